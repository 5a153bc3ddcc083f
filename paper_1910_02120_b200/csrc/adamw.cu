// One AdamW step over many tensors, states in 32 or in 8 bits (ist_adamw_step, see ist.h).
#include "../../include/ist.h"

#include <algorithm>
#include <cmath>
#include <mutex>
#include <type_traits>

#include "kernels.h"

using namespace ist;

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kChunk = 2048;                     // values that a block takes at a time
constexpr int kBlock = IST_ADAMW_BLOCK;          // values of an 8-bit state that share a base
constexpr int kNormBlocks = 1184;                // at most, per launch: each leaves one partial sum
constexpr int kSmallTable = 16, kTable = 400;    // tensors of a launch: the table is a kernel parameter (32,764 bytes at most)

struct Entry {
  float* p;
  const void* g;
  void* m;
  void* v;
  int16_t* mb;
  int16_t* vb;
  bf16* copy;
  int64_t n;
  float decay;
  uint32_t index;   // in the call; the top bit: all arrays are aligned for four values at a time
};
constexpr uint32_t kAligned = 0x80000000u;
constexpr uint32_t kInfinity = 0x7f800000u, kLargest = (kInfinity >> 20) - 1;

template <int CAP>
struct Table {
  int count;
  int per;                // blocks of kBlock values that a warp takes of a chunk (8-bit states)
  int chunk0[CAP + 1];    // first chunk of each tensor
  Entry e[CAP];
};

struct Args {
  float b1, c1, b2, c2, eps;             // c = 1 - b
  float lr, step_size, inv_root;         // lr, lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  double beta1, beta2;
  uint64_t step, seed;
  const int64_t* step_dev;
  const float* lr_dev;
  const double* partials;                // of the norm, or null
  int n_partials;
  double max_norm;
  float* norm_out;
};

constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;
__device__ __forceinline__ uint64_t mix64(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}
__device__ __forceinline__ uint64_t splitmix64(uint64_t seed, uint64_t i) { return mix64(seed + kGolden * i); }   // i-th output, from 1

__device__ __forceinline__ double power(double b, uint64_t t) {
  double r = 1.;
  for (; t; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}

// Sum over the block, the same in every thread; fixed order.
__device__ __forceinline__ double block_sum(double v, double* sh) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) s += sh[w];
  return s;
}

// What the whole step shares, worked out by every block.
struct Step {
  float lr, step_size, inv_root, clip;
  uint64_t key;
};
__device__ __forceinline__ Step begin_step(const Args& a) {
  __shared__ double sh[kWarps];
  Step s{a.lr, a.step_size, a.inv_root, 1.f, 0};
  uint64_t t = a.step;
  if (a.step_dev || a.lr_dev) {
    if (a.step_dev) t = (uint64_t)*a.step_dev;
    if (a.lr_dev) s.lr = *a.lr_dev;
    s.step_size = (float)((double)s.lr / (1. - power(a.beta1, t)));
    s.inv_root = (float)(1. / sqrt(1. - power(a.beta2, t)));
  }
  s.key = splitmix64(a.seed, t);
  if (a.partials) {
    double v = 0.;
    for (int i = threadIdx.x; i < a.n_partials; i += kThreads) v += a.partials[i];
    const double norm = sqrt(block_sum(v, sh));
    if (norm > a.max_norm) s.clip = (float)(a.max_norm / norm);
    if (a.norm_out && blockIdx.x == 0 && threadIdx.x == 0) *a.norm_out = (float)norm;
  }
  return s;
}

template <int CAP>
__device__ __forceinline__ int find_tensor(const Table<CAP>& t, int chunk) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.chunk0[mid] <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Four values from element i on; what lies at or behind n reads as zero and is not written.
template <typename T>
__device__ __forceinline__ void get4(const T* p, int64_t i, int64_t n, bool vec, float v[4]) {
  if (vec && i + 4 <= n) {
    load4(p + i, v);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = i + k < n ? to_float(p[i + k]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void put4(T* p, int64_t i, int64_t n, bool vec, const float v[4]) {
  if (vec && i + 4 <= n) {
    store4(p + i, v);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n) p[i + k] = from_float<T>(v[k]);
  }
}
__device__ __forceinline__ uint32_t get_codes(const uint8_t* p, int64_t i, int64_t n, bool vec) {
  if (vec && i + 4 <= n) return *reinterpret_cast<const uint32_t*>(p + i);
  uint32_t c = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (i + k < n) c |= (uint32_t)p[i + k] << (8 * k);
  return c;
}
__device__ __forceinline__ void put_codes(uint8_t* p, int64_t i, int64_t n, bool vec, uint32_t c) {
  if (vec && i + 4 <= n) {
    *reinterpret_cast<uint32_t*>(p + i) = c;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n) p[i + k] = (uint8_t)(c >> (8 * k));
  }
}

__device__ __forceinline__ void put8(float* p, int64_t i, int64_t n, bool vec, const float v[8]) {
  put4(p, i, n, vec, v);
  put4(p, i + 4, n, vec, v + 4);
}
__device__ __forceinline__ void put8(bf16* p, int64_t i, int64_t n, bool vec, const float v[8]) {
  if (vec && i + 8 <= n) {
    uint4 o;
    uint32_t* const w = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
      w[k] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p + i) = o;
  } else {
    put4(p, i, n, false, v);
    put4(p, i + 4, n, false, v + 4);
  }
}

// The moments' products and sums are rounded one by one, as elementary operations would be: 8-bit codes hang on their bits.
__device__ __forceinline__ void moments(const Args& a, float clip, float g, float* m, float* v) {
  g = __fmul_rn(g, clip);
  *m = __fadd_rn(__fmul_rn(a.b1, *m), __fmul_rn(a.c1, g));
  *v = __fadd_rn(__fmul_rn(a.b2, *v), __fmul_rn(__fmul_rn(a.c2, g), g));
}
// The root and the quotient by the hardware's approximations (2^-23 and 2^-22 of their values at most; the divisor is a normal
// number, eps at least): the change of a parameter is exact to a few units in its last place, and in the 8-bit step instructions
// are what the time goes to.
__device__ __forceinline__ float update(const Args& a, const Step& s, float decay, float p, float m, float v) {
  float root;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v));
  return fmaf(-s.step_size, __fdividef(m, fmaf(root, s.inv_root, a.eps)), fmaf(-s.lr * decay, p, p));
}

template <typename GT, int CAP>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Table<CAP> t, const Args a) {
  pdl_wait();
  pdl_trigger();
  const Step s = begin_step(a);
  for (int c = blockIdx.x; c < t.chunk0[t.count]; c += gridDim.x) {
    const int j = find_tensor(t, c);
    const Entry& e = t.e[j];
    const int64_t first = (int64_t)(c - t.chunk0[j]) * kChunk;
    const bool vec = e.index & kAligned;
    float* const em = (float*)e.m;
    float* const ev = (float*)e.v;
#pragma unroll
    for (int u = 0; u < kChunk / (4 * kThreads); ++u) {
      const int64_t i = first + (u * kThreads + threadIdx.x) * 4;
      if (i >= e.n) break;
      float p[4], g[4], m[4], v[4];
      get4(e.p, i, e.n, vec, p);
      get4((const GT*)e.g, i, e.n, vec, g);
      get4(em, i, e.n, vec, m);
      get4(ev, i, e.n, vec, v);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        moments(a, s.clip, g[k], &m[k], &v[k]);
        p[k] = update(a, s, e.decay, p[k], m[k], v[k]);
      }
      put4(e.p, i, e.n, vec, p);
      put4(em, i, e.n, vec, m);
      put4(ev, i, e.n, vec, v);
      if (e.copy) put4(e.copy, i, e.n, vec, p);
    }
  }
}

// Four codes of a block become values; see ist.h.  CHECKED: a base that no step makes reads as an infinity where it leaves
// fp32 (without it, as whatever number the sum's bits are).  The largest code is looked for in all four at once.
template <bool CHECKED>
__device__ __forceinline__ void decode_m4(uint32_t w, int base, float* m) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t c = (k == 3 ? w >> 4 : w << (20 - 8 * k)) & 0x07f00000u;
    uint32_t bits = CHECKED ? min((uint32_t)base + (c >> 20), kInfinity >> 20) << 20 : ((uint32_t)base << 20) + c;
    if (c == 0) bits = 0;
    m[k] = __uint_as_float(bits | ((w << (24 - 8 * k)) & 0x80000000u));
  }
  if (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (((w >> (8 * k)) & 127u) == 127u) m[k] = __uint_as_float(0x7fc00000u);
}
template <bool CHECKED>
__device__ __forceinline__ void decode_v4(uint32_t w, int base, float* v) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t c = (k == 3 ? w >> 4 : w << (20 - 8 * k)) & 0x0ff00000u;
    uint32_t bits = CHECKED ? min((uint32_t)base + (c >> 20), kInfinity >> 20) << 20 : ((uint32_t)base << 20) + c;
    if (c == 0) bits = 0;
    v[k] = __uint_as_float(bits);
  }
  if ((~w - 0x01010101u) & w & 0x80808080u)              // a byte of ~w is zero
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (((w >> (8 * k)) & 255u) == 255u) v[k] = __uint_as_float(kInfinity);
}
template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
  const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
  if (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
}
// Four bytes, one of each word's lowest.
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// A warp takes 128 values that share a base, four to a lane; a block takes a chunk, each of its warps t.per blocks of 128 in a
// row.  Where arrays are aligned, a lane's values come by asynchronous copies through shared memory, kStages - 1 blocks ahead (loads
// into registers cannot be waited for one after the other: 131 us for 20 M values with one block of loads ahead, TODO us
// this way).  Instructions, most of them integer ones, are what bounds the kernel then.  So blocks whose values are all finite
// and none near fp32's largest, which is to say all of a healthy run's, take a path without the cases of the others.
constexpr int kMostPer = 16, kStages = 4;

template <typename GT, int CAP>
__global__ void __launch_bounds__(kThreads) adamw8_kernel(const __grid_constant__ Table<CAP> t, const Args a) {
  pdl_wait();
  pdl_trigger();
  const Step s = begin_step(a);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kStage = kBlock * (4 + sizeof(GT) + 2);      // a block's p, g and codes
  extern __shared__ __align__(128) char rings[];
  char* const ring = rings + warp * (kStages * kStage);
  for (int c = blockIdx.x; c < t.chunk0[t.count]; c += gridDim.x) {
    const int j = find_tensor(t, c);
    const Entry& e = t.e[j];
    // from the warp's first value on
    const int64_t first = ((int64_t)(c - t.chunk0[j]) * kWarps + warp) * (t.per * kBlock), left = e.n - first;
    if (left <= 0) continue;
    float* const p = e.p + first;
    const GT* const g = (const GT*)e.g + first;
    uint8_t* const m = (uint8_t*)e.m + first;
    uint8_t* const v = (uint8_t*)e.v + first;
    bf16* const copy = e.copy ? e.copy + first : nullptr;
    int16_t* const mb = e.mb + first / kBlock;
    int16_t* const vb = e.vb + first / kBlock;
    const float decay = e.decay;
    // word w of the noise belongs to values 2 w and 2 w + 1
    const uint64_t noise = splitmix64(s.key, (e.index & ~kAligned) + 1ull) + kGolden * (uint64_t)(first / 2 + lane * 2 + 1);
    auto work = [&](auto fast, int u, float (&pf)[4], const float (&gf)[4], uint32_t mc, uint32_t vc, int mbase, int vbase) {
      float mf[4], vf[4];
      decode_m4<false>(mc, mbase, mf);
      decode_v4<false>(vc, vbase, vf);
      uint32_t mbits[4], vbits[4], mmax = 0, vmax = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        moments(a, s.clip, gf[k], &mf[k], &vf[k]);
        pf[k] = update(a, s, decay, pf[k], mf[k], vf[k]);
        mbits[k] = __float_as_uint(mf[k]) & 0x7fffffffu;
        vbits[k] = __float_as_uint(vf[k]);                       // of a number: the sign is zero
        mmax = max(mmax, mbits[k]);
        vmax = max(vmax, vbits[k]);
      }
      mmax = __reduce_max_sync(0xffffffffu, mmax);
      vmax = __reduce_max_sync(0xffffffffu, vmax);
      const bool special = max(mmax, vmax) >= kLargest << 20;
      if (special) {
        mmax = vmax = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          vbits[k] &= 0x7fffffffu;
          if (mbits[k] < kInfinity) mmax = max(mmax, mbits[k]);
          if (vbits[k] < kInfinity) vmax = max(vmax, vbits[k]);
        }
        mmax = __reduce_max_sync(0xffffffffu, mmax);
        vmax = __reduce_max_sync(0xffffffffu, vmax);
      }
      // the block's largest value, rounded up, gets the largest code but one
      const int nmb = max((int)(mmax >> 20) + 1 - 126, 0), nvb = max((int)(vmax >> 20) + 1 - 254, 0);
      const uint32_t mlow = 8u - ((uint32_t)nmb << 20), vlow = 8u - ((uint32_t)nvb << 20);
      uint32_t cm[4], cv[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint64_t w = mix64(noise + kGolden * (uint64_t)(u * (kBlock / 2) + k / 2));
        const uint32_t r = k & 1 ? (uint32_t)(w >> 32) : (uint32_t)w;
        const uint32_t mr = r << 4 & 0xffff0u, vr = r >> 12 & 0xffff0u;
        if (!special) {
          cm[k] = (uint32_t)max((int)(mbits[k] + mr + mlow), 0) >> 20;
          cv[k] = (uint32_t)max((int)(vbits[k] + vr + vlow), 0) >> 20;
        } else {
          cm[k] = mbits[k] >= kInfinity ? 127u : (uint32_t)max((int)min((mbits[k] + mr + 8u) >> 20, kLargest) - nmb, 0);
          cv[k] = vbits[k] >= kInfinity ? 255u : (uint32_t)max((int)min((vbits[k] + vr + 8u) >> 20, kLargest) - nvb, 0);
        }
        cv[k] = max(cv[k], min(vbits[k], 1u));                   // a divisor does not vanish
        if (cm[k]) cm[k] |= (__float_as_uint(mf[k]) >> 24) & 128u;
      }
      const uint32_t mw = pack4(cm[0], cm[1], cm[2], cm[3]), vw = pack4(cv[0], cv[1], cv[2], cv[3]);
      const int i = u * kBlock + lane * 4;
      if (fast) {
        store4(p + i, pf);
        if (copy) store4(copy + i, pf);
        *reinterpret_cast<uint32_t*>(m + i) = mw;
        *reinterpret_cast<uint32_t*>(v + i) = vw;
      } else {
        const bool vec = e.index & kAligned;
        put4(p, i, left, vec, pf);
        if (copy) put4(copy, i, left, vec, pf);
        put_codes(m, i, left, vec, mw);
        put_codes(v, i, left, vec, vw);
      }
      if (lane == 0) {
        mb[u] = (int16_t)nmb;
        vb[u] = (int16_t)nvb;
      }
    };
    const int blocks = (int)min((int64_t)t.per, ceil_div(left, kBlock));
    const int whole = e.index & kAligned ? (int)min((int64_t)t.per, left / kBlock) : 0;
    auto fetch = [&](int u) {
      if (u < whole) {
        char* const to = ring + (u % kStages) * kStage;
        const int i = u * kBlock + lane * 4;
        copy_async<16>(to + lane * 16, p + i);
        copy_async<4 * sizeof(GT)>(to + kBlock * 4 + lane * (4 * sizeof(GT)), g + i);
        copy_async<4>(to + kBlock * (4 + sizeof(GT)) + lane * 4, m + i);
        copy_async<4>(to + kBlock * (5 + sizeof(GT)) + lane * 4, v + i);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int u = 0; u < kStages - 1; ++u) fetch(u);
    // lane u has the first moment's base of block u, lane 16 + u the second's
    const int base = (lane & 15) < blocks ? (lane < 16 ? mb : vb)[lane & 15] : 0;
#pragma unroll 1
    for (int u = 0; u < whole; ++u) {
      fetch(u + kStages - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      const char* const from = ring + (u % kStages) * kStage;
      float pf[4], gf[4];
      load4(reinterpret_cast<const float*>(from) + lane * 4, pf);
      load4(reinterpret_cast<const GT*>(from + kBlock * 4) + lane * 4, gf);
      const uint32_t mc = reinterpret_cast<const uint32_t*>(from + kBlock * (4 + sizeof(GT)))[lane];
      const uint32_t vc = reinterpret_cast<const uint32_t*>(from + kBlock * (5 + sizeof(GT)))[lane];
      work(std::true_type(), u, pf, gf, mc, vc, __shfl_sync(0xffffffffu, base, u), __shfl_sync(0xffffffffu, base, 16 + u));
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll 1
    for (int u = whole; u < blocks; ++u) {
      const bool vec = e.index & kAligned;
      const int i = u * kBlock + lane * 4;
      float pf[4], gf[4];
      get4(p, i, left, vec, pf);
      get4(g, i, left, vec, gf);
      work(std::false_type(), u, pf, gf, get_codes(m, i, left, vec), get_codes(v, i, left, vec), __shfl_sync(0xffffffffu, base, u),
           __shfl_sync(0xffffffffu, base, 16 + u));
    }
  }
}

// Sum of squares of all gradients, a partial sum per block.  Eight squares at a time are added in fp32 and
// those sums in fp64; where fp32 overflows or comes near its smallest numbers the eight are taken in fp64.
template <typename GT, int CAP>
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const __grid_constant__ Table<CAP> t, int chunk, double* partials) {
  __shared__ double sh[kWarps];
  pdl_wait();
  pdl_trigger();
  double sum = 0.;
  constexpr int U = kChunk / (4 * kThreads);
  for (int c = blockIdx.x; c < t.chunk0[t.count]; c += gridDim.x) {
    const int j = find_tensor(t, c);
    const Entry& e = t.e[j];
    const bool vec = ((uintptr_t)e.g & (4 * sizeof(GT) - 1)) == 0;
#pragma unroll 1
    for (int at = 0; at < chunk; at += kChunk) {
      const int64_t first = (int64_t)(c - t.chunk0[j]) * chunk + at + threadIdx.x * 4, past = min(e.n, (int64_t)(c - t.chunk0[j] + 1) * chunk);
      float g[U][4];
#pragma unroll
      for (int u = 0; u < U; ++u) get4((const GT*)e.g, first + u * kThreads * 4, past, vec, g[u]);
      float q = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < 4; ++k) q = fmaf(g[u][k], g[u][k], q);
      if (q > 1e-30f && q < 1e37f)
        sum += q;
      else
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int k = 0; k < 4; ++k) sum += (double)g[u][k] * g[u][k];
    }
  }
  sum = block_sum(sum, sh);
  if (threadIdx.x == 0) partials[blockIdx.x] = sum;
}

// Eight values to a thread where a state's arrays allow it.
template <typename OT>
__global__ void __launch_bounds__(kThreads) state_values_kernel(const uint8_t* m, const int16_t* mb, const uint8_t* v,
                                                               const int16_t* vb, int64_t n, bool vec, OT* m_out, OT* v_out) {
  pdl_wait();
  pdl_trigger();
  const int64_t step = (int64_t)gridDim.x * kThreads * 8;
  for (int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 8; i < n; i += step) {
    uint32_t mc[2], vc[2];
    int mbase = 0, vbase = 0;
    if (m_out) {
      mbase = mb[i / kBlock];
#pragma unroll
      for (int h = 0; h < 2; ++h) mc[h] = get_codes(m, i + 4 * h, n, vec);
    }
    if (v_out) {
      vbase = vb[i / kBlock];
#pragma unroll
      for (int h = 0; h < 2; ++h) vc[h] = get_codes(v, i + 4 * h, n, vec);
    }
    float x[8];
    if (m_out) {
#pragma unroll
      for (int h = 0; h < 2; ++h) decode_m4<true>(mc[h], mbase, x + 4 * h);
      put8(m_out, i, n, vec, x);
    }
    if (v_out) {
#pragma unroll
      for (int h = 0; h < 2; ++h) decode_v4<true>(vc[h], vbase, x + 4 * h);
      put8(v_out, i, n, vec, x);
    }
  }
}

bool aligned(const void* p, int64_t bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// The next tensors of the call that fit a table, from `*at` on; empty ones and those without a gradient are passed over.
template <int CAP>
void fill(const ist_adamw_tensor* list, int64_t count, const ist_adamw_args& a, int64_t* at, Table<CAP>* t) {
  const int chunk = a.state_bits == 8 ? t->per * (kBlock * kWarps) : kChunk;
  const int64_t gs = a.grad_type == IST_T_BF16 ? 2 : 4, ss = a.state_bits == 8 ? 1 : 4;
  int64_t chunks = 0;
  t->count = 0;
  for (; *at < count && t->count < CAP; ++*at) {
    const ist_adamw_tensor& x = list[*at];
    if (x.n == 0 || !x.grad) continue;
    const int64_t more = ceil_div(x.n, chunk);
    if (chunks + more > (int64_t)1 << 30) break;     // at most 2^40 values in all: one tensor always fits
    Entry& e = t->e[t->count];
    e = Entry{x.param, x.grad, x.exp_avg, x.exp_avg_sq, x.exp_avg_base, x.exp_avg_sq_base, (bf16*)x.param_bf16, x.n,
              (float)x.weight_decay, (uint32_t)*at};
    if (aligned(x.param, 16) && aligned(x.grad, 4 * gs) && aligned(x.exp_avg, 4 * ss) && aligned(x.exp_avg_sq, 4 * ss) &&
        aligned(x.param_bf16, 8))
      e.index |= kAligned;
    t->chunk0[t->count++] = (int)chunks;
    chunks += more;
  }
  t->chunk0[t->count] = (int)chunks;
}

template <typename GT, int CAP>
cudaError_t launch8(const Table<CAP>& t, const Args& args, cudaStream_t stream) {
  constexpr int smem = kWarps * kStages * kBlock * (4 + sizeof(GT) + 2);
  static std::once_flag once;
  static cudaError_t ready = cudaSuccess;
  static int resident = 1;
  std::call_once(once, [] {
    ready = cudaFuncSetAttribute(adamw8_kernel<GT, CAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (ready == cudaSuccess) ready = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, adamw8_kernel<GT, CAP>, kThreads, smem);
    resident = std::max(resident, 1) * sm_count();
  });
  if (ready != cudaSuccess) return ready;
  return launch_pdl(adamw8_kernel<GT, CAP>, dim3((unsigned)std::min(t.chunk0[t.count], resident)), dim3(kThreads), smem, stream, t, args);
}

template <int CAP>
cudaError_t step_launches(const ist_adamw_tensor* list, int64_t count, int64_t values, const ist_adamw_args& a, Args args, double* partials,
                          cudaStream_t stream) {
  Table<CAP> t;
  t.count = t.chunk0[0] = 0;
  // chunks of eight blocks for each that the GPU holds, if there are so many values; a power of two
  t.per = 1;
  while (t.per < kMostPer && values > (int64_t)t.per * (kBlock * kWarps) * sm_count() * 8 * 4) t.per *= 2;
  cudaError_t e = cudaSuccess;
  const bool bf16_grad = a.grad_type == IST_T_BF16;
  auto blocks = [&](int per_sm) { return dim3((unsigned)std::min<int64_t>(t.chunk0[t.count], (int64_t)sm_count() * per_sm)); };
  bool ready = false;                     // the table holds the call's only part
  if (partials) {
    int64_t at = 0;
    while (at < count && e == cudaSuccess) {
      fill(list, count, a, &at, &t);
      ready = args.n_partials == 0 && at == count;
      if (t.count == 0) continue;
      const dim3 grid((unsigned)std::min<int64_t>(t.chunk0[t.count], kNormBlocks));
      double* const out = partials + args.n_partials;
      e = bf16_grad ? launch_pdl(grad_norm_kernel<bf16, CAP>, grid, dim3(kThreads), 0, stream, t, a.state_bits == 8 ? t.per * (kBlock * kWarps) : kChunk, out)
                    : launch_pdl(grad_norm_kernel<float, CAP>, grid, dim3(kThreads), 0, stream, t, a.state_bits == 8 ? t.per * (kBlock * kWarps) : kChunk, out);
      args.n_partials += (int)grid.x;
    }
    args.partials = partials;
  }
  int64_t at = 0;
  while (e == cudaSuccess && (ready || at < count)) {
    if (!ready) fill(list, count, a, &at, &t);
    if (t.count) {
      if (a.state_bits == 32)
        e = bf16_grad ? launch_pdl(adamw_kernel<bf16, CAP>, blocks(8), dim3(kThreads), 0, stream, t, args)
                      : launch_pdl(adamw_kernel<float, CAP>, blocks(8), dim3(kThreads), 0, stream, t, args);
      else
        e = bf16_grad ? launch8<bf16>(t, args, stream) : launch8<float>(t, args, stream);
      args.norm_out = nullptr;            // the first launch has written it
    }
    if (ready) break;
  }
  return e;
}

const char* bad_args(const ist_adamw_args& a) {
  if (a.state_bits != 32 && a.state_bits != 8) return "state_bits is 32 or 8";
  if (a.grad_type != IST_T_F32 && a.grad_type != IST_T_BF16) return "element types are IST_T_F32 and IST_T_BF16";
  if (!(a.beta1 >= 0. && a.beta1 < 1. && a.beta2 >= 0. && a.beta2 < 1.)) return "betas must be in [0, 1)";
  if (!((float)a.eps >= 1.17549435e-38f && std::isfinite((float)a.eps))) return "eps must be a positive normal number in fp32";
  if (!(a.max_norm >= 0.)) return "max_norm must be >= 0";
  if (!a.lr_dev && !std::isfinite((float)a.lr)) return "lr must be finite";
  if (!a.step_dev && a.step < 1) return "step must be >= 1";
  if (!aligned(a.step_dev, 8) || !aligned(a.lr_dev, 4) || !aligned(a.norm_out_dev, 4))
    return "step_dev, lr_dev and norm_out_dev must be aligned to their elements";
  return nullptr;
}
const char* bad_tensor(const ist_adamw_tensor& x, const ist_adamw_args& a) {
  if (x.n < 0 || x.n > (int64_t)1 << 40) return "n must be in 0..2^40";
  if (!std::isfinite((float)x.weight_decay)) return "weight_decay must be finite";
  if (x.n == 0 || !x.grad) return nullptr;
  if (!x.param || !x.exp_avg || !x.exp_avg_sq) return "null parameter or state";
  if (a.state_bits == 8 && (!x.exp_avg_base || !x.exp_avg_sq_base)) return "null base of an 8-bit state";
  const int64_t gs = a.grad_type == IST_T_BF16 ? 2 : 4, ss = a.state_bits == 8 ? 1 : 4;
  if (!aligned(x.param, 4) || !aligned(x.grad, gs) || !aligned(x.exp_avg, ss) || !aligned(x.exp_avg_sq, ss) ||
      !aligned(x.param_bf16, 2) || (a.state_bits == 8 && (!aligned(x.exp_avg_base, 2) || !aligned(x.exp_avg_sq_base, 2))))
    return "an array is not aligned to its elements";
  return nullptr;
}

}  // namespace

extern "C" size_t ist_adamw_workspace_bytes(int64_t count) {
  if (count < 0 || count > (int64_t)1 << 24) return 0;
  // one partial sum per block of the norm's launches: kTable tensors and 2^30 chunks at most each
  return (size_t)((ceil_div(count, kTable) + 1) * kNormBlocks * sizeof(double));
}

extern "C" ist_status ist_adamw_step(const ist_adamw_tensor* tensors_host, int64_t count, const ist_adamw_args* args,
                                     void* workspace_dev, size_t workspace_bytes, void* cuda_stream) {
  if (!args || (count > 0 && !tensors_host)) return fail_call(IST_ERR_ARG, "ist_adamw_step: null arguments");
  if (count < 0 || count > (int64_t)1 << 24) return fail_call(IST_ERR_ARG, "ist_adamw_step: count must be in 0..2^24");
  if (const char* why = bad_args(*args)) return fail_call(IST_ERR_ARG, "ist_adamw_step: %s", why);
  int64_t values = 0, live = 0;
  for (int64_t j = 0; j < count; ++j) {
    if (const char* why = bad_tensor(tensors_host[j], *args))
      return fail_call(IST_ERR_ARG, "ist_adamw_step: tensor %lld: %s", (long long)j, why);
    if (tensors_host[j].grad && tensors_host[j].n) {
      values += tensors_host[j].n;
      ++live;
    }
    if (values > (int64_t)1 << 40) return fail_call(IST_ERR_ARG, "ist_adamw_step: more than 2^40 values");
  }
  const bool clip = args->max_norm > 0.;
  if (clip && (!workspace_dev || workspace_bytes < ist_adamw_workspace_bytes(count) || !aligned(workspace_dev, 16)))
    return fail_call(IST_ERR_WORKSPACE, "ist_adamw_step: workspace too small or not aligned to 16 bytes (%lld bytes needed)",
                     (long long)ist_adamw_workspace_bytes(count));
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  cudaError_t e = cudaSuccess;
  if (live == 0) {
    if (clip && args->norm_out_dev) e = cudaMemsetAsync(args->norm_out_dev, 0, sizeof(float), stream);
  } else {
    Args k{};
    k.b1 = (float)args->beta1;
    k.c1 = (float)(1. - args->beta1);
    k.b2 = (float)args->beta2;
    k.c2 = (float)(1. - args->beta2);
    k.eps = (float)args->eps;
    k.lr = (float)args->lr;
    k.beta1 = args->beta1;
    k.beta2 = args->beta2;
    k.step = (uint64_t)args->step;
    k.seed = args->seed;
    k.step_dev = args->step_dev;
    k.lr_dev = args->lr_dev;
    k.step_size = (float)(args->lr / (1. - std::pow(args->beta1, (double)args->step)));
    k.inv_root = (float)(1. / std::sqrt(1. - std::pow(args->beta2, (double)args->step)));
    k.max_norm = args->max_norm;
    k.norm_out = args->norm_out_dev;
    double* const partials = clip ? (double*)workspace_dev : nullptr;
    e = live <= kSmallTable ? step_launches<kSmallTable>(tensors_host, count, values, *args, k, partials, stream)
                            : step_launches<kTable>(tensors_host, count, values, *args, k, partials, stream);
  }
  if (e != cudaSuccess) return fail_call(IST_ERR_CUDA, "ist_adamw_step: %s", cudaGetErrorString(e));
  return IST_OK;
}

extern "C" ist_status ist_adamw_state_values(const uint8_t* exp_avg, const int16_t* exp_avg_base, const uint8_t* exp_avg_sq,
                                             const int16_t* exp_avg_sq_base, int64_t n, int out_type, void* exp_avg_out_dev,
                                             void* exp_avg_sq_out_dev, void* cuda_stream) {
  const char* why = nullptr;
  const int64_t os = out_type == IST_T_BF16 ? 2 : 4;
  if (n < 0 || n > (int64_t)1 << 40) why = "n must be in 0..2^40";
  else if (out_type != IST_T_F32 && out_type != IST_T_BF16) why = "element types are IST_T_F32 and IST_T_BF16";
  else if (n && exp_avg_out_dev && (!exp_avg || !exp_avg_base)) why = "null codes or bases";
  else if (n && exp_avg_sq_out_dev && (!exp_avg_sq || !exp_avg_sq_base)) why = "null codes or bases";
  else if (!aligned(exp_avg_out_dev, os) || !aligned(exp_avg_sq_out_dev, os) || !aligned(exp_avg_base, 2) || !aligned(exp_avg_sq_base, 2))
    why = "an array is not aligned to its elements";
  if (why) return fail_call(IST_ERR_ARG, "ist_adamw_state_values: %s", why);
  if (n == 0 || (!exp_avg_out_dev && !exp_avg_sq_out_dev)) return IST_OK;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  const bool vec = (!exp_avg_out_dev || (aligned(exp_avg, 4) && aligned(exp_avg_out_dev, 16))) &&
                   (!exp_avg_sq_out_dev || (aligned(exp_avg_sq, 4) && aligned(exp_avg_sq_out_dev, 16)));
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(n, 8 * kThreads), (int64_t)sm_count() * 8));
  const cudaError_t e =
      out_type == IST_T_BF16
          ? launch_pdl(state_values_kernel<bf16>, grid, dim3(kThreads), 0, stream, exp_avg, exp_avg_base, exp_avg_sq,
                       exp_avg_sq_base, n, vec, (bf16*)exp_avg_out_dev, (bf16*)exp_avg_sq_out_dev)
          : launch_pdl(state_values_kernel<float>, grid, dim3(kThreads), 0, stream, exp_avg, exp_avg_base, exp_avg_sq,
                       exp_avg_sq_base, n, vec, (float*)exp_avg_out_dev, (float*)exp_avg_sq_out_dev);
  if (e != cudaSuccess) return fail_call(IST_ERR_CUDA, "ist_adamw_state_values: %s", cudaGetErrorString(e));
  return IST_OK;
}
