// One AdamW step over many tensors, states in 32 or in 8 bits (ist_adamw_step, see ist.h).
#include "../../include/ist.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.h"
#include "pairs.cuh"

namespace ist {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kChunk = 2048;                     // values that a block takes at a time
constexpr int kBlock = IST_ADAMW_BLOCK;          // values of an 8-bit state that share a base
constexpr int kNormBlocks = 1184;                // at most, per launch: each leaves one partial sum
// Tensors of a launch.  The table is a kernel parameter, which may be 32,764 bytes; launches of up to 4 KB cost the host least.
constexpr int kSmallTable = 16, kMiddleTable = 50, kTable = 400;

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

// The moments' products and sums are rounded one by one, as elementary operations would be: 8-bit codes hang on their bits.
__device__ __forceinline__ void moments(const Args& a, float clip, float g, float* m, float* v) {
  g = __fmul_rn(g, clip);
  *m = __fadd_rn(__fmul_rn(a.b1, *m), __fmul_rn(a.c1, g));
  *v = __fadd_rn(__fmul_rn(a.b2, *v), __fmul_rn(__fmul_rn(a.c2, g), g));
}
// The root and the reciprocal by the hardware's approximations (2^-23 of their values each; the divisor is a normal number, eps
// at least, and so is its reciprocal): the change of a parameter is exact to a few units in its last place, and in the
// 8-bit step instructions are what the time goes to.  TINY: eps is so small that roots of denormal numbers weigh beside it.
template <bool TINY>
__device__ __forceinline__ float root_of(float v) {
  float r;
  if (TINY)
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
  else
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float inverse(float a) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(a));
  return r;
}
__device__ __forceinline__ float update(const Args& a, const Step& s, float decay, float p, float m, float v) {
  return fmaf(-s.step_size, m * inverse(fmaf(root_of<true>(v), s.inv_root, a.eps)), fmaf(-s.lr * decay, p, p));
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
    if (vec) {
#pragma unroll
      for (int u = 0; u < kChunk / (4 * kThreads); ++u) {
        const int64_t i = first + (u * kThreads + threadIdx.x) * 4;
        if (i >= e.n) break;
        float p[4], g[4], m[4], v[4];
        get4(e.p, i, e.n, true, p);
        get4((const GT*)e.g, i, e.n, true, g);
        get4(em, i, e.n, true, m);
        get4(ev, i, e.n, true, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          moments(a, s.clip, g[k], &m[k], &v[k]);
          p[k] = update(a, s, e.decay, p[k], m[k], v[k]);
        }
        put4(e.p, i, e.n, true, p);
        put4(em, i, e.n, true, m);
        put4(ev, i, e.n, true, v);
        if (e.copy) put4(e.copy, i, e.n, true, p);
      }
    } else {
      // arrays that start anywhere: adjacent threads take adjacent values
#pragma unroll
      for (int u = 0; u < kChunk / (4 * kThreads); ++u) {
        const int64_t i = first + u * (4 * kThreads) + threadIdx.x;
        float p[4], g[4], m[4], v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int64_t at = i + k * kThreads;
          if (at < e.n) {
            p[k] = e.p[at];
            g[k] = to_float(((const GT*)e.g)[at]);
            m[k] = em[at];
            v[k] = ev[at];
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int64_t at = i + k * kThreads;
          if (at < e.n) {
            moments(a, s.clip, g[k], &m[k], &v[k]);
            p[k] = update(a, s, e.decay, p[k], m[k], v[k]);
            e.p[at] = p[k];
            em[at] = m[k];
            ev[at] = v[k];
            if (e.copy) e.copy[at] = from_float<bf16>(p[k]);
          }
        }
      }
    }
  }
}

// Four codes of a block become values; see ist.h.  Bases that no step makes read as infinities where they leave fp32.  TOP: the
// largest code, 127 or 255.  Not inlined: what seldom runs would otherwise be issued, predicated off, with what always does.
template <uint32_t TOP>
__device__ __noinline__ float4 decode_any4(uint32_t w, int base) {
  float x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t one = w >> (8 * k) & 255u, c = one & TOP;
    uint32_t bits = c == TOP ? (TOP == 127u ? 0x7fc00000u : kInfinity) : min((uint32_t)base + c, kInfinity >> 20) << 20;
    if (c == 0) bits = 0;
    x[k] = __uint_as_float(bits | (one & ~TOP) << 24);
  }
  return make_float4(x[0], x[1], x[2], x[3]);
}
// The same for bases that steps make: a code is multiplied into its place and the base is added, unless one of the four is zero or
// the largest.
__device__ __forceinline__ void decode_m4(uint32_t w, int base, float* m) {
  const uint32_t c = w & 0x7f7f7f7fu, sign = w & 0x80808080u, b = (uint32_t)base << 20;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    m[k] = __uint_as_float((__byte_perm(c, 0, 0x4440 + k) * (1u << 20) + b) | __byte_perm(sign, 0, 0x0444 + (k << 12)));
  if (((c + 0x01010101u) | ~(c + 0x7f7f7f7fu)) & 0x80808080u) {
    const float4 f = decode_any4<127>(w, base);
    m[0] = f.x; m[1] = f.y; m[2] = f.z; m[3] = f.w;
  }
}
__device__ __forceinline__ void decode_v4(uint32_t w, int base, float* v) {
  const uint32_t b = (uint32_t)base << 20;
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(__byte_perm(w, 0, 0x4440 + k) * (1u << 20) + b);
  if ((((w - 0x01010101u) & ~w) | ((~w - 0x01010101u) & w)) & 0x80808080u) {
    const float4 f = decode_any4<255>(w, base);
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
  }
}
// The top bytes of four words.
__device__ __forceinline__ uint32_t top4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

// Codes of four values, bits of their magnitudes and their noise given, where one of the block's is not finite or near fp32's largest.
__device__ __noinline__ uint32_t encode_special4(uint4 bits, uint4 noise, int base, uint32_t top) {
  const uint32_t b[4] = {bits.x, bits.y, bits.z, bits.w}, r[4] = {noise.x, noise.y, noise.z, noise.w};
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    w |= (b[k] >= kInfinity ? top : (uint32_t)max((int)min((b[k] + r[k] * 16u + 8u) >> 20, kLargest) - base, 0)) << (8 * k);
  return w;
}
// Zero codes of values that are not zero become the smallest code.
__device__ __noinline__ uint32_t lift_zeros4(uint32_t codes, uint4 bits) {
  const uint32_t b[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (b[k] && !(codes >> (8 * k) & 255u)) codes |= 1u << (8 * k);
  return codes;
}
// Largest of the bits that belong to numbers.
__device__ __noinline__ uint32_t largest_number(uint4 bits) {
  const uint32_t b[4] = {bits.x, bits.y, bits.z, bits.w};
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (b[k] < kInfinity) m = max(m, b[k]);
  return m;
}

// A warp takes 128 values that share a base, four to a lane; a block takes a chunk, each of its warps t.per blocks of 128 in a
// row.  Where arrays are aligned, a lane's values come by asynchronous copies through shared memory, kStages - 1 blocks ahead (loads
// into registers cannot be waited for one after the other: 118 us for 20 M values with one block of loads ahead, 84 us
// this way).  Instructions, most of them integer ones, are what bounds the kernel then.  So blocks whose values are all finite
// and none near fp32's largest, which is to say all of a healthy run's, take a path without the cases of the others.
constexpr int kMostPer = 16, kStages = 3;

template <bool TINY, typename GT, int CAP>
__device__ __forceinline__ void adamw8_chunks(const Table<CAP>& t, const Args& a, const Step& s, char* ring) {
  constexpr int kStage = kBlock * (4 + sizeof(GT) + 2);      // a block's p, g and codes
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const pair b1 = both(a.b1), c1 = both(a.c1), b2 = both(a.b2), c2 = both(a.c2), clip = both(s.clip);
  const pair inv_root = both(s.inv_root), eps = both(a.eps), step = both(-s.step_size);
  for (int c = blockIdx.x; c < t.chunk0[t.count]; c += gridDim.x) {
    const int j = find_tensor(t, c);
    const Entry& e = t.e[j];
    // the chunk's first value (the same for all threads), and where in the chunk this lane's first one is
    const int64_t first = (int64_t)(c - t.chunk0[j]) * (kWarps * t.per * kBlock);
    const uint32_t mine = warp * (t.per * kBlock) + lane * 4;
    const int64_t left = e.n - first - warp * (t.per * kBlock);
    if (left <= 0) continue;
    float* const p = e.p + first;
    const GT* const g = (const GT*)e.g + first;
    uint8_t* const m = (uint8_t*)e.m + first;
    uint8_t* const v = (uint8_t*)e.v + first;
    bf16* const copy = e.copy ? e.copy + first : nullptr;
    const pair decay = both(-s.lr * e.decay);
    const int blocks = (int)min((int64_t)t.per, ceil_div(left, kBlock));
    const int whole = e.index & kAligned ? (int)min((int64_t)t.per, left / kBlock) : 0;
    // word w of the noise belongs to values 2 w and 2 w + 1
    uint64_t noise = splitmix64(s.key, (e.index & ~kAligned) + 1ull) + kGolden * (uint64_t)((first + mine) / 2 + 1);
    // lane u has the first moment's base of block u, lane 16 + u the second's
    int16_t* const my_base = (lane < 16 ? e.mb : e.vb) + first / kBlock + warp * t.per + (lane & 15);
    const int base = (lane & 15) < blocks ? *my_base : 0;
    int new_base = 0;

    auto work = [&](int u, float (&pf)[4], const float (&gf)[4], uint32_t mc, uint32_t vc, uint32_t* mw, uint32_t* vw) {
      float mf[4], vf[4];
      decode_m4(mc, __shfl_sync(0xffffffffu, base, u), mf);
      decode_v4(vc, __shfl_sync(0xffffffffu, base, 16 + u), vf);
      uint32_t mbits[4], vbits[4], mmax = 0, vmax = 0;
      // the moments: the same operations, one rounding each, as in moments()
#pragma unroll
      for (int k = 0; k < 4; k += 2) {
        const pair gc = mul(make_pair2(gf[k], gf[k + 1]), clip);
        const pair mn = add_rounded(mul(b1, make_pair2(mf[k], mf[k + 1])), mul(c1, gc));
        const pair vn = add_rounded(mul(b2, make_pair2(vf[k], vf[k + 1])), mul(mul(c2, gc), gc));
        const pair d = fma(make_pair2(root_of<TINY>(first_of(vn)), root_of<TINY>(second_of(vn))), inv_root, eps);
        const pair q = mul(mn, make_pair2(inverse(first_of(d)), inverse(second_of(d))));
        const pair po = make_pair2(pf[k], pf[k + 1]), pn = fma(step, q, fma(decay, po, po));
        pf[k] = first_of(pn);
        pf[k + 1] = second_of(pn);
        mf[k] = first_of(mn);
        mf[k + 1] = second_of(mn);
        vbits[k] = __float_as_uint(first_of(vn));                  // of a number: the sign is zero
        vbits[k + 1] = __float_as_uint(second_of(vn));
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        mbits[k] = __float_as_uint(mf[k]) & 0x7fffffffu;
        mmax = max(mmax, mbits[k]);
        vmax = max(vmax, vbits[k]);
      }
      mmax = __reduce_max_sync(0xffffffffu, mmax);
      vmax = __reduce_max_sync(0xffffffffu, vmax);
      const bool special = max(mmax, vmax) >= kLargest << 20;
      if (special) {
#pragma unroll
        for (int k = 0; k < 4; ++k) vbits[k] &= 0x7fffffffu;
        mmax = __reduce_max_sync(0xffffffffu, largest_number(make_uint4(mbits[0], mbits[1], mbits[2], mbits[3])));
        vmax = __reduce_max_sync(0xffffffffu, largest_number(make_uint4(vbits[0], vbits[1], vbits[2], vbits[3])));
      }
      // the block's largest value, rounded up, gets the largest code but one
      const int nmb = max((int)(mmax >> 20) + 1 - 126, 0), nvb = max((int)(vmax >> 20) + 1 - 254, 0);
      if ((lane & 15) == u) new_base = lane < 16 ? nmb : nvb;
      const int mlow = 8 - (nmb << 20), vlow = 8 - (nvb << 20);
      uint32_t mr[4], vr[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint64_t w = mix64(noise + kGolden * (uint64_t)(k / 2));
        const uint32_t r = k & 1 ? (uint32_t)(w >> 32) : (uint32_t)w;
        mr[k] = r & 0xffffu;
        vr[k] = r >> 16;
      }
      noise += kGolden * (uint64_t)(kBlock / 2);
      uint32_t codes, out;
      if (!special) {
        uint32_t cm[4], cv[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {                                     // the code is the top byte
          cm[k] = (uint32_t)__viaddmax_s32((int)(mr[k] * 16u + mbits[k]), mlow, 0) * 16u;
          cv[k] = (uint32_t)__viaddmax_s32((int)(vr[k] * 16u + vbits[k]), vlow, 0) * 16u;
        }
        codes = top4(cm[0], cm[1], cm[2], cm[3]);
        out = top4(cv[0], cv[1], cv[2], cv[3]);
      } else {
        codes = encode_special4(make_uint4(mbits[0], mbits[1], mbits[2], mbits[3]), make_uint4(mr[0], mr[1], mr[2], mr[3]), nmb, 127u);
        out = encode_special4(make_uint4(vbits[0], vbits[1], vbits[2], vbits[3]), make_uint4(vr[0], vr[1], vr[2], vr[3]), nvb, 255u);
      }
      const uint32_t signs = top4(__float_as_uint(mf[0]), __float_as_uint(mf[1]), __float_as_uint(mf[2]), __float_as_uint(mf[3]));
      *mw = codes | (signs & (codes + 0x7f7f7f7fu) & 0x80808080u);      // a zero has no sign
      if ((out - 0x01010101u) & ~out & 0x80808080u)                     // a divisor does not vanish
        out = lift_zeros4(out, make_uint4(vbits[0], vbits[1], vbits[2], vbits[3]));
      *vw = out;
    };
    uint32_t in = 0, out = 0;                              // places in the ring of the next block to arrive and to be worked on
    auto fetch = [&](int u) {
      if (u < whole) {
        char* const to = ring + in;
        const uint32_t i = mine + u * kBlock;
        copy_async<16>(shared_address(to + lane * 16), p + i);
        copy_async<4 * sizeof(GT)>(shared_address(to + kBlock * 4 + lane * (4 * sizeof(GT))), g + i);
        copy_async<4>(shared_address(to + kBlock * (4 + sizeof(GT)) + lane * 4), m + i);
        copy_async<4>(shared_address(to + kBlock * (5 + sizeof(GT)) + lane * 4), v + i);
      }
      in = in == (kStages - 1) * kStage ? 0 : in + kStage;
      copy_commit();
    };
#pragma unroll
    for (int u = 0; u < kStages - 1; ++u) fetch(u);
#pragma unroll 1
    for (int u = 0; u < whole; ++u) {
      fetch(u + kStages - 1);
      copy_wait<kStages - 1>();
      const char* const from = ring + out;
      out = out == (kStages - 1) * kStage ? 0 : out + kStage;
      float pf[4], gf[4];
      load4(reinterpret_cast<const float*>(from) + lane * 4, pf);
      load4(reinterpret_cast<const GT*>(from + kBlock * 4) + lane * 4, gf);
      uint32_t mw = reinterpret_cast<const uint32_t*>(from + kBlock * (4 + sizeof(GT)))[lane];
      uint32_t vw = reinterpret_cast<const uint32_t*>(from + kBlock * (5 + sizeof(GT)))[lane];
      work(u, pf, gf, mw, vw, &mw, &vw);
      const uint32_t i = mine + u * kBlock;
      store4(p + i, pf);
      if (copy) store4(copy + i, pf);
      *reinterpret_cast<uint32_t*>(m + i) = mw;
      *reinterpret_cast<uint32_t*>(v + i) = vw;
    }
    copy_wait<0>();
#pragma unroll 1
    for (int u = whole; u < blocks; ++u) {
      const bool vec = e.index & kAligned;
      const int64_t i = mine + u * kBlock, n = e.n - first;
      float pf[4], gf[4];
      get4(p, i, n, vec, pf);
      get4(g, i, n, vec, gf);
      uint32_t mw, vw;
      work(u, pf, gf, get_codes(m, i, n, vec), get_codes(v, i, n, vec), &mw, &vw);
      put4(p, i, n, vec, pf);
      if (copy) put4(copy, i, n, vec, pf);
      put_codes(m, i, n, vec, mw);
      put_codes(v, i, n, vec, vw);
    }
    if ((lane & 15) < blocks) *my_base = (int16_t)new_base;
  }
}

template <typename GT, int CAP>
__global__ void __launch_bounds__(kThreads, 4) adamw8_kernel(const __grid_constant__ Table<CAP> t, const Args a) {
  extern __shared__ __align__(128) char rings[];
  char* const ring = rings + (threadIdx.x >> 5) * (kStages * kBlock * (4 + sizeof(GT) + 2));
  pdl_wait();
  pdl_trigger();
  const Step s = begin_step(a);
  // roots of denormal numbers are below 2^-63: beside a divisor of 2^-36 and more they do not show
  if (a.eps >= 0x1p-36f && s.inv_root <= 0x1p3f) adamw8_chunks<false, GT>(t, a, s, ring);
  else adamw8_chunks<true, GT>(t, a, s, ring);
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
      const int64_t first = (int64_t)(c - t.chunk0[j]) * chunk + at, past = min(e.n, (int64_t)(c - t.chunk0[j] + 1) * chunk);
      float g[U][4];
      if (vec) {
#pragma unroll
        for (int u = 0; u < U; ++u) get4((const GT*)e.g, first + (u * kThreads + threadIdx.x) * 4, past, true, g[u]);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int64_t i = first + (u * 4 + k) * kThreads + threadIdx.x;
            g[u][k] = i < past ? to_float(((const GT*)e.g)[i]) : 0.f;
          }
      }
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

template <typename OT>
__device__ __forceinline__ void write8(OT* out, const float* x) {
  if constexpr (sizeof(OT) == 2) {
    uint4 o;
    uint32_t* const w = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
      w[k] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(out) = o;
  } else {
    store4(out, x);
    store4(out + 4, x + 4);
  }
}
template <bool SIGNED>
__device__ __forceinline__ void decode4(uint32_t w, int base, float* x) {
  constexpr uint32_t kTop = SIGNED ? 127u : 255u;
  if ((uint32_t)base > kLargest - kTop) {
    const float4 f = decode_any4<kTop>(w, base);
    x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
  } else if (SIGNED) {
    decode_m4(w, base, x);
  } else {
    decode_v4(w, base, x);
  }
}
// The values of one state.  Where its arrays allow it, eight to a thread; four loads and the bases of a thread's runs are on
// their way together.
template <bool SIGNED, typename OT>
__device__ __forceinline__ void state_values(const uint8_t* codes, const int16_t* bases, int64_t n, bool vec, OT* out) {
  constexpr int U = 4;
  const int64_t step = (int64_t)gridDim.x * kThreads * 8;
  int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 8;
  for (; vec && i + (U - 1) * step + 8 <= n; i += U * step) {
    uint2 c[U];
    int base[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      c[u] = *reinterpret_cast<const uint2*>(codes + i + u * step);
      base[u] = bases[(uint64_t)(i + u * step) / kBlock];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[8];
      decode4<SIGNED>(c[u].x, base[u], x);
      decode4<SIGNED>(c[u].y, base[u], x + 4);
      write8(out + i + u * step, x);
    }
  }
  for (; vec && i + 8 <= n; i += step) {
    const uint2 c = *reinterpret_cast<const uint2*>(codes + i);
    const int base = bases[(uint64_t)i / kBlock];
    float x[8];
    decode4<SIGNED>(c.x, base, x);
    decode4<SIGNED>(c.y, base, x + 4);
    write8(out + i, x);
  }
  for (; i < n; i += step)
#pragma unroll 1
    for (int h = 0; h < 8 && i + h < n; h += 4) {
      float x[4];
      decode4<SIGNED>(get_codes(codes, i + h, n, false), bases[(uint64_t)i / kBlock], x);
      put4(out, i + h, n, false, x);
    }
}
template <typename OT>
__global__ void __launch_bounds__(kThreads) state_values_kernel(const uint8_t* m, const int16_t* mb, const uint8_t* v,
                                                               const int16_t* vb, int64_t n, bool vec, OT* m_out, OT* v_out) {
  pdl_wait();
  pdl_trigger();
  if (m_out) state_values<true>(m, mb, n, vec, m_out);
  if (v_out) state_values<false>(v, vb, n, vec, v_out);
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
  static OncePerDevice<KernelReady> once;
  const KernelReady ready = ready_here(once, [] {
    int per_sm = 1;
    cudaError_t e = cudaFuncSetAttribute(adamw8_kernel<GT, CAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, adamw8_kernel<GT, CAP>, kThreads, smem);
    return KernelReady{e, std::max(per_sm, 1) * sm_count()};
  });
  if (ready.error != cudaSuccess) return ready.error;
  return launch_pdl(adamw8_kernel<GT, CAP>, dim3((unsigned)std::min(t.chunk0[t.count], ready.resident)), dim3(kThreads), smem, stream, t, args);
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
  // the divisor, eps and a root of 2^91 at most, has a reciprocal that is a normal number too (see inverse)
  if (!((float)a.eps >= 0x1p-126f && (float)a.eps <= 0x1p125f)) return "eps must be in 2^-126..2^125";
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
}  // namespace ist

using namespace ist;

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
    e = live <= kSmallTable    ? step_launches<kSmallTable>(tensors_host, count, values, *args, k, partials, stream)
        : live <= kMiddleTable ? step_launches<kMiddleTable>(tensors_host, count, values, *args, k, partials, stream)
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
  const bool vec = (!exp_avg_out_dev || (aligned(exp_avg, 8) && aligned(exp_avg_out_dev, 16))) &&
                   (!exp_avg_sq_out_dev || (aligned(exp_avg_sq, 8) && aligned(exp_avg_sq_out_dev, 16)));
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
