// One AdamW step over many tensors, states in 32 or in 8 bits (ist_adamw_step, see ist.h).
#include "../../include/ist.h"

#include <algorithm>
#include <cmath>

#include "kernels.h"

using namespace ist;

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kChunk = 2048;                     // values that a block takes at a time
constexpr int kBlock = IST_ADAMW_BLOCK;          // values of an 8-bit state that share a base
constexpr int kNormBlocks = 592;                 // at most, per launch: each leaves one partial sum
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

__device__ __forceinline__ uint64_t splitmix64(uint64_t seed, uint64_t i) {   // the i-th output, from 1
  uint64_t z = seed + 0x9E3779B97F4A7C15ull * i;
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

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
__device__ __forceinline__ float update(const Args& a, const Step& s, float decay, float p, float m, float v) {
  const float root = fmaf(sqrtf(v), s.inv_root, a.eps);
  return fmaf(-s.step_size, m / root, fmaf(-s.lr * decay, p, p));
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

// A value of a block with this base; see ist.h.  A base that no step makes reads as an infinity where it leaves fp32.
__device__ __forceinline__ float decode_m(uint32_t c, uint32_t base) {
  const uint32_t k = c & 127u;
  uint32_t bits = k == 127u ? 0x7fc00000u : min(base + k, kInfinity >> 20) << 20;
  if (k == 0) bits = 0;
  return __uint_as_float(bits | (c & 128u) << 24);
}
__device__ __forceinline__ float decode_v(uint32_t c, uint32_t base) {
  uint32_t bits = c == 255u ? kInfinity : min(base + c, kInfinity >> 20) << 20;
  if (c == 0) bits = 0;
  return __uint_as_float(bits);
}
// bits: of the magnitude; r: 16 random bits.
__device__ __forceinline__ uint32_t encode(uint32_t bits, uint32_t r, int base, int top) {
  const int k = (int)min((bits + r * 16u + 8u) >> 20, kLargest) - base;
  return bits >= kInfinity ? (uint32_t)top : (uint32_t)max(k, 0);
}
__device__ __forceinline__ uint32_t warp_max(uint32_t v) {
  return __reduce_max_sync(0xffffffffu, v);
}

// A warp takes 128 values that share a base, four to a lane.
template <typename GT, int CAP>
__global__ void __launch_bounds__(kThreads) adamw8_kernel(const __grid_constant__ Table<CAP> t, const Args a) {
  pdl_wait();
  pdl_trigger();
  const Step s = begin_step(a);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int c = blockIdx.x; c < t.chunk0[t.count]; c += gridDim.x) {
    const int j = find_tensor(t, c);
    const Entry& e = t.e[j];
    const int64_t first = (int64_t)(c - t.chunk0[j]) * kChunk;
    const bool vec = e.index & kAligned;
    const uint64_t key = splitmix64(s.key, (e.index & ~kAligned) + 1ull);
    uint8_t* const em = (uint8_t*)e.m;
    uint8_t* const ev = (uint8_t*)e.v;
#pragma unroll
    for (int u = 0; u < kChunk / (kBlock * kWarps); ++u) {
      const int64_t start = first + (u * kWarps + warp) * kBlock, i = start + lane * 4;
      if (start >= e.n) break;
      const int64_t block = start / kBlock;
      float p[4], g[4], m[4], v[4];
      get4(e.p, i, e.n, vec, p);
      get4((const GT*)e.g, i, e.n, vec, g);
      const uint32_t mc = get_codes(em, i, e.n, vec), vc = get_codes(ev, i, e.n, vec);
      const uint32_t mb = (uint32_t)e.mb[block], vb = (uint32_t)e.vb[block];
      uint32_t mmax = 0, vmax = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        m[k] = decode_m((mc >> (8 * k)) & 255u, mb);
        v[k] = decode_v((vc >> (8 * k)) & 255u, vb);
        moments(a, s.clip, g[k], &m[k], &v[k]);
        p[k] = update(a, s, e.decay, p[k], m[k], v[k]);
        const uint32_t ma = __float_as_uint(m[k]) & 0x7fffffffu, va = __float_as_uint(v[k]) & 0x7fffffffu;
        if (ma < kInfinity) mmax = max(mmax, ma);
        if (va < kInfinity) vmax = max(vmax, va);
      }
      put4(e.p, i, e.n, vec, p);
      if (e.copy) put4(e.copy, i, e.n, vec, p);
      // the block's largest value, rounded up, gets the largest code but one
      const int nmb = max((int)(warp_max(mmax) >> 20) + 1 - 126, 0), nvb = max((int)(warp_max(vmax) >> 20) + 1 - 254, 0);
      uint32_t nmc = 0, nvc = 0;
#pragma unroll
      for (int k = 0; k < 4; k += 2) {
        const uint64_t w = splitmix64(key, (uint64_t)(i + k) / 2 + 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t r = (uint32_t)(w >> (32 * h));
          const uint32_t mbits = __float_as_uint(m[k + h]), vbits = __float_as_uint(v[k + h]) & 0x7fffffffu;
          uint32_t cm = encode(mbits & 0x7fffffffu, r & 0xffffu, nmb, 127);
          uint32_t cv = encode(vbits, r >> 16, nvb, 255);
          if (cm) cm |= (mbits >> 24) & 128u;
          if (vbits && !cv) cv = 1;
          nmc |= cm << (8 * (k + h));
          nvc |= cv << (8 * (k + h));
        }
      }
      put_codes(em, i, e.n, vec, nmc);
      put_codes(ev, i, e.n, vec, nvc);
      if (lane == 0) {
        e.mb[block] = (int16_t)nmb;
        e.vb[block] = (int16_t)nvb;
      }
    }
  }
}

// Sum of squares of all gradients, a partial sum per block.  Four squares at a time are added in fp32 and
// those sums in fp64; where fp32 overflows or comes near its smallest numbers the four are taken in fp64.
template <typename GT, int CAP>
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const __grid_constant__ Table<CAP> t, double* partials) {
  __shared__ double sh[kWarps];
  pdl_wait();
  pdl_trigger();
  double sum = 0.;
  for (int c = blockIdx.x; c < t.chunk0[t.count]; c += gridDim.x) {
    const int j = find_tensor(t, c);
    const Entry& e = t.e[j];
    const int64_t first = (int64_t)(c - t.chunk0[j]) * kChunk;
    const bool vec = ((uintptr_t)e.g & (4 * sizeof(GT) - 1)) == 0;
#pragma unroll
    for (int u = 0; u < kChunk / (4 * kThreads); ++u) {
      const int64_t i = first + (u * kThreads + threadIdx.x) * 4;
      if (i >= e.n) break;
      float g[4];
      get4((const GT*)e.g, i, e.n, vec, g);
      const float q = fmaf(g[0], g[0], fmaf(g[1], g[1], fmaf(g[2], g[2], g[3] * g[3])));
      if (q > 1e-30f && q < 1e37f)
        sum += q;
      else
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += (double)g[k] * g[k];
    }
  }
  sum = block_sum(sum, sh);
  if (threadIdx.x == 0) partials[blockIdx.x] = sum;
}

template <typename OT>
__global__ void __launch_bounds__(kThreads) state_values_kernel(const uint8_t* m, const int16_t* mb, const uint8_t* v,
                                                               const int16_t* vb, int64_t n, bool vec, OT* m_out, OT* v_out) {
  pdl_wait();
  pdl_trigger();
  for (int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * kThreads * 4) {
    float x[4];
    if (m_out) {
      const uint32_t c = get_codes(m, i, n, vec), base = (uint32_t)mb[i / kBlock];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = decode_m((c >> (8 * k)) & 255u, base);
      put4(m_out, i, n, vec, x);
    }
    if (v_out) {
      const uint32_t c = get_codes(v, i, n, vec), base = (uint32_t)vb[i / kBlock];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = decode_v((c >> (8 * k)) & 255u, base);
      put4(v_out, i, n, vec, x);
    }
  }
}

bool aligned(const void* p, int64_t bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// The next tensors of the call that fit a table, from `*at` on; empty ones and those without a gradient are passed over.
template <int CAP>
void fill(const ist_adamw_tensor* list, int64_t count, const ist_adamw_args& a, int64_t* at, Table<CAP>* t) {
  const int64_t gs = a.grad_type == IST_T_BF16 ? 2 : 4, ss = a.state_bits == 8 ? 1 : 4;
  int64_t chunks = 0;
  t->count = 0;
  for (; *at < count && t->count < CAP; ++*at) {
    const ist_adamw_tensor& x = list[*at];
    if (x.n == 0 || !x.grad) continue;
    const int64_t more = ceil_div(x.n, kChunk);
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

template <int CAP>
cudaError_t step_launches(const ist_adamw_tensor* list, int64_t count, const ist_adamw_args& a, Args args, double* partials,
                          cudaStream_t stream) {
  Table<CAP> t;
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
      e = bf16_grad ? launch_pdl(grad_norm_kernel<bf16, CAP>, grid, dim3(kThreads), 0, stream, t, out)
                    : launch_pdl(grad_norm_kernel<float, CAP>, grid, dim3(kThreads), 0, stream, t, out);
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
        e = bf16_grad ? launch_pdl(adamw8_kernel<bf16, CAP>, blocks(8), dim3(kThreads), 0, stream, t, args)
                      : launch_pdl(adamw8_kernel<float, CAP>, blocks(8), dim3(kThreads), 0, stream, t, args);
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
  if (!((float)a.eps > 0.f && std::isfinite((float)a.eps))) return "eps must be positive and finite in fp32";
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
    e = live <= kSmallTable ? step_launches<kSmallTable>(tensors_host, count, *args, k, partials, stream)
                            : step_launches<kTable>(tensors_host, count, *args, k, partials, stream);
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
  const bool vec = (!exp_avg_out_dev || (aligned(exp_avg, 4) && aligned(exp_avg_out_dev, 4 * os))) &&
                   (!exp_avg_sq_out_dev || (aligned(exp_avg_sq, 4) && aligned(exp_avg_sq_out_dev, 4 * os)));
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(n, 4 * kThreads), (int64_t)sm_count() * 8));
  const cudaError_t e =
      out_type == IST_T_BF16
          ? launch_pdl(state_values_kernel<bf16>, grid, dim3(kThreads), 0, stream, exp_avg, exp_avg_base, exp_avg_sq,
                       exp_avg_sq_base, n, vec, (bf16*)exp_avg_out_dev, (bf16*)exp_avg_sq_out_dev)
          : launch_pdl(state_values_kernel<float>, grid, dim3(kThreads), 0, stream, exp_avg, exp_avg_base, exp_avg_sq,
                       exp_avg_sq_base, n, vec, (float*)exp_avg_out_dev, (float*)exp_avg_sq_out_dev);
  if (e != cudaSuccess) return fail_call(IST_ERR_CUDA, "ist_adamw_state_values: %s", cudaGetErrorString(e));
  return IST_OK;
}
