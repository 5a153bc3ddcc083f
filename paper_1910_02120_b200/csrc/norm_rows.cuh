// What layer norm's two passes share: rows on their way through shared memory, sums over the threads of a row.
//
// TPR threads (8 ... 1024) take a row, each NV pieces of V adjacent elements, piece i of thread t being the row's piece
// t + i TPR.  Rows come in by asynchronous 16- or 8-byte copies, stages ahead of their use.  Where rows are aligned to
// pieces (V > 1) a thread copies exactly what it reads itself, so no barrier stands between the two.  Rows that start anywhere
// (V = 1) are copied in 16-byte pieces too, to the same offset from a 16-byte boundary as in memory, and their ends in
// single elements; then a barrier of the row's threads, and each reads elements TPR apart.
#pragma once

#include "kernels.h"

namespace ist {

constexpr int kNormThreads = 256;      // of a block, at least

struct NormForward {
  const void* x;
  void* y;
  int64_t x_ld, y_ld;
  int64_t site_rows;
  int sites, cols;
  const float* weight;
  const float* bias;
  float* mean;
  float* rstd;
  float eps;
};
struct NormBackward {
  const void* dy;
  const void* x;
  void* dx;
  int64_t dy_ld, x_ld, dx_ld;
  int64_t site_rows;
  int sites, cols;
  const float* weight;
  const float* mean;
  const float* rstd;
  // the sums over part p's rows of site s: [cols] at wsum and bsum + (p * sites + s) * sum_ld, either may be null
  float* wsum;
  float* bsum;
  int64_t sum_ld;
  int parts;
};

// norm_forward.cu, norm_backward.cu: false if no kernel takes rows of this width (nothing is launched).
bool norm_forward_rows(const NormForward& a, bool x_bf16, bool y_bf16, cudaStream_t stream, cudaError_t* e);
bool norm_backward_rows(const NormBackward& a, bool x_bf16, bool dy_bf16, cudaStream_t stream, cudaError_t* e);
constexpr int kNormWidest = 16384;     // wider rows have kernels of their own

namespace {

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
  if (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int BYTES> struct Raw;
template <> struct Raw<2> { typedef uint16_t type; };
template <> struct Raw<4> { typedef uint32_t type; };
template <> struct Raw<8> { typedef uint2 type; };
template <> struct Raw<16> { typedef uint4 type; };

// V adjacent elements as fp32.
template <typename T, int V>
__device__ __forceinline__ void unpack(const void* p, float* v) {
  typedef typename Raw<V * sizeof(T)>::type R;
  const R r = *reinterpret_cast<const R*>(p);
  if (sizeof(T) == 4) {
    const float* f = reinterpret_cast<const float*>(&r);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = f[k];
  } else if (V == 1) {
    v[0] = __uint_as_float((uint32_t) * reinterpret_cast<const uint16_t*>(&r) << 16);
  } else {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
    for (int k = 0; k < V / 2; ++k) {
      v[2 * k] = __uint_as_float(w[k] << 16);
      v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
  }
}
template <typename T, int V>
__device__ __forceinline__ void pack(T* p, const float* v) {
  typedef typename Raw<V * sizeof(T)>::type R;
  R r;
  if (sizeof(T) == 4) {
    float* f = reinterpret_cast<float*>(&r);
#pragma unroll
    for (int k = 0; k < V; ++k) f[k] = v[k];
  } else if (V == 1) {
    *reinterpret_cast<bf16*>(&r) = __float2bfloat16_rn(v[0]);
  } else {
    uint32_t* w = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
    for (int k = 0; k < V / 2; ++k) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
      w[k] = *reinterpret_cast<const uint32_t*>(&b);
    }
  }
  *reinterpret_cast<R*>(p) = r;
}
// V adjacent fp32 values of a weight, its own alignment aside.
template <int V>
__device__ __forceinline__ void load_vector(const float* p, bool wide, float* v) {
  if (V % 4 == 0 && wide) {
#pragma unroll
    for (int k = 0; k < V; k += 4) load4(p + k, v + k);
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = p[k];
  }
}

// A row's bytes in shared memory: room for its 16-byte pieces, whatever its offset from a boundary.
__host__ __device__ __forceinline__ constexpr int row_room(int cols, int size, bool anywhere) {
  return (cols * size + 15) / 16 * 16 + (anywhere ? 16 : 0);
}

// Starts the copies of a row.  Returns the offset of its first element in `buf`.
template <typename T, int V, int TPR>
__device__ __forceinline__ void fetch_row(const T* row, int cols, char* buf, int t) {
  if (V > 1) {
    for (int u = t * V; u < cols; u += TPR * V) copy_async<V * sizeof(T)>(shared_address(buf + u * sizeof(T)), row + u);
  } else {
    const uintptr_t first = (uintptr_t)row, last = first + (uintptr_t)cols * sizeof(T);
    const uintptr_t base = first & ~(uintptr_t)15, whole = (first + 15) & ~(uintptr_t)15, end = last & ~(uintptr_t)15;
    for (uintptr_t p = whole + 16 * t; p + 16 <= end; p += 16 * TPR)
      copy_async<16>(shared_address(buf + (p - base)), reinterpret_cast<const void*>(p));
    // the ends, in fp32 words; single bf16 elements among them are left to fetch_odd
    const uintptr_t head = whole < last ? whole : last;          // a short row may lie between two boundaries
    const uintptr_t word = (first + 3) & ~(uintptr_t)3;
    for (uintptr_t p = word + 4 * t; p + 4 <= head; p += 4 * TPR)
      copy_async<4>(shared_address(buf + (p - base)), reinterpret_cast<const void*>(p));
    if (end >= whole)
      for (uintptr_t p = end + 4 * t; p + 4 <= last; p += 4 * TPR)
        copy_async<4>(shared_address(buf + (p - base)), reinterpret_cast<const void*>(p));
  }
}
// bf16 rows that start or end in the middle of a 4-byte word: thread 0 and thread 1 of the row carry those elements.
template <typename T>
__device__ __forceinline__ uint16_t load_odd(const T* row, int cols, int t) {
  if (sizeof(T) == 4) return 0;
  const uintptr_t first = (uintptr_t)row, last = first + (uintptr_t)cols * sizeof(T);
  if (t == 0 && (first & 3)) return *reinterpret_cast<const uint16_t*>(row);
  if (t == 1 && (last & 3)) return *reinterpret_cast<const uint16_t*>(row + cols - 1);
  return 0;
}
template <typename T>
__device__ __forceinline__ void store_odd(const T* row, int cols, char* buf, int t, uint16_t v) {
  if (sizeof(T) == 4) return;
  const uintptr_t first = (uintptr_t)row, last = first + (uintptr_t)cols * sizeof(T), base = first & ~(uintptr_t)15;
  if (t == 0 && (first & 3)) *reinterpret_cast<uint16_t*>(buf + (first - base)) = v;
  if (t == 1 && (last & 3)) *reinterpret_cast<uint16_t*>(buf + (last - 2 - base)) = v;
}

// Sums of N values over the TPR threads of a row, left in all of them; the order is the same on every call.  sh: 2 buffers,
// used in turn, of [rows of the block][N][warps of a row].
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float* v, float* sh, int* turn) {
#pragma unroll
  for (int o = (TPR < 32 ? TPR : 32) / 2; o; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if (TPR > 32) {
    constexpr int W = TPR / 32;
    const int row = threadIdx.x / TPR, warp = threadIdx.x % TPR / 32, lane = threadIdx.x & 31;
    float* const b = sh + *turn * (blockDim.x / 32 * N) + row * N * W;
    *turn ^= 1;
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) b[i * W + warp] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (W <= 8) {
        float s = b[i * W];
#pragma unroll
        for (int w = 1; w < W; ++w) s += b[i * W + w];
        v[i] = s;
      } else {
        float s = lane < W ? b[i * W + lane] : 0.f;
#pragma unroll
        for (int o = W / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        v[i] = __shfl_sync(0xffffffffu, s, 0);
      }
    }
  }
}

template <int TPR>
__device__ __forceinline__ void row_barrier() {
  if (TPR <= 32) __syncwarp(); else __syncthreads();
}

// 1 / sqrt(a), the hardware's estimate improved by one Newton step.
__device__ __forceinline__ float inverse_root(float a) {
  const float r = rsqrtf(a);
  const float n = fmaf(r * 0.5f, fmaf(-a * r, r, 1.f), r);
  return isfinite(n) ? n : r;          // a infinite: 0, not 0 times infinity
}

}  // namespace
}  // namespace ist
