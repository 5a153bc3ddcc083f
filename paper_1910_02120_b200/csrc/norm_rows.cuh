// What layer norm's two passes share: rows on their way through shared memory, sums over the threads of a row.
//
// TPR threads (4 ... 512) of a block take a row, or its part where a cluster of blocks takes it, each NV pieces of V adjacent
// elements, piece i of thread t being piece t + i TPR.  Rows come in by asynchronous 16- or 8-byte copies, stages ahead of
// their use.  Where rows are aligned to pieces (V > 1) a thread copies exactly what it reads itself, so no barrier stands
// between the two.  Rows that start anywhere (V = 1) are copied in 16-byte pieces too, to the same offset from a 16-byte
// boundary as in memory, and their ends in single elements; then a barrier of the row's threads, and each reads elements TPR
// apart.  A thread takes RB rows at a time, whose sums go through the shuffles together.
//
// The arithmetic is on pairs of fp32 values (one instruction for two): one by one, issuing instructions took longer than the
// memory (bf16 rows of 2048, forward: 24 instructions an element, 35 us for 134 MB).
#pragma once

#include "kernels.h"
#include "pairs.cuh"
#include "tc_ptx.cuh"

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
  long long wait_limit;      // see Turn
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
  long long wait_limit;
};

// norm_forward.cu, norm_backward.cu: rows of up to kNormWidest elements.
cudaError_t norm_forward_rows(const NormForward& a, bool x_bf16, bool y_bf16, cudaStream_t stream);
cudaError_t norm_backward_rows(const NormBackward& a, bool x_bf16, bool dy_bf16, cudaStream_t stream);
// Whether a wait of theirs on the current device gave up since the last call; waits for the stream.
cudaError_t norm_forward_gave_up(cudaStream_t stream, bool* gave_up);
cudaError_t norm_backward_gave_up(cudaStream_t stream, bool* gave_up);
// norm_narrow.cu: rows of up to kNormNarrow elements.
cudaError_t norm_forward_narrow(const NormForward& a, bool x_bf16, bool y_bf16, cudaStream_t stream);
cudaError_t norm_backward_narrow(const NormBackward& a, bool x_bf16, bool dy_bf16, cudaStream_t stream);
constexpr int kNormNarrow = 16, kNormWidest = 65536;
// Blocks of a cluster that share a row of the second one.
inline int norm_cluster(int64_t cols) { return cols <= 8192 ? 1 : cols <= 16384 ? 2 : cols <= 32768 ? 4 : 8; }

namespace {

// Writes to the place in block `rank` of the cluster that corresponds to `at` in this one; the write itself tells that block's
// barrier, so no fence stands behind it (a cluster barrier would wait for all of the threads' stores to global memory too: 4096
// bf16 rows of 16384 shared by four blocks, backward, 189 us that way and 161 us this way).
__device__ __forceinline__ void send_cluster(float* at, uint64_t* bar, uint32_t rank, float v) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.f32 [%0], %1, [%2];"
               ::"r"(map_to_cta(at, rank)), "f"(v), "r"(map_to_cta(bar, rank)) : "memory");
}

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

// Columns of a block when a row is shared by a cluster of `cl`.
__host__ __device__ __forceinline__ constexpr int part_width(int cols, int cl) {
  return cl == 1 ? cols : ((cols + cl - 1) / cl + 7) / 8 * 8;
}
// A row's bytes in shared memory: room for its 16-byte pieces, whatever its offset from a boundary.  Rows that are copied in wide
// pieces by a warp or more take whole lines of 128 bytes (a warp's access that starts inside a line takes one turn more:
// fp32 rows of 1024, forward, 33 us and 39 us).
__host__ __device__ __forceinline__ constexpr int row_room(int cols, int size, bool anywhere) {
  const int bytes = cols * size, unit = bytes < 512 ? 16 : 128;
  return (bytes + (anywhere ? 15 : 0) + unit - 1) / unit * unit;
}

// Starts the copies of a row into `buf`.  LEAST: columns that it has at least.
template <typename T, int V, int NV, int TPR, int LEAST>
__device__ __forceinline__ void fetch_row(const T* row, int cols, char* buf, int t) {
  if (V > 1) {
    const T* const from = row + t * V;
    const uint32_t to = shared_address(buf) + t * (V * sizeof(T));
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if ((i + 1) * TPR * V <= LEAST || (t + i * TPR) * V < cols) copy_async<V * sizeof(T)>(to + i * (TPR * V * sizeof(T)), from + i * (TPR * V));
  } else {
    // from the 16-byte boundary at or before the row: whole 16-byte pieces, then up to three fp32 words at either end; single
    // bf16 elements outside these are left to load_odd
    constexpr int kPieces = (TPR * NV * (int)sizeof(T) / 16 + TPR) / TPR;
    const int off = (int)((uintptr_t)row & 15), end = off + cols * (int)sizeof(T);
    const char* const base = reinterpret_cast<const char*>(row) - off;
    const uint32_t to = shared_address(buf);
    const int head = (off + 15) >> 4, tail = end >> 4;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int p = head + t + i * TPR;
      if (p < tail) copy_async<16>(to + p * 16, base + p * 16);
    }
    if (t < 8) {
      const int p = t < 4 ? ((off + 3) >> 2) + t : tail * 4 + t - 4, past = t < 4 ? min(head * 4, end >> 2) : tail < head ? 0 : end >> 2;
      if (p < past) copy_async<4>(to + p * 4, base + p * 4);
    }
  }
}
// bf16 rows that start or end in the middle of a 4-byte word: thread 0 and thread 1 of the row carry those elements.
template <typename T>
__device__ __forceinline__ uint16_t load_odd(const T* row, int cols, int t) {
  if (sizeof(T) == 4) return 0;
  const int off = (int)((uintptr_t)row & 3) >> 1;
  const int at = t == 0 ? 0 : cols - 1;
  const bool mine = t == 0 ? off : t == 1 && ((off + cols) & 1);
  return mine ? *reinterpret_cast<const uint16_t*>(row + at) : (uint16_t)0;
}
template <typename T>
__device__ __forceinline__ void store_odd(const T* row, int cols, char* buf, int t, uint16_t v) {
  if (sizeof(T) == 4) return;
  const int off = (int)((uintptr_t)row & 15) >> 1;
  const int at = t == 0 ? 0 : cols - 1;
  const bool mine = t == 0 ? off & 1 : t == 1 && ((off + cols) & 1);
  if (mine) reinterpret_cast<uint16_t*>(buf)[off + at] = v;
}

constexpr int log2_of(int n) { return n <= 1 ? 0 : 1 + log2_of(n / 2); }

// Sums of N values (a power of two) over the TPR threads of a row and the CL blocks of a cluster, left in all of them; the
// order is the same on every call.  At each of the first steps a lane keeps half of the values and gives the other half
// to its partner, so that N values take N - 1 shuffles and one more for each step left, not one per value and step.
// RowSums: 2 buffers, used in turn, of [rows of the block][N][warps of a row in the cluster], N up to MOST.  A thread that
// writes a buffer again has read the sums of the use in between, to which every thread of the row contributed after reading
// this one, so one barrier per use is enough.
//
// A wait for other blocks' sums that does not end within wait_limit cycles makes them NaN and sets g_gave_up.  The block then
// neither announces nor sends sums any more (a barrier whose phase has not ended takes no second arrival, and counts only so many
// bytes), so the cluster's other threads give up in their turn; each waits out the limit once.  A negative limit is the self-test's:
// all blocks are silent from the start.
template <int THREADS, int CL, int MOST>
struct RowSums {
  float part[2 * (THREADS / 32) * CL * MOST];
  uint64_t bar[CL > 1 ? 2 : 1];
  volatile int silent;       // read ahead of the shuffles it is free; in a register it cost up to 13 % (1000 fp32 rows of 65536)
};
struct Turn {
  int buffer, parity;
  bool gave_up;
};
__device__ int g_gave_up;    // of this file's kernels
template <int CL, typename S>
__device__ __forceinline__ Turn begin_sums(S& sh, long long wait_limit) {
  if (CL > 1) {
    if (threadIdx.x == 0) {
      mbar_init(&sh.bar[0], 1);
      mbar_init(&sh.bar[CL > 1 ? 1 : 0], 1);
      sh.silent = wait_limit < 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    cluster_sync_all();
  }
  return Turn{0, 0, false};
}
// No block ends while another may write to its sums.  Where all waits ended, all sums that were sent have arrived; after one that
// gave up, others' may still be on their way when the last of the cluster gets here, and are given time.
template <int CL>
__device__ __forceinline__ void finish_sums(const Turn& turn) {
  if (CL == 1) return;
  cluster_sync_all();
  if (turn.gave_up) {
    const long long begin = clock64();
    while (clock64() - begin < 200000) {}
  }
}
// The sums' first half: everything up to where other warps' values are needed.
template <int TPR, int CL, int N, typename S>
__device__ __forceinline__ void begin_row_sums(float* v, S& sh, const Turn& turn) {
  constexpr int L = TPR < 32 ? TPR : 32;                   // lanes of a row within a warp
  const int lane = threadIdx.x & 31;
  const int silent = CL > 1 ? sh.silent : 0;
  int n = N, o = L / 2, mine = 0;                          // mine: the value this lane ends with
#pragma unroll
  for (int s = 0; s < log2_of(N < L ? N : L); ++s, o /= 2) {
    n /= 2;
    const bool up = lane & o;
    mine = mine * 2 + up;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float keep = up ? v[i + n] : v[i], give = up ? v[i] : v[i + n];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
  constexpr int kLeft = N < L ? 1 : N / L;                 // values that a lane has at the end
#pragma unroll
  for (; o; o /= 2)
#pragma unroll
    for (int i = 0; i < kLeft; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  constexpr int kSteps = log2_of(N < L ? N : L), kShare = L >> kSteps;     // lanes that hold the same values
  if (TPR <= 32) {
    if (N > 1) {
      float r[N];
#pragma unroll
      for (int i = 0; i < N; ++i) r[i] = __shfl_sync(0xffffffffu, v[i % kLeft], i / kLeft * kShare, L);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = r[i];
    }
    return;
  }
  constexpr int W = TPR / 32 * CL;
  const int row = threadIdx.x / TPR, warp = threadIdx.x % TPR / 32;
  float* const b = sh.part + turn.buffer * (sizeof(sh.part) / 8) + row * N * W;
  if (CL == 1) {
    if (lane % kShare == 0) b[mine * W + warp] = v[0];
  } else {
    uint64_t* const bar = &sh.bar[turn.buffer];
    if (threadIdx.x == 0 && !silent) mbar_expect_tx(bar, W * N * sizeof(float));
    if (lane % kShare == 0 && !silent)
#pragma unroll
      for (int q = 0; q < CL; ++q) send_cluster(b + mine * W + cluster_ctarank() * (TPR / 32) + warp, bar, q, v[0]);
  }
}
// Their second half: waits for the other warps and adds.
template <int TPR, int CL, int N, typename S>
__device__ __forceinline__ void end_row_sums(float* v, S& sh, Turn* turn, long long wait_limit) {
  if (TPR <= 32) return;
  constexpr int W = TPR / 32 * CL;
  const int row = threadIdx.x / TPR, lane = threadIdx.x & 31;
  const float* const b = sh.part + turn->buffer * (sizeof(sh.part) / 8) + row * N * W;
  if (CL == 1) {
    __syncthreads();
  } else {
    uint64_t* const bar = &sh.bar[turn->buffer];
    if (!turn->gave_up && !mbar_try_wait<true>(bar, turn->parity)) {
      const long long begin = clock64();
      while (!mbar_try_wait<true>(bar, turn->parity))
        if (clock64() - begin > (wait_limit < 0 ? -wait_limit : wait_limit)) {
          turn->gave_up = true;
          sh.silent = 1;
          *(volatile int*)&g_gave_up = 1;
          break;
        }
    }
    turn->parity ^= turn->buffer;          // the barrier's next use has the other parity
  }
  turn->buffer ^= 1;
  if (W < 8) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = b[i * W];
#pragma unroll
      for (int w = 1; w < W; ++w) s += b[i * W + w];
      v[i] = s;
    }
  } else {
    // a part of the warp's lanes for each value
    constexpr int G = 32 / N;
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < W; w += G)
      if (W >= G || lane % G < W) s += b[lane / G * W + w + lane % G];
#pragma unroll
    for (int o = G / 2; o; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xffffffffu, s, i * G);
  }
  if (CL > 1 && turn->gave_up)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __uint_as_float(0x7fc00000u);
}
template <int TPR, int CL, int N, typename S>
__device__ __forceinline__ void row_sums(float* v, S& sh, Turn* turn, long long wait_limit) {
  begin_row_sums<TPR, CL, N>(v, sh, *turn);
  end_row_sums<TPR, CL, N>(v, sh, turn, wait_limit);
}

inline cudaError_t read_gave_up(cudaStream_t stream, bool* gave_up) {
  int flag = 0;
  const int none = 0;
  cudaError_t e = cudaMemcpyFromSymbolAsync(&flag, g_gave_up, sizeof flag, 0, cudaMemcpyDeviceToHost, stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
  if (e == cudaSuccess && flag) {
    e = cudaMemcpyToSymbolAsync(g_gave_up, &none, sizeof none, 0, cudaMemcpyHostToDevice, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
  }
  *gave_up = flag != 0;
  return e;
}

// A launch that may start early (see launch_pdl), of clusters of `cluster` blocks.
template <typename A>
cudaError_t launch_rows(void (*kernel)(A), unsigned blocks, unsigned threads, size_t smem, unsigned cluster, cudaStream_t stream,
                        const A& args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args);
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
