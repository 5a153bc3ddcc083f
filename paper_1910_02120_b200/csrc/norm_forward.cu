// Layer norm's forward pass for rows that fit the threads of a block: a row is read once, into registers.
#include <algorithm>
#include <mutex>

#include "norm_rows.cuh"

namespace ist {
namespace {

template <typename XT, typename YT, int V, int NV, int TPR, int RB, int D>
__global__ void __launch_bounds__(TPR > kNormThreads ? TPR : kNormThreads) norm_forward_kernel(const NormForward a) {
  constexpr int kThreads = TPR > kNormThreads ? TPR : kNormThreads, kSlots = kThreads / TPR, kTile = kSlots * RB;
  constexpr int C = NV * V;
  constexpr bool kKeep = C <= 16 && RB * C <= 32;          // weight and bias stay in registers
  extern __shared__ __align__(16) char ring[];
  __shared__ float sh[2 * kThreads / 32 * RB * 2];
  const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
  const int cols = a.cols, room = row_room(cols, sizeof(XT), V == 1);
  const XT* const x = (const XT*)a.x;
  YT* const y = (YT*)a.y;
  const float inv = 1.f / (float)cols;
  const bool wide = (((uintptr_t)a.weight | (uintptr_t)a.bias) & 15) == 0 && cols % 4 == 0;
  // tiles of kTile rows of one site; a block takes a run of them
  const int64_t per_site = ceil_div(a.site_rows, kTile), tiles = per_site * a.sites;
  const int64_t first = tiles * blockIdx.x / gridDim.x, last = tiles * (blockIdx.x + 1) / gridDim.x;
  int turn = 0;

  // row j of this thread's slot in tile k; false if the site has no such row
  auto row_of = [&](int64_t k, int j, int64_t* r) {
    const int64_t site = k / per_site, in_site = (k - site * per_site) * kTile + slot * RB + j;
    *r = site * a.site_rows + in_site;
    return in_site < a.site_rows;
  };
  auto buffer = [&](int64_t k, int j) { return ring + (((k - first) % D * kSlots + slot) * RB + j) * room; };
  auto fetch = [&](int64_t k) {
    if (k < last) {
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        int64_t r;
        if (row_of(k, j, &r)) fetch_row<XT, V, TPR>(x + r * a.x_ld, cols, buffer(k, j), t);
      }
    }
    copy_commit();
  };
  uint16_t odd[RB];
  auto fetch_odd = [&](int64_t k) {
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      int64_t r;
      odd[j] = k < last && row_of(k, j, &r) ? load_odd(x + r * a.x_ld, cols, t) : (uint16_t)0;
    }
  };

  pdl_wait();
  pdl_trigger();
#pragma unroll
  for (int k = 0; k < D - 1; ++k) fetch(first + k);
  if (V == 1) fetch_odd(first);
  float w[kKeep ? C : 1], b[kKeep ? C : 1];
  int64_t held = -1;
  for (int64_t k = first; k < last; ++k) {
    fetch(k + D - 1);
    const int64_t site = k / per_site;
    const float* const ws = a.weight ? a.weight + site * cols : nullptr;
    const float* const bs = a.bias ? a.bias + site * cols : nullptr;
    auto vectors = [&](int i, float* wv, float* bv) {
      const int c = (t + i * TPR) * V;
#pragma unroll
      for (int e = 0; e < V; ++e) { wv[e] = 1.f; bv[e] = 0.f; }
      if (c < cols) {
        if (ws) load_vector<V>(ws + c, wide, wv);
        if (bs) load_vector<V>(bs + c, wide, bv);
      }
    };
    if (kKeep && site != held) {
#pragma unroll
      for (int i = 0; i < NV; ++i) vectors(i, w + i * V, b + i * V);
      held = site;
    }
    copy_wait<D - 1>();
    int64_t r[RB];
    bool live[RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) live[j] = row_of(k, j, &r[j]);
    if (V == 1) {
#pragma unroll
      for (int j = 0; j < RB; ++j)
        if (live[j]) store_odd(x + r[j] * a.x_ld, cols, buffer(k, j), t, odd[j]);
      row_barrier<TPR>();
      fetch_odd(k + 1);
    }
    float v[RB][C], s[RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      const char* const buf = buffer(k, j) + (V == 1 ? (uintptr_t)(x + r[j] * a.x_ld) & 15 : 0);
      s[j] = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (t + i * TPR) * V;
        if (c < cols) {
          unpack<XT, V>(buf + c * sizeof(XT), &v[j][i * V]);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) v[j][i * V + e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) s[j] += v[j][i * V + e];
      }
    }
    row_sums<TPR, RB>(s, sh, &turn);
    float q[2 * RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      const float mean = s[j] *= inv;
      float d1 = 0.f, d2 = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const bool in = (t + i * TPR) * V < cols;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = in ? v[j][i * V + e] - mean : 0.f;
          v[j][i * V + e] = d;
          d1 += d;
          d2 = fmaf(d, d, d2);
        }
      }
      q[j] = d1;
      q[RB + j] = d2;
    }
    row_sums<TPR, 2 * RB>(q, sh, &turn);
    float rstd[RB], shift[RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      const float rest = q[j] * inv;                        // what rounding left of the mean
      float var = fmaf(-rest, rest, q[RB + j] * inv);
      if (var < 0.f) var = 0.f;                             // a NaN stays one
      rstd[j] = inverse_root(var + a.eps);
      shift[j] = -rest * rstd[j];
      if (live[j] && t == 0) {
        if (a.mean) a.mean[r[j]] = s[j] + rest;
        if (a.rstd) a.rstd[r[j]] = rstd[j];
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * V;
      float wv[V], bv[V];
      if (kKeep) {
#pragma unroll
        for (int e = 0; e < V; ++e) { wv[e] = w[kKeep ? i * V + e : 0]; bv[e] = b[kKeep ? i * V + e : 0]; }
      } else {
        vectors(i, wv, bv);
      }
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = fmaf(fmaf(v[j][i * V + e], rstd[j], shift[j]), wv[e], bv[e]);
        if (live[j] && c < cols) pack<YT, V>(y + r[j] * a.y_ld + c, o);
      }
    }
    if (V == 1) row_barrier<TPR>();                         // the next fetch writes what this tile was read from
  }
  copy_wait<0>();
}

template <typename XT, typename YT, int V, int NV, int TPR, int RB, int D>
cudaError_t launch(const NormForward& a, cudaStream_t stream) {
  constexpr int kThreads = TPR > kNormThreads ? TPR : kNormThreads, kSlots = kThreads / TPR;
  const auto kernel = norm_forward_kernel<XT, YT, V, NV, TPR, RB, D>;
  const int smem = D * kSlots * RB * row_room(a.cols, sizeof(XT), V == 1);
  // the most that any width of this instance asks for, and how many blocks an SM holds then
  constexpr int kMost = D * kSlots * RB * row_room(TPR * V * NV, sizeof(XT), V == 1);
  static_assert(kMost <= 200 * 1024, "ring too large");
  static std::once_flag once;
  static cudaError_t ready = cudaSuccess;
  static int resident = 1;
  std::call_once(once, [&] {
    ready = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (ready == cudaSuccess) ready = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kernel, kThreads, kMost);
    if (resident < 1) resident = 1;
  });
  if (ready != cudaSuccess) return ready;
  const int64_t tiles = ceil_div(a.site_rows, kSlots * RB) * a.sites;
  const int64_t blocks = std::min<int64_t>(tiles, (int64_t)sm_count() * resident);
  return launch_pdl(kernel, dim3((unsigned)blocks), dim3(kThreads), smem, stream, a);
}

template <typename XT, typename YT>
bool dispatch(const NormForward& a, cudaStream_t stream, cudaError_t* e) {
  constexpr int V = sizeof(XT) == 2 && sizeof(YT) == 2 ? 8 : 4;
  auto fits = [&](const void* p, int64_t ld, int size) { return (((uintptr_t)p | (uintptr_t)(ld * size)) & (V * size - 1)) == 0; };
  const bool pieces = a.cols % V == 0 && fits(a.x, a.x_ld, sizeof(XT)) && fits(a.y, a.y_ld, sizeof(YT));
  const int n = a.cols;
#define TAKE(most, v, nv, tpr, rb, d) \
  if (n <= (most)) return *e = launch<XT, YT, v, nv, tpr, rb, d>(a, stream), true
  if (pieces) {
    TAKE(64, V, 1, 64 / V, 1, 4);
    TAKE(128, V, 1, 128 / V, 1, 4);
    TAKE(256, V, 8 / V, 32, 1, 4);
    TAKE(512, V, 16 / V, 32, 1, 4);
    TAKE(1024, V, 32 / V, 32, 1, 3);
    TAKE(2048, V, 16 / V, 128, 2, 3);
    TAKE(4096, V, 16 / V, 256, 2, 3);
    TAKE(8192, V, 16 / V, 512, 1, 3);
    TAKE(16384, V, 16 / V, 1024, 1, 2);
  } else {
    TAKE(8, 1, 1, 8, 1, 4);
    TAKE(64, 1, 2, 32, 1, 4);
    TAKE(256, 1, 8, 32, 1, 4);
    TAKE(1024, 1, 32, 32, 1, 3);
    TAKE(2048, 1, 16, 128, 2, 3);
    TAKE(4096, 1, 16, 256, 2, 3);
    TAKE(8192, 1, 16, 512, 1, 3);
    TAKE(16384, 1, 16, 1024, 1, 2);
  }
#undef TAKE
  return false;
}

}  // namespace

bool norm_forward_rows(const NormForward& a, bool x_bf16, bool y_bf16, cudaStream_t stream, cudaError_t* e) {
  return x_bf16 ? y_bf16 ? dispatch<bf16, bf16>(a, stream, e) : dispatch<bf16, float>(a, stream, e)
                : y_bf16 ? dispatch<float, bf16>(a, stream, e) : dispatch<float, float>(a, stream, e);
}

}  // namespace ist
