// Layer norm's way back for rows that fit the threads of a block: dy and x are read once, dx written, and the sums
// over rows that dweight and dbias need are kept in registers, a column always with the same thread.
#include <algorithm>
#include <mutex>

#include "norm_rows.cuh"

namespace ist {
namespace {

template <typename XT, typename DT, int V, int NV, int TPR, int RB, int D>
__global__ void __launch_bounds__(TPR > kNormThreads ? TPR : kNormThreads) norm_backward_kernel(const NormBackward a) {
  constexpr int kThreads = TPR > kNormThreads ? TPR : kNormThreads, kSlots = kThreads / TPR, kTile = kSlots * RB;
  constexpr int C = NV * V;
  extern __shared__ __align__(16) char ring[];
  __shared__ float sh[2 * kThreads / 32 * RB * 2];
  const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
  const int cols = a.cols, x_room = row_room(cols, sizeof(XT), V == 1), room = x_room + row_room(cols, sizeof(DT), V == 1);
  const int64_t site = blockIdx.x % a.sites, part = blockIdx.x / a.sites;
  // this block's rows of its site
  const int64_t begin = a.site_rows * part / a.parts, end = a.site_rows * (part + 1) / a.parts;
  const int64_t row0 = site * a.site_rows;
  const XT* const x = (const XT*)a.x + row0 * a.x_ld;
  const DT* const dy = (const DT*)a.dy + row0 * a.dy_ld;
  XT* const dx = a.dx ? (XT*)a.dx + row0 * a.dx_ld : nullptr;
  const float inv = 1.f / (float)cols;
  const int tiles = (int)ceil_div(end - begin, kTile);
  int turn = 0;

  auto row_of = [&](int k, int j) { return begin + (int64_t)k * kTile + slot * RB + j; };
  auto buffer = [&](int k, int j) { return ring + ((k % D * kSlots + slot) * RB + j) * room; };
  auto fetch = [&](int k) {
    if (k < tiles) {
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        const int64_t r = row_of(k, j);
        if (r < end) {
          fetch_row<XT, V, TPR>(x + r * a.x_ld, cols, buffer(k, j), t);
          fetch_row<DT, V, TPR>(dy + r * a.dy_ld, cols, buffer(k, j) + x_room, t);
        }
      }
    }
    copy_commit();
  };
  // what of the next tile is carried in registers: the rows' statistics, and elements that no copy takes
  float next_mean[RB], next_rstd[RB];
  uint16_t odd_x[RB], odd_d[RB];
  auto fetch_more = [&](int k) {
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      const int64_t r = row_of(k, j);
      const bool live = r < end;
      next_mean[j] = live ? a.mean[row0 + r] : 0.f;
      next_rstd[j] = live ? a.rstd[row0 + r] : 0.f;
      if (V == 1) {
        odd_x[j] = live ? load_odd(x + r * a.x_ld, cols, t) : (uint16_t)0;
        odd_d[j] = live ? load_odd(dy + r * a.dy_ld, cols, t) : (uint16_t)0;
      }
    }
  };

  pdl_wait();
  pdl_trigger();
#pragma unroll
  for (int k = 0; k < D - 1; ++k) fetch(k);
  fetch_more(0);
  float w[C], aw[C], ab[C];
  {
    const float* const ws = a.weight ? a.weight + site * cols : nullptr;
    const bool wide = ((uintptr_t)ws & 15) == 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * V;
#pragma unroll
      for (int e = 0; e < V; ++e) w[i * V + e] = 1.f;
      if (ws && c < cols) load_vector<V>(ws + c, wide, w + i * V);
    }
  }
#pragma unroll
  for (int e = 0; e < C; ++e) aw[e] = ab[e] = 0.f;
  for (int k = 0; k < tiles; ++k) {
    fetch(k + D - 1);
    copy_wait<D - 1>();
    float mean[RB], rstd[RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      mean[j] = next_mean[j];
      rstd[j] = next_rstd[j];
      const int64_t r = row_of(k, j);
      if (V == 1 && r < end) {
        store_odd(x + r * a.x_ld, cols, buffer(k, j), t, odd_x[j]);
        store_odd(dy + r * a.dy_ld, cols, buffer(k, j) + x_room, t, odd_d[j]);
      }
    }
    if (V == 1) row_barrier<TPR>();
    fetch_more(k + 1);
    float h[RB][C], g[RB][C], s[2 * RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      const int64_t r = row_of(k, j);
      const bool live = r < end;
      const char* const bx = buffer(k, j) + (V == 1 ? (uintptr_t)(x + r * a.x_ld) & 15 : 0);
      const char* const bd = buffer(k, j) + x_room + (V == 1 ? (uintptr_t)(dy + r * a.dy_ld) & 15 : 0);
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (t + i * TPR) * V;
        float xv[V], dv[V];
        if (live && c < cols) {
          unpack<XT, V>(bx + c * sizeof(XT), xv);
          unpack<DT, V>(bd + c * sizeof(DT), dv);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) { xv[e] = mean[j]; dv[e] = 0.f; }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int q = i * V + e;
          h[j][q] = (xv[e] - mean[j]) * rstd[j];
          aw[q] = fmaf(dv[e], h[j][q], aw[q]);
          ab[q] += dv[e];
          g[j][q] = dv[e] * w[q];
          s0 += g[j][q];
          s1 = fmaf(g[j][q], h[j][q], s1);
        }
      }
      s[j] = s0;
      s[RB + j] = s1;
    }
    if (dx) {
      row_sums<TPR, 2 * RB>(s, sh, &turn);
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        const int64_t r = row_of(k, j);
        if (r < end) {
          const float c0 = s[j] * inv, c1 = s[RB + j] * inv;
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * V;
            float o[V];
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] = rstd[j] * fmaf(-h[j][i * V + e], c1, g[j][i * V + e] - c0);
            if (c < cols) pack<XT, V>(dx + r * a.dx_ld + c, o);
          }
        }
      }
    }
    if (V == 1) row_barrier<TPR>();                         // the next fetch writes what this tile was read from
  }
  copy_wait<0>();
  if (!a.wsum && !a.bsum) return;
  // the slots' sums are joined in shared memory, slot after slot
  if (kSlots > 1) {
    __syncthreads();
    float* const f = reinterpret_cast<float*>(ring);        // [slot][2][C][TPR]
#pragma unroll
    for (int e = 0; e < C; ++e) {
      f[((slot * 2 + 0) * C + e) * TPR + t] = aw[e];
      f[((slot * 2 + 1) * C + e) * TPR + t] = ab[e];
    }
    __syncthreads();
    for (int q = threadIdx.x; q < 2 * C * TPR; q += kThreads) {
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < kSlots; ++u) sum += f[u * 2 * C * TPR + q];
      const int which = q / (C * TPR), e = q % (C * TPR) / TPR, tt = q % TPR;
      const int c = (tt + e / V * TPR) * V + e % V;
      float* const out = which ? a.bsum : a.wsum;
      if (out && c < cols) out[(part * a.sites + site) * a.sum_ld + c] = sum;
    }
  } else {
    const int64_t at = (part * a.sites + site) * a.sum_ld;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * V;
      if (c < cols) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (a.wsum) a.wsum[at + c + e] = aw[i * V + e];
          if (a.bsum) a.bsum[at + c + e] = ab[i * V + e];
        }
      }
    }
  }
}

template <typename XT, typename DT, int V, int NV, int TPR, int RB, int D>
cudaError_t launch(const NormBackward& a, cudaStream_t stream) {
  constexpr int kThreads = TPR > kNormThreads ? TPR : kNormThreads, kSlots = kThreads / TPR;
  const auto kernel = norm_backward_kernel<XT, DT, V, NV, TPR, RB, D>;
  constexpr int kJoin = kSlots > 1 ? kSlots * 2 * NV * V * TPR * 4 : 0;
  const int rows = D * kSlots * RB * (row_room(a.cols, sizeof(XT), V == 1) + row_room(a.cols, sizeof(DT), V == 1));
  constexpr int kMost = std::max(kJoin, D * kSlots * RB * (row_room(TPR * V * NV, sizeof(XT), V == 1) + row_room(TPR * V * NV, sizeof(DT), V == 1)));
  static_assert(kMost <= 225 * 1024, "ring too large");
  static std::once_flag once;
  static cudaError_t ready = cudaSuccess;
  std::call_once(once, [&] { ready = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost); });
  if (ready != cudaSuccess) return ready;
  return launch_pdl(kernel, dim3((unsigned)(a.sites * (int64_t)a.parts)), dim3(kThreads), std::max(rows, kJoin), stream, a);
}

template <typename XT, typename DT>
bool dispatch(const NormBackward& a, cudaStream_t stream, cudaError_t* e) {
  constexpr int V = sizeof(XT) == 2 && sizeof(DT) == 2 ? 8 : 4, S = sizeof(XT) + sizeof(DT);
  auto fits = [&](const void* p, int64_t ld, int size) { return (((uintptr_t)p | (uintptr_t)(ld * size)) & (V * size - 1)) == 0; };
  const bool pieces = a.cols % V == 0 && fits(a.x, a.x_ld, sizeof(XT)) && fits(a.dy, a.dy_ld, sizeof(DT)) &&
                      (!a.dx || fits(a.dx, a.dx_ld, sizeof(XT)));
  const int n = a.cols;
#define TAKE(most, v, nv, tpr, rb, d) \
  if (n <= (most)) return *e = launch<XT, DT, v, nv, tpr, rb, d>(a, stream), true
  if (pieces) {
    TAKE(64, V, 1, 64 / V, 1, 4);
    TAKE(128, V, 1, 128 / V, 1, 4);
    TAKE(256, V, 8 / V, 32, 1, 4);
    TAKE(512, V, 16 / V, 32, 1, 3);
    TAKE(1024, V, 16 / V, 64, 1, 3);
    TAKE(2048, V, 16 / V, 128, 1, 3);
    TAKE(4096, V, 16 / V, 256, 1, 3);
    TAKE(8192, V, 16 / V, 512, 1, 3);
    if constexpr (S < 8) TAKE(16384, V, 16 / V, 1024, 1, 2);
  } else {
    TAKE(8, 1, 1, 8, 1, 4);
    TAKE(64, 1, 2, 32, 1, 4);
    TAKE(256, 1, 8, 32, 1, 4);
    TAKE(512, 1, 16, 32, 1, 3);
    TAKE(1024, 1, 16, 64, 1, 3);
    TAKE(2048, 1, 16, 128, 1, 3);
    TAKE(4096, 1, 16, 256, 1, 3);
    TAKE(8192, 1, 16, 512, 1, 3);
    if constexpr (S < 8) TAKE(16384, 1, 16, 1024, 1, 2);
  }
#undef TAKE
  return false;
}

}  // namespace

bool norm_backward_rows(const NormBackward& a, bool x_bf16, bool dy_bf16, cudaStream_t stream, cudaError_t* e) {
  return x_bf16 ? dy_bf16 ? dispatch<bf16, bf16>(a, stream, e) : dispatch<bf16, float>(a, stream, e)
                : dy_bf16 ? dispatch<float, bf16>(a, stream, e) : dispatch<float, float>(a, stream, e);
}

}  // namespace ist
