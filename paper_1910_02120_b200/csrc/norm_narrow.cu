// Layer norm's two passes for rows of up to 16 elements: a thread takes a row, and a warp's rows together are whole lines.
#include <algorithm>

#include "norm_rows.cuh"

namespace ist {
namespace {

constexpr int kThreads = kNormThreads, kWarps = kThreads / 32;

// A row of up to NC elements; what lies behind its end is zero.  WIDE: NC elements, aligned to 16 bytes.
template <typename T, int NC, bool WIDE>
__device__ __forceinline__ void load_row(const T* row, int cols, float* v) {
  constexpr int E = 16 / sizeof(T);
  if constexpr (WIDE && NC % E == 0) {
#pragma unroll
    for (int c = 0; c < NC; c += E) unpack<T, E>(row + c, v + c);
  } else {
#pragma unroll
    for (int c = 0; c < NC; ++c) v[c] = WIDE || c < cols ? to_float(row[c]) : 0.f;
  }
}
template <typename T, int NC, bool WIDE>
__device__ __forceinline__ void store_row(T* row, int cols, const float* v) {
  constexpr int E = 16 / sizeof(T);
  if constexpr (WIDE && NC % E == 0) {
#pragma unroll
    for (int c = 0; c < NC; c += E) pack<T, E>(row + c, v + c);
  } else {
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (WIDE || c < cols) row[c] = from_float<T>(v[c]);
  }
}

template <typename XT, typename YT, int NC, bool WIDE>
__global__ void __launch_bounds__(kThreads) norm_forward_narrow_kernel(const NormForward a) {
  pdl_wait();
  pdl_trigger();
  const int cols = a.cols, rows = (int)(a.site_rows * a.sites), site_rows = (int)a.site_rows;
  const float inv = 1.f / (float)cols;
  float w[NC], b[NC];
  int held = -1;
  for (int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x; k < rows; k += (int64_t)gridDim.x * kThreads) {
    const int r = (int)k, site = r / site_rows;
    if (site != held) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        w[c] = a.weight && c < cols ? a.weight[(int64_t)site * cols + c] : 1.f;
        b[c] = a.bias && c < cols ? a.bias[(int64_t)site * cols + c] : 0.f;
      }
      held = site;
    }
    float v[NC], s = 0.f;
    load_row<XT, NC, WIDE>((const XT*)a.x + r * a.x_ld, cols, v);
#pragma unroll
    for (int c = 0; c < NC; ++c) s += v[c];
    // rounded as written, so that a call without statistics gives the same bits
    const float mean = __fmul_rn(s, inv);
    float d1 = 0.f, d2 = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      v[c] = WIDE || c < cols ? __fsub_rn(v[c], mean) : 0.f;
      d1 += v[c];
      d2 = fmaf(v[c], v[c], d2);
    }
    const float rest = __fmul_rn(d1, inv);              // what rounding left of the mean
    float var = fmaf(-rest, rest, __fmul_rn(d2, inv));
    if (var < 0.f) var = 0.f;                           // a NaN stays one
    const float rstd = inverse_root(var + a.eps), shift = __fmul_rn(-rest, rstd);
#pragma unroll
    for (int c = 0; c < NC; ++c) v[c] = fmaf(fmaf(v[c], rstd, shift), w[c], b[c]);
    store_row<YT, NC, WIDE>((YT*)a.y + r * a.y_ld, cols, v);
    if (a.mean) a.mean[r] = mean + rest;
    if (a.rstd) a.rstd[r] = rstd;
  }
}

template <typename XT, typename DT, int NC, bool WIDE>
__global__ void __launch_bounds__(kThreads) norm_backward_narrow_kernel(const NormBackward a) {
  __shared__ float sh[kWarps][2 * NC];
  pdl_wait();
  pdl_trigger();
  const int cols = a.cols, site = (int)(blockIdx.x % a.sites), part = (int)(blockIdx.x / a.sites);
  const int row0 = (int)(site * a.site_rows), begin = row0 + (int)(a.site_rows * part / a.parts);
  const int end = row0 + (int)(a.site_rows * (part + 1) / a.parts);
  const float inv = 1.f / (float)cols;
  float w[NC], aw[NC] = {}, ab[NC] = {};
#pragma unroll
  for (int c = 0; c < NC; ++c) w[c] = a.weight && c < cols ? a.weight[(int64_t)site * cols + c] : 1.f;
  for (int64_t k = begin + (int)threadIdx.x; k < end; k += kThreads) {
    const int r = (int)k;
    float h[NC], g[NC], s0 = 0.f, s1 = 0.f;
    load_row<XT, NC, WIDE>((const XT*)a.x + r * a.x_ld, cols, h);
    load_row<DT, NC, WIDE>((const DT*)a.dy + r * a.dy_ld, cols, g);
    const float mean = a.mean[r], rstd = a.rstd[r];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (WIDE || c < cols) {
        h[c] = (h[c] - mean) * rstd;
        aw[c] = fmaf(g[c], h[c], aw[c]);
        ab[c] += g[c];
        g[c] = __fmul_rn(g[c], w[c]);
        s0 += g[c];
        s1 = fmaf(g[c], h[c], s1);
      }
    }
    if (a.dx) {
      // rows of one or two elements have next to nothing left after the subtractions: every product is rounded as it was for
      // the sums, so that what cancels does
      const float m0 = s0 * inv, m1 = s1 * inv;
#pragma unroll
      for (int c = 0; c < NC; ++c) g[c] = rstd * __fsub_rn(__fsub_rn(g[c], m0), __fmul_rn(h[c], m1));
      store_row<XT, NC, WIDE>((XT*)a.dx + r * a.dx_ld, cols, g);
    }
  }
  if (!a.wsum && !a.bsum) return;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      aw[c] += __shfl_xor_sync(0xffffffffu, aw[c], o);
      ab[c] += __shfl_xor_sync(0xffffffffu, ab[c], o);
    }
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      sh[threadIdx.x >> 5][c] = aw[c];
      sh[threadIdx.x >> 5][NC + c] = ab[c];
    }
  __syncthreads();
  if (threadIdx.x < 2 * NC) {
    const int c = threadIdx.x % NC;
    float s = 0.f;
#pragma unroll
    for (int u = 0; u < kWarps; ++u) s += sh[u][threadIdx.x];
    float* const out = threadIdx.x < NC ? a.wsum : a.bsum;
    if (out && c < cols) out[((int64_t)part * a.sites + site) * a.sum_ld + c] = s;
  }
}

// Whether rows of `nc` elements can be moved in 16-byte pieces, or as elements that need no test.
bool wide_rows(const void* p, int64_t ld, int64_t size) { return ((uintptr_t)p & 15) == 0 && ld * size % 16 == 0; }

template <typename F>
void with_width(int cols, F f) {
  if (cols <= 4) f(std::integral_constant<int, 4>());
  else if (cols <= 8) f(std::integral_constant<int, 8>());
  else f(std::integral_constant<int, 16>());
}
template <typename XT, typename YT>
cudaError_t forward(const NormForward& a, cudaStream_t stream) {
  const bool wide = wide_rows(a.x, a.x_ld, sizeof(XT)) && wide_rows(a.y, a.y_ld, sizeof(YT));
  const int64_t blocks = std::min<int64_t>(ceil_div(a.site_rows * a.sites, kThreads), (int64_t)sm_count() * 8);
  cudaError_t e = cudaSuccess;
  with_width(a.cols, [&](auto nc) {
    constexpr int NC = decltype(nc)::value;
    e = launch_rows(wide && a.cols == NC ? norm_forward_narrow_kernel<XT, YT, NC, true> : norm_forward_narrow_kernel<XT, YT, NC, false>,
                    (unsigned)blocks, kThreads, 0, 1, stream, a);
  });
  return e;
}
template <typename XT, typename DT>
cudaError_t backward(const NormBackward& a, cudaStream_t stream) {
  const bool wide = wide_rows(a.x, a.x_ld, sizeof(XT)) && wide_rows(a.dy, a.dy_ld, sizeof(DT)) && (!a.dx || wide_rows(a.dx, a.dx_ld, sizeof(XT)));
  cudaError_t e = cudaSuccess;
  with_width(a.cols, [&](auto nc) {
    constexpr int NC = decltype(nc)::value;
    e = launch_rows(wide && a.cols == NC ? norm_backward_narrow_kernel<XT, DT, NC, true> : norm_backward_narrow_kernel<XT, DT, NC, false>,
                    (unsigned)((int64_t)a.sites * a.parts), kThreads, 0, 1, stream, a);
  });
  return e;
}

}  // namespace

cudaError_t norm_forward_narrow(const NormForward& a, bool x_bf16, bool y_bf16, cudaStream_t stream) {
  return x_bf16 ? y_bf16 ? forward<bf16, bf16>(a, stream) : forward<bf16, float>(a, stream)
                : y_bf16 ? forward<float, bf16>(a, stream) : forward<float, float>(a, stream);
}
cudaError_t norm_backward_narrow(const NormBackward& a, bool x_bf16, bool dy_bf16, cudaStream_t stream) {
  return x_bf16 ? dy_bf16 ? backward<bf16, bf16>(a, stream) : backward<bf16, float>(a, stream)
                : dy_bf16 ? backward<float, bf16>(a, stream) : backward<float, float>(a, stream);
}

}  // namespace ist
