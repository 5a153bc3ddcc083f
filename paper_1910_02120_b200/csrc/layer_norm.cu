// Layer normalisation of rows and its way back (ist_layer_norm_forward / _backward, see ist.h): argument checks, the choice of
// kernels, and the kernels for what the others do not take.
//
//   up to 16 columns     norm_narrow.cu                   a thread takes a row
//   up to 65,536         norm_forward.cu, _backward.cu    4 to 512 threads of a block, or a cluster of blocks, take a row, which is
//                                                         read once; rows that are aligned to pieces of 16 bytes and those that are not
//   wider                here                             a block takes a row and reads it three times (from L2 what that still holds of the
//                                                         rows at work); sums over rows in a launch of their own.  2000 fp32 rows of
//                                                         100,000: 1.10 ms, way back 1.69 ms, 0.22 of the copy rate
//
// The sums over a site's rows for dweight and dbias are taken part by part, a block each, and the parts' sums are added by one more
// launch (norm_join_kernel) in an order that shape, types, alignment and the number of SMs decide; no atomics.  All of it is bound by memory, and short
// of that by issuing instructions, the more so the narrower the types and the less aligned the rows.
#include "../../include/ist.h"

#include <algorithm>
#include <cmath>

#include "norm_rows.cuh"

namespace ist {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kColumns = 32, kLanes = 8;      // of the column kernels' blocks

// Sums of two values over the block, the same in every thread; fixed order.
__device__ __forceinline__ double2 block_sum(double2 v, double2* sh) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  double2 s = make_double2(0., 0.);
#pragma unroll
  for (int w = 0; w < kWarps; ++w) { s.x += sh[w].x; s.y += sh[w].y; }
  return s;
}

// Rows of any width.  Sums in fp64: a thread adds hundreds of values one after the other.
template <typename XT, typename YT>
__global__ void __launch_bounds__(kThreads) norm_forward_any_kernel(const XT* x, int64_t x_ld, int64_t rows, int64_t cols,
                                                                   int64_t site_rows, const float* weight,
                                                                   const float* bias, float eps, YT* y, int64_t y_ld,
                                                                   float* mean_out, float* rstd_out) {
  __shared__ double2 sh[kWarps];
  pdl_wait();
  pdl_trigger();
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const XT* xr = x + r * x_ld;
    double2 s = make_double2(0., 0.);
    for (int64_t j = threadIdx.x; j < cols; j += kThreads) s.x += to_float(xr[j]);
    const float mean = (float)(block_sum(s, sh).x / (double)cols);
    s = make_double2(0., 0.);
    for (int64_t j = threadIdx.x; j < cols; j += kThreads) {
      const float d = to_float(xr[j]) - mean;
      s.x += d;
      s.y += (double)d * d;
    }
    s = block_sum(s, sh);
    // what rounding left of the mean: taken out of the squares here and of the differences below
    const float rest = (float)(s.x / (double)cols);
    double var = s.y / (double)cols - (double)rest * rest;
    if (var < 0.) var = 0.;                              // a NaN stays one
    const float rstd = (float)(1. / sqrt(var + eps));
    const int64_t site = r / site_rows * cols;
    YT* yr = y + r * y_ld;
    for (int64_t j = threadIdx.x; j < cols; j += kThreads) {
      const float h = (to_float(xr[j]) - mean - rest) * rstd;
      yr[j] = from_float<YT>(fmaf(h, weight ? weight[site + j] : 1.f, bias ? bias[site + j] : 0.f));
    }
    if (threadIdx.x == 0) {
      if (mean_out) mean_out[r] = mean + rest;
      if (rstd_out) rstd_out[r] = rstd;
    }
  }
}

template <typename XT, typename DT>
__global__ void __launch_bounds__(kThreads) norm_backward_any_kernel(const DT* dy, int64_t dy_ld, const XT* x, int64_t x_ld,
                                                                    int64_t rows, int64_t cols, int64_t site_rows,
                                                                    const float* weight, const float* mean_in,
                                                                    const float* rstd_in, XT* dx, int64_t dx_ld) {
  __shared__ double2 sh[kWarps];
  pdl_wait();
  pdl_trigger();
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const XT* xr = x + r * x_ld;
    const DT* dr = dy + r * dy_ld;
    const float* wr = weight ? weight + r / site_rows * cols : nullptr;
    const float mean = mean_in[r], rstd = rstd_in[r];
    double2 s = make_double2(0., 0.);
    for (int64_t j = threadIdx.x; j < cols; j += kThreads) {
      const float g = to_float(dr[j]) * (wr ? wr[j] : 1.f);
      s.x += g;
      s.y += (double)g * ((to_float(xr[j]) - mean) * rstd);
    }
    s = block_sum(s, sh);
    const float c0 = (float)(s.x / (double)cols), c1 = (float)(s.y / (double)cols);
    XT* o = dx + r * dx_ld;
    for (int64_t j = threadIdx.x; j < cols; j += kThreads) {
      const float g = to_float(dr[j]) * (wr ? wr[j] : 1.f);
      o[j] = from_float<XT>(rstd * (g - c0 - (to_float(xr[j]) - mean) * rstd * c1));
    }
  }
}

// Sums over a part of a site's rows: part p of site s writes dweight's and dbias's [cols] at out + ((p * sites + s) * 2) * cols.
template <typename XT, typename DT>
__global__ void __launch_bounds__(kColumns* kLanes) norm_columns_any_kernel(const DT* dy, int64_t dy_ld, const XT* x,
                                                                           int64_t x_ld, int64_t cols, int64_t site_rows,
                                                                           int sites, int parts, const float* mean_in,
                                                                           const float* rstd_in, float* out) {
  __shared__ double sh[2][kLanes][kColumns + 1];
  pdl_wait();
  pdl_trigger();
  const int64_t chunks = ceil_div(cols, kColumns);
  const int64_t j = (int64_t)(blockIdx.x % chunks) * kColumns + threadIdx.x;
  const int64_t slab = blockIdx.x / chunks;          // part * sites + site
  const int64_t site = slab % sites, part = slab / sites;
  const int64_t first = site * site_rows + site_rows * part / parts, last = site * site_rows + site_rows * (part + 1) / parts;
  double sw = 0., sb = 0.;
  if (j < cols)
    for (int64_t r = first + threadIdx.y; r < last; r += kLanes) {
      const float d = to_float(dy[r * dy_ld + j]);
      sw += (double)d * ((to_float(x[r * x_ld + j]) - mean_in[r]) * rstd_in[r]);
      sb += d;
    }
  sh[0][threadIdx.y][threadIdx.x] = sw;
  sh[1][threadIdx.y][threadIdx.x] = sb;
  __syncthreads();
  if (threadIdx.y < 2 && j < cols) {
    double s = 0.;
#pragma unroll
    for (int u = 0; u < kLanes; ++u) s += sh[threadIdx.y][u][threadIdx.x];
    out[(slab * 2 + threadIdx.y) * cols + j] = (float)s;
  }
}

// dweight and dbias from the parts' sums.  LANES threads share the parts of four adjacent columns, so that all of a
// column's sums are on their way at once where there are many parts.  Many blocks of few loads each would be slower than the
// pass that leaves the sums (8 sites x 9 parts x 16384 columns: 55 us with 32 columns and 32 lanes to a block).
template <int LANES>
__global__ void __launch_bounds__(kThreads) norm_join_kernel(const float* parts_sums, int64_t cols, int sites, int parts,
                                                            float* dweight, float* dbias) {
  constexpr int kWide = kThreads / LANES * 4;             // columns of a block
  __shared__ float sh[LANES > 1 ? LANES : 1][kWide];
  pdl_wait();
  pdl_trigger();
  // blocks: [site][dweight, dbias][chunk of columns]
  const int64_t chunks = ceil_div(cols, kWide);
  const int x = threadIdx.x % (kThreads / LANES), lane = threadIdx.x / (kThreads / LANES);
  const int64_t first = (int64_t)(blockIdx.x % chunks) * kWide, j = first + x * 4, which = blockIdx.x / chunks % 2;
  const int64_t site = blockIdx.x / (chunks * 2), step = (int64_t)sites * 2 * cols;
  float* const out = which ? dbias : dweight;
  if (!out) return;
  const float* in = parts_sums + (site * 2 + which) * cols + j + lane * step;
  float s[4] = {};
  if (cols % 4 == 0) {
    if (j < cols)
#pragma unroll 4
      for (int p = lane; p < parts; p += LANES, in += LANES * step) {
        float v[4];
        load4(in, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] += v[k];
      }
  } else {
#pragma unroll 4
    for (int p = lane; p < parts; p += LANES, in += LANES * step)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (j + k < cols) s[k] += in[k];
  }
  if (LANES == 1) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (j + k < cols) out[site * cols + j + k] = s[k];
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) sh[lane][x * 4 + k] = s[k];
  __syncthreads();
  for (int c = threadIdx.x; c < kWide; c += kThreads)
    if (first + c < cols) {
      float t = 0.f;
#pragma unroll
      for (int u = 0; u < LANES; ++u) t += sh[u][c];
      out[site * cols + first + c] = t;
    }
}

// Rows of an array in memory: `rows` runs of `run` bytes, `pitch` bytes apart.
struct Span {
  const void* p;
  int64_t rows, run, pitch;
};
// Whether two arrays share a byte.  Rows of equal pitch that lie side by side in one buffer do not, nor does a single run that lies
// between rows.
bool overlap(const Span& a, const Span& b) {
  if (!a.p || !b.p || a.rows == 0 || b.rows == 0) return false;
  const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
  const uintptr_t ea = pa + (uintptr_t)((a.rows - 1) * a.pitch + a.run), eb = pb + (uintptr_t)((b.rows - 1) * b.pitch + b.run);
  if (ea <= pb || eb <= pa) return false;
  if (a.rows == 1 && b.rows == 1) return true;
  if (a.rows > 1 && b.rows > 1 && a.pitch != b.pitch) return true;
  const uintptr_t pitch = (uintptr_t)(a.rows > 1 ? a.pitch : b.pitch);
  const uintptr_t at = pb >= pa ? (pb - pa) % pitch : (pitch - (pa - pb) % pitch) % pitch;      // of b's runs behind a's
  return at < (uintptr_t)a.run || at + (uintptr_t)b.run > pitch;
}

int64_t element(int type) { return type == IST_T_BF16 ? 2 : 4; }
bool known(int type) { return type == IST_T_F32 || type == IST_T_BF16; }
bool aligned(const void* p, int64_t bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

const char* bad_rows(const void* p, int type, int64_t stride, int64_t rows, int64_t cols) {
  if (!known(type)) return "element types are IST_T_F32 and IST_T_BF16";
  if (rows == 0) return nullptr;
  if (!p) return "null rows";
  if (!aligned(p, element(type))) return "rows not aligned to their elements";
  if (stride < cols || stride > (int64_t)1 << 40) return "a row's stride must be in cols..2^40";
  if (stride > ((int64_t)1 << 48) / rows) return "rows * stride must be at most 2^48";
  return nullptr;
}
const char* bad_shape(int64_t rows, int64_t cols, int groups) {
  if (cols < 1 || cols > (int64_t)1 << 30) return "cols must be in 1..2^30";
  // row numbers are 32-bit, and run a few tiles past the last row
  if (rows < 0 || rows > ((int64_t)1 << 31) - 65536) return "rows must be in 0..2^31 - 65536";
  if (groups < 1 || rows % groups) return "groups must be >= 1 and divide rows";
  if (cols > ((int64_t)1 << 40) / groups) return "groups * cols must be at most 2^40";
  return nullptr;
}

// Parts that a site's rows are cut into for the sums over them: as many whole ones as the GPU holds blocks for, but 16,384 elements
// at least to a part.  The number of blocks is a multiple of the sites, so SMs stay idle where that does not come near theirs (40,000
// bf16 rows of 1024: 45 us of one site, 69 us of 75).
int parts_of(int64_t rows, int64_t cols, int groups) {
  const int64_t site_rows = rows / groups;
  int64_t parts, least;
  if (cols <= kNormNarrow) {
    parts = (int64_t)sm_count() * 4 / groups;
    least = 4 * kNormThreads;
  } else if (cols <= kNormWidest) {
    parts = (int64_t)sm_count() * (cols <= 256 ? 2 : 1) / norm_cluster(cols) / groups;
    least = ceil_div(16384, cols);
  } else {
    parts = ceil_div((int64_t)sm_count() * 8, ceil_div(cols, kColumns) * groups);
    least = 4 * kLanes;
  }
  return (int)std::max<int64_t>(1, std::min(parts, ceil_div(site_rows, least)));
}

template <typename F>
void with_types(int a, int b, F f) {
  if (a == IST_T_F32 && b == IST_T_F32) f(float(), float());
  else if (a == IST_T_F32) f(float(), bf16());
  else if (b == IST_T_F32) f(bf16(), float());
  else f(bf16(), bf16());
}

}  // namespace
}  // namespace ist

using namespace ist;

extern "C" ist_status ist_layer_norm_forward(const void* x_dev, int x_type, int64_t x_stride, int64_t rows, int64_t cols,
                                             int groups, const float* weight_dev, const float* bias_dev, float eps,
                                             void* y_dev, int y_type, int64_t y_stride, float* mean_out_dev,
                                             float* rstd_out_dev, void* cuda_stream) {
  const char* why = bad_shape(rows, cols, groups);
  if (!why) why = bad_rows(x_dev, x_type, x_stride, rows, cols);
  if (!why) why = bad_rows(y_dev, y_type, y_stride, rows, cols);
  if (!why && (!aligned(weight_dev, 4) || !aligned(bias_dev, 4) || !aligned(mean_out_dev, 4) || !aligned(rstd_out_dev, 4)))
    why = "weight, bias, mean and rstd must be aligned to 4 bytes";
  if (!why) {
    const Span x{x_dev, rows, cols * element(x_type), x_stride * element(x_type)};
    const Span y{y_dev, rows, cols * element(y_type), y_stride * element(y_type)};
    const Span in[] = {x, {weight_dev, 1, groups * cols * 4, 0}, {bias_dev, 1, groups * cols * 4, 0}};
    const Span out[] = {y, {mean_out_dev, rows ? 1 : 0, rows * 4, 0}, {rstd_out_dev, rows ? 1 : 0, rows * 4, 0}};
    for (int i = 0; i < 3 && !why; ++i) {
      for (int j = 0; j < 3; ++j)
        if (overlap(out[i], in[j])) why = "an output overlaps an input";
      for (int j = 0; j < i; ++j)
        if (overlap(out[i], out[j])) why = "outputs overlap";
    }
  }
  if (!why && !(eps > 0.f && std::isfinite(eps))) why = "eps must be positive and finite";
  if (why) return fail_call(IST_ERR_ARG, "ist_layer_norm_forward: %s", why);
  if (rows == 0) return IST_OK;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  cudaError_t e = cudaSuccess;
  if (cols <= kNormWidest) {
    const NormForward rows_args{x_dev, y_dev, x_stride, y_stride, rows / groups, groups, (int)cols, weight_dev, bias_dev,
                                mean_out_dev, rstd_out_dev, eps, kWaitLimitCycles};
    e = norm_forward_rows(rows_args, x_type == IST_T_BF16, y_type == IST_T_BF16, stream);
  } else {
    const unsigned blocks = (unsigned)std::min<int64_t>(rows, (int64_t)sm_count() * 8);
    with_types(x_type, y_type, [&](auto xt, auto yt) {
      using XT = decltype(xt);
      using YT = decltype(yt);
      e = launch_pdl(norm_forward_any_kernel<XT, YT>, dim3(blocks), dim3(kThreads), 0, stream, (const XT*)x_dev, x_stride,
                     rows, cols, rows / groups, weight_dev, bias_dev, eps, (YT*)y_dev, y_stride, mean_out_dev, rstd_out_dev);
    });
  }
  if (e != cudaSuccess) return fail_call(IST_ERR_CUDA, "ist_layer_norm_forward: %s", cudaGetErrorString(e));
  return IST_OK;
}

extern "C" size_t ist_layer_norm_workspace_bytes(int64_t rows, int64_t cols, int groups) {
  if (bad_shape(rows, cols, groups)) return 0;
  const int parts = parts_of(rows, cols, groups);
  if (cols <= kNormWidest && parts == 1) return 0;      // the sums are written where they belong
  return (size_t)(round_up((int64_t)parts * groups * 2 * cols * 4, 256));
}

extern "C" ist_status ist_layer_norm_backward(const void* dy_dev, int dy_type, int64_t dy_stride, const void* x_dev,
                                              int x_type, int64_t x_stride, int64_t rows, int64_t cols, int groups,
                                              const float* weight_dev, const float* mean_dev, const float* rstd_dev,
                                              void* dx_out_dev, int64_t dx_stride, float* dweight_out_dev,
                                              float* dbias_out_dev, void* workspace_dev, size_t workspace_bytes,
                                              void* cuda_stream) {
  const bool sums = dweight_out_dev || dbias_out_dev;
  const char* why = bad_shape(rows, cols, groups);
  if (!why) why = bad_rows(x_dev, x_type, x_stride, rows, cols);
  if (!why) why = bad_rows(dy_dev, dy_type, dy_stride, rows, cols);
  if (!why && dx_out_dev) why = bad_rows(dx_out_dev, x_type, dx_stride, rows, cols);
  if (!why && rows && !dx_out_dev && !sums) why = "no output is wanted";      // no rows: dx may have no address
  if (!why && rows && (!mean_dev || !rstd_dev)) why = "the forward pass's mean and rstd are needed";
  if (!why && (!aligned(weight_dev, 4) || !aligned(mean_dev, 4) || !aligned(rstd_dev, 4) || !aligned(dweight_out_dev, 4) ||
               !aligned(dbias_out_dev, 4)))
    why = "weight, mean, rstd, dweight and dbias must be aligned to 4 bytes";
  if (why) return fail_call(IST_ERR_ARG, "ist_layer_norm_backward: %s", why);
  const int64_t need = sums ? (int64_t)ist_layer_norm_workspace_bytes(rows, cols, groups) : 0;
  if (need && rows && (!workspace_dev || (int64_t)workspace_bytes < need || !aligned(workspace_dev, 16)))
    return fail_call(IST_ERR_WORKSPACE, "ist_layer_norm_backward: workspace too small or not aligned to 16 bytes (%lld bytes needed)",
                     (long long)need);
  {
    const int one = rows ? 1 : 0;
    const Span in[] = {{dy_dev, rows, cols * element(dy_type), dy_stride * element(dy_type)},
                       {x_dev, rows, cols * element(x_type), x_stride * element(x_type)},
                       {weight_dev, 1, groups * cols * 4, 0}, {mean_dev, one, rows * 4, 0}, {rstd_dev, one, rows * 4, 0}};
    const Span out[] = {{dx_out_dev, rows, cols * element(x_type), dx_stride * element(x_type)},
                        {dweight_out_dev, 1, groups * cols * 4, 0}, {dbias_out_dev, 1, groups * cols * 4, 0},
                        {need && rows ? workspace_dev : nullptr, 1, need, 0}};
    for (int i = 0; i < 4; ++i) {
      for (int j = 0; j < 5; ++j)
        if (overlap(out[i], in[j])) return fail_call(IST_ERR_ARG, "ist_layer_norm_backward: an output overlaps an input");
      for (int j = 0; j < i; ++j)
        if (overlap(out[i], out[j])) return fail_call(IST_ERR_ARG, "ist_layer_norm_backward: outputs overlap");
    }
  }
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  cudaError_t e = cudaSuccess;
  if (rows == 0) {
    if (dweight_out_dev) e = cudaMemsetAsync(dweight_out_dev, 0, (size_t)(groups * cols) * 4, stream);
    if (e == cudaSuccess && dbias_out_dev) e = cudaMemsetAsync(dbias_out_dev, 0, (size_t)(groups * cols) * 4, stream);
    if (e != cudaSuccess) return fail_call(IST_ERR_CUDA, "ist_layer_norm_backward: %s", cudaGetErrorString(e));
    return IST_OK;
  }
  const int64_t site_rows = rows / groups;
  const int64_t chunks = ceil_div(cols, kColumns);
  const int parts = parts_of(rows, cols, groups);
  if (chunks * groups * std::max(parts, 2) >= (int64_t)1 << 31)
    return fail_call(IST_ERR_UNSUPPORTED, "ist_layer_norm_backward: groups * cols is too large");
  float* const part_sums = (float*)workspace_dev;
  const bool join = sums && (parts > 1 || cols > kNormWidest);
  if (cols <= kNormWidest) {
    const NormBackward rows_args{dy_dev, x_dev, dx_out_dev, dy_stride, x_stride, dx_stride, site_rows, groups, (int)cols, weight_dev,
                                 mean_dev, rstd_dev, join ? part_sums : dweight_out_dev, join ? part_sums + cols : dbias_out_dev,
                                 join ? 2 * cols : cols, parts, kWaitLimitCycles};
    e = norm_backward_rows(rows_args, x_type == IST_T_BF16, dy_type == IST_T_BF16, stream);
  } else {
    with_types(x_type, dy_type, [&](auto xt, auto dt) {
      using XT = decltype(xt);
      using DT = decltype(dt);
      if (dx_out_dev)
        e = launch_pdl(norm_backward_any_kernel<XT, DT>, dim3((unsigned)std::min<int64_t>(rows, (int64_t)sm_count() * 8)),
                       dim3(kThreads), 0, stream, (const DT*)dy_dev, dy_stride, (const XT*)x_dev, x_stride, rows, cols, site_rows,
                       weight_dev, mean_dev, rstd_dev, (XT*)dx_out_dev, dx_stride);
      if (e == cudaSuccess && sums)
        e = launch_pdl(norm_columns_any_kernel<XT, DT>, dim3((unsigned)(chunks * groups * parts)), dim3(kColumns, kLanes), 0, stream,
                       (const DT*)dy_dev, dy_stride, (const XT*)x_dev, x_stride, cols, site_rows, groups, parts, mean_dev,
                       rstd_dev, part_sums);
    });
  }
  if (e == cudaSuccess && join) {
    // as many lanes as keep a thread at about eight parts
    auto blocks = [&](int lanes) { return dim3((unsigned)(ceil_div(cols, kThreads / lanes * 4) * groups * 2)); };
    auto launch_join = [&](auto kernel, int lanes) {
      return launch_pdl(kernel, blocks(lanes), dim3(kThreads), 0, stream, (const float*)part_sums, cols, groups, parts,
                        dweight_out_dev, dbias_out_dev);
    };
    e = parts <= 16 ? launch_join(norm_join_kernel<1>, 1) : parts <= 64 ? launch_join(norm_join_kernel<8>, 8)
                                                                       : launch_join(norm_join_kernel<32>, 32);
  }
  if (e != cudaSuccess) return fail_call(IST_ERR_CUDA, "ist_layer_norm_backward: %s", cudaGetErrorString(e));
  return IST_OK;
}

extern "C" ist_status ist_layer_norm_status(void* cuda_stream) {
  bool forward = false, backward = false;
  cudaError_t e = norm_forward_gave_up((cudaStream_t)cuda_stream, &forward);
  if (e == cudaSuccess) e = norm_backward_gave_up((cudaStream_t)cuda_stream, &backward);
  if (e != cudaSuccess) return fail_call(IST_ERR_CUDA, "ist_layer_norm_status: %s", cudaGetErrorString(e));
  if (forward || backward) return fail_call(IST_ERR_DEVICE_TIMEOUT, "ist_layer_norm_status: a wait of blocks that share a row gave up");
  return IST_OK;
}

extern "C" ist_status ist_selftest_layer_norm_wait(const float* x_dev, const float* dy_dev, const float* stats_dev, int64_t rows,
                                                   int64_t cols, float* out_dev, int64_t limit_cycles, void* cuda_stream) {
  const char* why = nullptr;
  if (rows < 1 || rows > 1 << 16) why = "rows must be in 1..65536";
  else if (cols <= 16384 || cols > kNormWidest) why = "cols must be in 16385..65536: rows that several blocks share";
  else if (!x_dev || !out_dev || (dy_dev && !stats_dev)) why = "null rows or statistics";
  else if (!aligned(x_dev, 4) || !aligned(dy_dev, 4) || !aligned(stats_dev, 4) || !aligned(out_dev, 4)) why = "not aligned to 4 bytes";
  else if (limit_cycles < 1 || limit_cycles > kWaitLimitCycles) why = "limit_cycles must be in 1..2e9";
  if (why) return fail_call(IST_ERR_ARG, "ist_selftest_layer_norm_wait: %s", why);
  cudaError_t e = cudaSuccess;
  if (!dy_dev) {
    const NormForward a{x_dev, out_dev, cols, cols, rows, 1, (int)cols, nullptr, nullptr, nullptr, nullptr, 1e-5f, -limit_cycles};
    e = norm_forward_rows(a, false, false, (cudaStream_t)cuda_stream);
  } else {
    const NormBackward a{dy_dev, x_dev, out_dev, cols, cols, cols, rows, 1, (int)cols, nullptr, stats_dev, stats_dev + rows, nullptr,
                         nullptr, cols, 1, -limit_cycles};
    e = norm_backward_rows(a, false, false, (cudaStream_t)cuda_stream);
  }
  if (e != cudaSuccess) return fail_call(IST_ERR_CUDA, "ist_selftest_layer_norm_wait: %s", cudaGetErrorString(e));
  return IST_OK;
}
