// Layer norm's forward pass for rows that fit the threads of a block or a cluster: a row is read once, into registers.
#include <algorithm>

#include "norm_rows.cuh"

namespace ist {
namespace {

// 51,200 bf16 rows of 1024: 36.6 us, 0.88 of the copy rate; 4096 fp32 rows of 16384 to bf16: 67 us, 0.92.  9600 fp32 rows of 1001,
// which start anywhere: 14.1 us, against 11.5 us for 1000 columns; 2^26 bf16 values in rows of 1001 64 us, of 1008 49 us.
template <typename XT, typename YT, int V, int NV, int TPR, int RB, int D, int CL, int LEAST>
__global__ void __launch_bounds__(TPR > kNormThreads ? TPR : kNormThreads) norm_forward_kernel(const NormForward a) {
  constexpr int kThreads = TPR > kNormThreads ? TPR : kNormThreads, kSlots = kThreads / TPR, kTile = kSlots * RB;
  constexpr int C = NV * V;
  constexpr bool FULL = LEAST == TPR * C;                  // of a block's columns: no piece is missing
  static_assert(C * (RB + 2) <= 96, "weight and bias stay in registers beside the rows");
  extern __shared__ __align__(128) char ring[];
  __shared__ RowSums<kThreads, CL, 2 * RB> sh;
  const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
  // columns of this block: the row's, or the part of them that is this block's in its cluster
  const int width = FULL ? TPR * C : part_width(a.cols, CL);
  const int c0 = CL > 1 ? (int)cluster_ctarank() * width : 0, cols = CL > 1 ? max(min(a.cols - c0, width), 0) : a.cols;
  const int room = row_room(width, sizeof(XT), V == 1);
  const XT* const x = (const XT*)a.x + c0;
  YT* const y = (YT*)a.y + c0;
  const float inv = 1.f / (float)a.cols;
  const bool wide = (((uintptr_t)a.weight | (uintptr_t)a.bias) & 15) == 0 && a.cols % 4 == 0;
  // tiles of kTile rows of one site; a block (or cluster) takes a run of them
  const int per_site = (int)ceil_div(a.site_rows, kTile), site_rows = (int)a.site_rows;
  const int64_t tiles = (int64_t)per_site * a.sites;
  const int64_t block = blockIdx.x / CL, blocks = gridDim.x / CL;
  const int64_t begin = tiles * block / blocks;
  int todo = (int)(tiles * (block + 1) / blocks - begin), to_fetch = todo;

  // The slot's rows of a tile: r, r + 1, ..., of which the first `left` are the site's.
  struct Walk {
    int site, tile, r, left;
  };
  auto start = [&](int64_t k) {
    Walk w;
    w.site = (int)(k / per_site);
    w.tile = (int)(k - (int64_t)w.site * per_site);
    w.left = site_rows - (w.tile * kTile + slot * RB);
    w.r = w.site * site_rows + w.tile * kTile + slot * RB;
    return w;
  };
  auto advance = [&](Walk& w) {
    w.r += kTile;
    w.left -= kTile;
    if (++w.tile == per_site) {
      w.tile = 0;
      ++w.site;
      w.left = site_rows - slot * RB;
      w.r = w.site * site_rows + slot * RB;
    }
  };
  Walk in = start(begin), at = in;
  int in_stage = 0, stage = 0;
  auto buffer = [&](int stage, int j) { return ring + ((stage * kSlots + slot) * RB + j) * room; };
  auto fetch = [&]() {
    if (to_fetch > 0) {
#pragma unroll
      for (int j = 0; j < RB; ++j)
        if (j < in.left) fetch_row<XT, V, NV, TPR, LEAST>(x + (int64_t)(in.r + j) * a.x_ld, cols, buffer(in_stage, j), t);
      --to_fetch;
      advance(in);
      if (++in_stage == D) in_stage = 0;
    }
    copy_commit();
  };
  uint16_t odd[RB];
  auto fetch_odd = [&](const Walk& w) {
#pragma unroll
    for (int j = 0; j < RB; ++j) odd[j] = j < w.left ? load_odd(x + (int64_t)(w.r + j) * a.x_ld, cols, t) : (uint16_t)0;
  };
  auto here = [&](int i) { return (i + 1) * TPR * V <= LEAST || (t + i * TPR) * V < cols; };

  Turn turn = begin_sums<CL>(sh, a.wait_limit);
  pdl_wait();
  pdl_trigger();
#pragma unroll
  for (int k = 0; k < D - 1; ++k) fetch();
  if (V == 1 && todo > 0) fetch_odd(at);
  pair w[C / 2], b[C / 2];
  int held = -1;
  auto vector = [&](const float* p, int site, float none, int i, float* out) {
#pragma unroll
    for (int e = 0; e < V; ++e) out[e] = none;
    if (p && here(i)) load_vector<V>(p + (int64_t)site * a.cols + c0 + (t + i * TPR) * V, wide, out);
  };
  for (; todo > 0; --todo) {
    fetch();
    if (at.site != held) {
      float f[C];
#pragma unroll
      for (int i = 0; i < NV; ++i) vector(a.weight, at.site, 1.f, i, f + i * V);
#pragma unroll
      for (int e = 0; e < C / 2; ++e) w[e] = make_pair2(f[2 * e], f[2 * e + 1]);
#pragma unroll
      for (int i = 0; i < NV; ++i) vector(a.bias, at.site, 0.f, i, f + i * V);
#pragma unroll
      for (int e = 0; e < C / 2; ++e) b[e] = make_pair2(f[2 * e], f[2 * e + 1]);
      held = at.site;
    }
    copy_wait<D - 1>();
    const Walk now = at;
    advance(at);
    if (V == 1) {
#pragma unroll
      for (int j = 0; j < RB; ++j)
        if (j < now.left) store_odd(x + (int64_t)(now.r + j) * a.x_ld, cols, buffer(stage, j), t, odd[j]);
      row_barrier<TPR>();
      if (todo > 1) fetch_odd(at);
    }
    pair v[RB][C / 2];
    float s[RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      const char* const buf =
          buffer(stage, j) + (V == 1 ? (int)((uintptr_t)(x + (int64_t)(now.r + j) * a.x_ld) & 15) : 0) + t * (V * (int)sizeof(XT));
      float f[C];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (here(i)) {
          unpack<XT, V>(buf + i * (TPR * V * sizeof(XT)), f + i * V);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) f[i * V + e] = 0.f;
        }
      }
      pair sum = v[j][0] = make_pair2(f[0], f[1]);
#pragma unroll
      for (int e = 1; e < C / 2; ++e) {
        v[j][e] = make_pair2(f[2 * e], f[2 * e + 1]);
        sum = add(sum, v[j][e]);
      }
      s[j] = first_of(sum) + second_of(sum);
    }
    row_sums<TPR, CL, RB>(s, sh, &turn, a.wait_limit);
    float q[2 * RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      s[j] *= inv;
      const pair minus = both(-s[j]);
      pair d1 = both(0.f), d2 = both(0.f);
#pragma unroll
      for (int e = 0; e < C / 2; ++e) {
        pair d = add(v[j][e], minus);
        if (!FULL) {
          const bool one = here(2 * e / V), two = V == 1 ? here(2 * e + 1) : one;
          d = make_pair2(one ? first_of(d) : 0.f, two ? second_of(d) : 0.f);
        }
        v[j][e] = d;
        d1 = add(d1, d);
        d2 = fma(d, d, d2);
      }
      q[j] = first_of(d1) + second_of(d1);
      q[RB + j] = first_of(d2) + second_of(d2);
    }
    row_sums<TPR, CL, 2 * RB>(q, sh, &turn, a.wait_limit);
    pair rstd[RB], shift[RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      const float rest = q[j] * inv;                        // what rounding left of the mean
      float var = fmaf(-rest, rest, q[RB + j] * inv);
      if (var < 0.f) var = 0.f;                             // a NaN stays one
      const float r = inverse_root(var + a.eps);
      rstd[j] = both(r);
      shift[j] = both(-rest * r);
      if (j < now.left && t == 0 && c0 == 0) {
        if (a.mean) a.mean[now.r + j] = s[j] + rest;
        if (a.rstd) a.rstd[now.r + j] = r;
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      // pairs of this piece; single elements (V = 1) are taken two pieces at a time
      constexpr int kPairs = V == 1 ? 1 : V / 2;
      if (V == 1 && i % 2) continue;
      const int p0 = V == 1 ? i / 2 : i * (V / 2);
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        float o[2 * kPairs];
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
          const pair r = fma(fma(v[j][p0 + e], rstd[j], shift[j]), w[p0 + e], b[p0 + e]);
          o[2 * e] = first_of(r);
          o[2 * e + 1] = second_of(r);
        }
        if (j < now.left) {
          YT* const to = y + (int64_t)(now.r + j) * a.y_ld + t * V;
          if (here(i)) pack<YT, V>(to + i * (TPR * V), o);
          if (V == 1 && here(i + 1)) pack<YT, V>(to + (i + 1) * TPR, o + 1);
        }
      }
    }
    if (++stage == D) stage = 0;
    if (V == 1) row_barrier<TPR>();                         // the next fetch writes what this tile was read from
  }
  copy_wait<0>();
  finish_sums<CL>(turn);
}

template <typename XT, typename YT, int V, int NV, int TPR, int RB, int D, int CL, int LEAST>
cudaError_t launch(const NormForward& a, cudaStream_t stream) {
  constexpr int kThreads = TPR > kNormThreads ? TPR : kNormThreads, kSlots = kThreads / TPR;
  const auto kernel = norm_forward_kernel<XT, YT, V, NV, TPR, RB, D, CL, LEAST>;
  // the most that any width of this instance asks for, and how many blocks an SM holds then
  constexpr int kMost = D * kSlots * RB * row_room(TPR * V * NV, sizeof(XT), V == 1);
  static_assert(kMost <= 225 * 1024, "ring too large");
  static OncePerDevice<KernelReady> once;
  const KernelReady ready = ready_here(once, [&] {
    int per_sm = 1;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kThreads, kMost);
    return KernelReady{e, std::max(1, sm_count() * per_sm / CL)};
  });
  if (ready.error != cudaSuccess) return ready.error;
  const int64_t tiles = ceil_div(a.site_rows, kSlots * RB) * a.sites;
  const int64_t blocks = std::min<int64_t>(tiles, ready.resident);
  const int smem = D * kSlots * RB * row_room(part_width(a.cols, CL), sizeof(XT), V == 1);
  return launch_rows(kernel, (unsigned)(blocks * CL), kThreads, smem, CL, stream, a);
}

template <typename XT, typename YT>
cudaError_t dispatch(const NormForward& a, cudaStream_t stream) {
  constexpr int V = sizeof(XT) == 2 && sizeof(YT) == 2 ? 8 : 4;
  auto fits = [&](const void* p, int64_t ld, int size) { return (((uintptr_t)p | (uintptr_t)(ld * size)) & (V * size - 1)) == 0; };
  const bool pieces = a.cols % V == 0 && fits(a.x, a.x_ld, sizeof(XT)) && fits(a.y, a.y_ld, sizeof(YT));
  const int n = a.cols;
  // Eight or sixteen columns a thread up to 4096 and two or four rows at a time, so that what a row costs is shared by 32 elements of a
  // thread; rows that start anywhere cost more, and a warp alone takes one of up to 1024 (bf16 rows of 1001: 34.9 us, 44.8 us with 64
  // threads a row and a barrier between them).  A row of 16384 goes to one block with 32 columns a thread (35 us for 134 MB read and 67
  // written): two blocks of 16 columns a thread exchange sums twice a row and took 57 us.
  // least: columns that are too many for the line before; 0 for a cluster's block, whose part of a row is little more than half of its
  // class at the least
#define TAKE(least, v, nv, tpr, rb, d, cl)                                                                             \
  if constexpr ((v) > 1)                                                                                               \
    if (n == (v) * (nv) * (tpr) * (cl)) return launch<XT, YT, v, nv, tpr, rb, d, cl, (v) * (nv) * (tpr)>(a, stream);   \
  if (n <= (v) * (nv) * (tpr) * (cl)) return launch<XT, YT, v, nv, tpr, rb, d, cl, least>(a, stream)
  if (pieces) {
    TAKE(0, V, 1, 32 / V, 4, 3, 1);
    TAKE(33, V, 1, 64 / V, 4, 3, 1);
    TAKE(65, V, 1, 128 / V, 4, 3, 1);
    TAKE(129, V, 8 / V, 32, 4, 3, 1);
    TAKE(257, V, 16 / V, 32, 2, 3, 1);
    TAKE(513, V, 16 / V, 64, 2, 3, 1);
    TAKE(1025, V, 16 / V, 128, 2, 3, 1);
    TAKE(2049, V, 16 / V, 256, 2, 3, 1);
    TAKE(4097, V, 16 / V, 512, 2, 2, 1);
    TAKE(8193, V, 32 / V, 512, 1, 3, 1);
    TAKE(0, V, 32 / V, 512, 1, 3, 2);
    TAKE(0, V, 32 / V, 512, 1, 3, 4);
  } else {
    TAKE(0, 1, 4, 8, 4, 3, 1);
    TAKE(33, 1, 8, 8, 4, 3, 1);
    TAKE(65, 1, 16, 8, 2, 3, 1);
    TAKE(129, 1, 16, 16, 2, 3, 1);
    TAKE(257, 1, 12, 32, 1, 4, 1);
    TAKE(385, 1, 16, 32, 1, 4, 1);
    TAKE(513, 1, 24, 32, 1, 3, 1);
    TAKE(769, 1, 32, 32, 1, 3, 1);
    TAKE(1025, 1, 12, 128, 1, 4, 1);
    TAKE(1537, 1, 16, 128, 1, 4, 1);
    TAKE(2049, 1, 16, 256, 2, 3, 1);
    TAKE(4097, 1, 16, 512, 2, 2, 1);
    TAKE(8193, 1, 32, 512, 1, 3, 1);
    TAKE(0, 1, 32, 512, 1, 3, 2);
    TAKE(0, 1, 32, 512, 1, 3, 4);
  }
#undef TAKE
  return cudaErrorInvalidValue;          // more than kNormWidest columns
}

}  // namespace

cudaError_t norm_forward_rows(const NormForward& a, bool x_bf16, bool y_bf16, cudaStream_t stream) {
  if (a.cols <= kNormNarrow) return norm_forward_narrow(a, x_bf16, y_bf16, stream);
  return x_bf16 ? y_bf16 ? dispatch<bf16, bf16>(a, stream) : dispatch<bf16, float>(a, stream)
                : y_bf16 ? dispatch<float, bf16>(a, stream) : dispatch<float, float>(a, stream);
}
cudaError_t norm_forward_gave_up(cudaStream_t stream, bool* gave_up) { return read_gave_up(stream, gave_up); }

}  // namespace ist
