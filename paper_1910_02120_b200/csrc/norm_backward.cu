// Layer norm's way back for rows that fit the threads of a block or a cluster: dy and x are read once, dx written, and
// the sums over rows that dweight and dbias need are kept in registers, a column always with the same thread.
#include <algorithm>

#include "norm_rows.cuh"

namespace ist {
namespace {

// 51,200 rows of 1024, x bf16 and dy fp32: 72 us with the join, 0.89 of the copy rate; 4096 bf16 rows of 16384: 84 us, 0.74 (one
// block an SM and one tile on its way at a time: neither memory nor the issue slots, 54 % of them used, run through); 9600 rows of 1001, which start anywhere: 28 us, against 21 us for 1000 columns.
//
// A tile is gone through twice: first for its sums, then, after the next tile's sums have been begun, for dx.  So the
// shuffles and the barrier of one tile's sums run beside the arithmetic of another, at the price of unpacking the rows twice
// (shared memory is not what bounds this) and of two tiles' rows kept.
template <typename XT, typename DT, int V, int NV, int TPR, int RB, int D, int CL, int LEAST>
__global__ void __launch_bounds__(NV * V == 16 ? 512 : kNormThreads) norm_backward_kernel(const NormBackward a) {
  constexpr int kThreads = NV * V == 16 ? 512 : kNormThreads, kSlots = kThreads / TPR, kTile = kSlots * RB;
  constexpr int C = NV * V, P = C / 2;
  constexpr bool FULL = LEAST == TPR * C;                  // of a block's columns: no piece is missing
  static_assert(D >= 3, "two tiles are in use while others arrive");
  extern __shared__ __align__(128) char ring[];
  __shared__ RowSums<kThreads, CL, 2 * RB> sh;
  const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
  // columns of this block: the row's, or the part of them that is this block's in its cluster
  const int width = FULL ? TPR * C : part_width(a.cols, CL);
  const int c0 = CL > 1 ? (int)cluster_ctarank() * width : 0, cols = CL > 1 ? max(min(a.cols - c0, width), 0) : a.cols;
  const int x_room = row_room(width, sizeof(XT), V == 1), room = x_room + row_room(width, sizeof(DT), V == 1);
  const int64_t block = blockIdx.x / CL;
  const int site = (int)(block % a.sites), part = (int)(block / a.sites);
  // this block's rows of its site
  const int row0 = (int)(site * a.site_rows), begin = row0 + (int)(a.site_rows * part / a.parts);
  const int end = row0 + (int)(a.site_rows * (part + 1) / a.parts);
  const XT* const x = (const XT*)a.x + c0;
  const DT* const dy = (const DT*)a.dy + c0;
  const float inv = 1.f / (float)a.cols;
  int r = begin + slot * RB, in_r = r, stage = 0, in_stage = 0;

  auto buffer = [&](int stage, int j) { return ring + ((stage * kSlots + slot) * RB + j) * room; };
  auto x_at = [&](int stage, int j, int r) {
    return buffer(stage, j) + (V == 1 ? (int)((uintptr_t)(x + (int64_t)(r + j) * a.x_ld) & 15) : 0) + t * (V * (int)sizeof(XT));
  };
  auto d_at = [&](int stage, int j, int r) {
    return buffer(stage, j) + x_room + (V == 1 ? (int)((uintptr_t)(dy + (int64_t)(r + j) * a.dy_ld) & 15) : 0) + t * (V * (int)sizeof(DT));
  };
  auto fetch = [&]() {
#pragma unroll
    for (int j = 0; j < RB; ++j)
      if (in_r + j < end) {
        fetch_row<XT, V, NV, TPR, LEAST>(x + (int64_t)(in_r + j) * a.x_ld, cols, buffer(in_stage, j), t);
        fetch_row<DT, V, NV, TPR, LEAST>(dy + (int64_t)(in_r + j) * a.dy_ld, cols, buffer(in_stage, j) + x_room, t);
      }
    in_r += kTile;
    if (++in_stage == D) in_stage = 0;
    copy_commit();
  };
  // what of the next tile is carried in registers: the rows' statistics, and elements that no copy takes
  float next_mean[RB], next_rstd[RB];
  uint16_t odd_x[RB], odd_d[RB];
  auto fetch_more = [&](int r) {
#pragma unroll
    for (int j = 0; j < RB; ++j) {
      const bool live = r + j < end;
      next_mean[j] = live ? a.mean[r + j] : 0.f;
      next_rstd[j] = live ? a.rstd[r + j] : 0.f;
      if (V == 1) {
        odd_x[j] = live ? load_odd(x + (int64_t)(r + j) * a.x_ld, cols, t) : (uint16_t)0;
        odd_d[j] = live ? load_odd(dy + (int64_t)(r + j) * a.dy_ld, cols, t) : (uint16_t)0;
      }
    }
  };
  auto here = [&](int i) { return (i + 1) * TPR * V <= LEAST || (t + i * TPR) * V < cols; };
  // kPairs pairs of elements from piece i on: a piece, or two single elements
  constexpr int kPairs = V == 1 ? 1 : V / 2, kStep = V == 1 ? 2 : 1;
  auto take = [&](const char* bx, const char* bd, int i, float* xv, float* dv) {
#pragma unroll
    for (int u = 0; u < kStep; ++u) {
      if (here(i + u)) {
        unpack<XT, V>(bx + (i + u) * (TPR * V * sizeof(XT)), xv + u * V);
        unpack<DT, V>(bd + (i + u) * (TPR * V * sizeof(DT)), dv + u * V);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) xv[u * V + e] = dv[u * V + e] = 0.f;     // dy = 0 leaves all sums as they are
      }
    }
  };

  Turn turn = begin_sums<CL>(sh, a.wait_limit);
  pdl_wait();
  pdl_trigger();
#pragma unroll
  for (int k = 0; k < D - 2; ++k) fetch();
  fetch_more(r);
  pair w[P], aw[P], ab[P];
  {
    const float* const ws = a.weight ? a.weight + (int64_t)site * a.cols + c0 : nullptr;
    const bool wide = ((uintptr_t)ws & 15) == 0;
    float f[C];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int e = 0; e < V; ++e) f[i * V + e] = 1.f;
      if (ws && here(i)) load_vector<V>(ws + (t + i * TPR) * V, wide, f + i * V);
    }
#pragma unroll
    for (int e = 0; e < P; ++e) {
      w[e] = make_pair2(f[2 * e], f[2 * e + 1]);
      aw[e] = ab[e] = both(0.f);
    }
  }
  const int tiles = (int)ceil_div(end - begin, kTile);
  float s[2 * RB], mean[RB], rstd[RB];          // of the tile whose dx is next
  for (int k = 0; k <= tiles; ++k) {
    float n[2 * RB], n_mean[RB], n_rstd[RB];    // of the tile whose sums are next
    if (k < tiles) {
      fetch();
      copy_wait<D - 2>();
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        n_mean[j] = next_mean[j];
        n_rstd[j] = next_rstd[j];
        if (V == 1 && r + j < end) {
          store_odd(x + (int64_t)(r + j) * a.x_ld, cols, buffer(stage, j), t, odd_x[j]);
          store_odd(dy + (int64_t)(r + j) * a.dy_ld, cols, buffer(stage, j) + x_room, t, odd_d[j]);
        }
      }
      if (V == 1) row_barrier<TPR>();
      fetch_more(r + kTile);
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        n[j] = n[RB + j] = 0.f;
        if (r + j >= end) continue;
        const char *const bx = x_at(stage, j, r), *const bd = d_at(stage, j, r);
        pair s0 = both(0.f), s1 = both(0.f);
        const pair rs = both(n_rstd[j]), minus = both(-n_mean[j]);
#pragma unroll
        for (int i = 0; i < NV; i += kStep) {
          float xv[2 * kPairs], dv[2 * kPairs];
          take(bx, bd, i, xv, dv);
#pragma unroll
          for (int e = 0; e < kPairs; ++e) {
            const int q = i * V / 2 + e;
            const pair d = make_pair2(dv[2 * e], dv[2 * e + 1]);
            const pair h = mul(add(make_pair2(xv[2 * e], xv[2 * e + 1]), minus), rs);
            const pair g = mul(d, w[q]);
            aw[q] = fma(d, h, aw[q]);
            ab[q] = add(ab[q], d);
            s0 = add(s0, g);
            s1 = fma(g, h, s1);
          }
        }
        n[j] = first_of(s0) + second_of(s0);
        n[RB + j] = first_of(s1) + second_of(s1);
      }
      if (a.dx) begin_row_sums<TPR, CL, 2 * RB>(n, sh, turn);
    }
    if (k > 0 && a.dx) {
      const int old = stage ? stage - 1 : D - 1, o_r = r - kTile;
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        if (o_r + j < end) {
          const char *const bx = x_at(old, j, o_r), *const bd = d_at(old, j, o_r);
          const pair m0 = both(-s[j] * inv), m1 = both(-s[RB + j] * inv), rs = both(rstd[j]), minus = both(-mean[j]);
          XT* const to = (XT*)a.dx + c0 + (int64_t)(o_r + j) * a.dx_ld + t * V;
#pragma unroll
          for (int i = 0; i < NV; i += kStep) {
            float xv[2 * kPairs], dv[2 * kPairs];
            take(bx, bd, i, xv, dv);
#pragma unroll
            for (int e = 0; e < kPairs; ++e) {
              const int q = i * V / 2 + e;
              const pair h = mul(add(make_pair2(xv[2 * e], xv[2 * e + 1]), minus), rs);
              const pair d = make_pair2(dv[2 * e], dv[2 * e + 1]);
              // rows of one or two elements have next to nothing left after the subtractions: there (V = 1) every product is
              // rounded as it was for the sums, so that what cancels does
              const pair o = V == 1 ? mul(add_rounded(add_rounded(mul(d, w[q]), m0), mul(h, m1)), rs)
                                    : mul(fma(h, m1, fma(d, w[q], m0)), rs);
              xv[2 * e] = first_of(o);
              xv[2 * e + 1] = second_of(o);
            }
#pragma unroll
            for (int u = 0; u < kStep; ++u)
              if (here(i + u)) pack<XT, V>(to + (i + u) * (TPR * V), xv + u * V);
          }
        }
      }
    }
    if (V == 1) row_barrier<TPR>();                         // the next fetch writes what the older tile was read from
    if (k < tiles) {
      if (a.dx) end_row_sums<TPR, CL, 2 * RB>(n, sh, &turn, a.wait_limit);
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        s[j] = n[j];
        s[RB + j] = n[RB + j];
        mean[j] = n_mean[j];
        rstd[j] = n_rstd[j];
      }
      if (++stage == D) stage = 0;
      r += kTile;
    }
  }
  copy_wait<0>();
  finish_sums<CL>(turn);
  if (!a.wsum && !a.bsum) return;
  const int64_t at = ((int64_t)part * a.sites + site) * a.sum_ld + c0;
  // the slots' sums are joined in shared memory, slot after slot
  if (kSlots > 1) {
    __syncthreads();
    float* const f = reinterpret_cast<float*>(ring);        // [slot][2][C][TPR]
#pragma unroll
    for (int e = 0; e < C; ++e) {
      f[((slot * 2 + 0) * C + e) * TPR + t] = e % 2 ? second_of(aw[e / 2]) : first_of(aw[e / 2]);
      f[((slot * 2 + 1) * C + e) * TPR + t] = e % 2 ? second_of(ab[e / 2]) : first_of(ab[e / 2]);
    }
    __syncthreads();
    for (int q = threadIdx.x; q < 2 * C * TPR; q += kThreads) {
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < kSlots; ++u) sum += f[u * 2 * C * TPR + q];
      const int which = q / (C * TPR), e = q % (C * TPR) / TPR, tt = q % TPR;
      const int c = (tt + e / V * TPR) * V + e % V;
      float* const out = which ? a.bsum : a.wsum;
      if (out && c < cols) out[at + c] = sum;
    }
  } else {
#pragma unroll
    for (int e = 0; e < C; ++e) {
      const int c = (t + e / V * TPR) * V + e % V;
      if (c < cols) {
        if (a.wsum) a.wsum[at + c] = e % 2 ? second_of(aw[e / 2]) : first_of(aw[e / 2]);
        if (a.bsum) a.bsum[at + c] = e % 2 ? second_of(ab[e / 2]) : first_of(ab[e / 2]);
      }
    }
  }
}

template <typename XT, typename DT, int V, int NV, int TPR, int RB, int D, int CL, int LEAST>
cudaError_t launch(const NormBackward& a, cudaStream_t stream) {
  constexpr int kThreads = NV * V == 16 ? 512 : kNormThreads, kSlots = kThreads / TPR;
  const auto kernel = norm_backward_kernel<XT, DT, V, NV, TPR, RB, D, CL, LEAST>;
  auto ring = [](int cols) { return D * kSlots * RB * (row_room(cols, sizeof(XT), V == 1) + row_room(cols, sizeof(DT), V == 1)); };
  constexpr int kJoin = kSlots > 1 ? kSlots * 2 * NV * V * TPR * 4 : 0;
  constexpr int kMost = std::max(kJoin, D * kSlots * RB * (row_room(TPR * V * NV, sizeof(XT), V == 1) + row_room(TPR * V * NV, sizeof(DT), V == 1)));
  static_assert(kMost <= 225 * 1024, "ring too large");
  static OncePerDevice<KernelReady> once;
  const KernelReady ready = ready_here(once, [&] {
    return KernelReady{cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost), 0};
  });
  if (ready.error != cudaSuccess) return ready.error;
  return launch_rows(kernel, (unsigned)((int64_t)a.sites * a.parts * CL), kThreads, std::max(ring(part_width(a.cols, CL)), kJoin), CL, stream, a);
}

template <typename XT, typename DT>
cudaError_t dispatch(const NormBackward& a, cudaStream_t stream) {
  constexpr int V = sizeof(XT) == 2 && sizeof(DT) == 2 ? 8 : 4;
  auto fits = [&](const void* p, int64_t ld, int size) { return (((uintptr_t)p | (uintptr_t)(ld * size)) & (V * size - 1)) == 0; };
  const bool pieces = a.cols % V == 0 && fits(a.x, a.x_ld, sizeof(XT)) && fits(a.dy, a.dy_ld, sizeof(DT)) &&
                      (!a.dx || fits(a.dx, a.dx_ld, sizeof(XT)));
  const int n = a.cols;
  // least: columns that are too many for the line before; 0 for a cluster's block, whose part of a row is little more than half of its
  // class at the least
#define TAKE(least, v, nv, tpr, rb, d, cl)                                                                             \
  if constexpr ((v) > 1)                                                                                               \
    if (n == (v) * (nv) * (tpr) * (cl)) return launch<XT, DT, v, nv, tpr, rb, d, cl, (v) * (nv) * (tpr)>(a, stream);   \
  if (n <= (v) * (nv) * (tpr) * (cl)) return launch<XT, DT, v, nv, tpr, rb, d, cl, least>(a, stream)
  // Sixteen columns a thread from 257 on, on 512 threads an SM: one block of 512 leaves half the parts' sums that two of 256 leave
  // (rows of 4096, bf16: 47.6 us and 40.6 us).  Two rows at a time where a stage of both types is small (36.9 us against 41 us for
  // bf16 rows of 1024), four rows up to 256 columns.
  // two tiles in use and one or two on their way, in the shared memory of two blocks (or one of 512 threads)
  constexpr int S = sizeof(XT) + sizeof(DT), D = S == 6 ? 4 : 3, R = S == 4 ? 2 : 1;
  if (pieces) {
    TAKE(0, V, 1, 32 / V, 4, 3, 1);
    TAKE(33, V, 1, 64 / V, 4, 3, 1);
    TAKE(65, V, 1, 128 / V, 4, 3, 1);
    TAKE(129, V, 8 / V, 32, 4, 3, 1);
    TAKE(257, V, 16 / V, 32, R, D, 1);
    TAKE(513, V, 16 / V, 64, R, D, 1);
    TAKE(1025, V, 16 / V, 128, R, D, 1);
    TAKE(2049, V, 16 / V, 256, R, D, 1);
    TAKE(4097, V, 16 / V, 512, R, D, 1);
    TAKE(0, V, 16 / V, 512, R, D, 2);
    TAKE(0, V, 16 / V, 512, R, D, 4);
    TAKE(0, V, 16 / V, 512, R, D, 8);
  } else {
    TAKE(0, 1, 4, 8, 4, 3, 1);
    TAKE(33, 1, 8, 8, 2, 3, 1);
    TAKE(65, 1, S == 4 ? 16 : 8, S == 4 ? 8 : 16, S == 4 ? 1 : 2, 3, 1);
    TAKE(129, 1, S == 4 ? 16 : 8, S == 4 ? 16 : 32, S == 4 ? 1 : 2, 3, 1);
    TAKE(257, 1, 16, 32, R, D, 1);
    TAKE(513, 1, 16, 64, R, D, 1);
    TAKE(1025, 1, 16, 128, R, D, 1);
    TAKE(2049, 1, 16, 256, R, D, 1);
    TAKE(4097, 1, 16, 512, R, D, 1);
    TAKE(0, 1, 16, 512, R, D, 2);
    TAKE(0, 1, 16, 512, R, D, 4);
    TAKE(0, 1, 16, 512, R, D, 8);
  }
#undef TAKE
  return cudaErrorInvalidValue;          // more than kNormWidest columns
}

}  // namespace

cudaError_t norm_backward_rows(const NormBackward& a, bool x_bf16, bool dy_bf16, cudaStream_t stream) {
  if (a.cols <= kNormNarrow) return norm_backward_narrow(a, x_bf16, dy_bf16, stream);
  return x_bf16 ? dy_bf16 ? dispatch<bf16, bf16>(a, stream) : dispatch<bf16, float>(a, stream)
                : dy_bf16 ? dispatch<float, bf16>(a, stream) : dispatch<float, float>(a, stream);
}
cudaError_t norm_backward_gave_up(cudaStream_t stream, bool* gave_up) { return read_gave_up(stream, gave_up); }

}  // namespace ist
