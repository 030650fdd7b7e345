// kernels_grad.hip -- the backward pass of the masked attention.
//
// With s_ij = scale q_i.k_j on the mask, p_ij = exp(s_ij - lse_i) (the
// probabilities, recomputed from the rows' log-sum-exp) and
//
//     dP_ij = dO_i.v_j,   delta_i = dO_i.O_i = sum_j p_ij dP_ij,
//     dS_ij = p_ij (dP_ij - delta_i),
//
// the gradients are dQ_i = scale sum_j dS_ij k_j, dK_j = scale sum_i dS_ij q_i
// and dV_j = sum_i p_ij dO_i.  Two kernels, each forming S and dP for itself:
// one walks the plan's query rows and sums dQ over their keys, the other walks
// the transposed plan's keys and sums dK and dV over their query rows.  That is
// 14 d flops a non-zero where one kernel would do with 10 d, but every sum has
// one owner: no atomics, no order that changes from run to run, no second pass
// over dQ.  The first kernel leaves each row's lse (times log2 e) and -delta in
// the caller's workspace for the second.
//
// A row with a single key has p = 1 whatever its score is: its dS is set to 0,
// which the difference of two roundings would only come near.
//
// Here: fp32, 32 query rows (or keys) a workgroup, its four wavefronts sharing out
// their units of 32 keys (or query rows; slice_ops.hpp).  kernels_grad_tiles.hip
// has bf16.  Bound by the matrix cores where the chip is full: they are 75 and 79%
// busy in dQ and dK, dV (full mask, L = 2048, d = 64, 16 heads: 250 and 310 us, 103
// and 111 TFLOP/s; a product of 8192^3 reaches 153), and by the longest slice where
// it is not (window 256 + 32 global, L = 2048, 12 heads: 77 and 94 us, 82 and 106 in
// the run of the next pairs).  Two sets of staged rows a wavefront, one loading while
// the other is used, gained nothing (86, 108 us), eight wavefronts a slice lost (95,
// 112 us).
#include <hip/hip_runtime.h>
#include <math.h>

#include "grad_ops.hpp"

namespace splat {
namespace {

constexpr int kThreads = 256;            // 4 wavefronts, one slice
constexpr int kMaxGridY = 32768;         // slices per launch dimension; more are looped over

// o[b][.] += sum over the staged rows of feature NB i + b times weight w.
template <int D>
__device__ __forceinline__ void add_staged(f32x16_t (&o)[D / 32], const char* stage, const Slice& s,
                                           const float (&w)[16]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    typename Mat<float, D>::V v;
    load_staged<float, D>(v, stage, s, j);
    Mat<float, D>::pv(o, v, w, j);
  }
}

// dot product of two rows in registers, over both halves
template <typename Row>
__device__ __forceinline__ float row_dot(const Row& x, const Row& y) {
  constexpr int N = sizeof(x.v) / sizeof(x.v[0]);
  float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e] = fmaf(x.v[t][e], y.v[t][e], d[e]);
  const float v = (d[0] + d[1]) + (d[2] + d[3]);
  return v + lane_xor32(v);
}

// LDS: each wavefront's staged rows of two matrices; then the partial sums.  d =
// 128: 128 KiB, one workgroup a CU.
template <int D>
constexpr int kStageBytes = kUnit * D * 4;
template <int D>
constexpr int kLds = kWavesPerGroup * 2 * kStageBytes<D>;
static_assert(kLds<64> >= kSumBytes<64> && kLds<128> >= kSumBytes<128>, "the sums fit");

// ------------------------------------------------------------------------ dQ
template <int D>
__global__ __launch_bounds__(kThreads, D == 64 ? 2 : 1) void k_grad_q_slices(
    const Group* __restrict__ groups, const int32_t* __restrict__ rows,
    const int32_t* __restrict__ row_ptr, const RowRuns* __restrict__ runs,
    const Tile* __restrict__ tiles, const uint64_t* __restrict__ masks, int L, int n_slices,
    const float* __restrict__ Q, const float* __restrict__ K, const float* __restrict__ V,
    const float* __restrict__ O, const float* __restrict__ dO, const float* __restrict__ lse,
    float scale, float* __restrict__ lse2, float* __restrict__ nd, float* __restrict__ dQ) {
  using M = Mat<float, D>;
  constexpr int NB = D / 32;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const size_t head = (size_t)blockIdx.x * L * D, heads_row = (size_t)blockIdx.x * L;
  const char *const Kh = (const char*)(K + head), *const Vh = (const char*)(V + head);
  const float sl2 = scale_size(scale);
  for (int sl = blockIdx.y; sl < n_slices; sl += gridDim.y) {
    Slice s;
    if (!s.open(sl, groups, rows, masks, L)) continue;
    typename M::Row q, g;
    const unsigned at = (unsigned)s.row * (D * 4u) + 16u * s.h;
    load_row<float, D>(q, (const char*)(Q + head), at);
    load_row<float, D>(g, (const char*)(dO + head), at);
    times_sign(q.v, scale_sign(scale));
    RowStat st;
    {
      typename M::Row o;
      load_row<float, D>(o, (const char*)(O + head), at);
      const bool some = row_ptr[s.row + 1] > row_ptr[s.row];
      st = RowStat{some ? lse[heads_row + s.row] * kLog2e : INFINITY, -row_dot(g, o)};
    }
    if (s.wave == 0 && s.h == 0 && s.row_valid)
      lse2[heads_row + s.row] = st.lse2, nd[heads_row + s.row] = st.nd;
    f32x16_t acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[b][r] = 0.f;

    char* const sk = lds + s.wave * 2 * kStageBytes<D>;
    char* const sv = sk + kStageBytes<D>;
    Units it;
    it.start(tiles + s.tb, s.nt, s.lane, s.wave, s.w);
    Unit u;
    bool more = it.next(u);
    while (more) {
      fetch_k<float, D>((float*)sk, Kh, s, u, L);
      fetch_k<float, D>((float*)sv, Vh, s, u, L);
      const uint32_t bits = s.bits(u) >> (4 * s.h);
      wait_loads();
      f32x16_t sc = dot_staged<float, D>(sk, s, q);
      const f32x16_t dp = dot_staged<float, D>(sv, s, g);
      if (!u.full)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = keep_if_bit(sc[r], bits, 8 * (r >> 2) + (r & 3));
      float w[16];
#pragma unroll
      for (int r = 0; r < 16; ++r)
        w[r] = exp2_hw(fmaf(sc[r], sl2, -st.lse2)) * (dp[r] + st.nd);
      add_staged<D>(acc, sk, s, w);
      more = it.next(u);
    }
    combine_rows<D, true>(
        lds, acc, s, scale, dQ + head, [&](int i) { return row_ptr[i + 1] - row_ptr[i] > 1; },
        [&](int i, int r) {
          const RowStat x{__shfl(st.lse2, r, 64), __shfl(st.nd, r, 64)};
          grad_q_row<float, D>(i, s.lane, runs, row_ptr, L, Q + head, K + head, V + head, dO + head,
                               x, scale, dQ + head);
        });
    __syncthreads();                     // LDS is reused by the next slice
  }
}

// ------------------------------------------------------------------ dK and dV
// The plan's roles exchanged: a slice is 32 keys, a unit 32 query rows, whose
// statistics are staged beside them.
template <int D>
__global__ __launch_bounds__(kThreads, D == 64 ? 2 : 1) void k_grad_kv_slices(
    const Group* __restrict__ groups, const int32_t* __restrict__ keys,
    const Tile* __restrict__ tiles, const uint64_t* __restrict__ masks, int L, int n_slices,
    const float* __restrict__ Q, const float* __restrict__ K, const float* __restrict__ V,
    const float* __restrict__ dO, float scale, const float* __restrict__ lse2,
    const float* __restrict__ nd, float* __restrict__ dK, float* __restrict__ dV) {
  using M = Mat<float, D>;
  constexpr int NB = D / 32;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const size_t head = (size_t)blockIdx.x * L * D, heads_row = (size_t)blockIdx.x * L;
  const char *const Qh = (const char*)(Q + head), *const Gh = (const char*)(dO + head);
  const float sl2 = scale_size(scale);
  for (int sl = blockIdx.y; sl < n_slices; sl += gridDim.y) {
    Slice s;
    if (!s.open(sl, groups, keys, masks, L)) continue;
    typename M::Row k, v;
    const unsigned at = (unsigned)s.row * (D * 4u) + 16u * s.h;
    load_row<float, D>(k, (const char*)(K + head), at);
    load_row<float, D>(v, (const char*)(V + head), at);
    times_sign(k.v, scale_sign(scale));
    f32x16_t ak[NB], av[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) ak[b][r] = av[b][r] = 0.f;

    char* const sq = lds + s.wave * 2 * kStageBytes<D>;
    char* const sg = sq + kStageBytes<D>;
    float* const stat = (float*)(lds + kLds<D> + s.wave * 256);
    const float* const mine = (s.h ? nd : lse2) + heads_row;
    Units it;
    it.start(tiles + s.tb, s.nt, s.lane, s.wave, s.w);
    Unit u;
    bool more = it.next(u);
    while (more) {
      fetch_k<float, D>((float*)sq, Qh, s, u, L);
      fetch_k<float, D>((float*)sg, Gh, s, u, L);
      dma4(mine + s.key(u, s.qi, L), (char*)stat);
      const uint32_t bits = s.bits(u) >> (4 * s.h);
      const uint32_t lone = u.full ? 0u : (uint32_t)tiles[s.tb + u.tile].pad[u.half] >> (4 * s.h);
      wait_loads();
      f32x16_t sc = dot_staged<float, D>(sq, s, k);
      const f32x16_t dp = dot_staged<float, D>(sg, s, v);
      if (!u.full)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = keep_if_bit(sc[r], bits, 8 * (r >> 2) + (r & 3));
      float p[16], w[16];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const f32x4_t l4 = *(const f32x4_t*)(stat + 8 * c + 4 * s.h);
        const f32x4_t n4 = *(const f32x4_t*)(stat + 32 + 8 * c + 4 * s.h);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * c + e;
          p[r] = exp2_hw(fmaf(sc[r], sl2, -l4[e]));
          w[r] = p[r] * (dp[r] + n4[e]);
        }
      }
      if (lone)
#pragma unroll
        for (int r = 0; r < 16; ++r) w[r] = zero_unless(w[r], ~lone, 8 * (r >> 2) + (r & 3));
      add_staged<D>(av, sg, s, p);
      add_staged<D>(ak, sq, s, w);
      more = it.next(u);
    }
    auto all = [](int) { return true; };
    const int first = s.w * kWaveRows;
    combine_rows<D, true>(lds, av, s, 1.f, dV + head, all, [&](int j, int r) {
      grad_kv_row<float, D, false>(j, first + r, s.lane, tiles + s.tb, s.nt, masks, L, Q + head,
                                   K + head, V + head, dO + head, lse2 + heads_row, nd + heads_row,
                                   scale, dV + head);
    });
    combine_rows<D, true>(lds, ak, s, scale, dK + head, all, [&](int j, int r) {
      grad_kv_row<float, D, true>(j, first + r, s.lane, tiles + s.tb, s.nt, masks, L, Q + head,
                                  K + head, V + head, dO + head, lse2 + heads_row, nd + heads_row,
                                  scale, dK + head);
    });
    __syncthreads();                     // LDS is reused by the next slice
  }
}

// ------------------------------------------------------------------ launches
dim3 slice_grid(int groups, int BH) {
  const int n = groups * kWavesPerGroup;
  return dim3(BH, n < kMaxGridY ? n : kMaxGridY);
}

template <int D>
hipError_t slices(const DevAcsr& a, int BH, const BwdArgs& x, float scale, hipStream_t st) {
  using T = float;
  float *const lse2 = x.ws, *const nd = x.ws + (size_t)BH * a.L;
  hipLaunchKernelGGL((k_grad_q_slices<D>), slice_grid(a.n_groups, BH), dim3(kThreads), kLds<D>, st,
                     a.groups, a.rows, a.row_ptr, a.runs, a.tiles, a.masks, a.L,
                     a.n_groups * kWavesPerGroup, (const T*)x.Q, (const T*)x.K, (const T*)x.V,
                     (const T*)x.O, (const T*)x.dO, x.lse, scale, lse2, nd, (T*)x.dQ);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_grad_kv_slices<D>), slice_grid(a.grad_groups, BH), dim3(kThreads),
                     kLds<D> + kWavesPerGroup * 256, st, a.grad_group, a.grad_rows, a.grad_tile,
                     a.grad_masks, a.L, a.grad_groups * kWavesPerGroup, (const T*)x.Q, (const T*)x.K,
                     (const T*)x.V, (const T*)x.dO, scale, lse2, nd, (T*)x.dK, (T*)x.dV);
  return hipGetLastError();
}

template <int D>
hipError_t allow_lds() {
  const hipError_t e = hipFuncSetAttribute((const void*)k_grad_q_slices<D>,
                                           hipFuncAttributeMaxDynamicSharedMemorySize, kLds<D>);
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute((const void*)k_grad_kv_slices<D>,
                             hipFuncAttributeMaxDynamicSharedMemorySize,
                             kLds<D> + kWavesPerGroup * 256);
}

}  // namespace

hipError_t bounds_collect_grad(uint32_t* bits, bool clear) { return dbg::collect(bits, clear); }

hipError_t prepare_bwd() {
  hipError_t e = allow_lds<64>();
  if (e == hipSuccess) e = allow_lds<128>();
  return e == hipSuccess ? prepare_bwd_tiles() : e;
}

hipError_t launch_bwd(const DevAcsr& a, int dtype, int BH, int d, const BwdArgs& x, float scale,
                      hipStream_t st) {
  if (dtype == 0)
    return d == 64 ? slices<64>(a, BH, x, scale, st) : slices<128>(a, BH, x, scale, st);
  const hipError_t e = launch_grad_q_tiles(a, BH, d, x, scale, st);
  return e == hipSuccess ? launch_grad_kv_tiles(a, BH, d, x, scale, st) : e;
}

}  // namespace splat
