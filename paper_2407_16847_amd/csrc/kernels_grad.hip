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
#include <hip/hip_runtime.h>
#include <math.h>

#include "slice_ops.hpp"

namespace splat {
namespace {

constexpr int kThreads = 256;            // 4 wavefronts, one slice
constexpr int kMaxGridY = 32768;         // slices per launch dimension; more are looped over
constexpr float kLog2e = 1.4426950408889634f;

// ----------------------------------------------------------------- operands
// o[b][.] += sum over the staged rows of feature NB i + b times weight w.  bf16:
// the weights are rounded to nearest even, half a step (2^-8 of each at most)
// as the rounding of the outputs.
template <typename T, int D>
__device__ __forceinline__ void add_staged(f32x16_t (&o)[D / 32], const char* stage, const Slice& s,
                                           const float (&w)[16]) {
  using M = Mat<T, D>;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    typename M::V v;
    load_staged<T, D>(v, stage, s, j);
    if constexpr (std::is_same<T, float>::value) {
      M::pv(o, v, w, j);
    } else {
      bf16x8_t p;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = (__bf16)w[8 * j + e];
#pragma unroll
      for (int b = 0; b < D / 32; ++b) o[b] = mfma32(M::vt(v, b), p, o[b]);
    }
  }
}

// dot product of two rows in registers, over both halves
template <typename Row>
__device__ __forceinline__ float row_dot(const Row& x, const Row& y) {
  constexpr int N = sizeof(x.v) / sizeof(x.v[0]), E = sizeof(x.v[0]) / sizeof(x.v[0][0]);
  float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int e = 0; e < E; ++e) d[e & 3] = fmaf((float)x.v[t][e], (float)y.v[t][e], d[e & 3]);
  const float v = (d[0] + d[1]) + (d[2] + d[3]);
  return v + lane_xor32(v);
}

// x where bit u of `word` is set, 0 elsewhere
__device__ __forceinline__ float zero_unless(float x, unsigned word, int u) {
  const unsigned m = (unsigned)__builtin_amdgcn_sbfe((int)word, u, 1);
  return __builtin_bit_cast(float, __builtin_bit_cast(unsigned, x) & m);
}

// What a row's scores need: log2 of the sum of its exponentials, and -delta.
// A row without keys has neither (its lse is -inf).
struct RowStat {
  float lse2, nd;
};

// ---------------------------------------------------------- one row, VALU
// Sums over the keys (or query rows) of one row by a wavefront, 64 of them at a
// time, a lane each: weight(j) for lanes that have one, then features by lanes.
template <typename T, int D>
struct RowSum {
  float acc[D / 64];
  __device__ __forceinline__ RowSum() {
#pragma unroll
    for (int b = 0; b < D / 64; ++b) acc[b] = 0.f;
  }
  // adds w of lane t times row j of lane t, for the lanes t in `which`
  __device__ __forceinline__ void add(uint64_t which, int j, float w, const T* X, int lane) {
#pragma unroll 1
    for (; which; which &= which - 1) {
      const int t = __builtin_ctzll(which);
      const float wt = __builtin_bit_cast(
          float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), t));
      const T* const x = X + (size_t)__builtin_amdgcn_readlane(j, t) * D;
#pragma unroll
      for (int b = 0; b < D / 64; ++b) acc[b] = fmaf(wt, (float)x[64 * b + lane], acc[b]);
    }
  }
  __device__ __forceinline__ void store(T* out, float f, int lane) {
#pragma unroll
    for (int b = 0; b < D / 64; ++b) store1(out + 64 * b + lane, acc[b] * f);
  }
};

// dQ of row i from its own keys alone (arrays of one head).
template <typename T, int D>
__device__ __attribute__((noinline)) void grad_q_row(int i, int lane, const RowRuns* runs,
                                                     const int32_t* row_ptr, int L, const T* Q,
                                                     const T* K, const T* V, const T* dO,
                                                     RowStat st, float scale, T* dQ) {
  const RowRuns rr = runs[i];
  const int n = row_ptr[i + 1] - row_ptr[i];
  const T *const q = Q + (size_t)i * D, *const g = dO + (size_t)i * D;
  RowSum<T, D> sum;
  for (int k0 = 0; n > 1 && k0 < n; k0 += 64) {
    const bool valid = k0 + lane < n;
    int j = 0;
    float w = 0.f;
    if (valid) {
      j = dbg::idx(col_of(rr, k0 + lane), L, dbg::kKey);
      const float p = exp2_hw(fmaf(dense_dot<T, D>(q, K + (size_t)j * D), scale * kLog2e, -st.lse2));
      w = p * (dense_dot<T, D>(g, V + (size_t)j * D) + st.nd);
    }
    sum.add(__ballot(valid), j, w, K, lane);
  }
  sum.store(dQ + (size_t)i * D, scale, lane);
}

// dK (KEYS) or dV of key j, the key `place` of its group, from the query rows
// that have it alone.
template <typename T, int D, bool KEYS>
__device__ __attribute__((noinline)) void grad_kv_row(int j, int place, int lane, const Tile* tiles,
                                                      int nt, const uint64_t* masks, int L,
                                                      const T* Q, const T* K, const T* V,
                                                      const T* dO, const float* lse2,
                                                      const float* nd, float scale, T* out) {
  RowSum<T, D> sum;
  for (int t = 0; t < nt; ++t) {
    const Tile tl = tiles[t];
    const int state = (tl.flags >> (kWaveShift + 2 * (place / kWaveRows))) & 3;
    if (state == kWaveEmpty) continue;
    uint64_t bits = state == kWaveFull ? ~0ull : masks[(size_t)tl.mask_block * kBM + place];
    if (KEYS) bits &= ~((uint64_t)(uint32_t)tl.pad[0] | (uint64_t)(uint32_t)tl.pad[1] << 32);
    const bool valid = (bits >> lane) & 1;
    int i = 0;
    float w = 0.f;
    if (valid) {
      i = dbg::idx(tl.kb + tl.ks * lane, L, dbg::kRow);
      w = exp2_hw(fmaf(dense_dot<T, D>(Q + (size_t)i * D, K + (size_t)j * D), scale * kLog2e,
                       -lse2[i]));
      if (KEYS) w *= dense_dot<T, D>(dO + (size_t)i * D, V + (size_t)j * D) + nd[i];
    }
    sum.add(bits, i, w, KEYS ? Q : dO, lane);
  }
  sum.store(out + (size_t)j * D, KEYS ? scale : 1.f, lane);
}

// ----------------------------------------------------------------- combining
// The wavefronts' partial sums, times f, written as whole rows: every thread
// sums features of one row, eight lanes along a row.  keep(row): whether the
// sums are the row's result, else it is 0.  The matrix cores multiply every
// staged row by every lane's weight, 0 where the mask has none, and 0 * inf is
// NaN: a row whose result is not finite is formed again(row, its place in the
// slice) from what the mask gives it alone.
template <int D>
constexpr int kSumStride = D + 4;        // floats of a row of partial sums
template <int D>
constexpr int kSumBytes = kWavesPerGroup * kWaveRows * kSumStride<D> * 4;

template <int D, typename T, typename F, typename G>
__device__ __forceinline__ void combine_rows(char* lds, const f32x16_t (&o)[D / 32], const Slice& s,
                                             float f, T* out, F&& keep, G&& again) {
  constexpr int NB = D / 32, OS = kSumStride<D>;
  float* const sums = (float*)lds;
  __syncthreads();                       // every wavefront has left its staged rows
  float* const mine = sums + (s.wave * kWaveRows + s.qi) * OS;
#pragma unroll
  for (int g = 0; g < 4; ++g)
#pragma unroll
    for (int c = 0; c < NB; ++c) {       // features NB (8 g + 4 h) + 4 c .. + 3
      f32x4_t v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = o[(4 * c + e) % NB][4 * g + (4 * c + e) / NB];
      *(f32x4_t*)(mine + NB * (8 * g + 4 * s.h) + 4 * c) = v;
    }
  __syncthreads();
  const int r = threadIdx.x >> 3;        // row of the slice
  const int row = (int)__shfl(s.row_valid ? s.row : -1, r & 31, 64);
  f32x4_t v[NB];
  float z = 0.f;
  bool is = false;
  if (row >= 0) {
    is = keep(row);
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int c = 4 * (threadIdx.x & 7) + 32 * k;
      v[k] = *(const f32x4_t*)(sums + r * OS + c);
#pragma unroll
      for (int w = 1; w < kWavesPerGroup; ++w)
        v[k] += *(const f32x4_t*)(sums + (w * kWaveRows + r) * OS + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[k][e] = is ? v[k][e] * f : 0.f;
        z = fmaf(v[k][e], 0.f, z);
      }
    }
  }
  const uint64_t bad = __ballot(z != z);
  if (row >= 0 && ((bad >> (s.lane & 56)) & 0xffu) == 0) {
#pragma unroll
    for (int k = 0; k < NB; ++k)
      store4<T>(out + (size_t)row * D + 4 * (threadIdx.x & 7) + 32 * k, v[k][0], v[k][1], v[k][2],
                v[k][3]);
  }
  if (bad != 0)
    for (int k = 0; k < 64; k += 8)
      if ((bad >> k) & 0xffu)
        again(__builtin_amdgcn_readlane(row, k), __builtin_amdgcn_readlane(r, k));
}

// The statistics of this lane's row, from its dO (in registers) and O.
template <typename T, int D>
__device__ __forceinline__ RowStat row_stat(const Slice& s, const typename Mat<T, D>::Row& g,
                                            const T* O, const float* lse) {
  typename Mat<T, D>::Row o;
  load_row<T, D>(o, (const char*)O, (unsigned)s.row * (D * (unsigned)sizeof(T)) + 16u * s.h);
  return RowStat{lse[s.row] * kLog2e, -row_dot(g, o)};
}

// ------------------------------------------------------------------------ dQ
// LDS: each wavefront's staged K and V rows; then the partial sums.
template <typename T, int D>
constexpr int kStageBytes = kUnit * D * (int)sizeof(T);
template <typename T, int D>
constexpr int kPairBytes = kWavesPerGroup * 2 * kStageBytes<T, D>;
template <typename T, int D>
constexpr int kSliceLds = kPairBytes<T, D> > kSumBytes<D> ? kPairBytes<T, D> : kSumBytes<D>;

template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 && D == 128 ? 1 : 2) void k_grad_q_slices(
    const Group* __restrict__ groups, const int32_t* __restrict__ rows,
    const int32_t* __restrict__ row_ptr, const RowRuns* __restrict__ runs,
    const Tile* __restrict__ tiles, const uint64_t* __restrict__ masks, int L, int n_slices,
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V,
    const T* __restrict__ O, const T* __restrict__ dO, const float* __restrict__ lse, float scale,
    float* __restrict__ lse2, float* __restrict__ nd, T* __restrict__ dQ) {
  using M = Mat<T, D>;
  constexpr int NB = D / 32;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const size_t head = (size_t)blockIdx.x * L * D, heads_row = (size_t)blockIdx.x * L;
  const char *const Kh = (const char*)(K + head), *const Vh = (const char*)(V + head);
  const float sl2 = scale * kLog2e;
  for (int sl = blockIdx.y; sl < n_slices; sl += gridDim.y) {
    Slice s;
    if (!s.open(sl, groups, rows, masks, L)) continue;
    typename M::Row q, g;
    const unsigned at = (unsigned)s.row * (D * (unsigned)sizeof(T)) + 16u * s.h;
    load_row<T, D>(q, (const char*)(Q + head), at);
    load_row<T, D>(g, (const char*)(dO + head), at);
    const RowStat st = row_stat<T, D>(s, g, O + head, lse + heads_row);
    if (s.wave == 0 && s.h == 0 && s.row_valid)
      lse2[heads_row + s.row] = st.lse2, nd[heads_row + s.row] = st.nd;
    f32x16_t acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[b][r] = 0.f;

    char* const sk = lds + s.wave * 2 * kStageBytes<T, D>;
    char* const sv = sk + kStageBytes<T, D>;
    Units it;
    it.start(tiles + s.tb, s.nt, s.lane, s.wave, s.w);
    Unit u;
    bool more = it.next(u);
    while (more) {
      fetch_k<T, D>((float*)sk, Kh, s, u, L);
      fetch_k<T, D>((float*)sv, Vh, s, u, L);
      const uint32_t bits = s.bits(u) >> (4 * s.h);
      wait_loads();
      const f32x16_t sc = dot_staged<T, D>(sk, s, q);
      const f32x16_t dp = dot_staged<T, D>(sv, s, g);
      float w[16];
#pragma unroll
      for (int r = 0; r < 16; ++r)
        w[r] = exp2_hw(fmaf(sc[r], sl2, -st.lse2)) * (dp[r] + st.nd);
      if (!u.full)
#pragma unroll
        for (int r = 0; r < 16; ++r) w[r] = zero_unless(w[r], bits, 8 * (r >> 2) + (r & 3));
      add_staged<T, D>(acc, sk, s, w);
      more = it.next(u);
    }
    combine_rows<D, T>(
        lds, acc, s, scale, dQ + head,
        [&](int i) { return row_ptr[i + 1] - row_ptr[i] > 1; },
        [&](int i, int r) {
          const RowStat x{__shfl(st.lse2, r, 64), __shfl(st.nd, r, 64)};
          grad_q_row<T, D>(i, s.lane, runs, row_ptr, L, Q + head, K + head, V + head, dO + head, x,
                           scale, dQ + head);
        });
    __syncthreads();                     // LDS is reused by the next slice
  }
}

// ------------------------------------------------------------------ dK and dV
// The plan's roles exchanged: a slice is 32 keys, a unit 32 query rows.
template <typename T, int D>
constexpr int kKvLds = kSliceLds<T, D> + kWavesPerGroup * 64 * 4;

template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 && D == 128 ? 1 : 2) void k_grad_kv_slices(
    const Group* __restrict__ groups, const int32_t* __restrict__ keys,
    const Tile* __restrict__ tiles, const uint64_t* __restrict__ masks, int L, int n_slices,
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V,
    const T* __restrict__ dO, float scale, const float* __restrict__ lse2,
    const float* __restrict__ nd, T* __restrict__ dK, T* __restrict__ dV) {
  using M = Mat<T, D>;
  constexpr int NB = D / 32;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const size_t head = (size_t)blockIdx.x * L * D, heads_row = (size_t)blockIdx.x * L;
  const char *const Qh = (const char*)(Q + head), *const Gh = (const char*)(dO + head);
  const float sl2 = scale * kLog2e;
  for (int sl = blockIdx.y; sl < n_slices; sl += gridDim.y) {
    Slice s;
    if (!s.open(sl, groups, keys, masks, L)) continue;
    typename M::Row k, v;
    const unsigned at = (unsigned)s.row * (D * (unsigned)sizeof(T)) + 16u * s.h;
    load_row<T, D>(k, (const char*)(K + head), at);
    load_row<T, D>(v, (const char*)(V + head), at);
    f32x16_t ak[NB], av[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) ak[b][r] = av[b][r] = 0.f;

    char* const sq = lds + s.wave * 2 * kStageBytes<T, D>;
    char* const sg = sq + kStageBytes<T, D>;
    float* const stat = (float*)(lds + kSliceLds<T, D>) + 64 * s.wave;
    const float* const mine = (s.h ? nd : lse2) + heads_row;
    Units it;
    it.start(tiles + s.tb, s.nt, s.lane, s.wave, s.w);
    Unit u;
    bool more = it.next(u);
    while (more) {
      fetch_k<T, D>((float*)sq, Qh, s, u, L);
      fetch_k<T, D>((float*)sg, Gh, s, u, L);
      stat[s.lane] = mine[s.key(u, s.qi, L)];
      const uint32_t bits = s.bits(u) >> (4 * s.h);
      const uint32_t lone = u.full ? 0u : (uint32_t)tiles[s.tb + u.tile].pad[u.half] >> (4 * s.h);
      wait_loads();
      const f32x16_t sc = dot_staged<T, D>(sq, s, k);
      const f32x16_t dp = dot_staged<T, D>(sg, s, v);
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
      if (!u.full)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          p[r] = zero_unless(p[r], bits, 8 * (r >> 2) + (r & 3));
          w[r] = zero_unless(w[r], bits & ~lone, 8 * (r >> 2) + (r & 3));
        }
      add_staged<T, D>(av, sg, s, p);
      add_staged<T, D>(ak, sq, s, w);
      more = it.next(u);
    }
    auto all = [](int) { return true; };
    const int first = s.w * kWaveRows;
    combine_rows<D, T>(lds, av, s, 1.f, dV + head, all, [&](int j, int r) {
      grad_kv_row<T, D, false>(j, first + r, s.lane, tiles + s.tb, s.nt, masks, L, Q + head,
                               K + head, V + head, dO + head, lse2 + heads_row, nd + heads_row,
                               scale, dV + head);
    });
    combine_rows<D, T>(lds, ak, s, scale, dK + head, all, [&](int j, int r) {
      grad_kv_row<T, D, true>(j, first + r, s.lane, tiles + s.tb, s.nt, masks, L, Q + head,
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

template <typename T, int D>
hipError_t bwd(const DevAcsr& a, int BH, const BwdArgs& x, float scale, hipStream_t st) {
  const T *Q = (const T*)x.Q, *K = (const T*)x.K, *V = (const T*)x.V, *O = (const T*)x.O,
          *dO = (const T*)x.dO;
  float *const lse2 = x.ws, *const nd = x.ws + (size_t)BH * a.L;
  hipLaunchKernelGGL((k_grad_q_slices<T, D>), slice_grid(a.n_groups, BH), dim3(kThreads),
                     (kSliceLds<T, D>), st, a.groups, a.rows, a.row_ptr, a.runs, a.tiles, a.masks,
                     a.L, a.n_groups * kWavesPerGroup, Q, K, V, O, dO, x.lse, scale, lse2, nd,
                     (T*)x.dQ);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_grad_kv_slices<T, D>), slice_grid(a.grad_groups, BH), dim3(kThreads),
                     (kKvLds<T, D>), st, a.grad_group, a.grad_rows, a.grad_tile, a.grad_masks, a.L,
                     a.grad_groups * kWavesPerGroup, Q, K, V, dO, scale, lse2, nd, (T*)x.dK,
                     (T*)x.dV);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t allow_lds() {
  hipError_t e = hipFuncSetAttribute((const void*)k_grad_q_slices<T, D>,
                                     hipFuncAttributeMaxDynamicSharedMemorySize, kSliceLds<T, D>);
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute((const void*)k_grad_kv_slices<T, D>,
                             hipFuncAttributeMaxDynamicSharedMemorySize, kKvLds<T, D>);
}

}  // namespace

hipError_t bounds_collect_grad(uint32_t* bits, bool clear) { return dbg::collect(bits, clear); }

hipError_t prepare_bwd() {
  hipError_t e = allow_lds<float, 64>();
  if (e == hipSuccess) e = allow_lds<float, 128>();
  if (e == hipSuccess) e = allow_lds<__bf16, 64>();
  if (e == hipSuccess) e = allow_lds<__bf16, 128>();
  return e;
}

hipError_t launch_bwd(const DevAcsr& a, int dtype, int BH, int d, const BwdArgs& x, float scale,
                      hipStream_t st) {
  if (dtype == 0)
    return d == 64 ? bwd<float, 64>(a, BH, x, scale, st) : bwd<float, 128>(a, BH, x, scale, st);
  return d == 64 ? bwd<__bf16, 64>(a, BH, x, scale, st) : bwd<__bf16, 128>(a, BH, x, scale, st);
}

}  // namespace splat
