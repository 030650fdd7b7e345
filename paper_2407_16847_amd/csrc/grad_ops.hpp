// grad_ops.hpp -- what the backward kernels share: a row's statistics, and the
// gradients of a single row or key by one wavefront.
#pragma once

#include "slice_ops.hpp"

namespace splat {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// scale log2(e) as a positive factor of the scores: its sign, and a zero one, go
// to the operand that stays in registers (exactly), so that scores set to -inf
// stay there.
__device__ __forceinline__ float scale_size(float scale) {
  return scale == 0.f ? 1.f : fabsf(scale) * kLog2e;
}
__device__ __forceinline__ float scale_sign(float scale) {
  return scale == 0.f ? 0.f : copysignf(1.f, scale);
}
template <typename V, int N>
__device__ __forceinline__ void times_sign(V (&x)[N], float sign) {
  constexpr int E = sizeof(V) / sizeof(x[0][0]);
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int e = 0; e < E; ++e)
      x[t][e] = (float)x[t][e] * sign;
}

// x where bit u of `word` is set, 0 elsewhere
__device__ __forceinline__ float zero_unless(float x, unsigned word, int u) {
  const unsigned m = (unsigned)__builtin_amdgcn_sbfe((int)word, u, 1);
  return __builtin_bit_cast(float, __builtin_bit_cast(unsigned, x) & m);
}

// What a row's scores need: log2 of the sum of its exponentials, and -delta.
// Scores that the mask leaves out are set to -inf; with lse2 = +inf for rows
// without keys (their lse is -inf) those too get p = 0 and not a NaN.
struct RowStat {
  float lse2, nd;
};

// -delta from a bf16 O carries O's rounding, an error e that is the same for all
// of a row's dS_ij = p_ij (dP_ij - delta): next to dS it is about 2^-9.3 / sqrt(n)
// for weight spread over n keys (and more where few of them have the weight).  Rows
// of 2 .. kFewKeys keys therefore sum their dS first, over the tiles of their group
// that such rows have keys in (Tile::pad), which with the exact delta is 0, and take
// that from delta.
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
  // adds w of lane t times row j of lane t, for the lanes t in `which`: eight rows'
  // loads in flight at a time (lanes without a row hold row 0)
  __device__ __forceinline__ void add(uint64_t which, int j, float w, const T* X, int lane) {
    if (!which) return;
    const int end = 64 - __builtin_clzll(which);
#pragma unroll 1
    for (int t0 = __builtin_ctzll(which); t0 < end; t0 += 8) {
      float x[8][D / 64];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const T* const r = X + (size_t)__builtin_amdgcn_readlane(j, min(t0 + e, 63)) * D;
#pragma unroll
        for (int b = 0; b < D / 64; ++b) x[e][b] = (float)r[64 * b + lane];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (t0 + e >= 64 || !((which >> (t0 + e)) & 1)) continue;
        const float wt = __builtin_bit_cast(
            float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), t0 + e));
#pragma unroll
        for (int b = 0; b < D / 64; ++b) acc[b] = fmaf(wt, x[e][b], acc[b]);
      }
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
// slice) from what the mask gives it alone.  Block b's output row i is feature
// 32 b + i, or NB i + b if INTERLEAVED (see slice_ops.hpp).
template <int D>
constexpr int kSumStride = D + 4;        // floats of a row of partial sums
template <int D>
constexpr int kSumBytes = kWavesPerGroup * kWaveRows * kSumStride<D> * 4;

template <int D, bool INTERLEAVED, typename T, typename S, typename F, typename G>
__device__ __forceinline__ void combine_rows(char* lds, const f32x16_t (&o)[D / 32], const S& s,
                                             float f, T* out, F&& keep, G&& again) {
  constexpr int NB = D / 32, OS = kSumStride<D>;
  float* const sums = (float*)lds;
  __syncthreads();                       // every wavefront has left its staged rows
  float* const mine = sums + (s.wave * kWaveRows + s.qi) * OS;
#pragma unroll
  for (int g = 0; g < 4; ++g)
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      f32x4_t v;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[e] = INTERLEAVED ? o[(4 * c + e) % NB][4 * g + (4 * c + e) / NB] : o[c][4 * g + e];
      const int r = 8 * g + 4 * s.h;     // the four output rows in a row
      *(f32x4_t*)(mine + (INTERLEAVED ? NB * r + 4 * c : 32 * c + r)) = v;
    }
  __syncthreads();
  const int r = threadIdx.x >> 3;        // row of the slice
  const int row = (int)__shfl(s.valid() ? s.row : -1, r & 31, 64);
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

}  // namespace
}  // namespace splat
