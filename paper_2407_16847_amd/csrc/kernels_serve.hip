// kernels_serve.hip -- rotary positions, the paged cache, and the attention of
// single query tokens over it.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "../../include/splat.h"
#include "serve_core.hpp"
#include "slice_ops.hpp"

namespace splat {
namespace {

constexpr int kThreads = 256;

// ------------------------------------------------- rotation and cache writing
// A thread owns one unit of a token: two 16-byte chunks that hold E pairs, or
// 2 E features past the rotated ones.  It reads their cosines and sines once and
// turns the unit of up to kMaxHeads heads, two heads' loads in flight at a time.
// Bound by memory: every element is read once and written once, whole 32-byte
// sectors, a token's units side by side.  The stores bypass the caches' usual order
// (nothing is read back here).  Rotation of Q and K, 4096 tokens, 16 + 16 heads of d =
// 64 in bf16, 4 sequences: 26.8 us, 5.05 TB/s, what a copy of 1 GiB reaches;
// ordinary stores 29.9, with nontemporal loads besides 33.1.  1000 tokens into the
// cache, d = 128, 8 sequences: 34.0 .. 35.7 us, 4.4 .. 4.6 TB/s; ordinary stores
// 39.6; four heads in flight and at most 8 a thread 34.7 .. 36.6.
constexpr int kInFlight = 2;
constexpr int kMaxHeads = 16;
constexpr int64_t kMaxRuns = 65000;

template <typename T>
struct Chunk;
template <>
struct Chunk<float> {
  static constexpr int E = 4;
  typedef f32x4_t vec_t;
};
template <>
struct Chunk<__bf16> {
  static constexpr int E = 8;
  typedef bf16x8_t vec_t;
};

// Several axes (AXES): each pair's angle stands in its axis's row of the table, 8 bytes at
// a time from the caches.  Q and K of 2 x 4096 tokens, 16 + 16 heads of d = 64 in bf16:
// 13.7 us in the kernel, 5.1 TB/s; 500 tokens into the cache, d = 128, 8 sequences: 19.9 us, 3.9 TB/s.
template <typename T, int D, bool INTER, bool AXES>
__global__ __launch_bounds__(kThreads) void k_heads(const HeadsArgs x, int per_block) {
  constexpr int E = Chunk<T>::E, U = D / (2 * E), TB = kThreads / U;
  using vec_t = typename Chunk<T>::vec_t;
  const int u = threadIdx.x % U;
  const int64_t n = (int64_t)blockIdx.x * TB + threadIdx.x / U;
  if (n >= (int64_t)x.B * x.T) return;
  const int b = (int)(n / x.T), t = (int)(n - (int64_t)b * x.T);
  const int64_t place = (int64_t)(x.first ? x.first[b] : 0) + t;
  const bool counts = !x.counts || t < x.counts[b];

  // where the unit's chunks lie, and its turn
  const bool turns = u < x.rot / (2 * E);
  const int c0 = (turns && !INTER ? u * E : 2 * u * E) * (int)sizeof(T);
  const int step = (turns && !INTER ? x.rot / 2 : E) * (int)sizeof(T);
  float co[E], si[E];
  if (AXES && turns) {
    int at[SPLAT_ROTARY_MAX_AXES];
#pragma unroll
    for (int a = 0; a < SPLAT_ROTARY_MAX_AXES; ++a)
      at[a] = x.positions[(int64_t)min(a, x.axes - 1) * x.B * x.T + n];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int a = x.axis[u * E + e];
      const int pos = a == 0 ? at[0] : a == 1 ? at[1] : a == 2 ? at[2] : at[3];
      const bool inside = pos >= 0 && pos < x.max_len;
      const f32x2_t v = *(const f32x2_t*)(x.angles + (int64_t)(inside ? pos : 0) * (x.rot / 2) + u * E + e);
      co[e] = inside ? v[0] : NAN, si[e] = inside ? (x.inverse ? -v[1] : v[1]) : NAN;
    }
  }
  if (!AXES && turns) {
    const int64_t pos = x.positions ? x.positions[n] : place;
    const bool inside = pos >= 0 && pos < x.max_len;
    const f32x4_t* a = (const f32x4_t*)(x.angles + (inside ? pos : 0) * (x.rot / 2) + u * E);
#pragma unroll
    for (int e = 0; e < E / 2; ++e) {
      const f32x4_t v = a[e];
      co[2 * e] = v[0], si[2 * e] = v[1], co[2 * e + 1] = v[2], si[2 * e + 1] = v[3];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (x.inverse) si[e] = -si[e];
      if (!inside) co[e] = si[e] = NAN;
    }
  }
  // the token's page in the cache, -1 if it has none
  const int page =
      x.pages && counts ? page_of(x.pages, b, x.max_pages, x.n_pages, x.page_shift, place) : -1;

  // blockIdx.y: a run of one tensor's heads
  int j = 0, run = blockIdx.y;
  while (run >= (x.job[j].heads + per_block - 1) / per_block)
    run -= (x.job[j].heads + per_block - 1) / per_block, ++j;
  const HeadsJob& job = x.job[j];
  const int first = run * per_block, last = min(first + per_block, job.heads);
  const bool rot = job.rotate && turns && counts;
  char* to = job.y + c0;
  int64_t next = job.yh;                // to the next head
  if (job.paged) {
    if (page < 0) return;
    to += (size_t)cache_row(page, job.heads, first, x.page_shift, place) * (D * sizeof(T));
    next = ((int64_t)D * (int)sizeof(T)) << x.page_shift;
  } else {
    to += b * job.yb + t * job.yt + first * job.yh;
  }
  const char* from = job.x + c0 + b * job.xb + t * job.xt + first * job.xh;
  for (int h0 = first; h0 < last; h0 += kInFlight) {
    vec_t v[kInFlight][2];
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      v[k][0] = vec_t{}, v[k][1] = vec_t{};
      if (h0 + k < last && counts) {
        v[k][0] = *(const vec_t*)(from + k * job.xh);
        v[k][1] = *(const vec_t*)(from + k * job.xh + step);
      }
    }
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      if (h0 + k >= last) continue;
      if (rot) {
        vec_t r[2];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          // pair e: elements e of both chunks, or 2 e and 2 e + 1 of them in a row
          const float p = (float)(INTER ? v[k][2 * e / E][2 * e % E] : v[k][0][e]);
          const float q = (float)(INTER ? v[k][2 * e / E][2 * e % E + 1] : v[k][1][e]);
          const float y0 = p * co[e] - q * si[e], y1 = q * co[e] + p * si[e];
          if (INTER) {
            r[2 * e / E][2 * e % E] = (T)y0, r[2 * e / E][2 * e % E + 1] = (T)y1;
          } else {
            r[0][e] = (T)y0, r[1][e] = (T)y1;
          }
        }
        v[k][0] = r[0], v[k][1] = r[1];
      }
      __builtin_nontemporal_store(v[k][0], (vec_t*)(to + k * next));
      __builtin_nontemporal_store(v[k][1], (vec_t*)(to + k * next + step));
    }
    from += kInFlight * job.xh, to += kInFlight * next;
  }
}

template <typename T, int D>
hipError_t heads_launch(const HeadsArgs& x, hipStream_t st) {
  constexpr int TB = kThreads / (D / (2 * Chunk<T>::E));
  const int64_t blocks = ((int64_t)x.B * x.T + TB - 1) / TB;
  int64_t heads = 0;
  for (int k = 0; k < x.n_jobs; ++k) heads += x.job[k].heads;
  // as many heads a thread as leave the chip eight workgroups a CU, and more where
  // their runs would pass a grid's second dimension
  int64_t per = blocks * heads / 2048;
  per = per < 1 ? 1 : per > kMaxHeads ? kMaxHeads : per;
  per = std::max(per, heads / kMaxRuns + 1);
  int64_t runs = 0;
  for (int k = 0; k < x.n_jobs; ++k) runs += (x.job[k].heads + per - 1) / per;
  const dim3 grid((unsigned)blocks, (unsigned)runs);
  auto* const k = x.axis ? (x.interleaved ? k_heads<T, D, true, true> : k_heads<T, D, false, true>)
                         : (x.interleaved ? k_heads<T, D, true, false> : k_heads<T, D, false, false>);
  hipLaunchKernelGGL(k, grid, dim3(kThreads), 0, st, x, (int)per);
  return hipGetLastError();
}

// ------------------------------------------------------------ one query token
// O = softmax(scale q K^T) V over the columns of one mask row, for up to 32
// query heads that share a head of K and V: the heads take the place of the 32
// query rows of a slice, so that K and V are read once for all of them and the
// products run on the matrix cores however many there are.  The row's columns
// are taken by rank, 32 a unit, each lane finding one key's page.  A workgroup
// has a contiguous range of a sequence's units, its wavefronts every fourth of
// them; ranges of one sequence are joined by a second kernel.  Bound by memory:
// K and V of the row's keys are read once, staged in LDS by loads that take whole
// rows.  32 sequences of 1000 .. 8192 keys, 32 heads over 8, d = 128, bf16: 117 us and
// 4.7 to join, 5.0 TB/s, what a copy of 1 GiB reaches (fp32: 274 in all, 4.4 TB/s; fp32,
// d = 64: 165, 3.7 TB/s); one sequence of a window's 577 keys 5.4 us and 4.0 to join, a
// chain of loads (row, pages, keys) with nothing to hide it.
constexpr int kHeadRows = 32;
constexpr int kMaxSplits = 64;

template <typename T, int D>
constexpr int kDecodeStage = kUnit * D * (int)sizeof(T);       // K or V of a unit
template <int D>
constexpr int kDecodeSum = kHeadRows * (D + 4) * 4;            // a wavefront's O
template <typename T, int D>
constexpr int kDecodeLds =
    4 * (2 * kDecodeStage<T, D> > kDecodeSum<D> ? 2 * kDecodeStage<T, D> : kDecodeSum<D>) +
    4 * 2 * kHeadRows * 4;

// Keys of sequence b's row: -1 for a length that is not one.
__device__ __forceinline__ int row_keys(const RowRuns* runs, int L, int len, int64_t room,
                                        RowRuns& rr) {
  if (len < 0 || len > L || len > room) return -1;
  if (len == 0) return 0;
  rr = runs[len - 1];
  return count_lt(rr, len);
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void k_decode(
    const RowRuns* __restrict__ runs, int L, int H, int heads, int chunks,
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V,
    const int32_t* __restrict__ pages, const int32_t* __restrict__ lengths, int max_pages,
    int n_pages, int page_shift, float sl2, T* __restrict__ O, float* __restrict__ ws) {
  using M = Mat<T, D>;
  constexpr int NB = D / 32, RB = D * (int)sizeof(T), CPR = RB / 16, RPL = 64 / CPR;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qi = lane & 31, h = lane >> 5;
  const int split = blockIdx.x, splits = gridDim.x;
  // blockIdx.y = (sequence, head of the cache, chunk of its query heads)
  const int chunk = blockIdx.y % chunks, bk = blockIdx.y / chunks;
  const int kh = bk % heads, b = bk / heads;
  const int group = H / heads, first = chunk * kHeadRows, mine = min(group - first, kHeadRows);
  const size_t row0 = (size_t)b * H + kh * group + first;      // of Q and O

  RowRuns rr;
  const int n = row_keys(runs, L, lengths[b], (int64_t)max_pages << page_shift, rr);
  const int units = n > 0 ? (n + kUnit - 1) / kUnit : 0;
  const int u1 = (int)((int64_t)units * (split + 1) / splits);
  int u = (int)((int64_t)units * split / splits) + wave;

  Slice s;
  s.lane = lane, s.qi = qi, s.h = h;
  typename M::Row q;
  load_row<T, D>(q, (const char*)(Q + row0 * D), (unsigned)(min(qi, mine - 1) * RB + 16 * h));
  f32x16_t o[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[c][r] = 0.f;
  float m = -INFINITY, l = 0.f;
  bool bad = n < 0;

  char* const sk = lds + wave * 2 * kDecodeStage<T, D>;
  char* const sv = sk + kDecodeStage<T, D>;
  // the row of the cache that holds this lane's key of unit u
  auto slot_of = [&](int unit) {
    const int j = dbg::idx(col_of(rr, min(unit * kUnit + qi, n - 1)), L, dbg::kKey);
    const int p = page_of(pages, b, max_pages, n_pages, page_shift, j);
    bad = bad || p < 0;
    return cache_row(p < 0 ? 0 : p, heads, kh, page_shift, j);
  };
  unsigned slot = u < u1 ? slot_of(u) : 0;
  for (; u < u1; u += 4) {
    wait_lds();   // the unit before it has left the rows that these loads fill
#pragma unroll
    for (int k = 0; k < kUnit / RPL; ++k) {
      const int r = RPL * k + lane / CPR;
      const size_t row = (size_t)(unsigned)__shfl((int)slot, r, 64) * RB;
      const int c = 16 * ((lane % CPR) ^ swz_row<CPR>(r));
      dma16((const char*)K + row + c, sk + kDmaBlock * k);
      dma16((const char*)V + row + c, sv + kDmaBlock * k);
    }
    const int count = min(n - u * kUnit, kUnit);
    if (u + 4 < u1) slot = slot_of(u + 4);
    wait_loads();
    const f32x16_t sc = dot_staged<T, D>(sk, s, q);
    float p[16], mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int k = 8 * (r >> 2) + 4 * h + (r & 3);
      p[r] = k < count ? sc[r] * sl2 : -INFINITY;
      mx = fmaxf(mx, p[r]);
    }
    mx = fmaxf(mx, lane_xor32(mx));
    const float mn = fmaxf(m, mx);
    const float mu = mn == -INFINITY ? 0.f : mn;   // every score so far -inf: weights 0
    if (__any(mn > m)) {
      const float alpha = exp2_hw(m - mu);
      l *= alpha;
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[c][r] *= alpha;
      m = mn;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = exp2_hw(p[r] - mu);
      l += p[r];
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      typename M::V v;
      load_staged<T, D>(v, sv, s, j);
      M::pv(o, v, p, j);
    }
  }
  l += lane_xor32(l);
  if (__any(bad)) l = NAN;

  // the wavefronts' (m, l, O) to one, rows of heads
  constexpr int OS = D + 4;
  float* const stat = (float*)(lds + kDecodeLds<T, D> - 4 * 2 * kHeadRows * 4);
  __syncthreads();
  float* const sum = (float*)lds + wave * kHeadRows * OS;
  if (qi < mine)
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        f32x4_t v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = o[(4 * c + e) % NB][4 * g + (4 * c + e) / NB];
        *(f32x4_t*)(sum + qi * OS + NB * (8 * g + 4 * h) + 4 * c) = v;
      }
  if (h == 0) stat[wave * 64 + qi] = m, stat[wave * 64 + 32 + qi] = l;
  __syncthreads();
  const int r = threadIdx.x >> 3;
  if (r >= mine) return;
  float mt = stat[r], f[4], lt = 0.f;
#pragma unroll
  for (int w = 1; w < 4; ++w) mt = fmaxf(mt, stat[w * 64 + r]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float mw = stat[w * 64 + r];
    f[w] = mw == -INFINITY ? 0.f : exp2_hw(mw - mt);
    lt += stat[w * 64 + 32 + r] * (mw == -INFINITY ? 1.f : f[w]);
  }
  // no key: 0; keys that all score -inf: NaN
  const float inv = n == 0 ? 0.f : 1.f / (lt == 0.f ? NAN : lt);
  float* const part = ws + ((row0 + r) * splits + split) * (D + 2);
#pragma unroll
  for (int k = 0; k < NB; ++k) {
    const int c = 4 * (threadIdx.x & 7) + 32 * k;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) v += *(const f32x4_t*)((const float*)lds + (w * kHeadRows + r) * OS + c) * f[w];
    if (splits == 1) {
      store4<T>(O + (row0 + r) * D + c, v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
    } else {
      *(f32x2_t*)(part + 2 + c) = f32x2_t{v[0], v[1]};
      *(f32x2_t*)(part + 4 + c) = f32x2_t{v[2], v[3]};
    }
  }
  if (splits > 1 && (threadIdx.x & 7) == 0)
    *(f32x2_t*)part = n == 0 ? f32x2_t{0.f, 1.f} : f32x2_t{mt, lt};
}

// One wavefront per (sequence, head): the splits' parts (m, l, O) to O, eight
// parts' loads in flight at a time (one after the other they took 10 us of a
// decode of one sequence).  A row without keys has parts (0, 1, 0).
template <typename T, int D>
__global__ __launch_bounds__(64) void k_decode_join(int splits, const float* __restrict__ ws,
                                                    T* __restrict__ O) {
  constexpr int STEP = 8;
  const int lane = threadIdx.x, row = blockIdx.x;
  const float* const part = ws + (size_t)row * splits * (D + 2);
  float m = -INFINITY, l = 0.f;
  if (lane < splits) {
    const f32x2_t ml = *(const f32x2_t*)(part + lane * (D + 2));
    m = ml[0], l = ml[1];
  }
  float acc[D / 64], x[STEP][D / 64];
#pragma unroll
  for (int b = 0; b < D / 64; ++b) acc[b] = 0.f;
  auto load = [&](int s0) {
#pragma unroll
    for (int k = 0; k < STEP; ++k)
#pragma unroll
      for (int b = 0; b < D / 64; ++b)
        x[k][b] = part[min(s0 + k, splits - 1) * (D + 2) + 2 + 64 * b + lane];
  };
  load(0);
  const float mt = wave_max(m), f = m == -INFINITY ? 0.f : exp2_hw(m - mt);
  const float lt = wave_sum(m == -INFINITY ? l : l * f);
  const float inv = 1.f / (lt == 0.f ? NAN : lt);   // keys that all score -inf: NaN
  for (int s0 = 0; s0 < splits; s0 += STEP) {
    if (s0) load(s0);
#pragma unroll
    for (int k = 0; k < STEP; ++k) {
      if (s0 + k >= splits) continue;
      const float fk = __builtin_bit_cast(
          float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), s0 + k));
#pragma unroll
      for (int b = 0; b < D / 64; ++b) acc[b] = fmaf(x[k][b], fk, acc[b]);
    }
  }
#pragma unroll
  for (int b = 0; b < D / 64; ++b) store1(O + (size_t)row * D + 64 * b + lane, acc[b] * inv);
}

int head_chunks(int H, int heads) { return (H / heads + kHeadRows - 1) / kHeadRows; }

template <typename T, int D>
hipError_t decode_launch(const DevAcsr& a, const DecodeArgs& x, hipStream_t st) {
  const int splits = decode_splits(a, x.B, x.H, x.heads), chunks = head_chunks(x.H, x.heads);
  const float sl2 = (float)((double)x.scale * 1.4426950408889634074);
  hipLaunchKernelGGL((k_decode<T, D>), dim3(splits, x.B * x.heads * chunks), dim3(kThreads),
                     (kDecodeLds<T, D>), st, a.runs, a.L, x.H, x.heads, chunks, (const T*)x.Q,
                     (const T*)x.K, (const T*)x.V, x.pages, x.lengths, x.max_pages, x.n_pages,
                     x.page_shift, sl2, (T*)x.O, x.ws);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  hipLaunchKernelGGL((k_decode_join<T, D>), dim3(x.B * x.H), dim3(64), 0, st, splits, x.ws, (T*)x.O);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t allow_lds() {
  return hipFuncSetAttribute((const void*)k_decode<T, D>, hipFuncAttributeMaxDynamicSharedMemorySize,
                             kDecodeLds<T, D>);
}

}  // namespace

hipError_t bounds_collect_serve(uint32_t* bits, bool clear) { return dbg::collect(bits, clear); }

hipError_t launch_heads(const HeadsArgs& x, int dtype, int d, hipStream_t st) {
  if (dtype == 0) return d == 64 ? heads_launch<float, 64>(x, st) : heads_launch<float, 128>(x, st);
  return d == 64 ? heads_launch<__bf16, 64>(x, st) : heads_launch<__bf16, 128>(x, st);
}

hipError_t prepare_decode() {
  hipError_t e = allow_lds<float, 64>();
  if (e == hipSuccess) e = allow_lds<float, 128>();
  if (e == hipSuccess) e = allow_lds<__bf16, 64>();
  if (e == hipSuccess) e = allow_lds<__bf16, 128>();
  return e;
}

// As many splits as fill the chip with two workgroups a CU while each wavefront
// keeps two units, between what a short row and a long one like best.  One / two /
// four units a wavefront: window 512 + 64 global at L = 4000, 16 heads, one
// sequence 10.4 / 8.5 / 7.8 us; every key of 8192, d = 128, 32 heads over 8, one
// sequence 21 / 15 / 17 us.  Twice and four times the workgroups for 32 sequences
// of 1000 .. 8192 keys: 130 -> 138, 150 us.
int decode_splits(const DevAcsr& a, int B, int H, int heads) {
  const int64_t groups = (int64_t)B * heads * head_chunks(H, heads);
  const int64_t units = (a.max_row_nnz + kUnit - 1) / kUnit;
  const int64_t s = std::min((512 + groups - 1) / groups, (units + 7) / 8);
  return (int)std::min<int64_t>(std::max<int64_t>(s, 1), kMaxSplits);
}

int64_t decode_workspace(const DevAcsr& a, int B, int H, int heads, int d) {
  const int splits = decode_splits(a, B, H, heads);
  return splits == 1 ? 0 : (int64_t)B * H * splits * (d + 2);
}

hipError_t launch_decode(const DevAcsr& a, int dtype, int d, const DecodeArgs& x, hipStream_t st) {
  if (dtype == 0)
    return d == 64 ? decode_launch<float, 64>(a, x, st) : decode_launch<float, 128>(a, x, st);
  return d == 64 ? decode_launch<__bf16, 64>(a, x, st) : decode_launch<__bf16, 128>(a, x, st);
}

}  // namespace splat
