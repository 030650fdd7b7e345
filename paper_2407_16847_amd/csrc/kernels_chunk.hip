// kernels_chunk.hip -- the attention of a chunk of new tokens over the paged cache.
//
// The chunk's n tokens are the last n of their sequence; token t has the mask's row
// p = length - n + t and its columns below the length:
//
//     s_ij = scale q_i.k_j    lse_i = ln sum_j exp(s_ij)    O_i = sum_j exp(s_ij - lse_i) v_j
//
// The query heads that share a head of the cache are rows of one block, token by
// token: row r of the sequence is token r / G, head r % G of the group of G.  A
// workgroup finds the keys that its rows need (chunk_plan.hpp) and walks them in
// units of 32.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "chunk_plan.hpp"
#include "serve_core.hpp"

namespace splat {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// One sequence's rows.
struct Chunk {
  int n, len, p0;     // tokens that count, the length, the first token's position
  bool bad;           // a length that is none
};
__device__ __forceinline__ Chunk chunk_of(const ChunkArgs& x, int L, int b) {
  Chunk c;
  c.n = x.counts ? min(max(x.counts[b], 0), x.T) : x.T;
  c.len = x.lengths[b];
  c.bad = c.len < c.n || c.len > L || c.len > ((int64_t)x.max_pages << x.page_shift);
  c.p0 = c.len - c.n;
  return c;
}

// i / G and the rest, for i below 2^24: the quotient by a reciprocal is off by one
// at most.
__device__ __forceinline__ int divide(int i, int G, float inv, int& rest) {
  int q = (int)((float)i * inv);
  rest = i - q * G;
  if (rest < 0) --q, rest += G;
  if (rest >= G) ++q, rest -= G;
  return q;
}

// The k-th longest sequence (the k-th, of more than 64): workgroups are dealt out in
// their grid's order, and the long ones had better not come last.
__device__ __forceinline__ int by_length(const int32_t* lengths, int B, int k) {
  if (B == 1 || B > 64) return k;
  const int lane = threadIdx.x & 63;
  const int len = lane < B ? lengths[lane] : 0;
  int rank = 0;
  for (int i = 0; i < B; ++i) {
    const int other = __builtin_amdgcn_readlane(len, i);
    rank += other > len || (other == len && i < lane);
  }
  return __builtin_ctzll(__ballot(lane < B && rank == k));
}

// Where a block's units are shared out, B * splits workgroups share out those of all
// sequences: each sequence has parts by its length (`splits` of them where there is one, or
// more than 64), at most x.cap.
struct Parts {
  int n, before;      // lane b: sequence b's parts, and those of the sequences before
};
__device__ __forceinline__ bool parts_vary(const ChunkArgs& x) { return x.cap != x.splits; }
__device__ __forceinline__ Parts parts_of(const ChunkArgs& x) {
  const int lane = threadIdx.x & 63;
  const int units = lane < x.B ? (min(max(x.lengths[lane], 1), x.most) + 31) / 32 : 0;
  int sum = units;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  Parts p;
  p.n = lane < x.B ? min(1 + units * (x.B * (x.splits - 1)) / sum, x.cap) : 0;
  int upto = p.n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(upto, o, 64);
    if (lane >= o) upto += y;
  }
  p.before = upto - p.n;
  return p;
}
// workgroup k of B * splits: its sequence (-1: none), part and how many of them
__device__ __forceinline__ int part_of(const ChunkArgs& x, int k, int& split, int& splits) {
  if (!parts_vary(x)) {
    splits = x.splits, split = k % splits;
    return k / splits;
  }
  const Parts p = parts_of(x);
  const uint64_t here = __ballot(k >= p.before && k < p.before + p.n);
  if (!here) return -1;
  const int b = __builtin_ctzll(here);
  splits = __builtin_amdgcn_readlane(p.n, b), split = k - __builtin_amdgcn_readlane(p.before, b);
  return b;
}

// What is read in the place of a key without a page, and then has no part in any row: the
// sequence's newest key, whose values are a token's where an unused page may hold anything
// (a NaN there would have every row formed again).
__device__ __forceinline__ unsigned spare_row(const ChunkArgs& x, int b, int kh, int len) {
  const int p = page_of(x.pages, b, x.max_pages, x.n_pages, x.page_shift, len - 1);
  return p < 0 ? 0u : cache_row(p, x.heads, kh, x.page_shift, len - 1);
}

// O and lse of one row by one wavefront, from the row's own keys alone.
template <typename T, int D>
__device__ __forceinline__ void row_alone(const ChunkArgs& x, const RowRuns& rr, int b, int kh, int len,
                                       const T* q, T* o, float* lse) {
  constexpr int NC = D / 64;
  const int lane = threadIdx.x & 63, n = count_lt(rr, len);
  float m = -__FLT_MAX__, l = n > 0 ? 0.f : 1.f, acc[NC];
  bool bad = false;
#pragma unroll
  for (int c = 0; c < NC; ++c) acc[c] = 0.f;
#pragma unroll 1
  for (int k0 = 0; k0 < n; k0 += 64) {
    const bool valid = k0 + lane < n;
    unsigned slot = 0;
    float s = -INFINITY;
    if (valid) {
      const int j = col_of(rr, k0 + lane);
      const int p = page_of(x.pages, b, x.max_pages, x.n_pages, x.page_shift, j);
      bad = bad || p < 0;
      slot = cache_row(max(p, 0), x.heads, kh, x.page_shift, j);
      // rare: few registers instead of many loads in flight
      const T* const k = (const T*)x.K + (size_t)slot * D;
      float dot = 0.f;
#pragma unroll 1
      for (int c = 0; c < D; c += 8)
#pragma unroll
        for (int e = 0; e < 8; ++e) dot = fmaf((float)q[c + e], (float)k[c + e], dot);
      s = dot * x.scale;
    }
    const float mn = fmaxf(m, wave_max(s));
    const float alpha = expf(m - mn), p = valid ? expf(s - mn) : 0.f;
    l = l * alpha + wave_sum(p);
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[c] *= alpha;
#pragma unroll 1
    for (int t = 0; t < min(64, n - k0); ++t) {
      const float pt = __shfl(p, t, 64);
      const T* const v = (const T*)x.V + (size_t)(unsigned)__shfl((int)slot, t, 64) * D;
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[c] = fmaf(pt, (float)v[64 * c + lane], acc[c]);
    }
    m = mn;
  }
  if (__any(bad)) l = NAN;
  // keys that all score -inf: 0 / 0, and lse -inf
  if (lane == 0) *lse = n == 0 ? -INFINITY : m + logf(l);
#pragma unroll
  for (int c = 0; c < NC; ++c) store1(o + 64 * c + lane, acc[c] / l);
}

template <typename T, int D>
__device__ __forceinline__ void redo_row(const ChunkArgs& x, const RowRuns* runs, int L, int b, int kh,
                                         const Chunk& c, int t, int g) {
  const int head = kh * x.group + g;
  const RowRuns rr = runs[dbg::idx(c.p0 + t, L, dbg::kRow)];
  row_alone<T, D>(x, rr, b, kh, c.len, (const T*)x.Q + b * x.qb + head * x.qh + t * x.qt,
                  (T*)x.O + b * x.ob + head * x.oh + t * x.ot,
                  x.lse + ((int64_t)b * x.H + head) * x.T + t);
}

// ------------------------------------------------------------------ slices
// A workgroup per 32 rows; its wavefronts take every fourth unit of the rows' keys
// and join at the end, and so do workgroups that share out a block's units.  Each
// wavefront keeps a softmax of its own (running maximum, sum, O): one pass over the
// keys.  Bound by HBM where sequences are long: 5 tokens of 16 sequences of 1000 .. 8192 keys, 32
// heads over 8, d = 128, bf16 59.6 us, 5.1 TB/s, what a copy of 1 GiB reaches, and 5.5 to join;
// else by the chain length, rows' runs, plan, pages, keys, products, some 8 us: 8 tokens of one
// sequence, 16 heads, under window 512 + 64 global, in five parts, 11.6 us with the joining launch.
// fp32, where each unit takes the matrix cores 2 us at d = 64: 300 tokens under a window of 256, 21.8 us.
constexpr int kRows = 32;

// Waits until at most N of this wavefront's loads are on their way.
template <int N>
__device__ __forceinline__ void loads_left() {
  static_assert(N < 64, "vmcnt field");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
  asm volatile("" ::: "memory");
}

template <typename T, int D>
constexpr int kStage = kUnit * D * (int)sizeof(T);       // K or V of a unit
template <typename T, int D>
constexpr int kSliceLds =
    4 * (2 * kStage<T, D> > kRows * (D + 4) * 4 ? 2 * kStage<T, D> : kRows * (D + 4) * 4) +
    4 * 2 * kRows * 4;

template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) * D > 256 ? 1 : 2) void k_chunk_slices(const RowRuns* __restrict__ runs, int L,
                                                           const ChunkArgs x) {
  using M = Mat<T, D>;
  constexpr int NB = D / 32, RB = D * (int)sizeof(T), CPR = RB / 16, RPL = 64 / CPR;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ uint64_t part[2 * kThreads / 64];
  __shared__ uint32_t redo;
  __shared__ RowEnds ends[4 * kRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qi = lane & 31, h = lane >> 5;
  // workgroups of one sequence and head share its keys: neighbours on a die
  const int kh = blockIdx.x % x.heads, rest = blockIdx.x / x.heads, shares = x.B * x.splits;
  const int block = x.blocks - 1 - rest / shares, G = x.group;
  int split, splits;
  const int b = part_of(x, rest % shares, split, splits);
  if (b < 0) return;
  const Chunk ch = chunk_of(x, L, b);
  const int r0 = block * kRows, rows = min(kRows, ch.n * G - r0);   // rows that count
  if (x.splits > 1 && rows <= 0) return;                 // the joining kernel clears the padding

  const int i = r0 + min(qi, max(rows - 1, 0)), t = i / G, g = i - t * G;
  RowsPlan plan(lds, L);
  char* const stage = lds + plan_bytes(L);
  int u0 = 0, u1 = 0;
  RowEnds& row = ends[wave * kRows + qi];
  bool dense = true;
  unsigned spare = 0;
  typename M::Row q;
  if (rows > 0 && !ch.bad && ch.len > 0) {
    const int t0 = r0 / G, t1 = (r0 + rows - 1) / G;
    dense = row.open(runs, dbg::idx(ch.p0 + t, L, dbg::kRow));
    load_row<T, D>(q, (const char*)((const T*)x.Q + b * x.qb + (kh * G + g) * x.qh + t * x.qt), 16u * h);
    spare = spare_row(x, b, kh, ch.len);
    plan_rows<kThreads>(plan, part, L, runs, ch.p0 + t0, t1 - t0 + 1, ch.len);
    u0 = (int)((int64_t)plan.n() * split / splits), u1 = (int)((int64_t)plan.n() * (split + 1) / splits);
  }
  const bool simple = __all(dense);
  Slice s;
  s.lane = lane, s.qi = qi, s.h = h;
  f32x16_t o[NB];
#pragma unroll
  for (int c = 0; c < NB; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[c][r] = 0.f;
  const float sl2 = x.scale * kLog2e;
  float m = -INFINITY, l = 0.f;
  bool bad = ch.bad;

  char* const sk = stage + wave * 2 * kStage<T, D>;
  char* const sv = sk + kStage<T, D>;
  // A wavefront has one K and one V unit in LDS: the next unit's K is loaded once the
  // scores are formed, its V once O is, so that loads are always on their way.  Pages
  // are looked up a unit ahead of that.
  constexpr int LOADS = kUnit / RPL;
  const int32_t* const table = x.pages + (int64_t)b * x.max_pages;
  auto key_of = [&](int u) {
    const int j = u < plan.dense ? min(32 * (plan.units()[u] & (int)(kFullUnit - 1)) + qi, ch.len - 1)
                                 : (int)plan.keys()[min(32 * (u - plan.dense) + qi, plan.gathered - 1)];
    return dbg::idx(j, L, dbg::kKey);
  };
  auto slot_of = [&](int u, int p, bool& found) {
    found = p >= 0 && p < x.n_pages;
    return found ? cache_row(p, x.heads, kh, x.page_shift, key_of(u)) : spare;
  };
  auto issue = [&](const void* from, unsigned slot, char* to) {
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      const int r = RPL * k + lane / CPR;
      const size_t row = (size_t)(unsigned)__shfl((int)slot, r, 64) * RB;
      dma16((const char*)from + row + 16 * ((lane % CPR) ^ swz_row<CPR>(r)), to + kDmaBlock * k);
    }
  };
  int u = u0 + wave, page = 0;
  bool found = true, next_found = true;
  unsigned slot = 0, next = 0;
  if (u < u1) {
    slot = slot_of(u, table[key_of(u) >> x.page_shift], found);
    issue(x.K, slot, sk);
    if (u + 4 < u1) page = table[key_of(u + 4) >> x.page_shift];
    issue(x.V, slot, sv);
  }
  for (; u < u1; u += 4) {
    const bool more = u + 4 < u1;
    // which of the unit's keys are the row's: bit r, the key of register r
    const uint32_t mine = register_bits(unit_word(plan, u, runs, row, simple, ch.len), h);
    const uint32_t lost = (uint32_t)__ballot(!found);   // keys without a page
    if (lost) bad = bad || (mine & register_bits(lost, h));
    loads_left<LOADS>();     // K is there
    const f32x16_t sc = dot_staged<T, D>(sk, s, q);
    if (more) {
      next = slot_of(u + 4, page, next_found);
      if (u + 8 < u1) page = table[key_of(u + 8) >> x.page_shift];
      wait_lds();            // K has been read
      issue(x.K, next, sk);
    }
    float p[16], mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = mine >> r & 1 ? sc[r] * sl2 : -INFINITY;
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
    if (more)
      loads_left<LOADS>();   // V is there
    else
      loads_left<0>();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      typename M::V v;
      load_staged<T, D>(v, sv, s, j);
      M::pv(o, v, p, j);
    }
    if (more) {
      wait_lds();            // V has been read
      issue(x.V, next, sv);
      slot = next, found = next_found;
    }
  }
  if (bad) l = NAN;
  l += lane_xor32(l);

  // the wavefronts' (m, l, O) to one
  constexpr int OS = D + 4;
  float* const stat = (float*)(stage + kSliceLds<T, D> - 4 * 2 * kRows * 4);
  if (threadIdx.x == 0) redo = 0;
  __syncthreads();
  float* const sum = (float*)stage + wave * kRows * OS;
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      f32x4_t v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = o[(4 * c + e) % NB][4 * k + (4 * c + e) / NB];
      *(f32x4_t*)(sum + qi * OS + NB * (8 * k + 4 * h) + 4 * c) = v;
    }
  if (h == 0) stat[wave * 64 + qi] = m, stat[wave * 64 + 32 + qi] = l;
  __syncthreads();
  const int r = threadIdx.x >> 3, ri = r0 + r, rt = ri / G, rg = ri - rt * G;
  float mt = stat[r], f[4], lt = 0.f;
#pragma unroll
  for (int w = 1; w < 4; ++w) mt = fmaxf(mt, stat[w * 64 + r]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float mw = stat[w * 64 + r];
    f[w] = mw == -INFINITY ? 0.f : exp2_hw(mw - mt);
    lt += stat[w * 64 + 32 + r] * (mw == -INFINITY ? 1.f : f[w]);
  }
  const int64_t head = (int64_t)b * x.H + kh * G + rg;
  if (x.splits > 1) {
    if (r >= rows) return;
    float* const to = x.ws + ((head * x.T + rt) * x.cap + split) * (D + 2);
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int c = 4 * (threadIdx.x & 7) + 32 * k;
      f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) v += *(const f32x4_t*)((const float*)stage + (w * kRows + r) * OS + c) * f[w];
      *(f32x2_t*)(to + 2 + c) = f32x2_t{v[0], v[1]};
      *(f32x2_t*)(to + 4 + c) = f32x2_t{v[2], v[3]};
    }
    if ((threadIdx.x & 7) == 0) *(f32x2_t*)to = f32x2_t{mt, lt};
    return;
  }
  if (ri < x.T * G) {
    T* const O = (T*)x.O + b * x.ob + (kh * G + rg) * x.oh + rt * x.ot;
    // a row without weight has no key, or is formed again
    const float inv = lt == 0.f ? 0.f : 1.f / lt;
    bool fine = r >= rows || ch.bad || (lt > 0.f && lt < INFINITY);
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int c = 4 * (threadIdx.x & 7) + 32 * k;
      f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) v += *(const f32x4_t*)((const float*)stage + (w * kRows + r) * OS + c) * f[w];
      v *= inv;
      if (r >= rows) v = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e) fine = fine && (r >= rows || ch.bad || fabsf(v[e]) < INFINITY);
      store4<T>(O + c, v[0], v[1], v[2], v[3]);
    }
    if ((threadIdx.x & 7) == 0)
      x.lse[head * x.T + rt] = r >= rows || lt == 0.f ? -INFINITY : kLn2 * (mt + log2f(lt));
    if (!fine) atomicOr(&redo, 1u << r);
  }
  __syncthreads();
  // rows that are not finite, or have no weight, from their own keys: what another
  // row's key holds does not reach them
  const uint32_t again = redo;
  for (int k = wave; k < kRows; k += 4)
    if (again >> k & 1) redo_row<T, D>(x, runs, L, b, kh, ch, (r0 + k) / G, (r0 + k) % G);
}

// ------------------------------------------------------------------- tiles
// bf16, many rows: a workgroup per 128 rows, 32 a wavefront, which share tiles of two
// units (64 keys) of K and V through a two-slot LDS ring, the next tile's loads
// in flight while this one is computed.  Products on v_mfma_f32_32x32x16_bf16:
// S^T = K Q^T, so that a lane has 32 scores of one row, and O^T += V^T P^T with P^T
// taken from the score registers.  A row's reference m stays while its tiles' sums
// stay below kSumLimit, without a look at the maximum: a tile past it (and a row's first)
// takes the exact maximum and rescales.
// P^T is rounded to bf16 as in the fused forward, which leaves an error of O of 0.0023 of its
// size where its own rounding leaves 0.0017.  A second product with what the rounding left brings that
// to 0.0017, at 413 us for 311 and 80 for 64 of the cases below.  O is divided by the sum of the weights
// before the rounding, so a feature is off by at most 2^-8 of the row's sum of w |v|; by the
// sum of the rounded ones it would be of w |v - O|: none where values are equal, but up to twice as
// much where they have both signs, at 2 to 3% more time.
// Bound by the matrix cores and the vector ALUs in turn, and by the longest blocks: 1024
// tokens of 4 sequences over 2048 .. 8192 keys, 32 heads over 8, d = 128 317 us, 875
// TFLOP/s (1232 in a product of 8192^3), the matrix cores 39% and the vector ALUs 41% busy; 2048
// tokens of 4 sequences under window 512 + 64 global, 16 heads, d = 64 60.5 us, 455 TFLOP/s: one
// uneven turn of 832 blocks, 2.2 of 4 wavefronts a SIMD.
// One 16-key step's products straight behind its exponentials, instead of a tile's behind all
// of them: 10% slower.  Without priority for the products: 4% slower.
constexpr int kTileRows = 128;
constexpr float kSumLimit = 4096.f;

// V^T of a tile's keys 16 J .. 16 (J + NJ) - 1 and one block of 32 features (the transposing
// reads of read_v_block).
template <int D, int J, int NJ, int K = 0>
__device__ __forceinline__ void read_v_part(unsigned at, bf16x8_t (&v)[NJ]) {
  constexpr int RB = 2 * D;
  if constexpr (K < NJ) {
    v[K] = __builtin_shufflevector(tr16_async_at<16 * (J + K) * RB>(at),
                                   tr16_async_at<16 * (J + K) * RB + 8 * RB>(at), 0, 1, 2, 3, 4, 5, 6, 7);
    read_v_part<D, J, NJ, K + 1>(at, v);
  }
}
// Waits until at most N of this wavefront's LDS reads are on their way; what was read
// before them depends on it.
template <int N>
__device__ __forceinline__ void part_wait(bf16x8_t (&v)[2]) {
  asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(v[0]), "+v"(v[1]) : "n"(N));
}
template <int N>
__device__ __forceinline__ void part_wait(bf16x8_t (&v)[4]) {
  asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]) : "n"(N));
}

// A tile's rows lie unpadded in LDS, their 16-byte chunks XOR-swizzled: K is read 16
// rows, one chunk each at a time, V 4 rows, 4 chunks each (transposed).  Rows of 256 bytes
// need a row's own place for that; two rows of 128 bytes share the banks (swz_k, swz_v).
template <int D>
__device__ __forceinline__ int place_k(int r) { return D == 128 ? r & 15 : swz_k(r); }
template <int D>
__device__ __forceinline__ int place_v(int r) { return D == 128 ? (r & 3) << 2 : swz_v(r); }

template <int D>
struct Ring {
  static constexpr int RB = 2 * D, CPR = RB / 16;       // bytes, 16-byte chunks of a row
  static constexpr int TB = 2 * kUnit * RB;             // bytes of a tile of K or V
  static constexpr int RPL = 64 / CPR;                  // rows a load
  static constexpr int N = 2 * kUnit / RPL / 4;         // loads a wavefront and tile of each
  static constexpr int LDS = 4 * TB;
};

// log2 of the rows in LDS a unit, for pages of 8 keys and more
__host__ __device__ constexpr int tiles_sub(int page_shift) {
  return page_shift < 3 || page_shift > 5 ? 0 : 5 - page_shift;
}

template <int D>
__global__ __launch_bounds__(kThreads, D == 64 ? 4 : 2) void k_chunk_tiles(
    const RowRuns* __restrict__ runs, int L, const ChunkArgs x) {
  using R = Ring<D>;
  constexpr int NKS = D / 16, NDB = D / 32, RB = R::RB;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ uint64_t part[2 * kThreads / 64];
  __shared__ uint32_t redo[4], lost;
  __shared__ RowEnds ends[kTileRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qi = lane & 31, h = lane >> 5;
  // the longest sequence's blocks first, of each the last (longest) first
  const int kh = blockIdx.x % x.heads, rest = blockIdx.x / x.heads, G = x.group;
  const int block = x.blocks - 1 - rest % x.blocks;
  int split = 0, splits = 1, b;
  if (x.splits > 1)
    b = part_of(x, rest / x.blocks, split, splits);
  else
    b = by_length(x.lengths, x.B, rest / x.blocks);
  if (b < 0) return;
  const Chunk ch = chunk_of(x, L, b);
  const int r0 = block * kTileRows, rows = min(kTileRows, ch.n * G - r0);   // rows that count
  if (x.splits > 1 && rows <= 0) return;                 // the joining kernel clears the padding

  int mine = wave * 32 + qi;                           // this lane's row of the block
  RowsPlan plan(lds, L, tiles_sub(x.page_shift));
  int u0 = 0, u1 = 0;
  RowEnds& row = ends[mine];
  bool dense = true;
  unsigned spare = 0;
  bf16x8_t q[NKS];
  char* const ring = lds + plan_bytes(L, tiles_sub(x.page_shift));
  if (rows > 0 && !ch.bad && ch.len > 0) {
    const int t0 = r0 / G, t1 = (r0 + rows - 1) / G;
    const int i = r0 + min(mine, rows - 1), t = i / G, g = i - t * G;
    const __bf16* const from = (const __bf16*)x.Q + b * x.qb + (kh * G + g) * x.qh + t * x.qt;
#pragma unroll
    for (int k = 0; k < NKS; ++k) q[k] = *(const bf16x8_t*)(from + 16 * k + 8 * h);
    dense = row.open(runs, dbg::idx(ch.p0 + t, L, dbg::kRow));
    spare = spare_row(x, b, kh, ch.len);
    plan_rows<kThreads>(plan, part, L, runs, ch.p0 + t0, t1 - t0 + 1, ch.len);
    u0 = (int)((int64_t)plan.n() * split / splits), u1 = (int)((int64_t)plan.n() * (split + 1) / splits);
  }
  const bool simple = __all(dense);
  if (threadIdx.x < 4) redo[threadIdx.x] = 0;
  if (threadIdx.x == 0) lost = 0;

  // K operand of key 32 * half + qi, chunk 2 * ks + h; V^T operand by transposing reads
  const int koff = qi * RB + 16 * (h ^ place_k<D>(qi));
  const int vr = 4 * h + ((lane & 15) >> 2);
  const int voff = vr * RB + 16 * ((2 * (lane >> 4 & 1) + (lane >> 1 & 1)) ^ place_v<D>(vr)) + 8 * (lane & 1);
  f32x16_t o[NDB];
#pragma unroll
  for (int c = 0; c < NDB; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[c][r] = 0.f;
  const float sl2 = x.scale * kLog2e;
  float m = 0.f, l = 0.f;
  bool set = false, found = true;          // the row has a reference; every page was one

  // Of unit u's keys this lane loads rows r = RPL * (wave + 4 k) % 32 + lane / CPR, k <
  // NU.  Where 8 keys or more lie in one page, the first row in the cache of each 8, 16 or 32 (a
  // multiple of as many) and, in its low bits, the last key stand in LDS from here on;
  // elsewhere pages are looked up a tile before they are needed, ahead of the tile's
  // loads, so that nothing waits for those.
  constexpr int NU = R::N / 2;             // loads of each a unit
  const int r_lane = lane / R::CPR;
  const int32_t* const table = x.pages + (int64_t)b * x.max_pages;
  const bool whole_pages = plan.gathered == 0 && x.page_shift >= 3;
  const int run = min(x.page_shift, 5), low = (1 << run) - 1;
  uint32_t* const unit_rows = (uint32_t*)lds;          // over the gathered keys
  if (whole_pages) {
    for (int k = (u0 << (5 - run)) + (int)threadIdx.x; k < u1 << (5 - run); k += kThreads) {
      const int u = k >> (5 - run), from = k & ((1 << (5 - run)) - 1);
      const int word = plan.units()[u] & (int)(kFullUnit - 1);
      const int kb = min(32 * word + (from << run), (ch.len - 1) & ~low);   // of keys that there are
      const int page = table[kb >> x.page_shift];
      const bool ok = page >= 0 && page < x.n_pages;
      found = found && ok;
      unit_rows[k] = ok ? cache_row(page, x.heads, kh, x.page_shift, kb) | min(low, ch.len - 1 - kb) : spare & ~(unsigned)low;
    }
    __syncthreads();
  }
  auto key_of = [&](int u, int k) {        // the key of load k
    const int r = (R::RPL * (wave + 4 * k)) % 32 + r_lane;
    const int j = u < plan.dense ? min(32 * (plan.units()[u] & (int)(kFullUnit - 1)) + r, ch.len - 1)
                                 : (int)plan.keys()[min(32 * (u - plan.dense) + r, plan.gathered - 1)];
    return dbg::idx(j, L, dbg::kKey);
  };
  auto pages_of = [&](int u, int (&p)[NU]) {
    if (whole_pages) return;
    u = min(u, u1 - 1);
#pragma unroll
    for (int k = 0; k < NU; ++k) p[k] = table[key_of(u, k) >> x.page_shift];
  };
  auto slots_of = [&](int u, const int (&p)[NU], unsigned (&slot)[NU]) {
    u = min(u, u1 - 1);
    if (whole_pages) {
#pragma unroll
      for (int k = 0; k < NU; ++k) {
        const int r = (R::RPL * (wave + 4 * k)) % 32 + r_lane;
        const uint32_t e = unit_rows[(u << (5 - run)) + (r >> run)];
        slot[k] = (e & ~(uint32_t)low) + min((uint32_t)(r & low), e & low);
      }
      return;
    }
#pragma unroll
    for (int k = 0; k < NU; ++k) {
      const bool ok = p[k] >= 0 && p[k] < x.n_pages;
      found = found && ok;
      slot[k] = ok ? cache_row(p[k], x.heads, kh, x.page_shift, key_of(u, k)) : spare;
    }
  };
  auto issue = [&](char* to, const unsigned (&slot)[2][NU]) {
#pragma unroll
    for (int k = 0; k < R::N; ++k) {
      const int bk = wave + 4 * k, r = bk * R::RPL + lane / R::CPR, c = lane % R::CPR;
      const unsigned row = slot[k / NU][k % NU];
      dma16((const char*)x.K + 16 * (c ^ place_k<D>(r)) + (uint64_t)row * RB, to + bk * kDmaBlock);
      dma16((const char*)x.V + 16 * (c ^ place_v<D>(r)) + (uint64_t)row * RB, to + R::TB + bk * kDmaBlock);
    }
  };
  unsigned slot[2][NU];
  int page[2][NU];
  const int nt = (u1 - u0 + 1) / 2;
  if (nt > 0) {
#pragma unroll
    for (int e = 0; e < 2; ++e) pages_of(u0 + e, page[e]), slots_of(u0 + e, page[e], slot[e]);
#pragma unroll
    for (int e = 0; e < 2; ++e) pages_of(u0 + 2 + e, page[e]);
    issue(ring, slot);
    ring_sync<0>();
  }
  for (int it = 0; it < nt; ++it) {
    const int u = u0 + 2 * it;
    const char* const sk = ring + (it & 1) * 2 * R::TB;
    if (it + 1 < nt) {
#pragma unroll
      for (int e = 0; e < 2; ++e) slots_of(u + 2 + e, page[e], slot[e]);
#pragma unroll
      for (int e = 0; e < 2; ++e) pages_of(u + 4 + e, page[e]);
      issue(ring + (~it & 1) * 2 * R::TB, slot);
    }
    // which of the tile's keys are the row's: bit r of 16 h', the key of register r of
    // half h'; the lanes' halves form a unit's word each
    uint32_t word = 0;
    if (u + h < u1) word = unit_word(plan, u + h, runs, row, simple, ch.len);
    const uint32_t other = __builtin_bit_cast(uint32_t, lane_xor32(__builtin_bit_cast(float, word)));
    // ... one unit after the other, or (d = 128) both at once
    auto pass = [&](auto FIRST) {
      constexpr int E = FIRST, NE = D == 64 ? 1 : 2;      // units E .. E + NE - 1
      const uint32_t seen = NE == 2 ? word | other : (h == E ? word : other);
      if (!__any(seen != 0)) return;
      const bool whole = NE == 2 ? __all(word == ~0u) : __all(seen == ~0u);
      __builtin_amdgcn_s_setprio(1);
      f32x16_t s[NE];
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        bf16x8_t ka[NKS];
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
          ka[ks] = *(const bf16x8_t*)(sk + (koff ^ (32 * ks)) + (E + e) * 32 * RB);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[e][r] = 0.f;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) s[e] = mfma32(ka[ks], q[ks], s[e]);
      }
      __builtin_amdgcn_s_setprio(0);
      // against the row's reference, in powers of 2
#pragma unroll
      for (int e = 0; e < NE; ++e)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[e][r] = fmaf(s[e][r], sl2, -m);
      if (!whole) {
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          const uint32_t bits = register_bits(h == E + e ? word : other, h);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[e][r] = keep_if_bit(s[e][r], bits, r);
        }
      }
      bf16x8_t pf[2 * NE];
      auto exps = [&]() {
        float l0 = 0.f, l1 = 0.f;
#pragma unroll
        for (int j = 0; j < 2 * NE; ++j) {
          float e8[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) e8[e] = exp2_hw(s[j >> 1][(j & 1) * 8 + e]);
          l0 += (e8[0] + e8[1]) + (e8[2] + e8[3]);
          l1 += (e8[4] + e8[5]) + (e8[6] + e8[7]);
          pf[j] = __builtin_bit_cast(bf16x8_t, u32x4_t{pack_bf16_rn(e8[0], e8[1]), pack_bf16_rn(e8[2], e8[3]),
                                                       pack_bf16_rn(e8[4], e8[5]), pack_bf16_rn(e8[6], e8[7])});
        }
        return l0 + l1;
      };
      float lt = exps();
      // (both halves of the lanes decide alike: a row's sum and its keys are theirs together)
      const float both = lt + lane_xor32(lt);
      if (__any(!(both <= kSumLimit) || (!set && seen != 0))) {
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < NE; ++e)
#pragma unroll
          for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[e][r]);
        mx = fmaxf(mx, lane_xor32(mx));
        // a row without weight has no reference yet
        const float up = !set ? (mx == -INFINITY ? 0.f : mx) : fmaxf(0.f, mx);
        const float alpha = set ? exp2_hw(-up) : 0.f;
        l *= alpha;
#pragma unroll
        for (int c = 0; c < NDB; ++c)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[c][r] *= alpha;
        set = set || mx != -INFINITY;
        m += up;
#pragma unroll
        for (int e = 0; e < NE; ++e)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[e][r] -= up;
        lt = exps();
      }
      l += lt;
      __builtin_amdgcn_s_setprio(1);
      // V^T a block of 32 features at a time, the next one's reads in flight
      const unsigned sv = lds_addr(sk + R::TB);
      bf16x8_t va[2][2 * NE];
      read_v_part<D, 2 * E, 2 * NE>(sv + voff, va[0]);
#pragma unroll
      for (int c = 0; c < NDB; ++c) {
        if (c + 1 < NDB) {
          read_v_part<D, 2 * E, 2 * NE>(sv + (voff ^ (64 * (c + 1))), va[(c + 1) & 1]);
          part_wait<4 * NE>(va[c & 1]);
        } else {
          part_wait<0>(va[c & 1]);
        }
#pragma unroll
        for (int j = 0; j < 2 * NE; ++j) o[c] = mfma32(va[c & 1][j], pf[j], o[c]);
      }
      __builtin_amdgcn_s_setprio(0);
    };
    pass(std::integral_constant<int, 0>());
    if constexpr (D == 64) pass(std::integral_constant<int, 1>());
    ring_sync<0>();
  }
  l += lane_xor32(l);
  if (__any(!found)) lost = 1;
  __syncthreads();
  // pages that are none, among those of the units' keys: the rows that have a key there are
  // NaN, and no others (a cache may have given up the pages behind its window, and a unit of the
  // window's first keys reach into them).  Bit k: key k of the unit.
  bool gone = ch.bad;
  if (lost) {
    uint32_t* const none = (uint32_t*)ring;
    for (int k0 = 0; k0 < 32 * (u1 - u0); k0 += kThreads) {
      const int u = min(u0 + (k0 + (int)threadIdx.x) / 32, u1 - 1);
      const int j = u < plan.dense ? min(32 * (plan.units()[u] & (int)(kFullUnit - 1)) + qi, ch.len - 1)
                                   : (int)plan.keys()[min(32 * (u - plan.dense) + qi, plan.gathered - 1)];
      const int p = table[dbg::idx(j, L, dbg::kKey) >> x.page_shift];
      const uint64_t out = __ballot(p < 0 || p >= x.n_pages);
      if (qi == 0) none[u - u0] = (uint32_t)(h == 0 ? out : out >> 32);
    }
    __syncthreads();
    for (int u = u0; u < u1; ++u) {
      const uint32_t bits = none[u - u0];
      if (bits) gone = gone || (unit_word(plan, u, runs, row, simple, ch.len) & bits);
    }
    __syncthreads();
  }
  if (gone) l = NAN;
  asm volatile("" : "+v"(mine));     // formed again, not kept through the loop
  const bool counts = mine < rows;
  const int ri = r0 + mine, rt = ri / G;
  const int64_t place = ((int64_t)b * x.H + kh * G + ri - rt * G) * x.T + rt;   // of lse
  if (x.splits > 1) {
    if (!counts) return;
    float* const to = x.ws + (place * x.cap + split) * (D + 2);
    if (h == 0) *(f32x2_t*)to = f32x2_t{set ? m : -INFINITY, l};
#pragma unroll
    for (int c = 0; c < NDB; ++c)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float* const at = to + 2 + 32 * c + 8 * k + 4 * h;
        *(f32x2_t*)at = f32x2_t{o[c][4 * k], o[c][4 * k + 1]};
        *(f32x2_t*)(at + 2) = f32x2_t{o[c][4 * k + 2], o[c][4 * k + 3]};
      }
    return;
  }
  // whole rows by way of the ring
  const float inv = l == 0.f ? 0.f : 1.f / l;
  bool fine = l > 0.f && l < INFINITY;
  constexpr int OS = RB + 16;
  char* const stage = ring + wave * 32 * OS;
#pragma unroll
  for (int c = 0; c < NDB; ++c)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = counts ? o[c][4 * k + e] * inv : 0.f;
        fine = fine && fabsf(v[e]) < INFINITY;
      }
      store4<__bf16>((__bf16*)(stage + qi * OS) + 32 * c + 8 * k + 4 * h, v[0], v[1], v[2], v[3]);
    }
  const uint64_t again = __ballot(counts && !gone && !fine);
  if (lane == 0) redo[wave] = (uint32_t)again | (uint32_t)(again >> 32);
  if (h == 0 && ri < x.T * G)
    x.lse[place] = !counts || l == 0.f ? -INFINITY : kLn2 * (m + log2f(l));
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 32 / R::RPL; ++k) {
    const int r = k * R::RPL + lane / R::CPR, ri = r0 + wave * 32 + r, rt = ri / G;
    if (ri >= x.T * G) continue;
    *(u32x4_t*)((char*)((__bf16*)x.O + b * x.ob + (kh * G + ri - rt * G) * x.oh + rt * x.ot) +
                16 * (lane % R::CPR)) = *(const u32x4_t*)(stage + r * OS + 16 * (lane % R::CPR));
  }
  __syncthreads();
  for (int k = 0; k < 32; ++k)
    if (redo[wave] >> k & 1) {
      const int ri = r0 + wave * 32 + k;
      redo_row<__bf16, D>(x, runs, L, b, kh, ch, ri / G, ri % G);
    }
}

// One wavefront per row (all T of them): the parts (m, l, O) of the workgroups that
// shared out its block's units to O and lse, eight parts' loads in flight at a time.
template <typename T, int D>
__global__ __launch_bounds__(64) void k_chunk_join(const RowRuns* __restrict__ runs, int L,
                                                   const ChunkArgs x) {
  constexpr int STEP = 8;
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x;
  const int t = (int)(row % x.T), head = (int)(row / x.T % x.H), b = (int)(row / x.T / x.H);
  const Chunk ch = chunk_of(x, L, b);
  T* const O = (T*)x.O + b * x.ob + head * x.oh + t * x.ot;
  if (t >= ch.n) {
#pragma unroll
    for (int c = 0; c < D / 64; ++c) store1(O + 64 * c + lane, 0.f);
    if (lane == 0) x.lse[row] = -INFINITY;
    return;
  }
  const int splits = parts_vary(x) ? __builtin_amdgcn_readlane(parts_of(x).n, b) : x.splits;
  const float* const part = x.ws + row * x.cap * (D + 2);
  float m = -INFINITY, l = 0.f;
  if (lane < splits) {
    const f32x2_t ml = *(const f32x2_t*)(part + lane * (D + 2));
    m = ml[0], l = ml[1];
  }
  float acc[D / 64], v[STEP][D / 64];
#pragma unroll
  for (int c = 0; c < D / 64; ++c) acc[c] = 0.f;
  auto load = [&](int s0) {
#pragma unroll
    for (int k = 0; k < STEP; ++k)
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
        v[k][c] = part[min(s0 + k, splits - 1) * (D + 2) + 2 + 64 * c + lane];
  };
  load(0);
  const float mt = wave_max(m), f = m == -INFINITY ? 0.f : exp2_hw(m - mt);
  const float lt = wave_sum(m == -INFINITY ? l : l * f);
  const float inv = lt == 0.f ? 0.f : 1.f / lt;
  for (int s0 = 0; s0 < splits; s0 += STEP) {
    if (s0) load(s0);
#pragma unroll
    for (int k = 0; k < STEP; ++k) {
      if (s0 + k >= splits) continue;
      const float fk = __builtin_bit_cast(
          float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), s0 + k));
#pragma unroll
      for (int c = 0; c < D / 64; ++c) acc[c] = fmaf(v[k][c], fk, acc[c]);
    }
  }
  bool fine = lt > 0.f && lt < INFINITY;
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    acc[c] *= inv;
    fine = fine && fabsf(acc[c]) < INFINITY;
    store1(O + 64 * c + lane, acc[c]);
  }
  if (lane == 0) x.lse[row] = lt == 0.f ? -INFINITY : kLn2 * (mt + log2f(lt));
  if (__any(!fine) && !ch.bad) redo_row<T, D>(x, runs, L, b, head / x.group, ch, t, head % x.group);
}

template <typename T, int D>
hipError_t chunk_launch(const DevAcsr& a, const ChunkArgs& x, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)x.blocks * x.B * x.heads * x.splits));
  if constexpr (sizeof(T) == 2) {
    if (x.tiles)
      hipLaunchKernelGGL((k_chunk_tiles<D>), grid, dim3(kThreads),
                         plan_bytes(a.L, tiles_sub(x.page_shift)) + Ring<D>::LDS, st, a.runs, a.L, x);
  }
  if (!x.tiles)
    hipLaunchKernelGGL((k_chunk_slices<T, D>), grid, dim3(kThreads), (plan_bytes(a.L) + kSliceLds<T, D>),
                       st, a.runs, a.L, x);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || x.splits == 1) return e;
  hipLaunchKernelGGL((k_chunk_join<T, D>), dim3((unsigned)((int64_t)x.B * x.H * x.T)), dim3(64), 0, st,
                     a.runs, a.L, x);
  return hipGetLastError();
}

// ------------------------------------------------------------ weights of keys
// w_j = decay w_j + sum over the chunk's rows and the group's heads of
// exp(s_ij - lse_i), the probabilities formed again from the rows' log-sum-exp: a
// lane has a row and 16 keys, sums over the rows it sees, and the lanes' sums meet
// at the end.
__device__ __forceinline__ void keys_sum(float (&acc)[16], int lane) {
  // register r's sum over the lanes of a half comes to those whose low bits are r
  // (picked by bits: the compiler made a selection by index of ?:, 900 instructions)
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    const uint32_t up = lane & o ? ~0u : 0u;
#pragma unroll
    for (int r = 0; r < o; ++r) {
      const uint32_t a = __builtin_bit_cast(uint32_t, acc[r]), b = __builtin_bit_cast(uint32_t, acc[r + o]);
      const float give = __builtin_bit_cast(float, (a & up) | (b & ~up));
      acc[r] = __builtin_bit_cast(float, (b & up) | (a & ~up)) + __shfl_xor(give, o, 64);
    }
  }
  acc[0] += __shfl_xor(acc[0], 16, 64);
}
// the key, of a unit, whose sum a lane then has
__device__ __forceinline__ int key_of_lane(int lane) {
  const int r = lane & 15;
  return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
}

// Few rows: the sequences' units of 32 keys are dealt out evenly, whatever the lengths: a
// workgroup has a contiguous share of those of one head (of 64 sequences at a time), its
// wavefronts every fourth, the next one's K on its way.  A unit's keys go over the
// sequence's rows 32 at a time, which are all read and multiplied where they see any.  K of every
// unit is read, also of one that no row sees: a window saves products, not bytes.  Bound by HBM: a token of 32 sequences of
// 1000 .. 8192 keys, 32 heads over 8, d = 128, bf16 72 us, 4.3 TB/s (77 with the launch);
// shares by sequence instead of by length 119.
template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) * D > 256 ? 1 : 2) void k_weigh(
    const RowRuns* __restrict__ runs, int L, const WeighArgs x) {
  using M = Mat<T, D>;
  constexpr int RB = D * (int)sizeof(T), CPR = RB / 16, RPL = 64 / CPR, LOADS = kUnit / RPL;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ RowEnds ends[4 * kRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qi = lane & 31, h = lane >> 5, G = x.c.group, kh = blockIdx.x;
  Slice s;
  s.lane = lane, s.qi = qi, s.h = h;
  char* const stage = lds + wave * 2 * kStage<T, D>;
  const float sl2 = x.c.scale * kLog2e;
  RowEnds& row = ends[wave * kRows + qi];
  const int mine = key_of_lane(lane);      // of a unit: the key whose sum this lane writes
  auto issue = [&](unsigned slot, char* to) {
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      const int r = RPL * k + lane / CPR;
      const size_t at = (size_t)(unsigned)__shfl((int)slot, r, 64) * RB;
      dma16((const char*)x.c.K + at + 16 * ((lane % CPR) ^ swz_row<CPR>(r)), to + kDmaBlock * k);
    }
  };
  for (int b0 = 0; b0 < x.c.B; b0 += 64) {
    // lane i: sequence b0 + i's length, tokens and the units before it
    int len = 0, n = 0;
    if (b0 + lane < x.c.B) {
      const Chunk c = chunk_of(x.c, L, b0 + lane);
      len = c.bad ? 0 : c.len, n = c.n;
    }
    int upto = (len + 31) / 32;
    const int own = upto;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o, 64);
      if (lane >= o) upto += y;
    }
    const int before = upto - own, all = __builtin_amdgcn_readlane(upto, 63);
    const int v1 = (int)((int64_t)all * (blockIdx.y + 1) / gridDim.y);
    int v = (int)((int64_t)all * blockIdx.y / gridDim.y) + wave;

    // unit v: its sequence, number and length there, the place of its key qi
    struct At {
      int i, u, len;
    };
    auto find = [&](int w) {
      At a;
      a.i = __builtin_ctzll(__ballot(upto > w));
      a.u = w - __builtin_amdgcn_readlane(before, a.i);
      a.len = __builtin_amdgcn_readlane(len, a.i);
      return a;
    };
    auto page_at = [&](const At& a) {
      return x.c.pages[(int64_t)(b0 + a.i) * x.c.max_pages + (min(32 * a.u + qi, a.len - 1) >> x.c.page_shift)];
    };
    auto slot_of = [&](const At& a, int p, bool& found) {
      found = p >= 0 && p < x.c.n_pages;
      return cache_row(found ? p : 0, x.c.heads, kh, x.c.page_shift, min(32 * a.u + qi, a.len - 1));
    };
    bool found = false, next_found = false, simple = true;
    int page = 0, buf = 0, have_i = -1, have_r = -1;
    unsigned slot = 0, next = 0;
    At at{0, 0, 0}, ahead{0, 0, 0};
    typename M::Row q;
    float lse = 0.f;
    wait_lds();
    if (v < v1) {
      at = find(v);
      slot = slot_of(at, page_at(at), found);
      if (v + 4 < v1) ahead = find(v + 4), page = page_at(ahead);
      issue(slot, stage);
    }
    for (; v < v1; v += 4, buf ^= 1) {
      const int tokens = __builtin_amdgcn_readlane(n, at.i), rows = tokens * G, p0 = at.len - tokens;
      const int kb = 32 * at.u, b = b0 + at.i;
      const unsigned to = (unsigned)__shfl((int)slot, mine, 64);
      const bool writes = __shfl((int)found, mine, 64) && (lane & 16) == 0 && kb + mine < at.len;
      float old = 0.f;
      if (writes && kb + mine < p0) old = x.w[to] * (tokens > 0 ? x.decay : 1.f);
      const At now = at;
      if (v + 4 < v1) {
        next = slot_of(ahead, page, next_found);
        at = ahead;
        if (v + 8 < v1) ahead = find(v + 8), page = page_at(ahead);
        wait_lds();              // the unit before has been read
        issue(next, stage + (buf ^ 1) * kStage<T, D>);
        loads_left<LOADS>();
      } else {
        loads_left<0>();
      }
      float acc[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[r] = 0.f;
      for (int r0 = 0; r0 < rows; r0 += kRows) {
        if (have_i != now.i || have_r != r0) {
          const int i = min(r0 + qi, rows - 1), t = i / G, head = kh * G + i - t * G;
          simple = __all(row.open(runs, dbg::idx(p0 + t, L, dbg::kRow)));
          load_row<T, D>(q, (const char*)((const T*)x.c.Q + b * x.c.qb + head * x.c.qh + t * x.c.qt), 16u * h);
          lse = x.c.lse[((int64_t)b * x.c.H + head) * x.c.T + t] * kLog2e;
          have_i = now.i, have_r = r0;
        }
        uint32_t word = keys_word(runs, row, simple, kb, min(32, now.len - kb));
        if (r0 + qi >= rows || lse == -INFINITY) word = 0;
        if (!__any(word != 0)) continue;
        const uint32_t bits = register_bits(word, h);
        const f32x16_t sc = dot_staged<T, D>(stage + buf * kStage<T, D>, s, q);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          acc[r] += exp2_hw(keep_if_bit(fmaf(sc[r], sl2, -lse), bits, r));
      }
      keys_sum(acc, lane);
      if (writes) x.out[to] = old + acc[0];
      slot = next, found = next_found;
    }
  }
}

// bf16, many rows: a workgroup has 64 keys, whose K stays in its wavefronts'
// registers, and goes over the rows that see any of them, 128 at a time through a two-slot
// LDS ring, 32 a wavefront.  A lane forms its row's word of one of the two units.
// 512 tokens of 4 sequences of 600 .. 4096 keys, 16 heads over 4, d = 64: 35 us, 229
// TFLOP/s: two to three workgroups a CU, each with some 8 us until its first products and
// 16 stages of exponentials (16 cycles each) behind half as many cycles of products.
template <int D>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void k_weigh_tiles(
    const RowRuns* __restrict__ runs, int L, const WeighArgs x) {
  constexpr int NKS = D / 16, RB = 2 * D, CPR = RB / 16, RPL = 64 / CPR, N = kTileRows / RPL / 4;
  extern __shared__ __attribute__((aligned(16))) char ring[];
  __shared__ float sums[4][2][32];
  __shared__ int span[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qi = lane & 31, h = lane >> 5, G = x.c.group;
  // a sequence's blocks of keys in a row, so that they lie on all of the chip's dies;
  // the longest sequence first; two dimensions, since 2^32 threads in one are refused
  const int bh = blockIdx.y, kb0 = 64 * blockIdx.x;
  const int kh = bh % x.c.heads, b = by_length(x.c.lengths, x.c.B, bh / x.c.heads);
  const Chunk ch = chunk_of(x.c, L, b);
  if (ch.bad || kb0 >= ch.len) return;
  const int rows = ch.n * G, kb = kb0 + 32 * h, nk = min(32, ch.len - kb);   // of the lane's words
  // the tokens that see a key of the workgroup's: from, to
  if (threadIdx.x == 0) span[0] = ch.n, span[1] = -1;
  __syncthreads();
  int from = ch.n, to = -1;
  for (int t = threadIdx.x; t < ch.n; t += kThreads) {
    const Run* const r = runs[dbg::idx(ch.p0 + t, L, dbg::kRow)].r;
    bool sees = false;
#pragma unroll
    for (int k = 0; k < SPLAT_MAX_RUNS; ++k)
      sees = sees || (r[k].count > 0 && r[k].start < kb0 + 64 && r[k].start + r[k].stride * (r[k].count - 1) >= kb0);
    if (sees) from = min(from, t), to = max(to, t);
  }
  if (to >= 0) atomicMin(&span[0], from), atomicMax(&span[1], to);
  auto slot_of = [&](int j, bool& found) {
    const int p = page_of(x.c.pages, b, x.c.max_pages, x.c.n_pages, x.c.page_shift, j);
    found = p >= 0;
    return cache_row(max(p, 0), x.c.heads, kh, x.c.page_shift, j);
  };
  __syncthreads();
  const int s0 = span[0] * G / kTileRows, s1 = span[1] < 0 ? s0 : (span[1] * G + G - 1) / kTileRows + 1;
  // K operand: key qi of each unit, chunk 2 ks + h
  bf16x8_t ka[2][NKS];
  if (s0 < s1) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      bool found;
      const unsigned slot = slot_of(min(kb0 + 32 * e + qi, ch.len - 1), found);
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks)
        ka[e][ks] = *(const bf16x8_t*)((const char*)x.c.K + (size_t)slot * RB + 32 * ks + 16 * h);
    }
  }

  // Rows are walked without divisions: R rows further are R / G tokens and R % G heads,
  // and a token more, G heads less, where the heads run over.
  const int64_t wrap = 2 * (x.c.qt - G * x.c.qh);
  // Q: this lane's row of each load, 4 RPL rows from one to the next, through all stages
  constexpr int RS = 4 * RPL;
  int qg;
  const int qr = s0 * kTileRows + wave * RPL + lane / CPR;
  const int qtok = divide(qr, G, 1.f / G, qg);
  const char* const q0 = (const char*)((const __bf16*)x.c.Q + b * x.c.qb + kh * G * x.c.qh);
  int64_t q_at = 2 * (qtok * x.c.qt + qg * x.c.qh);
  const int q_dg = RS % G;
  const int64_t q_step = 2 * (RS / G * x.c.qt + q_dg * x.c.qh);
  auto issue = [&](int st, char* at) {     // called for s0, s0 + 1, ..
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int bk = wave + 4 * k, r = bk * RPL + lane / CPR;
      const bool in = st * kTileRows + r < rows;
      dma16(q0 + (in ? q_at : 0) + 16 * ((lane % CPR) ^ place_k<D>(r)), at + bk * kDmaBlock);
      q_at += q_step, qg += q_dg;
      if (qg >= G) qg -= G, q_at += wrap;
    }
  };
  // ... and this lane's row of the wavefront's 32 of a stage, in the mask and of lse
  struct Row {
    RowRuns rr;
    float lse;
  };
  int rg, rt = divide(min(s0 * kTileRows + 32 * wave + qi, rows - 1), G, 1.f / G, rg);
  const int r_dt = kTileRows / G, r_dg = kTileRows % G;
  const float* const lse0 = x.c.lse + ((int64_t)b * x.c.H + kh * G) * x.c.T;
  auto fetch = [&]() {                     // of s0, then of each one after
    const Row w{runs[dbg::idx(ch.p0 + rt, L, dbg::kRow)], lse0[(int64_t)rg * x.c.T + rt] * kLog2e};
    rt += r_dt, rg += r_dg;
    if (rg >= G) rg -= G, ++rt;
    if (rt >= ch.n) rt = ch.n - 1, rg = G - 1;
    return w;
  };
  auto word_of = [&](int st, const Row& w) {
    uint32_t word = 0;
    if (st * kTileRows + 32 * wave + qi >= rows || w.lse == -INFINITY || nk <= 0) return word;
#pragma unroll
    for (int k = 0; k < SPLAT_MAX_RUNS; ++k) {
      const Run& r = w.rr.r[k];
      if (r.count <= 0) continue;
      if (r.stride == 1) {
        const int lo = max(r.start - kb, 0), hi = min(r.start + r.count - 1 - kb, nk - 1);
        if (lo <= hi) word |= (~0u << lo) & (~0u >> (31 - hi));
      } else {
        word |= (uint32_t)run_tile_bits(r, kb, 1, nk);
      }
    }
    return word;
  };

  float acc[2][16];
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[e][r] = 0.f;
  const float sl2 = x.c.scale * kLog2e;
  const int koff = (32 * wave + qi) * RB + 16 * (h ^ place_k<D>(qi));
  if (s0 < s1) {
    Row w = fetch();
    uint32_t word = word_of(s0, w);
    float lse = w.lse;
    w = fetch();
    issue(s0, ring);
    ring_sync<0>();
    for (int st = s0; st < s1; ++st) {
      const char* const sq = ring + ((st - s0) & 1) * kTileRows * RB;
      // the next stage's words, and the loads of the one after, ahead of its rows'
      const uint32_t next_word = word_of(st + 1, w);
      const float next_lse = w.lse;
      w = fetch();
      if (st + 1 < s1) issue(st + 1, ring + (~(st - s0) & 1) * kTileRows * RB);
      if (__any(word != 0)) {
        const uint32_t other = __builtin_bit_cast(uint32_t, lane_xor32(__builtin_bit_cast(float, word)));
        bf16x8_t qb[NKS];
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) qb[ks] = *(const bf16x8_t*)(sq + (koff ^ (32 * ks)));
        const bool whole = __all(word == ~0u);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          f32x16_t s;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
          for (int ks = 0; ks < NKS; ++ks) s = mfma32(ka[e][ks], qb[ks], s);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], sl2, -lse);
          if (!whole) {
            const uint32_t bits = register_bits(e == h ? word : other, h);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = keep_if_bit(s[r], bits, r);
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[e][r] += exp2_hw(s[r]);
        }
      }
      word = next_word, lse = next_lse;
      ring_sync<0>();
    }
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    keys_sum(acc[e], lane);
    if ((lane & 16) == 0) sums[wave][e][key_of_lane(lane)] = acc[e][0];
  }
  __syncthreads();
  const int j = kb0 + (int)threadIdx.x;
  if (threadIdx.x >= 64 || j >= ch.len) return;
  bool found;
  const unsigned at = slot_of(j, found);
  if (!found) return;
  const int e = threadIdx.x >> 5, k = threadIdx.x & 31;
  const float old = j < ch.p0 ? x.w[at] * (ch.n > 0 ? x.decay : 1.f) : 0.f;
  x.out[at] = old + ((sums[0][e][k] + sums[1][e][k]) + (sums[2][e][k] + sums[3][e][k]));
}

template <typename T, int D>
hipError_t weigh_launch(const DevAcsr& a, const WeighArgs& x, hipStream_t st) {
  const int64_t room = std::min<int64_t>((int64_t)x.c.max_pages << x.c.page_shift, a.L);
  const WeighShape s = weigh_shape(a, sizeof(T) == 2, x.c.B, x.c.H, x.c.heads, x.c.T, D, room);
  if constexpr (sizeof(T) == 2) {
    if (s.tiles) {
      hipLaunchKernelGGL((k_weigh_tiles<D>), dim3((unsigned)((room + 63) / 64), (unsigned)(x.c.B * x.c.heads)),
                         dim3(kThreads), (2 * kTileRows * 2 * D), st, a.runs, a.L, x);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((k_weigh<T, D>), dim3((unsigned)x.c.heads, (unsigned)s.parts), dim3(kThreads),
                     (8 * kStage<T, D>), st, a.runs, a.L, x);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t allow_lds() {
  const hipError_t e = hipFuncSetAttribute(
      (const void*)k_weigh<T, D>, hipFuncAttributeMaxDynamicSharedMemorySize, 8 * kStage<T, D>);
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute((const void*)k_chunk_slices<T, D>,
                             hipFuncAttributeMaxDynamicSharedMemorySize,
                             plan_bytes(SPLAT_MAX_L) + kSliceLds<T, D>);
}

template <int D>
hipError_t allow_tiles_lds() {
  const hipError_t e = hipFuncSetAttribute(
      (const void*)k_weigh_tiles<D>, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * kTileRows * 2 * D);
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute((const void*)k_chunk_tiles<D>, hipFuncAttributeMaxDynamicSharedMemorySize,
                             plan_bytes(SPLAT_MAX_L, 2) + Ring<D>::LDS);
}

}  // namespace

hipError_t bounds_collect_chunk(uint32_t* bits, bool clear) { return dbg::collect(bits, clear); }

hipError_t prepare_chunk() {
  hipError_t e = allow_lds<float, 64>();
  if (e == hipSuccess) e = allow_lds<float, 128>();
  if (e == hipSuccess) e = allow_lds<__bf16, 64>();
  if (e == hipSuccess) e = allow_lds<__bf16, 128>();
  if (e == hipSuccess) e = allow_tiles_lds<64>();
  if (e == hipSuccess) e = allow_tiles_lds<128>();
  return e;
}

// Sizes are those of a chunk's rows, which see the keys up to their own and the chunk's newer
// ones; a few global rows of the mask (DevAcsr) do not count, 300 tokens of 24 heads under a
// symmetric window of 255 with 4 global tokens 14.8 us, 26.3 counted by the longest row.
//
// Tiles for bf16 launches of more than 32 rows a head of the cache that are more slices than
// the chip takes nearly at once, whatever their keys: d = 64, 720 slices of 14 units tiles 32.3 us,
// slices 23.7, 816 of 2 20.0 and 16.9, 984 of 4 19.7 and 24.7, 1216 of 8 24.7 and 29.8; d = 128,
// 456 of 8 23.9 and 20.6, 640 of 8 29.4 and 29.2, 768 of 4 25.6 and 31.7, 984 of 4 20.6 and 30.8.  Fewer
// slices where they are long: tiles take a third of the time a row and key, but four wavefronts
// share one block's where slices have a unit each.  d = 64, 240 slices of 58 units 32.0 and 31.5, of
// 111 39.3 and 42.6, 416 of 58 41.5 and 36.7, of 111 50.4 and 59.5; d = 128, 240 of 33 32.5 and 33.0, of 58
// 38.3 and 40.5, 416 of 33 41.6 and 34.6, of 58 48.7 and 51.7.  And of those only launches of many units in
// all: d = 64, 48 of 111 23.9 and 21.7, 96 of 111 26.7 and 28.7; d = 128, 28.5 and 27.1, 33.4 and 37.1.
//
// A block's units are shared out among as many workgroups as the chip holds beside
// each other (more would take a second turn: 4 sequences of 16 fp32 tokens, 12 heads,
// 36.7 us where 30.7 were to be had) while each wavefront keeps two units, and not
// at all where joining costs more (about what 14 units of one workgroup take): 300
// fp32 tokens of 2 sequences under a window of 256, 12 heads, 27.4 us in two
// parts, 21.2 in one.  One sequence's 32 tokens over 2048 keys, 16 heads: two units a
// wavefront 13.1 us, four 15.6, eight 20.8; 16 tokens, 32 heads over 8, 8192 keys, d = 128:
// 23.0, 21.8, 28.5.  Few short blocks, a workgroup or less a CU in all, take one unit a wavefront:
// 8 tokens of one sequence, 16 heads, d = 64, 19 units, one part / two units / one unit a
// wavefront 13.8 / 14.0 / 12.3 us in bf16, 23.2 / 17.2 / 14.2 in fp32; 14 units 12.6 / 14.1 / 12.8 and
// 20.2 / 16.7 / 14.3, 7 units 10.1 / - / 12.3 and 17.6 / - / 17.2; d = 128 in fp32, 7 units 25.2 / - / 21.9.
ChunkShape chunk_shape(const DevAcsr& a, int dtype, int B, int H, int heads, int T, int d) {
  ChunkShape s;
  const int64_t rows = (int64_t)T * (H / heads);
  const int64_t slices = (rows + kRows - 1) / kRows * B * heads;
  auto keys = [&](int of) {      // that a block of so many rows has
    return std::min<int64_t>(std::min((int64_t)a.row_keys, (int64_t)a.past_keys + T) + of, a.L);
  };
  const int64_t slice_units = (keys(kRows) + kUnit - 1) / kUnit;
  const bool is_many = slices > (d == 64 ? 900 : 640);
  const bool is_long = slice_units >= (d == 64 ? 79 : 45) && slices * slice_units > (d == 64 ? 9000 : 6000);
  s.tiles = dtype == 1 && rows > 32 && (is_many || is_long);
  const int of = s.tiles ? kTileRows : kRows;
  s.blocks = (int32_t)((rows + of - 1) / of);
  const int64_t units = (keys(of) + kUnit - 1) / kUnit;
  const int64_t groups = (int64_t)s.blocks * B * heads, slots = s.tiles && d == 64 ? 1024 : 512;
  const int64_t n = std::min({std::max<int64_t>(slots / groups, 1), (units + 7) / 8, int64_t(64)});
  s.splits = units * (n - 1) <= 14 * n ? 1 : (int32_t)n;
  const int64_t each = (units + 3) / 4;
  if (!s.tiles && each > (dtype == 1 ? 4 : d == 64 ? 2 : 1) && each <= 16 && groups * each <= 256) s.splits = (int32_t)each;
  s.cap = s.splits == 1 || B == 1 || B > 64 ? s.splits : std::min(2 * s.splits, 64);
  s.most = (int32_t)keys(of);
  return s;
}

int64_t chunk_workspace(const ChunkShape& s, int B, int H, int T, int d) {
  return s.splits == 1 ? 0 : (int64_t)B * H * T * s.cap * (d + 2);
}

// parts: what the chip holds at a time by the workgroups' LDS, and no more, so that the shares are
// even: 32 sequences' tokens, 8 heads, d = 128, with twice as many workgroups 4% more time, four times
// 16%; 128 rows of 24 heads over 4096 keys 23.9 with 21 parts, 37.5 with 22, of which some
// take a second turn; d = 64 14.2 with 42, 18.4 with 21, 20.9 with 22.
//
// tiles: from how many rows on it pays to pass them through LDS for the keys' sake depends on whether
// all blocks of 64 keys are there at a time, and else on whether the mask has most keys (blocks
// skip the rows that see none of theirs).  us, units / tiles: d = 64, 4 heads of 4096 keys, 160 rows
// 10.7 / 11.3, 192 12.0 / 11.3, 256 14.7 / 11.5; 16 heads, every key, 320 rows 22.8 / 27.5, 448 29.6 / 30.2,
// 512 33.1 / 31.1, window 256, 192 rows 16.2 / 17.1, 256 19.9 / 18.1; 16 heads of 8 sequences, every
// key, 384 rows 134 / 155, 512 174 / 172.  d = 128, 4 heads, 128 rows 11.8 / 11.4, 192 15.7 / 12.7;
// 16 heads, every key, 320 rows 31.7 / 34.3, 384 36.7 / 34.8; 24 heads, window 256, 160 rows 30.3 / 32.0, 192
// 35.1 / 32.5.
WeighShape weigh_shape(const DevAcsr& a, int dtype, int B, int H, int heads, int T, int d, int64_t room) {
  const int64_t held = (1 << 17) / (d * (dtype == 1 ? 2 : 4));
  WeighShape s;
  const int64_t rows = (int64_t)T * (H / heads), blocks = (int64_t)B * heads * ((room + 63) / 64);
  const bool at_once = blocks <= (d == 64 ? 768 : 512), most = 2 * (int64_t)a.row_keys >= room;
  s.tiles = dtype == 1 && rows >= (at_once ? (d == 64 ? 192 : 144) : most ? (d == 64 ? 448 : 352) : d == 64 ? 240 : 192);
  s.parts = std::min((room + 4 * kUnit - 1) / (4 * kUnit) * B, std::max(held / heads, int64_t(1)));
  return s;
}

hipError_t launch_chunk(const DevAcsr& a, int dtype, int d, const ChunkArgs& x, hipStream_t st) {
  if (dtype == 0)
    return d == 64 ? chunk_launch<float, 64>(a, x, st) : chunk_launch<float, 128>(a, x, st);
  return d == 64 ? chunk_launch<__bf16, 64>(a, x, st) : chunk_launch<__bf16, 128>(a, x, st);
}

hipError_t launch_weigh(const DevAcsr& a, int dtype, int d, const WeighArgs& x, hipStream_t st) {
  if (dtype == 0)
    return d == 64 ? weigh_launch<float, 64>(a, x, st) : weigh_launch<float, 128>(a, x, st);
  return d == 64 ? weigh_launch<__bf16, 64>(a, x, st) : weigh_launch<__bf16, 128>(a, x, st);
}

}  // namespace splat
