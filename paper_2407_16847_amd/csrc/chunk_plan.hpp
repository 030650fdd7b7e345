// chunk_plan.hpp -- which keys a block of consecutive mask rows needs, found by a
// workgroup in LDS from the rows' runs.
//
// Keys are counted in words of 32 (a word is a unit of work).  A dense run covers whole words,
// counted by their two ends and summed up, and leaves bits in the two at its rims; a strided run leaves
// bits.  A word is then empty, full (every row has all its keys), partial, or, with at
// most kSparseKeys bits and no whole cover, sparse.  Where that saves half of them at least,
// the sparse words' keys are gathered into units of 32.  Every workgroup plans for
// itself, some 2 us under windows: a launch for it beforehand would cost as much, and the
// lengths are not known to the host.  4 tokens over every second key of 8192 / 65536, 8 heads,
// bf16: 21 / 46 us (every key 16 / 36; strided runs by one thread each, key by key: 213 / 1760).
#pragma once

#include "../../include/splat.h"
#include "slice_ops.hpp"

namespace splat {
namespace {

constexpr int kSparseKeys = 8;
constexpr uint32_t kFullUnit = 0x8000u;

// bytes of LDS for masks of L rows: the words' bits and cover, later the gathered
// keys (or 2^sub values of the caller's a unit) and the units
__host__ __device__ constexpr int plan_words(int L) { return (L + 31) / 32; }
__host__ __device__ constexpr int plan_bytes(int L, int sub = 0) {
  return (4 * (plan_words(L) << sub) + 4 * plan_words(L) + 4 + 15) / 16 * 16;
}

struct RowsPlan {
  char* lds;
  int words, front;        // words of the key axis; 32-bit values ahead of the units
  int dense, gathered;     // units of words, keys gathered
  // nothing yet; the arrays' addresses stay in sight of the compiler as ones in LDS
  __device__ __forceinline__ RowsPlan(char* at, int L, int sub = 0)
      : lds(at), words(plan_words(L)), front(words << sub), dense(0), gathered(0) {}
  // words of the key axis, kFullUnit set on full ones; gathered keys
  __device__ __forceinline__ uint16_t* units() const { return (uint16_t*)((int*)lds + front); }
  __device__ __forceinline__ uint16_t* keys() const { return (uint16_t*)lds; }
  __device__ __forceinline__ int n() const { return dense + (gathered + kUnit - 1) / kUnit; }
};

// 64-bit sums over the workgroup's threads before this one; `all`: the total.
template <int THREADS>
__device__ __forceinline__ uint64_t sums_before(uint64_t own, uint64_t* part, uint64_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t sum = own;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up((unsigned long long)sum, o, 64);
    if (lane >= o) sum += y;
  }
  if (lane == 63) part[wave] = sum;
  __syncthreads();
  uint64_t before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) before += part[w];
    all += part[w];
  }
  return before + sum - own;
}

// Rows p0 .. p0 + nt - 1 of the mask, keys below len (0 < len <= L).  Called by the
// whole workgroup; plan.lds: plan_bytes(L); part: 2 * THREADS / 64 values.
template <int THREADS>
__device__ __forceinline__ void plan_rows(RowsPlan& plan, uint64_t* part, int L, const RowRuns* runs,
                                          int p0, int nt, int len) {
  constexpr int kMost = SPLAT_MAX_L / 32 / THREADS;     // words a thread
  const int words = plan.words, W = (len + 31) >> 5, tid = threadIdx.x;
  uint32_t* const bits = (uint32_t*)plan.lds;
  int* const cover = (int*)plan.lds + plan.front;
  for (int i = tid; i < W; i += THREADS) bits[i] = 0;
  for (int i = tid; i <= W; i += THREADS) cover[i] = 0;
  // whether any run is strided; written again behind the barrier of the first sum
  uint64_t& strided = part[2 * THREADS / 64 - 1];
  if (tid == 0) strided = 0;
  __syncthreads();
  for (int k = tid; k < nt * SPLAT_MAX_RUNS; k += THREADS) {
    const int row = dbg::idx(p0 + k / SPLAT_MAX_RUNS, L, dbg::kRow), slot = k % SPLAT_MAX_RUNS;
    const Run r = runs[row].r[slot];
    if (r.count <= 0 || r.start >= len) continue;
    if (r.stride == 1 || r.count == 1) {
      const int s = r.start, e = imin(r.start + r.count - 1, len - 1);
      const int ws = (s + 31) >> 5, we = (e + 1) >> 5;
      if (ws < we) atomicAdd(&cover[ws], 1), atomicAdd(&cover[we], -1);
      if (ws >= we && (s >> 5) == (e >> 5)) {
        atomicOr(&bits[s >> 5], (~0u << (s & 31)) & (~0u >> (31 - (e & 31))));
      } else {
        if (s & 31) atomicOr(&bits[s >> 5], ~0u << (s & 31));
        if ((e + 1) & 31) atomicOr(&bits[(e + 1) >> 5], (1u << ((e + 1) & 31)) - 1u);
      }
      continue;
    }
    strided = 1;
  }
  __syncthreads();
  // Strided runs, a word a lane: each wavefront looks 64 runs over and takes every
  // (THREADS / 64)-th 64 words of them.  A row's run that the next row's continues is that one's.
  if (strided) {
    const int lane = tid & 63, wave = tid >> 6;
    for (int k0 = 0; k0 < nt * SPLAT_MAX_RUNS; k0 += 64) {
      const int k = min(k0 + lane, nt * SPLAT_MAX_RUNS - 1);
      const int row = dbg::idx(p0 + k / SPLAT_MAX_RUNS, L, dbg::kRow), slot = k % SPLAT_MAX_RUNS;
      Run r = runs[row].r[slot];
      bool marks = k0 + lane < nt * SPLAT_MAX_RUNS && r.count > 1 && r.stride != 1 && r.start < len;
      if (marks && row + 1 < p0 + nt) {
        const Run q = runs[row + 1].r[slot];
        marks = !(q.start == r.start && q.stride == r.stride && q.count >= r.count);
      }
      int turn = wave;
      for (uint64_t left = __ballot(marks); left; left &= left - 1) {
        const int from = __builtin_ctzll(left);
        const Run run{__builtin_amdgcn_readlane(r.start, from), __builtin_amdgcn_readlane(r.stride, from),
                      __builtin_amdgcn_readlane(r.count, from), 0};
        const int w0 = run.start >> 5, n = imin(run.start + run.stride * (run.count - 1), len - 1) / 32 - w0 + 1;
        for (int b = 0; b < n; b += 64, turn = (turn + 1) % (THREADS / 64)) {
          if (turn || b + lane >= n) continue;
          const int word = w0 + b + lane;
          const uint32_t have = (uint32_t)run_tile_bits(run, 32 * word, 1, imin(32, len - 32 * word));
          if (have) atomicOr(&bits[word], have);
        }
      }
    }
    __syncthreads();
  }
  // this thread's words
  const int per = (W + THREADS - 1) / THREADS, w0 = tid * per;
  uint32_t b[kMost];
  int c[kMost], sum = 0;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const bool in = i < per && w0 + i < W;
    b[i] = in ? bits[w0 + i] : 0u;
    c[i] = in ? cover[w0 + i] : 0;
    sum += c[i];
  }
  uint64_t all;
  int covered = (int)sums_before<THREADS>((uint64_t)(int64_t)sum, part, all);
  // dense units, sparse words and their keys, 16 bits each
  uint64_t own = 0;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    covered += c[i];
    c[i] = covered;       // rows that have the whole word
    const int n = __popc(b[i]);
    if (i >= per || w0 + i >= W || (c[i] == 0 && n == 0)) {
      c[i] = -1;
    } else if (c[i] == 0 && n <= kSparseKeys) {
      c[i] = -2;
      own += (1ull << 16) + ((uint64_t)n << 32);
    } else {
      own += 1;
    }
  }
  const uint64_t before = sums_before<THREADS>(own, part + THREADS / 64, all);
  const int sparse = (int)(all >> 16 & 0xffff), keys = (int)(all >> 32);
  const bool gather = keys <= 2 * words && 2 * ((keys + kUnit - 1) / kUnit) <= sparse;
  // every thread has read its words (the barrier of the second sum): units and keys take their place
  uint16_t *const to_units = plan.units(), *const to_keys = plan.keys();
  int u = (int)(before & 0xffff) + (gather ? 0 : (int)(before >> 16 & 0xffff)), k = (int)(before >> 32);
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    if (c[i] == -1) continue;
    if (c[i] == -2 && gather) {
      for (uint32_t x = b[i]; x; x &= x - 1) to_keys[k++] = (uint16_t)(32 * (w0 + i) + __ffs((int)x) - 1);
    } else {
      to_units[u++] = (uint16_t)((w0 + i) | (c[i] == nt ? kFullUnit : 0u));
    }
  }
  __syncthreads();
  plan.dense = (int)(all & 0xffff) + (gather ? 0 : sparse);
  plan.gathered = gather ? keys : 0;
}

// A row's runs as a lane finds them, in LDS since registers are short: both ends of
// each, 16 bits apiece, and the row's number.
struct RowEnds {
  u32x4_t ends;
  int row;
  // whether all of the row's runs have stride 1
  __device__ __forceinline__ bool open(const RowRuns* runs, int at) {
    bool dense = true;
    u32x4_t e;
#pragma unroll
    for (int k = 0; k < SPLAT_MAX_RUNS; ++k) {
      const Run r = runs[at].r[k];
      dense = dense && (r.stride == 1 || r.count <= 1);
      e[k] = r.count > 0 ? (uint32_t)r.start | (uint32_t)(r.start + r.stride * (r.count - 1)) << 16 : 1u;
    }
    ends = e, row = at;
    return dense;
  }
};
static_assert(SPLAT_MAX_RUNS == 4 && SPLAT_MAX_L <= 65536, "a run's ends are 16 bits");

// The row's keys among kb .. kb + nk - 1, bit k key kb + k; simple: every run in the
// wavefront has stride 1.
__device__ __forceinline__ uint32_t keys_word(const RowRuns* runs, const RowEnds& row, bool simple,
                                              int kb, int nk) {
  uint32_t word = 0;
  if (simple) {
    const u32x4_t ends = row.ends;
#pragma unroll
    for (int k = 0; k < SPLAT_MAX_RUNS; ++k) {
      const int lo = imax((int)(ends[k] & 0xffff) - kb, 0), hi = imin((int)(ends[k] >> 16) - kb, nk - 1);
      if (lo <= hi) word |= (~0u << lo) & (~0u >> (31 - hi));
    }
  } else {
    const Run* const r = runs[row.row].r;
#pragma unroll 1
    for (int k = 0; k < SPLAT_MAX_RUNS; ++k) word |= (uint32_t)run_tile_bits(r[k], kb, 1, nk);
  }
  return word;
}

// ... of unit u
__device__ __forceinline__ uint32_t unit_word(const RowsPlan& plan, int u, const RowRuns* runs,
                                              const RowEnds& row, bool simple, int len) {
  if (u < plan.dense) {
    const uint32_t unit = plan.units()[u];
    if (unit & kFullUnit) return ~0u;
    return keys_word(runs, row, simple, 32 * unit, imin(32, len - 32 * (int)unit));
  }
  uint32_t word = 0;
  const uint16_t* const keys = plan.keys() + 32 * (u - plan.dense);
  const int n = imin(32, plan.gathered - 32 * (u - plan.dense));
#pragma unroll 1
  for (int q = 0; q < SPLAT_MAX_RUNS; ++q) {
    const Run run = runs[row.row].r[q];
    if (run.count <= 0) continue;
    const float inv = __builtin_amdgcn_rcpf((float)run.stride);
#pragma unroll 4
    for (int k = 0; k < 32; ++k) {
      const int off = keys[imin(k, n - 1)] - run.start;
      // a multiple's quotient, below 2^16, is exact to 2^-7 before it is rounded
      const int t = (int)__builtin_rintf((float)off * inv);
      word |= (uint32_t)(off >= 0 && t < run.count && t * run.stride == off) << k;
    }
  }
  return word & (~0u >> (32 - n));
}

// A word's bits (bit k: key k) in the registers' order.
__device__ __forceinline__ uint32_t register_bits(uint32_t word, int h) {
  const uint32_t x = word >> (4 * h);
  return (x & 0xf) | (x >> 4 & 0xf0) | (x >> 8 & 0xf00) | (x >> 12 & 0xf000);
}

}  // namespace
}  // namespace splat
