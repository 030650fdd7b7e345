// slice_ops.hpp -- what the kernels whose workgroup owns 32 rows share: matrix
// operands of either type, a wavefront's units of work, its view of its slice.
// (Internal linkage throughout: the index checks' flags are per kernel file.)
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "bounds.hpp"
#include "launch.hpp"
#include "mfma_util.hpp"

namespace splat {
namespace {

using namespace mfma;

constexpr int kUnit = 32;                // keys per unit

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------- operands
template <typename T, int D>
struct Mat;

// fp32: v_mfma_f32_32x32x2_f32 (fp32 products, fp32 sums)
template <int D>
struct Mat<float, D> {
  static constexpr int NB = D / 32;
  typedef typename std::conditional<NB == 2, f32x2_t, f32x4_t>::type vrow_t;
  struct Row {               // features 8 t + 4 h .. + 3 of a Q or K row
    f32x4_t v[D / 8];
  };
  struct V {                 // features NB i .. of 8 key rows: half j of a unit
    vrow_t v[8];
  };
  static __device__ __forceinline__ f32x16_t dot(const Row& k, const Row& q) {
    f32x16_t s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int t = 0; t < D / 8; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.v[t][e], q.v[t][e], s, 0, 0, 0);
    return s;
  }
  static __device__ __forceinline__ void pv(f32x16_t (&o)[NB], const V& v, const float (&p)[16],
                                            int j) {
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int b = 0; b < NB; ++b)
        o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(v.v[r][b], p[8 * j + r], o[b], 0, 0, 0);
  }
};

// bf16: v_mfma_f32_32x32x16_bf16
template <int D>
struct Mat<__bf16, D> {
  static constexpr int NB = D / 32;
  typedef typename std::conditional<NB == 2, unsigned, u32x2_t>::type vrow_t;
  struct Row {               // features 16 t + 8 h .. + 7 of a Q or K row
    bf16x8_t v[D / 16];
  };
  struct V {                 // features NB i .. of 8 key rows: half j of a unit
    vrow_t v[8];
  };
  static __device__ __forceinline__ f32x16_t dot(const Row& k, const Row& q) {
    f32x16_t s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) s = mfma32(k.v[t], q.v[t], s);
    return s;
  }
  // block b's operand of the half's k-step: element e is key row e
  static __device__ __forceinline__ bf16x8_t vt(const V& v, int b) {
    u32x4_t a;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      unsigned x, y;
      if constexpr (NB == 2) {
        x = v.v[2 * e], y = v.v[2 * e + 1];
      } else {
        x = v.v[2 * e][b >> 1], y = v.v[2 * e + 1][b >> 1];
      }
      a[e] = __builtin_amdgcn_perm(y, x, (b & 1) ? 0x07060302u : 0x05040100u);
    }
    return __builtin_bit_cast(bf16x8_t, a);
  }
  // P as a bf16 high part plus a bf16 remainder: about 16 significant bits
  static __device__ __forceinline__ void pv(f32x16_t (&o)[NB], const V& v, const float (&p)[16],
                                            int j) {
    bf16x8_t hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi[e] = (__bf16)p[8 * j + e];
      lo[e] = (__bf16)(p[8 * j + e] - (float)hi[e]);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const bf16x8_t a = vt(v, b);
      o[b] = mfma32(a, hi, o[b]);
      o[b] = mfma32(a, lo, o[b]);
    }
  }
};

// K or Q row: 16-byte chunks 2 t + h, t < D * sizeof(T) / 32
template <typename T, int D>
__device__ __forceinline__ void load_row(typename Mat<T, D>::Row& x, const char* base,
                                         unsigned off) {
  constexpr int N = D * (int)sizeof(T) / 32;
#pragma unroll
  for (int t = 0; t < N; ++t)
    x.v[t] = *(const typename std::remove_reference<decltype(x.v[0])>::type*)(base + off + 32 * t);
}

// ------------------------------------------------------------ units of work
struct Unit {
  int kb, ks, n;       // keys kb + ks * u, u < n (n <= 32)
  int mask_block;
  int half;            // which half of the tile
  int tile;            // its place among the group's tiles
  bool full;           // every key in every row of the slice
};

// Walks the slice's non-empty tiles and yields this wavefront's units.  The
// 64 lanes hold 64 tile descriptors at a time, so a unit costs no dependent
// load.
struct Units {
  const Tile* tiles;   // the group's first tile
  int nt, base, rank, lane, wave, slice;
  uint64_t left;       // non-empty tiles of the current 64 not yet visited
  int4 d;
  int mb;

  __device__ __forceinline__ void fetch() {
    d = make_int4(0, 1, 0, 0);
    mb = -1;
    if (base + lane < nt) {
      const Tile* t = tiles + base + lane;
      d = *(const int4*)t;
      mb = t->mask_block;
    }
    left = __ballot(((d.w >> (kWaveShift + 2 * slice)) & 3) != kWaveEmpty);
  }
  __device__ __forceinline__ void start(const Tile* t, int n, int lane_, int wave_, int slice_) {
    tiles = t, nt = n, base = 0, rank = 0, lane = lane_, wave = wave_, slice = slice_;
    fetch();
  }
  __device__ __forceinline__ bool next(Unit& u) {
    const int half = wave & 1;
    while (true) {
      while (left == 0) {
        base += 64;
        if (base >= nt) return false;
        fetch();
      }
      const int t = __builtin_ctzll(left);
      left &= left - 1;
      const bool mine = (rank & 1) == (wave >> 1);
      ++rank;
      const int nk = __builtin_amdgcn_readlane(d.z, t) - kUnit * half;
      if (!mine || nk <= 0) continue;
      u.ks = __builtin_amdgcn_readlane(d.y, t);
      u.kb = __builtin_amdgcn_readlane(d.x, t) + u.ks * kUnit * half;
      u.n = min(nk, kUnit);
      u.mask_block = __builtin_amdgcn_readlane(mb, t);
      u.half = half;
      u.tile = base + t;
      const int st = (__builtin_amdgcn_readlane(d.w, t) >> (kWaveShift + 2 * slice)) & 3;
      u.full = st == kWaveFull;
      return true;
    }
  }
};

// A wavefront's view of its slice.
struct Slice {
  int lane, wave, qi, h, w;    // w: the slice's place in its group
  int row, tb, nt;
  bool row_valid;
  const uint32_t* masks;       // the slice's 32-bit mask words, two per row

  // false: the slice has no row
  __device__ __forceinline__ bool open(int s, const Group* groups, const int32_t* rows,
                                       const uint64_t* m, int L) {
    const Group grp = groups[s / kWavesPerGroup];
    w = s % kWavesPerGroup;
    if (w * kWaveRows >= grp.nrows) return false;
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    qi = lane & 31, h = lane >> 5;
    const int i = w * kWaveRows + qi;
    row_valid = i < grp.nrows;
    row = row_valid ? dbg::idx(rows[grp.row_off + i], L, dbg::kRow) : 0;
    tb = grp.tile_begin, nt = grp.tile_end - grp.tile_begin;
    masks = (const uint32_t*)m + 2 * i;
    return true;
  }
  __device__ __forceinline__ bool valid() const { return row_valid; }
  // the row's membership bits in a unit
  __device__ __forceinline__ uint32_t bits(const Unit& u) const {
    return u.full ? ~0u : masks[(size_t)u.mask_block * (2 * kBM) + u.half];
  }
  __device__ __forceinline__ int key(const Unit& u, int k, int L) const {
    return dbg::idx(u.kb + u.ks * min(k, u.n - 1), L, dbg::kKey);
  }
};

// waits for this wavefront's LDS reads, and for its loads from memory
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));
  asm volatile("" ::: "memory");
}

// A unit's K rows go from memory into the wavefront's own LDS, 1 KB of whole
// rows per load, and from there into the operand: loaded straight into the
// operand, each load would touch 32 rows, 32 bytes of each, and K would hold
// registers a unit ahead (d = 128: 862 us against 631, full mask, L = 2048,
// 32 heads).  The 16-byte chunks of row r sit XOR-ed with r % 16 (128-byte rows:
// r / 2 % 8), so that the operand reads (16 lanes, 16 rows) are free of bank
// conflicts.  Keys past the unit's end re-read its last.
template <int CPR>
__device__ __forceinline__ int swz_row(int r) { return CPR == 8 ? (r >> 1) & 7 : r & 15; }
template <typename T, int D>
__device__ __forceinline__ void fetch_k(float* stage, const char* Kh, const Slice& s, const Unit& u,
                                        int L) {
  constexpr int RB = D * (int)sizeof(T), CPR = RB / 16, RPL = 64 / CPR;
  wait_lds();   // the unit before it has left the LDS rows that these loads fill
#pragma unroll
  for (int k = 0; k < kUnit / RPL; ++k) {
    const int r = RPL * k + s.lane / CPR;
    const int c = (s.lane % CPR) ^ swz_row<CPR>(r);
    dma16(Kh + ((unsigned)s.key(u, r, L) * (unsigned)RB + 16u * c), (char*)stage + kDmaBlock * k);
  }
}
// Products of 32 staged rows (fetch_k) with this lane's row: the scores' layout
// of slice_ops, lane i's row against staged rows 8 (r/4) + 4 h + r % 4.
template <typename T, int D>
__device__ __forceinline__ f32x16_t dot_staged(const char* stage, const Slice& s,
                                               const typename Mat<T, D>::Row& x) {
  constexpr int RB = D * (int)sizeof(T);
  typedef typename std::remove_reference<decltype(x.v[0])>::type vec_t;
  const int off = s.qi * RB + 16 * (s.h ^ swz_row<RB / 16>(s.qi));
  f32x16_t acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;
#pragma unroll
  for (int t = 0; t < RB / 32; ++t) {
    const vec_t a = *(const vec_t*)(stage + (off ^ (32 * t)));
    if constexpr (std::is_same<T, float>::value) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], x.v[t][e], acc, 0, 0, 0);
    } else {
      acc = mfma32(a, x.v[t], acc);
    }
  }
  return acc;
}

// The staged rows as the transposed operand: features NB i .. NB i + NB - 1 of
// rows 16 j + 8 (r/4) + 4 h + r % 4, r < 8.  The swizzle of those rows is the
// lane's (by h) XOR a constant of r.
template <typename T, int D>
__device__ __forceinline__ void load_staged(typename Mat<T, D>::V& x, const char* stage,
                                            const Slice& s, int j) {
  using vrow_t = typename Mat<T, D>::vrow_t;
  constexpr int RB = D * (int)sizeof(T), CPR = RB / 16;
  const int at = (int)sizeof(vrow_t) * s.qi;
  const int chunk = (at >> 4) ^ (CPR == 8 ? 2 * s.h : 4 * s.h);
  const int base = 4 * s.h * RB + 16 * chunk + (at & 15);
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int k = 16 * j + 8 * (r >> 2) + (r & 3);
    x.v[r] = *(const vrow_t*)(stage + ((base ^ (16 * swz_row<CPR>(k))) + k * RB));
  }
}

// column of the k-th value of a row (k < row nnz)
__device__ __forceinline__ int col_of(const RowRuns& rr, int k) {
  int j = 0;
#pragma unroll
  for (int r = 0; r < SPLAT_MAX_RUNS; ++r) {
    const Run q = rr.r[r];
    if (k >= q.prefix && k < q.prefix + q.count) j = q.start + q.stride * (k - q.prefix);
  }
  return j;
}

__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__bf16* p, float v) { *p = (__bf16)v; }

// dot product of two rows in memory
template <typename T, int D>
__device__ __forceinline__ float dense_dot(const T* a, const T* b) {
  constexpr int E = 16 / (int)sizeof(T);
  typedef typename std::conditional<E == 4, f32x4_t, bf16x8_t>::type vec_t;
  float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int c = 0; c < D; c += E) {
    const vec_t x = *(const vec_t*)(a + c), y = *(const vec_t*)(b + c);
#pragma unroll
    for (int e = 0; e < E; ++e) d[e & 3] = fmaf((float)x[e], (float)y[e], d[e & 3]);
  }
  return (d[0] + d[1]) + (d[2] + d[3]);
}

// The fused forward of row i by one wavefront: scores by lanes over 64 keys at
// a time, O by lanes over the features; only the row's own keys are read.
// lse (if not null): the row's log-sum-exp.
template <int D, typename T, typename OutT>
__device__ __forceinline__ void fused_row(int i, int lane, const RowRuns* runs,
                                          const int32_t* row_ptr, int L, const T* Qh, const T* Kh,
                                          const T* Vh, float scale, OutT* Oh, float* lse) {
  constexpr int NC = D / 64;
  const RowRuns rr = runs[i];
  const int n = row_ptr[i + 1] - row_ptr[i];
  const T* const q = Qh + (size_t)i * D;
  // m: the largest score so far, from the lowest float on: against that a score
  // of -inf weighs 0 (against -inf itself NaN).  O of a row without keys is 0 / 1,
  // of one whose keys all score -inf 0 / 0.
  float m = -__FLT_MAX__, l = n > 0 ? 0.f : 1.f, acc[NC];
#pragma unroll
  for (int b = 0; b < NC; ++b) acc[b] = 0.f;
#pragma unroll 1
  for (int k0 = 0; k0 < n; k0 += 64) {
    const bool valid = k0 + lane < n;
    int j = 0;
    float x = -INFINITY;
    if (valid) {
      j = dbg::idx(col_of(rr, k0 + lane), L, dbg::kKey);
      x = dense_dot<T, D>(q, Kh + (size_t)j * D) * scale;
    }
    const float mn = fmaxf(m, wave_max(x));
    const float alpha = expf(m - mn);
    const float p = valid ? expf(x - mn) : 0.f;
    l = l * alpha + wave_sum(p);
#pragma unroll
    for (int b = 0; b < NC; ++b) acc[b] *= alpha;
    auto key = [&](int t) {
      const float pt = __builtin_bit_cast(
          float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, p), t));
      const T* const v = Vh + (size_t)__builtin_amdgcn_readlane(j, t) * D;
#pragma unroll
      for (int b = 0; b < NC; ++b) acc[b] = fmaf(pt, (float)v[64 * b + lane], acc[b]);
    };
    const int cnt = min(64, n - k0);
    int t = 0;
#pragma unroll 1
    for (; t + 8 <= cnt; t += 8)
#pragma unroll
      for (int e = 0; e < 8; ++e) key(t + e);
#pragma unroll 1
    for (; t < cnt; ++t) key(t);
    m = mn;
  }
  if (lse && lane == 0) lse[i] = n > 0 ? m + logf(l) : -INFINITY;
  const float inv = 1.f / l;
#pragma unroll
  for (int b = 0; b < NC; ++b) store1(Oh + (size_t)i * D + 64 * b + lane, acc[b] * inv);
}

}  // namespace
}  // namespace splat
