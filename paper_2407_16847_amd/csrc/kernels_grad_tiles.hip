// kernels_grad_tiles.hip -- the backward pass in bf16 (see kernels_grad.hip for the
// mathematics).
//
// A row's query vector and dO (or a key's K and V) stay in registers as the matrix
// cores' second operand; the rows it meets are staged in LDS and taken 32 at a
// time:
//
//     scores and dP of the 32 against this lane's row      2 d/16 MFMAs 32x32x16
//     p = exp2(s sl2 - lse2), dS = p (dP - delta)          in registers
//     dQ += dS K  (or dK += dS' Q and dV += p' dO)         d/16 (or d/8) MFMAs
//
// The last products take dS (and p) straight from the registers that formed
// them, rounded to nearest even bf16 (2^-8 of each at most, as the outputs); their
// other operand is the same staged rows, read transposed.
//
// A workgroup has a group of 128 rows, 32 a wavefront, and the group's tiles pass
// through a two-slot LDS ring, the next tile's loads issued while this one is
// computed.  A launch's longest groups (global rows and columns) may instead go to
// four workgroups each, of 32 rows, whose wavefronts share out the tiles' halves:
// 1.2 to 1.6 times the work a tile, but the chain of a group's tiles takes less than
// half as long (grad_long_groups, below).
//
// Measured, dQ and dK, dV, us, in a trace of passes one after the other: window 512 +
// 64 global, L = 4096, d = 64, 64 heads 122, 166 (880 and 870 TFLOP/s of their 6 d and
// 8 d flops a non-zero; a product of 8192^3 reaches 1187); dilated 2, L = 4096, d = 128,
// 16 heads 39, 45 (620, 710); strided+local 128, L = 2048, 24 heads 15, 24, the longest
// group's chain.  Pairs below are of one run each, on a colder chip.  For 32 x
// 32 elements a SIMD has 12 (16) matrix instructions, 384 (512) cycles; 16
// exponentials, multiply-adds and products and 8 (16) conversions, 416 (448) cycles;
// and a quarter of the CU's LDS reads, 12 (24) KB a wavefront, 384 (768) cycles.
// These take turns rather than run side by side, and what was tried to change that
// did not: both halves of a tile interleaved (dK, dV 193 to 223), a third wavefront a
// SIMD for dK, dV (28 registers spilled, or 16 with V in LDS), the statistics
// spread by the matrix cores instead of read from LDS (202 for 210, 189 for 186 of
// window 512 alone), transposed reads that do not wait for the next tile (210 for 199).
#include <hip/hip_runtime.h>
#include <math.h>

#include "grad_ops.hpp"

namespace splat {
namespace {

constexpr int kThreads = 256;           // 4 wavefronts

template <int D>
struct Geo {
  static constexpr int RB = 2 * D, CPR = RB / 16;        // bytes, 16-byte chunks of a row
  static constexpr int TB = kBN * RB;                    // bytes of a staged tile
  static constexpr int RPB = kDmaBlock / RB;             // rows per load
  static constexpr int SLOT = 2 * TB + kBM * 8 + 2 * kBN * 4;   // two tiles, row masks, statistics
  static constexpr int LDS = 2 * SLOT;
  // 32 rows a workgroup: a wavefront's 32 rows of two matrices and their
  // statistics; twice where two workgroups a CU still fit
  static constexpr int UB = 32 * RB;
  static constexpr int NBUF = D == 64 ? 2 : 1;
  static constexpr int UNIT = 2 * UB + 256;
  static constexpr int LONG = 4 * NBUF * UNIT > kSumBytes<D> ? 4 * NBUF * UNIT : kSumBytes<D>;
  static constexpr int LDS_LONG = LDS > LONG + 512 ? LDS : LONG + 512;
  // dK and dV, d = 128: K and the two sums leave no registers for V, which waits
  // in LDS (VB bytes a wavefront), and the ring's slots hold half a tile
  static constexpr bool kHalves = D == 128;
  static constexpr int VB = kHalves ? 32 * RB : 0;
  static constexpr int KV_RING = kHalves ? 2 * UNIT : LDS;
  static constexpr int KV_LDS = KV_RING + 4 * VB;
  static constexpr int KV_LONG = KV_LDS > LONG + VB ? KV_LDS : LONG + VB;
  // four wavefronts' staged rows of a result (store_rows)
  static constexpr int STAGE = 4 * 32 * (RB + 16);
  static_assert(STAGE <= LDS && STAGE <= KV_LDS, "the staged results fit");
};

// Place of chunk c of row r: c ^ swz(r).  Row reads take one chunk of 16 rows at a
// time, transposed reads four chunks of four rows: the 16 rows' places of a chunk
// are all the banks (two rows of d = 64, one of d = 128, span them once), and so
// are the places of any four rows 4k .. 4k + 3 and chunks 4b .. 4b + 3.
template <int D>
__device__ __forceinline__ int swz(int r) {
  return D == 64 ? ((r >> 2) & 3) | (((r >> 1) & 1) << 2) : ((r & 3) << 2) | ((r >> 2) & 3);
}

// A lane's row and the offsets of its operand reads in 32 staged rows.  Chunk and
// block enter a swizzled place by XOR: chunk 2 ks + h of row i is at off ^ 32 ks,
// block b of a transposed read at t ^ 64 b (of rows below 8, and from 8 on).
template <int D>
struct Lane {
  int lane, wave, qi, h, place, row;
  bool ok;
  unsigned off, t[2];
  // w: which 32 rows of the group
  __device__ __forceinline__ Lane(const Group& g, const int32_t* rows, int L, int wave_, int w) {
    constexpr int RB = 2 * D;
    lane = threadIdx.x & 63, wave = wave_;
    qi = lane & 31, h = lane >> 5;
    place = w * 32 + qi;
    ok = place < g.nrows;
    row = ok ? dbg::idx(rows[g.row_off + place], L, dbg::kRow) : 0;
    off = qi * RB + 16 * (h ^ swz<D>(qi));
    // lane i of 16 addresses row 4 h + i / 4, features 16 (lane / 16 % 2) + 4 (i % 4)
    const int i = lane & 15, rv = 4 * h + (i >> 2), cl = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
#pragma unroll
    for (int e = 0; e < 2; ++e) t[e] = rv * RB + 16 * (cl ^ swz<D>(rv + 8 * e)) + 8 * (i & 1);
  }
  __device__ __forceinline__ bool valid() const { return ok; }
};

template <typename T>
__device__ __forceinline__ T lds_read(unsigned at) {
  return *(const __attribute__((address_space(3))) T*)(uintptr_t)at;
}

// The addresses of a lane's reads in the staged rows from LDS address `rows` on;
// rows further on are a constant offset away, which the read itself adds.
template <int D>
struct Reads {
  unsigned row[D / 16], t[D / 32][2];
  __device__ __forceinline__ Reads(unsigned rows, const Lane<D>& l) {
    // d = 128 has no registers to keep both slots' addresses over the loop
    if (D == 128) asm volatile("" : "+s"(rows));
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) row[ks] = (rows + l.off) ^ (32 * ks);
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int e = 0; e < 2; ++e) t[b][e] = (rows + l.t[e]) ^ (64 * b);
  }
};

// acc + products of 32 staged rows, `at` bytes on, with this lane's row: registers
// r hold rows 8 (r/4) + 4 h + r % 4.
template <int D, typename X>
__device__ __forceinline__ f32x16_t row_products(const Reads<D>& l, unsigned at, const X& x,
                                                 f32x16_t acc) {
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) acc = mfma32(lds_read<bf16x8_t>(l.row[ks] + at), x[ks], acc);
  return acc;
}

// A lane's operand kept in LDS, 16 bytes a lane side by side.
struct Parked {
  unsigned at;
  __device__ __forceinline__ bf16x8_t operator[](int ks) const {
    return lds_read<bf16x8_t>(at + 1024 * ks);
  }
};

// o[b] += the staged rows, `at` bytes on, transposed (features 32 b + lane % 32),
// times the weights.  Two 16-bit 4 x 16 transpose reads give eight rows, 16 j +
// 8 (e/4) + 4 h + e % 4, as the weights' registers have them.  (The compiler waits
// for the loads in flight to LDS before the first of an iteration's transpose
// reads: half an iteration after they were issued.)
template <int D>
__device__ __forceinline__ void add_rows(f32x16_t (&o)[D / 32], const Reads<D>& l, unsigned at,
                                         const bf16x8_t (&w)[2]) {
  typedef __attribute__((address_space(3))) i16x4_t* p_t;
  constexpr int RB = 2 * D;
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const i16x4_t lo =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((p_t)(uintptr_t)(l.t[b][0] + at + 16 * j * RB));
      const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (p_t)(uintptr_t)(l.t[b][1] + at + (16 * j + 8) * RB));
      const bf16x8_t v =
          __builtin_shufflevector(__builtin_bit_cast(bf16x4_t, lo), __builtin_bit_cast(bf16x4_t, hi),
                                  0, 1, 2, 3, 4, 5, 6, 7);
      o[b] = mfma32(v, w[j], o[b]);
    }
}

__device__ __forceinline__ f32x16_t splat16(float v) {
  f32x16_t x;
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = v;
  return x;
}

__device__ __forceinline__ void pack(const float (&w)[16], bf16x8_t (&p)[2]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    u32x4_t u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = pack_bf16_rn(w[8 * j + 2 * e], w[8 * j + 2 * e + 1]);
    p[j] = __builtin_bit_cast(bf16x8_t, u);
  }
}

// Scores outside the lane's bits of the 32 staged rows set to -inf.
__device__ __forceinline__ void mask32(f32x16_t& s, unsigned bits, int h) {
  const unsigned word = bits >> (4 * h);
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = keep_if_bit(s[r], word, 8 * (r >> 2) + (r & 3));
}

// 32 staged keys (K's and V's rows k_at and v_at bytes on) for a query row: dQ, or
// (not ADD) the sum of dS.
template <int D, bool ADD>
__device__ __forceinline__ void q_rows(const Reads<D>& l, unsigned k_at, unsigned v_at, int h,
                                       const bf16x8_t (&q)[D / 16], const bf16x8_t (&go)[D / 16],
                                       const RowStat& st, float sl2, bool partial, unsigned bits,
                                       f32x16_t (&acc)[D / 32], float& sum) {
  f32x16_t s = row_products<D>(l, k_at, q, splat16(0.f));
  const f32x16_t dp = row_products<D>(l, v_at, go, splat16(st.nd));
  if (partial) mask32(s, bits, h);
  float w[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) w[r] = exp2_hw(fmaf(s[r], sl2, -st.lse2)) * dp[r];
  if constexpr (ADD) {
    bf16x8_t p[2];
    pack(w, p);
    add_rows<D>(acc, l, k_at, p);
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r)         // 0 * inf must not reach the sum
      sum += partial ? zero_unless(w[r], bits >> (4 * h), 8 * (r >> 2) + (r & 3)) : w[r];
  }
}

// 32 staged query rows for a key: dK and dV.  stat: LDS address of the rows' lse2;
// `apart` bytes on, their -delta.  v: the key's V, from registers or Parked.  lone:
// the rows that have a single key.
template <int D, typename X>
__device__ __forceinline__ void kv_rows(const Reads<D>& l, unsigned q_at, unsigned g_at,
                                        unsigned stat, int apart, int h, const bf16x8_t (&k)[D / 16],
                                        const X& v, float sl2, bool partial,
                                        unsigned bits, unsigned lone, f32x16_t (&ak)[D / 32],
                                        f32x16_t (&av)[D / 32]) {
  f32x16_t s = row_products<D>(l, q_at, k, splat16(0.f));
  f32x16_t dp;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const f32x4_t n4 = lds_read<f32x4_t>(stat + apart + 32 * c + 16 * h);
#pragma unroll
    for (int e = 0; e < 4; ++e) dp[4 * c + e] = n4[e];
  }
  dp = row_products<D>(l, g_at, v, dp);
  if (partial) mask32(s, bits, h);
  float p[16], w[16];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const f32x4_t l4 = lds_read<f32x4_t>(stat + 32 * c + 16 * h);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * c + e;
      p[r] = exp2_hw(fmaf(s[r], sl2, -l4[e]));
      w[r] = p[r] * dp[r];
    }
  }
  if (lone)
#pragma unroll
    for (int r = 0; r < 16; ++r) w[r] = zero_unless(w[r], ~lone >> (4 * h), 8 * (r >> 2) + (r & 3));
  bf16x8_t x[2];
  pack(p, x);
  add_rows<D>(av, l, g_at, x);
  pack(w, x);
  add_rows<D>(ak, l, q_at, x);
}

template <int D>
__device__ __forceinline__ void load_operand(bf16x8_t (&x)[D / 16], const __bf16* X, int row, int h) {
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) x[ks] = *(const bf16x8_t*)(X + (size_t)row * D + ks * 16 + h * 8);
}

template <int N>
__device__ __forceinline__ void zero(f32x16_t (&a)[N]) {
#pragma unroll
  for (int b = 0; b < N; ++b) a[b] = splat16(0.f);
}

// ------------------------------------------------------------------- staging
// This wavefront's share of a tile's loads: rows of A and B, the masks of the
// group's rows where some need them and, with STAT, the tile rows' statistics.
// Rows past the tile's end re-read its last.
template <int D, bool STAT>
__device__ __forceinline__ void issue_tile(char* slot, const Tile& tl, const __bf16* A,
                                           const __bf16* B, const uint64_t* masks, const float* lse2,
                                           const float* nd, int L, int wave, int lane) {
  using G = Geo<D>;
  const int last = tl.nk - 1;
  const char* a = (const char*)(A + (size_t)tl.kb * D);
  const char* b = (const char*)(B + (size_t)tl.kb * D);
#pragma unroll
  for (int k = 0; k < G::TB / kDmaBlock / 4; ++k) {
    const int blk = wave + 4 * k;
    const int r = blk * G::RPB + lane / G::CPR;
    const int row = dbg::idx(tl.kb + tl.ks * min(r, last), L, dbg::kKey);
    const unsigned off =
        (unsigned)(row - tl.kb) * (unsigned)G::RB + 16u * ((lane % G::CPR) ^ swz<D>(r));
    dma16(a + off, slot + blk * kDmaBlock);
    dma16(b + off, slot + G::TB + blk * kDmaBlock);
  }
  if (tl.mask_block >= 0) {
    const uint64_t* m = masks + (size_t)tl.mask_block * kBM + wave * 32 + 2 * lane;
    if (lane < 16) dma16(m, slot + 2 * G::TB + wave * 256);
  }
  if (STAT && wave < 2) {
    const int row = dbg::idx(tl.kb + tl.ks * min(lane, last), L, dbg::kRow);
    dma4((wave ? nd : lse2) + row, slot + 2 * G::TB + kBM * 8 + wave * (kBN * 4));
  }
}

// A wavefront's unit of 32 rows of A and B into its own LDS; with stat (lse2 for
// lanes below 32, -delta for the others), the rows' statistics behind them.
template <int D>
__device__ __forceinline__ void issue_unit(char* to, const __bf16* A, const __bf16* B,
                                           const float* stat, const Slice& s, const Unit& u, int L) {
  using G = Geo<D>;
#pragma unroll
  for (int k = 0; k < G::UB / kDmaBlock; ++k) {
    const int r = k * G::RPB + s.lane / G::CPR;
    const size_t off = (unsigned)s.key(u, r, L) * (unsigned)G::RB + 16u * ((s.lane % G::CPR) ^ swz<D>(r));
    dma16((const char*)A + off, to + k * kDmaBlock);
    dma16((const char*)B + off, to + G::UB + k * kDmaBlock);
  }
  if (stat) dma4(stat + s.key(u, s.qi, L), to + 2 * G::UB);
}

// The ring over a group's tiles: f(slot, tile, its state for this wavefront).
template <int D, bool STAT, typename F>
__device__ __forceinline__ void for_tiles(char* lds, const Tile* tiles, int nt, const __bf16* A,
                                          const __bf16* B, const uint64_t* masks, const float* lse2,
                                          const float* nd, int L, int wave, int lane, F&& f) {
  using G = Geo<D>;
  Tile now = tiles[0], next = tiles[min(1, nt - 1)];   // read one iteration ahead
  issue_tile<D, STAT>(lds, now, A, B, masks, lse2, nd, L, wave, lane);
  ring_sync<0>();
  for (int i = 0; i < nt; ++i) {
    char* const slot = lds + (i & 1) * G::SLOT;
    const Tile tl = now;
    now = next;
    if (i + 1 < nt)
      issue_tile<D, STAT>(lds + ((i + 1) & 1) * G::SLOT, next, A, B, masks, lse2, nd, L, wave, lane);
    next = tiles[min(i + 2, nt - 1)];
    const int state = (tl.flags >> (kWaveShift + 2 * wave)) & 3;
    if (state != kWaveEmpty) f(slot, tl, state);
    // the next tile has landed, and every wavefront is done with this slot
    ring_sync<0>();
  }
}

// The ring over the halves of a group's tiles: f(slot, half, tile, state, bits of
// this lane's row in the half).  stat as issue_unit's; the row masks come straight
// to registers.
template <int D, typename F>
__device__ __forceinline__ void for_halves(char* lds, const Tile* tiles, int nt, const __bf16* A,
                                           const __bf16* B, const uint64_t* masks, const float* stat,
                                           int L, int wave, int lane, int place, F&& f) {
  using G = Geo<D>;
  constexpr int PER = G::UB / kDmaBlock / 4;    // loads of a wavefront, half tile and matrix
  auto issue = [&](const Tile& x, int e, char* slot) {
    const int last = x.nk - 1;
    const char* a = (const char*)(A + (size_t)x.kb * D);
    const char* b = (const char*)(B + (size_t)x.kb * D);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int blk = wave * PER + k, r = blk * G::RPB + lane / G::CPR;
      const int row = dbg::idx(x.kb + x.ks * min(32 * e + r, last), L, dbg::kKey);
      const unsigned off =
          (unsigned)(row - x.kb) * (unsigned)G::RB + 16u * ((lane % G::CPR) ^ swz<D>(r));
      dma16(a + off, slot + blk * kDmaBlock);
      dma16(b + off, slot + G::UB + blk * kDmaBlock);
    }
    if (wave == 0) {
      const int row = dbg::idx(x.kb + x.ks * min(32 * e + (lane & 31), last), L, dbg::kRow);
      dma4(stat + row, slot + 2 * G::UB);
    }
  };
  auto mask_of = [&](const Tile& x) {
    return x.mask_block >= 0 ? masks[(size_t)x.mask_block * kBM + place] : ~0ull;
  };
  char* const slot[2] = {lds, lds + G::UNIT};
  Tile now = tiles[0], next = tiles[min(1, nt - 1)];
  uint64_t bits = mask_of(now);
  issue(now, 0, slot[0]);
  for (int i = 0; i < nt; ++i) {
    const Tile tl = now;
    const int state = (tl.flags >> (kWaveShift + 2 * wave)) & 3;
    now = next;
    next = tiles[min(i + 2, nt - 1)];
    const uint64_t mine = bits;
    ring_sync<0>();                 // a slot has landed, the other one is free
    if (tl.nk > 32) issue(tl, 1, slot[1]);
    if (state != kWaveEmpty) f(lds_addr(slot[0]), 0, tl, state, (unsigned)mine);
    ring_sync<0>();
    if (i + 1 < nt) bits = mask_of(now), issue(now, 0, slot[0]);
    if (state != kWaveEmpty && tl.nk > 32)
      f(lds_addr(slot[1]), 1, tl, state, (unsigned)(mine >> 32));
  }
  __syncthreads();                  // LDS is used again
}

// This wavefront's units of a slice: f(their LDS address, unit, bits of this
// lane's row, lone rows).
template <int D, typename F>
__device__ __forceinline__ void for_units(char* lds, const Tile* tiles, const Slice& s, const __bf16* A,
                                          const __bf16* B, const float* stat, int L, F&& f) {
  using G = Geo<D>;
  char* const mine = lds + s.wave * G::NBUF * G::UNIT;
  Units it;
  it.start(tiles, s.nt, s.lane, s.wave, s.w);
  Unit u, nu;
  bool more = it.next(u);
  uint32_t bits = 0, lone = 0, nbits = 0, nlone = 0;
  auto issue = [&](const Unit& x, int buf) {
    nbits = s.bits(x);
    nlone = x.full || !stat ? 0u : (uint32_t)tiles[x.tile].pad[x.half];
    wait_lds();
    issue_unit<D>(mine + buf * G::UNIT, A, B, stat, s, x, L);
  };
  if (more) issue(u, 0);
  for (int buf = 0; more; u = nu) {
    wait_loads();
    bits = nbits, lone = nlone;
    more = it.next(nu);
    if (G::NBUF == 2 && more) issue(nu, buf ^ 1);
    f(lds_addr(mine + buf * G::UNIT), u, bits, lone);
    if (G::NBUF == 1 && more) issue(nu, 0);
    if (G::NBUF == 2) buf ^= 1;
  }
}

// This wavefront's 32 rows of a result (features 32 b + 8 (r/4) + 4 h + r % 4 of
// the lane's row), times f, through its part of LDS to memory as whole rows; 0 for
// rows with `none`.  Returns the rows that are not finite, which stay unwritten.
template <int D>
__device__ __forceinline__ uint64_t store_rows(char* stage, const f32x16_t (&o)[D / 32], float f,
                                               bool none, const Lane<D>& x, int nrows, __bf16* out) {
  constexpr int RS = 2 * D + 16, CPR = 2 * D / 16;   // staged row stride, chunks of a row
  float z = 0.f;
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = none ? 0.f : o[b][4 * g + e] * f;
        z = fmaf(v[e], 0.f, z);
      }
      store4<__bf16>((__bf16*)(stage + x.qi * RS + (b * 32 + g * 8 + 4 * x.h) * 2), v[0], v[1], v[2],
                     v[3]);
    }
  uint64_t bad = __ballot(x.ok && z != z);
  bad = (bad | bad >> 32) & 0xffffffffu;
  const int n = nrows - x.wave * 32;
#pragma unroll
  for (int k = 0; k < 32 * CPR / 64; ++k) {
    const int idx = k * 64 + x.lane, r = idx / CPR, c = idx % CPR;
    const int row = __shfl(x.row, r);
    const u32x4_t v = *(const u32x4_t*)(stage + r * RS + c * 16);
    if (r < n && !((bad >> r) & 1)) store16_nt((char*)(out + (size_t)row * D) + c * 16, v);
  }
  return bad;
}

// ------------------------------------------------------------------------ dQ
template <int D>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void k_grad_q_tiles(
    const Group* __restrict__ groups, const int32_t* __restrict__ rows,
    const int32_t* __restrict__ row_ptr, const RowRuns* __restrict__ runs,
    const Tile* __restrict__ tiles, const uint64_t* __restrict__ masks, int L, int BH, int n_long,
    const __bf16* __restrict__ Q, const __bf16* K, const __bf16* V, const __bf16* __restrict__ O,
    const __bf16* __restrict__ dO, const float* __restrict__ lse, float scale,
    float* __restrict__ lse2, float* __restrict__ nd, __bf16* __restrict__ dQ) {
  using G = Geo<D>;
  extern __shared__ __attribute__((aligned(256))) char lds[];
  const int item = blockIdx.x / BH, bh = blockIdx.x - item * BH;
  const bool shared = item < n_long * kWavesPerGroup;   // 32 rows for the workgroup
  const Group grp = groups[shared ? item / kWavesPerGroup : item - n_long * (kWavesPerGroup - 1)];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = shared ? item % kWavesPerGroup : wave;
  if (shared && w * kWaveRows >= grp.nrows) return;
  const Lane<D> x(grp, rows, L, wave, w);
  const size_t head = (size_t)bh * L * D, head_rows = (size_t)bh * L;
  const __bf16 *const Kh = K + head, *const Vh = V + head;
  const float sl2 = scale_size(scale);

  bf16x8_t q[D / 16], go[D / 16];
  load_operand<D>(q, Q + head, x.row, x.h);
  load_operand<D>(go, dO + head, x.row, x.h);
  times_sign(q, scale_sign(scale));
  const int keys = row_ptr[x.row + 1] - row_ptr[x.row];
  RowStat st;
  {
    bf16x8_t o[D / 16];
    load_operand<D>(o, O + head, x.row, x.h);
    float d0 = 0.f, d1 = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        d0 = fmaf((float)o[ks][e], (float)go[ks][e], d0);
        d1 = fmaf((float)o[ks][e + 1], (float)go[ks][e + 1], d1);
      }
    const float d = d0 + d1;
    st = RowStat{keys > 0 ? lse[head_rows + x.row] * kLog2e : INFINITY, -(d + lane_xor32(d))};
  }
  f32x16_t acc[D / 32];
  zero(acc);
  const Tile* const mine = tiles + grp.tile_begin;
  const int nt = grp.tile_end - grp.tile_begin;
  // see grad_ops.hpp: the tiles of rows of few keys, and whether this lane's is one
  const int few_first = nt > 0 ? mine[0].pad[0] : 0, few_tiles = nt > 0 ? mine[0].pad[1] : 0;
  const bool few = keys > 1 && keys <= kFewKeys, any_few = __any(few && x.ok);
  const bool writes = x.h == 0 && x.ok && (!shared || wave == 0);

  auto again = [&](int i, int r) {
    const RowStat y{__shfl(st.lse2, r), __shfl(st.nd, r)};
    grad_q_row<__bf16, D>(i, x.lane, runs, row_ptr, L, Q + head, Kh, Vh, dO + head, y, scale,
                          dQ + head);
  };
  if (!shared) {
    auto sweep = [&](auto add, const Tile* from, int n) {
      float sum = 0.f;
      for_tiles<D, false>(lds, from, n, Kh, Vh, masks, nullptr, nullptr, L, wave, x.lane,
                          [&](const char* slot, const Tile&, int state) {
        if (!decltype(add)::value && !any_few) return;
        uint64_t bits = ~0ull;
        if (state == kWavePartial) bits = *(const uint64_t*)(slot + 2 * G::TB + x.place * 8);
        const Reads<D> at(lds_addr(slot), x);
#pragma unroll
        for (int e = 0; e < 2; ++e)
          q_rows<D, decltype(add)::value>(at, e * G::UB, G::TB + e * G::UB, x.h, q, go, st, sl2,
                                          state == kWavePartial, (unsigned)(bits >> (32 * e)), acc,
                                          sum);
      });
      return sum + lane_xor32(sum);
    };
    if (few_tiles > 0) {
      const float sum = sweep(std::false_type(), mine + few_first, few_tiles);
      if (few) st.nd -= sum;
    }
    if (writes) lse2[head_rows + x.row] = st.lse2, nd[head_rows + x.row] = st.nd;
    if (nt > 0) sweep(std::true_type(), mine, nt);
    uint64_t bad = store_rows<D>(lds + wave * 32 * (2 * D + 16), acc, scale, keys <= 1, x, grp.nrows,
                                 dQ + head);
    for (; bad; bad &= bad - 1) {
      const int r = __builtin_ctzll(bad);
      again(__builtin_amdgcn_readlane(x.row, r), r);
    }
    return;
  }
  Slice s;
  s.lane = x.lane, s.wave = wave, s.qi = x.qi, s.h = x.h, s.w = w;
  s.masks = (const uint32_t*)masks + 2 * x.place;
  auto sweep = [&](auto add, const Tile* from, int n) {
    float sum = 0.f;
    s.nt = n;
    for_units<D>(lds, from, s, Kh, Vh, nullptr, L,
                 [&](unsigned at, const Unit& u, uint32_t bits, uint32_t) {
      q_rows<D, decltype(add)::value>(Reads<D>(at, x), 0, G::UB, x.h, q, go, st, sl2, !u.full, bits, acc, sum);
    });
    return sum + lane_xor32(sum);
  };
  if (any_few) {   // the same in all four wavefronts: they have the same rows
    float* const part = (float*)(lds + G::LONG);
    const float sum = sweep(std::false_type(), mine + few_first, few_tiles);
    if (x.h == 0) part[wave * 32 + x.qi] = sum;
    __syncthreads();
    if (few) st.nd -= (part[x.qi] + part[32 + x.qi]) + (part[64 + x.qi] + part[96 + x.qi]);
  }
  if (writes) lse2[head_rows + x.row] = st.lse2, nd[head_rows + x.row] = st.nd;
  sweep(std::true_type(), mine, nt);
  combine_rows<D, false>(lds, acc, x, scale, dQ + head,
                         [&](int i) { return row_ptr[i + 1] - row_ptr[i] > 1; }, again);
}

// ------------------------------------------------------------------ dK and dV
// The plan's roles exchanged: rows are keys, a tile is 64 query rows, whose
// statistics come with it.
template <int D>
__global__ __launch_bounds__(kThreads, 2) void k_grad_kv_tiles(
    const Group* __restrict__ groups, const int32_t* __restrict__ keys,
    const Tile* __restrict__ tiles, const uint64_t* __restrict__ masks, int L, int BH, int n_long,
    const __bf16* Q, const __bf16* __restrict__ K, const __bf16* __restrict__ V, const __bf16* dO,
    float scale, const float* lse2, const float* nd, __bf16* __restrict__ dK,
    __bf16* __restrict__ dV) {
  using G = Geo<D>;
  extern __shared__ __attribute__((aligned(256))) char lds[];
  const int item = blockIdx.x / BH, bh = blockIdx.x - item * BH;
  const bool shared = item < n_long * kWavesPerGroup;
  const Group grp = groups[shared ? item / kWavesPerGroup : item - n_long * (kWavesPerGroup - 1)];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w = shared ? item % kWavesPerGroup : wave;
  if (shared && w * kWaveRows >= grp.nrows) return;
  const Lane<D> x(grp, keys, L, wave, w);
  const size_t head = (size_t)bh * L * D, head_rows = (size_t)bh * L;
  const __bf16 *const Qh = Q + head, *const Gh = dO + head;
  const float *const l2 = lse2 + head_rows, *const ndh = nd + head_rows;
  const float sl2 = scale_size(scale);

  bf16x8_t k[D / 16], v[D / 16];
  load_operand<D>(k, K + head, x.row, x.h);
  load_operand<D>(v, V + head, x.row, x.h);
  times_sign(k, scale_sign(scale));
  // the parked V lies behind the ring, or behind the units of all wavefronts
  const unsigned parked =
      lds_addr(lds) + (shared ? G::LONG : G::KV_RING + wave * G::VB) + 16 * x.lane;
  // (Not for a group without tiles: store_rows stages all wavefronts' rows from the
  // start of LDS, past the ring, and only a ring's end has a barrier before that.)
  const int nt = grp.tile_end - grp.tile_begin;
  if (G::kHalves && nt > 0 && (!shared || wave == 0))
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      *(__attribute__((address_space(3))) bf16x8_t*)(uintptr_t)(parked + 1024 * ks) = v[ks];
  if (G::kHalves && shared) __syncthreads();
  auto v_of = [&]() -> decltype(auto) {
    if constexpr (G::kHalves) return Parked{parked};
    else return (v);
  };
  f32x16_t ak[D / 32], av[D / 32];
  zero(ak), zero(av);
  const Tile* const mine = tiles + grp.tile_begin;

  auto again_v = [&](int j, int r) {
    grad_kv_row<__bf16, D, false>(j, w * 32 + r, x.lane, mine, nt, masks, L, Qh, K + head, V + head,
                                  Gh, l2, ndh, scale, dV + head);
  };
  auto again_k = [&](int j, int r) {
    grad_kv_row<__bf16, D, true>(j, w * 32 + r, x.lane, mine, nt, masks, L, Qh, K + head, V + head,
                                 Gh, l2, ndh, scale, dK + head);
  };
  if (!shared) {
    if constexpr (G::kHalves) {
      if (nt > 0)
        for_halves<D>(lds, mine, nt, Qh, Gh, masks, x.h ? ndh : l2, L, wave, x.lane, x.place,
                      [&](unsigned at, int e, const Tile& tl, int state, unsigned bits) {
          kv_rows<D>(Reads<D>(at, x), 0, G::UB, at + 2 * G::UB, 128, x.h, k, v_of(), sl2,
                     state == kWavePartial, bits, (unsigned)tl.pad[e], ak, av);
        });
    } else if (nt > 0) {
      for_tiles<D, true>(lds, mine, nt, Qh, Gh, masks, l2, ndh, L, wave, x.lane,
                         [&](const char* slot, const Tile& tl, int state) {
        uint64_t bits = ~0ull;
        if (state == kWavePartial) bits = *(const uint64_t*)(slot + 2 * G::TB + x.place * 8);
        const Reads<D> at(lds_addr(slot), x);
        const unsigned stat = lds_addr(slot) + 2 * G::TB + kBM * 8;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          kv_rows<D>(at, e * G::UB, G::TB + e * G::UB, stat + e * 128, kBN * 4, x.h, k, v_of(),
                     sl2, state == kWavePartial, (unsigned)(bits >> (32 * e)),
                     (unsigned)tl.pad[e], ak, av);
      });
    }
    char* const stage = lds + wave * 32 * (2 * D + 16);
    uint64_t bad_v = store_rows<D>(stage, av, 1.f, false, x, grp.nrows, dV + head);
    wait_lds();
    uint64_t bad_k = store_rows<D>(stage, ak, scale, false, x, grp.nrows, dK + head);
    for (; bad_v; bad_v &= bad_v - 1) {
      const int r = __builtin_ctzll(bad_v);
      again_v(__builtin_amdgcn_readlane(x.row, r), r);
    }
    for (; bad_k; bad_k &= bad_k - 1) {
      const int r = __builtin_ctzll(bad_k);
      again_k(__builtin_amdgcn_readlane(x.row, r), r);
    }
    return;
  }
  Slice s;
  s.lane = x.lane, s.wave = wave, s.qi = x.qi, s.h = x.h, s.w = w, s.nt = nt;
  s.masks = (const uint32_t*)masks + 2 * x.place;
  for_units<D>(lds, mine, s, Qh, Gh, x.h ? ndh : l2, L,
               [&](unsigned at, const Unit& u, uint32_t bits, uint32_t lone) {
    kv_rows<D>(Reads<D>(at, x), 0, G::UB, at + 2 * G::UB, 128, x.h, k, v_of(), sl2, !u.full, bits, lone, ak, av);
  });
  auto all = [](int) { return true; };
  combine_rows<D, false>(lds, av, x, 1.f, dV + head, all, again_v);
  combine_rows<D, false>(lds, ak, x, scale, dK + head, all, again_k);
}

// ------------------------------------------------------------------ launches
template <int D>
hipError_t tiles_q(const DevAcsr& a, int BH, const BwdArgs& x, float scale, hipStream_t st) {
  float *const lse2 = x.ws, *const nd = x.ws + (size_t)BH * a.L;
  const int n = grad_long_groups(a, false, BH, D);
  hipLaunchKernelGGL((k_grad_q_tiles<D>), dim3((a.n_groups + n * (kWavesPerGroup - 1)) * BH),
                     dim3(kThreads), n ? Geo<D>::LDS_LONG : Geo<D>::LDS, st, a.groups, a.rows,
                     a.row_ptr, a.runs, a.tiles, a.masks, a.L, BH, n, (const __bf16*)x.Q,
                     (const __bf16*)x.K, (const __bf16*)x.V, (const __bf16*)x.O, (const __bf16*)x.dO,
                     x.lse, scale, lse2, nd, (__bf16*)x.dQ);
  return hipGetLastError();
}

template <int D>
hipError_t tiles_kv(const DevAcsr& a, int BH, const BwdArgs& x, float scale, hipStream_t st) {
  const float *const lse2 = x.ws, *const nd = x.ws + (size_t)BH * a.L;
  const int n = grad_long_groups(a, true, BH, D);
  hipLaunchKernelGGL((k_grad_kv_tiles<D>), dim3((a.grad_groups + n * (kWavesPerGroup - 1)) * BH),
                     dim3(kThreads), n ? Geo<D>::KV_LONG : Geo<D>::KV_LDS, st, a.grad_group, a.grad_rows,
                     a.grad_tile, a.grad_masks, a.L, BH, n, (const __bf16*)x.Q, (const __bf16*)x.K,
                     (const __bf16*)x.V, (const __bf16*)x.dO, scale, lse2, nd, (__bf16*)x.dK,
                     (__bf16*)x.dV);
  return hipGetLastError();
}

template <int D>
hipError_t allow_lds() {
  const hipError_t e = hipFuncSetAttribute((const void*)k_grad_q_tiles<D>,
                                           hipFuncAttributeMaxDynamicSharedMemorySize,
                                           Geo<D>::LDS_LONG);
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute((const void*)k_grad_kv_tiles<D>,
                             hipFuncAttributeMaxDynamicSharedMemorySize, Geo<D>::KV_LONG);
}

}  // namespace

// How many of a launch's groups, the longest, go to four workgroups each.  A
// choice takes the longest of its work at throughput, the chain of the longest
// group that one workgroup has and the chain of the longest of the others;
// microseconds a tile, measured on full masks and window + global ones.  dQ and
// dK, dV with none / the longest / all: window 512 + 64 global, L = 4096, d = 64,
// 16 heads 80, 101 / 50, 58 / 67, 75 us, 64 heads 136, 184 / 156, 186 / 245, 274;
// strided+local 128, L = 2048, 24 heads 16, 49 / -, 25 / 26, 27; dilated 2, L =
// 4096, d = 128, 16 heads 42, 48 / - / 72, 81; full, L = 777, d = 128, 16 heads 29,
// 41 / - / 24, 27.
int grad_long_groups(const DevAcsr& a, bool kv, int BH, int d) {
  struct Cost {
    double all, all_shared, chain, chain_shared;
  };
  static constexpr Cost cost[2][2] = {{{3.6e-3, 5.9e-3, 1.0, 0.42}, {8.5e-3, 10e-3, 2.1, 0.9}},
                                      {{4.6e-3, 6.8e-3, 1.3, 0.5}, {10e-3, 11.6e-3, 3.0, 1.1}}};
  const Cost& c = cost[kv][d == 128];
  const TileRun* runs = kv ? a.grad_lengths : a.lengths;
  const int n = kv ? a.n_grad_lengths : a.n_lengths;
  double rest = kv ? a.grad_tiles : a.n_tiles, longs = 0;
  double best = 0;
  int take = 0, groups = 0;
  for (int k = 0; k <= n; ++k) {
    const double work = (c.all * rest + c.all_shared * longs) * BH;
    const double chain = k < n ? c.chain * runs[k].tiles : 0;
    const double shared = k > 0 ? c.chain_shared * runs[0].tiles : 0;
    const double t = fmax(work, fmax(chain, shared));
    if (k == 0 || t < best) best = t, take = groups;
    if (k == n) break;
    const double tiles = (double)runs[k].tiles * runs[k].groups;
    rest -= tiles, longs += tiles, groups += runs[k].groups;
  }
  // the work-items of a launch stay below 2^32
  const int64_t all = kv ? a.grad_groups : a.n_groups;
  return (all + (kWavesPerGroup - 1) * (int64_t)take) * BH < (1 << 24) ? take : 0;
}

hipError_t bounds_collect_grad_tiles(uint32_t* bits, bool clear) { return dbg::collect(bits, clear); }

hipError_t prepare_bwd_tiles() {
  const hipError_t e = allow_lds<64>();
  return e == hipSuccess ? allow_lds<128>() : e;
}

hipError_t launch_grad_q_tiles(const DevAcsr& a, int BH, int d, const BwdArgs& x, float scale,
                               hipStream_t st) {
  return d == 64 ? tiles_q<64>(a, BH, x, scale, st) : tiles_q<128>(a, BH, x, scale, st);
}

hipError_t launch_grad_kv_tiles(const DevAcsr& a, int BH, int d, const BwdArgs& x, float scale,
                                hipStream_t st) {
  return d == 64 ? tiles_kv<64>(a, BH, x, scale, st) : tiles_kv<128>(a, BH, x, scale, st);
}

}  // namespace splat
