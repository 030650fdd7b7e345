// kernels_evict.hip -- a cache brought back to a budget: the keys of each head that
// gathered the most attention weight stay, in their order.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/splat.h"
#include "bounds.hpp"
#include "launch.hpp"
#include "mfma_util.hpp"
#include "serve_core.hpp"

namespace splat {
namespace {

using mfma::u32x4_t;

// ------------------------------------------------------------- which keys stay
// One workgroup per (sequence, head of the cache).  The weights, as integers in the
// same order, stay in registers; the K-th largest of them is found 8 bits at a time from
// the top, by histograms of those that agree with it so far.  Equal weights at that value
// stay from the lowest place on.  Bound by latency: pages and weights one behind the other, two
// barriers and a scan a digit, two scans for the places: 8.8 us for 4096 weights a head,
// 15 for 8192 (bit by bit, 32 counts over the workgroup: 20 and 32).
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;

// The weights' order as that of unsigned integers: a NaN is the largest, -0 is 0.
__device__ __forceinline__ uint32_t order_of(float w) {
  if (w != w) return 0xffffffffu;
  const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A row of the cache, checked against its size in a checked build.
__device__ __forceinline__ uint32_t row_of(const EvictArgs& x, int page, int h, int j) {
  return dbg::idx(cache_row(page, x.heads, h, x.page_shift, j),
                  ((uint32_t)x.n_pages * (uint32_t)x.heads) << x.page_shift, dbg::kKey);
}

// Exclusive prefix sums of n values in LDS (n <= kSelThreads), all of which
// every thread sees afterwards.
__device__ __forceinline__ void scan(int* x, int n, int* wave_sums) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int own = t < n ? x[t] : 0;
  int sum = own;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(sum, o, 64);
    if (lane >= o) sum += y;
  }
  if (lane == 63) wave_sums[wave] = sum;
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) before += w < wave ? wave_sums[w] : 0;
  if (t < n) x[t] = before + sum - own;
  __syncthreads();
}

template <int V>
__global__ __launch_bounds__(kSelThreads) void k_evict_select(const EvictArgs x) {
  __shared__ int part[V * kSelWaves], sums[kSelWaves], hist[256], found[3];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = blockIdx.x / x.heads, h = blockIdx.x - b * x.heads;
  int n = x.lengths[b];
  if (n < 0 || n > SPLAT_MAX_L || n > ((int64_t)x.max_pages << x.page_shift)) n = -1;
  if (h == 0 && tid == 0) x.left[b] = min(n, x.budget);
  int32_t* const kept = x.kept + (int64_t)blockIdx.x * x.budget;
  if (n <= x.budget) {
    for (int i = tid; i < x.budget; i += kSelThreads) kept[i] = i < n ? i : -1;
    return;
  }
  // place v * kSelThreads + tid of the sequence; the middle ones compete for `room`
  const int last = n - x.recent, room = x.budget - x.first - x.recent;
  uint32_t key[V];
  constexpr int STEP = V < 16 ? V : 16;    // pages' and weights' loads in flight
#pragma unroll
  for (int v0 = 0; v0 < V; v0 += STEP) {
    if (v0 * kSelThreads >= n) break;
    int page[STEP];
#pragma unroll
    for (int v = 0; v < STEP; ++v)
      page[v] = x.pages[(int64_t)b * x.max_pages +
                        dbg::idx(min((v0 + v) * kSelThreads + tid, n - 1) >> x.page_shift, x.max_pages, dbg::kRow)];
#pragma unroll
    for (int v = 0; v < STEP; ++v) {
      const bool ok = page[v] >= 0 && page[v] < x.n_pages;
      const int j = min((v0 + v) * kSelThreads + tid, n - 1);
      const float w = x.w[row_of(x, ok ? page[v] : 0, h, j)];
      key[v0 + v] = ok ? order_of(w) : 0;  // a place without a page goes first
    }
  }
  auto middle = [&](int v) {
    const int j = v * kSelThreads + tid;
    return j >= x.first && j < last;
  };
  // `least`: the room-th largest of the middle ones, or a value that as many reach;
  // `above`: how many surely stay; ties: more equal it than may stay
  uint32_t least = 0;
  int above = 0;
  bool ties = false;
  for (int shift = 24; room > 0 && shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (v * kSelThreads >= n) break;
      if (middle(v) && (uint64_t)(key[v] ^ least) >> (shift + 8) == 0) atomicAdd(&hist[key[v] >> shift & 255], 1);
    }
    __syncthreads();
    if (wave == 0) {                       // lane l: digits 255 - 4 l and the three below
      int c[4], own = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) c[e] = hist[255 - 4 * lane - e], own += c[e];
      int upto = own;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(upto, o, 64);
        if (lane >= o) upto += y;
      }
      int before = above + upto - own;
      if (before < room && before + own >= room)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (before < room && before + c[e] >= room) found[0] = 255 - 4 * lane - e, found[1] = before, found[2] = c[e];
          before += c[e];
        }
    }
    __syncthreads();
    least |= (uint32_t)found[0] << shift, above = found[1];
    ties = above + found[2] > room;
    if (!ties) break;                      // all that begin so stay
  }
  // places in order: 64 at a time by (v, wave)
  const uint64_t before = ((uint64_t)1 << lane) - 1;
  auto ranks = [&](auto&& takes) {
    for (int k = tid; k < V * kSelWaves; k += kSelThreads) part[k] = 0;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (v * kSelThreads >= n) break;
      const uint64_t m = __ballot(takes(v));
      if (lane == 0) part[v * kSelWaves + wave] = __popcll(m);
    }
    __syncthreads();
    scan(part, V * kSelWaves, sums);
  };
  auto equal = [&](int v) { return middle(v) && key[v] == least; };
  if (ties) ranks(equal);
  uint64_t keep = 0;        // bit v: the place stays
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (v * kSelThreads >= n) break;
    const int j = v * kSelThreads + tid;
    bool stays = middle(v) ? room > 0 && key[v] >= least : j < n;
    if (ties) {
      const int rank = part[v * kSelWaves + wave] + __popcll(__ballot(equal(v)) & before);
      stays = stays && !(equal(v) && rank >= room - above);
    }
    keep |= (uint64_t)stays << v;
  }
  __syncthreads();
  ranks([&](int v) { return (keep >> v & 1) != 0; });
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (v * kSelThreads >= n) break;
    const bool stays = keep >> v & 1;
    const int rank = part[v * kSelWaves + wave] + __popcll(__ballot(stays) & before);
    if (stays) kept[dbg::idx(rank, x.budget, dbg::kValue)] = v * kSelThreads + tid;
  }
}

// ------------------------------------------------------------ where they move
// To pages of their own: a thread has a 16-byte chunk of kMoveRows rows of K and of V.
// Bound by HBM: 4096 rows of 256 bytes of K and V, 8 heads, 16 sequences 92 us, 5.3 TB/s.
constexpr int kMoveThreads = 256, kMoveRows = 4;

template <int RB>
__global__ __launch_bounds__(kMoveThreads) void k_evict_move(const EvictArgs x) {
  constexpr int LPR = RB / 16, RPP = kMoveThreads / LPR;
  const int b = blockIdx.y / x.heads, h = blockIdx.y - b * x.heads;
  const int chunk = threadIdx.x % LPR;
  const int i0 = blockIdx.x * (RPP * kMoveRows) + threadIdx.x / LPR;
  uint32_t src[kMoveRows], dst[kMoveRows];
  bool moves[kMoveRows];
  u32x4_t k[kMoveRows], v[kMoveRows];
  float w[kMoveRows];
#pragma unroll
  for (int r = 0; r < kMoveRows; ++r) {
    const int i = i0 + r * RPP;
    const int j = i < x.budget ? x.kept[(int64_t)blockIdx.y * x.budget + i] : -1;
    const int p = j < 0 ? -1 : page_of(x.pages, b, x.max_pages, x.n_pages, x.page_shift, j);
    const int q = j < 0 ? -1 : page_of(x.to, b, x.max_to, x.n_pages, x.page_shift, i);
    moves[r] = p >= 0 && q >= 0;
    src[r] = moves[r] ? row_of(x, p, h, j) : 0;
    dst[r] = moves[r] ? row_of(x, q, h, i) : 0;
  }
#pragma unroll
  for (int r = 0; r < kMoveRows; ++r) {
    if (!moves[r]) continue;
    k[r] = *(const u32x4_t*)(x.k + (size_t)src[r] * RB + 16 * chunk);
    v[r] = *(const u32x4_t*)(x.v + (size_t)src[r] * RB + 16 * chunk);
    if (chunk == 0) w[r] = x.w[src[r]];
  }
#pragma unroll
  for (int r = 0; r < kMoveRows; ++r) {
    if (!moves[r]) continue;
    mfma::store16_nt(x.k + (size_t)dst[r] * RB + 16 * chunk, k[r]);
    mfma::store16_nt(x.v + (size_t)dst[r] * RB + 16 * chunk, v[r]);
    if (chunk == 0) x.w[dst[r]] = w[r];
  }
}

// In place: the rows' order makes a row's new place never come after its old one.  A
// workgroup has 64 bytes of every row of K or V (or the weights) of one (sequence, head) and
// takes the rows in batches: once a batch is read its places may be written, since
// what later batches read lies behind them.  16 sequences of 2000 .. 8192 tokens to 4096, 8
// heads, d = 128, bf16: 139 us with the selection, to pages of their own 116; one of
// 4096 to 2048, 16 heads, d = 64 45 us and 15: batches of 256 rows one after the other.
constexpr int kSlab = 64;

template <typename T, int LPR>
__device__ __forceinline__ void move_in_place(const EvictArgs& x, int b, int h, char* base, int RB,
                                              int at) {
  constexpr int RPP = kMoveThreads / LPR;
  const int32_t* const kept = x.kept + (int64_t)blockIdx.y * x.budget;
  const int n = x.left[b];
  for (int i0 = 0; i0 < n; i0 += RPP * kMoveRows) {
    T v[kMoveRows];
    char* to[kMoveRows];
#pragma unroll
    for (int r = 0; r < kMoveRows; ++r) {
      const int i = i0 + r * RPP + threadIdx.x / LPR;
      to[r] = nullptr;
      if (i >= n) continue;
      const int j = kept[i];
      const int p = page_of(x.pages, b, x.max_pages, x.n_pages, x.page_shift, j);
      const int q = page_of(x.pages, b, x.max_pages, x.n_pages, x.page_shift, i);
      if (j == i || p < 0 || q < 0) continue;
      v[r] = *(const T*)(base + (size_t)row_of(x, p, h, j) * RB + at);
      to[r] = base + (size_t)row_of(x, q, h, i) * RB + at;
    }
    // the whole batch is in registers before any of its places is written
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));
    asm volatile("" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kMoveRows; ++r)
      if (to[r]) *(T*)to[r] = v[r];
  }
}

__global__ __launch_bounds__(kMoveThreads) void k_evict_in_place(const EvictArgs x, int RB) {
  const int b = blockIdx.y / x.heads, h = blockIdx.y - b * x.heads;
  const int slabs = RB / kSlab, job = blockIdx.x;
  if (job == 2 * slabs) {
    move_in_place<float, 1>(x, b, h, (char*)x.w, 4, 0);
    return;
  }
  constexpr int LPR = kSlab / 16;
  move_in_place<u32x4_t, LPR>(x, b, h, job < slabs ? x.k : x.v, RB,
                              kSlab * (job % slabs) + 16 * (threadIdx.x % LPR));
}

template <int RB>
void move_launch(const EvictArgs& x, hipStream_t st) {
  constexpr int rows = kMoveThreads / (RB / 16) * kMoveRows;
  hipLaunchKernelGGL(k_evict_move<RB>, dim3((x.budget + rows - 1) / rows, x.B * x.heads),
                     dim3(kMoveThreads), 0, st, x);
}

}  // namespace

hipError_t bounds_collect_evict(uint32_t* bits, bool clear) { return dbg::collect(bits, clear); }

hipError_t launch_evict(const EvictArgs& x, int row_bytes, hipStream_t st) {
  const int64_t room = std::min<int64_t>((int64_t)x.max_pages << x.page_shift, SPLAT_MAX_L);
  auto* const select = room <= 4 * kSelThreads    ? k_evict_select<4>
                       : room <= 16 * kSelThreads ? k_evict_select<16>
                                                  : k_evict_select<SPLAT_MAX_L / kSelThreads>;
  hipLaunchKernelGGL(select, dim3(x.B * x.heads), dim3(kSelThreads), 0, st, x);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (!x.to)
    hipLaunchKernelGGL(k_evict_in_place, dim3(2 * row_bytes / kSlab + 1, x.B * x.heads),
                       dim3(kMoveThreads), 0, st, x, row_bytes);
  else if (row_bytes == 128)
    move_launch<128>(x, st);
  else if (row_bytes == 256)
    move_launch<256>(x, st);
  else
    move_launch<512>(x, st);
  return hipGetLastError();
}

}  // namespace splat
