// Attention of query tokens over the paged cache (pp_attn_forward).
//
// out = sum_j softmax_j(scale q.k_j) v_j, one pass over the keys with a running
// maximum and sum.  With few query rows per key (single tokens, groups of heads
// over one cache head) it is bound by reading K and V from device memory.
//
// A unit is 8 or 16 query rows (tokens x the heads of a group) of one sequence and
// cache head; its keys come in tiles (64 rows of 16-bit values, 32 of fp32).
// All units' tiles in a row are cut into equal runs, one per CTA, whatever the
// sequences' lengths: each CTA reads the same number of bytes, and only the host's
// launch size is known before.  A unit cut between CTAs is joined by the one that
// finishes last, in a fixed order (in two levels where it spans many CTAs).
//
// A producer warp looks up pages and has TMA copy their rows, as 128-byte
// swizzled columns, into a ring; four warps take a quarter of each tile's keys
// each: scores by mma.sync, a softmax of their own, then the product with V, and
// join at the end of a unit.  mma.sync and not tcgen05: at most 16 rows meet a
// key, and the copies set the pace.  With 16-bit values the products are
// transposed (m16n8k16: keys x rows, then values x rows), so that groups of up to
// 8 rows fill an instruction.  fp32 takes plain fp32 multiply-adds, for 2, 4 or 8
// rows: mma.sync in tf32 runs no faster on this GPU, and needs three products and
// 16 rows (48 us against 22 in the fp32 case below).
//
// Measured, of a copy rate of 6.8 TB/s: 8 sequences of 65536 keys, 32 heads of 128
// over 8 (f16) 303 us, 7.1 TB/s; 48 of up to 8192 (bf16) 143 us, 6.1 TB/s; 32 tokens
// over 32 selected pages of 64 each (bf16) 45 us, 5.9 TB/s; fp32, 16 of up to 2500, 8
// heads of 96 over 4: 22 us, 3.2 TB/s.  One sequence of 777 keys: 10 us, a chain of
// launch, lengths, page table, copy, tile and join.
//
// Over a cache in 8 bits a tile is 128 keys.  Codes are whole numbers, exact in f16, so
// all products are f16's: queries of other types are scaled by a power of two per row (bf16
// has fewer bits than f16, and fp32 comes as three f16 parts), a page's key scale goes into
// its scores, and its value scale to the 32 keys' products that a warp adds up (where pages
// are smaller the largest of their scales, and the weights of the others are less, down to
// 2^-6; pages beyond that come again as a tile of their own).  A byte becomes f16 by two
// instructions for two: placed below the exponent of 1024, and 1152 taken
// off.  At half the bytes a key the instructions count: weights are taken from the last
// maximum while they fit, 8 rows to a unit leave registers for three CTAs per SM, and what is
// rare lies behind the loop.  8 sequences of 65536 keys (f16) 168 us, 6.4 TB/s (260 at
// first); 48 of up to 8192 (bf16) 79 us, 5.5 TB/s (114); the same in fp32 93 us, three
// products where 16 bits have one; one of 777 keys 10.8 us.
//
// With a window, a unit's tiles are those of the first keys and of its rows' windows; what
// lies between is not looked up.  32 tokens over 4096 of 32768 keys and 16 first ones (bf16):
// 85 us, 6.3 TB/s.
#pragma once

#include <algorithm>
#include <cmath>

#include "attn.cuh"
#include "internal.h"

namespace ppc_row {

using namespace ppc;
using namespace ppc_ptx;
using namespace ppc_attn;

constexpr int kRows = 16;      // query rows of a unit at most
constexpr int kUp = 15;        // f16 weights are up to 2^15 (a warp's m is never behind its keys)
constexpr int kGroup = 16;     // parts of a unit joined at once
constexpr int kMaxCtas = 512;  // kGroup^2 parts and more
constexpr int kJoin = kMaxCtas / kGroup;
constexpr float kUp8 = 12.f;      // over codes, weights are up to 2^12 when m is set, and stay
constexpr float kMost8 = 32768.f; // up to this with it
constexpr float kNone = -3e38f;   // m before there is one: any weight from it is too large
constexpr float kNear = 64.f;     // pages whose value scales lie within this share a product: they have 2^-6 of f16's range at the least

// Cell: what the cache holds, T or codes of 8 bits
template <class T, class Cell, int DP, int RB>
struct Shape {
  static constexpr bool EIGHT = sizeof(Cell) == 1;
  static constexpr bool MM = EIGHT || sizeof(T) == 2;  // products by mma.sync
  static constexpr int E = sizeof(Cell);
  static constexpr int NT = EIGHT && sizeof(T) == 4 ? 3 : 1;  // f16 parts of a query
  static constexpr int R = MM ? 8 * RB : RB;    // query rows of a unit
  static constexpr int TK = EIGHT ? kTileKeys8 : MM ? 64 : 32;  // keys per tile
  static constexpr int LOG_TK = TK == 128 ? 7 : TK == 64 ? 6 : 5;
  static constexpr int WARPS = 4;               // that compute; one more copies
  static constexpr int THREADS = WARPS * 32 + 32;
  static constexpr int KW = TK / WARPS;         // keys per warp
  // A change of unit, in tiles: some 8 us under way (queries, joining, stores), of 2 a tile.  Without it CTAs that get many short
  // units are the last to end: 48 sequences of up to 8192 keys, one of them idle, took 84 us with it and 102 without.  (Not where it would
  // move the joins of calls from before it.)
  template <bool WIN>
  static constexpr int EXTRA = EIGHT ? 3 : WIN ? 2 : 0;
  static constexpr int PIECES = TK / 8;         // boxes down a tile at most (pages of 8)
  static constexpr int COL = E * DP < 128 ? 64 : 128;  // bytes of a column
  static constexpr int CH = COL / E;            // values of it
  static constexpr int NCH = DP / CH;
  static constexpr int TILE = TK * DP * E;      // bytes of a K or V tile
  static constexpr int CTAS = EIGHT && RB == 1 && NT == 1 && DP <= 128 ? 3 : DP <= 128 ? 2 : 1;
  static constexpr int QS = MM ? 0 : R * DP * 4;  // fp32 queries stay in shared memory
  static constexpr int AS = DP + 4;             // row stride of the joining buffers, free of bank conflicts
  static constexpr int NB = R <= 8 && CTAS < 3 ? 2 : 1;  // joining buffers
  static constexpr int ACC = NB * R * AS * 4;
  // as many stages as fit: with 228 KB per SM, 1 KB of it taken and 6 KB static per CTA, 190 KB are in flight (16 bits)
  static constexpr int STAGES = (233472 / CTAS - 1024 - (EIGHT ? 4096 : 6144) - 1024 - ACC - QS) / (2 * TILE);
  static constexpr int SMEM = STAGES * 2 * TILE + ACC + QS + 1024;
  static constexpr int PART = kRows * DP + 2 * kRows;  // floats of a partial result
  static_assert(!MM || NT * R * (DP + 8) * 2 <= ACC, "queries pass through the joining buffers");
};

constexpr int kMore = 2, kTurn = 4;
// Sums over codes are of values as they are.  With scales up to this none of up to 2^31 weights of 2^15 leaves fp32; where a unit of rows
// meets larger ones, its sums go on as multiples of 2^51 (the largest scales come to 2^70 then)
constexpr float kHuge = 0x1p70f, kLess = 0x1p-51f;
template <int PIECES>
struct Stage {          // what the producer says of a tile
  int have[PIECES];     // keys of each piece that the call may use
  int full;             // all of them (1); of codes also: the tile comes once more, with its other pieces (kMore); from here on the
                        // scales, and the unit's sums, are multiples of 2^51 (kTurn)
  float ks[PIECES], vs[PIECES];  // their scales, of codes
};

__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a));
}
__device__ __forceinline__ void ldsm4t(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a));
}
template <class T>
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two numbers as the type's largest ones that are no larger (of numbers from 0 on).
template <class T>
__device__ __forceinline__ uint32_t pack_down(float x, float y) {
  uint32_t r;
  if constexpr (std::is_same<T, __half>::value) asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  else asm("cvt.rz.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  return r;
}
template <class T>
constexpr float kLeast = std::is_same<T, __half>::value ? 0x1p-24f : 0x1p-126f;  // its smallest number (bf16: normal one)
// An 8 x 8 matrix of 16-bit values over the warp, two per lane, transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// Where chunk c of a key's codes lies in a tile.
template <class S>
__device__ __forceinline__ int place8(int key, int c) {
  if constexpr (S::COL == 64) return key * 64 + ((c ^ (key >> 1 & 3)) << 4);
  else return c / 8 * S::TK * 128 + key * 128 + ((c % 8 ^ (key & 7)) << 4);
}

// Walks the units' tiles in their one order (whole: in runs that end with their unit).  An item is a sequence, or a token where pages are selected for each
// token; its units are (R rows, head) pairs of kt tiles each.
struct Walk {
  int base;  // its first place in the order
  int item, t0, n, len, rows, units;
  int kt;    // tiles of a unit
  int st;    // with a window: the first st of them are the first keys'
  int span;  // places of a unit in the order: its tiles and what a change of unit costs in tiles, or whole runs of tiles
  int places;
};
template <bool WIN, int EXTRA>
__device__ __forceinline__ void load_item(const AttnParams& p, int TK, int R, int whole, int i, Walk& w) {
  w.item = i;
  int seen;
  if (p.sel) {
    const Seen s = seen_keys(i, p.T, p.B, p.starts, p.lens, p.width * p.page, p.causal, p.status);
    w.t0 = i;
    w.n = 1;
    w.len = s.keys;
    seen = min(p.keep, (s.keys + p.page - 1) >> p.log_page) << p.log_page;
  } else {
    w.t0 = p.starts ? p.starts[i] : i;
    w.n = p.starts ? p.starts[i + 1] - w.t0 : 1;
    int len = p.lens[i];
    const int most = p.width * p.page;
    if (len < 0 || len > most) {
      atomicOr(p.status, PP_CACHE_BAD_LENGTH);
      len = min(max(len, 0), most);
    }
    if (p.starts && ((i == 0 && w.t0 != 0) || (i == p.B - 1 && w.t0 + w.n != p.T))) atomicOr(p.status, PP_CACHE_BAD_LENGTH);
    if (w.t0 < 0 || w.n < 0 || w.t0 > p.T - w.n) w.n = -1;  // ranges that do not fit: the call does nothing
    w.len = len;
    seen = len;
  }
  w.rows = max(w.n, 0) * p.G.d;
  w.units = (w.rows + R - 1) / R * p.H;
  w.kt = max(1, (seen + TK - 1) / TK);
  w.st = 0;
  if (WIN) {  // a unit's tokens' windows together, wherever in a tile they begin
    const int tokens = p.causal ? min(max(w.n, 1), (R - 2) / p.G.d + 2) : 1;
    w.st = min(w.kt, (min(p.sinks, seen) + TK - 1) / TK);
    w.kt = min(w.kt, w.st + (min(p.window, seen) + tokens + TK - 3) / TK + 1);
  }
  w.span = whole ? (w.kt + whole - 1) / whole * whole : w.kt + EXTRA;
  w.places = w.units * w.span;
}

template <class T, class Cell, int DP, int RB, bool WIN>
__global__ void __launch_bounds__(Shape<T, Cell, DP, RB>::THREADS, Shape<T, Cell, DP, RB>::CTAS)
    attn_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv) {
  using S = Shape<T, Cell, DP, RB>;
  using W = std::conditional_t<S::EIGHT, __half, T>;  // of the weights
  constexpr int TK = S::TK, KW = S::KW, ST = S::STAGES, R = S::R, kWarps = S::WARPS, kThreads = S::THREADS, EX = S::template EXTRA<WIN>;
  extern __shared__ unsigned char raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  float* acc = reinterpret_cast<float*>(smem + ST * 2 * S::TILE);
  [[maybe_unused]] float* qs = acc + S::NB * R * S::AS;
  __shared__ alignas(8) uint64_t full_bar[ST], empty_bar[ST];
  __shared__ Stage<S::PIECES> stage[ST];
  __shared__ float wm[kWarps][kRows], wl[kWarps][kRows], rm[kRows], rl[kRows];
  __shared__ float wts[R][kJoin + 1], sums[R][kJoin + 1];
  __shared__ int scan[4][kThreads / 32], last_flag, dead;
  // keys with values that are not finite, a bit each: 16 from lim_min on, and 16 from the first row's window on
  __shared__ unsigned unfit;
  [[maybe_unused]] __shared__ float row_scale[kRows];
  [[maybe_unused]] __shared__ int turned[kWarps];  // where the unit ends whose sums a warp has as multiples of 2^51
  __shared__ Walk found;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const int NI = p.sel ? p.T : p.B;

  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mk) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mv) : "memory");
    dead = 0;
    for (int i = 0; i < kWarps; ++i) turned[i] = -1;
    for (int i = 0; i < ST; ++i) {
      mbar_init(su32(&full_bar[i]), S::EIGHT ? 2 : 1);  // the copies, and the scales
      mbar_init(su32(&empty_bar[i]), kWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  after_previous();
  // Every thread looks after a run of items; of few, every warp for itself, so that no warp waits for another.
  const bool small = NI <= 128;
  const int team = small ? 32 : kThreads, me = small ? lane : tid;
  const int per = (NI + team - 1) / team;
  const int i0 = min(NI, me * per), i1 = min(NI, i0 + per);
  int tiles = 0, units = 0;
  bool bad_range = false;
  Walk w;
  // what the passes below ask of an item; of up to four kept, as each load of a length waits a microsecond
  constexpr int KEEP = EX ? 4 : 1;
  int kept_kt[KEEP] = {}, kept_units[KEEP] = {};
  const bool kept = per <= KEEP;
  auto each_item = [&](auto f) {  // f(tiles of a unit, units)
    if (kept) {
#pragma unroll
      for (int j = 0; j < KEEP; ++j)
        if (i0 + j < i1) f(kept_kt[j], kept_units[j]);
    } else {
      for (int i = i0; i < i1; ++i) {
        load_item<WIN, EX>(p, TK, R, 0, i, w);
        f(w.kt, w.units);
      }
    }
  };
  auto span_of = [&](int kt, int whole) { return whole ? (kt + whole - 1) / whole * whole : kt + EX; };
  if (kept) {
#pragma unroll
    for (int j = 0; j < KEEP; ++j)
      if (i0 + j < i1) {
        load_item<WIN, EX>(p, TK, R, 0, i0 + j, w);
        kept_kt[j] = w.kt;
        kept_units[j] = w.units;
        bad_range = bad_range || w.n < 0;
      }
    each_item([&](int kt, int n) {
      tiles += n * (kt + EX);
      units += n;
    });
  } else {
    for (int i = i0; i < i1; ++i) {
      load_item<WIN, EX>(p, TK, R, 0, i, w);
      tiles += w.places;
      units += w.units;
      bad_range = bad_range || w.n < 0;
    }
  }
  const int grid = gridDim.x;
  // sums of N numbers over the team
  auto sums_of = [&](auto& v) {
    constexpr int N = sizeof(v) / sizeof(int);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __reduce_add_sync(~0u, v[i]);
    if (small) return;
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) scan[i][warp] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0;
#pragma unroll
      for (int j = 0; j < kThreads / 32; ++j) v[i] += scan[i][j];
    }
    __syncthreads();
  };
  int all[3] = {tiles, units, bad_range};
  sums_of(all);
  if (all[2]) {
    if (tid == 0) atomicOr(p.status, PP_CACHE_BAD_LENGTH);
    return;
  }
  // Equal runs; one of a single tile (but of 128 keys) would spend more on joining than on its keys.  Where every unit can have CTAs of its
  // own with runs not much longer (up to 1.4 times, which the copies of the other CTAs make up for), runs end with
  // their unit: a CTA that changes units waits some 3 us for queries, joining and stores.
  int run = max((all[0] + grid - 1) / grid, TK == 128 ? 1 : 2), whole = 0;
  if (all[1] <= grid) {
    const int own = max(run - EX, 1), longer[4] = {own, own + own / 10 + 1, own + own / 4 + 1, own + own * 2 / 5 + 2};
    int ctas[4] = {};
    each_item([&](int kt, int n) {
#pragma unroll
      for (int j = 0; j < 4; ++j) ctas[j] += n * ((kt + longer[j] - 1) / longer[j]);
    });
    sums_of(ctas);
#pragma unroll
    for (int j = 3; j >= 0; --j)
      if (ctas[j] <= grid && (int64_t)longer[j] * grid <= INT32_MAX) whole = longer[j];  // places are counted in 32 bits
    if (whole) run = whole;
  }
  // a scan places the items in the one order
  int mine = 0;
  each_item([&](int kt, int n) { mine += n * span_of(kt, whole); });
  int before = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int up = __shfl_up_sync(~0u, before, d);
    if (lane >= d) before += up;
  }
  int total = __shfl_sync(~0u, before, 31);
  if (!small) {
    if (lane == 31) scan[0][warp] = before;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) {
      if (i < warp) before += scan[0][i];
      total += scan[0][i];
    }
  }
  before -= mine;
  if ((int64_t)blockIdx.x * run >= total) return;
  const int x0 = blockIdx.x * run, x1 = x0 + min(total - x0, run);
  const bool has = x0 >= before && x0 < before + mine;
  if (has) {
    for (int i = i0;; ++i) {
      if (per > 1) {
        load_item<WIN, EX>(p, TK, R, whole, i, w);
      } else {
        w.span = span_of(w.kt, whole);
        w.places = w.units * w.span;
      }
      if (x0 < before + w.places) break;
      before += w.places;
    }
    w.base = before;
    if (!small) found = w;
  }
  if (small) {
    const int from = __ffs(__ballot_sync(~0u, has)) - 1;
    w.base = __shfl_sync(~0u, w.base, from);
    w.item = __shfl_sync(~0u, w.item, from);
    w.t0 = __shfl_sync(~0u, w.t0, from);
    w.n = __shfl_sync(~0u, w.n, from);
    w.len = __shfl_sync(~0u, w.len, from);
    w.rows = __shfl_sync(~0u, w.rows, from);
    w.units = __shfl_sync(~0u, w.units, from);
    w.kt = __shfl_sync(~0u, w.kt, from);
    w.st = __shfl_sync(~0u, w.st, from);
    w.span = __shfl_sync(~0u, w.span, from);
    w.places = __shfl_sync(~0u, w.places, from);
  }
  __syncthreads();  // the barriers are set up, too
  if (!small) w = found;
  const int log_br = min(p.log_page, S::LOG_TK), BR = 1 << log_br, pieces = TK >> log_br;
  const float sl = p.scale * 1.44269504f;  // softmax in powers of two

  // the unit at x: its rows, head and tiles up to this CTA's end
  auto settle = [&](int x) {
    while (x - w.base >= w.places) {
      const int b = w.base + w.places;
      load_item<WIN, EX>(p, TK, R, whole, w.item + 1, w);
      w.base = b;
    }
  };

  // keys that row r of w's rows may see; with a window, how many tiles lie between a unit's first keys and its window's first
  auto limit_of = [&](int r) {
    return p.causal && !p.sel ? min(w.len, max(0, w.len - w.n + p.G.div(r) + 1)) : w.len;
  };
  auto gap_of = [&](int r0) { return max(0, (max(0, limit_of(r0) - p.window) >> S::LOG_TK) - w.st); };

  if (warp == kWarps) {
    // ---- producer.  Pages are looked up 32 pieces at a time, a lane each, so that the latency of the lists and tables
    // is paid once in 32 / pieces tiles
    int s = 0;
    uint32_t ph = 1;  // an empty ring
    const int log_pc = S::LOG_TK - log_br;
    for (int x = x0; x < x1;) {
      settle(x);
      const int u = (x - w.base) / w.span, h = p.by_head.mod(u);
      const int k0 = x - w.base - u * w.span, next = x + min(w.span - k0, x1 - x), k1 = min(w.kt, k0 + next - x);
      if (EX && k0 >= k1) {  // no tiles of it
        x = next;
        continue;
      }
      const int b = p.sel ? seen_keys(w.t0, p.T, p.B, p.starts, p.lens, p.width * p.page, p.causal, p.status).b : w.item;
      const int* row = p.table + (int64_t)b * p.width;
      const int* list = p.sel ? p.sel + ((int64_t)w.t0 * p.H + h) * p.keep : nullptr;
      int gap = 0, end = w.len, low = 0;  // with a window: the unit's keys end and begin here
      if (WIN) {
        const int r0 = p.by_head.div(u) * R;
        gap = gap_of(r0);
        end = limit_of(min(r0 + R, w.rows) - 1);
        low = limit_of(r0) - p.window;
      }
      int have32 = 0, y32 = 0;
      [[maybe_unused]] bool huge = false;
      [[maybe_unused]] float ks32 = 0.f, vs32 = 0.f;
      for (int k = k0; k < k1; ++k) {
        const int in32 = (k - k0) << log_pc & 31;  // the tile's first piece among the 32
        if (in32 == 0) {
          have32 = 0;
          ks32 = vs32 = 0.f;
          // key of the sequence, or of the list's pages in a row
          int64_t key = (int64_t)k * TK + lane * BR;
          bool some = key < (int64_t)k1 * TK;
          if (WIN) {
            if (k + (lane * BR >> S::LOG_TK) >= w.st) key += (int64_t)gap * TK;
            some = some && (key < p.sinks || key + BR > low);
          }
          if (some) {
            const int off = (int)key & (p.page - 1);
            int at = (int)(key >> p.log_page);
            bool ok = true;
            if (list) {
              ok = at < p.keep;
              at = ok ? list[at] : -1;
              if (at >= p.width) atomicOr(p.status, PP_CACHE_BAD_PAGE);
              ok = at >= 0 && at < p.width;
            }
            have32 = ok ? max(0, min(BR, end - at * p.page - off)) : 0;
            if (have32 > 0) {
              const int id = row[at];
              if (id < 0 || id >= p.pages) {
                atomicOr(p.status, PP_CACHE_BAD_PAGE);
                have32 = 0;
              }
              y32 = (int)(((int64_t)id * p.H + h) * p.page) + off;
              if constexpr (S::EIGHT) {  // on their way while the copies are
                if (have32 > 0) {
                  ks32 = p.ks[(int64_t)id * p.H + h];
                  vs32 = p.vs[(int64_t)id * p.H + h];
                }
              }
            }
          }
        }
        const int have = __shfl_sync(~0u, have32, in32 + (lane & pieces - 1));
        const int y = __shfl_sync(~0u, y32, in32 + (lane & pieces - 1));
        // The pieces that the stage has: all that are there; over codes those of similar value scales (as their products share one,
        // and a row may not see, or hardly, the page that has the largest), and the others in stages of their own behind it
        unsigned live = __ballot_sync(~0u, lane < pieces && have > 0);
        bool whole = __all_sync(~0u, have == BR), again;
        do {
          again = false;
          if (!*(volatile int*)&dead && !wait(su32(&empty_bar[s]), ph)) dead = 1;
          __syncwarp();
          const bool go = !*(volatile int*)&dead;
          if constexpr (!S::EIGHT) {
            if (lane < pieces) stage[s].have[lane] = have;
            if (lane == 0) stage[s].full = whole;
            __syncwarp();
          }
          if (lane == 0) mbar_arrive_expect_tx(su32(&full_bar[s]), go ? __popc(live) * 2 * BR * DP * S::E : 0);
          __syncwarp();
          const uint32_t dst = su32(smem + s * 2 * S::TILE);
          const int boxes = pieces * S::NCH * 2, j = lane & pieces - 1;  // box i: piece i % pieces, column and pool i / pieces
          for (int i = lane; i < boxes; i += 32) {
            const int c = (i >> log_pc) % S::NCH, v = (i >> log_pc) / S::NCH;
            if (go && (live >> j & 1))
              copy_box(dst + v * S::TILE + c * TK * S::COL + j * BR * S::COL, v ? &mv : &mk, c * S::CH, y, su32(&full_bar[s]));
          }
          if constexpr (S::EIGHT) {
            const float ks = __shfl_sync(~0u, ks32, in32 + (lane & pieces - 1)), all = __shfl_sync(~0u, vs32, in32 + (lane & pieces - 1));
            const bool turn = !huge && __any_sync(~0u, all > kHuge);
            huge = huge || turn;
            const float vs = huge ? all * kLess : all;
            bool taken = live >> j & 1;  // with the largest scale among its warp's keys that no stage has had
            if (BR < S::KW) {
              float top = taken ? fabsf(vs) : 0.f;
              for (int d = 1; BR * d < S::KW; d <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
              taken = taken && (vs == 0.f || !(fabsf(vs) * kNear < top));  // the largest at the least, whatever the scales hold
              live &= ~__ballot_sync(~0u, taken);
              again = (live & ((1u << pieces) - 1)) != 0;
            }
            if (lane < pieces) {
              stage[s].have[lane] = taken ? have : 0;
              stage[s].ks[lane] = ks;
              stage[s].vs[lane] = taken ? vs : 0.f;
            }
            if (lane == 0) stage[s].full = (again ? kMore : whole) | (turn ? kTurn : 0);
            __syncwarp();
            if (lane == 0) mbar_arrive(su32(&full_bar[s]));
          }
          __syncwarp();
          if (++s == ST) {
            s = 0;
            ph ^= 1;
          }
          whole = false;
        } while (S::EIGHT && again);
      }
      x = next;
    }
    if (p.sel && p.starts && blockIdx.x == 0) check_ranges(p.starts, p.T, p.B, lane, 32, p.status);
    return;
  }

  // ---- consumers
  // A lane's sums: mma, values i * 16 + g, + 8 (of codes, 2g, + 1) of rows 8 rb + 2t, + 1 (o[rb][i]); fp32, four values from (lane + 32 i) * 4
  // on of every row (o[r][i]).
  constexpr int NO = S::MM ? DP / 16 : (DP + 127) / 128, OB = S::MM ? RB : R, NR = S::MM ? 2 * RB : R;
  const int g = lane / 4, t = lane % 4;
  // the r-th of the lane's NR rows
  auto row_of = [&](int r) { return S::MM ? (r >> 1) * 8 + 2 * t + (r & 1) : r; };
  const T* q = static_cast<const T*>(p.q);
  [[maybe_unused]] const bool q16 = ((reinterpret_cast<uintptr_t>(q) & 15) | (p.q_ts & (sizeof(T) == 4 ? 3 : 7)) | (p.q_hs & (sizeof(T) == 4 ? 3 : 7))) == 0;
  int s = 0;
  uint32_t ph = 0;
  bool timed_out = false;
  for (int x = x0; x < x1;) {
    settle(x);
    const int u = (x - w.base) / w.span, h = p.by_head.mod(u), r0 = p.by_head.div(u) * R;
    const int k0 = x - w.base - u * w.span, next = x + min(w.span - k0, x1 - x), k1 = min(w.kt, k0 + next - x);
    if (EX && k0 >= k1) {
      x = next;
      continue;
    }
    const int nrows = min(R, w.rows - r0);
    const bool listed = p.sel != nullptr;
    // keys that a row of the unit may see
    auto limit = [&](int r) { return limit_of(r0 + r); };
    const int gap = WIN ? gap_of(r0) : 0;
    int lim[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) lim[r] = limit(min(row_of(r), nrows - 1));
    const int lim_min = limit(0), lim_max = limit(nrows - 1);
    // the row's queries: token r / G of the unit's, head r % G of the group's
    auto qrow = [&](int r) {
      return q + (w.t0 + p.G.div(r0 + r)) * p.q_ts + (int64_t)(h * p.G.d + p.G.mod(r0 + r)) * p.q_hs;
    };
    [[maybe_unused]] uint32_t qf[S::NT][S::MM ? RB : 1][S::MM ? DP / 16 : 1][2];
    [[maybe_unused]] float slr[NR];  // of codes: softmax in powers of two and the row's own power
    if (tid == 0) unfit = 0;
    if constexpr (S::EIGHT) {
      // a row is DP / 8 lanes of one warp; f16 as it is, others times a power of two that brings the row's largest to 2^14
      __half* stage_q = reinterpret_cast<__half*>(acc);
      constexpr int L = DP / 8;
#pragma unroll 1
      for (int i = tid; i < R * L; i += kWarps * 32) {
        const int r = i / L, d = i % L * 8;
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = 0.f;
        if (r < nrows && d < p.D) {
          const T* from = qrow(r) + d;
          if (q16) {
            constexpr int V = 16 / sizeof(T);
#pragma unroll
            for (int e = 0; e < 8; e += V) {
              const Vec<T, V> v = *reinterpret_cast<const Vec<T, V>*>(from + e);
#pragma unroll
              for (int j = 0; j < V; ++j) f[e + j] = to_f32(v.v[j]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = to_f32(from[e]);
          }
        }
        float up = 1.f, back = 1.f;
        if constexpr (!std::is_same<T, __half>::value) {
          int top = 0;  // the largest exponent, of infinities and NaN the largest finite one
#pragma unroll
          for (int e = 0; e < 8; ++e) top = max(top, min(__float_as_int(fabsf(f[e])) >> 23, 254));
#pragma unroll
          for (int m = 1; m < L; m <<= 1) top = max(top, __shfl_xor_sync(~0u, top, m));
          top = max(top, 16);  // rows below 2^-111 keep fewer bits
          up = __int_as_float((127 + 14 + 127 - top) << 23);
          back = __int_as_float((top - 14) << 23);
        }
        if (i % L == 0) row_scale[r] = back;
#pragma unroll
        for (int n = 0; n < S::NT; ++n) {
          Vec<__half, 8> y;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float z = n == 0 ? f[e] * up : f[e];
            y.v[e] = __float2half_rn(z);
            f[e] = z - __half2float(y.v[e]);
          }
          *reinterpret_cast<Vec<__half, 8>*>(stage_q + (n * R + r) * (DP + 8) + d) = y;
        }
      }
      group_sync<kWarps * 32>();
#pragma unroll
      for (int n = 0; n < S::NT; ++n)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int kk = 0; kk < DP / 16; ++kk) {
            const uint2 v = *reinterpret_cast<const uint2*>(stage_q + (n * R + rb * 8 + g) * (DP + 8) + kk * 16 + 4 * t);
            qf[n][rb][kk][0] = v.x;
            qf[n][rb][kk][1] = v.y;
          }
#pragma unroll
      for (int r = 0; r < NR; ++r) slr[r] = sl * row_scale[row_of(r)];
      group_sync<kWarps * 32>();
    } else if constexpr (S::MM) {
      // through the joining buffer, free here, so that each value is read once and 16 bytes at a time where they lie so
      T* stage_q = reinterpret_cast<T*>(acc);
      for (int i = tid; i < R * (DP / 8); i += kWarps * 32) {
        const int r = i / (DP / 8), d = i % (DP / 8) * 8;
        Vec<T, 8> v = {};
        if (r < nrows && d < p.D) {
          const T* from = qrow(r) + d;
          if (q16) {
            v = *reinterpret_cast<const Vec<T, 8>*>(from);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v.v[e] = from[e];
          }
        }
        *reinterpret_cast<Vec<T, 8>*>(stage_q + r * (DP + 8) + d) = v;
      }
      group_sync<kWarps * 32>();
      // matrices of 8 rows x 8 values, four at a time: b0, b1 of two steps
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const uint32_t at = su32(stage_q + (rb * 8 + lane % 8) * (DP + 8) + lane / 8 * 8);
#pragma unroll
        for (int kk = 0; kk < DP / 16; kk += 2) {
          uint32_t f[4];
          ldsm4(at + kk * 32, f);
          qf[0][rb][kk][0] = f[0];
          qf[0][rb][kk][1] = f[1];
          qf[0][rb][kk + 1][0] = f[2];
          qf[0][rb][kk + 1][1] = f[3];
        }
      }
      group_sync<kWarps * 32>();
    } else {
      group_sync<kWarps * 32>();  // the last unit's are read
      for (int i = tid; i < R * DP; i += kWarps * 32) {
        const int r = i / DP, d = i % DP;
        qs[i] = r < nrows && d < p.D ? to_f32(qrow(r)[d]) : 0.f;
      }
      group_sync<kWarps * 32>();
    }
    float o[OB][NO][4];
#pragma unroll
    for (int rb = 0; rb < OB; ++rb)
#pragma unroll
      for (int i = 0; i < NO; ++i) o[rb][i][0] = o[rb][i][1] = o[rb][i][2] = o[rb][i][3] = 0.f;
    float m[NR], l[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      m[r] = S::EIGHT ? kNone : -INFINITY;
      l[r] = 0.f;
    }

    for (int k = k0; k < k1;) {
      if (!*(volatile int*)&dead && !wait(su32(&full_bar[s]), ph)) dead = 1;
      __syncwarp();
      timed_out = timed_out || *(volatile int*)&dead;
      const uint32_t kt = su32(smem + s * 2 * S::TILE), vt = kt + S::TILE;
      const Stage<S::PIECES>& sg = stage[s];
      const int from = (WIN && k >= w.st ? k + gap : k) * TK;  // the tile's first key
      k += S::EIGHT && !timed_out ? !(sg.full & kMore) : 1;
      const bool clean = (S::EIGHT ? sg.full & 1 : sg.full) && (listed || (from + TK <= lim_min && (!WIN || from >= lim_max - p.window || from + TK <= p.sinks)));
      // a key of the tile that row r of the lane's may not use; keys whose values have to be 0, as no row uses them
      auto hidden = [&](int j, int r) {
        return (j & (BR - 1)) >= sg.have[j >> log_br] || (!listed && from + j >= lim[r]) ||
               (WIN && from + j < lim[r] - p.window && from + j >= p.sinks);
      };
      if (!S::EIGHT && !clean) {  // 0 x the values that a row does not see has to be 0
#pragma unroll
        for (int i = 0; i < KW; ++i) {
          const int j = warp * KW + i;
          unsigned char* v = smem + s * 2 * S::TILE + S::TILE + j * 128;
          const int key = from + j;
          const bool edge = WIN && key < lim_max - p.window && key >= p.sinks;  // before some rows' windows
          bool zero = (j & (BR - 1)) >= sg.have[j >> log_br] || (!listed && key >= lim_max) || (edge && key < lim_min - p.window);
          if (!zero && !listed && (key >= lim_min || edge)) {  // some rows see it
            for (int c = lane; c < S::NCH * 8; c += 32)
              zero = zero || not_finite<T>(*reinterpret_cast<const uint4*>(v + c / 8 * TK * 128 + c % 8 * 16));
            zero = __any_sync(~0u, zero);
            if (zero && lane == 0) atomicOr(&unfit, 1u << (key >= lim_min ? key - lim_min : 16 + key - (lim_min - p.window)));
          }
          if (zero)
            for (int c = lane; c < S::NCH * 8; c += 32) *reinterpret_cast<uint4*>(v + c / 8 * TK * 128 + c % 8 * 16) = make_uint4(0, 0, 0, 0);
        }
        __syncwarp();
      }
      float f[NR];
      bool moved = false;
      // row r's m after keys of up to mx, the factor of what came before it, and where exponents are taken from
      auto raise = [&](int r, float mx) {
        mx = fmaxf(m[r], lower(mx, kLift<W, kUp>));
        const float at = mx == -INFINITY ? 0.f : mx;
        f[r] = ex2(m[r] - at);
        moved = moved || m[r] != mx;
        m[r] = mx;
        return at;
      };
      if constexpr (S::EIGHT) {
        // ---- scores of this warp's keys, 16 at a time: sc[.][rb] is keys g (0, 1) and g + 8 (2, 3) by the lane's two rows
        constexpr int SL = KW / 16;
        float sc[SL][RB][4] = {}, x[SL][RB][4];
        float ks[SL][2], vs[SL][2];  // scales of keys g and g + 8
#pragma unroll
        for (int z = 0; z < SL; ++z) {
          const int slab = warp * KW + 16 * z, key = slab + lane % 16;
#pragma unroll
          for (int kk = 0; kk < DP / 16; kk += 2) {  // 16 values of a key are a chunk of 16 bytes: two at a time
            uint32_t c[4], a[4];
            ldsm4(kt + place8<S>(key, kk + lane / 16), c);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              f16_in_order(c[2 * i], a[0], a[2]);
              f16_in_order(c[2 * i + 1], a[1], a[3]);
#pragma unroll
              for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int n = S::NT - 1; n >= 0; --n) mma16<W>(sc[z][rb], a, qf[n][rb][kk + i][0], qf[n][rb][kk + i][1]);
            }
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            ks[z][i] = sg.ks[slab + 8 * i >> log_br];
            vs[z][i] = sg.vs[slab + 8 * i >> log_br];
          }
        }
        auto masked = [&](int z, int rb, int e) { return !clean && hidden(warp * KW + 16 * z + g + 8 * (e >> 1), 2 * rb + (e & 1)); };
        // ---- softmax over what this warp has seen: with m as it is, and only where a weight would leave f16 once more with the
        // scores' maximum looked for and m 2^12 below it (each step rounded by itself there, as the maximum's are)
        float top = 0.f;
#pragma unroll
        for (int z = 0; z < SL; ++z)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int r = 2 * rb + (e & 1);
              x[z][rb][e] = fmaf(sc[z][rb][e], ks[z][e >> 1] * slr[r], -m[r]);
            }
        // (what is rare is kept out of the way: the loop is long for the instruction cache)
        if (__builtin_expect(!clean, 0)) {
#pragma unroll
          for (int z = 0; z < SL; ++z)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (masked(z, rb, e)) x[z][rb][e] = -INFINITY;
        }
#pragma unroll
        for (int z = 0; z < SL; ++z)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              x[z][rb][e] = ex2(x[z][rb][e]);
              top = fmaxf(top, x[z][rb][e]);
            }
        const bool turn = sg.full & kTurn;
        if (__builtin_expect(__any_sync(~0u, top > kMost8) || turn, 0)) {
          if (turn && lane == 0) turned[warp] = next;
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            float mx = -INFINITY;
#pragma unroll
            for (int z = 0; z < SL; ++z)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                float& y = sc[z][r >> 1][2 * i + (r & 1)];
                y = masked(z, r >> 1, 2 * i + (r & 1)) ? -INFINITY : __fmul_rn(__fmul_rn(y, ks[z][i]), slr[r]);
                mx = fmaxf(mx, y);
              }
            mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 4));
            mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 8));
            mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 16));
            const float to = fmaxf(m[r], lower(mx, kUp8)), f = ex2(m[r] - to);
            m[r] = to;
            l[r] *= f;
#pragma unroll
            for (int z = 0; z < SL; ++z)
#pragma unroll
              for (int i = 0; i < 2; ++i) x[z][r >> 1][2 * i + (r & 1)] = ex2(__fadd_rn(sc[z][r >> 1][2 * i + (r & 1)], -to));
#pragma unroll
            for (int i = 0; i < NO; ++i) {
              o[r >> 1][i][r & 1] *= turn ? f * kLess : f;
              o[r >> 1][i][2 + (r & 1)] *= turn ? f * kLess : f;
            }
          }
        }
        // ---- their product with V.  A weight as two halves in f16, the first rounded down, so that it keeps 21 bits (some 2^-24 of
        // up to 2^15 at the least); of several pages' scales the largest, and the others' weights less
        float vmax = 0.f;
#pragma unroll
        for (int z = 0; z < SL; ++z) vmax = fmaxf(vmax, fmaxf(vs[z][0], vs[z][1]));
        const bool differ = 8 << log_br - 3 < KW && vmax > 0.f;
#pragma unroll
        for (int z = 0; z < SL; ++z)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int e = 0; e < 4; ++e) l[2 * rb + (e & 1)] += x[z][rb][e];
        if (__builtin_expect(differ, 0)) {
#pragma unroll
          for (int z = 0; z < SL; ++z)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float f = vs[z][e >> 1] / vmax;
#pragma unroll
              for (int rb = 0; rb < RB; ++rb) x[z][rb][e] *= f;
            }
        }
        uint32_t bh[SL][RB][2], bl[SL][RB][2];
#pragma unroll
        for (int z = 0; z < SL; ++z)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float a = x[z][rb][2 * i], b = x[z][rb][2 * i + 1];
              const uint32_t hi = pack_down<W>(a, b);
              Vec<W, 2> two;
              memcpy(&two, &hi, 4);
              const float2 back = get2(two, 0);
              bh[z][rb][i] = transpose8(hi);  // keys x rows to rows x keys
              bl[z][rb][i] = transpose8(pack<W>(a - back.x, b - back.y));
            }
#pragma unroll
        for (int i0 = 0; i0 < NO; i0 += 2) {
          float sum[2][RB][4] = {};
#pragma unroll
          for (int z = 0; z < SL; ++z) {
            uint32_t c[4], a[4];
            ldsm4t(vt + place8<S>(warp * KW + 16 * z + lane % 16, i0 + lane / 16), c);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              f16_by_parity(c[2 * i], a[0], a[1]);
              f16_by_parity(c[2 * i + 1], a[2], a[3]);
#pragma unroll
              for (int rb = 0; rb < RB; ++rb) {
                mma16<W>(sum[i][rb], a, bl[z][rb][0], bl[z][rb][1]);
                mma16<W>(sum[i][rb], a, bh[z][rb][0], bh[z][rb][1]);
              }
            }
          }
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[rb][i0 + i][e] = fmaf(sum[i][rb][e], vmax, o[rb][i0 + i][e]);
        }
      } else if constexpr (S::MM) {
        // ---- scores of this warp's keys: sc[rb] is keys g (0, 1) and g + 8 (2, 3) by the lane's two rows
        float sc[RB][4], odd[RB][4];  // every other step apart: two chains of products instead of one
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[rb][e] = odd[rb][e] = 0.f;
        {
          const int key = warp * KW + lane % 16;
#pragma unroll
          for (int kk = 0; kk < DP / 16; ++kk) {
            uint32_t a[4];
            ldsm4(kt + kk / 4 * TK * 128 + key * 128 + ((((kk % 4) * 2 + lane / 16) ^ (key & 7)) << 4), a);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) mma16<T>(kk % 2 ? odd[rb] : sc[rb], a, qf[0][rb][kk][0], qf[0][rb][kk][1]);
          }
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sc[rb][e] = __fmul_rn(sc[rb][e] + odd[rb][e], sl);
            if (!clean && hidden(warp * KW + g + 8 * (e >> 1), 2 * rb + (e & 1))) sc[rb][e] = -INFINITY;
          }
        // ---- softmax over what this warp has seen
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          float &s0 = sc[r >> 1][r & 1], &s1 = sc[r >> 1][2 + (r & 1)];
          float mx = fmaxf(s0, s1);
          mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 16));
          const float at = raise(r, mx);
          s0 = ex2(s0 - at);
          s1 = ex2(s1 - at);
          l[r] = l[r] * f[r] + (s0 + s1);
        }
        if (__any_sync(~0u, moved)) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int i = 0; i < NO; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[rb][i][e] *= f[2 * rb + (e & 1)];
        }
        // ---- their product with V.  The weights as two halves of the inputs' type, so that they keep 16 bits in bf16 and 21
        // in f16 (fewer below 2^-14, of up to 2^15, and some 2^-24 at the least): bound by the copies, the kernel has the time,
        // and the output's own rounding stays the largest error.  The first half is rounded down and the second above 0, so
        // that neither is 0 or negative beside an infinite value
        uint32_t bh[RB][2], bl[RB][2];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float a = sc[rb][2 * i], b = sc[rb][2 * i + 1];
            const uint32_t hi = pack_down<T>(a, b);
            Vec<T, 2> two;
            memcpy(&two, &hi, 4);
            const float2 back = get2(two, 0);
            bh[rb][i] = transpose8(hi);  // keys x rows to rows x keys
            bl[rb][i] = transpose8(pack<T>(a > 0.f ? fmaxf(a - back.x, kLeast<T>) : 0.f, b > 0.f ? fmaxf(b - back.y, kLeast<T>) : 0.f));
          }
        const int key = warp * KW + (lane / 16) * 8 + lane % 8;
#pragma unroll
        for (int i = 0; i < NO; ++i) {
          uint32_t a[4];
          ldsm4t(vt + i / 4 * TK * 128 + key * 128 + (((i % 4 * 2 + (lane / 8 & 1)) ^ (key & 7)) << 4), a);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            mma16<T>(o[rb][i], a, bl[rb][0], bl[rb][1]);
            mma16<T>(o[rb][i], a, bh[rb][0], bh[rb][1]);
          }
        }
      } else {
        // ---- scores: lane (g, t) has a quarter of key g, 16 bytes at a time.  Which ones goes by where they lie: of each
        // column's eight, 2t + (g & 1) and its neighbour, so that eight lanes meet eight banks
        const int key = warp * KW + g;
        const float* kp = reinterpret_cast<const float*>(smem + s * 2 * S::TILE) + key * 32;
        float sc[R];
#pragma unroll
        for (int r = 0; r < R; ++r) sc[r] = 0.f;
        const int columns = (p.D + 31) / 32;
#pragma unroll 2
        for (int c = 0; c < columns; ++c) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int at = 2 * t + ((g & 1) ^ e);
            const float4 a = *reinterpret_cast<const float4*>(kp + c * TK * 32 + at * 4);
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const float4 b = *reinterpret_cast<const float4*>(qs + r * DP + c * 32 + ((at ^ (key & 7)) << 2));
              sc[r] = fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, fmaf(a.w, b.w, sc[r]))));
            }
          }
        }
        // ---- softmax over what this warp has seen
#pragma unroll
        for (int r = 0; r < R; ++r) {
          sc[r] += __shfl_xor_sync(~0u, sc[r], 1);
          sc[r] = __fmul_rn(sc[r] + __shfl_xor_sync(~0u, sc[r], 2), sl);
          if (!clean && hidden(key, r)) sc[r] = -INFINITY;
          float mx = sc[r];
          mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 16));
          sc[r] = ex2(sc[r] - raise(r, mx));
          l[r] = l[r] * f[r] + sc[r];
        }
        if (moved) {
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < NO; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[r][i][e] *= f[r];
        }
        // ---- their product with V: key after key, a lane's four values of each
#pragma unroll
        for (int i = 0; i < NO; ++i) {
          const int c = DP == 64 ? lane % 16 : lane + 32 * i;  // of 64 values, two lanes have the same
          const float* vp = reinterpret_cast<const float*>(smem + s * 2 * S::TILE + S::TILE) + c / 8 * TK * 32;
#pragma unroll
          for (int j = 0; j < KW; ++j) {
            const int row = warp * KW + j;
            const float4 v = *reinterpret_cast<const float4*>(vp + row * 32 + ((c % 8 ^ (row & 7)) << 2));
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const float w = __shfl_sync(~0u, sc[r], j * 4);
              o[r][i][0] = fmaf(w, v.x, o[r][i][0]);
              o[r][i][1] = fmaf(w, v.y, o[r][i][1]);
              o[r][i][2] = fmaf(w, v.z, o[r][i][2]);
              o[r][i][3] = fmaf(w, v.w, o[r][i][3]);
            }
          }
        }
      }
      if (!S::EIGHT && !clean) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the zeros before the next copy
      __syncwarp();
      if (lane == 0) mbar_arrive(su32(&empty_bar[s]));
      if (++s == ST) {
        s = 0;
        ph ^= 1;
      }
    }

    // ---- the four warps' parts into one
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      l[r] += __shfl_xor_sync(~0u, l[r], 4);
      l[r] += __shfl_xor_sync(~0u, l[r], 8);
      l[r] += __shfl_xor_sync(~0u, l[r], 16);
      if (S::EIGHT && l[r] == 0.f) m[r] = -INFINITY;
      if (S::MM ? g == 0 : lane == 0) {
        wm[warp][row_of(r)] = m[r];
        wl[warp][row_of(r)] = l[r];
      }
    }
    group_sync<kWarps * 32>();
    [[maybe_unused]] float grain = S::EIGHT && turned[warp] == next ? 1.f / kLess : 1.f;  // what 1 of the sums is (every warp met the turn)
    float f[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) mx = fmaxf(mx, wm[i][row_of(r)]);
      f[r] = m[r] == -INFINITY ? 0.f : ex2(m[r] - mx);
    }
    if (tid < R) {
      float mx = -INFINITY, sum = 0.f;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) mx = fmaxf(mx, wm[i][tid]);
#pragma unroll
      for (int i = 0; i < kWarps; ++i)  // without keys 0 x 0; of scores that are all NaN, NaN
        sum += wl[i][tid] * (wm[i][tid] == -INFINITY ? 0.f : ex2(wm[i][tid] - mx));
      rm[tid] = mx;
      rl[tid] = sum;
    }
    // warp i adds to buffer i % NB in round i / NB
#pragma unroll
    for (int round = 0; round < kWarps / S::NB; ++round) {
      if (warp / S::NB == round && !(!S::MM && DP == 64 && lane >= 16)) {
        float* buf = acc + warp % S::NB * R * S::AS;
#pragma unroll
        for (int rb = 0; rb < OB; ++rb) {
          constexpr int C = 8;  // read together, then written: not one after the other
#pragma unroll
          for (int i0 = 0; i0 < NO; i0 += C) {
            float v[C][4];
            auto place = [&](int i, int e) {
              return S::MM ? buf + row_of(2 * rb + (e & 1)) * S::AS + i * 16 + (S::EIGHT ? 2 * g + (e >> 1) : g + 8 * (e >> 1))
                               : buf + rb * S::AS + (DP == 64 ? lane % 16 : lane + 32 * i) * 4 + e;
            };
#pragma unroll
            for (int i = 0; i < C && i0 + i < NO; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) v[i][e] = round == 0 ? 0.f : *place(i0 + i, e);
#pragma unroll
            for (int i = 0; i < C && i0 + i < NO; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) *place(i0 + i, e) = v[i][e] + o[rb][i0 + i][e] * f[S::MM ? 2 * rb + (e & 1) : rb];
          }
        }
      }
      group_sync<kWarps * 32>();
    }
    if constexpr (S::NB == 2) {
      for (int i = tid; i < nrows * (DP / 4); i += kWarps * 32) {
        float4* a = reinterpret_cast<float4*>(acc + i / (DP / 4) * S::AS + i % (DP / 4) * 4);
        const float4 b = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a) + R * S::AS);
        *a = make_float4(a->x + b.x, a->y + b.y, a->z + b.z, a->w + b.w);
      }
      group_sync<kWarps * 32>();
    }
    if (!S::EIGHT && unfit) {
      for (int r = warp; r < nrows; r += kWarps) {
        const int past = limit(r) - lim_min;
        unsigned last = unfit & 0xFFFFu & ((1u << past) - 1);
        if (WIN && past > p.window)  // a window shorter than the unit's tokens
          last &= ~((1u << (past - p.window)) - 1) | (p.sinks > lim_min ? (1u << min(16, p.sinks - lim_min)) - 1 : 0u);
        const int* table = p.table + (int64_t)w.item * p.width;
        add_keys<T, DP>(p, qrow(r), table, h, lim_min, last, sl, rm[r], acc + r * S::AS);
        if (WIN) add_keys<T, DP>(p, qrow(r), table, h, lim_min - p.window, unfit >> 16 >> past << past, sl, rm[r], acc + r * S::AS);
      }
      group_sync<kWarps * 32>();
    }

    // ---- out, or joined with the unit's other parts
    auto rows_out = [&]() {
      const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 15) == 0;
      for (int i = tid; i < nrows * (p.D / 4); i += kWarps * 32) {
        const int r = i / (p.D / 4), d = i % (p.D / 4) * 4;
        const float4 v = *reinterpret_cast<const float4*>(acc + r * S::AS + d);
        const float n = rl[r] > 0.f || rl[r] != rl[r] ? 1.f / rl[r] : 0.f;
        const float to = S::EIGHT ? grain : 1.f;
        Vec<T, 4> y = {from_f32<T>(v.x * n * to), from_f32<T>(v.y * n * to), from_f32<T>(v.z * n * to), from_f32<T>(v.w * n * to)};
        T* dst = static_cast<T*>(p.out) +
                 ((int64_t)(w.t0 + p.G.div(r0 + r)) * p.H * p.G.d + h * p.G.d + p.G.mod(r0 + r)) * p.D + d;
        if (wide) {
          *reinterpret_cast<Vec<T, 4>*>(dst) = y;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) dst[e] = y.v[e];
        }
      }
      if (p.lse && tid < nrows)
        p.lse[(int64_t)(w.t0 + p.G.div(r0 + tid)) * p.H * p.G.d + h * p.G.d + p.G.mod(r0 + tid)] =
            rl[tid] == 0.f ? -INFINITY : log_sum<W, kUp>(rm[tid], rl[tid]);
    };
    const int first = w.base + u * w.span;  // the unit's first place
    const int c0 = first / run, parts = (first + w.kt - 1) / run - c0 + 1;
    if (parts == 1) {
      rows_out();
    } else {
      auto slot = [&](int part) {
        return p.partial + (int64_t)(part == 0 ? 2 * c0 + 1 : 2 * (c0 + part)) * S::PART;
      };
      constexpr int kGrain = kRows * DP + kRows - 1;  // (over codes there are 8 rows, and the last maximum's place is free)
      static_assert(!S::EIGHT || R < kRows, "the grain's place");
      auto store = [&](float* to) {
        for (int i = tid; i < nrows * (DP / 4); i += kWarps * 32) {
          const int r = i / (DP / 4), d = i % (DP / 4) * 4;
          __stcg(reinterpret_cast<float4*>(to + r * DP + d), *reinterpret_cast<const float4*>(acc + r * S::AS + d));
        }
        if (tid < nrows) {
          __stcg(to + kRows * DP + tid, rm[tid]);
          __stcg(to + kRows * DP + kRows + tid, rl[tid]);
        }
        if (S::EIGHT && tid == 0) __stcg(to + kGrain, grain);
      };
      // the last of `of` to come here; what the others stored is then there to read
      // (one thread's release behind the barrier is every thread's)
      auto last_of = [&](int* counter, int of) {
        group_sync<kWarps * 32>();
        if (tid == 0) {
          int was;
          asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(was) : "l"(counter) : "memory");
          if (was == of - 1) *counter = 0;
          last_flag = was == of - 1;
        }
        group_sync<kWarps * 32>();
        return last_flag != 0;
      };
      // n parts, step apart, into acc, rm and rl: in their order, whoever comes last
      auto join = [&](int part, int n, int step) {
        // over codes in the parts' largest grain: what the sums of one count there
        auto in_grain = [&](float c, float of) { return S::EIGHT && grain != of ? c * kLess : c; };
        if (EX > 0 && R <= 8 && n <= kGroup) {  // 16 lanes to a row, a part each
          const int r = tid / kGroup, i = tid % kGroup;
          const bool in = r < nrows && i < n;
          const float* from = slot(part + (in ? i : 0) * step) + kRows * DP + (in ? r : 0);
          const float pm = in ? __ldcg(from) : -INFINITY, pl = in ? __ldcg(from + kRows) : 0.f;
          const float of = S::EIGHT && i < n ? __ldcg(slot(part + i * step) + kGrain) : 1.f;
          if constexpr (S::EIGHT) grain = __any_sync(~0u, of != 1.f) ? 1.f / kLess : 1.f;  // (a warp has every part)
          float mx = pm;
#pragma unroll
          for (int d = 1; d < kGroup; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, d));
          const float c = pm == -INFINITY ? 0.f : ex2(pm - mx);
          float sum = c * pl;  // NaN stays NaN
#pragma unroll
          for (int d = 1; d < kGroup; d <<= 1) sum += __shfl_xor_sync(~0u, sum, d);
          if (in) wts[r][i] = in_grain(c, of);
          if (i == 0 && r < nrows) {
            rm[r] = mx;
            rl[r] = sum;
          }
        } else {
          for (int i = tid; i < n * kRows; i += kWarps * 32) {  // row i % 16 of part i / 16
            const float* from = slot(part + i / kRows * step) + kRows * DP + i % kRows;
            if (i % kRows < nrows) {
              wts[i % kRows][i / kRows] = __ldcg(from);
              sums[i % kRows][i / kRows] = __ldcg(from + kRows);
            }
          }
          if constexpr (S::EIGHT) {
            bool any = false;
            for (int i = lane; i < n; i += 32) any = any || __ldcg(slot(part + i * step) + kGrain) != 1.f;
            grain = __any_sync(~0u, any) ? 1.f / kLess : 1.f;
          }
          group_sync<kWarps * 32>();
          if (tid < nrows) {
            float mx = -INFINITY, sum = 0.f;
            for (int i = 0; i < n; ++i) mx = fmaxf(mx, wts[tid][i]);
            for (int i = 0; i < n; ++i) {
              const float c = wts[tid][i] == -INFINITY ? 0.f : ex2(wts[tid][i] - mx);
              wts[tid][i] = S::EIGHT ? in_grain(c, __ldcg(slot(part + i * step) + kGrain)) : c;
              sum += c * sums[tid][i];  // NaN stays NaN
            }
            rm[tid] = mx;
            rl[tid] = sum;
          }
        }
        group_sync<kWarps * 32>();
        for (int i = tid; i < nrows * (DP / 4); i += kWarps * 32) {
          const int r = i / (DP / 4), d = i % (DP / 4) * 4;
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
          for (int j = 0; j < n; ++j) {
            const float4 a = __ldcg(reinterpret_cast<const float4*>(slot(part + j * step) + r * DP + d));
            const float c = wts[r][j];
            v.x += c * a.x;
            v.y += c * a.y;
            v.z += c * a.z;
            v.w += c * a.w;
          }
          *reinterpret_cast<float4*>(acc + r * S::AS + d) = v;
        }
        group_sync<kWarps * 32>();
      };
      const int part = (int)blockIdx.x - c0, group = part / kGroup, groups = (parts + kGroup - 1) / kGroup;
      store(slot(part));
      const int gn = min(kGroup, parts - group * kGroup);
      if (last_of(p.counters + 3 * (c0 + group * kGroup) + (group > 0), gn)) {
        join(group * kGroup, gn, 1);
        if (groups == 1) {
          rows_out();
        } else {
          store(slot(group * kGroup));
          if (last_of(p.counters + 3 * c0 + 2, groups)) {
            join(0, groups, kGroup);
            rows_out();
          }
        }
      }
    }
    group_sync<kWarps * 32>();  // acc is free
    x = next;
  }
  if (timed_out) {
    if (lane == 0) atomicOr(p.status, PP_CACHE_TIMEOUT);
    if (tid == 0)  // copies still in flight end before the CTA does
      for (int i = 0; i < ST; ++i) wait(su32(&full_bar[i]), 0), wait(su32(&full_bar[i]), 1);
  }
}

template <class T, class Cell, int DP, int RB, bool WIN>
cudaError_t prepare_one() {
  return cudaFuncSetAttribute(attn_kernel<T, Cell, DP, RB, WIN>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<T, Cell, DP, RB>::SMEM);
}

template <class T, class Cell, int DP, int RB, bool WIN>
cudaError_t launch(const AttnParams& p, const pp_cache& c, int sms, cudaStream_t stream) {
  // all tiles, at most: they are counted in 32 bits
  using S = Shape<T, Cell, DP, RB>;
  constexpr int R = S::R, TK = S::TK;
  const int64_t units = (p.sel ? (int64_t)p.T * ((p.G.d + R - 1) / R) : ((int64_t)p.T * p.G.d + (int64_t)p.B * (R - 1)) / R) * p.H;
  const int64_t deep = ((int64_t)(p.sel ? std::min(p.width, p.keep) : p.width) * p.page + TK - 1) / TK;
  if (units >= INT32_MAX / (deep + S::template EXTRA<WIN>)) return cudaErrorNotSupported;
  const int grid = std::min(sms * S::CTAS, kMaxCtas);
  return launch_after(attn_kernel<T, Cell, DP, RB, WIN>, dim3(grid), S::THREADS, S::SMEM, stream, 1, p, c.mk, c.mv);
}

// Units of as many rows as a sequence (or, with selected pages, a token) has, up to 8 or 16; in fp32 and over codes up to 8.
template <class T, class Cell, int DP, bool WIN>
cudaError_t by_rows(const AttnParams& p, const pp_cache& c, int sms, cudaStream_t stream) {
  const int64_t rows = p.sel || !p.starts ? p.G.d : ((int64_t)p.T * p.G.d + p.B - 1) / p.B;
  if constexpr (sizeof(Cell) == 1) {
    return launch<T, Cell, DP, 1, WIN>(p, c, sms, stream);
  } else if constexpr (sizeof(T) == 2) {
    return rows <= 8 ? launch<T, Cell, DP, 1, WIN>(p, c, sms, stream) : launch<T, Cell, DP, 2, WIN>(p, c, sms, stream);
  } else {
    return rows <= 2   ? launch<T, Cell, DP, 2, WIN>(p, c, sms, stream)
           : rows <= 4 ? launch<T, Cell, DP, 4, WIN>(p, c, sms, stream)
                       : launch<T, Cell, DP, 8, WIN>(p, c, sms, stream);
  }
}

template <class T, class Cell, bool WIN>
cudaError_t by_head(const AttnParams& p, const pp_cache& c, int sms, cudaStream_t stream) {
  return p.D <= 64    ? by_rows<T, Cell, 64, WIN>(p, c, sms, stream)
         : p.D <= 128 ? by_rows<T, Cell, 128, WIN>(p, c, sms, stream)
                      : by_rows<T, Cell, 256, WIN>(p, c, sms, stream);
}

template <class T, class Cell, int RB, bool WIN>
cudaError_t prepare_rows() {
  cudaError_t e = prepare_one<T, Cell, 64, RB, WIN>();
  if (e == cudaSuccess) e = prepare_one<T, Cell, 128, RB, WIN>();
  if (e == cudaSuccess) e = prepare_one<T, Cell, 256, RB, WIN>();
  return e;
}

template <class T, class Cell, bool WIN>
cudaError_t prepare_type() {
  cudaError_t e;
  if constexpr (sizeof(Cell) == 1) {
    e = prepare_rows<T, Cell, 1, WIN>();
  } else if constexpr (sizeof(T) == 2) {
    e = prepare_rows<T, Cell, 1, WIN>();
    if (e == cudaSuccess) e = prepare_rows<T, Cell, 2, WIN>();
  } else {
    e = prepare_rows<T, Cell, 2, WIN>();
    if (e == cudaSuccess) e = prepare_rows<T, Cell, 4, WIN>();
    if (e == cudaSuccess) e = prepare_rows<T, Cell, 8, WIN>();
  }
  return e;
}

}  // namespace ppc_row
