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
// over 8 (f16) 308 us, 7.0 TB/s; 48 of up to 8192 (bf16) 151 us, 5.7 TB/s; 32 tokens
// over 32 selected pages of 64 each (bf16) 45 us, 5.9 TB/s; fp32, 16 of up to 2500, 8
// heads of 96 over 4: 22 us, 3.2 TB/s.  One sequence of 777 keys: 11 us, a chain of
// launch, lengths, page table, copy, tile and join.
#include <algorithm>
#include <cmath>

#include "attn.cuh"
#include "internal.h"

namespace {

using namespace ppc;
using namespace ppc_ptx;
using namespace ppc_attn;

constexpr int kRows = 16;      // query rows of a unit at most
constexpr int kWarps = 4;      // that compute; one more copies
constexpr int kThreads = kWarps * 32 + 32;
constexpr int kUp = 15;        // f16 weights are up to 2^15 (a warp's m is never behind its keys)
constexpr int kGroup = 16;     // parts of a unit joined at once
constexpr int kMaxCtas = 512;  // kGroup^2 parts and more
constexpr int kJoin = kMaxCtas / kGroup;

template <class T, int DP, int RB>
struct Shape {
  static constexpr int E = sizeof(T);
  static constexpr int R = E == 4 ? RB : 8 * RB;  // query rows of a unit
  static constexpr int TK = E == 4 ? 32 : 64;   // keys per tile
  static constexpr int LOG_TK = E == 4 ? 5 : 6;
  static constexpr int KW = TK / kWarps;        // keys per warp
  static constexpr int CH = 128 / E;            // values per 128-byte column
  static constexpr int NCH = DP / CH;
  static constexpr int TILE = TK * DP * E;      // bytes of a K or V tile
  static constexpr int CTAS = DP <= 128 ? 2 : 1;
  static constexpr int QS = E == 4 ? R * DP * 4 : 0;  // fp32 queries stay in shared memory
  static constexpr int AS = DP + 4;             // row stride of the joining buffers, free of bank conflicts
  static constexpr int NB = R <= 8 ? 2 : 1;     // joining buffers
  static constexpr int ACC = NB * R * AS * 4;
  // as many stages as fit: with 228 KB per SM, 1 KB of it taken and 6 KB static per CTA, 190 KB are in flight (16 bits)
  static constexpr int STAGES = (233472 / CTAS - 1024 - 6144 - 1024 - ACC - QS) / (2 * TILE);
  static constexpr int SMEM = STAGES * 2 * TILE + ACC + QS + 1024;
  static constexpr int PART = kRows * DP + 2 * kRows;  // floats of a partial result
};

struct Stage {          // what the producer says of a tile
  int have[kPieces];    // keys of each piece that the call may use
  int full;             // all of them
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
// Walks the units' tiles in their one order (whole: in runs that end with their unit).  An item is a sequence, or a token where pages are selected for each
// token; its units are (R rows, head) pairs of kt tiles each.
struct Walk {
  int base;  // its first place in the order
  int item, t0, n, len, rows, units;
  int kt;    // tiles of a unit
  int span;  // places of a unit in the order: its tiles, or whole runs of them
  int places;
};
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
  w.span = whole ? (w.kt + whole - 1) / whole * whole : w.kt;
  w.places = w.units * w.span;
}

template <class T, int DP, int RB>
__global__ void __launch_bounds__(kThreads, Shape<T, DP, RB>::CTAS)
    attn_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv) {
  using S = Shape<T, DP, RB>;
  constexpr int TK = S::TK, KW = S::KW, ST = S::STAGES, R = S::R;
  extern __shared__ unsigned char raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  float* acc = reinterpret_cast<float*>(smem + ST * 2 * S::TILE);
  [[maybe_unused]] float* qs = acc + S::NB * R * S::AS;
  __shared__ alignas(8) uint64_t full_bar[ST], empty_bar[ST];
  __shared__ Stage stage[ST];
  __shared__ float wm[kWarps][kRows], wl[kWarps][kRows], rm[kRows], rl[kRows];
  __shared__ float wts[kRows][kJoin + 1], sums[kRows][kJoin + 1];
  __shared__ int scan[4][kThreads / 32], last_flag, dead;
  __shared__ unsigned unfit;  // keys from lim_min on with values that are not finite, a bit each
  __shared__ Walk found;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const int NI = p.sel ? p.T : p.B;

  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mk) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mv) : "memory");
    dead = 0;
    for (int i = 0; i < ST; ++i) {
      mbar_init(su32(&full_bar[i]), 1);
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
  for (int i = i0; i < i1; ++i) {
    load_item(p, TK, R, 0, i, w);
    tiles += w.places;
    units += w.units;
    bad_range = bad_range || w.n < 0;
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
  // Equal runs; one of a single tile would spend more on joining than on its keys.  Where every unit can have CTAs of its
  // own with runs not much longer (up to 1.4 times, which the copies of the other CTAs make up for), runs end with
  // their unit: a CTA that changes units waits some 3 us for queries, joining and stores.
  int run = max((all[0] + grid - 1) / grid, 2), whole = 0;
  if (all[1] <= grid) {
    const int longer[4] = {run, run + run / 10 + 1, run + run / 4 + 1, run + run * 2 / 5 + 2};
    int ctas[4] = {};
    for (int i = i0; i < i1; ++i) {
      if (per > 1) load_item(p, TK, R, 0, i, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) ctas[j] += w.units * ((w.kt + longer[j] - 1) / longer[j]);
    }
    sums_of(ctas);
#pragma unroll
    for (int j = 3; j >= 0; --j)
      if (ctas[j] <= grid && (int64_t)longer[j] * grid <= INT32_MAX) whole = longer[j];  // places are counted in 32 bits
    if (whole) run = whole;
  }
  // a scan places the items in the one order
  int mine = 0;
  for (int i = i0; i < i1; ++i) {
    if (per > 1 || whole) load_item(p, TK, R, whole, i, w);
    mine += w.places;
  }
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
      if (per > 1) load_item(p, TK, R, whole, i, w);
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
      load_item(p, TK, R, whole, w.item + 1, w);
      w.base = b;
    }
  };

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
      const int b = p.sel ? seen_keys(w.t0, p.T, p.B, p.starts, p.lens, p.width * p.page, p.causal, p.status).b : w.item;
      const int* row = p.table + (int64_t)b * p.width;
      const int* list = p.sel ? p.sel + ((int64_t)w.t0 * p.H + h) * p.keep : nullptr;
      int have32 = 0, y32 = 0;
      for (int k = k0; k < k1; ++k) {
        const int in32 = (k - k0) << log_pc & 31;  // the tile's first piece among the 32
        if (in32 == 0) {
          have32 = 0;
          // key of the sequence, or of the list's pages in a row
          const int64_t key = (int64_t)k * TK + lane * BR;
          if (key < (int64_t)k1 * TK) {
            const int off = (int)key & (p.page - 1);
            int at = (int)(key >> p.log_page);
            bool ok = true;
            if (list) {
              ok = at < p.keep;
              at = ok ? list[at] : -1;
              if (at >= p.width) atomicOr(p.status, PP_CACHE_BAD_PAGE);
              ok = at >= 0 && at < p.width;
            }
            have32 = ok ? max(0, min(BR, w.len - at * p.page - off)) : 0;
            if (have32 > 0) {
              const int id = row[at];
              if (id < 0 || id >= p.pages) {
                atomicOr(p.status, PP_CACHE_BAD_PAGE);
                have32 = 0;
              }
              y32 = (int)(((int64_t)id * p.H + h) * p.page) + off;
            }
          }
        }
        const int have = __shfl_sync(~0u, have32, in32 + (lane & pieces - 1));
        const int y = __shfl_sync(~0u, y32, in32 + (lane & pieces - 1));
        const unsigned live = __ballot_sync(~0u, lane < pieces && have > 0);
        const bool whole = __all_sync(~0u, have == BR);
        if (!*(volatile int*)&dead && !wait(su32(&empty_bar[s]), ph)) dead = 1;
        __syncwarp();
        const bool go = !*(volatile int*)&dead;
        if (lane < pieces) stage[s].have[lane] = have;
        if (lane == 0) stage[s].full = whole;
        __syncwarp();
        if (lane == 0) mbar_arrive_expect_tx(su32(&full_bar[s]), go ? __popc(live) * 2 * BR * DP * S::E : 0);
        __syncwarp();
        const uint32_t dst = su32(smem + s * 2 * S::TILE);
        const int boxes = pieces * S::NCH * 2, j = lane & pieces - 1;  // box i: piece i % pieces, column and pool i / pieces
        for (int i = lane; i < boxes; i += 32) {
          const int c = (i >> log_pc) % S::NCH, v = (i >> log_pc) / S::NCH;
          if (go && (live >> j & 1))
            copy_box(dst + v * S::TILE + c * TK * 128 + j * BR * 128, v ? &mv : &mk, c * S::CH, y, su32(&full_bar[s]));
        }
        __syncwarp();
        if (++s == ST) {
          s = 0;
          ph ^= 1;
        }
      }
      x = next;
    }
    if (p.sel && p.starts && blockIdx.x == 0) check_ranges(p.starts, p.T, p.B, lane, 32, p.status);
    return;
  }

  // ---- consumers
  // A lane's sums: 16 bits, values i * 16 + g, + 8 of rows 8 rb + 2t, + 1 (o[rb][i]); fp32, four values from (lane + 32 i) * 4
  // on of every row (o[r][i]).
  constexpr int NO = S::E == 2 ? DP / 16 : (DP + 127) / 128, OB = S::E == 2 ? RB : R, NR = S::E == 2 ? 2 * RB : R;
  const int g = lane / 4, t = lane % 4;
  // the r-th of the lane's NR rows
  auto row_of = [&](int r) { return S::E == 2 ? (r >> 1) * 8 + 2 * t + (r & 1) : r; };
  const T* q = static_cast<const T*>(p.q);
  [[maybe_unused]] const bool q16 = ((reinterpret_cast<uintptr_t>(q) & 15) | (p.q_ts & 7) | (p.q_hs & 7)) == 0;
  int s = 0;
  uint32_t ph = 0;
  bool timed_out = false;
  for (int x = x0; x < x1;) {
    settle(x);
    const int u = (x - w.base) / w.span, h = p.by_head.mod(u), r0 = p.by_head.div(u) * R;
    const int k0 = x - w.base - u * w.span, next = x + min(w.span - k0, x1 - x), k1 = min(w.kt, k0 + next - x);
    const int nrows = min(R, w.rows - r0);
    const bool listed = p.sel != nullptr;
    // keys that a row of the unit may see
    auto limit = [&](int r) {
      return p.causal && !listed ? min(w.len, max(0, w.len - w.n + p.G.div(r0 + r) + 1)) : w.len;
    };
    int lim[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) lim[r] = limit(min(row_of(r), nrows - 1));
    const int lim_min = limit(0), lim_max = limit(nrows - 1);
    // the row's queries: token r / G of the unit's, head r % G of the group's
    auto qrow = [&](int r) {
      return q + (w.t0 + p.G.div(r0 + r)) * p.q_ts + (int64_t)(h * p.G.d + p.G.mod(r0 + r)) * p.q_hs;
    };
    [[maybe_unused]] uint32_t qf[S::E == 2 ? RB : 1][S::E == 2 ? DP / 16 : 1][2];
    if (tid == 0) unfit = 0;
    if constexpr (S::E == 2) {
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
          qf[rb][kk][0] = f[0];
          qf[rb][kk][1] = f[1];
          qf[rb][kk + 1][0] = f[2];
          qf[rb][kk + 1][1] = f[3];
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
      m[r] = -INFINITY;
      l[r] = 0.f;
    }

    for (int k = k0; k < k1; ++k) {
      if (!*(volatile int*)&dead && !wait(su32(&full_bar[s]), ph)) dead = 1;
      __syncwarp();
      timed_out = timed_out || *(volatile int*)&dead;
      const uint32_t kt = su32(smem + s * 2 * S::TILE), vt = kt + S::TILE;
      const Stage& sg = stage[s];
      const bool clean = sg.full && (listed || (k + 1) * TK <= lim_min);
      // a key of the tile that row r of the lane's may not use; keys whose values have to be 0, as no row uses them
      auto hidden = [&](int j, int r) { return (j & (BR - 1)) >= sg.have[j >> log_br] || (!listed && k * TK + j >= lim[r]); };
      if (!clean) {  // 0 x the values that a row does not see has to be 0
#pragma unroll
        for (int i = 0; i < KW; ++i) {
          const int j = warp * KW + i;
          unsigned char* v = smem + s * 2 * S::TILE + S::TILE + j * 128;
          bool zero = (j & (BR - 1)) >= sg.have[j >> log_br] || (!listed && k * TK + j >= lim_max);
          if (!zero && !listed && k * TK + j >= lim_min) {  // some rows see it
            for (int c = lane; c < S::NCH * 8; c += 32)
              zero = zero || not_finite<T>(*reinterpret_cast<const uint4*>(v + c / 8 * TK * 128 + c % 8 * 16));
            zero = __any_sync(~0u, zero);
            if (zero && lane == 0) atomicOr(&unfit, 1u << (k * TK + j - lim_min));
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
        mx = fmaxf(m[r], lower(mx, kLift<T, kUp>));
        const float at = mx == -INFINITY ? 0.f : mx;
        f[r] = ex2(m[r] - at);
        moved = moved || m[r] != mx;
        m[r] = mx;
        return at;
      };
      if constexpr (S::E == 2) {
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
            for (int rb = 0; rb < RB; ++rb) mma16<T>(kk % 2 ? odd[rb] : sc[rb], a, qf[rb][kk][0], qf[rb][kk][1]);
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
      if (!clean) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the zeros before the next copy
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
      if (S::E == 2 ? g == 0 : lane == 0) {
        wm[warp][row_of(r)] = m[r];
        wl[warp][row_of(r)] = l[r];
      }
    }
    group_sync<kWarps * 32>();
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
      if (warp / S::NB == round && !(S::E == 4 && DP == 64 && lane >= 16)) {
        float* buf = acc + warp % S::NB * R * S::AS;
#pragma unroll
        for (int rb = 0; rb < OB; ++rb) {
          constexpr int C = 8;  // read together, then written: not one after the other
#pragma unroll
          for (int i0 = 0; i0 < NO; i0 += C) {
            float v[C][4];
            auto place = [&](int i, int e) {
              return S::E == 2 ? buf + row_of(2 * rb + (e & 1)) * S::AS + i * 16 + g + 8 * (e >> 1)
                               : buf + rb * S::AS + (DP == 64 ? lane % 16 : lane + 32 * i) * 4 + e;
            };
#pragma unroll
            for (int i = 0; i < C && i0 + i < NO; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) v[i][e] = round == 0 ? 0.f : *place(i0 + i, e);
#pragma unroll
            for (int i = 0; i < C && i0 + i < NO; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) *place(i0 + i, e) = v[i][e] + o[rb][i0 + i][e] * f[S::E == 2 ? 2 * rb + (e & 1) : rb];
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
    if (unfit) {
      for (int r = warp; r < nrows; r += kWarps)
        add_keys<T, DP>(p, qrow(r), p.table + (int64_t)w.item * p.width, h, lim_min, unfit & ((1u << (limit(r) - lim_min)) - 1), sl, rm[r],
                        acc + r * S::AS);
      group_sync<kWarps * 32>();
    }

    // ---- out, or joined with the unit's other parts
    auto rows_out = [&]() {
      const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 15) == 0;
      for (int i = tid; i < nrows * (p.D / 4); i += kWarps * 32) {
        const int r = i / (p.D / 4), d = i % (p.D / 4) * 4;
        const float4 v = *reinterpret_cast<const float4*>(acc + r * S::AS + d);
        const float n = rl[r] > 0.f || rl[r] != rl[r] ? 1.f / rl[r] : 0.f;
        Vec<T, 4> y = {from_f32<T>(v.x * n), from_f32<T>(v.y * n), from_f32<T>(v.z * n), from_f32<T>(v.w * n)};
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
            rl[tid] == 0.f ? -INFINITY : log_sum<T, kUp>(rm[tid], rl[tid]);
    };
    const int first = w.base + u * w.span;  // the unit's first place
    const int c0 = first / run, parts = (first + w.span - 1) / run - c0 + 1;
    if (parts == 1) {
      rows_out();
    } else {
      auto slot = [&](int part) {
        return p.partial + (int64_t)(part == 0 ? 2 * c0 + 1 : 2 * (c0 + part)) * S::PART;
      };
      auto store = [&](float* to) {
        for (int i = tid; i < nrows * (DP / 4); i += kWarps * 32) {
          const int r = i / (DP / 4), d = i % (DP / 4) * 4;
          __stcg(reinterpret_cast<float4*>(to + r * DP + d), *reinterpret_cast<const float4*>(acc + r * S::AS + d));
        }
        if (tid < nrows) {
          __stcg(to + kRows * DP + tid, rm[tid]);
          __stcg(to + kRows * DP + kRows + tid, rl[tid]);
        }
      };
      // the last of `of` to come here; what the others stored is then there to read
      auto last_of = [&](int* counter, int of) {
        __threadfence();
        group_sync<kWarps * 32>();
        if (tid == 0) {
          const int was = atomicAdd(counter, 1);
          if (was == of - 1) *counter = 0;
          __threadfence();
          last_flag = was == of - 1;
        }
        group_sync<kWarps * 32>();
        return last_flag != 0;
      };
      // n parts, step apart, into acc, rm and rl: in their order, whoever comes last
      auto join = [&](int part, int n, int step) {
        for (int i = tid; i < n * kRows; i += kWarps * 32) {  // row i % 16 of part i / 16
          const float* from = slot(part + i / kRows * step) + kRows * DP + i % kRows;
          if (i % kRows < nrows) {
            wts[i % kRows][i / kRows] = __ldcg(from);
            sums[i % kRows][i / kRows] = __ldcg(from + kRows);
          }
        }
        group_sync<kWarps * 32>();
        if (tid < nrows) {
          float mx = -INFINITY, sum = 0.f;
          for (int i = 0; i < n; ++i) mx = fmaxf(mx, wts[tid][i]);
          for (int i = 0; i < n; ++i) {
            const float c = wts[tid][i] == -INFINITY ? 0.f : ex2(wts[tid][i] - mx);
            wts[tid][i] = c;
            sum += c * sums[tid][i];  // NaN stays NaN
          }
          rm[tid] = mx;
          rl[tid] = sum;
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

template <class T, int DP, int RB>
cudaError_t prepare_one() {
  return cudaFuncSetAttribute(attn_kernel<T, DP, RB>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<T, DP, RB>::SMEM);
}

template <class T, int DP, int RB>
cudaError_t launch(const AttnParams& p, const pp_cache& c, int sms, cudaStream_t stream) {
  // all tiles, at most: they are counted in 32 bits
  constexpr int R = Shape<T, DP, RB>::R, TK = Shape<T, DP, RB>::TK;
  const int64_t units = (p.sel ? (int64_t)p.T * ((p.G.d + R - 1) / R) : ((int64_t)p.T * p.G.d + (int64_t)p.B * (R - 1)) / R) * p.H;
  const int64_t deep = ((int64_t)(p.sel ? std::min(p.width, p.keep) : p.width) * p.page + TK - 1) / TK;
  if (units >= INT32_MAX / deep) return cudaErrorNotSupported;
  const int grid = std::min(sms * Shape<T, DP, RB>::CTAS, kMaxCtas);
  return launch_after(attn_kernel<T, DP, RB>, dim3(grid), kThreads, Shape<T, DP, RB>::SMEM, stream, 1, p, c.mk, c.mv);
}

// Units of as many rows as a sequence (or, with selected pages, a token) has, up to 8 or 16; in fp32 up to 8.
template <class T, int DP>
cudaError_t by_rows(const AttnParams& p, const pp_cache& c, int sms, cudaStream_t stream) {
  const int64_t rows = p.sel || !p.starts ? p.G.d : ((int64_t)p.T * p.G.d + p.B - 1) / p.B;
  if constexpr (sizeof(T) == 2) {
    return rows <= 8 ? launch<T, DP, 1>(p, c, sms, stream) : launch<T, DP, 2>(p, c, sms, stream);
  } else {
    return rows <= 2   ? launch<T, DP, 2>(p, c, sms, stream)
           : rows <= 4 ? launch<T, DP, 4>(p, c, sms, stream)
                       : launch<T, DP, 8>(p, c, sms, stream);
  }
}

template <class T>
cudaError_t by_head(const AttnParams& p, const pp_cache& c, int sms, cudaStream_t stream) {
  return p.D <= 64    ? by_rows<T, 64>(p, c, sms, stream)
         : p.D <= 128 ? by_rows<T, 128>(p, c, sms, stream)
                      : by_rows<T, 256>(p, c, sms, stream);
}

template <class T, int RB>
cudaError_t prepare_type() {
  cudaError_t e = prepare_one<T, 64, RB>();
  if (e == cudaSuccess) e = prepare_one<T, 128, RB>();
  if (e == cudaSuccess) e = prepare_one<T, 256, RB>();
  return e;
}

DeviceOnce g_attn_once;

}  // namespace

namespace ppc {

AttnSpace attn_space(int dtype, int D, int sms) {
  const int DP = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  const size_t ctas = (size_t)std::min(sms * (DP <= 128 ? 2 : 1), kMaxCtas);
  return {ctas * 3 * 4, ctas * 2 * (kRows * DP + 2 * kRows) * 4, tile_space(dtype, D, sms)};
}

cudaError_t attn_prepare() {
  return g_attn_once.run([](int) {
    cudaError_t e = tile_prepare();
    if (e == cudaSuccess) e = prepare_type<float, 2>();
    if (e == cudaSuccess) e = prepare_type<float, 4>();
    if (e == cudaSuccess) e = prepare_type<float, 8>();
    if (e == cudaSuccess) e = prepare_type<__half, 1>();
    if (e == cudaSuccess) e = prepare_type<__half, 2>();
    if (e == cudaSuccess) e = prepare_type<__nv_bfloat16, 1>();
    if (e == cudaSuccess) e = prepare_type<__nv_bfloat16, 2>();
    return e;
  });
}

}  // namespace ppc

extern "C" pp_status pp_attn_forward(const pp_cache* cache, int T, const void* q, int64_t q_ts, int64_t q_hs, int Hq,
                                     int B, const int32_t* starts, const int32_t* table, int width, const int32_t* lens,
                                     float scale, int flags, const int32_t* sel, int keep, void* out, float* lse,
                                     void* stream) {
  if (!cache || T < 0 || B < 0 || Hq < 1 || Hq % cache->H || width < 1 || q_ts < 0 || q_hs < 0 || !std::isfinite(scale) ||
      (flags & ~PP_ATTN_CAUSAL) || (sel ? keep < 1 : keep != 0))
    return PP_ERR_INVALID_ARG;
  const uintptr_t al = (uintptr_t)dtype_size(cache->dtype) - 1;
  if (T > 0 && (!q || !table || !lens || !out || B < 1 || (!starts && T != B) || (reinterpret_cast<uintptr_t>(q) & al) ||
                (reinterpret_cast<uintptr_t>(out) & al) || (reinterpret_cast<uintptr_t>(lse) & 3)))
    return PP_ERR_INVALID_ARG;
  if (T == 0) return PP_OK;
  if ((int64_t)width * cache->page > INT32_MAX - 256) return PP_ERR_UNSUPPORTED;  // the end of a tile is counted in 32 bits, too
  const int sms = device_sms();
  if (sms <= 0) return PP_ERR_CUDA;
  const pp_cache& c = *cache;
  const int G = Hq / c.H;
  if ((int64_t)T * G >= INT32_MAX) return PP_ERR_UNSUPPORTED;
  AttnParams p = {q,     q_ts,   q_hs,        c.k,        c.v,     starts, table, lens, sel,  out, lse, c.status, c.counters,
                  c.partial, scale, T, B, c.H, c.D, c.page, log2_of(c.page), c.pages, width, keep, flags & PP_ATTN_CAUSAL,
                  FastDiv(G), FastDiv(c.H), FastDiv(std::max(keep, 1)), 1, nullptr, nullptr};
  const cudaStream_t s = (cudaStream_t)stream;
  const cudaError_t e = tile_applicable(p, c.dtype, sms) ? tile_launch(p, c, sms, s)
                        : c.dtype == PP_F32 ? by_head<float>(p, c, sms, s)
                        : c.dtype == PP_F16 ? by_head<__half>(p, c, sms, s)
                                            : by_head<__nv_bfloat16>(p, c, sms, s);
  return e == cudaSuccess ? PP_OK : e == cudaErrorNotSupported ? PP_ERR_UNSUPPORTED : PP_ERR_CUDA;
}
