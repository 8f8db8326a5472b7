// Attention of query tokens over the paged cache (pp_attn_forward).
//
// out = sum_j softmax_j(scale q.k_j) v_j, one pass over the keys with a running
// maximum and sum.  With few query rows per key (single tokens, groups of heads
// over one cache head) it is bound by reading K and V from device memory.
//
// A unit is 16 query rows (tokens x the heads of a group) of one sequence and
// cache head; its keys come in tiles (64 rows of 16-bit values, 32 of fp32).
// All units' tiles in a row are cut into equal runs, one per CTA, whatever the
// sequences' lengths: each CTA reads the same number of bytes, and only the host's
// launch size is known before.  A unit cut between CTAs is joined by the one that
// finishes last, in a fixed order (in two levels where it spans many CTAs).
//
// A producer warp looks up pages and has TMA copy their rows, as 128-byte
// swizzled columns, into a ring; four warps take a quarter of each tile's keys
// each: scores by mma.sync m16n8k16 (fp32: three tf32 products), a softmax of
// their own, then the product with V, and join at the end of a unit.  mma.sync
// and not tcgen05: at most 16 rows meet a key, and the copies set the pace.
#include <algorithm>
#include <cmath>

#include "cache.h"
#include "internal.h"
#include "tc_ptx.cuh"

namespace {

using namespace ppc;
using namespace ppc_ptx;

constexpr int kRows = 16;      // query rows of a unit
constexpr int kWarps = 4;      // that compute; one more copies
constexpr int kThreads = kWarps * 32 + 32;
constexpr int kGroup = 16;     // parts of a unit joined at once
constexpr int kMaxCtas = 512;  // kGroup^2 parts and more
constexpr int kJoin = kMaxCtas / kGroup;
constexpr int kPieces = 8;     // boxes down a tile at most (pages of 8)

struct AttnParams {
  const void* q;
  int64_t q_ts, q_hs;
  const void *k, *v;
  const int *starts, *table, *lens, *sel;
  void* out;
  float* lse;
  int* status;
  int* counters;   // [CTAs][3], zero between calls
  float* partial;  // [CTAs][2] x (16 rows of DP sums, 16 maxima, 16 totals)
  float scale;
  int T, B, H, G, D, page, pages, width, keep, causal;
};

template <class T, int DP>
struct Shape {
  static constexpr int E = sizeof(T);
  static constexpr int TK = E == 4 ? 32 : 64;   // keys per tile
  static constexpr int KW = TK / kWarps;        // keys per warp
  static constexpr int CH = 128 / E;            // values per 128-byte column
  static constexpr int NCH = DP / CH;
  static constexpr int TILE = TK * DP * E;      // bytes of a K or V tile
  static constexpr int CTAS = DP <= 128 ? 2 : 1;
  static constexpr int QS = E == 4 ? kRows * (DP + 4) * 4 : 0;  // fp32 queries stay in shared memory
  static constexpr int AS = DP + 8;             // row stride of the joining buffer: rows 8 banks apart
  static constexpr int ACC = kRows * AS * 4;
  // as many stages as fit: with 228 KB per SM, 1 KB of it taken and 6 KB static per CTA, 190 KB are in flight (16 bits)
  static constexpr int STAGES = (233472 / CTAS - 1024 - 6144 - 1024 - ACC - QS) / (2 * TILE);
  static constexpr int SMEM = STAGES * 2 * TILE + ACC + QS + 1024;
  static constexpr int PART = kRows * DP + 2 * kRows;  // floats of a partial result
};

struct Stage {          // what the producer says of a tile
  int have[kPieces];    // keys of each piece that the call may use
  int full;             // all of them
};

__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) {
  for (long i = 0; i < PP_WAIT_POLLS; ++i)
    if (mbar_try(bar, parity)) return true;
  return false;
}

__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* m, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(m), "r"(x), "r"(y), "r"(bar)
      : "memory");
}

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
__device__ __forceinline__ void mma8(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// v = hi + lo with hi exact in tf32; the dropped part of lo is below 2^-21 |v|
__device__ __forceinline__ void split_tf32(float v, uint32_t& hi, uint32_t& lo) {
  const float h = tf32_hi(v);
  hi = __float_as_uint(h);
  lo = __float_as_uint(v - h);
}
// c += a b with fp32 operands as three tf32 products (lo lo, below 2^-22, is left out)
__device__ __forceinline__ void mma8x3(float (&c)[4], const uint32_t (&ah)[4], const uint32_t (&al)[4], float b0, float b1) {
  uint32_t h0, l0, h1, l1;
  split_tf32(b0, h0, l0);
  split_tf32(b1, h1, l1);
  mma8(c, al, h0, h1);
  mma8(c, ah, l0, l1);
  mma8(c, ah, h0, h1);
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <class T>
__device__ __forceinline__ uint32_t pack(float a, float b) {
  T v[2] = {from_f32<T>(a), from_f32<T>(b)};
  uint32_t r;
  memcpy(&r, v, 4);
  return r;
}

// Walks the units' tiles in their one order.  An item is a sequence, or a token where pages are selected for each
// token; its units are (16 rows, head) pairs of kt tiles each.
struct Walk {
  int64_t base;  // its first tile in the order
  int item, t0, n, len, rows, kt;
  int64_t units;
};
__device__ __forceinline__ void load_item(const AttnParams& p, int TK, int i, Walk& w) {
  w.item = i;
  int seen;
  if (p.sel) {
    const Seen s = seen_keys(i, p.T, p.B, p.starts, p.lens, p.width * p.page, p.causal, p.status);
    w.t0 = i;
    w.n = 1;
    w.len = s.keys;
    seen = min(p.keep, (s.keys + p.page - 1) / p.page) * p.page;
  } else {
    w.t0 = p.starts ? p.starts[i] : i;
    w.n = p.starts ? p.starts[i + 1] - w.t0 : 1;
    int len = p.lens[i];
    const int most = p.width * p.page;
    if (w.t0 < 0 || w.n < 0 || w.t0 + (int64_t)w.n > p.T || len < 0 || len > most) {
      atomicOr(p.status, PP_CACHE_BAD_LENGTH);
      if (w.t0 < 0 || w.n < 0 || w.t0 + (int64_t)w.n > p.T) w.n = 0;
      len = min(max(len, 0), most);
    }
    w.len = len;
    seen = len;
  }
  w.rows = w.n * p.G;
  w.units = (int64_t)((w.rows + kRows - 1) / kRows) * p.H;
  w.kt = max(1, (seen + TK - 1) / TK);
}

// One row's attention over keys j0 .. j1 - 1 of a sequence by one warp, one key after the other.
template <class T, int DP>
__device__ __noinline__ void redo_row(const AttnParams& p, const T* q, const int* row, int h, int j0, int j1, float sl,
                                      float* acc, float* rm, float* rl) {
  const int lane = threadIdx.x % 32;
  float o[DP / 32], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) o[i] = 0.f;
  for (int j = j0; j < j1; ++j) {
    const int id = row[j / p.page];
    if (id < 0 || id >= p.pages) continue;
    const int64_t at = (((int64_t)id * p.H + h) * p.page + j % p.page) * p.D;
    float x = 0.f;
    for (int d = lane; d < p.D; d += 32) x += to_f32(q[d]) * to_f32(static_cast<const T*>(p.k)[at + d]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    x *= sl;
    const float mx = fmaxf(m, x), ref = mx == -INFINITY ? 0.f : mx, f = ex2(m - ref), e = ex2(x - ref);
    m = mx;
    l = l * f + e;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
      if (lane + 32 * i < p.D) o[i] = o[i] * f + e * to_f32(static_cast<const T*>(p.v)[at + lane + 32 * i]);
  }
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) acc[lane + 32 * i] = o[i];
  if (lane == 0) {
    *rm = m;
    *rl = l;
  }
}

template <class T, int DP>
__global__ void __launch_bounds__(kThreads, Shape<T, DP>::CTAS)
    attn_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap mk,
                const __grid_constant__ CUtensorMap mv) {
  using S = Shape<T, DP>;
  constexpr int TK = S::TK, KW = S::KW, ST = S::STAGES;
  extern __shared__ unsigned char raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  float* acc = reinterpret_cast<float*>(smem + ST * 2 * S::TILE);
  [[maybe_unused]] float* qs = acc + kRows * S::AS;
  __shared__ alignas(8) uint64_t full_bar[ST], empty_bar[ST];
  __shared__ Stage stage[ST];
  __shared__ float wm[kWarps][kRows], wl[kWarps][kRows], rm[kRows], rl[kRows];
  __shared__ float wts[kRows][kJoin + 1], sums[kRows][kJoin + 1];
  __shared__ int64_t scan[kThreads / 32];
  __shared__ int64_t found_base;
  __shared__ int found_item, last_flag, dead;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const int NI = p.sel ? p.T : p.B;

  if (tid == 0) {
    dead = 0;
    found_item = -1;
    for (int i = 0; i < ST; ++i) {
      mbar_init(su32(&full_bar[i]), 1);
      mbar_init(su32(&empty_bar[i]), kWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // every thread sums a run of items; a scan of the sums places them in the one order
  const int per = (NI + kThreads - 1) / kThreads;
  const int i0 = min(NI, tid * per), i1 = min(NI, i0 + per);
  int64_t mine = 0;
  Walk w;
  for (int i = i0; i < i1; ++i) {
    load_item(p, TK, i, w);
    mine += w.units * w.kt;
  }
  int64_t before = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(~0u, before, d);
    if (lane >= d) before += o;
  }
  if (lane == 31) scan[warp] = before;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) {
    if (i < warp) before += scan[i];
    total += scan[i];
  }
  before -= mine;
  // equal runs; one of a single tile would spend more on joining than on its keys
  const int64_t run = max((total + gridDim.x - 1) / (int64_t)gridDim.x, (int64_t)2);
  const int64_t x0 = (int64_t)blockIdx.x * run, x1 = min(total, x0 + run);
  if (x0 >= total) return;
  if (x0 >= before && x0 < before + mine) {
    for (int i = i0;; ++i) {
      load_item(p, TK, i, w);
      const int64_t c = w.units * w.kt;
      if (x0 < before + c) {
        found_item = i;
        found_base = before;
        break;
      }
      before += c;
    }
  }
  __syncthreads();
  load_item(p, TK, found_item, w);
  w.base = found_base;
  const int BR = min(p.page, TK), pieces = TK / BR;
  const float sl = p.scale * 1.44269504f;  // softmax in powers of two

  // the unit at x: its rows, head and tiles up to this CTA's end
  auto settle = [&](int64_t x) {
    while (x - w.base >= w.units * w.kt) {
      const int64_t b = w.base + w.units * w.kt;
      load_item(p, TK, w.item + 1, w);
      w.base = b;
    }
  };

  if (warp == kWarps) {
    // ---- producer: lane j < pieces looks after piece j of each tile
    int s = 0;
    uint32_t ph = 1;  // an empty ring
    for (int64_t x = x0; x < x1;) {
      settle(x);
      const int64_t u = (x - w.base) / w.kt;
      const int h = (int)(u % p.H), k0 = (int)((x - w.base) % w.kt), k1 = (int)min((int64_t)w.kt, k0 + x1 - x);
      const int b = p.sel ? seen_keys(w.t0, p.T, p.B, p.starts, p.lens, p.width * p.page, p.causal, p.status).b : w.item;
      const int* row = p.table + (int64_t)b * p.width;
      const int* list = p.sel ? p.sel + ((int64_t)w.t0 * p.H + h) * p.keep : nullptr;
      for (int k = k0; k < k1; ++k) {
        int have = 0;
        int64_t y = 0;
        if (lane < pieces) {
          const int key = k * TK + lane * BR, off = key % p.page;  // key of the sequence, or of the list's pages in a row
          int at = key / p.page;
          bool ok = true;
          if (list) {
            ok = at < p.keep;
            at = ok ? list[at] : -1;
            if (at >= p.width) atomicOr(p.status, PP_CACHE_BAD_PAGE);
            ok = at >= 0 && at < p.width;
          }
          have = ok ? min(BR, w.len - at * p.page - off) : 0;
          if (have > 0) {
            const int id = row[at];
            if (id < 0 || id >= p.pages) {
              atomicOr(p.status, PP_CACHE_BAD_PAGE);
              have = 0;
            }
            y = ((int64_t)id * p.H + h) * p.page + off;
          }
          have = max(have, 0);
        }
        const unsigned live = __ballot_sync(~0u, have > 0), whole = __ballot_sync(~0u, have == BR);
        if (!*(volatile int*)&dead && !wait(su32(&empty_bar[s]), ph)) dead = 1;
        __syncwarp();
        const bool go = !*(volatile int*)&dead;
        if (lane < pieces) stage[s].have[lane] = have;
        if (lane == 0) stage[s].full = __popc(whole) == pieces;
        __syncwarp();
        if (lane == 0) mbar_arrive_expect_tx(su32(&full_bar[s]), go ? __popc(live) * 2 * BR * DP * S::E : 0);
        __syncwarp();
        const uint32_t dst = su32(smem + s * 2 * S::TILE);
        const int boxes = pieces * S::NCH * 2;  // box i: piece i % pieces, column and pool i / pieces
        for (int i = lane; i - lane < boxes; i += 32) {
          const int j = i % pieces, c = i / pieces % S::NCH, v = i / pieces / S::NCH;
          const int yy = __shfl_sync(~0u, (int)y, j);
          if (go && i < boxes && (live >> j & 1))
            copy_box(dst + v * S::TILE + c * TK * 128 + j * BR * 128, v ? &mv : &mk, c * S::CH, yy, su32(&full_bar[s]));
        }
        __syncwarp();
        if (++s == ST) {
          s = 0;
          ph ^= 1;
        }
      }
      x += k1 - k0;
    }
    return;
  }

  // ---- consumers
  constexpr int NT = KW / 8, ND = DP / 8;
  const int g = lane / 4, t = lane % 4;
  const T* q = static_cast<const T*>(p.q);
  const bool even = ((reinterpret_cast<uintptr_t>(q) & 3) | (p.q_ts & 1) | (p.q_hs & 1)) == 0;
  int s = 0;
  uint32_t ph = 0;
  bool timed_out = false;
  for (int64_t x = x0; x < x1;) {
    settle(x);
    const int64_t u = (x - w.base) / w.kt;
    const int h = (int)(u % p.H), r0 = (int)(u / p.H) * kRows;
    const int k0 = (int)((x - w.base) % w.kt), k1 = (int)min((int64_t)w.kt, k0 + x1 - x);
    const int nrows = min(kRows, w.rows - r0);
    const bool listed = p.sel != nullptr;
    // keys that a row of the unit may see
    auto limit = [&](int r) {
      return p.causal && !listed ? min(w.len, max(0, w.len - w.n + (r0 + r) / p.G + 1)) : w.len;
    };
    const int lim[2] = {limit(min(g, nrows - 1)), limit(min(g + 8, nrows - 1))};
    const int lim_min = limit(0), lim_max = limit(nrows - 1);
    // the row's queries: token r / G of the unit's, head r % G of the group's
    auto qrow = [&](int r) {
      return q + (w.t0 + (r0 + r) / p.G) * p.q_ts + (int64_t)(h * p.G + (r0 + r) % p.G) * p.q_hs;
    };
    [[maybe_unused]] uint32_t qf[S::E == 2 ? DP / 16 : 1][4];
    if constexpr (S::E == 2) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int r = g + 8 * half;
        const T* x = qrow(min(r, nrows - 1));
#pragma unroll
        for (int kk = 0; kk < DP / 16; ++kk)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int d = kk * 16 + e * 8 + 2 * t;
            uint32_t v = 0;
            if (r < nrows && d < p.D) {
              if (even) {
                v = *reinterpret_cast<const uint32_t*>(x + d);
              } else {
                T two[2] = {x[d], x[d + 1]};
                memcpy(&v, two, 4);
              }
            }
            qf[kk][half + 2 * e] = v;
          }
      }
    } else {
      group_sync<kWarps * 32>();  // the last unit's are read
      for (int i = tid; i < kRows * DP; i += kWarps * 32) {
        const int r = i / DP, d = i % DP;
        qs[r * (DP + 4) + d] = r < nrows && d < p.D ? to_f32(qrow(r)[d]) : 0.f;
      }
      group_sync<kWarps * 32>();
    }
    float o[ND][4];
#pragma unroll
    for (int i = 0; i < ND; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    for (int k = k0; k < k1; ++k) {
      if (!*(volatile int*)&dead && !wait(su32(&full_bar[s]), ph)) dead = 1;
      __syncwarp();
      timed_out = timed_out || *(volatile int*)&dead;
      const uint32_t kt = su32(smem + s * 2 * S::TILE), vt = kt + S::TILE;
      // ---- scores of this warp's keys
      float sc[NT][4];
#pragma unroll
      for (int i = 0; i < NT; ++i) sc[i][0] = sc[i][1] = sc[i][2] = sc[i][3] = 0.f;
      if constexpr (S::E == 2) {
        const int key = warp * KW + (lane / 16) * 8 + lane % 8;
#pragma unroll
        for (int kk = 0; kk < DP / 16; ++kk) {
          uint32_t b[4];
          ldsm4(kt + kk / 4 * TK * 128 + key * 128 + ((((kk % 4) * 2 + (lane / 8 & 1)) ^ (key & 7)) << 4), b);
          mma16<T>(sc[0], qf[kk], b[0], b[1]);
          mma16<T>(sc[1], qf[kk], b[2], b[3]);
        }
      } else {
        const int key = warp * KW + g;
        const float* kp = reinterpret_cast<const float*>(smem + s * 2 * S::TILE);
#pragma unroll 4
        for (int kk = 0; kk < DP / 8; ++kk) {
          const float* row = kp + kk / 4 * TK * 32 + key * 32;
          const int c = kk % 4 * 2;
          uint32_t ah[4], al[4];
          split_tf32(qs[g * (DP + 4) + kk * 8 + t], ah[0], al[0]);
          split_tf32(qs[(g + 8) * (DP + 4) + kk * 8 + t], ah[1], al[1]);
          split_tf32(qs[g * (DP + 4) + kk * 8 + t + 4], ah[2], al[2]);
          split_tf32(qs[(g + 8) * (DP + 4) + kk * 8 + t + 4], ah[3], al[3]);
          mma8x3(sc[0], ah, al, row[((c ^ (key & 7)) << 2) + t], row[(((c + 1) ^ (key & 7)) << 2) + t]);
        }
      }
      const Stage& sg = stage[s];
      const bool clean = sg.full && (listed || (k + 1) * TK <= lim_min);
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sc[i][e] *= sl;
          if (!clean) {
            const int j = warp * KW + i * 8 + 2 * t + (e & 1);
            if (j % BR >= sg.have[j / BR] || (!listed && k * TK + j >= lim[e >> 1])) sc[i][e] = -INFINITY;
          }
        }
      if (!clean) {  // values that no row sees: 0 x them has to be 0
#pragma unroll
        for (int i = 0; i < KW; ++i) {
          const int j = warp * KW + i;
          if (j % BR >= sg.have[j / BR] || (!listed && k * TK + j >= lim_max))
            for (int c = lane; c < S::NCH * 8; c += 32)
              *reinterpret_cast<uint4*>(smem + s * 2 * S::TILE + S::TILE + c / 8 * TK * 128 + j * 128 + c % 8 * 16) =
                  make_uint4(0, 0, 0, 0);
        }
        __syncwarp();
      }
      // ---- softmax over what this warp has seen
      float f[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float mx = fmaxf(sc[0][2 * r], sc[0][2 * r + 1]);
        if (NT == 2) mx = fmaxf(mx, fmaxf(sc[NT - 1][2 * r], sc[NT - 1][2 * r + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 1));
        mx = fmaxf(m[r], fmaxf(mx, __shfl_xor_sync(~0u, mx, 2)));
        const float at = mx == -INFINITY ? 0.f : mx;
        f[r] = ex2(m[r] - at);
        m[r] = mx;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          sc[i][2 * r] = ex2(sc[i][2 * r] - at);
          sc[i][2 * r + 1] = ex2(sc[i][2 * r + 1] - at);
          sum += sc[i][2 * r] + sc[i][2 * r + 1];
        }
        l[r] = l[r] * f[r] + sum;
      }
      if (__any_sync(~0u, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
        for (int i = 0; i < ND; ++i) {
          o[i][0] *= f[0];
          o[i][1] *= f[0];
          o[i][2] *= f[1];
          o[i][3] *= f[1];
        }
      }
      // ---- their product with V
      if constexpr (S::E == 2) {
        // the weights as two halves of the inputs' type, so that they keep 16 bits and more (22 in f16): bound by the
        // copies, the kernel has the time, and the output's own rounding stays the largest error
        uint32_t ph4[4], pl4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = sc[i / 2][i % 2 * 2], b = sc[i / 2][i % 2 * 2 + 1];
          ph4[i] = pack<T>(a, b);
          T two[2];
          memcpy(two, &ph4[i], 4);
          pl4[i] = pack<T>(a - to_f32(two[0]), b - to_f32(two[1]));
        }
        const int key = warp * KW + (lane / 8 & 1) * 8 + lane % 8;
#pragma unroll
        for (int i = 0; i < ND; i += 2) {
          uint32_t b[4];
          ldsm4t(vt + i / 8 * TK * 128 + key * 128 + (((i % 8 + lane / 16) ^ (key & 7)) << 4), b);
          mma16<T>(o[i], ph4, b[0], b[1]);
          mma16<T>(o[i + 1], ph4, b[2], b[3]);
          mma16<T>(o[i], pl4, b[0], b[1]);
          mma16<T>(o[i + 1], pl4, b[2], b[3]);
        }
      } else {
        // columns t and t + 4 of the product's left side are keys 2t and 2t + 1: the sum does not mind
        uint32_t ah[4], al[4];
        split_tf32(sc[0][0], ah[0], al[0]);
        split_tf32(sc[0][2], ah[1], al[1]);
        split_tf32(sc[0][1], ah[2], al[2]);
        split_tf32(sc[0][3], ah[3], al[3]);
        const float* vp = reinterpret_cast<const float*>(smem + s * 2 * S::TILE + S::TILE);
        const int key = warp * KW + 2 * t;
#pragma unroll
        for (int i = 0; i < ND; ++i) {
          const float* row = vp + i / 4 * TK * 32 + key * 32;
          const int c = i % 4 * 2 + g / 4;
          mma8x3(o[i], ah, al, row[((c ^ (key & 7)) << 2) + g % 4], row[32 + ((c ^ (key + 1 & 7)) << 2) + g % 4]);
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
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(~0u, l[r], 1);
      l[r] += __shfl_xor_sync(~0u, l[r], 2);
      if (t == 0) {
        wm[warp][g + 8 * r] = m[r];
        wl[warp][g + 8 * r] = l[r];
      }
    }
    group_sync<kWarps * 32>();
    float f[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int row = g + 8 * r;
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) mx = fmaxf(mx, wm[i][row]);
      f[r] = m[r] == -INFINITY ? 0.f : ex2(m[r] - mx);
      if (warp == 0 && t == 0) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) sum += wm[i][row] == -INFINITY ? 0.f : wl[i][row] * ex2(wm[i][row] - mx);
        rm[row] = mx;
        rl[row] = sum;
      }
    }
#pragma unroll 1
    for (int i = 0; i < kWarps; ++i) {
      if (warp == i) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if (g + 8 * r >= nrows) continue;
          float* row = acc + (g + 8 * r) * S::AS + 2 * t;
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            float2 v = i == 0 ? make_float2(0.f, 0.f) : *reinterpret_cast<float2*>(row + d * 8);
            v.x += o[d][2 * r] * f[r];
            v.y += o[d][2 * r + 1] * f[r];
            *reinterpret_cast<float2*>(row + d * 8) = v;
          }
        }
      }
      group_sync<kWarps * 32>();
    }
    // a product with 0 of a value that is not finite, at a key that this row does not see and another does: such rows again
    if (lim_min != lim_max) {
      bool bad = false;
      for (int i = tid; i < nrows * p.D; i += kWarps * 32) bad = bad || !isfinite(acc[i / p.D * S::AS + i % p.D]);
      if (group_any<kWarps * 32>(bad)) {
        for (int r = warp; r < nrows; r += kWarps)
          redo_row<T, DP>(p, qrow(r), p.table + (int64_t)w.item * p.width, h, k0 * TK, min(k1 * TK, limit(r)), sl,
                          acc + r * S::AS, rm + r, rl + r);
        group_sync<kWarps * 32>();
      }
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
                 ((int64_t)(w.t0 + (r0 + r) / p.G) * p.H * p.G + h * p.G + (r0 + r) % p.G) * p.D + d;
        if (wide) {
          *reinterpret_cast<Vec<T, 4>*>(dst) = y;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) dst[e] = y.v[e];
        }
      }
      if (p.lse && tid < nrows)
        p.lse[(int64_t)(w.t0 + (r0 + tid) / p.G) * p.H * p.G + h * p.G + (r0 + tid) % p.G] =
            rl[tid] == 0.f ? -INFINITY : rm[tid] * 0.693147181f + logf(rl[tid]);
    };
    const int64_t first = w.base + u * w.kt;  // the unit's first tile
    const int c0 = (int)(first / run), parts = (int)((first + w.kt - 1) / run) - c0 + 1;
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
            sum += c == 0.f ? 0.f : c * sums[tid][i];
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
    x += k1 - k0;
  }
  if (timed_out) {
    if (lane == 0) atomicOr(p.status, PP_CACHE_TIMEOUT);
    if (tid == 0)  // copies still in flight end before the CTA does
      for (int i = 0; i < ST; ++i) wait(su32(&full_bar[i]), 0), wait(su32(&full_bar[i]), 1);
  }
}

template <class T, int DP>
cudaError_t prepare_one() {
  return cudaFuncSetAttribute(attn_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<T, DP>::SMEM);
}

template <class T, int DP>
cudaError_t launch(const AttnParams& p, const pp_cache& c, int sms, cudaStream_t stream) {
  const int grid = std::min(sms * Shape<T, DP>::CTAS, kMaxCtas);
  attn_kernel<T, DP><<<grid, kThreads, Shape<T, DP>::SMEM, stream>>>(p, c.mk, c.mv);
  return cudaGetLastError();
}

template <class T>
cudaError_t by_head(const AttnParams& p, const pp_cache& c, int sms, cudaStream_t stream) {
  return p.D <= 64    ? launch<T, 64>(p, c, sms, stream)
         : p.D <= 128 ? launch<T, 128>(p, c, sms, stream)
                      : launch<T, 256>(p, c, sms, stream);
}

template <class T>
cudaError_t prepare_type() {
  cudaError_t e = prepare_one<T, 64>();
  if (e == cudaSuccess) e = prepare_one<T, 128>();
  if (e == cudaSuccess) e = prepare_one<T, 256>();
  return e;
}

DeviceOnce g_attn_once;

}  // namespace

namespace ppc {

AttnSpace attn_space(int, int D, int sms) {
  const int DP = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  const size_t ctas = (size_t)std::min(sms * (DP <= 128 ? 2 : 1), kMaxCtas);
  return {ctas * 3 * 4, ctas * 2 * (kRows * DP + 2 * kRows) * 4};
}

cudaError_t attn_prepare() {
  return g_attn_once.run([](int) {
    cudaError_t e = prepare_type<float>();
    if (e == cudaSuccess) e = prepare_type<__half>();
    if (e == cudaSuccess) e = prepare_type<__nv_bfloat16>();
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
  if ((int64_t)width * cache->page > INT32_MAX) return PP_ERR_UNSUPPORTED;
  const int sms = device_sms();
  if (sms <= 0) return PP_ERR_CUDA;
  const pp_cache& c = *cache;
  AttnParams p = {q, q_ts, q_hs, c.k, c.v, starts, table, lens, sel, out, lse, c.status, c.counters, c.partial, scale, T, B, c.H,
                  Hq / c.H, c.D, c.page, c.pages, width, keep, flags & PP_ATTN_CAUSAL};
  const cudaStream_t s = (cudaStream_t)stream;
  const cudaError_t e = c.dtype == PP_F32   ? by_head<float>(p, c, sms, s)
                        : c.dtype == PP_F16 ? by_head<__half>(p, c, sms, s)
                                            : by_head<__nv_bfloat16>(p, c, sms, s);
  return e == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}
