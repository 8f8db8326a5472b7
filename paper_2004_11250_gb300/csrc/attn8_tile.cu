// Attention for many query tokens over a cache in 8 bits: two tiles of 128 query
// rows to a CTA on the tensor cores (tcgen05), for 16-bit types and heads of up to
// 128 values.
//
// The tensor cores take codes as f16, in which they are exact, so somebody has to
// turn each byte into two.  Four warps do so once for two tiles: they load a block of
// 64 keys (the next one's while they write this one's), and write it as the swizzled
// operands that a copy of f16 would have made.  Per block and tile, as in attn_tile.cu:
//   S = Q K^T            128 x 64, queries in f16 (bf16 times a power of two per row)
//   P = 2^(S ks - m) vs  a thread per row; ks, vs are the page's scales, vs over the
//                        largest of the tile's pages, so that P stays below its bound
//   O += P V             P from TMEM (over S's own columns), V from shared memory
// and O is multiplied by the largest vs over the row's sum at the end.  Codes are
// finite, so a key that a row does not see adds 0 whatever it holds.
#include <algorithm>
#include <type_traits>

#include "attn_tc.cuh"
#include "internal.h"

namespace {

using namespace ppc_attn;

constexpr int kRowsT = 128;                       // query rows of a tile
constexpr int kSoft = 2 * kRowsT;                 // threads of the softmax
constexpr int kTurn = 128;                        // that turn codes into f16; then a multiplying warp, and three that idle
constexpr int kThreads8 = kSoft + kTurn + 128;
// Registers of a thread at launch, and after they are shared out by warpgroups: a row of 64 scores wants more than 128.
constexpr int kRegs = 128, kRegsSoft = 176, kRegsTurn = 96, kRegsMul = 64;
static_assert(2 * kRegsSoft + kRegsTurn + kRegsMul == 4 * kRegs && kThreads8 * kRegs == 65536, "what the block was launched with");
constexpr int kKeys = 64;                         // keys per block
constexpr int kStages = 2;                        // of K and of V
constexpr int kInfo = 8;                          // blocks whose notes are kept: the turning warps are up to 4 ahead of the softmax
constexpr int kSplits = 8;                        // shares of a tile's blocks at most
constexpr int kUp = 13;                           // weights are up to 2^13 where m is not behind, and 2^2 times that
constexpr float kGrow = 2.f;

template <int DP>
struct Shape8 {
  static constexpr int Q = kRowsT * DP * 2, KV = kKeys * DP * 2;
  static constexpr int SMEM = 2 * Q + 2 * kStages * KV + 1024;
  static constexpr int COLS = 512;  // TMEM: O of the tiles at 0 and 128, S at 256, 320 and 384, 448
};

struct alignas(16) Note {  // of a block
  float ks[8], vs[8];      // scales of each 8 keys; vs over the largest
  uint16_t valid[4];       // keys that are there, a bit each
};

template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// 16 codes as 16 f16 (attn_row.cuh has the same by bytes' parity)
__device__ __forceinline__ uint32_t f16_pair(uint32_t biased, uint32_t bytes) {
  const uint32_t w = __byte_perm(biased, 0x64646464u, bytes);  // 1024 + code + 128
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&w), __float2half2_rn(1152.f));
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 f16_of8(uint32_t a, uint32_t b) {
  a ^= 0x80808080u;
  b ^= 0x80808080u;
  return make_uint4(f16_pair(a, 0x4140), f16_pair(a, 0x4342), f16_pair(b, 0x4140), f16_pair(b, 0x4342));
}

template <class T, int DP>
__global__ void __launch_bounds__(kThreads8, 1) attn8_tile_kernel(const __grid_constant__ AttnParams p) {
  using S = Shape8<DP>;
  constexpr int CHUNK_Q = kRowsT * 128, CHUNK_KV = kKeys * 128;  // bytes of 64 values of every row
  extern __shared__ unsigned char raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  unsigned char* kbuf = smem + 2 * S::Q;
  unsigned char* vbuf = kbuf + kStages * S::KV;
  __shared__ alignas(8) uint64_t q_full[2], k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages], s_full[2][2],
      p_full[2][2], pv_done[2], note_full[kInfo];
  __shared__ Note notes[kInfo];
  __shared__ float row_scale[kSoft], most[kThreads8 / 32];
  __shared__ uint32_t tmem_s;
  __shared__ int scan[kThreads8 / 32], tile_of[4], dead;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;

  // ---- which tiles: those of a sequence's last tokens, which see the most keys, come first
  const int T1 = kRowsT / p.G.d, TT = 2 * T1;  // tokens of a tile, of the CTA's two
  const int z = blockIdx.x % p.splits, h = blockIdx.x / p.splits % p.H, order = blockIdx.x / p.splits / p.H;
  if (tid == 0) {
    dead = 0;
    tile_of[0] = -1;
  }
  __syncthreads();
  after_previous();
  const int per = (p.B + kThreads8 - 1) / kThreads8, b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
  int mine = 0;
  bool bad = false;
  for (int b = b0; b < b1; ++b) {
    const int s0 = p.starts[b], n = p.starts[b + 1] - s0;
    bad = bad || s0 < 0 || n < 0 || s0 > p.T - n;
    if ((b == 0 && s0 != 0) || (b == p.B - 1 && s0 + n != p.T)) atomicOr(p.status, PP_CACHE_BAD_LENGTH);
    mine += (max(n, 0) + TT - 1) / TT;
  }
  int before = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int up = __shfl_up_sync(~0u, before, d);
    if (lane >= d) before += up;
  }
  if (lane == 31) scan[warp] = before;
  if (__syncthreads_or(bad)) {
    if (tid == 0) atomicOr(p.status, PP_CACHE_BAD_LENGTH);
    return;
  }
  int total = 0;
#pragma unroll
  for (int i = 0; i < kThreads8 / 32; ++i) {
    if (i < warp) before += scan[i];
    total += scan[i];
  }
  before -= mine;
  if (order >= total) return;
  const int want = total - 1 - order;
  if (want >= before && want < before + mine) {
    for (int b = b0;; ++b) {
      const int s0 = p.starts[b], n = p.starts[b + 1] - s0, c = (n + TT - 1) / TT;
      if (want < before + c) {
        tile_of[0] = b;
        tile_of[1] = s0;
        tile_of[2] = n;
        tile_of[3] = (want - before) * TT;
        break;
      }
      before += c;
    }
  }
  __syncthreads();
  const int b = tile_of[0], t0 = tile_of[1] + tile_of[3], nt = min(TT, tile_of[2] - tile_of[3]);
  int len = p.lens[b];
  const int all = p.width * p.page;
  if (len < 0 || len > all) {
    if (tid == 0) atomicOr(p.status, PP_CACHE_BAD_LENGTH);
    len = min(max(len, 0), all);
  }
  // keys that token i of the two tiles sees
  auto limit = [&](int i) { return p.causal ? min(len, max(0, len - tile_of[2] + tile_of[3] + i + 1)) : len; };
  const int lim_min = limit(0), lim_max = limit(nt - 1);
  const int* table = p.table + (int64_t)b * p.width;
  // the first key of a window, and the blocks between the first keys' and the windows'
  const int low = max(0, lim_min - p.window), sink_blocks = (min(p.sinks, lim_max) + 63) >> 6, gap = max(0, (low >> 6) - sink_blocks);
  const int blocks = ((lim_max + 63) >> 6) - gap, first = (int)((int64_t)blocks * z / p.splits), n = (int)((int64_t)blocks * (z + 1) / p.splits) - first;
  auto key_of = [&](int k) { return (first + k < sink_blocks ? first + k : first + k + gap) << 6; };  // of the share's block k
  const bool two = nt > T1;
  // a negative scale goes into the queries, and so does 0 (with no queries, any scale): sl > 0
  const float sl = p.scale == 0.f ? 1.f : fabsf(p.scale) * 1.44269504f;

  // ---- set up
  if (warp == (kSoft + kTurn) / 32) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(su32(&tmem_s)), "n"(S::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(su32(&q_full[i]), kRowsT);
      mbar_init(su32(&pv_done[i]), 1);
      for (int j = 0; j < 2; ++j) {
        mbar_init(su32(&s_full[i][j]), 1);
        mbar_init(su32(&p_full[i][j]), kRowsT);
      }
    }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(su32(&k_full[i]), kTurn);
      mbar_init(su32(&k_empty[i]), 1);
      mbar_init(su32(&v_full[i]), kTurn);
      mbar_init(su32(&v_empty[i]), 1);
    }
    for (int i = 0; i < kInfo; ++i) mbar_init(su32(&note_full[i]), kTurn);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // the largest scale of values among the pages that some token sees
  float vtop = 0.f;
  {
    const int sinks = min(p.sinks, lim_max), pages0 = (sinks + p.page - 1) >> p.log_page, from = max(pages0, low >> p.log_page);
    const int count = pages0 + max(0, ((lim_max + p.page - 1) >> p.log_page) - from);
    for (int i = tid; i < count; i += kThreads8) {
      const int id = table[i < pages0 ? i : i - pages0 + from];
      if (id >= 0 && id < p.pages) vtop = fmaxf(vtop, p.vs[(int64_t)id * p.H + h]);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) vtop = fmaxf(vtop, __shfl_xor_sync(~0u, vtop, d));
    if (lane == 0) most[warp] = vtop;
  }
  tm_fence_before();
  __syncthreads();
  tm_fence_after();
#pragma unroll
  for (int i = 0; i < kThreads8 / 32; ++i) vtop = fmaxf(vtop, most[i]);
  const uint32_t tmem = tmem_s;
  // a bounded wait; after one gave up none waits any more
  auto hold = [&](uint64_t* bar, uint32_t parity) {
    if (mbar_try(su32(bar), parity) || *(volatile int*)&dead) return;
    if (!wait(su32(bar), parity)) dead = 1;
  };

  if (warp >= (kSoft + kTurn) / 32) {
    // ---- products
    fewer_registers<kRegsMul>();
    if (warp == (kSoft + kTurn) / 32) {
    const uint32_t leader = elect();
    const uint32_t qa = desc_lo(su32(smem), 16), kb = desc_lo(su32(kbuf), 16), vb = desc_lo(su32(vbuf), CHUNK_KV);
    auto scores = [&](int g) {
      const int st = g % kStages;
      hold(&k_full[st], g / kStages & 1);
      tm_fence_after();
      const uint32_t kd = kb + st * (S::KV >> 4);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (t && !two) break;
        const uint32_t to = tmem + 256 + t * 128 + (g & 1) * 64;
#pragma unroll
        for (int kk = 0; kk < DP / 16; ++kk)
          mma_ss(to, qa + (t * S::Q + kk / 4 * CHUNK_Q + kk % 4 * 32 >> 4), kd + (kk / 4 * CHUNK_KV + kk % 4 * 32 >> 4),
                 idesc<__half>(kRowsT, kKeys, false), kk > 0, leader);
        commit(su32(&s_full[t][g & 1]), leader);
      }
      commit(su32(&k_empty[st]), leader);
    };
    if (n > 0) {
      hold(&q_full[0], 0);
      if (two) hold(&q_full[1], 0);
      scores(0);
    }
    for (int g = 0; g < n; ++g) {
      const int st = g % kStages;
      if (g + 1 < n) scores(g + 1);
      hold(&v_full[st], g / kStages & 1);
      const uint32_t vd = vb + st * (S::KV >> 4);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (t && !two) break;
        hold(&p_full[t][g & 1], g >> 1 & 1);
        tm_fence_after();
        const uint32_t pt = tmem + 256 + t * 128 + (g & 1) * 64;
#pragma unroll
        for (int kk = 0; kk < kKeys / 16; ++kk)
          mma_ts(tmem + t * 128, pt + kk * 8, vd + (kk * 2048 >> 4), idesc<__half>(kRowsT, DP, true), g > 0 || kk > 0, leader);
        commit(su32(&pv_done[t]), leader);
      }
      commit(su32(&v_empty[st]), leader);
    }
    }
  } else if (warp >= kSoft / 32) {
    fewer_registers<kRegsTurn>();
    // ---- codes to f16: a warp has 16 keys of a block, which lie on one page, or on two of 8
    constexpr int CPR = DP / 16, RPL = 32 / CPR, NI = 16 / RPL;  // chunks of 16 codes to a row, rows to a load, loads
    const int w = warp - kSoft / 32, c = lane % CPR, r = lane / CPR;
    const bool in = c * 16 < p.D;
    struct Place {
      int64_t cell[2];  // of each 8 keys: (page id * H + h), -1: no key that is there
    };
    auto look = [&](int k) {
      Place at;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        at.cell[j] = -1;
        const int key = k < n ? key_of(k) + w * 16 + j * 8 : INT32_MAX;
        if (key < lim_max && (key < p.sinks || key + 8 > low)) {
          const int id = table[key >> p.log_page];
          if (id >= 0 && id < p.pages) at.cell[j] = (int64_t)id * p.H + h;
          else atomicOr(p.status, PP_CACHE_BAD_PAGE);
        }
      }
      return at;
    };
    auto load = [&](const void* pool, const Place& at, int k, uint4 (&x)[NI]) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int row = i * RPL + r;
        const int64_t cell = at.cell[row >> 3];
        x[i] = make_uint4(0, 0, 0, 0);
        if (in && cell >= 0)
          x[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const int8_t*>(pool) + (cell * p.page + (key_of(k) + w * 16 + row & p.page - 1)) * p.D + c * 16));
      }
    };
    auto write = [&](unsigned char* to, const uint4 (&x)[NI]) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int key = w * 16 + i * RPL + r;
        unsigned char* row = to + c / 4 * CHUNK_KV + key * 128;
        const uint4 lo = f16_of8(x[i].x, x[i].y), hi = f16_of8(x[i].z, x[i].w);
        // lanes of the second column write their halves the other way round, so that eight lanes meet eight banks
        const int e = DP == 128 ? c >> 2 : 0;
        *reinterpret_cast<uint4*>(row + ((c % 4 * 2 + e ^ key & 7) << 4)) = e ? hi : lo;
        *reinterpret_cast<uint4*>(row + ((c % 4 * 2 + 1 - e ^ key & 7) << 4)) = e ? lo : hi;
      }
    };
    const float vinv = vtop > 0.f ? 1.f / vtop : 0.f;
    uint4 kx[NI], vx[NI];
    Place here = look(0), next;
    if (n > 0) {
      load(p.k, here, 0, kx);
      load(p.v, here, 0, vx);
    }
    for (int g = 0; g < n; ++g) {
      const int st = g % kStages;
      const uint32_t ph = (g / kStages + 1) & 1;
      next = look(g + 1);
      hold(&k_empty[st], ph);
      if (lane < 2) {
        const int64_t cell = lane ? here.cell[1] : here.cell[0];
        notes[g % kInfo].ks[w * 2 + lane] = cell >= 0 ? p.ks[cell] : 0.f;
        notes[g % kInfo].vs[w * 2 + lane] = cell >= 0 ? p.vs[cell] * vinv : 0.f;
        if (lane == 0) notes[g % kInfo].valid[w] = (here.cell[0] >= 0 ? 0xFFu : 0u) | (here.cell[1] >= 0 ? 0xFF00u : 0u);
      }
      mbar_arrive(su32(&note_full[g % kInfo]));
      write(kbuf + st * S::KV, kx);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive(su32(&k_full[st]));
      if (g + 1 < n) load(p.k, next, g + 1, kx);
      hold(&v_empty[st], ph);
      write(vbuf + st * S::KV, vx);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive(su32(&v_full[st]));
      if (g + 1 < n) load(p.v, next, g + 1, vx);
      here = next;
    }
  } else {
    // ---- queries, then the softmax, a thread per row
    more_registers<kRegsSoft>();
    const int t = warp / 4, tr = tid % kRowsT, rows = (t ? nt - T1 : min(nt, T1)) * p.G.d;  // the tile, its row, its rows
    const bool some = rows > 0;
    const int base = t0 + t * T1;
    if (some) {
      // f16 as it is; bf16 times a power of two that brings the row's largest to 2^14.  A row is DP / 8 lanes
      constexpr int L = DP / 8, U = 4;
      const T* q = static_cast<const T*>(p.q);
      const bool wide = ((reinterpret_cast<uintptr_t>(q) & 15) | (p.q_ts & 7) | (p.q_hs & 7)) == 0;
      const float sign = p.scale < 0.f ? -1.f : p.scale == 0.f ? 0.f : 1.f;
#pragma unroll 1
      for (int i0 = tr; i0 < kRowsT * L; i0 += U * kRowsT) {
        Vec<T, 8> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int r = (i0 + u * kRowsT) / L, d = (i0 + u * kRowsT) % L * 8;
          const int fr = min(r, rows - 1);
          const T* from = q + (base + p.G.div(fr)) * p.q_ts + (int64_t)(h * p.G.d + p.G.mod(fr)) * p.q_hs + min(d, p.D - 8);
          if (wide) {
            v[u] = *reinterpret_cast<const Vec<T, 8>*>(from);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u].v[e] = from[e];
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int r = (i0 + u * kRowsT) / L, c = (i0 + u * kRowsT) % L;
          const bool used = r < rows && c * 8 < p.D;
          float f[8], up = 1.f, back = 1.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = used ? to_f32(v[u].v[e]) : 0.f;
          if constexpr (!std::is_same<T, __half>::value) {
            int top = 16;  // the largest exponent, of infinities and NaN the largest finite one; rows below 2^-111 keep fewer bits
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, min(__float_as_int(fabsf(f[e])) >> 23, 254));
#pragma unroll
            for (int m = 1; m < L; m <<= 1) top = max(top, __shfl_xor_sync(~0u, top, m));
            up = __int_as_float((268 - top) << 23);
            back = __int_as_float((top - 14) << 23);
          }
          if (c == 0) row_scale[t * kRowsT + r] = back;
          Vec<__half, 8> y;
#pragma unroll
          for (int e = 0; e < 8; ++e) y.v[e] = __float2half_rn(sign == 0.f ? 0.f : f[e] * (up * sign));
          *reinterpret_cast<Vec<__half, 8>*>(smem + t * S::Q + c / 8 * CHUNK_Q + r * 128 + ((c % 8 ^ (r & 7)) << 4)) = y;
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive(su32(&q_full[t]));
      // the rows of this tile's four warps
      asm volatile("bar.sync %0, %1;" ::"r"(1 + t), "n"(kRowsT) : "memory");
    }
    const bool live_row = tr < rows;
    const int tok = live_row ? t * T1 + p.G.div(tr) : 0;
    const int lim = live_row ? limit(tok) : 0;
    const float slr = some ? sl * row_scale[t * kRowsT + tr] : 0.f;
    const uint32_t row_tm = tmem + t * 128 + ((uint32_t)(warp % 4 * 32) << 16), s_tm = row_tm + 256;  // its sums, its scores
    float m = -INFINITY, l = 0.f;
    for (int g = 0; some && g < n; ++g) {
      const int key = key_of(g);
      const Note& note = notes[g % kInfo];
      hold(&note_full[g % kInfo], g / kInfo & 1);
      uint64_t see = *reinterpret_cast<const uint64_t*>(note.valid);
      see &= live_row ? below(lim - key) & (~below(lim - key - p.window) | below(p.sinks - key)) : 0;
      const bool part = __any_sync(~0u, live_row && see != ~0ull), none = __all_sync(~0u, see == 0);
      hold(&s_full[t][g & 1], g >> 1 & 1);
      __syncwarp();
      tm_fence_after();
      const uint32_t tm = s_tm + (g & 1) * 64;
      uint32_t w[32];
      bool waited = false;
      if (none) {
#pragma unroll
        for (int i = 0; i < 32; ++i) w[i] = 0;
      } else {
        float x[64];
        tm_ld32(tm, reinterpret_cast<float(&)[32]>(x[0]));
        tm_ld32(tm + 32, reinterpret_cast<float(&)[32]>(x[32]));
        float ks[8], vs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          ks[j] = __fmul_rn(note.ks[j], slr);
          vs[j] = note.vs[j];
        }
        tm_wait_ld();
        const uint64_t zero = pack2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 32; ++i)  // a product plus 0, so that it is rounded before the maximum is taken from it
          unpack2(fma2(pack2(x[2 * i], x[2 * i + 1]), pack2(ks[i / 4], ks[i / 4]), zero), x[2 * i], x[2 * i + 1]);
        if (part) {
#pragma unroll
          for (int i = 0; i < 64; ++i)
            if (!((i < 32 ? (uint32_t)see : (uint32_t)(see >> 32)) >> (i & 31) & 1)) x[i] = -INFINITY;
        }
        float top[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          top[c] = fmaxf(x[c], x[c + 4]);
#pragma unroll
          for (int i = 8; i < 64; i += 8) top[c] = fmaxf(top[c], fmaxf(x[i + c], x[i + c + 4]));
        }
        const float mx = lower(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), (float)kUp);
        const bool grow = mx > __fadd_rd(m, kGrow);  // from -infinity, too
        if (__any_sync(~0u, grow)) {
          const float to = fmaxf(m, mx), f = to == -INFINITY ? 1.f : ex2(m - to);
          m = to;
          l *= f;
          if (g > 0) {  // the sums so far, in TMEM
            hold(&pv_done[t], (g - 1) & 1);
            waited = true;
            __syncwarp();
            tm_fence_after();
#pragma unroll
            for (int c = 0; c < DP; c += 32) {
              float o[32];
              tm_ld32(row_tm + c, o);
              tm_wait_ld();
              uint32_t r[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(o[i] * f);
              tm_st32(row_tm + c, r);
            }
            tm_wait_st();
          }
        }
        const float at = m == -INFINITY ? 0.f : m;
        const uint64_t at2 = pack2(-at, -at);
        uint64_t sum[4] = {};
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          float a, c;
          unpack2(add2(pack2(x[2 * i], x[2 * i + 1]), at2), a, c);
          a = ex2(a);
          c = ex2(c);
          sum[i & 3] = add2(sum[i & 3], pack2(a, c));
          unpack2(fma2(pack2(a, c), pack2(vs[i / 4], vs[i / 4]), zero), a, c);
          w[i] = pack<__half>(a, c);
        }
        float a, c;
        unpack2(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), a, c);
        l += a + c;
      }
      tm_st32(tm, w);
      tm_wait_st();
      // each block's products with V are waited for, and in order, so that a parity names one of two phases
      if (g > 0 && !waited) hold(&pv_done[t], (g - 1) & 1);
      tm_fence_before();
      mbar_arrive(su32(&p_full[t][g & 1]));
    }

    // ---- out
    if (some) {
      if (n > 0) hold(&pv_done[t], (n - 1) & 1);
      __syncwarp();
      tm_fence_after();
      const int64_t cell = (int64_t)(base + p.G.div(live_row ? tr : 0)) * p.H * p.G.d + h * p.G.d + p.G.mod(live_row ? tr : 0);
      const bool parts = p.splits > 1;
      // (the joining kernel takes bf16's sums as not lifted)
      const float lift = std::is_same<T, __half>::value ? 1.f : 1.f / (float)(1 << kUp);
      const float scale = parts ? vtop * lift : l == 0.f ? 0.f : vtop / l;
      const int64_t at = (int64_t)z * p.T * p.H * p.G.d + cell;
      T* dst = static_cast<T*>(p.out) + cell * p.D;
      const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 15) == 0;
#pragma unroll
      for (int c = 0; c < DP; c += 32) {
        float o[32];
        if (n > 0) {
          tm_ld32(row_tm + c, o);
          tm_wait_ld();
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = 0.f;
        }
        if (!live_row) continue;
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] *= scale;
        if (parts) {
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            *reinterpret_cast<float4*>(p.split_sums + at * DP + c + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
        } else {
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            if (c + i >= p.D) continue;
            Vec<T, 8> y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y.v[e] = from_f32<T>(o[i + e]);
            if (wide) {
              *reinterpret_cast<Vec<T, 8>*>(dst + c + i) = y;
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) dst[c + i + e] = y.v[e];
            }
          }
        }
      }
      if (live_row) {
        if (parts) p.split_stats[at] = make_float2(lift == 1.f ? m : m + (float)kUp, l * lift);
        else if (p.lse) p.lse[cell] = l == 0.f ? -INFINITY : log_sum<__half, kUp>(m, l);
      }
    }
    tm_fence_before();
  }
  __syncthreads();
  if (dead && tid == 0) {
    atomicOr(p.status, PP_CACHE_TIMEOUT);
    // products still in flight end before the CTA does
    for (int i = 0; i < 2; ++i)
      for (uint32_t ph = 0; ph < 2; ++ph) wait(su32(&pv_done[i]), ph);
  }
  if (warp == (kSoft + kTurn) / 32) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::COLS));
  }
}

template <class T, int DP>
cudaError_t prepare_one() {
  // warps that ask for more registers than the block has would wait for ever: it has to be launched with what they add up to
  cudaFuncAttributes at;
  const cudaError_t e = cudaFuncGetAttributes(&at, attn8_tile_kernel<T, DP>);
  if (e != cudaSuccess) return e;
  if (at.numRegs != kRegs) return cudaErrorInvalidConfiguration;
  return cudaFuncSetAttribute(attn8_tile_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape8<DP>::SMEM);
}

template <class T, int DP>
cudaError_t launch(const AttnParams& p, int64_t grid, cudaStream_t stream) {
  const cudaError_t e = launch_after(attn8_tile_kernel<T, DP>, dim3((unsigned)grid), kThreads8, Shape8<DP>::SMEM, stream, 1, p);
  return e != cudaSuccess || p.splits == 1 ? e : tile_join(p, std::is_same<T, __half>::value ? PP_F16 : PP_BF16, stream);
}

// Pairs of tiles of a call at most: each sequence adds at most one that is not full.
int64_t most_pairs(const AttnParams& p) { return ((int64_t)p.T / (2 * (kRowsT / p.G.d)) + std::min(p.T, p.B)) * p.H; }

}  // namespace

namespace ppc_attn {

bool tile8_applicable(const AttnParams& p, int dtype, int sms) {
  if (dtype == PP_F32 || p.D > 128 || p.G.d > 64 || !p.starts) return false;
  const int64_t few = 2 * sms / kSplits, pairs = most_pairs(p), units = ((int64_t)p.T * p.G.d + 15) / 16 * p.H;
  return few < units && pairs * 8 <= units * 9;
}

cudaError_t tile8_prepare() {
  cudaError_t e = prepare_one<__half, 64>();
  if (e == cudaSuccess) e = prepare_one<__half, 128>();
  if (e == cudaSuccess) e = prepare_one<__nv_bfloat16, 64>();
  if (e == cudaSuccess) e = prepare_one<__nv_bfloat16, 128>();
  return e;
}

cudaError_t tile8_launch(AttnParams p, const pp_cache& c, int sms, cudaStream_t stream) {
  const int TT = 2 * (kRowsT / p.G.d), DP = p.D <= 64 ? 64 : 128;
  const int64_t pairs = most_pairs(p);  // CTAs beyond the last tile leave
  // Few tiles are split along their blocks, up to one CTA per SM, while a share can have 4 blocks; the shares' sums have room for
  // two tiles per SM.
  const int64_t cells = (int64_t)p.T * p.H * p.G.d, room = (int64_t)2 * sms * kRowsT;
  const int64_t keys = std::min<int64_t>((int64_t)p.width * p.page, (int64_t)p.window + p.sinks + TT + 2 * kKeys);
  const int64_t splits = std::min({(int64_t)kSplits, sms / pairs, keys / kKeys / 4, room / cells});
  p.splits = (int)std::max<int64_t>(1, splits);
  p.split_sums = c.tiles;
  p.split_stats = reinterpret_cast<float2*>(c.tiles + room * DP);
  const int64_t grid = pairs * p.splits;
  if (grid > INT32_MAX) return cudaErrorInvalidValue;
  return c.dtype == PP_F16 ? (DP == 64 ? launch<__half, 64>(p, grid, stream) : launch<__half, 128>(p, grid, stream))
                           : (DP == 64 ? launch<__nv_bfloat16, 64>(p, grid, stream) : launch<__nv_bfloat16, 128>(p, grid, stream));
}

}  // namespace ppc_attn
