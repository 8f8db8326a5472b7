// Attention for many query tokens over a cache in 8 bits: two tiles of 128 query
// rows to a CTA on the tensor cores (tcgen05), for 16-bit types and heads of up to
// 128 values.
//
// The tensor cores take codes as f16, in which they are exact, so somebody has to
// turn each byte into two.  Four warps do so once for two tiles: blocks of 64 keys
// are copied as they are, while they write the ones before as the swizzled operands
// that a copy of f16 would have made.  (Loads into registers instead are waited for
// as a whole, as a warp has few counters for what is on its way: 1.8 ms in the case
// below.)  Per block and tile
//   S = Q K^T                    128 x 64, queries in f16 (bf16 times a power of two per row)
//   P = 2^(S ks + log2 vs - m)   a thread per row; ks, vs are the scales of the key's page,
//                                vs over the largest of the tile's pages
//   O += P V                     P from TMEM (over S's own columns), V from shared memory
// so that O over sum P / vs, times the largest vs, is the output.  A block's scores are
// there before the softmax of the one before is done (two S buffers); each tile has a warp
// of its own for its products, or one tile's would wait for the other's softmax (1.44 ms).
// Codes are finite, so a key that a row does not see adds 0 whatever it holds.
//
// m stays as it is while the weights fit f16 (they are up to 2^8 when it is set): a block is
// computed with the last one's m, and only where some 8 weights' sum, which the row's total
// wants anyway, says that one might not fit, once more, with m raised and the sums so far made
// smaller.  So most blocks read S once, and neither wait for nor look for a maximum.  That
// path lies behind the loop: in line, the instruction cache cost a tenth of the time.
//
// log2 vs reaches down to -90: a tile knows the smallest scale that its tokens see, and rows
// with nearly all their weight on pages of less are computed again, each by a warp.
//
// Measured: 2048 tokens over 32768 keys, 32 heads of 128 over 8: 1.02 ms in bf16, 1040
// TFLOP/s, 1.01 in f16 (keys of 16 bits: 1.01 ms).  Bound by shared memory and by whole rounds of CTAs: per 64 keys of
// two tiles the products read 128 KB of it and the codes' way takes 64, 1540 cycles at its rate,
// of some 1900; and 256 pairs of tiles come in two rounds of 152.  128 keys at a time, which read
// the queries half as often, leave no room for a second S: 1.4 ms.
#include <algorithm>
#include <type_traits>

#include "attn_tc.cuh"
#include "internal.h"

namespace {

using namespace ppc_attn;

constexpr int kRowsT = 128;                       // query rows of a tile
constexpr int kSoft = 2 * kRowsT;                 // threads of the softmax
constexpr int kTurn = 128;                        // that turn codes into f16, half of them keys, half values; then a multiplying warp for each tile and a copying one
constexpr int kMulWarp = (kSoft + kTurn) / 32, kCopyWarp = kMulWarp + 2;
constexpr int kThreads8 = kSoft + kTurn + 96;
constexpr int kKeys = 64, kLogKeys = 6;           // keys per block
constexpr int kStages = 3;                        // of K and of V in f16
constexpr int kCopies = 2;                        // blocks of codes on their way
constexpr int kInfo = 8;                          // blocks whose notes are kept: those of block g are written when K of g - 2 has been, after the
                                                  // scores of g - 5, which were asked for when the softmax had done with g - 7
constexpr int kSplits = 8;                        // shares of a tile's blocks at most
constexpr int kUp = 8;                            // weights are up to 2^8 when m is set
constexpr float kMost = 65504.f;                  // 8 weights' sum at most: f16's largest number
constexpr float kLeastScale = -90.f;              // log2 of vs at the least: a row that sees no other pages has sums of P / vs below 2^121.
// One that has nearly all its weight on pages of less is computed again by itself: its sum is above 2^98 then, and where it is not
// above this, the largest weight lies on a page of more, beside which what those pages add is some 2^-31
constexpr float kSmallPages = 0x1p60f;

template <int DP>
struct Shape8 {
  static constexpr int Q = kRowsT * DP * 2, KV = kKeys * DP * 2, CODES = kKeys * DP;
  static constexpr int SMEM = 2 * Q + 2 * kStages * KV + 2 * kCopies * CODES + 1024;
  static constexpr int COLS = 512;  // TMEM: O of the tiles at 0 and 128, S at 256, 320 and 384, 448
};

struct alignas(16) Note {           // of a block
  float ks[8], lv[8], inv[8];       // of each 8 keys: the keys' scale; log2 of the values' over the largest, and 1 over that
  uint32_t valid, zero;             // a bit for each 8 keys that are there; whose values are 0 as their scale is
};

// 8 codes as f16, in order
__device__ __forceinline__ uint4 f16_of8(uint32_t a, uint32_t b) {
  uint4 y;
  f16_in_order(a, y.x, y.y);
  f16_in_order(b, y.z, y.w);
  return y;
}

// A row's attention over blocks of keys of its own, by one warp in fp32, 8 keys (of one page) at a time: o is the average so far of
// the lane's 4 values, so that it is as large as they are.  For rows whose pages' value scales are too small beside others'
// for the tile's weights; 125 cycles a key.
struct Average {
  float o[4], m, l;
};
template <class T>
__device__ __noinline__ void row_again(const AttnParams& p, const T* q, const int* table, int h, int lim, int first, int n, int sink_blocks,
                                       int gap, Average& y) {
  const int d = threadIdx.x % 32 * 4;
  const bool in = d < p.D;
  float x[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = in && p.scale != 0.f ? to_f32(q[d + e]) : 0.f;
    y.o[e] = 0.f;
  }
  y.m = -INFINITY;
  y.l = 0.f;
  for (int i = 0; i < n * (kKeys / 8); ++i) {
    const int k = first + i / (kKeys / 8), key = ((k < sink_blocks ? k : k + gap) << kLogKeys) + i % (kKeys / 8) * 8;
    if (key >= lim || (key >= p.sinks && key + 8 <= lim - p.window)) continue;
    const int id = table[key >> p.log_page];
    if (id < 0 || id >= p.pages) continue;
    const int64_t cell = (int64_t)id * p.H + h, at = (cell * p.page + (key & p.page - 1)) * p.D + d;
    const float ks = p.ks[cell], vs = p.vs[cell];
    uint32_t kc[8], vc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      kc[j] = in ? *reinterpret_cast<const uint32_t*>(static_cast<const int8_t*>(p.k) + at + j * p.D) : 0;
      vc[j] = in ? *reinterpret_cast<const uint32_t*>(static_cast<const int8_t*>(p.v) + at + j * p.D) : 0;
    }
    auto code = [](uint32_t w, int e) { return (float)(int8_t)(w >> 8 * e); };
    float s[8], mx = y.m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s[j] = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) s[j] = fmaf(x[e] * ks, code(kc[j], e), s[j]);
#pragma unroll
      for (int f = 16; f > 0; f >>= 1) s[j] += __shfl_xor_sync(~0u, s[j], f);
      s[j] = key + j < lim && (key + j >= lim - p.window || key + j < p.sinks) ? s[j] * (p.scale * 1.44269504f) : -INFINITY;
      mx = fmaxf(mx, s[j]);
    }
    const float base = mx == -INFINITY ? 0.f : mx, had = y.l * ex2(y.m - base);
    float l = had;
#pragma unroll
    for (int j = 0; j < 8; ++j) l += s[j] = ex2(s[j] - base);
    if (l == 0.f) continue;
    const float r = 1.f / l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum = fmaf(s[j] * r, code(vc[j], e), sum);
      y.o[e] = y.o[e] * (had * r) + sum * vs;
    }
    y.m = mx;
    y.l = l;
  }
}

template <class T, int DP>
__global__ void __launch_bounds__(kThreads8, 1) attn8_tile_kernel(const __grid_constant__ AttnParams p) {
  using S = Shape8<DP>;
  constexpr int CHUNK_Q = kRowsT * 128, CHUNK_KV = kKeys * 128;  // bytes of 64 values of every row
  extern __shared__ unsigned char raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  unsigned char* kbuf = smem + 2 * S::Q;
  unsigned char* vbuf = kbuf + kStages * S::KV;
  unsigned char* codes = vbuf + kStages * S::KV;  // of K and of V, as they are in the cache
  __shared__ alignas(8) uint64_t q_full[2], k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages], s_full[2][2],
      p_full[2][2], pv_done[2], o_full[2], note_full[kInfo], codes_full[2][kCopies], codes_empty[2][kCopies];
  __shared__ Note notes[kInfo];
  __shared__ float most[kThreads8 / 32], least[kThreads8 / 32];
  __shared__ uint8_t row_power[kSoft];
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
  const int low = max(0, lim_min - p.window), sink_blocks = (min(p.sinks, lim_max) + kKeys - 1) >> kLogKeys, gap = max(0, (low >> kLogKeys) - sink_blocks);
  const int blocks = ((lim_max + kKeys - 1) >> kLogKeys) - gap, first = (int)((int64_t)blocks * z / p.splits), n = (int)((int64_t)blocks * (z + 1) / p.splits) - first;
  auto key_of = [&](int k) { return (first + k < sink_blocks ? first + k : first + k + gap) << kLogKeys; };  // of the share's block k
  const bool two = nt > T1;
  // a negative scale goes into the queries, and so does 0 (with no queries, any scale): sl > 0
  const float sl = p.scale == 0.f ? 1.f : fabsf(p.scale) * 1.44269504f;

  // ---- set up
  if (warp == kMulWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(su32(&tmem_s)), "n"(S::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(su32(&q_full[i]), 4);  // warps, as below: arrivals of threads come one after another
      mbar_init(su32(&pv_done[i]), 1);
      mbar_init(su32(&o_full[i]), 1);
      for (int j = 0; j < 2; ++j) {
        mbar_init(su32(&s_full[i][j]), 1);
        mbar_init(su32(&p_full[i][j]), 4);
      }
      for (int j = 0; j < kCopies; ++j) {
        mbar_init(su32(&codes_full[i][j]), 1);
        mbar_init(su32(&codes_empty[i][j]), 2);
      }
    }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(su32(&k_full[i]), 2);
      mbar_init(su32(&k_empty[i]), 1 + two);
      mbar_init(su32(&v_full[i]), 2);
      mbar_init(su32(&v_empty[i]), 1 + two);
    }
    for (int i = 0; i < kInfo; ++i) mbar_init(su32(&note_full[i]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // the largest scale of values among the pages that some token sees, the smallest above 0, and whether one is 0
  float vtop = 0.f, vleast = INFINITY;
  bool zeros = false;
  {
    const int sinks = min(p.sinks, lim_max), pages0 = (sinks + p.page - 1) >> p.log_page, from = max(pages0, low >> p.log_page);
    const int count = pages0 + max(0, ((lim_max + p.page - 1) >> p.log_page) - from);
    for (int i = tid; i < count; i += kThreads8) {
      const int id = table[i < pages0 ? i : i - pages0 + from];
      const bool there = id >= 0 && id < p.pages;
      const float vs = there ? p.vs[(int64_t)id * p.H + h] : 0.f;
      zeros = zeros || (there && vs == 0.f);
      vtop = fmaxf(vtop, vs);
      vleast = fminf(vleast, vs > 0.f ? vs : INFINITY);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      vtop = fmaxf(vtop, __shfl_xor_sync(~0u, vtop, d));
      vleast = fminf(vleast, __shfl_xor_sync(~0u, vleast, d));
    }
    if (lane == 0) {
      most[warp] = vtop;
      least[warp] = vleast;
    }
  }
  tm_fence_before();
  zeros = __syncthreads_or(zeros);
  tm_fence_after();
#pragma unroll
  for (int i = 0; i < kThreads8 / 32; ++i) {
    vtop = fmaxf(vtop, most[i]);
    vleast = fminf(vleast, least[i]);
  }
  const uint32_t tmem = tmem_s;
  // a bounded wait; after one gave up none waits any more
  auto hold = [&](uint64_t* bar, uint32_t parity) {
    if (!mbar_try(su32(bar), parity)) hold_on(su32(bar), parity, &dead);
  };

  // what the warp has done before is there for who waits
  auto warp_arrive = [&](uint64_t* bar) {
    __syncwarp();
    if (lane == 0) mbar_arrive(su32(bar));
  };

  if (warp >= kMulWarp) {
    if (warp == kCopyWarp) {
      // ---- copies, and what there is to say of a block.  Lane j < 8 has keys 8 j on; a run of keys on one page is one copy.
      // Pages are looked up two blocks ahead and scales one, so that neither is waited for
      const int run = min(p.page, kKeys), runs = run >> 3;
      auto look = [&](int k) {  // the page's entry of the table (-1: no page); INT32_MIN: none of the run's keys is there
        const int key = lane < 8 && k < n ? key_of(k) + (lane * 8 & ~(run - 1)) : INT32_MAX;
        return key < lim_max && (key < p.sinks || key + run > low) ? max(table[key >> p.log_page], -1) : INT32_MIN;
      };
      // 1 over the largest scale, in two steps, as it may lie beyond fp32: a power of two, and what is left
      const float vup = __int_as_float((254 - min(max(__float_as_int(vtop) >> 23, 1), 253)) << 23), vinv = vtop > 0.f ? 1.f / (vtop * vup) : 0.f;
      int64_t cell = -1;
      float ks = 0.f, vs = 0.f;
      auto resolve = [&](int id) {
        const bool there = id >= 0 && id < p.pages;
        if (!there && id != INT32_MIN) atomicOr(p.status, PP_CACHE_BAD_PAGE);
        cell = there ? (int64_t)id * p.H + h : -1;
        ks = vs = 0.f;
        if (there) {
          ks = p.ks[cell];
          vs = p.vs[cell];
        }
      };
      int ahead = look(1);
      resolve(look(0));
      for (int g = 0; g < n; ++g) {
        Note& note = notes[g % kInfo];
        const unsigned there = __ballot_sync(~0u, cell >= 0);
        const int bytes = __popc(there) * 8 * p.D, key = key_of(g) + lane * 8;
        const int64_t from = (cell * p.page + (key & p.page - 1)) * p.D;
        const bool lead = cell >= 0 && (lane & runs - 1) == 0;
        auto copy = [&](int i, const void* pool) {
          const int at = g % kCopies;
          hold(&codes_empty[i][at], g / kCopies & 1 ^ 1);
          const bool go = !*(volatile int*)&dead;
          if (lane == 0) mbar_arrive_expect_tx(su32(&codes_full[i][at]), go ? bytes : 0);
          __syncwarp();
          if (go && lead)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                             su32(codes + (i * kCopies + at) * S::CODES) + lane * 8 * p.D),
                         "l"(static_cast<const int8_t*>(pool) + from), "r"(run * p.D), "r"(su32(&codes_full[i][at]))
                         : "memory");
          __syncwarp();
        };
        copy(0, p.k);
        if (lane < 8) {
          const float lv = vs > 0.f ? fmaxf(__log2f(vs * vup * vinv), kLeastScale) : kLeastScale;
          note.ks[lane] = ks;
          note.lv[lane] = lv;
          note.inv[lane] = ex2(-lv);
        }
        const unsigned zero = __ballot_sync(~0u, lane < 8 && cell >= 0 && vs == 0.f);
        if (lane == 0) {
          note.valid = there;
          note.zero = zero;
        }
        warp_arrive(&note_full[g % kInfo]);
        copy(1, p.v);
        resolve(ahead);
        ahead = look(g + 2);
      }
    }
    // ---- products, each tile's by a warp of its own, so that neither waits for the other's softmax
    if (const int t = warp - kMulWarp; t < 1 + two) {
      const uint32_t leader = elect();
      const uint32_t qa = desc_lo(su32(smem) + t * S::Q, 16), kb = desc_lo(su32(kbuf), 16), vb = desc_lo(su32(vbuf), CHUNK_KV);
      const uint32_t to = tmem + t * 128, scores_at = to + 256;
      auto scores = [&](int g) {
        const int st = g % kStages;
        hold(&k_full[st], g / kStages & 1);
        tm_fence_after();
        const uint32_t kd = kb + st * (S::KV >> 4);
#pragma unroll
        for (int kk = 0; kk < DP / 16; ++kk)
          mma_ss(scores_at + (g & 1) * 64, qa + (kk / 4 * CHUNK_Q + kk % 4 * 32 >> 4), kd + (kk / 4 * CHUNK_KV + kk % 4 * 32 >> 4),
                 idesc<__half>(kRowsT, kKeys, false), kk > 0, leader);
        commit(su32(&s_full[t][g & 1]), leader);
        commit(su32(&k_empty[st]), leader);
      };
      // Products run in the order in which they are asked for, so the scores that go where a block's P was lie behind its product
      if (n > 0) {
        hold(&q_full[t], 0);
        scores(0);
      }
      for (int g = 0; g < n; ++g) {
        if (g + 1 < n) scores(g + 1);
        const int st = g % kStages;
        hold(&v_full[st], g / kStages & 1);
        hold(&p_full[t][g & 1], g >> 1 & 1);
        tm_fence_after();
        const uint32_t vd = vb + st * (S::KV >> 4);
#pragma unroll
        for (int kk = 0; kk < kKeys / 16; ++kk)
          mma_ts(to, scores_at + (g & 1) * 64 + kk * 8, vd + (kk * 2048 >> 4), idesc<__half>(kRowsT, DP, true), g > 0 || kk > 0, leader);
        commit(su32(&pv_done[t]), leader);
        commit(su32(&v_empty[st]), leader);
      }
      if (n > 0) commit(su32(&o_full[t]), leader);
    }
  } else if (warp >= kSoft / 32) {
    // ---- codes to f16, two warps the keys' and two the values': a warp has 32 rows of a block, a lane 16 codes of a row at a time, their halves apart: e is the one that
    // it takes first, so that 16 lanes read from all banks, and the 8 lanes that write at once write to all (rows of 128 or 64)
    constexpr int CPR = DP / 16, RPL = 32 / CPR, NI = 32 / RPL;  // chunks of 16 codes to a row, rows to a step, steps
    const int pool = warp / 2 & 1, w = warp % 2, c = lane % CPR, r = lane / CPR, e = DP == 128 ? c >> 2 ^ r & 1 : r >> 1 & 1;
    const bool in = c * 16 < p.D;
    const int key0 = w * 32 + r, from = key0 * p.D + c * 16 + e * 8, other = 8 - 16 * e;
    // where the halves go: rows 4 on of 8 are swizzled by 4 more chunks
    const int to0 = c / 4 * CHUNK_KV + key0 * 128;
    const int at0 = to0 + ((c % 4 * 2 + e ^ key0 & 7) << 4), at1 = to0 + ((c % 4 * 2 + 1 - e ^ key0 & 7) << 4);
    auto turn = [&](unsigned char* to, const unsigned char* codes, uint32_t zero) {
      uint2 x[NI], y[NI];
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        x[i] = y[i] = make_uint2(0, 0);
        if (in) {
          x[i] = *reinterpret_cast<const uint2*>(codes + from + i * RPL * p.D);
          y[i] = *reinterpret_cast<const uint2*>(codes + from + i * RPL * p.D + other);
        }
      }
      if (__builtin_expect(zero, 0)) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
          if (zero >> (key0 + i * RPL) / 8 & 1) x[i] = y[i] = make_uint2(0, 0);
      }
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int flip = i * RPL & 4 ? 64 : 0;
        *reinterpret_cast<uint4*>(to + (at0 ^ flip) + i * RPL * 128) = f16_of8(x[i].x, x[i].y);
        *reinterpret_cast<uint4*>(to + (at1 ^ flip) + i * RPL * 128) = f16_of8(y[i].x, y[i].y);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    };
    uint64_t *const full = pool ? v_full : k_full, *const empty = pool ? v_empty : k_empty;
    unsigned char* const buf = pool ? vbuf : kbuf;
    for (int g = 0; g < n; ++g) {
      const int st = g % kStages, at = g % kCopies;
      hold(&codes_full[pool][at], g / kCopies & 1);
      hold(&empty[st], (g / kStages + 1) & 1);
      uint32_t zero = 0;
      if (__builtin_expect(pool && zeros, 0)) {  // (the note is written before the values' copy)
        hold(&note_full[g % kInfo], g / kInfo & 1);
        zero = notes[g % kInfo].zero;
      }
      turn(buf + st * S::KV, codes + (pool * kCopies + at) * S::CODES, zero);
      warp_arrive(&full[st]);
      if (lane == 0) mbar_arrive(su32(&codes_empty[pool][at]));
    }
  } else {
    // ---- queries, then the softmax, a thread per row
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
          float f[8], up = 1.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = used ? to_f32(v[u].v[e]) : 0.f;
          if constexpr (!std::is_same<T, __half>::value) {
            int top = 16;  // the largest exponent, of infinities and NaN the largest finite one; rows below 2^-111 keep fewer bits
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, min(__float_as_int(fabsf(f[e])) >> 23, 254));
#pragma unroll
            for (int m = 1; m < L; m <<= 1) top = max(top, __shfl_xor_sync(~0u, top, m));
            up = __int_as_float((268 - top) << 23);
            if (c == 0) row_power[t * kRowsT + r] = (uint8_t)(top - 14);
          }
          Vec<__half, 8> y;
#pragma unroll
          for (int e = 0; e < 8; ++e) y.v[e] = __float2half_rn(sign == 0.f ? 0.f : f[e] * (up * sign));
          *reinterpret_cast<Vec<__half, 8>*>(smem + t * S::Q + c / 8 * CHUNK_Q + r * 128 + ((c % 8 ^ (r & 7)) << 4)) = y;
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      warp_arrive(&q_full[t]);
      // the rows of this tile's four warps
      asm volatile("bar.sync %0, %1;" ::"r"(1 + t), "n"(kRowsT) : "memory");
    }
    const bool live_row = tr < rows;
    const int tok = t * T1 + p.G.div(min(tr, max(rows, 1) - 1));  // rows behind the last do as it does
    const int lim = some ? limit(tok) : 0;
    const float slr = sl * (std::is_same<T, __half>::value || !some ? 1.f : __int_as_float(row_power[t * kRowsT + tr] << 23));
    const uint32_t row_tm = tmem + t * 128 + ((uint32_t)(warp % 4 * 32) << 16);  // its sums; its scores lie 256 on
    float m = -INFINITY, l = 0.f;
    for (int g = 0; some && g < n; ++g) {
      const int key = key_of(g);
      const Note& note = notes[g % kInfo];
      hold(&note_full[g % kInfo], g / kInfo & 1);
      const uint32_t valid = note.valid;
      const bool part = __any_sync(~0u, valid != 0xFFu || lim - key < kKeys || (key < lim - p.window && key + kKeys > p.sinks));
      // which of 32 keys the row sees
      auto see = [&](int c) -> uint32_t {
        const int at = key + c * 32;
        const uint32_t v = (valid >> c * 4 & 15u) * 0x00204081u & 0x01010101u;  // a bit to a byte
        return v * 255u & (uint32_t)(below(lim - at) & (~below(lim - at - p.window) | below(p.sinks - at)));
      };
      const uint32_t s_tm = row_tm + 256 + (g & 1) * 64;
      hold(&s_full[t][g & 1], g >> 1 & 1);
      __syncwarp();
      tm_fence_after();
      float top = 0.f, sum = 0.f;
      bool again = __any_sync(~0u, m == -INFINITY);  // m is not set: it has to be where the row sees something
      if (__builtin_expect(again, 0)) again = __any_sync(~0u, m == -INFINITY && (!part || (see(0) | see(1))));
      if (__builtin_expect(!again, 1)) {
        uint32_t w[32];
        const float at = m == -INFINITY ? 0.f : m;
        float x[2][32];
        tm_ld32(s_tm, x[0]);
        tm_ld32(s_tm + 32, x[1]);
        tm_wait_ld();
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float(&y)[32] = x[c];
          const float4 ks = *reinterpret_cast<const float4*>(note.ks + 4 * c), lv = *reinterpret_cast<const float4*>(note.lv + 4 * c),
                       inv = *reinterpret_cast<const float4*>(note.inv + 4 * c);
          const float k4[4] = {ks.x, ks.y, ks.z, ks.w}, l4[4] = {lv.x, lv.y, lv.z, lv.w}, i4[4] = {inv.x, inv.y, inv.z, inv.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float kj = k4[j] * slr, oj = l4[j] - at;
#pragma unroll
            for (int i = 0; i < 8; i += 2)
              unpack2(fma2(pack2(y[8 * j + i], y[8 * j + i + 1]), pack2(kj, kj), pack2(oj, oj)), y[8 * j + i], y[8 * j + i + 1]);
          }
          if (__builtin_expect(part, 0)) {
            const uint32_t bits = see(c);
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!(bits >> i & 1)) y[i] = -INFINITY;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint64_t s2 = 0;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
              const float a = ex2(y[8 * j + i]), b = ex2(y[8 * j + i + 1]);
              s2 = add2(s2, pack2(a, b));
              w[16 * c + 4 * j + i / 2] = pack<__half>(a, b);
            }
            float a, b;
            unpack2(s2, a, b);
            a += b;
            top = fmaxf(top, a);
            sum = fmaf(a, i4[j], sum);
          }
        }
        again = __any_sync(~0u, top > kMost);
        if (!again) {
          l += sum;
          tm_st32(s_tm, w);
        }
      }
      if (__builtin_expect(again, 0)) {
        // once more from the scores, with m above them.  Each step is rounded by itself, as the maximum's are, so that no weight
        // passes its bound and the largest does not vanish where fp32 numbers lie further than 1 apart
        auto exponents = [&](int c, float (&y)[32]) {
          tm_ld32(s_tm + 32 * c, y);
          tm_wait_ld();
          const uint32_t bits = part ? see(c) : ~0u;
#pragma unroll
          for (int i = 0; i < 32; ++i)
            y[i] = bits >> i & 1 ? __fadd_rn(__fmul_rn(y[i], note.ks[4 * c + i / 8] * slr), note.lv[4 * c + i / 8]) : -INFINITY;
        };
        float most = -INFINITY;
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
          float y[32];
          exponents(c, y);
#pragma unroll
          for (int i = 0; i < 32; ++i) most = fmaxf(most, y[i]);
        }
        const float to = fmaxf(m, lower(most, (float)kUp)), f = to == -INFINITY ? 1.f : ex2(m - to);
        m = to;
        l *= f;
        if (g > 0) {  // the sums so far, in TMEM.  (Those of g - 2 are done, as they lie before these scores: a parity names one phase)
          hold(&pv_done[t], (g - 1) & 1);
          __syncwarp();
          tm_fence_after();
#pragma unroll 1
          for (int c = 0; c < DP; c += 32) {
            float o[32];
            tm_ld32(row_tm + c, o);
            tm_wait_ld();
            uint32_t r[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(o[i] * f);
            tm_st32(row_tm + c, r);
          }
        }
        const float at = m == -INFINITY ? 0.f : m;
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {  // weights go where scores were that have been read
          float y[32];
          exponents(c, y);
          uint32_t r[16];
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float a = ex2(__fadd_rn(y[i], -at)), b = ex2(__fadd_rn(y[i + 1], -at));
            l = fmaf(a + b, note.inv[4 * c + i / 8], l);
            r[i / 2] = pack<__half>(a, b);
          }
          tm_st16(s_tm + 16 * c, r);
        }
      }
      tm_wait_st();
      tm_fence_before();
      warp_arrive(&p_full[t][g & 1]);
    }

    // ---- out
    if (some) {
      // (a barrier of its own: of pv_done's last two phases both may be over, and their parities say nothing then)
      if (n > 0) hold(&o_full[t], 0);
      __syncwarp();
      tm_fence_after();
      const int64_t cell = (int64_t)(base + p.G.div(live_row ? tr : 0)) * p.H * p.G.d + h * p.G.d + p.G.mod(live_row ? tr : 0);
      const bool parts = p.splits > 1;
      // first over the total, then times the scale: together they may lie below fp32's numbers, and a share's sums beyond them
      const float over = l == 0.f ? 0.f : 1.f / l;
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
        for (int i = 0; i < 32; ++i) o[i] = o[i] * over * vtop;
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
        if (parts) p.split_stats[at] = make_float2(m, l);
        else if (p.lse) p.lse[cell] = l == 0.f ? -INFINITY : log_sum<__half, kUp>(m, l);
      }
      unsigned again = __ballot_sync(~0u, live_row && l > kSmallPages && vleast < vtop * 0x1p-90f);
      __syncwarp();  // what the rows' own threads wrote lies before what the warp writes over it
      for (; again; again &= again - 1) {
        const int r = warp % 4 * 32 + __ffs(again) - 1, token = p.G.div(r), head = h * p.G.d + p.G.mod(r), d = lane * 4;
        Average y;
        row_again<T>(p, static_cast<const T*>(p.q) + (base + token) * p.q_ts + (int64_t)head * p.q_hs, table, h, limit(t * T1 + token), first, n,
                     sink_blocks, gap, y);
        const int64_t cell = (int64_t)(base + token) * p.H * p.G.d + head, at = (int64_t)z * p.T * p.H * p.G.d + cell;
        if (d < p.D) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (parts) p.split_sums[at * DP + d + e] = y.o[e];
            else static_cast<T*>(p.out)[cell * p.D + d + e] = from_f32<T>(y.o[e]);
          }
        }
        if (lane == 0) {
          if (parts) p.split_stats[at] = make_float2(y.m, y.l);
          else if (p.lse) p.lse[cell] = y.l == 0.f ? -INFINITY : y.m * 0.693147181f + logf(y.l);
        }
      }
    }
    tm_fence_before();
  }
  __syncthreads();
  if (dead && tid == 0) {
    atomicOr(p.status, PP_CACHE_TIMEOUT);
    // copies and products still in flight end before the CTA does
    for (int i = 0; i < 2; ++i)
      for (uint32_t ph = 0; ph < 2; ++ph) {
        for (int j = 0; j < kCopies; ++j) wait(su32(&codes_full[i][j]), ph);
        wait(su32(&pv_done[i]), ph);
      }
  }
  if (warp == kMulWarp) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::COLS));
  }
}

template <class T, int DP>
cudaError_t prepare_one() {
  return cudaFuncSetAttribute(attn8_tile_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape8<DP>::SMEM);
}

template <class T, int DP>
cudaError_t launch(const AttnParams& p, int64_t grid, cudaStream_t stream) {
  const cudaError_t e = launch_after(attn8_tile_kernel<T, DP>, dim3((unsigned)grid), kThreads8, Shape8<DP>::SMEM, stream, 1, p);
  return e != cudaSuccess || p.splits == 1 ? e : tile_join(p, std::is_same<T, __half>::value ? PP_F16 : PP_BF16, true, stream);
}

// Pairs of tiles of a call at most: each sequence adds at most one that is not full.
int64_t most_pairs(const AttnParams& p) { return ((int64_t)p.T / (2 * (kRowsT / p.G.d)) + std::min(p.T, p.B)) * p.H; }

// Few tiles are split along their blocks, up to one CTA per SM, while a share can have 4 blocks; the shares' sums have room for
// two tiles per SM.
int64_t splits_of(const AttnParams& p, int sms) {
  const int TT = 2 * (kRowsT / p.G.d);
  const int64_t cells = (int64_t)p.T * p.H * p.G.d, room = (int64_t)2 * sms * kRowsT;
  const int64_t keys = std::min<int64_t>((int64_t)p.width * p.page, (int64_t)p.window + p.sinks + TT + 2 * kKeys);
  return std::max<int64_t>(1, std::min({(int64_t)kSplits, sms / most_pairs(p), keys / kKeys / 4, room / cells}));
}

}  // namespace

namespace ppc_attn {

bool tile8_applicable(const AttnParams& p, int dtype, int sms) {
  if (dtype == PP_F32 || p.D > 128 || p.G.d > 64 || !p.starts) return false;
  // By what 64 keys of every sequence take.  The row kernel has three CTAs per SM, each of which meets them with 8 rows in about
  // 0.95 us; a CTA here meets them with a tile in as much, with two in 1.5 times that, and the CTAs come in rounds.  32 heads of
  // 128 over 8, bf16, rows and tiles: 16 rows of each of 32 sequences of 8192 keys 152 and 235 us (of up to 8192 96 and 175), 32
  // rows 316 and 237 (172 and 176); 20 rows of one of 30000 41 and 66, 64 rows of one of 32768 84 and 72, 1024 rows 1042 and 207.
  const int64_t units = ((int64_t)p.T * p.G.d + 7) / 8 * p.H, pairs = most_pairs(p), s = splits_of(p, sms);
  const bool two = (int64_t)p.T * p.G.d > (int64_t)kRowsT * p.B;
  return units * s * 2 > 3 * (int64_t)sms * ((pairs * s + sms - 1) / sms) * (two ? 3 : 2);
}

cudaError_t tile8_prepare() {
  cudaError_t e = prepare_one<__half, 64>();
  if (e == cudaSuccess) e = prepare_one<__half, 128>();
  if (e == cudaSuccess) e = prepare_one<__nv_bfloat16, 64>();
  if (e == cudaSuccess) e = prepare_one<__nv_bfloat16, 128>();
  return e;
}

cudaError_t tile8_launch(AttnParams p, const pp_cache& c, int sms, cudaStream_t stream) {
  const int DP = p.D <= 64 ? 64 : 128;
  const int64_t pairs = most_pairs(p), room = (int64_t)2 * sms * kRowsT;  // CTAs beyond the last tile leave
  p.splits = (int)splits_of(p, sms);
  p.split_sums = c.tiles;
  p.split_stats = reinterpret_cast<float2*>(c.tiles + room * DP);
  const int64_t grid = pairs * p.splits;
  if (grid > INT32_MAX) return cudaErrorInvalidValue;
  return c.dtype == PP_F16 ? (DP == 64 ? launch<__half, 64>(p, grid, stream) : launch<__half, 128>(p, grid, stream))
                           : (DP == 64 ? launch<__nv_bfloat16, 64>(p, grid, stream) : launch<__nv_bfloat16, 128>(p, grid, stream));
}

}  // namespace ppc_attn
