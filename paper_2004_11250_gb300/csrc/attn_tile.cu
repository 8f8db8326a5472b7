// Attention for many query tokens: tiles of 128 query rows on the tensor cores
// (tcgen05), for 16-bit types and heads of up to 128 values.
//
// A CTA has the rows of one cache head: the heads of its group for as many
// consecutive tokens as give up to 128 rows, one row per TMEM lane.  Keys come in
// blocks of 64 (whole pages, or pieces of one).  Per block
//   S = Q K^T       128 x 64, operands in shared memory, sums in TMEM
//   P = 2^(S - m)   a thread per row: no exchange between lanes
//   O += P V        P from TMEM (over S's own columns), V from shared memory
// The score product of a block runs while the softmax of the one before it does
// (two S buffers), and two CTAs share an SM, so one's softmax hides behind the
// other's products.  m is only raised, and O rescaled in TMEM, when a row's
// maximum has grown by more than 2^8 (2^2 in f16): the weights stay below a bound,
// and both they and their sums are divided in the end.  P is rounded to the inputs'
// type, as the tensor cores want it: 11 bits in f16, 8 in bf16, where the sums have
// 24 (a second half would double the products).  f16 weights are taken 2^13 times as
// large, so that all down to 2^-27 of the row's largest have their 11 bits, and
// those above 2^-38 some.
//
// Where pages are selected for each token, the tile reads the union of its tokens'
// pages once, and a bit per (page, token) says which rows use it: neighbouring
// tokens select mostly the same pages, and a gather per token would read each of
// them through L2 again (2048 tokens over 512 pages: 17 GB).  Few tiles are split
// along their blocks, and a second kernel joins the shares.
//
// Measured: 2048 tokens, 32 heads of 128 over 8, 32 of 512 pages of 64 each (bf16):
// 296 us, 905 TFLOP/s of the products over the unions (125 pages per 32 tokens);
// 303 us in f16, whose rows are rescaled more often.
// Bound by latency in the softmax: 2.7 warps per scheduler wait for their loads from
// tensor memory, at 1.5 instructions per cycle and SM; the tensor pipe is busy 36 %
// of the time.  All 32768 keys: 998 us, 1060 TFLOP/s.  3 chunks of 333 tokens, 8 heads
// of 64, 20 pages of 32 each (f16): 37 us, split in four (71 us whole).
#include <algorithm>
#include <type_traits>

#include "attn.cuh"
#include "internal.h"

namespace {

using namespace ppc_attn;

constexpr int kRowsT = 128;            // query rows of a tile
constexpr int kSoft = 128;             // threads of the softmax; then a copying and a multiplying warp
constexpr int kThreadsT = kSoft + 64;
constexpr int kKeys = 64;              // keys per block
constexpr int kStages = 2;             // of K and of V
constexpr int kEnds = 3;               // blocks with keys that some tokens of a tile see and others do not, at most: 127 keys
constexpr int kInfo = 4;               // blocks that the copying warp may be ahead of the softmax, and one
constexpr int kMaskWords = 2048;       // token bits of the pages in one window
constexpr int kAhead = 8;              // entries of the tokens' lists in flight per thread
constexpr int kSplits = 8;             // shares of a tile's blocks at most
constexpr int kUp = 13;                // f16 weights are up to 2^13 where m is not behind, and 2^2 times that
template <class T>
constexpr float kGrow = std::is_same<T, __half>::value ? 2.f : 8.f;  // log2 of how far a row's weights may pass their bound

template <int DP>
struct TileShape {
  static constexpr int Q = kRowsT * DP * 2, KV = kKeys * DP * 2;
  static constexpr int SMEM = Q + 2 * kStages * KV + kMaskWords * 4 + kMaskWords * 2 + 1024;
  static constexpr int COLS = 256;     // TMEM: O at 0 .. DP - 1, S at 128 and 192
};

struct Block {          // what the copying warp says of a block
  int have[kPieces];
  int full;  // every row sees all of it (or may, of selected pages)
  int end;   // 1 + which of the last blocks, with keys that some tokens see and others do not; 0: none of them
};

// Shared-memory descriptors of 128-byte swizzled operands.  K-major (Q, K): rows of 128 bytes, groups of 8 rows 1024
// bytes apart.  MN-major (V): 128 bytes of values per key, groups of 8 keys 1024 bytes apart, the next 64 values `lbo`
// bytes on.
constexpr uint32_t kDescHi = (1024 >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo) { return ((addr >> 4) & 0x3FFF) | (lbo >> 4) << 16; }
template <class T>
__host__ __device__ constexpr uint32_t idesc(int m, int n, bool b_mn) {
  const uint32_t f = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  return (1u << 4) | (f << 7) | (f << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// Copies, products and commits of a whole warp, issued by its leader.  The warp stays together, so that the operands are in
// uniform registers, as the instructions want them: behind a branch of one lane each is moved there first, and an issue
// took some 100 cycles.
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t id, uint32_t acc, uint32_t leader) {
  asm volatile(
      "{ .reg .pred p, q; .reg .b64 x, y; setp.ne.b32 p, %5, 0; setp.ne.b32 q, %6, 0; mov.b64 x, {%1, %4}; mov.b64 y, {%2, %4};"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p; }" ::"r"(d),
      "r"(a), "r"(b), "r"(id), "r"(kDescHi), "r"(acc), "r"(leader)
      : "memory");
}
// the left operand in TMEM
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t id, uint32_t acc, uint32_t leader) {
  asm volatile(
      "{ .reg .pred p, q; .reg .b64 y; setp.ne.b32 p, %5, 0; setp.ne.b32 q, %6, 0; mov.b64 y, {%2, %4};"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p; }" ::"r"(d),
      "r"(a), "r"(b), "r"(id), "r"(kDescHi), "r"(acc), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar, uint32_t leader) {
  asm volatile(
      "{ .reg .pred q; setp.ne.b32 q, %1, 0; @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0]; }" ::"r"(bar),
      "r"(leader)
      : "memory");
}
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* m, int x, int y, uint32_t bar, uint32_t leader) {
  asm volatile(
      "{ .reg .pred q; setp.ne.b32 q, %5, 0;"
      " @q cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4]; }" ::"r"(dst),
      "l"(m), "r"(x), "r"(y), "r"(bar), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void expect(uint32_t bar, int bytes, uint32_t leader) {
  asm volatile(
      "{ .reg .pred q; setp.ne.b32 q, %2, 0; @q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1; }" ::"r"(bar), "r"(bytes),
      "r"(leader)
      : "memory");
}
__device__ __forceinline__ uint32_t elect() {
  uint32_t r;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xFFFFFFFF; selp.u32 %0, 1, 0, p; }" : "=r"(r));
  return r;
}
__device__ __forceinline__ void tm_ld32(uint32_t a, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
      "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(a));
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tm_st32(uint32_t a, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
      "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
      "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
      "r"(r[31]), "r"(a)
      : "memory");
}
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// One row's attention over its selected pages, by one warp, 4 keys at a time: of a row whose product met a value that is not
// finite, on a page of the tile's union that may not be its own.  A lane has 4 of the row's values.
template <class T>
__device__ __noinline__ void redo_row(const AttnParams& p, const T* q, const int* table, const int* list, int h, int keys,
                                      float sl, T* out, float* lse) {
  constexpr int U = 4;
  const int lane = threadIdx.x % 32, P = (keys + p.page - 1) >> p.log_page, d = lane * 4;
  const bool in = d < p.D;
  float qv[4], o[4] = {}, m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) qv[i] = in ? to_f32(q[d + i]) : 0.f;
  for (int e = 0; e < min(p.keep, P); ++e) {
    const int w = list[e];
    if (w < 0 || w >= P) continue;
    const int id = table[w];
    if (id < 0 || id >= p.pages) continue;
    const int n = min(p.page, keys - w * p.page);
    for (int j = 0; j < n; j += U) {
      Vec<T, 4> k[U], v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {  // beyond the last key, the last once more
        const int64_t at = (((int64_t)id * p.H + h) * p.page + min(j + u, n - 1)) * p.D + (in ? d : 0);
        k[u] = *reinterpret_cast<const Vec<T, 4>*>(static_cast<const T*>(p.k) + at);
        v[u] = *reinterpret_cast<const Vec<T, 4>*>(static_cast<const T*>(p.v) + at);
      }
      float x[U], mx = m;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        x[u] = 0.f;
        if (in)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[u] += qv[i] * to_f32(k[u].v[i]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) x[u] += __shfl_xor_sync(~0u, x[u], s);
        x[u] = j + u < n ? __fmul_rn(x[u], sl) : -INFINITY;  // rounded before the maximum is taken from it
        mx = fmaxf(mx, x[u]);
      }
      const float ref = mx == -INFINITY ? 0.f : mx, f = ex2(m - ref);
      m = mx;
      l *= f;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float c = ex2(x[u] - ref);
        l += c;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += c * to_f32(v[u].v[i]);
      }
    }
  }
  const float n = l == 0.f ? 0.f : 1.f / l;
  if (in)
#pragma unroll
    for (int i = 0; i < 4; ++i) out[d + i] = from_f32<T>(o[i] * n);
  if (lse && lane == 0) *lse = l == 0.f ? -INFINITY : m * 0.693147181f + logf(l);  // m is the largest here
}

// Values of a block that meet a weight of 0 for being out of sight have to be 0: of keys that no row sees, and where `unfit`
// is not null (some rows see keys that others do not) of those that hold a value that is not finite, which are noted there, a
// bit each.  Two threads per key, a warp per 16 keys.
template <class T, int DP>
__device__ __noinline__ void zero_values(unsigned char* v, const Block& bl, int log_br, uint16_t* unfit) {
  constexpr int C = DP / 16;  // 16-byte pieces of a thread
  const int tid = threadIdx.x, key = tid / 2, c0 = tid % 2 * C;
  const bool there = (key & (1 << log_br) - 1) < bl.have[key >> log_br];
  auto piece = [&](int i) { return reinterpret_cast<uint4*>(v + (c0 + i) / 8 * kKeys * 128 + key * 128 + (c0 + i) % 8 * 16); };
  bool odd = false;
  if (unfit) {
#pragma unroll
    for (int i = 0; i < C; ++i) odd |= not_finite<T>(*piece((i ^ key) & C - 1));  // rows lie in the same banks
    odd = (__shfl_xor_sync(~0u, odd, 1) || odd) && there;
    unsigned bits = 0;
    if (const unsigned every = __ballot_sync(~0u, odd))
      for (int i = 0; i < 16; ++i) bits |= (every >> 2 * i & 1) << i;
    if (bits && tid % 32 == 0) unfit[tid / 32] = (uint16_t)bits;
  }
  if (odd || !there) {
#pragma unroll
    for (int i = 0; i < C; ++i) *piece(i) = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
}

// what a wait comes to that does not find its phase complete at once
__device__ __noinline__ void hold_on(uint32_t bar, uint32_t parity, volatile int* dead) {
  if (!*dead && !wait(bar, parity)) *dead = 1;
}

template <class T, int DP>
__global__ void __launch_bounds__(kThreadsT, 2)
    attn_tile_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap mk,
                     const __grid_constant__ CUtensorMap mv) {
  using S = TileShape<DP>;
  constexpr int CHUNK_Q = kRowsT * 128, CHUNK_KV = kKeys * 128;  // bytes of 64 values of every row
  extern __shared__ unsigned char raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  unsigned char* kbuf = smem + S::Q;
  unsigned char* vbuf = kbuf + kStages * S::KV;
  uint32_t* masks = reinterpret_cast<uint32_t*>(vbuf + kStages * S::KV);
  uint16_t* list = reinterpret_cast<uint16_t*>(masks + kMaskWords);
  __shared__ alignas(8) uint64_t q_full, k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages], s_full[2],
      p_full[2], pv_done;
  __shared__ Block info[kInfo];
  __shared__ alignas(8) uint64_t info_full[kInfo];
  __shared__ int2 found[32];
  __shared__ uint32_t tmem_s;
  __shared__ int scan[kThreadsT / 32], tile_of[4], dead;
  __shared__ alignas(8) uint16_t unfit[kEnds][4];  // keys of the last blocks with values that are not finite, a bit each, and 16 a word
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;

  // ---- which tile: those of a sequence's last tokens, which see the most keys, come first
  const int TT = kRowsT / p.G.d;  // tokens per tile
  const int z = blockIdx.x % p.splits, h = blockIdx.x / p.splits % p.H, order = blockIdx.x / p.splits / p.H;
  if (tid == 0) {
    dead = 0;
    tile_of[0] = -1;
  }
  __syncthreads();
  after_previous();
  const int per = (p.B + kThreadsT - 1) / kThreadsT, b0 = min(p.B, tid * per), b1 = min(p.B, b0 + per);
  int mine = 0;
  bool bad = false;
  for (int b = b0; b < b1; ++b) {
    const int s0 = p.starts ? p.starts[b] : b, n = p.starts ? p.starts[b + 1] - s0 : 1;
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
  for (int i = 0; i < kThreadsT / 32; ++i) {
    if (i < warp) before += scan[i];
    total += scan[i];
  }
  before -= mine;
  if (order >= total) return;
  const int want = total - 1 - order;
  if (want >= before && want < before + mine) {
    for (int b = b0;; ++b) {
      const int s0 = p.starts ? p.starts[b] : b, n = p.starts ? p.starts[b + 1] - s0 : 1, c = (n + TT - 1) / TT;
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
  const int b = tile_of[0], t0 = tile_of[1] + tile_of[3], nt = min(TT, tile_of[2] - tile_of[3]), rows = nt * p.G.d;
  int len = p.lens[b];
  const int most = p.width * p.page;
  if (len < 0 || len > most) {
    if (tid == 0) atomicOr(p.status, PP_CACHE_BAD_LENGTH);
    len = min(max(len, 0), most);
  }
  // keys that token i of the tile sees
  auto limit = [&](int i) { return p.causal ? min(len, max(0, len - tile_of[2] + tile_of[3] + i + 1)) : len; };
  const int lim_min = limit(0), lim_max = limit(nt - 1), P = (lim_max + p.page - 1) >> p.log_page;
  const int* table = p.table + (int64_t)b * p.width;
  const int log_br = min(p.log_page, 6), BR = 1 << log_br, log_pc = 6 - log_br, pieces = 1 << log_pc;
  const int log_pp = p.log_page - log_br;  // pieces per page
  // a negative scale goes into the queries, and so does 0 (with no queries, any scale): sl > 0
  const float sl = p.scale == 0.f ? 1.f : fabsf(p.scale) * 1.44269504f;

  // ---- set up
  if (warp == 5) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(su32(&tmem_s)), "n"(S::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (tid < kEnds * 4) unfit[tid / 4][tid % 4] = 0;
  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mk) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mv) : "memory");
    mbar_init(su32(&q_full), kSoft);
    mbar_init(su32(&pv_done), 1);
    for (int i = 0; i < kStages; ++i) {
      mbar_init(su32(&k_full[i]), 1);
      mbar_init(su32(&k_empty[i]), 1);
      mbar_init(su32(&v_full[i]), 1);
      mbar_init(su32(&v_empty[i]), 1);
    }
    for (int i = 0; i < kInfo; ++i) mbar_init(su32(&info_full[i]), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(su32(&s_full[i]), 1);
      mbar_init(su32(&p_full[i]), kSoft);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tm_fence_before();
  __syncthreads();
  tm_fence_after();
  const uint32_t tmem = tmem_s;
  // a bounded wait; after one gave up none waits any more
  auto hold = [&](uint64_t* bar, uint32_t parity) {
    if (!mbar_try(su32(bar), parity)) hold_on(su32(bar), parity, &dead);
  };

  const T* q = static_cast<const T*>(p.q);
  if (warp < 4) {  // the queries, swizzled as a copy would
    auto fill = [&](auto wide) {  // one kind of load, without branches between those in flight
      constexpr int U = 8;
      for (int i0 = tid; i0 < kRowsT * (DP / 8); i0 += U * kSoft) {
        Vec<T, 8> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int r = (i0 + u * kSoft) / (DP / 8), c = (i0 + u * kSoft) % (DP / 8);
          const int from_r = min(r, rows - 1), from_c = min(c * 8, p.D - 8);
          const T* from = q + (t0 + p.G.div(from_r)) * p.q_ts + (int64_t)(h * p.G.d + p.G.mod(from_r)) * p.q_hs + from_c;
          if constexpr (decltype(wide)::value) {
            v[u] = *reinterpret_cast<const Vec<T, 8>*>(from);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u].v[e] = from[e];
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int r = (i0 + u * kSoft) / (DP / 8), c = (i0 + u * kSoft) % (DP / 8);
          if (r >= rows || c * 8 >= p.D || p.scale == 0.f) v[u] = {};
          if (p.scale < 0.f) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u].v[e] = from_f32<T>(-to_f32(v[u].v[e]));
          }
          *reinterpret_cast<Vec<T, 8>*>(smem + c / 8 * CHUNK_Q + r * 128 + ((c % 8 ^ (r & 7)) << 4)) = v[u];
        }
      }
    };
    if (((reinterpret_cast<uintptr_t>(q) & 15) | (p.q_ts & 7) | (p.q_hs & 7)) == 0)
      fill(std::true_type{});
    else
      fill(std::false_type{});
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    mbar_arrive(su32(&q_full));
  }

  // softmax state of the thread's row
  const int tok = min(p.G.div(tid), nt - 1);
  const bool live_row = tid < rows;
  const int lim = warp < 4 ? limit(tok) : 0;
  float m = -INFINITY, l = 0.f;
  const uint32_t row_tm = tmem + ((uint32_t)(warp * 32) << 16);

  // the first block with keys that some tokens see and others do not (of selected pages each may be one)
  const bool dense = !p.sel;
  const int ends = dense && lim_min < lim_max ? lim_min >> 6 : INT32_MAX / 2;
  const int words = (TT + 31) / 32, window = p.sel ? kMaskWords / words : INT32_MAX;
  int done = 0;  // blocks before this window
  for (int w0 = 0; w0 < P; w0 = p.sel ? w0 + window : P) {
    int npieces = (lim_max + BR - 1) >> log_br;  // of the window: all, or those of the listed pages
    if (p.sel) {
      const int wn = min(window, P - w0);
      __syncthreads();
      for (int i = tid; i < wn * words; i += kThreadsT) masks[i] = 0;
      __syncthreads();
      const int* lists = p.sel + ((int64_t)t0 * p.H + h) * p.keep;
      constexpr int U = kAhead;
      for (int i0 = tid; i0 < nt * p.keep; i0 += U * kThreadsT) {
        int tk[U], w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + u * kThreadsT;
          tk[u] = p.by_keep.div(i);
          w[u] = i < nt * p.keep ? lists[(int64_t)tk[u] * p.H * p.keep + p.by_keep.mod(i)] : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int Pt = (limit(tk[u]) + p.page - 1) >> p.log_page, e = p.by_keep.mod(i0 + u * kThreadsT);
          if (w[u] >= p.width) atomicOr(p.status, PP_CACHE_BAD_PAGE);
          if (e < Pt && w[u] >= w0 && w[u] < w0 + wn && w[u] < Pt) atomicOr(&masks[(w[u] - w0) * words + tk[u] / 32], 1u << (tk[u] % 32));
        }
      }
      __syncthreads();
      // the pages that some token uses, in order
      const int each = (wn + kThreadsT - 1) / kThreadsT, a0 = min(wn, tid * each), a1 = min(wn, a0 + each);
      int used = 0;
      auto any = [&](int w) {
        uint32_t v = 0;
        for (int i = 0; i < words; ++i) v |= masks[w * words + i];
        return v != 0;
      };
      for (int w = a0; w < a1; ++w) used += any(w);
      int at = used;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(~0u, at, d);
        if (lane >= d) at += up;
      }
      if (lane == 31) scan[warp] = at;
      __syncthreads();
      int sum = 0;
#pragma unroll
      for (int i = 0; i < kThreadsT / 32; ++i) {
        if (i < warp) at += scan[i];
        sum += scan[i];
      }
      at -= used;
      for (int w = a0; w < a1; ++w)
        if (any(w)) list[at++] = (uint16_t)w;
      __syncthreads();
      npieces = sum << log_pp;
    }
    // this CTA's share of the window's blocks, and its first piece
    const int blocks = (npieces + pieces - 1) >> log_pc, first = blocks * z / p.splits;
    const int n = blocks * (z + 1) / p.splits - first, i0 = first << log_pc;
    // piece i of the window: its first key, -1 beyond the last
    auto key_of = [&](int i) {
      if (i >= npieces) return -1;
      return p.sel ? ((w0 + list[i >> log_pp]) << p.log_page) + ((i & (1 << log_pp) - 1) << log_br) : i << log_br;
    };

    if (warp == 4) {
      // ---- copies.  Pages are looked up 32 pieces at a time, a lane each; the warp's leader then has the blocks
      // copied
      const uint32_t leader = elect();
      for (int k0 = 0; k0 < n; k0 += 32 >> log_pc) {
        const int key = key_of(i0 + (k0 << log_pc) + lane);
        int have = key < 0 ? 0 : max(0, min(BR, lim_max - key)), y = 0;
        if (have > 0) {
          const int id = table[key >> p.log_page];
          if (id < 0 || id >= p.pages) {
            atomicOr(p.status, PP_CACHE_BAD_PAGE);
            have = 0;
          }
          y = (int)(((int64_t)id * p.H + h) * p.page) + (key & (p.page - 1));
        }
        __syncwarp();
        found[lane] = make_int2(have, y);
        __syncwarp();
        const int k1 = min(n, k0 + (32 >> log_pc));
        for (int k = k0; k < k1; ++k) {
          const int g = done + k, st = g % kStages;
          const uint32_t ph = (g / kStages + 1) & 1;
          const int2* at = found + ((k - k0) << log_pc);
          hold(&k_empty[st], ph);
          // the softmax is done with what was said of block g - 4: the scores of g - 2, just found done, were asked for after
          // it
          int bytes = 0, full = 1;
          for (int j = 0; j < pieces; ++j) {
            const int some = at[j].x;
            if (lane == 0) info[g % kInfo].have[j] = some;
            full &= some == BR;
            bytes += some > 0 ? BR * DP * 2 : 0;
          }
          if (lane == 0) {
            info[g % kInfo].full = full && first + k < ends;
            info[g % kInfo].end = max(0, first + k - ends + 1);
            mbar_arrive(su32(&info_full[g % kInfo]));
          }
          if (*(volatile int*)&dead) bytes = 0;
          auto copy = [&](const CUtensorMap* m, uint32_t to, uint32_t bar) {
            expect(bar, bytes, leader);
            for (int j = 0; j < pieces; ++j) {
              const int2 piece = at[j];
              if (bytes == 0 || piece.x <= 0) continue;
#pragma unroll
              for (int c = 0; c < DP / 64; ++c) copy_box(to + c * CHUNK_KV + j * BR * 128, m, c * 64, piece.y, bar, leader);
            }
          };
          copy(&mk, su32(kbuf) + st * S::KV, su32(&k_full[st]));
          hold(&v_empty[st], ph);
          if (*(volatile int*)&dead) bytes = 0;
          copy(&mv, su32(vbuf) + st * S::KV, su32(&v_full[st]));
        }
        __syncwarp();
      }
    } else if (warp == 5) {
      // ---- products
      const uint32_t leader = elect();
      const uint32_t qa = desc_lo(su32(smem), 16), kb = desc_lo(su32(kbuf), 16), vb = desc_lo(su32(vbuf), CHUNK_KV);
      auto scores = [&](int k) {
        const int g = done + k, st = g % kStages;
        hold(&k_full[st], g / kStages & 1);
        tm_fence_after();
        const uint32_t kd = kb + st * (S::KV >> 4), to = tmem + 128 + (g & 1) * 64;
#pragma unroll
        for (int kk = 0; kk < DP / 16; ++kk)
          mma_ss(to, qa + (kk / 4 * CHUNK_Q + kk % 4 * 32 >> 4), kd + (kk / 4 * CHUNK_KV + kk % 4 * 32 >> 4),
                 idesc<T>(kRowsT, kKeys, false), kk > 0, leader);
        commit(su32(&k_empty[st]), leader);
        commit(su32(&s_full[g & 1]), leader);
      };
      if (n > 0) {
        if (done == 0) hold(&q_full, 0);
        scores(0);
      }
      for (int k = 0; k < n; ++k) {
        const int g = done + k, st = g % kStages;
        if (k + 1 < n) scores(k + 1);
        hold(&v_full[st], g / kStages & 1);
        hold(&p_full[g & 1], g >> 1 & 1);
        tm_fence_after();
        const uint32_t vd = vb + st * (S::KV >> 4), pt = tmem + 128 + (g & 1) * 64;
#pragma unroll
        for (int kk = 0; kk < kKeys / 16; ++kk)
          mma_ts(tmem, pt + kk * 8, vd + (kk * 2048 >> 4), idesc<T>(kRowsT, DP, true), g > 0 || kk > 0, leader);
        commit(su32(&v_empty[st]), leader);
        commit(su32(&pv_done), leader);
      }
    } else {
      // ---- softmax, a thread per row
      for (int k = 0; k < n; ++k) {
        const int g = done + k, st = g % kStages;
        // which of the block's keys the row sees, a bit each
        uint64_t see = 0;
        const Block& bl = info[g % kInfo];
        if (log_pc == 0) {  // a page, or a piece of one
          const int key = key_of(i0 + k);
          bool on = live_row && key >= 0;
          if (on && p.sel) on = masks[list[i0 + k >> log_pp] * words + tok / 32] >> (tok % 32) & 1;
          hold(&info_full[g % kInfo], g / kInfo & 1);
          const int c = on ? min(bl.have[0], lim - key) : 0;
          see = c >= 64 ? ~0ull : c > 0 ? (1ull << c) - 1 : 0;
        } else {
          hold(&info_full[g % kInfo], g / kInfo & 1);
#pragma unroll 1
          for (int j = 0; j < pieces; ++j) {
            const int i = i0 + (k << log_pc) + j, key = key_of(i);
            bool on = live_row && key >= 0;
            if (on && p.sel) on = masks[list[i >> log_pp] * words + tok / 32] >> (tok % 32) & 1;
            const int c = on ? min(bl.have[j], lim - key) : 0;
            if (c > 0) see |= ((1ull << c) - 1) << (j << log_br);
          }
        }
        // (with all pages, a row that sees nothing of a block is masked, too, whatever the keys hold)
        const bool part = __any_sync(~0u, live_row && see != ~0ull && (see != 0 || dense)), none = __all_sync(~0u, see == 0);
        hold(&s_full[g & 1], g >> 1 & 1);
        __syncwarp();
        tm_fence_after();
        const uint32_t tm = row_tm + 128 + (g & 1) * 64;
        uint32_t w[32];
        bool waited = false;
        if (none) {
#pragma unroll
          for (int i = 0; i < 32; ++i) w[i] = 0;
        } else {
          float x[64];
          tm_ld32(tm, reinterpret_cast<float(&)[32]>(x[0]));
          tm_ld32(tm + 32, reinterpret_cast<float(&)[32]>(x[32]));
          tm_wait_ld();
          // rows that see all or nothing need no mask: the latter's exponents are taken from infinity below
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
          const float mx = see ? lower(__fmul_rn(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), sl), kLift<T, kUp>) : -INFINITY;
          const bool grow = mx > __fadd_rd(m, kGrow<T>);  // from -infinity, too
          if (__any_sync(~0u, grow)) {
            const float to = fmaxf(m, mx), f = to == -INFINITY ? 1.f : ex2(m - to);
            m = to;
            l *= f;
            if (g > 0) {  // the sums so far, in TMEM
              hold(&pv_done, (g - 1) & 1);
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
          const float at = see ? (m == -INFINITY ? 0.f : m) : INFINITY;
          const uint64_t sl2 = pack2(sl, sl), at2 = pack2(-at, -at);
          uint64_t sum[4] = {};
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float a, c;
            // scaled as the maximum is and then taken from it, not in one step (a product plus 0, so that the two are not merged):
            // where scores are so large that fp32 numbers lie further than 1 apart, no weight passes its bound and the largest
            // does not vanish
            unpack2(add2(fma2(pack2(x[2 * i], x[2 * i + 1]), sl2, pack2(0.f, 0.f)), at2), a, c);
            a = ex2(a);
            c = ex2(c);
            sum[i & 3] = add2(sum[i & 3], pack2(a, c));
            w[i] = pack<T>(a, c);
          }
          float a, c;
          unpack2(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), a, c);
          l += a + c;
        }
        tm_st32(tm, w);
        if (!bl.full) {
          hold(&v_full[st], g / kStages & 1);
          __syncwarp();
          zero_values<T, DP>(vbuf + st * S::KV, bl, log_br, bl.end ? unfit[bl.end - 1] : nullptr);
        }
        tm_wait_st();
        // each block's products with V are waited for, and in order, so that a parity names one of two phases; those of the
        // block before are done by now
        if (g > 0 && !waited) hold(&pv_done, (g - 1) & 1);
        tm_fence_before();
        mbar_arrive(su32(&p_full[g & 1]));
      }
    }
    done += n;
  }

  // ---- out
  if (warp < 4) {
    if (done > 0) hold(&pv_done, (done - 1) & 1);
    group_sync<kSoft>();  // what was said of the last blocks' keys
    tm_fence_after();
    // the keys of end block e that row r's token sees and whose values are still missing
    auto missing = [&](int e, int limit_of) -> uint64_t {
      const int c = limit_of - (ends + e) * 64;
      const uint64_t bits = *reinterpret_cast<const uint64_t*>(unfit[e]);
      return c >= 64 ? bits : c > 0 ? bits & ((1ull << c) - 1) : 0;
    };
    uint64_t some = 0;
    if (dense)
#pragma unroll
      for (int e = 0; e < kEnds; ++e) some |= missing(e, lim);
    const unsigned lacking = __ballot_sync(~0u, live_row && some != 0);
    auto cell_of = [&](int r, int tk) { return (int64_t)(t0 + tk) * p.H * p.G.d + h * p.G.d + p.G.mod(r); };
    auto queries_of = [&](int r, int tk) { return q + (t0 + tk) * p.q_ts + (int64_t)(h * p.G.d + p.G.mod(r)) * p.q_hs; };
    const int64_t cell = (int64_t)(t0 + p.G.div(live_row ? tid : 0)) * p.H * p.G.d + h * p.G.d + p.G.mod(live_row ? tid : 0);
    if (p.splits > 1) {  // sums as they are, for the joining kernel
      const int64_t at = (int64_t)z * p.T * p.H * p.G.d + cell;
#pragma unroll
      for (int c = 0; c < DP; c += 32) {
        float o[32];
        if (done > 0) {
          tm_ld32(row_tm + c, o);
          tm_wait_ld();
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = 0.f;
        }
        if (live_row)
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            *reinterpret_cast<float4*>(p.split_sums + at * DP + c + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
      }
      if (live_row) p.split_stats[at] = make_float2(m, l);
    } else {
      T* dst = static_cast<T*>(p.out) + cell * p.D;
      const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 15) == 0;
      const float scale = l == 0.f ? 0.f : 1.f / l;
      bool odd = false;
#pragma unroll
      for (int c = 0; c < DP; c += 32) {
        float o[32];
        if (done > 0) {
          tm_ld32(row_tm + c, o);
          tm_wait_ld();
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
          if (c + i >= p.D || !live_row) continue;
          Vec<T, 8> y;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            odd = odd || !isfinite(o[i + e]);
            y.v[e] = from_f32<T>(o[i + e] * scale);
          }
          if (wide) {
            *reinterpret_cast<Vec<T, 8>*>(dst + c + i) = y;
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) dst[c + i + e] = y.v[e];
          }
        }
      }
      if (p.lse && live_row) p.lse[cell] = l == 0.f ? -INFINITY : log_sum<T, kUp>(m, l);
      unsigned again = __ballot_sync(~0u, odd && live_row && p.sel);
      __syncwarp();  // what the rows' own threads wrote lies before what the warp writes over it
      for (; again; again &= again - 1) {
        const int r = warp * 32 + __ffs(again) - 1, tk = p.G.div(r);
        redo_row<T>(p, queries_of(r, tk), table, p.sel + ((int64_t)(t0 + tk) * p.H + h) * p.keep, h, limit(tk), p.scale * 1.44269504f,
                    static_cast<T*>(p.out) + cell_of(r, tk) * p.D, p.lse ? p.lse + cell_of(r, tk) : nullptr);
      }
    }
    __syncwarp();
    for (unsigned left = lacking; left; left &= left - 1) {
      const int from = __ffs(left) - 1, r = warp * 32 + from, tk = p.G.div(r);
      const float mr = __shfl_sync(~0u, m, from), n = 1.f / __shfl_sync(~0u, l, from);
      const int64_t at = cell_of(r, tk);
      // into the row's sums for the joining kernel, or beside (where the queries were, whose products are done)
      float* sums = p.splits > 1 ? p.split_sums + ((int64_t)z * p.T * p.H * p.G.d + at) * DP : reinterpret_cast<float*>(smem) + warp * DP;
      if (p.splits == 1)
        for (int d = lane; d < p.D; d += 32) sums[d] = 0.f;
      for (int e = 0; e < kEnds; ++e)
        add_keys<T, DP>(p, queries_of(r, tk), table, h, (ends + e) * 64, missing(e, limit(tk)), p.scale * 1.44269504f, mr, sums);
      if (p.splits == 1) {
        T* dst = static_cast<T*>(p.out) + at * p.D;
        for (int d = lane; d < p.D; d += 32) dst[d] = from_f32<T>(to_f32(dst[d]) + sums[d] * n);
      }
    }
    tm_fence_before();
  }
  __syncthreads();
  if (dead && tid == 0) {
    atomicOr(p.status, PP_CACHE_TIMEOUT);
    // copies and products still in flight end before the CTA does
    for (int i = 0; i < kStages; ++i)
      for (uint32_t ph = 0; ph < 2; ++ph) wait(su32(&k_full[i]), ph), wait(su32(&v_full[i]), ph);
    for (uint32_t ph = 0; ph < 2; ++ph) wait(su32(&pv_done), ph);
  }
  if (warp == 5) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::COLS));
  }
}

// The splits' sums of a row into its output: a warp per (token, query head).
template <class T, int DP>
__global__ void __launch_bounds__(256) attn_tile_join_kernel(const __grid_constant__ AttnParams p) {
  after_previous();
  const int Hq = p.H * p.G.d, lane = threadIdx.x % 32;
  const int64_t cells = (int64_t)p.T * Hq, cell = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
  if (cell >= cells) return;
  float m = -INFINITY, l = 0.f;
  float2 st[kSplits];
#pragma unroll
  for (int z = 0; z < kSplits; ++z) {
    st[z] = z < p.splits ? p.split_stats[z * cells + cell] : make_float2(-INFINITY, 0.f);
    m = fmaxf(m, st[z].x);
  }
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  const int d = lane * 4 < DP ? lane * 4 : 0;
#pragma unroll
  for (int z = 0; z < kSplits; ++z) {
    if (st[z].y == 0.f) continue;
    const float w = ex2(st[z].x - m);
    const float4 a = *reinterpret_cast<const float4*>(p.split_sums + (z * cells + cell) * DP + d);
    l += w * st[z].y;
    o.x += w * a.x;
    o.y += w * a.y;
    o.z += w * a.z;
    o.w += w * a.w;
  }
  const bool in = lane * 4 < p.D;
  const bool odd = in && !(isfinite(o.x) && isfinite(o.y) && isfinite(o.z) && isfinite(o.w));
  const int t = (int)(cell / Hq), hq = (int)(cell - (int64_t)t * Hq);
  T* out = static_cast<T*>(p.out) + cell * p.D;
  float* lse = p.lse ? p.lse + cell : nullptr;
  if (p.sel && __any_sync(~0u, odd)) {
    const Seen s = seen_keys(t, p.T, p.B, p.starts, p.lens, p.width * p.page, p.causal, p.status);
    const int h = p.G.div(hq);
    redo_row<T>(p, static_cast<const T*>(p.q) + t * p.q_ts + (int64_t)hq * p.q_hs, p.table + (int64_t)s.b * p.width,
                p.sel + ((int64_t)t * p.H + h) * p.keep, h, s.keys, p.scale * 1.44269504f, out, lse);
    return;
  }
  const float n = l == 0.f ? 0.f : 1.f / l;
  if (in) {
    const Vec<T, 4> y = {from_f32<T>(o.x * n), from_f32<T>(o.y * n), from_f32<T>(o.z * n), from_f32<T>(o.w * n)};
    if ((reinterpret_cast<uintptr_t>(p.out) & 7) == 0) {
      *reinterpret_cast<Vec<T, 4>*>(out + d) = y;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) out[d + e] = y.v[e];
    }
  }
  if (lse && lane == 0) *lse = l == 0.f ? -INFINITY : log_sum<T, kUp>(m, l);
}

template <class T, int DP>
cudaError_t prepare_one() {
  return cudaFuncSetAttribute(attn_tile_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, TileShape<DP>::SMEM);
}

template <class T, int DP>
cudaError_t launch(const AttnParams& p, const pp_cache& c, int64_t grid, cudaStream_t stream) {
  const cudaError_t e = launch_after(attn_tile_kernel<T, DP>, dim3((unsigned)grid), kThreadsT, TileShape<DP>::SMEM, stream, 1,
                                     p, c.mk, c.mv);
  if (e != cudaSuccess || p.splits == 1) return e;
  const int64_t cells = (int64_t)p.T * p.H * p.G.d;
  return launch_after(attn_tile_join_kernel<T, DP>, dim3((unsigned)((cells + 7) / 8)), 256, 0, stream, 1, p);
}

}  // namespace

namespace ppc_attn {

// Tiles of a call at most: each sequence adds at most one that is not full.
static int64_t most_tiles(const AttnParams& p) { return ((int64_t)p.T / (kRowsT / p.G.d) + std::min(p.T, p.B)) * p.H; }

bool tile_applicable(const AttnParams& p, int dtype, int sms) {
  if (dtype == PP_F32 || p.D > 128 || p.G.d > 64 || !p.starts) return false;
  // a tile's list entries are counted in 32 bits
  if (p.sel && (int64_t)(kRowsT / p.G.d) * p.keep > INT32_MAX - 2 * kAhead * kThreadsT) return false;
  // Units of rows (attn.cu) share the keys' length among all CTAs, but meet each key with 16 rows (one token's, where pages
  // are selected) at about 1 us per 64 keys and CTA; a tile meets it with 128 in about the same, split 8 times at most.
  // Selected pages: neighbouring tokens' together are some four times one token's.
  // How tokens are spread over sequences is not known here.  Where sequences have less than a unit's 16 rows each (then
  // there can be more than 9 tiles to 8 units), a tile would hold no more rows than a unit and be walked whole by one CTA:
  // one token each of 32 sequences, of which one has 65536 keys, 32 heads of 128 over 8: 101 us by units, 956 by tiles.
  // With 4 tokens each of 32 sequences of up to 8192: 171 us by units, 143 by tiles.
  const int64_t few = 2 * sms / kSplits, tiles = most_tiles(p);
  const int64_t units = p.sel ? (int64_t)p.T * ((p.G.d + 7) / 8) * p.H : ((int64_t)p.T * p.G.d + 15) / 16 * p.H;
  return p.sel ? std::max(tiles, few) * 4 < units : few < units && tiles * 8 <= units * 9;
}

cudaError_t tile_prepare() {
  cudaError_t e = prepare_one<__half, 64>();
  if (e == cudaSuccess) e = prepare_one<__half, 128>();
  if (e == cudaSuccess) e = prepare_one<__nv_bfloat16, 64>();
  if (e == cudaSuccess) e = prepare_one<__nv_bfloat16, 128>();
  return e;
}

size_t tile_space(int dtype, int D, int sms) {
  return dtype == PP_F32 || D > 128 ? 0 : (size_t)2 * sms * kRowsT * ((D <= 64 ? 64 : 128) + 2) * 4;
}

cudaError_t tile_launch(AttnParams p, const pp_cache& c, int sms, cudaStream_t stream) {
  const int TT = kRowsT / p.G.d, DP = p.D <= 64 ? 64 : 128;
  const int64_t tiles = most_tiles(p);  // CTAs beyond the last tile leave
  // Few tiles are split along their blocks, up to two CTAs per SM, while a share can have 4 blocks (a CTA spends the time of
  // about 8 on its queries and masks, but side by side with the others).  3 chunks of 333 tokens, 8 heads of 64: 71 us
  // whole, 35 in four shares; 119 tokens of 2 heads over 1720 keys, with their selection: 50 us whole, 31 in shares.
  const int64_t cells = (int64_t)p.T * p.H * p.G.d, room = (int64_t)2 * sms * kRowsT;
  const int64_t pages = p.sel ? std::min<int64_t>(p.width, (int64_t)TT * p.keep) : p.width;
  const int64_t splits = std::min({(int64_t)kSplits, 2 * sms / tiles, pages * p.page / kKeys / 4, room / cells});
  p.splits = (int)std::max<int64_t>(1, splits);
  p.split_sums = c.tiles;
  p.split_stats = reinterpret_cast<float2*>(c.tiles + room * DP);
  const int64_t grid = tiles * p.splits;
  if (grid > INT32_MAX) return cudaErrorInvalidValue;
  return c.dtype == PP_F16 ? (DP == 64 ? launch<__half, 64>(p, c, grid, stream) : launch<__half, 128>(p, c, grid, stream))
                           : (DP == 64 ? launch<__nv_bfloat16, 64>(p, c, grid, stream)
                                       : launch<__nv_bfloat16, 128>(p, c, grid, stream));
}

}  // namespace ppc_attn
