// Selection of the pages worth reading (pp_cache_select).
//
// score = scale (p . codes[0] + m . codes[1]) with whole numbers: p and m sum the
// positive and the negative parts of the group's rounded queries, so the sum over
// the 2 D codes of a page is one integer below 2^24, exact in any order and in
// fp32 products of f16 values up to 2048 as well.  Scores are compared as integers
// of the same order, equal ones by page.
//
// Two kernels: for single tokens, integer products by a cluster per (token, head),
// bound by reading the codes once; for many tokens, 16 of them at a time on the
// tensor cores (mma.sync m16n8k16, f16), bound by neither bytes nor products but
// by instructions: the codes' conversion and the search for the keep-th largest score
// (in 8-bit products, m16n8k32 with the integers as 128 hi + lo: 96 us against 71).
//
// Measured, 32 heads over 8, D = 128: one token over 625 pages 7.7 us, 32 tokens over up
// to 512 pages 12.4 us (chains of latencies), 2048 tokens over 512 pages 71 us (132 in a
// table of 2048, whose scores leave an SM one block; 600 in a wider one, token by token).
#include <algorithm>

#include "cache.h"
#include "internal.h"
#include "tc_ptx.cuh"

namespace {

using namespace ppc;
using namespace ppc_ptx;

constexpr int kThreads = 256;

struct SelectParams {
  const void* q;
  int64_t q_ts, q_hs;
  const int *starts, *table, *lens;
  const int8_t* codes;
  const float* scales;
  int* sel;
  int* status;
  int T, B, H, G, D, page, pages, width, first, last, keep, Q, causal;
};

// A score as an integer of the same order; NaN as the lowest.
__device__ __forceinline__ uint32_t ordered(float v) {
  if (v != v) v = -INFINITY;
  const uint32_t u = __float_as_uint(v + 0.f);  // one zero
  return u >> 31 ? ~u : u | 0x80000000u;
}

// The integers of token t's queries of head h, by one warp: store(d, up, down) for every value d of the head.  A lane
// takes 8 values of every per-th head of the group; the largest first, then the rounded ones, summed over the group.
// Loads are asked for together and without conditions (a clamped place instead), so that they wait for memory once.
template <class T, bool WIDE, class F>
__device__ __forceinline__ void group_values(const T* q, int64_t q_hs, int G, int g0, int per, bool in, F&& use) {
  constexpr int U = 4;
  for (int g = g0; g - g0 < G; g += U * per) {
    Vec<T, 8> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const T* from = q + min(g + u * per, G - 1) * q_hs;
      if (WIDE) {
        v[u] = *reinterpret_cast<const Vec<T, 8>*>(from);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[u].v[i] = from[i];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (in && g + u * per < G)
#pragma unroll
        for (int i = 0; i < 8; ++i) use(i, to_f32(v[u].v[i]));
  }
}
template <class T, bool WIDE, class F>
__device__ __forceinline__ void query_codes_of(const SelectParams& p, const T* q, int lane, F&& store) {
  const int chunks = p.D / 8;
  int span = 2;
  while (span < chunks) span *= 2;
  const int c = lane & (span - 1), per = 32 / span;
  const bool in = c < chunks;
  const T* from = q + min(c, chunks - 1) * 8;
  float m = 0.f;
  group_values<T, WIDE>(from, p.q_hs, p.G, lane / span, per, in, [&](int, float v) {
    m = fabsf(v) <= 3.402823466e38f ? fmaxf(m, fabsf(v)) : INFINITY;  // a NaN too
  });
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
  const bool zero = !(m >= kTiny) || m == INFINITY;
  const float r = zero ? 0.f : __fdiv_rn((float)p.Q, m);
  int up[8] = {}, down[8] = {};
  if (!zero)
    group_values<T, WIDE>(from, p.q_hs, p.G, lane / span, per, in, [&](int i, float v) {
      const int k = (int)rintf(__fmul_rn(v, r));
      up[i] += max(k, 0);
      down[i] += min(k, 0);
    });
  for (int d = span; d < 32; d *= 2)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      up[i] += __shfl_xor_sync(~0u, up[i], d);
      down[i] += __shfl_xor_sync(~0u, down[i], d);
    }
  if (lane < chunks)
#pragma unroll
    for (int i = 0; i < 8; ++i) store(c * 8 + i, up[i], down[i]);
}
template <class T, class F>
__device__ __forceinline__ void query_codes(const SelectParams& p, int t, int h, int lane, F&& store) {
  const T* q = static_cast<const T*>(p.q) + t * p.q_ts + (int64_t)h * p.G * p.q_hs;
  if (((reinterpret_cast<uintptr_t>(q) | (uintptr_t)(p.q_hs * sizeof(T))) & (sizeof(Vec<T, 8>) - 1)) == 0)
    query_codes_of<T, true>(p, q, lane, store);
  else
    query_codes_of<T, false>(p, q, lane, store);
}

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}

// Single tokens: a cluster per (token, head), its CTAs sharing the pages.  Bound by reading the codes, 2 D bytes a page:
// a lane keeps 16 of the query's integers, as 128 hi + lo, and meets 16 codes of every page with four-way integer products.  The first
// CTA has all scores in shared memory and finds the keep-th largest digit by digit (8 bits each).
template <class T>
__global__ void __launch_bounds__(kThreads) select_kernel(const SelectParams p) {
  extern __shared__ uint32_t key[];
  __shared__ __align__(16) int8_t code[2][512];  // lo (0 .. 127) and hi of the query's integers
  __shared__ uint2 ends[8 * kThreads / 32];  // the least and the largest key of every warp of the cluster
  __shared__ int hist[256], warp_sum[kThreads / 32], digit_of, left_of;
  const int rank = cluster_rank(), ranks = cluster_size();
  const int t = blockIdx.x / ranks, h = blockIdx.y, tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  after_previous();
  const Seen s = seen_keys(t, p.T, p.B, p.starts, p.lens, p.width * p.page, p.causal, p.status);
  const int P = (s.keys + p.page - 1) / p.page;
  int* out = p.sel + ((int64_t)t * p.H + h) * p.keep;
  // by a warp that waits for the queries' integers
  auto ranges = [&]() {
    if (p.starts && blockIdx.x == 0 && h == 0 && warp == kThreads / 32 - 1) check_ranges(p.starts, p.T, p.B, lane, 32, p.status);
  };
  if (P <= p.keep) {  // the whole cluster
    ranges();
    if (rank == 0)
      for (int i = tid; i < p.keep; i += kThreads) out[i] = i < P ? i : -1;
    return;
  }
  // every CTA of the cluster has begun before one writes to the first's shared memory
  if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  // candidates: pages first .. P - last - 1; this CTA's are from .. to - 1.  Their ids first, where the scores will be
  const int N = P - p.first - p.last, share = (N + ranks - 1) / ranks, from = min(N, rank * share), to = min(N, from + share);
  const int* row = p.table + (int64_t)s.b * p.width + p.first;
  for (int w = from + tid; w < to; w += kThreads) key[w] = (uint32_t)row[w];
  if (warp == 0)
    query_codes<T>(p, t, h, lane, [&](int d, int up, int down) {
      code[0][d] = (int8_t)(up & 127);
      code[1][d] = (int8_t)(up >> 7);
      code[0][p.D + d] = (int8_t)(down & 127);
      code[1][p.D + d] = (int8_t)(down >> 7);
    });
  ranges();
  __syncwarp();
  if (ranks > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  __syncthreads();
  // 2 D / 16 lanes a page, in a power of two
  const int chunks = p.D / 8;
  int span = 2;
  while (span < chunks) span *= 2;
  const int at = lane % span, per = 32 / span;  // pages per warp at a time
  int4 lo = make_int4(0, 0, 0, 0), hi = lo;
  if (at < chunks) {
    lo = reinterpret_cast<const int4*>(code[0])[at];
    hi = reinterpret_cast<const int4*>(code[1])[at];
  }
  const uint32_t keys0 = map_rank((uint32_t)__cvta_generic_to_shared(key), 0);
  uint32_t mn = ~0u, mx = 0;  // of the keys that this warp makes
  constexpr int U = 8;
  for (int w0 = from + warp * U * per; w0 < to; w0 += (kThreads / 32) * U * per) {
    int4 c[U];
    float sc[U];
    bool bad[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // no conditions around the loads, so that they are under way together: page 0 in the place of what is none
      const int w = w0 + u * per + lane / span, id = (int)key[min(w, to - 1)];
      const bool good = id >= 0 && id < p.pages;
      const int64_t cell = (int64_t)(good ? id : 0) * p.H + h;
      c[u] = *reinterpret_cast<const int4*>(p.codes + cell * 2 * p.D + min(at, chunks - 1) * 16);
      sc[u] = p.scales[cell];
      bad[u] = !good;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!bad[u]) continue;
      sc[u] = nanf("");
      if (at == 0 && w0 + u * per + lane / span < to) atomicOr(p.status, PP_CACHE_BAD_PAGE);
    }
    __syncwarp();  // the ids are read before scores take their places
    int sum[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      sum[u] = __dp4a(hi.x, c[u].x, __dp4a(hi.y, c[u].y, __dp4a(hi.z, c[u].z, __dp4a(hi.w, c[u].w, 0)))) * 128;
      sum[u] = __dp4a(lo.x, c[u].x, __dp4a(lo.y, c[u].y, __dp4a(lo.z, c[u].z, __dp4a(lo.w, c[u].w, sum[u]))));
    }
    for (int d = span / 2; d > 0; d >>= 1)
#pragma unroll
      for (int u = 0; u < U; ++u) sum[u] += __shfl_xor_sync(~0u, sum[u], d);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int w = w0 + u * per + lane / span;
      const uint32_t v = ordered(__fmul_rn((float)sum[u], sc[u]));
      mn = min(mn, w < to ? v : ~0u);
      mx = max(mx, w < to ? v : 0);
      if (at == 0 && w < to) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(keys0 + 4 * w), "r"(v) : "memory");
    }
  }
  mn = __reduce_min_sync(~0u, mn);
  mx = __reduce_max_sync(~0u, mx);
  if (lane == 0)
    asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(map_rank((uint32_t)__cvta_generic_to_shared(&ends[rank * (kThreads / 32) + warp]), 0)),
                 "r"(mn), "r"(mx) : "memory");
  if (ranks > 1)
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  else
    __syncthreads();
  if (rank != 0) return;
  // the need-th largest key: thr, with `need` of those equal to it (under the mask of the bits found), digit by digit of 8
  // bits below the bits that all keys have in common
  int need = p.keep - p.first - p.last;
  for (int i = 0; i < ranks * (kThreads / 32); ++i) {
    mn = min(mn, ends[i].x);
    mx = max(mx, ends[i].y);
  }
  int low = 32 - __clz(mn ^ mx);  // bits not found yet
  uint32_t mask = low == 32 ? 0 : ~0u << low, thr = mx & mask;
  while (low > 0 && need > 0) {
    const int bits = min(low, 8), shift = low - bits;
    low = shift;
    hist[tid] = 0;
    __syncthreads();
    for (int w = tid; w < N; w += kThreads)
      if ((key[w] & mask) == thr) atomicAdd(&hist[key[w] >> shift & (1 << bits) - 1], 1);
    __syncthreads();
    const int have = hist[255 - tid];  // digits from the largest down
    int sum = have;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(~0u, sum, d);
      if (lane >= d) sum += o;
    }
    if (lane == 31) warp_sum[warp] = sum;
    __syncthreads();
    for (int i = 0; i < warp; ++i) sum += warp_sum[i];
    if (sum >= need && sum - have < need) {
      digit_of = 255 - tid;
      left_of = need - (sum - have);
    }
    __syncthreads();
    thr |= (uint32_t)digit_of << shift;
    mask |= (1u << bits) - 1 << shift;
    need = left_of;
    if (hist[digit_of] == need) break;  // all that start like this
    __syncthreads();
  }
  __syncthreads();
  // each thread a run of pages, in order: those above thr, and the first `need` equal to it
  const int len = (N + kThreads - 1) / kThreads, w0 = min(N, tid * len), w1 = min(N, w0 + len);
  int above = 0, equal = 0;
  if (p.keep > p.first + p.last)
    for (int w = w0; w < w1; ++w) {
      const uint32_t v = key[w] & mask;
      above += v > thr;
      equal += v == thr;
    }
  int sum = above | equal << 16;  // above < 2^11, equal <= 2^15
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(~0u, sum, d);
    if (lane >= d) sum += o;
  }
  if (lane == 31) warp_sum[warp] = sum;
  __syncthreads();
  for (int i = 0; i < warp; ++i) sum += warp_sum[i];
  sum -= above | equal << 16;
  int a = sum & 0xFFFF, e = (uint32_t)sum >> 16;
  if (p.keep > p.first + p.last)
    for (int w = w0; w < w1; ++w) {
      const uint32_t v = key[w] & mask;
      if (v > thr || (v == thr && e < need)) out[p.first + a + min(e, need)] = p.first + w;
      a += v > thr;
      e += v == thr;
    }
  for (int i = tid; i < p.first; i += kThreads) out[i] = i;
  for (int i = tid; i < p.last; i += kThreads) out[p.keep - p.last + i] = P - p.last + i;
}

// ---- many tokens: a block per (16 tokens, head)

constexpr int kTokens = 16;
constexpr int kTileWidth = 2048;  // pages whose scores fit: 16 x 2048 x 4 bytes
constexpr int kExact = 2048;      // whole numbers up to this are exact in f16

// Four codes as two pairs of f16: a byte plus 128 is the low byte of 1024 + byte, less 1152.
__device__ __forceinline__ void codes_f16(uint32_t x, uint32_t& lo, uint32_t& hi) {
  const uint32_t u = x ^ 0x80808080u, a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
  const __half2 bias = __half2half2(__ushort_as_half(0x6480));
  const __half2 l = __hsub2(*reinterpret_cast<const __half2*>(&a), bias), h = __hsub2(*reinterpret_cast<const __half2*>(&b), bias);
  lo = *reinterpret_cast<const uint32_t*>(&l);
  hi = *reinterpret_cast<const uint32_t*>(&h);
}

// The `need` best of N keys, by one warp: their places plus `first`, ascending, to out.  A lane has every 32nd key in
// registers; the largest thr that `need` keys reach is found bit by bit, below the bits that all keys have in common.
template <int M>
__device__ __forceinline__ void best_of(const uint32_t* key, int N, int need, int first, int lane, int* out) {
  uint32_t k[M], mn = ~0u, mx = 0;
#pragma unroll
  for (int i = 0; i < M; ++i) {
    const int w = lane + 32 * i;
    k[i] = w < N ? key[w] : 0;  // no score is that low
    if (w < N) {
      mn = min(mn, k[i]);
      mx = max(mx, k[i]);
    }
  }
  mn = __reduce_min_sync(~0u, mn);
  mx = __reduce_max_sync(~0u, mx);
  const int top = 32 - __clz(mn ^ mx);  // bits that differ
  uint32_t thr = top == 32 ? 0 : mx >> top << top;
  bool exact = false;
  for (int bit = top - 1; bit >= 0 && !exact; --bit) {
    const uint32_t at = thr | 1u << bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) n += k[i] >= at;
    n = __reduce_add_sync(~0u, n);
    if (n >= need) thr = at;
    exact = n == need;
  }
  int equal = need;  // of those equal to thr, that many
  if (!exact) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) n += k[i] > thr;
    equal = need - __reduce_add_sync(~0u, n);
  }
  const unsigned below = (1u << lane) - 1;
  int at = 0;
#pragma unroll
  for (int i = 0; i < M; ++i) {
    const int w = lane + 32 * i;
    if (w - lane >= N) break;
    const bool in = w < N, same = in && k[i] == thr;
    const unsigned same_of = __ballot_sync(~0u, same);
    const bool take = in && (k[i] > thr || (same && __popc(same_of & below) < equal));
    const unsigned take_of = __ballot_sync(~0u, take);
    if (take) out[at + __popc(take_of & below)] = first + w;
    at += __popc(take_of);
    equal -= min(equal, __popc(same_of));
  }
}

template <class T>
__global__ void __launch_bounds__(kThreads, 3) select_tile_kernel(const SelectParams p) {
  extern __shared__ uint32_t key[];  // [16][stride] scores
  __shared__ __align__(16) __half code[kTokens * (512 + 4)];
  __shared__ int row_b[kTokens], row_P[kTokens];
  const int t0 = blockIdx.x * kTokens, h = blockIdx.y, tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  const int nt = min(kTokens, p.T - t0), D2 = 2 * p.D, cs = D2 + 4, stride = p.width + 4;  // rows 2 and 4 banks apart
  after_previous();
  // ---- the tokens' sequences, a lane each, and their integers, a warp per token
  if (warp == 0 && lane < kTokens) {
    Seen s = {-1, 0};
    if (lane < nt) s = seen_keys(t0 + lane, p.T, p.B, p.starts, p.lens, p.width * p.page, p.causal, p.status);
    row_b[lane] = s.b;
    row_P[lane] = (s.keys + p.page - 1) / p.page;
  }
  if (warp == 1 && p.starts && blockIdx.x == 0 && h == 0) check_ranges(p.starts, p.T, p.B, lane, 32, p.status);
  __syncthreads();
  for (int r = warp; r < kTokens; r += kThreads / 32) {
    auto store = [&](int d, int up, int down) {
      code[r * cs + d] = __int2half_rn(up);
      code[r * cs + p.D + d] = __int2half_rn(down);
    };
    if (r < nt && row_P[r] > p.keep) {
      query_codes<T>(p, t0 + r, h, lane, store);
    } else {
      for (int d = lane; d < p.D; d += 32) store(d, 0, 0);
    }
  }
  __syncthreads();
  // ---- scores, sequence by sequence of the tile; a warp takes 32 pages at a time.  The sum does not mind the order of
  // the 2 D terms: lane t of a quad has bytes 16 t .. 16 t + 15 of each 64, four of them in each of four products.
  const int g = lane / 4, t = lane % 4;
  for (int r0 = 0; r0 < nt;) {
    const int b = row_b[r0];
    int r1 = r0, P = 0;
    for (; r1 < nt && row_b[r1] == b; ++r1) P = max(P, row_P[r1]);
    const int w1 = P <= p.keep ? 0 : P - p.last;
    const int* row = p.table + (int64_t)b * p.width;
    for (int w0 = p.first + warp * 32; w0 < w1; w0 += kThreads) {
      float c[4][4] = {};
      // no conditions around the loads, so that they are under way together: page 0 in the place of what is none
      float scale[4];
      const int8_t* from[4];
      int id[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) id[j] = row[min(w0 + j * 8 + g, w1 - 1)];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t cell = (int64_t)(id[j] >= 0 && id[j] < p.pages ? id[j] : 0) * p.H + h;
        scale[j] = p.scales[cell];
        from[j] = p.codes + cell * D2;
      }
      for (int d0 = 0; d0 < D2; d0 += 64) {
        const bool in = d0 + t * 16 < D2;
        uint4 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const uint4*>(from[j] + (in ? d0 + t * 16 : 0));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint2 lo = make_uint2(0, 0), hi = lo;
          if (in) {
            lo = *reinterpret_cast<const uint2*>(code + g * cs + d0 + t * 16 + i * 4);
            hi = *reinterpret_cast<const uint2*>(code + (g + 8) * cs + d0 + t * 16 + i * 4);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t b0, b1;
            codes_f16(i == 0 ? x[j].x : i == 1 ? x[j].y : i == 2 ? x[j].z : x[j].w, b0, b1);
            asm volatile(
                "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                : "+f"(c[j][0]), "+f"(c[j][1]), "+f"(c[j][2]), "+f"(c[j][3])
                : "r"(lo.x), "r"(hi.x), "r"(lo.y), "r"(hi.y), "r"(b0), "r"(b1));
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (id[j] < 0 || id[j] >= p.pages) {
          scale[j] = nanf("");
          if (t == 0 && w0 + j * 8 + g < w1) atomicOr(p.status, PP_CACHE_BAD_PAGE);
        }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float sc = __shfl_sync(~0u, scale[j], (2 * t + (e & 1)) * 4);
          const int r = g + 8 * (e >> 1), w = w0 + j * 8 + 2 * t + (e & 1);
          if (r >= r0 && r < r1 && w < w1) key[r * stride + w] = ordered(__fmul_rn(c[j][e], sc));
        }
    }
    r0 = r1;
  }
  __syncthreads();
  // ---- the keep best of each token, a warp per token
  for (int r = warp; r < nt; r += kThreads / 32) {
    const int P = row_P[r], N = P - p.first - p.last;
    const int need = p.keep - p.first - p.last;
    int* out = p.sel + ((int64_t)(t0 + r) * p.H + h) * p.keep;
    if (P <= p.keep) {
      for (int i = lane; i < p.keep; i += 32) out[i] = i < P ? i : -1;
      continue;
    }
    if (need > 0) {
      const uint32_t* k = key + r * stride + p.first;
      if (N <= 8 * 32)
        best_of<8>(k, N, need, p.first, lane, out + p.first);
      else if (N <= 16 * 32)
        best_of<16>(k, N, need, p.first, lane, out + p.first);
      else if (N <= 32 * 32)
        best_of<32>(k, N, need, p.first, lane, out + p.first);
      else
        best_of<64>(k, N, need, p.first, lane, out + p.first);
    }
    for (int i = lane; i < p.first; i += 32) out[i] = i;
    for (int i = lane; i < p.last; i += 32) out[p.keep - p.last + i] = P - p.last + i;
  }
}

template <class T>
cudaError_t prepare_type() {
  cudaError_t e = cudaFuncSetAttribute(select_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 131072);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(select_tile_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTokens * (kTileWidth + 4) * 4);
  return e;
}

template <class T>
cudaError_t launch(const SelectParams& p, int sms, cudaStream_t stream) {
  // Many tokens per sequence: 16 of them meet a page's codes at once (2048 tokens, 512 pages: 571 us by single tokens).
  // Not where a sum of queries passes what f16 holds exactly, nor where the scores of 16 tokens do not fit.
  if (p.starts && (int64_t)p.T >= (int64_t)p.B * 4 && p.Q * p.G <= kExact && p.width <= kTileWidth) {
    const dim3 grid((p.T + kTokens - 1) / kTokens, p.H);
    return launch_after(select_tile_kernel<T>, grid, kThreads, (size_t)kTokens * (p.width + 4) * 4, stream, 1, p);
  }
  // CTAs per (token, head): more where there are few, so that long tables are read by enough of them
  int ranks = 1;
  while (ranks < 8 && (int64_t)p.T * p.H * ranks * 2 <= sms * 2 && p.width >= ranks * 2 * 128) ranks *= 2;
  if ((int64_t)p.T * ranks > INT32_MAX) return cudaErrorInvalidValue;
  return launch_after(select_kernel<T>, dim3(p.T * ranks, p.H), kThreads, (size_t)p.width * 4, stream, ranks, p);
}

DeviceOnce g_select_once;

}  // namespace

namespace ppc {

cudaError_t select_prepare() {
  return g_select_once.run([](int) {
    cudaError_t e = prepare_type<float>();
    if (e == cudaSuccess) e = prepare_type<__half>();
    if (e == cudaSuccess) e = prepare_type<__nv_bfloat16>();
    return e;
  });
}

}  // namespace ppc

extern "C" pp_status pp_cache_select(const pp_cache* cache, int T, const void* q, int64_t q_ts, int64_t q_hs, int Hq,
                                     int B, const int32_t* starts, const int32_t* table, int width, const int32_t* lens,
                                     int flags, int first, int last, int keep, int32_t* sel, void* stream) {
  if (!cache || !cache->codes || T < 0 || B < 0 || Hq < 1 || Hq % cache->H || width < 1 || q_ts < 0 || q_hs < 0 ||
      first < 0 || last < 1 || keep < 1 || (int64_t)first + last > keep || (flags & ~PP_ATTN_CAUSAL))
    return PP_ERR_INVALID_ARG;
  if (T > 0 && (!q || !table || !lens || !sel || B < 1 || (!starts && T != B) ||
                (reinterpret_cast<uintptr_t>(q) & (dtype_size(cache->dtype) - 1))))
    return PP_ERR_INVALID_ARG;
  const int G = Hq / cache->H;
  const int64_t Q = std::min<int64_t>(127, (1 << 24) / ((int64_t)127 * cache->D * G));
  if (width > 32768 || keep > 1024 || Q < 1) return PP_ERR_UNSUPPORTED;
  if (T == 0) return PP_OK;
  const int sms = device_sms();
  if (sms <= 0) return PP_ERR_CUDA;
  SelectParams p = {q, q_ts, q_hs, starts, table, lens, cache->codes, cache->scales, sel, cache->status, T, B, cache->H, G,
                    cache->D, cache->page, cache->pages, width, first, last, keep, (int)Q, flags & PP_ATTN_CAUSAL};
  const cudaStream_t s = (cudaStream_t)stream;
  const cudaError_t e = cache->dtype == PP_F32   ? launch<float>(p, sms, s)
                        : cache->dtype == PP_F16 ? launch<__half>(p, sms, s)
                                                 : launch<__nv_bfloat16>(p, sms, s);
  return e == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}
