// The paged cache in 8 bits: new keys and values quantised as they are written
// (pp_cache_append) and read back (pp_cache_read).
//
// A page's values of one head are whole numbers of -127 .. 127 times one fp32 scale,
// a 127th of the largest value written since the page's first token.  Tokens come in
// order, so a page may have to take a larger value than its scale holds: the codes
// that it has are then rounded again to the new scale, by the same block that writes
// the new ones.  Every step is one fp32 operation, rounded to nearest: codes and
// scales depend on nothing but the values and how they were split into calls.
#include <algorithm>
#include <cmath>

#include "cache.h"
#include "internal.h"

namespace {

using namespace ppc;

struct AppendParams {
  const void* x[2];  // keys, values
  int64_t ts[2], hs[2];
  int8_t* codes[2];
  float* scales[2];
  const int *starts, *table, *lens;
  int* status;
  int T, B, H, D, page, log_page, pages, width;
  FastDiv row;  // by the 8-value chunks of a row
};

constexpr int kThreads = 128;
constexpr int kHeld = 8;       // chunks of 8 values that a thread keeps between the two passes: a page of 64 x 128

template <class T, bool WIDE>
__device__ __forceinline__ void load8(const T* x, float (&v)[8]) {
  constexpr int V = 16 / sizeof(T);
  if constexpr (WIDE) {
#pragma unroll
    for (int i = 0; i < 8; i += V) {
      const Vec<T, V> a = *reinterpret_cast<const Vec<T, V>*>(x + i);
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const float2 f = get2(a, e / 2);
        v[i + e] = f.x;
        v[i + e + 1] = f.y;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32(x[i]);
  }
}

__device__ __forceinline__ uint32_t code(float v) {
  return (uint32_t)__float2int_rn(fminf(fmaxf(v, -127.f), 127.f)) & 255u;
}
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float r) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i / 4] |= code(__fmul_rn(v[i], r)) << i % 4 * 8;
  return make_uint2(w[0], w[1]);
}

// One block per page that a sequence's new tokens fall in, head, and pool: the largest new value, the page's scale, its
// older codes where the scale has grown, then the new codes.  The values stay in registers in between (pages of up to
// 64 x 128; of larger ones the rest is read again, out of L2).
template <class T, bool WIDE>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ AppendParams p) {
  __shared__ float most[kThreads / 32];
  after_previous();
  const int h = blockIdx.y, pool = blockIdx.z, tid = threadIdx.x;
  int b = blockIdx.x, s0 = b, n = 1, i = 0;
  if (p.starts) {
    // A sequence whose tokens begin at s has the blocks from s / page + 2 b on: no fewer than the pages that they fall in
    const int at = blockIdx.x;
    auto base = [&](int b) { return (min(max(p.starts[b], 0), p.T) >> p.log_page) + 2 * b; };
    int lo = 0, hi = p.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (base(mid) <= at) lo = mid; else hi = mid;
    }
    b = lo;
    s0 = p.starts[b];
    n = p.starts[b + 1] - s0;
    i = at - base(b);
    if (at == 0 && h == 0 && pool == 0) check_ranges(p.starts, p.T, p.B, tid, kThreads, p.status);
    if (s0 < 0 || n < 0 || s0 > p.T - n || i < 0) return;
  }
  const int len = p.lens[b];
  if (len < 0 || len > p.width << p.log_page) {
    if (tid == 0 && i == 0) atomicOr(p.status, PP_CACHE_BAD_LENGTH);
    return;
  }
  // positions of the new tokens: from .. len - 1, of which this block has those of one page
  const int from = len - n, page_of = (max(from, 0) >> p.log_page) + i;
  if (len == 0 || page_of > (len - 1) >> p.log_page) return;
  const int lo = max(max(from, 0), page_of << p.log_page), hi = min(len - (page_of << p.log_page), p.page) + (page_of << p.log_page);
  if (lo >= hi) return;
  const int id = p.table[(int64_t)b * p.width + page_of];
  if (id < 0 || id >= p.pages) {
    if (tid == 0) atomicOr(p.status, PP_CACHE_BAD_PAGE);
    return;
  }
  const int64_t cell = (int64_t)id * p.H + h;
  const int at = lo & (p.page - 1);
  int8_t* codes = p.codes[pool] + cell * p.page * p.D;
  const float had = at ? p.scales[pool][cell] : 0.f;
  const int64_t ts = p.ts[pool];
  const T* x = static_cast<const T*>(p.x[pool]) + (s0 + lo - from) * ts + h * p.hs[pool];
  const int chunks = (hi - lo) * p.row.d;
  auto chunk = [&](int c, float (&v)[8]) {
    const int r = p.row.div(c);
    load8<T, WIDE>(x + r * ts + (c - r * p.row.d) * 8, v);
  };

  float a = 0.f;
  bool odd = false;
  auto largest = [&](float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (!isfinite(v[e])) {
        v[e] = 0.f;
        odd = true;
      }
      a = fmaxf(a, fabsf(v[e]));
    }
  };
  float held[kHeld][8];
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (tid + j * kThreads < chunks) chunk(tid + j * kThreads, held[j]);
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (tid + j * kThreads < chunks) largest(held[j]);
  for (int c = tid + kHeld * kThreads; c < chunks; c += kThreads) {
    float v[8];
    chunk(c, v);
    largest(v);
  }
  if (__syncthreads_or(odd) && tid == 0) atomicOr(p.status, PP_CACHE_NOT_FINITE);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) a = fmaxf(a, __shfl_xor_sync(~0u, a, d));
  if (tid % 32 == 0) most[tid / 32] = a;
  __syncthreads();  // every thread has read the scale, too
#pragma unroll
  for (int j = 0; j < kThreads / 32; ++j) a = fmaxf(a, most[j]);

  const float now = fmaxf(had, a >= kTiny ? __fmul_rn(a, 1.f / 127.f) : 0.f);
  const float r = now > 0.f ? __fdiv_rn(1.f, now) : 0.f;
  if (at && now > had) {
    const float f = __fdiv_rn(had, now);
    for (int c = tid; c < at * p.row.d; c += kThreads) {
      uint2 w = *reinterpret_cast<const uint2*>(codes + c * 8);
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)((e < 4 ? w.x : w.y) >> e % 4 * 8);
      *reinterpret_cast<uint2*>(codes + c * 8) = codes8(v, f);
    }
  }
  uint2* to = reinterpret_cast<uint2*>(codes + at * p.D);  // rows follow each other
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (tid + j * kThreads < chunks) to[tid + j * kThreads] = codes8(held[j], r);
  for (int c = tid + kHeld * kThreads; c < chunks; c += kThreads) {
    float v[8];
    chunk(c, v);
    largest(v);  // what is not finite is 0
    to[c] = codes8(v, r);
  }
  if (tid == 0 && (!at || now != had)) p.scales[pool][cell] = now;
}

// ---- reading back: a block has `tokens` tokens, of which a lane each looks up the place, then every thread takes 8 codes of
// a head at a time.  Bound by its writes.
constexpr int kReadThreads = 256;
constexpr int kMostTokens = 32;

struct ReadParams {
  const int8_t* codes[2];
  const float* scales[2];
  void* out[2];
  const int *starts, *table, *lens;
  int* status;
  int T, B, H, D, page, log_page, pages, width, tokens;
  FastDiv row, heads;  // by the chunks of a row, by H
};

template <class T, bool WIDE>
__global__ void __launch_bounds__(kReadThreads) read_kernel(const __grid_constant__ ReadParams p) {
  __shared__ int place[kMostTokens];  // page id * page + offset; -1: no such key
  after_previous();
  const int t0 = blockIdx.x * p.tokens, nt = min(p.tokens, p.T - t0), tid = threadIdx.x;
  if (tid < nt) {
    const int most = p.width << p.log_page;
    const Seen s = seen_keys(t0 + tid, p.T, p.B, p.starts, p.lens, most, true, p.status);
    int at = -1;
    if (s.keys > 0) {  // the token's own key is the last that it sees
      const int id = p.table[(int64_t)s.b * p.width + (s.keys - 1 >> p.log_page)];
      if (id < 0 || id >= p.pages) atomicOr(p.status, PP_CACHE_BAD_PAGE);
      else at = (id << p.log_page) + (s.keys - 1 & p.page - 1);
    }
    place[tid] = at;
  }
  if (p.starts && blockIdx.x == 0) check_ranges(p.starts, p.T, p.B, tid, kReadThreads, p.status);
  __syncthreads();
  const int per = p.row.d * p.H, all = nt * per;  // chunks of a token, of the block
  constexpr int U = 4;
#pragma unroll 1
  for (int pool = 0; pool < 2; ++pool) {
    T* out = static_cast<T*>(p.out[pool]);
    if (!out) continue;
    out += (int64_t)t0 * per * 8;
    for (int c0 = tid; c0 < all; c0 += U * kReadThreads) {
      uint2 w[U];
      float s[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = min(c0 + u * kReadThreads, all - 1);
        const int row = p.row.div(c), t = p.heads.div(row), h = row - t * p.H, at = place[t];
        const int id = max(at, 0) >> p.log_page;
        const int64_t cell = (int64_t)id * p.H + h;
        w[u] = *reinterpret_cast<const uint2*>(p.codes[pool] + (cell * p.page + (max(at, 0) & p.page - 1)) * p.D + (c - row * p.row.d) * 8);
        s[u] = p.scales[pool][cell];
        if (at < 0) {
          w[u] = make_uint2(0, 0);
          s[u] = 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u * kReadThreads;
        if (c >= all) break;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __fmul_rn((float)(int8_t)((e < 4 ? w[u].x : w[u].y) >> e % 4 * 8), s[u]);
        constexpr int V = 16 / sizeof(T);
        T* to = out + (int64_t)c * 8;
        if constexpr (WIDE) {
#pragma unroll
          for (int i = 0; i < 8; i += V) {
            Vec<T, V> y;
#pragma unroll
            for (int e = 0; e < V; e += 2) put2(y, e / 2, v[i + e], v[i + e + 1]);
            *reinterpret_cast<Vec<T, V>*>(to + i) = y;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) to[e] = from_f32<T>(v[e]);
        }
      }
    }
  }
}

// What both calls ask of their sequences.
pp_status check_sequences(const pp_cache* cache, int T, int B, const int32_t* starts, const int32_t* table, int width,
                          const int32_t* lens) {
  if (!cache || T < 0 || B < 0 || width < 1) return PP_ERR_INVALID_ARG;
  if (T > 0 && (!table || !lens || B < 1 || (!starts && T != B))) return PP_ERR_INVALID_ARG;
  if (!cache->scales8[0] || (int64_t)width * cache->page > INT32_MAX - 256) return PP_ERR_UNSUPPORTED;
  return PP_OK;
}

// f(pointer to an element) of the cache's type, with rows on 16-byte boundaries or not
template <class F>
cudaError_t by_type(int dtype, bool wide, F f) {
  auto with = [&](auto* t) { return wide ? f(t, std::true_type{}) : f(t, std::false_type{}); };
  return dtype == PP_F32   ? with((float*)nullptr)
         : dtype == PP_F16 ? with((__half*)nullptr)
                           : with((__nv_bfloat16*)nullptr);
}

}  // namespace

extern "C" {

pp_status pp_cache_append(const pp_cache* cache, int T, const void* k, int64_t k_ts, int64_t k_hs, const void* v, int64_t v_ts,
                          int64_t v_hs, int B, const int32_t* starts, const int32_t* table, int width, const int32_t* lens,
                          void* stream) {
  const pp_status st = check_sequences(cache, T, B, starts, table, width, lens);
  if (st != PP_OK) return st;
  const pp_cache& c = *cache;
  const uintptr_t al = (uintptr_t)dtype_size(c.dtype) - 1, at = reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v);
  if (k_ts < 0 || k_hs < 0 || v_ts < 0 || v_hs < 0 || (T > 0 && (!k || !v || (at & al)))) return PP_ERR_INVALID_ARG;
  if (T == 0) return PP_OK;
  AppendParams p = {{k, v},     {k_ts, v_ts}, {k_hs, v_hs}, {static_cast<int8_t*>(c.k), static_cast<int8_t*>(c.v)},
                    {c.scales8[0], c.scales8[1]}, starts, table, lens, c.status, T, B, c.H, c.D, c.page, log2_of(c.page), c.pages,
                    width, FastDiv(c.D / 8)};
  const int64_t blocks = starts ? (int64_t)T / c.page + 2 * (int64_t)B : T;
  if (blocks > INT32_MAX) return PP_ERR_UNSUPPORTED;
  const int64_t strides = (k_ts | k_hs | v_ts | v_hs) * dtype_size(c.dtype);
  const cudaError_t e = by_type(c.dtype, ((at | (uintptr_t)strides) & 15) == 0, [&](auto* t, auto wide) {
    using E = std::remove_pointer_t<decltype(t)>;
    return launch_after(append_kernel<E, decltype(wide)::value>, dim3((unsigned)blocks, c.H, 2), kThreads, 0, (cudaStream_t)stream, 1, p);
  });
  return e == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

pp_status pp_cache_read(const pp_cache* cache, int T, int B, const int32_t* starts, const int32_t* table, int width,
                        const int32_t* lens, void* k_out, void* v_out, void* stream) {
  const pp_status st = check_sequences(cache, T, B, starts, table, width, lens);
  if (st != PP_OK) return st;
  const pp_cache& c = *cache;
  const uintptr_t al = (uintptr_t)dtype_size(c.dtype) - 1, at = reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out);
  if (at & al) return PP_ERR_INVALID_ARG;
  if (T == 0 || (!k_out && !v_out)) return PP_OK;
  const int sms = device_sms();
  if (sms <= 0) return PP_ERR_CUDA;
  // few tokens a block each, so that all SMs have some; a block's chunks are counted in 32 bits (65535 heads of 256: 2^26)
  const int tokens = std::min(kMostTokens, std::max(1, T / (8 * sms)));
  ReadParams p = {{static_cast<const int8_t*>(c.k), static_cast<const int8_t*>(c.v)}, {c.scales8[0], c.scales8[1]}, {k_out, v_out},
                  starts, table, lens, c.status, T, B, c.H, c.D, c.page, log2_of(c.page), c.pages, width, tokens, FastDiv(c.D / 8),
                  FastDiv(c.H)};
  const cudaError_t e = by_type(c.dtype, (at & 15) == 0, [&](auto* t, auto wide) {
    using E = std::remove_pointer_t<decltype(t)>;
    return launch_after(read_kernel<E, decltype(wide)::value>, dim3((unsigned)((T + tokens - 1) / tokens)), kReadThreads, 0,
                        (cudaStream_t)stream, 1, p);
  });
  return e == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

}  // extern "C"
