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
  int64_t items;  // (span of a page's new tokens, pool, head)
  FastDiv row;    // by the 16-byte chunks of a row
};

constexpr int kThreads = 128;
constexpr int kHeld = 8;  // chunks of 16 bytes that a thread keeps between the two passes

// A chunk of 16 bytes of a token's values, and 0 for those that are not finite.
template <class T, bool WIDE>
__device__ __forceinline__ uint4 load_chunk(const T* x) {
  constexpr int V = 16 / sizeof(T);
  if constexpr (WIDE) {
    return *reinterpret_cast<const uint4*>(x);
  } else {
    Vec<T, V> v;
#pragma unroll
    for (int i = 0; i < V; ++i) v.v[i] = x[i];
    return *reinterpret_cast<const uint4*>(&v);
  }
}
// The bits of positive numbers are ordered as they are, so a chunk's largest |x| is a maximum of whole numbers, two 16-bit ones
// at a time; what is not finite comes out on top.
template <class T>
constexpr uint32_t kNotFinite = sizeof(T) == 4 ? 0x7F800000u : std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
template <class T>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t w) {
  if constexpr (sizeof(T) == 4) return max(a, w & 0x7FFFFFFFu);
  else return __vmaxu2(a, w & 0x7FFF7FFFu);
}
template <class T>
__device__ __forceinline__ uint32_t largest_bits(uint32_t a) {  // of both halves
  if constexpr (sizeof(T) == 4) return a;
  else return max(a & 0xFFFFu, a >> 16);
}
template <class T>
__device__ __forceinline__ uint4 finite_only(uint4 w) {
  auto f = [](uint32_t x) {
    if constexpr (sizeof(T) == 4) return (x & 0x7FFFFFFFu) >= kNotFinite<T> ? 0u : x;
    else return ((x & 0x7FFFu) >= kNotFinite<T> ? 0u : x & 0xFFFFu) | ((x >> 16 & 0x7FFFu) >= kNotFinite<T> ? 0u : x & 0xFFFF0000u);
  };
  return make_uint4(f(w.x), f(w.y), f(w.z), f(w.w));
}
template <class T>
__device__ __forceinline__ float of_bits(uint32_t b) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(b);
  else if constexpr (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((unsigned short)b));
  else return __uint_as_float(b << 16);
}

// rint(v r) of values that stay within 127.5, as the low byte: added to 1.5 x 2^23, a product is rounded to a whole number (half to
// even) in the lowest bits.  In two steps: the product is rounded first.
__device__ __forceinline__ uint32_t code(float v, float r) {
  return __float_as_uint(__fadd_rn(__fmul_rn(v, r), 12582912.f));
}
__device__ __forceinline__ uint32_t four(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
template <class T>
__device__ __forceinline__ void store_codes(int8_t* to, uint4 w, float r) {
  Vec<T, 16 / sizeof(T)> v;
  memcpy(&v, &w, 16);
  uint32_t c[16 / sizeof(T)];
#pragma unroll
  for (int i = 0; i < 16 / (int)sizeof(T); i += 2) {
    const float2 f = get2(v, i / 2);
    c[i] = code(f.x, r);
    c[i + 1] = code(f.y, r);
  }
  if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(to) = four(c[0], c[1], c[2], c[3]);
  else *reinterpret_cast<uint2*>(to) = make_uint2(four(c[0], c[1], c[2], c[3]), four(c[4], c[5], c[6], c[7]));
}

// A team of threads (a warp, or the block of four) has the new tokens of one page, head and pool: their largest value, the page's
// scale, its older codes where the scale has grown, then the new codes.  What the threads hold stays in registers in between
// (64 tokens of 128 in 16 bits for a block; the rest is read again, out of L2).  Bound by reading the tokens once: 16384 of 8
// heads of 128 (f16) 19.5 us, 5.2 TB/s.
template <class T, bool WIDE, int TEAM>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int V = 16 / sizeof(T);
  __shared__ uint32_t most[kThreads / 32];
  after_previous();
  const int tid = threadIdx.x % TEAM;
  const int64_t item = (int64_t)blockIdx.x * (kThreads / TEAM) + threadIdx.x / TEAM;
  if (p.starts && blockIdx.x == 0) check_ranges(p.starts, p.T, p.B, threadIdx.x, kThreads, p.status);
  if (item >= p.items) return;
  const int at_span = (int)(item / (2 * p.H)), rest = (int)(item - (int64_t)at_span * 2 * p.H), pool = rest >= p.H, h = rest - pool * p.H;
  int b = at_span, s0 = b, n = 1, i = 0;
  if (p.starts) {
    // A sequence whose tokens begin at s has the spans from s / page + 2 b on: no fewer than the pages that they fall in
    auto base = [&](int b) { return (min(max(p.starts[b], 0), p.T) >> p.log_page) + 2 * b; };
    int lo = 0, hi = p.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (base(mid) <= at_span) lo = mid; else hi = mid;
    }
    b = lo;
    s0 = p.starts[b];
    n = p.starts[b + 1] - s0;
    i = at_span - base(b);
    if (s0 < 0 || n < 0 || s0 > p.T - n || i < 0) return;
  }
  const int len = p.lens[b];
  if (len < 0 || len > p.width << p.log_page) {
    if (tid == 0 && i == 0) atomicOr(p.status, PP_CACHE_BAD_LENGTH);
    return;
  }
  // positions of the new tokens: from .. len - 1, of which the team has those of one page
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
  const T* x = static_cast<const T*>(p.x[pool]) + (s0 + (lo - from)) * ts + h * p.hs[pool];
  const int row = p.row.d, chunks = (hi - lo) * row;
  auto chunk = [&](int c) {
    const int r = p.row.div(c);
    return load_chunk<T, WIDE>(x + r * ts + (c - r * row) * V);
  };

  uint32_t a = 0;
  auto largest = [&](uint4 w) { a = larger<T>(larger<T>(larger<T>(larger<T>(a, w.x), w.y), w.z), w.w); };
  uint4 held[kHeld];
#pragma unroll
  for (int j = 0; j < kHeld; ++j) held[j] = tid + j * TEAM < chunks ? chunk(tid + j * TEAM) : make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int j = 0; j < kHeld; ++j) largest(held[j]);
  for (int c = tid + kHeld * TEAM; c < chunks; c += TEAM) largest(chunk(c));
  auto over_team = [&](uint32_t a) {
    a = __reduce_max_sync(~0u, largest_bits<T>(a));
    if constexpr (TEAM > 32) {
      __syncthreads();  // (the last one's have been read)
      if (tid % 32 == 0) most[tid / 32] = a;
      __syncthreads();  // every thread has read the scale, too
#pragma unroll
      for (int j = 0; j < TEAM / 32; ++j) a = max(a, most[j]);
    }
    return a;
  };
  a = over_team(a);
  const bool odd = a >= kNotFinite<T>;
  if (odd) {  // once more without what is not finite
    if (tid == 0) atomicOr(p.status, PP_CACHE_NOT_FINITE);
    a = 0;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      held[j] = finite_only<T>(held[j]);
      largest(held[j]);
    }
    for (int c = tid + kHeld * TEAM; c < chunks; c += TEAM) largest(finite_only<T>(chunk(c)));
    a = over_team(a);
  }

  const float big = of_bits<T>(a), now = fmaxf(had, big >= kTiny ? __fmul_rn(big, 1.f / 127.f) : 0.f);
  const float r = now > 0.f ? __fdiv_rn(1.f, now) : 0.f;
  if (at && now > had) {
    const float f = __fdiv_rn(had, now);
    for (int c = tid; c < at * (p.D / 8); c += TEAM) {
      const uint2 w = *reinterpret_cast<const uint2*>(codes + c * 8);
      uint32_t v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = code((float)(int8_t)((e < 4 ? w.x : w.y) >> e % 4 * 8), f);
      *reinterpret_cast<uint2*>(codes + c * 8) = make_uint2(four(v[0], v[1], v[2], v[3]), four(v[4], v[5], v[6], v[7]));
    }
  }
  int8_t* to = codes + at * p.D;  // rows follow each other
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (tid + j * TEAM < chunks) store_codes<T>(to + (tid + j * TEAM) * V, held[j], r);
  for (int c = tid + kHeld * TEAM; c < chunks; c += TEAM) store_codes<T>(to + c * V, odd ? finite_only<T>(chunk(c)) : chunk(c), r);
  if (TEAM == 32) __syncwarp();  // every thread has read the scale
  if (tid == 0 && (!at || now != had)) p.scales[pool][cell] = now;
}

// ---- reading back: a block has `tokens` tokens, of which a lane each looks up the place, then every thread takes 16 codes of
// a head at a time.  Bound by its writes, which are 32 bytes of a thread at once: 8 sequences of 8192 tokens, 8 heads of 128
// (bf16), 68 us, 5.9 TB/s; written 16 bytes at a time fp32 took 1.3 times as long.
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
__global__ void __launch_bounds__(kReadThreads, 6) read_kernel(const __grid_constant__ ReadParams p) {
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
    out += (int64_t)t0 * per * 16;
    for (int c0 = tid; c0 < all; c0 += U * kReadThreads) {
      uint4 w[U];
      float s[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = min(c0 + u * kReadThreads, all - 1);
        const int row = p.row.div(c), t = p.heads.div(row), h = row - t * p.H, at = place[t];
        const int id = max(at, 0) >> p.log_page;
        const int64_t cell = (int64_t)id * p.H + h;
        w[u] = *reinterpret_cast<const uint4*>(p.codes[pool] + (cell * p.page + (max(at, 0) & p.page - 1)) * p.D + (c - row * p.row.d) * 16);
        s[u] = p.scales[pool][cell];
        if (at < 0) {
          w[u] = make_uint4(0, 0, 0, 0);
          s[u] = 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u * kReadThreads;
        if (c >= all) break;
        const uint32_t word[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
        float v[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = __fmul_rn((float)(int8_t)(word[e / 4] >> e % 4 * 8), s[u]);
        T* to = out + (int64_t)c * 16;
        if constexpr (WIDE) {
          uint32_t y[4 * sizeof(T)];
#pragma unroll
          for (int i = 0; i < 4 * (int)sizeof(T); ++i) {
            if constexpr (sizeof(T) == 4) y[i] = __float_as_uint(v[i]);
            else y[i] = pack<T>(v[2 * i], v[2 * i + 1]);
          }
#pragma unroll
          for (int i = 0; i < 4 * (int)sizeof(T); i += 8)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + i * 4 / sizeof(T)), "r"(y[i]), "r"(y[i + 1]),
                         "r"(y[i + 2]), "r"(y[i + 3]), "r"(y[i + 4]), "r"(y[i + 5]), "r"(y[i + 6]), "r"(y[i + 7])
                         : "memory");
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) to[e] = from_f32<T>(v[e]);
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

// f(pointer to an element) of the cache's type, with rows on wide boundaries or not
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
                    width, 0, FastDiv(c.D * dtype_size(c.dtype) / 16)};
  const int64_t spans = starts ? (int64_t)T / c.page + 2 * (int64_t)B : T;
  p.items = spans * 2 * c.H;
  // A warp where it can hold a page's new tokens (16 of 128 in 16 bits), else a block: 16384 tokens into pages of 16, 8 heads of 128
  // (f16), took 70 us by blocks and take 21 by warps
  const bool small = (int64_t)(starts ? std::min(c.page, T) : 1) * p.row.d <= 32 * kHeld;
  const int64_t blocks = small ? (p.items + kThreads / 32 - 1) / (kThreads / 32) : p.items;
  if (spans > INT32_MAX || blocks > INT32_MAX) return PP_ERR_UNSUPPORTED;
  const int64_t strides = (k_ts | k_hs | v_ts | v_hs) * dtype_size(c.dtype);
  const cudaError_t e = by_type(c.dtype, ((at | (uintptr_t)strides) & 15) == 0, [&](auto* t, auto wide) {
    using E = std::remove_pointer_t<decltype(t)>;
    constexpr bool W = decltype(wide)::value;
    return launch_after(small ? append_kernel<E, W, 32> : append_kernel<E, W, kThreads>, dim3((unsigned)blocks), kThreads, 0,
                        (cudaStream_t)stream, 1, p);
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
                  starts, table, lens, c.status, T, B, c.H, c.D, c.page, log2_of(c.page), c.pages, width, tokens, FastDiv(c.D / 16),
                  FastDiv(c.H)};
  const cudaError_t e = by_type(c.dtype, (at & 31) == 0, [&](auto* t, auto wide) {
    using E = std::remove_pointer_t<decltype(t)>;
    return launch_after(read_kernel<E, decltype(wide)::value>, dim3((unsigned)((T - 1) / tokens + 1)), kReadThreads, 0,
                        (cudaStream_t)stream, 1, p);
  });
  return e == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

}  // extern "C"
