// Internal declarations of the decoder operators: element types, the rotation
// plan and the paged cache.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "ppconv.h"

struct pp_rope {
  int D = 0, pairs = 0, axes = 0, interleaved = 0;
  // per pair: the turn per position as a 64-bit fraction (2^64 = one turn), and its axis
  const uint64_t* turn = nullptr;
  const uint8_t* axis = nullptr;
  void* dmem = nullptr;
};

struct pp_cache {
  int dtype = 0, pages = 0, page = 0, H = 0, D = 0;
  void* k = nullptr;
  void* v = nullptr;
  int8_t* codes = nullptr;
  float* scales = nullptr;
  void* dmem = nullptr;   // status word, counters and partial results
  int* status = nullptr;
  int* counters = nullptr;   // zero between calls
  float* partial = nullptr;
  float* tiles = nullptr;
  CUtensorMap mk, mv;        // the pools as rows of D values; boxes of one 128-byte column of a page's rows
};

namespace ppc {

// The row kernel's keys per tile (attn.cu): 64 rows of 16-bit values, 32 of fp32.
inline int tile_keys(int dtype) { return dtype == PP_F32 ? 32 : 64; }
// Device bytes that attention needs beside the status word: counters, partial results, shares of tiles.
struct AttnSpace {
  size_t counters, partial, tiles;
};
AttnSpace attn_space(int dtype, int D, int sms);
cudaError_t attn_prepare();
cudaError_t select_prepare();

// Launches that may begin while the stream's kernel before them ends (programmatic dependent launch): their kernels call
// after_previous() before they touch any memory, and let the next one begin at once.  A step's calls are small and follow
// each other, so a launch's latency hides behind the kernel before it.
template <class... P, class... A>
cudaError_t launch_after(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, int cluster, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim = {(unsigned)cluster, 1, 1};
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
__device__ __forceinline__ void after_previous() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

inline int dtype_size(int dtype) { return dtype == PP_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == PP_F32 || dtype == PP_F16 || dtype == PP_BF16; }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Division of numbers below 2^31 by a number known on the host: n / d = (n m / 2^32 + n) / 2^shift with the round-up
// multiplier m of Granlund and Montgomery.  A general division is tens of dependent instructions.
struct FastDiv {
  uint32_t m;
  int shift, d;
  FastDiv(int by = 1) : m(0), shift(0), d(by) {
    while ((int64_t(1) << shift) < by) ++shift;
    m = (uint32_t)((((uint64_t(1) << shift) - (uint64_t)by) << 32) / (uint64_t)by + 1);
  }
  __device__ __forceinline__ int div(int n) const { return (int)((__umulhi((uint32_t)n, m) + (uint32_t)n) >> shift); }
  __device__ __forceinline__ int mod(int n) const { return n - div(n) * d; }
};
inline int log2_of(int n) {
  int s = 0;
  while ((1 << s) < n) ++s;
  return s;
}

constexpr float kTiny = 0x1p-100f;  // a page's or query's largest value below which it counts as 0: 127 / a stays finite

// V consecutive elements moved as one (up to 16 bytes).
template <class T, int V>
struct alignas(sizeof(T) * V) Vec {
  T v[V];
};

// Two neighbours of a vector at once, as the word that holds them: one conversion instruction where the type has one for
// two (bf16 to fp32 is a shift or a mask).
template <class T, int V>
__device__ __forceinline__ float2 get2(const Vec<T, V>& a, int i) {
  if constexpr (sizeof(T) == 4) {
    return make_float2(a.v[2 * i], a.v[2 * i + 1]);
  } else {
    const uint32_t w = reinterpret_cast<const uint32_t*>(&a)[i];
    if constexpr (std::is_same<T, __half>::value) return __half22float2(*reinterpret_cast<const __half2*>(&w));
    else return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  }
}
template <class T>
__device__ __forceinline__ uint32_t pack(float x, float y) {
  if constexpr (std::is_same<T, __half>::value) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}
template <class T, int V>
__device__ __forceinline__ void put2(Vec<T, V>& a, int i, float x, float y) {
  if constexpr (sizeof(T) == 4) {
    a.v[2 * i] = x;
    a.v[2 * i + 1] = y;
  } else {
    reinterpret_cast<uint32_t*>(&a)[i] = pack<T>(x, y);
  }
}

// A token of a call on the cache: its sequence and how many of that sequence's keys it sees.
struct Seen {
  int b, keys;
};
// starts null: token t is sequence t.  Lengths and ranges that do not fit are cut to what does, and recorded.
__device__ __forceinline__ Seen seen_keys(int t, int T, int B, const int* __restrict__ starts,
                                          const int* __restrict__ lens, int most, bool causal, int* status) {
  int b = t, n = 1, i = 0;
  if (starts) {
    int lo = 0, hi = B;  // the last b with starts[b] <= t
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (starts[mid] <= t) lo = mid; else hi = mid;
    }
    b = lo;
    const int s0 = starts[b], s1 = starts[b + 1];
    n = s1 - s0;
    i = t - s0;
    if (s0 < 0 || s1 > T || i < 0 || i >= n) {  // no sequence has this token, or one has others that there are not
      atomicOr(status, PP_CACHE_BAD_LENGTH);
      return {b, 0};
    }
  }
  int len = lens[b];
  if (len < 0 || len > most) {
    atomicOr(status, PP_CACHE_BAD_LENGTH);
    len = len < 0 ? 0 : most;
  }
  const int keys = causal ? len - n + i + 1 : len;
  return {b, keys < 0 ? 0 : keys};
}

// Records token ranges that do not fit, of which a call by tokens meets only those that its tokens fall in: by the threads
// of one block.
__device__ __forceinline__ void check_ranges(const int* __restrict__ starts, int T, int B, int tid, int threads, int* status) {
  bool bad = tid == 0 && (starts[0] != 0 || starts[B] != T);
  for (int b = tid; b < B; b += threads) bad = bad || starts[b] > starts[b + 1];
  if (bad) atomicOr(status, PP_CACHE_BAD_LENGTH);
}

}  // namespace ppc
