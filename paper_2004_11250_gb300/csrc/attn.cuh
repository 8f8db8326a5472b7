// What the two attention kernels share: a call's parameters, bounded waits, box copies.
#pragma once

#include <cmath>
#include <type_traits>

#include "cache.h"
#include "tc_ptx.cuh"

namespace ppc_attn {

using namespace ppc;
using namespace ppc_ptx;

constexpr int kPieces = 8;  // boxes down a tile at most (pages of 8)

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
  int T, B, H, D, page, log_page, pages, width, keep, causal;
  FastDiv G, by_head, by_keep;  // by the group's heads, by H, by keep
  // tiles: shares that their blocks are split into, and the rows' sums and (maximum, total) of each share
  int splits;
  float* split_sums;
  float2* split_stats;
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

// The weights 2^(s - m) of a row may be rounded to the inputs' type before their product with V.  f16 has its 11 bits down
// to 2^-14 and nothing below 2^-25, and keys far below a row's largest count by their number: m is taken that many powers
// of two below the largest, so that the weights fill f16's range from above (its largest number is just below 2^16).
// Their sum is of the same weights, so m need not be the largest for it.
template <class T, int UP>
constexpr float kLift = std::is_same<T, __half>::value ? (float)UP : 0.f;
// x - n, no less than that: beyond 2^24 fp32 holds no difference of n, and a weight must not pass its bound
__device__ __forceinline__ float lower(float x, float n) { return __fadd_ru(x, -n); }
// log of a row's sum `l` of weights taken from m
template <class T, int UP>
__device__ __forceinline__ float log_sum(float m, float l) {
  constexpr float n = kLift<T, UP>;
  return (m + n) * 0.693147181f + logf(l * (n == 0.f ? 1.f : 1.f / (float)(1 << UP)));
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Whether some of 16 bytes of values are not finite.
template <class T>
__device__ __forceinline__ bool not_finite(uint4 v) {
  if constexpr (sizeof(T) == 4) {
    const float* f = reinterpret_cast<const float*>(&v);
    return !(isfinite(f[0]) && isfinite(f[1]) && isfinite(f[2]) && isfinite(f[3]));
  } else {  // an exponent of ones carries into the sign's place
    constexpr uint32_t e = std::is_same<T, __half>::value ? 0x7C007C00u : 0x7F807F80u, one = e & ~(e << 1) & 0x7FFF7FFFu;
    return (((v.x & e) + one) | ((v.y & e) + one) | ((v.z & e) + one) | ((v.w & e) + one)) & 0x80008000u;
  }
}

// Values that are not finite, at a key that some rows of a unit or tile see and others do not, would reach the others as 0 x
// NaN.  Such a key's values are zeroed in shared memory, and its weight times them is added to each row that sees it when the
// row is done: those of the keys first + i with bit i set to sums of a row of queries q and its m, by one warp.
template <class T, int DP>
__device__ __noinline__ void add_keys(const AttnParams& p, const T* q, const int* table, int h, int first, uint64_t keys, float sl,
                                      float m, float* sums) {
  const int lane = threadIdx.x % 32;
  for (; keys; keys &= keys - 1) {
    const int key = first + __ffsll(keys) - 1;
    const int64_t at = (((int64_t)table[key >> p.log_page] * p.H + h) * p.page + (key & (p.page - 1))) * p.D;
    float x = 0.f;
    for (int d = lane; d < p.D; d += 32) x += to_f32(q[d]) * to_f32(static_cast<const T*>(p.k)[at + d]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    const float w = ex2(__fmul_rn(x, sl) - (m == -INFINITY ? 0.f : m));
    for (int d = lane; d < p.D; d += 32) sums[d] += w * to_f32(static_cast<const T*>(p.v)[at + d]);
  }
}

// attn_tile.cu: tiles of 128 query rows on the tensor cores, for 16-bit types and heads of up to 128.
bool tile_applicable(const AttnParams& p, int dtype, int sms);
cudaError_t tile_prepare();
size_t tile_space(int dtype, int D, int sms);  // device bytes of the shares' sums
cudaError_t tile_launch(AttnParams p, const pp_cache& c, int sms, cudaStream_t stream);

}  // namespace ppc_attn
