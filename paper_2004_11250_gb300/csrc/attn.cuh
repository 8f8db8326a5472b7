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
// attn_tile.cu: tiles of 128 query rows on the tensor cores, for 16-bit types and heads of up to 128.
bool tile_applicable(const AttnParams& p, int dtype, int sms);
cudaError_t tile_prepare();
size_t tile_space(int dtype, int D, int sms);  // device bytes of the shares' sums
cudaError_t tile_launch(AttnParams p, const pp_cache& c, int sms, cudaStream_t stream);

}  // namespace ppc_attn
