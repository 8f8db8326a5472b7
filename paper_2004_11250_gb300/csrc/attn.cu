// Attention of query tokens over the paged cache (pp_attn_forward).
//
// One block per (token, head): each warp takes every fourth key, a lane up to 8
// values of the head, with a running maximum and sum; the warps join at the end.
#include <cmath>

#include "cache.h"
#include "internal.h"

namespace {

using namespace ppc;

constexpr int kWarps = 4;

struct AttnParams {
  const void* q;
  int64_t q_ts, q_hs;
  const void *k, *v;
  const int *starts, *table, *lens, *sel;
  void* out;
  float* lse;
  int* status;
  float scale;
  int T, B, H, G, D, page, pages, width, keep, causal;
};

template <class T>
__global__ void __launch_bounds__(kWarps * 32) attn_kernel(const AttnParams p) {
  __shared__ float acc[kWarps][256], ms[kWarps], ls[kWarps];
  const int t = blockIdx.x, hq = blockIdx.y, h = hq / p.G, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const Seen s = seen_keys(t, p.T, p.B, p.starts, p.lens, p.width * p.page, p.causal, p.status);
  const int P = (s.keys + p.page - 1) / p.page;
  const T* q = static_cast<const T*>(p.q) + t * p.q_ts + (int64_t)hq * p.q_hs;
  float fq[8], o[8], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    fq[i] = lane + 32 * i < p.D ? to_f32(q[lane + 32 * i]) : 0.f;
    o[i] = 0.f;
  }
  const int n = p.sel ? p.keep : P;
  for (int e = 0; e < n; ++e) {
    int w = e;
    if (p.sel) {
      w = p.sel[((int64_t)t * p.H + h) * p.keep + e];
      if (w < 0) continue;
      if (w >= p.width) {
        atomicOr(p.status, PP_CACHE_BAD_PAGE);
        continue;
      }
      if (w >= P) continue;
    }
    const int id = p.table[(int64_t)s.b * p.width + w];
    if (id < 0 || id >= p.pages) {
      atomicOr(p.status, PP_CACHE_BAD_PAGE);
      continue;
    }
    const int64_t base = ((int64_t)id * p.H + h) * p.page;
    const int have = min(p.page, s.keys - w * p.page);
    for (int i = warp; i < have; i += kWarps) {
      const T* k = static_cast<const T*>(p.k) + (base + i) * p.D;
      const T* v = static_cast<const T*>(p.v) + (base + i) * p.D;
      float x = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (lane + 32 * j < p.D) x += fq[j] * to_f32(k[lane + 32 * j]);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
      x *= p.scale;
      const float mn = fmaxf(m, x), c = m == mn ? 1.f : __expf(m - mn), w1 = __expf(x - mn);
      m = mn;
      l = l * c + w1;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (lane + 32 * j < p.D) o[j] = o[j] * c + w1 * to_f32(v[lane + 32 * j]);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[warp][lane + 32 * j] = o[j];
  if (lane == 0) {
    ms[warp] = m;
    ls[warp] = l;
  }
  __syncthreads();
  float mx = -INFINITY, sum = 0.f;
  for (int i = 0; i < kWarps; ++i) mx = fmaxf(mx, ms[i]);
  float f[kWarps];
  for (int i = 0; i < kWarps; ++i) {
    f[i] = ls[i] > 0.f ? __expf(ms[i] - mx) : 0.f;
    sum += ls[i] * f[i];
  }
  T* out = static_cast<T*>(p.out) + ((int64_t)t * p.H * p.G + hq) * p.D;
  for (int d = threadIdx.x; d < p.D; d += kWarps * 32) {
    float y = 0.f;
    for (int i = 0; i < kWarps; ++i) y += acc[i][d] * f[i];
    out[d] = from_f32<T>(sum > 0.f ? y / sum : 0.f);
  }
  if (p.lse && threadIdx.x == 0) p.lse[(int64_t)t * p.H * p.G + hq] = sum > 0.f ? mx + logf(sum) : -INFINITY;
}

}  // namespace

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
  const pp_cache& c = *cache;
  AttnParams p = {q, q_ts, q_hs, c.k, c.v, starts, table, lens, sel, out, lse, c.status, scale, T, B, c.H, Hq / c.H, c.D,
                  c.page, c.pages, width, keep, flags & PP_ATTN_CAUSAL};
  const dim3 grid(T, Hq);
  const cudaStream_t s = (cudaStream_t)stream;
  if (c.dtype == PP_F32)
    attn_kernel<float><<<grid, kWarps * 32, 0, s>>>(p);
  else if (c.dtype == PP_F16)
    attn_kernel<__half><<<grid, kWarps * 32, 0, s>>>(p);
  else
    attn_kernel<__nv_bfloat16><<<grid, kWarps * 32, 0, s>>>(p);
  return cudaGetLastError() == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}
