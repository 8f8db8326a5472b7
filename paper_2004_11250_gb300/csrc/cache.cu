// The paged cache: its handle, page summaries and page selection
// (pp_cache_create, pp_cache_summarize, pp_cache_select).
#include <algorithm>
#include <cmath>
#include <new>

#include "cache.h"
#include "internal.h"

namespace {

using namespace ppc;

constexpr float kTiny = 0x1p-100f;  // largest key value below which a page counts as 0: 127 / a stays finite

// One block per (page, head), a thread per value of the head.
template <class T>
__global__ void summarize_kernel(const T* __restrict__ k, const int* __restrict__ ids, int pages, int page, int H, int D,
                                 int8_t* __restrict__ codes, float* __restrict__ scales, int* status) {
  const int id = ids[blockIdx.x], h = blockIdx.y, d = threadIdx.x;
  if (id < 0 || id >= pages) {
    if (d == 0) atomicOr(status, PP_CACHE_BAD_PAGE);
    return;
  }
  __shared__ float big;
  __shared__ int odd;
  if (d == 0) {
    big = 0.f;
    odd = 0;
  }
  __syncthreads();
  const int64_t cell = (int64_t)id * H + h;
  const T* x = k + cell * page * D;
  float mx = to_f32(x[d]), mn = mx;
  bool bad = false;
  for (int i = 0; i < page; ++i) {
    const float v = to_f32(x[(int64_t)i * D + d]);
    bad = bad || !isfinite(v);
    mx = fmaxf(mx, v);
    mn = fminf(mn, v);
  }
  if (bad) atomicOr(&odd, 1);
  atomicMax(reinterpret_cast<int*>(&big), __float_as_int(fmaxf(fabsf(mx), fabsf(mn))));  // not negative: ordered as integers
  __syncthreads();
  const float a = big;
  const bool zero = odd || !(a >= kTiny);
  const float r = zero ? 0.f : __fdiv_rn(127.f, a);
  int8_t* c = codes + cell * 2 * D;
  c[d] = zero ? 0 : (int8_t)fminf(ceilf(__fmul_rn(mx, r)), 127.f);
  c[D + d] = zero ? 0 : (int8_t)fmaxf(floorf(__fmul_rn(mn, r)), -127.f);
  if (d == 0) scales[cell] = odd ? nanf("") : __fmul_rn(a, 1.f / 127.f);
}

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

// One block per (token, head): scores in shared memory, the best found one by one.
template <class T>
__global__ void __launch_bounds__(256) select_kernel(const SelectParams p) {
  extern __shared__ float score[];
  __shared__ short cp[256], cm[256];
  __shared__ float big;
  __shared__ int odd;
  __shared__ float wv[8];
  __shared__ int wi[8];
  const int t = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  const Seen s = seen_keys(t, p.T, p.B, p.starts, p.lens, p.width * p.page, p.causal, p.status);
  const int P = (s.keys + p.page - 1) / p.page;
  int* out = p.sel + ((int64_t)t * p.H + h) * p.keep;
  if (P <= p.keep) {
    for (int i = tid; i < p.keep; i += 256) out[i] = i < P ? i : -1;
    return;
  }
  if (tid == 0) {
    big = 0.f;
    odd = 0;
  }
  __syncthreads();
  const T* q = static_cast<const T*>(p.q) + t * p.q_ts + (int64_t)h * p.G * p.q_hs;
  if (tid < p.D) {
    float m = 0.f;
    for (int g = 0; g < p.G; ++g) {
      const float v = to_f32(q[g * p.q_hs + tid]);
      if (!isfinite(v)) odd = 1;
      m = fmaxf(m, fabsf(v));
    }
    atomicMax(reinterpret_cast<int*>(&big), __float_as_int(m));
  }
  __syncthreads();
  const bool zero = odd || !(big >= kTiny);
  const float r = zero ? 0.f : __fdiv_rn((float)p.Q, big);
  if (tid < p.D) {
    int a = 0, b = 0;
    for (int g = 0; g < p.G; ++g) {
      const int c = zero ? 0 : (int)rintf(__fmul_rn(to_f32(q[g * p.q_hs + tid]), r));
      a += max(c, 0);
      b += min(c, 0);
    }
    cp[tid] = (short)a;
    cm[tid] = (short)b;
  }
  __syncthreads();
  for (int w = tid; w < P; w += 256) {
    float v = INFINITY;
    if (w >= p.first && w < P - p.last) {
      const int id = p.table[(int64_t)s.b * p.width + w];
      v = -INFINITY;
      if (id < 0 || id >= p.pages) {
        atomicOr(p.status, PP_CACHE_BAD_PAGE);
      } else {
        const int64_t cell = (int64_t)id * p.H + h;
        const int8_t* c = p.codes + cell * 2 * p.D;
        int sum = 0;
        for (int d = 0; d < p.D; ++d) sum += cp[d] * c[d] + cm[d] * c[p.D + d];
        v = __fmul_rn((float)sum, p.scales[cell]);
        if (v != v) v = -INFINITY;
      }
    }
    score[w] = v;
  }
  __syncthreads();
  // the keep best: the largest left, of equal ones the lowest, taken out (NaN) until enough are
  for (int n = 0; n < p.keep; ++n) {
    float best = -INFINITY;
    int at = INT32_MAX;
    for (int w = tid; w < P; w += 256) {
      const float v = score[w];
      if (v == v && (v > best || at == INT32_MAX)) {
        best = v;
        at = w;
      }
    }
    for (int d = 16; d > 0; d >>= 1) {
      const float v = __shfl_xor_sync(~0u, best, d);
      const int a = __shfl_xor_sync(~0u, at, d);
      if (a != INT32_MAX && (at == INT32_MAX || v > best || (v == best && a < at))) {
        best = v;
        at = a;
      }
    }
    if (tid % 32 == 0) {
      wv[tid / 32] = best;
      wi[tid / 32] = at;
    }
    __syncthreads();
    if (tid == 0) {
      for (int i = 1; i < 8; ++i)
        if (wi[i] != INT32_MAX && (at == INT32_MAX || wv[i] > best || (wv[i] == best && wi[i] < at))) {
          best = wv[i];
          at = wi[i];
        }
      score[at] = nanf("");
    }
    __syncthreads();
  }
  if (tid == 0) {
    int n = 0;
    for (int w = 0; w < P; ++w)
      if (score[w] != score[w]) out[n++] = w;
  }
}

DeviceOnce g_select_once;

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// A pool as [pages * H * page][D]: boxes of 128 bytes by up to a tile of one page's rows, zeros beyond D.
bool pool_map(CUtensorMap* m, const pp_cache& c, void* pool) {
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult q;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
      q != cudaDriverEntryPointSuccess)
    return false;
  const int e = dtype_size(c.dtype);
  const cuuint64_t dims[2] = {(cuuint64_t)c.D, (cuuint64_t)c.pages * c.H * c.page};
  const cuuint64_t strides[1] = {(cuuint64_t)c.D * e};
  const cuuint32_t box[2] = {(cuuint32_t)(128 / e), (cuuint32_t)std::min(c.page, tile_keys(c.dtype))};
  const cuuint32_t estr[2] = {1, 1};
  const CUtensorMapDataType t = c.dtype == PP_F32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                : c.dtype == PP_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                    : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  return reinterpret_cast<EncodeTiledFn>(fn)(m, t, 2, pool, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

extern "C" {

pp_status pp_cache_create(int dtype, int pages, int page, int H, int D, void* k, void* v, int8_t* codes, float* scales,
                          pp_cache** out) {
  if (!out || !k || !v || !dtype_ok(dtype) || pages < 1 || H < 1 || D < 1 || page < 1 || !codes != !scales)
    return PP_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | reinterpret_cast<uintptr_t>(codes) |
       reinterpret_cast<uintptr_t>(scales)) & 15)
    return PP_ERR_INVALID_ARG;
  if (page < 8 || page > 256 || (page & (page - 1)) || D % 8 || D < 16 || D > 256 || H > 65535 ||
      (int64_t)pages * page >= (int64_t)INT32_MAX / H)
    return PP_ERR_UNSUPPORTED;
  pp_cache* c = new (std::nothrow) pp_cache;
  if (!c) return PP_ERR_OOM;
  c->dtype = dtype;
  c->pages = pages;
  c->page = page;
  c->H = H;
  c->D = D;
  c->k = k;
  c->v = v;
  c->codes = codes;
  c->scales = scales;
  const int sms = device_sms();
  if (sms <= 0 || attn_prepare() != cudaSuccess || !pool_map(&c->mk, *c, k) || !pool_map(&c->mv, *c, v)) {
    delete c;
    return PP_ERR_CUDA;
  }
  const AttnSpace space = attn_space(dtype, D, sms);
  const size_t head = 256 + (space.counters + 255) / 256 * 256;
  cudaError_t e = cudaMalloc(&c->dmem, head + space.partial);
  if (e != cudaSuccess) {
    cudaGetLastError();
    delete c;
    return e == cudaErrorMemoryAllocation ? PP_ERR_OOM : PP_ERR_CUDA;
  }
  e = cudaMemset(c->dmem, 0, head);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    pp_cache_destroy(c);
    return PP_ERR_CUDA;
  }
  c->status = static_cast<int*>(c->dmem);
  c->counters = reinterpret_cast<int*>(static_cast<char*>(c->dmem) + 256);
  c->partial = reinterpret_cast<float*>(static_cast<char*>(c->dmem) + head);
  *out = c;
  return PP_OK;
}

void pp_cache_destroy(pp_cache* cache) {
  if (!cache) return;
  cudaFree(cache->dmem);
  delete cache;
}

pp_status pp_cache_device_status(const pp_cache* cache, int* device_error) {
  if (!cache || !device_error) return PP_ERR_INVALID_ARG;
  int v = 0;
  if (cudaDeviceSynchronize() != cudaSuccess ||
      cudaMemcpy(&v, cache->status, sizeof(v), cudaMemcpyDeviceToHost) != cudaSuccess ||
      cudaMemset(cache->status, 0, sizeof(v)) != cudaSuccess)
    return PP_ERR_CUDA;
  *device_error = v;
  return PP_OK;
}

pp_status pp_cache_summarize(const pp_cache* cache, const int32_t* ids, int n, void* stream) {
  if (!cache || n < 0 || !cache->codes || (n > 0 && !ids)) return PP_ERR_INVALID_ARG;
  if (n == 0) return PP_OK;
  const cudaStream_t s = (cudaStream_t)stream;
  const dim3 grid(n, cache->H);
  const pp_cache& c = *cache;
  if (c.dtype == PP_F32)
    summarize_kernel<<<grid, c.D, 0, s>>>(static_cast<const float*>(c.k), ids, c.pages, c.page, c.H, c.D, c.codes,
                                          c.scales, c.status);
  else if (c.dtype == PP_F16)
    summarize_kernel<<<grid, c.D, 0, s>>>(static_cast<const __half*>(c.k), ids, c.pages, c.page, c.H, c.D, c.codes,
                                          c.scales, c.status);
  else
    summarize_kernel<<<grid, c.D, 0, s>>>(static_cast<const __nv_bfloat16*>(c.k), ids, c.pages, c.page, c.H, c.D,
                                          c.codes, c.scales, c.status);
  return cudaGetLastError() == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

pp_status pp_cache_select(const pp_cache* cache, int T, const void* q, int64_t q_ts, int64_t q_hs, int Hq, int B,
                          const int32_t* starts, const int32_t* table, int width, const int32_t* lens, int flags,
                          int first, int last, int keep, int32_t* sel, void* stream) {
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
  const cudaError_t e = g_select_once.run([](int) {
    cudaError_t r = cudaFuncSetAttribute(select_kernel<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, 131072);
    if (r == cudaSuccess)
      r = cudaFuncSetAttribute(select_kernel<__half>, cudaFuncAttributeMaxDynamicSharedMemorySize, 131072);
    if (r == cudaSuccess)
      r = cudaFuncSetAttribute(select_kernel<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, 131072);
    return r;
  });
  if (e != cudaSuccess) return PP_ERR_CUDA;
  SelectParams p = {q, q_ts, q_hs, starts, table, lens, cache->codes, cache->scales, sel, cache->status, T, B, cache->H, G,
                    cache->D, cache->page, cache->pages, width, first, last, keep, (int)Q, flags & PP_ATTN_CAUSAL};
  const dim3 grid(T, cache->H);
  const cudaStream_t s = (cudaStream_t)stream;
  const size_t smem = (size_t)width * 4;
  if (cache->dtype == PP_F32)
    select_kernel<float><<<grid, 256, smem, s>>>(p);
  else if (cache->dtype == PP_F16)
    select_kernel<__half><<<grid, 256, smem, s>>>(p);
  else
    select_kernel<__nv_bfloat16><<<grid, 256, smem, s>>>(p);
  return cudaGetLastError() == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

}  // extern "C"
