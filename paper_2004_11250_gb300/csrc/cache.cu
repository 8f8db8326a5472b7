// The paged cache: its handle and page summaries (pp_cache_create,
// pp_cache_summarize).
#include <algorithm>
#include <cmath>
#include <new>

#include "cache.h"
#include "internal.h"

namespace {

using namespace ppc;

constexpr int kThreads = 256;

// ---- summaries: one block per (page, head).  Bound by reading the page's keys once: a thread takes 16 bytes of every
// R-th row, then thread d joins the R partial extremes of value d.  32 pages of 64 keys, 8 heads of 128 (bf16): 4.7 us, 0.9
// TB/s, a launch and two latencies.
template <class T>
__global__ void __launch_bounds__(kThreads) summarize_kernel(const T* __restrict__ k, const int* __restrict__ ids,
                                                             int pages, int page, int H, int D,
                                                             int8_t* __restrict__ codes, float* __restrict__ scales,
                                                             int* status) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float hi[kThreads * V], lo[kThreads * V];
  __shared__ float big[kThreads / 32];
  after_previous();
  const int id = ids[blockIdx.x], h = blockIdx.y, tid = threadIdx.x;
  if (id < 0 || id >= pages) {
    if (tid == 0) atomicOr(status, PP_CACHE_BAD_PAGE);
    return;
  }
  const int64_t cell = (int64_t)id * H + h;
  const int lanes = D / V, R = kThreads / lanes, row = tid / lanes, d0 = tid % lanes * V;
  bool bad = false;
  if (row < R) {
    float mx[V], mn[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      mx[i] = -INFINITY;
      mn[i] = INFINITY;
    }
    const T* x = k + cell * page * D + d0;
#pragma unroll 4
    for (int r = row; r < page; r += R) {
      const Vec<T, V> v = *reinterpret_cast<const Vec<T, V>*>(x + (int64_t)r * D);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float f = to_f32(v.v[i]);
        bad = bad || !isfinite(f);
        mx[i] = fmaxf(mx[i], f);
        mn[i] = fminf(mn[i], f);
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      hi[row * D + d0 + i] = mx[i];
      lo[row * D + d0 + i] = mn[i];
    }
  }
  const bool odd = __syncthreads_or(bad);
  float mx = -INFINITY, mn = INFINITY, a = 0.f;
  if (tid < D) {
    const int used = min(R, page);
    for (int r = 0; r < used; ++r) {
      mx = fmaxf(mx, hi[r * D + tid]);
      mn = fminf(mn, lo[r * D + tid]);
    }
    a = fmaxf(fabsf(mx), fabsf(mn));
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) a = fmaxf(a, __shfl_xor_sync(~0u, a, d));
  if (tid % 32 == 0) big[tid / 32] = a;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) a = fmaxf(a, big[i]);
  const bool zero = odd || !(a >= kTiny);
  const float r = zero ? 0.f : __fdiv_rn(127.f, a);
  if (tid < D) {
    int8_t* c = codes + cell * 2 * D;
    c[tid] = zero ? 0 : (int8_t)fminf(ceilf(__fmul_rn(mx, r)), 127.f);
    c[D + tid] = zero ? 0 : (int8_t)fmaxf(floorf(__fmul_rn(mn, r)), -127.f);
  }
  if (tid == 0) scales[cell] = odd ? nanf("") : __fmul_rn(a, 1.f / 127.f);
}

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
  if (sms <= 0 || attn_prepare() != cudaSuccess || select_prepare() != cudaSuccess || !pool_map(&c->mk, *c, k) || !pool_map(&c->mv, *c, v)) {
    delete c;
    return PP_ERR_CUDA;
  }
  const AttnSpace space = attn_space(dtype, D, sms);
  const size_t head = 256 + (space.counters + 255) / 256 * 256;
  const size_t partial = (space.partial + 255) / 256 * 256;
  cudaError_t e = cudaMalloc(&c->dmem, head + partial + space.tiles);
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
  c->tiles = reinterpret_cast<float*>(static_cast<char*>(c->dmem) + head + partial);
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
  // The word is clear before the call returns: nothing orders a memset on the default stream before the next kernel of
  // another stream, whose bits it would take away
  if (cudaDeviceSynchronize() != cudaSuccess ||
      cudaMemcpy(&v, cache->status, sizeof(v), cudaMemcpyDeviceToHost) != cudaSuccess ||
      (v && (cudaMemset(cache->status, 0, sizeof(v)) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess)))
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
  auto run = [&](auto* k) {
    using T = std::remove_const_t<std::remove_pointer_t<decltype(k)>>;
    return launch_after(summarize_kernel<T>, grid, kThreads, 0, s, 1, k, ids, c.pages, c.page, c.H, c.D, c.codes, c.scales,
                        c.status);
  };
  const cudaError_t e = c.dtype == PP_F32   ? run(static_cast<const float*>(c.k))
                        : c.dtype == PP_F16 ? run(static_cast<const __half*>(c.k))
                                            : run(static_cast<const __nv_bfloat16*>(c.k));
  return e == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

}  // extern "C"
