// The paged cache: its handle, page summaries and page selection
// (pp_cache_create, pp_cache_summarize, pp_cache_select).
#include <algorithm>
#include <cmath>
#include <new>

#include "cache.h"
#include "internal.h"
#include "tc_ptx.cuh"

namespace {

using namespace ppc;
using namespace ppc_ptx;

constexpr float kTiny = 0x1p-100f;  // largest value below which a page or query counts as 0: 127 / a stays finite

constexpr int kThreads = 256;

// ---- summaries: one block per (page, head).  Bound by reading the page's keys once: a thread takes 16 bytes of every
// R-th row, then thread d joins the R partial extremes of value d.
template <class T>
__global__ void __launch_bounds__(kThreads) summarize_kernel(const T* __restrict__ k, const int* __restrict__ ids,
                                                             int pages, int page, int H, int D,
                                                             int8_t* __restrict__ codes, float* __restrict__ scales,
                                                             int* status) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float hi[kThreads * V], lo[kThreads * V];
  __shared__ float big[kThreads / 32];
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

// ---- selection

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

// A group's queries as sums of integers: value d of up [D] and down [D] for token t and head h, by nthr threads of which
// this is thread i.  big: the largest |q| of the group (infinity if one is not finite).
template <class T>
__device__ __forceinline__ float largest_query(const SelectParams& p, int t, int h, int i, int nthr) {
  const T* q = static_cast<const T*>(p.q) + t * p.q_ts + (int64_t)h * p.G * p.q_hs;
  float m = 0.f;
  for (int j = i; j < p.G * p.D; j += nthr) {
    const float v = fabsf(to_f32(q[j / p.D * p.q_hs + j % p.D]));
    m = v <= 3.402823466e38f ? fmaxf(m, v) : INFINITY;  // a NaN too
  }
  return m;
}
template <class T>
__device__ __forceinline__ void query_codes(const SelectParams& p, int t, int h, float big, int d, int& up, int& down) {
  const T* q = static_cast<const T*>(p.q) + t * p.q_ts + (int64_t)h * p.G * p.q_hs + d;
  up = down = 0;
  if (!(big >= kTiny) || big == INFINITY) return;
  const float r = __fdiv_rn((float)p.Q, big);
  for (int g = 0; g < p.G; ++g) {
    const int c = (int)rintf(__fmul_rn(to_f32(q[g * p.q_hs]), r));
    up += max(c, 0);
    down += min(c, 0);
  }
}

__device__ __forceinline__ int dot2_lo(int a, int b, int c) {  // c + a's two 16-bit halves times b's bytes 0 and 1
  int d;
  asm("dp2a.lo.s32.s32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ int dot2_hi(int a, int b, int c) {
  int d;
  asm("dp2a.hi.s32.s32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}

// Single tokens: a cluster per (token, head), its CTAs sharing the pages.  Bound by reading the codes, 2 D bytes a page:
// a lane keeps 16 of the query's integers and meets 16 codes of every page with two-way integer products.  The first
// CTA has all scores in shared memory and finds the keep-th largest digit by digit (8 bits each).
template <class T>
__global__ void __launch_bounds__(kThreads) select_kernel(const SelectParams p) {
  extern __shared__ uint32_t key[];
  __shared__ __align__(16) short code[512];
  __shared__ float big[kThreads / 32];
  __shared__ int hist[256], warp_sum[kThreads / 32], digit_of, left_of;
  const int rank = cluster_rank(), ranks = cluster_size();
  const int t = blockIdx.x / ranks, h = blockIdx.y, tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  const Seen s = seen_keys(t, p.T, p.B, p.starts, p.lens, p.width * p.page, p.causal, p.status);
  const int P = (s.keys + p.page - 1) / p.page;
  int* out = p.sel + ((int64_t)t * p.H + h) * p.keep;
  if (P <= p.keep) {  // the whole cluster
    if (rank == 0)
      for (int i = tid; i < p.keep; i += kThreads) out[i] = i < P ? i : -1;
    return;
  }
  float m = largest_query<T>(p, t, h, tid, kThreads);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
  if (lane == 0) big[warp] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) m = fmaxf(m, big[i]);
  if (tid < p.D) {
    int up, down;
    query_codes<T>(p, t, h, m, tid, up, down);
    code[tid] = (short)up;
    code[p.D + tid] = (short)down;
  }
  __syncthreads();
  // candidates: pages first .. P - last - 1; 2 D / 16 lanes a page, in a power of two
  const int N = P - p.first - p.last, chunks = p.D / 8;
  int span = 2;
  while (span < chunks) span *= 2;
  const int at = lane % span, per = 32 / span;  // pages per warp at a time
  int mine[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) mine[i] = at < chunks ? reinterpret_cast<const int*>(code)[at * 8 + i] : 0;
  const int* row = p.table + (int64_t)s.b * p.width + p.first;
  const uint32_t keys0 = map_rank((uint32_t)__cvta_generic_to_shared(key), 0);
  const int step = (kThreads / 32) * per;
  constexpr int U = 4;
  for (int w0 = (rank * U * (kThreads / 32) + warp * U) * per; w0 < N; w0 += ranks * U * step) {
    int4 c[U];
    float sc[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int w = w0 + u * per + lane / span;
      c[u] = make_int4(0, 0, 0, 0);
      sc[u] = nanf("");
      if (w < N) {
        const int id = row[w];
        if (id < 0 || id >= p.pages) {
          if (at == 0) atomicOr(p.status, PP_CACHE_BAD_PAGE);
        } else {
          const int64_t cell = (int64_t)id * p.H + h;
          if (at < chunks) c[u] = *reinterpret_cast<const int4*>(p.codes + cell * 2 * p.D + at * 16);
          sc[u] = p.scales[cell];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int sum = dot2_hi(mine[1], c[u].x, dot2_lo(mine[0], c[u].x, 0));
      sum = dot2_hi(mine[3], c[u].y, dot2_lo(mine[2], c[u].y, sum));
      sum = dot2_hi(mine[5], c[u].z, dot2_lo(mine[4], c[u].z, sum));
      sum = dot2_hi(mine[7], c[u].w, dot2_lo(mine[6], c[u].w, sum));
      for (int d = span / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
      const int w = w0 + u * per + lane / span;
      if (at == 0 && w < N)
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(keys0 + 4 * w), "r"(ordered(__fmul_rn((float)sum, sc[u]))) : "memory");
    }
  }
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (rank != 0) return;
  // the need-th largest key: thr, with `need` of those equal to it (under the mask of the digits found)
  int need = p.keep - p.first - p.last;
  uint32_t thr = 0, mask = 0;
  for (int shift = 24; shift >= 0 && need > 0; shift -= 8) {
    hist[tid] = 0;
    __syncthreads();
    for (int w = tid; w < N; w += kThreads)
      if ((key[w] & mask) == thr) atomicAdd(&hist[key[w] >> shift & 255], 1);
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
    mask |= 255u << shift;
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
  auto run = [&](auto* k) {
    summarize_kernel<<<grid, kThreads, 0, s>>>(k, ids, c.pages, c.page, c.H, c.D, c.codes, c.scales, c.status);
  };
  if (c.dtype == PP_F32)
    run(static_cast<const float*>(c.k));
  else if (c.dtype == PP_F16)
    run(static_cast<const __half*>(c.k));
  else
    run(static_cast<const __nv_bfloat16*>(c.k));
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
  const int sms = device_sms();
  if (sms <= 0) return PP_ERR_CUDA;
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
  // CTAs per (token, head): more where there are few, so that long tables are read by enough of them
  int ranks = 1;
  while (ranks < 8 && (int64_t)T * cache->H * ranks * 2 <= sms * 2 && width >= ranks * 2 * 128) ranks *= 2;
  if ((int64_t)T * ranks > INT32_MAX) return PP_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(T * ranks, cache->H);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)width * 4;
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim = {(unsigned)ranks, 1, 1};
  cfg.attrs = at;
  cfg.numAttrs = 1;
  const cudaError_t r = cache->dtype == PP_F32   ? cudaLaunchKernelEx(&cfg, select_kernel<float>, p)
                        : cache->dtype == PP_F16 ? cudaLaunchKernelEx(&cfg, select_kernel<__half>, p)
                                                 : cudaLaunchKernelEx(&cfg, select_kernel<__nv_bfloat16>, p);
  return r == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

}  // extern "C"
