// Attention of query tokens over the paged cache: the calls (pp_attn_forward,
// pp_attn_window), and the row kernel over fp32, f16 and bf16 without a window.
#include "attn_row.cuh"

namespace {

using namespace ppc_row;

DeviceOnce g_attn_once;

// What both calls ask, and their kernels.  window below 0: none.
pp_status attend(const pp_cache* cache, int T, const void* q, int64_t q_ts, int64_t q_hs, int Hq, int B, const int32_t* starts,
                 const int32_t* table, int width, const int32_t* lens, float scale, int flags, const int32_t* sel, int keep,
                 int window, int sinks, void* out, float* lse, void* stream) {
  if (!cache || T < 0 || B < 0 || Hq < 1 || Hq % cache->H || width < 1 || q_ts < 0 || q_hs < 0 || !std::isfinite(scale) ||
      (flags & ~PP_ATTN_CAUSAL) || (sel ? keep < 1 : keep != 0))
    return PP_ERR_INVALID_ARG;
  const uintptr_t al = (uintptr_t)dtype_size(cache->dtype) - 1;
  if (T > 0 && (!q || !table || !lens || !out || B < 1 || (!starts && T != B) || (reinterpret_cast<uintptr_t>(q) & al) ||
                (reinterpret_cast<uintptr_t>(out) & al) || (reinterpret_cast<uintptr_t>(lse) & 3)))
    return PP_ERR_INVALID_ARG;
  const bool eight = cache->scales8[0] != nullptr;
  if (sel && eight) return PP_ERR_UNSUPPORTED;
  if (T == 0) return PP_OK;
  if ((int64_t)width * cache->page > INT32_MAX - 256) return PP_ERR_UNSUPPORTED;  // the end of a tile is counted in 32 bits, too
  const int sms = device_sms();
  if (sms <= 0) return PP_ERR_CUDA;
  const pp_cache& c = *cache;
  const int G = Hq / c.H;
  if ((int64_t)T * G >= INT32_MAX) return PP_ERR_UNSUPPORTED;
  const int most = width * c.page;
  const bool windowed = window >= 0 && window < most;
  AttnParams p = {q,     q_ts,   q_hs,        c.k,        c.v,     starts, table, lens, sel,  out, lse, c.status, c.counters,
                  c.partial, scale, T, B, c.H, c.D, c.page, log2_of(c.page), c.pages, width, keep, flags & PP_ATTN_CAUSAL,
                  FastDiv(G), FastDiv(c.H), FastDiv(std::max(keep, 1)), 1, nullptr, nullptr,
                  windowed ? window : most, windowed ? std::min(sinks, most) : 0, c.scales8[0], c.scales8[1]};
  const cudaStream_t s = (cudaStream_t)stream;
  const cudaError_t e = eight ? (tile8_applicable(p, c.dtype, sms) ? tile8_launch(p, c, sms, s) : rows8_launch(p, c, sms, s))
                        : tile_applicable(p, c.dtype, sms) ? tile_launch(p, c, sms, s)
                        : windowed ? rows_window_launch(p, c, sms, s)
                                   : rows_launch(p, c, sms, s);
  return e == cudaSuccess ? PP_OK : e == cudaErrorNotSupported ? PP_ERR_UNSUPPORTED : PP_ERR_CUDA;
}

}  // namespace

namespace ppc_attn {

cudaError_t rows_launch(const AttnParams& p, const pp_cache& c, int sms, cudaStream_t stream) {
  return c.dtype == PP_F32   ? by_head<float, float, false>(p, c, sms, stream)
         : c.dtype == PP_F16 ? by_head<__half, __half, false>(p, c, sms, stream)
                             : by_head<__nv_bfloat16, __nv_bfloat16, false>(p, c, sms, stream);
}

}  // namespace ppc_attn

namespace ppc {

AttnSpace attn_space(int dtype, int D, int sms) {
  const int DP = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  const size_t ctas = (size_t)std::min(sms * (DP <= 128 ? 3 : 1), kMaxCtas);
  return {ctas * 3 * 4, ctas * 2 * (kRows * DP + 2 * kRows) * 4, tile_space(dtype, D, sms)};
}

cudaError_t attn_prepare() {
  return g_attn_once.run([](int) {
    cudaError_t e = tile_prepare();
    if (e == cudaSuccess) e = prepare_type<float, float, false>();
    if (e == cudaSuccess) e = prepare_type<__half, __half, false>();
    if (e == cudaSuccess) e = prepare_type<__nv_bfloat16, __nv_bfloat16, false>();
    if (e == cudaSuccess) e = rows_window_prepare();
    if (e == cudaSuccess) e = rows8_prepare();
    if (e == cudaSuccess) e = tile8_prepare();
    return e;
  });
}

}  // namespace ppc

extern "C" pp_status pp_attn_forward(const pp_cache* cache, int T, const void* q, int64_t q_ts, int64_t q_hs, int Hq,
                                     int B, const int32_t* starts, const int32_t* table, int width, const int32_t* lens,
                                     float scale, int flags, const int32_t* sel, int keep, void* out, float* lse,
                                     void* stream) {
  return attend(cache, T, q, q_ts, q_hs, Hq, B, starts, table, width, lens, scale, flags, sel, keep, -1, 0, out, lse, stream);
}

extern "C" pp_status pp_attn_window(const pp_cache* cache, int T, const void* q, int64_t q_ts, int64_t q_hs, int Hq,
                                    int B, const int32_t* starts, const int32_t* table, int width, const int32_t* lens,
                                    float scale, int flags, int window, int sinks, void* out, float* lse, void* stream) {
  if (window < 1 || sinks < 0) return PP_ERR_INVALID_ARG;
  return attend(cache, T, q, q_ts, q_hs, Hq, B, starts, table, width, lens, scale, flags, nullptr, 0, window, sinks, out, lse, stream);
}
