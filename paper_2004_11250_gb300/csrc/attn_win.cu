// The row kernel (attn_row.cuh) over fp32, f16 and bf16 with a sliding window.
#include "attn_row.cuh"

namespace ppc_attn {

using namespace ppc_row;

cudaError_t rows_window_launch(const AttnParams& p, const pp_cache& c, int sms, cudaStream_t stream) {
  return c.dtype == PP_F32   ? by_head<float, float, true>(p, c, sms, stream)
         : c.dtype == PP_F16 ? by_head<__half, __half, true>(p, c, sms, stream)
                             : by_head<__nv_bfloat16, __nv_bfloat16, true>(p, c, sms, stream);
}

cudaError_t rows_window_prepare() {
  cudaError_t e = prepare_type<float, float, true>();
  if (e == cudaSuccess) e = prepare_type<__half, __half, true>();
  if (e == cudaSuccess) e = prepare_type<__nv_bfloat16, __nv_bfloat16, true>();
  return e;
}

}  // namespace ppc_attn
