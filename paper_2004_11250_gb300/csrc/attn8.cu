// The row kernel (attn_row.cuh) over a cache in 8 bits, with a window (or one of all keys).
#include "attn_row.cuh"

namespace ppc_attn {

using namespace ppc_row;

cudaError_t rows8_launch(const AttnParams& p, const pp_cache& c, int sms, cudaStream_t stream) {
  return c.dtype == PP_F32   ? by_head<float, int8_t, true>(p, c, sms, stream)
         : c.dtype == PP_F16 ? by_head<__half, int8_t, true>(p, c, sms, stream)
                             : by_head<__nv_bfloat16, int8_t, true>(p, c, sms, stream);
}

cudaError_t rows8_prepare() {
  cudaError_t e = prepare_type<float, int8_t, true>();
  if (e == cudaSuccess) e = prepare_type<__half, int8_t, true>();
  if (e == cudaSuccess) e = prepare_type<__nv_bfloat16, int8_t, true>();
  return e;
}

}  // namespace ppc_attn
