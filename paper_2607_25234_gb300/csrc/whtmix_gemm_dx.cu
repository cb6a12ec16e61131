// whtmix_gemm_dx.cu -- the input gradient's instances of whtmix_gemm.cuh: dx = dp W, both operands as they lie.
#include "whtmix_gemm.cuh"

namespace whtmix {
namespace linear {

cudaError_t gemm_dx(const Gemm& g, int bn, int sms, cudaStream_t stream) {
  return gemm_by_width<false, false, true, __nv_bfloat16>(g, bn, sms, stream);
}

}  // namespace linear
}  // namespace whtmix
