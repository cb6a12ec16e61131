// whtmix_gemm_gated.cu -- the instances of whtmix_gemm_gated.cuh with bf16 operands, bf16 and float output.
#include "whtmix_gemm_gated.cuh"

namespace whtmix {
namespace linear {

cudaError_t gemm_gated(const Gated& g, bool out_f32, int bn, bool four, int sms, cudaStream_t stream) {
  return out_f32 ? gated_by_width<false, float>(g, bn, four, sms, stream) : gated_by_width<false, __nv_bfloat16>(g, bn, four, sms, stream);
}

}  // namespace linear
}  // namespace whtmix
