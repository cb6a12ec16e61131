// whtmix_gemm_gated_e4m3.cu -- the instances of whtmix_gemm_gated.cuh with 8-bit operands, bf16 and float output.
#include "whtmix_gemm_gated.cuh"

namespace whtmix {
namespace linear {

cudaError_t gemm_gated_e4m3(const Gated& g, bool out_f32, int bn, bool four, int sms, cudaStream_t stream) {
  return out_f32 ? gated_by_width<true, float>(g, bn, four, sms, stream) : gated_by_width<true, __nv_bfloat16>(g, bn, four, sms, stream);
}

}  // namespace linear
}  // namespace whtmix
