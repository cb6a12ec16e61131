// whtmix_gemm_e4m3.cu -- the forward products' instances of whtmix_gemm.cuh: 8-bit operands, bf16 and float output.
#include "whtmix_gemm.cuh"

namespace whtmix {
namespace linear {

cudaError_t gemm_e4m3(const Gemm& g, bool out_f32, int bn, int sms, cudaStream_t stream) {
  return out_f32 ? gemm_by_width<true, false, false, float>(g, bn, sms, stream) : gemm_by_width<true, false, false, __nv_bfloat16>(g, bn, sms, stream);
}

}  // namespace linear
}  // namespace whtmix
