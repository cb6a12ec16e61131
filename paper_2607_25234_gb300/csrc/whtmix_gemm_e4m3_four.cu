// whtmix_gemm_e4m3_four.cu -- the forward products' instances of whtmix_gemm.cuh with four epilogue groups: 8-bit operands, bf16 and float output.
#include "whtmix_gemm.cuh"

namespace whtmix {
namespace linear {

cudaError_t gemm_e4m3_four(const Gemm& g, bool out_f32, int bn, int sms, cudaStream_t stream) {
  return out_f32 ? gemm_four<true, float>(g, bn, sms, stream) : gemm_four<true, __nv_bfloat16>(g, bn, sms, stream);
}

}  // namespace linear
}  // namespace whtmix
