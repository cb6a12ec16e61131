// whtmix_gemm_fwd.cu -- the forward products' instances of whtmix_gemm.cuh: bf16 and e4m3 operands, bf16 and float output.
#include "whtmix_gemm.cuh"

namespace whtmix {
namespace linear {

template <bool E4M3, typename O>
static cudaError_t by_width(const Gemm& g, int bn, int sms, cudaStream_t stream) {
  switch (bn) {
    case 64: return launch_gemm<E4M3, false, false, 64, O>(g, sms, stream);
    case 128: return launch_gemm<E4M3, false, false, 128, O>(g, sms, stream);
    default: return launch_gemm<E4M3, false, false, 256, O>(g, sms, stream);
  }
}

cudaError_t gemm_forward(const Gemm& g, bool e4m3, bool out_f32, int bn, int sms, cudaStream_t stream) {
  if (e4m3) return out_f32 ? by_width<true, float>(g, bn, sms, stream) : by_width<true, __nv_bfloat16>(g, bn, sms, stream);
  return out_f32 ? by_width<false, float>(g, bn, sms, stream) : by_width<false, __nv_bfloat16>(g, bn, sms, stream);
}

}  // namespace linear
}  // namespace whtmix
