// whtmix_gemm_bwd.cu -- the backward products' instances of whtmix_gemm.cuh: dx = dp W and dw = dp^T x, operands as they lie.
#include "whtmix_gemm.cuh"

namespace whtmix {
namespace linear {

cudaError_t gemm_dx(const Gemm& g, int bn, int sms, cudaStream_t stream) {
  switch (bn) {
    case 64: return launch_gemm<false, false, true, 64, __nv_bfloat16>(g, sms, stream);
    case 128: return launch_gemm<false, false, true, 128, __nv_bfloat16>(g, sms, stream);
    default: return launch_gemm<false, false, true, 256, __nv_bfloat16>(g, sms, stream);
  }
}

template <typename O>
static cudaError_t dw_by_width(const Gemm& g, int bn, int sms, cudaStream_t stream) {
  switch (bn) {
    case 64: return launch_gemm<false, true, true, 64, O>(g, sms, stream);
    case 128: return launch_gemm<false, true, true, 128, O>(g, sms, stream);
    default: return launch_gemm<false, true, true, 256, O>(g, sms, stream);
  }
}
cudaError_t gemm_dw(const Gemm& g, bool out_f32, int bn, int sms, cudaStream_t stream) {
  return out_f32 ? dw_by_width<float>(g, bn, sms, stream) : dw_by_width<__nv_bfloat16>(g, bn, sms, stream);
}

}  // namespace linear
}  // namespace whtmix
