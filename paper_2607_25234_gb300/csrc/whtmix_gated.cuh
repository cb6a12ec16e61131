// whtmix_gated.cuh -- the gated feed-forward half's launches (whtmix_gated.cu), in the arguments of whtmix_linear.cuh: N is the number of
// hidden channels; W is [2 N, K], N gate rows and then N value rows, and so are w_scale, bias, dw and db; p is [T, 2 N].
//
//   g = s_x s_w x Wg^T + bg,  u = s_x s_w x Wu^T + bu,  y = act(g) u                                          (no residual)
//   backward, from p = [g, u]:  dp = [dy u act'(g), dy act(g)],  dx = dp W,  dw = dp^T x,  db = sum over rows of dp
#pragma once

#include "whtmix_linear.cuh"

namespace whtmix {
namespace linear {

size_t gated_forward_workspace(const Forward& a, int sms);
cudaError_t gated_forward(const Forward& a, void* ws, unsigned int* err, int sms, cudaStream_t stream);
size_t gated_backward_workspace(const Backward& a, int sms);
cudaError_t gated_backward(const Backward& a, void* ws, unsigned int* err, int sms, cudaStream_t stream);

}  // namespace linear
}  // namespace whtmix
