// whtmix_linear.cuh -- the linear layer's arguments and launches (whtmix_linear.cu, which calls the products of whtmix_gemm*.cu and
// whtmix_few.cu), shared with the host side of the C ABI.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>

namespace whtmix {
namespace linear {

enum Activation { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

// gelu in its tanh form: z sigmoid(2 u), u = sqrt(2 / pi) (z + 0.044715 z^3);  silu: z sigmoid(z).
constexpr float GELU_2A = 1.5957691216057308f, GELU_B = 0.044715f;

// y = act(s_x s_w x W^T + b) + r:  x [T, K], W [N, K], y and r [T, N], p = s_x s_w x W^T + b before the activation.
struct Forward {
  const void *x, *w;
  const float *x_scale, *w_scale;  // e4m3 only
  const float* bias;               // or null
  const void* r;                   // or null, y's type
  void* p;                         // bf16, or null
  void* y;                         // bf16, or float (out_f32)
  long long T, xs, ws, rs, ps, ys;  // row strides in elements
  int K, N, act;
  bool e4m3, out_f32;
};
// dp = dy act'(p);  dx = dp W;  dw = dp^T x;  db = sum over rows of dp
struct Backward {
  const void *x, *w, *dy, *p;  // p null where act is none
  void *dx, *dw;               // each or null; dw bf16, or float (dw_f32)
  float* db;                   // or null
  long long T, xs, ws, dys, ps, dxs;
  int K, N, act;
  bool dw_f32;
  bool split_dx = false;  // dx's contraction over N may be split over CTAs, as dw's over T is
};

size_t forward_workspace(const Forward& a, int sms);
cudaError_t forward(const Forward& a, void* ws, unsigned int* err, int sms, cudaStream_t stream);
size_t backward_workspace(const Backward& a, int sms);
cudaError_t backward(const Backward& a, void* ws, unsigned int* err, int sms, cudaStream_t stream);

}  // namespace linear
}  // namespace whtmix
