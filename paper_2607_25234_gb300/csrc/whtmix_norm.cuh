// whtmix_norm.cuh -- arguments and launches of the RMS norm kernels (whtmix_norm.cu), shared with the host side of the C ABI.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>

namespace whtmix {
namespace norm {

// Rows of D elements; strides count elements from one row to the next.
struct Forward {
  const void* x;
  const void* r;  // residual, or null
  const float* w;
  void* h;       // x + r, or null
  void* y;       // same type as x, or e4m3
  float* scale;  // e4m3 only: one a row
  long long T, xs, rs, hs, ys;
  int D;
  float eps;
};
struct Backward {
  const void* h;
  const float* w;
  const void* dy;
  const void* dh;  // gradient that reaches h directly, or null
  void* dx;
  float* dw;
  void* ws;  // as many bytes as backward_workspace says
  long long T, hs, ys, ds, xs;  // strides of h, dy, dh, dx
  int D;
  float eps;
};

cudaError_t forward(const Forward& a, bool bf16, bool to_e4m3, int sms, cudaStream_t stream);
cudaError_t backward_workspace(const Backward& a, bool bf16, int sms, size_t* bytes);  // (of a its ws is not read)
// out[e] = the sum over `parts` of part[p][e], e < D, in a fixed order (also the linear layer's bias gradient)
cudaError_t add_rows(const float* part, float* out, int D, int parts, cudaStream_t stream);
cudaError_t backward(const Backward& a, bool bf16, int sms, cudaStream_t stream);

}  // namespace norm
}  // namespace whtmix
