// whtmix_layer_norm.cuh -- arguments and launches of the layer norm kernels (whtmix_layer_norm.cu), shared with the host side of the
// C ABI.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>

namespace whtmix {
namespace norm {

// Rows of D elements; strides count elements from one row to the next.
struct LayerForward {
  const void* x;
  const void* r;  // residual, or null
  const float* w;
  const float* b;  // or null
  void* h;         // x + r, or null
  void* y;         // same type as x, or e4m3
  float* scale;    // e4m3 only: one a row
  long long T, xs, rs, hs, ys;
  int D;
  float eps;
};
struct LayerBackward {
  const void* h;
  const float* w;
  const void* dy;
  const void* dh;  // gradient that reaches h directly, or null
  void* dx;
  float* dw;
  float* db;    // or null
  void* ws;     // as many bytes as layer_backward_workspace says
  long long T, hs, ys, ds, xs;  // strides of h, dy, dh, dx
  int D;
  float eps;
};

// err: the word that a wait that gave up leaves its mark in
cudaError_t layer_forward(const LayerForward& a, bool bf16, bool to_e4m3, unsigned int* err, int sms, cudaStream_t stream);
cudaError_t layer_backward_workspace(const LayerBackward& a, bool bf16, int sms, size_t* bytes);  // (of a its ws is not read)
cudaError_t layer_backward(const LayerBackward& a, bool bf16, unsigned int* err, int sms, cudaStream_t stream);

}  // namespace norm
}  // namespace whtmix
