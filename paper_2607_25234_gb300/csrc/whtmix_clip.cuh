// whtmix_clip.cuh -- arguments and launches of the common norm of many tensors and of the scaling by it (whtmix_clip.cu), shared
// with the host side of the C ABI.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>

namespace whtmix {
namespace clip {

struct Item {
  const void* in;
  void* out;  // in itself, or memory apart from it; null for the norm alone
  long long n;
  bool bf16;  // else float
};
// norm = sqrt(sum of all squares);  out = in min(1, max_norm / (norm + 1e-6)) where `scale`
struct Call {
  const Item* items;  // host memory; none is empty
  long long count;
  float* norm;  // or null
  float max_norm;
  bool scale;
};

size_t workspace(const Call& a, int sms);  // may be 0
cudaError_t run(const Call& a, void* ws, int sms, cudaStream_t stream);

}  // namespace clip
}  // namespace whtmix
