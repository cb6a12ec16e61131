// whtmix_few.cuh -- the linear layer's forward for few tokens or few tiles (whtmix_few.cu): x and W (at x, w) with 16-byte aligned
// rows, everything else as whtmix_linear.cuh has it.
#pragma once

#include "whtmix_linear.cuh"

namespace whtmix {
namespace linear {

bool use_few(long long T, int N, int sms);
cudaError_t forward_few(const Forward& a, const void* x, long long xs, const void* w, long long ws, unsigned int* err, int sms,
                        cudaStream_t stream);

}  // namespace linear
}  // namespace whtmix
