// whtmix_few.cuh -- the linear layer's forward for up to FEW_TOKENS tokens (whtmix_few.cu); any size and alignment, no workspace.
#pragma once

#include "whtmix_linear.cuh"

namespace whtmix {
namespace linear {

constexpr int FEW_TOKENS = 64;
cudaError_t forward_few(const Forward& a, int sms, cudaStream_t stream);

}  // namespace linear
}  // namespace whtmix
