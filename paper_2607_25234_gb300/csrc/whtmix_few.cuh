// whtmix_few.cuh -- the linear layer's forward for few tokens (whtmix_few.cu): x and W (at x, w) with 16-byte aligned
// rows, everything else as whtmix_linear.cuh has it.
#pragma once

#include "whtmix_linear.cuh"

namespace whtmix {
namespace linear {

// T tokens, K in blocks of 128 bytes.  Measured against whtmix_gemm.cuh (us, gelu, [T, K] x [N, K]): 100 tokens, K = 256, N = 1024
// 7.1 and 5.1, K = 1024 6.2 and 8.4; 250 tokens, K = 1024, N = 4096 12.6 and 8.7, K = N = 4096 19.0 and 22.7; 500 tokens,
// K = N = 4096 24.7 and 25.0, K = N = 1024 10.3 and 8.6.
bool use_few(long long T, int kblocks);
cudaError_t forward_few(const Forward& a, const void* x, long long xs, const void* w, long long ws, unsigned int* err, int sms,
                        cudaStream_t stream);

}  // namespace linear
}  // namespace whtmix
