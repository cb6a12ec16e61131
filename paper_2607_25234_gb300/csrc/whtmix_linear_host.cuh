// whtmix_linear_host.cuh -- host pieces of the linear layer (whtmix_linear.cu) that the gated half's calls (whtmix_gated.cu) take too.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace whtmix {
namespace linear {

// dst [rows, pitch] = src [rows, cols], zeros beyond cols; stride, cols, pitch in bytes, pitch a multiple of 16
struct Copy {
  uint8_t* dst;
  const uint8_t* src;
  long long rows, stride, cols, pitch;
  __host__ __device__ long long chunks() const { return rows * (pitch / 16); }
};
inline Copy copy_of(void* dst, const void* src, long long rows, int cols, long long stride, int pitch, int es) {
  return {static_cast<uint8_t*>(dst), static_cast<const uint8_t*>(src), rows, stride * es, static_cast<long long>(cols) * es,
          static_cast<long long>(pitch) * es};
}
// up to two copies (dst null: none) in one launch
cudaError_t to_pitch(const Copy& a, const Copy& b, int sms, cudaStream_t stream);

inline size_t align256(size_t v) { return (v + 255) & ~size_t{255}; }
inline int pitch_of(int cols, int es) { return (cols + 16 / es - 1) / (16 / es) * (16 / es); }
inline int ceil_div(long long a, long long b) { return static_cast<int>((a + b - 1) / b); }

struct Plan {
  int bn, splits;
};
Plan plan_product(long long M, int N, int kblocks, int sms, int max_splits);

}  // namespace linear
}  // namespace whtmix
