// whtmix_unaligned.cuh -- 16 bytes from any address in two aligned loads, for rows that do not start on 16-byte boundaries.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace whtmix {

// The bytes of a matrix, first to one past its last: an aligned load that would reach outside takes its bytes one by one.
struct Span {
  const uint8_t *lo, *hi;
};

static __device__ __noinline__ uint4 granule_bytes(const uint8_t* a, const uint8_t* lo, const uint8_t* hi) {
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (a + i >= lo && a + i < hi) w[i >> 2] |= static_cast<uint32_t>(a[i]) << (8 * (i & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 granule(const uint8_t* a, const Span s) {
  return a >= s.lo && a + 16 <= s.hi ? *reinterpret_cast<const uint4*>(a) : granule_bytes(a, s.lo, s.hi);
}

// Bytes p .. p + 15 (those outside the span are zero).
__device__ __forceinline__ uint4 load16(const uint8_t* p, const Span s) {
  const uint32_t m = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 15u;
  const uint4 a = granule(p - m, s);
  if (m == 0) return a;
  const uint4 b = granule(p - m + 16, s);
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (m & 8u) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (m & 4u) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  const uint32_t bits = 8 * (m & 3u);
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                    __funnelshift_r(w[3], w[4], bits));
}

// The first `bytes` (0 .. 16) of u, zeros beyond.
__device__ __forceinline__ uint4 keep(uint4 u, int bytes) {
  auto word = [&](uint32_t w, int at) { return bytes >= at + 4 ? w : bytes <= at ? 0u : w & (0xffffffffu >> (8 * (at + 4 - bytes))); };
  return make_uint4(word(u.x, 0), word(u.y, 4), word(u.z, 8), word(u.w, 12));
}

}  // namespace whtmix
