// whtmix_unaligned.cuh -- 16 bytes from any address: two aligned loads, shifted into place.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace whtmix {

// The bytes of a matrix, first to one past its last: an aligned load that would reach outside takes its bytes one by one.
struct Span {
  const uint8_t *lo, *hi;
};
__device__ __forceinline__ Span span_of(const void* p, long long rows, long long stride, long long cols, int es) {
  const uint8_t* b = static_cast<const uint8_t*>(p);
  return {b, b + ((rows - 1) * stride + cols) * es};
}

// Bytes s .. s + 4 W - 1 (0 < s < 4 W) of the 2 W words w, into the first W of them.
template <int W>
__device__ __forceinline__ void shift_bytes(uint32_t (&w)[2 * W], uint32_t s) {
  if constexpr (W >= 4) {
    if (s & 8u) {
#pragma unroll
      for (int i = 0; i + 2 < 2 * W; ++i) w[i] = w[i + 2];
    }
  }
  if constexpr (W >= 2) {
    if (s & 4u) {
#pragma unroll
      for (int i = 0; i + 1 < 2 * W; ++i) w[i] = w[i + 1];
    }
  }
#pragma unroll
  for (int i = 0; i < W; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 8 * (s & 3u));
}

// Bytes p .. p + 15 in two steps, so that many lanes' and vectors' loads are in flight before the first is used: the two aligned
// granules, loaded where they lie in the span, and the bytes of them (outside the span: zeros; only there byte by byte).
struct Granules {
  uint4 a, b;
};
__device__ __forceinline__ Granules fetch16(const uint8_t* p, const Span s) {
  const uint8_t* q = p - (static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 15u);
  Granules g{make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
  if (q >= s.lo && q + 16 <= s.hi) g.a = *reinterpret_cast<const uint4*>(q);
  if (q != p && q + 32 <= s.hi) g.b = *reinterpret_cast<const uint4*>(q + 16);
  return g;
}
static __device__ __noinline__ uint4 bytes16(const uint8_t* p, const uint8_t* lo, const uint8_t* hi) {
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (p + i >= lo && p + i < hi) w[i >> 2] |= static_cast<uint32_t>(p[i]) << (8 * (i & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 finish16(const Granules g, const uint8_t* p, const Span s) {
  const uint32_t m = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 15u;
  if (p - m < s.lo || p - m + (m ? 32 : 16) > s.hi) return bytes16(p, s.lo, s.hi);
  if (m == 0) return g.a;
  uint32_t w[8] = {g.a.x, g.a.y, g.a.z, g.a.w, g.b.x, g.b.y, g.b.z, g.b.w};
  shift_bytes<4>(w, m);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The first `bytes` (0 .. 16) of u, zeros beyond.
__device__ __forceinline__ uint4 keep(uint4 u, int bytes) {
  auto word = [&](uint32_t w, int at) { return bytes >= at + 4 ? w : bytes <= at ? 0u : w & (0xffffffffu >> (8 * (at + 4 - bytes))); };
  return make_uint4(word(u.x, 0), word(u.y, 4), word(u.z, 8), word(u.w, 12));
}

}  // namespace whtmix
