// whtmix_norm.cu -- RMS norm with the residual's addition, its 8-bit output, and its backward.
//
//   h = x + r,   y_d = h_d w_d / sqrt(mean(h^2) + eps)                              one row of D channels
//   8 bits: s = max_d |y_d| / 448,  q_d = e4m3(y_d / s).  1 / sqrt(mean + eps) cancels in y_d / s, so that the q are taken
//   from h_d w_d and its largest magnitude, which is found in the same reduction as the sum of squares.
//   backward, with rstd = 1 / sqrt(mean(h^2) + eps) and a = dy w:
//     dx = rstd a - h rstd^3 mean(a h) + dh,      dw = sum over rows of dy h rstd
//
// All of it is bound by memory: a row is read once into registers (packed as stored), its sums meet in one reduction, and it is
// written once.  TPR threads hold a row, NV 16-byte vectors each; up to 32 threads a row need no shared memory.  Sums are
// float32 in a fixed order.  dw: every thread keeps its columns' sums over the rows that its CTA takes, the CTAs' partial rows
// are added up by k_dw in a fixed order.  Rows that are not 16-byte aligned are read and written in aligned 16-byte accesses
// all the same, but for their ends, short ones that lie one behind another several at a time (k_rms_flat, k_rms_bwd_flat); rows
// beyond 2048 vectors (an unaligned row touches one more) are read twice (k_rms_long, k_rms_bwd_long).
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <map>
#include <mutex>
#include <tuple>
#include <type_traits>
#include <utility>

#include "whtmix_kernels.cuh"
#include "whtmix_norm.cuh"

namespace whtmix {
namespace norm {

constexpr float E4M3_MAX = 448.f;
constexpr int MAX_VECTORS = 2048;  // vectors of a row that fit the threads' registers
constexpr int LONG_THREADS = 512;

template <typename T> struct Io;
template <> struct Io<float> {
  static constexpr int V = 4;
  static __device__ __forceinline__ float get(const void* p, long long i) { return static_cast<const float*>(p)[i]; }
  static __device__ __forceinline__ void put(void* p, long long i, float v) { static_cast<float*>(p)[i] = v; }
  static __device__ __forceinline__ void unpack(uint4 u, float (&f)[4]) {
    f[0] = __uint_as_float(u.x), f[1] = __uint_as_float(u.y), f[2] = __uint_as_float(u.z), f[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <> struct Io<__nv_bfloat16> {
  static constexpr int V = 8;
  static __device__ __forceinline__ float get(const void* p, long long i) {
    return __uint_as_float(static_cast<uint32_t>(static_cast<const unsigned short*>(p)[i]) << 16);
  }
  static __device__ __forceinline__ void put(void* p, long long i, float v) {
    static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  }
  static __device__ __forceinline__ void unpack(uint4 u, float (&f)[8]) {
    const uint32_t a[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) f[2 * j] = __uint_as_float(a[j] << 16), f[2 * j + 1] = __uint_as_float(a[j] & 0xffff0000u);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t a[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
      a[j] = *reinterpret_cast<uint32_t*>(&b);
    }
    return make_uint4(a[0], a[1], a[2], a[3]);
  }
};

// Unaligned rows' gains and sums in shared memory: the places of a vector slots_of() words apart, so that a warp's lanes, whose
// vectors follow one another, touch consecutive words whatever the row's offset; a slot before and one after take the elements of a
// cut vector that are not the row's.
template <int V>
__host__ __device__ constexpr int slots_of(int D) { return (D + V - 1) / V + 2; }
template <int V>
__device__ __forceinline__ int column_at(int c, int D) { return c % V * slots_of<V>(D) + c / V + 1; }
// Where elements 0 .. V - 1 of the vector that starts at -off lie; V elements on each is the next word.
template <int V>
struct Places {
  int at[V];
  __device__ __forceinline__ Places(int off, int D) {
#pragma unroll
    for (int j = 0; j < V; ++j) at[j] = ((j - off) & (V - 1)) * slots_of<V>(D) + (j < off ? 0 : 1);
  }
};

// The addresses of a matrix, first to one past its last.
struct Bounds {
  uintptr_t lo, hi;
};
template <typename T>
__device__ __forceinline__ Bounds bounds_of(const void* p, long long rows, long long stride, int D) {
  const T* b = static_cast<const T*>(p);
  return {reinterpret_cast<uintptr_t>(b), reinterpret_cast<uintptr_t>(b + (rows - 1) * stride + D)};
}

// Vector k of thread `lane` of a row's TPR: V consecutive elements, from at(lane, k) - off on.  AL: rows are 16-byte aligned, whole
// vectors (off = 0).  Otherwise off is the row's distance from the 16-byte boundary before it, so that the vectors lie on such
// boundaries all the same: the first and the last of a row are cut, and go element by element.  So do all vectors of a matrix
// whose rows do not lie like the others' (same = false).
template <typename T, bool AL, int TPR>
struct Row {
  static constexpr int V = Io<T>::V;
  static __device__ __forceinline__ int at(int lane, int k) { return (lane + TPR * k) * V; }
  static __device__ __forceinline__ int offset(const T* p) {
    return AL ? 0 : static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
  }
  static __device__ __forceinline__ bool whole(int e, int D, bool same) { return AL ? e < D : same && e >= 0 && e + V <= D; }
  // a vector of the row that lies in the matrix whole, cut or not
  static __device__ __forceinline__ bool loadable(const T* p, int e, const Bounds& b, bool same, int D) {
    const uintptr_t q = reinterpret_cast<uintptr_t>(p + e);
    return AL ? e < D : same && e > -V && e < D && q >= b.lo && q + 16 <= b.hi;
  }
  // the NV vectors of a row as they lie in memory, and their values (what a cut one holds of other rows is zero; element by element
  // only at the ends of the matrix)
  template <int NV>
  static __device__ __forceinline__ void fetch(const T* p, const Bounds& b, int lane, int off, bool same, int D, uint4 (&u)[NV]) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int e = at(lane, k) - off;
      u[k] = make_uint4(0u, 0u, 0u, 0u);
      if (loadable(p, e, b, same, D)) u[k] = *reinterpret_cast<const uint4*>(p + e);
    }
  }
  static __device__ __forceinline__ void values(const T* p, const Bounds& b, int lane, int k, int off, bool same, int D, uint4 u,
                                                float (&f)[V]) {
    Io<T>::unpack(u, f);
    if constexpr (!AL) {
      const int e = at(lane, k) - off;
      if (!whole(e, D, same)) {
        const bool loaded = loadable(p, e, b, same, D);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          if (e + j < 0 || e + j >= D)
            f[j] = 0.f;
          else if (!loaded)
            f[j] = Io<T>::get(p, e + j);
        }
      }
    }
  }
  static __device__ __forceinline__ void store(T* p, int lane, int k, int off, bool same, int D, const float (&f)[V]) {
    const int e = at(lane, k) - off;
    if (whole(e, D, same)) {
      *reinterpret_cast<uint4*>(p + e) = Io<T>::pack(f);
    } else if constexpr (!AL) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (e + j >= 0 && e + j < D) Io<T>::put(p, e + j, f[j]);
    }
  }
  // AL: from w; otherwise from its copy in shared memory (gains_to_shared)
  static __device__ __forceinline__ void gains(const float* w, const Places<V>& at_, int lane, int k, int off, int D, float (&f)[V]) {
    const int e = at(lane, k) - off;
    if constexpr (AL) {
#pragma unroll
      for (int j = 0; j < V; j += 4) {
        const float4 v = e < D ? __ldg(reinterpret_cast<const float4*>(w + e + j)) : make_float4(0.f, 0.f, 0.f, 0.f);
        f[j] = v.x, f[j + 1] = v.y, f[j + 2] = v.z, f[j + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = e < D ? w[at_.at[j] + lane + TPR * k] : 0.f;
    }
  }
  static __device__ __forceinline__ void store_e4m3(uint8_t* p, int lane, int k, int off, bool same, int D, const float (&f)[V]) {
    const int e = at(lane, k) - off;
    uint32_t u[V / 4];
#pragma unroll
    for (int j = 0; j < V / 4; ++j)
      u[j] = static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(make_float2(f[4 * j], f[4 * j + 1]), __NV_SATFINITE, __NV_E4M3)) |
             static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(make_float2(f[4 * j + 2], f[4 * j + 3]), __NV_SATFINITE, __NV_E4M3)) << 16;
    if (whole(e, D, same)) {
      if constexpr (V == 8)
        *reinterpret_cast<uint2*>(p + e) = make_uint2(u[0], u[1]);
      else
        *reinterpret_cast<uint32_t*>(p + e) = u[0];
    } else if constexpr (!AL) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (e + j >= 0 && e + j < D) p[e + j] = static_cast<uint8_t>(u[j / 4] >> (8 * (j & 3)));
    }
  }
};
template <int V, int BLOCK>
__device__ __forceinline__ void gains_to_shared(float* s, const float* w, int D) {
  for (int i = threadIdx.x; i < V * slots_of<V>(D); i += BLOCK) s[i] = 0.f;
  __syncthreads();
  for (int i = threadIdx.x; i < D; i += BLOCK) s[column_at<V>(i, D)] = __ldg(w + i);
}
// Which matrices of an unaligned call lie like the first one (x; h in the backward).
struct Same {
  bool a, b, c;
};

// Sum of a and sum of b (or, MAXB, the largest b by its bits: magnitudes, where a NaN is above infinity) over a row's TPR
// threads, the same value in each.
template <int TPR, bool MAXB>
__device__ __forceinline__ void row_reduce(float& a, float& b) {
  constexpr int W = TPR < 32 ? TPR : 32;
  auto join = [](float u, float v) {
    return MAXB ? __uint_as_float(max(__float_as_uint(u), __float_as_uint(v))) : u + v;
  };
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    b = join(b, __shfl_xor_sync(0xffffffffu, b, o));
  }
  if constexpr (TPR > 32) {
    __shared__ float sa[TPR / 32], sb[TPR / 32];
    __syncthreads();  // the previous row's values have been read
    if ((threadIdx.x & 31) == 0) sa[threadIdx.x >> 5] = a, sb[threadIdx.x >> 5] = b;
    __syncthreads();
    a = sa[0], b = sb[0];
#pragma unroll
    for (int i = 1; i < TPR / 32; ++i) a += sa[i], b = join(b, sb[i]);
  }
}

// 448 / top would overflow for a row of magnitudes below TINY: such a row is scaled up by a power of two first (exact).
constexpr float TINY = 1e-30f, LIFT = 0x1p80f;
__device__ __forceinline__ float to_e4m3_range(float top, float lift) { return top == 0.f ? 0.f : E4M3_MAX / (top * lift); }

__device__ __forceinline__ float magnitude(float v) { return __uint_as_float(__float_as_uint(v) & 0x7fffffffu); }

template <int TPR> constexpr int BLOCK_OF = TPR > 32 ? TPR : 256;  // threads a CTA

// A thread's gains, where its columns are the same in every row and they are few (else they come again with each row).
template <typename R, bool AL, int NV>
struct Kept {
  static constexpr bool KEEP = AL && NV <= 2;
  float w[KEEP ? NV : 1][R::V];
  __device__ __forceinline__ void fill(const float* g, int lane, int D) {
    if constexpr (KEEP) {
#pragma unroll
      for (int k = 0; k < NV; ++k) R::gains(g, Places<R::V>(0, D), lane, k, 0, D, w[k]);
    }
  }
  __device__ __forceinline__ void get(const float* g, const Places<R::V>& at, int lane, int k, int off, int D, float (&f)[R::V]) const {
    if constexpr (KEEP) {
#pragma unroll
      for (int j = 0; j < R::V; ++j) f[j] = w[k][j];
    } else {
      R::gains(g, at, lane, k, off, D, f);
    }
  }
};

// The next row's loads are issued before this row's sums are complete.
template <typename T, bool Q8, bool AL, int TPR, int NV>
__global__ void __launch_bounds__(BLOCK_OF<TPR>) k_rms(const Forward a, const Same same) {
  constexpr int V = Io<T>::V, BLOCK = BLOCK_OF<TPR>, ROWS = BLOCK / TPR;
  using R = Row<T, AL, TPR>;
  extern __shared__ float s_w[];  // unaligned rows: the gains
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const float inv_d = 1.f / static_cast<float>(a.D);
  pdl_wait();
  // A short launch lets the next kernel come in at once (24 rows to 8 bits and their product, time on the GPU,
  // 12.4 -> 11.0 us); a long one would have it wait in the SMs' way.
  const bool short_launch = gridDim.x < 128;
  if (short_launch) pdl_trigger();
  if constexpr (!AL) {
    gains_to_shared<V, BLOCK>(s_w, a.w, a.D);
    __syncthreads();
  }
  const float* gains = AL ? a.w : s_w;
  Kept<R, AL, NV> kept;
  kept.fill(gains, lane, a.D);
  const long long step = static_cast<long long>(gridDim.x) * ROWS;
  const Bounds bx = bounds_of<T>(a.x, a.T, a.xs, a.D), br = bounds_of<T>(a.r, a.T, a.rs, a.D);
  uint4 ux[NV], ur[NV];
  auto fetch = [&](long long t) {
    const T *x = static_cast<const T*>(a.x) + t * a.xs, *r = static_cast<const T*>(a.r) + t * a.rs;
    const int D = t < a.T ? a.D : 0;  // a row past the end holds no elements
    R::fetch(x, bx, lane, R::offset(x), true, D, ux);
    if (a.r) R::fetch(r, br, lane, R::offset(x), same.a, D, ur);
  };
  fetch(static_cast<long long>(blockIdx.x) * ROWS + group);
  for (long long base = static_cast<long long>(blockIdx.x) * ROWS; base < a.T; base += step) {
    const long long t = base + group;
    const int D = t < a.T ? a.D : 0;
    const T *x = static_cast<const T*>(a.x) + t * a.xs, *r = static_cast<const T*>(a.r) + t * a.rs;
    const int off = R::offset(x);
    const Places<V> places(off, a.D);
    float h[NV][V];
    float sq = 0.f, top = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      R::values(x, bx, lane, k, off, true, D, ux[k], h[k]);
      if (a.r) {
        float f[V];
        R::values(r, br, lane, k, off, same.a, D, ur[k], f);
#pragma unroll
        for (int j = 0; j < V; ++j) h[k][j] += f[j];
        if (a.h) R::store(static_cast<T*>(a.h) + t * a.hs, lane, k, off, same.b, D, h[k]);
      }
    }
    fetch(t + step);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float w[V];
      kept.get(gains, places, lane, k, off, a.D, w);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        sq += h[k][j] * h[k][j];
        h[k][j] *= w[j];
        if (Q8) top = __uint_as_float(max(__float_as_uint(top), __float_as_uint(magnitude(h[k][j]))));
      }
    }
    row_reduce<TPR, true>(sq, top);
    const float rstd = rsqrtf(sq * inv_d + a.eps);
    const float lift = Q8 && top < TINY ? LIFT : 1.f;
    const float f = Q8 ? to_e4m3_range(top, lift) : rstd;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int j = 0; j < V; ++j) h[k][j] = Q8 ? h[k][j] * lift * f : h[k][j] * f;
      if constexpr (Q8)
        R::store_e4m3(static_cast<uint8_t*>(a.y) + t * a.ys, lane, k, off, same.c, D, h[k]);
      else
        R::store(static_cast<T*>(a.y) + t * a.ys, lane, k, off, same.c, D, h[k]);
    }
    if (Q8 && lane == 0 && t < a.T) a.scale[t] = top * rstd * (1.f / E4M3_MAX);
  }
  if (!short_launch) pdl_trigger();
}

// Rows too long for the registers: a CTA a row, read twice (the second time from L2).  Element loads.
template <typename T, bool Q8>
__global__ void __launch_bounds__(LONG_THREADS) k_rms_long(const Forward a) {
  pdl_wait();
  for (long long t = blockIdx.x; t < a.T; t += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + t * a.xs;
    const T* r = static_cast<const T*>(a.r) + t * a.rs;
    float sq = 0.f, top = 0.f;
    for (int e = threadIdx.x; e < a.D; e += LONG_THREADS) {
      const float h = Io<T>::get(x, e) + (a.r ? Io<T>::get(r, e) : 0.f);
      sq += h * h;
      if (Q8) top = __uint_as_float(max(__float_as_uint(top), __float_as_uint(magnitude(h * __ldg(a.w + e)))));
    }
    row_reduce<LONG_THREADS, true>(sq, top);
    const float rstd = rsqrtf(sq / static_cast<float>(a.D) + a.eps);
    const float lift = Q8 && top < TINY ? LIFT : 1.f;
    const float f = Q8 ? to_e4m3_range(top, lift) : rstd;
    for (int e = threadIdx.x; e < a.D; e += LONG_THREADS) {
      const float h = Io<T>::get(x, e) + (a.r ? Io<T>::get(r, e) : 0.f);
      if (a.r && a.h) Io<T>::put(static_cast<T*>(a.h) + t * a.hs, e, h);
      const float v = h * __ldg(a.w + e) * lift * f;
      if constexpr (Q8)
        (static_cast<uint8_t*>(a.y) + t * a.ys)[e] = __nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3);
      else
        Io<T>::put(static_cast<T*>(a.y) + t * a.ys, e, v);
    }
    if (Q8 && threadIdx.x == 0) a.scale[t] = top * rstd * (1.f / E4M3_MAX);
  }
  pdl_trigger();
}

// dx, and this CTA's partial row of dw: part[blockIdx.x][0 .. D).  Aligned rows: a thread's columns are the same in every row,
// their sums stay in its registers.  Unaligned ones: in shared memory, one set for each of the CTA's row groups (dynamic).
template <typename T, bool AL, int TPR, int NV>
__global__ void __launch_bounds__(BLOCK_OF<TPR>) k_rms_bwd(const Backward a, const Same same) {
  constexpr int V = Io<T>::V, BLOCK = BLOCK_OF<TPR>, ROWS = BLOCK / TPR;
  using R = Row<T, AL, TPR>;
  extern __shared__ float s_acc[];  // unaligned rows: the sums, then the gains
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const float inv_d = 1.f / static_cast<float>(a.D);
  float acc[AL ? NV : 1][V] = {};
  const int set = V * slots_of<V>(a.D);
  float* mine = s_acc + (AL ? 0 : group * set);
  if constexpr (!AL) {
    for (int i = lane; i < set; i += TPR) mine[i] = 0.f;
  }
  float* s_w = s_acc + ROWS * set;
  pdl_wait();
  if constexpr (!AL) {
    gains_to_shared<V, BLOCK>(s_w, a.w, a.D);
    __syncthreads();
  }
  const float* gains = AL ? a.w : s_w;
  Kept<R, AL, NV> kept;
  kept.fill(gains, lane, a.D);
  const long long step = static_cast<long long>(gridDim.x) * ROWS;
  const Bounds bh = bounds_of<T>(a.h, a.T, a.hs, a.D), bd = bounds_of<T>(a.dy, a.T, a.ys, a.D), bg = bounds_of<T>(a.dh, a.T, a.ds, a.D);
  uint4 uh[NV], ud[NV];
  auto fetch = [&](long long t) {
    const T *hp = static_cast<const T*>(a.h) + t * a.hs, *dp = static_cast<const T*>(a.dy) + t * a.ys;
    const int D = t < a.T ? a.D : 0;
    R::fetch(hp, bh, lane, R::offset(hp), true, D, uh);
    R::fetch(dp, bd, lane, R::offset(hp), same.a, D, ud);
  };
  fetch(static_cast<long long>(blockIdx.x) * ROWS + group);
  for (long long base = static_cast<long long>(blockIdx.x) * ROWS; base < a.T; base += step) {
    const long long t = base + group;
    const int D = t < a.T ? a.D : 0;
    float h[NV][V], d[NV][V];
    float sq = 0.f, ah = 0.f;
    const T *hp = static_cast<const T*>(a.h) + t * a.hs, *dp = static_cast<const T*>(a.dy) + t * a.ys;
    const int off = R::offset(hp);
    const Places<V> places(off, a.D);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      R::values(hp, bh, lane, k, off, true, D, uh[k], h[k]);
      R::values(dp, bd, lane, k, off, same.a, D, ud[k], d[k]);
    }
    uint4 ug[NV];
    const T* gp = static_cast<const T*>(a.dh) + t * a.ds;
    if (a.dh) R::fetch(gp, bg, lane, off, same.b, D, ug);
    fetch(t + step);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float w[V];
      kept.get(gains, places, lane, k, off, a.D, w);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        sq += h[k][j] * h[k][j];
        ah += d[k][j] * w[j] * h[k][j];
      }
    }
    row_reduce<TPR, false>(sq, ah);  // (more than a warp a row: a barrier, behind which the last row's columns are added)
    if constexpr (!AL && TPR <= 32) __syncwarp();
    const float rstd = t < a.T ? rsqrtf(sq * inv_d + a.eps) : 0.f;  // (a row past the end adds nothing to dw, with eps = 0 either)
    const float c = rstd * rstd * rstd * (ah * inv_d);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float w[V], o[V] = {};
      kept.get(gains, places, lane, k, off, a.D, w);
      if (a.dh) R::values(gp, bg, lane, k, off, same.b, D, ug[k], o);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float g = d[k][j] * (h[k][j] * rstd);
        if constexpr (AL) {
          acc[k][j] += g;
        } else {
          if (R::at(lane, k) - off < D) mine[places.at[j] + lane + TPR * k] += g;
        }
        o[j] += rstd * (d[k][j] * w[j]) - c * h[k][j];
      }
      R::store(static_cast<T*>(a.dx) + t * a.xs, lane, k, off, same.c, D, o);
    }
  }
  // the CTA's row groups hold the same columns: added in ascending group order
  float* part = static_cast<float*>(a.ws) + static_cast<long long>(blockIdx.x) * a.D;
  if constexpr (!AL) {
    __syncthreads();
    for (int e = threadIdx.x; e < a.D; e += BLOCK) {
      const float* s = s_acc + column_at<V>(e, a.D);
      float sum = s[0];
#pragma unroll 4
      for (int g = 1; g < ROWS; ++g) sum += s[g * set];
      part[e] = sum;
    }
  } else if constexpr (ROWS == 1) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (R::at(lane, k) + j < a.D) part[R::at(lane, k) + j] = acc[k][j];
  } else {
    __shared__ float s[ROWS][TPR][V + 1];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < V; ++j) s[group][lane][j] = acc[k][j];
      __syncthreads();
      for (int i = threadIdx.x; i < TPR * V; i += BLOCK) {
        const int l = i / V, j = i % V;
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < ROWS; ++g) sum += s[g][l][j];
        if (R::at(l, k) + j < a.D) part[R::at(l, k) + j] = sum;
      }
    }
  }
  pdl_trigger();
}

// Rows too long for the registers: dx (DX) by a CTA a row; coef[t] = rstd for k_dw_long.
template <typename T, bool DX>
__global__ void __launch_bounds__(LONG_THREADS) k_rms_bwd_long(const Backward a, float* __restrict__ coef) {
  pdl_wait();
  for (long long t = blockIdx.x; t < a.T; t += gridDim.x) {
    const T* h = static_cast<const T*>(a.h) + t * a.hs;
    const T* dy = static_cast<const T*>(a.dy) + t * a.ys;
    float sq = 0.f, ah = 0.f;
    for (int e = threadIdx.x; e < a.D; e += LONG_THREADS) {
      const float v = Io<T>::get(h, e);
      sq += v * v;
      ah += Io<T>::get(dy, e) * __ldg(a.w + e) * v;
    }
    row_reduce<LONG_THREADS, false>(sq, ah);
    const float inv_d = 1.f / static_cast<float>(a.D), rstd = rsqrtf(sq * inv_d + a.eps);
    const float c = rstd * rstd * rstd * (ah * inv_d);
    if constexpr (DX) {
      for (int e = threadIdx.x; e < a.D; e += LONG_THREADS) {
        float o = a.dh ? Io<T>::get(static_cast<const T*>(a.dh) + t * a.ds, e) : 0.f;
        o += rstd * (Io<T>::get(dy, e) * __ldg(a.w + e)) - c * Io<T>::get(h, e);
        Io<T>::put(static_cast<T*>(a.dx) + t * a.xs, e, o);
      }
    }
    if (threadIdx.x == 0) coef[t] = rstd;
  }
  pdl_trigger();
}
// part[blockIdx.y][e] = sum over the rows of chunk blockIdx.y of dy h rstd
template <typename T>
__global__ void __launch_bounds__(256) k_dw_long(const Backward a, const float* coef, int chunks) {
  pdl_wait();
  const int e = blockIdx.x * 256 + threadIdx.x;
  const long long t0 = a.T * blockIdx.y / chunks, t1 = a.T * (blockIdx.y + 1) / chunks;
  float sum = 0.f;
  if (e < a.D) {
    for (long long t = t0; t < t1; ++t)
      sum += Io<T>::get(static_cast<const T*>(a.dy) + t * a.ys, e) * (Io<T>::get(static_cast<const T*>(a.h) + t * a.hs, e) * coef[t]);
    (static_cast<float*>(a.ws) + static_cast<long long>(blockIdx.y) * a.D)[e] = sum;
  }
  pdl_trigger();
}

// dw[e] = the sum of `parts` partial rows: 32 runs of consecutive rows, each in ascending order, then the run sums in
// ascending order.  A CTA takes 32 columns.
constexpr int DW_RUNS = 32;
__global__ void __launch_bounds__(32 * DW_RUNS) k_dw(const float* part, float* __restrict__ dw, int D, int parts) {
  __shared__ float s[DW_RUNS][33];
  pdl_wait();
  const int lane = threadIdx.x & 31, g = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
  const int p0 = parts * g / DW_RUNS, p1 = parts * (g + 1) / DW_RUNS;
  float sum = 0.f;
  if (e < D) {
    int p = p0;
    for (; p + 8 <= p1; p += 8) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = __ldcg(part + static_cast<long long>(p + u) * D + e);
#pragma unroll
      for (int u = 0; u < 8; ++u) sum += v[u];
    }
    for (; p < p1; ++p) sum += __ldcg(part + static_cast<long long>(p) * D + e);
  }
  s[g][lane] = sum;
  __syncthreads();
  if (g == 0 && e < D) {
    float total = s[0][lane];
#pragma unroll
    for (int i = 1; i < DW_RUNS; ++i) total += s[i][lane];
    dw[e] = total;
  }
  pdl_trigger();
}

// ---- contiguous rows of an odd length ----
// V rows of a contiguous matrix (V elements in 16 bytes) are D whole vectors: a CTA takes them as they lie, thread v vectors v,
// v + BLOCK, ..  A vector holds elements of one row or, cut, of two (D >= V); its row, its cut and its gains are the same in every
// group, the gains in shared memory in the vectors' order.  Each vector leaves the sums of its part of one row and of the next one in
// shared memory, a warp adds a row's up.  Measured against the rows' own kernels (above), us: [21680, 177] bf16 with a residual 15.9
// and 7.5 (floor 4.5), its backward 21.4 and 15.9; [1300, 177] 3.4 and 2.8.  As many warps as rows at least: with six for 177 vectors
// it took 9.3.
template <typename T>
struct Flat {
  static constexpr int V = Io<T>::V;
  static __device__ __forceinline__ void gains(float* s, const float* w, int D) {
    for (int i = threadIdx.x; i < V * D; i += blockDim.x) s[(((i % V) >> 2) * D + i / V) * 4 + (i & 3)] = __ldg(w + i % D);
  }
  static __device__ __forceinline__ void gain(const float* s, int v, int D, float (&f)[V]) {
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
      const float4 u = reinterpret_cast<const float4*>(s)[q * D + v];
      f[4 * q] = u.x, f[4 * q + 1] = u.y, f[4 * q + 2] = u.z, f[4 * q + 3] = u.w;
    }
  }
  // elements e .. e + V - 1 of the group at p, those from n on zero
  static __device__ __forceinline__ uint4 load(const T* p, int e, int n) {
    if (e + V <= n) return *reinterpret_cast<const uint4*>(p + e);
    float f[V] = {};
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (e + j < n) f[j] = Io<T>::get(p, e + j);
    return Io<T>::pack(f);
  }
  static __device__ __forceinline__ void store(T* p, int e, int n, const float (&f)[V]) {
    if (e + V <= n) {
      *reinterpret_cast<uint4*>(p + e) = Io<T>::pack(f);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (e + j < n) Io<T>::put(p, e + j, f[j]);
    }
  }
  // row r's sum of the vectors' first parts, by one warp; the same value in each lane
  static __device__ __forceinline__ float row_sum(const float* first, int r, int D) {
    float sum = 0.f;
    const int end = ((r + 1) * D + V - 1) / V;
    for (int v = (r * D + V - 1) / V + (threadIdx.x & 31); v < end; v += 32) sum += first[v];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return sum;
  }
};

template <typename T, int BLOCK, int NV>
__global__ void __launch_bounds__(BLOCK) k_rms_flat(const Forward a) {
  using F = Flat<T>;
  constexpr int V = F::V;
  extern __shared__ __align__(16) float s_w[];  // the gains, then the vectors' sums
  __shared__ float s_second[V], s_rstd[V];
  const int D = a.D, warp = threadIdx.x >> 5;
  const float inv_d = 1.f / static_cast<float>(D);
  float* s_first = s_w + V * D;
  int row[NV], cut[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int e = V * (static_cast<int>(threadIdx.x) + BLOCK * k);
    row[k] = e / D;
    cut[k] = min(V, (row[k] + 1) * D - e);
  }
  if (threadIdx.x < V) s_second[threadIdx.x] = 0.f;
  pdl_wait();
  F::gains(s_w, a.w, D);
  __syncthreads();
  const long long groups = (a.T + V - 1) / V;
  auto elements = [&](long long g) { return static_cast<int>(min(static_cast<long long>(V), a.T - g * V)) * D; };
  uint4 ux[NV], ur[NV];
  auto fetch = [&](long long g) {
    if (g >= groups) return;
    const int n = elements(g);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int e = V * (static_cast<int>(threadIdx.x) + BLOCK * k);
      if (e >= V * D) continue;
      ux[k] = F::load(static_cast<const T*>(a.x) + g * V * D, e, n);
      if (a.r) ur[k] = F::load(static_cast<const T*>(a.r) + g * V * D, e, n);
    }
  };
  fetch(blockIdx.x);
  for (long long g = blockIdx.x; g < groups; g += gridDim.x) {
    const int n = elements(g);
    float h[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = threadIdx.x + BLOCK * k;
      if (v >= D) continue;
      Io<T>::unpack(ux[k], h[k]);
      if (a.r) {
        float f[V];
        Io<T>::unpack(ur[k], f);
#pragma unroll
        for (int j = 0; j < V; ++j) h[k][j] += f[j];
        if (a.h) F::store(static_cast<T*>(a.h) + g * V * D, V * v, n, h[k]);
      }
      float first = 0.f, second = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float s = h[k][j] * h[k][j];
        if (j < cut[k]) first += s; else second += s;
      }
      s_first[v] = first;
      if (cut[k] < V) s_second[row[k] + 1] = second;
    }
    fetch(g + gridDim.x);
    __syncthreads();
    for (int r = warp; r < V; r += BLOCK / 32) {
      const float sum = F::row_sum(s_first, r, D) + s_second[r];
      if ((threadIdx.x & 31) == 0) s_rstd[r] = rsqrtf(sum * inv_d + a.eps);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = threadIdx.x + BLOCK * k;
      if (v >= D) continue;
      const float ra = s_rstd[row[k]], rb = s_rstd[min(row[k] + 1, V - 1)];
      float w[V];
      F::gain(s_w, v, D, w);
#pragma unroll
      for (int j = 0; j < V; ++j) h[k][j] = h[k][j] * w[j] * (j < cut[k] ? ra : rb);
      F::store(static_cast<T*>(a.y) + g * V * D, V * v, n, h[k]);
    }
  }
  pdl_trigger();
}

// dw: a thread's places in the group have the same columns in every group, their sums stay in its registers; at the end the V
// rows' sums of a column are added in ascending order.
template <typename T, int BLOCK>
__global__ void __launch_bounds__(BLOCK) k_rms_bwd_flat(const Backward a) {
  using F = Flat<T>;
  constexpr int V = F::V, NV = 1;
  extern __shared__ __align__(16) float s_w[];  // the gains (at the end the columns' sums), then the vectors' two sums
  __shared__ float s_second[2][V], s_rstd[V], s_c[V];
  const int D = a.D, warp = threadIdx.x >> 5;
  const float inv_d = 1.f / static_cast<float>(D);
  float *s_sq = s_w + V * D, *s_ah = s_sq + D;
  int row[NV], cut[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int e = V * (static_cast<int>(threadIdx.x) + BLOCK * k);
    row[k] = e / D;
    cut[k] = min(V, (row[k] + 1) * D - e);
  }
  if (threadIdx.x < V) s_second[0][threadIdx.x] = s_second[1][threadIdx.x] = 0.f;
  pdl_wait();
  F::gains(s_w, a.w, D);
  __syncthreads();
  const long long groups = (a.T + V - 1) / V;
  auto elements = [&](long long g) { return static_cast<int>(min(static_cast<long long>(V), a.T - g * V)) * D; };
  float acc[NV][V] = {};
  uint4 uh[NV], ud[NV];
  auto fetch = [&](long long g) {
    if (g >= groups) return;
    const int n = elements(g);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int e = V * (static_cast<int>(threadIdx.x) + BLOCK * k);
      if (e >= V * D) continue;
      uh[k] = F::load(static_cast<const T*>(a.h) + g * V * D, e, n);
      ud[k] = F::load(static_cast<const T*>(a.dy) + g * V * D, e, n);
    }
  };
  fetch(blockIdx.x);
  for (long long g = blockIdx.x; g < groups; g += gridDim.x) {
    const int n = elements(g);
    float h[NV][V], d[NV][V];
    uint4 ug[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = threadIdx.x + BLOCK * k;
      if (v >= D) continue;
      Io<T>::unpack(uh[k], h[k]);
      Io<T>::unpack(ud[k], d[k]);
      if (a.dh) ug[k] = F::load(static_cast<const T*>(a.dh) + g * V * D, V * v, n);
    }
    fetch(g + gridDim.x);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = threadIdx.x + BLOCK * k;
      if (v >= D) continue;
      float w[V], sq[2] = {}, ah[2] = {};
      F::gain(s_w, v, D, w);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float s = h[k][j] * h[k][j], t = d[k][j] * w[j] * h[k][j];
        if (j < cut[k]) sq[0] += s, ah[0] += t; else sq[1] += s, ah[1] += t;
      }
      s_sq[v] = sq[0], s_ah[v] = ah[0];
      if (cut[k] < V) s_second[0][row[k] + 1] = sq[1], s_second[1][row[k] + 1] = ah[1];
    }
    __syncthreads();
    for (int r = warp; r < V; r += BLOCK / 32) {
      const float sq = F::row_sum(s_sq, r, D) + s_second[0][r], ah = F::row_sum(s_ah, r, D) + s_second[1][r];
      const float rstd = r * D < n ? rsqrtf(sq * inv_d + a.eps) : 0.f;  // (a row past the end adds nothing to dw)
      if ((threadIdx.x & 31) == 0) s_rstd[r] = rstd, s_c[r] = rstd * rstd * rstd * (ah * inv_d);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = threadIdx.x + BLOCK * k;
      if (v >= D) continue;
      const int next = min(row[k] + 1, V - 1);
      const float ra = s_rstd[row[k]], rb = s_rstd[next], ca = s_c[row[k]], cb = s_c[next];
      float w[V], o[V] = {};
      F::gain(s_w, v, D, w);
      if (a.dh) Io<T>::unpack(ug[k], o);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float rstd = j < cut[k] ? ra : rb, c = j < cut[k] ? ca : cb;
        acc[k][j] += d[k][j] * (h[k][j] * rstd);
        o[j] += rstd * (d[k][j] * w[j]) - c * h[k][j];
      }
      F::store(static_cast<T*>(a.dx) + g * V * D, V * v, n, o);
    }
  }
  __syncthreads();  // the gains have been read
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = threadIdx.x + BLOCK * k;
    if (v >= D) continue;
#pragma unroll
    for (int j = 0; j < V; ++j) s_w[V * v + j] = acc[k][j];
  }
  __syncthreads();
  float* part = static_cast<float*>(a.ws) + static_cast<long long>(blockIdx.x) * D;
  for (int e = threadIdx.x; e < D; e += BLOCK) {
    float sum = s_w[e];
#pragma unroll
    for (int r = 1; r < V; ++r) sum += s_w[r * D + e];
    part[e] = sum;
  }
  pdl_trigger();
}

// ---- host ----

// Threads a row and vectors a thread for rows of n vectors: at most 128 vectors stay within a warp (no shared memory).  Few rows
// (fewer than SMs) take more threads each: a row's latency is the call's.
template <class F>
cudaError_t by_length(int n, bool few, F&& f) {
#define WHTMIX_ROW(TPR, NV) f(std::integral_constant<int, TPR>(), std::integral_constant<int, NV>())
  if (n <= 8) return WHTMIX_ROW(8, 1);
  if (n <= 16) return WHTMIX_ROW(16, 1);
  if (n <= 32) return WHTMIX_ROW(32, 1);
  if (few) {
    if (n <= 128) return WHTMIX_ROW(128, 1);
    if (n <= 512) return WHTMIX_ROW(512, 1);
  }
  if (n <= 64) return WHTMIX_ROW(32, 2);
  if (n <= 128) return WHTMIX_ROW(32, 4);
  if (n <= 256) return WHTMIX_ROW(128, 2);
  if (n <= 384) return WHTMIX_ROW(128, 3);
  if (n <= 512) return WHTMIX_ROW(256, 2);
  if (n <= 768) return WHTMIX_ROW(256, 3);
  if (n <= 1024) return WHTMIX_ROW(256, 4);
  if (n <= 1536) return WHTMIX_ROW(512, 3);
  return WHTMIX_ROW(512, 4);
}
// The backward's: more registers a vector (its sums and two inputs), so one a thread up to 512 vectors.
template <class F>
cudaError_t by_length_backward(int n, F&& f) {
  if (n <= 8) return WHTMIX_ROW(8, 1);
  if (n <= 16) return WHTMIX_ROW(16, 1);
  if (n <= 32) return WHTMIX_ROW(32, 1);
  if (n <= 64) return WHTMIX_ROW(32, 2);
  if (n <= 128) return WHTMIX_ROW(128, 1);
  if (n <= 256) return WHTMIX_ROW(256, 1);
  if (n <= 512) return WHTMIX_ROW(512, 1);
  if (n <= 1024) return WHTMIX_ROW(512, 2);
  if (n <= 1536) return WHTMIX_ROW(512, 3);
  return WHTMIX_ROW(512, 4);
#undef WHTMIX_ROW
}

// 16-byte vectors of a row; an unaligned one may touch one more
int vectors(int D, bool bf16, bool al) {
  const int v = bf16 ? 8 : 4;
  return (D + v - 1) / v + (al ? 0 : 1);
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// rows of `es`-byte elements at p, `stride` elements apart, all start on a 16-byte boundary
bool rows_aligned(const void* p, long long stride, size_t es, size_t to = 16) {
  return !p || (aligned(p, to) && (static_cast<unsigned long long>(stride) * es) % to == 0);
}

// rows q lie like rows p: the same distance from a 16-byte boundary, row for row
bool rows_same(const void* p, long long ps, const void* q, long long qs, size_t es) {
  return !q || (((reinterpret_cast<uintptr_t>(p) - reinterpret_cast<uintptr_t>(q)) & 15u) == 0 && (ps - qs) * static_cast<long long>(es) % 16 == 0);
}

// CTAs for T rows, `rows` at a time: at most as many as are resident at once, so that each takes its even share (with four
// times the SMs where three fit, a backward of 131072 rows of 256 took 66 us).
unsigned grid_rows(long long T, int rows, int resident) {
  const long long need = (T + rows - 1) / rows;
  return static_cast<unsigned>(need < resident ? need : resident);
}
// Resident CTAs of a kernel on the whole device, asked once for each kernel and size.  Its shared-memory limit, which belongs to the
// kernel and not to a size, is raised first and never lowered: calls of other widths, on other threads too, go on under it.
cudaError_t resident_ctas(const void* kernel, int block, size_t smem, int sms, int* out) {
  static std::mutex mu;
  static std::map<std::tuple<int, const void*, size_t>, int> known;
  static std::map<std::pair<int, const void*>, size_t> limits;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  std::lock_guard<std::mutex> lock(mu);
  int& n = known[{dev, kernel, smem}];
  if (n == 0) {
    size_t& limit = limits[{dev, kernel}];
    if (limit == 0) {  // until it is raised: 48 KB less what the kernel declares itself
      cudaFuncAttributes own;
      if ((e = cudaFuncGetAttributes(&own, kernel)) != cudaSuccess) return e;
      limit = 48 * 1024 - own.sharedSizeBytes;
    }
    if (smem > limit) {
      if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem))) != cudaSuccess) return e;
      limit = smem;
    }
    int per_sm = 0;
    if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, block, smem)) != cudaSuccess) return e;
    if (per_sm < 1) return cudaErrorLaunchOutOfResources;
    n = per_sm * sms;
  }
  *out = n;
  return cudaSuccess;
}

template <int N>
using Int = std::integral_constant<int, N>;
// The longest rows that go this way.  Row kernels and these, us: forward [20000, 1001] bf16 40.1 and 32.1, [5200, 1001] f32 16.6 and
// 17.7; backward [21680, 177] bf16 21.4 and 15.8, [20000, 333] f32 42.3 and 49.8, [20000, 500] bf16 29.7 and 35.7.
template <typename T>
constexpr int FLAT_FORWARD = 2048 / sizeof(T);
constexpr int FLAT_BACKWARD = 256;
// A contiguous matrix of odd rows and enough groups of them, every matrix on a 16-byte boundary: k_rms_flat's and k_rms_bwd_flat's.
template <typename T>
bool flat(long long T_, int D, int most, int sms) {
  constexpr int V = Io<T>::V;
  return D % V != 0 && D >= V && D <= most && T_ >= static_cast<long long>(V) * (D > 512 ? 2 * sms : sms);
}
bool contiguous(const void* p, long long stride, int D) { return !p || (stride == D && aligned(p, 16)); }
template <typename T, bool Q8>
cudaError_t forward_t(const Forward& a, int sms, cudaStream_t stream) {
  constexpr int V = Io<T>::V;
  const size_t es = sizeof(T);
  const bool al = a.D % V == 0 && aligned(a.w, 16) && rows_aligned(a.x, a.xs, es) && rows_aligned(a.r, a.rs, es) &&
                  rows_aligned(a.r ? a.h : nullptr, a.hs, es) && (Q8 ? rows_aligned(a.y, a.ys, 1, V) : rows_aligned(a.y, a.ys, es));
  const int n = vectors(a.D, es == 2, al);
  Forward c = a;
  if constexpr (!Q8) {
    if (flat<T>(a.T, a.D, FLAT_FORWARD<T>, sms) && contiguous(a.x, a.xs, a.D) && contiguous(a.r, a.rs, a.D) &&
        contiguous(a.r ? a.h : nullptr, a.hs, a.D) && contiguous(a.y, a.ys, a.D)) {
      const void* k = nullptr;
      int block = 0;
      auto take = [&](auto threads, auto nv) {
        block = decltype(threads)::value;
        k = reinterpret_cast<const void*>(k_rms_flat<T, decltype(threads)::value, decltype(nv)::value>);
      };
      if (a.D <= 64) take(Int<64>(), Int<1>());
      else if (a.D <= 128) take(Int<128>(), Int<1>());
      else if (a.D <= 256) take(Int<256>(), Int<1>());
      else if (a.D <= 512) take(Int<256>(), Int<2>());
      else if constexpr (FLAT_FORWARD<T> > 512) take(Int<512>(), Int<2>());
      const size_t smem = static_cast<size_t>(V + 1) * a.D * 4;  // at most 36 KB
      int resident = 0;
      const cudaError_t e = resident_ctas(k, block, smem, sms, &resident);
      if (e != cudaSuccess) return e;
      void* args[] = {&c};
      return launch_pdl(k, grid_rows(a.T, V, resident), block, smem, stream, args);
    }
  }
  if (n > MAX_VECTORS) {
    void* args[] = {&c};
    return launch_pdl(reinterpret_cast<const void*>(k_rms_long<T, Q8>), grid_rows(a.T, 1, 4 * sms), LONG_THREADS, 0, stream, args);
  }
  // (8 bits: a vector's V bytes start on a multiple of V)
  const bool same_y = Q8 ? (reinterpret_cast<uintptr_t>(a.y) - reinterpret_cast<uintptr_t>(a.x) / es) % V == 0 && (a.ys - a.xs) % V == 0
                         : rows_same(a.x, a.xs, a.y, a.ys, es);
  Same same{rows_same(a.x, a.xs, a.r, a.rs, es), rows_same(a.x, a.xs, a.r ? a.h : nullptr, a.hs, es), same_y};
  return by_length(n, a.T < sms, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, BLOCK = BLOCK_OF<TPR>;
    const void* k = al ? reinterpret_cast<const void*>(k_rms<T, Q8, true, TPR, NV>)
                       : reinterpret_cast<const void*>(k_rms<T, Q8, false, TPR, NV>);
    void* args[] = {&c, &same};
    const size_t smem = al ? 0 : static_cast<size_t>(V) * slots_of<V>(a.D) * 4;  // at most 64 KB
    int resident = 0;
    const cudaError_t e = resident_ctas(k, BLOCK, smem, sms, &resident);
    if (e != cudaSuccess) return e;
    return launch_pdl(k, grid_rows(a.T, BLOCK / TPR, resident), BLOCK, smem, stream, args);
  });
}

cudaError_t forward(const Forward& a, bool bf16, bool to_e4m3, int sms, cudaStream_t stream) {
  if (a.T <= 0) return cudaSuccess;
  if (bf16) return to_e4m3 ? forward_t<__nv_bfloat16, true>(a, sms, stream) : forward_t<__nv_bfloat16, false>(a, sms, stream);
  return to_e4m3 ? forward_t<float, true>(a, sms, stream) : forward_t<float, false>(a, sms, stream);
}

// Chunks of rows of k_dw_long.
int long_parts(long long T) { return static_cast<int>(T < 64 ? T : 64); }

template <typename T>
bool backward_aligned(const Backward& a) {
  const size_t es = sizeof(T);
  return a.D % Io<T>::V == 0 && aligned(a.w, 16) && rows_aligned(a.h, a.hs, es) && rows_aligned(a.dy, a.ys, es) &&
         rows_aligned(a.dh, a.ds, es) && rows_aligned(a.dx, a.xs, es);
}

// A call's kernel, its shared memory and its CTAs, each of which leaves a partial row of dw.
struct BackwardPlan {
  const void* kernel;
  size_t smem;
  int block, parts;
};
template <typename T>
cudaError_t backward_plan(const Backward& a, int n, bool al, int sms, BackwardPlan* p) {
  if (flat<T>(a.T, a.D, FLAT_BACKWARD, sms) && contiguous(a.h, a.hs, a.D) && contiguous(a.dy, a.ys, a.D) && contiguous(a.dh, a.ds, a.D) &&
      contiguous(a.dx, a.xs, a.D)) {
    constexpr int V = Io<T>::V;
    p->kernel = a.D <= 64    ? reinterpret_cast<const void*>(k_rms_bwd_flat<T, 64>)
                : a.D <= 128 ? reinterpret_cast<const void*>(k_rms_bwd_flat<T, 128>)
                             : reinterpret_cast<const void*>(k_rms_bwd_flat<T, 256>);
    p->block = a.D <= 64 ? 64 : a.D <= 128 ? 128 : 256;
    p->smem = static_cast<size_t>(V + 2) * a.D * 4;
    int resident = 0;
    const cudaError_t e = resident_ctas(p->kernel, p->block, p->smem, sms, &resident);
    if (e == cudaSuccess) p->parts = static_cast<int>(grid_rows(a.T, V, resident));
    return e;
  }
  return by_length_backward(n, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, BLOCK = BLOCK_OF<TPR>;
    p->kernel = al ? reinterpret_cast<const void*>(k_rms_bwd<T, true, TPR, NV>) : reinterpret_cast<const void*>(k_rms_bwd<T, false, TPR, NV>);
    p->smem = al ? 0 : static_cast<size_t>(BLOCK / TPR + 1) * Io<T>::V * slots_of<Io<T>::V>(a.D) * 4;  // at most 129 KB
    p->block = BLOCK;
    int resident = 0;
    const cudaError_t e = resident_ctas(p->kernel, BLOCK, p->smem, sms, &resident);
    if (e == cudaSuccess) p->parts = static_cast<int>(grid_rows(a.T, BLOCK / TPR, resident));
    return e;
  });
}

template <typename T>
static cudaError_t workspace_t(const Backward& a, int sms, size_t* bytes) {
  const bool al = backward_aligned<T>(a);
  const int n = vectors(a.D, sizeof(T) == 2, al);
  if (n > MAX_VECTORS) {
    *bytes = static_cast<size_t>(long_parts(a.T)) * a.D * 4 + static_cast<size_t>(a.T) * 4;
    return cudaSuccess;
  }
  BackwardPlan p;
  const cudaError_t e = backward_plan<T>(a, n, al, sms, &p);
  if (e == cudaSuccess) *bytes = static_cast<size_t>(p.parts) * a.D * 4;
  return e;
}
cudaError_t backward_workspace(const Backward& a, bool bf16, int sms, size_t* bytes) {
  return bf16 ? workspace_t<__nv_bfloat16>(a, sms, bytes) : workspace_t<float>(a, sms, bytes);
}

cudaError_t add_rows(const float* part, float* out, int D, int parts, cudaStream_t stream) {
  void* args[] = {&part, &out, &D, &parts};
  return launch_pdl(reinterpret_cast<const void*>(k_dw), static_cast<unsigned>((D + 31) / 32), 32 * DW_RUNS, 0, stream, args);
}

template <typename T>
cudaError_t backward_t(const Backward& a, int sms, cudaStream_t stream) {
  const size_t es = sizeof(T);
  const bool al = backward_aligned<T>(a);
  const int n = vectors(a.D, es == 2, al);
  int parts = long_parts(a.T);
  Backward c = a;
  cudaError_t e;
  if (n > MAX_VECTORS) {
    float* coef = static_cast<float*>(a.ws) + static_cast<size_t>(parts) * a.D;
    // dw reads dy: where dx takes dy's place, the coefficients alone come first and dx last.  [1000, 20001] bf16, us: 96, and 71 where
    // dx is another matrix; with dx written by the threads that add up a column's dw both took 139.
    const bool over_dy = a.dx == a.dy;
    const void *with_dx = reinterpret_cast<const void*>(k_rms_bwd_long<T, true>), *without = reinterpret_cast<const void*>(k_rms_bwd_long<T, false>);
    void* args[] = {&c, &coef};
    auto rows = [&](const void* k) { return launch_pdl(k, grid_rows(a.T, 1, 4 * sms), LONG_THREADS, 0, stream, args); };
    if ((e = rows(over_dy ? without : with_dx)) != cudaSuccess) return e;
    k_dw_long<T><<<dim3((a.D + 255) / 256, parts), 256, 0, stream>>>(c, coef, parts);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    if (over_dy) e = rows(with_dx);
  } else {
    Same same{rows_same(a.h, a.hs, a.dy, a.ys, es), rows_same(a.h, a.hs, a.dh, a.ds, es), rows_same(a.h, a.hs, a.dx, a.xs, es)};
    BackwardPlan p;
    if ((e = backward_plan<T>(a, n, al, sms, &p)) != cudaSuccess) return e;
    parts = p.parts;
    void* args[] = {&c, &same};  // (the flat kernel takes the first alone)
    e = launch_pdl(p.kernel, static_cast<unsigned>(parts), p.block, p.smem, stream, args);
  }
  if (e != cudaSuccess) return e;
  return add_rows(static_cast<const float*>(a.ws), a.dw, a.D, parts, stream);
}

cudaError_t backward(const Backward& a, bool bf16, int sms, cudaStream_t stream) {
  return bf16 ? backward_t<__nv_bfloat16>(a, sms, stream) : backward_t<float>(a, sms, stream);
}

}  // namespace norm
}  // namespace whtmix
