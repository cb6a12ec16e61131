// whtmix_rows.cuh -- rows of channels in registers: what the RMS norm's (whtmix_norm.cu) and the layer norm's (whtmix_layer_norm.cu)
// kernels share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <map>
#include <mutex>
#include <tuple>
#include <type_traits>
#include <utility>

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
inline int vectors(int D, bool bf16, bool al) {
  const int v = bf16 ? 8 : 4;
  return (D + v - 1) / v + (al ? 0 : 1);
}

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// rows of `es`-byte elements at p, `stride` elements apart, all start on a 16-byte boundary
inline bool rows_aligned(const void* p, long long stride, size_t es, size_t to = 16) {
  return !p || (aligned(p, to) && (static_cast<unsigned long long>(stride) * es) % to == 0);
}

// rows q lie like rows p: the same distance from a 16-byte boundary, row for row
inline bool rows_same(const void* p, long long ps, const void* q, long long qs, size_t es) {
  return !q || (((reinterpret_cast<uintptr_t>(p) - reinterpret_cast<uintptr_t>(q)) & 15u) == 0 && (ps - qs) * static_cast<long long>(es) % 16 == 0);
}

// CTAs for T rows, `rows` at a time: at most as many as are resident at once, so that each takes its even share (with four
// times the SMs where three fit, a backward of 131072 rows of 256 took 66 us).
inline unsigned grid_rows(long long T, int rows, int resident) {
  const long long need = (T + rows - 1) / rows;
  return static_cast<unsigned>(need < resident ? need : resident);
}
// Resident CTAs of a kernel on the whole device, asked once for each kernel and size.  Its shared-memory limit, which belongs to the
// kernel and not to a size, is raised first and never lowered: calls of other widths, on other threads too, go on under it.
inline cudaError_t resident_ctas(const void* kernel, int block, size_t smem, int sms, int* out) {
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

}  // namespace norm
}  // namespace whtmix
