// whtmix_layer_norm.cu -- layer norm with the residual's addition, its 8-bit output, and its backward.
//
//   h = x + r,  m = mean(h),  c = h - m,  rstd = 1 / sqrt(mean(c^2) + eps),  y = c rstd w + b                one row of D channels
//   8 bits: s = max_d |y_d| / 448,  q_d = e4m3(y_d / s)
//   backward, with n = c rstd and a = dy w:
//     dx = rstd (a - mean(a) - n mean(a n)) + dh,      dw = sum over rows of dy n,      db = sum over rows of dy
//
// Bound by memory: a row is read once into registers (packed as stored) and written once.  The variance is taken from the
// differences to the mean, in a second reduction over the registers: as a difference of two sums it would lose what a mean far from
// zero takes.  Of the backward's sums only the mean stands alone, the other three share a reduction.  Layouts, unaligned rows and
// the sums over rows as whtmix_norm.cu has them (whtmix_rows.cuh), with two sets of column sums; rows beyond the registers are
// read several times, from L2 (k_ln_long, k_ln_bwd_long).
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "whtmix_kernels.cuh"
#include "whtmix_layer_norm.cuh"
#include "whtmix_rows.cuh"
#include "whtmix_tc.cuh"
#include "whtmix_tma.cuh"
#include "whtmix_unaligned.cuh"

namespace whtmix {
namespace norm {

// `bytes` (a multiple of 16) between shared and global memory, both on 16-byte boundaries.
__device__ __forceinline__ void bulk_load(void* s, const void* g, int bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(tc::smem_u32(s)), "l"(g), "r"(bytes), "r"(tc::smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void bulk_store(void* g, const void* s, int bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(g), "r"(tc::smem_u32(s)), "r"(bytes) : "memory");
}

// Finite rows whose sums leave float32's range: where var + eps is not within [1 / FAR, FAR], or no number, the row is taken again with its
// values times a power of two (exact, but for elements too small to count):
//   s h - mean(s h) = s c,     c rstd = s c r,     rstd = s r,     r = 1 / sqrt(mean((s c)^2) + s^2 eps)
// DOWN leaves the squares of 2^24 of float32's largest below 2^122, UP the smallest's above 2^-138.  For a row in range s = 1.  The check is a
// vote and a branch in every row, 0 to 10 % of a kernel's time ([131072, 256] bf16 backward with dh 44.8 -> 45.7 us), 20 % at the most ([64800, 64]
// float32 to 8 bits 8.1 -> 9.8).
constexpr float FAR = 0x1p100f, DOWN = 0x1p-80f, UP = 0x1p80f;
__device__ __forceinline__ bool in_range(float v) { return v >= 1.f / FAR && v <= FAR; }
// s, from var + eps and the mean.  (Equal values of 2^20 and more with an eps below 1 / FAR: c is 0 as it is.)
__device__ __forceinline__ float range_of(float v, float mean) {
  return in_range(v) ? 1.f : v < 1.f / FAR ? fabsf(mean) < 0x1p20f ? UP : 1.f : DOWN;
}
// s^2 eps; DOWN keeps an eps from vanishing, for equal values whose sum was infinite (c = 0; any other c is 1 and more there)
__device__ __forceinline__ float eps_of(float eps, float by) {
  const float e = eps * by * by;
  return by < 1.f && eps > 0.f ? fmaxf(e, 0x1p-90f) : e;
}
// Whether b holds for one of the rows that this one shares a warp with (LANES threads a row; more than a warp: in all of a CTA's it is the
// same): what follows takes all lanes.
template <int LANES>
__device__ __forceinline__ bool any_row(bool b) {
  if constexpr (LANES > 32) return b;
  return __any_sync(0xffffffffu, b);
}
// mean(s h) and r for k_ln_columns.  s rides along in r's sign and, below 1 or above, its size: 2^-50 <= r <= 2^45 with DOWN, 2^-30 <= r with UP.
__device__ __forceinline__ float2 coefficients(float mean, float r, float by) {
  return make_float2(mean, by == 1.f ? r : by < 1.f ? r * -0x1p-60f : r * -0x1p40f);
}

// The sums of a[0 .. N - 1] (MAXB: the largest by its bits) over a row's TPR threads, the same value in each.  STEP numbers a row's
// reductions: each has its own shared memory, so that one barrier a reduction is enough (whoever writes a step's again has passed
// the next step's barrier, behind every read of it; a row has two steps at least).
template <int TPR, int STEP, bool MAXB, int N>
__device__ __forceinline__ void row_join(float (&a)[N]) {
  constexpr int W = TPR < 32 ? TPR : 32;
  auto join = [](float u, float v) { return MAXB ? __uint_as_float(max(__float_as_uint(u), __float_as_uint(v))) : u + v; };
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = join(a[i], __shfl_xor_sync(0xffffffffu, a[i], o));
  if constexpr (TPR > 32) {
    __shared__ float s[N][TPR / 32];
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) s[i][threadIdx.x >> 5] = a[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      a[i] = s[i][0];
#pragma unroll
      for (int j = 1; j < TPR / 32; ++j) a[i] = join(a[i], s[i][j]);
    }
  }
}

// c = h - mean for the elements of vector k, zero for those that are not the row's.
template <typename R, bool AL>
__device__ __forceinline__ void center(const float (&h)[R::V], float (&c)[R::V], float mean, int lane, int k, int off, int D) {
  const int e = R::at(lane, k) - off;
  if (AL ? e < D : e >= 0 && e + R::V <= D) {  // (a whole vector, nearly always)
#pragma unroll
    for (int j = 0; j < R::V; ++j) c[j] = h[j] - mean;
  } else {
#pragma unroll
    for (int j = 0; j < R::V; ++j) c[j] = !AL && e + j >= 0 && e + j < D ? h[j] - mean : 0.f;
  }
}

// CTAs an SM that k_ln's registers are bounded for (0: as they come), so that the way of rows out of range costs none of them.  As they come
// and bounded, us: [16384, 768] float32 37.2 and 35.4, [8192, 4096] 88.8 and 82.4; to 8 bits [4096, 6144] 78.3 and 59.8, odd [2000, 2999]
// 27.1 and 25.0.
template <typename T, bool Q8, bool AL, int TPR, int NV>
constexpr int ln_ctas() {
  if constexpr (!AL) return TPR != 256 ? 0 : NV == 2 ? (sizeof(T) == 4 && Q8 ? 4 : 3) : NV == 3 && sizeof(T) == 4 && Q8 ? 3 : 0;
  if constexpr (sizeof(T) == 2) return 0;
  constexpr int registers = NV == 1 ? (Q8 ? 64 : 48) : NV == 2 ? (Q8 ? 72 : 64) : NV == 3 ? (Q8 && TPR == 512 ? 64 : 72) : 80;
  return 65536 / BLOCK_OF<TPR> / registers;
}
// Rows of k_ln on their way to a thread.  One and two for rows of one float32 vector a lane, at 40 and 48 registers (8 bits: 56 and 64), us:
// [64800, 128] 11.2 and 10.8 (9.7 without the check of each row's range, which keeps the loads from moving), with residual 23.4 and
// 20.2 (19.7), to 8 bits 26.4 and 18.9 (19.1).
template <typename T, bool AL, int TPR, int NV>
constexpr int LN_AHEAD = sizeof(T) == 4 && AL && TPR <= 32 && NV == 1 ? 2 : 1;
template <typename T, bool Q8, bool AL, int TPR, int NV>
__global__ void __launch_bounds__(BLOCK_OF<TPR>, ln_ctas<T, Q8, AL, TPR, NV>()) k_ln(const LayerForward a, const Same same) {
  constexpr int V = Io<T>::V, BLOCK = BLOCK_OF<TPR>, ROWS = BLOCK / TPR;
  using R = Row<T, AL, TPR>;
  extern __shared__ float s_w[];  // unaligned rows: the gains, then the shifts
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const float inv_d = 1.f / static_cast<float>(a.D);
  // A short launch lets the next kernel come in at once: its launch, its barriers and its tensor memory are set up beside this one's rows
  // (24 rows to 8 bits and their gated product 19.7 -> 19.4 us); a long one would have it wait in the SMs' way.  This comes before the wait:
  // the kernel before this one may still be writing, so that no kernel reads global data in front of its own pdl_wait.
  const bool short_launch = gridDim.x < 128;
  if (short_launch) pdl_trigger();
  pdl_wait();
  const int set = V * slots_of<V>(a.D);
  if constexpr (!AL) {
    gains_to_shared<V, BLOCK>(s_w, a.w, a.D);
    if (a.b) gains_to_shared<V, BLOCK>(s_w + set, a.b, a.D);
    __syncthreads();
  }
  const float *gains = AL ? a.w : s_w, *shifts = AL || !a.b ? a.b : s_w + set;
  Kept<R, AL, NV> kept_w, kept_b = {};
  kept_w.fill(gains, lane, a.D);
  if (a.b) kept_b.fill(shifts, lane, a.D);
  const long long step = static_cast<long long>(gridDim.x) * ROWS;
  const Bounds bx = bounds_of<T>(a.x, a.T, a.xs, a.D), br = bounds_of<T>(a.r, a.T, a.rs, a.D);
  constexpr int AHEAD = LN_AHEAD<T, AL, TPR, NV>;
  uint4 ux[AHEAD][NV], ur[AHEAD][NV];  // the next rows
  auto fetch = [&](long long t, int i) {
    const T *x = static_cast<const T*>(a.x) + t * a.xs, *r = static_cast<const T*>(a.r) + t * a.rs;
    const int D = t < a.T ? a.D : 0;  // a row past the end holds no elements
    R::fetch(x, bx, lane, R::offset(x), true, D, ux[i]);
    if (a.r) R::fetch(r, br, lane, R::offset(x), same.a, D, ur[i]);
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) fetch(static_cast<long long>(blockIdx.x) * ROWS + group + i * step, i);
  for (long long base = static_cast<long long>(blockIdx.x) * ROWS; base < a.T; base += step) {
    const long long t = base + group;
    const int D = t < a.T ? a.D : 0;
    const T *x = static_cast<const T*>(a.x) + t * a.xs, *r = static_cast<const T*>(a.r) + t * a.rs;
    const int off = R::offset(x);
    const Places<V> places(off, a.D);
    float h[NV][V], sum[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      R::values(x, bx, lane, k, off, true, D, ux[0][k], h[k]);
      if (a.r) {
        float f[V];
        R::values(r, br, lane, k, off, same.a, D, ur[0][k], f);
#pragma unroll
        for (int j = 0; j < V; ++j) h[k][j] += f[j];
        if (a.h) R::store(static_cast<T*>(a.h) + t * a.hs, lane, k, off, same.b, D, h[k]);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) sum[0] += h[k][j];
    }
#pragma unroll
    for (int i = 1; i < AHEAD; ++i)
#pragma unroll
      for (int k = 0; k < NV; ++k) ux[i - 1][k] = ux[i][k], ur[i - 1][k] = ur[i][k];
    fetch(t + AHEAD * step, AHEAD - 1);
    row_join<TPR, 0, false>(sum);
    float mean = sum[0] * inv_d, sq[1];
    auto squares = [&] {
      sq[0] = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float c[V];
        center<R, AL>(h[k], c, mean, lane, k, off, a.D);
#pragma unroll
        for (int j = 0; j < V; ++j) sq[0] += c[j] * c[j];
      }
    };
    squares();
    row_join<TPR, 1, false>(sq);
    float v = sq[0] * inv_d + a.eps;
    if (any_row<TPR>(!in_range(v))) {
      const float by = range_of(v, mean);
      sum[0] = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) sum[0] += h[k][j] *= by;
      row_join<TPR, 3, false>(sum);
      mean = sum[0] * inv_d;
      squares();
      row_join<TPR, 4, false>(sq);
      v = sq[0] * inv_d + eps_of(a.eps, by);
    }
    const float rstd = rsqrtf(v);
    float top[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float w[V], b[V] = {};
      kept_w.get(gains, places, lane, k, off, a.D, w);
      if (a.b) kept_b.get(shifts, places, lane, k, off, a.D, b);
      if constexpr (Q8) {
        center<R, AL>(h[k], h[k], mean, lane, k, off, a.D);  // what is not the row's counts as 0 in `top`
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) h[k][j] -= mean;
      }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        h[k][j] = h[k][j] * rstd * w[j] + b[j];
        if (Q8) top[0] = __uint_as_float(max(__float_as_uint(top[0]), __float_as_uint(magnitude(h[k][j]))));
      }
      if constexpr (!Q8) R::store(static_cast<T*>(a.y) + t * a.ys, lane, k, off, same.c, D, h[k]);
    }
    if constexpr (Q8) {
      row_join<TPR, 2, true>(top);
      const float lift = top[0] < TINY ? LIFT : 1.f, f = to_e4m3_range(top[0], lift);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
#pragma unroll
        for (int j = 0; j < V; ++j) h[k][j] = h[k][j] * lift * f;
        R::store_e4m3(static_cast<uint8_t*>(a.y) + t * a.ys, lane, k, off, same.c, D, h[k]);
      }
      if (lane == 0 && t < a.T) a.scale[t] = top[0] * (1.f / E4M3_MAX);
    }
  }
  if (!short_launch) pdl_trigger();
}

// A long row's sum of f(e) by LONG_THREADS threads, 32 terms at a time: a thread's own sum stays short.
template <class F>
__device__ __forceinline__ float sum_along(int D, F&& f) {
  float total = 0.f;
  for (int e0 = threadIdx.x; e0 < D; e0 += 32 * LONG_THREADS) {
    float s = 0.f;
#pragma unroll 4
    for (int i = 0; i < 32; ++i) {
      const int e = e0 + i * LONG_THREADS;
      if (e < D) s += f(e);
    }
    total += s;
  }
  return total;
}

// Rows too long for the registers: a CTA a row.  Element loads.  (Four CTAs an SM, where 40 registers leave three: [2000, 12001] float32 with residual
// 109 -> 98 us; 8 bits would spill.)
template <typename T, bool Q8>
__global__ void __launch_bounds__(LONG_THREADS, Q8 ? 3 : 4) k_ln_long(const LayerForward a) {
  pdl_wait();
  const float inv_d = 1.f / static_cast<float>(a.D);
  for (long long t = blockIdx.x; t < a.T; t += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + t * a.xs;
    const T* r = static_cast<const T*>(a.r) + t * a.rs;
    auto h = [&](int e) { return Io<T>::get(x, e) + (a.r ? Io<T>::get(r, e) : 0.f); };
    float sum[1] = {sum_along(a.D, h)};
    row_join<LONG_THREADS, 0, false>(sum);
    float mean = sum[0] * inv_d, by = 1.f;
    float sq[1] = {sum_along(a.D, [&](int e) {
      const float c = h(e) - mean;
      return c * c;
    })};
    row_join<LONG_THREADS, 1, false>(sq);
    float v = sq[0] * inv_d + a.eps;
    if (!in_range(v)) {
      by = range_of(v, mean);
      sum[0] = sum_along(a.D, [&](int e) { return h(e) * by; });
      row_join<LONG_THREADS, 3, false>(sum);
      mean = sum[0] * inv_d;
      sq[0] = sum_along(a.D, [&](int e) {
        const float c = h(e) * by - mean;
        return c * c;
      });
      row_join<LONG_THREADS, 4, false>(sq);
      v = sq[0] * inv_d + eps_of(a.eps, by);
    }
    const float rstd = rsqrtf(v);
    auto y = [&](float u, int e) { return (u * by - mean) * rstd * __ldg(a.w + e) + (a.b ? __ldg(a.b + e) : 0.f); };
    float top[1] = {0.f}, lift = 1.f, f = 1.f;
    if constexpr (Q8) {
      for (int e = threadIdx.x; e < a.D; e += LONG_THREADS)
        top[0] = __uint_as_float(max(__float_as_uint(top[0]), __float_as_uint(magnitude(y(h(e), e)))));
      row_join<LONG_THREADS, 2, true>(top);
      lift = top[0] < TINY ? LIFT : 1.f, f = to_e4m3_range(top[0], lift);
      if (threadIdx.x == 0) a.scale[t] = top[0] * (1.f / E4M3_MAX);
    }
    for (int e = threadIdx.x; e < a.D; e += LONG_THREADS) {
      const float v = h(e), o = y(v, e);  // (before h or y take x's place)
      if (a.r && a.h) Io<T>::put(static_cast<T*>(a.h) + t * a.hs, e, v);
      if constexpr (Q8)
        (static_cast<uint8_t*>(a.y) + t * a.ys)[e] = __nv_cvt_float_to_fp8(o * lift * f, __NV_SATFINITE, __NV_E4M3);
      else
        Io<T>::put(static_cast<T*>(a.y) + t * a.ys, e, o);
    }
  }
  pdl_trigger();
}

// Rows on their way to a thread of k_ln_bwd, 48 KB a CTA of 256 threads: registers for one row ahead (113 of them, two CTAs an SM) keep too
// little in flight: [131072, 256] bf16 with dh 59.5 us, this way 49.2.
template <int BLOCK, int NV>
constexpr int LN_DEPTH = NV == 1 ? 4 : 2;

// dx, and this CTA's partial row of dw and of db: part[blockIdx.x][0 .. 2 D).  Aligned rows: a thread's columns are the same in every
// row, their sums stay in its registers.  Unaligned ones, and rows of more vectors than that leaves registers for: in shared memory,
// two sets for each of the CTA's row groups (dynamic), or, where those would cost more than reading h and dy again, not here (SUMS): coef[t]
// = mean and rstd for k_ln_columns.
// (Odd rows on 256 threads are kept to 80 registers, three CTAs an SM: left alone they take 152, and one CTA an SM cannot hide what a row
// waits for: [20000, 601] float32 167 -> 127 us before such rows went as tiles.  Aligned float32 rows of one vector a lane are bounded as k_ln's are.)
template <typename T, bool AL, int TPR, int NV, bool SUMS>
__global__ void __launch_bounds__(BLOCK_OF<TPR>, !AL && TPR == 256 && NV == 1 ? 3 : AL && NV == 1 && TPR == 512 ? 2 : AL && NV == 1 && sizeof(T) == 4 ? (TPR == 128 ? 8 : 65536 / 80 / BLOCK_OF<TPR>) : 1) k_ln_bwd(const LayerBackward a, const Same same, float2* coef) {
  static_assert(SUMS || !AL, "the sums of aligned rows stay in registers");
  constexpr int V = Io<T>::V, BLOCK = BLOCK_OF<TPR>, ROWS = BLOCK / TPR;
  using R = Row<T, AL, TPR>;
  extern __shared__ __align__(16) float s_acc[];  // unaligned: a group's sums for dw, then for db; behind all groups' the gains.  Aligned: the rows
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const float inv_d = 1.f / static_cast<float>(a.D);
  float acc_w[AL ? NV : 1][V] = {}, acc_b[AL ? NV : 1][V] = {};
  const int set = V * slots_of<V>(a.D);
  float *own_w = s_acc + (AL ? 0 : 2 * group * set), *own_b = own_w + (AL ? 0 : set);
  if constexpr (!AL && SUMS) {
    for (int i = lane; i < 2 * set; i += TPR) own_w[i] = 0.f;
  }
  float* s_w = s_acc + (SUMS ? 2 * ROWS * set : 0);
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
  // the row's vectors: aligned rows come through shared memory, DEPTH of them on their way (a thread's own places: nobody else waits),
  // unaligned ones through registers, one row ahead
  constexpr int DEPTH = LN_DEPTH<BLOCK, NV>;
  uint4* ring = reinterpret_cast<uint4*>(s_acc) + threadIdx.x;
  auto place = [&](int i, int m, int k) { return ring + ((i * 3 + m) * NV + k) * BLOCK; };
  uint4 uh[AL ? 1 : NV], ud[AL ? 1 : NV], un[AL ? 1 : NV];
  auto fetch = [&](long long t, int i) {
    const T *hp = static_cast<const T*>(a.h) + t * a.hs, *dp = static_cast<const T*>(a.dy) + t * a.ys, *gp = static_cast<const T*>(a.dh) + t * a.ds;
    const int D = t < a.T ? a.D : 0;
    if constexpr (AL) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int e = R::at(lane, k), n = e < D ? 16 : 0;  // (0: zeros)
        const T* from[3] = {n ? hp + e : static_cast<const T*>(a.h), n ? dp + e : static_cast<const T*>(a.dy), n ? gp + e : static_cast<const T*>(a.dh)};
#pragma unroll
        for (int m = 0; m < 3; ++m)
          if (m < 2 || a.dh)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(place(i, m, k))), "l"(from[m]), "r"(n) : "memory");
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    } else {
      R::fetch(hp, bh, lane, R::offset(hp), true, D, uh);
      R::fetch(dp, bd, lane, R::offset(hp), same.a, D, ud);
      if (a.dh) R::fetch(gp, bg, lane, R::offset(hp), same.b, D, un);
    }
  };
  const long long first = static_cast<long long>(blockIdx.x) * ROWS;
#pragma unroll
  for (int i = 0; i < (AL ? DEPTH - 1 : 1); ++i) fetch(first + i * step + group, i);
  int turn = 0;
  for (long long base = first; base < a.T; base += step, turn = (turn + 1) % DEPTH) {
    const long long t = base + group;
    const int D = t < a.T ? a.D : 0;
    float h[NV][V], d[NV][V], sum[1] = {0.f};
    const T *hp = static_cast<const T*>(a.h) + t * a.hs, *dp = static_cast<const T*>(a.dy) + t * a.ys, *gp = static_cast<const T*>(a.dh) + t * a.ds;
    const int off = R::offset(hp);
    const Places<V> places(off, a.D);
    uint4 ug[NV];
    if constexpr (AL) {
      fetch(t + (DEPTH - 1) * step, (turn + DEPTH - 1) % DEPTH);
      asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        Io<T>::unpack(*place(turn, 0, k), h[k]);
        Io<T>::unpack(*place(turn, 1, k), d[k]);
        if (a.dh) ug[k] = *place(turn, 2, k);
      }
    } else {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        R::values(hp, bh, lane, k, off, true, D, uh[k], h[k]);
        R::values(dp, bd, lane, k, off, same.a, D, ud[k], d[k]);
        ug[k] = un[k];
      }
      fetch(t + step, 0);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) sum[0] += h[k][j];
    row_join<TPR, 0, false>(sum);
    float mean = sum[0] * inv_d, by = 1.f;
    float s[3] = {};  // of c^2, a, a c
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float w[V];
      kept.get(gains, places, lane, k, off, a.D, w);
      center<R, AL>(h[k], h[k], mean, lane, k, off, a.D);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float g = d[k][j] * w[j];
        s[0] += h[k][j] * h[k][j];
        s[1] += g;
        s[2] += g * h[k][j];
      }
    }
    row_join<TPR, 1, false>(s);  // (more than a warp a row: a barrier, behind which the last row's columns are added)
    if constexpr (!AL && TPR <= 32) __syncwarp();
    float v = s[0] * inv_d + a.eps;
    if (any_row<TPR>(!in_range(v))) {
      by = range_of(v, mean);
      sum[0] = 0.f;
      if constexpr (AL) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          Io<T>::unpack(*place(turn, 0, k), h[k]);
#pragma unroll
          for (int j = 0; j < V; ++j) sum[0] += h[k][j] *= by;
        }
      } else {
#pragma unroll 1
        for (int e = lane; e < D; e += TPR) sum[0] += Io<T>::get(hp, e) * by;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int e = R::at(lane, k) - off;
#pragma unroll
          for (int j = 0; j < V; ++j) h[k][j] = e + j >= 0 && e + j < D ? Io<T>::get(hp, e + j) * by : 0.f;
        }
      }
      row_join<TPR, 3, false>(sum);
      mean = sum[0] * inv_d;
      float again[2] = {};
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float w[V];
        kept.get(gains, places, lane, k, off, a.D, w);
        center<R, AL>(h[k], h[k], mean, lane, k, off, a.D);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          again[0] += h[k][j] * h[k][j];
          again[1] += d[k][j] * w[j] * h[k][j];
        }
      }
      row_join<TPR, 4, false>(again);
      s[2] = again[1];
      v = again[0] * inv_d + eps_of(a.eps, by);
    }
    const float rstd = t < a.T ? rsqrtf(v) : 0.f;  // (a row past the end adds nothing to dw, with eps = 0 either)
    const float ma = s[1] * inv_d, q = rstd * rstd * (s[2] * inv_d), rdx = rstd * by;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float w[V], o[V] = {};
      kept.get(gains, places, lane, k, off, a.D, w);
      if (a.dh) R::values(gp, bg, lane, k, off, same.b, D, ug[k], o);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float g = d[k][j] * (h[k][j] * rstd);
        if constexpr (AL) {
          acc_w[k][j] += g;
          acc_b[k][j] += d[k][j];
        } else if (SUMS && R::at(lane, k) - off < D) {
          own_w[places.at[j] + lane + TPR * k] += g;
          own_b[places.at[j] + lane + TPR * k] += d[k][j];
        }
        o[j] += rdx * (d[k][j] * w[j] - ma - q * h[k][j]);
      }
      if (SUMS || a.dx) R::store(static_cast<T*>(a.dx) + t * a.xs, lane, k, off, same.c, D, o);
    }
    if (!SUMS && lane == 0 && t < a.T) coef[t] = coefficients(mean, rstd, by);
  }
  if constexpr (!SUMS) {
    pdl_trigger();
    return;
  }
  if constexpr (AL) asm volatile("cp.async.wait_all;" ::: "memory");
  // the CTA's row groups hold the same columns: added in ascending group order
  float* part = static_cast<float*>(a.ws) + static_cast<long long>(blockIdx.x) * 2 * a.D;
  if constexpr (!AL) {
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.D; i += BLOCK) {
      const int e = i < a.D ? i : i - a.D;
      const float* from = s_acc + (i < a.D ? 0 : set) + column_at<V>(e, a.D);
      float sum = from[0];
#pragma unroll 4
      for (int g = 1; g < ROWS; ++g) sum += from[2 * g * set];
      part[i] = sum;
    }
  } else if constexpr (ROWS == 1) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < V; j += 4) {
        const int e = R::at(lane, k) + j;
        if (e >= a.D) continue;
        *reinterpret_cast<float4*>(part + e) = make_float4(acc_w[k][j], acc_w[k][j + 1], acc_w[k][j + 2], acc_w[k][j + 3]);
        *reinterpret_cast<float4*>(part + a.D + e) = make_float4(acc_b[k][j], acc_b[k][j + 1], acc_b[k][j + 2], acc_b[k][j + 3]);
      }
  } else {
    __shared__ float s[ROWS][TPR][V + 1];
    auto put = [&](const float (&acc)[AL ? NV : 1][V], float* to) {
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
          if (R::at(l, k) + j < a.D) to[R::at(l, k) + j] = sum;
        }
      }
    };
    put(acc_w, part);
    put(acc_b, part + a.D);
  }
  pdl_trigger();
}

// Rows too long for the registers: dx (DX) by a CTA a row; coef[t] = mean and rstd for k_ln_columns.
template <typename T, bool DX>
__global__ void __launch_bounds__(LONG_THREADS) k_ln_bwd_long(const LayerBackward a, float2* __restrict__ coef) {
  pdl_wait();
  const float inv_d = 1.f / static_cast<float>(a.D);
  for (long long t = blockIdx.x; t < a.T; t += gridDim.x) {
    const T* h = static_cast<const T*>(a.h) + t * a.hs;
    const T* dy = static_cast<const T*>(a.dy) + t * a.ys;
    float sum[1] = {sum_along(a.D, [&](int e) { return Io<T>::get(h, e); })};
    row_join<LONG_THREADS, 0, false>(sum);
    float mean = sum[0] * inv_d, by = 1.f;
    auto centred = [&](int e) { return Io<T>::get(h, e) * by - mean; };
    auto square = [&](int e) {
      const float c = centred(e);
      return c * c;
    };
    auto product = [&](int e) { return Io<T>::get(dy, e) * __ldg(a.w + e) * centred(e); };
    float s[3];
    s[0] = sum_along(a.D, square);
    s[1] = s[2] = 0.f;
    if constexpr (DX) {
      s[1] = sum_along(a.D, [&](int e) { return Io<T>::get(dy, e) * __ldg(a.w + e); });
      s[2] = sum_along(a.D, product);
    }
    row_join<LONG_THREADS, 1, false>(s);
    float v = s[0] * inv_d + a.eps;
    if (!in_range(v)) {
      by = range_of(v, mean);
      sum[0] = sum_along(a.D, [&](int e) { return Io<T>::get(h, e) * by; });
      row_join<LONG_THREADS, 3, false>(sum);
      mean = sum[0] * inv_d;
      float again[2] = {sum_along(a.D, square), DX ? sum_along(a.D, product) : 0.f};
      row_join<LONG_THREADS, 4, false>(again);
      s[2] = again[1];
      v = again[0] * inv_d + eps_of(a.eps, by);
    }
    const float rstd = rsqrtf(v), ma = s[1] * inv_d, q = rstd * rstd * (s[2] * inv_d), rdx = rstd * by;
    if constexpr (DX) {
      for (int e = threadIdx.x; e < a.D; e += LONG_THREADS) {
        float o = a.dh ? Io<T>::get(static_cast<const T*>(a.dh) + t * a.ds, e) : 0.f;
        o += rdx * (Io<T>::get(dy, e) * __ldg(a.w + e) - ma - q * centred(e));
        Io<T>::put(static_cast<T*>(a.dx) + t * a.xs, e, o);
      }
    }
    if (threadIdx.x == 0) coef[t] = coefficients(mean, rstd, by);
  }
  pdl_trigger();
}
// part[blockIdx.y][e], [D + e] = sums over the rows of chunk blockIdx.y of dy n and dy.  A CTA takes a strip of 32 vectors, a thread the V
// columns of one in every eighth row of the chunk, wherever the rows start.
constexpr int COLUMN_THREADS = 256, COLUMN_CTAS = 3;
template <typename T>
__global__ void __launch_bounds__(COLUMN_THREADS, COLUMN_CTAS) k_ln_columns(const LayerBackward a, const float2* coef, int chunks) {
  constexpr int V = Io<T>::V, G = COLUMN_THREADS / 32;  // rows at a time
  __shared__ float s[2][G][32][V + 1];
  const int lane = threadIdx.x & 31, g = threadIdx.x >> 5, c0 = (blockIdx.x * 32 + lane) * V;
  const long long t0 = a.T * blockIdx.y / chunks, t1 = a.T * (blockIdx.y + 1) / chunks;
  const int left = min(16, (a.D - c0) * static_cast<int>(sizeof(T)));  // bytes of the vector that are the row's
  pdl_wait();
  const Span sh = span_of(a.h, a.T, a.hs, a.D, sizeof(T)), sd = span_of(a.dy, a.T, a.ys, a.D, sizeof(T));
  float dw[V] = {}, db[V] = {};
  for (long long t = t0 + g; t < t1 && left > 0; t += G) {
    const uint8_t *hp = reinterpret_cast<const uint8_t*>(static_cast<const T*>(a.h) + t * a.hs + c0),
                  *dp = reinterpret_cast<const uint8_t*>(static_cast<const T*>(a.dy) + t * a.ys + c0);
    const Granules uh = fetch16(hp, sh), ud = fetch16(dp, sd);
    float2 c = coef[t];
    float h[V], d[V], by = 1.f;
    if (c.y < 0.f) {  // a row that is taken times a power of two (coefficients)
      by = c.y > -1.f ? DOWN : UP;
      c.y *= c.y > -1.f ? -0x1p60f : -0x1p-40f;
    }
    Io<T>::unpack(finish16(uh, hp, sh), h);
    Io<T>::unpack(keep(finish16(ud, dp, sd), left), d);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (c0 + j < a.D) dw[j] += d[j] * (fmaf(h[j], by, -c.x) * c.y);
      db[j] += d[j];
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) s[0][g][lane][j] = dw[j], s[1][g][lane][j] = db[j];
  __syncthreads();
  float* part = static_cast<float*>(a.ws) + static_cast<long long>(blockIdx.y) * 2 * a.D;
  for (int i = threadIdx.x; i < 2 * 32 * V; i += COLUMN_THREADS) {
    const int which = i / (32 * V), l = i % (32 * V) / V, j = i % V, e = blockIdx.x * 32 * V + l * V + j;
    float sum = s[which][0][l][j];
#pragma unroll
    for (int k = 1; k < G; ++k) sum += s[which][k][l][j];
    if (e < a.D) part[which * a.D + e] = sum;
  }
  pdl_trigger();
}

// dw[e] and db[e] (or null) = the sums of `parts` partial rows of 2 D: 32 runs of consecutive rows, each in ascending order, then the
// run sums in ascending order.  A CTA takes 32 columns.
constexpr int DWDB_RUNS = 32;
__global__ void __launch_bounds__(32 * DWDB_RUNS) k_dwdb(const float* part, float* dw, float* db, int D, int parts) {
  __shared__ float s[DWDB_RUNS][33];
  pdl_wait();
  const int lane = threadIdx.x & 31, g = threadIdx.x >> 5, e = blockIdx.x * 32 + lane, n = db ? 2 * D : D;
  const int p0 = parts * g / DWDB_RUNS, p1 = parts * (g + 1) / DWDB_RUNS;
  float sum = 0.f;
  if (e < n) {
    const float* q = part + e;
    for (int p = p0; p < p1; p += 16) {  // (the last ones too: a load at a time is the latency of each)
      float v[16];
#pragma unroll
      for (int u = 0; u < 16; ++u)
        if (p + u < p1) v[u] = __ldcg(q + static_cast<long long>(p + u) * 2 * D);
#pragma unroll
      for (int u = 0; u < 16; ++u)
        if (p + u < p1) sum += v[u];
    }
  }
  s[g][lane] = sum;
  __syncthreads();
  if (g == 0 && e < n) {
    float total = s[0][lane];
#pragma unroll
    for (int i = 1; i < DWDB_RUNS; ++i) total += s[i][lane];
    if (e < D) dw[e] = total; else db[e - D] = total;
  }
  pdl_trigger();
}

// ---- contiguous rows of an odd length ----
// Rows that are no whole 16-byte pieces, one behind another: tiles of 8, 16 or 32 rows (whole pieces together) come and go as they
// lie, in bulk copies (three stages, each with a place for every matrix read; what is computed takes a read one's place), and between
// the two LANES lanes take a row's elements, lane l those at l, l + LANES, ..: neither the rows' offsets nor their cut vectors cost anything, and
// a lane's columns are the same in every row.  NE: elements a lane.
constexpr int TILE_THREADS = 256, TILE_STAGES = 3;

// Rows of a tile, about 10 KB of a matrix.
template <typename T>
__host__ __device__ constexpr int tile_rows(int D) {
  const int bytes = D * static_cast<int>(sizeof(T));
  return bytes <= 320 ? 32 : bytes <= 640 ? 16 : 8;  // (64 rows up to 320 bytes: [64000, 77] float32 17.4 -> 25.5 us; 16: 18.9)
}
template <typename T>
__host__ __device__ constexpr int tile_bytes(int D) { return tile_rows<T>(D) * D * static_cast<int>(sizeof(T)); }

// Of a lane's NE elements the first SURE are inside every row that by_columns sends here (more than LANES SURE channels).
template <int NE>
constexpr int SURE = NE == 4 ? 0 : NE == 6 ? 4 : NE == 8 ? 6 : NE == 12 ? 8 : NE == 16 ? 12 : NE == 32 ? 16 : 32;

// A contiguous matrix [T, D] that is copied tile by tile.  The last tile's bytes beyond whole 16-byte pieces go element by element.
template <typename T>
struct Tiles {
  const void* p;
  long long rows;
  int D;
  __device__ __forceinline__ int bytes(long long tile) const {
    const long long left = rows - tile * tile_rows<T>(D);
    return left < tile_rows<T>(D) ? static_cast<int>(left) * D * static_cast<int>(sizeof(T)) : tile_bytes<T>(D);
  }
  __device__ __forceinline__ uint8_t* at(long long tile) const {
    return const_cast<uint8_t*>(static_cast<const uint8_t*>(p)) + tile * tile_bytes<T>(D);
  }
  // by one thread; the bytes that will arrive at the barrier
  __device__ __forceinline__ uint32_t load(long long tile, unsigned char* s, uint64_t* bar) const {
    const int n = bytes(tile) & ~15;
    if (n) bulk_load(s, at(tile), n, bar);
    return static_cast<uint32_t>(n);
  }
  // what a bulk copy leaves out, by the first threads; before (STORE: behind) a barrier
  template <bool STORE>
  __device__ __forceinline__ void ends(long long tile, unsigned char* s) const {
    const int n = bytes(tile), e = (n & ~15) / static_cast<int>(sizeof(T)) + static_cast<int>(threadIdx.x);
    if (threadIdx.x < 16 / sizeof(T) && e * static_cast<int>(sizeof(T)) < n) {
      T *g = reinterpret_cast<T*>(at(tile)) + e, *m = reinterpret_cast<T*>(s) + e;
      if (STORE) *g = *m; else *m = *g;
    }
  }
  __device__ __forceinline__ void store(long long tile, const unsigned char* s) const {  // by one thread
    const int n = bytes(tile) & ~15;
    if (n) bulk_store(at(tile), s, n);
  }
};

// The sums of a[0 .. N - 1] over a row's LANES lanes, the same value in each.
template <int LANES, int N>
__device__ __forceinline__ void lanes_join(float (&a)[N]) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] += __shfl_xor_sync(0xffffffffu, a[i], o);
}

// Stages of a kernel whose tiles have M matrices read: who loads, waits and stores.
template <typename T, int M>
struct Stages {
  unsigned char* smem;
  uint64_t* full;  // TILE_STAGES barriers
  Tiles<T> in[M];
  int live;  // matrices of a call
  int D;
  __device__ __forceinline__ unsigned char* place(int stage, int m) const { return smem + (stage * live + m) * tile_bytes<T>(D); }
  __device__ __forceinline__ void load(long long tile, int stage) const {  // thread 0
    uint32_t n = 0;
    for (int m = 0; m < live; ++m) n += static_cast<uint32_t>(in[m].bytes(tile) & ~15);
    tma::expect_tx(&full[stage], n);
    for (int m = 0; m < live; ++m) in[m].load(tile, place(stage, m), &full[stage]);
  }
  __device__ __forceinline__ void ends(long long tile, int stage) const {
    for (int m = 0; m < live; ++m) in[m].template ends<false>(tile, place(stage, m));
  }
};

// Q8: the bytes go out as they are made, to rows of any stride.  (With the 8-bit gated product behind it, bf16 and a residual: [86832, 74] by
// row kernels 63.1 us, by tiles 41.3; [30859, 575] 104.6 and 66.6.)
template <typename T, bool Q8, int LANES, int NE>
__global__ void __launch_bounds__(TILE_THREADS) k_ln_tile(const LayerForward a, unsigned int* err) {
  constexpr int ROWS = TILE_THREADS / LANES;  // at a time
  extern __shared__ __align__(128) unsigned char s_tiles[];
  __shared__ uint64_t full[TILE_STAGES];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, D = a.D, R = tile_rows<T>(D);
  const float inv_d = 1.f / static_cast<float>(D);
  const long long tiles = (a.T + R - 1) / R;
  if (threadIdx.x == 0) {
    for (int s = 0; s < TILE_STAGES; ++s) tc::mbar_init(&full[s], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  pdl_wait();
  const Stages<T, 2> st{s_tiles, full, {{a.x, a.T, D}, {a.r, a.T, D}}, a.r ? 2 : 1, D};
  const Tiles<T> y{a.y, a.T, D}, h_out{a.h, a.T, D};
  constexpr bool KEEP = NE <= 32;  // gains and shifts in registers, or from L1 with each row
  float kept_w[KEEP ? NE : 1], kept_b[KEEP ? NE : 1];
  if constexpr (KEEP) {
#pragma unroll
    for (int k = 0; k < NE; ++k) {
      const int e = lane + LANES * k;
      kept_w[k] = e < D ? __ldg(a.w + e) : 0.f;
      kept_b[k] = a.b && e < D ? __ldg(a.b + e) : 0.f;
    }
  }
  // y's element k of a lane (inside the row), from c rstd
  auto affine = [&](float n, int k) {
    if constexpr (KEEP) return n * kept_w[k] + kept_b[k];
    return n * __ldg(a.w + lane + LANES * k) + (a.b ? __ldg(a.b + lane + LANES * k) : 0.f);
  };
  if (threadIdx.x == 0) {
    for (int i = 0; i < TILE_STAGES - 1; ++i)
      if (blockIdx.x + static_cast<long long>(i) * gridDim.x < tiles) st.load(blockIdx.x + static_cast<long long>(i) * gridDim.x, i);
  }
  unsigned bad = 0;
  uint32_t it = 0;
  for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x, ++it) {
    const int s = it % TILE_STAGES;
    st.ends(tile, s);
    if (!bad && !tma::wait(&full[s], (it / TILE_STAGES) & 1)) bad |= 1;
    __syncthreads();  // the ends too
    T *xs = reinterpret_cast<T*>(st.place(s, 0)), *rs = reinterpret_cast<T*>(st.place(s, st.live - 1));
#pragma unroll 1
    for (int r0 = 0; r0 < R; r0 += ROWS) {
      const int at = (r0 + group) * D + lane;
      float v[NE], sum[1] = {0.f};
#pragma unroll
      for (int k = 0; k < NE; ++k) {
        const bool in = k < SURE<NE> || lane + LANES * k < D;
        v[k] = in ? Io<T>::get(xs, at + LANES * k) : 0.f;
        if (a.r && in) {
          v[k] += Io<T>::get(rs, at + LANES * k);
          Io<T>::put(rs, at + LANES * k, v[k]);
        }
        sum[0] += v[k];
      }
      lanes_join<LANES>(sum);
      float mean = sum[0] * inv_d, sq[1];
      auto squares = [&] {
        sq[0] = 0.f;
#pragma unroll
        for (int k = 0; k < NE; ++k) {
          const float c = k < SURE<NE> || lane + LANES * k < D ? v[k] - mean : 0.f;
          sq[0] += c * c;
        }
        lanes_join<LANES>(sq);
      };
      squares();
      const float var = sq[0] * inv_d + a.eps;
      float rstd = rsqrtf(var);
      auto finish = [&] {
#pragma unroll
        for (int k = 0; k < NE; ++k)
          if (k < SURE<NE> || lane + LANES * k < D) Io<T>::put(xs, at + LANES * k, affine((v[k] - mean) * rstd, k));
      };
      // (few elements a lane: y before the check, which then costs less, [10000, 501] bf16 9.05 and 8.6 us; many: [20000, 1500] 66.6 and 92)
      constexpr bool LATE = !Q8 && NE <= 16;
      if constexpr (LATE) finish();
      if (any_row<LANES>(!in_range(var))) {
        const float by = range_of(var, mean);
        sum[0] = 0.f;
#pragma unroll
        for (int k = 0; k < NE; ++k) sum[0] += v[k] *= by;
        lanes_join<LANES>(sum);
        mean = sum[0] * inv_d;
        squares();
        rstd = rsqrtf(sq[0] * inv_d + eps_of(a.eps, by));
        if constexpr (LATE) finish();
      }
      if constexpr (Q8) {
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < NE; ++k) {
          if (k < SURE<NE> || lane + LANES * k < D) {
            v[k] = affine((v[k] - mean) * rstd, k);
            top = max(top, __float_as_uint(magnitude(v[k])));
          }
        }
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const long long t = tile * R + r0 + group;
        if (t < a.T) {
          const float most = __uint_as_float(top), lift = most < TINY ? LIFT : 1.f, f = to_e4m3_range(most, lift);
          uint8_t* y8 = static_cast<uint8_t*>(a.y) + t * a.ys + lane;
#pragma unroll
          for (int k = 0; k < NE; ++k)
            if (k < SURE<NE> || lane + LANES * k < D) y8[LANES * k] = __nv_cvt_float_to_fp8(v[k] * lift * f, __NV_SATFINITE, __NV_E4M3);
          if (lane == 0) a.scale[t] = most * (1.f / E4M3_MAX);
        }
      } else if constexpr (!LATE) {
        finish();
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
      if constexpr (!Q8) y.store(tile, reinterpret_cast<unsigned char*>(xs));
      if (a.r && a.h) h_out.store(tile, reinterpret_cast<unsigned char*>(rs));
      tma::commit();
      const long long next = tile + static_cast<long long>(TILE_STAGES - 1) * gridDim.x;
      if (next < tiles) {
        asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");  // the last tile has left the stage
        st.load(next, (it + TILE_STAGES - 1) % TILE_STAGES);
      }
    }
    if constexpr (!Q8) y.template ends<true>(tile, reinterpret_cast<unsigned char*>(xs));
    if (a.r && a.h) h_out.template ends<true>(tile, reinterpret_cast<unsigned char*>(rs));
  }
  if (threadIdx.x == 0) {
    tma::wait_done();
    // a wait that gave up: the copies in flight have landed before the CTA can end
    for (uint32_t j = it > TILE_STAGES ? it - TILE_STAGES : 0; bad && j < it; ++j) (void)tma::wait(&full[j % TILE_STAGES], (j / TILE_STAGES) & 1);
    if (bad) atomicOr(err, bad);
  }
  pdl_trigger();
}

template <typename T, int LANES, int NE>
__global__ void __launch_bounds__(TILE_THREADS) k_ln_bwd_tile(const LayerBackward a, unsigned int* err) {
  constexpr int ROWS = TILE_THREADS / LANES;  // at a time
  extern __shared__ __align__(128) unsigned char s_tiles[];
  __shared__ uint64_t full[TILE_STAGES];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, D = a.D, R = tile_rows<T>(D);
  const float inv_d = 1.f / static_cast<float>(D);
  const long long tiles = (a.T + R - 1) / R;
  if (threadIdx.x == 0) {
    for (int s = 0; s < TILE_STAGES; ++s) tc::mbar_init(&full[s], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  pdl_wait();
  const Stages<T, 3> st{s_tiles, full, {{a.h, a.T, D}, {a.dy, a.T, D}, {a.dh, a.T, D}}, a.dh ? 3 : 2, D};
  const Tiles<T> dx{a.dx, a.T, D};
  float w[NE], acc_w[NE], acc_b[NE];
#pragma unroll
  for (int k = 0; k < NE; ++k) {
    const int e = lane + LANES * k;
    w[k] = e < D ? __ldg(a.w + e) : 0.f;
    acc_w[k] = acc_b[k] = 0.f;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < TILE_STAGES - 1; ++i)
      if (blockIdx.x + static_cast<long long>(i) * gridDim.x < tiles) st.load(blockIdx.x + static_cast<long long>(i) * gridDim.x, i);
  }
  unsigned bad = 0;
  uint32_t it = 0;
  for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x, ++it) {
    const int s = it % TILE_STAGES, rows = static_cast<int>(min(static_cast<long long>(R), a.T - tile * R));
    st.ends(tile, s);
    if (!bad && !tma::wait(&full[s], (it / TILE_STAGES) & 1)) bad |= 1;
    __syncthreads();  // the ends too
    const T *hs = reinterpret_cast<const T*>(st.place(s, 0)), *gs = reinterpret_cast<const T*>(st.place(s, 2));
    T* ds = reinterpret_cast<T*>(st.place(s, 1));
#pragma unroll 1
    for (int r0 = 0; r0 < R; r0 += ROWS) {
      const bool live = r0 + group < rows;  // (a row past the end adds nothing to dw and db)
      const int at = (r0 + group) * D + lane;
      float c[NE], d[NE], sum[1] = {0.f};
#pragma unroll
      for (int k = 0; k < NE; ++k) {
        const bool in = live && (k < SURE<NE> || lane + LANES * k < D);
        c[k] = in ? Io<T>::get(hs, at + LANES * k) : 0.f;
        d[k] = in ? Io<T>::get(ds, at + LANES * k) : 0.f;
        sum[0] += c[k];
      }
      lanes_join<LANES>(sum);
      const float mean = sum[0] * inv_d;
      float q[3] = {};  // sums of c^2, a, a c
#pragma unroll
      for (int k = 0; k < NE; ++k) {
        c[k] = k < SURE<NE> || lane + LANES * k < D ? c[k] - mean : 0.f;
        const float g = d[k] * w[k];
        q[0] += c[k] * c[k];
        q[1] += g;
        q[2] += g * c[k];
      }
      lanes_join<LANES>(q);
      float v = q[0] * inv_d + a.eps, by = 1.f;
      if (any_row<LANES>(!in_range(v))) {
        by = range_of(v, mean);
        const int end = live ? D - lane : 0;
        sum[0] = 0.f;
#pragma unroll 1
        for (int e = 0; e < end; e += LANES) sum[0] += Io<T>::get(hs, at + e) * by;
        lanes_join<LANES>(sum);
        const float m = sum[0] * inv_d;
        float again[2] = {};
#pragma unroll
        for (int k = 0; k < NE; ++k) {
          c[k] = LANES * k < end ? Io<T>::get(hs, at + LANES * k) * by - m : 0.f;
          again[0] += c[k] * c[k];
          again[1] += d[k] * w[k] * c[k];
        }
        lanes_join<LANES>(again);
        q[2] = again[1];
        v = again[0] * inv_d + eps_of(a.eps, by);
      }
      const float rstd = live ? rsqrtf(v) : 0.f;
      const float ma = q[1] * inv_d, m = rstd * rstd * (q[2] * inv_d), rdx = rstd * by;
#pragma unroll
      for (int k = 0; k < NE; ++k) {
        acc_w[k] += d[k] * (c[k] * rstd);
        acc_b[k] += d[k];
        if (live && (k < SURE<NE> || lane + LANES * k < D))
          Io<T>::put(ds, at + LANES * k, rdx * (d[k] * w[k] - ma - m * c[k]) + (a.dh ? Io<T>::get(gs, at + LANES * k) : 0.f));
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
      dx.store(tile, reinterpret_cast<unsigned char*>(ds));
      tma::commit();
      const long long next = tile + static_cast<long long>(TILE_STAGES - 1) * gridDim.x;
      if (next < tiles) {
        asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");  // the last tile has left the stage
        st.load(next, (it + TILE_STAGES - 1) % TILE_STAGES);
      }
    }
    dx.template ends<true>(tile, reinterpret_cast<unsigned char*>(ds));
  }
  if (threadIdx.x == 0) {
    tma::wait_done();
    // a wait that gave up: the copies in flight have landed before the CTA can end
    for (uint32_t j = it > TILE_STAGES ? it - TILE_STAGES : 0; bad && j < it; ++j) (void)tma::wait(&full[j % TILE_STAGES], (j / TILE_STAGES) & 1);
    if (bad) atomicOr(err, bad);
  }
  __syncthreads();  // the stages are free: every load has been waited for, every store has left
  // the row groups hold the same columns: added in ascending group order
  float* s_acc = reinterpret_cast<float*>(s_tiles);  // [group][2][D]
  float* part = static_cast<float*>(a.ws) + static_cast<long long>(blockIdx.x) * 2 * D;
#pragma unroll
  for (int k = 0; k < NE; ++k) {
    const int e = lane + LANES * k;
    if (e < D) s_acc[(2 * group) * D + e] = acc_w[k], s_acc[(2 * group + 1) * D + e] = acc_b[k];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += TILE_THREADS) {
    float sum = s_acc[i];
#pragma unroll 4
    for (int g = 1; g < ROWS; ++g) sum += s_acc[2 * g * D + i];
    part[i] = sum;
  }
  pdl_trigger();
}

// The same for wider rows, a warp a row: dx (null: not) and coef[t] = mean and rstd for k_ln_columns, the column sums of which would not fit
// the registers.  Gains in shared memory, two or three stages.  (Whole backward, row kernels and this, us: [20000, 601] float32 128 and 65,
// [28453, 1356] bf16 with dh 242 and 132, [5000, 1001] bf16 25.3 and 19.6, [8000, 1601] float32 115 and 78, bf16 78 and 56.)
constexpr int WIDE_ROWS = TILE_THREADS / 32;
template <int NE>
constexpr int WIDE_SURE = NE == 20 ? 16 : NE == 24 ? 20 : NE == 32 ? 24 : NE == 40 ? 32 : NE == 48 ? 40 : 48;
template <typename T, int NE>
__global__ void __launch_bounds__(TILE_THREADS, NE <= 24 ? 3 : NE <= 40 ? 2 : 1) k_ln_dx_tile(const LayerBackward a, float2* coef, int stages, unsigned int* err) {
  extern __shared__ __align__(128) unsigned char s_tiles[];
  __shared__ uint64_t full[TILE_STAGES];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = a.D;
  const float inv_d = 1.f / static_cast<float>(D);
  const long long tiles = (a.T + WIDE_ROWS - 1) / WIDE_ROWS;
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) tc::mbar_init(&full[s], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  pdl_wait();
  const Stages<T, 3> st{s_tiles, full, {{a.h, a.T, D}, {a.dy, a.T, D}, {a.dh, a.T, D}}, a.dh ? 3 : 2, D};
  const Tiles<T> dx{a.dx, a.T, D};
  float* s_w = reinterpret_cast<float*>(s_tiles + stages * st.live * tile_bytes<T>(D));
  for (int e = threadIdx.x; e < D; e += TILE_THREADS) s_w[e] = __ldg(a.w + e);  // (behind the first tile's barrier)
  if (threadIdx.x == 0) {
    for (int i = 0; i < stages - 1; ++i)
      if (blockIdx.x + static_cast<long long>(i) * gridDim.x < tiles) st.load(blockIdx.x + static_cast<long long>(i) * gridDim.x, i);
  }
  unsigned bad = 0;
  uint32_t it = 0;
  int s = 0;
  for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x, ++it, s = s + 1 == stages ? 0 : s + 1) {
    if (threadIdx.x == 0) {
      const long long next = tile + static_cast<long long>(stages - 1) * gridDim.x;
      if (next < tiles) {
        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // the last tile has left the stage
        st.load(next, s == 0 ? stages - 1 : s - 1);
      }
    }
    st.ends(tile, s);
    if (!bad && !tma::wait(&full[s], (it / stages) & 1)) bad |= 1;
    __syncthreads();  // the ends and the gains too
    const long long t = tile * WIDE_ROWS + warp;
    if (t < a.T) {
      const T* hs = reinterpret_cast<const T*>(st.place(s, 0)) + warp * D + lane;
      const T* gs = reinterpret_cast<const T*>(st.place(s, 2)) + warp * D + lane;
      T* ds = reinterpret_cast<T*>(st.place(s, 1)) + warp * D + lane;
      const float* ws = s_w + lane;
      float c[NE], d[NE], sum[1] = {0.f};
#pragma unroll
      for (int k = 0; k < NE; ++k) {
        const bool in = k < WIDE_SURE<NE> || lane + 32 * k < D;
        c[k] = in ? Io<T>::get(hs, 32 * k) : 0.f;
        d[k] = in ? Io<T>::get(ds, 32 * k) : 0.f;
        sum[0] += c[k];
      }
      lanes_join<32>(sum);
      float mean = sum[0] * inv_d, by = 1.f;
      float q[3] = {};  // sums of c^2, a, a c
#pragma unroll
      for (int k = 0; k < NE; ++k) {
        const bool in = k < WIDE_SURE<NE> || lane + 32 * k < D;
        c[k] = in ? c[k] - mean : 0.f;
        const float g = in ? d[k] * ws[32 * k] : 0.f;
        q[0] += c[k] * c[k];
        q[1] += g;
        q[2] += g * c[k];
      }
      lanes_join<32>(q);
      float v = q[0] * inv_d + a.eps;
      if (any_row<32>(!in_range(v))) {
        by = range_of(v, mean);
        sum[0] = 0.f;
#pragma unroll 1
        for (int e = 0; lane + e < D; e += 32) sum[0] += Io<T>::get(hs, e) * by;
        lanes_join<32>(sum);
        mean = sum[0] * inv_d;
        float again[2] = {};
#pragma unroll
        for (int k = 0; k < NE; ++k) c[k] = k < WIDE_SURE<NE> || lane + 32 * k < D ? Io<T>::get(hs, 32 * k) * by - mean : 0.f;
#pragma unroll 1
        for (int e = 0; lane + e < D; e += 32) {
          const float u = Io<T>::get(hs, e) * by - mean;
          again[0] += u * u;
          again[1] += Io<T>::get(ds, e) * ws[e] * u;
        }
        lanes_join<32>(again);
        q[2] = again[1];
        v = again[0] * inv_d + eps_of(a.eps, by);
      }
      const float rstd = rsqrtf(v), ma = q[1] * inv_d, m = rstd * rstd * (q[2] * inv_d), rdx = rstd * by;
      if (a.dx) {
#pragma unroll
        for (int k = 0; k < NE; ++k)
          if (k < WIDE_SURE<NE> || lane + 32 * k < D)
            Io<T>::put(ds, 32 * k, rdx * (d[k] * ws[32 * k] - ma - m * c[k]) + (a.dh ? Io<T>::get(gs, 32 * k) : 0.f));
      }
      if (lane == 0) coef[t] = coefficients(mean, rstd, by);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    if (a.dx) {
      if (threadIdx.x == 0) {
        dx.store(tile, reinterpret_cast<unsigned char*>(st.place(s, 1)));
        tma::commit();
      }
      dx.template ends<true>(tile, reinterpret_cast<unsigned char*>(st.place(s, 1)));
    }
  }
  if (threadIdx.x == 0) {
    tma::wait_done();
    // a wait that gave up: the copies in flight have landed before the CTA can end
    const uint32_t n = stages;
    for (uint32_t j = it > n ? it - n : 0; bad && j < it; ++j) (void)tma::wait(&full[j % n], (j / n) & 1);
    if (bad) atomicOr(err, bad);
  }
  pdl_trigger();
}

// ---- host ----

// The longest rows that go as tiles, and the least of them (two tiles an SM).  Rows of whole vectors stay with their own kernels
// (backward, us, tiles read by vectors and row kernels: [131072, 256] bf16 69.1 and 59.6, [128000, 64] float32 21.4 and 20.8).
// Forward with a residual, row kernels and tiles: [20000, 1500] bf16 72.1 and 64.7, [2500, 1101] 12.7 and 9.8, [8000, 1101] float32 34.6 and
// 29.7, but [10000, 2001] bf16 37.6 and 47.7; to 8 bits with its gated product [8000, 1501] 57.3 and 59.3.
constexpr int TILE_FORWARD = 1536, TILE_FORWARD_Q8 = 1024, TILE_BACKWARD = 512, TILE_WIDE = 2048;
constexpr size_t WIDE_SMEM = 220 * 1024;  // an SM's, less what its CTAs declare themselves
template <typename T>
static bool tiled(long long rows, int D, int most, int sms) {
  return D % Io<T>::V != 0 && D >= 8 && D <= most && rows >= 2ll * tile_rows<T>(D) * sms;
}
static bool contiguous(const void* p, long long stride, int D) { return !p || (stride == D && aligned(p, 16)); }
// Lanes a row and elements a lane for rows of D.
template <class F>
static void by_columns(int D, F&& f) {
#define WHTMIX_LANES(L, N) f(std::integral_constant<int, L>(), std::integral_constant<int, N>())
  if (D <= 32) WHTMIX_LANES(8, 4);
  else if (D <= 48) WHTMIX_LANES(8, 6);
  else if (D <= 64) WHTMIX_LANES(8, 8);
  else if (D <= 96) WHTMIX_LANES(16, 6);
  else if (D <= 128) WHTMIX_LANES(16, 8);
  else if (D <= 192) WHTMIX_LANES(32, 6);
  else if (D <= 256) WHTMIX_LANES(32, 8);
  else if (D <= 384) WHTMIX_LANES(32, 12);
  else if (D <= 512) WHTMIX_LANES(32, 16);
  else if (D <= 1024) WHTMIX_LANES(32, 32);
  else WHTMIX_LANES(32, 48);
#undef WHTMIX_LANES
}

template <typename T, bool Q8>
static cudaError_t forward_t(const LayerForward& a, unsigned int* err, int sms, cudaStream_t stream) {
  constexpr int V = Io<T>::V;
  const size_t es = sizeof(T);
  const bool al = a.D % V == 0 && aligned(a.w, 16) && (!a.b || aligned(a.b, 16)) && rows_aligned(a.x, a.xs, es) && rows_aligned(a.r, a.rs, es) &&
                  rows_aligned(a.r ? a.h : nullptr, a.hs, es) && (Q8 ? rows_aligned(a.y, a.ys, 1, V) : rows_aligned(a.y, a.ys, es));
  const int n = vectors(a.D, es == 2, al);
  LayerForward c = a;
  const size_t stages = static_cast<size_t>(TILE_STAGES) * (a.r ? 2 : 1) * tile_bytes<T>(a.D);
  if (tiled<T>(a.T, a.D, Q8 ? TILE_FORWARD_Q8 : TILE_FORWARD, sms) && stages <= WIDE_SMEM && contiguous(a.x, a.xs, a.D) && contiguous(a.r, a.rs, a.D) &&
      contiguous(a.r ? a.h : nullptr, a.hs, a.D) && (Q8 || contiguous(a.y, a.ys, a.D))) {
    const void* k = nullptr;
    by_columns(a.D, [&](auto lanes, auto ne) {
      constexpr int LANES = decltype(lanes)::value, NE = decltype(ne)::value;
      if constexpr (LANES * NE <= (Q8 ? TILE_FORWARD_Q8 : TILE_FORWARD)) k = reinterpret_cast<const void*>(k_ln_tile<T, Q8, LANES, NE>);
    });
    int resident = 0;
    const cudaError_t e = resident_ctas(k, TILE_THREADS, stages, sms, &resident);
    if (e != cudaSuccess) return e;
    void* args[] = {&c, &err};
    return launch_pdl(k, grid_rows(a.T, tile_rows<T>(a.D), resident), TILE_THREADS, stages, stream, args);
  }
  if (n > MAX_VECTORS) {
    void* args[] = {&c};
    return launch_pdl(reinterpret_cast<const void*>(k_ln_long<T, Q8>), grid_rows(a.T, 1, 4 * sms), LONG_THREADS, 0, stream, args);
  }
  // (8 bits: a vector's V bytes start on a multiple of V)
  const bool same_y = Q8 ? (reinterpret_cast<uintptr_t>(a.y) - reinterpret_cast<uintptr_t>(a.x) / es) % V == 0 && (a.ys - a.xs) % V == 0
                         : rows_same(a.x, a.xs, a.y, a.ys, es);
  Same same{rows_same(a.x, a.xs, a.r, a.rs, es), rows_same(a.x, a.xs, a.r ? a.h : nullptr, a.hs, es), same_y};
  return by_length(n, a.T < sms, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, BLOCK = BLOCK_OF<TPR>;
    const void* k = al ? reinterpret_cast<const void*>(k_ln<T, Q8, true, TPR, NV>) : reinterpret_cast<const void*>(k_ln<T, Q8, false, TPR, NV>);
    void* args[] = {&c, &same};
    const size_t smem = al ? 0 : static_cast<size_t>(a.b ? 2 : 1) * V * slots_of<V>(a.D) * 4;  // at most 128 KB
    int resident = 0;
    const cudaError_t e = resident_ctas(k, BLOCK, smem, sms, &resident);
    if (e != cudaSuccess) return e;
    return launch_pdl(k, grid_rows(a.T, BLOCK / TPR, resident), BLOCK, smem, stream, args);
  });
}

cudaError_t layer_forward(const LayerForward& a, bool bf16, bool to_e4m3, unsigned int* err, int sms, cudaStream_t stream) {
  if (a.T <= 0) return cudaSuccess;
  if (bf16) return to_e4m3 ? forward_t<__nv_bfloat16, true>(a, err, sms, stream) : forward_t<__nv_bfloat16, false>(a, err, sms, stream);
  return to_e4m3 ? forward_t<float, true>(a, err, sms, stream) : forward_t<float, false>(a, err, sms, stream);
}

// Chunks of rows of k_ln_columns: one wave, eight rows each at least.
template <typename T>
static int column_chunks(const LayerBackward& a, int sms) {
  const long long strips = (a.D + 32 * Io<T>::V - 1) / (32 * Io<T>::V), rows = (a.T + 7) / 8;
  long long most = (static_cast<long long>(COLUMN_CTAS) * sms + strips - 1) / strips;
  if (most > 256) most = 256;
  return static_cast<int>(rows < most ? rows : most);
}
template <typename T>
static cudaError_t columns(const LayerBackward& a, float2* coef, int chunks, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((a.D + 32 * Io<T>::V - 1) / (32 * Io<T>::V)), static_cast<unsigned>(chunks));
  cfg.blockDim = dim3(COLUMN_THREADS);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_ln_columns<T>, a, static_cast<const float2*>(coef), chunks);
}

// How a backward call's rows are taken: aligned with the sums in registers up to MAX_SUMMED vectors (512 threads have 128 registers each),
// else as unaligned ones.  (1024 threads with one vector each: [11870, 4696] bf16 148 -> 230 us.)
template <typename T>
constexpr int MAX_SUMMED = sizeof(T) == 4 ? 2048 : 1024;
struct LayerRows {
  bool al;
  int n;  // vectors
  bool apart;  // the sums by k_ln_columns
};
template <typename T>
static LayerRows layer_rows(const LayerBackward& a) {
  const size_t es = sizeof(T);
  const bool al = a.D % Io<T>::V == 0 && aligned(a.w, 16) && rows_aligned(a.h, a.hs, es) && rows_aligned(a.dy, a.ys, es) &&
                  rows_aligned(a.dh, a.ds, es) && rows_aligned(a.dx, a.xs, es) && vectors(a.D, es == 2, true) <= MAX_SUMMED<T>;
  const int n = vectors(a.D, es == 2, al);
  // Odd rows of more than 64 vectors and enough of them: [5000, 1001] bf16 31.1 -> 25.2 us; of more than 512 it does not pay
  // ([12856, 5565] 362 -> 399).
  return {al, n, n > MAX_VECTORS || (!al && n > 64 && n <= 512 && a.T * a.D >= 1ll << 20)};
}

// A call's kernel, its shared memory and its CTAs, each of which leaves a partial row of dw and db.
struct LayerPlan {
  const void* kernel;
  size_t smem;
  int block, parts;
  bool tiles;
  int wide;  // stages of k_ln_dx_tile, or 0
};

// Stages of k_ln_dx_tile for a call, its kernel and shared memory; 0 where two do not fit or the rows are not for it.
template <typename T>
static int wide_tiles(const LayerBackward& a, int sms, const void** kernel, size_t* smem) {
  if (!tiled<T>(a.T, a.D, TILE_WIDE, sms) || a.D <= TILE_BACKWARD || !contiguous(a.h, a.hs, a.D) || !contiguous(a.dy, a.ys, a.D) ||
      !contiguous(a.dh, a.ds, a.D) || !contiguous(a.dx, a.xs, a.D))
    return 0;
  const size_t stage = static_cast<size_t>(a.dh ? 3 : 2) * tile_bytes<T>(a.D), gains = static_cast<size_t>(a.D) * 4;
  const int most = static_cast<int>((WIDE_SMEM - gains) / stage), pair = static_cast<int>((WIDE_SMEM / 2 - gains) / stage);
  const int stages = pair >= 2 ? pair : most;  // two CTAs an SM before a third stage
  if (stages < 2) return 0;
  const int used = stages < TILE_STAGES ? stages : TILE_STAGES;
  *smem = used * stage + gains;
  auto k = [](auto ne) { return reinterpret_cast<const void*>(k_ln_dx_tile<T, decltype(ne)::value>); };
  const int ne = (a.D + 31) / 32;
  *kernel = ne <= 20 ? k(Int<20>()) : ne <= 24 ? k(Int<24>()) : ne <= 32 ? k(Int<32>()) : ne <= 40 ? k(Int<40>()) : ne <= 48 ? k(Int<48>()) : k(Int<64>());
  return used;
}
template <typename T>
static cudaError_t layer_plan(const LayerBackward& a, const LayerRows& rows, int sms, LayerPlan* p) {
  const size_t stages = static_cast<size_t>(TILE_STAGES) * (a.dh ? 3 : 2) * tile_bytes<T>(a.D);  // at most 144 KB
  p->tiles = tiled<T>(a.T, a.D, TILE_BACKWARD, sms) && contiguous(a.h, a.hs, a.D) && contiguous(a.dy, a.ys, a.D) &&
             contiguous(a.dh, a.ds, a.D) && contiguous(a.dx, a.xs, a.D);
  if (p->tiles) {
    by_columns(a.D, [&](auto lanes, auto ne) {
      constexpr int LANES = decltype(lanes)::value, NE = decltype(ne)::value;
      if constexpr (LANES * NE <= TILE_BACKWARD) p->kernel = reinterpret_cast<const void*>(k_ln_bwd_tile<T, LANES, NE>);
      const size_t sums = static_cast<size_t>(TILE_THREADS / LANES) * 2 * a.D * 4;  // in the stages' place at the end
      p->smem = stages > sums ? stages : sums;
    });
    p->block = TILE_THREADS;
    int resident = 0;
    const cudaError_t e = resident_ctas(p->kernel, TILE_THREADS, p->smem, sms, &resident);
    if (e == cudaSuccess) p->parts = static_cast<int>(grid_rows(a.T, tile_rows<T>(a.D), resident));
    return e;
  }
  if (rows.apart && (p->wide = wide_tiles<T>(a, sms, &p->kernel, &p->smem)) > 0) {
    p->block = TILE_THREADS;
    int resident = 0;
    const cudaError_t e = resident_ctas(p->kernel, TILE_THREADS, p->smem, sms, &resident);
    if (e == cudaSuccess) p->parts = static_cast<int>(grid_rows(a.T, WIDE_ROWS, resident));
    return e;
  }
  auto take = [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, BLOCK = BLOCK_OF<TPR>;
    constexpr bool ALIGNED = NV * TPR <= MAX_SUMMED<T>, ODD = TPR != 192 && TPR != 384;
    if (rows.al) {
      if constexpr (ALIGNED) p->kernel = reinterpret_cast<const void*>(k_ln_bwd<T, true, TPR, NV, true>);
    } else if constexpr (ODD) {
      p->kernel = reinterpret_cast<const void*>(k_ln_bwd<T, false, TPR, NV, true>);
      if constexpr (TPR * NV > 64 && TPR * NV <= 512) {
        if (rows.apart) p->kernel = reinterpret_cast<const void*>(k_ln_bwd<T, false, TPR, NV, false>);
      }
    }
    p->smem = rows.al ? static_cast<size_t>(LN_DEPTH<BLOCK, NV>) * 3 * NV * BLOCK * 16  // at most 192 KB
                      : static_cast<size_t>(rows.apart ? 1 : 2 * (BLOCK / TPR) + 1) * Io<T>::V * slots_of<Io<T>::V>(a.D) * 4;  // at most 193 KB
    p->block = BLOCK;
    int resident = 0;
    const cudaError_t e = resident_ctas(p->kernel, BLOCK, p->smem, sms, &resident);
    if (e == cudaSuccess) p->parts = static_cast<int>(grid_rows(a.T, BLOCK / TPR, resident));
    return e;
  };
  // (aligned rows in registers: threads in steps of two thirds too, [5288, 2232] bf16 41.5 us with 512 of them and 34.7 with 384)
  if (rows.al && rows.n > 128 && rows.n <= 192) return take(Int<192>(), Int<1>());
  if (rows.al && rows.n > 256 && rows.n <= 384) return take(Int<384>(), Int<1>());
  if (rows.al && rows.n > 512 && rows.n <= 768) return take(Int<384>(), Int<2>());
  return by_length_backward(rows.n, take);
}

template <typename T>
static cudaError_t workspace_t(const LayerBackward& a, int sms, size_t* bytes) {
  const LayerRows rows = layer_rows<T>(a);
  LayerPlan p{};
  if (rows.n <= MAX_VECTORS) {
    const cudaError_t e = layer_plan<T>(a, rows, sms, &p);
    if (e != cudaSuccess) return e;
  }
  const bool apart = rows.apart && !p.tiles;
  *bytes = static_cast<size_t>(apart ? column_chunks<T>(a, sms) : p.parts) * 2 * a.D * 4 + (apart ? static_cast<size_t>(a.T) * 8 : 0);
  return cudaSuccess;
}
cudaError_t layer_backward_workspace(const LayerBackward& a, bool bf16, int sms, size_t* bytes) {
  return bf16 ? workspace_t<__nv_bfloat16>(a, sms, bytes) : workspace_t<float>(a, sms, bytes);
}

template <typename T>
static cudaError_t backward_t(const LayerBackward& a, unsigned int* err, int sms, cudaStream_t stream) {
  const size_t es = sizeof(T);
  const LayerRows rows = layer_rows<T>(a);
  LayerBackward c = a;
  LayerPlan p{};
  cudaError_t e = cudaSuccess;
  if (rows.n <= MAX_VECTORS && (e = layer_plan<T>(a, rows, sms, &p)) != cudaSuccess) return e;
  const bool apart = rows.apart && !p.tiles;
  int parts = apart ? column_chunks<T>(a, sms) : p.parts;
  float2* coef = apart ? reinterpret_cast<float2*>(static_cast<float*>(a.ws) + static_cast<size_t>(parts) * 2 * a.D) : nullptr;
  if (rows.n > MAX_VECTORS) {
    // dw reads dy: where dx takes dy's place, the coefficients alone come first and dx last
    const bool over_dy = a.dx == a.dy;
    const void *with_dx = reinterpret_cast<const void*>(k_ln_bwd_long<T, true>), *without = reinterpret_cast<const void*>(k_ln_bwd_long<T, false>);
    void* args[] = {&c, &coef};
    auto take = [&](const void* k) { return launch_pdl(k, grid_rows(a.T, 1, 4 * sms), LONG_THREADS, 0, stream, args); };
    if ((e = take(over_dy ? without : with_dx)) != cudaSuccess) return e;
    if ((e = columns<T>(a, coef, parts, stream)) != cudaSuccess) return e;
    if (over_dy) e = take(with_dx);
  } else {
    Same same{rows_same(a.h, a.hs, a.dy, a.ys, es), rows_same(a.h, a.hs, a.dh, a.ds, es), rows_same(a.h, a.hs, a.dx, a.xs, es)};
    void *args[] = {&c, &same, &coef}, *tile_args[] = {&c, &err}, *wide_args[] = {&c, &coef, &p.wide, &err};
    auto take = [&] { return launch_pdl(p.kernel, static_cast<unsigned>(p.parts), p.block, p.smem, stream, p.tiles ? tile_args : p.wide ? wide_args : args); };
    // (dw reads dy, as above)
    const bool over_dy = apart && a.dx == a.dy;
    if (over_dy) c.dx = nullptr;
    e = take();
    if (e == cudaSuccess && apart) e = columns<T>(a, coef, parts, stream);
    if (e == cudaSuccess && over_dy) c.dx = a.dx, e = take();
  }
  if (e != cudaSuccess) return e;
  const float* part = static_cast<const float*>(a.ws);
  float *dw = a.dw, *db = a.db;
  int D = a.D;
  void* args[] = {&part, &dw, &db, &D, &parts};
  return launch_pdl(reinterpret_cast<const void*>(k_dwdb), static_cast<unsigned>(((db ? 2 * D : D) + 31) / 32), 32 * DWDB_RUNS, 0, stream, args);
}

cudaError_t layer_backward(const LayerBackward& a, bool bf16, unsigned int* err, int sms, cudaStream_t stream) {
  return bf16 ? backward_t<__nv_bfloat16>(a, err, sms, stream) : backward_t<float>(a, err, sms, stream);
}

}  // namespace norm
}  // namespace whtmix
