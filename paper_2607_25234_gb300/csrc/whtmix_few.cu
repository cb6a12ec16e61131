// whtmix_few.cu -- the linear layer's product for a few tokens (up to 64): y = act(s_x s_w x W^T + b) + r, bound by reading W once.
//
// W goes from memory to registers in 16-byte loads and into mma.sync from there (its rows are the product's rows, the tokens its
// columns): no shared memory, no conversion, nothing between the loads and the products, and every warp keeps 16 KB and more in
// flight.  A lane holds 16 consecutive bytes of k of a row of W and of x alike; the order of k within a product is immaterial.
// A CTA of 8 warps takes 16 MT rows of W, its warps take blocks of 64 bytes of k in turn; the K axis is also divided over the
// CTAs of a cluster, so that a small W occupies every SM.  The warps' sums meet in shared memory, the cluster's through
// distributed shared memory, each in a fixed order.
// tcgen05 would need W staged in shared memory for products that are idle most of the time: with few tokens the 128-row tiles of
// whtmix_gemm.cuh take 11.6 us for [1, 1024] x [4096, 1024] (8 MB) and 19.5 us for 24 tokens of 4096 8-bit channels to 8192.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "whtmix_few.cuh"
#include "whtmix_gemm.cuh"
#include "whtmix_unaligned.cuh"

namespace whtmix {
namespace linear {

constexpr int FEW_WARPS = 8, FEW_THREADS = 32 * FEW_WARPS;
template <int NT>
struct Few {
  static constexpr int MT = 2, ROWS = 16 * MT, TOKENS = 8 * NT, PITCH = ROWS + 4;
  static constexpr int DEPTH = NT == 1 ? 4 : NT == 2 ? 3 : 2;  // 64-byte blocks of k a warp has in flight
  static constexpr size_t SMEM = static_cast<size_t>(FEW_WARPS) * TOKENS * PITCH * 4;
};

template <bool E4M3>
__device__ __forceinline__ void mma_few(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (E4M3)
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// VEC: rows of x and W are 16-byte aligned and whole multiples of 16 bytes.
template <bool E4M3, int NT, bool VEC, typename O>
__global__ void __launch_bounds__(FEW_THREADS, NT <= 4 && VEC ? 2 : 1) k_few(const Forward a, int splits) {
  using F = Few<NT>;
  constexpr int MT = F::MT, ES = E4M3 ? 1 : 2;
  extern __shared__ __align__(16) float s_sum[];
  namespace cg = cooperative_groups;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int rank = blockIdx.x % splits, n0 = blockIdx.x / splits * F::ROWS;
  const int T = static_cast<int>(a.T);
  const long long row_bytes = static_cast<long long>(a.K) * ES;
  const int blocks = static_cast<int>((row_bytes + 63) / 64);
  const int b0 = static_cast<int>(static_cast<long long>(blocks) * rank / splits), b1 = static_cast<int>(static_cast<long long>(blocks) * (rank + 1) / splits);
  const uint8_t *x = static_cast<const uint8_t*>(a.x), *w = static_cast<const uint8_t*>(a.w);
  const Span sx = span_of(x, a.T, a.xs, a.K, ES), sw = span_of(w, a.N, a.ws, a.K, ES);
  using Raw = typename std::conditional<VEC, uint4, Granules>::type;
  auto fetch = [&](Raw& u, const uint8_t* base, long long pitch, int row, int rows, int block, const Span& span) {
    const long long at = 64ll * block + 16 * c;
    u = Raw{};
    if (row >= rows || at >= row_bytes) return;
    const uint8_t* p = base + row * pitch * ES + at;
    if constexpr (VEC)
      u = *reinterpret_cast<const uint4*>(p);
    else
      u = fetch16(p, span);
  };
  auto finish = [&](const Raw& u, const uint8_t* base, long long pitch, int row, int rows, int block, const Span& span) -> uint4 {
    if constexpr (VEC) {
      return u;
    } else {
      const long long at = 64ll * block + 16 * c;
      if (row >= rows || at >= row_bytes) return make_uint4(0u, 0u, 0u, 0u);
      const uint4 v = finish16(u, base + row * pitch * ES + at, span);
      return row_bytes - at >= 16 ? v : keep(v, static_cast<int>(row_bytes - at));
    }
  };
  float acc[MT][NT][4] = {};
  constexpr int DEPTH = VEC ? F::DEPTH : 1;
  Raw wr[DEPTH][MT][2], xr[DEPTH][NT];
  auto load = [&](Raw (&wb)[MT][2], Raw (&xb)[NT], int block) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) fetch(wb[m][h], w, a.ws, n0 + 16 * m + 8 * h + g, a.N, block, sw);
#pragma unroll
    for (int n = 0; n < NT; ++n) fetch(xb[n], x, a.xs, 8 * n + g, T, block, sx);
  };
  auto multiply = [&](const Raw (&wb)[MT][2], const Raw (&xb)[NT], int block) {
    uint4 u[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) u[m][h] = finish(wb[m][h], w, a.ws, n0 + 16 * m + 8 * h + g, a.N, block, sw);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint4 v = finish(xb[n], x, a.xs, 8 * n + g, T, block, sx);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        mma_few<E4M3>(acc[m][n], u[m][0].x, u[m][1].x, u[m][0].y, u[m][1].y, v.x, v.y);
        mma_few<E4M3>(acc[m][n], u[m][0].z, u[m][1].z, u[m][0].w, u[m][1].w, v.z, v.w);
      }
    }
  };
  pdl_wait();
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) {
    const int block = b0 + warp + FEW_WARPS * d;
    if (block < b1) load(wr[d], xr[d], block);
  }
  for (int first = b0 + warp; first < b1; first += FEW_WARPS * DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int block = first + FEW_WARPS * d, next = block + FEW_WARPS * DEPTH;
      if (block < b1) {
        multiply(wr[d], xr[d], block);
        if (next < b1) load(wr[d], xr[d], next);
      }
    }
  }
  // the warps' sums, then the cluster's
  float* mine = s_sum + warp * F::TOKENS * F::PITCH;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) mine[(8 * n + 2 * c + (j & 1)) * F::PITCH + 16 * m + g + 8 * (j >> 1)] = acc[m][n][j];
  __syncthreads();
  constexpr int ALL = F::TOKENS * F::ROWS;
  for (int i = threadIdx.x; i < ALL; i += FEW_THREADS) {
    const int at = i / F::ROWS * F::PITCH + i % F::ROWS;
    float sum = s_sum[at];
#pragma unroll
    for (int k = 1; k < FEW_WARPS; ++k) sum += s_sum[k * F::TOKENS * F::PITCH + at];
    s_sum[at] = sum;
  }
  if (splits > 1) cg::this_cluster().sync();
  const int tokens = min(T, F::TOKENS), live = tokens * F::ROWS;
  for (int i = live * rank / splits + threadIdx.x; i < live * (rank + 1) / splits; i += FEW_THREADS) {
    const int t = i / F::ROWS, n = n0 + i % F::ROWS, at = t * F::PITCH + i % F::ROWS;
    float z = 0.f;
    if (splits == 1) {
      z = s_sum[at];
    } else {
      for (int k = 0; k < splits; ++k) z += *cg::this_cluster().map_shared_rank(s_sum + at, k);
    }
    if (n >= a.N) continue;
    if (E4M3) z *= a.x_scale[t] * a.w_scale[n];
    if (a.bias) z += a.bias[n];
    if (a.p) static_cast<__nv_bfloat16*>(a.p)[t * a.ps + n] = __float2bfloat16_rn(z);
    z = activate(z, a.act);
    if (a.r) z += static_cast<float>(static_cast<const O*>(a.r)[t * a.rs + n]);
    static_cast<O*>(a.y)[t * a.ys + n] = static_cast<O>(z);
  }
  if (splits > 1) cg::this_cluster().sync();  // the others have read this CTA's sums
  pdl_trigger();
}

template <bool E4M3, int NT, bool VEC, typename O>
static cudaError_t launch_few(const Forward& a, int sms, cudaStream_t stream) {
  using F = Few<NT>;
  auto k = k_few<E4M3, NT, VEC, O>;
  static std::atomic<uint64_t> raised{0};
  cudaError_t e = raise_smem(reinterpret_cast<const void*>(k), F::SMEM, raised);
  if (e != cudaSuccess) return e;
  // the K axis over 1, 2, 4 or 8 CTAs where the rows alone leave SMs idle, with a block of k a warp at least
  const long long tiles = (a.N + F::ROWS - 1) / F::ROWS, blocks = (static_cast<long long>(a.K) * (E4M3 ? 1 : 2) + 63) / 64;
  int splits = 1;
  while (splits < 8 && tiles * splits * 2 <= 2ll * sms && blocks >= 2ll * FEW_WARPS * splits) splits *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(tiles * splits));
  cfg.blockDim = dim3(FEW_THREADS);
  cfg.dynamicSmemBytes = F::SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(splits);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, k, a, splits);
}

template <bool E4M3, bool VEC, typename O>
static cudaError_t by_tokens(const Forward& a, int sms, cudaStream_t stream) {
  if (a.T <= 8) return launch_few<E4M3, 1, VEC, O>(a, sms, stream);
  if (a.T <= 16) return launch_few<E4M3, 2, VEC, O>(a, sms, stream);
  if (a.T <= 32) return launch_few<E4M3, 4, VEC, O>(a, sms, stream);
  return launch_few<E4M3, 8, VEC, O>(a, sms, stream);
}

template <bool E4M3, typename O>
static cudaError_t by_alignment(const Forward& a, int sms, cudaStream_t stream) {
  const int es = E4M3 ? 1 : 2;
  const bool vec = (static_cast<long long>(a.K) * es) % 16 == 0 && tma::mappable(a.x, a.T, a.xs, es) && tma::mappable(a.w, a.N, a.ws, es);
  return vec ? by_tokens<E4M3, true, O>(a, sms, stream) : by_tokens<E4M3, false, O>(a, sms, stream);
}

cudaError_t forward_few(const Forward& a, int sms, cudaStream_t stream) {
  if (a.e4m3) return a.out_f32 ? by_alignment<true, float>(a, sms, stream) : by_alignment<true, __nv_bfloat16>(a, sms, stream);
  return a.out_f32 ? by_alignment<false, float>(a, sms, stream) : by_alignment<false, __nv_bfloat16>(a, sms, stream);
}

}  // namespace linear
}  // namespace whtmix
