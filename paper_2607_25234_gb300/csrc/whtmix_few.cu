// whtmix_few.cu -- the linear layer's product for few tokens (use_few), where whtmix_gemm.cuh would have few tiles or wait for W:
// y = act(s_x s_w x W^T + b) + r, bound by reading W and the latencies of one short chain.
//
// The roles of whtmix_gemm.cuh exchanged: 128 rows of W are the product's M, 16, 32, 64 or 128 tokens its N, so that with few
// tokens every load in flight is a weight's.  A CTA takes 128 rows of W, the tokens of one tile and a share of K; the CTAs that
// share a tile form a cluster (up to 8), two CTAs fit an SM.  Warp 4 keeps a ring of TMA loads full, warp 5 issues the products
// into tensor memory, warps 0-3 move the accumulator (a thread a row of W) to shared memory; then each CTA of the cluster adds
// its share of the tile's tokens from all of them, in rank order, applies the epilogue and stores 128 consecutive channels a warp.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "whtmix_few.cuh"
#include "whtmix_gemm.cuh"

namespace whtmix {
namespace linear {

constexpr int FEW_THREADS = 192, FEW_ROWS = 128;

struct Few {
  CUtensorMap tw, tx;
  void* y;
  const void* r;
  void* p;
  long long ys, rs, ps;
  const float *bias, *sx, *sw;  // scales of the rows of x and W, or null
  int T, N, kblocks, splits, tiles_n, act;
  bool vec;  // rows of y, r and p lie on whole fours of channels
  unsigned int* err;
};

template <int TN>
constexpr uint32_t FEW_STAGE = (FEW_ROWS + TN) * 128;
template <int TN>
constexpr int FEW_STAGES = TN <= 32 ? 5 : TN == 64 ? 4 : 3;  // at most 100 KB: two CTAs an SM
template <int TN>  // the ring, or the tile's sums that take its place
constexpr size_t FEW_SMEM = FEW_STAGES<TN> * FEW_STAGE<TN>;
static_assert(FEW_SMEM<128> >= 128 * FEW_ROWS * 4 && FEW_SMEM<16> >= 16 * FEW_ROWS * 4, "a tile's sums fit the ring");

// four consecutive channels
template <typename O>
struct Four;
template <>
struct Four<float> {
  static __device__ __forceinline__ void load(const void* p, long long i, float (&f)[4]) {
    const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
    f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w;
  }
  static __device__ __forceinline__ void store(void* p, long long i, const float (&f)[4]) {
    *reinterpret_cast<float4*>(static_cast<float*>(p) + i) = make_float4(f[0], f[1], f[2], f[3]);
  }
};
template <>
struct Four<__nv_bfloat16> {
  static __device__ __forceinline__ void load(const void* p, long long i, float (&f)[4]) {
    const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(p) + i);
    f[0] = __uint_as_float(u.x << 16), f[1] = __uint_as_float(u.x & 0xffff0000u);
    f[2] = __uint_as_float(u.y << 16), f[3] = __uint_as_float(u.y & 0xffff0000u);
  }
  static __device__ __forceinline__ void store(void* p, long long i, const float (&f)[4]) {
    __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p) + i) =
        make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
  }
};

// GATED: a tile's 128 rows of W are 64 of the gate's and the 64 of the value's that belong to the same channels; lanes 0-15 of a
// warp take the gate's sums, lanes 16-31 the value's, and the gate's lanes store four channels of y.
template <bool E4M3, int TN, typename O, bool GATED>
__global__ void __launch_bounds__(FEW_THREADS) k_few(const __grid_constant__ Few a) {
  constexpr int OUT = GATED ? FEW_ROWS / 2 : FEW_ROWS;  // channels of a tile
  constexpr int BK = E4M3 ? 128 : 64, S = FEW_STAGES<TN>;
  constexpr uint32_t IDESC = (1u << 4) | (E4M3 ? 0u : (1u << 7) | (1u << 10)) | (static_cast<uint32_t>(TN >> 3) << 17) | ((128u >> 4) << 24);
  constexpr int COLS = TN < 32 ? 32 : TN;  // tensor-memory columns
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ uint64_t full[S], empty[S], dfull;
  __shared__ uint32_t tmem_slot;
  namespace cg = cooperative_groups;
  const uint32_t ring = tc::smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = blockIdx.x % a.splits, tile = blockIdx.x / a.splits;
  const int n0 = tile % a.tiles_n * OUT, t0 = tile / a.tiles_n * TN, tokens = min(TN, a.T - t0);
  const int k0 = static_cast<int>(static_cast<long long>(a.kblocks) * rank / a.splits);
  const int k1 = static_cast<int>(static_cast<long long>(a.kblocks) * (rank + 1) / a.splits);
  if (warp == 0) tc::tmem_alloc(&tmem_slot, COLS);
  if (tid == 32) {
    for (int s = 0; s < S; ++s) tc::mbar_init(&full[s], 1), tc::mbar_init(&empty[s], 1);
    tc::mbar_init(&dfull, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma::prefetch(&a.tw);
    tma::prefetch(&a.tx);
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  pdl_wait();
  pdl_trigger();  // (tensor memory is allocated) the next kernel comes in beside this one: a chain of [1, 1024] to 4096 5.8 -> 4.8 us a link
  const uint32_t tmem = tmem_slot;
  unsigned bad = 0;
  if (warp == 4) {
    if (lane == 0) {
      int i = 0;
      for (const int n = k1 - k0; i < n; ++i) {
        const int s = i % S;
        if (!tma::wait(&empty[s], ((i / S) & 1) ^ 1)) {
          bad |= 1;
          break;
        }
        const uint32_t st = ring + s * FEW_STAGE<TN>;
        tma::expect_tx(&full[s], FEW_STAGE<TN>);
        tma::load_2d(st, &a.tw, (k0 + i) * BK, n0, &full[s]);
        if constexpr (GATED) tma::load_2d(st + OUT * 128, &a.tw, (k0 + i) * BK, a.N + n0, &full[s]);
        tma::load_2d(st + FEW_ROWS * 128, &a.tx, (k0 + i) * BK, t0, &full[s]);
      }
      // the copies in flight have landed before the CTA can end, whichever warp has given up
      for (int j = i > S ? i - S : 0; j < i; ++j)
        if (!tma::wait(&full[j % S], (j / S) & 1)) bad |= 1;
    }
  } else if (warp == 5) {
    if (lane == 0) {
      for (int kb = k0; kb < k1; ++kb) {
        const int i = kb - k0, s = i % S;
        if (!tma::wait(&full[s], (i / S) & 1)) {
          bad |= 2;
          break;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t sw = ring + s * FEW_STAGE<TN>, sx = sw + FEW_ROWS * 128;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          const uint32_t acc = i > 0 || ks > 0;
          if constexpr (E4M3)
            mma_e4m3(tmem, tc::sw128_desc(sw + ks * 32), tc::sw128_desc(sx + ks * 32), IDESC, acc);
          else
            tc::mma_bf16(tmem, tc::sw128_desc(sw + ks * 32), tc::sw128_desc(sx + ks * 32), IDESC, acc);
        }
        tc::mma_commit(&empty[s]);
      }
      tc::mma_commit(&dfull);
      // every product has completed before the tensor memory is freed, also where warps 0-3 have given up
      if (!tma::wait(&dfull, 0)) bad |= 2;
    }
  }
  float* sums = reinterpret_cast<float*>(smem);  // [token][row of W]
  if (warp < 4) {
    // the products have completed: the accumulator can be read, the ring is free
    if (!tma::wait(&dfull, 0)) bad |= 4;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    __syncwarp();
#pragma unroll
    for (int c = 0; c < TN; c += 16) {
      if (c < tokens) {
        float v[16];
        tc::tmem_ld16(tmem + (static_cast<uint32_t>(32 * warp) << 16) + c, v);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
        for (int j = 0; j < 16; ++j) sums[(c + j) * FEW_ROWS + tid] = v[j];
      }
    }
  }
  cg::cluster_group cluster = cg::this_cluster();
  if (a.splits > 1) cluster.sync(); else __syncthreads();
  const int n = n0 + (4 * lane) % OUT, live = min(4, a.N - n), wn = n + (4 * lane < OUT ? 0 : a.N);  // channel, row of W
  float bias[4] = {}, sw[4] = {1.f, 1.f, 1.f, 1.f};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (j < live && a.bias) bias[j] = a.bias[wn + j];
    if (j < live && a.sw) sw[j] = a.sw[wn + j];
  }
  const bool vec = a.vec && live == 4;
  const int tt0 = tokens * rank / a.splits, tt1 = tokens * (rank + 1) / a.splits;
  auto finish = [&](int tt, float4 sum) {
    const long long t = t0 + tt;
    float z[4] = {sum.x, sum.y, sum.z, sum.w}, r[4] = {};
    if (a.r) {
      if (vec) {
        Four<O>::load(a.r, t * a.rs + n, r);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < live) r[j] = static_cast<float>(static_cast<const O*>(a.r)[t * a.rs + n + j]);
      }
    }
    const float sx = a.sx ? a.sx[t] : 1.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] = (a.sx ? z[j] * sx * sw[j] : z[j]) + bias[j];
    if (a.p) {
      if (vec) {
        Four<__nv_bfloat16>::store(a.p, t * a.ps + wn, z);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < live) static_cast<__nv_bfloat16*>(a.p)[t * a.ps + wn + j] = __float2bfloat16_rn(z[j]);
      }
    }
    float u[4] = {1.f, 1.f, 1.f, 1.f};
    if constexpr (GATED) {
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] = __shfl_down_sync(0xffffffffu, z[j], 16);
      if (lane >= 16) return;
    }
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      activate(z[j], z[j + 1], a.act);
      if constexpr (GATED)
        z[j] *= u[j], z[j + 1] *= u[j + 1];
      else
        z[j] += r[j], z[j + 1] += r[j + 1];
    }
    if (vec) {
      Four<O>::store(a.y, t * a.ys + n, z);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < live) static_cast<O*>(a.y)[t * a.ys + n + j] = static_cast<O>(z[j]);
    }
  };
  // 16 loads of the cluster's sums in flight: 16 / splits tokens at a time
  auto add_up = [&](auto splits) {
    constexpr int SPLITS = decltype(splits)::value, U = 16 / SPLITS < 4 ? 16 / SPLITS : 4;
    const float* from[SPLITS];
#pragma unroll
    for (int k = 0; k < SPLITS; ++k) from[k] = SPLITS == 1 ? sums : cluster.map_shared_rank(sums, k);
    for (int base = tt0 + warp; base < tt1; base += U * (FEW_THREADS / 32)) {
      float4 part[U][SPLITS];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < SPLITS; ++k) {
          const int tt = base + u * (FEW_THREADS / 32);
          if (tt < tt1) part[u][k] = *reinterpret_cast<const float4*>(from[k] + tt * FEW_ROWS + 4 * lane);
        }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int tt = base + u * (FEW_THREADS / 32);
        if (tt < tt1) {
          float4 z = part[u][0];
#pragma unroll
          for (int k = 1; k < SPLITS; ++k) z.x += part[u][k].x, z.y += part[u][k].y, z.z += part[u][k].z, z.w += part[u][k].w;
          finish(tt, z);
        }
      }
    }
  };
  switch (a.splits) {
    case 1: add_up(std::integral_constant<int, 1>()); break;
    case 2: add_up(std::integral_constant<int, 2>()); break;
    case 4: add_up(std::integral_constant<int, 4>()); break;
    default: add_up(std::integral_constant<int, 8>()); break;
  }
  if (a.splits > 1) cluster.sync();  // the others have read this CTA's sums
  if (bad) atomicOr(a.err, bad << 24);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 0) tc::tmem_dealloc(tmem, COLS);
}

template <bool E4M3, int TN, typename O, bool GATED>
static cudaError_t launch_few(const Few& f, int sms, cudaStream_t stream) {
  auto k = k_few<E4M3, TN, O, GATED>;
  static std::atomic<uint64_t> raised{0};
  cudaError_t e = raise_smem(reinterpret_cast<const void*>(k), FEW_SMEM<TN>, raised);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(f.tiles_n * ((f.T + TN - 1) / TN) * f.splits));
  cfg.blockDim = dim3(FEW_THREADS);
  cfg.dynamicSmemBytes = FEW_SMEM<TN>;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(f.splits);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = f.splits > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k, f);
}

template <bool E4M3, typename O, bool GATED>
static cudaError_t by_tokens(const Few& f, int tn, int sms, cudaStream_t stream) {
  switch (tn) {
    case 16: return launch_few<E4M3, 16, O, GATED>(f, sms, stream);
    case 32: return launch_few<E4M3, 32, O, GATED>(f, sms, stream);
    case 64: return launch_few<E4M3, 64, O, GATED>(f, sms, stream);
    default: return launch_few<E4M3, 128, O, GATED>(f, sms, stream);
  }
}
template <bool GATED>
static cudaError_t by_types(const Few& f, const Forward& a, int tn, int sms, cudaStream_t stream) {
  if (a.e4m3) return a.out_f32 ? by_tokens<true, float, GATED>(f, tn, sms, stream) : by_tokens<true, __nv_bfloat16, GATED>(f, tn, sms, stream);
  return a.out_f32 ? by_tokens<false, float, GATED>(f, tn, sms, stream) : by_tokens<false, __nv_bfloat16, GATED>(f, tn, sms, stream);
}

bool use_few(long long T, int kblocks) { return T <= 64 || (T <= 128 && kblocks >= 8) || (T <= 256 && kblocks >= 32); }

cudaError_t forward_few(const Forward& a, const void* x, long long xs, const void* w, long long ws, bool gated, unsigned int* err, int sms,
                        cudaStream_t stream) {
  const int es = a.e4m3 ? 1 : 2, os = a.out_f32 ? 4 : 2, tn = a.T <= 16 ? 16 : a.T <= 32 ? 32 : a.T <= 64 ? 64 : 128;
  Few f{};
  f.y = a.y, f.r = a.r, f.p = a.p, f.ys = a.ys, f.rs = a.rs, f.ps = a.ps;
  f.bias = a.bias, f.sx = a.x_scale, f.sw = a.w_scale;
  f.T = static_cast<int>(a.T), f.N = a.N, f.act = a.act, f.err = err;
  auto fours = [&](const void* p, long long stride, int size) {
    return !p || (reinterpret_cast<uintptr_t>(p) % (4 * size) == 0 && (a.T == 1 || stride % 4 == 0));
  };
  f.vec = fours(a.y, a.ys, os) && fours(a.r, a.rs, os) && fours(a.p, a.ps, 2) && !(gated && a.p && a.N % 4);
  f.kblocks = static_cast<int>((static_cast<long long>(a.K) * es + 127) / 128);
  const int out = gated ? FEW_ROWS / 2 : FEW_ROWS;
  f.tiles_n = (a.N + out - 1) / out;
  // the K axis over 1, 2, 4 or 8 CTAs while two CTAs an SM are not reached and each keeps two blocks
  const long long tiles = static_cast<long long>(f.tiles_n) * ((a.T + tn - 1) / tn);
  f.splits = 1;
  while (f.splits < 8 && tiles * f.splits * 2 <= 2ll * sms && f.kblocks >= 4 * f.splits) f.splits *= 2;
  // (gated: a pair of CTAs a tile costs more than it gives for more than a few tokens on a short K axis, or where the tiles alone nearly
  // fill the SMs.  One CTA and two, us, bf16, K and N: 1 token 1024, 5464 7.1 and 6.4; 32 tokens 1024, 8192 9.9 and 11.0; 64 tokens 1024,
  // 5464 11.1 and 13.1, 4096, 5464 26.5 and 25.9, 4096, 8192 30.2 and 31.7)
  if (gated && f.splits == 2 && ((a.T > 8 && f.kblocks < 32) || (a.T > 16 && 4 * tiles > 3ll * sms))) f.splits = 1;
  if (!tma::encode_rows(&f.tw, w, es, gated ? 2ll * a.N : a.N, a.K, ws, out) || !tma::encode_rows(&f.tx, x, es, a.T, a.K, xs, tn))
    return cudaErrorInvalidValue;
  return gated ? by_types<true>(f, a, tn, sms, stream) : by_types<false>(f, a, tn, sms, stream);
}

}  // namespace linear
}  // namespace whtmix
