// whtmix_gemm_dp.cu -- the linear layer's backward down to dx in one pass: dp = dy act'(p), the bias's partial sums and dx = dp W, for
// K <= 256, where one tile of columns holds all of dx's.
//
// One persistent CTA per SM, 512 threads, tiles of 128 tokens, N in blocks of 64 channels:
//   warp 0      TMA loads of a block of dy and p (128 x 64) and of W (64 rows of it, BN columns), three or four stages;
//   warps 8-15  read dy and p in shared memory, write bf16(dy act'(p)) over dy, where it lies as the product's operand wants it,
//               and add up the block's columns unrounded; the block also goes out to memory by TMA, for dw;
//   warp 1      four tcgen05.mma a block, dp with k along its rows, W with n along its rows, as they lie;
//   warps 4-7   the accumulator (two tiles' worth) to dx, as whtmix_gemm.cuh.
// Bound by memory: dy and p are read once and dp is written once, where a kernel for dp and a product that reads it again moved a
// third more.
#include "whtmix_gemm.cuh"

namespace whtmix {
namespace linear {

constexpr int DP_THREADS = 512;
template <int BN>
struct DpRing {
  static constexpr uint32_t TILE = 128 * 128, STAGE = 2 * TILE + BN * 128;
  static constexpr int STAGES = BN == 256 ? 3 : 4;
  static constexpr size_t SMEM = STAGES * STAGE + PANEL_BYTES;
};
template <int BN>
struct DpBars {
  uint64_t full[DpRing<BN>::STAGES], ready[DpRing<BN>::STAGES], empty[DpRing<BN>::STAGES], dfull[2], dempty[2];
};

template <int BN, int ACT>
__global__ void __launch_bounds__(DP_THREADS, 1) k_dx_dp(const __grid_constant__ DpProduct a) {
  using R = DpRing<BN>;
  constexpr int S = R::STAGES;
  constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | (static_cast<uint32_t>(BN >> 3) << 17) | ((128u >> 4) << 24);
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ DpBars<BN> bars;
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(16) float s_sum[2][8][64];  // the warps' column sums of a block, and of the next
  const uint32_t ring = tc::smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == 0) tc::tmem_alloc(&tmem_slot, 2 * BN);
  if (tid == 32) {
    for (int s = 0; s < S; ++s) {
      tc::mbar_init(&bars.full[s], 1);
      tc::mbar_init(&bars.ready[s], 1);
      tc::mbar_init(&bars.empty[s], a.store_dp ? 2 : 1);  // the products, and dp's way out
    }
    for (int s = 0; s < 2; ++s) tc::mbar_init(&bars.dfull[s], 1), tc::mbar_init(&bars.dempty[s], 4);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma::prefetch(&a.tdy);
    tma::prefetch(&a.tp);
    tma::prefetch(&a.tw);
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  pdl_wait();
  const uint32_t tmem = tmem_slot;
  unsigned bad = 0;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      for (int tile = blockIdx.x; tile < a.tiles_m && !bad; tile += gridDim.x)
        for (int kb = 0; kb < a.kblocks; ++kb, ++it) {
          const int s = it % S;
          if (!tma::wait(&bars.empty[s], ((it / S) & 1) ^ 1)) {
            bad |= 1;
            break;
          }
          const uint32_t st = ring + s * R::STAGE;
          tma::expect_tx(&bars.full[s], R::STAGE);
          tma::load_2d(st, &a.tdy, kb * 64, tile * GEMM_BM, &bars.full[s]);
          tma::load_2d(st + R::TILE, &a.tp, kb * 64, tile * GEMM_BM, &bars.full[s]);
#pragma unroll
          for (int i = 0; i < BN / 64; ++i) tma::load_2d(st + 2 * R::TILE + i * 8192, &a.tw, 64 * i, kb * 64, &bars.full[s]);
        }
      // the copies in flight have landed before the CTA can end
      for (uint32_t j = it > S ? it - S : 0; j < it; ++j)
        if (!tma::wait(&bars.full[j % S], (j / S) & 1)) bad |= 1;
    }
  } else if (warp == 1) {
    if (lane == 0) {
      uint32_t it = 0, i = 0;
      for (int tile = blockIdx.x; tile < a.tiles_m && !bad; tile += gridDim.x, ++i) {
        const int d = i & 1;
        if (!tma::wait(&bars.dempty[d], ((i >> 1) & 1) ^ 1)) {
          bad |= 2;
          break;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (int kb = 0; kb < a.kblocks; ++kb, ++it) {
          const int s = it % S;
          if (!tma::wait(&bars.ready[s], (it / S) & 1)) {
            bad |= 4;
            break;
          }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t sa = ring + s * R::STAGE, sb = sa + 2 * R::TILE;
#pragma unroll
          for (int ks = 0; ks < 4; ++ks)
            tc::mma_bf16(tmem + d * BN, tc::sw128_desc(sa + ks * 32), mn_major_desc(sb + ks * 2048, 8192), IDESC, kb > 0 || ks > 0);
          tc::mma_commit(&bars.empty[s]);
        }
        tc::mma_commit(&bars.dfull[d]);
      }
      // every product has completed before the tensor memory is freed
      for (uint32_t j = i > 2 ? i - 2 : 0; j < i; ++j)
        if (!tma::wait(&bars.dfull[j & 1], (j >> 1) & 1)) bad |= 2;
    }
  } else if (warp >= 8) {
    const int t = tid - 256, w = warp - 8, q = t & 7, r0 = t >> 3;  // 16 bytes q of rows r0, r0 + 32, ..
    uint32_t it = 0;
    int leaving = -1;  // thread 0: the stage whose dp is on its way out
    for (int tile = blockIdx.x; tile < a.tiles_m; tile += gridDim.x)
      for (int kb = 0; kb < a.kblocks; ++kb, ++it) {
        const int s = it % S;
        if (!bad && !tma::wait(&bars.full[s], (it / S) & 1)) bad |= 8;  // (after one wait has given up none is waited for)
        unsigned char* dy = smem + s * R::STAGE;
        float sum[8] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = r0 + 32 * i;
          const uint32_t at = r * 128 + ((q ^ (r & 7)) << 4);
          const uint4 u = *reinterpret_cast<const uint4*>(dy + at), v = *reinterpret_cast<const uint4*>(dy + R::TILE + at);
          const uint32_t du[4] = {u.x, u.y, u.z, u.w}, zu[4] = {v.x, v.y, v.z, v.w};
          uint32_t h[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float d0 = __uint_as_float(du[j] << 16), d1 = __uint_as_float(du[j] & 0xffff0000u);
            times_slope(d0, d1, __uint_as_float(zu[j] << 16), __uint_as_float(zu[j] & 0xffff0000u), ACT);
            sum[2 * j] += d0, sum[2 * j + 1] += d1;
            __nv_bfloat162 b = __floats2bfloat162_rn(d0, d1);
            h[j] = *reinterpret_cast<uint32_t*>(&b);
          }
          *reinterpret_cast<uint4*>(dy + at) = make_uint4(h[0], h[1], h[2], h[3]);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if (a.part) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 8);
            sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 16);
          }
          if (lane < 8) {
            float4* o = reinterpret_cast<float4*>(&s_sum[it & 1][w][8 * q]);
            o[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            o[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
          }
        }
        asm volatile("bar.sync 2, 256;" ::: "memory");
        if (t == 0) {
          tma::arrive(&bars.ready[s]);
          if (a.store_dp) {
            if (leaving >= 0) {
              tma::wait_read();
              tma::arrive(&bars.empty[leaving]);
            }
            tma::store_2d(&a.tdp, kb * 64, tile * GEMM_BM, ring + s * R::STAGE);
            tma::commit();
            leaving = s;
          }
        }
        if (a.part && t >= 64 && t < 128 && kb * 64 + t - 64 < a.N) {
          const int c = t - 64;
          float total = s_sum[it & 1][0][c];
#pragma unroll
          for (int k = 1; k < 8; ++k) total += s_sum[it & 1][k][c];
          a.part[static_cast<long long>(tile) * a.N + kb * 64 + c] = total;
        }
      }
    if (t == 0 && leaving >= 0) {
      tma::wait_done();
      tma::arrive(&bars.empty[leaving]);
    }
  } else if (warp >= 4) {
    const int gt = tid - 128, row = 32 * (warp & 3) + lane;
    unsigned char* st = smem + S * R::STAGE;
    const uint32_t lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16;
    uint32_t i = 0;
    for (int tile = blockIdx.x; tile < a.tiles_m; tile += gridDim.x, ++i) {
      const int d = i & 1, m0 = tile * GEMM_BM, panels = (a.K + 63) / 64;
      if (!bad && !tma::wait(&bars.dfull[d], (i >> 1) & 1)) bad |= 16;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      __syncwarp();
      for (int p = 0; p < panels; ++p) {
        float v[64];
        tmem_ld32(tmem + lanes + d * BN + p * 64, v);
        tmem_ld32(tmem + lanes + d * BN + p * 64 + 32, v + 32);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
        if (p + 1 == panels) {  // the accumulator has been read
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) tma::arrive(&bars.dempty[d]);
        }
        if (gt == 0) tma::wait_read();  // the last store has read the panel
        asm volatile("bar.sync 1, 128;" ::: "memory");
        panel_put<8>(st, row, 0, v, __nv_bfloat16());
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (a.dx_plain) {
          panel_plain<__nv_bfloat16, true>(st, a.dx, a.dxs, m0, a.M, p * 64, a.K, gt);
        } else if (gt == 0) {
          tma::store_2d(&a.tdx, p * 64, m0, tc::smem_u32(st));
          tma::commit();
        }
      }
    }
    if (gt == 0) tma::wait_done();
  }
  if (bad) atomicOr(a.err, bad << 8);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  pdl_trigger();
  if (warp == 0) tc::tmem_dealloc(tmem, 2 * BN);
}

template <int BN, int ACT>
static cudaError_t launch(const DpProduct& g, int sms, cudaStream_t stream) {
  const void* k = reinterpret_cast<const void*>(k_dx_dp<BN, ACT>);
  static std::atomic<uint64_t> raised{0};
  const cudaError_t e = raise_smem(k, DpRing<BN>::SMEM, raised);
  if (e != cudaSuccess) return e;
  DpProduct c = g;
  void* args[] = {&c};
  return launch_pdl(k, static_cast<unsigned>(g.tiles_m < sms ? g.tiles_m : sms), DP_THREADS, DpRing<BN>::SMEM, stream, args);
}
template <int BN>
static cudaError_t by_act(const DpProduct& g, int sms, cudaStream_t stream) {
  switch (g.act) {
    case ACT_RELU: return launch<BN, ACT_RELU>(g, sms, stream);
    case ACT_GELU: return launch<BN, ACT_GELU>(g, sms, stream);
    case ACT_SILU: return launch<BN, ACT_SILU>(g, sms, stream);
    default: return cudaErrorInvalidValue;
  }
}
cudaError_t gemm_dp(const DpProduct& g, int sms, cudaStream_t stream) {
  return g.K <= 64 ? by_act<64>(g, sms, stream) : g.K <= 128 ? by_act<128>(g, sms, stream) : by_act<256>(g, sms, stream);
}

}  // namespace linear
}  // namespace whtmix
