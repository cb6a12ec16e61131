// whtmix_gemm_gated_dp.cu -- the gated half's backward down to dx in one pass: dp = [dg, du] = [dy u act'(g), dy act(g)], the bias's partial
// sums and dx = dg Wg + du Wu, for K <= 256, where one tile of columns holds all of dx's.
//
// One persistent CTA per SM, 512 threads, tiles of 128 tokens, the hidden channels in blocks of 64:
//   warp 0      TMA loads of a block of dy, g and u (128 x 64 each), two or three stages;
//   warp 2      TMA loads of its rows of Wg and of Wu (64 rows of BN columns each), a ring of three;
//   warps 8-15  read the block in shared memory, write bf16 dg over g and du over u, where they lie as the products' operand wants
//               them (why in bf16: k_gated_dp), and add up the block's columns unrounded;
//   warp 3      both go out to memory by TMA as well, for dw (a warp of its own: the stage is free again as soon as they have left);
//   warp 1      four tcgen05.mma for each of the two, dg and du with k along their rows, W with n along its rows, as they lie;
//   warps 4-7   the accumulator (two tiles' worth) to dx, as whtmix_gemm.cuh.
// Bound by memory: dy and p are read once and dp is written once, where a kernel for dp and a product that reads it again move a third more.
#include "whtmix_gemm_gated.cuh"

namespace whtmix {
namespace linear {

constexpr int GDP_THREADS = 512;
template <int BN>
struct GdpRing {
  // ([65536, 128] to 344, two and three stages: 85.4 and 76.9 us.  256 columns, [131072, 256] to 688: W's units of 32 KB leave room for
  // two stages, 258 us; three stages and units of 16 KB 297; three stages, two units and dx stored from the registers 260; pairs of CTAs
  // that share W, three stages 279)
  static constexpr int STAGES = BN == 256 ? 2 : 3, UNITS = 3;
  static constexpr uint32_t TILE = 128 * 128, STAGE = 3 * TILE, UNIT = BN * 128;
  static constexpr uint32_t W = STAGES * STAGE, PANEL = W + UNITS * UNIT;
  static constexpr size_t SMEM = PANEL + PANEL_BYTES;
};
template <int BN>
struct GdpBars {
  uint64_t full[GdpRing<BN>::STAGES], ready[GdpRing<BN>::STAGES], empty[GdpRing<BN>::STAGES];
  uint64_t wfull[GdpRing<BN>::UNITS], wempty[GdpRing<BN>::UNITS], dfull[2], dempty[2];
};

template <int BN, int ACT>
__global__ void __launch_bounds__(GDP_THREADS, 1) k_dx_gated(const __grid_constant__ GatedDp a) {
  using R = GdpRing<BN>;
  constexpr int S = R::STAGES, U = R::UNITS;
  constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | (static_cast<uint32_t>(BN >> 3) << 17) | ((128u >> 4) << 24);
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ GdpBars<BN> bars;
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(16) float s_sum[2][8][128];  // the warps' column sums of a block, dg's and du's, and of the next
  const uint32_t ring = tc::smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == 0) tc::tmem_alloc(&tmem_slot, 2 * BN);
  if (tid == 32) {
    for (int s = 0; s < S; ++s) {
      tc::mbar_init(&bars.full[s], 1);
      tc::mbar_init(&bars.ready[s], 1);
      tc::mbar_init(&bars.empty[s], a.store_dp ? 2 : 1);  // the products, and dp's way out
    }
    for (int s = 0; s < U; ++s) tc::mbar_init(&bars.wfull[s], 1), tc::mbar_init(&bars.wempty[s], 1);
    for (int s = 0; s < 2; ++s) tc::mbar_init(&bars.dfull[s], 1), tc::mbar_init(&bars.dempty[s], 4);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma::prefetch(&a.tdy);
    tma::prefetch(&a.tg);
    tma::prefetch(&a.tu);
    tma::prefetch(&a.twg);
    tma::prefetch(&a.twu);
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
          tma::load_2d(st + R::TILE, &a.tg, kb * 64, tile * GEMM_BM, &bars.full[s]);
          tma::load_2d(st + 2 * R::TILE, &a.tu, kb * 64, tile * GEMM_BM, &bars.full[s]);
        }
      // the copies in flight have landed before the CTA can end
      for (uint32_t j = it > S ? it - S : 0; j < it; ++j)
        if (!tma::wait(&bars.full[j % S], (j / S) & 1)) bad |= 1;
    }
  } else if (warp == 2) {
    if (lane == 0) {
      uint32_t it = 0;
      for (int tile = blockIdx.x; tile < a.tiles_m && !bad; tile += gridDim.x)
        for (int u = 0; u < 2 * a.kblocks; ++u, ++it) {
          const int s = it % U;
          if (!tma::wait(&bars.wempty[s], ((it / U) & 1) ^ 1)) {
            bad |= 1;
            break;
          }
          const uint32_t st = ring + R::W + s * R::UNIT;
          tma::expect_tx(&bars.wfull[s], R::UNIT);
#pragma unroll
          for (int i = 0; i < BN / 64; ++i) tma::load_2d(st + i * 8192, u & 1 ? &a.twu : &a.twg, 64 * i, (u >> 1) * 64, &bars.wfull[s]);
        }
      for (uint32_t j = it > U ? it - U : 0; j < it; ++j)
        if (!tma::wait(&bars.wfull[j % U], (j / U) & 1)) bad |= 1;
    }
  } else if (warp == 1) {
    if (lane == 0) {
      uint32_t it = 0, wit = 0, i = 0;
      for (int tile = blockIdx.x; tile < a.tiles_m && !bad; tile += gridDim.x, ++i) {
        const int d = i & 1;
        if (!tma::wait(&bars.dempty[d], ((i >> 1) & 1) ^ 1)) {
          bad |= 2;
          break;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (int kb = 0; kb < a.kblocks && !bad; ++kb, ++it) {
          const int s = it % S;
          if (!tma::wait(&bars.ready[s], (it / S) & 1)) {
            bad |= 4;
            break;
          }
#pragma unroll
          for (int half = 0; half < 2; ++half, ++wit) {
            const int w = wit % U;
            if (!tma::wait(&bars.wfull[w], (wit / U) & 1)) {
              bad |= 4;
              break;
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t sa = ring + s * R::STAGE + (1 + half) * R::TILE, sb = ring + R::W + w * R::UNIT;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              tc::mma_bf16(tmem + d * BN, tc::sw128_desc(sa + ks * 32), mn_major_desc(sb + ks * 2048, 8192), IDESC, kb > 0 || half > 0 || ks > 0);
            tc::mma_commit(&bars.wempty[w]);
          }
          tc::mma_commit(&bars.empty[s]);
        }
        tc::mma_commit(&bars.dfull[d]);
      }
      // every product has completed before the tensor memory is freed
      for (uint32_t j = i > 2 ? i - 2 : 0; j < i; ++j)
        if (!tma::wait(&bars.dfull[j & 1], (j >> 1) & 1)) bad |= 2;
    }
  } else if (warp == 3) {
    if (lane == 0 && a.store_dp) {
      uint32_t it = 0;
      for (int tile = blockIdx.x; tile < a.tiles_m && !bad; tile += gridDim.x)
        for (int kb = 0; kb < a.kblocks; ++kb, ++it) {
          const int s = it % S;
          if (!tma::wait(&bars.ready[s], (it / S) & 1)) {
            bad |= 8;
            break;
          }
          tma::store_2d(&a.tdg, kb * 64, tile * GEMM_BM, ring + s * R::STAGE + R::TILE);
          tma::store_2d(&a.tdu, kb * 64, tile * GEMM_BM, ring + s * R::STAGE + 2 * R::TILE);
          tma::commit();
          tma::wait_read();
          tma::arrive(&bars.empty[s]);
        }
      tma::wait_done();
    }
  } else if (warp >= 8) {
    const int t = tid - 256, w = warp - 8, q = t & 7, r0 = t >> 3;  // 16 bytes q of rows r0, r0 + 32, ..
    uint32_t it = 0;
    for (int tile = blockIdx.x; tile < a.tiles_m; tile += gridDim.x)
      for (int kb = 0; kb < a.kblocks; ++kb, ++it) {
        const int s = it % S;
        if (!bad && !tma::wait(&bars.full[s], (it / S) & 1)) bad |= 8;  // (after one wait has given up none is waited for)
        unsigned char* dy = smem + s * R::STAGE;
        float sum_g[8] = {}, sum_u[8] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = r0 + 32 * i;
          const uint32_t at = r * 128 + ((q ^ (r & 7)) << 4);
          const uint4 dv = *reinterpret_cast<const uint4*>(dy + at), gv = *reinterpret_cast<const uint4*>(dy + R::TILE + at),
                      uv = *reinterpret_cast<const uint4*>(dy + 2 * R::TILE + at);
          const uint32_t dw[4] = {dv.x, dv.y, dv.z, dv.w}, gw[4] = {gv.x, gv.y, gv.z, gv.w}, uw[4] = {uv.x, uv.y, uv.z, uv.w};
          uint32_t hg[4], hu[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float d0 = __uint_as_float(dw[j] << 16), d1 = __uint_as_float(dw[j] & 0xffff0000u), v0, v1;
            gate_gradients(d0, d1, v0, v1, __uint_as_float(gw[j] << 16), __uint_as_float(gw[j] & 0xffff0000u), __uint_as_float(uw[j] << 16),
                           __uint_as_float(uw[j] & 0xffff0000u), ACT);
            sum_g[2 * j] += d0, sum_g[2 * j + 1] += d1;
            sum_u[2 * j] += v0, sum_u[2 * j + 1] += v1;
            __nv_bfloat162 b = __floats2bfloat162_rn(d0, d1), c = __floats2bfloat162_rn(v0, v1);
            hg[j] = *reinterpret_cast<uint32_t*>(&b), hu[j] = *reinterpret_cast<uint32_t*>(&c);
          }
          *reinterpret_cast<uint4*>(dy + R::TILE + at) = make_uint4(hg[0], hg[1], hg[2], hg[3]);
          *reinterpret_cast<uint4*>(dy + 2 * R::TILE + at) = make_uint4(hu[0], hu[1], hu[2], hu[3]);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if (a.part) {
          // four lanes hold sums of the same 16 columns: each pass hands half of them over, so that each ends with four columns' sums
          float h[8], o[4];
          const bool up = lane & 8, top = lane & 16;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float other = __shfl_xor_sync(0xffffffffu, up ? sum_g[j] : sum_u[j], 8);
            h[j] = (up ? sum_u[j] : sum_g[j]) + other;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float other = __shfl_xor_sync(0xffffffffu, top ? h[j] : h[4 + j], 16);
            o[j] = (top ? h[4 + j] : h[j]) + other;
          }
          *reinterpret_cast<float4*>(&s_sum[it & 1][w][(up ? 64 : 0) + 8 * q + (top ? 4 : 0)]) = make_float4(o[0], o[1], o[2], o[3]);
        }
        asm volatile("bar.sync 2, 256;" ::: "memory");
        if (t == 0) tma::arrive(&bars.ready[s]);
        if (a.part && t >= 128 && kb * 64 + (t & 63) < a.N) {
          const int c = t - 128;
          float total = s_sum[it & 1][0][c];
#pragma unroll
          for (int k = 1; k < 8; ++k) total += s_sum[it & 1][k][c];
          a.part[static_cast<long long>(tile) * 2 * a.N + (c < 64 ? 0 : a.N) + kb * 64 + (c & 63)] = total;
        }
      }
  } else if (warp >= 4) {
    const int gt = tid - 128, row = 32 * (warp & 3) + lane;
    unsigned char* st = smem + R::PANEL;
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
static cudaError_t launch(const GatedDp& g, int sms, cudaStream_t stream) {
  const void* k = reinterpret_cast<const void*>(k_dx_gated<BN, ACT>);
  static std::atomic<uint64_t> raised{0};
  const cudaError_t e = raise_smem(k, GdpRing<BN>::SMEM, raised);
  if (e != cudaSuccess) return e;
  GatedDp c = g;
  void* args[] = {&c};
  return launch_pdl(k, static_cast<unsigned>(g.tiles_m < sms ? g.tiles_m : sms), GDP_THREADS, GdpRing<BN>::SMEM, stream, args);
}
template <int BN>
static cudaError_t by_act(const GatedDp& g, int sms, cudaStream_t stream) {
  switch (g.act) {
    case ACT_NONE: return launch<BN, ACT_NONE>(g, sms, stream);
    case ACT_RELU: return launch<BN, ACT_RELU>(g, sms, stream);
    case ACT_GELU: return launch<BN, ACT_GELU>(g, sms, stream);
    default: return launch<BN, ACT_SILU>(g, sms, stream);
  }
}
cudaError_t gemm_gated_dp(const GatedDp& g, int sms, cudaStream_t stream) {
  return g.K <= 64 ? by_act<64>(g, sms, stream) : g.K <= 128 ? by_act<128>(g, sms, stream) : by_act<256>(g, sms, stream);
}

}  // namespace linear
}  // namespace whtmix
