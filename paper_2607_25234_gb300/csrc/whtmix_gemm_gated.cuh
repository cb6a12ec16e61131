// whtmix_gemm_gated.cuh -- both products of a gated feed-forward half, its activation and their product in one kernel.
//
//   g = s_m s_n sum over k of A[m, k] B[n, k] + b_n,   u = the same with row N + n of B,   y = act(g) u          (p = [g, u])
//
// whtmix_gemm.cuh's pipeline (warp 0 loads, warp 1 issues tcgen05 products, epilogue groups on alternate tiles), with a tile's B of
// OUT rows of the gate's weights and the OUT rows of the value's that belong to the same channels: column c of the accumulator is the
// gate, column OUT + c the value of output channel n0 + c.  A is read once for both, and neither g nor u goes out to memory where p
// is not wanted.  OUT = 64 or 128 (accumulators of 128 or 256 columns); PAIR: two CTAs on 256 x 128 channels, the first one's rows of B
// the gate's, the second one's the value's.
// Gate rows read past N (the last tile's) are the value's first ones: their columns are never stored.
#pragma once

#include "whtmix_gemm.cuh"

namespace whtmix {
namespace linear {

struct Gated {
  CUtensorMap ta, tb, ty, tg, tu;  // tg, tu: the halves of p
  // plain accesses where a matrix has no tensor map (elements, strides in elements)
  void* y;
  void* p;
  long long ys, ps;
  const float *bias, *sm, *sn;  // sm, sn: scales of the rows of A and B, or null
  int M, N, kblocks, tiles_m, tiles_n, band, act;
  bool has_p, y_plain, p_plain;
  unsigned int* err;
};

// d0 = d0 u0 act'(z0), v0 = d0 act(z0), and the same for the other value (one logistic function for value and slope; limits as in
// activate and times_slope).
__device__ __forceinline__ void gate_gradients(float& d0, float& d1, float& v0, float& v1, float z0, float z1, float u0, float u1, int act) {
  v0 = d0, v1 = d1;
  d0 *= u0, d1 *= u1;
  if (act == ACT_NONE) {
    v0 *= z0, v1 *= z1;
  } else if (act == ACT_RELU) {
    v0 *= z0 < 0.f ? 0.f : z0, v1 *= z1 < 0.f ? 0.f : z1;
    d0 = z0 > 0.f ? d0 : d0 * 0.f, d1 = z1 > 0.f ? d1 : d1 * 0.f;
  } else {
    const Pair zv = pair(above(z0, GATE_LOW), above(z1, GATE_LOW)), z = pair(between(z0, GATE_LOW, GATE_HIGH), between(z1, GATE_LOW, GATE_HIGH));
    const Logistic l = logistic2(gate_exponent(z, act));
    Pair g = z * (l.e * l.s);
    if (act == ACT_GELU) g = g * fma(z * z, pair(3.f * GELU_2A * GELU_B, 3.f * GELU_2A * GELU_B), pair(GELU_2A, GELU_2A));
    unpair(pair(d0, d1) * (l.s * (g + pair(1.f, 1.f))), d0, d1);
    unpair(pair(v0, v1) * (zv * l.s), v0, v1);
  }
}

// (the ring, two panels and what is declared here are an SM's 227 KB to the last: one set of biases and scales a group)
template <bool E4M3, int BN, bool PAIR, int GROUPS, typename O>
__global__ void __launch_bounds__(GEMM_THREADS<GROUPS>, 1) k_gated(const __grid_constant__ Gated a) {
  static_assert(!PAIR || BN == 256, "a pair's tile is 256 x 256");
  static_assert(GROUPS == 2 || (GROUPS == 4 && !PAIR), "two or four epilogue groups");
  constexpr int OUT = BN / 2, TEAM = GROUPS / 2;  // groups on a tile
  using R = Ring<BN, PAIR, GROUPS>;
  constexpr int CTAS = PAIR ? 2 : 1, TILE_M = CTAS * GEMM_BM;
  constexpr int S = R::STAGES, BK = E4M3 ? 128 : 64, PW = Panel<O>::W, PANELS = OUT / PW;
  constexpr uint32_t IDESC = (1u << 4) | (E4M3 ? 0u : (1u << 7) | (1u << 10)) | (static_cast<uint32_t>(BN >> 3) << 17) |
                             (static_cast<uint32_t>(TILE_M >> 4) << 24);
  constexpr int CH = GROUPS == 2 ? 32 : 16, Q = CH * static_cast<int>(sizeof(O)) / 16;  // columns of each half in registers, their pieces
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ GemmBars<BN, PAIR, GROUPS> bars;
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(16) float s_bias[GROUPS][2][PW], s_scale[GROUPS][2][PW];  // of a group's panel: gate, value
  const uint32_t ring = tc::smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int items = a.tiles_m * a.tiles_n;
  const int unit = blockIdx.x / CTAS, units = gridDim.x / CTAS, rank = PAIR ? blockIdx.x % 2 : 0;
  const bool alternate = items > units;
  if (warp == 0) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(&tmem_slot)), "r"(2 * BN) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      tc::tmem_alloc(&tmem_slot, 2 * BN);
    }
  }
  if (tid == 32) {
    for (int s = 0; s < S; ++s) tc::mbar_init(&bars.full[s], 1), tc::mbar_init(&bars.empty[s], 1);
    for (int s = 0; s < 2; ++s) tc::mbar_init(&bars.dfull[s], 1), tc::mbar_init(&bars.dempty[s], CTAS * (alternate ? 4 * TEAM : 4 * GROUPS));
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma::prefetch(&a.ta);
    tma::prefetch(&a.tb);
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if constexpr (PAIR) tma::cluster_sync();  // the other CTA's barriers are set up
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  pdl_wait();
  const uint32_t tmem = tmem_slot;
  // item -> tile: bands of `band` tiles down, m fastest in a band, so that the tiles at work together are a near square of the output
  // ([8192, 4096] to 8192, whose W does not fit L2: 660 us a row of tiles at a time, 570 in bands of 16)
  auto place = [&](int item, int& m0, int& n0) {
    const int per = a.band * a.tiles_n, b = item / per, i = item - b * per, rows = min(a.band, a.tiles_m - b * a.band), n = i / rows;
    m0 = (b * a.band + i - n * rows) * TILE_M + rank * GEMM_BM;  // this CTA's rows
    n0 = n * OUT;
  };
  unsigned bad = 0;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      for (int item = unit; item < items && !bad; item += units) {
        int m0, n0;
        place(item, m0, n0);
        for (int kb = 0; kb < a.kblocks; ++kb, ++it) {
          const int s = it % S;
          if (!tma::wait(&bars.empty[s], ((it / S) & 1) ^ 1)) {
            bad |= 1;
            break;
          }
          const uint32_t sa = ring + s * R::STAGE, sb = sa + R::A;
          if (rank == 0) tma::expect_tx(&bars.full[s], CTAS * R::STAGE);
          if constexpr (PAIR) {
            const uint32_t full = tma::in_cta(tc::smem_u32(&bars.full[s]), 0);
            tma::load_2d_pair(sa, &a.ta, kb * BK, m0, full);
            tma::load_2d_pair(sb, &a.tb, kb * BK, rank * a.N + n0, full);
          } else {
            tma::load_2d(sa, &a.ta, kb * BK, m0, &bars.full[s]);
            tma::load_2d(sb, &a.tb, kb * BK, n0, &bars.full[s]);
            tma::load_2d(sb + OUT * 128, &a.tb, kb * BK, a.N + n0, &bars.full[s]);
          }
        }
      }
      // the copies in flight have landed before the CTA can end
      for (uint32_t j = it > S ? it - S : 0; rank == 0 && j < it; ++j)
        if (!tma::wait(&bars.full[j % S], (j / S) & 1)) bad |= 1;
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      uint32_t it = 0, i = 0;
      for (int item = unit; item < items && !bad; item += units, ++i) {
        const int d = i & 1;
        if (!tma::wait(&bars.dempty[d], ((i >> 1) & 1) ^ 1)) {
          bad |= 2;
          break;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (int kb = 0; kb < a.kblocks; ++kb, ++it) {
          const int s = it % S;
          if (!tma::wait(&bars.full[s], (it / S) & 1)) {
            bad |= 4;
            break;
          }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t sa = ring + s * R::STAGE, sb = sa + R::A;
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {  // 32 bytes of k
            const uint64_t da = tc::sw128_desc(sa + ks * 32), db = tc::sw128_desc(sb + ks * 32);
            const uint32_t acc = kb > 0 || ks > 0;
            if constexpr (PAIR)
              mma_pair<E4M3>(tmem + d * BN, da, db, IDESC, acc);
            else if constexpr (E4M3)
              mma_e4m3(tmem + d * BN, da, db, IDESC, acc);
            else
              tc::mma_bf16(tmem + d * BN, da, db, IDESC, acc);
          }
          if constexpr (PAIR) commit_pair(&bars.empty[s]); else tc::mma_commit(&bars.empty[s]);
        }
        if constexpr (PAIR) commit_pair(&bars.dfull[d]); else tc::mma_commit(&bars.dfull[d]);
      }
      // every product has completed before the tensor memory is freed
      for (uint32_t j = i > 2 ? i - 2 : 0; j < i; ++j)
        if (!tma::wait(&bars.dfull[j & 1], (j >> 1) & 1)) bad |= 2;
    }
  } else if (warp >= 4) {
    const int g = (warp - 4) >> 2, gt = tid - 128 - 128 * g, row = 32 * (warp & 3) + lane;
    unsigned char* st = smem + RING_BYTES<GROUPS> + g * PANEL_BYTES;
    const uint32_t st_u = tc::smem_u32(st), lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16;
    auto sync_group = [&] { asm volatile("bar.sync %0, 128;" ::"r"(1 + g) : "memory"); };
    auto wait = [&](uint64_t* b, uint32_t parity) {  // (after one wait has given up none is waited for)
      if (!bad && !tma::wait(b, parity)) bad |= 8;
    };
    // the group's tiles (a CTA with one tile: its every other panel), and of the next one's columns gt, gt + 128 the bias and scale, of
    // its row the scale: on their way while a tile is stored
    const int step = alternate ? TEAM : GROUPS, p0 = alternate ? g % TEAM : g, stride = alternate ? 2 * units : units;
    auto accumulator_read = [&](int d) {
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        if constexpr (PAIR)
          tma::arrive_in(tma::in_cta(tc::smem_u32(&bars.dempty[d]), 0));
        else
          tma::arrive(&bars.dempty[d]);
      }
    };
    constexpr int HELD = BN / 128;
    float next_bias[HELD], next_scale[HELD], next_sm = 1.f;
    auto fetch = [&](int item) {
      if (item >= items) return;
      int m0, n0;
      place(item, m0, n0);
#pragma unroll
      for (int j = 0; j < HELD; ++j) {
        const int c = 128 * j + gt, n = n0 + c % OUT, r = c < OUT ? n : a.N + n;
        next_bias[j] = a.bias && n < a.N ? __ldg(a.bias + r) : 0.f;
        next_scale[j] = a.sn && n < a.N ? __ldg(a.sn + r) : 1.f;
      }
      if (a.sm) next_sm = m0 + row < a.M ? __ldg(a.sm + m0 + row) : 1.f;
    };
    const int first = unit + (alternate ? g / TEAM * units : 0);
    uint32_t i = alternate ? g / TEAM : 0;
    fetch(first);
    for (int item = first; item < items; item += stride, i += alternate ? 2 : 1) {
      int m0, n0;
      place(item, m0, n0);
      const int d = i & 1, panels = min(PANELS, (a.N - n0 + PW - 1) / PW);
      const float sm = next_sm;
      bool waited = false;
      float bias[HELD], scale[HELD];
#pragma unroll
      for (int j = 0; j < HELD; ++j) bias[j] = next_bias[j], scale[j] = next_scale[j];
      fetch(item + stride);
      for (int p = p0; p < panels; p += step) {
        const int col0 = n0 + p * PW;
        // the panel's columns' bias and scale, by the threads that hold them (the last panel's readers are behind its barrier)
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
          const int c = (128 * j + gt) % OUT - p * PW, half = (128 * j + gt) / OUT;
          if (c >= 0 && c < PW) s_bias[g][half][c] = bias[j], s_scale[g][half][c] = scale[j];
        }
        sync_group();
        auto panel_free = [&] {  // the last store has read the panel
          if (gt == 0) tma::wait_read();
          sync_group();
        };
        if (!waited) {
          wait(&bars.dfull[d], (i >> 1) & 1);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          waited = true;
        }
        // columns c0 .. of the panel in one half, scaled, with their bias
        auto load = [&](int half, int c0, float (&v)[CH]) {
          const uint32_t from = tmem + lanes + d * BN + half * OUT + p * PW + c0;
          if constexpr (CH == 32)
            tmem_ld32(from, v);
          else
            tc::tmem_ld16(from, v);
        };
        auto finish = [&](int half, int c0, float (&v)[CH]) {
          if (a.sm) {
            const float* ss = s_scale[g][half] + c0;
#pragma unroll
            for (int c = 0; c < CH; c += 4) {
              const float4 s = *reinterpret_cast<const float4*>(ss + c);
              unpair(pair(v[c], v[c + 1]) * (pair(sm, sm) * pair(s.x, s.y)), v[c], v[c + 1]);
              unpair(pair(v[c + 2], v[c + 3]) * (pair(sm, sm) * pair(s.z, s.w)), v[c + 2], v[c + 3]);
            }
          }
          if (a.bias) {
            const float* sb = s_bias[g][half] + c0;
#pragma unroll
            for (int c = 0; c < CH; c += 4) {
              const float4 b = *reinterpret_cast<const float4*>(sb + c);
              unpair(pair(v[c], v[c + 1]) + pair(b.x, b.y), v[c], v[c + 1]);
              unpair(pair(v[c + 2], v[c + 3]) + pair(b.z, b.w), v[c + 2], v[c + 3]);
            }
          }
        };
        if constexpr (PW == 64) {
          if (a.has_p) {
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
              panel_free();
#pragma unroll
              for (int c0 = 0; c0 < PW; c0 += CH) {
                float v[CH];
                __syncwarp();
                load(half, c0, v);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                finish(half, c0, v);
                panel_put<Q>(st, row, c0 / 8, v, O());
              }
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              sync_group();
              if (a.p_plain) {
                panel_plain<__nv_bfloat16, true>(st, static_cast<__nv_bfloat16*>(a.p) + static_cast<long long>(half) * a.N, a.ps, m0, a.M, col0, a.N, gt);
              } else if (gt == 0 && (!PAIR || m0 < a.M)) {
                tma::store_2d(half ? &a.tu : &a.tg, col0, m0, st_u);
                tma::commit();
              }
            }
          }
        }
#pragma unroll
        for (int c0 = 0; c0 < PW; c0 += CH) {
          float v[CH], u[CH];
          __syncwarp();
          load(0, c0, v);
          load(1, c0, u);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          if (c0 + CH == PW && p + step >= panels) accumulator_read(d);
          finish(0, c0, v);
          finish(1, c0, u);
          switch (a.act) {
#define WHTMIX_ACT(A)                                             \
  case A:                                                         \
    _Pragma("unroll") for (int c = 0; c < CH; c += 2) activate(v[c], v[c + 1], A); \
    break
            WHTMIX_ACT(ACT_RELU);
            WHTMIX_ACT(ACT_GELU);
            WHTMIX_ACT(ACT_SILU);
#undef WHTMIX_ACT
            default: break;
          }
#pragma unroll
          for (int c = 0; c < CH; c += 2) unpair(pair(v[c], v[c + 1]) * pair(u[c], u[c + 1]), v[c], v[c + 1]);
          if (c0 == 0) panel_free();
          panel_put<Q>(st, row, c0 * static_cast<int>(sizeof(O)) / 16, v, O());
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        sync_group();
        if (a.y_plain) {
          panel_plain<O, true>(st, a.y, a.ys, m0, a.M, col0, a.N, gt);
        } else if (gt == 0 && (!PAIR || m0 < a.M)) {
          tma::store_2d(&a.ty, col0, m0, st_u);
          tma::commit();
        }
      }
      if (!waited) {  // no panel of this tile for this group
        wait(&bars.dfull[d], (i >> 1) & 1);
        accumulator_read(d);
      }
    }
    if (gt == 0) tma::wait_done();
  }
  if (bad) atomicOr(a.err, bad << 16);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if constexpr (PAIR) tma::cluster_sync();  // neither CTA ends while the other's products or arrivals reach into it
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  pdl_trigger();
  if (warp == 0) {
    if constexpr (PAIR)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * BN) : "memory");
    else
      tc::tmem_dealloc(tmem, 2 * BN);
  }
}

// One instance's launch: a persistent grid of at most one CTA per SM.
template <bool E4M3, int BN, bool PAIR, typename O, int GROUPS = 2>
cudaError_t launch_gated(const Gated& g, int sms, cudaStream_t stream) {
  auto k = k_gated<E4M3, BN, PAIR, GROUPS, O>;
  static std::atomic<uint64_t> raised{0};
  const cudaError_t e = raise_smem(reinterpret_cast<const void*>(k), GEMM_SMEM<GROUPS>, raised);
  if (e != cudaSuccess) return e;
  constexpr int CTAS = PAIR ? 2 : 1;
  const long long items = static_cast<long long>(g.tiles_m) * g.tiles_n, most = sms / CTAS;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(CTAS * (items < most ? items : most)));
  cfg.blockDim = dim3(GEMM_THREADS<GROUPS>);
  cfg.dynamicSmemBytes = GEMM_SMEM<GROUPS>;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CTAS;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CTAS;
  return cudaLaunchKernelEx(&cfg, k, g);
}

// By accumulator width: 128, 256, or TILE_PAIR; `four` epilogue groups only with 256.
template <bool E4M3, typename O>
cudaError_t gated_by_width(const Gated& g, int bn, bool four, int sms, cudaStream_t stream) {
  switch (bn) {
    case 128: return launch_gated<E4M3, 128, false, O>(g, sms, stream);
    case 256: return four ? launch_gated<E4M3, 256, false, O, 4>(g, sms, stream) : launch_gated<E4M3, 256, false, O>(g, sms, stream);
    default: return launch_gated<E4M3, 256, true, O>(g, sms, stream);
  }
}

// whtmix_gemm_gated_dp.cu: dp = [dg, du], its column sums and dx = dp W in one pass, for K <= 256 (one tile of columns).
// part [tiles_m, 2 N]: the 128-token tiles' sums of unrounded dp, or null; tdg, tdu, dp's halves, are written where store_dp.
struct GatedDp {
  CUtensorMap tdy, tg, tu, twg, twu, tdg, tdu, tdx;
  float* part;
  void* dx;
  long long dxs;
  int M, N, K, tiles_m, kblocks, act;
  bool store_dp, dx_plain;
  unsigned int* err;
};
cudaError_t gemm_gated_dp(const GatedDp& g, int sms, cudaStream_t stream);

// whtmix_gemm_gated.cu, whtmix_gemm_gated_e4m3.cu
cudaError_t gemm_gated(const Gated& g, bool out_f32, int bn, bool four, int sms, cudaStream_t stream);
cudaError_t gemm_gated_e4m3(const Gated& g, bool out_f32, int bn, bool four, int sms, cudaStream_t stream);

}  // namespace linear
}  // namespace whtmix
