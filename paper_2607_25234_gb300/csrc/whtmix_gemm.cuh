// whtmix_gemm.cuh -- matrix products on the 5th-generation tensor cores with the linear layer's epilogue.
//
//   C[m, n] = sum over k of A[m, k] B[n, k]        y = act(s_m s_n C + b_n) + r
//
// One persistent CTA per SM, 384 or 640 threads, tiles of 128 x BN (BN = 64, 128, 256) in turn, the K axis in blocks of 128 bytes:
//   warp 0     TMA loads of A and B blocks into a ring of stages (192 or 144 KB in all);
//   warp 1     four tcgen05.mma a block (fp32 accumulators in tensor memory, two tiles' worth: the next tile's products run
//              while the last one's accumulator is read);
//   warps 4-11 epilogue, two groups of four warps, which take every other tile (a CTA with one tile: every other panel of it); a
//   (4-19)     panel is 128 bytes of each of the 128 rows: accumulator -> registers, the epilogue, shared memory, TMA store.  Four
//              groups: two to a tile, 32 columns at a time in registers.
//              On panels of one tile both groups work in step and wait for the special-function unit together; a tile apart,
//              one's stores cover the other's arithmetic.
// A and B may lie with k along a row (the forward; A of dx = dp W) or with m / n along a row (B of dx; both of dw = dp^T x, the
// contraction down the rows): the panels are multiplied as they lie.  What lies past an edge reads as zero and is not stored, so
// that every size runs; rows that are not 16-byte aligned are stored (and the residual read) with plain accesses, through the
// same shared-memory panel.
// PAIR: the two CTAs of a cluster share a tile of 256 x 256.  Each loads its 128 rows of A and 128 of the 256 rows of B, the first
// one's warp 1 issues cta_group::2 products that read both CTAs' shared memory, and each CTA's tensor memory takes its 128 rows:
// a third less comes from L2 and out of shared memory than with two tiles of 128 x 256.
// Splits: item s of a split tile takes its share of the K blocks and stores fp32 partial rows [s * split_rows + m] (added to a
// residual that lies the same way); the caller adds them up in a fixed order.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "whtmix_kernels.cuh"
#include "whtmix_linear.cuh"
#include "whtmix_tc.cuh"
#include "whtmix_tma.cuh"

namespace whtmix {
namespace linear {

struct Gemm {
  CUtensorMap ta, tb, ty, tr, tp;
  // plain accesses where a matrix has no tensor map (y_plain and so on; elements, strides in elements)
  void* y;
  const void* r;
  void* p;
  long long ys, rs, ps;
  const float *bias, *sm, *sn;  // sm, sn: scales of the rows of A and B, or null
  int M, N, kblocks, tiles_m, tiles_n, splits, split_rows, act;
  bool has_r, has_p, y_plain, r_plain, p_plain;
  unsigned int* err;
};

constexpr int GEMM_BM = 128;
constexpr uint32_t PANEL_BYTES = 128 * 128;
template <int GROUPS>
constexpr int GEMM_THREADS = 128 + 128 * GROUPS;
// the stages' bytes, a panel for each epilogue group behind them: with 3 or 5 KB static an SM's 227 KB at most
template <int GROUPS>
constexpr uint32_t RING_BYTES = (GROUPS == 2 ? 192 : 144) * 1024;
template <int GROUPS>
constexpr size_t GEMM_SMEM = RING_BYTES<GROUPS> + GROUPS * PANEL_BYTES;

template <int BN, bool PAIR, int GROUPS>
struct Ring {
  static constexpr uint32_t A = GEMM_BM * 128, B = (PAIR ? BN / 2 : BN) * 128, STAGE = A + B;
  static constexpr int STAGES = RING_BYTES<GROUPS> / STAGE;  // two groups: 4, 6, 8, a pair's 6; four: 3, 4
};

template <int BN, bool PAIR, int GROUPS>
struct GemmBars {
  uint64_t full[Ring<BN, PAIR, GROUPS>::STAGES], empty[Ring<BN, PAIR, GROUPS>::STAGES], dfull[2], dempty[2], rfull[GROUPS];
};

__device__ __forceinline__ void tmem_ld32(uint32_t ta, float* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
               "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
                 "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]),
                 "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]),
                 "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
               : "r"(ta) : "memory");
}

// Panels with m or n along their 128-byte rows: 64 elements of it a panel, `panel` bytes to the next 64, 1024 to the next 8 k.
__device__ __forceinline__ uint64_t mn_major_desc(uint32_t addr, uint32_t panel) {
  return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(panel >> 4) << 16) |
         (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
template <bool E4M3>
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (E4M3)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// The products so far have completed: an arrival at this barrier in both CTAs.
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(tc::smem_u32(bar)), "h"(static_cast<uint16_t>(3)) : "memory");
}
__device__ __forceinline__ void mma_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

// Two values at once (packed float32 arithmetic: half the instructions).
struct Pair {
  uint64_t v;
};
__device__ __forceinline__ Pair pair(float a, float b) {
  Pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(Pair p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.v)); }
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}

// s = 1 / (1 + e) for both of e = 2^t.  A reciprocal takes the special-function unit twice an exponential's time (measured: 16 and 32
// results a clock and SM), so one serves two values: 1 / (d0 d1) times the other.  t is cut at 60, so that the product stays finite
// and a NaN becomes a number that leaves the other value alone (the caller multiplies by its own z, which is NaN then too).
struct Logistic {
  Pair s, e;
};
__device__ __forceinline__ Logistic logistic2(Pair t) {
  float t0, t1, e0, e1, d0, d1, r;
  unpair(t, t0, t1);
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(fminf(t0, 60.f)));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(fminf(t1, 60.f)));
  const Pair e = pair(e0, e1);
  unpair(e + pair(1.f, 1.f), d0, d1);
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d0 * d1));
  return {pair(r, r) * pair(d1, d0), e};
}
// max(z, lo), NaN for NaN: below lo the products with logistic2 (at least 2^-60) stay next to nothing, infinities too
__device__ __forceinline__ float above(float z, float lo) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(z), "f"(lo));
  return r;
}
constexpr float LOG2E = 1.4426950408889634f, GATE_LOW = -64.f;
// the exponent of two in gelu's and silu's z / (1 + 2^t)
__device__ __forceinline__ Pair gate_exponent(Pair z, int act) {
  constexpr float A = -GELU_2A * LOG2E, B = A * GELU_B;
  if (act == ACT_GELU) return z * fma(z * z, pair(B, B), pair(A, A));
  return z * pair(-LOG2E, -LOG2E);
}
__device__ __forceinline__ void activate(float& z0, float& z1, int act) {
  if (act == ACT_RELU) {
    z0 = z0 < 0.f ? 0.f : z0, z1 = z1 < 0.f ? 0.f : z1;
  } else if (act != ACT_NONE) {
    const Pair z = pair(above(z0, GATE_LOW), above(z1, GATE_LOW));
    unpair(z * logistic2(gate_exponent(z, act)).s, z0, z1);
  }
}

// d0 *= act'(z0), d1 *= act'(z1).  gelu and silu: s (1 + z (1 - s) u'), s = 1 / (1 + e), e = 2^t.  1 - s is taken as e s: the shared
// reciprocal leaves s a unit or so off 1, which z u' (of the third degree in gelu) would make 1 % at z = 100.  z is held in
// [GATE_LOW, GATE_HIGH], beyond which the slope is 0 and 1 in float32 (e s is 0 from z = 9.8 on in gelu, from 87.4 on in silu; at
// GATE_LOW s, cut at 2^-60, leaves 5e-14 at most): left as it is, z u' would outgrow both, and 0 times an infinity be NaN.
constexpr float GATE_HIGH = 128.f;
__device__ __forceinline__ float between(float z, float lo, float hi) {  // NaN for NaN
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(above(z, lo)), "f"(hi));
  return r;
}
__device__ __forceinline__ void times_slope(float& d0, float& d1, float z0, float z1, int act) {
  if (act == ACT_RELU) {
    d0 = z0 > 0.f ? d0 : d0 * 0.f, d1 = z1 > 0.f ? d1 : d1 * 0.f;
    return;
  }
  const Pair z = pair(between(z0, GATE_LOW, GATE_HIGH), between(z1, GATE_LOW, GATE_HIGH));
  const Logistic l = logistic2(gate_exponent(z, act));
  Pair g = z * (l.e * l.s);
  if (act == ACT_GELU) g = g * fma(z * z, pair(3.f * GELU_2A * GELU_B, 3.f * GELU_2A * GELU_B), pair(GELU_2A, GELU_2A));
  unpair(pair(d0, d1) * (l.s * (g + pair(1.f, 1.f))), d0, d1);
}

template <typename O> struct Panel;  // a 128-byte row of the output
template <> struct Panel<__nv_bfloat16> {
  static constexpr int W = 64;
};
template <> struct Panel<float> {
  static constexpr int W = 32;
};

// byte of element c of row r of a swizzled panel
template <typename O>
__device__ __forceinline__ uint32_t panel_at(int r, int c) {
  constexpr int E = 16 / sizeof(O);
  return r * 128 + (((c / E) ^ (r & 7)) << 4) + (c % E) * static_cast<int>(sizeof(O));
}

// The group's 128 threads copy a panel between shared memory and rows m0 .. of an unaligned matrix, up to 16 elements a thread
// in flight.
template <typename O, bool STORE>
__device__ __forceinline__ void panel_plain(unsigned char* s, void* g, long long stride, int m0, int M, int col0, int N, int gt) {
  constexpr int C = Panel<O>::W / 32, ROWS = 16 / C;
  const int lane = gt & 31, warp = gt >> 5, rows = min(GEMM_BM, M - m0);
  O* base = static_cast<O*>(g) + static_cast<long long>(m0) * stride + col0 + lane;
  for (int r0 = warp; r0 < rows; r0 += 4 * ROWS) {
    O v[ROWS][C];
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int r = r0 + 4 * i;
        const bool in = r < rows && col0 + lane + 32 * c < N;
        if (STORE)
          v[i][c] = *reinterpret_cast<O*>(s + panel_at<O>(r & (GEMM_BM - 1), lane + 32 * c));
        else
          v[i][c] = in ? base[r * stride + 32 * c] : O(0.f);
      }
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int r = r0 + 4 * i;
        if (!STORE)
          *reinterpret_cast<O*>(s + panel_at<O>(r & (GEMM_BM - 1), lane + 32 * c)) = v[i][c];
        else if (r < rows && col0 + lane + 32 * c < N)
          base[r * stride + 32 * c] = v[i][c];
      }
  }
}

// 16-byte pieces q0 .. q0 + Q - 1 of a row of a panel
template <int Q>
__device__ __forceinline__ void panel_put(unsigned char* s, int row, int q0, const float* v, __nv_bfloat16) {
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    uint32_t h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      __nv_bfloat162 b = __floats2bfloat162_rn(v[8 * q + 2 * j], v[8 * q + 2 * j + 1]);
      h[j] = *reinterpret_cast<uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(s + row * 128 + (((q0 + q) ^ (row & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
  }
}
template <int Q>
__device__ __forceinline__ void panel_put(unsigned char* s, int row, int q0, const float* v, float) {
#pragma unroll
  for (int q = 0; q < Q; ++q)
    *reinterpret_cast<float4*>(s + row * 128 + (((q0 + q) ^ (row & 7)) << 4)) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
}
template <int Q>
__device__ __forceinline__ void panel_add(const unsigned char* s, int row, int q0, float* v, __nv_bfloat16) {
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const uint4 u = *reinterpret_cast<const uint4*>(s + row * 128 + (((q0 + q) ^ (row & 7)) << 4));
    const uint32_t a[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[8 * q + 2 * j] += __uint_as_float(a[j] << 16);
      v[8 * q + 2 * j + 1] += __uint_as_float(a[j] & 0xffff0000u);
    }
  }
}
template <int Q>
__device__ __forceinline__ void panel_add(const unsigned char* s, int row, int q0, float* v, float) {
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const float4 u = *reinterpret_cast<const float4*>(s + row * 128 + (((q0 + q) ^ (row & 7)) << 4));
    v[4 * q] += u.x, v[4 * q + 1] += u.y, v[4 * q + 2] += u.z, v[4 * q + 3] += u.w;
  }
}

// E4M3: A and B are e4m3 (else bf16); A_MN, B_MN: m / n along the rows of A / B (bf16 only); O: the output's type.
// GROUPS: epilogue groups.
template <bool E4M3, bool A_MN, bool B_MN, int BN, bool PAIR, int GROUPS, typename O>
__global__ void __launch_bounds__(GEMM_THREADS<GROUPS>, 1) k_gemm(const __grid_constant__ Gemm a) {
  static_assert(!E4M3 || (!A_MN && !B_MN), "8-bit operands lie with k along their rows");
  static_assert(!PAIR || BN == 256, "a pair's tile is 256 x 256");
  static_assert(GROUPS == 2 || (GROUPS == 4 && !PAIR), "two or four epilogue groups");
  using R = Ring<BN, PAIR, GROUPS>;
  constexpr int CTAS = PAIR ? 2 : 1, TILE_M = CTAS * GEMM_BM;
  constexpr int S = R::STAGES, BK = E4M3 ? 128 : 64, PW = Panel<O>::W, PANELS = BN / PW;
  constexpr uint32_t IDESC = (1u << 4) | (E4M3 ? 0u : (1u << 7) | (1u << 10)) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) |
                             (static_cast<uint32_t>(BN >> 3) << 17) | (static_cast<uint32_t>(TILE_M >> 4) << 24);
  extern __shared__ __align__(1024) unsigned char smem[];
  constexpr int TEAM = GROUPS / 2;  // groups on a tile
  constexpr int CH = GROUPS == 2 || PW < 32 ? PW : 32, Q = CH * static_cast<int>(sizeof(O)) / 16;  // columns in registers, their pieces
  __shared__ GemmBars<BN, PAIR, GROUPS> bars;
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(16) float s_bias[GROUPS][2][PW], s_scale[GROUPS][2][PW];  // of a group's panel and its next
  const uint32_t ring = tc::smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int items = a.tiles_m * a.tiles_n * a.splits;
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
    for (int s = 0; s < GROUPS; ++s) tc::mbar_init(&bars.rfull[s], 1);
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
  // item -> tile (n fastest) and split (slowest)
  auto place = [&](int item, int& m0, int& n0, int& split) {
    const int tile = item % (a.tiles_m * a.tiles_n);
    split = item / (a.tiles_m * a.tiles_n);
    m0 = tile / a.tiles_n * TILE_M + rank * GEMM_BM;  // this CTA's rows
    n0 = tile % a.tiles_n * BN;
  };
  auto first_block = [&](int split) { return static_cast<int>(static_cast<long long>(a.kblocks) * split / a.splits); };
  unsigned bad = 0;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      for (int item = unit; item < items && !bad; item += units) {
        int m0, n0, split;
        place(item, m0, n0, split);
        const int k1 = first_block(split + 1), b0 = PAIR ? n0 + rank * (BN / 2) : n0;
        for (int kb = first_block(split); kb < k1; ++kb, ++it) {
          const int s = it % S;
          if (!tma::wait(&bars.empty[s], ((it / S) & 1) ^ 1)) {
            bad |= 1;
            break;
          }
          const uint32_t sa = ring + s * R::STAGE, sb = sa + R::A;
          if (rank == 0) tma::expect_tx(&bars.full[s], CTAS * R::STAGE);
          const uint32_t full = PAIR ? tma::in_cta(tc::smem_u32(&bars.full[s]), 0) : 0;
          auto load = [&](uint32_t dst, const CUtensorMap* tm, int x, int y) {
            if constexpr (PAIR)
              tma::load_2d_pair(dst, tm, x, y, full);
            else
              tma::load_2d(dst, tm, x, y, &bars.full[s]);
          };
          if constexpr (A_MN) {
#pragma unroll
            for (int i = 0; i < GEMM_BM / 64; ++i) load(sa + i * 8192, &a.ta, m0 + 64 * i, kb * BK);
          } else {
            load(sa, &a.ta, kb * BK, m0);
          }
          if constexpr (B_MN) {
#pragma unroll
            for (int i = 0; i < BN / CTAS / 64; ++i) load(sb + i * 8192, &a.tb, b0 + 64 * i, kb * BK);
          } else {
            load(sb, &a.tb, kb * BK, b0);
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
        int m0, n0, split;
        place(item, m0, n0, split);
        const int d = i & 1, k0 = first_block(split), k1 = first_block(split + 1);
        if (!tma::wait(&bars.dempty[d], ((i >> 1) & 1) ^ 1)) {
          bad |= 2;
          break;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (int kb = k0; kb < k1; ++kb, ++it) {
          const int s = it % S;
          if (!tma::wait(&bars.full[s], (it / S) & 1)) {
            bad |= 4;
            break;
          }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t sa = ring + s * R::STAGE, sb = sa + R::A;
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {  // 32 bytes of k
            const uint64_t da = A_MN ? mn_major_desc(sa + ks * 2048, 8192) : tc::sw128_desc(sa + ks * 32);
            const uint64_t db = B_MN ? mn_major_desc(sb + ks * 2048, 8192) : tc::sw128_desc(sb + ks * 32);
            const uint32_t acc = kb > k0 || ks > 0;
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
    uint32_t i = 0, loads = 0;
    auto sync_group = [&] { asm volatile("bar.sync %0, 128;" ::"r"(1 + g) : "memory"); };
    auto wait = [&](uint64_t* b, uint32_t parity) {  // (after one wait has given up none is waited for)
      if (!bad && !tma::wait(b, parity)) bad |= 8;
    };
    // the group's tiles, and of the next one's columns gt, gt + 128 the bias and scale, of its row the scale: on their way while a
    // tile is stored
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
    constexpr int HELD = (BN + 127) / 128;
    float next_bias[HELD], next_scale[HELD], next_sm = 1.f;
    auto fetch = [&](int item) {
      if (item >= items) return;
      int m0, n0, split;
      place(item, m0, n0, split);
#pragma unroll
      for (int j = 0; j < HELD; ++j) {
        const int c = n0 + 128 * j + gt;
        next_bias[j] = a.bias && c < a.N ? __ldg(a.bias + c) : 0.f;
        next_scale[j] = a.sn && c < a.N ? __ldg(a.sn + c) : 1.f;
      }
      if (a.sm) next_sm = m0 + row < a.M ? __ldg(a.sm + m0 + row) : 1.f;
    };
    const int first = unit + (alternate ? g / TEAM * units : 0);
    if (alternate) i = g / TEAM;
    fetch(first);
    for (int item = first; item < items; item += stride, i += alternate ? 2 : 1) {
      int m0, n0, split;
      place(item, m0, n0, split);
      const int d = i & 1, yrow = split * a.split_rows + m0;
      const bool none = first_block(split) == first_block(split + 1);  // no K block: a sum of nothing
      const int panels = min(PANELS, (a.N - n0 + PW - 1) / PW);
      const float sm = next_sm;
      bool waited = false;
      int turn = 0;
      float bias[HELD], scale[HELD];
#pragma unroll
      for (int j = 0; j < HELD; ++j) bias[j] = next_bias[j], scale[j] = next_scale[j];
      fetch(item + stride);
      auto put_cols = [&](int p, int b) {  // of panel p, by the threads that hold its columns
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
          const int c = 128 * j + gt - p * PW;
          if (c >= 0 && c < PW) s_bias[g][b][c] = bias[j], s_scale[g][b][c] = scale[j];
        }
      };
      put_cols(p0, 0);
      sync_group();
      for (int p = p0; p < panels; p += step, turn ^= 1) {
        const int col0 = n0 + p * PW;
        put_cols(p + step, turn ^ 1);  // (the last panel's readers are behind its barrier)
        auto panel_free = [&] {  // the last store has read the panel
          if (gt == 0) tma::wait_read();
          sync_group();
        };
        auto load_r = [&] {
          if (a.r_plain) {
            panel_plain<O, false>(st, const_cast<void*>(a.r), a.rs, m0, a.M, col0, a.N, gt);
          } else if (gt == 0) {
            tma::expect_tx(&bars.rfull[g], PANEL_BYTES);
            tma::load_2d(st_u, &a.tr, col0, yrow, &bars.rfull[g]);
          }
        };
        if (a.has_r && !a.has_p) {
          panel_free();
          load_r();
        }
        if (!waited) {
          wait(&bars.dfull[d], (i >> 1) & 1);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          waited = true;
        }
        const float *sb = s_bias[g][turn], *ss = s_scale[g][turn];
        float v[CH];
        auto values = [&](int c0) {  // columns c0 .. of the panel before the activation
          __syncwarp();
#pragma unroll
          for (int c = 0; c < CH; c += 32) tmem_ld32(tmem + lanes + d * BN + p * PW + c0 + c, v + c);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          if (none) {
#pragma unroll
            for (int c = 0; c < CH; ++c) v[c] = 0.f;
          }
          if (a.sm) {
#pragma unroll
            for (int c = 0; c < CH; c += 4) {
              const float4 s = *reinterpret_cast<const float4*>(ss + c0 + c);
              unpair(pair(v[c], v[c + 1]) * (pair(sm, sm) * pair(s.x, s.y)), v[c], v[c + 1]);
              unpair(pair(v[c + 2], v[c + 3]) * (pair(sm, sm) * pair(s.z, s.w)), v[c + 2], v[c + 3]);
            }
          }
          if (a.bias) {
#pragma unroll
            for (int c = 0; c < CH; c += 4) {
              const float4 b = *reinterpret_cast<const float4*>(sb + c0 + c);
              unpair(pair(v[c], v[c + 1]) + pair(b.x, b.y), v[c], v[c + 1]);
              unpair(pair(v[c + 2], v[c + 3]) + pair(b.z, b.w), v[c + 2], v[c + 3]);
            }
          }
        };
        if constexpr (PW == 64) {
          if (a.has_p) {
            panel_free();
#pragma unroll
            for (int c0 = 0; c0 < PW; c0 += CH) {
              values(c0);
              panel_put<Q>(st, row, c0 / 8, v, O());
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            sync_group();
            if (a.p_plain) {
              panel_plain<__nv_bfloat16, true>(st, a.p, a.ps, m0, a.M, col0, a.N, gt);
            } else if (gt == 0 && (!PAIR || m0 < a.M)) {
              tma::store_2d(&a.tp, col0, m0, st_u);
              tma::commit();
              tma::wait_read();
            }
            sync_group();
            if (a.has_r) load_r();
          }
        }
#pragma unroll
        for (int c0 = 0; c0 < PW; c0 += CH) {
          if (CH < PW || !a.has_p) values(c0);  // (a whole panel's are still there)
          if (c0 + CH == PW && p + step >= panels) accumulator_read(d);
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
          if (a.has_r) {
            if (c0 == 0) {
              if (a.r_plain)
                sync_group();
              else
                wait(&bars.rfull[g], loads++ & 1);
            }
            panel_add<Q>(st, row, c0 * static_cast<int>(sizeof(O)) / 16, v, O());
          } else if (c0 == 0 && !a.has_p) {
            panel_free();
          }
          panel_put<Q>(st, row, c0 * static_cast<int>(sizeof(O)) / 16, v, O());
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        sync_group();
        if (a.y_plain) {
          panel_plain<O, true>(st, a.y, a.ys, m0, a.M, col0, a.N, gt);
        } else if (gt == 0 && (!PAIR || m0 < a.M)) {
          tma::store_2d(&a.ty, col0, yrow, st_u);
          tma::commit();
        }
      }
      if (!waited) {  // no panel of this tile for this group
        wait(&bars.dfull[d], (i >> 1) & 1);
        accumulator_read(d);
      }
    }
    if (gt == 0) tma::wait_done();
    if (bad && loads && !tma::wait(&bars.rfull[g], (loads - 1) & 1)) bad |= 16;  // a residual panel in flight
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

// Raises a kernel's shared-memory limit once a device; `raised` holds the devices (of the first 64) where that is done.
inline cudaError_t raise_smem(const void* kernel, size_t bytes, std::atomic<uint64_t>& raised) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (bit && (raised.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
  if (e == cudaSuccess) raised.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// One instance's launch: a persistent grid of at most one CTA per SM.
template <bool E4M3, bool A_MN, bool B_MN, int BN, bool PAIR, typename O, int GROUPS = 2>
cudaError_t launch_gemm(const Gemm& g, int sms, cudaStream_t stream) {
  auto k = k_gemm<E4M3, A_MN, B_MN, BN, PAIR, GROUPS, O>;
  static std::atomic<uint64_t> raised{0};
  const cudaError_t e = raise_smem(reinterpret_cast<const void*>(k), GEMM_SMEM<GROUPS>, raised);
  if (e != cudaSuccess) return e;
  constexpr int CTAS = PAIR ? 2 : 1;
  const long long items = static_cast<long long>(g.tiles_m) * g.tiles_n * g.splits, most = sms / CTAS;
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

// The products by tile width: 64, 128, 256, or TILE_PAIR, two CTAs on 256 x 256.
constexpr int TILE_PAIR = 512;
inline int tile_rows(int bn) { return bn == TILE_PAIR ? 2 * GEMM_BM : GEMM_BM; }
inline int tile_cols(int bn) { return bn == TILE_PAIR ? 256 : bn; }
inline int tile_b_rows(int bn) { return bn == TILE_PAIR ? 128 : bn; }  // of B that a CTA loads
template <bool E4M3, bool A_MN, bool B_MN, typename O>
cudaError_t gemm_by_width(const Gemm& g, int bn, int sms, cudaStream_t stream) {
  switch (bn) {
    case 64: return launch_gemm<E4M3, A_MN, B_MN, 64, false, O>(g, sms, stream);
    case 128: return launch_gemm<E4M3, A_MN, B_MN, 128, false, O>(g, sms, stream);
    case 256: return launch_gemm<E4M3, A_MN, B_MN, 256, false, O>(g, sms, stream);
    default: return launch_gemm<E4M3, A_MN, B_MN, 256, true, O>(g, sms, stream);
  }
}

// bn 128 or 256
template <bool E4M3, typename O>
cudaError_t gemm_four(const Gemm& g, int bn, int sms, cudaStream_t stream) {
  return bn == 128 ? launch_gemm<E4M3, false, false, 128, false, O, 4>(g, sms, stream) : launch_gemm<E4M3, false, false, 256, false, O, 4>(g, sms, stream);
}

// whtmix_gemm_fwd.cu, whtmix_gemm_e4m3.cu: y from x and W; whtmix_gemm_dx.cu (A with k, B with n along its rows); whtmix_gemm_dw.cu
// (both m / n)
cudaError_t gemm_forward(const Gemm& g, bool out_f32, int bn, int sms, cudaStream_t stream);
cudaError_t gemm_e4m3(const Gemm& g, bool out_f32, int bn, int sms, cudaStream_t stream);
// whtmix_gemm_four.cu, whtmix_gemm_e4m3_four.cu: the same with four epilogue groups
cudaError_t gemm_forward_four(const Gemm& g, bool out_f32, int bn, int sms, cudaStream_t stream);
cudaError_t gemm_e4m3_four(const Gemm& g, bool out_f32, int bn, int sms, cudaStream_t stream);
cudaError_t gemm_dx(const Gemm& g, int bn, int sms, cudaStream_t stream);
cudaError_t gemm_dw(const Gemm& g, bool out_f32, int bn, int sms, cudaStream_t stream);

// whtmix_gemm_dp.cu: dp = dy act'(p), its column sums and dx = dp W in one pass, for K <= 256 (one tile of columns) and an
// activation.  part [tiles_m, N]: the 128-token tiles' sums of unrounded dp, or null; tdp's map is written where store_dp.
struct DpProduct {
  CUtensorMap tdy, tp, tw, tdp, tdx;
  float* part;
  void* dx;
  long long dxs;
  int M, N, K, tiles_m, kblocks, act;
  bool store_dp, dx_plain;
  unsigned int* err;
};
cudaError_t gemm_dp(const DpProduct& g, int sms, cudaStream_t stream);

}  // namespace linear
}  // namespace whtmix
