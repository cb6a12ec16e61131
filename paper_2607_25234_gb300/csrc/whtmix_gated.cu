// whtmix_gated.cu -- host side of the gated feed-forward half (whtmix_gated.cuh) and the pass that makes dp = [dy u act'(g), dy act(g)] with
// the bias's gradient.  The backward's products are the linear layer's, without an activation: dp and W have 2 N columns and rows.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "whtmix_few.cuh"
#include "whtmix_gated.cuh"
#include "whtmix_gemm_gated.cuh"
#include "whtmix_linear_host.cuh"
#include "whtmix_norm.cuh"
#include "whtmix_unaligned.cuh"

namespace whtmix {
namespace linear {

constexpr int THREADS_256 = 256;

// CTAs of k_gated_dp an SM.  Two, three and four, whole backward, us: [65536, 512] to 1408 450, 391 and 422; [20000, 512] to 608 93, 81 and
// 88, to 601 135, 113 and 127; [8192, 1024] to 2736 203, 199 and 198, to 2733 261, 253 and 246; [27104, 184] to 5238 904, 851 and 810.
constexpr int DP_CTAS = 3;

// Rows on their way to a thread of k_gated_dp with many of them, in shared memory: a place for each of dy, g and u a lane, for unaligned
// rows one more a row.  With fewer than DP_RING rows a thread they come through registers, one at a time.  Registers and ring, dp alone, us:
// [8192, 2736] (24 rows a thread) 61.9 and 46.4, [5456, 2240] (13) 31.6 and 23.1, [2003, 3776] (8) 22.7 and 19.4, [20000, 200] (6) 10.6 and 11.9, [20000, 104] (3) 6.6 and 8.0;
// unaligned [27104, 5238] (154) 706 and 592, [8192, 2733] (24) 119.3 and 103.8, [3001, 777] (3) 15.0 and 17.6.  With 16 rows, whole backward,
// [20000, 512] to 608 83.5 and 81.2, unaligned to 601 111.8 and 113.4: the one rule for both costs the latter 1.5 %.
constexpr int DP_DEPTH = 4, DP_RING = 8;
template <bool AL, int TX>
constexpr int DP_PLACES = THREADS_256 / TX * (AL ? TX : TX + 1);
template <bool AL, int TX>
constexpr size_t DP_SMEM = size_t{DP_DEPTH} * 3 * DP_PLACES<AL, TX> * 16;

// dp goes to bf16: the products behind it take both operands in one type, and W and x are bf16 (dp in two bf16 parts would double them).
// dx and dw are off by 2.3e-3 of their norm for it, by 1.7e-3, their own rounding, with dp in 32 bits; db sums the 32 bits.
// dp[t, n], dp[t, N + n] = bf16 of both gradients; part[chunk][n], [N + n] = the chunk's rows' float32 sums of them, before the rounding.
// A CTA takes 8 TX channels (a thread 8) and the rows of chunk blockIdx.y, 256 / TX at a time.  dp, part: or null.  AL: dy, p and dp
// have 16-byte aligned rows and halves.  Unaligned rows come as the whole 16-byte granules around them: a lane takes its own, and the
// next lane's for the bytes it misses.
template <bool AL, int TX, bool RING>
__global__ void __launch_bounds__(THREADS_256, DP_CTAS) k_gated_dp(const Backward a, __nv_bfloat16* dp, long long dps, float* part, int chunks) {
  constexpr int G = THREADS_256 / TX, PITCH = AL ? TX : TX + 1;  // rows at a time, places a row
  extern __shared__ __align__(16) uint4 s_ring[];
  __shared__ float s[G][TX][9];
  const int lane = threadIdx.x % TX, g = threadIdx.x / TX, c0 = (blockIdx.x * TX + lane) * 8;
  const long long t0 = a.T * blockIdx.y / chunks, t1 = a.T * (blockIdx.y + 1) / chunks;
  float acc_g[8] = {}, acc_u[8] = {};
  pdl_wait();
  const uint16_t *dy = static_cast<const uint16_t*>(a.dy), *p = static_cast<const uint16_t*>(a.p);
  auto place = [&](int i, int m) { return s_ring + (i * 3 + m) * DP_PLACES<AL, TX> + g * PITCH + lane; };
  // a row's granules: of each the bytes from the matrix's first to the row's last, zeros beyond
  auto fetch = [&](long long t, int i) {
    const uint16_t *matrix[3] = {dy, p, p}, *row[3] = {dy + t * a.dys, p + t * a.ps, p + t * a.ps + a.N};
#pragma unroll
    for (int m = 0; m < 3; ++m) {
      const uint8_t *lo = reinterpret_cast<const uint8_t*>(matrix[m]), *end = reinterpret_cast<const uint8_t*>(row[m] + a.N);
      const uint8_t* q = reinterpret_cast<const uint8_t*>(row[m] + c0);
      q -= reinterpret_cast<uintptr_t>(q) & 15u;
#pragma unroll
      for (int extra = 0; extra < (AL ? 1 : 2); ++extra, q += 16) {
        if (extra && lane < TX - 1) continue;
        uint4* to = place(i, m) + extra;
        const int n = t >= t1 || q >= end ? 0 : end - q < 16 ? static_cast<int>(end - q) : 16;
        if (AL || n == 0 || q >= lo) {
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(to)), "l"(n ? q : lo - (reinterpret_cast<uintptr_t>(lo) & 15u)), "r"(n) : "memory");
        } else {  // the matrix starts inside it
#pragma unroll 1
          for (int j = 0; j < 8; ++j) reinterpret_cast<uint16_t*>(to)[j] = q + 2 * j >= lo && q + 2 * j < end ? *reinterpret_cast<const uint16_t*>(q + 2 * j) : 0;
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto unpack = [&](const uint32_t* w, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f[2 * j] = __uint_as_float(w[j] << 16), f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
  };
  auto values = [&](const uint4* from, const uint16_t* row, float (&f)[8]) {
    const uint4 u = *from;
    uint32_t w[8] = {u.x, u.y, u.z, u.w};
    if constexpr (!AL) {
      const uint32_t r = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row + c0)) & 15u;
      if (r) {
        const uint4 v = from[1];
        w[4] = v.x, w[5] = v.y, w[6] = v.z, w[7] = v.w;
        shift_bytes<4>(w, r);
      }
    }
    unpack(w, f);
  };
  // the same through registers
  const Span sd = span_of(a.dy, a.T, a.dys, a.N, 2), sp = span_of(a.p, a.T, a.ps, 2 * a.N, 2);
  using Raw = typename std::conditional<AL, uint4, Granules>::type;
  auto load = [&](const uint16_t* row, const Span& s, bool in) {
    Raw u = Raw{};
    if (in && c0 < a.N) {
      if constexpr (AL)
        u = *reinterpret_cast<const uint4*>(row + c0);
      else
        u = fetch16(reinterpret_cast<const uint8_t*>(row + c0), s);
    }
    return u;
  };
  auto loaded = [&](const Raw& raw, const uint16_t* row, const Span& s, bool in, float (&f)[8]) {
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (AL)
      u = raw;
    else if (in && c0 < a.N)
      u = keep(finish16(raw, reinterpret_cast<const uint8_t*>(row + c0), s), min(16, 2 * (a.N - c0)));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    unpack(w, f);
  };
  // Eight values at column c0 of a half that starts s elements behind a 16-byte boundary (dp's rows start on one): whole vectors lie s
  // elements lower, their first s values are the lane before's.  What no vector holds, at the ends of a strip and of the half, goes
  // element by element.  ([3001, 777] with every element on its own: 31 us)
  const uint32_t segment = TX == 32 ? 0xffffffffu : ((1u << TX) - 1u) << (threadIdx.x & 31u & ~static_cast<uint32_t>(TX - 1));
  auto store = [&](__nv_bfloat16* o, int s, const float (&f)[8]) {
    const int left = a.N - c0;
    uint32_t h[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
      h[4 + j] = *reinterpret_cast<uint32_t*>(&b);
    }
    bool whole = left >= 8, next = true;  // this lane's vector, and the next one's
    if constexpr (!AL) {
      if (s > 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) h[j] = __shfl_up_sync(segment, h[4 + j], 1, TX);
        shift_bytes<4>(h, static_cast<uint32_t>(16 - 2 * s));
#pragma unroll
        for (int j = 0; j < 4; ++j) h[4 + j] = h[j];
        whole = lane > 0 && left >= 8 - s, next = lane < TX - 1 && left - 8 >= 8 - s;
      }
    }
    if (whole) *reinterpret_cast<uint4*>(o + c0 - s) = make_uint4(h[4], h[5], h[6], h[7]);
    if constexpr (!AL) {
      if (!whole || !next) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < left && (j < 8 - s ? !whole : !next)) o[c0 + j] = __float2bfloat16_rn(f[j]);
      }
    }
  };
  if constexpr (RING) {
#pragma unroll
    for (int i = 0; i < DP_DEPTH - 1; ++i) fetch(t0 + i * G + g, i);
  }
  int turn = 0;
  for (long long base = t0; base < t1; base += G, turn = (turn + 1) % DP_DEPTH) {
    const long long t = base + g;
    const uint16_t *rd = dy + t * a.dys, *rz = p + t * a.ps, *ru = rz + a.N;
    float d[8], z[8], u[8], v[8];
    if constexpr (RING) {
      asm volatile("cp.async.wait_group %0;" ::"n"(DP_DEPTH - 2) : "memory");
      if constexpr (!AL) __syncwarp();  // the other lanes' granules are there, and those of the last row have been read
      fetch(t + (DP_DEPTH - 1) * G, (turn + DP_DEPTH - 1) % DP_DEPTH);
      values(place(turn, 0), rd, d);
      values(place(turn, 1), rz, z);
      values(place(turn, 2), ru, u);
    } else {
      const bool in = t < t1;
      const Raw xd = load(rd, sd, in), xz = load(rz, sp, in), xu = load(ru, sp, in);
      loaded(xd, rd, sd, in, d);
      loaded(xz, rz, sp, in, z);
      loaded(xu, ru, sp, in, u);
    }
#pragma unroll
    for (int j = 0; j < 8; j += 2) gate_gradients(d[j], d[j + 1], v[j], v[j + 1], z[j], z[j + 1], u[j], u[j + 1], a.act);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc_g[j] += d[j], acc_u[j] += v[j];
    if (dp && t < t1) {
      store(dp + t * dps, 0, d);
      store(dp + t * dps + a.N, a.N % 8, v);
    }
  }
  if constexpr (RING) asm volatile("cp.async.wait_all;" ::: "memory");
  if (part) {
    auto add = [&](const float (&acc)[8], float* to) {
      __syncthreads();  // the last sums have been read
#pragma unroll
      for (int j = 0; j < 8; ++j) s[g][lane][j] = acc[j];
      __syncthreads();
      if (threadIdx.x < 8 * TX) {
        float sum = 0.f;
#pragma unroll 8
        for (int i = 0; i < G; ++i) sum += s[i][threadIdx.x >> 3][threadIdx.x & 7];
        const int c = blockIdx.x * 8 * TX + threadIdx.x;
        if (c < a.N) to[c] = sum;
      }
    };
    float* row = part + static_cast<long long>(blockIdx.y) * 2 * a.N;
    add(acc_g, row);
    add(acc_u, row + a.N);
  }
  pdl_trigger();
}

// ---- host ----

struct GatedForwardPlan {
  bool pad_x, pad_w;
  int kp;
  size_t x_off, w_off, total;
};
static GatedForwardPlan plan_forward(const Forward& a) {
  GatedForwardPlan f{};
  const int es = a.e4m3 ? 1 : 2;
  f.kp = pitch_of(a.K, es);
  f.pad_x = !tma::mappable(a.x, a.T, a.xs, es);
  f.pad_w = !tma::mappable(a.w, 2ll * a.N, a.ws, es);
  if (f.pad_x) f.x_off = f.total, f.total += align256(static_cast<size_t>(a.T) * f.kp * es);
  if (f.pad_w) f.w_off = f.total, f.total += align256(static_cast<size_t>(2ll * a.N) * f.kp * es);
  return f;
}

// Calls for whtmix_few.cu: few tokens; a long K axis and tiles of 64 channels that four CTAs each can share; or few tiles for a long K
// axis, which the tiled products would walk along on their own.  The tiled products and those, us, bf16, K and N: 32 tokens 1024, 8192
// 9.5 and 9.9; 64 tokens 1024, 2736 8.4 and 9.3, 4096, 4096 23.7 and 18.6, 4096, 8192 26.5 and 30.2; 100 tokens 2048, 5464 14.6 and 22.6;
// 171 tokens 7448, 1176 44.7 and 27.5; 500 tokens 2048, 144 13.3 and 9.2, 7448, 1176 45.0 and 55.4; 3200 tokens 4096, 64 23.2 and 15.2,
// 2048, 144 13.8 and 28.9.  Beyond three tiles for four SMs the tiled products fill the SMs on their own: 512 tokens 32768, 1600 157.0 and 117.1;
// 1024 tokens 16384, 1024 81.7 and 100.6; 128 tokens 16384, 8192 98.8 and 113.7.
static bool few_tokens(long long T, int N, int kblocks, int sms) {
  const long long tiles = static_cast<long long>(ceil_div(N, 64)) * ceil_div(T, 128);
  return T <= 32 || (T <= 64 && kblocks >= 32 && 4 * tiles <= 2ll * sms) || (5 * tiles <= 3ll * kblocks && 4 * tiles <= 3ll * sms);
}

// Four epilogue groups instead of two, at the price of a shorter ring, where the epilogue is longer than a tile's products.  Two and
// four, us: [64800, 128] to 344, gelu 26.0 and 22.6, with p 40.5 and 33.9; [64800, 256] to 688 with p 74.7 and 66.2; [64800, 384] to
// 1024 77.8 and 81.8, with p 117 and 108; [32768, 512] to 1408 64.3 and 72.3, with p 95.8 and 89.3; [32768, 768] to 2048 with p 155
// and 162.
static bool four_groups(const Gated& g, int sms) {
  return g.kblocks <= (g.has_p ? 8 : 4) && static_cast<long long>(g.tiles_m) * g.tiles_n > sms;
}

size_t gated_forward_workspace(const Forward& a, int) { return plan_forward(a).total; }

cudaError_t gated_forward(const Forward& a, void* ws, unsigned int* err, int sms, cudaStream_t stream) {
  const GatedForwardPlan f = plan_forward(a);
  const int es = a.e4m3 ? 1 : 2, os = a.out_f32 ? 4 : 2;
  const void *x = a.x, *w = a.w;
  long long xs = a.xs, wst = a.ws;
  Copy cx{}, cw{};
  if (f.pad_x) {
    x = static_cast<char*>(ws) + f.x_off, xs = f.kp;
    cx = copy_of(static_cast<char*>(ws) + f.x_off, a.x, a.T, a.K, a.xs, f.kp, es);
  }
  if (f.pad_w) {
    w = static_cast<char*>(ws) + f.w_off, wst = f.kp;
    cw = copy_of(static_cast<char*>(ws) + f.w_off, a.w, 2ll * a.N, a.K, a.ws, f.kp, es);
  }
  const cudaError_t e = to_pitch(cx, cw, sms, stream);
  if (e != cudaSuccess) return e;
  if (few_tokens(a.T, a.N, ceil_div(a.K, 128 / es), sms)) return forward_few(a, x, xs, w, wst, true, err, sms, stream);
  Gated g{};
  g.kblocks = ceil_div(a.K, 128 / es);
  // a product of 2 N columns by its clocks, 128 of them a tile at least
  Plan pl = plan_product(a.T, 2 * a.N, g.kblocks, sms, 1);
  if (pl.bn < 128) pl.bn = 128;
  // Rows that are no whole 128-byte lines cost twice the way out of L2, of which a pair needs less: [15944, 408] to 5456 171 and 138 us
  // (with p 207 and 195), where [64800, 384] to 1024 takes 78 and 84; [6192, 216] to 6272 with p, 4 K blocks, 73 and 81.
  const bool lines = static_cast<unsigned long long>(xs) * es % 128 == 0 && static_cast<unsigned long long>(wst) * es % 128 == 0;
  if (pl.bn == 256 && !lines && g.kblocks > 4 && static_cast<long long>(ceil_div(a.T, 256)) * ceil_div(a.N, 128) >= sms) pl.bn = TILE_PAIR;
  const int out = tile_cols(pl.bn) / 2;
  g.tiles_m = ceil_div(a.T, tile_rows(pl.bn)), g.tiles_n = ceil_div(a.N, out);
  g.band = 16;
  g.M = static_cast<int>(a.T), g.N = a.N, g.act = a.act;
  g.bias = a.bias, g.sm = a.x_scale, g.sn = a.w_scale;
  g.y = a.y, g.p = a.p, g.ys = a.ys, g.ps = a.ps;
  g.has_p = a.p != nullptr;
  g.y_plain = !tma::storable(a.y, a.T, a.N, a.ys, os);
  // (its halves apart: a store of the gate's last columns must not reach the value's first ones)
  __nv_bfloat16* value = static_cast<__nv_bfloat16*>(a.p) + (a.p ? a.N : 0);
  g.p_plain = a.p && !(tma::storable(a.p, a.T, a.N, a.ps, 2) && tma::storable(value, a.T, a.N, a.ps, 2));
  g.err = err;
  if (!tma::encode_rows(&g.ta, x, es, a.T, a.K, xs, GEMM_BM) || !tma::encode_rows(&g.tb, w, es, 2ll * a.N, a.K, wst, out) ||
      (!g.y_plain && !tma::encode_rows(&g.ty, a.y, os, a.T, a.N, a.ys, GEMM_BM)) ||
      (g.has_p && !g.p_plain && (!tma::encode_rows(&g.tg, a.p, 2, a.T, a.N, a.ps, GEMM_BM) || !tma::encode_rows(&g.tu, value, 2, a.T, a.N, a.ps, GEMM_BM))))
    return cudaErrorInvalidValue;
  const bool four = four_groups(g, sms);
  return a.e4m3 ? gemm_gated_e4m3(g, a.out_f32, pl.bn, four, sms, stream) : gemm_gated(g, a.out_f32, pl.bn, four, sms, stream);
}

// Threads a row of k_gated_dp, eight channels each: 32 unless they would be idle in a third of the last strip's places, and eight where one
// CTA a strip takes all rows.  32 and 8, dp alone, us: [128224, 150] 104.2 and 81.4, [60000, 176] 25.3 and 22.3, [3001, 301] 9.3 and
// 8.1, but [20000, 601] 58.1 and 75.9, [3001, 777] 15.1 and 18.2; [128, 1408] in one chunk 12.0 and 4.7, [64, 149] 14.6 and 6.2.
static int dp_lanes(long long T, int N) {
  if (N <= 64 || T <= 128) return 8;
  if (N <= 128) return 16;
  return 3 * ceil_div(N, 256) * 256 >= 4 * ceil_div(N, 64) * 64 ? 8 : 32;
}

// dp and db's partial sums (fused: and dx), then the linear layer's products of them with W and x.
struct GatedBackwardPlan {
  bool fused;         // whtmix_gemm_gated_dp.cu
  Backward products;  // (its dy and workspace are filled in when the call runs)
  int np, chunks;     // pitch of dp; db's chunks of rows
  bool pad_w, pad_x;  // fused: W, x to a 16-byte pitch, in one launch
  size_t dp_off, db_off, w_off, x_off, products_off, total;
};
static GatedBackwardPlan plan_backward(const Backward& a, int sms) {
  GatedBackwardPlan b{};
  b.np = pitch_of(2 * a.N, 2);
  auto take = [&](size_t bytes) {
    const size_t off = b.total;
    b.total += align256(bytes);
    return off;
  };
  // one pass over dy and p instead of a kernel for dp and a product that reads it again; tiles of 128 tokens on half the SMs at least,
  // dy's rows and both halves' on 16-byte boundaries
  b.fused = a.dx && a.K <= 256 && a.N % 8 == 0 && tma::mappable(a.dy, a.T, a.dys, 2) && tma::mappable(a.p, a.T, a.ps, 2) &&
            2ll * ceil_div(a.T, GEMM_BM) >= sms;
  b.products = a;
  b.products.N = 2 * a.N, b.products.act = ACT_NONE, b.products.p = nullptr, b.products.db = nullptr;
  b.products.dy = nullptr, b.products.dys = b.np;  // (on a 16-byte boundary)
  b.products.split_dx = true;
  if (b.fused) {
    b.products.dx = nullptr;
    b.pad_x = a.dw && !tma::mappable(a.x, a.T, a.xs, 2);
    if (b.pad_x) b.x_off = take(static_cast<size_t>(a.T) * pitch_of(a.K, 2) * 2), b.products.x = nullptr, b.products.xs = pitch_of(a.K, 2);
  }
  if (b.products.dx || a.dw) {
    b.dp_off = take(static_cast<size_t>(a.T) * b.np * 2);
    b.products_off = take(backward_workspace(b.products, sms));
  }
  if (b.fused) {
    b.chunks = ceil_div(a.T, GEMM_BM);
    b.pad_w = !tma::mappable(a.w, 2ll * a.N, a.ws, 2);
    if (b.pad_w) b.w_off = take(static_cast<size_t>(2ll * a.N) * pitch_of(a.K, 2) * 2);
  } else {
    const int tx = dp_lanes(a.T, a.N), strips = ceil_div(a.N, 8 * tx), rows = ceil_div(a.T, 512 / tx), most = (DP_CTAS * sms + strips - 1) / strips;  // one wave
    b.chunks = rows < most ? rows : most;
    if (b.chunks > 65535) b.chunks = 65535;
    if (a.T <= 128) b.chunks = 1;  // db comes whole from one CTA a strip: a launch less
  }
  if (a.db && b.chunks > 1) b.db_off = take(static_cast<size_t>(b.chunks) * 2 * a.N * 4);
  return b;
}

size_t gated_backward_workspace(const Backward& a, int sms) { return plan_backward(a, sms).total; }

// dp, dx and db's partial sums
static cudaError_t fused_backward(const Backward& a, const GatedBackwardPlan& b, char* base, float* part, unsigned int* err, int sms,
                                  cudaStream_t stream) {
  const __nv_bfloat16* w = static_cast<const __nv_bfloat16*>(a.w);
  long long wst = a.ws;
  const int kp = pitch_of(a.K, 2);
  const Copy cx = b.pad_x ? copy_of(base + b.x_off, a.x, a.T, a.K, a.xs, kp, 2) : Copy{};
  const Copy cw = b.pad_w ? copy_of(base + b.w_off, a.w, 2ll * a.N, a.K, a.ws, kp, 2) : Copy{};
  const cudaError_t e = to_pitch(cx, cw, sms, stream);
  if (e != cudaSuccess) return e;
  if (b.pad_w) w = reinterpret_cast<const __nv_bfloat16*>(base + b.w_off), wst = kp;
  const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(a.p);
  __nv_bfloat16* dp = a.dw ? reinterpret_cast<__nv_bfloat16*>(base + b.dp_off) : nullptr;
  GatedDp g{};
  g.M = static_cast<int>(a.T), g.N = a.N, g.K = a.K, g.tiles_m = ceil_div(a.T, GEMM_BM), g.kblocks = ceil_div(a.N, 64), g.act = a.act;
  g.part = part;
  g.store_dp = dp != nullptr;
  g.dx = a.dx, g.dxs = a.dxs, g.dx_plain = !tma::storable(a.dx, a.T, a.K, a.dxs, 2);
  g.err = err;
  if (!tma::encode_rows(&g.tdy, a.dy, 2, a.T, a.N, a.dys, GEMM_BM) || !tma::encode_rows(&g.tg, p, 2, a.T, a.N, a.ps, GEMM_BM) ||
      !tma::encode_rows(&g.tu, p + a.N, 2, a.T, a.N, a.ps, GEMM_BM) || !tma::encode_rows(&g.twg, w, 2, a.N, a.K, wst, 64) ||
      !tma::encode_rows(&g.twu, w + static_cast<size_t>(a.N) * wst, 2, a.N, a.K, wst, 64) ||
      (dp && (!tma::encode_rows(&g.tdg, dp, 2, a.T, a.N, b.np, GEMM_BM) || !tma::encode_rows(&g.tdu, dp + a.N, 2, a.T, a.N, b.np, GEMM_BM))) ||
      (!g.dx_plain && !tma::encode_rows(&g.tdx, a.dx, 2, a.T, a.K, a.dxs, GEMM_BM)))
    return cudaErrorInvalidValue;
  return gemm_gated_dp(g, sms, stream);
}

cudaError_t gated_backward(const Backward& a, void* ws, unsigned int* err, int sms, cudaStream_t stream) {
  const GatedBackwardPlan b = plan_backward(a, sms);
  char* base = static_cast<char*>(ws);
  Backward c = a;
  __nv_bfloat16* dp = b.products.dx || a.dw ? reinterpret_cast<__nv_bfloat16*>(base + b.dp_off) : nullptr;
  float* part = !a.db ? nullptr : b.chunks > 1 ? reinterpret_cast<float*>(base + b.db_off) : a.db;
  int chunks = b.chunks;
  cudaError_t e;
  if (b.fused) {
    e = fused_backward(a, b, base, part, err, sms, stream);
  } else {
    long long np = b.np;
    const bool al = a.N % 8 == 0 && tma::mappable(a.dy, a.T, a.dys, 2) && tma::mappable(a.p, a.T, a.ps, 2);
    cudaLaunchConfig_t cfg = {};
    const int tx = dp_lanes(a.T, a.N);
    cfg.gridDim = dim3(ceil_div(a.N, 8 * tx), chunks);
    cfg.blockDim = dim3(THREADS_256);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const bool ring = a.T * tx >= static_cast<long long>(DP_RING) * THREADS_256 * chunks;
    auto launch = [&](auto aligned, auto lanes) {
      constexpr bool AL = decltype(aligned)::value;
      constexpr int TX = decltype(lanes)::value;
      if (!ring) return cudaLaunchKernelEx(&cfg, k_gated_dp<AL, TX, false>, c, dp, np, part, chunks);
      static std::atomic<uint64_t> raised{0};
      const cudaError_t r = raise_smem(reinterpret_cast<const void*>(k_gated_dp<AL, TX, true>), DP_SMEM<AL, TX>, raised);
      cfg.dynamicSmemBytes = DP_SMEM<AL, TX>;
      return r != cudaSuccess ? r : cudaLaunchKernelEx(&cfg, k_gated_dp<AL, TX, true>, c, dp, np, part, chunks);
    };
    auto by_lanes = [&](auto aligned) {
      return tx == 8    ? launch(aligned, std::integral_constant<int, 8>())
             : tx == 16 ? launch(aligned, std::integral_constant<int, 16>())
                        : launch(aligned, std::integral_constant<int, 32>());
    };
    e = al ? by_lanes(std::true_type()) : by_lanes(std::false_type());
  }
  if (e != cudaSuccess) return e;
  if (a.db && chunks > 1 && (e = norm::add_rows(part, a.db, 2 * a.N, chunks, stream)) != cudaSuccess) return e;
  if (!dp) return cudaSuccess;
  Backward products = b.products;
  products.dy = dp;
  if (b.pad_x) products.x = base + b.x_off;
  return backward(products, base + b.products_off, err, sms, stream);
}

}  // namespace linear
}  // namespace whtmix
