// whtmix_linear.cu -- host side of the linear layer (y = act(x W^T + b) + r and its backward) and the passes around its products:
// rows copied to a 16-byte pitch where the tensor maps need one, dp = dy act'(p) with the bias's gradient, the sum of a split
// weight gradient's partial products.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "whtmix_few.cuh"
#include "whtmix_gemm.cuh"
#include "whtmix_linear.cuh"
#include "whtmix_linear_host.cuh"
#include "whtmix_norm.cuh"
#include "whtmix_unaligned.cuh"

namespace whtmix {
namespace linear {

constexpr int THREADS_256 = 256;

// ---- rows to a 16-byte pitch ----
// dst [rows, pitch] = src [rows, cols] (stride elements a row), zeros beyond cols; a thread writes 16 bytes.  pitch is a multiple of
// 16 bytes.  Up to two matrices a launch.
template <typename I>  // 32-bit places where they suffice
__global__ void __launch_bounds__(THREADS_256) k_pitch(const Copy a, const Copy b, long long na, long long n) {
  constexpr int U = 4;
  pdl_wait();
  const I step = static_cast<I>(gridDim.x) * THREADS_256;
  for (I i0 = static_cast<I>(blockIdx.x) * THREADS_256 + threadIdx.x; i0 < static_cast<I>(n); i0 += U * step) {
    Granules g[U];
    const uint8_t* p[U];
    uint8_t* q[U];
    int left[U];
    Span span[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const I i = i0 + u * step;
      left[u] = -1;
      if (i < static_cast<I>(n)) {
        const bool first = i < static_cast<I>(na);
        const Copy& m = first ? a : b;
        const I j = first ? i : i - static_cast<I>(na), per_row = static_cast<I>(m.pitch >> 4), r = j / per_row;
        const long long c = static_cast<long long>(j - r * per_row) * 16;
        p[u] = m.src + static_cast<long long>(r) * m.stride + c;
        q[u] = m.dst + static_cast<long long>(r) * m.pitch + c;
        left[u] = static_cast<int>(m.cols - c < 16 ? m.cols - c : 16);
        span[u] = Span{m.src, m.src + (m.rows - 1) * m.stride + m.cols};
        g[u] = fetch16(p[u], span[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (left[u] >= 0) *reinterpret_cast<uint4*>(q[u]) = keep(finish16(g[u], p[u], span[u]), left[u]);
  }
  pdl_trigger();
}

cudaError_t to_pitch(const Copy& a, const Copy& b, int sms, cudaStream_t stream) {
  long long na = a.dst ? a.chunks() : 0, n = na + (b.dst ? b.chunks() : 0);
  if (n == 0) return cudaSuccess;
  const long long need = (n + 4 * THREADS_256 - 1) / (4 * THREADS_256), most = 4ll * sms;
  Copy ca = a, cb = b;
  void* args[] = {&ca, &cb, &na, &n};
  return launch_pdl(n < (1ll << 30) ? reinterpret_cast<const void*>(k_pitch<uint32_t>) : reinterpret_cast<const void*>(k_pitch<unsigned long long>), static_cast<unsigned>(need < most ? need : most), THREADS_256, 0, stream, args);
}

// ---- dp and db ----
// dp[t, n] = bf16(dy act'(p)); part[chunk][n] = the chunk's rows' float32 sum of dy act'(p), before the rounding.  A CTA takes
// 8 TX columns (a thread 8) and the rows of chunk blockIdx.y, 256 / TX at a time.  dp, part: or null.
template <bool AL, int TX>
__global__ void __launch_bounds__(THREADS_256, AL ? 4 : 3) k_dp(const Backward a, __nv_bfloat16* dp, long long dps, float* part, int chunks) {
  constexpr int G = THREADS_256 / TX;  // rows at a time
  __shared__ float s[G][TX][9];
  const int lane = threadIdx.x % TX, g = threadIdx.x / TX, c0 = (blockIdx.x * TX + lane) * 8;
  const long long t0 = a.T * blockIdx.y / chunks, t1 = a.T * (blockIdx.y + 1) / chunks;
  float acc[8] = {};
  pdl_wait();
  const uint16_t *dy = static_cast<const uint16_t*>(a.dy), *p = static_cast<const uint16_t*>(a.p);
  const Span sd = span_of(a.dy, a.T, a.dys, a.N, 2), sp = span_of(a.p, a.T, a.ps, a.N, 2);
  using Raw = typename std::conditional<AL, uint4, Granules>::type;
  auto fetch = [&](const uint16_t* row, const Span& s) {
    Raw u = Raw{};
    if (c0 < a.N) {
      if constexpr (AL)
        u = *reinterpret_cast<const uint4*>(row + c0);
      else
        u = fetch16(reinterpret_cast<const uint8_t*>(row + c0), s);
    }
    return u;
  };
  auto values = [&](const Raw& raw, const uint16_t* row, const Span& s, float (&f)[8]) {
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (AL)
      u = raw;
    else if (c0 < a.N)
      u = keep(finish16(raw, reinterpret_cast<const uint8_t*>(row + c0), s), min(16, 2 * (a.N - c0)));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) f[2 * j] = __uint_as_float(w[j] << 16), f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
  };
  constexpr int U = 2;  // rows in flight
  for (long long first = t0 + g; first < t1; first += G * U) {
    Raw ud[U], uz[U];
#pragma unroll
    for (int r = 0; r < U; ++r) {
      const long long t = first + G * r;
      if (t < t1) {
        ud[r] = fetch(dy + t * a.dys, sd);
        if (a.act != ACT_NONE) uz[r] = fetch(p + t * a.ps, sp);
      }
    }
#pragma unroll
    for (int r = 0; r < U; ++r) {
      const long long t = first + G * r;
      if (t >= t1) break;
      float d[8];
      values(ud[r], dy + t * a.dys, sd, d);
      if (a.act != ACT_NONE) {
        float z[8];
        values(uz[r], p + t * a.ps, sp, z);
#pragma unroll
        for (int j = 0; j < 8; j += 2) times_slope(d[j], d[j + 1], z[j], z[j + 1], a.act);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += d[j];
      if (dp) {  // (its pitch holds whole vectors)
        uint32_t h[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          __nv_bfloat162 b = __floats2bfloat162_rn(d[2 * j], d[2 * j + 1]);
          h[j] = *reinterpret_cast<uint32_t*>(&b);
        }
        if (c0 < a.N) *reinterpret_cast<uint4*>(dp + t * dps + c0) = make_uint4(h[0], h[1], h[2], h[3]);
      }
    }
  }
  if (part) {
#pragma unroll
    for (int j = 0; j < 8; ++j) s[g][lane][j] = acc[j];
    __syncthreads();
    if (threadIdx.x < 8 * TX) {
      float sum = 0.f;
#pragma unroll 8
      for (int i = 0; i < G; ++i) sum += s[i][threadIdx.x >> 3][threadIdx.x & 7];
      const int c = blockIdx.x * 8 * TX + threadIdx.x;
      if (c < a.N) part[static_cast<long long>(blockIdx.y) * a.N + c] = sum;
    }
  }
  pdl_trigger();
}

// ---- the sum of a split product ----
// out [rows, cols] (out_stride elements a row) = sum over s of part[s * split_rows + row][pitch].  A CTA takes 256 / G fours of columns; its G groups
// of threads sum runs of consecutive splits, each in ascending order, then the run sums are added in ascending order.  Many splits
// take G = 8: with a thread for all the splits of its four, 152 splits of [77, 488] took 12.5 us.
template <typename O, int G>
__global__ void __launch_bounds__(THREADS_256) k_sum_splits(O* __restrict__ out, const float* part, int rows, int cols, int pitch,
                                                            int split_rows, int splits, long long out_stride) {
  constexpr int L = THREADS_256 / G;
  __shared__ float4 s[G][L];
  pdl_wait();
  const int lane = threadIdx.x % L, g = threadIdx.x / L, quads = (cols + 3) / 4;
  const int s0 = splits * g / G, s1 = splits * (g + 1) / G;
  const long long n = static_cast<long long>(rows) * quads;
  for (long long base = static_cast<long long>(blockIdx.x) * L; base < n; base += static_cast<long long>(gridDim.x) * L) {
    const long long i = base + lane;
    const int r = static_cast<int>(i / quads), c = static_cast<int>(i - static_cast<long long>(r) * quads) * 4;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < n) {
      const float4* p = reinterpret_cast<const float4*>(part + (static_cast<long long>(s0) * split_rows + r) * pitch + c);
      const long long step = static_cast<long long>(split_rows) * pitch / 4;
      int k = s0;
      for (; k + 8 <= s1; k += 8, p += 8 * step) {
        float4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = __ldcg(p + u * step);
#pragma unroll
        for (int u = 0; u < 8; ++u) sum.x += v[u].x, sum.y += v[u].y, sum.z += v[u].z, sum.w += v[u].w;
      }
#pragma unroll 4
      for (; k < s1; ++k, p += step) {
        const float4 v = __ldcg(p);
        sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
      }
    }
    if constexpr (G > 1) {
      __syncthreads();  // the last round's sums have been read
      s[g][lane] = sum;
      __syncthreads();
    }
    if (g == 0 && i < n) {
#pragma unroll
      for (int k = 1; k < G; ++k) {
        const float4 v = s[k][lane];
        sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
      }
      const float f[4] = {sum.x, sum.y, sum.z, sum.w};
      O* o = out + static_cast<long long>(r) * out_stride + c;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < cols) o[j] = static_cast<O>(f[j]);
    }
  }
  pdl_trigger();
}

// ---- host ----

static cudaError_t sum_splits(void* out, bool f32, long long out_stride, const float* part, int rows, int cols, int pitch, int split_rows,
                              int splits, int sms, cudaStream_t stream) {
  void* args[] = {&out, &part, &rows, &cols, &pitch, &split_rows, &splits, &out_stride};
  const bool many = splits >= 16;
  const long long n = static_cast<long long>(rows) * ceil_div(cols, 4), need = (n + (many ? 31 : 255)) / (many ? 32 : 256);
  return launch_pdl(f32 ? (many ? reinterpret_cast<const void*>(k_sum_splits<float, 8>) : reinterpret_cast<const void*>(k_sum_splits<float, 1>))
                        : (many ? reinterpret_cast<const void*>(k_sum_splits<__nv_bfloat16, 8>)
                                : reinterpret_cast<const void*>(k_sum_splits<__nv_bfloat16, 1>)),
                    static_cast<unsigned>(need < 8ll * sms ? need : 8ll * sms), THREADS_256, 0, stream, args);
}

// Tile width and splits of a product of M rows, N columns and kblocks K blocks.  A block of a tile costs BLOCK clocks of an SM (of a
// pair of them), not in proportion to its width: the operands' way from L2 and out of shared memory bounds the narrow tiles
// (measured at [8192, 4096] x [4096, 4096]: 545 clocks at 256 columns, 450 at 128; a pair's 256 x 256 takes 470).  A tile costs about
// TILE_CLOCKS besides, more where two CTAs wait for each other, a split product's partial tiles their way through memory.  Pairs
// against single tiles, us: that product 157.7 and 168.5; [8192, 1024] x [1024, 1024] 18.7 and 17.2; 64800 tokens of 128 channels to
// 512 32.2 and 28.6: long K axes take pairs, short ones do not.
Plan plan_product(long long M, int N, int kblocks, int sms, int max_splits) {
  constexpr double TILE_CLOCKS = 1500.0, PAIR_TILE_CLOCKS = 3700.0;
  Plan best{256, 1};
  double best_cost = 1e300;
  for (int bn = TILE_PAIR; bn >= 64; bn >>= 1) {
    const int units = bn == TILE_PAIR ? sms / 2 : sms;  // tiles at a time
    const long long tiles = static_cast<long long>(ceil_div(M, tile_rows(bn))) * ceil_div(N, tile_cols(bn));
    const double block = bn == TILE_PAIR ? 470.0 : bn == 256 ? 545.0 : bn == 128 ? 450.0 : 400.0;
    // one split, or as many as fill 1 .. 4 waves
    for (int w = 0; w <= 4; ++w) {
      const long long fill = w == 0 ? 1 : static_cast<long long>(w) * units / tiles;
      const int s = static_cast<int>(fill < max_splits ? (fill < kblocks ? fill : kblocks) : (max_splits < kblocks ? max_splits : kblocks));
      if (s < 1 || (w > 0 && s == 1)) continue;
      const double waves = ceil_div(tiles * s, units);
      // partial tiles: written and read back, 8 bytes an element, at about 3000 bytes a clock for the whole device
      const double join = s > 1 ? 4000.0 + static_cast<double>(tiles) * tile_rows(bn) * tile_cols(bn) * s * 8.0 / 3000.0 : 0.0;
      const double cost = waves * (ceil_div(kblocks, s) * block + (bn == TILE_PAIR ? PAIR_TILE_CLOCKS : TILE_CLOCKS)) + join;
      if (cost < best_cost * 0.999) best_cost = cost, best = {bn, s};
    }
  }
  return best;
}

// Four epilogue groups instead of two, at the price of a shorter ring: where the epilogue is longer than a tile's products, with few
// K blocks and several tiles a CTA, or with a residual that is read element by element.  Two and four, us: [64800, 128] to 512, gelu
// 28.8 and 25.3; [16384, 320] to 1024, gelu 19.7 and 19.3, 512 22.8 and 23.4; [2000, 256] to 1024, one tile a CTA, 5.9 and 6.4;
// [12360, 578] to 2849 with a residual of odd rows 117.7 and 94.1, [9000, 4001] to 1001 112.9 and 113.2.
static bool four_groups(const Gemm& g, int sms) {
  return g.r_plain || (g.kblocks <= 6 && static_cast<long long>(g.tiles_m) * g.tiles_n > sms);
}

struct ForwardPlan {
  bool pad_x, pad_w;
  int kp;
  size_t x_off, w_off, total;
};
static ForwardPlan plan_forward(const Forward& a) {
  ForwardPlan f{};
  const int es = a.e4m3 ? 1 : 2;
  f.kp = pitch_of(a.K, es);
  f.pad_x = !tma::mappable(a.x, a.T, a.xs, es);
  f.pad_w = !tma::mappable(a.w, a.N, a.ws, es);
  if (f.pad_x) f.x_off = f.total, f.total += align256(static_cast<size_t>(a.T) * f.kp * es);
  if (f.pad_w) f.w_off = f.total, f.total += align256(static_cast<size_t>(a.N) * f.kp * es);
  return f;
}

size_t forward_workspace(const Forward& a, int) { return plan_forward(a).total; }

cudaError_t forward(const Forward& a, void* ws, unsigned int* err, int sms, cudaStream_t stream) {
  const ForwardPlan f = plan_forward(a);
  const int es = a.e4m3 ? 1 : 2, os = a.out_f32 ? 4 : 2;
  const void *x = a.x, *w = a.w;
  long long xs = a.xs, wst = a.ws;
  cudaError_t e;
  Copy cx{}, cw{};
  if (f.pad_x) {
    x = static_cast<char*>(ws) + f.x_off, xs = f.kp;
    cx = copy_of(static_cast<char*>(ws) + f.x_off, a.x, a.T, a.K, a.xs, f.kp, es);
  }
  if (f.pad_w) {
    w = static_cast<char*>(ws) + f.w_off, wst = f.kp;
    cw = copy_of(static_cast<char*>(ws) + f.w_off, a.w, a.N, a.K, a.ws, f.kp, es);
  }
  if ((e = to_pitch(cx, cw, sms, stream)) != cudaSuccess) return e;
  if (use_few(a.T, ceil_div(a.K, 128 / es))) return forward_few(a, x, xs, w, wst, false, err, sms, stream);
  Gemm g{};
  g.kblocks = ceil_div(a.K, 128 / es);
  const Plan pl = plan_product(a.T, a.N, g.kblocks, sms, 1);
  g.tiles_m = ceil_div(a.T, tile_rows(pl.bn)), g.tiles_n = ceil_div(a.N, tile_cols(pl.bn));
  g.splits = 1;
  g.M = static_cast<int>(a.T), g.N = a.N, g.act = a.act;
  g.bias = a.bias, g.sm = a.x_scale, g.sn = a.w_scale;
  g.y = a.y, g.r = a.r, g.p = a.p, g.ys = a.ys, g.rs = a.rs, g.ps = a.ps;
  g.has_r = a.r != nullptr, g.has_p = a.p != nullptr;
  g.y_plain = !tma::storable(a.y, a.T, a.N, a.ys, os);
  g.r_plain = a.r && !tma::mappable(a.r, a.T, a.rs, os);
  g.p_plain = a.p && !tma::storable(a.p, a.T, a.N, a.ps, 2);
  g.err = err;
  if (!tma::encode_rows(&g.ta, x, es, a.T, a.K, xs, GEMM_BM) || !tma::encode_rows(&g.tb, w, es, a.N, a.K, wst, tile_b_rows(pl.bn)) ||
      (!g.y_plain && !tma::encode_rows(&g.ty, a.y, os, a.T, a.N, a.ys, GEMM_BM)) ||
      (g.has_r && !g.r_plain && !tma::encode_rows(&g.tr, a.r, os, a.T, a.N, a.rs, GEMM_BM)) ||
      (g.has_p && !g.p_plain && !tma::encode_rows(&g.tp, a.p, 2, a.T, a.N, a.ps, GEMM_BM)))
    return cudaErrorInvalidValue;
  if ((pl.bn == 128 || pl.bn == 256) && four_groups(g, sms))
    return a.e4m3 ? gemm_e4m3_four(g, a.out_f32, pl.bn, sms, stream) : gemm_forward_four(g, a.out_f32, pl.bn, sms, stream);
  return a.e4m3 ? gemm_e4m3(g, a.out_f32, pl.bn, sms, stream) : gemm_forward(g, a.out_f32, pl.bn, sms, stream);
}

// Threads a row of k_dp, eight columns each.
static int dp_lanes(int N) { return N <= 64 ? 8 : N <= 128 ? 16 : 32; }

struct BackwardPlan {
  bool fused;  // dp, db's partial sums and dx in one kernel (whtmix_gemm_dp.cu)
  bool own_dp, pad_x, pad_w;
  int np, kp, chunks;  // pitches of dp, and of x and W; db's chunks of rows
  Plan dx, dw;
  int dx_split_rows, split_rows;
  size_t dp_off, x_off, w_off, db_off, dx_off, dw_off, total;
};
static BackwardPlan plan_backward(const Backward& a, int sms) {
  BackwardPlan b{};
  b.np = pitch_of(a.N, 2), b.kp = pitch_of(a.K, 2);
  b.own_dp = (a.dx || a.dw) && (a.act != ACT_NONE || !tma::mappable(a.dy, a.T, a.dys, 2));
  // one pass over dy and p instead of a kernel for dp and a product that reads it again; tiles of 128 tokens on half the SMs at least
  b.fused = a.dx && a.act != ACT_NONE && a.K <= 256 && tma::mappable(a.dy, a.T, a.dys, 2) && tma::mappable(a.p, a.T, a.ps, 2) &&
            2ll * ceil_div(a.T, GEMM_BM) >= sms;
  b.pad_x = a.dw && !tma::mappable(a.x, a.T, a.xs, 2);
  b.pad_w = a.dx && !tma::mappable(a.w, a.N, a.ws, 2);
  auto take = [&](size_t bytes) {
    const size_t off = b.total;
    b.total += align256(bytes);
    return off;
  };
  if (b.fused ? a.dw != nullptr : b.own_dp) b.dp_off = take(static_cast<size_t>(a.T) * b.np * 2);
  if (b.pad_x) b.x_off = take(static_cast<size_t>(a.T) * b.kp * 2);
  if (b.pad_w) b.w_off = take(static_cast<size_t>(a.N) * b.kp * 2);
  if (b.fused) {
    b.chunks = ceil_div(a.T, GEMM_BM);
    if (a.db) b.db_off = take(static_cast<size_t>(b.chunks) * a.N * 4);
  } else if (a.db || b.own_dp) {
    const int strips = ceil_div(a.N, 8 * dp_lanes(a.N)), rows = ceil_div(a.T, 512 / dp_lanes(a.N)), most = (4 * sms + strips - 1) / strips;  // one wave
    b.chunks = rows < most ? rows : most;
    if (b.chunks > 65535) b.chunks = 65535;
    if (a.T <= 128) b.chunks = 1;  // db comes whole from one CTA a strip: a launch less
    if (a.db && b.chunks > 1) b.db_off = take(static_cast<size_t>(b.chunks) * a.N * 4);
  }
  if (a.dx && !b.fused) {
    b.dx = plan_product(a.T, a.K, ceil_div(a.N, 64), sms, a.split_dx ? 2 * sms : 1);
    b.dx_split_rows = ceil_div(a.T, tile_rows(b.dx.bn)) * tile_rows(b.dx.bn);
    if (b.dx.splits > 1) b.dx_off = take(static_cast<size_t>(b.dx.splits) * b.dx_split_rows * pitch_of(a.K, 4) * 4);
  }
  if (a.dw) {
    b.dw = plan_product(a.N, a.K, ceil_div(a.T, 64), sms, 2 * sms);
    b.split_rows = ceil_div(a.N, tile_rows(b.dw.bn)) * tile_rows(b.dw.bn);
    if (b.dw.splits > 1) b.dw_off = take(static_cast<size_t>(b.dw.splits) * b.split_rows * pitch_of(a.K, 4) * 4);
  }
  return b;
}

size_t backward_workspace(const Backward& a, int sms) { return plan_backward(a, sms).total; }

cudaError_t backward(const Backward& a, void* ws, unsigned int* err, int sms, cudaStream_t stream) {
  const BackwardPlan b = plan_backward(a, sms);
  char* base = static_cast<char*>(ws);
  const Copy cx = b.pad_x ? copy_of(base + b.x_off, a.x, a.T, a.K, a.xs, b.kp, 2) : Copy{};
  const Copy cw = b.pad_w ? copy_of(base + b.w_off, a.w, a.N, a.K, a.ws, b.kp, 2) : Copy{};
  cudaError_t e = to_pitch(cx, cw, sms, stream);
  if (e != cudaSuccess) return e;
  const void* dp = a.dy;
  long long dps = a.dys;
  if (b.fused) {
    void* d = a.dw ? base + b.dp_off : nullptr;
    DpProduct g{};
    g.M = static_cast<int>(a.T), g.N = a.N, g.K = a.K, g.tiles_m = b.chunks, g.kblocks = ceil_div(a.N, 64), g.act = a.act;
    g.part = a.db ? reinterpret_cast<float*>(base + b.db_off) : nullptr;
    g.store_dp = d != nullptr;
    g.dx = a.dx, g.dxs = a.dxs, g.dx_plain = !tma::storable(a.dx, a.T, a.K, a.dxs, 2);
    g.err = err;
    if (!tma::encode_rows(&g.tdy, a.dy, 2, a.T, a.N, a.dys, GEMM_BM) || !tma::encode_rows(&g.tp, a.p, 2, a.T, a.N, a.ps, GEMM_BM) ||
        !tma::encode_rows(&g.tw, b.pad_w ? base + b.w_off : a.w, 2, a.N, a.K, b.pad_w ? b.kp : a.ws, 64) ||
        (d && !tma::encode_rows(&g.tdp, d, 2, a.T, b.np, b.np, GEMM_BM)) ||
        (!g.dx_plain && !tma::encode_rows(&g.tdx, a.dx, 2, a.T, a.K, a.dxs, GEMM_BM)))
      return cudaErrorInvalidValue;
    if ((e = gemm_dp(g, sms, stream)) != cudaSuccess) return e;
    if (d) dp = d, dps = b.np;
    if (a.db && (e = norm::add_rows(g.part, a.db, a.N, b.chunks, stream)) != cudaSuccess) return e;
  } else if (a.db || b.own_dp) {
    Backward c = a;
    __nv_bfloat16* d = b.own_dp ? reinterpret_cast<__nv_bfloat16*>(base + b.dp_off) : nullptr;
    float* part = !a.db ? nullptr : b.chunks > 1 ? reinterpret_cast<float*>(base + b.db_off) : a.db;
    long long np = b.np;
    int chunks = b.chunks;
    const bool al = a.N % 8 == 0 && tma::mappable(a.dy, a.T, a.dys, 2) && (a.act == ACT_NONE || tma::mappable(a.p, a.T, a.ps, 2));
    cudaLaunchConfig_t cfg = {};
    const int tx = dp_lanes(a.N);
    cfg.gridDim = dim3(ceil_div(a.N, 8 * tx), chunks);
    cfg.blockDim = dim3(THREADS_256);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg,
                           tx == 8    ? (al ? k_dp<true, 8> : k_dp<false, 8>)
                           : tx == 16 ? (al ? k_dp<true, 16> : k_dp<false, 16>)
                                      : (al ? k_dp<true, 32> : k_dp<false, 32>),
                           c, d, np, part, chunks);
    if (e != cudaSuccess) return e;
    if (b.own_dp) dp = d, dps = b.np;
    if (a.db && chunks > 1 && (e = norm::add_rows(part, a.db, a.N, chunks, stream)) != cudaSuccess) return e;
  }
  if (a.dx && !b.fused) {
    Gemm g{};
    g.kblocks = ceil_div(a.N, 64);
    g.tiles_m = ceil_div(a.T, tile_rows(b.dx.bn)), g.tiles_n = ceil_div(a.K, tile_cols(b.dx.bn));
    g.splits = b.dx.splits;
    g.split_rows = g.splits > 1 ? b.dx_split_rows : 0;
    g.M = static_cast<int>(a.T), g.N = a.K;
    g.err = err;
    const bool split = g.splits > 1;
    const int os = split ? 4 : 2;
    void* out = split ? static_cast<void*>(base + b.dx_off) : a.dx;
    const long long rows = split ? static_cast<long long>(g.splits) * b.dx_split_rows : a.T, stride = split ? pitch_of(a.K, 4) : a.dxs;
    g.y = out, g.ys = stride, g.y_plain = !split && !tma::storable(a.dx, a.T, a.K, a.dxs, 2);
    if (!tma::encode_rows(&g.ta, dp, 2, a.T, a.N, dps, GEMM_BM) ||
        !tma::encode_rows(&g.tb, b.pad_w ? base + b.w_off : a.w, 2, a.N, a.K, b.pad_w ? b.kp : a.ws, 64) ||
        (!g.y_plain && !tma::encode_rows(&g.ty, out, os, rows, a.K, stride, GEMM_BM)))
      return cudaErrorInvalidValue;
    if ((e = gemm_dx(g, split, b.dx.bn, sms, stream)) != cudaSuccess) return e;
    if (split && (e = sum_splits(a.dx, false, a.dxs, static_cast<const float*>(out), static_cast<int>(a.T), a.K, pitch_of(a.K, 4), b.dx_split_rows,
                                 g.splits, sms, stream)) != cudaSuccess)
      return e;
  }
  if (a.dw) {
    Gemm g{};
    g.kblocks = ceil_div(a.T, 64);
    g.tiles_m = ceil_div(a.N, tile_rows(b.dw.bn)), g.tiles_n = ceil_div(a.K, tile_cols(b.dw.bn));
    g.splits = b.dw.splits;
    g.split_rows = b.split_rows;
    g.M = a.N, g.N = a.K;
    g.err = err;
    const bool split = g.splits > 1;
    const int os = split || a.dw_f32 ? 4 : 2;
    void* out = split ? static_cast<void*>(base + b.dw_off) : a.dw;
    const long long rows = split ? static_cast<long long>(g.splits) * b.split_rows : a.N;
    int pitch = split ? pitch_of(a.K, 4) : a.K;
    g.y = out, g.ys = pitch, g.y_plain = !split && !tma::storable(out, rows, a.K, pitch, os);  // (a partial row's end may be written over)
    if (!tma::encode_rows(&g.ta, dp, 2, a.T, a.N, dps, 64) ||
        !tma::encode_rows(&g.tb, b.pad_x ? base + b.x_off : a.x, 2, a.T, a.K, b.pad_x ? b.kp : a.xs, 64) ||
        (!g.y_plain && !tma::encode_rows(&g.ty, out, os, rows, a.K, pitch, GEMM_BM)))
      return cudaErrorInvalidValue;
    if ((e = gemm_dw(g, os == 4, b.dw.bn, sms, stream)) != cudaSuccess) return e;
    if (split)
      e = sum_splits(a.dw, a.dw_f32, a.K, static_cast<const float*>(out), a.N, a.K, pitch, b.split_rows, g.splits, sms, stream);
  }
  return e;
}

}  // namespace linear
}  // namespace whtmix
