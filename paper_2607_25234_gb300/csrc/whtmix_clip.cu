// whtmix_clip.cu -- the common norm of many tensors and their scaling by it (clipping of a step's gradients).
//
//   norm = sqrt(sum over all tensors and elements of g^2),   out = g min(1, max_norm / (norm + 1e-6))
//
// Bound by memory: the gradients are read for the norm and again for the scaling.  A tensor is cut into chunks of CHUNK 16-byte
// vectors, counted from the 16-byte boundary at or before its first element, so that every load is aligned whatever its address; a
// CTA takes a run of chunks, the next one's loads on their way while it works on one.  A table of the tensors goes along as a kernel
// parameter (a captured graph keeps it), a launch for every MAX of them.  The scaling takes a run in descending order, the last chunks
// read first; ascending it takes as long (0.6 GB 280 and 279 us, 67 MB 33.9 and 33.5).  Short lists stay in one cluster's registers
// between the two.
// A thread's squares of one chunk are added in float32, those sums in float32 with a compensation (float64 additions are slow
// here: two a clock and SM), the threads' sums in float64; values whose squares leave float32's range are scaled by a power of two
// first, so that every finite gradient has its finite norm.  Every CTA of the scaling adds up the partial
// sums itself, in the same order: no atomics, results repeat bit for bit.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "whtmix_clip.cuh"
#include "whtmix_kernels.cuh"

namespace whtmix {
namespace clip {

constexpr int CLIP_THREADS = 256, VECTORS = 4, CHUNK = CLIP_THREADS * VECTORS;
constexpr int CLIP_CTAS = 4;  // an SM
// tensors a launch: a small table for the usual list, a large one (15 KB of parameters) for long ones
constexpr int FEW = 64, MANY = 480;
constexpr float CLIP_EPS = 1e-6f;

struct Entry {
  const uint8_t* in;
  uint8_t* out;
  long long bytes;
  int first;  // its first chunk; the top bit: bf16
};
constexpr int BF16_BIT = static_cast<int>(0x80000000u);
template <int MAX>
struct Table {
  Entry e[MAX];
  int count, chunks;
  bool in_place;  // every tensor of it
};

// A thread's vectors of a chunk.
struct Piece {
  const uint8_t *base, *lo, *hi;  // base: this thread's first vector; the tensor's bytes
  long long shift;                // out - in
  bool bf16;
};
// The tensor of a chunk: the last one whose first chunk is not beyond it.
template <int MAX>
__device__ __forceinline__ int tensor_of(const Table<MAX>& t, int chunk) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((t.e[mid].first & ~BF16_BIT) <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}
__device__ __forceinline__ Piece piece_of(const Entry& e, int chunk) {
  Piece p;
  p.lo = e.in, p.hi = e.in + e.bytes;
  p.base = e.in - (reinterpret_cast<uintptr_t>(e.in) & 15u) + (static_cast<long long>(chunk - (e.first & ~BF16_BIT)) * CHUNK + threadIdx.x) * 16;
  p.shift = e.out - e.in;
  p.bf16 = e.first < 0;
  return p;
}
// The chunks of a run, one after another (UP) or from its last to its first.
template <int MAX, bool UP>
struct Run {
  const Table<MAX>& t;
  int chunk, end, i;  // end: one beyond the last to come
  __device__ __forceinline__ Run(const Table<MAX>& table) : t(table) {
    const int first = static_cast<int>(static_cast<long long>(t.chunks) * blockIdx.x / gridDim.x);
    const int last = static_cast<int>(static_cast<long long>(t.chunks) * (blockIdx.x + 1) / gridDim.x);  // (never empty)
    chunk = UP ? first : last - 1, end = UP ? last : first - 1;
    i = tensor_of(t, chunk);
  }
  __device__ __forceinline__ bool more() const { return chunk != end; }
  // this chunk, and on to the next one
  __device__ __forceinline__ Piece take() {
    const Entry e = t.e[i];
    const Piece p = piece_of(e, chunk);
    if (UP) {
      ++chunk;
      if (i + 1 < t.count && (t.e[i + 1].first & ~BF16_BIT) <= chunk) ++i;  // (a tensor has a chunk at least)
    } else {
      --chunk;
      if (chunk < (e.first & ~BF16_BIT)) --i;
    }
    return p;
  }
};
__device__ __forceinline__ const uint8_t* vector_at(const Piece& p, int u) { return p.base + u * (CLIP_THREADS * 16); }
// the vector at q, zeros outside the tensor
__device__ __forceinline__ uint4 load(const Piece& p, const uint8_t* q) {
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (q >= p.lo && q + 16 <= p.hi) {
    v = *reinterpret_cast<const uint4*>(q);
  } else if (q + 16 > p.lo && q < p.hi) {  // a tensor's first or last vector, in halves of words (elements are aligned)
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (q + 2 * i >= p.lo && q + 2 * i < p.hi) w[i >> 1] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(q + 2 * i)) << (16 * (i & 1));
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return v;
}
__device__ __forceinline__ void load_all(const Piece& p, uint4 (&u)[VECTORS]) {
#pragma unroll
  for (int k = 0; k < VECTORS; ++k) u[k] = load(p, vector_at(p, k));
}

// sum of the squares of s times the values of u, two accumulators
__device__ __forceinline__ float squares(const uint4 (&u)[VECTORS], bool bf16, float s) {
  float a = 0.f, b = 0.f;
#pragma unroll
  for (int k = 0; k < VECTORS; ++k) {
    const uint32_t w[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (bf16) {
        const float x = __uint_as_float(w[j] << 16) * s, y = __uint_as_float(w[j] & 0xffff0000u) * s;
        a = fmaf(x, x, a), b = fmaf(y, y, b);
      } else {
        const float x = __uint_as_float(w[j]) * s;
        if (j & 1) b = fmaf(x, x, b); else a = fmaf(x, x, a);
      }
    }
  }
  return a + b;
}
// A thread's sum: float32 with the rounding errors beside it, and in float64 what lies beyond [2^-100, 2^90] (2^37 chunks in range
// stay finite).  Beyond, the squares are taken again with the values scaled by 2^110 (all of them are below 2^-50 then) or 2^-72.
struct Sum {
  float s = 0.f, err = 0.f;
  double far = 0.0;
  __device__ __forceinline__ void add(const uint4 (&u)[VECTORS], bool bf16) {
    const float v = squares(u, bf16, 1.f);
    if (v >= 0x1p-100f && v <= 0x1p90f) {
      const float y = v - err, t = s + y;
      err = (t - s) - y;
      s = t;
      return;
    }
    uint32_t any = 0;
#pragma unroll
    for (int k = 0; k < VECTORS; ++k) any |= u[k].x | u[k].y | u[k].z | u[k].w;
    if ((any & 0x7fff7fffu) == 0 && (bf16 || (any & 0x7fffffffu) == 0)) return;
    const bool tiny = v < 1.f;
    far += static_cast<double>(squares(u, bf16, tiny ? 0x1p110f : 0x1p-72f)) * (tiny ? 0x1p-220 : 0x1p144);
  }
};

// The CTA's sum, in thread 0.  float64 operations are taken by as few warps as there are values: all threads' own would be 3 us here.
__device__ __forceinline__ double add_up(Sum a) {
  __shared__ float2 s[CLIP_THREADS / 32];
  __shared__ double s_far[CLIP_THREADS / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float hi = a.s, lo = -a.err;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {  // sums of two float32, what rounding takes from the first kept in the second
    const float h = __shfl_xor_sync(0xffffffffu, hi, o), l = __shfl_xor_sync(0xffffffffu, lo, o);
    const float t = hi + h, b = t - hi;
    lo += l + ((hi - (t - b)) + (h - b));
    hi = t;
  }
  const bool far = __any_sync(0xffffffffu, a.far != 0.0);  // (NaN too)
  if (far) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a.far += __shfl_xor_sync(0xffffffffu, a.far, o);
  }
  if (lane == 0) s[warp] = make_float2(hi, lo), s_far[warp] = far ? a.far : 0.0;
  __syncthreads();
  double sum = 0.0;
  if (warp == 0) {
    const float2 v = lane < CLIP_THREADS / 32 ? s[lane] : make_float2(0.f, 0.f);
    sum = static_cast<double>(v.x) + static_cast<double>(v.y) + (lane < CLIP_THREADS / 32 ? s_far[lane] : 0.0);
#pragma unroll
    for (int o = CLIP_THREADS / 64; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  }
  return sum;
}
// The sum of the parts, in the first warp.
__device__ __forceinline__ double add_parts(const double* part, int parts) {
  double a = 0.0;
  for (int i = threadIdx.x; i < parts; i += 32) a += __ldcg(part + i);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
  return a;
}

// The root of the sum and the factor min(1, max_norm / (norm + 1e-6)), NaN for NaN.  A factor below 2^-120 (norms that float32 does not
// hold) loses its digits as a float32: there `ratio` is to be used.
struct Scale {
  float norm, f;
  double ratio;  // 0 where f does
  __device__ __forceinline__ void set(double sum, float max_norm) {
    ratio = 0.0;
    if (sum >= 0x1p-120 && sum <= 0x1p120) {
      norm = sqrtf(static_cast<float>(sum));
      const float r = max_norm / (norm + CLIP_EPS);
      f = r >= 1.f ? 1.f : r;
    } else {
      const double root = sqrt(sum), r = max_norm / (root + CLIP_EPS);
      norm = static_cast<float>(root), f = r >= 1.0 ? 1.f : static_cast<float>(r);
      if (r < 0x1p-120) ratio = r;
    }
  }
};

// part[blockIdx.x] = the sum of squares of this CTA's chunks
template <int MAX>
__global__ void __launch_bounds__(CLIP_THREADS, CLIP_CTAS) k_squares(const __grid_constant__ Table<MAX> t, double* part) {
  pdl_wait();
  Run<MAX, true> run(t);
  Sum sum;
  Piece p = run.take();
  uint4 u[VECTORS];
  load_all(p, u);
  while (run.more()) {
    const bool bf16 = p.bf16;
    uint4 next[VECTORS];
    p = run.take();
    load_all(p, next);
    sum.add(u, bf16);
#pragma unroll
    for (int k = 0; k < VECTORS; ++k) u[k] = next[k];
  }
  sum.add(u, p.bf16);
  const double all = add_up(sum);
  if (threadIdx.x == 0) part[blockIdx.x] = all;
  pdl_trigger();
}

// *total = the sum of the parts, *norm its root (each or null); one warp
__global__ void __launch_bounds__(32) k_total(const double* part, int parts, double* total, float* norm) {
  pdl_wait();
  const double sum = add_parts(part, parts);
  if (threadIdx.x == 0) {
    Scale s;
    s.set(sum, 0.f);
    if (total) *total = sum;
    if (norm) *norm = s.norm;
  }
  pdl_trigger();
}

// f(x) of each value of u, to the piece's place
template <class F>
__device__ __forceinline__ void store_mapped(const Piece& p, const uint4 (&u)[VECTORS], F&& f) {
#pragma unroll
  for (int k = 0; k < VECTORS; ++k) {
    uint32_t w[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (p.bf16) {
        __nv_bfloat162 b = __floats2bfloat162_rn(f(__uint_as_float(w[j] << 16)), f(__uint_as_float(w[j] & 0xffff0000u)));
        w[j] = *reinterpret_cast<uint32_t*>(&b);
      } else {
        w[j] = __float_as_uint(f(__uint_as_float(w[j])));
      }
    }
    const uint8_t* q = vector_at(p, k);
    uint8_t* o = const_cast<uint8_t*>(q) + p.shift;
    if (q >= p.lo && q + 16 <= p.hi && (p.shift & 15) == 0) {
      *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
    } else if (q + 16 > p.lo && q < p.hi) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (q + 2 * j >= p.lo && q + 2 * j < p.hi) *reinterpret_cast<uint16_t*>(o + 2 * j) = static_cast<uint16_t>(w[j >> 1] >> (16 * (j & 1)));
    }
  }
}
// (the far products kept out of the usual path: on both sides of a choice an element they took 1.25 ms of 0.6 GB)
static __device__ __noinline__ float times_far(float x, double ratio) { return static_cast<float>(x * ratio); }
__device__ __forceinline__ void store_scaled(const Piece& p, const uint4 (&u)[VECTORS], const Scale& s) {
  if (s.ratio != 0.0)
    store_mapped(p, u, [&](float x) { return times_far(x, s.ratio); });
  else
    store_mapped(p, u, [&](float x) { return x * s.f; });
}

// The first chunk is on its way while the parts are added up.
template <int MAX>
__global__ void __launch_bounds__(CLIP_THREADS, CLIP_CTAS) k_scale(const __grid_constant__ Table<MAX> t, const double* part, int parts,
                                                                   float max_norm, float* norm) {
  pdl_wait();
  Run<MAX, false> run(t);
  Piece p = run.take();
  uint4 u[VECTORS];
  load_all(p, u);
  __shared__ Scale s_scale;
  if (threadIdx.x < 32) {
    const double sum = add_parts(part, parts);
    if (threadIdx.x == 0) s_scale.set(sum, max_norm);
  }
  __syncthreads();
  const Scale s = s_scale;
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = s.norm;
  if (s.f == 1.f && t.in_place) return;
  while (run.more()) {
    const Piece at = p;
    uint4 next[VECTORS];
    p = run.take();
    load_all(p, next);
    store_scaled(at, u, s);
#pragma unroll
    for (int k = 0; k < VECTORS; ++k) u[k] = next[k];
  }
  store_scaled(p, u, s);
  pdl_trigger();
}

// ---- few chunks ----
// Lists of up to SMALL chunks: one cluster holds them all in registers between the sum and the scaling; its CTAs put their sums into
// one another's shared memory, behind a barrier of the cluster that the loads hide (a CTA's shared memory is there once it has
// started) and before another.  One launch, no scratch.
constexpr int CLUSTER = 8, HELD = 3, SMALL = CLUSTER * HELD;
__global__ void __launch_bounds__(CLIP_THREADS) k_clip_few(const __grid_constant__ Table<FEW> t, float max_norm, float* norm, int scale) {
  __shared__ double s_all[CLUSTER];
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = static_cast<int>(cluster.block_rank());
  cluster.barrier_arrive();  // waited for before the first store to another CTA: by then all have started
  pdl_wait();
  Piece p[HELD];
  uint4 u[HELD][VECTORS];
  Sum sum;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int c = rank + CLUSTER * i;
    if (c < t.chunks) {
      p[i] = piece_of(t.e[tensor_of(t, c)], c);
      load_all(p[i], u[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (rank + CLUSTER * i < t.chunks) sum.add(u[i], p[i].bf16);
  const double mine = __shfl_sync(0xffffffffu, add_up(sum), 0);
  cluster.barrier_wait();
  if (threadIdx.x < CLUSTER) *cluster.map_shared_rank(&s_all[rank], threadIdx.x) = mine;
  cluster.sync();
  __shared__ Scale s_scale;
  if (threadIdx.x == 0) {
    double all = s_all[0];
#pragma unroll
    for (int i = 1; i < CLUSTER; ++i) all += s_all[i];
    s_scale.set(all, max_norm);
  }
  __syncthreads();
  const Scale s = s_scale;
  if (norm && rank == 0 && threadIdx.x == 0) *norm = s.norm;
  if (scale && !(s.f == 1.f && t.in_place)) {
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (rank + CLUSTER * i < t.chunks) store_scaled(p[i], u[i], s);
  }
  pdl_trigger();
}

// ---- host ----

constexpr int PARTS_AT_ONCE = 4096;  // more are added up once, before the scaling

static long long chunks_of(const Item& i) {
  const long long bytes = i.n * (i.bf16 ? 2 : 4) + static_cast<long long>(reinterpret_cast<uintptr_t>(i.in) & 15u);
  return (bytes + 16ll * CHUNK - 1) / (16ll * CHUNK);
}
static int ctas(long long chunks, int sms) {
  const long long most = static_cast<long long>(CLIP_CTAS) * sms;
  return static_cast<int>(chunks < most ? chunks : most);
}

// f(table, its CTAs) for each launch's tensors, in order; stops at an error
template <int MAX, class F>
static cudaError_t each(const Call& a, int sms, F&& f) {
  Table<MAX> t;
  t.count = 0, t.chunks = 0, t.in_place = true;
  for (long long i = 0; i < a.count; ++i) {
    const Item& m = a.items[i];
    t.e[t.count++] = {static_cast<const uint8_t*>(m.in), static_cast<uint8_t*>(m.out ? m.out : const_cast<void*>(m.in)), m.n * (m.bf16 ? 2 : 4),
                      t.chunks | (m.bf16 ? BF16_BIT : 0)};
    t.chunks += static_cast<int>(chunks_of(m));
    t.in_place = t.in_place && m.out == m.in;
    if (t.count == MAX || i + 1 == a.count || t.chunks + chunks_of(a.items[i + 1]) >= (1ll << 31)) {
      const cudaError_t e = f(t, ctas(t.chunks, sms));
      if (e != cudaSuccess) return e;
      t.count = 0, t.chunks = 0, t.in_place = true;
    }
  }
  return cudaSuccess;
}
template <int MAX>
static long long parts_of(const Call& a, int sms) {
  long long n = 0;
  (void)each<MAX>(a, sms, [&](Table<MAX>&, int grid) {
    n += grid;
    return cudaSuccess;
  });
  return n;
}
static bool long_list(const Call& a) { return a.count > FEW; }

// A list for one cluster.
static bool few_chunks(const Call& a) {
  long long chunks = 0;
  for (long long i = 0; i < a.count && chunks <= SMALL; ++i) chunks += chunks_of(a.items[i]);
  return !long_list(a) && chunks <= SMALL;
}
static cudaError_t run_few(const Call& a, int sms, cudaStream_t stream) {
  return each<FEW>(a, sms, [&](Table<FEW>& t, int) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CLUSTER);
    cfg.blockDim = dim3(CLIP_THREADS);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CLUSTER;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_clip_few, t, a.max_norm, a.norm, a.scale ? 1 : 0);
  });
}

size_t workspace(const Call& a, int sms) {
  if (few_chunks(a)) return 0;
  return (1 + (long_list(a) ? parts_of<MANY>(a, sms) : parts_of<FEW>(a, sms))) * sizeof(double);
}

template <int MAX>
static cudaError_t run_t(const Call& a, void* ws, int sms, cudaStream_t stream) {
  double *total = static_cast<double*>(ws), *part = total + 1;
  int parts = 0;
  cudaError_t e = each<MAX>(a, sms, [&](Table<MAX>& t, int grid) {
    double* p = part + parts;
    parts += grid;
    void* args[] = {&t, &p};
    return launch_pdl(reinterpret_cast<const void*>(k_squares<MAX>), static_cast<unsigned>(grid), CLIP_THREADS, 0, stream, args);
  });
  if (e != cudaSuccess) return e;
  const double* from = part;
  float* norm = a.norm;
  if (!a.scale || parts > PARTS_AT_ONCE) {
    double* to = a.scale ? total : nullptr;
    void* args[] = {&from, &parts, &to, &norm};
    if ((e = launch_pdl(reinterpret_cast<const void*>(k_total), 1, 32, 0, stream, args)) != cudaSuccess || !a.scale) return e;
    from = total, parts = 1, norm = nullptr;
  }
  float max_norm = a.max_norm;
  return each<MAX>(a, sms, [&](Table<MAX>& t, int grid) {
    void* args[] = {&t, &from, &parts, &max_norm, &norm};
    const cudaError_t r = launch_pdl(reinterpret_cast<const void*>(k_scale<MAX>), static_cast<unsigned>(grid), CLIP_THREADS, 0, stream, args);
    norm = nullptr;
    return r;
  });
}
cudaError_t run(const Call& a, void* ws, int sms, cudaStream_t stream) {
  if (few_chunks(a)) return run_few(a, sms, stream);
  return long_list(a) ? run_t<MANY>(a, ws, sms, stream) : run_t<FEW>(a, ws, sms, stream);
}

}  // namespace clip
}  // namespace whtmix
