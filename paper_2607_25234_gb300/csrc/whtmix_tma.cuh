// whtmix_tma.cuh -- TMA pieces of the matrix products: tensor maps of row-major matrices (host), tile loads and stores (device).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "whtmix_tc.cuh"

namespace whtmix {
namespace tma {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// cuTensorMapEncodeTiled through the runtime's driver entry point (no link against libcuda); null where it is missing.
inline EncodeTiledFn encode_fn() {
  static const EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ok = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
                    q == cudaDriverEntryPointSuccess;
    return reinterpret_cast<EncodeTiledFn>(ok ? p : nullptr);
  }();
  return fn;
}

// A row-major matrix can be a tensor map: 16-byte aligned rows (one row needs no stride).
inline bool mappable(const void* base, long long rows, long long stride, int es) {
  return (reinterpret_cast<uintptr_t>(base) & 15u) == 0 && (rows == 1 || (static_cast<unsigned long long>(stride) * es) % 16 == 0);
}

// A tensor map of it can be stored to: a store writes whole 16-byte pieces, zeros beyond the last column (a load's columns end
// where the map's do), so that only rows of whole pieces leave what follows them alone.
inline bool storable(const void* base, long long rows, long long cols, long long stride, int es) {
  return mappable(base, rows, stride, es) && static_cast<unsigned long long>(cols) * es % 16 == 0;
}

// [rows, cols] of es-byte elements (1: bytes, 2: bf16, 4: float), `stride` elements a row; boxes of box_rows rows x 128 bytes,
// 128-byte swizzle.  What lies outside reads as zero and is not written.
inline bool encode_rows(CUtensorMap* tm, const void* base, int es, long long rows, long long cols, long long stride, int box_rows) {
  const EncodeTiledFn f = encode_fn();
  if (!f) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t pitch = rows == 1 ? (static_cast<cuuint64_t>(cols) * es + 15) / 16 * 16 : static_cast<cuuint64_t>(stride) * es;
  const cuuint64_t strides[1] = {pitch};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(128 / es), static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t steps[2] = {1, 1};
  const CUtensorMapDataType type =
      es == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : es == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
  return f(tm, type, 2, const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Phase `parity` of an mbarrier, waited for at most WAIT_NS; false if it did not complete by then.
constexpr unsigned long long WAIT_NS = 1000000000ull;  // 1 s
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
__device__ __forceinline__ bool wait(uint64_t* b, uint32_t parity) {
  const uint32_t bar = tc::smem_u32(b);
  if (try_wait(bar, parity)) return true;
  unsigned long long t0, t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t0));
  do {
#pragma unroll 1
    for (int i = 0; i < 32; ++i)
      if (try_wait(bar, parity)) return true;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  } while (t - t0 < WAIT_NS);
  return false;
}

__device__ __forceinline__ void arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(tc::smem_u32(b)) : "memory");
}
__device__ __forceinline__ void expect_tx(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(tc::smem_u32(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void load_2d(uint32_t sdst, const CUtensorMap* tm, int x, int y, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(sdst), "l"(tm), "r"(x), "r"(y), "r"(tc::smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void store_2d(const CUtensorMap* tm, int x, int y, uint32_t ssrc) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
               ::"l"(tm), "r"(x), "r"(y), "r"(ssrc) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void wait_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void prefetch(const CUtensorMap* tm) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(tm) : "memory");
}

// ---- two CTAs of a cluster on one tile ----
// The address in CTA `rank` of the cluster of what lies at `addr` in this one.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void arrive_in(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// Into this CTA's shared memory, counted at a barrier of the pair's first CTA.
__device__ __forceinline__ void load_2d_pair(uint32_t sdst, const CUtensorMap* tm, int x, int y, uint32_t cluster_bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
               ::"r"(sdst), "l"(tm), "r"(x), "r"(y), "r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

}  // namespace tma
}  // namespace whtmix
