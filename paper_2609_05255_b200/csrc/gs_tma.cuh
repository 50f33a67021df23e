// Tiled copies by the tensor memory accelerator, and waits for them.  Included inside namespace gs's unnamed namespace after
// gs_tcgen05.cuh, by translation units that include <cuda.h>.  Copies go to the CTA that issues them, never to others of a cluster.
//
// A matrix of 16-bit values, row-major with rows `ld` elements apart, is copied in boxes of 64 columns (128 bytes: the span
// of the 128-byte swizzle, which moves the 16-byte chunk c of a row r of the box to c ^ (r mod 8)) and a number of rows.  What a box
// has outside the matrix is zero on the way in and left alone on the way out.
#pragma once

namespace tma {

constexpr int kBoxCols = 64;
constexpr uint32_t kRowBytes = 128;

// Made on the host for every call: it holds the addresses that the call was given.  False where the driver refuses it.
inline bool make_map(CUtensorMap *map, int dtype, const void *base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  typedef CUresult (*Encode)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                             const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void *f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<Encode>(f);
  }();
  if (!encode) return false;
  if (rows <= 1) ld = (cols + 7) / 8 * 8;      // (no second row to find)
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {(cuuint32_t)kBoxCols, (cuuint32_t)box_rows}, step[2] = {1, 1};
  return encode(map, dtype == GS_TYPE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides, box,
                step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

#ifdef __CUDACC__
// `col` is a multiple of kBoxCols: every copy starts on a 16-byte boundary.
__device__ __forceinline__ void load(uint32_t dst, const CUtensorMap *map, int col, int row, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(col), "r"(row), "r"(bar) : "memory");
}
__device__ __forceinline__ void store(const CUtensorMap *map, int col, int row, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(col), "r"(row), "r"(src) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kLeft) : "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
// kCluster: what the other CTA of a cluster wrote before it arrived is visible, too.
template <bool kCluster = false>
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
  uint32_t done;
  if (kCluster)
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
// Waits for a phase, at most 2^32 cycles (about two seconds) or until another role of the CTA has given up.  Who gives up says so
// in *dead: everybody's waits then end, and the CTA leaves in order.
template <bool kCluster = false>
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile uint32_t *dead) {
  if (try_wait<kCluster>(bar, parity)) return true;
  const long long begin = clock64();
  while (!try_wait<kCluster>(bar, parity)) {
    if (*dead) return false;
    if (clock64() - begin > (1ll << 32)) {
      *dead = 1u;
      return false;
    }
  }
  return true;
}
// The same without a word to the others: for what has to end before a CTA leaves.
__device__ __forceinline__ void settle(uint32_t bar, uint32_t parity) {
  const long long begin = clock64();
  while (!try_wait(bar, parity) && clock64() - begin < (1ll << 28)) {}
}
#endif

}  // namespace tma
