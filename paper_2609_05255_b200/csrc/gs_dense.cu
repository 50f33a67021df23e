// Dense layers over the rows of a matrix, forward and backward, on the 5th-generation tensor cores.
//
//   forward    z = x W^T + b (fp32);  preact = z rounded, where it is kept;  y = act(z) + residual, rounded once
//   backward   dz = dy act'(preact);  dx = dz W;  dW = dz^T x (fp32);  db = sum over rows of dz (fp32)
//
// Operands are fp16 or bf16, accumulators fp32 in tensor memory.  Rows are many (a row per Gaussian) and the widths those of
// small networks, so up to widths of about 256 the bytes of x, y, dy, preact and dx bound the layer, beyond that the tensor
// cores.  Everything row-shaped moves by TMA in boxes of 64 columns with the 128-byte swizzle, which the MMAs read as it is:
// rows and columns that the matrices do not have come as zeros and are not written.
//
// k_dense_rows (forward and dx): a persistent CTA per SM owns one tile of output columns and walks over tiles of 128 rows.
// One thread issues the loads, one the MMAs, four warps take accumulators out of tensor memory (two of them, so that the next tile's
// products run meanwhile) into swizzled tiles that leave by TMA.  The weights of the column tile stay in shared memory for the
// whole walk where they fit, else they come with every step.
// k_dense_weights (dW, db): the contraction runs over the rows, which are split over the CTAs; both operands are read MN-major, as
// they lie in memory.  The CTAs' sums go to the workspace and are added in a fixed order by k_dense_sums: no atomics, the same bits
// from run to run.
//
// In both backward kernels eight warps turn the tile of dy in shared memory into dz, in place, with the tile of preact beside
// it: elementwise, so the layout does not matter.  dz is an fp32 product; rounded to 16 bits it would cost dW its fp32 accuracy and dx half
// again the error of its own rounding.  So for the smooth activations it becomes two or three operands that sum up to
// it: high, and what the rounding left (which takes the place of preact); three for the weights in bf16, whose two would keep 16 bits.
// For dW in fp16 what is left is scaled by 2^11 (it would fall below fp16's range) and summed in an accumulator of its own.
// Without activation, and with ReLU, dz is dy or 0: exact as it is.
//
// Waits are bounded (tma::wait): one that runs out sets *timeout, and the CTA leaves without its results.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gs_device.cuh"

namespace gs {
namespace {

#include "gs_rows.cuh"
#include "gs_tcgen05.cuh"
#include "gs_tma.cuh"

constexpr int kRows = 128;                    // rows of a tile of k_dense_rows, lanes of tensor memory
constexpr int kStep = 64;                     // columns (k_dense_rows) or rows (k_dense_weights) of a pipeline step
constexpr uint32_t kTileBytes = kRows * tma::kRowBytes;       // 128 x 64 values
constexpr uint32_t kBoxBytes = kStep * tma::kRowBytes;        // 64 x 64 values
constexpr int kMaxStages = 8;
constexpr uint32_t kSmemMost = 232448;        // 227 KB

enum { kWarpLoad = 0, kWarpMma = 1, kWarpResidual = 2, kWarpEpilogue = 4, kWarpTransform = 8 };
constexpr int kTransformThreads = 256;
enum { kWarpWorker = 4, kWorkerWarps = 8 };   // of k_dense_weights, behind the warps that load and issue

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float logistic(float x) { return rcp_approx(1.f + ex2_approx(-1.4426950408889634f * x)); }
// gelu(z) = z logistic(2 sqrt(2 / pi) (z + 0.044715 z^3)), the tanh form
__device__ __forceinline__ float gelu_arg(float z) { return z * fmaf(0.07135481627159806f, z * z, 1.5957691216057308f); }
__device__ __forceinline__ float activate(int act, float z) {
  if (act == GS_DENSE_RELU) return z < 0.f ? 0.f : z;      // (a NaN stays)
  if (act == GS_DENSE_SILU) return z * logistic(z);
  if (act == GS_DENSE_GELU) return z * logistic(gelu_arg(z));
  return z;
}
// act' of the smooth ones.  Beyond |z| = 128 it is 1 or 0 in fp32; the clamp keeps z^3 finite (and a NaN a NaN).
__device__ __forceinline__ float activate_grad(int act, float z) {
  z = z > 128.f ? 128.f : z < -128.f ? -128.f : z;
  const float gelu = act == GS_DENSE_GELU ? 1.f : 0.f;
  const float p = logistic(act == GS_DENSE_GELU ? gelu_arg(z) : z);
  const float slope = fmaf(gelu, fmaf(0.21406444881479418f, z * z, 0.5957691216057308f), 1.f);     // of the logistic's argument
  return fmaf(z * p * (1.f - p), slope, p);
}

// Shared-memory matrix descriptors for the 128-byte swizzle.  K-major (a row holds 64 elements of the contraction): groups of
// eight rows are 1024 bytes apart (stride byte offset); 16 elements on is 32 bytes on.  MN-major (a row is one element of
// the contraction and holds 64 of M or N): groups of eight rows are 1024 bytes apart (stride byte offset), the next 64
// of M or N a box further (leading byte offset); 16 elements of the contraction on is 2048 bytes on.
__device__ __forceinline__ uint64_t desc_swizzled(uint32_t addr, uint32_t leading) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(leading >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// Operand formats of the instruction descriptor (bits 7-9 and 10-12): 0 fp16, 1 bf16.
template <class T> __host__ __device__ constexpr uint32_t idesc_of(int n, bool a_mn, bool b_mn) {
  return tc::idesc(kRows, n, a_mn, b_mn) | (sizeof(T) == 2 && !__is_same(T, __half) ? (1u << 7) | (1u << 10) : 0u);
}

__device__ __forceinline__ void load32(uint32_t taddr, float v[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(r[k]);
}
__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// dz of eight values: part 0 high, then what is left; in place of dy (a), preact (b) and at c.
// kParts: 1 ReLU, 2 or 3 smooth; kScale: the second part times 2^11.  dz itself is added to sums where there are any.
template <class T, int kParts, bool kScale, bool kSums>
__device__ __forceinline__ void transform_chunk(unsigned char *a, unsigned char *b, unsigned char *c, int act, float *sums) {
  uint4 dy = *reinterpret_cast<const uint4 *>(a), z = *reinterpret_cast<const uint4 *>(b), third = make_uint4(0u, 0u, 0u, 0u);
  uint32_t *dw = &dy.x, *zw = &z.x, *tw = &third.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 d = widen2<T>(dw[i]), p = widen2<T>(zw[i]);
    if (kParts == 1) {
      const float2 v = make_float2(p.x > 0.f ? d.x : 0.f, p.y > 0.f ? d.y : 0.f);
      dw[i] = narrow2<T>(v.x, v.y);
      if (kSums) { sums[2 * i] += v.x; sums[2 * i + 1] += v.y; }
    } else {
      float2 v = make_float2(d.x * activate_grad(act, p.x), d.y * activate_grad(act, p.y));
      if (kSums) { sums[2 * i] += v.x; sums[2 * i + 1] += v.y; }
      dw[i] = narrow2<T>(v.x, v.y);
      float2 f = widen2<T>(dw[i]);
      v.x -= f.x; v.y -= f.y;
      zw[i] = kScale ? narrow2<T>(v.x * 2048.f, v.y * 2048.f) : narrow2<T>(v.x, v.y);
      if (kParts == 3) {
        f = widen2<T>(zw[i]);
        tw[i] = narrow2<T>(v.x - f.x, v.y - f.y);
      }
    }
  }
  *reinterpret_cast<uint4 *>(a) = dy;
  if (kParts >= 2) *reinterpret_cast<uint4 *>(b) = z;
  if (kParts == 3) *reinterpret_cast<uint4 *>(c) = third;
}

struct RowsArgs {
  CUtensorMap a, z, b, out, keep, residual;     // x or dy; preact (backward); W; y or dx; preact (forward); residual
  const float *bias;
  void *out_rows, *keep_rows;                   // y or dx, preact: for the columns behind the last multiple of 8
  int64_t ld_out, ld_keep;
  int rows;
  int out_cols, m_tiles, n_tiles, k_blocks, k;   // k: length of the contraction
  int bn;                                       // columns of a tile, at most 256
  uint32_t b_bytes;                             // of one step's weights
  int stages, resident, staging;                // staging: tiles per output on their way out, 1 or 2
  int act, has_keep, has_residual;
  uint32_t tmem_cols;
  unsigned long long *timeout;
};

struct RowsBarriers {
  uint64_t full[kMaxStages], ready[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], res_full[2], res_empty[2], weights, drained;
  uint32_t tmem, dead, ok, pad;
};

// kForward: B is W [out, in], K-major, and the epilogue has bias, activation, residual and kept pre-activation.  Else B is W
// [contraction, out], MN-major, A is dz in kParts parts (0: dy as it is).
template <class T, bool kForward, int kParts>
__global__ void __launch_bounds__(kParts ? 512 : 256, 1) k_dense_rows(const __grid_constant__ RowsArgs a) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char *smem = smem_raw + ((1024u - (tc::smem_addr(smem_raw) & 1023u)) & 1023u);
  constexpr uint32_t kStageA = kParts ? 2 * kTileBytes : kTileBytes;
  const uint32_t stage_bytes = kStageA + (a.resident ? 0u : a.b_bytes);
  unsigned char *stages = smem + (a.resident ? (uint32_t)a.k_blocks * a.b_bytes : 0u);
  unsigned char *out_tiles = stages + (uint32_t)a.stages * stage_bytes;
  unsigned char *keep_tiles = out_tiles + (uint32_t)a.staging * kTileBytes;
  unsigned char *res_tiles = keep_tiles + (a.has_keep ? (uint32_t)a.staging * kTileBytes : 0u);
  float *bias = reinterpret_cast<float *>(res_tiles + (a.has_residual ? (uint32_t)a.staging * kTileBytes : 0u));
  RowsBarriers &bars = *reinterpret_cast<RowsBarriers *>(bias + 256);
  volatile uint32_t *dead = &bars.dead;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [](const uint64_t &b) { return tc::smem_addr(&b); };

  if (threadIdx.x == 0) {
    for (int s = 0; s < a.stages; ++s) { tma::init(bar(bars.full[s]), 1); tma::init(bar(bars.ready[s]), kTransformThreads / 32); tma::init(bar(bars.empty[s]), 1); }
    for (int i = 0; i < 2; ++i) {
      tma::init(bar(bars.acc_full[i]), 1); tma::init(bar(bars.acc_empty[i]), 4);
      tma::init(bar(bars.res_full[i]), 1); tma::init(bar(bars.res_empty[i]), 1);
    }
    tma::init(bar(bars.weights), 1); tma::init(bar(bars.drained), 1);
    bars.dead = 0u;
    tc::fence_barrier_init();
  }
  if (warp == kWarpMma) tc::tmem_alloc(&bars.tmem, a.tmem_cols);
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = bars.tmem;
  dependency_wait();

  const int n_tile = blockIdx.x % a.n_tiles, n0 = n_tile * a.bn;
  const int m_first = blockIdx.x / a.n_tiles, m_step = gridDim.x / a.n_tiles;
  const uint32_t acc_cols = (uint32_t)(a.bn + 63) & ~63u;
  const int chunks = (min(a.bn, a.out_cols - n0) + 63) / 64;

  if (warp == kWarpLoad) {
    if (lane == 0) {
      auto load_weights = [&](uint32_t dst, int kb, uint32_t b) {
        if (kForward) tma::load(dst, &a.b, kb * kStep, n0, b);
        else for (int j = 0; j * 64 < a.bn; ++j) tma::load(dst + j * kBoxBytes, &a.b, n0 + j * 64, kb * kStep, b);
      };
      if (a.resident) {
        tma::expect(bar(bars.weights), (uint32_t)a.k_blocks * a.b_bytes);
        for (int kb = 0; kb < a.k_blocks; ++kb) load_weights(tc::smem_addr(smem) + kb * a.b_bytes, kb, bar(bars.weights));
      }
      uint32_t it = 0;
      bool ok = true;
      for (int m = m_first; ok && m < a.m_tiles; m += m_step)
        for (int kb = 0; kb < a.k_blocks; ++kb, ++it) {
          const uint32_t s = it % a.stages;
          if (!(ok = tma::wait(bar(bars.empty[s]), (it / a.stages & 1u) ^ 1u, dead))) break;
          const uint32_t dst = tc::smem_addr(stages) + s * stage_bytes, f = bar(bars.full[s]);
          tma::expect(f, stage_bytes);
          tma::load(dst, &a.a, kb * kStep, m * kRows, f);
          if (kParts) tma::load(dst + kTileBytes, &a.z, kb * kStep, m * kRows, f);
          if (!a.resident) load_weights(dst + kStageA, kb, f);
        }
      if (!ok) {                          // copies in flight land before the CTA leaves
        for (uint32_t k = it > (uint32_t)a.stages ? it - a.stages : 0u; k < it; ++k)
          for (int t = 0; t < (1 << 16) && !tma::try_wait(bar(bars.full[k % a.stages]), k / a.stages & 1u); ++t) {}
      }
      if (a.resident)
        for (int t = 0; t < (1 << 20) && !tma::try_wait(bar(bars.weights), 0u); ++t) {}
    }
  } else if (warp == kWarpMma) {
    if (lane == 0) {
      const uint32_t desc = idesc_of<T>((a.bn + 15) & ~15, false, !kForward);
      uint32_t it = 0, tile = 0;
      bool ok = !a.resident || m_first >= a.m_tiles || tma::wait(bar(bars.weights), 0u, dead);
      for (int m = m_first; ok && m < a.m_tiles; m += m_step, ++tile) {
        const uint32_t buf = tile & 1u;
        if (!(ok = tma::wait(bar(bars.acc_empty[buf]), (tile >> 1 & 1u) ^ 1u, dead))) break;
        tc::fence_after_sync();
        const uint32_t d = tmem + buf * acc_cols;
        for (int kb = 0; kb < a.k_blocks; ++kb, ++it) {
          const uint32_t s = it % a.stages;
          if (!(ok = tma::wait(kParts ? bar(bars.ready[s]) : bar(bars.full[s]), it / a.stages & 1u, dead))) break;
          tc::fence_after_sync();
          const uint32_t A = tc::smem_addr(stages) + s * stage_bytes;
          const uint32_t B = a.resident ? tc::smem_addr(smem) + kb * a.b_bytes : A + kStageA;
          const int steps = min(4, (a.k - kb * kStep + 15) / 16);
#pragma unroll
          for (int p = 0; p < (kParts == 2 ? 2 : 1); ++p)
            for (int ks = 0; ks < steps; ++ks)
              tc::mma(d, desc_swizzled(A + p * kTileBytes + ks * 32, 16), kForward ? desc_swizzled(B + ks * 32, 16) : desc_swizzled(B + ks * 2048, kBoxBytes),
                      (kb | p | ks) ? 1u : 0u, desc);
          tc::commit(bar(bars.empty[s]));
        }
        if (ok) tc::commit(bar(bars.acc_full[buf]));
      }
      // products in flight end before tensor memory is given back
      tc::commit(bar(bars.drained));
      for (int t = 0; t < (1 << 20) && !tma::try_wait(bar(bars.drained), 0u); ++t) {}
    }
  } else if (kForward && warp == kWarpResidual) {
    if (lane == 0 && a.has_residual) {
      uint32_t it = 0;
      bool ok = true;
      for (int m = m_first; ok && m < a.m_tiles; m += m_step)
        for (int c = 0; c < chunks; ++c, ++it) {
          const uint32_t s = it % a.staging;
          if (!(ok = tma::wait(bar(bars.res_empty[s]), (it / a.staging & 1u) ^ 1u, dead))) break;
          tma::expect(bar(bars.res_full[s]), kTileBytes);
          tma::load(tc::smem_addr(res_tiles) + s * kTileBytes, &a.residual, n0 + c * 64, m * kRows, bar(bars.res_full[s]));
        }
      if (!ok)
        for (uint32_t k = it > (uint32_t)a.staging ? it - a.staging : 0u; k < it; ++k)
          for (int t = 0; t < (1 << 16) && !tma::try_wait(bar(bars.res_full[k % a.staging]), k / a.staging & 1u); ++t) {}
    }
  } else if (warp >= kWarpEpilogue && warp < kWarpTransform) {
    const int tid = threadIdx.x - kWarpEpilogue * 32;              // = lane of tensor memory = row of the tile
    if (kForward)
      for (int c = tid; c < 256; c += 128) bias[c] = a.bias && c < a.bn && n0 + c < a.out_cols ? __ldg(a.bias + n0 + c) : 0.f;
    // A copy out of shared memory writes whole 16-byte chunks: the columns behind the last multiple of 8 go one by one.
    const int tail = a.out_cols & 7, whole = a.out_cols - tail;
    auto store_tail = [&](void *rows, int64_t ld, int m, const float *w) {
      const int row = m * kRows + tid;
      if (row >= a.rows) return;
      T *p = static_cast<T *>(rows) + (int64_t)row * ld + whole;
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < tail) p[i] = narrow<T>(w[i]);
    };
    uint32_t it = 0, tile = 0;
    bool ok = true;
    for (int m = m_first; ok && m < a.m_tiles; m += m_step, ++tile) {
      const uint32_t buf = tile & 1u;
      for (int c = 0; c < chunks; ++c, ++it) {
        const uint32_t s = it % a.staging;
        if (tid == 0) {
          bool all = c > 0 || tma::wait(bar(bars.acc_full[buf]), tile >> 1 & 1u, dead);
          if (kForward && a.has_residual) all = all && tma::wait(bar(bars.res_full[s]), it / a.staging & 1u, dead);
          if (a.staging == 2) tma::stores_read<1>(); else tma::stores_read<0>();
          bars.ok = all ? 1u : 0u;
        }
        named_sync(1, 128);
        if (!(ok = *(volatile uint32_t *)&bars.ok != 0u)) break;
        tc::fence_after_sync();
        unsigned char *out = out_tiles + s * kTileBytes + tid * tma::kRowBytes, *keep = keep_tiles + s * kTileBytes + tid * tma::kRowBytes;
        const unsigned char *res = res_tiles + s * kTileBytes + tid * tma::kRowBytes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float v[32];
          load32(tmem + buf * acc_cols + c * 64 + h * 32 + ((uint32_t)(tid & 96) << 16), v);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t at = (uint32_t)((h * 4 + q) ^ (tid & 7)) * 16u;
            float *w = v + q * 8;
            if (kForward) {
              const float4 b0 = *reinterpret_cast<const float4 *>(bias + c * 64 + h * 32 + q * 8), b1 = *reinterpret_cast<const float4 *>(bias + c * 64 + h * 32 + q * 8 + 4);
              w[0] += b0.x; w[1] += b0.y; w[2] += b0.z; w[3] += b0.w;
              w[4] += b1.x; w[5] += b1.y; w[6] += b1.z; w[7] += b1.w;
              if (a.has_keep) {
                *reinterpret_cast<uint4 *>(keep + at) = pack<T>(w);
                if (tail && n0 + c * 64 + h * 32 + q * 8 == whole) store_tail(a.keep_rows, a.ld_keep, m, w);
              }
#pragma unroll
              for (int i = 0; i < 8; ++i) w[i] = activate(a.act, w[i]);
              if (a.has_residual) {
                float r[8];
                unpack<T>(*reinterpret_cast<const uint4 *>(res + at), r);
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] += r[i];
              }
            }
            *reinterpret_cast<uint4 *>(out + at) = pack<T>(w);
            if (tail && n0 + c * 64 + h * 32 + q * 8 == whole) store_tail(a.out_rows, a.ld_out, m, w);
          }
        }
        tc::fence_before_sync();
        tc::fence_generic_writes();
        if (c == chunks - 1 && lane == 0) tma::arrive(bar(bars.acc_empty[buf]));
        named_sync(1, 128);
        if (tid == 0) {
          const bool any = n0 + c * 64 < whole;
          if (any) tma::store(&a.out, n0 + c * 64, m * kRows, tc::smem_addr(out_tiles) + s * kTileBytes);
          if (kForward && a.has_keep && any) tma::store(&a.keep, n0 + c * 64, m * kRows, tc::smem_addr(keep_tiles) + s * kTileBytes);
          tma::store_commit();
          if (kForward && a.has_residual) tma::arrive(bar(bars.res_empty[s]));
        }
      }
    }
    if (tid == 0) tma::stores_done();
  } else if (kParts && warp >= kWarpTransform) {
    const int t = threadIdx.x - kWarpTransform * 32;
    uint32_t it = 0;
    bool ok = true;
    for (int m = m_first; ok && m < a.m_tiles; m += m_step)
      for (int kb = 0; kb < a.k_blocks; ++kb, ++it) {
        const uint32_t s = it % a.stages;
        if (!(ok = __all_sync(0xffffffffu, tma::wait(bar(bars.full[s]), it / a.stages & 1u, dead)))) break;
        unsigned char *A = stages + s * stage_bytes;
#pragma unroll
        for (int u = 0; u < (int)(kTileBytes / 16 / kTransformThreads); ++u) {
          const uint32_t at = (uint32_t)(u * kTransformThreads + t) * 16u;
          transform_chunk<T, kParts, false, false>(A + at, A + kTileBytes + at, nullptr, a.act, nullptr);
        }
        tc::fence_generic_writes();
        __syncwarp();
        if (lane == 0) tma::arrive(bar(bars.ready[s]));
      }
  }
  __syncwarp();
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  if (threadIdx.x == 0 && bars.dead) *a.timeout = 1ull;
  if (warp == kWarpMma) tc::tmem_free(tmem, a.tmem_cols);
}

// ---- dW and db ---------------------------------------------------------------------------------------------------
struct WeightsArgs {
  CUtensorMap dy, z, x;
  int n, k, n_tiles, k_tiles, splits, row_blocks;
  int bk;                         // columns of x of a tile, at most 256
  int stages, act, want_db;
  int ld;                         // row length of the partial sums
  float *partials, *db_partials;  // [splits, n, ld], [splits, n]
  uint32_t tmem_cols;
  unsigned long long *timeout;
};
constexpr int kFlush = 8;                       // steps of 64 rows after which an accumulator is emptied
struct WeightsBarriers {
  uint64_t full[kMaxStages], ready[kMaxStages], empty[kMaxStages], sum_full[2], sum_empty[2], done;
  uint32_t tmem, dead, pad[2];
};

// kParts: 0 dy is dz; 1 ReLU; 2 and 3 smooth activations in so many parts.  kScale: what is left lies 2^11 higher.
//
// The tensor core cuts off what an addition leaves below the accumulator's last bit, so over thousands of additions the sums
// shrink: 1M rows in 74 splits were 9e-5 off.  So the accumulator of dz, or of its high part, is emptied every 8 steps, after
// 32 additions, into fp32 registers of the eight worker warps, which round to nearest (two accumulators in turn where there
// is one part: 4e-7 off).  The other parts have an accumulator of their own, which loses as much of 2^-8 as much.
template <class T, int kParts, bool kScale>
__global__ void __launch_bounds__(384, 1) k_dense_weights(const __grid_constant__ WeightsArgs a) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char *smem = smem_raw + ((1024u - (tc::smem_addr(smem_raw) & 1023u)) & 1023u);
  constexpr bool kLow = kParts >= 2;
  constexpr uint32_t kStageA = (kParts == 3 ? 3 : kParts ? 2 : 1) * 2 * kBoxBytes;
  const int x_boxes = (a.bk + 63) / 64;
  const uint32_t stage_bytes = kStageA + x_boxes * kBoxBytes;
  float *sums = reinterpret_cast<float *>(smem + a.stages * stage_bytes);  // [16, 128]
  WeightsBarriers &bars = *reinterpret_cast<WeightsBarriers *>(sums + 16 * 128);
  volatile uint32_t *dead = &bars.dead;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [](const uint64_t &b) { return tc::smem_addr(&b); };

  if (threadIdx.x == 0) {
    for (int s = 0; s < a.stages; ++s) { tma::init(bar(bars.full[s]), 1); tma::init(bar(bars.ready[s]), kWorkerWarps); tma::init(bar(bars.empty[s]), 1); }
    for (int i = 0; i < 2; ++i) { tma::init(bar(bars.sum_full[i]), 1); tma::init(bar(bars.sum_empty[i]), kWorkerWarps); }
    tma::init(bar(bars.done), 1);
    bars.dead = 0u;
    tc::fence_barrier_init();
  }
  if (warp == kWarpMma) tc::tmem_alloc(&bars.tmem, a.tmem_cols);
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = bars.tmem;
  dependency_wait();

  const int tiles = a.n_tiles * a.k_tiles, tile = blockIdx.x % tiles, split = blockIdx.x / tiles;
  const int n0 = tile / a.k_tiles * kRows, k0 = tile % a.k_tiles * a.bk;
  const int first = (int)((int64_t)a.row_blocks * split / a.splits), count = (int)((int64_t)a.row_blocks * (split + 1) / a.splits) - first;
  const int dz_boxes = a.n - n0 > 64 ? 2 : 1, cols = min(a.bk, a.k - k0), boxes = (cols + 63) / 64;
  const bool db = a.want_db && k0 == 0, touched = kParts || db;      // the workers look at every step
  const uint32_t second = a.bk > 128 ? 256u : 128u;                  // columns of the second accumulator

  if (warp < kWarpWorker) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == kWarpLoad && lane == 0) {
      int it = 0;
      bool ok = true;
      for (; it < count; ++it) {
        const int s = it % a.stages, r = first + it;
        if (!(ok = tma::wait(bar(bars.empty[s]), (it / a.stages & 1) ^ 1, dead))) break;
        const uint32_t dst = tc::smem_addr(smem) + s * stage_bytes, f = bar(bars.full[s]);
        tma::expect(f, (uint32_t)(dz_boxes * (kParts ? 2 : 1) + boxes) * kBoxBytes);
        for (int j = 0; j < dz_boxes; ++j) {
          tma::load(dst + j * kBoxBytes, &a.dy, n0 + j * 64, r * kStep, f);
          if (kParts) tma::load(dst + (2 + j) * kBoxBytes, &a.z, n0 + j * 64, r * kStep, f);
        }
        for (int j = 0; j < boxes; ++j) tma::load(dst + kStageA + j * kBoxBytes, &a.x, k0 + j * 64, r * kStep, f);
      }
      if (!ok)
        for (int k = it > a.stages ? it - a.stages : 0; k < it; ++k)
          for (int t = 0; t < (1 << 16) && !tma::try_wait(bar(bars.full[k % a.stages]), k / a.stages & 1); ++t) {}
    } else if (warp == kWarpMma && lane == 0) {
      const uint32_t desc = idesc_of<T>((cols + 15) & ~15, true, true);
      for (int it = 0; it < count; ++it) {
        const int s = it % a.stages, group = it / kFlush;
        // accumulator of this group: one of two in turn, or the first one always
        const int buf = kLow ? 0 : group & 1, use = kLow ? group : group >> 1;
        if (!tma::wait(touched ? bar(bars.ready[s]) : bar(bars.full[s]), it / a.stages & 1, dead)) break;
        const uint32_t A = tc::smem_addr(smem) + s * stage_bytes, B = A + kStageA;
        auto part = [&](int p, uint32_t d, bool add) {
#pragma unroll
          for (int ks = 0; ks < 4; ++ks)
            tc::mma(d, desc_swizzled(A + p * 2 * kBoxBytes + ks * 2048, kBoxBytes), desc_swizzled(B + ks * 2048, kBoxBytes), add || ks ? 1u : 0u, desc);
        };
        tc::fence_after_sync();
        if (kLow) part(1, tmem + second, it > 0);
        if (kParts == 3) part(2, tmem + second, true);
        if (it % kFlush == 0 && !tma::wait(bar(bars.sum_empty[buf]), (use & 1) ^ 1, dead)) break;
        tc::fence_after_sync();
        part(0, tmem + buf * second, it % kFlush > 0);
        tc::commit(bar(bars.empty[s]));
        if (it % kFlush == kFlush - 1 || it == count - 1) tc::commit(bar(bars.sum_full[buf]));
      }
      // products in flight end before tensor memory is given back
      tc::commit(bar(bars.done));
      for (int t = 0; t < (1 << 20) && !tma::try_wait(bar(bars.done), 0u); ++t) {}
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    // As a holder of sums: rows (lanes of tensor memory) 32 (warp % 4) + lane, columns from 128 * half on.  As a maker of dz:
    // the eight columns 16 bytes chunk & 7 of box chunk >> 3 of rows t / 16, 16 further, ...: always the same columns.
    const int t = threadIdx.x - kWarpWorker * 32, half = t >> 7, n = n0 + (t & 127);
    const uint32_t lanes = tmem + ((uint32_t)(t & 96) << 16) + half * 128;
    const int chunk = (t & 7) | (t >> 4 & 8), row0 = (t >> 3) & 15;
    float mine[8], acc[128];
#pragma unroll
    for (int i = 0; i < 8; ++i) mine[i] = 0.f;
#pragma unroll
    for (int i = 0; i < 128; ++i) acc[i] = 0.f;
    bool ok = true;
    auto flush = [&](int group) {
      const int buf = kLow ? 0 : group & 1, use = kLow ? group : group >> 1;
      ok = __all_sync(0xffffffffu, tma::wait(bar(bars.sum_full[buf]), use & 1, dead));
      if (!ok) return;
      tc::fence_after_sync();
#pragma unroll
      for (int c = 0; c < 128; c += 32)
        if (half * 128 + c < cols) {
          float v[32];
          load32(lanes + buf * second + c, v);
#pragma unroll
          for (int i = 0; i < 32; ++i) acc[c + i] += v[i];
        }
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tma::arrive(bar(bars.sum_empty[buf]));
    };
    // an accumulator is emptied a step after its last one was made ready: the products have time
    for (int it = 0; ok && it < count; ++it) {
      if (touched) {
        const int s = it % a.stages;
        if (!(ok = __all_sync(0xffffffffu, tma::wait(bar(bars.full[s]), it / a.stages & 1, dead)))) break;
        unsigned char *A = smem + s * stage_bytes + (chunk >> 3) * kBoxBytes;
        if ((chunk >> 3) < dz_boxes) {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int row = row0 + 16 * u;
            const uint32_t at = (uint32_t)row * tma::kRowBytes + (uint32_t)((chunk & 7) ^ (row & 7)) * 16u;
            if constexpr (kParts > 0) {
              transform_chunk<T, kParts, kScale, true>(A + at, A + 2 * kBoxBytes + at, A + 4 * kBoxBytes + at, a.act, mine);
            } else {
              float v[8];
              unpack<T>(*reinterpret_cast<const uint4 *>(A + at), v);
#pragma unroll
              for (int i = 0; i < 8; ++i) mine[i] += v[i];
            }
          }
        }
        if (kParts) tc::fence_generic_writes();
        __syncwarp();
        if (lane == 0) tma::arrive(bar(bars.ready[s]));
      }
      if (it % kFlush == 0 && it > 0) flush(it / kFlush - 1);
    }
    if (ok && count > 0) flush((count - 1) / kFlush);
    if (ok && n < a.n) {
      float *out = a.partials + ((size_t)split * a.n + n) * a.ld + k0 + half * 128;
#pragma unroll
      for (int c = 0; c < 128; c += 32)
        if (half * 128 + c < cols) {
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            if (half * 128 + c + i < cols) *reinterpret_cast<float4 *>(out + c + i) = make_float4(acc[c + i], acc[c + i + 1], acc[c + i + 2], acc[c + i + 3]);
        }
    }
    if constexpr (kLow) {
      // (all products have completed with the last group's: the high part's are issued last)
      if (__any_sync(0xffffffffu, ok && count > 0 && n < a.n)) {
        float *out = a.partials + ((size_t)split * a.n + n) * a.ld + k0 + half * 128;
#pragma unroll
        for (int c = 0; c < 128; c += 32)
          if (half * 128 + c < cols) {
            float v[32];
            load32(lanes + second + c, v);
            if (n < a.n) {
#pragma unroll
              for (int i = 0; i < 32; i += 4)
                if (half * 128 + c + i < cols) {
                  float4 w = *reinterpret_cast<const float4 *>(out + c + i);
                  constexpr float k = kScale ? 1.f / 2048.f : 1.f;
                  w.x = fmaf(v[i], k, w.x); w.y = fmaf(v[i + 1], k, w.y); w.z = fmaf(v[i + 2], k, w.z); w.w = fmaf(v[i + 3], k, w.w);
                  *reinterpret_cast<float4 *>(out + c + i) = w;
                }
            }
          }
      }
    }
    if (db) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sums[row0 * 128 + chunk * 8 + i] = mine[i];
      named_sync(2, kWorkerWarps * 32);
      if (t < 128 && n < a.n) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v += sums[i * 128 + t];
        a.db_partials[(size_t)split * a.n + n] = v;
      }
    }
  }
  __syncwarp();
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  if (threadIdx.x == 0 && bars.dead) *a.timeout = 1ull;
  if (warp == kWarpMma) tc::tmem_free(tmem, a.tmem_cols);
}

// dW [n, k] and db [n] from the splits' sums, added in their order.
__global__ void __launch_bounds__(256) k_dense_sums(const float *partials, const float *db_partials, int splits, int n, int k, int ld, float *dw, float *db) {
  dependency_wait();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, count = (int64_t)n * ld, stride = count;
  if (i < count) {
    const int row = (int)(i / ld), col = (int)(i % ld);
    if (col < k) {
      double s = 0.0;
      for (int p = 0; p < splits; ++p) s += (double)__ldcs(partials + p * stride + i);
      dw[(int64_t)row * k + col] = (float)s;
    }
  } else if (db && i - count < n) {
    double s = 0.0;
    for (int p = 0; p < splits; ++p) s += (double)__ldcs(db_partials + (int64_t)p * n + (i - count));
    db[i - count] = (float)s;
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
uint32_t tmem_columns(uint32_t n) {
  uint32_t c = 32;
  while (c < n) c *= 2;
  return c;
}

// The shape of a call of k_dense_rows: tile width, weights resident or not, pipeline depth.
bool plan_rows(RowsArgs &a, bool forward, bool transform, int num_sms, uint32_t &smem, int &grid) {
  const uint32_t stage_a = transform ? 2 * kTileBytes : kTileBytes;
  const int outputs = 1 + a.has_keep + a.has_residual;
  auto shape = [&](int bn) {
    a.bn = bn;
    a.n_tiles = ceil_div(a.out_cols, bn);
    a.b_bytes = forward ? (uint32_t)bn * tma::kRowBytes : (uint32_t)ceil_div(bn, 64) * kBoxBytes;
    const uint32_t fixed = 1024 + 1024 + sizeof(RowsBarriers);
    for (int resident = 1; resident >= 0; --resident)
      for (int want = 3; want >= 2; --want)             // rather a deeper pipeline than a second tile on its way out
      for (int staging = 2; staging >= 1; --staging) {
        const uint32_t used = fixed + (uint32_t)(outputs * staging) * kTileBytes + (resident ? (uint32_t)a.k_blocks * a.b_bytes : 0u);
        const uint32_t stage = stage_a + (resident ? 0u : a.b_bytes);
        if (used + want * stage > kSmemMost) continue;
        int stages = (int)((kSmemMost - used) / stage);
        if (stages > kMaxStages) stages = kMaxStages;
        a.resident = resident; a.staging = staging; a.stages = stages;
        smem = used + (uint32_t)stages * stage;
        return true;
      }
    return false;
  };
  // Wide tiles read the rows once; narrower ones where there are fewer tiles than SMs.  Results leave in boxes of 64 columns, so tiles
  // beside one another are a multiple of that.
  int bn = a.out_cols <= 256 ? (a.out_cols + 15) / 16 * 16 : 256;
  while (bn > 64 && (int64_t)a.m_tiles * ceil_div(a.out_cols, bn) * 2 <= num_sms) bn = (bn / 2 + 63) / 64 * 64;
  if (!forward) bn = (bn + 63) / 64 * 64;
  if (!shape(bn)) return false;
  a.tmem_cols = tmem_columns(2u * (((uint32_t)bn + 63u) & ~63u));
  int groups = num_sms / a.n_tiles;
  if (groups < 1) groups = 1;
  if (groups > a.m_tiles) groups = a.m_tiles;
  grid = groups * a.n_tiles;
  return true;
}

template <class T, bool kForward, int kParts>
void run_rows(const RowsArgs &a, uint32_t smem, int grid, cudaStream_t st) {
  cudaFuncSetAttribute(k_dense_rows<T, kForward, kParts>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  launch_chained(k_dense_rows<T, kForward, kParts>, grid, kParts ? 512 : 256, smem, st, a);
}

template <class T>
int fwd(const DenseArgs &d, int num_sms, cudaStream_t st) {
  RowsArgs a;
  a.bias = d.bias; a.out_cols = d.out; a.k = d.in; a.k_blocks = ceil_div(d.in, kStep); a.m_tiles = ceil_div(d.rows, kRows);
  a.rows = (int)d.rows; a.out_rows = d.y; a.ld_out = d.ld_y; a.keep_rows = d.preact; a.ld_keep = d.ld_preact;
  a.act = d.act; a.has_keep = d.preact != nullptr; a.has_residual = d.residual != nullptr; a.timeout = d.timeout;
  uint32_t smem;
  int grid;
  if (!plan_rows(a, true, false, num_sms, smem, grid)) return -1;
  if (!tma::make_map(&a.a, d.dtype, d.x, d.rows, d.in, d.ld_x, kRows) || !tma::make_map(&a.b, d.dtype, d.w, d.out, d.in, d.ld_w, a.bn) ||
      (d.out >= 8 && !tma::make_map(&a.out, d.dtype, d.y, d.rows, d.out & ~7, d.ld_y, kRows)) ||
      (d.out >= 8 && a.has_keep && !tma::make_map(&a.keep, d.dtype, d.preact, d.rows, d.out & ~7, d.ld_preact, kRows)) ||
      (a.has_residual && !tma::make_map(&a.residual, d.dtype, d.residual, d.rows, d.out, d.ld_residual, kRows)))
    return -1;
  run_rows<T, true, 0>(a, smem, grid, st);
  return 1;
}

// Rows are split so that every SM has a tile; a split has at least 512 rows.  The workspace's size is asked for without a
// context: it is for kSplitSms SMs, and no more are used.
constexpr int kSplitSms = 160;
struct WeightsPlan { int n_tiles, k_tiles, bk, splits, ld; };
WeightsPlan plan_weights(int64_t rows, int in, int out, int num_sms) {
  WeightsPlan p;
  p.bk = in < 256 ? (in + 15) / 16 * 16 : 256;
  p.n_tiles = ceil_div(out, kRows);
  p.k_tiles = ceil_div(in, p.bk);
  int splits = num_sms / (p.n_tiles * p.k_tiles);
  const int most = ceil_div(rows, 512);
  if (splits > most) splits = most;
  p.splits = splits < 1 ? 1 : splits;
  p.ld = (in + 3) / 4 * 4;
  return p;
}

template <class T, int kParts, bool kScale>
void run_weights(WeightsArgs &a, cudaStream_t st) {
  const uint32_t stage = ((kParts == 3 ? 3u : kParts ? 2u : 1u) * 2u + (uint32_t)ceil_div(a.bk, 64)) * kBoxBytes;
  const uint32_t fixed = 1024 + 16 * 128 * 4 + sizeof(WeightsBarriers);
  a.stages = (int)((kSmemMost - fixed) / stage);
  if (a.stages > kMaxStages) a.stages = kMaxStages;
  const uint32_t smem = fixed + a.stages * stage;
  a.tmem_cols = a.bk > 128 ? 512u : 256u;
  cudaFuncSetAttribute(k_dense_weights<T, kParts, kScale>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  launch_chained(k_dense_weights<T, kParts, kScale>, a.n_tiles * a.k_tiles * a.splits, 384, smem, st, a);
}

template <class T>
int bwd(const DenseArgs &d, int num_sms, cudaStream_t st) {
  constexpr bool kHalf = __is_same(T, __half);
  const bool plain = d.act == GS_DENSE_NONE, relu = d.act == GS_DENSE_RELU;
  int launches = 0;
  if (d.dx) {
    RowsArgs a;
    a.bias = nullptr; a.out_cols = d.in; a.k = d.out; a.k_blocks = ceil_div(d.out, kStep); a.m_tiles = ceil_div(d.rows, kRows);
    a.rows = (int)d.rows; a.out_rows = d.dx; a.ld_out = d.ld_dx; a.keep_rows = nullptr; a.ld_keep = 0;
    a.act = d.act; a.has_keep = a.has_residual = 0; a.timeout = d.timeout;
    uint32_t smem;
    int grid;
    if (!plan_rows(a, false, !plain, num_sms, smem, grid)) return -1;
    if (!tma::make_map(&a.a, d.dtype, d.dy, d.rows, d.out, d.ld_dy, kRows) || !tma::make_map(&a.b, d.dtype, d.w, d.out, d.in, d.ld_w, kStep) ||
        (d.in >= 8 && !tma::make_map(&a.out, d.dtype, d.dx, d.rows, d.in & ~7, d.ld_dx, kRows)) ||
        (!plain && !tma::make_map(&a.z, d.dtype, d.preact_in, d.rows, d.out, d.ld_preact, kRows)))
      return -1;
    if (plain) run_rows<T, false, 0>(a, smem, grid, st);
    else if (relu) run_rows<T, false, 1>(a, smem, grid, st);
    else run_rows<T, false, 2>(a, smem, grid, st);
    ++launches;
  }
  if (d.dw) {
    const WeightsPlan p = plan_weights(d.rows, d.in, d.out, num_sms < kSplitSms ? num_sms : kSplitSms);
    WeightsArgs a;
    a.n = d.out; a.k = d.in; a.n_tiles = p.n_tiles; a.k_tiles = p.k_tiles; a.splits = p.splits; a.bk = p.bk; a.ld = p.ld;
    a.row_blocks = ceil_div(d.rows, kStep); a.act = d.act; a.want_db = d.db != nullptr; a.timeout = d.timeout;
    a.partials = d.partials;
    a.db_partials = d.partials + (size_t)p.splits * d.out * p.ld;
    if (!tma::make_map(&a.dy, d.dtype, d.dy, d.rows, d.out, d.ld_dy, kStep) || !tma::make_map(&a.x, d.dtype, d.x, d.rows, d.in, d.ld_x, kStep) ||
        (!plain && !tma::make_map(&a.z, d.dtype, d.preact_in, d.rows, d.out, d.ld_preact, kStep)))
      return -1;
    if (plain) run_weights<T, 0, false>(a, st);
    else if (relu) run_weights<T, 1, false>(a, st);
    else if constexpr (kHalf) run_weights<T, 2, true>(a, st);
    else run_weights<T, 3, false>(a, st);
    launch_chained(k_dense_sums, ceil_div((int64_t)d.out * p.ld + (d.db ? d.out : 0), 256), 256, 0, st, (const float *)a.partials,
                   (const float *)a.db_partials, p.splits, d.out, d.in, p.ld, d.dw, d.db);
    launches += 2;
  }
  return launches;
}

}  // namespace

size_t dense_partials(int64_t rows, int in, int out) {
  const WeightsPlan p = plan_weights(rows, in, out, kSplitSms);
  return (size_t)p.splits * out * (p.ld + 1);
}
int launch_dense_fwd(const DenseArgs &a, int num_sms, cudaStream_t st) { return a.dtype == GS_TYPE_F16 ? fwd<__half>(a, num_sms, st) : fwd<__nv_bfloat16>(a, num_sms, st); }
int launch_dense_bwd(const DenseArgs &a, int num_sms, cudaStream_t st) { return a.dtype == GS_TYPE_F16 ? bwd<__half>(a, num_sms, st) : bwd<__nv_bfloat16>(a, num_sms, st); }

}  // namespace gs
