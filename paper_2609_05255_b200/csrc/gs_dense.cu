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
// In fp16 what is left is scaled by 2^11 (it would fall below fp16's range: unscaled, dx lost all but 11 bits of gradients below 2^-13) and
// summed in an accumulator of its own.
// Without activation, and with ReLU, dz is dy or 0: exact as it is.
//
// Waits are bounded (tma::wait): one that runs out sets *timeout, and the CTA leaves without its results.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

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
constexpr int kMaxStages = 12;
constexpr uint32_t kSmemMost = 232448;        // 227 KB

enum { kWarpLoad = 0, kWarpMma = 1, kWarpResidual = 2, kWarpEpilogue = 4 };
constexpr int kTransformThreads = 256;
enum { kWarpWorker = 4, kWorkerWarps = 8 };   // of k_dense_weights, behind the warps that load and issue

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// logistic(x) of two values, from -log2(e) x
__device__ __forceinline__ float2 logistic2(float2 t) {
  t = add2(make_float2(ex2_approx(t.x), ex2_approx(t.y)), both(1.f));
  return make_float2(rcp_approx(t.x), rcp_approx(t.y));
}
constexpr float kMinusLog2e = -1.4426950408889634f;
// gelu(z) = z logistic(u), u = 2 sqrt(2 / pi) (z + 0.044715 z^3): the tanh form.  -log2(e) u:
__device__ __forceinline__ float2 gelu_arg2(float2 z, float2 zz) {
  return mul2(z, fma2(zz, both(0.07135481627159806f * kMinusLog2e), both(1.5957691216057308f * kMinusLog2e)));
}
template <int kAct>
__device__ __forceinline__ void activate8(float2 z[4]) {
  if constexpr (kAct == GS_DENSE_RELU) {
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = make_float2(z[i].x < 0.f ? 0.f : z[i].x, z[i].y < 0.f ? 0.f : z[i].y);      // (a NaN stays)
  } else if constexpr (kAct == GS_DENSE_SILU) {
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = mul2(z[i], logistic2(mul2(z[i], both(kMinusLog2e))));
  } else if constexpr (kAct == GS_DENSE_GELU) {
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = mul2(z[i], logistic2(gelu_arg2(z[i], mul2(z[i], z[i]))));
  }
}
// act' of the smooth ones: p + z p (1 - p) u', 1 - p by one fused operation.  p or 1 - p is 0 before a product overflows, but for z^2 of
// gelu in bf16 (kWide), which is held below 1e30; a NaN stays one.
template <int kAct, bool kWide>
__device__ __forceinline__ void activate_grad8(float2 z[4]) {
  if constexpr (kAct == GS_DENSE_SILU) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = logistic2(mul2(z[i], both(kMinusLog2e)));
      z[i] = fma2(mul2(z[i], p), fma2(p, both(-1.f), both(1.f)), p);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float2 zz = mul2(z[i], z[i]);
      if (kWide) zz = make_float2(fminf(zz.x, 1e30f), fminf(zz.y, 1e30f));
      const float2 p = logistic2(gelu_arg2(z[i], zz));
      const float2 slope = fma2(zz, both(0.21406444881479418f), both(1.5957691216057308f));
      z[i] = fma2(mul2(mul2(z[i], p), fma2(p, both(-1.f), both(1.f))), slope, p);
    }
  }
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
template <class T, int kAct, int kParts, bool kScale, bool kSums>
__device__ __forceinline__ void transform_chunk(unsigned char *a, unsigned char *b, unsigned char *c, uint4 dy, uint4 z, float2 *sums) {
  uint4 third;
  uint32_t *dw = &dy.x, *zw = &z.x, *tw = &third.x;
  float2 g[4];
  unpack<T>(z, &g[0].x);
  if constexpr (kParts > 1) activate_grad8<kAct, !__is_same(T, __half)>(g);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 d = widen2<T>(dw[i]);
    float2 v = kParts == 1 ? make_float2(g[i].x > 0.f ? d.x : 0.f, g[i].y > 0.f ? d.y : 0.f) : mul2(d, g[i]);
    if (kSums) sums[i] = add2(sums[i], v);
    dw[i] = narrow2<T>(v.x, v.y);
    if (kParts >= 2) {
      v = fma2(widen2<T>(dw[i]), both(-1.f), v);
      if (kScale) v = mul2(v, both(2048.f));
      zw[i] = narrow2<T>(v.x, v.y);
    }
    if (kParts == 3) {
      v = fma2(widen2<T>(zw[i]), both(-1.f), v);
      tw[i] = narrow2<T>(v.x, v.y);
    }
  }
  *reinterpret_cast<uint4 *>(a) = dy;
  if (kParts >= 2) *reinterpret_cast<uint4 *>(b) = z;
  if (kParts == 3) *reinterpret_cast<uint4 *>(c) = third;
}
__device__ __forceinline__ uint4 shared16(const unsigned char *p) { return *reinterpret_cast<const uint4 *>(p); }

// A place in a ring of stages and the parity of the passes over it, moved on without divisions: what one thread does for a step
// (wait, descriptors, four MMAs, commit) is a chain of dependent instructions, and at 650 cycles a step it was the bound (20 011
// rows of 1024 to 1024 in 56 us instead of 48).
struct Ring {
  uint32_t s = 0, parity = 0;
  __device__ __forceinline__ void next(uint32_t stages) {
    if (++s == stages) { s = 0; parity ^= 1u; }
  }
};

// Pairs: the two CTAs of a cluster work on two row tiles with one MMA of 256 rows, which the first of them issues; each holds its own
// rows and half of the weights, and its own rows' accumulator.  Barriers that the first one's MMA thread waits on get arrivals of both, its
// commits arrive at both.
namespace pair {
__device__ __forceinline__ uint32_t rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void sync() { asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory"); }
// At the first CTA's barrier of the same place.  (Not as a release at cluster scope, which takes 1 us a step: what the arrival tells
// of is read by the tensor core of the SM that wrote it, behind the writers' fence to the async proxy.)
__device__ __forceinline__ void arrive_first(uint32_t bar) {
  asm volatile("{\n\t.reg .b32 remote;\n\tmapa.shared::cluster.u32 remote, %0, 0;\n\tmbarrier.arrive.shared::cluster.b64 _, [remote];\n\t}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t accumulate, uint32_t desc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(desc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tmem_alloc(uint32_t *slot, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_addr(slot)), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
}
}  // namespace pair

struct RowsArgs {
  CUtensorMap a, z, b, out, keep, residual;     // x or dy; preact (backward); W; y or dx; preact (forward); residual
  const float *bias;
  void *out_rows, *keep_rows;                   // y or dx, preact: for the columns behind the last multiple of 8
  int64_t ld_out, ld_keep;
  int rows;
  int out_cols, m_tiles, n_tiles, k_blocks, k;   // k: length of the contraction
  int bn;                                       // columns of a tile, at most 256
  uint32_t b_bytes;                             // of one step's weights
  int stages, resident;
  int out_slots, keep_slots;                    // tiles of y (where the residual arrives) and preact on their way out: 2 or 4
  int has_keep, has_residual;
  int accumulators;                             // that tiles take in turn: 2, or 1 where the two parts' fill tensor memory
  uint32_t tmem_cols;
  unsigned long long *timeout;
};

struct RowsBarriers {
  uint64_t full[kMaxStages], ready[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], res_full[4], res_empty[4], weights, weights_both, drained;
  uint32_t tmem, dead, ok[2];
};

// Warps that take tiles out: two groups, which take chunks of 64 columns in turn, so that one computes while the other waits at its
// barriers.  In the forward, whose activation is the work, a group has eight warps, two for each 32 lanes of tensor memory.
// (One group of four: 943 us instead of 507, and 319 with the residual landing where y leaves, for 1M rows of 256 to 256 in bf16
// with SiLU, residual and kept pre-activation.)
template <bool kForward> constexpr int kGroupWarps = kForward ? 8 : 4;
template <bool kForward, int kParts> constexpr int kRowsThreads = 32 * (kWarpEpilogue + 2 * kGroupWarps<kForward>) + (kParts ? kTransformThreads : 0);

// kForward: B is W [out, in], K-major, and the epilogue has bias, activation, residual and kept pre-activation.  Else B is W
// [contraction, out], MN-major, A is dz in kParts parts (0: dy as it is).  (The activation is the kernel's: chosen inside, between
// two unrolled bodies, it kept the values from overlapping.)
// In fp16 the second part lies 2^11 higher, in the accumulator behind the first one's.
template <bool kForward, int kAct> constexpr int kRowsParts = kForward || kAct == GS_DENSE_NONE ? 0 : kAct == GS_DENSE_RELU ? 1 : 2;
template <class T, bool kForward, int kAct, bool kPair>
__global__ void __launch_bounds__((kRowsThreads<kForward, kRowsParts<kForward, kAct>>), 1) k_dense_rows(const __grid_constant__ RowsArgs a) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char *smem = smem_raw + ((1024u - (tc::smem_addr(smem_raw) & 1023u)) & 1023u);
  constexpr int kParts = kRowsParts<kForward, kAct>;
  constexpr bool kScale = kParts == 2 && __is_same(T, __half);
  static_assert(!kPair || kParts > 0, "pairs make dz");
  constexpr uint32_t kStageA = kParts ? 2 * kTileBytes : kTileBytes;
  const uint32_t stage_bytes = kStageA + (a.resident ? 0u : a.b_bytes);
  unsigned char *stages = smem + (a.resident ? (uint32_t)a.k_blocks * a.b_bytes : 0u);
  unsigned char *out_tiles = stages + (uint32_t)a.stages * stage_bytes;
  unsigned char *keep_tiles = out_tiles + (uint32_t)a.out_slots * kTileBytes;
  float *bias = reinterpret_cast<float *>(keep_tiles + (uint32_t)a.keep_slots * kTileBytes);
  RowsBarriers &bars = *reinterpret_cast<RowsBarriers *>(bias + 256);
  volatile uint32_t *dead = &bars.dead;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kGroup = kGroupWarps<kForward>, kWarpTransform = kWarpEpilogue + 2 * kGroup;
  auto bar = [](const uint64_t &b) { return tc::smem_addr(&b); };
  const uint32_t rank = kPair ? pair::rank() : 0u;
  constexpr int kCtas = kPair ? 2 : 1;
  const int worker = blockIdx.x / kCtas, workers = gridDim.x / kCtas;
  const int n_tile = worker % a.n_tiles, n0 = n_tile * a.bn, b0 = n0 + (int)rank * (a.bn / 2);     // b0: this CTA's share of the weights
  const int b_cols = a.bn / kCtas;
  const int m_first = worker / a.n_tiles * kCtas + (int)rank, m_step = workers / a.n_tiles * kCtas;
  const int m_end = (a.m_tiles + kCtas - 1) / kCtas * kCtas;      // (a tile behind the last one reads zeros and writes nothing)
  const uint32_t acc_cols = (uint32_t)(a.bn + 63) & ~63u, acc_stride = kScale ? 2 * acc_cols : acc_cols;
  // the accumulator of this CTA's tile-th tile, and its pass over it
  auto acc_of = [&](uint32_t tile) { return kScale && a.accumulators == 1 ? 0u : tile & 1u; };
  auto acc_use = [&](uint32_t tile) { return kScale && a.accumulators == 1 ? tile : tile >> 1; };
  const int chunks = (min(a.bn, a.out_cols - n0) + 63) / 64;
  // One accumulator and one chunk: the groups that take tiles out have one every other pass, but a parity tells only neighbouring passes
  // apart, so a group follows the passes of the other, too, and the accumulator is empty when it has seen them.
  const bool follow = kScale && a.accumulators == 1 && chunks == 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < a.stages; ++s) { tma::init(bar(bars.full[s]), 1); tma::init(bar(bars.ready[s]), kCtas * kTransformThreads / 32); tma::init(bar(bars.empty[s]), 1); }
    for (int i = 0; i < 2; ++i) { tma::init(bar(bars.acc_full[i]), 1); tma::init(bar(bars.acc_empty[i]), kCtas * (chunks * kGroup + (follow ? 1 : 0))); }
    for (int i = 0; i < 4; ++i) { tma::init(bar(bars.res_full[i]), 1); tma::init(bar(bars.res_empty[i]), 1); }
    tma::init(bar(bars.weights), 1); tma::init(bar(bars.weights_both), 1); tma::init(bar(bars.drained), 1);
    bars.dead = 0u;
    tc::fence_barrier_init();
  }
  if (warp == kWarpMma) {
    if (kPair) pair::tmem_alloc(&bars.tmem, a.tmem_cols); else tc::tmem_alloc(&bars.tmem, a.tmem_cols);
  }
  tc::fence_before_sync();
  __syncthreads();
  if (kPair) pair::sync();                // the other's barriers exist, too
  tc::fence_after_sync();
  const uint32_t tmem = bars.tmem;
  dependency_wait();

  if (warp == kWarpLoad) {
    if (lane == 0) {
      auto load_weights = [&](uint32_t dst, int kb, uint32_t b) {
        if (kForward) tma::load(dst, &a.b, kb * kStep, b0, b);
        else for (int j = 0; j * 64 < b_cols; ++j) tma::load(dst + j * kBoxBytes, &a.b, b0 + j * 64, kb * kStep, b);
      };
      if (a.resident) {
        tma::expect(bar(bars.weights), (uint32_t)a.k_blocks * a.b_bytes);
        for (int kb = 0; kb < a.k_blocks; ++kb) load_weights(tc::smem_addr(smem) + kb * a.b_bytes, kb, bar(bars.weights));
      }
      uint32_t it = 0;
      Ring at;
      bool ok = true;
      const uint32_t dst0 = tc::smem_addr(stages), full0 = bar(bars.full[0]), empty0 = bar(bars.empty[0]);
      for (int m = m_first; ok && m < m_end; m += m_step)
        for (int kb = 0; kb < a.k_blocks; ++kb, ++it, at.next(a.stages)) {
          if (!(ok = tma::wait(empty0 + at.s * 8, at.parity ^ 1u, dead))) break;
          const uint32_t dst = dst0 + at.s * stage_bytes, f = full0 + at.s * 8;
          tma::expect(f, stage_bytes);
          tma::load(dst, &a.a, kb * kStep, m * kRows, f);
          if (kParts) tma::load(dst + kTileBytes, &a.z, kb * kStep, m * kRows, f);
          if (!a.resident) load_weights(dst + kStageA, kb, f);
        }
      if (!ok) {                          // copies in flight land before the CTA leaves
        for (uint32_t k = it > (uint32_t)a.stages ? it - a.stages : 0u; k < it; ++k)
          tma::settle(bar(bars.full[k % a.stages]), k / a.stages & 1u);
      }
      if (a.resident)
        tma::settle(bar(bars.weights), 0u);
    }
  } else if (warp == kWarpMma) {
    if (kPair && rank != 0) {
      // the second CTA's: tells the first when its weights have landed (its steps are told by those who make dz of them)
      if (lane == 0) {
        if (tma::wait(bar(bars.weights), 0u, dead)) pair::arrive_first(bar(bars.weights_both));
        tma::settle(bar(bars.drained), 0u);
      }
    } else if (lane == 0) {
      const uint32_t desc = (kPair ? 1u << 27 : 0u) + idesc_of<T>((a.bn + 15) & ~15, false, !kForward);     // (bits 24 on: rows / 16)
      auto mma = [](uint32_t d, uint64_t da, uint64_t db, uint32_t add, uint32_t desc) {
        if (kPair) pair::mma(d, da, db, add, desc); else tc::mma(d, da, db, add, desc);
      };
      auto commit = [](uint32_t b) {
        if (kPair) pair::commit(b); else tc::commit(b);
      };
      // descriptors of the first stage and of the first step's weights; further on is an addition (in 16 bytes) to the address field
      constexpr uint64_t kNextB = kForward ? 2 : 128;
      const uint64_t a_desc = desc_swizzled(tc::smem_addr(stages), 16), stage16 = stage_bytes >> 4, b16 = a.resident ? a.b_bytes >> 4 : 0u;
      const uint64_t b_desc = desc_swizzled(a.resident ? tc::smem_addr(smem) : tc::smem_addr(stages) + kStageA, kForward ? 16 : kBoxBytes);
      const uint32_t ready0 = kParts ? bar(bars.ready[0]) : bar(bars.full[0]), empty0 = bar(bars.empty[0]);
      const int last_steps = (a.k - (a.k_blocks - 1) * kStep + 15) / 16;
      uint32_t tile = 0;
      Ring at;
      bool ok = !a.resident || (tma::wait(bar(bars.weights), 0u, dead) && (!kPair || tma::wait<kPair>(bar(bars.weights_both), 0u, dead)));
      for (int m = m_first; ok && m < m_end; m += m_step, ++tile) {
        const uint32_t buf = acc_of(tile);
        if (!(ok = tma::wait<kPair>(bar(bars.acc_empty[buf]), (acc_use(tile) & 1u) ^ 1u, dead))) break;
        const uint32_t d = tmem + buf * acc_stride;
        for (int kb = 0; kb < a.k_blocks; ++kb, at.next(a.stages)) {
          const uint64_t da = a_desc + at.s * stage16, db = b_desc + (a.resident ? kb * b16 : at.s * stage16);
          if (!(ok = tma::wait<kPair>(ready0 + at.s * 8, at.parity, dead))) break;
          tc::fence_after_sync();
          const int steps = kb == a.k_blocks - 1 ? last_steps : 4;
#pragma unroll
          for (int p = 0; p < (kParts == 2 ? 2 : 1); ++p)
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              if (ks < steps) mma(kScale && p ? d + acc_cols : d, da + p * (kTileBytes >> 4) + ks * 2, db + ks * kNextB, (p && !kScale) || ks ? 1u : (uint32_t)kb, desc);
          commit(empty0 + at.s * 8);
        }
        if (ok) commit(bar(bars.acc_full[buf]));
      }
      // products in flight end before tensor memory is given back
      commit(bar(bars.drained));
      tma::settle(bar(bars.drained), 0u);
    }
  } else if (kForward && warp == kWarpResidual) {
    if (lane == 0 && a.has_residual) {
      uint32_t it = 0;
      Ring at;
      bool ok = true;
      for (int m = m_first; ok && m < m_end; m += m_step)
        for (int c = 0; c < chunks; ++c, ++it, at.next(a.out_slots)) {
          const uint32_t s = at.s;
          if (!(ok = tma::wait(bar(bars.res_empty[s]), at.parity ^ 1u, dead))) break;
          tma::expect(bar(bars.res_full[s]), kTileBytes);
          tma::load(tc::smem_addr(out_tiles) + s * kTileBytes, &a.residual, n0 + c * 64, m * kRows, bar(bars.res_full[s]));
        }
      if (!ok)
        for (uint32_t k = it > (uint32_t)a.out_slots ? it - a.out_slots : 0u; k < it; ++k)
          tma::settle(bar(bars.res_full[k % a.out_slots]), k / a.out_slots & 1u);
    }
  } else if (warp >= kWarpEpilogue && warp < kWarpTransform) {
    const int group = (warp - kWarpEpilogue) / kGroup, tid = threadIdx.x - (kWarpEpilogue + group * kGroup) * 32;
    const int row = tid & 127;                                     // of the tile = lane of tensor memory
    const int threads = kGroup * 32;
    if (kForward) {
      if (group == 0 && tid < 256) bias[tid] = a.bias && tid < a.bn && n0 + tid < a.out_cols ? __ldg(a.bias + n0 + tid) : 0.f;
      named_sync(3, 2 * threads);
    }
    // A copy out of shared memory writes whole 16-byte chunks: the columns behind the last multiple of 8 go one by one.
    const int tail = a.out_cols & 7, whole = a.out_cols - tail;
    auto store_tail = [&](void *rows, int64_t ld, int m, const float *w) {
      const int r = m * kRows + row;
      if (r >= a.rows) return;
      T *p = static_cast<T *>(rows) + (int64_t)r * ld + whole;
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < tail) p[i] = narrow<T>(w[i]);
    };
    const bool behind = a.out_slots == 4 && a.keep_slots != 2;     // a group's last copies may still read while it fills the other slots
    uint32_t tile = 0, before = 4;
    Ring at;
    bool ok = true;
    for (int m = m_first; ok && m < m_end; m += m_step, ++tile) {
      const uint32_t buf = acc_of(tile);
      for (int c = 0; c < chunks; ++c, at.next(a.out_slots)) {
        const uint32_t s = at.s;
        if ((int)(s & 1u) != group) {
          if (follow) {
            if (tid == 0 && tma::wait(bar(bars.acc_full[buf]), acc_use(tile) & 1u, dead)) {
              if (kPair) pair::arrive_first(bar(bars.acc_empty[buf])); else tma::arrive(bar(bars.acc_empty[buf]));
            }
            __syncwarp();
          }
          continue;
        }
        if (tid == 0) {
          if (kForward && a.has_residual) {                        // the slot before is free for the residual of a chunk to come
            tma::stores_read<0>();
            if (before < 4) tma::arrive(bar(bars.res_empty[before]));
            before = s;
          } else if (behind) {
            tma::stores_read<1>();
          } else {
            tma::stores_read<0>();
          }
          bool all = tma::wait(bar(bars.acc_full[buf]), acc_use(tile) & 1u, dead);
          if (kForward && a.has_residual) all = all && tma::wait(bar(bars.res_full[s]), at.parity, dead);
          bars.ok[group] = all ? 1u : 0u;
        }
        named_sync(1 + group, threads);
        if (!(ok = *(volatile uint32_t *)&bars.ok[group] != 0u)) break;
        tc::fence_after_sync();
        const uint32_t ks = a.keep_slots == 4 ? s : (uint32_t)group;
        unsigned char *out = out_tiles + s * kTileBytes + row * tma::kRowBytes, *keep = keep_tiles + ks * kTileBytes + row * tma::kRowBytes;
#pragma unroll
        for (int half = 0; half < (kGroup == 8 ? 1 : 2); ++half) {
          const int h = kGroup == 8 ? tid >> 7 : half;
          float2 v[16];
          const uint32_t from = tmem + buf * acc_stride + c * 64 + h * 32 + ((uint32_t)(tid & 96) << 16);
          load32(from, &v[0].x);
          if constexpr (kScale) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              float2 l[8];
              tc::load16(from + acc_cols + q * 16, &l[0].x);
#pragma unroll
              for (int i = 0; i < 8; ++i) v[q * 8 + i] = fma2(l[i], both(1.f / 2048.f), v[q * 8 + i]);
            }
          }
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t in = (uint32_t)((h * 4 + q) ^ (row & 7)) * 16u;
            const int col = c * 64 + h * 32 + q * 8;
            float2 *w = v + q * 4;
            if (kForward) {
              const float4 b0 = *reinterpret_cast<const float4 *>(bias + col), b1 = *reinterpret_cast<const float4 *>(bias + col + 4);
              w[0] = add2(w[0], make_float2(b0.x, b0.y)); w[1] = add2(w[1], make_float2(b0.z, b0.w));
              w[2] = add2(w[2], make_float2(b1.x, b1.y)); w[3] = add2(w[3], make_float2(b1.z, b1.w));
              if (a.has_keep) {
                *reinterpret_cast<uint4 *>(keep + in) = pack<T>(&w[0].x);
                if (tail && n0 + col == whole) store_tail(a.keep_rows, a.ld_keep, m, &w[0].x);
              }
              activate8<kAct>(w);
              if (a.has_residual) {
                float2 r[4];
                unpack<T>(*reinterpret_cast<const uint4 *>(out + in), &r[0].x);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = add2(w[i], r[i]);
              }
            }
            *reinterpret_cast<uint4 *>(out + in) = pack<T>(&w[0].x);
            if (tail && n0 + col == whole) store_tail(a.out_rows, a.ld_out, m, &w[0].x);
          }
        }
        tc::fence_before_sync();
        tc::fence_generic_writes();
        if (lane == 0) {
          if (kPair) pair::arrive_first(bar(bars.acc_empty[buf])); else tma::arrive(bar(bars.acc_empty[buf]));
        }
        named_sync(1 + group, threads);
        if (tid == 0) {
          const bool any = n0 + c * 64 < whole;
          if (any) tma::store(&a.out, n0 + c * 64, m * kRows, tc::smem_addr(out_tiles) + s * kTileBytes);
          if (kForward && a.has_keep && any) tma::store(&a.keep, n0 + c * 64, m * kRows, tc::smem_addr(keep_tiles) + ks * kTileBytes);
          tma::store_commit();
        }
      }
    }
    if (tid == 0) tma::stores_done();
  } else if (kParts && warp >= kWarpTransform) {
    const int t = threadIdx.x - kWarpTransform * 32;
    Ring at;
    bool ok = true;
    for (int m = m_first; ok && m < m_end; m += m_step)
      for (int kb = 0; kb < a.k_blocks; ++kb, at.next(a.stages)) {
        const uint32_t s = at.s;
        if (!(ok = __all_sync(0xffffffffu, tma::wait(bar(bars.full[s]), at.parity, dead)))) break;
        unsigned char *A = stages + s * stage_bytes;
        constexpr int kChunks = (int)(kTileBytes / 16 / kTransformThreads);
        uint4 dy[kChunks], z[kChunks];
#pragma unroll
        for (int u = 0; u < kChunks; ++u) {
          dy[u] = shared16(A + (u * kTransformThreads + t) * 16);
          z[u] = shared16(A + kTileBytes + (u * kTransformThreads + t) * 16);
        }
#pragma unroll
        for (int u = 0; u < kChunks; ++u) {
          unsigned char *p = A + (u * kTransformThreads + t) * 16;
          transform_chunk<T, kAct, kParts, kScale, false>(p, p + kTileBytes, nullptr, dy[u], z[u], nullptr);
        }
        tc::fence_generic_writes();
        __syncwarp();
        if (lane == 0) {
          if (kPair) pair::arrive_first(bar(bars.ready[s])); else tma::arrive(bar(bars.ready[s]));
        }
      }
  }
  __syncwarp();
  tc::fence_before_sync();
  __syncthreads();
  if (kPair) pair::sync();                // nobody leaves while the other may still arrive here
  tc::fence_after_sync();
  if (threadIdx.x == 0 && bars.dead) *a.timeout = 1ull;
  if (warp == kWarpMma) {
    if (kPair) pair::tmem_free(tmem, a.tmem_cols); else tc::tmem_free(tmem, a.tmem_cols);
  }
}

// ---- dW and db ---------------------------------------------------------------------------------------------------
struct WeightsArgs {
  CUtensorMap dy, z, x;
  int n, k, n_tiles, k_tiles, splits, row_blocks;
  int bk;                         // columns of x of a tile, at most 256
  int stages, want_db;
  int ld;                         // row length of the partial sums
  float *partials, *db_partials;  // [splits, n, ld], [splits, n]
  uint32_t tmem_cols;
  unsigned long long *timeout;
};
constexpr int kWStep = 64;                      // rows of a step (32: 221 us instead of 173 without activation)
constexpr uint32_t kWBoxBytes = kWStep * tma::kRowBytes;
constexpr int kFlush = 8;                       // steps after which an accumulator is emptied
struct WeightsBarriers {
  uint64_t full[kMaxStages], ready[kMaxStages], empty[kMaxStages], sum_full[2], sum_empty[2], third_empty[2], done;
  uint32_t tmem, dead, pad[2];
};

// Parts of dz: 0 it is dy; 1 ReLU; 2 (fp16, what is left lies 2^11 higher) and 3 (bf16) smooth activations.
template <class T>
__host__ __device__ constexpr int weight_parts(int act) {
  return act == GS_DENSE_NONE ? 0 : act == GS_DENSE_RELU ? 1 : __is_same(T, __half) ? 2 : 3;
}
//
// The tensor core cuts off what an addition leaves below the accumulator's last bit, so over thousands of additions the sums
// shrink: 1M rows in 74 splits were 9e-5 off.  So the accumulator of dz, or of its high part, is emptied every 8 steps, after
// 32 additions, into fp32 registers of the eight worker warps, which round to nearest (two accumulators in turn where there
// is one part: 2e-7 to 7e-7 off).  The other parts have an accumulator of their own, which loses as much of 2^-8 as much.
template <class T, int kAct, bool kPair>
__global__ void __launch_bounds__(384, 1) k_dense_weights(const __grid_constant__ WeightsArgs a) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char *smem = smem_raw + ((1024u - (tc::smem_addr(smem_raw) & 1023u)) & 1023u);
  constexpr int kParts = weight_parts<T>(kAct);
  constexpr bool kLow = kParts >= 2, kScale = kParts == 2;
  constexpr uint32_t kStageA = (kParts ? 2 : 1) * 2 * kWBoxBytes;
  static_assert(!kPair || kParts > 0, "pairs make dz");
  constexpr int kCtas = kPair ? 2 : 1;
  const uint32_t rank = kPair ? pair::rank() : 0u;
  const int x_boxes = (a.bk / kCtas + 63) / 64;
  const uint32_t stage_bytes = kStageA + x_boxes * kWBoxBytes;
  // the third part of dz, in two buffers in turn: it is needed for a short time, and in the stages it would cost one of three
  // (397 us instead of 362 for 1M rows of 256 to 256 with SiLU)
  unsigned char *thirds = smem + a.stages * stage_bytes;
  WeightsBarriers &bars = *reinterpret_cast<WeightsBarriers *>(thirds + (kParts == 3 ? 4 * kWBoxBytes : 0u));
  float *sums = reinterpret_cast<float *>(smem);          // [16, 128], at the end, when the stages have served
  volatile uint32_t *dead = &bars.dead;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [](const uint64_t &b) { return tc::smem_addr(&b); };

  if (threadIdx.x == 0) {
    for (int s = 0; s < a.stages; ++s) { tma::init(bar(bars.full[s]), 1); tma::init(bar(bars.ready[s]), kCtas * kWorkerWarps); tma::init(bar(bars.empty[s]), 1); }
    for (int i = 0; i < 2; ++i) { tma::init(bar(bars.sum_full[i]), 1); tma::init(bar(bars.sum_empty[i]), kCtas * kWorkerWarps); tma::init(bar(bars.third_empty[i]), 1); }
    tma::init(bar(bars.done), 1);
    bars.dead = 0u;
    tc::fence_barrier_init();
  }
  if (warp == kWarpMma) {
    if (kPair) pair::tmem_alloc(&bars.tmem, a.tmem_cols); else tc::tmem_alloc(&bars.tmem, a.tmem_cols);
  }
  tc::fence_before_sync();
  __syncthreads();
  if (kPair) pair::sync();
  tc::fence_after_sync();
  const uint32_t tmem = bars.tmem;
  dependency_wait();

  const int tiles = a.n_tiles / kCtas * a.k_tiles, tile = blockIdx.x / kCtas % tiles, split = blockIdx.x / kCtas / tiles;
  const int n0 = (tile / a.k_tiles * kCtas + (int)rank) * kRows, k0 = tile % a.k_tiles * a.bk, b0 = k0 + (int)rank * (a.bk / 2);
  const int first = (int)((int64_t)a.row_blocks * split / a.splits), count = (int)((int64_t)a.row_blocks * (split + 1) / a.splits) - first;
  const int dz_boxes = a.n - n0 > 64 ? 2 : 1, cols = min(a.bk, a.k - k0), boxes = kPair ? x_boxes : (cols + 63) / 64;
  const bool db = a.want_db && k0 == 0, touched = kParts || db;      // the workers look at every step
  const uint32_t second = a.bk > 128 ? 256u : 128u;                  // columns of the second accumulator

  if (warp < kWarpWorker) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == kWarpLoad && lane == 0) {
      int it = 0;
      bool ok = true;
      Ring at;
      const uint32_t dst0 = tc::smem_addr(smem), full0 = bar(bars.full[0]), empty0 = bar(bars.empty[0]);
      for (; it < count; ++it, at.next(a.stages)) {
        const int r = first + it;
        if (!(ok = tma::wait(empty0 + at.s * 8, at.parity ^ 1u, dead))) break;
        const uint32_t dst = dst0 + at.s * stage_bytes, f = full0 + at.s * 8;
        tma::expect(f, (uint32_t)(dz_boxes * (kParts ? 2 : 1) + boxes) * kWBoxBytes);
        for (int j = 0; j < dz_boxes; ++j) {
          tma::load(dst + j * kWBoxBytes, &a.dy, n0 + j * 64, r * kWStep, f);
          if (kParts) tma::load(dst + (2 + j) * kWBoxBytes, &a.z, n0 + j * 64, r * kWStep, f);
        }
        for (int j = 0; j < boxes; ++j) tma::load(dst + kStageA + j * kWBoxBytes, &a.x, b0 + j * 64, r * kWStep, f);
      }
      if (!ok)
        for (int k = it > a.stages ? it - a.stages : 0; k < it; ++k)
          tma::settle(bar(bars.full[k % a.stages]), k / a.stages & 1);
    } else if (warp == kWarpMma && lane == 0 && rank != 0) {
      tma::settle(bar(bars.done), 0u);
    } else if (warp == kWarpMma && lane == 0) {
      const uint32_t desc = (kPair ? 1u << 27 : 0u) + idesc_of<T>(kPair ? 256 : (cols + 15) & ~15, true, true);
      auto commit = [](uint32_t b) {
        if (kPair) pair::commit(b); else tc::commit(b);
      };
      const uint64_t a_desc = desc_swizzled(tc::smem_addr(smem), kWBoxBytes), b_desc = a_desc + (kStageA >> 4), stage16 = stage_bytes >> 4;
      const uint64_t third_desc = desc_swizzled(tc::smem_addr(thirds), kWBoxBytes);
      const uint32_t ready0 = touched ? bar(bars.ready[0]) : bar(bars.full[0]), empty0 = bar(bars.empty[0]);
      Ring at;
      for (int it = 0; it < count; ++it, at.next(a.stages)) {
        const int group = it / kFlush;
        // accumulator of this group: one of two in turn, or the first one always
        const int buf = kLow ? 0 : group & 1, use = kLow ? group : group >> 1;
        const uint64_t da = a_desc + at.s * stage16, db = b_desc + at.s * stage16;
        if (!tma::wait<kPair>(ready0 + at.s * 8, at.parity, dead)) break;
        auto part = [&](uint64_t dz, uint32_t d, bool add) {
#pragma unroll
          for (int ks = 0; ks < kWStep / 16; ++ks) {
            if (kPair) pair::mma(d, dz + ks * 128, db + ks * 128, add || ks ? 1u : 0u, desc);
            else tc::mma(d, dz + ks * 128, db + ks * 128, add || ks ? 1u : 0u, desc);
          }
        };
        tc::fence_after_sync();
        if (kParts == 3) {
          part(third_desc + (it & 1) * (2 * kWBoxBytes >> 4), tmem + second, it > 0);
          commit(bar(bars.third_empty[it & 1]));
        }
        if (kLow) part(da + (2 * kWBoxBytes >> 4), tmem + second, kParts == 3 || it > 0);
        if (it % kFlush == 0 && !tma::wait<kPair>(bar(bars.sum_empty[buf]), (use & 1) ^ 1, dead)) break;
        tc::fence_after_sync();
        part(da, tmem + buf * second, it % kFlush > 0);
        commit(empty0 + at.s * 8);
        if (it % kFlush == kFlush - 1 || it == count - 1) commit(bar(bars.sum_full[buf]));
      }
      // products in flight end before tensor memory is given back
      commit(bar(bars.done));
      tma::settle(bar(bars.done), 0u);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    // As a holder of sums: rows (lanes of tensor memory) 32 (warp % 4) + lane, columns from 128 * half on.  As a maker of dz:
    // the eight columns 16 bytes chunk & 7 of box chunk >> 3 of rows t / 16, 16 further, ...: always the same columns.
    const int t = threadIdx.x - kWarpWorker * 32, half = t >> 7, n = n0 + (t & 127);
    const uint32_t lanes = tmem + ((uint32_t)(t & 96) << 16) + half * 128;
    const int chunk = (t & 7) | (t >> 4 & 8), row0 = (t >> 3) & 15;
    float2 mine[4];
    float acc[128];
#pragma unroll
    for (int i = 0; i < 4; ++i) mine[i] = make_float2(0.f, 0.f);
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
      if (lane == 0) {
        if (kPair) pair::arrive_first(bar(bars.sum_empty[buf])); else tma::arrive(bar(bars.sum_empty[buf]));
      }
    };
    // an accumulator is emptied a step after its last one was made ready: the products have time
    Ring at;
    for (int it = 0; ok && it < count; ++it, at.next(a.stages)) {
      if (touched) {
        const int s = at.s;
        if (!(ok = __all_sync(0xffffffffu, tma::wait(bar(bars.full[s]), at.parity, dead)))) break;
        unsigned char *A = smem + s * stage_bytes + (chunk >> 3) * kWBoxBytes;
        // (rows 16 apart have the same swizzle)
        if (kParts == 3 && !(ok = __all_sync(0xffffffffu, tma::wait(bar(bars.third_empty[it & 1]), (it >> 1 & 1) ^ 1, dead)))) break;
        auto in = [&](int u) { return A + (row0 + 16 * u) * (int)tma::kRowBytes + (((chunk & 7) ^ (row0 & 7)) * 16); };
        const ptrdiff_t third = thirds + (it & 1) * (2 * kWBoxBytes) - (smem + s * stage_bytes);
        if ((chunk >> 3) < dz_boxes) {
#pragma unroll
          for (int u = 0; u < kWStep / 16; u += 2) {
            const uint4 dy0 = shared16(in(u)), dy1 = shared16(in(u + 1));
            if constexpr (kParts > 0) {
              const uint4 z0 = shared16(in(u) + 2 * kWBoxBytes), z1 = shared16(in(u + 1) + 2 * kWBoxBytes);
              transform_chunk<T, kAct, kParts, kScale, true>(in(u), in(u) + 2 * kWBoxBytes, in(u) + third, dy0, z0, mine);
              transform_chunk<T, kAct, kParts, kScale, true>(in(u + 1), in(u + 1) + 2 * kWBoxBytes, in(u + 1) + third, dy1, z1, mine);
            } else {
              float2 v[4], w[4];
              unpack<T>(dy0, &v[0].x);
              unpack<T>(dy1, &w[0].x);
#pragma unroll
              for (int i = 0; i < 4; ++i) mine[i] = add2(mine[i], add2(v[i], w[i]));
            }
          }
        }
        if (kParts) tc::fence_generic_writes();
        __syncwarp();
        if (lane == 0) {
          if (kPair) pair::arrive_first(bar(bars.ready[s])); else tma::arrive(bar(bars.ready[s]));
        }
      }
      if (it % kFlush == 0 && it > 0) flush(it / kFlush - 1);
    }
    if (ok && count > 0) flush((count - 1) / kFlush);
    if constexpr (kLow) {
      // (all products have completed with the last group's: the high part's are issued last)
      if (ok && count > 0) {
#pragma unroll
        for (int c = 0; c < 128; c += 32)
          if (half * 128 + c < cols) {
            float v[32];
            load32(lanes + second + c, v);
            constexpr float k = kScale ? 1.f / 2048.f : 1.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[c + i] = fmaf(v[i], k, acc[c + i]);
          }
      }
    }
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
    named_sync(2, kWorkerWarps * 32);                        // (every worker has seen the last products complete)
    if (db) {
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<float2 *>(sums + row0 * 128 + chunk * 8 + 2 * i) = mine[i];
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
  if (kPair) pair::sync();
  tc::fence_after_sync();
  if (threadIdx.x == 0 && bars.dead) *a.timeout = 1ull;
  if (warp == kWarpMma) {
    if (kPair) pair::tmem_free(tmem, a.tmem_cols); else tc::tmem_free(tmem, a.tmem_cols);
  }
}

// dW [n, k] and db [n] from the splits' sums, four values a lane.  Many splits are taken by 16 groups of lanes, so that many loads are in
// flight (256 to 8 with 148 splits: the weights' gradient 35 us instead of 39), whose sums are added in their order; few
// by one (1024 to 1024 with 4: 61 instead of 87).  The last CTAs take db.
template <int kGroups>
__global__ void __launch_bounds__(512) k_dense_sums(const float *partials, const float *db_partials, int splits, int n, int k, int ld, int blocks, float *dw, float *db) {
  constexpr int kLanes = 512 / kGroups, kValues = 4 * kLanes;
  __shared__ double part[kGroups > 1 ? kGroups : 1][kGroups > 1 ? kValues : 1];
  dependency_wait();
  const bool bias = (int)blockIdx.x >= blocks;
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int64_t count = bias ? n : (int64_t)n * ld, first = (int64_t)(bias ? blockIdx.x - blocks : blockIdx.x) * kValues;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  if (!bias) {
    const int64_t i = first + lane * 4;                       // (rows of partial sums are a multiple of four values)
    if (i < count) {
#pragma unroll 4
      for (int p = group; p < splits; p += kGroups) {
        const float4 v = __ldcs(reinterpret_cast<const float4 *>(partials + p * count + i));
        s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
      }
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (first + lane * 4 + q < count)
        for (int p = group; p < splits; p += kGroups) s[q] += __ldcs(db_partials + p * count + first + lane * 4 + q);
  }
  auto put = [&](int64_t i, double v) {
    if (i >= count) return;
    if (bias) {
      db[i] = (float)v;
    } else {
      const int row = (int)(i / ld), col = (int)(i % ld);
      if (col < k) dw[(int64_t)row * k + col] = (float)v;
    }
  };
  if constexpr (kGroups == 1) {
#pragma unroll
    for (int q = 0; q < 4; ++q) put(first + lane * 4 + q, s[q]);
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) part[group][lane * 4 + q] = s[q];
    __syncthreads();
    if (threadIdx.x < kValues) {
      double t = part[0][threadIdx.x];
#pragma unroll
      for (int g = 1; g < kGroups; ++g) t += part[g][threadIdx.x];
      put(first + threadIdx.x, t);
    }
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
uint32_t tmem_columns(uint32_t n) {
  uint32_t c = 32;
  while (c < n) c *= 2;
  return c;
}

// The shape of a call of k_dense_rows: tile width, weights resident or not, pipeline depth.  False where it does not fit.
bool shape_rows(RowsArgs &a, bool forward, bool transform, int bn, int ctas, bool resident, int want, uint32_t &smem) {
  a.bn = bn;
  a.n_tiles = ceil_div(a.out_cols, bn);
  a.b_bytes = forward ? (uint32_t)(bn / ctas) * tma::kRowBytes : (uint32_t)ceil_div(bn / ctas, 64) * kBoxBytes;
  a.resident = resident;
  const uint32_t stage = (transform ? 2 : 1) * kTileBytes + (resident ? 0u : a.b_bytes);
  const uint64_t fixed = 1024 + 1024 + sizeof(RowsBarriers) + (resident ? (uint64_t)a.k_blocks * a.b_bytes : 0u);
  // (where the weights come with every step, a step more before a tile more on its way out: 20 011 rows of 1024 to 1024 41.7 us instead of 44.2)
  for (a.out_slots = resident ? 4 : 2; a.out_slots >= 2; a.out_slots -= 2) {
    a.keep_slots = !a.has_keep ? 0 : a.has_residual ? 2 : a.out_slots;
    const uint64_t used = fixed + (uint64_t)(a.out_slots + a.keep_slots) * kTileBytes;
    if (used + (uint64_t)want * stage > kSmemMost) continue;
    a.stages = (int)((kSmemMost - used) / stage);
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    smem = (uint32_t)used + (uint32_t)a.stages * stage;
    return true;
  }
  return false;
}
// The number of CTAs that share a tile's weights, or 0.  scaled: the second part of dz has accumulators of its own.
int plan_rows(RowsArgs &a, bool forward, bool transform, bool scaled, int num_sms, uint32_t &smem, int &grid) {
  // Wide tiles read the rows once; narrower ones where there are fewer tiles than SMs.  Results leave in boxes of 64 columns, so tiles
  // beside one another are a multiple of that.
  int bn = a.out_cols <= 256 ? (a.out_cols + 15) / 16 * 16 : 256, ctas = 1;
  while (bn > 64 && (int64_t)a.m_tiles * ceil_div(a.out_cols, bn) * 2 <= num_sms) bn = (bn / 2 + 63) / 64 * 64;
  if (!forward) bn = (bn + 63) / 64 * 64;
  const int narrow = bn > 128 ? 128 : bn;
  // Where dz is made, tiles of more than 128 columns by pairs of CTAs, each with half of the weights, which leaves room for three or
  // four steps of dy and preact instead of two: dx of 1M rows of 256 to 256 in bf16 with SiLU 295 us instead of 353, with ReLU 237
  // instead of 287.  Four steps where the second part has its own accumulator and the next tile's products wait for this one's to leave: fp16
  // 335 us instead of 357 with three (308 with both parts in one accumulator, without the bits that fp16 then loses).  Without dz the steps are small and the first CTA's wait for both costs more than it brings: 181 instead of
  // 164, forward with residual 350 instead of 313, 20 011 rows of 1024 to 1024 55 instead of 50.
  if (transform && bn > 128 && a.m_tiles >= 2 &&
      ((scaled && shape_rows(a, forward, transform, 256, 2, true, 4, smem)) || shape_rows(a, forward, transform, 256, 2, true, 3, smem)))
    ctas = 2;
  // Else resident weights, up to six steps of a narrower tile if need be (forward, 300 000 rows of 256 to 256 with residual and kept
  // pre-activation 103 us instead of 153; 100 000 of 320 to 512 85 instead of 110), beyond that weights that come with every step
  // rather than two looks at the rows (100 000 of 512 to 512 65 instead of 83).
  if (ctas == 1 && !(shape_rows(a, forward, transform, bn, 1, true, 3, smem) || (a.k_blocks <= 6 && shape_rows(a, forward, transform, narrow, 1, true, 3, smem)) ||
                     shape_rows(a, forward, transform, bn, 1, false, 3, smem) || shape_rows(a, forward, transform, narrow, 1, true, 3, smem) ||
                     shape_rows(a, forward, transform, narrow, 1, false, 2, smem)))
    return 0;
  const uint32_t acc = (((uint32_t)a.bn + 63u) & ~63u) * (scaled ? 2u : 1u);
  a.accumulators = 2u * acc <= 512u ? 2 : 1;
  a.tmem_cols = tmem_columns((uint32_t)a.accumulators * acc);
  const int tiles = ceil_div(a.m_tiles, ctas);
  int groups = num_sms / ctas / a.n_tiles;
  if (groups < 1) groups = 1;
  if (groups > tiles) groups = tiles;
  grid = groups * a.n_tiles * ctas;
  return ctas;
}

// Once for every kernel and device: all of the SM's shared memory may be asked for.
template <class Kernel>
void opt_in(Kernel kernel, std::atomic<uint64_t> &devices) {
  int device = 0;
  cudaGetDevice(&device);
  const uint64_t bit = 1ull << (device & 63);
  if (device < 64 && (devices.load(std::memory_order_relaxed) & bit)) return;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost) == cudaSuccess) devices.fetch_or(bit, std::memory_order_relaxed);
}
// As launch_chained, in clusters of two where asked for.
template <class Args>
void launch(void (*kernel)(Args), int grid, int threads, uint32_t smem, bool pairs, cudaStream_t st, const Args &a) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = threads; cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = pairs ? 2 : 1;
  cudaLaunchKernelEx(&cfg, kernel, a);
}
template <class T, bool kForward, int kAct, bool kPair>
void run_rows_as(const RowsArgs &a, uint32_t smem, int grid, cudaStream_t st) {
  static std::atomic<uint64_t> devices{0};
  opt_in(k_dense_rows<T, kForward, kAct, kPair>, devices);
  launch(k_dense_rows<T, kForward, kAct, kPair>, grid, kRowsThreads<kForward, kRowsParts<kForward, kAct>>, smem, kPair, st, a);
}
template <class T, bool kForward>
void run_rows(int act, const RowsArgs &a, uint32_t smem, int grid, cudaStream_t st) {
  if (act == GS_DENSE_NONE) run_rows_as<T, kForward, GS_DENSE_NONE, false>(a, smem, grid, st);
  else if (act == GS_DENSE_RELU) run_rows_as<T, kForward, GS_DENSE_RELU, false>(a, smem, grid, st);
  else if (act == GS_DENSE_SILU) run_rows_as<T, kForward, GS_DENSE_SILU, false>(a, smem, grid, st);
  else run_rows_as<T, kForward, GS_DENSE_GELU, false>(a, smem, grid, st);
}
template <class T>
void run_pairs(int act, const RowsArgs &a, uint32_t smem, int grid, cudaStream_t st) {
  if (act == GS_DENSE_RELU) run_rows_as<T, false, GS_DENSE_RELU, true>(a, smem, grid, st);
  else if (act == GS_DENSE_SILU) run_rows_as<T, false, GS_DENSE_SILU, true>(a, smem, grid, st);
  else run_rows_as<T, false, GS_DENSE_GELU, true>(a, smem, grid, st);
}

template <class T>
int fwd(const DenseArgs &d, int num_sms, cudaStream_t st) {
  RowsArgs a;
  a.bias = d.bias; a.out_cols = d.out; a.k = d.in; a.k_blocks = ceil_div(d.in, kStep); a.m_tiles = ceil_div(d.rows, kRows);
  a.rows = (int)d.rows; a.out_rows = d.y; a.ld_out = d.ld_y; a.keep_rows = d.preact; a.ld_keep = d.ld_preact;
  a.has_keep = d.preact != nullptr; a.has_residual = d.residual != nullptr; a.timeout = d.timeout;
  uint32_t smem;
  int grid;
  if (!plan_rows(a, true, false, false, num_sms, smem, grid)) return -1;
  if (!tma::make_map(&a.a, d.dtype, d.x, d.rows, d.in, d.ld_x, kRows) || !tma::make_map(&a.b, d.dtype, d.w, d.out, d.in, d.ld_w, a.bn) ||
      (d.out >= 8 && !tma::make_map(&a.out, d.dtype, d.y, d.rows, d.out & ~7, d.ld_y, kRows)) ||
      (d.out >= 8 && a.has_keep && !tma::make_map(&a.keep, d.dtype, d.preact, d.rows, d.out & ~7, d.ld_preact, kRows)) ||
      (a.has_residual && !tma::make_map(&a.residual, d.dtype, d.residual, d.rows, d.out, d.ld_residual, kRows)))
    return -1;
  run_rows<T, true>(d.act, a, smem, grid, st);
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

template <class T, int kAct, bool kPair>
void run_weights_as(WeightsArgs &a, cudaStream_t st) {
  constexpr int kParts = weight_parts<T>(kAct);
  if (kPair) a.bk = 256;
  const uint32_t stage = ((kParts ? 2u : 1u) * 2u + (uint32_t)ceil_div(kPair ? a.bk / 2 : a.bk, 64)) * kWBoxBytes;
  const uint32_t fixed = 1024 + (kParts == 3 ? 4 * kWBoxBytes : 0u) + sizeof(WeightsBarriers);
  a.stages = (int)((kSmemMost - fixed) / stage);
  if (a.stages > kMaxStages) a.stages = kMaxStages;
  a.tmem_cols = a.bk > 128 ? 512u : 256u;
  static std::atomic<uint64_t> devices{0};
  opt_in(k_dense_weights<T, kAct, kPair>, devices);
  launch(k_dense_weights<T, kAct, kPair>, a.n_tiles * a.k_tiles * a.splits, 384, fixed + a.stages * stage, kPair, st, a);
}
template <class T, int kAct>
void run_weights(WeightsArgs &a, cudaStream_t st) {
  // Where dz is made, an even number of feature tiles over more than 128 columns of x: by pairs, each CTA with half of x.  1M rows of 256
  // to 256 with SiLU in fp16 301 us instead of 355, in bf16 (three parts: arithmetic bounds it) 349 instead of 357, with ReLU 234
  // instead of 230; 20 011 rows of 1024 to 1024 with ReLU 82 instead of 91.
  if constexpr (kAct != GS_DENSE_NONE) {
    if (a.n_tiles % 2 == 0 && a.bk > 128) return run_weights_as<T, kAct, true>(a, st);
  }
  run_weights_as<T, kAct, false>(a, st);
}

// Every tensor map is made before the first launch: a call whose map the driver refuses launches nothing.
template <class T>
int bwd(const DenseArgs &d, int num_sms, cudaStream_t st) {
  const bool plain = d.act == GS_DENSE_NONE;
  int launches = 0;
  RowsArgs a;
  uint32_t smem = 0;
  int grid = 0, ctas = 0;
  if (d.dx) {
    a.bias = nullptr; a.out_cols = d.in; a.k = d.out; a.k_blocks = ceil_div(d.out, kStep); a.m_tiles = ceil_div(d.rows, kRows);
    a.rows = (int)d.rows; a.out_rows = d.dx; a.ld_out = d.ld_dx; a.keep_rows = nullptr; a.ld_keep = 0;
    a.has_keep = a.has_residual = 0; a.timeout = d.timeout;
    ctas = plan_rows(a, false, !plain, d.dtype == GS_TYPE_F16 && (d.act == GS_DENSE_SILU || d.act == GS_DENSE_GELU), num_sms, smem, grid);
    if (!ctas) return -1;
    if (!tma::make_map(&a.a, d.dtype, d.dy, d.rows, d.out, d.ld_dy, kRows) || !tma::make_map(&a.b, d.dtype, d.w, d.out, d.in, d.ld_w, kStep) ||
        (d.in >= 8 && !tma::make_map(&a.out, d.dtype, d.dx, d.rows, d.in & ~7, d.ld_dx, kRows)) ||
        (!plain && !tma::make_map(&a.z, d.dtype, d.preact_in, d.rows, d.out, d.ld_preact, kRows)))
      return -1;
  }
  WeightsArgs w;
  if (d.dw) {
    const WeightsPlan p = plan_weights(d.rows, d.in, d.out, num_sms < kSplitSms ? num_sms : kSplitSms);
    w.n = d.out; w.k = d.in; w.n_tiles = p.n_tiles; w.k_tiles = p.k_tiles; w.splits = p.splits; w.bk = p.bk; w.ld = p.ld;
    w.row_blocks = ceil_div(d.rows, kWStep); w.want_db = d.db != nullptr; w.timeout = d.timeout;
    w.partials = d.partials;
    w.db_partials = d.partials + (size_t)p.splits * d.out * p.ld;
    if (!tma::make_map(&w.dy, d.dtype, d.dy, d.rows, d.out, d.ld_dy, kWStep) || !tma::make_map(&w.x, d.dtype, d.x, d.rows, d.in, d.ld_x, kWStep) ||
        (!plain && !tma::make_map(&w.z, d.dtype, d.preact_in, d.rows, d.out, d.ld_preact, kWStep)))
      return -1;
  }
  if (d.dx) {
    if (ctas == 2) run_pairs<T>(d.act, a, smem, grid, st);
    else run_rows<T, false>(d.act, a, smem, grid, st);
    ++launches;
  }
  if (d.dw) {
    if (d.act == GS_DENSE_NONE) run_weights<T, GS_DENSE_NONE>(w, st);
    else if (d.act == GS_DENSE_RELU) run_weights<T, GS_DENSE_RELU>(w, st);
    else if (d.act == GS_DENSE_SILU) run_weights<T, GS_DENSE_SILU>(w, st);
    else run_weights<T, GS_DENSE_GELU>(w, st);
    auto sum = [&](auto kernel, int values) {
      const int blocks = ceil_div((int64_t)d.out * w.ld, values);
      launch_chained(kernel, blocks + (d.db ? ceil_div(d.out, values) : 0), 512, 0, st, (const float *)w.partials, (const float *)w.db_partials, w.splits, d.out, d.in,
                     w.ld, blocks, d.dw, d.db);
    };
    if (w.splits >= 16) sum(k_dense_sums<16>, 128);
    else sum(k_dense_sums<1>, 2048);
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
