// The global norm over many gradient tensors and the tensors scaled to a largest norm.
//
//   s_i = sum of the buffers of tensor i (fp32, in the order given);  norm = sqrt(sum over all elements of s^2)
//   scale = 1 if norm <= max_norm, else max_norm / norm (0 if the norm is not finite);  out_i = scale s_i
//
// k_grad_squares walks a common space of 8192-element chunks of all tensors with a persistent grid and leaves a sum per CTA;
// the sums are added in a fixed order by k_grad_norm (one CTA) or by every CTA of k_grad_scale for itself, so no atomics and
// the same bits from run to run.  Bound by the bytes of the gradients, once for the norm and once more for what follows (which
// finds them in the L2 as long as they fit there).
//
// The squares are summed in 64 bits: 2^30 elements of one size lose nothing, and gradients whose squares leave fp32's range
// (|g| above 2^63 or below 2^-63) keep their norm.  Conversions to 64 bits run at an eighth of the fp32 rate, so eight squares are first summed in
// fp32 where the largest of them lies well inside the range (what underflows beside it is below 2^-40 of the sum); else each is
// taken in 64 bits.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gs_device.cuh"

namespace gs {
namespace {

#include "gs_rows.cuh"

constexpr int kGradThreads = 256;
constexpr int kGradChunk = 8192;          // elements

struct GradEntry {
  const void *grad;
  void *out;
  uint64_t count;
  uint32_t chunk_start;                   // chunks of the tensors before
  uint16_t more_start;                    // its further buffers in the table of pointers
  uint8_t num_more, dtype;
  uint32_t head;                          // elements before the first 16-byte boundary; 2^32 - 1 where the buffers' boundaries differ:
                                          // element by element then
};
// The tables travel as kernel parameters: nothing to allocate or copy, and a captured launch keeps its own.
template <int kTensors, int kMore>
struct GradArgs {
  int num_tensors;
  uint32_t chunks;
  GradEntry t[kTensors];
  const void *more[kMore];
};
using GradArgsSmall = GradArgs<64, 128>;
using GradArgsLarge = GradArgs<GS_GRAD_MAX_TENSORS, GS_GRAD_MAX_BUFFERS>;
static_assert(sizeof(GradArgsLarge) <= 32000, "kernel parameters end at 32764 bytes");

template <class Args>
__device__ __forceinline__ int entry_of(const Args &a, uint32_t chunk) {
  int lo = 0, hi = a.num_tensors - 1;     // last entry with chunk_start <= chunk
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.t[mid].chunk_start <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Calls vec(values, element) for whole vectors and one(value, element) for single elements of the sums s of a chunk.  Several vectors
// are asked for before the first is used: four, or with further buffers (kMore) those of four buffers at one or two places (one
// buffer after another is waited for one after another: the norm of eight buffers of 25M elements took about 195 us, 113 so; 122 are
// the bytes' time).
template <class T, bool kMore, class Args, class Vec, class One>
__device__ __forceinline__ void chunk_sums(const Args &a, const GradEntry &t, uint32_t chunk, Vec vec, One one) {
  constexpr int V = kVecOf<T>, U = kMore ? 8 / V : 4, B = kMore ? 4 : 1;
  const T *g = static_cast<const T *>(t.grad);
  const uint64_t head = t.head == 0xffffffffu ? t.count : t.head;
  const uint64_t begin = (uint64_t)(chunk - t.chunk_start) * kGradChunk, end = min(begin + kGradChunk, t.count);
  // vectors start at head + i V: those that start inside [begin, end) and are whole belong to the chunk, so do the single elements
  const uint64_t first = begin <= head ? head : head + (begin - head + V - 1) / V * V;
  const uint64_t last = t.count < head + V ? head : head + (t.count - head) / V * V;      // end of the whole vectors
  const uint64_t stop = min(end, last);
  const int vectors = first < stop ? (int)((stop - first + V - 1) / V) : 0;
  const int buffers = 1 + (kMore ? t.num_more : 0);
  for (int v0 = threadIdx.x; v0 < vectors; v0 += U * kGradThreads) {
    const uint64_t e0 = first + (uint64_t)v0 * V;
    if constexpr (!kMore) {
      uint4 raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (v0 + u * kGradThreads < vectors) raw[u] = *reinterpret_cast<const uint4 *>(g + e0 + u * kGradThreads * V);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (v0 + u * kGradThreads < vectors) {
          float s[V];
          unpack<T>(raw[u], s);
          vec(s, e0 + u * kGradThreads * V);
        }
    } else {
      float s[U][V];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) s[u][i] = -0.f;           // (adds nothing, also to a zero of either sign)
#pragma unroll 1
      for (int k0 = 0; k0 < buffers; k0 += B) {
        uint4 raw[B][U];
#pragma unroll
        for (int k = 0; k < B; ++k) {
          const T *p = (k0 + k > 0 && k0 + k < buffers ? static_cast<const T *>(a.more[t.more_start + k0 + k - 1]) : g) + e0;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            raw[k][u] = make_uint4(0u, 0u, 0u, 0u);
            if (k0 + k < buffers && v0 + u * kGradThreads < vectors) raw[k][u] = *reinterpret_cast<const uint4 *>(p + u * kGradThreads * V);
          }
        }
#pragma unroll
        for (int k = 0; k < B; ++k)
          if (k0 + k < buffers) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
              float x[V];
              unpack<T>(raw[k][u], x);
#pragma unroll
              for (int i = 0; i < V; ++i) s[u][i] += x[i];
            }
          }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (v0 + u * kGradThreads < vectors) vec(s[u], e0 + u * kGradThreads * V);
    }
  }
  auto single = [&](uint64_t e) {
    float s = widen(g[e]);
    for (int k = 0; k < buffers - 1; ++k) s += widen(static_cast<const T *>(a.more[t.more_start + k])[e]);
    one(s, e);
  };
  for (uint64_t e = begin + threadIdx.x; e < min(end, head); e += kGradThreads) single(e);
  for (uint64_t e = max(begin, max(last, head)) + threadIdx.x; e < end; e += kGradThreads) single(e);
}

template <int V, bool kInRange = false>
__device__ __forceinline__ double squares(const float s[V]) {
  float most = kInRange ? 1.f : 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (!kInRange) most = fmaxf(most, fabsf(s[i]));
  // a NaN is dropped by fmaxf, but not by the sum: fp32 or 64 bits, it comes through
  if (most < 0x1p60f && (most > 0x1p-40f || most == 0.f)) {
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) q = fmaf(s[i], s[i], q);
    return (double)q;
  }
  double q = 0.0;
#pragma unroll
  for (int i = 0; i < V; ++i) q = fma((double)s[i], (double)s[i], q);
  return q;
}

__device__ __forceinline__ double block_sum(double q, double *shared) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = q;
  __syncthreads();
  q = shared[0];
#pragma unroll
  for (int w = 1; w < kGradThreads / 32; ++w) q += shared[w];
  return q;
}

struct Clip { float norm, scale; };
__device__ __forceinline__ Clip clip_of(double squares, float max_norm) {
  const double norm = sqrt(squares);
  Clip c;
  c.norm = (float)norm;
  c.scale = !isfinite(c.norm) ? 0.f : norm <= (double)max_norm ? 1.f : (float)((double)max_norm / norm);
  return c;
}
// Of the CTAs' sums; every thread of the CTA gets it.
__device__ __forceinline__ Clip clip_from_partials(const double *partials, int count, float max_norm, double *shared) {
  double q = 0.0;
  for (int i = threadIdx.x; i < count; i += kGradThreads) q += __ldcg(partials + i);
  return clip_of(block_sum(q, shared), max_norm);
}

template <class Args, bool kMore>
__global__ void __launch_bounds__(kGradThreads, kMore ? 3 : 4) k_grad_squares(const __grid_constant__ Args a, double *partials) {
  __shared__ double shared[kGradThreads / 32];
  dependency_wait();
  double q = 0.0;
  for (uint32_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const GradEntry &t = a.t[entry_of(a, chunk)];
    auto one = [&](float s, uint64_t) { q = fma((double)s, (double)s, q); };
    if (t.dtype == GS_TYPE_F32) chunk_sums<float, kMore>(a, t, chunk, [&](const float *s, uint64_t) { q += squares<4>(s); }, one);
    else if (t.dtype == GS_TYPE_F16) chunk_sums<__half, kMore>(a, t, chunk, [&](const float *s, uint64_t) { q += squares<8, !kMore>(s); }, one);   // (2^-48 to 2^32)
    else chunk_sums<__nv_bfloat16, kMore>(a, t, chunk, [&](const float *s, uint64_t) { q += squares<8>(s); }, one);
  }
  q = block_sum(q, shared);
  if (threadIdx.x == 0) partials[blockIdx.x] = q;
}

__global__ void __launch_bounds__(kGradThreads) k_grad_norm(const double *partials, int count, float max_norm, float *clip) {
  __shared__ double shared[kGradThreads / 32];
  dependency_wait();
  const Clip c = clip_from_partials(partials, count, max_norm, shared);
  if (threadIdx.x == 0) { clip[0] = c.norm; clip[1] = c.scale; }
}

template <class T, bool kMore, class Args>
__device__ __forceinline__ void scale_chunk(const Args &a, const GradEntry &t, uint32_t chunk, float scale) {
  constexpr int V = kVecOf<T>;
  T *out = static_cast<T *>(t.out);
  if (scale == 1.f && t.out == t.grad && t.num_more == 0) return;
  chunk_sums<T, kMore>(
      a, t, chunk,
      [&](float *s, uint64_t e) {
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = scale > 0.f ? s[i] * scale : 0.f;
        *reinterpret_cast<uint4 *>(out + e) = pack<T>(s);
      },
      [&](float s, uint64_t e) { out[e] = narrow<T>(scale > 0.f ? s * scale : 0.f); });
}
template <class Args, bool kMore>
__global__ void __launch_bounds__(kGradThreads, kMore ? 3 : 4) k_grad_scale(const __grid_constant__ Args a, const double *partials, int count, float max_norm,
                                                             float *clip) {
  __shared__ double shared[kGradThreads / 32];
  dependency_wait();
  const Clip c = clip_from_partials(partials, count, max_norm, shared);
  if (blockIdx.x == 0 && threadIdx.x == 0) { clip[0] = c.norm; clip[1] = c.scale; }
  // from the end on: what the norm has read last is in the L2
  for (uint32_t back = blockIdx.x; back < a.chunks; back += gridDim.x) {
    const uint32_t chunk = a.chunks - 1 - back;
    const GradEntry &t = a.t[entry_of(a, chunk)];
    if (t.dtype == GS_TYPE_F32) scale_chunk<float, kMore>(a, t, chunk, c.scale);
    else if (t.dtype == GS_TYPE_F16) scale_chunk<__half, kMore>(a, t, chunk, c.scale);
    else scale_chunk<__nv_bfloat16, kMore>(a, t, chunk, c.scale);
  }
}

template <class Args>
int run(const GsGradTensor *tensors, int num_tensors, bool scale, float max_norm, float *clip, double *partials, int num_sms, cudaStream_t st) {
  Args a;
  a.num_tensors = 0; a.chunks = 0;
  int more = 0;
  for (int i = 0; i < num_tensors; ++i) {
    const GsGradTensor &s = tensors[i];
    if (s.count == 0) continue;
    GradEntry &d = a.t[a.num_tensors++];
    d.grad = s.grad; d.out = scale ? s.out : nullptr; d.count = (uint64_t)s.count;
    d.chunk_start = a.chunks; d.more_start = (uint16_t)more; d.num_more = (uint8_t)s.num_more_grads; d.dtype = (uint8_t)s.dtype;
    const uintptr_t at = reinterpret_cast<uintptr_t>(s.grad) & 15u;
    bool same = !scale || (reinterpret_cast<uintptr_t>(s.out) & 15u) == at;
    for (int k = 0; k < s.num_more_grads; ++k) {
      a.more[more++] = s.more_grads[k];
      same = same && (reinterpret_cast<uintptr_t>(s.more_grads[k]) & 15u) == at;
    }
    const uint32_t size = s.dtype == GS_TYPE_F32 ? 4u : 2u;
    const uint64_t head = at ? (16u - at) / size : 0u;
    d.head = !same ? 0xffffffffu : (uint32_t)(head < d.count ? head : d.count);
    a.chunks += (uint32_t)((d.count + kGradChunk - 1) / kGradChunk);
  }
  const uint32_t wave = (uint32_t)num_sms * (more ? 3u : 4u), most = wave < (uint32_t)kGradPartials ? wave : (uint32_t)kGradPartials;
  const uint32_t grid = a.chunks < most ? (a.chunks ? a.chunks : 1u) : most;
  launch_chained(more ? k_grad_squares<Args, true> : k_grad_squares<Args, false>, grid, kGradThreads, 0, st, a, partials);
  if (scale) launch_chained(more ? k_grad_scale<Args, true> : k_grad_scale<Args, false>, grid, kGradThreads, 0, st, a, (const double *)partials, (int)grid, max_norm, clip);
  else launch_chained(k_grad_norm, 1, kGradThreads, 0, st, (const double *)partials, (int)grid, max_norm, clip);
  return 2;
}

}  // namespace

// Host side of gs_grad_norm (scale false) and gs_clip_grads: the C entry point has checked the arguments.
int launch_grad_clip(const GsGradTensor *tensors, int num_tensors, bool scale, float max_norm, float *clip, double *partials, int num_sms, cudaStream_t st) {
  int more = 0;
  for (int i = 0; i < num_tensors; ++i) more += tensors[i].num_more_grads;
  if (num_tensors <= 64 && more <= 128) return run<GradArgsSmall>(tensors, num_tensors, scale, max_norm, clip, partials, num_sms, st);
  return run<GradArgsLarge>(tensors, num_tensors, scale, max_norm, clip, partials, num_sms, st);
}

}  // namespace gs
