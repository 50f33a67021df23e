// Layer norm over the rows of a matrix, forward and backward.
//
//   mean, var of a row;  rstd = 1 / sqrt(var + eps);  h = (x - mean) rstd;  y = h gamma + beta
//   backward: g = dy gamma;  dx = rstd (g - avg(g) - h avg(g h));  dgamma = sum over rows of dy h;  dbeta = sum over rows of dy
//
// A pure stream: forward reads x and writes y once, backward reads x and dy and writes dx once, so HBM bounds it.  A row
// lives in the registers of a group of lanes (1 to 32 of a warp, or the 256 of a CTA), as the vectors of 16 bytes it was
// loaded in; the variance is taken about the mean in a second pass over the registers, which loses nothing where the mean is
// large against the spread.  All sums in fp32, two operations an instruction (add2 and the like): with one each the arithmetic
// was the bound (1M rows of 256 took 349 us forward, 432 backward; together with the row fetched ahead, the exchanges
// written out and running pointers 176 and 269, 90 and 88 % of the copy rate).  The grid is persistent: a lane keeps its columns from row to row, so
// gamma and beta stay in registers, and in the backward so do its sums for dgamma and dbeta, which leave as one row of partial
// sums per CTA and are added up by k_layer_norm_sums in a fixed order (no atomics: the same bits from run to run).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gs_device.cuh"

namespace gs {
namespace {

#include "gs_rows.cuh"

constexpr int kNormThreads = 256;
constexpr int kNormPartialRows = 960;     // most CTAs of the backward

// CTAs per SM, of as many registers as the elements of a lane need, and no more CTAs than are resident: 1M rows of 256 in bf16
// forward 189 us with three, 221 with four (spills), 308 with two; backward in fp16 282 with two, 324 with the compiler's choice.  (Some
// layouts spill at these counts: aligned ones up to 216 bytes a thread forward and 84 backward, both in fp32, unaligned ones of 32 elements
// a thread 252 and 128.)
__host__ __device__ constexpr int fwd_ctas(int elements) { return elements <= 4 ? 6 : elements <= 8 ? 4 : elements <= 16 ? 3 : 2; }
__host__ __device__ constexpr int bwd_ctas(int elements) { return elements <= 4 ? 4 : elements <= 8 ? 3 : elements <= 16 ? 2 : 1; }

// How a row is laid over lanes: `lanes` of them with NV vectors of V elements each, vector j of lane l at column (j lanes + l) V.
// V is a whole 16-byte vector, or 1 where rows are not aligned.
template <class T, int V, int NV>
struct Row {
  uint4 raw[V > 1 ? NV : 1];
  float one[V > 1 ? 1 : NV];
  // whole vectors; of the row's last one what is there (zero beyond)
  __device__ __forceinline__ void load(const T *p, int lane, int lanes, int cols, bool live) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * lanes + lane) * V;
      if constexpr (V > 1) {
        raw[j] = make_uint4(0u, 0u, 0u, 0u);
        if (live && c + V <= cols) raw[j] = __ldcs(reinterpret_cast<const uint4 *>(p + c));
        else if (live && c < cols) {
          float v[V];
#pragma unroll
          for (int i = 0; i < V; ++i) v[i] = c + i < cols ? widen(p[c + i]) : 0.f;
          raw[j] = pack<T>(v);
        }
      } else {
        one[j] = live && c < cols ? widen(p[c]) : 0.f;
      }
    }
  }
  __device__ __forceinline__ void get(float2 v[V * NV / 2]) const {
    if constexpr (V > 1) {
#pragma unroll
      for (int j = 0; j < NV; ++j) unpack<T>(raw[j], &v[j * V / 2].x);
    } else {
#pragma unroll
      for (int j = 0; j < NV / 2; ++j) v[j] = make_float2(one[2 * j], one[2 * j + 1]);
    }
  }
};
// A lane's values to where they belong.
template <class T, int V, int NV>
__device__ __forceinline__ void put(T *p, int lane, int lanes, int cols, const float2 v2[V * NV / 2]) {
  const float *v = &v2[0].x;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * lanes + lane) * V;
    if constexpr (V > 1) {
      if (c + V <= cols) { __stcs(reinterpret_cast<uint4 *>(p + c), pack<T>(v + j * V)); continue; }
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (c + i < cols) p[c + i] = narrow<T>(v[j * V + i]);
  }
}

// Sums over a group; the same in every lane.  (The steps are written out: a loop over them was a third of a row's instructions.)
template <bool kBlock>
__device__ __forceinline__ float2 group_sum2(float2 v, int lanes, float2 *shared) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (kBlock || lanes > o) v = add2(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
  if constexpr (kBlock) {
    __syncthreads();
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = shared[0];
#pragma unroll
    for (int w = 1; w < kNormThreads / 32; ++w) v = add2(v, shared[w]);
  }
  return v;
}
template <bool kBlock>
__device__ __forceinline__ float group_sum(float v, int lanes, float2 *shared) {
  if constexpr (kBlock) {
    return group_sum2<true>(make_float2(v, 0.f), lanes, shared).x;
  } else {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      if (lanes > o) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  }
}

// A lane's values of a parameter vector.
template <int V, int NV>
__device__ __forceinline__ void columns(const float *p, float fallback, int lane, int lanes, int cols, float2 out2[V * NV / 2]) {
  float *out = &out2[0].x;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (j * lanes + lane) * V + i;
      out[j * V + i] = p && c < cols ? __ldg(p + c) : fallback;
    }
}

// The next row is asked for before this one's sums are taken, where a row is short enough for the registers.
template <class T, int V, int NV, bool kBlock>
__global__ void __launch_bounds__(kNormThreads, fwd_ctas(V * NV)) k_layer_norm_fwd(LayerNormArgs a, int lanes) {
  __shared__ float2 shared[kNormThreads / 32];
  constexpr int P = V * NV / 2;
  dependency_wait();
  const int group = kBlock ? 0 : threadIdx.x / lanes, lane = kBlock ? threadIdx.x : threadIdx.x & (lanes - 1);
  const int groups = kBlock ? 1 : kNormThreads / lanes;
  float2 gamma[P], beta[P];
  columns<V, NV>(a.gamma, 1.f, lane, lanes, a.cols, gamma);
  columns<V, NV>(a.beta, 0.f, lane, lanes, a.cols, beta);
  const float inv = 1.f / (float)a.cols;
  const bool ragged = lanes * NV * V != a.cols;
  const int64_t step = (int64_t)gridDim.x * groups;
  int64_t row = (int64_t)blockIdx.x * groups + group;
  Row<T, V, NV> x;
  const T *from = static_cast<const T *>(a.x) + row * a.ld_x;
  T *to = static_cast<T *>(a.y) + row * a.ld_out;
  const int64_t from_step = step * a.ld_x, to_step = step * a.ld_out;
  x.load(from, lane, lanes, a.cols, row < a.rows);
  for (int64_t row0 = (int64_t)blockIdx.x * groups; row0 < a.rows; row0 += step, row += step, to += to_step) {
    float2 v[P];
    x.get(v);
    from += from_step;
    x.load(from, lane, lanes, a.cols, row + step < a.rows);
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < P; ++i) s = add2(s, v[i]);
    const float mean = group_sum<kBlock>(s.x + s.y, lanes, shared) * inv;
    s = make_float2(0.f, 0.f);
    const float2 minus = both(-mean);
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = add2(v[i], minus);
    if (ragged) {
#pragma unroll
      for (int e = 0; e < 2 * P; ++e)
        if (((e / V) * lanes + lane) * V + e % V >= a.cols) (&v[0].x)[e] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) s = fma2(v[i], v[i], s);
    const float rstd = rsqrtf(fmaf(group_sum<kBlock>(s.x + s.y, lanes, shared), inv, a.eps));
    if (row < a.rows) {
#pragma unroll
      for (int i = 0; i < P; ++i) v[i] = fma2(mul2(v[i], both(rstd)), gamma[i], beta[i]);
      put<T, V, NV>(to, lane, lanes, a.cols, v);
      if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
      }
    }
  }
}

template <class T, int V, int NV, bool kBlock, bool kParams>
__global__ void __launch_bounds__(kNormThreads, bwd_ctas(V * NV)) k_layer_norm_bwd(LayerNormArgs a, int lanes) {
  __shared__ float2 shared[kNormThreads / 32];
  constexpr int P = V * NV / 2;
  dependency_wait();
  const int group = kBlock ? 0 : threadIdx.x / lanes, lane = kBlock ? threadIdx.x : threadIdx.x & (lanes - 1);
  const int groups = kBlock ? 1 : kNormThreads / lanes;
  float2 gamma[P], sum_g[P], sum_b[P];
  columns<V, NV>(a.gamma, 1.f, lane, lanes, a.cols, gamma);
#pragma unroll
  for (int i = 0; i < P; ++i) sum_g[i] = sum_b[i] = make_float2(0.f, 0.f);
  const float inv = 1.f / (float)a.cols;
  const int64_t step = (int64_t)gridDim.x * groups;
  int64_t row = (int64_t)blockIdx.x * groups + group;
  Row<T, V, NV> x, dy;
  float mean, rstd;
  const T *from_x = static_cast<const T *>(a.x) + row * a.ld_x, *from_dy = static_cast<const T *>(a.dy) + row * a.ld_dy;
  T *to = a.dx ? static_cast<T *>(a.dx) + row * a.ld_out : nullptr;
  const int64_t x_step = step * a.ld_x, dy_step = step * a.ld_dy, to_step = a.dx ? step * a.ld_out : 0;
  auto fetch = [&](int64_t r) {
    const bool live = r < a.rows;
    x.load(from_x, lane, lanes, a.cols, live);
    dy.load(from_dy, lane, lanes, a.cols, live);
    from_x += x_step; from_dy += dy_step;
    mean = live ? __ldg(a.mean + r) : 0.f;
    rstd = live ? __ldg(a.rstd + r) : 0.f;
  };
  fetch(row);
  for (int64_t row0 = (int64_t)blockIdx.x * groups; row0 < a.rows; row0 += step, row += step, to += to_step) {
    float2 h[P], g[P];
    x.get(h);
    dy.get(g);
    const float2 minus = both(-mean), r = both(rstd);
    fetch(row + step);
    float2 s = make_float2(0.f, 0.f), t = s;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      // the sum of g h as rstd times that of g (x - mean): columns behind the row's end have g = 0 and x = 0, so their terms are 0 (their h
      // would be -mean rstd, which may be infinite)
      const float2 d = add2(h[i], minus);
      h[i] = mul2(d, r);
      if (kParams) {
        sum_g[i] = fma2(g[i], h[i], sum_g[i]);
        sum_b[i] = add2(sum_b[i], g[i]);
      }
      g[i] = mul2(g[i], gamma[i]);
      s = add2(s, g[i]);
      t = fma2(g[i], d, t);
    }
    const float2 sums = group_sum2<kBlock>(make_float2(s.x + s.y, (t.x + t.y) * r.x), lanes, shared);
    if (row < a.rows && a.dx) {
      const float2 avg_g = both(-sums.x * inv), avg_gh = both(-sums.y * inv);
#pragma unroll
      for (int i = 0; i < P; ++i) g[i] = mul2(add2(fma2(h[i], avg_gh, g[i]), avg_g), r);
      put<T, V, NV>(to, lane, lanes, a.cols, g);
    }
  }
  if constexpr (kParams) {
    // one row [2, cols] per CTA: the groups' sums of a column added in their order
    constexpr int E = 2 * P;
    const float *gs = &sum_g[0].x, *bs = &sum_b[0].x;
    float *out = a.partials + (size_t)blockIdx.x * 2 * a.cols;
    if constexpr (kBlock) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int c = ((e / V) * lanes + lane) * V + e % V;
        if (c < a.cols) { out[c] = gs[e]; out[a.cols + c] = bs[e]; }
      }
    } else {
      __shared__ float part[kNormThreads];
      // (sums of a warp's groups by shuffles, then of the warps through shared memory)
#pragma unroll
      for (int e = 0; e < 2 * E; ++e) {
        float v = e < E ? gs[e < E ? e : 0] : bs[e < E ? 0 : e - E];
        for (int o = lanes; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        __syncthreads();
        part[threadIdx.x] = v;
        __syncthreads();
        const int l = threadIdx.x, k = e % E;
        if (l < lanes) {
          float t = part[l];
#pragma unroll
          for (int w = 1; w < kNormThreads / 32; ++w) t += part[32 * w + l];
          const int c = ((k / V) * lanes + l) * V + k % V;
          if (c < a.cols) out[(e < E ? 0 : a.cols) + c] = t;
        }
      }
    }
  }
}

// Adds the CTAs' rows of partial sums: 32 columns per CTA, eight warps over the rows.
__global__ void __launch_bounds__(256) k_layer_norm_sums(const float *partials, int count, int cols, float *dgamma, float *dbeta) {
  __shared__ double part[8][32];
  dependency_wait();
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
  double s = 0.0;
  if (c < 2 * cols)
    for (int r = w; r < count; r += 8) s += (double)__ldcg(partials + (size_t)r * 2 * cols + c);
  part[w][threadIdx.x & 31] = s;
  __syncthreads();
  if (w == 0 && c < 2 * cols) {
    for (int k = 1; k < 8; ++k) s += part[k][threadIdx.x & 31];
    float *out = c < cols ? dgamma : dbeta;
    if (out) out[c < cols ? c : c - cols] = (float)s;
  }
}

// Rows per pass of a CTA and the layout over lanes for a number of vectors per row.
int lanes_for(int vectors, int nv) {
  int lanes = 1;
  while (lanes * nv < vectors) lanes *= 2;
  return lanes;
}

template <class T, int V, int NV, bool kBlock>
int fwd(const LayerNormArgs &a, int lanes, int num_sms, cudaStream_t st) {
  const int64_t groups = kBlock ? 1 : kNormThreads / lanes, want = (a.rows + groups - 1) / groups;
  const int64_t most = (int64_t)num_sms * fwd_ctas(V * NV);
  launch_chained(k_layer_norm_fwd<T, V, NV, kBlock>, (unsigned)(want < most ? want : most), kNormThreads, 0, st, a, lanes);
  return 1;
}
int bwd_grid(int64_t rows, int groups) {
  const int64_t want = (rows + groups - 1) / groups;
  return (int)(want < kNormPartialRows ? want : kNormPartialRows);
}
template <class T, int V, int NV, bool kBlock>
int bwd(const LayerNormArgs &a, int lanes, int num_sms, cudaStream_t st) {
  int grid = bwd_grid(a.rows, kBlock ? 1 : kNormThreads / lanes);
  const int most = num_sms * bwd_ctas(V * NV);
  if (grid > most) grid = most;
  if (!a.dgamma && !a.dbeta) {
    launch_chained(k_layer_norm_bwd<T, V, NV, kBlock, false>, grid, kNormThreads, 0, st, a, lanes);
    return 1;
  }
  launch_chained(k_layer_norm_bwd<T, V, NV, kBlock, true>, grid, kNormThreads, 0, st, a, lanes);
  launch_chained(k_layer_norm_sums, (2 * a.cols + 31) / 32, 256, 0, st, (const float *)a.partials, grid, a.cols, a.dgamma, a.dbeta);
  return 2;
}

bool vectors_fit(const void *p, int64_t ld, int64_t rows, int size) {
  return !p || ((reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows <= 1 || (ld * size) % 16 == 0));
}

template <class T>
int fwd_any(const LayerNormArgs &a, int num_sms, cudaStream_t st) {
  constexpr int V = kVecOf<T>;
  const bool vec = vectors_fit(a.x, a.ld_x, a.rows, sizeof(T)) && vectors_fit(a.y, a.ld_out, a.rows, sizeof(T));
  const int n = vec ? (a.cols + V - 1) / V : a.cols;
  if (vec) {
    constexpr int few = 16 / V, most = 32 / V;    // vectors of a lane that holds 16 or 32 elements
    // a row in a warp as long as it fits its registers (100 000 rows of 1024 in bf16 in a CTA's: 192 us), then in as few of a CTA's as it takes
    if (n <= 4) return fwd<T, V, 1, false>(a, lanes_for(n, 1), num_sms, st);
    if (n <= 32 * few) return fwd<T, V, few, false>(a, lanes_for(n, few), num_sms, st);
    if (n <= 32 * most) return fwd<T, V, most, false>(a, lanes_for(n, most), num_sms, st);
    if (n <= kNormThreads * few) return fwd<T, V, few, true>(a, kNormThreads, num_sms, st);
    return fwd<T, V, most, true>(a, kNormThreads, num_sms, st);
  }
  if (n <= 4) return fwd<T, 1, 2, false>(a, lanes_for(n, 2), num_sms, st);
  if (n <= 128) return fwd<T, 1, 4, false>(a, lanes_for(n, 4), num_sms, st);
  if (n <= 2048) return fwd<T, 1, 8, true>(a, kNormThreads, num_sms, st);
  return fwd<T, 1, 32, true>(a, kNormThreads, num_sms, st);
}
template <class T>
int bwd_any(const LayerNormArgs &a, int num_sms, cudaStream_t st) {
  constexpr int V = kVecOf<T>;
  const bool vec = vectors_fit(a.x, a.ld_x, a.rows, sizeof(T)) && vectors_fit(a.dy, a.ld_dy, a.rows, sizeof(T)) &&
                   vectors_fit(a.dx, a.ld_out, a.rows, sizeof(T));
  const int n = vec ? (a.cols + V - 1) / V : a.cols;
  if (vec) {
    constexpr int few = 16 / V, most = 32 / V;    // vectors of a lane that holds 16 or 32 elements
    if (n <= 4) return bwd<T, V, 1, false>(a, lanes_for(n, 1), num_sms, st);
    if (n <= 32 * few) return bwd<T, V, few, false>(a, lanes_for(n, few), num_sms, st);
    if (n <= 32 * most) return bwd<T, V, most, false>(a, lanes_for(n, most), num_sms, st);
    if (n <= kNormThreads * few) return bwd<T, V, few, true>(a, kNormThreads, num_sms, st);
    return bwd<T, V, most, true>(a, kNormThreads, num_sms, st);
  }
  if (n <= 4) return bwd<T, 1, 2, false>(a, lanes_for(n, 2), num_sms, st);
  if (n <= 128) return bwd<T, 1, 4, false>(a, lanes_for(n, 4), num_sms, st);
  if (n <= 2048) return bwd<T, 1, 8, true>(a, kNormThreads, num_sms, st);
  return bwd<T, 1, 32, true>(a, kNormThreads, num_sms, st);
}

}  // namespace

size_t layer_norm_partials(int64_t rows, int cols) { return (size_t)(rows < kNormPartialRows ? rows : kNormPartialRows) * 2 * (size_t)cols; }

int launch_layer_norm_fwd(const LayerNormArgs &a, int num_sms, cudaStream_t st) {
  if (a.dtype == GS_TYPE_F32) return fwd_any<float>(a, num_sms, st);
  if (a.dtype == GS_TYPE_F16) return fwd_any<__half>(a, num_sms, st);
  return fwd_any<__nv_bfloat16>(a, num_sms, st);
}
int launch_layer_norm_bwd(const LayerNormArgs &a, int num_sms, cudaStream_t st) {
  if (a.dtype == GS_TYPE_F32) return bwd_any<float>(a, num_sms, st);
  if (a.dtype == GS_TYPE_F16) return bwd_any<__half>(a, num_sms, st);
  return bwd_any<__nv_bfloat16>(a, num_sms, st);
}

}  // namespace gs
