// Norm of many tensors, clipping by it, and the Adam update.
#include "row_io.h"
#include "update.h"

namespace aecct {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ double block_sum(double v, double *lds) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
  __syncthreads();
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) v += lds[w];
  return v;
}

// The tensor of unit u, from that of an earlier unit.
template <int N>
__device__ __forceinline__ int tensor_of(const Units<N> &t, int u, int k) {
  if (u < t.unit0[k + 1]) return k;
  int lo = k + 1, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (t.unit0[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Four values of any type; n of them are there.
__device__ __forceinline__ void load4(const void *p, int type, int64_t i, int64_t n, float (&f)[4]) {
  const int k = n >= 4 ? 4 : (int)n;
  if (type == 0) load_part<float, 4>((const float *)p + i, k, f);
  else if (type == 1) load_part<bf16_t, 4>((const bf16_t *)p + i, k, f);
  else load_part<f16_t, 4>((const f16_t *)p + i, k, f);
}
__device__ __forceinline__ void store4(void *p, int type, int64_t i, int64_t n, const float (&f)[4]) {
  const int k = n >= 4 ? 4 : (int)n;
  if (type == 0) store_part<float, 4>((float *)p + i, k, f);
  else if (type == 1) store_part<bf16_t, 4>((bf16_t *)p + i, k, f);
  else store_part<f16_t, 4>((f16_t *)p + i, k, f);
}

constexpr int kSteps = kUnit / (4 * kThreads);   // of four values a thread in a unit

// Sum of squares of a unit's values from i0 on, n in all: 16 bytes a load.
template <class T>
__device__ __forceinline__ double unit_squares(const T *g, int64_t n) {
  constexpr int V = 16 / sizeof(T), J = kUnit / (V * kThreads);
  float f[J][V];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int i = (j * kThreads + (int)threadIdx.x) * V;
    load_part<T, V>(g + i, n - i >= V ? V : (int)(n - i), f[j]);
  }
  double s = 0, q = 0;
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      s += (double)f[j][i] * (double)f[j][i];
      q += (double)f[j][i + 1] * (double)f[j][i + 1];
    }
  return s + q;
}

template <int N>
__global__ __launch_bounds__(kThreads) void k_sum_squares(SumTable<N> t, double *part, const int64_t *step, int64_t *next) {
  __shared__ double lds[kThreads / 64];
  if (step && blockIdx.x == 0 && threadIdx.x == 0) *next = *step + 1;
  double s = 0;
  int k = 0;
  for (int u = blockIdx.x; u < t.unit0[t.n]; u += gridDim.x) {
    k = tensor_of(t, u, k);
    const int64_t i0 = (int64_t)(u - t.unit0[k]) * kUnit, n = t.count[k] - i0;
    if (t.type[k] == 0) s += unit_squares((const float *)t.g[k] + i0, n);
    else if (t.type[k] == 1) s += unit_squares((const bf16_t *)t.g[k] + i0, n);
    else s += unit_squares((const f16_t *)t.g[k] + i0, n);
  }
  s = block_sum(s, lds);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The norm from the blocks' sums; every block that asks gets the same bits.
__device__ __forceinline__ double norm_of(const double *part, int parts, double *lds) {
  double s = 0;
  for (int i = threadIdx.x; i < parts; i += 8 * kThreads) {   // eight loads in flight: this is all latency
    double v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = i + j * kThreads < parts ? part[i + j * kThreads] : 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) s += v[j];
  }
  return sqrt(block_sum(s, lds));
}

__global__ __launch_bounds__(kThreads) void k_norm(const double *part, int parts, float *norm) {
  __shared__ double lds[kThreads / 64];
  const double n = norm_of(part, parts, lds);
  if (threadIdx.x == 0) *norm = (float)n;
}

// min(1, max_norm / norm), and 1 for a norm that is not finite
__device__ __forceinline__ float clip_factor(double norm, double max_norm) {
  return norm > max_norm && norm <= 1.7976931348623157e308 ? (float)(max_norm / norm) : 1.0f;
}

template <int N>
__global__ __launch_bounds__(kThreads) void k_clip(ClipTable<N> t, const double *part, int parts, double max_norm, float *norm) {
  __shared__ double lds[kThreads / 64];
  const double n = norm_of(part, parts, lds);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
  const float f = clip_factor(n, max_norm);
  int k = 0;
  for (int u = blockIdx.x; u < t.unit0[t.n]; u += gridDim.x) {
    k = tensor_of(t, u, k);
    const int64_t i0 = (int64_t)(u - t.unit0[k]) * kUnit + 4 * threadIdx.x, c = t.count[k];
    float g[kSteps][4];
#pragma unroll
    for (int j = 0; j < kSteps; ++j) load4(t.g[k], t.type[k], i0 + 4 * kThreads * j, c - i0 - 4 * kThreads * j, g[j]);
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) g[j][i] *= f;
      store4(t.out[k], t.out_type[k], i0 + 4 * kThreads * j, c - i0 - 4 * kThreads * j, g[j]);
    }
  }
}

__global__ void k_next_step(const int64_t *step, int64_t *next) { *next = *step + 1; }

template <int N>
__global__ __launch_bounds__(kThreads) void k_adam(AdamTable<N> t, const double *part, int parts, AdamScalars o,
                                                   const int64_t *next, int64_t *step, float *norm) {
  __shared__ double lds[kThreads / 64];
  float f = 1.0f;
  if (parts) {
    const double n = norm_of(part, parts, lds);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    if (!(n <= 1.7976931348623157e308)) return;
    if (o.max_norm > 0) f = clip_factor(n, o.max_norm);
  }
  const int64_t now = *next;
  if (step && blockIdx.x == 0 && threadIdx.x == 0) *step = now;
  const double lr = o.lr_device ? (double)*o.lr_device : o.lr;
  const float size = (float)(lr / (1 - pow(o.beta1, (double)now))), root = (float)(1 / sqrt(1 - pow(o.beta2, (double)now)));
  const float b1 = (float)o.beta1, c1 = (float)(1 - o.beta1), b2 = (float)o.beta2, c2 = (float)(1 - o.beta2);
  const float decay = (float)(lr * o.weight_decay), eps = (float)o.eps;
  int k = 0;
  for (int u = blockIdx.x; u < t.unit0[t.n]; u += gridDim.x) {
    k = tensor_of(t, u, k);
    const int64_t i0 = (int64_t)(u - t.unit0[k]) * kUnit + 4 * threadIdx.x, c = t.count[k];
#pragma unroll 2
    for (int j = 0; j < kSteps; ++j) {
      const int64_t at = i0 + 4 * kThreads * j, left = c - at;
      const int n = left >= 4 ? 4 : (int)left;
      float g[4], p[4], m[4], v[4];
      load4(t.g[k], t.type[k], at, left, g);
      load_part<float, 4>(t.p[k] + at, n, p);
      load_part<float, 4>(t.m[k] + at, n, m);
      load_part<float, 4>(t.v[k] + at, n, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = g[i] * f;
        m[i] = fmaf(b1, m[i], c1 * x);
        v[i] = fmaf(b2, v[i], c2 * (x * x));
        p[i] -= fmaf(decay, p[i], size * m[i] / fmaf(sqrtf(v[i]), root, eps));
      }
      store_part<float, 4>(t.m[k] + at, n, m);
      store_part<float, 4>(t.v[k] + at, n, v);
      store_part<float, 4>(t.p[k] + at, n, p);
      if (t.copy[k]) store4(t.copy[k], t.copy_type[k], at, left, p);
    }
  }
}

int grid_of(int units, int most) { return units < 1 ? 1 : units < most ? units : most; }

// The shorter form of a table of at most kFew ranges.
template <int N>
void few(const Units<N> &t, Units<kFew> &f) {
  f.n = t.n;
  for (int i = 0; i <= t.n; ++i) f.unit0[i] = t.unit0[i];
  for (int i = 0; i < t.n; ++i) {
    f.count[i] = t.count[i];
    f.type[i] = t.type[i];
  }
}

}  // namespace

hipError_t launch_sum_squares(const SumTable<kSumRanges> &t, double *part, int blocks, const int64_t *step, int64_t *next,
                              hipStream_t s) {
  if (t.n <= kFew) {
    SumTable<kFew> f;
    few(t, f);
    for (int i = 0; i < t.n; ++i) f.g[i] = t.g[i];
    k_sum_squares<<<blocks, kThreads, 0, s>>>(f, part, step, next);
  } else {
    k_sum_squares<<<blocks, kThreads, 0, s>>>(t, part, step, next);
  }
  return hipGetLastError();
}
hipError_t launch_norm(const double *part, int parts, float *norm, hipStream_t s) {
  k_norm<<<1, kThreads, 0, s>>>(part, parts, norm);
  return hipGetLastError();
}
hipError_t launch_clip(const ClipTable<kClipRanges> &t, const double *part, int parts, double max_norm, float *norm,
                       int cu_count, hipStream_t s) {
  const int grid = grid_of(t.unit0[t.n], 8 * cu_count);
  if (t.n <= kFew) {
    ClipTable<kFew> f;
    few(t, f);
    for (int i = 0; i < t.n; ++i) {
      f.g[i] = t.g[i];
      f.out[i] = t.out[i];
      f.out_type[i] = t.out_type[i];
    }
    k_clip<<<grid, kThreads, 0, s>>>(f, part, parts, max_norm, norm);
  } else {
    k_clip<<<grid, kThreads, 0, s>>>(t, part, parts, max_norm, norm);
  }
  return hipGetLastError();
}
hipError_t launch_next_step(const int64_t *step, int64_t *next, hipStream_t s) {
  k_next_step<<<1, 1, 0, s>>>(step, next);
  return hipGetLastError();
}
hipError_t launch_adam(const AdamTable<kAdamRanges> &t, const double *part, int parts, const AdamScalars &o,
                       const int64_t *next, int64_t *step, float *norm, int cu_count, hipStream_t s) {
  const int grid = grid_of(t.unit0[t.n], 8 * cu_count);
  if (t.n <= kFew) {
    AdamTable<kFew> f;
    few(t, f);
    for (int i = 0; i < t.n; ++i) {
      f.g[i] = t.g[i];
      f.p[i] = t.p[i];
      f.m[i] = t.m[i];
      f.v[i] = t.v[i];
      f.copy[i] = t.copy[i];
      f.copy_type[i] = t.copy_type[i];
    }
    k_adam<<<grid, kThreads, 0, s>>>(f, part, parts, o, next, step, norm);
  } else {
    k_adam<<<grid, kThreads, 0, s>>>(t, part, parts, o, next, step, norm);
  }
  return hipGetLastError();
}

}  // namespace aecct
