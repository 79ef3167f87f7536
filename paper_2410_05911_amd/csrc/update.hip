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

// The tensor that unit u belongs to.
template <int N>
__device__ __forceinline__ int tensor_of(const Units<N> &t, int u) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (t.unit0[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ float load_typed(const void *p, int type, int64_t i) {
  return type == 0 ? ((const float *)p)[i] : type == 1 ? (float)((const bf16_t *)p)[i] : (float)((const f16_t *)p)[i];
}
__device__ __forceinline__ void store_typed(void *p, int type, int64_t i, float v) {
  if (type == 0) ((float *)p)[i] = v;
  else if (type == 1) ((bf16_t *)p)[i] = (bf16_t)v;
  else ((f16_t *)p)[i] = (f16_t)v;
}

__global__ __launch_bounds__(kThreads) void k_sum_squares(SumTable t, double *part) {
  __shared__ double lds[kThreads / 64];
  double s = 0;
  for (int u = blockIdx.x; u < t.unit0[t.n]; u += gridDim.x) {
    const int k = tensor_of(t, u);
    const int64_t i0 = (int64_t)(u - t.unit0[k]) * kUnit, n = t.count[k];
    for (int64_t i = i0 + threadIdx.x; i < i0 + kUnit && i < n; i += kThreads) {
      const double g = load_typed(t.g[k], t.type[k], i);
      s += g * g;
    }
  }
  s = block_sum(s, lds);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The norm from the blocks' sums; every block that asks gets the same bits.
__device__ __forceinline__ double norm_of(const double *part, int parts, double *lds) {
  double s = 0;
  for (int i = threadIdx.x; i < parts; i += kThreads) s += part[i];
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

__global__ __launch_bounds__(kThreads) void k_clip(ClipTable t, const double *part, int parts, double max_norm, float *norm) {
  __shared__ double lds[kThreads / 64];
  const double n = norm_of(part, parts, lds);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
  const float f = clip_factor(n, max_norm);
  for (int u = blockIdx.x; u < t.unit0[t.n]; u += gridDim.x) {
    const int k = tensor_of(t, u);
    const int64_t i0 = (int64_t)(u - t.unit0[k]) * kUnit, c = t.count[k];
    for (int64_t i = i0 + threadIdx.x; i < i0 + kUnit && i < c; i += kThreads)
      store_typed(t.out[k], t.out_type[k], i, load_typed(t.g[k], t.type[k], i) * f);
  }
}

__global__ void k_next_step(const int64_t *step, int64_t *next) { *next = *step + 1; }

__global__ __launch_bounds__(kThreads) void k_adam(AdamTable t, const double *part, int parts, AdamScalars o,
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
  for (int u = blockIdx.x; u < t.unit0[t.n]; u += gridDim.x) {
    const int k = tensor_of(t, u);
    const int64_t i0 = (int64_t)(u - t.unit0[k]) * kUnit, c = t.count[k];
    for (int64_t i = i0 + threadIdx.x; i < i0 + kUnit && i < c; i += kThreads) {
      const float g = load_typed(t.g[k], t.type[k], i) * f;
      const float m = fmaf(b1, t.m[k][i], c1 * g), v = fmaf(b2, t.v[k][i], c2 * (g * g));
      const float p0 = t.p[k][i];
      const float p = p0 - fmaf(decay, p0, size * m / fmaf(sqrtf(v), root, eps));
      t.m[k][i] = m;
      t.v[k][i] = v;
      t.p[k][i] = p;
      if (t.copy[k]) store_typed(t.copy[k], t.copy_type[k], i, p);
    }
  }
}

int grid_of(int units, int most) { return units < 1 ? 1 : units < most ? units : most; }

}  // namespace

hipError_t launch_sum_squares(const SumTable &t, double *part, int blocks, hipStream_t s) {
  k_sum_squares<<<blocks, kThreads, 0, s>>>(t, part);
  return hipGetLastError();
}
hipError_t launch_norm(const double *part, int parts, float *norm, hipStream_t s) {
  k_norm<<<1, kThreads, 0, s>>>(part, parts, norm);
  return hipGetLastError();
}
hipError_t launch_clip(const ClipTable &t, const double *part, int parts, double max_norm, float *norm, int cu_count,
                       hipStream_t s) {
  k_clip<<<grid_of(t.unit0[t.n], 8 * cu_count), kThreads, 0, s>>>(t, part, parts, max_norm, norm);
  return hipGetLastError();
}
hipError_t launch_next_step(const int64_t *step, int64_t *next, hipStream_t s) {
  k_next_step<<<1, 1, 0, s>>>(step, next);
  return hipGetLastError();
}
hipError_t launch_adam(const AdamTable &t, const double *part, int parts, const AdamScalars &o, const int64_t *next,
                       int64_t *step, float *norm, int cu_count, hipStream_t s) {
  k_adam<<<grid_of(t.unit0[t.n], 8 * cu_count), kThreads, 0, s>>>(t, part, parts, o, next, step, norm);
  return hipGetLastError();
}

}  // namespace aecct
