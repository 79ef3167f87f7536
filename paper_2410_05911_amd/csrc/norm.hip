// Root-mean-square norm of rows with the residual's addition and Eq. 2 codes, and its gradient.
#include "device_common.h"
#include "norm.h"
#include "row_io.h"

namespace aecct {
namespace {

constexpr int kWaves = 16;
constexpr int kThreads = 64 * kWaves;   // one block a row

struct SumOp {
  template <class S>
  static __device__ __forceinline__ S join(S a, S b) { return a + b; }
};
struct MaxOp {
  static __device__ __forceinline__ uint32_t join(uint32_t a, uint32_t b) { return max(a, b); }
};

// Joins v over the block in a fixed order; every thread gets the result.
template <class Op, class S>
__device__ __forceinline__ S block_join(S v, S *lds) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) v = Op::join(v, __shfl_xor(v, m));
  __syncthreads();
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) v = Op::join(v, lds[w]);
  return v;
}

// rho = 1 / sqrt(mean(h^2) + eps) from the fp32 sum of squares ss.  Where that sum overflowed, or is so small that
// squares were lost below fp32's range, h is scaled by a power of two, `unit`, and summed again; rho is then that of the
// scaled row (h rho is the same) and 1 / sqrt(mean(h^2) + eps) = rho unit.
template <int N>
__device__ __forceinline__ float row_rho(float ss, float (&h)[N], int d, float eps, float &unit, float *lds) {
  unit = 1.0f;
  if (ss >= 1e-24f && ss <= 1e37f) return 1.0f / sqrtf(ss / (float)d + eps);
  unit = ss < 1.0f ? 0x1p100f : 0x1p-100f;
  ss = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    h[i] *= unit;
    ss = fmaf(h[i], h[i], ss);
  }
  ss = block_join<SumOp>(ss, lds);
  return (float)(1.0 / sqrt((double)ss / d + (double)eps * unit * unit));
}

template <class T>
__device__ __forceinline__ float load_gain(const void *gain, bool f32, int c) {
  return f32 ? ((const float *)gain)[c] : (float)((const T *)gain)[c];
}

// Q / alpha for values scaled by `up`, a power of two that keeps the quotient finite for the smallest alphas.
__device__ __forceinline__ float code_scale(float alpha, float most, float &up) {
  up = alpha < 0x1p-60f ? 0x1p60f : 1.0f;
  return alpha == 0.0f ? 0.0f : most / (alpha * up);
}
__device__ __forceinline__ uint8_t code_of(float y, float q, float alpha, int code) {
  if (code == 1) return alpha == alpha ? (uint8_t)quant_bits(y, q) : 0;
  return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(y * q, y * q, 0, false);
}

// A row a block; thread t holds columns t, t + 1024, ...
template <class T, int N>
__global__ __launch_bounds__(kThreads) void k_rms_norm(NormRows a) {
  __shared__ float lds4[kWaves];
  __shared__ uint32_t lmax[65536 / 32];
  const int t = threadIdx.x;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *x = (const T *)a.x + r * a.ldx, *res = (const T *)a.res + r * a.ldres;
    float h[N];
    float ss = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = t + i * kThreads;
      h[i] = c < a.d ? (float)x[c] + (a.res ? (float)res[c] : 0.0f) : 0.0f;
      if (a.h && c < a.d) ((T *)a.h)[r * a.ldh + c] = (T)h[i];
      ss = fmaf(h[i], h[i], ss);
    }
    float unit;
    const float rho = row_rho(block_join<SumOp>(ss, lds4), h, a.d, a.eps, unit, lds4);
    for (int k = t; k < a.alphas; k += kThreads) lmax[k] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = t + i * kThreads;
      if (c < a.d) {
        h[i] = h[i] * rho;
        if (a.gain) h[i] *= load_gain<T>(a.gain, a.gain_f32, c);
        if (a.y) ((T *)a.y)[r * a.ldy + c] = (T)h[i];
        if (a.code) atomicMax(&lmax[c / a.group], __builtin_bit_cast(uint32_t, fabsf(h[i])));
      }
    }
    if (!a.code) continue;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = t + i * kThreads;
      if (c < a.d) {
        const float alpha = __builtin_bit_cast(float, lmax[c / a.group]);
        float up;
        const float q = code_scale(alpha, a.code == 1 ? 127.0f : 448.0f, up);
        a.codes[r * a.ldcodes + c] = code_of(h[i] * up, q, alpha, a.code);
        if (c % a.group == 0) a.alpha[r * a.alphas + c / a.group] = alpha;
      }
    }
    __syncthreads();
  }
}

// The gradient, a row a block; block b sums its rows' dy xh per column and leaves it in part[b].
template <class T, int N>
__global__ __launch_bounds__(kThreads) void k_rms_norm_grad(NormGradRows a) {
  __shared__ float lds4[kWaves];
  const int t = threadIdx.x;
  float dg[N];
#pragma unroll
  for (int i = 0; i < N; ++i) dg[i] = 0;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *h = (const T *)a.h + r * a.ldh, *dy = (const T *)a.dy + r * a.lddy;
    const T *dres = (const T *)a.dres + r * a.lddres;
    float x[N], g[N];
    float ss = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = t + i * kThreads;
      x[i] = c < a.d ? (float)h[c] : 0.0f;
      g[i] = c < a.d ? (float)dy[c] : 0.0f;
      ss = fmaf(x[i], x[i], ss);
    }
    float unit;
    const float rho = row_rho(block_join<SumOp>(ss, lds4), x, a.d, a.eps, unit, lds4), rho1 = rho * unit;
    float dot = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = t + i * kThreads;
      x[i] *= rho;
      dg[i] = fmaf(g[i], x[i], dg[i]);
      if (c < a.d && a.gain) g[i] *= load_gain<T>(a.gain, a.gain_f32, c);
      dot = fmaf(g[i], x[i], dot);
    }
    const float m = block_join<SumOp>(dot, lds4) / (float)a.d;
    if (!a.dh) continue;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = t + i * kThreads;
      if (c < a.d) ((T *)a.dh)[r * a.lddh + c] = (T)(rho1 * fmaf(-m, x[i], g[i]) + (a.dres ? (float)dres[c] : 0.0f));
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = t + i * kThreads;
    if (c < a.d) a.part[(int64_t)blockIdx.x * a.d + c] = dg[i];
  }
}

// dgain[c] = the sum of `rows` partial rows, in ascending order.
__global__ void k_rms_norm_dgain(const float *part, int rows, int d, float *dgain) {
  const int c = blockIdx.x * 64 + threadIdx.x;
  if (c >= d) return;
  float s = 0;
  for (int r = 0; r < rows; ++r) s += part[(int64_t)r * d + c];
  dgain[c] = s;
}

template <class T>
hipError_t norm_type(const NormRows &a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.rows < (1 << 20) ? a.rows : (1 << 20));
  const int n = (a.d + kThreads - 1) / kThreads;
  if (n <= 1) k_rms_norm<T, 1><<<grid, kThreads, 0, s>>>(a);
  else if (n <= 4) k_rms_norm<T, 4><<<grid, kThreads, 0, s>>>(a);
  else if (n <= 16) k_rms_norm<T, 16><<<grid, kThreads, 0, s>>>(a);
  else k_rms_norm<T, 64><<<grid, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

template <class T>
hipError_t grad_type(const NormGradRows &a, hipStream_t s) {
  const int64_t blocks = norm_grad_part_rows(a.rows, a.d);
  const unsigned grid = (unsigned)blocks;
  const int n = (a.d + kThreads - 1) / kThreads;
  if (grid) {
    if (n <= 1) k_rms_norm_grad<T, 1><<<grid, kThreads, 0, s>>>(a);
    else if (n <= 4) k_rms_norm_grad<T, 4><<<grid, kThreads, 0, s>>>(a);
    else if (n <= 16) k_rms_norm_grad<T, 16><<<grid, kThreads, 0, s>>>(a);
    else k_rms_norm_grad<T, 64><<<grid, kThreads, 0, s>>>(a);
  }
  if (a.part) k_rms_norm_dgain<<<(a.d + 63) / 64, 64, 0, s>>>(a.part, (int)grid, a.d, a.dgain);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rms_norm(int type, const NormRows &a, int cu_count, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  return type == 0 ? norm_type<float>(a, s) : type == 1 ? norm_type<bf16_t>(a, s) : norm_type<f16_t>(a, s);
}

int64_t norm_grad_part_rows(int64_t rows, int d) { return rows < 512 ? rows : 512; }

hipError_t launch_rms_norm_grad(int type, const NormGradRows &a, int cu_count, hipStream_t s) {
  return type == 0 ? grad_type<float>(a, s) : type == 1 ? grad_type<bf16_t>(a, s) : grad_type<f16_t>(a, s);
}

}  // namespace aecct
