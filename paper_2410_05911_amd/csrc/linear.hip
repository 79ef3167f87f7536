// Linear maps: which tile and how many splits a product takes, and what its gradient needs besides products.
#include "gemm.h"

namespace aecct {

GemmPlan plan_gemm(int type, int64_t m, int64_t n, int64_t k, bool across_a, bool across_b, int64_t ldb) {
  GemmPlan p{false, 1, 1, 0};
  const int64_t size = type == AECCT_F32 ? 4 : type == kCodeType + AECCT_CODE_I8 ? 1 : 2;   // of a value in LDS
  if (m <= kFewRows && !across_a && ldb < (int64_t)1 << 30) {
    p.few = true;
    const int64_t t = (n + 63) / 64, rounds = (k + kFewRound - 1) / kFewRound;
    // Weights of less than 4 MB are read in less time than a second launch takes.
    if (across_b && m > 0 && t < 512 && n * k * size >= ((int64_t)4 << 20)) {
      p.splits = (int)(1024 / t < rounds ? 1024 / t : rounds);
      if (p.splits > 16) p.splits = 16;
      if (p.splits > 1) p.part_bytes = (size_t)(p.splits * m * n * 4);
    }
    return p;
  }
  auto tiles = [&](int t) { return (m + kTileSide[t][0] - 1) / kTileSide[t][0] * ((n + kTileSide[t][1] - 1) / kTileSide[t][1]); };
  if (tiles(1) < 192) p.tile = 0;
  else if (tiles(2) >= 256 && k * size >= 1024) p.tile = 2;
  const int64_t t = tiles(p.tile), kt = (k * size + 127) / 128;
  if (t > 0 && t < 256) {
    int64_t s = (512 + t - 1) / t;
    if (s > kt / 4) s = kt / 4;
    if (s > 64) s = 64;
    p.splits = s > 1 ? (int)s : 1;
  }
  if (p.splits > 1) p.part_bytes = (size_t)(p.splits * m * n * 4);
  return p;
}

hipError_t launch_gemm(int type, const Gemm &g, const GemmPlan &plan, hipStream_t s) {
  if (g.m == 0 || g.n == 0) return hipSuccess;
  switch (type) {
    case AECCT_F32: return launch_gemm_f32(g, plan, s);
    case AECCT_BF16: return launch_gemm_bf16(g, plan, s);
    case AECCT_F16: return launch_gemm_f16(g, plan, s);
    case kCodeType + AECCT_CODE_I8: return launch_gemm_i8(g, plan, s);
    case kCodeType + AECCT_CODE_E4M3: return launch_gemm_e4m3(g, plan, s);
    default: return hipErrorInvalidValue;
  }
}

namespace {

// act'(z).  Where a factor is 0 the other may be infinite: such a product's limit is 0.
__device__ __forceinline__ float slope(float z, int act, bool f32) {
  if (act == kActRelu) return z > 0.0f ? 1.0f : z != z ? z : 0.0f;
  if (act == kActGelu) {
    float e;
    const float phi = normal(z, e), density = e * 0.39894228040143268f;
    return (f32 ? 0.5f * (1.0f + erff(z * 0.70710678118654752f)) : phi) + (density == 0.0f ? 0.0f : z * density);
  }
  const float p = logistic(z), q = logistic(-z);   // q = 1 - p
  if (p == 0.0f || q == 0.0f) return p;
  return p * (1.0f + z * q);
}

constexpr int kSlopeColumns = 128;   // 16 threads of 8 values a row, 16 rows at once

template <class T>
__global__ __launch_bounds__(256) void k_slope(Slope a) {
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * kSlopeColumns + c * 8;
  const int count = a.n - n0 < 8 ? (int)(a.n - n0) : 8;
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (count > 0) {
    for (int64_t row = (int64_t)blockIdx.y * 16 + r; row < a.rows; row += (int64_t)gridDim.y * 16) {
      float d[8];
      load_part<T, 8>((const T *)a.dy + row * a.lddy + n0, count, d);
      if (a.z) {
        float z[8];
        load_part<T, 8>((const T *)a.z + row * a.ldz + n0, count, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] *= slope(z[i], a.act, sizeof(T) == 4);
        if (a.dz) store_part<T, 8>((T *)a.dz + row * a.lddz + n0, count, d);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += d[i];
    }
  }
  if (!a.part) return;
  __shared__ float s[16][kSlopeColumns + 4];
#pragma unroll
  for (int i = 0; i < 8; ++i) s[r][c * 8 + i] = sum[i];
  __syncthreads();
  if (threadIdx.x < kSlopeColumns) {
    const int64_t n = (int64_t)blockIdx.x * kSlopeColumns + threadIdx.x;
    float t = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += s[i][threadIdx.x];
    if (n < a.n) a.part[(int64_t)blockIdx.y * a.n + n] = t;
  }
}

// 16 columns a block, 16 threads each.
__global__ __launch_bounds__(256) void k_column_sum(const float *part, int64_t blocks, int64_t n, float *out) {
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int64_t at = (int64_t)blockIdx.x * 16 + c;
  float t = 0;
  if (at < n)
    for (int64_t b = r; b < blocks; b += 16) t += part[b * n + at];
  __shared__ float s[16][17];
  s[r][c] = t;
  __syncthreads();
  if (r || at >= n) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) t += s[i][c];
  out[at] = t;
}

}  // namespace

int64_t slope_blocks(int64_t rows, int64_t n) {
  const int64_t across = (n + kSlopeColumns - 1) / kSlopeColumns;
  int64_t b = (1024 + across - 1) / across;
  const int64_t most = (rows + 15) / 16;
  if (b > most) b = most;
  return b < 1 ? 1 : b;
}

hipError_t launch_slope(int type, const Slope &a, hipStream_t s) {
  const int64_t blocks = slope_blocks(a.rows, a.n);
  const dim3 grid((unsigned)((a.n + kSlopeColumns - 1) / kSlopeColumns), (unsigned)blocks);
  switch (type) {
    case AECCT_F32: k_slope<float><<<grid, 256, 0, s>>>(a); break;
    case AECCT_BF16: k_slope<bf16_t><<<grid, 256, 0, s>>>(a); break;
    case AECCT_F16: k_slope<f16_t><<<grid, 256, 0, s>>>(a); break;
    default: return hipErrorInvalidValue;
  }
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || !a.part) return err;
  k_column_sum<<<dim3((unsigned)((a.n + 15) / 16)), 256, 0, s>>>(a.part, blocks, a.n, a.dbias);
  return hipGetLastError();
}

}  // namespace aecct
