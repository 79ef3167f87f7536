// Linear maps with an epilogue and their gradients: what linear_host.cpp hands to the kernels.
#pragma once

#include <cstddef>
#include <cstdint>

#include <hip/hip_runtime.h>

namespace aecct {

enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };

// out[m][n] = sum over k of a(m, k) b(n, k).  Strides in values.  A factor lies along k (value (row, k) at row ld + k) or
// across k (at k ld + row).
struct Factor {
  const void *p;
  int64_t ld;
  bool across;
};
// What becomes of a sum: v = sum alpha[m] / q scale[n] + bias[n], z = v, y = act(v) + res.
struct Epilogue {
  const float *alpha, *scale, *bias;   // or null
  float per_q;                         // 1 / q
  int act;
  int type;                            // aecct_dtype of res, z and y
  const void *res;                     // or null
  void *z;                             // or null
  void *y;
  int64_t ldres, ldz, ldy;
};
struct Gemm {
  int m, n, k;                         // at most 2^28; offsets in memory take 64 bits
  Factor a, b;
  Epilogue e;
  void *part;                          // fp32 (int8 factors: int32) [splits][m][n], or null: one split
  int splits;
};
// type: aecct_dtype, or 16 + aecct_code for codes.
constexpr int kCodeType = 16;
struct GemmPlan {
  bool few;                            // few rows by vector instructions
  int tile;                            // else: which tile
  int splits;
  size_t part_bytes;
};
GemmPlan plan_gemm(int type, int64_t m, int64_t n, int64_t k, bool across_a, bool across_b, int64_t ldb);
hipError_t launch_gemm(int type, const Gemm &g, const GemmPlan &plan, hipStream_t s);
hipError_t launch_gemm_f32(const Gemm &g, const GemmPlan &plan, hipStream_t s);
hipError_t launch_gemm_bf16(const Gemm &g, const GemmPlan &plan, hipStream_t s);
hipError_t launch_gemm_f16(const Gemm &g, const GemmPlan &plan, hipStream_t s);
hipError_t launch_gemm_i8(const Gemm &g, const GemmPlan &plan, hipStream_t s);
hipError_t launch_gemm_e4m3(const Gemm &g, const GemmPlan &plan, hipStream_t s);

// dz = dy act'(z) (not written where act is none) and the sums of its columns.
struct Slope {
  int64_t rows, n;
  int act;
  const void *dy, *z;
  int64_t lddy, ldz;
  void *dz;                            // [rows][lddz], or null
  int64_t lddz;
  float *part;                         // [slope_blocks][n], or null: no sums
  float *dbias;
};
int64_t slope_blocks(int64_t rows, int64_t n);
hipError_t launch_slope(int type, const Slope &a, hipStream_t s);

}  // namespace aecct
