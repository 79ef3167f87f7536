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
  bool packed;                         // its lines are whole pieces, zeros behind their ends
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
// whole: both factors are whole 16-byte pieces.
GemmPlan plan_gemm(int type, int64_t m, int64_t n, int64_t k, bool across_a, bool across_b, int64_t ldb, bool whole);
// The products alone, one or two of them (the gradient's): the sums of splits are left in `part` for launch_finish.
hipError_t launch_gemm(int type, const Gemm *g, const GemmPlan *plan, int count, hipStream_t s);
hipError_t launch_gemm_f32(const Gemm *g, const GemmPlan *plan, int count, hipStream_t s);
hipError_t launch_gemm_bf16(const Gemm *g, const GemmPlan *plan, int count, hipStream_t s);
hipError_t launch_gemm_f16(const Gemm *g, const GemmPlan *plan, int count, hipStream_t s);
hipError_t launch_gemm_i8(const Gemm *g, const GemmPlan *plan, int count, hipStream_t s);
hipError_t launch_gemm_e4m3(const Gemm *g, const GemmPlan *plan, int count, hipStream_t s);

// dz = dy act'(z) (not written where act is none) and the sums of its columns.
struct Slope {
  int rows, n;                         // rows 0 of n 0: not asked for
  int act;
  const void *dy, *z;
  int64_t lddy, ldz;
  void *dz;                            // [rows][lddz], or null
  int64_t lddz;
  float *part;                         // [blocks][n], or null: no sums
  int blocks;                          // slope_blocks(rows, n)
};
int64_t slope_blocks(int64_t rows, int64_t n);
// A matrix of `lines` lines of `width` values, copied to lines that are whole 16-byte pieces, zeros behind their ends; e4m3 values
// become fp16.
struct Pack {
  const void *from;
  int64_t ld;
  int lines, width;                    // lines 0: not asked for
  void *to;
  int64_t ldto;
};
// Values of a line in the copy, of types as GemmPlan's.
inline int type_bytes(int type) { return type == 0 ? 4 : type == kCodeType + 1 ? 1 : 2; }   // as multiplied
inline int64_t packed_line(int type, int64_t width) {
  const int64_t e = 16 / type_bytes(type);
  return (width + e - 1) / e * e;
}
// Whether a matrix has to be copied for the products that take whole pieces.
inline bool ragged(int type, int64_t ld, int64_t width) {
  const int64_t e = 16 / type_bytes(type);
  return type == kCodeType + 2 || ld % e != 0 || width % e != 0;
}
struct Prepare {
  Slope slope;
  Pack pack[3];
};
hipError_t launch_prepare(int type, const Prepare &p, hipStream_t s);
// What is left after the products: the splits' sums with their epilogues, the column sums of launch_prepare.
struct Finish {
  Gemm g[2];                           // part null: not asked for
  const float *part;                   // [blocks][n], or null
  int blocks, n;
  float *out;
};
hipError_t launch_finish(int type, const Finish &f, hipStream_t s);

}  // namespace aecct
