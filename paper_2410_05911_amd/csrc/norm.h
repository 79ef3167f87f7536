// Root-mean-square norm of rows and its gradient: what norm_host.cpp hands to the kernels of norm.hip.
#pragma once

#include <cstddef>
#include <cstdint>

#include <hip/hip_runtime.h>

namespace aecct {

struct NormRows {
  int64_t rows;
  int d;
  float eps;
  bool gain_f32;               // gain is fp32, else of the rows' type
  int code;                    // aecct_code
  int group;                   // columns of one alpha (d: the whole row)
  int alphas;                  // alphas a row
  const void *x, *res, *gain;
  void *h, *y;
  uint8_t *codes;
  float *alpha;
  int64_t ldx, ldres, ldh, ldy, ldcodes;
  bool past_in, past_out;      // inputs are read, outputs written past the caches
};
hipError_t launch_rms_norm(int type, const NormRows &a, int cu_count, hipStream_t s);

struct NormGradRows {
  int64_t rows;
  int d;
  float eps;
  bool gain_f32;
  const void *h, *dy, *dres, *gain;
  void *dh;
  int64_t ldh, lddy, lddres, lddh;
  float *part;                 // partial sums of dgain, or null: no dgain
  float *dgain;
  bool past_in;
};
// Blocks at most, so rows of the partial sums: norm_grad_part_rows(rows, d) of d floats each.
int64_t norm_grad_part_rows(int64_t rows, int d);
hipError_t launch_rms_norm_grad(int type, const NormGradRows &a, int cu_count, hipStream_t s);

}  // namespace aecct
