// Norm, clipping and Adam update of lists of tensors: what update_host.cpp hands to the kernels of update.hip.
#pragma once

#include <cstddef>
#include <cstdint>

#include <hip/hip_runtime.h>

namespace aecct {

// A list is cut into units of kUnit values, none of which spans two tensors; a launch takes the tensors of one
// table, passed by value.  Tensor i has units unit0[i] .. unit0[i + 1).
constexpr int kUnit = 4096;
constexpr int kSumTensors = 160, kClipTensors = 96, kAdamTensors = 56;
constexpr int kMaxSumBlocks = 2048;

template <int N>
struct Units {
  int n;                  // tensors
  int unit0[N + 1];
  int64_t count[N];
  uint8_t type[N];        // of the tensor read (aecct_dtype)
};
struct SumTable : Units<kSumTensors> {
  const void *g[kSumTensors];
};
struct ClipTable : Units<kClipTensors> {
  const void *g[kClipTensors];
  void *out[kClipTensors];
  uint8_t out_type[kClipTensors];
};
struct AdamTable : Units<kAdamTensors> {
  const void *g[kAdamTensors];
  float *p[kAdamTensors], *m[kAdamTensors], *v[kAdamTensors];
  void *copy[kAdamTensors];
  uint8_t copy_type[kAdamTensors];
};
struct AdamScalars {
  double lr, beta1, beta2, eps, weight_decay, max_norm;
  const float *lr_device;
};

// Sums of squares of the table's tensors, one double a block, to part[0 .. blocks).
hipError_t launch_sum_squares(const SumTable &t, double *part, int blocks, hipStream_t s);
// *norm from `parts` sums.
hipError_t launch_norm(const double *part, int parts, float *norm, hipStream_t s);
hipError_t launch_clip(const ClipTable &t, const double *part, int parts, double max_norm, float *norm, int cu_count,
                       hipStream_t s);
// *next = *step + 1
hipError_t launch_next_step(const int64_t *step, int64_t *next, hipStream_t s);
// parts = 0: no norm.  step (of one launch of a call, else null) and norm (may be null) are written.
hipError_t launch_adam(const AdamTable &t, const double *part, int parts, const AdamScalars &o, const int64_t *next,
                       int64_t *step, float *norm, int cu_count, hipStream_t s);

}  // namespace aecct
