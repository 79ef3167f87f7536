// Norm, clipping and Adam update of lists of tensors: what update_host.cpp hands to the kernels of update.hip.
#pragma once

#include <cstddef>
#include <cstdint>

#include <hip/hip_runtime.h>

namespace aecct {

// A list is cut into units of a table's unit_of(type) values, none of which spans two ranges; a launch takes the ranges of one
// table, passed by value.  A range is a tensor, or tensors that lie back to back.  Range i has units unit0[i] ..
// unit0[i + 1).
// The most ranges of a table keep it below 4 KB; tables of up to kFew are passed in a shorter form.
constexpr int kFew = 24, kSumRanges = 160, kClipRanges = 96, kAdamRanges = 56;
constexpr int kMaxSumBlocks = 2048;

template <int N>
struct Units {
  static constexpr int kMost = N;
  int n;                  // ranges
  int unit0[N + 1];
  int64_t count[N];
  uint8_t type[N];        // of the values read (aecct_dtype)
};
template <int N>
struct SumTable : Units<N> {
  static constexpr int kUnitBytes = 16384;
  static constexpr int unit_of(int type) { return type == 0 ? kUnitBytes / 4 : kUnitBytes / 2; }
  const void *g[N];
};
template <int N>
struct ClipTable : Units<N> {
  static constexpr int kUnit = 4096;
  static constexpr int unit_of(int) { return kUnit; }
  const void *g[N];
  void *out[N];
  uint8_t out_type[N];
};
template <int N>
struct AdamTable : Units<N> {
  static constexpr int kUnit = 1024;
  static constexpr int unit_of(int) { return kUnit; }
  const void *g[N];
  float *p[N], *m[N], *v[N];
  void *copy[N];
  uint8_t copy_type[N];
};
// What an update needs of the number of updates made.
struct AdamNow {
  int64_t step;          // t, this update included
  float grow1, root2;    // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
};
struct AdamScalars {
  double lr, beta1, beta2, eps, weight_decay, max_norm;
  const float *lr_device;
};

// Sums of squares of the table's values, one double a block, to part[0 .. blocks); with now, *now from *step too.
// alone: no pass over the values follows.
hipError_t launch_sum_squares(const SumTable<kSumRanges> &t, double *part, int blocks, bool alone, const int64_t *step,
                              AdamNow *now, const AdamScalars &o, hipStream_t s);
// *norm from `parts` sums.
hipError_t launch_norm(const double *part, int parts, float *norm, hipStream_t s);
hipError_t launch_clip(const ClipTable<kClipRanges> &t, const double *part, int parts, double max_norm, float *norm,
                       int cu_count, hipStream_t s);
hipError_t launch_now(const int64_t *step, AdamNow *now, const AdamScalars &o, hipStream_t s);
// parts = 0: no norm.  step (of one launch of a call, else null) and norm (may be null) are written.
hipError_t launch_adam(const AdamTable<kAdamRanges> &t, const double *part, int parts, const AdamScalars &o,
                       const AdamNow *now, int64_t *step, float *norm, int cu_count, hipStream_t s);

}  // namespace aecct
