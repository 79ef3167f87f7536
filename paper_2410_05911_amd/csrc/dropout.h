// Dropout from a counter-based generator: what dropout_host.cpp hands to the kernel.
#pragma once

#include <cstdint>

#include <hip/hip_runtime.h>

namespace aecct {

struct Dropout {
  int64_t rows, d;
  uint32_t below;              // a value is dropped where its word is below this
  float scale;                 // 1 / (1 - p)
  uint64_t seed, offset;
  const int64_t *offset_device;   // or null: offset
  const void *x, *res;
  void *y;
  int64_t ldx, ldres, ldy;
};
hipError_t launch_dropout(int type, const Dropout &a, hipStream_t s);

}  // namespace aecct
