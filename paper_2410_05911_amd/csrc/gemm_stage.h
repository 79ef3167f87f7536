// Pieces of 16 bytes from rows at any address, for tiles in LDS.
#pragma once

#include "mfma.h"

namespace aecct {

// The first `n` values at p, the others 0.
template <class T>
__device__ __forceinline__ u32x4 some_values(const char *p, int n) {
  unsigned __int128 v = 0;
#pragma unroll 1
  for (int i = n - 1; i >= 0; --i) {
    if constexpr (sizeof(T) == 4) v = v << 32 | *(const uint32_t *)(p + 4 * i);
    if constexpr (sizeof(T) == 2) v = v << 16 | *(const uint16_t *)(p + 2 * i);
    if constexpr (sizeof(T) == 1) v = v << 8 | *(const uint8_t *)(p + i);
  }
  return __builtin_bit_cast(u32x4, v);
}
__device__ __forceinline__ u32x4 any16(const char *p) {   // at any address
  u32x4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}

}  // namespace aecct
