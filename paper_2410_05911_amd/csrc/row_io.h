// Loads and stores of fp32, bf16 and fp16 values for the row and list kernels (norm.hip, update.hip).  A vector of
// V values at any address aligned to one value: gfx950 takes wide global accesses at any byte address, so an
// odd row or tensor start needs no variant of its own.
#pragma once

#include <cstdint>
#include <cstring>

#include <hip/hip_runtime.h>

namespace aecct {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

template <class T, int V>
struct alignas(sizeof(T)) Vec {
  T v[V];
};

template <class T, int V>
__device__ __forceinline__ void load_vec(const T *p, float (&f)[V]) {
  Vec<T, V> t;
  __builtin_memcpy(&t, p, sizeof(t));
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = (float)t.v[i];
}

template <class T, int V>
__device__ __forceinline__ void store_vec(T *p, const float (&f)[V]) {
  Vec<T, V> t;
#pragma unroll
  for (int i = 0; i < V; ++i) t.v[i] = (T)f[i];
  __builtin_memcpy(p, &t, sizeof(t));
}

// The first `n` (clamped to 0..V) of V values; the others are 0 (load) or left alone (store).
template <class T, int V>
__device__ __forceinline__ void load_part(const T *p, int n, float (&f)[V]) {
  if (n >= V) {
    load_vec<T, V>(p, f);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = i < n ? (float)p[i] : 0.0f;
  }
}
template <class T, int V>
__device__ __forceinline__ void store_part(T *p, int n, const float (&f)[V]) {
  if (n >= V) {
    store_vec<T, V>(p, f);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) p[i] = (T)f[i];
  }
}

}  // namespace aecct
