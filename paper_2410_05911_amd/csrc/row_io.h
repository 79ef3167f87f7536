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

// B bytes (8 or 16) at any 2-byte address; NT: marked as not to be used again soon.
template <int B>
struct Wide {
  typedef uint32_t type __attribute__((ext_vector_type(B / 4), aligned(2)));
};
template <int B, bool NT>
__device__ __forceinline__ void copy_in(const void *p, uint32_t *w) {
  if constexpr (NT && (B == 8 || B == 16)) {
    const typename Wide<B>::type t = __builtin_nontemporal_load((const typename Wide<B>::type *)p);
    __builtin_memcpy(w, &t, B);
  } else {
    __builtin_memcpy(w, p, B);
  }
}
template <int B, bool NT>
__device__ __forceinline__ void copy_out(void *p, const void *w) {
  if constexpr (NT && (B == 8 || B == 16)) {
    typename Wide<B>::type t;
    __builtin_memcpy(&t, w, B);
    __builtin_nontemporal_store(t, (typename Wide<B>::type *)p);
  } else {
    __builtin_memcpy(p, w, B);
  }
}

template <class T, int V, bool NT = false>
__device__ __forceinline__ void store_vec(T *p, const float (&f)[V]) {
  Vec<T, V> t;
#pragma unroll
  for (int i = 0; i < V; ++i) t.v[i] = (T)f[i];
  copy_out<(int)sizeof(t), NT>(p, &t);
}

// The same in two steps, for values that are read ahead: as stored, two 16-bit values a register, then as fp32.
template <class T, int V>
struct Raw {
  uint32_t w[V * sizeof(T) / 4];
};
template <class T, int V, bool NT = false>
__device__ __forceinline__ void load_raw(const T *p, Raw<T, V> &r) {
  copy_in<(int)sizeof(r.w), NT>(p, r.w);
}
// Waits for the loads issued so far, and with them the stores, which the same counter counts.  Behind a branch that few threads take it keeps the wait inside: otherwise the
// registers that it loaded may still be written where the paths meet, and every wavefront waits there, also for what it
// wanted to load ahead (gradient of 100000 x 200 bf16 35 -> 26 us).  0x0f70: no load or store to memory left, the other counters as they are.
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// `bytes` < 4 W bytes from p into the W words, the rest 0, as loads of 16, 8, 4 and 2 bytes at most once each.  (Value by
// value the ends of rows of 5007 bf16 values took half as long as the rows.)
template <int W>
__device__ __forceinline__ void bytes_in(const void *p, int bytes, uint32_t (&w)[W]) {
  const char *const q = (const char *)p;
  if constexpr (W == 8) {
    uint32_t a[4] = {0, 0, 0, 0}, rest[4];
    if (bytes & 16) __builtin_memcpy(a, q, 16);
    bytes_in<4>(q + (bytes & 16), bytes & 15, rest);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = bytes & 16 ? a[i] : rest[i];
      w[4 + i] = bytes & 16 ? rest[i] : 0u;
    }
  } else {
    uint32_t a[2] = {0, 0}, b = 0;
    uint16_t c = 0;
    if (W == 4 && bytes & 8) __builtin_memcpy(a, q, 8);
    if (bytes & 4) __builtin_memcpy(&b, q + (bytes & 8), 4);
    if (bytes & 2) __builtin_memcpy(&c, q + (bytes & 12), 2);
    const uint32_t low = bytes & 4 ? b : c, high = bytes & 4 ? c : 0u;   // the words after the 8 bytes
    if constexpr (W == 4) {
      w[0] = bytes & 8 ? a[0] : low;
      w[1] = bytes & 8 ? a[1] : high;
      w[2] = bytes & 8 ? low : 0u;
      w[3] = bytes & 8 ? high : 0u;
    } else {
      w[0] = low;
      w[1] = high;
    }
  }
}
template <class T, int V>   // the first n < V values (none for n < 0), the others 0
__device__ __forceinline__ void load_raw_part(const T *p, int n, Raw<T, V> &r) {
  bytes_in(p, n > 0 ? n * (int)sizeof(T) : 0, r.w);
  wait_loads();
}
// Value i + n of r to value i, 0 where there is none; 0 < n < V.
template <class T, int V>
__device__ __forceinline__ void move_down(Raw<T, V> &r, int n) {
  constexpr int W = V * (int)sizeof(T) / 4;
  const int words = sizeof(T) == 4 ? n : n / 2;
  if (sizeof(T) == 2 && n % 2) {
#pragma unroll
    for (int i = 0; i < W; ++i) r.w[i] = (r.w[i] >> 16) | (i + 1 < W ? r.w[i + 1] << 16 : 0u);
  }
#pragma unroll
  for (int k = 1; k < W; k *= 2) {
    if (words & k) {
#pragma unroll
      for (int i = 0; i < W; ++i) r.w[i] = i + k < W ? r.w[i + k] : 0u;
    }
  }
}
template <class T, int V>
__device__ __forceinline__ void unpack(const Raw<T, V> &r, float (&f)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if constexpr (sizeof(T) == 4) {
      f[i] = __builtin_bit_cast(float, r.w[i]);
    } else if constexpr (__is_same(T, bf16_t)) {
      f[i] = __builtin_bit_cast(float, i % 2 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
    } else {
      f[i] = (float)__builtin_bit_cast(f16_t, (uint16_t)(r.w[i / 2] >> (16 * (i % 2))));
    }
  }
}

template <class T, int V, bool NT = false>
__device__ __forceinline__ void load_vec(const T *p, float (&f)[V]) {
  Raw<T, V> r;
  load_raw<T, V, NT>(p, r);
  unpack<T, V>(r, f);
}

// The first `n` (clamped to 0..V) of V values; the others are 0 (load) or left alone (store).
template <class T, int V, bool NT = false>
__device__ __forceinline__ void load_part(const T *p, int n, float (&f)[V]) {
  Raw<T, V> r;
  if (n >= V) load_raw<T, V, NT>(p, r);
  else load_raw_part<T, V>(p, n, r);
  unpack<T, V>(r, f);
}
template <class T, int V, bool NT = false>
__device__ __forceinline__ void store_part(T *p, int n, const float (&f)[V]) {
  if (n >= V) {
    store_vec<T, V, NT>(p, f);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) p[i] = (T)f[i];
  }
}

}  // namespace aecct
