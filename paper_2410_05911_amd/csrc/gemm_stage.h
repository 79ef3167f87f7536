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

// Waits until at most N of the loads issued so far are not there yet.
template <int N>
__device__ __forceinline__ void wait_loads_but() {
  static_assert(N < 64, "the counter's bits");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
}
// A block's barrier behind which its LDS accesses are done, that leaves loads from memory on their way.
__device__ __forceinline__ void barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Loads that go to LDS without passing through registers: 16 bytes a lane from byte `offset` of a buffer (zeros from `size` on) to
// the wavefront's place `lds` + 16 lane.  Written as assembly because the compiler waits for such loads before any read of LDS,
// whichever part of it that reads; here wait_loads() says when they have to be there.  (They write no vector registers;
// m0 is the wavefront's place.  One instruction has to lie between the write of m0 and its use.)
struct BufferOf {
  u32x4 r;
  __device__ __forceinline__ BufferOf(const void *p, uint32_t size) {
    const uint64_t a = (uint64_t)(uintptr_t)p;
    r = u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a), (uint32_t)__builtin_amdgcn_readfirstlane((int)(a >> 32)) & 0xffffu,
              size, 0x00020000u};
  }
  __device__ __forceinline__ void to_lds(char *lds, uint32_t offset) const {
    const uint32_t at = (uint32_t)(uintptr_t)AECCT_LDS(char, lds);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(offset), "s"(r) : "memory", "m0");
  }
};

}  // namespace aecct
