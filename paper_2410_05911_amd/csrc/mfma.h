// Matrix products of 32 x 32 tiles on the matrix instructions, for the types of the linear maps and of cross attention.
//
// A chunk is 16 bytes of consecutive k (8 16-bit, 16 8-bit, 4 fp32 values) of one row.  In a step each half h = lane / 32
// of the wavefront holds chunk 2 s + h of row lane % 32 of both factors: the instructions pair values of equal position
// in equal halves, so any order of k that both factors share gives the product.  D's row of register i is
// 8 (i / 4) + 4 h + i % 4 (of the first factor), its column lane % 32 (of the second).
#pragma once

#include <cstdint>

#include <hip/hip_runtime.h>

#include "row_io.h"

namespace aecct {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));
struct e4m3_t {
  uint8_t bits;
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

template <class T>
struct Product {
  typedef f32x16 Acc;
};
template <>
struct Product<int8_t> {
  typedef i32x16 Acc;
};

// acc += a b over one step of chunks.  (There is none for e4m3: the instructions on 8-bit floats add products of very different size
// with about 17 bits, sums of 64 products of full-scale codes came out 1.5e-5 off; those on fp16 lose nothing of that size.)
template <class T>
__device__ __forceinline__ void step(typename Product<T>::Acc &acc, u32x4 a, u32x4 b) {
  if constexpr (sizeof(T) == 4) {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], acc, 0, 0, 0);
  } else if constexpr (__is_same(T, bf16_t)) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
  } else if constexpr (__is_same(T, f16_t)) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
  } else {
    static_assert(__is_same(T, int8_t), "e4m3 goes as fp16");
    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), acc, 0, 0, 0);
  }
}

// Eight e4m3 values as fp16, which holds all of them.
__device__ __forceinline__ u32x4 widen(uint32_t low, uint32_t high) {
  typedef _Float16 two __attribute__((ext_vector_type(2)));
  const two a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(low, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(low, 1.0f, true),
            c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(high, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(high, 1.0f, true);
  return u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
               __builtin_bit_cast(uint32_t, d)};
}

// Value `i` of four e4m3 values.
__device__ __forceinline__ float e4m3_value(uint32_t w, int i) {
  typedef float two __attribute__((ext_vector_type(2)));
  const two v = i < 2 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  const float low = v[0], high = v[1];
  return i % 2 ? high : low;
}

// ---- tiles in LDS
// "Along k": a row of the tile is 128 bytes of k, its chunk c at place c ^ (row / 2 % 8): LDS serves 16 lanes of 16 bytes at once where
// they fall on all of its banks, and 16 rows of two to 256 bytes do.
__device__ __forceinline__ int along_swap(int row) { return row >> 1 & 7; }
__device__ __forceinline__ int along_k(int row, int chunk) { return row * 128 + ((chunk ^ along_swap(row)) << 4); }
template <class T>
__device__ __forceinline__ u32x4 frag_k(const char *tile, int row, int chunk) {
  return *(const u32x4 *)(tile + along_k(row, chunk));
}

// "Across k": a line of the tile is PITCH bytes of rows at one k.  Its bytes are exchanged (exclusive or of the offset) so
// that the lines that one read spans fall on different banks: 4 lines of 64 bytes for 16-bit values, 8 of 32 for 8-bit
// values, 2 of 128 for fp32.
template <class T, int PITCH>
__device__ __forceinline__ int line_swap(int k) {
  static_assert(PITCH % (32 * sizeof(T)) == 0, "a fragment is 32 rows");
  if constexpr (sizeof(T) == 2) return PITCH >= 256 ? (k & 3) << 6 : PITCH == 128 ? (k >> 1 & 1) << 6 : 0;
  if constexpr (sizeof(T) == 1) return PITCH >= 256 ? (k & 7) << 5 : PITCH == 128 ? (k >> 1 & 3) << 5 : PITCH == 64 ? (k >> 2 & 1) << 5 : 0;
  return PITCH >= 256 ? (k >> 2 & 1) << 7 : 0;
}
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
#define AECCT_LDS(type, p) ((__attribute__((address_space(3))) type *)(p))
// 8 bytes a lane: of the 16 lanes of a group lane l reads part l % (16 / lines) of line l / (16 / lines); the group's lane l
// gets column l, its values in the order of the lines.  All lanes have to take part.
__device__ __forceinline__ uint64_t columns16(const char *p) {
  return __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(AECCT_LDS(s16x4, p)));
}
__device__ __forceinline__ uint64_t columns8(const char *p) {
  return __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr8_b64_v2i32(AECCT_LDS(i32x2, p)));
}
__device__ __forceinline__ u32x4 pair64(uint64_t a, uint64_t b) {
  return u32x4{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
}
// Rows row0 + lane % 32 of chunk `chunk`.  (line_swap is the same for all lines that a lane reads of a chunk.)
template <class T, int PITCH>
__device__ __forceinline__ u32x4 frag_n(const char *tile, int row0, int chunk) {
  const int lane = threadIdx.x & 63, l = lane & 15, sixteen = lane & 16;
  if constexpr (sizeof(T) == 2) {
    const char *const p = tile + (chunk * 8 + (l >> 2)) * PITCH + (((row0 + sixteen + (l & 3) * 4) * 2) ^ line_swap<T, PITCH>(l >> 2));
    return pair64(columns16(p), columns16(p + 4 * PITCH));
  } else if constexpr (sizeof(T) == 1) {
    const char *const p = tile + (chunk * 16 + (l >> 1)) * PITCH + ((row0 + sixteen + (l & 1) * 8) ^ line_swap<T, PITCH>(l >> 1));
    return pair64(columns8(p), columns8(p + 8 * PITCH));
  } else {
    const char *const p = tile + chunk * 4 * PITCH + (((row0 + (lane & 31)) * 4) ^ line_swap<T, PITCH>(chunk * 4));
    u32x4 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = *(const uint32_t *)(p + i * PITCH);
    return f;
  }
}

// ---- values of a stored type
__device__ __forceinline__ uint32_t pack2(float a, float b, bf16_t) {
  typedef __bf16 two __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, two{(__bf16)a, (__bf16)b});
}
__device__ __forceinline__ uint32_t pack2(float a, float b, f16_t) {
  typedef _Float16 two __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, two{(_Float16)a, (_Float16)b});
}

}  // namespace aecct
