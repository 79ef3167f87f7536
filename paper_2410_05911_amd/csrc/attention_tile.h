// Tiles of keys and queries in LDS, and the products of attention on them, for the forward pass and the gradient.
//
// A tile is 32 rows (or several times 32) of RB bytes, d values padded by zeros to 32, 64, 128, 192 or 256.  The 16-byte chunks of a row
// are exchanged by the row's number, so that the reads of one chunk of 32 rows and those of 4 rows' columns fall on
// different banks alike.
#pragma once

#include "../../include/aecct.h"
#include "attention.h"
#include "gemm_stage.h"
#include "mfma.h"

namespace aecct {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

template <int RB>
__device__ __forceinline__ int exchange(int row) {
  static_assert(RB % 128 == 0 || RB == 64, "chunks stay in their row");
  if constexpr (RB % 256 == 0) return ((row & 3) << 2 | (row >> 2 & 3)) << 4;
  return RB >= 128 ? ((row & 3) << 1 | (row >> 2 & 1)) << 4 : ((row & 2) | (row >> 2 & 1)) << 4;
}
// The lane, for LDS addresses.  In fp32 rows of 33 to 64 and of more than 128 values take it as a new value each time: the addresses of a
// tile, the same for every tile, are then computed where they are used instead of being kept over the loop, for which 60 to 200
// registers a lane were spilled (128 x 256 on 128 keys, 8 heads of 64, a band: 163 -> 104 us, its gradient 527 -> 311; 8 x 1024 on
// 1024, 16/4 heads of 256: 2204 -> 1763).  Between, where nothing spills, computing them again costs 5 %.
template <class T, int RB>
__device__ __forceinline__ int lane_of() {
  int lane = threadIdx.x & 63;
  if constexpr (sizeof(T) == 4 && (RB == 256 || RB >= 768)) asm volatile("" : "+v"(lane));
  return lane;
}
// Chunk `chunk` of row `row`: of a product along d.
template <int RB>
__device__ __forceinline__ u32x4 row_chunk(const char *tile, int row, int chunk) {
  return *(const u32x4 *)(tile + row * RB + ((chunk << 4) ^ exchange<RB>(row)));
}
// Columns d0 + lane % 32 of 16-bit rows 16 t + {4 h .. + 3, 8 + 4 h .. + 3}: the order in which a lane's registers 8 t .. 8 t + 7 hold
// the rows of a 32 x 32 result, which is the other factor.
template <int RB>
__device__ __forceinline__ u32x4 column_chunk(const char *tile, int row0, int t, int d0) {
  const int lane = threadIdx.x & 63, l = lane & 15, row = row0 + 16 * t + 4 * (lane >> 5) + (l >> 2);
  const int col = (d0 + (lane & 16) + (l & 3) * 4) * 2;
  return pair64(columns16(tile + row * RB + (col ^ exchange<RB>(row))),
                columns16(tile + (row + 8) * RB + (col ^ exchange<RB>(row + 8))));
}
// The row of a 32 x 32 result that register i of a lane in half h holds.
__device__ __forceinline__ int row_of(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// acc[f] += the tile's columns (32 f + 0..31) times p, over the 32 rows from row0 on; p a result's registers.
//
// fp32 rows of 129 to 256 values, one wavefront a SIMD: what a step reads from LDS is asked for before the step ahead of it is
// multiplied, and the barriers keep it there: left alone, the compiler either waits for each or asks for so many that registers are
// spilled (8 x 1024 on 1024, 16/4 heads of 256 1768 -> 1259 us, gradient of 4 x 1024 on 1024, 8/4 of 160 1117 -> 1096).  TIGHT (dq and
// dk of more than 192 values: three times 128 registers are kept) has none for that; there a branch a step stops at d, and with
// it the compiler's looking ahead (2 x 1024 on 1024, 8/4 of 256: dq 412 us, without the branches 494).
template <class T, int RB, bool TIGHT, int FD>
__device__ __forceinline__ void add_columns(f32x16 (&acc)[FD], const char *tile, int row0, const float (&p)[16], int d) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const u32x4 b = {pack2(p[8 * t], p[8 * t + 1], T()), pack2(p[8 * t + 2], p[8 * t + 3], T()),
                       pack2(p[8 * t + 4], p[8 * t + 5], T()), pack2(p[8 * t + 6], p[8 * t + 7], T())};
#pragma unroll
      for (int f = 0; f < FD; ++f) step<T>(acc[f], column_chunk<RB>(tile, row0, t, 32 * f), b);
    }
  } else {
    const int lane = lane_of<T, RB>(), h = lane >> 5;
    auto value = [&](int i, int f) {
      const int row = row0 + row_of(i, h);
      return *(const float *)(tile + row * RB + (((32 * f + (lane & 31)) * 4) ^ exchange<RB>(row)));
    };
    if constexpr (RB >= 768 && !TIGHT) {
      float v[2][FD];
#pragma unroll
      for (int f = 0; f < FD; ++f) v[0][f] = value(0, f);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (i < 15) {
#pragma unroll
          for (int f = 0; f < FD; ++f) v[(i + 1) & 1][f] = value(i + 1, f);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < FD; ++f) {
          acc[f] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[i & 1][f], p[i], acc[f], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int f = 0; f < FD; ++f) {
          if (TIGHT && f && 32 * f >= d) break;
          acc[f] = __builtin_amdgcn_mfma_f32_32x32x2f32(value(i, f), p[i], acc[f], 0, 0, 0);
        }
    }
  }
}
// The product of the tile's 32 rows from row0 on with a lane's row held in registers (chunks 2 s + h).
template <class T, int RB, bool TIGHT>
__device__ __forceinline__ f32x16 times_rows(const char *tile, int row0, const u32x4 (&r)[RB / 32], int d) {
  const int lane = lane_of<T, RB>();
  f32x16 s;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = 0;
  auto chunk = [&](int c) { return row_chunk<RB>(tile, row0 + (lane & 31), 2 * c + (lane >> 5)); };
  if constexpr (sizeof(T) == 4 && RB >= 768 && !TIGHT) {
    constexpr int G = 2;
    u32x4 x[2][G];
#pragma unroll
    for (int j = 0; j < G; ++j) x[0][j] = chunk(j);
#pragma unroll
    for (int c = 0; c < RB / 32; c += G) {
      if (c + G < RB / 32) {
#pragma unroll
        for (int j = 0; j < G; ++j) x[(c / G + 1) & 1][j] = chunk(c + G + j);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < G; ++j) step<T>(s, x[c / G & 1][j], r[c + j]);
      __builtin_amdgcn_sched_barrier(0);
    }
  } else {
#pragma unroll
    for (int c = 0; c < RB / 32; ++c) {
      if (TIGHT && c && 8 * c >= d) break;
      step<T>(s, chunk(c), r[c]);
    }
  }
  return s;
}

// Both halves' values of x: theirs is the same in lanes l and l + 32.
__device__ __forceinline__ void both_halves(float x, float &low, float &high) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t a = r[0], b = r[1];
  low = __builtin_bit_cast(float, a);
  high = __builtin_bit_cast(float, b);
}
__device__ __forceinline__ float max_halves(float x) {
  float a, b;
  both_halves(x, a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float sum_halves(float x) {
  float a, b;
  both_halves(x, a, b);
  return a + b;
}

// ---- masks that leave few pairs (a Tanner graph's): fp32 tiles go pair by pair, each lane through its own row's keys (or its key's
// rows), where the matrix instructions would take 64 DP clocks for 32 x 32 pairs, a pair of one lane about 240 + 8 DP.  To 64 values a
// row, in dk and dv to 32: a key, its value and both sums leave no registers there (128 x 256 on 128 keys, 8 heads of 64, a Tanner
// graph: the gradient with pairs in dk and dv too 500 us and more, without 299).
template <class T, int RB>
__host__ __device__ constexpr bool pairwise() { return sizeof(T) == 4 && RB <= 256; }
constexpr int kFewPairs = 4;   // of a lane, for 32 keys or rows
// The lane's half of a row of a tile: chunks 2 c + h, which are also the columns that its sums of a result's columns are for.  Read once
// for a product and for a sum (LDS is what bounds these loops).
template <int RB>
struct HalfRow {
  f32x4 x[RB / 32];
  __device__ __forceinline__ HalfRow(const char *tile, int row, int d) {
    const int h = lane_of<float, RB>() >> 5;
#pragma unroll
    for (int c = 0; c < RB / 32; ++c) {
      if (8 * c >= d) break;
      x[c] = __builtin_bit_cast(f32x4, row_chunk<RB>(tile, row, 2 * c + h));
    }
  }
  // Half of the product with the row in the lane's registers.
  __device__ __forceinline__ float dot(const u32x4 (&r)[RB / 32], int d) const {
    float s = 0;
#pragma unroll
    for (int c = 0; c < RB / 32; ++c) {
      if (8 * c >= d) break;
      const f32x4 y = __builtin_bit_cast(f32x4, r[c]);
#pragma unroll
      for (int i = 0; i < 4; ++i) s = fmaf(x[c][i], y[i], s);
    }
    return s;
  }
  template <int FD>
  __device__ __forceinline__ void add_to(f32x16 (&acc)[FD], float w, int d) const {
#pragma unroll
    for (int c = 0; c < RB / 32; ++c) {
      if (8 * c >= d) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[c >> 2][4 * (c & 3) + i] = fmaf(w, x[c][i], acc[c >> 2][4 * (c & 3) + i]);
    }
  }
};
// Bit k of lane r's word to bit r of lane k's, in each half of the wavefront.
__device__ __forceinline__ uint32_t turn_bits(uint32_t x) {
  uint32_t m = 0x0000ffffu;
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
    const uint32_t y = (uint32_t)__shfl_xor((int)x, s);
    x = threadIdx.x & s ? (x & ~m) | ((y & ~m) >> s) : (x & m) | ((y & m) << s);
    m ^= m << (s >> 1);
  }
  return x;
}

// 16 bytes of a row of d values from chunk `chunk` on, zeros behind its end; `end` is where the tensor's memory ends.
template <class T>
__device__ __forceinline__ u32x4 row_piece(const char *row, int chunk, int d, const char *end) {
  constexpr int E = 16 / (int)sizeof(T);
  const int n = d - chunk * E;
  if (n <= 0) return u32x4{0, 0, 0, 0};
  const char *const p = row + chunk * 16;
  if (n >= E) return any16(p);
  if (p + 16 > end) return some_values<T>(p, n);
  u32x4 v = any16(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      if (i >= n) v[i] = 0;
    } else {
      v[i] = 2 * i + 1 < n ? v[i] : 2 * i < n ? v[i] & 0xffffu : 0u;
    }
  }
  return v;
}
__device__ __forceinline__ const char *end_of(const Heads &t, int64_t batch, int64_t length, int64_t heads, int d, int size) {
  return (const char *)t.p + ((batch - 1) * t.batch + (length - 1) * t.row + (heads - 1) * t.head + d) * size;
}

// Blocks in an order that keeps those of one XCD (every eighth) on neighbouring numbers, which share their keys.
__device__ __forceinline__ uint32_t near_block(uint32_t block, uint32_t blocks) {
  const uint32_t share = blocks / 8;
  return block < share * 8 ? block % 8 * share + block / 8 : block;
}
__device__ __forceinline__ int length_of(const Attention &a, uint32_t b) {
  if (!a.lengths) return (int)a.keys;
  const int l = a.lengths[b];
  return max(0, min(l, (int)a.keys));
}

// Whether a tensor's rows are whole 16-byte pieces at 16-byte addresses, and the offsets in a tile of 256 rows within 2^31.
template <class T>
bool direct_ok(const Heads &t, const Attention &a) {
  constexpr int64_t E = 16 / sizeof(T);
  return (uintptr_t)t.p % 16 == 0 && (t.packed || a.d % E == 0) && t.batch % E == 0 && t.row % E == 0 && t.head % E == 0 &&
         t.row < ((int64_t)1 << 22) / (int64_t)sizeof(T);
}
// Tiles of KT keys (or values) of one pair, on their way to LDS: DIRECT by loads whose out-of-range offsets give the zeros behind d and
// past the length, else through registers.  What lies past the length is never read: its weights are 0, and 0 times it may be NaN.
template <class T, int RB, int KT, int NT, bool DIRECT>
struct Keys {
  static constexpr int CH = RB / 16, PER = (KT * CH + NT - 1) / NT, E = 16 / (int)sizeof(T);
  static constexpr uint32_t OUT = 0x80000000u;
  const char *p, *end;
  int64_t stride;              // bytes of a row
  int length, d;
  uint32_t at[DIRECT ? PER : 1];
  u32x4 v[DIRECT ? 1 : PER];
  static __device__ __forceinline__ void place(int i, int &row, int &chunk) {
    const int slot = threadIdx.x + i * NT;
    row = slot / CH;
    chunk = (((slot % CH) << 4) ^ exchange<RB>(row)) >> 4;
  }
  __device__ __forceinline__ Keys(const Heads &t, const Attention &a, uint32_t b, uint32_t kh, int length)
      : p((const char *)t.p + (b * t.batch + kh * t.head) * (int64_t)sizeof(T)),
        end(end_of(t, a.batch, a.keys, a.kv_heads, a.d, sizeof(T))), stride(t.row * (int64_t)sizeof(T)), length(length), d(a.d) {
    if constexpr (DIRECT) {
      static_assert(KT * CH % NT == 0, "whole pieces");
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        int row, chunk;
        place(i, row, chunk);
        at[i] = chunk * E < d ? (uint32_t)(row * stride + chunk * 16) : OUT;
      }
    }
  }
  __device__ __forceinline__ void load(char *lds, int t) {
    if constexpr (DIRECT) {
      const BufferOf r(p + (int64_t)t * KT * stride, OUT);
      const int left = length - t * KT, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        uint32_t offset = at[i];
        if (left < KT) {
          int row, chunk;
          place(i, row, chunk);
          if (row >= left) offset = OUT;
        }
        r.to_lds(lds + (i * NT + wave * 64) * 16, offset);
      }
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        int row, chunk;
        place(i, row, chunk);
        const int64_t key = (int64_t)t * KT + row;
        v[i] = u32x4{0, 0, 0, 0};
        if (row < KT && key < length) v[i] = row_piece<T>(p + key * stride, chunk, d, end);
      }
    }
  }
  __device__ __forceinline__ void store(char *lds) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int slot = threadIdx.x + i * NT;
      if (PER * NT == KT * CH || slot < KT * CH) *(u32x4 *)(lds + slot * 16) = v[i];
    }
  }
};

// Whether any of ROWS rows from row `first` on may attend any of KEYS keys from key0 on, by the tiles of 32 queries that they fall in (one
// more at each end, and behind the last query).  No branch between the loads: they are on their way together.
template <int ROWS, int KEYS>
__device__ __forceinline__ bool any_flag(const Attention &a, uint32_t first, int key0) {
  const uint32_t queries = (uint32_t)a.queries, tiles = (queries + 31) / 32, key_tiles = (uint32_t)words_of(a.keys) / 2;
  constexpr int C = KEYS <= 64 ? 1 : KEYS / 64;     // key0 is a multiple of KEYS
  uint32_t q = first % queries / 32;
  int any = 0;
#pragma unroll
  for (int i = 0; i < (ROWS + 31) / 32 + 2; ++i) {
#pragma unroll
    for (int c = 0; c < C; ++c) any |= a.flags[(int64_t)q * key_tiles + min((uint32_t)key0 / 64 + c, key_tiles - 1)];
    q = q + 1 == tiles ? 0 : q + 1;
  }
  return any != 0;
}

template <class T>
__device__ __forceinline__ void store_values4(T *p, int n, float a, float b, float c, float d) {
  const float v[4] = {a, b, c, d};
  store_part<T, 4>(p, n, v);
}

}  // namespace aecct
