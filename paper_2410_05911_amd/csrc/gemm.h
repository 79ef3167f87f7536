// The product of two factors, a block of BM x BN outputs a workgroup: tiles of 128 bytes of k of both factors go through LDS
// twice over (one is read by the matrix instructions while the next one is on its way), each wavefront sums 32 x 32
// blocks of the outputs in its registers.
//
// The first factor of a matrix instruction is b and the second a: a lane then holds one row m of the output and groups
// of four consecutive columns n, and reads and writes the epilogue's tensors four values at a time.
#pragma once

#include <cmath>

#include "../../include/aecct.h"
#include "linear.h"
#include "gemm_stage.h"
#include "mfma.h"

namespace aecct {

// ---- activations, in fp32
// 2^(hi + lo), lo small; 1 / x, after a step of Newton's where F32.
__device__ __forceinline__ float exp2_of(float hi, float lo) {
  const float e = __builtin_amdgcn_exp2f(hi);
  return fmaf(e, lo * 0.69314718f, e);
}
template <bool F32>
__device__ __forceinline__ float inverse(float x) {
  const float r = __builtin_amdgcn_rcpf(x);
  return F32 ? fmaf(fmaf(-x, r, 1.0f), r, r) : r;
}
// The normal distribution Phi(z) and e = e^(-z^2 / 2).  Its tail, half of erfc(x) at x = |z| / sqrt(2), is e times a polynomial in
// 1 / (1 + c x), x to 9.6.  For fp32 outputs its coefficients are fitted here to 3e-8 of erfc(x), and the exponent is taken in two
// parts: z Phi(z) is within 7 2^-24 of itself from -12.5 on (with erfcf and expf in their place the epilogue took 23 registers more and
// a compute unit one block less: 49152 x 128 -> 512 int8, ReLU, 31 -> 42 us).  For 16 bits they are fitted for the smallest error
// against the larger of 1.4e-7 and 2^-14 of erfc(x), an eighth of fp16's half step where Phi is small (with one coefficient less,
// fitted for 1.5e-7 alone, GELU at -4 was off by 2 half steps of fp16 and below -7 by several of bf16).  |z| is
// bounded in fp32 so that both parts of the exponent stay finite.
template <bool F32>
__device__ __forceinline__ float normal(float z, float &e) {
  const float a = F32 && fabsf(z) > 100.0f ? 100.0f : fabsf(z), x = a * 0.70710678118654752f;
  const float t = inverse<F32>(fmaf(F32 ? 0.48f : 0.412f, x, 1.0f));
  float p;
  if constexpr (F32) {
    const float s = a * a, c = -0.72134752f, hi = s * c;     // -log2(e) / 2 is c - 9.63e-9
    e = exp2_of(hi, fmaf(s, c, -hi) + fmaf(fmaf(a, a, -s), c, s * -9.6298e-9f));
    p = fmaf(t, -0.052127723f, 0.27955455f);
    p = fmaf(t, p, -0.5505261f);
    p = fmaf(t, p, 0.41219106f);
    p = fmaf(t, p, -0.094040006f);
    p = fmaf(t, p, 0.23274627f);
    p = fmaf(t, p, 0.22962034f);
    p = fmaf(t, p, 0.27181336f);
    p = fmaf(t, p, 0.2707682f);
  } else {
    e = __builtin_amdgcn_exp2f(x * x * -1.4426950408889634f);
    p = fmaf(t, -0.17485723f, 0.55085403f);
    p = fmaf(t, p, -0.1636966f);
    p = fmaf(t, p, 0.3475389f);
    p = fmaf(t, p, 0.20564933f);
    p = fmaf(t, p, 0.23451155f);
  }
  const float tail = 0.5f * (p * t) * e;
  return z > 0.0f ? 1.0f - tail : tail;
}
// 1 / (1 + e^-z) and q = 1 - that, each from e^-|z|, so that the smaller one keeps its bits and does not vanish before e^-|z| does.
template <bool F32>
__device__ __forceinline__ float logistic(float z, float &q) {
  const float a = F32 && fabsf(z) > 200.0f ? 200.0f : fabsf(z), c = -1.44269502f, hi = a * c;     // -log2(e) is c - 1.926e-8
  const float e = F32 ? exp2_of(hi, fmaf(a, c, -hi) + a * -1.92596e-8f) : __builtin_amdgcn_exp2f(hi);
  const float large = inverse<F32>(1.0f + e), small = e * large;
  q = z < 0.0f ? large : small;
  return z < 0.0f ? small : large;
}
template <bool F32>
__device__ __forceinline__ float activate(float z, int act) {
  float other;
  if (act == kActRelu) return z > 0.0f || z != z ? z : 0.0f;
  if (act == kActGelu) return z * normal<F32>(z, other);
  if (act == kActSilu) return z * logistic<F32>(z, other);
  return z;
}

// ---- V values of a stored type, at any address aligned to one
template <int V>
__device__ __forceinline__ void load_values(int type, const void *p, int64_t at, int n, float (&f)[V]) {
  if (type == 0) load_part<float, V>((const float *)p + at, n, f);
  else if (type == 1) load_part<bf16_t, V>((const bf16_t *)p + at, n, f);
  else load_part<f16_t, V>((const f16_t *)p + at, n, f);
}
template <int V>
__device__ __forceinline__ void store_values(int type, void *p, int64_t at, int n, const float (&f)[V]) {
  if (type == 0) store_part<float, V>((float *)p + at, n, f);
  else if (type == 1) store_part<bf16_t, V>((bf16_t *)p + at, n, f);
  else store_part<f16_t, V>((f16_t *)p + at, n, f);
}

// What the epilogue takes of V columns (n0 .. n0 + count, count <= V).
template <int V>
struct Columns {
  float scale[V], bias[V];
  __device__ __forceinline__ Columns(const Epilogue &e, int64_t n0, int count) {
#pragma unroll
    for (int i = 0; i < V; ++i) scale[i] = bias[i] = 0;
    if (e.alpha) load_part<float, V>(e.scale + n0, count, scale);
    if (e.bias) load_part<float, V>(e.bias + n0, count, bias);
  }
};
// The epilogue of those columns' values of row m; F32: of an fp32 output.
template <bool F32, int V>
__device__ __forceinline__ void finish(const Epilogue &e, const Columns<V> &of, int64_t m, int64_t n0, int count, float (&v)[V]) {
  float r[V];
  if (e.res) load_values<V>(e.type, e.res, m * e.ldres + n0, count, r);
  if (e.alpha) {
    const float a = e.alpha[m] * e.per_q;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = v[i] * a * of.scale[i];
  }
  if (e.bias) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += of.bias[i];
  }
  if (e.z) store_values<V>(e.type, e.z, m * e.ldz + n0, count, v);
  if (e.act != kActNone) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = activate<F32>(v[i], e.act);
  }
  if (e.res) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += r[i];
  }
  store_values<V>(e.type, e.y, m * e.ldy + n0, count, v);
}
template <int V>
__device__ __forceinline__ void finish(const Epilogue &e, int64_t m, int64_t n0, int count, float (&v)[V]) {
  if (e.type == AECCT_F32) finish<true>(e, Columns<V>(e, n0, count), m, n0, count, v);
  else finish<false>(e, Columns<V>(e, n0, count), m, n0, count, v);
}

// ---- staging: 16-byte pieces of a factor's tile, slot by slot
// E values of the stored type S at p as the product's type T: all of them, or the first n.
template <class T, class S>
__device__ __forceinline__ u32x4 piece(const char *p) {
  if constexpr (__is_same(S, e4m3_t)) {
    uint32_t v[2];
    __builtin_memcpy(v, p, 8);
    return widen(v[0], v[1]);
  } else {
    return any16(p);
  }
}
template <class T, class S>
__device__ __forceinline__ u32x4 piece(const char *p, int n) {
  const u32x4 v = some_values<S>(p, n);
  if constexpr (__is_same(S, e4m3_t)) return widen(v[0], v[1]);
  return v;
}

// A tile of ROWS rows from row0 on, of values stored as S and multiplied as T: where slot `slot` of its LDS lies in the factor.
template <class T, class S, bool ACROSS, int ROWS>
struct Tile {
  static constexpr int E = 16 / (int)sizeof(T), KT = 128 / (int)sizeof(T), PITCH = ROWS * (int)sizeof(T);
  static constexpr int SLOTS = ROWS * 8;
  // The row (first of them) and the k (first of them) that the slot holds, relative to the tile.
  static __device__ __forceinline__ void place(int slot, int &row, int &k) {
    if constexpr (ACROSS) {
      constexpr int PER = PITCH / 16;
      k = slot / PER;
      row = ((slot % PER) ^ (line_swap<T, PITCH>(k) >> 4)) * E;
    } else {
      row = slot >> 3;
      k = ((slot & 7) ^ along_swap(row)) * E;
    }
  }
  // The slot's values: zeros past `k_end`, anything for rows past `rows`.  k_all: the factor's k, where its memory ends.
  static __device__ __forceinline__ u32x4 fetch(const char *p, int64_t ld, int64_t rows, int64_t k_all, int64_t row0, int64_t k0,
                                                int64_t k_end, int slot) {
    int r, c;
    place(slot, r, c);
    const int64_t k = k0 + c;
    if constexpr (ACROSS) {
      const int64_t row = row0 + r;
      if (k >= k_end || row >= rows) return u32x4{0, 0, 0, 0};
      const int64_t at = k * ld + row, left = (k_all - 1) * ld + rows - at;   // values to the end of the memory
      return left >= E ? piece<T, S>(p + at * (int64_t)sizeof(S)) : piece<T, S>(p + at * (int64_t)sizeof(S), (int)left);
    } else {
      if (k >= k_end) return u32x4{0, 0, 0, 0};
      const int64_t row = row0 + r < rows ? row0 + r : rows - 1;
      const char *const q = p + (row * ld + k) * (int64_t)sizeof(S);
      return k + E <= k_end ? piece<T, S>(q) : piece<T, S>(q, (int)(k_end - k));
    }
  }
  static __device__ __forceinline__ u32x4 frag(const char *tile, int row0, int chunk) {
    if constexpr (ACROSS) return frag_n<T, PITCH>(tile, row0, chunk);
    else return frag_k<T>(tile, row0 + (threadIdx.x & 31), chunk);
  }
};

// Orders a wavefront's LDS accesses before and after among its lanes (they run in order; the compiler must not move them).
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Blocks in an order that keeps those of one XCD (every eighth block) on neighbouring numbers.  (Numbers of blocks and tiles are 32-bit:
// a 64-bit division takes 150 instructions, and several of them a microsecond of a small product.)
__device__ __forceinline__ uint32_t near_tile(uint32_t block, uint32_t all) {
  const uint32_t share = all / 8;
  return block < share * 8 ? block % 8 * share + block / 8 : block;
}
// Tiles in such an order, bands of 8 rows of tiles, column by column.
__device__ __forceinline__ void tile_of(uint32_t block, uint32_t tm, uint32_t tn, uint32_t &im, uint32_t &in) {
  const uint32_t at = near_tile(block, tm * tn);
  const uint32_t band = at / (8 * tn), first = band * 8, height = min(tm - first, 8u), rest = at - band * 8 * tn;
  in = rest / height;
  im = first + rest - in * height;
}
// A block's tile and its share of k: whole tiles of k to each split; only the last one has a ragged end.
struct Share {
  int m0, n0, k0, k1, split;
  template <int BM, int BN, int KT>
  static __device__ __forceinline__ Share of(const Gemm &g, uint32_t block) {
    const uint32_t tm = (uint32_t)(g.m + BM - 1) / BM, tn = (uint32_t)(g.n + BN - 1) / BN, tiles = tm * tn;
    const uint32_t split = g.splits > 1 ? block / tiles : 0, kt = (uint32_t)(g.k + KT - 1) / KT;
    uint32_t im, in, first = 0, last = kt;
    tile_of(block - split * tiles, tm, tn, im, in);
    if (g.splits > 1) {
      first = kt * split / (uint32_t)g.splits;
      last = kt * (split + 1) / (uint32_t)g.splits;
    }
    return {(int)(im * BM), (int)(in * BN), (int)(first * KT), min(g.k, (int)(last * KT)), (int)split};
  }
};

// 32 rows of sums in LDS through the epilogue, V neighbouring columns a lane: four of fp32 outputs and sums, eight of 16-bit ones.
template <int V, int FN, int TURNS>
__device__ __forceinline__ void finish_strip(const Gemm &g, const float *strip, int split, int m0, int n0) {
  constexpr int LD = FN * 32 + 4, PER = FN * 32 / V, STEP = 64 / PER;   // lanes a row, rows at once
  const int lane = threadIdx.x & 63, c = lane % PER * V, n = n0 + c, count = min(g.n - n, V);
  const Columns<V> columns(g.e, n, g.part ? 0 : count);
#pragma unroll TURNS
  for (int at = 0; at < 32; at += STEP) {
    const int row = at + lane / PER, m = m0 + row;
    if (m >= g.m || count <= 0) continue;
    float v[V];
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const f32x4 x = *(const f32x4 *)(strip + row * LD + c + i);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[i + r] = x[r];
    }
    if (g.part) store_part<float, V>((float *)g.part + ((int64_t)split * g.m + m) * g.n + n, count, v);
    else finish<V == 4>(g.e, columns, m, n, count, v);
  }
}
// A wavefront's FM x FN sums from (m0, n0) on through the epilogue: 32 rows at a time go through LDS, so that a lane then has 16 bytes of
// neighbouring outputs and neighbouring lanes a row's (stored as they lie in registers, in pieces of 16 or 8 bytes 32 rows apart,
// 49152 x 128 -> 512 to fp32 took 89 us; in pieces of 16 bytes 32 apart 38).  All wavefronts of the block are done with the
// tiles in LDS before.
template <class T, int FM, int FN>
__device__ __forceinline__ void finish_block(const Gemm &g, typename Product<T>::Acc (&acc)[FM][FN], char *lds, int split, int m0, int n0) {
  constexpr int LD = FN * 32 + 4;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  float *const strip = (float *)lds + (threadIdx.x >> 6) * (32 * LD);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < FM; ++i) {
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const auto sum = acc[i][j][4 * q + r];
          v[r] = g.part ? __builtin_bit_cast(float, sum) : (float)sum;   // int32 partial sums travel as their bits
        }
        *(f32x4 *)(strip + (lane & 31) * LD + j * 32 + 8 * q + 4 * h) = v;
      }
    wave_sync();
    if (g.part || g.e.type == AECCT_F32) finish_strip<4, FN, 4>(g, strip, split, m0 + i * 32, n0);
    else finish_strip<8, FN, (FM * FN <= 4 ? 4 : 2)>(g, strip, split, m0 + i * 32, n0);
    wave_sync();
  }
}

// A factor's tiles on their way through registers: a thread's slots as 32-bit offsets from the tile's begin, where the tile is whole
// (values past a row's end may be read, not past the memory's: rows that are not there give outputs that are not there).
template <class T, class S, bool ACROSS, int ROWS, int NT>
struct Through {
  typedef Tile<T, S, ACROSS, ROWS> Place;
  static constexpr int COUNT = Place::SLOTS / NT;
  uint32_t at[COUNT];
  const Factor &f;
  int64_t rows, k_all, row0;
  bool near;
  __device__ __forceinline__ Through(const Factor &f, int64_t rows, int64_t k_all, int64_t row0)
      : f(f), rows(rows), k_all(k_all), row0(row0) {
    near = f.ld < ((int64_t)1 << 30) / (ROWS > Place::KT ? ROWS : Place::KT) / (int64_t)sizeof(S);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      int r, k;
      Place::place(threadIdx.x + i * NT, r, k);
      if constexpr (!ACROSS) r = row0 + r < rows ? r : (int)(rows - 1 - row0);
      at[i] = (uint32_t)((ACROSS ? k * f.ld + r : r * f.ld + k) * (int64_t)sizeof(S));
    }
  }
  // The tile of k0, of which k_end is the end.
  __device__ __forceinline__ void load(u32x4 (&v)[COUNT], int64_t k0, int64_t k_end) const {
    bool whole = near && k0 + Place::KT <= k_end;
    if constexpr (ACROSS) whole = whole && (k0 + Place::KT - 1) * f.ld + row0 + ROWS <= (k_all - 1) * f.ld + rows;
    if (whole) {
      const char *const p = (const char *)f.p + (ACROSS ? k0 * f.ld + row0 : row0 * f.ld + k0) * (int64_t)sizeof(S);
#pragma unroll
      for (int i = 0; i < COUNT; ++i) v[i] = piece<T, S>(p + at[i]);
    } else {
#pragma unroll
      for (int i = 0; i < COUNT; ++i)
        v[i] = Place::fetch((const char *)f.p, f.ld, rows, k_all, row0, k0, k_end, threadIdx.x + i * NT);
    }
  }
};

template <class T, class S, bool AA, bool BA, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN * 64) void k_gemm(Gemm g) {
  typedef Tile<T, S, AA, BM> TA;
  typedef Tile<T, S, BA, BN> TB;
  constexpr int NT = WM * WN * 64, FM = BM / WM / 32, FN = BN / WN / 32, KT = TA::KT;
  constexpr int CA = TA::SLOTS / NT, CB = TB::SLOTS / NT, BYTES = (BM + BN) * 128;
  constexpr int AHEAD = CA + CB <= 4 ? 3 : 1;   // tiles on their way in registers
  static_assert(TA::SLOTS % NT == 0 && TB::SLOTS % NT == 0, "whole slots");
  __shared__ __attribute__((aligned(16))) char lds[2 * BYTES];
  const Share at = Share::of<BM, BN, KT>(g, blockIdx.x);
  const int m0 = at.m0, n0 = at.n0, k0 = at.k0, k1 = at.k1, split = at.split;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5;
  const int wm = wave / WN * (FM * 32), wn = wave % WN * (FN * 32);
  const Through<T, S, AA, BM, NT> ta(g.a, g.m, g.k, m0);
  const Through<T, S, BA, BN, NT> tb(g.b, g.n, g.k, n0);

  typename Product<T>::Acc acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;

  u32x4 ra[AHEAD][CA], rb[AHEAD][CB];
#pragma unroll
  for (int d = 0; d < AHEAD; ++d) {
    if (k0 + d * KT < k1) {
      ta.load(ra[d], k0 + d * KT, k1);
      tb.load(rb[d], k0 + d * KT, k1);
    }
  }
  int buf = 0;
  for (int k = k0; k < k1;) {
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) {
      if (k >= k1) break;
      char *const la = lds + buf * BYTES, *const lb = la + BM * 128;
#pragma unroll
      for (int i = 0; i < CA; ++i) *(u32x4 *)(la + (threadIdx.x + i * NT) * 16) = ra[d][i];
#pragma unroll
      for (int i = 0; i < CB; ++i) *(u32x4 *)(lb + (threadIdx.x + i * NT) * 16) = rb[d][i];
      __syncthreads();   // also: no wavefront reads the other buffer any more when the next round writes it
      if (k + AHEAD * KT < k1) {
        ta.load(ra[d], k + AHEAD * KT, k1);
        tb.load(rb[d], k + AHEAD * KT, k1);
      }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      u32x4 fa[FM];
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[i] = TA::frag(la, wm + i * 32, 2 * s + h);
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const u32x4 fb = TB::frag(lb, wn + j * 32, 2 * s + h);
#pragma unroll
        for (int i = 0; i < FM; ++i) step<T>(acc[i][j], fb, fa[i]);
      }
    }
      k += KT;
      buf ^= 1;
    }
  }
  finish_block<T, FM, FN>(g, acc, lds, split, m0 + wm, n0 + wn);
}

// The same product where both factors' rows begin at 16-byte addresses and are whole 16-byte pieces: the pieces go from memory to LDS
// without passing through registers, by buffer loads whose out-of-range offsets give the zeros of a ragged end.
template <class T, bool ACROSS, int ROWS, int NT>
struct Direct {
  typedef Tile<T, T, ACROSS, ROWS> Place;
  static constexpr int COUNT = Place::SLOTS / NT;
  static constexpr uint32_t OUT = 0x80000000u;   // offsets from here on are out of range
  uint32_t at[COUNT];
  const char *p;
  int64_t step;
  __device__ __forceinline__ void init(const Factor &f, int64_t rows, int64_t row0, int64_t k0) {
    p = (const char *)f.p + (ACROSS ? k0 * f.ld + row0 : row0 * f.ld + k0) * (int64_t)sizeof(T);
    step = (ACROSS ? Place::KT * f.ld : Place::KT) * (int64_t)sizeof(T);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      int r, k;
      Place::place(threadIdx.x + i * NT, r, k);
      if constexpr (ACROSS) {
        at[i] = row0 + r < rows ? (uint32_t)((k * f.ld + r) * (int64_t)sizeof(T)) : OUT;
      } else {
        const int64_t row = row0 + r < rows ? r : rows - 1 - row0;
        at[i] = (uint32_t)((row * f.ld + k) * (int64_t)sizeof(T));
      }
    }
  }
  // The next tile into LDS; `left` of its k are there.
  __device__ __forceinline__ void load(char *lds, int left) {
    const BufferOf r(p, OUT);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      uint32_t offset = at[i];
      if (left < Place::KT) {
        int row, k;
        Place::place(threadIdx.x + i * NT, row, k);
        if (k >= left) offset = OUT;
      }
      r.to_lds(lds + (i * NT + wave * 64) * 16, offset);
    }
    p += step;
  }
};

// STAGES tiles of LDS: while one is multiplied, STAGES - 2 lie ready or are on their way beside the one being asked for.
template <int BM, int BN, int WM, int WN, int STAGES>
struct DirectShape {
  static constexpr int BYTES = (BM + BN) * 128, STRIPS = WM * WN * 32 * (BN / WN + 4) * 4;   // a stage; what finish_block takes
  static constexpr int LDS = STAGES * BYTES > STRIPS ? STAGES * BYTES : STRIPS;
};
template <class T, bool AA, bool BA, int BM, int BN, int WM, int WN, int STAGES>
__device__ __forceinline__ void gemm_direct(const Gemm &g, uint32_t block, char *lds) {
  typedef Tile<T, T, AA, BM> TA;
  typedef Tile<T, T, BA, BN> TB;
  constexpr int NT = WM * WN * 64, FM = BM / WM / 32, FN = BN / WN / 32, KT = TA::KT, BYTES = (BM + BN) * 128;
  const Share at = Share::of<BM, BN, KT>(g, block);
  const int m0 = at.m0, n0 = at.n0, k0 = at.k0, k1 = at.k1, split = at.split;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5;
  const int wm = wave / WN * (FM * 32), wn = wave % WN * (FN * 32);
  Direct<T, AA, BM, NT> da;
  Direct<T, BA, BN, NT> db;
  da.init(g.a, g.m, m0, k0);
  db.init(g.b, g.n, n0, k0);

  typename Product<T>::Acc acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
  constexpr int AHEAD = STAGES > 1 ? STAGES - 1 : 1;   // one stage: for a k of one tile
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    if (k0 + i * KT < k1) {
      da.load(lds + i * BYTES, k1 - k0 - i * KT);
      db.load(lds + i * BYTES + BM * 128, k1 - k0 - i * KT);
    }
  }
  int buf = 0, free = AHEAD;
  for (int k = k0; k < k1; k += KT) {
    // Loads come back in order: the tile is there when only those of the tiles after it are left.
    if (k + (AHEAD - 1) * KT < k1) wait_loads_but<(AHEAD - 1) * (Direct<T, AA, BM, NT>::COUNT + Direct<T, BA, BN, NT>::COUNT)>();
    else wait_loads();
    barrier();   // the tile is there for all, and nobody reads the one before it any more
    const char *const la = lds + buf * BYTES, *const lb = la + BM * 128;
    if (k + AHEAD * KT < k1) {
      da.load(lds + free * BYTES, k1 - k - AHEAD * KT);
      db.load(lds + free * BYTES + BM * 128, k1 - k - AHEAD * KT);
    }
    buf = buf + 1 == STAGES ? 0 : buf + 1;
    free = free + 1 == STAGES ? 0 : free + 1;
    u32x4 fa[2][FM], fb[2][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) fa[0][i] = TA::frag(la, wm + i * 32, h);
#pragma unroll
    for (int j = 0; j < FN; ++j) fb[0][j] = TB::frag(lb, wn + j * 32, h);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s < 3) {
#pragma unroll
        for (int i = 0; i < FM; ++i) fa[(s + 1) & 1][i] = TA::frag(la, wm + i * 32, 2 * s + 2 + h);
#pragma unroll
        for (int j = 0; j < FN; ++j) fb[(s + 1) & 1][j] = TB::frag(lb, wn + j * 32, 2 * s + 2 + h);
      }
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) step<T>(acc[i][j], fb[s & 1][j], fa[s & 1][i]);
    }
    if constexpr (sizeof(T) < 4) {
      constexpr int READS = (AA ? 2 : 1) * FM + (BA ? 2 : 1) * FN, EACH = (READS + FM * FN - 1) / (FM * FN);
      __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
#pragma unroll
      for (int s = 0; s < 3; ++s) {
#pragma unroll
        for (int i = 0; i < FM * FN; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
        }
      }
      __builtin_amdgcn_sched_group_barrier(0x008, FM * FN, 0);
    }
  }
  finish_block<T, FM, FN>(g, acc, lds, split, m0 + wm, n0 + wn);
}

template <class T, bool AA, bool BA, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WM *WN * 64) void k_gemm_direct(Gemm g) {
  __shared__ __attribute__((aligned(16))) char lds[DirectShape<BM, BN, WM, WN, STAGES>::LDS];
  gemm_direct<T, AA, BA, BM, BN, WM, WN, STAGES>(g, blockIdx.x, lds);
}
// A gradient's two products in one launch: small ones leave compute units idle one after the other.
template <class T, bool BA>
__global__ __launch_bounds__(256) void k_gemm_two(Gemm g0, Gemm g1, uint32_t blocks0) {
  __shared__ __attribute__((aligned(16))) char lds[DirectShape<64, 64, 2, 2, 4>::LDS];
  if (blockIdx.x < blocks0) gemm_direct<T, false, BA, 64, 64, 2, 2, 4>(g0, blockIdx.x, lds);
  else gemm_direct<T, true, true, 64, 64, 2, 2, 4>(g1, blockIdx.x - blocks0, lds);
}

// ---- few rows: the weights are read once, by vector instructions
constexpr int kFewRows = 4, kFewRound = 256;   // k of a split at least

// V values of the stored type S: as they lie in memory (the first n), and as the type they are summed in.
template <class S, int V>
struct Stored {
  static constexpr int W = V * (int)sizeof(S) / 4;
  uint32_t w[W];
  __device__ __forceinline__ void load(const char *p) { __builtin_memcpy(w, p, V * sizeof(S)); }
  __device__ __forceinline__ void load(const char *p, int n) {
    if (n >= V) {
      load(p);
      return;
    }
#pragma unroll
    for (int j = 0; j < W; j += 4) {
      const u32x4 x = some_values<S>(p + 4 * j, min(n - j * 4 / (int)sizeof(S), 16 / (int)sizeof(S)));
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (j + i < W) w[j + i] = x[i];
    }
  }
  template <class A>
  __device__ __forceinline__ void numbers(A (&f)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if constexpr (sizeof(S) == 4) f[i] = __builtin_bit_cast(float, w[i]);
      else if constexpr (__is_same(S, bf16_t)) f[i] = __builtin_bit_cast(float, i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
      else if constexpr (__is_same(S, f16_t)) f[i] = (float)__builtin_bit_cast(f16_t, (uint16_t)(w[i / 2] >> (16 * (i % 2))));
      else if constexpr (__is_same(S, int8_t)) f[i] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
      else f[i] = e4m3_value(w[i / 4], i % 4);
    }
  }
};
template <class S>
struct SumOf {
  typedef float type;
};
template <>
struct SumOf<int8_t> {
  typedef int32_t type;
};
template <class S, class A>
__device__ __forceinline__ A number(const S *p) {
  if constexpr (__is_same(S, e4m3_t)) return e4m3_value(p->bits, 0);
  else return (A)*p;
}
__device__ __forceinline__ uint64_t mul_wide(int a, uint32_t b) { return (uint64_t)(uint32_t)a * b; }
template <class A>
__device__ __forceinline__ A add_product(A a, A x, A w) {
  if constexpr (__is_same(A, float)) return fmaf(x, w, a);
  else return a + x * w;
}

// Weights across k: a block takes 64 columns, so whole lines of 128 bytes in 16 bits, eight threads a line of them and 32 lines at once;
// x goes through LDS as numbers.  k is split over blocks: a compute unit alone gets about 30 GB/s (one row of 4096 x 4096 bf16 in
// blocks that sum all of k: 64 columns each 18 us, 32 columns 15, 16 columns, a quarter of a line, 13).
template <class S, int R, int NT>
__global__ __launch_bounds__(NT) void k_few_across(Gemm g) {
  typedef typename SumOf<S>::type A;
  constexpr int LINES = NT / 8, AT = 8, ROUND = LINES * AT;   // loads on their way, k of a round
  __shared__ __attribute__((aligned(16))) A sx[ROUND][R];
  const uint32_t tn = (uint32_t)(g.n + 63) / 64, at = near_tile(blockIdx.x, gridDim.x);
  const int split = (int)(at / tn), line = threadIdx.x >> 3, col = (threadIdx.x & 7) * 8;
  const int n0 = (int)(at - split * tn) * 64 + col, count = min(g.n - n0, 8);
  const uint32_t rounds = (uint32_t)(g.k + ROUND - 1) / ROUND;
  const int begin = (int)(rounds * split / (uint32_t)g.splits) * ROUND,
            end = min(g.k, (int)(rounds * (split + 1) / (uint32_t)g.splits) * ROUND);
  A acc[R][8];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[r][i] = 0;
  const S *const px = (const S *)g.a.p;
  const char *const pw = (const char *)g.b.p + n0 * (int64_t)sizeof(S);
  const uint32_t step = (uint32_t)(g.b.ld * (int64_t)sizeof(S));   // below 2^32: plan_gemm takes few rows with ldb < 2^30 only
  for (int k0 = begin; k0 < end; k0 += ROUND) {
    Stored<S, 8> w[AT];
    if (count == 8) {
      // Lines past the end are the last one again: no branch, so that all loads are on their way before one is waited for.
#pragma unroll
      for (int j = 0; j < AT; ++j) w[j].load(pw + mul_wide(min(k0 + line + j * LINES, end - 1), step));
    }
    __builtin_amdgcn_sched_barrier(0);
    if (k0 != begin) __syncthreads();
    for (int i = threadIdx.x; i < ROUND && k0 + i < end; i += NT) {
#pragma unroll
      for (int r = 0; r < R; ++r) sx[i][r] = r < g.m ? number<S, A>(px + r * g.a.ld + k0 + i) : (A)0;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < AT; ++j) {
      const int k = k0 + line + j * LINES;
      if (k >= end) break;
      if (count < 8) w[j].load(pw + mul_wide(k, step), count);
      A f[8];
      w[j].numbers(f);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const A x = sx[line + j * LINES][r];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[r][i] = add_product(acc[r][i], x, f[i]);
      }
    }
  }
  // The lines' sums: eight of them in a wavefront by exchanges, then over the wavefronts.
  __shared__ A part[NT / 64][R][64];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      A v = acc[r][i];
#pragma unroll
      for (int x = 8; x < 64; x *= 2) v += __shfl_xor(v, x);
      if ((threadIdx.x & 63) < 8) part[threadIdx.x >> 6][r][col + i] = v;
    }
  __syncthreads();
  const int r = threadIdx.x >> 3;
  if (r >= R || r >= g.m || count <= 0) return;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    A t = part[0][r][col + i];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) t += part[w][r][col + i];
    v[i] = g.part ? __builtin_bit_cast(float, t) : (float)t;
  }
  if (g.part) store_part<float, 8>((float *)g.part + ((int64_t)split * g.m + r) * g.n + n0, count, v);
  else finish<8>(g.e, r, n0, count, v);
}

// Weights along k: a wavefront takes two columns.
template <class S, int R>
__global__ __launch_bounds__(256) void k_few_along(Gemm g) {
  typedef typename SumOf<S>::type A;
  constexpr int E = 16 / (int)sizeof(S);
  const int lane = threadIdx.x & 63;
  const int n0 = ((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6)) * 2;
  if (n0 >= g.n) return;
  const int64_t n1 = n0 + 1 < g.n ? n0 + 1 : n0;
  const char *const px = (const char *)g.a.p, *const p0 = (const char *)g.b.p + (int64_t)n0 * g.b.ld * (int64_t)sizeof(S),
             *const p1 = (const char *)g.b.p + n1 * g.b.ld * (int64_t)sizeof(S);
  A acc[R][2];
#pragma unroll
  for (int r = 0; r < R; ++r) acc[r][0] = acc[r][1] = 0;
  for (int k = lane * E; k < g.k; k += 64 * E) {
    const int n = min(g.k - k, E);
    Stored<S, E> v0, v1, v;
    v0.load(p0 + k * (int64_t)sizeof(S), n);
    v1.load(p1 + k * (int64_t)sizeof(S), n);
    A w0[E], w1[E], x[E];
    v0.numbers(w0);
    v1.numbers(w1);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r >= g.m) break;
      v.load(px + (r * g.a.ld + k) * (int64_t)sizeof(S), n);
      v.numbers(x);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        acc[r][0] = add_product(acc[r][0], x[i], w0[i]);
        acc[r][1] = add_product(acc[r][1], x[i], w1[i]);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      A v = acc[r][c];
#pragma unroll
      for (int x = 1; x < 64; x *= 2) v += __shfl_xor(v, x);
      acc[r][c] = v;
    }
  if (lane == 0) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r >= g.m) break;
      float v[4] = {(float)acc[r][0], (float)acc[r][1], 0, 0};
      finish<4>(g.e, r, n0, g.n - n0 < 2 ? 1 : 2, v);
    }
  }
}
template <class S, int R>
hipError_t launch_few_rows(const Gemm &g, hipStream_t s) {
  // Blocks that sum all of k need its lines on their way at once: 1024 x 1024 bf16 8.1 us in blocks of 256 threads, 5 in those of 1024.
  if (!g.b.across) k_few_along<S, R><<<dim3((unsigned)((g.n + 7) / 8)), 256, 0, s>>>(g);
  else if (g.splits == 1) k_few_across<S, R, 1024><<<dim3((unsigned)((g.n + 63) / 64)), 1024, 0, s>>>(g);
  else k_few_across<S, R, 256><<<dim3((unsigned)((g.n + 63) / 64 * g.splits)), 256, 0, s>>>(g);
  return hipGetLastError();
}
template <class S>
hipError_t launch_few(const Gemm &g, hipStream_t s) {
  return g.m == 1 ? launch_few_rows<S, 1>(g, s) : g.m == 2 ? launch_few_rows<S, 2>(g, s) : launch_few_rows<S, 4>(g, s);
}

template <int BM, int BN>
unsigned blocks_of(const Gemm &g) {
  return (unsigned)((int64_t)((g.m + BM - 1) / BM) * ((g.n + BN - 1) / BN) * g.splits);
}
template <class T, class S, bool AA, bool BA, int BM, int BN, int WM, int WN>
hipError_t launch_tile(const Gemm &g, hipStream_t s) {
  k_gemm<T, S, AA, BA, BM, BN, WM, WN><<<dim3(blocks_of<BM, BN>(g)), dim3(WM * WN * 64), 0, s>>>(g);
  return hipGetLastError();
}
template <class T, bool AA, bool BA, int BM, int BN, int WM, int WN, int STAGES>
hipError_t launch_direct(const Gemm &g, hipStream_t s) {
  k_gemm_direct<T, AA, BA, BM, BN, WM, WN, STAGES><<<dim3(blocks_of<BM, BN>(g)), dim3(WM * WN * 64), 0, s>>>(g);
  return hipGetLastError();
}

// Whether k_gemm_direct takes a factor of `rows` rows: whole pieces at 16-byte addresses, offsets in a tile of 256 rows within 2^31.
template <class T>
bool direct_ok(const Factor &f, int rows, int k) {
  constexpr int64_t E = 16 / sizeof(T);
  return (uintptr_t)f.p % 16 == 0 && f.ld % E == 0 && (f.packed || (f.across ? rows : k) % E == 0) &&
         f.ld < ((int64_t)1 << 22) / (int64_t)sizeof(T);
}
template <class T>
bool direct_ok(const Gemm &g) {
  return direct_ok<T>(g.a, g.m, g.k) && direct_ok<T>(g.b, g.n, g.k);
}

// The tiles that plan_gemm chooses from.  What a tile of BM x BN costs beside its products is reading BM + BN lines of k: with 256 x 256
// and eight wavefronts of 128 x 64 the matrix instructions are busy 63 % of the clocks, which fall to 1.75 GHz under them (8192 x 4096
// x 4096 bf16 245 us a product, 1.1 PFLOP/s; with 128 x 128 415 us).  The two stages of it fill LDS, so one block a compute unit, whose
// epilogue nothing overlaps: about 60 of the 1040 us of 16384 x 4096 -> 8192 with GELU and z.  Where 256 x 256 would leave compute units
// idle, or k is short, 128 x 128 with two blocks a unit (49152 x 128 -> 512 int8 49 -> 41 us); for small products 64 x 64 with four
// stages, as their time is loads' latency.
constexpr int kTileSide[3][2] = {{64, 64}, {128, 128}, {256, 256}};
template <class T, class S, bool AA, bool BA>
hipError_t launch_layout(const Gemm &g, const GemmPlan &p, hipStream_t s) {
  if ((__is_same(T, S) || g.a.packed) && direct_ok<T>(g)) {
    if constexpr (sizeof(T) < 4) {
      if (p.tile == 2) return launch_direct<T, AA, BA, 256, 256, 2, 4, 2>(g, s);
    }
    if constexpr (!AA) {
      if (p.tile >= 1 && g.k * (int64_t)sizeof(T) <= 128) return launch_direct<T, AA, BA, 128, 128, 2, 2, 1>(g, s);
    }
    if (p.tile >= 1) return launch_direct<T, AA, BA, 128, 128, 2, 2, 2>(g, s);
    return launch_direct<T, AA, BA, 64, 64, 2, 2, 4>(g, s);
  }
  if (p.tile == 0) return launch_tile<T, S, AA, BA, 64, 64, 2, 2>(g, s);
  return launch_tile<T, S, AA, BA, 128, 128, 2, 2>(g, s);
}
// Codes are never a gradient's factor, so a of theirs lies along k.
template <class T, class S>
hipError_t launch_one(const Gemm &g, const GemmPlan &p, hipStream_t s) {
  if (g.m == 0 || g.n == 0) return hipSuccess;
  if (p.few) return g.a.across ? hipErrorInvalidValue : launch_few<S>(g, s);
  if constexpr (sizeof(S) > 1) {
    if (g.a.across && g.b.across) return launch_layout<T, S, true, true>(g, p, s);
  }
  if (g.a.across) return hipErrorInvalidValue;
  return g.b.across ? launch_layout<T, S, false, true>(g, p, s) : launch_layout<T, S, false, false>(g, p, s);
}
template <class T, class S = T>
hipError_t launch_type(const Gemm *g, const GemmPlan *p, int count, hipStream_t s) {
  if constexpr (sizeof(S) > 1) {
    if (count == 2 && !p[0].few && !p[1].few && p[0].tile == 0 && p[1].tile == 0 && g[0].m > 0 && direct_ok<T>(g[0]) && direct_ok<T>(g[1])) {
      const unsigned first = blocks_of<64, 64>(g[0]), all = first + blocks_of<64, 64>(g[1]);
      if (g[0].b.across) k_gemm_two<T, true><<<dim3(all), 256, 0, s>>>(g[0], g[1], first);
      else k_gemm_two<T, false><<<dim3(all), 256, 0, s>>>(g[0], g[1], first);
      return hipGetLastError();
    }
  }
  for (int i = 0; i < count; ++i) {
    const hipError_t err = launch_one<T, S>(g[i], p[i], s);
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace aecct
