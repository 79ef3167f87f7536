// Linear maps: which tile and how many splits a product takes, and what its gradient needs besides products.
#include <type_traits>

#include "gemm.h"

namespace aecct {

namespace {

// fp32: the matrix instructions' time is nearly all there is, so what counts is the blocks of the fullest compute unit.  Microseconds by
// what was measured (512 x 512 x 512 to 4096 x 4096 x 4096, 26 x 6912 -> 4096, 7717 x 5144 -> 128): a tile of k of 128 x 128 outputs
// 2.0, of 64 x 64 0.6 beside others and 0.7 alone; joining splits 4 and what their sums take at 6.5 TB/s.  (With the rule for 16 bits 288
// blocks of 128 x 128 took two rounds: 2048 x 2048 -> 2304 257 us, k split in five 183; 1280 x 4096 -> 3840 504 and 334; 672 x 6352 ->
// 1024 122 and 94.)
void plan_f32(GemmPlan &p, int64_t m, int64_t n, int64_t tiles64, int64_t tiles128, int64_t kt) {
  double best = 0;
  for (int tile = 0; tile < 2; ++tile)
    for (int64_t s = 1; s <= 64; ++s) {
      const int64_t blocks = (tile ? tiles128 : tiles64) * s, rounds = (blocks + 255) / 256;
      if (s > 1 && (kt / s < 4 || rounds > 8)) break;
      const double each = tile ? 2.0 : rounds > 1 ? 0.6 : 0.7;
      const double time = (double)(rounds * ((kt + s - 1) / s)) * each + (s > 1 ? 4 + (double)(s * m * n) * 8 / 6.5e6 : 0);
      if ((tile == 0 && s == 1) || time < best) {
        best = time;
        p.tile = tile;
        p.splits = (int)s;
      }
    }
  if (p.splits > 1) p.part_bytes = (size_t)(p.splits * m * n * 4);
}

}  // namespace

GemmPlan plan_gemm(int type, int64_t m, int64_t n, int64_t k, bool across_a, bool across_b, int64_t ldb, bool whole) {
  GemmPlan p{false, 1, 1, 0};
  const int64_t size = type == AECCT_F32 ? 4 : type == kCodeType + AECCT_CODE_I8 ? 1 : 2;   // of a value in LDS
  if (m <= kFewRows && !across_a && ldb < (int64_t)1 << 30) {
    p.few = true;
    const int64_t t = (n + 63) / 64, rounds = (k + kFewRound - 1) / kFewRound;
    // Weights of less than 4 MB are read in less time than a second launch takes.
    if (across_b && m > 0 && t < 512 && n * k * size >= ((int64_t)4 << 20)) {
      p.splits = (int)(1024 / t < rounds ? 1024 / t : rounds);
      if (p.splits > 16) p.splits = 16;
      if (p.splits > 1) p.part_bytes = (size_t)(p.splits * m * n * 4);
    }
    return p;
  }
  auto tiles = [&](int t) { return (m + kTileSide[t][0] - 1) / kTileSide[t][0] * ((n + kTileSide[t][1] - 1) / kTileSide[t][1]); };
  if (type == AECCT_F32) {
    plan_f32(p, m, n, tiles(0), tiles(1), (k + 31) / 32);
    return p;
  }
  if (tiles(1) < 192) p.tile = 0;
  else if (tiles(2) >= 256 && k * size >= 1024) p.tile = 2;
  const int64_t t = tiles(p.tile), kt = (k * size + 127) / 128;
  // k is split where that fills the card (two blocks a compute unit), not into less than what a launch that joins the sums costs: 16
  // tiles where pieces go past the registers, four tiles ahead, 4 where they go through them.  (Gradient of 1001 x 777 -> 1333 fp16 with
  // 4 in both: 32.8 us, with 16: 28.)
  if (t > 0 && t < 256) {
    int64_t s = 512 / t;
    if (s > kt / (whole ? 16 : 4)) s = kt / (whole ? 16 : 4);
    if (s > 64) s = 64;
    p.splits = s > 1 ? (int)s : 1;
  }
  if (p.splits > 1) p.part_bytes = (size_t)(p.splits * m * n * 4);
  return p;
}

hipError_t launch_gemm(int type, const Gemm *g, const GemmPlan *plan, int count, hipStream_t s) {
  switch (type) {
    case AECCT_F32: return launch_gemm_f32(g, plan, count, s);
    case AECCT_BF16: return launch_gemm_bf16(g, plan, count, s);
    case AECCT_F16: return launch_gemm_f16(g, plan, count, s);
    case kCodeType + AECCT_CODE_I8: return launch_gemm_i8(g, plan, count, s);
    case kCodeType + AECCT_CODE_E4M3: return launch_gemm_e4m3(g, plan, count, s);
    default: return hipErrorInvalidValue;
  }
}

namespace {

// act'(z).  Where a factor is 0 the other may be infinite: such a product's limit is 0.
template <bool F32>
__device__ __forceinline__ float slope(float z, int act) {
  if (act == kActRelu) return z > 0.0f ? 1.0f : z != z ? z : 0.0f;
  if (act == kActGelu) {
    float e;
    const float phi = normal<F32>(z, e), density = e * 0.39894228040143268f;
    return phi + (density == 0.0f ? 0.0f : z * density);
  }
  float q;
  const float p = logistic<F32>(z, q);
  if (p == 0.0f || q == 0.0f) return p;
  return p * (1.0f + z * q);
}

constexpr int kSlopeColumns = 128;   // 16 threads of 8 values a row, 16 rows at once

// dz is rounded to the type, as the products take it: dx and dw are what the formula gives with that dz, 2.35e-3 (bf16) and 2.9e-4 (fp16) of
// their norms from 64 bits where their own rounding alone is 1.66e-3 and 2.1e-4; a second product of what the rounding leaves
// would double the gradient's time.  The sums take dz unrounded.
template <class T>
__device__ __forceinline__ void slope_block(const Slope &a, uint32_t block, uint32_t across) {
  const uint32_t by = block / across, bx = block - by * across;
  const int64_t stride = a.blocks * 16;
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int n0 = (int)bx * kSlopeColumns + c * 8, count = min(a.n - n0, 8);
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (count > 0) {
    for (int64_t row = (int64_t)by * 16 + r; row < a.rows; row += stride) {
      float d[8];
      load_part<T, 8>((const T *)a.dy + row * a.lddy + n0, count, d);
      if (a.z) {
        float z[8];
        load_part<T, 8>((const T *)a.z + row * a.ldz + n0, count, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] *= slope<sizeof(T) == 4>(z[i], a.act);
        if (a.dz) {   // zeros behind the row's end
          float e[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) e[i] = i < count ? d[i] : 0.0f;
          store_part<T, 8>((T *)a.dz + row * a.lddz + n0, (int)a.lddz - n0, e);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += d[i];
    }
  }
  if (!a.part) return;
  __shared__ float s[16][kSlopeColumns + 4];
#pragma unroll
  for (int i = 0; i < 8; ++i) s[r][c * 8 + i] = sum[i];
  __syncthreads();
  if (threadIdx.x < kSlopeColumns) {
    const int n = (int)bx * kSlopeColumns + threadIdx.x;
    float t = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += s[i][threadIdx.x];
    if (n < a.n) a.part[(int64_t)by * a.n + n] = t;
  }
}
// Pieces of the copy, one a thread and turn.
template <class S>
__device__ __forceinline__ void pack_block(const Pack &a, uint32_t block, uint32_t blocks) {
  constexpr int E = __is_same(S, e4m3_t) ? 8 : 16 / (int)sizeof(S), OUT = __is_same(S, e4m3_t) ? 2 : (int)sizeof(S);
  typedef std::conditional_t<__is_same(S, e4m3_t), f16_t, S> T;
  const uint32_t per = (uint32_t)(a.ldto / E);
  const uint64_t all = (uint64_t)a.lines * per;
  for (uint64_t at = (uint64_t)block * 256 + threadIdx.x; at < all; at += (uint64_t)blocks * 256) {
    const uint32_t line = at >> 32 == 0 ? (uint32_t)at / per : (uint32_t)(at / per), c = (uint32_t)(at - (uint64_t)line * per);
    const char *const p = (const char *)a.from + ((int64_t)line * a.ld + c * E) * (int64_t)sizeof(S);
    const int n = a.width - (int)c * E;
    const u32x4 v = n >= E ? piece<T, S>(p) : n > 0 ? piece<T, S>(p, n) : u32x4{0, 0, 0, 0};
    *(u32x4 *)((char *)a.to + ((int64_t)line * a.ldto + c * E) * OUT) = v;
  }
}
struct PrepareGrid {
  uint32_t across, slope, pack[3];     // blocks
};
template <class S>
__global__ __launch_bounds__(256) void k_prepare(Prepare p, PrepareGrid grid) {
  uint32_t block = blockIdx.x;
  if constexpr (sizeof(S) > 1) {
    if (block < grid.slope) {
      slope_block<S>(p.slope, block, grid.across);
      return;
    }
    block -= grid.slope;
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (block < grid.pack[i]) {
      pack_block<S>(p.pack[i], block, grid.pack[i]);
      return;
    }
    block -= grid.pack[i];
  }
}

// The splits' sums of four outputs a thread, in the order of the splits, and the epilogue.
template <bool INT>
__device__ __forceinline__ void join_block(const Gemm &g, uint32_t block) {
  const uint32_t per = (uint32_t)(g.n + 3) / 4, at = block * 256 + threadIdx.x;
  const int m = (int)(at / per), n = (int)(at - m * per) * 4;
  if (m >= g.m) return;
  const int count = min(g.n - n, 4);
  float v[4] = {0, 0, 0, 0};
  int32_t w[4] = {0, 0, 0, 0};
  const float *const part = (const float *)g.part + (int64_t)m * g.n + n;
  for (int s = 0; s < g.splits; s += 8) {
    float p[8][4];
#pragma unroll
    for (int j = 0; j < 8; ++j) load_part<float, 4>(part + (int64_t)min(s + j, g.splits - 1) * g.m * g.n, count, p[j]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (s + j >= g.splits) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (INT) w[i] += __builtin_bit_cast(int32_t, p[j][i]);
        else v[i] += p[j][i];
      }
    }
  }
  if constexpr (INT) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)w[i];
  }
  finish<4>(g.e, m, n, count, v);
}
// 16 columns of the column sums, 16 threads each.
__device__ __forceinline__ void column_block(const Finish &f, uint32_t block) {
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, at = (int)block * 16 + c;
  float t = 0;
  if (at < f.n)
    for (int b = r; b < f.blocks; b += 16) t += f.part[(int64_t)b * f.n + at];
  __shared__ float s[16][17];
  s[r][c] = t;
  __syncthreads();
  if (r || at >= f.n) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) t += s[i][c];
  f.out[at] = t;
}
template <bool INT>
__global__ __launch_bounds__(256) void k_finish(Finish f, uint32_t first, uint32_t second) {
  if (blockIdx.x < first) join_block<INT>(f.g[0], blockIdx.x);
  else if (blockIdx.x < second) join_block<INT>(f.g[1], blockIdx.x - first);
  else column_block(f, blockIdx.x - second);
}

}  // namespace

int64_t slope_blocks(int64_t rows, int64_t n) {
  const int64_t across = (n + kSlopeColumns - 1) / kSlopeColumns;
  int64_t b = (1024 + across - 1) / across;
  const int64_t most = (rows + 15) / 16;
  if (b > most) b = most;
  return b < 1 ? 1 : b;
}

hipError_t launch_prepare(int type, const Prepare &p, hipStream_t s) {
  PrepareGrid grid{};
  if (p.slope.n) {
    grid.across = (uint32_t)((p.slope.n + kSlopeColumns - 1) / kSlopeColumns);
    grid.slope = grid.across * (uint32_t)slope_blocks(p.slope.rows, p.slope.n);
  }
  int64_t all = grid.slope;
  for (int i = 0; i < 3; ++i) {
    const int64_t pieces = (int64_t)p.pack[i].lines * (p.pack[i].ldto / (16 / type_bytes(type)));
    grid.pack[i] = p.pack[i].lines ? (uint32_t)(pieces < (int64_t)1 << 24 ? (pieces + 255) / 256 : 1 << 16) : 0;
    all += grid.pack[i];
  }
  if (all == 0) return hipSuccess;
  const dim3 blocks((unsigned)all);
  switch (type) {
    case AECCT_F32: k_prepare<float><<<blocks, 256, 0, s>>>(p, grid); break;
    case AECCT_BF16: k_prepare<bf16_t><<<blocks, 256, 0, s>>>(p, grid); break;
    case AECCT_F16: k_prepare<f16_t><<<blocks, 256, 0, s>>>(p, grid); break;
    case kCodeType + AECCT_CODE_I8: k_prepare<int8_t><<<blocks, 256, 0, s>>>(p, grid); break;
    case kCodeType + AECCT_CODE_E4M3: k_prepare<e4m3_t><<<blocks, 256, 0, s>>>(p, grid); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_finish(int type, const Finish &f, hipStream_t s) {
  uint32_t blocks[3] = {0, 0, 0};
  for (int i = 0; i < 2; ++i)
    if (f.g[i].part) blocks[i] = (uint32_t)(((int64_t)f.g[i].m * ((f.g[i].n + 3) / 4) + 255) / 256);
  if (f.part) blocks[2] = (uint32_t)((f.n + 15) / 16);
  const uint32_t all = blocks[0] + blocks[1] + blocks[2];
  if (all == 0) return hipSuccess;
  if (type == kCodeType + AECCT_CODE_I8) k_finish<true><<<dim3(all), 256, 0, s>>>(f, blocks[0], blocks[0] + blocks[1]);
  else k_finish<false><<<dim3(all), 256, 0, s>>>(f, blocks[0], blocks[0] + blocks[1]);
  return hipGetLastError();
}

}  // namespace aecct
