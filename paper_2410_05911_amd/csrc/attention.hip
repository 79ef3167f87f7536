// Cross attention in one pass over the keys: o = softmax(scale q k^T) v with the running maximum and sum of each row (softmax in
// base 2, on scores times log2(e)).
//
// A wavefront takes 32 rows (queries of the heads that share a key head).  It computes the scores turned, keys by rows, so that a
// lane holds 16 keys of one row: the maximum and sum are taken in registers with one exchange between the halves, and the
// weights are, as they lie, the second factor of the product with the values.
//
// What bounds it: many rows, the matrix instructions (50 % of the clocks) and the vector ones (52 %, half of them exponentials), which
// two wavefronts a SIMD overlap little (2 x 4096 queries on 2111 keys, 32 heads of 128, bf16: 290 us, 0.89 PFLOP/s; one wavefront a
// SIMD 577).  Scores a tile ahead in the same wavefront, wavefront priorities and sums that begin with kept zeros were measured
// without gain.  Few rows, memory: one query on 8192 keys, 16 sequences, 8 key heads of 128, bf16 in 89 us (4.5 TB/s).
//
// With 16-bit types the weights are rounded to the type, as the matrix instructions take them; their sum takes them unrounded.  o is then as
// far from 64 bits as two such roundings (bf16 2.3e-3 of its norm, fp16 2.8e-4), its own alone 1.66e-3 and 2.1e-4: two
// products instead, of the weights and of what their rounding leaves, would add half the matrix instructions again.
#include "attention_tile.h"

namespace aecct {
namespace {

// In fp16 the weights are taken times 2^10, so that those of long rows stay in its normal range (at most 2^10, the sum in
// fp32 takes the factor out again).
template <class T>
__device__ constexpr float weight_shift() { return __is_same(T, f16_t) ? 10.0f : 0.0f; }

// How far a row's scores (times log2(e)) may pass its reference before the sums are scaled down to a new one: weights stay below 2^8,
// in fp16 with its factor below 2^15.  Most tiles then leave the sums alone.
template <class T>
__device__ constexpr float slack() { return __is_same(T, f16_t) ? 5.0f : 8.0f; }

// WQ wavefronts take 32 rows each and share the tiles of keys, or (WQ = 1) WK wavefronts the same 32 rows and different keys.
// DIRECT: keys and values go from memory to LDS past the registers, a tile ahead where two fit.  Rows of 128 bytes are held to the
// registers of three wavefronts a SIMD (four: they spill, 256 x 128 under a Tanner graph 26 -> 34 us), wider ones to those of two.
template <class T, int DP, int WQ, int WK, bool MASK, bool DIRECT>
__global__ __launch_bounds__(WQ *WK * 64, DP * sizeof(T) <= 128 ? 3 : DP * sizeof(T) <= 256 ? 2 : 1) void k_attention(Attention a) {
  constexpr int RB = DP * (int)sizeof(T), FD = DP / 32, NT = WQ * WK * 64;
  constexpr int SUB = WK == 1 && RB <= 256 ? 2 : 1, KT = 32 * SUB * WK;   // keys of a tile
  constexpr int STAGES = DIRECT && 4 * KT * RB <= 131072 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) char lds[STAGES * 2 * KT * RB];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5;
  const int wq = WK == 1 ? wave : 0, wk = WK == 1 ? 0 : wave;
  const uint32_t group = a.heads / a.kv_heads, queries = (uint32_t)a.queries, rows = group * queries;
  const uint32_t row_blocks = (rows + 32 * WQ - 1) / (32 * WQ), pairs = (uint32_t)a.batch * a.kv_heads;
  const uint32_t at = near_block(blockIdx.x, gridDim.x), rest = at / row_blocks, row_block = at - rest * row_blocks;
  const uint32_t pair = a.splits > 1 ? rest / (uint32_t)a.splits : rest, split = rest - pair * (uint32_t)a.splits * (a.splits > 1);
  const uint32_t b = pair / (uint32_t)a.kv_heads, kh = pair - b * a.kv_heads;
  const int length = length_of(a, b);
  // This block's tiles of keys.
  const int tiles = (length + KT - 1) / KT;
  int t0 = 0, t1 = tiles;
  if (a.splits > 1) {
    t0 = (int)((uint32_t)tiles * split / (uint32_t)a.splits);
    t1 = (int)((uint32_t)tiles * (split + 1) / (uint32_t)a.splits);
  }
  // This lane's row.
  const uint32_t r = row_block * (32 * WQ) + wq * 32 + (lane & 31), rc = min(r, rows - 1);
  const uint32_t head = kh * group + rc / queries, query = rc % queries;
  const bool idle = row_block * (32 * WQ) + wq * 32 >= rows;   // the whole wavefront's rows are past the last
  Keys<T, RB, KT, NT, DIRECT> keys(a.k, a, b, kh, length), values(a.v, a, b, kh, length);
  const int words = (int)words_of(a.keys);
  const uint32_t *const mask = MASK ? a.words + (int64_t)query * words + wk * SUB : nullptr;
  // Tiles of keys that none of the block's rows may attend are passed over: 64 tiles are looked up at once.
  uint64_t want = 0;
  int want0 = t0 - 64;
  auto from = [&](int t) {   // the first tile to be done from t on
    if constexpr (!MASK) return t;
    while (t < t1) {
      if (t - want0 >= 64) {
        want0 = t;
        want = __ballot(any_flag<32 * WQ, KT>(a, row_block * (32 * WQ), min(t + lane, t1 - 1) * KT) && t + lane < t1);
      }
      const uint64_t left = want >> (t - want0);
      if (left) return t + __builtin_ctzll(left);
      t = want0 + 64;
    }
    return t1;
  };

  f32x16 acc[FD];
#pragma unroll
  for (int f = 0; f < FD; ++f)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[f][i] = 0;
  float m = -INFINITY, sum = 0;   // the row's reference, and its sum of 2^(score - reference)
  const float to2 = a.scale * kLog2e;

  // Scales the sums down to a new reference where a score passes the old one by too much.
  auto refer = [&](float top) {
    if (!__any(top > m + slack<T>())) return;
    const float now = top > m + slack<T>() ? top : m;
    // A row that has met no key it may attend keeps the reference -inf; its weights are 2^-inf = 0.
    const float down = __builtin_amdgcn_exp2f(m - (now == -INFINITY ? 0.0f : now));
    m = now;
    sum *= down;
#pragma unroll
    for (int f = 0; f < FD; ++f)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[f][i] *= down;
  };

  int t = from(t0), buf = 0;
  uint32_t w[SUB] = {}, w_next[SUB] = {};   // what the lane's row may attend of the tile
  auto look = [&](int t, uint32_t (&w)[SUB]) {
    if constexpr (MASK) {
#pragma unroll
      for (int u = 0; u < SUB; ++u) w[u] = t * (KT / 32) + wk * SUB + u < words ? mask[t * (KT / 32) + u] : 0;
    }
  };
  if (t < t1) {
    if constexpr (!DIRECT || STAGES == 2) {
      keys.load(lds, t);
      values.load(lds + KT * RB, t);
    }
    look(t, w_next);
  }
  // (behind the first tile, which is on its way by now)
  u32x4 q[RB / 32];
  {
    const char *const p = (const char *)a.q.p + (b * a.q.batch + query * a.q.row + head * a.q.head) * (int64_t)sizeof(T);
    const char *const end = end_of(a.q, a.batch, a.queries, a.heads, a.d, sizeof(T));
#pragma unroll
    for (int c = 0; c < RB / 32; ++c) q[c] = row_piece<T>(p, 2 * c + h, a.d, end);
  }
  while (t < t1) {
    const int next = from(t + 1);
    char *const lk = lds + buf * 2 * KT * RB, *const lv = lk + KT * RB;
#pragma unroll
    for (int u = 0; u < SUB; ++u) w[u] = w_next[u];
    if constexpr (DIRECT && STAGES == 2) {
      wait_loads();
      barrier();         // the tile is there for all, and nobody reads the other one any more
      if (next < t1) {
        keys.load(lds + (buf ^ 1) * 2 * KT * RB, next);
        values.load(lds + (buf ^ 1) * 2 * KT * RB + KT * RB, next);
      }
      buf ^= 1;
    } else if constexpr (DIRECT) {
      barrier();         // the tile before has been read
      keys.load(lk, t);
      values.load(lv, t);
      wait_loads();
      barrier();
    } else {
      barrier();
      keys.store(lk);
      values.store(lv);
      barrier();
      if (next < t1) {
        keys.load(nullptr, next);
        values.load(nullptr, next);
      }
    }
    if (next < t1) look(next, w_next);
    const int key0 = t * KT + wk * 32 * SUB;
    bool none = idle || key0 >= length;
    if constexpr (MASK) {
      uint32_t any = 0;
#pragma unroll
      for (int u = 0; u < SUB; ++u) any |= w[u];
      none = none || !__any(any != 0);
    }
    bool dense = !none;
    if constexpr (MASK && pairwise<T, RB>()) {
      uint64_t in = w[0];
      if constexpr (SUB == 2) in |= (uint64_t)w[1] << 32;
      if (key0 + 32 * SUB > length) in = length > key0 ? in & (((uint64_t)1 << (length - key0)) - 1) : 0;
      if (dense && !__any(__popcll(in) > kFewPairs * SUB)) {
        dense = false;
        while (__any(in != 0)) {
          const int j = in ? __builtin_ctzll(in) : 0, row = wk * SUB * 32 + j;
          const float score = sum_halves(HalfRow<RB>(lk, row, a.d).dot(q, a.d)) * to2;
          const float s = in ? score : -INFINITY;
          refer(s);
          const float p = __builtin_amdgcn_exp2f(s - (m == -INFINITY ? 0.0f : m));
          sum += h == 0 ? p : 0.0f;      // both halves have it
          // (a lane that has no pair left: no value that it may not see)
          if (in) HalfRow<RB>(lv, row, a.d).add_to(acc, p, a.d);
          in &= in - 1;
        }
      }
    }
    if (dense) {
      float s[SUB][16];
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const f32x16 x = times_rows<T, RB, false>(lk, (wk * SUB + u) * 32, q, a.d);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[u][i] = x[i];
      }
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const int k0 = key0 + u * 32;
        if constexpr (MASK) {
          uint32_t in = w[u];
          if (k0 + 32 > length) in = length > k0 ? in & ((1u << (length - k0)) - 1) : 0;
          if (pairwise<T, RB>() || !__all(in == ~0u)) {   // (where pairs are taken one by one this branch costs the registers of a wavefront)
            in >>= 4 * h;
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (!(in >> row_of(i, 0) & 1)) s[u][i] = -INFINITY;
          }
        } else if (k0 + 32 > length) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (k0 + row_of(i, h) >= length) s[u][i] = -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
      }
      top = max_halves(top) * to2;
      refer(top);
      const float lift = (m == -INFINITY ? 0.0f : m) - weight_shift<T>();
      float part[4] = {0, 0, 0, 0};
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[u][i] = __builtin_amdgcn_exp2f(fmaf(s[u][i], to2, -lift));
          part[i & 3] += s[u][i];
        }
        add_columns<T, RB, false>(acc, lv, (wk * SUB + u) * 32, s[u], a.d);
      }
      sum += (part[0] + part[1]) + (part[2] + part[3]);
    }
    t = next;
  }
  sum = sum_halves(sum);

  if constexpr (WK > 1) {
    // The wavefronts' shares of the keys are joined through LDS.
    constexpr int LD = DP;
    static_assert(STAGES * 2 * KT * RB >= WK * 32 * LD * 4, "the sums fit where the tiles were");
    __shared__ float ml[WK][32][2];
    __syncthreads();
    if (h == 0) {
      ml[wk][lane][0] = m;
      ml[wk][lane][1] = sum;
    }
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < WK; ++w) top = fmaxf(top, ml[w][lane & 31][0]);
    const float base = top == -INFINITY ? 0.0f : top;
    sum = 0;
#pragma unroll
    for (int w = 0; w < WK; ++w) sum += ml[w][lane & 31][1] * __builtin_amdgcn_exp2f(ml[w][lane & 31][0] - base);
    const float down = __builtin_amdgcn_exp2f(m - base);
    m = top;
    float *const o = (float *)lds;
#pragma unroll
    for (int f = 0; f < FD; ++f)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        f32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = acc[f][i + j] * down;
        // groups of four values exchanged by the row, so that the 32 rows fall on different banks
        *(f32x4 *)(o + (wk * 32 + (lane & 31)) * LD + ((32 * f + row_of(i, h)) ^ ((lane & 7) << 2))) = v;
      }
    __syncthreads();
    // Wavefront w finishes the columns of its share of f.
#pragma unroll
    for (int f = 0; f < FD; ++f) {
      if (f % WK != wk) continue;
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        f32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WK; ++w)
          v += *(const f32x4 *)(o + (w * 32 + (lane & 31)) * LD + ((32 * f + row_of(i, h)) ^ ((lane & 7) << 2)));
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[f][i + j] = v[j];
      }
    }
  }

  if (r >= rows) return;
  if (a.splits > 1) {
    const int64_t at_row = (int64_t)(split * pairs + pair) * rows + r;
    if (h == 0 && wk == 0) {
      a.part_ml[at_row * 2] = m;
      a.part_ml[at_row * 2 + 1] = sum;
    }
    float *const o = a.part_o + at_row * DP;
#pragma unroll
    for (int f = 0; f < FD; ++f) {
      if (WK > 1 && f % WK != wk) continue;
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(f32x4 *)(o + 32 * f + row_of(i, h)) = f32x4{acc[f][i], acc[f][i + 1], acc[f][i + 2], acc[f][i + 3]};
    }
    return;
  }
  const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
  if (a.lse && h == 0 && wk == 0)
    a.lse[(int64_t)(b * a.heads + head) * queries + query] = sum == 0.0f ? -INFINITY : (m + (__log2f(sum) - weight_shift<T>())) * kLn2;
  T *const o = (T *)a.o.p + b * a.o.batch + query * a.o.row + head * a.o.head;
#pragma unroll
  for (int f = 0; f < FD; ++f) {
    if (WK > 1 && f % WK != wk) continue;
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int c = 32 * f + row_of(i, h);
      if (c < a.d) store_values4<T>(o + c, a.d - c, acc[f][i] * over, acc[f][i + 1] * over, acc[f][i + 2] * over, acc[f][i + 3] * over);
    }
  }
}

// The splits' sums of four columns of a row a thread, in the order of the splits.
template <class T>
__global__ __launch_bounds__(256) void k_join_attention(Attention a, int dp) {
  const uint32_t group = a.heads / a.kv_heads, per = dp / 4, queries = (uint32_t)a.queries, rows = group * queries;
  const int64_t all = (int64_t)a.batch * a.kv_heads * rows;
  const uint32_t at = blockIdx.x * 256 + threadIdx.x, row = at / per, c = (at - row * per) * 4;
  if (row >= all) return;
  float m = -INFINITY, sum = 0;
  for (int s = 0; s < a.splits; ++s) m = fmaxf(m, a.part_ml[(s * all + row) * 2]);
  const float base = m == -INFINITY ? 0.0f : m;
  float v[4] = {0, 0, 0, 0};
  for (int s = 0; s < a.splits; ++s) {
    const float down = __builtin_amdgcn_exp2f(a.part_ml[(s * all + row) * 2] - base);
    sum += a.part_ml[(s * all + row) * 2 + 1] * down;
    const f32x4 o = *(const f32x4 *)(a.part_o + (s * all + row) * dp + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += o[i] * down;
  }
  const uint32_t pair = row / rows, r = row - pair * rows, b = pair / (uint32_t)a.kv_heads;
  const uint32_t head = (pair - b * a.kv_heads) * group + r / queries, query = r % queries;
  const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
  if (a.lse && c == 0)
    a.lse[(int64_t)(b * a.heads + head) * queries + query] = sum == 0.0f ? -INFINITY : (m + (__log2f(sum) - weight_shift<T>())) * kLn2;
  if ((int)c < a.d)
    store_values4<T>((T *)a.o.p + b * a.o.batch + query * a.o.row + head * a.o.head + c, a.d - (int)c, v[0] * over, v[1] * over,
                     v[2] * over, v[3] * over);
}

// Nonzero bytes of w as its four low bits.
__device__ __forceinline__ uint32_t nonzero4(uint32_t w) {
  const uint32_t t = ((((w & 0x7f7f7f7fu) + 0x7f7f7f7fu) | w) >> 7) & 0x01010101u;
  return (t * 0x01020408u) >> 24 & 15u;
}
// The mask in words of 32 keys (0 past the last), and whether any of 32 queries may attend any of 64 keys.  A wavefront takes 32
// queries and two such tiles of keys.
__global__ __launch_bounds__(64) void k_pack_mask(Attention a) {
  const int lane = threadIdx.x, h = lane >> 5;
  const uint32_t words = (uint32_t)words_of(a.keys), tiles = words / 2, per = (tiles + 1) / 2;
  const uint32_t qt = blockIdx.x / per, t = (blockIdx.x - qt * per) * 2 + h, query = qt * 32 + (lane & 31);
  uint64_t w = 0;
  if (query < a.queries && t < tiles) {
    const int64_t k0 = (int64_t)t * 64;
    const int n = a.keys - k0 < 64 ? (int)(a.keys - k0) : 64;
    const char *const p = (const char *)a.mask + (int64_t)query * a.ldmask + k0;
    u32x4 v[4];
    if (n == 64) {
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = any16(p + 16 * c);
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if (n >= 16 * c + 16) v[c] = any16(p + 16 * c);
        else v[c] = some_values<uint8_t>(p + 16 * c, n - 16 * c);
      }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = v[c][i];
        w |= (uint64_t)nonzero4(x) << (16 * c + 4 * i);
      }
    *(uint64_t *)(a.words + (int64_t)query * words + t * 2) = w;
  }
  const uint64_t any = __ballot(w != 0);
  if ((lane & 31) == 0 && t < tiles) a.flags[(int64_t)qt * tiles + t] = (uint32_t)(any >> (32 * h)) != 0;
}

struct PackGrid {
  uint32_t blocks[4];
};
// Pieces of the copies, one a thread and turn.
template <class T>
__global__ __launch_bounds__(256) void k_pack_heads(PackHeadsAll all, PackGrid grid) {
  constexpr int E = 16 / (int)sizeof(T);
  uint32_t block = blockIdx.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (block >= grid.blocks[i]) {
      block -= grid.blocks[i];
      continue;
    }
    const PackHeads &p = all.t[i];
    const uint32_t per = p.line / E, row_pieces = per * p.heads;
    const uint64_t pieces = (uint64_t)p.batch * p.length * row_pieces;
    const char *const end = end_of(p.from, p.batch, p.length, p.heads, p.d, sizeof(T));
    for (uint64_t at = (uint64_t)block * 256 + threadIdx.x; at < pieces; at += (uint64_t)grid.blocks[i] * 256) {
      const uint64_t row = at >> 32 ? at / row_pieces : (uint32_t)at / row_pieces;
      const uint32_t rest = (uint32_t)(at - row * row_pieces), head = rest / per, c = rest - head * per;
      const uint32_t b = row >> 32 ? (uint32_t)(row / p.length) : (uint32_t)row / (uint32_t)p.length;
      const int64_t n = (int64_t)row - (int64_t)b * p.length;
      if (p.lengths && n >= p.lengths[b]) continue;
      const char *const from = (const char *)p.from.p + (b * p.from.batch + n * p.from.row + head * p.from.head) * (int64_t)sizeof(T);
      *(u32x4 *)((char *)p.to + at * 16) = row_piece<T>(from, (int)c, p.d, end);
    }
    return;
  }
}

template <class T, int DP, int WQ, int WK>
hipError_t launch_shape(const Attention &a, hipStream_t s) {
  const int64_t rows = (int64_t)(a.heads / a.kv_heads) * a.queries;
  const int64_t blocks = (rows + 32 * WQ - 1) / (32 * WQ) * a.batch * a.kv_heads * a.splits;
  const bool direct = direct_ok<T>(a.k, a) && direct_ok<T>(a.v, a);
  if (a.mask && direct) k_attention<T, DP, WQ, WK, true, true><<<dim3((unsigned)blocks), WQ * WK * 64, 0, s>>>(a);
  else if (a.mask) k_attention<T, DP, WQ, WK, true, false><<<dim3((unsigned)blocks), WQ * WK * 64, 0, s>>>(a);
  else if (direct) k_attention<T, DP, WQ, WK, false, true><<<dim3((unsigned)blocks), WQ * WK * 64, 0, s>>>(a);
  else k_attention<T, DP, WQ, WK, false, false><<<dim3((unsigned)blocks), WQ * WK * 64, 0, s>>>(a);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || a.splits == 1) return err;
  const int64_t threads = rows * a.batch * a.kv_heads * (DP / 4);
  k_join_attention<T><<<dim3((unsigned)((threads + 255) / 256)), 256, 0, s>>>(a, DP);
  return hipGetLastError();
}
// Over 128 fp32 values a row: tiles of four wavefronts' keys do not fit in LDS, so few rows run as many do.
template <class T, int DP>
hipError_t launch_rows(const Attention &a, bool few, hipStream_t s) {
  if constexpr (DP * sizeof(T) <= 512) {
    if (few) return launch_shape<T, DP, 1, 4>(a, s);
  }
  return launch_shape<T, DP, 4, 1>(a, s);
}
template <class T>
hipError_t launch_type(const Attention &a, bool few, hipStream_t s) {
  switch (d_of(a.d)) {
    case 32: return launch_rows<T, 32>(a, few, s);
    case 64: return launch_rows<T, 64>(a, few, s);
    case 128: return launch_rows<T, 128>(a, few, s);
    case 192: return launch_rows<T, 192>(a, few, s);
    default: return launch_rows<T, 256>(a, few, s);
  }
}

}  // namespace

AttentionPlan plan_attention(int type, int64_t batch, int64_t queries, int64_t keys, int heads, int kv_heads, int d, bool masked) {
  AttentionPlan p{};
  const int dp = d_of(d);
  const int64_t rows = (int64_t)(heads / kv_heads) * queries, pairs = batch * kv_heads;
  const int64_t wide = (rows + 127) / 128 * pairs;
  p.few = wide < 256 && !(type == AECCT_F32 && dp > 128);
  const int64_t blocks = p.few ? (rows + 31) / 32 * pairs : wide;
  // At least 512 keys a split, about four blocks a compute unit.
  int64_t splits = blocks > 0 ? 1024 / blocks : 1;
  if (splits > keys / 512) splits = keys / 512;
  if (splits > 64) splits = 64;
  p.splits = splits > 1 && blocks < 512 ? (int)splits : 1;
  if (masked) {
    p.words = (size_t)(queries * words_of(keys)) * 4;
    p.flags = (size_t)((queries + 31) / 32 * (words_of(keys) / 2));
  }
  if (p.splits > 1) {
    p.part_o = (size_t)(p.splits * pairs * rows * dp) * 4;
    p.part_ml = (size_t)(p.splits * pairs * rows) * 8;
  }
  return p;
}

hipError_t launch_mask(const Attention &a, hipStream_t s) {
  const int64_t tiles = words_of(a.keys) / 2;
  k_pack_mask<<<dim3((unsigned)((a.queries + 31) / 32 * ((tiles + 1) / 2))), 64, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pack_heads(int type, const PackHeadsAll &p, hipStream_t s) {
  PackGrid grid{};
  uint32_t all = 0;
  for (int i = 0; i < 4; ++i) {
    const int64_t pieces = p.t[i].length ? p.t[i].batch * p.t[i].length * p.t[i].heads * (p.t[i].line / (16 / (type == AECCT_F32 ? 4 : 2))) : 0;
    grid.blocks[i] = (uint32_t)(pieces < (int64_t)1 << 24 ? (pieces + 255) / 256 : 1 << 16);
    all += grid.blocks[i];
  }
  if (all == 0) return hipSuccess;
  switch (type) {
    case AECCT_F32: k_pack_heads<float><<<dim3(all), 256, 0, s>>>(p, grid); break;
    case AECCT_BF16: k_pack_heads<bf16_t><<<dim3(all), 256, 0, s>>>(p, grid); break;
    case AECCT_F16: k_pack_heads<f16_t><<<dim3(all), 256, 0, s>>>(p, grid); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_attention(int type, const Attention &a, const AttentionPlan &p, hipStream_t s) {
  if (a.mask) {
    const hipError_t err = launch_mask(a, s);
    if (err != hipSuccess) return err;
  }
  switch (type) {
    case AECCT_F32: return launch_type<float>(a, p.few, s);
    case AECCT_BF16: return launch_type<bf16_t>(a, p.few, s);
    case AECCT_F16: return launch_type<f16_t>(a, p.few, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace aecct
