// Cross attention in one pass over the keys: o = softmax(scale q k^T) v with the running maximum and sum of each row (softmax in
// base 2, on scores times log2(e)).
//
// A wavefront takes 32 rows (queries of the heads that share a key head).  It computes the scores turned, keys by rows, so that a
// lane holds 16 keys of one row: the maximum and sum are taken in registers with one exchange between the halves, and the
// weights are, as they lie, the second factor of the product with the values.
#include "attention_tile.h"

namespace aecct {
namespace {

// In fp16 the weights are taken times 2^10, so that those of long rows stay in its normal range (at most 2^10, the sum in
// fp32 takes the factor out again).
template <class T>
__device__ constexpr float weight_shift() { return __is_same(T, f16_t) ? 10.0f : 0.0f; }

template <class T, int DP, int WQ, int WK, bool MASK>
__global__ __launch_bounds__(WQ *WK * 64) void k_attention(Attention a) {
  constexpr int RB = DP * (int)sizeof(T), FD = DP / 32, NT = WQ * WK * 64;
  constexpr int SUB = WK == 1 && RB <= 256 ? 2 : 1, KT = 32 * SUB * WK;   // keys of a tile
  constexpr int PER = KT * RB / 16 / NT, CH = RB / 16;                    // pieces a thread and a row
  static_assert(KT * RB / 16 % NT == 0, "whole pieces");
  __shared__ __attribute__((aligned(16))) char lds[2 * KT * RB];
  char *const lk = lds, *const lv = lds + KT * RB;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5;
  const int wq = WK == 1 ? wave : 0, wk = WK == 1 ? 0 : wave;
  const int group = a.heads / a.kv_heads;
  const int64_t rows = group * a.queries, row_blocks = (rows + 32 * WQ - 1) / (32 * WQ);
  const int64_t at = near_block(blockIdx.x, gridDim.x);
  const int64_t row_block = at % row_blocks, rest = at / row_blocks, pairs = a.batch * a.kv_heads;
  const int64_t pair = rest / a.splits;
  const int split = (int)(rest % a.splits);
  const int64_t b = pair / a.kv_heads;
  const int kh = (int)(pair % a.kv_heads);
  int64_t length = a.keys;
  if (a.lengths) {
    const int64_t l = a.lengths[b];
    length = l < 0 ? 0 : l < length ? l : length;
  }
  // This block's tiles of keys.
  const int64_t tiles = (length + KT - 1) / KT, t0 = tiles * split / a.splits, t1 = tiles * (split + 1) / a.splits;
  // This lane's row.
  const int64_t r = row_block * (32 * WQ) + wq * 32 + (lane & 31), rc = r < rows ? r : rows - 1;
  const int64_t head = kh * group + rc / a.queries, query = rc % a.queries;
  const bool idle = row_block * (32 * WQ) + wq * 32 >= rows;   // the whole wavefront's rows are past the last
  u32x4 q[RB / 32];
  {
    const char *const p = (const char *)a.q.p + (b * a.q.batch + query * a.q.row + head * a.q.head) * (int64_t)sizeof(T);
    const char *const end = end_of(a.q, a.batch, a.queries, a.heads, a.d, sizeof(T));
#pragma unroll
    for (int c = 0; c < RB / 32; ++c) q[c] = row_piece<T>(p, 2 * c + h, a.d, end);
  }
  const char *const pk = (const char *)a.k.p + (b * a.k.batch + kh * a.k.head) * (int64_t)sizeof(T);
  const char *const pv = (const char *)a.v.p + (b * a.v.batch + kh * a.v.head) * (int64_t)sizeof(T);
  const char *const ek = end_of(a.k, a.batch, a.keys, a.kv_heads, a.d, sizeof(T));
  const char *const ev = end_of(a.v, a.batch, a.keys, a.kv_heads, a.d, sizeof(T));
  const int64_t words = words_of(a.keys), flag_tiles = words / 2;
  const uint8_t *const flags = MASK ? a.flags + (row_block * WQ + wq) * flag_tiles : nullptr;
  // Tiles of keys that none of the block's rows may attend are passed over: 64 tiles are looked up at once.
  uint64_t want = 0;
  int64_t want0 = t0 - 64;
  auto from = [&](int64_t t) {   // the first tile to be done from t on
    if constexpr (!MASK) return t;
    while (t < t1) {
      if (t - want0 >= 64) {
        want0 = t;
        want = __ballot(t + lane < t1 && any_flag(a.flags, row_block * WQ, WQ, (rows + 31) / 32, (t + lane) * KT, KT, flag_tiles));
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
  float m = -INFINITY, sum = 0;
  const float to2 = a.scale * kLog2e;

  u32x4 ck[PER], cv[PER];
  auto load = [&](int64_t t) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int slot = threadIdx.x + i * NT, row = slot / CH, chunk = slot % CH;
      const int64_t key = t * KT + row;
      ck[i] = cv[i] = u32x4{0, 0, 0, 0};
      if (key < length) {   // keys past the length are never read: their weights are 0, and 0 times what lies there may be NaN
        ck[i] = row_piece<T>(pk + key * a.k.row * (int64_t)sizeof(T), chunk, a.d, ek);
        cv[i] = row_piece<T>(pv + key * a.v.row * (int64_t)sizeof(T), chunk, a.d, ev);
      }
    }
  };
  int64_t t = from(t0);
  if (t < t1) load(t);
  while (t < t1) {
    const int64_t next = from(t + 1);
    __syncthreads();   // the tile before has been read
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int slot = threadIdx.x + i * NT, row = slot / CH, chunk = slot % CH;
      const int to = row * RB + ((chunk << 4) ^ exchange<RB>(row));
      *(u32x4 *)(lk + to) = ck[i];
      *(u32x4 *)(lv + to) = cv[i];
    }
    __syncthreads();
    if (next < t1) load(next);
    const int64_t key0 = t * KT + wk * 32 * SUB;
    int flag = 2;
    if constexpr (MASK) flag = !idle && key0 < length ? flags[key0 / 64] : 0;
    if (!idle && key0 < length && flag != 0) {
      float s[SUB][16];
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const f32x16 x = times_rows<T, RB>(lk, (wk * SUB + u) * 32, q);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[u][i] = x[i];
        const int64_t k0 = key0 + u * 32;
        if (k0 + 32 > length) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (k0 + row_of(i, h) >= length) s[u][i] = -INFINITY;
        }
        if constexpr (MASK) {
          if (flag == 1) {
            const uint32_t w = a.words[query * words + k0 / 32] >> (4 * h);
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (!(w >> row_of(i, 0) & 1)) s[u][i] = -INFINITY;
          }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
      }
      top = fmaxf(m, max_halves(top) * to2);
      // A row that has met no key it may attend keeps the maximum -inf; its weights are 2^-inf = 0.
      const float base = top == -INFINITY ? 0.0f : top;
      if (__any(top != m)) {
        const float down = __builtin_amdgcn_exp2f(m - base);
        sum *= down;
#pragma unroll
        for (int f = 0; f < FD; ++f)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[f][i] *= down;
      }
      m = top;
      const float lift = base - weight_shift<T>();
      float part = 0;
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[u][i] = __builtin_amdgcn_exp2f(fmaf(s[u][i], to2, -lift));
          part += s[u][i];
        }
        add_columns<T, RB, FD>(acc, lv, (wk * SUB + u) * 32, s[u]);
      }
      sum += part;
    }
    t = next;
  }
  sum = sum_halves(sum);

  if constexpr (WK > 1) {
    // The wavefronts' shares of the keys are joined through LDS.
    constexpr int LD = DP;
    static_assert(2 * KT * RB >= WK * 32 * LD * 4, "the sums fit where the tiles were");
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
    const int64_t at_row = ((int64_t)split * pairs + pair) * rows + r;
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
    a.lse[(b * a.heads + head) * a.queries + query] = sum == 0.0f ? -INFINITY : (m + (__log2f(sum) - weight_shift<T>())) * kLn2;
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
  const int group = a.heads / a.kv_heads, per = dp / 4;
  const int64_t rows = group * a.queries, pairs = a.batch * a.kv_heads, all = pairs * rows;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / per;
  const int c = (int)(at % per) * 4;
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
  const int64_t pair = row / rows, r = row % rows, b = pair / a.kv_heads;
  const int64_t head = pair % a.kv_heads * group + r / a.queries, query = r % a.queries;
  const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
  if (a.lse && c == 0)
    a.lse[(b * a.heads + head) * a.queries + query] = sum == 0.0f ? -INFINITY : (m + (__log2f(sum) - weight_shift<T>())) * kLn2;
  if (c < a.d)
    store_values4<T>((T *)a.o.p + b * a.o.batch + query * a.o.row + head * a.o.head + c, a.d - c, v[0] * over, v[1] * over,
                     v[2] * over, v[3] * over);
}

// Nonzero bytes of w as its four low bits.
__device__ __forceinline__ uint32_t nonzero4(uint32_t w) {
  const uint32_t t = ((((w & 0x7f7f7f7fu) + 0x7f7f7f7fu) | w) >> 7) & 0x01010101u;
  return (t * 0x01020408u) >> 24 & 15u;
}
// The mask in words of 32 keys, and what each 32 rows may attend of each 64 keys.  A wavefront takes 32 rows and two such tiles of
// keys; bits past the last key are 0 in the words, and do not count in the flags.
__global__ __launch_bounds__(64) void k_pack_mask(Attention a) {
  const int lane = threadIdx.x, h = lane >> 5;
  const int64_t rows = (int64_t)(a.heads / a.kv_heads) * a.queries, words = words_of(a.keys), tiles = words / 2;
  const int64_t per = (tiles + 1) / 2, rt = blockIdx.x / per, t = blockIdx.x % per * 2 + h;
  const int64_t r = rt * 32 + (lane & 31);
  const bool live = r < rows && t < tiles;
  uint64_t w = 0, full = ~(uint64_t)0;
  if (live) {
    const int64_t k0 = t * 64;
    const int n = a.keys - k0 < 64 ? (int)(a.keys - k0) : 64;
    if (n < 64) full = ((uint64_t)1 << n) - 1;
    const uint8_t *const p = a.mask + (r % a.queries) * a.ldmask + k0;
    if (n == 64) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const u32x4 v = any16((const char *)p + 16 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = v[i];
          w |= (uint64_t)nonzero4(x) << (16 * c + 4 * i);
        }
      }
    } else {
      for (int i = 0; i < n; ++i) w |= (uint64_t)(p[i] != 0) << i;
    }
    if (r < a.queries) *(uint64_t *)(a.words + r * words + t * 2) = w;
  }
  const uint64_t any = __ballot(live && w != 0), gap = __ballot(live && w != full);
  if ((lane & 31) == 0 && t < tiles) {
    const uint32_t x = (uint32_t)(any >> (32 * h)), y = (uint32_t)(gap >> (32 * h));
    a.flags[rt * tiles + t] = x == 0 ? 0 : y == 0 ? 2 : 1;
  }
}

template <class T, int DP, int WQ, int WK>
hipError_t launch_shape(const Attention &a, hipStream_t s) {
  const int64_t rows = (int64_t)(a.heads / a.kv_heads) * a.queries;
  const int64_t blocks = (rows + 32 * WQ - 1) / (32 * WQ) * a.batch * a.kv_heads * a.splits;
  if (a.mask) k_attention<T, DP, WQ, WK, true><<<dim3((unsigned)blocks), WQ * WK * 64, 0, s>>>(a);
  else k_attention<T, DP, WQ, WK, false><<<dim3((unsigned)blocks), WQ * WK * 64, 0, s>>>(a);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || a.splits == 1) return err;
  const int64_t threads = rows * a.batch * a.kv_heads * (DP / 4);
  k_join_attention<T><<<dim3((unsigned)((threads + 255) / 256)), 256, 0, s>>>(a, DP);
  return hipGetLastError();
}
// 256 fp32 values a row: tiles of four wavefronts' keys do not fit in LDS, so few rows run as many do.
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
    default: return launch_rows<T, 256>(a, few, s);
  }
}

}  // namespace

AttentionPlan plan_attention(int type, int64_t batch, int64_t queries, int64_t keys, int heads, int kv_heads, int d, bool masked) {
  AttentionPlan p{};
  const int dp = d_of(d);
  const int64_t rows = (int64_t)(heads / kv_heads) * queries, pairs = batch * kv_heads;
  const int64_t wide = (rows + 127) / 128 * pairs;
  p.few = wide < 256 && !(type == AECCT_F32 && dp == 256);
  const int64_t blocks = p.few ? (rows + 31) / 32 * pairs : wide;
  // At least 512 keys a split, about four blocks a compute unit.
  int64_t splits = blocks > 0 ? 1024 / blocks : 1;
  if (splits > keys / 512) splits = keys / 512;
  if (splits > 64) splits = 64;
  p.splits = splits > 1 && blocks < 512 ? (int)splits : 1;
  if (masked) {
    p.words = (size_t)(queries * words_of(keys)) * 4;
    p.flags = (size_t)((rows + 31) / 32 * (words_of(keys) / 2));
  }
  if (p.splits > 1) {
    p.part_o = (size_t)(p.splits * pairs * rows * dp) * 4;
    p.part_ml = (size_t)(p.splits * pairs * rows) * 8;
  }
  return p;
}

hipError_t launch_mask(const Attention &a, hipStream_t s) {
  const int64_t rows = (int64_t)(a.heads / a.kv_heads) * a.queries, tiles = words_of(a.keys) / 2;
  k_pack_mask<<<dim3((unsigned)((rows + 31) / 32 * ((tiles + 1) / 2))), 64, 0, s>>>(a);
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
