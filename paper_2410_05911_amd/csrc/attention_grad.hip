// The gradient of cross attention from its output and the logarithms of its rows' sums:
//   p = exp(scale q k^T - lse),  D = sum of dout o over d,  ds = p (dout v^T - D),
//   dq = scale ds k,  dk = scale ds^T q,  dv = p^T dout.
// dk and dv sum over rows and dq over keys, so they are two kernels, each of which computes p and ds for itself: seven products in
// place of five, and no sums in memory whose order could change.  Every sum over the heads that share a key head is one over rows.
//
// As in the forward pass the scores are computed so that a lane's registers are the second factor of the products that follow:
// keys by rows for dq, rows by keys for dk and dv.
//
// With 16-bit types p and ds are rounded to the type, as the matrix instructions take them: dq, dk and dv are what the formula gives with
// those rounded weights, rounded once more, 2.4e-3 (bf16) and 3.0e-4 (fp16) of their norms from 64 bits where an output's rounding alone
// is 1.66e-3 and 2.1e-4.  What a second product with the rest would gain is not worth 3 products more beside 7.
//
// Measured: 2 x 2049 queries on 1531 keys, 16 heads of 64 on 4 key heads, a band of a quarter, bf16: dq 27 us, dk and dv 46, their join
// 10, all 85; 128 x 256 on 128 keys, 8 heads of 16, three keys a query, fp32: 34 and 52, all 87.  Both are bound by the instructions
// and latencies of short loops (dq has 9 tiles of keys a block, dk and dv 8 to 16 of rows), not by memory.
#include "attention_tile.h"

namespace aecct {
namespace {

// In fp16 p is taken times 2^14 (it is at most 1), and ds times a power of two that each lane keeps below 2^15 for its own row or
// key and takes out of the sum so far when it shrinks: small gradients stay in fp16's normal range, large ones do not overflow.
template <class T>
__device__ constexpr float p_shift() { return __is_same(T, f16_t) ? 14.0f : 0.0f; }
template <class T, int FD>
struct Scaled {
  float by = 0x1p100f;
  __device__ __forceinline__ void apply(float (&ds)[16], f32x16 (&acc)[FD]) {
    if constexpr (__is_same(T, f16_t)) {
      float most = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(ds[i]));
      most = max_halves(most);
      if (__any(most * by >= 0x1p15f)) {
        const float now = most * by >= 0x1p15f ? fmaxf(__builtin_amdgcn_ldexpf(1.0f, 15 - __builtin_amdgcn_frexp_expf(most)), 0x1p-100f) : by;
        const float down = now / by;
#pragma unroll
        for (int f = 0; f < FD; ++f)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[f][i] *= down;
        by = now;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) ds[i] *= by;
    }
  }
  __device__ __forceinline__ float out() const { return __is_same(T, f16_t) ? 1.0f / by : 1.0f; }
};

// What a row of p and ds is taken from: lse, in 16-bit types times log2(e) (a row that attends nothing: infinity, so that its weights
// are 0) and D.
template <class T>
__device__ __forceinline__ void row_terms(float lse, float sum, float &l, float &dd) {
  l = lse == -INFINITY ? INFINITY : sizeof(T) == 4 ? lse : lse * kLog2e;
  dd = lse == -INFINITY ? 0.0f : sum;
}
// p of a score s, times 2^shift.  In fp32 the score's distance from lse is taken before it is multiplied by log2(e): it is small where p is
// not, while lse log2(e) alone, rounded, moves a row's p by up to 2^-24 of |lse log2(e)| (2 queries on 24 keys of 64 values: dv off by
// 2.6e-7 of its norm, so 2.1e-7; what is left is the scores' own sums).
template <class T>
__device__ __forceinline__ float weight(float s, float scale, float l, float shift) {
  if constexpr (sizeof(T) == 4) return __builtin_amdgcn_exp2f(fmaf(s, scale, -l) * kLog2e);
  else return __builtin_amdgcn_exp2f(fmaf(s, scale * kLog2e, shift - l));
}
// The sum of the products of two pieces of 16 bytes.
template <class T>
__device__ __forceinline__ float dot(u32x4 x, u32x4 y, float sum) {
  Raw<T, 16 / sizeof(T)> a, b;
  float f[16 / sizeof(T)], g[16 / sizeof(T)];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a.w[i] = x[i];
    b.w[i] = y[i];
  }
  unpack<T, 16 / sizeof(T)>(a, f);
  unpack<T, 16 / sizeof(T)>(b, g);
#pragma unroll
  for (int i = 0; i < (int)(16 / sizeof(T)); ++i) sum = fmaf(f[i], g[i], sum);
  return sum;
}
// The rows' terms where dq, which takes them along, is not asked for: 16 lanes a row.
template <class T>
__global__ __launch_bounds__(256) void k_attention_rows(AttentionGrad g) {
  const Attention &a = g.a;
  const uint32_t group = a.heads / a.kv_heads, queries = (uint32_t)a.queries, rows = group * queries;
  const uint32_t row = blockIdx.x * 16 + (threadIdx.x >> 4), pair = row / rows, r = row - pair * rows, b = pair / (uint32_t)a.kv_heads;
  if (b >= a.batch) return;
  const uint32_t head = (pair - b * a.kv_heads) * group + r / queries, query = r % queries;
  const char *const o = (const char *)a.o.p + (b * a.o.batch + query * a.o.row + head * a.o.head) * (int64_t)sizeof(T);
  const char *const d = (const char *)g.dout.p + (b * g.dout.batch + query * g.dout.row + head * g.dout.head) * (int64_t)sizeof(T);
  const char *const eo = end_of(a.o, a.batch, a.queries, a.heads, a.d, sizeof(T));
  const char *const ed = end_of(g.dout, a.batch, a.queries, a.heads, a.d, sizeof(T));
  float sum = 0;
  for (int c = threadIdx.x & 15; c * (int)(16 / sizeof(T)) < a.d; c += 16)
    sum = dot<T>(row_piece<T>(o, c, a.d, eo), row_piece<T>(d, c, a.d, ed), sum);
#pragma unroll
  for (int i = 1; i < 16; i *= 2) sum += __shfl_xor(sum, i);
  if ((threadIdx.x & 15) == 0) {
    float l, dd;
    row_terms<T>(a.lse[(int64_t)(b * a.heads + head) * queries + query], sum, l, dd);
    g.rows[(int64_t)row * 2] = l;
    g.rows[(int64_t)row * 2 + 1] = dd;
  }
}

// dq: a wavefront takes 32 rows, tiles of keys pass through LDS.  It leaves the rows' terms for dk and dv.
template <class T, int DP, bool MASK, bool DIRECT>
__global__ __launch_bounds__(256, DP * sizeof(T) <= 128 ? 3 : DP * sizeof(T) <= 256 ? 2 : 1) void k_attention_dq(AttentionGrad g) {
  constexpr int RB = DP * (int)sizeof(T), FD = DP / 32, NT = 256, SUB = RB <= 256 ? 2 : 1, KT = 32 * SUB;
  constexpr int STAGES = DIRECT && 4 * KT * RB <= 131072 ? 2 : 1;
  const Attention &a = g.a;
  __shared__ __attribute__((aligned(16))) char lds[STAGES * 2 * KT * RB];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5;
  const uint32_t group = a.heads / a.kv_heads, queries = (uint32_t)a.queries, rows = group * queries, row_blocks = (rows + 127) / 128;
  const uint32_t at = near_block(blockIdx.x, gridDim.x), rest = at / row_blocks, row_block = at - rest * row_blocks;
  const uint32_t pair = g.splits_q > 1 ? rest / (uint32_t)g.splits_q : rest, split = g.splits_q > 1 ? rest - pair * g.splits_q : 0;
  const uint32_t b = pair / (uint32_t)a.kv_heads, kh = pair - b * a.kv_heads;
  const int length = length_of(a, b), tiles = (length + KT - 1) / KT;
  int t0 = 0, t1 = tiles;
  if (g.splits_q > 1) {
    t0 = (int)((uint32_t)tiles * split / (uint32_t)g.splits_q);
    t1 = (int)((uint32_t)tiles * (split + 1) / (uint32_t)g.splits_q);
  }
  const uint32_t r = row_block * 128 + wave * 32 + (lane & 31), rc = min(r, rows - 1);
  const uint32_t head = kh * group + rc / queries, query = rc % queries;
  const bool idle = row_block * 128 + wave * 32 >= rows;
  Keys<T, RB, KT, NT, DIRECT> keys(a.k, a, b, kh, length), values(a.v, a, b, kh, length);
  const int words = (int)words_of(a.keys);
  const uint32_t *const mask = MASK ? a.words + (int64_t)query * words : nullptr;
  uint64_t want = 0;
  int want0 = t0 - 64;
  auto from = [&](int t) {
    if constexpr (!MASK) return t;
    while (t < t1) {
      if (t - want0 >= 64) {
        want0 = t;
        want = __ballot(any_flag<128, KT>(a, row_block * 128, min(t + lane, t1 - 1) * KT) && t + lane < t1);
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
  Scaled<T, FD> scaled;
  uint32_t w[SUB] = {}, w_next[SUB] = {};
  auto look = [&](int t, uint32_t (&w)[SUB]) {
    if constexpr (MASK) {
#pragma unroll
      for (int u = 0; u < SUB; ++u) w[u] = t * SUB + u < words ? mask[t * SUB + u] : 0;
    }
  };
  int t = from(t0), buf = 0;
  if (t < t1) {
    if constexpr (!DIRECT || STAGES == 2) {
      keys.load(lds, t);
      values.load(lds + KT * RB, t);
    }
    look(t, w_next);
  }
  // (behind the first tile, which is on its way by now)
  u32x4 q[RB / 32], dout[RB / 32];
  float dd = 0, l;
  {
    const char *const p = (const char *)a.q.p + (b * a.q.batch + query * a.q.row + head * a.q.head) * (int64_t)sizeof(T);
    const char *const pd = (const char *)g.dout.p + (b * g.dout.batch + query * g.dout.row + head * g.dout.head) * (int64_t)sizeof(T);
    const char *const po = (const char *)a.o.p + (b * a.o.batch + query * a.o.row + head * a.o.head) * (int64_t)sizeof(T);
    const char *const end = end_of(a.q, a.batch, a.queries, a.heads, a.d, sizeof(T));
    const char *const endd = end_of(g.dout, a.batch, a.queries, a.heads, a.d, sizeof(T));
    const char *const endo = end_of(a.o, a.batch, a.queries, a.heads, a.d, sizeof(T));
#pragma unroll
    for (int c = 0; c < RB / 32; ++c) {
      q[c] = row_piece<T>(p, 2 * c + h, a.d, end);
      dout[c] = row_piece<T>(pd, 2 * c + h, a.d, endd);
      dd = dot<T>(row_piece<T>(po, 2 * c + h, a.d, endo), dout[c], dd);
    }
    row_terms<T>(a.lse[(int64_t)(b * a.heads + head) * queries + query], sum_halves(dd), l, dd);
    if (h == 0 && r < rows && split == 0) {
      g.rows[((int64_t)pair * rows + r) * 2] = l;
      g.rows[((int64_t)pair * rows + r) * 2 + 1] = dd;
    }
  }
  while (t < t1) {
    const int next = from(t + 1);
    char *const lk = lds + buf * 2 * KT * RB, *const lv = lk + KT * RB;
#pragma unroll
    for (int u = 0; u < SUB; ++u) w[u] = w_next[u];
    if constexpr (DIRECT && STAGES == 2) {
      wait_loads();
      barrier();
      if (next < t1) {
        keys.load(lds + (buf ^ 1) * 2 * KT * RB, next);
        values.load(lds + (buf ^ 1) * 2 * KT * RB + KT * RB, next);
      }
      buf ^= 1;
    } else if constexpr (DIRECT) {
      barrier();
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
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      const int k0 = t * KT + u * 32;
      uint32_t in = MASK ? w[u] : ~0u;
      if (k0 + 32 > length) in = length > k0 ? in & ((1u << (length - k0)) - 1) : 0;
      if (idle || !__any(in != 0)) continue;
      if constexpr (MASK && pairwise<T, RB>()) {
        if (!__any(__popc(in) > kFewPairs)) {
          while (__any(in != 0)) {
            const int row = u * 32 + (in ? __builtin_ctz(in) : 0);
            const float dp = sum_halves(HalfRow<RB>(lv, row, a.d).dot(dout, a.d));
            const HalfRow<RB> key(lk, row, a.d);
            const float s = sum_halves(key.dot(q, a.d));
            const float ds = weight<T>(s, a.scale, l, 0.0f) * (dp - dd);
            if (in) key.add_to(acc, ds, a.d);
            in &= in - 1;
          }
          continue;
        }
      }
      const f32x16 s = times_rows<T, RB, RB == 1024>(lk, u * 32, q, a.d), dp = times_rows<T, RB, RB == 1024>(lv, u * 32, dout, a.d);
      float ds[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) ds[i] = weight<T>(s[i], a.scale, l, 0.0f) * (dp[i] - dd);
      if (!__all(in == ~0u)) {
        in >>= 4 * h;
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] = in >> row_of(i, 0) & 1 ? ds[i] : 0.0f;
      }
      scaled.apply(ds, acc);
      if constexpr (sizeof(T) == 4 && RB <= 512) {
        // In fp32 a tile's sums begin anew: one chain over all keys adds up to twice the error of a product in blocks (3000 keys 1.2e-6).
        f32x16 fresh[FD];
#pragma unroll
        for (int f = 0; f < FD; ++f)
#pragma unroll
          for (int i = 0; i < 16; ++i) fresh[f][i] = 0;
        add_columns<T, RB, RB == 1024>(fresh, lk, u * 32, ds, a.d);
#pragma unroll
        for (int f = 0; f < FD; ++f)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[f][i] += fresh[f][i];
      } else {
        add_columns<T, RB, RB == 1024>(acc, lk, u * 32, ds, a.d);
      }
    }
    t = next;
  }
  if (r >= rows) return;
  const float out = a.scale * scaled.out();
  if (g.splits_q > 1) {
    float *const o = g.part_q + ((int64_t)(split * (uint32_t)a.batch * a.kv_heads + pair) * rows + r) * DP;
#pragma unroll
    for (int f = 0; f < FD; ++f)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(f32x4 *)(o + 32 * f + row_of(i, h)) = f32x4{acc[f][i] * out, acc[f][i + 1] * out, acc[f][i + 2] * out, acc[f][i + 3] * out};
    return;
  }
  T *const o = (T *)g.dq.p + b * g.dq.batch + query * g.dq.row + head * g.dq.head;
#pragma unroll
  for (int f = 0; f < FD; ++f)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int c = 32 * f + row_of(i, h);
      if (c < a.d) store_values4<T>(o + c, a.d - c, acc[f][i] * out, acc[f][i + 1] * out, acc[f][i + 2] * out, acc[f][i + 3] * out);
    }
}

// Tiles of 32 rows (queries of the heads of a key head) of one pair on their way to LDS, as Keys.
template <class T, int RB, bool DIRECT>
struct RowsOf {
  static constexpr int NT = 256, CH = RB / 16, PER = (32 * CH + NT - 1) / NT, E = 16 / (int)sizeof(T);
  static constexpr uint32_t OUT = 0x80000000u;
  const char *p, *end;
  int64_t row_stride, head_stride;
  uint32_t rows, queries;
  int d;
  u32x4 v[DIRECT ? 1 : PER];
  __device__ __forceinline__ RowsOf(const Heads &t, const Attention &a, uint32_t b, uint32_t kh)
      : p((const char *)t.p + (b * t.batch + kh * (a.heads / a.kv_heads) * t.head) * (int64_t)sizeof(T)),
        end(end_of(t, a.batch, a.queries, a.heads, a.d, sizeof(T))), row_stride(t.row * (int64_t)sizeof(T)),
        head_stride(t.head * (int64_t)sizeof(T)), rows((uint32_t)(a.heads / a.kv_heads) * (uint32_t)a.queries),
        queries((uint32_t)a.queries), d(a.d) {}
  __device__ __forceinline__ void load(char *lds, int t) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const BufferOf buffer(p, OUT);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int slot = threadIdx.x + i * NT, row = slot / CH, chunk = (((slot % CH) << 4) ^ exchange<RB>(row)) >> 4;
      const uint32_t r = t * 32 + row, head = r / queries, query = r - head * queries;
      const bool there = r < rows && row < 32;
      if constexpr (DIRECT) {
        // The last wavefronts of a tile of less than 256 pieces have none.
        if (32 * CH >= NT || wave * 64 < 32 * CH) {
          const uint32_t at = query * (uint32_t)row_stride + head * (uint32_t)head_stride + chunk * 16;
          buffer.to_lds(lds + (i * NT + wave * 64) * 16, there && chunk * E < d ? at : OUT);
        }
      } else {
        v[i] = u32x4{0, 0, 0, 0};
        if (there) v[i] = row_piece<T>(p + query * row_stride + head * head_stride, chunk, d, end);
      }
    }
  }
  __device__ __forceinline__ void store(char *lds) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int slot = threadIdx.x + i * NT;
      if (slot < 32 * CH) *(u32x4 *)(lds + slot * 16) = v[i];
    }
  }
};
// Whether RowsOf takes a tensor past the registers: whole 16-byte pieces, and a sequence's offsets within 2^31.
template <class T>
bool direct_rows(const Heads &t, const Attention &a) {
  constexpr int64_t E = 16 / sizeof(T);
  return (uintptr_t)t.p % 16 == 0 && (t.packed || a.d % E == 0) && t.batch % E == 0 && t.row % E == 0 && t.head % E == 0 &&
         t.row * (a.queries - 1) + t.head * a.heads + a.d < ((int64_t)1 << 31) / (int64_t)sizeof(T);
}

// dk and dv (DK, DV: which of them): a wavefront takes 32 keys, tiles of 32 rows pass through LDS.
template <class T, int DP, bool MASK, bool DK, bool DV, bool DIRECT>
__global__ __launch_bounds__(256, DP * sizeof(T) <= (DIRECT ? 256 : 128) ? 2 : 1) void k_attention_dkv(AttentionGrad g) {
  constexpr int RB = DP * (int)sizeof(T), FD = DP / 32, RT = 32, STAGES = DIRECT ? 2 : 1;
  const Attention &a = g.a;
  __shared__ __attribute__((aligned(16))) char lds[STAGES * 2 * RT * RB];
  __shared__ __attribute__((aligned(16))) float rl[2][32], rd[2][32];
  __shared__ __attribute__((aligned(16))) uint32_t rw[2][4][32];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5;
  const uint32_t group = a.heads / a.kv_heads, queries = (uint32_t)a.queries, rows = group * queries;
  const uint32_t key_blocks = (uint32_t)((a.keys + 127) / 128), pairs = (uint32_t)a.batch * a.kv_heads;
  const uint32_t at = near_block(blockIdx.x, gridDim.x), rest = at / key_blocks, key_block = at - rest * key_blocks;
  const uint32_t pair = g.splits > 1 ? rest / (uint32_t)g.splits : rest, split = g.splits > 1 ? rest - pair * g.splits : 0;
  const uint32_t b = pair / (uint32_t)a.kv_heads, kh = pair - b * a.kv_heads;
  const int length = length_of(a, b), key0 = key_block * 128 + wave * 32, key = key0 + (lane & 31);
  // Every splits-th tile of rows, so that under a band each split has its share of those that a key meets.
  const int tiles = (int)((rows + RT - 1) / RT), by = g.splits;
  int t1 = (tiles - (int)split + by - 1) / by;
  if ((int)(key_block * 128) >= length) t1 = 0;   // a block whose keys are all past the length has nothing to sum
  const bool idle = key0 >= length, mine = key < length;
  const int words = (int)words_of(a.keys);
  uint64_t want = 0;
  int want0 = -64;
  auto from = [&](int t) {
    if constexpr (!MASK) return t;
    while (t < t1) {
      if (t - want0 >= 64) {
        want0 = t;
        want = __ballot(any_flag<RT, 128>(a, (min(t + lane, t1 - 1) * by + split) * RT, key_block * 128) && t + lane < t1);
      }
      const uint64_t left = want >> (t - want0);
      if (left) return t + __builtin_ctzll(left);
      t = want0 + 64;
    }
    return t1;
  };
  f32x16 ak[DK ? FD : 1], av[DV ? FD : 1];
#pragma unroll
  for (int f = 0; f < FD; ++f)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (DK) ak[f][i] = 0;
      if constexpr (DV) av[f][i] = 0;
    }
  Scaled<T, DK ? FD : 1> scaled;
  RowsOf<T, RB, DIRECT> qs(a.q, a, b, kh), ds_(g.dout, a, b, kh);
  float nl = 0, nd = 0;
  uint32_t nw = 0;
  // The terms and mask words of a tile's rows, a row a lane (rows past the last have the weights 2^-inf = 0).
  auto look = [&](int t) {
    const uint32_t r = (t * by + split) * RT + (lane & 31);
    nl = r < rows ? g.rows[((int64_t)pair * rows + r) * 2] : INFINITY;
    nd = r < rows ? g.rows[((int64_t)pair * rows + r) * 2 + 1] : 0.0f;
    if constexpr (MASK) nw = r < rows && key0 < a.keys ? a.words[(int64_t)(r % queries) * words + key0 / 32] : 0;
  };
  int t = from(0), buf = 0;
  if (t < t1) {
    qs.load(lds, t * by + split);
    ds_.load(lds + RT * RB, t * by + split);
    look(t);
  }
  // (behind the first tile, which is on its way by now)
  u32x4 k[RB / 32], v[DK ? RB / 32 : 1];
  {
    const char *const pk = (const char *)a.k.p + (b * a.k.batch + key * a.k.row + kh * a.k.head) * (int64_t)sizeof(T);
    const char *const pv = (const char *)a.v.p + (b * a.v.batch + key * a.v.row + kh * a.v.head) * (int64_t)sizeof(T);
    const char *const ek = end_of(a.k, a.batch, a.keys, a.kv_heads, a.d, sizeof(T));
    const char *const ev = end_of(a.v, a.batch, a.keys, a.kv_heads, a.d, sizeof(T));
#pragma unroll
    for (int c = 0; c < RB / 32; ++c) {
      k[c] = u32x4{0, 0, 0, 0};
      if (mine) k[c] = row_piece<T>(pk, 2 * c + h, a.d, ek);
      if constexpr (DK) {
        v[c] = u32x4{0, 0, 0, 0};
        if (mine) v[c] = row_piece<T>(pv, 2 * c + h, a.d, ev);
      }
    }
  }
  for (int turn = 0; t < t1; turn ^= 1) {
    const int next = from(t + 1);
    char *const lq = lds + buf * 2 * RT * RB, *const ld = lq + RT * RB;
    uint32_t any = nw;
    if constexpr (DIRECT) {
      wait_loads();
    } else {
      barrier();   // the tile before has been read
      qs.store(lq);
      ds_.store(ld);
    }
    if (lane < 32) {
      if (wave == 0) {
        rl[turn][lane] = nl;
        rd[turn][lane] = nd;
      }
      if constexpr (MASK) rw[turn][wave][lane] = nw;
    }
    barrier();     // the tile is there for all (DIRECT: and nobody reads the other one any more)
    if (next < t1) {
      qs.load(lds + (DIRECT ? buf ^ 1 : 0) * 2 * RT * RB, next * by + split);
      ds_.load(lds + (DIRECT ? buf ^ 1 : 0) * 2 * RT * RB + RT * RB, next * by + split);
      look(next);
    }
    if constexpr (DIRECT) buf ^= 1;
    bool dense = !idle && (!MASK || __any(any != 0));
    if constexpr (MASK && DK && DV && pairwise<T, RB>() && RB <= 128) {
      if (dense && !__any(__popc(any) > 16)) {
        uint32_t in = turn_bits(any);    // the rows of the tile that may attend the lane's key
        if (!mine) in = 0;
        if (!__any(__popc(in) > kFewPairs)) {
          dense = false;
          while (__any(in != 0)) {
            const int row = in ? __builtin_ctz(in) : 0;
            const HalfRow<RB> q(lq, row, a.d), dout(ld, row, a.d);
            const float s = sum_halves(q.dot(k, a.d)), dp = sum_halves(dout.dot(v, a.d));
            const float p = weight<T>(s, a.scale, rl[turn][row], 0.0f), ds = p * (dp - rd[turn][row]);
            if (in) {
              dout.add_to(av, p, a.d);
              q.add_to(ak, ds, a.d);
            }
            in &= in - 1;
          }
        }
      }
    }
    if (dense) {
      const f32x16 s = times_rows<T, RB, RB == 1024 && DK>(lq, 0, k, a.d);
      f32x16 dp;
      if constexpr (DK) dp = times_rows<T, RB, RB == 1024 && DK>(ld, 0, v, a.d);
      float p[16], ds[16];
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const f32x4 l = *(const f32x4 *)(&rl[turn][row_of(i, h)]), dd = *(const f32x4 *)(&rd[turn][row_of(i, h)]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          p[i + j] = weight<T>(s[i + j], a.scale, l[j], p_shift<T>());
          if constexpr (DK) ds[i + j] = p[i + j] * (dp[i + j] - dd[j]);
        }
      }
      if (!__all(mine && (!MASK || any == ~0u))) {
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          u32x4 w = {~0u, ~0u, ~0u, ~0u};
          if constexpr (MASK) w = *(const u32x4 *)(&rw[turn][wave][row_of(i, h)]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const bool in = mine && (w[j] >> (lane & 31) & 1);
            p[i + j] = in ? p[i + j] : 0.0f;
            if constexpr (DK) ds[i + j] = in ? ds[i + j] : 0.0f;
          }
        }
      }
      if constexpr (DV) add_columns<T, RB, RB == 1024 && DK>(av, ld, 0, p, a.d);
      if constexpr (DK) {
        scaled.apply(ds, ak);
        add_columns<T, RB, RB == 1024 && DK>(ak, lq, 0, ds, a.d);
      }
    }
    t = next;
  }
  if (key >= a.keys) return;
  constexpr float down = __is_same(T, f16_t) ? 0x1p-14f : 1.0f;   // 2^-p_shift
  const float outk = a.scale * scaled.out() * down;
  if (g.part) {
    float *const pk = g.part + (((int64_t)split * 2 * pairs + pair) * a.keys + key) * DP, *const pv = pk + (int64_t)pairs * a.keys * DP;
#pragma unroll
    for (int f = 0; f < FD; ++f)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int c = 32 * f + row_of(i, h);
        if constexpr (DK) *(f32x4 *)(pk + c) = f32x4{ak[f][i] * outk, ak[f][i + 1] * outk, ak[f][i + 2] * outk, ak[f][i + 3] * outk};
        if constexpr (DV) *(f32x4 *)(pv + c) = f32x4{av[f][i] * down, av[f][i + 1] * down, av[f][i + 2] * down, av[f][i + 3] * down};
      }
    return;
  }
  T *const ok = (T *)g.dk.p + b * g.dk.batch + key * g.dk.row + kh * g.dk.head;
  T *const ov = (T *)g.dv.p + b * g.dv.batch + key * g.dv.row + kh * g.dv.head;
#pragma unroll
  for (int f = 0; f < FD; ++f)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int c = 32 * f + row_of(i, h);
      if (c >= a.d) continue;
      if constexpr (DK) store_values4<T>(ok + c, a.d - c, ak[f][i] * outk, ak[f][i + 1] * outk, ak[f][i + 2] * outk, ak[f][i + 3] * outk);
      if constexpr (DV) store_values4<T>(ov + c, a.d - c, av[f][i] * down, av[f][i + 1] * down, av[f][i + 2] * down, av[f][i + 3] * down);
    }
}

// The splits' sums of four columns of a row's dq a thread, in the order of the splits.
template <class T>
__global__ __launch_bounds__(256) void k_join_dq(AttentionGrad g, int dp) {
  const Attention &a = g.a;
  const uint32_t group = a.heads / a.kv_heads, per = dp / 4, queries = (uint32_t)a.queries, rows = group * queries;
  const uint32_t all = (uint32_t)a.batch * a.kv_heads * rows, at = blockIdx.x * 256 + threadIdx.x, row = at / per;
  const int c = (int)(at - row * per) * 4;
  if (row >= all || c >= a.d) return;
  float v[4] = {0, 0, 0, 0};
  for (int s = 0; s < g.splits_q; ++s) {
    const f32x4 x = *(const f32x4 *)(g.part_q + ((int64_t)s * all + row) * dp + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += x[i];
  }
  const uint32_t pair = row / rows, r = row - pair * rows, b = pair / (uint32_t)a.kv_heads;
  const uint32_t head = (pair - b * a.kv_heads) * group + r / queries, query = r % queries;
  store_values4<T>((T *)g.dq.p + b * g.dq.batch + query * g.dq.row + head * g.dq.head + c, a.d - c, v[0], v[1], v[2], v[3]);
}
// The splits' sums of four columns of a key's dk or dv a thread, in the order of the splits.
template <class T>
__global__ __launch_bounds__(256) void k_join_dkv(AttentionGrad g, int dp) {
  const Attention &a = g.a;
  const uint32_t per = dp / 4, keys = (uint32_t)a.keys, all = (uint32_t)a.batch * a.kv_heads * keys;
  const uint32_t at = blockIdx.x * 256 + threadIdx.x, row = at / per;
  const int c = (int)(at - row * per) * 4;
  if (row >= 2 * all || c >= a.d) return;
  float v[4] = {0, 0, 0, 0};
  for (int s = 0; s < g.splits; ++s) {
    const f32x4 x = *(const f32x4 *)(g.part + ((int64_t)s * 2 * all + row) * dp + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += x[i];
  }
  const Heads &o = row < all ? g.dk : g.dv;
  const uint32_t pk = row < all ? row : row - all, pair = pk / keys, key = pk - pair * keys, b = pair / (uint32_t)a.kv_heads;
  store_values4<T>((T *)o.p + b * o.batch + key * o.row + (pair - b * a.kv_heads) * o.head + c, a.d - c, v[0], v[1], v[2], v[3]);
}

template <class T, int DP, bool MASK, bool DIRECT>
void launch_dkv(const AttentionGrad &g, dim3 grid, hipStream_t s) {
  // Rows of 256 values, or 192 in fp32, leave no registers for both sums beside a key and its value.
  if constexpr (DP == 256 || DP * sizeof(T) > 512) {
    k_attention_dkv<T, DP, MASK, true, false, DIRECT><<<grid, 256, 0, s>>>(g);
    k_attention_dkv<T, DP, MASK, false, true, DIRECT><<<grid, 256, 0, s>>>(g);
  } else {
    k_attention_dkv<T, DP, MASK, true, true, DIRECT><<<grid, 256, 0, s>>>(g);
  }
}
template <class T, int DP, bool MASK>
hipError_t launch_shape(const AttentionGrad &g, hipStream_t s) {
  const Attention &a = g.a;
  const int64_t rows = (int64_t)(a.heads / a.kv_heads) * a.queries, pairs = a.batch * a.kv_heads;
  hipError_t err = hipSuccess;
  if (rows) {
    const dim3 grid((unsigned)((rows + 127) / 128 * pairs * g.splits_q));
    if (!g.dq.p) k_attention_rows<T><<<dim3((unsigned)((rows * pairs + 15) / 16)), 256, 0, s>>>(g);
    else if (direct_ok<T>(a.k, a) && direct_ok<T>(a.v, a)) k_attention_dq<T, DP, MASK, true><<<grid, 256, 0, s>>>(g);
    else k_attention_dq<T, DP, MASK, false><<<grid, 256, 0, s>>>(g);
    if ((err = hipGetLastError()) != hipSuccess) return err;
    if (g.dq.p && g.splits_q > 1) {
      k_join_dq<T><<<dim3((unsigned)((rows * pairs * (DP / 4) + 255) / 256)), 256, 0, s>>>(g, DP);
      if ((err = hipGetLastError()) != hipSuccess) return err;
    }
  }
  if (!g.dk.p) return err;
  const dim3 grid((unsigned)((a.keys + 127) / 128 * pairs * g.splits));
  if (direct_rows<T>(a.q, a) && direct_rows<T>(g.dout, a)) launch_dkv<T, DP, MASK, true>(g, grid, s);
  else launch_dkv<T, DP, MASK, false>(g, grid, s);
  if ((err = hipGetLastError()) != hipSuccess || !g.part) return err;
  const int64_t threads = 2 * pairs * a.keys * (DP / 4);
  k_join_dkv<T><<<dim3((unsigned)((threads + 255) / 256)), 256, 0, s>>>(g, DP);
  return hipGetLastError();
}
template <class T>
hipError_t launch_type(const AttentionGrad &g, hipStream_t s) {
  switch (d_of(g.a.d)) {
    case 32: return g.a.mask ? launch_shape<T, 32, true>(g, s) : launch_shape<T, 32, false>(g, s);
    case 64: return g.a.mask ? launch_shape<T, 64, true>(g, s) : launch_shape<T, 64, false>(g, s);
    case 128: return g.a.mask ? launch_shape<T, 128, true>(g, s) : launch_shape<T, 128, false>(g, s);
    case 192: return g.a.mask ? launch_shape<T, 192, true>(g, s) : launch_shape<T, 192, false>(g, s);
    default: return g.a.mask ? launch_shape<T, 256, true>(g, s) : launch_shape<T, 256, false>(g, s);
  }
}

}  // namespace

// Splits of `blocks` blocks that take `tiles` tiles each, at most `most`: as many as make `fill` blocks.  fp32 rows of more than 64 values
// (`alone`) leave a compute unit room for one block, so what counts there is the rounds of 256 blocks, each of its tiles and about two more for its begin and end (gradient of 2 x 1024 on 1024, 8/4 heads of 256,
// with 768 and 512 blocks 1068 us, by rounds 915; 79 x 96 on 7, 32/4 of 128, 316 blocks unsplit 659, by rounds 533).
static int splits_of(bool alone, int64_t blocks, int64_t tiles, int64_t most, int64_t fill) {
  if (most > 32) most = 32;
  if (blocks <= 0 || most < 2) return 1;
  if (!alone) {
    const int64_t s = fill / blocks < most ? fill / blocks : most;
    return s > 1 ? (int)s : 1;
  }
  if (blocks > 1 << 16) return 1;      // many rounds either way
  int64_t best = 1, least = 0;
  for (int64_t s = 1; s <= most; ++s) {
    const int64_t time = (blocks * s + 255) / 256 * ((tiles + s - 1) / s + 2);
    if (s == 1 || time < least) best = s, least = time;
  }
  return (int)best;
}

AttentionGradPlan plan_attention_grad(int type, int64_t batch, int64_t queries, int64_t keys, int heads, int kv_heads, int d,
                                      bool masked) {
  AttentionGradPlan p{};
  const int64_t rows = (int64_t)(heads / kv_heads) * queries, pairs = batch * kv_heads;
  const bool alone = type == AECCT_F32 && d > 64;
  p.splits = splits_of(alone, (keys + 127) / 128 * pairs, (rows + 31) / 32, rows / 128, 768);
  if (masked) {
    p.words = (size_t)(queries * words_of(keys)) * 4;
    p.flags = (size_t)((queries + 31) / 32 * (words_of(keys) / 2));
  }
  p.rows = (size_t)(rows * pairs) * 8;
  if (p.splits > 1) p.part = (size_t)(p.splits * 2 * pairs * keys * d_of(d)) * 4;
  // dq's blocks of 128 rows, where they are few, split the keys: at least 256 keys each.
  p.splits_q = splits_of(alone, (rows + 127) / 128 * pairs, (keys + 31) / 32, keys / 256, 512);
  if (p.splits_q > 1) p.part_q = (size_t)(p.splits_q * pairs * rows * d_of(d)) * 4;
  return p;
}

hipError_t launch_attention_grad(int type, const AttentionGrad &g, hipStream_t s) {
  if (g.a.mask) {
    const hipError_t err = launch_mask(g.a, s);
    if (err != hipSuccess) return err;
  }
  switch (type) {
    case AECCT_F32: return launch_type<float>(g, s);
    case AECCT_BF16: return launch_type<bf16_t>(g, s);
    case AECCT_F16: return launch_type<f16_t>(g, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace aecct
