// The gradient of cross attention from its output and the logarithms of its rows' sums:
//   p = exp(scale q k^T - lse),  D = sum of dout o over d,  ds = p (dout v^T - D),
//   dq = scale ds k,  dk = scale ds^T q,  dv = p^T dout.
// dk and dv sum over rows and dq over keys, so they are two kernels, each of which computes p and ds for itself: seven products in
// place of five, and no sums in memory whose order could change.  Every sum over the heads that share a key head is one over rows.
//
// As in the forward pass the scores are computed so that a lane's registers are the second factor of the products that follow:
// keys by rows for dq, rows by keys for dk and dv.
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

// lse log2(e) (a row that attends nothing: infinity, so that its weights are 0) and D, a wavefront a row.
template <class T>
__global__ __launch_bounds__(256) void k_attention_rows(AttentionGrad g) {
  const Attention &a = g.a;
  const int lane = threadIdx.x & 63, group = a.heads / a.kv_heads;
  const int64_t rows = group * a.queries, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows * a.batch * a.kv_heads) return;
  const int64_t pair = row / rows, r = row % rows, b = pair / a.kv_heads;
  const int64_t head = pair % a.kv_heads * group + r / a.queries, query = r % a.queries;
  const T *const o = (const T *)a.o.p + b * a.o.batch + query * a.o.row + head * a.o.head;
  const T *const d = (const T *)g.dout.p + b * g.dout.batch + query * g.dout.row + head * g.dout.head;
  float sum = 0;
  for (int c = lane; c < a.d; c += 64) sum = fmaf((float)o[c], (float)d[c], sum);
#pragma unroll
  for (int i = 1; i < 64; i *= 2) sum += __shfl_xor(sum, i);
  if (lane == 0) {
    const float lse = a.lse[(b * a.heads + head) * a.queries + query];
    g.rows[row * 2] = lse == -INFINITY ? INFINITY : lse * kLog2e;
    g.rows[row * 2 + 1] = lse == -INFINITY ? 0.0f : sum;
  }
}

// dq: a wavefront takes 32 rows, tiles of 32 keys pass through LDS.
template <class T, int DP, bool MASK>
__global__ __launch_bounds__(256) void k_attention_dq(AttentionGrad g) {
  constexpr int RB = DP * (int)sizeof(T), FD = DP / 32, NT = 256, KT = 32, CH = RB / 16, PER = (KT * CH + NT - 1) / NT;
  const Attention &a = g.a;
  __shared__ __attribute__((aligned(16))) char lds[2 * KT * RB];
  char *const lk = lds, *const lv = lds + KT * RB;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5, group = a.heads / a.kv_heads;
  const int64_t rows = group * a.queries, row_blocks = (rows + 127) / 128;
  const int64_t at = near_block(blockIdx.x, gridDim.x), row_block = at % row_blocks, pair = at / row_blocks, b = pair / a.kv_heads;
  const int kh = (int)(pair % a.kv_heads);
  const int64_t length = length_of(a, b), t1 = (length + KT - 1) / KT;
  const int64_t r = row_block * 128 + wave * 32 + (lane & 31), rc = r < rows ? r : rows - 1;
  const int64_t head = kh * group + rc / a.queries, query = rc % a.queries;
  const bool idle = row_block * 128 + wave * 32 >= rows;
  u32x4 q[RB / 32], dout[RB / 32];
  {
    const char *const p = (const char *)a.q.p + (b * a.q.batch + query * a.q.row + head * a.q.head) * (int64_t)sizeof(T);
    const char *const pd = (const char *)g.dout.p + (b * g.dout.batch + query * g.dout.row + head * g.dout.head) * (int64_t)sizeof(T);
    const char *const end = end_of(a.q, a.batch, a.queries, a.heads, a.d, sizeof(T));
    const char *const endd = end_of(g.dout, a.batch, a.queries, a.heads, a.d, sizeof(T));
#pragma unroll
    for (int c = 0; c < RB / 32; ++c) {
      q[c] = row_piece<T>(p, 2 * c + h, a.d, end);
      dout[c] = row_piece<T>(pd, 2 * c + h, a.d, endd);
    }
  }
  const float l2 = g.rows[(pair * rows + rc) * 2], dd = g.rows[(pair * rows + rc) * 2 + 1], to2 = a.scale * kLog2e;
  const char *const pk = (const char *)a.k.p + (b * a.k.batch + kh * a.k.head) * (int64_t)sizeof(T);
  const char *const pv = (const char *)a.v.p + (b * a.v.batch + kh * a.v.head) * (int64_t)sizeof(T);
  const char *const ek = end_of(a.k, a.batch, a.keys, a.kv_heads, a.d, sizeof(T));
  const char *const ev = end_of(a.v, a.batch, a.keys, a.kv_heads, a.d, sizeof(T));
  const int64_t words = words_of(a.keys), flag_tiles = words / 2;
  uint64_t want = 0;
  int64_t want0 = -64;
  auto from = [&](int64_t t) {
    if constexpr (!MASK) return t;
    while (t < t1) {
      if (t - want0 >= 64) {
        want0 = t;
        want = __ballot(t + lane < t1 && any_flag(a.flags, row_block * 4, 4, (rows + 31) / 32, (t + lane) * KT, KT, flag_tiles));
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
  u32x4 ck[PER], cv[PER];
  auto load = [&](int64_t t) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int slot = threadIdx.x + i * NT, row = slot / CH, chunk = slot % CH;
      const int64_t key = t * KT + row;
      ck[i] = cv[i] = u32x4{0, 0, 0, 0};
      if (row < KT && key < length) {
        ck[i] = row_piece<T>(pk + key * a.k.row * (int64_t)sizeof(T), chunk, a.d, ek);
        cv[i] = row_piece<T>(pv + key * a.v.row * (int64_t)sizeof(T), chunk, a.d, ev);
      }
    }
  };
  int64_t t = from(0);
  if (t < t1) load(t);
  while (t < t1) {
    const int64_t next = from(t + 1);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int slot = threadIdx.x + i * NT, row = slot / CH, chunk = slot % CH;
      if (row >= KT) continue;
      const int to = row * RB + ((chunk << 4) ^ exchange<RB>(row));
      *(u32x4 *)(lk + to) = ck[i];
      *(u32x4 *)(lv + to) = cv[i];
    }
    __syncthreads();
    if (next < t1) load(next);
    const int64_t k0 = t * KT;
    int flag = 2;
    if constexpr (MASK) flag = !idle ? a.flags[(row_block * 4 + wave) * flag_tiles + k0 / 64] : 0;
    if (!idle && flag != 0) {
      const f32x16 s = times_rows<T, RB>(lk, 0, q), dp = times_rows<T, RB>(lv, 0, dout);
      uint32_t w = ~0u;
      if (k0 + 32 > length) w = (1u << (length - k0)) - 1;
      if constexpr (MASK) {
        if (flag == 1) w &= a.words[query * words + k0 / 32];
      }
      w >>= 4 * h;
      float ds[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[i], to2, -l2));
        ds[i] = w >> row_of(i, 0) & 1 ? p * (dp[i] - dd) : 0.0f;
      }
      scaled.apply(ds, acc);
      add_columns<T, RB, FD>(acc, lk, 0, ds);
    }
    t = next;
  }
  if (r >= rows) return;
  const float out = a.scale * scaled.out();
  T *const o = (T *)g.dq.p + b * g.dq.batch + query * g.dq.row + head * g.dq.head;
#pragma unroll
  for (int f = 0; f < FD; ++f)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int c = 32 * f + row_of(i, h);
      if (c < a.d) store_values4<T>(o + c, a.d - c, acc[f][i] * out, acc[f][i + 1] * out, acc[f][i + 2] * out, acc[f][i + 3] * out);
    }
}

// dk and dv (DK, DV: which of them): a wavefront takes 32 keys, tiles of 32 rows pass through LDS.
template <class T, int DP, bool MASK, bool DK, bool DV>
__global__ __launch_bounds__(256) void k_attention_dkv(AttentionGrad g) {
  constexpr int RB = DP * (int)sizeof(T), FD = DP / 32, NT = 256, RT = 32, CH = RB / 16, PER = (RT * CH + NT - 1) / NT;
  const Attention &a = g.a;
  __shared__ __attribute__((aligned(16))) char lds[2 * RT * RB];
  __shared__ __attribute__((aligned(16))) float rl[32], rd[32];
  __shared__ __attribute__((aligned(16))) uint32_t rw[4][32];
  char *const lq = lds, *const ld = lds + RT * RB;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5, group = a.heads / a.kv_heads;
  const int64_t rows = group * a.queries, key_blocks = (a.keys + 127) / 128, pairs = a.batch * a.kv_heads;
  const int64_t at = near_block(blockIdx.x, gridDim.x), key_block = at % key_blocks, rest = at / key_blocks;
  const int64_t pair = rest / g.splits, b = pair / a.kv_heads;
  const int split = (int)(rest % g.splits), kh = (int)(pair % a.kv_heads);
  const int64_t length = length_of(a, b), key = key_block * 128 + wave * 32 + (lane & 31), key0 = key_block * 128 + wave * 32;
  const int64_t tiles = (rows + RT - 1) / RT, t0 = tiles * split / g.splits;
  // A block whose keys are all past the length has nothing to sum.
  const int64_t t1 = key_block * 128 < length ? tiles * (split + 1) / g.splits : t0;
  const bool idle = key0 >= length;
  const float to2 = a.scale * kLog2e;
  u32x4 k[RB / 32], v[DK ? RB / 32 : 1];
  {
    const char *const pk = (const char *)a.k.p + (b * a.k.batch + key * a.k.row + kh * a.k.head) * (int64_t)sizeof(T);
    const char *const pv = (const char *)a.v.p + (b * a.v.batch + key * a.v.row + kh * a.v.head) * (int64_t)sizeof(T);
    const char *const ek = end_of(a.k, a.batch, a.keys, a.kv_heads, a.d, sizeof(T));
    const char *const ev = end_of(a.v, a.batch, a.keys, a.kv_heads, a.d, sizeof(T));
#pragma unroll
    for (int c = 0; c < RB / 32; ++c) {
      k[c] = u32x4{0, 0, 0, 0};
      if (key < length) k[c] = row_piece<T>(pk, 2 * c + h, a.d, ek);
      if constexpr (DK) {
        v[c] = u32x4{0, 0, 0, 0};
        if (key < length) v[c] = row_piece<T>(pv, 2 * c + h, a.d, ev);
      }
    }
  }
  const int64_t words = words_of(a.keys), flag_tiles = words / 2;
  uint64_t want = 0;
  int64_t want0 = t0 - 64;
  auto from = [&](int64_t t) {
    if constexpr (!MASK) return t;
    while (t < t1) {
      if (t - want0 >= 64) {
        want0 = t;
        want = __ballot(t + lane < t1 && any_flag(a.flags, t + lane, 1, tiles, key_block * 128, 128, flag_tiles));
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
  const char *const pq = (const char *)a.q.p + b * a.q.batch * (int64_t)sizeof(T);
  const char *const pd = (const char *)g.dout.p + b * g.dout.batch * (int64_t)sizeof(T);
  const char *const eq = end_of(a.q, a.batch, a.queries, a.heads, a.d, sizeof(T));
  const char *const ed = end_of(g.dout, a.batch, a.queries, a.heads, a.d, sizeof(T));
  u32x4 cq[PER], cd[PER];
  float nl = 0, nd = 0;
  uint32_t nw = 0;
  auto load = [&](int64_t t) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int slot = threadIdx.x + i * NT, row = slot / CH, chunk = slot % CH;
      const int64_t r = t * RT + row;
      cq[i] = cd[i] = u32x4{0, 0, 0, 0};
      if (row < RT && r < rows) {
        const int64_t head = kh * group + r / a.queries, query = r % a.queries;
        cq[i] = row_piece<T>(pq + (query * a.q.row + head * a.q.head) * (int64_t)sizeof(T), chunk, a.d, eq);
        cd[i] = row_piece<T>(pd + (query * g.dout.row + head * g.dout.head) * (int64_t)sizeof(T), chunk, a.d, ed);
      }
    }
    if (lane < 32) {
      const int64_t r = t * RT + lane;
      // rows past the last have the weights 2^-inf = 0
      nl = r < rows ? g.rows[(pair * rows + r) * 2] : INFINITY;
      nd = r < rows ? g.rows[(pair * rows + r) * 2 + 1] : 0.0f;
      if constexpr (MASK) nw = r < rows && key0 < a.keys ? a.words[r % a.queries * words + key0 / 32] : 0;
    }
  };
  int64_t t = from(t0);
  if (t < t1) load(t);
  while (t < t1) {
    const int64_t next = from(t + 1);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int slot = threadIdx.x + i * NT, row = slot / CH, chunk = slot % CH;
      if (row >= RT) continue;
      const int to = row * RB + ((chunk << 4) ^ exchange<RB>(row));
      *(u32x4 *)(lq + to) = cq[i];
      *(u32x4 *)(ld + to) = cd[i];
    }
    if (lane < 32) {
      if (wave == 0) {
        rl[lane] = nl;
        rd[lane] = nd;
      }
      if constexpr (MASK) rw[wave][lane] = nw;
    }
    __syncthreads();
    if (next < t1) load(next);
    bool none = idle;
    if constexpr (MASK) none = none || a.flags[t * flag_tiles + key0 / 64] == 0;
    if (!none) {
      const f32x16 s = times_rows<T, RB>(lq, 0, k);
      f32x16 dp;
      if constexpr (DK) dp = times_rows<T, RB>(ld, 0, v);
      float p[16], ds[16];
      const bool mine = key < length;
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const f32x4 l2 = *(const f32x4 *)(rl + row_of(i, h)), dd = *(const f32x4 *)(rd + row_of(i, h));
        u32x4 w = {~0u, ~0u, ~0u, ~0u};
        if constexpr (MASK) w = *(const u32x4 *)(&rw[wave][row_of(i, h)]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool in = mine && (!MASK || (w[j] >> (lane & 31) & 1));
          p[i + j] = in ? __builtin_amdgcn_exp2f(fmaf(s[i + j], to2, p_shift<T>() - l2[j])) : 0.0f;
          if constexpr (DK) ds[i + j] = in ? p[i + j] * (dp[i + j] - dd[j]) : 0.0f;
        }
      }
      if constexpr (DV) add_columns<T, RB, FD>(av, ld, 0, p);
      if constexpr (DK) {
        scaled.apply(ds, ak);
        add_columns<T, RB, FD>(ak, lq, 0, ds);
      }
    }
    t = next;
  }
  if (key >= a.keys) return;
  constexpr float down = __is_same(T, f16_t) ? 0x1p-14f : 1.0f;   // 2^-p_shift
  const float outk = a.scale * scaled.out() * down;
  if (g.part) {
    float *const pk = g.part + (((int64_t)split * 2 * pairs + pair) * a.keys + key) * DP, *const pv = pk + pairs * a.keys * DP;
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

// The splits' sums of four columns of a key's dk or dv a thread, in the order of the splits.
template <class T>
__global__ __launch_bounds__(256) void k_join_dkv(AttentionGrad g, int dp) {
  const Attention &a = g.a;
  const int64_t pairs = a.batch * a.kv_heads, at = (int64_t)blockIdx.x * 256 + threadIdx.x, per = dp / 4, all = pairs * a.keys;
  const int64_t row = at / per;
  const int c = (int)(at % per) * 4;
  if (row >= 2 * all || c >= a.d) return;
  float v[4] = {0, 0, 0, 0};
  for (int s = 0; s < g.splits; ++s) {
    const f32x4 x = *(const f32x4 *)(g.part + (s * 2 * all + row) * dp + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += x[i];
  }
  const Heads &o = row < all ? g.dk : g.dv;
  const int64_t pk = row < all ? row : row - all, pair = pk / a.keys, key = pk % a.keys;
  store_values4<T>((T *)o.p + pair / a.kv_heads * o.batch + key * o.row + pair % a.kv_heads * o.head + c, a.d - c, v[0], v[1], v[2], v[3]);
}

template <class T, int DP, bool MASK>
hipError_t launch_shape(const AttentionGrad &g, hipStream_t s) {
  const Attention &a = g.a;
  const int64_t rows = (int64_t)(a.heads / a.kv_heads) * a.queries, pairs = a.batch * a.kv_heads;
  hipError_t err = hipSuccess;
  if (rows) {
    k_attention_rows<T><<<dim3((unsigned)((rows * pairs + 3) / 4)), 256, 0, s>>>(g);
    if ((err = hipGetLastError()) != hipSuccess) return err;
    if (g.dq.p) {
      k_attention_dq<T, DP, MASK><<<dim3((unsigned)((rows + 127) / 128 * pairs)), 256, 0, s>>>(g);
      if ((err = hipGetLastError()) != hipSuccess) return err;
    }
  }
  if (!g.dk.p) return err;
  const dim3 grid((unsigned)((a.keys + 127) / 128 * pairs * g.splits));
  // Rows of 256 fp32 values leave no registers for both sums beside a key and its value.
  if constexpr (DP * sizeof(T) > 512) {
    k_attention_dkv<T, DP, MASK, true, false><<<grid, 256, 0, s>>>(g);
    if ((err = hipGetLastError()) != hipSuccess) return err;
    k_attention_dkv<T, DP, MASK, false, true><<<grid, 256, 0, s>>>(g);
  } else {
    k_attention_dkv<T, DP, MASK, true, true><<<grid, 256, 0, s>>>(g);
  }
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
    default: return g.a.mask ? launch_shape<T, 256, true>(g, s) : launch_shape<T, 256, false>(g, s);
  }
}

}  // namespace

AttentionGradPlan plan_attention_grad(int type, int64_t batch, int64_t queries, int64_t keys, int heads, int kv_heads, int d,
                                      bool masked) {
  AttentionGradPlan p{};
  const int64_t rows = (int64_t)(heads / kv_heads) * queries, pairs = batch * kv_heads, blocks = (keys + 127) / 128 * pairs;
  int64_t splits = blocks > 0 ? 768 / blocks : 1;
  if (splits > rows / 256) splits = rows / 256;
  if (splits > 32) splits = 32;
  p.splits = splits > 1 ? (int)splits : 1;
  if (masked) {
    p.words = (size_t)(queries * words_of(keys)) * 4;
    p.flags = (size_t)((rows + 31) / 32 * (words_of(keys) / 2));
  }
  p.rows = (size_t)(rows * pairs) * 8;
  if (p.splits > 1) p.part = (size_t)(p.splits * 2 * pairs * keys * d_of(d)) * 4;
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
