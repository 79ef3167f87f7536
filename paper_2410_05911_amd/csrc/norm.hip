// Root-mean-square norm of rows with the residual's addition and Eq. 2 codes, and its gradient.
//
// With h = x + res, rho = 1 / sqrt(mean(h^2) + eps) and y = h rho gain a row needs two sums over its columns (of h^2, and
// for the gradient of dy gain h) or a sum and a maximum, and then one multiple of what it read.  Both directions are bound
// by device memory: a row is read once into registers, its two sums are joined together, and it is written.  A row is held
// by TPR threads, NV vectors of 16 bytes a thread: 8 to 64 lanes of a wavefront for short rows (several rows a wavefront,
// no barrier), a block of 256 to 1024 threads for long ones, two passes beyond 16384 columns.
//
// Measured on an MI355X, where a copy of 1 GB runs at 5.1 TB/s and one that fits its caches at 6 to 8: the norm of 16384
// rows of 8192 bf16 to e4m3 codes 170 us (5.5 TB/s; about 30 vector instructions a value, 0.6 of
// the time), of 49152 rows of 128 fp32 to int8 codes 14.5 us (5.6 TB/s), of 16384 rows of 4096 bf16 81 us (6.6 TB/s);
// the gradient of the last 71 us (5.7 TB/s); of one row 3 to 4 us, all latency.
#include <algorithm>

#include "device_common.h"
#include "norm.h"
#include "row_io.h"

namespace aecct {
namespace {

// ---- joins over the lanes of a row -----------------------------------------------------------------------------
struct Sum {
  static __device__ __forceinline__ float join(float a, float b) { return a + b; }
};
struct Max {   // of non-negative floats, whose bits order like them; NaN is above all
  static __device__ __forceinline__ float join(float a, float b) {
    return __builtin_bit_cast(float, max(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)));
  }
};
struct Largest {   // of any floats
  static __device__ __forceinline__ float join(float a, float b) { return fmaxf(a, b); }
};
template <class Op, int CTRL>
__device__ __forceinline__ float dpp_join(float v) {
  return Op::join(v, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true)));
}
template <class Op, int M>
__device__ __forceinline__ float swap_join(float v) {
  uint32_t a, b;
  lane_swap_pair<M>(__builtin_bit_cast(uint32_t, v), a, b);
  return Op::join(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
// Over each aligned group of `lanes` (4 to 64, a power of two) lanes of a wavefront; the same bits in every lane: the
// pairs of quads, then mirrored halves of 8 and of 16 lanes, then the swaps of 16 and of 32.
template <class Op>
__device__ __forceinline__ float lanes_join(float v, int lanes) {
  v = dpp_join<Op, 0xB1>(v);    // quad_perm [1, 0, 3, 2]
  v = dpp_join<Op, 0x4E>(v);    // quad_perm [2, 3, 0, 1]
  if (lanes >= 8) v = dpp_join<Op, 0x141>(v);   // row_half_mirror
  if (lanes >= 16) v = dpp_join<Op, 0x140>(v);  // row_mirror
  if (lanes >= 32) v = swap_join<Op, 16>(v);
  if (lanes >= 64) v = swap_join<Op, 32>(v);
  return v;
}
// Two values of a row, the first a sum, joined over its TPR threads in a fixed order, the second by Op2.
template <class Op2, int TPR>
__device__ __forceinline__ void row_join(float &a, float &b, float2 *lds) {
  a = lanes_join<Sum>(a, TPR < 64 ? TPR : 64);
  b = lanes_join<Op2>(b, TPR < 64 ? TPR : 64);
  if constexpr (TPR > 64) {
    __syncthreads();   // the last join's values are read
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = float2{a, b};
    __syncthreads();
    a = lds[0].x;
    b = lds[0].y;
#pragma unroll
    for (int w = 1; w < TPR / 64; ++w) {
      a += lds[w].x;
      b = Op2::join(b, lds[w].y);
    }
  }
}

// 1 / sqrt(mean + eps): the hardware's reciprocal square root, within 2^-23 of it for normal arguments.
__device__ __forceinline__ float near_rho(float ss, float inv_d, float eps) {
  return __builtin_amdgcn_rsqf(fmaf(ss, inv_d, eps));
}
__device__ __forceinline__ bool in_range(float s) { return s >= 1e-24f && s <= 1e37f; }

// rho in [2^k, 2^(k + 1)); -1 for 0, infinity and NaN, which the scaling leaves what they are
__device__ __forceinline__ int exponent_of(float rho) { return __builtin_amdgcn_frexp_expf(rho) - 1; }

// A row's rho = 1 / sqrt(mean(h^2) + eps) where the plain fp32 sum of squares is out of range: h is scaled by a power of
// two first, `unit`, and by a second that takes rho into [1, 2), so that products with h stay in range; h rho is
// unchanged and the rho of the row as it was is rho unit.
__device__ __forceinline__ float far_up(float ss) { return in_range(ss) ? 1.0f : ss < 1.0f ? 0x1p100f : 0x1p-100f; }
__device__ __forceinline__ float far_rho_of(float ss, float up, float inv_d, float eps, float &more) {
  float rho;
  int e = 0;
  if (up > 1.0f && eps >= 1e-30f) {   // eps up^2 would overflow: the mean as it was, to which tiny squares add little
    rho = __builtin_amdgcn_rsqf(fmaf(ss * 0x1p-100f * 0x1p-100f, inv_d, eps));
    e = -100;
  } else {
    rho = __builtin_amdgcn_rsqf(fmaf(ss, inv_d, eps * up * up));
  }
  const int k = exponent_of(rho);
  more = ldexpf(1.0f, e + k);
  return ldexpf(rho, -k);
}
template <int TPR, int N>
__device__ __forceinline__ float far_rho(float ss, float (&h)[N], float inv_d, float eps, float &unit, float2 *lds) {
  const float up = far_up(ss);
  float none = 0;
  ss = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    h[i] *= up;
    ss = fmaf(h[i], h[i], ss);
  }
  row_join<Sum, TPR>(ss, none, lds);
  float more;
  const float rho = far_rho_of(ss, up, inv_d, eps, more);
#pragma unroll
  for (int i = 0; i < N; ++i) h[i] *= more;
  unit = up * more;
  return rho;
}

// Products h gain below this are taken of h 2^k instead, and rho 2^-k, with k such that rho 2^-k lies in [2^-100, 2^-99):
// |h rho| is at most 2^8, so h 2^k cannot overflow, and wherever |h gain rho| is not below fp32's smallest number, h 2^k gain
// is above 2^-51 and its rounding error a normal number too.
constexpr float kTiny = 0x1p-60f;
template <int N>
__device__ __forceinline__ float lift(float *h, float rho) {   // scales h, returns rho for it
  const int k = 100 + exponent_of(rho);
#pragma unroll
  for (int i = 0; i < N; ++i) h[i] = ldexpf(h[i], k);
  return ldexpf(rho, -k);
}

// Where a thread's columns lie: vector j starts at column col(j).  A row of d = V k + tail values ends in a vector of
// `tail` values, the jt-th of one lane; only that lane runs the code for it, once for all j.
template <int V, int TPR, int NV>
struct Columns {
  int d, lane, tail, jt;
  bool last;   // this lane holds the short vector
  __device__ __forceinline__ Columns(int d, int lane)
      : d(d), lane(lane), tail(d % V), jt(d / V / TPR), last(tail && jt < NV && d / V % TPR == lane) {}
  __device__ __forceinline__ int col(int j) const { return (j * TPR + lane) * V; }
  __device__ __forceinline__ bool full(int j) const { return col(j) + V <= d; }
  // PAST: past the caches.  ENDS, for rows of d >= V values that no thread writes before all have settled theirs: the
  // short vector is read as the V values that end the row, by one load as the others', and nothing waits until settle()
  // moves them to their place (20000 rows of 5007 bf16 values 102 -> 80 us, their gradient 146 -> 119).
  template <bool PAST, bool ENDS, class T>
  __device__ __forceinline__ void load(const T *p, bool live, Raw<T, V> (&v)[NV]) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = col(j);
      if (live && (ENDS ? c < d : full(j))) load_raw<T, V, PAST>(p + (ENDS && c > d - V ? d - V : c), v[j]);
      else v[j] = Raw<T, V>{};
    }
    if constexpr (!ENDS) {
      if (live && last) {
        Raw<T, V> t;
        load_raw_part<T, V>(p + col(jt), tail, t);
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (j == jt) v[j] = t;
      }
    }
  }
  template <class T>
  __device__ __forceinline__ void settle(Raw<T, V> (&v)[NV]) const {
    if (last) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (j == jt) move_down(v[j], V - tail);
    }
  }
  template <class T, class F>   // f(j, v): the V values of vector j
  __device__ __forceinline__ void store(T *p, bool live, bool past, F f) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float v[V];
      f(j, v);
      if (live && full(j)) {
        if (past) store_vec<T, V, true>(p + col(j), v);
        else store_vec<T, V>(p + col(j), v);
      }
      if (live && last && j == jt) store_part<T, V>(p + col(j), tail, v);
    }
  }
  template <class T>
  __device__ __forceinline__ void gain(const void *p, bool f32, float (&g)[NV * V]) const {
    if (!p) {
#pragma unroll
      for (int i = 0; i < NV * V; ++i) g[i] = 1.0f;
    } else if (f32) {
      Raw<float, V> v[NV];
      load<false, false>((const float *)p, true, v);
#pragma unroll
      for (int j = 0; j < NV; ++j) unpack<float, V>(v[j], (float (&)[V])g[j * V]);
    } else {
      Raw<T, V> v[NV];
      load<false, false>((const T *)p, true, v);
#pragma unroll
      for (int j = 0; j < NV; ++j) unpack<T, V>(v[j], (float (&)[V])g[j * V]);
    }
  }
};

// Which of a block's rows this thread works on; one row a wavefront or a block is told to the compiler as such.
template <int TPR, int BLOCK>
__device__ __forceinline__ int row_of_block() {
  if constexpr (TPR == BLOCK) return 0;
  else if constexpr (TPR == 64) return __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  else return threadIdx.x / TPR;
}

// ---- codes -----------------------------------------------------------------------------------------------------
// code = round(p Q / A) with p = h gain and A = max |p|: rho is a factor of both y and alpha and drops out.  Everything is
// taken with its rounding error beside it, p + e and A + E, and the quotient as (p + e)(q + q1), q a near Q / A and q1
// what it lacks: a code then differs from the exact one only where the quotient is within 2^-24 of a tie.  A row, or a group
// of its columns, whose products h gain are tiny is scaled first (kTiny), since neither they nor their errors need be
// numbers of fp32.
constexpr float kNoTail = -3e38f;
// max |p| of each vector of a thread's values
template <int V, int NV>
__device__ __forceinline__ float vector_max(const float *h, const float *g, float (&m)[NV]) {
  float A = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    m[j] = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) m[j] = Max::join(m[j], fabsf(h[j * V + i] * g[j * V + i]));
    A = Max::join(A, m[j]);
  }
  return A;
}
// The largest rounding error among the values whose |p| is A.
template <int N>
__device__ __forceinline__ float tail_of(float A, const float *h, const float *g) {
  float E = kNoTail;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float p = fabsf(h[i]) * fabsf(g[i]), e = fmaf(fabsf(h[i]), fabsf(g[i]), -p);
    E = p == A ? fmaxf(E, e) : E;
  }
  return E;
}
struct CodeScale {
  float up, q, q1;   // up: a power of two that keeps q1 a normal number
};
__device__ __forceinline__ CodeScale code_scale(float alpha, float A, float E, float most) {
  CodeScale s;
  s.up = A > 0x1p60f ? 0x1p-60f : 1.0f;
  const float b = A * s.up, r = __builtin_amdgcn_rcpf(b), t = E > kNoTail ? E * s.up : 0.0f;
  s.q = most * r;
  s.q1 = b <= 3e38f ? fmaf(-s.q, t, fmaf(-s.q, b, most)) * r : 0.0f;
  if (!(alpha > 0)) {   // codes 0, or NaN where alpha is: of every value, also where rho alone is 0 or NaN
    s.q = alpha;
    s.q1 = 0;
  }
  return s;
}
template <int V>
__device__ __forceinline__ void codes_of(int code, float alpha, float A, float E, const float *h, const float *g,
                                         uint32_t (&w)[V / 4]) {
  const CodeScale s = code_scale(alpha, A, E, code == 1 ? 127.0f : 448.0f);
  float v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float p = h[i] * g[i], e = fmaf(h[i], g[i], -p);
    v[i] = fmaf(p, s.q, fmaf(p, s.q1, e * s.q));
  }
  if (s.up != 1.0f) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float x = h[i] * s.up, p = x * g[i], e = fmaf(x, g[i], -p);
      v[i] = fmaf(p, s.q, fmaf(p, s.q1, e * s.q));
    }
  }
  if (code == 1) {
    const uint32_t keep = alpha == alpha ? 0xffffffffu : 0u;
    uint32_t b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = quant_bits(v[i], 1.0f);
#pragma unroll
    for (int i = 0; i < V / 4; ++i) w[i] = pack4(b[4 * i], b[4 * i + 1], b[4 * i + 2], b[4 * i + 3]) & keep;
  } else {
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
      const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], lo, true);
    }
  }
}
template <int V>
__device__ __forceinline__ void store_codes(uint8_t *to, int n, const uint32_t (&w)[V / 4]) {
  if (n >= V) {
    __builtin_memcpy(to, w, V);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) to[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// ---- the norm ---------------------------------------------------------------------------------------------------
// y and the codes of a row's columns from `off` on, those that cols holds.  h is used up.
template <class T, int V, int TPR, int NV>
__device__ __forceinline__ void write_norm(const NormRows &a, const Columns<V, TPR, NV> &cols, int off, int64_t r, bool live,
                                           float (&h)[NV * V], const float (&g)[NV * V], const float (&m)[NV], float A,
                                           float E, float rho) {
  if (a.y)
    cols.store((T *)a.y + r * a.ldy + off, live, a.past_out, [&](int j, float (&v)[V]) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = h[j * V + i] * g[j * V + i] * rho;
    });
  if (!a.code) return;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = off + cols.col(j), lanes = a.group / V;
    float B = A, F = E, rho_j = rho;
    if (a.alphas > 1) {
      B = lanes_join<Max>(m[j], lanes);
      if (B < kTiny) {   // the row's own maximum is not
        float t[1];
        rho_j = lift<V>(h + j * V, rho);
        B = lanes_join<Max>(vector_max<V, 1>(h + j * V, g + j * V, t), lanes);
      }
      F = lanes_join<Largest>(tail_of<V>(B, h + j * V, g + j * V), lanes);
    }
    const float alpha = B * rho_j;
    uint32_t w[V / 4];
    codes_of<V>(a.code, alpha, B, F, h + j * V, g + j * V, w);
    uint8_t *to = a.codes + r * a.ldcodes + c;
    if (live && cols.full(j)) __builtin_memcpy(to, w, V);
    if (live && cols.last && j == cols.jt) store_codes<V>(to, cols.tail, w);
    if (live && c < a.d && c % a.group == 0) a.alpha[r * a.alphas + c / a.group] = alpha;
  }
}

// A block takes every gridDim.x-th of its sets of rows; the next one's inputs are read before the present one is joined
// and written (loads issued ahead of the stores, so that waiting for them does not wait for the stores): 16384 x 8192
// bf16 182 -> 175 us, its gradient 125 -> 108 at 4096 columns.  What waits stays as it was stored, 16-bit values two to a
// register.
template <class T, int TPR, int NV, int BLOCK, int WAVES, bool PAST, bool ENDS>
__global__ __launch_bounds__(BLOCK, WAVES) void k_rms_norm(NormRows a) {
  constexpr int V = 16 / sizeof(T), RPB = BLOCK / TPR;
  __shared__ float2 lds[BLOCK / 64];
  const int lane = threadIdx.x % TPR, sub = row_of_block<TPR, BLOCK>();
  const float inv_d = 1.0f / (float)a.d;
  const Columns<V, TPR, NV> cols(a.d, lane);
  const int64_t step = (int64_t)gridDim.x * RPB;
  Raw<T, V> nx[NV], nres[NV];
  const auto fetch = [&](int64_t r) {
    cols.template load<PAST, ENDS>((const T *)a.x + r * a.ldx, RPB == 1 || r < a.rows, nx);
    if (a.res) {
      // one stream of reads from the memory at a time: 20000 x 5000 bf16 157 -> 150 us (x + one row for all 126, waiting 188)
      if (PAST && a.ldx && a.ldres) wait_loads();
      cols.template load<PAST, ENDS>((const T *)a.res + r * a.ldres, RPB == 1 || r < a.rows, nres);
    }
  };
  fetch((int64_t)blockIdx.x * RPB + sub);
  float g[NV * V];
  cols.template gain<T>(a.gain, a.gain_f32, g);
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += step) {
    const int64_t r = r0 + sub;
    const bool live = RPB == 1 || r < a.rows;
    float h[NV * V];
    float ss = 0, A = 0;
    if (ENDS) cols.settle(nx);
    if (ENDS && a.res) cols.settle(nres);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float (&v)[V] = (float (&)[V])h[j * V];
      unpack<T, V>(nx[j], v);
      if (a.res) {
        float w[V];
        unpack<T, V>(nres[j], w);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += w[i];
      }
    }
    if (r0 + step < a.rows) fetch(r + step);
    const auto store_h = [&] {
      if (a.h)
        cols.store((T *)a.h + r * a.ldh, live, a.past_out, [&](int j, float (&v)[V]) {
#pragma unroll
          for (int i = 0; i < V; ++i) v[i] = h[j * V + i];
        });
    };
    if (!ENDS) store_h();
#pragma unroll
    for (int i = 0; i < NV * V; ++i) ss = fmaf(h[i], h[i], ss);
    float m[NV];
    A = vector_max<V, NV>(h, g, m);
    row_join<Max, TPR>(ss, A, lds);
    if (ENDS) store_h();   // behind the join: h may lie on an input, whose row's last lane reads columns of its neighbour's
    float rho = near_rho(ss, inv_d, a.eps);
    if (!in_range(ss) || !(A >= kTiny && A <= 1e37f)) {
      float unit, none = 0;
      rho = far_rho<TPR>(ss, h, inv_d, a.eps, unit, lds);
      A = vector_max<V, NV>(h, g, m);
      row_join<Max, TPR>(none, A, lds);
      if (A < kTiny) {   // tiny gains
        rho = lift<NV * V>(h, rho);
        A = vector_max<V, NV>(h, g, m);
        row_join<Max, TPR>(none, A, lds);
      }
    }
    float E = kNoTail;
    if (a.code && a.alphas == 1) {
      float none = 0;
      E = tail_of<NV * V>(A, h, g);
      row_join<Largest, TPR>(none, E, lds);
    }
    write_norm<T, V, TPR, NV>(a, cols, 0, r, live, h, g, m, A, E, rho);
  }
}

// Rows too long for registers, a block of 1024 threads each, 16 values a thread at a time: the first pass reads the row
// and writes nothing, the second reads it again (from the caches) and writes; a thread reads and writes the same columns,
// so h and y may lie on the inputs here too.
constexpr int kWideThreads = 1024, kWideValues = 16, kWideStep = kWideThreads * kWideValues;
template <class T>
__device__ __forceinline__ const void *gain_at(const void *gain, bool f32, int off) {
  return !gain ? nullptr : f32 ? (const void *)((const float *)gain + off) : (const void *)((const T *)gain + off);
}

template <class T>
__global__ __launch_bounds__(kWideThreads) void k_rms_norm_wide(NormRows a) {
  constexpr int V = 16 / sizeof(T), NV = kWideValues / V, N = kWideValues;
  using Cols = Columns<V, kWideThreads, NV>;
  __shared__ float2 lds[kWideThreads / 64];
  const float inv_d = 1.0f / (float)a.d;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const auto read = [&](const Cols &cols, int off, float (&h)[N], float (&g)[N]) {
      Raw<T, V> x[NV], res[NV];
      cols.template load<false, false>((const T *)a.x + r * a.ldx + off, true, x);
      if (a.res) cols.template load<false, false>((const T *)a.res + r * a.ldres + off, true, res);
      cols.template gain<T>(gain_at<T>(a.gain, a.gain_f32, off), a.gain_f32, g);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float (&v)[V] = (float (&)[V])h[j * V];
        unpack<T, V>(x[j], v);
        if (a.res) {
          float w[V];
          unpack<T, V>(res[j], w);
#pragma unroll
          for (int i = 0; i < V; ++i) v[i] += w[i];
        }
      }
    };
    float ss, A, E;
    const auto sums = [&](float up, float more) {
      ss = A = 0;
      E = kNoTail;
      for (int off = 0; off < a.d; off += kWideStep) {
        float h[N], g[N];
        read(Cols(a.d - off, threadIdx.x), off, h, g);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          h[i] = h[i] * up * more;
          ss = fmaf(h[i], h[i], ss);
          const float p = fabsf(h[i]) * fabsf(g[i]), e = fmaf(fabsf(h[i]), fabsf(g[i]), -p), B = Max::join(A, p);
          E = B != A ? e : p == A ? fmaxf(E, e) : E;
          A = B;
        }
      }
      const float own = A;
      row_join<Max, kWideThreads>(ss, A, lds);
      if (a.code) {
        float none = 0;
        E = own == A ? E : kNoTail;
        row_join<Largest, kWideThreads>(none, E, lds);
      }
    };
    sums(1.0f, 1.0f);
    float rho = near_rho(ss, inv_d, a.eps), up = 1.0f, more = 1.0f;
    if (!in_range(ss) || !(A >= kTiny && A <= 1e37f)) {
      up = far_up(ss);
      sums(up, 1.0f);
      rho = far_rho_of(ss, up, inv_d, a.eps, more);
      sums(up, more);
      if (A < kTiny) {
        rho = lift<1>(&more, rho);
        sums(up, more);
      }
    }
    for (int off = 0; off < a.d; off += kWideStep) {
      const Cols cols(a.d - off, threadIdx.x);
      float h[N], g[N];
      read(cols, off, h, g);
      if (a.h)
        cols.store((T *)a.h + r * a.ldh + off, true, a.past_out, [&](int j, float (&v)[V]) {
#pragma unroll
          for (int i = 0; i < V; ++i) v[i] = h[j * V + i];
        });
#pragma unroll
      for (int i = 0; i < N; ++i) h[i] = h[i] * up * more;
      float m[NV];
      (void)vector_max<V, NV>(h, g, m);
      write_norm<T, V, kWideThreads, NV>(a, cols, off, r, true, h, g, m, A, E, rho);
    }
  }
}

// ---- its gradient ------------------------------------------------------------------------------------------------
// Block b sums dy xh over its rows per column and leaves the sums in part[b].
// AHEAD: the next rows are read ahead, as above.  Where 128 registers do not hold everything (16 values a thread, two to a
// register while they wait, and a join over a whole block), each thread keeps its gains in LDS: 9000 x 16384 fp16 167 us,
// with some registers spilled to memory instead 239.  Rows of one wavefront need none (60000 x 1000 fp16 66 us, with 76).
template <class T, int TPR, int NV, int BLOCK, int WAVES, bool AHEAD, bool PAST, bool ENDS>
__global__ __launch_bounds__(BLOCK, WAVES) void k_rms_norm_grad(NormGradRows a) {
  constexpr int V = 16 / sizeof(T), RPB = BLOCK / TPR, N = NV * V;
  __shared__ float2 lds[BLOCK / 64];
  const int lane = threadIdx.x % TPR, sub = row_of_block<TPR, BLOCK>();
  const float inv_d = 1.0f / (float)a.d;
  const Columns<V, TPR, NV> cols(a.d, lane);
  const int64_t step = (int64_t)gridDim.x * RPB;
  Raw<T, V> nh[NV], ndy[NV];
  const auto fetch = [&](int64_t r) {
    cols.template load<PAST, ENDS>((const T *)a.h + r * a.ldh, RPB == 1 || r < a.rows, nh);
    cols.template load<PAST, ENDS>((const T *)a.dy + r * a.lddy, RPB == 1 || r < a.rows, ndy);
  };
  if constexpr (AHEAD) fetch((int64_t)blockIdx.x * RPB + sub);
  constexpr bool GAIN_LDS = sizeof(T) == 2 && NV == 2 && TPR > 64;
  __shared__ float4 gain_lds[GAIN_LDS ? N / 4 * BLOCK : 1];
  float g[N], dg[N];
  cols.template gain<T>(a.gain, a.gain_f32, g);
  if constexpr (GAIN_LDS) {   // read again by the thread that wrote it only
#pragma unroll
    for (int i = 0; i < N / 4; ++i) gain_lds[i * BLOCK + threadIdx.x] = float4{g[4 * i], g[4 * i + 1], g[4 * i + 2], g[4 * i + 3]};
  }
  const auto gains = [&](int j, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
      if constexpr (GAIN_LDS) {
        const float4 q = gain_lds[(j * (V / 4) + i) * BLOCK + threadIdx.x];
        v[4 * i] = q.x, v[4 * i + 1] = q.y, v[4 * i + 2] = q.z, v[4 * i + 3] = q.w;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[4 * i + k] = g[j * V + 4 * i + k];
      }
    }
  };
#pragma unroll
  for (int i = 0; i < N; ++i) dg[i] = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += step) {
    const int64_t r = r0 + sub;
    const bool live = RPB == 1 || r < a.rows;
    float h[N], dy[N];
    Raw<T, V> res[NV];
    float ss = 0, dot = 0;
    if constexpr (!AHEAD) fetch(r);
    if (a.dres) cols.template load<PAST, ENDS>((const T *)a.dres + r * a.lddres, live, res);
    if (ENDS) cols.settle(nh);
    if (ENDS) cols.settle(ndy);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      unpack<T, V>(nh[j], (float (&)[V])h[j * V]);
      unpack<T, V>(ndy[j], (float (&)[V])dy[j * V]);
    }
    if (AHEAD && r0 + step < a.rows) fetch(r + step);
    const auto add_dot = [&] {
      dot = 0;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float w[V];
        gains(j, w);
#pragma unroll
        for (int i = 0; i < V; ++i) dot = fmaf(dy[j * V + i] * w[i], h[j * V + i], dot);
      }
    };
#pragma unroll
    for (int i = 0; i < N; ++i) ss = fmaf(h[i], h[i], ss);
    add_dot();
    if (ENDS && a.dres) cols.settle(res);   // before the join: behind it the others write dh, perhaps where dres lies
    row_join<Sum, TPR>(ss, dot, lds);
    float rho = near_rho(ss, inv_d, a.eps), unit = 1.0f;
    if (!in_range(ss) || !(fabsf(dot) <= 1e37f)) {
      float none = 0;
      rho = far_rho<TPR>(ss, h, inv_d, a.eps, unit, lds);
      add_dot();
      row_join<Sum, TPR>(dot, none, lds);
    }
    const float m = dot * rho * inv_d, rho1 = rho * unit;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      h[i] *= rho;
      if (live) dg[i] = fmaf(dy[i], h[i], dg[i]);
    }
    if (a.dh)
      cols.store((T *)a.dh + r * a.lddh, live, false, [&](int j, float (&o)[V]) {
        float w[V], gj[V];
        gains(j, gj);
        if (a.dres) unpack<T, V>(res[j], w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          o[i] = rho1 * fmaf(-m, h[j * V + i], dy[j * V + i] * gj[i]);
          if (a.dres) o[i] += w[i];
        }
      });
  }
  if (!a.part) return;
  if constexpr (RPB > 1) {   // the block's rows in a fixed order
    __shared__ float sums[BLOCK * N];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) sums[sub * TPR * N + (j * TPR + lane) * V + i] = dg[j * V + i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.d; c += BLOCK) {
      float s = sums[c];
      for (int k = 1; k < RPB; ++k) s += sums[k * TPR * N + c];
      a.part[(int64_t)blockIdx.x * a.d + c] = s;
    }
  } else {
    cols.store(a.part + (int64_t)blockIdx.x * a.d, true, false, [&](int j, float (&v)[V]) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = dg[j * V + i];
    });
  }
}

// Rows too long for registers: two passes as above.  The block's sums of dgain do not stay in registers either: its
// partial row in memory is added to, each column by one thread.
template <class T>
__global__ __launch_bounds__(kWideThreads) void k_rms_norm_grad_wide(NormGradRows a) {
  constexpr int V = 16 / sizeof(T), N = kWideValues, NV = N / V, STEP = kWideThreads * N;
  using Cols = Columns<V, kWideThreads, NV>;
  __shared__ float2 lds[kWideThreads / 64];
  const float inv_d = 1.0f / (float)a.d;
  float *const part = a.part + (int64_t)blockIdx.x * a.d;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const auto read = [&](const Cols &cols, int off, float (&h)[N], float (&dy)[N], float (&g)[N]) {
      Raw<T, V> x[NV], y[NV];
      cols.template load<false, false>((const T *)a.h + r * a.ldh + off, true, x);
      cols.template load<false, false>((const T *)a.dy + r * a.lddy + off, true, y);
      cols.template gain<T>(gain_at<T>(a.gain, a.gain_f32, off), a.gain_f32, g);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        unpack<T, V>(x[j], (float (&)[V])h[j * V]);
        unpack<T, V>(y[j], (float (&)[V])dy[j * V]);
      }
    };
    float ss, dot;
    const auto sums = [&](float up, float more) {
      ss = dot = 0;
      for (int off = 0; off < a.d; off += STEP) {
        float h[N], dy[N], g[N];
        read(Cols(a.d - off, threadIdx.x), off, h, dy, g);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          h[i] = h[i] * up * more;
          ss = fmaf(h[i], h[i], ss);
          dot = fmaf(dy[i] * g[i], h[i], dot);
        }
      }
      row_join<Sum, kWideThreads>(ss, dot, lds);
    };
    sums(1.0f, 1.0f);
    float rho = near_rho(ss, inv_d, a.eps), up = 1.0f, more = 1.0f;
    if (!in_range(ss) || !(fabsf(dot) <= 1e37f)) {
      up = far_up(ss);
      sums(up, 1.0f);
      rho = far_rho_of(ss, up, inv_d, a.eps, more);
      sums(up, more);
    }
    const float m = dot * rho * inv_d, rho1 = rho * (up * more);
    for (int off = 0; off < a.d; off += STEP) {
      const Cols cols(a.d - off, threadIdx.x);
      float h[N], dy[N], g[N];
      Raw<T, V> res[NV];
      if (a.dres) cols.template load<false, false>((const T *)a.dres + r * a.lddres + off, true, res);
      read(cols, off, h, dy, g);
#pragma unroll
      for (int i = 0; i < N; ++i) h[i] = h[i] * up * more * rho;
      if (a.dh)
        cols.store((T *)a.dh + r * a.lddh + off, true, false, [&](int j, float (&o)[V]) {
          float w[V];
          if (a.dres) unpack<T, V>(res[j], w);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            o[i] = rho1 * fmaf(-m, h[j * V + i], dy[j * V + i] * g[j * V + i]);
            if (a.dres) o[i] += w[i];
          }
        });
      if (a.part) {
        Raw<float, V> sum[NV];
        if (r != blockIdx.x) {
          cols.template load<false, false>(part + off, true, sum);
        } else {
#pragma unroll
          for (int j = 0; j < NV; ++j) sum[j] = Raw<float, V>{};
        }
        cols.store(part + off, true, false, [&](int j, float (&o)[V]) {
          unpack<float, V>(sum[j], o);
#pragma unroll
          for (int i = 0; i < V; ++i) o[i] = fmaf(dy[j * V + i], h[j * V + i], o[i]);
        });
      }
    }
  }
}

// dgain[c] = the sum of `rows` partial rows: 16 columns a block, 64 threads a column, thread k the rows k, k + 64, ...
__global__ __launch_bounds__(1024) void k_rms_norm_dgain(const float *part, int rows, int d, float *dgain) {
  __shared__ float lds[1024];
  const int c = blockIdx.x * 16 + threadIdx.x % 16;
  float s = 0;
  for (int r = threadIdx.x / 16; r < rows; r += 64 * 8) {   // eight loads in flight
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c < d && r + 64 * j < rows ? part[(int64_t)(r + 64 * j) * d + c] : 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s += v[j];
  }
  lds[threadIdx.x] = s;
  for (int half = 512; half >= 16; half /= 2) {
    __syncthreads();
    if (threadIdx.x < half) lds[threadIdx.x] += lds[threadIdx.x + half];
  }
  if (threadIdx.x < 16 && c < d) dgain[c] = lds[threadIdx.x];
}

// ---- launches ----------------------------------------------------------------------------------------------------
// f.run<TPR, NV, BLOCK>() for the narrowest shape that holds d values of V a vector, f.wide() past the widest.  Eight
// values a thread where a row fits a wavefront or less, so two vectors in fp32 (one: 49152 x 128 14.8 -> 14.3 us with two)
// and one in 16 bits (with two the gradient of 100000 x 200 26 -> 37 us, of 100000 x 512 55 -> 77).  Long rows have two
// vectors a thread in the norm (with one 16384 x 8192 bf16 to codes 173 -> 221 us, 2000 x 8192 23 -> 25) and one in the
// gradient (F::kThin), which holds more of each.  That pays for few rows and for widths that fill their threads: with two
// 777 x 5003 fp16 18.4 us, with one 15.9, 2000 x 8192 bf16 25.9 and 23.4, 20000 x 8192 193 and 177, 4096 x 2048 fp32 22.0
// and 20.7, 16384 x 4096 bf16 73.9 and 69.2; many rows a little wider than a power of two lose: 20000 x 5003 bf16 136 and
// 147, 20000 x 2100 57 and 67.
template <int V, class F>
hipError_t by_width(int d, const F &f) {
  const int n = (d + V - 1) / V;   // vectors a row
  if (n <= 8) return f.template run<8, 1, 256>();
  if constexpr (V == 4) {
    if (n <= 16) return f.template run<8, 2, 256>();
    if (n <= 32) return f.template run<16, 2, 256>();
    if (n <= 64) return f.template run<32, 2, 256>();
  } else {
    if (n <= 16) return f.template run<16, 1, 256>();
    if (n <= 32) return f.template run<32, 1, 256>();
    if (n <= 64) return f.template run<64, 1, 256>();
  }
  if (n <= 128) return f.template run<64, 2, 256>();
  if (n <= 256) return f.template run<256, 1, 256>();
  if constexpr (F::kThin) {
    if (n <= 512) return f.template run<512, 1, 512>();
    if (n <= 1024) return f.template run<1024, 1, 1024>();
  } else {
    if (n <= 512) return f.template run<256, 2, 256>();
    if (n <= 1024) return f.template run<512, 2, 512>();
  }
  if (n <= 2048) return f.template run<1024, 2, 1024>();
  if constexpr (V == 4) {
    if (n <= 4096) return f.template run<1024, 4, 1024>();
  }
  return f.wide();
}
// Blocks for `sets` sets of rows, at most `most`, each with as many sets as any other but the last.
unsigned even_grid(int64_t sets, int64_t most) {
  const int64_t rounds = (sets + most - 1) / most;
  return rounds > 1 ? (unsigned)((sets + rounds - 1) / rounds) : (unsigned)sets;
}

template <class T>
struct NormLaunch {
  static constexpr bool kThin = false;
  const NormRows &a;
  int cu_count;
  hipStream_t s;
  template <int TPR, int NV, int BLOCK>
  hipError_t run() const {
    // Wavefronts a SIMD, as many as need no scratch; a block of 1024 brings four at a time (six: 10000 x 5000 fp32 64 -> 92 us).
    constexpr int V = 16 / sizeof(T), W = NV * V <= 4 ? 8 : NV * V <= 8 && BLOCK < 1024 ? 6 : 4;
    const int64_t blocks = (a.rows + BLOCK / TPR - 1) / (BLOCK / TPR), most = (int64_t)cu_count * (W * 256 / BLOCK);
    constexpr bool ENDS = !(V == 4 && NV == 4);   // no registers left for it there
    const unsigned grid = even_grid(blocks, most);
    if constexpr (TPR == 8 && NV == 1) {
      if (a.d < V) {
        k_rms_norm<T, TPR, NV, BLOCK, W, false, false><<<grid, BLOCK, 0, s>>>(a);
        return hipGetLastError();
      }
    }
    if (a.past_in) k_rms_norm<T, TPR, NV, BLOCK, W, true, ENDS><<<grid, BLOCK, 0, s>>>(a);
    else k_rms_norm<T, TPR, NV, BLOCK, W, false, ENDS><<<grid, BLOCK, 0, s>>>(a);
    return hipGetLastError();
  }
  hipError_t wide() const {
    k_rms_norm_wide<T><<<even_grid(a.rows, cu_count), kWideThreads, 0, s>>>(a);
    return hipGetLastError();
  }
};

constexpr int kPartRows = 1024;   // blocks of the gradient, so rows of its partial sums, at most
template <class T>
struct NormGradLaunch {
  static constexpr bool kThin = true;
  const NormGradRows &a;
  int cu_count;
  hipStream_t s;
  template <int TPR, int NV, int BLOCK>
  hipError_t run() const {
    // Wavefronts a SIMD; with two vectors in five 400000 x 128 fp32 takes 106 us, not 100.  Blocks of 512 and 1024 threads bring
    // two and four at a time, so of five they get four.
    constexpr int V = 16 / sizeof(T), W = NV == 1 ? 5 : 4;
    constexpr bool AHEAD = !(V == 4 && NV == 4);   // fp32 does not shrink while it waits: no registers left
    const int64_t blocks = (a.rows + BLOCK / TPR - 1) / (BLOCK / TPR);
    int64_t most = (int64_t)cu_count * (W * 256 / BLOCK);
    if (most > kPartRows) most = kPartRows;
    // Each block leaves a row of partial sums, so long rows go to fewer blocks, of four rows if that leaves two for each
    // CU (3001 x 2048 fp16 16.1 -> 15.1 us, 700 x 900 fp32 8.6 -> 7.5); with many rows all the blocks hide more
    // (20000 x 2048 fp16 48 us, with half of them 53).
    if (TPR >= 256 && most > blocks / 4) most = std::max(blocks / 4, std::min<int64_t>(most, 2 * cu_count));
    const unsigned grid = even_grid(blocks, most);
    if constexpr (TPR == 8 && NV == 1) {
      if (grid && a.d < V) {
        k_rms_norm_grad<T, TPR, NV, BLOCK, W, AHEAD, false, false><<<grid, BLOCK, 0, s>>>(a);
        return dgain(grid);
      }
    }
    if (grid && a.past_in) k_rms_norm_grad<T, TPR, NV, BLOCK, W, AHEAD, true, AHEAD><<<grid, BLOCK, 0, s>>>(a);
    else if (grid) k_rms_norm_grad<T, TPR, NV, BLOCK, W, AHEAD, false, AHEAD><<<grid, BLOCK, 0, s>>>(a);
    return dgain(grid);
  }
  hipError_t wide() const {
    const unsigned grid = even_grid(a.rows, cu_count < kPartRows ? cu_count : kPartRows);
    if (grid) k_rms_norm_grad_wide<T><<<grid, kWideThreads, 0, s>>>(a);
    return dgain(grid);
  }
  hipError_t dgain(unsigned rows) const {
    if (a.part) k_rms_norm_dgain<<<(a.d + 15) / 16, 1024, 0, s>>>(a.part, (int)rows, a.d, a.dgain);
    return hipGetLastError();
  }
};

}  // namespace

hipError_t launch_rms_norm(int type, const NormRows &a, int cu_count, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  if (type == 0) return by_width<4>(a.d, NormLaunch<float>{a, cu_count, s});
  if (type == 1) return by_width<8>(a.d, NormLaunch<bf16_t>{a, cu_count, s});
  return by_width<8>(a.d, NormLaunch<f16_t>{a, cu_count, s});
}

int64_t norm_grad_part_rows(int64_t rows, int d) { return rows < kPartRows ? rows : kPartRows; }

hipError_t launch_rms_norm_grad(int type, const NormGradRows &a, int cu_count, hipStream_t s) {
  if (type == 0) return by_width<4>(a.d, NormGradLaunch<float>{a, cu_count, s});
  if (type == 1) return by_width<8>(a.d, NormGradLaunch<bf16_t>{a, cu_count, s});
  return by_width<8>(a.d, NormGradLaunch<f16_t>{a, cu_count, s});
}

}  // namespace aecct
