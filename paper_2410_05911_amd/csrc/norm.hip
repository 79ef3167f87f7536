// Root-mean-square norm of rows with the residual's addition and Eq. 2 codes, and its gradient.
//
// Both are bound by device memory: a row is read once into registers, reduced there, and written.  A row is held by
// TPR threads, NV vectors of 16 bytes a thread: 8 to 64 lanes of a wavefront for short rows (several rows a
// wavefront, no barrier), a block of 256 or 1024 threads for long ones.
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
// Two values of a row joined over its TPR threads, the second by Op2.
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

// A row's rho = 1 / sqrt(mean(h^2) + eps) where the plain fp32 sum of squares is out of range: h is scaled by a power of
// two first, `unit`, and by a second that takes rho into [1, 2), so that products with h stay in range; h rho is
// unchanged and the rho of the row as it was is rho unit.
__device__ __forceinline__ float far_up(float ss) { return in_range(ss) ? 1.0f : ss < 1.0f ? 0x1p100f : 0x1p-100f; }
__device__ __forceinline__ float far_rho_of(float ss, float up, int d, float eps, float &more) {
  const float rho = (float)(1.0 / sqrt((double)ss / d + (double)eps * up * up));
  const int e = rho > 0 && rho < __builtin_inff() ? __builtin_amdgcn_frexp_expf(rho) - 1 : 0;
  more = ldexpf(1.0f, e);
  return ldexpf(rho, -e);
}
template <int TPR, int N>
__device__ __forceinline__ float far_rho(float ss, float (&h)[N], int d, float eps, float &unit, float2 *lds) {
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
  const float rho = far_rho_of(ss, up, d, eps, more);
#pragma unroll
  for (int i = 0; i < N; ++i) h[i] *= more;
  unit = up * more;
  return rho;
}

template <class T, int V>
__device__ __forceinline__ void load_gain(const void *gain, bool f32, int c, int n, float (&g)[V]) {
  if (!gain) {
#pragma unroll
    for (int i = 0; i < V; ++i) g[i] = 1.0f;
  } else if (f32) {
    load_part<float, V>((const float *)gain + c, n, g);
  } else {
    load_part<T, V>((const T *)gain + c, n, g);
  }
}

// ---- codes -----------------------------------------------------------------------------------------------------
// code = round(p Q / A) with p = h gain and A = max |p|: rho is a factor of both y and alpha and drops out.  The quotient
// is taken as (p + e)(q + q1), e the rounding error of p, q a near quotient Q / A and q1 its remainder's: a code then
// differs from the exact one only where the quotient is within about 2^-24 of a tie.  `up` keeps A and q normal numbers.
struct CodeScale {
  float up, q, q1;
};
__device__ __forceinline__ CodeScale code_scale(float A, float most) {
  CodeScale s;
  s.up = A < 0x1p-60f ? 0x1p60f : A > 0x1p60f ? 0x1p-60f : 1.0f;
  const float b = A * s.up, r = __builtin_amdgcn_rcpf(b);
  s.q = A == 0.0f ? 0.0f : most * r;
  s.q1 = A == 0.0f || !(b <= 3e38f) ? 0.0f : fmaf(-s.q, b, most) * r;
  return s;
}
template <int V>
__device__ __forceinline__ void store_codes(uint8_t *to, int n, int code, float A, const float *h, const float *g) {
  const CodeScale s = code_scale(A, code == 1 ? 127.0f : 448.0f);
  uint32_t w[V / 4];
  float v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float x = h[i] * s.up, p = x * g[i], e = fmaf(x, g[i], -p);
    v[i] = fmaf(p, s.q, fmaf(p, s.q1, e * s.q));
  }
  if (code == 1) {
    const uint32_t keep = A == A ? 0xffffffffu : 0u;
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
  if (n >= V) {
    __builtin_memcpy(to, w, V);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) to[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// ---- the norm ---------------------------------------------------------------------------------------------------
template <class T, int TPR, int NV, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_rms_norm(NormRows a) {
  constexpr int V = 16 / sizeof(T), RPB = BLOCK / TPR;
  __shared__ float2 lds[BLOCK / 64];
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const float inv_d = 1.0f / (float)a.d;
  float g[NV * V];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * TPR + lane) * V;
    load_gain<T, V>(a.gain, a.gain_f32, c, a.d - c, (float (&)[V])g[j * V]);
  }
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB) {
    const int64_t r = r0 + sub;
    const bool live = r < a.rows;
    float h[NV * V];
    float ss = 0, A = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * TPR + lane) * V, n = live ? a.d - c : 0;
      float (&v)[V] = (float (&)[V])h[j * V];
      load_part<T, V>((const T *)a.x + r * a.ldx + c, n, v);
      if (a.res) {
        float w[V];
        load_part<T, V>((const T *)a.res + r * a.ldres + c, n, w);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += w[i];
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * TPR + lane) * V, n = live ? a.d - c : 0;
      float (&v)[V] = (float (&)[V])h[j * V];
      if (a.h) store_part<T, V>((T *)a.h + r * a.ldh + c, n, v);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        ss = fmaf(v[i], v[i], ss);
        A = Max::join(A, fabsf(v[i] * g[j * V + i]));
      }
    }
    row_join<Max, TPR>(ss, A, lds);
    float rho = near_rho(ss, inv_d, a.eps);
    if (!in_range(ss) || !(A >= 0x1p-60f && A <= 1e37f)) {
      float unit, none = 0;
      rho = far_rho<TPR>(ss, h, a.d, a.eps, unit, lds);
      A = 0;
#pragma unroll
      for (int i = 0; i < NV * V; ++i) A = Max::join(A, fabsf(h[i] * g[i]));
      row_join<Max, TPR>(none, A, lds);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * TPR + lane) * V, n = live ? a.d - c : 0;
      if (a.y) {
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = h[j * V + i] * g[j * V + i] * rho;
        store_part<T, V>((T *)a.y + r * a.ldy + c, n, y);
      }
      if (a.code) {
        float B = A;
        if (a.alphas > 1) {
          B = 0;
#pragma unroll
          for (int i = 0; i < V; ++i) B = Max::join(B, fabsf(h[j * V + i] * g[j * V + i]));
          B = lanes_join<Max>(B, a.group / V);
        }
        store_codes<V>(a.codes + r * a.ldcodes + c, n, a.code, B, h + j * V, g + j * V);
        if (n > 0 && c % a.group == 0) a.alpha[r * a.alphas + c / a.group] = B * rho;
      }
    }
  }
}

// Rows too long for registers, a block of 1024 threads each: the first pass reads the row and writes nothing, the
// second reads it again (from the caches) and writes; a thread reads and writes the same columns, so h and y may lie on
// the inputs here too.
constexpr int kWideThreads = 1024;
template <class T>
__global__ __launch_bounds__(kWideThreads) void k_rms_norm_wide(NormRows a) {
  constexpr int V = 16 / sizeof(T), STEP = kWideThreads * V;
  __shared__ float2 lds[kWideThreads / 64];
  const int c0 = threadIdx.x * V;
  const float inv_d = 1.0f / (float)a.d;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *x = (const T *)a.x + r * a.ldx, *res = (const T *)a.res + r * a.ldres;
    const auto load_h = [&](int c, float (&h)[V]) {
      load_part<T, V>(x + c, a.d - c, h);
      if (a.res) {
        float w[V];
        load_part<T, V>(res + c, a.d - c, w);
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] += w[i];
      }
    };
    float ss, A;
    const auto sums = [&](float up, float more) {
      ss = A = 0;
      for (int c = c0; c < a.d; c += STEP) {
        float h[V], g[V];
        load_h(c, h);
        load_gain<T, V>(a.gain, a.gain_f32, c, a.d - c, g);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          h[i] = h[i] * up * more;
          ss = fmaf(h[i], h[i], ss);
          A = Max::join(A, fabsf(h[i] * g[i]));
        }
      }
      row_join<Max, kWideThreads>(ss, A, lds);
    };
    sums(1.0f, 1.0f);
    float rho = near_rho(ss, inv_d, a.eps), up = 1.0f, more = 1.0f;
    if (!in_range(ss) || !(A >= 0x1p-60f && A <= 1e37f)) {
      up = far_up(ss);
      sums(up, 1.0f);
      rho = far_rho_of(ss, up, a.d, a.eps, more);
      sums(up, more);
    }
    // every thread of a wavefront takes part in a group's maximum: columns past the row are zeros
    for (int c = c0; c - c0 < a.d; c += STEP) {
      const int n = a.d - c;
      float h[V], g[V];
      load_gain<T, V>(a.gain, a.gain_f32, c, n, g);
      load_h(c, h);
      if (a.h) store_part<T, V>((T *)a.h + r * a.ldh + c, n, h);
#pragma unroll
      for (int i = 0; i < V; ++i) h[i] = h[i] * up * more;
      if (a.y) {
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = h[i] * g[i] * rho;
        store_part<T, V>((T *)a.y + r * a.ldy + c, n, y);
      }
      if (a.code) {
        float B = A;
        if (a.alphas > 1) {
          B = 0;
#pragma unroll
          for (int i = 0; i < V; ++i) B = Max::join(B, fabsf(h[i] * g[i]));
          B = lanes_join<Max>(B, a.group / V);
        }
        store_codes<V>(a.codes + r * a.ldcodes + c, n, a.code, B, h, g);
        if (n > 0 && c % a.group == 0) a.alpha[r * a.alphas + c / a.group] = B * rho;
      }
    }
  }
}

// ---- its gradient ------------------------------------------------------------------------------------------------
// Block b sums dy xh over its rows per column and leaves the sums in part[b].
template <class T, int TPR, int NV, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_rms_norm_grad(NormGradRows a) {
  constexpr int V = 16 / sizeof(T), RPB = BLOCK / TPR, N = NV * V;
  __shared__ float2 lds[BLOCK / 64];
  const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const float inv_d = 1.0f / (float)a.d;
  float g[N], dg[N];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (j * TPR + lane) * V;
    load_gain<T, V>(a.gain, a.gain_f32, c, a.d - c, (float (&)[V])g[j * V]);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) dg[i] = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB) {
    const int64_t r = r0 + sub;
    const bool live = r < a.rows;
    float h[N], dy[N];
    float ss = 0, dot = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * TPR + lane) * V, n = live ? a.d - c : 0;
      load_part<T, V>((const T *)a.h + r * a.ldh + c, n, (float (&)[V])h[j * V]);
      load_part<T, V>((const T *)a.dy + r * a.lddy + c, n, (float (&)[V])dy[j * V]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      ss = fmaf(h[i], h[i], ss);
      dot = fmaf(dy[i] * g[i], h[i], dot);
    }
    row_join<Sum, TPR>(ss, dot, lds);
    float rho = near_rho(ss, inv_d, a.eps), unit = 1.0f;
    if (!in_range(ss) || !(fabsf(dot) <= 1e37f)) {
      float none = 0;
      rho = far_rho<TPR>(ss, h, a.d, a.eps, unit, lds);
      dot = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) dot = fmaf(dy[i] * g[i], h[i], dot);
      row_join<Sum, TPR>(dot, none, lds);
    }
    const float m = dot * rho * inv_d, rho1 = rho * unit;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * TPR + lane) * V, n = live ? a.d - c : 0;
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int k = j * V + i;
        const float xh = h[k] * rho;
        if (live) dg[k] = fmaf(dy[k], xh, dg[k]);
        o[i] = rho1 * fmaf(-m, xh, dy[k] * g[k]);
      }
      if (a.dh) {
        if (a.dres) {
          float w[V];
          load_part<T, V>((const T *)a.dres + r * a.lddres + c, n, w);
#pragma unroll
          for (int i = 0; i < V; ++i) o[i] += w[i];
        }
        store_part<T, V>((T *)a.dh + r * a.lddh + c, n, o);
      }
    }
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
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * TPR + lane) * V;
      store_part<float, V>(a.part + (int64_t)blockIdx.x * a.d + c, a.d - c, (float (&)[V])dg[j * V]);
    }
  }
}

// Rows too long for registers: two passes as above; the block's partial row is added to in memory, each column by one
// thread.
template <class T>
__global__ __launch_bounds__(kWideThreads) void k_rms_norm_grad_wide(NormGradRows a) {
  constexpr int V = 16 / sizeof(T), STEP = kWideThreads * V;
  __shared__ float2 lds[kWideThreads / 64];
  const int c0 = threadIdx.x * V;
  const float inv_d = 1.0f / (float)a.d;
  float *part = a.part + (int64_t)blockIdx.x * a.d;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *ph = (const T *)a.h + r * a.ldh, *pdy = (const T *)a.dy + r * a.lddy;
    float ss, dot;
    const auto sums = [&](float up, float more) {
      ss = dot = 0;
      for (int c = c0; c < a.d; c += STEP) {
        float h[V], dy[V], g[V];
        load_part<T, V>(ph + c, a.d - c, h);
        load_part<T, V>(pdy + c, a.d - c, dy);
        load_gain<T, V>(a.gain, a.gain_f32, c, a.d - c, g);
#pragma unroll
        for (int i = 0; i < V; ++i) {
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
      rho = far_rho_of(ss, up, a.d, a.eps, more);
      sums(up, more);
    }
    const float m = dot * rho * inv_d, rho1 = rho * (up * more);
    for (int c = c0; c < a.d; c += STEP) {
      const int n = a.d - c;
      float h[V], dy[V], g[V], o[V];
      load_part<T, V>(ph + c, n, h);
      load_part<T, V>(pdy + c, n, dy);
      load_gain<T, V>(a.gain, a.gain_f32, c, n, g);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        h[i] = h[i] * up * more * rho;
        o[i] = rho1 * fmaf(-m, h[i], dy[i] * g[i]);
      }
      if (a.dh) {
        if (a.dres) {
          float w[V];
          load_part<T, V>((const T *)a.dres + r * a.lddres + c, n, w);
#pragma unroll
          for (int i = 0; i < V; ++i) o[i] += w[i];
        }
        store_part<T, V>((T *)a.dh + r * a.lddh + c, n, o);
      }
      if (a.part) {
        float s[V];
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = 0;
        if (r != blockIdx.x) load_part<float, V>(part + c, n, s);
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = fmaf(dy[i], h[i], s[i]);
        store_part<float, V>(part + c, n, s);
      }
    }
  }
}

// dgain[c] = the sum of `rows` partial rows: 16 columns a block, 16 threads a column, thread k the rows k, k + 16, ...
__global__ __launch_bounds__(256) void k_rms_norm_dgain(const float *part, int rows, int d, float *dgain) {
  __shared__ float lds[256];
  const int c = blockIdx.x * 16 + threadIdx.x % 16;
  float s = 0;
  if (c < d)
    for (int r = threadIdx.x / 16; r < rows; r += 16) s += part[(int64_t)r * d + c];
  lds[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x < 16 && c < d) {
    for (int k = 1; k < 16; ++k) s += lds[16 * k + threadIdx.x];
    dgain[c] = s;
  }
}

// ---- launches ----------------------------------------------------------------------------------------------------
// f.run<TPR, NV, BLOCK>() for the narrowest shape that holds d values of V a vector, f.wide() past the widest.
template <int V, class F>
hipError_t by_width(int d, const F &f) {
  const int n = (d + V - 1) / V;   // vectors a row
  if (n <= 8) return f.template run<8, 1, 256>();
  if (n <= 16) return f.template run<16, 1, 256>();
  if (n <= 32) return f.template run<32, 1, 256>();
  if (n <= 64) return f.template run<64, 1, 256>();
  if (n <= 128) return f.template run<64, 2, 256>();
  if (n <= 256) return f.template run<256, 1, 256>();
  if (n <= 512) return f.template run<256, 2, 256>();
  if (n <= 1024) return f.template run<256, 4, 256>();
  if (n <= 2048) return f.template run<1024, 2, 1024>();
  if constexpr (V == 4) {
    if (n <= 4096) return f.template run<1024, 4, 1024>();
  }
  return f.wide();
}

template <class T>
struct NormLaunch {
  const NormRows &a;
  int cu_count;
  hipStream_t s;
  template <int TPR, int NV, int BLOCK>
  hipError_t run() const {
    const int64_t blocks = (a.rows + BLOCK / TPR - 1) / (BLOCK / TPR), most = (int64_t)cu_count * (2048 / BLOCK);
    k_rms_norm<T, TPR, NV, BLOCK><<<(unsigned)(blocks < most ? blocks : most), BLOCK, 0, s>>>(a);
    return hipGetLastError();
  }
  hipError_t wide() const {
    const int64_t most = 2 * (int64_t)cu_count;
    k_rms_norm_wide<T><<<(unsigned)(a.rows < most ? a.rows : most), kWideThreads, 0, s>>>(a);
    return hipGetLastError();
  }
};

constexpr int kPartRows = 1024;
template <class T>
struct NormGradLaunch {
  const NormGradRows &a;
  int cu_count;
  hipStream_t s;
  template <int TPR, int NV, int BLOCK>
  hipError_t run() const {
    const int64_t blocks = (a.rows + BLOCK / TPR - 1) / (BLOCK / TPR);
    int64_t most = (int64_t)cu_count * (1024 / BLOCK);
    if (most > kPartRows) most = kPartRows;
    const unsigned grid = (unsigned)(blocks < most ? blocks : most);
    if (grid) k_rms_norm_grad<T, TPR, NV, BLOCK><<<grid, BLOCK, 0, s>>>(a);
    return dgain(grid);
  }
  hipError_t wide() const {
    const int64_t most = cu_count < kPartRows ? cu_count : kPartRows;
    const unsigned grid = (unsigned)(a.rows < most ? a.rows : most);
    if (grid) k_rms_norm_grad_wide<T><<<grid, kWideThreads, 0, s>>>(a);
    return dgain(grid);
  }
  hipError_t dgain(unsigned rows) const {
    if (a.part) k_rms_norm_dgain<<<(a.d + 15) / 16, 256, 0, s>>>(a.part, (int)rows, a.d, a.dgain);
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
