// Norm of many tensors, clipping by it, and the Adam update.
//
// All are bound by device memory; a list is worked on as one range of units, whatever its tensors' sizes.  The norm
// needs every value before any is scaled, so clipping and the update are two launches: sums of squares, one double a
// block, then a pass in which every block adds those sums up in the same order (2048 doubles, eight loads in flight)
// while its first unit's values are on their way.  Squares and sums are fp64, so that no finite gradient is out of
// range.  Measured on an MI355X (a copy of 1 GB 5.1 TB/s, reads alone 6.4): the norm of 250e6 fp32 values 155 us
// (6.4 TB/s), the update of 120e6 parameters from bf16 gradients with clipping and bf16 copies 45 + 605 us (5.5 TB/s in
// the second), of the 2.1e6 parameters of LDPC(256,128) 5 + 12 us.
#include "row_io.h"
#include "update.h"

namespace aecct {
namespace {

constexpr int kThreads = 256;
// The last pass over a list reads and writes what nothing here uses again: marked so, it leaves the values that it
// has still to read in the cache (clipping 250e6 fp32 values 562 -> 504 us, the update of 120e6 with clipping
// 790 -> 710; of 10e6 66 -> 59).  Clipping 5e6 to 15e6 values, which fit the cache, would take 3 to 4 us of 20 to 36 less
// without, clipping 2e6 1 us more.  The sum that precedes such a pass is not marked (with it 15 us less for 1 GB, lost again after it).
constexpr bool kLast = true;

__device__ __forceinline__ double block_sum(double v, double *lds) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
  __syncthreads();
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int w = 1; w < kThreads / 64; ++w) v += lds[w];
  return v;
}

// The range of unit u, from that of a later unit.  Units are taken from the last to the first: the pass that follows a sum
// of squares meets the values that the sum read last first, while they are still in the cache.
template <int N>
__device__ __forceinline__ int range_of(const Units<N> &t, int u, int k) {
  if (u >= t.unit0[k]) return k;
  int lo = 0, hi = k - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (t.unit0[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
template <int N>
__device__ __forceinline__ int range_after(const Units<N> &t, int u, int k) {   // from that of an earlier unit
  if (u < t.unit0[k + 1]) return k;
  int lo = k + 1, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (t.unit0[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Four values of any type; n of them are there.
__device__ __forceinline__ void load4(const void *p, int type, int64_t i, int64_t n, float (&f)[4]) {
  const int k = n >= 4 ? 4 : (int)n;
  if (type == 0) load_part<float, 4, kLast>((const float *)p + i, k, f);
  else if (type == 1) load_part<bf16_t, 4, kLast>((const bf16_t *)p + i, k, f);
  else load_part<f16_t, 4, kLast>((const f16_t *)p + i, k, f);
}
__device__ __forceinline__ void store4(void *p, int type, int64_t i, int64_t n, const float (&f)[4]) {
  const int k = n >= 4 ? 4 : (int)n;
  if (type == 0) store_part<float, 4, kLast>((float *)p + i, k, f);
  else if (type == 1) store_part<bf16_t, 4, kLast>((bf16_t *)p + i, k, f);
  else store_part<f16_t, 4, kLast>((f16_t *)p + i, k, f);
}

// The unit of a thread of the sums: four vectors of 16 bytes, read a unit ahead of their use (eight, not read ahead: 191 us
// for 250e6 fp32 values where these take 155 to 167).
struct SumUnit {
  Raw<float, 4> w[4];
  template <class T, bool NT>
  __device__ __forceinline__ void load(const T *g, int64_t n) {
    constexpr int V = 16 / sizeof(T);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = (j * kThreads + (int)threadIdx.x) * V;
      Raw<T, V> r;
      if (i + V <= n) load_raw<T, V, NT>(g + i, r);
      else load_raw_part<T, V>(g + i, (int)(n - i), r);
      __builtin_memcpy(w[j].w, r.w, 16);
    }
  }
  template <class T>
  __device__ __forceinline__ void add_squares(double &s, double &q) const {
    constexpr int V = 16 / sizeof(T);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      Raw<T, V> r;
      __builtin_memcpy(r.w, w[j].w, 16);
      float f[V];
      unpack<T, V>(r, f);
#pragma unroll
      for (int i = 0; i < V; i += 2) {
        s = fma((double)f[i], (double)f[i], s);
        q = fma((double)f[i + 1], (double)f[i + 1], q);
      }
    }
  }
};

__device__ __forceinline__ void set_now(AdamNow *now, const int64_t *step, const AdamScalars &o) {
  const int64_t t = *step + 1;
  now->step = t;
  now->grow1 = (float)(1 / (1 - pow(o.beta1, (double)t)));
  now->root2 = (float)(1 / sqrt(1 - pow(o.beta2, (double)t)));
}
__global__ void k_now(const int64_t *step, AdamNow *now, AdamScalars o) { set_now(now, step, o); }

template <int N, bool NT>   // NT: no pass over the values follows
__global__ __launch_bounds__(kThreads) void k_sum_squares(SumTable<N> t, double *part, const int64_t *step, AdamNow *now,
                                                          AdamScalars o) {
  __shared__ double lds[kThreads / 64];
  if (now && blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) set_now(now, step, o);
  double s = 0, q = 0;
  SumUnit x;
  int k = 0;
  const auto fetch = [&](int u) {
    k = range_after(t, u, k);
    const int type = t.type[k];
    const int64_t i0 = (int64_t)(u - t.unit0[k]) * t.unit_of(type), n = t.count[k] - i0;
    if (type == 0) x.load<float, NT>((const float *)t.g[k] + i0, n);
    else x.load<bf16_t, NT>((const bf16_t *)t.g[k] + i0, n);
    return type;
  };
  const int units = t.unit0[t.n];
  int u = blockIdx.x, type = 0;
  if (u < units) type = fetch(u);
  while (u < units) {
    const SumUnit y = x;
    const int ty = type;
    u += gridDim.x;
    if (u < units) type = fetch(u);
    if (ty == 0) y.add_squares<float>(s, q);
    else if (ty == 1) y.add_squares<bf16_t>(s, q);
    else y.add_squares<f16_t>(s, q);
  }
  s = block_sum(s + q, lds);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The norm from the blocks' sums; every block that asks gets the same bits.
__device__ __forceinline__ double norm_of(const double *part, int parts, double *lds) {
  double s = 0;
  for (int i = threadIdx.x; i < parts; i += 8 * kThreads) {   // eight loads in flight: this is all latency
    double v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = i + j * kThreads < parts ? part[i + j * kThreads] : 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) s += v[j];
  }
  return sqrt(block_sum(s, lds));
}

__global__ __launch_bounds__(kThreads) void k_norm(const double *part, int parts, float *norm) {
  __shared__ double lds[kThreads / 64];
  const double n = norm_of(part, parts, lds);
  if (threadIdx.x == 0) *norm = (float)n;
}

// min(1, max_norm / norm), and 1 for a norm that is not finite.  A factor near or below the end of fp32's normal range is
// taken in two, the first a power of two, the second normal for every factor above 2^-275: no value is left of the largest
// gradient below that.
struct Factor {
  float up = 1.0f, f = 1.0f;
  __device__ __forceinline__ float of(float g) const { return g * up * f; }
};
__device__ __forceinline__ Factor clip_factor(double norm, double max_norm) {
  Factor r;
  if (norm > max_norm && norm <= 1.7976931348623157e308) {
    const double f = max_norm / norm;
    const int k = f < 0x1p-190 ? 149 : f < 0x1p-100 ? 64 : 0;
    r.up = ldexpf(1.0f, -k);
    r.f = (float)ldexp(f, k);
  }
  return r;
}

template <int N>
__global__ __launch_bounds__(kThreads) void k_clip(ClipTable<N> t, const double *part, int parts, double max_norm, float *norm) {
  __shared__ double lds[kThreads / 64];
  const double n = norm_of(part, parts, lds);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
  const Factor f = clip_factor(n, max_norm);
  int k = t.n - 1;
  for (int u = t.unit0[t.n] - 1 - (int)blockIdx.x; u >= 0; u -= gridDim.x) {
    k = range_of(t, u, k);
    const int64_t i0 = (int64_t)(u - t.unit0[k]) * t.kUnit + 4 * threadIdx.x, c = t.count[k];
    constexpr int kSteps = ClipTable<N>::kUnit / (4 * kThreads);
    float g[kSteps][4];
#pragma unroll
    for (int j = 0; j < kSteps; ++j) load4(t.g[k], t.type[k], i0 + 4 * kThreads * j, c - i0 - 4 * kThreads * j, g[j]);
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) g[j][i] = f.of(g[j][i]);
      store4(t.out[k], t.out_type[k], i0 + 4 * kThreads * j, c - i0 - 4 * kThreads * j, g[j]);
    }
  }
}

// Four values of each tensor a thread in a unit; the next unit's are read before the present ones are worked on, the
// first unit's before the norm is known.  Units of 1024 values, so that 2.1e6 parameters fill the card (of 4096: 15.1 us, of
// 1024 13.7); the powers of beta are taken once, by the sums' last block (by every block here: 19.9 us).
template <int N>
__global__ __launch_bounds__(kThreads) void k_adam(AdamTable<N> t, const double *part, int parts, AdamScalars o,
                                                   const AdamNow *now, int64_t *step, float *norm) {
  __shared__ double lds[kThreads / 64];
  Raw<float, 4> np, nm, nv, ng;   // ng: two words for a 16-bit type
  int k = t.n - 1;
  const auto at_of = [&](int u) { return (int64_t)(u - t.unit0[k]) * t.kUnit + 4 * threadIdx.x; };
  const auto fetch = [&](int u) {
    k = range_of(t, u, k);
    const int64_t at = at_of(u), left = t.count[k] - at;
    if (left >= 4) {
      load_raw<float, 4, kLast>(t.p[k] + at, np);
      load_raw<float, 4, kLast>(t.m[k] + at, nm);
      load_raw<float, 4, kLast>(t.v[k] + at, nv);
      if (t.type[k] == 0) load_raw<float, 4, kLast>((const float *)t.g[k] + at, ng);
      else copy_in<8, kLast>((const bf16_t *)t.g[k] + at, ng.w);
    } else {
      const int n = (int)left;
      load_raw_part<float, 4>(t.p[k] + at, n, np);
      load_raw_part<float, 4>(t.m[k] + at, n, nm);
      load_raw_part<float, 4>(t.v[k] + at, n, nv);
      if (t.type[k] == 0) {
        load_raw_part<float, 4>((const float *)t.g[k] + at, n, ng);
      } else {
        Raw<bf16_t, 4> h;
        load_raw_part<bf16_t, 4>((const bf16_t *)t.g[k] + at, n, h);
        ng.w[0] = h.w[0];
        ng.w[1] = h.w[1];
      }
    }
  };
  int u = t.unit0[t.n] - 1 - (int)blockIdx.x;
  if (u >= 0) fetch(u);
  Factor f;
  if (parts) {
    const double n = norm_of(part, parts, lds);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    if (!(n <= 1.7976931348623157e308)) return;
    if (o.max_norm > 0) f = clip_factor(n, o.max_norm);
  }
  if (step && blockIdx.x == 0 && threadIdx.x == 0) *step = now->step;
  const float lr = o.lr_device ? *o.lr_device : (float)o.lr, size = lr * now->grow1, root = now->root2;
  const float b1 = (float)o.beta1, c1 = (float)(1 - o.beta1), b2 = (float)o.beta2, c2 = (float)(1 - o.beta2);
  const float decay = lr * (float)o.weight_decay, eps = (float)o.eps;
  while (u >= 0) {
    float g[4], p[4], m[4], v[4];
    const int kc = k;
    const int64_t at = at_of(u), left = t.count[k] - at;
    unpack<float, 4>(np, p);
    unpack<float, 4>(nm, m);
    unpack<float, 4>(nv, v);
    if (t.type[k] == 0) {
      unpack<float, 4>(ng, g);
    } else if (t.type[k] == 1) {
      const Raw<bf16_t, 4> h{{ng.w[0], ng.w[1]}};
      unpack<bf16_t, 4>(h, g);
    } else {
      const Raw<f16_t, 4> h{{ng.w[0], ng.w[1]}};
      unpack<f16_t, 4>(h, g);
    }
    u -= gridDim.x;
    if (u >= 0) fetch(u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = f.of(g[i]);
      m[i] = fmaf(b1, m[i], c1 * x);
      v[i] = fmaf(b2, v[i], c2 * x * x);   // x * x alone would leave fp32's range first
      p[i] -= fmaf(decay, p[i], size * m[i] / fmaf(sqrtf(v[i]), root, eps));
    }
    const int n = left >= 4 ? 4 : (int)left;
    store_part<float, 4, kLast>(t.m[kc] + at, n, m);
    store_part<float, 4, kLast>(t.v[kc] + at, n, v);
    store_part<float, 4, kLast>(t.p[kc] + at, n, p);
    if (t.copy[kc]) store4(t.copy[kc], t.copy_type[kc], at, left, p);
  }
}

int grid_of(int units, int most) { return units < 1 ? 1 : units < most ? units : most; }

// The shorter form of a table of at most kFew ranges.
template <int N>
void few(const Units<N> &t, Units<kFew> &f) {
  f.n = t.n;
  for (int i = 0; i <= t.n; ++i) f.unit0[i] = t.unit0[i];
  for (int i = 0; i < t.n; ++i) {
    f.count[i] = t.count[i];
    f.type[i] = t.type[i];
  }
}

}  // namespace

hipError_t launch_sum_squares(const SumTable<kSumRanges> &t, double *part, int blocks, bool alone, const int64_t *step,
                              AdamNow *now, const AdamScalars &o, hipStream_t s) {
  if (t.n <= kFew) {
    SumTable<kFew> f;
    few(t, f);
    for (int i = 0; i < t.n; ++i) f.g[i] = t.g[i];
    if (alone) k_sum_squares<kFew, true><<<blocks, kThreads, 0, s>>>(f, part, step, now, o);
    else k_sum_squares<kFew, false><<<blocks, kThreads, 0, s>>>(f, part, step, now, o);
  } else {
    if (alone) k_sum_squares<kSumRanges, true><<<blocks, kThreads, 0, s>>>(t, part, step, now, o);
    else k_sum_squares<kSumRanges, false><<<blocks, kThreads, 0, s>>>(t, part, step, now, o);
  }
  return hipGetLastError();
}
hipError_t launch_norm(const double *part, int parts, float *norm, hipStream_t s) {
  k_norm<<<1, kThreads, 0, s>>>(part, parts, norm);
  return hipGetLastError();
}
hipError_t launch_clip(const ClipTable<kClipRanges> &t, const double *part, int parts, double max_norm, float *norm,
                       int cu_count, hipStream_t s) {
  const int grid = grid_of(t.unit0[t.n], 8 * cu_count);
  if (t.n <= kFew) {
    ClipTable<kFew> f;
    few(t, f);
    for (int i = 0; i < t.n; ++i) {
      f.g[i] = t.g[i];
      f.out[i] = t.out[i];
      f.out_type[i] = t.out_type[i];
    }
    k_clip<<<grid, kThreads, 0, s>>>(f, part, parts, max_norm, norm);
  } else {
    k_clip<<<grid, kThreads, 0, s>>>(t, part, parts, max_norm, norm);
  }
  return hipGetLastError();
}
hipError_t launch_now(const int64_t *step, AdamNow *now, const AdamScalars &o, hipStream_t s) {
  k_now<<<1, 1, 0, s>>>(step, now, o);
  return hipGetLastError();
}
hipError_t launch_adam(const AdamTable<kAdamRanges> &t, const double *part, int parts, const AdamScalars &o,
                       const AdamNow *now, int64_t *step, float *norm, int cu_count, hipStream_t s) {
  const int grid = grid_of(t.unit0[t.n], 8 * cu_count);
  if (t.n <= kFew) {
    AdamTable<kFew> f;
    few(t, f);
    for (int i = 0; i < t.n; ++i) {
      f.g[i] = t.g[i];
      f.p[i] = t.p[i];
      f.m[i] = t.m[i];
      f.v[i] = t.v[i];
      f.copy[i] = t.copy[i];
      f.copy_type[i] = t.copy_type[i];
    }
    k_adam<<<grid, kThreads, 0, s>>>(f, part, parts, o, now, step, norm);
  } else {
    k_adam<<<grid, kThreads, 0, s>>>(t, part, parts, o, now, step, norm);
  }
  return hipGetLastError();
}

}  // namespace aecct
