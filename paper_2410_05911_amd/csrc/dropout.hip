// Dropout whose mask is never stored: y = x kept / (1 - p) + res.  Value i of the tensor (row by row) takes word i % 4 of
// Philox4x32-7's block with the counter (i / 4, offset) and the key `seed` (Salmon, Moraes, Dror and Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC 2011), so any call with the same numbers, also on a gradient, drops the same values.
//
// Eight values a thread, so 16-byte accesses in 16 bits and two blocks of words; where rows begin inside a block, three.  Bound by
// memory (16384 x 8192 bf16 with residual 136 us, 5.9 TB/s; the words' products and exclusive ors take 60 % of the clocks beside),
// small calls by the launch (5888 x 32 fp32: 3 us on the GPU, 7.5 with the host).
#include "../../include/aecct.h"
#include "dropout.h"
#include "row_io.h"

namespace aecct {
namespace {

// Seven rounds: the high and low halves of two 32 x 32-bit products change places.
__device__ __forceinline__ void philox(uint64_t block, uint64_t offset, uint64_t seed, uint32_t (&w)[4]) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)q;
    c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  w[0] = c0;
  w[1] = c1;
  w[2] = c2;
  w[3] = c3;
}

// Eight values a thread.  WHOLE: rows begin at the first word of a block (d % 4 = 0, or all values are one row).
template <class T, bool WHOLE>
__global__ __launch_bounds__(256) void k_dropout(Dropout a) {
  const int64_t per = (a.d + 7) / 8, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= a.rows * per) return;
  int64_t row = 0, chunk = at;
  if (a.rows > 1) {
    // an unsigned 32-bit division is a quarter of a 64-bit one
    if ((uint64_t)at >> 32 == 0 && per >> 32 == 0) {
      row = (uint32_t)at / (uint32_t)per;
      chunk = (uint32_t)at % (uint32_t)per;
    } else {
      row = at / per;
      chunk = at % per;
    }
  }
  const int64_t c = chunk * 8;
  const int count = a.d - c < 8 ? (int)(a.d - c) : 8;
  const uint64_t first = (uint64_t)row * (uint64_t)a.d + (uint64_t)c;
  const uint64_t offset = a.offset_device ? (uint64_t)*a.offset_device : a.offset;
  Raw<T, 8> rx, rr;
  float v[8], r[8];
  const T *const px = (const T *)a.x + row * a.ldx + c, *const pr = (const T *)a.res + row * a.ldres + c;
  if (count == 8) {
    load_raw<T, 8>(px, rx);
    if (a.res) load_raw<T, 8>(pr, rr);
  } else {
    load_raw_part<T, 8>(px, count, rx);
    if (a.res) load_raw_part<T, 8>(pr, count, rr);
  }
  uint32_t w[12];
#pragma unroll
  for (int b = 0; b < (WHOLE ? 2 : 3); ++b) {
    uint32_t t[4];
    philox(first / 4 + b, offset, a.seed, t);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[4 * b + i] = t[i];
  }
  if constexpr (!WHOLE) {   // word first % 4 to the front
#pragma unroll
    for (int by = 1; by <= 2; by *= 2) {
      if (first & by) {
#pragma unroll
        for (int i = 0; i + by < 12; ++i) w[i] = w[i + by];
      }
    }
  }
  unpack<T, 8>(rx, v);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = w[i] >= a.below ? v[i] * a.scale : 0.0f;
  if (a.res) {
    unpack<T, 8>(rr, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += r[i];
  }
  store_part<T, 8>((T *)a.y + row * a.ldy + c, count, v);
}

template <class T>
hipError_t launch(Dropout a, hipStream_t s) {
  if (a.ldx == a.d && a.ldy == a.d && (!a.res || a.ldres == a.d)) {
    a.d *= a.rows;
    a.rows = 1;
  }
  const dim3 grid((unsigned)((a.rows * ((a.d + 7) / 8) + 255) / 256));
  if (a.rows == 1 || a.d % 4 == 0) k_dropout<T, true><<<grid, 256, 0, s>>>(a);
  else k_dropout<T, false><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(int type, const Dropout &a, hipStream_t s) {
  switch (type) {
    case AECCT_F32: return launch<float>(a, s);
    case AECCT_BF16: return launch<bf16_t>(a, s);
    case AECCT_F16: return launch<f16_t>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace aecct
