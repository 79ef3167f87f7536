// Entry point of dropout: argument checks, then the launch.
#include <cstdint>

#include <hip/hip_runtime.h>

#include "../../include/aecct.h"
#include "dropout.h"
#include "spans.h"

namespace {

using aecct::overlap;
using aecct::Span;

constexpr int64_t kMaxRows = (int64_t)1 << 40, kMaxSpan = (int64_t)1 << 56;   // no byte offset overflows
constexpr int64_t kMaxChunks = ((int64_t)1 << 32) - 512;                     // of 8 values: threads of a grid

bool stride_ok(const void *p, int64_t rows, int64_t ld, int64_t least) {
  return !p || (ld >= least && ld <= kMaxSpan / (rows > 0 ? rows : 1));
}

}  // namespace

extern "C" aecct_status aecct_dropout(const aecct_dropout_args *a, void *stream) {
  if (!a || a->rows < 0 || a->rows > kMaxRows || a->d < 1) return AECCT_ERR_INVALID_ARG;
  if (a->type != AECCT_F32 && a->type != AECCT_BF16 && a->type != AECCT_F16) return AECCT_ERR_INVALID_ARG;
  if (!(a->p >= 0.0 && a->p < 1.0)) return AECCT_ERR_INVALID_ARG;
  if (a->d > kMaxRows || (a->rows && (a->d + 7) / 8 > kMaxChunks / a->rows)) return AECCT_ERR_UNSUPPORTED;
  if (a->rows == 0) return AECCT_OK;
  if (!a->x || !a->y) return AECCT_ERR_INVALID_ARG;
  if (!stride_ok(a->x, a->rows, a->ldx, 0) || !stride_ok(a->res, a->rows, a->ldres, 0) || !stride_ok(a->y, a->rows, a->ldy, a->d))
    return AECCT_ERR_INVALID_ARG;
  const int64_t size = a->type == AECCT_F32 ? 4 : 2;
  const Span x{a->x, a->rows, a->d * size, a->ldx * size}, res{a->res, a->rows, a->d * size, a->ldres * size},
      y{a->y, a->rows, a->d * size, a->ldy * size}, off{a->offset_device, 1, 8, 0};
  if ((overlap(y, x) && !same(y, x)) || (overlap(y, res) && !same(y, res)) || overlap(y, off)) return AECCT_ERR_INVALID_ARG;
  const aecct::Dropout d{a->rows, a->d, (uint32_t)(a->p * 4294967296.0), (float)(1.0 / (1.0 - a->p)), a->seed, a->offset,
                         a->offset_device, a->x, a->res, a->y, a->ldx, a->ldres, a->ldy};
  return aecct::launch_dropout(a->type, d, (hipStream_t)stream) == hipSuccess ? AECCT_OK : AECCT_ERR_DEVICE;
}
