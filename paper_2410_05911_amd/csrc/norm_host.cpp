// Entry points of the root-mean-square norm and its gradient: argument checks, then the launch.
#include <cmath>
#include <cstdint>

#include <hip/hip_runtime.h>

#include "../../include/aecct.h"
#include "norm.h"

namespace {

constexpr int64_t kMaxWidth = 65536;      // a row is held in a block's registers
constexpr int64_t kMaxRows = (int64_t)1 << 40, kMaxSpan = (int64_t)1 << 56;   // values: no byte offset overflows
constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

bool type_ok(int32_t t) { return t == AECCT_F32 || t == AECCT_BF16 || t == AECCT_F16; }
int64_t type_size(int32_t t) { return t == AECCT_F32 ? 4 : 2; }

// `rows` rows of `width` bytes, `pitch` bytes apart.
struct Rows {
  const void *p;
  int64_t rows, width, pitch;
  uintptr_t begin() const { return (uintptr_t)p; }
  uintptr_t end() const { return rows > 0 ? begin() + (uintptr_t)((rows - 1) * pitch + width) : begin(); }
};
bool same(const Rows &a, const Rows &b) { return a.p == b.p && a.width == b.width && (a.pitch == b.pitch || a.rows <= 1); }
// Whether two regions may share a byte: their spans do, unless both are columns of rows of one pitch that lie side
// by side.
bool overlap(const Rows &a, const Rows &b) {
  if (!a.p || !b.p || a.begin() >= b.end() || b.begin() >= a.end()) return false;
  if (a.pitch != b.pitch || a.pitch <= 0) return true;
  const uintptr_t pitch = (uintptr_t)a.pitch;
  const uintptr_t off = b.begin() >= a.begin() ? (b.begin() - a.begin()) % pitch
                                               : (pitch - (a.begin() - b.begin()) % pitch) % pitch;
  return !(off >= (uintptr_t)a.width && off + (uintptr_t)b.width <= pitch);
}

bool stride_ok(const void *p, int64_t rows, int64_t ld, int64_t least) {
  return !p || (ld >= least && ld <= kMaxSpan / (rows > 0 ? rows : 1));
}

// Which sizes go past the 256 MB of cache between the chip and its memory.  Inputs of more than half of it will not be
// found there again, and leave it to the outputs if they go past (16384 x 4096 bf16 with residual: 102 -> 81 us); smaller
// ones often lie there still, from the kernel that made them (49152 x 128 fp32: 14.7 us, past it 16.3).  Outputs go past
// it where they are well over its size (16384 x 8192 to 8-bit codes 183 -> 170 us; 16384 x 4096, 268 MB, 81 -> 94).
constexpr int64_t kPastInputs = (int64_t)128 << 20, kPastOutputs = (int64_t)384 << 20;

}  // namespace

extern "C" {

aecct_status aecct_rms_norm(const aecct_rms_norm_args *a, void *stream) {
  if (!a || a->rows < 0 || a->rows > kMaxRows || a->d < 1 || !type_ok(a->type)) return AECCT_ERR_INVALID_ARG;
  if (a->gain_type != AECCT_F32 && a->gain_type != a->type) return AECCT_ERR_INVALID_ARG;
  if (!(a->eps >= 0.0f) || !std::isfinite(a->eps)) return AECCT_ERR_INVALID_ARG;
  if (a->code_type != AECCT_CODE_NONE && a->code_type != AECCT_CODE_I8 && a->code_type != AECCT_CODE_E4M3)
    return AECCT_ERR_INVALID_ARG;
  if (a->group != 0 && a->group != 32 && a->group != 64 && a->group != 128) return AECCT_ERR_INVALID_ARG;
  const bool coded = a->code_type != AECCT_CODE_NONE;
  if (a->d > kMaxWidth) return AECCT_ERR_UNSUPPORTED;
  if (a->rows == 0) return AECCT_OK;
  if (coded != (a->codes != nullptr) || coded != (a->alpha != nullptr)) return AECCT_ERR_INVALID_ARG;
  if (!a->x || (!a->h && !a->y && !coded)) return AECCT_ERR_INVALID_ARG;
  if (!stride_ok(a->x, a->rows, a->ldx, 0) || !stride_ok(a->res, a->rows, a->ldres, 0) || !stride_ok(a->h, a->rows, a->ldh, a->d) ||
      !stride_ok(a->y, a->rows, a->ldy, a->d) || !stride_ok(a->codes, a->rows, a->ldcodes, a->d))
    return AECCT_ERR_INVALID_ARG;
  const int64_t size = type_size(a->type), group = a->group && a->group < a->d ? a->group : a->d;
  const int64_t alphas = (a->d + group - 1) / group;
  const Rows x{a->x, a->rows, a->d * size, a->ldx * size}, res{a->res, a->rows, a->d * size, a->ldres * size},
      gain{a->gain, 1, a->d * type_size(a->gain_type), 0};
  const Rows out[4] = {{a->h, a->rows, a->d * size, a->ldh * size},
                       {a->y, a->rows, a->d * size, a->ldy * size},
                       {a->codes, a->rows, a->d, a->ldcodes},
                       {a->alpha, a->rows, 4 * alphas, 4 * alphas}};
  for (int i = 0; i < 4; ++i) {
    for (int k = 0; k < i; ++k)
      if (overlap(out[i], out[k])) return AECCT_ERR_INVALID_ARG;
    if (overlap(out[i], gain) || (overlap(out[i], x) && !(i < 2 && same(out[i], x))) ||
        (overlap(out[i], res) && !(i < 2 && same(out[i], res))))
      return AECCT_ERR_INVALID_ARG;
  }
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    return AECCT_ERR_DEVICE;
  const int64_t values = a->rows * a->d, in_bytes = values * size * (a->res ? 2 : 1),
                out_bytes = values * (size * ((a->h ? 1 : 0) + (a->y ? 1 : 0)) + (coded ? 1 : 0));
  const aecct::NormRows n{a->rows, (int)a->d, a->eps, a->gain_type == AECCT_F32, a->code_type, (int)group, (int)alphas,
                          a->x, a->res, a->gain, a->h, a->y, (uint8_t *)a->codes, a->alpha, a->ldx, a->ldres, a->ldh,
                          a->ldy, a->ldcodes, in_bytes > kPastInputs, out_bytes > kPastOutputs};
  return aecct::launch_rms_norm(a->type, n, cus, (hipStream_t)stream) == hipSuccess ? AECCT_OK : AECCT_ERR_DEVICE;
}

aecct_status aecct_rms_norm_grad_workspace_size(int64_t rows, int64_t d, size_t *bytes) {
  if (!bytes || rows < 0 || rows > kMaxRows || d < 1) return AECCT_ERR_INVALID_ARG;
  if (d > kMaxWidth) return AECCT_ERR_UNSUPPORTED;
  *bytes = kAlign + align_up((size_t)aecct::norm_grad_part_rows(rows, (int)d) * (size_t)d * 4);
  return AECCT_OK;
}

aecct_status aecct_rms_norm_grad(const aecct_rms_norm_grad_args *a, void *workspace, size_t workspace_bytes,
                                 void *stream) {
  if (!a || a->rows < 0 || a->rows > kMaxRows || a->d < 1 || !type_ok(a->type)) return AECCT_ERR_INVALID_ARG;
  if (a->gain_type != AECCT_F32 && a->gain_type != a->type) return AECCT_ERR_INVALID_ARG;
  if (!(a->eps >= 0.0f) || !std::isfinite(a->eps)) return AECCT_ERR_INVALID_ARG;
  if (a->d > kMaxWidth) return AECCT_ERR_UNSUPPORTED;
  if ((a->rows && (!a->h || !a->dy)) || (!a->dh && !a->dgain)) return AECCT_ERR_INVALID_ARG;
  if (!stride_ok(a->h, a->rows, a->ldh, 0) || !stride_ok(a->dy, a->rows, a->lddy, 0) || !stride_ok(a->dres, a->rows, a->lddres, 0) ||
      !stride_ok(a->dh, a->rows, a->lddh, a->d))
    return AECCT_ERR_INVALID_ARG;
  const int64_t size = type_size(a->type);
  const Rows in[4] = {{a->h, a->rows, a->d * size, a->ldh * size},
                      {a->dy, a->rows, a->d * size, a->lddy * size},
                      {a->dres, a->rows, a->d * size, a->lddres * size},
                      {a->gain, 1, a->d * type_size(a->gain_type), 0}};
  const Rows dh{a->dh, a->rows, a->d * size, a->lddh * size}, dgain{a->dgain, 1, 4 * a->d, 0};
  if (overlap(dh, dgain)) return AECCT_ERR_INVALID_ARG;
  for (int i = 0; i < 4; ++i)
    if (overlap(dgain, in[i]) || (overlap(dh, in[i]) && !(i < 3 && same(dh, in[i])))) return AECCT_ERR_INVALID_ARG;
  float *part = nullptr;
  if (a->dgain) {
    size_t need = 0;
    (void)aecct_rms_norm_grad_workspace_size(a->rows, a->d, &need);
    if (workspace_bytes < need) return AECCT_ERR_WORKSPACE_TOO_SMALL;
    if (!workspace) return AECCT_ERR_INVALID_ARG;
    const Rows ws{workspace, 1, (int64_t)need, 0};
    if (overlap(ws, dh) || overlap(ws, dgain)) return AECCT_ERR_INVALID_ARG;
    for (int i = 0; i < 4; ++i)
      if (overlap(ws, in[i])) return AECCT_ERR_INVALID_ARG;
    part = (float *)align_up((size_t)(uintptr_t)workspace);
  }
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    return AECCT_ERR_DEVICE;
  const int64_t values = a->rows * a->d;
  const aecct::NormGradRows n{a->rows, (int)a->d, a->eps, a->gain_type == AECCT_F32, a->h, a->dy, a->dres, a->gain, a->dh,
                              a->ldh, a->lddy, a->lddres, a->lddh, part, a->dgain,
                              values * size * (a->dres ? 3 : 2) > kPastInputs};
  return aecct::launch_rms_norm_grad(a->type, n, cus, (hipStream_t)stream) == hipSuccess ? AECCT_OK : AECCT_ERR_DEVICE;
}

}  // extern "C"
