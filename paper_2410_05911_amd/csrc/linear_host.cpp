// Entry points of the linear maps and their gradients: argument checks, workspaces, launches.
#include <cstdint>

#include <hip/hip_runtime.h>

#include "../../include/aecct.h"
#include "linear.h"
#include "spans.h"

namespace {

using aecct::overlap;
using aecct::Span;

constexpr int64_t kMaxRows = (int64_t)1 << 40, kMaxSpan = (int64_t)1 << 56;   // no byte offset overflows
constexpr int64_t kMaxWidth = (int64_t)1 << 20;
constexpr int64_t kMaxIntWidth = 131071;       // |sum of products of two int8| < 2^31
constexpr int64_t kMaxTiles = (int64_t)1 << 22;   // of 64 x 64 outputs: the grid's threads stay below 2^32
constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

bool type_ok(int32_t t) { return t == AECCT_F32 || t == AECCT_BF16 || t == AECCT_F16; }
int64_t type_size(int32_t t) { return t == AECCT_F32 ? 4 : 2; }
bool stride_ok(const void *p, int64_t rows, int64_t ld, int64_t least) {
  return !p || (ld >= least && ld <= kMaxSpan / (rows > 0 ? rows : 1));
}
bool too_large(int64_t m, int64_t n) { return (m + 63) / 64 > kMaxTiles / ((n + 63) / 64); }

aecct_status sizes_ok(int64_t rows, int64_t in, int64_t out) {
  if (rows < 0 || rows > kMaxRows || in < 1 || out < 1) return AECCT_ERR_INVALID_ARG;
  if (in > kMaxWidth || out > kMaxWidth || too_large(rows, in > out ? in : out) || too_large(in, out)) return AECCT_ERR_UNSUPPORTED;
  return AECCT_OK;
}

aecct_status check_linear(const aecct_linear_map_args *a) {
  if (!a) return AECCT_ERR_INVALID_ARG;
  if (a->code_type != AECCT_CODE_NONE && a->code_type != AECCT_CODE_I8 && a->code_type != AECCT_CODE_E4M3)
    return AECCT_ERR_INVALID_ARG;
  if (!type_ok(a->y_type) || (a->code_type == AECCT_CODE_NONE && a->type != a->y_type)) return AECCT_ERR_INVALID_ARG;
  if (a->act < AECCT_ACT_NONE || a->act > AECCT_ACT_SILU || (a->w_turned != 0 && a->w_turned != 1)) return AECCT_ERR_INVALID_ARG;
  const aecct_status s = sizes_ok(a->rows, a->in, a->out);
  if (s != AECCT_OK) return s;
  return a->code_type == AECCT_CODE_I8 && a->in > kMaxIntWidth ? AECCT_ERR_UNSUPPORTED : AECCT_OK;
}
int kind(const aecct_linear_map_args *a) { return a->code_type == AECCT_CODE_NONE ? a->type : aecct::kCodeType + a->code_type; }
aecct::GemmPlan plan(const aecct_linear_map_args *a) {
  return aecct::plan_gemm(kind(a), a->rows, a->out, a->in, false, !a->w_turned, a->ldw);
}

aecct_status check_grad(const aecct_linear_map_grad_args *a) {
  if (!a || !type_ok(a->type) || (a->dw_type != AECCT_F32 && a->dw_type != a->type)) return AECCT_ERR_INVALID_ARG;
  if (a->act < AECCT_ACT_NONE || a->act > AECCT_ACT_SILU || (a->w_turned != 0 && a->w_turned != 1)) return AECCT_ERR_INVALID_ARG;
  return sizes_ok(a->rows, a->in, a->out);
}
// What a gradient's workspace holds: dz, the splits' sums of one product after the other, the column sums.
struct GradWork {
  aecct::GemmPlan dx, dw;
  int64_t lddz;
  size_t dz, part, sums, total;
};
GradWork grad_work(const aecct_linear_map_grad_args *a) {
  GradWork w{};
  w.dx = aecct::plan_gemm(a->type, a->rows, a->in, a->out, false, a->w_turned, a->ldw);
  w.dw = aecct::plan_gemm(a->type, a->in, a->out, a->rows, true, true, 0);
  w.lddz = (a->out + 63) / 64 * 64;
  w.dz = a->act != AECCT_ACT_NONE ? align_up((size_t)(a->rows * w.lddz * type_size(a->type))) : 0;
  const size_t p = a->dx ? w.dx.part_bytes : 0, q = a->dw ? w.dw.part_bytes : 0;
  w.part = align_up(p > q ? p : q);
  w.sums = a->dbias ? align_up((size_t)(aecct::slope_blocks(a->rows, a->out) * a->out) * 4) : 0;
  w.total = w.dz + w.part + w.sums;
  if (w.total) w.total += kAlign;
  return w;
}

}  // namespace

extern "C" {

aecct_status aecct_linear_map_workspace_size(const aecct_linear_map_args *a, size_t *bytes) {
  if (!bytes) return AECCT_ERR_INVALID_ARG;
  const aecct_status s = check_linear(a);
  if (s != AECCT_OK) return s;
  const size_t part = plan(a).part_bytes;
  *bytes = part ? kAlign + align_up(part) : 0;
  return AECCT_OK;
}

aecct_status aecct_linear_map(const aecct_linear_map_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  const aecct_status s = check_linear(a);
  if (s != AECCT_OK) return s;
  if (a->rows == 0) return AECCT_OK;
  const bool coded = a->code_type != AECCT_CODE_NONE;
  if (!a->x || !a->w || !a->y || coded != (a->alpha != nullptr) || coded != (a->scale != nullptr)) return AECCT_ERR_INVALID_ARG;
  const int64_t lines = a->w_turned ? a->out : a->in, across = a->w_turned ? a->in : a->out;
  if (!stride_ok(a->x, a->rows, a->ldx, 0) || !stride_ok(a->w, lines, a->ldw, across) ||
      !stride_ok(a->res, a->rows, a->ldres, 0) || !stride_ok(a->z, a->rows, a->ldz, a->out) ||
      !stride_ok(a->y, a->rows, a->ldy, a->out))
    return AECCT_ERR_INVALID_ARG;
  const int64_t size = coded ? 1 : type_size(a->type), ysize = type_size(a->y_type);
  const Span in[6] = {{a->x, a->rows, a->in * size, a->ldx * size},
                      {a->w, lines, across * size, a->ldw * size},
                      {a->alpha, 1, 4 * a->rows, 0},
                      {a->scale, 1, 4 * a->out, 0},
                      {a->bias, 1, 4 * a->out, 0},
                      {a->res, a->rows, a->out * ysize, a->ldres * ysize}};
  const Span out[2] = {{a->z, a->rows, a->out * ysize, a->ldz * ysize}, {a->y, a->rows, a->out * ysize, a->ldy * ysize}};
  if (overlap(out[0], out[1])) return AECCT_ERR_INVALID_ARG;
  for (int i = 0; i < 6; ++i)
    for (int k = 0; k < 2; ++k)
      if (overlap(out[k], in[i]) && !(i == 5 && k == 1 && same(out[k], in[i]))) return AECCT_ERR_INVALID_ARG;
  const aecct::GemmPlan p = plan(a);
  void *part = nullptr;
  if (p.part_bytes) {
    const size_t need = kAlign + align_up(p.part_bytes);
    if (workspace_bytes < need) return AECCT_ERR_WORKSPACE_TOO_SMALL;
    if (!workspace) return AECCT_ERR_INVALID_ARG;
    const Span ws{workspace, 1, (int64_t)need, 0};
    for (const Span &t : in)
      if (overlap(ws, t)) return AECCT_ERR_INVALID_ARG;
    if (overlap(ws, out[0]) || overlap(ws, out[1])) return AECCT_ERR_INVALID_ARG;
    part = (void *)align_up((size_t)(uintptr_t)workspace);
  }
  const float q = a->code_type == AECCT_CODE_I8 ? 127.0f : 448.0f;
  const aecct::Gemm g{(int)a->rows, (int)a->out, (int)a->in, {a->x, a->ldx, false}, {a->w, a->ldw, !a->w_turned},
                      {a->alpha, a->scale, a->bias, 1.0f / q, a->act, a->y_type, a->res, a->z, a->y, a->ldres, a->ldz, a->ldy},
                      part, p.splits};
  return aecct::launch_gemm(kind(a), g, p, (hipStream_t)stream) == hipSuccess ? AECCT_OK : AECCT_ERR_DEVICE;
}

aecct_status aecct_linear_map_grad_workspace_size(const aecct_linear_map_grad_args *a, size_t *bytes) {
  if (!bytes) return AECCT_ERR_INVALID_ARG;
  const aecct_status s = check_grad(a);
  if (s != AECCT_OK) return s;
  *bytes = grad_work(a).total;
  return AECCT_OK;
}

aecct_status aecct_linear_map_grad(const aecct_linear_map_grad_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  const aecct_status st = check_grad(a);
  if (st != AECCT_OK) return st;
  if (!a->dx && !a->dw && !a->dbias) return AECCT_ERR_INVALID_ARG;
  const bool sloped = a->act != AECCT_ACT_NONE;
  if (a->rows && (!a->dy || (a->dx && !a->w) || (a->dw && !a->x) || sloped != (a->z != nullptr))) return AECCT_ERR_INVALID_ARG;
  const int64_t lines = a->w_turned ? a->out : a->in, across = a->w_turned ? a->in : a->out;
  if (!stride_ok(a->x, a->rows, a->ldx, 0) || !stride_ok(a->w, lines, a->ldw, across) ||
      !stride_ok(a->dy, a->rows, a->lddy, 0) || !stride_ok(a->z, a->rows, a->ldz, 0) ||
      !stride_ok(a->dx, a->rows, a->lddx, a->in) || !stride_ok(a->dw, a->in, a->lddw, a->out))
    return AECCT_ERR_INVALID_ARG;
  const int64_t size = type_size(a->type), wsize = type_size(a->dw_type);
  const Span in[4] = {{a->x, a->rows, a->in * size, a->ldx * size},
                      {a->w, lines, across * size, a->ldw * size},
                      {a->dy, a->rows, a->out * size, a->lddy * size},
                      {a->z, a->rows, a->out * size, a->ldz * size}};
  const Span out[3] = {{a->dx, a->rows, a->in * size, a->lddx * size},
                       {a->dw, a->in, a->out * wsize, a->lddw * wsize},
                       {a->dbias, 1, 4 * a->out, 0}};
  for (int i = 0; i < 3; ++i) {
    for (int k = 0; k < i; ++k)
      if (overlap(out[i], out[k])) return AECCT_ERR_INVALID_ARG;
    for (const Span &t : in)
      if (overlap(out[i], t)) return AECCT_ERR_INVALID_ARG;
  }
  const GradWork w = grad_work(a);
  char *dz = nullptr, *part = nullptr, *sums = nullptr;
  if (w.total) {
    if (workspace_bytes < w.total) return AECCT_ERR_WORKSPACE_TOO_SMALL;
    if (!workspace) return AECCT_ERR_INVALID_ARG;
    const Span ws{workspace, 1, (int64_t)w.total, 0};
    for (const Span &t : in)
      if (overlap(ws, t)) return AECCT_ERR_INVALID_ARG;
    for (const Span &t : out)
      if (overlap(ws, t)) return AECCT_ERR_INVALID_ARG;
    dz = (char *)align_up((size_t)(uintptr_t)workspace);
    part = dz + w.dz;
    sums = part + w.part;
  }
  const hipStream_t s = (hipStream_t)stream;
  const bool need_dz = sloped && (a->dx || a->dw);
  if (need_dz || a->dbias) {
    const aecct::Slope v{a->rows, a->out, a->act, a->dy, a->z, a->lddy, a->ldz, need_dz ? dz : nullptr, w.lddz,
                         a->dbias ? (float *)sums : nullptr, a->dbias};
    if (aecct::launch_slope(a->type, v, s) != hipSuccess) return AECCT_ERR_DEVICE;
  }
  const void *const d = need_dz ? (const void *)dz : a->dy;
  const int64_t ldd = need_dz ? w.lddz : a->lddy;
  if (a->dx && a->rows) {
    const aecct::Gemm g{(int)a->rows, (int)a->in, (int)a->out, {d, ldd, false}, {a->w, a->ldw, a->w_turned != 0},
                        {nullptr, nullptr, nullptr, 0.0f, 0, a->type, nullptr, nullptr, a->dx, 0, 0, a->lddx},
                        w.dx.part_bytes ? part : nullptr, w.dx.splits};
    if (aecct::launch_gemm(a->type, g, w.dx, s) != hipSuccess) return AECCT_ERR_DEVICE;
  }
  if (a->dw) {
    const aecct::Gemm g{(int)a->in, (int)a->out, (int)a->rows, {a->x, a->ldx, true}, {d, ldd, true},
                        {nullptr, nullptr, nullptr, 0.0f, 0, a->dw_type, nullptr, nullptr, a->dw, 0, 0, a->lddw},
                        w.dw.part_bytes ? part : nullptr, w.dw.splits};
    if (aecct::launch_gemm(a->type, g, w.dw, s) != hipSuccess) return AECCT_ERR_DEVICE;
  }
  return AECCT_OK;
}

}  // extern "C"
