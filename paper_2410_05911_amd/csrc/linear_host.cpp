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
// Factors that are no whole 16-byte pieces are copied into such where that pays: where the product takes longer than the launch that copies
// them, and each copied value enters so many products that its reading and writing is less than what the product gains.  A map in 16
// or 8 bits, from 300 products a value on (bf16 1295 x 7731 -> 1082, 580 a value, 114 -> 88 us; 9987 x 4929 -> 187, 184 a value, copied
// 77, as it lies 64), in fp32 from 2000 on (2001 x 1001 -> 2601, 1130 a value, copied 124 us, as it lies 119; 6081 x 2480 -> 4735, 6081 a
// value, 1143 and 1180).  A gradient, which reads a factor across its lines, from 160 on (7717 x 5137 -> 128, 126 a value, fp32 279 and 231, bf16 94 and 75; 1001 x 777 ->
// 1333, 330 a value, fp32 77 and 92, bf16 25.5 and 39).
constexpr double kPackWork = 4e9, kPackMap = 300, kPackMap32 = 2000, kPackGrad = 160;
// A forward map's workspace: copies of ragged factors, the splits' sums.
struct MapWork {
  aecct::GemmPlan plan;
  bool pack_x, pack_w;
  int64_t ldx, ldw;
  size_t x, w, part, total;
};
MapWork map_work(const aecct_linear_map_args *a) {
  MapWork m{};
  const int t = kind(a);
  const int64_t lines = a->w_turned ? a->out : a->in, across = a->w_turned ? a->in : a->out;
  const bool ragged_x = aecct::ragged(t, a->ldx, a->in), ragged_w = aecct::ragged(t, a->ldw, across),
             pack = 2.0 * a->rows * a->in * a->out >= kPackWork &&
                    (double)a->rows * a->in * a->out >=
                        (t == AECCT_F32 ? kPackMap32 : kPackMap) *
                            ((ragged_x ? (double)a->rows * a->in : 0) + (ragged_w ? (double)a->in * a->out : 0));
  m.plan = aecct::plan_gemm(t, a->rows, a->out, a->in, false, !a->w_turned, a->ldw, pack || !(ragged_x || ragged_w));
  if (!m.plan.few && pack) {
    m.pack_x = ragged_x;
    m.pack_w = ragged_w;
  }
  m.ldx = aecct::packed_line(t, a->in);
  m.ldw = aecct::packed_line(t, across);
  m.x = m.pack_x ? align_up((size_t)(a->rows * m.ldx * aecct::type_bytes(t))) : 0;
  m.w = m.pack_w ? align_up((size_t)(lines * m.ldw * aecct::type_bytes(t))) : 0;
  m.part = align_up(m.plan.part_bytes);
  m.total = m.x + m.w + m.part;
  if (m.total) m.total += kAlign;
  return m;
}

aecct_status check_grad(const aecct_linear_map_grad_args *a) {
  if (!a || !type_ok(a->type) || (a->dw_type != AECCT_F32 && a->dw_type != a->type)) return AECCT_ERR_INVALID_ARG;
  if (a->act < AECCT_ACT_NONE || a->act > AECCT_ACT_SILU || (a->w_turned != 0 && a->w_turned != 1)) return AECCT_ERR_INVALID_ARG;
  return sizes_ok(a->rows, a->in, a->out);
}
// What a gradient's workspace holds: dz, copies of ragged factors, the splits' sums of both products, the column sums.
struct GradWork {
  aecct::GemmPlan dx, dw;
  bool need_dz, pack_x, pack_w, pack_dy;
  int64_t lddz, ldx, ldw;
  size_t dz, x, w, part_dx, part_dw, sums, total;
};
GradWork grad_work(const aecct_linear_map_grad_args *a) {
  GradWork w{};
  const int t = a->type, size = aecct::type_bytes(t);
  const int64_t lines = a->w_turned ? a->out : a->in, across = a->w_turned ? a->in : a->out;
  w.need_dz = a->act != AECCT_ACT_NONE && (a->dx || a->dw);
  w.lddz = aecct::packed_line(t, a->out);
  const bool ragged_x = aecct::ragged(t, a->ldx, a->in), ragged_w = aecct::ragged(t, a->ldw, across),
             ragged_d = !w.need_dz && aecct::ragged(t, a->lddy, a->out);
  const double values = (a->dw && ragged_x ? (double)a->rows * a->in : 0) + (a->dx && ragged_w ? (double)a->in * a->out : 0) +
                        (ragged_d ? (double)a->rows * a->out : 0);
  // (a first launch for dz or the sums is there anyway)
  const bool pack = (w.need_dz || a->dbias || 2.0 * a->rows * a->in * a->out >= kPackWork) &&
                    (double)a->rows * a->in * a->out >= kPackGrad * values;
  w.dx = aecct::plan_gemm(t, a->rows, a->in, a->out, false, a->w_turned, a->ldw, pack || !(ragged_w || ragged_d));
  w.dw = aecct::plan_gemm(t, a->in, a->out, a->rows, true, true, 0, pack || !(ragged_x || ragged_d));
  if (pack) {
    w.pack_x = a->dw && ragged_x;
    w.pack_w = a->dx && !w.dx.few && ragged_w;
    w.pack_dy = ragged_d && (a->dw || (a->dx && !w.dx.few));
  }
  w.ldx = aecct::packed_line(t, a->in);
  w.ldw = aecct::packed_line(t, across);
  w.dz = w.need_dz || w.pack_dy ? align_up((size_t)(a->rows * w.lddz * size)) : 0;
  w.x = w.pack_x ? align_up((size_t)(a->rows * w.ldx * size)) : 0;
  w.w = w.pack_w ? align_up((size_t)(lines * w.ldw * size)) : 0;
  w.part_dx = a->dx ? align_up(w.dx.part_bytes) : 0;
  w.part_dw = a->dw ? align_up(w.dw.part_bytes) : 0;
  w.sums = a->dbias ? align_up((size_t)(aecct::slope_blocks(a->rows, a->out) * a->out) * 4) : 0;
  w.total = w.dz + w.x + w.w + w.part_dx + w.part_dw + w.sums;
  if (w.total) w.total += kAlign;
  return w;
}

}  // namespace

extern "C" {

aecct_status aecct_linear_map_workspace_size(const aecct_linear_map_args *a, size_t *bytes) {
  if (!bytes) return AECCT_ERR_INVALID_ARG;
  const aecct_status s = check_linear(a);
  if (s != AECCT_OK) return s;
  *bytes = map_work(a).total;
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
  const MapWork m = map_work(a);
  char *ws = nullptr;
  if (m.total) {
    if (workspace_bytes < m.total) return AECCT_ERR_WORKSPACE_TOO_SMALL;
    if (!workspace) return AECCT_ERR_INVALID_ARG;
    const Span all{workspace, 1, (int64_t)m.total, 0};
    for (const Span &t : in)
      if (overlap(all, t)) return AECCT_ERR_INVALID_ARG;
    if (overlap(all, out[0]) || overlap(all, out[1])) return AECCT_ERR_INVALID_ARG;
    ws = (char *)align_up((size_t)(uintptr_t)workspace);
  }
  aecct::Factor x{a->x, a->ldx, false, false}, w{a->w, a->ldw, !a->w_turned, false};
  aecct::Prepare prepare{};
  if (m.pack_x) {
    prepare.pack[0] = {a->x, a->ldx, (int)a->rows, (int)a->in, ws, m.ldx};
    x = {ws, m.ldx, false, true};
  }
  if (m.pack_w) {
    prepare.pack[1] = {a->w, a->ldw, (int)lines, (int)across, ws + m.x, m.ldw};
    w = {ws + m.x, m.ldw, !a->w_turned, true};
  }
  const float q = a->code_type == AECCT_CODE_I8 ? 127.0f : 448.0f;
  const aecct::Gemm g{(int)a->rows, (int)a->out, (int)a->in, x, w,
                      {a->alpha, a->scale, a->bias, 1.0f / q, a->act, a->y_type, a->res, a->z, a->y, a->ldres, a->ldz, a->ldy},
                      m.plan.part_bytes ? ws + m.x + m.w : nullptr, m.plan.splits};
  const hipStream_t st = (hipStream_t)stream;
  const int t = kind(a);
  if ((m.pack_x || m.pack_w) && aecct::launch_prepare(t, prepare, st) != hipSuccess) return AECCT_ERR_DEVICE;
  if (aecct::launch_gemm(t, &g, &m.plan, 1, st) != hipSuccess) return AECCT_ERR_DEVICE;
  if (!g.part) return AECCT_OK;
  aecct::Finish f{};
  f.g[0] = g;
  return aecct::launch_finish(t, f, st) == hipSuccess ? AECCT_OK : AECCT_ERR_DEVICE;
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
  char *ws = nullptr;
  if (w.total) {
    if (workspace_bytes < w.total) return AECCT_ERR_WORKSPACE_TOO_SMALL;
    if (!workspace) return AECCT_ERR_INVALID_ARG;
    const Span all{workspace, 1, (int64_t)w.total, 0};
    for (const Span &t : in)
      if (overlap(all, t)) return AECCT_ERR_INVALID_ARG;
    for (const Span &t : out)
      if (overlap(all, t)) return AECCT_ERR_INVALID_ARG;
    ws = (char *)align_up((size_t)(uintptr_t)workspace);
  }
  char *const dz = ws, *const cx = dz + w.dz, *const cw = cx + w.x, *const part_dx = cw + w.w, *const part_dw = part_dx + w.part_dx,
       *const sums = part_dw + w.part_dw;
  const hipStream_t s = (hipStream_t)stream;
  const bool turned = a->w_turned != 0;
  aecct::Factor x{a->x, a->ldx, true, false}, m{a->w, a->ldw, turned, false}, d{a->dy, a->lddy, false, false};
  aecct::Prepare prepare{};
  if (w.need_dz || a->dbias)
    prepare.slope = {(int)a->rows, (int)a->out, a->act, a->dy, a->z, a->lddy, a->ldz, w.need_dz ? dz : nullptr, w.lddz,
                     a->dbias ? (float *)sums : nullptr, (int)aecct::slope_blocks(a->rows, a->out)};
  if (w.pack_x) {
    prepare.pack[0] = {a->x, a->ldx, (int)a->rows, (int)a->in, cx, w.ldx};
    x = {cx, w.ldx, true, true};
  }
  if (w.pack_w) {
    prepare.pack[1] = {a->w, a->ldw, (int)lines, (int)across, cw, w.ldw};
    m = {cw, w.ldw, turned, true};
  }
  if (w.pack_dy) prepare.pack[2] = {a->dy, a->lddy, (int)a->rows, (int)a->out, dz, w.lddz};
  if (w.pack_dy || w.need_dz) d = {dz, w.lddz, false, true};
  if (aecct::launch_prepare(a->type, prepare, s) != hipSuccess) return AECCT_ERR_DEVICE;
  aecct::Gemm g[2];
  aecct::GemmPlan plan[2];
  int count = 0;
  if (a->dx && a->rows) {
    plan[count] = w.dx;
    g[count++] = {(int)a->rows, (int)a->in, (int)a->out, d, m,
                  {nullptr, nullptr, nullptr, 0.0f, 0, a->type, nullptr, nullptr, a->dx, 0, 0, a->lddx},
                  w.dx.part_bytes ? part_dx : nullptr, w.dx.splits};
  }
  if (a->dw) {
    aecct::Factor dt = d;
    dt.across = true;
    plan[count] = w.dw;
    g[count++] = {(int)a->in, (int)a->out, (int)a->rows, x, dt,
                  {nullptr, nullptr, nullptr, 0.0f, 0, a->dw_type, nullptr, nullptr, a->dw, 0, 0, a->lddw},
                  w.dw.part_bytes ? part_dw : nullptr, w.dw.splits};
  }
  if (aecct::launch_gemm(a->type, g, plan, count, s) != hipSuccess) return AECCT_ERR_DEVICE;
  aecct::Finish f{};
  for (int i = 0; i < count; ++i) f.g[i] = g[i];
  if (a->dbias) {
    f.part = (const float *)sums;
    f.blocks = (int)aecct::slope_blocks(a->rows, a->out);
    f.n = (int)a->out;
    f.out = a->dbias;
  }
  return aecct::launch_finish(a->type, f, s) == hipSuccess ? AECCT_OK : AECCT_ERR_DEVICE;
}

}  // extern "C"
