// Entry points of the gradient norm, clipping and the Adam update over lists of tensors: argument checks, the
// tables of the launches, the launches.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include <hip/hip_runtime.h>

#include "../../include/aecct.h"
#include "update.h"

namespace {

using namespace aecct;

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

constexpr int64_t kMaxCount = (int64_t)1 << 40;   // values of a tensor
constexpr int kMaxUnits = 1 << 30;                // of a launch

int64_t type_size(int32_t t) { return t == AECCT_F32 ? 4 : 2; }
bool tensor_ok(const aecct_tensor &t) {
  return t.count >= 0 && t.count <= kMaxCount && (t.data || t.count == 0) &&
         (t.type == AECCT_F32 || t.type == AECCT_BF16 || t.type == AECCT_F16);
}
bool list_ok(const aecct_tensor *t, int32_t n) {
  if (n < 0 || (n > 0 && !t)) return false;
  for (int i = 0; i < n; ++i)
    if (!tensor_ok(t[i])) return false;
  return true;
}
bool same_counts(const aecct_tensor *a, const aecct_tensor *b, int32_t n) {
  for (int i = 0; i < n; ++i)
    if (a[i].count != b[i].count) return false;
  return true;
}

// Whether a tensor of the written lists shares a byte with another tensor of any of the lists (the read list may
// overlap itself).
struct Span {
  uintptr_t begin, end;
  bool written;
};
bool span_of(const aecct_tensor &t, bool written, Span &s) {
  s = Span{(uintptr_t)t.data, (uintptr_t)t.data + (uintptr_t)(t.count * type_size(t.type)), written};
  return t.count > 0;
}
bool conflict(std::vector<Span> &v) {
  // lists usually come in ascending order of addresses already, one after the other
  if (!std::is_sorted(v.begin(), v.end(), [](const Span &a, const Span &b) { return a.begin < b.begin; }))
    std::sort(v.begin(), v.end(), [](const Span &a, const Span &b) { return a.begin < b.begin; });
  uintptr_t any = 0, written = 0;   // the furthest ends so far
  for (const Span &s : v) {
    if (s.begin < written || (s.written && s.begin < any)) return true;
    any = std::max(any, s.end);
    if (s.written) written = std::max(written, s.end);
  }
  return false;
}

int64_t units_of(int64_t count) { return (count + kUnit - 1) / kUnit; }

// Calls f(first, end) for every run of tensors that one launch takes.
template <class F>
hipError_t for_launches(const aecct_tensor *t, int32_t n, int most, F f) {
  for (int i = 0; i < n;) {
    int k = i;
    int64_t units = 0;
    while (k < n && k - i < most && units + units_of(t[k].count) <= kMaxUnits) units += units_of(t[k++].count);
    const hipError_t e = f(i, k);
    if (e != hipSuccess) return e;
    i = k;
  }
  return hipSuccess;
}
template <class Table>
void add_units(Table &t, const aecct_tensor &x) {
  t.count[t.n] = x.count;
  t.type[t.n] = (uint8_t)x.type;
  t.unit0[t.n + 1] = t.unit0[t.n] + (int)units_of(x.count);
  ++t.n;
}

size_t sum_launches(int32_t n) { return ((size_t)n + kSumTensors - 1) / kSumTensors; }
size_t need_bytes(int32_t n) { return 2 * kAlign + std::max<size_t>(1, sum_launches(n)) * kMaxSumBlocks * sizeof(double); }

struct Work {
  int64_t *next;
  double *part;
};
Work work_of(void *workspace) {
  unsigned char *w = (unsigned char *)align_up((size_t)(uintptr_t)workspace);
  return Work{(int64_t *)w, (double *)(w + kAlign)};
}

hipError_t sums(const aecct_tensor *g, int32_t n, double *part, int &parts, hipStream_t s) {
  parts = 0;
  return for_launches(g, n, kSumTensors, [&](int i, int k) {
    SumTable t;
    t.n = 0;
    t.unit0[0] = 0;
    for (; i < k; ++i)
      if (g[i].count) {
        t.g[t.n] = g[i].data;
        add_units(t, g[i]);
      }
    if (!t.n) return hipSuccess;
    const int blocks = std::min(t.unit0[t.n], kMaxSumBlocks);
    const hipError_t e = launch_sum_squares(t, part + parts, blocks, s);
    parts += blocks;
    return e;
  });
}

aecct_status st(hipError_t e) { return e == hipSuccess ? AECCT_OK : AECCT_ERR_DEVICE; }
aecct_status device_cus(int &cus) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    return AECCT_ERR_DEVICE;
  return AECCT_OK;
}

}  // namespace

extern "C" {

aecct_status aecct_update_workspace_size(int32_t n, size_t *bytes) {
  if (!bytes || n < 0) return AECCT_ERR_INVALID_ARG;
  *bytes = need_bytes(n);
  return AECCT_OK;
}

aecct_status aecct_grad_norm(const aecct_tensor *grads, int32_t n, float *norm, void *workspace, size_t workspace_bytes,
                             void *stream) {
  if (!list_ok(grads, n) || !norm) return AECCT_ERR_INVALID_ARG;
  const uintptr_t at = (uintptr_t)norm;
  for (int i = 0; i < n; ++i) {
    Span x;
    if (span_of(grads[i], false, x) && x.begin < at + sizeof(float) && at < x.end) return AECCT_ERR_INVALID_ARG;
  }
  if (workspace_bytes < need_bytes(n)) return AECCT_ERR_WORKSPACE_TOO_SMALL;
  if (!workspace) return AECCT_ERR_INVALID_ARG;
  const Work w = work_of(workspace);
  hipStream_t s = (hipStream_t)stream;
  int parts = 0;
  const hipError_t e = sums(grads, n, w.part, parts, s);
  return st(e != hipSuccess ? e : launch_norm(w.part, parts, norm, s));
}

aecct_status aecct_grad_clip(const aecct_tensor *grads, const aecct_tensor *out, int32_t n, double max_norm, float *norm,
                             void *workspace, size_t workspace_bytes, void *stream) {
  if (!out) out = grads;
  if (!list_ok(grads, n) || !list_ok(out, n) || !same_counts(grads, out, n) || !norm || !(max_norm >= 0))
    return AECCT_ERR_INVALID_ARG;
  if (workspace_bytes < need_bytes(n)) return AECCT_ERR_WORKSPACE_TOO_SMALL;
  if (!workspace) return AECCT_ERR_INVALID_ARG;
  try {
    std::vector<Span> v;
    v.reserve(2 * (size_t)n + 1);
    Span x;
    for (int i = 0; i < n; ++i)
      if (span_of(out[i], true, x)) v.push_back(x);
    for (int i = 0; i < n; ++i)
      if (!(grads[i].data == out[i].data && grads[i].type == out[i].type) && span_of(grads[i], false, x)) v.push_back(x);
    v.push_back(Span{(uintptr_t)norm, (uintptr_t)(norm + 1), true});
    if (conflict(v)) return AECCT_ERR_INVALID_ARG;
  } catch (const std::bad_alloc &) {
    return AECCT_ERR_OUT_OF_MEMORY;
  }
  int cus = 0;
  if (device_cus(cus) != AECCT_OK) return AECCT_ERR_DEVICE;
  const Work w = work_of(workspace);
  hipStream_t s = (hipStream_t)stream;
  int parts = 0;
  hipError_t e = sums(grads, n, w.part, parts, s);
  if (e != hipSuccess) return st(e);
  if (!parts) return st(launch_norm(w.part, 0, norm, s));
  return st(for_launches(grads, n, kClipTensors, [&](int i, int k) {
    ClipTable t;
    t.n = 0;
    t.unit0[0] = 0;
    for (; i < k; ++i)
      if (grads[i].count) {
        t.g[t.n] = grads[i].data;
        t.out[t.n] = out[i].data;
        t.out_type[t.n] = (uint8_t)out[i].type;
        add_units(t, grads[i]);
      }
    return t.n ? launch_clip(t, w.part, parts, max_norm, norm, cus, s) : hipSuccess;
  }));
}

aecct_status aecct_adam_step(const aecct_tensor *params, const aecct_tensor *m, const aecct_tensor *v,
                             const aecct_tensor *grads, const aecct_tensor *copies, int32_t n,
                             const aecct_adam_options *opt, int64_t *step, float *norm, void *workspace,
                             size_t workspace_bytes, void *stream) {
  if (!list_ok(params, n) || !list_ok(m, n) || !list_ok(v, n) || !list_ok(grads, n) || (copies && !list_ok(copies, n)) ||
      !opt || !step)
    return AECCT_ERR_INVALID_ARG;
  if (!same_counts(params, m, n) || !same_counts(params, v, n) || !same_counts(params, grads, n)) return AECCT_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i)
    if (params[i].type != AECCT_F32 || m[i].type != AECCT_F32 || v[i].type != AECCT_F32 ||
        (copies && copies[i].count && copies[i].count != params[i].count))
      return AECCT_ERR_INVALID_ARG;
  if ((!opt->lr_device && !std::isfinite(opt->lr)) || !(opt->beta1 >= 0 && opt->beta1 < 1) ||
      !(opt->beta2 >= 0 && opt->beta2 < 1) || !(opt->eps >= 0 && std::isfinite(opt->eps)) ||
      !std::isfinite(opt->weight_decay) || !(opt->max_norm >= 0))
    return AECCT_ERR_INVALID_ARG;
  if (workspace_bytes < need_bytes(n)) return AECCT_ERR_WORKSPACE_TOO_SMALL;
  if (!workspace) return AECCT_ERR_INVALID_ARG;
  try {
    std::vector<Span> all;
    all.reserve(5 * (size_t)n + 2);
    Span x;
    const aecct_tensor *lists[5] = {params, m, v, copies, grads};
    for (int l = 0; l < 5; ++l)
      for (int i = 0; lists[l] && i < n; ++i)
        if (span_of(lists[l][i], l < 4, x)) all.push_back(x);
    all.push_back(Span{(uintptr_t)step, (uintptr_t)(step + 1), true});
    if (norm) all.push_back(Span{(uintptr_t)norm, (uintptr_t)(norm + 1), true});
    if (conflict(all)) return AECCT_ERR_INVALID_ARG;
  } catch (const std::bad_alloc &) {
    return AECCT_ERR_OUT_OF_MEMORY;
  }
  int cus = 0;
  if (device_cus(cus) != AECCT_OK) return AECCT_ERR_DEVICE;
  const Work w = work_of(workspace);
  hipStream_t s = (hipStream_t)stream;
  int parts = 0;
  hipError_t e = launch_next_step(step, w.next, s);
  if (e == hipSuccess && (opt->max_norm > 0 || norm)) e = sums(grads, n, w.part, parts, s);
  if (e != hipSuccess) return st(e);
  const AdamScalars o{opt->lr, opt->beta1, opt->beta2, opt->eps, opt->weight_decay, opt->max_norm, opt->lr_device};
  bool first = true;
  auto launch = [&](const AdamTable &t) {
    const hipError_t r = launch_adam(t, w.part, parts, o, w.next, first ? step : nullptr, first ? norm : nullptr, cus, s);
    first = false;
    return r;
  };
  e = for_launches(params, n, kAdamTensors, [&](int i, int k) {
    AdamTable t;
    t.n = 0;
    t.unit0[0] = 0;
    for (; i < k; ++i)
      if (params[i].count) {
        t.g[t.n] = grads[i].data;
        t.p[t.n] = (float *)params[i].data;
        t.m[t.n] = (float *)m[i].data;
        t.v[t.n] = (float *)v[i].data;
        t.copy[t.n] = copies && copies[i].count ? copies[i].data : nullptr;
        t.copy_type[t.n] = copies ? (uint8_t)copies[i].type : 0;
        add_units(t, grads[i]);
      }
    return t.n ? launch(t) : hipSuccess;
  });
  if (e == hipSuccess && first) {   // no value at all: the step counts, the norm is 0
    AdamTable t;
    t.n = 0;
    t.unit0[0] = 0;
    e = launch(t);
    if (e == hipSuccess && norm) e = launch_norm(w.part, 0, norm, s);
  }
  return st(e);
}

}  // extern "C"
