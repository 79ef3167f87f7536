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

constexpr int64_t kMaxCount = (int64_t)1 << 40;   // values of a list: its sums then need no more launches than its ranges ask for
constexpr int64_t kMaxUnits = (int64_t)1 << 30;   // of a launch: a tensor of 2^40 values is as many units of 1024

int64_t type_size(int32_t t) { return t == AECCT_F32 ? 4 : 2; }
bool tensor_ok(const aecct_tensor &t) {
  return t.count >= 0 && t.count <= kMaxCount && (t.data || t.count == 0) &&
         (t.type == AECCT_F32 || t.type == AECCT_BF16 || t.type == AECCT_F16);
}
bool list_ok(const aecct_tensor *t, int32_t n) {
  if (n < 0 || (n > 0 && !t)) return false;
  int64_t count = 0;
  for (int i = 0; i < n; ++i)
    if (!tensor_ok(t[i]) || (count += t[i].count) > kMaxCount) return false;
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
struct Spans {
  std::vector<Span> v;
  explicit Spans(size_t most) { v.reserve(most); }
  static bool before(const Span &a, const Span &b) { return a.begin < b.begin; }
  // Adds a list (without tensors that are `but`'s own), which usually lies in ascending order already.
  void add(const aecct_tensor *t, int32_t n, bool written, const aecct_tensor *but = nullptr) {
    const size_t old = v.size();
    Span x;
    for (int i = 0; i < n; ++i)
      if (!(but && t[i].data == but[i].data && t[i].type == but[i].type) && span_of(t[i], written, x)) v.push_back(x);
    join(old);
  }
  void add(const void *p, size_t bytes, bool written = true) {
    v.push_back(Span{(uintptr_t)p, (uintptr_t)p + bytes, written});
    join(v.size() - 1);
  }
  void join(size_t old) {
    if (!std::is_sorted(v.begin() + old, v.end(), before)) std::sort(v.begin() + old, v.end(), before);
    if (old && old < v.size() && before(v[old], v[old - 1])) std::inplace_merge(v.begin(), v.begin() + old, v.end(), before);
  }
  bool meets(const void *p, size_t bytes) const {   // whether any span of the lists shares a byte with these
    const uintptr_t begin = (uintptr_t)p, end = begin + bytes;
    bool any = false;
    for (const Span &s : v) any |= s.begin < end && begin < s.end;
    return any;
  }
  bool conflict() const {
    uintptr_t any = 0, written = 0;   // the furthest ends so far
    for (const Span &s : v) {
      if (s.begin < written || (s.written && s.begin < any)) return true;
      any = std::max(any, s.end);
      if (s.written) written = std::max(written, s.end);
    }
    return false;
  }
};

// Whether tensor b follows a run of `count` values at a.
bool follows(const void *a, int64_t count, int32_t type, const aecct_tensor &b) {
  return b.type == type && (uintptr_t)a + (uintptr_t)(count * type_size(type)) == (uintptr_t)b.data;
}

// Fills tables with a list's tensors, one table a launch: extends(t, i) whether tensor i goes on where the table's last
// range ends, put(t, i) sets a new range's addresses, launch(t).
template <class Table, class Extends, class Put, class Launch>
hipError_t for_tables(const aecct_tensor *list, int32_t n, Extends extends, Put put, Launch launch) {
  const auto units_of = [](int64_t count, int type) { return (count + Table::unit_of(type) - 1) / Table::unit_of(type); };
  Table t;
  t.n = 0;
  t.unit0[0] = 0;
  for (int i = 0; i < n; ++i) {
    if (list[i].count == 0) continue;
    if (t.n && extends(t, i)) {
      const int64_t count = t.count[t.n - 1] + list[i].count, units = t.unit0[t.n - 1] + units_of(count, t.type[t.n - 1]);
      if (units <= kMaxUnits) {
        t.count[t.n - 1] = count;
        t.unit0[t.n] = (int)units;
        continue;
      }
    }
    if (t.n == Table::kMost || t.unit0[t.n] + units_of(list[i].count, list[i].type) > kMaxUnits) {
      const hipError_t e = launch(t);
      if (e != hipSuccess) return e;
      t.n = 0;
    }
    put(t, i);
    t.count[t.n] = list[i].count;
    t.type[t.n] = (uint8_t)list[i].type;
    t.unit0[t.n + 1] = t.unit0[t.n] + (int)units_of(list[i].count, list[i].type);
    ++t.n;
  }
  return t.n ? launch(t) : hipSuccess;
}

size_t sum_launches(int32_t n) { return ((size_t)n + kSumRanges - 1) / kSumRanges; }
size_t need_bytes(int32_t n) { return 2 * kAlign + std::max<size_t>(1, sum_launches(n)) * kMaxSumBlocks * sizeof(double); }

struct Work {
  AdamNow *now;
  double *part;
};
Work work_of(void *workspace) {
  unsigned char *w = (unsigned char *)align_up((size_t)(uintptr_t)workspace);
  return Work{(AdamNow *)w, (double *)(w + kAlign)};
}

// The norm's partial sums, and *w.now from *step if that is given.
hipError_t sums(const aecct_tensor *g, int32_t n, const Work &w, int &parts, bool alone, const int64_t *step,
                const AdamScalars &o, hipStream_t s) {
  parts = 0;
  using Table = SumTable<kSumRanges>;
  const hipError_t e = for_tables<Table>(
      g, n, [&](const Table &t, int i) { return follows(t.g[t.n - 1], t.count[t.n - 1], t.type[t.n - 1], g[i]); },
      [&](Table &t, int i) { t.g[t.n] = g[i].data; },
      [&](const Table &t) {
        const int blocks = std::min(t.unit0[t.n], kMaxSumBlocks);
        const hipError_t r = launch_sum_squares(t, w.part + parts, blocks, alone, step, step && !parts ? w.now : nullptr, o, s);
        parts += blocks;
        return r;
      });
  return e == hipSuccess && !parts && step ? launch_now(step, w.now, o, s) : e;
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
  const uintptr_t at = (uintptr_t)norm, ws = (uintptr_t)workspace, ws_end = ws + need_bytes(n);
  bool on_norm = false, on_ws = at < ws_end && ws < at + sizeof(float);
  for (int i = 0; i < n; ++i) {
    Span x;
    if (!span_of(grads[i], false, x)) continue;
    on_norm = on_norm || (x.begin < at + sizeof(float) && at < x.end);
    on_ws = on_ws || (x.begin < ws_end && ws < x.end);
  }
  if (on_norm) return AECCT_ERR_INVALID_ARG;
  if (workspace_bytes < need_bytes(n)) return AECCT_ERR_WORKSPACE_TOO_SMALL;
  if (!workspace || on_ws) return AECCT_ERR_INVALID_ARG;
  const Work w = work_of(workspace);
  hipStream_t s = (hipStream_t)stream;
  int parts = 0;
  const hipError_t e = sums(grads, n, w, parts, true, nullptr, AdamScalars{}, s);
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
    Spans v(2 * (size_t)n + 1);
    v.add(out, n, true);
    v.add(grads, n, false, out);
    v.add(norm, sizeof(float));
    if (v.conflict() || v.meets(workspace, need_bytes(n))) return AECCT_ERR_INVALID_ARG;
  } catch (const std::bad_alloc &) {
    return AECCT_ERR_OUT_OF_MEMORY;
  }
  int cus = 0;
  if (device_cus(cus) != AECCT_OK) return AECCT_ERR_DEVICE;
  const Work w = work_of(workspace);
  hipStream_t s = (hipStream_t)stream;
  int parts = 0;
  const hipError_t e = sums(grads, n, w, parts, false, nullptr, AdamScalars{}, s);
  if (e != hipSuccess) return st(e);
  if (!parts) return st(launch_norm(w.part, 0, norm, s));
  using Table = ClipTable<kClipRanges>;
  return st(for_tables<Table>(
      grads, n,
      [&](const Table &t, int i) {
        const int k = t.n - 1;
        return follows(t.g[k], t.count[k], t.type[k], grads[i]) && follows(t.out[k], t.count[k], t.out_type[k], out[i]);
      },
      [&](Table &t, int i) {
        t.g[t.n] = grads[i].data;
        t.out[t.n] = out[i].data;
        t.out_type[t.n] = (uint8_t)out[i].type;
      },
      [&](const Table &t) { return launch_clip(t, w.part, parts, max_norm, norm, cus, s); }));
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
    Spans spans(5 * (size_t)n + 3);
    spans.add(params, n, true);
    spans.add(m, n, true);
    spans.add(v, n, true);
    if (copies) spans.add(copies, n, true);
    spans.add(grads, n, false);
    spans.add(step, sizeof(int64_t));
    if (norm) spans.add(norm, sizeof(float));
    if (opt->lr_device) spans.add(opt->lr_device, sizeof(float), false);
    if (spans.conflict() || spans.meets(workspace, need_bytes(n))) return AECCT_ERR_INVALID_ARG;
  } catch (const std::bad_alloc &) {
    return AECCT_ERR_OUT_OF_MEMORY;
  }
  int cus = 0;
  if (device_cus(cus) != AECCT_OK) return AECCT_ERR_DEVICE;
  const Work w = work_of(workspace);
  hipStream_t s = (hipStream_t)stream;
  int parts = 0;
  const AdamScalars o{opt->lr, opt->beta1, opt->beta2, opt->eps, opt->weight_decay, opt->max_norm, opt->lr_device};
  hipError_t e = opt->max_norm > 0 || norm ? sums(grads, n, w, parts, false, step, o, s) : launch_now(step, w.now, o, s);
  if (e != hipSuccess) return st(e);
  using Table = AdamTable<kAdamRanges>;
  bool first = true;
  const auto launch = [&](const Table &t) {
    const hipError_t r = launch_adam(t, w.part, parts, o, w.now, first ? step : nullptr, first ? norm : nullptr, cus, s);
    first = false;
    return r;
  };
  const auto copy_of = [&](int i) { return copies && copies[i].count ? copies[i].data : nullptr; };
  e = for_tables<Table>(
      grads, n,
      [&](const Table &t, int i) {
        const int k = t.n - 1;
        const int64_t c = t.count[k];
        return follows(t.g[k], c, t.type[k], grads[i]) && follows(t.p[k], c, AECCT_F32, params[i]) &&
               follows(t.m[k], c, AECCT_F32, m[i]) && follows(t.v[k], c, AECCT_F32, v[i]) &&
               (t.copy[k] ? copy_of(i) && follows(t.copy[k], c, t.copy_type[k], copies[i]) : !copy_of(i));
      },
      [&](Table &t, int i) {
        t.g[t.n] = grads[i].data;
        t.p[t.n] = (float *)params[i].data;
        t.m[t.n] = (float *)m[i].data;
        t.v[t.n] = (float *)v[i].data;
        t.copy[t.n] = copy_of(i);
        t.copy_type[t.n] = copies ? (uint8_t)copies[i].type : 0;
      },
      launch);
  if (e == hipSuccess && first) {   // no value at all: the step counts, the norm is 0
    Table t;
    t.n = 0;
    t.unit0[0] = 0;
    e = launch(t);
    if (e == hipSuccess && norm) e = launch_norm(w.part, 0, norm, s);
  }
  return st(e);
}

}  // extern "C"
