// Entry points of cross attention and its gradient: argument checks, workspaces, launches.
#include <cmath>
#include <cstdint>

#include <hip/hip_runtime.h>

#include "../../include/aecct.h"
#include "attention.h"
#include "spans.h"

namespace {

using aecct::overlap;
using aecct::Span;

constexpr int64_t kMaxCount = (int64_t)1 << 30, kMaxSpan = (int64_t)1 << 56;   // no byte offset overflows
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 512;                      // of a grid
constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

bool type_ok(int32_t t) { return t == AECCT_F32 || t == AECCT_BF16 || t == AECCT_F16; }
int64_t type_size(int32_t t) { return t == AECCT_F32 ? 4 : 2; }

aecct_status check_sizes(int64_t batch, int64_t queries, int64_t keys, int32_t heads, int32_t kv_heads, int32_t d, int32_t type,
                         float scale, bool masked) {
  if (batch < 0 || queries < 0 || keys < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads || d < 1 || !type_ok(type))
    return AECCT_ERR_INVALID_ARG;
  if (!(scale > 0.0f) || !std::isfinite(scale)) return AECCT_ERR_INVALID_ARG;
  if (d > 256 || batch > kMaxCount || queries > kMaxCount || keys > kMaxCount || heads > (1 << 20)) return AECCT_ERR_UNSUPPORTED;
  // Threads of the largest grids: 256 for 32 rows of a pair or 128 keys (times the splits, which only few blocks take), 16 for a row's
  // terms, and with a mask, which all heads share, 64 for 32 queries and 128 keys.
  const __int128 rows = (__int128)(heads / kv_heads) * queries, pairs = (__int128)batch * kv_heads;
  const __int128 blocks = (rows + 31) / 32 * pairs, masks = masked ? ((__int128)queries + 31) / 32 * ((keys + 127) / 128 + 1) : 0;
  const __int128 keyed = ((__int128)keys + 127) / 128 * pairs;
  if (blocks > kMaxThreads / 256 || masks > kMaxThreads / 64 || keyed > kMaxThreads / 256 || rows * pairs > kMaxThreads / 16)
    return AECCT_ERR_UNSUPPORTED;
  return AECCT_OK;
}

// The memory of a [batch][length][heads][d] tensor, from its first value to its last.
struct Box {
  int64_t batch, length, heads, d;
};
struct Dim {
  int64_t n, stride;
};
// The dimensions longer than one, in the order of their strides.
int dims_of(const aecct_heads &t, const Box &n, Dim (&dims)[3]) {
  int count = 0;
  for (const Dim &x : {Dim{n.heads, t.head}, Dim{n.length, t.row}, Dim{n.batch, t.batch}}) {
    if (x.n <= 1) continue;
    int i = count++;
    for (; i > 0 && dims[i - 1].stride > x.stride; --i) dims[i] = dims[i - 1];
    dims[i] = x;
  }
  return count;
}
bool strides_ok(const aecct_heads &t, const Box &n, bool out) {
  if (!t.data || n.batch == 0 || n.length == 0) return true;
  if (t.batch < 0 || t.row < 0 || t.head < 0) return false;
  if (t.batch > kMaxSpan / n.batch || t.row > kMaxSpan / n.length || t.head > kMaxSpan / n.heads) return false;
  if (!out) return true;
  // An output's values lie apart: each step of a dimension goes over all of the ones inside it.
  Dim dims[3];
  const int count = dims_of(t, n, dims);
  int64_t reach = n.d;
  for (int i = 0; i < count; ++i) {
    if (dims[i].stride < reach) return false;
    reach += (dims[i].n - 1) * dims[i].stride;
  }
  return true;
}
Span span_of(const aecct_heads &t, const Box &n, int64_t size) {
  if (!t.data || n.batch == 0 || n.length == 0) return {nullptr, 0, 0, 0};
  return {t.data, 1, ((n.batch - 1) * t.batch + (n.length - 1) * t.row + (n.heads - 1) * t.head + n.d) * size, 0};
}
// Whether two outputs of one box may share a byte: their spans do, unless their strides are equal and they lie side by side at some
// dimension (as k and v of one projection do, or heads in turn): inside it one ends before the other begins, and each step
// of it and of those around it goes over both.
bool mix(const aecct_heads &s, const Span &x, const aecct_heads &t, const Span &y, const Box &n, int64_t size) {
  if (!overlap(x, y)) return false;
  Dim dims[3], others[3];
  const int count = dims_of(s, n, dims);
  (void)dims_of(t, n, others);
  for (int i = 0; i < count; ++i)
    if (dims[i].n != others[i].n || dims[i].stride != others[i].stride) return true;
  const int64_t off = (int64_t)(x.begin() <= y.begin() ? y.begin() - x.begin() : x.begin() - y.begin());
  int64_t reach = n.d * size;              // of one of them
  for (int at = 0; at < count && off >= reach; ++at) {
    int64_t both = off + reach;
    int i = at;
    for (; i < count && dims[i].stride * size >= both; ++i) both += (dims[i].n - 1) * dims[i].stride * size;
    if (i == count) return false;
    reach += (dims[at].n - 1) * dims[at].stride * size;
  }
  return true;
}

// Attention of at least this many operations, or on this many bytes of keys, first has tensors whose rows are no whole 16-byte pieces
// copied into such (2 x 1000 on 1500 keys of 177 fp16 268 -> 92 us, its gradient 419 -> 291; a launch of 5 us and the
// tensors read and written once more).
constexpr double kPackWork = 1e9, kPackBytes = 4e6;
bool worth_packing(int64_t batch, int64_t queries, int64_t keys, int32_t heads, int32_t kv_heads, int32_t d, int64_t size) {
  return 4.0 * batch * heads * queries * keys * d >= kPackWork || 2.0 * batch * keys * kv_heads * d * size >= kPackBytes;
}
// Bytes of a tensor's copy, 0 where it needs none.
size_t copy_bytes(bool worth, const aecct_heads &t, const Box &n, int64_t size) {
  if (!worth || n.length == 0 || !aecct::ragged_heads((int)size, t.batch, t.row, t.head, (int)n.d)) return 0;
  const int64_t e = 16 / size;
  return align_up((size_t)(n.batch * n.length * n.heads * ((n.d + e - 1) / e * e) * size));
}
// Has the copy made at `to` (bytes > 0), and takes it in the tensor's place.
void take_copy(aecct::PackHeads &job, aecct::Heads &t, const Box &n, int64_t size, const int32_t *lengths, char *to, size_t bytes) {
  if (!bytes) return;
  const int64_t e = 16 / size, line = (n.d + e - 1) / e * e;
  job.from = t;
  job.batch = n.batch, job.length = n.length, job.heads = (int)n.heads, job.d = (int)n.d, job.line = (int)line;
  job.lengths = lengths, job.to = to;
  t.p = to, t.batch = n.length * n.heads * line, t.row = n.heads * line, t.head = line, t.packed = true;
}

aecct::Heads heads_of(const aecct_heads &t) { return {t.data, t.batch, t.row, t.head}; }

}  // namespace

extern "C" {

aecct_status aecct_cross_attention_workspace_size(const aecct_cross_attention_args *a, size_t *bytes) {
  if (!a || !bytes) return AECCT_ERR_INVALID_ARG;
  const aecct_status s = check_sizes(a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, a->type, a->scale, a->mask);
  if (s != AECCT_OK) return s;
  const aecct::AttentionPlan p =
      aecct::plan_attention(a->type, a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, a->mask != nullptr);
  const int64_t size = type_size(a->type);
  const Box bk{a->batch, a->keys, a->kv_heads, a->d};
  const bool worth = worth_packing(a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, size);
  const size_t need = align_up(p.words) + align_up(p.flags) + align_up(p.part_o) + align_up(p.part_ml) +
                      copy_bytes(worth, a->k, bk, size) + copy_bytes(worth, a->v, bk, size);
  *bytes = need ? need + kAlign : 0;
  return AECCT_OK;
}

aecct_status aecct_cross_attention(const aecct_cross_attention_args *a, void *workspace, size_t workspace_bytes, void *stream) {
  if (!a) return AECCT_ERR_INVALID_ARG;
  const aecct_status st = check_sizes(a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, a->type, a->scale, a->mask);
  if (st != AECCT_OK) return st;
  if (a->batch == 0 || a->queries == 0) return AECCT_OK;
  if (!a->q.data || !a->o.data || (a->keys && (!a->k.data || !a->v.data))) return AECCT_ERR_INVALID_ARG;
  const Box bq{a->batch, a->queries, a->heads, a->d}, bk{a->batch, a->keys, a->kv_heads, a->d};
  if (!strides_ok(a->q, bq, false) || !strides_ok(a->k, bk, false) || !strides_ok(a->v, bk, false) || !strides_ok(a->o, bq, true))
    return AECCT_ERR_INVALID_ARG;
  const bool masked = a->mask && a->keys;
  if (masked && (a->ldmask < 0 || a->ldmask > kMaxSpan / a->queries)) return AECCT_ERR_INVALID_ARG;
  const int64_t size = type_size(a->type);
  const Span in[5] = {span_of(a->q, bq, size), span_of(a->k, bk, size), span_of(a->v, bk, size), {a->lengths, 1, 4 * a->batch, 0},
                      {masked ? a->mask : nullptr, 1, (a->queries - 1) * a->ldmask + a->keys, 0}};
  const Span o = span_of(a->o, bq, size), lse{a->lse, 1, 4 * a->batch * a->heads * a->queries, 0};
  if (overlap(o, lse)) return AECCT_ERR_INVALID_ARG;
  for (const Span &t : in)
    if (overlap(o, t) || overlap(lse, t)) return AECCT_ERR_INVALID_ARG;
  const aecct::AttentionPlan p = aecct::plan_attention(a->type, a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, masked);
  size_t need = 0;
  (void)aecct_cross_attention_workspace_size(a, &need);
  char *ws = nullptr;
  if (need) {
    if (workspace_bytes < need) return AECCT_ERR_WORKSPACE_TOO_SMALL;
    if (!workspace) return AECCT_ERR_INVALID_ARG;
    const Span w{workspace, 1, (int64_t)need, 0};
    for (const Span &t : in)
      if (overlap(w, t)) return AECCT_ERR_INVALID_ARG;
    if (overlap(w, o) || overlap(w, lse)) return AECCT_ERR_INVALID_ARG;
    ws = (char *)align_up((size_t)(uintptr_t)workspace);
  }
  aecct::Attention x{a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, a->scale, heads_of(a->q), heads_of(a->k),
                     heads_of(a->v), heads_of(a->o), a->lengths, masked ? a->mask : nullptr, a->ldmask, nullptr, nullptr, a->lse,
                     p.splits, nullptr, nullptr};
  x.words = (uint32_t *)ws;
  x.flags = (uint8_t *)ws + align_up(p.words);
  x.part_o = (float *)(x.flags + align_up(p.flags));
  x.part_ml = (float *)((char *)x.part_o + align_up(p.part_o));
  const bool worth = worth_packing(a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, size);
  const size_t ck = copy_bytes(worth, a->k, bk, size), cv = copy_bytes(worth, a->v, bk, size);
  char *const copies = (char *)x.part_ml + align_up(p.part_ml);
  aecct::PackHeadsAll jobs{};
  take_copy(jobs.t[0], x.k, bk, size, a->lengths, copies, ck);
  take_copy(jobs.t[1], x.v, bk, size, a->lengths, copies + ck, cv);
  if (aecct::launch_pack_heads(a->type, jobs, (hipStream_t)stream) != hipSuccess) return AECCT_ERR_DEVICE;
  return aecct::launch_attention(a->type, x, p, (hipStream_t)stream) == hipSuccess ? AECCT_OK : AECCT_ERR_DEVICE;
}

aecct_status aecct_cross_attention_grad_workspace_size(const aecct_cross_attention_grad_args *a, size_t *bytes) {
  if (!a || !bytes) return AECCT_ERR_INVALID_ARG;
  const aecct_status s = check_sizes(a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, a->type, a->scale, a->mask);
  if (s != AECCT_OK) return s;
  const aecct::AttentionGradPlan p =
      aecct::plan_attention_grad(a->type, a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, a->mask != nullptr);
  const int64_t size = type_size(a->type);
  const Box bq{a->batch, a->queries, a->heads, a->d}, bk{a->batch, a->keys, a->kv_heads, a->d};
  const bool worth = worth_packing(a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, size);
  const size_t need = align_up(p.words) + align_up(p.flags) + align_up(p.rows) + align_up(p.part) + align_up(p.part_q) +
                      copy_bytes(worth, a->k, bk, size) + copy_bytes(worth, a->v, bk, size) + copy_bytes(worth, a->q, bq, size) +
                      copy_bytes(worth, a->dout, bq, size);
  *bytes = need ? need + kAlign : 0;
  return AECCT_OK;
}

aecct_status aecct_cross_attention_grad(const aecct_cross_attention_grad_args *a, void *workspace, size_t workspace_bytes,
                                        void *stream) {
  if (!a) return AECCT_ERR_INVALID_ARG;
  const aecct_status st = check_sizes(a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, a->type, a->scale, a->mask);
  if (st != AECCT_OK) return st;
  if (a->batch == 0) return AECCT_OK;
  const bool some_q = a->queries > 0, some_k = a->keys > 0;
  if ((some_q && (!a->q.data || !a->o.data || !a->dout.data || !a->lse)) || (some_k && (!a->k.data || !a->v.data)))
    return AECCT_ERR_INVALID_ARG;
  if ((some_q && some_k && !a->dq.data && !a->dk.data) || (a->dk.data != nullptr) != (a->dv.data != nullptr))
    return AECCT_ERR_INVALID_ARG;
  const Box bq{a->batch, a->queries, a->heads, a->d}, bk{a->batch, a->keys, a->kv_heads, a->d};
  if (!strides_ok(a->q, bq, false) || !strides_ok(a->k, bk, false) || !strides_ok(a->v, bk, false) || !strides_ok(a->o, bq, false) ||
      !strides_ok(a->dout, bq, false) || !strides_ok(a->dq, bq, true) || !strides_ok(a->dk, bk, true) || !strides_ok(a->dv, bk, true))
    return AECCT_ERR_INVALID_ARG;
  const bool masked = a->mask && some_k && some_q;
  if (masked && (a->ldmask < 0 || a->ldmask > kMaxSpan / a->queries)) return AECCT_ERR_INVALID_ARG;
  const int64_t size = type_size(a->type);
  const Span in[8] = {span_of(a->q, bq, size), span_of(a->k, bk, size), span_of(a->v, bk, size), span_of(a->o, bq, size),
                      span_of(a->dout, bq, size), {a->lse, 1, 4 * a->batch * a->heads * a->queries, 0},
                      {a->lengths, 1, 4 * a->batch, 0}, {masked ? a->mask : nullptr, 1, (a->queries - 1) * a->ldmask + a->keys, 0}};
  const Span dq = span_of(a->dq, bq, size), dk = span_of(a->dk, bk, size), dv = span_of(a->dv, bk, size);
  if (overlap(dq, dk) || overlap(dq, dv) || mix(a->dk, dk, a->dv, dv, bk, size)) return AECCT_ERR_INVALID_ARG;
  for (const Span &t : in)
    if (overlap(dq, t) || overlap(dk, t) || overlap(dv, t)) return AECCT_ERR_INVALID_ARG;
  const aecct::AttentionGradPlan p =
      aecct::plan_attention_grad(a->type, a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, masked);
  size_t need = 0;
  (void)aecct_cross_attention_grad_workspace_size(a, &need);
  char *ws = nullptr;
  if (need) {
    if (workspace_bytes < need) return AECCT_ERR_WORKSPACE_TOO_SMALL;
    if (!workspace) return AECCT_ERR_INVALID_ARG;
    const Span w{workspace, 1, (int64_t)need, 0};
    for (const Span &t : in)
      if (overlap(w, t)) return AECCT_ERR_INVALID_ARG;
    if (overlap(w, dq) || overlap(w, dk) || overlap(w, dv)) return AECCT_ERR_INVALID_ARG;
    ws = (char *)align_up((size_t)(uintptr_t)workspace);
  }
  aecct::AttentionGrad x{};
  x.a = {a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, a->scale, heads_of(a->q), heads_of(a->k), heads_of(a->v),
         heads_of(a->o), a->lengths, masked ? a->mask : nullptr, a->ldmask, nullptr, nullptr, (float *)a->lse, 1, nullptr, nullptr};
  x.a.words = (uint32_t *)ws;
  x.a.flags = (uint8_t *)ws + align_up(p.words);
  x.rows = (float *)(x.a.flags + align_up(p.flags));
  x.splits = p.splits;
  x.part = p.part ? (float *)((char *)x.rows + align_up(p.rows)) : nullptr;
  x.splits_q = p.splits_q;
  x.part_q = (float *)((char *)x.rows + align_up(p.rows) + align_up(p.part));
  x.dout = heads_of(a->dout);
  x.dq = heads_of(a->dq);
  x.dk = heads_of(a->dk);
  x.dv = heads_of(a->dv);
  if (!some_k) x.dk.p = x.dv.p = nullptr;
  const bool worth = worth_packing(a->batch, a->queries, a->keys, a->heads, a->kv_heads, a->d, size);
  const size_t ck = copy_bytes(worth, a->k, bk, size), cv = copy_bytes(worth, a->v, bk, size), cq = copy_bytes(worth, a->q, bq, size),
               cd = copy_bytes(worth, a->dout, bq, size);
  char *const copies = (char *)x.part_q + align_up(p.part_q);
  aecct::PackHeadsAll jobs{};
  take_copy(jobs.t[0], x.a.k, bk, size, a->lengths, copies, ck);
  take_copy(jobs.t[1], x.a.v, bk, size, a->lengths, copies + ck, cv);
  take_copy(jobs.t[2], x.a.q, bq, size, nullptr, copies + ck + cv, cq);
  take_copy(jobs.t[3], x.dout, bq, size, nullptr, copies + ck + cv + cq, cd);
  if (aecct::launch_pack_heads(a->type, jobs, (hipStream_t)stream) != hipSuccess) return AECCT_ERR_DEVICE;
  return aecct::launch_attention_grad(a->type, x, (hipStream_t)stream) == hipSuccess ? AECCT_OK : AECCT_ERR_DEVICE;
}

}  // extern "C"
