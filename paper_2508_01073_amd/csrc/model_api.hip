// extern "C" entry points of the operators over walk tokens: host-side argument
// checks, then the launchers. The declarations, argument meanings and error
// behaviour are in rdf2v.h.

#include <climits>
#include <cmath>
#include <initializer_list>
#include <utility>

#include "model.hpp"

namespace {

constexpr int64_t kInt32Limit = int64_t(1) << 31;
// Most elements of one array of a call: keeps every byte offset and size exact
// in 64 bits, and is far beyond any device memory.
constexpr int64_t kMaxElements = int64_t(1) << 56;
constexpr int64_t kMaxStride = int64_t(1) << 56;

bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool dtype_ok(int32_t dtype) { return dtype == RDF2V_F32 || dtype == RDF2V_BF16; }
size_t dtype_size(int32_t dtype) { return dtype == RDF2V_BF16 ? 2 : 4; }

// a * b for non-negative a and b, at most `most`; -1 beyond.
int64_t product(int64_t a, int64_t b, int64_t most) { return a >= 0 && (b == 0 || a <= most / b) ? a * b : -1; }

rdf2v_status check_sizes(const rdf2v_attention *a, bool step) {
  if (a == nullptr || a->rows < 0 || (!step && a->length < 0)) return RDF2V_ERR_INVALID_ARGUMENT;
  if (a->heads < 1 || a->heads > 65535 || a->kv_heads < 1 || a->heads % a->kv_heads != 0)
    return RDF2V_ERR_INVALID_ARGUMENT;
  if (a->dk < 1 || a->dk > RDF2V_MAX_HEAD_SIZE || a->dv < 1 || a->dv > RDF2V_MAX_HEAD_SIZE)
    return RDF2V_ERR_INVALID_ARGUMENT;
  if (!dtype_ok(a->dtype)) return RDF2V_ERR_INVALID_ARGUMENT;
  if (a->rows >= kInt32Limit || (!step && a->length >= kInt32Limit)) return RDF2V_ERR_TOO_LARGE;
  const int64_t per_row = int64_t(a->heads) * RDF2V_MAX_HEAD_SIZE * RDF2V_MAX_HEAD_SIZE;
  int64_t n = product(a->rows, per_row, kMaxElements);
  if (n >= 0 && !step) n = product(a->rows * a->length, int64_t(a->heads) * RDF2V_MAX_HEAD_SIZE, kMaxElements);
  return n < 0 ? RDF2V_ERR_TOO_LARGE : RDF2V_OK;
}

rdf2v_status check_attention(const rdf2v_attention *a, bool step) {
  const rdf2v_status st = check_sizes(a, step);
  if (st != RDF2V_OK) return st;
  if (!std::isfinite(a->scale)) return RDF2V_ERR_INVALID_ARGUMENT;
  if (a->rows > 0 && (a->log_decay == nullptr || !aligned(a->log_decay, 4))) return RDF2V_ERR_INVALID_ARGUMENT;
  if (!step && !aligned(a->len, 4)) return RDF2V_ERR_INVALID_ARGUMENT;
  return RDF2V_OK;
}

bool stride_ok(int64_t s) { return s > -kMaxStride && s < kMaxStride; }

bool view_ok(const rdf2v_heads_view *v, int32_t dtype, bool empty) {
  if (v == nullptr) return false;
  if (!stride_ok(v->row_stride) || !stride_ok(v->token_stride) || !stride_ok(v->head_stride)) return false;
  return (empty || v->data != nullptr) && aligned(v->data, dtype_size(dtype));
}

rdf2v_status check_workspace(const void *workspace, size_t bytes, size_t need) {
  if (need == 0) return RDF2V_OK;
  return workspace == nullptr || bytes < need || !aligned(workspace, 256) ? RDF2V_ERR_WORKSPACE : RDF2V_OK;
}

// Whether [a, a + an) and [b, b + bn) share a byte.
bool overlap(const void *a, size_t an, const void *b, size_t bn) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x <= y ? y - x < an : x - y < bn;
}

// An array of a call: where it lies, of how many bytes. Null or empty: it overlaps nothing.
struct Span {
  const void *data;
  size_t bytes;
};
bool overlap(const Span &a, const Span &b) {
  return a.data != nullptr && b.data != nullptr && a.bytes != 0 && b.bytes != 0 &&
         overlap(a.data, a.bytes, b.data, b.bytes);
}
bool same(const Span &a, const Span &b) { return a.data == b.data; }

// The bytes of a view as boxes inside boxes: count[i] boxes every step[i] bytes, those of the last level
// `bytes` long.
struct Boxes {
  __int128 step[3];
  int64_t count[3];
  __int128 bytes;
};

// Whether boxes of the levels from `level` on, the first of them at byte `at`, have a byte in [lo, hi).
bool boxes_reach(const Boxes &x, int level, __int128 at, __int128 lo, __int128 hi) {
  if (level == 3) return at < hi && at + x.bytes > lo;
  if (x.count[level] == 1) return boxes_reach(x, level + 1, at, lo, hi);
  __int128 size = x.bytes;  // from a box's first byte to its last
  for (int i = level + 1; i < 3; ++i) size += x.step[i] * (x.count[i] - 1);
  const __int128 all = size + x.step[level] * (x.count[level] - 1);
  if (at >= hi || at + all <= lo) return false;
  if (x.step[level] < size) return true;  // the boxes lie in one another: taken as one
  // Of the boxes that reach into the interval all but the first and the last lie in it.
  const __int128 first = at >= lo ? 0 : (lo - at) / x.step[level];
  __int128 last = (hi - 1 - at) / x.step[level];
  if (last > x.count[level] - 1) last = x.count[level] - 1;
  if (last - first > 1) return true;
  for (__int128 i = first; i <= last; ++i)
    if (boxes_reach(x, level + 1, at + i * x.step[level], lo, hi)) return true;
  return false;
}

// Whether a view of rows x tokens x heads of `size` values has a byte in an array. What lies between a view's
// values is not its own: another slice of the projection, say.
bool overlap(const rdf2v_heads_view &v, const rdf2v_attention &a, int heads, int size, const Span &out) {
  if (out.data == nullptr || out.bytes == 0 || a.rows == 0 || a.length == 0) return false;
  const int64_t value = int64_t(dtype_size(a.dtype));
  const int64_t strides[3] = {v.row_stride, v.token_stride, v.head_stride}, counts[3] = {a.rows, a.length, heads};
  Boxes x{};
  x.bytes = __int128(size) * value;
  __int128 at = __int128(reinterpret_cast<uintptr_t>(v.data));
  for (int i = 0; i < 3; ++i) {
    const __int128 step = __int128(strides[i]) * value;
    if (step < 0) at += step * (counts[i] - 1);  // from the lowest byte upwards
    x.step[i] = step < 0 ? -step : step;
    x.count[i] = step == 0 ? 1 : counts[i];
    if (x.count[i] == 1) x.step[i] = 0;
  }
  for (int i = 0; i < 2; ++i)  // the widest first
    for (int j = 0; j < 2 - i; ++j)
      if (x.step[j] < x.step[j + 1]) {
        std::swap(x.step[j], x.step[j + 1]);
        std::swap(x.count[j], x.count[j + 1]);
      }
  const __int128 lo = __int128(reinterpret_cast<uintptr_t>(out.data));
  return boxes_reach(x, 0, at, lo, lo + __int128(out.bytes));
}

size_t state_bytes(const rdf2v_attention &a) { return size_t(a.rows) * a.heads * a.dk * a.dv * 4; }
size_t head_bytes(const rdf2v_attention &a, int heads, int size) {
  return size_t(a.rows) * a.length * heads * size * dtype_size(a.dtype);
}

// Whether a view has a byte in one of the outputs.
bool reads(const rdf2v_heads_view &v, const rdf2v_attention &a, int heads, int size, std::initializer_list<Span> outs) {
  for (const Span &out : outs)
    if (overlap(v, a, heads, size, out)) return true;
  return false;
}

}  // namespace

RDF2V_API size_t rdf2v_decay_attention_workspace_size(const rdf2v_attention *a) {
  return check_sizes(a, false) == RDF2V_OK ? rdf2v::decay_attention_workspace_bytes(*a, false) : 0;
}

RDF2V_API size_t rdf2v_decay_attention_backward_workspace_size(const rdf2v_attention *a) {
  return check_sizes(a, false) == RDF2V_OK ? rdf2v::decay_attention_workspace_bytes(*a, true) : 0;
}

RDF2V_API rdf2v_status rdf2v_decay_attention(const rdf2v_attention *a, const rdf2v_heads_view *q,
                                             const rdf2v_heads_view *k, const rdf2v_heads_view *v,
                                             const float *state, void *out, float *state_out, void *workspace,
                                             size_t workspace_bytes, int32_t *status_dev, void *stream) {
  rdf2v_status st = check_attention(a, false);
  if (st != RDF2V_OK) return st;
  const bool empty = a->rows == 0 || a->length == 0;
  if (!view_ok(q, a->dtype, empty) || !view_ok(k, a->dtype, empty) || !view_ok(v, a->dtype, empty))
    return RDF2V_ERR_INVALID_ARGUMENT;
  if ((!empty && out == nullptr) || !aligned(out, dtype_size(a->dtype)) || !aligned(state, 4) ||
      !aligned(state_out, 4))
    return RDF2V_ERR_INVALID_ARGUMENT;
  st = check_workspace(workspace, workspace_bytes, rdf2v::decay_attention_workspace_bytes(*a, false));
  if (st != RDF2V_OK) return st;
  if (a->rows == 0) return RDF2V_OK;
  const size_t states = state_bytes(*a);
  const Span o = {out, head_bytes(*a, a->heads, a->dv)}, s = {state, states}, so = {state_out, states};
  if (overlap(o, s) || overlap(o, so) || (overlap(s, so) && !same(s, so))) return RDF2V_ERR_INVALID_ARGUMENT;
  if (reads(*q, *a, a->heads, a->dk, {o, so}) || reads(*k, *a, a->kv_heads, a->dk, {o, so}) ||
      reads(*v, *a, a->kv_heads, a->dv, {o, so}))
    return RDF2V_ERR_INVALID_ARGUMENT;
  return rdf2v::launch_decay_attention(*a, *q, *k, *v, state, out, state_out, workspace, status_dev,
                                       static_cast<hipStream_t>(stream));
}

RDF2V_API rdf2v_status rdf2v_decay_attention_backward(const rdf2v_attention *a, const rdf2v_heads_view *q,
                                                      const rdf2v_heads_view *k, const rdf2v_heads_view *v,
                                                      const rdf2v_heads_view *dout, const float *state,
                                                      const float *dstate_out, void *dq, void *dk, void *dv,
                                                      float *dstate, void *workspace, size_t workspace_bytes,
                                                      int32_t *status_dev, void *stream) {
  rdf2v_status st = check_attention(a, false);
  if (st != RDF2V_OK) return st;
  const bool empty = a->rows == 0 || a->length == 0;
  if (!view_ok(q, a->dtype, empty) || !view_ok(k, a->dtype, empty) || !view_ok(v, a->dtype, empty) ||
      !view_ok(dout, a->dtype, empty))
    return RDF2V_ERR_INVALID_ARGUMENT;
  if (!empty && (dq == nullptr || dk == nullptr || dv == nullptr)) return RDF2V_ERR_INVALID_ARGUMENT;
  const size_t size = dtype_size(a->dtype);
  if (!aligned(dq, size) || !aligned(dk, size) || !aligned(dv, size) || !aligned(state, 4) ||
      !aligned(dstate_out, 4) || !aligned(dstate, 4))
    return RDF2V_ERR_INVALID_ARGUMENT;
  st = check_workspace(workspace, workspace_bytes, rdf2v::decay_attention_workspace_bytes(*a, true));
  if (st != RDF2V_OK) return st;
  if (a->rows == 0) return RDF2V_OK;
  const size_t states = state_bytes(*a);
  const Span s = {state, states}, dso = {dstate_out, states}, ds = {dstate, states},
             gq = {dq, head_bytes(*a, a->heads, a->dk)}, gk = {dk, head_bytes(*a, a->kv_heads, a->dk)},
             gv = {dv, head_bytes(*a, a->kv_heads, a->dv)};
  if (overlap(gq, gk) || overlap(gq, gv) || overlap(gk, gv) || overlap(ds, s) ||
      (overlap(ds, dso) && !same(ds, dso)))
    return RDF2V_ERR_INVALID_ARGUMENT;
  for (const Span *g : {&gq, &gk, &gv})
    if (overlap(*g, s) || overlap(*g, dso) || overlap(*g, ds)) return RDF2V_ERR_INVALID_ARGUMENT;
  if (reads(*q, *a, a->heads, a->dk, {gq, gk, gv, ds}) || reads(*k, *a, a->kv_heads, a->dk, {gq, gk, gv, ds}) ||
      reads(*v, *a, a->kv_heads, a->dv, {gq, gk, gv, ds}) || reads(*dout, *a, a->heads, a->dv, {gq, gk, gv, ds}))
    return RDF2V_ERR_INVALID_ARGUMENT;
  return rdf2v::launch_decay_attention_backward(*a, *q, *k, *v, *dout, state, dstate_out, dq, dk, dv, dstate,
                                                workspace, status_dev, static_cast<hipStream_t>(stream));
}

RDF2V_API rdf2v_status rdf2v_decay_attention_step(const rdf2v_attention *a, const rdf2v_heads_view *q,
                                                  const rdf2v_heads_view *k, const rdf2v_heads_view *v,
                                                  const float *state, int64_t num_states, const int32_t *parents,
                                                  void *out, float *state_out, int32_t *status_dev, void *stream) {
  const rdf2v_status st = check_attention(a, true);
  if (st != RDF2V_OK) return st;
  const bool empty = a->rows == 0;
  if (!view_ok(q, a->dtype, empty) || !view_ok(k, a->dtype, empty) || !view_ok(v, a->dtype, empty))
    return RDF2V_ERR_INVALID_ARGUMENT;
  if (num_states < 0 || (parents == nullptr && num_states != a->rows)) return RDF2V_ERR_INVALID_ARGUMENT;
  if (num_states >= kInt32Limit ||
      product(num_states, int64_t(a->heads) * a->dk * a->dv, kMaxElements) < 0)
    return RDF2V_ERR_TOO_LARGE;
  if (empty) return RDF2V_OK;
  if (out == nullptr || state_out == nullptr || (num_states > 0 && state == nullptr))
    return RDF2V_ERR_INVALID_ARGUMENT;
  if (!aligned(out, dtype_size(a->dtype)) || !aligned(state, 4) || !aligned(state_out, 4) || !aligned(parents, 4))
    return RDF2V_ERR_INVALID_ARGUMENT;
  const size_t state_bytes = size_t(a->heads) * a->dk * a->dv * 4;
  if ((parents != nullptr || state != state_out) &&
      overlap(state, num_states * state_bytes, state_out, a->rows * state_bytes))
    return RDF2V_ERR_INVALID_ARGUMENT;
  return rdf2v::launch_decay_attention_step(*a, *q, *k, *v, state, num_states, parents, out, state_out, status_dev,
                                            static_cast<hipStream_t>(stream));
}

namespace {

rdf2v_status check_beam_sizes(int64_t groups, int32_t beams, int64_t vocab, int32_t num_out) {
  if (groups < 0 || beams < 1 || beams > RDF2V_MAX_BEAMS || num_out < 1 || num_out > RDF2V_MAX_BEAMS || vocab < 1)
    return RDF2V_ERR_INVALID_ARGUMENT;
  return vocab >= kInt32Limit || groups >= kInt32Limit / beams ? RDF2V_ERR_TOO_LARGE : RDF2V_OK;
}

}  // namespace

RDF2V_API size_t rdf2v_beam_select_workspace_size(int64_t groups, int32_t beams, int64_t vocab, int32_t num_out) {
  if (check_beam_sizes(groups, beams, vocab, num_out) != RDF2V_OK) return 0;
  return rdf2v::beam_select_workspace_bytes(groups, beams, vocab, num_out);
}

RDF2V_API rdf2v_status rdf2v_beam_select(const void *logits, int64_t logits_stride, int32_t dtype,
                                         const float *scores, const int32_t *finished, int64_t groups, int32_t beams,
                                         int64_t vocab, int32_t num_out, float *scores_out, int32_t *tokens_out,
                                         int32_t *parents_out, void *workspace, size_t workspace_bytes,
                                         int32_t *status_dev, void *stream) {
  rdf2v_status st = check_beam_sizes(groups, beams, vocab, num_out);
  if (st != RDF2V_OK) return st;
  if (!dtype_ok(dtype) || logits_stride < vocab) return RDF2V_ERR_INVALID_ARGUMENT;
  if (product(groups * beams, logits_stride, kMaxElements) < 0) return RDF2V_ERR_TOO_LARGE;
  if (groups == 0) return RDF2V_OK;
  if (logits == nullptr || scores == nullptr || scores_out == nullptr || tokens_out == nullptr ||
      parents_out == nullptr)
    return RDF2V_ERR_INVALID_ARGUMENT;
  if (!aligned(logits, dtype_size(dtype)) || !aligned(scores, 4) || !aligned(finished, 4) ||
      !aligned(scores_out, 4) || !aligned(tokens_out, 4) || !aligned(parents_out, 4))
    return RDF2V_ERR_INVALID_ARGUMENT;
  // rows of a group are read after other groups have been written
  const size_t in_bytes = size_t(groups) * beams * 4, out_bytes = size_t(groups) * num_out * 4;
  if ((scores != scores_out || num_out != beams) && overlap(scores, in_bytes, scores_out, out_bytes))
    return RDF2V_ERR_INVALID_ARGUMENT;
  st = check_workspace(workspace, workspace_bytes,
                       rdf2v::beam_select_workspace_bytes(groups, beams, vocab, num_out));
  if (st != RDF2V_OK) return st;
  return rdf2v::launch_beam_select(logits, logits_stride, dtype, scores, finished, groups, beams, vocab, num_out,
                                   scores_out, tokens_out, parents_out, workspace, status_dev,
                                   static_cast<hipStream_t>(stream));
}

RDF2V_API rdf2v_status rdf2v_beam_reorder(const void *src, int64_t num_src, int64_t row_bytes, const int32_t *parents,
                                          int64_t num_rows, void *dst, int32_t *status_dev, void *stream) {
  if (num_src < 0 || num_rows < 0 || row_bytes < 0) return RDF2V_ERR_INVALID_ARGUMENT;
  if (num_src >= kInt32Limit || num_rows >= kInt32Limit || product(num_src, row_bytes, kMaxElements) < 0 ||
      product(num_rows, row_bytes, kMaxElements) < 0)
    return RDF2V_ERR_TOO_LARGE;
  if (num_rows == 0 || row_bytes == 0) return RDF2V_OK;
  if ((num_src > 0 && src == nullptr) || parents == nullptr || dst == nullptr || !aligned(parents, 4))
    return RDF2V_ERR_INVALID_ARGUMENT;
  if (overlap(src, size_t(num_src) * row_bytes, dst, size_t(num_rows) * row_bytes))
    return RDF2V_ERR_INVALID_ARGUMENT;
  return rdf2v::launch_beam_reorder(src, num_src, row_bytes, parents, num_rows, dst, status_dev,
                                    static_cast<hipStream_t>(stream));
}

namespace {

rdf2v_status check_distill_sizes(int64_t rows, int64_t vocab, int32_t top, int32_t dtype) {
  if (rows < 0 || vocab < 1 || top < 0 || top > RDF2V_MAX_TEACHER_TOP || !dtype_ok(dtype))
    return RDF2V_ERR_INVALID_ARGUMENT;
  return rows >= kInt32Limit || vocab >= kInt32Limit ? RDF2V_ERR_TOO_LARGE : RDF2V_OK;
}

rdf2v_status check_distill(const rdf2v::DistillArgs &a) {
  const rdf2v_status st = check_distill_sizes(a.rows, a.vocab, a.top, a.dtype);
  if (st != RDF2V_OK) return st;
  if (!std::isfinite(a.temperature) || !(a.temperature > 0.0f)) return RDF2V_ERR_INVALID_ARGUMENT;
  if (a.stride < a.vocab || (a.dlogits != nullptr && a.dstride < a.vocab)) return RDF2V_ERR_INVALID_ARGUMENT;
  if (product(a.rows, a.stride, kMaxElements) < 0 ||
      (a.dlogits != nullptr && product(a.rows, a.dstride, kMaxElements) < 0))
    return RDF2V_ERR_TOO_LARGE;
  if (a.rows == 0) return RDF2V_OK;
  if (a.logits == nullptr || (a.top > 0 && (a.ids == nullptr || a.teacher == nullptr)))
    return RDF2V_ERR_INVALID_ARGUMENT;
  const size_t size = dtype_size(a.dtype);
  if (!aligned(a.logits, size) || !aligned(a.dlogits, size) || !aligned(a.ids, 4) || !aligned(a.teacher, 4) ||
      !aligned(a.dloss, 4) || !aligned(a.loss, 4) || !aligned(a.lse, 4) || !aligned(a.lse_in, 4))
    return RDF2V_ERR_INVALID_ARGUMENT;
  // in place element by element, or apart
  if (a.dlogits != nullptr && (a.dlogits != a.logits || a.dstride != a.stride) &&
      overlap(a.logits, ((a.rows - 1) * a.stride + a.vocab) * size, a.dlogits,
              ((a.rows - 1) * a.dstride + a.vocab) * size))
    return RDF2V_ERR_INVALID_ARGUMENT;
  return RDF2V_OK;
}

}  // namespace

RDF2V_API size_t rdf2v_distill_workspace_size(int64_t rows, int64_t vocab, int32_t top, int32_t dtype) {
  if (check_distill_sizes(rows, vocab, top, dtype) != RDF2V_OK) return 0;
  return rdf2v::distill_workspace_bytes(rows, vocab, top, dtype);
}

RDF2V_API rdf2v_status rdf2v_distill_loss(const void *logits, int64_t logits_stride, int32_t dtype,
                                          const int32_t *ids, const float *teacher, int64_t rows, int64_t vocab,
                                          int32_t top, float temperature, float *loss, float *lse,
                                          const float *dloss, void *dlogits, int64_t dlogits_stride, void *workspace,
                                          size_t workspace_bytes, int32_t *status_dev, void *stream) {
  if ((dloss == nullptr) != (dlogits == nullptr) && rows > 0) return RDF2V_ERR_INVALID_ARGUMENT;
  if ((loss == nullptr || lse == nullptr) && rows > 0) return RDF2V_ERR_INVALID_ARGUMENT;
  const rdf2v::DistillArgs a{logits, ids,           teacher,        dloss, nullptr, loss, lse,   dlogits,
                             status_dev, logits_stride, dlogits_stride, rows,  vocab,   top,  dtype, temperature};
  rdf2v_status st = check_distill(a);
  if (st != RDF2V_OK) return st;
  st = check_workspace(workspace, workspace_bytes, rdf2v::distill_workspace_bytes(rows, vocab, top, dtype));
  if (st != RDF2V_OK) return st;
  if (rows == 0) return RDF2V_OK;
  return rdf2v::launch_distill(a, workspace, static_cast<hipStream_t>(stream));
}

RDF2V_API rdf2v_status rdf2v_distill_loss_backward(const void *logits, int64_t logits_stride, int32_t dtype,
                                                   const int32_t *ids, const float *teacher, int64_t rows,
                                                   int64_t vocab, int32_t top, float temperature, const float *lse,
                                                   const float *dloss, void *dlogits, int64_t dlogits_stride,
                                                   void *workspace, size_t workspace_bytes, int32_t *status_dev,
                                                   void *stream) {
  if ((lse == nullptr || dloss == nullptr || dlogits == nullptr) && rows > 0) return RDF2V_ERR_INVALID_ARGUMENT;
  const rdf2v::DistillArgs a{logits, ids,           teacher,        dloss, lse,   nullptr, nullptr, dlogits,
                             status_dev, logits_stride, dlogits_stride, rows,  vocab, top,     dtype,   temperature};
  rdf2v_status st = check_distill(a);
  if (st != RDF2V_OK) return st;
  st = check_workspace(workspace, workspace_bytes, rdf2v::distill_workspace_bytes(rows, vocab, top, dtype));
  if (st != RDF2V_OK) return st;
  if (rows == 0) return RDF2V_OK;
  return rdf2v::launch_distill(a, workspace, static_cast<hipStream_t>(stream));
}
