// extern "C" entry points of the operators of a model's layers: host-side
// argument checks, then the launchers. The declarations, argument meanings and
// error behaviour are in rdf2v.h.

#include "checks.hpp"
#include "layer.hpp"

using namespace rdf2v;

namespace {

rdf2v_heads_view one_head(const rdf2v_tokens_view &v) { return {v.data, v.row_stride, v.token_stride, 0}; }

bool view_ok(const rdf2v_tokens_view *v, int32_t dtype, bool empty) {
  if (v == nullptr) return false;
  const rdf2v_heads_view h = one_head(*v);
  return rdf2v::view_ok(&h, dtype, empty);
}

// What a call reads and writes.
class Arrays {
 public:
  void view(const rdf2v_tokens_view &v, int64_t rows, int64_t length, int64_t channels, int32_t dtype) {
    view(one_head(v), rows, length, 1, channels, dtype);
  }
  void view(const rdf2v_heads_view &v, int64_t rows, int64_t length, int64_t heads, int64_t size, int32_t dtype) {
    views_[num_views_++] = ViewBoxes(v, rows, length, heads, size, dtype);
  }
  void in(const void *data, size_t bytes) { ins_[num_ins_++] = {data, bytes}; }
  void out(const void *data, size_t bytes) { outs_[num_outs_++] = {data, bytes}; }

  // Whether an output shares a byte with an input or another output, but for `may` lying where `over` does.
  bool clash(const void *may = nullptr, const void *over = nullptr) const {
    for (int i = 0; i < num_outs_; ++i) {
      for (int j = 0; j < i; ++j)
        if (overlap(outs_[i], outs_[j])) return true;
      for (int j = 0; j < num_ins_; ++j) {
        const bool same = may != nullptr && may == over && outs_[i].data == may && ins_[j].data == over &&
                          outs_[i].bytes == ins_[j].bytes;
        if (!same && overlap(outs_[i], ins_[j])) return true;
      }
      for (int j = 0; j < num_views_; ++j)
        if (views_[j].reach(outs_[i])) return true;
    }
    return false;
  }

 private:
  ViewBoxes views_[8];
  Span ins_[12], outs_[12];
  int num_views_ = 0, num_ins_ = 0, num_outs_ = 0;
};

// Of rows and length that a call takes, and as many values of `wide` for each token.
rdf2v_status check_rows(int64_t rows, int64_t length, int64_t wide) {
  if (rows < 0 || length < 0) return RDF2V_ERR_INVALID_ARGUMENT;
  if (rows >= kInt32Limit || length >= kInt32Limit) return RDF2V_ERR_TOO_LARGE;
  return product(rows * (length + 1), wide, kMaxElements) < 0 ? RDF2V_ERR_TOO_LARGE : RDF2V_OK;
}

bool num_states_ok(int64_t num_states, int64_t rows, const int32_t *parents) {
  return num_states >= 0 && (parents != nullptr || num_states == rows);
}

// ---- causal convolution ---------------------------------------------------

rdf2v_status check_conv_sizes(const rdf2v_conv *a, bool step) {
  if (a == nullptr || a->channels < 1 || a->width < 1 || a->width > RDF2V_MAX_CONV_WIDTH || !dtype_ok(a->dtype))
    return RDF2V_ERR_INVALID_ARGUMENT;
  return check_rows(a->rows, step ? 1 : a->length, int64_t(a->channels) * RDF2V_MAX_CONV_WIDTH * 2);
}

rdf2v_status check_conv(const rdf2v_conv *a, bool step) {
  const rdf2v_status st = check_conv_sizes(a, step);
  if (st != RDF2V_OK) return st;
  if ((a->rows > 0 && a->weight == nullptr) || !aligned(a->weight, 4) || !aligned(a->bias, 4))
    return RDF2V_ERR_INVALID_ARGUMENT;
  return step || aligned(a->len, 4) ? RDF2V_OK : RDF2V_ERR_INVALID_ARGUMENT;
}

size_t conv_state_bytes(const rdf2v_conv &a, int64_t rows) {
  return size_t(rows) * (a.width - 1) * a.channels * dtype_size(a.dtype);
}

void conv_parameters(Arrays &all, const rdf2v_conv &a, bool step) {
  all.in(a.weight, size_t(a.channels) * a.width * 4);
  all.in(a.bias, size_t(a.channels) * 4);
  if (!step) all.in(a.len, size_t(a.rows) * 4);
}

// ---- selective scan -------------------------------------------------------

rdf2v_status check_scan_sizes(const rdf2v_scan *a, bool step) {
  if (a == nullptr || a->channels < 1 || a->groups < 1 || a->groups > 65535 || a->channels % a->groups != 0 ||
      a->states < 1 || a->states > RDF2V_MAX_SCAN_STATES || !dtype_ok(a->dtype))
    return RDF2V_ERR_INVALID_ARGUMENT;
  if (a->channels > 1 << 28) return RDF2V_ERR_TOO_LARGE;
  return check_rows(a->rows, step ? 1 : a->length, int64_t(a->channels) * RDF2V_MAX_SCAN_STATES * 8);
}

rdf2v_status check_scan(const rdf2v_scan *a, const rdf2v_tokens_view *x, const rdf2v_tokens_view *dt,
                        const rdf2v_heads_view *b, const rdf2v_heads_view *c, const rdf2v_tokens_view *gate,
                        bool step) {
  const rdf2v_status st = check_scan_sizes(a, step);
  if (st != RDF2V_OK) return st;
  if ((a->rows > 0 && a->a == nullptr) || !aligned(a->a, 4) || !aligned(a->dt_bias, 4) || !aligned(a->skip, 4) ||
      (!step && !aligned(a->len, 4)))
    return RDF2V_ERR_INVALID_ARGUMENT;
  const bool empty = a->rows == 0 || (!step && a->length == 0);
  if (!view_ok(x, a->dtype, empty) || !view_ok(dt, a->dtype, empty) || !rdf2v::view_ok(b, a->dtype, empty) ||
      !rdf2v::view_ok(c, a->dtype, empty) || (gate != nullptr && !view_ok(gate, a->dtype, empty)))
    return RDF2V_ERR_INVALID_ARGUMENT;
  return RDF2V_OK;
}

ScanInputs scan_inputs(Arrays &all, const rdf2v_scan &a, const rdf2v_tokens_view &x, const rdf2v_tokens_view &dt,
                       const rdf2v_heads_view &b, const rdf2v_heads_view &c, const rdf2v_tokens_view *gate,
                       bool step) {
  const int64_t length = step ? 1 : a.length;
  ScanInputs in{x, dt, gate != nullptr ? *gate : rdf2v_tokens_view{nullptr, 0, 0}, b, c};
  all.view(x, a.rows, length, a.channels, a.dtype);
  all.view(dt, a.rows, length, a.channels, a.dtype);
  all.view(in.gate, a.rows, length, a.channels, a.dtype);
  all.view(b, a.rows, length, a.groups, a.states, a.dtype);
  all.view(c, a.rows, length, a.groups, a.states, a.dtype);
  all.in(a.a, size_t(a.channels) * a.states * 4);
  all.in(a.dt_bias, size_t(a.channels) * 4);
  all.in(a.skip, size_t(a.channels) * 4);
  if (!step) all.in(a.len, size_t(a.rows) * 4);
  return in;
}

size_t scan_state_bytes(const rdf2v_scan &a, int64_t rows) { return size_t(rows) * a.channels * a.states * 4; }

// ---- residual norm --------------------------------------------------------

rdf2v_status check_norm_sizes(const rdf2v_norm *a) {
  if (a == nullptr || a->channels < 1 || a->channels > RDF2V_MAX_NORM_CHANNELS || !dtype_ok(a->dtype) ||
      (a->residual_dtype != a->dtype && a->residual_dtype != RDF2V_F32))
    return RDF2V_ERR_INVALID_ARGUMENT;
  return check_rows(a->rows, a->length, a->channels);
}

rdf2v_status check_norm(const rdf2v_norm *a, const rdf2v_tokens_view *x, const rdf2v_tokens_view *residual) {
  const rdf2v_status st = check_norm_sizes(a);
  if (st != RDF2V_OK) return st;
  if (!std::isfinite(a->eps) || a->eps < 0.0f || !(a->drop >= 0.0) || !(a->drop < 1.0 - 0x1p-32) || a->row_begin < 0 ||
      a->row_begin > INT64_MAX - a->rows)
    return RDF2V_ERR_INVALID_ARGUMENT;
  const bool empty = a->rows == 0 || a->length == 0;
  if ((!empty && a->weight == nullptr) || !aligned(a->weight, 4) || !aligned(a->bias, 4) || !aligned(a->scale, 4) ||
      !aligned(a->seed_offset, 8) || !aligned(a->len, 4))
    return RDF2V_ERR_INVALID_ARGUMENT;
  if (!view_ok(x, a->dtype, empty) || (residual != nullptr && !view_ok(residual, a->residual_dtype, empty)))
    return RDF2V_ERR_INVALID_ARGUMENT;
  return RDF2V_OK;
}

void norm_inputs(Arrays &all, const rdf2v_norm &a, const rdf2v_tokens_view &x, const rdf2v_tokens_view &residual) {
  all.view(x, a.rows, a.length, a.channels, a.dtype);
  all.view(residual, a.rows, a.length, a.channels, a.residual_dtype);
  all.in(a.weight, size_t(a.channels) * 4);
  all.in(a.bias, size_t(a.channels) * 4);
  all.in(a.scale, size_t(a.channels) * 4);
  all.in(a.seed_offset, 8);
  all.in(a.len, size_t(a.rows) * 4);
}

}  // namespace

RDF2V_API size_t rdf2v_causal_conv_backward_workspace_size(const rdf2v_conv *a) {
  return check_conv_sizes(a, false) == RDF2V_OK ? causal_conv_backward_workspace_bytes(*a) : 0;
}

RDF2V_API rdf2v_status rdf2v_causal_conv(const rdf2v_conv *a, const rdf2v_tokens_view *x, const void *state, void *out,
                                         void *state_out, int32_t *status_dev, void *stream) {
  const rdf2v_status st = check_conv(a, false);
  if (st != RDF2V_OK) return st;
  const bool empty = a->rows == 0 || a->length == 0;
  const size_t size = dtype_size(a->dtype);
  if (!view_ok(x, a->dtype, empty) || (!empty && out == nullptr) || !aligned(out, size) || !aligned(state, size) ||
      !aligned(state_out, size))
    return RDF2V_ERR_INVALID_ARGUMENT;
  if (a->rows == 0) return RDF2V_OK;
  Arrays all;
  all.view(*x, a->rows, a->length, a->channels, a->dtype);
  all.in(state, conv_state_bytes(*a, a->rows));
  conv_parameters(all, *a, false);
  all.out(out, size_t(a->rows) * a->length * a->channels * size);
  all.out(state_out, conv_state_bytes(*a, a->rows));
  if (all.clash()) return RDF2V_ERR_INVALID_ARGUMENT;
  return launch_causal_conv(*a, *x, state, out, state_out, status_dev, static_cast<hipStream_t>(stream));
}

RDF2V_API rdf2v_status rdf2v_causal_conv_backward(const rdf2v_conv *a, const rdf2v_tokens_view *x,
                                                  const rdf2v_tokens_view *dout, const void *state,
                                                  const void *dstate_out, void *dx, float *dweight, float *dbias,
                                                  void *dstate, void *workspace, size_t workspace_bytes,
                                                  int32_t *status_dev, void *stream) {
  rdf2v_status st = check_conv(a, false);
  if (st != RDF2V_OK) return st;
  const bool empty = a->rows == 0 || a->length == 0;
  const size_t size = dtype_size(a->dtype);
  if (!view_ok(x, a->dtype, empty) || !view_ok(dout, a->dtype, empty) || (!empty && dx == nullptr) ||
      dweight == nullptr || !aligned(dx, size) || !aligned(dweight, 4) || !aligned(dbias, 4) ||
      !aligned(state, size) || !aligned(dstate_out, size) || !aligned(dstate, size))
    return RDF2V_ERR_INVALID_ARGUMENT;
  st = check_workspace(workspace, workspace_bytes, causal_conv_backward_workspace_bytes(*a));
  if (st != RDF2V_OK) return st;
  Arrays all;
  all.view(*x, a->rows, a->length, a->channels, a->dtype);
  all.view(*dout, a->rows, a->length, a->channels, a->dtype);
  all.in(state, conv_state_bytes(*a, a->rows));
  all.in(dstate_out, conv_state_bytes(*a, a->rows));
  conv_parameters(all, *a, false);
  all.out(dx, size_t(a->rows) * a->length * a->channels * size);
  all.out(dweight, size_t(a->channels) * a->width * 4);
  all.out(dbias, size_t(a->channels) * 4);
  all.out(dstate, conv_state_bytes(*a, a->rows));
  if (all.clash()) return RDF2V_ERR_INVALID_ARGUMENT;
  return launch_causal_conv_backward(*a, *x, *dout, state, dstate_out, dx, dweight, dbias, dstate, workspace,
                                     status_dev, static_cast<hipStream_t>(stream));
}

RDF2V_API rdf2v_status rdf2v_causal_conv_step(const rdf2v_conv *a, const rdf2v_tokens_view *x, const void *state,
                                              int64_t num_states, const int32_t *parents, void *out, void *state_out,
                                              int32_t *status_dev, void *stream) {
  const rdf2v_status st = check_conv(a, true);
  if (st != RDF2V_OK) return st;
  const bool empty = a->rows == 0, held = a->width > 1;
  const size_t size = dtype_size(a->dtype);
  if (!view_ok(x, a->dtype, empty) || !num_states_ok(num_states, a->rows, parents)) return RDF2V_ERR_INVALID_ARGUMENT;
  if (num_states >= kInt32Limit || product(num_states, int64_t(a->channels) * a->width, kMaxElements) < 0)
    return RDF2V_ERR_TOO_LARGE;
  if (empty) return RDF2V_OK;
  if (out == nullptr || (held && (state_out == nullptr || (num_states > 0 && state == nullptr))) ||
      !aligned(out, size) || !aligned(state, size) || !aligned(state_out, size) || !aligned(parents, 4))
    return RDF2V_ERR_INVALID_ARGUMENT;
  Arrays all;
  all.view(*x, a->rows, 1, a->channels, a->dtype);
  all.in(state, conv_state_bytes(*a, num_states));
  all.in(parents, size_t(a->rows) * 4);
  conv_parameters(all, *a, true);
  all.out(out, size_t(a->rows) * a->channels * size);
  all.out(state_out, conv_state_bytes(*a, a->rows));
  if (parents == nullptr ? all.clash(state_out, state) : all.clash()) return RDF2V_ERR_INVALID_ARGUMENT;
  return launch_causal_conv_step(*a, *x, state, num_states, parents, out, state_out, status_dev,
                                 static_cast<hipStream_t>(stream));
}

RDF2V_API size_t rdf2v_selective_scan_workspace_size(const rdf2v_scan *a) {
  return check_scan_sizes(a, false) == RDF2V_OK ? selective_scan_workspace_bytes(*a, false) : 0;
}

RDF2V_API size_t rdf2v_selective_scan_backward_workspace_size(const rdf2v_scan *a) {
  return check_scan_sizes(a, false) == RDF2V_OK ? selective_scan_workspace_bytes(*a, true) : 0;
}

RDF2V_API rdf2v_status rdf2v_selective_scan(const rdf2v_scan *a, const rdf2v_tokens_view *x,
                                            const rdf2v_tokens_view *dt, const rdf2v_heads_view *b,
                                            const rdf2v_heads_view *c, const rdf2v_tokens_view *gate,
                                            const float *state, void *out, float *state_out, void *workspace,
                                            size_t workspace_bytes, int32_t *status_dev, void *stream) {
  rdf2v_status st = check_scan(a, x, dt, b, c, gate, false);
  if (st != RDF2V_OK) return st;
  const size_t size = dtype_size(a->dtype);
  if ((a->rows > 0 && a->length > 0 && out == nullptr) || !aligned(out, size) || !aligned(state, 4) ||
      !aligned(state_out, 4))
    return RDF2V_ERR_INVALID_ARGUMENT;
  st = check_workspace(workspace, workspace_bytes, selective_scan_workspace_bytes(*a, false));
  if (st != RDF2V_OK) return st;
  if (a->rows == 0) return RDF2V_OK;
  Arrays all;
  const ScanInputs in = scan_inputs(all, *a, *x, *dt, *b, *c, gate, false);
  all.in(state, scan_state_bytes(*a, a->rows));
  all.out(out, size_t(a->rows) * a->length * a->channels * size);
  all.out(state_out, scan_state_bytes(*a, a->rows));
  if (all.clash(state_out, state)) return RDF2V_ERR_INVALID_ARGUMENT;
  return launch_selective_scan(*a, in, state, out, state_out, workspace, status_dev,
                               static_cast<hipStream_t>(stream));
}

RDF2V_API rdf2v_status rdf2v_selective_scan_backward(const rdf2v_scan *a, const rdf2v_tokens_view *x,
                                                     const rdf2v_tokens_view *dt, const rdf2v_heads_view *b,
                                                     const rdf2v_heads_view *c, const rdf2v_tokens_view *gate,
                                                     const rdf2v_tokens_view *dout, const float *state,
                                                     const float *dstate_out, const rdf2v_scan_gradients *grads,
                                                     void *workspace, size_t workspace_bytes, int32_t *status_dev,
                                                     void *stream) {
  rdf2v_status st = check_scan(a, x, dt, b, c, gate, false);
  if (st != RDF2V_OK) return st;
  const bool empty = a->rows == 0 || a->length == 0;
  if (!view_ok(dout, a->dtype, empty) || grads == nullptr || grads->da == nullptr) return RDF2V_ERR_INVALID_ARGUMENT;
  const rdf2v_scan_gradients &g = *grads;
  const size_t size = dtype_size(a->dtype);
  if (!empty && (g.dx == nullptr || g.ddt == nullptr || g.db == nullptr || g.dc == nullptr ||
                 (g.dgate == nullptr) != (gate == nullptr)))
    return RDF2V_ERR_INVALID_ARGUMENT;
  for (const void *p : {g.dx, g.ddt, g.db, g.dc, g.dgate})
    if (!aligned(p, size)) return RDF2V_ERR_INVALID_ARGUMENT;
  for (const float *p : {state, dstate_out, static_cast<const float *>(g.da), static_cast<const float *>(g.ddt_bias),
                         static_cast<const float *>(g.dskip), static_cast<const float *>(g.dstate)})
    if (!aligned(p, 4)) return RDF2V_ERR_INVALID_ARGUMENT;
  st = check_workspace(workspace, workspace_bytes, selective_scan_workspace_bytes(*a, true));
  if (st != RDF2V_OK) return st;
  Arrays all;
  const ScanInputs in = scan_inputs(all, *a, *x, *dt, *b, *c, gate, false);
  all.view(*dout, a->rows, a->length, a->channels, a->dtype);
  all.in(state, scan_state_bytes(*a, a->rows));
  all.in(dstate_out, scan_state_bytes(*a, a->rows));
  const size_t wide = size_t(a->rows) * a->length * a->channels * size,
               narrow = size_t(a->rows) * a->length * a->groups * a->states * size;
  all.out(g.dx, wide);
  all.out(g.ddt, wide);
  all.out(g.dgate, wide);
  all.out(g.db, narrow);
  all.out(g.dc, narrow);
  all.out(g.da, size_t(a->channels) * a->states * 4);
  all.out(g.ddt_bias, size_t(a->channels) * 4);
  all.out(g.dskip, size_t(a->channels) * 4);
  all.out(g.dstate, scan_state_bytes(*a, a->rows));
  if (all.clash(g.dstate, dstate_out)) return RDF2V_ERR_INVALID_ARGUMENT;
  return launch_selective_scan_backward(*a, in, *dout, state, dstate_out, g, workspace, status_dev,
                                        static_cast<hipStream_t>(stream));
}

RDF2V_API rdf2v_status rdf2v_selective_scan_step(const rdf2v_scan *a, const rdf2v_tokens_view *x,
                                                 const rdf2v_tokens_view *dt, const rdf2v_heads_view *b,
                                                 const rdf2v_heads_view *c, const rdf2v_tokens_view *gate,
                                                 const float *state, int64_t num_states, const int32_t *parents,
                                                 void *out, float *state_out, int32_t *status_dev, void *stream) {
  const rdf2v_status st = check_scan(a, x, dt, b, c, gate, true);
  if (st != RDF2V_OK) return st;
  if (!num_states_ok(num_states, a->rows, parents)) return RDF2V_ERR_INVALID_ARGUMENT;
  if (num_states >= kInt32Limit || product(num_states, int64_t(a->channels) * a->states, kMaxElements) < 0)
    return RDF2V_ERR_TOO_LARGE;
  if (a->rows == 0) return RDF2V_OK;
  const size_t size = dtype_size(a->dtype);
  if (out == nullptr || state_out == nullptr || (num_states > 0 && state == nullptr) || !aligned(out, size) ||
      !aligned(state, 4) || !aligned(state_out, 4) || !aligned(parents, 4))
    return RDF2V_ERR_INVALID_ARGUMENT;
  Arrays all;
  const ScanInputs in = scan_inputs(all, *a, *x, *dt, *b, *c, gate, true);
  all.in(state, scan_state_bytes(*a, num_states));
  all.in(parents, size_t(a->rows) * 4);
  all.out(out, size_t(a->rows) * a->channels * size);
  all.out(state_out, scan_state_bytes(*a, a->rows));
  if (parents == nullptr ? all.clash(state_out, state) : all.clash()) return RDF2V_ERR_INVALID_ARGUMENT;
  return launch_selective_scan_step(*a, in, state, num_states, parents, out, state_out, status_dev,
                                    static_cast<hipStream_t>(stream));
}

RDF2V_API size_t rdf2v_residual_norm_backward_workspace_size(const rdf2v_norm *a) {
  return check_norm_sizes(a) == RDF2V_OK ? residual_norm_backward_workspace_bytes(*a) : 0;
}

RDF2V_API rdf2v_status rdf2v_residual_norm(const rdf2v_norm *a, const rdf2v_tokens_view *x,
                                           const rdf2v_tokens_view *residual, void *out, void *hidden, float *stats,
                                           int32_t *status_dev, void *stream) {
  const rdf2v_status st = check_norm(a, x, residual);
  if (st != RDF2V_OK) return st;
  const size_t size = dtype_size(a->dtype), wide = dtype_size(a->residual_dtype);
  if (!aligned(out, size) || !aligned(hidden, wide) || !aligned(stats, 4)) return RDF2V_ERR_INVALID_ARGUMENT;
  if (a->rows == 0 || a->length == 0) return RDF2V_OK;
  if (out == nullptr) return RDF2V_ERR_INVALID_ARGUMENT;
  const rdf2v_tokens_view from = residual != nullptr ? *residual : rdf2v_tokens_view{nullptr, 0, 0};
  Arrays all;
  norm_inputs(all, *a, *x, from);
  const size_t tokens = size_t(a->rows) * a->length;
  all.out(out, tokens * a->channels * size);
  all.out(hidden, tokens * a->channels * wide);
  all.out(stats, tokens * 8);
  if (all.clash()) return RDF2V_ERR_INVALID_ARGUMENT;
  return launch_residual_norm(*a, *x, from, out, hidden, stats, status_dev, static_cast<hipStream_t>(stream));
}

RDF2V_API rdf2v_status rdf2v_residual_norm_backward(const rdf2v_norm *a, const rdf2v_tokens_view *x,
                                                    const rdf2v_tokens_view *residual, const float *stats,
                                                    const rdf2v_tokens_view *dout, const rdf2v_tokens_view *dhidden,
                                                    void *dx, void *dresidual, float *dweight, float *dbias,
                                                    float *dscale, void *workspace, size_t workspace_bytes,
                                                    int32_t *status_dev, void *stream) {
  rdf2v_status st = check_norm(a, x, residual);
  if (st != RDF2V_OK) return st;
  const bool empty = a->rows == 0 || a->length == 0;
  const size_t size = dtype_size(a->dtype), wide = dtype_size(a->residual_dtype);
  if (!view_ok(dout, a->dtype, empty) || (dhidden != nullptr && !view_ok(dhidden, a->residual_dtype, empty)) ||
      (!empty && (stats == nullptr || dx == nullptr)) || dweight == nullptr || !aligned(stats, 4) ||
      !aligned(dx, size) || !aligned(dresidual, wide) || !aligned(dweight, 4) || !aligned(dbias, 4) ||
      !aligned(dscale, 4))
    return RDF2V_ERR_INVALID_ARGUMENT;
  st = check_workspace(workspace, workspace_bytes, residual_norm_backward_workspace_bytes(*a));
  if (st != RDF2V_OK) return st;
  const rdf2v_tokens_view none = {nullptr, 0, 0}, from = residual != nullptr ? *residual : none,
                          dh = dhidden != nullptr ? *dhidden : none;
  Arrays all;
  norm_inputs(all, *a, *x, from);
  all.view(*dout, a->rows, a->length, a->channels, a->dtype);
  all.view(dh, a->rows, a->length, a->channels, a->residual_dtype);
  const size_t tokens = size_t(a->rows) * a->length, each = size_t(a->channels) * 4;
  all.in(stats, tokens * 8);
  all.out(dx, tokens * a->channels * size);
  all.out(dresidual, tokens * a->channels * wide);
  all.out(dweight, each);
  all.out(dbias, each);
  all.out(dscale, each);
  if (all.clash()) return RDF2V_ERR_INVALID_ARGUMENT;
  return launch_residual_norm_backward(*a, *x, from, stats, *dout, dh, dx, dresidual, dweight, dbias, dscale,
                                       workspace, status_dev, static_cast<hipStream_t>(stream));
}
