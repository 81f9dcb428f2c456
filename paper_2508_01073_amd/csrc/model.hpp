// Helpers and launchers of the operators over walk tokens (decay attention,
// beam selection, distillation). The extern "C" entry points in model_api.hip
// validate arguments and call the launchers, which only enqueue.
#pragma once

#include "common.hpp"
#include "grid.hpp"

namespace rdf2v {

typedef __bf16 bf16;

// Values of the two element types as float32, and float32 rounded to them (to
// nearest even).
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16 x) { return float(x); }
template <class T>
__device__ __forceinline__ T from_f32(float x) {
  return T(x);
}

// ---- decay attention ------------------------------------------------------

size_t decay_attention_workspace_bytes(const rdf2v_attention &a, bool backward);
rdf2v_status launch_decay_attention(const rdf2v_attention &a, const rdf2v_heads_view &q, const rdf2v_heads_view &k,
                                    const rdf2v_heads_view &v, const float *state, void *out, float *state_out,
                                    void *workspace, int32_t *status_dev, hipStream_t stream);
rdf2v_status launch_decay_attention_backward(const rdf2v_attention &a, const rdf2v_heads_view &q,
                                             const rdf2v_heads_view &k, const rdf2v_heads_view &v,
                                             const rdf2v_heads_view &dout, const float *state,
                                             const float *dstate_out, void *dq, void *dk, void *dv, float *dstate,
                                             void *workspace, int32_t *status_dev, hipStream_t stream);
rdf2v_status launch_decay_attention_step(const rdf2v_attention &a, const rdf2v_heads_view &q,
                                         const rdf2v_heads_view &k, const rdf2v_heads_view &v, const float *state,
                                         int64_t num_states, const int32_t *parents, void *out, float *state_out,
                                         int32_t *status_dev, hipStream_t stream);

// ---- beam selection -------------------------------------------------------

size_t beam_select_workspace_bytes(int64_t groups, int32_t beams, int64_t vocab, int32_t num_out);
rdf2v_status launch_beam_select(const void *logits, int64_t stride, int32_t dtype, const float *scores,
                                const int32_t *finished, int64_t groups, int32_t beams, int64_t vocab,
                                int32_t num_out, float *scores_out, int32_t *tokens_out, int32_t *parents_out,
                                void *workspace, int32_t *status_dev, hipStream_t stream);
rdf2v_status launch_beam_reorder(const void *src, int64_t num_src, int64_t row_bytes, const int32_t *parents,
                                 int64_t num_rows, void *dst, int32_t *status_dev, hipStream_t stream);

// ---- distillation ---------------------------------------------------------

struct DistillArgs {
  const void *logits;
  const int32_t *ids;
  const float *teacher;
  const float *dloss;       // gradient wanted: not null, and dlogits too
  const float *lse_in;      // gradient alone: the row statistics of the loss call
  float *loss, *lse;        // loss wanted
  void *dlogits;
  int32_t *status;
  int64_t stride, dstride, rows, vocab;
  int32_t top, dtype;
  float temperature;
};
size_t distill_workspace_bytes(int64_t rows, int64_t vocab, int32_t top, int32_t dtype);
rdf2v_status launch_distill(const DistillArgs &a, void *workspace, hipStream_t stream);

}  // namespace rdf2v
