// Launchers of the operators of a model's layers (causal convolution, selective
// scan, residual norm). The extern "C" entry points in layer_api.hip validate
// arguments and call the launchers, which only enqueue.
#pragma once

#include "model.hpp"

namespace rdf2v {

size_t causal_conv_backward_workspace_bytes(const rdf2v_conv &a);
rdf2v_status launch_causal_conv(const rdf2v_conv &a, const rdf2v_tokens_view &x, const void *state, void *out,
                                void *state_out, int32_t *status_dev, hipStream_t stream);
rdf2v_status launch_causal_conv_backward(const rdf2v_conv &a, const rdf2v_tokens_view &x,
                                         const rdf2v_tokens_view &dout, const void *state, const void *dstate_out,
                                         void *dx, float *dweight, float *dbias, void *dstate, void *workspace,
                                         int32_t *status_dev, hipStream_t stream);
rdf2v_status launch_causal_conv_step(const rdf2v_conv &a, const rdf2v_tokens_view &x, const void *state,
                                     int64_t num_states, const int32_t *parents, void *out, void *state_out,
                                     int32_t *status_dev, hipStream_t stream);

// The inputs that the selective scan calls share; gate.data is null without a gate.
struct ScanInputs {
  rdf2v_tokens_view x, dt, gate;
  rdf2v_heads_view b, c;
};
size_t selective_scan_workspace_bytes(const rdf2v_scan &a, bool backward);
rdf2v_status launch_selective_scan(const rdf2v_scan &a, const ScanInputs &in, const float *state, void *out,
                                   float *state_out, void *workspace, int32_t *status_dev, hipStream_t stream);
rdf2v_status launch_selective_scan_backward(const rdf2v_scan &a, const ScanInputs &in, const rdf2v_tokens_view &dout,
                                            const float *state, const float *dstate_out,
                                            const rdf2v_scan_gradients &grads, void *workspace, int32_t *status_dev,
                                            hipStream_t stream);
rdf2v_status launch_selective_scan_step(const rdf2v_scan &a, const ScanInputs &in, const float *state,
                                        int64_t num_states, const int32_t *parents, void *out, float *state_out,
                                        int32_t *status_dev, hipStream_t stream);

// residual.data and dhidden.data may be null.
size_t residual_norm_backward_workspace_bytes(const rdf2v_norm &a);
rdf2v_status launch_residual_norm(const rdf2v_norm &a, const rdf2v_tokens_view &x, const rdf2v_tokens_view &residual,
                                  void *out, void *hidden, float *stats, int32_t *status_dev, hipStream_t stream);
rdf2v_status launch_residual_norm_backward(const rdf2v_norm &a, const rdf2v_tokens_view &x,
                                           const rdf2v_tokens_view &residual, const float *stats,
                                           const rdf2v_tokens_view &dout, const rdf2v_tokens_view &dhidden, void *dx,
                                           void *dresidual, float *dweight, float *dbias, float *dscale,
                                           void *workspace, int32_t *status_dev, hipStream_t stream);

}  // namespace rdf2v
