// Distillation from a teacher's top logits on gfx950.
//
// With p the softmax of the teacher's entries over the temperature tau and q
// that of the logits over the whole vocabulary,
//   loss = tau^2 (sum_k p_k log p_k - sum_k p_k z_{id_k} / tau + lse)
//   dlogits = dloss tau (q - p)
// so a row needs its log-sum-exp, the logits at the teacher's ids, and for the
// gradient one more pass over the row.

#include "model.hpp"

namespace rdf2v {
namespace {

constexpr int kThreads = 256;
constexpr float kInf = __builtin_huge_valf();

template <class Op>
__device__ __forceinline__ float block_reduce(float x, float *scratch, Op op) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) x = op(x, __shfl_xor(x, off, kWave));
  __syncthreads();
  if (lane_id() == 0) scratch[threadIdx.x / kWave] = x;
  __syncthreads();
  x = scratch[0];
#pragma unroll
  for (int i = 1; i < kThreads / kWave; ++i) x = op(x, scratch[i]);
  return x;
}
__device__ __forceinline__ float block_max(float x, float *scratch) {
  return block_reduce(x, scratch, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float block_add(float x, float *scratch) {
  return block_reduce(x, scratch, [](float a, float b) { return a + b; });
}

// One workgroup to a row.
template <class T>
__global__ __launch_bounds__(kThreads) void distill_kernel(DistillArgs a, int64_t first) {
  __shared__ float p[RDF2V_MAX_TEACHER_TOP];
  __shared__ float zk[RDF2V_MAX_TEACHER_TOP];
  __shared__ int32_t id[RDF2V_MAX_TEACHER_TOP];
  __shared__ float scratch[kThreads / kWave];
  const int64_t row = first + blockIdx.x;
  const T *z = static_cast<const T *>(a.logits) + row * a.stride;
  const float inv_tau = 1.0f / a.temperature;
  float top = -kInf;
  for (int k = threadIdx.x; k < a.top; k += kThreads) {
    int32_t i = a.ids[row * a.top + k];
    if (int64_t(i) >= a.vocab) {
      if (a.status != nullptr) atomicOr(a.status, RDF2V_STATUS_ID_OUT_OF_RANGE);
      i = -1;
    }
    const float t = a.teacher[row * a.top + k] * inv_tau;
    if (t == -kInf) i = -1;
    id[k] = i;
    p[k] = t;
    zk[k] = i >= 0 ? to_f32(z[i]) * inv_tau : 0.0f;
    if (i >= 0) top = fmaxf(top, t);
  }
  float any = 0.0f;
  for (int k = threadIdx.x; k < a.top; k += kThreads) any = id[k] >= 0 ? 1.0f : any;
  const bool valid = block_max(any, scratch) > 0.0f;
  T *dz = a.dlogits == nullptr ? nullptr : static_cast<T *>(a.dlogits) + row * a.dstride;
  if (!valid) {
    if (threadIdx.x == 0 && a.loss != nullptr) a.loss[row] = a.lse[row] = 0.0f;
    if (dz != nullptr)
      for (int64_t j = threadIdx.x; j < a.vocab; j += kThreads) dz[j] = from_f32<T>(0.0f);
    return;
  }
  top = block_max(top, scratch);
  float sum = 0.0f;
  for (int k = threadIdx.x; k < a.top; k += kThreads) sum += id[k] >= 0 ? expf(p[k] - top) : 0.0f;
  const float lse_t = top + logf(block_add(sum, scratch));
  float lse;
  if (a.loss != nullptr) {
    float m = -kInf, s = 0.0f;
    for (int64_t j = threadIdx.x; j < a.vocab; j += kThreads) m = fmaxf(m, to_f32(z[j]) * inv_tau);
    m = block_max(m, scratch);
    for (int64_t j = threadIdx.x; j < a.vocab; j += kThreads)
      s += m == -kInf ? 0.0f : expf(to_f32(z[j]) * inv_tau - m);
    s = block_add(s, scratch);
    lse = m == -kInf ? -kInf : m + logf(s);
    float loss = 0.0f;
    for (int k = threadIdx.x; k < a.top; k += kThreads) {
      const float log_p = p[k] - lse_t, pk = expf(log_p);
      if (id[k] >= 0) loss += pk * (log_p - (zk[k] == -kInf ? -kInf : zk[k] - lse));
    }
    loss = block_add(loss, scratch);
    if (threadIdx.x == 0) {
      a.loss[row] = a.temperature * a.temperature * loss;
      a.lse[row] = lse;
    }
  } else {
    lse = a.lse_in[row];
  }
  if (dz == nullptr) return;
  const float w = a.dloss[row] * a.temperature;
  for (int64_t j = threadIdx.x; j < a.vocab; j += kThreads) {
    const float x = to_f32(z[j]) * inv_tau;
    dz[j] = from_f32<T>(w * (x == -kInf ? 0.0f : expf(x - lse)));
  }
  __syncthreads();
  // every occurrence of an id writes the same value
  for (int k = threadIdx.x; k < a.top; k += kThreads) {
    if (id[k] < 0) continue;
    float pj = 0.0f;
    for (int m = 0; m < a.top; ++m)
      if (id[m] == id[k]) pj += expf(p[m] - lse_t);
    dz[id[k]] = from_f32<T>(w * ((zk[k] == -kInf ? 0.0f : expf(zk[k] - lse)) - pj));
  }
}

}  // namespace

size_t distill_workspace_bytes(int64_t, int64_t, int32_t, int32_t) { return 0; }

rdf2v_status launch_distill(const DistillArgs &a, void *, hipStream_t stream) {
  return for_each_launch(a.rows, kThreads, 1, [&](int64_t first, int64_t count) {
    if (a.dtype == RDF2V_BF16)
      distill_kernel<bf16><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(a, first);
    else
      distill_kernel<float><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(a, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

}  // namespace rdf2v
