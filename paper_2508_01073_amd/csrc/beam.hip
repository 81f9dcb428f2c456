// Beam search's selection and the reordering of states on gfx950.
//
// Of a beam only its num_out largest logits can be chosen, so a row of logits
// is reduced to those and its log-sum-exp, and a group's beams are merged by
// total. Places are compared as (value descending, index ascending), a total
// order, so the choice does not depend on the order of the work.

#include "model.hpp"

namespace rdf2v {
namespace {

constexpr int kThreads = 256;
constexpr float kInf = __builtin_huge_valf();

// Descending (value, -index) as one unsigned number: larger is better.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t index) {
  const uint32_t b = __float_as_uint(x + 0.0f);  // -0 becomes +0
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return uint64_t(o) << 32 | (0xffffffffu - index);
}
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t o = uint32_t(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint32_t key_index(uint64_t key) { return 0xffffffffu - uint32_t(key); }

template <class V, class Op>
__device__ __forceinline__ V block_reduce(V x, V *scratch, Op op) {
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

// A logit that can be chosen, or -inf.
__device__ __forceinline__ float usable(float x, bool &bad) {
  if (x < kInf) return x;
  bad = true;
  return -kInf;
}

// One workgroup to a row: its log-sum-exp and its num_out best places.
template <class T>
__global__ __launch_bounds__(kThreads) void beam_rows_kernel(const T *logits, int64_t stride, const float *scores,
                                                             const int32_t *finished, int64_t vocab, int num_out,
                                                             float *lse, uint64_t *best, int32_t *status,
                                                             int64_t first) {
  __shared__ float fscratch[kThreads / kWave];
  __shared__ uint64_t kscratch[kThreads / kWave];
  const int64_t row = first + blockIdx.x;
  if (!(scores[row] > -kInf) || (finished != nullptr && finished[row] != 0)) return;
  const T *z = logits + row * stride;
  bool bad = false;
  float m = -kInf, s = 0.0f;
  for (int64_t j = threadIdx.x; j < vocab; j += kThreads) m = fmaxf(m, usable(to_f32(z[j]), bad));
  if (bad && status != nullptr) atomicOr(status, RDF2V_STATUS_BAD_VALUE);
  m = block_reduce(m, fscratch, [](float a, float b) { return fmaxf(a, b); });
  for (int64_t j = threadIdx.x; j < vocab; j += kThreads) {
    const float x = usable(to_f32(z[j]), bad);
    s += x == -kInf ? 0.0f : expf(x - m);
  }
  s = block_reduce(s, fscratch, [](float a, float b) { return a + b; });
  if (threadIdx.x == 0) lse[row] = m + logf(s);
  uint64_t last = ~uint64_t(0);
  for (int k = 0; k < num_out; ++k) {
    uint64_t key = 0;
    for (int64_t j = threadIdx.x; j < vocab; j += kThreads) {
      const float x = usable(to_f32(z[j]), bad);
      const uint64_t c = x == -kInf ? 0 : order_key(x, uint32_t(j));
      if (c < last && c > key) key = c;
    }
    last = block_reduce(key, kscratch, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
    if (threadIdx.x == 0) best[row * num_out + k] = last;
  }
}

// One workgroup to a group: its beams' candidates by total.
__global__ __launch_bounds__(kThreads) void beam_merge_kernel(const float *scores, const int32_t *finished, int beams,
                                                              int num_out, const float *lse, const uint64_t *best,
                                                              float *scores_out, int32_t *tokens_out,
                                                              int32_t *parents_out, int64_t first) {
  __shared__ float total[RDF2V_MAX_BEAMS * RDF2V_MAX_BEAMS];
  __shared__ uint64_t kscratch[kThreads / kWave];
  const int64_t group = first + blockIdx.x, row0 = group * beams;
  const int count = beams * num_out;
  for (int c = threadIdx.x; c < count; c += kThreads) {
    const int64_t row = row0 + c / num_out;
    const float score = scores[row];
    float t = -kInf;
    if (score > -kInf) {
      if (finished != nullptr && finished[row] != 0) {
        t = c % num_out == 0 ? score : -kInf;
      } else {
        const uint64_t key = best[row * num_out + c % num_out];
        if (key != 0) t = score + (key_value(key) - lse[row]);
      }
    }
    total[c] = t;
  }
  __syncthreads();
  uint64_t last = ~uint64_t(0);
  for (int k = 0; k < num_out; ++k) {
    uint64_t key = 0;
    for (int c = threadIdx.x; c < count; c += kThreads) {
      const uint64_t x = total[c] > -kInf ? order_key(total[c], uint32_t(c)) : 0;
      if (x < last && x > key) key = x;
    }
    last = block_reduce(key, kscratch, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
    if (threadIdx.x == 0) {
      const int64_t to = group * num_out + k;
      int32_t token = -1;
      int64_t row = row0;
      if (last != 0) {
        const uint32_t c = key_index(last);
        row = row0 + c / num_out;
        if (finished == nullptr || finished[row] == 0) token = int32_t(key_index(best[row * num_out + c % num_out]));
      }
      scores_out[to] = last != 0 ? key_value(last) : -kInf;
      tokens_out[to] = token;
      parents_out[to] = int32_t(row);
    }
  }
}

// One workgroup copies up to kCopy units of one row.
constexpr int kCopy = kThreads * 4;

template <class U>
__global__ __launch_bounds__(kThreads) void reorder_kernel(const U *src, int64_t num_src, int64_t units,
                                                           const int32_t *parents, U *dst, int32_t *status,
                                                           int64_t first) {
  const int64_t parts = (units + kCopy - 1) / kCopy, block = first + blockIdx.x;
  const int64_t row = block / parts, part = block % parts;
  const int64_t from = parents[row];
  const bool ok = from >= 0 && from < num_src;
  if (!ok && part == 0 && threadIdx.x == 0 && status != nullptr) atomicOr(status, RDF2V_STATUS_ID_OUT_OF_RANGE);
#pragma unroll
  for (int i = 0; i < kCopy / kThreads; ++i) {
    const int64_t u = part * kCopy + i * kThreads + threadIdx.x;
    if (u < units) dst[row * units + u] = ok ? src[from * units + u] : U{};
  }
}

template <class U>
rdf2v_status reorder(const void *src, int64_t num_src, int64_t row_bytes, const int32_t *parents, int64_t num_rows,
                     void *dst, int32_t *status, hipStream_t stream) {
  const int64_t units = row_bytes / int64_t(sizeof(U)), parts = (units + kCopy - 1) / kCopy;
  return for_each_launch(num_rows * parts, kThreads, 1, [&](int64_t first, int64_t count) {
    reorder_kernel<U><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(
        static_cast<const U *>(src), num_src, units, parents, static_cast<U *>(dst), status, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

}  // namespace

size_t beam_select_workspace_bytes(int64_t groups, int32_t beams, int64_t, int32_t num_out) {
  const size_t rows = size_t(groups) * beams;
  return align_up(rows * num_out * sizeof(uint64_t), 256) + align_up(rows * sizeof(float), 256);
}

rdf2v_status launch_beam_select(const void *logits, int64_t stride, int32_t dtype, const float *scores,
                                const int32_t *finished, int64_t groups, int32_t beams, int64_t vocab,
                                int32_t num_out, float *scores_out, int32_t *tokens_out, int32_t *parents_out,
                                void *workspace, int32_t *status_dev, hipStream_t stream) {
  const int64_t rows = groups * beams;
  uint64_t *best = static_cast<uint64_t *>(workspace);
  float *lse = reinterpret_cast<float *>(static_cast<char *>(workspace) +
                                         align_up(size_t(rows) * num_out * sizeof(uint64_t), 256));
  rdf2v_status st = for_each_launch(rows, kThreads, 1, [&](int64_t first, int64_t count) {
    if (dtype == RDF2V_BF16)
      beam_rows_kernel<bf16><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(
          static_cast<const bf16 *>(logits), stride, scores, finished, vocab, num_out, lse, best, status_dev, first);
    else
      beam_rows_kernel<float><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(
          static_cast<const float *>(logits), stride, scores, finished, vocab, num_out, lse, best, status_dev, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
  if (st != RDF2V_OK) return st;
  return for_each_launch(groups, kThreads, 1, [&](int64_t first, int64_t count) {
    beam_merge_kernel<<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(
        scores, finished, beams, num_out, lse, best, scores_out, tokens_out, parents_out, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

rdf2v_status launch_beam_reorder(const void *src, int64_t num_src, int64_t row_bytes, const int32_t *parents,
                                 int64_t num_rows, void *dst, int32_t *status_dev, hipStream_t stream) {
  const uintptr_t low = reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst) | uintptr_t(row_bytes);
  if ((low & 15) == 0) return reorder<uint4>(src, num_src, row_bytes, parents, num_rows, dst, status_dev, stream);
  if ((low & 3) == 0) return reorder<uint32_t>(src, num_src, row_bytes, parents, num_rows, dst, status_dev, stream);
  return reorder<uint8_t>(src, num_src, row_bytes, parents, num_rows, dst, status_dev, stream);
}

}  // namespace rdf2v
