// Distillation from a teacher's top logits on gfx950.
//
// With p the softmax of the teacher's entries over the temperature tau and q
// that of the logits over the whole vocabulary,
//   loss = tau^2 (sum_k p_k (log p_k - z_{id_k} / tau) + lse)
//   dlogits = dloss tau (q - p)
// so a row needs its log-sum-exp, the logits at the teacher's ids, and for the
// gradient one more look at the row. HBM-bound: the floor is one read, and one
// write for the gradient. A row that fits the registers of a workgroup stays
// there between the two looks. A longer one is cut into slices of a workgroup
// each, in two launches over some rows at a time; the second goes backwards, so
// that about half of what it reads is still in the Infinity Cache (256 MB).
//
// The gradient at the teacher's ids is written after the row's q, by the
// workgroup that wrote that q, so it is rounded once; every occurrence of a
// repeated id writes the same value.

#include "logits.hpp"

namespace rdf2v {
namespace {

constexpr int kVectors = 8;  // 16-byte loads of a thread, all in flight
constexpr int kSliceThreads = 256;
constexpr int64_t kSlice = int64_t(kVectors) * kSliceThreads;  // vectors of a slice of a long row
constexpr int64_t kLargest = int64_t(kVectors) * 1024;         // vectors of a row that stays in registers
// Bytes of logits between the two looks. Of 1 GB of bfloat16 logits and their
// gradient, both looks took 669 us at 96 MB (the ends of 22 launches), 586 at
// 192 MB and 578 without batches; with the second look backwards 590 at 200 MB,
// 543 at 400 MB and 550 without batches.
constexpr int64_t kCached = int64_t(400) << 20;
constexpr float kLog2e = 1.44269504088896341f;

// What the two launches over a long row hand on, for each row.
struct Workspace {
  float2 *parts;  // [rows][slices] largest logit, sum of exponentials over it
  float *zk;      // [rows][top] the logits at the teacher's ids, over tau
  int64_t slices;
};

// A row's teacher entries: every wave computes their log-sum-exp for itself, as
// the largest and the logarithm of the sum over it: their sum would lose the
// latter, and the entries' differences, beside large logits. `each(k, id, t)` is
// called by one lane of the calling wave for each.
struct Teacher {
  float most, log_sum, inv_tau;
  bool valid;
  __device__ __forceinline__ float log_p(float t) const { return fmaf(t - most, inv_tau, -log_sum); }
};
template <class Each>
__device__ __forceinline__ Teacher read_teacher(const DistillArgs &a, int64_t row, float inv_tau, bool report,
                                                Each each) {
  float most = -kInf, sum = 0.0f;
  bool any = false;
  for (int k = lane_id(); k < a.top; k += kWave) {
    int32_t id = a.ids[row * a.top + k];
    const float t = a.teacher[row * a.top + k];
    if (int64_t(id) >= a.vocab) {
      if (report && a.status != nullptr) atomicOr(a.status, RDF2V_STATUS_ID_OUT_OF_RANGE);
      id = -1;
    }
    if (t == -kInf) id = -1;
    each(k, id, t);
    if (id < 0) continue;
    any = true;
    const float up = fmaxf(most, t);
    sum = sum * (most == -kInf ? 0.0f : expf((most - up) * inv_tau)) + expf((t - up) * inv_tau);
    most = up;
  }
  const float top = wave_max(most);
  sum = wave_sum(any ? sum * expf((most - top) * inv_tau) : 0.0f);
  return {top, logf(sum), inv_tau, __ballot(any) != 0};
}

// Calls take(words, i, whether the vector is there) for the vectors of this thread.
template <class T, int THREADS>
struct Slice {
  Words x[kVectors];
  float rest;

  // Vectors begin .. end of a row and, for the workgroup that has them, the values after the row's last.
  __device__ __forceinline__ void load(const T *z, int64_t begin, int64_t end, int64_t rest_at, int64_t vocab) {
#pragma unroll
    for (int i = 0; i < kVectors; ++i)
      if (begin + i * THREADS < end) x[i] = Row<T>::load(z, end, begin + i * THREADS + threadIdx.x);
    rest = rest_at < vocab ? to_f32(z[rest_at]) : -kInf;
  }
  // (largest, sum of exponentials over it) of this thread's values over tau
  __device__ __forceinline__ float2 fold(int64_t begin, int64_t end, float inv_tau) {
    float top = rest;
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
      if (begin + i * THREADS >= end) break;
#pragma unroll
      for (int j = 0; j < Row<T>::kPer; ++j) top = fmaxf(top, Row<T>::value(x[i], j));
    }
    const float from = top == -kInf ? 0.0f : top, c = inv_tau * kLog2e;
    float sum = __builtin_amdgcn_exp2f((rest - from) * c);
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
      if (begin + i * THREADS >= end) break;
      asm volatile("" : "+v"(x[i]));  // made from the words anew: kept, the values would cost registers
#pragma unroll
      for (int j = 0; j < Row<T>::kPer; ++j)
        sum += __builtin_amdgcn_exp2f((Row<T>::value(x[i], j) - from) * c);
    }
    return make_float2(top * inv_tau, sum);
  }
  __device__ __forceinline__ void store(T *dz, int64_t begin, int64_t end, int64_t rest_at, int64_t vocab,
                                        float inv_tau, float lse, float w) {
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
      if (begin + i * THREADS >= end) break;
      asm volatile("" : "+v"(x[i]));
      const int64_t v = begin + i * THREADS + threadIdx.x;
      if (v >= end) break;
      typedef T vec __attribute__((ext_vector_type(Row<T>::kPer)));
      typedef uint32_t Unaligned __attribute__((ext_vector_type(4), aligned(2)));
      vec y;
#pragma unroll
      for (int j = 0; j < Row<T>::kPer; ++j) y[j] = from_f32<T>(w * q(Row<T>::value(x[i], j), inv_tau, lse));
      __builtin_nontemporal_store(__builtin_bit_cast(Words, y), reinterpret_cast<Unaligned *>(dz + v * Row<T>::kPer));
    }
    if (rest_at < vocab) dz[rest_at] = from_f32<T>(w * q(rest, inv_tau, lse));
  }
  static __device__ __forceinline__ float q(float z, float inv_tau, float lse) {
    return __builtin_amdgcn_exp2f(fmaf(z, inv_tau, -lse) * kLog2e);
  }
};

// Zeros for a row without entries.
template <class T, int THREADS>
__device__ __forceinline__ void store_zeros(T *dz, int64_t begin, int64_t end, int64_t rest_at, int64_t vocab) {
  typedef uint32_t Unaligned __attribute__((ext_vector_type(4), aligned(2)));
  for (int64_t v = begin + threadIdx.x; v < end; v += THREADS)
    __builtin_nontemporal_store(Words{0, 0, 0, 0}, reinterpret_cast<Unaligned *>(dz + v * Row<T>::kPer));
  if (rest_at < vocab) dz[rest_at] = from_f32<T>(0.0f);
}

// (largest, sum) pairs of all threads, in every thread. One barrier.
template <int THREADS>
__device__ __forceinline__ float2 block_fold(float2 x, float2 *scratch) {
  const float most = wave_max(x.x);
  const float sum = wave_sum(x.y * (x.x == -kInf && most == -kInf ? 1.0f : expf(x.x - most)));
  if (THREADS == kWave) return make_float2(most, sum);
  if (lane_id() == 0) scratch[threadIdx.x / kWave] = make_float2(most, sum);
  __syncthreads();
  float top = scratch[0].x, all = 0.0f;
#pragma unroll
  for (int i = 1; i < THREADS / kWave; ++i) top = fmaxf(top, scratch[i].x);
#pragma unroll
  for (int i = 0; i < THREADS / kWave; ++i)
    all += scratch[i].y * (scratch[i].x == top ? 1.0f : expf(scratch[i].x - top));
  return make_float2(top, all);
}

__device__ __forceinline__ float log_sum(float2 x) { return x.x == -kInf && x.y == 0.0f ? -kInf : x.x + logf(x.y); }

// What row_loss and the gradient at the ids read; ids that count are not negative.
struct Entries {
  const float *t, *zk;  // zk is over tau
  const int32_t *id;
};

// The loss of a row, by one wave.
__device__ __forceinline__ float row_loss(const DistillArgs &a, const Entries &e, const Teacher &teacher, float lse) {
  float loss = 0.0f;
  for (int k = lane_id(); k < a.top; k += kWave) {
    if (e.id[k] < 0) continue;
    const float log_p = teacher.log_p(e.t[k]), p = expf(log_p);
    // a p that is too small for float32 is not 0: nothing times a number, infinite where q is 0
    if (p == 0.0f)
      loss += e.zk[k] == -kInf ? kInf : 0.0f;
    else
      loss += p * (log_p - (e.zk[k] == -kInf ? -kInf : e.zk[k] - lse));
  }
  return a.temperature * a.temperature * wave_sum(loss);
}

// The gradient at the ids in [lo, hi).
template <class T, int THREADS>
__device__ __forceinline__ void store_entries(const DistillArgs &a, const Entries &e, T *dz, int64_t lo, int64_t hi,
                                              const Teacher &teacher, float lse, float w) {
  for (int k = threadIdx.x; k < a.top; k += THREADS) {
    const int32_t id = e.id[k];
    if (id < 0 || id < lo || id >= hi) continue;
    float p = 0.0f;
    for (int m = 0; m < a.top; ++m)
      if (e.id[m] == id) p += expf(teacher.log_p(e.t[m]));
    dz[id] = from_f32<T>(w * (__builtin_amdgcn_exp2f((e.zk[k] - lse) * kLog2e) - p));
  }
}

// One workgroup to a row that stays in its registers. 4,352 rows of 10,100
// bfloat16 logits, loss and gradient: 41 us, 4.0 TB/s.
template <class T, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_row_kernel(DistillArgs a, int64_t first) {
  extern __shared__ float shared[];
  float *t = shared, *zk = shared + a.top;
  int32_t *id = reinterpret_cast<int32_t *>(shared + 2 * a.top);
  __shared__ float2 scratch[THREADS / kWave];
  const int64_t row = first + blockIdx.x;
  const T *z = static_cast<const T *>(a.logits) + row * a.stride;
  T *dz = a.dlogits == nullptr ? nullptr : static_cast<T *>(a.dlogits) + row * a.dstride;
  const float inv_tau = 1.0f / a.temperature;
  const int64_t whole = a.vocab / Row<T>::kPer, rest_at = whole * Row<T>::kPer + threadIdx.x;
  const bool first_wave = threadIdx.x < kWave;
  const Teacher teacher = read_teacher(a, row, inv_tau, first_wave, [&](int k, int32_t i, float x) {
    if (!first_wave) return;
    t[k] = x;
    id[k] = i;
    zk[k] = i >= 0 ? to_f32(z[i]) * inv_tau : 0.0f;
  });
  if (!teacher.valid) {
    if (threadIdx.x == 0 && a.loss != nullptr) a.loss[row] = a.lse[row] = 0.0f;
    if (dz != nullptr) store_zeros<T, THREADS>(dz, 0, whole, rest_at, a.vocab);
    return;
  }
  Slice<T, THREADS> slice;
  slice.load(z, 0, whole, rest_at, a.vocab);
  float lse;
  if (a.loss != nullptr) {
    lse = log_sum(block_fold<THREADS>(slice.fold(0, whole, inv_tau), scratch));
    if (first_wave) {
      const float loss = row_loss(a, {t, zk, id}, teacher, lse);
      if (threadIdx.x == 0) {
        a.loss[row] = loss;
        a.lse[row] = lse;
      }
    }
  } else {
    lse = a.lse_in[row];
  }
  if (dz == nullptr) return;
  __syncthreads();  // in place: the logits at the ids have been read
  const float w = a.dloss[row] * a.temperature, from = lse == -kInf ? 0.0f : lse;  // all masked: q = 0
  slice.store(dz, 0, whole, rest_at, a.vocab, inv_tau, from, w);
  __syncthreads();
  store_entries<T, THREADS>(a, {t, zk, id}, dz, 0, a.vocab, teacher, from, w);
}

// One workgroup to a slice of a long row: its part of the log-sum-exp, and with
// the first slice the logits at the ids, which an in-place gradient overwrites.
// 510 rows of 1,000,200 bfloat16 logits (1 GB, and as much gradient): 545 us
// for both looks, of which this one takes two fifths.
template <class T>
__global__ __launch_bounds__(kSliceThreads) void distill_stats_kernel(DistillArgs a, Workspace ws, int64_t first) {
  __shared__ float2 scratch[kSliceThreads / kWave];
  const int64_t slices = a.loss != nullptr ? ws.slices : 1;  // the gradient alone needs the first only
  const int64_t block = first + blockIdx.x, row = block / slices, at = block % slices;
  const T *z = static_cast<const T *>(a.logits) + row * a.stride;
  const float inv_tau = 1.0f / a.temperature;
  const bool gather = at == 0 && threadIdx.x < kWave;
  const Teacher teacher = read_teacher(a, row, inv_tau, gather, [&](int k, int32_t i, float) {
    if (gather) ws.zk[row * a.top + k] = i >= 0 ? to_f32(z[i]) * inv_tau : 0.0f;
  });
  if (!teacher.valid || a.loss == nullptr) return;
  const int64_t whole = a.vocab / Row<T>::kPer, per = (whole + slices - 1) / slices;
  const int64_t begin = at * per, end = min(whole, begin + per);
  const int64_t rest_at = at == 0 ? whole * Row<T>::kPer + threadIdx.x : a.vocab;
  Slice<T, kSliceThreads> slice;
  slice.load(z, begin, end, rest_at, a.vocab);
  const float2 part = block_fold<kSliceThreads>(slice.fold(begin, end, inv_tau), scratch);
  if (threadIdx.x == 0) ws.parts[row * slices + at] = part;
}

// One workgroup to a slice of a long row: its gradient; with the first slice
// the loss.
template <class T>
__global__ __launch_bounds__(kSliceThreads) void distill_grad_kernel(DistillArgs a, Workspace ws, int64_t first) {
  extern __shared__ float shared[];
  float *t = shared, *zk = shared + a.top;
  int32_t *id = reinterpret_cast<int32_t *>(shared + 2 * a.top);
  const int64_t slices = a.dlogits != nullptr ? ws.slices : 1;  // the loss alone needs the first only
  const int64_t block = first + (gridDim.x - 1 - blockIdx.x);  // backwards: the rows read last are cached
  const int64_t row = block / slices, at = block % slices;
  const T *z = static_cast<const T *>(a.logits) + row * a.stride;
  T *dz = a.dlogits == nullptr ? nullptr : static_cast<T *>(a.dlogits) + row * a.dstride;
  const float inv_tau = 1.0f / a.temperature;
  const int64_t whole = a.vocab / Row<T>::kPer, per = (whole + ws.slices - 1) / ws.slices;
  const int64_t begin = at * per, end = min(whole, begin + per);
  const int64_t rest_at = at == 0 ? whole * Row<T>::kPer + threadIdx.x : a.vocab;
  const bool first_wave = threadIdx.x < kWave;
  const Teacher teacher = read_teacher(a, row, inv_tau, false, [&](int k, int32_t i, float x) {
    if (!first_wave) return;
    t[k] = x;
    id[k] = i;
    zk[k] = ws.zk[row * a.top + k];
  });
  if (!teacher.valid) {
    if (at == 0 && threadIdx.x == 0 && a.loss != nullptr) a.loss[row] = a.lse[row] = 0.0f;
    if (dz != nullptr) store_zeros<T, kSliceThreads>(dz, begin, end, rest_at, a.vocab);
    return;
  }
  Slice<T, kSliceThreads> slice;
  if (dz != nullptr) slice.load(z, begin, end, rest_at, a.vocab);
  float lse;
  if (a.loss != nullptr) {
    // every wave joins the row's parts for itself
    float2 x = make_float2(-kInf, 0.0f);
    for (int64_t i = lane_id(); i < ws.slices; i += kWave) {
      const float2 y = ws.parts[row * ws.slices + i];
      const float up = fmaxf(x.x, y.x);
      const float keep = x.x == up ? 1.0f : expf(x.x - up), add = y.x == up ? 1.0f : expf(y.x - up);
      x = make_float2(up, x.y * keep + y.y * add);
    }
    const float most = wave_max(x.x);
    lse = log_sum(make_float2(most, wave_sum(x.y * (x.x == most ? 1.0f : expf(x.x - most)))));
    if (at == 0 && first_wave) {
      const float loss = row_loss(a, {t, zk, id}, teacher, lse);
      if (threadIdx.x == 0) {
        a.loss[row] = loss;
        a.lse[row] = lse;
      }
    }
  } else {
    lse = a.lse_in[row];
  }
  if (dz == nullptr) return;
  const float w = a.dloss[row] * a.temperature, from = lse == -kInf ? 0.0f : lse;  // all masked: q = 0
  slice.store(dz, begin, end, rest_at, a.vocab, inv_tau, from, w);
  __syncthreads();
  const Entries e{t, zk, id};
  store_entries<T, kSliceThreads>(a, e, dz, begin * Row<T>::kPer, end * Row<T>::kPer, teacher, from, w);
  if (at == 0) store_entries<T, kSliceThreads>(a, e, dz, whole * Row<T>::kPer, a.vocab, teacher, from, w);
}

int64_t row_vectors(int64_t vocab, int32_t dtype) { return vocab / (dtype == RDF2V_BF16 ? 8 : 4); }
int64_t slice_count(int64_t vocab, int32_t dtype) { return (row_vectors(vocab, dtype) + kSlice - 1) / kSlice; }

size_t entry_bytes(const DistillArgs &a) { return size_t(a.top) * 12; }

template <class T, int THREADS>
rdf2v_status launch_rows(const DistillArgs &a, hipStream_t stream) {
  return for_each_launch(a.rows, THREADS, 1, [&](int64_t first, int64_t count) {
    distill_row_kernel<T, THREADS>
        <<<dim3(unsigned(count)), dim3(THREADS), entry_bytes(a), stream>>>(a, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

template <class T>
rdf2v_status launch(const DistillArgs &a, void *workspace, hipStream_t stream) {
  const int64_t vectors = row_vectors(a.vocab, a.dtype);
  if (vectors <= int64_t(kVectors) * kWave) return launch_rows<T, kWave>(a, stream);
  if (vectors <= kSlice) return launch_rows<T, kSliceThreads>(a, stream);
  if (vectors <= kLargest) return launch_rows<T, 1024>(a, stream);
  Workspace ws{};
  ws.slices = slice_count(a.vocab, a.dtype);
  ws.parts = static_cast<float2 *>(workspace);
  ws.zk = reinterpret_cast<float *>(static_cast<char *>(workspace) +
                                    align_up(size_t(a.rows) * ws.slices * sizeof(float2), 256));
  int64_t batch = a.dlogits == nullptr || a.loss == nullptr ? a.rows : kCached / (a.vocab * int64_t(sizeof(T)));
  if (batch < 1) batch = 1;
  for (int64_t row = 0; row < a.rows; row += batch) {
    const int64_t rows = a.rows - row < batch ? a.rows - row : batch;
    const int64_t stats = a.loss != nullptr ? ws.slices : 1, grads = a.dlogits != nullptr ? ws.slices : 1;
    rdf2v_status st = for_each_launch(rows * stats, kSliceThreads, 1, [&](int64_t first, int64_t count) {
      distill_stats_kernel<T>
          <<<dim3(unsigned(count)), dim3(kSliceThreads), 0, stream>>>(a, ws, row * stats + first);
      RDF2V_LAUNCH_CHECK();
      return RDF2V_OK;
    });
    if (st != RDF2V_OK) return st;
    st = for_each_launch(rows * grads, kSliceThreads, 1, [&](int64_t first, int64_t count) {
      distill_grad_kernel<T>
          <<<dim3(unsigned(count)), dim3(kSliceThreads), entry_bytes(a), stream>>>(a, ws, row * grads + first);
      RDF2V_LAUNCH_CHECK();
      return RDF2V_OK;
    });
    if (st != RDF2V_OK) return st;
  }
  return RDF2V_OK;
}

}  // namespace

size_t distill_workspace_bytes(int64_t rows, int64_t vocab, int32_t top, int32_t dtype) {
  if (row_vectors(vocab, dtype) <= kLargest) return 0;
  return align_up(size_t(rows) * slice_count(vocab, dtype) * sizeof(float2), 256) +
         align_up(size_t(rows) * top * sizeof(float), 256);
}

rdf2v_status launch_distill(const DistillArgs &a, void *workspace, hipStream_t stream) {
  return a.dtype == RDF2V_BF16 ? launch<bf16>(a, workspace, stream) : launch<float>(a, workspace, stream);
}

}  // namespace rdf2v
