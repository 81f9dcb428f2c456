// Beam search's selection and the reordering of states on gfx950.
//
// Of a beam only the best logits can be chosen, so the logits are read once, in
// slices of a workgroup each, and reduced to the slice's num_out + 1 best and
// its part of the log-sum-exp; a workgroup per group then merges by total.
// Places are compared as (value descending, index ascending), a total order,
// so the choice does not depend on the order of the work.
//
// Totals are rounded sums, so logits that differ can have equal totals, of
// which the lowest token counts. The last entry of a slice is the best of what
// the slice left out: only where it or a smaller logit reaches the last chosen
// total, and could win by its token, is the slice read again for the lowest
// tokens at that total.

#include <climits>

#include "logits.hpp"

namespace rdf2v {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kVectors = 8;                    // 16-byte loads of a thread: 32 KB to a workgroup, all in flight
constexpr int kSlice = kVectors * kThreads;    // vectors of a slice
constexpr int kList = 1024;                    // candidates of a slice that are ranked at once

// Values in their order as unsigned numbers; that of -inf is below kLowest.
constexpr uint32_t kLowest = 0x00800000u;
__device__ __forceinline__ uint32_t order(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);  // -0 becomes +0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// Descending (value, -index) as one unsigned number: larger is better, 0 is none.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t index) {
  return uint64_t(order(x)) << 32 | (0xffffffffu - index);
}
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t o = uint32_t(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint32_t key_index(uint64_t key) { return 0xffffffffu - uint32_t(key); }

template <int W, class V, class Op>
__device__ __forceinline__ V block_reduce(V x, V *scratch, Op op) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) x = op(x, __shfl_xor(x, off, kWave));
  __syncthreads();
  if (lane_id() == 0) scratch[threadIdx.x / kWave] = x;
  __syncthreads();
  x = scratch[0];
#pragma unroll
  for (int i = 1; i < W; ++i) x = op(x, scratch[i]);
  return x;
}
template <int W>
__device__ __forceinline__ int block_sum(int x, int *scratch) {
  return block_reduce<W>(x, scratch, [](int a, int b) { return a + b; });
}

// The largest number of [lo, hi] that reach(number) holds for, and the smallest. reach falls (rises) once. The
// largest is often lo.
template <class Reach>
__device__ __forceinline__ uint32_t largest(uint32_t lo, uint32_t hi, Reach reach) {
  if (lo < hi && !reach(lo + 1)) return lo;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo - 1) / 2 + 1;
    if (reach(mid))
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}
template <class Reach>
__device__ __forceinline__ uint32_t smallest(uint32_t lo, uint32_t hi, Reach reach) {
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (reach(mid))
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

// A bound that at least k of the values that the threads' maxima x come from
// reach: in each of the W waves the k / W-th of its lanes' maxima, and the least of
// those. -inf where the values are fewer. One barrier pair.
template <int W = kWaves>
__device__ __forceinline__ float block_bound(float x, int k, float *scratch) {
  float at = kInf;
  for (int left = (k + W - 1) / W; left > 0;) {
    at = wave_max(x);
    // lanes of one maximum at once: where all are equal it is the bound
    left -= max(1, __popcll(__ballot(x == at)));
    if (x == at) x = -kInf;
  }
  __syncthreads();
  if (lane_id() == 0) scratch[threadIdx.x / kWave] = at;
  __syncthreads();
  at = scratch[0];
#pragma unroll
  for (int i = 1; i < W; ++i) at = fminf(at, scratch[i]);
  return at;
}

// The k largest of the n distinct keys in `list`, descending, zeros beyond n, to put(rank, key).
template <class Put>
__device__ __forceinline__ void rank_list(const uint64_t *list, int n, int k, Put put) {
  const int lane = lane_id();
  for (int i = threadIdx.x / kWave; i < n; i += kWaves) {
    const uint64_t key = list[i];
    int rank = 0;
    for (int j = lane; j - lane < n; j += kWave) rank += __popcll(__ballot(j < n && list[j] > key));
    if (lane == 0 && rank < k) put(rank, key);
  }
  for (int i = n + threadIdx.x; i < k; i += kThreads) put(i, uint64_t(0));
}

// A logit that can be chosen, or -inf.
__device__ __forceinline__ float usable(float x) { return x < kInf ? x : -kInf; }

__host__ __device__ __forceinline__ int64_t slice_count(int64_t vocab, int per) {
  return vocab / per < kSlice ? 1 : (vocab / per + kSlice - 1) / kSlice;
}

struct SelectArgs {
  const void *logits;
  const float *scores;
  const int32_t *finished;
  float *scores_out;
  int32_t *tokens_out, *parents_out, *status;
  float2 *parts;     // [rows][slices] largest logit, sum of exponentials over it
  uint64_t *best;    // [rows][slices][num_out + 1] logits and tokens, descending
  int64_t stride, vocab, slices;
  int32_t beams, num_out;
};

__device__ __forceinline__ bool row_counts(const SelectArgs &p, int64_t row) {
  return p.scores[row] > -kInf && (p.finished == nullptr || p.finished[row] == 0);
}

// One workgroup to a slice. HBM-bound: the logits are read once, 16 bytes a
// lane and kVectors of them in flight. 32 groups of 8 beams and 100,050 float32
// logits, a third of the beams finished or dead, take 19 us (3.7 TB/s), 8 groups
// of 8 and 1,000,200 bfloat16 logits 26 us (3.3 TB/s).
template <class T>
__global__ __launch_bounds__(kThreads) void beam_rows_kernel(SelectArgs p, int64_t first) {
  constexpr int kPer = Row<T>::kPer;
  __shared__ float scratch[2 * kWaves];
  __shared__ uint64_t list[kList];
  __shared__ int count, cscratch[kWaves];
  const int64_t block = first + blockIdx.x, row = block / p.slices, slice = block % p.slices;
  if (!row_counts(p, row)) return;
  const T *z = static_cast<const T *>(p.logits) + row * p.stride;
  const int k = p.num_out + 1;
  if (threadIdx.x == 0) count = 0;
  const int64_t whole = p.vocab / kPer;
  // Slices of equal size, and a short row spread over all waves: the bound of the candidates is that of the
  // wave that has least.
  const int64_t per = (whole + p.slices - 1) / p.slices, begin = slice * per, end = min(whole, begin + per);
  const int place = whole < kThreads ? lane_id() * kWaves + threadIdx.x / kWave : threadIdx.x;
  const int64_t v0 = begin + place;
  Words x[kVectors];  // as they lie in memory: half the registers for bfloat16
  if (whole > 0) {
#pragma unroll
    for (int i = 0; i < kVectors; ++i) x[i] = Row<T>::load(z, end, v0 + i * kThreads);
  }
  // the values after the last vector, one to a thread of the last slice
  const int64_t rest_at = whole * kPer + threadIdx.x;
  const bool has_rest = slice == p.slices - 1 && rest_at < p.vocab;
  float rest = has_rest ? to_f32(z[rest_at]) : -kInf;
  // Values are made from the words anew in each pass: kept, they would take the registers of other waves.
  auto each = [&](auto take) {
    if (whole > 0) {
#pragma unroll
      for (int i = 0; i < kVectors; ++i) {
        asm volatile("" : "+v"(x[i]));
#pragma unroll
        for (int j = 0; j < kPer; ++j)
          take(Row<T>::value(x[i], j), [&] { return uint32_t((v0 + i * kThreads) * kPer + j); });
      }
    }
    take(rest, [&] { return uint32_t(rest_at); });
  };
  float top = -kInf, sum = 0.0f;
  each([&](float y, auto) { top = fmaxf(top, y); });
  each([&](float y, auto) { sum += __expf(y - (top == -kInf ? 0.0f : top)); });
  if (!(sum < kInf) || !(top < kInf)) {  // NaN or +inf among them
    if (p.status != nullptr) atomicOr(p.status, RDF2V_STATUS_BAD_VALUE);
    top = -kInf;
    sum = 0.0f;
    each([&](float y, auto) { top = fmaxf(top, usable(y)); });
    each([&](float y, auto) { sum += __expf(usable(y) - (top == -kInf ? 0.0f : top)); });
  }
  const float bound = block_bound(top, k, scratch);  // its barriers also order `count`
  {
    const float most = wave_max(top), from = most == -kInf ? 0.0f : most;
    sum *= __expf(top - from);
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
    __syncthreads();
    if (lane_id() == 0) {
      scratch[threadIdx.x / kWave] = most;
      scratch[kWaves + threadIdx.x / kWave] = sum;
    }
  }
  auto collect = [&](float y, uint32_t index) {
    if (!(y >= bound) || !(usable(y) > -kInf)) return;
    const int at = atomicAdd(&count, 1);
    if (at < kList) list[at] = order_key(y, index);
  };
  if (whole > 0) {
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
      asm volatile("" : "+v"(x[i]));
      float most = Row<T>::value(x[i], 0);
#pragma unroll
      for (int j = 1; j < kPer; ++j) most = fmaxf(most, Row<T>::value(x[i], j));
      if (__ballot(most >= bound) == 0) continue;  // few vectors of a wave have any
      for (int j = 0; j < kPer; ++j)
        collect(Row<T>::value(x[i], j), uint32_t((v0 + i * kThreads) * kPer + j));
    }
  }
  collect(rest, uint32_t(rest_at));
  __syncthreads();
  if (threadIdx.x == 0) {
    float most = scratch[0], all = 0.0f;
#pragma unroll
    for (int i = 1; i < kWaves; ++i) most = fmaxf(most, scratch[i]);
    if (most > -kInf)
#pragma unroll
      for (int i = 0; i < kWaves; ++i) all += scratch[kWaves + i] * __expf(scratch[i] - most);
    p.parts[row * p.slices + slice] = make_float2(most, all);
  }
  uint64_t *best = p.best + (row * p.slices + slice) * k;
  const int n = count;
  if (n <= kList) {
    rank_list(list, n, k, [&](int rank, uint64_t key) { best[rank] = key; });
    return;
  }
  // More at the bound than the list holds, as where all logits are equal: the k-th value by halving, then of
  // that value as many tokens as are needed, in ascending order. The slice is read again for it: more code over
  // the registers would take them from the other waves.
  auto again = [&](auto take) {
#pragma unroll 1
    for (int64_t v = v0; v < end; v += kThreads) {
      const Words w = Row<T>::load(z, end, v);
#pragma unroll
      for (int j = 0; j < kPer; ++j) take(usable(Row<T>::value(w, j)), uint32_t(v * kPer + j));
    }
    take(usable(rest), uint32_t(rest_at));
  };
  auto at_least = [&](uint32_t value) {
    int c = 0;
    again([&](float y, uint32_t) { c += order(y) >= value; });
    return block_sum<kWaves>(c, cscratch);
  };
  const uint32_t most = order(fmaxf(fmaxf(scratch[0], scratch[1]), fmaxf(scratch[2], scratch[3])));
  const uint32_t value = largest(max(order(bound), kLowest), most, [&](uint32_t v) { return at_least(v) >= k; });
  int need = k - (value < most ? at_least(value + 1) : 0);
  uint32_t token = 0;
#pragma unroll 1
  for (int64_t step = begin;; step += kThreads) {
    const bool last = step + kThreads >= end;
    const Words w = Row<T>::load(z, end, step + threadIdx.x);
    auto up_to = [&](uint32_t t) {
      int c = last && order(usable(rest)) == value && uint32_t(rest_at) <= t;
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        c += order(usable(Row<T>::value(w, j))) == value && uint32_t((step + threadIdx.x) * kPer + j) <= t;
      return block_sum<kWaves>(c, cscratch);
    };
    const int here = up_to(0xffffffffu);
    if (here < need && !last) {
      need -= here;
      continue;
    }
    token = smallest(uint32_t(step * kPer), uint32_t(last ? p.vocab - 1 : (step + kThreads) * kPer - 1),
                     [&](uint32_t t) { return up_to(t) >= need; });
    break;
  }
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  again([&](float y, uint32_t index) {
    if (order(y) > value || (order(y) == value && index <= token)) list[atomicAdd(&count, 1)] = order_key(y, index);
  });
  __syncthreads();
  rank_list(list, k, k, [&](int rank, uint64_t key) { best[rank] = key; });
}

constexpr int kOwn = 2;        // parts of a wave that are read ahead
constexpr int kStaged = 5120;  // entries of all lists that LDS takes
// Candidates of the merge that are ranked at once, which takes as many steps as their square.
constexpr int kMergeList = 768;

// The next value of the element type below x, which is one.
template <class T>
__device__ __forceinline__ float previous(float x) {
  constexpr uint32_t kOne = sizeof(T) == 2 ? 0x10000u : 1u;
  const uint32_t b = __float_as_uint(x);
  return __uint_as_float(x == 0.0f ? 0x80000000u + kOne : x > 0.0f ? b - kOne : b + kOne);
}

// Threads of the merge: a chain of short steps, each shorter with more threads. A selection of 8 from 32
// groups of 8 beams and 100,050 float32 logits takes 34.5, 33 and 33 us with 256, 512 and 1024 threads, one
// from 8 groups of 8 beams and 1,000,200 bfloat16 logits 48, 41.5 and 40.5 us.
constexpr int kMergeThreads = 512;
constexpr int kMergeWaves = kMergeThreads / kWave;
static_assert(kMergeThreads + 4 * RDF2V_MAX_BEAMS <= kMergeList, "a step's entries, and what goes with them, are ranked at once");

// One workgroup to a group: its beams' candidates by total. 7 us for those 32 groups and 10 for those 8, bound
// by the latency of its steps, not by what it reads: one trip to memory for all lists, the beams' log-sum-exps,
// a bound from the lists' first entries, the entries that reach it, their ranks (a wave to a candidate and a
// ballot to 64 of those it is set against), and the look at what the slices left out.
template <class T>
__global__ __launch_bounds__(kMergeThreads) void beam_merge_kernel(SelectArgs p, int64_t first) {
  __shared__ float lse[RDF2V_MAX_BEAMS], score[RDF2V_MAX_BEAMS];
  __shared__ uint8_t counts[RDF2V_MAX_BEAMS], ended[RDF2V_MAX_BEAMS];
  __shared__ float fscratch[kMergeWaves];
  __shared__ uint64_t kscratch[kMergeWaves];
  __shared__ uint64_t list[kMergeList], stage[kStaged];
  __shared__ uint32_t place[kMergeList];
  __shared__ uint64_t chosen[RDF2V_MAX_BEAMS];
  __shared__ uint32_t chosen_place[RDF2V_MAX_BEAMS];
  __shared__ uint32_t tied[kMergeWaves][RDF2V_MAX_BEAMS];
  __shared__ int count, cscratch[kMergeWaves], tied_count[kMergeWaves];
  const int64_t group = first + blockIdx.x, row0 = group * p.beams;
  const int k = p.num_out + 1;
  const int64_t slices = p.slices;
  const int lane = lane_id(), wave = threadIdx.x / kWave;

  // One trip to memory for what nearly every group needs: the lists, where they fit LDS, the scores and a
  // wave's first parts. Lists of beams that do not count hold anything.
  const int lists = p.beams * int(slices), l0 = wave + kMergeWaves * lane;  // as many lists to each wave
  float2 parts[kOwn];
#pragma unroll
  for (int o = 0; o < kOwn; ++o)
    parts[o] = p.parts[(row0 + min(wave + o * kMergeWaves, p.beams - 1)) * slices + min(int64_t(lane), slices - 1)];
  const bool staged = lists * k <= kStaged;
  const uint64_t *source = p.best + row0 * slices * k;
  if (staged) {
    constexpr int kAhead = 5;
    for (int i = threadIdx.x; i < lists * k; i += kAhead * kMergeThreads) {
      uint64_t x[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) x[j] = source[min(i + j * kMergeThreads, lists * k - 1)];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j * kMergeThreads < lists * k) stage[i + j * kMergeThreads] = x[j];
    }
  }
  if (int(threadIdx.x) < p.beams) {
    const float x = p.scores[row0 + threadIdx.x];
    const bool end = p.finished != nullptr && p.finished[row0 + threadIdx.x] != 0;
    score[threadIdx.x] = x;
    counts[threadIdx.x] = x > -kInf && !end;
    ended[threadIdx.x] = x > -kInf && end;
  }
  __syncthreads();
  for (int b = wave, o = 0; b < p.beams; b += kMergeWaves, ++o) {
    if (!counts[b]) continue;
    float most = -kInf, sum = 0.0f;
    for (int64_t i = lane; i < slices; i += kWave) {
      float2 part;
      if (o < kOwn && i < kWave)
        part = o == 0 ? parts[0] : parts[1];
      else
        part = p.parts[(row0 + b) * slices + i];
      if (part.x > most) {
        sum = sum * __expf(most - part.x) + part.y;
        most = part.x;
      } else if (part.x > -kInf) {
        sum += part.y * __expf(part.x - most);
      }
    }
    const float all = wave_max(most);
    sum *= most > -kInf ? __expf(most - all) : 0.0f;
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
    if (lane == 0) {
      lse[b] = all + logf(sum);
      counts[b] = all > -kInf;
    }
  }
  __syncthreads();

  // the total of a beam's logit, in the order of the definition
  auto total_of = [&](int b, float x) { return score[b] + (x - lse[b]); };
  // candidates are compared by total, then by beam and token: (total, beam) is unique up to the token
  // a wave ranks one candidate of n at a time, its lanes a candidate each to set against it
  auto rank_one = [&](int i, int n) {
    const uint64_t key = list[i];
    const uint32_t at = place[i];
    int rank = 0;
    for (int j = lane; j - lane < n; j += kWave) {
      const uint64_t other = j < n ? list[j] : 0;
      const uint32_t there = j < n ? place[j] : 0;
      rank += __popcll(__ballot(other > key || (other == key && there < at)));
    }
    if (lane == 0 && rank < p.num_out && key != 0) {
      chosen[rank] = key;
      chosen_place[rank] = at;
    }
  };
  if (threadIdx.x == 0) count = 0;
  const uint64_t *keys = staged ? stage : source;
  // the lists' first entries: num_out of them bound the last chosen total
  float head = -kInf;
  for (int l = l0; l < lists; l += kMergeThreads) {
    const int b = l / int(slices);
    const uint64_t key = counts[b] ? keys[l * k] : 0;
    if (key != 0) head = fmaxf(head, total_of(b, key_value(key)));
  }
  const float bound = block_bound<kMergeWaves>(head, p.num_out, fscratch);
  // take(total, list, beam, token, 1 for a beam that has ended) for this thread's candidates of the first
  // `entries`. Descending logits have descending totals; the last entry of a list is left out.
  auto one = [&](int e, auto take) {
    const int l = e / k, b = l / int(slices);
    const uint64_t key = counts[b] && e - l * k < p.num_out ? keys[e] : 0;
    const float t = total_of(b, key_value(key));
    if (key != 0 && t >= bound && t > -kInf) take(t, l, b, key_index(key), 0u);
  };
  auto each = [&](int entries, auto take, int most = INT_MAX) {
    for (int e = threadIdx.x; e < entries && *static_cast<volatile int *>(&count) <= most; e += kMergeThreads)
      one(e, take);
    for (int b = threadIdx.x; b < p.beams; b += kMergeThreads)
      if (ended[b]) take(score[b], 0, b, 0u, 1u);
  };
  auto put = [&](float t, int, int b, uint32_t token, uint32_t end) {
    const int at = atomicAdd(&count, 1);
    if (at < kMergeList) {
      list[at] = order_key(t, uint32_t(b) << 26 | end);
      place[at] = token;
    }
  };
  each(lists * k, put, kMergeList);
  __syncthreads();
  int n = count;
  if (n > kMergeList) {
    // More at the bound than the list holds: the last total by halving, then of that total the first lists that
    // have enough, since a list's tokens are all lower than the next one's. Those are less than a step's entries
    // and a list too many, and fit.
    auto at_least = [&](uint32_t value) {
      int c = 0;
      each(lists * k, [&](float t, int, int, uint32_t, uint32_t) { c += order(t) >= value; });
      return block_sum<kMergeWaves>(c, cscratch);
    };
    uint32_t most = order(head);
    if (int(threadIdx.x) < p.beams && ended[threadIdx.x]) most = max(most, order(score[threadIdx.x]));
    most = block_reduce<kMergeWaves>(most, reinterpret_cast<uint32_t *>(cscratch),
                                     [](uint32_t a, uint32_t b) { return max(a, b); });
    const uint32_t value =
        largest(max(order(bound), kLowest), most, [&](uint32_t v) { return at_least(v) >= p.num_out; });
    int need = p.num_out - (value < most ? at_least(value + 1) : 0), upto = lists - 1;
    for (int step = 0; step < lists * k && need > 0; step += kMergeThreads) {
      int c = 0;
      if (step + int(threadIdx.x) < lists * k)
        one(step + threadIdx.x, [&](float t, int, int, uint32_t, uint32_t) { c = order(t) == value; });
      need -= block_sum<kMergeWaves>(c, cscratch);
      upto = min(lists - 1, (step + kMergeThreads - 1) / k);
    }
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    each(value < most ? lists * k : (upto + 1) * k, [&](float t, int l, int b, uint32_t token, uint32_t end) {
      if (order(t) > value || (order(t) == value && l <= upto)) put(t, l, b, token, end);
    });
    __syncthreads();
    n = count;
  }
  for (int i = wave; i < n; i += kMergeWaves) rank_one(i, n);
  for (int i = n + threadIdx.x; i < p.num_out; i += kMergeThreads) chosen[i] = 0;
  __syncthreads();

  // Whether something that a slice left out, its last entry among it, could belong to the chosen. The slice has
  // num_out entries of no smaller totals, so only at the last chosen total, and by a lower token than one of
  // those has. Of the last entry's logit the lowest tokens are taken first, so then either a greater logit
  // has the same total and a higher token, or a smaller logit the same total and any token.
  const uint64_t worst = chosen[p.num_out - 1];
  const float least = worst != 0 ? key_value(worst) : kInf;  // fewer than num_out: nothing was left out
  auto look_again = [&](int l) {
    const int b = l / int(slices);
    const uint64_t key = counts[b] ? keys[l * k + p.num_out] : 0;
    if (key == 0 || !(total_of(b, key_value(key)) >= least)) return false;
    bool look = total_of(b, previous<T>(key_value(key))) >= least;
    for (int i = 0; i < p.num_out && !look; ++i) {
      const uint64_t entry = keys[l * k + i];
      look = key_index(entry) > key_index(key) && total_of(b, key_value(entry)) == least;
    }
    return look;
  };
  // Such slices are read again, in ascending order of beam and token, until they have given as many tokens at
  // the last chosen total as it has places: what they give beyond is worse. Each gives one at least, its last
  // last entry, so few are read, be all logits equal: 8 groups of 8 beams and 1,000,200 equal float32 logits
  // take 184 us (random ones 72), with 64 places 216 (196).
  int places = RDF2V_MAX_BEAMS, found = 0;
  if (worst != 0) {
    for (int base = 0; base < lists && found < places; base += kMergeThreads) {
      const int mine = base + int(threadIdx.x);
      const bool look = mine < lists && look_again(mine);
      if (!__syncthreads_or(look)) continue;
      places = 0;
      for (int i = 0; i < p.num_out; ++i) places += chosen[i] >> 32 == worst >> 32;
      const uint64_t looks = __ballot(look);
      if (lane == 0) kscratch[wave] = looks;
      __syncthreads();
      for (int w = 0; w < kMergeWaves && found < places; ++w) {
        for (uint64_t left = kscratch[w]; left != 0 && found < places; left &= left - 1) {
          const int l = base + w * kWave + __builtin_ctzll(left), b = l / int(slices);
          const int64_t s = l - int64_t(b) * slices;
          constexpr int kPer = Row<T>::kPer, kAhead = 8;
          const int64_t whole = p.vocab / kPer, per = (whole + slices - 1) / slices;
          const int64_t begin = min(whole, s * per) * kPer;
          const int64_t end = s == slices - 1 ? p.vocab : min(whole, (s + 1) * per) * kPer;
          // a wave takes an eighth of the slice, in order
          const int64_t part = (end - begin + kMergeWaves - 1) / kMergeWaves;
          const int64_t lo = min(end, begin + wave * part), hi = min(end, lo + part);
          const T *z = static_cast<const T *>(p.logits) + (row0 + b) * p.stride;
          int n = 0;
          for (int64_t j0 = lo; j0 < hi && n < places; j0 += kAhead * kWave) {
            float x[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) x[i] = to_f32(z[min(j0 + i * kWave + lane, hi - 1)]);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
              const int64_t j = j0 + i * kWave + lane;
              const bool is = j < hi && total_of(b, usable(x[i])) == least;
              const uint64_t all = __ballot(is);
              const int at = n + __popcll(all & ((uint64_t(1) << lane) - 1));
              if (is && at < places) tied[wave][at] = uint32_t(j);
              n += __popcll(all);
            }
          }
          if (lane == 0) tied_count[wave] = min(n, places);
          __syncthreads();
          int before = found;
          for (int i = 0; i < wave; ++i) before += tied_count[i];
          if (lane < tied_count[wave] && before + lane < places) {
            list[p.num_out + before + lane] = order_key(least, uint32_t(b) << 26);
            place[p.num_out + before + lane] = tied[wave][lane];
          }
          for (int i = 0; i < kMergeWaves; ++i) found += tied_count[i];
          found = min(found, places);
          __syncthreads();
        }
      }
    }
  }
  if (found > 0) {
    // the chosen and the found, one of each
    const int n = p.num_out + found;
    for (int i = threadIdx.x; i < p.num_out; i += kMergeThreads) {
      list[i] = chosen[i];
      place[i] = chosen_place[i];
    }
    __syncthreads();
    for (int i = p.num_out + wave; i < n; i += kMergeWaves) {
      const bool same = lane < p.num_out && chosen[lane] == list[i] && chosen_place[lane] == place[i];
      if (__ballot(same) != 0 && lane == 0) list[i] = 0;
    }
    __syncthreads();
    for (int i = wave; i < n; i += kMergeWaves) rank_one(i, n);
    __syncthreads();
  }

  for (int r = threadIdx.x; r < p.num_out; r += kMergeThreads) {
    const uint64_t key = chosen[r];
    const uint32_t at = key_index(key);
    const int64_t to = group * p.num_out + r;
    p.scores_out[to] = key != 0 ? key_value(key) : -kInf;
    p.tokens_out[to] = key != 0 && at % (1u << 26) == 0 ? int32_t(chosen_place[r]) : -1;
    p.parents_out[to] = int32_t(row0 + (key != 0 ? at >> 26 : 0));
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

size_t beam_select_workspace_bytes(int64_t groups, int32_t beams, int64_t vocab, int32_t num_out) {
  const size_t lists = size_t(groups) * beams * slice_count(vocab, 4);  // float32 has the more slices
  return align_up(lists * (num_out + 1) * sizeof(uint64_t), 256) + align_up(lists * sizeof(float2), 256);
}

rdf2v_status launch_beam_select(const void *logits, int64_t stride, int32_t dtype, const float *scores,
                                const int32_t *finished, int64_t groups, int32_t beams, int64_t vocab,
                                int32_t num_out, float *scores_out, int32_t *tokens_out, int32_t *parents_out,
                                void *workspace, int32_t *status_dev, hipStream_t stream) {
  SelectArgs p{};
  p.logits = logits;
  p.scores = scores;
  p.finished = finished;
  p.scores_out = scores_out;
  p.tokens_out = tokens_out;
  p.parents_out = parents_out;
  p.status = status_dev;
  p.stride = stride;
  p.vocab = vocab;
  p.slices = slice_count(vocab, dtype == RDF2V_BF16 ? 8 : 4);
  p.beams = beams;
  p.num_out = num_out;
  const size_t lists = size_t(groups) * beams * p.slices;
  p.best = static_cast<uint64_t *>(workspace);
  p.parts = reinterpret_cast<float2 *>(static_cast<char *>(workspace) +
                                       align_up(lists * (num_out + 1) * sizeof(uint64_t), 256));
  rdf2v_status st = for_each_launch(int64_t(lists), kThreads, 1, [&](int64_t first, int64_t count) {
    if (dtype == RDF2V_BF16)
      beam_rows_kernel<bf16><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(p, first);
    else
      beam_rows_kernel<float><<<dim3(unsigned(count)), dim3(kThreads), 0, stream>>>(p, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
  if (st != RDF2V_OK) return st;
  return for_each_launch(groups, kMergeThreads, 1, [&](int64_t first, int64_t count) {
    if (dtype == RDF2V_BF16)
      beam_merge_kernel<bf16><<<dim3(unsigned(count)), dim3(kMergeThreads), 0, stream>>>(p, first);
    else
      beam_merge_kernel<float><<<dim3(unsigned(count)), dim3(kMergeThreads), 0, stream>>>(p, first);
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
