// Sums of partial results over workgroups on gfx950: parameters' gradients are sums over all tokens, which
// workgroups leave as one partial sum each. Added up in a fixed order, so that the same inputs give the same bits.
#include "vectors.hpp"

namespace rdf2v {
namespace {

constexpr int kValues = 16, kRanks = 64;  // values of a workgroup, threads of a value
constexpr int kWaves = kValues * kRanks / kWave;

// A value's threads take every 64th part each, eight loads in flight. Held in 64 bits: the parts are few, and their
// sum is rounded once. 1,024 parts of 903 values: 20 us with 16 threads to each of 64 values of a workgroup, which
// leaves 15 workgroups, 5 us so.
__global__ __launch_bounds__(kValues *kRanks) void part_sums_kernel(PartSums a, int64_t first) {
  constexpr int kAhead = 8;
  __shared__ double sums[kWaves][kValues];
  const int value = threadIdx.x % kValues, rank = threadIdx.x / kValues;
  const int64_t n = a.count[0] + a.count[1] + a.count[2], at = (first + blockIdx.x) * kValues + value;
  double sum = 0.0;
  if (at < n)
    for (int64_t p = rank; p < a.parts; p += kAhead * kRanks) {
      float x[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) x[k] = p + k * kRanks < a.parts ? a.partial[(p + k * kRanks) * n + at] : 0.0f;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) sum += x[k];
    }
  for (int m = kValues; m < kWave; m *= 2) sum += __shfl_xor(sum, m, kWave);
  if (threadIdx.x % kWave < kValues) sums[threadIdx.x / kWave][value] = sum;
  __syncthreads();
  if (threadIdx.x >= kValues || at >= n) return;
  for (int w = 1; w < kWaves; ++w) sum += sums[w][value];
  int64_t i = at;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    if (i < a.count[k]) {
      if (a.out[k] != nullptr) a.out[k][i] = float(sum);
      return;
    }
    i -= a.count[k];
  }
}

}  // namespace

rdf2v_status launch_part_sums(const PartSums &a, hipStream_t stream) {
  const int64_t n = a.count[0] + a.count[1] + a.count[2];
  return for_each_launch((n + kValues - 1) / kValues, kValues * kRanks, 1, [&](int64_t first, int64_t count) {
    part_sums_kernel<<<dim3(unsigned(count)), dim3(kValues * kRanks), 0, stream>>>(a, first);
    RDF2V_LAUNCH_CHECK();
    return RDF2V_OK;
  });
}

}  // namespace rdf2v
