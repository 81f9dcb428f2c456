// Sums of partial results over workgroups on gfx950: parameters' gradients are sums over all tokens, which
// workgroups leave as one partial sum each. Added up in a fixed order, so that the same inputs give the same bits.
#include "vectors.hpp"

namespace rdf2v {
namespace {

constexpr int kValues = 64, kRanks = 16;

// 64 values of a workgroup; 16 threads to a value, each takes every sixteenth part. Held in 64 bits: the parts
// are few, and their sum is rounded once.
__global__ __launch_bounds__(kValues *kRanks) void part_sums_kernel(PartSums a) {
  __shared__ double sums[kRanks][kValues];
  const int lane = threadIdx.x % kValues, rank = threadIdx.x / kValues;
  const int64_t n = a.count[0] + a.count[1] + a.count[2], at = int64_t(blockIdx.x) * kValues + lane;
  double sum = 0.0;
  if (at < n)
    for (int64_t p = rank; p < a.parts; p += kRanks) sum += a.partial[p * n + at];
  sums[rank][lane] = sum;
  __syncthreads();
  if (rank != 0 || at >= n) return;
  for (int r = 1; r < kRanks; ++r) sum += sums[r][lane];
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
  if (n == 0) return RDF2V_OK;
  const int64_t blocks = (n + kValues - 1) / kValues;
  if (blocks * kValues * kRanks > kMaxLaunchThreads) return RDF2V_ERR_TOO_LARGE;
  hipLaunchKernelGGL(part_sums_kernel, dim3(uint32_t(blocks)), dim3(kValues * kRanks), 0, stream, a);
  RDF2V_LAUNCH_CHECK();
  return RDF2V_OK;
}

}  // namespace rdf2v
