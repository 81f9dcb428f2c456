// Rows of channels as vectors of a few values, what the layer operators read and write them with.
#pragma once

#include "model.hpp"

namespace rdf2v {

// N values of a row from `p` on, of which `n` are there (the others read as 0 and are not written). Loads need
// no alignment beyond the element's.
template <class T, int N>
__device__ __forceinline__ void load_values(const T *p, int n, float (&x)[N]) {
  typedef T Vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  if (n >= N) {
    const Vec v = *reinterpret_cast<const Vec *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = to_f32(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = i < n ? to_f32(p[i]) : 0.0f;
  }
}
template <class T, int N>
__device__ __forceinline__ void store_values(T *p, int n, const float (&x)[N]) {
  typedef T Vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  if (n >= N) {
    Vec v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = from_f32<T>(x[i]);
    *reinterpret_cast<Vec *>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = from_f32<T>(x[i]);
  }
}

// The same in flight, as they lie in memory: half the registers where they are of 16 bits.
template <class T, int N>
struct Values {
  typedef T Vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  Vec v;
  __device__ __forceinline__ void load(const T *p, int n) {
    if (n >= N) {
      v = *reinterpret_cast<const Vec *>(p);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = i < n ? p[i] : T(0.0f);
    }
  }
  __device__ __forceinline__ float operator[](int i) const { return to_f32(v[i]); }
};

// A row's length as the caller gives it, kept within [0, length]; `report`: one thread of a call for each row.
__device__ __forceinline__ int64_t row_length(const int32_t *len, int64_t row, int64_t length, bool report,
                                              int32_t *status) {
  if (len == nullptr) return length;
  const int64_t l = len[row];
  if (l >= 0 && l <= length) return l;
  if (report && status != nullptr) atomicOr(status, RDF2V_STATUS_BAD_LENGTH);
  return l < 0 ? 0 : length;
}

// 2^x, the hardware's: off by about 1 unit in the last place, denormal results are 0.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// e^x for x <= 0 to about 2 units in the last place: the rounding of x log2 e, and what log2 e itself lacks in
// 24 bits, would cost |x| of them. 0 below -150, and for what is no number: callers put that in again.
__device__ __forceinline__ float exp_negative(float x) {
  x = __builtin_amdgcn_fmed3f(x, -150.0f, 0.0f);
  const float t = x * kLog2e, rest = fmaf(x, 1.92596299e-8f, fmaf(x, kLog2e, -t)), r = exp2_fast(t);
  return fmaf(r, rest * kLn2, r);
}

// 1 / (1 + e^-x) as a factor beside x: a number also where x is none. With it the slope of x sigmoid(x).
__device__ __forceinline__ float sigmoid(float x) {
  const float e = exp_negative(-fabsf(x)), d = __builtin_amdgcn_rcpf(1.0f + e);
  return x < 0.0f ? e * d : d;
}
__device__ __forceinline__ float silu_slope(float x, float s) { return s * fmaf(x, 1.0f - s, 1.0f); }

// Sums over the parts of partial results: values [parts][n] float32, in the order of the parts, to up to three
// arrays that lie one behind the other in a part's n values.
struct PartSums {
  const float *partial;
  int64_t parts;
  int64_t count[3];
  float *out[3];  // null: not wanted
};
rdf2v_status launch_part_sums(const PartSums &a, hipStream_t stream);

}  // namespace rdf2v
