// Rows of logits: what beam selection and distillation read them with.
#pragma once

#include "model.hpp"

namespace rdf2v {

constexpr float kInf = __builtin_huge_valf();

// Largest value of a wave's lanes, in every lane: the row scan of
// wave_inclusive_sum with the maximum.
__device__ __forceinline__ float wave_max(float x) {
  const int none = __float_as_int(-kInf);
#define RDF2V_MAX_STEP(CTRL, ROWS) \
  x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(none, __float_as_int(x), CTRL, ROWS, 0xf, false)));
  RDF2V_MAX_STEP(0x111, 0xf)
  RDF2V_MAX_STEP(0x112, 0xf)
  RDF2V_MAX_STEP(0x114, 0xf)
  RDF2V_MAX_STEP(0x118, 0xf)
  RDF2V_MAX_STEP(0x142, 0xa)
  RDF2V_MAX_STEP(0x143, 0xc)
#undef RDF2V_MAX_STEP
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), kWave - 1));
}

// Sum over a wave's lanes, in every lane.
__device__ __forceinline__ float wave_sum(float x) {
#define RDF2V_ADD_STEP(CTRL, ROWS) \
  x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROWS, 0xf, false));
  RDF2V_ADD_STEP(0x111, 0xf)
  RDF2V_ADD_STEP(0x112, 0xf)
  RDF2V_ADD_STEP(0x114, 0xf)
  RDF2V_ADD_STEP(0x118, 0xf)
  RDF2V_ADD_STEP(0x142, 0xa)
  RDF2V_ADD_STEP(0x143, 0xc)
#undef RDF2V_ADD_STEP
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), kWave - 1));
}

// A row as whole 16-byte vectors and the values after the last of them. Vectors
// start with the row, whatever its alignment (global loads need none), so that
// sums do not depend on where a row lies.
typedef uint32_t Words __attribute__((ext_vector_type(4)));
template <class T>
struct Row {
  static constexpr int kPer = 16 / sizeof(T);
  typedef uint32_t Unaligned __attribute__((ext_vector_type(4), aligned(2)));
  // Vector v of the first `end` ones of a row; -inf beyond.
  static __device__ __forceinline__ Words load(const T *row, int64_t end, int64_t v) {
    constexpr uint32_t kNone = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
    const Words x = *reinterpret_cast<const Unaligned *>(row + min(v, end - 1) * kPer);
    return v < end ? x : Words{kNone, kNone, kNone, kNone};
  }
  static __device__ __forceinline__ float value(const Words &x, int j) {
    if (sizeof(T) == 4) return __uint_as_float(x[j]);
    return __uint_as_float(j % 2 ? x[j / 2] & 0xffff0000u : x[j / 2] << 16);
  }
};

}  // namespace rdf2v
