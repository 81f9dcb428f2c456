// Host-side checks that the entry points of the operators over walk tokens share.
#pragma once

#include <climits>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <initializer_list>
#include <utility>

#include "rdf2v.h"

namespace rdf2v {

constexpr int64_t kInt32Limit = int64_t(1) << 31;
// Most elements of one array of a call: keeps every byte offset and size exact
// in 64 bits, and is far beyond any device memory.
constexpr int64_t kMaxElements = int64_t(1) << 56;
constexpr int64_t kMaxStride = int64_t(1) << 56;

inline bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline bool dtype_ok(int32_t dtype) { return dtype == RDF2V_F32 || dtype == RDF2V_BF16; }
inline size_t dtype_size(int32_t dtype) { return dtype == RDF2V_BF16 ? 2 : 4; }

// a * b for non-negative a and b, at most `most`; -1 beyond.
inline int64_t product(int64_t a, int64_t b, int64_t most) { return a >= 0 && (b == 0 || a <= most / b) ? a * b : -1; }

inline bool stride_ok(int64_t s) { return s > -kMaxStride && s < kMaxStride; }

inline bool view_ok(const rdf2v_heads_view *v, int32_t dtype, bool empty) {
  if (v == nullptr) return false;
  if (!stride_ok(v->row_stride) || !stride_ok(v->token_stride) || !stride_ok(v->head_stride)) return false;
  return (empty || v->data != nullptr) && aligned(v->data, dtype_size(dtype));
}

inline rdf2v_status check_workspace(const void *workspace, size_t bytes, size_t need) {
  if (need == 0) return RDF2V_OK;
  return workspace == nullptr || bytes < need || !aligned(workspace, 256) ? RDF2V_ERR_WORKSPACE : RDF2V_OK;
}

// Whether [a, a + an) and [b, b + bn) share a byte.
inline bool overlap(const void *a, size_t an, const void *b, size_t bn) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x <= y ? y - x < an : x - y < bn;
}

// An array of a call: where it lies, of how many bytes. Null or empty: it overlaps nothing.
struct Span {
  const void *data;
  size_t bytes;
};
inline bool overlap(const Span &a, const Span &b) {
  return a.data != nullptr && b.data != nullptr && a.bytes != 0 && b.bytes != 0 &&
         overlap(a.data, a.bytes, b.data, b.bytes);
}
inline bool same(const Span &a, const Span &b) { return a.data == b.data; }

// The bytes of a view as boxes inside boxes: count[i] boxes every step[i] bytes, those of the last level
// `bytes` long.
struct Boxes {
  __int128 step[3];
  int64_t count[3];
  __int128 bytes;
};

// Whether boxes of the levels from `level` on, the first of them at byte `at`, have a byte in [lo, hi).
inline bool boxes_reach(const Boxes &x, int level, __int128 at, __int128 lo, __int128 hi) {
  if (level == 3) return at < hi && at + x.bytes > lo;
  if (x.count[level] == 1) return boxes_reach(x, level + 1, at, lo, hi);
  __int128 size = x.bytes;  // from a box's first byte to its last
  for (int i = level + 1; i < 3; ++i) size += x.step[i] * (x.count[i] - 1);
  const __int128 all = size + x.step[level] * (x.count[level] - 1);
  if (at >= hi || at + all <= lo) return false;
  if (x.step[level] < size) return true;  // the boxes lie in one another: taken as one
  // Of the boxes that reach into the interval all but the first and the last lie in it.
  const __int128 first = at >= lo ? 0 : (lo - at) / x.step[level];
  __int128 last = (hi - 1 - at) / x.step[level];
  if (last > x.count[level] - 1) last = x.count[level] - 1;
  if (last - first > 1) return true;
  for (__int128 i = first; i <= last; ++i)
    if (boxes_reach(x, level + 1, at + i * x.step[level], lo, hi)) return true;
  return false;
}

// A view of rows x tokens x heads of `size` values as boxes. What lies between a view's values is not its own:
// another slice of the projection, say.
struct ViewBoxes {
  Boxes x{};
  __int128 at = 0;
  bool empty = true;

  ViewBoxes() = default;
  ViewBoxes(const rdf2v_heads_view &v, int64_t rows, int64_t length, int64_t heads, int64_t size, int32_t dtype) {
    if (rows == 0 || length == 0 || v.data == nullptr) return;
    empty = false;
    const int64_t value = int64_t(dtype_size(dtype));
    const int64_t strides[3] = {v.row_stride, v.token_stride, v.head_stride}, counts[3] = {rows, length, heads};
    x.bytes = __int128(size) * value;
    at = __int128(reinterpret_cast<uintptr_t>(v.data));
    for (int i = 0; i < 3; ++i) {
      const __int128 step = __int128(strides[i]) * value;
      if (step < 0) at += step * (counts[i] - 1);  // from the lowest byte upwards
      x.step[i] = step < 0 ? -step : step;
      x.count[i] = step == 0 ? 1 : counts[i];
      if (x.count[i] == 1) x.step[i] = 0;
    }
    for (int i = 0; i < 2; ++i)  // the widest first
      for (int j = 0; j < 2 - i; ++j)
        if (x.step[j] < x.step[j + 1]) {
          std::swap(x.step[j], x.step[j + 1]);
          std::swap(x.count[j], x.count[j + 1]);
        }
  }

  // Whether the view has a byte in an array.
  bool reach(const Span &out) const {
    if (empty || out.data == nullptr || out.bytes == 0) return false;
    const __int128 lo = __int128(reinterpret_cast<uintptr_t>(out.data));
    return boxes_reach(x, 0, at, lo, lo + __int128(out.bytes));
  }
};

}  // namespace rdf2v
