// Host-side check that a call's outputs overlap neither its inputs nor each other.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace moe {

struct Span {                                    // p NULL or no bytes: nothing
  const void* p;
  int64_t bytes;
};

// `rows` rows of `row` bytes, `stride` bytes apart.
inline Span span_rows(const void* p, int64_t rows, int64_t stride, int64_t row) {
  return {p, rows > 0 ? (rows - 1) * stride + row : 0};
}

inline bool span_meets(const Span& a, const Span& b) {
  if (!a.p || !b.p || a.bytes <= 0 || b.bytes <= 0) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x < y ? (uint64_t)(y - x) < (uint64_t)a.bytes : (uint64_t)(x - y) < (uint64_t)b.bytes;
}

// Rows of one stride may lie between each other (slices of one buffer).
inline bool rows_meet(const void* a, const void* b, int64_t rows, int64_t stride_a, int64_t stride_b,
                      int64_t row) {
  if (!span_meets(span_rows(a, rows, stride_a, row), span_rows(b, rows, stride_b, row))) return false;
  if (stride_a != stride_b) return true;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  const int64_t gap = (int64_t)((x < y ? y - x : x - y) % (uint64_t)stride_a);
  return gap < row || stride_a - gap < row;
}

template <size_t N, size_t M>
inline bool spans_apart(const Span (&outs)[N], const Span (&ins)[M]) {
  for (size_t i = 0; i < N; ++i) {
    for (size_t j = 0; j < M; ++j)
      if (span_meets(outs[i], ins[j])) return false;
    for (size_t j = i + 1; j < N; ++j)
      if (span_meets(outs[i], outs[j])) return false;
  }
  return true;
}

}  // namespace moe
