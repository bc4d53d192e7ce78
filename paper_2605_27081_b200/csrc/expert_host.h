// Host side shared by the operators on tokens sorted by expert: argument checks.
#pragma once

#include "logit_rows_host.h"

namespace remoe {
namespace sorted {

// A matrix of `n` rows: its address, the distance of its rows, and the alignment that its type asks for.  One without rows may be null.
inline bool bad_matrix(const void* p, int64_t stride, int64_t n, int64_t columns, int size) {
  return (!p && n > 0) || rows::misaligned(p, size) || (n > 1 && stride < columns);
}

// Widest access (16 bytes at most) that every row of a matrix starts on.
inline int access_width(const void* p, int64_t stride, int64_t n, int size) {
  const uint64_t bits = reinterpret_cast<uintptr_t>(p) | (n > 1 ? (uint64_t)stride * size : 0) | 16;
  return (int)(bits & (~bits + 1));
}

}  // namespace sorted
}  // namespace remoe
