// Rows of a tensor of any number of dimensions, whose last one is a row (plain C++).
#pragma once

#include <stdint.h>

namespace unif {

// The `n` dimensions in front of the last one as rows: how many, and the elements from each to the
// next (cols for a single one or none). False where they do not lie at one distance, or at one below cols: rows of
// an expanded tensor are one row in memory, at distance 0.
inline bool rows_at_one_distance(const int64_t* sizes, const int64_t* strides, int n, int64_t cols, int64_t* rows,
                                 int64_t* distance) {
  bool found = false;
  *rows = 1;
  *distance = cols;
  for (int i = 0; i < n; ++i)
    if (sizes[i] == 0) {
      *rows = 0;
      return true;
    }
  for (int i = n - 1; i >= 0; --i) {
    if (sizes[i] > 1) {
      if (!found) *distance = strides[i];
      found = true;
      if (*distance < cols || strides[i] != *distance * *rows) return false;
    }
    *rows *= sizes[i];
  }
  return true;
}

}  // namespace unif
