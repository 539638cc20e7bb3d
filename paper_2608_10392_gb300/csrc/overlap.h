// Whether arrays of a call share memory (plain C++): a result that is written while other parts of the
// call still read is refused.
#pragma once

#include <stdint.h>

#include <initializer_list>

namespace unif {

// Rows of `width` bytes, `pitch` bytes apart; NULL is no array.
struct Block {
  const void* p;
  int64_t pitch, width, rows;
};
inline Block flat(const void* p, int64_t bytes) { return {p, bytes, bytes, 1}; }

// Columns of one wider array, each its own, do not share memory. (Arrays of several rows at different
// distances do as soon as their ranges meet.)
inline bool overlap(const Block& a, const Block& b) {
  if (!a.p || !b.p || a.rows < 1 || b.rows < 1 || a.width < 1 || b.width < 1) return false;
  if (reinterpret_cast<uintptr_t>(b.p) < reinterpret_cast<uintptr_t>(a.p)) return overlap(b, a);
  const uintptr_t apart = reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p);
  if (apart >= (uint64_t)((a.rows - 1) * a.pitch + a.width)) return false;  // b begins behind a
  if (a.rows == 1) return true;
  if (b.rows > 1 && a.pitch != b.pitch) return true;
  const int64_t in_row = (int64_t)(apart % (uint64_t)a.pitch);  // where b begins in a row of a
  return in_row < a.width || in_row + b.width > a.pitch;
}

inline bool overlap_any(const Block& a, std::initializer_list<Block> others) {
  for (const Block& b : others)
    if (overlap(a, b)) return true;
  return false;
}

}  // namespace unif
