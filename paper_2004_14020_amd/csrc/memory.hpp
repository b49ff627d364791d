// The memory that one call reads and writes: nothing it writes may overlap anything else of the call.
#pragma once

#include <algorithm>
#include <cstdint>

#include "caramel.h"

namespace caramel {

// Buffers are rows of equal length, `pitch` bytes apart; those in one piece are a single row.  What lies between the rows is not the
// buffer's, so that workers' rows may interleave in one array.  Buffers of several rows all have the same pitch within a call
// (a call has one kind of them).
struct Memory {
  struct Span {
    uint64_t lo, hi, row, pitch;
    bool written;
  };
  Span spans[4 * CARAMEL_MAX_WORLD + 1];  // four buffers of every worker, and a workspace
  uint32_t n = 0;

  void add(uint64_t at, uint64_t bytes, bool written) {
    if (bytes) spans[n++] = {at, at + bytes, bytes, bytes, written};
  }
  // no more than the last row's columns belong to it
  void add_rows(uint64_t at, uint64_t rows, uint64_t pitch, uint64_t columns, uint64_t elem_size, bool written) {
    if (rows) spans[n++] = {at, at + ((rows - 1) * pitch + columns) * elem_size, columns * elem_size, pitch * elem_size, written};
  }
  // x begins first, and y before x ends.
  static bool share(const Span& x, const Span& y) {
    const uint64_t down = (y.lo - x.lo) / x.pitch, right = (y.lo - x.lo) % x.pitch;
    const bool next = (down + 1) * x.pitch < x.hi - x.lo;  // x has a row after the one that y begins beside
    return right < x.row || (next && right + y.row > x.pitch);
  }
  bool overlap() {
    std::sort(spans, spans + n, [](const Span& x, const Span& y) { return x.lo < y.lo; });
    for (uint32_t i = 0; i < n; ++i)
      for (uint32_t j = i + 1; j < n && spans[j].lo < spans[i].hi; ++j)
        if ((spans[i].written || spans[j].written) && share(spans[i], spans[j])) return true;
    return false;
  }
};

}  // namespace caramel
