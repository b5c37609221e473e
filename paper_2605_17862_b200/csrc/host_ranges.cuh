// Address ranges of the tensors of a call, and whether a written one meets another.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <numeric>
#include <vector>

#include "../../include/fopd.h"

namespace fopd {

struct Range {
  uintptr_t lo, hi, row;  // row: pitch in bytes (0: one row, or rows without a gap)
  uintptr_t width;        // bytes of a row
  int32_t tensor;
  bool written;
};

static inline Range range_of(const void *p, int64_t rows, int64_t cols, int64_t row_stride, uintptr_t esz, int32_t i, bool written) {
  const bool dense = rows == 1 || row_stride == cols;
  const uintptr_t a = (uintptr_t)p;
  const uintptr_t width = (uintptr_t)(dense ? rows * cols : cols) * esz, pitch = dense ? 0 : (uintptr_t)row_stride * esz;
  return {a, a + (uintptr_t)(rows - 1) * pitch + width, pitch, width, i, written};
}

// Column blocks and rows of one wider matrix overlap as ranges but not as elements.  The distance of a row of b behind a
// row of a is b.lo - a.lo and any multiples of both pitches, that is of their greatest common divisor (the other's where
// one has a single row): no row of b meets one of a if within that distance b's row lies behind a's and ends before the
// next.  a starts first.
static inline bool disjoint_columns(const Range &a, const Range &b) {
  const uintptr_t pitch = std::gcd(a.row, b.row);
  if (pitch == 0) return false;
  const uintptr_t shift = (b.lo - a.lo) % pitch;
  return shift >= a.width && shift + b.width <= pitch;
}

// Whether a written range meets another one; inputs (or in place) and outputs apart: each is usually in order already.
static inline int check_ranges(std::vector<Range> &in, std::vector<Range> &out) {
  const auto before = [](const Range &a, const Range &b) { return a.lo < b.lo; };
  std::vector<Range> r;
  for (std::vector<Range> *v : {&in, &out})
    if (!std::is_sorted(v->begin(), v->end(), before)) std::sort(v->begin(), v->end(), before);
  if (out.empty()) {
    r.swap(in);
  } else {
    r.resize(in.size() + out.size());
    std::merge(in.begin(), in.end(), out.begin(), out.end(), r.begin(), before);
  }
  // open: ranges that reach beyond the start of the next one
  std::vector<Range> open;
  for (const Range &b : r) {
    size_t k = 0;
    for (const Range &a : open) {
      if (a.hi <= b.lo) continue;
      if ((a.written || b.written) && !disjoint_columns(a, b)) return FOPD_ERR_ALIAS;
      open[k++] = a;
    }
    open.resize(k);
    open.push_back(b);
  }
  return FOPD_OK;
}

}  // namespace fopd
