// row_parts.hpp -- how a sum over rows is divided into K steps and parts (plain C++, for the host and the kernels).
//
// There may be 2^31 - 1 rows: whole steps of them end past what an int holds, so their ends are counted unsigned.
#pragma once
#include <stdint.h>

#include "plan_types.hpp"

namespace moe {

// K steps of n elements, the last one perhaps not full.
constexpr int steps_of(int n) { return (int)(((uint32_t)n + kTileK - 1) / kTileK); }

struct RowPart {
  int row0, rows;
};

// Part `part` of the rows [lo, hi) in `split` parts of whole K steps, of which the last ones may be empty.
constexpr RowPart row_part(int lo, int hi, int split, int part) {
  const uint32_t n = (uint32_t)hi - (uint32_t)lo, each = ((uint32_t)steps_of((int)n) + (uint32_t)split - 1) / (uint32_t)split * kTileK;
  const uint32_t before = (uint32_t)part * each, skip = before < n ? before : n;
  return RowPart{lo + (int)skip, (int)(each < n - skip ? each : n - skip)};
}

// Which of n rows is element `lane` of K step `step`: the last step starts early, so that it ends with the rows, and with
// fewer rows than a step's it repeats the last one, as a step past the last one does.
constexpr int row_of_step(int step, int lane, int n) {
  const uint32_t from = (uint32_t)step * kTileK, last = n > kTileK ? (uint32_t)n - kTileK : 0;
  const uint32_t at = (from < last ? from : last) + (uint32_t)lane;
  return (int)(at < (uint32_t)n ? at : (uint32_t)n - 1);
}

}  // namespace moe
