// Device-side view of a batch of sequences: which sequence a row belongs to, where
// a key lies.  Whatever the tables hold, no access leaves its operand: row and key
// ranges are clamped to the call's, page numbers to the cache's.
#pragma once
#include "common.h"
#include "kernels.h"

namespace dif {

// Rows [lo, hi) of sequence s, within the call's.
__device__ __forceinline__ void seq_rows(const KeyView& kv, int s, int* lo, int* hi) {
  *lo = min(max(kv.row_off[s], 0), kv.rows);
  *hi = min(max(kv.row_off[s + 1], *lo), kv.rows);
}

// The sequence that row `row` belongs to (ascending offsets): the last one whose rows
// begin at or before it, found by the 64 lanes together, 64 offsets a step.
__device__ __forceinline__ int seq_of_row(const KeyView& kv, int row) {
  const int lane = threadIdx.x & 63;
  int base = 0, n = kv.n_seqs;
  while (n > 64) {
    const int step = (n + 63) / 64, at = lane * step;
    const bool before = at < n && kv.row_off[base + at] <= row;
    const int last = max((int)__popcll(__ballot(before)) - 1, 0);
    base += last * step;
    n = min(step, n - last * step);
  }
  const bool before = lane < n && kv.row_off[base + lane] <= row;
  return base + max((int)__popcll(__ballot(before)) - 1, 0);
}

}  // namespace dif
