// The last step of a bias gradient: the sum of its partial sums, by groups of rows.
#pragma once

#include "linear.h"

namespace morello {

constexpr int kSumColumns = 8;      // columns of a warp: 32 bytes, a sector, of every row of partial sums

// A warp takes kSumColumns columns of a group at a time, four lanes to a column: strided runs of the parts, then the
// four in lane order.  The same sums in the same order whoever calls it.
__device__ __forceinline__ void column_sums(const ColumnSums& c, int64_t warp, int64_t warps, int lane) {
  constexpr int kRuns = 32 / kSumColumns;
  const int64_t octets = (c.width + kSumColumns - 1) / kSumColumns;
  for (int64_t at = warp; at < c.groups * octets; at += warps) {
    const int64_t g = at / octets, col = (at - g * octets) * kSumColumns + lane % kSumColumns;
    int64_t first = 0, last = c.parts;
    if (c.offsets) {
      first = c.offsets[g] / kSlopeRows;
      last = first + (c.counts[g] + kSlopeRows - 1) / kSlopeRows;
    }
    float s = 0.f;
    if (col < c.width) {
#pragma unroll 4
      for (int64_t i = first + lane / kSumColumns; i < last; i += kRuns) s += c.partial[i * c.width + col];
    }
    float total = 0.f;
#pragma unroll
    for (int r = 0; r < kRuns; ++r) total += __shfl_sync(0xffffffffu, s, r * kSumColumns + lane % kSumColumns);
    if (lane < kSumColumns && col < c.width) {
      float* dst = c.db + g * c.width + col;
      *dst = c.accumulate ? *dst + total : total;
    }
  }
}

}  // namespace morello
