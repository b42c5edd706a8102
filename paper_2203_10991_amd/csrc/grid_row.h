// Workgroups in one row that may be longer than a dimension of a grid, which holds fewer than 2^32 threads: rows of 2^21 workgroups under each other.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

namespace nm {

constexpr int GRID_ROW_BITS = 21;            // (2^31 threads in workgroups of 1024)

// x and the number of rows for `wgs` workgroups, up to 2^31: the last row's last ones may be none
inline unsigned grid_row(int64_t wgs) { return (unsigned)std::min<int64_t>(wgs, 1 << GRID_ROW_BITS); }
inline unsigned grid_rows(int64_t wgs) { return (unsigned)((wgs + (1 << GRID_ROW_BITS) - 1) >> GRID_ROW_BITS); }
__device__ __forceinline__ uint32_t grid_place(uint32_t x, uint32_t row) { return row << GRID_ROW_BITS | x; }

}  // namespace nm
