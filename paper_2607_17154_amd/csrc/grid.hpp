// Launches of any number of workgroups.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ordermoe {

// The grid of n workgroups of at most 512 threads.  A launch has fewer than 2^32 threads
// along an axis, so past 2^22 workgroups (2^31 threads) they go along two.
constexpr int GRID_ROW = 22;
inline dim3 grid_of(int64_t n) {
    const int64_t row = (int64_t)1 << GRID_ROW;
    return n <= row ? dim3((unsigned)n) : dim3((unsigned)row, (unsigned)((n + row - 1) / row));
}
// A workgroup's number in it (those of the last row may lie past n).  Rows have a fixed length:
// reading gridDim costs a small kernel a memory access before its first address.
__device__ inline uint32_t block_number() { return (blockIdx.y << GRID_ROW) + blockIdx.x; }

}  // namespace ordermoe
