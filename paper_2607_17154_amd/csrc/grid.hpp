// Launches of any number of workgroups.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ordermoe {

// The grid of n workgroups of at most 512 threads.  A launch has fewer than 2^32 threads
// along an axis, so past 2^22 workgroups (2^31 threads) they go along two.
inline dim3 grid_of(int64_t n) {
    const int64_t rows = (n + (1 << 22) - 1) >> 22;
    return rows <= 1 ? dim3((unsigned)n) : dim3((unsigned)((n + rows - 1) / rows), (unsigned)rows);
}
// a workgroup's number in it (the last ones may lie past n)
__device__ inline uint32_t block_number() { return blockIdx.y * gridDim.x + blockIdx.x; }

}  // namespace ordermoe
