// Pieces shared by the expert-layer kernels: the row groups read from `ends`,
// the padded row positions of token planes, BF16 packing, and the host-side
// limits.
#pragma once

#include "../../include/emu_experts.h"
#include "common.cuh"

namespace emu {

constexpr int kMaxGroups = 1024;      // groups of one call: their bounds are kept in shared memory
constexpr int kRowPad = 16;           // a group's rows in padded planes start and end at multiples of one MMA's K

// First padded row of a group whose first row is `start`.  Groups never
// overlap: from one group to the next the position grows by
// ceil16(start + n) - ceil16(start) + 16, a multiple of 16 above n.
__host__ __device__ __forceinline__ int64_t padded_start(int64_t start, int g)
{
    return (start + kRowPad - 1) / kRowPad * kRowPad + (int64_t)kRowPad * g;
}
inline int64_t padded_rows(int64_t rows, int64_t G) { return padded_start(rows, (int)G) + kRowPad; }

// Group bounds in shared memory: starts[g] .. starts[g + 1] are the rows of
// group g, from `ends` clamped to [0, rows] and made non-decreasing, so that
// no value in `ends` can lead out of the row range.  Called by all threads of
// a block (blockDim.x >= 32); ends with a barrier.  Returns (in every thread)
// whether some entry had to be changed.
__device__ __forceinline__ bool load_groups(const int32_t *__restrict__ ends, int G, int rows, int *starts)
{
    bool bad = false;
    for (int g = threadIdx.x; g < G; g += blockDim.x) {
        const int e = ends[g];
        bad |= e < 0 || e > rows || (g > 0 && ends[g - 1] > e);
        starts[g + 1] = min(max(e, 0), rows);
    }
    if (threadIdx.x == 0) starts[0] = 0;
    const int any = __syncthreads_or(bad ? 1 : 0);
    if (any) {                                        // rare: running maximum of the bounds
        if (threadIdx.x == 0)
            for (int g = 1; g <= G; ++g) starts[g] = max(starts[g], starts[g - 1]);
        __syncthreads();
    }
    return any != 0;
}

// The group of row r: the g with bound[g] <= r < bound[g + 1] (bounds
// non-decreasing, bound[0] <= r < bound[G]).
__device__ __forceinline__ int find_group(const int *bound, int G, int r)
{
    int lo = 0, hi = G - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (r < bound[mid + 1]) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

}  // namespace emu
