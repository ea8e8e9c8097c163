// Lists of tensors that travel with a launch's arguments, and sums over a block, for the kernels that work on many tensors.
#pragma once
#include "st_common.hpp"

namespace st {

// The last tensor that begins at or before the tile (tensors without values own no tile and are not in the list).  Every lane looks at a
// few of them: one trip to memory, where a search by halves takes one after the other.
template <int MOST> __device__ __forceinline__ int tensor_of(const unsigned* first, int n, unsigned tile)
{
    const int lane = threadIdx.x & 63;
    int before = 0;
#pragma unroll
    for (int c = 0; c < MOST; c += 64) {
        const bool there = c + lane < n;
        before += __popcll(__ballot(there && first[there ? c + lane : 0] <= tile));
    }
    return before - 1;
}

__device__ __forceinline__ double block_sum(double s, double* sums)      // of 256 threads, in one order; to every thread
{
#pragma unroll
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    return (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

}  // namespace st
