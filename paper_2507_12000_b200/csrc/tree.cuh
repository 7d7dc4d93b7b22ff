// A sequence's drafted tree in shared memory (sm_100a).
#pragma once

#include "dssd_device.cuh"

namespace dssd {

constexpr int kMaxNodes = DSSD_TREE_MAX_NODES;

// parent[j] for j = 1 .. N-1: the node above, or -1 where there is no node j; parent[0] = 0.  A node whose parent is not below it, or not
// there, is not there either; *bad is then set.  All threads of the CTA (at least N) call it; ends with a barrier.
__device__ __forceinline__ void load_tree(const int32_t *parents, long long b, int N, short *parent, int *bad)
{
    const int t = threadIdx.x;
    if (t == 0) *bad = 0;
    __syncthreads();
    if (t < N) {
        int p = t - 1;
        if (t > 0 && parents) {
            p = ld_after(parents + b * (N - 1) + t - 1);
            if (p >= t) {
                *bad = 1;  // (every writer stores the same value)
                p = -1;
            }
        }
        parent[t] = (short)(t == 0 ? 0 : (p < 0 ? -1 : p));
    }
    __syncthreads();
    // up to the root: parents are below their nodes, so this ends
    int up = t < N ? t : 0;
    while (up > 0) up = parent[up];
    __syncthreads();
    if (t < N && up < 0 && parent[t] >= 0) {
        *bad = 1;
        parent[t] = -1;
    }
    __syncthreads();
}

}  // namespace dssd
