// Trees of drafted tokens: who sees whom, and at which position.
//
//   node t of row b hangs from node parents[b,t] < t, or directly from the row's history where that is no node before it
//   masks[b,t]      bit u: u is t or one of the nodes it hangs from
//   positions[b,t]  lens[b] - n_new[b] + depth(t) + offset[b]: nodes of one depth are alternatives for one position
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/csd.h"
#include "csd_common.cuh"
#include "csd_ptx.cuh"

namespace csd {
namespace tree {

struct PlanParams {
    const int *parents;                    // null: a chain
    long long parent_stride;               // between rows; 0: one tree for all
    int T;
    const int *lens, *n_new, *offset;
    unsigned long long *masks;
    int *positions;
};

// A block per row, a thread per node.  Ancestors by doubling: six rounds reach the root of any tree of 64 nodes.  Latency alone, once per step.
__global__ void __launch_bounds__(CSD_TREE_MAX_NODES) plan_kernel(const PlanParams p)
{
    __shared__ unsigned long long seen[CSD_TREE_MAX_NODES];
    __shared__ int up[CSD_TREE_MAX_NODES];
    ptx::wait_for_stream();
    const int b = blockIdx.x, t = threadIdx.x;
    const int news = p.n_new ? max(ptx::ld_written(p.n_new + b), 0) : p.T;
    const bool there = t < p.T && t < news;
    int parent = -1;
    if (there) parent = p.parents ? ptx::ld_written(p.parents + b * p.parent_stride + t) : t - 1;
    if (parent >= t) parent = -1;
    unsigned long long mine = there ? 1ull << t : 0ull;
    seen[t] = mine;
    up[t] = parent;
    __syncthreads();
#pragma unroll 1
    for (int round = 0; round < 6; ++round) {
        if (parent >= 0) {
            mine |= seen[parent];
            parent = up[parent];
        }
        __syncthreads();
        seen[t] = mine;
        up[t] = parent;
        __syncthreads();
    }
    if (t >= p.T) return;
    const long long at = static_cast<long long>(b) * p.T + t;
    p.masks[at] = mine;
    if (p.positions)
        p.positions[at] = there ? ptx::ld_written(p.lens + b) - news + (p.offset ? ptx::ld_written(p.offset + b) : 0) + __popcll(mine) - 1 : 0;
}

}  // namespace tree
}  // namespace csd
