// Which tokens of a row stay, and their way together: the accepted path of a tree, and what a budget leaves of a long row.
//
// Tokens only ever move to lower places of their own row, in every layer, and what moves where is settled before anything moves.  A
// place may be both a source and a target, so the order matters: a thread moves the same 16 bytes of every token (path), or a block the
// same head of every token with a barrier between a piece's loads and its stores (eviction); no two blocks touch the same bytes.
//
// Bound: memory for the moves, latency for the choice (a few dependent passes over 4 bytes per place).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/csd.h"
#include "csd_common.cuh"
#include "csd_pages.cuh"
#include "csd_ptx.cuh"

namespace csd {
namespace keep {

using pages::View;

// Keys and values of a cache as the moves address them, in elements of two bytes.
struct Pool {
    char *k, *v;
    long long layer, page, head, token;    // strides in bytes
    int layers, heads, vecs;               // vecs: 16-byte vectors of a head
};

// ---- the accepted path -----------------------------------------------------------------------------------------

constexpr int kPathThreads = 128;

struct PathParams {
    View v;
    Pool pool;
    const int *accept_len, *path;
    int T;
};

// How many of the row's granted tokens stay: the accepted ones and the root, as far as the path names them in ascending order.  One
// warp; lane i and i + 32 hold entries i and i + 32 of the path.
__device__ __forceinline__ int path_kept(const PathParams &p, int r, int granted, int (&entry)[2], bool &bad)
{
    const int lane = threadIdx.x & 31;
    const int keep = min(max(ptx::ld_written(p.accept_len + r), -1), granted - 1) + 1;
    const int *path = p.path + static_cast<long long>(r) * p.T;
    int fine = 0;
    bool all = true;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = lane + 32 * k;
        entry[k] = i < p.T ? ptx::ld_written(path + i) : -1;
        const int before = i == 0 ? -1 : (i <= p.T ? ptx::ld_written(path + i - 1) : 0x7fffffff);
        const bool ok = i < keep && i < p.T && entry[k] > before && entry[k] >= 0 && entry[k] < granted;
        const unsigned int not_ok = __ballot_sync(kFull, !ok);
        if (all) fine += not_ok ? __ffs(not_ok) - 1 : 32;
        all = all && not_ok == 0u;
    }
    fine = min(fine, keep);
    bad = fine < keep;
    return fine;
}

// grid (blocks over a token's vectors in all layers, rows).  A thread owns one 16-byte vector of every token: it reads token path[i]'s before it
// writes token i's, in ascending i, and path[i] >= i, so what it still has to read is never overwritten.
__global__ void __launch_bounds__(kPathThreads) path_move_kernel(const PathParams p)
{
    __shared__ long long from_off[CSD_TREE_MAX_NODES], to_off[CSD_TREE_MAX_NODES];     // of the tokens that move
    __shared__ int n_moves;
    ptx::wait_for_stream();
    const int r = blockIdx.y, lane = threadIdx.x & 31;
    if (threadIdx.x < 32) {
        const int granted = p.v.granted[r], base = p.v.lens[r] - granted;
        const int *row = p.v.table + static_cast<long long>(r) * p.v.max_pages;
        int entry[2], at = 0;
        bool bad;
        const int n = granted > 0 ? path_kept(p, r, granted, entry, bad) : 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = lane + 32 * k;
            bool moves = i < n && entry[k] != i;
            long long from = 0, to = 0;
            if (moves) {
                const int a = base + entry[k], b = base + i;
                const int pa = row[a >> p.v.page_shift], pb = row[b >> p.v.page_shift];
                moves = pa >= 0 && pa < p.v.n_pages && pb >= 0 && pb < p.v.n_pages;
                if (!moves) atomicOr(p.v.flags, CSD_CACHE_BAD_PAGE);
                from = pa * p.pool.page + (a & (p.v.page_size - 1)) * p.pool.token;
                to = pb * p.pool.page + (b & (p.v.page_size - 1)) * p.pool.token;
            }
            const unsigned int m = __ballot_sync(kFull, moves);
            if (moves) {
                const int j = at + __popc(m & ((1u << lane) - 1u));
                from_off[j] = from;
                to_off[j] = to;
            }
            at += __popc(m);
        }
        if (lane == 0) n_moves = at;
    }
    __syncthreads();
    const int n = n_moves;
    if (n == 0) return;
    const int per_plane = p.pool.heads * p.pool.vecs, all = 2 * p.pool.layers * per_plane;
    for (int c = blockIdx.x * kPathThreads + threadIdx.x; c < all; c += gridDim.x * kPathThreads) {
        const int plane = c / per_plane, in_plane = c - plane * per_plane, h = in_plane / p.pool.vecs, vec = in_plane - h * p.pool.vecs;
        char *base = ((plane & 1) ? p.pool.v : p.pool.k) + (plane >> 1) * p.pool.layer + h * p.pool.head + vec * 16;
        for (int i = 0; i < n; i += 4) {
            uint4 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k < n) x[k] = ptx::ld_written(reinterpret_cast<const uint4 *>(base + from_off[i + k]));
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i + k < n) *reinterpret_cast<uint4 *>(base + to_off[i + k]) = x[k];
        }
    }
}

// The bookkeeping after the moves: a block per row.
__global__ void __launch_bounds__(pages::kRowThreads) path_commit_kernel(const PathParams p)
{
    __shared__ int kept;
    ptx::wait_for_stream();
    const int r = blockIdx.x;
    const int len = p.v.lens[r], granted = max(p.v.granted[r], 0);
    if (threadIdx.x < 32) {
        int entry[2];
        bool bad;
        const int n = path_kept(p, r, granted, entry, bad);
        if (threadIdx.x == 0) {
            kept = n;
            if (bad) atomicOr(p.v.flags, CSD_CACHE_BAD_PATH);
        }
    }
    __syncthreads();
    pages::shorten(p.v, r, len, len - granted + kept);
}

}  // namespace keep
}  // namespace csd
