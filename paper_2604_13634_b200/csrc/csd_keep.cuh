// Which tokens of a row stay, and their way together: the accepted path of a tree, and what a budget leaves of a long row.
//
// Tokens only ever move to lower places of their own row, in every layer, and what moves where is settled before anything moves.  A
// place may be both a source and a target, so the order matters: a thread moves the same 16 bytes of every token (path), or a block the
// same head of every token with a barrier between a piece's loads and its stores (eviction); no two blocks touch the same bytes.
//
// Bound: memory for the moves, latency for the choice (a few dependent passes over 4 bytes per place).  A path of one row in 32 layers takes 6.1 to 7.1 us,
// 64 paths in 28 layers 19.3 to 20.4 (35 MB read and written); cutting 16 rows of about 1021 tokens to 1008 in 16 layers 69 to 72 us, of
// which the moves of 147 MB read and written take 50 and the choice 11; 8 prompts of 6000 to 16384 to 4096 in 4 layers 151 to 155 us, 128 and 19.
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
using ptx::cluster_rank;
using ptx::cluster_size;
using ptx::st_cluster;

// Keys and values of a cache as the moves address them, in elements of two bytes.
struct Pool {
    char *k, *v;
    long long layer, page, head, token;    // strides in bytes
    int layers, heads, vecs;               // vecs: 16-byte vectors of a head
};

// Tokens of a row, as far as its table reaches: the arrays are the caller's memory, and what they say is bounded before it becomes an address.
__device__ __forceinline__ int row_len(const View &v, int r) { return min(max(ptx::ld_written(v.lens + r), 0), v.max_pages << v.page_shift); }

// ---- clusters ----

__device__ __forceinline__ unsigned int in_block(const void *mine, unsigned int rank) { return ptx::in_block(ptx::smem_u32(mine), rank); }
__device__ __forceinline__ void add_cluster(unsigned int addr, unsigned int v)
{
    asm volatile("red.shared::cluster.add.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
// All threads of all blocks of the cluster.
__device__ __forceinline__ void cluster_meet(unsigned int blocks)
{
    if (blocks == 1)
        __syncthreads();
    else
        ptx::cluster_meet();
}

// ---- the accepted path -----------------------------------------------------------------------------------------

constexpr int kPathThreads = 512, kPathBlocks = 8;      // blocks of a cluster, which has a row

struct PathParams {
    View v;
    Pool pool;
    const int *accept_len, *path;
    int T;
    float *mass;                           // null: none
    long long mass_stride;
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

// A cluster has a row.  A thread owns 16-byte vectors of every token: it reads token path[i]'s before it writes token i's, in ascending i, and
// path[i] >= i, so what it still has to read is never overwritten.  Every block works out for itself what moves where; once all have, the first
// does the bookkeeping, beside the moves: pages that it frees are only given away by later launches.
__global__ void __launch_bounds__(kPathThreads) path_kernel(const PathParams p)
{
    __shared__ long long from_off[CSD_TREE_MAX_NODES], to_off[CSD_TREE_MAX_NODES];     // of the tokens that move
    __shared__ int n_moves, n_kept;
    ptx::wait_for_stream();
    const unsigned int rank = cluster_rank();
    const int r = blockIdx.x / kPathBlocks, tid = threadIdx.x, lane = tid & 31;
    const int len = row_len(p.v, r), granted = min(max(ptx::ld_written(p.v.granted + r), 0), len);
    if (tid < 32) {
        const int base = len - granted;
        const int *row = p.v.table + static_cast<long long>(r) * p.v.max_pages;
        int entry[2], at = 0;
        bool bad;
        const int n = path_kept(p, r, granted, entry, bad);
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
        if (p.mass && rank == 0) {
            // the new tokens' masses go with them: all are read before one is written; those of the dropped ones become 0
            float *const mass = p.mass + r * p.mass_stride + base;
            float x[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) x[k] = lane + 32 * k < n ? mass[entry[k]] : 0.f;
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (lane + 32 * k < n) mass[lane + 32 * k] = x[k];
            for (int i = n + lane; i < granted; i += 32) mass[i] = 0.f;
        }
        if (lane == 0) {
            n_moves = at;
            n_kept = n;
            if (bad && rank == 0) atomicOr(p.v.flags, CSD_CACHE_BAD_PATH);
        }
    }
    cluster_meet(kPathBlocks);                       // no block reads the tables any more
    if (rank == 0) pages::shorten(p.v, r, len, len - granted + n_kept, kPathThreads);
    const int n = n_moves;
    if (n == 0) return;
    const int per_plane = p.pool.heads * p.pool.vecs, all = 2 * p.pool.layers * per_plane;
    for (int c = static_cast<int>(rank) * kPathThreads + tid; c < all; c += kPathBlocks * kPathThreads) {
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

// ---- a budget --------------------------------------------------------------------------------------------------
//
// A row of len > keep tokens keeps its first S (sinks), its last R (recent), and of the places between the W = keep - S - R with the
// largest mass (lowest place on ties).  New places: with F = S + W, the recent tokens become the last, F .. keep - 1, in order; a chosen
// place below F stays; the chosen places from F on (movers), in ascending order, fill the places below F that were not chosen (holes),
// in ascending order.  So as many tokens move as the row loses at most, and R.

constexpr int kPickThreads = 512, kPickWarps = kPickThreads / 32, kBins = 2048, kMostBlocks = 8;
constexpr int kKeys = 6144;                // keys that a block keeps in shared memory; a larger share is read again

struct RowPlan {
    int early, front;                      // pairs [0, early): movers from places below `keep`; [early, front): the others; then the recent tokens
    int from, to, recent;                  // which go from place `from` to place `to`
    int len, keep;                         // tokens before and after (equal: nothing happens)
};

struct EvictParams {
    View v;
    Pool pool;
    float *mass;
    long long mass_stride;
    const int *keep_rows;                  // null: `keep` for every row
    int keep, sinks, recent, width;        // width: columns of kept, pairs and offsets
    int *kept, *evicted;
    RowPlan *plans;                        // [rows]
    int2 *pairs;                           // [rows, width] mover, hole: places
    longlong2 *offsets;                    // [rows, width] where from and where to within a layer's pool, in bytes; -1: no such page
};

// Masses in descending order are keys in descending order; NaN below everything, one zero.
__device__ __forceinline__ unsigned int mass_key(float x)
{
    if (x != x) return 0u;
    const unsigned int u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
struct PickShared {
    unsigned int keys[kKeys];
    __align__(16) unsigned int mine[kBins];            // counts of this block, read four at a time
    __align__(16) unsigned int all[kBins];             // of the cluster (the first block's)
    unsigned int of_warp[kPickWarps][2], of_block[2][kMostBlocks][2];
    unsigned int found[3], refused[kMostBlocks], scan[kPickWarps];      // found: digit, how many with it are chosen, how many have it
};

// What the warps before this one, in all blocks before and in this, have counted (two counts at once), and everything.
__device__ __forceinline__ void before_me(PickShared &s, int &turn, unsigned int rank, unsigned int blocks, unsigned int a, unsigned int b, unsigned int (&before)[2],
                                          unsigned int (&total)[2])
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();
    if (lane == 0) {
        s.of_warp[warp][0] = a;
        s.of_warp[warp][1] = b;
    }
    __syncthreads();
    const unsigned int x = lane < kPickWarps ? s.of_warp[lane][0] : 0u, y = lane < kPickWarps ? s.of_warp[lane][1] : 0u;
    total[0] = __reduce_add_sync(kFull, x);
    total[1] = __reduce_add_sync(kFull, y);
    before[0] = __reduce_add_sync(kFull, lane < warp ? x : 0u);
    before[1] = __reduce_add_sync(kFull, lane < warp ? y : 0u);
    if (blocks == 1) return;
    if (warp == 0 && lane < static_cast<int>(blocks)) {
        const unsigned int to = in_block(s.of_block[turn][rank], lane);
        st_cluster(to, total[0]);
        st_cluster(to + 4, total[1]);
    }
    cluster_meet(blocks);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const unsigned int z = lane < static_cast<int>(blocks) ? s.of_block[turn][lane][k] : 0u;
        total[k] = __reduce_add_sync(kFull, z);
        before[k] += __reduce_add_sync(kFull, lane < static_cast<int>(rank) ? z : 0u);
    }
    turn ^= 1;
}

// Finds the key of the W-th largest of the M places from S on, and how many of those that have it are chosen: rounds over digits of 11, 11
// and 10 bits, fewer where a digit settles it.  A cluster of blocks has the row; each warp of it a run of the places.
__global__ void __launch_bounds__(kPickThreads) evict_pick_kernel(const EvictParams p)
{
    __shared__ PickShared s;
    const unsigned int rank = cluster_rank(), blocks = cluster_size();
    if (blocks > 1) ptx::cluster_arrive();                             // that all blocks run is waited for behind the stream
    ptx::wait_for_stream();
    const int r = blockIdx.x / blocks, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int len = row_len(p.v, r);
    int keep = min(max(p.keep_rows ? ptx::ld_written(p.keep_rows + r) : p.keep, 0), p.width);
    if (blocks > 1) {
        ptx::cluster_wait();
        // as the first block has read them: whatever another stream may do meanwhile, all blocks meet at the same barriers
        if (rank == 0 && tid < static_cast<int>(blocks)) {
            const unsigned int to = in_block(s.found, tid);
            st_cluster(to, static_cast<unsigned int>(len));
            st_cluster(to + 4, static_cast<unsigned int>(keep));
        }
        cluster_meet(blocks);
        len = static_cast<int>(s.found[0]);
        keep = static_cast<int>(s.found[1]);
    }
    int *const kept = p.kept + static_cast<long long>(r) * p.width;
    const int threads = static_cast<int>(blocks) * kPickThreads, my = static_cast<int>(rank) * kPickThreads + tid;
    if (len <= keep) {
        for (int i = my; i < p.width; i += threads) kept[i] = i < len ? i : -1;
        if (my == 0) {
            p.plans[r] = {0, 0, 0, 0, 0, len, len};
            p.evicted[r] = 0;
        }
        return;
    }
    const int R = min(max(p.recent, 0), keep), S = min(max(p.sinks, 0), keep - R), W = keep - S - R, F = S + W, M = len - R - S;
    const float *const mass = p.mass + r * p.mass_stride;
    const int warps = static_cast<int>(blocks) * kPickWarps, me = static_cast<int>(rank) * kPickWarps + warp;
    auto run_from = [&](int w) { return S + static_cast<int>(static_cast<long long>(M) * w / warps); };
    const int p0 = run_from(me), p1 = run_from(me + 1), b0 = run_from(static_cast<int>(rank) * kPickWarps), b1 = run_from(static_cast<int>(rank + 1) * kPickWarps);
    auto load = [&](int j) { return mass_key(__int_as_float(ptx::ld_written(reinterpret_cast<const int *>(mass) + j))); };
    const bool cached = b1 - b0 <= kKeys;
    if (cached && W > 0) {
        for (int j = p0 + lane; j < p1; j += 32 * 8) {
            unsigned int k[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) k[e] = j + 32 * e < p1 ? load(j + 32 * e) : 0u;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (j + 32 * e < p1) s.keys[j + 32 * e - b0] = k[e];
        }
        __syncwarp();                                                  // (a warp reads its own run alone)
    }
    auto key_at = [&](int j) { return cached ? s.keys[j - b0] : load(j); };

    // ---- the key that decides ----
    // places with a key above `prefix` (in the bits above `shift`) are chosen, and `left` of the `ties` that have it
    unsigned int prefix = 0u, left = static_cast<unsigned int>(W), ties = 0u;
    int shift = 0, turn = 0;
    if (W > 0) {
#pragma unroll 1
        for (int round = 0; round < 3; ++round) {
            const int bits = round == 2 ? 10 : 11;
            const unsigned int above = round == 0 ? 0u : 0xffffffffu << (round == 1 ? 21 : 10);
            shift = round == 0 ? 21 : (round == 1 ? 10 : 0);
            for (int i = tid; i < kBins; i += kPickThreads) s.mine[i] = s.all[i] = 0u;
            cluster_meet(blocks);
            for (int j = p0 + lane; j < p1; j += 32 * 8) {
                unsigned int k[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) k[e] = j + 32 * e < p1 ? key_at(j + 32 * e) : 0u;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (j + 32 * e < p1 && (k[e] & above) == prefix) atomicAdd(&s.mine[(k[e] >> shift) & ((1u << bits) - 1u)], 1u);
            }
            __syncthreads();
            if (blocks > 1) {
                for (int i = tid; i < kBins; i += kPickThreads)
                    if (s.mine[i]) add_cluster(in_block(&s.all[i], 0), s.mine[i]);
                cluster_meet(blocks);
            }
            if (rank == 0) {
                // from the highest bin down: thread t has bins 4 t' .. 4 t' + 3 with t' = 511 - t
                const unsigned int *const count = blocks == 1 ? s.mine : s.all;
                const int c0 = 4 * (kPickThreads - 1 - tid);
                const uint4 q = *reinterpret_cast<const uint4 *>(count + c0);
                const unsigned int c[4] = {q.w, q.z, q.y, q.x};
                const unsigned int sum = c[0] + c[1] + c[2] + c[3];
                unsigned int inc = sum;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const unsigned int o = __shfl_up_sync(kFull, inc, d);
                    if (lane >= d) inc += o;
                }
                if (lane == 31) s.scan[warp] = inc;
                __syncthreads();
                unsigned int at = inc - sum + __reduce_add_sync(kFull, lane < warp ? s.scan[lane] : 0u);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (at < left && left <= at + c[e]) {                      // one thread and bin
                        for (unsigned int b = 0; b < blocks; ++b) {
                            const unsigned int to = in_block(s.found, b);
                            st_cluster(to, static_cast<unsigned int>(c0 + 3 - e));
                            st_cluster(to + 4, left - at);
                            st_cluster(to + 8, c[e]);
                        }
                    }
                    at += c[e];
                }
            }
            cluster_meet(blocks);
            prefix |= s.found[0] << shift;
            left = s.found[1];
            ties = s.found[2];
            if (left == ties) break;                                       // all of them: what follows the digit does not matter
        }
    }
    unsigned int before[2], total[2], first_tie = 0u;
    const bool all_ties = left == ties;                                    // (W = 0: nothing is chosen)
    if (!all_ties) {
        unsigned int mine = 0u;
        for (int j = p0 + lane; j < p1; j += 32) mine += key_at(j) == prefix ? 1u : 0u;
        before_me(s, turn, rank, blocks, __reduce_add_sync(kFull, mine), 0u, before, total);
        first_tie = before[0];
    }
    const unsigned int digits = prefix >> shift;
    auto walk = [&](auto visit) {
        unsigned int tie = first_tie;
        for (int j0 = p0; j0 < p1; j0 += 32) {
            const int j = j0 + lane;
            const unsigned int k = j < p1 && W > 0 ? key_at(j) >> shift : 0u;
            bool chosen = j < p1 && W > 0 && (all_ties ? k >= digits : k > digits);
            if (!all_ties) {
                const bool same = j < p1 && k == digits;
                const unsigned int m = __ballot_sync(kFull, same);
                if (same && tie + __popc(m & ((1u << lane) - 1u)) < left) chosen = true;
                tie += __popc(m);
            }
            visit(j, j < p1 && !chosen && j < F, chosen && j >= F, chosen && j < F);
        }
    };
    // ---- holes and movers counted; are the pages that would be written the row's own? ----
    const int *const table = p.v.table + static_cast<long long>(r) * p.v.max_pages;
    auto own_page = [&](int place) {
        const int page = table[place >> p.v.page_shift];
        return page < 0 || page >= p.v.n_pages || p.v.refs[page] <= 1;        // (no page: nothing will be written)
    };
    unsigned int holes = 0u, movers = 0u;
    bool foreign = false;
    walk([&](int j, bool hole, bool mover, bool) {
        holes += __popc(__ballot_sync(kFull, hole));
        movers += __popc(__ballot_sync(kFull, mover));
        if (hole) foreign |= !own_page(j);
    });
    for (int i = (F >> p.v.page_shift) + my; i << p.v.page_shift < keep && R > 0; i += threads) foreign |= !own_page(i << p.v.page_shift);
    const int refuse_here = __syncthreads_or(foreign ? 1 : 0);
    if (tid < static_cast<int>(blocks)) st_cluster(in_block(&s.refused[rank], tid), static_cast<unsigned int>(refuse_here));
    before_me(s, turn, rank, blocks, holes, movers, before, total);
    bool refused = false;
    for (unsigned int q = 0; q < blocks; ++q) refused |= s.refused[q] != 0u;
    if (refused) {
        for (int i = my; i < p.width; i += threads) kept[i] = i < len ? i : -1;
        if (my == 0) {
            atomicOr(p.v.flags, CSD_CACHE_SHARED);
            p.plans[r] = {0, 0, 0, 0, 0, len, len};
            p.evicted[r] = 0;
        }
        return;
    }
    // ---- where everything goes ----
    int2 *const pairs = p.pairs + static_cast<long long>(r) * p.width;
    longlong2 *const offsets = p.offsets + static_cast<long long>(r) * p.width;
    const int front = static_cast<int>(total[1]);
    bool lost = false;
    auto offset_of = [&](int place) -> long long {
        const int page = table[place >> p.v.page_shift];
        if (page < 0 || page >= p.v.n_pages) {
            lost = true;
            return -1;
        }
        return page * p.pool.page + (place & (p.v.page_size - 1)) * p.pool.token;
    };
    unsigned int hole_at = before[0], mover_at = before[1];
    walk([&](int j, bool hole, bool mover, bool stays) {
        const unsigned int mh = __ballot_sync(kFull, hole), mm = __ballot_sync(kFull, mover), below = (1u << lane) - 1u;
        if (hole) {
            const int at = hole_at + __popc(mh & below);
            __stcg(&pairs[at].y, j);
            __stcg(&offsets[at].y, offset_of(j));
        }
        if (mover) {
            const int at = mover_at + __popc(mm & below);
            __stcg(&pairs[at].x, j);
            __stcg(&offsets[at].x, offset_of(j));
        }
        if (stays) kept[j] = j;
        if (j == keep && j < p1) p.plans[r].early = static_cast<int>(mover_at) + __popc(mm & below);     // (the warp whose run has that place)
        hole_at += __popc(mh);
        mover_at += __popc(mm);
    });
    for (int i = my; i < S; i += threads) kept[i] = i;
    for (int i = F + my; i < p.width; i += threads) kept[i] = i < keep ? len - keep + i : -1;
    for (int i = my; i < R; i += threads) {
        longlong2 o;
        o.x = offset_of(len - R + i);
        o.y = offset_of(F + i);
        offsets[front + i] = o;
    }
    if (lost) atomicOr(p.v.flags, CSD_CACHE_BAD_PAGE);
    if (my == 0) {
        RowPlan *const plan = p.plans + r;
        if (keep >= len - R) plan->early = front;                           // every mover comes from below `keep`
        plan->front = front;
        plan->from = len - R;
        plan->to = F;
        plan->recent = R;
        plan->len = len;
        plan->keep = keep;
        p.evicted[r] = len - keep;
    }
    cluster_meet(blocks);
    for (int i = my; i < front; i += threads) {
        const int2 m = __ldcg(pairs + i);
        kept[m.y] = m.x;
    }
}

// The moves.  Movers from places beyond the row's new end can go at any time, in any number of blocks: nothing else touches where they come
// from or go to.  The others make room for the recent tokens and go before these: a team of threads does both for one head of the keys or values of one
// layer of one row, first those movers, then, after a barrier, the recent tokens in pieces: a piece's loads, a barrier, its stores.  A team is a
// warp where there are warps' worth of such heads (16 rows of 16 layers with 8 heads: 69 us for the call, 81 with blocks), else a block (8 rows of 4
// layers: 150, with warps 182).  Loads in flight per thread and blocks per SM: 8 and 2, 4 and 4 (exchanged: 74 and 154).
constexpr int kMoveThreads = 256;
template <int kTeam>
constexpr int kMoveBlocks = kTeam == 32 ? 2 : 4;     // per SM

template <int kTeam>
__global__ void __launch_bounds__(kMoveThreads, kMoveBlocks<kTeam>) evict_move_kernel(const EvictParams p)
{
    __shared__ int active[CSD_CACHE_MAX_ROWS];
    __shared__ int of_warp[kMoveThreads / 32];
    ptx::wait_for_stream();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // the rows that lose tokens, in order
    int n_active = 0;
    for (int r0 = 0; r0 < p.v.rows; r0 += kMoveThreads) {
        const int r = r0 + tid;
        const bool on = r < p.v.rows && ptx::ld_written(&p.plans[r].len) != ptx::ld_written(&p.plans[r].keep);
        const unsigned int m = __ballot_sync(kFull, on);
        if (lane == 0) of_warp[warp] = __popc(m);
        __syncthreads();
        int at = n_active;
        for (int w = 0; w < kMoveThreads / 32; ++w) {
            if (w < warp) at += of_warp[w];
            n_active += of_warp[w];
        }
        if (on) active[at + __popc(m & ((1u << lane) - 1u))] = r;
        __syncthreads();
    }
    const int units = 2 * p.pool.layers * p.pool.heads + 1;
    const int mine = tid % kTeam;
    const int tokens = kTeam / p.pool.vecs, sub = mine / p.pool.vecs, vec = mine - sub * p.pool.vecs;       // tokens of a piece
    const bool works = sub < tokens;
    auto team_sync = [&]() {
        if constexpr (kTeam == 32)
            __syncwarp();
        else
            __syncthreads();
    };
    // a unit's late movers are shared out over so many teams that all have something to do
    constexpr int kTeams = kMoveThreads / kTeam, kMoveAtOnce = kTeam == 32 ? 8 : 4;
    const long long teams = static_cast<long long>(gridDim.x) * kTeams, whole = static_cast<long long>(n_active) * units;
    const int parts = whole > 0 ? static_cast<int>(min(max(2 * teams / whole, 1ll), 8ll)) : 1;
    for (long long w = static_cast<long long>(blockIdx.x) * kTeams + tid / kTeam; w < whole * parts; w += teams) {
        const int part = static_cast<int>(w / whole);
        const long long w1 = w - part * whole;
        const int r = active[w1 / units], unit = static_cast<int>(w1 % units);
        const RowPlan plan = p.plans[r];
        if (unit == units - 1) {
            if (part != 0) continue;
            const int2 *const pairs = p.pairs + static_cast<long long>(r) * p.width;
            float *const mass = p.mass + r * p.mass_stride;
            for (int i = mine; i < plan.front; i += kTeam) {
                const int2 m = pairs[i];
                mass[m.y] = mass[m.x];
            }
            team_sync();
            for (int i0 = 0; i0 < plan.recent; i0 += kTeam) {
                const int i = i0 + mine;
                const float x = i < plan.recent ? mass[plan.from + i] : 0.f;
                team_sync();
                if (i < plan.recent) mass[plan.to + i] = x;
            }
            team_sync();
            for (int i = plan.keep + mine; i < plan.len; i += kTeam) mass[i] = 0.f;
            continue;
        }
        const int plane = unit / p.pool.heads, h = unit - plane * p.pool.heads;
        char *const base = ((plane & 1) ? p.pool.v : p.pool.k) + (plane >> 1) * p.pool.layer + h * p.pool.head + vec * 16;
        const longlong2 *const offsets = p.offsets + static_cast<long long>(r) * p.width;
        // pairs [first, end) in turn: the early movers, the recent tokens, this block's share of the late movers.  The next offsets are fetched ahead; of
        // the recent tokens no thread stores before all have loaded.
        for (int phase = part == 0 ? 0 : 2; phase < 3; ++phase) {
            int first = 0, end = plan.early;
            if (phase == 1) {
                team_sync();
                first = plan.front;
                end = plan.front + plan.recent;
            } else if (phase == 2) {
                const int late = plan.front - plan.early, shares = parts == 1 ? 1 : parts - 1, share = parts == 1 ? 0 : part - 1;
                if (share < 0) break;
                first = plan.early + static_cast<int>(static_cast<long long>(late) * share / shares);
                end = plan.early + static_cast<int>(static_cast<long long>(late) * (share + 1) / shares);
            }
            longlong2 o[kMoveAtOnce];
            auto fetch = [&](int i0) {
#pragma unroll
                for (int k = 0; k < kMoveAtOnce; ++k) {
                    const int i = i0 + k * tokens + sub;
                    o[k] = make_longlong2(-1, -1);
                    if (works && i < end) o[k] = offsets[i];
                }
            };
            fetch(first);
            for (int i0 = first; i0 < end; i0 += tokens * kMoveAtOnce) {
                uint4 x[kMoveAtOnce];
                long long to[kMoveAtOnce];
#pragma unroll
                for (int k = 0; k < kMoveAtOnce; ++k) {
                    to[k] = o[k].x >= 0 ? o[k].y : -1;
                    if (to[k] >= 0) x[k] = ptx::ld_written_once(base + o[k].x);
                }
                fetch(i0 + tokens * kMoveAtOnce);
                if (phase == 1) team_sync();
#pragma unroll
                for (int k = 0; k < kMoveAtOnce; ++k)
                    if (to[k] >= 0) *reinterpret_cast<uint4 *>(base + to[k]) = x[k];
            }
        }
    }
}

// The bookkeeping after the moves: a block per row.
__global__ void __launch_bounds__(pages::kRowThreads) evict_finish_kernel(const EvictParams p)
{
    ptx::wait_for_stream();
    const int r = blockIdx.x;
    const int len = ptx::ld_written(&p.plans[r].len), keep = ptx::ld_written(&p.plans[r].keep);
    pages::shorten(p.v, r, len, keep);
}

}  // namespace keep
}  // namespace csd
