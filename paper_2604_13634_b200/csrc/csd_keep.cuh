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

// ---- a budget --------------------------------------------------------------------------------------------------
//
// A row of len > keep tokens keeps its first S (sinks), its last R (recent), and of the places between the W = keep - S - R with the
// largest mass (lowest place on ties).  New places: with F = S + W, the recent tokens become the last, F .. keep - 1, in order; a chosen
// place below F stays; the chosen places from F on (movers), in ascending order, fill the places below F that were not chosen (holes),
// in ascending order.  So as many tokens move as the row loses at most, and R.

constexpr int kPickThreads = 512, kPickWarps = kPickThreads / 32, kBins = 2048, kMostBlocks = 8;

struct RowPlan {
    int front;                             // movers; pairs[0 .. front)
    int from, to, recent;                  // the last `recent` tokens go from place `from` to place `to`
    int len, keep;                         // tokens before and after (equal: nothing happens)
};

struct EvictParams {
    View v;
    Pool pool;
    float *mass;
    long long mass_stride;
    const int *keep_rows;                  // null: `keep` for every row
    int keep, sinks, recent, width;        // width: columns of kept and of pairs
    int *kept, *evicted;
    RowPlan *plans;                        // [rows]
    int2 *pairs;                           // [rows, width] mover, hole
};

// Masses in descending order are keys in descending order; NaN below everything, one zero.
__device__ __forceinline__ unsigned int mass_key(float x)
{
    if (x != x) return 0u;
    const unsigned int u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ unsigned int cluster_rank()
{
    unsigned int r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ unsigned int cluster_size()
{
    unsigned int r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ unsigned int in_block(const void *mine, unsigned int rank)
{
    unsigned int r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(ptx::smem_u32(mine)), "r"(rank));
    return r;
}
__device__ __forceinline__ void st_cluster(unsigned int addr, unsigned int v)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void add_cluster(unsigned int addr, unsigned int v)
{
    asm volatile("red.shared::cluster.add.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
// All threads of all blocks of the cluster; also the block's own barrier.
__device__ __forceinline__ void cluster_meet()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

struct PickShared {
    unsigned int mine[kBins], all[kBins];              // counts of this block; of the cluster (the first block's)
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
    if (warp == 0) {
        const unsigned int x = __reduce_add_sync(kFull, lane < kPickWarps ? s.of_warp[lane][0] : 0u), y = __reduce_add_sync(kFull, lane < kPickWarps ? s.of_warp[lane][1] : 0u);
        if (lane < static_cast<int>(blocks)) {
            const unsigned int to = in_block(s.of_block[turn][rank], lane);
            st_cluster(to, x);
            st_cluster(to + 4, y);
        }
    }
    cluster_meet();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        before[k] = total[k] = 0u;
        for (unsigned int r = 0; r < blocks; ++r) {
            total[k] += s.of_block[turn][r][k];
            if (r < rank) before[k] += s.of_block[turn][r][k];
        }
        for (int w = 0; w < warp; ++w) before[k] += s.of_warp[w][k];
    }
    turn ^= 1;
}

// Finds the key of the W-th largest of the places [first, first + n) and how many of those that have it are chosen: three rounds over
// digits of 11, 11 and 10 bits.  A cluster of blocks has the row; each warp of it a run of the places.
__global__ void __launch_bounds__(kPickThreads) evict_pick_kernel(const EvictParams p)
{
    __shared__ PickShared s;
    ptx::wait_for_stream();
    const unsigned int rank = cluster_rank(), blocks = cluster_size();
    const int r = blockIdx.x / blocks, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int len = p.v.lens[r];
    const int keep = min(max(p.keep_rows ? ptx::ld_written(p.keep_rows + r) : p.keep, 0), p.width);
    int *const kept = p.kept + static_cast<long long>(r) * p.width;
    const int threads = static_cast<int>(blocks) * kPickThreads, my = static_cast<int>(rank) * kPickThreads + tid;
    if (len <= keep) {
        for (int i = my; i < p.width; i += threads) kept[i] = i < len ? i : -1;
        if (my == 0) {
            p.plans[r] = {0, 0, 0, 0, len, len};
            p.evicted[r] = 0;
        }
        return;
    }
    const int R = min(max(p.recent, 0), keep), S = min(max(p.sinks, 0), keep - R), W = keep - S - R, F = S + W, M = len - R - S;
    const float *const mass = p.mass + r * p.mass_stride;
    const int warps = static_cast<int>(blocks) * kPickWarps, me = static_cast<int>(rank) * kPickWarps + warp;
    const int p0 = S + static_cast<int>(static_cast<long long>(M) * me / warps), p1 = S + static_cast<int>(static_cast<long long>(M) * (me + 1) / warps);
    auto key_at = [&](int j) { return mass_key(__int_as_float(ptx::ld_written(reinterpret_cast<const int *>(mass) + j))); };

    // ---- the key that decides ----
    unsigned int prefix = 0u, left = static_cast<unsigned int>(W), ties = 0u;        // of the places with this prefix, `left` are chosen
    int turn = 0;
    if (W > 0) {
#pragma unroll 1
        for (int round = 0; round < 3; ++round) {
            const int shift = round == 0 ? 21 : (round == 1 ? 10 : 0), bits = round == 2 ? 10 : 11;
            const unsigned int above = round == 0 ? 0u : 0xffffffffu << (shift + bits);
            for (int i = tid; i < kBins; i += kPickThreads) s.mine[i] = s.all[i] = 0u;
            cluster_meet();
            for (int j = p0 + lane; j < p1; j += 32 * 8) {
                unsigned int k[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) k[e] = j + 32 * e < p1 ? key_at(j + 32 * e) : 0u;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (j + 32 * e < p1 && (k[e] & above) == prefix) atomicAdd(&s.mine[(k[e] >> shift) & ((1u << bits) - 1u)], 1u);
            }
            __syncthreads();
            for (int i = tid; i < kBins; i += kPickThreads)
                if (s.mine[i]) add_cluster(in_block(&s.all[i], 0), s.mine[i]);
            cluster_meet();
            if (rank == 0) {
                // from the highest bin down: thread t has bins 4 t' .. 4 t' + 3 with t' = 511 - t
                const int b0 = 4 * (kPickThreads - 1 - tid);
                const unsigned int c[4] = {s.all[b0 + 3], s.all[b0 + 2], s.all[b0 + 1], s.all[b0]};
                const unsigned int sum = c[0] + c[1] + c[2] + c[3];
                unsigned int inc = sum;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const unsigned int o = __shfl_up_sync(kFull, inc, d);
                    if (lane >= d) inc += o;
                }
                if (lane == 31) s.scan[warp] = inc;
                __syncthreads();
                unsigned int at = inc - sum;
                for (int w = 0; w < warp; ++w) at += s.scan[w];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (at < left && left <= at + c[e]) {                      // one thread and bin
                        for (unsigned int q = 0; q < blocks; ++q) {
                            const unsigned int to = in_block(s.found, q);
                            st_cluster(to, static_cast<unsigned int>(b0 + 3 - e));
                            st_cluster(to + 4, left - at);
                            st_cluster(to + 8, c[e]);
                        }
                    }
                    at += c[e];
                }
            }
            cluster_meet();
            prefix |= s.found[0] << shift;
            left = s.found[1];
            ties = s.found[2];
        }
    }
    // a place is chosen if its key is above `prefix`, or is it and fewer than `left` such places come before it
    unsigned int before[2], total[2], first_tie = 0u;
    const bool all_ties = W > 0 && left == ties;
    if (W > 0 && !all_ties) {
        unsigned int mine = 0u;
        for (int j = p0 + lane; j < p1; j += 32) mine += key_at(j) == prefix ? 1u : 0u;
        before_me(s, turn, rank, blocks, __reduce_add_sync(kFull, mine), 0u, before, total);
        first_tie = before[0];
    }
    auto walk = [&](auto visit) {
        unsigned int tie = first_tie;
        for (int j0 = p0; j0 < p1; j0 += 32) {
            const int j = j0 + lane;
            const unsigned int k = j < p1 && W > 0 ? key_at(j) : 0u;
            const bool same = j < p1 && W > 0 && k == prefix;
            const unsigned int m = __ballot_sync(kFull, same);
            const bool chosen = j < p1 && W > 0 && (k > prefix || (same && (all_ties || tie + __popc(m & ((1u << lane) - 1u)) < left)));
            tie += __popc(m);
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
            p.plans[r] = {0, 0, 0, 0, len, len};
            p.evicted[r] = 0;
        }
        return;
    }
    // ---- where everything goes ----
    int2 *const pairs = p.pairs + static_cast<long long>(r) * p.width;
    unsigned int hole_at = before[0], mover_at = before[1];
    walk([&](int j, bool hole, bool mover, bool stays) {
        const unsigned int mh = __ballot_sync(kFull, hole), mm = __ballot_sync(kFull, mover), below = (1u << lane) - 1u;
        if (hole) __stcg(&pairs[hole_at + __popc(mh & below)].y, j);
        if (mover) __stcg(&pairs[mover_at + __popc(mm & below)].x, j);
        if (stays) kept[j] = j;
        hole_at += __popc(mh);
        mover_at += __popc(mm);
    });
    for (int i = my; i < S; i += threads) kept[i] = i;
    for (int i = F + my; i < p.width; i += threads) kept[i] = i < keep ? len - keep + i : -1;
    if (my == 0) {
        p.plans[r] = {static_cast<int>(total[1]), len - R, F, R, len, keep};
        p.evicted[r] = len - keep;
    }
    cluster_meet();
    for (int i = my; i < static_cast<int>(total[1]); i += threads) {
        const int2 m = __ldcg(pairs + i);
        kept[m.y] = m.x;
    }
}

// The moves: a block has one head of the keys or values of one layer of one row (or the row's masses) at a time.  First the movers, whose
// targets nothing else reads; then, after a barrier, the recent tokens in pieces: a piece's loads, a barrier, its stores.
constexpr int kMoveThreads = 256, kMoveAtOnce = 4;

__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const EvictParams p)
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
    const int tokens = kMoveThreads / p.pool.vecs, sub = tid / p.pool.vecs, vec = tid - sub * p.pool.vecs;       // tokens of a piece
    for (long long w = blockIdx.x; w < static_cast<long long>(n_active) * units; w += gridDim.x) {
        const int r = active[w / units], unit = static_cast<int>(w % units);
        const RowPlan plan = p.plans[r];
        const int2 *const pairs = p.pairs + static_cast<long long>(r) * p.width;
        if (unit == units - 1) {
            float *const mass = p.mass + r * p.mass_stride;
            for (int i = tid; i < plan.front; i += kMoveThreads) {
                const int2 m = pairs[i];
                mass[m.y] = mass[m.x];
            }
            __syncthreads();
            for (int i0 = 0; i0 < plan.recent; i0 += kMoveThreads) {
                const int i = i0 + tid;
                const float x = i < plan.recent ? mass[plan.from + i] : 0.f;
                __syncthreads();
                if (i < plan.recent) mass[plan.to + i] = x;
            }
            __syncthreads();
            for (int i = plan.keep + tid; i < plan.len; i += kMoveThreads) mass[i] = 0.f;
            continue;
        }
        const int plane = unit / p.pool.heads, h = unit - plane * p.pool.heads;
        char *const base = ((plane & 1) ? p.pool.v : p.pool.k) + (plane >> 1) * p.pool.layer + h * p.pool.head + vec * 16;
        const int *const table = p.v.table + static_cast<long long>(r) * p.v.max_pages;
        auto slot = [&](int place) -> char * {
            const int page = table[place >> p.v.page_shift];
            return page < 0 || page >= p.v.n_pages ? nullptr : base + page * p.pool.page + (place & (p.v.page_size - 1)) * p.pool.token;
        };
        bool lost = false;
        uint4 x[kMoveAtOnce];
        for (int i0 = 0; i0 < plan.front; i0 += tokens * kMoveAtOnce) {
            char *to[kMoveAtOnce];
#pragma unroll
            for (int k = 0; k < kMoveAtOnce; ++k) {
                const int i = i0 + k * tokens + sub;
                to[k] = nullptr;
                if (sub < tokens && i < plan.front) {
                    const int2 m = pairs[i];
                    const char *from = slot(m.x);
                    to[k] = slot(m.y);
                    if (!from) to[k] = nullptr;
                    lost |= !to[k];
                    if (to[k]) x[k] = ptx::ld_written_once(from);
                }
            }
#pragma unroll
            for (int k = 0; k < kMoveAtOnce; ++k)
                if (to[k]) *reinterpret_cast<uint4 *>(to[k]) = x[k];
        }
        __syncthreads();
        for (int i0 = 0; i0 < plan.recent; i0 += tokens * kMoveAtOnce) {
            char *to[kMoveAtOnce];
#pragma unroll
            for (int k = 0; k < kMoveAtOnce; ++k) {
                const int i = i0 + k * tokens + sub;
                to[k] = nullptr;
                if (sub < tokens && i < plan.recent) {
                    const char *from = slot(plan.from + i);
                    to[k] = slot(plan.to + i);
                    if (!from) to[k] = nullptr;
                    lost |= !to[k];
                    if (to[k]) x[k] = ptx::ld_written_once(from);
                }
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kMoveAtOnce; ++k)
                if (to[k]) *reinterpret_cast<uint4 *>(to[k]) = x[k];
        }
        if (lost) atomicOr(p.v.flags, CSD_CACHE_BAD_PAGE);
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
