// How much attention each place of a row has received: the weights of its newest tokens' queries, summed over tokens and heads.
//
//   mass[b,j] += sum_{t,h} exp(scale q[b,t,h].k[b,j,h / g] - lse[b,t,h])      over the tokens that see place j
//
// The softmax's sums are known (lse), so the keys alone are read once more: half of the bytes of attention, and no value is touched.
// Bound: memory for large batches of up to about 64 query rows to a key head.  96 rows of 500 to 4000 tokens, 8 key heads of 128, 36 query rows
// each: 83 to 86 us, 5.3 TB/s; one row of 131071 and one token 54.8 us, 4.9 TB/s; one row of 700 10.7 to 11.7 us.  Beyond, latency from scores to
// exponentials and back, with one set of query rows instead of two; and every further pass loads the keys again (from L2), as its loop lies outside
// the loads.  32 rows of 500 to 4000, 8 key heads of 128 (147 MB of keys, 23 us): with 4, 36, 64, 100 and 128 query rows 43, 44, 47, 58 and 62
// us, in two passes with 132, 192 and 256 81, 92 and 108; with 128 and 132 neither DRAM nor any unit of the SM is more than 40 % busy.
//
//   A tile is 128 places of a row and key head, and the FIRST operand of the product: S = K Q^T (tcgen05.mma, M = 128 places, N = the
//   head's query rows), so that a thread finds all scores of one place in its own lane of tensor memory and adds their exponentials
//   without an exchange.  Up to kMostRows query rows at a time (those that 32 KiB hold: 64 of 256 elements); more are further passes.
//   The places of all rows, in tiles, are split evenly over clusters of blocks; a cluster's blocks share its tiles' key heads among
//   themselves.  A run of up to kRunTiles tiles keeps its sums in shared memory over all heads of a block; at its end the blocks' sums are
//   added in the order of the blocks through distributed shared memory.  No atomics: results are bit-reproducible for given lengths.
//   warps 0..3  a thread per place: scores from tensor memory, exponentials, sums; they also fetch the query rows of the next pass
//   warp 4      one thread issues the products
//   warp 5      loads keys page by page (TMA), 64 elements of 128 places to a slot of the ring
// Waits inside a block are bounded, and a block whose wait runs out still meets the others at the cluster's barriers.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/csd.h"
#include "csd_attention.cuh"
#include "csd_common.cuh"
#include "csd_ptx.cuh"

namespace csd {
namespace mass {

using attention::Cursor;
using ptx::cluster_meet;
using ptx::mbar_arrive;
using ptx::mbar_expect_tx;
using ptx::mbar_init;
using ptx::mbar_wait;
using ptx::smem_u32;

constexpr int kTile = 128, kThreads = 192, kBlocksPerSm = 2, kMaxSlots = 8, kRunTiles = 16, kMostRows = 128;
constexpr int kSlotBytes = kTile * 128;
constexpr unsigned int kCols = 256;        // tensor memory: two buffers of up to kMostRows columns

struct Params {
    attention::Params a;                   // the cache's and the queries' fields
    const float *lse;                      // [B, T, Hq]
    float *mass;
    long long mass_stride;
    int fresh;
    int q_rows;                            // query rows of a pass: a multiple of 16, at most kMostRows
};

// A cluster's share of the tiles: runs of at most kRunTiles tiles of one row.
struct Tiles {
    const int *base;
    int B, x, x1, b;
    __device__ __forceinline__ Tiles(const int *base_, int B_, int cluster, int clusters) : base(base_), B(B_)
    {
        const long long total = base[B];
        x = static_cast<int>(total * cluster / clusters);
        x1 = static_cast<int>(total * (cluster + 1) / clusters);
        int lo = 0, hi = B - 1;            // the last row that begins at or before x
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (base[mid] <= x) lo = mid; else hi = mid - 1;
        }
        b = lo;
    }
    __device__ __forceinline__ bool next(int &row, int &j0, int &n)
    {
        if (x >= x1) return false;
        while (base[b + 1] <= x) ++b;
        row = b;
        j0 = x - base[b];
        n = min(min(x1, base[b + 1]) - x, kRunTiles);
        x += n;
        return true;
    }
};

__device__ __forceinline__ int ld_cluster(const int *mine, unsigned int rank)
{
    int v;
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(ptx::in_block(smem_u32(mine), rank)) : "memory");
    return v;
}

template <typename T>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
mass_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ Params p)
{
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bar_words[2 * kMaxSlots + 5];
    __shared__ __align__(16) float less[2][kMostRows];                   // -lse log2(e) of a pass's query rows; -inf: the row adds nothing
    __shared__ __align__(16) uint4 sees[2][kMostRows];                   // who sees it: new tokens' places 0 .. 31 and 32 .. 63, places before them, none
    __shared__ unsigned int tmem_base_slot;
    __shared__ int give_up_flag;
    volatile int *give_up = &give_up_flag;
    const attention::Params &a = p.a;

    const unsigned int rank = ptx::cluster_rank(), blocks = ptx::cluster_size();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned int rows_bytes = static_cast<unsigned int>(a.halves * p.q_rows * 128);
    const unsigned int q_smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const unsigned int ring = q_smem + a.q_buffers * rows_bytes;
    float *const acc = reinterpret_cast<float *>(smem_raw + (ring - smem_u32(smem_raw)) + a.n_stages * kSlotBytes);     // [kRunTiles][kTile]
    int *const base = reinterpret_cast<int *>(acc + kRunTiles * kTile);                                                  // [B + 1]
    const unsigned int bars = smem_u32(bar_words);
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (kMaxSlots + s); };
    auto s_full = [&](int k) { return bars + 8u * (2 * kMaxSlots + (k & 1)); };
    auto s_empty = [&](int k) { return bars + 8u * (2 * kMaxSlots + 2 + (k & 1)); };
    const unsigned int q_ready = bars + 8u * (2 * kMaxSlots + 4);
    auto q_at = [&](int pass) { return q_smem + (a.q_buffers == 2 ? pass & 1 : 0) * rows_bytes; };

    if (tid == 0) {
        give_up_flag = 0;
        for (int s = 0; s < a.n_stages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int k = 0; k < 2; ++k) {
            mbar_init(s_full(k), 1);
            mbar_init(s_empty(k), 4);
        }
        mbar_init(q_ready, 4);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    }
    if (warp == 1) {
        ptx::tmem_alloc(smem_u32(&tmem_base_slot), kCols);
        ptx::tmem_relinquish();
    }
    ptx::wait_for_stream();
    for (int b = tid; b < a.B; b += kThreads) {
        const int len = attention::row_len(a, b), news = attention::row_news(a, b);
        base[b + 1] = news > 0 ? (len + kTile - 1) / kTile : 0;
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    if (warp == 0) attention::scan_tiles(base, a.B);
    __syncthreads();
    if (blocks > 1) {
        // the first block's, for all: whatever another stream may do to the lengths meanwhile, all blocks have the same runs and barriers
        cluster_meet();
        if (rank != 0)
            for (int b = tid; b <= a.B; b += kThreads) base[b] = ld_cluster(base + b, 0);
        cluster_meet();
    }
    const unsigned int tmem = tmem_base_slot;
    Tiles tiles(base, a.B, static_cast<int>(blockIdx.x / blocks), static_cast<int>(gridDim.x / blocks));
    int b, j0, n;

    if (warp == 5) {
        // ---- page loads ----
        const int per_tile = kTile / a.box_rows;
        const unsigned int box_bytes = static_cast<unsigned int>(a.box_rows) * 128u;
        Cursor at = {0, 0u};
        bool ok = true;
        while (tiles.next(b, j0, n)) {
            const int len = attention::row_len(a, b), rows = min(a.T, attention::row_news(a, b)) * a.group;
            for (int h = static_cast<int>(rank); h < a.Hkv && ok; h += static_cast<int>(blocks))
                for (int r0 = 0; r0 < rows && ok; r0 += p.q_rows) {
                    int page = attention::tile_page<kTile>(a, b, j0, len, lane, per_tile);
                    for (int i = 0; i < n && ok; ++i) {
                        const int here = page, j = j0 + i;
                        if (i + 1 < n) page = attention::tile_page<kTile>(a, b, j + 1, len, lane, per_tile);
                        const unsigned int there = __ballot_sync(kFull, here >= 0);
                        const int in_page = a.box_rows == kTile ? (j * kTile) & ((1 << a.page_shift) - 1) : 0;
                        for (int hf = 0; hf < a.halves && ok; ++hf) {
                            int fine = 1;
                            if (lane == 0) {
                                fine = mbar_wait(empty(at.slot), at.round ^ 1u, give_up) ? 1 : 0;
                                if (fine) mbar_expect_tx(full(at.slot), static_cast<unsigned int>(__popc(there)) * box_bytes);
                            }
                            ok = __shfl_sync(kFull, fine, 0) != 0;
                            if (ok && here >= 0)
                                attention::tma_load_page(ring + at.slot * kSlotBytes + lane * box_bytes, &map_k, full(at.slot), hf * 64, in_page, h, here);
                            at.next(a.n_stages);
                        }
                    }
                }
            if (blocks > 1) {
                cluster_meet();
                cluster_meet();
            }
        }
        // every commit aimed at the slots' barriers has landed before the block ends
        if (lane == 0)
            for (int k = 0; k < a.n_stages && ok; ++k, at.next(a.n_stages)) ok = mbar_wait(empty(at.slot), at.round ^ 1u, give_up);
    } else if (warp == 4) {
        // ---- products ----
        // (written out for each number of 64-element columns; elements beyond dim are zeros)
        Cursor at = {0, 0u};
        int k = 0, pass = 0;
        bool ok = true;
        auto issue = [&](auto columns, int rows) {
            constexpr int kColumns = decltype(columns)::value;
            for (int h = static_cast<int>(rank); h < a.Hkv && ok; h += static_cast<int>(blocks))
                for (int r0 = 0; r0 < rows && ok; r0 += p.q_rows, ++pass) {
                    const unsigned int idesc = attention::tc_instr<T>(kTile, (min(p.q_rows, rows - r0) + 15) / 16 * 16, false);
                    ok = mbar_wait(q_ready, pass & 1, give_up);
                    for (int i = 0; i < n && ok; ++i, ++k) {
                        if (!(ok = mbar_wait(s_empty(k), ((k >> 1) & 1) ^ 1, give_up))) break;
                        const unsigned int d = tmem + (k & 1) * kMostRows;
                        const unsigned long long q_desc = ptx::operand_desc(q_at(pass)), q_column = static_cast<unsigned long long>(p.q_rows * 128 >> 4);
#pragma unroll
                        for (int c = 0; c < kColumns; ++c) {
                            if (!ok || !(ok = mbar_wait(full(at.slot), at.round, give_up))) break;
                            ptx::tc_fence_after();
                            const unsigned long long kd = ptx::operand_desc(ring + at.slot * kSlotBytes), qd = q_desc + c * q_column;
#pragma unroll
                            for (int e = 0; e < 4; ++e)                             // 16 elements further: 32 bytes
                                attention::tc_mma_ss(d, kd + 2 * e, qd + 2 * e, idesc, c == 0 && e == 0 ? 0u : 1u);
                            ptx::tc_commit(empty(at.slot));
                            at.next(a.n_stages);
                        }
                        if (ok) ptx::tc_commit(s_full(k));
                    }
                }
        };
        const bool issuer = ptx::elect_one();
        while (tiles.next(b, j0, n)) {
            const int rows = min(a.T, attention::row_news(a, b)) * a.group;
            if (issuer) {
                if (a.halves == 1)
                    issue(attention::Columns<1>(), rows);
                else if (a.halves == 2)
                    issue(attention::Columns<2>(), rows);
                else if (a.halves == 3)
                    issue(attention::Columns<3>(), rows);
                else
                    issue(attention::Columns<4>(), rows);
            }
            if (blocks > 1) {
                cluster_meet();
                cluster_meet();
            }
        }
    } else {
        // ---- a thread per place ----
        const unsigned int my_lanes = static_cast<unsigned int>(32 * warp) << 16;
        const unsigned long long sc2 = pack2(a.scale_log2, a.scale_log2);
        // a pass: the query rows r0 .. of key head h of row b
        struct Pass {
            int b, h, r0, rows, len, news;                               // rows: all of the head
        };
        auto here_of = [&](const Pass &x) { return min(p.q_rows, x.rows - x.r0); };
        auto fetch = [&](const Pass &x, int pass) {                      // its query rows on their way to shared memory
            const int rows_here = here_of(x), chunks = a.halves * 8, at_once = 32 / chunks, sub = lane / chunks, ch = lane - sub * chunks;
            if (sub >= at_once) return;
            for (int r = warp * at_once + sub; r < rows_here; r += 4 * at_once) {
                const int rr = x.r0 + r, tok = rr / a.group, head = x.h * a.group + rr - tok * a.group;
                const unsigned int to = q_at(pass) + (ch >> 3) * (p.q_rows * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
                const bool there = ch * 8 < a.D;
                const T *from = static_cast<const T *>(a.q) + x.b * a.qb + tok * a.qt + head * a.qh + (there ? ch * 8 : 0);
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
            }
        };
        auto fetched = [&]() {
            asm volatile("cp.async.wait_all;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(q_ready);
        };
        // thread r looks after query row r of a pass.  Loaded a pass ahead and not looked at before its turn, so that nothing waits here.
        struct Column {
            int tok, lse;                                                // tok -1: no row, or a token without a place
            int2 mask;
        };
        auto column = [&](const Pass &x) {
            Column c = {-1, 0, make_int2(0, 0)};
            if (tid >= here_of(x)) return c;
            const int rr = x.r0 + tid, tok = rr / a.group, head = x.h * a.group + rr - tok * a.group;
            if (x.len - x.news + tok < 0) return c;
            const long long at = static_cast<long long>(x.b) * a.T + tok;
            c.tok = tok;
            c.lse = ptx::ld_written(reinterpret_cast<const int *>(p.lse) + at * a.Hq + head);
            if (a.masks) c.mask = ptx::ld_written(reinterpret_cast<const int2 *>(a.masks) + at);
            return c;
        };
        // the passes in order, a pass ahead of the work
        Tiles ahead = tiles;
        Pass coming = {0, 0, 0, 0, 0, 0};
        int ahead_j0, ahead_n;
        bool more = false;
        auto advance = [&]() {
            if (more) {
                coming.r0 += p.q_rows;
                if (coming.r0 < coming.rows) return;
                coming.r0 = 0;
                coming.h += static_cast<int>(blocks);
                if (coming.h < a.Hkv) return;
            }
            more = ahead.next(coming.b, ahead_j0, ahead_n);
            if (!more) return;
            coming.h = static_cast<int>(rank);
            coming.r0 = 0;
            coming.len = attention::row_len(a, coming.b);
            coming.news = attention::row_news(a, coming.b);
            coming.rows = min(a.T, coming.news) * a.group;
        };
        const bool two = a.q_buffers == 2;
        Column mine = {-1, 0, make_int2(0, 0)};
        advance();
        if (more) {
            mine = column(coming);
            if (two) {
                fetch(coming, 0);
                fetched();
            }
        }
        int k = 0, pass = 0;
        while (tiles.next(b, j0, n)) {
            const Pass row = coming;                                      // the run's first pass
            const int first = row.len - row.news;
            for (int h = static_cast<int>(rank); h < a.Hkv; h += static_cast<int>(blocks))
                for (int r0 = 0; r0 < row.rows; r0 += p.q_rows, ++pass) {
                    const Pass now = coming;
                    const int here = here_of(now), buf = pass & 1;
                    if (!two) {                                           // (the pass before has been read by its products: its scores are there)
                        fetch(now, pass);
                        fetched();
                    }
                    const float lse = __int_as_float(mine.lse);
                    const float minus = mine.tok < 0 || lse == -INFINITY ? -INFINITY : -lse * kLog2e;
                    less[buf][tid] = minus;
                    const bool dead = minus == -INFINITY;
                    const unsigned long long bits = a.masks ? attention::existing(mine.mask, now.len, now.news) : (mine.tok < 63 ? (2ull << max(mine.tok, 0)) - 1ull : ~0ull);
                    sees[buf][tid] = dead ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(static_cast<unsigned int>(bits), static_cast<unsigned int>(bits >> 32), ~0u, 0u);
                    // (two sets: a warp may be a pass ahead of another, never two, for every pass has this barrier)
                    int any_dead;
                    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(any_dead) : "r"(dead && tid < here ? 1 : 0) : "memory");
                    advance();
                    if (more) {
                        mine = column(coming);
                        if (two) fetch(coming, pass + 1);
                    }
                    for (int i = 0; i < n; ++i, ++k) {
                        const int key = (j0 + i) * kTile + tid;
                        const bool careful = any_dead != 0 || (j0 + i + 1) * kTile > first;    // some row adds nothing, or does not see all places
                        mbar_wait(s_full(k), (k >> 1) & 1, give_up);
                        ptx::tc_fence_after();
                        const unsigned int at = tmem + my_lanes + (k & 1) * kMostRows;
                        float sum = 0.f;
                        int c = 0;
                        if (!careful) {
                            unsigned long long sum0 = pack2(0.f, 0.f), sum1 = sum0;
                            for (; c + 32 <= here; c += 32) {
                                float x[32];
                                ptx::tmem_ld32(at + c, x);
#pragma unroll
                                for (int e = 0; e < 32; e += 4) {
                                    const ulonglong2 l2 = *reinterpret_cast<const ulonglong2 *>(&less[buf][c + e]);
                                    float y0, y1, y2, y3;
                                    unpack2(fma2(pack2(x[e], x[e + 1]), sc2, l2.x), y0, y1);
                                    unpack2(fma2(pack2(x[e + 2], x[e + 3]), sc2, l2.y), y2, y3);
                                    sum0 = add2(sum0, pack2(ex2_approx(y0), ex2_approx(y1)));
                                    sum1 = add2(sum1, pack2(ex2_approx(y2), ex2_approx(y3)));
                                }
                            }
                            float s0, s1;
                            unpack2(add2(sum0, sum1), s0, s1);
                            sum = s0 + s1;
                        }
                        // rows that do not exist or add nothing, and places that a row does not see: whatever was computed for them is left out
                        const int u = key - first;
                        const unsigned int *const word = reinterpret_cast<const unsigned int *>(&sees[buf][0]) + (u < 0 ? 2 : min(u >> 5, 2) + (u >= 64 ? 1 : 0));
                        auto picked = [&](int c1, const auto &x, auto width) {
#pragma unroll
                            for (int e = 0; e < decltype(width)::value; ++e) {
                                const float w = ex2_approx(__fmaf_rn(x[e], a.scale_log2, less[buf][c1 + e]));
                                sum += word[4 * (c1 + e)] >> (u & 31) & 1u ? w : 0.f;
                            }
                        };
                        for (; c + 16 < here; c += 32) {
                            float x[32];
                            ptx::tmem_ld32(at + c, x);
                            picked(c, x, attention::Columns<32>());
                        }
                        if (c < here) {
                            float x[16];
                            ptx::tmem_ld16(at + c, x);
                            picked(c, x, attention::Columns<16>());
                        }
                        ptx::tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(s_empty(k));
                        float *const to = acc + i * kTile + tid;
                        *to = h == static_cast<int>(rank) && r0 == 0 ? sum : *to + sum;
                        if (i == 0 && two && more) fetched();             // the products may run on into the next pass
                    }
                }
            // ---- the run's places ----
            float *const mass = p.mass + b * p.mass_stride;
            if (blocks > 1) cluster_meet();
            for (int i = static_cast<int>(rank); i < n; i += static_cast<int>(blocks)) {
                const int key = (j0 + i) * kTile + tid;
                float sum = 0.f;
                if (blocks > 1)
                    for (unsigned int r = 0; r < blocks; ++r) sum += __int_as_float(ld_cluster(reinterpret_cast<const int *>(acc) + i * kTile + tid, r));
                else
                    sum = acc[i * kTile + tid];
                if (key < row.len) {
                    const float was = p.fresh && key >= first ? 0.f : __int_as_float(ptx::ld_written(reinterpret_cast<const int *>(mass) + key));
                    mass[key] = was + sum;
                }
            }
            if (blocks > 1) cluster_meet();
        }
        ptx::tc_fence_before();
    }
    __syncthreads();
    if (*give_up) {                                                  // a wait ran out
        if (lane == 0) atomicOr(a.flags, CSD_CACHE_INTERNAL);
        ptx::linger();
        __syncthreads();
    }
    if (warp == 1) ptx::tmem_dealloc(tmem, kCols);
}

}  // namespace mass
}  // namespace csd
