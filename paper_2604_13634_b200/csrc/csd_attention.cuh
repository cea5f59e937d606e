// Attention of a row's newest tokens over its paged keys and values, split over the length and joined.
//
//   out[b,t,h] = sum_j w_j v_j,  w = softmax_j(scale q.k_j),  over the places j <= lens[b] - n_new[b] + t
//   lse[b,t,h] = ln sum_j exp(scale q.k_j)
//
// A run of places gives a part (m, l, O) = (max_j x_j, sum_j 2^(x_j - m), sum_j 2^(x_j - m) v_j) with x = scale log2(e) q.k, and
// parts join as M = max m_i, L = sum l_i 2^(m_i - M), O = sum O_i 2^(m_i - M) / L.
//
// Bound: memory (each key and value is read once; T g query rows share it, g = query heads per key head).
//
//   attention_kernel  persistent.  The tiles (kTile places of one row and key head) of all rows and heads, laid out row after
//                     row, are split evenly and contiguously over the blocks, whatever the rows' lengths are (read on the
//                     device), so a block works on a run of tiles of a few (row, head) units.
//       producer warp  puts the tile's keys and values, page by page, into a ring of shared-memory stages by TMA (boxes of
//                     64 elements x the places of one page, 128-byte swizzle; elements beyond dim read as zero)
//       consumer warps KG x RG of them: a warp owns 16 MT of the unit's query rows and 16 NK of a tile's places, with
//                     its own running (m, l, O) in registers: no exchange between warps until the unit ends.  Products
//                     are mma.sync m16n8k16 (16 x 8 x 16) with float32 accumulators: a tile has at most 128 query rows, the
//                     tensor pipe is far from its limit while the tiles stream.
//     At the end of a unit the KG warps of a row group join through a ring stage; a unit that lies in one block whole is
//     written out, otherwise the part goes to the workspace.
//   attention_join_kernel  joins the parts of the units that were split (at most one begins in each block), a warp per query row, in
//                     the order of the places.
// No block waits for another; waits inside a block are bounded.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/csd.h"
#include "csd_common.cuh"
#include "csd_ptx.cuh"
#include "csd_rope.cuh"

namespace csd {
namespace attention {

using ptx::mbar_arrive;
using ptx::mbar_expect_tx;
using ptx::mbar_init;
using ptx::mbar_wait;
using ptx::smem_u32;
using rope::from_f32;

constexpr int kMaxStages = 12;
constexpr float kLn2 = 0.6931471805599453f;

// What the first block of a split unit leaves for the join: parts lie in slot 2 c + 1 of that block and slots 2 (c + i) of the next ones.
struct Split {
    int unit;                 // (row * heads + head) * row tiles + row tile
    int parts;                // 0: no split unit begins in this block
};

struct Params {
    const void *q;
    void *out;
    float *lse;
    int B, T, Hq, Hkv, D, group, rows;     // rows: T * group query rows of a unit
    int row_tiles;                         // of kRows query rows each
    long long qb, qt, qh;
    int page_shift, n_pages, max_pages;
    int box_rows;                          // places of a TMA box: min(page, kTile)
    const int *table, *lens, *n_new;
    unsigned int *flags;
    float scale_log2;
    int n_stages, min_tiles;
    Split *splits;                         // [gridDim.x]
    float *parts;                          // [2 gridDim.x] slots of kRows * (DP + 2) floats
};

template <typename T_, int DP_, int MT_, int NK_, int KG_, int RG_, int kBlocksPerSm_>
struct Config {
    using T = T_;
    static constexpr int DP = DP_, MT = MT_, NK = NK_, KG = KG_, RG = RG_, kBlocksPerSm = kBlocksPerSm_;
    static constexpr int kTile = 16 * NK * KG;
    static constexpr int kRows = 16 * MT * RG;
    static constexpr int kWarps = KG * RG;
    // Registers move between warpgroups of four warps: the producer's gives up what it does not need.
    static constexpr int kThreads = 32 * (kWarps + 4);
    static constexpr int kGroups = kWarps / 4 + 1;
    static constexpr int kLaunchRegs = 65536 / (kThreads * kBlocksPerSm) / 8 * 8;          // per thread, as launched (the host checks)
    static constexpr bool kMoveRegs = kLaunchRegs < 232;
    static constexpr int kProducerRegs = 40;
    static constexpr int kConsumerRegs = (kGroups * kLaunchRegs - kProducerRegs) / (kGroups - 1) / 8 * 8;
    static_assert(kWarps % 4 == 0 && (!kMoveRegs || (kConsumerRegs <= 240 && kConsumerRegs * (kGroups - 1) + kProducerRegs <= kGroups * kLaunchRegs)),
                  "register split");
    static constexpr int kHalves = DP / 64;                        // 128-byte columns of a tile
    static constexpr int kTileBytes = kTile * DP * 2;               // keys or values of a stage
    static constexpr int kStageBytes = 2 * kTileBytes;
    static constexpr int kQBytes = kRows * DP * 2;
    static constexpr int kMlBytes = KG * kRows * 8;
    static constexpr int kSlotFloats = kRows * (DP + 2);
    static constexpr bool kQInRegisters = MT == 1 && DP <= 128;
    // joining warps: KG / 2 buffers of the block's rows fit in a stage, column by column block if need be
    static constexpr int kJoinBytes = KG / 2 * kRows * DP * 4;
    static constexpr int kJoinPasses = KG == 1 ? 1 : (kJoinBytes + kStageBytes - 1) / kStageBytes;
    static constexpr int kNt = DP / 8;                              // column tiles of 8
    static constexpr int kNtPass = kNt / kJoinPasses;
    static_assert(kNt % kJoinPasses == 0, "column passes");
};

__device__ __forceinline__ void tma_load_page(unsigned int dst, const CUtensorMap *map, unsigned int bar, int d, int place, int head, int page)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
                 "l"(map), "r"(bar), "r"(d), "r"(place), "r"(head), "r"(page)
                 : "memory");
}
__device__ __forceinline__ void ldsm4(unsigned int (&r)[4], unsigned int addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(unsigned int (&r)[4], unsigned int addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const unsigned int (&a)[4], unsigned int b0, unsigned int b1);
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const unsigned int (&a)[4], unsigned int b0, unsigned int b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__half>(float (&c)[4], const unsigned int (&a)[4], unsigned int b0, unsigned int b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <typename T>
__device__ __forceinline__ unsigned int pack_pair(float lo, float hi);
template <>
__device__ __forceinline__ unsigned int pack_pair<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned int *>(&v);
}
template <>
__device__ __forceinline__ unsigned int pack_pair<__half>(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const unsigned int *>(&v);
}
// Two elements with those that are an infinity or NaN (exponent field all ones) replaced by zero.
template <typename T>
struct ExponentBits;
template <>
struct ExponentBits<__nv_bfloat16> {
    static constexpr unsigned int value = 0x7f80u;
};
template <>
struct ExponentBits<__half> {
    static constexpr unsigned int value = 0x7c00u;
};
template <typename T>
__device__ __forceinline__ unsigned int finite_only(unsigned int two)
{
    constexpr unsigned int e = ExponentBits<T>::value;
    if ((two & e) == e) two &= 0xffff0000u;
    if ((two & (e << 16)) == (e << 16)) two &= 0x0000ffffu;
    return two;
}

__device__ __forceinline__ void consumer_barrier(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }

// Walks a block's run of tiles: row b, key head h, row tile rt, tile j of n.
struct Walk {
    int b, h, rt, j, n;
};

// base[b]: tiles of the rows before b (one head, one row tile).  Tile t of all lies in row b with base[b] hr <= t < base[b+1] hr.
__device__ __forceinline__ Walk walk_to(long long t, const int *base, int B, int Hkv, int row_tiles)
{
    const long long hr = static_cast<long long>(Hkv) * row_tiles;
    int lo = 0, hi = B - 1;                              // the last b with base[b] * hr <= t has tiles
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (base[mid] * hr <= t) lo = mid; else hi = mid - 1;
    }
    Walk w;
    w.b = lo;
    w.n = base[lo + 1] - base[lo];
    const long long rest = t - base[lo] * hr;
    const int hrt = static_cast<int>(rest / w.n);
    w.j = static_cast<int>(rest - static_cast<long long>(hrt) * w.n);
    w.h = hrt / row_tiles;
    w.rt = hrt - w.h * row_tiles;
    return w;
}

__device__ __forceinline__ void walk_next(Walk &w, const int *base, int B, int Hkv, int row_tiles)
{
    if (++w.j < w.n) return;
    w.j = 0;
    if (++w.rt < row_tiles) return;
    w.rt = 0;
    if (++w.h < Hkv) return;
    w.h = 0;
    do {
        ++w.b;
    } while (w.b < B && base[w.b + 1] == base[w.b]);
    w.n = w.b < B ? base[w.b + 1] - base[w.b] : 1;
}

__device__ __forceinline__ int row_len(const Params &p, int b) { return min(max(__ldg(p.lens + b), 0), p.max_pages << p.page_shift); }
__device__ __forceinline__ int row_news(const Params &p, int b) { return p.n_new ? min(max(__ldg(p.n_new + b), 0), p.T) : p.T; }

template <typename C>
__global__ void __launch_bounds__(C::kThreads, C::kBlocksPerSm)
attention_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Params p)
{
    using T = typename C::T;
    constexpr int DP = C::DP, MT = C::MT, NK = C::NK, KG = C::KG, RG = C::RG, kTile = C::kTile;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bar_words[3 * kMaxStages];
    __shared__ int give_up_flag;
    volatile int *give_up = &give_up_flag;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned int ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const unsigned int q_smem = ring + p.n_stages * C::kStageBytes;
    unsigned char *after_q = smem_raw + (q_smem - smem_u32(smem_raw)) + C::kQBytes;
    float2 *ml = reinterpret_cast<float2 *>(after_q);                              // [KG][kRows]
    int *base = reinterpret_cast<int *>(after_q + C::kMlBytes);                    // [B + 1]
    const unsigned int bars = smem_u32(bar_words);
    auto full_k = [&](int s) { return bars + 8u * s; };
    auto full_v = [&](int s) { return bars + 8u * (kMaxStages + s); };
    auto empty = [&](int s) { return bars + 8u * (2 * kMaxStages + s); };

    if (tid == 0) {
        give_up_flag = 0;
        for (int s = 0; s < p.n_stages; ++s) {
            mbar_init(full_k(s), 1);
            mbar_init(full_v(s), 1);
            mbar_init(empty(s), C::kWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        p.splits[blockIdx.x].parts = 0;
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // tiles of each row; rows without any give zeros
    for (int b = tid; b < p.B; b += C::kThreads) {
        const int len = row_len(p, b), news = row_news(p, b);
        base[b + 1] = news > 0 ? (len + kTile - 1) / kTile : 0;
    }
    __syncthreads();
    if (warp == 0) {
        int sum = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            int v = b0 + lane < p.B ? base[b0 + lane + 1] : 0;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(kFull, v, d);
                if (lane >= d) v += o;
            }
            if (b0 + lane < p.B) base[b0 + lane + 1] = sum + v;
            sum += __shfl_sync(kFull, v, 31);
        }
        if (lane == 0) base[0] = 0;
    }
    __syncthreads();
    const int units_per_row = p.Hkv * p.row_tiles;
    const long long total = static_cast<long long>(base[p.B]) * units_per_row;
    long long G = gridDim.x;
    if (total < G * p.min_tiles) G = max(1ll, total / p.min_tiles);
    const long long c = blockIdx.x;
    const long long t0 = c < G ? c * total / G : total, t1 = c < G ? (c + 1) * total / G : total;

    if (warp >= C::kWarps) {
        // ---- producer: one warp of its group ----
        if constexpr (C::kMoveRegs) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kProducerRegs));
        if (warp == C::kWarps && t0 < t1) {
            Walk w = walk_to(t0, base, p.B, p.Hkv, p.row_tiles);
            const int per_tile = kTile / p.box_rows;               // pages of a tile (1 where a page is larger)
            const unsigned int box_bytes = static_cast<unsigned int>(p.box_rows) * 128u;
            int len = row_len(p, w.b), len_of = w.b;
            // lane f < per_tile looks after page f of the tile; its id is fetched a tile ahead
            auto fetch = [&](const Walk &x, int x_len) {
                const int place = x.j * kTile + lane * p.box_rows;
                int id = -1;                                        // nothing to load
                if (lane < per_tile && place < x_len) {
                    id = __ldg(p.table + static_cast<long long>(x.b) * p.max_pages + (place >> p.page_shift));
                    if (id < 0 || id >= p.n_pages) {                // reads as zeros: outside the tensor map
                        atomicOr(p.flags, CSD_CACHE_BAD_PAGE);
                        id = p.n_pages;
                    }
                }
                return id;
            };
            int id = fetch(w, len);
            int it = 0;
            for (long long t = t0; t < t1; ++t, ++it) {
                const Walk now = w;
                const int my_page = id;
                const bool unit_ends = now.j + 1 == now.n || t + 1 == t1;
                if (t + 1 < t1) {
                    walk_next(w, base, p.B, p.Hkv, p.row_tiles);
                    if (w.b != len_of) {
                        len = row_len(p, w.b);
                        len_of = w.b;
                    }
                    id = fetch(w, len);
                }
                const int s = it % p.n_stages;
                const unsigned int there = __ballot_sync(kFull, my_page >= 0);
                bool ok = true;
                if (lane == 0) {
                    ok = mbar_wait(empty(s), ((it / p.n_stages) & 1) ^ 1, give_up);
                    if (ok) {
                        const unsigned int bytes = static_cast<unsigned int>(__popc(there)) * box_bytes * C::kHalves;
                        mbar_expect_tx(full_k(s), bytes);
                        mbar_expect_tx(full_v(s), bytes);
                    }
                }
                ok = __shfl_sync(kFull, ok ? 1 : 0, 0) != 0;
                if (!ok) break;
                if (my_page >= 0) {
                    const int in_page = p.box_rows == kTile ? (now.j * kTile) & ((1 << p.page_shift) - 1) : 0;
                    const unsigned int at = ring + s * C::kStageBytes + lane * box_bytes;
#pragma unroll
                    for (int hf = 0; hf < C::kHalves; ++hf)
                        tma_load_page(at + hf * (kTile * 128), &map_k, full_k(s), hf * 64, in_page, now.h, my_page);
#pragma unroll
                    for (int hf = 0; hf < C::kHalves; ++hf)
                        tma_load_page(at + C::kTileBytes + hf * (kTile * 128), &map_v, full_v(s), hf * 64, in_page, now.h, my_page);
                }
                if (unit_ends && KG > 1) {                           // the consumers join through the next stage
                    ++it;
                    const int sj = it % p.n_stages;
                    if (lane == 0) {
                        ok = mbar_wait(empty(sj), ((it / p.n_stages) & 1) ^ 1, give_up);
                        if (ok) {
                            mbar_arrive(full_k(sj));
                            mbar_arrive(full_v(sj));
                        }
                    }
                    ok = __shfl_sync(kFull, ok ? 1 : 0, 0) != 0;
                    if (!ok) break;
                }
            }
        }
    } else {
        // ---- consumers ----
        if constexpr (C::kMoveRegs) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kConsumerRegs));
        const int rg = warp / KG, kg = warp % KG;
        const int g = lane >> 2, qd = lane & 3;
        const int cthreads = C::kWarps * 32;
        // zeros for rows that have nothing to read
        for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
            if (base[b + 1] != base[b]) continue;
            const long long row0 = static_cast<long long>(b) * p.T * p.Hq;
            uint4 *o = reinterpret_cast<uint4 *>(static_cast<T *>(p.out) + row0 * p.D);
            const int vecs = p.T * p.Hq * p.D / 8;
            for (int i = tid; i < vecs; i += cthreads) o[i] = make_uint4(0, 0, 0, 0);
            if (p.lse)
                for (int i = tid; i < p.T * p.Hq; i += cthreads) p.lse[row0 + i] = -INFINITY;
        }
        Walk w;
        if (t0 < t1) w = walk_to(t0, base, p.B, p.Hkv, p.row_tiles);
        int it = 0;
        const int swz = lane & 7;
        const unsigned int k_lane = (16 * NK * kg + ((lane >> 4) << 3) + swz) * 128u, k_chunk = (lane >> 3) & 1;
        const unsigned int v_lane = (16 * NK * kg + (((lane >> 3) & 1) << 3) + swz) * 128u, v_chunk = lane >> 4;
        const unsigned int q_lane = (16 * MT * rg + (((lane >> 3) & 1) << 3) + swz) * 128u, q_chunk = lane >> 4;

        for (long long t = t0; t < t1;) {
            // ---- a unit, or the part of one that lies in this block ----
            const int b = w.b, h = w.h, rt = w.rt, j0 = w.j;
            const int j1 = static_cast<int>(min(static_cast<long long>(w.n), j0 + (t1 - t)));
            const int len = row_len(p, b), news = row_news(p, b);
            const int rows_here = min(C::kRows, p.rows - rt * C::kRows);
            // its query rows: row r is token r / group, query head h * group + r % group
            for (int i = tid; i < C::kRows * (DP / 8); i += cthreads) {
                const int r = i / (DP / 8), ch = i % (DP / 8);
                uint4 x = make_uint4(0, 0, 0, 0);
                if (r < rows_here && ch * 8 < p.D) {
                    const int rr = rt * C::kRows + r, tok = rr / p.group, hh = h * p.group + rr - tok * p.group;
                    x = __ldg(reinterpret_cast<const uint4 *>(static_cast<const T *>(p.q) + b * p.qb + tok * p.qt + hh * p.qh + ch * 8));
                }
                const unsigned int at = q_smem + (ch >> 3) * (C::kRows * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
            }
            consumer_barrier(cthreads);
            int limit[MT][2];                                       // last place that the thread's rows see; -1: none
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const int r = 16 * (MT * rg + mt) + g + 8 * hh, rr = rt * C::kRows + r;
                    const int tok = rr / p.group;
                    limit[mt][hh] = r < rows_here && tok < news ? len - news + tok : -1;
                }
            unsigned int qf[C::kQInRegisters ? DP / 16 : 1][4];
            if constexpr (C::kQInRegisters) {
#pragma unroll
                for (int ks = 0; ks < DP / 16; ++ks)
                    ldsm4(qf[ks], q_smem + (ks >> 2) * (C::kRows * 128) + q_lane + ((((ks & 3) * 2 + q_chunk) ^ swz) << 4));
            }
            float o[MT][C::kNt][4], m[MT][2], l[MT][2];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int nt = 0; nt < C::kNt; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[mt][nt][e] = 0.f;
                m[mt][0] = m[mt][1] = -INFINITY;
                l[mt][0] = l[mt][1] = 0.f;
            }

            for (int j = j0; j < j1; ++j, ++it) {
                const int s = it % p.n_stages;
                const unsigned int parity = (it / p.n_stages) & 1;
                const unsigned int k_at = ring + s * C::kStageBytes, v_at = k_at + C::kTileBytes;
                const int key0 = j * kTile + 16 * NK * kg;          // the warp's first place
                float x[MT][2 * NK][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int n = 0; n < 2 * NK; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[mt][n][e] = 0.f;
                mbar_wait(full_k(s), parity, give_up);
                const bool any = key0 < len;                         // nothing of the warp's places exists otherwise
                if (any) {
#pragma unroll
                    for (int ks = 0; ks < DP / 16; ++ks) {
                        unsigned int qa[MT][4];
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            if constexpr (C::kQInRegisters) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) qa[mt][e] = qf[ks][e];
                            } else {
                                ldsm4(qa[mt], q_smem + (ks >> 2) * (C::kRows * 128) + q_lane + mt * (16 * 128) + ((((ks & 3) * 2 + q_chunk) ^ swz) << 4));
                            }
                        }
#pragma unroll
                        for (int nk = 0; nk < NK; ++nk) {
                            unsigned int kb[4];
                            ldsm4(kb, k_at + (ks >> 2) * (kTile * 128) + k_lane + nk * (16 * 128) + ((((ks & 3) * 2 + k_chunk) ^ swz) << 4));
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) {
                                mma16816<T>(x[mt][2 * nk], qa[mt], kb[0], kb[1]);
                                mma16816<T>(x[mt][2 * nk + 1], qa[mt], kb[2], kb[3]);
                            }
                        }
                    }
                }
                // scores in powers of two; places that a row does not see become -inf whatever was computed for them
                const bool edge = key0 + 16 * NK - 1 > len - news;   // some row does not see all of the warp's places
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int n = 0; n < 2 * NK; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            x[mt][n][e] *= p.scale_log2;
                            if (edge && key0 + 8 * n + 2 * qd + (e & 1) > limit[mt][e >> 1]) x[mt][n][e] = -INFINITY;
                        }
                unsigned int pa[MT][NK][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    float mx[2], f[2], at0[2];
                    bool grew = false;
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        float v = x[mt][0][2 * hh];
#pragma unroll
                        for (int n = 0; n < 2 * NK; ++n) v = fmaxf(v, fmaxf(x[mt][n][2 * hh], x[mt][n][2 * hh + 1]));
                        v = fmaxf(v, __shfl_xor_sync(kFull, v, 1));
                        v = fmaxf(v, __shfl_xor_sync(kFull, v, 2));
                        mx[hh] = fmaxf(m[mt][hh], v);
                        grew |= mx[hh] > m[mt][hh];
                        at0[hh] = mx[hh] == -INFINITY ? 0.f : mx[hh];
                    }
                    if (__any_sync(kFull, grew)) {
#pragma unroll
                        for (int hh = 0; hh < 2; ++hh) {
                            f[hh] = ex2_approx(m[mt][hh] - at0[hh]);
                            l[mt][hh] *= f[hh];
                            m[mt][hh] = mx[hh];
                        }
#pragma unroll
                        for (int nt = 0; nt < C::kNt; ++nt) {
                            o[mt][nt][0] *= f[0];
                            o[mt][nt][1] *= f[0];
                            o[mt][nt][2] *= f[1];
                            o[mt][nt][3] *= f[1];
                        }
                    }
#pragma unroll
                    for (int n = 0; n < 2 * NK; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            x[mt][n][e] = ex2_approx(x[mt][n][e] - at0[e >> 1]);
                            l[mt][e >> 1] += x[mt][n][e];
                        }
                    // the weights go into the second product in the cache's type: relative error 2^-9 (2^-12) of each, of random
                    // sign, where the result itself is rounded to that type; the sum l is taken before the rounding
#pragma unroll
                    for (int nk = 0; nk < NK; ++nk) {
                        pa[mt][nk][0] = pack_pair<T>(x[mt][2 * nk][0], x[mt][2 * nk][1]);
                        pa[mt][nk][1] = pack_pair<T>(x[mt][2 * nk][2], x[mt][2 * nk][3]);
                        pa[mt][nk][2] = pack_pair<T>(x[mt][2 * nk + 1][0], x[mt][2 * nk + 1][1]);
                        pa[mt][nk][3] = pack_pair<T>(x[mt][2 * nk + 1][2], x[mt][2 * nk + 1][3]);
                    }
                }
                mbar_wait(full_v(s), parity, give_up);
                bool odd_values = false, wrote = false;
                if (any && edge) {
                    // A weight of zero does not silence an infinity or NaN.  Places beyond the row hold anything: zeroed here.
                    // Places of later new tokens are seen by some rows only: if one holds such a value, the product leaves it
                    // out (the other rows' results keep their bits) and the rows that see it get it afterwards.
                    bool odd = false;
                    for (int i = lane; i < 16 * NK * (DP / 8); i += 32) {
                        const int r = i / (DP / 8), ch = i % (DP / 8), key = key0 + r;
                        const unsigned int at = v_at + (ch >> 3) * (kTile * 128) + (16 * NK * kg + r) * 128 + (((ch & 7) ^ (r & 7)) << 4);
                        if (key >= len) {
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0u) : "memory");
                            wrote = true;
                        } else if (key > len - news) {
                            unsigned int y[4];
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]) : "r"(at) : "memory");
                            odd |= finite_only<T>(y[0]) != y[0] || finite_only<T>(y[1]) != y[1] || finite_only<T>(y[2]) != y[2] || finite_only<T>(y[3]) != y[3];
                        }
                    }
                    __syncwarp();
                    odd_values = __any_sync(kFull, odd);
                }
                if (any) {
#pragma unroll
                    for (int nk = 0; nk < NK; ++nk)
#pragma unroll
                        for (int n2 = 0; n2 < C::kNt / 2; ++n2) {
                            unsigned int vb[4];
                            ldsm4_trans(vb, v_at + (n2 >> 2) * (kTile * 128) + v_lane + nk * (16 * 128) + ((((n2 & 3) * 2 + v_chunk) ^ swz) << 4));
                            if (odd_values) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) vb[e] = finite_only<T>(vb[e]);
                            }
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) {
                                mma16816<T>(o[mt][2 * n2], pa[mt][nk], vb[0], vb[1]);
                                mma16816<T>(o[mt][2 * n2 + 1], pa[mt][nk], vb[2], vb[3]);
                            }
                        }
                }
                if (odd_values) {                                    // what was left out, for the rows that see it
                    for (int r = 0; r < 16 * NK && key0 + r < len; ++r) {
                        const int src = (lane & ~3) | ((r & 7) >> 1);
                        float wt[MT][2];
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int hh = 0; hh < 2; ++hh) {
                                wt[mt][hh] = 0.f;
#pragma unroll
                                for (int n = 0; n < 2 * NK; ++n)
#pragma unroll
                                    for (int e = 0; e < 2; ++e) {
                                        const float y = __shfl_sync(kFull, x[mt][n][2 * hh + e], src);
                                        if (n == (r >> 3) && e == (r & 1)) wt[mt][hh] = y;
                                    }
                            }
#pragma unroll
                        for (int nt = 0; nt < C::kNt; ++nt) {
                            const unsigned int at = v_at + (nt >> 3) * (kTile * 128) + (16 * NK * kg + r) * 128 + (((nt & 7) ^ (r & 7)) << 4) + 4 * qd;
                            unsigned int two;
                            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(two) : "r"(at) : "memory");
                            const unsigned int kept = finite_only<T>(two);
                            const T *pair = reinterpret_cast<const T *>(&two);
                            const float v0 = rope::to_f32(pair[0]), v1 = rope::to_f32(pair[1]);
                            const bool odd0 = (two ^ kept) & 0xffffu, odd1 = (two ^ kept) & 0xffff0000u;
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                                for (int hh = 0; hh < 2; ++hh)
                                    if (key0 + r <= limit[mt][hh]) {
                                        if (odd0) o[mt][nt][2 * hh] += wt[mt][hh] * v0;
                                        if (odd1) o[mt][nt][2 * hh + 1] += wt[mt][hh] * v1;
                                    }
                        }
                    }
                }
                // zeros written here are ordered before the TMA writes that reuse the stage
                if (wrote) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(empty(s));
            }

            // ---- the unit's rows: join the KG warps of a row group ----
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    l[mt][hh] += __shfl_xor_sync(kFull, l[mt][hh], 1);
                    l[mt][hh] += __shfl_xor_sync(kFull, l[mt][hh], 2);
                    if (limit[mt][hh] < 0) {                          // a row without a token, or one that sees nothing
                        m[mt][hh] = -INFINITY;
                        l[mt][hh] = 0.f;
#pragma unroll
                        for (int nt = 0; nt < C::kNt; ++nt) o[mt][nt][2 * hh] = o[mt][nt][2 * hh + 1] = 0.f;
                    }
                    if (KG > 1 && qd == 0) ml[kg * C::kRows + 16 * (MT * rg + mt) + g + 8 * hh] = make_float2(m[mt][hh], l[mt][hh]);
                }
            if constexpr (KG > 1) {
                consumer_barrier(cthreads);                           // also: every warp is done with the tiles before
                const unsigned int buf = ring + (it % p.n_stages) * C::kStageBytes;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        const int r = 16 * (MT * rg + mt) + g + 8 * hh;
                        float M = -INFINITY, L = 0.f;
#pragma unroll
                        for (int k = 0; k < KG; ++k) M = fmaxf(M, ml[k * C::kRows + r].x);
#pragma unroll
                        for (int k = 0; k < KG; ++k) {
                            const float2 y = ml[k * C::kRows + r];
                            L += y.y * (y.x == -INFINITY ? 0.f : ex2_approx(y.x - M));
                        }
                        const float f = m[mt][hh] == -INFINITY ? 0.f : ex2_approx(m[mt][hh] - M);
#pragma unroll
                        for (int nt = 0; nt < C::kNt; ++nt) {
                            o[mt][nt][2 * hh] *= f;
                            o[mt][nt][2 * hh + 1] *= f;
                        }
                        m[mt][hh] = M;
                        l[mt][hh] = L;
                    }
#pragma unroll
                for (int pass = 0; pass < C::kJoinPasses; ++pass)
#pragma unroll
                    for (int half = KG / 2; half >= 1; half /= 2) {
                        if (pass > 0 || half < KG / 2) consumer_barrier(cthreads);
                        const int pair = kg % half;
                        const unsigned int at = buf + ((pair * RG + rg) * MT * C::kNtPass * 32 + lane) * 16;
                        if (kg >= half && kg < 2 * half) {
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                                for (int nt = 0; nt < C::kNtPass; ++nt) {
                                    const float(&y)[4] = o[mt][pass * C::kNtPass + nt];
                                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at + (mt * C::kNtPass + nt) * 512), "f"(y[0]), "f"(y[1]),
                                                 "f"(y[2]), "f"(y[3])
                                                 : "memory");
                                }
                        }
                        consumer_barrier(cthreads);
                        if (kg < half) {
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                                for (int nt = 0; nt < C::kNtPass; ++nt) {
                                    float y[4];
                                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                                                 : "=f"(y[0]), "=f"(y[1]), "=f"(y[2]), "=f"(y[3])
                                                 : "r"(at + (mt * C::kNtPass + nt) * 512)
                                                 : "memory");
#pragma unroll
                                    for (int e = 0; e < 4; ++e) o[mt][pass * C::kNtPass + nt][e] += y[e];
                                }
                        }
                    }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(empty(it % p.n_stages));
                ++it;
            }
            const bool whole = j0 == 0 && j1 == w.n;
            const int unit = (b * p.Hkv + h) * p.row_tiles + rt;
            if (kg == 0) {
                const int slot = 2 * static_cast<int>(c) + (j0 == 0 ? 1 : 0);
                float *part = p.parts + static_cast<long long>(slot) * C::kSlotFloats;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        const int r = 16 * (MT * rg + mt) + g + 8 * hh;
                        if (r >= rows_here) continue;
                        const float L = l[mt][hh];
                        if (whole) {
                            const int rr = rt * C::kRows + r, tok = rr / p.group, head = h * p.group + rr - tok * p.group;
                            const long long row = (static_cast<long long>(b) * p.T + tok) * p.Hq + head;
                            const float inv = L == 0.f ? 0.f : 1.f / L;
                            unsigned int *out = reinterpret_cast<unsigned int *>(static_cast<T *>(p.out) + row * p.D);
#pragma unroll
                            for (int nt = 0; nt < C::kNt; ++nt)
                                if (nt * 8 < p.D) out[nt * 4 + qd] = pack_pair<T>(o[mt][nt][2 * hh] * inv, o[mt][nt][2 * hh + 1] * inv);
                            if (p.lse && qd == 0) p.lse[row] = L == 0.f ? -INFINITY : (fmaxf(m[mt][hh], -3e38f) + log2f(L)) * kLn2;
                        } else {
#pragma unroll
                            for (int nt = 0; nt < C::kNt; ++nt)
                                if (nt * 8 < p.D)
                                    __stcg(reinterpret_cast<float2 *>(part + r * DP + nt * 8 + 2 * qd), make_float2(o[mt][nt][2 * hh], o[mt][nt][2 * hh + 1]));
                            if (qd == 0) __stcg(reinterpret_cast<float2 *>(part + C::kRows * DP + 2 * r), make_float2(m[mt][hh], L));
                        }
                    }
                if (!whole && j0 == 0 && warp == 0 && lane == 0) {
                    // the unit's last tile is (unit's first tile of all) + n - 1; the block that owns it ends the parts
                    const long long last = t - j0 + w.n - 1;
                    const int end = static_cast<int>(((last + 1) * G - 1) / total);
                    p.splits[blockIdx.x].unit = unit;
                    p.splits[blockIdx.x].parts = end - static_cast<int>(c) + 1;
                }
            }
            t += j1 - j0;
            w.j = j1 - 1;
            if (t < t1) walk_next(w, base, p.B, p.Hkv, p.row_tiles);
            if constexpr (KG == 1) consumer_barrier(cthreads);          // the query rows in shared memory are done with
        }
    }
    if (*give_up && tid % 32 == 0) atomicOr(p.flags, CSD_CACHE_INTERNAL);
}

// Joins the parts of split units.  Block (c, y): the unit that begins in block c of the kernel before, query rows 8 y ..; a warp per row.
template <typename T, int DP>
__global__ void __launch_bounds__(256) attention_join_kernel(const Params p, int rows_per_tile)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int c = blockIdx.x, lane = threadIdx.x & 31;
    const int r = blockIdx.y * 8 + (threadIdx.x >> 5);
    const int unit = __ldcg(&p.splits[c].unit), n = __ldcg(&p.splits[c].parts);
    if (n == 0) return;
    const int rt = unit % p.row_tiles, bh = unit / p.row_tiles, b = bh / p.Hkv, h = bh - b * p.Hkv;
    if (r >= min(rows_per_tile, p.rows - rt * rows_per_tile)) return;
    const long long slot_floats = static_cast<long long>(rows_per_tile) * (DP + 2);
    auto slot = [&](int i) { return p.parts + slot_floats * (i == 0 ? 2 * c + 1 : 2 * (c + i)); };
    float M = -INFINITY;
    for (int i = lane; i < n; i += 32) M = fmaxf(M, __ldcg(slot(i) + rows_per_tile * DP + 2 * r));
#pragma unroll
    for (int d = 16; d; d >>= 1) M = fmaxf(M, __shfl_xor_sync(kFull, M, d));
    constexpr int E = DP / 32;                                          // columns of a lane: 2, 4 or 8, side by side
    float o[E], L = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    for (int i0 = 0; i0 < n; i0 += 32) {
        float wt = 0.f, wl = 0.f;
        if (i0 + lane < n) {
            const float2 y = __ldcg(reinterpret_cast<const float2 *>(slot(i0 + lane) + rows_per_tile * DP + 2 * r));
            wt = y.x == -INFINITY ? 0.f : ex2_approx(y.x - M);
            wl = y.y * wt;
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) wl += __shfl_xor_sync(kFull, wl, d);
        L += wl;
        const int here = min(32, n - i0);
#pragma unroll 8
        for (int i = 0; i < here; ++i) {
            const float f = __shfl_sync(kFull, wt, i);
            const float *from = slot(i0 + i) + r * DP + lane * E;
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                if (lane * E + e < p.D) {
                    const float2 y = __ldcg(reinterpret_cast<const float2 *>(from + e));
                    o[e] += f * y.x;
                    o[e + 1] += f * y.y;
                }
            }
        }
    }
    const int rr = rt * rows_per_tile + r, tok = rr / p.group, head = h * p.group + rr - tok * p.group;
    const long long row = (static_cast<long long>(b) * p.T + tok) * p.Hq + head;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    unsigned int *out = reinterpret_cast<unsigned int *>(static_cast<T *>(p.out) + row * p.D);
#pragma unroll
    for (int e = 0; e < E; e += 2)
        if (lane * E + e < p.D) out[(lane * E + e) / 2] = pack_pair<T>(o[e] * inv, o[e + 1] * inv);
    if (p.lse && lane == 0) p.lse[row] = L == 0.f ? -INFINITY : (fmaxf(M, -3e38f) + log2f(L)) * kLn2;
}

}  // namespace attention
}  // namespace csd
