// Attention of a row's newest tokens over its paged keys and values, split over the length and joined.
//
//   out[b,t,h] = sum_j w_j v_j,  w = softmax_j(scale q.k_j),  over the places j <= lens[b] - n_new[b] + t
//   lse[b,t,h] = ln sum_j exp(scale q.k_j)
//
// A run of places gives a part (m, l, O) = (max_j x_j, sum_j 2^(x_j - m), sum_j 2^(x_j - m) v_j) with x = scale log2(e) q.k, and
// parts join as M = max m_i, L = sum l_i 2^(m_i - M), O = sum O_i 2^(m_i - M) / L.
//
// Bound: memory (each key and value is read once; T g query rows share it, g = query heads per key head); for a short cache the
// latency of the chain lengths -> page ids -> tiles -> join, 9.7 us with one row of 700 tokens.
// Measured with keys and values of 0.1 to 1.2 GB, bf16, 8 key heads of 128: 6.0 TB/s for one row of 131071 tokens and one new token
// (89.7 us, 32 query heads), 5.9 for 128 rows of 500 to 4000 with nine (203 us), 5.2 for 32 ragged rows up to 8191 with six (104 us),
// 3.2 for one row of 30001 with 72 query rows to a key head (39.0 us: half of it is the start, the parts' way out and the join).
//
// Two kernels, by query rows to a key head and row of the cache: up to 16 fit one mma.sync tile held in registers; beyond, up to 128 rows
// share a tensor-memory tile.  With pages of 16 tokens, first kernel and second: 32 ragged rows up to 8191 tokens, dim 128: 97 us and 105
// with 10 query rows, 96 and 106 with 15, 97 and 107 with 16, 156 and 105 with 20, 166 and 107 with 30; 128 rows of 500 to 4000, dim 64:
// 110 and 162 with 8 and 16, 194 and 167 with 20, 197 and 171 with 32; 32 rows up to 4095, dim 256: 108 and 128 with 8, 119 and 127 with 16,
// 202 and 130 with 20.  Beyond 16 the first kernel has a second row tile, which reads every key again.
//
//   attention_kernel  persistent.  The tiles (kTile places of one row and key head) of all rows and heads, laid out row after
//                     row, are split evenly and contiguously over the blocks, whatever the rows' lengths are (read on the
//                     device), so a block works on a run of tiles of a few (row, head) units.
//       producer warp  puts the tile's keys and values, page by page, into a ring of shared-memory stages by TMA (boxes of
//                     64 elements x the places of one page, 128-byte swizzle; elements beyond dim read as zero)
//       consumer warps four: a warp owns 16 NK of a tile's places, against all of the unit's query rows (at most 16), with its
//                     own running (m, l, O) in registers: no exchange between warps until the unit ends.  Products are
//                     mma.sync m16n8k16 with float32 accumulators: with 16 query rows the tensor pipe is at a tenth of its
//                     limit while the tiles stream.
//     At the end of a unit the warps join through a ring stage that the producer hands over; a unit that lies in one block whole is written out, otherwise
//     the part goes to the workspace.
//   attention_join_kernel  joins the parts of the units that were split (at most one begins in each block).  A launch of its own: joining
//                     in the last block to finish a unit was slower (103.6 us against 94 for one row of 131071 tokens, 36.9
//                     against 30.6 for 16 rows with a key head to every query head), a chain of cold reads at the end of the slowest block.
// No block waits for another; waits inside a block are bounded, and a block whose wait runs out stays until what it sent for has landed.
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

// What the first block of a split unit leaves for the join: its parts lie in slot 2 first + 1 and slots 2 (first + i), i = 1 .. parts - 1.
struct Split {
    int unit;                 // (row * heads + head) * row tiles + row tile
    int first;                // that block
    int parts;                // 0: not split
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
    int n_stages;
    int run_cost;                          // what beginning and ending a unit costs a block, in tiles
    int by_unit;                           // splits are indexed by unit (no more units than blocks), else by first block
    Split *splits;                         // [min(units, gridDim.x)]
    float *parts;                          // [2 gridDim.x] slots of kRows * (DP + 2) floats
    // the tensor-memory kernel alone
    int tile_rows;                         // query rows of a row tile: a multiple of 8, at most 128
    int q_buffers;                         // sets of query rows: 2, or 1 where they would leave too few slots
    int halves, d16;                       // 64-element columns of a tile; dim rounded up to 16
    int part_stride;                       // floats between rows of a part
    const void *k_pool, *v_pool;           // of this layer
    long long pool_page, pool_head, pool_token;
};

// A variant of the mma.sync kernel: dim padded to DP, 16 NK places to a warp and tile.
template <typename T_, int DP_, int NK_, int kBlocksPerSm_>
struct Config {
    using T = T_;
    static constexpr int DP = DP_, NK = NK_, kBlocksPerSm = kBlocksPerSm_;
    static constexpr int kWarps = 4;
    static constexpr int kTile = 16 * NK * kWarps;
    static constexpr int kRows = 16;
    // Registers move between warpgroups of four warps: the producer's gives up what it does not need.
    static constexpr int kThreads = 32 * (kWarps + 4);
    static constexpr int kGroups = kWarps / 4 + 1;
    static constexpr int kLaunchRegs = 65536 / (kThreads * kBlocksPerSm) / 8 * 8;          // per thread, as launched (the host checks)
    static constexpr bool kMoveRegs = kLaunchRegs < 232;
    static constexpr int kProducerRegs = 40;
    static constexpr int kConsumerRegs = (kGroups * kLaunchRegs - kProducerRegs) / (kGroups - 1) / 8 * 8;
    static_assert(!kMoveRegs || (kConsumerRegs <= 240 && kConsumerRegs * (kGroups - 1) + kProducerRegs <= kGroups * kLaunchRegs), "register split");
    static constexpr int kHalves = DP / 64;                        // 128-byte columns of a tile
    static constexpr int kTileBytes = kTile * DP * 2;               // keys or values of a stage
    static constexpr int kStageBytes = 2 * kTileBytes;
    static constexpr int kQBytes = kRows * DP * 2;
    static constexpr int kMlBytes = kWarps * kRows * 8;
    static constexpr int kSlotFloats = kRows * (DP + 2);
    static constexpr bool kQInRegisters = DP <= 128;
    static constexpr int kNt = DP / 8;                              // column tiles of 8
    static_assert(kWarps * kRows * DP * 4 <= kStageBytes, "the warps' sums fit in a stage");
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
// Weights go into the second product in the cache's type: a relative error of 2^-9 (bfloat16) or 2^-12 (float16) of each, of random
// sign, where the result itself is rounded to that type; the sum l is taken before the rounding.  Float16 steps by 2^-24 below 2^-14, and
// what is below 2^-25 of the largest weight would be counted in l and dropped from the product (0.4 % of the result for 131072 places
// of 2^-25).  So a row's reference m lies this many powers of two below the maximum: O and l carry the factor, their quotient and
// m + log2 l do not.  Float16 holds 2^15; in the kernel whose reference may lag by 2^kLag that much is left for it.  What remains is
// at most 2^-39 of the largest weight per place, or 2^-32.
constexpr int kLag = 8;
template <typename T>
__device__ __forceinline__ constexpr float raised(int lag)
{
    return ExponentBits<T>::value == 0x7c00u ? static_cast<float>(lag == 0 ? 14 : 15 - lag) : 0.f;
}
template <typename T>
__device__ __forceinline__ unsigned int finite_only(unsigned int two)
{
    constexpr unsigned int e = ExponentBits<T>::value;
    if ((two & e) == e) two &= 0xffff0000u;
    if ((two & (e << 16)) == (e << 16)) two &= 0x0000ffffu;
    return two;
}

__device__ __forceinline__ void consumer_barrier(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }

// A place in a ring of slots that are taken in order: the slot, and the parity of the round.
struct Cursor {
    int slot;
    unsigned int round;
    __device__ __forceinline__ void next(int slots)
    {
        if (++slot == slots) {
            slot = 0;
            round ^= 1u;
        }
    }
};

// The split.  A unit of n tiles counts n + run_cost positions, the first run_cost of them empty: what its beginning and its end
// cost a block.  The positions of all units are split evenly over the blocks; a block's share [x, x1) is a few runs of tiles.
struct Run {
    int b, h, rt;             // row, key head, row tile
    int j0, ns, n;            // first tile, tiles here, tiles of the unit
    int at;                   // position of the unit's first tile
};

struct Runs {
    const int *base;          // base[b]: positions of the rows before b (one head, one row tile)
    int B, Hkv, row_tiles, cost;
    int b, h, rt;
    int x, x1, unit;          // next position, end of the share, first position of the unit

    __device__ __forceinline__ void begin(const Params &p, const int *base_, int x0, int end)
    {
        base = base_;
        B = p.B;
        Hkv = p.Hkv;
        row_tiles = p.row_tiles;
        cost = p.run_cost;
        x = x0;
        x1 = end;
        b = h = rt = 0;
        unit = 0;
        if (x >= x1) return;
        const int hr = Hkv * row_tiles;
        int lo = 0, hi = B - 1;                              // the last row whose positions begin at or before x has some
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (base[mid] * hr <= x) lo = mid; else hi = mid - 1;
        }
        b = lo;
        const int each = base[b + 1] - base[b];
        const int hrt = static_cast<int>(static_cast<unsigned int>(x - base[b] * hr) / static_cast<unsigned int>(each));
        unit = base[b] * hr + hrt * each;
        h = hrt / row_tiles;
        rt = hrt - h * row_tiles;
    }

    __device__ __forceinline__ bool next(Run &r)
    {
        while (x < x1) {
            const int each = base[b + 1] - base[b];
            r.b = b;
            r.h = h;
            r.rt = rt;
            r.n = each - cost;
            r.at = unit + cost;
            r.j0 = max(x - r.at, 0);
            r.ns = min(r.n, x1 - r.at) - r.j0;
            unit += each;
            x = unit;
            if (++rt == row_tiles) {
                rt = 0;
                if (++h == Hkv) {
                    h = 0;
                    do {
                        ++b;
                    } while (b < B && base[b + 1] == base[b]);
                }
            }
            if (r.ns > 0) return true;
        }
        return false;
    }
};

__device__ __forceinline__ int row_len(const Params &p, int b) { return min(max(ptx::ld_written(p.lens + b), 0), p.max_pages << p.page_shift); }
// (may be more than T: a pass over the first T of them)
__device__ __forceinline__ int row_news(const Params &p, int b) { return p.n_new ? max(ptx::ld_written(p.n_new + b), 0) : p.T; }

// base[b + 1] holds the positions of row b; becomes base[b] = positions of the rows before b.  One warp.
__device__ __forceinline__ void scan_tiles(int *base, int B)
{
    const int lane = threadIdx.x & 31;
    int sum = 0;
    for (int b0 = 0; b0 < B; b0 += 32) {
        int v = b0 + lane < B ? base[b0 + lane + 1] : 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(kFull, v, d);
            if (lane >= d) v += o;
        }
        if (b0 + lane < B) base[b0 + lane + 1] = sum + v;
        sum += __shfl_sync(kFull, v, 31);
    }
    if (lane == 0) base[0] = 0;
}

// The page that lane f < per_tile looks after in a tile; -1: nothing to load.
template <int kTile>
__device__ __forceinline__ int tile_page(const Params &p, int b, int j, int len, int lane, int per_tile)
{
    const int place = j * kTile + lane * p.box_rows;
    if (lane >= per_tile || place >= len) return -1;
    const int id = ptx::ld_written(p.table + static_cast<long long>(b) * p.max_pages + (place >> p.page_shift));
    if (id >= 0 && id < p.n_pages) return id;
    atomicOr(p.flags, CSD_CACHE_BAD_PAGE);
    return p.n_pages;                                    // outside the tensor map: reads as zeros
}

// This block's share of the positions, and the block that a position belongs to.  The host sees to it that positions fit in 31 bits:
// divisions of 64 bits here and in Runs cost a microsecond before the first load.
struct Share {
    unsigned int total, blocks, each, more;              // total = each blocks + more; every one of these blocks has a position at least
    int x0, x1;
    __device__ __forceinline__ Share(const Params &p, const int *base)
    {
        total = static_cast<unsigned int>(base[p.B] * p.Hkv * p.row_tiles);
        blocks = max(min(gridDim.x, total), 1u);
        each = total / blocks;
        more = total - each * blocks;
        x0 = from(min(blockIdx.x, blocks));
        x1 = from(min(blockIdx.x + 1, blocks));
    }
    __device__ __forceinline__ int from(unsigned int c) const { return static_cast<int>(c * each + c * more / blocks); }
    __device__ __forceinline__ int owner(int x) const
    {
        unsigned int c = static_cast<unsigned int>(static_cast<float>(x) / static_cast<float>(total) * static_cast<float>(blocks));
        while (c > 0 && from(c) > x) --c;                // at most a step or two: the quotient is good to 2^-22 of the blocks
        while (from(c + 1) <= x) ++c;
        return static_cast<int>(c);
    }
};

// The block with a unit's first tile says whether it was split.
__device__ __forceinline__ void note_split(const Params &p, const Share &s, const Run &r)
{
    if (r.j0 != 0) return;
    const int unit = (r.b * p.Hkv + r.h) * p.row_tiles + r.rt;
    const int parts = r.ns == r.n ? 0 : s.owner(r.at + r.n - 1) - static_cast<int>(blockIdx.x) + 1;
    if (!p.by_unit && parts == 0) return;
    Split *to = p.splits + (p.by_unit ? unit : static_cast<int>(blockIdx.x));
    to->unit = unit;
    to->first = blockIdx.x;
    to->parts = parts;
}

// Zeros for rows that have nothing to read.
template <typename T>
__device__ __forceinline__ void zero_empty_rows(const Params &p, const int *base, int tid, int threads)
{
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
        if (base[b + 1] != base[b]) continue;
        if (p.by_unit)
            for (int i = tid; i < p.Hkv * p.row_tiles; i += threads) p.splits[b * p.Hkv * p.row_tiles + i].parts = 0;
        const long long row0 = static_cast<long long>(b) * p.T * p.Hq;
        uint4 *o = reinterpret_cast<uint4 *>(static_cast<T *>(p.out) + row0 * p.D);
        const int vecs = p.T * p.Hq * p.D / 8;
        for (int i = tid; i < vecs; i += threads) o[i] = make_uint4(0, 0, 0, 0);
        if (p.lse)
            for (int i = tid; i < p.T * p.Hq; i += threads) p.lse[row0 + i] = -INFINITY;
    }
}

// Adds w v for the infinities and NaN among 32 elements (from c0) of the values in places [from, to], which the product left
// out, to one row's accumulators; w is computed again.  Rare: straight from global memory.
template <typename T>
__device__ __noinline__ void add_left_out(const Params &p, int b, int h, int tok, int head, int c0, int from, int to, float m, float (&o)[32])
{
    const T *q = static_cast<const T *>(p.q) + b * p.qb + tok * p.qt + head * p.qh;
    for (int key = from; key <= to; ++key) {
        const int page = ptx::ld_written(p.table + static_cast<long long>(b) * p.max_pages + (key >> p.page_shift));
        if (page < 0 || page >= p.n_pages) continue;
        const long long at = page * p.pool_page + h * p.pool_head + (key & ((1 << p.page_shift) - 1)) * p.pool_token;
        const T *k = static_cast<const T *>(p.k_pool) + at, *v = static_cast<const T *>(p.v_pool) + at;
        float x = 0.f;
        for (int d = 0; d < p.D; ++d) x += rope::to_f32(q[d]) * rope::to_f32(k[d]);
        const float w = ex2_approx(x * p.scale_log2 - m);
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            if (c0 + e >= p.D) break;
            const float y = rope::to_f32(v[c0 + e]);
            if (!isfinite(y)) o[e] += w * y;
        }
    }
}

template <typename C>
__global__ void __launch_bounds__(C::kThreads, C::kBlocksPerSm)
attention_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Params p)
{
    using T = typename C::T;
    constexpr int DP = C::DP, NK = C::NK, kTile = C::kTile;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bar_words[3 * kMaxStages];
    __shared__ int give_up_flag;
    volatile int *give_up = &give_up_flag;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned int ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const unsigned int q_smem = ring + p.n_stages * C::kStageBytes;
    unsigned char *after_q = smem_raw + (q_smem - smem_u32(smem_raw)) + C::kQBytes;
    float2 *ml = reinterpret_cast<float2 *>(after_q);                              // [kWarps][kRows]
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
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    }
    ptx::wait_for_stream();
    if (tid == 0 && !p.by_unit) p.splits[blockIdx.x].parts = 0;
    // tiles of each row; rows without any give zeros
    for (int b = tid; b < p.B; b += C::kThreads) {
        const int len = row_len(p, b), news = row_news(p, b);
        base[b + 1] = news > 0 && len > 0 ? (len + kTile - 1) / kTile + p.run_cost : 0;
    }
    __syncthreads();
    if (warp == 0) scan_tiles(base, p.B);
    __syncthreads();
    const Share share(p, base);

    if (warp >= C::kWarps) {
        // ---- producer: one warp of its group ----
        if constexpr (C::kMoveRegs) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kProducerRegs));
        if (warp == C::kWarps) {
            Runs runs;
            runs.begin(p, base, share.x0, share.x1);
            Run r, rn;
            bool more = runs.next(r);
            const int per_tile = kTile / p.box_rows;               // pages of a tile (1 where a page is larger)
            const unsigned int box_bytes = static_cast<unsigned int>(p.box_rows) * 128u;
            int len = more ? row_len(p, r.b) : 0;
            // page ids are fetched a tile ahead
            int id = more ? tile_page<kTile>(p, r.b, r.j0, len, lane, per_tile) : -1;
            Cursor at_ring = {0, 0u};
            bool ok = true;
            while (more && ok) {
                const bool follows = runs.next(rn);
                const int len_next = follows ? row_len(p, rn.b) : 0;
                for (int i = 0; i < r.ns && ok; ++i) {
                    const int page = id, j = r.j0 + i;
                    id = i + 1 < r.ns ? tile_page<kTile>(p, r.b, j + 1, len, lane, per_tile)
                                      : (follows ? tile_page<kTile>(p, rn.b, rn.j0, len_next, lane, per_tile) : -1);
                    const int s = at_ring.slot;
                    const unsigned int there = __ballot_sync(kFull, page >= 0);
                    if (lane == 0) {
                        ok = mbar_wait(empty(s), at_ring.round ^ 1u, give_up);
                        if (ok) {
                            const unsigned int bytes = static_cast<unsigned int>(__popc(there)) * box_bytes * C::kHalves;
                            mbar_expect_tx(full_k(s), bytes);
                            mbar_expect_tx(full_v(s), bytes);
                        }
                    }
                    ok = __shfl_sync(kFull, ok ? 1 : 0, 0) != 0;
                    if (ok && page >= 0) {
                        const int in_page = p.box_rows == kTile ? (j * kTile) & ((1 << p.page_shift) - 1) : 0;
                        const unsigned int at = ring + s * C::kStageBytes + lane * box_bytes;
#pragma unroll
                        for (int hf = 0; hf < C::kHalves; ++hf) tma_load_page(at + hf * (kTile * 128), &map_k, full_k(s), hf * 64, in_page, r.h, page);
#pragma unroll
                        for (int hf = 0; hf < C::kHalves; ++hf)
                            tma_load_page(at + C::kTileBytes + hf * (kTile * 128), &map_v, full_v(s), hf * 64, in_page, r.h, page);
                    }
                    at_ring.next(p.n_stages);
                }
                if (ok) {                                            // the consumers join through the next stage, once it is theirs
                    const int sj = at_ring.slot;
                    if (lane == 0) {
                        ok = mbar_wait(empty(sj), at_ring.round ^ 1u, give_up);
                        if (ok) {
                            mbar_arrive(full_k(sj));
                            mbar_arrive(full_v(sj));
                        }
                    }
                    at_ring.next(p.n_stages);
                    ok = __shfl_sync(kFull, ok ? 1 : 0, 0) != 0;
                }
                if (lane == 0) note_split(p, share, r);
                r = rn;
                len = len_next;
                more = follows;
            }
        }
    } else {
        // ---- consumers ----
        if constexpr (C::kMoveRegs) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kConsumerRegs));
        const int g = lane >> 2, qd = lane & 3;
        const int cthreads = C::kWarps * 32;
        zero_empty_rows<T>(p, base, tid, cthreads);
        Runs runs;
        runs.begin(p, base, share.x0, share.x1);
        Run run, next;
        Cursor at_ring = {0, 0u};
        constexpr int kFetch = C::kRows * (DP / 8) / (C::kWarps * 32);       // 16-byte pieces of the query rows for a thread
        uint4 fetched[kFetch];
        auto fetch = [&](const Run &x) {
            const int here = min(C::kRows, p.rows - x.rt * C::kRows);
#pragma unroll
            for (int k = 0; k < kFetch; ++k) {
                const int i = tid + k * C::kWarps * 32, r = i / (DP / 8), ch = i % (DP / 8);
                fetched[k] = make_uint4(0, 0, 0, 0);
                if (r < here && ch * 8 < p.D) {
                    const int rr = x.rt * C::kRows + r, tok = rr / p.group, head = x.h * p.group + rr - tok * p.group;
                    fetched[k] = ptx::ld_written(reinterpret_cast<const uint4 *>(static_cast<const T *>(p.q) + x.b * p.qb + tok * p.qt + head * p.qh + ch * 8));
                }
            }
        };
        bool more = runs.next(next);
        if (more) fetch(next);
        const int swz = lane & 7;
        const unsigned int k_lane = (16 * NK * warp + ((lane >> 4) << 3) + swz) * 128u, k_chunk = (lane >> 3) & 1;
        const unsigned int v_lane = (16 * NK * warp + (((lane >> 3) & 1) << 3) + swz) * 128u, v_chunk = lane >> 4;
        const unsigned int q_lane = ((((lane >> 3) & 1) << 3) + swz) * 128u, q_chunk = lane >> 4;

        while (more) {
            run = next;
            more = runs.next(next);
            // ---- a unit, or the part of one that lies in this block ----
            const int b = run.b, h = run.h, rt = run.rt, j0 = run.j0, j1 = run.j0 + run.ns;
            const int len = row_len(p, b), news = row_news(p, b);
            const int rows_here = min(C::kRows, p.rows - rt * C::kRows);
            // its query rows, on their way since the run before began: row r is token r / group, query head h * group + r % group
#pragma unroll
            for (int k = 0; k < kFetch; ++k) {
                const int i = tid + k * C::kWarps * 32, r = i / (DP / 8), ch = i % (DP / 8);
                const unsigned int at = q_smem + (ch >> 3) * (C::kRows * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(fetched[k].x), "r"(fetched[k].y), "r"(fetched[k].z), "r"(fetched[k].w) : "memory");
            }
            if (more) fetch(next);
            consumer_barrier(cthreads);
            int limit[2];                                           // last place that the thread's rows see; -1: none
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const int r = g + 8 * hh, rr = rt * C::kRows + r, tok = rr / p.group;
                limit[hh] = r < rows_here && tok < news ? len - news + tok : -1;
            }
            unsigned int qf[C::kQInRegisters ? DP / 16 : 1][4];
            if constexpr (C::kQInRegisters) {
#pragma unroll
                for (int ks = 0; ks < DP / 16; ++ks)
                    ldsm4(qf[ks], q_smem + (ks >> 2) * (C::kRows * 128) + q_lane + ((((ks & 3) * 2 + q_chunk) ^ swz) << 4));
            }
            float o[C::kNt][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
            for (int nt = 0; nt < C::kNt; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][e] = 0.f;

            for (int j = j0; j < j1; ++j, at_ring.next(p.n_stages)) {
                const int s = at_ring.slot;
                const unsigned int parity = at_ring.round;
                const unsigned int k_at = ring + s * C::kStageBytes, v_at = k_at + C::kTileBytes;
                const int key0 = j * kTile + 16 * NK * warp;          // the warp's first place
                float x[2 * NK][4];
#pragma unroll
                for (int n = 0; n < 2 * NK; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[n][e] = 0.f;
                mbar_wait(full_k(s), parity, give_up);
                const bool any = key0 < len;                         // nothing of the warp's places exists otherwise
                if (any) {
#pragma unroll
                    for (int ks = 0; ks < DP / 16; ++ks) {
                        unsigned int qa[4];
                        if constexpr (C::kQInRegisters) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) qa[e] = qf[ks][e];
                        } else {
                            ldsm4(qa, q_smem + (ks >> 2) * (C::kRows * 128) + q_lane + ((((ks & 3) * 2 + q_chunk) ^ swz) << 4));
                        }
#pragma unroll
                        for (int nk = 0; nk < NK; ++nk) {
                            unsigned int kb[4];
                            ldsm4(kb, k_at + (ks >> 2) * (kTile * 128) + k_lane + nk * (16 * 128) + ((((ks & 3) * 2 + k_chunk) ^ swz) << 4));
                            mma16816<T>(x[2 * nk], qa, kb[0], kb[1]);
                            mma16816<T>(x[2 * nk + 1], qa, kb[2], kb[3]);
                        }
                    }
                }
                // scores in powers of two; places that a row does not see become -inf whatever was computed for them
                const bool edge = key0 + 16 * NK - 1 > len - news;   // some row does not see all of the warp's places
#pragma unroll
                for (int n = 0; n < 2 * NK; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[n][e] *= p.scale_log2;
                        if (edge && key0 + 8 * n + 2 * qd + (e & 1) > limit[e >> 1]) x[n][e] = -INFINITY;
                    }
                float mx[2], at0[2];
                bool grew = false;
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    float v = x[0][2 * hh];
#pragma unroll
                    for (int n = 0; n < 2 * NK; ++n) v = fmaxf(v, fmaxf(x[n][2 * hh], x[n][2 * hh + 1]));
                    v = fmaxf(v, __shfl_xor_sync(kFull, v, 1));
                    v = fmaxf(v, __shfl_xor_sync(kFull, v, 2));
                    mx[hh] = fmaxf(m[hh], v - raised<T>(0));
                    grew |= mx[hh] > m[hh];
                    at0[hh] = mx[hh] == -INFINITY ? 0.f : mx[hh];
                }
                if (__any_sync(kFull, grew)) {
                    float f[2];
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        f[hh] = ex2_approx(m[hh] - at0[hh]);
                        l[hh] *= f[hh];
                        m[hh] = mx[hh];
                    }
#pragma unroll
                    for (int nt = 0; nt < C::kNt; ++nt) {
                        o[nt][0] *= f[0];
                        o[nt][1] *= f[0];
                        o[nt][2] *= f[1];
                        o[nt][3] *= f[1];
                    }
                }
#pragma unroll
                for (int n = 0; n < 2 * NK; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[n][e] = ex2_approx(x[n][e] - at0[e >> 1]);
                        l[e >> 1] += x[n][e];
                    }
                unsigned int pa[NK][4];
#pragma unroll
                for (int nk = 0; nk < NK; ++nk) {
                    pa[nk][0] = pack_pair<T>(x[2 * nk][0], x[2 * nk][1]);
                    pa[nk][1] = pack_pair<T>(x[2 * nk][2], x[2 * nk][3]);
                    pa[nk][2] = pack_pair<T>(x[2 * nk + 1][0], x[2 * nk + 1][1]);
                    pa[nk][3] = pack_pair<T>(x[2 * nk + 1][2], x[2 * nk + 1][3]);
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
                        const unsigned int at = v_at + (ch >> 3) * (kTile * 128) + (16 * NK * warp + r) * 128 + (((ch & 7) ^ (r & 7)) << 4);
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
                            mma16816<T>(o[2 * n2], pa[nk], vb[0], vb[1]);
                            mma16816<T>(o[2 * n2 + 1], pa[nk], vb[2], vb[3]);
                        }
                }
                if (odd_values) {                                    // what was left out, for the rows that see it
                    for (int r = 0; r < 16 * NK && key0 + r < len; ++r) {
                        const int src = (lane & ~3) | ((r & 7) >> 1);
                        float wt[2];
#pragma unroll
                        for (int hh = 0; hh < 2; ++hh) {
                            wt[hh] = 0.f;
#pragma unroll
                            for (int n = 0; n < 2 * NK; ++n)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const float y = __shfl_sync(kFull, x[n][2 * hh + e], src);
                                    if (n == (r >> 3) && e == (r & 1)) wt[hh] = y;
                                }
                        }
#pragma unroll
                        for (int nt = 0; nt < C::kNt; ++nt) {
                            const unsigned int at = v_at + (nt >> 3) * (kTile * 128) + (16 * NK * warp + r) * 128 + (((nt & 7) ^ (r & 7)) << 4) + 4 * qd;
                            unsigned int two;
                            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(two) : "r"(at) : "memory");
                            const unsigned int kept = finite_only<T>(two);
                            const T *pair = reinterpret_cast<const T *>(&two);
                            const float v0 = rope::to_f32(pair[0]), v1 = rope::to_f32(pair[1]);
                            const bool odd0 = (two ^ kept) & 0xffffu, odd1 = (two ^ kept) & 0xffff0000u;
#pragma unroll
                            for (int hh = 0; hh < 2; ++hh)
                                if (key0 + r <= limit[hh]) {
                                    if (odd0) o[nt][2 * hh] += wt[hh] * v0;
                                    if (odd1) o[nt][2 * hh + 1] += wt[hh] * v1;
                                }
                        }
                    }
                }
                // zeros written here are ordered before the TMA writes that reuse the stage
                if (wrote) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(empty(s));
            }

            // ---- the unit's rows: the warps' sums meet in the next stage, and the rows leave from there side by side ----
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                l[hh] += __shfl_xor_sync(kFull, l[hh], 1);
                l[hh] += __shfl_xor_sync(kFull, l[hh], 2);
                if (limit[hh] < 0) {                                  // a row without a token, or one that sees nothing
                    m[hh] = -INFINITY;
                    l[hh] = 0.f;
                }
                if (qd == 0) ml[warp * C::kRows + g + 8 * hh] = make_float2(m[hh], l[hh]);
            }
            // The stage is handed over by the producer: without this wait the arrivals on empty() below could come before the producer's
            // test of the phase before, which by parity then reads as still open.
            mbar_wait(full_k(at_ring.slot), at_ring.round, give_up);
            consumer_barrier(cthreads);                               // every warp is done with the tiles before
            // element (row, column) of a warp's sums; the columns' order within a row is turned by the row, so that the eight rows a
            // warp writes at once fall on different banks
            float *sums = reinterpret_cast<float *>(smem_raw + (ring - smem_u32(smem_raw)) + at_ring.slot * C::kStageBytes);
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const int r = g + 8 * hh;
                if (r < rows_here) {
#pragma unroll
                    for (int nt = 0; nt < C::kNt; ++nt)
                        *reinterpret_cast<float2 *>(sums + (warp * C::kRows + r) * DP + ((nt * 8) ^ ((r & 3) << 3)) + 2 * qd) =
                            limit[hh] < 0 ? make_float2(0.f, 0.f) : make_float2(o[nt][2 * hh], o[nt][2 * hh + 1]);
                }
            }
            consumer_barrier(cthreads);
            const bool whole = run.ns == run.n;
            float *part = p.parts + static_cast<long long>(2 * static_cast<int>(blockIdx.x) + (j0 == 0 ? 1 : 0)) * C::kSlotFloats;
            for (int i = tid; i < rows_here * (DP / 4); i += cthreads) {
                const int r = i / (DP / 4), c = i % (DP / 4) * 4;
                float2 y[C::kWarps];
                float M = -INFINITY, L = 0.f;
#pragma unroll
                for (int k = 0; k < C::kWarps; ++k) {
                    y[k] = ml[k * C::kRows + r];
                    M = fmaxf(M, y[k].x);
                }
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int k = 0; k < C::kWarps; ++k) {
                    // (a warp that has seen nothing adds nothing; one whose scores were all NaN keeps its NaN)
                    const float f = y[k].x == -INFINITY ? (y[k].y == 0.f ? 0.f : y[k].y) : ex2_approx(y[k].x - M);
                    const float4 z = *reinterpret_cast<const float4 *>(sums + (k * C::kRows + r) * DP + (c ^ ((r & 3) << 3)));
                    L += y[k].y * f;
                    sum.x += z.x * f;
                    sum.y += z.y * f;
                    sum.z += z.z * f;
                    sum.w += z.w * f;
                }
                if (c < p.D) {
                    if (whole) {
                        const int rr = rt * C::kRows + r, tok = rr / p.group, head = h * p.group + rr - tok * p.group;
                        const long long row = (static_cast<long long>(b) * p.T + tok) * p.Hq + head;
                        const float inv = L == 0.f ? 0.f : 1.f / L;
                        *reinterpret_cast<uint2 *>(static_cast<T *>(p.out) + row * p.D + c) =
                            make_uint2(pack_pair<T>(sum.x * inv, sum.y * inv), pack_pair<T>(sum.z * inv, sum.w * inv));
                        if (p.lse && c == 0) p.lse[row] = L == 0.f ? -INFINITY : (fmaxf(M, -3e38f) + log2f(L)) * kLn2;
                    } else {
                        __stcg(reinterpret_cast<float4 *>(part + r * DP + c), sum);
                        if (c == 0) __stcg(reinterpret_cast<float2 *>(part + C::kRows * DP + 2 * r), make_float2(M, L));
                    }
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(empty(at_ring.slot));
            at_ring.next(p.n_stages);
        }
    }
    // a wait ran out (whoever noticed stays, and so does the block)
    if (*give_up) {
        if (tid % 32 == 0) atomicOr(p.flags, CSD_CACHE_INTERNAL);
        ptx::linger();
    }
}

// ---- more than 16 query rows per key head: products on the tensor-memory path -------------------------------------------
//
// The same split over the blocks, parts and join; inside a block
//   warps 0..3  softmax: a thread owns a query row of the row tile.  It reads the row's 64 scores of a tile from tensor memory,
//               writes the weights back there in the cache's type, and keeps (m, l) in registers
//   warp 4      one thread issues the products: S = Q K^T (tcgen05.mma, M = 128 or 64 query rows, N = 64 places, both operands from
//               shared memory) into one of two score buffers, O += P V (P from tensor memory, V read with places as its K)
//   warp 5      the page loads
// Two blocks per SM (one beyond dim 128, whose accumulators take more than half of the tensor memory): while one waits for its scores
// or ends a unit, the other keeps the memory busy.  One block with two such sets that took a run's tiles in turn was slower, 247 us
// against 221 at that time for 1024 units of 8 to 63 tiles: both sets stop at a unit's end together.
// The next run's query rows are fetched, and its first scores computed, while this one ends (where two sets of query rows fit).
// A row tile is always computed as 128 rows (kM), or 64 where these suffice and pay: rows that do not exist read whatever follows in
// shared memory and feed accumulator rows that nobody reads.  Of 128 rows a softmax warp's quarter of the tensor memory holds 32, of
// 64 it holds 16, in its first 16 lanes.  Each query row twice, against either half of a tile's places, took 225 us against 206 (36
// query rows of 128): the products' issue and reads, not the weights, are what a tile waits for (with dim 64 the pipe is busy for
// half of the time).
// The reference of a row stays while no score exceeds it by more than kLag powers of two (weights up to 2^kLag, raised as above, are
// harmless in float32 sums and in either cache type) and jumps to the tile's maximum when one does, so the accumulators in tensor memory are rescaled a few times per unit, not per tile.
constexpr int kTcTile = 64;
constexpr int kTcThreads = 192;
constexpr int kTcMaxSlots = 16;
constexpr unsigned int kTcScoreCols = 64, kTcOutCol = 128;     // tensor memory: scores at 0 and 64 (weights over them), output from 128

template <typename T>
__device__ __forceinline__ unsigned int tc_instr(int m, int n, bool b_mn_major)
{
    constexpr unsigned int type = sizeof(T) == 2 && ExponentBits<T>::value == 0x7f80u ? 1u : 0u;     // 1: bf16, 0: f16
    return (1u << 4) | (type << 7) | (type << 10) | (b_mn_major ? 1u << 16 : 0u) | (static_cast<unsigned int>(n >> 3) << 17) | (static_cast<unsigned int>(m >> 4) << 24);
}
// Values as the second operand: rows of 64 elements (128 bytes, swizzled) are K, the elements within them N.
__device__ __forceinline__ unsigned long long value_desc(unsigned int smem_addr, unsigned int column_bytes)
{
    unsigned long long d = 0;
    d |= static_cast<unsigned long long>((smem_addr & 0x3FFFFu) >> 4);
    d |= static_cast<unsigned long long>(column_bytes >> 4) << 16;           // to the next 64 elements of N
    d |= static_cast<unsigned long long>(1024 >> 4) << 32;                   // to the next 8 places of K
    d |= 1ull << 46;
    d |= 2ull << 61;
    return d;
}
__device__ __forceinline__ void tc_mma_ss(unsigned int d, unsigned long long a, unsigned long long b, unsigned int idesc, unsigned int accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                 "r"(idesc), "r"(accumulate)
                 : "memory");
}
__device__ __forceinline__ void tc_mma_ts(unsigned int d, unsigned int a, unsigned long long b, unsigned int idesc, unsigned int accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b),
                 "r"(idesc), "r"(accumulate)
                 : "memory");
}
// Order of the loads of a run of n tiles, and of the products: K0, K1, V0, K2, V1, ..., K(n-1), V(n-2), V(n-1).  The
// number of V(k) among them:
__device__ __forceinline__ int v_item(int k, int n) { return k == n - 1 ? 2 * n - 1 : 2 * k + 2; }

// The query rows of a unit into shared memory, asynchronously: rows of 128 bytes, swizzled, 64 elements of all rows after one another.
template <typename T>
__device__ __forceinline__ void fetch_rows(const Params &p, const Run &ru, unsigned int to, int warp, int warps, int lane)
{
    const int rows_here = min(p.tile_rows, p.rows - ru.rt * p.tile_rows);
    const int chunks = p.halves * 8, at_once = 32 / chunks, sub = lane / chunks, ch = lane - sub * chunks;
    if (sub >= at_once) return;                                    // (24 pieces leave lanes over)
    for (int r = warp * at_once + sub; r < rows_here; r += warps * at_once) {
        const int rr = ru.rt * p.tile_rows + r, tok = rr / p.group, head = ru.h * p.group + rr - tok * p.group;
        const unsigned int at = to + (ch >> 3) * (p.tile_rows * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
        const bool there = ch * 8 < p.D;                            // elements beyond dim: zeros
        const T *from = static_cast<const T *>(p.q) + ru.b * p.qb + tok * p.qt + head * p.qh + (there ? ch * 8 : 0);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(from), "r"(there ? 16 : 0) : "memory");
    }
}

template <typename T, int kBlocksPerSm, int kM>
__global__ void __launch_bounds__(kTcThreads, kBlocksPerSm)
attention_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Params p)
{
    static_assert(kM == 64 || kM == 128, "rows of a product");
    constexpr int kWarpRows = kM / 4;                            // query rows of a softmax warp, in its first lanes
    constexpr unsigned int kCols = kBlocksPerSm == 2 ? 256 : 512;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bar_words[2 * kTcMaxSlots + 7];
    __shared__ unsigned int tmem_base_slot;
    __shared__ int give_up_flag, odd_run;
    volatile int *give_up = &give_up_flag;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const unsigned int rows_bytes = static_cast<unsigned int>(p.halves * p.tile_rows * 128);
    const unsigned int q_smem = (smem_u32(smem_raw) + 1023u) & ~1023u;              // one or two sets of query rows
    const unsigned int ring = q_smem + p.q_buffers * rows_bytes;
    const unsigned int slot_bytes = static_cast<unsigned int>(p.halves) * (kTcTile * 128);
    int *base = reinterpret_cast<int *>(smem_raw + (ring - smem_u32(smem_raw)) + p.n_stages * slot_bytes);      // [B + 1]
    const unsigned int bars = smem_u32(bar_words);
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (kTcMaxSlots + s); };
    auto s_full = [&](int k) { return bars + 8u * (2 * kTcMaxSlots + (k & 1)); };
    auto p_ready = [&](int k) { return bars + 8u * (2 * kTcMaxSlots + 2 + (k & 1)); };
    // (two, taken in turn: a wait by parity is sound while the barrier is in the phase waited for or the one after it, and the scores
    // of tile k, whose product is issued after the output product of tile k - 2, say that the barrier's phase before is over)
    auto pv_done = [&](int k) { return bars + 8u * (2 * kTcMaxSlots + 4 + (k & 1)); };
    const unsigned int q_ready = bars + 8u * (2 * kTcMaxSlots + 6);
    auto slot_at = [&](int s) { return ring + s * slot_bytes; };
    auto q_at = [&](int run) { return q_smem + (p.q_buffers == 2 ? run & 1 : 0) * rows_bytes; };

    if (tid == 0) {
        give_up_flag = 0;
        odd_run = 0;
        for (int s = 0; s < p.n_stages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int k = 0; k < 2; ++k) {
            mbar_init(s_full(k), 1);
            mbar_init(p_ready(k), 4);
            mbar_init(pv_done(k), 1);
        }
        mbar_init(q_ready, 4);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    }
    if (warp == 1) {
        ptx::tmem_alloc(smem_u32(&tmem_base_slot), kCols);
        ptx::tmem_relinquish();
    }
    ptx::wait_for_stream();
    if (tid == 0 && !p.by_unit) p.splits[blockIdx.x].parts = 0;
    for (int b = tid; b < p.B; b += kTcThreads) {
        const int len = row_len(p, b), news = row_news(p, b);
        base[b + 1] = news > 0 && len > 0 ? (len + kTcTile - 1) / kTcTile + p.run_cost : 0;
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    if (warp == 0) scan_tiles(base, p.B);
    __syncthreads();
    const unsigned int tmem = tmem_base_slot;
    const Share share(p, base);

    if (warp == 5) {
        // ---- page loads ----
        Runs runs;
        runs.begin(p, base, share.x0, share.x1);
        Run r, rn;
        bool ok = true;
        const int per_tile = kTcTile / p.box_rows;               // pages of a tile (1 where a page is larger)
        const unsigned int box_bytes = static_cast<unsigned int>(p.box_rows) * 128u;
        Cursor at = {0, 0u};
        auto load = [&](const CUtensorMap *map, int h, int j, int page) {
            const unsigned int there = __ballot_sync(kFull, page >= 0);
            int fine = 1;
            if (lane == 0) {
                fine = mbar_wait(empty(at.slot), at.round ^ 1u, give_up) ? 1 : 0;
                if (fine) mbar_expect_tx(full(at.slot), static_cast<unsigned int>(__popc(there)) * box_bytes * p.halves);
            }
            fine = __shfl_sync(kFull, fine, 0);
            if (fine && page >= 0) {
                const int in_page = p.box_rows == kTcTile ? (j * kTcTile) & ((1 << p.page_shift) - 1) : 0;
                const unsigned int to = slot_at(at.slot) + lane * box_bytes;
                for (int hf = 0; hf < p.halves; ++hf) tma_load_page(to + hf * (kTcTile * 128), map, full(at.slot), hf * 64, in_page, h, page);
            }
            at.next(p.n_stages);
            return fine != 0;
        };
        bool more = runs.next(r);
        int len = more ? row_len(p, r.b) : 0;
        int id = more ? tile_page<kTcTile>(p, r.b, r.j0, len, lane, per_tile) : -1;      // fetched a tile ahead
        while (more && ok) {
            const bool follows = runs.next(rn);
            const int len_next = follows ? row_len(p, rn.b) : 0;
            int before = -1;                                      // the page of the tile whose values are still to be loaded
            for (int i = 0; i < r.ns && ok; ++i) {
                const int page = id, j = r.j0 + i;
                const bool last = i + 1 == r.ns;
                id = !last ? tile_page<kTcTile>(p, r.b, j + 1, len, lane, per_tile)
                           : (follows ? tile_page<kTcTile>(p, rn.b, rn.j0, len_next, lane, per_tile) : -1);
                ok = load(&map_k, r.h, j, page);
                if (ok && i > 0) ok = load(&map_v, r.h, j - 1, before);
                if (ok && last) ok = load(&map_v, r.h, j, page);
                before = page;
            }
            if (lane == 0) note_split(p, share, r);
            r = rn;
            len = len_next;
            more = follows;
        }
        // every commit aimed at the slots' barriers has landed before the block ends
        if (lane == 0)
            for (int k = 0; k < p.n_stages && ok; ++k, at.next(p.n_stages)) ok = mbar_wait(empty(at.slot), at.round ^ 1u, give_up);
    } else if (warp == 4) {
        // ---- products ----
        if (lane == 0) {
            Runs runs;
            runs.begin(p, base, share.x0, share.x1);
            Run r;
            const unsigned int idesc_qk = tc_instr<T>(kM, kTcTile, false), idesc_pv = tc_instr<T>(kM, p.d16, true);
            const unsigned long long half_q = static_cast<unsigned long long>((p.tile_rows * 128) >> 4), half_k = (kTcTile * 128) >> 4;
            Cursor at = {0, 0u};                               // the loads are used in the order in which they are made
            int mine = 0;                                      // tiles of the runs before
            bool ok = true;
            for (int run = 0; ok && runs.next(r); ++run) {
                const int n = r.ns;
                const unsigned long long q_desc = ptx::operand_desc(q_at(run));
                ok = mbar_wait(q_ready, run & 1, give_up);
                for (int i = 0; i <= n && ok; ++i) {
                    if (i < n) {
                        const int k = mine + i;
                        if (!(ok = mbar_wait(full(at.slot), at.round, give_up))) break;
                        ptx::tc_fence_after();
                        const unsigned int d = tmem + (k & 1) * kTcScoreCols;
                        unsigned long long qd = q_desc, kd = ptx::operand_desc(slot_at(at.slot));
                        for (int left = p.d16; left > 0; left -= 64, qd += half_q, kd += half_k) {
                            tc_mma_ss(d, qd, kd, idesc_qk, left == p.d16 ? 0u : 1u);      // 16 elements further: 32 bytes
                            if (left > 16) tc_mma_ss(d, qd + 2, kd + 2, idesc_qk, 1u);
                            if (left > 32) tc_mma_ss(d, qd + 4, kd + 4, idesc_qk, 1u);
                            if (left > 48) tc_mma_ss(d, qd + 6, kd + 6, idesc_qk, 1u);
                        }
                        ptx::tc_commit(empty(at.slot));
                        ptx::tc_commit(s_full(k));
                        at.next(p.n_stages);
                    }
                    if (i > 0) {
                        const int k = mine + i - 1;
                        if (!(ok = mbar_wait(p_ready(k), (k >> 1) & 1, give_up))) break;
                        if (!(ok = mbar_wait(full(at.slot), at.round, give_up))) break;
                        ptx::tc_fence_after();
                        const unsigned int d = tmem + kTcOutCol, w = tmem + (k & 1) * kTcScoreCols;
                        const unsigned long long vd = value_desc(slot_at(at.slot), kTcTile * 128);
                        tc_mma_ts(d, w, vd, idesc_pv, i > 1 ? 1u : 0u);                  // 16 places further: 2 KiB
                        tc_mma_ts(d, w + 8, vd + 128, idesc_pv, 1u);
                        tc_mma_ts(d, w + 16, vd + 256, idesc_pv, 1u);
                        tc_mma_ts(d, w + 24, vd + 384, idesc_pv, 1u);
                        ptx::tc_commit(empty(at.slot));
                        ptx::tc_commit(pv_done(k));
                        at.next(p.n_stages);
                    }
                }
                mine += n;
            }
        }
    } else {
        // ---- softmax, rows in and out ----
        const int warp_row = kWarpRows * warp, r = lane < kWarpRows ? warp_row + lane : kM;      // the thread's query row of the row tile
        zero_empty_rows<T>(p, base, tid, 128);
        Runs runs;
        runs.begin(p, base, share.x0, share.x1);
        Run ru, next;
        bool more = runs.next(next);
        const unsigned int my_lanes = static_cast<unsigned int>(32 * warp) << 16, my_out = tmem + my_lanes + kTcOutCol;
        // query rows on their way; and: they are there, scores may be computed
        auto fetch = [&](const Run &x, int run) { fetch_rows<T>(p, x, q_at(run), warp, 4, lane); };
        auto fetched = [&]() {
            asm volatile("cp.async.wait_all;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(q_ready);
        };
        const bool ahead = p.q_buffers == 2;
        if (more && ahead) {
            fetch(next, 0);
            fetched();
        }
        int items = 0, mine = 0;                                    // loads of the runs before; tiles so far
        for (int run = 0; more; ++run) {
            ru = next;
            more = runs.next(next);
            const int b = ru.b, h = ru.h, rt = ru.rt, j0 = ru.j0, ns = ru.ns;
            const int len = row_len(p, b), news = row_news(p, b);
            const int rows_here = min(p.tile_rows, p.rows - rt * p.tile_rows);
            ptx::tc_fence_before();
            consumer_barrier(128);                                   // the accumulators and staged rows of the run before have been read
            ptx::tc_fence_after();
            if (!ahead) {
                fetch(ru, run);
                fetched();
            } else if (more) {
                fetch(next, run + 1);
            }
            const int rr = rt * p.tile_rows + r, tok = rr / p.group;
            const int limit = r < rows_here && tok < news ? len - news + tok : -1;
            const bool warp_has = warp_row < rows_here;
            float m = 0.f, l = 0.f;                              // l == 0: nothing seen yet, m is arbitrary

            for (int i = 0; i < ns; ++i, ++mine) {
                const int key0 = (j0 + i) * kTcTile;
                const bool edge = key0 + kTcTile - 1 > len - news;
                const unsigned int s_at = tmem + my_lanes + (mine & 1) * kTcScoreCols;
                mbar_wait(s_full(mine), (mine >> 1) & 1, give_up);
                ptx::tc_fence_after();
                float f = 1.f;                                   // on what has been accumulated
                if (warp_has) {
                    float x[32], y[32];
                    ptx::tmem_ld64(s_at, x, y);
                    const unsigned long long sc2 = pack2(p.scale_log2, p.scale_log2), m2 = pack2(-m, -m);
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        unpack2(fma2(pack2(x[j], x[j + 1]), sc2, m2), x[j], x[j + 1]);
                        unpack2(fma2(pack2(y[j], y[j + 1]), sc2, m2), y[j], y[j + 1]);
                    }
                    if (edge) {
                        const int left = limit - key0;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            if (j > left) x[j] = -INFINITY;
                            if (32 + j > left) y[j] = -INFINITY;
                        }
                    }
                    float mx = fmaxf(x[0], y[0]), my = fmaxf(x[1], y[1]);
#pragma unroll
                    for (int j = 2; j < 32; j += 2) {
                        mx = fmaxf(mx, fmaxf(x[j], y[j]));
                        my = fmaxf(my, fmaxf(x[j + 1], y[j + 1]));
                    }
                    mx = fmaxf(mx, my);
                    float up = 0.f;
                    if (limit >= 0) {
                        if (l == 0.f) {
                            up = mx == -INFINITY ? 0.f : mx - raised<T>(kLag);
                        } else if (mx > raised<T>(kLag) + kLag) {
                            up = mx - raised<T>(kLag);
                            f = ex2_approx(-up);
                        }
                    }
                    if (__any_sync(kFull, up != 0.f)) {
                        m += up;
                        l *= f;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            x[j] -= up;
                            y[j] -= up;
                        }
                    }
                    unsigned int w2[32];
                    unsigned long long sum0 = pack2(0.f, 0.f), sum1 = sum0;
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        const float a0 = ex2_approx(x[j]), a1 = ex2_approx(x[j + 1]), b0 = ex2_approx(y[j]), b1 = ex2_approx(y[j + 1]);
                        sum0 = add2(sum0, pack2(a0, a1));
                        sum1 = add2(sum1, pack2(b0, b1));
                        w2[j / 2] = pack_pair<T>(a0, a1);
                        w2[16 + j / 2] = pack_pair<T>(b0, b1);
                    }
                    float s0, s1;
                    unpack2(add2(sum0, sum1), s0, s1);
                    l += s0 + s1;
                    ptx::tmem_st32(s_at, w2);
                }
                if (warp_has) {
                    if (__any_sync(kFull, f != 1.f)) {
                        // the product before has to be complete; the next one waits for these weights
                        mbar_wait(pv_done(mine - 1), ((mine - 1) >> 1) & 1, give_up);
                        ptx::tc_fence_after();
                        for (int c0 = 0; c0 < p.d16; c0 += 32) {
                            float o[32];
                            unsigned int w2[32];
                            ptx::tmem_ld32(my_out + c0, o);
#pragma unroll
                            for (int j = 0; j < 32; ++j) w2[j] = __float_as_uint(o[j] * f);
                            ptx::tmem_st32(my_out + c0, w2);
                        }
                    }
                    ptx::tmem_wait_st();
                }
                if (edge) {
                    // A weight of zero does not silence an infinity or NaN in the values.  Places beyond the row hold anything:
                    // zeroed.  Such a value in a place of a later new token is left out here and handed to the rows that see it at the end.
                    // (The loads up to the tile's keys have been consumed: with four slots that includes this slot's load before.)
                    const int item = items + v_item(i, ns), s = item % p.n_stages;
                    mbar_wait(full(s), (item / p.n_stages) & 1, give_up);
                    const unsigned int v_at = slot_at(s);
                    const int from = max(len - news + 1 - key0, 0), chunks = p.halves * 8;
                    for (int c = tid; c < (kTcTile - from) * chunks; c += 128) {
                        const int kr = from + c / chunks, ch = c % chunks;
                        const unsigned int at = v_at + (ch >> 3) * (kTcTile * 128) + kr * 128 + (((ch & 7) ^ (kr & 7)) << 4);
                        unsigned int v[4] = {0u, 0u, 0u, 0u}, z[4] = {0u, 0u, 0u, 0u};
                        bool store = key0 + kr >= len;
                        if (!store) {
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                z[e] = finite_only<T>(v[e]);
                                store |= z[e] != v[e];
                            }
                            if (store) odd_run = run + 1;
                        }
                        if (store) asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(z[0]), "r"(z[1]), "r"(z[2]), "r"(z[3]) : "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_ready(mine));
            }
            if (ahead && more) fetched();

            // ---- the run's rows ----
            if (ns > 1) mbar_wait(pv_done(mine - 2), ((mine - 2) >> 1) & 1, give_up);
            mbar_wait(pv_done(mine - 1), ((mine - 1) >> 1) & 1, give_up);
            ptx::tc_fence_after();
            consumer_barrier(128);                                   // odd_run of all four warps
            const bool odd = *static_cast<volatile int *>(&odd_run) == run + 1;
            const bool whole = ns == ru.n;
            const bool seen = limit >= 0 && l != 0.f;                // (NaN counts as seen)
            const int head = h * p.group + rr - tok * p.group;
            const long long row = (static_cast<long long>(b) * p.T + tok) * p.Hq + head;
            float *part = p.parts + static_cast<long long>(2 * static_cast<int>(blockIdx.x) + (j0 == 0 ? 1 : 0)) * p.tile_rows * (p.part_stride + 2);
            if (warp_has) {
                // A thread has a row, memory wants rows side by side: each warp turns its 32 rows round in shared memory, where the
                // run's query rows were, which every product has read.
                const float inv = seen ? (whole ? 1.f / l : 1.f) : 0.f;
                const int pitch = p.halves * 128, warp_rows = min(kWarpRows, rows_here - warp_row);
                const unsigned int out_smem = q_at(run), my_row = out_smem + r * pitch;
                const int cols = whole ? p.halves * 64 : p.halves * 32;                        // of a pass: what a staged row holds
                const int lanes_row = p.halves * 8, at_once = 32 / lanes_row, sub = lane / lanes_row, ch = lane - sub * lanes_row;
                for (int pass0 = 0; pass0 < p.D; pass0 += cols) {
                    const int pass1 = min(pass0 + cols, p.D);
                    for (int c0 = pass0; c0 < pass1; c0 += 32) {
                        float o[32];
                        ptx::tmem_ld32(my_out + c0, o);
                        if (odd && seen) {
                            float z[32];
#pragma unroll
                            for (int e = 0; e < 32; ++e) z[e] = o[e];
                            add_left_out<T>(p, b, h, tok, head, c0, max(len - news + 1, j0 * kTcTile), min(limit, (j0 + ns) * kTcTile - 1), m, z);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = z[e];
                        }
                        if (r < rows_here) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = seen ? o[e] * inv : 0.f;
                            if (whole) {
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(my_row + ((((c0 - pass0) / 8 + e) ^ (r & 7)) << 4)),
                                                 "r"(pack_pair<T>(o[8 * e], o[8 * e + 1])), "r"(pack_pair<T>(o[8 * e + 2], o[8 * e + 3])),
                                                 "r"(pack_pair<T>(o[8 * e + 4], o[8 * e + 5])), "r"(pack_pair<T>(o[8 * e + 6], o[8 * e + 7]))
                                                 : "memory");
                            } else {
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(my_row + ((((c0 - pass0) / 4 + e) ^ (r & 7)) << 4)),
                                                 "f"(o[4 * e]), "f"(o[4 * e + 1]), "f"(o[4 * e + 2]), "f"(o[4 * e + 3])
                                                 : "memory");
                            }
                        }
                    }
                    __syncwarp();
                    // lanes_row lanes a row, 16 bytes each
                    const int d = pass0 + (whole ? ch * 8 : ch * 4);
                    const bool do_it = sub < at_once && d < pass1;
                    char *to = whole ? reinterpret_cast<char *>(static_cast<T *>(p.out) + d) : reinterpret_cast<char *>(part + warp_row * p.part_stride + d);
                    const long long row_bytes = whole ? row * p.D * static_cast<long long>(sizeof(T)) : static_cast<long long>(lane) * p.part_stride * 4;
                    for (int w0 = 0; w0 < warp_rows; w0 += 4 * at_once) {
                        uint4 v[4];
                        long long off[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int wr = w0 + k * at_once + sub, r2 = warp_row + wr;
                            off[k] = __shfl_sync(kFull, row_bytes, wr & 31);
                            if (do_it && wr < warp_rows)
                                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[k].x), "=r"(v[k].y), "=r"(v[k].z), "=r"(v[k].w) : "r"(out_smem + r2 * pitch + ((ch ^ (r2 & 7)) << 4)) : "memory");
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (do_it && w0 + k * at_once + sub < warp_rows) __stcg(reinterpret_cast<uint4 *>(to + off[k]), v[k]);
                    }
                    __syncwarp();
                }
                if (r < rows_here) {
                    if (!whole)
                        __stcg(reinterpret_cast<float2 *>(part + static_cast<long long>(p.tile_rows) * p.part_stride + 2 * r), make_float2(seen ? m : -INFINITY, seen ? l : 0.f));
                    else if (p.lse)
                        p.lse[row] = seen ? (m + log2f(l)) * kLn2 : -INFINITY;
                }
            }
            items += 2 * ns;
        }
        ptx::tc_fence_before();
    }
    __syncthreads();
    if (*give_up) {                                                  // a wait ran out
        if (lane == 0) atomicOr(p.flags, CSD_CACHE_INTERNAL);
        ptx::linger();
        __syncthreads();
    }
    if (warp == 1) ptx::tmem_dealloc(tmem, kCols);
}

// Joins the parts of split units: block (x, y) kJoinRows query rows of one of them.  The weights of all parts and rows first (a
// thread per part and row), then each warp sums every fourth part, the rows side by side, so that a row of 40 parts costs a
// few memory latencies and not forty; the four sums are added in order.  Four rows to a block, or one where units have many parts.
constexpr int kJoinThreads = 128, kMaxGrid = 512;

template <typename T, int DP, int kJoinRows>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const Params p, int tile_rows)
{
    __shared__ float2 part_ml[kMaxGrid][kJoinRows];                     // (m, l), then (weight, l)
    __shared__ float red[4][kJoinRows], sums[4][kJoinRows];
    __shared__ __align__(16) float rows[4][kJoinRows][DP];
    ptx::wait_for_stream();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Split sp = {ptx::ld_written(&p.splits[blockIdx.x].unit), ptx::ld_written(&p.splits[blockIdx.x].first), ptx::ld_written(&p.splits[blockIdx.x].parts)};
    const int n = sp.parts;
    if (n == 0) return;
    const int rt = sp.unit % p.row_tiles, bh = sp.unit / p.row_tiles, b = bh / p.Hkv, h = bh - b * p.Hkv;
    const int r0 = blockIdx.y * kJoinRows, here = min(kJoinRows, min(tile_rows, p.rows - rt * tile_rows) - r0);
    if (here <= 0) return;
    const long long slot_floats = static_cast<long long>(tile_rows) * (DP + 2);
    auto slot = [&](int i) { return p.parts + slot_floats * (i == 0 ? 2 * sp.first + 1 : 2 * (sp.first + i)); };
    const int row = tid % kJoinRows;
    float M = -INFINITY, L = 0.f;
    for (int i = tid / kJoinRows; i < n; i += kJoinThreads / kJoinRows) {
        const float2 ml = row < here ? __ldcg(reinterpret_cast<const float2 *>(slot(i) + tile_rows * DP + 2 * (r0 + row))) : make_float2(-INFINITY, 0.f);
        part_ml[i][row] = ml;
        M = fmaxf(M, ml.x);
    }
#pragma unroll
    for (int d = kJoinRows; d < 32; d <<= 1) M = fmaxf(M, __shfl_xor_sync(kFull, M, d));
    if (lane < kJoinRows) red[warp][row] = M;
    __syncthreads();
    M = fmaxf(fmaxf(red[0][row], red[1][row]), fmaxf(red[2][row], red[3][row]));
    for (int i = tid / kJoinRows; i < n; i += kJoinThreads / kJoinRows) {
        const float2 ml = part_ml[i][row];
        const float w = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - M);
        part_ml[i][row].x = w;
        L += w * ml.y;
    }
#pragma unroll
    for (int d = kJoinRows; d < 32; d <<= 1) L += __shfl_xor_sync(kFull, L, d);
    if (lane < kJoinRows) sums[warp][row] = L;
    __syncthreads();
    constexpr int E = DP / 32;                                          // columns of a lane: 2, 4 or 8, side by side
    float o[kJoinRows][E];
#pragma unroll
    for (int k = 0; k < kJoinRows; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) o[k][e] = 0.f;
    const bool mine = lane * E < p.D;
#pragma unroll (kJoinRows == 1 ? 8 : 4)
    for (int i = warp; i < n; i += 4) {
        const float *from = slot(i) + r0 * DP + lane * E;
#pragma unroll
        for (int k = 0; k < kJoinRows; ++k) {
            if (k < here && mine) {
                const float w = part_ml[i][k].x;
                if constexpr (E == 2) {
                    const float2 y = __ldcg(reinterpret_cast<const float2 *>(from + k * DP));
                    o[k][0] += w * y.x;
                    o[k][1] += w * y.y;
                } else {
#pragma unroll
                    for (int e = 0; e < E; e += 4) {
                        const float4 y = __ldcg(reinterpret_cast<const float4 *>(from + k * DP + e));
                        o[k][e] += w * y.x;
                        o[k][e + 1] += w * y.y;
                        o[k][e + 2] += w * y.z;
                        o[k][e + 3] += w * y.w;
                    }
                }
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kJoinRows; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) rows[warp][k][lane * E + e] = o[k][e];
    __syncthreads();
    if (warp >= here) return;
    // warp k finishes row k
    L = (sums[0][warp] + sums[1][warp]) + (sums[2][warp] + sums[3][warp]);
    const int rr = rt * tile_rows + r0 + warp, tok = rr / p.group, head = h * p.group + rr - tok * p.group;
    const long long to = (static_cast<long long>(b) * p.T + tok) * p.Hq + head;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    unsigned int *out = reinterpret_cast<unsigned int *>(static_cast<T *>(p.out) + to * p.D);
    for (int d = 2 * lane; d < p.D; d += 64) {
        float2 y = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            y.x += rows[w][warp][d];
            y.y += rows[w][warp][d + 1];
        }
        out[d / 2] = pack_pair<T>(y.x * inv, y.y * inv);
    }
    if (p.lse && lane == 0) {
        const float m = fmaxf(fmaxf(red[0][warp], red[1][warp]), fmaxf(red[2][warp], red[3][warp]));
        p.lse[to] = L == 0.f ? -INFINITY : (fmaxf(m, -3e38f) + log2f(L)) * kLn2;
    }
}

}  // namespace attention
}  // namespace csd
