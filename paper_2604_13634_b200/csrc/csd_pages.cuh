// The pages of a key-value cache: which page holds which tokens of which row, kept on the device beside the pool.
//
//   table[row, i]  page of the row's tokens i * page_size ..; -1 where the row has none
//   lens[row]      tokens in the row;  ceil(lens / page_size) entries of the table are in use
//   refs[page]     rows that use the page (0: free)
//   free_bits      bit p set: page p is free (the same fact as refs[p] == 0, kept packed so that a block can scan it)
//
// Every result is a function of the state and the arguments alone, not of the order in which atomics land: pages are
// handed out lowest id first, to rows in index order; a page becomes free when its count is zero after ALL decrements
// of a call; counts only meet commutative adds.  Nothing here synchronises, so the accepted lengths of a verification
// step drive it without leaving the device.
//
// Bounds: the bookkeeping kernels are latency (a few dependent reads and one block-wide scan); pages_copy_kernel,
// which moves page contents over all layers, is memory.  Fork, extension and truncation of 64 rows with 48 page copies over 16 layers
// take 23.1 us, of which the copies' 101 MB need 15.4.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/csd.h"
#include "csd_common.cuh"
#include "csd_ptx.cuh"

namespace csd {
namespace pages {

constexpr int kBlock = 1024;           // the bookkeeping block
constexpr int kMaxRows = 4096;
constexpr int kRowThreads = 256;       // of the kernels with a block per row
constexpr int kCopyThreads = 256;
constexpr int kCopyBytes = 32 * 16 * 8;   // what a warp moves at a time: eight 16-byte vectors per lane

struct View {
    int rows, max_pages, n_pages, page_size, page_shift, words;
    int *table, *lens, *granted, *refs;
    unsigned int *free_bits;
    unsigned int *flags;
    int *n_moves;                      // page copies wanted by the call before pages_copy_kernel
    int *moves;                        // [2 n_moves]: source, destination   (scratch)
    int *list;                         // [n_pages]: free pages handed out; or where a page went   (scratch)
    int *staged;                       // [rows, max_pages + 1]: tables and lengths of a fork   (scratch)
};

__device__ __forceinline__ int pages_of(int tokens, int shift) { return static_cast<int>((static_cast<unsigned int>(tokens) + ((1u << shift) - 1u)) >> shift); }

// Exclusive scan over a block of 1024 threads; `total` is the sum.  Two barriers; `slots` holds 33 words.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long *slots, unsigned long long &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long inc = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long o = __shfl_up_sync(kFull, inc, d);
        if (lane >= d) inc += o;
    }
    __syncthreads();                   // the slots of a scan before this one have been read
    if (lane == 31) slots[warp] = inc;
    __syncthreads();
    const unsigned long long w = slots[lane];
    unsigned long long winc = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long o = __shfl_up_sync(kFull, winc, d);
        if (lane >= d) winc += o;
    }
    total = __shfl_sync(kFull, winc, 31);
    return __shfl_sync(kFull, winc - w, warp) + inc - v;
}

// Room for n_new[row] more tokens (or `uniform` for every row).  All rows or none: if the free pages do not suffice,
// or a row would need more than max_pages, nothing changes, granted is 0 and a flag says so.
//   need(row) = ceil((len + n) / page) - ceil(len / page) + copied(row)
//   copied(row): the last page is partly filled and still shared at the row's turn, i.e. refs - (rows before it that
//   take a copy of the same page) > 1; the last of them keeps the page.
__global__ void __launch_bounds__(kBlock, 1) extend_kernel(const View v, const int *n_new, int uniform)
{
    constexpr int kRowsEach = kMaxRows / kBlock;     // rows of a thread: consecutive, so that scans follow the rows
    constexpr int kListed = 4096;                    // pages handed out that stay in shared memory; a longer list goes to scratch
    __shared__ __align__(16) int tail[kMaxRows];     // the shared last page a row would have to copy, or -1; later: its first page in the list
    __shared__ unsigned long long slots[32];
    __shared__ int short_list[kListed];
    __shared__ int bad;
    ptx::wait_for_stream();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (v.rows + kBlock - 1) / kBlock, r0 = tid * per;
    // everything that is needed and does not depend on anything, at once
    const unsigned int first_bits = tid < v.words ? v.free_bits[tid] : 0u;
    int len[kRowsEach], n[kRowsEach], page[kRowsEach];
#pragma unroll
    for (int k = 0; k < kRowsEach; ++k) {
        const bool there = k < per && r0 + k < v.rows;
        len[k] = there ? v.lens[r0 + k] : 0;
        n[k] = there ? max(n_new ? ptx::ld_written(n_new + r0 + k) : uniform, 0) : 0;
    }
    if (tid == 0) bad = 0;
    for (int r = tid; r < ((v.rows + 3) & ~3); r += kBlock) tail[r] = -1;
    __syncthreads();
    unsigned int complaint = 0;
#pragma unroll
    for (int k = 0; k < kRowsEach; ++k) {
        page[k] = -1;
        if (n[k] == 0) continue;
        if (static_cast<long long>(len[k]) + n[k] > (static_cast<long long>(v.max_pages) << v.page_shift))
            complaint |= CSD_CACHE_ROW_FULL;
        else if (len[k] & (v.page_size - 1))
            page[k] = v.table[static_cast<long long>(r0 + k) * v.max_pages + (len[k] >> v.page_shift)];
    }
    int users[kRowsEach];
#pragma unroll
    for (int k = 0; k < kRowsEach; ++k) {
        users[k] = 0;
        if (n[k] == 0 || !(len[k] & (v.page_size - 1)) || (complaint & CSD_CACHE_ROW_FULL)) continue;
        if (page[k] < 0 || page[k] >= v.n_pages) {
            complaint |= CSD_CACHE_BAD_PAGE;
            continue;
        }
        users[k] = v.refs[page[k]];
        if (users[k] > 1) tail[r0 + k] = page[k];
    }
    if (complaint) {
        atomicOr(v.flags, complaint);
        bad = 1;
    }
    __syncthreads();
    const bool refuse_shape = bad != 0;
    unsigned long long mine = 0;                     // pages wanted | page copies << 32
    int need[kRowsEach];
    unsigned int copied = 0;                         // bit k: row r0 + k copies
#pragma unroll
    for (int k = 0; k < kRowsEach; ++k) {
        need[k] = 0;
        if (n[k] == 0 || refuse_shape) continue;
        const int r = r0 + k;
        need[k] = pages_of(len[k] + n[k], v.page_shift) - pages_of(len[k], v.page_shift);
        if (users[k] > 1) {                          // how many rows before it have the same last page
            int before = 0;
            const int4 *t4 = reinterpret_cast<const int4 *>(tail);
            for (int j = 0; j < (r >> 2); ++j) {
                const int4 q = t4[j];
                before += (q.x == page[k]) + (q.y == page[k]) + (q.z == page[k]) + (q.w == page[k]);
            }
            for (int j = r & ~3; j < r; ++j) before += tail[j] == page[k];
            if (users[k] - before > 1) {
                copied |= 1u << k;
                mine += 1ull + (1ull << 32);
            }
        }
        mine += static_cast<unsigned int>(need[k]);
    }
    unsigned long long total2;
    const unsigned long long first2 = block_scan(mine, slots, total2);
    const int total = static_cast<int>(total2 & 0xffffffffu), total_moves = static_cast<int>(total2 >> 32);
    int *list = total <= kListed ? short_list : v.list;
    // the `total` lowest free pages, in order
    int found = 0;
    for (int w0 = 0; w0 < v.words && found < total; w0 += kBlock) {
        const int w = w0 + tid;
        unsigned int bits = w0 == 0 ? first_bits : (w < v.words ? v.free_bits[w] : 0u);
        unsigned long long sum;
        int at = found + static_cast<int>(block_scan(static_cast<unsigned long long>(__popc(bits)), slots, sum));
        while (bits && at < total) {
            list[at++] = w * 32 + __ffs(bits) - 1;
            bits &= bits - 1;
        }
        found += static_cast<int>(sum);
    }
    const bool refuse = refuse_shape || found < total;
    __syncthreads();                                 // the list is complete; tail has been read
    if (refuse) {
        if (tid == 0) {
            if (!refuse_shape) atomicOr(v.flags, CSD_CACHE_FULL);
            *v.n_moves = 0;
        }
        for (int r = tid; r < v.rows; r += kBlock) v.granted[r] = 0;
        return;
    }
    {
        int at = static_cast<int>(first2 & 0xffffffffu), mv = static_cast<int>(first2 >> 32);
#pragma unroll
        for (int k = 0; k < kRowsEach; ++k) {
            if (k >= per || r0 + k >= v.rows) continue;
            const int r = r0 + k;
            if ((copied >> k) & 1u) {
                const int dst = list[at++];
                v.moves[2 * mv] = page[k];
                v.moves[2 * mv + 1] = dst;
                ++mv;
                v.table[static_cast<long long>(r) * v.max_pages + (len[k] >> v.page_shift)] = dst;
                atomicSub(v.refs + page[k], 1);
            }
            v.lens[r] = len[k] + n[k];
            v.granted[r] = n[k];
            tail[r] = at;
            at += need[k];
            // a few new pages: here; more: a warp per row, below
            if (need[k] <= 2)
                for (int j = 0; j < need[k]; ++j) v.table[static_cast<long long>(r) * v.max_pages + pages_of(len[k], v.page_shift) + j] = list[at - need[k] + j];
        }
    }
    if (tid == 0) *v.n_moves = total_moves;
    for (int j = tid; j < total; j += kBlock) {
        const int p = list[j];
        v.refs[p] = 1;
        atomicAnd(v.free_bits + (p >> 5), ~(1u << (p & 31)));
    }
    bool many = false;
#pragma unroll
    for (int k = 0; k < kRowsEach; ++k) many |= need[k] > 2;
    if (__syncthreads_or(many ? 1 : 0) == 0) return;
    for (int r = warp; r < v.rows; r += kBlock / 32) {
        const int more_to = v.granted[r], now = v.lens[r], held = pages_of(now - more_to, v.page_shift), more = pages_of(now, v.page_shift) - held;
        if (more <= 2) continue;
        for (int j = lane; j < more; j += 32) v.table[static_cast<long long>(r) * v.max_pages + held + j] = list[tail[r] + j];
    }
}

__device__ __forceinline__ void release(const View &v, int page)
{
    if (page < 0 || page >= v.n_pages) {
        atomicOr(v.flags, CSD_CACHE_BAD_PAGE);
        return;
    }
    if (atomicSub(v.refs + page, 1) == 1) atomicOr(v.free_bits + (page >> 5), 1u << (page & 31));
}

// A row of len tokens keeps `to` of them.  All threads of a block.
__device__ __forceinline__ void shorten(const View &v, int r, int len, int to, int threads = kRowThreads)
{
    const int first = pages_of(to, v.page_shift), held = pages_of(len, v.page_shift);
    int *row = v.table + static_cast<long long>(r) * v.max_pages;
    for (int i = first + threadIdx.x; i < held; i += threads) {
        release(v, row[i]);
        row[i] = -1;
    }
    __syncthreads();                                 // every thread has read the row's length and grant
    if (threadIdx.x == 0) {
        v.lens[r] = to;
        v.granted[r] = 0;
    }
}

// Rows become shorter: to new_lens[row], or (commit) by the tokens of the last extension that the verification did
// not keep: granted - min(granted, accept_len + 1).  A row never grows here.
__global__ void __launch_bounds__(kRowThreads) truncate_kernel(const View v, const int *new_lens, const int *accept_len)
{
    ptx::wait_for_stream();
    const int r = blockIdx.x;
    const int len = v.lens[r];
    int to;
    if (accept_len) {
        // (bounded before one is added: any accepted count will do, 2^31 - 1 for "all" among them)
        const int n = v.granted[r], kept = min(max(ptx::ld_written(accept_len + r), -1), n - 1) + 1;
        to = len - (n - kept);
    } else {
        to = ptx::ld_written(new_lens + r);
    }
    shorten(v, r, len, min(max(to, 0), len));
}

// Rows continue other rows' pages.  First launch: stage the new tables and count the new references; second launch,
// after all of them: drop the old ones and put the staged tables in place.  Entries that stay the same are left alone.
__global__ void __launch_bounds__(kRowThreads) fork_stage_kernel(const View v, const int *parent)
{
    ptx::wait_for_stream();
    const int r = blockIdx.x;
    int p = ptx::ld_written(parent + r);
    if (p >= v.rows) {
        if (threadIdx.x == 0) atomicOr(v.flags, CSD_CACHE_BAD_ROW);
        p = r;
    }
    const int len = p >= 0 ? v.lens[p] : 0;
    int *to = v.staged + static_cast<long long>(r) * (v.max_pages + 1);
    if (threadIdx.x == 0) to[v.max_pages] = len;
    if (p == r) return;
    const int *from = v.table + static_cast<long long>(p < 0 ? 0 : p) * v.max_pages, *own = v.table + static_cast<long long>(r) * v.max_pages;
    const int held = pages_of(len, v.page_shift), own_held = pages_of(v.lens[r], v.page_shift);
    for (int i = threadIdx.x; i < held; i += kRowThreads) {
        const int page = from[i];
        to[i] = page;
        if (page < 0 || page >= v.n_pages)
            atomicOr(v.flags, CSD_CACHE_BAD_PAGE);
        else if (i >= own_held || own[i] != page)
            atomicAdd(v.refs + page, 1);
    }
}

__global__ void __launch_bounds__(kRowThreads) fork_commit_kernel(const View v, const int *parent)
{
    ptx::wait_for_stream();
    const int r = blockIdx.x;
    const int p = ptx::ld_written(parent + r);
    const int *to = v.staged + static_cast<long long>(r) * (v.max_pages + 1);
    if (p != r && p < v.rows) {
        int *own = v.table + static_cast<long long>(r) * v.max_pages;
        const int len = to[v.max_pages];
        const int held = pages_of(len, v.page_shift), own_held = pages_of(v.lens[r], v.page_shift);
        for (int i = threadIdx.x; i < max(held, own_held); i += kRowThreads) {
            const int old = i < own_held ? own[i] : -1, now = i < held ? to[i] : -1;
            if (old == now) continue;
            if (i < own_held) release(v, old);
            own[i] = now;
        }
        __syncthreads();                             // every thread has read the row's old length
        if (threadIdx.x == 0) v.lens[r] = len;
    }
    if (threadIdx.x == 0) v.granted[r] = 0;
}

// With n_live pages in use: the i-th lowest page in use at or above n_live moves to the i-th lowest free page below.
__global__ void __launch_bounds__(kBlock, 1) compact_kernel(const View v)
{
    ptx::wait_for_stream();
    __shared__ unsigned long long slots[32];
    const int tid = threadIdx.x;
    unsigned long long mine = 0, n_free;
    for (int w = tid; w < v.words; w += kBlock) mine += static_cast<unsigned int>(__popc(v.free_bits[w]));
    block_scan(mine, slots, n_free);
    const int n_live = v.n_pages - static_cast<int>(n_free);
    int holes = 0, high = 0;                         // found so far
    for (int w0 = 0; w0 < v.words; w0 += kBlock) {
        const int w = w0 + tid;
        unsigned int lo = 0, hi = 0;                 // free pages below n_live; pages in use from n_live on
        if (w < v.words) {
            const unsigned int bits = v.free_bits[w];
            const int there = min(32, v.n_pages - 32 * w);
            const unsigned int real = there >= 32 ? 0xffffffffu : (1u << there) - 1u;
            const int below = min(max(n_live - 32 * w, 0), 32);
            const unsigned int under = below >= 32 ? 0xffffffffu : (1u << below) - 1u;
            lo = bits & real & under;
            hi = ~bits & real & ~under;
        }
        unsigned long long sum;
        const unsigned long long at = block_scan(static_cast<unsigned long long>(__popc(lo)) | static_cast<unsigned long long>(__popc(hi)) << 32, slots, sum);
        int a = holes + static_cast<int>(at & 0xffffffffu), b = high + static_cast<int>(at >> 32);
        for (; lo; lo &= lo - 1) v.moves[2 * a++ + 1] = w * 32 + __ffs(lo) - 1;
        for (; hi; hi &= hi - 1) v.moves[2 * b++] = w * 32 + __ffs(hi) - 1;
        holes += static_cast<int>(sum & 0xffffffffu);
        high += static_cast<int>(sum >> 32);
    }
    const int n = min(holes, high);                  // the two are the same number
    __syncthreads();
    for (int j = tid; j < n; j += kBlock) {
        const int src = v.moves[2 * j], dst = v.moves[2 * j + 1];
        v.list[src] = dst;
        v.refs[dst] = v.refs[src];
        v.refs[src] = 0;
    }
    for (int w = tid; w < v.words; w += kBlock) {
        const int there = min(32, v.n_pages - 32 * w), below = min(max(n_live - 32 * w, 0), 32);
        const unsigned int real = there >= 32 ? 0xffffffffu : (1u << there) - 1u;
        v.free_bits[w] = real & ~(below >= 32 ? 0xffffffffu : (1u << below) - 1u);
    }
    if (tid == 0) *v.n_moves = n;
    // how many pages are in use, for the launch that renames them in the tables
    if (tid == 0) v.moves[2 * n] = n_live;
}

// Tables after a compaction: pages from n_live on have moved.
__global__ void __launch_bounds__(kRowThreads) rename_kernel(const View v)
{
    ptx::wait_for_stream();
    const int r = blockIdx.x;
    const int n_live = v.moves[2 * *v.n_moves];
    const int held = pages_of(v.lens[r], v.page_shift);
    int *row = v.table + static_cast<long long>(r) * v.max_pages;
    for (int i = threadIdx.x; i < held; i += kRowThreads) {
        const int page = row[i];
        if (page >= n_live && page < v.n_pages) row[i] = v.list[page];
    }
}

// Counts and free bits from tables and lengths.  Entries beyond a row's length become -1.
__global__ void __launch_bounds__(kRowThreads) rebuild_count_kernel(const View v)
{
    ptx::wait_for_stream();
    const int r = blockIdx.x;
    int len = v.lens[r];
    if (len < 0 || len > static_cast<long long>(v.max_pages) << v.page_shift) {
        if (threadIdx.x == 0) atomicOr(v.flags, CSD_CACHE_ROW_FULL);
        len = len < 0 ? 0 : v.max_pages << v.page_shift;
    }
    int *row = v.table + static_cast<long long>(r) * v.max_pages;
    const int held = pages_of(len, v.page_shift);
    for (int i = threadIdx.x; i < v.max_pages; i += kRowThreads) {
        if (i >= held) {
            row[i] = -1;
        } else if (row[i] < 0 || row[i] >= v.n_pages) {
            atomicOr(v.flags, CSD_CACHE_BAD_PAGE);
        } else {
            atomicAdd(v.refs + row[i], 1);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        v.lens[r] = len;
        v.granted[r] = 0;
    }
}

__global__ void __launch_bounds__(kRowThreads) rebuild_bits_kernel(const View v)
{
    ptx::wait_for_stream();
    const int p = blockIdx.x * kRowThreads + threadIdx.x;
    const unsigned int bits = __ballot_sync(kFull, p < v.n_pages && v.refs[p] == 0);
    if ((threadIdx.x & 31) == 0 && p / 32 < v.words) v.free_bits[p / 32] = bits;
}

struct CopyParams {
    char *k, *v;
    long long layer_bytes, page_stride_bytes;
    int page_bytes, layers, pieces;                  // pieces of kCopyBytes in a page
    const int *n_moves, *moves;
};

// Page contents: grid.y is a layer's keys or values.  A warp moves up to 4 KiB at a time, eight 16-byte loads in flight per
// lane, neighbouring warps neighbouring pieces of a page.  2.6 GB (2500 pages of 32 KB in 16 planes, read and written): 412 to 420 us, 6.2
// to 6.4 TB/s, of the 430 to 445 us of the compaction that asked for them.
__global__ void __launch_bounds__(kCopyThreads) pages_copy_kernel(const CopyParams p)
{
    ptx::wait_for_stream();
    const int lane = threadIdx.x & 31;
    const int n = *p.n_moves * p.pieces;             // (the host has seen to it that this fits)
    char *pool = ((blockIdx.y & 1) ? p.v : p.k) + static_cast<long long>(blockIdx.y >> 1) * p.layer_bytes + lane * 16;
    const int warps = gridDim.x * (kCopyThreads / 32);
    for (int it = blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); it < n; it += warps) {
        const int move = it / p.pieces, piece = it - move * p.pieces;
        const int2 m = ptx::ld_written(reinterpret_cast<const int2 *>(p.moves) + move);
        char *base = pool + static_cast<long long>(piece) * kCopyBytes;
        const char *from = base + m.x * p.page_stride_bytes;
        char *to = base + m.y * p.page_stride_bytes;
        const int left = p.page_bytes - piece * kCopyBytes - lane * 16;
        uint4 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 512 < left) x[j] = ptx::ld_written_once(from + j * 512);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 512 < left) __stcs(reinterpret_cast<uint4 *>(to + j * 512), x[j]);
    }
}

}  // namespace pages
}  // namespace csd
