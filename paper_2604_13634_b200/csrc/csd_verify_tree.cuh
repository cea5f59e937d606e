// The verification loop of Algorithm 1 (greedy) on a tree of drafted tokens.
//
//   c = 0; repeat: t* = argmax z[c]; c' = a child of c with token t* (lowest index), else the child d that memory and gate let through
//   (T[(d, t*)] >= lambda, z[c,d] - z[c,t*] >= ln tau) with the largest z[c,d] (lowest index on ties); until there is none
//
// Only the logit rows of the nodes that the walk visits are read: (accepted + 1) V elements of a batch row, where a pass over all nodes
// would read T V.  The price is a chain of dependent passes, one per accepted token.  A thread-block cluster has a batch row: every block
// reduces its share of the node's logits to (max, lowest index), hands it to all others through distributed shared memory (once all are
// known to run: they meet as the kernel begins), and after one cluster barrier each of them knows t* and, where a child has that token, the next node.  Where none has, the first block alone asks the
// memory (another stream may be updating it: two answers could differ) and a second barrier spreads what it decided.  All blocks of a
// cluster take the same branches, so they meet at the same barriers, which the hardware schedules together and which always end.
//
// Bound: that chain.  48 rows of up to 40 nodes over 151936 bf16 logits, at most 8 of them visited in a row: 36 to 37 us (137 rows, 42 MB; all
// 983 rows would be 299 MB, 46 us at the copy rate), 4 us a node with memory look-ups at every second; 11.4 to 12.1 us for one row and three
// nodes of 128256.  48 rows are 384 blocks of which 296 run at a time, so that some rows begin when others have ended.
// Sending for the rows of two children while a node's are reduced: 41 us.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/csd.h"
#include "csd_common.cuh"
#include "csd_ocm.cuh"
#include "csd_ptx.cuh"

namespace csd {
namespace verify_tree {

using ptx::cluster_meet;
using ptx::in_block;
using ptx::st_cluster;

constexpr int kThreads = 512, kWarps = kThreads / 32, kMaxCluster = 8, kNodes = CSD_TREE_MAX_NODES;
constexpr int kAtOnce = 8;                 // 16-byte loads in flight per thread: all of a row of 262144 bf16 logits, shared by eight blocks

struct Params {
    const void *logits;
    int T, V;
    long long stride_b, stride_t, parent_stride;
    const int *tokens, *parents, *n_nodes;
    OcmView ocm;
    float log_tau;
    int *accept_len, *next_token, *path;
    unsigned char *rescued;
    int *rej_d, *rej_t;
};

// A maximum as an unsigned number in the same order, and the lowest index that has it; `odd`: a NaN was seen.
struct Best {
    unsigned int key;
    int index, odd;
};
__device__ __forceinline__ unsigned int ordered(float x)
{
    const unsigned int u = __float_as_uint(x + 0.0f);                 // (one zero)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(unsigned int k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ Best warp_best(const Best &x)
{
    Best r;
    r.key = __reduce_max_sync(kFull, x.key);
    r.index = __reduce_min_sync(kFull, x.key == r.key ? x.index : 0x7fffffff);
    r.odd = __any_sync(kFull, x.odd) ? 1 : 0;
    return r;
}

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
template <typename T>
struct Lane;                               // a 16-byte vector of logits
template <>
struct Lane<float> {
    static constexpr int kN = 4;
    static __device__ __forceinline__ float largest(const uint4 &v)
    {
        return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)), max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    static __device__ __forceinline__ float one(const float *p) { return __uint_as_float(static_cast<unsigned int>(ptx::ld_written(reinterpret_cast<const int *>(p)))); }
    static __device__ __forceinline__ int first(const uint4 &v, float m)
    {
        return __uint_as_float(v.x) == m ? 0 : (__uint_as_float(v.y) == m ? 1 : (__uint_as_float(v.z) == m ? 2 : 3));
    }
};
template <>
struct Lane<__nv_bfloat16> {
    static constexpr int kN = 8;
    static __device__ __forceinline__ float lo(unsigned int w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float hi(unsigned int w) { return __uint_as_float(w & 0xffff0000u); }
    static __device__ __forceinline__ unsigned int max2(unsigned int a, unsigned int b)
    {
        unsigned int r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ float largest(const uint4 &v)
    {
        const unsigned int w = max2(max2(v.x, v.y), max2(v.z, v.w));
        return max_nan(lo(w), hi(w));
    }
    static __device__ __forceinline__ float one(const __nv_bfloat16 *p)
    {
        unsigned short u;
        asm volatile("ld.global.u16 %0, [%1];" : "=h"(u) : "l"(p));
        return __uint_as_float(static_cast<unsigned int>(u) << 16);
    }
    static __device__ __forceinline__ int first(const uint4 &v, float m)
    {
        const unsigned int w[4] = {v.x, v.y, v.z, v.w};
        int at = 7;
#pragma unroll
        for (int j = 3; j >= 0; --j) {
            if (hi(w[j]) == m) at = 2 * j + 1;
            if (lo(w[j]) == m) at = 2 * j;
        }
        return at;
    }
};

// This warp's share of a logit row: (max, lowest index) of it.
template <typename T>
__device__ __forceinline__ Best row_share(const T *row, int V, unsigned int rank, unsigned int blocks)
{
    constexpr int N = Lane<T>::kN;
    const int tid = threadIdx.x;
    // elements up to the first 16-byte boundary, whole vectors, the rest
    const int head = min(V, static_cast<int>((16u - (static_cast<unsigned int>(reinterpret_cast<uintptr_t>(row)) & 15u)) % 16u / sizeof(T)));
    const int n_vec = (V - head) / N;
    const uint4 *vec = reinterpret_cast<const uint4 *>(row + head);
    const int v0 = static_cast<int>(static_cast<long long>(n_vec) * rank / blocks), v1 = static_cast<int>(static_cast<long long>(n_vec) * (rank + 1) / blocks);
    float m = -INFINITY;
    int at = 0x7fffffff;
    bool odd = false;
    uint4 best = make_uint4(0u, 0u, 0u, 0u);
    for (int v = v0 + tid; v < v1; v += kThreads * kAtOnce) {
        uint4 x[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            if (v + j * kThreads < v1) x[j] = ptx::ld_written_once(vec + v + j * kThreads);
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (v + j * kThreads < v1) {
                const float y = Lane<T>::largest(x[j]);
                odd |= y != y;
                if (y > m) {
                    m = y;
                    at = v + j * kThreads;
                    best = x[j];
                }
            }
        }
    }
    int index = at == 0x7fffffff ? at : head + at * N + Lane<T>::first(best, m);
    // the ragged ends: the first block has the elements before the vectors, the last one those behind them
    auto single = [&](int i) {
        const float y = Lane<T>::one(row + i);
        odd |= y != y;
        if (y > m || (y == m && i < index)) {
            m = y;
            index = i;
        }
    };
    if (rank == 0 && tid < head) single(tid);
    if (rank == blocks - 1 && head + n_vec * N + tid < V) single(head + n_vec * N + tid);
    const Best mine = {ordered(m), index, odd ? 1 : 0};
    return warp_best(mine);
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) verify_tree_kernel(const Params p)
{
    __shared__ int token[kNodes], parent[kNodes];
    __shared__ Best of_warps[2][kMaxCluster * kWarps];                  // of all warps of the cluster, this block's copy
    __shared__ int decision, n_shared;
    __shared__ int path[kNodes], rec_d[kNodes], rec_t[kNodes], rescued[kNodes];        // the first block's
    ptx::cluster_arrive();                                              // that all blocks run is waited for behind the stream
    ptx::wait_for_stream();
    const unsigned int rank = ptx::cluster_rank(), blocks = ptx::cluster_size();
    const int b = blockIdx.x / blocks, tid = threadIdx.x, lane = tid & 31;
    // The tree is read by the first block and handed to the others: whatever another stream may do to it meanwhile, all walk the same one
    // and meet at the same barriers.
    const bool hands_over = rank == 0 && tid < kNodes;
    int nodes = 0, tok = -1, up = -1;
    if (hands_over) {
        nodes = min(p.n_nodes ? ptx::ld_written(p.n_nodes + b) : p.T, p.T);
        if (tid < p.T) {
            tok = ptx::ld_written(p.tokens + static_cast<long long>(b) * p.T + tid);
            up = ptx::ld_written(p.parents + b * p.parent_stride + tid);
        }
    }
    if (tid < kNodes) {
        path[tid] = rec_d[tid] = rec_t[tid] = -1;
        rescued[tid] = 0;
    }
    ptx::cluster_wait();
    if (hands_over) {
        for (unsigned int q = 0; q < blocks; ++q) {
            st_cluster(in_block(ptx::smem_u32(&token[tid]), q), static_cast<unsigned int>(tok));
            st_cluster(in_block(ptx::smem_u32(&parent[tid]), q), static_cast<unsigned int>(up));
            if (tid == 0) st_cluster(in_block(ptx::smem_u32(&n_shared), q), static_cast<unsigned int>(nodes));
        }
    }
    cluster_meet();
    const int n = n_shared;
    int length = 0, cur = n > 0 ? 0 : -1, star = -1, matches = 0, records = 0;
    unsigned int complaint = 0;
    while (cur >= 0) {
        if (tid == 0) path[length] = cur;
        const T *row = static_cast<const T *>(p.logits) + b * p.stride_b + cur * p.stride_t;
        const Best share = row_share<T>(row, p.V, rank, blocks);
        Best *const slots = of_warps[length & 1];                       // (read by all before the barrier after the next one)
        if (lane < static_cast<int>(blocks)) {
            const unsigned int to = in_block(ptx::smem_u32(&slots[rank * kWarps + (tid >> 5)]), lane);
            st_cluster(to, share.key);
            st_cluster(to + 4, static_cast<unsigned int>(share.index));
            st_cluster(to + 8, static_cast<unsigned int>(share.odd));
        }
        cluster_meet();
        Best all = {0u, 0x7fffffff, 0};
        for (int w = lane; w < static_cast<int>(blocks) * kWarps; w += 32) {
            const Best x = slots[w];
            if (x.key > all.key || (x.key == all.key && x.index < all.index)) {
                all.key = x.key;
                all.index = x.index;
            }
            all.odd |= x.odd;
        }
        all = warp_best(all);
        const float m = unordered(all.key);
        star = all.index == 0x7fffffff ? 0 : all.index;                 // (nothing above minus infinity: the lowest)
        if (all.odd || !isfinite(m)) complaint |= CSD_FLAG_NAN_LOGIT;
        ++length;
        // children of the node: lane and lane + 32
        int next = -1;
        bool child[2], any = false;
#pragma unroll
        for (int k = 1; k >= 0; --k) {
            const int t = lane + 32 * k;
            child[k] = t > cur && t < n && parent[t] == cur;
            const unsigned int same = __ballot_sync(kFull, child[k] && token[t] == star);
            if (same) next = 32 * k + __ffs(same) - 1;
            any |= __any_sync(kFull, child[k]);
        }
        if (next >= 0) {
            ++matches;
        } else if (any) {
            if (rank == 0 && tid < 32) {
                unsigned int best_key = 0u;                            // (below the key of every logit)
                int best_at = 0x7fffffff;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int t = lane + 32 * k;
                    if (!child[k]) continue;
                    const int d = token[t];
                    if (d < 0 || d >= p.V) {
                        complaint |= CSD_FLAG_BAD_DRAFT;
                        continue;
                    }
                    rec_d[t] = d;
                    rec_t[t] = star;
                    ++records;
                    const float zd = Lane<T>::one(row + d);
                    const unsigned int count = ocm_lookup(p.ocm, make_key(d, star));
                    const bool safe = static_cast<double>(zd) - static_cast<double>(m) >= static_cast<double>(p.log_tau);
                    if (count >= p.ocm.lambda && safe && ordered(zd) > best_key) {
                        best_key = ordered(zd);
                        best_at = t;
                    }
                }
                const unsigned int top = __reduce_max_sync(kFull, best_key);
                const int at = __reduce_min_sync(kFull, best_key == top ? best_at : 0x7fffffff);
                next = top == 0u ? -1 : at;
                if (lane == 0 && next >= 0) rescued[next] = 1;
                if (lane < static_cast<int>(blocks)) st_cluster(in_block(ptx::smem_u32(&decision), lane), static_cast<unsigned int>(next));
            }
            cluster_meet();
            next = decision;
        }
        cur = next;
    }
    if (rank != 0) return;
    __syncthreads();
    if (tid < p.T) {
        const long long at = static_cast<long long>(b) * p.T + tid;
        p.path[at] = path[tid];
        p.rescued[at] = static_cast<unsigned char>(rescued[tid]);
        p.rej_d[at] = rec_d[tid];
        p.rej_t[at] = rec_t[tid];
    }
    if (tid >= 32) return;
    records = __reduce_add_sync(kFull, records);
    const int rescues = __popc(__ballot_sync(kFull, rescued[lane] != 0)) + __popc(__ballot_sync(kFull, rescued[lane + 32] != 0));
    complaint = __reduce_or_sync(kFull, complaint);
    if (lane == 0) {
        p.accept_len[b] = max(length - 1, 0);
        p.next_token[b] = star;
        OcmStatsDev *st = p.ocm.stats;
        if (b == 0) atomicAdd(&st->steps, 1ull);
        if (n > 1) atomicAdd(&st->positions, static_cast<unsigned long long>(n - 1));
        if (matches) atomicAdd(&st->matches, static_cast<unsigned long long>(matches));
        if (rescues) atomicAdd(&st->rescues, static_cast<unsigned long long>(rescues));
        if (records) atomicAdd(&st->rejections, static_cast<unsigned long long>(records));
        if (complaint) atomicOr(&st->flags, complaint);
    }
}

}  // namespace verify_tree
}  // namespace csd
