// Attention of a row's newest tokens over its paged keys and values.
//
//   out[b,t,h] = sum_j w_j v_j,  w = softmax_j(scale q.k_j),  over the places j <= lens[b] - n_new[b] + t
//   lse[b,t,h] = ln sum_j exp(scale q.k_j)
//
// A token that sees nothing gives zeros and lse = -inf.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/csd.h"
#include "csd_common.cuh"
#include "csd_rope.cuh"

namespace csd {
namespace attention {

using rope::from_f32;
using rope::to_f32;

struct Params {
    const void *q;
    const void *k_pool, *v_pool;           // of this layer
    void *out;
    float *lse;
    int B, T, Hq, Hkv, D, group;
    long long qb, qt, qh;
    long long pool_page, pool_head, pool_token;
    int page_shift, n_pages, max_pages;
    const int *table, *lens, *n_new;
    unsigned int *flags;
    float scale;
};

// One block per (row, token, query head); its warps share the places out.
template <typename T>
__global__ void __launch_bounds__(128) attention_simple_kernel(const Params p)
{
    __shared__ float sm[4], sl[4], so[4][256];
    const int h = blockIdx.x % p.Hq, bt = blockIdx.x / p.Hq;
    const int b = bt / p.T, t = bt % p.T;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int news = p.n_new ? p.n_new[b] : p.T;
    const int last = t < news ? p.lens[b] - news + t : -1;
    const T *q = static_cast<const T *>(p.q) + b * p.qb + t * p.qt + h * p.qh;
    float qr[8], acc[8], m = -INFINITY, l = 0.f;
    for (int i = 0; i < 8; ++i) {
        const int d = lane + 32 * i;
        qr[i] = d < p.D ? to_f32(q[d]) * p.scale : 0.f;
        acc[i] = 0.f;
    }
    for (int j = warp; j <= last; j += 4) {
        const int slot = j >> p.page_shift;
        const int page = slot < p.max_pages ? p.table[static_cast<long long>(b) * p.max_pages + slot] : -1;
        if (page < 0 || page >= p.n_pages) {
            if (lane == 0) atomicOr(p.flags, CSD_CACHE_BAD_PAGE);
            continue;
        }
        const long long at = page * p.pool_page + (h / p.group) * p.pool_head + (j & ((1 << p.page_shift) - 1)) * p.pool_token;
        const T *k = static_cast<const T *>(p.k_pool) + at, *v = static_cast<const T *>(p.v_pool) + at;
        float s = 0.f;
        for (int i = 0; i < 8; ++i) {
            const int d = lane + 32 * i;
            if (d < p.D) s += qr[i] * to_f32(k[d]);
        }
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
        const float mn = fmaxf(m, s), at0 = mn == -INFINITY ? 0.f : mn, f = expf(m - at0), w = expf(s - at0);   // a NaN score stays one
        l = l * f + w;
        for (int i = 0; i < 8; ++i) {
            const int d = lane + 32 * i;
            if (d < p.D) acc[i] = acc[i] * f + w * to_f32(v[d]);
        }
        m = mn;
    }
    if (lane == 0) {
        sm[warp] = m;
        sl[warp] = l;
    }
    for (int i = 0; i < 8; ++i) so[warp][lane + 32 * i] = acc[i];
    __syncthreads();
    float M = -INFINITY, L = 0.f;
    for (int w = 0; w < 4; ++w) M = fmaxf(M, sm[w]);
    const float M0 = M == -INFINITY ? 0.f : M;
    for (int w = 0; w < 4; ++w) L += sl[w] == 0.f ? 0.f : sl[w] * expf(fmaxf(sm[w], -3e38f) - fmaxf(M0, -3e38f));
    const long long row = (static_cast<long long>(b) * p.T + t) * p.Hq + h;
    for (int d = threadIdx.x; d < p.D; d += 128) {
        float o = 0.f;
        for (int w = 0; w < 4; ++w) o += sl[w] == 0.f ? 0.f : so[w][d] * expf(fmaxf(sm[w], -3e38f) - fmaxf(M0, -3e38f));
        static_cast<T *>(p.out)[row * p.D + d] = from_f32<T>(L == 0.f ? 0.f : o / L);
    }
    if (p.lse && threadIdx.x == 0) p.lse[row] = L == 0.f ? -INFINITY : M0 + logf(L);
}

}  // namespace attention
}  // namespace csd
