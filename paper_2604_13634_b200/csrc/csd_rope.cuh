// Rotary positions: pairs of a head's elements turned by an angle proportional to the token's position, and the
// serving form that also puts the new keys and values into their page slots.
//
//   a = p theta_i,  i < rot/2;   y0 = m (x0 cos a - x1 sin a),  y1 = m (x1 cos a + x0 sin a)
//   half layout: (x0, x1) = (x[i], x[i + rot/2]);  interleaved: (x[2i], x[2i + 1]);  elements from rot on pass through.
//   A rotation is orthogonal, so the gradient is the rotation by -a with the same factor m.
//
// The angle: theta_i is kept as a 64-bit fraction of a turn, so p * step mod 2^64 IS the angle, exactly reduced at any
// position (a float32 product p * theta is off by 2^-24 p theta: 0.008 rad at p = 131072).  The top 32 bits are
// rounded to float32 once and go to sincospif; sums and products are float32, rounded once to the output's type.
//
// Bound: memory (every element read once, written once).  A thread owns one unit (P = 16 bytes' worth of pairs: two
// 16-byte vectors, neighbouring lanes neighbouring vectors) of up to kHeads heads of one token, so the P sines and
// cosines of a unit are paid once for kHeads heads.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/csd.h"
#include "csd_ptx.cuh"

namespace csd {
namespace rope {

constexpr int kThreads = 256;
constexpr int kHeads = 4;              // heads per thread

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// P elements that travel together
template <typename T, int P>
struct alignas(sizeof(T) * P) Pack {
    T e[P];
};

struct Turn {
    const unsigned long long *steps;   // [rot / 2] fraction of a turn per position, times 2^64
    int rot;                           // rotated elements of a head (even, 0 .. D)
    float magnitude;
};

// Where the elements of unit u lie: [a, a + P) and, if second, [b, b + P).  Units [0, turning) rotate, the rest copy.
struct Unit {
    int a, b;
    bool turns, second;
};

template <int P, bool kHalf>
__device__ __forceinline__ Unit unit_at(int u, int rot, int D)
{
    Unit r;
    const int turning = rot / (2 * P);
    r.turns = u < turning;
    r.second = true;
    if (r.turns) {
        r.a = kHalf ? u * P : 2 * u * P;
        r.b = kHalf ? rot / 2 + u * P : r.a + P;
    } else {
        r.a = rot + 2 * (u - turning) * P;
        r.b = r.a + P;
        r.second = r.b < D;
    }
    return r;
}

template <int P, bool kHalf>
__device__ __forceinline__ void angles(const Turn &t, int u, long long position, bool inverse, float (&c)[P], float (&s)[P])
{
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const unsigned long long phase = static_cast<unsigned long long>(position) * __ldg(t.steps + u * P + j);
        const float half_turns = static_cast<float>(static_cast<int>(phase >> 32)) * 0x1p-31f;     // angle / pi, in [-1, 1]
        sincospif(half_turns, &s[j], &c[j]);
        s[j] *= inverse ? -t.magnitude : t.magnitude;
        c[j] *= t.magnitude;
    }
}

// Two vectors of a rotating unit.  Pair j of the unit: (a[j], b[j]) in the half layout; consecutive elements of the
// run a, b in the interleaved one.
template <typename T, int P, bool kHalf>
__device__ __forceinline__ void turn(Pack<T, P> &a, Pack<T, P> &b, const float (&c)[P], const float (&s)[P])
{
#pragma unroll
    for (int j = 0; j < P; ++j) {
        T *x0 = kHalf ? &a.e[j] : (2 * j < P ? &a.e[2 * j < P ? 2 * j : 0] : &b.e[2 * j < P ? 0 : 2 * j - P]);
        T *x1 = kHalf ? &b.e[j] : (2 * j + 1 < P ? &a.e[2 * j + 1 < P ? 2 * j + 1 : 0] : &b.e[2 * j + 1 < P ? 0 : 2 * j + 1 - P]);
        const float f0 = to_f32(*x0), f1 = to_f32(*x1);
        // one product rounded, one fused: spelled out so that every variant of the kernel gives the same bits
        *x0 = from_f32<T>(__fmaf_rn(f0, c[j], -__fmul_rn(f1, s[j])));
        *x1 = from_f32<T>(__fmaf_rn(f1, c[j], __fmul_rn(f0, s[j])));
    }
}

struct RopeParams {
    const void *x;
    void *y;
    int B, S, H, D;
    long long xb, xs, xh, yb, ys, yh;      // strides in elements
    const int *positions;
    long long pb, ps;
    Turn turn;
    int inverse;
    int units, groups;                     // units of a head, groups of kHeads heads
    long long threads;
};

template <typename T, int P, bool kHalf>
__global__ void __launch_bounds__(kThreads) rope_kernel(const RopeParams p)
{
    ptx::wait_for_stream();
    const long long at = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    if (at >= p.threads) return;
    const long long tg = at / p.units;
    const int u = static_cast<int>(at - tg * p.units);
    const long long token = tg / p.groups;
    const int h0 = static_cast<int>(tg - token * p.groups) * kHeads;
    const int b = static_cast<int>(token / p.S), s = static_cast<int>(token - static_cast<long long>(b) * p.S);
    const T *x = static_cast<const T *>(p.x) + b * p.xb + s * p.xs;
    T *y = static_cast<T *>(p.y) + b * p.yb + s * p.ys;
    const Unit un = unit_at<P, kHalf>(u, p.turn.rot, p.D);
    Pack<T, P> a[kHeads], c2[kHeads];
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
        if (h0 + k < p.H) {
            const T *xh = x + (h0 + k) * p.xh;
            a[k] = *reinterpret_cast<const Pack<T, P> *>(xh + un.a);
            if (un.second) c2[k] = *reinterpret_cast<const Pack<T, P> *>(xh + un.b);
        }
    }
    if (un.turns) {
        float cs[P], sn[P];
        angles<P, kHalf>(p.turn, u, __ldg(p.positions + b * p.pb + s * p.ps), p.inverse != 0, cs, sn);
#pragma unroll
        for (int k = 0; k < kHeads; ++k) turn<T, P, kHalf>(a[k], c2[k], cs, sn);
    }
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
        if (h0 + k < p.H) {
            T *yh = y + (h0 + k) * p.yh;
            *reinterpret_cast<Pack<T, P> *>(yh + un.a) = a[k];
            if (un.second) *reinterpret_cast<Pack<T, P> *>(yh + un.b) = c2[k];
        }
    }
}

struct AppendParams {
    const void *q, *k, *v;
    void *q_out, *k_pool, *v_pool;         // pools: of this layer
    int B, T, Hq, Hkv, D;
    long long qb, qt, qh, kb, kt, kh, vb, vt, vh;
    long long pool_page, pool_head, pool_token;
    int page_shift, n_pages, max_pages;
    const int *table, *lens, *n_new;
    unsigned int *flags;
    Turn turn;
    int units, q_groups, kv_groups;
    long long threads;
};

// One launch for the new tokens' queries (turned, to q_out), keys (turned, to their page slots) and values (to their
// page slots).  Token t of row b lies at place lens[b] - n_new[b] + t; one that does not exist (t >= n_new[b], or a
// negative place) gets a zero query and touches no page.
template <typename T, int P, bool kHalf>
__global__ void __launch_bounds__(kThreads) rope_append_kernel(const AppendParams p)
{
    ptx::wait_for_stream();
    const long long at = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    if (at >= p.threads) return;
    const int groups = p.q_groups + 2 * p.kv_groups;
    const long long tg = at / p.units;
    const int u = static_cast<int>(at - tg * p.units);
    const long long token = tg / groups;
    int g = static_cast<int>(tg - token * groups);
    const int b = static_cast<int>(token / p.T), t = static_cast<int>(token - static_cast<long long>(b) * p.T);
    const int which = g < p.q_groups ? 0 : (g < p.q_groups + p.kv_groups ? 1 : 2);
    g -= which == 0 ? 0 : (which == 1 ? p.q_groups : p.q_groups + p.kv_groups);
    const int h0 = g * kHeads, H = which == 0 ? p.Hq : p.Hkv;
    const T *x = which == 0 ? static_cast<const T *>(p.q) + b * p.qb + t * p.qt
                            : (which == 1 ? static_cast<const T *>(p.k) + b * p.kb + t * p.kt : static_cast<const T *>(p.v) + b * p.vb + t * p.vt);
    const long long xh = which == 0 ? p.qh : (which == 1 ? p.kh : p.vh);
    const Unit un = unit_at<P, kHalf>(u, p.turn.rot, p.D);
    const int news = p.n_new ? __ldg(p.n_new + b) : p.T;
    const int place = __ldg(p.lens + b) - news + t;
    const bool real = t < news && place >= 0;
    if (!real && which != 0) return;
    Pack<T, P> a[kHeads], c2[kHeads];
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
        if (h0 + k < H && real) {
            const T *xr = x + (h0 + k) * xh;
            a[k] = *reinterpret_cast<const Pack<T, P> *>(xr + un.a);
            if (un.second) c2[k] = *reinterpret_cast<const Pack<T, P> *>(xr + un.b);
        } else {
#pragma unroll
            for (int j = 0; j < P; ++j) a[k].e[j] = c2[k].e[j] = from_f32<T>(0.f);
        }
    }
    T *y;
    long long yh;
    if (which == 0) {
        y = static_cast<T *>(p.q_out) + token * p.Hq * p.D;
        yh = p.D;
    } else {
        const int slot = place >> p.page_shift;
        const int page = slot < p.max_pages ? __ldg(p.table + static_cast<long long>(b) * p.max_pages + slot) : -1;
        if (page < 0 || page >= p.n_pages) {                      // a table that does not hold its row's tokens
            atomicOr(p.flags, CSD_CACHE_BAD_PAGE);
            return;
        }
        y = static_cast<T *>(which == 1 ? p.k_pool : p.v_pool) + page * p.pool_page + (place & ((1 << p.page_shift) - 1)) * p.pool_token;
        yh = p.pool_head;
    }
    if (un.turns && which != 2 && real) {
        float cs[P], sn[P];
        angles<P, kHalf>(p.turn, u, place, false, cs, sn);
#pragma unroll
        for (int k = 0; k < kHeads; ++k) turn<T, P, kHalf>(a[k], c2[k], cs, sn);
    }
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
        if (h0 + k < H) {
            T *yr = y + (h0 + k) * yh;
            *reinterpret_cast<Pack<T, P> *>(yr + un.a) = a[k];
            if (un.second) *reinterpret_cast<Pack<T, P> *>(yr + un.b) = c2[k];
        }
    }
}

}  // namespace rope
}  // namespace csd
