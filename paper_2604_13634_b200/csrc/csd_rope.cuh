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
// Bound: memory (every element read once, written once).  A block has a few whole tokens.  Its threads first put the tokens' sines
// and cosines into shared memory, one per pair and token; then each thread turns one unit (P = 16 bytes' worth of pairs: two
// 16-byte vectors, neighbouring lanes neighbouring vectors) of kHeads heads, whose loads it has issued before.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/csd.h"
#include "csd_common.cuh"
#include "csd_ptx.cuh"

namespace csd {
namespace rope {

constexpr int kThreads = 256;          // a block
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

// Cosine and sine of one pair's angle, times the magnitude.
__device__ __forceinline__ float2 angle(const Turn &t, int pair, int position, bool inverse)
{
    const unsigned long long phase = static_cast<unsigned long long>(static_cast<long long>(position)) * __ldg(t.steps + pair);
    const float half_turns = static_cast<float>(static_cast<int>(phase >> 32)) * 0x1p-31f;         // angle / pi, in [-1, 1]
    float s, c;
    sincospif(half_turns, &s, &c);
    return make_float2(c * t.magnitude, s * (inverse ? -t.magnitude : t.magnitude));
}

// A unit in registers: two vectors of P elements.  Pair j: (a[j], b[j]) in the half layout; consecutive elements of the run a, b in
// the interleaved one.  One product rounded, one fused, spelled out so that every variant gives the same bits.
template <typename T, int P>
struct Vec;

template <typename T>
struct Vec<T, 1> {
    T v;
};
template <>
struct Vec<float, 4> {
    float4 v;
};
template <>
struct Vec<__nv_bfloat16, 8> {
    uint4 v;
};
template <>
struct Vec<__half, 8> {
    uint4 v;
};

template <bool kHalf, typename T>
__device__ __forceinline__ void turn(Vec<T, 1> &a, Vec<T, 1> &b, const float2 (&cs)[1])
{
    const float f0 = to_f32(a.v), f1 = to_f32(b.v);
    a.v = from_f32<T>(__fmaf_rn(f0, cs[0].x, -__fmul_rn(f1, cs[0].y)));
    b.v = from_f32<T>(__fmaf_rn(f1, cs[0].x, __fmul_rn(f0, cs[0].y)));
}

__device__ __forceinline__ void turn_pair(float &x0, float &x1, const float2 &cs)
{
    const float f0 = x0, f1 = x1;
    x0 = __fmaf_rn(f0, cs.x, -__fmul_rn(f1, cs.y));
    x1 = __fmaf_rn(f1, cs.x, __fmul_rn(f0, cs.y));
}

template <bool kHalf>
__device__ __forceinline__ void turn(Vec<float, 4> &a, Vec<float, 4> &b, const float2 (&cs)[4])
{
    if constexpr (kHalf) {
        turn_pair(a.v.x, b.v.x, cs[0]);
        turn_pair(a.v.y, b.v.y, cs[1]);
        turn_pair(a.v.z, b.v.z, cs[2]);
        turn_pair(a.v.w, b.v.w, cs[3]);
    } else {
        turn_pair(a.v.x, a.v.y, cs[0]);
        turn_pair(a.v.z, a.v.w, cs[1]);
        turn_pair(b.v.x, b.v.y, cs[2]);
        turn_pair(b.v.z, b.v.w, cs[3]);
    }
}

template <typename T>
__device__ __forceinline__ float2 unpack_word(unsigned int w);
template <>
__device__ __forceinline__ float2 unpack_word<__nv_bfloat16>(unsigned int w)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <>
__device__ __forceinline__ float2 unpack_word<__half>(unsigned int w)
{
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
template <typename T>
__device__ __forceinline__ unsigned int pack_word(float lo, float hi);
template <>
__device__ __forceinline__ unsigned int pack_word<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned int *>(&v);
}
template <>
__device__ __forceinline__ unsigned int pack_word<__half>(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const unsigned int *>(&v);
}

// two pairs (a.lo, b.lo), (a.hi, b.hi) on packed arithmetic
template <typename T>
__device__ __forceinline__ void turn_words_half(unsigned int &a, unsigned int &b, const float2 &cs0, const float2 &cs1)
{
    const float2 fa = unpack_word<T>(a), fb = unpack_word<T>(b);
    const unsigned long long x = pack2(fa.x, fa.y), y = pack2(fb.x, fb.y), c = pack2(cs0.x, cs1.x), s = pack2(cs0.y, cs1.y), n = pack2(-cs0.y, -cs1.y);
    float r0, r1;
    unpack2(fma2(x, c, mul2(y, n)), r0, r1);
    a = pack_word<T>(r0, r1);
    unpack2(fma2(y, c, mul2(x, s)), r0, r1);
    b = pack_word<T>(r0, r1);
}
// one pair (a.lo, a.hi)
template <typename T>
__device__ __forceinline__ void turn_word_interleaved(unsigned int &a, const float2 &cs)
{
    const float2 f = unpack_word<T>(a);
    float r0, r1;
    unpack2(fma2(pack2(f.x, f.y), pack2(cs.x, cs.x), mul2(pack2(f.y, f.x), pack2(-cs.y, cs.y))), r0, r1);
    a = pack_word<T>(r0, r1);
}

template <bool kHalf, typename T>
__device__ __forceinline__ void turn(Vec<T, 8> &a, Vec<T, 8> &b, const float2 (&cs)[8])
{
    if constexpr (kHalf) {
        turn_words_half<T>(a.v.x, b.v.x, cs[0], cs[1]);
        turn_words_half<T>(a.v.y, b.v.y, cs[2], cs[3]);
        turn_words_half<T>(a.v.z, b.v.z, cs[4], cs[5]);
        turn_words_half<T>(a.v.w, b.v.w, cs[6], cs[7]);
    } else {
        turn_word_interleaved<T>(a.v.x, cs[0]);
        turn_word_interleaved<T>(a.v.y, cs[1]);
        turn_word_interleaved<T>(a.v.z, cs[2]);
        turn_word_interleaved<T>(a.v.w, cs[3]);
        turn_word_interleaved<T>(b.v.x, cs[4]);
        turn_word_interleaved<T>(b.v.y, cs[5]);
        turn_word_interleaved<T>(b.v.z, cs[6]);
        turn_word_interleaved<T>(b.v.w, cs[7]);
    }
}

// Which token, unit and group of heads a thread has: `per_token` threads a token, `tokens` tokens to a block (grid.y > 1 where a
// token takes more than a block).  32-bit quotients only: the 64-bit ones of a flat index cost more than the rotation.
struct Places {
    int per_token, tokens;
    int n_tokens;
};

struct Place {
    int token, unit, group, in_block;
    bool ok;
};

// cosines and sines of a block's tokens: element (token, j, u) is pair u P + j, so that neighbouring units are neighbours
constexpr int kMaxRot = 4096;
constexpr int kTable = kMaxRot / 2;        // tokens * rot / 2 <= threads * P <= this, too

__device__ __forceinline__ Place place_of(const Places &p, int units)
{
    Place r;
    int i = threadIdx.x;
    r.in_block = 0;
    if (p.tokens > 1) {
        r.in_block = i / p.per_token;
        i -= r.in_block * p.per_token;
    } else {
        i += blockIdx.y * kThreads;
    }
    r.token = blockIdx.x * p.tokens + r.in_block;
    r.group = i / units;
    r.unit = i - r.group * units;
    r.ok = r.in_block < p.tokens && i < p.per_token && r.token < p.n_tokens;
    return r;
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
    int units;                             // of a head
    Places at;
};

template <typename T, int P, bool kHalf>
__global__ void __launch_bounds__(kThreads, 3) rope_kernel(const RopeParams p)
{
    __shared__ float2 table[kTable];
    ptx::wait_for_stream();
    const Place at = place_of(p.at, p.units);
    const int u = at.unit, h0 = at.group * kHeads, pairs = p.turn.rot / 2, turning = pairs / P;
    const Unit un = unit_at<P, kHalf>(u, p.turn.rot, p.D);
    Vec<T, P> a[kHeads], c[kHeads];
    int b = 0, s = 0;
    if (at.ok) {
        b = at.token / p.S;
        s = at.token - b * p.S;
        const T *x = static_cast<const T *>(p.x) + b * p.xb + s * p.xs;
#pragma unroll
        for (int k = 0; k < kHeads; ++k) {
            if (h0 + k < p.H) {
                const T *xh = x + (h0 + k) * p.xh;
                a[k] = *reinterpret_cast<const Vec<T, P> *>(xh + un.a);
                if (un.second) c[k] = *reinterpret_cast<const Vec<T, P> *>(xh + un.b);
            }
        }
    }
    for (int i = threadIdx.x; i < p.at.tokens * pairs; i += kThreads) {
        const int k = i / pairs, pair = i - k * pairs, token = blockIdx.x * p.at.tokens + k;
        if (token < p.at.n_tokens) {
            const int tb = token / p.S, ts = token - tb * p.S;
            table[k * pairs + (pair % P) * turning + pair / P] = angle(p.turn, pair, __ldg(p.positions + tb * p.pb + ts * p.ps), p.inverse != 0);
        }
    }
    __syncthreads();
    if (!at.ok) return;
    if (un.turns) {
        float2 cs[P];
#pragma unroll
        for (int j = 0; j < P; ++j) cs[j] = table[at.in_block * pairs + j * turning + u];
#pragma unroll
        for (int k = 0; k < kHeads; ++k) turn<kHalf>(a[k], c[k], cs);
    }
    T *y = static_cast<T *>(p.y) + b * p.yb + s * p.ys;
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
        if (h0 + k < p.H) {
            T *yh = y + (h0 + k) * p.yh;
            *reinterpret_cast<Vec<T, P> *>(yh + un.a) = a[k];
            if (un.second) *reinterpret_cast<Vec<T, P> *>(yh + un.b) = c[k];
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
    Places at;
};

// One launch for the new tokens' queries (turned, to q_out), keys (turned, to their page slots) and values (to their
// page slots).  Token t of row b lies at place lens[b] - n_new[b] + t; one that does not exist (t >= n_new[b], or a
// negative place) gets a zero query and touches no page.
template <typename T, int P, bool kHalf>
__global__ void __launch_bounds__(kThreads, 3) rope_append_kernel(const AppendParams p)
{
    __shared__ float2 table[kTable];
    ptx::wait_for_stream();
    const Place at = place_of(p.at, p.units);
    const int u = at.unit, pairs = p.turn.rot / 2, turning = pairs / P;
    const Unit un = unit_at<P, kHalf>(u, p.turn.rot, p.D);
    const int b = at.token / p.T, t = at.token - b * p.T;
    const int which = at.group < p.q_groups ? 0 : (at.group < p.q_groups + p.kv_groups ? 1 : 2);
    const int h0 = (at.group - (which == 0 ? 0 : (which == 1 ? p.q_groups : p.q_groups + p.kv_groups))) * kHeads;
    const int H = which == 0 ? p.Hq : p.Hkv;
    Vec<T, P> a[kHeads], c[kHeads];
    int place = 0, page = -1;
    bool real = false;
    if (at.ok) {
        const T *x = which == 0 ? static_cast<const T *>(p.q) + b * p.qb + t * p.qt
                                : (which == 1 ? static_cast<const T *>(p.k) + b * p.kb + t * p.kt : static_cast<const T *>(p.v) + b * p.vb + t * p.vt);
        const long long xh = which == 0 ? p.qh : (which == 1 ? p.kh : p.vh);
        // (rows and tokens that do not exist are read too: they lie in the caller's tensor)
#pragma unroll
        for (int k = 0; k < kHeads; ++k) {
            if (h0 + k < H) {
                const T *xr = x + (h0 + k) * xh;
                a[k] = *reinterpret_cast<const Vec<T, P> *>(xr + un.a);
                if (un.second) c[k] = *reinterpret_cast<const Vec<T, P> *>(xr + un.b);
            }
        }
        const int news = p.n_new ? __ldg(p.n_new + b) : p.T;
        place = __ldg(p.lens + b) - news + t;
        real = t < news && place >= 0;
        if (which != 0 && real) {
            const int slot = place >> p.page_shift;
            page = slot < p.max_pages ? __ldg(p.table + static_cast<long long>(b) * p.max_pages + slot) : -1;
        }
    }
    for (int i = threadIdx.x; i < p.at.tokens * pairs; i += kThreads) {
        const int k = i / pairs, pair = i - k * pairs, token = blockIdx.x * p.at.tokens + k;
        if (token < p.at.n_tokens) {
            const int tb = token / p.T, tt = token - tb * p.T;
            table[k * pairs + (pair % P) * turning + pair / P] =
                angle(p.turn, pair, __ldg(p.lens + tb) - (p.n_new ? __ldg(p.n_new + tb) : p.T) + tt, false);
        }
    }
    __syncthreads();
    if (!at.ok || (which != 0 && !real)) return;
    T *y;
    long long yh;
    if (which == 0) {
        y = static_cast<T *>(p.q_out) + static_cast<long long>(at.token) * p.Hq * p.D;
        yh = p.D;
    } else {
        if (page < 0 || page >= p.n_pages) {                      // a table that does not hold its row's tokens
            atomicOr(p.flags, CSD_CACHE_BAD_PAGE);
            return;
        }
        y = static_cast<T *>(which == 1 ? p.k_pool : p.v_pool) + page * p.pool_page + (place & ((1 << p.page_shift) - 1)) * p.pool_token;
        yh = p.pool_head;
    }
    if (un.turns && which != 2) {
        float2 cs[P];
#pragma unroll
        for (int j = 0; j < P; ++j) cs[j] = table[at.in_block * pairs + j * turning + u];
#pragma unroll
        for (int k = 0; k < kHeads; ++k) turn<kHalf>(a[k], c[k], cs);
    }
    if (!real) {
#pragma unroll
        for (int k = 0; k < kHeads; ++k) a[k] = c[k] = Vec<T, P>();
    }
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
        if (h0 + k < H) {
            T *yr = y + (h0 + k) * yh;
            *reinterpret_cast<Vec<T, P> *>(yr + un.a) = a[k];
            if (un.second) *reinterpret_cast<Vec<T, P> *>(yr + un.b) = c[k];
        }
    }
}

}  // namespace rope
}  // namespace csd
