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
// 268 MB of bf16 (4 x 4096 tokens, 32 heads of 128): 44.0 us, 6.1 TB/s.  16 MB of float32 (2 x 1023 tokens, 12 heads of 80 of which 32
// turn): 5.9 us, start and one pass.
// Where rot does not divide into such units but rows are made of whole vectors, a thread has one vector of kHeads heads instead:
// 38.4 us (interleaved; 90.7 pair by pair) for 170 MB with 66 of 168 elements turned; 268 MB with 126 of 128 turned in 45.9 us
// interleaved and 72 us half, where 128 of 128 take 44.0.  Pair by pair only where rows themselves are not whole vectors.
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

// Which token, unit and group of heads a thread has: `per_token` threads a token, `tokens` tokens to a block, or (grid.y > 1)
// `groups` groups of heads of one token to a block: a head lies in one block whole, so that a barrier can part its reads and its
// writes (0: heads of more units than a block has threads, whose units are read and written by one thread each).  32-bit quotients only: the 64-bit ones of a flat index cost more than the rotation.
struct Places {
    int per_token, tokens, groups;
    int n_tokens;
};

struct Place {
    int token, unit, group, in_block;
    bool ok;
};

// cosines and sines of a block's tokens: element (token, j, u) is pair u P + j, so that neighbouring units are neighbours
constexpr int kMaxRot = 4096;
constexpr int kTable = kMaxRot / 2 + 8;    // tokens * (rot / 2, rounded up to P) <= threads * P <= this, too

__device__ __forceinline__ Place place_of(const Places &p, int units)
{
    Place r;
    int i = threadIdx.x;
    r.in_block = 0;
    if (p.tokens > 1) {
        r.in_block = i / p.per_token;
        i -= r.in_block * p.per_token;
    } else {
        const int taken = p.groups > 0 ? p.groups * units : kThreads;
        if (i >= taken) r.in_block = 1;                            // (no token of its own: not ok below)
        i += blockIdx.y * taken;
    }
    r.token = blockIdx.x * p.tokens + r.in_block;
    r.group = i / units;
    r.unit = i - r.group * units;
    r.ok = r.in_block < p.tokens && i < p.per_token && r.token < p.n_tokens;
    return r;
}

// One 16-byte vector of a head's row, from element e0, as four words of W = 1 (float32) or 2 elements.  Its elements' partners: in
// the interleaved layout their neighbours; in the half layout other threads' elements (e < rot/2 pairs with e + rot/2), handed over in
// shared memory, word j of every thread's vector of head k in plane (k, j), so that lanes read neighbours.  Elements from rot on
// keep their bits.  With W = 2 and rot/2 odd a word's partners lie in two words, the upper half of one and the lower of another.
template <typename T>
struct Loose {
    static constexpr int W = 4 / static_cast<int>(sizeof(T));
    unsigned int w[4];

    __device__ __forceinline__ void load(const T *row, int e0)
    {
        const uint4 v = *reinterpret_cast<const uint4 *>(row + e0);
        w[0] = v.x;
        w[1] = v.y;
        w[2] = v.z;
        w[3] = v.w;
    }
    __device__ __forceinline__ void store(T *row, int e0) const { *reinterpret_cast<uint4 *>(row + e0) = make_uint4(w[0], w[1], w[2], w[3]); }
    __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0u; }
    __device__ __forceinline__ void hand_over(unsigned int *planes, int k) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) planes[(k * 4 + j) * kThreads + threadIdx.x] = w[j];
    }
};

// What a vector's elements are multiplied by, and where their partners lie: for all heads the same.
template <typename T, bool kHalf>
struct LooseTurn {
    static constexpr int W = Loose<T>::W, P = 4 * W;
    float2 cs[kHalf ? P : P / 2];
    int at[kHalf ? 4 : 1], at_next[kHalf && W == 2 ? 4 : 1];

    static __device__ __forceinline__ int place(int element, int first) { return element / W % 4 * kThreads + first + element / P; }

    // table: pair i at (i % P) * columns + i / P
    __device__ __forceinline__ LooseTurn(const float2 *table, int columns, int e0, int rot)
    {
        const int half = rot / 2, first = static_cast<int>(threadIdx.x) - e0 / P;           // the thread with the row's first vector
#pragma unroll
        for (int j = 0; j < (kHalf ? P : P / 2); ++j) {
            const int e = e0 + j, i = kHalf ? (e < half ? e : e - half) : e0 / 2 + j;
            if (kHalf ? e < rot : i < half) {
                cs[j] = table[(i % P) * columns + i / P];
                if (kHalf && e < half) cs[j].y = -cs[j].y;         // x0 cos - x1 sin: the product with the sign changed is the same product
            }
        }
        if constexpr (kHalf) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int e = e0 + j * W;
                if (e < rot) {
                    at[j] = place(e < half ? e + half : e - half, first);
                    if constexpr (W == 2) at_next[j] = place(e + 1 < half ? e + 1 + half : e + 1 - half, first);
                }
            }
        }
    }
    __device__ __forceinline__ void apply(Loose<T> &v, const unsigned int *planes, int k, int e0, int rot) const
    {
        if constexpr (kHalf) {
            const unsigned int *of_head = planes + k * 4 * kThreads;
            const bool odd = (rot / 2) & 1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (e0 + j * W < rot) {
                    unsigned int y = of_head[at[j]];
                    if constexpr (W == 1) {
                        v.w[j] = __float_as_uint(__fmaf_rn(__uint_as_float(v.w[j]), cs[j].x, __fmul_rn(__uint_as_float(y), cs[j].y)));
                    } else {
                        if (odd) y = __funnelshift_r(y, of_head[at_next[j]], 16);
                        const float2 fx = unpack_word<T>(v.w[j]), fy = unpack_word<T>(y);
                        float r0, r1;
                        unpack2(fma2(pack2(fx.x, fx.y), pack2(cs[2 * j].x, cs[2 * j + 1].x), mul2(pack2(fy.x, fy.y), pack2(cs[2 * j].y, cs[2 * j + 1].y))), r0, r1);
                        v.w[j] = pack_word<T>(r0, r1);
                    }
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < P / 2; ++j)
                if (e0 + 2 * j < rot) {
                    if constexpr (W == 1) {
                        float x = __uint_as_float(v.w[2 * j]), y = __uint_as_float(v.w[2 * j + 1]);
                        turn_pair(x, y, cs[j]);
                        v.w[2 * j] = __float_as_uint(x);
                        v.w[2 * j + 1] = __float_as_uint(y);
                    } else {
                        turn_word_interleaved<T>(v.w[j], cs[j]);
                    }
                }
        }
    }
};

// The two shapes of a thread's work under one interface: whole units (kLoose false) and single vectors.
template <typename T, int P, bool kHalf, bool kLoose>
struct Piece;
template <typename T, int P, bool kHalf>
struct Piece<T, P, kHalf, false> {
    Vec<T, P> a, c;
    static __device__ __forceinline__ int columns(int rot) { return rot / 2 / P; }
    __device__ __forceinline__ void load(const T *row, int u, int rot, int D)
    {
        const Unit un = unit_at<P, kHalf>(u, rot, D);
        a = *reinterpret_cast<const Vec<T, P> *>(row + un.a);
        if (un.second) c = *reinterpret_cast<const Vec<T, P> *>(row + un.b);
    }
    __device__ __forceinline__ void turn_by(const float2 (&cs)[P]) { turn<kHalf>(a, c, cs); }
    __device__ __forceinline__ void store(T *row, int u, int rot, int D) const
    {
        const Unit un = unit_at<P, kHalf>(u, rot, D);
        *reinterpret_cast<Vec<T, P> *>(row + un.a) = a;
        if (un.second) *reinterpret_cast<Vec<T, P> *>(row + un.b) = c;
    }
    __device__ __forceinline__ void zero() { a = c = Vec<T, P>(); }
};
template <typename T, int P, bool kHalf>
struct Piece<T, P, kHalf, true> {
    Loose<T> v;
    static __device__ __forceinline__ int columns(int rot) { return (rot / 2 + P - 1) / P; }
    __device__ __forceinline__ void load(const T *row, int u, int, int) { v.load(row, u * P); }
    __device__ __forceinline__ void store(T *row, int u, int, int) const { v.store(row, u * P); }
    __device__ __forceinline__ void zero() { v.zero(); }
};

// All heads of a thread turned by its token's table.
template <typename T, int P, bool kHalf, bool kLoose, int kHeads_>
__device__ __forceinline__ void turn_all(Piece<T, P, kHalf, kLoose> (&x)[kHeads_], const float2 *table, const unsigned int *planes, int u, int rot, int D)
{
    const int columns = Piece<T, P, kHalf, kLoose>::columns(rot);
    if constexpr (kLoose) {
        const LooseTurn<T, kHalf> by(table, columns, u * P, rot);
#pragma unroll
        for (int k = 0; k < kHeads_; ++k) by.apply(x[k].v, planes, k, u * P, rot);
    } else if (unit_at<P, kHalf>(u, rot, D).turns) {
        float2 cs[P];
#pragma unroll
        for (int j = 0; j < P; ++j) cs[j] = table[j * columns + u];
#pragma unroll
        for (int k = 0; k < kHeads_; ++k) x[k].turn_by(cs);
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
    int units;                             // of a head
    Places at;
};

template <typename T, int P, bool kHalf, bool kLoose>
__global__ void __launch_bounds__(kThreads, 3) rope_kernel(const RopeParams p)
{
    using Mine = Piece<T, P, kHalf, kLoose>;
    __shared__ float2 table[kTable];
    __shared__ unsigned int planes[kLoose && kHalf ? kThreads * kHeads * 4 : 1];
    ptx::wait_for_stream();
    const Place at = place_of(p.at, p.units);
    const int u = at.unit, h0 = at.group * kHeads, pairs = p.turn.rot / 2, columns = Mine::columns(p.turn.rot), each = columns * P;
    Mine x[kHeads];
    int b = 0, s = 0;
    if (at.ok) {
        b = at.token / p.S;
        s = at.token - b * p.S;
        const T *from = static_cast<const T *>(p.x) + b * p.xb + s * p.xs;
#pragma unroll
        for (int k = 0; k < kHeads; ++k)
            if (h0 + k < p.H) {
                x[k].load(from + (h0 + k) * p.xh, u, p.turn.rot, p.D);
                if constexpr (kLoose && kHalf) x[k].v.hand_over(planes, k);
            }
    }
    for (int i = threadIdx.x; i < p.at.tokens * pairs; i += kThreads) {
        const int k = i / pairs, pair = i - k * pairs, token = blockIdx.x * p.at.tokens + k;
        if (token < p.at.n_tokens) {
            const int tb = token / p.S, ts = token - tb * p.S;
            table[k * each + (pair % P) * columns + pair / P] = angle(p.turn, pair, ptx::ld_written(p.positions + tb * p.pb + ts * p.ps), p.inverse != 0);
        }
    }
    __syncthreads();                       // the table is complete; and every element has been read (y may be x)
    if (!at.ok) return;
    turn_all<T, P, kHalf, kLoose>(x, table + at.in_block * each, planes, u, p.turn.rot, p.D);
    T *to = static_cast<T *>(p.y) + b * p.yb + s * p.ys;
#pragma unroll
    for (int k = 0; k < kHeads; ++k)
        if (h0 + k < p.H) x[k].store(to + (h0 + k) * p.yh, u, p.turn.rot, p.D);
}

struct AppendParams {
    const void *q, *k, *v;
    void *q_out, *k_pool, *v_pool;         // pools: of this layer
    int B, T, Hq, Hkv, D;
    long long qb, qt, qh, kb, kt, kh, vb, vt, vh;
    long long pool_page, pool_head, pool_token;
    int page_shift, n_pages, max_pages;
    const int *table, *lens, *n_new;
    const int *positions;                  // [B, T] what the tokens are turned by; null: their places
    unsigned int *flags;
    Turn turn;
    int units, q_groups, kv_groups;
    Places at;
};

// One launch for the new tokens' queries (turned, to q_out), keys (turned, to their page slots) and values (to their
// page slots).  Token t of row b lies at place lens[b] - n_new[b] + t; one that does not exist (t >= n_new[b], or a
// negative place) gets a zero query and touches no page.
// Bound: latency for one token (2.6 us: launch, length, page id, store), memory beyond (9.2 us for 28 MB: 128 rows of nine tokens, 32 +
// 2 x 8 heads of 128, where the chain of those reads is a third and 132 of the 576 blocks run as a second wave).
template <typename T, int P, bool kHalf, bool kLoose>
__global__ void __launch_bounds__(kThreads, 3) rope_append_kernel(const AppendParams p)
{
    using Mine = Piece<T, P, kHalf, kLoose>;
    __shared__ float2 table[kTable];
    __shared__ unsigned int planes[kLoose && kHalf ? kThreads * kHeads * 4 : 1];
    ptx::wait_for_stream();
    const Place at = place_of(p.at, p.units);
    const int u = at.unit, pairs = p.turn.rot / 2, columns = Mine::columns(p.turn.rot), each = columns * P;
    const int b = at.token / p.T, t = at.token - b * p.T;
    const int which = at.group < p.q_groups ? 0 : (at.group < p.q_groups + p.kv_groups ? 1 : 2);
    const int h0 = (at.group - (which == 0 ? 0 : (which == 1 ? p.q_groups : p.q_groups + p.kv_groups))) * kHeads;
    const int H = which == 0 ? p.Hq : p.Hkv;
    Mine x[kHeads];
    int place = 0, page = -1;
    bool real = false;
    if (at.ok) {
        const T *from = which == 0 ? static_cast<const T *>(p.q) + b * p.qb + t * p.qt
                                   : (which == 1 ? static_cast<const T *>(p.k) + b * p.kb + t * p.kt : static_cast<const T *>(p.v) + b * p.vb + t * p.vt);
        const long long head = which == 0 ? p.qh : (which == 1 ? p.kh : p.vh);
        // (rows and tokens that do not exist are read too: they lie in the caller's tensor)
#pragma unroll
        for (int k = 0; k < kHeads; ++k)
            if (h0 + k < H) {
                x[k].load(from + (h0 + k) * head, u, p.turn.rot, p.D);
                if constexpr (kLoose && kHalf) x[k].v.hand_over(planes, k);
            }
        const int news = p.n_new ? ptx::ld_written(p.n_new + b) : p.T;
        place = ptx::ld_written(p.lens + b) - news + t;
        real = t < news && place >= 0;
        if (which != 0 && real) {
            const int slot = place >> p.page_shift;
            page = slot < p.max_pages ? ptx::ld_written(p.table + static_cast<long long>(b) * p.max_pages + slot) : -1;
        }
    }
    for (int i = threadIdx.x; i < p.at.tokens * pairs; i += kThreads) {
        const int k = i / pairs, pair = i - k * pairs, token = blockIdx.x * p.at.tokens + k;
        if (token < p.at.n_tokens) {
            const int tb = token / p.T, tt = token - tb * p.T;
            const int position = p.positions ? ptx::ld_written(p.positions + static_cast<long long>(tb) * p.T + tt)
                                             : ptx::ld_written(p.lens + tb) - (p.n_new ? ptx::ld_written(p.n_new + tb) : p.T) + tt;
            table[k * each + (pair % P) * columns + pair / P] = angle(p.turn, pair, position, false);
        }
    }
    __syncthreads();                       // the table is complete; and every element has been read (q_out may be q)
    if (!at.ok || (which != 0 && !real)) return;
    T *to;
    long long head;
    if (which == 0) {
        to = static_cast<T *>(p.q_out) + static_cast<long long>(at.token) * p.Hq * p.D;
        head = p.D;
    } else {
        if (page < 0 || page >= p.n_pages) {                      // a table that does not hold its row's tokens
            atomicOr(p.flags, CSD_CACHE_BAD_PAGE);
            return;
        }
        to = static_cast<T *>(which == 1 ? p.k_pool : p.v_pool) + page * p.pool_page + (place & ((1 << p.page_shift) - 1)) * p.pool_token;
        head = p.pool_head;
    }
    if (which != 2) turn_all<T, P, kHalf, kLoose>(x, table + at.in_block * each, planes, u, p.turn.rot, p.D);
    if (!real) {
#pragma unroll
        for (int k = 0; k < kHeads; ++k) x[k].zero();
    }
#pragma unroll
    for (int k = 0; k < kHeads; ++k)
        if (h0 + k < H) x[k].store(to + (h0 + k) * head, u, p.turn.rot, p.D);
}

}  // namespace rope
}  // namespace csd
