// Packed matrices: values in 8-bit floating point (e4m3: sign, 4 exponent bits, 3 mantissa bits) with one
// power-of-two scale per block of 128 values of a row, and what reads and writes them value by value.
//
// With e the smallest integer for which a block's largest magnitude is at most 448 * 2^e (448 = 1.75 * 2^8 is
// the largest e4m3 number), a value x is stored as the e4m3 number nearest to x * 2^-e.  The scale is a power of
// two, so x * 2^-e and code * 2^e are exact and the one rounding is the code's own: at most 2^-4 of the value
// above 2^-6 * 2^e, at most 2^-10 * 2^e below.  A scale of 32 bits would bring every block's largest value to exactly 448,
// which buys a floating-point code less than one binade of its 15 at the small end and nothing else, and
// would cost a multiply per product and block; a power of two goes into the matrix instruction as its scale operand.
//
// Every kernel here moves each byte once and is bound by HBM bandwidth, but for tanh and GELU from 8 bits to 16, which arithmetic bounds (unpack of 8192 x 4096:
// none and ReLU 17 us, logistic and SiLU 18, tanh 24, GELU 25; activation gradients 26, of GELU 30).
#pragma once
#include "common.hip.h"

namespace gtopk {

constexpr int kPackBlock = 128;             // values per scale
constexpr int kLaneVals = 8;                // consecutive values a lane handles: 16 lanes cover one block
constexpr int kPackThreads = 256;           // 16 blocks of 128 side by side

typedef uint32_t uint32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t uint32x4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

// dense matrices hold one of three types; they need only that type's own alignment, and rows at any stride
struct F32 { typedef float T; };
struct BF16 { typedef __bf16 T; };
struct F16 { typedef _Float16 T; };

template <class D> using Eight = typename D::T __attribute__((ext_vector_type(kLaneVals)));

// 8 consecutive values; p is aligned to one value (global memory takes wide accesses at any address)
template <class D>
__device__ __forceinline__ Eight<D> load_eight(const typename D::T* p) {
    struct __attribute__((packed)) Loose { Eight<D> v; };
    return reinterpret_cast<const Loose*>(p)->v;
}
template <class D>
__device__ __forceinline__ void load8(const typename D::T* p, float (&v)[kLaneVals]) {
    const Eight<D> x = load_eight<D>(p);
#pragma unroll
    for (int j = 0; j < kLaneVals; ++j) v[j] = (float)x[j];
}
template <class D>
__device__ __forceinline__ void store8(typename D::T* p, const float (&v)[kLaneVals]) {
    typedef typename D::T T;
    typedef T Vec __attribute__((ext_vector_type(kLaneVals)));
    struct __attribute__((packed)) Loose { Vec v; };
    Vec x;
#pragma unroll
    for (int j = 0; j < kLaneVals; ++j) x[j] = (T)v[j];      // to nearest, ties to even
    reinterpret_cast<Loose*>(p)->v = x;
}
// the same of the n < 8 values that a row's end leaves; 0 behind them
template <class D>
__device__ __forceinline__ void load_some(const typename D::T* p, int n, float (&v)[kLaneVals]) {
#pragma unroll
    for (int j = 0; j < kLaneVals; ++j) v[j] = j < n ? (float)p[j] : 0.0f;
}
template <class D>
__device__ __forceinline__ void store_some(typename D::T* p, int n, const float (&v)[kLaneVals]) {
#pragma unroll
    for (int j = 0; j < kLaneVals; ++j)
        if (j < n) p[j] = (typename D::T)v[j];
}

// 4 consecutive values, of which a row's end leaves `left`
template <class D>
__device__ __forceinline__ void store4(typename D::T* p, int64_t left, floatx4 v) {
    typedef typename D::T T;
    typedef T Vec __attribute__((ext_vector_type(4)));
    struct __attribute__((packed)) Loose { Vec v; };
    if (left >= 4) {
        Vec x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = (T)v[j];
        reinterpret_cast<Loose*>(p)->v = x;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) p[j] = (T)v[j];
    }
}

// 2^(s - 127); 255 stands for NaN
__device__ __forceinline__ float scale_value(uint32_t s) {
    return __uint_as_float(s == 0u ? 0x00400000u : s == 255u ? 0x7FC00000u : s << 23);
}
// the stored exponent e + 127 for a block whose largest finite magnitude has these bits
__device__ __forceinline__ uint32_t scale_for(uint32_t top) {
    const int s = (int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return s < 0 ? 0u : (uint32_t)s;
}
// 2^-e of a stored exponent that scale_for returned (0 .. 247)
__device__ __forceinline__ float inverse_scale(uint32_t s) { return __uint_as_float((254u - s) << 23); }

__device__ __forceinline__ bool finite_bits(uint32_t b) { return (b & 0x7F800000u) != 0x7F800000u; }

// bits of the largest finite magnitude among 8 values
__device__ __forceinline__ uint32_t top_of(const float (&v)[kLaneVals]) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < kLaneVals; ++j) {
        const uint32_t b = __float_as_uint(v[j]) & kAbs;
        if (finite_bits(b) && b > top) top = b;
    }
    return top;
}
// maximum over the 16 lanes of a DPP row, in all of them (row_ror:n = 0x120 + n)
__device__ __forceinline__ uint32_t row_largest(uint32_t v) {
    auto with = [&](uint32_t x) { v = x > v ? x : v; };
    with(dpp_moved<0x128, 0xf>(v));
    with(dpp_moved<0x124, 0xf>(v));
    with(dpp_moved<0x122, 0xf>(v));
    with(dpp_moved<0x121, 0xf>(v));
    return v;
}
// the codes of 8 values; what is not finite becomes the NaN code (e4m3 has no infinity), so that an overflow
// in the forward pass reaches the gradients instead of passing for a large value
__device__ __forceinline__ uint32x2 encode8(const float (&v)[kLaneVals], float inv) {
    float y[kLaneVals];
#pragma unroll
    for (int j = 0; j < kLaneVals; ++j)
        y[j] = finite_bits(__float_as_uint(v[j])) ? v[j] * inv : __uint_as_float(0x7FC00000u);
    uint32x2 c;
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    c[0] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
    c[1] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], w, true);
    return c;
}
__device__ __forceinline__ void decode8(uint32x2 c, float scale, float (&v)[kLaneVals]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], false);
        const floatx2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], true);
        v[4 * h] = lo[0] * scale;
        v[4 * h + 1] = lo[1] * scale;
        v[4 * h + 2] = hi[0] * scale;
        v[4 * h + 3] = hi[1] * scale;
    }
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// the lower (upper) two codes of a word as bf16 numbers times a power of two: exact down to 2^-126, below that
// rounded to a multiple of 2^-133.  (The word is taken whole: taking the vector's elements apart gives the first one twice.)
template <bool UPPER>
__device__ __forceinline__ uint32_t decode2(uint32_t c, float scale) {
    const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, UPPER);
    return __builtin_bit_cast(uint32_t, v);
}

// keeps the instructions that compute v in front of what follows
__device__ __forceinline__ void pin(floatx4& v) {
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("" : "+v"(v));
#endif
}

// Number `id` of `count` so that the ids that one XCD gets (id % 8, blocks are dealt out in turn) are consecutive numbers
__device__ __forceinline__ uint32_t by_xcd(uint32_t id, uint32_t count) {
    const uint32_t xcd = id % 8, each = count / 8, more = count % 8;
    return xcd * each + (xcd < more ? xcd : more) + id / 8;
}

// tile `t` of tiles_m x tiles_n: columns of `high` tiles, one column of tiles after the other, so that the tiles that are
// worked on side by side are about as many down as across and share their rows of A and B in an XCD's L2
__device__ __forceinline__ void tile_at(uint32_t t, uint32_t tiles_m, uint32_t tiles_n, uint32_t high, uint32_t& m, uint32_t& n) {
    const uint32_t band = t / (high * tiles_n), first = band * high, in = t - band * high * tiles_n;
    const uint32_t rows = tiles_m - first < high ? tiles_m - first : high;
    m = first + in % rows;
    n = in / rows;
}

// How the 16 blocks of 128 that a thread block covers lie in the matrix: 2^side_log2 of them side by side, the rest below
struct PackGrid {
    int64_t rows, cols;
    uint32_t nb;                            // blocks of 128 per row
    uint32_t side_log2;
};
// Rows whose loads a thread has under way before the first one's work: with 16 bytes per row and lane two are the better (unpack of
// 8192 x 4096 to bf16: 17.5 us with one, 16.2 with two, 16.5 with four), with 32 bytes one is (to fp32: 25.9, 28.7, 28.1).
constexpr int rows_ahead(size_t value_bytes) { return value_bytes == 4 ? 1 : 2; }
// load(u, row, block of the row, lane's first column), then work(..) of the same, for every block of 128, 16 lanes per block, all
// lanes of a block together
template <int ROWS, class L, class W>
__device__ __forceinline__ void for_blocks(const PackGrid& g, L load, W work) {
    const uint32_t item = threadIdx.x / 16, lane = threadIdx.x % 16;
    const uint32_t kb = (blockIdx.x << g.side_log2) + (item & ((1u << g.side_log2) - 1u));
    const uint32_t deep = (kPackThreads / 16) >> g.side_log2;      // rows per thread block and turn
    if (kb >= g.nb) return;
    const int64_t col = (int64_t)kb * kPackBlock + lane * kLaneVals;
    for (int64_t row = (int64_t)blockIdx.y * deep * ROWS + (item >> g.side_log2); row < g.rows; row += (int64_t)gridDim.y * deep * ROWS) {
#pragma unroll
        for (int u = 0; u < ROWS; ++u)
            if (row + u * deep < g.rows) load(u, row + u * deep, kb, col);
#pragma unroll
        for (int u = 0; u < ROWS; ++u)
            if (row + u * deep < g.rows) work(u, row + u * deep, kb, col);
    }
}
// the lane's values of a row of a dense matrix, 0 behind its end
template <class D>
__device__ __forceinline__ Eight<D> load_row(const typename D::T* p, int64_t left) {
    Eight<D> v;
    if (left >= kLaneVals) {
        v = load_eight<D>(p);
    } else {
#pragma unroll
        for (int j = 0; j < kLaneVals; ++j) v[j] = j < left ? p[j] : (typename D::T)0.0f;
    }
    return v;
}
template <class D>
__device__ __forceinline__ void store_row(typename D::T* p, int64_t left, const float (&v)[kLaneVals]) {
    if (left >= kLaneVals) store8<D>(p, v);
    else store_some<D>(p, (int)left, v);
}

template <class D>
__global__ __launch_bounds__(kPackThreads) void k_pack_rows(
        const typename D::T* __restrict__ x, int64_t stride, PackGrid g, uint8_t* __restrict__ codes, int64_t code_stride,
        uint8_t* __restrict__ scales, int64_t scale_stride) {
    constexpr int kRows = rows_ahead(sizeof(typename D::T));
    Eight<D> in[kRows];
    for_blocks<kRows>(g, [&](int u, int64_t row, uint32_t, int64_t col) { in[u] = load_row<D>(x + row * stride + col, g.cols - col); },
               [&](int u, int64_t row, uint32_t kb, int64_t col) {
        float v[kLaneVals];
#pragma unroll
        for (int j = 0; j < kLaneVals; ++j) v[j] = (float)in[u][j];
        const uint32_t s = scale_for(row_largest(top_of(v)));
        *reinterpret_cast<uint32x2*>(codes + row * code_stride + col) = encode8(v, inverse_scale(s));
        if (threadIdx.x % 16 == 0) scales[row * scale_stride + kb] = (uint8_t)s;
    });
}

// ---- f and f' of the layer's activation, in 32 bits -----------------------------------
// Written for the rate of the memory: some twenty operations per value, each function from one exponential and one reciprocal.
// FINE, for fp32 results: the exponentials' arguments are corrected for what their own rounding lost, as results would otherwise be off by |x| (GELU:
// x^2) 2^-24 far out; 16-bit ones are rounded to 2^-9 or 2^-12, more than that wherever the result is not 0.  (8192 x 4096 to fp32 with / without
// the correction, in us: unpack tanh 29.2 / 27.7, GELU 31.1 / 27.8, logistic and SiLU 28; activation gradients all 50, bound by HBM.)

// 2^(t + rest)
template <bool FINE>
__device__ __forceinline__ float exp2_of(float t, float rest) {
    const float e = __builtin_amdgcn_exp2f(t);                 // off by 2^-23, 0 for a result below 2^-126
    return FINE ? fmaf(e, rest * 0.69314718055994531f, e) : e;
}
// e^-a of an a >= 0
template <bool FINE>
__device__ __forceinline__ float exp_minus(float a) {
    constexpr float kLog2E = 1.44269504088896341f, kLog2EBehind = (float)(1.44269504088896341 - (double)kLog2E);
    if constexpr (FINE) a = a > 128.0f ? 128.0f : a;           // (an infinity has no remainder; a NaN stays)
    const float t = a * -kLog2E;
    return exp2_of<FINE>(t, FINE ? fmaf(a, -kLog2EBehind, fmaf(a, -kLog2E, -t)) : 0.0f);
}
__device__ __forceinline__ float reciprocal(float x) { return __builtin_amdgcn_rcpf(x); }                     // off by 2^-23
// 1 / (1 + e^-x), without cancellation at either end
template <bool FINE>
__device__ __forceinline__ float logistic(float x) {
    const float e = exp_minus<FINE>(fabsf(x)), r = reciprocal(1.0f + e);
    return x < 0.0f ? e * r : r;
}
// tanh x = (1 - e) / (1 + e) with e = exp(-2 |x|); below 1/4, where 1 - e cancels, the Taylor series to x^9 (the next term is 2^-26 there)
template <bool FINE>
__device__ __forceinline__ float tanh_of(float x) {
    const float e = exp_minus<FINE>(2.0f * fabsf(x)), far = copysignf((1.0f - e) * reciprocal(1.0f + e), x), s = x * x;
    float p = fmaf(s, 62.0f / 2835.0f, -17.0f / 315.0f);
    p = fmaf(s, p, 2.0f / 15.0f);
    p = fmaf(s, p, -1.0f / 3.0f);
    return fabsf(x) < 0.25f ? fmaf(x * s, p, x) : far;
}
// Phi(-|x|) = erfc(z) / 2 with z = |x| / sqrt 2, and e^(-x^2 / 2), as tail * bell.  For z >= 0, erfc(z) = e^(-z^2) t p(t) with
// t = 1 / (1 + 0.3 z); p has degree 8, fitted to erfc(z) e^(z^2) / t for z up to 10.5 with weights that level the relative error:
// 2^-24.3 in 64 bits, evaluated in fp32 at most 9e-7, that with the reciprocal a step off.  (p is halved here.)
template <bool FINE>
__device__ __forceinline__ float normal_tail(float x, float& bell) {
    constexpr double kPower = -0.72134752044448170;            // e^(-x^2 / 2) = 2^(kPower x^2)
    constexpr float kNear = (float)kPower, kBehind = (float)(kPower - (double)kNear);
    const float t = reciprocal(fmaf(0.3f * 0.70710678118654752f, fabsf(x), 1.0f));
    const float a = FINE && fabsf(x) > 16.0f ? 16.0f : x;      // (2^-184 there; a NaN stays)
    const float square = a * a, power = square * kNear;
    bell = exp2_of<FINE>(power, FINE ? fmaf(square, kBehind, fmaf(fmaf(a, a, -square), kNear, fmaf(square, kNear, -power))) : 0.0f);
    float p = -0.06477917730808258f;
    p = fmaf(p, t, 0.2428741753101349f);
    p = fmaf(p, t, -0.256346195936203f);
    p = fmaf(p, t, 0.2741190791130066f);
    p = fmaf(p, t, -0.04752312600612640f);
    p = fmaf(p, t, 0.10755722969770432f);
    p = fmaf(p, t, 0.07414228469133377f);
    p = fmaf(p, t, 0.0853620097041130f);
    p = fmaf(p, t, 0.08459369838237762f);
    return p * t;
}

// Values of 2^128 and more decode to infinities.  Where a factor falls to 0 far out (from |x| = 104 on at the latest), x beside it is cut off
// behind that, as an infinity times 0 is NaN.  (A NaN of x is in the other factor.)
constexpr float kFarOut = 1e4f;
__device__ __forceinline__ float near_size(float x) { return fminf(fabsf(x), kFarOut); }
__device__ __forceinline__ float near_value(float x) { return fminf(fmaxf(x, -kFarOut), kFarOut); }

// (a NaN gives NaN in every branch)
template <int ACT, bool FINE>
__device__ __forceinline__ float act_value(float x) {
    if constexpr (ACT == GTOPK_ACT_RELU) return x < 0.0f ? 0.0f : x;
    if constexpr (ACT == GTOPK_ACT_TANH) return tanh_of<FINE>(x);
    if constexpr (ACT == GTOPK_ACT_SIGMOID) return logistic<FINE>(x);
    if constexpr (ACT == GTOPK_ACT_SILU) return fmaxf(x, -kFarOut) * logistic<FINE>(x);
    if constexpr (ACT == GTOPK_ACT_GELU) {
        float bell;                                // x Phi(x) = max(x, 0) - |x| Phi(-|x|)
        const float tail = normal_tail<FINE>(x, bell);
        return fmaf(-near_size(x) * bell, tail, fmaxf(x, 0.0f));
    }
    return x;
}
template <int ACT, bool FINE>
__device__ __forceinline__ float act_slope(float x) {
    if constexpr (ACT == GTOPK_ACT_RELU) return x > 0.0f ? 1.0f : x <= 0.0f ? 0.0f : x;
    if constexpr (ACT == GTOPK_ACT_TANH) {         // 1 - tanh^2 = 4 e / (1 + e)^2
        const float e = exp_minus<FINE>(2.0f * fabsf(x)), r = reciprocal(1.0f + e);
        return 4.0f * e * r * r;
    }
    if constexpr (ACT == GTOPK_ACT_SIGMOID || ACT == GTOPK_ACT_SILU) {
        const float e = exp_minus<FINE>(fabsf(x)), r = reciprocal(1.0f + e), slope = e * r * r;
        return ACT == GTOPK_ACT_SIGMOID ? slope : fmaf(near_value(x), slope, x < 0.0f ? e * r : r);
    }
    if constexpr (ACT == GTOPK_ACT_GELU) {
        float bell;
        const float below = normal_tail<FINE>(x, bell) * bell;
        return fmaf(near_value(x) * 0.39894228040143268f, bell, x < 0.0f ? below : 1.0f - below);
    }
    return x == x ? 1.0f : x;
}

template <class D> constexpr bool kFine = sizeof(typename D::T) == 4;

template <class D, int ACT>
__global__ __launch_bounds__(kPackThreads) void k_unpack(
        const uint8_t* __restrict__ codes, int64_t code_stride, const uint8_t* __restrict__ scales, int64_t scale_stride,
        PackGrid g, typename D::T* __restrict__ out, int64_t stride) {
    constexpr int kRows = rows_ahead(sizeof(typename D::T));
    uint32x2 c[kRows];
    uint32_t s[kRows];
    for_blocks<kRows>(g, [&](int u, int64_t row, uint32_t kb, int64_t col) {
        c[u] = *reinterpret_cast<const uint32x2*>(codes + row * code_stride + col);
        s[u] = scales[row * scale_stride + kb];
    }, [&](int u, int64_t row, uint32_t, int64_t col) {
        float v[kLaneVals];
        decode8(c[u], scale_value(s[u]), v);
#pragma unroll
        for (int j = 0; j < kLaneVals; ++j) v[j] = act_value<ACT, kFine<D>>(v[j]);
        store_row<D>(out + row * stride + col, g.cols - col, v);
    });
}

// dx may be dy: a lane reads its values before it writes them, and nobody else touches them
template <class D, int ACT>
__global__ __launch_bounds__(kPackThreads) void k_activation_grad(
        const uint8_t* __restrict__ codes, int64_t code_stride, const uint8_t* __restrict__ scales, int64_t scale_stride,
        PackGrid g, const typename D::T* dy, int64_t dy_stride, typename D::T* dx, int64_t dx_stride) {
    constexpr int kRows = rows_ahead(sizeof(typename D::T));
    uint32x2 c[kRows];
    uint32_t s[kRows];
    Eight<D> in[kRows];
    for_blocks<kRows>(g, [&](int u, int64_t row, uint32_t kb, int64_t col) {
        in[u] = load_row<D>(dy + row * dy_stride + col, g.cols - col);
        c[u] = *reinterpret_cast<const uint32x2*>(codes + row * code_stride + col);
        s[u] = scales[row * scale_stride + kb];
    }, [&](int u, int64_t row, uint32_t, int64_t col) {
        float v[kLaneVals];
        decode8(c[u], scale_value(s[u]), v);
#pragma unroll
        for (int j = 0; j < kLaneVals; ++j) v[j] = (float)in[u][j] * act_slope<ACT, kFine<D>>(v[j]);
        store_row<D>(dx + row * dx_stride + col, g.cols - col, v);
    });
}

// One thread block per tile of 128 x 128.  Of the tile a thread holds rows 64 h + 16 wave + 4 (lane / 16) + (0 .. 3),
// h = 0, 1, and 8 columns: four rows, so that the transposed codes come out as whole words.
constexpr int kTilePitch = kPackBlock / 4 + 1;      // words per row of the transposed tile in LDS: one extra spreads the banks
template <class D>
__global__ __launch_bounds__(kPackThreads) void k_pack_tiles(
        const typename D::T* __restrict__ x, int64_t stride, int64_t rows, int64_t cols, uint8_t* __restrict__ codes,
        int64_t code_stride, uint8_t* __restrict__ scales, int64_t scale_stride, uint8_t* __restrict__ codes_t,
        int64_t code_t_stride, uint8_t* __restrict__ scales_t, int64_t scale_t_stride, uint32_t nbc, uint64_t tiles) {
    __shared__ uint32_t s_t[kPackBlock * kTilePitch];
    __shared__ uint32_t s_top[kPackThreads / kWave];
    const uint32_t wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    for (uint64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t tr = (int64_t)(tile / nbc), tc = (int64_t)(tile % nbc);
        const int64_t col = tc * kPackBlock + (lane % 16) * kLaneVals;
        const int64_t left = cols - col;
        float v[8][kLaneVals];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t row = tr * kPackBlock + (i / 4) * 64 + wave * 16 + (lane / 16) * 4 + i % 4;
            const typename D::T* p = x + row * stride + col;
            if (row < rows && left >= kLaneVals) load8<D>(p, v[i]);
            else load_some<D>(p, row < rows ? (int)left : 0, v[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t t = top_of(v[i]);
            top = t > top ? t : top;
        }
        top = wave_largest(top);
        if (lane == 0) s_top[wave] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPackThreads / kWave; ++i) top = s_top[i] > top ? s_top[i] : top;
        const uint32_t s = scale_for(top);
        const float inv = inverse_scale(s);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t row0 = tr * kPackBlock + h * 64 + wave * 16 + (lane / 16) * 4;
            uint32x2 c[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[i] = encode8(v[h * 4 + i], inv);
                if (codes && row0 + i < rows) *reinterpret_cast<uint32x2*>(codes + (row0 + i) * code_stride + col) = c[i];
            }
            if (codes_t) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {      // 4 x 4 bytes turned: word j holds column j of the four rows
                    const uint32_t ab02 = __builtin_amdgcn_perm(c[1][q], c[0][q], 0x06020400u), ab13 = __builtin_amdgcn_perm(c[1][q], c[0][q], 0x07030501u);
                    const uint32_t cd02 = __builtin_amdgcn_perm(c[3][q], c[2][q], 0x06020400u), cd13 = __builtin_amdgcn_perm(c[3][q], c[2][q], 0x07030501u);
                    uint32_t* t = s_t + ((lane % 16) * kLaneVals + q * 4) * kTilePitch + (h * 64 + wave * 16 + (lane / 16) * 4) / 4;
                    t[0] = __builtin_amdgcn_perm(cd02, ab02, 0x05040100u);
                    t[kTilePitch] = __builtin_amdgcn_perm(cd13, ab13, 0x05040100u);
                    t[2 * kTilePitch] = __builtin_amdgcn_perm(cd02, ab02, 0x07060302u);
                    t[3 * kTilePitch] = __builtin_amdgcn_perm(cd13, ab13, 0x07060302u);
                }
            }
        }
        // the scale of the tile, once for each of its rows, so that readers need not know about tiles
        if (codes && threadIdx.x < kPackBlock && tr * kPackBlock + threadIdx.x < rows)
            scales[(tr * kPackBlock + threadIdx.x) * scale_stride + tc] = (uint8_t)s;
        if (codes_t && threadIdx.x >= kPackBlock && tc * kPackBlock + (threadIdx.x - kPackBlock) < cols)
            scales_t[(tc * kPackBlock + (threadIdx.x - kPackBlock)) * scale_t_stride + tr] = (uint8_t)s;
        __syncthreads();
        if (codes_t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = i * 8 + threadIdx.x / 32, w = threadIdx.x % 32;
                const int64_t row = tc * kPackBlock + r;
                if (row < cols) *reinterpret_cast<uint32_t*>(codes_t + row * code_t_stride + tr * kPackBlock + w * 4) = s_t[r * kTilePitch + w];
            }
        }
        __syncthreads();                   // the next tile writes s_top and s_t
    }
}

}  // namespace gtopk
