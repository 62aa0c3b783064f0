// Weight gradients of P workers from packed activations, into the workers' gradient rows:
//   dW_w[n][k] = sum over the rows t of worker w of dY[t][n] * X[t][k]
//
// The sum runs over the rows, and X's scales change from row to row, so X is decoded: an e4m3 number times a
// power of two is a bf16 number, exactly, and dY is one (bf16), the sum of two (fp16) or of three (fp32).  The
// products of bf16 numbers are exact and v_mfma_f32_16x16x32_bf16 adds them in fp32 (measured: terms down to 2^-23 of
// the largest are kept wherever they stand, where the instruction for e4m3 numbers keeps 2^-13 within eight).
#pragma once
#include "packed.hip.h"

namespace gtopk {

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));

// first and last + 1 row of worker w; whatever begin[] holds, 0 <= first <= last <= rows
__device__ __forceinline__ void rows_of_worker(const int32_t* begin, int64_t rows, uint32_t P, uint32_t w, int64_t& first, int64_t& last) {
    if (begin) {
        first = begin[w];
        last = begin[w + 1];
        first = first < 0 ? 0 : first > rows ? rows : first;
        last = last < first ? first : last > rows ? rows : last;
    } else {
        const int64_t each = rows / P;
        first = each * w;
        last = first + each;
    }
}

// a value as a sum of bf16 numbers: its leading 8 bits, the next 8, the last 8 (cut off, so that no part overflows)
template <class D> struct Parts;
template <> struct Parts<BF16> { static constexpr int n = 1; };
template <> struct Parts<F16> { static constexpr int n = 2; };
template <> struct Parts<F32> { static constexpr int n = 3; };

// bits of the parts of two values, packed: part[i] = low half from a, high half from b
template <int N>
__device__ __forceinline__ void split2(float a, float b, uint32_t (&part)[N]) {
    auto lead = [](float v) {
        const uint32_t u = __float_as_uint(v);
        return v != v ? u | 0x00400000u : u;        // NaN: the bit that is kept must not be 0
    };
    const bool fa = finite_bits(__float_as_uint(a)), fb = finite_bits(__float_as_uint(b));
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t ua = lead(a), ub = lead(b);
        part[i] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);
        a = fa ? a - __uint_as_float(ua & 0xFFFF0000u) : 0.0f;
        b = fb ? b - __uint_as_float(ub & 0xFFFF0000u) : 0.0f;
    }
}

// 16 codes as bf16 numbers, exactly
__device__ __forceinline__ void decode16(uint32x4 c, float scale, uint32x4& lo, uint32x4& hi) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        lo[2 * i] = decode2<false>(c[i], scale);
        lo[2 * i + 1] = decode2<true>(c[i], scale);
        hi[2 * i] = decode2<false>(c[2 + i], scale);
        hi[2 * i + 1] = decode2<true>(c[2 + i], scale);
    }
}

// What a block loads ahead: kRows rows of the tile's columns of dY and X.
constexpr int kGradRows = 32;

// A block computes BN x BK values of one worker (rows of dW from dY's columns, columns from X's) over all of its rows,
// or over one of `splits` equal shares of them, with waves of WN x WK.  kGradRows rows at a time lie in one of two LDS
// buffers while the next ones are on their way to registers.  In LDS both are bf16 with their rows as in
// memory; ds_read_b64_tr_b16 gives each lane four rows' values of one column, which is what the
// matrix instruction wants.  (Which 8 of the 32 rows a lane holds is free as long as both operands agree: the
// four groups of 16 lanes take rows 4 g .. 4 g + 3 and 16 + 4 g .. , so that with 8 words between the rows'
// banks 16 lanes' pieces of 32 bytes fall on all of them.)
template <class D, int BN, int BK, int WN, int WK>
__global__ __launch_bounds__((BN / WN) * (BK / WK) * kWave, 2) void k_weight_grad(
        const typename D::T* __restrict__ dy, int64_t dy_stride, const uint8_t* __restrict__ codes, int64_t code_stride,
        const uint8_t* __restrict__ scales, int64_t scale_stride, int64_t rows, const int32_t* __restrict__ begin, uint32_t P,
        int64_t N, int64_t K, float* __restrict__ grad, int64_t grad_stride, int accumulate, uint32_t splits, int64_t split_stride,
        uint32_t tiles_n, uint32_t tiles_k, uint32_t jobs) {
    constexpr int kParts = Parts<D>::n;
    constexpr int kWavesK = BK / WK, kThreads = (BN / WN) * kWavesK * kWave;
    constexpr int TN = WN / 16, TK = WK / 16;
    constexpr int kPitchD = BN + 16, kPitchX = BK + 16;                    // values; 8 words more than a multiple of the banks
    constexpr int kLoadsD = kGradRows * BN / 8 / kThreads, kLoadsX = kGradRows * BK / 16 / kThreads;
    static_assert(kLoadsD * kThreads * 8 == kGradRows * BN && kLoadsX * kThreads * 16 == kGradRows * BK, "whole loads");
    static_assert(BK % kPackBlock == 0, "a lane's 16 codes lie in one block of 128");
    __shared__ __align__(16) uint16_t s_d[2][kParts][kGradRows * kPitchD];
    __shared__ __align__(16) uint16_t s_x[2][kGradRows * kPitchX];

    const uint32_t wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const uint32_t wn = (wave / kWavesK) * WN, wk = (wave % kWavesK) * WK;
    for (uint32_t id = blockIdx.x; id < jobs; id += gridDim.x) {
        uint32_t job = id;
        const uint32_t tile_k = job % tiles_k;
        job /= tiles_k;
        const uint32_t tile_n = job % tiles_n;
        job /= tiles_n;
        const uint32_t split = job % splits, w = job / splits;
        const int64_t n0 = (int64_t)tile_n * BN, k0 = (int64_t)tile_k * BK;
        int64_t first, last;
        rows_of_worker(begin, rows, P, w, first, last);
        if (splits > 1) {                  // shares of whole steps
            const int64_t share = ((last - first + splits - 1) / splits + kGradRows - 1) / kGradRows * kGradRows;
            first = first + share * split < last ? first + share * split : last;
            last = first + share < last ? first + share : last;
        }
        const int32_t steps = (int32_t)((last - first + kGradRows - 1) / kGradRows);

        // this thread's pieces: 8 values of dY at column n_at of rows r, r + kThreads * 8 / BN, ..; 16 codes likewise
        const uint32_t n_at = threadIdx.x % (BN / 8) * 8, d_row = threadIdx.x / (BN / 8);
        const uint32_t k_at = threadIdx.x % (BK / 16) * 16, x_row = threadIdx.x / (BK / 16);
        const int64_t n_left = N - (n0 + n_at);
        const bool k_in = k0 + k_at < (K + kPackBlock - 1) / kPackBlock * kPackBlock;
        const typename D::T* d_from = dy + (first + d_row) * dy_stride + n0 + n_at;
        const uint8_t* x_from = codes + (first + x_row) * code_stride + k0 + k_at;
        const uint8_t* s_from = scales + (first + x_row) * scale_stride + (k0 + k_at) / kPackBlock;
        float d_next[kLoadsD][kLaneVals];
        uint32x4 x_next[kLoadsX];
        uint32_t s_next[kLoadsX];
        auto load = [&](int32_t step) {
            const int64_t left = last - first - (int64_t)step * kGradRows;     // rows from this step on
#pragma unroll
            for (int i = 0; i < kLoadsD; ++i) {
                const int r = d_row + i * (kThreads * 8 / BN);
                const typename D::T* p = d_from + ((int64_t)step * kGradRows + i * (kThreads * 8 / BN)) * dy_stride;
                if (r < left && n_left >= kLaneVals) load8<D>(p, d_next[i]);
                else load_some<D>(p, r < left ? (int)n_left : 0, d_next[i]);
            }
#pragma unroll
            for (int i = 0; i < kLoadsX; ++i) {
                const int r = x_row + i * (kThreads * 16 / BK);
                const int64_t at = (int64_t)step * kGradRows + i * (kThreads * 16 / BK);
                x_next[i] = uint32x4{0u, 0u, 0u, 0u};
                s_next[i] = 127u;
                if (r < left && k_in) {
                    x_next[i] = *reinterpret_cast<const uint32x4*>(x_from + at * code_stride);
                    s_next[i] = s_from[at * scale_stride];
                }
            }
        };
        auto stage = [&](int buf) {
#pragma unroll
            for (int i = 0; i < kLoadsD; ++i) {
                uint32x4 word[kParts];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t part[kParts];
                    split2(d_next[i][2 * j], d_next[i][2 * j + 1], part);
#pragma unroll
                    for (int q = 0; q < kParts; ++q) word[q][j] = part[q];
                }
#pragma unroll
                for (int q = 0; q < kParts; ++q)
                    *reinterpret_cast<uint32x4*>(s_d[buf][q] + (d_row + i * (kThreads * 8 / BN)) * kPitchD + n_at) = word[q];
            }
#pragma unroll
            for (int i = 0; i < kLoadsX; ++i) {
                uint32x4 lo, hi;
                decode16(x_next[i], scale_value(s_next[i]), lo, hi);
                uint32x4* to = reinterpret_cast<uint32x4*>(s_x[buf] + (x_row + i * (kThreads * 16 / BK)) * kPitchX + k_at);
                to[0] = lo;
                to[1] = hi;
            }
        };
        // eight rows' values of column `at` + lane % 16
        auto operand = [&](const uint16_t* from, int pitch, uint32_t at) {
            const uint16_t* p = from + (lane / 16 * 4 + lane % 16 / 4) * pitch + at + lane % 4 * 4;
            typedef __attribute__((address_space(3))) shortx4* Lds;
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + 16 * pitch));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        };

        floatx4 sum[TK][TN] = {};
        if (steps > 0) {
            load(0);
            stage(0);
            __syncthreads();
        }
        for (int32_t step = 0; step < steps; ++step) {
            const int buf = step % 2;
            if (step + 1 < steps) load(step + 1);
            bf16x8 x[TK];
#pragma unroll
            for (int i = 0; i < TK; ++i) x[i] = operand(s_x[buf], kPitchX, wk + i * 16);
#pragma unroll
            for (int q = 0; q < kParts; ++q) {
                bf16x8 d[TN];
#pragma unroll
                for (int j = 0; j < TN; ++j) d[j] = operand(s_d[buf][q], kPitchD, wn + j * 16);
#pragma unroll
                for (int i = 0; i < TK; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i], d[j], sum[i][j], 0, 0, 0);
            }
            if (step + 1 < steps) stage(buf ^ 1);
            __syncthreads();
        }
        // a lane holds four consecutive columns of a row of dW
        float* const to = grad + w * grad_stride + split * split_stride;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = n0 + wn + j * 16 + lane % 16;
            if (n >= N) continue;
#pragma unroll
            for (int i = 0; i < TK; ++i) {
                const int64_t k = k0 + wk + i * 16 + lane / 16 * 4;
                if (k >= K) continue;
                float* p = to + n * K + k;
                floatx4 v = sum[i][j];
                if (accumulate) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (k + r < K) v[r] = p[r] + v[r];
                }
                store4<F32>(p, K - k, v);
            }
        }
    }
}

// the sum of the shares, in their order
__global__ __launch_bounds__(kPackThreads) void k_join_shares(const float* __restrict__ part, uint32_t splits, int64_t split_stride,
                                                              int64_t part_stride, int64_t values, float* __restrict__ grad,
                                                              int64_t grad_stride, int accumulate) {
    const float* from = part + blockIdx.y * part_stride;
    float* to = grad + blockIdx.y * grad_stride;
    for (int64_t i = ((int64_t)blockIdx.x * kPackThreads + threadIdx.x) * 4; i < values; i += (int64_t)gridDim.x * kPackThreads * 4) {
        floatx4 v = *reinterpret_cast<const floatx4*>(from + i);       // the shares' rows are padded to fours
        for (uint32_t s = 1; s < splits; ++s) v += *reinterpret_cast<const floatx4*>(from + s * split_stride + i);
        if (accumulate) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (i + r < values) v[r] = to[i + r] + v[r];
        }
        store4<F32>(to + i, values - i, v);
    }
}

}  // namespace gtopk
