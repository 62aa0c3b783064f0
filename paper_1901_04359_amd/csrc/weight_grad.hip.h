// Weight gradients of P workers from packed activations, into the workers' gradient rows:
//   dW_w[n][k] = sum over the rows t of worker w of dY[t][n] * X[t][k]
//
// The sum runs over the rows, and X's scales change from row to row, so X is decoded: an e4m3 number times a
// power of two is a bf16 number, exactly, and dY is one (bf16), the sum of two (fp16) or of three (fp32).  The
// products of bf16 numbers are exact and v_mfma_f32_16x16x32_bf16 adds them in fp32 (measured: terms down to 2^-23 of
// the largest are kept wherever they stand, where the instruction for e4m3 numbers keeps 2^-13 within eight).
// An X of 2^128 or more decodes to an infinity, times which a part of dY that is 0 gives a NaN.  (Looking for sums that are not finite and computing
// them again, as products do, costs registers that writing needs: 16 workers, 64 rows each, 4096 x 9216 487 us, so 414.)
#pragma once
#include "packed.hip.h"

namespace gtopk {

typedef short shortx4 __attribute__((ext_vector_type(4)));

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

// the parts of 8 values, 8 numbers of 16 bits each
__device__ __forceinline__ void parts_of(Eight<BF16> v, uint32x4 (&part)[1]) { part[0] = __builtin_bit_cast(uint32x4, v); }
template <class T, int N>
__device__ __forceinline__ void parts_of(T v, uint32x4 (&part)[N]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        // (a signalling NaN, whose upper half may be that of an infinity, becomes a quiet one)
        float a = __builtin_canonicalizef((float)v[2 * j]), b = __builtin_canonicalizef((float)v[2 * j + 1]);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
            part[i][j] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);
            if (i + 1 < N) {
                a -= __uint_as_float(ua & 0xFFFF0000u);
                b -= __uint_as_float(ub & 0xFFFF0000u);
                if (i == 0) {              // behind an infinity nothing is left
                    a = finite_bits(ua) ? a : 0.0f;
                    b = finite_bits(ub) ? b : 0.0f;
                }
            }
        }
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

// two values (a word): the first n from block 0, the rest from block 1
__device__ __forceinline__ uint32_t two_blocks(uint32_t in0, uint32_t in1, int n) {
    return n >= 2 ? in0 : n <= 0 ? in1 : (in0 & 0xFFFFu) | (in1 & 0xFFFF0000u);
}

constexpr int kGradRows = 32;               // rows of dY and X in one step

// A block computes BN x BK values of one worker (rows of dW from dY's columns, columns from X's) over all of its rows,
// or over one of `splits` equal shares of them, with waves of WN x WK.  kGradRows rows at a time lie in one of two LDS
// buffers; the rows of the next two steps are on their way to registers.  In LDS both matrices are bf16 with their rows as in
// memory; ds_read_b64_tr_b16 gives each lane four rows' values of one column, which is what the
// matrix instruction wants.  (Which 8 of the 32 rows a lane holds is free as long as both operands agree: the
// four groups of 16 lanes take rows 4 g .. 4 g + 3 and 16 + 4 g .. , so that with 8 words between the rows'
// banks 16 lanes' pieces of 32 bytes fall on all of them.)
// Tiles of 128 x 128 with four waves: where workers have few rows, writing dW bounds the call, and three blocks per compute unit
// overlap one's stores with another's loads (16 workers, 64 rows each, 4096 x 9216: 2.4 GB, nearly all of it written, in 409 us =
// 6.0 TB/s; a fill writes 6.9).  Tiles of 128 x 256 with eight waves where they don't and dY is fp16 or fp32, as taking it apart is what costs there
// (half of the steps' vector instructions).  Tiles of 256 x 256 with eight waves for long sums in
// bf16: half the LDS traffic and loads per product (16384 rows, 4096 x 4096: 464 us = 1.18 PFLOP/s, with tiles of 128 677 us);
// there (kAhead) dY's columns are read, and the next rows staged, while the matrix instructions run (8192 rows, 8192 x 8192: 963 us,
// all reads before them 1026; 64 rows a step need more than the registers), also behind the last step, which would cost
// a quarter of the call where workers have two steps.
// LINES: K is a multiple of 32, so dW's rows all begin at the same place in a memory line, but a layer may lie anywhere in its
// worker's row.  Tiles that begin where lines do have whole lines to write, which go past the caches; a line written in two pieces
// by two blocks costs more than twice (4096 x 9216 from an odd place: 484 us without LINES).
template <class D, int BN, int BK, int WN, int WK, bool LINES>
__global__ __launch_bounds__((BN / WN) * (BK / WK) * kWave, BN * BK == 256 * 256 ? 1 : Parts<D>::n == 1 ? 3 : 2) void k_weight_grad(
        const typename D::T* __restrict__ dy, int64_t dy_stride, const uint8_t* __restrict__ codes, int64_t code_stride,
        const uint8_t* __restrict__ scales, int64_t scale_stride, int64_t rows, const int32_t* __restrict__ begin, uint32_t P,
        int64_t N, int64_t K, float* __restrict__ grad, int64_t grad_stride, int accumulate, uint32_t splits, int64_t split_stride,
        uint32_t tiles_n, uint32_t tiles_k, uint32_t band, uint32_t jobs) {
    constexpr int kParts = Parts<D>::n;
    constexpr int kWavesK = BK / WK, kThreads = (BN / WN) * kWavesK * kWave;
    constexpr int TN = WN / 16, TK = WK / 16;
    constexpr int kPitchD = BN + 16, kPitchX = BK + 16;                    // values; 8 words more than a multiple of the banks
    constexpr int kLoadsD = kGradRows * BN / 8 / kThreads, kLoadsX = kGradRows * BK / 16 / kThreads;
    static_assert(kLoadsD * kThreads * 8 == kGradRows * BN && kLoadsX * kThreads * 16 == kGradRows * BK, "whole loads");
    static_assert(BK % kPackBlock == 0, "a lane's 16 codes lie in one block of 128, or in two with LINES");
    constexpr bool kAhead = BN * BK == 256 * 256;
    constexpr int kPitchOut = WK + 4;                                      // floats
    static_assert((BN / WN) * kWavesK * 16 * kPitchOut * 2 <= 2 * kGradRows * (kParts * kPitchD + kPitchX), "the result's rows fit the same memory");
    __shared__ __align__(16) uint16_t s_rows[2 * kGradRows * (kParts * kPitchD + kPitchX)];
    uint16_t* const s_d = s_rows;                                          // [2][kParts][kGradRows][kPitchD]
    uint16_t* const s_x = s_rows + 2 * kParts * kGradRows * kPitchD;       // [2][kGradRows][kPitchX]

    const uint32_t wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const uint32_t wn = (wave / kWavesK) * WN, wk = (wave % kWavesK) * WK;
    for (uint32_t id = blockIdx.x; id < jobs; id += gridDim.x) {
        // Equal shares: an XCD gets whole workers, whose rows then lie in its L2 (TB/s with 64 rows of every worker, whole / spread out:
        // 4096 x 1024 5.9 / 5.5, 1000 x 4096 5.8 / 5.3, 4096 x 9217 4.9 / 4.6, larger ones alike).  Uneven ones: every worker's tiles are
        // spread over all XCDs (the shares of 1501 rows by seven random cuts, 1000 x 4096 in fp32, tiles of 128: 76 us, by XCD 167).
        const uint32_t tiles = tiles_n * tiles_k, spread = begin ? tiles * splits : jobs, at = id / spread * spread;
        uint32_t job = at + by_xcd(id - at, spread);
        uint32_t tile_n, tile_k;
        tile_at(job % tiles, tiles_k, tiles_n, band, tile_k, tile_n);
        job /= tiles;
        const uint32_t split = job % splits, w = job / splits;
        float* const to = grad + w * grad_stride + split * split_stride;
        // (LINES: the tile's columns start where a memory line of dW's rows does, up to 31 columns before a block of 128)
        const int64_t n0 = (int64_t)tile_n * BN, k0 = (int64_t)tile_k * BK - (LINES ? (int64_t)((uintptr_t)to / 4 % 32) : 0);
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
        const int64_t k_first = k0 + k_at, k_end = (K + kPackBlock - 1) / kPackBlock * kPackBlock;
        const bool k_in = LINES ? k_first > -16 && k_first < k_end : k_first < k_end, k_whole = !LINES || (k_first >= 0 && k_first + 16 <= k_end);
        // (LINES: 16 codes may lie in two blocks of 128, the first `k_cut` in the first one)
        const int64_t block0 = LINES && k_first < 0 ? 0 : k_first / kPackBlock;
        const uint32_t block1 = !LINES || k_first + 15 >= k_end ? 0u : (uint32_t)((k_first + 15) / kPackBlock - block0);
        const int k_cut = block1 ? (int)((block0 + 1) * kPackBlock - k_first) : 16;
        const typename D::T* d_from = dy + (first + d_row) * dy_stride + n0 + n_at;
        const uint8_t* x_from = codes + (first + x_row) * code_stride + k_first;
        const uint8_t* s_from = scales + (first + x_row) * scale_stride + block0;
        int32_t left = (int32_t)(last - first);    // rows that have not been loaded
        // two steps' rows on their way, as they lie in memory: taken apart when they are staged
        Eight<D> d_next[2][kLoadsD];
        uint32x4 x_next[2][kLoadsX];
        uint32_t s_next[2][kLoadsX];
        auto load = [&](int set) __attribute__((always_inline)) {      // the next step's rows
#pragma unroll
            for (int i = 0; i < kLoadsD; ++i) {
                const bool in = (int)d_row + i * (kThreads * 8 / BN) < left;
                const typename D::T* p = d_from + i * (kThreads * 8 / BN) * dy_stride;
                if (in && n_left >= kLaneVals) {
                    d_next[set][i] = load_eight<D>(p);
                } else {
#pragma unroll
                    for (int j = 0; j < kLaneVals; ++j) d_next[set][i][j] = in && j < n_left ? p[j] : (typename D::T)0.0f;
                }
            }
#pragma unroll
            for (int i = 0; i < kLoadsX; ++i) {
                x_next[set][i] = uint32x4{0u, 0u, 0u, 0u};
                s_next[set][i] = 127u;
                if ((int)x_row + i * (kThreads * 16 / BK) < left && k_in) {
                    const uint8_t* p = x_from + i * (kThreads * 16 / BK) * code_stride;
                    const uint8_t* q = s_from + i * (kThreads * 16 / BK) * scale_stride;
                    if (k_whole) {
                        struct __attribute__((packed)) Loose { uint32x4 v; };
                        x_next[set][i] = LINES ? reinterpret_cast<const Loose*>(p)->v : *reinterpret_cast<const uint32x4*>(p);
                    } else {               // at a row's ends: what lies outside the row is not read
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (k_first + e >= 0 && k_first + e < k_end) x_next[set][i][e / 4] |= (uint32_t)p[e] << (e % 4 * 8);
                    }
                    s_next[set][i] = LINES ? q[0] | (uint32_t)q[block1] << 8 : q[0];
                }
            }
            d_from += kGradRows * dy_stride;
            x_from += kGradRows * code_stride;
            s_from += kGradRows * scale_stride;
            left -= kGradRows;
        };
        auto stage = [&](int buf, int set) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kLoadsD; ++i) {
                uint32x4 word[kParts];
                parts_of(d_next[set][i], word);
#pragma unroll
                for (int q = 0; q < kParts; ++q)
                    *reinterpret_cast<uint32x4*>(s_d + ((buf * kParts + q) * kGradRows + d_row + i * (kThreads * 8 / BN)) * kPitchD + n_at) = word[q];
            }
#pragma unroll
            for (int i = 0; i < kLoadsX; ++i) {
                uint32x4 lo, hi;
                decode16(x_next[set][i], scale_value(LINES ? s_next[set][i] & 255u : s_next[set][i]), lo, hi);
                if (LINES && k_cut < 16) {
                    uint32x4 lo1, hi1;
                    decode16(x_next[set][i], scale_value(s_next[set][i] >> 8), lo1, hi1);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        lo[e] = two_blocks(lo[e], lo1[e], k_cut - 2 * e);
                        hi[e] = two_blocks(hi[e], hi1[e], k_cut - 8 - 2 * e);
                    }
                }
                uint32x4* to = reinterpret_cast<uint32x4*>(s_x + (buf * kGradRows + x_row + i * (kThreads * 16 / BK)) * kPitchX + k_at);
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
        auto step_at = [&](int32_t step, int buf) __attribute__((always_inline)) {
            bf16x8 x[TK];
#pragma unroll
            for (int i = 0; i < TK; ++i) x[i] = operand(s_x + buf * kGradRows * kPitchX, kPitchX, wk + i * 16);
            if constexpr (kAhead) {
                // dY's columns are read 16 at a time, while the products of the ones before run
                static_assert(!kAhead || (kParts == 1 && TN > 4), "one part; columns to stage and to load beside");
                const uint16_t* const in_d = s_d + buf * kGradRows * kPitchD;
                bf16x8 d = operand(in_d, kPitchD, wn);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const bf16x8 d_next_column = j + 1 < TN ? operand(in_d, kPitchD, wn + (j + 1) * 16) : d;
                    if (j == 2) stage(buf ^ 1, buf ^ 1);
                    if (j == 4) load(buf ^ 1);
#pragma unroll
                    for (int i = 0; i < TK; ++i) sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i], d, sum[i][j], 0, 0, 0);
                    d = d_next_column;
                    // these products here and not behind the next reads
#pragma unroll
                    for (int i = 0; i < TK; ++i) pin(sum[i][j]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
#pragma unroll
                for (int q = 0; q < kParts; ++q) {
                    bf16x8 d[TN];
#pragma unroll
                    for (int j = 0; j < TN; ++j) d[j] = operand(s_d + (buf * kParts + q) * kGradRows * kPitchD, kPitchD, wn + j * 16);
#pragma unroll
                    for (int i = 0; i < TK; ++i)
#pragma unroll
                        for (int j = 0; j < TN; ++j) sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i], d[j], sum[i][j], 0, 0, 0);
                }
                if (step + 1 < steps) {
                    stage(buf ^ 1, buf ^ 1);
                    load(buf ^ 1);         // (rows behind the last one are not read)
                }
            }
            __syncthreads();
        };
        if (steps > 0) {
            load(0);
            load(1);
            stage(0, 0);
            load(0);
            __syncthreads();
        }
        int32_t step = 0;
        for (; step + 2 <= steps; step += 2) {
            step_at(step, 0);
            step_at(step + 1, 1);
        }
        if (step < steps) step_at(step, 0);
        // A lane holds four consecutive columns of a row of dW, and a wave's store would write pieces of 64 bytes of 16 rows; by way
        // of LDS (each wave its own part, 16 rows at a time) it writes 4 WK bytes of a row at a stretch.
        float* const s_out = reinterpret_cast<float*>(s_rows) + wave * 16 * kPitchOut;
        constexpr int kAcross = WK / 4;        // lanes per row
#pragma unroll
        for (int j = 0; j < TN; ++j) {
#pragma unroll
            for (int i = 0; i < TK; ++i) *reinterpret_cast<floatx4*>(s_out + lane % 16 * kPitchOut + i * 16 + lane / 16 * 4) = sum[i][j];
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int r = 0; r < 16; r += kWave / kAcross) {
                const int row = r + lane / kAcross, col = lane % kAcross * 4;
                floatx4 v = *reinterpret_cast<const floatx4*>(s_out + row * kPitchOut + col);
                const int64_t n = n0 + wn + j * 16 + row, k = k0 + wk + col;
                if (n >= N || k >= K) continue;
                float* p = to + n * K + k;
                if constexpr (LINES) {
                    const int64_t line = k - col % 32;
                    if (line >= 0 && line + 32 <= K) {         // a whole line: past the caches
                        floatx4* const q = reinterpret_cast<floatx4*>(p);
                        if (accumulate) v = *q + v;
                        __builtin_nontemporal_store(v, q);
                    } else {                   // the lines that two rows share
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (k + e >= 0 && k + e < K) p[e] = accumulate ? p[e] + v[e] : v[e];
                    }
                } else {
                    if (accumulate) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (k + e < K) v[e] = p[e] + v[e];
                    }
                    store4<F32>(p, K - k, v);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (id + gridDim.x < jobs) __syncthreads();        // the next job's rows go where the result's were
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
