// C = A B^T of two packed matrices:
//   C[m][n] = sum over blocks b of 2^(ea[m][b] + eb[n][b]) * (sum over k in b of a[m][k] * b[n][k])
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 codes and takes a power-of-two scale for
// every row of either operand, so one block of 128 is one instruction with its scales, and the sum over
// blocks stays in the fp32 accumulators.  A lane l gives 32 codes of row l % 16; which 32 of the 128 does not
// matter as long as both operands agree, and all four lanes of a row give the same scale.
#pragma once
#include <type_traits>

#include "packed.hip.h"

namespace gtopk {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef int intx4 __attribute__((ext_vector_type(4)));

// The instruction for e4m3 numbers lines up the eight products of consecutive k with the largest of them and keeps 13 bits
// below its leading one (measured: 2^-13 of it is added, 2^-14 lost; the sums of eight, and they with the accumulator, add
// as fp32 numbers).  On activations and weights that is 3e-5 to 7e-5 of the result in norm, where a 16-bit result's rounding is 2^-9 or 2^-12 at most (a
// sum that cancels loses more).  A result in fp32 is not rounded like that, so there the codes are decoded to bf16 numbers, which hold them and
// their scales exactly, and multiplied at half the rate by the instruction for those, which keeps 23 bits.  Without tiles (k_product_thin) all types are: reading
// B bounds the call (us, cut / exact, 1 x 4096 x 9216 9.94 / 9.86; 16 x 4096 x 9216 13.5 / 13.6; 32 x 4096 x 4096 10.1 / 10.3).  With tiles exact
// products would cost 16-bit results 10 to 90 % (64 x 4096 x 9216 17.2 / 24.0; 256 x 4096 x 4096 19.6 / 22.4; 2048 x 4096 x 9216 72 / 135).
template <class D> struct Exact { static constexpr bool value = false; };
template <> struct Exact<F32> { static constexpr bool value = true; };

struct PackedMatrix {
    const uint8_t* codes;
    const uint8_t* scales;
    uint32_t code_stride, scale_stride;     // bytes
};

// Bytes from `from` + offset + at into LDS, 16 or 4 per lane, lane l's to `to` + 16 l or 4 l (all but `offset` are uniform).  Buffer loads add
// the three by themselves; with a global load's address of 64 bits per lane the large tiles lose 4 % (8192^3 429 us, so 409).
typedef __amdgpu_buffer_rsrc_t Source;
__device__ __forceinline__ Source source(const uint8_t* from) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, (int)0xFFFFFFFFu, 0x00027000);     // bytes, up to 2^32 of them
}
__device__ __forceinline__ void load_to_lds16(Source from, uint32_t offset, uint32_t at, uint8_t* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, (int)offset, (int)at, 0, 0);
}
__device__ __forceinline__ void load_to_lds4(Source from, uint32_t offset, uint32_t at, uint8_t* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 4, (int)offset, (int)at, 0, 0);
}

// 8 codes as bf16 numbers, exactly
__device__ __forceinline__ bf16x8 decode_bf16(int c0, int c1, float scale) {
    uint32x4 u;
    u[0] = decode2<false>((uint32_t)c0, scale);
    u[1] = decode2<true>((uint32_t)c0, scale);
    u[2] = decode2<false>((uint32_t)c1, scale);
    u[3] = decode2<true>((uint32_t)c1, scale);
    return __builtin_bit_cast(bf16x8, u);
}

// A row's 32 codes of one block of 128 as the matrix instruction takes them, with the row's scale (the lowest byte of `scale`)
template <bool EXACT> struct Operand;
template <> struct Operand<false> { intx8 codes; uint32_t scale; };
template <> struct Operand<true> { bf16x8 values[4]; };
template <bool EXACT>
__device__ __forceinline__ Operand<EXACT> prepare(intx8 codes, uint32_t scale) {
    Operand<EXACT> x;
    if constexpr (EXACT) {
        const float f = scale_value(scale & 255u);
#pragma unroll
        for (int q = 0; q < 4; ++q) x.values[q] = decode_bf16(codes[2 * q], codes[2 * q + 1], f);
    } else {
        x.codes = codes;
        x.scale = scale;
    }
    return x;
}
// sum + one block of 128: B's row is the instruction's first operand, so a lane holds four consecutive columns of C
template <bool EXACT>
__device__ __forceinline__ floatx4 multiply(const Operand<EXACT>& b, const Operand<EXACT>& a, floatx4 sum) {
    if constexpr (EXACT) {
#pragma unroll
        for (int q = 0; q < 4; ++q) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.values[q], a.values[q], sum, 0, 0, 0);
        return sum;
    } else {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.codes, a.codes, sum, 0, 0, 0, (int)b.scale, 0, (int)a.scale);
    }
}

// `none` stays 0 while all values are finite: one operation each
__device__ __forceinline__ void note_lost(float& none, floatx4 v) {
#pragma unroll
    for (int r = 0; r < 4; ++r) none = fmaf(v[r], 0.0f, none);
}
// With a scale from 247 on a value may be 2^128 or more, which decodes to a bf16 infinity; a sum that it enters is not finite.  Such sums are computed
// once more with the scales of both rows applied together, to products of the bare codes, one block of 128 after the other as
// it lies in memory (2048 x 4096 x 9216 to fp32: a NaN in one row of A costs the look at the scales, 202 us instead of 150, such a scale there 390).  This adds
// one; 32 codes per lane at a and b, their rows' scales at a_scale and b_scale.  (A lane's four results are of B's
// rows 4 quarter .. 4 quarter + 3, whose scales lanes of those numbers have.)
__device__ __forceinline__ intx8 codes_at(const uint8_t* p) {
    const intx4 lo = *reinterpret_cast<const intx4*>(p), hi = *reinterpret_cast<const intx4*>(p + 16);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ floatx4 add_far(const uint8_t* b, uint32_t b_scale, const uint8_t* a, uint32_t a_scale, floatx4 sum) {
    const floatx4 part = multiply<true>(prepare<true>(codes_at(b), 127u), prepare<true>(codes_at(a), 127u), floatx4{});
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const uint32_t of_b = (uint32_t)__shfl((int)b_scale, (int)(lane_id() / 16 * 4) + r);
        sum[r] += a_scale == 255u || of_b == 255u ? __uint_as_float(0x7FC00000u) : __builtin_ldexpf(part[r], (int)(a_scale + of_b) - 254);
    }
    return sum;
}
// v, with those of its values that are not finite taken from `again`
__device__ __forceinline__ floatx4 mended(floatx4 v, floatx4 again) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = finite_bits(__float_as_uint(v[r])) ? v[r] : again[r];
    return v;
}

// A block computes BM x BN values with BM/WM x BN/WN waves of WM x WN each.  A block of 128 of the tile's rows of A and B
// goes straight from global memory into one of two LDS buffers while the matrix instructions work on the other; the scales
// of four blocks go together (a word per row: fetched one by one they would be as many requests as the codes).
// Tiles of 128 x 128 with four waves, two blocks per compute unit: 2048 x 4096 x 9216 to bf16 in 72 to 79 us = 2.0 to 2.1 PFLOP/s, 8192^3 in 509; to
// fp32 142 to 149 and 929.  What bounds them is the way into LDS: of 8192^3's 509 us the loads alone take 407, the matrix instructions
// alone 282, all but the loads 337.  Tiles of 256 x 256 with eight waves, one block per compute unit, need half the loads: 409 to 419 us = 2.6 to 2.7
// PFLOP/s, to fp32 773 to 792 = 1.4 (the matrix instructions of either type at 0.87 of what a library product of 8192^3 reaches).  (Calls in a row on the
// same buffers; by turns on buffers that no cache holds, 8192^3 447 and 786 us, 2048 x 4096 x 9216 92 and 146.)  Their waves read
// A 16 rows at a time, for the registers (kStream).  Slower: 256 x 128 with eight waves 80 us for the first size, with three LDS buffers
// 81; 256 x 256 with four waves 493 us for 8192^3; decoding B's rows for fp32 once per half block of A's 187 us for the first
// size, nothing gained with large tiles.
// In LDS a row's 16-byte pieces are exchanged by the row's number (piece p lies at p ^ (row / 2 % 8)): rows are 128
// bytes apart, and without that a wave's lanes would read from an eighth of the banks.  Rows behind the
// matrix's end are read as its last row and not written.  Grid: x the tiles, y shares of `share` blocks of 128 (a multiple of 4, or
// all of them), each written to a result of its own.
template <class D, bool EXACT, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * kWave, 1) void k_product(
        PackedMatrix a, PackedMatrix b, int64_t M, int64_t N, uint32_t blocks, typename D::T* __restrict__ out, int64_t out_stride,
        uint32_t tiles_m, uint32_t tiles_n, uint32_t share) {
    constexpr int kWavesN = BN / WN, kWaves = (BM / WM) * kWavesN, kThreads = kWaves * kWave;
    constexpr int TM = WM / 16, TN = WN / 16;
    constexpr bool kStream = TM > 4;         // A's rows are read 16 at a time, while the products of the ones before run
    constexpr int kScaleLoads = (BM + BN + kThreads - 1) / kThreads;
    constexpr int kStage = (BM + BN) * kPackBlock;
    constexpr int kLoads = kStage / 16 / kThreads;                 // 16-byte pieces per thread and stage
    static_assert(kStage % (16 * kThreads) == 0 && BM % (kThreads / 8) == 0, "whole loads, none of which has rows of both matrices");
    // arrays of their own, so that the compiler can tell a load into one from a read of another
    __shared__ __align__(128) uint8_t s_codes0[kStage];
    __shared__ __align__(128) uint8_t s_codes1[kStage];
    __shared__ __align__(128) uint8_t s_scales[2][kScaleLoads * kThreads * 4];      // a word per row: four blocks' scales

    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const uint32_t first = blockIdx.y * share, nb = blocks - first < share ? blocks - first : share;     // this share's blocks of 128
    out += blockIdx.y * M * out_stride;
    uint32_t tile_m, tile_n;
    tile_at(by_xcd(blockIdx.x, tiles_m * tiles_n), tiles_m, tiles_n, 2048 / BM, tile_m, tile_n);
    tile_m = __builtin_amdgcn_readfirstlane(tile_m);
    tile_n = __builtin_amdgcn_readfirstlane(tile_n);
    const int64_t m0 = (int64_t)tile_m * BM, n0 = (int64_t)tile_n * BN;
    const uint8_t* const a_base = a.codes + m0 * a.code_stride + (int64_t)first * kPackBlock;
    const uint8_t* const b_base = b.codes + n0 * b.code_stride + (int64_t)first * kPackBlock;
    const uint32_t a_last = (uint32_t)(M - m0 < BM ? M - m0 - 1 : BM - 1), b_last = (uint32_t)(N - n0 < BN ? N - n0 - 1 : BN - 1);

    const Source a_from = source(a_base), b_from = source(b_base);
    uint32_t offset[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const uint32_t r = (i * kThreads + threadIdx.x) / 8, piece = (threadIdx.x % 8) ^ (r / 2 % 8);
        const bool of_a = i * kThreads / 8 < BM;
        const uint32_t row = of_a ? (r < a_last ? r : a_last) : (r - BM < b_last ? r - BM : b_last);
        offset[i] = row * (of_a ? a.code_stride : b.code_stride) + piece * 16;
    }
    // a word of four scales per row (which can be read in fours to the end); a wave's rows are of one matrix
    Source scales_from[kScaleLoads];
    uint32_t scale_offset[kScaleLoads];
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        const uint32_t r = i * kThreads + threadIdx.x;
        const bool of_a = i * kThreads + wave * kWave < BM;
        scales_from[i] = source((of_a ? a.scales + m0 * a.scale_stride : b.scales + n0 * b.scale_stride) + first);  // (a multiple of 4)
        scale_offset[i] = of_a ? (r < a_last ? r : a_last) * a.scale_stride : (r - BM < b_last ? r - BM : b_last) * b.scale_stride;
    }
    auto fetch = [&](uint32_t kb, uint8_t* stage) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            load_to_lds16(i * kThreads / 8 < BM ? a_from : b_from, offset[i], kb * kPackBlock, stage + (i * kThreads + wave * kWave) * 16);
    };
    auto fetch_scales = [&](uint32_t kb, uint8_t* to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) load_to_lds4(scales_from[i], scale_offset[i], kb, to + (i * kThreads + wave * kWave) * 4);
    };

    const uint32_t wm = (wave / kWavesN) * WM, wn = (wave % kWavesN) * WN;
    const uint32_t in16 = lane % 16, quarter = lane / 16;
    // the lane's two pieces of a row (of which the subtiles' first row is a multiple of 16)
    const uint32_t piece0 = in16 * kPackBlock + ((2 * quarter) ^ (in16 / 2)) * 16, piece1 = in16 * kPackBlock + ((2 * quarter + 1) ^ (in16 / 2)) * 16;
    auto operand = [&](const uint8_t* stage, uint32_t row) __attribute__((always_inline)) {
        const uint8_t* p = stage + row * kPackBlock;
        const intx4 lo = *reinterpret_cast<const intx4*>(p + piece0), hi = *reinterpret_cast<const intx4*>(p + piece1);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    floatx4 sum[TM][TN] = {};
    uint32_t sa[TM], sb[TN];
    fetch(0, s_codes0);
    fetch_scales(0, s_scales[0]);
    auto block = [&](uint32_t kb, int in4, const uint8_t* here, uint8_t* free) __attribute__((always_inline)) {
        // what this wave fetched is in LDS (a barrier alone does not wait for loads into LDS), and behind the barrier what all did;
        // the other buffer has been read
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (in4 == 0) {
            const uint32_t* from = reinterpret_cast<const uint32_t*>(s_scales[kb / 4 % 2]);
#pragma unroll
            for (int i = 0; i < TM; ++i) sa[i] = from[wm + i * 16 + in16];
#pragma unroll
            for (int j = 0; j < TN; ++j) sb[j] = from[BM + wn + j * 16 + in16];
        }
        const uint32_t after = kb + 1 < nb ? kb + 1 : nb - 1, after_scales = kb + 1 < nb ? kb + 1 : kb & ~3u;
        if constexpr (kStream) {
            intx8 vb[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) vb[j] = operand(here, BM + wn + j * 16);
            intx8 va = operand(here, wm);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const intx8 va_next = i + 1 < TM ? operand(here, wm + (i + 1) * 16) : va;
                if (i == 0) fetch(after, free);
                if (in4 == 3 && i == TM - 1) fetch_scales(after_scales, s_scales[(kb + 1) / 4 % 2]);
                const Operand<EXACT> xa = prepare<EXACT>(va, sa[i] >> (8 * in4));
#pragma unroll
                for (int j = 0; j < TN; ++j) sum[i][j] = multiply<EXACT>(prepare<EXACT>(vb[j], sb[j] >> (8 * in4)), xa, sum[i][j]);
                va = va_next;
                // these products here and not behind the next reads: the compiler moves them as far down as it may
#pragma unroll
                for (int j = 0; j < TN; ++j) pin(sum[i][j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            intx8 va[TM], vb[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) vb[j] = operand(here, BM + wn + j * 16);
#pragma unroll
            for (int i = 0; i < TM; ++i) va[i] = operand(here, wm + i * 16);
            __builtin_amdgcn_sched_barrier(0);         // the loads behind the reads that the first products wait for
            fetch(after, free);
            if (in4 == 3) fetch_scales(after_scales, s_scales[(kb + 1) / 4 % 2]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) sum[i][j] = multiply<EXACT>(prepare<EXACT>(vb[j], sb[j] >> (8 * in4)), prepare<EXACT>(va[i], sa[i] >> (8 * in4)), sum[i][j]);
        }
    };
    for (uint32_t kb = 0; kb < nb; kb += 4) {
        block(kb, 0, s_codes0, s_codes1);
        if (kb + 1 < nb) block(kb + 1, 1, s_codes1, s_codes0);
        if (kb + 2 < nb) block(kb + 2, 2, s_codes0, s_codes1);
        if (kb + 3 < nb) block(kb + 3, 3, s_codes1, s_codes0);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // the last loads into LDS, which nobody reads, end before the block does
    float none = 0.0f;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + wm + i * 16 + in16;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = n0 + wn + j * 16 + quarter * 4;
            if constexpr (EXACT) note_lost(none, sum[i][j]);
            if (m < M && n < N) store4<D>(out + m * out_stride + n, N - n, sum[i][j]);
        }
    }
    if constexpr (EXACT) {
        if (!__ballot(none != 0.0f)) return;
        // (an infinity or a NaN: each subtile again, if a scale of its rows may be the cause)
        for (int t = 0; t < TM * TN; ++t) {
            const uint32_t row_a = wm + t / TN * 16 + in16, row_b = wn + t % TN * 16 + in16;
            const uint32_t ra = row_a < a_last ? row_a : a_last, rb = row_b < b_last ? row_b : b_last;
            const uint8_t *pa = a_base + (int64_t)ra * a.code_stride + quarter * 32, *pb = b_base + (int64_t)rb * b.code_stride + quarter * 32;
            const uint8_t *qa = a.scales + (m0 + ra) * a.scale_stride + first, *qb = b.scales + (n0 + rb) * b.scale_stride + first;
            bool far = false;
            for (uint32_t kb = quarter; kb < nb; kb += 4) far = far || (qa[kb] >= 247u && qa[kb] != 255u) || (qb[kb] >= 247u && qb[kb] != 255u);
            if (!__ballot(far)) continue;
            floatx4 again = {};
            for (uint32_t kb = 0; kb < nb; ++kb) again = add_far(pb + (uint64_t)kb * kPackBlock, qb[kb], pa + (uint64_t)kb * kPackBlock, qa[kb], again);
            const int64_t m = m0 + row_a, n = n0 + wn + t % TN * 16 + quarter * 4;
            if (m < M && n < N) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    typename D::T* const p = out + m * out_stride + n + r;
                    if (n + r < N && !finite_bits(__float_as_uint((float)*p))) *p = (typename D::T)again[r];
                }
            }
        }
    }
}

// Few rows of A (at most 16 TM): what counts is reading B once at the memory's rate (1 x 4096 x 9216: 38 MB in 9.1 to 9.8 us with the host's
// part of the call; 1 x 16384 x 9216: 151 MB in 30 us = 5.0 TB/s).  A block computes 16 columns of C
// with kThinWaves waves that share out the blocks of 128 among them and read both matrices straight into registers, kThinAhead
// blocks of 128 at a time, so that a compute unit has some 64 KB of B under way; the waves' sums are joined in LDS, in their order.
constexpr int kThinWaves = 8;
constexpr int kThinAhead = 4;
template <class D, int TM>
__global__ __launch_bounds__(kThinWaves * kWave) void k_product_thin(PackedMatrix a, PackedMatrix b, int64_t M, int64_t N, uint32_t nb,
                                                                   typename D::T* __restrict__ out, int64_t out_stride) {
    constexpr int kAhead = TM > 1 ? kThinAhead / 2 : kThinAhead;
    __shared__ floatx4 s_sum[kThinWaves][TM][kWave];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, in16 = lane % 16, quarter = lane / 16;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int64_t n = n0 + in16 < N ? n0 + in16 : N - 1;
    const uint8_t* const b_row = b.codes + n * b.code_stride + quarter * 32;
    const uint8_t* const b_scale = b.scales + n * b.scale_stride;
    const uint8_t *a_row[TM], *a_scale[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = i * 16 + in16 < M ? i * 16 + in16 : M - 1;
        a_row[i] = a.codes + m * a.code_stride + quarter * 32;
        a_scale[i] = a.scales + m * a.scale_stride;
    }
    floatx4 sum[TM] = {};
    for (uint32_t k0 = wave; k0 < nb; k0 += kThinWaves * kAhead) {
        intx8 va[kAhead][TM], vb[kAhead];
        uint32_t sa[kAhead][TM], sb[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {         // behind the last block the last one once more, which is not used
            const uint32_t kb = k0 + u * kThinWaves < nb ? k0 + u * kThinWaves : nb - 1;
            vb[u] = codes_at(b_row + (uint64_t)kb * kPackBlock);
            sb[u] = b_scale[kb];
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                va[u][i] = codes_at(a_row[i] + (uint64_t)kb * kPackBlock);
                sa[u][i] = a_scale[i][kb];
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (k0 + u * kThinWaves < nb) {
#pragma unroll
                for (int i = 0; i < TM; ++i) sum[i] = multiply<true>(prepare<true>(vb[u], sb[u]), prepare<true>(va[u][i], sa[u][i]), sum[i]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        float none = 0.0f;
        note_lost(none, sum[i]);
        if (__ballot(none != 0.0f)) {
            floatx4 again = {};
            for (uint32_t kb = wave; kb < nb; kb += kThinWaves)
                again = add_far(b_row + (uint64_t)kb * kPackBlock, b_scale[kb], a_row[i] + (uint64_t)kb * kPackBlock, a_scale[i][kb], again);
            sum[i] = mended(sum[i], again);
        }
        s_sum[wave][i][lane] = sum[i];
    }
    __syncthreads();
    for (int i = wave; i < TM; i += kThinWaves) {
        floatx4 v = s_sum[0][i][lane];
#pragma unroll
        for (int w = 1; w < kThinWaves; ++w) v += s_sum[w][i][lane];
        const int64_t m = i * 16 + in16, at = n0 + quarter * 4;
        if (m < M && at < N) store4<D>(out + m * out_stride + at, N - at, v);
    }
}

// the sum of the shares, in their order; their rows lie `stride` apart, a multiple of 4
template <class D>
__global__ __launch_bounds__(kPackThreads) void k_join_products(const float* __restrict__ part, uint32_t shares, int64_t share_stride,
                                                                int64_t stride, int64_t N, typename D::T* __restrict__ out, int64_t out_stride) {
    const float* from = part + blockIdx.y * stride;
    for (int64_t n = ((int64_t)blockIdx.x * kPackThreads + threadIdx.x) * 4; n < N; n += (int64_t)gridDim.x * kPackThreads * 4) {
        floatx4 v = *reinterpret_cast<const floatx4*>(from + n);
        for (uint32_t s = 1; s < shares; ++s) v += *reinterpret_cast<const floatx4*>(from + s * share_stride + n);
        store4<D>(out + blockIdx.y * out_stride + n, N - n, v);
    }
}

}  // namespace gtopk
