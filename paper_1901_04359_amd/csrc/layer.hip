// What lies before the hot path in an iteration (Algorithm 4 lines 2-3, where the gradients come from): a layer's
// activations packed to 8 bits, the products that read them, and the weight gradients of P workers written into
// the gradient rows that gtopk_step takes.  The C ABI's side of packed.hip.h, product.hip.h and weight_grad.hip.h.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "gtopk.h"
#include "common.hip.h"
#include "packed.hip.h"
#include "product.hip.h"
#include "weight_grad.hip.h"

using namespace gtopk;

namespace {

constexpr int64_t kMaxSide = 0x7FFFFFFF;            // rows and columns of a matrix
constexpr int64_t kMaxCodeStride = 1 << 23;         // of a product's operands (also of their scales): a tile's rows at offsets of 32 bits
constexpr int64_t kMaxTiles = (1 << 24) - 1;        // of 128 x 128 in a product: fewer than 2^32 threads in a launch
constexpr int64_t kMaxThinColumns = 1 << 26;
constexpr uint64_t kMaxBlocks = 1u << 22;           // blocks of a launch; kernels walk what is left

inline bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline uint32_t grid_for(uint64_t jobs) { return (uint32_t)(jobs < kMaxBlocks ? jobs : kMaxBlocks); }
inline int launch_status() { return hipGetLastError() == hipSuccess ? GTOPK_OK : GTOPK_EHIP; }
inline size_t value_bytes(int32_t dtype) { return dtype == GTOPK_F32 ? 4 : 2; }
inline int value_parts(int32_t dtype) { return dtype == GTOPK_BF16 ? 1 : dtype == GTOPK_F16 ? 2 : 3; }
inline bool dtype_ok(int32_t dtype) { return dtype == GTOPK_F32 || dtype == GTOPK_BF16 || dtype == GTOPK_F16; }
inline bool act_ok(int32_t act) { return act >= GTOPK_ACT_NONE && act <= GTOPK_ACT_GELU; }
inline bool side_ok(int64_t n, int64_t least) { return n >= least && n <= kMaxSide; }
inline bool packed_strides_ok(int64_t cols, int64_t code_stride, int64_t scale_stride) {
    const int64_t nb = ceil_div(cols, kPackBlock);
    return code_stride >= nb * kPackBlock && code_stride % kPackBlock == 0 && scale_stride >= nb && scale_stride % 4 == 0;
}
inline bool packed_aligned(const uint8_t* codes, const uint8_t* scales) { return aligned(codes, 16) && aligned(scales, 4); }

// calls launch(F32{}), launch(BF16{}) or launch(F16{})
template <class L>
void by_type(int32_t dtype, L launch) {
    if (dtype == GTOPK_F32) launch(F32{});
    else if (dtype == GTOPK_BF16) launch(BF16{});
    else launch(F16{});
}

// calls launch(std::integral_constant<int, act>{})
template <class L>
void by_act(int32_t act, L launch) {
    switch (act) {
        case GTOPK_ACT_RELU: return launch(std::integral_constant<int, GTOPK_ACT_RELU>{});
        case GTOPK_ACT_TANH: return launch(std::integral_constant<int, GTOPK_ACT_TANH>{});
        case GTOPK_ACT_SIGMOID: return launch(std::integral_constant<int, GTOPK_ACT_SIGMOID>{});
        case GTOPK_ACT_SILU: return launch(std::integral_constant<int, GTOPK_ACT_SILU>{});
        case GTOPK_ACT_GELU: return launch(std::integral_constant<int, GTOPK_ACT_GELU>{});
        default: return launch(std::integral_constant<int, GTOPK_ACT_NONE>{});
    }
}

PackGrid pack_grid(int64_t rows, int64_t cols, int32_t dtype, dim3* grid) {
    PackGrid g;
    g.rows = rows;
    g.cols = cols;
    g.nb = (uint32_t)ceil_div(cols, kPackBlock);
    g.side_log2 = 0;
    while (g.side_log2 < 4 && (1u << g.side_log2) < g.nb) ++g.side_log2;
    const int64_t deep = ((kPackThreads / 16) >> g.side_log2) * rows_ahead(value_bytes(dtype)), down = ceil_div(rows, deep);
    *grid = dim3((uint32_t)ceil_div(g.nb, 1 << g.side_log2), (uint32_t)(down < 65535 ? down : 65535));
    return g;
}

// How a product is computed: few rows of A without tiles, else tiles of 128 x 128, and where they are too few for the
// chip's 256 compute units (two blocks each), shares of K, joined from the workspace.
struct ProductPlan {
    bool thin, large;                               // large: tiles of 256 x 256, one block per compute unit
    uint32_t tiles_m, tiles_n, share, shares;       // blocks of 128 per share
    int64_t stride;                                 // of a share's result
};
// (us, without tiles / with, where 16-bit results lose bits: 32 x 4096 x 9216 16.1 / 15.5; 17 rows 12.9 / 15.0; 64 rows 24.6 / 16.9)
constexpr int64_t kThinRows = 32;
// blocks of 128 per share, at least; a multiple of 4.  (us with 4, 8, 16: 128 x 4096 x 4096 17.5, 15.2, 17.6; 1024^3 12.7, 9.2, 9.2;
// 64 x 4096 x 9216 16.9, 16.9, 22.1; 512 x 1000 x 4096 16.2, 15.5, 17.4, and 22.9 in one piece)
constexpr uint32_t kProductShare = 8;
ProductPlan product_plan(int64_t M, int64_t N, int64_t K) {
    ProductPlan g;
    const uint32_t nb = (uint32_t)ceil_div(K, kPackBlock);
    g.thin = M <= kThinRows;
    g.tiles_m = (uint32_t)ceil_div(M, 128);
    g.tiles_n = (uint32_t)ceil_div(N, 128);
    g.stride = ceil_div(N, 4) * 4;
    // A round of large tiles over the chip takes 1.67 times as long as one of small ones, two to a compute unit, and does twice as much (us,
    // small / large: 8192^3 509 / 409; 4096^3 71 / 57; 8187 x 9216 x 4096 305 / 272, to fp32 538 / 494; 2048 x 4096 x 9216, half a round of large
    // ones, 72 / 111).
    const uint64_t tiles_large = (uint64_t)ceil_div(M, 256) * ceil_div(N, 256);
    g.large = !g.thin && 5 * ((tiles_large + 255) / 256) < 3 * (((uint64_t)g.tiles_m * g.tiles_n + 511) / 512);
    g.share = nb;
    g.shares = 1;
    if (g.large) {
        g.tiles_m = (uint32_t)ceil_div(M, 256);
        g.tiles_n = (uint32_t)ceil_div(N, 256);
        return g;
    }
    const uint64_t tiles = (uint64_t)g.tiles_m * g.tiles_n;
    uint64_t want = g.thin || tiles == 0 ? 1 : 512 / tiles;
    if (want > nb / kProductShare) want = nb / kProductShare;
    g.share = want > 1 ? (uint32_t)ceil_div(ceil_div(nb, (int64_t)want), 4) * 4 : nb;
    g.shares = (uint32_t)ceil_div(nb, g.share);
    return g;
}

// How the weight gradient's sums are cut: tiles of every worker's gradient, and where they are too few for the chip's 256 compute
// units, shares of the rows, joined from the workspace.
struct GradPlan {
    bool big;                           // tiles of 256 x 256, one block per compute unit; else 128 x 128, two or three
    uint32_t tiles_n, tiles_k, splits;
    int64_t part_stride;                // values of one worker's share
    uint64_t jobs;
};
constexpr uint64_t kMaxJobs = 0x3FFFFFFF;
constexpr int64_t kGradShareRows = 256, kGradShareRowsBig = 1024;   // rows of a share, at least
constexpr int64_t kGradRowsBig = 512;                               // rows of a worker from which on large tiles are weighed
// Tiles across in a band (tile_at) where products bound the call and L2 has to hold dY and X.  Whole rows of tiles where writing does, or
// where two tiles write one memory line.  (us, 2 / 4 / 8 / 16 / whole rows.  fp32, tiles of 128 x 256: 8192 rows, 8192 x 8192 2877 / 2818 / 2810 / 2831 /
// 2879; four workers of 2048 rows, 4096 x 4096 747 / 730 / 752 / 754 / 758.  bf16, large tiles, the same two: 1005 / 984 / 972 / 961 / 973; 292 / 273 /
// 285 / 286 / 284.)
constexpr uint32_t kGradBand = 4;
GradPlan grad_plan_of(bool big, int64_t rows, int32_t P, int64_t N, int64_t K) {
    GradPlan g;
    const int64_t side = big ? 256 : 128;
    g.big = big;
    g.tiles_n = (uint32_t)ceil_div(N, side);
    g.tiles_k = (uint32_t)ceil_div(K, side);
    const uint64_t blocks = (uint64_t)g.tiles_n * g.tiles_k * (uint64_t)P;
    const int64_t most = rows / P / (big ? kGradShareRowsBig : kGradShareRows), want = (int64_t)((big ? 256 : 512) / blocks);
    g.splits = (uint32_t)(want < most ? want : most);
    if (g.splits < 1) g.splits = 1;
    g.part_stride = ceil_div(N * K, 4) * 4;
    g.jobs = blocks * g.splits;
    return g;
}
// Large tiles in bf16 (an fp16 or fp32 dY's two or three parts do not fit the registers beside their sums).
// Without shares: a round of large tiles over the chip takes as long as 3.5 small ones per compute unit (us with 2048 rows: 70 a round; small ones
// 96, 108, 124, 147, 165, 181, 239 with 4, 5, 6, 7, 8, 9, 12 per compute unit), with fewer rows somewhat longer.  (small / large, 512 and 2048 rows: 4096
// x 4096 35 / 30 and 97 / 70; 5120 x 5120 52 / 52 and 147 / 132; 4096 x 5120 39 / 51 and 108 / 136; 4096 x 9216 67 / 82 and 182 / 207; 8192 x 8192
// 108 / 112 and 316 / 289; 256 rows of 16 workers, 4096 x 4096 307 / 338.)
// In shares: from 1024 rows per share on, if they keep three quarters of the chip at work; from 2048 on if small ones need no shares.  (One worker, rows per large
// share: 1024 x 1024 512: 39 / 42, 1024: 59 / 55; 2048 x 2048 512: 41 / 43, 1024: 62 / 57; 2048 x 4096 1024: 52 / 60, 2048: 95 / 87; 4 workers, 1024 x 1024
// 512: 40 / 43, 1024: 61 / 57.)
GradPlan grad_plan(bool bf16, int64_t rows, int32_t P, int64_t N, int64_t K) {
    const GradPlan small = grad_plan_of(false, rows, P, N, K);
    if (!bf16 || rows / P < kGradRowsBig) return small;
    const GradPlan large = grad_plan_of(true, rows, P, N, K);
    const bool gain = large.splits == 1 ? 7 * ((large.jobs + 255) / 256) <= 2 * ((small.jobs + 255) / 256)
                                        : large.jobs >= 192 && (small.splits > 1 || rows / P / large.splits >= 2 * kGradShareRowsBig);
    return gain ? large : small;
}

// Tiles that begin where memory lines do and write them past the caches (LINES), `aligned`: every row of dW begins with a line; else the last of up to 31
// more columns.  They need rows of whole lines (K a multiple of 32), and pay where writing bounds the call (rows times the parts of a dY value) and
// the result is more than the 256 MB of the memory-side cache hold.  (us, without / with LINES, workers x N x K, rows of every worker, in bf16 unless
// stated.  Aligned: 16 x 2048 x 2048 64: 58 / 51, 256: 100 / 79, 384: 117 / 115; fp32 64: 75 / 69, 86: 85 / 89, 128: 97 / 101; fp16 128: 82 / 81, 192: 95 /
// 106; 256 x 512 x 512 64: 70 / 54; half of it and less, 8 x 2048 x 2048 64: 29.5 / 29.4, 256: 40 / 42; 8 x 1000 x 4096 64: 30 / 32.
// Not aligned: 4 x 4096 x 9216 64: 130 / 117, 128: 169 / 138, 384: 266 / 274; 32 x 2048 x 2048 64: 133 / 108, 128: 154 / 136; 64 x 1024 x 1024 64: 67 /
// 64, 128: 84 / 82, 256: 107 / 117; 512 x 512 x 512 64: 156 / 141, 128: 179 / 184, 256: 217 / 301; 8 x 1000 x 4096 64: 30 / 36; fp32 16 x 4096 x 4096
// 22: 263 / 222, 43: 302 / 293; 4 x 4096 x 9216 22: 136 / 124, 43: 154 / 162; 16 x 2048 x 2048 22: 64 / 66; fp16 24 x 1000 x 4096 32: 89 / 85, 64: 105 / 109.)
constexpr int64_t kGradWriteRows = 256;
bool grad_lines(int parts, int64_t rows_each, int32_t P, int64_t N, int64_t K, bool aligned) {
    if (K % 32 != 0 || rows_each * parts > kGradWriteRows || P * N < ((1 << 26) + K - 1) / K) return false;
    return aligned || (parts == 1 ? rows_each <= 128 && K >= 1024 : rows_each * parts <= 64 && K >= 4096);
}

}  // namespace

extern "C" {

int gtopk_pack_rows(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t stride, uint8_t* codes,
                    int64_t code_stride, uint8_t* scales, int64_t scale_stride, void* stream) {
    if (!dtype_ok(dtype) || !side_ok(rows, 0) || !side_ok(cols, 1) || stride < cols) return GTOPK_EINVAL;
    if (!packed_strides_ok(cols, code_stride, scale_stride)) return GTOPK_EINVAL;
    if (rows == 0) return GTOPK_OK;
    if (!x || !codes || !scales) return GTOPK_EINVAL;
    if (!aligned(x, value_bytes(dtype)) || !packed_aligned(codes, scales)) return GTOPK_EALIGN;
    dim3 grid;
    const PackGrid g = pack_grid(rows, cols, dtype, &grid);
    by_type(dtype, [&](auto d) {
        using D = decltype(d);
        hipLaunchKernelGGL(k_pack_rows<D>, grid, dim3(kPackThreads), 0, (hipStream_t)stream, (const typename D::T*)x, stride, g,
                           codes, code_stride, scales, scale_stride);
    });
    return launch_status();
}

int gtopk_pack_tiles(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t stride, uint8_t* codes,
                     int64_t code_stride, uint8_t* scales, int64_t scale_stride, uint8_t* codes_t, int64_t code_t_stride,
                     uint8_t* scales_t, int64_t scale_t_stride, void* stream) {
    if (!dtype_ok(dtype) || !side_ok(rows, 0) || !side_ok(cols, 1) || stride < cols) return GTOPK_EINVAL;
    if (rows == 0) return GTOPK_OK;
    if (!x || (!codes && !codes_t) || (codes == nullptr) != (scales == nullptr) || (codes_t == nullptr) != (scales_t == nullptr))
        return GTOPK_EINVAL;
    if ((codes && !packed_strides_ok(cols, code_stride, scale_stride)) || (codes_t && !packed_strides_ok(rows, code_t_stride, scale_t_stride)))
        return GTOPK_EINVAL;
    if (!aligned(x, value_bytes(dtype)) || !packed_aligned(codes, scales) || !packed_aligned(codes_t, scales_t)) return GTOPK_EALIGN;
    const uint32_t nbc = (uint32_t)ceil_div(cols, kPackBlock);
    const uint64_t tiles = (uint64_t)ceil_div(rows, kPackBlock) * nbc;
    by_type(dtype, [&](auto d) {
        using D = decltype(d);
        hipLaunchKernelGGL(k_pack_tiles<D>, dim3(grid_for(tiles)), dim3(kPackThreads), 0, (hipStream_t)stream,
                           (const typename D::T*)x, stride, rows, cols, codes, code_stride, scales, scale_stride, codes_t,
                           code_t_stride, scales_t, scale_t_stride, nbc, tiles);
    });
    return launch_status();
}

int gtopk_unpack(const uint8_t* codes, int64_t code_stride, const uint8_t* scales, int64_t scale_stride, int64_t rows,
                 int64_t cols, int32_t act, void* out, int32_t dtype, int64_t out_stride, void* stream) {
    if (!dtype_ok(dtype) || !act_ok(act) || !side_ok(rows, 0) || !side_ok(cols, 1) || out_stride < cols) return GTOPK_EINVAL;
    if (!packed_strides_ok(cols, code_stride, scale_stride)) return GTOPK_EINVAL;
    if (rows == 0) return GTOPK_OK;
    if (!codes || !scales || !out) return GTOPK_EINVAL;
    if (!packed_aligned(codes, scales) || !aligned(out, value_bytes(dtype))) return GTOPK_EALIGN;
    dim3 grid;
    const PackGrid g = pack_grid(rows, cols, dtype, &grid);
    by_type(dtype, [&](auto d) {
        using D = decltype(d);
        by_act(act, [&](auto f) {
            hipLaunchKernelGGL((k_unpack<D, decltype(f)::value>), grid, dim3(kPackThreads), 0, (hipStream_t)stream, codes,
                               code_stride, scales, scale_stride, g, (typename D::T*)out, out_stride);
        });
    });
    return launch_status();
}

int gtopk_activation_grad(const uint8_t* codes, int64_t code_stride, const uint8_t* scales, int64_t scale_stride,
                          int64_t rows, int64_t cols, int32_t act, const void* dy, int64_t dy_stride, void* dx,
                          int64_t dx_stride, int32_t dtype, void* stream) {
    if (!dtype_ok(dtype) || !act_ok(act) || !side_ok(rows, 0) || !side_ok(cols, 1) || dy_stride < cols || dx_stride < cols)
        return GTOPK_EINVAL;
    if (!packed_strides_ok(cols, code_stride, scale_stride)) return GTOPK_EINVAL;
    if (rows == 0) return GTOPK_OK;
    if (!codes || !scales || !dy || !dx || (dy == dx && dy_stride != dx_stride)) return GTOPK_EINVAL;
    if (!packed_aligned(codes, scales) || !aligned(dy, value_bytes(dtype)) || !aligned(dx, value_bytes(dtype))) return GTOPK_EALIGN;
    dim3 grid;
    const PackGrid g = pack_grid(rows, cols, dtype, &grid);
    by_type(dtype, [&](auto d) {
        using D = decltype(d);
        by_act(act, [&](auto f) {
            hipLaunchKernelGGL((k_activation_grad<D, decltype(f)::value>), grid, dim3(kPackThreads), 0, (hipStream_t)stream, codes,
                               code_stride, scales, scale_stride, g, (const typename D::T*)dy, dy_stride, (typename D::T*)dx, dx_stride);
        });
    });
    return launch_status();
}

size_t gtopk_product_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (!side_ok(M, 0) || !side_ok(N, 1) || !side_ok(K, 1) || K > kMaxCodeStride) return 0;
    const ProductPlan g = product_plan(M, N, K);
    if (g.thin ? N > kMaxThinColumns : ceil_div(M, 128) * ceil_div(N, 128) > kMaxTiles) return 0;
    return 256 + (g.shares > 1 ? (size_t)g.shares * M * g.stride * sizeof(float) : 0);
}

int gtopk_scaled_product(const uint8_t* a_codes, int64_t a_code_stride, const uint8_t* a_scales, int64_t a_scale_stride,
                         const uint8_t* b_codes, int64_t b_code_stride, const uint8_t* b_scales, int64_t b_scale_stride,
                         int64_t M, int64_t N, int64_t K, void* out, int32_t dtype, int64_t out_stride, void* ws,
                         size_t ws_bytes, void* stream) {
    const size_t need = gtopk_product_workspace_bytes(M, N, K);
    if (!need || !dtype_ok(dtype) || out_stride < N) return GTOPK_EINVAL;
    if (!packed_strides_ok(K, a_code_stride, a_scale_stride) || !packed_strides_ok(K, b_code_stride, b_scale_stride)) return GTOPK_EINVAL;
    if (a_code_stride > kMaxCodeStride || b_code_stride > kMaxCodeStride || a_scale_stride > kMaxCodeStride || b_scale_stride > kMaxCodeStride)
        return GTOPK_EINVAL;
    if (M == 0) return GTOPK_OK;
    if (!a_codes || !a_scales || !b_codes || !b_scales || !out || !ws) return GTOPK_EINVAL;
    if (!packed_aligned(a_codes, a_scales) || !packed_aligned(b_codes, b_scales) || !aligned(out, value_bytes(dtype)) || !aligned(ws, 16))
        return GTOPK_EALIGN;
    if (ws_bytes < need) return GTOPK_EWORKSPACE;
    const PackedMatrix a{a_codes, a_scales, (uint32_t)a_code_stride, (uint32_t)a_scale_stride};
    const PackedMatrix b{b_codes, b_scales, (uint32_t)b_code_stride, (uint32_t)b_scale_stride};
    const uint32_t nb = (uint32_t)ceil_div(K, kPackBlock);
    const ProductPlan g = product_plan(M, N, K);
    hipStream_t st = (hipStream_t)stream;
    by_type(dtype, [&](auto d) {
        using D = decltype(d);
        typename D::T* const to = (typename D::T*)out;
        if (g.thin) {
            const dim3 grid((uint32_t)ceil_div(N, 16)), block(kThinWaves * kWave);
            if (M <= 16) hipLaunchKernelGGL((k_product_thin<D, 1>), grid, block, 0, st, a, b, M, N, nb, to, out_stride);
            else hipLaunchKernelGGL((k_product_thin<D, 2>), grid, block, 0, st, a, b, M, N, nb, to, out_stride);
            return;
        }
        if (g.large) {
            hipLaunchKernelGGL((k_product<D, Exact<D>::value, 256, 256, 128, 64>), dim3(g.tiles_m * g.tiles_n), dim3(512), 0, st, a, b, M, N,
                               nb, to, out_stride, g.tiles_m, g.tiles_n, nb);
            return;
        }
        if (g.shares == 1) {
            hipLaunchKernelGGL((k_product<D, Exact<D>::value, 128, 128, 64, 64>), dim3(g.tiles_m * g.tiles_n), dim3(256), 0, st, a, b, M, N,
                               nb, to, out_stride, g.tiles_m, g.tiles_n, nb);
            return;
        }
        hipLaunchKernelGGL((k_product<F32, Exact<D>::value, 128, 128, 64, 64>), dim3(g.tiles_m * g.tiles_n, g.shares), dim3(256), 0, st, a, b,
                           M, N, nb, (float*)ws, g.stride, g.tiles_m, g.tiles_n, g.share);
        hipLaunchKernelGGL(k_join_products<D>, dim3((uint32_t)ceil_div(g.stride, 4 * kPackThreads), (uint32_t)M), dim3(kPackThreads), 0, st,
                           (const float*)ws, g.shares, M * g.stride, g.stride, N, to, out_stride);
    });
    return launch_status();
}

size_t gtopk_weight_grad_workspace_bytes(int64_t rows, int32_t P, int64_t N, int64_t K) {
    if (!side_ok(rows, 0) || P < 1 || P > 32768 || !side_ok(N, 1) || !side_ok(K, 1)) return 0;
    size_t most = 0;                    // of the plans of all types
    for (int bf16 = 0; bf16 < 2; ++bf16) {
        const GradPlan g = grad_plan(bf16 != 0, rows, P, N, K);
        if (g.jobs > kMaxJobs) return 0;
        const size_t bytes = 256 + (g.splits > 1 ? (size_t)g.splits * P * g.part_stride * sizeof(float) : 0);
        if (bytes > most) most = bytes;
    }
    return most;
}

int gtopk_weight_grad(const void* dy, int32_t dtype, int64_t dy_stride, const uint8_t* codes, int64_t code_stride,
                      const uint8_t* scales, int64_t scale_stride, int64_t rows, const int32_t* row_begin, int32_t P, int64_t N,
                      int64_t K, float* grad, int64_t grad_stride, int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
    const size_t need = gtopk_weight_grad_workspace_bytes(rows, P, N, K);
    if (!need || !dtype_ok(dtype) || dy_stride < N || !packed_strides_ok(K, code_stride, scale_stride)) return GTOPK_EINVAL;
    if ((P > 1 && grad_stride < N * K) || (!row_begin && rows % P != 0)) return GTOPK_EINVAL;
    if ((rows > 0 && (!dy || !codes || !scales)) || !grad || !ws) return GTOPK_EINVAL;
    if (!aligned(dy, value_bytes(dtype)) || !packed_aligned(codes, scales) || !aligned(row_begin, 4) || !aligned(grad, 4) || !aligned(ws, 16))
        return GTOPK_EALIGN;
    if (ws_bytes < need) return GTOPK_EWORKSPACE;
    const GradPlan g = grad_plan(dtype == GTOPK_BF16, rows, P, N, K);
    const bool split = g.splits > 1;
    float* const to = split ? (float*)ws : grad;
    const int64_t to_stride = split ? g.part_stride : grad_stride, split_stride = split ? g.part_stride * P : 0;
    const int parts = value_parts(dtype);
    const bool aligned_rows = K % 32 == 0 && to_stride % 32 == 0 && aligned(to, 128);
    const bool writes = rows / P * parts <= kGradWriteRows;
    const bool lines = grad_lines(parts, rows / P, P, N, K, aligned_rows);
    // An fp16 or fp32 dY is taken apart once per tile: twice as wide ones, with eight waves, where writing does not bound the call (us, 128 /
    // 256 wide, fp32 and fp16: 8192 rows, 4096 x 4096 821 / 679 and 614 / 503; 188 rows of 8 workers, 1000 x 4096 66 / 56 and 57 / 51; 150 rows of 4, 1000 x
    // 1024 15.5 / 14.0 and 13.9 / 12.5; 200 of 16, 2000 x 128, where half of a tile is empty, 18.9 / 18.3 and 16.5 / 15.6; 64 of 16, 4096 x 9217 637 / 647 and
    // 615 / 577; 64 of 32, 128 x 128 7.6 / 7.8 and 7.1 / 7.3.  bf16, 64 rows of 16 workers, 4096 x 9217: 484 / 505.)
    const bool wide = !lines && dtype != GTOPK_BF16;
    const uint32_t tiles_k = wide ? (uint32_t)ceil_div(K, 256) : lines && !aligned_rows ? (uint32_t)ceil_div(K + 31, 128) : g.tiles_k;
    const uint32_t jobs = g.tiles_n * tiles_k * (uint32_t)P * g.splits, band = writes || !aligned_rows ? tiles_k : kGradBand;
    hipStream_t st = (hipStream_t)stream;
    by_type(dtype, [&](auto d) {
        using D = decltype(d);
        auto launch = [&](auto kernel, int threads) {
            hipLaunchKernelGGL(kernel, dim3(grid_for(jobs)), dim3(threads), 0, st, (const typename D::T*)dy, dy_stride, codes, code_stride,
                               scales, scale_stride, rows, row_begin, (uint32_t)P, N, K, to, to_stride, split ? 0 : accumulate != 0,
                               g.splits, split_stride, g.tiles_n, tiles_k, band, jobs);
        };
        if (lines) launch(k_weight_grad<D, 128, 128, 64, 64, true>, 256);
        else if constexpr (Parts<D>::n > 1) launch(k_weight_grad<D, 128, 256, 64, 64, false>, 512);
        else if (g.big) launch(k_weight_grad<D, 256, 256, 128, 64, false>, 512);
        else launch(k_weight_grad<D, 128, 128, 64, 64, false>, 256);
    });
    if (split) {
        const int64_t blocks = ceil_div(N * K, 4 * kPackThreads);
        hipLaunchKernelGGL(k_join_shares, dim3((uint32_t)(blocks < 4096 ? blocks : 4096), (uint32_t)P), dim3(kPackThreads), 0, st,
                           (const float*)ws, g.splits, g.part_stride * P, g.part_stride, N * K, grad, grad_stride, accumulate != 0);
    }
    return launch_status();
}

}  // extern "C"
