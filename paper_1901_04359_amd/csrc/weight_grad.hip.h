// Weight gradients of P workers from packed activations, into the workers' gradient rows:
//   dW_w[n][k] = sum over the rows t of worker w of dY[t][n] * X[t][k]
#pragma once
#include "packed.hip.h"

namespace gtopk {

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

// one value per thread, sixteen rows at a time in LDS
template <class D>
__global__ __launch_bounds__(256) void k_weight_grad(
        const typename D::T* __restrict__ dy, int64_t dy_stride, const uint8_t* __restrict__ codes, int64_t code_stride,
        const uint8_t* __restrict__ scales, int64_t scale_stride, int64_t rows, const int32_t* __restrict__ begin, uint32_t P,
        int64_t N, int64_t K, float* __restrict__ grad, int64_t grad_stride, int accumulate, uint32_t tiles_k, uint64_t tiles) {
    __shared__ float s_d[16][17], s_x[16][17];
    const uint32_t r = threadIdx.x / 16, l = threadIdx.x % 16;
    for (uint64_t job = blockIdx.x; job < tiles * P; job += gridDim.x) {
        const uint32_t w = (uint32_t)(job / tiles);
        const uint64_t tile = job % tiles;
        const int64_t n0 = (int64_t)(tile / tiles_k) * 16, k0 = (int64_t)(tile % tiles_k) * 16;
        int64_t first, last;
        rows_of_worker(begin, rows, P, w, first, last);
        float sum = 0.0f;
        for (int64_t t0 = first; t0 < last; t0 += 16) {
            const int64_t t = t0 + r;
            const bool in = t < last;
            s_d[r][l] = in && n0 + l < N ? (float)dy[t * dy_stride + n0 + l] : 0.0f;
            float x = 0.0f;
            if (in && k0 + l < K)
                x = __builtin_amdgcn_cvt_f32_fp8((int)codes[t * code_stride + k0 + l], 0) * scale_value(scales[t * scale_stride + k0 / kPackBlock]);
            s_x[r][l] = x;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 16; ++j) sum += s_d[j][r] * s_x[j][l];
            __syncthreads();
        }
        if (n0 + r < N && k0 + l < K) {
            float* g = grad + w * grad_stride + (n0 + r) * K + k0 + l;
            *g = accumulate ? *g + sum : sum;
        }
    }
}

}  // namespace gtopk
