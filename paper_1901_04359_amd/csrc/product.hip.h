// C = A B^T of two packed matrices:
//   C[m][n] = sum over blocks b of 2^(ea[m][b] + eb[n][b]) * (sum over k in b of a[m][k] * b[n][k])
#pragma once
#include "packed.hip.h"

namespace gtopk {

// one value per thread, a block of 128 of sixteen rows of A and of B at a time in LDS
template <class D>
__global__ __launch_bounds__(256) void k_product(
        const uint8_t* __restrict__ a, int64_t a_stride, const uint8_t* __restrict__ a_scales, int64_t a_scale_stride,
        const uint8_t* __restrict__ b, int64_t b_stride, const uint8_t* __restrict__ b_scales, int64_t b_scale_stride,
        int64_t M, int64_t N, uint32_t nb, typename D::T* __restrict__ out, int64_t out_stride, uint32_t tiles_n, uint64_t tiles) {
    __shared__ float s_a[16][kPackBlock + 1], s_b[16][kPackBlock + 1];
    const uint32_t r = threadIdx.x / 16, l = threadIdx.x % 16;
    for (uint64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t m0 = (int64_t)(tile / tiles_n) * 16, n0 = (int64_t)(tile % tiles_n) * 16;
        float sum = 0.0f;
        for (uint32_t kb = 0; kb < nb; ++kb) {
            float v[kLaneVals] = {}, w[kLaneVals] = {};
            const int64_t col = (int64_t)kb * kPackBlock + l * kLaneVals;
            if (m0 + r < M)
                decode8(*reinterpret_cast<const uint32x2*>(a + (m0 + r) * a_stride + col), scale_value(a_scales[(m0 + r) * a_scale_stride + kb]), v);
            if (n0 + r < N)
                decode8(*reinterpret_cast<const uint32x2*>(b + (n0 + r) * b_stride + col), scale_value(b_scales[(n0 + r) * b_scale_stride + kb]), w);
#pragma unroll
            for (int j = 0; j < kLaneVals; ++j) {
                s_a[r][l * kLaneVals + j] = v[j];
                s_b[r][l * kLaneVals + j] = w[j];
            }
            __syncthreads();
            for (int k = 0; k < kPackBlock; ++k) sum += s_a[r][k] * s_b[l][k];
            __syncthreads();
        }
        if (m0 + r < M && n0 + l < N) out[(m0 + r) * out_stride + n0 + l] = (typename D::T)sum;
    }
}

}  // namespace gtopk
