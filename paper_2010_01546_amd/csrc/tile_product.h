#pragma once
#include "fw_internal.h"

namespace fw {

// C[r][c] = sum_k A[r][k] B[c][k] for operands in any order of their axes (strides ars, aks and brs, bks in entries); each finished
// element goes to epi(r, c, sum).  A workgroup owns 64 x 64 results, a thread 4 x 4 of them.
template <class TA, class TB, class Acc, class Epi>
__global__ __launch_bounds__(256) void strided_product_kernel(const TA* __restrict__ A, size_t ars, size_t aks, const TB* __restrict__ B,
                                                              size_t brs, size_t bks, int R, int C, int K, Epi epi) {
    __shared__ Acc a[16][65], b[16][65];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const long long r0 = (long long)blockIdx.y * 64, c0 = (long long)blockIdx.x * 64;
    Acc acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += 16) {
        for (int e = tid; e < 1024; e += 256) {
            const int kk = e & 15, rr = e >> 4, k = k0 + kk;
            a[kk][rr] = k < K && r0 + rr < R ? (Acc)A[(size_t)(r0 + rr) * ars + (size_t)k * aks] : (Acc)0;
            b[kk][rr] = k < K && c0 + rr < C ? (Acc)B[(size_t)(c0 + rr) * brs + (size_t)k * bks] : (Acc)0;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < 16; ++kk)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += a[kk][ty + 16 * i] * b[kk][tx + 16 * j];
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (r0 + ty + 16 * i < R && c0 + tx + 16 * j < C) epi((int)(r0 + ty + 16 * i), (int)(c0 + tx + 16 * j), acc[i][j]);
}

template <class Acc, class TA, class TB, class Epi>
fw_status strided_product(const TA* A, size_t ars, size_t aks, const TB* B, size_t brs, size_t bks, int R, int C, int K, Epi epi, hipStream_t st) {
    for (long long r0 = 0; r0 < R; r0 += 64 * 32768ll) {      // the grid's second axis ends at 65535
        const int rows = (int)(R - r0 < 64 * 32768ll ? R - r0 : 64 * 32768ll);
        auto shifted = [=] __device__(int r, int c, Acc v) { epi(r + r0, c, v); };
        hipLaunchKernelGGL((strided_product_kernel<TA, TB, Acc, decltype(shifted)>), dim3((C + 63) / 64, (rows + 63) / 64), dim3(256), 0, st,
                           A + (size_t)r0 * ars, ars, aks, B, brs, bks, rows, C, K, shifted);
        FW_LAUNCH_CHECK();
    }
    return FW_OK;
}

}  // namespace fw
