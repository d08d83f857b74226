// A plain batched matrix product on the CUDA cores, C = alpha A B + beta C, any strides, fp32 sums.
#pragma once

#include "lm_ops.h"

namespace a2 {

template <class T>
struct Strided {
    T* p;
    int64_t row, col, mat;  // strides in elements
};

template <class TA, class TB, class TC>
__global__ void __launch_bounds__(256) k_matmul(Strided<const TA> a, Strided<const TB> b, Strided<TC> c, int64_t m, int64_t n, int64_t k,
                                                float alpha, float beta) {
    __shared__ float as[16][65], bs[16][65];
    const int64_t i0 = (int64_t)blockIdx.y * 64, j0 = (int64_t)blockIdx.x * 64;
    const TA* ap = a.p + blockIdx.z * a.mat;
    const TB* bp = b.p + blockIdx.z * b.mat;
    TC* cp = c.p + blockIdx.z * c.mat;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float sum[4][4] = {};
    for (int64_t k0 = 0; k0 < k; k0 += 16) {
        for (int e = threadIdx.x; e < 64 * 16; e += 256) {
            const int r = a.col == 1 ? e / 16 : e % 64, q = a.col == 1 ? e % 16 : e / 64;
            as[q][r] = i0 + r < m && k0 + q < k ? widen(ap[(i0 + r) * a.row + (k0 + q) * a.col]) : 0.0f;
            const int r2 = b.col == 1 ? e / 64 : e % 16, q2 = b.col == 1 ? e % 64 : e / 16;
            bs[r2][q2] = j0 + q2 < n && k0 + r2 < k ? widen(bp[(k0 + r2) * b.row + (j0 + q2) * b.col]) : 0.0f;
        }
        __syncthreads();
        float part[4][4] = {};  // sixteen products first: the long sum then has a sixteenth of the roundings
#pragma unroll
        for (int q = 0; q < 16; ++q)
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) part[u][v] = fmaf(as[q][ty * 4 + u], bs[q][tx * 4 + v], part[u][v]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int v = 0; v < 4; ++v) sum[u][v] += part[u][v];
        __syncthreads();
    }
    for (int u = 0; u < 4; ++u)
        for (int v = 0; v < 4; ++v) {
            const int64_t i = i0 + ty * 4 + u, j = j0 + tx * 4 + v;
            if (i >= m || j >= n) continue;
            TC* at = cp + i * c.row + j * c.col;
            *at = narrow<TC>(alpha * sum[u][v] + (beta != 0.0f ? beta * widen(*at) : 0.0f));
        }
}

template <class TA, class TB, class TC>
void matmul(Strided<const TA> a, Strided<const TB> b, Strided<TC> c, int64_t m, int64_t n, int64_t k, int64_t mats, float alpha, float beta,
            cudaStream_t s) {
    if (m <= 0 || n <= 0 || mats <= 0) return;
    k_matmul<TA, TB, TC><<<dim3((unsigned)ceil_div(n, 64), (unsigned)ceil_div(m, 64), (unsigned)mats), 256, 0, s>>>(a, b, c, m, n, k, alpha, beta);
}

}  // namespace a2
