// Orthogonalisation of a batch of matrices by Newton-Schulz products.
#include <algorithm>

#include "lm_ops.h"
#include "simple_matmul.cuh"

namespace a2 {

namespace {

struct Layout {
    float *x0, *x1, *gram, *poly;
    double* norm;
};

int64_t layout(int64_t mats, int64_t rows, int64_t cols, void* ws, Layout* out) {
    const int64_t m = std::min(rows, cols);
    Carver w(ws);
    Layout l{};
    l.x0 = w.take<float>(mats * rows * cols);
    l.x1 = w.take<float>(mats * rows * cols);
    l.gram = w.take<float>(mats * m * m);
    l.poly = w.take<float>(mats * m * m);
    l.norm = w.take<double>(mats);
    if (out) *out = l;
    return w.used;
}

// One CTA a matrix: Frobenius norm with 64-bit sums, then X0 = G / (norm + eps), laid out [min, max].
template <class T>
__global__ void __launch_bounds__(1024) k_normalize(const T* in, int64_t stride, int64_t pitch, int64_t rows, int64_t cols, bool turn, double eps, float* x0) {
    __shared__ double part[32];
    const T* g = in + blockIdx.x * stride;
    float* x = x0 + blockIdx.x * rows * cols;
    double sum = 0.0;
    for (int64_t e = threadIdx.x; e < rows * cols; e += 1024) {
        const double v = widen(g[e / cols * pitch + e % cols]);
        sum += v * v;
    }
    for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = sum;
    __syncthreads();
    double all = 0.0;
    for (int w = 0; w < 32; ++w) all += part[w];
    const double by = sqrt(all) + eps;
    for (int64_t e = threadIdx.x; e < rows * cols; e += 1024) {
        const int64_t i = e / cols, j = e % cols;
        x[turn ? j * rows + i : e] = by > 0.0 ? (float)(widen(g[i * pitch + j]) / by) : by == 0.0 ? 0.0f : NAN;
    }
}

// out = s x, back in the caller's layout.
template <class T>
__global__ void k_scatter(const float* x0, int64_t rows, int64_t cols, bool turn, float scale, T* out, int64_t stride, int64_t pitch) {
    const float* x = x0 + blockIdx.y * rows * cols;
    T* o = out + blockIdx.y * stride;
    for (int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; e < rows * cols; e += (int64_t)gridDim.x * blockDim.x) {
        const int64_t i = e / cols, j = e % cols;
        o[i * pitch + j] = narrow<T>(scale * x[turn ? j * rows + i : e]);
    }
}

__global__ void k_copy(const float* a, float* b, int64_t n) {
    for (int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; e < n; e += (int64_t)gridDim.x * blockDim.x) b[e] = a[e];
}

template <class T>
cudaError_t typed(const OrthogonalizeArgs& a, const Layout& l, cudaStream_t s) {
    const bool turn = a.rows > a.cols;
    const int64_t m = std::min(a.rows, a.cols), n = std::max(a.rows, a.cols);
    k_normalize<T><<<(unsigned)a.n_mats, 1024, 0, s>>>(static_cast<const T*>(a.in), a.in_stride, a.in_pitch, a.rows, a.cols, turn, a.eps, l.x0);
    float *x = l.x0, *y = l.x1;
    for (int step = 0; step < a.steps; ++step) {
        matmul<float, float, float>({x, n, 1, m * n}, {x, 1, n, m * n}, {l.gram, m, 1, m * m}, m, m, n, a.n_mats, 1.0f, 0.0f, s);
        k_copy<<<1024, 256, 0, s>>>(l.gram, l.poly, a.n_mats * m * m);
        matmul<float, float, float>({l.gram, m, 1, m * m}, {l.gram, m, 1, m * m}, {l.poly, m, 1, m * m}, m, m, m, a.n_mats, a.cc, a.cb, s);
        k_copy<<<1024, 256, 0, s>>>(x, y, a.n_mats * m * n);
        matmul<float, float, float>({l.poly, m, 1, m * m}, {x, n, 1, m * n}, {y, n, 1, m * n}, m, n, m, a.n_mats, 1.0f, a.ca, s);
        std::swap(x, y);
    }
    k_scatter<T><<<dim3(512, (unsigned)a.n_mats), 256, 0, s>>>(x, a.rows, a.cols, turn, a.scale, static_cast<T*>(a.out), a.out_stride, a.out_pitch);
    return cudaGetLastError();
}

}  // namespace

int64_t orthogonalize_workspace(int64_t n_mats, int64_t rows, int64_t cols, int32_t) { return layout(n_mats, rows, cols, nullptr, nullptr); }

cudaError_t run_orthogonalize(const OrthogonalizeArgs& a, void* workspace, cudaStream_t s) {
    Layout l;
    layout(a.n_mats, a.rows, a.cols, workspace, &l);
    return a.dtype == A2_BF16 ? typed<__nv_bfloat16>(a, l, s) : typed<float>(a, l, s);
}

}  // namespace a2
