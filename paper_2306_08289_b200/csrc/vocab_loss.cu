// Softmax cross entropy over a large vocabulary, in pieces of the vocabulary, with its gradients.
#include <algorithm>

#include "lm_ops.h"
#include "simple_matmul.cuh"

namespace a2 {

namespace {

constexpr int64_t kPiece = 2048;  // vocabulary rows a piece

__global__ void k_start(float* top, float* sum, float* target, int64_t n) {
    const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (t < n) {
        top[t] = -INFINITY;
        sum[t] = 0.0f;
        target[t] = 0.0f;
    }
}

// One warp a token: the running maximum and sum of exponentials over one piece's logits.
__global__ void k_statistics(const float* z, int64_t n, int64_t piece, int64_t v0, const int32_t* targets, float* top, float* sum, float* target) {
    const int64_t t = (int64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32;
    const int lane = threadIdx.x % 32;
    if (t >= n) return;
    float m = -INFINITY;
    for (int64_t j = lane; j < piece; j += 32) m = fmaxf(m, z[t * kPiece + j]);
    for (int o = 16; o; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    m = fmaxf(m, top[t]);
    float s = 0.0f;
    for (int64_t j = lane; j < piece; j += 32) s += expf(z[t * kPiece + j] - m);
    for (int o = 16; o; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) {
        sum[t] = sum[t] * (top[t] == m ? 1.0f : expf(top[t] - m)) + s;
        top[t] = m;
        const int64_t y = (int64_t)targets[t] - v0;
        if (y >= 0 && y < piece) target[t] = z[t * kPiece + y];
    }
}

__global__ void k_finish(const float* top, const float* sum, const float* target, const int32_t* targets, int64_t n, int64_t vocab, float* loss,
                         float* lse) {
    const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (t >= n) return;
    const float l = top[t] + logf(sum[t]);
    lse[t] = l;
    loss[t] = targets[t] >= 0 && targets[t] < vocab ? l - target[t] : 0.0f;
}

__global__ void k_probabilities(float* z, int64_t n, int64_t piece, int64_t v0, int64_t vocab, const int32_t* targets, const float* lse,
                                const float* weights, float scale) {
    const int64_t t = blockIdx.x;
    const int64_t y = targets[t];
    const bool live = y >= 0 && y < vocab;
    const float g = live ? scale * (weights ? weights[t] : 1.0f) : 0.0f;
    for (int64_t j = threadIdx.x; j < piece; j += blockDim.x)
        z[t * kPiece + j] = live ? g * (expf(z[t * kPiece + j] - lse[t]) - (v0 + j == y ? 1.0f : 0.0f)) : 0.0f;
}

template <class T>
__global__ void k_store(const float* from, int64_t rows, int64_t width, T* to, int64_t pitch) {
    for (int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; e < rows * width; e += (int64_t)gridDim.x * blockDim.x)
        to[e / width * pitch + e % width] = narrow<T>(from[e]);
}

// A token without a target adds nothing to any gradient, whatever its hidden state holds.
template <class T>
__global__ void k_live_rows(const T* h, int64_t n, int64_t width, int64_t pitch, int64_t vocab, const int32_t* targets, float* to) {
    for (int64_t e = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; e < n * width; e += (int64_t)gridDim.x * blockDim.x) {
        const int64_t y = targets[e / width];
        to[e] = y >= 0 && y < vocab ? widen(h[e / width * pitch + e % width]) : 0.0f;
    }
}

struct Layout {
    float *z, *top, *sum, *target, *dh, *live;
};
int64_t layout(int64_t n, int64_t width, bool with_grad, void* ws, Layout* out) {
    Carver w(ws);
    Layout l{};
    l.z = w.take<float>(n * kPiece);
    l.top = w.take<float>(n);
    l.sum = w.take<float>(n);
    l.target = w.take<float>(n);
    if (with_grad) l.dh = w.take<float>(n * width);
    if (with_grad) l.live = w.take<float>(n * width);
    if (out) *out = l;
    return w.used;
}

template <class T>
cudaError_t typed(const VocabLossArgs& a, const Layout& l, cudaStream_t s) {
    const int64_t n = a.n_tokens;
    auto* h = static_cast<const T*>(a.hidden);
    auto* w = static_cast<const T*>(a.head);
    auto logits = [&](int64_t v0, int64_t piece) {
        matmul<T, T, float>({h, a.hidden_pitch, 1, 0}, {w + v0 * a.head_pitch, 1, a.head_pitch, 0}, {l.z, kPiece, 1, 0}, n, piece, a.width, 1,
                            1.0f, 0.0f, s);
    };
    if (n > 0) k_start<<<(unsigned)ceil_div(n, 256), 256, 0, s>>>(l.top, l.sum, l.target, n);
    for (int64_t v0 = 0; v0 < a.vocab && n > 0; v0 += kPiece) {
        const int64_t piece = std::min(kPiece, a.vocab - v0);
        logits(v0, piece);
        k_statistics<<<(unsigned)ceil_div(n, 8), 256, 0, s>>>(l.z, n, piece, v0, a.targets, l.top, l.sum, l.target);
    }
    if (n > 0) k_finish<<<(unsigned)ceil_div(n, 256), 256, 0, s>>>(l.top, l.sum, l.target, a.targets, n, a.vocab, a.loss, a.lse);
    if (!a.grad_hidden && !a.grad_head) return cudaGetLastError();
    if (n > 0) k_live_rows<T><<<1024, 256, 0, s>>>(h, n, a.width, a.hidden_pitch, a.vocab, a.targets, l.live);
    for (int64_t v0 = 0; v0 < a.vocab; v0 += kPiece) {
        const int64_t piece = std::min(kPiece, a.vocab - v0);
        if (n > 0) {
            logits(v0, piece);
            k_probabilities<<<(unsigned)n, 256, 0, s>>>(l.z, n, piece, v0, a.vocab, a.targets, a.lse, a.weights, a.scale);
        }
        if (a.grad_head)
            matmul<float, float, T>({l.z, 1, kPiece, 0}, {l.live, a.width, 1, 0},
                                {static_cast<T*>(a.grad_head) + v0 * a.grad_head_pitch, a.grad_head_pitch, 1, 0}, piece, a.width, n, 1, 1.0f,
                                0.0f, s);
        if (a.grad_hidden)
            matmul<float, T, float>({l.z, kPiece, 1, 0}, {w + v0 * a.head_pitch, a.head_pitch, 1, 0}, {l.dh, a.width, 1, 0}, n, a.width, piece,
                                    1, 1.0f, v0 == 0 ? 0.0f : 1.0f, s);
    }
    if (a.grad_hidden && n > 0)
        k_store<T><<<(unsigned)std::min<int64_t>(ceil_div(n * a.width, 256), 4096), 256, 0, s>>>(l.dh, n, a.width, static_cast<T*>(a.grad_hidden),
                                                                                                 a.grad_hidden_pitch);
    return cudaGetLastError();
}

}  // namespace

int64_t vocab_loss_workspace(int64_t n_tokens, int64_t width, int64_t, bool with_grad, int32_t) {
    return layout(n_tokens, width, with_grad, nullptr, nullptr);
}

cudaError_t run_vocab_loss(const VocabLossArgs& a, void* workspace, cudaStream_t s) {
    Layout l;
    layout(a.n_tokens, a.width, a.grad_hidden || a.grad_head, workspace, &l);
    return a.dtype == A2_BF16 ? typed<__nv_bfloat16>(a, l, s) : typed<float>(a, l, s);
}

}  // namespace a2
