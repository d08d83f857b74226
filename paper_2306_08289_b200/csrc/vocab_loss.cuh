// What the two forms of the vocabulary loss share.
#pragma once

#include <cmath>

#include "lm_ops.h"

namespace a2 {

// Few tokens times few columns: see vocab_loss_few.cu. The rule and the workspace know nothing of alignment or gradients, so that a loss
// is the same bits with and without them.
bool vocab_loss_is_few(int64_t n_tokens, int64_t width, int64_t vocab, int32_t dtype);
int64_t vocab_loss_few_workspace(int64_t n_tokens, int64_t width, int64_t vocab, bool with_grad);
cudaError_t run_vocab_loss_few(const VocabLossArgs& a, void* workspace, cudaStream_t s);

namespace {

constexpr float kLog2E = 1.4426950408889634f;
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ bool is_token(int32_t y, int64_t vocab) { return y >= 0 && y < vocab; }

// Joins the statistics of the parts: 32 tokens a CTA, its warps over the parts.
constexpr int kFinishWarps = 16;
__global__ void __launch_bounds__(kFinishWarps * 32) k_finish(const float2* partial, int parts, const float* at_target,
                                                const int32_t* targets, const int32_t* poisoned, int64_t n, int64_t vocab,
                                                float* __restrict__ loss, float* __restrict__ lse) {
    ptx::chained();
    __shared__ float2 joined[kFinishWarps][32];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t t = (int64_t)blockIdx.x * 32 + lane;
    float top = -INFINITY, sum = 0.0f;
    // eight parts at a time: their loads and exponentials do not wait for one another
    for (int p0 = warp; t < n && p0 < parts; p0 += 8 * kFinishWarps) {
        float2 p[8];
        float next = top;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int at = p0 + k * kFinishWarps;
            p[k] = at < parts ? partial[(int64_t)at * n + t] : make_float2(-INFINITY, 0.0f);
            next = fmaxf(next, p[k].x);
        }
        const float base = next == -INFINITY ? 0.0f : next;
        sum *= exp2_fast((top - base) * kLog2E);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += p[k].y * exp2_fast((p[k].x - base) * kLog2E);
        top = next;
    }
    joined[warp][lane] = make_float2(top, sum);
    __syncthreads();
    if (warp == 0 && t < n) {
        for (int w = 1; w < kFinishWarps; ++w) top = fmaxf(top, joined[w][lane].x);
        const float base = top == -INFINITY ? 0.0f : top;
        sum = 0.0f;
        for (int w = 0; w < kFinishWarps; ++w) sum += joined[w][lane].y * exp2_fast((joined[w][lane].x - base) * kLog2E);
        const float l = poisoned && poisoned[t] ? NAN : top + logf(sum);
        lse[t] = l;
        loss[t] = is_token(targets[t], vocab) ? l - at_target[t] : 0.0f;
    }
}

// The same of tokens whose logits lie in the workspace; with gradients also turns them into P. A CTA a token and kRowColumns
// columns. partial: [n][parts].
constexpr int kRowThreads = 128, kRowColumns = 2048;

__device__ __forceinline__ float block_reduce(float v, bool sum, float* shared) {
    for (int o = 16; o; o /= 2) {
        const float w = __shfl_xor_sync(0xffffffffu, v, o);
        v = sum ? v + w : fmaxf(v, w);
    }
    __syncthreads();
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = v;
    __syncthreads();
    v = shared[0];
    for (int w = 1; w < kRowThreads / 32; ++w) v = sum ? v + shared[w] : fmaxf(v, shared[w]);
    return v;
}

template <class Sink>
__global__ void __launch_bounds__(kRowThreads) k_rows(const VocabLossArgs a, const float2* partial, int parts, const float* at_target,
                                                      const int32_t* poisoned, bool probabilities, const float* z, int64_t z_ld, Sink sink) {
    ptx::chained();
    __shared__ float shared[kRowThreads / 32];
    const int64_t t = blockIdx.x;
    const float2* mine = partial + t * parts;
    float top = -INFINITY, sum = 0.0f;
    for (int p = threadIdx.x; p < parts; p += kRowThreads) top = fmaxf(top, mine[p].x);
    top = block_reduce(top, false, shared);
    const float base = top == -INFINITY ? 0.0f : top;
    for (int p = threadIdx.x; p < parts; p += kRowThreads) sum += mine[p].y * exp2_fast((mine[p].x - base) * kLog2E);
    sum = block_reduce(sum, true, shared);
    const float lse = poisoned && poisoned[t] ? NAN : top + logf(sum);
    const int64_t y = a.targets[t];
    const bool live = is_token((int32_t)y, a.vocab);
    if (threadIdx.x == 0 && blockIdx.y == 0) {
        a.lse[t] = lse;
        a.loss[t] = live ? lse - at_target[t] : 0.0f;
    }
    if (!probabilities) return;
    const auto row = sink.row(t);
    const int64_t c0 = (int64_t)blockIdx.y * kRowColumns;
    // two columns a thread; z_ld is even, and what is written past the vocabulary is padding
#pragma unroll 4
    for (int64_t c = c0 + threadIdx.x * 2; c < min(c0 + kRowColumns, a.vocab); c += kRowThreads * 2) {
        const float2 l = *reinterpret_cast<const float2*>(z + t * z_ld + c);
        const float p = exp2_fast((l.x - lse) * kLog2E), q = exp2_fast((l.y - lse) * kLog2E);
        if (live) row(c, c == y ? p - 1.0f : p, c + 1 == y ? q - 1.0f : q);
        else row.none(c);
    }
}

template <class Sink>
[[nodiscard]] cudaError_t launch_rows(const VocabLossArgs& a, const float2* partial, int parts, const float* at_target, const int32_t* poisoned, const float* z, int64_t z_ld,
                        bool with_grad, const Sink& sink, cudaStream_t s) {
    return launch_chained(k_rows<Sink>, dim3((unsigned)a.n_tokens, with_grad ? (unsigned)ceil_div(a.vocab, kRowColumns) : 1u), kRowThreads, 0, s, a, partial,
                          parts, at_target, poisoned, with_grad, z, z_ld, sink);
}

}  // namespace

}  // namespace a2
