// The vocabulary loss of few tokens, few columns, or both: products on the CUDA cores in fp32 straight from the rows, logits kept in
// the workspace (64 MB at most) and turned into P there. Two launches forward and one to three for the gradients, where the tensor-core
// form needs up to ten and pads 256 rows; what bounds it is latency, or reading the head.
#include <algorithm>

#include "vocab_loss.cuh"

namespace a2 {

namespace {

constexpr int kM = 32, kN = 64, kK = 32;  // a CTA's tile
constexpr int kFewThreads = 128;          // 16 x 8 threads of 4 x 4 sums
constexpr int kPitch = kK + 4;            // floats: rows 16 bytes apart modulo 128, so that eight threads' rows are free of conflicts

// sums[u][v] += sum over k in [0, depth) of a(m, k) b(n, k), m = ty * 4 + u, n = tx + 16 * v. A_K, B_K: neighbouring k lie side by side
// in memory (else neighbouring m or n do). The loaders return 0 outside. kParts: every kPartK of a long row are added up by themselves
// first, since one chain would round every term to the size of the whole sum (2 x 356 x 1,753: loss 2.3e-6 from 64 bits, with parts 4e-7).
constexpr int kPartK = 4 * kK;
template <bool A_K, bool B_K, bool kParts, class LoadA, class LoadB>
__device__ __forceinline__ void tile_product(float (&sums)[4][4], int64_t depth, LoadA a, LoadB b) {
    __shared__ __align__(16) float as[kM * kPitch], bs[kN * kPitch];
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, tx = tid % 16, ty = tid / 16;
    float ra[kM / 4], rb[kN / 4], whole[4][4] = {};
    auto fetch = [&](int64_t k0) {
#pragma unroll
        for (int i = 0; i < kM / 4; ++i) {
            const int other = warp + 4 * i;  // a warp reads 32 neighbours of one m (or of one k)
            ra[i] = A_K ? a(other, k0 + lane) : a(lane, k0 + other);
        }
#pragma unroll
        for (int i = 0; i < kN / 4; ++i) {
            const int other = warp + 4 * i;
            rb[i] = B_K ? b(other, k0 + lane) : b(lane + 32 * (other / kK), k0 + other % kK);
        }
    };
    fetch(0);
    for (int64_t k0 = 0; k0 < depth; k0 += kK) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kM / 4; ++i) as[A_K ? (warp + 4 * i) * kPitch + lane : lane * kPitch + warp + 4 * i] = ra[i];
#pragma unroll
        for (int i = 0; i < kN / 4; ++i) {
            const int other = warp + 4 * i;
            bs[B_K ? other * kPitch + lane : (lane + 32 * (other / kK)) * kPitch + other % kK] = rb[i];
        }
        __syncthreads();
        if (k0 + kK < depth) fetch(k0 + kK);
        if (kParts && k0 > 0 && k0 % kPartK == 0)
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    whole[u][v] += sums[u][v];
                    sums[u][v] = 0.0f;
                }
#pragma unroll
        for (int k = 0; k < kK; k += 4) {
            float4 x[4], y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = *reinterpret_cast<const float4*>(as + (ty * 4 + u) * kPitch + k);
#pragma unroll
            for (int v = 0; v < 4; ++v) y[v] = *reinterpret_cast<const float4*>(bs + (tx + 16 * v) * kPitch + k);
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    sums[u][v] = fmaf(x[u].x, y[v].x, sums[u][v]);
                    sums[u][v] = fmaf(x[u].y, y[v].y, sums[u][v]);
                    sums[u][v] = fmaf(x[u].z, y[v].z, sums[u][v]);
                    sums[u][v] = fmaf(x[u].w, y[v].w, sums[u][v]);
                }
        }
    }
    if (kParts)
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int v = 0; v < 4; ++v) sums[u][v] += whole[u][v];
}

// Logits of 32 tokens x 64 vocabulary rows, and each token's maximum and sum of exponentials over the 64.
template <class T>
__global__ void __launch_bounds__(kFewThreads) k_few_logits(const VocabLossArgs a, float* __restrict__ z, int64_t z_ld, float2* __restrict__ partial,
                                                            float* __restrict__ at_target) {
    ptx::chained();
    const T* hidden = static_cast<const T*>(a.hidden);
    const T* head = static_cast<const T*>(a.head);
    const int64_t parts = (a.vocab + kN - 1) / kN, part = blockIdx.x % parts;  // along the vocabulary first
    const int64_t t0 = blockIdx.x / parts * kM, v0 = part * kN;
    float sums[4][4] = {};
    tile_product<true, true, true>(
        sums, a.width, [&](int m, int64_t k) { return t0 + m < a.n_tokens && k < a.width ? widen(hidden[(t0 + m) * a.hidden_pitch + k]) : 0.0f; },
        [&](int n, int64_t k) { return v0 + n < a.vocab && k < a.width ? widen(head[(v0 + n) * a.head_pitch + k]) : 0.0f; });
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int64_t t = t0 + ty * 4 + u;
        const bool row = t < a.n_tokens;
        const int64_t y = row ? a.targets[t] : -1;
        float most = -INFINITY;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int64_t c = v0 + tx + 16 * v;
            if (c >= a.vocab) {
                sums[u][v] = -INFINITY;
            } else if (row) {
                z[t * z_ld + c] = sums[u][v];
                if (c == y) at_target[t] = sums[u][v];
            }
            most = fmaxf(most, sums[u][v]);
        }
        for (int o = 8; o; o /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        const float base = most == -INFINITY ? 0.0f : most;
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < 4; ++v) sum += exp2_fast((sums[u][v] - base) * kLog2E);
        for (int o = 8; o; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (tx == 0 && row) partial[t * parts + part] = make_float2(most, sum);
    }
}

// P in place of the logits, with the gradients' factor in it.
struct FewSink {
    float* z;
    int64_t z_ld;
    float scale;
    const float* weights;
    struct Row {
        float* z;
        float g;
        __device__ __forceinline__ void operator()(int64_t c, float p, float q) const { *reinterpret_cast<float2*>(z + c) = make_float2(g * p, g * q); }
        __device__ __forceinline__ void none(int64_t c) const { *reinterpret_cast<float2*>(z + c) = make_float2(0.0f, 0.0f); }
    };
    __device__ __forceinline__ Row row(int64_t t) const { return {z + t * z_ld, scale * (weights ? weights[t] : 1.0f)}; }
};

// Both gradients: CTAs 0 .. head_ctas - 1 make tiles of grad_head (32 vocabulary rows x 64 columns over a part of the tokens), the others
// tiles of grad_hidden (32 tokens x 64 columns over a part of the vocabulary).
struct Split {
    int64_t tiles;  // of a part
    int parts;
    int64_t depth;  // of a part
    float* sums;    // [parts][rows][width] with several parts
};
struct FewGradArgs {
    VocabLossArgs loss;
    const float* p;
    int64_t p_ld, columns;  // tile columns
    Split head, hidden;
};

template <class T>
__global__ void __launch_bounds__(kFewThreads) k_few_gradients(const FewGradArgs g) {
    ptx::chained();
    const VocabLossArgs& a = g.loss;
    const T* hidden = static_cast<const T*>(a.hidden);
    const T* head = static_cast<const T*>(a.head);
    const int64_t head_ctas = g.head.tiles * g.head.parts;
    const bool of_head = (int64_t)blockIdx.x < head_ctas;
    const Split& s = of_head ? g.head : g.hidden;
    const int64_t unit = of_head ? blockIdx.x : blockIdx.x - head_ctas, part = unit / s.tiles, tile = unit % s.tiles;
    const int64_t r0 = tile / g.columns * kM, c0 = tile % g.columns * kN, first = part * s.depth;
    const int64_t rows = of_head ? a.vocab : a.n_tokens, depth = min(s.depth, (of_head ? a.n_tokens : a.vocab) - first);
    float sums[4][4] = {};
    if (of_head)
        tile_product<false, false, false>(
            sums, depth, [&](int m, int64_t k) { return r0 + m < a.vocab && k < depth ? g.p[(first + k) * g.p_ld + r0 + m] : 0.0f; },
            [&](int n, int64_t k) {  // a token without a target adds nothing, whatever its row holds
                if (c0 + n >= a.width || k >= depth) return 0.0f;
                const float h = widen(hidden[(first + k) * a.hidden_pitch + c0 + n]);
                return is_token(a.targets[first + k], a.vocab) ? h : 0.0f;
            });
    else
        tile_product<true, false, false>(
            sums, depth, [&](int m, int64_t k) { return r0 + m < a.n_tokens && k < depth ? g.p[(r0 + m) * g.p_ld + first + k] : 0.0f; },
            [&](int n, int64_t k) { return c0 + n < a.width && k < depth ? widen(head[(first + k) * a.head_pitch + c0 + n]) : 0.0f; });
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    T* out = static_cast<T*>(of_head ? a.grad_head : a.grad_hidden);
    const int64_t pitch = of_head ? a.grad_head_pitch : a.grad_hidden_pitch;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int64_t r = r0 + ty * 4 + u, c = c0 + tx + 16 * v;
            if (r >= rows || c >= a.width) continue;
            // a token without a target has a zero row, also where the head holds what is not finite
            const float sum = of_head || is_token(a.targets[r], a.vocab) ? sums[u][v] : 0.0f;
            if (s.parts > 1) s.sums[(part * rows + r) * a.width + c] = sum;
            else out[r * pitch + c] = narrow<T>(sum);
        }
}

template <class T>
__global__ void __launch_bounds__(256) k_few_join(const float* __restrict__ sums, int parts, int64_t n, int64_t width, T* __restrict__ out, int64_t pitch) {
    ptx::chained();
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n * width; e += (int64_t)gridDim.x * 256) {
        float sum = 0.0f;
#pragma unroll 8
        for (int p = 0; p < parts; ++p) sum += sums[p * n * width + e];
        out[e / width * pitch + e % width] = narrow<T>(sum);
    }
}

struct Layout {
    float *z, *at_target;
    float2* partial;
    int64_t z_ld;
    Split head, hidden;
};

constexpr int64_t kCtas = 148 * 4;  // CTAs that keep the GPU busy
Split split(int64_t rows, int64_t depth, int64_t width, Carver& w) {
    Split s{};
    s.tiles = std::max<int64_t>(1, ceil_div(rows, kM) * ceil_div(width, kN));
    const int64_t parts = std::max<int64_t>(1, std::min(kCtas / s.tiles, ceil_div(depth, 4 * kK)));
    s.depth = round_up(ceil_div(depth, parts), kK);
    s.parts = (int)ceil_div(depth, s.depth);
    if (s.parts > 1) s.sums = w.take<float>(s.parts * rows * width);
    return s;
}

int64_t layout(int64_t n, int64_t width, int64_t vocab, bool with_grad, void* ws, Layout* out) {
    Carver w(ws);
    Layout l{};
    l.z_ld = round_up(vocab, 32);
    l.z = w.take<float>(n * l.z_ld);
    l.at_target = w.take<float>(n);
    l.partial = w.take<float2>(ceil_div(vocab, kN) * n);
    if (with_grad) {
        l.head = split(vocab, n, width, w);
        l.hidden = split(n, vocab, width, w);
    }
    if (out) *out = l;
    return w.used;
}

template <class T>
cudaError_t typed(const VocabLossArgs& a, const Layout& l, cudaStream_t s) {
    const int64_t n = a.n_tokens, parts = ceil_div(a.vocab, kN);
    const bool with_grad = a.grad_hidden || a.grad_head;
    A2_CUDA_TRY(launch_chained(k_few_logits<T>, dim3((unsigned)(parts * ceil_div(n, kM))), kFewThreads, 0, s, a, l.z, l.z_ld, l.partial, l.at_target));
    A2_CUDA_TRY(launch_rows(a, l.partial, (int)parts, l.at_target, nullptr, l.z, l.z_ld, with_grad, FewSink{l.z, l.z_ld, a.scale, a.weights}, s));
    if (!with_grad) return cudaSuccess;
    FewGradArgs g{a, l.z, l.z_ld, ceil_div(a.width, kN), l.head, l.hidden};
    if (!a.grad_head) g.head.parts = 0;
    if (!a.grad_hidden) g.hidden.parts = 0;
    A2_CUDA_TRY(launch_chained(k_few_gradients<T>, dim3((unsigned)(g.head.tiles * g.head.parts + g.hidden.tiles * g.hidden.parts)), kFewThreads, 0, s, g));
    auto join = [&](const Split& p, int64_t rows, void* out, int64_t pitch) {
        if (p.parts <= 1) return cudaSuccess;
        return launch_chained(k_few_join<T>, dim3((unsigned)std::min<int64_t>(ceil_div(rows * a.width, 256), kCtas)), 256, 0, s, p.sums, p.parts, rows,
                              a.width, static_cast<T*>(out), pitch);
    };
    A2_CUDA_TRY(join(g.head, a.vocab, a.grad_head, a.grad_head_pitch));
    return join(g.hidden, n, a.grad_hidden, a.grad_hidden_pitch);
}

}  // namespace

// Where this form is the faster one, by T V H and the head's size, gradients included (measured, us, this form / tensor cores):
// fp32 rows, T V H = 2^25 8 x 8,000 x 512: 82 / 98; 2^25.4 300 x 500 x 300: 45 / 89; 2^27 64 x 16,000 x 128: 79 / 86; 2^28 128 x 4,000 x
// 512: 122 / 99. bf16 rows need no words there, so less is gained: 2^22 32 x 1,000 x 128: 33 / 49; 2^24.6 100 x 1,000 x 256: 52 / 54; 2^25.4
// 300 x 500 x 300: 72 / 55; a large head is read faster by the copies of that form: 2^24 1 x 32,000 x 512: 304 / 101; and a wide row is a
// long chain of steps of 32 columns here, 2 us each: 2^21 64 x 64 x 512: 54 / 40.
bool vocab_loss_is_few(int64_t n, int64_t width, int64_t vocab, int32_t dtype) {
    if (n == 0 || n * vocab > (int64_t(1) << 24)) return false;
    if (dtype == A2_F32) return n * vocab * width <= int64_t(1) << 27;
    return n * vocab * width <= int64_t(1) << 24 && vocab * width <= int64_t(1) << 20 && width <= 256;
}

int64_t vocab_loss_few_workspace(int64_t n, int64_t width, int64_t vocab, bool with_grad) { return layout(n, width, vocab, with_grad, nullptr, nullptr); }

cudaError_t run_vocab_loss_few(const VocabLossArgs& a, void* workspace, cudaStream_t s) {
    Layout l;
    layout(a.n_tokens, a.width, a.vocab, a.grad_hidden || a.grad_head, workspace, &l);
    return a.dtype == A2_BF16 ? typed<__nv_bfloat16>(a, l, s) : typed<float>(a, l, s);
}

}  // namespace a2
