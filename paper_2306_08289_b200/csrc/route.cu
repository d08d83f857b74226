// Routing of tokens to experts and its gradient. For a token's logits z over the experts:
//   score s = softmax(z) or sigmoid(z),  key = s + bias (without a bias: z, which orders alike),
//   of the groups of experts the `top_groups` best are open (by their best key, or the sum of their two best),
//   ids = the k best keys of the open groups, the lowest expert first where keys are equal,
//   weights = scale * s (divided by the chosen scores' sum: renormalised).
#include <algorithm>
#include <cfloat>

#include "lm_ops.h"

namespace a2 {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr unsigned kAll = 0xffffffffu;

// Numbers as unsigned integers in the same order, above zero: zero stands for an expert that cannot be chosen.
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);  // -0 is 0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t ordered(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);
    return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ float number(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
__device__ __forceinline__ double number(uint64_t u) { return __longlong_as_double((long long)(u >> 63 ? u & 0x7fffffffffffffffull : ~u)); }

__device__ __forceinline__ uint32_t warp_max(uint32_t v) { return __reduce_max_sync(kAll, v); }
__device__ __forceinline__ uint64_t warp_max(uint64_t v) {
    const uint32_t high = __reduce_max_sync(kAll, (uint32_t)(v >> 32));
    const uint32_t low = __reduce_max_sync(kAll, (uint32_t)(v >> 32) == high ? (uint32_t)v : 0u);
    return (uint64_t)high << 32 | low;
}
template <class F>
__device__ __forceinline__ F warp_sum(F v) {
#pragma unroll
    for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(kAll, v, d);
    return v;
}
__device__ __forceinline__ float warp_most(float v) { return number(warp_max(ordered(v))); }

template <class F>
struct Ordered;
template <>
struct Ordered<float> {
    using Type = uint32_t;
};
template <>
struct Ordered<double> {
    using Type = uint64_t;
};

// A logit as the kernels use it: -inf (no expert) for NaN and what is at or below the type's lowest value, as masks are written.
template <class T>
__device__ __forceinline__ float logit(T v) {
    const float x = widen(v);
    return x > (sizeof(T) == 2 ? -0x1.fep127f : -FLT_MAX) ? fminf(x, FLT_MAX) : -INFINITY;
}

struct RouteKernelArgs {
    const void* logits;
    int64_t pitch, n;
    int experts, k;
    bool sigmoid, renormalize;
    const float* bias;
    int groups, group_size, top_groups;
    bool two_best;  // a group's score is the sum of its two best keys
    float scale;
    int32_t* ids;
    float* weights;
    int32_t* counts;
};

// The choice among a warp's experts: groups by their keys, experts by `rank` (the keys, or without a bias the logits). Lane j gets the j-th expert
// (or -1). Expert e lies in lane e % 32, place e / 32. `off_key` and `off_rank` bound the errors (0: exact). Returns whether a decision is
// closer than they allow.
template <class F, int N, class Same>
__device__ __forceinline__ bool choose(const RouteKernelArgs& a, const F (&key)[N], F off_key, const F (&rank_by)[N], F off_rank, const bool (&live)[N], F* staged,
                                       int& mine, const Same& same) {
    using U = typename Ordered<F>::Type;
    const int lane = threadIdx.x % 32;
    bool doubt = false;
    U u[N];
#pragma unroll
    for (int j = 0; j < N; ++j) u[j] = live[j] ? ordered(rank_by[j]) : U(0);
    if (a.groups > 1) {
        // keys through shared memory (a word in 33 left out against bank conflicts): `share` lanes look through a group
        __syncwarp();
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j * 32 + lane < a.experts) staged[j * 33 + lane] = live[j] ? key[j] : -(F)INFINITY;
        __syncwarp();
        int share = 1;
        while (share * 2 * a.groups <= 32) share *= 2;
        const int group = lane / share;
        F first = -(F)INFINITY, second = -(F)INFINITY;
        if (group < a.groups)
            for (int i = lane % share; i < a.group_size; i += share) {
                const int e = group * a.group_size + i;
                const F v = staged[e + e / 32];
                second = v > first ? first : (v > second ? v : second);
                first = v > first ? v : first;
            }
        for (int d = share / 2; d > 0; d /= 2) {
            const F f = __shfl_xor_sync(kAll, first, d), s = __shfl_xor_sync(kAll, second, d);
            const F low = f > first ? first : f;
            second = second > s ? second : s;
            second = low > second ? low : second;
            first = f > first ? f : first;
        }
        const F score = a.two_best && a.group_size > 1 ? first + second : first;
        int rank = 0;
        for (int g = 0; g < a.groups; ++g) {
            const F other = __shfl_sync(kAll, score, g * share);
            rank += other > score || (other == score && g < group);
        }
        const bool leads = group < a.groups && lane % share == 0;
        const unsigned open = __ballot_sync(kAll, leads && rank < a.top_groups);
        if (off_key > 0 && a.top_groups < a.groups) {
            const int last = __ffs(__ballot_sync(kAll, leads && rank == a.top_groups - 1)) - 1, next = __ffs(__ballot_sync(kAll, leads && rank == a.top_groups)) - 1;
            const F in = __shfl_sync(kAll, score, last), out = __shfl_sync(kAll, score, next);
            if (out > -(F)INFINITY) doubt = !(in - out > 4 * off_key + fabs(in) * (F)0x1p-21);
        }
        const uint32_t magic = (1u << 20) / a.group_size + 1;  // e / group_size for e * group_size < 2^20
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int g = (int)(((uint32_t)(j * 32 + lane) * magic) >> 20);
            if (j * 32 + lane < a.experts && !(open >> (g * share) & 1)) u[j] = 0;
        }
    }
    mine = -1;
    U best = 0;
    int at = 0;
    auto look = [&] {
        best = 0;
#pragma unroll
        for (int j = N - 1; j >= 0; --j)
            if (u[j] >= best) best = u[j], at = j;
    };
    look();
    F before = 0;
    int expert_before = -1;
    const int rounds = off_rank > 0 ? a.k + 1 : a.k;
    for (int r = 0; r < rounds; ++r) {
        const U top = warp_max(best);
        if (top == 0) break;
        const int expert = (int)__reduce_min_sync(kAll, best == top ? (unsigned)(at * 32 + lane) : 0xffffffffu);
        if (off_rank > 0) {
            const F now = number(top);
            if (r > 0 && !(before - now > 2 * off_rank + fabs(now) * (F)0x1p-22) && !same(expert_before, expert)) doubt = true;
            before = now;
            expert_before = expert;
        }
        if (r < a.k && lane == r) mine = expert;
        if (lane == expert % 32) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j == expert / 32) u[j] = 0;
            look();
        }
    }
    return doubt;
}

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }

// Keys closer to one another than fp32 scores can tell apart: the whole choice again in 64 bits. Rare.
template <class T, int N>
__device__ __noinline__ int choose_in_doubt(const RouteKernelArgs& a, const T* row, double* staged) {
    const int lane = threadIdx.x % 32;
    double z[N], key[N];
    bool live[N];
    double most = -INFINITY;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int e = j * 32 + lane;
        z[j] = e < a.experts ? (double)logit(row[e]) : -(double)INFINITY;
        live[j] = z[j] > -(double)INFINITY;
        most = fmax(most, z[j]);
    }
    if (a.sigmoid) {
#pragma unroll
        for (int j = 0; j < N; ++j) key[j] = 1.0 / (1.0 + exp(-z[j]));
    } else {
#pragma unroll
        for (int d = 16; d > 0; d /= 2) most = fmax(most, __shfl_xor_sync(kAll, most, d));
        double total = 0.0;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            key[j] = live[j] ? exp(z[j] - most) : 0.0;
            total += key[j];
        }
        total = warp_sum(total);
#pragma unroll
        for (int j = 0; j < N; ++j) key[j] = key[j] / total;
    }
    if (a.bias) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (live[j]) {
                key[j] += (double)a.bias[j * 32 + lane];
                live[j] = key[j] > -(double)INFINITY;
                key[j] = fmin(key[j], DBL_MAX);
            }
    }
    int mine;
    const auto never = [](int, int) { return false; };
    if (a.bias)
        choose<double, N>(a, key, 0.0, key, 0.0, live, staged, mine, never);
    else
        choose<double, N>(a, key, 0.0, z, 0.0, live, staged, mine, never);
    return mine;
}

// ---------------------------------------------------------------------------------------------
// A warp takes a token: its logits lie in registers, a round of the choice is a maximum over the warp and the lowest expert that has
// it. Scores are fp32; where a decision is closer than their errors, the row is chosen again in 64 bits, so that the choice is that of
// exact scores. Experts are counted in shared memory and added to `counts`, which an earlier kernel has cleared (ALONE: one CTA writes them).
// ---------------------------------------------------------------------------------------------
template <class T, int N, bool ALONE, int THREADS>
__global__ void __launch_bounds__(THREADS) k_route(const RouteKernelArgs a) {
    extern __shared__ double memory[];  // groups: a row of keys for every warp; then the counts
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int staged_words = a.groups > 1 ? N * 33 : 0;
    double* staged = memory + warp * staged_words;
    int* counts = reinterpret_cast<int*>(memory + THREADS / 32 * staged_words);
    if (ALONE) {
        ptx::chained();
    } else if (!a.counts) {
        ptx::chained();
    }  // else k_clear before it has waited for all that came before
    if (a.counts) {
        for (int e = threadIdx.x; e < a.experts; e += THREADS) counts[e] = 0;
        __syncthreads();
    }
    const float off = a.bias || a.two_best ? (a.sigmoid ? 0x1p-22f : (N + 16) * 0x1p-24f) : 0.0f;
    for (int64_t token = (int64_t)blockIdx.x * (THREADS / 32) + warp; token < a.n; token += (int64_t)gridDim.x * (THREADS / 32)) {
        const T* row = static_cast<const T*>(a.logits) + token * a.pitch;
        float z[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int e = j * 32 + lane;
            z[j] = e < a.experts ? logit(row[e]) : -INFINITY;
        }
        float most = 0.0f, total = 1.0f;
        if (!a.sigmoid && (off > 0.0f || !a.renormalize)) {
            most = z[0];
#pragma unroll
            for (int j = 1; j < N; ++j) most = fmaxf(most, z[j]);
            most = warp_most(most);
            if (most == -INFINITY) most = 0.0f;
            total = 0.0f;
#pragma unroll
            for (int j = 0; j < N; ++j) total += expf(z[j] - most);
            total = warp_sum(total);
        }
        bool live[N];
#pragma unroll
        for (int j = 0; j < N; ++j) live[j] = z[j] > -INFINITY;
        int mine;
        auto same = [&](int p, int q) {  // equal in every respect: no rounding has made them so
            return logit(row[p]) == logit(row[q]) && (!a.bias || a.bias[p] == a.bias[q]);
        };
        bool doubt = false;
        if (off > 0.0f) {
            float key[N], rank_by[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                key[j] = a.sigmoid ? sigmoid(z[j]) : expf(z[j] - most) / total;
                if (a.bias && live[j]) {
                    key[j] += a.bias[j * 32 + lane];
                    live[j] = key[j] > -INFINITY;  // a bias of -inf or NaN switches an expert off
                    key[j] = fminf(key[j], FLT_MAX);
                }
            }
            if (!a.bias) {
#pragma unroll
                for (int j = 0; j < N; ++j) rank_by[j] = z[j];
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) rank_by[j] = key[j];
            }
            doubt = choose<float, N>(a, key, off, rank_by, a.bias ? off : 0.0f, live, reinterpret_cast<float*>(staged), mine, same);
        } else {
            choose<float, N>(a, z, 0.0f, z, 0.0f, live, reinterpret_cast<float*>(staged), mine, same);
        }
        if (doubt) {
            __syncwarp();
            mine = choose_in_doubt<T, N>(a, row, staged);
        }
        // lane j < k: the j-th expert's weight
        const bool chosen = mine >= 0;
        const float x = chosen ? logit(row[mine]) : -INFINITY;
        float w;
        if (a.sigmoid) {
            w = chosen ? sigmoid(x) : 0.0f;
            if (a.renormalize) {
                float sum = warp_sum(w);
                if (sum < 0x1p-100f) {  // scores at the end of fp32's range: their ratios by their logarithms, which are then the logits
                    const float top = warp_most(x);
                    w = chosen ? expf(x - top) : 0.0f;
                    sum = warp_sum(w);
                }
                w = chosen ? w / sum : 0.0f;
            }
        } else if (a.renormalize) {
            const float top = warp_most(x);
            w = chosen ? expf(x - top) : 0.0f;
            const float sum = warp_sum(w);
            w = chosen ? w / sum : 0.0f;
        } else {
            w = chosen ? expf(x - most) / total : 0.0f;
        }
        if (lane < a.k) {
            a.ids[token * a.k + lane] = mine;
            a.weights[token * a.k + lane] = w * a.scale;
            if (a.counts && chosen) atomicAdd(&counts[mine], 1);
        }
    }
    if (!a.counts) return;
    __syncthreads();
    if (!ALONE) ptx::chained();
    for (int e = threadIdx.x; e < a.experts; e += THREADS) {
        if (ALONE)
            a.counts[e] = counts[e];
        else if (counts[e])
            atomicAdd(&a.counts[e], counts[e]);
    }
}

__global__ void __launch_bounds__(1024) k_clear(int32_t* counts, int n) {
    ptx::wait_previous();
    ptx::release_next();  // the next kernel does not wait before it reads: all it reads was done before this one
    if ((int)threadIdx.x < n) counts[threadIdx.x] = 0;
}

template <class T, int N>
cudaError_t launch_route(const RouteKernelArgs& a, cudaStream_t s) {
    const size_t staged = a.groups > 1 ? (size_t)N * 33 * 8 : 0, counted = a.counts ? (size_t)a.experts * 4 : 0;
    constexpr int64_t kAlone = N <= 8 ? 64 : 32;  // tokens of one CTA
    if (a.n <= kAlone && N <= 8) {
        constexpr int kMost = N <= 8 ? 512 : kThreads;
        return launch_chained(k_route<T, N, true, kMost>, dim3(1), kMost, staged * (kMost / 32) + counted, s, a);
    }
    if (a.counts) A2_CUDA_TRY(launch_chained(k_clear, dim3(1), 1024, 0, s, a.counts, a.experts));
    const int64_t ctas = std::min<int64_t>(ceil_div(a.n, kWarps), (int64_t)multiprocessors() * (N <= 8 ? 8 : N <= 16 ? 4 : 2));
    auto* kernel = k_route<T, N, false, kThreads>;
    const size_t smem = staged * kWarps + counted;
    if (smem > 48 * 1024)
        A2_CUDA_TRY(cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    return launch_chained(kernel, dim3((unsigned)ctas), kThreads, smem, s, a);
}

template <class T>
cudaError_t route_typed(const RouteArgs& r, cudaStream_t s) {
    const RouteKernelArgs a{r.logits, r.logits_pitch, r.n, r.experts, r.k, r.score == A2_SCORE_SIGMOID, r.renormalize, r.bias, r.groups, r.experts / r.groups,
                            r.top_groups, r.group_score == A2_GROUP_TWO_BEST && r.groups > 1, r.scale, r.ids, r.weights, r.counts};
    const int places = (r.experts + 31) / 32;
    if (places <= 1) return launch_route<T, 1>(a, s);
    if (places <= 2) return launch_route<T, 2>(a, s);
    if (places <= 4) return launch_route<T, 4>(a, s);
    if (places <= 8) return launch_route<T, 8>(a, s);
    if (places <= 16) return launch_route<T, 16>(a, s);
    return launch_route<T, 32>(a, s);
}

// ---------------------------------------------------------------------------------------------
// Gradient, a warp a token. With n_j the chosen scores divided by their sum where they are renormalised and h_j = scale * g_j * s_j (n_j):
//   renormalised   d/d log s_j = n_j scale (g_j - sum_m n_m g_m), which sums to zero: the chosen logits alone have a gradient,
//                  that (softmax) or that times 1 - s_j (sigmoid);
//   sigmoid        dz_j = h_j (1 - s_j);      softmax  dz_e = [e chosen] h_e - s_e sum_m h_m for every expert.
// ---------------------------------------------------------------------------------------------
struct RouteGradKernelArgs {
    const void* logits;
    int64_t pitch;
    const int32_t* ids;
    const float* grad_weights;
    int64_t n;
    int experts, k;
    bool sigmoid, renormalize;
    float scale;
    void* out;
    int64_t out_pitch;
};

template <class T, int N>
__global__ void __launch_bounds__(kThreads) k_route_grad(const RouteGradKernelArgs a) {
    ptx::chained();
    const int lane = threadIdx.x % 32;
    for (int64_t token = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; token < a.n; token += (int64_t)gridDim.x * kWarps) {
        const T* row = static_cast<const T*>(a.logits) + token * a.pitch;
        T* out = static_cast<T*>(a.out) + token * a.out_pitch;
        int mine = lane < a.k ? a.ids[token * a.k + lane] : -1;
        if (mine >= a.experts) mine = -1;
        const float x = mine >= 0 ? logit(row[mine]) : -INFINITY;
        const bool chosen = x > -INFINITY;
        const float g = chosen ? a.grad_weights[token * a.k + lane] * a.scale : 0.0f;
        float d[N];
#pragma unroll
        for (int j = 0; j < N; ++j) d[j] = 0.0f;
        float h;
        if (a.renormalize) {
            float p = a.sigmoid && chosen ? sigmoid(x) : 0.0f;
            float sum = a.sigmoid ? warp_sum(p) : 0.0f;
            if (sum < 0x1p-100f) {  // softmax, or scores at the end of fp32's range
                const float top = warp_most(x);
                p = chosen ? expf(x - top) : 0.0f;
                sum = warp_sum(p);
            }
            p = chosen ? p / sum : 0.0f;  // the sum of a token without an expert is zero
            h = p * (g - warp_sum(p * g));
            if (a.sigmoid && chosen) h *= sigmoid(-x);
        } else if (a.sigmoid) {
            h = chosen ? g * sigmoid(x) * sigmoid(-x) : 0.0f;
        } else {
            float most = -INFINITY;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int e = j * 32 + lane;
                d[j] = e < a.experts ? logit(row[e]) : -INFINITY;
                most = fmaxf(most, d[j]);
            }
            most = warp_most(most);
            if (most == -INFINITY) most = 0.0f;
            float total = 0.0f;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                d[j] = expf(d[j] - most);
                total += d[j];
            }
            total = warp_sum(total);
            const float one = total > 0.0f ? 1.0f / total : 0.0f;
            h = chosen ? g * expf(x - most) * one : 0.0f;
            const float all = warp_sum(h) * one;
#pragma unroll
            for (int j = 0; j < N; ++j) d[j] = -d[j] * all;
        }
        if (!chosen) mine = -1;
        for (int c = 0; c < a.k; ++c) {
            const int e = __shfl_sync(kAll, mine, c);
            const float v = __shfl_sync(kAll, h, c);
            if (e >= 0 && e % 32 == lane) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (j == e / 32) d[j] += v;
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int e = j * 32 + lane;
            if (e < a.experts) out[e] = narrow<T>(d[j]);
        }
    }
}

template <class T>
cudaError_t route_grad_typed(const RouteGradArgs& r, cudaStream_t s) {
    const RouteGradKernelArgs a{r.logits, r.logits_pitch, r.ids, r.grad_weights, r.n, r.experts, r.k, r.score == A2_SCORE_SIGMOID, r.renormalize, r.scale,
                                r.grad_logits, r.grad_logits_pitch};
    const int places = (r.experts + 31) / 32;
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(r.n, kWarps), (int64_t)multiprocessors() * 8));
    auto* kernel = places <= 1   ? k_route_grad<T, 1>
                   : places <= 2 ? k_route_grad<T, 2>
                   : places <= 4 ? k_route_grad<T, 4>
                   : places <= 8 ? k_route_grad<T, 8>
                   : places <= 16 ? k_route_grad<T, 16>
                                  : k_route_grad<T, 32>;
    return launch_chained(kernel, grid, kThreads, 0, s, a);
}

__global__ void __launch_bounds__(1024) k_no_tokens(int32_t* counts, int n) {
    ptx::chained();
    if ((int)threadIdx.x < n) counts[threadIdx.x] = 0;
}

}  // namespace

cudaError_t run_route(const RouteArgs& a, cudaStream_t s) {
    if (a.n == 0) return a.counts ? launch_chained(k_no_tokens, dim3(1), 1024, 0, s, a.counts, a.experts) : cudaSuccess;
    return a.dtype == A2_BF16 ? route_typed<__nv_bfloat16>(a, s) : route_typed<float>(a, s);
}

cudaError_t run_route_grad(const RouteGradArgs& a, cudaStream_t s) {
    if (a.n == 0) return cudaSuccess;
    return a.dtype == A2_BF16 ? route_grad_typed<__nv_bfloat16>(a, s) : route_grad_typed<float>(a, s);
}

}  // namespace a2
