// Routing of tokens to experts and its gradient. For a token's logits z over the experts:
//   score s = softmax(z) or sigmoid(z),  key = s + bias (without a bias: z, which orders alike),
//   of the groups of experts the `top_groups` best are open (by their best key, or the sum of their two best),
//   ids = the k best keys of the open groups, the lowest expert first where keys are equal,
//   weights = scale * s (divided by the chosen scores' sum: renormalised).
#include <algorithm>
#include <cfloat>
#include <climits>

#include "lm_ops.h"

namespace a2 {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr unsigned kAll = 0xffffffffu;

// Floats as unsigned integers in the same order, above zero: zero stands for an expert that cannot be chosen.
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);  // -0 is 0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float number(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

__device__ __forceinline__ uint32_t warp_max(uint32_t v) { return __reduce_max_sync(kAll, v); }
template <class F>
__device__ __forceinline__ F warp_sum(F v) {
#pragma unroll
    for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(kAll, v, d);
    return v;
}
__device__ __forceinline__ float warp_most(float v) { return number(warp_max(ordered(v))); }

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
    int share, per;  // lanes of a group (a power of two), experts of a lane
    bool two_best;   // a group's score is the sum of its two best keys
    bool wide;       // a lane's logits may be read 16 bytes at a time
    float scale;
    int32_t* ids;
    float* weights;
    int32_t* counts;
};

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }

// Better of two experts by key; the lower one where keys are equal.
__device__ __forceinline__ bool before(double key, int expert, double key2, int expert2) { return key > key2 || (key == key2 && expert < expert2); }

// Keys closer to one another than fp32 scores can tell apart: the whole choice again in 64 bits. Rare, so short rather than fast. `first` and `count` are
// this lane's experts. Lane j gets the j-th expert (or -1).
template <class T, int N>
__device__ __noinline__ int choose_in_doubt(const RouteKernelArgs& a, const T* row, int first, int count) {
    const int lane = threadIdx.x % 32;
    double key[N], rank[N];  // of groups and of experts
    double most = -(double)INFINITY;
    for (int j = 0; j < N; ++j) {
        rank[j] = j < count ? (double)logit(row[first + j]) : -(double)INFINITY;
        most = fmax(most, rank[j]);
    }
    for (int d = 16; d > 0; d /= 2) most = fmax(most, __shfl_xor_sync(kAll, most, d));
    double total = 0.0;
    for (int j = 0; j < N; ++j) {
        const bool live = rank[j] > -(double)INFINITY;
        key[j] = !live ? 0.0 : a.sigmoid ? 1.0 / (1.0 + exp(-rank[j])) : exp(rank[j] - most);
        total += key[j];
    }
    total = warp_sum(total);
    for (int j = 0; j < N; ++j) {
        if (!(rank[j] > -(double)INFINITY)) {
            key[j] = -(double)INFINITY;
            continue;
        }
        if (!a.sigmoid) key[j] /= total;
        if (a.bias) {
            key[j] += (double)a.bias[first + j];
            key[j] = key[j] > -(double)INFINITY ? fmin(key[j], DBL_MAX) : -(double)INFINITY;  // NaN: not available
            rank[j] = key[j];
        }
        if (!a.bias && !a.two_best) key[j] = rank[j];
    }
    if (a.groups > 1) {
        double best = -(double)INFINITY, second = best;
        for (int j = 0; j < N; ++j) {
            second = fmax(second, fmin(best, key[j]));
            best = fmax(best, key[j]);
        }
        for (int d = a.share / 2; d > 0; d /= 2) {
            const double b = __shfl_xor_sync(kAll, best, d), s = __shfl_xor_sync(kAll, second, d);
            second = fmax(fmin(best, b), fmax(second, s));
            best = fmax(best, b);
        }
        const double score = a.two_best && a.group_size > 1 ? best + second : best;
        int place = 0;
        for (int g = 0; g < a.groups; ++g) place += before(__shfl_sync(kAll, score, g * a.share), g, score, lane / a.share);
        if (place >= a.top_groups)
            for (int j = 0; j < N; ++j) rank[j] = -(double)INFINITY;
    }
    int mine = -1;
    for (int r = 0; r < a.k; ++r) {
        double best = -(double)INFINITY;
        int expert = INT_MAX;
        for (int j = 0; j < N; ++j)
            if (rank[j] > best) best = rank[j], expert = first + j;
        for (int d = 16; d > 0; d /= 2) {
            const double b = __shfl_xor_sync(kAll, best, d);
            const int e = __shfl_xor_sync(kAll, expert, d);
            if (before(b, e, best, expert)) best = b, expert = e;
        }
        if (expert == INT_MAX) break;
        if (lane == r) mine = expert;
        if (expert >= first && expert < first + count) rank[expert - first] = -(double)INFINITY;
    }
    return mine;
}

// Sorts descending: Batcher's odd-even merges.
template <int N>
__device__ __forceinline__ void sort(uint32_t (&u)[N]) {
#pragma unroll
    for (int p = 1; p < N; p *= 2)
#pragma unroll
        for (int q = p; q >= 1; q /= 2)
#pragma unroll
            for (int j = q % p; j + q < N; j += 2 * q)
#pragma unroll
                for (int i = 0; i < q; ++i)
                    if (j + i + q < N && (j + i) / (2 * p) == (j + i + q) / (2 * p)) {
                        const uint32_t x = u[j + i], y = u[j + i + q];
                        u[j + i] = max(x, y);
                        u[j + i + q] = min(x, y);
                    }
}

// ---------------------------------------------------------------------------------------------
// A warp takes a token. Lane l has the experts first .. first + count of group l / share in registers, as keys in 32 bits whose lowest bits are replaced by the
// expert's place in the lane (lower places larger), sorted; a round of the choice is a maximum over the heads of the lanes' lists, and the lowest lane that has
// it, which is the lowest expert. Keys are fp32 scores less those bits. Where a decision is closer than their errors, the row is chosen
// again in 64 bits, so that the choice is that of exact scores; without a bias keys are the logits, and only what is equal but for the lost bits is in
// doubt. Experts are counted in shared memory and added to `counts`, which an earlier kernel has cleared (ALONE: one CTA writes them).
// Bound by instructions: scores (two special functions an element), sorting, and about 20 for each round.
// ---------------------------------------------------------------------------------------------
constexpr int ctas_of(int n) { return n <= 8 ? 4 : n <= 16 ? 3 : 2; }  // a multiprocessor, of kThreads

template <class T, int N, bool ALONE, int THREADS>
__global__ void __launch_bounds__(THREADS, ALONE ? 1 : ctas_of(N)) k_route(const __grid_constant__ RouteKernelArgs a) {
    constexpr uint32_t kPlace = N - 1;
    constexpr bool kSorted = N <= 16;  // longer lists: the maximum is looked for again in each round
    constexpr float kLost = N * 0x1p-23f;
    constexpr int V = 16 / sizeof(T);
    extern __shared__ int counts[];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    if (ALONE || !a.counts) ptx::chained();  // else k_clear before it has waited for all that came before
    if (a.counts) {
        for (int e = threadIdx.x; e < a.experts; e += THREADS) counts[e] = 0;
        __syncthreads();
    }
    const int group = lane / a.share, skip = lane % a.share * a.per;
    const int first = group * a.group_size + skip;
    const int count = group < a.groups ? max(0, min(a.per, a.group_size - skip)) : 0;
    float bias[N];
#pragma unroll
    for (int j = 0; j < N; ++j) bias[j] = a.bias && j < count ? a.bias[first + j] : 0.0f;
    const bool scored = a.bias || a.two_best;
    const float off = a.sigmoid ? 0x1p-21f : (N + 24) * 0x1p-24f;  // of a score: approximate exponential and reciprocal, sums of N + 5 terms
    const bool exact = !a.bias;                                   // experts are ranked by their logits
    const int rounds = exact && sizeof(T) == 2 ? a.k : a.k + 1;   // bf16 logits have no bits to lose
    for (int64_t token = (int64_t)blockIdx.x * (THREADS / 32) + warp; token < a.n; token += (int64_t)gridDim.x * (THREADS / 32)) {
        const T* row = static_cast<const T*>(a.logits) + token * a.pitch;
        float z[N];
        if (N % V == 0 && a.wide) {
#pragma unroll
            for (int j = 0; j < N; j += V) {
                Pack<T, V> p;
                if (j < count) p = *reinterpret_cast<const Pack<T, V>*>(row + first + j);
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (j + i < N) z[j + i] = j < count ? logit(p.v[i]) : -INFINITY;
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) z[j] = j < count ? logit(row[first + j]) : -INFINITY;
        }
        float most = 0.0f, total = 1.0f;
        if (!a.sigmoid && (scored || !a.renormalize)) {
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
        bool doubt = false;
        uint32_t u[N];
        float best = -INFINITY, second = -INFINITY;
        if (scored) {
            const float one = 1.0f / total;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float key = (a.sigmoid ? __fdividef(1.0f, 1.0f + __expf(-z[j])) : __expf(z[j] - most) * one) + bias[j];
                // a bias of -inf or NaN switches an expert off
                const bool live = z[j] > -INFINITY && key > -INFINITY;
                key = live ? fminf(key, FLT_MAX) : -INFINITY;
                second = fmaxf(second, fminf(best, key));
                best = fmaxf(best, key);
                u[j] = !live ? 0u : (ordered(exact ? z[j] : key) & ~kPlace) | (kPlace - j);
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                best = fmaxf(best, z[j]);
                u[j] = z[j] > -INFINITY ? (ordered(z[j]) & ~kPlace) | (kPlace - j) : 0u;
            }
        }
        if (a.groups > 1) {
            for (int d = a.share / 2; d > 0; d /= 2) {
                const float b = __shfl_xor_sync(kAll, best, d), s = __shfl_xor_sync(kAll, second, d);
                second = fmaxf(fminf(best, b), fmaxf(second, s));
                best = fmaxf(best, b);
            }
            const float score = a.two_best && a.group_size > 1 ? best + second : best;
            int place = 0;
            for (int g = 0; g < a.groups; ++g) {
                const float other = __shfl_sync(kAll, score, g * a.share);
                place += other > score || (other == score && g < group);
            }
            if (scored && a.top_groups < a.groups) {
                const unsigned in = __ballot_sync(kAll, group < a.groups && place == a.top_groups - 1), out = __ballot_sync(kAll, group < a.groups && place == a.top_groups);
                const float last = __shfl_sync(kAll, score, __ffs(in) - 1), next = __shfl_sync(kAll, score, __ffs(out) - 1);
                doubt = next > -INFINITY && !(last - next > 4.0f * off + fabsf(last) * 0x1p-21f);
            }
            if (place >= a.top_groups) {
#pragma unroll
                for (int j = 0; j < N; ++j) u[j] = 0;
            }
        }
        if constexpr (kSorted) sort<N>(u);
        auto head_of = [&] {
            if constexpr (kSorted) return u[0];
            uint32_t h = u[0];
#pragma unroll
            for (int j = 1; j < N; ++j) h = max(h, u[j]);
            return h;
        };
        int mine = -1, last_expert = -1;
        uint32_t head = head_of(), last = 0;
        for (int r = 0; r < rounds; ++r) {
            const uint32_t here = head & ~kPlace;
            const uint32_t top = warp_max(here);
            if (top == 0) break;
            const int winner = __ffs(__ballot_sync(kAll, here == top)) - 1;
            const int expert = __shfl_sync(kAll, first + (int)(kPlace - (head & kPlace)), winner);
            if (r > 0) {
                const float now = number(top);
                const bool close = exact ? sizeof(T) == 4 && top == last : !(number(last) - now > 2.0f * off + fabsf(now) * (2.0f * kLost + 0x1p-22f));
                // equal in every respect: no rounding has made them so
                if (close && !(logit(row[last_expert]) == logit(row[expert]) && (!a.bias || a.bias[last_expert] == a.bias[expert]))) doubt = true;
            }
            last = top;
            last_expert = expert;
            if (r < a.k && lane == r) mine = expert;
            if (lane == winner) {
                if constexpr (kSorted) {
#pragma unroll
                    for (int j = 0; j + 1 < N; ++j) u[j] = u[j + 1];
                    u[N - 1] = 0;
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j) u[j] = u[j] == head ? 0u : u[j];
                }
                head = head_of();
            }
        }
        if (__any_sync(kAll, doubt)) mine = choose_in_doubt<T, N>(a, row, first, count);
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

constexpr int64_t kAlone = 64;  // tokens of one CTA: four rounds of its 16 warps are as long as the launch that it saves

template <class T, int N>
cudaError_t launch_route(const RouteKernelArgs& a, cudaStream_t s) {
    const size_t counted = a.counts ? (size_t)a.experts * 4 : 0;
    if constexpr (N <= 8)
        if (a.n <= kAlone) return launch_chained(k_route<T, N, true, 512>, dim3(1), 512, counted, s, a);
    if (a.counts) A2_CUDA_TRY(launch_chained(k_clear, dim3(1), 1024, 0, s, a.counts, a.experts));
    const int64_t ctas = std::min<int64_t>(ceil_div(a.n, kWarps), (int64_t)multiprocessors() * ctas_of(N));
    return launch_chained(k_route<T, N, false, kThreads>, dim3((unsigned)ctas), kThreads, counted, s, a);
}

template <class T>
cudaError_t route_typed(const RouteArgs& r, cudaStream_t s) {
    const int size = r.experts / r.groups;
    int share = 1;
    while (share * 2 * r.groups <= 32) share *= 2;
    const int per = (int)ceil_div(size, share);
    constexpr int V = 16 / sizeof(T);
    const bool wide = per % V == 0 && size % V == 0 && reinterpret_cast<uintptr_t>(r.logits) % 16 == 0 && r.logits_pitch % V == 0;
    const RouteKernelArgs a{r.logits, r.logits_pitch, r.n, r.experts, r.k, r.score == A2_SCORE_SIGMOID, r.renormalize, r.bias, r.groups, size, r.top_groups, share, per,
                            r.group_score == A2_GROUP_TWO_BEST && r.groups > 1, wide, r.scale, r.ids, r.weights, r.counts};
    if (per <= 1) return launch_route<T, 1>(a, s);
    if (per <= 2) return launch_route<T, 2>(a, s);
    if (per <= 4) return launch_route<T, 4>(a, s);
    if (per <= 8) return launch_route<T, 8>(a, s);
    if (per <= 16) return launch_route<T, 16>(a, s);
    if (per <= 32) return launch_route<T, 32>(a, s);
    return launch_route<T, 64>(a, s);  // groups that leave up to half of the lanes idle
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
__global__ void __launch_bounds__(kThreads) k_route_grad(const __grid_constant__ RouteGradKernelArgs a) {
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
            const int place = e >= 0 && e % 32 == lane ? e / 32 : N;
#pragma unroll
            for (int j = 0; j < N; ++j) d[j] += j == place ? v : 0.0f;
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
