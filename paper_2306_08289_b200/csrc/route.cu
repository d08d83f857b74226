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
constexpr unsigned kAll = 0xffffffffu;

// Floats as unsigned integers in the same order. The sign is spread by a product rather than a shift: the pipe of shifts, comparisons and selections
// is what these kernels are short of.
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);  // -0 is 0
    int sign;
    asm("mul.hi.s32 %0, %1, 2;" : "=r"(sign) : "r"(b));
    return b ^ ((uint32_t)sign | 0x80000000u);
}
__device__ __forceinline__ float number(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

// A token's experts lie over LANES lanes of a warp (8, 16 or 32; the tokens of a warp work side by side): reductions over those.
template <int LANES, class F>
__device__ __forceinline__ F lanes_sum(F v) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d /= 2) v += __shfl_xor_sync(kAll, v, d);
    return v;
}
template <int LANES>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d /= 2) v = fmaxf(v, __shfl_xor_sync(kAll, v, d));
    return v;
}
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
    if constexpr (LANES == 32) {
        return __reduce_max_sync(kAll, v);
    } else {
#pragma unroll
        for (int d = LANES / 2; d > 0; d /= 2) v = max(v, __shfl_xor_sync(kAll, v, d));
        return v;
    }
}

// A logit (widened) as the kernels use it: -inf (no expert) for NaN and what is at or below the type's lowest value, as masks are written; of fp32 that is what its
// lowest 8 bits do not tell from it, for keys lose up to 6 of them.
template <class T>
__device__ __forceinline__ float lowest_of() {
    return sizeof(T) == 2 ? -0x1.fep127f : -0x1.fffep127f;
}
template <class T>
__device__ __forceinline__ float logit(float x) {
    return x > lowest_of<T>() ? fminf(x, FLT_MAX) : -INFINITY;
}

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }

// Approximate ones, of single instructions: off by 2^-22 of their results and by what rounding x * log2(e) does.
__device__ __forceinline__ float near_exp(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * 1.4426950408889634f));
    return y;
}
// Of the dense gradient: rows of fp32 take the accurate one, whose error does not grow with the distance from the largest logit (30,011 x 161: 14.3 us, 12.8 with the
// other); rows of bf16 keep 8 bits of it, and the approximate one is right to 2^-17 wherever it is above 2^-126 (13.5 us, 15.1 with the accurate one).
template <class T>
__device__ __forceinline__ float row_exp(float x) {
    return sizeof(T) == 4 ? expf(x) : near_exp(x);
}
__device__ __forceinline__ float near_reciprocal(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct RouteKernelArgs {
    const void* logits;
    int64_t pitch, n;
    int experts, k;
    bool sigmoid, renormalize;
    const float* bias;
    int groups, group_size, top_groups;
    int share_log, per;  // lanes of a group (a power of two), experts of a lane
    bool two_best;       // a group's score is the sum of its two best keys
    bool wide;           // a lane's logits may be read 16 bytes at a time
    float scale;
    int32_t* ids;
    float* weights;
    int32_t* counts;
};

// Better of two experts by key; the lower one where keys are equal.
__device__ __forceinline__ bool before(double key, int expert, double key2, int expert2) { return key > key2 || (key == key2 && expert < expert2); }

// Keys closer to one another than fp32 scores can tell apart: the whole choice again in 64 bits. Rare, so short rather than fast. `first` and `count` are
// this lane's experts. Lane j of a token gets the j-th expert (or -1).
template <class T, int LANES, int N>
__device__ __noinline__ int choose_in_doubt(const RouteKernelArgs& a, const T* row, int first, int count) {
    const int lane = threadIdx.x % LANES, base = threadIdx.x % 32 - lane;
    double key[N], rank[N];  // of groups and of experts
    double most = -(double)INFINITY;
    for (int j = 0; j < N; ++j) {
        rank[j] = j < count ? (double)logit<T>(widen(row[first + j])) : -(double)INFINITY;
        most = fmax(most, rank[j]);
    }
    for (int d = LANES / 2; d > 0; d /= 2) most = fmax(most, __shfl_xor_sync(kAll, most, d));
    double total = 0.0;
    for (int j = 0; j < N; ++j) {
        const bool live = rank[j] > -(double)INFINITY;
        key[j] = !live ? 0.0 : a.sigmoid ? 1.0 / (1.0 + exp(-rank[j])) : exp(rank[j] - most);
        total += key[j];
    }
    total = lanes_sum<LANES>(total);
    for (int j = 0; j < N; ++j) {
        if (!(rank[j] > -(double)INFINITY)) {
            key[j] = -(double)INFINITY;
            continue;
        }
        if (!a.sigmoid) key[j] /= total;
        if (a.bias) {
            const float bias = a.bias[first + j];
            key[j] = bias > lowest_of<T>() ? key[j] + (double)fminf(bias, FLT_MAX) : -(double)INFINITY;
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
        for (int d = (1 << a.share_log) / 2; d > 0; d /= 2) {
            const double b = __shfl_xor_sync(kAll, best, d), s = __shfl_xor_sync(kAll, second, d);
            second = fmax(fmin(best, b), fmax(second, s));
            best = fmax(best, b);
        }
        const double score = a.two_best && a.group_size > 1 ? best + second : best;
        int place = 0;
        for (int g = 0; g < a.groups; ++g) place += before(__shfl_sync(kAll, score, base + (g << a.share_log)), g, score, lane >> a.share_log);
        if (place >= a.top_groups)
            for (int j = 0; j < N; ++j) rank[j] = -(double)INFINITY;
    }
    int mine = -1;
    for (int r = 0; r < a.k; ++r) {
        double best = -(double)INFINITY;
        int expert = INT_MAX;
        for (int j = 0; j < N; ++j)
            if (rank[j] > best) best = rank[j], expert = first + j;
        for (int d = LANES / 2; d > 0; d /= 2) {
            const double b = __shfl_xor_sync(kAll, best, d);
            const int e = __shfl_xor_sync(kAll, expert, d);
            if (before(b, e, best, expert)) best = b, expert = e;
        }
        if (lane == r && expert != INT_MAX) mine = expert;
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
// LANES lanes take a token. Lane l has the experts first .. first + count of group l >> share_log in registers, as keys in 32 bits whose lowest bits are
// replaced by the expert's place in the lane (lower places larger), sorted; a round of the choice is a maximum over the heads of the lanes' lists, and the
// lowest lane that has it, which is the lowest expert. Keys are fp32 scores less those bits. Where a decision is closer than their errors, the token's experts are
// chosen again in 64 bits, so that the choice is that of exact scores; without a bias keys are the logits, and only what is equal but
// for the lost bits is in doubt. Experts are counted in shared memory and added to `counts`, which an earlier kernel has cleared (ALONE: one CTA writes
// them). Bound by instructions, nearly half of them comparisons, selections and logic, of which a multiprocessor takes two warps' a cycle: 823 a token of 256 experts
// with sigmoid scores, a bias, 8 groups and 8 choices (367 of that kind), which is 24 us of issue slots and 21 of that pipe; and by the rounds, each a chain of a reduction, a ballot and a shuffle
// with one token a warp (issue slots 63 % busy): 32,768 tokens of fp32 44 us, for 6 us of memory. Without groups 38 us, by softmax without a bias 30, one
// choice of those 20. LANES: 65,536 tokens of 64 experts, 2 chosen, over 8 lanes, four tokens a warp, 13 us; over 32 lanes 26. 256 experts over 16 lanes 58 us (lists of 16 to sort and to move).
// ---------------------------------------------------------------------------------------------
constexpr int kAloneThreads = 512;
template <int N>
constexpr int kCtasOf = N <= 8 ? 4 : N <= 16 ? 3 : 2;  // a multiprocessor, of kThreads

template <class T, int LANES, int N, bool ALONE>
__global__ void __launch_bounds__(ALONE ? kAloneThreads : kThreads, ALONE ? 1 : kCtasOf<N>) k_route(const __grid_constant__ RouteKernelArgs a) {
    constexpr int kTokens = 32 / LANES, kThreadCount = ALONE ? kAloneThreads : kThreads;  // tokens of a warp
    constexpr unsigned kSegment = LANES == 32 ? kAll : (1u << (LANES % 32)) - 1u;
    constexpr uint32_t kPlace = N - 1;
    constexpr uint32_t kNone = sizeof(T) == 4 ? 0x008000ffu : 0x0080ffffu;  // what a key is above, if its expert is available: ordered(lowest_of<T>())
    constexpr bool kSorted = N <= 16;  // longer lists: the maximum is looked for again in each round
    constexpr float kLost = N * 0x1p-23f;
    constexpr int V = 16 / sizeof(T);
    __shared__ alignas(16) float biases[LANES * N];
    extern __shared__ int counts[];
    const int lane = threadIdx.x % LANES, base = threadIdx.x % 32 - lane;
    ptx::chained();
    if (a.counts)
        for (int e = threadIdx.x; e < a.experts; e += kThreadCount) counts[e] = 0;
    auto first_of = [&](int l) { return (l >> a.share_log) * a.group_size + (l & ((1 << a.share_log) - 1)) * a.per; };
    const int group = lane >> a.share_log, first = first_of(lane);
    const int count = group < a.groups ? max(0, min(a.per, (group + 1) * a.group_size - first)) : 0;
    const bool scored = a.bias || a.two_best;
    if (threadIdx.x < LANES)  // a bias may switch an expert off like a logit
#pragma unroll
        for (int j = 0; j < N; ++j) biases[lane * N + j] = !a.bias || j >= count ? 0.0f : a.bias[first + j] > lowest_of<T>() ? fminf(a.bias[first + j], FLT_MAX) : -INFINITY;
    __syncthreads();
    const float off = a.sigmoid ? 0x1p-21f : (N + 24) * 0x1p-24f;  // of a score: approximate exponential and reciprocal, sums of N + 5 terms
    const bool exact = !a.bias;                                   // experts are ranked by their logits
    const bool checked = !exact || sizeof(T) == 4;                // bf16 logits have no bits to lose
    constexpr int64_t kStep = kThreadCount / 32 * kTokens;        // tokens of a CTA
    for (int64_t here = (int64_t)blockIdx.x * kStep; here < a.n; here += (int64_t)gridDim.x * kStep) {
        const int64_t wanted = here + threadIdx.x / LANES;
        if (here + threadIdx.x / 32 * kTokens >= a.n) break;     // none of the warp's tokens
        const int64_t token = wanted < a.n ? wanted : a.n - 1;   // a warp's last ones work along
        const T* row = static_cast<const T*>(a.logits) + token * a.pitch;
        float z[N];
        constexpr uint32_t kNothing = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;  // -inf
        if (N % V == 0 && a.wide) {
#pragma unroll
            for (int j = 0; j < N; j += V) {
                Words p{kNothing, kNothing, kNothing, kNothing};
                if (j < count) p = *reinterpret_cast<const Words*>(row + first + j);
                float f[V];
                unpack<T>(p, f);
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (j + i < N) z[j + i] = f[i];
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                z[j] = -INFINITY;
                if (j < count) z[j] = widen(row[first + j]);
            }
        }
        float most = 0.0f, total = 1.0f;
        if (!a.sigmoid && (scored || !a.renormalize)) {
#pragma unroll
            for (int j = 0; j < N; ++j) z[j] = logit<T>(z[j]);
            most = z[0];
#pragma unroll
            for (int j = 1; j < N; ++j) most = fmaxf(most, z[j]);
            most = lanes_max<LANES>(most);
            if (most == -INFINITY) most = 0.0f;
            total = 0.0f;
#pragma unroll
            for (int j = 0; j < N; ++j) total += expf(z[j] - most);
            total = lanes_sum<LANES>(total);
        }
        bool doubt = false;
        uint32_t u[N];
        auto place = [&](int j, float key) { u[j] = (ordered(key) & ~kPlace) | (kPlace - j); };
        if (a.bias) {
            const float one = 1.0f / total;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float score = a.sigmoid ? near_reciprocal(1.0f + near_exp(-z[j])) : near_exp(z[j] - most) * one;
                place(j, z[j] > lowest_of<T>() ? score + biases[lane * N + j] : -INFINITY);
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float known = fmaxf(z[j], -INFINITY);                     // NaN is -inf
                place(j, sizeof(T) == 4 ? fminf(known, FLT_MAX) : known);  // +inf the largest float, which bf16 does not have beside it
            }
        }
        if constexpr (kSorted) sort<N>(u);
        bool open = true;  // this lane's group
        auto head_of = [&] {
            uint32_t h = u[0];
            if constexpr (!kSorted) {
#pragma unroll
                for (int j = 1; j < N; ++j) h = max(h, u[j]);
            }
            return h;
        };
        if (a.groups > 1) {
            // a lane's two best keys, less the lost bits; -inf for what is not available
            auto value = [&](uint32_t v) { return v > kNone ? fminf(number(v & ~kPlace), FLT_MAX) : -INFINITY; };
            uint32_t u0 = head_of(), u1 = kSorted && N > 1 ? u[N > 1 ? 1 : 0] : 0;
            if constexpr (!kSorted) {
#pragma unroll
                for (int j = 0; j < N; ++j) u1 = u[j] == u0 ? u1 : max(u1, u[j]);
            }
            float best = value(u0), second = value(u1);
            if (scored && !a.bias) {  // lists of logits, but groups by scores
                best = second = -INFINITY;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float v = logit<T>(z[j]);
                    second = fmaxf(second, fminf(best, v));
                    best = fmaxf(best, v);
                }
                auto score = [&](float v) { return v == -INFINITY ? v : a.sigmoid ? near_reciprocal(1.0f + near_exp(-v)) : near_exp(v - most) / total; };
                best = score(best), second = score(second);
            }
            for (int d = (1 << a.share_log) / 2; d > 0; d /= 2) {
                const float b = __shfl_xor_sync(kAll, best, d);
                if (a.two_best) {
                    const float s = __shfl_xor_sync(kAll, second, d);
                    second = fmaxf(fminf(best, b), fmaxf(second, s));
                }
                best = fmaxf(best, b);
            }
            const float score = a.two_best && a.group_size > 1 ? best + second : best;
            // the best groups one after the other; a group's number in the lowest bits, so that no two are equal and the lowest is first
            uint32_t mine = group < a.groups ? (ordered(score) & ~31u) | (31 - group) : 0u, last = 0;
            open = false;
            for (int r = 0; r < a.top_groups; ++r) {
                last = lanes_max<LANES>(mine);
                if (mine == last) open = true, mine = 0;
            }
            const uint32_t next = lanes_max<LANES>(mine);
            if (a.top_groups < a.groups && (next | 31u) != (ordered(-INFINITY) | 31u)) {
                // the border's scores without 5 bits (unscored ones of bf16 have none there), of keys without those of their places
                const float in = number(last & ~31u), out = number(next & ~31u);
                doubt = !scored ? sizeof(T) == 4 && !(in - out > fabsf(in) * (2.0f * kLost + 0x1p-17f))
                                : !(in - out > 4.0f * off + fabsf(in) * (4.0f * kLost + 0x1p-17f));
            }
            // a lane whose group is closed never wins a round, so of its sorted list the head alone is looked at
#pragma unroll
            for (int j = 0; j < (kSorted ? 1 : N); ++j) u[j] = open ? u[j] : 0u;
        }
        // lane r keeps the r-th round's key and lane; all keep those of the best that is left, for the check of what was left out
        uint32_t head = head_of(), key = 0, top = 0;
        int from = 0, winner = 0;
        auto best_of_lanes = [&] {
            top = lanes_max<LANES>(head);
            const unsigned hits = __ballot_sync(kAll, (head ^ top) <= kPlace) >> base & kSegment;  // equal but for the places
            winner = __ffs(hits) - 1;
            top = __shfl_sync(kAll, head, base + winner);
        };
        for (int r = 0; r < a.k; ++r) {
            best_of_lanes();
            if (lane == r) key = top, from = winner;
            const bool won = lane == winner;
            if constexpr (kSorted) {
#pragma unroll
                for (int j = 0; j < N; ++j) u[j] = won ? (j + 1 < N ? u[j + 1] : 0u) : u[j];
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) u[j] = won && u[j] == head ? 0u : u[j];
            }
            head = head_of();
        }
        if (checked) best_of_lanes();
        const uint32_t key_next = top;
        const int from_next = winner;
        auto expert_of = [&](uint32_t key, int from) { return first_of(from) + (int)(kPlace - (key & kPlace)); };
        int mine = lane < a.k && key > kNone ? expert_of(key, from) : -1;
        if (checked) {
            // whether the better of two keys, less the lost bits, may not be so; what is equal in every respect has not been made so by rounding
            auto close = [&](uint32_t better, uint32_t worse) {
                const float low = number(worse);
                return exact ? better == worse : !(number(better) - low > 2.0f * off + fabsf(low) * (2.0f * kLost + 0x1p-22f));
            };
            auto same = [&](int x, int y) { return logit<T>(widen(row[x])) == logit<T>(widen(row[y])) && (!a.bias || a.bias[x] == a.bias[y]); };
            const uint32_t after = __shfl_down_sync(kAll, key, 1), behind = lane + 1 < a.k ? after : key_next;
            const int after_from = __shfl_down_sync(kAll, from, 1);
            bool tied = false;  // the last one that is chosen, with the first that is not
            if (mine >= 0 && behind > kNone && close(key & ~kPlace, behind & ~kPlace)) {
                const bool equal = same(mine, expert_of(behind, lane + 1 < a.k ? after_from : from_next));
                doubt = doubt || !equal;
                tied = equal && lane + 1 == a.k;
            }
            // such a tie says nothing about the others that are not chosen: those in it may hide a better one
            if (__any_sync(kAll, tied)) {
                const int last = base + a.k - 1;
                const uint32_t chosen_key = __shfl_sync(kAll, key, last) & ~kPlace;
                const int chosen = __shfl_sync(kAll, mine, last);
                if (__shfl_sync(kAll, (int)tied, last) && open)
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (u[j] > kNone && close(chosen_key, u[j] & ~kPlace) && !same(chosen, first + (int)(kPlace - (u[j] & kPlace)))) doubt = true;
            }
        }
        const unsigned doubts = __ballot_sync(kAll, doubt);
        if (doubts) {
            const int again = choose_in_doubt<T, LANES, N>(a, row, first, count);
            if (doubts >> base & kSegment) mine = lane < a.k ? again : -1;
        }
        // lane j < k: the j-th expert's weight
        const bool chosen = mine >= 0;
        const float x = chosen ? logit<T>(widen(row[mine])) : -INFINITY;
        float w;
        if (a.sigmoid) {
            w = chosen ? sigmoid(x) : 0.0f;
            if (a.renormalize) {
                float sum = lanes_sum<LANES>(w);
                const bool low = sum < 0x1p-100f;  // scores at the end of fp32's range: their ratios by their logarithms, which are then the logits
                if (__any_sync(kAll, low)) {
                    const float top = lanes_max<LANES>(x);
                    const float ratio = chosen ? expf(x - top) : 0.0f, ratios = lanes_sum<LANES>(ratio);
                    if (low) w = ratio, sum = ratios;
                }
                w = chosen ? w / sum : 0.0f;
            }
        } else if (a.renormalize) {
            const float top = lanes_max<LANES>(x);
            w = chosen ? expf(x - top) : 0.0f;
            const float sum = lanes_sum<LANES>(w);
            w = chosen ? w / sum : 0.0f;
        } else {
            w = chosen ? expf(x - most) / total : 0.0f;
        }
        if (lane < a.k && wanted < a.n) {
            a.ids[token * a.k + lane] = mine;
            a.weights[token * a.k + lane] = w * a.scale;
            if (a.counts && chosen) atomicAdd(&counts[mine], 1);
        }
    }
    if (!a.counts) return;
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += kThreadCount) {
        if (ALONE)
            a.counts[e] = counts[e];
        else if (counts[e])
            atomicAdd(&a.counts[e], counts[e]);
    }
}

__global__ void __launch_bounds__(1024) k_clear(int32_t* counts, int n) {
    ptx::chained();
    if ((int)threadIdx.x < n) counts[threadIdx.x] = 0;
}

template <class T, int LANES, int N>
cudaError_t launch_route(const RouteKernelArgs& a, cudaStream_t s) {
    const size_t counted = a.counts ? (size_t)a.experts * 4 : 0;
    if constexpr (N <= 8)  // few tokens, at most four rounds of its warps: one CTA, and no launch to clear the counts
        if (a.n <= kAloneThreads / LANES * 4 && a.n <= 64) return launch_chained(k_route<T, LANES, N, true>, dim3(1), kAloneThreads, counted, s, a);
    if (a.counts) A2_CUDA_TRY(launch_chained(k_clear, dim3(1), 1024, 0, s, a.counts, a.experts));
    const int64_t ctas = std::min<int64_t>(ceil_div(a.n, kThreads / LANES), (int64_t)multiprocessors() * kCtasOf<N>);
    return launch_chained(k_route<T, LANES, N, false>, dim3((unsigned)ctas), kThreads, counted, s, a);
}

template <class T>
cudaError_t route_typed(const RouteArgs& r, cudaStream_t s) {
    const int size = r.experts / r.groups;
    // the fewest lanes that have no more than 8 experts each, and a lane for every group and every chosen expert
    int lanes = 8, share_log = 0, per = 0;
    for (;; lanes *= 2) {
        share_log = 0;
        while ((2 << share_log) * r.groups <= lanes) ++share_log;
        per = (int)ceil_div(size, 1 << share_log);
        if (lanes == 32 || (r.groups <= lanes && r.k <= lanes && per <= 8)) break;
    }
    constexpr int V = 16 / sizeof(T);
    const bool wide = per % V == 0 && size % V == 0 && reinterpret_cast<uintptr_t>(r.logits) % 16 == 0 && r.logits_pitch % V == 0;
    const RouteKernelArgs a{r.logits, r.logits_pitch, r.n, r.experts, r.k, r.score == A2_SCORE_SIGMOID, r.renormalize, r.bias, r.groups, size, r.top_groups, share_log,
                            per, r.group_score == A2_GROUP_TWO_BEST && r.groups > 1, wide, r.scale, r.ids, r.weights, r.counts};
    if (lanes == 8) return per <= 2 ? launch_route<T, 8, 2>(a, s) : per <= 4 ? launch_route<T, 8, 4>(a, s) : launch_route<T, 8, 8>(a, s);
    if (lanes == 16) return launch_route<T, 16, 8>(a, s);
    if (per <= 8) return launch_route<T, 32, 8>(a, s);
    if (per <= 16) return launch_route<T, 32, 16>(a, s);
    if (per <= 32) return launch_route<T, 32, 32>(a, s);
    return launch_route<T, 32, 64>(a, s);  // groups that leave up to half of the lanes idle
}

// ---------------------------------------------------------------------------------------------
// Gradient. With n_j the chosen scores divided by their sum where they are renormalised and h_j = scale * g_j * s_j (n_j):
//   renormalised   d/d log s_j = n_j scale (g_j - sum_m n_m g_m), which sums to zero: the chosen logits alone have a gradient,
//                  that (softmax) or that times 1 - s_j (sigmoid);
//   sigmoid        dz_j = h_j (1 - s_j);      softmax  dz_e = [e chosen] h_e - s_e sum_m h_m for every expert.
// LANES lanes take a token, lane j its j-th chosen expert, and all of them the row of the gradient, in vectors of 16 bytes (WIDE) or element by
// element, side by side; then each chosen expert's lane writes that element once more, with the expert's own part. (Handing every expert to the lane that has
// its element takes 2 N + 2 instructions each: 30,011 x 161, softmax not renormalised, 6 chosen, 24 us that way, 13 so, both with the approximate exponential.) In place: a warp has read all that it needs of a
// token's row before it writes. With the accurate one it is 14.3 us (2.8 TB/s): rows of 161 are read and written element by element; 128 experts in whole vectors, 8 chosen and
// renormalised, 8,192 tokens: 4 us, as long as a small kernel takes.
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

template <class T, int LANES, int N, bool WIDE>
__global__ void __launch_bounds__(kThreads) k_route_grad(const __grid_constant__ RouteGradKernelArgs a) {
    constexpr int kStep = kThreads / LANES, V = WIDE ? 16 / (int)sizeof(T) : 1;
    static_assert(N % V == 0, "whole vectors");
    ptx::chained();
    const int lane = threadIdx.x % LANES, base = threadIdx.x % 32 - lane;
    auto column = [&](int j) { return (j / V * LANES + lane) * V; };  // of the vector of place j
    for (int64_t here = (int64_t)blockIdx.x * kStep; here < a.n; here += (int64_t)gridDim.x * kStep) {
        const int64_t wanted = here + threadIdx.x / LANES;
        if (here + threadIdx.x / 32 * (32 / LANES) >= a.n) break;
        const int64_t token = wanted < a.n ? wanted : a.n - 1;
        const T* row = static_cast<const T*>(a.logits) + token * a.pitch;
        T* out = static_cast<T*>(a.out) + token * a.out_pitch;
        int mine = lane < a.k ? a.ids[token * a.k + lane] : -1;
        const bool named = mine >= 0 && mine < a.experts;
        float g = named ? a.grad_weights[token * a.k + lane] * a.scale : 0.0f;
        const float x = named ? logit<T>(widen(row[mine])) : -INFINITY;
        const bool chosen = x > -INFINITY;
        if (!chosen) mine = -1, g = 0.0f;
        float d[N], h, rest = 0.0f;  // the row without the chosen experts' own part; that, and what the row has at this lane's expert
#pragma unroll
        for (int j = 0; j < N; ++j) d[j] = 0.0f;
        if (a.renormalize) {
            const float top = lanes_max<LANES>(x);
            float p = chosen ? expf(x - top) : 0.0f;
            float sum = lanes_sum<LANES>(p);
            if (a.sigmoid) {
                const float s = chosen ? sigmoid(x) : 0.0f, scores = lanes_sum<LANES>(s);
                if (!(scores < 0x1p-100f)) p = s, sum = scores;  // else ratios by the scores' logarithms, which are then the logits
            }
            p = chosen ? p / sum : 0.0f;  // the sum of a token without an expert is zero
            h = p * (g - lanes_sum<LANES>(p * g));
            if (a.sigmoid && chosen) h *= sigmoid(-x);
        } else if (a.sigmoid) {
            h = chosen ? g * sigmoid(x) * sigmoid(-x) : 0.0f;
        } else {
            float most = -INFINITY;
#pragma unroll
            for (int j = 0; j < N; j += V) {
                const bool in = column(j) < a.experts;
                float f[V];
                if constexpr (WIDE)
                    unpack<T>(in ? *reinterpret_cast<const Words*>(row + column(j)) : Words{}, f);
                else
                    f[0] = in ? widen(row[column(j)]) : 0.0f;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    d[j + i] = in ? logit<T>(f[i]) : -INFINITY;
                    most = fmaxf(most, d[j + i]);
                }
            }
            most = lanes_max<LANES>(most);
            if (most == -INFINITY) most = 0.0f;
            float total = 0.0f;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                d[j] = row_exp<T>(d[j] - most);
                total += d[j];
            }
            total = lanes_sum<LANES>(total);
            const float one = total > 0.0f ? 1.0f / total : 0.0f, s = chosen ? row_exp<T>(x - most) : 0.0f;
            h = g * s * one;
            const float all = lanes_sum<LANES>(h) * -one;
#pragma unroll
            for (int j = 0; j < N; ++j) d[j] *= all;
            rest = s * all;
        }
        // an expert that a token has twice: the first of the two lanes has their sum, in order
        const unsigned alike = __match_any_sync(kAll, chosen ? base << 16 | mine : -1 - (int)(threadIdx.x % 32));
        bool writes = chosen && wanted < a.n;
        if (__any_sync(kAll, __popc(alike) > 1)) {
            float sum = 0.0f;
            for (int c = 0; c < 32; ++c) {
                const float v = __shfl_sync(kAll, h, c);
                if (alike >> c & 1) sum += v;
            }
            h = sum;
            writes = writes && __ffs(alike) - 1 == (int)(threadIdx.x % 32);
        }
#pragma unroll
        for (int j = 0; j < N; j += V) {
            if (column(j) >= a.experts || wanted >= a.n) continue;
            if constexpr (WIDE) {
                float f[V];
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] = d[j + i];
                *reinterpret_cast<Words*>(out + column(j)) = pack<T>(f);
            } else {
                out[column(j)] = narrow<T>(d[j]);
            }
        }
        __syncwarp();  // orders the warp's writes: the chosen experts' come second
        if (writes) out[mine] = narrow<T>(rest + h);
        __syncwarp();  // and before what the next token's lanes read, where it is in place
    }
}

template <class T, int LANES, int N>
cudaError_t launch_route_grad(const RouteGradKernelArgs& a, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const bool wide = a.experts % V == 0 && a.pitch % V == 0 && a.out_pitch % V == 0 && reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 &&
                      reinterpret_cast<uintptr_t>(a.out) % 16 == 0;
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(a.n, kThreads / LANES), (int64_t)multiprocessors() * 8));
    return launch_chained(wide ? k_route_grad<T, LANES, N, true> : k_route_grad<T, LANES, N, false>, grid, kThreads, 0, s, a);
}

template <class T>
cudaError_t route_grad_typed(const RouteGradArgs& r, cudaStream_t s) {
    const RouteGradKernelArgs a{r.logits, r.logits_pitch, r.ids, r.grad_weights, r.n, r.experts, r.k, r.score == A2_SCORE_SIGMOID, r.renormalize, r.scale,
                                r.grad_logits, r.grad_logits_pitch};
    if (r.experts <= 64 && r.k <= 8) return launch_route_grad<T, 8, 8>(a, s);
    if (r.experts <= 128 && r.k <= 16) return launch_route_grad<T, 16, 8>(a, s);
    if (r.experts <= 256) return launch_route_grad<T, 32, 8>(a, s);
    if (r.experts <= 512) return launch_route_grad<T, 32, 16>(a, s);
    return launch_route_grad<T, 32, 32>(a, s);
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
