// Softmax cross entropy over a large vocabulary, in pieces of the vocabulary, with its gradients:
//   z_tv = <h_t, W_v>, lse_t = log sum_v exp z_tv, loss_t = lse_t - z_ty,
//   P_tv = g_t (exp(z_tv - lse_t) - [v = y_t]), dh = P W, dW = P^T h.
// Four products of 2 T V H operations (three without the recomputed logits), all on the tensor cores; the logits
// live in tensor memory only. The first product's epilogue keeps each token's maximum and sum of exponentials of 128 columns;
// k_finish joins them. The gradient goes through the vocabulary in pieces: logits again, P of the piece into the workspace as
// the 16-bit operand of the other two products.
#include <algorithm>

#include "gemm_sm100.cuh"

namespace a2 {

namespace {

constexpr float kLog2E = 1.4426950408889634f;
constexpr int kPScale = 14;  // P / max |P| <= 1 is held at this power of two with fp32 rows

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Scalars found by k_scan, as bits of non-negative floats (their order is that of the bits).
struct Scan {
    uint32_t hidden, head, weight;  // largest finite magnitude of each
};

// The power of two that puts `amax` into [2^14, 2^15).
__device__ __forceinline__ int word_exponent(uint32_t amax_bits) { return amax_bits ? 14 - ilogbf(__uint_as_float(amax_bits)) : 0; }

// v * 2^e in two factors, so that no intermediate leaves the range unless the result does.
struct PowerOfTwo {
    float a, b;
    __device__ __forceinline__ explicit PowerOfTwo(int e) {
        e = max(-250, min(250, e));
        a = ldexpf(1.0f, e / 2);
        b = ldexpf(1.0f, e - e / 2);
    }
    __device__ __forceinline__ float operator()(float v) const { return v * a * b; }
};

__device__ __forceinline__ bool is_token(int32_t y, int64_t vocab) { return y >= 0 && y < vocab; }

// ---- operands -----------------------------------------------------------------------------------
struct PrepareArgs {
    const void* hidden;
    const void* head;
    const int32_t* targets;
    const float* weights;
    int64_t n, width, vocab, hidden_pitch, head_pitch;
    Scan* scan;          // NULL: neither fp32 rows nor weights
    void *h0, *h1;       // hidden's words [n, ld] (h1 NULL with bf16 rows), or NULL: not wanted
    void *w0, *w1;       // head's words [vocab, ld], or NULL
    int64_t ld;
    float* rate;         // g_t / max |g|, 0 for tokens without a target; NULL without gradients
    int32_t* poisoned;   // tokens without a target whose hidden row is not finite: the row is taken as zero, its lse as NaN
};

template <class T>
__device__ __forceinline__ uint32_t scan_rows(const T* p, int64_t rows, int64_t width, int64_t pitch, int64_t warp, int64_t warps) {
    uint32_t most = 0;
    for (int64_t r = warp; r < rows; r += warps)
        for (int64_t c = threadIdx.x % 32; c < width; c += 32) {
            const uint32_t bits = __float_as_uint(fabsf(widen(p[r * pitch + c])));
            if (bits < 0x7f800000u) most = max(most, bits);
        }
    return most;
}

__device__ __forceinline__ void publish(uint32_t most, uint32_t* to) {
    most = __reduce_max_sync(0xffffffffu, most);
    if (threadIdx.x % 32 == 0 && most) atomicMax(to, most);
}

// Largest finite magnitudes. The head's and hidden's are needed for fp32 rows alone.
template <class T>
__global__ void __launch_bounds__(256) k_scan(PrepareArgs a) {
    const int64_t warp = (int64_t)blockIdx.x * 8 + threadIdx.x / 32, warps = (int64_t)gridDim.x * 8;
    if (sizeof(T) == 4) {
        publish(scan_rows(static_cast<const T*>(a.hidden), a.n, a.width, a.hidden_pitch, warp, warps), &a.scan->hidden);
        publish(scan_rows(static_cast<const T*>(a.head), a.vocab, a.width, a.head_pitch, warp, warps), &a.scan->head);
    }
    if (a.weights) {
        uint32_t most = 0;
        for (int64_t t = warp * 32 + threadIdx.x % 32; t < a.n; t += warps * 32) {
            const uint32_t bits = __float_as_uint(fabsf(a.weights[t]));
            if (is_token(a.targets[t], a.vocab) && bits < 0x7f800000u) most = max(most, bits);
        }
        publish(most, &a.scan->weight);
    }
}

__device__ __forceinline__ void split_words(float x, __half& hi, __half& lo) {
    hi = __float2half_rn(x);
    const float back = __half2float(hi);
    lo = __float2half_rn(isfinite(back) ? x - back : 0.0f);
}

template <class T>
__device__ __forceinline__ void pack_row(const T* from, void* to0, void* to1, int64_t at, int64_t width, int64_t ld, int e, bool zero) {
    for (int64_t c = threadIdx.x % 32; c < width; c += 32) {
        const float x = zero ? 0.0f : widen(from[c]);
        if constexpr (sizeof(T) == 4) {
            __half hi, lo;
            split_words(scalbnf(x, e), hi, lo);
            static_cast<__half*>(to0)[at * ld + c] = hi;
            static_cast<__half*>(to1)[at * ld + c] = lo;
        } else {
            static_cast<__nv_bfloat16*>(to0)[at * ld + c] = narrow<__nv_bfloat16>(x);
        }
    }
}

// The operands of the products in the workspace, a warp a row: two words of fp32 rows, a copy of bf16 ones where
// TMA cannot read them in place. A token without a target must add nothing to dW = P^T h: 0 * NaN would, so such a row of hidden
// becomes zero when it holds anything that is not finite.
template <class T>
__global__ void __launch_bounds__(256) k_pack(PrepareArgs a) {
    const int64_t warp = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    if (warp < a.n) {
        const bool live = is_token(a.targets[warp], a.vocab);
        if (a.rate && threadIdx.x % 32 == 0) {
            const float most = a.weights ? __uint_as_float(a.scan->weight) : 1.0f;
            a.rate[warp] = !live ? 0.0f : !a.weights ? 1.0f : most > 0.0f ? a.weights[warp] / most : a.weights[warp];
        }
        if (!a.h0) return;
        const T* from = static_cast<const T*>(a.hidden) + warp * a.hidden_pitch;
        bool bad = false;
        if (!live) {
            for (int64_t c = threadIdx.x % 32; c < a.width; c += 32) bad |= !isfinite(widen(from[c]));
            bad = __any_sync(0xffffffffu, bad);
        }
        if (threadIdx.x % 32 == 0) a.poisoned[warp] = bad;
        pack_row(from, a.h0, a.h1, warp, a.width, a.ld, a.h1 ? word_exponent(a.scan->hidden) : 0, bad);
    } else if (a.w0 && warp - a.n < a.vocab) {
        const int64_t v = warp - a.n;
        pack_row(static_cast<const T*>(a.head) + v * a.head_pitch, a.w0, a.w1, v, a.width, a.ld, a.w1 ? word_exponent(a.scan->head) : 0, false);
    }
}

// ---- epilogues ----------------------------------------------------------------------------------
// Statistics of 128 columns of one token, by one thread.
template <bool kWords>
struct StatisticsEpi {
    struct Args {
        float2* partial;  // [2 * tile columns][n]: maximum, sum of exp(z - maximum)
        float* at_target;
        const int32_t* targets;
        const Scan* scan;
        int64_t n, vocab;
    };
    const Args& a;
    int64_t row, col0;
    int64_t target;
    float top = -INFINITY, sum = 0.0f;
    PowerOfTwo unscale;
    __device__ __forceinline__ StatisticsEpi(const Args& args, int, int row0, int col, int lane, float*)
        : a(args), row((int64_t)row0 + lane), col0(col), unscale(kWords ? -(word_exponent(args.scan->hidden) + word_exponent(args.scan->head)) : 0) {
        target = row < a.n ? a.targets[row] : -1;
    }
    __device__ __forceinline__ void chunk(int c, float (&v)[32]) {
        const int64_t col = col0 + c * 32;
        if (kWords)
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] = unscale(v[k]);
        if (col + 32 > a.vocab)
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (col + k >= a.vocab) v[k] = -INFINITY;
        if (target >= col && target < col + 32 && target < a.vocab) {
            float z = 0.0f;
#pragma unroll
            for (int k = 0; k < 32; ++k) z = target == col + k ? v[k] : z;
            a.at_target[row] = z;
        }
        float most = v[0];
#pragma unroll
        for (int k = 1; k < 32; ++k) most = fmaxf(most, v[k]);
        const float next = fmaxf(top, most);
        const float base = next == -INFINITY ? 0.0f : next;
        float part[4] = {};
#pragma unroll
        for (int k = 0; k < 32; ++k) part[k % 4] += exp2_fast((v[k] - base) * kLog2E);
        sum = sum * exp2_fast((top - base) * kLog2E) + ((part[0] + part[1]) + (part[2] + part[3]));
        top = next;
    }
    __device__ __forceinline__ void finish() {
        if (row < a.n) a.partial[(col0 / 128) * a.n + row] = make_float2(top, sum);
    }
};

// P of a piece, as the 16-bit operand of the gradients' products: row-major [n, ld], which dh = P W reads K-major and
// dW = P^T h reads MN-major.
template <bool kWords>
struct ProbabilityEpi {
    struct Args {
        void *p0, *p1;
        int64_t ld;
        const int32_t* targets;
        const float* lse;
        const float* rate;
        const Scan* scan;
        int64_t n, vocab, v0;
    };
    const Args& a;
    int64_t row, col0;
    int64_t target;
    float lse = 0.0f, rate = 0.0f;
    PowerOfTwo unscale;
    __device__ __forceinline__ ProbabilityEpi(const Args& args, int, int row0, int col, int lane, float*)
        : a(args), row((int64_t)row0 + lane), col0(col), unscale(kWords ? -(word_exponent(args.scan->hidden) + word_exponent(args.scan->head)) : 0) {
        target = -1;
        if (row < a.n) {
            lse = a.lse[row];
            rate = a.rate[row];
            const int64_t y = a.targets[row];
            if (is_token((int32_t)y, a.vocab)) target = y - a.v0;
            else rate = 0.0f;
        }
    }
    __device__ __forceinline__ void chunk(int c, float (&v)[32]) {
        if (row >= a.n) return;
        const int64_t col = col0 + c * 32;
        const bool live = target >= 0 || rate != 0.0f;
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            const float z = kWords ? unscale(v[k]) : v[k];
            float p = exp2_fast((z - lse) * kLog2E);
            p = rate * (target == col + k ? p - 1.0f : p);
            v[k] = live ? p : 0.0f;
        }
        const int64_t at = row * a.ld + col;
        if constexpr (kWords) {
            Pack<__half, 16> hi, lo;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
#pragma unroll
                for (int k = 0; k < 16; ++k) split_words(v[g * 16 + k] * (float)(1 << kPScale), hi.v[k], lo.v[k]);
                *reinterpret_cast<Pack<__half, 16>*>(static_cast<__half*>(a.p0) + at + g * 16) = hi;
                *reinterpret_cast<Pack<__half, 16>*>(static_cast<__half*>(a.p1) + at + g * 16) = lo;
            }
        } else {
            Pack<__nv_bfloat16, 16> o;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
#pragma unroll
                for (int k = 0; k < 16; ++k) o.v[k] = narrow<__nv_bfloat16>(v[g * 16 + k]);
                *reinterpret_cast<Pack<__nv_bfloat16, 16>*>(static_cast<__nv_bfloat16*>(a.p0) + at + g * 16) = o;
            }
        }
    }
    __device__ __forceinline__ void finish() {}
};

// A gradient's tile: out = factor * (sums of the earlier pieces + this one), or those sums kept for the next piece.
template <class T>
struct GradientEpi {
    struct Args {
        T* out;  // NULL: keep
        int64_t pitch, rows, cols;
        float* kept;  // [rows, kept_ld], or NULL with a single piece
        int64_t kept_ld;
        bool add;  // kept holds earlier pieces
        const Scan* scan;
        bool of_hidden;  // which word scale the other operand has: grad_hidden's is head's
        bool weighted;
        float scale;
    };
    const Args& a;
    int64_t row0, col0;
    int lane;
    float* staging;
    float last;
    PowerOfTwo unscale;
    static __device__ __forceinline__ int exponent(const Args& a) {
        if (sizeof(T) != 4) return 0;
        return -(kPScale + word_exponent(a.of_hidden ? a.scan->head : a.scan->hidden));
    }
    __device__ __forceinline__ GradientEpi(const Args& args, int, int row, int col, int lane_, float* staging_)
        : a(args), row0(row), col0(col), lane(lane_), staging(staging_), unscale(exponent(args)) {
        const float most = a.weighted ? __uint_as_float(a.scan->weight) : 1.0f;
        last = a.scale * (most > 0.0f ? most : 1.0f);
    }
    __device__ __forceinline__ void chunk(int c, float (&v)[32]) {
        const int64_t col = col0 + c * 32, row = row0 + lane;
        if (a.kept && row < a.rows) {  // kept_ld is a multiple of 256: no column check
            float* k = a.kept + row * a.kept_ld + col;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                Pack<float, 8>* at = reinterpret_cast<Pack<float, 8>*>(k + g * 8);
                Pack<float, 8> o;
                if (a.add) o = *at;
#pragma unroll
                for (int e = 0; e < 8; ++e) o.v[e] = v[g * 8 + e] = a.add ? o.v[e] + v[g * 8 + e] : v[g * 8 + e];
                if (!a.out) *at = o;
            }
        }
        if (!a.out) return;
        // through shared memory, so that a row's 32 columns are written side by side whatever the alignment
#pragma unroll
        for (int k = 0; k < 32; ++k) staging[lane * kStagePitch + k] = sizeof(T) == 4 ? unscale(v[k]) * last : v[k] * last;
        __syncwarp();
        if (col + lane < a.cols) {
            T* to = a.out + row0 * a.pitch + col + lane;
            const int rows = (int)min((int64_t)32, a.rows - row0);
#pragma unroll 8
            for (int r = 0; r < rows; ++r) to[r * a.pitch] = narrow<T>(staging[r * kStagePitch + lane]);
        }
        __syncwarp();
    }
    __device__ __forceinline__ void finish() {}
};

// Joins the statistics of the parts: 32 tokens a CTA, eight warps over the parts.
__global__ void __launch_bounds__(256) k_finish(const float2* __restrict__ partial, int parts, const float* __restrict__ at_target,
                                                const int32_t* __restrict__ targets, const int32_t* __restrict__ poisoned, int64_t n, int64_t vocab,
                                                float* __restrict__ loss, float* __restrict__ lse) {
    __shared__ float2 joined[8][32];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t t = (int64_t)blockIdx.x * 32 + lane;
    float top = -INFINITY, sum = 0.0f;
    auto join = [&](float2 p) {
        const float next = fmaxf(top, p.x);
        const float base = next == -INFINITY ? 0.0f : next;
        sum = sum * exp2_fast((top - base) * kLog2E) + p.y * exp2_fast((p.x - base) * kLog2E);
        top = next;
    };
    if (t < n)
#pragma unroll 4
        for (int p = warp; p < parts; p += 8) join(partial[(int64_t)p * n + t]);
    joined[warp][lane] = make_float2(top, sum);
    __syncthreads();
    if (warp == 0 && t < n) {
        for (int w = 1; w < 8; ++w) join(joined[w][lane]);
        const float l = poisoned && poisoned[t] ? NAN : top + logf(sum);
        lse[t] = l;
        loss[t] = is_token(targets[t], vocab) ? l - at_target[t] : 0.0f;
    }
}

// ---- layout and launches ------------------------------------------------------------------------
constexpr int kFlush = 8;  // K blocks a promoted sum stays in tensor memory: 32 steps of the tensor core

struct Layout {
    Scan* scan;
    void *h0, *h1, *w0, *w1, *p0, *p1;
    float2* partial;
    float *at_target, *rate, *kept;
    int32_t* poisoned;
    int64_t ld, p_ld, kept_ld, piece;
};

// Vocabulary rows of a piece: as many as keep P within kPieceBytes, fewer where that fills the pairs of CTAs better.
// Cost in units of (tile of 256 x 256) x (K of 256) a pair.
constexpr int64_t kPieceBytes = 160ll << 20;
constexpr int64_t kPairs = 74;
int64_t piece_rows(int64_t n, int64_t width, int64_t vocab, int64_t words) {
    const int64_t tm = std::max<int64_t>(1, ceil_div(n, kTileM)), tw = ceil_div(width, kTileN), tv = ceil_div(vocab, kTileN);
    const int64_t most = std::min(tv, std::max<int64_t>(1, kPieceBytes / (tm * kTileM * kTileN * 2 * words)));
    int64_t best = most, least = INT64_MAX;
    for (int64_t q = most; q >= std::max<int64_t>(1, most / 2); --q) {
        const int64_t pieces = ceil_div(tv, q);
        const int64_t cost = pieces * (ceil_div(tm * q, kPairs) * tw + ceil_div(tm * tw, kPairs) * q + ceil_div(q * tw, kPairs) * tm);
        if (cost < least) least = cost, best = q;
    }
    return best * kTileN;
}

int64_t layout(int64_t n, int64_t width, int64_t vocab, bool with_grad, int32_t dtype, void* ws, Layout* out) {
    const int64_t words = dtype == A2_F32 ? 2 : 1;
    Carver w(ws);
    Layout l{};
    l.ld = round_up(width, 64);
    l.scan = w.take<Scan>(1);
    l.h0 = w.take<uint16_t>(n * l.ld);
    l.w0 = w.take<uint16_t>(vocab * l.ld);
    if (words == 2) {
        l.h1 = w.take<uint16_t>(n * l.ld);
        l.w1 = w.take<uint16_t>(vocab * l.ld);
    }
    l.partial = w.take<float2>(2 * ceil_div(vocab, kTileN) * n);
    l.at_target = w.take<float>(n);
    l.poisoned = w.take<int32_t>(n);
    if (with_grad) {
        l.piece = piece_rows(n, width, vocab, words);
        l.p_ld = l.piece;
        l.rate = w.take<float>(n);
        l.p0 = w.take<uint16_t>(n * l.p_ld);
        if (words == 2) l.p1 = w.take<uint16_t>(n * l.p_ld);
        l.kept_ld = round_up(width, kTileN);
        if (l.piece < vocab) l.kept = w.take<float>(n * l.kept_ld);
    }
    if (out) *out = l;
    return w.used;
}

template <class T>
cudaError_t typed(const VocabLossArgs& a, Layout l, cudaStream_t s) {
    constexpr bool kWords = sizeof(T) == 4;
    const int64_t n = a.n_tokens;
    const bool with_grad = a.grad_hidden || a.grad_head;
    cudaError_t e = cudaSuccess;
    if (n == 0) {
        if (!a.grad_head) return cudaSuccess;
        return cudaMemset2DAsync(a.grad_head, a.grad_head_pitch * sizeof(T), 0, a.width * sizeof(T), a.vocab, s);
    }
    // operands: in place where TMA can read them (bf16, 16-byte rows), else from the workspace
    auto in_place = [](const void* p, int64_t pitch) { return !kWords && reinterpret_cast<uintptr_t>(p) % 16 == 0 && pitch % 8 == 0; };
    const bool hidden_in_place = in_place(a.hidden, a.hidden_pitch) && !a.grad_head;
    const bool head_in_place = in_place(a.head, a.head_pitch);
    PrepareArgs prep{a.hidden, a.head, a.targets, a.weights, n, a.width, a.vocab, a.hidden_pitch, a.head_pitch, nullptr, nullptr, nullptr,
                     nullptr,  nullptr, l.ld, with_grad ? l.rate : nullptr, l.poisoned};
    const bool weighted = with_grad && a.weights;
    if (!with_grad) prep.weights = nullptr;
    if (kWords || weighted) prep.scan = l.scan;
    if (!hidden_in_place) prep.h0 = l.h0, prep.h1 = l.h1;
    if (!head_in_place) prep.w0 = l.w0, prep.w1 = l.w1;
    if (prep.scan) {
        e = cudaMemsetAsync(l.scan, 0, sizeof(Scan), s);
        if (e != cudaSuccess) return e;
        const int64_t rows = kWords ? n + a.vocab : ceil_div(n, 32);
        k_scan<T><<<(unsigned)std::min<int64_t>(ceil_div(rows, 8), 148 * 8), 256, 0, s>>>(prep);
    }
    if (prep.h0 || prep.w0 || prep.rate) k_pack<T><<<(unsigned)ceil_div(n + (prep.w0 ? a.vocab : 0), 8), 256, 0, s>>>(prep);

    auto words = [&](const void* mine, void* w0, void* w1, bool here, int64_t pitch, int64_t row0, int64_t rows, int64_t cols, bool mn) {
        // rows x cols from row0 on; K-major: rows are M or N and columns K; MN-major: the other way round
        const int64_t ld = here ? pitch : l.ld;
        const uint16_t* p = static_cast<const uint16_t*>(here ? mine : w0) + row0 * ld;
        const uint16_t* lo = kWords ? static_cast<const uint16_t*>(w1) + row0 * ld : nullptr;
        return Operand{p, lo, mn ? cols : rows, mn ? rows : cols, ld, 0, mn};
    };
    auto hidden = [&](bool mn) { return words(a.hidden, l.h0, l.h1, hidden_in_place, a.hidden_pitch, 0, n, a.width, mn); };
    auto head = [&](int64_t v0, int64_t rows, bool mn) { return words(a.head, l.w0, l.w1, head_in_place, a.head_pitch, v0, rows, a.width, mn); };
    const int flush = kWords ? kFlush : 0;

    GemmArgs g;
    // the loss is fp32 with either storage type, so its sums are promoted with both
    e = make_gemm(hidden(false), head(0, a.vocab, false), 1, !kWords, false, kFlush, &g);
    if (e != cudaSuccess) return e;
    const typename StatisticsEpi<kWords>::Args stats{l.partial, l.at_target, a.targets, l.scan, n, a.vocab};
    e = launch_gemm<StatisticsEpi<kWords>, true>(g, stats, s);
    if (e != cudaSuccess) return e;
    k_finish<<<(unsigned)ceil_div(n, 32), 256, 0, s>>>(l.partial, (int)(2 * ceil_div(a.vocab, kTileN)), l.at_target, a.targets,
                                                      hidden_in_place ? nullptr : l.poisoned, n, a.vocab, a.loss, a.lse);
    if (!with_grad) return cudaGetLastError();

    for (int64_t v0 = 0; v0 < a.vocab; v0 += l.piece) {
        const int64_t rows = std::min(l.piece, a.vocab - v0);
        const bool first = v0 == 0, final = v0 + rows == a.vocab;
        e = make_gemm(hidden(false), head(v0, rows, false), 1, !kWords, false, flush, &g);
        if (e != cudaSuccess) return e;
        const typename ProbabilityEpi<kWords>::Args prob{l.p0, l.p1, l.p_ld, a.targets, a.lse, l.rate, l.scan, n, a.vocab, v0};
        e = launch_gemm<ProbabilityEpi<kWords>, kWords>(g, prob, s);
        if (e != cudaSuccess) return e;
        if (a.grad_head) {
            const Operand p{l.p0, l.p1, rows, n, l.p_ld, 0, true};
            e = make_gemm(p, hidden(true), 1, !kWords, false, flush, &g);
            if (e != cudaSuccess) return e;
            const typename GradientEpi<T>::Args grad{static_cast<T*>(a.grad_head) + v0 * a.grad_head_pitch, a.grad_head_pitch, rows, a.width, nullptr,
                                                     0, false, l.scan, false, weighted, a.scale};
            e = launch_gemm<GradientEpi<T>, kWords>(g, grad, s);
            if (e != cudaSuccess) return e;
        }
        if (a.grad_hidden) {
            const Operand p{l.p0, l.p1, n, rows, l.p_ld, 0, false};
            e = make_gemm(p, head(v0, rows, true), 1, !kWords, false, flush, &g);
            if (e != cudaSuccess) return e;
            const typename GradientEpi<T>::Args grad{final ? static_cast<T*>(a.grad_hidden) : nullptr, a.grad_hidden_pitch, n, a.width,
                                                     first && final ? nullptr : l.kept, l.kept_ld, !first, l.scan, true, weighted, a.scale};
            e = launch_gemm<GradientEpi<T>, kWords>(g, grad, s);
            if (e != cudaSuccess) return e;
        }
    }
    return cudaGetLastError();
}

}  // namespace

int64_t vocab_loss_workspace(int64_t n_tokens, int64_t width, int64_t vocab, bool with_grad, int32_t dtype) {
    return layout(n_tokens, width, vocab, with_grad, dtype, nullptr, nullptr);
}

cudaError_t run_vocab_loss(const VocabLossArgs& a, void* workspace, cudaStream_t s) {
    Layout l;
    layout(a.n_tokens, a.width, a.vocab, a.grad_hidden || a.grad_head, a.dtype, workspace, &l);
    return a.dtype == A2_BF16 ? typed<__nv_bfloat16>(a, l, s) : typed<float>(a, l, s);
}

}  // namespace a2
