// Softmax cross entropy over a large vocabulary, in pieces of the vocabulary, with its gradients:
//   z_tv = <h_t, W_v>, lse_t = log sum_v exp z_tv, loss_t = lse_t - z_ty,
//   P_tv = g_t (exp(z_tv - lse_t) - [v = y_t]), dh = P W, dW = P^T h.
// Four products of 2 T V H operations (three without the recomputed logits), all on the tensor cores; the logits
// live in tensor memory only (a few of them, 64 MB at most, are kept where that is faster). The first product's epilogue keeps each token's maximum and sum of exponentials of 128 columns;
// k_finish joins them. The gradient goes through the vocabulary in pieces: logits again, P of the piece into the workspace as
// the 16-bit operand of the other two products.
#include <algorithm>
#include <type_traits>

#include "gemm_sm100.cuh"
#include "vocab_loss.cuh"

namespace a2 {

namespace {

constexpr int kPScale = 14;  // P / max |P| <= 1 is held at this power of two with fp32 rows

// Largest finite magnitudes, as bits of non-negative floats (their order is that of the bits): of a CTA of k_scan, or of all.
struct alignas(16) Scan {
    uint32_t hidden, head, weight;  // hidden: of the tokens with a target
};
constexpr int kScanCtas = 148, kScanThreads = 1024;

// The power of two that puts `amax` into [2^14, 2^15).
__device__ __forceinline__ int word_exponent(uint32_t amax_bits) { return amax_bits ? 14 - ilogbf(__uint_as_float(amax_bits)) : 0; }

// ---- operands -----------------------------------------------------------------------------------
struct PrepareArgs {
    const void* hidden;
    const void* head;
    const int32_t* targets;
    const float* weights;
    int64_t n, width, vocab, hidden_pitch, head_pitch;
    Scan* scan;          // NULL: neither fp32 rows nor weights
    Scan* scan_parts;    // [kScanCtas]
    void *h0, *h1;       // hidden's words [n, ld] (h1 NULL with bf16 rows), or NULL: not wanted
    void *w0, *w1;       // head's words [vocab, ld], or NULL
    int64_t ld;
    float* rate;         // g_t / max |g|, 0 for tokens without a target; NULL without gradients
    bool hidden_fours, head_fours;  // four columns can be read at once
    int32_t* exponents;  // of the words of each row of hidden
    int32_t* poisoned;   // tokens without a target whose hidden row is not finite: the row is taken as zero, its lse as NaN
};

template <class T>
__device__ __forceinline__ uint32_t scan_rows(const T* p, bool aligned, int64_t rows, int64_t width, int64_t pitch, int64_t warp, int64_t warps,
                                              const int32_t* targets, int64_t vocab) {
    uint32_t most = 0;
    auto see = [&](T x) {
        const uint32_t bits = __float_as_uint(fabsf(widen(x)));
        if (bits < 0x7f800000u) most = max(most, bits);
    };
    for (int64_t r = warp; r < rows; r += warps) {
        if (targets && !is_token(targets[r], vocab)) continue;
        const T* row = p + r * pitch;
        if (aligned) {
            int64_t c = threadIdx.x % 32 * 4;
#pragma unroll 4
            for (; c + 4 <= width; c += 128) {
                const Pack<T, 4> x = *reinterpret_cast<const Pack<T, 4>*>(row + c);
#pragma unroll
                for (int k = 0; k < 4; ++k) see(x.v[k]);
            }
            for (int k = 0; k < 4 && c + k < width; ++k) see(row[c + k]);
        } else {
#pragma unroll 8
            for (int64_t c = threadIdx.x % 32; c < width; c += 32) see(row[c]);
        }
    }
    return most;
}

// The head's and hidden's are needed for fp32 rows alone.
template <class T>
__global__ void __launch_bounds__(kScanThreads) k_scan(PrepareArgs a) {
    ptx::chained();
    __shared__ Scan warps_found[kScanThreads / 32];
    const int64_t warp = (int64_t)blockIdx.x * (kScanThreads / 32) + threadIdx.x / 32, warps = (int64_t)gridDim.x * (kScanThreads / 32);
    Scan most{};
    if (sizeof(T) == 4) {
        most.hidden = scan_rows(static_cast<const T*>(a.hidden), a.hidden_fours, a.n, a.width, a.hidden_pitch, warp, warps,
                                a.targets, a.vocab);
        most.head = scan_rows(static_cast<const T*>(a.head), a.head_fours, a.vocab, a.width, a.head_pitch, warp, warps, nullptr, 0);
    }
    if (a.weights)
        for (int64_t t = warp * 32 + threadIdx.x % 32; t < a.n; t += warps * 32) {
            const uint32_t bits = __float_as_uint(fabsf(a.weights[t]));
            if (is_token(a.targets[t], a.vocab) && bits < 0x7f800000u) most.weight = max(most.weight, bits);
        }
    auto reduce = [](Scan& m) {
        m.hidden = __reduce_max_sync(0xffffffffu, m.hidden);
        m.head = __reduce_max_sync(0xffffffffu, m.head);
        m.weight = __reduce_max_sync(0xffffffffu, m.weight);
    };
    reduce(most);
    if (threadIdx.x % 32 == 0) warps_found[threadIdx.x / 32] = most;
    __syncthreads();
    if (threadIdx.x < 32) {
        most = threadIdx.x < kScanThreads / 32 ? warps_found[threadIdx.x] : Scan{};
        reduce(most);
        if (threadIdx.x == 0) a.scan_parts[blockIdx.x] = most;
    }
}

// The largest of the parts, by every warp for itself.
__device__ __forceinline__ Scan join_scan(const Scan* parts) {
    Scan most{};
    for (int p = threadIdx.x % 32; p < kScanCtas; p += 32) {
        const Scan s = parts[p];
        most.hidden = max(most.hidden, s.hidden);
        most.head = max(most.head, s.head);
        most.weight = max(most.weight, s.weight);
    }
    most.hidden = __reduce_max_sync(0xffffffffu, most.hidden);
    most.head = __reduce_max_sync(0xffffffffu, most.head);
    most.weight = __reduce_max_sync(0xffffffffu, most.weight);
    return most;
}

// Four columns a lane; `aligned`: they can be read at once. ld is a multiple of 64: what a lane writes past the width is padding.
template <class T>
__device__ __forceinline__ void pack_row(const T* from, bool aligned, void* to0, void* to1, int64_t at, int64_t width, int64_t ld, int e, bool zero) {
    const PowerOfTwo up(e);
#pragma unroll 4
    for (int64_t c = threadIdx.x % 32 * 4; c < width; c += 128) {
        Pack<T, 4> x;
        if (aligned && c + 4 <= width) {
            x = *reinterpret_cast<const Pack<T, 4>*>(from + c);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) x.v[k] = c + k < width ? from[c + k] : narrow<T>(0.0f);
        }
        if (zero)
#pragma unroll
            for (int k = 0; k < 4; ++k) x.v[k] = narrow<T>(0.0f);
        if constexpr (sizeof(T) == 4) {
            Pack<__half, 4> h, l;
#pragma unroll
            for (int k = 0; k < 4; ++k) split_words(up(x.v[k]), h.v[k], l.v[k]);
            *reinterpret_cast<Pack<__half, 4>*>(static_cast<__half*>(to0) + at * ld + c) = h;
            *reinterpret_cast<Pack<__half, 4>*>(static_cast<__half*>(to1) + at * ld + c) = l;
        } else {
            *reinterpret_cast<Pack<T, 4>*>(static_cast<T*>(to0) + at * ld + c) = x;
        }
    }
}

template <class T>
bool fours_aligned(const void* p, int64_t pitch) {
    return reinterpret_cast<uintptr_t>(p) % (4 * sizeof(T)) == 0 && pitch % 4 == 0;
}

// The operands of the products in the workspace, a warp a row: two words of fp32 rows, a copy of bf16 ones where
// TMA cannot read them in place. A token without a target must add nothing to dW = P^T h: 0 * NaN would, so such a row of hidden
// becomes zero when it holds anything that is not finite. Nor may it weigh on the others' precision: all tokens with a target share
// one power of two (dW adds them up), one without has its own.
template <class T>
__global__ void __launch_bounds__(256) k_pack(PrepareArgs a) {
    ptx::chained();
    const int64_t warp = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    Scan scan{};
    if (a.scan) {
        scan = join_scan(a.scan_parts);
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.scan = scan;  // for the epilogues
    }
    const int64_t rows = a.n + (a.w0 ? a.vocab : 0);
    for (int64_t r = warp; r < rows; r += (int64_t)gridDim.x * 8) {
        if (r >= a.n) {
            const int64_t v = r - a.n;
            pack_row(static_cast<const T*>(a.head) + v * a.head_pitch, a.head_fours, a.w0, a.w1, v, a.width, a.ld, a.w1 ? word_exponent(scan.head) : 0,
                     false);
            continue;
        }
        const bool live = is_token(a.targets[r], a.vocab);
        if (a.rate && threadIdx.x % 32 == 0) {
            const float most = a.weights ? __uint_as_float(scan.weight) : 1.0f;
            a.rate[r] = !live ? 0.0f : !a.weights ? 1.0f : most > 0.0f ? a.weights[r] / most : a.weights[r];
        }
        if (!a.h0) continue;
        const T* from = static_cast<const T*>(a.hidden) + r * a.hidden_pitch;
        uint32_t most = scan.hidden;
        bool bad = false;
        if (!live) {
            most = 0;
            for (int64_t c = threadIdx.x % 32; c < a.width; c += 32) most = max(most, __float_as_uint(fabsf(widen(from[c]))));
            most = __reduce_max_sync(0xffffffffu, most);
            bad = most >= 0x7f800000u;
        }
        const int e = a.h1 && !bad ? word_exponent(most) : 0;
        if (threadIdx.x % 32 == 0) {
            a.poisoned[r] = bad;
            if (a.h1) a.exponents[r] = e;
        }
        pack_row(from, a.hidden_fours, a.h0, a.h1, r, a.width, a.ld, e, bad);
    }
}

// ---- epilogues ----------------------------------------------------------------------------------
// Statistics of 128 columns of one token, by one thread.
template <bool kWords, bool kKeep>
struct StatisticsEpi {
    struct Args {
        float2* partial;  // maximum, sum of exp(z - maximum) of each token and part (128 columns)
        int64_t row_stride, part_stride;
        float* z;         // [n, z_ld], where the logits are kept
        int64_t z_ld;
        float* at_target;
        const int32_t* targets;
        const Scan* scan;
        const int32_t* exponents;
        int64_t n, vocab;
    };
    const Args& a;
    int64_t row0, row, col0;
    int64_t target;
    int lane;
    float* staging;
    float top = -INFINITY, sum = 0.0f;
    PowerOfTwo unscale;
    __device__ __forceinline__ StatisticsEpi(const Args& args, const Tile& t, int row_, int col, int lane_, float* staging_)
        : a(args), row0(row_), row((int64_t)row_ + lane_), col0(col), lane(lane_), staging(staging_), unscale(kWords && row < args.n ? -(args.exponents[row] + word_exponent(args.scan->head)) : 0) {
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
        if (kKeep && row0 < a.n && col < a.vocab) {
            turn_columns(staging, v, lane);
            float* to = a.z + row0 * a.z_ld + col + lane;
            if (col + lane < a.vocab)
#pragma unroll
                for (int r = 0; r < 32; ++r)
                    if (row0 + r < a.n) to[r * a.z_ld] = v[r];
        }
    }
    __device__ __forceinline__ void finish() {
        if (row < a.n) a.partial[col0 / 128 * a.part_stride + row * a.row_stride] = make_float2(top, sum);
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
        const int32_t* exponents;
        int64_t n, vocab, v0;
    };
    const Args& a;
    int64_t row0, row, col0;
    int64_t target;
    int lane;
    float* staging;
    float lse = 0.0f, rate = 0.0f;
    PowerOfTwo unscale;
    __device__ __forceinline__ ProbabilityEpi(const Args& args, const Tile& t, int row_, int col, int lane_, float* staging_)
        : a(args),
          row0(row_),
          row((int64_t)row_ + lane_),
          col0(col),
          lane(lane_),
          staging(staging_),
          unscale(kWords && row < args.n ? -(args.exponents[row] + word_exponent(args.scan->head)) : 0) {
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
        if (row0 >= a.n) return;
        const int64_t col = col0 + c * 32;
        const bool live = target >= 0 || rate != 0.0f;
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            const float z = kWords ? unscale(v[k]) : v[k];
            float p = exp2_fast((z - lse) * kLog2E);
            p = rate * (target == col + k ? p - 1.0f : p);
            v[k] = live ? p : 0.0f;
        }
        const int64_t at = row0 * a.ld + col;
        const int rows = (int)min((int64_t)32, a.n - row0);
        if constexpr (kWords) {
            __half hi[32], lo[32];
#pragma unroll
            for (int k = 0; k < 32; k += 2)
                split_pair(v[k] * (float)(1 << kPScale), v[k + 1] * (float)(1 << kPScale), hi[k], hi[k + 1], lo[k], lo[k + 1]);
            store_rows16(staging, hi, static_cast<__half*>(a.p0) + at, a.ld, rows, lane);
            store_rows16(reinterpret_cast<char*>(staging) + 2048, lo, static_cast<__half*>(a.p1) + at, a.ld, rows, lane);
        } else {
            __nv_bfloat16 o[32];
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = narrow<__nv_bfloat16>(v[k]);
            store_rows16(staging, o, static_cast<__nv_bfloat16*>(a.p0) + at, a.ld, rows, lane);
        }
    }
    __device__ __forceinline__ void finish() {}
};

// What turns a gradient's sums into the gradient: the words' scales, the caller's, and the largest weight.
struct GradientScale {
    const Scan* scan;
    bool of_hidden;  // the other operand is head (grad_hidden) or hidden (grad_head)
    bool weighted;
    float scale;
    // of grad_hidden's rows, else NULL: a token without a target has a zero row, also where the head holds what is not finite and 0 * NaN came in
    const int32_t* targets;
    int64_t vocab;
    __device__ __forceinline__ bool zero_row(int64_t r) const { return targets && !is_token(targets[r], vocab); }
};
template <class T>
struct GradientFactor {
    PowerOfTwo unscale;
    float last;
    static __device__ __forceinline__ int exponent(const GradientScale& s) {
        return sizeof(T) == 4 ? -(kPScale + word_exponent(s.of_hidden ? s.scan->head : s.scan->hidden)) : 0;
    }
    __device__ __forceinline__ explicit GradientFactor(const GradientScale& s) : unscale(exponent(s)) {
        const float most = s.weighted ? __uint_as_float(s.scan->weight) : 1.0f;
        last = s.scale * (most > 0.0f ? most : 1.0f);
    }
    __device__ __forceinline__ T operator()(float v) const { return narrow<T>((sizeof(T) == 4 ? unscale(v) : v) * last); }
};

// P from kept logits.
template <bool kWords>
struct WordSink {
    void *p0, *p1;
    int64_t ld;
    const float* rate;
    struct Row {
        void *p0, *p1;
        float rate;
        __device__ __forceinline__ void operator()(int64_t c, float p, float q) const {
            if constexpr (kWords) {
                Pack<__half, 2> h, l;
                split_pair(rate * p * (float)(1 << kPScale), rate * q * (float)(1 << kPScale), h.v[0], h.v[1], l.v[0], l.v[1]);
                *reinterpret_cast<Pack<__half, 2>*>(static_cast<__half*>(p0) + c) = h;
                *reinterpret_cast<Pack<__half, 2>*>(static_cast<__half*>(p1) + c) = l;
            } else {
                *reinterpret_cast<Pack<__nv_bfloat16, 2>*>(static_cast<__nv_bfloat16*>(p0) + c) = {narrow<__nv_bfloat16>(rate * p), narrow<__nv_bfloat16>(rate * q)};
            }
        }
        __device__ __forceinline__ void none(int64_t c) const {
            *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p0) + c) = 0;
            if (kWords) *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p1) + c) = 0;
        }
    };
    __device__ __forceinline__ Row row(int64_t t) const {
        return {static_cast<uint16_t*>(p0) + t * ld, kWords ? static_cast<uint16_t*>(p1) + t * ld : nullptr, rate[t]};
    }
};

// A gradient's tile: out = factor * (sums of the earlier pieces + this one), or those sums kept for later.
template <class T>
struct GradientEpi {
    struct Args {
        T* out;  // NULL: keep
        int64_t pitch, rows, cols;
        float* kept;  // [parts of K][rows][kept_ld], or NULL with a single piece in one part
        int64_t kept_ld;
        bool add;  // kept holds earlier pieces
        GradientScale scale;
    };
    const Args& a;
    int64_t row0, col0;
    int lane;
    float* staging;
    float* kept;
    GradientFactor<T> factor;
    unsigned zero;  // rows of zeros, a bit each
    __device__ __forceinline__ GradientEpi(const Args& args, const Tile& t, int row, int col, int lane_, float* staging_)
        : a(args), row0(row), col0(col), lane(lane_), staging(staging_), kept(a.kept ? a.kept + t.split * a.rows * a.kept_ld : nullptr), factor(a.scale) {
        zero = __ballot_sync(0xffffffffu, row0 + lane < a.rows && a.scale.zero_row(row0 + lane));
    }
    __device__ __forceinline__ void chunk(int c, float (&v)[32]) {
        const int64_t col = col0 + c * 32 + lane;
        if (row0 >= a.rows || col0 + c * 32 >= a.cols) return;
        turn_columns(staging, v, lane);
        if (col >= a.cols) return;
        const int rows = (int)min((int64_t)32, a.rows - row0);
        float* keep = kept + row0 * a.kept_ld + col;
        if (a.add) {  // all loads before the first store
            float before[32];
#pragma unroll
            for (int r = 0; r < 32; ++r) before[r] = r < rows ? keep[r * a.kept_ld] : 0.0f;
#pragma unroll
            for (int r = 0; r < 32; ++r) v[r] += before[r];
        }
        T* to = a.out + row0 * a.pitch + col;
#pragma unroll
        for (int r = 0; r < 32; ++r)
            if (r < rows) {
                if (a.out) to[r * a.pitch] = zero >> r & 1 ? narrow<T>(0.0f) : factor(v[r]);
                else keep[r * a.kept_ld] = v[r];
            }
    }
    __device__ __forceinline__ void finish() {}
};

// Adds up the parts of K of a gradient, in order.
template <class T>
__global__ void __launch_bounds__(256) k_join_parts(const float* __restrict__ kept, int parts, int64_t kept_ld, int64_t some, int64_t rows, int64_t cols, T* __restrict__ out,
                                                    int64_t pitch, GradientScale scale) {
    ptx::chained();
    const GradientFactor<T> factor(scale);
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x, r = blockIdx.y;
    if (c >= cols || r >= some) return;
    float sum = 0.0f;
#pragma unroll 4
    for (int p = 0; p < parts; ++p) sum += kept[(p * rows + r) * kept_ld + c];
    out[r * pitch + c] = scale.zero_row(r) ? narrow<T>(0.0f) : factor(sum);
}

// ---- layout and launches ------------------------------------------------------------------------
// K blocks a promoted sum stays in tensor memory: 16 steps of the tensor core with fp32 rows, for the loss of bf16 rows 32, or 16 where
// reading the sums back more often costs little: all tiles have a pair of CTAs at once, or one tile holds all tokens and reading the head
// bounds the product. The loss of bf16 rows, stays of 16 / 8 / 4 blocks: us and the error (root mean square over the tokens, of loss and
// lse) as a multiple of a plain fp32 form's: 4,096 x 50,003 x 1,024 316 (2.8, 3.0) / 332 (1.4, 1.8) / 341 (0.7, 1.3); 256 x 50,003 x 1,024
// 35.1 (2.7, 3.1) / 37.6 (1.2, 1.9) / 37.8 (0.7, 1.4); 64 x 20,000 x 768 22.8 (2.7, 2.6) / 24.1 (1.7, 2.1) / 21.7 (1.1, 1.2); 2,000 x 5,003
// x 1,024 30.1 (2.9, 3.5) / 31.5 (1.4, 1.9) / 32.8 (0.7, 1.2); 2,000 x 356 x 1,753 28.8 (1.7, 2.4) / 28.6 (0.9, 1.2) / 28.1 (0.5, 0.6); 300
// x 300 x 512, the product alone, 12.2 (1.9, 3.1) / 12.2 / 13.0 (0.9, 1.7).
constexpr int kFlush = 4, kFlushLoss = 8, kFlushLossFewTiles = 4;

struct Layout {
    Scan *scan, *scan_parts;
    void *h0, *h1, *w0, *w1, *p0, *p1;
    float2* partial;
    float *at_target, *rate, *kept, *head_kept, *z;
    int32_t *exponents, *poisoned;
    int64_t ld, p_ld, kept_ld, piece, z_ld;
    bool keep;  // the logits, from the statistics to P
    int hidden_parts, head_parts;  // of K, in the gradients' products
    bool together;                 // both in one launch
};

// Vocabulary rows of a piece: as many as keep P within kPieceBytes, fewer where that fills the pairs of CTAs better.
// Cost in units of (tile of 256 x 256) x (K of 256) a pair.
constexpr int64_t kPieceBytes = 160ll << 20;
constexpr int64_t kPairs = 74;
// Few logits (64 MB as floats, half of that with bf16 rows, whose products cost a third) are kept: P then costs a pass over them and not
// another product. Loss and gradients, us, kept / made again, tokens x vocabulary x width. fp32 rows: 333 x 5,003 x 201 76 / 87; 2,000 x 4,000 x
// 512 137 / 162; 1,000 x 16,000 x 1,024 387 / 449; 200 x 60,000 x 80 211 / 212; 1 x 200,064 x 768 1,178 / 1,432; 64 x 200,064 x 512 881 / 1,010;
// 64 x 262,144 x 2,048 4,042 / 4,808. bf16: 333 x 5,003 x 201 47 / 47; 2,000 x 4,000 x 512 78 / 74; 128 x 50,000 x 512 147 / 140; 200 x 40,000 x 80
// 99 / 82; 1 x 262,144 x 768 612 / 703; 16 x 400,003 x 768 923 / 1,026; 25 x 327,681 x 2,048 1,772 / 2,037: with bf16 rows it pays for few tokens
// against a large vocabulary, where a product pads them to 256, and costs up to a fifth where width is small against that.
// A vocabulary of a few tiles would leave the pass mostly launch.
constexpr int64_t kKeepLogits = int64_t(1) << 24, kKeepVocab = 512;
constexpr int64_t kLeastBlocks = 8;  // of K in a part: less would leave its tile mostly epilogue
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
    l.scan_parts = w.take<Scan>(kScanCtas);
    l.h0 = w.take<uint16_t>(n * l.ld);
    l.w0 = w.take<uint16_t>(vocab * l.ld);
    if (words == 2) {
        l.h1 = w.take<uint16_t>(n * l.ld);
        l.w1 = w.take<uint16_t>(vocab * l.ld);
    }
    l.partial = w.take<float2>(2 * ceil_div(vocab, kTileN) * n);
    l.at_target = w.take<float>(n);
    l.keep = n * vocab <= kKeepLogits / (words == 2 ? 1 : 2) && vocab >= kKeepVocab;
    l.z_ld = round_up(vocab, 32);
    if (l.keep && with_grad) l.z = w.take<float>(n * l.z_ld);
    l.exponents = w.take<int32_t>(n);
    l.poisoned = w.take<int32_t>(n);
    if (with_grad) {
        // kept logits become P in one launch, so then a piece is the whole vocabulary: at most as many elements as logits
        l.piece = l.keep ? round_up(vocab, kTileN) : piece_rows(n, width, vocab, words);
        l.p_ld = l.piece;
        l.rate = w.take<float>(n);
        l.p0 = w.take<uint16_t>(n * l.p_ld);
        if (words == 2) l.p1 = w.take<uint16_t>(n * l.p_ld);
        l.kept_ld = round_up(width, kTileN);
        const int64_t rows = std::min(l.piece, vocab), across = ceil_div(width, kTileN);
        const int64_t hidden_tiles = ceil_div(n, kTileM) * across, hidden_blocks = ceil_div(rows, kBlockK);
        const int64_t head_tiles = ceil_div(rows, kTileM) * across, head_blocks = ceil_div(n, kBlockK);
        l.together = l.piece >= vocab && hidden_tiles + head_tiles <= kPairs;
        if (l.together) {  // one launch: a part's share of the blocks of K is what a pair of CTAs gets of all of them
            const int64_t target = std::max(kLeastBlocks, ceil_div(hidden_tiles * hidden_blocks + head_tiles * head_blocks, kPairs));
            l.hidden_parts = (int)std::max<int64_t>(1, hidden_blocks / target);
            l.head_parts = (int)std::max<int64_t>(1, head_blocks / target);
        } else {
            l.hidden_parts = split_parts(hidden_tiles, hidden_blocks, kPairs, kLeastBlocks);
            l.head_parts = split_parts(head_tiles, head_blocks, kPairs, kLeastBlocks);
        }
        const int64_t kept_rows = l.piece < vocab || l.hidden_parts > 1 ? n * l.hidden_parts : 0;
        l.kept = w.take<float>(kept_rows * l.kept_ld);
        l.head_kept = w.take<float>(l.head_parts > 1 ? rows * l.head_parts * l.kept_ld : 0);
    }
    if (out) *out = l;
    return w.used;
}

template <class T>
cudaError_t typed(const VocabLossArgs& a, Layout l, cudaStream_t s) {
    constexpr bool kWords = sizeof(T) == 4;
    const int64_t n = a.n_tokens;
    const bool with_grad = a.grad_hidden || a.grad_head;
    if (n == 0) {
        if (!a.grad_head) return cudaSuccess;
        return cudaMemset2DAsync(a.grad_head, a.grad_head_pitch * sizeof(T), 0, a.width * sizeof(T), a.vocab, s);
    }
    // operands: in place where TMA can read them (bf16, 16-byte rows), else from the workspace
    auto in_place = [](const void* p, int64_t pitch) { return !kWords && reinterpret_cast<uintptr_t>(p) % 16 == 0 && pitch % 8 == 0 && pitch < (int64_t(1) << 38); };
    const bool hidden_in_place = in_place(a.hidden, a.hidden_pitch) && !a.grad_head;
    const bool head_in_place = in_place(a.head, a.head_pitch);
    PrepareArgs prep{a.hidden, a.head, a.targets, a.weights, n, a.width, a.vocab, a.hidden_pitch, a.head_pitch, nullptr, l.scan_parts, nullptr, nullptr,
                     nullptr, nullptr, l.ld, with_grad ? l.rate : nullptr, fours_aligned<T>(a.hidden, a.hidden_pitch), fours_aligned<T>(a.head, a.head_pitch),
                     l.exponents, l.poisoned};
    const bool weighted = with_grad && a.weights;
    if (!with_grad) prep.weights = nullptr;
    if (kWords || weighted) prep.scan = l.scan;
    if (!hidden_in_place) prep.h0 = l.h0, prep.h1 = l.h1;
    if (!head_in_place) prep.w0 = l.w0, prep.w1 = l.w1;
    if (prep.scan) A2_CUDA_TRY(launch_chained(k_scan<T>, dim3(kScanCtas), kScanThreads, 0, s, prep));
    if (prep.h0 || prep.w0 || prep.rate)
        A2_CUDA_TRY(launch_chained(k_pack<T>, dim3((unsigned)std::min<int64_t>(ceil_div(n + (prep.w0 ? a.vocab : 0), 8), 148 * 8)), 256, 0, s, prep));

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
    const int64_t tiles_m = ceil_div(n, kTileM), tiles = tiles_m * ceil_div(a.vocab, kTileN);
    const int flush_loss = kWords ? kFlush : tiles_m == 1 || tiles <= kPairs ? kFlushLossFewTiles : kFlushLoss;
    A2_CUDA_TRY(make_gemm(hidden(false), head(0, a.vocab, false), 1, !kWords, false, flush_loss, 1, &g));
    const int parts = (int)(2 * ceil_div(a.vocab, kTileN));
    auto statistics = [&](auto keep) {
        using Epi = StatisticsEpi<kWords, decltype(keep)::value>;
        return launch_gemm<Epi, true>(
            g, typename Epi::Args{l.partial, l.keep ? parts : 1, l.keep ? 1 : n, l.z, l.z_ld, l.at_target, a.targets, l.scan, l.exponents, n, a.vocab}, s);
    };
    A2_CUDA_TRY(l.z ? statistics(std::true_type{}) : statistics(std::false_type{}));
    const int32_t* poisoned = hidden_in_place ? nullptr : l.poisoned;
    if (l.keep) {
        A2_CUDA_TRY(launch_rows(a, l.partial, parts, l.at_target, poisoned, l.z, l.z_ld, with_grad, WordSink<kWords>{l.p0, l.p1, l.p_ld, l.rate}, s));
    } else {
        A2_CUDA_TRY(launch_chained(k_finish, dim3((unsigned)ceil_div(n, 32)), kFinishWarps * 32, 0, s, l.partial, parts, l.at_target, a.targets, poisoned, n,
                               a.vocab, a.loss, a.lse));
    }
    if (!with_grad) return cudaSuccess;

    auto join = [&](const float* kept, int parts, int64_t rows, T* out, int64_t pitch, const GradientScale& of_all) {
        for (int64_t r = 0; r < rows; r += 65535) {  // the grid's second dimension ends there
            const int64_t some = std::min<int64_t>(65535, rows - r);
            GradientScale scale = of_all;
            if (scale.targets) scale.targets += r;
            A2_CUDA_TRY(launch_chained(k_join_parts<T>, dim3((unsigned)ceil_div(a.width, 256), (unsigned)some), 256, 0, s, kept + r * l.kept_ld, parts,
                                   l.kept_ld, some, rows, a.width, out + r * pitch, pitch, scale));
        }
        return cudaSuccess;
    };
    for (int64_t v0 = 0; v0 < a.vocab; v0 += l.piece) {
        const int64_t rows = std::min(l.piece, a.vocab - v0);
        const bool first = v0 == 0, final = v0 + rows == a.vocab;
        if (!l.keep) {
            A2_CUDA_TRY(make_gemm(hidden(false), head(v0, rows, false), 1, !kWords, false, flush, 1, &g));
            const typename ProbabilityEpi<kWords>::Args prob{l.p0, l.p1, l.p_ld, a.targets, a.lse, l.rate, l.scan, l.exponents, n, a.vocab, v0};
            A2_CUDA_TRY((launch_gemm<ProbabilityEpi<kWords>, kWords>(g, prob, s)));
        }
        using Grad = GradientEpi<T>;
        GemmArgs of_head, of_hidden;
        const GradientScale head_scale{l.scan, false, weighted, a.scale, nullptr, 0}, hidden_scale{l.scan, true, weighted, a.scale, a.targets, a.vocab};
        T* head_out = a.grad_head ? static_cast<T*>(a.grad_head) + v0 * a.grad_head_pitch : nullptr;
        T* hidden_out = static_cast<T*>(a.grad_hidden);
        const bool head_parts = l.head_parts > 1, hidden_parts = l.hidden_parts > 1;
        const typename Grad::Args head_args{head_parts ? nullptr : head_out, a.grad_head_pitch, rows, a.width, l.head_kept, l.kept_ld, false, head_scale};
        const typename Grad::Args hidden_args{final && !hidden_parts ? hidden_out : nullptr, a.grad_hidden_pitch, n, a.width, l.kept, l.kept_ld, !first,
                                              hidden_scale};
        if (a.grad_head) A2_CUDA_TRY(make_gemm(Operand{l.p0, l.p1, rows, n, l.p_ld, 0, true}, hidden(true), 1, !kWords, false, flush, l.head_parts, &of_head));
        if (a.grad_hidden) {
            // part p of every piece adds to the sums of part p; a short last piece may have fewer parts, but none without a block
            const int here = (int)std::min<int64_t>(l.hidden_parts, ceil_div(rows, kBlockK));
            A2_CUDA_TRY(make_gemm(Operand{l.p0, l.p1, n, rows, l.p_ld, 0, false}, head(v0, rows, true), 1, !kWords, false, flush, here, &of_hidden));
        }
        if (l.together && a.grad_head && a.grad_hidden) {  // the longer sums first
            A2_CUDA_TRY((rows >= n ? launch_gemms<Grad, kWords>(of_hidden, hidden_args, of_head, head_args, s)
                               : launch_gemms<Grad, kWords>(of_head, head_args, of_hidden, hidden_args, s)));
        } else {
            if (a.grad_head) A2_CUDA_TRY((launch_gemm<Grad, kWords>(of_head, head_args, s)));
            if (a.grad_hidden) A2_CUDA_TRY((launch_gemm<Grad, kWords>(of_hidden, hidden_args, s)));
        }
        if (a.grad_head && head_parts) A2_CUDA_TRY(join(l.head_kept, l.head_parts, rows, head_out, a.grad_head_pitch, head_scale));
        if (a.grad_hidden && hidden_parts && final) A2_CUDA_TRY(join(l.kept, l.hidden_parts, n, hidden_out, a.grad_hidden_pitch, hidden_scale));
    }
    return cudaSuccess;
}

}  // namespace

int64_t vocab_loss_workspace(int64_t n_tokens, int64_t width, int64_t vocab, bool with_grad, int32_t dtype) {
    if (vocab_loss_is_few(n_tokens, width, vocab, dtype)) return vocab_loss_few_workspace(n_tokens, width, vocab, with_grad);
    return layout(n_tokens, width, vocab, with_grad, dtype, nullptr, nullptr);
}

cudaError_t run_vocab_loss(const VocabLossArgs& a, void* workspace, cudaStream_t s) {
    if (vocab_loss_is_few(a.n_tokens, a.width, a.vocab, a.dtype)) return run_vocab_loss_few(a, workspace, s);
    Layout l;
    layout(a.n_tokens, a.width, a.vocab, a.grad_hidden || a.grad_head, a.dtype, workspace, &l);
    return a.dtype == A2_BF16 ? typed<__nv_bfloat16>(a, l, s) : typed<float>(a, l, s);
}

}  // namespace a2
