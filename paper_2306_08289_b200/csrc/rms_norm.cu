// Root-mean-square norm with the residual's addition, y = s / sqrt(mean s^2 + eps) w with s = x + r, its output in 8 bits, and its gradient
//   hat = s rstd,  c = mean(hat w g),  dx = rstd (w g - hat c) + ds,  dw = sum over rows of g hat.
#include <cuda_fp8.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "lm_ops.h"

namespace a2 {

int multiprocessors() {
    static std::atomic<int> known[64];
    int device = 0, sms = 0;
    if (cudaGetDevice(&device) != cudaSuccess) return 1;
    if (device < 64 && known[device].load() > 0) return known[device].load();
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || sms < 1) return 1;
    if (device < 64) known[device].store(sms);
    return sms;
}

namespace {

constexpr float kE4m3Most = 448.0f;
constexpr float kScaleLeast = 0x1p-126f;  // of a block of zeros: its values are zeros whatever the scale, and no division by zero follows

// ---------------------------------------------------------------------------------------------
// A row's columns lie over a group of `group` threads: thread t holds the vectors t, t + group, ... of 16 bytes, K of them. A row that starts `shift`
// elements after a 16-byte boundary is read from that boundary on (the vectors of all matrices of a call then start on boundaries, if
// all rows are shifted alike): the first and the last vector are cut at the row's ends. WIDE = false finds a vector in two units of 16 bytes and writes element by
// element.
// ---------------------------------------------------------------------------------------------
// Groups are a power of two up to a warp, or whole warps. A thread's group in its CTA, its place in it:
struct Place {
    int mine, t;
    __device__ explicit Place(unsigned group) {
        mine = blockDim.x == group ? 0 : threadIdx.x / group;
        t = threadIdx.x - mine * group;
    }
};

__device__ __forceinline__ unsigned mask_of(int group) {  // of the lanes of this thread's group
    const int lane = threadIdx.x % 32;
    return group >= 32 ? 0xffffffffu : ((1u << group) - 1u) << (lane & ~(group - 1));
}

// Sums (or maxima of magnitudes) of COUNT values over a group, the same bits in every thread. `slot` changes from one such reduction to the
// next (0, 1, 0, ...), so that one barrier each is enough: that of the CTA, or with SEVERAL groups of more than a warp in it (at most 15) that of the
// group's warps. Those groups do not wait for one another: a warp has two places of its own in a slot, whatever COUNT is, so that one group's maximum never lies where
// another's sums do. A kernel that does not know its barriers' numbers reserves all of a CTA's, which only few CTAs a multiprocessor can have.
constexpr int kPlaces = 2;  // of a warp, in a slot
template <bool MAX, bool SEVERAL, int COUNT>
__device__ __forceinline__ void over_group(float (&v)[COUNT], int group, int mine, int slot, float (*shared)[32 * kPlaces]) {
    static_assert(COUNT <= kPlaces, "places of a warp");
    const unsigned mask = mask_of(group);
    auto join = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
#pragma unroll
    for (int d = 16; d > 0; d /= 2)
        if (d < group)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] = join(v[i], __shfl_xor_sync(mask, v[i], d));
    if (group <= 32) return;
    const int warps = group / 32, lane = threadIdx.x % 32;
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < COUNT; ++i) shared[slot][threadIdx.x / 32 * kPlaces + i] = v[i];
    if constexpr (SEVERAL)
        asm volatile("bar.sync %0, %1;" ::"r"(mine + 1), "r"(group) : "memory");
    else
        __syncthreads();
    const int first = SEVERAL ? mine * warps : 0;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = lane < warps ? shared[slot][(first + lane) * kPlaces + i] : 0.0f;  // zero is neutral for both
#pragma unroll
    for (int d = 16; d > 0; d /= 2)
        if (d < warps)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] = join(v[i], __shfl_xor_sync(0xffffffffu, v[i], d));
    // warps that are no power of two: lanes past them hold other sums
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = __shfl_sync(0xffffffffu, v[i], 0);
}
template <bool MAX, bool SEVERAL>
__device__ __forceinline__ float over_group(float v, int group, int mine, int slot, float (*shared)[32 * kPlaces]) {
    float one[1] = {v};
    over_group<MAX, SEVERAL, 1>(one, group, mine, slot, shared);
    return one[0];
}

// Rows whose squares leave the range of floats are multiplied by a power of two first, and rstd is that of the scaled row.
__device__ __forceinline__ bool in_range(float squares, float eps_sum) { return squares < 0x1p120f && squares + eps_sum > 0x1p-90f; }
template <class T>
__device__ __forceinline__ float most_of(uint32_t word) {  // the larger magnitude of a word's elements
    if constexpr (sizeof(T) == 4)
        return fabsf(__uint_as_float(word));
    else
        return fmaxf(fabsf(__uint_as_float(word << 16)), fabsf(__uint_as_float(word & 0xffff0000u)));
}
__device__ __forceinline__ float power_below(float most) {  // 2^-e for most in [2^e, 2^(e+1))
    if (!(most > 0.0f) || isinf(most)) return 1.0f;
    int e;
    frexpf(most, &e);
    return ldexpf(1.0f, max(-126, min(126, 1 - e)));
}
__device__ __forceinline__ float rstd_of(float mean) { return __frsqrt_rn(mean); }  // 1 / sqrt, rounded once
__device__ __forceinline__ float scaled_rstd(float by, float squares, int width, float eps) {
    const double mean = (double)squares / (double)width + (double)eps * by * by;
    return mean > 0.0 ? (float)(1.0 / sqrt(mean)) : isnan(mean) ? (float)mean : 0.0f;  // a row of zeros with eps = 0 gives zeros
}

__device__ __forceinline__ float scale_of(float most) { return fmaxf(__fdiv_rn(most, kE4m3Most), kScaleLeast); }

// Off by a unit in the last place at most; a scale and its reciprocal are both in the range of floats.
__device__ __forceinline__ float near_reciprocal(float scale) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(scale));
    return r;
}

// The 8 bits nearest to v / scale, four values a word. A division a value would cost more than all else there is to do with it, so each is multiplied by two factors,
// one below and one above 1 / scale: products and their roundings keep the order, the quotient's lies between them, and where both give the same 8 bits these are the
// quotient's. The others (one value in 10^5) are divided. 8,192 x 2,048 bf16 in blocks of 128, with residual: 26.2 us, of which that certainty and the scale's own division
// take 2.9 (23.3 with one product by the approximate reciprocal, which gives some values their other neighbour).
template <int H>
struct Halves {
    float2 v[H];
};
template <int H>
__device__ __noinline__ Pack<uint32_t, H / 2> divided(const Halves<H> h, float scale) {
    Pack<uint32_t, H / 2> q;
#pragma unroll
    for (int k = 0; k < H; ++k) {
        const uint32_t pair = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(h.v[k].x, scale), __fdiv_rn(h.v[k].y, scale)), __NV_SATFINITE, __NV_E4M3);
        q.v[k / 2] = k % 2 ? q.v[k / 2] | pair << 16 : pair;
    }
    return q;
}
template <int H>
__device__ __forceinline__ Pack<uint32_t, H / 2> to_8_bits(const float2 (&v)[H], float scale) {
    const float inverse = near_reciprocal(scale), below = inverse * (1.0f - 0x1p-22f), above = inverse * (1.0f + 0x1p-22f);
    Pack<uint32_t, H / 2> q;
    uint32_t differ = 0;
#pragma unroll
    for (int k = 0; k < H; ++k) {
        const uint32_t pair = __nv_cvt_float2_to_fp8x2(mul2(v[k], two(below)), __NV_SATFINITE, __NV_E4M3);
        differ |= pair ^ __nv_cvt_float2_to_fp8x2(mul2(v[k], two(above)), __NV_SATFINITE, __NV_E4M3);
        q.v[k / 2] = k % 2 ? q.v[k / 2] | pair << 16 : pair;
    }
    if (differ) {
        Halves<H> h;
#pragma unroll
        for (int k = 0; k < H; ++k) h.v[k] = v[k];
        q = divided<H>(h, scale);
    }
    return q;
}

struct NormKernelArgs {
    const void *x, *residual, *weight;
    int64_t x_pitch, residual_pitch, n;
    int width;
    float eps, one_over_width;
    void *sum, *out;
    int64_t sum_pitch, out_pitch;
    float* scales;
    int block_log, blocks, group;
    bool wide_weight, wide_out;
};

// ---------------------------------------------------------------------------------------------
// Forward. Bound by memory: x and r are read once, s and y written once, the row stays in registers as floats in between. A group holds one
// row. MODE 0: y in the rows' type. 1: e4m3 with a scale for every 2^block_log columns, whose vectors lie in neighbouring lanes. 2: e4m3 with one
// scale a row. Sums are in fp32; s is rounded only where it is stored, y is formed from what it was before.
// With residual, 16,384 x 4,096 fp32: 158 us (6.8 TB/s); 16,384 x 2,048 bf16: 41 us (6.5 TB/s). To 8 bits in blocks of 128, with residual: 8,192 x 2,048 bf16 26 us (4.5 TB/s;
// instructions and what one waits for another: two thirds of the issue slots), fp32 39 us (5.6 TB/s); with a scale a row 25 and 35.
// Few threads a row (two to four vectors each) because what a row costs besides its vectors is paid by every warp; the
// figures stand at the choice. Times here and below are of launches replayed from a graph, one behind the other.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t bits_of(const float* p) { return __float_as_uint(*p); }
__device__ __forceinline__ uint32_t bits_of(const __nv_bfloat16* p) { return *reinterpret_cast<const uint16_t*>(p); }

// How rows lie: vectors are found in two units each; on boundaries, the ends cut; or on boundaries and all K vectors of all threads whole.
enum Lie { kAnywhere, kWide, kFull };

// A thread's vectors of a row.
template <class T, Lie LIE, int K>
struct Columns {
    static constexpr bool WIDE = LIE != kAnywhere;
    int first, step, width;  // the column of vector 0, columns from one vector to the next
    bool cut;                // one of them is cut at the row's ends
    __device__ Columns(const void* row, int t, int group, int w) {
        first = t * kVec<T> - (LIE == kWide ? (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T)) : 0);
        step = group * kVec<T>;
        width = w;
        cut = LIE == kAnywhere || (LIE == kWide && first < 0);
        if (LIE == kWide)
#pragma unroll
            for (int j = 0; j < K; ++j) cut = cut || (at(j) < w && at(j) + kVec<T> > w);
    }
    __device__ int at(int j) const { return first + j * step; }
    __device__ bool in(int j) const { return LIE == kFull || at(j) < width; }
    // Loads K vectors, all of them before anything is done with one: zeros past the row's ends.
    __device__ void load(Words (&p)[K], const T* row) const {
#pragma unroll
        for (int j = 0; j < K; ++j) {
            p[j] = Words{};
            if (in(j)) p[j] = WIDE ? *reinterpret_cast<const Words*>(row + at(j)) : load_anywhere(row, at(j), width);
        }
    }
    __device__ void clear_past_ends(Words (&p)[K]) const {
        if (!WIDE || !cut) return;
#pragma unroll
        for (int j = 0; j < K; ++j) p[j] = within<T>(p[j], at(j), width);
    }
    __device__ void store(T* row, int j, const Words& p) const {
        if (WIDE && !cut)
            *reinterpret_cast<Words*>(row + at(j)) = p;
        else if (WIDE && at(j) >= 0 && at(j) + kVec<T> <= width)
            *reinterpret_cast<Words*>(row + at(j)) = p;
        else
            store_cut(row, at(j), width, p);
    }
    // A vector of the weight, which may start elsewhere.
    __device__ Words load_weight(const T* w, int j, bool wide) const {
        if (wide && !cut && (LIE == kFull || first % kVec<T> == 0)) return *reinterpret_cast<const Words*>(w + at(j));
        if (at(j) >= 0) return load_anywhere(w, at(j), width);
        Words p{};  // the vector that begins before the row
#pragma unroll
        for (int k = 0; k < kVec<T>; ++k)
            if (at(j) + k >= 0 && at(j) + k < width) p.w[k * sizeof(T) / 4] |= bits_of(w + at(j) + k) << (k * sizeof(T) % 4 * 8);
        return p;
    }
};

template <class T, Lie LIE, int K, int MODE, int THREADS>
__global__ void __launch_bounds__(THREADS, 1) k_norm(const __grid_constant__ NormKernelArgs a) {
    constexpr int V = kVec<T>, H = V / 2;
    __shared__ float shared[2][32 * kPlaces];
    ptx::chained();
    const int group = a.group, width = a.width;
    const int mine = group > 32 ? 0 : threadIdx.x >> (31 - __clz(group)), t = group > 32 ? threadIdx.x : threadIdx.x & (group - 1);
    const int64_t row = group > 32 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (blockDim.x / group) + mine;
    if (row >= a.n) return;  // whole groups, which are CTAs where they are more than a warp
    const T* x = static_cast<const T*>(a.x) + row * a.x_pitch;
    const T* w = static_cast<const T*>(a.weight);
    const Columns<T, LIE, K> columns(x, t, group, width);

    float2 v[K][H];
    {
        Words px[K], pr[K];
        columns.load(px, x);
        if (a.residual) columns.load(pr, static_cast<const T*>(a.residual) + row * a.residual_pitch);
        columns.clear_past_ends(px);
#pragma unroll
        for (int j = 0; j < K; ++j) unpack<T>(px[j], v[j]);
        if (a.residual) {
            columns.clear_past_ends(pr);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                float2 other[H];
                unpack<T>(pr[j], other);
#pragma unroll
                for (int k = 0; k < H; ++k) v[j][k] = add2(v[j][k], other[k]);
            }
        }
        if (a.sum) {
            T* sum = static_cast<T*>(a.sum) + row * a.sum_pitch;
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (columns.in(j)) columns.store(sum, j, pack<T>(v[j]));
        }
    }
    auto squares_of = [&] {
        float2 q = two(0.0f);
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int k = 0; k < H; ++k) q = fma2(v[j][k], v[j][k], q);
        return q.x + q.y;
    };
    auto most_of_row = [&] {
        float most = 0.0f;
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int k = 0; k < H; ++k) most = fmaxf(most, fmaxf(fabsf(v[j][k].x), fabsf(v[j][k].y)));
        return most;
    };
    const float squares = over_group<false, false>(squares_of(), group, mine, 0, shared);
    float rstd;
    if (in_range(squares, a.eps * (float)width)) {
        rstd = rstd_of(fmaf(squares, a.one_over_width, a.eps));
    } else {
        const float by = power_below(over_group<true, false>(most_of_row(), group, mine, 1, shared));
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int k = 0; k < H; ++k) v[j][k] = mul2(v[j][k], two(by));
        rstd = scaled_rstd(by, over_group<false, false>(squares_of(), group, mine, 0, shared), width, a.eps);
    }
#pragma unroll
    for (int j = 0; j < K; ++j) {
#pragma unroll
        for (int k = 0; k < H; ++k) v[j][k] = mul2(v[j][k], two(rstd));
        if (!columns.in(j)) continue;
        if (w) {
            float2 by_weight[H];
            unpack<T>(columns.load_weight(w, j, a.wide_weight), by_weight);
#pragma unroll
            for (int k = 0; k < H; ++k) v[j][k] = mul2(v[j][k], by_weight[k]);
        }
        if (MODE == 0) columns.store(static_cast<T*>(a.out) + row * a.out_pitch, j, pack<T>(v[j]));
    }
    if constexpr (MODE != 0) {
        uint8_t* out = static_cast<uint8_t*>(a.out) + row * a.out_pitch;
        float* scales = a.scales + row * a.blocks;
        float most = 0.0f, scale = 0.0f;
        if (MODE == 2) {
            scale = scale_of(over_group<true, false>(most_of_row(), group, mine, 1, shared));
            if (t == 0) scales[0] = scale;
        }
        const unsigned mask = mask_of(group);
        const int lanes = (1 << a.block_log) / V;  // a power of two
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int c = columns.at(j);
            if (MODE == 1) {  // vectors past the row's end hold zeros (or NaN, which maxima pass over)
                most = 0.0f;
#pragma unroll
                for (int k = 0; k < H; ++k) most = fmaxf(most, fmaxf(fabsf(v[j][k].x), fabsf(v[j][k].y)));
#pragma unroll
                for (int d = 16; d > 0; d /= 2)
                    if (d < lanes) most = fmaxf(most, __shfl_xor_sync(mask, most, d));
                scale = scale_of(most);
                if ((t & (lanes - 1)) == 0 && columns.in(j)) scales[c >> a.block_log] = scale;
            }
            if (!columns.in(j)) continue;
            const Pack<uint32_t, V / 4> q = to_8_bits<H>(v[j], scale);
            if (a.wide_out && c >= 0 && c + V <= width && c % V == 0) {
                *reinterpret_cast<Pack<uint32_t, V / 4>*>(out + c) = q;
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (c + k >= 0 && c + k < width) out[c + k] = (uint8_t)(q.v[k / 4] >> (k % 4 * 8));
            }
        }
    }
}

template <class T>
bool aligned16(const void* p, int64_t pitch) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && pitch * sizeof(T) % 16 == 0;
}

// Whether the rows of two matrices always start equally far from a 16-byte boundary.
template <class T>
bool alike(const void* p, int64_t p_pitch, const void* q, int64_t q_pitch, int64_t n) {
    return reinterpret_cast<uintptr_t>(p) % 16 == reinterpret_cast<uintptr_t>(q) % 16 && (n <= 1 || (p_pitch - q_pitch) * (int64_t)sizeof(T) % 16 == 0);
}

// Vectors of a thread and threads of a group for rows of `vecs` vectors: few vectors a thread while rows are short (short chains of
// latency), more for long rows (fewer warps to join).
struct Shape {
    int k, group;
};
// Threads of a CTA: one group of more than a warp, or several smaller ones.
int cta_threads(const Shape& shape) { return shape.group > 32 ? shape.group : 128; }

Shape shape_of(int64_t vecs, int64_t one, int64_t two, int64_t four, int least) {
    const int k = vecs <= one ? 1 : vecs <= two ? 2 : vecs <= four ? 4 : 8;
    const int64_t threads = ceil_div(vecs, k);
    int group = least;
    if (threads <= 32)
        while (group < threads) group *= 2;
    else
        group = (int)round_up(threads, 32);
    return {k, group};
}

template <class T>
bool is_full(const void* x, int64_t pitch, int64_t width, const Shape& shape) {
    return aligned16<T>(x, pitch) && width == (int64_t)shape.k * shape.group * kVec<T>;
}

template <class T, Lie LIE, int MODE>
cudaError_t launch_norm(NormKernelArgs& a, const Shape& shape, cudaStream_t s) {
    const unsigned threads = cta_threads(shape);
    const dim3 grid((unsigned)ceil_div(a.n, threads / shape.group));
    a.group = shape.group;
    constexpr Lie kLong = LIE == kFull ? kWide : LIE;  // the longest rows are not told apart
    switch (shape.k) {
        case 1: return launch_chained(k_norm<T, LIE, 1, MODE, 512>, grid, threads, 0, s, a);
        case 2: return launch_chained(k_norm<T, LIE, 2, MODE, 512>, grid, threads, 0, s, a);
        case 4: return launch_chained(k_norm<T, LIE, 4, MODE, 512>, grid, threads, 0, s, a);
        default: return launch_chained(k_norm<T, kLong, 8, MODE, (sizeof(T) == 2 ? 512 : 1024)>, grid, threads, 0, s, a);
    }
}

template <class T>
cudaError_t norm_typed(const NormArgs& n, cudaStream_t s) {
    constexpr int V = kVec<T>;
    const int block_log = n.block == 128 ? 7 : n.block == 64 ? 6 : 5;
    NormKernelArgs a{n.x, n.residual, n.weight, n.x_pitch, n.residual_pitch, n.n, (int)n.width, n.eps, 1.0f / (float)n.width, n.sum, n.out, n.sum_pitch, n.out_pitch, n.scales, block_log,
                     n.block ? (int)ceil_div(n.width, n.block) : 1, 0, reinterpret_cast<uintptr_t>(n.weight) % 16 == 0, false};
    bool wide = (!n.residual || alike<T>(n.x, n.x_pitch, n.residual, n.residual_pitch, n.n)) && (!n.sum || alike<T>(n.x, n.x_pitch, n.sum, n.sum_pitch, n.n));
    if (n.scales)
        a.wide_out = reinterpret_cast<uintptr_t>(n.out) % V == 0 && n.out_pitch % V == 0;
    else
        wide = wide && alike<T>(n.x, n.x_pitch, n.out, n.out_pitch, n.n);
    int64_t vecs = ceil_div(n.width, V);
    if (wide && !aligned16<T>(n.x, n.x_pitch)) {
        // a block's vectors start at its first column; a row that takes one vector more has to fit too
        if (n.block || n.width + V > kMaxNormWidth)
            wide = false;
        else
            vecs = ceil_div(n.width + V - 1, V);
    }
    // Rows of more than 32 vectors have two a thread (65,536 x 512 bf16 with a residual 41 us, 69 with one, which takes two warps a row). Rows of fp32 have four from 65 vectors on: 33.5 M elements in rows of 1,024 without a residual 41 us, 45 with two, in rows of 260 60 and 134, to 8 bits 70 and 79, with a residual 80 both ways. Rows of bf16 stay with
    // two: one row of 2,048 takes 2.5 us, 2.9 with four, and 16,384 with a residual 41 both ways; many rows without a residual would be faster with four (24 us, 27 with two).
    const Shape shape = shape_of(vecs, 32, sizeof(T) == 2 ? 1024 : 64, 2048, std::max<int>(8, (int)(n.block / V)));
    const Lie lie = !wide ? kAnywhere : is_full<T>(n.x, n.x_pitch, n.width, shape) ? kFull : kWide;
    auto launch = [&](auto mode) {
        constexpr int kMode = decltype(mode)::value;
        return lie == kFull ? launch_norm<T, kFull, kMode>(a, shape, s) : lie == kWide ? launch_norm<T, kWide, kMode>(a, shape, s) : launch_norm<T, kAnywhere, kMode>(a, shape, s);
    };
    if (!n.scales) return launch(std::integral_constant<int, 0>{});
    return n.block ? launch(std::integral_constant<int, 1>{}) : launch(std::integral_constant<int, 2>{});
}

// ---------------------------------------------------------------------------------------------
// Values from their 8 bits and scales. Bound by memory's latency, one load of 16 bytes a thread before the conversions: 8,192 x 2,048 to bf16 8.9 us where the values lie in L2, 13.5 from
// DRAM (3.7 TB/s); to fp32 20.5 us. Rows off boundaries go value by value: 8,192 x 2,049 28.8 us.
// ---------------------------------------------------------------------------------------------
constexpr int kBack = 16;  // values a thread takes at a time; blocks are multiples of it

template <class T>
__global__ void __launch_bounds__(256) k_dequantize(const uint8_t* values, int64_t values_pitch, const float* scales, int64_t n,
                                                    int width, int block_log, int blocks, T* __restrict__ out, int64_t out_pitch, int group) {
    ptx::chained();
    const int64_t row = (int64_t)blockIdx.x * (256 / group) + threadIdx.x / group;
    if (row >= n) return;
    auto value = [](uint8_t b) { return __half2float(__half(__nv_cvt_fp8_to_halfraw(b, __NV_E4M3))); };
#pragma unroll 2
    for (int c = (int)threadIdx.x % group * kBack; c < width; c += group * kBack) {
        const float scale = scales[row * blocks + (blocks > 1 ? c >> block_log : 0)];
        const uint8_t* q = values + row * values_pitch + c;
        T* o = out + row * out_pitch + c;
        if (c + kBack <= width) {
            const Words p = *reinterpret_cast<const Words*>(q);
            constexpr int V = kVec<T>;
#pragma unroll
            for (int k = 0; k < kBack; k += V) {
                float y[V];
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const __half2_raw two = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(p.w[(k + e) / 4] >> ((k + e) % 4 * 8)), __NV_E4M3);
                    const float2 f = __half22float2(__half2(two));
                    y[e] = f.x * scale, y[e + 1] = f.y * scale;
                }
                *reinterpret_cast<Words*>(o + k) = pack<T>(y);
            }
        } else {
            for (int k = 0; k < kBack && c + k < width; ++k) o[k] = narrow<T>(value(q[k]) * scale);
        }
    }
}

// Rows anywhere: neighbouring threads take neighbouring values.
template <class T>
__global__ void __launch_bounds__(256) k_dequantize_single(const uint8_t* values, int64_t values_pitch, const float* scales, int64_t n,
                                                           int width, int block_log, int blocks, T* __restrict__ out, int64_t out_pitch, int group) {
    ptx::chained();
    const int64_t row = (int64_t)blockIdx.x * (256 / group) + threadIdx.x / group;
    if (row >= n) return;
    constexpr int kAtOnce = 8;
    for (int c = (int)threadIdx.x % group; c < width; c += kAtOnce * group) {
        float f[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {  // all loads before the first store
            const int at = c + k * group;
            if (at < width) f[k] = __half2float(__half(__nv_cvt_fp8_to_halfraw(values[row * values_pitch + at], __NV_E4M3))) * scales[row * blocks + (blocks > 1 ? at >> block_log : 0)];
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (c + k * group < width) out[row * out_pitch + c + k * group] = narrow<T>(f[k]);
    }
}

template <class T>
cudaError_t dequantize_typed(const DequantizeArgs& a, cudaStream_t s) {
    const int blocks = a.block ? (int)ceil_div(a.width, a.block) : 1, block_log = a.block == 128 ? 7 : a.block == 64 ? 6 : 5;
    const bool wide = reinterpret_cast<uintptr_t>(a.values) % kBack == 0 && a.values_pitch % kBack == 0 && aligned16<T>(a.out, a.out_pitch);
    int group = 1;
    while (group < 256 && group * (wide ? 2 * kBack : 8) < a.width) group *= 2;
    return launch_chained(wide ? k_dequantize<T> : k_dequantize_single<T>, dim3((unsigned)ceil_div(a.n, 256 / group)), 256, 0, s, a.values, a.values_pitch,
                          a.scales, a.n, (int)a.width, block_log, blocks, static_cast<T*>(a.out), a.out_pitch, group);
}

// ---------------------------------------------------------------------------------------------
// Gradient. Bound by memory: g, s and ds are read once, dx written once. CTAs walk over rows a fixed number apart and keep their part of dw for the
// columns of each thread in registers; the parts go to the workspace and a second kernel adds them up in order. A slot (a group's sequence of rows)
// has rows a multiple of 8 apart, so that all of them start equally far from a 16-byte boundary and a thread's columns stay the same.
// The reductions over a row leave the loads idle, so the rows to come are brought to shared memory meanwhile: every thread copies the vectors that
// it will itself read, kStages rows deep, and waits for its own copies alone.
// Long rows (LEAN) have no room for that: they keep x and g in registers and dw in shared memory, every thread its own.
// 16,384 x 2,048 bf16 with ds: 51 us (5.3 TB/s), 16,384 x 1,024 fp32: 46 us (5.8 TB/s), of which the second kernel is 4 to 6; without the copies ahead the
// first took 108 us. What holds bf16 back is one CTA of 16 warps a multiprocessor (124 registers: the row, its gradient, the weight and dw as floats), whose
// issue slots are 60 % busy. 2,000 x 16,384 fp32 (LEAN): 149 us (3.5 TB/s).
// ---------------------------------------------------------------------------------------------
template <int K>
constexpr int kStagesOf = K <= 2 ? 3 : 2;

__device__ __forceinline__ void copy_ahead(void* to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((unsigned)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void close_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_copies() {
    asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float load_of_cta(const float* p, unsigned cta) {  // from the place p of another CTA's shared memory
    uint32_t at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(cta));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}

struct NormGradKernelArgs {
    const void *g, *x, *weight, *ds;
    int64_t g_pitch, x_pitch, ds_pitch, n;
    int width;
    float eps, one_over_width;
    void* dx;
    int64_t dx_pitch;
    float* parts;  // [CTAs][width], or NULL without a gradient of the weight, or if the CTAs are one cluster and join their parts themselves:
    void* dw;      // the gradient of the weight then, else NULL
    int64_t slots, x_step, g_step, ds_step, dx_step;  // elements from one row of a slot to the next
    int group;
    bool wide_weight;
};

template <class T, Lie LIE, int K, bool LEAN, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS) k_norm_grad(const __grid_constant__ NormGradKernelArgs a) {
    constexpr int V = kVec<T>, H = V / 2, kStages = kStagesOf<K>;
    constexpr bool WIDE = LIE != kAnywhere;
    __shared__ float shared[2][32 * kPlaces];
    extern __shared__ uint4 memory[];  // LEAN: every thread's part of dw. Else rows to come, and at the end, with several groups a CTA, a row of dw for each
    ptx::chained();
    const int group = a.group, width = a.width, groups = blockDim.x / group;
    const Place place(group);
    const int t = place.t, mine = place.mine;
    const int64_t first = (int64_t)blockIdx.x * groups + mine;
    const T* x = static_cast<const T*>(a.x) + first * a.x_pitch;
    const T* g = static_cast<const T*>(a.g) + first * a.g_pitch;
    const T* ds = static_cast<const T*>(a.ds) + first * a.ds_pitch;
    T* dx = static_cast<T*>(a.dx) + first * a.dx_pitch;
    const Columns<T, LIE, K> columns(x, t, group, width);
    // the vectors of one row: [stage][matrix][j][thread]
    auto ahead = [&](int stage, int matrix, int j) -> Words& { return reinterpret_cast<Words*>(memory)[((stage * 3 + matrix) * K + j) * blockDim.x + threadIdx.x]; };
    auto bring_row = [&](int stage, const T* x, const T* g, const T* ds) {
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if (!columns.in(j)) continue;
            if (WIDE) {
                copy_ahead(&ahead(stage, 0, j), x + columns.at(j));
                copy_ahead(&ahead(stage, 1, j), g + columns.at(j));
                if (a.ds) copy_ahead(&ahead(stage, 2, j), ds + columns.at(j));
            } else {
                ahead(stage, 0, j) = load_anywhere(x, columns.at(j), width);
                ahead(stage, 1, j) = load_anywhere(g, columns.at(j), width);
                if (a.ds) ahead(stage, 2, j) = load_anywhere(ds, columns.at(j), width);
            }
        }
    };
    float2 p[K][H], dw[LEAN ? 1 : K][H];
    auto own = [&](int j, int q) -> float4& { return reinterpret_cast<float4*>(memory)[(j * (V / 4) + q) * blockDim.x + threadIdx.x]; };  // LEAN
    auto load_weight = [&](int j) {
        if (a.weight && columns.in(j)) {
            unpack<T>(columns.load_weight(static_cast<const T*>(a.weight), j, a.wide_weight), p[j]);
        } else {
#pragma unroll
            for (int k = 0; k < H; ++k) p[j][k] = two(1.0f);
        }
    };
    int64_t coming = first;  // the next row to bring, with the three pointers
    if constexpr (!LEAN) {
#pragma unroll
        for (int s = 0; s + 1 < kStages; ++s) {
            if (coming < a.n) bring_row(s, x, g, ds);
            close_copies();
            coming += a.slots, x += a.x_step, g += a.g_step, ds += a.ds_step;
        }
#pragma unroll
        for (int j = 0; j < K; ++j) {
            load_weight(j);
#pragma unroll
            for (int k = 0; k < H; ++k) dw[j][k] = two(0.0f);
        }
    } else {
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int q = 0; q < V / 4; ++q) own(j, q) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    int slot = 0, stage = 0;
    for (int64_t row = first; row < a.n; row += a.slots, dx += a.dx_step) {
        float2 s[K][H], u[K][H];  // the row and its grad_out
        Words px[K], pg[K];
        if constexpr (LEAN) {
            columns.load(px, x);
            columns.load(pg, g);
            columns.clear_past_ends(px);
            columns.clear_past_ends(pg);
        } else {
            if (coming < a.n) bring_row(stage == 0 ? kStages - 1 : stage - 1, x, g, ds);
            close_copies();
            coming += a.slots, x += a.x_step, g += a.g_step, ds += a.ds_step;
            wait_copies<kStages - 1>();
#pragma unroll
            for (int j = 0; j < K; ++j) {
                px[j] = pg[j] = Words{};
                if (columns.in(j)) px[j] = ahead(stage, 0, j), pg[j] = ahead(stage, 1, j);
            }
            columns.clear_past_ends(px);
            columns.clear_past_ends(pg);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                unpack<T>(px[j], s[j]);
                unpack<T>(pg[j], u[j]);
            }
        }
        // by: a power of two that the row is multiplied by, one but for rows whose squares leave the range of floats
        float v[2];
        auto sums = [&](float by) {
            float2 q = two(0.0f), c = two(0.0f);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                if constexpr (LEAN) {
                    unpack<T>(px[j], s[j]);
                    unpack<T>(pg[j], u[j]);
                    load_weight(j);
                }
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    if (by != 1.0f) s[j][k] = mul2(s[j][k], two(by));
                    q = fma2(s[j][k], s[j][k], q);
                    c = fma2(s[j][k], mul2(u[j][k], p[j][k]), c);
                }
            }
            v[0] = q.x + q.y, v[1] = c.x + c.y;
            over_group<false, true, 2>(v, group, mine, slot, shared);
            slot ^= 1;
        };
        sums(1.0f);
        float by = 1.0f, rstd;
        if (in_range(v[0], a.eps * (float)width)) {
            rstd = rstd_of(fmaf(v[0], a.one_over_width, a.eps));
        } else {
            float most = 0.0f;
#pragma unroll
            for (int j = 0; j < K; ++j) {
                if constexpr (LEAN) unpack<T>(px[j], s[j]);
#pragma unroll
                for (int k = 0; k < H; ++k) most = fmaxf(most, fmaxf(fabsf(s[j][k].x), fabsf(s[j][k].y)));
            }
            by = power_below(over_group<true, true>(most, group, mine, slot, shared));
            slot ^= 1;
            sums(by);
            rstd = scaled_rstd(by, v[0], width, a.eps);
        }
        // dx = w g rstd - h (c rstd) + ds, where rstd of the row itself is `by` times that of the scaled one
        const float true_rstd = rstd * by, back = -(v[1] * rstd * a.one_over_width) * true_rstd;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if (!columns.in(j)) continue;
            float2 d[H];
            if constexpr (LEAN) {
                unpack<T>(!a.ds ? Words{} : WIDE ? *reinterpret_cast<const Words*>(ds + columns.at(j)) : load_anywhere(ds, columns.at(j), width), d);
                unpack<T>(px[j], s[j]);
                unpack<T>(pg[j], u[j]);
                if (by != 1.0f) {
#pragma unroll
                    for (int k = 0; k < H; ++k) s[j][k] = mul2(s[j][k], two(by));
                }
                load_weight(j);
            } else {
                unpack<T>(a.ds ? ahead(stage, 2, j) : Words{}, d);
            }
#pragma unroll
            for (int k = 0; k < H; ++k) {
                const float2 hat = mul2(s[j][k], two(rstd));
                d[k] = fma2(mul2(u[j][k], two(true_rstd)), p[j][k], fma2(hat, two(back), d[k]));
                if constexpr (LEAN)
                    s[j][k] = hat;
                else
                    dw[j][k] = fma2(u[j][k], hat, dw[j][k]);
            }
            if constexpr (LEAN) {
#pragma unroll
                for (int q = 0; q < V / 4; ++q) {
                    const float4 f = own(j, q);
                    const float2 low = fma2(u[j][2 * q], s[j][2 * q], make_float2(f.x, f.y)), high = fma2(u[j][2 * q + 1], s[j][2 * q + 1], make_float2(f.z, f.w));
                    own(j, q) = make_float4(low.x, low.y, high.x, high.y);
                }
            }
            if (a.dx) columns.store(dx, j, pack<T>(d));
        }
        if constexpr (LEAN)
            x += a.x_step, g += a.g_step, ds += a.ds_step;
        else
            stage = stage + 1 == kStages ? 0 : stage + 1;
    }
    if (!a.parts && !a.dw) return;
    float* rows = reinterpret_cast<float*>(memory);
    const bool one_cluster = !LEAN && a.dw;
    if (!LEAN && (groups > 1 || one_cluster)) {
        wait_copies<0>();
        __syncthreads();  // the place of the rows to come is free
    }
    float* part = one_cluster ? rows + (groups > 1 ? groups * width : 0) : a.parts + (int64_t)blockIdx.x * width;
    float* to = groups > 1 ? rows + mine * width : part;
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
        for (int k = 0; k < H; ++k) {
            float2 f;
            if constexpr (LEAN)
                f = k % 2 ? make_float2(own(j, k / 2).z, own(j, k / 2).w) : make_float2(own(j, k / 2).x, own(j, k / 2).y);
            else
                f = dw[j][k];
            const int c = columns.at(j) + 2 * k;
            if (c >= 0 && c < width) to[c] = f.x;
            if (c + 1 >= 0 && c + 1 < width) to[c + 1] = f.y;
        }
    if (groups > 1) {
        __syncthreads();
        for (int c = threadIdx.x; c < width; c += blockDim.x) {
            float sum = 0.0f;
            for (int q = 0; q < groups; ++q) sum += rows[q * width + c];
            part[c] = sum;
        }
    }
    if (!one_cluster) return;
    // the columns are shared out over the CTAs of the cluster; sixteen lanes take a column, each the part of one CTA
    cluster_barrier();
    const int q = threadIdx.x % 16, columns_at_once = blockDim.x / 16;
    for (int i = 0; i * (int)gridDim.x < width; i += columns_at_once) {
        const int c = (i + (int)threadIdx.x / 16) * gridDim.x + blockIdx.x;
        float sum = c < width && q < (int)gridDim.x ? load_of_cta(part + c, q) : 0.0f;
#pragma unroll
        for (int d = 8; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (q == 0 && c < width) static_cast<T*>(a.dw)[c] = narrow<T>(sum);
    }
    cluster_barrier();  // no CTA ends while another reads its memory
}

// dw from the CTAs' parts: 32 columns a CTA, every warp a share of the parts, joined in order.
template <class T>
__global__ void __launch_bounds__(1024) k_norm_join(const float* parts, int64_t count, int64_t width, T* __restrict__ dw) {
    __shared__ float sums[32][33];
    ptx::chained();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (c < width)
#pragma unroll 8
        for (int64_t q = warp; q < count; q += 32) sum += parts[q * width + c];
    sums[warp][lane] = sum;
    __syncthreads();
    sum = sums[lane][warp];
#pragma unroll
    for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    const int64_t to = (int64_t)blockIdx.x * 32 + warp;
    if (lane == 0 && to < width) dw[to] = narrow<T>(sum);
}

template <class T>
Shape grad_shape(int64_t width, bool shifted) {  // shifted: rows may start behind a 16-byte boundary, and take a vector more
    return shape_of(ceil_div(width + (shifted ? kVec<T> - 1 : 0), kVec<T>), 32, 1024, 2048, 8);
}

// The first kernel's launch. A CTA has as many groups as make 512 threads, for a part of dw each CTA is written and read again; fewer where there are not rows
// enough to give each multiprocessor some. At most as many CTAs as are resident at once (two a multiprocessor with one vector a thread, else one); where a
// group has several rows, so many that the slots are a multiple of 8.
// With few rows they are one cluster of up to 16 CTAs, which joins its parts of dw itself: no workspace, and no second launch.
constexpr int kClusterRows = 2;  // of a group, at most: 1,001 x 201 fp32 (four rows each) 9.5 us in one launch, 6.7 in two

struct GradLaunch {
    int groups;
    int64_t ctas;
    bool one_cluster;
};
GradLaunch grad_launch(int64_t n, const Shape& shape, bool lean, bool with_weight) {
    const int most_groups = std::max(1, 512 / shape.group);
    if (!lean && with_weight && n <= (int64_t)16 * most_groups * kClusterRows)
        return {most_groups, std::min<int64_t>(16, std::max<int64_t>(1, ceil_div(n, most_groups))), true};
    const int64_t sms = multiprocessors(), resident = sms * (shape.k == 1 ? 2 : 1);
    const int whole = std::max(1, 32 / shape.group);  // groups of a warp
    int groups = (int)std::min<int64_t>(most_groups, round_up(std::max<int64_t>(ceil_div(n, sms), 1), whole));
    const int64_t ctas = ceil_div(n, groups);
    if (ctas <= resident) return {groups, std::max<int64_t>(ctas, 1), false};
    int64_t most = resident;
    while (most * groups % 8) --most;
    return {groups, std::max<int64_t>(most, 1), false};
}
template <class T>
bool is_lean(const Shape& shape) {
    return shape.k > (sizeof(T) == 2 ? 2 : 4);
}

template <class T, Lie LIE, int K, bool LEAN, int THREADS>
cudaError_t launch_grad_kernel(const NormGradKernelArgs& a, unsigned ctas, unsigned threads, cudaStream_t s) {
    constexpr int kCtas = !LEAN && K == 1 ? 2 : 1;
    constexpr size_t each = LEAN ? K * kVec<T> * 4 : kStagesOf<K> * 3 * K * 16, most = each * THREADS;  // bytes of a thread
    static std::atomic<uint64_t> allowed{0};
    auto* kernel = k_norm_grad<T, LIE, K, LEAN, THREADS, kCtas>;
    A2_CUDA_TRY(allow_shared_memory(reinterpret_cast<const void*>(kernel), (int)most, allowed));
    if (a.dw) {
        static std::atomic<uint64_t> clusters{0};
        if (ctas > 8) A2_CUDA_TRY(allow_large_clusters(reinterpret_cast<const void*>(kernel), clusters));
        return launch_clusters(kernel, dim3(ctas), threads, each * threads, ctas, s, a);
    }
    return launch_chained(kernel, dim3(ctas), threads, each * threads, s, a);  // rows of dw of several groups, and their sum, take less: K vectors of floats a thread
}

template <class T, Lie LIE>
cudaError_t launch_norm_grad(NormGradKernelArgs& a, const Shape& shape, const GradLaunch& launch, cudaStream_t s) {
    const unsigned threads = launch.groups * shape.group, ctas = (unsigned)launch.ctas;
    a.group = shape.group;
    a.slots = launch.ctas * launch.groups;
    a.x_step = a.slots * a.x_pitch, a.g_step = a.slots * a.g_pitch, a.ds_step = a.slots * a.ds_pitch, a.dx_step = a.slots * a.dx_pitch;
    constexpr Lie kLong = LIE == kFull ? kWide : LIE;
    switch (shape.k) {
        case 1: return launch_grad_kernel<T, LIE, 1, false, 512>(a, ctas, threads, s);
        case 2: return launch_grad_kernel<T, LIE, 2, false, 512>(a, ctas, threads, s);
        case 4: return launch_grad_kernel<T, LIE, 4, sizeof(T) == 2, 512>(a, ctas, threads, s);
        default: break;
    }
    if (threads <= 512) return launch_grad_kernel<T, kLong, 8, true, 512>(a, ctas, threads, s);
    return launch_grad_kernel<float, kLong, 8, true, 1024>(a, ctas, threads, s);  // rows of fp32 alone are that long
}

template <class T>
cudaError_t norm_grad_typed(const NormGradArgs& n, void* workspace, cudaStream_t s) {
    const bool aligned = aligned16<T>(n.x, n.x_pitch), room = n.width + kVec<T> <= kMaxNormWidth;
    const bool wide = alike<T>(n.x, n.x_pitch, n.grad_out, n.grad_out_pitch, n.n) && (!n.grad_sum || alike<T>(n.x, n.x_pitch, n.grad_sum, n.grad_sum_pitch, n.n)) &&
                      (!n.grad_x || alike<T>(n.x, n.x_pitch, n.grad_x, n.grad_x_pitch, n.n)) && (aligned || room);
    const Shape shape = grad_shape<T>(n.width, wide && !aligned);
    const GradLaunch launch = grad_launch(n.n, shape, is_lean<T>(shape), n.grad_weight != nullptr);
    const bool parts = n.grad_weight && !launch.one_cluster;
    NormGradKernelArgs a{n.grad_out, n.x, n.weight, n.grad_sum, n.grad_out_pitch, n.x_pitch, n.grad_sum_pitch, n.n, (int)n.width, n.eps, 1.0f / (float)n.width, n.grad_x, n.grad_x_pitch,
                         parts ? Carver(workspace).take<float>(launch.ctas * n.width) : nullptr, launch.one_cluster ? n.grad_weight : nullptr, 0, 0, 0, 0, 0, 0,
                         reinterpret_cast<uintptr_t>(n.weight) % 16 == 0};
    const cudaError_t e = !wide ? launch_norm_grad<T, kAnywhere>(a, shape, launch, s)
                          : is_full<T>(n.x, n.x_pitch, n.width, shape) ? launch_norm_grad<T, kFull>(a, shape, launch, s) : launch_norm_grad<T, kWide>(a, shape, launch, s);
    A2_CUDA_TRY(e);
    if (!parts) return cudaSuccess;
    return launch_chained(k_norm_join<T>, dim3((unsigned)ceil_div(n.width, 32)), 1024, 0, s, a.parts, launch.ctas, n.width, static_cast<T*>(n.grad_weight));
}

}  // namespace

cudaError_t run_norm(const NormArgs& a, cudaStream_t s) {
    if (a.n == 0) return cudaSuccess;
    return a.dtype == A2_BF16 ? norm_typed<__nv_bfloat16>(a, s) : norm_typed<float>(a, s);
}

cudaError_t run_dequantize(const DequantizeArgs& a, cudaStream_t s) {
    if (a.n == 0) return cudaSuccess;
    return a.dtype == A2_BF16 ? dequantize_typed<__nv_bfloat16>(a, s) : dequantize_typed<float>(a, s);
}

int64_t norm_grad_workspace(int64_t n, int64_t width, bool with_weight, int32_t dtype) {
    if (!with_weight) return 0;
    Carver c(nullptr);
    int64_t most = 0;
    for (const bool shifted : {false, true}) {
        if (shifted && width + 8 > kMaxNormWidth) continue;
        const Shape shape = dtype == A2_BF16 ? grad_shape<__nv_bfloat16>(width, shifted) : grad_shape<float>(width, shifted);
        const GradLaunch launch = grad_launch(n, shape, dtype == A2_BF16 ? is_lean<__nv_bfloat16>(shape) : is_lean<float>(shape), true);
        if (!launch.one_cluster) most = std::max(most, launch.ctas);
    }
    if (most == 0) return 0;
    c.take<float>(most * width);
    return c.used;
}

cudaError_t run_norm_grad(const NormGradArgs& a, void* workspace, cudaStream_t s) {
    return a.dtype == A2_BF16 ? norm_grad_typed<__nv_bfloat16>(a, workspace, s) : norm_grad_typed<float>(a, workspace, s);
}

}  // namespace a2
