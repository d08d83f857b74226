// Root-mean-square norm with the residual's addition, y = s / sqrt(mean s^2 + eps) w with s = x + r, its output in 8 bits, and its gradient
//   hat = s rstd,  c = mean(hat w g),  dx = rstd (w g - hat c) + ds,  dw = sum over rows of g hat.
#include <cuda_fp8.h>

#include <algorithm>
#include <atomic>

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
// all rows are shifted alike): the first and the last vector are cut at the row's ends, element by element. WIDE = false reads all vectors
// element by element.
// ---------------------------------------------------------------------------------------------
template <class T>
constexpr int kVec = 16 / sizeof(T);

template <class T, bool WIDE>
__device__ __forceinline__ void load(Pack<T, kVec<T>>& to, const T* row, int64_t c, int64_t width) {
    if (WIDE && c >= 0 && c + kVec<T> <= width) {
        to = *reinterpret_cast<const Pack<T, kVec<T>>*>(row + c);
    } else {
#pragma unroll
        for (int k = 0; k < kVec<T>; ++k) to.v[k] = c + k >= 0 && c + k < width ? row[c + k] : narrow<T>(0.0f);
    }
}
template <class T, bool WIDE>
__device__ __forceinline__ void store(T* row, int64_t c, int64_t width, const Pack<T, kVec<T>>& from) {
    if (WIDE && c >= 0 && c + kVec<T> <= width) {
        *reinterpret_cast<Pack<T, kVec<T>>*>(row + c) = from;
    } else {
#pragma unroll
        for (int k = 0; k < kVec<T>; ++k)
            if (c + k >= 0 && c + k < width) row[c + k] = from.v[k];
    }
}

// Sums (or maxima) of two values over a group, the same bits in every thread. Groups of more than a warp are whole CTAs; `slot` changes from
// one such reduction to the next (0, 1, 0, ...), so that one barrier each is enough.
template <bool MAX>
__device__ __forceinline__ float2 over_group(float2 v, int group, int slot, float2 (*shared)[32]) {
    const int lane = threadIdx.x % 32;
    const int span = group < 32 ? group : 32;
    const unsigned mask = span == 32 ? 0xffffffffu : ((1u << span) - 1u) << (lane & ~(span - 1));
    auto join = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
    for (int d = span / 2; d > 0; d /= 2) {
        v.x = join(v.x, __shfl_xor_sync(mask, v.x, d));
        v.y = join(v.y, __shfl_xor_sync(mask, v.y, d));
    }
    if (group <= 32) return v;
    const int warps = group / 32;
    if (lane == 0) shared[slot][threadIdx.x / 32] = v;
    __syncthreads();
    v = lane < warps ? shared[slot][lane] : make_float2(0.0f, 0.0f);  // zero is neutral for both: maxima are of magnitudes
    for (int d = 16; d > 0; d /= 2) {
        v.x = join(v.x, __shfl_xor_sync(0xffffffffu, v.x, d));
        v.y = join(v.y, __shfl_xor_sync(0xffffffffu, v.y, d));
    }
    return v;
}

// rstd as a product of two factors, `by` a power of two: values whose squares leave the range of floats are scaled first.
struct Rstd {
    float by, r;
};
__device__ __forceinline__ bool in_range(float squares, float eps_sum) { return squares < 0x1p120f && squares + eps_sum > 0x1p-90f; }
__device__ __forceinline__ float power_below(float most) {  // 2^-e for most in [2^e, 2^(e+1))
    if (!(most > 0.0f) || isinf(most)) return 1.0f;
    int e;
    frexpf(most, &e);
    return ldexpf(1.0f, max(-126, min(126, 1 - e)));
}
__device__ __forceinline__ Rstd scaled_rstd(float by, float squares, int64_t width, float eps) {
    const double mean = (double)squares / (double)width + (double)eps * by * by;
    return {by, mean > 0.0 ? (float)(1.0 / sqrt(mean)) : (isnan(mean) ? (float)mean : 0.0f)};  // a row of zeros with eps = 0 gives zeros
}

struct NormKernelArgs {
    const void *x, *residual, *weight;
    int64_t x_pitch, residual_pitch, n, width;
    float eps;
    void *sum, *out;
    int64_t sum_pitch, out_pitch;
    float* scales;
    int64_t block, blocks;
    int group;
    bool wide_weight, wide_out;
};

// ---------------------------------------------------------------------------------------------
// Forward. Bound by memory: x and r are read once, s and y written once, the row stays in registers as floats in between. A group holds one
// row. MODE 0: y in the rows' type. 1: e4m3 with a scale for every `block` columns, whose vectors lie in neighbouring lanes. 2: e4m3 with one
// scale a row. Sums are in fp32; s is rounded only where it is stored, y is formed from what it was before.
// ---------------------------------------------------------------------------------------------
template <class T, bool WIDE, int K, int MODE, int THREADS>
__global__ void __launch_bounds__(THREADS) k_norm(const NormKernelArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float2 shared[2][32];
    ptx::chained();
    const int group = a.group;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / group) + threadIdx.x / group;
    if (row >= a.n) return;  // whole groups, and whole CTAs where a group is one
    const int t = threadIdx.x % group;
    const T* x = static_cast<const T*>(a.x) + row * a.x_pitch;
    const T* r = static_cast<const T*>(a.residual) + row * a.residual_pitch;
    T* sum = static_cast<T*>(a.sum) + row * a.sum_pitch;
    const T* w = static_cast<const T*>(a.weight);
    const int shift = WIDE ? (int)(reinterpret_cast<uintptr_t>(x) % 16 / sizeof(T)) : 0;

    float v[K][V];
    {
        Pack<T, V> px[K], pr[K];
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int64_t c = (int64_t)(j * group + t) * V - shift;
            if (c < a.width) load<T, WIDE>(px[j], x, c, a.width);
        }
        if (a.residual) {
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const int64_t c = (int64_t)(j * group + t) * V - shift;
                if (c < a.width) load<T, WIDE>(pr[j], r, c, a.width);
            }
        }
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int64_t c = (int64_t)(j * group + t) * V - shift;
#pragma unroll
            for (int k = 0; k < V; ++k) v[j][k] = c < a.width ? widen(px[j].v[k]) : 0.0f;
            if (a.residual && c < a.width) {
#pragma unroll
                for (int k = 0; k < V; ++k) v[j][k] += widen(pr[j].v[k]);
            }
            if (a.sum && c < a.width) {
                Pack<T, V> p;
#pragma unroll
                for (int k = 0; k < V; ++k) p.v[k] = narrow<T>(v[j][k]);
                store<T, WIDE>(sum, c, a.width, p);
            }
        }
    }
    float squares = 0.0f;
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) squares = fmaf(v[j][k], v[j][k], squares);
    squares = over_group<false>(make_float2(squares, 0.0f), group, 0, shared).x;
    int slot = 1;
    Rstd rstd{1.0f, 0.0f};
    if (in_range(squares, a.eps * (float)a.width)) {
        rstd.r = 1.0f / sqrtf(squares / (float)a.width + a.eps);
    } else {
        float most = 0.0f;
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int k = 0; k < V; ++k) most = fmaxf(most, fabsf(v[j][k]));
        const float by = power_below(over_group<true>(make_float2(most, 0.0f), group, 1, shared).x);
        float again = 0.0f;
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int k = 0; k < V; ++k) again = fmaf(v[j][k] * by, v[j][k] * by, again);
        rstd = scaled_rstd(by, over_group<false>(make_float2(again, 0.0f), group, 0, shared).x, a.width, a.eps);
    }
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const int64_t c = (int64_t)(j * group + t) * V - shift;
        if (c >= a.width) continue;
        Pack<T, V> pw;
        if (w) {
            if (a.wide_weight && shift == 0)
                load<T, true>(pw, w, c, a.width);
            else
                load<T, false>(pw, w, c, a.width);
        }
#pragma unroll
        for (int k = 0; k < V; ++k) {
            v[j][k] = v[j][k] * rstd.by * rstd.r;
            if (w) v[j][k] *= widen(pw.v[k]);
        }
        if (MODE == 0) {
            Pack<T, V> p;
#pragma unroll
            for (int k = 0; k < V; ++k) p.v[k] = narrow<T>(v[j][k]);
            store<T, WIDE>(static_cast<T*>(a.out) + row * a.out_pitch, c, a.width, p);
        }
    }
    if constexpr (MODE != 0) {
        uint8_t* out = static_cast<uint8_t*>(a.out) + row * a.out_pitch;
        float most_of_row = 0.0f;
        if (MODE == 2) {
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k) most_of_row = fmaxf(most_of_row, fabsf(v[j][k]));
            most_of_row = over_group<true>(make_float2(most_of_row, 0.0f), group, slot, shared).x;
        }
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int64_t c = (int64_t)(j * group + t) * V - shift;
            float most = most_of_row;
            if (MODE == 1) {  // vectors past the row's end hold zeros
                const int lanes = (int)a.block / V;
                const int span = group < 32 ? group : 32, lane = threadIdx.x % 32;
                const unsigned mask = span == 32 ? 0xffffffffu : ((1u << span) - 1u) << (lane & ~(span - 1));
#pragma unroll
                for (int k = 0; k < V; ++k) most = fmaxf(most, fabsf(v[j][k]));
                for (int d = lanes / 2; d > 0; d /= 2) most = fmaxf(most, __shfl_xor_sync(mask, most, d));
            }
            if (c >= a.width) continue;
            const float scale = fmaxf(most / kE4m3Most, kScaleLeast);
            const float inverse = 1.0f / scale;
            const int64_t block = MODE == 1 ? c / a.block : 0;
            if (MODE == 1 ? c % a.block == 0 : (j == 0 && t == 0)) a.scales[row * a.blocks + block] = scale;
            Pack<uint8_t, V> q;
#pragma unroll
            for (int k = 0; k < V; ++k) q.v[k] = __nv_cvt_float_to_fp8(v[j][k] * inverse, __NV_SATFINITE, __NV_E4M3);
            if (a.wide_out && shift == 0 && c + V <= a.width) {
                *reinterpret_cast<Pack<uint8_t, V>*>(out + c) = q;
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (c + k >= 0 && c + k < a.width) out[c + k] = q.v[k];
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

template <class T, bool WIDE, int MODE>
cudaError_t launch_norm(NormKernelArgs& a, const Shape& shape, cudaStream_t s) {
    const unsigned threads = cta_threads(shape);
    const dim3 grid((unsigned)ceil_div(a.n, threads / shape.group));
    a.group = shape.group;
    switch (shape.k) {
        case 1: return launch_chained(k_norm<T, WIDE, 1, MODE, 512>, grid, threads, 0, s, a);
        case 2: return launch_chained(k_norm<T, WIDE, 2, MODE, 512>, grid, threads, 0, s, a);
        case 4: return launch_chained(k_norm<T, WIDE, 4, MODE, 512>, grid, threads, 0, s, a);
        default: return launch_chained(k_norm<T, WIDE, 8, MODE, (sizeof(T) == 2 ? 512 : 1024)>, grid, threads, 0, s, a);
    }
}

template <class T>
cudaError_t norm_typed(const NormArgs& n, cudaStream_t s) {
    constexpr int V = kVec<T>;
    NormKernelArgs a{n.x, n.residual, n.weight, n.x_pitch, n.residual_pitch, n.n, n.width, n.eps, n.sum, n.out, n.sum_pitch, n.out_pitch, n.scales, n.block,
                     n.block ? ceil_div(n.width, n.block) : 1, 0, reinterpret_cast<uintptr_t>(n.weight) % 16 == 0, false};
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
    const Shape shape = sizeof(T) == 2 ? shape_of(vecs, 256, 1024, 2048, std::max<int>(8, (int)(n.block / V)))
                                       : shape_of(vecs, 128, 512, 2048, std::max<int>(8, (int)(n.block / V)));
    if (!n.scales) return wide ? launch_norm<T, true, 0>(a, shape, s) : launch_norm<T, false, 0>(a, shape, s);
    if (n.block) return wide ? launch_norm<T, true, 1>(a, shape, s) : launch_norm<T, false, 1>(a, shape, s);
    return wide ? launch_norm<T, true, 2>(a, shape, s) : launch_norm<T, false, 2>(a, shape, s);
}

// ---------------------------------------------------------------------------------------------
// Values from their 8 bits and scales. Bound by memory.
// ---------------------------------------------------------------------------------------------
constexpr int kBack = 8;  // values a thread

template <class T, bool WIDE>
__global__ void __launch_bounds__(256) k_dequantize(const uint8_t* __restrict__ values, int64_t values_pitch, const float* __restrict__ scales, int64_t n,
                                                    int64_t width, int64_t block, int64_t blocks, int64_t pieces, T* __restrict__ out, int64_t out_pitch) {
    ptx::chained();
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = at / pieces, c = at % pieces * kBack;
    if (row >= n) return;
    const float scale = scales[row * blocks + (block ? c / block : 0)];  // blocks are multiples of a thread's values
    const uint8_t* q = values + row * values_pitch + c;
    T* o = out + row * out_pitch + c;
    auto value = [&](uint8_t b) {
        const __half_raw h = __nv_cvt_fp8_to_halfraw(b, __NV_E4M3);
        return narrow<T>(__half2float(__half(h)) * scale);
    };
    if (WIDE && c + kBack <= width) {
        const Pack<uint8_t, kBack> p = *reinterpret_cast<const Pack<uint8_t, kBack>*>(q);
        constexpr int V = kVec<T>;
#pragma unroll
        for (int k = 0; k < kBack; k += V) {
            Pack<T, V> y;
#pragma unroll
            for (int e = 0; e < V; ++e) y.v[e] = value(p.v[k + e]);
            *reinterpret_cast<Pack<T, V>*>(o + k) = y;
        }
    } else {
        for (int k = 0; k < kBack && c + k < width; ++k) o[k] = value(q[k]);
    }
}

template <class T>
cudaError_t dequantize_typed(const DequantizeArgs& a, cudaStream_t s) {
    const int64_t pieces = ceil_div(a.width, kBack), blocks = a.block ? ceil_div(a.width, a.block) : 1;
    const bool wide = reinterpret_cast<uintptr_t>(a.values) % kBack == 0 && a.values_pitch % kBack == 0 && aligned16<T>(a.out, a.out_pitch);
    return launch_chained(wide ? k_dequantize<T, true> : k_dequantize<T, false>, dim3((unsigned)ceil_div(a.n * pieces, 256)), 256, 0, s, a.values, a.values_pitch,
                          a.scales, a.n, a.width, a.block, blocks, pieces, static_cast<T*>(a.out), a.out_pitch);
}

// ---------------------------------------------------------------------------------------------
// Gradient. Bound by memory: g, s and ds are read once, dx written once. CTAs walk over rows a fixed number apart and keep their part of dw for the
// columns of each thread, in registers (in shared memory for long rows, LEAN); the parts go to the workspace and a second kernel adds
// them up in order. A slot (a group's sequence of rows) has rows a multiple of 8 apart, so that all of them start equally far from a
// 16-byte boundary and a thread's columns stay the same.
// ---------------------------------------------------------------------------------------------
struct NormGradKernelArgs {
    const void *g, *x, *weight, *ds;
    int64_t g_pitch, x_pitch, ds_pitch, n, width;
    float eps;
    void* dx;
    int64_t dx_pitch;
    float* parts;  // [CTAs][width], or NULL without a gradient of the weight
    int64_t slots;
    int group;
};

template <class T, bool WIDE, int K, bool LEAN, int THREADS>
__global__ void __launch_bounds__(THREADS) k_norm_grad(const NormGradKernelArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float2 shared[2][32];
    extern __shared__ float columns[];  // LEAN: this CTA's dw. Else, with several groups a CTA: one row of dw for each
    ptx::chained();
    const int group = a.group, groups = blockDim.x / group, t = threadIdx.x % group, mine = threadIdx.x / group;
    const int64_t first = (int64_t)blockIdx.x * groups + mine;
    const T* w = static_cast<const T*>(a.weight);
    const int shift = WIDE ? (int)(reinterpret_cast<uintptr_t>(static_cast<const T*>(a.x) + first * a.x_pitch) % 16 / sizeof(T)) : 0;
    Pack<T, V> pw[LEAN ? 1 : K];
    float dw[LEAN ? 1 : K][V];
    if (!LEAN) {
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int64_t c = (int64_t)(j * group + t) * V - shift;
            if (w && c < a.width) load<T, false>(pw[LEAN ? 0 : j], w, c, a.width);
#pragma unroll
            for (int k = 0; k < V; ++k) dw[LEAN ? 0 : j][k] = 0.0f;
        }
    } else if (a.parts) {
        for (int64_t c = threadIdx.x; c < a.width; c += blockDim.x) columns[c] = 0.0f;
        __syncthreads();
    }
    int slot = 0;
    for (int64_t row = first; row < a.n; row += a.slots) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_pitch;
        const T* g = static_cast<const T*>(a.g) + row * a.g_pitch;
        const T* ds = static_cast<const T*>(a.ds) + row * a.ds_pitch;
        T* dx = static_cast<T*>(a.dx) + row * a.dx_pitch;
        Pack<T, V> px[K], pg[K];
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int64_t c = (int64_t)(j * group + t) * V - shift;
            if (c < a.width) {
                load<T, WIDE>(px[j], x, c, a.width);
                load<T, WIDE>(pg[j], g, c, a.width);
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k) px[j].v[k] = pg[j].v[k] = narrow<T>(0.0f);
            }
        }
        auto weights = [&](int j, int64_t c) {
            Pack<T, V> p;
            if (!LEAN) return pw[LEAN ? 0 : j];
            if (w && c < a.width)
                load<T, false>(p, w, c, a.width);
            return p;
        };
        auto sums = [&](float by) {
            float2 v = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const int64_t c = (int64_t)(j * group + t) * V - shift;
                if (c >= a.width) continue;
                const Pack<T, V> p = weights(j, c);
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float s = widen(px[j].v[k]) * by;
                    const float wg = widen(pg[j].v[k]) * (w ? widen(p.v[k]) : 1.0f);
                    v.x = fmaf(s, s, v.x);
                    v.y = fmaf(s, wg, v.y);
                }
            }
            v = over_group<false>(v, group, slot, shared);
            slot ^= 1;
            return v;
        };
        float2 v = sums(1.0f);
        Rstd rstd{1.0f, 0.0f};
        if (in_range(v.x, a.eps * (float)a.width)) {
            rstd.r = 1.0f / sqrtf(v.x / (float)a.width + a.eps);
        } else {
            float most = 0.0f;
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int k = 0; k < V; ++k) most = fmaxf(most, fabsf(widen(px[j].v[k])));
            most = over_group<true>(make_float2(most, 0.0f), group, slot, shared).x;
            slot ^= 1;
            const float by = power_below(most);
            v = sums(by);
            rstd = scaled_rstd(by, v.x, a.width, a.eps);
        }
        const float c_mean = v.y * rstd.r / (float)a.width;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int64_t c = (int64_t)(j * group + t) * V - shift;
            if (c >= a.width) continue;
            const Pack<T, V> p = weights(j, c);
            Pack<T, V> pd, o;
            if (a.ds) load<T, WIDE>(pd, ds, c, a.width);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float hat = widen(px[j].v[k]) * rstd.by * rstd.r, gk = widen(pg[j].v[k]);
                const float wg = w ? gk * widen(p.v[k]) : gk;
                float d = (wg - hat * c_mean) * rstd.r * rstd.by;
                if (a.ds) d += widen(pd.v[k]);
                o.v[k] = narrow<T>(d);
                if (!LEAN)
                    dw[LEAN ? 0 : j][k] = fmaf(gk, hat, dw[LEAN ? 0 : j][k]);
                else if (a.parts && c + k >= 0 && c + k < a.width)
                    columns[c + k] = fmaf(gk, hat, columns[c + k]);
            }
            if (a.dx) store<T, WIDE>(dx, c, a.width, o);
        }
    }
    if (!a.parts) return;
    float* part = a.parts + (int64_t)blockIdx.x * a.width;
    if (LEAN) {
        __syncthreads();
        for (int64_t c = threadIdx.x; c < a.width; c += blockDim.x) part[c] = columns[c];
        return;
    }
    float* to = groups > 1 ? columns + mine * a.width : part;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const int64_t c = (int64_t)(j * group + t) * V - shift;
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (c + k >= 0 && c + k < a.width) to[c + k] = dw[LEAN ? 0 : j][k];
    }
    if (groups > 1) {
        __syncthreads();
        for (int64_t c = threadIdx.x; c < a.width; c += blockDim.x) {
            float sum = 0.0f;
            for (int q = 0; q < groups; ++q) sum += columns[q * a.width + c];
            part[c] = sum;
        }
    }
}

// dw from the CTAs' parts: 32 columns a CTA, every warp a share of the parts, joined in order.
template <class T>
__global__ void __launch_bounds__(1024) k_norm_join(const float* __restrict__ parts, int64_t count, int64_t width, T* __restrict__ dw) {
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

constexpr int kGradThreads = 2048 / 2;  // threads of a multiprocessor's CTAs

template <class T>
Shape grad_shape(int64_t width) {
    return shape_of(ceil_div(width + (width + kVec<T> <= kMaxNormWidth ? kVec<T> - 1 : 0), kVec<T>), 512, 1024, 2048, 8);
}

// CTAs of the first kernel: enough to fill the GPU, at most one row for each group, a multiple of 8 where a group has several rows.
int64_t grad_ctas(int64_t n, const Shape& shape) {
    const int threads = cta_threads(shape), groups = threads / shape.group;
    const int64_t full = (int64_t)multiprocessors() * std::max(1, kGradThreads / threads);
    const int64_t needed = ceil_div(n, groups);
    return needed <= full ? std::max<int64_t>(needed, 1) : round_up(full, 8);
}

template <class T, bool WIDE>
cudaError_t launch_norm_grad(NormGradKernelArgs& a, const Shape& shape, int64_t ctas, cudaStream_t s) {
    const unsigned threads = cta_threads(shape);
    const int groups = threads / shape.group;
    a.group = shape.group;
    a.slots = ctas * groups;
    const dim3 grid((unsigned)ctas);
    const size_t several = groups > 1 && a.parts ? (size_t)groups * a.width * 4 : 0, whole = a.parts ? (size_t)a.width * 4 : 0;
    auto lean = [&](auto* kernel) -> cudaError_t {
        A2_CUDA_TRY(cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMaxNormWidth * 4));
        return launch_chained(kernel, grid, threads, whole, s, a);
    };
    switch (shape.k) {
        case 1: return launch_chained(k_norm_grad<T, WIDE, 1, false, 512>, grid, threads, several, s, a);
        case 2: return launch_chained(k_norm_grad<T, WIDE, 2, false, 512>, grid, threads, several, s, a);
        case 4: return lean(k_norm_grad<T, WIDE, 4, true, 512>);
        default: break;
    }
    if (threads <= 512) return lean(k_norm_grad<T, WIDE, 8, true, 512>);
    return lean(k_norm_grad<float, WIDE, 8, true, 1024>);  // rows of fp32 alone are that long
}

template <class T>
cudaError_t norm_grad_typed(const NormGradArgs& n, void* workspace, cudaStream_t s) {
    const Shape shape = grad_shape<T>(n.width);
    const int64_t ctas = grad_ctas(n.n, shape);
    NormGradKernelArgs a{n.grad_out, n.x, n.weight, n.grad_sum, n.grad_out_pitch, n.x_pitch, n.grad_sum_pitch, n.n, n.width, n.eps, n.grad_x, n.grad_x_pitch,
                         n.grad_weight ? Carver(workspace).take<float>(ctas * n.width) : nullptr, 0, 0};
    const bool wide = alike<T>(n.x, n.x_pitch, n.grad_out, n.grad_out_pitch, n.n) && (!n.grad_sum || alike<T>(n.x, n.x_pitch, n.grad_sum, n.grad_sum_pitch, n.n)) &&
                      (!n.grad_x || alike<T>(n.x, n.x_pitch, n.grad_x, n.grad_x_pitch, n.n)) && (aligned16<T>(n.x, n.x_pitch) || n.width + kVec<T> <= kMaxNormWidth);
    A2_CUDA_TRY((wide ? launch_norm_grad<T, true>(a, shape, ctas, s) : launch_norm_grad<T, false>(a, shape, ctas, s)));
    if (!n.grad_weight) return cudaSuccess;
    return launch_chained(k_norm_join<T>, dim3((unsigned)ceil_div(n.width, 32)), 1024, 0, s, a.parts, ctas, n.width, static_cast<T*>(n.grad_weight));
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
    c.take<float>(grad_ctas(n, dtype == A2_BF16 ? grad_shape<__nv_bfloat16>(width) : grad_shape<float>(width)) * width);
    return c.used;
}

cudaError_t run_norm_grad(const NormGradArgs& a, void* workspace, cudaStream_t s) {
    return a.dtype == A2_BF16 ? norm_grad_typed<__nv_bfloat16>(a, workspace, s) : norm_grad_typed<float>(a, workspace, s);
}

}  // namespace a2
