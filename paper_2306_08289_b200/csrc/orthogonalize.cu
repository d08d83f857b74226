// Orthogonalisation of a batch of matrices by Newton-Schulz products: X = G / (|G|_F + eps), then
//   A = X X^T,  B = (a - q) I + b A + c A^2,  X <- q X + B X
// (the same for any q; one in the middle of the polynomial's range makes B, and so its rounding, smallest) on the smaller side m <= n. All three products run on the tensor cores; A and B are symmetric, so only tiles on and below
// the diagonal are computed and the others are written as their transposes: 3 m^2 n + m^3 operations a step instead of
// 4 m^2 n + 2 m^3. A tall matrix (rows > cols) stays as it lies: Y = X^T, A = Y^T Y, Y <- q Y + Y B.
//
// The intermediates are fp16 words at power-of-two scales: one word with bf16 rows (11 bits; bf16 words would lose 8 times as
// much per rounding, and the roundings of small singular values grow up to a^steps), two with fp32 rows. X's elements are bounded by
// its largest singular value, so the scale 2^14 leaves it room up to 4; the entry point refuses coefficients that
// leave that room. The first X keeps G's own bits: it is stored as G 2^e and its true scale u is a factor of the epilogues.
#include <algorithm>
#include <cmath>

#include "gemm_sm100.cuh"

namespace a2 {

namespace {

constexpr float kScale = 16384.0f;  // 2^14
// 65504 / 2^14 = 3.998 bounds X, A = X X^T and B; the rest is for rounding
constexpr double kMostSingular = 1.95, kMostPoly = 3.9;

// What the kernels know of each matrix.
struct MatScale {
    float u;  // X0 = u * (the stored words)
    int e;    // stored words = G * 2^e
    int r;    // |X0|_F <= 2^r, r <= 0: far below zero when eps outweighs the norm
};

// |X_k|_F <= 2^r(k): the scale of the stored words of X_k, k >= 1, is 2^(14 - r(k)), so that a matrix far smaller than eps
// keeps its bits.
__device__ __forceinline__ int next_bound(int r, float a, float b, float c) {
    if (r >= 0) return 0;
    const float s = ldexpf(1.0f, 2 * r);
    const float growth = fabsf(a) + fabsf(b) * s + fabsf(c) * s * s;
    return min(0, r + (growth > 1.0f ? ilogbf(growth) + 1 : 0));
}

struct Poly {
    float a, b, c, q;
    int step;  // 0 .. steps - 1
};

// Value of one stored unit of X at step `step`, and of the next X's stored unit.
__device__ __forceinline__ void units(const MatScale& s, const Poly& p, float* now, float* next) {
    int r = s.r;
    for (int k = 0; k < p.step; ++k) r = next_bound(r, p.a, p.b, p.c);
    *now = p.step == 0 ? s.u : ldexpf(1.0f, r - 14);
    *next = ldexpf(1.0f, next_bound(r, p.a, p.b, p.c) - 14);
}

// ---- norm and first words ------------------------------------------------------------------------
constexpr int kNormThreads = 256;

template <class T>
__global__ void __launch_bounds__(kNormThreads) k_norm(const T* __restrict__ in, int64_t stride, int64_t pitch, int64_t rows, int64_t cols,
                                                       double* __restrict__ partial) {
    __shared__ double part[kNormThreads / 32];
    const T* g = in + blockIdx.y * stride;
    double sum = 0.0;
    const int64_t warp = (int64_t)blockIdx.x * (kNormThreads / 32) + threadIdx.x / 32, warps = (int64_t)gridDim.x * (kNormThreads / 32);
    for (int64_t i = warp; i < rows; i += warps) {
#pragma unroll 4
        for (int64_t j = threadIdx.x % 32; j < cols; j += 32) {
            const double v = widen(g[i * pitch + j]);  // the squares of fp32 values may leave fp32
            sum += v * v;
        }
    }
    for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double all = 0.0;
        for (int w = 0; w < kNormThreads / 32; ++w) all += part[w];
        partial[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = all;
    }
}

__device__ __forceinline__ void split_words(float x, __half& hi, __half& lo) {
    hi = __float2half_rn(x);
    const float back = __half2float(hi);
    lo = __float2half_rn(isfinite(back) ? x - back : 0.0f);
}

__device__ __forceinline__ MatScale mat_scale(const double* partial, int parts, double eps) {
    double all = 0.0;
    for (int p = 0; p < parts; ++p) all += partial[p];
    const double norm = sqrt(all), by = norm + eps;
    if (!(norm <= 1e300)) return {NAN, 0, 0};
    if (norm == 0.0) return {0.0f, 0, 0};
    const int e = 13 - ilogb(norm);  // norm * 2^e in [2^13, 2^14)
    return {(float)(1.0 / (ldexp(by, e))), e, min(0, ilogb(norm / by) + 1)};
}

// Words of G 2^e, [rows, ld].
template <class T>
__global__ void __launch_bounds__(kNormThreads) k_first_words(const T* __restrict__ in, int64_t stride, int64_t pitch, int64_t rows, int64_t cols,
                                                              const double* __restrict__ partial, int parts, double eps, __half* __restrict__ hi,
                                                              __half* __restrict__ lo, int64_t ld, MatScale* __restrict__ scales) {
    __shared__ MatScale shared;
    if (threadIdx.x == 0) {
        shared = mat_scale(partial + (int64_t)blockIdx.y * parts, parts, eps);
        if (blockIdx.x == 0) scales[blockIdx.y] = shared;
    }
    __syncthreads();
    const int e = shared.e;
    const T* g = in + blockIdx.y * stride;
    const int64_t base = (int64_t)blockIdx.y * rows * ld;
    const int64_t warp = (int64_t)blockIdx.x * (kNormThreads / 32) + threadIdx.x / 32, warps = (int64_t)gridDim.x * (kNormThreads / 32);
    for (int64_t i = warp; i < rows; i += warps)
#pragma unroll 4
        for (int64_t j = threadIdx.x % 32; j < cols; j += 32) {
            __half h, l;
            split_words(scalbnf(widen(g[i * pitch + j]), e), h, l);
            hi[base + i * ld + j] = h;
            if (lo) lo[base + i * ld + j] = l;
        }
}

// steps = 0: the normalised matrix itself.
template <class T>
__global__ void __launch_bounds__(kNormThreads) k_normalized(const __half* hi, const __half* lo, int64_t ld, int64_t rows, int64_t cols,
                                                             const MatScale* scales, float scale, T* out, int64_t stride, int64_t pitch) {
    const float by = scales[blockIdx.y].u * scale;
    const int64_t base = (int64_t)blockIdx.y * rows * ld;
    const int64_t warp = (int64_t)blockIdx.x * (kNormThreads / 32) + threadIdx.x / 32, warps = (int64_t)gridDim.x * (kNormThreads / 32);
    for (int64_t i = warp; i < rows; i += warps)
        for (int64_t j = threadIdx.x % 32; j < cols; j += 32) {
            const int64_t at = base + i * ld + j;
            out[blockIdx.y * stride + i * pitch + j] = narrow<T>((__half2float(hi[at]) + (lo ? __half2float(lo[at]) : 0.0f)) * by);
        }
}

// ---- epilogues ------------------------------------------------------------------------------------
// A matrix of one or two words in the workspace; ld is a multiple of 64, rows of `mats` matrices one after another.
struct Words {
    __half* hi;
    __half* lo;  // or NULL
    int64_t ld, stride;
};

__device__ __forceinline__ void read_words(const Words& w, int64_t at, float (&x)[32]) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        const Pack<__half, 16> h = *reinterpret_cast<const Pack<__half, 16>*>(w.hi + at + g * 16);
#pragma unroll
        for (int k = 0; k < 16; ++k) x[g * 16 + k] = __half2float(h.v[k]);
        if (w.lo) {
            const Pack<__half, 16> l = *reinterpret_cast<const Pack<__half, 16>*>(w.lo + at + g * 16);
#pragma unroll
            for (int k = 0; k < 16; ++k) x[g * 16 + k] += __half2float(l.v[k]);
        }
    }
}
__device__ __forceinline__ void write_words(const Words& w, int64_t at, const float (&x)[32]) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        Pack<__half, 16> h, l;
#pragma unroll
        for (int k = 0; k < 16; ++k) split_words(x[g * 16 + k], h.v[k], l.v[k]);
        *reinterpret_cast<Pack<__half, 16>*>(w.hi + at + g * 16) = h;
        if (w.lo) *reinterpret_cast<Pack<__half, 16>*>(w.lo + at + g * 16) = l;
    }
}

// A = X X^T (kQuadratic false) or B = (a - q) I + b A + c A^2 (true), symmetric: tiles below the diagonal are written twice.
template <bool kQuadratic>
struct SymmetricEpi {
    struct Args {
        Words from, to;  // from: A, for B
        int64_t m;
        const MatScale* scales;
        Poly poly;
    };
    const Args& a;
    int64_t row0, col0, mat;
    int lane;
    bool mirror;
    float factor;
    __device__ __forceinline__ SymmetricEpi(const Args& args, int b, int row, int col, int lane_, float*)
        : a(args), row0(row), col0(col), mat(b), lane(lane_), mirror(row / kTileM != col / kTileN) {
        if (kQuadratic) {
            factor = a.poly.c / kScale;
        } else {
            float now, next;
            units(a.scales[b], a.poly, &now, &next);
            factor = kScale * now * now;
        }
    }
    __device__ __forceinline__ void chunk(int c, float (&v)[32]) {
        const int64_t col = col0 + c * 32, row = row0 + lane;
        if (row >= a.m || col >= a.m) return;
        const int64_t at = mat * a.to.stride + row * a.to.ld + col;
        if (kQuadratic) {
            float x[32];
            read_words(a.from, at, x);
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] = a.poly.b * x[k] + factor * v[k] + (row == col + k ? (a.poly.a - a.poly.q) * kScale : 0.0f);
        } else {
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] *= factor;
        }
        write_words(a.to, at, v);
        if (mirror) {  // col < row0: all 32 columns lie inside the matrix
            const int64_t turned = mat * a.to.stride + col * a.to.ld + row;
#pragma unroll
            for (int k = 0; k < 32; ++k) {
                __half h, l;
                split_words(v[k], h, l);
                a.to.hi[turned + k * a.to.ld] = h;
                if (a.to.lo) a.to.lo[turned + k * a.to.ld] = l;
            }
        }
    }
    __device__ __forceinline__ void finish() {}
};

// X <- q X + B X; the last step writes the caller's matrix.
template <class T>
struct UpdateEpi {
    struct Args {
        Words from, to;
        int64_t rows, cols;
        const MatScale* scales;
        Poly poly;
        T* out;  // last step, else NULL
        int64_t stride, pitch;
        float scale;
    };
    const Args& a;
    int64_t row0, col0, mat;
    int lane;
    float* staging;
    float factor;
    __device__ __forceinline__ UpdateEpi(const Args& args, int b, int row, int col, int lane_, float* staging_)
        : a(args), row0(row), col0(col), mat(b), lane(lane_), staging(staging_) {
        float now, next;
        units(a.scales[b], a.poly, &now, &next);
        factor = a.out ? a.scale * now : now / next;
    }
    __device__ __forceinline__ void chunk(int c, float (&v)[32]) {
        const int64_t col = col0 + c * 32, row = row0 + lane;
        if (col >= a.cols) return;
        if (row < a.rows) {
            const int64_t at = mat * a.from.stride + row * a.from.ld + col;
            float x[32];
            read_words(a.from, at, x);
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] = (a.poly.q * x[k] + v[k] / kScale) * factor;
            if (!a.out) write_words(a.to, at, v);
        }
        if (!a.out) return;
#pragma unroll
        for (int k = 0; k < 32; ++k) staging[lane * kStagePitch + k] = v[k];
        __syncwarp();
        if (col + lane < a.cols) {
            T* to = a.out + mat * a.stride + row0 * a.pitch + col + lane;
            const int rows = (int)min((int64_t)32, a.rows - row0);
#pragma unroll 8
            for (int r = 0; r < rows; ++r) to[r * a.pitch] = narrow<T>(staging[r * kStagePitch + lane]);
        }
        __syncwarp();
    }
    __device__ __forceinline__ void finish() {}
};

// ---- layout and launches ---------------------------------------------------------------------------
constexpr int kFlush = 4;  // K blocks a sum stays in tensor memory with fp32 rows: 16 steps of the tensor core

struct Layout {
    double* partial;
    MatScale* scales;
    Words x, y, gram, poly;
    int64_t parts;
};

int64_t layout(int64_t mats, int64_t rows, int64_t cols, int32_t dtype, void* ws, Layout* out) {
    const int64_t m = std::min(rows, cols);
    Carver w(ws);
    Layout l{};
    l.parts = std::max<int64_t>(1, std::min<int64_t>({ceil_div(rows, 8), ceil_div(148 * 8, mats > 0 ? mats : 1), 256}));
    l.partial = w.take<double>(mats * l.parts);
    l.scales = w.take<MatScale>(mats);
    auto take = [&](int64_t r, int64_t c) {
        Words v{};
        v.ld = round_up(c, 64);
        v.stride = r * v.ld;
        v.hi = w.take<__half>(mats * v.stride);
        if (dtype == A2_F32) v.lo = w.take<__half>(mats * v.stride);
        return v;
    };
    l.x = take(rows, cols);
    l.y = take(rows, cols);
    l.gram = take(m, m);
    l.poly = take(m, m);
    if (out) *out = l;
    return w.used;
}

template <class T>
cudaError_t typed(const OrthogonalizeArgs& a, Layout l, cudaStream_t s) {
    constexpr bool kWords = sizeof(T) == 4;
    const int flush = kWords ? kFlush : 0;
    const bool tall = a.rows > a.cols;
    const int64_t m = std::min(a.rows, a.cols), n = std::max(a.rows, a.cols);
    const dim3 grid((unsigned)l.parts, (unsigned)a.n_mats);
    k_norm<T><<<grid, kNormThreads, 0, s>>>(static_cast<const T*>(a.in), a.in_stride, a.in_pitch, a.rows, a.cols, l.partial);
    k_first_words<T><<<grid, kNormThreads, 0, s>>>(static_cast<const T*>(a.in), a.in_stride, a.in_pitch, a.rows, a.cols, l.partial, (int)l.parts,
                                                   a.eps, l.x.hi, l.x.lo, l.x.ld, l.scales);
    if (a.steps == 0)
        k_normalized<T><<<grid, kNormThreads, 0, s>>>(l.x.hi, l.x.lo, l.x.ld, a.rows, a.cols, l.scales, a.scale, static_cast<T*>(a.out), a.out_stride,
                                                      a.out_pitch);
    auto operand = [](const Words& w, int64_t rows, int64_t k, bool mn) { return Operand{w.hi, w.lo, rows, k, w.ld, w.stride, mn}; };
    Words x = l.x, y = l.y;
    for (int step = 0; step < a.steps; ++step) {
        const Poly poly{a.ca, a.cb, a.cc, a.center, step};
        GemmArgs g;
        const Operand side = operand(x, m, n, tall);
        cudaError_t e = make_gemm(side, side, a.n_mats, false, true, flush, &g);
        if (e != cudaSuccess) return e;
        e = launch_gemm<SymmetricEpi<false>, kWords>(g, {l.gram, l.gram, m, l.scales, poly}, s);
        if (e != cudaSuccess) return e;
        const Operand gram = operand(l.gram, m, m, false);
        e = make_gemm(gram, gram, a.n_mats, false, true, flush, &g);
        if (e != cudaSuccess) return e;
        e = launch_gemm<SymmetricEpi<true>, kWords>(g, {l.gram, l.poly, m, l.scales, poly}, s);
        if (e != cudaSuccess) return e;
        const Operand b = operand(l.poly, m, m, false);
        e = tall ? make_gemm(operand(x, a.rows, m, false), b, a.n_mats, false, false, flush, &g)
                 : make_gemm(b, operand(x, n, m, true), a.n_mats, false, false, flush, &g);
        if (e != cudaSuccess) return e;
        const bool last = step + 1 == a.steps;
        e = launch_gemm<UpdateEpi<T>, kWords>(
            g, {x, y, a.rows, a.cols, l.scales, poly, last ? static_cast<T*>(a.out) : nullptr, a.out_stride, a.out_pitch, a.scale}, s);
        if (e != cudaSuccess) return e;
        std::swap(x, y);
    }
    return cudaGetLastError();
}

}  // namespace

bool orthogonalize_range(double a, double b, double c, int steps, double* center) {
    // singular values start in [0, 1]; how far each step's polynomial takes them, on a grid
    double reach = 1.0, low = 0.0, high = 0.0;
    *center = a;
    for (int step = 0; step < steps; ++step) {
        double next = reach;
        low = high = 0.0;
        for (int k = 0; k <= 4096; ++k) {
            const double x = reach * k / 4096, s = x * x, p = b * s + c * s * s;
            low = std::min(low, p);
            high = std::max(high, p);
            next = std::max(next, std::abs(x * (a + p)));
        }
        *center = a + (low + high) / 2;
        if (!(next <= kMostSingular) || !((high - low) / 2 <= kMostPoly)) return false;
        if (next == reach) break;
        reach = next;
    }
    return true;
}

int64_t orthogonalize_workspace(int64_t n_mats, int64_t rows, int64_t cols, int32_t dtype) {
    return layout(n_mats, rows, cols, dtype, nullptr, nullptr);
}

cudaError_t run_orthogonalize(const OrthogonalizeArgs& a, void* workspace, cudaStream_t s) {
    Layout l;
    layout(a.n_mats, a.rows, a.cols, a.dtype, workspace, &l);
    return a.dtype == A2_BF16 ? typed<__nv_bfloat16>(a, l, s) : typed<float>(a, l, s);
}

}  // namespace a2
