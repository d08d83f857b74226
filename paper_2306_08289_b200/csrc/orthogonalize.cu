// Orthogonalisation of a batch of matrices by Newton-Schulz products: X = G / (|G|_F + eps), then
//   A = X X^T,  B = a I + b A + c A^2,  X <- B X
// on the smaller side m <= n. All three products run on the tensor cores; A and B are symmetric, so only tiles on and below
// the diagonal are computed and stored, and a product reads the others as the transposes of those: 3 m^2 n + m^3 operations a
// step instead of 4 m^2 n + 2 m^3. A tall matrix (rows > cols) stays as it lies: Y = X^T, A = Y^T Y, Y <- Y B.
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

// What the kernels know of each matrix. Powers of two are kept as exponents: when eps outweighs the norm they lie far below the
// smallest float.
struct MatScale {
    float u;  // X0 = u * 2^k * (the stored words)
    int k;
    int e;  // stored words = G * 2^e
    int r;  // |X0|_F <= 2^r, r <= 0
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
    float a, b, c;
    int step;  // 0 .. steps - 1
};

// 2^e for e <= 127, zero below the normal numbers.
__device__ __forceinline__ float power_of_two(int e) { return e < -126 ? 0.0f : __int_as_float((e + 127) << 23); }

// A stored unit of X at step `step` is worth u * 2^k, one of the next X 2^next.
struct Units {
    float u;
    int k, next;
    __device__ __forceinline__ Units(const MatScale& s, const Poly& p) {
        int r = s.r;
        for (int i = 0; i < p.step; ++i) r = next_bound(r, p.a, p.b, p.c);
        u = p.step == 0 ? s.u : 1.0f;
        k = p.step == 0 ? s.k : r - 14;
        next = next_bound(r, p.a, p.b, p.c) - 14;
    }
    // What sums of words of X times words of X become in A's words (2^14).
    __device__ __forceinline__ float gram() const { return kScale * u * u * power_of_two(2 * k); }
};

// v * scale * u * 2^k, in factors that leave the range only if the result does.
struct Scaled {
    float a, b;
    __device__ __forceinline__ Scaled(float scale, float u, int k) {
        int e = 0;
        const float m = frexpf(scale, &e);
        const PowerOfTwo up(e + k);
        a = m * u * up.a;
        b = up.b;
    }
    __device__ __forceinline__ float operator()(float v) const { return v * a * b; }
};

// ---- norm and first words ------------------------------------------------------------------------
constexpr int kNormThreads = 256;

// Columns j .. j + VEC - 1 of a row, 0 past its end. Only whole groups are read at once, and those only where rows allow it (VEC = 1 else).
template <class T, int VEC>
__device__ __forceinline__ Pack<T, VEC> read_columns(const T* row, int64_t j, int64_t cols) {
    if (j + VEC <= cols) return *reinterpret_cast<const Pack<T, VEC>*>(row + j);
    Pack<T, VEC> x;
#pragma unroll
    for (int k = 0; k < VEC; ++k) x.v[k] = j + k < cols ? row[j + k] : narrow<T>(0.0f);
    return x;
}

template <class T, int VEC>
__global__ void __launch_bounds__(kNormThreads) k_norm(const T* in, int64_t stride, int64_t pitch, int64_t rows, int64_t cols,
                                                       double* __restrict__ partial) {
    ptx::chained();
    __shared__ double part[kNormThreads / 32];
    const T* g = in + blockIdx.y * stride;
    double sum = 0.0;
    const int64_t warp = (int64_t)blockIdx.x * (kNormThreads / 32) + threadIdx.x / 32, warps = (int64_t)gridDim.x * (kNormThreads / 32);
    for (int64_t i = warp; i < rows; i += warps) {
#pragma unroll 4
        for (int64_t j = threadIdx.x % 32 * VEC; j < cols; j += 32 * VEC) {
            const Pack<T, VEC> x = read_columns<T, VEC>(g + i * pitch, j, cols);
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                const double v = widen(x.v[k]);  // the squares of fp32 values may leave fp32
                sum += v * v;
            }
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

__device__ __forceinline__ MatScale mat_scale(double squares, double eps) {
    const double norm = sqrt(squares), by = fmin(norm + eps, 1.7e308);
    if (!(norm <= 1e300)) return {NAN, 0, 0, 0};
    if (norm == 0.0) return {0.0f, 0, 0, 0};
    const int n = ilogb(norm), d = ilogb(by), e = 13 - n;  // norm * 2^e in [2^13, 2^14)
    const double norm1 = ldexp(norm, -n), by1 = ldexp(by, -d);  // in [1, 2)
    return {(float)(1.0 / by1), -d - e, e, min(0, n - d + (norm1 >= by1 ? 1 : 0))};
}

// Words of G 2^e, [rows, ld].
template <class T, int VEC>
__global__ void __launch_bounds__(kNormThreads) k_first_words(const T* in, int64_t stride, int64_t pitch, int64_t rows, int64_t cols,
                                                              const double* partial, int parts, double eps, __half* __restrict__ hi, __half* __restrict__ lo, int64_t ld,
                                                              MatScale* __restrict__ scales) {
    ptx::chained();
    __shared__ MatScale shared;
    if (threadIdx.x < 32) {
        double sum = 0.0;
        for (int p = threadIdx.x; p < parts; p += 32) sum += partial[(int64_t)blockIdx.y * parts + p];
        for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (threadIdx.x == 0) {
            shared = mat_scale(sum, eps);
            if (blockIdx.x == 0) scales[blockIdx.y] = shared;
        }
    }
    __syncthreads();
    const PowerOfTwo up(shared.e);
    const T* g = in + blockIdx.y * stride;
    const int64_t base = (int64_t)blockIdx.y * rows * ld;
    const int64_t warp = (int64_t)blockIdx.x * (kNormThreads / 32) + threadIdx.x / 32, warps = (int64_t)gridDim.x * (kNormThreads / 32);
    for (int64_t i = warp; i < rows; i += warps)
#pragma unroll 4
        for (int64_t j = threadIdx.x % 32 * VEC; j < cols; j += 32 * VEC) {
            const Pack<T, VEC> x = read_columns<T, VEC>(g + i * pitch, j, cols);
            Pack<__half, VEC> h, l;
#pragma unroll
            for (int k = 0; k < VEC; ++k) split_words(up(widen(x.v[k])), h.v[k], l.v[k]);
            *reinterpret_cast<Pack<__half, VEC>*>(hi + base + i * ld + j) = h;  // ld is a multiple of 64: the last ones may be padding
            if (lo) *reinterpret_cast<Pack<__half, VEC>*>(lo + base + i * ld + j) = l;
        }
}

// steps = 0: the normalised matrix itself.
template <class T>
__global__ void __launch_bounds__(kNormThreads) k_normalized(const __half* hi, const __half* lo, int64_t ld, int64_t rows, int64_t cols,
                                                             const MatScale* scales, float scale, T* out, int64_t stride, int64_t pitch) {
    ptx::chained();
    const Scaled by(scale, scales[blockIdx.y].u, scales[blockIdx.y].k);
    const int64_t base = (int64_t)blockIdx.y * rows * ld;
    const int64_t warp = (int64_t)blockIdx.x * (kNormThreads / 32) + threadIdx.x / 32, warps = (int64_t)gridDim.x * (kNormThreads / 32);
    for (int64_t i = warp; i < rows; i += warps)
        for (int64_t j = threadIdx.x % 32; j < cols; j += 32) {
            const int64_t at = base + i * ld + j;
            out[blockIdx.y * stride + i * pitch + j] = narrow<T>(by(__half2float(hi[at]) + (lo ? __half2float(lo[at]) / kLowUp : 0.0f)));
        }
}

// ---- epilogues ------------------------------------------------------------------------------------
// A matrix of one or two words in the workspace; ld is a multiple of 64, rows of `mats` matrices one after another.
struct Words {
    __half* hi;
    __half* lo;  // or NULL
    int64_t ld, stride;
};

// Words of 32 x 32 values, a row a lane (staging: 4 KB).
__device__ __forceinline__ void write_words(const Words& w, int64_t at, const float (&x)[32], int rows, int lane, float* staging) {
    __half h[32], l[32];
#pragma unroll
    for (int k = 0; k < 32; k += 2) split_pair(x[k], x[k + 1], h[k], h[k + 1], l[k], l[k + 1]);
    char* s = reinterpret_cast<char*>(staging);
    store_rows16(s, h, w.hi + at, w.ld, rows, lane);
    if (w.lo) store_rows16(s + 2048, l, w.lo + at, w.ld, rows, lane);
}

// A = X X^T (kQuadratic false) or B = a I + b A + c A^2 (true), symmetric: tiles above the diagonal are
// neither computed nor stored.
template <bool kQuadratic>
struct SymmetricEpi {
    struct Args {
        Words from, to;  // from: A, for B
        int64_t m;
        const MatScale* scales;
        Poly poly;
        float* parts;  // A alone: sums of the parts of K, [parts][matrix][m][ld], or NULL when K is whole
        int64_t part_stride;
    };
    const Args& a;
    int64_t row0, col0, mat, split;
    int lane;
    float* staging;
    float factor;
    __device__ __forceinline__ SymmetricEpi(const Args& args, const Tile& t, int row, int col, int lane_, float* staging_)
        : a(args), row0(row), col0(col), mat(t.b), split(t.split), lane(lane_), staging(staging_) {
        if (kQuadratic) {
            factor = a.poly.c / kScale;
        } else {
            factor = Units(a.scales[mat], a.poly).gram();
        }
    }
    __device__ __forceinline__ void chunk(int c, float (&v)[32]) {
        const int64_t col = col0 + c * 32;
        if (row0 >= a.m || col >= a.m) return;  // rows of `to` are padded to 64 columns: only rows need care
        const int rows = (int)min((int64_t)32, a.m - row0);
        const int64_t at = mat * a.to.stride + row0 * a.to.ld + col;
        if (!kQuadratic && a.parts) {
            turn_columns(staging, v, lane);
            float* to = a.parts + split * a.part_stride + at + lane;
#pragma unroll
            for (int r = 0; r < 32; ++r)
                if (r < rows) to[r * a.to.ld] = v[r];
            return;
        }
        if (kQuadratic) {
            __half x[32];
            load_rows16(staging, x, a.from.hi + at, a.from.ld, rows, lane);
#pragma unroll
            for (int k = 0; k < 32; ++k)
                v[k] = a.poly.b * __half2float(x[k]) + factor * v[k] + (row0 + lane == col + k ? a.poly.a * kScale : 0.0f);
            if (a.from.lo) {
                load_rows16(staging, x, a.from.lo + at, a.from.ld, rows, lane);
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] += a.poly.b / kLowUp * __half2float(x[k]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] *= factor;
        }
        write_words(a.to, at, v, rows, lane, staging);
    }
    __device__ __forceinline__ void finish() {}
};

// Adds up the parts of A = X X^T, in order, on and below the diagonal tiles. Two columns a thread.
__global__ void __launch_bounds__(256) k_join_gram(const float* parts, int n_parts, int64_t part_stride, Words to, int64_t m,
                                                   const MatScale* scales, Poly poly) {
    ptx::chained();
    const int64_t row = blockIdx.y, mat = blockIdx.z, col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 2;
    if (col >= m || col / kTileN > row / kTileM) return;
    const float factor = Units(scales[mat], poly).gram();
    const int64_t at = mat * to.stride + row * to.ld + col;  // ld is even: the second column may be padding
    float x = 0.0f, y = 0.0f;
#pragma unroll 4
    for (int p = 0; p < n_parts; ++p) {
        const float2 v = *reinterpret_cast<const float2*>(parts + p * part_stride + at);
        x += v.x;
        y += v.y;
    }
    Pack<__half, 2> h, l;
    split_pair(x * factor, y * factor, h.v[0], h.v[1], l.v[0], l.v[1]);
    *reinterpret_cast<Pack<__half, 2>*>(to.hi + at) = h;
    if (to.lo) *reinterpret_cast<Pack<__half, 2>*>(to.lo + at) = l;
}

// X <- B X; the last step writes the caller's matrix.
template <class T>
struct UpdateEpi {
    struct Args {
        Words to;
        int64_t rows, cols;
        const MatScale* scales;
        Poly poly;
        T* out;  // last step, else NULL
        int64_t stride, pitch;
        float scale;
    };
    const Args& a;
    int row0, col0, mat;
    int lane;
    float* staging;
    float factor, rest;  // rest: the caller's matrix alone
    __device__ __forceinline__ UpdateEpi(const Args& args, const Tile& t, int row, int col, int lane_, float* staging_)
        : a(args), row0(row), col0(col), mat(t.b), lane(lane_), staging(staging_), rest(1.0f) {
        const Units x(a.scales[mat], a.poly);
        if (a.out) {
            const Scaled by(a.scale, x.u, x.k - 14);
            factor = by.a;
            rest = by.b;
        } else {
            factor = x.u * power_of_two(x.k - x.next - 14);  // both bound the same X: about 2^-14
        }
    }
    __device__ __forceinline__ void chunk(int c, float (&v)[32]) {
        const int col = col0 + c * 32;
        if (row0 >= a.rows || col >= a.cols) return;
        const int rows = (int)min((int64_t)32, a.rows - row0);
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] *= factor;
        if (!a.out) {
            write_words(a.to, mat * a.to.stride + row0 * a.to.ld + col, v, rows, lane, staging);
            return;
        }
        turn_columns(staging, v, lane);
        if (col + lane < a.cols) {
            T* to = a.out + mat * a.stride + row0 * a.pitch + col + lane;
#pragma unroll
            for (int r = 0; r < 32; ++r)
                if (r < rows) to[r * a.pitch] = narrow<T>(v[r] * rest);
        }
    }
    __device__ __forceinline__ void finish() {}
};

// ---- layout and launches ---------------------------------------------------------------------------
constexpr int64_t kPairs = 74, kLeastBlocks = 6;  // pairs of CTAs; fewest blocks of K worth a part (of three passes; four times that of one)
// K blocks a sum stays in tensor memory with fp32 rows, in the products of A, A^2 and B X. What A^2's sums lose goes into every singular value and is what
// the result's error follows; A's hardly show. 16 x 1,001 x 512, us, and 80 to 120 matrices of 129 to 1,200 a side, how many are over 1.5 times as far
// from 64 bits as a plain fp32 form and the median of that ratio: stays of 2, 2, 2 477 us, 47 of 80, 1.61; 1, 2, 2 494, 48 of 80, 1.64; 2, 1, 2 490, 1 of 80,
// 1.07; 4, 1, 2 483, 1 of 120, 1.05; 4, 1, 1 497, none, 0.96; 8, 1, 1 495, none, 1.17. The worst ratios are those of m up to 256, where a block more or
// less of B X costs little: one block there.
constexpr int kFlushGram = 4, kFlushPoly = 1, kFlushUpdate = 2;
int update_flush(int64_t m) { return m <= kTileM ? 1 : kFlushUpdate; }

struct Layout {
    double* partial;
    MatScale* scales;
    Words x, y, gram, poly;
    int64_t parts;
    int gram_parts;  // of K = n in A = X X^T, so that few matrices fill the GPU
    float* gram_sums;
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
    const int64_t side = ceil_div(m, kTileM);
    l.gram_parts = split_parts(mats * side * (side + 1) / 2, ceil_div(std::max(rows, cols), kBlockK), kPairs, dtype == A2_F32 ? kLeastBlocks : 4 * kLeastBlocks);
    if (l.gram_parts > 1) l.gram_sums = w.take<float>(l.gram_parts * mats * l.gram.stride);
    if (out) *out = l;
    return w.used;
}

template <class T>
cudaError_t typed(const OrthogonalizeArgs& a, Layout l, cudaStream_t s) {
    constexpr bool kWords = sizeof(T) == 4;
    auto flush = [](int blocks) { return kWords ? blocks : 0; };
    const bool tall = a.rows > a.cols;
    const int64_t m = std::min(a.rows, a.cols), n = std::max(a.rows, a.cols);
    const dim3 grid((unsigned)l.parts, (unsigned)a.n_mats);
    constexpr int kVec = 16 / sizeof(T);
    const bool aligned = reinterpret_cast<uintptr_t>(a.in) % 16 == 0 && a.in_pitch % kVec == 0 && (a.n_mats == 1 || a.in_stride % kVec == 0);
    A2_CUDA_TRY(launch_chained(aligned ? k_norm<T, kVec> : k_norm<T, 1>, grid, kNormThreads, 0, s, static_cast<const T*>(a.in), a.in_stride, a.in_pitch, a.rows,
                           a.cols, l.partial));
    A2_CUDA_TRY(launch_chained(aligned ? k_first_words<T, kVec> : k_first_words<T, 1>, grid, kNormThreads, 0, s, static_cast<const T*>(a.in), a.in_stride,
                           a.in_pitch, a.rows, a.cols, l.partial, (int)l.parts, a.eps, l.x.hi, l.x.lo, l.x.ld, l.scales));
    if (a.steps == 0)
        return launch_chained(k_normalized<T>, grid, kNormThreads, 0, s, l.x.hi, l.x.lo, l.x.ld, a.rows, a.cols, l.scales, a.scale, static_cast<T*>(a.out),
                              a.out_stride, a.out_pitch);
    // X goes back and forth between two buffers: two of each product that reads it
    auto operand = [](const Words& w, int64_t rows, int64_t k, bool mn) { return Operand{w.hi, w.lo, rows, k, w.ld, w.stride, mn}; };
    Operand gram = operand(l.gram, m, m, false), b = operand(l.poly, m, m, false);
    gram.symmetric = b.symmetric = true;
    const Words x[2] = {l.x, l.y};
    GemmArgs make_gram[2], make_poly, update[2];
    A2_CUDA_TRY(make_gemm(gram, gram, a.n_mats, false, true, flush(kFlushPoly), 1, &make_poly));
    for (int k = 0; k < 2 && k < a.steps; ++k) {
        const Operand side = operand(x[k], m, n, tall);
        A2_CUDA_TRY(make_gemm(side, side, a.n_mats, false, true, flush(kFlushGram), l.gram_parts, &make_gram[k]));
        A2_CUDA_TRY(tall ? make_gemm(operand(x[k], a.rows, m, false), b, a.n_mats, false, false, flush(update_flush(m)), 1, &update[k])
                         : make_gemm(b, operand(x[k], n, m, true), a.n_mats, false, false, flush(update_flush(m)), 1, &update[k]));
    }
    const int64_t part_stride = a.n_mats * l.gram.stride;
    for (int step = 0; step < a.steps; ++step) {
        const Poly poly{a.ca, a.cb, a.cc, step};
        const bool last = step + 1 == a.steps;
        A2_CUDA_TRY((launch_gemm<SymmetricEpi<false>, kWords>(
            make_gram[step % 2], {l.gram, l.gram, m, l.scales, poly, l.gram_parts > 1 ? l.gram_sums : nullptr, part_stride}, s)));
        if (l.gram_parts > 1)  // only with fewer tiles than pairs, so m and the matrices fit a grid
            A2_CUDA_TRY(launch_chained(k_join_gram, dim3((unsigned)ceil_div(m, 512), (unsigned)m, (unsigned)a.n_mats), 256, 0, s, l.gram_sums, l.gram_parts,
                                   part_stride, l.gram, m, l.scales, poly));
        A2_CUDA_TRY((launch_gemm<SymmetricEpi<true>, kWords>(make_poly, {l.gram, l.poly, m, l.scales, poly, nullptr, 0}, s)));
        A2_CUDA_TRY((launch_gemm<UpdateEpi<T>, kWords>(
            update[step % 2],
            {x[1 - step % 2], a.rows, a.cols, l.scales, poly, last ? static_cast<T*>(a.out) : nullptr, a.out_stride, a.out_pitch, a.scale}, s)));
    }
    return cudaSuccess;
}

// ---- narrow matrices: all steps in one cluster -------------------------------------------------------
// m <= 128: a cluster of up to 16 CTAs holds a matrix, 256 columns of X a CTA, and runs all steps in one launch. X, A and B stay in
// shared memory as the two-word operands of the tensor core (with either storage type: the products cost little here), the sums in
// tensor memory. X is kept [m, 256] in 64-column blocks of 128-byte swizzled rows, which the tensor core reads K-major for X X^T and
// MN-major for B X. Every CTA makes its columns' part of A = X X^T; the parts are added up in CTA order, a share of the rows by each
// CTA, and every CTA takes the whole of A from the shares and forms B by itself. Bound by that chain: three products, their
// epilogues and two exchanges a step. Five steps, fp32, us, this form / the products above: 16 x 64 x 64 30 / 149; 512 x 64 x 64 116 / 600; 3 x 21 x
// 2,579 54 / 192; 14 x 3,802 x 42 164 / 295; 8 x 282 x 97 97 / 209; 64 x 100 x 1,000 213 / 417; 16 x 128 x 4,096 382 / 484; 64 x 128 x 4,096 1,326 /
// 1,240: only many matrices of the widest kind, which fill the GPU either way, would be a little faster above. Its errors: 16 x 64 x 64 1.4e-6,
// where a plain fp32 form has 1.1e-6; of 100 matrices the median of that ratio is 1.3, the largest 2.0. With a fourth pass (lo * lo) and sums of four
// steps at a time the median is 1.05 and the largest 1.8, but the first size then takes 34 us and the last 1,465.
constexpr int kNarrowM = 128, kNarrowN = 256, kNarrowCtas = 16;
constexpr int kNarrowThreads = 256;
constexpr int kBlockBytes = kNarrowM * 128;  // 128 rows of 64 fp16 columns
constexpr int kWordBytes = (kNarrowM / 64) * kBlockBytes;         // a word of A or B
constexpr int kSquareBytes = kNarrowM * (kNarrowM + 4) * 4 + 64;  // two of them, or a part of A as floats (and what a last load reads past it)
static_assert(2 * kWordBytes <= kSquareBytes, "A's words and its part share their place");
constexpr int kNarrowSmem = 2 * (kNarrowN / 64) * kBlockBytes + kSquareBytes + 1024;
constexpr int kNarrowLowUp = 1;  // all passes share one accumulator: tensor memory has no room for another, so low words keep their size
static_assert(kNarrowSmem <= 227 * 1024 - 512, "shared memory of one CTA, with room for the static part");

// Byte offset of columns col .. col + 7 of a row.
__device__ __forceinline__ uint32_t swizzled(int row, int col) {
    return (uint32_t)(col / 64) * kBlockBytes + row * 128 + ((((col % 64) / 8) ^ (row % 8)) * 16);
}

__device__ __forceinline__ float4 load_remote(uint32_t addr, int cta) {
    uint32_t remote;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(cta));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote) : "memory");
    return v;
}
__device__ __forceinline__ double load_remote_double(uint32_t addr, int cta) {
    uint32_t remote;
    double v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(cta));
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(remote) : "memory");
    return v;
}

struct NarrowArgs {
    int64_t in_stride, in_pitch, out_stride, out_pitch;
    int rows, cols, steps;
    int ctas, chunk;  // of a matrix; columns of X a CTA, a multiple of 64
    bool tall;
    Poly poly;
    double eps;
    float scale;
    int* gave_up;
};

// D = A B^T or A B over K = 16 * k_steps in the three passes of two-word operands; one thread.
__device__ __forceinline__ void narrow_product(uint32_t d, const uint32_t (&a)[2], const uint32_t (&b)[2], bool b_mn, int k_steps, uint32_t idesc) {
    for (int pass = 0; pass < 3; ++pass) {
        const uint32_t pa = a[pass == 0], pb = b[pass == 1];  // lo hi, hi lo, hi hi
        for (int k = 0; k < k_steps; ++k) {
            const uint32_t along = (uint32_t)(k / 4) * kBlockBytes + (k % 4) * 32;  // K-major: 32 bytes, then the next block
            const uint64_t da = operand_desc(pa + along, false);
            const uint64_t db = b_mn ? operand_desc(pb + k * 2048, true, kBlockBytes) : operand_desc(pb + along, false);
            ptx::mma_one(d, da, db, idesc, pass > 0 || k > 0);
        }
    }
}

template <class T>
__global__ void __launch_bounds__(kNarrowThreads, 1) k_narrow(const T* in, T* out, const NarrowArgs g) {
    extern __shared__ char raw[];
    __shared__ double part[kNarrowThreads / 32];
    __shared__ double squares;
    __shared__ uint64_t bar_word;
    __shared__ uint32_t tmem_slot;
    __shared__ MatScale scale;
    char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rank = g.ctas > 1 ? (int)ptx::cta_rank() : 0, mat = blockIdx.x / g.ctas;
    const int m = g.tall ? g.cols : g.rows;
    const int first = rank * g.chunk, n = min(g.chunk, (g.tall ? g.rows : g.cols) - first);  // this CTA's columns of X
    const int m16 = (m + 15) / 16 * 16, n16 = (n + 15) / 16 * 16, blocks = (n + 63) / 64;
    char* xw[2] = {smem, smem + (kNarrowN / 64) * kBlockBytes};
    char* square = smem + 2 * (kNarrowN / 64) * kBlockBytes;
    char* aw[2] = {square, square + kWordBytes};
    // [m16][m16 + 4] in A's place while it is made: rows 16 bytes apart modulo 128, so that eight lanes' rows are free of conflicts
    float* gram_part = reinterpret_cast<float*>(square);
    const int pitch = m16 + 4, share = (m + g.ctas - 1) / g.ctas;
    const uint32_t xs[2] = {ptx::smem_addr(xw[0]), ptx::smem_addr(xw[1])}, as[2] = {ptx::smem_addr(aw[0]), ptx::smem_addr(aw[1])};
    const uint32_t bar = ptx::smem_addr(&bar_word);
    auto sync_matrix = [&] {  // all CTAs of the matrix
        if (g.ctas > 1) ptx::cluster_sync();
        else __syncthreads();
    };

    if (threadIdx.x == 0) {
        ptx::bar_init(bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(ptx::smem_addr(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        ptx::fence_before();
    }
    ptx::chained();
    // element (i, j) of this CTA's columns of X
    const T* from = in + mat * g.in_stride + (g.tall ? first * g.in_pitch : first);
    T* to = out + mat * g.out_stride + (g.tall ? first * g.out_pitch : first);
    const int my_rows = g.tall ? n : g.rows, my_cols = g.tall ? g.cols : n;
    // the norm
    double sum = 0.0;
    for (int i = warp; i < my_rows; i += kNarrowThreads / 32)
        for (int j = lane; j < my_cols; j += 32) {
            const double v = widen(from[i * g.in_pitch + j]);
            sum += v * v;
        }
    for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double all = 0.0;
        for (int w = 0; w < kNarrowThreads / 32; ++w) all += part[w];
        squares = all;
    }
    sync_matrix();
    if (threadIdx.x == 0) {
        double all = 0.0;
        for (int c = 0; c < g.ctas; ++c) all += g.ctas > 1 ? load_remote_double(ptx::smem_addr(&squares), c) : squares;
        scale = mat_scale(all, g.eps);
    }
    __syncthreads();
    ptx::fence_after();
    const uint32_t tmem = tmem_slot;
    // first words, zeros around the matrix: rows to a multiple of 16, columns to a multiple of 64. Eight columns a thread; the tall
    // matrix is read along its rows, which are X's columns
    const PowerOfTwo up(scale.e);
    for (int k = threadIdx.x; k < m16 * blocks * 8; k += kNarrowThreads) {
        const int i = g.tall ? k % m16 : k / (blocks * 8), j = (g.tall ? k / m16 : k % (blocks * 8)) * 8;
        Pack<__half, 8> hi, lo;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const bool inside = i < m && j + q < n;
            const float v = inside ? widen(g.tall ? from[(j + q) * g.in_pitch + i] : from[i * g.in_pitch + j + q]) : 0.0f;
            split_words<kNarrowLowUp>(up(v), hi.v[q], lo.v[q]);
        }
        const uint32_t at = swizzled(i, j);
        *reinterpret_cast<Pack<__half, 8>*>(xw[0] + at) = hi;
        *reinterpret_cast<Pack<__half, 8>*>(xw[1] + at) = lo;
    }

    const int quad = warp % 4, half = warp / 4;
    const int row = quad * 32 + lane;
    const bool mine = quad * 32 < m;  // warps of padding rows have nothing to write
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t to_square = instruction_desc(false, false, false, 128, m16), to_wide = instruction_desc(false, false, true, 128, n16);
    uint32_t phase = 0;
    bool ok = true;  // once a wait has run out no further product is made, but every CTA still comes to every barrier
    // one product: operands written by everybody, MMAs by one thread, everybody waits
    auto product = [&](uint32_t d, const uint32_t (&a)[2], const uint32_t (&b)[2], bool b_mn, int k_steps, uint32_t idesc) {
        ptx::fence_before();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0 && ok) {
            ptx::fence_after();
            narrow_product(d, a, b, b_mn, k_steps, idesc);
            ptx::commit_one(bar);
        }
        __syncwarp();
        if (ok) ok = ptx::bar_wait(bar, phase & 1, g.gave_up);
        ++phase;
        ptx::fence_after();
        ok = __syncthreads_or(!ok) == 0;
    };
    auto write8 = [&](char* const (&to)[2], int col, const float* v) {
        Pack<__half, 8> hi, lo;
#pragma unroll
        for (int q = 0; q < 8; q += 2) split_pair<kNarrowLowUp>(v[q], v[q + 1], hi.v[q], hi.v[q + 1], lo.v[q], lo.v[q + 1]);
        const uint32_t at = swizzled(row, col);
        *reinterpret_cast<Pack<__half, 8>*>(to[0] + at) = hi;
        *reinterpret_cast<Pack<__half, 8>*>(to[1] + at) = lo;
    };
    Poly poly = g.poly;
    for (poly.step = 0; poly.step < g.steps; ++poly.step) {
        const Units x(scale, poly);
        const bool last = poly.step + 1 == g.steps;
        const float gram = x.gram();
        product(tmem, xs, xs, false, n16 / 16, to_square);
        float total[2][32];  // of A, this thread's columns half * 32 .. and half * 32 + 64 ..
        if (g.ctas > 1) {
            for (int col = half * 32; mine && col < m16; col += 64) {
                float v[32];
                ptx::tmem_load32(v, lanes + col);
                ptx::tmem_load_wait();
#pragma unroll
                for (int k = 0; k < 32; k += 4)
                    if (row < m16 && col + k < m16) *reinterpret_cast<float4*>(gram_part + row * pitch + col + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
            }
            sync_matrix();
            // this CTA's rows, in place: nobody else reads its part of them
            for (int k = threadIdx.x; k < share * (m16 / 4); k += kNarrowThreads) {
                const int r = rank * share + k / (m16 / 4), c = k % (m16 / 4) * 4;
                if (r >= m) break;
                const uint32_t at = ptx::smem_addr(gram_part + r * pitch + c);
                float4 all = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
                for (int q = 0; q < g.ctas; ++q) {
                    const float4 v = load_remote(at, q);
                    all.x += v.x;
                    all.y += v.y;
                    all.z += v.z;
                    all.w += v.w;
                }
                *reinterpret_cast<float4*>(gram_part + r * pitch + c) = all;
            }
            sync_matrix();
            const int r = min(row, m - 1);
            const uint32_t at = ptx::smem_addr(gram_part + r * pitch);
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (mine && half * 32 + c * 64 < m16)
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        const float4 v = load_remote(at + (half * 32 + c * 64 + k) * 4, r / share);
                        total[c][k] = row < m ? v.x : 0.0f;
                        total[c][k + 1] = row < m ? v.y : 0.0f;
                        total[c][k + 2] = row < m ? v.z : 0.0f;
                        total[c][k + 3] = row < m ? v.w : 0.0f;
                    }
            sync_matrix();  // A's words go where its parts lie
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int col = half * 32 + c * 64;
            if (!mine || col >= m16) continue;
            float v[32];
            if (g.ctas > 1) {
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] = total[c][k];
            } else {
                ptx::tmem_load32(v, lanes + col);
                ptx::tmem_load_wait();
            }
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] *= gram;
            uint64_t keep[16];  // A itself, for B
#pragma unroll
            for (int k = 0; k < 16; ++k) asm volatile("mov.b64 %0, {%1, %2};" : "=l"(keep[k]) : "f"(v[2 * k]), "f"(v[2 * k + 1]));
            ptx::tmem_store_pairs(lanes + col, keep);
#pragma unroll
            for (int k = 0; k < 32; k += 8)
                if (col + k < m16) write8(aw, col + k, v + k);
        }
        ptx::tmem_store_wait();
        product(tmem + 128, as, as, false, m16 / 16, to_square);
        for (int col = half * 32; mine && col < m16; col += 64) {
            float v[32], w[32];
            ptx::tmem_load32(v, lanes + col);
            ptx::tmem_load32(w, lanes + 128 + col);
            ptx::tmem_load_wait();
#pragma unroll
            for (int k = 0; k < 32; ++k)
                v[k] = poly.b * v[k] + poly.c / kScale * w[k] + (row == col + k && row < m ? poly.a * kScale : 0.0f);
#pragma unroll
            for (int k = 0; k < 32; k += 8)
                if (col + k < m16) write8(aw, col + k, v + k);
        }
        product(tmem + 256, as, xs, true, m16 / 16, to_wide);
        const Scaled factor(last ? g.scale : 1.0f, x.u, x.k - 14 - (last ? 0 : x.next));
        for (int col = half * 32; mine && col < n16; col += 64) {
            float v[32];
            ptx::tmem_load32(v, lanes + 256 + col);
            ptx::tmem_load_wait();
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] = factor(v[k]);
            if (!last) {  // rows of padding keep their zeros: what they hold in tensor memory is not a product of anything
#pragma unroll
                for (int k = 0; k < 32; k += 8)
                    if (row < m && col + k < n16) write8(xw, col + k, v + k);
                continue;
            }
            if (g.tall) {  // lanes lie along the caller's columns
                if (row < m)
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (col + k < n) to[(col + k) * g.out_pitch + row] = narrow<T>(v[k]);
            } else {  // through shared memory (B is done with), so that a row's columns are written side by side
                turn_columns(reinterpret_cast<float*>(aw[0]) + warp * 32 * kStagePitch, v, lane);
                if (col + lane < n)
#pragma unroll
                    for (int r = 0; r < 32; ++r)
                        if (quad * 32 + r < m) to[(quad * 32 + r) * g.out_pitch + col + lane] = narrow<T>(v[r]);
            }
        }
    }
    if (g.steps == 0) {
        const Scaled by(g.scale, scale.u, scale.k);
        for (int i = warp; i < my_rows; i += kNarrowThreads / 32)
            for (int j = lane; j < my_cols; j += 32)
                to[i * g.out_pitch + j] = narrow<T>(by(up(widen(from[i * g.in_pitch + j]))));
    }
    ptx::fence_before();
    sync_matrix();  // no CTA leaves while another may read its shared memory
    if (warp == 0) {
        ptx::fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

template <class T>
cudaError_t narrow_typed(const OrthogonalizeArgs& a, cudaStream_t s) {
    const int64_t n = std::max(a.rows, a.cols);
    const int ctas = (int)ceil_div(n, kNarrowN);
    NarrowArgs g{a.in_stride, a.in_pitch, a.out_stride, a.out_pitch, (int)a.rows, (int)a.cols, a.steps, ctas, (int)round_up(ceil_div(n, ctas), 64),
                 a.rows > a.cols, {a.ca, a.cb, a.cc, 0}, a.eps, a.scale, nullptr};
    g.ctas = (int)ceil_div(n, g.chunk);
    static std::atomic<uint64_t> allowed, clusters;
    A2_CUDA_TRY(gave_up_flag(&g.gave_up));
    A2_CUDA_TRY(allow_shared_memory(reinterpret_cast<const void*>(k_narrow<T>), kNarrowSmem, allowed));
    A2_CUDA_TRY(allow_large_clusters(reinterpret_cast<const void*>(k_narrow<T>), clusters));
    return launch_clusters(k_narrow<T>, dim3((unsigned)(a.n_mats * g.ctas)), kNarrowThreads, kNarrowSmem, (unsigned)g.ctas, s, static_cast<const T*>(a.in),
                           static_cast<T*>(a.out), g);
}

bool is_narrow(int64_t rows, int64_t cols) { return std::min(rows, cols) <= kNarrowM && std::max(rows, cols) <= kNarrowN * kNarrowCtas; }

}  // namespace

bool orthogonalize_range(double a, double b, double c, int steps) {
    // singular values start in [0, 1]; x p(x^2), p(s) = a + b s + c s^2, takes them step by step to at most its extremes: at the end
    // of the interval and where a + 3 b s + 5 c s^2 = 0. p's own extremes: at both ends and at s = -b / 2c.
    auto p = [&](double s) { return std::abs(a + b * s + c * s * s); };
    double reach = 1.0;
    for (int step = 0; step < steps; ++step) {
        const double end = reach * reach, turn = c != 0.0 ? -b / (2 * c) : -1.0;
        if (!(p(0.0) <= kMostPoly && p(end) <= kMostPoly && !(turn > 0.0 && turn < end && p(turn) > kMostPoly))) return false;
        double roots[2] = {b != 0.0 ? -a / (3 * b) : -1.0, -1.0};
        const double disc = 9 * b * b - 20 * a * c;
        if (c != 0.0) {
            roots[0] = disc >= 0.0 ? (-3 * b + std::sqrt(disc)) / (10 * c) : -1.0;
            roots[1] = disc >= 0.0 ? (-3 * b - std::sqrt(disc)) / (10 * c) : -1.0;
        }
        double next = std::max(reach, reach * p(end));
        for (double s : roots)
            if (s > 0.0 && s < end) next = std::max(next, std::sqrt(s) * p(s));
        if (!(next <= kMostSingular)) return false;
        if (next == reach) break;
        reach = next;
    }
    return true;
}

int64_t orthogonalize_workspace(int64_t n_mats, int64_t rows, int64_t cols, int32_t dtype) {
    return is_narrow(rows, cols) ? 0 : layout(n_mats, rows, cols, dtype, nullptr, nullptr);
}

cudaError_t run_orthogonalize(const OrthogonalizeArgs& a, void* workspace, cudaStream_t s) {
    if (is_narrow(a.rows, a.cols)) return a.dtype == A2_BF16 ? narrow_typed<__nv_bfloat16>(a, s) : narrow_typed<float>(a, s);
    Layout l;
    layout(a.n_mats, a.rows, a.cols, a.dtype, workspace, &l);
    return a.dtype == A2_BF16 ? typed<__nv_bfloat16>(a, l, s) : typed<float>(a, l, s);
}

}  // namespace a2
