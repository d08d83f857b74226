// Norm of a gradient that is spread over many tensors, and its clipping: norm = sqrt(sum of squares of all elements of all tensors), out = in * min(1, max_norm / norm); for
// each worker's part of the tensors by itself.
#include <algorithm>
#include <type_traits>

#include "lm_ops.h"

namespace a2 {

namespace {

// ---------------------------------------------------------------------------------------------
// Bound by memory: read once for the norm, read again and written once for the clipping. A worker's elements are cut into chunks of kChunkBytes, tensor after tensor;
// every CTA has a run of consecutive chunks, over all workers, and leaves a sum for each worker it meets: CTA b and worker w at place b + w, which no other pair
// has, since runs follow one another. Sums are joined in order.
// 134 M elements, two thirds bf16 (340 MB), to other tensors: 165 us, 58 for the norm (5.9 TB/s) and 98 to 103 for the scaling (6.5 TB/s, a copy's rate); 135 M fp32
// 81 and 170. In place and not clipped 87. 16 workers of 4.5 MB: 35 us. The first reading leaves what it reads in the L2 cache where a second one follows (10 M fp32 clipped
// 17.8 us, 20.3 without), and not where the norms are all (135 M fp32: 80.6 us, 82.6 with it). The second reading goes in the order of the first: against it, with
// what was read last kept in the cache by hints, took the same (60 M fp32 113.3 us both ways) or more (16 workers of 34 MB 264 us, 258 in order).
// ---------------------------------------------------------------------------------------------
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kChunkBytes = 16384;   // four loads of 16 bytes in flight for each of 256 threads
constexpr int kCtas = 6;             // a multiprocessor
constexpr int64_t kMany = 2;         // chunks of a run from which on the scaling is a launch of its own shape, after one that joins the norms
constexpr int kFew = 48;             // tensors that are described in a kernel's parameters; more in the workspace
constexpr int kStored = 240;         // tensors that a launch brings there
constexpr int64_t kSmallChunks = 4;  // chunks of a worker that one CTA takes alone

struct Tensor {
    const void* in;
    void* out;
    int64_t worker_stride, out_worker_stride, rows, cols, pitch, out_pitch;
    int64_t first_chunk;  // of the worker's
    int32_t bf16;
    int32_t wide;  // rows may be read 16 bytes at a time: one row (from the boundary before it), or all rows on boundaries
};

struct Few {
    Tensor tensor[kFew];
};
struct Stored {
    Tensor tensor[kStored];
};

struct alignas(16) Factor {
    float by, then;      // two factors: one alone may lie below the range of floats where the result does not
    int32_t zero, nothing;  // nothing: by one
};

struct ClipKernelArgs {
    int64_t n_tensors, workers, worker_chunks, chunks;
    int64_t run, longer_runs;  // chunks of a CTA's run, and how many runs have one more
    double* sums;
    Factor* factors;  // of the workers, where the scaling is a launch of its own shape
    float* norms;
    double max_norm;
    bool zero_nonfinite, clip;
};

__global__ void __launch_bounds__(kStored) k_store(const __grid_constant__ Stored from, Tensor* to, int n) {
    ptx::chained();
    if ((int)threadIdx.x < n) to[threadIdx.x] = from.tensor[threadIdx.x];
}

// The first runs have a chunk more than the others.
__device__ __forceinline__ int64_t run_start(const ClipKernelArgs& a, int64_t cta) { return cta * a.run + min(cta, a.longer_runs); }
__device__ __forceinline__ int64_t run_of(const ClipKernelArgs& a, int64_t chunk) {
    const int64_t longer = a.longer_runs * (a.run + 1);
    return chunk < longer ? chunk / (a.run + 1) : a.longer_runs + (chunk - longer) / a.run;
}

template <int THREADS>
__device__ __forceinline__ double cta_sum(double v, double* shared) {
#pragma unroll
    for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) v += shared[w];
    return v;
}

// The sum of the squares of vectors. In fp32 where that neither overflows nor loses what lies below its range, as it hardly ever does; else in 64 bits.
template <class T, int COUNT>
__device__ __forceinline__ double squares(const Words (&p)[COUNT]) {
    constexpr int V = kVec<T>;
    float q[COUNT];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        float2 v[V / 2], sum = two(0.0f);
        unpack<T>(p[i], v);
#pragma unroll
        for (int k = 0; k < V / 2; ++k) sum = fma2(v[k], v[k], sum);
        q[i] = sum.x + sum.y;
    }
#pragma unroll
    for (int n = COUNT / 2; n > 0; n /= 2)
#pragma unroll
        for (int i = 0; i < n; ++i) q[i] += q[i + n];
    if (q[0] > 0x1p-60f && q[0] < 0x1p120f) return q[0];
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        float v[V];
        unpack<T>(p[i], v);
#pragma unroll
        for (int k = 0; k < V; ++k) d += (double)v[k] * (double)v[k];
    }
    return d;
}

// Walks over a chunk: `vectors(in, out)` gets the addresses of COUNT vectors of the calling thread, `element(in, out)` of single elements.
constexpr int kBatch = 4;

template <class T, int THREADS, class Vectors, class Element>
__device__ __forceinline__ void over_chunk(const Tensor& t, int64_t worker, int64_t chunk, const Vectors& vectors, const Element& element) {
    constexpr int V = 16 / sizeof(T), kChunk = kChunkBytes / sizeof(T);
    const T* in = static_cast<const T*>(t.in) + worker * t.worker_stride;
    T* out = static_cast<T*>(t.out) + worker * t.out_worker_stride;
    const int64_t all = t.rows * t.cols;
    if (t.wide && t.rows == 1) {
        const int64_t start = chunk * kChunk - (int64_t)(reinterpret_cast<uintptr_t>(in) % 16 / sizeof(T));
        constexpr int kCount = kChunk / V / THREADS;
        if (start >= 0 && start + kChunk <= all) {
            vectors(std::integral_constant<int, kCount>{}, [&](int i) { return start + (int64_t)(i * THREADS + (int)threadIdx.x) * V; }, in, [&](int i) { return start + (int64_t)(i * THREADS + (int)threadIdx.x) * V; }, out);
            return;
        }
        for (int i = threadIdx.x; i < kChunk / V; i += THREADS) {
            const int64_t e = start + i * V;
            if (e >= all) break;
            if (e >= 0 && e + V <= all) {
                vectors(std::integral_constant<int, 1>{}, [&](int) { return e; }, in, [&](int) { return e; }, out);
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (e + k >= 0 && e + k < all) element(in + e + k, out + e + k);
            }
        }
        return;
    }
    // rows: the chunk's first element, from which the others are found in 32 bits
    const int64_t first = chunk * kChunk;
    const int64_t row0 = first / t.cols, col0 = first % t.cols;
    const int count = (int)(all - first < kChunk ? all - first : kChunk);
    auto at = [&](int i, int64_t pitch) {
        int64_t row = row0, col = col0 + i;
        if (t.cols >= kChunk) {
            if (col >= t.cols) ++row, col -= t.cols;
        } else {
            const unsigned r = (unsigned)col / (unsigned)t.cols;
            row += r;
            col -= (int64_t)r * t.cols;
        }
        return row * pitch + col;
    };
    if (t.wide) {
        int i = threadIdx.x * V;
        for (; i + (kBatch - 1) * THREADS * V < count; i += kBatch * THREADS * V)
            vectors(std::integral_constant<int, kBatch>{}, [&](int k) { return at(i + k * THREADS * V, t.pitch); }, in, [&](int k) { return at(i + k * THREADS * V, t.out_pitch); }, out);
        for (; i < count; i += THREADS * V)
            vectors(std::integral_constant<int, 1>{}, [&](int) { return at(i, t.pitch); }, in, [&](int) { return at(i, t.out_pitch); }, out);
    } else {
#pragma unroll 4
        for (int i = threadIdx.x; i < count; i += THREADS) element(in + at(i, t.pitch), out + at(i, t.out_pitch));
    }
}

// Words that nobody reads again soon leave the L2 cache first.
__device__ __forceinline__ Words load_once(const void* p) {
    const uint4 v = __ldcs(static_cast<const uint4*>(p));
    return {v.x, v.y, v.z, v.w};
}
__device__ __forceinline__ void store_once(void* p, const Words& v) { __stcs(static_cast<uint4*>(p), make_uint4(v.w[0], v.w[1], v.w[2], v.w[3])); }

template <class T, int THREADS>
__device__ __forceinline__ double chunk_squares(const Tensor& t, int64_t worker, int64_t chunk, bool keep) {
    double sum = 0.0;
    over_chunk<T, THREADS>(
        t, worker, chunk,
        [&](auto count, auto from, const T* in, auto, T*) {
            constexpr int kCount = decltype(count)::value;
            Words p[kCount];
#pragma unroll
            for (int i = 0; i < kCount; ++i) p[i] = keep ? *reinterpret_cast<const Words*>(in + from(i)) : load_once(in + from(i));
            sum += squares<T, kCount>(p);
        },
        [&](const T* in, T*) {
            const double v = widen(*in);
            sum += v * v;
        });
    return sum;
}

__device__ __forceinline__ Factor factor_of(const ClipKernelArgs& a, double norm) {
    if (!isfinite(norm)) return {1.0f, 1.0f, a.zero_nonfinite, !a.zero_nonfinite};
    if (norm <= a.max_norm) return {1.0f, 1.0f, false, true};
    const double factor = a.max_norm / norm;
    if (factor < 0x1p-100) return {(float)(factor * 0x1p100), 0x1p-100f, false, false};
    return {(float)factor, 1.0f, false, false};
}

template <class T, int THREADS, class F>
__device__ __forceinline__ void scale_chunk(const Tensor& t, int64_t worker, int64_t chunk, const F& factor) {
    constexpr int V = 16 / sizeof(T);
    over_chunk<T, THREADS>(
        t, worker, chunk,
        [&](auto count, auto from, const T* in, auto to, T* out) {
            constexpr int kCount = decltype(count)::value;
            Words p[kCount];
#pragma unroll
            for (int i = 0; i < kCount; ++i) p[i] = load_once(in + from(i));
            const Factor f = factor();
#pragma unroll
            for (int i = 0; i < kCount; ++i) {
                float v[V];
                unpack<T>(p[i], v);
#pragma unroll
                for (int k = 0; k < V; ++k) v[k] = f.zero ? 0.0f : v[k] * f.by * f.then;
                store_once(out + to(i), pack<T>(v));
            }
        },
        [&](const T* in, T* out) {
            const Factor f = factor();
            *out = narrow<T>(f.zero ? 0.0f : widen(*in) * f.by * f.then);
        });
}

// `factor()` gives the factor: it is asked for after the loads that do not need it.
template <int THREADS, class F>
__device__ __forceinline__ void scale(const Tensor& t, int64_t worker, int64_t chunk, const F& factor) {
    if (t.bf16)
        scale_chunk<__nv_bfloat16, THREADS>(t, worker, chunk, factor);
    else
        scale_chunk<float, THREADS>(t, worker, chunk, factor);
}

// The tensor that a worker's chunk belongs to: the last one that begins at it or before. (Each lane with an entry of its own would read a kernel's
// parameters one lane after the other.)
__device__ __forceinline__ int tensor_of(const Tensor* table, int64_t n, int64_t chunk) {
    int low = 0, high = (int)n - 1;
    while (low < high) {
        const int mid = (low + high + 1) / 2;
        if (table[mid].first_chunk <= chunk)
            low = mid;
        else
            high = mid - 1;
    }
    return low;
}

template <bool FEW>
__global__ void __launch_bounds__(kThreads, kCtas) k_squares(const __grid_constant__ ClipKernelArgs a, const __grid_constant__ Few few, const Tensor* stored) {
    __shared__ double shared[kWarps];
    ptx::chained();
    const Tensor* table = FEW ? few.tensor : stored;
    const int64_t cta = blockIdx.x, end = run_start(a, cta + 1);
    int64_t chunk = run_start(a, cta);
    while (chunk < end) {
        const int64_t worker = chunk / a.worker_chunks, worker_end = min(end, (worker + 1) * a.worker_chunks);
        int64_t c = chunk - worker * a.worker_chunks;
        int t = tensor_of(table, a.n_tensors, c);
        double sum = 0.0;
        for (; chunk < worker_end; ++chunk, ++c) {
            while (t + 1 < a.n_tensors && table[t + 1].first_chunk <= c) ++t;
            const Tensor& tensor = table[t];
            sum += tensor.bf16 ? chunk_squares<__nv_bfloat16, kThreads>(tensor, worker, c - tensor.first_chunk, a.clip)
                               : chunk_squares<float, kThreads>(tensor, worker, c - tensor.first_chunk, a.clip);
        }
        sum = cta_sum<kThreads>(sum, shared);
        if (threadIdx.x == 0) a.sums[cta + worker] = sum;
    }
}

__device__ __forceinline__ double norm_of(const ClipKernelArgs& a, int64_t worker, double* shared) {
    const int64_t from = run_of(a, worker * a.worker_chunks), to = run_of(a, (worker + 1) * a.worker_chunks - 1);
    double sum = 0.0;
    for (int64_t b = from + threadIdx.x; b <= to; b += kThreads) sum += a.sums[b + worker];
    return sqrt(cta_sum<kThreads>(sum, shared));
}

template <bool FEW>
__global__ void __launch_bounds__(kThreads, kCtas) k_scale(const __grid_constant__ ClipKernelArgs a, const __grid_constant__ Few few, const Tensor* stored) {
    __shared__ double shared[kWarps];
    ptx::chained();
    const Tensor* table = FEW ? few.tensor : stored;
    const int64_t cta = blockIdx.x, end = run_start(a, cta + 1);
    int64_t chunk = run_start(a, cta);
    while (chunk < end) {
        const int64_t worker = chunk / a.worker_chunks, worker_end = min(end, (worker + 1) * a.worker_chunks);
        const double norm = norm_of(a, worker, shared);
        if (chunk == worker * a.worker_chunks && threadIdx.x == 0) a.norms[worker] = (float)norm;
        const Factor f = factor_of(a, norm);
        int64_t c = chunk - worker * a.worker_chunks;
        int t = tensor_of(table, a.n_tensors, c);
        for (; chunk < worker_end; ++chunk, ++c) {
            while (t + 1 < a.n_tensors && table[t + 1].first_chunk <= c) ++t;
            if (!f.nothing || table[t].in != table[t].out) scale<kThreads>(table[t], worker, c - table[t].first_chunk, [&] { return f; });
        }
    }
}

// Norms alone, of a CTA each; with the factors where a kernel that scales follows.
__global__ void __launch_bounds__(kThreads) k_norms(const __grid_constant__ ClipKernelArgs a) {
    __shared__ double shared[kWarps];
    ptx::chained();
    const double norm = a.chunks ? norm_of(a, blockIdx.x, shared) : 0.0;
    if (threadIdx.x != 0) return;
    a.norms[blockIdx.x] = (float)norm;
    if (a.clip) a.factors[blockIdx.x] = factor_of(a, norm);
}

// A chunk a CTA: while one waits for its loads, others write (134 M bf16: 128 us with the norm, 133 with a few chunks each). In place, where mostly nothing has to be done, a
// few chunks each, which are sooner over then.
__device__ __forceinline__ void scale_one(const ClipKernelArgs& a, const Tensor* table, int64_t chunk) {
    const int64_t worker = a.workers == 1 ? 0 : chunk / a.worker_chunks, c = chunk - worker * a.worker_chunks;
    const uint4 factor = *reinterpret_cast<const uint4*>(a.factors + worker);
    const Tensor& t = table[tensor_of(table, a.n_tensors, c)];
    if (t.in == t.out && reinterpret_cast<const Factor*>(&factor)->nothing) return;
    scale<kThreads>(t, worker, c - t.first_chunk, [&] { return *reinterpret_cast<const Factor*>(&factor); });
}

template <bool FEW>
__global__ void __launch_bounds__(kThreads, 5) k_scale_chunks(const __grid_constant__ ClipKernelArgs a, const __grid_constant__ Few few, const Tensor* stored) {
    ptx::chained();
    scale_one(a, FEW ? few.tensor : stored, blockIdx.x);
}

template <bool FEW>
__global__ void __launch_bounds__(kThreads) k_scale_in_place(const __grid_constant__ ClipKernelArgs a, const __grid_constant__ Few few, const Tensor* stored) {
    ptx::chained();
    if (a.workers == 1 && a.factors[0].nothing) return;
    for (int64_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) scale_one(a, FEW ? few.tensor : stored, chunk);
}

// Few elements a worker: both steps in one launch, a CTA a worker.
constexpr int kSmallThreads = 1024;

template <bool FEW>
__global__ void __launch_bounds__(kSmallThreads) k_small(const __grid_constant__ ClipKernelArgs a, const __grid_constant__ Few few, const Tensor* stored) {
    __shared__ double shared[kSmallThreads / 32];
    ptx::chained();
    const Tensor* table = FEW ? few.tensor : stored;
    const int64_t worker = blockIdx.x;
    double sum = 0.0;
    for (int64_t c = 0, t = 0; c < a.worker_chunks; ++c) {
        while (t + 1 < a.n_tensors && table[t + 1].first_chunk <= c) ++t;
        const Tensor& tensor = table[t];
        sum += tensor.bf16 ? chunk_squares<__nv_bfloat16, kSmallThreads>(tensor, worker, c - tensor.first_chunk, true)
                           : chunk_squares<float, kSmallThreads>(tensor, worker, c - tensor.first_chunk, true);
    }
    const double norm = sqrt(cta_sum<kSmallThreads>(sum, shared));
    if (threadIdx.x == 0) a.norms[worker] = (float)norm;
    if (!a.clip) return;
    const Factor f = factor_of(a, norm);
    for (int64_t c = 0, t = 0; c < a.worker_chunks; ++c) {
        while (t + 1 < a.n_tensors && table[t + 1].first_chunk <= c) ++t;
        if (!f.nothing || table[t].in != table[t].out) scale<kSmallThreads>(table[t], worker, c - table[t].first_chunk, [&] { return f; });
    }
}

int64_t most_ctas() { return (int64_t)multiprocessors() * kCtas; }

bool on_boundaries(const void* p, int64_t pitch, int64_t size) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && pitch * size % 16 == 0; }

// How a tensor is read, and its chunks.
int64_t describe(const a2cid2_gradient_t& g, bool clip, int64_t workers, Tensor& t) {
    const int64_t size = g.storage_dtype == A2_BF16 ? 2 : 4, chunk = kChunkBytes / size;
    t = {g.in, clip ? g.out : const_cast<void*>(g.in), g.worker_stride, clip ? g.out_worker_stride : g.worker_stride, g.rows, g.cols, g.pitch,
         clip ? g.out_pitch : g.pitch, 0, g.storage_dtype == A2_BF16, 0};
    if (t.rows > 1 && t.pitch == t.cols && t.out_pitch == t.cols) t.cols *= t.rows, t.rows = 1;
    const int64_t all = t.rows * t.cols;
    if (all == 0) return 0;
    if (t.rows == 1) {
        const uintptr_t apart = reinterpret_cast<uintptr_t>(t.in) - reinterpret_cast<uintptr_t>(t.out);
        t.wide = apart % 16 == 0 && (workers == 1 || (t.worker_stride - t.out_worker_stride) * size % 16 == 0);
    } else {
        t.wide = on_boundaries(t.in, t.pitch, size) && on_boundaries(t.out, t.out_pitch, size) && t.cols * size % 16 == 0 &&
                 (workers == 1 || (t.worker_stride * size % 16 == 0 && t.out_worker_stride * size % 16 == 0));
    }
    // a row that starts behind a boundary may take a part of a chunk more
    return ceil_div(all + (t.wide && t.rows == 1 ? 16 / size - 1 : 0), chunk);
}

}  // namespace

int64_t clip_workspace(int64_t n_tensors, int64_t workers) {
    Carver c(nullptr);
    c.take<double>(most_ctas() + workers);
    c.take<Factor>(workers);
    if (n_tensors > kFew) c.take<Tensor>(n_tensors);
    return c.used;
}

cudaError_t run_clip(const ClipArgs& r, void* workspace, cudaStream_t s) {
    if (r.workers == 0) return cudaSuccess;
    Carver carver(workspace);
    ClipKernelArgs a{0, r.workers, 0, 0, 1, 0, carver.take<double>(most_ctas() + r.workers), carver.take<Factor>(r.workers), r.norms, r.max_norm, r.zero_nonfinite, r.clip};
    Few few{};
    Stored part{};
    Tensor* table = r.n_tensors > kFew ? carver.take<Tensor>(r.n_tensors) : nullptr;
    int held = 0;
    int64_t stored = 0;
    bool in_place = true;
    auto bring = [&]() -> cudaError_t {
        A2_CUDA_TRY(launch_chained(k_store, dim3(1), kStored, 0, s, part, table + stored, held));
        stored += held;
        held = 0;
        return cudaSuccess;
    };
    for (int64_t i = 0; i < r.n_tensors; ++i) {
        Tensor t;
        const int64_t chunks = describe(r.tensors[i], r.clip, r.workers, t);
        if (chunks == 0) continue;
        t.first_chunk = a.worker_chunks;
        a.worker_chunks += chunks;
        ++a.n_tensors;
        in_place = in_place && t.in == t.out;
        (table ? part.tensor : few.tensor)[held++] = t;
        if (table && held == kStored) A2_CUDA_TRY(bring());
    }
    if (table && held) A2_CUDA_TRY(bring());
    a.chunks = a.worker_chunks * a.workers;
    const unsigned workers = (unsigned)a.workers;
    if (a.chunks == 0) return launch_chained(k_norms, dim3(workers), kThreads, 0, s, a);
    if (a.worker_chunks <= kSmallChunks) return launch_chained(table ? k_small<false> : k_small<true>, dim3(workers), kSmallThreads, 0, s, a, few, table);
    const int64_t ctas = std::min(a.chunks, most_ctas());
    a.run = a.chunks / ctas, a.longer_runs = a.chunks % ctas;
    A2_CUDA_TRY(launch_chained(table ? k_squares<false> : k_squares<true>, dim3((unsigned)ctas), kThreads, 0, s, a, few, table));
    const bool many = a.run >= kMany && a.chunks < (int64_t(1) << 31);  // CTAs of a launch
    if (!r.clip || many) A2_CUDA_TRY(launch_chained(k_norms, dim3(workers), kThreads, 0, s, a));
    if (!r.clip) return cudaSuccess;
    if (many && in_place)
        return launch_chained(table ? k_scale_in_place<false> : k_scale_in_place<true>, dim3((unsigned)std::min(a.chunks, 4 * ctas)), kThreads, 0, s, a, few, table);
    if (many) return launch_chained(table ? k_scale_chunks<false> : k_scale_chunks<true>, dim3((unsigned)a.chunks), kThreads, 0, s, a, few, table);
    return launch_chained(table ? k_scale<false> : k_scale<true>, dim3((unsigned)ctas), kThreads, 0, s, a, few, table);
}

}  // namespace a2
