// Internal declarations of the language-model operators (embedding, vocabulary loss, orthogonalisation).
// The entry points in lm_api.cu validate; the functions below launch. All return a cudaError_t.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <utility>

#include "a2cid2.h"

namespace a2 {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

// Cuts a workspace into 256-byte aligned pieces. With a NULL base it only adds the sizes up.
struct Carver {
    char* base;
    int64_t used = 0;
    explicit Carver(void* p) : base(static_cast<char*>(p)) {}
    template <class T>
    T* take(int64_t n) {
        T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used += round_up(n * (int64_t)sizeof(T), 256);
        return p;
    }
};

struct EmbedArgs {
    const void* table;
    int64_t vocab, width, table_pitch;
    const int32_t* ids;
    int64_t n_ids;
    float scale;
    void* out;
    int64_t out_pitch;
    int32_t dtype;
};
cudaError_t run_embed(const EmbedArgs& a, cudaStream_t s);

struct EmbedGradArgs {
    const void* grad_out;
    int64_t grad_out_pitch;
    const int32_t* ids;
    int64_t n_ids, vocab, width;
    float scale;
    bool accumulate;
    void* grad_table;
    int64_t grad_table_pitch;
    int32_t dtype;
};
int64_t embed_grad_workspace(int64_t vocab, int64_t width, int64_t n_ids);
cudaError_t run_embed_grad(const EmbedGradArgs& a, void* workspace, cudaStream_t s);

struct VocabLossArgs {
    const void* hidden;
    int64_t hidden_pitch;
    const void* head;
    int64_t head_pitch;
    const int32_t* targets;
    int64_t n_tokens, width, vocab;
    const float* weights;
    float scale;
    float* loss;
    float* lse;
    void* grad_hidden;
    int64_t grad_hidden_pitch;
    void* grad_head;
    int64_t grad_head_pitch;
    int32_t dtype;
};
int64_t vocab_loss_workspace(int64_t n_tokens, int64_t width, int64_t vocab, bool with_grad, int32_t dtype);
cudaError_t run_vocab_loss(const VocabLossArgs& a, void* workspace, cudaStream_t s);

struct OrthogonalizeArgs {
    const void* in;
    int64_t in_stride, in_pitch;
    int64_t n_mats, rows, cols;
    int32_t steps;
    float ca, cb, cc;
    double eps;
    float scale;
    void* out;
    int64_t out_stride, out_pitch;
    int32_t dtype;
};
// Whether the steps keep singular values of [0, 1], and the polynomial there, inside what the fp16 intermediates hold.
bool orthogonalize_range(double a, double b, double c, int steps);
int64_t orthogonalize_workspace(int64_t n_mats, int64_t rows, int64_t cols, int32_t dtype);
cudaError_t run_orthogonalize(const OrthogonalizeArgs& a, void* workspace, cudaStream_t s);

int multiprocessors();  // of the current device

// Allows a kernel its dynamic shared memory, once for each device (`done`: which of them).
[[nodiscard]] cudaError_t allow_shared_memory(const void* kernel, int bytes, std::atomic<uint64_t>& done);
[[nodiscard]] cudaError_t allow_large_clusters(const void* kernel, std::atomic<uint64_t>& done);  // more than 8 CTAs

constexpr int64_t kMaxNormWidth = 32768;  // columns of a normalised row: it is held in the registers of a CTA

struct NormArgs {
    const void* x;
    int64_t x_pitch;
    const void* residual;  // or NULL
    int64_t residual_pitch;
    const void* weight;  // or NULL
    int64_t n, width;
    float eps;
    void* sum;  // or NULL
    int64_t sum_pitch;
    void* out;  // rows of the storage type; with `scales` of 8 bits
    int64_t out_pitch;
    float* scales;  // [n][blocks], or NULL
    int64_t block;  // columns of a scale, 0: a row
    int32_t dtype;
};
cudaError_t run_norm(const NormArgs& a, cudaStream_t s);

struct DequantizeArgs {
    const uint8_t* values;
    int64_t values_pitch;
    const float* scales;
    int64_t n, width, block;
    void* out;
    int64_t out_pitch;
    int32_t dtype;
};
cudaError_t run_dequantize(const DequantizeArgs& a, cudaStream_t s);

struct NormGradArgs {
    const void* grad_out;
    int64_t grad_out_pitch;
    const void* x;
    int64_t x_pitch;
    const void* weight;    // or NULL
    const void* grad_sum;  // or NULL
    int64_t grad_sum_pitch;
    int64_t n, width;
    float eps;
    void* grad_x;  // or NULL
    int64_t grad_x_pitch;
    void* grad_weight;  // or NULL
    int32_t dtype;
};
int64_t norm_grad_workspace(int64_t n, int64_t width, bool with_weight, int32_t dtype);
cudaError_t run_norm_grad(const NormGradArgs& a, void* workspace, cudaStream_t s);

constexpr int64_t kMaxExperts = 1024;  // a lane of a warp holds 32 of them
constexpr int64_t kMaxChosen = 32;     // one a lane
constexpr int64_t kMaxGroups = 32;

struct RouteArgs {
    const void* logits;
    int64_t logits_pitch, n;
    int experts, k;
    int score;          // A2_SCORE_*
    const float* bias;  // or NULL
    int groups, top_groups, group_score;
    bool renormalize;
    float scale;
    int32_t* ids;
    float* weights;
    int32_t* counts;  // or NULL
    int32_t dtype;
};
cudaError_t run_route(const RouteArgs& a, cudaStream_t s);

struct RouteGradArgs {
    const void* logits;
    int64_t logits_pitch;
    const int32_t* ids;
    const float* grad_weights;
    int64_t n;
    int experts, k;
    int score;
    bool renormalize;
    float scale;
    void* grad_logits;
    int64_t grad_logits_pitch;
    int32_t dtype;
};
cudaError_t run_route_grad(const RouteGradArgs& a, cudaStream_t s);

struct ClipArgs {
    const a2cid2_gradient_t* tensors;  // host
    int64_t n_tensors, workers;
    bool clip;  // else the norms alone
    double max_norm;
    bool zero_nonfinite;
    float* norms;
};
int64_t clip_workspace(int64_t n_tensors, int64_t workers);
cudaError_t run_clip(const ClipArgs& a, void* workspace, cudaStream_t s);

// Ends a function at the first launch that fails: what would follow reads what that launch was to write.
#define A2_CUDA_TRY(call)                            \
    do {                                             \
        const cudaError_t e__ = (call);              \
        if (e__ != cudaSuccess) return e__;          \
    } while (0)

// Whether a product gave up a wait on the current device since the last check that said so. Waits for nothing.
bool products_gave_up();
[[nodiscard]] cudaError_t check_products(cudaStream_t s, bool* gave_up);  // waits for the stream, and forgets what it reports

#ifdef __CUDACC__
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Starts a kernel that may begin before its predecessor in the stream has ended; the kernel itself calls wait_previous() before it
// touches memory.
template <class... P, class... A>
[[nodiscard]] cudaError_t launch_clusters(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, unsigned cluster, cudaStream_t s, A&&... args) {
    cudaLaunchConfig_t config{};
    config.gridDim = grid;
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = smem;
    config.stream = s;
    cudaLaunchAttribute attributes[2]{};
    attributes[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attributes[0].val.programmaticStreamSerializationAllowed = 1;
    attributes[1].id = cudaLaunchAttributeClusterDimension;
    attributes[1].val.clusterDim.x = cluster;
    attributes[1].val.clusterDim.y = attributes[1].val.clusterDim.z = 1;
    config.attrs = attributes;
    config.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&config, kernel, static_cast<P>(args)...);
}
template <class... P, class... A>
[[nodiscard]] cudaError_t launch_chained(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t s, A&&... args) {
    return launch_clusters(kernel, grid, threads, smem, 1, s, std::forward<A>(args)...);
}

namespace ptx {
// Kernels of one operator are launched so that one may start while its predecessor ends: it sets itself up, lets its own
// successor do the same, and waits until everything before it is done and visible. Such a kernel's inputs are no `const T* __restrict__`: that lets the
// compiler read them through the read-only cache and before the wait, which is right only for what nobody writes while the kernel lives, and its life begins before the
// predecessor's writes end. (Results may be __restrict__.)
__device__ __forceinline__ void release_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void chained() {
    release_next();
    wait_previous();
}
}  // namespace ptx

template <class T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
    T v[VEC];
};

// 16 bytes of a row as they lie in memory. Kept in words where paths with and without whole vectors meet: as single bf16 elements they would take
// a register and several instructions each.
struct alignas(16) Words {
    uint32_t w[4];
};
template <class T>
constexpr int kVec = 16 / sizeof(T);

__device__ __forceinline__ void unpack(const Words& p, float (&v)[4], float) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(p.w[i]);
}
__device__ __forceinline__ void unpack(const Words& p, float (&v)[8], __nv_bfloat16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(p.w[i] << 16);
        v[2 * i + 1] = __uint_as_float(p.w[i] & 0xffff0000u);
    }
}
template <class T>
__device__ __forceinline__ void unpack(const Words& p, float (&v)[kVec<T>]) {
    unpack(p, v, T());
}
__device__ __forceinline__ Words pack(const float (&v)[4], float) {
    Words p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p.w[i] = __float_as_uint(v[i]);
    return p;
}
__device__ __forceinline__ Words pack(const float (&v)[8], __nv_bfloat16) {
    Words p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 two = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        p.w[i] = *reinterpret_cast<const uint32_t*>(&two);
    }
    return p;
}
template <class T>
__device__ __forceinline__ Words pack(const float (&v)[kVec<T>]) {
    return pack(v, T());
}

// Two floats at a time: one instruction on this architecture.
__device__ __forceinline__ uint64_t bits(float2 v) { return *reinterpret_cast<const uint64_t*>(&v); }
__device__ __forceinline__ float2 floats(uint64_t b) { return *reinterpret_cast<const float2*>(&b); }
__device__ __forceinline__ float2 two(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
    return floats(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
    return floats(r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
    return floats(r);
}
template <class T>
__device__ __forceinline__ void unpack(const Words& p, float2 (&v)[kVec<T> / 2]) {
    float one[kVec<T>];
    unpack<T>(p, one);
#pragma unroll
    for (int i = 0; i < kVec<T> / 2; ++i) v[i] = make_float2(one[2 * i], one[2 * i + 1]);
}
template <class T>
__device__ __forceinline__ Words pack(const float2 (&v)[kVec<T> / 2]) {
    float one[kVec<T>];
#pragma unroll
    for (int i = 0; i < kVec<T> / 2; ++i) one[2 * i] = v[i].x, one[2 * i + 1] = v[i].y;
    return pack<T>(one);
}

// What of a vector at column c lies in a row. Vectors that begin before the row or end past it, and such as do not lie on a 16-byte boundary, are read in whole
// units of 16 bytes that hold an element of the row (memory comes in larger units than that, so what is next to the row is there) and cleared of
// what is not the row's; they are written element by element.
template <class T>
__device__ __forceinline__ Words within(Words p, int c, int width) {
#pragma unroll
    for (int k = 0; k < kVec<T>; ++k)
        if (c + k < 0 || c + k >= width) p.w[k * sizeof(T) / 4] &= sizeof(T) == 4 ? 0u : k % 2 ? 0xffffu : 0xffff0000u;
    return p;
}
// A vector at column c >= 0 of a row, wherever it lies.
template <class T>
__device__ __forceinline__ Words load_anywhere(const T* row, int c, int width) {
    const uintptr_t from = reinterpret_cast<uintptr_t>(row + c), unit = from & ~(uintptr_t)15;
    const int skip = (int)(from - unit);  // bytes
    const int last = min(c + kVec<T>, width) - 1;
    const Words low = *reinterpret_cast<const Words*>(unit);
    const Words high = reinterpret_cast<uintptr_t>(row + last) >= unit + 16 ? *reinterpret_cast<const Words*>(unit + 16) : Words{};
    uint32_t w[8] = {low.w[0], low.w[1], low.w[2], low.w[3], high.w[0], high.w[1], high.w[2], high.w[3]};
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = skip & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = skip & 4 ? w[i + 1] : w[i];
    Words p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p.w[i] = sizeof(T) == 4 ? w[i] : __funnelshift_r(w[i], w[i + 1], skip % 4 * 8);
    return within<T>(p, c, width);
}
template <class T>
__device__ __forceinline__ void store_cut(T* row, int c, int width, const Words& p) {
#pragma unroll
    for (int k = 0; k < kVec<T>; ++k) {
        if (c + k < 0 || c + k >= width) continue;
        if constexpr (sizeof(T) == 4)
            reinterpret_cast<uint32_t*>(row)[c + k] = p.w[k];
        else
            reinterpret_cast<uint16_t*>(row)[c + k] = (uint16_t)(p.w[k / 2] >> (k % 2 * 16));
    }
}
#endif

}  // namespace a2
