// Internal declarations of the language-model operators (embedding, vocabulary loss, orthogonalisation).
// The entry points in lm_api.cu validate; the functions below launch. All return a cudaError_t.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

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
// successor do the same, and waits until everything before it is done and visible.
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
#endif

}  // namespace a2
