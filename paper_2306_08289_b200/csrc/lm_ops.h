// Internal declarations of the language-model operators (embedding, vocabulary loss, orthogonalisation).
// The entry points in lm_api.cu validate; the functions below launch. All return a cudaError_t.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

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
    float center;  // of orthogonalize_range
    double eps;
    float scale;
    void* out;
    int64_t out_stride, out_pitch;
    int32_t dtype;
};
// Whether the steps keep singular values of [0, 1], and the polynomial, inside what the fp16 intermediates hold; the
// polynomial's middle.
bool orthogonalize_range(double a, double b, double c, int steps, double* center);
int64_t orthogonalize_workspace(int64_t n_mats, int64_t rows, int64_t cols, int32_t dtype);
cudaError_t run_orthogonalize(const OrthogonalizeArgs& a, void* workspace, cudaStream_t s);

cudaError_t products_gave_up(cudaStream_t s, bool* out);  // waits for the stream; whether a product ever gave up on this device

#ifdef __CUDACC__
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <class T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
    T v[VEC];
};
#endif

}  // namespace a2
