// C ABI of the norm, the routing and the clipping: argument checks, then the launches of rms_norm.cu, route.cu and clip.cu.
#include <algorithm>
#include <memory>
#include <new>

#include "lm_checks.h"

namespace {

constexpr int64_t kMaxTensors = 65536;

int check_rows(int64_t n, int64_t width) {
    A2_CHECK(n >= 0 && width >= 1, A2_EINVAL, "need width >= 1 and no negative count");
    A2_CHECK(n <= kMaxRows, A2_ERANGE, "more than %lld rows", (long long)kMaxRows);
    A2_CHECK(width <= a2::kMaxNormWidth, A2_ERANGE, "width beyond %lld", (long long)a2::kMaxNormWidth);
    return A2_OK;
}

int check_eps(double eps) {
    A2_CHECK(std::isfinite((float)eps) && eps >= 0, A2_EINVAL, "need eps >= 0, finite in fp32");
    return A2_OK;
}

int check_block(int64_t block) {
    A2_CHECK(block == 0 || block == 32 || block == 64 || block == 128, A2_EINVAL, "block is 32, 64, 128 or 0 for whole rows");
    return A2_OK;
}

int check_vector(const char* name, const void* p, int32_t dtype) {
    A2_CHECK(reinterpret_cast<uintptr_t>(p) % (dtype == A2_BF16 ? 2 : 4) == 0, A2_EINVAL, "%s is not aligned to its elements", name);
    return A2_OK;
}

// Of two buffers that may be one: then with one pitch.
int check_in_place(const char* name, const void* p, int64_t p_pitch, const void* q, int64_t q_pitch, int64_t n) {
    A2_CHECK(!p || p != q || p_pitch == q_pitch || n <= 1, A2_EINVAL, "%s in place needs the same pitch", name);
    return A2_OK;
}

int check_norm(const void* x, int64_t x_pitch, const void* residual, int64_t residual_pitch, const void* weight, int64_t n, int64_t width, double eps, const void* sum,
               int64_t sum_pitch, int32_t dtype) {
    A2_TRY(check_type(dtype));
    A2_TRY(check_rows(n, width));
    A2_TRY(check_eps(eps));
    A2_TRY(check_matrix("x", x, n, width, x_pitch, dtype));
    if (residual) A2_TRY(check_matrix("residual", residual, n, width, residual_pitch, dtype));
    A2_TRY(check_vector("weight", weight, dtype));
    if (sum) A2_TRY(check_matrix("sum", sum, n, width, sum_pitch, dtype));
    A2_TRY(check_in_place("sum", sum, sum_pitch, x, x_pitch, n));
    return check_in_place("sum", sum, sum_pitch, residual, residual_pitch, n);
}

int check_bytes(const char* name, const void* p, int64_t n, int64_t width, int64_t pitch) {
    A2_CHECK(p || n == 0, A2_EINVAL, "%s is NULL", name);
    A2_CHECK(pitch >= width && pitch <= kMaxPitch, A2_EINVAL, "pitch of %s must be at least its width", name);
    return A2_OK;
}

int check_score(int32_t score) {
    A2_CHECK(score == A2_SCORE_SOFTMAX || score == A2_SCORE_SIGMOID, A2_EINVAL, "unknown score");
    return A2_OK;
}

int check_experts(int64_t n, int64_t experts, int64_t k) {
    A2_CHECK(n >= 0 && experts >= 1 && k >= 1 && k <= experts, A2_EINVAL, "need 1 <= k <= n_experts and no negative count");
    A2_CHECK(n <= kMaxRows, A2_ERANGE, "more than %lld tokens", (long long)kMaxRows);
    A2_CHECK(experts <= a2::kMaxExperts && k <= a2::kMaxChosen, A2_ERANGE, "more than %d experts or %d chosen ones", (int)a2::kMaxExperts, (int)a2::kMaxChosen);
    return A2_OK;
}

int check_tensor_counts(int64_t n_tensors, int64_t workers) {
    A2_CHECK(n_tensors >= 0 && workers >= 0, A2_EINVAL, "a negative count");
    A2_CHECK(n_tensors <= kMaxTensors && workers <= kMaxMats, A2_ERANGE, "more than %lld tensors or %lld workers", (long long)kMaxTensors, (long long)kMaxMats);
    return A2_OK;
}

// One side of a tensor of a gradient.
int check_side(const char* name, const void* p, const a2cid2_gradient_t& t, int64_t pitch, int64_t stride, int64_t workers) {
    A2_CHECK(p || t.rows * t.cols == 0 || workers == 0, A2_EINVAL, "%s of a tensor is NULL", name);
    A2_CHECK(reinterpret_cast<uintptr_t>(p) % (t.storage_dtype == A2_BF16 ? 2 : 4) == 0, A2_EINVAL, "%s of a tensor is not aligned to its elements", name);
    A2_CHECK(t.rows <= 1 || (pitch >= t.cols && pitch <= kMaxPitch), A2_EINVAL, "pitch of %s of a tensor must be at least its columns", name);
    A2_CHECK(workers <= 1 || t.rows * t.cols == 0 || (stride >= (t.rows - 1) * (t.rows > 1 ? pitch : 0) + t.cols && stride <= kMaxPitch), A2_EINVAL,
             "the stride from worker to worker must be at least a tensor's extent");
    return A2_OK;
}

int check_gradients(const a2cid2_gradient_t* tensors, int64_t n_tensors, int64_t workers, bool clip) {
    A2_TRY(check_tensor_counts(n_tensors, workers));
    A2_CHECK(tensors || n_tensors == 0, A2_EINVAL, "tensors is NULL");
    double all = 0.0;
    for (int64_t i = 0; i < n_tensors; ++i) {
        const a2cid2_gradient_t& t = tensors[i];
        A2_CHECK(t.storage_dtype == A2_F32 || t.storage_dtype == A2_BF16, A2_EINVAL, "unknown storage type of a tensor");
        A2_CHECK(t.rows >= 0 && t.cols >= 0, A2_EINVAL, "a negative size of a tensor");
        A2_CHECK((double)t.rows * (double)t.cols <= 0x1p40, A2_ERANGE, "a tensor of more than 2^40 elements");
        all += (double)t.rows * (double)t.cols;
        A2_TRY(check_side("in", t.in, t, t.pitch, t.worker_stride, workers));
        if (!clip) continue;
        A2_TRY(check_side("out", t.out, t, t.out_pitch, t.out_worker_stride, workers));
        A2_CHECK(t.in != t.out || ((t.rows <= 1 || t.pitch == t.out_pitch) && (workers <= 1 || t.worker_stride == t.out_worker_stride)), A2_EINVAL,
                 "in place needs the same stride and pitch on both sides");
    }
    A2_CHECK(all <= 0x1p44, A2_ERANGE, "more than 2^44 elements");  // chunks of all workers are numbered in 64 bits with room
    if (!clip || n_tensors < 2) return A2_OK;
    // the same place twice would be scaled twice
    std::unique_ptr<const void*[]> outs(new (std::nothrow) const void*[n_tensors]);
    A2_CHECK(outs, A2_ENOMEM, "no memory for %lld addresses", (long long)n_tensors);
    int64_t count = 0;
    for (int64_t i = 0; i < n_tensors; ++i)
        if (tensors[i].rows * tensors[i].cols > 0) outs[count++] = tensors[i].out;
    std::sort(outs.get(), outs.get() + count, std::less<const void*>());
    A2_CHECK(std::adjacent_find(outs.get(), outs.get() + count) == outs.get() + count || workers == 0, A2_EINVAL, "two tensors have the same out");
    return A2_OK;
}

}  // namespace

extern "C" {

int a2cid2_rms_norm(const void* x, int64_t x_pitch, const void* residual, int64_t residual_pitch, const void* weight, int64_t n, int64_t width, double eps,
                    void* sum, int64_t sum_pitch, void* out, int64_t out_pitch, int32_t storage_dtype, void* cuda_stream) {
    A2_TRY(check_norm(x, x_pitch, residual, residual_pitch, weight, n, width, eps, sum, sum_pitch, storage_dtype));
    A2_TRY(check_matrix("out", out, n, width, out_pitch, storage_dtype));
    A2_TRY(check_in_place("out", out, out_pitch, x, x_pitch, n));
    A2_TRY(check_in_place("out", out, out_pitch, residual, residual_pitch, n));
    A2_CHECK(!sum || sum != out || n == 0, A2_EINVAL, "sum and out are the same");
    A2_TRY(check_complete());
    const a2::NormArgs a{x, x_pitch, residual, residual_pitch, weight, n, width, (float)eps, sum, sum_pitch, out, out_pitch, nullptr, 0, storage_dtype};
    return status(a2::run_norm(a, (cudaStream_t)cuda_stream), "root-mean-square norm");
}

int a2cid2_rms_norm_e4m3(const void* x, int64_t x_pitch, const void* residual, int64_t residual_pitch, const void* weight, int64_t n, int64_t width, double eps,
                         void* sum, int64_t sum_pitch, int64_t block, void* values, int64_t values_pitch, float* scales, int32_t storage_dtype,
                         void* cuda_stream) {
    A2_TRY(check_norm(x, x_pitch, residual, residual_pitch, weight, n, width, eps, sum, sum_pitch, storage_dtype));
    A2_TRY(check_block(block));
    A2_TRY(check_bytes("values", values, n, width, values_pitch));
    A2_CHECK(scales || n == 0, A2_EINVAL, "scales is NULL");
    A2_TRY(check_floats("scales", scales));
    A2_TRY(check_complete());
    const a2::NormArgs a{x, x_pitch, residual, residual_pitch, weight, n, width, (float)eps, sum, sum_pitch, values, values_pitch, scales, block, storage_dtype};
    return status(a2::run_norm(a, (cudaStream_t)cuda_stream), "root-mean-square norm");
}

int a2cid2_dequantize_e4m3(const void* values, int64_t values_pitch, const float* scales, int64_t n, int64_t width, int64_t block, void* out, int64_t out_pitch,
                           int32_t storage_dtype, void* cuda_stream) {
    A2_TRY(check_type(storage_dtype));
    A2_TRY(check_rows(n, width));
    A2_TRY(check_block(block));
    A2_TRY(check_bytes("values", values, n, width, values_pitch));
    A2_CHECK(scales || n == 0, A2_EINVAL, "scales is NULL");
    A2_TRY(check_floats("scales", scales));
    A2_TRY(check_matrix("out", out, n, width, out_pitch, storage_dtype));
    A2_TRY(check_complete());
    const a2::DequantizeArgs a{static_cast<const uint8_t*>(values), values_pitch, scales, n, width, block, out, out_pitch, storage_dtype};
    return status(a2::run_dequantize(a, (cudaStream_t)cuda_stream), "values from 8 bits");
}

int a2cid2_rms_norm_grad_workspace(int64_t n, int64_t width, int32_t with_weight, int32_t storage_dtype, int64_t* bytes) {
    A2_CHECK(bytes, A2_EINVAL, "bytes is NULL");
    A2_TRY(check_type(storage_dtype));
    A2_TRY(check_rows(n, width));
    *bytes = a2::norm_grad_workspace(n, width, with_weight != 0, storage_dtype);
    return A2_OK;
}

int a2cid2_rms_norm_grad(const void* grad_out, int64_t grad_out_pitch, const void* x, int64_t x_pitch, const void* weight, const void* grad_sum,
                         int64_t grad_sum_pitch, int64_t n, int64_t width, double eps, void* grad_x, int64_t grad_x_pitch, void* grad_weight,
                         int32_t storage_dtype, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    A2_TRY(check_type(storage_dtype));
    A2_TRY(check_rows(n, width));
    A2_TRY(check_eps(eps));
    A2_TRY(check_matrix("grad_out", grad_out, n, width, grad_out_pitch, storage_dtype));
    A2_TRY(check_matrix("x", x, n, width, x_pitch, storage_dtype));
    A2_TRY(check_vector("weight", weight, storage_dtype));
    A2_TRY(check_vector("grad_weight", grad_weight, storage_dtype));
    if (grad_sum) A2_TRY(check_matrix("grad_sum", grad_sum, n, width, grad_sum_pitch, storage_dtype));
    if (grad_x) A2_TRY(check_matrix("grad_x", grad_x, n, width, grad_x_pitch, storage_dtype));
    A2_TRY(check_in_place("grad_x", grad_x, grad_x_pitch, grad_out, grad_out_pitch, n));
    A2_TRY(check_in_place("grad_x", grad_x, grad_x_pitch, grad_sum, grad_sum_pitch, n));
    A2_TRY(check_in_place("grad_x", grad_x, grad_x_pitch, x, x_pitch, n));
    A2_TRY(check_workspace(workspace, workspace_bytes, a2::norm_grad_workspace(n, width, grad_weight != nullptr, storage_dtype)));
    A2_TRY(check_complete());
    const a2::NormGradArgs a{grad_out, grad_out_pitch, x, x_pitch, weight, grad_sum, grad_sum_pitch, n, width, (float)eps, grad_x, grad_x_pitch, grad_weight,
                             storage_dtype};
    return status(a2::run_norm_grad(a, workspace, (cudaStream_t)cuda_stream), "gradient of the norm");
}

int a2cid2_route(const void* logits, int64_t logits_pitch, int64_t n, int64_t n_experts, int64_t k, int32_t score, const float* bias, int64_t groups,
                 int64_t top_groups, int32_t group_score, int32_t renormalize, double scale, int32_t* ids, float* weights, int32_t* counts,
                 int32_t storage_dtype, void* cuda_stream) {
    A2_TRY(check_type(storage_dtype));
    A2_TRY(check_experts(n, n_experts, k));
    A2_TRY(check_score(score));
    A2_TRY(check_number("scale", scale));
    A2_CHECK(group_score == A2_GROUP_BEST || group_score == A2_GROUP_TWO_BEST, A2_EINVAL, "unknown score of groups");
    A2_CHECK(groups >= 1 && n_experts % groups == 0 && top_groups >= 1 && top_groups <= groups, A2_EINVAL,
             "groups must divide the experts, and 1 <= top_groups <= groups");
    A2_CHECK(groups <= a2::kMaxGroups, A2_ERANGE, "more than %d groups", (int)a2::kMaxGroups);
    A2_CHECK(k <= n_experts / groups * top_groups, A2_EINVAL, "k is more than the experts of the open groups");
    A2_TRY(check_matrix("logits", logits, n, n_experts, logits_pitch, storage_dtype));
    A2_TRY(check_floats("bias", bias));
    A2_TRY(check_ids("ids", ids, n));
    A2_CHECK(weights || n == 0, A2_EINVAL, "weights is NULL");
    A2_TRY(check_floats("weights", weights));
    if (counts) A2_TRY(check_ids("counts", counts, n_experts));
    A2_TRY(check_complete());
    const a2::RouteArgs a{logits, logits_pitch, n, (int)n_experts, (int)k, score, bias, (int)groups, (int)top_groups, group_score, renormalize != 0, (float)scale, ids,
                          weights, counts, storage_dtype};
    return status(a2::run_route(a, (cudaStream_t)cuda_stream), "routing");
}

int a2cid2_route_grad(const void* logits, int64_t logits_pitch, const int32_t* ids, const float* grad_weights, int64_t n, int64_t n_experts, int64_t k, int32_t score,
                      int32_t renormalize, double scale, void* grad_logits, int64_t grad_logits_pitch, int32_t storage_dtype, void* cuda_stream) {
    A2_TRY(check_type(storage_dtype));
    A2_TRY(check_experts(n, n_experts, k));
    A2_TRY(check_score(score));
    A2_TRY(check_number("scale", scale));
    A2_TRY(check_matrix("logits", logits, n, n_experts, logits_pitch, storage_dtype));
    A2_TRY(check_ids("ids", ids, n));
    A2_CHECK(grad_weights || n == 0, A2_EINVAL, "grad_weights is NULL");
    A2_TRY(check_floats("grad_weights", grad_weights));
    A2_TRY(check_matrix("grad_logits", grad_logits, n, n_experts, grad_logits_pitch, storage_dtype));
    A2_TRY(check_in_place("grad_logits", grad_logits, grad_logits_pitch, logits, logits_pitch, n));
    A2_TRY(check_complete());
    const a2::RouteGradArgs a{logits, logits_pitch, ids, grad_weights, n, (int)n_experts, (int)k, score, renormalize != 0, (float)scale, grad_logits,
                              grad_logits_pitch, storage_dtype};
    return status(a2::run_route_grad(a, (cudaStream_t)cuda_stream), "gradient of the routing");
}

int a2cid2_clip_gradients_workspace(int64_t n_tensors, int64_t workers, int64_t* bytes) {
    A2_CHECK(bytes, A2_EINVAL, "bytes is NULL");
    A2_TRY(check_tensor_counts(n_tensors, workers));
    *bytes = a2::clip_workspace(n_tensors, workers);
    return A2_OK;
}

int a2cid2_gradient_norms(const a2cid2_gradient_t* tensors, int64_t n_tensors, int64_t workers, float* norms, void* workspace, int64_t workspace_bytes,
                          void* cuda_stream) {
    A2_TRY(check_gradients(tensors, n_tensors, workers, false));
    A2_CHECK(norms || workers == 0, A2_EINVAL, "norms is NULL");
    A2_TRY(check_floats("norms", norms));
    A2_TRY(check_workspace(workspace, workspace_bytes, a2::clip_workspace(n_tensors, workers)));
    A2_TRY(check_complete());
    const a2::ClipArgs a{tensors, n_tensors, workers, false, 0.0, false, norms};
    return status(a2::run_clip(a, workspace, (cudaStream_t)cuda_stream), "gradient norms");
}

int a2cid2_clip_gradients(const a2cid2_gradient_t* tensors, int64_t n_tensors, int64_t workers, double max_norm, int32_t zero_nonfinite, float* norms,
                          void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    A2_TRY(check_gradients(tensors, n_tensors, workers, true));
    A2_CHECK(max_norm >= 0, A2_EINVAL, "need max_norm >= 0");
    A2_CHECK(norms || workers == 0, A2_EINVAL, "norms is NULL");
    A2_TRY(check_floats("norms", norms));
    A2_TRY(check_workspace(workspace, workspace_bytes, a2::clip_workspace(n_tensors, workers)));
    A2_TRY(check_complete());
    const a2::ClipArgs a{tensors, n_tensors, workers, true, max_norm, zero_nonfinite != 0, norms};
    return status(a2::run_clip(a, workspace, (cudaStream_t)cuda_stream), "clipping");
}

}  // extern "C"
