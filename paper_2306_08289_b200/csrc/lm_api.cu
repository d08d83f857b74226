// C ABI of the language-model operators: argument checks, then the launches of embed.cu, vocab_loss.cu and
// orthogonalize.cu.
#include "lm_checks.h"

extern "C" {

int a2cid2_embed(const void* table, int64_t vocab, int64_t width, int64_t table_pitch, const int32_t* ids, int64_t n_ids,
                 double scale, void* out, int64_t out_pitch, int32_t storage_dtype, void* cuda_stream) {
    A2_TRY(check_type(storage_dtype));
    A2_TRY(check_table_sizes(vocab, width, n_ids));
    A2_TRY(check_number("scale", scale));
    A2_TRY(check_matrix("table", table, vocab, width, table_pitch, storage_dtype));
    A2_TRY(check_ids("ids", ids, n_ids));
    A2_TRY(check_matrix("out", out, n_ids, width, out_pitch, storage_dtype));
    A2_TRY(check_complete());
    const a2::EmbedArgs a{table, vocab, width, table_pitch, ids, n_ids, (float)scale, out, out_pitch, storage_dtype};
    return status(a2::run_embed(a, (cudaStream_t)cuda_stream), "embedding lookup");
}

int a2cid2_embed_grad_workspace(int64_t vocab, int64_t width, int64_t n_ids, int64_t* bytes) {
    A2_CHECK(bytes, A2_EINVAL, "bytes is NULL");
    A2_TRY(check_table_sizes(vocab, width, n_ids));
    A2_CHECK(n_ids <= kMaxSorted, A2_ERANGE, "more than %lld ids in a gradient", (long long)kMaxSorted);
    *bytes = a2::embed_grad_workspace(vocab, width, n_ids);
    return A2_OK;
}

int a2cid2_embed_grad(const void* grad_out, int64_t grad_out_pitch, const int32_t* ids, int64_t n_ids, int64_t vocab,
                      int64_t width, double scale, int32_t accumulate, void* grad_table, int64_t grad_table_pitch,
                      int32_t storage_dtype, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    A2_TRY(check_type(storage_dtype));
    A2_TRY(check_table_sizes(vocab, width, n_ids));
    A2_CHECK(n_ids <= kMaxSorted, A2_ERANGE, "more than %lld ids in a gradient", (long long)kMaxSorted);
    A2_TRY(check_number("scale", scale));
    A2_TRY(check_matrix("grad_out", grad_out, n_ids, width, grad_out_pitch, storage_dtype));
    A2_TRY(check_ids("ids", ids, n_ids));
    A2_TRY(check_matrix("grad_table", grad_table, vocab, width, grad_table_pitch, storage_dtype));
    A2_TRY(check_workspace(workspace, workspace_bytes, a2::embed_grad_workspace(vocab, width, n_ids)));
    A2_TRY(check_complete());
    const a2::EmbedGradArgs a{grad_out, grad_out_pitch, ids, n_ids, vocab, width, (float)scale, accumulate != 0, grad_table, grad_table_pitch,
                              storage_dtype};
    return status(a2::run_embed_grad(a, workspace, (cudaStream_t)cuda_stream), "embedding gradient");
}

int a2cid2_vocab_loss_workspace(int64_t n_tokens, int64_t width, int64_t vocab, int32_t with_grad, int32_t storage_dtype,
                                int64_t* bytes) {
    A2_CHECK(bytes, A2_EINVAL, "bytes is NULL");
    A2_TRY(check_type(storage_dtype));
    A2_TRY(check_table_sizes(vocab, width, n_tokens));
    A2_TRY(check_tiles(n_tokens, vocab));
    *bytes = a2::vocab_loss_workspace(n_tokens, width, vocab, with_grad != 0, storage_dtype);
    return A2_OK;
}

int a2cid2_vocab_loss(const void* hidden, int64_t hidden_pitch, const void* head, int64_t head_pitch, const int32_t* targets,
                      int64_t n_tokens, int64_t width, int64_t vocab, const float* weights, double scale, float* loss,
                      float* lse, void* grad_hidden, int64_t grad_hidden_pitch, void* grad_head, int64_t grad_head_pitch,
                      int32_t storage_dtype, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    A2_TRY(check_type(storage_dtype));
    A2_TRY(check_table_sizes(vocab, width, n_tokens));
    A2_TRY(check_tiles(n_tokens, vocab));
    A2_TRY(check_number("scale", scale));
    A2_TRY(check_matrix("hidden", hidden, n_tokens, width, hidden_pitch, storage_dtype));
    A2_TRY(check_matrix("head", head, vocab, width, head_pitch, storage_dtype));
    A2_TRY(check_ids("targets", targets, n_tokens));
    A2_CHECK((loss && lse) || n_tokens == 0, A2_EINVAL, "loss or lse is NULL");
    A2_TRY(check_floats("loss", loss));
    A2_TRY(check_floats("lse", lse));
    A2_TRY(check_floats("weights", weights));
    if (grad_hidden) A2_TRY(check_matrix("grad_hidden", grad_hidden, n_tokens, width, grad_hidden_pitch, storage_dtype));
    if (grad_head) A2_TRY(check_matrix("grad_head", grad_head, vocab, width, grad_head_pitch, storage_dtype));
    const bool with_grad = grad_hidden || grad_head;
    A2_TRY(check_workspace(workspace, workspace_bytes, a2::vocab_loss_workspace(n_tokens, width, vocab, with_grad, storage_dtype)));
    A2_TRY(check_complete());
    const a2::VocabLossArgs a{hidden, hidden_pitch, head, head_pitch, targets, n_tokens, width, vocab, weights, (float)scale, loss, lse,
                              grad_hidden, grad_hidden_pitch, grad_head, grad_head_pitch, storage_dtype};
    return status(a2::run_vocab_loss(a, workspace, (cudaStream_t)cuda_stream), "vocabulary loss");
}

int a2cid2_orthogonalize_workspace(int64_t n_mats, int64_t rows, int64_t cols, int32_t storage_dtype, int64_t* bytes) {
    A2_CHECK(bytes, A2_EINVAL, "bytes is NULL");
    A2_TRY(check_type(storage_dtype));
    A2_TRY(check_batch_sizes(n_mats, rows, cols));
    *bytes = a2::orthogonalize_workspace(n_mats, rows, cols, storage_dtype);
    return A2_OK;
}

int a2cid2_orthogonalize(const void* in, int64_t in_stride, int64_t in_pitch, int64_t n_mats, int64_t rows, int64_t cols,
                         int32_t steps, double a, double b, double c, double eps, double scale, void* out, int64_t out_stride,
                         int64_t out_pitch, int32_t storage_dtype, void* workspace, int64_t workspace_bytes,
                         void* cuda_stream) {
    A2_TRY(check_type(storage_dtype));
    A2_TRY(check_batch_sizes(n_mats, rows, cols));
    A2_CHECK(steps >= 0 && steps <= 1000, A2_EINVAL, "need 0 <= steps <= 1000");
    A2_TRY(check_number("a", a));
    A2_TRY(check_number("b", b));
    A2_TRY(check_number("c", c));
    A2_TRY(check_number("scale", scale));
    A2_CHECK(std::isfinite(eps) && eps >= 0, A2_EINVAL, "need eps >= 0");
    A2_CHECK(a2::orthogonalize_range(a, b, c, steps), A2_EINVAL,
             "the coefficients take singular values of [0, 1] beyond 1.95 or the polynomial beyond 3.9");
    A2_TRY(check_matrix("in", in, n_mats, cols, in_pitch, storage_dtype));
    A2_TRY(check_matrix("out", out, n_mats, cols, out_pitch, storage_dtype));
    // matrices of a batch may not share elements: a matrix takes (rows - 1) * pitch + cols of them
    A2_CHECK(n_mats <= 1 || (in_stride >= (rows - 1) * in_pitch + cols && out_stride >= (rows - 1) * out_pitch + cols), A2_EINVAL,
             "the stride from matrix to matrix must be at least a matrix's extent");
    A2_CHECK(in_stride <= kMaxPitch && out_stride <= kMaxPitch, A2_ERANGE, "a stride beyond %lld", (long long)kMaxPitch);
    A2_CHECK(in != out || n_mats == 0 || (in_pitch == out_pitch && (n_mats == 1 || in_stride == out_stride)), A2_EINVAL,
             "in place needs the same stride and pitch on both sides");
    A2_TRY(check_workspace(workspace, workspace_bytes, a2::orthogonalize_workspace(n_mats, rows, cols, storage_dtype)));
    if (n_mats == 0) return A2_OK;
    A2_TRY(check_complete());
    const a2::OrthogonalizeArgs args{in, in_stride, in_pitch, n_mats, rows, cols, steps, (float)a, (float)b, (float)c, eps, (float)scale, out,
                                     out_stride, out_pitch, storage_dtype};
    return status(a2::run_orthogonalize(args, workspace, (cudaStream_t)cuda_stream), "orthogonalisation");
}

int a2cid2_operators_check(void* cuda_stream) {
    bool gave_up = false;
    A2_TRY(status(a2::check_products((cudaStream_t)cuda_stream, &gave_up), "operators check"));
    A2_CHECK(!gave_up, A2_ECUDA, "a product gave up waiting for its operands: results since the last check may be incomplete");
    return A2_OK;
}

}  // extern "C"
