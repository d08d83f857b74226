// C ABI of the language-model operators: argument checks, then the launches of embed.cu, vocab_loss.cu and
// orthogonalize.cu.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "a2cid2_internal.h"
#include "lm_ops.h"

namespace {

int fail(int code, const char* format, ...) {
    char text[256];
    va_list args;
    va_start(args, format);
    std::vsnprintf(text, sizeof text, format, args);
    va_end(args);
    try {
        a2::set_thread_error(text);
    } catch (...) {  // no memory for the text: the code alone has to do
    }
    return code;
}

int status(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return A2_OK;
    (void)cudaGetLastError();  // reported here, and not once more by whoever asks next
    return fail(A2_ECUDA, "%s: %s (%s)", what, cudaGetErrorName(e), cudaGetErrorString(e));
}

constexpr int64_t kMaxRows = int64_t(1) << 30;        // ids, tokens, vocabulary rows
constexpr int64_t kMaxSorted = int64_t(1) << 26;      // ids of a gradient: every tile of the sort reads the counts of all tiles
constexpr int64_t kMaxWidth = int64_t(1) << 20;       // columns of a matrix
constexpr int64_t kMaxMats = 65535;                   // matrices of a batch
constexpr int64_t kMaxPitch = int64_t(1) << 40;       // elements; keeps row * pitch inside 64 bits with room

#define A2_CHECK(ok, code, ...)                        \
    do {                                               \
        if (!(ok)) return fail((code), __VA_ARGS__);   \
    } while (0)

int check_type(int32_t dtype) {
    A2_CHECK(dtype == A2_F32 || dtype == A2_BF16, A2_EINVAL, "unknown storage type");
    return A2_OK;
}

// A matrix of `rows` rows: `p` may be NULL only when it has none.
int check_matrix(const char* name, const void* p, int64_t rows, int64_t width, int64_t pitch, int32_t dtype) {
    A2_CHECK(p || rows == 0, A2_EINVAL, "%s is NULL", name);
    A2_CHECK(reinterpret_cast<uintptr_t>(p) % (dtype == A2_BF16 ? 2 : 4) == 0, A2_EINVAL, "%s is not aligned to its elements", name);
    A2_CHECK(pitch >= width && pitch <= kMaxPitch, A2_EINVAL, "pitch of %s must be at least its width", name);
    return A2_OK;
}

int check_ids(const char* name, const int32_t* p, int64_t n) {
    A2_CHECK(p || n == 0, A2_EINVAL, "%s is NULL", name);
    A2_CHECK(reinterpret_cast<uintptr_t>(p) % 4 == 0, A2_EINVAL, "%s is not aligned to its elements", name);
    return A2_OK;
}

int check_floats(const char* name, const float* p) {
    A2_CHECK(reinterpret_cast<uintptr_t>(p) % 4 == 0, A2_EINVAL, "%s is not aligned to its elements", name);
    return A2_OK;
}

// A parameter the kernels use as a float.
int check_number(const char* name, double v) {
    A2_CHECK(std::isfinite((float)v), A2_EINVAL, "%s must be finite in fp32", name);
    return A2_OK;
}

int check_workspace(const void* p, int64_t have, int64_t need) {
    A2_CHECK(have >= need, A2_EINVAL, "workspace of %lld bytes, %lld needed", (long long)have, (long long)need);
    A2_CHECK(p || need == 0, A2_EINVAL, "workspace is NULL");
    A2_CHECK(reinterpret_cast<uintptr_t>(p) % 256 == 0, A2_EINVAL, "workspace must be 256-byte aligned");
    return A2_OK;
}

int check_table_sizes(int64_t vocab, int64_t width, int64_t n_ids) {
    A2_CHECK(vocab >= 1 && width >= 1 && n_ids >= 0, A2_EINVAL, "need vocab >= 1, width >= 1 and no negative count");
    A2_CHECK(vocab <= kMaxRows && n_ids <= kMaxRows, A2_ERANGE, "more than %lld rows", (long long)kMaxRows);
    A2_CHECK(width <= kMaxWidth, A2_ERANGE, "width beyond %lld", (long long)kMaxWidth);
    return A2_OK;
}

// A product that gave up a wait has left a result incomplete: nothing more is queued until the caller has been told.
int check_complete() {
    A2_CHECK(!a2::products_gave_up(), A2_ECUDA, "a product of an earlier call gave up a wait: its results are incomplete (a2cid2_operators_check)");
    return A2_OK;
}

// The products count their tiles in 32 bits.
int check_tiles(int64_t n_tokens, int64_t vocab) {
    A2_CHECK(a2::ceil_div(n_tokens, 256) * a2::ceil_div(vocab, 256) < (int64_t(1) << 30), A2_ERANGE, "n_tokens * vocab beyond 2^46");
    return A2_OK;
}

int check_batch_sizes(int64_t n_mats, int64_t rows, int64_t cols) {
    A2_CHECK(n_mats >= 0 && rows >= 1 && cols >= 1, A2_EINVAL, "need rows >= 1, cols >= 1 and no negative count");
    A2_CHECK(n_mats <= kMaxMats, A2_ERANGE, "more than %lld matrices", (long long)kMaxMats);
    A2_CHECK(rows <= kMaxWidth && cols <= kMaxWidth, A2_ERANGE, "a side beyond %lld", (long long)kMaxWidth);
    return A2_OK;
}

#define A2_TRY(call)              \
    do {                          \
        const int rc__ = (call);  \
        if (rc__ != A2_OK) return rc__; \
    } while (0)

}  // namespace

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
