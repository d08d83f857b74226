// Argument checks of the language-model operators' C entry points: each gives A2_OK, or a status whose text it has set. Included once by every file
// of entry points.
#pragma once

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "a2cid2_internal.h"
#include "lm_ops.h"

namespace {

[[maybe_unused]] int fail(int code, const char* format, ...) {
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

[[maybe_unused]] int status(cudaError_t e, const char* what) {
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

[[maybe_unused]] int check_type(int32_t dtype) {
    A2_CHECK(dtype == A2_F32 || dtype == A2_BF16, A2_EINVAL, "unknown storage type");
    return A2_OK;
}

// A matrix of `rows` rows: `p` may be NULL only when it has none.
[[maybe_unused]] int check_matrix(const char* name, const void* p, int64_t rows, int64_t width, int64_t pitch, int32_t dtype) {
    A2_CHECK(p || rows == 0, A2_EINVAL, "%s is NULL", name);
    A2_CHECK(reinterpret_cast<uintptr_t>(p) % (dtype == A2_BF16 ? 2 : 4) == 0, A2_EINVAL, "%s is not aligned to its elements", name);
    A2_CHECK(pitch >= width && pitch <= kMaxPitch, A2_EINVAL, "pitch of %s must be at least its width", name);
    return A2_OK;
}

[[maybe_unused]] int check_ids(const char* name, const int32_t* p, int64_t n) {
    A2_CHECK(p || n == 0, A2_EINVAL, "%s is NULL", name);
    A2_CHECK(reinterpret_cast<uintptr_t>(p) % 4 == 0, A2_EINVAL, "%s is not aligned to its elements", name);
    return A2_OK;
}

[[maybe_unused]] int check_floats(const char* name, const float* p) {
    A2_CHECK(reinterpret_cast<uintptr_t>(p) % 4 == 0, A2_EINVAL, "%s is not aligned to its elements", name);
    return A2_OK;
}

// A parameter the kernels use as a float.
[[maybe_unused]] int check_number(const char* name, double v) {
    A2_CHECK(std::isfinite((float)v), A2_EINVAL, "%s must be finite in fp32", name);
    return A2_OK;
}

[[maybe_unused]] int check_workspace(const void* p, int64_t have, int64_t need) {
    A2_CHECK(have >= need, A2_EINVAL, "workspace of %lld bytes, %lld needed", (long long)have, (long long)need);
    A2_CHECK(p || need == 0, A2_EINVAL, "workspace is NULL");
    A2_CHECK(reinterpret_cast<uintptr_t>(p) % 256 == 0, A2_EINVAL, "workspace must be 256-byte aligned");
    return A2_OK;
}

[[maybe_unused]] int check_table_sizes(int64_t vocab, int64_t width, int64_t n_ids) {
    A2_CHECK(vocab >= 1 && width >= 1 && n_ids >= 0, A2_EINVAL, "need vocab >= 1, width >= 1 and no negative count");
    A2_CHECK(vocab <= kMaxRows && n_ids <= kMaxRows, A2_ERANGE, "more than %lld rows", (long long)kMaxRows);
    A2_CHECK(width <= kMaxWidth, A2_ERANGE, "width beyond %lld", (long long)kMaxWidth);
    return A2_OK;
}

// A product that gave up a wait has left a result incomplete: nothing more is queued until the caller has been told.
[[maybe_unused]] int check_complete() {
    A2_CHECK(!a2::products_gave_up(), A2_ECUDA, "a product of an earlier call gave up a wait: its results are incomplete (a2cid2_operators_check)");
    return A2_OK;
}

// The products count their tiles in 32 bits.
[[maybe_unused]] int check_tiles(int64_t n_tokens, int64_t vocab) {
    A2_CHECK(a2::ceil_div(n_tokens, 256) * a2::ceil_div(vocab, 256) < (int64_t(1) << 30), A2_ERANGE, "n_tokens * vocab beyond 2^46");
    return A2_OK;
}

[[maybe_unused]] int check_batch_sizes(int64_t n_mats, int64_t rows, int64_t cols) {
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
