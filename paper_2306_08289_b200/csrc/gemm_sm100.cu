// Host side of the tensor-core products: tensor maps, launch shape, the flag of kernels that gave up a wait.
#include <mutex>

#include "gemm_sm100.cuh"

namespace a2 {

namespace {

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder() {
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

// Boxes of 64 x `box_rows` (128 bytes a row) of a [mats][rows][inner] array of 16-bit elements.
cudaError_t make_map(const void* p, bool bf16, int64_t inner, int64_t rows, int64_t pitch, int64_t mats, int64_t stride, int box_rows, CUtensorMap* out) {
    const EncodeTiled encode = encoder();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)mats};
    const cuuint64_t strides[2] = {(cuuint64_t)pitch * 2, (cuuint64_t)(mats > 1 ? stride : pitch * rows) * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
    const CUresult r = encode(out, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(p), dims, strides,
                              box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t operand_maps(const Operand& o, bool bf16, int64_t mats, CUtensorMap (&out)[2]) {
    const int64_t inner = o.mn ? o.rows : o.k, rows = o.mn ? o.k : o.rows;
    for (int w = 0; w < 2; ++w) {
        const void* p = w && o.lo ? o.lo : o.p;
        const cudaError_t e = make_map(p, bf16, inner, rows, o.pitch, mats, o.stride, o.mn ? kBlockK : 128, &out[w]);
        if (e != cudaSuccess) return e;
        if (!o.lo) {
            out[1] = out[0];
            break;
        }
    }
    return cudaSuccess;
}

}  // namespace

// What the launches ask of a device, looked up at its first product.
namespace {
constexpr int kMaxDevices = 64;
std::atomic<int> g_clusters[kMaxDevices];
std::mutex g_flags_mutex;
std::atomic<int*> g_flags;  // one a device (the last one for all further), in pinned host memory that every device can write; never freed
}  // namespace

cudaError_t gave_up_flag(int** out) {
    int device = 0;
    A2_CUDA_TRY(cudaGetDevice(&device));
    if (!g_flags.load()) {
        std::lock_guard<std::mutex> lock(g_flags_mutex);
        if (!g_flags.load()) {
            // the caller's stream may be under capture: this allocation is no part of it
            cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
            A2_CUDA_TRY(cudaThreadExchangeStreamCaptureMode(&mode));
            void* p = nullptr;
            const cudaError_t e = cudaHostAlloc(&p, kMaxDevices * sizeof(int), cudaHostAllocPortable | cudaHostAllocMapped);
            A2_CUDA_TRY(cudaThreadExchangeStreamCaptureMode(&mode));
            if (e != cudaSuccess) return e;
            for (int k = 0; k < kMaxDevices; ++k) static_cast<int*>(p)[k] = 0;
            g_flags.store(static_cast<int*>(p));
        }
    }
    // with unified addressing the devices know the memory by its host address
    *out = g_flags.load() + std::min(device, kMaxDevices - 1);
    return cudaSuccess;
}

bool products_gave_up() {
    int device = 0;
    const int* flags = g_flags.load();
    if (!flags || cudaGetDevice(&device) != cudaSuccess) return false;
    return *static_cast<const volatile int*>(flags + std::min(device, kMaxDevices - 1)) != 0;
}

int gemm_clusters() {
    int device = 0, sms = 0;
    if (cudaGetDevice(&device) != cudaSuccess) return 1;
    if (device < kMaxDevices && g_clusters[device].load() > 0) return g_clusters[device].load();
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return 1;
    const int clusters = sms >= 2 ? sms / 2 : 1;
    if (device < kMaxDevices) g_clusters[device].store(clusters);
    return clusters;
}

namespace {
cudaError_t set_once(const void* kernel, cudaFuncAttribute attribute, int value, std::atomic<uint64_t>& done) {
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const uint64_t bit = device < kMaxDevices ? uint64_t(1) << device : 0;
    if (done.load() & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, attribute, value);
    if (e == cudaSuccess) done.fetch_or(bit);
    return e;
}
}  // namespace

cudaError_t allow_shared_memory(const void* kernel, int bytes, std::atomic<uint64_t>& done) {
    return set_once(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes, done);
}
cudaError_t allow_large_clusters(const void* kernel, std::atomic<uint64_t>& done) {
    return set_once(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1, done);
}

cudaError_t make_gemm(const Operand& a, const Operand& b, int64_t mats, bool bf16, bool lower, int flush, int splits, GemmArgs* g) {
    cudaError_t e = operand_maps(a, bf16, mats, g->a);
    if (e == cudaSuccess) e = operand_maps(b, bf16, mats, g->b);
    auto mirror = [&](Operand o, CUtensorMap(&out)[2]) {
        if (e != cudaSuccess || !o.symmetric) return;
        o.mn = true;
        e = operand_maps(o, bf16, mats, out);
    };
    mirror(a, g->a_mirror);
    mirror(b, g->b_mirror);
    if (e != cudaSuccess) return e;
    e = gave_up_flag(&g->gave_up);
    if (e != cudaSuccess) return e;
    g->tiles_m = (int32_t)ceil_div(a.rows, kTileM);
    g->tiles_n = (int32_t)ceil_div(b.rows, kTileN);
    g->batch = (int32_t)mats;
    g->k_blocks = (int32_t)ceil_div(a.k, kBlockK);
    g->splits = splits;
    g->passes = a.lo ? 3 : 1;
    g->flush = flush > 0 ? flush : g->k_blocks * g->passes;
    g->idesc = instruction_desc(bf16, false, false, kTileM, kTileN);  // the kernel adds the MN-major bits
    g->a_mn = a.mn;
    g->b_mn = b.mn;
    g->a_sym = a.symmetric;
    g->b_sym = b.symmetric;
    g->lower = lower;
    return cudaSuccess;
}

cudaError_t check_products(cudaStream_t s, bool* gave_up) {
    A2_CUDA_TRY(cudaStreamSynchronize(s));
    *gave_up = products_gave_up();
    if (!*gave_up) return cudaSuccess;
    int* flag = nullptr;
    A2_CUDA_TRY(gave_up_flag(&flag));
    *static_cast<volatile int*>(flag) = 0;
    return cudaSuccess;
}

}  // namespace a2
