// Stands in for the CUDA runtime calls of the language-model operators (linked with --wrap), so that their host side runs without a GPU:
// launches are counted, and one of them can be made to fail.
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdlib>
#include <string>

namespace {
int g_launches = 0, g_fail_at = -1, g_bad_maps = 0;
void* g_host = nullptr;
std::string g_text;

cudaError_t queue() { return g_launches++ == g_fail_at ? cudaErrorLaunchOutOfResources : cudaSuccess; }

// Refuses what the driver would refuse, and counts it.
CUresult encode(CUtensorMap*, CUtensorMapDataType, cuuint32_t rank, void* base, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box,
                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
    bool ok = rank == 3 && reinterpret_cast<uintptr_t>(base) % 16 == 0;
    for (cuuint32_t k = 0; k < rank; ++k) ok = ok && dims[k] >= 1 && dims[k] <= (cuuint64_t(1) << 32) && box[k] >= 1 && box[k] <= 256;
    for (cuuint32_t k = 0; k + 1 < rank; ++k) ok = ok && strides[k] % 16 == 0 && strides[k] < (cuuint64_t(1) << 40);
    g_bad_maps += !ok;
    return ok ? CUDA_SUCCESS : CUDA_ERROR_INVALID_VALUE;
}
}  // namespace

namespace a2 {
void set_thread_error(const std::string& text) { g_text = text; }
}  // namespace a2

extern "C" {
void fake_reset(int fail_at) {
    g_launches = g_bad_maps = 0;
    g_fail_at = fail_at;
    g_text.clear();
}
int fake_launches() { return g_launches; }
int fake_bad_maps() { return g_bad_maps; }
const char* fake_error_text() { return g_text.c_str(); }

cudaError_t __wrap_cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void*, void**) {
    if (c->gridDim.x == 0 || c->gridDim.y == 0 || c->gridDim.y > 65535 || c->gridDim.z > 65535) return cudaErrorInvalidConfiguration;
    return queue();
}
cudaError_t __wrap_cudaMemset2DAsync(void*, size_t, int, size_t, size_t, cudaStream_t) { return queue(); }
cudaError_t __wrap_cudaGetDevice(int* device) {
    *device = 0;
    return cudaSuccess;
}
cudaError_t __wrap_cudaDeviceGetAttribute(int* value, cudaDeviceAttr, int) {
    *value = 148;  // the only one asked for: the number of multiprocessors
    return cudaSuccess;
}
cudaError_t __wrap_cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t __wrap_cudaHostAlloc(void** p, size_t bytes, unsigned int) {
    *p = g_host = std::calloc(1, bytes);
    return cudaSuccess;
}
int* fake_host_memory() { return static_cast<int*>(g_host); }
cudaError_t __wrap_cudaThreadExchangeStreamCaptureMode(cudaStreamCaptureMode*) { return cudaSuccess; }
cudaError_t __wrap_cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t __wrap_cudaGetDriverEntryPointByVersion(const char*, void** p, unsigned int, unsigned long long, cudaDriverEntryPointQueryResult* found) {
    *p = reinterpret_cast<void*>(encode);
    *found = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
cudaError_t __wrap_cudaGetLastError() { return cudaSuccess; }
}
