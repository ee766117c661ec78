// A CUDA runtime of a few functions for tests of ops_api.cu's host side without a device: every call is written down, any of
// them can be made to fail, device memory is host memory.  The launches of the operators are written down too.
#include <cuda_runtime.h>

#include <cstdlib>
#include <cstring>
#include <string>

#include "ops.cuh"

namespace {
std::string g_log, g_fail, g_error;
cudaError_t g_last = cudaSuccess;

cudaError_t call(const char* name, cudaError_t failure = cudaErrorMemoryAllocation) {
    g_log += name;
    g_log += '\n';
    if (g_fail != name) return cudaSuccess;
    return g_last = failure;
}
}  // namespace

extern "C" {
const char* fake_log() { return g_log.c_str(); }
const char* fake_error() { return g_error.c_str(); }
void fake_reset(const char* fail) { g_log.clear(); g_fail = fail; g_last = cudaSuccess; }
int fake_last() { return (int)g_last; }

cudaError_t cudaGetDeviceCount(int* n) { *n = 1; return cudaSuccess; }
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, enum cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaGetLastError() { const cudaError_t e = g_last; g_last = cudaSuccess; return e; }
const char* cudaGetErrorString(cudaError_t) { return "made to fail"; }
cudaError_t cudaMalloc(void** p, size_t n) {
    const cudaError_t e = call("malloc");
    if (e == cudaSuccess) *p = std::malloc(n ? n : 1);
    return e;
}
cudaError_t cudaFree(void* p) { std::free(p); return cudaSuccess; }
cudaError_t cudaMemset(void* p, int v, size_t n) {
    const cudaError_t e = call("memset");
    if (e == cudaSuccess) std::memset(p, v, n);
    return e;
}
cudaError_t cudaMemcpy(void* d, const void* s, size_t n, enum cudaMemcpyKind) {
    const cudaError_t e = call("memcpy");
    if (e == cudaSuccess) std::memcpy(d, s, n);
    return e;
}
cudaError_t cudaMemcpyAsync(void* d, const void* s, size_t n, enum cudaMemcpyKind, cudaStream_t) {
    const cudaError_t e = call("memcpy async");
    if (e == cudaSuccess) std::memcpy(d, s, n);
    return e;
}
cudaError_t cudaMemsetAsync(void* p, int v, size_t n, cudaStream_t) {
    const cudaError_t e = call("memset async");
    if (e == cudaSuccess) std::memset(p, v, n);
    return e;
}
cudaError_t cudaMemset2DAsync(void* p, size_t pitch, int v, size_t width, size_t height, cudaStream_t) {
    const cudaError_t e = call("memset 2d");
    if (e == cudaSuccess) for (size_t r = 0; r < height; ++r) std::memset(static_cast<char*>(p) + r * pitch, v, width);
    return e;
}
cudaError_t cudaStreamSynchronize(cudaStream_t) { return call("synchronize", cudaErrorUnknown); }
cudaError_t cudaDeviceSynchronize() { return call("synchronize", cudaErrorUnknown); }

void cerar_internal_set_error(const char* msg) { g_error = msg; }
}

namespace cerar {
cudaError_t launch_fp8_quantize(const QuantizeArgs&, cerar_type_t, cudaStream_t, uint64_t* n) { ++*n; return call("launch", cudaErrorLaunchFailure); }
cudaError_t launch_fp8_matmul(const MatmulArgs&, int, cudaStream_t, uint64_t* n) { ++*n; return call("launch", cudaErrorLaunchFailure); }
int fp8_matmul_tile(int64_t, int64_t, int64_t, bool, int, int* split) { *split = 1; return 128; }
cudaError_t launch_grad_norm(const NormArgs&, int, cudaStream_t, uint64_t* n) { ++*n; return call("launch", cudaErrorLaunchFailure); }
cudaError_t launch_adamw(const AdamwArgs&, int, int, int, int, cudaStream_t, uint64_t* n) { ++*n; return call("launch", cudaErrorLaunchFailure); }
cudaError_t launch_set_grads(TensorRec*, int64_t, int, void* const*, cudaStream_t, uint64_t* n) { ++*n; return call("launch", cudaErrorLaunchFailure); }
}  // namespace cerar
