// The handle behind cerar_ops_t, and what the files with C entries on it share: error texts and checks.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>
#include <string>

#include "../../include/cerar.h"

extern "C" void cerar_internal_set_error(const char* msg);    // api.cu: text behind cerar_last_error()

struct cerar_ops {
    int device = -1;
    int num_sms = 0;
    int* d_status = nullptr;                   // 0, STATUS_TIMEOUT or STATUS_BEYOND
    uint64_t launches = 0;
};

namespace cerar {

inline cerar_status_t fail(cerar_status_t s, const char* msg) {
    cerar_internal_set_error(msg);
    return s;
}
inline cerar_status_t cuda_fail(cudaError_t e, const char* what) {
    cudaGetLastError();      // reported here: left where it is, the next check of somebody else's launch would find it
    try {
        cerar_internal_set_error((std::string(what) + ": " + cudaGetErrorString(e)).c_str());
    } catch (...) {
    }
    return e == cudaErrorMemoryAllocation ? CERAR_ERR_NOMEM : CERAR_ERR_CUDA;
}
inline cerar_status_t check_ops(const cerar_ops* o) {
    if (!o) return fail(CERAR_ERR_INVALID_ARG, "ops handle is NULL");
    int dev = -1;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(e, "current device");
    if (dev != o->device)
        return fail(CERAR_ERR_CUDA, "the device the ops handle was created on must be current");
    return CERAR_OK;
}
inline bool type_ok(int t) { return t == CERAR_TYPE_F32 || t == CERAR_TYPE_BF16; }
inline int type_bytes(int t) { return t == CERAR_TYPE_F32 ? 4 : 2; }
inline bool misaligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

}  // namespace cerar
