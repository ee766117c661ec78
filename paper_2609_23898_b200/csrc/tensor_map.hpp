// Host side of tensor maps: the driver's encoder, looked up at run time (the library does not link the driver).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

namespace cerar {
namespace tc {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// (Looked up once, by whichever host thread comes first; others that come meanwhile wait for it.)
inline EncodeTiledFn get_encode_fn() {
    static const EncodeTiledFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        const bool found = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
                           q == cudaDriverEntryPointSuccess;
        return found ? reinterpret_cast<EncodeTiledFn>(p) : nullptr;
    }();
    return fn;
}

// One map.  The encoder wants a current context, which a host thread does not have before its first call of the runtime that needs
// one; only there, it is tried again with the thread's device made current.
template <typename... Args>
inline bool encode_tiled(Args... args) {
    const EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    if (fn(args...) == CUDA_SUCCESS) return true;
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && cudaSetDevice(dev) == cudaSuccess && fn(args...) == CUDA_SUCCESS;
}

}  // namespace tc
}  // namespace cerar
