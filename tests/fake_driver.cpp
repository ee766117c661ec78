// The driver's tensor-map encoder as tensor_map.hpp looks it up: slow to find, and refusing a host thread that has made no
// device current, as the driver does.  test_tensor_map_host.py builds this without a device.
#include <atomic>
#include <chrono>
#include <thread>
#include <vector>

#include "tensor_map.hpp"

namespace {
std::atomic<int> g_lookups{0};
thread_local bool t_current = false;

CUresult encode(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
    return t_current ? CUDA_SUCCESS : CUDA_ERROR_INVALID_CONTEXT;
}
}  // namespace

extern "C" {
#undef cudaGetDriverEntryPoint
cudaError_t cudaGetDriverEntryPoint(const char*, void** p, unsigned long long, cudaDriverEntryPointQueryResult* q) {
    ++g_lookups;
    std::this_thread::sleep_for(std::chrono::milliseconds(50));
    *p = reinterpret_cast<void*>(encode);
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaSetDevice(int) { t_current = true; return cudaSuccess; }

// how many of n threads that start together get the encoder
int found_by(int n) {
    std::vector<std::thread> t;
    std::atomic<int> ready{0}, found{0};
    for (int i = 0; i < n; ++i)
        t.emplace_back([&] {
            ++ready;
            while (ready < n) { }
            if (cerar::tc::get_encode_fn()) ++found;
        });
    for (auto& x : t) x.join();
    return found;
}
// a map by a thread whose first call this is
int first_map_of_a_thread() {
    bool ok = false;
    std::thread([&] {
        CUtensorMap m;
        ok = cerar::tc::encode_tiled(&m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2u, (void*)nullptr, (const cuuint64_t*)nullptr, (const cuuint64_t*)nullptr,
                                     (const cuuint32_t*)nullptr, (const cuuint32_t*)nullptr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                     CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    }).join();
    return ok;
}
int lookups() { return g_lookups; }
}
