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
int lookups() { return g_lookups; }
}
