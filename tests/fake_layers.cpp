// The launches of the layers' operators, written down beside fake_cuda.cpp's functions: layers_api.cu's host side without a device.
#include <cuda_runtime.h>

#include <string>

#include "ops.cuh"

extern "C" {
void fake_reset(const char*);
const char* fake_log();
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t);
}

namespace {
std::string g_launches;
int g_fail = 0;
cudaError_t launch(const char* name, uint64_t* n) {
    g_launches += name;
    g_launches += '\n';
    ++*n;
    return g_fail ? cudaErrorLaunchFailure : cudaSuccess;
}
}  // namespace

extern "C" {
const char* fake_launches() { return g_launches.c_str(); }
void fake_launches_reset(int fail) { g_launches.clear(); g_fail = fail; }
}

namespace cerar {
cudaError_t launch_embed(const EmbedArgs&, int, cudaStream_t, uint64_t* n) { return launch("embed", n); }
size_t embed_grad_workspace(int64_t tokens, int64_t, int64_t) { return tokens ? 1024 : 0; }
cudaError_t launch_embed_grad(const EmbedGradArgs&, int, cudaStream_t, uint64_t* n) { return launch("embed_grad", n); }
size_t head_norm_grad_workspace(int count, int dim) { return (size_t)count * dim * 4; }
cudaError_t launch_head_norm(const HeadNormArgs&, int, cudaStream_t, uint64_t* n) { return launch("head_norm", n); }
cudaError_t launch_head_norm_grad(const HeadNormArgs&, void*, int, cudaStream_t, uint64_t* n) { return launch("head_norm_grad", n); }
cudaError_t launch_rotation_table(const double*, int, int64_t, int64_t, float*, int, cudaStream_t, uint64_t* n) { return launch("rotation", n); }
cudaError_t launch_matmul16(const Matmul16Args&, int, cudaStream_t, uint64_t* n) { return launch("matmul", n); }
int matmul16_tile(int64_t, int64_t, int64_t, int, int* split) { *split = 1; return 0; }
cudaError_t launch_align(const AlignArgs*, int, cudaStream_t, uint64_t* n) { return launch("align", n); }
cudaError_t launch_gated_in(const GatedInArgs&, int, cudaStream_t, uint64_t* n) { return launch("gated_in", n); }
cudaError_t launch_gated_grad(const GatedGradArgs&, int, cudaStream_t, uint64_t* n) { return launch("gated_grad", n); }
size_t gated_kept_bytes(int64_t tokens, int64_t hidden) { return (size_t)(tokens * hidden * 6); }
}  // namespace cerar
