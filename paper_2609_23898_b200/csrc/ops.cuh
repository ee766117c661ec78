// Launch descriptors of the training-step operators (8-bit products and conversions, gradient norm, AdamW).
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/cerar.h"

namespace cerar {

constexpr int FP8_BLOCK = 128;          // values that share a scale

// Power-of-two scale exponent of the 8-bit format from the bit pattern of a block's largest finite magnitude:
// the smallest e with amax 2^-e <= 448, within [-100, 100]; 0 for a block of zeros.
// amax = f 2^E with f in [0.5, 1): 448 = 0.875 * 2^9, so e = E - 9 if f <= 0.875 (a fraction field up to 0x600000), else E - 8.
__host__ __device__ __forceinline__ int fp8_scale_exponent(uint32_t amax_bits) {
    if (amax_bits == 0u) return 0;
    const int E = (int)(amax_bits >> 23) - 126;
    const int e = ((amax_bits & 0x7FFFFFu) <= 0x600000u) ? E - 9 : E - 8;
    return e < -100 ? -100 : (e > 100 ? 100 : e);      // (a subnormal maximum has E = -126 here: -100 as well)
}

struct QuantizeArgs {
    const void* x;
    int64_t ldx, rows, cols;
    int vec;                             // x can be read four elements at a time
    uint8_t* codes[3];                   // by cerar_scaling_t; null = not wanted
    float* scales[3];
    int64_t ld[3], lds[3];
};
cudaError_t launch_fp8_quantize(const QuantizeArgs& a, cerar_type_t type, cudaStream_t s, uint64_t* launches);

struct MatmulArgs {
    cerar_fp8_matrix_t A, B;
    int trans_a, trans_b;
    void* C;
    int64_t ldc;
    int64_t M, N, K;
    int type, accumulate;
    int* status;
};
cudaError_t launch_fp8_matmul(const MatmulArgs& a, int num_sms, cudaStream_t s, uint64_t* launches);
int fp8_matmul_tile(int64_t M, int64_t N, int64_t K, bool pow2, int num_sms, int* split);

// One tensor of a set as the kernels see it.
struct TensorRec {
    void* param;
    float* master;
    void* grad;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    int64_t numel;
    int64_t block0;                      // first state block of this tensor, counted over the set
    float lr_scale, weight_decay;
    int param_type, grad_type;
    int vec, gvec;                       // all pointers but the gradient's / the gradient's are aligned for four elements at a time
    int unused[2];                       // (a multiple of 16 bytes)
};
__host__ __device__ inline bool grad_vec(const void* p, int type) { return (reinterpret_cast<uintptr_t>(p) & (type == CERAR_TYPE_F32 ? 15u : 7u)) == 0; }
// Work is cut into chunks of up to `steps` times 2048 consecutive elements of one tensor; a list names the tensor and the chunk's
// place inside it, so that a block finds its work with two dependent loads however many tensors there are.
constexpr int CHUNK = 2048;
struct ChunkRef {
    int tensor;
    int index;                           // element offset / CHUNK
};
// Groups of tensors that one optimizer kernel instance serves: parameter kind x gradient type.
enum { PARAM_F32 = 0, PARAM_BF16 = 1, PARAM_MASTER = 2 /* bf16 with a binary32 copy */, PARAM_KINDS = 3 };

struct NormArgs {
    const TensorRec* tensors;
    const ChunkRef* chunks;
    int64_t nchunks;
    int steps;
    double* partial;                     // one per block
    unsigned* ticket;                    // zero between calls
    float max_norm;
    float* clip;
};
cudaError_t launch_grad_norm(const NormArgs& a, int blocks, cudaStream_t s, uint64_t* launches);

struct AdamwArgs {
    const TensorRec* tensors;
    const ChunkRef* chunks;
    int64_t nchunks;
    int steps;
    const float* clip;
    float lr, beta1, beta2, eps;         // and what the host derives from them in binary64:
    float one_minus_beta1, one_minus_beta2, step_size /* lr / (1 - beta1^step) */, root_scale /* (1 - beta2^step)^-1/2 */;
    float minus_zero;                    // -0
    uint64_t seed;
};
cudaError_t launch_adamw(const AdamwArgs& a, int param_kind, int grad_type, int state_bits, int num_sms, cudaStream_t s,
                         uint64_t* launches);
cudaError_t launch_set_grads(TensorRec* tensors, int64_t first, int count, void* const* grads, cudaStream_t s,
                             uint64_t* launches);
constexpr int SET_GRADS_MAX = 256;       // pointers per launch

}  // namespace cerar
