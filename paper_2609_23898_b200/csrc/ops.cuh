// Launch descriptors of the training-step operators (8-bit products and conversions, gradient norm, AdamW; embedding, head norms,
// bfloat16 products and the gated block made of them).
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/cerar.h"

namespace cerar {

constexpr int FP8_BLOCK = 128;          // values that share a scale

// What kernels leave in a handle's status word.
enum { STATUS_TIMEOUT = 2, STATUS_BEYOND = 3 };

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

struct EmbedArgs {
    const void* table;
    int64_t vocab, width, ld;
    const void* ids;
    int id_bytes;
    int64_t tokens;
    float scale;
    void* y;
    int64_t ldy;
    int type, y_type;
    int* status;
};
cudaError_t launch_embed(const EmbedArgs& a, int num_sms, cudaStream_t s, uint64_t* launches);

struct EmbedGradArgs {
    const void* dy;
    int64_t lddy;
    const void* ids;
    int id_bytes;
    int64_t tokens;
    float scale;
    void* dtable;
    int64_t vocab, width, ld;
    int type, d_type, accumulate;
    void* workspace;
    int* status;
};
size_t embed_grad_workspace(int64_t tokens, int64_t vocab, int64_t width);
cudaError_t launch_embed_grad(const EmbedGradArgs& a, int num_sms, cudaStream_t s, uint64_t* launches);

struct HeadPart {                        // queries or keys
    const void *x, *dy, *w;              // w: null where all are one
    void* y;                             // or dx
    void* dw;
    int64_t x_token, x_head, dy_token, dy_head, y_token, y_head;
    int heads;
};
struct HeadNormArgs {
    HeadPart part[2];
    int count;
    int64_t tokens, period;              // token t has position number t % period
    int dim, rotated, neighbours;
    float eps;
    const float2* table;                 // [table_rows][rotated / 2]: cosine, sine
    int64_t table_rows;
    const void* positions;               // null: the position is the number
    int position_bytes;
    int type, w_type, dw_type, accumulate;
    int* status;
};
constexpr int HEAD_NORM_BLOCKS = 1024;   // of each part, at most, in the gradient
size_t head_norm_grad_workspace(int count, int dim);
cudaError_t launch_head_norm(const HeadNormArgs& a, int num_sms, cudaStream_t s, uint64_t* launches);
cudaError_t launch_head_norm_grad(const HeadNormArgs& a, void* workspace, int num_sms, cudaStream_t s, uint64_t* launches);
cudaError_t launch_rotation_table(const double* freqs, int pairs, int64_t first, int64_t rows, float* table, int num_sms, cudaStream_t s, uint64_t* launches);


// C = op(A) op(B) of bfloat16 matrices; rows on 16-byte boundaries, M, N, K above zero
struct Matmul16Args {
    const void *A, *B;
    int64_t lda, ldb;
    bool trans_a, trans_b;
    int64_t M, N, K;
    void* C;
    int64_t ldc;
    int type, accumulate;
    int* status;
    // after: the kernel in front is a product with `followed` that this one has nothing to do with, and what this one needs was complete before that
    // one began; it may run beside that one's last blocks and waits for it at its own end
    int after, followed;
};
cudaError_t launch_matmul16(const Matmul16Args& a, int num_sms, cudaStream_t s, uint64_t* launches);
int matmul16_tile(int64_t M, int64_t N, int64_t K, int num_sms, int* split);
struct AlignArgs {                       // a bfloat16 matrix whose rows are copied to rows on 16-byte boundaries
    const void* src;
    void* dst;
    int64_t rows, cols, ld, ldd;
};
constexpr int ALIGN_MAX = 4;
cudaError_t launch_align(const AlignArgs* items, int count, cudaStream_t s, uint64_t* launches);
struct GatedInArgs {
    const void *x, *w;
    int64_t ldx, ldw;
    int64_t tokens, width, hidden;
    int act;
    void *h, *kept;                      // kept: null where nothing is
    int64_t ldh;
    int* status;
};
cudaError_t launch_gated_in(const GatedInArgs& a, int num_sms, cudaStream_t s, uint64_t* launches);
struct GatedGradArgs {
    const void *dy, *w, *kept;
    int64_t lddy, ldw;
    int64_t tokens, width, hidden;
    int act;
    void *dgu, *h;                       // h: null where it is not wanted
    int64_t lddgu, ldh;
    int* status;
};
size_t gated_kept_bytes(int64_t tokens, int64_t hidden);
cudaError_t launch_gated_grad(const GatedGradArgs& a, int num_sms, cudaStream_t s, uint64_t* launches);

}  // namespace cerar
