// C ABI of the training-step operators: handles, argument checks, launches.
#include <cuda_runtime.h>

#include <cmath>
#include <new>
#include <string>
#include <vector>

#include "../../include/cerar.h"
#include "ops.cuh"
#include "ops_handle.hpp"

using cerar::check_ops;
using cerar::cuda_fail;
using cerar::fail;
using cerar::misaligned;
using cerar::type_bytes;
using cerar::type_ok;

struct cerar_tensors {
    cerar_ops* ops = nullptr;
    int64_t count = 0;
    int state_bits = 0;
    int64_t nchunks = 0;
    int steps = 1;                             // a chunk has up to steps * CHUNK elements
    cerar::TensorRec* d_tensors = nullptr;
    cerar::ChunkRef* d_chunks = nullptr;       // grouped by (parameter kind, gradient type)
    double* d_partial = nullptr;
    unsigned* d_ticket = nullptr;
    int norm_blocks = 0;
    std::vector<int64_t> numel;                // host copies for the checks of set_grads
    std::vector<int> grad_type;
    struct Group { int kind, grad_type; int64_t first, nchunks; };
    std::vector<Group> groups;
};

namespace {

cerar_status_t check_matrix(const cerar_fp8_matrix_t* m) {
    if (!m) return fail(CERAR_ERR_INVALID_ARG, "8-bit matrix is NULL");
    if (m->scaling < CERAR_BY_ROW || m->scaling > CERAR_BY_BLOCK) return fail(CERAR_ERR_INVALID_ARG, "8-bit matrix: unknown scaling");
    if (m->rows < 0 || m->cols < 0) return fail(CERAR_ERR_SHAPE, "8-bit matrix: negative size");
    if (m->rows > 0x7FFFFF00 || m->cols > 0x7FFFFF00) return fail(CERAR_ERR_SHAPE, "8-bit matrix: sizes are limited to 2^31 - 256");
    if (m->rows == 0 || m->cols == 0) return CERAR_OK;
    if (!m->codes || !m->scales) return fail(CERAR_ERR_INVALID_ARG, "8-bit matrix: codes or scales are NULL");
    if (misaligned(m->codes, 16)) return fail(CERAR_ERR_INVALID_ARG, "8-bit matrix: codes must start on a 16-byte boundary");
    if (misaligned(m->scales, 4)) return fail(CERAR_ERR_INVALID_ARG, "8-bit matrix: scales must be aligned to 4 bytes");
    if (m->ld < m->cols || m->ld % 16) return fail(CERAR_ERR_SHAPE, "8-bit matrix: ld must be a multiple of 16 and at least cols");
    if (m->ld >= (int64_t)1 << 40) return fail(CERAR_ERR_SHAPE, "8-bit matrix: ld is limited to 2^40 bytes");
    const int64_t per = m->scaling == CERAR_BY_ROW ? m->rows : m->scaling == CERAR_BY_COLUMN ? m->cols : (m->cols + 127) / 128;
    if (m->lds < per) return fail(CERAR_ERR_SHAPE, "8-bit matrix: lds is too small for this scaling");
    return CERAR_OK;
}

// What was copied or set on the legacy stream is on the device when this returns.  cudaMemcpy from pageable memory and cudaMemset may
// return earlier, and the caller's streams need not wait for that one (torch's do not).
cudaError_t set_up_done() { return cudaStreamSynchronize(cudaStreamLegacy); }

}  // namespace

extern "C" {

cerar_status_t cerar_ops_create(cerar_ops_t** out) {
    if (!out) return fail(CERAR_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    int count = 0;
    cudaError_t e = cudaGetDeviceCount(&count);
    if (e != cudaSuccess || count == 0) {
        cudaGetLastError();
        return fail(CERAR_ERR_CUDA, "no CUDA device");
    }
    cerar_ops* o = new (std::nothrow) cerar_ops;
    if (!o) return fail(CERAR_ERR_NOMEM, "out of host memory");
    if ((e = cudaGetDevice(&o->device)) == cudaSuccess &&
        (e = cudaDeviceGetAttribute(&o->num_sms, cudaDevAttrMultiProcessorCount, o->device)) == cudaSuccess &&
        (e = cudaMalloc(&o->d_status, sizeof(int))) == cudaSuccess &&
        (e = cudaMemset(o->d_status, 0, sizeof(int))) == cudaSuccess)
        e = set_up_done();
    if (e != cudaSuccess) {
        const cerar_status_t st = cuda_fail(e, "ops set-up");
        cerar_ops_destroy(o);
        return st;
    }
    *out = o;
    return CERAR_OK;
}

void cerar_ops_destroy(cerar_ops_t* o) {
    if (!o) return;
    if (o->d_status) cudaFree(o->d_status);
    delete o;
}

cerar_status_t cerar_ops_status(cerar_ops_t* o, cerar_stream_t stream) {
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    int flag = 0;
    cudaError_t e = cudaMemcpyAsync(&flag, o->d_status, sizeof(int), cudaMemcpyDeviceToHost, (cudaStream_t)stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_fail(e, "status read");
    if (flag == 0) return CERAR_OK;
    cudaMemsetAsync(o->d_status, 0, sizeof(int), (cudaStream_t)stream);
    if (flag == cerar::STATUS_BEYOND) return fail(CERAR_ERR_BOUNDS, "a token or a position beyond the end of its table");
    return fail(CERAR_ERR_TIMEOUT, "a kernel gave up on a bounded wait");
}

uint64_t cerar_ops_launch_count(const cerar_ops_t* o) { return o ? o->launches : 0; }

cerar_status_t cerar_fp8_quantize(cerar_ops_t* o, const void* x, cerar_type_t type, int64_t ldx, const cerar_fp8_matrix_t* out,
                                  int count, cerar_stream_t stream) {
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    if (!type_ok(type)) return fail(CERAR_ERR_INVALID_ARG, "unknown element type");
    if (!out || count < 1 || count > 3) return fail(CERAR_ERR_INVALID_ARG, "1 to 3 output matrices are wanted");
    cerar::QuantizeArgs a = {};
    a.x = x; a.ldx = ldx; a.rows = out[0].rows; a.cols = out[0].cols;
    for (int i = 0; i < count; ++i) {
        if ((st = check_matrix(out + i)) != CERAR_OK) return st;
        if (out[i].rows != a.rows || out[i].cols != a.cols) return fail(CERAR_ERR_SHAPE, "output matrices of different sizes");
        const int f = out[i].scaling;
        if (a.codes[f]) return fail(CERAR_ERR_INVALID_ARG, "two output matrices with the same scaling");
        a.codes[f] = out[i].codes; a.scales[f] = out[i].scales; a.ld[f] = out[i].ld; a.lds[f] = out[i].lds;
    }
    if (a.rows == 0 || a.cols == 0) return CERAR_OK;
    if (!x) return fail(CERAR_ERR_INVALID_ARG, "x is NULL");
    if (ldx < a.cols) return fail(CERAR_ERR_SHAPE, "ldx must be at least the number of columns");
    if (misaligned(x, type_bytes(type))) return fail(CERAR_ERR_INVALID_ARG, "x is not aligned to its elements");
    a.vec = !misaligned(x, 4 * type_bytes(type)) && ldx % 4 == 0;
    const cudaError_t e = cerar::launch_fp8_quantize(a, type, (cudaStream_t)stream, &o->launches);
    return e == cudaSuccess ? CERAR_OK : cuda_fail(e, "fp8 quantize launch");
}

cerar_status_t cerar_fp8_matmul(cerar_ops_t* o, const cerar_fp8_matrix_t* A, int trans_a, const cerar_fp8_matrix_t* B, int trans_b,
                                void* C, cerar_type_t type, int64_t ldc, int accumulate, cerar_stream_t stream) {
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    if (!type_ok(type)) return fail(CERAR_ERR_INVALID_ARG, "unknown element type");
    if ((st = check_matrix(A)) != CERAR_OK || (st = check_matrix(B)) != CERAR_OK) return st;
    cerar::MatmulArgs a = {};
    a.A = *A; a.B = *B; a.trans_a = trans_a != 0; a.trans_b = trans_b != 0;
    a.M = trans_a ? A->cols : A->rows; a.K = trans_a ? A->rows : A->cols;
    a.N = trans_b ? B->rows : B->cols;
    if ((trans_b ? B->cols : B->rows) != a.K) return fail(CERAR_ERR_SHAPE, "the summed dimensions of A and B differ");
    if (A->scaling != CERAR_BY_BLOCK && A->scaling != (trans_a ? CERAR_BY_COLUMN : CERAR_BY_ROW))
        return fail(CERAR_ERR_INVALID_ARG, "A must be scaled along the summed dimension (by row, transposed by column) or by block");
    if (B->scaling != CERAR_BY_BLOCK && B->scaling != (trans_b ? CERAR_BY_ROW : CERAR_BY_COLUMN))
        return fail(CERAR_ERR_INVALID_ARG, "B must be scaled along the summed dimension (by column, transposed by row) or by block");
    if (a.M == 0 || a.N == 0) return CERAR_OK;
    if (!C) return fail(CERAR_ERR_INVALID_ARG, "C is NULL");
    if (misaligned(C, type_bytes(type))) return fail(CERAR_ERR_INVALID_ARG, "C is not aligned to its elements");
    if (ldc < a.N) return fail(CERAR_ERR_SHAPE, "ldc must be at least the number of columns of C");
    a.C = C; a.ldc = ldc; a.type = type; a.accumulate = accumulate != 0; a.status = o->d_status;
    cudaError_t e = cudaSuccess;
    if (a.K == 0) {                       // an empty sum
        if (!a.accumulate)
            e = cudaMemset2DAsync(C, (size_t)ldc * type_bytes(type), 0, (size_t)a.N * type_bytes(type), (size_t)a.M, (cudaStream_t)stream);
    } else {
        e = cerar::launch_fp8_matmul(a, o->num_sms, (cudaStream_t)stream, &o->launches);
    }
    return e == cudaSuccess ? CERAR_OK : cuda_fail(e, "fp8 matmul launch");
}

int cerar_fp8_matmul_tile(int64_t M, int64_t N, int64_t K, int pow2, int num_sms, int* split) {
    if (M < 1 || N < 1 || K < 1 || M > 0x7FFFFF00 || N > 0x7FFFFF00 || K > 0x7FFFFF00 || num_sms < 1 || !split) return -1;
    return cerar::fp8_matmul_tile(M, N, K, pow2 != 0, num_sms, split);
}

cerar_status_t cerar_tensors_create(cerar_ops_t* o, int64_t count, const cerar_tensor_t* tensors, int state_bits,
                                    cerar_tensors_t** out) {
    if (!out) return fail(CERAR_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    if (count < 0 || count > 0x7FFFFFFF || (count > 0 && !tensors)) return fail(CERAR_ERR_INVALID_ARG, "bad tensor list");
    if (state_bits != 0 && state_bits != 8 && state_bits != 32) return fail(CERAR_ERR_INVALID_ARG, "state_bits must be 0, 8 or 32");
    for (int64_t i = 0; i < count; ++i) {
        const cerar_tensor_t& t = tensors[i];
        if (t.numel < 0 || t.numel >= (int64_t)1 << 40) return fail(CERAR_ERR_SHAPE, "tensor with a negative or too large size");
        if (!type_ok(t.grad_type) || (state_bits && !type_ok(t.param_type))) return fail(CERAR_ERR_INVALID_ARG, "tensor of unknown type");
        if (t.numel == 0) continue;
        if (!t.grad || misaligned(t.grad, type_bytes(t.grad_type))) return fail(CERAR_ERR_INVALID_ARG, "gradient NULL or not aligned to its elements");
        if (!state_bits) continue;
        if (!t.param || misaligned(t.param, type_bytes(t.param_type))) return fail(CERAR_ERR_INVALID_ARG, "parameter NULL or not aligned to its elements");
        if (t.master && t.param_type != CERAR_TYPE_BF16) return fail(CERAR_ERR_INVALID_ARG, "a master copy belongs to a bfloat16 parameter");
        if (misaligned(t.master, 4)) return fail(CERAR_ERR_INVALID_ARG, "master copy not aligned to its elements");
        const uintptr_t sa = state_bits == 32 ? 4 : 1;
        if (!t.m || !t.v || misaligned(t.m, sa) || misaligned(t.v, sa)) return fail(CERAR_ERR_INVALID_ARG, "state NULL or not aligned to its elements");
        if (state_bits == 8 && (!t.m_scale || !t.v_scale || misaligned(t.m_scale, 4) || misaligned(t.v_scale, 4)))
            return fail(CERAR_ERR_INVALID_ARG, "8-bit states need scales aligned to 4 bytes");
        if (!std::isfinite(t.lr_scale) || !std::isfinite(t.weight_decay)) return fail(CERAR_ERR_INVALID_ARG, "lr_scale or weight_decay is not finite");
    }
    cerar_tensors* set = new (std::nothrow) cerar_tensors;
    if (!set) return fail(CERAR_ERR_NOMEM, "out of host memory");
    cudaError_t e = cudaSuccess;
    try {
        std::vector<cerar::TensorRec> recs((size_t)count);
        std::vector<cerar::ChunkRef> chunks;
        int64_t block = 0, total = 0;
        bool plain_bf16 = false;
        for (int64_t i = 0; i < count; ++i) {
            total += tensors[i].numel;
            plain_bf16 = plain_bf16 || (state_bits && tensors[i].param_type == CERAR_TYPE_BF16 && !tensors[i].master);
        }
        // Long chunks where there are many (16 per SM): memory serves longer runs better (32-bit states 6.1 -> 6.4 TB/s).  Sets with
        // 8-bit states, whose step is bound by its instructions and short of registers, keep short ones (4.6 against 5.0 TB/s), and so do
        // sets with bfloat16 parameters without master copies (6.4 against 6.65).
        set->steps = state_bits != 8 && !plain_bf16 && total >= (int64_t)o->num_sms * 16 * 4 * cerar::CHUNK ? 4 : 1;
        for (int64_t i = 0; i < count; ++i) {
            const cerar_tensor_t& t = tensors[i];
            recs[i] = cerar::TensorRec{t.param, t.master, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.numel, block, t.lr_scale, t.weight_decay,
                                       t.param_type, t.grad_type, 0, cerar::grad_vec(t.grad, t.grad_type) ? 1 : 0, {0, 0}};
            const uintptr_t sa = state_bits == 32 ? 16 : 4;
            recs[i].vec = !misaligned(t.m, sa) && !misaligned(t.v, sa) && !misaligned(t.master, 16) &&
                          !misaligned(t.param, t.param_type == CERAR_TYPE_F32 ? 16 : 8);
            block += (t.numel + CERAR_STATE_BLOCK - 1) / CERAR_STATE_BLOCK;
            set->numel.push_back(t.numel);
            set->grad_type.push_back(t.grad_type);
        }
        for (int kind = 0; kind < cerar::PARAM_KINDS; ++kind)
            for (int gt = 0; gt < 2; ++gt) {
                const size_t first = chunks.size();
                for (int64_t i = 0; i < count; ++i) {
                    const cerar_tensor_t& t = tensors[i];
                    const int k = !state_bits || t.param_type == CERAR_TYPE_F32 ? cerar::PARAM_F32 : t.master ? cerar::PARAM_MASTER : cerar::PARAM_BF16;
                    if (k != kind || t.grad_type != gt) continue;
                    for (int64_t c = 0; c * cerar::CHUNK < t.numel; c += set->steps) chunks.push_back(cerar::ChunkRef{(int)i, (int)c});
                }
                if (chunks.size() > first) set->groups.push_back({kind, gt, (int64_t)first, (int64_t)(chunks.size() - first)});
            }
        set->ops = o; set->count = count; set->state_bits = state_bits; set->nchunks = (int64_t)chunks.size();
        const int64_t most = (int64_t)o->num_sms * 8;
        set->norm_blocks = (int)(set->nchunks < 1 ? 1 : set->nchunks < most ? set->nchunks : most);
        if ((e = cudaMalloc(&set->d_tensors, sizeof(cerar::TensorRec) * (recs.size() + 1))) == cudaSuccess &&
            (e = cudaMalloc(&set->d_chunks, sizeof(cerar::ChunkRef) * (chunks.size() + 1))) == cudaSuccess &&
            (e = cudaMalloc(&set->d_partial, sizeof(double) * set->norm_blocks)) == cudaSuccess &&
            (e = cudaMalloc(&set->d_ticket, sizeof(unsigned))) == cudaSuccess &&
            (e = cudaMemset(set->d_ticket, 0, sizeof(unsigned))) == cudaSuccess &&
            (e = cudaMemcpy(set->d_tensors, recs.data(), sizeof(cerar::TensorRec) * recs.size(), cudaMemcpyHostToDevice)) == cudaSuccess &&
            (e = cudaMemcpy(set->d_chunks, chunks.data(), sizeof(cerar::ChunkRef) * chunks.size(), cudaMemcpyHostToDevice)) == cudaSuccess)
            e = set_up_done();
    } catch (const std::bad_alloc&) {
        cerar_tensors_destroy(set);
        return fail(CERAR_ERR_NOMEM, "out of host memory");
    }
    if (e != cudaSuccess) {
        st = cuda_fail(e, "tensor set");
        cerar_tensors_destroy(set);
        return st;
    }
    *out = set;
    return CERAR_OK;
}

void cerar_tensors_destroy(cerar_tensors_t* set) {
    if (!set) return;
    cudaFree(set->d_tensors);
    cudaFree(set->d_chunks);
    cudaFree(set->d_partial);
    cudaFree(set->d_ticket);
    delete set;
}

cerar_status_t cerar_tensors_set_grads(cerar_tensors_t* set, void* const* grads, cerar_stream_t stream) {
    if (!set) return fail(CERAR_ERR_INVALID_ARG, "tensor set is NULL");
    cerar_status_t st = check_ops(set->ops);
    if (st != CERAR_OK) return st;
    if (set->count > 0 && !grads) return fail(CERAR_ERR_INVALID_ARG, "grads is NULL");
    for (int64_t i = 0; i < set->count; ++i)
        if (set->numel[i] && (!grads[i] || misaligned(grads[i], type_bytes(set->grad_type[i]))))
            return fail(CERAR_ERR_INVALID_ARG, "gradient NULL or not aligned to its elements");
    for (int64_t i = 0; i < set->count; i += cerar::SET_GRADS_MAX) {
        const int n = (int)(set->count - i < cerar::SET_GRADS_MAX ? set->count - i : cerar::SET_GRADS_MAX);
        const cudaError_t e = cerar::launch_set_grads(set->d_tensors, i, n, grads + i, (cudaStream_t)stream, &set->ops->launches);
        if (e != cudaSuccess) return cuda_fail(e, "set_grads launch");
    }
    return CERAR_OK;
}

cerar_status_t cerar_grad_norm(cerar_tensors_t* set, float max_norm, float* clip, cerar_stream_t stream) {
    if (!set) return fail(CERAR_ERR_INVALID_ARG, "tensor set is NULL");
    cerar_status_t st = check_ops(set->ops);
    if (st != CERAR_OK) return st;
    if (!clip || misaligned(clip, 4)) return fail(CERAR_ERR_INVALID_ARG, "clip must be three floats of device memory");
    if (std::isnan(max_norm)) return fail(CERAR_ERR_INVALID_ARG, "max_norm is NaN");
    cerar::NormArgs a = {set->d_tensors, set->d_chunks, set->nchunks, set->steps, set->d_partial, set->d_ticket, max_norm, clip};
    const cudaError_t e = cerar::launch_grad_norm(a, set->norm_blocks, (cudaStream_t)stream, &set->ops->launches);
    return e == cudaSuccess ? CERAR_OK : cuda_fail(e, "grad norm launch");
}

cerar_status_t cerar_adamw_step(cerar_tensors_t* set, const cerar_adamw_options_t* opt, const float* clip, cerar_stream_t stream) {
    if (!set || !opt) return fail(CERAR_ERR_INVALID_ARG, "tensor set or options are NULL");
    cerar_status_t st = check_ops(set->ops);
    if (st != CERAR_OK) return st;
    if (!set->state_bits) return fail(CERAR_ERR_STATE, "the set was created without optimizer states");
    if (misaligned(clip, 4)) return fail(CERAR_ERR_INVALID_ARG, "clip is not aligned to its elements");
    if (!std::isfinite(opt->lr) || !(opt->beta1 >= 0.0 && opt->beta1 < 1.0) || !(opt->beta2 >= 0.0 && opt->beta2 < 1.0) ||
        !(opt->eps >= 0.0 && std::isfinite(opt->eps)) || opt->step < 1)
        return fail(CERAR_ERR_INVALID_ARG, "AdamW wants a finite lr, betas in [0, 1), a finite eps >= 0 and a step from 1 on");
    cerar::AdamwArgs a = {};
    a.tensors = set->d_tensors; a.steps = set->steps; a.clip = clip;
    a.minus_zero = -0.f;
    a.lr = (float)opt->lr; a.beta1 = (float)opt->beta1; a.beta2 = (float)opt->beta2; a.eps = (float)opt->eps; a.seed = opt->seed;
    a.one_minus_beta1 = (float)(1.0 - opt->beta1);
    a.one_minus_beta2 = (float)(1.0 - opt->beta2);
    a.step_size = (float)(opt->lr / (1.0 - std::pow(opt->beta1, (double)opt->step)));
    a.root_scale = (float)(1.0 / std::sqrt(1.0 - std::pow(opt->beta2, (double)opt->step)));
    for (const auto& g : set->groups) {
        a.chunks = set->d_chunks + g.first;
        a.nchunks = g.nchunks;
        const cudaError_t e = cerar::launch_adamw(a, g.kind, g.grad_type, set->state_bits, set->ops->num_sms, (cudaStream_t)stream, &set->ops->launches);
        if (e != cudaSuccess) return cuda_fail(e, "AdamW launch");
    }
    return CERAR_OK;
}

}  // extern "C"
