// C ABI of the layers' operators (embedding, head norms, bfloat16 products, gated block): argument checks, launches.
#include <cuda_runtime.h>

#include <cmath>

#include "../../include/cerar.h"
#include "ops.cuh"
#include "ops_handle.hpp"

using cerar::check_ops;
using cerar::cuda_fail;
using cerar::fail;
using cerar::misaligned;
using cerar::type_bytes;
using cerar::type_ok;

namespace {

constexpr int64_t TOKENS_MAX = 0x7FFFFF00, SIZE_MAX_ = 0x7FFFFF00, LD_MAX = (int64_t)1 << 40;

cerar_status_t check_ids(const void* ids, int id_bytes, int64_t tokens, int64_t vocab, int64_t width) {
    if (id_bytes != 4 && id_bytes != 8) return fail(CERAR_ERR_INVALID_ARG, "ids of 4 or 8 bytes are wanted");
    if (tokens < 0 || tokens > TOKENS_MAX || vocab < 0 || vocab > SIZE_MAX_ || width < 0 || width > SIZE_MAX_)
        return fail(CERAR_ERR_SHAPE, "embedding: negative sizes, or above 2^31 - 256");
    if (tokens > 0 && (!ids || misaligned(ids, (uintptr_t)id_bytes))) return fail(CERAR_ERR_INVALID_ARG, "ids NULL or not aligned to their elements");
    return CERAR_OK;
}
// rows x width of `type`, ld elements between rows
cerar_status_t check_rows(const void* p, int type, int64_t rows, int64_t width, int64_t ld, const char* null_text) {
    if (!type_ok(type)) return fail(CERAR_ERR_INVALID_ARG, "unknown element type");
    if (rows == 0 || width == 0) return CERAR_OK;
    if (!p || misaligned(p, type_bytes(type))) return fail(CERAR_ERR_INVALID_ARG, null_text);
    if (rows > 1 && (ld < width || ld > LD_MAX)) return fail(CERAR_ERR_SHAPE, "rows overlap, or lie more than 2^40 elements apart");
    return CERAR_OK;
}

cerar_status_t check_heads(const cerar_heads_t* parts, int count, cerar_type_t type, int64_t tokens, int dim, bool grad, cerar::HeadNormArgs& a) {
    if (!type_ok(type)) return fail(CERAR_ERR_INVALID_ARG, "unknown element type");
    if (!parts || count < 1 || count > 2) return fail(CERAR_ERR_INVALID_ARG, "1 or 2 groups of heads are wanted");
    if (tokens < 0 || tokens > TOKENS_MAX) return fail(CERAR_ERR_SHAPE, "a negative number of tokens, or above 2^31 - 256");
    if (dim < 2 || dim > CERAR_HEAD_DIM_MAX || dim % 2) return fail(CERAR_ERR_SHAPE, "the values of a head must be an even number from 2 to 512");
    a.count = count; a.tokens = tokens; a.dim = dim; a.type = type;
    for (int i = 0; i < count; ++i) {
        const cerar_heads_t& h = parts[i];
        if (h.heads < 0 || h.heads > 0xFFFF) return fail(CERAR_ERR_SHAPE, "a negative number of heads, or above 65535");
        auto rows_ok = [&](const void* p, int64_t token, int64_t head) {
            if (!p || misaligned(p, type_bytes(type))) return false;
            return token > -LD_MAX && token < LD_MAX && head > -LD_MAX && head < LD_MAX;
        };
        // written rows: no two of them may lie over one another
        auto apart = [&](int64_t token, int64_t head) {
            const int64_t t = token < 0 ? -token : token, d = head < 0 ? -head : head;
            if (h.heads < 2) return tokens < 2 || t >= dim;
            if (tokens < 2) return d >= dim;
            return (d >= dim && t >= d * (h.heads - 1) + dim) || (t >= dim && d >= t * (tokens - 1) + dim);
        };
        if (tokens > 0 && h.heads > 0) {
            if (!rows_ok(h.x, h.x_token, h.x_head) || !rows_ok(h.y, h.y_token, h.y_head) || (grad && !rows_ok(h.dy, h.dy_token, h.dy_head)))
                return fail(CERAR_ERR_INVALID_ARG, "heads: a pointer is NULL or not aligned to its elements, or strides are above 2^40");
            if (!apart(h.y_token, h.y_head)) return fail(CERAR_ERR_SHAPE, "heads: rows that are written overlap");
        }
        cerar::HeadPart& p = a.part[i];
        p = {h.x, h.dy, h.w, h.y, grad ? h.dw : nullptr, h.x_token, h.x_head, h.dy_token, h.dy_head, h.y_token, h.y_head, (int)h.heads};
    }
    return CERAR_OK;
}
cerar_status_t check_rotation(const cerar_rotation_t* r, int dim, cerar::HeadNormArgs& a) {
    if (!r) return fail(CERAR_ERR_INVALID_ARG, "rotation is NULL");
    if (r->rotated < 0 || r->rotated > dim || r->rotated % 2) return fail(CERAR_ERR_SHAPE, "the values that are turned must be an even number up to the head's");
    if (r->period < 1) return fail(CERAR_ERR_SHAPE, "period must be at least 1");
    if (r->rows < 0 || (r->rotated > 0 && (!r->table || misaligned(r->table, 8)))) return fail(CERAR_ERR_INVALID_ARG, "rotation table NULL, not aligned to 8 bytes, or of a negative length");
    if (r->positions && ((r->position_bytes != 4 && r->position_bytes != 8) || misaligned(r->positions, (uintptr_t)r->position_bytes)))
        return fail(CERAR_ERR_INVALID_ARG, "positions of 4 or 8 bytes, aligned, are wanted");
    a.rotated = r->rotated; a.neighbours = r->neighbours != 0; a.period = r->period;
    a.table = reinterpret_cast<const float2*>(r->table);
    a.table_rows = r->rotated > 0 ? r->rows : (int64_t)1 << 62;          // (nothing is looked up: any position will do)
    a.positions = r->positions; a.position_bytes = r->position_bytes;
    return CERAR_OK;
}

// A bfloat16 operand of a product: rows x cols, read by tensor-map copies
cerar_status_t check_operand(const void* p, int64_t rows, int64_t cols, int64_t ld) {
    if (rows < 0 || cols < 0 || rows > SIZE_MAX_ || cols > SIZE_MAX_) return fail(CERAR_ERR_SHAPE, "matrix: sizes from 0 to 2^31 - 256 are wanted");
    if (rows == 0 || cols == 0) return CERAR_OK;
    if (!p || misaligned(p, 16)) return fail(CERAR_ERR_INVALID_ARG, "matrix: NULL, or not on a 16-byte boundary");
    if (ld < cols || ld % 8 || ld >= (int64_t)1 << 39) return fail(CERAR_ERR_SHAPE, "matrix: ld must be a multiple of 8, at least the number of columns and below 2^39");
    return CERAR_OK;
}

// ---- the gated block: its operands as the products read them, and what it makes on the way, in one workspace

struct Mat {                                                 // rows of bfloat16, 16-byte aligned
    void* p;
    int64_t ld;
};
struct Block {
    Mat x, w_in, w_out, dy, h, dgu;
    cerar::AlignArgs copies[cerar::ALIGN_MAX];
    int count;
    int64_t bytes;
};
cerar_status_t check_gated(const cerar_gated_t& g, bool backward) {
    if (g.tokens < 0 || g.tokens > TOKENS_MAX || g.width < 0 || g.width > SIZE_MAX_ || g.outputs < 0 || g.outputs > SIZE_MAX_ || g.hidden < 0 || g.hidden > SIZE_MAX_ / 2)
        return fail(CERAR_ERR_SHAPE, "gated block: negative sizes, above 2^31 - 256, or hidden above 2^30 - 128");
    if (g.activation < CERAR_ACT_SILU || g.activation > CERAR_ACT_RELU) return fail(CERAR_ERR_INVALID_ARG, "unknown activation");
    cerar_status_t st;
    const bool x = !backward || g.dw_in, w_in = !backward || g.dx;
    if ((x && (st = check_rows(g.x, CERAR_TYPE_BF16, g.tokens, g.width, g.ldx, "x NULL or not aligned to its elements")) != CERAR_OK) ||
        (w_in && (st = check_rows(g.w_in, CERAR_TYPE_BF16, 2 * g.hidden, g.width, g.ldw_in, "w_in NULL or not aligned to its elements")) != CERAR_OK) ||
        (st = check_rows(g.w_out, CERAR_TYPE_BF16, g.outputs, g.hidden, g.ldw_out, "w_out NULL or not aligned to its elements")) != CERAR_OK)
        return st;
    if (misaligned(g.kept, 16) || (backward && !g.kept && g.tokens > 0 && g.hidden > 0 && g.outputs > 0))
        return fail(CERAR_ERR_INVALID_ARG, "kept NULL where it is needed, or not on a 16-byte boundary");
    if (!backward) return check_rows(g.y, CERAR_TYPE_BF16, g.tokens, g.outputs, g.ldy, "y NULL or not aligned to its elements");
    if ((st = check_rows(g.dy, CERAR_TYPE_BF16, g.tokens, g.outputs, g.lddy, "dy NULL or not aligned to its elements")) != CERAR_OK ||
        (g.dx && (st = check_rows(g.dx, CERAR_TYPE_BF16, g.tokens, g.width, g.lddx, "dx not aligned to its elements")) != CERAR_OK) ||
        (g.dw_in && (st = check_rows(g.dw_in, (int)g.dw_in_type, 2 * g.hidden, g.width, g.lddw_in, "dw_in not aligned to its elements")) != CERAR_OK) ||
        (g.dw_out && (st = check_rows(g.dw_out, (int)g.dw_out_type, g.outputs, g.hidden, g.lddw_out, "dw_out not aligned to its elements")) != CERAR_OK))
        return st;
    return CERAR_OK;
}
// false: the workspace would have more than 2^62 bytes
bool lay_out(const cerar_gated_t& g, bool backward, void* workspace, Block& b) {
    b = {};
    unsigned char* at = static_cast<unsigned char*>(workspace);
    bool fits = true;
    auto take = [&](int64_t rows, int64_t cols, Mat& m) {
        m.ld = (cols + 7) & ~(int64_t)7;
        const __int128 size = (__int128)rows * m.ld * 2 + 255;
        if (b.bytes + size > (__int128)1 << 62) { fits = false; return; }
        m.p = at + b.bytes;
        b.bytes += (int64_t)size & ~(int64_t)255;
    };
    auto operand = [&](const void* p, int64_t rows, int64_t cols, int64_t ld, Mat& m) {
        if (rows == 0 || cols == 0) { m = {nullptr, 8}; return; }
        if (rows < 2) ld = (cols + 7) & ~(int64_t)7;
        if (!misaligned(p, 16) && ld % 8 == 0) { m = {const_cast<void*>(p), ld}; return; }
        take(rows, cols, m);
        b.copies[b.count++] = {p, m.p, rows, cols, ld, m.ld};
    };
    const bool empty = g.tokens == 0 || g.hidden == 0 || g.outputs == 0;
    if (backward && empty) return true;
    if (!backward || g.dw_in) operand(g.x, g.tokens, g.width, g.ldx, b.x);
    if (!backward || g.dx) operand(g.w_in, 2 * g.hidden, g.width, g.ldw_in, b.w_in);
    operand(g.w_out, g.outputs, g.hidden, g.ldw_out, b.w_out);
    if (backward) {
        operand(g.dy, g.tokens, g.outputs, g.lddy, b.dy);
        take(g.tokens, 2 * g.hidden, b.dgu);
        if (g.dw_out) take(g.tokens, g.hidden, b.h);
    } else {
        take(g.tokens, g.hidden, b.h);
    }
    return fits;
}
cerar_status_t check_workspace(const cerar_gated_t& g, bool backward, void* workspace, size_t bytes, Block& b) {
    if (!lay_out(g, backward, workspace, b)) return fail(CERAR_ERR_TOO_LARGE, "gated block: a workspace above 2^62 bytes");
    if (b.bytes > 0 && (!workspace || misaligned(workspace, 16))) return fail(CERAR_ERR_INVALID_ARG, "workspace NULL or not aligned to 16 bytes");
    if ((int64_t)bytes < b.bytes) return fail(CERAR_ERR_SHAPE, "the workspace is too small");
    return CERAR_OK;
}
// C (+)= op(a) op(b); an empty sum is zero
cudaError_t product(cerar_ops* o, const Mat& a, bool trans_a, const Mat& b, bool trans_b, int64_t M, int64_t N, int64_t K, void* C, int type, int64_t ldc, bool accumulate, cudaStream_t s,
                    bool after = false, bool followed = false) {
    if (M == 0 || N == 0) return cudaSuccess;
    if (K == 0)
        return accumulate ? cudaSuccess : cudaMemset2DAsync(C, (size_t)(M > 1 ? ldc : N) * type_bytes(type), 0, (size_t)N * type_bytes(type), (size_t)M, s);
    return cerar::launch_matmul16({a.p, b.p, a.ld, b.ld, trans_a, trans_b, M, N, K, C, ldc, type, accumulate ? 1 : 0, o->d_status, after ? 1 : 0, followed ? 1 : 0}, o->num_sms, s, &o->launches);
}

// Memory from the first to behind the last element of a matrix (above zero rows and columns)
struct Span {
    uintptr_t from, to;
};
Span span_of(const void* p, int64_t rows, int64_t cols, int64_t ld, int size) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    return {at, at + ((uintptr_t)(rows - 1) * (uintptr_t)ld + (uintptr_t)cols) * (uintptr_t)size};      // (ld up to 2^40: no signed overflow)
}
Span span_of(const Mat& m, int64_t rows, int64_t cols) { return span_of(m.p, rows, cols, m.ld, 2); }
// Products that run beside one another: since the last one that waited, what each writes and what it reads.
struct Beside {
    struct { Span out, a, b; } running[3];
    int count = 0;
    // Whether the next product may begin beside them.  Where it may not it waits for the one in front, which ends after those in front of it.
    bool add(const Span& out, const Span& a, const Span& b) {
        auto meet = [](const Span& x, const Span& y) { return x.from < y.to && y.from < x.to; };
        bool free = count > 0;
        for (int i = 0; i < count; ++i)
            if (meet(out, running[i].out) || meet(out, running[i].a) || meet(out, running[i].b) || meet(a, running[i].out) || meet(b, running[i].out)) free = false;
        if (!free) count = 0;
        running[count++] = {out, a, b};
        return free;
    }
};

}  // namespace

extern "C" {

cerar_status_t cerar_embed(cerar_ops_t* o, const void* table, cerar_type_t type, int64_t vocab, int64_t width, int64_t ld, const void* ids,
                           int id_bytes, int64_t tokens, float scale, void* y, cerar_type_t y_type, int64_t ldy, cerar_stream_t stream) {
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    if ((st = check_ids(ids, id_bytes, tokens, vocab, width)) != CERAR_OK ||
        (st = check_rows(table, type, vocab, width, ld, "table NULL or not aligned to its elements")) != CERAR_OK ||
        (st = check_rows(y, y_type, tokens, width, ldy, "y NULL or not aligned to its elements")) != CERAR_OK)
        return st;
    if (tokens == 0 || width == 0) return CERAR_OK;
    const cerar::EmbedArgs a = {table, vocab, width, ld, ids, id_bytes, tokens, scale, y, ldy, type, y_type, o->d_status};
    const cudaError_t e = cerar::launch_embed(a, o->num_sms, (cudaStream_t)stream, &o->launches);
    return e == cudaSuccess ? CERAR_OK : cuda_fail(e, "embed launch");
}

size_t cerar_embed_grad_workspace(int64_t tokens, int64_t vocab, int64_t width) {
    if (tokens < 0 || tokens > TOKENS_MAX || vocab < 0 || vocab > SIZE_MAX_ || width < 0 || width > SIZE_MAX_) return 0;
    return cerar::embed_grad_workspace(tokens, vocab, width);
}

cerar_status_t cerar_embed_grad(cerar_ops_t* o, const void* dy, cerar_type_t type, int64_t lddy, const void* ids, int id_bytes, int64_t tokens,
                                float scale, void* dtable, cerar_type_t d_type, int64_t vocab, int64_t width, int64_t ld, int accumulate,
                                void* workspace, size_t workspace_bytes, cerar_stream_t stream) {
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    if ((st = check_ids(ids, id_bytes, tokens, vocab, width)) != CERAR_OK ||
        (st = check_rows(dy, type, tokens, width, lddy, "dy NULL or not aligned to its elements")) != CERAR_OK ||
        (st = check_rows(dtable, d_type, vocab, width, ld, "dtable NULL or not aligned to its elements")) != CERAR_OK)
        return st;
    if (vocab == 0 || width == 0 || (tokens == 0 && accumulate)) return CERAR_OK;
    const size_t need = cerar::embed_grad_workspace(tokens, vocab, width);
    if (need > 0 && (!workspace || misaligned(workspace, 16))) return fail(CERAR_ERR_INVALID_ARG, "workspace NULL or not aligned to 16 bytes");
    if (workspace_bytes < need) return fail(CERAR_ERR_SHAPE, "the workspace is too small");
    const cerar::EmbedGradArgs a = {dy, lddy, ids, id_bytes, tokens, scale, dtable, vocab, width, ld, type, d_type, accumulate != 0, workspace, o->d_status};
    const cudaError_t e = cerar::launch_embed_grad(a, o->num_sms, (cudaStream_t)stream, &o->launches);
    return e == cudaSuccess ? CERAR_OK : cuda_fail(e, "embed gradient launch");
}

cerar_status_t cerar_rotation_table(cerar_ops_t* o, const double* freqs, int pairs, int64_t first, int64_t rows, float* table, cerar_stream_t stream) {
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    if (pairs < 0 || pairs > CERAR_HEAD_DIM_MAX / 2 || rows < 0 || rows > TOKENS_MAX) return fail(CERAR_ERR_SHAPE, "rotation table: up to 256 pairs and 2^31 - 256 positions");
    if (pairs == 0 || rows == 0) return CERAR_OK;
    if (!freqs) return fail(CERAR_ERR_INVALID_ARG, "freqs is NULL");
    for (int i = 0; i < pairs; ++i)
        if (!std::isfinite(freqs[i])) return fail(CERAR_ERR_INVALID_ARG, "a frequency is not finite");
    if (!table || misaligned(table, 8)) return fail(CERAR_ERR_INVALID_ARG, "table NULL or not aligned to 8 bytes");
    const cudaError_t e = cerar::launch_rotation_table(freqs, pairs, first, rows, table, o->num_sms, (cudaStream_t)stream, &o->launches);
    return e == cudaSuccess ? CERAR_OK : cuda_fail(e, "rotation table launch");
}

cerar_status_t cerar_head_norm(cerar_ops_t* o, cerar_type_t type, const cerar_heads_t* parts, int count, cerar_type_t w_type, int64_t tokens, int dim,
                               float eps, const cerar_rotation_t* rotation, cerar_stream_t stream) {
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    cerar::HeadNormArgs a = {};
    if ((st = check_heads(parts, count, type, tokens, dim, false, a)) != CERAR_OK || (st = check_rotation(rotation, dim, a)) != CERAR_OK) return st;
    if (!type_ok(w_type)) return fail(CERAR_ERR_INVALID_ARG, "unknown element type");
    for (int i = 0; i < count; ++i)
        if (misaligned(parts[i].w, type_bytes(w_type))) return fail(CERAR_ERR_INVALID_ARG, "w is not aligned to its elements");
    if (!(eps > 0.f) || !std::isfinite(eps)) return fail(CERAR_ERR_INVALID_ARG, "eps must be positive and finite");
    if (tokens == 0) return CERAR_OK;
    a.eps = eps; a.w_type = w_type; a.status = o->d_status;
    const cudaError_t e = cerar::launch_head_norm(a, o->num_sms, (cudaStream_t)stream, &o->launches);
    return e == cudaSuccess ? CERAR_OK : cuda_fail(e, "head norm launch");
}

size_t cerar_head_norm_grad_workspace(int count, int dim) {
    if (count < 1 || count > 2 || dim < 2 || dim > CERAR_HEAD_DIM_MAX) return 0;
    return cerar::head_norm_grad_workspace(count, dim);
}

cerar_status_t cerar_head_norm_grad(cerar_ops_t* o, cerar_type_t type, const cerar_heads_t* parts, int count, cerar_type_t w_type, cerar_type_t dw_type,
                                    int accumulate, int64_t tokens, int dim, float eps, const cerar_rotation_t* rotation, void* workspace,
                                    size_t workspace_bytes, cerar_stream_t stream) {
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    cerar::HeadNormArgs a = {};
    if ((st = check_heads(parts, count, type, tokens, dim, true, a)) != CERAR_OK || (st = check_rotation(rotation, dim, a)) != CERAR_OK) return st;
    if (!type_ok(w_type) || !type_ok(dw_type)) return fail(CERAR_ERR_INVALID_ARG, "unknown element type");
    for (int i = 0; i < count; ++i)
        if (misaligned(parts[i].w, type_bytes(w_type)) || misaligned(parts[i].dw, type_bytes(dw_type)))
            return fail(CERAR_ERR_INVALID_ARG, "w or dw is not aligned to its elements");
    if (count > 1 && parts[0].dw && parts[1].dw && parts[0].dw != parts[1].dw) {
        const uintptr_t q = reinterpret_cast<uintptr_t>(parts[0].dw), k = reinterpret_cast<uintptr_t>(parts[1].dw);
        if ((q < k ? k - q : q - k) < (uintptr_t)dim * type_bytes(dw_type)) return fail(CERAR_ERR_SHAPE, "dw of the two groups overlap without being the same");
    }
    if (!(eps > 0.f) || !std::isfinite(eps)) return fail(CERAR_ERR_INVALID_ARG, "eps must be positive and finite");
    const size_t need = cerar::head_norm_grad_workspace(count, dim);
    if (!workspace || misaligned(workspace, 16)) return fail(CERAR_ERR_INVALID_ARG, "workspace NULL or not aligned to 16 bytes");
    if (workspace_bytes < need) return fail(CERAR_ERR_SHAPE, "the workspace is too small");
    a.eps = eps; a.w_type = w_type; a.dw_type = dw_type; a.accumulate = accumulate != 0; a.status = o->d_status;
    const cudaError_t e = cerar::launch_head_norm_grad(a, workspace, o->num_sms, (cudaStream_t)stream, &o->launches);
    return e == cudaSuccess ? CERAR_OK : cuda_fail(e, "head norm gradient launch");
}

cerar_status_t cerar_matmul_bf16(cerar_ops_t* o, const void* A, int64_t lda, int trans_a, const void* B, int64_t ldb, int trans_b, int64_t M, int64_t N,
                                 int64_t K, void* C, cerar_type_t type, int64_t ldc, int accumulate, cerar_stream_t stream) {
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    if ((st = check_operand(A, trans_a ? K : M, trans_a ? M : K, lda)) != CERAR_OK || (st = check_operand(B, trans_b ? N : K, trans_b ? K : N, ldb)) != CERAR_OK ||
        (st = check_rows(C, type, M, N, ldc, "C NULL or not aligned to its elements")) != CERAR_OK)
        return st;
    if (M == 0 || N == 0) return CERAR_OK;
    const cudaError_t e = product(o, {const_cast<void*>(A), lda}, trans_a != 0, {const_cast<void*>(B), ldb}, trans_b != 0, M, N, K, C, type, ldc, accumulate != 0, (cudaStream_t)stream);
    return e == cudaSuccess ? CERAR_OK : cuda_fail(e, "bfloat16 matmul launch");
}

int cerar_matmul_bf16_tile(int64_t M, int64_t N, int64_t K, int num_sms, int* split) {
    if (M < 1 || N < 1 || K < 1 || M > SIZE_MAX_ || N > SIZE_MAX_ || K > SIZE_MAX_ || num_sms < 1 || !split) return -1;
    return cerar::matmul16_tile(M, N, K, num_sms, split);
}

cerar_status_t cerar_align_bf16(cerar_ops_t* o, const cerar_rows_t* items, int count, cerar_stream_t stream) {
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    if (!items || count < 1 || count > cerar::ALIGN_MAX) return fail(CERAR_ERR_INVALID_ARG, "1 to 4 matrices are wanted");
    cerar::AlignArgs a[cerar::ALIGN_MAX];
    for (int i = 0; i < count; ++i) {
        const cerar_rows_t& m = items[i];
        if (m.rows < 0 || m.cols < 0 || m.rows > SIZE_MAX_ || m.cols > SIZE_MAX_) return fail(CERAR_ERR_SHAPE, "matrix: sizes from 0 to 2^31 - 256 are wanted");
        if ((st = check_rows(m.src, CERAR_TYPE_BF16, m.rows, m.cols, m.ld, "src NULL or not aligned to its elements")) != CERAR_OK) return st;
        if (m.rows > 0 && m.cols > 0) {
            if (!m.dst || misaligned(m.dst, 16)) return fail(CERAR_ERR_INVALID_ARG, "dst NULL, or not on a 16-byte boundary");
            if (m.ldd % 8 || m.ldd < m.cols || m.ldd > LD_MAX) return fail(CERAR_ERR_SHAPE, "ldd must be a multiple of 8 and at least the number of columns");
        }
        a[i] = {m.src, m.dst, m.cols > 0 ? m.rows : 0, m.cols, m.ld, m.ldd};
    }
    const cudaError_t e = cerar::launch_align(a, count, (cudaStream_t)stream, &o->launches);
    return e == cudaSuccess ? CERAR_OK : cuda_fail(e, "row copy launch");
}

size_t cerar_gated_kept_bytes(int64_t tokens, int64_t hidden) {
    if (tokens < 0 || tokens > TOKENS_MAX || hidden < 0 || hidden > SIZE_MAX_ / 2) return 0;
    return cerar::gated_kept_bytes(tokens, hidden);
}

size_t cerar_gated_workspace(const cerar_gated_t* g, int backward) {
    Block b;
    return g && check_gated(*g, backward != 0) == CERAR_OK && lay_out(*g, backward != 0, nullptr, b) ? (size_t)b.bytes : 0;
}

cerar_status_t cerar_gated_forward(cerar_ops_t* o, const cerar_gated_t* g, void* workspace, size_t workspace_bytes, cerar_stream_t stream) {
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    if (!g) return fail(CERAR_ERR_INVALID_ARG, "the block's description is NULL");
    if ((st = check_gated(*g, false)) != CERAR_OK) return st;
    if (g->tokens == 0 || g->outputs == 0) return CERAR_OK;
    Block b;
    if ((st = check_workspace(*g, false, workspace, workspace_bytes, b)) != CERAR_OK) return st;
    const cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e = cerar::launch_align(b.copies, b.count, s, &o->launches);
    if (e == cudaSuccess && g->hidden > 0 && g->width == 0) {            // empty sums: g = u = 0, and act(0) 0 = 0
        e = cudaMemsetAsync(b.h.p, 0, (size_t)g->tokens * b.h.ld * 2, s);
        if (e == cudaSuccess && g->kept) e = cudaMemsetAsync(g->kept, 0, cerar::gated_kept_bytes(g->tokens, g->hidden), s);
    } else if (e == cudaSuccess && g->hidden > 0) {
        e = cerar::launch_gated_in({b.x.p, b.w_in.p, b.x.ld, b.w_in.ld, g->tokens, g->width, g->hidden, (int)g->activation, b.h.p, g->kept, b.h.ld, o->d_status}, o->num_sms, s, &o->launches);
    }
    if (e == cudaSuccess) e = product(o, b.h, false, b.w_out, true, g->tokens, g->outputs, g->hidden, g->y, CERAR_TYPE_BF16, g->ldy, false, s);
    return e == cudaSuccess ? CERAR_OK : cuda_fail(e, "gated block launch");
}

cerar_status_t cerar_gated_backward(cerar_ops_t* o, const cerar_gated_t* g, void* workspace, size_t workspace_bytes, cerar_stream_t stream) {
    cerar_status_t st = check_ops(o);
    if (st != CERAR_OK) return st;
    if (!g) return fail(CERAR_ERR_INVALID_ARG, "the block's description is NULL");
    if ((st = check_gated(*g, true)) != CERAR_OK) return st;
    Block b;
    if ((st = check_workspace(*g, true, workspace, workspace_bytes, b)) != CERAR_OK) return st;
    const cudaStream_t s = (cudaStream_t)stream;
    const int64_t t = g->tokens, d = g->width, f = g->hidden, n = g->outputs;
    cudaError_t e = cerar::launch_align(b.copies, b.count, s, &o->launches);
    const bool reached = t > 0 && f > 0 && n > 0;                        // otherwise every sum below is empty
    if (e == cudaSuccess && reached)
        e = cerar::launch_gated_grad({b.dy.p, b.w_out.p, g->kept, b.dy.ld, b.w_out.ld, t, n, f, (int)g->activation, b.dgu.p, b.h.p, b.dgu.ld, b.h.ld, o->d_status}, o->num_sms, s, &o->launches);
    // The three products need what the one above made and not one another's results: the first waits for it, the others begin where blocks of the
    // one in front have left, unless a result lies over what those in front read or write (dx over dy).
    Beside beside;
    if (e == cudaSuccess && g->dw_out) {
        const bool early = reached && beside.add(span_of(g->dw_out, n, f, g->lddw_out, type_bytes((int)g->dw_out_type)), span_of(b.dy, t, n), span_of(b.h, t, f));
        e = product(o, b.dy, true, b.h, false, n, f, reached ? t : 0, g->dw_out, (int)g->dw_out_type, g->lddw_out, g->accumulate != 0, s, early, g->dx || g->dw_in);
    }
    if (e == cudaSuccess && g->dx) {
        const bool early = reached && d > 0 && beside.add(span_of(g->dx, t, d, g->lddx, 2), span_of(b.dgu, t, 2 * f), span_of(b.w_in, 2 * f, d));
        e = product(o, b.dgu, false, b.w_in, false, t, d, reached ? 2 * f : 0, g->dx, CERAR_TYPE_BF16, g->lddx, false, s, early, g->dw_in != nullptr);
    }
    if (e == cudaSuccess && g->dw_in) {
        const bool early = reached && d > 0 && beside.add(span_of(g->dw_in, 2 * f, d, g->lddw_in, type_bytes((int)g->dw_in_type)), span_of(b.dgu, t, 2 * f), span_of(b.x, t, d));
        e = product(o, b.dgu, true, b.x, false, 2 * f, d, reached ? t : 0, g->dw_in, (int)g->dw_in_type, g->lddw_in, g->accumulate != 0, s, early);
    }
    return e == cudaSuccess ? CERAR_OK : cuda_fail(e, "gated block gradient launch");
}

}  // extern "C"
