// Products of bfloat16 matrices on the tensor cores, and the two of a gated feed-forward block that carry its elementwise part
// (cerar_matmul_bf16, cerar_gated_forward, cerar_gated_backward; sm_100a: TMA + tcgen05 + TMEM).
//
//   plain   C (+)= op(A) op(B)
//   gate    [g u] = x W^T in one accumulator, h = act(g) u: a tile holds the same columns of both projections side by side
//   grad    dh = dy W_out in the accumulator, dg = dh u act'(g) and du = dh act(g) from the kept g and u
//
// A tile of C is 256 x 256 or 256 x 128 by a pair of blocks (cta_group::2, each with its 128 rows of A and half of B), or 128 x 128 by one.  At 256 x 256
// a k of 64 costs the tensor cores 256 clk and each block 32 KB of shared memory written and read; two accumulators fill tensor memory, so
// that a tile is written while the next one's products run.  Operands are read in place whichever of their dimensions is contiguous.
//
//   warp 0     producer: TMA loads of the stages (64 values of k: rows of 128 bytes in the 128-byte swizzle)
//   warp 1     issues the products; owns the tensor memory
//   warps 4-11 take the sums out (32 lanes of tensor memory, half of the tile's columns each), finish them in binary32 and write
// (Warps 2, 3 complete the warpgroup that hands most of its registers to the others.)
//
// The accumulator drops what does not fit its 24 bits instead of rounding, an error that grows with the number of additions, so plain sums of more
// than SEGMENT blocks of k are put together in registers.  (The gate's results have 16 bits, 24 at most: their sums stay in one piece, so that
// GRAD can take dh out of tensor memory as it goes.)
// Few tiles, long sums: a cluster of S blocks or pairs shares a tile, each sums 1/S of the blocks of k, and the partial tiles are added through
// distributed shared memory, in a fixed order.
// Every wait is bounded; one that runs out sets the status word and the block leaves through the common exit.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>

#include "kernels.cuh"
#include "mma_tile.cuh"
#include "ops.cuh"
#include "packed.cuh"

namespace cerar {
namespace {

using namespace mma;
using namespace packed;
typedef __nv_bfloat16 bf16;

constexpr int BK = 64;                                  // values of k in a stage: rows of 128 bytes
constexpr int UK = 16;                                  // of one product
constexpr int WARP_EPI0 = 4, THREADS = 32 * (WARP_EPI0 + EPI_WARPS), MAX_SPLIT = 8;      // blocks of a (portable) cluster
// registers per thread: 128 x 56 + 256 x 224 = 384 x 168, what the block is launched with
constexpr int REGS_FEW = 56, REGS_MANY = 224;
constexpr uint32_t A_BYTES = BM * BK * 2, PART = 64 * BK * 2;      // an operand lies in parts of 64 of its own rows or columns
constexpr int SEGMENT = 64;                             // 4096 values of k: 256 additions

enum { PLAIN = 0, GATE = 1, GRAD = 2 };

struct Kept {
    unsigned char* at;
    int64_t blocks;                                    // of 32 columns, in a row of blocks
};
struct Params {
    void* C;                                           // PLAIN: C; GATE: h; GRAD: [dg du]
    int64_t ldc;
    Kept kept;                                         // GATE: where g and u go (null: nowhere); GRAD: where they are
    bf16* h;                                           // GRAD: h, or null
    int64_t ldh;
    int M, N, kblocks;                                 // N: columns of C (GATE, GRAD: of h)
    int tiles_m, tiles_n, group_m;
    uint32_t tiles;
    int a_mn, b_mn;                                    // 1: the operand's own dimension (m or n) is the contiguous one
    int accumulate, c_vec, c_pair;                     // rows of C start on 16-byte, on 4-byte boundaries
    int four;                                          // GRAD: rows of dg, du and h on 8-byte boundaries
    int act;
    int stages, split;
    uint32_t a_bytes;                                  // what a load of A brings (few rows: those only; the others' sums are made of
                                                       // whatever lies there, row by row, and not stored)
    int early;                                         // 1: the next kernel of the stream may set itself up meanwhile
    int after, followed;                               // 1: the kernel in front has nothing to do with this one; nor has the one behind
    int* status;
};

template <int CG>
__device__ __forceinline__ void mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 1)
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
                     " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
                     " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

// a barrier of this block, or the one at the same place in both blocks of the pair (bits of `blocks`)
template <int CG>
__device__ __forceinline__ void commit_to(uint32_t bar, uint32_t blocks) {
    if constexpr (CG == 1) tc_commit(bar);
    else asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)blocks) : "memory");
}

// ---------------------------------------------------------------- activations
//
// In binary32, two values at a time (one instruction for both, where there is one).  The exponential and the reciprocal are the hardware's, some
// 2^-22 of themselves off, far below the step of a bfloat16 result.

__device__ __forceinline__ uint64_t exp2_2(uint64_t x) {
    float a, b;
    parts(x, a, b);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    return two_of(a, b);
}
__device__ __forceinline__ uint64_t rcp_2(uint64_t x) {
    float a, b;
    parts(x, a, b);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    return two_of(a, b);
}
constexpr float LOG2E = 1.44269504f;

template <int ACT> struct Act;
template <> struct Act<CERAR_ACT_SILU> {
    static __device__ __forceinline__ uint64_t part(uint64_t g) { return rcp_2(add2(exp2_2(mul2(g, all(-LOG2E))), all(1.f))); }
    static __device__ __forceinline__ uint64_t value(uint64_t g) { return mul2(g, part(g)); }
    static __device__ __forceinline__ void both(uint64_t g, uint64_t& a, uint64_t& d) {
        const uint64_t s = part(g);
        a = mul2(g, s);
        d = mad2(a, mad2(s, all(-1.f), all(1.f)), s);
    }
};
// g Phi(g).  Phi(-|g|) = erfc(z) / 2 with z = |g| / sqrt 2, and erfc(z) = t e^(-z^2 + P(t)), t = 1 / (1 + z / 2), P of degree 9: the
// Chebyshev fit published in Numerical Recipes (erfcc, relative error below 1.2e-7 for all z), its coefficients here times log2 e.
template <> struct Act<CERAR_ACT_GELU> {
    static __device__ __forceinline__ void fit(uint64_t g, uint64_t& t, uint64_t& square, uint64_t& p) {
        const uint64_t z = mul2(g & 0x7FFFFFFF7FFFFFFFull, all(0.70710678f));
        t = rcp_2(mad2(z, all(0.5f), all(1.f)));
        square = mul2(mul2(z, all(-LOG2E)), z);
        p = mad2(t, all(0.17087277f * LOG2E), all(-0.82215223f * LOG2E));
        p = mad2(t, p, all(1.48851587f * LOG2E));
        p = mad2(t, p, all(-1.13520398f * LOG2E));
        p = mad2(t, p, all(0.27886807f * LOG2E));
        p = mad2(t, p, all(-0.18628806f * LOG2E));
        p = mad2(t, p, all(0.09678418f * LOG2E));
        p = mad2(t, p, all(0.37409196f * LOG2E));
        p = mad2(t, p, all(1.00002368f * LOG2E));
        p = mad2(t, p, all(-1.26551223f * LOG2E - 1.f));                 // (- 1: half of erfc)
    }
    // Phi(g) from Phi(-|g|)
    static __device__ __forceinline__ uint64_t side(uint64_t g, uint64_t low) {
        const uint64_t high = mad2(low, all(-1.f), all(1.f));
        float g0, g1, l0, l1, h0, h1;
        parts(g, g0, g1); parts(low, l0, l1); parts(high, h0, h1);
        return two_of(g0 < 0.f ? l0 : h0, g1 < 0.f ? l1 : h1);
    }
    static __device__ __forceinline__ uint64_t value(uint64_t g) {
        uint64_t t, square, p;
        fit(g, t, square, p);
        return mul2(g, side(g, mul2(t, exp2_2(add2(square, p)))));
    }
    static __device__ __forceinline__ void both(uint64_t g, uint64_t& a, uint64_t& d) {
        uint64_t t, square, p;
        fit(g, t, square, p);
        const uint64_t e = exp2_2(square);                               // e^(-g^2 / 2)
        const uint64_t phi = side(g, mul2(mul2(t, e), exp2_2(p)));
        a = mul2(g, phi);
        d = mad2(mul2(g, all(0.39894228f)), e, phi);
    }
};
template <> struct Act<CERAR_ACT_GELU_TANH> {          // g / (1 + e^-2v) with v = sqrt(2 / pi) (g + 0.044715 g^3): (1 + tanh v) / 2 is that quotient
    static constexpr float FAR_OUT = 1e6f;             // of g^2: |v| is above 10^7 there
    static __device__ __forceinline__ uint64_t part(uint64_t g, uint64_t gg) {
        return rcp_2(add2(exp2_2(mul2(mul2(g, all(-1.5957691f * LOG2E)), mad2(gg, all(0.044715f), all(1.f)))), all(1.f)));
    }
    static __device__ __forceinline__ uint64_t value(uint64_t g) { return mul2(g, part(g, mul2(g, g))); }
    static __device__ __forceinline__ void both(uint64_t g, uint64_t& a, uint64_t& d) {
        // Far out s is 0 or 1 and the derivative too: g s (1 - s), which is zero there, has a finite factor as long as the square is finite
        // (g may be up to the end of the range).
        float x, y;
        parts(mul2(g, g), x, y);
        const uint64_t gg = two_of(fminf(x, FAR_OUT), fminf(y, FAR_OUT)), s = part(g, gg);
        a = mul2(g, s);
        const uint64_t rest = mul2(a, mad2(s, all(-1.f), all(1.f)));
        d = mad2(rest, mad2(gg, all(1.5957691f * 0.134145f), all(1.5957691f)), s);
    }
};
template <> struct Act<CERAR_ACT_RELU> {
    static __device__ __forceinline__ float one(float g) { return g > 0.f ? g : g != g ? g : 0.f; }
    static __device__ __forceinline__ uint64_t value(uint64_t g) {
        float x, y;
        parts(g, x, y);
        return two_of(one(x), one(y));
    }
    static __device__ __forceinline__ void both(uint64_t g, uint64_t& a, uint64_t& d) {
        float x, y;
        parts(g, x, y);
        a = two_of(one(x), one(y));
        d = two_of(x > 0.f ? 1.f : 0.f, y > 0.f ? 1.f : 0.f);
    }
};
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
    if (act == CERAR_ACT_SILU) f(Act<CERAR_ACT_SILU>());
    else if (act == CERAR_ACT_GELU) f(Act<CERAR_ACT_GELU>());
    else if (act == CERAR_ACT_GELU_TANH) f(Act<CERAR_ACT_GELU_TANH>());
    else f(Act<CERAR_ACT_RELU>());
}

// ---------------------------------------------------------------- what is kept for the backward pass
//
// g and u in 24 bits: sign, exponent and 15 bits of the fraction, rounded to nearest (2^-16 of themselves off).  Kept in bfloat16 their rounding would
// be the largest part of the error of dx and dw_in (3.0e-3 instead of 2.3e-3 of the norm); h is made again from them, so that no more is kept
// than g, u and h in bfloat16 would be.
// They lie in blocks of 32 rows x 32 columns, 6 KB each: the upper 16 bits of g in pieces of 16 bytes (8 columns), piece j of row r at
// (32 j + r) 16; the same of u; the lower 8 bits of g in pieces of 16 columns; the same of u.  A warp that holds a row per lane so reads and writes
// 512 bytes at a time with no exchange between lanes, and a block is one run of memory (in rows of their own the reads came in pieces of 64 bytes
// that were a row of the matrix apart: 16384 x 8192 x 2048 562 us).

constexpr int64_t KEPT_BLOCK = 6144;
__device__ __forceinline__ unsigned char* kept_block(const Kept& k, int row, int col) { return k.at + ((int64_t)(row >> 5) * k.blocks + (col >> 5)) * KEPT_BLOCK; }
__device__ __forceinline__ uint32_t to24(float x) {    // (a carry into the exponent is right; NaN keeps its upper bits)
    const uint32_t b = __float_as_uint(x);
    return x != x ? b | 0x00400000u : b + 0x80u;
}
__device__ __forceinline__ uint32_t highs(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x7632); }
__device__ __forceinline__ uint32_t lows(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0051), __byte_perm(c, d, 0x0051), 0x5410);
}
// values 2 i and 2 i + 1 of four, from their upper and lower bits
__device__ __forceinline__ uint64_t pair_of(uint32_t h, uint32_t low, int i) {
    const uint32_t x = __byte_perm(h, low, i ? 0x1066 : 0x1044) & 0xFFFFFF00u, y = __byte_perm(h, low, i ? 0x3277 : 0x3255) & 0xFFFFFF00u;
    return two_of(__uint_as_float(x), __uint_as_float(y));
}
// four neighbouring values of one row
struct Four {
    uint2 high;
    uint32_t low;
};
__device__ __forceinline__ Four load_kept(const Kept& k, int which, int row, int col) {
    const unsigned char* b = kept_block(k, row, col);
    const int r = row & 31, c = col & 31;
    return {__ldg(reinterpret_cast<const uint2*>(b + which * 2048 + ((c >> 3) * 32 + r) * 16 + (c & 7) * 2)),
            __ldg(reinterpret_cast<const uint32_t*>(b + 4096 + which * 1024 + ((c >> 4) * 32 + r) * 16 + (c & 15)))};
}
__device__ __forceinline__ void store_kept(const Kept& k, int which, int row, int col, const float* v) {
    unsigned char* b = kept_block(k, row, col);
    const int r = row & 31, c = col & 31;
    const uint32_t x = to24(v[0]), y = to24(v[1]), z = to24(v[2]), w = to24(v[3]);
    *reinterpret_cast<uint2*>(b + which * 2048 + ((c >> 3) * 32 + r) * 16 + (c & 7) * 2) = make_uint2(highs(x, y), highs(z, w));
    *reinterpret_cast<uint32_t*>(b + 4096 + which * 1024 + ((c >> 4) * 32 + r) * 16 + (c & 15)) = lows(x, y, z, w);
}
// 32 values of a lane's row to a block, and the loads of both g's and u's
__device__ __forceinline__ void store_kept32(unsigned char* block, int which, const float* v) {
    const int lane = threadIdx.x & 31;
    uint32_t low[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t b[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = to24(v[8 * j + e]);
        *reinterpret_cast<uint4*>(block + which * 2048 + (j * 32 + lane) * 16) = make_uint4(highs(b[0], b[1]), highs(b[2], b[3]), highs(b[4], b[5]), highs(b[6], b[7]));
        low[2 * j] = lows(b[0], b[1], b[2], b[3]);
        low[2 * j + 1] = lows(b[4], b[5], b[6], b[7]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
        *reinterpret_cast<uint4*>(block + 4096 + which * 1024 + (j * 32 + lane) * 16) = make_uint4(low[4 * j], low[4 * j + 1], low[4 * j + 2], low[4 * j + 3]);
}
struct Kept32 {
    uint4 high[2][4], low[2][2];
};
__device__ __forceinline__ void load_kept32(const unsigned char* block, Kept32& k) {     // (volatile: issued here, not where they are used)
    const unsigned char* at = block + (threadIdx.x & 31) * 16;
    auto load = [](const unsigned char* p, uint4& q) { asm volatile("ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p)); };
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int j = 0; j < 4; ++j) load(at + which * 2048 + j * 512, k.high[which][j]);
#pragma unroll
        for (int j = 0; j < 2; ++j) load(at + 4096 + which * 1024 + j * 512, k.low[which][j]);
    }
}
__device__ __forceinline__ uint32_t word(const uint4& q, int i) { return i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w; }
// values 2 i and 2 i + 1 (i < 16) of g (which = 0) or u
__device__ __forceinline__ uint64_t pair_of(const Kept32& k, int which, int i) {
    return pair_of(word(k.high[which][i >> 2], i & 3), word(k.low[which][i >> 3], (i >> 1) & 3), i & 1);
}

// ---------------------------------------------------------------- writing

// Rows row0 .. row0 + 31 (those below M) and columns col0 .. col0 + W - 1 (those below N) of a bfloat16 matrix; the warp holds row (lane)'s values.
template <int W>
__device__ __forceinline__ void write_rows(uint32_t staging, bf16* c, int64_t ld, int M, int N, int row0, int col0, const float* v, bool vec) {
    const int lane = threadIdx.x & 31;
    const int nrows = M - row0 < 32 ? M - row0 : 32, n = N - col0 < W ? N - col0 : W;
    if (nrows <= 0 || n <= 0) return;
    __syncwarp();
#pragma unroll
    for (int j = 0; j < W / 8; ++j) {
        const uint4 q = Out<bf16>::pack(v + j * 8);
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(staging + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
    }
    __syncwarp();
    if (vec) {
        constexpr int PER_ROW = W / 8, ROWS = 32 / PER_ROW;
        const int j = lane % PER_ROW;
#pragma unroll
        for (int it = 0; it < 32 / ROWS; ++it) {
            const int r = it * ROWS + lane / PER_ROW;
            uint4 q;
            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(staging + r * 128 + ((j ^ (r & 7)) << 4)) : "memory");
            if (r >= nrows) continue;
            bf16* dst = c + (int64_t)(row0 + r) * ld + col0 + j * 8;
            if (8 * j + 8 <= n) {
                *reinterpret_cast<uint4*>(dst) = q;
            } else {
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (8 * j + e < n) reinterpret_cast<unsigned short*>(dst)[e] = (unsigned short)(e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xFFFFu);
            }
        }
    } else {
        // Rows on other boundaries: 16 bytes at a time from the first boundary inside the row on, its ends element by element.
        constexpr int PER_ROW = W / 8, ROWS = 32 / PER_ROW;
        const int j = lane % PER_ROW;
        auto element = [&](int r, int e) {
            uint16_t q;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(q) : "r"(staging + r * 128 + (((e >> 3) ^ (r & 7)) << 4) + (e & 7) * 2) : "memory");
            return q;
        };
#pragma unroll 1
        for (int it = 0; it < 32 / ROWS; ++it) {
            const int r = it * ROWS + lane / PER_ROW;
            if (r >= nrows) continue;
            uint16_t* dst = reinterpret_cast<uint16_t*>(c + (int64_t)(row0 + r) * ld + col0);
            const int gap = (int)(8u - (uint32_t)(reinterpret_cast<uintptr_t>(dst) >> 1)) & 7, first = gap < n ? gap : n;
            const int whole = (n - first) >> 3, rest = (n - first) & 7, e0 = first + 8 * j;
            if (j < whole) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = (uint32_t)element(r, e0 + 2 * i) | (uint32_t)element(r, e0 + 2 * i + 1) << 16;
                *reinterpret_cast<uint4*>(dst + e0) = make_uint4(w[0], w[1], w[2], w[3]);
            }
#pragma unroll
            for (int i = j; i < 8; i += PER_ROW) {
                if (i < first) dst[i] = element(r, i);
                if (i < rest) dst[first + 8 * whole + i] = element(r, first + 8 * whole + i);
            }
        }
    }
}

// Four columns of a row to bfloat16, `n` of them there
__device__ __forceinline__ void store4(bf16* p, int n, bool vec, uint64_t lo, uint64_t hi) {
    float v[4];
    parts(lo, v[0], v[1]);
    parts(hi, v[2], v[3]);
    if (vec && n >= 4) {
        *reinterpret_cast<uint2*>(p) = make_uint2(Out<bf16>::two(v[0], v[1]), Out<bf16>::two(v[2], v[3]));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) p[e] = __float2bfloat16_rn(v[e]);
    }
}
// dg, du and h of four columns from dh and the kept g and u
template <typename A>
__device__ __forceinline__ void write_grad4(const Params& p, A act, int row, int col, const uint64_t* dh, const Four& g, const Four& u) {
    const int n = p.N - col;
    uint64_t dg[2], du[2], h[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint64_t a, d;
        const uint64_t up = pair_of(i ? u.high.y : u.high.x, u.low, i);
        act.both(pair_of(i ? g.high.y : g.high.x, g.low, i), a, d);
        dg[i] = mul2(mul2(dh[i], up), d);
        du[i] = mul2(dh[i], a);
        h[i] = mul2(a, up);
    }
    bf16* c = static_cast<bf16*>(p.C) + (int64_t)row * p.ldc + col;
    store4(c, n, p.four, dg[0], dg[1]);
    store4(c + p.N, n, p.four, du[0], du[1]);
    if (p.h) store4(p.h + (int64_t)row * p.ldh + col, n, p.four, h[0], h[1]);
}

// The whole tile's sums of this warp: rows row0 .. row0 + 31, CW columns, in registers.
template <int KIND, int BN, typename C>
__device__ __forceinline__ void write_tile(const Params& p, uint32_t staging, int row0, int tn, int half, float* acc) {
    constexpr int CW = BN / 2;
    const int lane = threadIdx.x & 31;
    if constexpr (KIND == PLAIN) {
        constexpr int SLAB = 8 * Out<C>::PER16;
        if (sizeof(C) == 2 && !p.accumulate && !p.c_vec) {
#pragma unroll
            for (int c = 0; c < CW / 64; ++c) write_rows<64>(staging, reinterpret_cast<bf16*>(p.C), p.ldc, p.M, p.N, row0, tn * BN + half * CW + c * 64, acc + c * 64, false);
            return;
        }
#pragma unroll
        for (int c = 0; c < CW / SLAB; ++c) write_slab<C>(p, staging, row0, tn * BN + half * CW + c * SLAB, acc + c * SLAB);
    } else if constexpr (KIND == GATE) {
        constexpr int FW = BN / 4;                      // columns of h: acc holds their g, then their u
        const int col0 = tn * (BN / 2) + half * FW, nrows = p.M - row0 < 32 ? p.M - row0 : 32;
        if (nrows <= 0 || col0 >= p.N) return;
        if (p.kept.at && lane < nrows) {
            unsigned char* block = kept_block(p.kept, row0, col0);
#pragma unroll
            for (int c = 0; c < FW; c += 32) {
                if (col0 + c >= p.N) break;
                store_kept32(block + c / 32 * KEPT_BLOCK, 0, acc + c);
                store_kept32(block + c / 32 * KEPT_BLOCK, 1, acc + FW + c);
            }
        }
        with_act(p.act, [&](auto act) {
#pragma unroll
            for (int j = 0; j < FW; j += 2) parts(mul2(act.value(two_of(acc[j], acc[j + 1])), two_of(acc[FW + j], acc[FW + j + 1])), acc[j], acc[j + 1]);
        });
        write_rows<FW>(staging, static_cast<bf16*>(p.C), p.ldc, p.M, p.N, row0, col0, acc, p.c_vec);
    }
}

// GRAD: dh comes from tensor memory (`from`: this warp's lanes and columns) 32 columns at a time, a row per lane, as g and u do; those of the next 32
// columns are on their way meanwhile (next: of the first).
template <int BN, typename A, typename Release>
__device__ __forceinline__ void write_grad(const Params& p, A act, uint32_t staging, uint32_t from, int row0, int col0, Kept32& next, Release release) {
    constexpr int CW = BN / 2;
    const bool there = row0 + (int)(threadIdx.x & 31) < p.M;
#pragma unroll 1
    for (int h = 0; h < CW / 32; ++h) {
        const int col = col0 + h * 32;
        uint32_t v[32];
        ld32_start(from + h * 32, v);
        const Kept32 now = next;
        if (h + 1 < CW / 32 && there && col + 32 < p.N) load_kept32(kept_block(p.kept, row0, col + 32), next);
        ld32_done(v);
        if (h + 1 == CW / 32) release();
        if (row0 >= p.M || col >= p.N) continue;
        float dg[32], du[32], hv[32];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint64_t dh = two_of(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), up = pair_of(now, 1, i);
            uint64_t a, d;
            act.both(pair_of(now, 0, i), a, d);
            parts(mul2(mul2(dh, up), d), dg[2 * i], dg[2 * i + 1]);
            parts(mul2(dh, a), du[2 * i], du[2 * i + 1]);
            parts(mul2(a, up), hv[2 * i], hv[2 * i + 1]);
        }
        bf16* c = static_cast<bf16*>(p.C);
        write_rows<32>(staging, c, p.ldc, p.M, p.N, row0, col, dg, p.c_vec);
        write_rows<32>(staging, c + p.N, p.ldc, p.M, p.N, row0, col, du, p.c_vec);
        if (p.h) write_rows<32>(staging, p.h, p.ldh, p.M, p.N, row0, col, hv, p.c_vec);
    }
}

// A tile whose sum is split over a cluster: every block leaves the rows of its partial tile that exist in its stages (free by then), row
// r at r * BN floats, 16-byte pieces exchanged by the row so that lanes do not meet in a bank ...
template <int BN>
__device__ __forceinline__ void store_partial(uint32_t smem, int rows, int row, int col, int n, const float* v) {
    if (row >= rows) return;
    const uint32_t base = smem + (uint32_t)row * (BN * 4u);
#pragma unroll
    for (int j = 0; j < n / 4; ++j)
        asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(base + ((uint32_t)((col / 4 + j) ^ (row & 7)) << 4)), "f"(v[4 * j]), "f"(v[4 * j + 1]),
                     "f"(v[4 * j + 2]), "f"(v[4 * j + 3]) : "memory");
}
template <int CG>
__device__ __forceinline__ float4 add_piece(const Params& p, uint32_t at, int pair_rank) {
    float4 w[MAX_SPLIT / CG];
#pragma unroll
    for (int q = 0; q < MAX_SPLIT / CG; ++q)
        if (q < p.split) w[q] = ld_cluster4(at, q * CG + pair_rank);
    float4 v = w[0];
#pragma unroll
    for (int q = 1; q < MAX_SPLIT / CG; ++q)
        if (q < p.split) { v.x += w[q].x; v.y += w[q].y; v.z += w[q].z; v.w += w[q].w; }
    return v;
}
// ... and adds every split-th run of 32 pieces (a warp's) of all partial tiles, in the order of their blocks of k.
template <int CG, int KIND, int BN, typename C>
__device__ __noinline__ void add_partials(const Params& p, uint32_t smem, int row0, int tn, int rows, int rank, int pair_rank, int thread) {
    constexpr int PER_ROW = KIND == GATE ? BN / 8 : BN / 4;
    const int pieces = rows * PER_ROW;
    for (int run = (thread >> 5) * p.split + rank; run * 32 < pieces; run += EPI_WARPS * p.split) {
        const int i = run * 32 + (thread & 31);
        if (i >= pieces) continue;
        const int r = i / PER_ROW, j = i % PER_ROW, row = row0 + r;
        const uint32_t base = smem + (uint32_t)r * (BN * 4u);
        const float4 v4 = add_piece<CG>(p, base + ((uint32_t)(j ^ (r & 7)) << 4), pair_rank);
        const float v[4] = {v4.x, v4.y, v4.z, v4.w};
        const int col = tn * (PER_ROW * 4) + 4 * j, n = p.N - col;
        if constexpr (KIND == PLAIN) {
            C* dst = static_cast<C*>(p.C) + (int64_t)row * p.ldc + col;
            if (p.c_vec && !p.accumulate && n >= 4) {
                if constexpr (sizeof(C) == 4) *reinterpret_cast<float4*>(dst) = v4;
                else *reinterpret_cast<uint2*>(dst) = make_uint2(Out<C>::two(v[0], v[1]), Out<C>::two(v[2], v[3]));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < n) dst[e] = (C)(p.accumulate ? (float)dst[e] + v[e] : v[e]);
            }
        } else if constexpr (KIND == GATE) {
            // a row's columns of g are followed by the same ones of u
            const float4 u4 = add_piece<CG>(p, base + ((uint32_t)((j + PER_ROW) ^ (r & 7)) << 4), pair_rank);
            const float u[4] = {u4.x, u4.y, u4.z, u4.w};
            if (p.kept.at && n > 0) {
                store_kept(p.kept, 0, row, col, v);
                store_kept(p.kept, 1, row, col, u);
            }
            if (n > 0)
                with_act(p.act, [&](auto act) {
                    store4(static_cast<bf16*>(p.C) + (int64_t)row * p.ldc + col, n, p.c_vec, mul2(act.value(two_of(v[0], v[1])), two_of(u[0], u[1])),
                           mul2(act.value(two_of(v[2], v[3])), two_of(u[2], u[3])));
                });
        } else {
            if (n > 0) {
                const uint64_t dh[2] = {two_of(v[0], v[1]), two_of(v[2], v[3])};
                const Four g = load_kept(p.kept, 0, row, col), u = load_kept(p.kept, 1, row, col);
                with_act(p.act, [&](auto act) { write_grad4(p, act, row, col, dh, g, u); });
            }
        }
    }
}

template <int CG, int BN, int KIND, typename C>
__global__ void __launch_bounds__(THREADS, 1)
matmul16_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ Params p) {
    constexpr int CW = BN / 2;                           // columns of the accumulator per writing warp
    constexpr int B_ROWS = BN / CG;                      // of the tile of B, in this block
    constexpr uint32_t STAGE = A_BYTES + B_ROWS * BK * 2;
    extern __shared__ unsigned char smem_dyn[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t smem = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    const uint32_t staging0 = smem + (uint32_t)p.stages * STAGE;
    const uint32_t bars = staging0 + EPI_WARPS * STAGING;
    const uint32_t full = bars, empty = full + 8u * p.stages, acc_full = empty + 8u * p.stages, acc_empty = acc_full + 16u, slot = acc_empty + 16u;

    if (threadIdx.x == 0) {
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        for (int s = 0; s < p.stages; ++s) { mbar_init(full + 8u * s, 1); mbar_init(empty + 8u * s, 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(acc_full + 8u * b, 1); mbar_init(acc_empty + 8u * b, CG * EPI_WARPS); }
        mbar_init_fence();
    }
    if (warp == 1) {
        if constexpr (CG == 1) {
            tc_alloc(slot, 512u);
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(512u) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();               // the other block's barriers are there before anything is sent to them
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(slot));
    if (p.early && !p.followed) grid_dependents_may_launch();
    if (!p.after) grid_dependency_wait();
    if (p.followed) grid_dependents_may_launch();        // (behind the wait: what ran before this kernel is then complete for that one too)

    // a cluster is `split` blocks, or pairs of blocks (CG = 2: tiles of 256 rows), that share the sum of a tile
    const int crank = CG == 2 || p.split > 1 ? (int)cluster_rank() : 0;
    const int pair_rank = crank % CG, rank = crank / CG, leader = crank - pair_rank;
    const uint32_t csize = CG * p.split;
    const uint32_t t0 = blockIdx.x / csize, tstep = gridDim.x / csize;
    const int kb0 = (int)((int64_t)p.kblocks * rank / p.split), kb1 = (int)((int64_t)p.kblocks * (rank + 1) / p.split);
    const int segment = KIND == PLAIN ? SEGMENT : kb1;   // (kb0 + kb1 is behind the end)
    bool failed = false;

    if (warp < WARP_EPI0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FEW));
        if (warp == 0) {
            if (lane == 0) {
                if (p.after) asm volatile("fence.proxy.async;" ::: "memory");
                uint32_t s = 0, ph = 1;
                for (uint32_t t = t0; t < p.tiles && !failed; t += tstep) {
                    int tm, tn;
                    tile_of(p, t, tm, tn);
                    const int m0 = (tm * CG + pair_rank) * BM;
                    // first row or column of every part of 64 of B: GATE takes its first half from g's weights, its second from u's
                    int n0 = tn * BN + pair_rank * B_ROWS, n1 = n0 + 64;
                    if constexpr (KIND == GATE) {
                        n0 = tn * (BN / 2) + pair_rank * p.N;
                        n1 = CG == 2 ? n0 + 64 : n0 + p.N;
                    }
                    for (int kb = kb0; kb < kb1; ++kb) {
                        if (!wait_soon(empty + 8u * s, ph)) { failed = true; break; }
                        const uint32_t a = smem + s * STAGE, b = a + A_BYTES;
                        if (pair_rank == 0) mbar_arrive_expect_tx(full + 8u * s, CG * (p.a_bytes + B_ROWS * BK * 2));       // what both blocks load
                        const uint32_t bar = CG == 1 ? full + 8u * s : in_block(full + 8u * s, leader);
                        if (p.a_mn) {
                            tma_load_operand<CG>(a, &map_a, m0, kb * BK, bar);
                            tma_load_operand<CG>(a + PART, &map_a, m0 + 64, kb * BK, bar);
                        } else {
                            tma_load_operand<CG>(a, &map_a, kb * BK, m0, bar);
                        }
                        if (p.b_mn) {
                            tma_load_operand<CG>(b, &map_b, n0, kb * BK, bar);
                            if (B_ROWS > 64) tma_load_operand<CG>(b + PART, &map_b, n1, kb * BK, bar);
                        } else {
                            tma_load_operand<CG>(b, &map_b, kb * BK, n0, bar);
                            if (B_ROWS > 64) tma_load_operand<CG>(b + PART, &map_b, kb * BK, n1, bar);
                        }
                        if (++s == (uint32_t)p.stages) { s = 0; ph ^= 1u; }
                    }
                }
            }
        } else if (warp == 1) {
            if (pair_rank == 0) {
                // The whole warp goes through the loop and one lane issues: what the products are made from then stays in uniform registers.
                const uint32_t one = elect_one();
                // D binary32, A and B bfloat16, M = 128 CG, N = BN
                const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)p.a_mn << 15) | ((uint32_t)p.b_mn << 16) | ((uint32_t)(BN >> 3) << 17) |
                                       ((uint32_t)(CG * BM >> 4) << 24);
                // 16 values of k further: 32 bytes in a row of k, or 16 rows of 128 bytes
                const uint64_t a_step = p.a_mn ? (UK * 128u) >> 4 : (UK * 2u) >> 4, b_step = p.b_mn ? (UK * 128u) >> 4 : (UK * 2u) >> 4;
                const uint64_t desc0 = swizzled_desc(smem, PART);
                uint32_t s = 0, ph = 0, seg = 0;
                for (uint32_t t = t0; t < p.tiles && !failed; t += tstep)
                    for (int k0 = kb0; k0 < kb1 && !failed; k0 += segment, ++seg) {
                        const uint32_t buf = seg & 1u, d = tmem + buf * 256u;
                        if (!warp_wait_soon(acc_empty + 8u * buf, ((seg >> 1) & 1u) ^ 1u)) { failed = true; break; }
                        const int k1 = k0 + segment < kb1 ? k0 + segment : kb1;
                        for (int kb = k0; kb < k1; ++kb) {
                            if (!warp_wait_soon(full + 8u * s, ph)) { failed = true; break; }
                            tc_fence_after();
                            const uint64_t da = desc0 + (uint64_t)(s * (STAGE >> 4)), db = da + (A_BYTES >> 4);
                            if (one) {
#pragma unroll
                                for (int k = 0; k < BK / UK; ++k) mma_bf16<CG>(d, da + k * a_step, db + k * b_step, idesc, kb != k0 || k != 0);
                                commit_to<CG>(empty + 8u * s, 3u << leader);
                                if (kb + 1 == k1) commit_to<CG>(acc_full + 8u * buf, 3u << leader);
                            }
                            __syncwarp();
                            if (++s == (uint32_t)p.stages) { s = 0; ph ^= 1u; }
                        }
                    }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_MANY));
        const int quad = warp & 3, half = (warp - WARP_EPI0) >> 2;
        const uint32_t staging = staging0 + (uint32_t)(warp - WARP_EPI0) * STAGING;
        const uint32_t freed = CG == 1 ? acc_empty : in_block(acc_empty, leader);
        uint32_t seg = 0;
        for (uint32_t t = t0; t < p.tiles && !failed; t += tstep) {
            int tm, tn;
            tile_of(p, t, tm, tn);
            const int row0 = (tm * CG + pair_rank) * BM + quad * 32;
            if constexpr (KIND == GRAD) {                // (one segment: see SEGMENT)
                const uint32_t buf = seg & 1u, from = tmem + ((uint32_t)(quad * 32) << 16) + buf * 256u + half * CW;
                const int col0 = tn * BN + half * CW;
                Kept32 next = {};
                if (p.split == 1 && row0 + lane < p.M && col0 < p.N) load_kept32(kept_block(p.kept, row0, col0), next);
                if (!warp_wait_soon(acc_full + 8u * buf, (seg >> 1) & 1u)) { failed = true; break; }
                tc_fence_after();
                auto release = [&] {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive<CG>(freed + 8u * buf);
                };
                if (p.split == 1) {
                    with_act(p.act, [&](auto act) { write_grad<BN>(p, act, staging, from, row0, col0, next, release); });
                } else {
#pragma unroll 1
                    for (int c = 0; c < CW / 32; ++c) {
                        uint32_t v[32];
                        ld32_start(from + c * 32, v);
                        ld32_done(v);
                        store_partial<BN>(smem, p.M - (tm * CG + pair_rank) * BM, quad * 32 + lane, half * CW + c * 32, 32, reinterpret_cast<const float*>(v));
                    }
                    release();
                }
                ++seg;
                continue;
            }
            float acc[CW];
            for (int k0 = kb0; k0 < kb1; k0 += segment, ++seg) {
                const uint32_t buf = seg & 1u;
                if (!warp_wait_soon(acc_full + 8u * buf, (seg >> 1) & 1u)) { failed = true; break; }
                tc_fence_after();
                const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16) + buf * 256u;
#pragma unroll
                for (int c = 0; c < CW / 32; ++c) {
                    // GATE: this warp's columns of g, then the same ones of u
                    const uint32_t col = KIND != GATE ? half * CW + c * 32 : c * 32 < CW / 2 ? half * (CW / 2) + c * 32 : CW + half * (CW / 2) + c * 32 - CW / 2;
                    uint32_t v[32];
                    ld32_start(from + col, v);
                    ld32_done(v);
                    if (c == CW / 32 - 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) arrive<CG>(freed + 8u * buf);
                    }
                    if (k0 == kb0) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) acc[c * 32 + j] = __uint_as_float(v[j]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) acc[c * 32 + j] += __uint_as_float(v[j]);
                    }
                }
            }
            if (failed) break;
            if (KIND != GRAD && p.split == 1) {
                write_tile<KIND, BN, C>(p, staging, row0, tn, half, acc);
                __syncwarp();
            } else if constexpr (KIND == GATE) {
                store_partial<BN>(smem, p.M - (tm * CG + pair_rank) * BM, quad * 32 + lane, half * (CW / 2), CW / 2, acc);
                store_partial<BN>(smem, p.M - (tm * CG + pair_rank) * BM, quad * 32 + lane, CW + half * (CW / 2), CW / 2, acc + CW / 2);
            } else {
                store_partial<BN>(smem, p.M - (tm * CG + pair_rank) * BM, quad * 32 + lane, half * CW, CW, acc);
            }
        }
    }
    __syncwarp();
    if (p.split > 1) {
        cluster_sync();
        if (warp >= WARP_EPI0) {
            int tm, tn;                                  // (one tile per cluster)
            tile_of(p, t0, tm, tn);
            const int row0 = (tm * CG + pair_rank) * BM;
            add_partials<CG, KIND, BN, C>(p, smem, row0, tn, p.M - row0 < BM ? p.M - row0 : BM, rank, pair_rank, threadIdx.x - 32 * WARP_EPI0);
        }
        __syncwarp();
    }
    if (CG == 2 || p.split > 1) {
        tc_fence_before();
        cluster_sync();                                  // no block leaves while another reads its part or sends to it
        tc_fence_after();
    }
    if (p.after) grid_dependency_wait();                 // this kernel's end is the end of those in front too
    leave<CG>(p, failed, warp, lane, tmem);
}

bool make_map_16bit(CUtensorMap* m, const void* x, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
    const cuuint64_t dim[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {(cuuint32_t)BK, (cuuint32_t)box_rows}, step[2] = {1, 1};
    return encode_tiled(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(x), dim, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

// ---------------------------------------------------------------- few rows
//
// Up to sixteen rows of A against weights whose rows are the sums' terms (B transposed): the weights are read once and that is all there is to it.
// A block takes 16 rows of B (GATE: of both halves), its warps every W-th run of 32 terms of them, straight from memory into the operands of
// mma.sync (16 weights' rows x 8 tokens): a lane's 16 bytes are 8 neighbouring terms of one row, and since both operands name the terms in the
// same order, any order will do.  The warps' sums are added in their order.  The next kernel may set itself up meanwhile.
// (Scalar multiply-adds were bound by unpacking from two rows on: 4 x 16384 x 2048 in 29 us, one row 14.6.)
constexpr int FEW_ROWS = 16, FEW_AHEAD = 4;
constexpr int64_t FEW_TERMS = 65536;                   // a warp's sum is then at most 256 additions, as in a tile
// Weights up to this size: they come in pieces of 64 bytes, which costs nothing while latency is what counts (2048 x 512: 5.0 -> 3.1 us, 2048 x 2048:
// 7.1 -> 4.9), but does where bandwidth does (4096 x 2048: 8.2 -> 8.9, 4096 x 8192: 16.7 -> 27.5).
constexpr int64_t FEW_BYTES = 12 << 20;
struct FewParams {
    const bf16 *A, *B;
    int64_t lda, ldb;
    int M, K;
    int64_t N;
};
// 8 terms of a row from k on; zeros from K on (rows are 16-byte aligned: the 16 bytes hold a term of the row)
template <bool ONCE>
__device__ __forceinline__ uint4 load_terms(const bf16* row, int k, int K) {
    uint4 q = make_uint4(0u, 0u, 0u, 0u);
    if (k >= K) return q;
    if constexpr (ONCE) asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(row + k));
    else q = __ldg(reinterpret_cast<const uint4*>(row + k));
    if (k + 8 > K) {
        const int n = K - k;
        auto cut = [&](uint32_t w, int i) { return n >= 2 * i + 2 ? w : n == 2 * i + 1 ? w & 0xFFFFu : 0u; };
        q = make_uint4(cut(q.x, 0), cut(q.y, 1), cut(q.z, 2), cut(q.w, 3));
    }
    return q;
}
__device__ __forceinline__ void mma_16x8(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// W warps; NT groups of 8 rows of A
template <int NT, int W, int KIND, typename C>
__global__ void __launch_bounds__(32 * W) few_rows_kernel(const FewParams f, const Params p) {
    constexpr int H = KIND == GATE ? 2 : 1;
    __shared__ float sums[W][H][NT][32][4];
    grid_dependents_may_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const bf16 *b[H][2], *a[NT];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int64_t n = n0 + g + 8 * r;           // (rows behind the last: the last one's, not stored)
            b[h][r] = f.B + (h * f.N + (n < f.N ? n : f.N - 1)) * f.ldb;
        }
#pragma unroll
    for (int t = 0; t < NT; ++t) a[t] = f.A + (8 * t + g < f.M ? 8 * t + g : f.M - 1) * f.lda;
    grid_dependency_wait();
    float acc[H][NT][4] = {};
    for (int k0 = warp * (32 * FEW_AHEAD) + c * 8; k0 - c * 8 < f.K; k0 += 32 * W * FEW_AHEAD) {
        uint4 w[FEW_AHEAD][H][2], x[FEW_AHEAD][NT];
#pragma unroll
        for (int i = 0; i < FEW_AHEAD; ++i)
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) w[i][h][r] = load_terms<true>(b[h][r], k0 + i * 32, f.K);
#pragma unroll
        for (int i = 0; i < FEW_AHEAD; ++i)
#pragma unroll
            for (int t = 0; t < NT; ++t) x[i][t] = load_terms<false>(a[t], k0 + i * 32, f.K);
#pragma unroll
        for (int i = 0; i < FEW_AHEAD; ++i)
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    mma_16x8(acc[h][t], w[i][h][0].x, w[i][h][1].x, w[i][h][0].y, w[i][h][1].y, x[i][t].x, x[i][t].y);
                    mma_16x8(acc[h][t], w[i][h][0].z, w[i][h][1].z, w[i][h][0].w, w[i][h][1].w, x[i][t].z, x[i][t].w);
                }
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int t = 0; t < NT; ++t)
            *reinterpret_cast<float4*>(sums[warp][h][t][lane]) = make_float4(acc[h][t][0], acc[h][t][1], acc[h][t][2], acc[h][t][3]);
    __syncthreads();
    // value i of lane l: column n0 + l / 4 + 8 (i / 2) of the result, row 2 (l % 4) + i % 2 (of the group of 8)
    for (int i = threadIdx.x; i < NT * 128; i += 32 * W) {
        const int t = i >> 7, j = i & 127, l = ((j >> 3) & 7) * 4 + ((j >> 1) & 3), e = (j >> 6) * 2 + (j & 1);
        const int64_t n = n0 + (l >> 2) + 8 * (e >> 1);
        const int m = 8 * t + 2 * (l & 3) + (e & 1);
        if (m >= f.M || n >= f.N) continue;
        float v[H];
#pragma unroll
        for (int h = 0; h < H; ++h) {
            v[h] = sums[0][h][t][l][e];
#pragma unroll
            for (int q = 1; q < W; ++q) v[h] += sums[q][h][t][l][e];
        }
        if constexpr (KIND == GATE) {
            if (p.kept.at) {
                unsigned char* k = kept_block(p.kept, m, (int)n);
                const int col = (int)n & 31;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t bits = to24(v[h]);
                    *reinterpret_cast<uint16_t*>(k + h * 2048 + ((col >> 3) * 32 + m) * 16 + (col & 7) * 2) = (uint16_t)(bits >> 16);
                    k[4096 + h * 1024 + ((col >> 4) * 32 + m) * 16 + (col & 15)] = (unsigned char)(bits >> 8);
                }
            }
            with_act(p.act, [&](auto act) {
                float h, other;
                parts(mul2(act.value(two_of(v[0], v[0])), two_of(v[1], v[1])), h, other);
                static_cast<bf16*>(p.C)[m * p.ldc + n] = __float2bfloat16_rn(h);
            });
        } else {
            C* q = static_cast<C*>(p.C) + m * p.ldc + n;
            *q = (C)(p.accumulate ? (float)*q + v[0] : v[0]);
        }
    }
}
// Warps per block: enough for sixteen per SM, and for sums that stay within 256 additions.
template <int NT, int KIND, typename C>
cudaError_t launch_few(const FewParams& f, const Params& p, int num_sms, cudaStream_t s) {
    const int64_t blocks = (f.N + 15) / 16;
    const dim3 grid((unsigned)blocks);
    if (blocks * 4 >= 16 * num_sms && f.K <= FEW_TERMS / 4) return launch_pdl(few_rows_kernel<NT, 4, KIND, C>, grid, dim3(128), 0, s, f, p);
    if (blocks * 8 >= 16 * num_sms && f.K <= FEW_TERMS / 2) return launch_pdl(few_rows_kernel<NT, 8, KIND, C>, grid, dim3(256), 0, s, f, p);
    return launch_pdl(few_rows_kernel<NT, 16, KIND, C>, grid, dim3(512), 0, s, f, p);
}
template <int KIND, typename C>
cudaError_t launch_few_rows(const FewParams& f, const Params& p, int num_sms, cudaStream_t s) {
    return f.M <= 8 ? launch_few<1, KIND, C>(f, p, num_sms, s) : launch_few<2, KIND, C>(f, p, num_sms, s);
}

typedef void (*Kernel)(CUtensorMap, CUtensorMap, Params);
constexpr int MAX_SMEM = 232448, KERNELS = 12;

cudaError_t launch_one(Kernel kern, int which, int cluster, size_t smem, const CUtensorMap& ma, const CUtensorMap& mb, const Params& p, int grid, cudaStream_t s) {
    // Once per kernel and device (a call costs the host more than the rest of this function): every launch is allowed the most.
    static std::atomic<uint64_t> allowed[KERNELS];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
    if (!(allowed[which].load(std::memory_order_relaxed) & bit)) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SMEM);
        if (e != cudaSuccess) return e;
        allowed[which].fetch_or(bit, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = g_tune_pdl_off ? 0 : 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)cluster, 1, 1};
    cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, ma, mb, p);
}

// Tile and split, from a model of what was measured (ns, B200): a block of k costs 274 in a tile of 256 x 256 and 190 in one of 256 x 128, by pairs,
// and 238 in one of 128 x 128; a turn of tiles 1600, 950 and 950 more; pairs start 1150 and 800 later than single blocks; adding partial
// tiles up 300, 500 and 900 and for full tiles 3200, 1600 and 2000 more.  (M x N x K in us, forms in this order, alone and with the best split:
// 128 x 4096 x 2048: 15.2, 11.2, 12.0; 12.3 (3), 10.7 (2), 8.9 (4).  4096 x 4096 x 1024: 26.6, 30.0, 34.7.  256 x 256 x 8192: 41.4, 28.8,
// 34.5; 17.7 (4), 12.8 (4), 11.0 (8).)
// Clusters do not fill the GPU's groups of SMs: of 148 SMs those of 2, 3 .. 8 blocks were found to use 148, 135, 132, 130, 132, 105 and 120 at a
// time (one more cluster takes a second turn: 10.6 -> 18.9 us); the rule stays a little below that.
enum { PAIR_256 = 0, PAIR_128 = 1, SINGLE_128 = 2 };
struct Shape { int form, split; };
Shape choose_shape(int64_t M, int64_t N, int64_t kblocks, int num_sms) {
    static constexpr int BLOCK[3] = {274, 190, 238}, TURN[3] = {1600, 950, 950}, START[3] = {1150, 800, 0}, ADD[3] = {300, 500, 900}, ADD_FULL[3] = {3200, 1600, 2000};
    static constexpr int USABLE[MAX_SPLIT + 1] = {0, 100, 100, 85, 87, 81, 81, 66, 76};        // percent of the SMs, by the blocks of a cluster
    Shape best{PAIR_256, 1};
    int64_t cost = INT64_MAX;
    for (int form = 0; form < 3; ++form) {
        const int blocks = form == SINGLE_128 ? 1 : 2, rows = blocks * BM, columns = form == PAIR_256 ? 256 : 128;
        const int64_t tiles = ((M + rows - 1) / rows) * ((N + columns - 1) / columns);
        if (blocks > num_sms) continue;
        for (int q = 1; q * blocks <= MAX_SPLIT && q <= kblocks; ++q) {
            const int64_t slots = num_sms / (q * blocks);
            if (q > 1 && tiles * q * blocks * 100 > (int64_t)num_sms * USABLE[q * blocks]) break;
            const int64_t turns = q > 1 ? 1 : (tiles + slots - 1) / slots;
            const int64_t c = START[form] + turns * ((kblocks + q - 1) / q * BLOCK[form] + TURN[form]) + (q > 1 ? ADD[form] + ADD_FULL[form] * (M < rows ? M : rows) / rows : 0);
            if (c < cost) { cost = c; best = {form, q}; }
        }
    }
    return best;
}

template <int KIND, typename C>
Kernel kernel_of(int form) {
    return form == PAIR_256 ? matmul16_kernel<2, 256, KIND, C> : form == PAIR_128 ? matmul16_kernel<2, 128, KIND, C> : matmul16_kernel<1, 128, KIND, C>;
}

bool on(const void* p, int64_t ld, int64_t bytes, int64_t size) { return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * size % bytes == 0; }

// p: the output's part is filled in.  N: columns of the accumulators all tiles together (GATE: twice those of h).
cudaError_t launch(Params p, int kind, int type, const void* A, int64_t lda, bool trans_a, const void* B, int64_t ldb, bool trans_b, int64_t M, int64_t N, int64_t K,
                   int* status, int num_sms, cudaStream_t s, uint64_t* launches) {
    // (the blocks of few rows let the next kernel in before they wait: not where one follows that relies on their wait)
    if (kind != GRAD && !p.followed && !trans_a && trans_b && M <= FEW_ROWS && K <= FEW_TERMS && N * K * 2 <= FEW_BYTES) {
        const FewParams f = {static_cast<const bf16*>(A), static_cast<const bf16*>(B), lda, ldb, (int)M, (int)K, kind == GATE ? N / 2 : N};
        const cudaError_t e = kind == GATE ? launch_few_rows<GATE, bf16>(f, p, num_sms, s) : type == CERAR_TYPE_F32 ? launch_few_rows<PLAIN, float>(f, p, num_sms, s)
                                                                                             : launch_few_rows<PLAIN, bf16>(f, p, num_sms, s);
        if (e == cudaSuccess) ++*launches;
        return e;
    }
    if (!get_encode_fn()) return cudaErrorNotSupported;
    p.M = (int)M; p.kblocks = (int)((K + BK - 1) / BK); p.status = status;
    const Shape shape = choose_shape(M, N, p.kblocks, num_sms);
    const bool paired = shape.form != SINGLE_128;
    const int BN = shape.form == PAIR_256 ? 256 : 128, rows = paired ? 2 * BM : BM, columns = kind == GATE ? BN / 2 : BN;
    p.N = (int)(kind == GATE ? N / 2 : N);
    p.tiles_m = (p.M + rows - 1) / rows;
    p.tiles_n = (p.N + columns - 1) / columns;
    if ((int64_t)p.tiles_m * p.tiles_n > 0x3FFFFFFF) return cudaErrorInvalidConfiguration;
    p.tiles = (uint32_t)p.tiles_m * (uint32_t)p.tiles_n;
    p.split = shape.split;
    p.group_m = paired ? 8 : 16;
    const uint32_t stage = A_BYTES + (uint32_t)(paired ? BN / 2 : BN) * BK * 2;
    const size_t fixed = 1024 + EPI_WARPS * STAGING + 512;
    p.stages = (int)((MAX_SMEM - fixed) / stage);
    p.a_mn = trans_a; p.b_mn = !trans_b;
    const int a_rows = !p.a_mn && p.M < BM ? (p.M + 7) & ~7 : BM;
    p.a_bytes = (uint32_t)a_rows * BK * 2;
    CUtensorMap ma, mb;
    if (!make_map_16bit(&ma, A, trans_a ? K : M, trans_a ? M : K, lda, p.a_mn ? BK : a_rows) ||
        !make_map_16bit(&mb, B, trans_b ? N : K, trans_b ? K : N, ldb, 64))
        return cudaErrorInvalidValue;
    const int cluster = (paired ? 2 : 1) * p.split, most = num_sms / cluster;
    const int grid = cluster * (p.split > 1 || (int)p.tiles < most ? (int)p.tiles : most);
    p.early = p.split > 1 || (int64_t)p.tiles * cluster <= num_sms;      // (one turn: the next kernel's blocks come where this one's have left)
    const Kernel kern = kind == GATE ? kernel_of<GATE, bf16>(shape.form) : kind == GRAD ? kernel_of<GRAD, bf16>(shape.form)
                        : type == CERAR_TYPE_F32 ? kernel_of<PLAIN, float>(shape.form) : kernel_of<PLAIN, bf16>(shape.form);
    const int which = 3 * (kind == PLAIN ? (type == CERAR_TYPE_F32 ? 0 : 1) : kind + 1) + shape.form;
    const cudaError_t e = launch_one(kern, which, cluster, fixed + (size_t)p.stages * stage, ma, mb, p, grid, s);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace

int matmul16_tile(int64_t M, int64_t N, int64_t K, int num_sms, int* split) {
    const Shape shape = choose_shape(M, N, (K + BK - 1) / BK, num_sms);
    *split = shape.split;
    return shape.form;
}

cudaError_t launch_matmul16(const Matmul16Args& a, int num_sms, cudaStream_t s, uint64_t* launches) {
    Params p = {};
    const int64_t size = a.type == CERAR_TYPE_F32 ? 4 : 2;
    p.C = a.C; p.ldc = a.ldc; p.accumulate = a.accumulate; p.after = a.after; p.followed = a.followed;
    p.c_vec = on(a.C, a.ldc, 16, size);
    p.c_pair = on(a.C, a.ldc, 4, size);
    return launch(p, PLAIN, a.type, a.A, a.lda, a.trans_a, a.B, a.ldb, a.trans_b, a.M, a.N, a.K, a.status, num_sms, s, launches);
}

namespace {
Kept kept_of(const void* p, int64_t hidden) { return {static_cast<unsigned char*>(const_cast<void*>(p)), (hidden + 31) / 32}; }
}  // namespace
size_t gated_kept_bytes(int64_t tokens, int64_t hidden) { return (size_t)((tokens + 31) / 32) * (size_t)((hidden + 31) / 32) * KEPT_BLOCK; }

cudaError_t launch_gated_in(const GatedInArgs& a, int num_sms, cudaStream_t s, uint64_t* launches) {
    Params p = {};
    p.C = a.h; p.ldc = a.ldh; p.act = a.act;
    if (a.kept) p.kept = kept_of(a.kept, a.hidden);
    p.c_vec = on(a.h, a.ldh, 16, 2);
    return launch(p, GATE, CERAR_TYPE_BF16, a.x, a.ldx, false, a.w, a.ldw, true, a.tokens, 2 * a.hidden, a.width, a.status, num_sms, s, launches);
}

cudaError_t launch_gated_grad(const GatedGradArgs& a, int num_sms, cudaStream_t s, uint64_t* launches) {
    Params p = {};
    p.C = a.dgu; p.ldc = a.lddgu; p.kept = kept_of(a.kept, a.hidden); p.h = static_cast<bf16*>(a.h); p.ldh = a.ldh; p.act = a.act;
    p.four = on(a.dgu, a.lddgu, 8, 2) && (!a.h || on(a.h, a.ldh, 8, 2)) && a.hidden % 4 == 0;
    p.c_vec = on(a.dgu, a.lddgu, 16, 2) && (!a.h || on(a.h, a.ldh, 16, 2)) && a.hidden % 8 == 0;
    return launch(p, GRAD, CERAR_TYPE_BF16, a.dy, a.lddy, false, a.w, a.ldw, false, a.tokens, a.hidden, a.width, a.status, num_sms, s, launches);
}

// ---------------------------------------------------------------- copies to rows on 16-byte boundaries
//
// What tensor-map copies cannot read in place.  A thread writes 16 bytes and reads them as single elements (pairs, where rows start on 4-byte
// boundaries), of which the first-level cache serves all but the first.  Several matrices go in one launch.

namespace {
constexpr int ALIGN_THREADS = 256, ALIGN_CHUNKS = 4;
struct AlignItems {
    AlignArgs m[ALIGN_MAX];
    uint32_t first[ALIGN_MAX + 1];                     // blocks in front of each
};
__global__ void __launch_bounds__(ALIGN_THREADS) align_kernel(const AlignItems items) {
    grid_dependency_wait();
    int i = 0;
    while (blockIdx.x >= items.first[i + 1]) ++i;
    const AlignArgs& m = items.m[i];
    const uint32_t chunks = (uint32_t)(m.cols + 7) / 8;
    const int64_t total = m.rows * chunks;
    const bool pairs = (reinterpret_cast<uintptr_t>(m.src) & 3) == 0 && (m.ld & 1) == 0;
    int64_t at = (int64_t)(blockIdx.x - items.first[i]) * (ALIGN_THREADS * ALIGN_CHUNKS) + threadIdx.x;
    uint32_t w[ALIGN_CHUNKS][4];
    uint16_t* dst[ALIGN_CHUNKS];
#pragma unroll
    for (int c = 0; c < ALIGN_CHUNKS; ++c, at += ALIGN_THREADS) {
        dst[c] = nullptr;
        if (at >= total) continue;
        const int64_t row = total < 0x7FFFFFFF ? (int64_t)((uint32_t)at / chunks) : at / chunks;
        const int64_t col = (at - row * chunks) * 8;
        const uint16_t* src = static_cast<const uint16_t*>(m.src) + row * m.ld + col;
        dst[c] = static_cast<uint16_t*>(m.dst) + row * m.ldd + col;
        const int n = (int)(m.cols - col < 8 ? m.cols - col : 8);
        if (pairs && n == 8) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[c][e] = __ldg(reinterpret_cast<const uint32_t*>(src) + e);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[c][e] = (2 * e < n ? (uint32_t)__ldg(src + 2 * e) : 0u) | (2 * e + 1 < n ? (uint32_t)__ldg(src + 2 * e + 1) << 16 : 0u);
        }
    }
#pragma unroll
    for (int c = 0; c < ALIGN_CHUNKS; ++c)
        if (dst[c]) *reinterpret_cast<uint4*>(dst[c]) = make_uint4(w[c][0], w[c][1], w[c][2], w[c][3]);
}
}  // namespace

cudaError_t launch_align(const AlignArgs* items, int count, cudaStream_t s, uint64_t* launches) {
    AlignItems a = {};
    int64_t blocks = 0;
    for (int i = 0; i < count; ++i) {
        a.m[i] = items[i];
        blocks += (items[i].rows * ((items[i].cols + 7) / 8) + ALIGN_THREADS * ALIGN_CHUNKS - 1) / (ALIGN_THREADS * ALIGN_CHUNKS);
        if (blocks > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
        a.first[i + 1] = (uint32_t)blocks;
    }
    for (int i = count; i < ALIGN_MAX; ++i) a.first[i + 1] = (uint32_t)blocks;
    if (blocks == 0) return cudaSuccess;
    const cudaError_t e = launch_pdl(align_kernel, dim3((unsigned)blocks), dim3(ALIGN_THREADS), 0, s, a);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace cerar
