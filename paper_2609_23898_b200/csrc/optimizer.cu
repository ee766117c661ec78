// Gradient norm and AdamW over a set of tensors (cerar_grad_norm, cerar_adamw_step).
//
// Both are one pass over memory: the norm reads every gradient once (4 or 2 bytes per element), the step reads and writes each
// parameter and state once.  A set is cut into chunks of 2048 elements of one tensor each, in one list for all tensors, so one
// launch serves hundreds of tensors and every SM has work whatever their sizes; blocks take chunks in turn.
//
// In a chunk warp w owns the 256 elements 256 w .. 256 w + 255: lane l has elements 4 l .. 4 l + 3 and 128 + 4 l .. 128 + 4 l + 3 of
// them, so every access of a warp is contiguous, and the 256 elements that share a scale of the 8-bit states belong to one warp.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "kernels.cuh"
#include "ops.cuh"
#include "ptx.cuh"

namespace cerar {
namespace {

constexpr int THREADS = 256;
constexpr int PER_WARP = CERAR_STATE_BLOCK;
static_assert(CHUNK == (THREADS / 32) * PER_WARP, "one state block per warp and chunk");

// n (1..4) consecutive elements as binary32, the rest zero; vec: all four exist and are aligned
__device__ __forceinline__ void load4(float* x, const float* p, int n, bool vec) {
    if (vec) {
        const float4 v = __ldcs(reinterpret_cast<const float4*>(p));
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = j < n ? __ldcs(p + j) : 0.f;
    }
}
__device__ __forceinline__ void load4(float* x, const __nv_bfloat16* p, int n, bool vec) {
    if (vec) {
        const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p));
        x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xFFFF0000u);
        x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xFFFF0000u);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = j < n ? __bfloat162float(p[j]) : 0.f;
    }
}
__device__ __forceinline__ void store4(float* p, const float* x, int n, bool vec) {
    if (vec) {
        __stcs(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3]));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) if (j < n) p[j] = x[j];
    }
}
__device__ __forceinline__ void store4_bf16(__nv_bfloat16* p, const uint32_t* b, int n, bool vec) {   // b: 16-bit patterns
    if (vec) {
        __stcs(reinterpret_cast<uint2*>(p), make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16)));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) if (j < n) reinterpret_cast<uint16_t*>(p)[j] = (uint16_t)b[j];
    }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int n, bool vec) {
    if (vec) return __ldcs(reinterpret_cast<const uint32_t*>(p));
    uint32_t v = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) if (j < n) v |= (uint32_t)p[j] << (8 * j);
    return v;
}
__device__ __forceinline__ void store_codes(uint8_t* p, uint32_t v, int n, bool vec) {
    if (vec) { __stcs(reinterpret_cast<uint32_t*>(p), v); return; }
#pragma unroll
    for (int j = 0; j < 4; ++j) if (j < n) p[j] = (uint8_t)(v >> (8 * j));
}

// ---------------------------------------------------------------- gradient norm

__device__ __forceinline__ double block_sum(double s, double* sh) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) s += sh[w];
    __syncthreads();
    return s;
}

// Squares are summed eight at a time in binary32 and from there in binary64.  A group whose sum leaves the range where
// binary32 squares are good (overflow, underflow, NaN) is done again in binary64 from the registers.
__device__ __forceinline__ double sum8(const float* x) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(x[j], x[j], s);
    if (s > 1e-25f && s < 1e37f) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) d = fma((double)x[j], (double)x[j], d);
    return d;
}

// Sum over n consecutive gradients of what this thread reads of them.  The order does not matter here, so a run that starts
// off a 16-byte boundary is read from the boundary below on, in whole groups of four elements that hold at least one of the run's,
// and what does not belong to the run counts as zero.
template <typename G>
__device__ __forceinline__ double sum_squares(const G* g, int n) {
    constexpr uintptr_t GROUP = 4 * sizeof(G);
    const int head = (int)((reinterpret_cast<uintptr_t>(g) & (GROUP - 1)) / sizeof(G));
    g -= head;
    n += head;
    double sum = 0.0;
    for (int at = (int)(threadIdx.x >> 5) * PER_WARP + 4 * (int)(threadIdx.x & 31); at < n; at += CHUNK) {
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        load4(x, g + at, 4, true);
        if (at + 128 < n) load4(x + 4, g + at + 128, 4, true);
        if (at < head || at + 132 > n) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = at + (j & 3) + (j >> 2) * 128;
                if (i < head || i >= n) x[j] = 0.f;
            }
        }
        sum += sum8(x);
    }
    return sum;
}

__global__ void __launch_bounds__(THREADS) grad_norm_kernel(const __grid_constant__ NormArgs a) {
    __shared__ double sh[THREADS / 32];
    __shared__ bool last;
    ptx::grid_dependency_wait();
    double sum = 0.0;
    for (int64_t c = blockIdx.x; c < a.nchunks; c += gridDim.x) {
        const ChunkRef ref = a.chunks[c];
        const TensorRec& t = a.tensors[ref.tensor];
        const int64_t begin = (int64_t)ref.index * CHUNK;
        const int64_t n = t.numel - begin < (int64_t)a.steps * CHUNK ? t.numel - begin : (int64_t)a.steps * CHUNK;
        if (t.grad_type == CERAR_TYPE_F32) sum += sum_squares(static_cast<const float*>(t.grad) + begin, (int)n);
        else sum += sum_squares(static_cast<const __nv_bfloat16*>(t.grad) + begin, (int)n);
    }
    sum = block_sum(sum, sh);
    // the block that arrives last adds the partial sums of all blocks, in their order
    if (threadIdx.x == 0) {
        a.partial[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double s = 0.0;
    for (unsigned b = threadIdx.x; b < gridDim.x; b += THREADS) s += __ldcg(a.partial + b);
    s = block_sum(s, sh);
    if (threadIdx.x == 0) {
        const float norm = (float)sqrt(s);
        const bool finite = norm <= 3.4028234e38f;                     // false for NaN too
        a.clip[0] = norm;
        a.clip[1] = !finite ? 0.f : a.max_norm > 0.f ? fminf(1.f, a.max_norm / (norm + 1e-6f)) : 1.f;
        a.clip[2] = finite ? 1.f : 0.f;
        *a.ticket = 0u;
    }
}

// ---------------------------------------------------------------- AdamW

// Multiply and xor-shift rounds: every input bit reaches every output bit.  Shifts and multipliers are published: C. Wellons, "Prospecting
// for Hash Functions", 2018 (a search for 32-bit hashes of this form with little bias).
__device__ __forceinline__ uint32_t scramble(uint32_t h) {
    h = (h ^ (h >> 16)) * 0x7FEB352Du;
    h = (h ^ (h >> 15)) * 0x846CA68Bu;
    return h ^ (h >> 16);
}
// random bits of a state block; element i of it then uses scramble(key + i * 0x9E3779B9)
__device__ __forceinline__ uint32_t block_key(int64_t block, uint64_t seed, uint32_t stream) {
    return scramble((uint32_t)block * 0x9E3779B1u + ((uint32_t)(block >> 32) + 1u) * 0x7FEB352Du + (uint32_t)seed * 0x85157AF5u +
                    (uint32_t)(seed >> 32) * 0xC2B2AE35u + stream * 0x632BE5ABu);
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Two binary32 numbers in a 64-bit register and the instructions that work on both.
__device__ __forceinline__ uint64_t two(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void split2(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2x(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// Values of four e4m3 codes times a scale (the conversion goes through binary16, which holds them all).
__device__ __forceinline__ void code_values(uint32_t codes, float scale, float* x) {
    uint32_t lo, hi;
    asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}\n" : "=r"(lo), "=r"(hi) : "r"(codes));
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    const uint64_t s2 = two(scale, scale);
    split2(mul2(two(a.x, a.y), s2), x[0], x[1]);
    split2(mul2(two(b.x, b.y), s2), x[2], x[3]);
}
__device__ __forceinline__ float max_nan(float a, float b) {           // NaN if one of them is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t sign_bytes(float a, float b) {     // bytes 0 and 1: 0xFF where a, b are negative, else 0
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, 0xFBFB;" : "=r"(r) : "r"(__float_as_uint(a)), "r"(__float_as_uint(b)));
    return r;
}
__device__ __forceinline__ uint32_t bytes4(const uint32_t* c) {        // four numbers below 256 in the bytes of a word
    return __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
}
__device__ __forceinline__ float pick(const float* x, int j) {         // x[j] of eight, without an array in memory
    float v = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) v = j == i ? x[i] : v;
    return v;
}
// Moments below this (2^14) have a scale exponent up to 6, so that 2^-e 2^-120 is a normal binary32 number.
constexpr uint32_t LARGE_STATE = (127u + 14u) << 23;
// Code of y, |y| <= 448, rounded away from zero with the probability of the part that is cut off: times 2^-120 the code is the
// top of the binary32 number, and 16 random bits (plus half of their last place) are added to the 20 bits below it.
__device__ __forceinline__ uint32_t random_code(float y, uint32_t bits16) {
    const uint32_t b = __float_as_uint(y), sign = (b >> 24) & 0x80u;
    if ((b & 0x7FFFFFFFu) >= 0x7F800000u) return sign | 0x7Fu;
    const uint32_t c = (__float_as_uint(fabsf(y) * 0x1p-120f) + ((bits16 << 4) + 8u)) >> 20;
    return sign | min(c, 0x7Eu);
}
__device__ __forceinline__ uint32_t finite_magnitude(float x) {
    const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
}

// FULL: all 256 elements exist and everything but the gradient is aligned for four at a time; nothing is checked element by element.
template <int PK, typename G, int BITS, bool FULL>
__device__ __forceinline__ void adamw_warp(const AdamwArgs& a, const TensorRec& t, int64_t e0 /* first element of the warp's block */, float coef,
                                           bool vec, bool gvec) {
    const int lane = threadIdx.x & 31;
    const int64_t left = t.numel - e0 - 4 * lane;
    const int n0 = FULL || left >= 4 ? 4 : (int)max((int64_t)0, left), n1 = FULL || left >= 132 ? 4 : (int)max((int64_t)0, left - 128);
    const int64_t i0 = e0 + 4 * lane, i1 = i0 + 128;
    const bool v0 = FULL || (vec && n0 == 4), v1 = FULL || (vec && n1 == 4), g0 = gvec && n0 == 4, g1 = gvec && n1 == 4;
    float g[8], p[8], m[8], v[8];
    uint32_t mc[2], vc[2];
    float msc = 0.f, vsc = 0.f;
    const G* gp = static_cast<const G*>(t.grad);
    load4(g, gp + i0, n0, g0);
    load4(g + 4, gp + i1, n1, g1);
    if constexpr (PK == PARAM_BF16) {
        const __nv_bfloat16* pp = static_cast<const __nv_bfloat16*>(t.param);
        load4(p, pp + i0, n0, v0);
        load4(p + 4, pp + i1, n1, v1);
    } else {
        const float* pp = PK == PARAM_MASTER ? t.master : static_cast<const float*>(t.param);
        load4(p, pp + i0, n0, v0);
        load4(p + 4, pp + i1, n1, v1);
    }
    if constexpr (BITS == 32) {
        load4(m, static_cast<const float*>(t.m) + i0, n0, v0);
        load4(m + 4, static_cast<const float*>(t.m) + i1, n1, v1);
        load4(v, static_cast<const float*>(t.v) + i0, n0, v0);
        load4(v + 4, static_cast<const float*>(t.v) + i1, n1, v1);
    } else {
        mc[0] = load_codes(static_cast<const uint8_t*>(t.m) + i0, n0, v0);
        mc[1] = load_codes(static_cast<const uint8_t*>(t.m) + i1, n1, v1);
        vc[0] = load_codes(static_cast<const uint8_t*>(t.v) + i0, n0, v0);
        vc[1] = load_codes(static_cast<const uint8_t*>(t.v) + i1, n1, v1);
        msc = t.m_scale[e0 / PER_WARP];
        vsc = t.v_scale[e0 / PER_WARP];
        code_values(mc[0], msc, m);
        code_values(mc[1], msc, m + 4);
        code_values(vc[0], vsc, v);
        code_values(vc[1], vsc, v + 4);
#pragma unroll
        for (int j = 0; j < 8; j += 2) split2(mul2(two(v[j], v[j + 1]), two(v[j], v[j + 1])), v[j], v[j + 1]);
    }
    const float step = a.step_size * t.lr_scale, keep = 1.f - a.lr * t.lr_scale * t.weight_decay;
    const uint64_t coef2 = two(coef, coef), b1 = two(a.beta1, a.beta1), c1 = two(a.one_minus_beta1, a.one_minus_beta1), b2 = two(a.beta2, a.beta2),
                   c2 = two(a.one_minus_beta2, a.one_minus_beta2), keep2 = two(keep, keep), rs2 = two(a.root_scale, a.root_scale), eps2 = two(a.eps, a.eps);
    // a b + (-0) rounded once is the product a b; written as a product it is contracted with the sum behind it, and the states differ
    // in the last place from the formula's, now and then in the code that is kept.  -0 comes from the host: known here, it is folded away
    const uint64_t nil = two(a.minus_zero, a.minus_zero);
    float r[8];
    float mtop = 0.f, rtop = 0.f;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        // two elements per instruction; each product and sum rounded by itself (no contraction), as the formula is written
        const uint64_t g2 = mul2(two(g[j], g[j + 1]), coef2);
        const uint64_t m2 = add2(fma2x(two(m[j], m[j + 1]), b1, nil), fma2x(g2, c1, nil));
        const uint64_t v2 = add2(fma2x(two(v[j], v[j + 1]), b2, nil), fma2x(mul2(g2, g2), c2, nil));
        split2(m2, m[j], m[j + 1]);
        split2(v2, v[j], v[j + 1]);
#pragma unroll
        for (int i = j; i < j + 2; ++i) {
            // The root of an 8-bit state decides which code is kept and is rounded to nearest.  Otherwise only the update sees it, and it
            // is an approximation (2^-23), as the quotient below is (2 units in the last place): the update is within 2^-21 of the formula's,
            // and usually far smaller than the parameter it is added to.  Rounded to nearest both are branches, eight of each per
            // thread: 65,536 elements 3.95 -> 4.32 us, bfloat16 parameters without copies 900 -> 983 (2.7e8 elements, 32-bit states) and
            // 957 -> 1000 (8-bit states), while 1.41e9 binary32 elements gain (6240 -> 5960).
            if constexpr (BITS == 8) r[i] = __fsqrt_rn(v[i]);
            else asm("sqrt.approx.f32 %0, %1;" : "=f"(r[i]) : "f"(v[i]));
        }
        float d0, d1, q0, q1;
        split2(fma2x(two(r[j], r[j + 1]), rs2, eps2), d0, d1);
        split2(mul2(two(p[j], p[j + 1]), keep2), q0, q1);
        p[j] = fmaf(-step, __fdividef(m[j], d0), q0);
        p[j + 1] = fmaf(-step, __fdividef(m[j + 1], d1), q1);
        if constexpr (BITS == 8) {
            mtop = max_nan(mtop, max_nan(fabsf(m[j]), fabsf(m[j + 1])));
            rtop = max_nan(rtop, max_nan(r[j], r[j + 1]));
        }
    }
    if constexpr (BITS == 32) {
        store4(static_cast<float*>(t.m) + i0, m, n0, v0);
        store4(static_cast<float*>(t.m) + i1, m + 4, n1, v1);
        store4(static_cast<float*>(t.v) + i0, v, n0, v0);
        store4(static_cast<float*>(t.v) + i1, v + 4, n1, v1);
    } else {
        uint32_t mmax = __reduce_max_sync(0xffffffffu, __float_as_uint(mtop)), rmax = __reduce_max_sync(0xffffffffu, __float_as_uint(rtop));
        const uint32_t key = block_key(t.block0 + e0 / PER_WARP, a.seed, 0u) + (uint32_t)lane * (4u * 0x9E3779B9u);
        int em, er;
        mc[0] = mc[1] = vc[0] = vc[1] = 0u;
        if (mmax < LARGE_STATE && rmax < LARGE_STATE) {
            // everything is finite, and 2^-e 2^-120 is a number: one product brings the code to the top of the binary32 number
            em = fp8_scale_exponent(mmax);
            er = fp8_scale_exponent(rmax);
            const float im = pow2f(-em) * 0x1p-120f, ir = pow2f(-er) * 0x1p-120f;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                uint32_t cm[4], cr[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = 4 * q + i;
                    const uint32_t h = scramble(key + (uint32_t)(q * 128 + i) * 0x9E3779B9u);
                    cm[i] = (__float_as_uint(fabsf(m[j]) * im) + (((h >> 12) & 0xFFFF0u) | 8u)) >> 20;
                    cr[i] = max((__float_as_uint(r[j] * ir) + (((h << 4) & 0xFFFF0u) | 8u)) >> 20, min(__float_as_uint(r[j]), 1u));
                }
                // four codes to a word; the signs come from the top bytes of m, spread over a byte each by the permutation
                const uint32_t neg = __byte_perm(sign_bytes(m[4 * q], m[4 * q + 1]), sign_bytes(m[4 * q + 2], m[4 * q + 3]), 0x5410);
                mc[q] = bytes4(cm) | (neg & 0x80808080u);
                vc[q] = bytes4(cr);
            }
        } else {
            mmax = rmax = 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j) { mmax = max(mmax, finite_magnitude(m[j])); rmax = max(rmax, finite_magnitude(r[j])); }
            em = fp8_scale_exponent(__reduce_max_sync(0xffffffffu, mmax));
            er = fp8_scale_exponent(__reduce_max_sync(0xffffffffu, rmax));
            const float im = pow2f(-em), ir = pow2f(-er);
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
                const uint32_t h = scramble(key + (uint32_t)((j >> 2) * 128 + (j & 3)) * 0x9E3779B9u);
                const float mj = pick(m, j), rj = pick(r, j);
                const uint32_t cm = random_code(mj * im, h >> 16) << (8 * (j & 3));
                uint32_t c = random_code(rj * ir, h & 0xFFFFu);
                if (rj > 0.f) c = max(c, 1u);
                c <<= 8 * (j & 3);
                if (j < 4) { mc[0] |= cm; vc[0] |= c; } else { mc[1] |= cm; vc[1] |= c; }
            }
        }
        store_codes(static_cast<uint8_t*>(t.m) + i0, mc[0], n0, v0);
        store_codes(static_cast<uint8_t*>(t.m) + i1, mc[1], n1, v1);
        store_codes(static_cast<uint8_t*>(t.v) + i0, vc[0], n0, v0);
        store_codes(static_cast<uint8_t*>(t.v) + i1, vc[1], n1, v1);
        if (lane == 0) { t.m_scale[e0 / PER_WARP] = pow2f(em); t.v_scale[e0 / PER_WARP] = pow2f(er); }
    }
    if constexpr (PK == PARAM_F32 || PK == PARAM_MASTER) {
        float* pp = PK == PARAM_MASTER ? t.master : static_cast<float*>(t.param);
        store4(pp + i0, p, n0, v0);
        store4(pp + i1, p + 4, n1, v1);
    }
    if constexpr (PK == PARAM_MASTER || PK == PARAM_BF16) {
        // the copy is rounded to nearest; a parameter without one is rounded up or down at random, since a step is far
        // smaller than the distance of two bfloat16 numbers (0.4 %) and rounding to nearest would lose it every time
        const uint32_t key = PK == PARAM_BF16 ? block_key(t.block0 + e0 / PER_WARP, a.seed, 1u) : 0u;
        uint32_t b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (PK == PARAM_MASTER) {
                b[j] = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(p[j]));
            } else {
                const uint32_t h = scramble(key + (uint32_t)((j >> 2) * 128 + 4 * lane + (j & 3)) * 0x9E3779B9u);
                const uint32_t u = __float_as_uint(p[j]);
                b[j] = (u & 0x7FFFFFFFu) >= 0x7F800000u ? (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(p[j])) : (u + (h >> 16)) >> 16;
            }
        }
        __nv_bfloat16* pp = static_cast<__nv_bfloat16*>(t.param);
        store4_bf16(pp + i0, b, n0, v0);
        store4_bf16(pp + i1, b + 4, n1, v1);
    }
}

// Blocks per SM: two where the step streams 28 bytes per element and more (longer runs of each, 6.4 against 6.2 TB/s for binary32
// parameters and states), else four.
template <int PK, int BITS>
constexpr int blocks_per_sm() { return BITS == 32 && PK != PARAM_BF16 ? 2 : 4; }

template <int PK, typename G, int BITS>
__global__ void __launch_bounds__(THREADS, (blocks_per_sm<PK, BITS>())) adamw_kernel(const __grid_constant__ AdamwArgs a) {
    ptx::grid_dependency_wait();
    float coef = 1.f;
    if (a.clip) {
        if (a.clip[2] == 0.f) return;
        coef = a.clip[1];
    }
    const int warp = threadIdx.x >> 5;
    for (int64_t c = blockIdx.x; c < a.nchunks; c += gridDim.x) {
        const ChunkRef ref = a.chunks[c];
        const TensorRec t = a.tensors[ref.tensor];
        int64_t e0 = (int64_t)ref.index * CHUNK + warp * PER_WARP;
#pragma unroll 1
        for (int step = 0; step < (BITS == 32 ? a.steps : 1) && e0 < t.numel; ++step, e0 += CHUNK) {
            if ((BITS == 8 || PK != PARAM_BF16) && t.vec && e0 + PER_WARP <= t.numel) adamw_warp<PK, G, BITS, true>(a, t, e0, coef, true, t.gvec);
            else adamw_warp<PK, G, BITS, false>(a, t, e0, coef, t.vec, t.gvec);
        }
    }
}

struct GradPointers { void* p[SET_GRADS_MAX]; };
__global__ void set_grads_kernel(TensorRec* tensors, int64_t first, int count, const __grid_constant__ GradPointers g) {
    ptx::grid_dependency_wait();
    if ((int)threadIdx.x >= count) return;
    TensorRec& t = tensors[first + threadIdx.x];
    t.grad = g.p[threadIdx.x];
    t.gvec = grad_vec(t.grad, t.grad_type);
}

template <int PK, typename G, int BITS>
cudaError_t launch_kind(const AdamwArgs& a, int num_sms, cudaStream_t s) {
    const int64_t most = (int64_t)num_sms * blocks_per_sm<PK, BITS>(), blocks = a.nchunks < most ? a.nchunks : most;
    return launch_pdl(adamw_kernel<PK, G, BITS>, dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
}
template <int PK>
cudaError_t launch_types(const AdamwArgs& a, int grad_type, int bits, int num_sms, cudaStream_t s) {
    if (grad_type == CERAR_TYPE_F32)
        return bits == 32 ? launch_kind<PK, float, 32>(a, num_sms, s) : launch_kind<PK, float, 8>(a, num_sms, s);
    return bits == 32 ? launch_kind<PK, __nv_bfloat16, 32>(a, num_sms, s) : launch_kind<PK, __nv_bfloat16, 8>(a, num_sms, s);
}

}  // namespace

cudaError_t launch_grad_norm(const NormArgs& a, int blocks, cudaStream_t s, uint64_t* launches) {
    const cudaError_t e = launch_pdl(grad_norm_kernel, dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
    if (e == cudaSuccess) ++*launches;
    return e;
}

cudaError_t launch_adamw(const AdamwArgs& a, int param_kind, int grad_type, int state_bits, int num_sms, cudaStream_t s,
                         uint64_t* launches) {
    if (a.nchunks == 0) return cudaSuccess;
    const cudaError_t e = param_kind == PARAM_F32    ? launch_types<PARAM_F32>(a, grad_type, state_bits, num_sms, s)
                          : param_kind == PARAM_BF16 ? launch_types<PARAM_BF16>(a, grad_type, state_bits, num_sms, s)
                                                     : launch_types<PARAM_MASTER>(a, grad_type, state_bits, num_sms, s);
    if (e == cudaSuccess) ++*launches;
    return e;
}

cudaError_t launch_set_grads(TensorRec* tensors, int64_t first, int count, void* const* grads, cudaStream_t s, uint64_t* launches) {
    GradPointers g = {};
    for (int i = 0; i < count; ++i) g.p[i] = grads[i];
    const cudaError_t e = launch_pdl(set_grads_kernel, dim3(1), dim3(SET_GRADS_MAX), 0, s, tensors, first, count, g);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace cerar
