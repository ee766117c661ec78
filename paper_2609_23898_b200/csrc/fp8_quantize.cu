// Conversion of a matrix to 8 bits with a power-of-two scale per 128 values (cerar_fp8_quantize).
//
//   s = 2^e, e = min { e : max |x| 2^-e <= 448 } over a block;   code = e4m3(x 2^-e), nearest even
//
// x 2^-e is exact in binary32 (away from underflow), so the only rounding is that of the code.  A block is
// 128 values of a row, 128 values of a column, or 128 x 128 values; every wanted form is made from one
// reading of x.  Nothing but bytes bounds this: 2 or 4 in, 1 out per form and element.
//
// One CTA per 128 x 128 tile, the tile in registers: a warp holds 16 (or 8) consecutive rows, lane l the columns 4 l .. 4 l + 3 of
// each, so a warp reads whole row segments (256 or 512 contiguous bytes) and stores 128.
// A row's maximum is one warp reduction; a column's goes through shared memory once; all forms are stored row-major, as the
// products read them, so nothing is transposed.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "kernels.cuh"
#include "ops.cuh"
#include "ptx.cuh"

namespace cerar {
namespace {

constexpr int T = FP8_BLOCK;             // tile edge
// Warps of a CTA and CTAs per SM: what keeps a tile's values in registers and as many loads on their way as possible.  Measured
// (16384 x 8192, by row / by column / both, TB/s): bfloat16 8 warps x 3 6.1 / 6.0 / 5.5, 8 x 4 6.4 / 6.3 / 4.4 (spills with two forms),
// 8 x 2 6.1 / 4.9 / 4.9; binary32 16 x 2 6.7 / 5.8 / 5.9, 16 x 1 6.7 / 4.0 / 4.4.
template <typename X> constexpr int kWarps = sizeof(X) == 2 ? 8 : 16;
template <typename X, int FORMS> constexpr int kPerSm = sizeof(X) == 4 ? 2 : (FORMS & (FORMS - 1)) == 0 ? 4 : 3;
constexpr uint32_t INF = 0x7F800000u;

__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Four values of one row as they are in memory; their largest magnitudes, column by column (Top) and together (row_top), as the
// bit patterns of binary32 numbers, which order like the magnitudes, with infinity and NaN above all numbers.
template <typename X> struct Four;
template <> struct Four<float> {
    float4 v;
    struct Top { float t[4] = {0.f, 0.f, 0.f, 0.f}; };
    static __device__ __forceinline__ float larger(float a, float b) {    // NaN if one of them is
        float r;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
        return r;
    }
    static __device__ __forceinline__ float finite(float x) { return (__float_as_uint(x) & 0x7FFFFFFFu) < INF ? x : 0.f; }
    __device__ __forceinline__ void clear() { v = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const float* p) { v = __ldcs(reinterpret_cast<const float4*>(p)); }
    // from an address that is not on a 16-byte boundary: the two groups of 16 bytes that hold the four values
    __device__ __forceinline__ void load_across(const float* p) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15;
        const float4 w = __ldg(reinterpret_cast<const float4*>(a)), u = __ldg(reinterpret_cast<const float4*>(a) + 1);
        switch ((reinterpret_cast<uintptr_t>(p) >> 2) & 3u) {
            case 1: v = make_float4(w.y, w.z, w.w, u.x); break;
            case 2: v = make_float4(w.z, w.w, u.x, u.y); break;
            default: v = make_float4(w.w, u.x, u.y, u.z); break;
        }
    }
    static constexpr uintptr_t GROUP = 15;
    __device__ __forceinline__ void set(int j, float x) { (&v.x)[j] = x; }
    __device__ __forceinline__ void get(float* x) const { x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
    __device__ __forceinline__ Four finite_only() const { Four f; f.v = make_float4(finite(v.x), finite(v.y), finite(v.z), finite(v.w)); return f; }
    __device__ __forceinline__ void fold(Top& t) const {
        t.t[0] = larger(t.t[0], fabsf(v.x)); t.t[1] = larger(t.t[1], fabsf(v.y));
        t.t[2] = larger(t.t[2], fabsf(v.z)); t.t[3] = larger(t.t[3], fabsf(v.w));
    }
    __device__ __forceinline__ uint32_t row_top() const {
        return __float_as_uint(larger(larger(fabsf(v.x), fabsf(v.y)), larger(fabsf(v.z), fabsf(v.w))));
    }
    static __device__ __forceinline__ void bits(const Top& t, uint32_t* b) {
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = __float_as_uint(t.t[j]);
    }
};
template <> struct Four<__nv_bfloat16> {
    uint2 v;
    struct Top { uint32_t x = 0u, y = 0u; };                              // two 16-bit patterns each
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ uint32_t finite(uint32_t x) {
        return ((x & 0x7F80u) == 0x7F80u ? 0u : x & 0xFFFFu) | ((x & 0x7F800000u) == 0x7F800000u ? 0u : x & 0xFFFF0000u);
    }
    __device__ __forceinline__ void clear() { v = make_uint2(0u, 0u); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = __ldcs(reinterpret_cast<const uint2*>(p)); }
    __device__ __forceinline__ void load_across(const __nv_bfloat16* p) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)7;
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(a)), u = __ldg(reinterpret_cast<const uint2*>(a) + 1);
        switch ((reinterpret_cast<uintptr_t>(p) >> 1) & 3u) {
            case 1: v = make_uint2(__funnelshift_r(w.x, w.y, 16), __funnelshift_r(w.y, u.x, 16)); break;
            case 2: v = make_uint2(w.y, u.x); break;
            default: v = make_uint2(__funnelshift_r(w.y, u.x, 16), __funnelshift_r(u.x, u.y, 16)); break;
        }
    }
    static constexpr uintptr_t GROUP = 7;
    __device__ __forceinline__ void set(int j, __nv_bfloat16 x) {
        const uint32_t b = (uint32_t)__bfloat16_as_ushort(x) << (16 * (j & 1));
        if (j < 2) v.x |= b; else v.y |= b;
    }
    __device__ __forceinline__ void get(float* x) const {
        x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xFFFF0000u);
        x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xFFFF0000u);
    }
    __device__ __forceinline__ Four finite_only() const { Four f; f.v = make_uint2(finite(v.x), finite(v.y)); return f; }
    __device__ __forceinline__ void fold(Top& t) const { t.x = larger(t.x, v.x & 0x7FFF7FFFu); t.y = larger(t.y, v.y & 0x7FFF7FFFu); }
    __device__ __forceinline__ uint32_t row_top() const {
        const uint32_t h = larger(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu);
        return max(h << 16, h & 0xFFFF0000u);
    }
    static __device__ __forceinline__ void bits(const Top& t, uint32_t* b) {
        b[0] = t.x << 16; b[1] = t.x & 0xFFFF0000u; b[2] = t.y << 16; b[3] = t.y & 0xFFFF0000u;
    }
};

// Four scaled values to four codes.  BAD: there may be values that are not finite, which become NaN: x * 0 is NaN exactly there
// (the conversion by itself would turn an infinity into 448).
template <bool BAD>
__device__ __forceinline__ uint32_t codes4(const float* x, const float* inv) {
    uint16_t lo, hi;
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = BAD ? fmaf(x[j], inv[j], x[j] * 0.f) : x[j] * inv[j];
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(y[1]), "f"(y[0]));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(y[3]), "f"(y[2]));
    uint32_t r;
    asm("mov.b32 %0, {%1, %2};" : "=r"(r) : "h"(lo), "h"(hi));
    return r;
}
__device__ __forceinline__ void store_codes(uint8_t* dst, uint32_t v, int n) {
    if (n >= 4) { *reinterpret_cast<uint32_t*>(dst) = v; return; }
#pragma unroll
    for (int j = 0; j < 3; ++j) if (j < n) dst[j] = (uint8_t)(v >> (8 * j));
}

// FORMS: bit per cerar_scaling_t
template <typename X, int FORMS>
__global__ void __launch_bounds__(32 * kWarps<X>, (kPerSm<X, FORMS>)) fp8_quantize_kernel(const __grid_constant__ QuantizeArgs a, uint32_t tiles_c) {
    constexpr int WARPS = kWarps<X>, ROWS = T / WARPS;
    constexpr bool BY_ROW = FORMS & (1 << CERAR_BY_ROW), BY_COL = FORMS & (1 << CERAR_BY_COLUMN), BY_BLK = FORMS & (1 << CERAR_BY_BLOCK);
    __shared__ uint32_t colmax[BY_COL || BY_BLK ? WARPS : 1][T];
    ptx::grid_dependency_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
    const int64_t r0 = (int64_t)tr * T + warp * ROWS, c0 = (int64_t)tc * T + 4 * lane;
    const int64_t left = a.cols - c0;
    const int nc = left >= 4 ? 4 : left > 0 ? (int)left : 0;          // columns of this thread that exist
    const int nr = (int)(a.rows - r0 < ROWS ? (a.rows > r0 ? a.rows - r0 : 0) : ROWS);   // rows of this warp that exist

    Four<X> v[ROWS];
    const X* src = static_cast<const X*>(a.x) + r0 * a.ldx + c0;
    // a tile inside the matrix needs no bounds, row by row (the same for the whole CTA)
    const bool whole = (int64_t)(tr + 1) * T <= a.rows && (int64_t)(tc + 1) * T <= a.cols;
    if (whole && a.vec) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i, src += a.ldx) v[i].load(src);
    } else if (a.vec && nc == 4) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            v[i].clear();
            if (i < nr) v[i].load(src + i * a.ldx);
        }
    } else if (nc == 4) {
        // rows that start anywhere: where they start is the same for the whole warp, row by row
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const X* p = src + i * a.ldx;
            v[i].clear();
            if (i < nr) {
                if ((reinterpret_cast<uintptr_t>(p) & Four<X>::GROUP) == 0) v[i].load(p);
                else v[i].load_across(p);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            v[i].clear();
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i < nr && j < nc) v[i].set(j, src[i * a.ldx + j]);
        }
    }

    // largest magnitudes: of each of this lane's columns, and lane i's of row i (lanes 0 .. ROWS - 1)
    typename Four<X>::Top top;
    uint32_t cm[4], row_top = 0u;
    auto look = [&](auto finite_only) {
        top = typename Four<X>::Top();
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const Four<X> f = decltype(finite_only)::value ? v[i].finite_only() : v[i];
            if constexpr (BY_COL || BY_BLK) f.fold(top);
            if constexpr (BY_ROW) {
                const uint32_t t = __reduce_max_sync(0xffffffffu, f.row_top());
                if (lane == i) row_top = t;
            }
        }
        Four<X>::bits(top, cm);
    };
    look(std::false_type());
    const bool bad = __any_sync(0xffffffffu, BY_ROW ? row_top >= INF : max(max(cm[0], cm[1]), max(cm[2], cm[3])) >= INF);
    if (bad) look(std::true_type());                                    // rare: once more, over the finite values only

    auto put = [&](int form, auto inv_of_row) {
        uint8_t* dst = a.codes[form] + r0 * a.ld[form] + c0;
        const int64_t ld = a.ld[form];
        if (whole && !bad) {
#pragma unroll
            for (int i = 0; i < ROWS; ++i, dst += ld) {
                float x[4], inv[4];
                v[i].get(x);
                inv_of_row(i, inv);
                *reinterpret_cast<uint32_t*>(dst) = codes4<false>(x, inv);
            }
        } else {
#pragma unroll
            for (int i = 0; i < ROWS; ++i, dst += ld) {
                float x[4], inv[4];
                v[i].get(x);
                inv_of_row(i, inv);
                const uint32_t q = codes4<true>(x, inv);
                if (i < nr) store_codes(dst, q, nc);
            }
        }
    };
    if constexpr (BY_ROW) {
        const int e = fp8_scale_exponent(row_top);
        const float inv = pow2f(-e);
        if (lane < nr) a.scales[CERAR_BY_ROW][tc * a.lds[CERAR_BY_ROW] + r0 + lane] = pow2f(e);
        put(CERAR_BY_ROW, [&](int i, float* k) { k[0] = k[1] = k[2] = k[3] = __shfl_sync(0xffffffffu, inv, i); });
    }
    if constexpr (BY_COL || BY_BLK) {
        *reinterpret_cast<uint4*>(&colmax[warp][4 * lane]) = make_uint4(cm[0], cm[1], cm[2], cm[3]);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const uint4 q = *reinterpret_cast<const uint4*>(&colmax[w][4 * lane]);
            cm[0] = max(cm[0], q.x); cm[1] = max(cm[1], q.y); cm[2] = max(cm[2], q.z); cm[3] = max(cm[3], q.w);
        }
    }
    if constexpr (BY_COL) {
        float inv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = fp8_scale_exponent(cm[j]);
            inv[j] = pow2f(-e);
            if (warp == 0 && j < nc) a.scales[CERAR_BY_COLUMN][tr * a.lds[CERAR_BY_COLUMN] + c0 + j] = pow2f(e);
        }
        put(CERAR_BY_COLUMN, [&](int, float* k) { k[0] = inv[0]; k[1] = inv[1]; k[2] = inv[2]; k[3] = inv[3]; });
    }
    if constexpr (BY_BLK) {
        const int e = fp8_scale_exponent(__reduce_max_sync(0xffffffffu, max(max(cm[0], cm[1]), max(cm[2], cm[3]))));
        const float inv = pow2f(-e);
        put(CERAR_BY_BLOCK, [&](int, float* k) { k[0] = k[1] = k[2] = k[3] = inv; });
        if (threadIdx.x == 0) a.scales[CERAR_BY_BLOCK][tr * a.lds[CERAR_BY_BLOCK] + tc] = pow2f(e);
    }
}

template <typename X>
cudaError_t launch_forms(const QuantizeArgs& a, int forms, dim3 grid, uint32_t tiles_c, cudaStream_t s);

template <typename X, int FORMS>
cudaError_t launch_one(const QuantizeArgs& a, dim3 grid, uint32_t tiles_c, cudaStream_t s) {
    return launch_pdl(fp8_quantize_kernel<X, FORMS>, grid, dim3(32 * kWarps<X>), 0, s, a, tiles_c);
}
template <typename X>
cudaError_t launch_forms(const QuantizeArgs& a, int forms, dim3 grid, uint32_t tiles_c, cudaStream_t s) {
    switch (forms) {
        case 1: return launch_one<X, 1>(a, grid, tiles_c, s);
        case 2: return launch_one<X, 2>(a, grid, tiles_c, s);
        case 3: return launch_one<X, 3>(a, grid, tiles_c, s);
        case 4: return launch_one<X, 4>(a, grid, tiles_c, s);
        case 5: return launch_one<X, 5>(a, grid, tiles_c, s);
        case 6: return launch_one<X, 6>(a, grid, tiles_c, s);
        default: return launch_one<X, 7>(a, grid, tiles_c, s);
    }
}

}  // namespace

cudaError_t launch_fp8_quantize(const QuantizeArgs& a, cerar_type_t type, cudaStream_t s, uint64_t* launches) {
    const int64_t tiles_r = (a.rows + T - 1) / T, tiles_c = (a.cols + T - 1) / T;
    if (tiles_r == 0 || tiles_c == 0) return cudaSuccess;
    if (tiles_r * tiles_c > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    int forms = 0;
    for (int f = 0; f < 3; ++f) if (a.codes[f]) forms |= 1 << f;
    const dim3 grid((unsigned)(tiles_r * tiles_c));
    const cudaError_t e = type == CERAR_TYPE_F32 ? launch_forms<float>(a, forms, grid, (uint32_t)tiles_c, s)
                                                 : launch_forms<__nv_bfloat16>(a, forms, grid, (uint32_t)tiles_c, s);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace cerar
