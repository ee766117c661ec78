// Conversion of a matrix to 8 bits with a power-of-two scale per 128 values (cerar_fp8_quantize).
//
//   s = 2^e, e = min { e : max |x| 2^-e <= 448 } over a block;   code = e4m3(x 2^-e), nearest even
//
// x 2^-e is exact in binary32 (away from underflow), so the only rounding is that of the code.  A block is
// 128 values of a row, 128 values of a column, or 128 x 128 values; every wanted form is made from one
// reading of x.  Nothing but bytes bounds this: 2 or 4 in, 1 out per form and element.
//
// One CTA per 128 x 128 tile, the tile in registers: warp w holds rows 16 w .. 16 w + 15, lane l the columns 4 l .. 4 l + 3 of
// each, so a warp reads whole row segments (256 or 512 contiguous bytes) and stores 128.
// A row's maximum is one warp reduction; a column's goes through shared memory once; all forms are stored row-major, as the
// products read them, so nothing is transposed.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "kernels.cuh"
#include "ops.cuh"
#include "ptx.cuh"

namespace cerar {
namespace {

constexpr int T = FP8_BLOCK;             // tile edge
constexpr int WARPS = 8, ROWS = T / WARPS;
constexpr uint32_t INF = 0x7F800000u;

__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Four values of one row as they are in memory, and as binary32.
template <typename X> struct Four;
template <> struct Four<float> {
    float4 v;
    __device__ __forceinline__ void clear() { v = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const float* p) { v = __ldcs(reinterpret_cast<const float4*>(p)); }
    __device__ __forceinline__ void set(int j, float x) { (&v.x)[j] = x; }
    __device__ __forceinline__ void get(float* x) const { x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
};
template <> struct Four<__nv_bfloat16> {
    uint2 v;
    __device__ __forceinline__ void clear() { v = make_uint2(0u, 0u); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = __ldcs(reinterpret_cast<const uint2*>(p)); }
    __device__ __forceinline__ void set(int j, __nv_bfloat16 x) {
        const uint32_t b = (uint32_t)__bfloat16_as_ushort(x) << (16 * (j & 1));
        if (j < 2) v.x |= b; else v.y |= b;
    }
    __device__ __forceinline__ void get(float* x) const {
        x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xFFFF0000u);
        x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xFFFF0000u);
    }
};

// Four scaled values to four codes.  bad: there may be values that are not finite, which become NaN: x * 0 is NaN exactly there
// (the conversion by itself would turn an infinity into 448).
__device__ __forceinline__ uint32_t codes4(const float* x, const float* inv, bool bad) {
    uint16_t lo, hi;
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = x[j] * inv[j];
    if (bad) {
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] += x[j] * 0.f;
    }
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(y[1]), "f"(y[0]));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(y[3]), "f"(y[2]));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}
__device__ __forceinline__ void store_codes(uint8_t* dst, uint32_t v, int n) {
    if (n >= 4) { *reinterpret_cast<uint32_t*>(dst) = v; return; }
#pragma unroll
    for (int j = 0; j < 3; ++j) if (j < n) dst[j] = (uint8_t)(v >> (8 * j));
}

// FORMS: bit per cerar_scaling_t
template <typename X, int FORMS>
__global__ void __launch_bounds__(32 * WARPS, sizeof(X) == 2 ? 3 : 2) fp8_quantize_kernel(const __grid_constant__ QuantizeArgs a, uint32_t tiles_c) {
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
#pragma unroll
    for (int i = 0; i < ROWS; ++i) v[i].clear();
    if (a.vec && nc == 4) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
            if (i < nr) v[i].load(src + i * a.ldx);
    } else {
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i < nr && j < nc) v[i].set(j, src[i * a.ldx + j]);
    }

    uint32_t cm[4] = {0u, 0u, 0u, 0u};
    bool bad = false;
    float row_scale = 1.f;                                             // of row `lane` of this warp (lanes 0 .. ROWS - 1)
    uint8_t* dst = BY_ROW ? a.codes[CERAR_BY_ROW] + r0 * a.ld[CERAR_BY_ROW] + c0 : nullptr;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        float x[4];
        v[i].get(x);
        uint32_t m[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) m[j] = __float_as_uint(x[j]) & 0x7FFFFFFFu;
        if (max(max(m[0], m[1]), max(m[2], m[3])) >= INF) {           // rare: only finite magnitudes count
            bad = true;
#pragma unroll
            for (int j = 0; j < 4; ++j) if (m[j] >= INF) m[j] = 0u;
        }
        if constexpr (BY_COL || BY_BLK) {
#pragma unroll
            for (int j = 0; j < 4; ++j) cm[j] = max(cm[j], m[j]);
        }
        if constexpr (BY_ROW) {
            const int e = fp8_scale_exponent(__reduce_max_sync(0xffffffffu, max(max(m[0], m[1]), max(m[2], m[3]))));
            if (lane == i) row_scale = pow2f(e);
            const float k = pow2f(-e), inv[4] = {k, k, k, k};
            if (i < nr) store_codes(dst + i * a.ld[CERAR_BY_ROW], codes4(x, inv, bad), nc);
        }
    }
    if constexpr (BY_ROW) {
        if (lane < nr) a.scales[CERAR_BY_ROW][tc * a.lds[CERAR_BY_ROW] + r0 + lane] = row_scale;
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
        float inv[4], sc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) { const int e = fp8_scale_exponent(cm[j]); inv[j] = pow2f(-e); sc[j] = pow2f(e); }
        uint8_t* dc = a.codes[CERAR_BY_COLUMN] + r0 * a.ld[CERAR_BY_COLUMN] + c0;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            float x[4];
            v[i].get(x);
            if (i < nr) store_codes(dc + i * a.ld[CERAR_BY_COLUMN], codes4(x, inv, bad), nc);
        }
        if (warp == 0) {
            float* s = a.scales[CERAR_BY_COLUMN] + tr * a.lds[CERAR_BY_COLUMN] + c0;
#pragma unroll
            for (int j = 0; j < 4; ++j) if (j < nc) s[j] = sc[j];
        }
    }
    if constexpr (BY_BLK) {
        const int e = fp8_scale_exponent(__reduce_max_sync(0xffffffffu, max(max(cm[0], cm[1]), max(cm[2], cm[3]))));
        const float k = pow2f(-e), inv[4] = {k, k, k, k};
        uint8_t* db = a.codes[CERAR_BY_BLOCK] + r0 * a.ld[CERAR_BY_BLOCK] + c0;
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            float x[4];
            v[i].get(x);
            if (i < nr) store_codes(db + i * a.ld[CERAR_BY_BLOCK], codes4(x, inv, bad), nc);
        }
        if (threadIdx.x == 0) a.scales[CERAR_BY_BLOCK][tr * a.lds[CERAR_BY_BLOCK] + tc] = pow2f(e);
    }
}

template <typename X>
cudaError_t launch_forms(const QuantizeArgs& a, int forms, dim3 grid, uint32_t tiles_c, cudaStream_t s);

template <typename X, int FORMS>
cudaError_t launch_one(const QuantizeArgs& a, dim3 grid, uint32_t tiles_c, cudaStream_t s) {
    return launch_pdl(fp8_quantize_kernel<X, FORMS>, grid, dim3(32 * WARPS), 0, s, a, tiles_c);
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
