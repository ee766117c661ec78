// Product of two 8-bit matrices with a scale per 128 values along the summed dimension (cerar_fp8_matmul).
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include "kernels.cuh"
#include "ops.cuh"
#include "ptx.cuh"

namespace cerar {
namespace {

// operand as op(X)[row][k] with row = m or n: codes at row * rs + k * ks, scale of (row, block b) at (row / rd) * srs + b * sbs
struct Operand {
    const uint8_t* codes;
    const float* scales;
    int64_t rs, ks, srs, sbs;
    int rd;
};
__device__ __forceinline__ float value(uint8_t c) { return __half2float(__half(__nv_cvt_fp8_to_halfraw(c, __NV_E4M3))); }

constexpr int TM = 64, TN = 64, TK = 32;

template <typename C>
__global__ void __launch_bounds__(256) fp8_matmul_kernel(const __grid_constant__ Operand A, const __grid_constant__ Operand B, C* c, int64_t ldc,
                                                         int64_t M, int64_t N, int64_t K, int accumulate) {
    __shared__ float as[TK][TM + 1], bs[TK][TN + 1];
    ptx::grid_dependency_wait();
    const int64_t m0 = (int64_t)blockIdx.y * TM, n0 = (int64_t)blockIdx.x * TN;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {}, part[4][4] = {};
    for (int64_t k0 = 0; k0 < K; k0 += TK) {
        for (int i = threadIdx.x; i < TM * TK; i += 256) {
            const int r = i / TK, k = i % TK;
            as[k][r] = m0 + r < M && k0 + k < K ? value(A.codes[(m0 + r) * A.rs + (k0 + k) * A.ks]) : 0.f;
            bs[k][r] = n0 + r < N && k0 + k < K ? value(B.codes[(n0 + r) * B.rs + (k0 + k) * B.ks]) : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < TK; ++k)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) part[i][j] = fmaf(as[k][ty * 4 + i], bs[k][tx * 4 + j], part[i][j]);
        __syncthreads();
        if ((k0 + TK) % FP8_BLOCK == 0 || k0 + TK >= K) {
            const int64_t b = k0 / FP8_BLOCK;
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) {
                    const int64_t m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
                    if (m < M && n < N)
                        acc[i][j] = fmaf(A.scales[m / A.rd * A.srs + b * A.sbs] * part[i][j], B.scales[n / B.rd * B.srs + b * B.sbs], acc[i][j]);
                    part[i][j] = 0.f;
                }
        }
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int64_t m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
            if (m >= M || n >= N) continue;
            C& dst = c[m * ldc + n];
            dst = (C)(accumulate ? (float)dst + acc[i][j] : acc[i][j]);
        }
}

// rows_are_k: the summed dimension runs down the rows of the stored matrix
Operand operand(const cerar_fp8_matrix_t& m, bool rows_are_k) {
    Operand o;
    o.codes = m.codes; o.scales = m.scales;
    o.rs = rows_are_k ? 1 : m.ld; o.ks = rows_are_k ? m.ld : 1;
    o.rd = m.scaling == CERAR_BY_BLOCK ? FP8_BLOCK : 1;
    if (m.scaling == CERAR_BY_BLOCK) { o.srs = rows_are_k ? 1 : m.lds; o.sbs = rows_are_k ? m.lds : 1; }
    else { o.srs = 1; o.sbs = m.lds; }
    return o;
}

}  // namespace

cudaError_t launch_fp8_matmul(const MatmulArgs& a, int, cudaStream_t s, uint64_t* launches) {
    const dim3 grid((unsigned)((a.N + TN - 1) / TN), (unsigned)((a.M + TM - 1) / TM));
    const Operand A = operand(a.A, a.trans_a), B = operand(a.B, !a.trans_b);
    const cudaError_t e = a.type == CERAR_TYPE_F32
        ? launch_pdl(fp8_matmul_kernel<float>, grid, dim3(256), 0, s, A, B, (float*)a.C, a.ldc, a.M, a.N, a.K, a.accumulate)
        : launch_pdl(fp8_matmul_kernel<__nv_bfloat16>, grid, dim3(256), 0, s, A, B, (__nv_bfloat16*)a.C, a.ldc, a.M, a.N, a.K, a.accumulate);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace cerar
