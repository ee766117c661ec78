// Product of two 8-bit matrices with a scale per 128 values along the summed dimension (cerar_fp8_matmul; sm_100a:
// TMA + tcgen05 + TMEM).
//
//   C[m,n] (+)= sum_b sA(m,b) sB(b,n) P_b[m,n],     P_b[m,n] = sum_{k in block b} A[m,k] B[k,n]
//
// P_b is four tcgen05.mma kind::f8f6f4 (128 x BN x 32) into tensor memory.  The scales differ from block to block, so P_b is
// taken out after every block, multiplied by its scales and added to the running sum in registers (binary32), while the
// tensor core works on the next block in the other half of tensor memory.  At 128 x 256 x 128 the products take 512 clk; taking
// them out is 256 columns per warp quadrant (256 clk) and 64 packed multiply-adds per warp (twice that with a scale per
// column of B), done by two warps per quadrant.  Taking out is what bounds this form (tensor pipe 52 % active; 31 % with a scale
// per column).  Measured on B200, bfloat16 results: 8192^3 530 us (2070 TFLOP/s), 890 us with a scale per column of B.
//
// Where all scales are powers of two the tensor core multiplies by them itself and nothing is taken out before 16 blocks of k are
// summed up: fp8_matmul_pow2_kernel below, 8192^3 416 us (2640 TFLOP/s), 16384 x 8192 x 2048 234 us (2350).  In a long
// loop the power limit decides (8192^3: 485 us at 1.27 GHz); the library's own 8-bit product takes 413 and 197 us at these sizes, so
// with short sums (16 blocks of k: one segment per tile) there is something left in the hand-over from tile to tile.
//
// Operands come in as tiles of 128 bytes of one dimension by 128 (or BN) of the other, in the 128-byte swizzle that the
// tensor core reads, whichever dimension is contiguous in memory: a transposed operand is read in place (the "MN-major" form).
//
//   warp 0     producer: TMA loads of the stages
//   warp 1     issues the products; owns the tensor memory
//   warps 4-11 take the partial products out, scale, add; write the tile of C.  Warp w reads lanes 32 (w % 4) .. of tensor memory; the
//              two warps of a quadrant share the columns.  A warp writes C through 4 KB of shared memory of its own, so
//              that rows leave in 128-byte pieces; the products of the next tile go on meanwhile.
// (Warps 2, 3 only complete the warpgroup that hands most of its registers to the other two: 128 sums per thread need more than
// the 168 of an even share.)
//
// Few tiles, long sums: a cluster of S blocks shares a tile, each sums 1/S of the blocks of k, and the partial tiles are added
// through distributed shared memory, in a fixed order.
// Every wait is bounded; one that runs out sets the status word and the block leaves through the common exit.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>

#include "kernels.cuh"
#include "mma_tile.cuh"
#include "ops.cuh"

namespace cerar {
namespace {

using namespace mma;

constexpr int BK = FP8_BLOCK;
constexpr int WARP_EPI0 = 4;
constexpr int MAX_SPLIT = 8;                            // blocks that share the sum of a tile (a portable cluster)
// registers per thread: 128 x 56 + 256 x 224 = 384 x 168, what the block is launched with
constexpr int REGS_FEW = 56, REGS_MANY = 224;
constexpr int THREADS = 32 * (WARP_EPI0 + EPI_WARPS);
constexpr uint32_t A_BYTES = BM * BK;
// (an epilogue warp's staging rows also hold the column scales of B)

// scale of (row or column i, block b) at scales[(i / div) * si + b * sb]
struct Scales {
    const float* p;
    int64_t si, sb;
    int shift;                                         // div = 1 << shift (1 or 128)
};
struct Params {
    Scales sa, sb;
    void* C;
    int64_t ldc;
    int M, N, kblocks;
    int tiles_m, tiles_n, group_m;
    uint32_t tiles;
    int a_mn, b_mn;                                    // 1: the operand's own dimension (m or n) is the contiguous one
    int accumulate, c_vec, c_pair;                     // rows of C start on 16-byte, on 4-byte boundaries
    int stages, split;
    uint32_t a_bytes;                                  // what a load of A brings (a matrix of few rows: those rows only; the others'
                                                       // sums are made of whatever lies there, row by row, and not stored)
    int early;                                         // 1: the next kernel of the stream may set itself up meanwhile (on SMs that this one leaves free)
    int* status;
};

__device__ __forceinline__ void mma_f8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// two sums at a time (one instruction): a += x * y
__device__ __forceinline__ uint64_t pair(uint32_t x, uint32_t y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(x), "r"(y));
    return r;
}
__device__ __forceinline__ void fma_pair(uint64_t& a, uint64_t x, uint64_t y) { asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(a) : "l"(x), "l"(y)); }
__device__ __forceinline__ uint64_t mul_pair(uint64_t x, uint64_t y) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
// The producer's thread: the stages of every block of k of every tile of this CTA.
template <int BN>
__device__ __forceinline__ void produce(const Params& p, const CUtensorMap& map_a, const CUtensorMap& map_b, uint32_t smem, uint32_t full, uint32_t empty,
                                        uint32_t t0, uint32_t tstep, int kb0, int kb1, bool& failed) {
    constexpr uint32_t STAGE = A_BYTES + BN * BK;
    const uint32_t loaded = p.a_bytes + BN * BK;
    uint32_t it = 0;
    for (uint32_t t = t0; t < p.tiles && !failed; t += tstep) {
        int tm, tn;
        tile_of(p, t, tm, tn);
        const int m0 = tm * BM, n0 = tn * BN;
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
            const uint32_t s = it % p.stages, ph = (it / p.stages) & 1u;
            if (!wait_soon(empty + 8u * s, ph ^ 1u)) { failed = true; break; }
            const uint32_t a = smem + s * STAGE, b = a + A_BYTES, bar = full + 8u * s;
            mbar_arrive_expect_tx(bar, loaded);
            if (p.a_mn) tma_load_2d(a, &map_a, m0, kb * BK, bar);
            else tma_load_2d(a, &map_a, kb * BK, m0, bar);
            if (p.b_mn) {
#pragma unroll
                for (int j = 0; j < BN / 128; ++j) tma_load_2d(b + j * (128 * BK), &map_b, n0 + j * 128, kb * BK, bar);
            } else {
                tma_load_2d(b, &map_b, kb * BK, n0, bar);
            }
        }
    }
}

// A tile whose sum is split over a cluster: every block leaves the rows of its partial tile that exist in its stages (free by then),
// row r at r * BN floats, 16-byte pieces exchanged by the row so that lanes do not meet in a bank ...
template <int BN>
__device__ __forceinline__ void store_partial(uint32_t smem, int rows, int row, int col, int n, const uint32_t* v) {
    if (row >= rows) return;
    const uint32_t base = smem + (uint32_t)row * (BN * 4u);
#pragma unroll
    for (int j = 0; j < n / 4; ++j)
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(base + ((uint32_t)((col / 4 + j) ^ (row & 7)) << 4)), "r"(v[4 * j]), "r"(v[4 * j + 1]),
                     "r"(v[4 * j + 2]), "r"(v[4 * j + 3]) : "memory");
}
// ... and adds every split-th run of 32 pieces (a warp's) of all partial tiles, in the order of their blocks of k.
template <int BN, typename C>
__device__ __forceinline__ void add_partials(const Params& p, uint32_t smem, int tm, int tn, int rows, int rank, int thread) {
    C* c = static_cast<C*>(p.C);
    const int pieces = rows * (BN / 4);
    for (int run = (thread >> 5) * p.split + rank; run * 32 < pieces; run += EPI_WARPS * p.split) {
        const int i = run * 32 + (thread & 31);         // (pieces is a multiple of 32)
        const int r = i / (BN / 4), j = i % (BN / 4);
        const uint32_t at = smem + (uint32_t)r * (BN * 4u) + ((uint32_t)(j ^ (r & 7)) << 4);
        float4 w[MAX_SPLIT];
#pragma unroll
        for (int q = 0; q < MAX_SPLIT; ++q)
            if (q < p.split) w[q] = ld_cluster4(at, q);
        float4 v = w[0];
#pragma unroll
        for (int q = 1; q < MAX_SPLIT; ++q)
            if (q < p.split) { v.x += w[q].x; v.y += w[q].y; v.z += w[q].z; v.w += w[q].w; }
        const int n0 = tn * BN + 4 * j;
        C* dst = c + (int64_t)(tm * BM + r) * p.ldc + n0;
        const float x[4] = {v.x, v.y, v.z, v.w};
        if (p.c_vec && !p.accumulate && n0 + 4 <= p.N) {
            if constexpr (sizeof(C) == 4) *reinterpret_cast<float4*>(dst) = v;
            else *reinterpret_cast<uint2*>(dst) = make_uint2(Out<C>::two(v.x, v.y), Out<C>::two(v.z, v.w));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n0 + e < p.N) dst[e] = (C)(p.accumulate ? (float)dst[e] + x[e] : x[e]);
        }
    }
}

// BVEC: a scale per column of B (otherwise one for the warp's columns, which lie in one block)
template <int BN, bool BVEC, typename C>
__global__ void __launch_bounds__(THREADS, 1)
fp8_matmul_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ Params p) {
    constexpr int CW = BN / 2;                          // columns of a tile per epilogue warp
    constexpr uint32_t B_BYTES = BN * BK, STAGE = A_BYTES + B_BYTES;
    constexpr int NBUF = 512 / BN;                      // partial products in tensor memory
    extern __shared__ unsigned char smem_dyn[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t smem = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    const uint32_t staging0 = smem + (uint32_t)p.stages * STAGE;
    const uint32_t bars = staging0 + EPI_WARPS * STAGING;
    const uint32_t full = bars, empty = full + 8u * p.stages, acc_full = empty + 8u * p.stages, acc_empty = acc_full + 8u * NBUF;
    const uint32_t slot = acc_empty + 8u * NBUF;

    if (threadIdx.x == 0) {
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        for (int s = 0; s < p.stages; ++s) { mbar_init(full + 8u * s, 1); mbar_init(empty + 8u * s, 1); }
        for (int b = 0; b < NBUF; ++b) { mbar_init(acc_full + 8u * b, 1); mbar_init(acc_empty + 8u * b, EPI_WARPS); }
        mbar_init_fence();
    }
    if (warp == 1) tc_alloc(slot, 512u);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(slot));
    if (p.early) grid_dependents_may_launch();
    grid_dependency_wait();

    const int rank = p.split > 1 ? (int)cluster_rank() : 0;
    const uint32_t t0 = blockIdx.x / p.split, tstep = gridDim.x / p.split;
    const int kb0 = (int)((int64_t)p.kblocks * rank / p.split), kb1 = (int)((int64_t)p.kblocks * (rank + 1) / p.split);
    bool failed = false;

    if (warp < WARP_EPI0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FEW));
        if (warp == 0) {
            if (lane == 0) produce<BN>(p, map_a, map_b, smem, full, empty, t0, tstep, kb0, kb1, failed);
        } else if (warp == 1) {
            // The whole warp goes through the loop and one lane issues: everything the products are made from is then the same in all
            // lanes, as far as the compiler can see too, and stays in uniform registers, which is where the instruction takes
            // its operands from (a lone lane moves them there one by one, product by product).
            const uint32_t one = elect_one();
            // D binary32, A and B e4m3, M = 128, N = BN
            const uint32_t idesc = (1u << 4) | ((uint32_t)p.a_mn << 15) | ((uint32_t)p.b_mn << 16) | ((uint32_t)(BN >> 3) << 17) | ((128u >> 4) << 24);
            // 32 values of k further: 32 bytes in a row of k, or 32 rows of 128 bytes
            const uint64_t a_step = p.a_mn ? (32u * 128u) >> 4 : 32u >> 4, b_step = p.b_mn ? (32u * 128u) >> 4 : 32u >> 4;
            const uint64_t desc0 = swizzled_desc(smem, BK * 128);
            uint32_t s = 0, ph = 0, buf = 0, bph = 1;
            for (uint32_t t = t0; t < p.tiles && !failed; t += tstep)
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!warp_wait_soon(acc_empty + 8u * buf, bph) || !warp_wait_soon(full + 8u * s, ph)) { failed = true; break; }
                    tc_fence_after();
                    const uint64_t da = desc0 + (uint64_t)(s * (STAGE >> 4)), db = da + (A_BYTES >> 4);
                    if (one) {
#pragma unroll
                        for (int k = 0; k < BK / 32; ++k) mma_f8(tmem + buf * BN, da + k * a_step, db + k * b_step, idesc, k != 0);
                        tc_commit(empty + 8u * s);
                        tc_commit(acc_full + 8u * buf);
                    }
                    __syncwarp();
                    if (++s == (uint32_t)p.stages) { s = 0; ph ^= 1u; }
                    if (++buf == NBUF) { buf = 0; bph ^= 1u; }
                }
        }
        __syncwarp();
        if (p.split > 1) { cluster_sync(); cluster_sync(); }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_MANY));
        const int quad = warp & 3, half = (warp - WARP_EPI0) >> 2;
        const uint32_t staging = staging0 + (uint32_t)(warp - WARP_EPI0) * STAGING;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        uint32_t it = 0;
        for (uint32_t t = t0; t < p.tiles && !failed; t += tstep) {
            int tm, tn;
            tile_of(p, t, tm, tn);
            const int row = tm * BM + quad * 32 + lane, col0 = tn * BN + half * CW;
            // scales of this row and of these columns; rows and columns beyond the matrix use the last one's (their sums are not stored)
            const float* sa = p.sa.p + (int64_t)((row < p.M ? row : p.M - 1) >> p.sa.shift) * p.sa.si;
            const float* sb = p.sb.p + (int64_t)((col0 < p.N ? col0 : p.N - 1) >> p.sb.shift) * p.sb.si;
            uint64_t acc2[CW / 2];                        // the sums, in pairs
#pragma unroll
            for (int j = 0; j < CW / 2; ++j) acc2[j] = 0ull;
            float a_next = __ldg(sa + kb0 * p.sa.sb), b_next = 1.f;
            float bv[CW / 32];
            if constexpr (!BVEC) b_next = __ldg(sb + kb0 * p.sb.sb);
            auto column_scales = [&](int kb) {
#pragma unroll
                for (int j = 0; j < CW / 32; ++j) {
                    const int n = col0 + j * 32 + lane;
                    bv[j] = __ldg(p.sb.p + (n < p.N ? n : p.N - 1) + kb * p.sb.sb);
                }
            };
            if constexpr (BVEC) column_scales(kb0);
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const uint32_t buf = it % NBUF, bph = (it / NBUF) & 1u;
                const uint64_t s = pair(__float_as_uint(a_next * b_next), __float_as_uint(a_next * b_next));
                if (kb + 1 < kb1) {
                    a_next = __ldg(sa + (kb + 1) * p.sa.sb);
                    if constexpr (!BVEC) b_next = __ldg(sb + (kb + 1) * p.sb.sb);
                }
                if constexpr (BVEC) {
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < CW / 32; ++j) asm volatile("st.shared.f32 [%0], %1;" ::"r"(staging + 4u * (j * 32 + lane)), "f"(bv[j]) : "memory");
                    __syncwarp();
                    if (kb + 1 < kb1) column_scales(kb + 1);
                }
                if (!warp_wait_soon(acc_full + 8u * buf, bph)) { failed = true; break; }
                tc_fence_after();
                // the next 16 columns are on their way while these are added (32 at a time leave no registers for the loop's own
                // variables beside 128 sums: 8192^3 745 us instead of 570)
                uint32_t v[2][16];
                const uint32_t from = tmem + lanes + buf * BN + half * CW;
                ld16_start(from, v[0]);
#pragma unroll
                for (int c = 0; c < CW / 16; ++c) {
                    uint32_t* x = v[c & 1];
                    uint64_t q[8];                       // the column scales of these 16, in pairs
                    if constexpr (BVEC) {
#pragma unroll
                        for (int j = 0; j < 8; j += 2)
                            asm volatile("ld.shared.v2.b64 {%0,%1}, [%2];" : "=l"(q[j]), "=l"(q[j + 1]) : "r"(staging + 4u * (c * 16 + 2 * j)));
                    }
                    ld16_done(x);
                    if (c < CW / 16 - 1) {
                        ld16_start(from + (c + 1) * 16, v[(c + 1) & 1]);
                    } else {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(acc_empty + 8u * buf);
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) fma_pair(acc2[c * 8 + j], BVEC ? mul_pair(s, q[j]) : s, pair(x[2 * j], x[2 * j + 1]));
                }
            }
            if (failed) break;
            float acc[CW];
#pragma unroll
            for (int j = 0; j < CW; j += 2) asm("mov.b64 {%0, %1}, %2;" : "=f"(acc[j]), "=f"(acc[j + 1]) : "l"(acc2[j / 2]));
            if (p.split == 1) {
                constexpr int SLAB = 8 * Out<C>::PER16;
#pragma unroll
                for (int c = 0; c < CW / SLAB; ++c) write_slab<C>(p, staging, tm * BM + quad * 32, col0 + c * SLAB, acc + c * SLAB);
                __syncwarp();
            } else {
                store_partial<BN>(smem, p.M - tm * BM, quad * 32 + lane, half * CW, CW, reinterpret_cast<const uint32_t*>(acc));
            }
        }
        __syncwarp();
        if (p.split > 1) {
            cluster_sync();
            int tm, tn;                                 // (one tile per cluster)
            tile_of(p, t0, tm, tn);
            add_partials<BN, C>(p, smem, tm, tn, p.M - tm * BM < BM ? p.M - tm * BM : BM, rank, threadIdx.x - 32 * WARP_EPI0);
            __syncwarp();
            cluster_sync();                             // no block leaves while another reads its part
        }
    }
    leave(p, failed, warp, lane, tmem);
}

// ---------------------------------------------------------------- scales that are powers of two
//
// The tensor core multiplies by such scales itself (kind::mxf8f6f4.block_scale: one 8-bit exponent per row and 32 values of k, from
// tensor memory), so the sum over all blocks stays in the accumulator, nothing is taken out in between, and a tile costs its
// products alone.  The exponents of 128 rows are 4 columns of 32 lanes (row r in lane r % 32 of column r / 32), present in
// all four lane quadrants; a 32-bit word holds those of four blocks of k, which the instruction picks from by number.
//
//   warp 0       producer, warp 1 issues the products, as above
//   warps 4-7    read the scales of four blocks of k (a warp each, a group ahead), exchange their exponents through shared
//                memory and put them into tensor memory, every warp into its quadrant.  A scale that is no power of two
//                (the caller said they all are) becomes the exponent that means NaN, and so do the results it touches
//   warps 8-15   write the tile of C
// Two accumulators of 256 columns and the exponents do not fit into 512 columns: the accumulators overlap by 32 columns,
// which are written out first; the products of the next tile wait for those only.
constexpr int POW2_THREADS = 512, WARP_SCALE0 = 4, WARP_OUT0 = 8;
// registers per thread: 128 x 56 + 128 x 72 + 256 x 192 = 512 x 128, what the block is launched with
constexpr int POW2_REGS_ISSUE = 56, POW2_REGS_SCALE = 72, POW2_REGS_OUT = 192;
// blocks of k that stay in the accumulator: it drops what does not fit its 24 bits instead of rounding, an error that
// grows with every addition (K = 16384: 1.2e-6 of a sum's norm), so longer sums are put together in registers
constexpr int SEGMENT = 16;
constexpr uint32_t SF_WORDS = 12 * 128;                  // shared memory of the exponents of a group
constexpr uint32_t SF_COL = 480, SF_BUF = 16;            // exponents: two buffers of 4 (A) and, 8 further, 8 (B) columns

template <int CG>
__device__ __forceinline__ void mma_mxf8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    if constexpr (CG == 1)
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
                     " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
                     " tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
__device__ __forceinline__ uint32_t exponent_of(float s) {
    const uint32_t b = __float_as_uint(s), e = b >> 23;
    return (b & 0x807FFFFFu) == 0u && e >= 1u && e <= 254u ? e : 0xFFu;
}

template <int CG, int BN, typename C>
__global__ void __launch_bounds__(POW2_THREADS, 1)
fp8_matmul_pow2_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ Params p) {
    constexpr int CW = BN / 2;                           // columns per output warp
    constexpr int B_ROWS = BN / CG;                      // of the tile of B, in this block
    constexpr uint32_t STAGE = A_BYTES + B_ROWS * BK;
    constexpr uint32_t OVERLAP = BN == 256 ? 32 : 0, D1 = BN - OVERLAP;       // first column of the second accumulator
    constexpr int SLAB = 8 * Out<C>::PER16;
    extern __shared__ unsigned char smem_dyn[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t smem = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    const uint32_t staging0 = smem + (uint32_t)p.stages * STAGE;
    const uint32_t bars = staging0 + EPI_WARPS * STAGING;
    const uint32_t full = bars, empty = full + 8u * p.stages, acc_full = empty + 8u * p.stages, acc_empty = acc_full + 16u, over_empty = acc_empty + 16u;
    const uint32_t sf_full = over_empty + 8u, sf_empty = sf_full + 16u, slot = sf_empty + 16u;

    if (threadIdx.x == 0) {
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        for (int s = 0; s < p.stages; ++s) { mbar_init(full + 8u * s, 1); mbar_init(empty + 8u * s, 1); }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full + 8u * b, 1); mbar_init(acc_empty + 8u * b, CG * EPI_WARPS);
            mbar_init(sf_full + 8u * b, CG * 4); mbar_init(sf_empty + 8u * b, 1);
        }
        mbar_init(over_empty, CG * EPI_WARPS / 2);
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
    if (p.early) grid_dependents_may_launch();
    grid_dependency_wait();

    // a cluster is a pair of blocks that share a tile of 256 rows (CG = 2), or `split` blocks that share the sum of a tile
    const int crank = CG == 2 || p.split > 1 ? (int)cluster_rank() : 0;
    const int pair_rank = CG == 2 ? crank : 0, rank = CG == 2 ? 0 : crank;
    const uint32_t csize = CG == 2 ? 2 : p.split;
    const uint32_t t0 = blockIdx.x / csize, tstep = gridDim.x / csize;
    const int kb0 = (int)((int64_t)p.kblocks * rank / p.split), kb1 = (int)((int64_t)p.kblocks * (rank + 1) / p.split);
    bool failed = false;

    if (warp < WARP_SCALE0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(POW2_REGS_ISSUE));
        if (warp == 0) {
            if (lane == 0) {
                uint32_t it = 0;
                for (uint32_t t = t0; t < p.tiles && !failed; t += tstep) {
                    int tm, tn;
                    tile_of(p, t, tm, tn);
                    const int m0 = (tm * CG + pair_rank) * BM, n0 = tn * BN + pair_rank * B_ROWS;
                    for (int kb = kb0; kb < kb1; ++kb, ++it) {
                        const uint32_t s = it % p.stages, ph = (it / p.stages) & 1u;
                        if (!wait_soon(empty + 8u * s, ph ^ 1u)) { failed = true; break; }
                        const uint32_t a = smem + s * STAGE, b = a + A_BYTES;
                        if (pair_rank == 0) mbar_arrive_expect_tx(full + 8u * s, CG * (p.a_bytes + B_ROWS * BK));       // what both blocks load
                        const uint32_t bar = CG == 1 ? full + 8u * s : in_block(full + 8u * s, 0);
                        if (p.a_mn) tma_load_operand<CG>(a, &map_a, m0, kb * BK, bar);
                        else tma_load_operand<CG>(a, &map_a, kb * BK, m0, bar);
                        if (p.b_mn) {
#pragma unroll
                            for (int j = 0; j < B_ROWS / 128; ++j) tma_load_operand<CG>(b + j * (128 * BK), &map_b, n0 + j * 128, kb * BK, bar);
                        } else {
                            tma_load_operand<CG>(b, &map_b, kb * BK, n0, bar);
                        }
                    }
                }
            }
        } else if (warp == 1) {
            if (pair_rank == 0) {                        // (the whole warp, one lane issuing: see above)
                const uint32_t one = elect_one();
                // exponents of 8 bits, A and B e4m3, M = 128 CG, N = BN
                const uint32_t idesc0 = (1u << 23) | ((uint32_t)p.a_mn << 15) | ((uint32_t)p.b_mn << 16) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(CG * BM >> 4) << 24);
                const uint64_t a_step = p.a_mn ? (32u * 128u) >> 4 : 32u >> 4, b_step = p.b_mn ? (32u * 128u) >> 4 : 32u >> 4;
                const uint64_t desc0 = swizzled_desc(smem, BK * 128);
                uint32_t s = 0, ph = 0, seg = 0, group = 0;
                for (uint32_t t = t0; t < p.tiles && !failed; t += tstep) {
                    uint32_t id = 0;                     // block of k within its group of four
                    for (int k0 = kb0; k0 < kb1 && !failed; k0 += SEGMENT, ++seg) {
                        const uint32_t buf = seg & 1u;
                        if (!warp_wait_soon(acc_empty + 8u * buf, ((seg >> 1) & 1u) ^ 1u)) { failed = true; break; }
                        if (OVERLAP && !warp_wait_soon(over_empty, (seg & 1u) ^ 1u)) { failed = true; break; }
                        const uint32_t d = tmem + buf * D1;
                        const int k1 = k0 + SEGMENT < kb1 ? k0 + SEGMENT : kb1;
                        for (int kb = k0; kb < k1; ++kb) {
                            const uint32_t sbuf = group & 1u;
                            if (id == 0u && !warp_wait_soon(sf_full + 8u * sbuf, (group >> 1) & 1u)) { failed = true; break; }
                            if (!warp_wait_soon(full + 8u * s, ph)) { failed = true; break; }
                            tc_fence_after();
                            const uint64_t da = desc0 + (uint64_t)(s * (STAGE >> 4)), db = da + (A_BYTES >> 4);
                            const uint32_t sf = tmem + SF_COL + sbuf * SF_BUF, idesc = idesc0 | (id << 4) | (id << 29);
                            const bool last = id == 3u || kb + 1 == kb1;
                            if (one) {
#pragma unroll
                                for (int k = 0; k < BK / 32; ++k) mma_mxf8<CG>(d, da + k * a_step, db + k * b_step, idesc, sf, sf + 8, kb != k0 || k != 0);
                                commit<CG>(empty + 8u * s);
                                if (last) commit<CG>(sf_empty + 8u * sbuf);
                                if (kb + 1 == k1) commit<CG>(acc_full + 8u * buf);
                            }
                            __syncwarp();
                            if (++s == (uint32_t)p.stages) { s = 0; ph ^= 1u; }
                            if (last) ++group;
                            id = (id + 1) & 3u;
                        }
                    }
                }
            }
        }
    } else if (warp < WARP_OUT0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(POW2_REGS_SCALE));
        constexpr int NW = 4 + BN / 32;                  // words of exponents per lane
        const uint32_t ready = CG == 1 ? sf_full : in_block(sf_full, 0), words = slot + 16u;
        uint32_t group = 0;
        for (uint32_t t = t0; t < p.tiles; t += tstep) {
            int tm, tn;
            tile_of(p, t, tm, tn);
            // this lane's rows and columns; warp w reads block w of every group of four, one group ahead
            const float *a[4], *b[BN / 32];
            const int w = warp - WARP_SCALE0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int m = (tm * CG + pair_rank) * BM + j * 32 + lane;
                a[j] = p.sa.p + (int64_t)((m < p.M ? m : p.M - 1) >> p.sa.shift) * p.sa.si;
            }
#pragma unroll
            for (int j = 0; j < BN / 32; ++j) {
                const int n = tn * BN + j * 32 + lane;
                b[j] = p.sb.p + (int64_t)((n < p.N ? n : p.N - 1) >> p.sb.shift) * p.sb.si;
            }
            float x[NW];
            auto load = [&](int kb) {
                const int k = kb + w < kb1 ? kb + w : kb1 - 1;
#pragma unroll
                for (int j = 0; j < NW; ++j) x[j] = j < 4 ? __ldg(a[j < 4 ? j : 0] + k * p.sa.sb) : __ldg(b[j < 4 ? 0 : j - 4] + k * p.sb.sb);
            };
            load(kb0);
            for (int kb = kb0; kb < kb1; kb += 4, ++group) {
                bar_sync(1, 128);                        // the words of the group before have been read
#pragma unroll
                for (int j = 0; j < NW; ++j)
                    asm volatile("st.shared.u8 [%0], %1;" ::"r"(words + (uint32_t)(j * 128 + lane * 4 + w)), "r"(exponent_of(x[j])) : "memory");
                if (kb + 4 < kb1) load(kb + 4);
                bar_sync(1, 128);
                uint32_t e[NW];
#pragma unroll
                for (int j = 0; j < NW; ++j) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(e[j]) : "r"(words + (uint32_t)(j * 128 + lane * 4)) : "memory");
                const uint32_t sbuf = group & 1u;
                if (!failed && !warp_wait_soon(sf_empty + 8u * sbuf, ((group >> 1) & 1u) ^ 1u)) failed = true;     // (goes on for the barriers' sake)
                tc_fence_after();
                const uint32_t to = tmem + ((uint32_t)((warp & 3) * 32) << 16) + SF_COL + sbuf * SF_BUF;
                tc_st_cols<4>(to, e);
                tc_st_cols<BN / 32>(to + 8, e + 4);
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive<CG>(ready + 8u * sbuf);
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(POW2_REGS_OUT));
        const int quad = warp & 3, half = (warp - WARP_OUT0) >> 2;
        const uint32_t staging = staging0 + (uint32_t)(warp - WARP_OUT0) * STAGING;
        const uint32_t freed = CG == 1 ? acc_empty : in_block(acc_empty, 0), over_freed = CG == 1 ? over_empty : in_block(over_empty, 0);
        // columns of this warp, 32 at a time, from the shared ones on: the last 32 of the first accumulator and the first 32 of the
        // second are taken out first, so the warps of the second half go backwards
        const int first = half ? BN - 32 : 0, step = half ? -32 : 32;
        uint32_t seg = 0;
        for (uint32_t t = t0; t < p.tiles && !failed; t += tstep) {
            int tm, tn;
            tile_of(p, t, tm, tn);
            float acc[CW];
#pragma unroll
            for (int j = 0; j < CW; ++j) acc[j] = 0.f;
            for (int k0 = kb0; k0 < kb1; k0 += SEGMENT, ++seg) {
                const uint32_t buf = seg & 1u;
                if (!warp_wait_soon(acc_full + 8u * buf, (seg >> 1) & 1u)) { failed = true; break; }
                tc_fence_after();
                const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16) + buf * D1 + first;
#pragma unroll
                for (int c = 0; c < CW / 32; ++c) {
                    uint32_t v[32];
                    ld32_start(from + c * step, v);
                    ld32_done(v);
                    if (c == 0 && OVERLAP && half != (int)buf) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) arrive<CG>(over_freed);
                    }
                    if (c == CW / 32 - 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) arrive<CG>(freed + 8u * buf);
                    }
#pragma unroll
                    for (int j = 0; j < 32; ++j) acc[c * 32 + j] += __uint_as_float(v[j]);
                }
            }
            if (failed) break;
            if (CG == 2 || p.split == 1) {
                const int row0 = (tm * CG + pair_rank) * BM + quad * 32, col0 = tn * BN + (half ? BN - SLAB : 0);
#pragma unroll
                for (int c = 0; c < CW / SLAB; ++c)
                    write_slab<C>(p, staging, row0, col0 + (half ? -c : c) * SLAB, acc + c * SLAB, SLAB == 64 && half ? 4 : 0);
            } else {
#pragma unroll
                for (int c = 0; c < CW / 32; ++c) store_partial<BN>(smem, p.M - tm * BM, quad * 32 + lane, first + c * step, 32, reinterpret_cast<const uint32_t*>(acc + 32 * c));
            }
            __syncwarp();
        }
    }
    __syncwarp();
    if (CG == 1 && p.split > 1) {
        cluster_sync();
        if (warp >= WARP_OUT0) {
            int tm, tn;                                  // (one tile per cluster)
            tile_of(p, t0, tm, tn);
            add_partials<BN, C>(p, smem, tm, tn, p.M - tm * BM < BM ? p.M - tm * BM : BM, rank, threadIdx.x - 32 * WARP_OUT0);
        }
        __syncwarp();
        cluster_sync();
    }
    if constexpr (CG == 2) {
        tc_fence_before();
        cluster_sync();                                  // nothing is sent to a block that has left
        tc_fence_after();
    }
    leave<CG>(p, failed, warp, lane, tmem);
}

bool make_map_8bit(CUtensorMap* m, const cerar_fp8_matrix_t& x, int box_rows) {
    const cuuint64_t dim[2] = {(cuuint64_t)x.cols, (cuuint64_t)x.rows}, stride[1] = {(cuuint64_t)x.ld};
    const cuuint32_t box[2] = {(cuuint32_t)BK, (cuuint32_t)box_rows}, step[2] = {1, 1};
    return encode_tiled(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, x.codes, dim, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

// rows_are_k: the summed dimension runs down the rows of the stored matrix
Scales scales_of(const cerar_fp8_matrix_t& m, bool rows_are_k) {
    if (m.scaling != CERAR_BY_BLOCK) return {m.scales, 1, m.lds, 0};
    return rows_are_k ? Scales{m.scales, 1, m.lds, 7} : Scales{m.scales, m.lds, 1, 7};
}

typedef void (*Kernel)(CUtensorMap, CUtensorMap, Params);

constexpr int KERNELS = 12, MAX_SMEM = 232448;

cudaError_t launch_one(Kernel kern, int which, int b_rows, int threads, int cluster, const CUtensorMap& ma, const CUtensorMap& mb, const Params& p, int grid, cudaStream_t s) {
    const size_t smem = 1024 + (size_t)p.stages * (A_BYTES + b_rows * BK) + EPI_WARPS * STAGING + 512 + SF_WORDS;
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
    cfg.gridDim = dim3((unsigned)grid); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = g_tune_pdl_off ? 0 : 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)cluster, 1, 1};
    cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, ma, mb, p);
}
template <typename C>
Kernel kernel_for(bool wide, bool pow2, bool bvec) {
    if (pow2) return wide ? fp8_matmul_pow2_kernel<2, 256, C> : fp8_matmul_pow2_kernel<1, 128, C>;
    if (bvec) return wide ? fp8_matmul_kernel<256, true, C> : fp8_matmul_kernel<128, true, C>;
    return wide ? fp8_matmul_kernel<256, false, C> : fp8_matmul_kernel<128, false, C>;
}

// Tile and split.  The times are a model (ns, B200) of what was measured: a block of k costs 420 in a tile of 256 x 256 (by a pair of
// blocks) and 315 in one of 128 x 128 where the tensor core applies the scales, 640 in 128 x 256 and 400 in 128 x 128 where it does
// not; a tile's end costs about 800; adding up partial tiles 800 and 2000 more for 128 full rows (16 tiles of 16 blocks of k, us
// for split 1, 2, 3, 4, 6: 9.3, 10.0, 9.1, 8.0, 7.9; one row, 16 tiles of 64: 24.7, 15.3, 12.2, 10.2, 10.6).  Large clusters do not
// fill the GPU's groups of SMs: 128 blocks in clusters of 8 take two turns (14 us instead of 8), 108 in clusters of 4 do not.
struct Shape { bool wide; int split; };
Shape choose_shape(int M, int N, int kblocks, bool pow2, int num_sms) {
    const int64_t m = (M + BM - 1) / BM, n = (N + 127) / 128, narrow = m * n;
    const int64_t wide = pow2 ? ((m + 1) / 2) * ((n + 1) / 2) : m * ((n + 1) / 2), wide_slots = pow2 ? num_sms / 2 : num_sms;
    Shape best{true, 1};
    int64_t cost = ((wide + wide_slots - 1) / wide_slots) * ((int64_t)kblocks * (pow2 ? 420 : 640) + 1600);
    for (int q = 1; q <= MAX_SPLIT && q <= kblocks; ++q) {
        if (q > 1 && narrow * q * 100 > (int64_t)num_sms * (q == 2 ? 100 : q <= 4 ? 82 : 65)) continue;
        const int64_t waves = q > 1 ? 1 : (narrow + num_sms - 1) / num_sms;
        const int64_t c = waves * ((int64_t)((kblocks + q - 1) / q) * (pow2 ? 315 : 400) + 800) + (q > 1 ? 800 + 2000 * (M < BM ? M : BM) / BM : 0);
        if (c < cost) { cost = c; best = {false, q}; }
    }
    return best;
}

}  // namespace

int fp8_matmul_tile(int64_t M, int64_t N, int64_t K, bool pow2, int num_sms, int* split) {
    const Shape shape = choose_shape((int)M, (int)N, (int)((K + BK - 1) / BK), pow2, num_sms);
    *split = shape.split;
    return shape.wide ? 256 : 128;
}

cudaError_t launch_fp8_matmul(const MatmulArgs& a, int num_sms, cudaStream_t s, uint64_t* launches) {
    if (!get_encode_fn()) return cudaErrorNotSupported;
    Params p = {};
    const bool bvec = a.B.scaling != CERAR_BY_BLOCK, pow2 = a.A.pow2 && a.B.pow2;
    p.M = (int)a.M; p.N = (int)a.N; p.kblocks = (int)((a.K + BK - 1) / BK);
    const Shape shape = choose_shape(p.M, p.N, p.kblocks, pow2, num_sms);
    const bool wide = shape.wide, paired = wide && pow2;                   // paired: tiles of 256 rows, by two blocks
    const int BN = wide ? 256 : 128, rows = paired ? 2 * BM : BM, b_rows = paired ? BN / 2 : BN;
    p.tiles_m = (p.M + rows - 1) / rows;
    p.tiles_n = (p.N + BN - 1) / BN;
    if ((int64_t)p.tiles_m * p.tiles_n > 0x3FFFFFFF) return cudaErrorInvalidConfiguration;
    p.tiles = (uint32_t)p.tiles_m * (uint32_t)p.tiles_n;
    p.split = shape.split;
    p.group_m = paired ? 8 : 16;
    p.stages = wide && !paired ? 4 : 6;
    p.a_mn = a.trans_a; p.b_mn = !a.trans_b;
    p.sa = scales_of(a.A, a.trans_a);
    p.sb = scales_of(a.B, !a.trans_b);
    p.C = a.C; p.ldc = a.ldc; p.accumulate = a.accumulate; p.status = a.status;
    const int64_t size = a.type == CERAR_TYPE_F32 ? 4 : 2;
    p.c_vec = (reinterpret_cast<uintptr_t>(a.C) & 15u) == 0 && (a.ldc * size) % 16 == 0;
    p.c_pair = (reinterpret_cast<uintptr_t>(a.C) & 3u) == 0 && (a.ldc * size) % 4 == 0;
    CUtensorMap ma, mb;
    const int a_rows = !p.a_mn && p.M < BM ? (p.M + 7) & ~7 : BM;
    p.a_bytes = (uint32_t)a_rows * BK;
    if (!make_map_8bit(&ma, a.A, p.a_mn ? BK : a_rows) || !make_map_8bit(&mb, a.B, p.b_mn ? BK : b_rows)) return cudaErrorInvalidValue;
    const int cluster = paired ? 2 : p.split, most = num_sms / cluster;
    const int grid = cluster * (p.split > 1 || (int)p.tiles < most ? (int)p.tiles : most);
    p.early = 2 * grid <= num_sms;
    const Kernel kern = a.type == CERAR_TYPE_F32 ? kernel_for<float>(wide, pow2, bvec) : kernel_for<__nv_bfloat16>(wide, pow2, bvec);
    const cudaError_t e = launch_one(kern, (pow2 ? 0 : bvec ? 1 : 2) * 4 + wide * 2 + (a.type == CERAR_TYPE_F32), b_rows, pow2 ? POW2_THREADS : THREADS, cluster, ma, mb, p, grid, s);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace cerar
