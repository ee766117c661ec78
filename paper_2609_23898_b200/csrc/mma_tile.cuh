// What the tile kernels of the products share (8-bit and bfloat16 operands): bounded waits, operand loads, descriptors, reads of tensor
// memory, pairs of blocks, and the writing of a tile of C.  Rows of operand tiles are 128 bytes in the 128-byte swizzle.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "ops.cuh"
#include "tc_common.cuh"

namespace cerar {
namespace mma {

using namespace tc;

constexpr int BM = 128;                                 // rows of a tile in a block
constexpr int EPI_WARPS = 8;
constexpr uint32_t STAGING = 32 * 128;                 // shared memory of a writing warp: 32 rows of 128 bytes

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// The bounded wait of this file: an attempt lets the warp sleep until the phase is there or about 20 us have passed, so that
// waiting warps leave the issue slots and the shared-memory port to the others; the timer is looked at after the first attempt.
__device__ __forceinline__ bool try_wait_asleep(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(bar), "r"(parity), "r"(20000u) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool wait_soon(uint32_t bar, uint32_t parity) {
    unsigned long long start = 0;
    for (;;) {
        for (int i = 0; i < 16; ++i)
            if (try_wait_asleep(bar, parity)) return true;
        const unsigned long long now = global_ns();
        if (start == 0) start = now;
        else if (now - start > WAIT_LIMIT_NS) return false;
    }
}
__device__ __forceinline__ bool warp_wait_soon(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_soon(bar, parity) ? 1 : 0) != 0; }
__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) { asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory"); }
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(r));
    return r;
}
// Shared-memory descriptor of a tile in the 128-byte swizzle.  Summed dimension contiguous: rows of 128 bytes, groups of 8 rows
// 1024 bytes apart.  The other dimension contiguous: groups of 8 k 1024 bytes apart, blocks of 128 bytes of rows or columns `block` bytes apart.
__device__ __forceinline__ uint64_t swizzled_desc(uint32_t saddr, uint32_t block) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | (uint64_t)(block >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 |
           (uint64_t)1 << 46 /* sm_100 descriptor */ | (uint64_t)2 << 61 /* 128-byte swizzle */;
}
// 32 columns of this warp's lanes of tensor memory; the values may be used after ld32_done, which names them so that no use of
// them is moved in front of the wait
__device__ __forceinline__ void ld32_start(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
__device__ __forceinline__ void ld32_done(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
          "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
          "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
          "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}
__device__ __forceinline__ void ld16_start(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void ld16_done(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
          "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t saddr, uint32_t rank) {
    uint32_t ra;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(saddr), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(ra) : "memory");
    return v;
}

// tile number -> (row tile, column tile): column by column inside bands of group_m row tiles, so that the tiles that run at the
// same time share operand tiles in L2
template <typename P>
__device__ __forceinline__ void tile_of(const P& p, uint32_t t, int& tm, int& tn) {
    const uint32_t per_band = (uint32_t)(p.group_m * p.tiles_n);
    const int band = (int)(t / per_band);
    const int first = band * p.group_m;
    const int rows = p.tiles_m - first < p.group_m ? p.tiles_m - first : p.group_m;
    const int r = (int)(t - band * per_band);
    tm = first + r % rows;
    tn = r / rows;
}

template <typename C> struct Out;
template <> struct Out<float> {
    static constexpr int PER16 = 4;                    // elements in 16 bytes
    static __device__ __forceinline__ uint4 pack(const float* v) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};
template <> struct Out<__nv_bfloat16> {
    static constexpr int PER16 = 8;
    static __device__ __forceinline__ uint32_t two(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const float* v) { return make_uint4(two(v[0], v[1]), two(v[2], v[3]), two(v[4], v[5]), two(v[6], v[7])); }
};

// Rows row0 .. row0 + 31 (those below M) of C, columns col0 .. col0 + n - 1 of a slab of 128 bytes per row: the warp holds row
// (lane)'s values in v[0 .. SLAB) (flip = 4: of a slab of 64 columns the second 32 come first in v).  With accumulate the slab of C is read and added in binary32 before the one rounding.
template <typename C, typename P>
__device__ __forceinline__ void write_slab(const P& p, uint32_t staging, int row0, int col0, const float* v, int flip = 0) {
    constexpr int PER16 = Out<C>::PER16, SLAB = 8 * PER16;
    const int lane = threadIdx.x & 31;
    const int nrows = p.M - row0 < 32 ? p.M - row0 : 32, n = p.N - col0 < SLAB ? p.N - col0 : SLAB;
    if (nrows <= 0 || n <= 0) return;
    C* c = static_cast<C*>(p.C);
    __syncwarp();
    if (!p.accumulate) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint4 q = Out<C>::pack(v + j * PER16);
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(staging + lane * 128 + ((j ^ flip ^ (lane & 7)) << 4)), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
        }
        __syncwarp();
        if (p.c_vec && n == SLAB) {
#pragma unroll
            for (int it = 0; it < 8; ++it) {
                const int r = it * 4 + (lane >> 3), j = lane & 7;
                uint4 q;
                asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(staging + r * 128 + ((j ^ (r & 7)) << 4)) : "memory");
                if (r < nrows) *reinterpret_cast<uint4*>(c + (int64_t)(row0 + r) * p.ldc + col0 + j * PER16) = q;
            }
        } else if (sizeof(C) == 2 && p.c_pair) {
            // rows that start on 4-byte boundaries: two elements at a time
            const int e = 2 * lane;
            for (int r = 0; r < nrows; ++r) {
                uint32_t q;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(q) : "r"(staging + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4) : "memory");
                C* dst = c + (int64_t)(row0 + r) * p.ldc + col0 + e;
                if (e + 1 < n) *reinterpret_cast<uint32_t*>(dst) = q;
                else if (e < n) *reinterpret_cast<uint16_t*>(dst) = (uint16_t)q;
            }
        } else {
            for (int r = 0; r < nrows; ++r)
                for (int e = lane; e < n; e += 32) {
                    const uint32_t at = staging + r * 128 + (((e / PER16) ^ (r & 7)) << 4) + (e % PER16) * sizeof(C);
                    C* dst = c + (int64_t)(row0 + r) * p.ldc + col0 + e;
                    if constexpr (sizeof(C) == 4) {
                        float q;
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(q) : "r"(at) : "memory");
                        *dst = q;
                    } else {
                        uint16_t q;
                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(q) : "r"(at) : "memory");
                        *reinterpret_cast<uint16_t*>(dst) = q;
                    }
                }
        }
    } else {
        // binary32 through the staging rows, 32 columns at a time
#pragma unroll
        for (int h = 0; h < SLAB / 32; ++h) {
            const int hc = (h ^ (flip >> 2)) * 32;                         // first column of these 32
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 8; ++j)
                asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(staging + lane * 128 + ((j ^ (lane & 7)) << 4)), "f"(v[h * 32 + 4 * j]), "f"(v[h * 32 + 4 * j + 1]),
                             "f"(v[h * 32 + 4 * j + 2]), "f"(v[h * 32 + 4 * j + 3]) : "memory");
            __syncwarp();
            if (p.c_vec && n == SLAB) {
                // (all reads of C before the first store to it: they are independent, which the compiler cannot know)
                constexpr int W = sizeof(C);                                // 32-bit words of four elements
                uint32_t old[8][W];
#pragma unroll
                for (int it = 0; it < 8; ++it) {
                    const int r = it * 4 + (lane >> 3), j = lane & 7;
                    const C* src = c + (int64_t)(row0 + r) * p.ldc + col0 + hc + j * 4;
                    if (r < nrows) {
                        if constexpr (W == 4) *reinterpret_cast<uint4*>(old[it]) = *reinterpret_cast<const uint4*>(src);
                        else *reinterpret_cast<uint2*>(old[it]) = *reinterpret_cast<const uint2*>(src);
                    }
                }
#pragma unroll
                for (int it = 0; it < 8; ++it) {
                    const int r = it * 4 + (lane >> 3), j = lane & 7;
                    float4 q;
                    asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w) : "r"(staging + r * 128 + ((j ^ (r & 7)) << 4)) : "memory");
                    if (r < nrows) {
                        C* dst = c + (int64_t)(row0 + r) * p.ldc + col0 + hc + j * 4;
                        if constexpr (sizeof(C) == 4) {
                            *reinterpret_cast<float4*>(dst) = make_float4(__uint_as_float(old[it][0]) + q.x, __uint_as_float(old[it][1]) + q.y,
                                                                          __uint_as_float(old[it][2]) + q.z, __uint_as_float(old[it][3]) + q.w);
                        } else {
                            const uint32_t o0 = old[it][0], o1 = old[it][1];
                            *reinterpret_cast<uint2*>(dst) = make_uint2(
                                Out<C>::two(__uint_as_float(o0 << 16) + q.x, __uint_as_float(o0 & 0xFFFF0000u) + q.y),
                                Out<C>::two(__uint_as_float(o1 << 16) + q.z, __uint_as_float(o1 & 0xFFFF0000u) + q.w));
                        }
                    }
                }
            } else {
                const int e = hc + lane;
                C* at = c + (int64_t)row0 * p.ldc + col0 + e;
#pragma unroll 1
                for (int r0 = 0; r0 < nrows; r0 += 8) {                    // (eight reads of C before their stores)
                    float old[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) old[i] = e < n && r0 + i < nrows ? (float)at[(r0 + i) * p.ldc] : 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int r = r0 + i;
                        float q;
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(q) : "r"(staging + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4) : "memory");
                        if (e < n && r < nrows) at[r * p.ldc] = (C)(old[i] + q);
                    }
                }
            }
        }
    }
}

// a barrier of this block (CG = 1), or the one at the same place in both blocks of the pair
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
    if constexpr (CG == 1) tc_commit(bar);
    else asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ uint32_t in_block(uint32_t saddr, uint32_t rank) {     // the same place in the shared memory of another block of the cluster
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
    return r;
}
template <int CG>
__device__ __forceinline__ void arrive(uint32_t bar) {                            // CG = 2: an address from in_block
    if constexpr (CG == 1) mbar_arrive(bar);
    else asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void tma_load_operand(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if constexpr (CG == 1) tma_load_2d(dst, map, x, y, bar);
    else asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// The common exit: every warp comes here, whatever it waited for in vain.
template <int CG = 1, typename P>
__device__ __forceinline__ void leave(const P& p, bool failed, int warp, int lane, uint32_t tmem) {
    if (failed) {
        if (lane == 0) atomicExch(p.status, STATUS_TIMEOUT);
        const unsigned long long start = global_ns();
        while (global_ns() - start < 2000000ull) { }    // let copies and products in flight finish
    }
    if (!p.early) grid_dependents_may_launch();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        if constexpr (CG == 1) tc_dealloc(tmem, 512u);
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

}  // namespace mma
}  // namespace cerar
