// Norms of queries and keys for each head, with the rotation by position in the same pass, and their gradient
// (cerar_head_norm, cerar_head_norm_grad).  Per row x of `dim` values (one head of one token):
//
//   r = (mean x^2 + eps)^-1/2,  n = r x,  z = w n,   y = z with the pairs (a, b) of its first `rotated` values turned:
//                                                    (a cos - b sin, b cos + a sin), angles from a table by the token's position
//   dz = dy turned back,  dw += sum over rows of dz n,  dn = w dz,  dx = r (dn - n mean(dn n))
//
// Memory bound: forward reads and writes every value once, backward reads x and dy and writes dx; r is computed again from x, which
// has to be read anyway.  A row belongs to a group of 1 .. 32 threads; a thread holds two chunks of it that contain both parts
// of its pairs (the two halves' same places, or neighbours), so that nothing but the sums crosses threads.  The group goes through
// several heads of one token with the weights and the rotation, worked into one another, in registers; the loads of a few heads are on their
// way together.  With p = dz x the gradient needs sum x^2 and sum w p only, one exchange for both: dw += r p, dx = r w dz - x r^3 mean(w p).
// dw is summed in registers over all rows of a thread, then over the block in a fixed order; a second launch adds the blocks up.
// (A grid of heads by tokens: two 64-bit divisions per row cost as many instructions as the row's arithmetic.)
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "kernels.cuh"
#include "ops.cuh"
#include "packed.cuh"
#include "ptx.cuh"

namespace cerar {
namespace {

using namespace packed;
using namespace ptx;

constexpr int THREADS = 128;

// CH elements of a row as they lie in memory (aligned to the chunk), as binary32, and back with one rounding.  Plain loads, not read-only ones: a row may be
// written where it was read (a thread writes the very places that it has read before).
template <typename T, int CH> struct Chunk;
template <int CH> struct Chunk<float, CH> {
    uint32_t q[CH];
    __device__ __forceinline__ void load(const float* p) {
        if constexpr (CH == 4) *reinterpret_cast<uint4*>(q) = *reinterpret_cast<const uint4*>(p);
        else if constexpr (CH == 2) *reinterpret_cast<uint2*>(q) = *reinterpret_cast<const uint2*>(p);
        else q[0] = __float_as_uint(*p);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < CH; ++i) q[i] = 0u;
    }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(q[i]); }
    __device__ __forceinline__ uint64_t two(int i) const { return two_of(__uint_as_float(q[2 * i]), __uint_as_float(q[2 * i + 1])); }
    static __device__ __forceinline__ void store(float* p, const float* v) {
        if constexpr (CH == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        else if constexpr (CH == 2) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
        else p[0] = v[0];
    }
};
template <int CH> struct Chunk<__nv_bfloat16, CH> {
    static constexpr int WORDS = CH > 1 ? CH / 2 : 1;
    uint32_t q[WORDS];
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        if constexpr (CH == 8) *reinterpret_cast<uint4*>(q) = *reinterpret_cast<const uint4*>(p);
        else if constexpr (CH == 4) *reinterpret_cast<uint2*>(q) = *reinterpret_cast<const uint2*>(p);
        else if constexpr (CH == 2) q[0] = *reinterpret_cast<const uint32_t*>(p);
        else q[0] = *reinterpret_cast<const unsigned short*>(p);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) q[i] = 0u;
    }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? q[i / 2] & 0xFFFF0000u : q[i / 2] << 16); }
    __device__ __forceinline__ uint64_t two(int i) const { return of_bf16(q[i]); }
    static __device__ __forceinline__ uint32_t word(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* v) {
        if constexpr (CH == 8) *reinterpret_cast<uint4*>(p) = make_uint4(word(v[0], v[1]), word(v[2], v[3]), word(v[4], v[5]), word(v[6], v[7]));
        else if constexpr (CH == 4) *reinterpret_cast<uint2*>(p) = make_uint2(word(v[0], v[1]), word(v[2], v[3]));
        else if constexpr (CH == 2) *reinterpret_cast<uint32_t*>(p) = word(v[0], v[1]);
        else p[0] = __float2bfloat16_rn(v[0]);
    }
};

struct Work {                                  // how a launch is cut up
    int log_lanes;                             // threads per row
    int chunks;                                // chunks of half a row
    int run;                                   // heads of a token that a group goes through
    int runs[2], rows;                         // of each part, of both
    int w_vec;                                 // weights are aligned to whole chunks
    float* partial;                            // gradient of w: [part][block][dim]
};

// Where a thread's chunk c lies: the offsets of its two halves, whether its pairs are turned, and their number.
struct Place {
    int a, b;
    bool turned;
    int pair;
};
__device__ __forceinline__ Place place(const HeadNormArgs& p, int c, int ch) {
    const int h = p.rotated / 2, first = c * ch;
    if (p.neighbours) return {2 * first, 2 * first + ch, 2 * first < p.rotated, first};
    if (first < h) return {first, h + first, true, first};
    return {p.rotated + first - h, p.rotated + first - h + (p.dim - p.rotated) / 2, false, 0};
}
// Position of token t: below zero where it is padding; beyond the table it is reported and taken for padding.
__device__ __forceinline__ int64_t position_of(const HeadNormArgs& p, uint32_t t) {
    const uint32_t i = p.period > t ? t : t % (uint32_t)p.period;
    int64_t at = i;
    if (p.positions) at = p.position_bytes == 8 ? __ldg(static_cast<const long long*>(p.positions) + i) : (int64_t)__ldg(static_cast<const int*>(p.positions) + i);
    if (at >= p.table_rows) {
        atomicCAS(p.status, 0, STATUS_BEYOND);
        return -1;
    }
    return at;
}
// A thread's part of a row: NCH times two chunks, in CH packed pairs of neighbours each.  The value that each one is turned with lies in the
// other chunk's same place, or next to it (neighbours; chunks of one value).
template <typename T, int CH, int NCH> struct Raw {
    Chunk<T, CH> a[NCH], b[NCH];
    __device__ __forceinline__ void load(const T* row, const Place* at, const bool* mine) {
#pragma unroll
        for (int j = 0; j < NCH; ++j)
            if (mine[j]) {
                a[j].load(row + at[j].a);
                b[j].load(row + at[j].b);
            }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < NCH; ++j) { a[j].clear(); b[j].clear(); }
    }
    __device__ __forceinline__ void take(uint64_t (*v)[CH]) const {
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            if constexpr (CH == 1) {
                v[j][0] = two_of(a[j].get(0), b[j].get(0));
            } else {
#pragma unroll
                for (int m = 0; m < CH / 2; ++m) { v[j][m] = a[j].two(m); v[j][CH / 2 + m] = b[j].two(m); }
            }
        }
    }
};
// What values m are turned with: zero where they are not turned, or zero times an infinite neighbour would be NaN.
template <int CH, bool NEIGHBOURS>
__device__ __forceinline__ uint64_t partner(const uint64_t* v, int m, bool turned) {
    return !turned ? 0ull : NEIGHBOURS || CH == 1 ? swapped(v[m]) : v[(m + CH / 2) % CH];
}
template <typename T, int CH>
__device__ __forceinline__ void store_pairs(T* row, const Place& at, const uint64_t* v) {
    float f[2 * CH];
#pragma unroll
    for (int m = 0; m < CH; ++m) parts(v[m], f[2 * m], f[2 * m + 1]);
    Chunk<T, CH>::store(row + at.a, f);
    Chunk<T, CH>::store(row + at.b, f + CH);
}
// Cosine and sine for every one of a thread's values: y = v c + partner s, the sine negative for the first of a pair.  sign = -1: turned back.
template <int CH, bool NEIGHBOURS>
__device__ __forceinline__ void rotation_of(const HeadNormArgs& p, int64_t pos, const Place& at, bool mine, float sign, float* c, float* s) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const float2 turn = pos >= 0 && mine && at.turned ? __ldg(p.table + pos * (p.rotated / 2) + at.pair + i) : make_float2(1.f, 0.f);
        const int f = NEIGHBOURS ? 2 * i : i, g = NEIGHBOURS ? 2 * i + 1 : CH + i;
        c[f] = c[g] = turn.x;
        s[f] = -sign * turn.y;
        s[g] = sign * turn.y;
    }
}

// The 2 CH weights of a thread's chunk
template <typename W, int CH>
__device__ __forceinline__ void load_weights(const W* w, const Place& at, bool vec, float* v) {
    if (vec) {
        Chunk<W, CH> a, b;
        a.load(w + at.a);
        b.load(w + at.b);
#pragma unroll
        for (int e = 0; e < CH; ++e) { v[e] = a.get(e); v[CH + e] = b.get(e); }
    } else {
#pragma unroll
        for (int e = 0; e < 2 * CH; ++e) v[e] = (float)w[e < CH ? at.a + e : at.b + e - CH];
    }
}
template <int CH>
__device__ __forceinline__ void weights(const HeadNormArgs& p, const void* w, const Place& at, bool vec, float* v) {
    if (w == nullptr) {
#pragma unroll
        for (int e = 0; e < 2 * CH; ++e) v[e] = 1.f;
    } else if (p.w_type == CERAR_TYPE_F32) {
        if constexpr (CH <= 4) load_weights<float, CH>(static_cast<const float*>(w), at, vec, v);
        else {                                  // (chunks of 8 binary32 values: two of 4)
            load_weights<float, 4>(static_cast<const float*>(w), {at.a, at.a + 4, false, 0}, vec, v);
            load_weights<float, 4>(static_cast<const float*>(w), {at.b, at.b + 4, false, 0}, vec, v + 8);
        }
    } else {
        load_weights<__nv_bfloat16, CH>(static_cast<const __nv_bfloat16*>(w), at, vec, v);
    }
}

// NCH: chunks per thread.  DEPTH: heads whose loads are on their way.  NEIGHBOURS: which values are a pair.  WHOLE: all of them are turned (as a value of the launch it costs
// 16384 x 40 x 128 in bfloat16 56.6 -> 57.7 us).
// A block: a run of heads (the faster index, so that whole tokens are read at a time) of some tokens.  Threads without a token (a chunk) stay, with zeros: they share their warp's sums.
template <typename T, int CH, int NCH, int DEPTH, bool NEIGHBOURS, bool WHOLE>
__global__ void __launch_bounds__(THREADS) head_norm_kernel(const HeadNormArgs p, const Work wk) {
    grid_dependency_wait();
    const uint32_t column = blockIdx.x / wk.rows;
    const int row = (int)(blockIdx.x - column * wk.rows), part = row < wk.runs[0] ? 0 : 1;
    const HeadPart& h = p.part[part];
    const int lanes = 1 << wk.log_lanes, lane = threadIdx.x & (lanes - 1);
    const int64_t t = (int64_t)column * (THREADS >> wk.log_lanes) + (threadIdx.x >> wk.log_lanes);
    const bool there = t < p.tokens;
    const int first = (row - (part ? wk.runs[0] : 0)) * wk.run, last = first + wk.run < h.heads ? first + wk.run : h.heads;
    Place at[NCH];
    bool mine[NCH];
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const int c = lane + j * lanes;
        mine[j] = there && c < wk.chunks;
        at[j] = place(p, mine[j] ? c : 0, CH);
    }
    const T* x = static_cast<const T*>(h.x) + t * h.x_token + first * h.x_head;
    T* y = static_cast<T*>(h.y) + t * h.y_token + first * h.y_head;
    Raw<T, CH, NCH> raw[DEPTH];
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
        raw[i].clear();
        if (first + i < last) raw[i].load(x, at, mine);
        x += h.x_head;
    }
    // y = r (v vc + partner vs): weights and rotation in one
    const int64_t pos = there ? position_of(p, (uint32_t)t) : -1;
    uint64_t vc[NCH][CH], vs[NCH][CH];
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        float w[2 * CH], c[2 * CH], s[2 * CH];
        weights<CH>(p, h.w, at[j], wk.w_vec, w);
        rotation_of<CH, NEIGHBOURS>(p, pos, at[j], mine[j], 1.f, c, s);
        uint64_t pw[CH];
#pragma unroll
        for (int m = 0; m < CH; ++m) pw[m] = two_of(w[2 * m], w[2 * m + 1]);
#pragma unroll
        for (int m = 0; m < CH; ++m) {
            vc[j][m] = mul2(pw[m], two_of(c[2 * m], c[2 * m + 1]));
            vs[j][m] = mul2(partner<CH, NEIGHBOURS>(pw, m, WHOLE || at[j].turned), two_of(s[2 * m], s[2 * m + 1]));
            if (pos < 0) vc[j][m] = vs[j][m] = 0ull;                 // (padding: zero whatever the weights are)
        }
    }
    const float inv_dim = 1.f / (float)p.dim;
    for (int head0 = first; head0 < last; head0 += DEPTH)
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            if (head0 + i >= last) break;
            uint64_t v[NCH][CH], sum2 = 0ull;
            if (pos < 0) raw[i].clear();        // (padding may hold anything)
            raw[i].take(v);
            if (head0 + i + DEPTH < last) raw[i].load(x, at, mine);
            x += h.x_head;
#pragma unroll
            for (int j = 0; j < NCH; ++j)
#pragma unroll
                for (int m = 0; m < CH; ++m) sum2 = mad2(v[j][m], v[j][m], sum2);
            float sum, other;
            parts(sum2, sum, other);
            sum += other;
            for (int o = lanes >> 1; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const uint64_t r = all(rsqrtf(fmaf(sum, inv_dim, p.eps)));
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                uint64_t z[CH];
#pragma unroll
                for (int m = 0; m < CH; ++m) z[m] = mul2(r, mad2(v[j][m], vc[j][m], mul2(partner<CH, NEIGHBOURS>(v[j], m, WHOLE || at[j].turned), vs[j][m])));
                if (mine[j]) store_pairs<T, CH>(y, at[j], z);
            }
            y += h.y_head;
        }
}

template <typename T, int CH, int NCH, int DEPTH, bool NEIGHBOURS, bool WHOLE>
__global__ void __launch_bounds__(THREADS) head_norm_grad_kernel(const HeadNormArgs p, const Work wk) {
    extern __shared__ float sums[];                              // [groups of the block][dim]: their shares of dw
    grid_dependency_wait();
    const uint32_t column = blockIdx.x / wk.rows, columns = gridDim.x / wk.rows;
    const int row = (int)(blockIdx.x - column * wk.rows), part = row < wk.runs[0] ? 0 : 1;
    const HeadPart& h = p.part[part];
    const int lanes = 1 << wk.log_lanes, lane = threadIdx.x & (lanes - 1), per_block = THREADS >> wk.log_lanes;
    const int run = row - (part ? wk.runs[0] : 0), first = run * wk.run, last = first + wk.run < h.heads ? first + wk.run : h.heads;
    Place at[NCH];
    uint64_t w[NCH][CH], dw[NCH][CH];
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const int c = lane + j * lanes;
        at[j] = place(p, c < wk.chunks ? c : 0, CH);
        float f[2 * CH];
        weights<CH>(p, h.w, at[j], wk.w_vec, f);
#pragma unroll
        for (int m = 0; m < CH; ++m) {
            w[j][m] = two_of(f[2 * m], f[2 * m + 1]);
            dw[j][m] = 0ull;
        }
    }
    const float inv_dim = 1.f / (float)p.dim;
    for (int64_t t0 = (int64_t)column * per_block; t0 < p.tokens; t0 += (int64_t)columns * per_block) {
        const int64_t t = t0 + (threadIdx.x >> wk.log_lanes);
        bool mine[NCH];
#pragma unroll
        for (int j = 0; j < NCH; ++j) mine[j] = t < p.tokens && lane + j * lanes < wk.chunks;
        const T* x = static_cast<const T*>(h.x) + t * h.x_token + first * h.x_head;
        const T* dy = static_cast<const T*>(h.dy) + t * h.dy_token + first * h.dy_head;
        T* dx = static_cast<T*>(h.y) + t * h.y_token + first * h.y_head;
        Raw<T, CH, NCH> rx[DEPTH], ry[DEPTH];
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            rx[i].clear();
            ry[i].clear();
            if (first + i < last) {
                rx[i].load(x, at, mine);
                ry[i].load(dy, at, mine);
            }
            x += h.x_head;
            dy += h.dy_head;
        }
        const int64_t pos = t < p.tokens ? position_of(p, (uint32_t)t) : -1;
        uint64_t vc[NCH][CH], vs[NCH][CH];
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            float c[2 * CH], s[2 * CH];
            rotation_of<CH, NEIGHBOURS>(p, pos, at[j], mine[j], -1.f, c, s);
#pragma unroll
            for (int m = 0; m < CH; ++m) {
                vc[j][m] = two_of(c[2 * m], c[2 * m + 1]);
                vs[j][m] = two_of(s[2 * m], s[2 * m + 1]);
            }
        }
        for (int head0 = first; head0 < last; head0 += DEPTH)
#pragma unroll
            for (int i = 0; i < DEPTH; ++i) {
                if (head0 + i >= last) break;
                if (pos < 0) {                  // (padding may hold anything)
                    rx[i].clear();
                    ry[i].clear();
                }
                uint64_t v[NCH][CH], dz[NCH][CH], square2 = 0ull, dot2 = 0ull;
                rx[i].take(v);
                {
                    uint64_t g[NCH][CH];
                    ry[i].take(g);
                    if (head0 + i + DEPTH < last) {
                        rx[i].load(x, at, mine);
                        ry[i].load(dy, at, mine);
                    }
                    x += h.x_head;
                    dy += h.dy_head;
#pragma unroll
                    for (int j = 0; j < NCH; ++j)
#pragma unroll
                        for (int m = 0; m < CH; ++m) dz[j][m] = mad2(g[j][m], vc[j][m], mul2(partner<CH, NEIGHBOURS>(g[j], m, WHOLE || at[j].turned), vs[j][m]));
                }
#pragma unroll
                for (int j = 0; j < NCH; ++j)
#pragma unroll
                    for (int m = 0; m < CH; ++m) {
                        square2 = mad2(v[j][m], v[j][m], square2);
                        dot2 = mad2(mul2(w[j][m], dz[j][m]), v[j][m], dot2);
                    }
                float square, dot, other;
                parts(square2, square, other);
                square += other;
                parts(dot2, dot, other);
                dot += other;
                for (int o = lanes >> 1; o; o >>= 1) {
                    square += __shfl_xor_sync(0xffffffffu, square, o);
                    dot += __shfl_xor_sync(0xffffffffu, dot, o);
                }
                const float r = rsqrtf(fmaf(square, inv_dim, p.eps));
                const uint64_t r2 = all(r), back = all(-(dot * inv_dim) * r * r * r);
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    uint64_t u[CH];
#pragma unroll
                    for (int m = 0; m < CH; ++m) {
                        const uint64_t rz = mul2(r2, dz[j][m]);
                        dw[j][m] = mad2(rz, v[j][m], dw[j][m]);
                        u[m] = mad2(v[j][m], back, mul2(rz, w[j][m]));
                    }
                    if (pos < 0)                // (zero whatever the weights are)
#pragma unroll
                        for (int m = 0; m < CH; ++m) u[m] = 0ull;
                    if (mine[j]) store_pairs<T, CH>(dx, at[j], u);
                }
                dx += h.y_head;
            }
    }
    if (h.dw == nullptr) return;                                 // (the same for the whole block)
    float* share = sums + (threadIdx.x >> wk.log_lanes) * p.dim;
#pragma unroll
    for (int j = 0; j < NCH; ++j)
        if (lane + j * lanes < wk.chunks)
#pragma unroll
            for (int m = 0; m < CH; ++m) {
                float f[2];
                parts(dw[j][m], f[0], f[1]);
#pragma unroll
                for (int i = 0; i < 2; ++i) share[2 * m + i < CH ? at[j].a + 2 * m + i : at[j].b + 2 * m + i - CH] = f[i];
            }
    __syncthreads();
    float* out = wk.partial + ((int64_t)part * HEAD_NORM_BLOCKS + (int64_t)run * columns + column) * p.dim;
    for (int c = threadIdx.x; c < p.dim; c += THREADS) {
        float v = 0.f;
        for (int g = 0; g < per_block; ++g) v += sums[g * p.dim + c];
        out[c] = v;
    }
}

// The same for bfloat16 in whole 16-byte chunks, one to a thread's half.  Rows, and a token's part of the table, are on their way in shared memory, in
// slots of the thread's own (nothing has to be waited for but its own copies): AHEAD heads of the block's sequence of tokens and heads, over the
// ends of tokens, and no register holds them.  16384 x 40 x 128 in a loop 87 us, 5.9 TB/s, and 95 with L2 flushed before each pass (two heads of one token ahead
// in registers, and the table's latency at each token: 104 and 112; in a loop one or three heads here 99 and 86, 4096 x 20 x 256 with one to
// three 35, 32, 33; four blocks per SM in one turn, eight in two: 90).  Copies go through L1, or the halves of a 32-byte piece come from L2 twice (neighbours: 144).  binary32 has twice the bytes per
// instruction and is slower this way (168 -> 196).
constexpr int AHEAD = 2, SLOTS = AHEAD + 1, AHEAD_BLOCKS = 4;
__device__ __forceinline__ void copy16(uint32_t to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ void shared16(uint32_t from, uint32_t* q) {
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]) : "r"(from) : "memory");
}
constexpr int PIECE = 16 * THREADS;                              // 16 bytes of every thread
constexpr int TURN = 4;                                          // pieces of a chunk's eight pairs (cos, sin)
constexpr int RING_BYTES = (SLOTS * 4 + 2 * TURN) * PIECE;

template <bool NEIGHBOURS, bool WHOLE>
__global__ void __launch_bounds__(THREADS, AHEAD_BLOCKS) head_norm_grad_ahead_kernel(const HeadNormArgs p, const Work wk) {
    using T = __nv_bfloat16;
    constexpr int CH = 8;
    extern __shared__ __align__(16) float sums[];                // the ring; in the end [groups of the block][dim]: their shares of dw
    grid_dependency_wait();
    const uint32_t column = blockIdx.x / wk.rows, columns = gridDim.x / wk.rows;
    const int row = (int)(blockIdx.x - column * wk.rows), part = row < wk.runs[0] ? 0 : 1;
    const HeadPart& h = p.part[part];
    const int lanes = 1 << wk.log_lanes, lane = threadIdx.x & (lanes - 1), per_block = THREADS >> wk.log_lanes;
    const int run = row - (part ? wk.runs[0] : 0), first = run * wk.run, len = (first + wk.run < h.heads ? first + wk.run : h.heads) - first;
    const bool mine = lane < wk.chunks;
    const Place at = place(p, mine ? lane : 0, CH);
    uint64_t w[CH], dw[CH];
    {
        float f[2 * CH];
        weights<CH>(p, h.w, at, wk.w_vec, f);
#pragma unroll
        for (int m = 0; m < CH; ++m) {
            w[m] = two_of(f[2 * m], f[2 * m + 1]);
            dw[m] = 0ull;
        }
    }
    const float inv_dim = 1.f / (float)p.dim;
    const int64_t t0 = (int64_t)column * per_block, step = (int64_t)columns * per_block;
    const int64_t items = t0 < p.tokens ? (p.tokens - t0 + step - 1) / step * len : 0;       // the same for the whole block
    const int dist = len < AHEAD ? len : AHEAD;                  // (no further than into the next token)
    const uint32_t own = smem_u32(sums) + 16 * threadIdx.x, turns = own + SLOTS * 4 * PIECE;

    // what is brought next: token it, its head ih; positions of that token and the one behind it
    int64_t it = t0 + (threadIdx.x >> wk.log_lanes), left = items;
    int64_t pos_in = -1, pos_next = it < p.tokens ? position_of(p, (uint32_t)it) : -1;
    int ih = 0, slot_in = 0, turn_in = 0;
    const T *x = nullptr, *dy = nullptr;
    auto bring = [&]() {
        if (left > 0) {
            --left;
            if (ih == 0) {
                pos_in = pos_next;
                if (pos_in >= 0 && mine && at.turned) {
                    const float2* from = p.table + pos_in * (p.rotated / 2) + at.pair;
#pragma unroll
                    for (int i = 0; i < TURN; ++i) copy16(turns + (turn_in * TURN + i) * PIECE, from + 2 * i);
                }
                turn_in ^= 1;
                x = static_cast<const T*>(h.x) + it * h.x_token + first * h.x_head;
                dy = static_cast<const T*>(h.dy) + it * h.dy_token + first * h.dy_head;
                it += step;
                pos_next = it < p.tokens ? position_of(p, (uint32_t)it) : -1;
            }
            if (pos_in >= 0 && mine) {
                const uint32_t to = own + slot_in * 4 * PIECE;
                copy16(to, x + at.a);
                copy16(to + PIECE, x + at.b);
                copy16(to + 2 * PIECE, dy + at.a);
                copy16(to + 3 * PIECE, dy + at.b);
            }
            x += h.x_head;
            dy += h.dy_head;
            slot_in = slot_in + 1 == SLOTS ? 0 : slot_in + 1;
            if (++ih == len) ih = 0;
        }
        copies_done();
    };
    for (int i = 0; i < dist; ++i) bring();

    int64_t pos = -1, t = t0 + (threadIdx.x >> wk.log_lanes);
    int head = 0, slot = 0, turn = 0;
    T* dx = nullptr;
    uint64_t vc[CH], vs[CH];
    for (int64_t k = 0; k < items; ++k) {
        if (dist == AHEAD) copies_wait<AHEAD - 1>();
        else copies_wait<0>();
        if (head == 0) {
            pos = pos_in;                                        // (what is on its way is of this token as yet)
            dx = static_cast<T*>(h.y) + t * h.y_token + first * h.y_head;
            t += step;
            float q[2 * CH];                                     // cosine and sine of each pair
#pragma unroll
            for (int i = 0; i < CH; ++i) { q[2 * i] = 1.f; q[2 * i + 1] = 0.f; }
            if (pos >= 0 && mine && at.turned)
#pragma unroll
                for (int i = 0; i < TURN; ++i) shared16(turns + (turn * TURN + i) * PIECE, reinterpret_cast<uint32_t*>(q) + 4 * i);
            turn ^= 1;
            float c[2 * CH], s[2 * CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int f = NEIGHBOURS ? 2 * i : i, g = NEIGHBOURS ? 2 * i + 1 : CH + i;
                c[f] = c[g] = q[2 * i];
                s[f] = q[2 * i + 1];
                s[g] = -q[2 * i + 1];
            }
#pragma unroll
            for (int m = 0; m < CH; ++m) {
                vc[m] = two_of(c[2 * m], c[2 * m + 1]);
                vs[m] = two_of(s[2 * m], s[2 * m + 1]);
            }
        }
        Raw<T, CH, 1> rx, ry;
        rx.clear();                                              // (padding may hold anything)
        ry.clear();
        if (pos >= 0 && mine) {
            const uint32_t from = own + slot * 4 * PIECE;
            shared16(from, rx.a[0].q);
            shared16(from + PIECE, rx.b[0].q);
            shared16(from + 2 * PIECE, ry.a[0].q);
            shared16(from + 3 * PIECE, ry.b[0].q);
        }
        slot = slot + 1 == SLOTS ? 0 : slot + 1;
        bring();                                                 // into the slot of the head before this one
        uint64_t v[1][CH], dz[CH], square2 = 0ull, dot2 = 0ull;
        rx.take(v);
        {
            uint64_t g[1][CH];
            ry.take(g);
#pragma unroll
            for (int m = 0; m < CH; ++m) dz[m] = mad2(g[0][m], vc[m], mul2(partner<CH, NEIGHBOURS>(g[0], m, WHOLE || at.turned), vs[m]));
        }
#pragma unroll
        for (int m = 0; m < CH; ++m) {
            square2 = mad2(v[0][m], v[0][m], square2);
            dot2 = mad2(mul2(w[m], dz[m]), v[0][m], dot2);
        }
        float square, dot, other;
        parts(square2, square, other);
        square += other;
        parts(dot2, dot, other);
        dot += other;
        for (int o = lanes >> 1; o; o >>= 1) {
            square += __shfl_xor_sync(0xffffffffu, square, o);
            dot += __shfl_xor_sync(0xffffffffu, dot, o);
        }
        const float r = rsqrtf(fmaf(square, inv_dim, p.eps));
        const uint64_t r2 = all(r), back = all(-(dot * inv_dim) * r * r * r);
        uint64_t u[CH];
#pragma unroll
        for (int m = 0; m < CH; ++m) {
            const uint64_t rz = mul2(r2, dz[m]);
            dw[m] = mad2(rz, v[0][m], dw[m]);
            u[m] = mad2(v[0][m], back, mul2(rz, w[m]));
        }
        if (pos < 0)                                             // (zero whatever the weights are)
#pragma unroll
            for (int m = 0; m < CH; ++m) u[m] = 0ull;
        if (mine && t - step < p.tokens) store_pairs<T, CH>(dx, at, u);
        dx += h.y_head;
        if (++head == len) head = 0;
    }
    if (h.dw == nullptr) return;                                 // (the same for the whole block)
    __syncthreads();                                             // (nothing is on its way to the ring: all of it has been waited for)
    float* share = sums + (threadIdx.x >> wk.log_lanes) * p.dim;
    if (mine)
#pragma unroll
        for (int m = 0; m < CH; ++m) {
            float f[2];
            parts(dw[m], f[0], f[1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) share[2 * m + i < CH ? at.a + 2 * m + i : at.b + 2 * m + i - CH] = f[i];
        }
    __syncthreads();
    float* out = wk.partial + ((int64_t)part * HEAD_NORM_BLOCKS + (int64_t)run * columns + column) * p.dim;
    for (int c = threadIdx.x; c < p.dim; c += THREADS) {
        float v = 0.f;
        for (int g = 0; g < per_block; ++g) v += sums[g * p.dim + c];
        out[c] = v;
    }
}

// dw (+)= the blocks' shares, in their order: a block per 32 columns of a part, or of both where they have one dw; a warp per run of blocks.
constexpr int FOLD_WARPS = 32;
__global__ void __launch_bounds__(32 * FOLD_WARPS) head_norm_fold_kernel(const HeadNormArgs p, const Work wk, int columns) {
    __shared__ float sums[FOLD_WARPS][32];
    grid_dependency_wait();
    const int part = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * 32 + lane;
    void* dw = p.part[part].dw;
    if (dw == nullptr) return;
    float v = 0.f;
    for (int q = part; q < (gridDim.y == 1 ? p.count : part + 1) && c < p.dim; ++q) {
        const int n = columns * wk.runs[q], b0 = (int)((int64_t)n * warp / FOLD_WARPS), b1 = (int)((int64_t)n * (warp + 1) / FOLD_WARPS);
        const float* from = wk.partial + (int64_t)q * HEAD_NORM_BLOCKS * p.dim + c;
#pragma unroll 8
        for (int b = b0; b < b1; ++b) v += from[(int64_t)b * p.dim];
    }
    sums[warp][lane] = v;
    __syncthreads();
    if (warp != 0 || c >= p.dim) return;
    for (int i = 1; i < FOLD_WARPS; ++i) v += sums[i][lane];
    if (p.dw_type == CERAR_TYPE_F32) {
        float* q = static_cast<float*>(dw) + c;
        *q = p.accumulate ? *q + v : v;
    } else {
        __nv_bfloat16* q = static_cast<__nv_bfloat16*>(dw) + c;
        *q = __float2bfloat16_rn(p.accumulate ? __bfloat162float(*q) + v : v);
    }
}

// The largest chunk (elements, at most 16 bytes) that both halves' turned and unturned values consist of and that all rows are aligned to.
int chunk_of(const HeadNormArgs& p, int64_t size, bool grad) {
    for (int ch = (int)(16 / size); ch > 1; ch /= 2) {
        const int64_t bytes = ch * size;
        bool ok = (p.rotated / 2) % ch == 0 && (p.dim / 2) % ch == 0;
        if (grad && ch == 8 && p.rotated > 0) ok = ok && reinterpret_cast<uintptr_t>(p.table) % 16 == 0;      // (read in such pieces)
        for (int i = 0; i < p.count && ok; ++i) {
            const HeadPart& h = p.part[i];
            auto fits = [&](const void* q, int64_t token, int64_t head) {
                return reinterpret_cast<uintptr_t>(q) % bytes == 0 && (p.tokens < 2 || token * size % bytes == 0) && (h.heads < 2 || head * size % bytes == 0);
            };
            if (h.heads == 0) continue;
            ok = fits(h.x, h.x_token, h.x_head) && fits(h.y, h.y_token, h.y_head) && (!grad || fits(h.dy, h.dy_token, h.dy_head));
        }
        if (ok) return ch;
    }
    return 1;
}

template <typename T, int CH, int NCH, int DEPTH, bool NEIGHBOURS, bool WHOLE>
cudaError_t launch_form(const HeadNormArgs& p, bool grad, float* partial, int num_sms, cudaStream_t s, uint64_t* launches) {
    Work wk = {};
    wk.chunks = (p.dim / 2 + CH - 1) / CH;
    constexpr bool ahead = std::is_same<T, __nv_bfloat16>::value && CH == 8;      // (the gradient)
    while (((int64_t)NCH << wk.log_lanes) < wk.chunks) ++wk.log_lanes;
    const int per_block = THREADS >> wk.log_lanes;
    const int64_t columns = (p.tokens + per_block - 1) / per_block;
    wk.w_vec = 1;
    for (int i = 0; i < p.count; ++i) wk.w_vec = wk.w_vec && reinterpret_cast<uintptr_t>(p.part[i].w) % (p.w_type == CERAR_TYPE_F32 ? (CH < 4 ? CH * 4 : 16) : CH * 2) == 0;
    // Eight heads a run share a token's weights and rotation (sixteen where six are loaded at a time); two where there are not enough runs for
    // four blocks per SM.
    // (In the gradient runs are also counted by the blocks whose shares of dw are kept.)
    auto count = [&](int run) {
        wk.run = run;
        for (int i = 0; i < 2; ++i) wk.runs[i] = i < p.count ? (p.part[i].heads + run - 1) / run : 0;
        return wk.runs[0] + wk.runs[1];
    };
    int rows = count(2);
    if (columns * rows >= 4 * num_sms || rows > 256) rows = count(DEPTH > 4 && !grad ? 16 : 8);
    while (rows > (grad ? 256 : 65536)) rows = count(2 * wk.run);
    wk.partial = partial;
    int64_t grid = columns;
    if (grad) {
        const int64_t most = (int64_t)num_sms * (ahead ? AHEAD_BLOCKS : 6) / (rows > 0 ? rows : 1), kept = HEAD_NORM_BLOCKS / (wk.runs[0] > wk.runs[1] ? wk.runs[0] : wk.runs[1] > 0 ? wk.runs[1] : 1);
        if (grid > most) grid = most < 1 ? 1 : most;
        if (grid > kept) grid = kept;
    }
    cudaError_t e = cudaSuccess;
    if (grid > 0 && rows > 0) {
        if (grid * rows > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
        wk.rows = rows;
        const dim3 blocks((unsigned)(grid * rows));
        if (!grad) e = launch_pdl(head_norm_kernel<T, CH, NCH, DEPTH, NEIGHBOURS, WHOLE>, blocks, dim3(THREADS), 0, s, p, wk);
        else if constexpr (ahead) e = launch_pdl(head_norm_grad_ahead_kernel<NEIGHBOURS, WHOLE>, blocks, dim3(THREADS), (size_t)RING_BYTES, s, p, wk);
        else e = launch_pdl(head_norm_grad_kernel<T, CH, NCH, DEPTH, NEIGHBOURS, WHOLE>, blocks, dim3(THREADS), (size_t)per_block * p.dim * 4, s, p, wk);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    if (grad && (p.part[0].dw || (p.count > 1 && p.part[1].dw))) {
        const bool one = p.count > 1 && p.part[0].dw == p.part[1].dw;
        e = launch_pdl(head_norm_fold_kernel, dim3((unsigned)((p.dim + 31) / 32), one ? 1u : (unsigned)p.count), dim3(32 * FOLD_WARPS), 0, s, p, wk, (int)grid);
        if (e == cudaSuccess) ++*launches;
    }
    return e;
}

template <typename T, int CH, int NCH, int DEPTH>
cudaError_t launch_pairs(const HeadNormArgs& p, bool grad, float* partial, int num_sms, cudaStream_t s, uint64_t* launches) {
    auto form = p.rotated == p.dim ? p.neighbours ? launch_form<T, CH, NCH, DEPTH, true, true> : launch_form<T, CH, NCH, DEPTH, false, true>
                                   : p.neighbours ? launch_form<T, CH, NCH, DEPTH, true, false> : launch_form<T, CH, NCH, DEPTH, false, false>;
    return form(p, grad, partial, num_sms, s, launches);
}

// Chunks of 16 bytes go with one or two per thread (half a row is at most 256 values); shorter ones with more, so that a row still fits a warp.
// Heads on their way: as many as registers hold (16384 x 40 x 128 in us, forward bfloat16 with 1, 2, 4, 6, 8: 67, 71, 61, 56, 62; binary32 with
// 1, 2: 120, 107; gradient binary32 200, 167; bfloat16's with 8 values per chunk has its own way).
cudaError_t launch(const HeadNormArgs& p, bool grad, float* partial, int num_sms, cudaStream_t s, uint64_t* launches) {
    if (p.type == CERAR_TYPE_F32) {
        switch (chunk_of(p, 4, grad)) {
            case 4: return launch_pairs<float, 4, 2, 2>(p, grad, partial, num_sms, s, launches);
            case 2: return launch_pairs<float, 2, 4, 1>(p, grad, partial, num_sms, s, launches);
            default: return launch_pairs<float, 1, 8, 1>(p, grad, partial, num_sms, s, launches);
        }
    }
    switch (chunk_of(p, 2, grad)) {
        case 8: return launch_pairs<__nv_bfloat16, 8, 1, 6>(p, grad, partial, num_sms, s, launches);
        case 4: return launch_pairs<__nv_bfloat16, 4, 2, 1>(p, grad, partial, num_sms, s, launches);
        case 2: return launch_pairs<__nv_bfloat16, 2, 4, 1>(p, grad, partial, num_sms, s, launches);
        default: return launch_pairs<__nv_bfloat16, 1, 8, 1>(p, grad, partial, num_sms, s, launches);
    }
}

constexpr int TABLE_PAIRS = CERAR_HEAD_DIM_MAX / 2;
struct Frequencies {
    double f[TABLE_PAIRS];
};
// Angles in binary64: at position 10^6 a binary32 angle is off by up to 0.03.
__global__ void __launch_bounds__(THREADS) rotation_kernel(const Frequencies f, int pairs, int64_t first, int64_t rows, float2* table) {
    grid_dependency_wait();
    for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < rows * pairs; i += (int64_t)gridDim.x * THREADS) {
        const int64_t row = i / pairs;
        double s, c;
        sincos((double)(first + row) * f.f[i - row * pairs], &s, &c);
        table[i] = make_float2((float)c, (float)s);
    }
}

}  // namespace

size_t head_norm_grad_workspace(int count, int dim) { return (size_t)count * HEAD_NORM_BLOCKS * dim * 4; }

cudaError_t launch_head_norm(const HeadNormArgs& a, int num_sms, cudaStream_t s, uint64_t* launches) { return launch(a, false, nullptr, num_sms, s, launches); }
cudaError_t launch_head_norm_grad(const HeadNormArgs& a, void* workspace, int num_sms, cudaStream_t s, uint64_t* launches) {
    return launch(a, true, static_cast<float*>(workspace), num_sms, s, launches);
}

cudaError_t launch_rotation_table(const double* freqs, int pairs, int64_t first, int64_t rows, float* table, int num_sms, cudaStream_t s, uint64_t* launches) {
    Frequencies f = {};
    for (int i = 0; i < pairs; ++i) f.f[i] = freqs[i];
    const int64_t blocks = (rows * pairs + THREADS - 1) / THREADS, most = (int64_t)num_sms * 32;
    const cudaError_t e = launch_pdl(rotation_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(THREADS), 0, s, f, pairs, first, rows, reinterpret_cast<float2*>(table));
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace cerar
