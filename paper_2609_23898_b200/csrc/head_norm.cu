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

#include "kernels.cuh"
#include "ops.cuh"
#include "ptx.cuh"

namespace cerar {
namespace {

using namespace ptx;

constexpr int THREADS = 256;

// CH elements as binary32, and back with one rounding; aligned to the chunk
template <typename T, int CH> struct Chunk;
template <int CH> struct Chunk<float, CH> {
    uint32_t q[CH];
    __device__ __forceinline__ void load(const float* p) {
        if constexpr (CH == 4) *reinterpret_cast<uint4*>(q) = __ldg(reinterpret_cast<const uint4*>(p));
        else if constexpr (CH == 2) *reinterpret_cast<uint2*>(q) = __ldg(reinterpret_cast<const uint2*>(p));
        else q[0] = __float_as_uint(__ldg(p));
    }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(q[i]); }
    static __device__ __forceinline__ void store(float* p, const float* v) {
        if constexpr (CH == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        else if constexpr (CH == 2) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
        else p[0] = v[0];
    }
};
template <int CH> struct Chunk<__nv_bfloat16, CH> {
    uint32_t q[CH > 1 ? CH / 2 : 1];
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        if constexpr (CH == 8) *reinterpret_cast<uint4*>(q) = __ldg(reinterpret_cast<const uint4*>(p));
        else if constexpr (CH == 4) *reinterpret_cast<uint2*>(q) = __ldg(reinterpret_cast<const uint2*>(p));
        else if constexpr (CH == 2) q[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
        else q[0] = __ldg(reinterpret_cast<const unsigned short*>(p));
    }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? q[i / 2] & 0xFFFF0000u : q[i / 2] << 16); }
    static __device__ __forceinline__ uint32_t two(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* v) {
        if constexpr (CH == 8) *reinterpret_cast<uint4*>(p) = make_uint4(two(v[0], v[1]), two(v[2], v[3]), two(v[4], v[5]), two(v[6], v[7]));
        else if constexpr (CH == 4) *reinterpret_cast<uint2*>(p) = make_uint2(two(v[0], v[1]), two(v[2], v[3]));
        else if constexpr (CH == 2) *reinterpret_cast<uint32_t*>(p) = two(v[0], v[1]);
        else p[0] = __float2bfloat16_rn(v[0]);
    }
};

struct Work {                                  // how a launch is cut up
    int log_lanes;                             // threads per row
    int chunks;                                // chunks of half a row
    int run;                                   // heads of a token that a group goes through
    int runs[2];                               // of each part
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
// pair i of the 2 CH values of a chunk (halves: same places of its two parts; neighbours: next to one another)
template <int CH> __device__ __forceinline__ constexpr int first_of(bool neighbours, int i) { return neighbours ? 2 * i : i; }
template <int CH> __device__ __forceinline__ constexpr int second_of(bool neighbours, int i) { return neighbours ? 2 * i + 1 : CH + i; }

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

// NCH: chunks per thread.  HEADS: heads whose loads are on their way together.  NEIGHBOURS: which values are a pair.
// blockIdx.y: a run of heads of a part; blockIdx.x: tokens.
template <typename T, int CH, int NCH, int HEADS, bool NEIGHBOURS>
__global__ void __launch_bounds__(THREADS) head_norm_kernel(const HeadNormArgs p, const Work wk) {
    grid_dependency_wait();
    const int part = (int)blockIdx.y < wk.runs[0] ? 0 : 1;
    const HeadPart& h = p.part[part];
    const int lanes = 1 << wk.log_lanes, lane = threadIdx.x & (lanes - 1);
    const int64_t t = (int64_t)blockIdx.x * (THREADS >> wk.log_lanes) + (threadIdx.x >> wk.log_lanes);
    const bool there = t < p.tokens;            // (threads without a token stay: they share their warp's sums)
    const int first = ((int)blockIdx.y - (part ? wk.runs[0] : 0)) * wk.run, last = there ? (first + wk.run < h.heads ? first + wk.run : h.heads) : first;
    Place at[NCH];
    bool mine[NCH];
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const int c = lane + j * lanes;
        mine[j] = c < wk.chunks;
        at[j] = place(p, mine[j] ? c : 0, CH);
    }
    const T* x = static_cast<const T*>(h.x) + t * h.x_token + first * h.x_head;
    T* y = static_cast<T*>(h.y) + t * h.y_token + first * h.y_head;
    Chunk<T, CH> xa[HEADS][NCH], xb[HEADS][NCH];
    auto load = [&](int head) {
#pragma unroll
        for (int i = 0; i < HEADS; ++i)
#pragma unroll
            for (int j = 0; j < NCH; ++j)
                if (head + i < last && mine[j]) {
                    xa[i][j].load(x + i * h.x_head + at[j].a);
                    xb[i][j].load(x + i * h.x_head + at[j].b);
                }
    };
    load(first);
    // y_a = r (x_a ac - x_b bs), y_b = r (x_b bc + x_a as)
    const int64_t pos = there ? position_of(p, (uint32_t)t) : -1;
    float ac[NCH][CH], as[NCH][CH], bc[NCH][CH], bs[NCH][CH];
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        float w[2 * CH];
        weights<CH>(p, h.w, at[j], wk.w_vec, w);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const float2 turn = pos < 0 ? make_float2(0.f, 0.f) : mine[j] && at[j].turned ? __ldg(p.table + pos * (p.rotated / 2) + at[j].pair + i) : make_float2(1.f, 0.f);
            const float a = w[first_of<CH>(NEIGHBOURS, i)], b = w[second_of<CH>(NEIGHBOURS, i)];
            ac[j][i] = a * turn.x; as[j][i] = a * turn.y; bc[j][i] = b * turn.x; bs[j][i] = b * turn.y;
        }
    }
    const float inv_dim = 1.f / (float)p.dim;
    // (every warp goes through all heads of the run: its groups share sums)
    for (int head = first; head < first + wk.run; head += HEADS) {
        if (head != first) load(head);
        float sum[HEADS];
#pragma unroll
        for (int i = 0; i < HEADS; ++i) {
            sum[i] = 0.f;
            if (head + i < last && pos >= 0) {
#pragma unroll
                for (int j = 0; j < NCH; ++j)
                    if (mine[j])
#pragma unroll
                        for (int e = 0; e < CH; ++e) {
                            sum[i] = fmaf(xa[i][j].get(e), xa[i][j].get(e), sum[i]);
                            sum[i] = fmaf(xb[i][j].get(e), xb[i][j].get(e), sum[i]);
                        }
            }
        }
        for (int o = lanes >> 1; o; o >>= 1)
#pragma unroll
            for (int i = 0; i < HEADS; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
#pragma unroll
        for (int i = 0; i < HEADS; ++i) {
            if (head + i >= last) break;
            const float r = rsqrtf(fmaf(sum[i], inv_dim, p.eps));
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                float z[2 * CH];
#pragma unroll
                for (int e = 0; e < CH; ++e) {
                    constexpr bool N = NEIGHBOURS;
                    const int f = first_of<CH>(N, e), g = second_of<CH>(N, e);
                    const float a = pos < 0 ? 0.f : f < CH ? xa[i][j].get(f < CH ? f : 0) : xb[i][j].get(f < CH ? 0 : f - CH);
                    const float b = pos < 0 ? 0.f : g < CH ? xa[i][j].get(g < CH ? g : 0) : xb[i][j].get(g < CH ? 0 : g - CH);
                    z[f] = r * fmaf(a, ac[j][e], -(b * bs[j][e]));
                    z[g] = r * fmaf(b, bc[j][e], a * as[j][e]);
                }
                if (mine[j]) {
                    Chunk<T, CH>::store(y + i * h.y_head + at[j].a, z);
                    Chunk<T, CH>::store(y + i * h.y_head + at[j].b, z + CH);
                }
            }
        }
        x += HEADS * h.x_head;
        y += HEADS * h.y_head;
    }
}

template <typename T, int CH, int NCH, int HEADS, bool NEIGHBOURS>
__global__ void __launch_bounds__(THREADS) head_norm_grad_kernel(const HeadNormArgs p, const Work wk) {
    extern __shared__ float sums[];                              // [groups of the block][dim]: their shares of dw
    grid_dependency_wait();
    const int part = (int)blockIdx.y < wk.runs[0] ? 0 : 1;
    const HeadPart& h = p.part[part];
    const int lanes = 1 << wk.log_lanes, lane = threadIdx.x & (lanes - 1), per_block = THREADS >> wk.log_lanes;
    const int run = (int)blockIdx.y - (part ? wk.runs[0] : 0), first = run * wk.run;
    Place at[NCH];
    float w[NCH][2 * CH], dw[NCH][2 * CH];
    bool mine[NCH];
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const int c = lane + j * lanes;
        mine[j] = c < wk.chunks;
        at[j] = place(p, mine[j] ? c : 0, CH);
        weights<CH>(p, h.w, at[j], wk.w_vec, w[j]);
#pragma unroll
        for (int e = 0; e < 2 * CH; ++e) dw[j][e] = 0.f;
    }
    const float inv_dim = 1.f / (float)p.dim;
    for (int64_t t0 = (int64_t)blockIdx.x * per_block; t0 < p.tokens; t0 += (int64_t)gridDim.x * per_block) {
        const int64_t t = t0 + (threadIdx.x >> wk.log_lanes);
        const bool there = t < p.tokens;
        const int last = there ? (first + wk.run < h.heads ? first + wk.run : h.heads) : first;
        const T* x = static_cast<const T*>(h.x) + t * h.x_token + first * h.x_head;
        const T* dy = static_cast<const T*>(h.dy) + t * h.dy_token + first * h.dy_head;
        T* dx = static_cast<T*>(h.y) + t * h.y_token + first * h.y_head;
        Chunk<T, CH> xa[HEADS][NCH], xb[HEADS][NCH], ya[HEADS][NCH], yb[HEADS][NCH];
        auto load = [&](int head) {
#pragma unroll
            for (int i = 0; i < HEADS; ++i)
#pragma unroll
                for (int j = 0; j < NCH; ++j)
                    if (head + i < last && mine[j]) {
                        xa[i][j].load(x + i * h.x_head + at[j].a);
                        xb[i][j].load(x + i * h.x_head + at[j].b);
                        ya[i][j].load(dy + i * h.dy_head + at[j].a);
                        yb[i][j].load(dy + i * h.dy_head + at[j].b);
                    }
        };
        load(first);
        const int64_t pos = there ? position_of(p, (uint32_t)t) : -1;
        float2 turn[NCH][CH];
#pragma unroll
        for (int j = 0; j < NCH; ++j)
#pragma unroll
            for (int i = 0; i < CH; ++i)
                turn[j][i] = pos >= 0 && mine[j] && at[j].turned ? __ldg(p.table + pos * (p.rotated / 2) + at[j].pair + i) : make_float2(1.f, 0.f);
        for (int head = first; head < first + wk.run; head += HEADS) {
            if (head != first) load(head);
#pragma unroll
            for (int i = 0; i < HEADS; ++i) {
                // (padding takes no part: its values are not looked at, NaN among them)
                const bool live = head + i < last && pos >= 0;
                float v[NCH][2 * CH], dz[NCH][2 * CH], square = 0.f, dot = 0.f;
#pragma unroll
                for (int j = 0; j < NCH; ++j)
#pragma unroll
                    for (int e = 0; e < CH; ++e) {
                        const int f = first_of<CH>(NEIGHBOURS, e), g = second_of<CH>(NEIGHBOURS, e);
                        const bool in = live && mine[j];
                        const float a = in ? f < CH ? ya[i][j].get(f < CH ? f : 0) : yb[i][j].get(f < CH ? 0 : f - CH) : 0.f;
                        const float b = in ? g < CH ? ya[i][j].get(g < CH ? g : 0) : yb[i][j].get(g < CH ? 0 : g - CH) : 0.f;
                        v[j][f] = in ? f < CH ? xa[i][j].get(f < CH ? f : 0) : xb[i][j].get(f < CH ? 0 : f - CH) : 0.f;
                        v[j][g] = in ? g < CH ? xa[i][j].get(g < CH ? g : 0) : xb[i][j].get(g < CH ? 0 : g - CH) : 0.f;
                        dz[j][f] = fmaf(a, turn[j][e].x, b * turn[j][e].y);
                        dz[j][g] = fmaf(b, turn[j][e].x, -(a * turn[j][e].y));
                    }
#pragma unroll
                for (int j = 0; j < NCH; ++j)
#pragma unroll
                    for (int e = 0; e < 2 * CH; ++e) {
                        square = fmaf(v[j][e], v[j][e], square);
                        dot = fmaf(w[j][e] * dz[j][e], v[j][e], dot);
                    }
                for (int o = lanes >> 1; o; o >>= 1) {
                    square += __shfl_xor_sync(0xffffffffu, square, o);
                    dot += __shfl_xor_sync(0xffffffffu, dot, o);
                }
                if (!live && head + i >= last) continue;
                const float r = rsqrtf(fmaf(square, inv_dim, p.eps)), back = -(dot * inv_dim) * r * r * r;
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    float u[2 * CH];
#pragma unroll
                    for (int e = 0; e < 2 * CH; ++e) {
                        const float rz = r * dz[j][e];
                        dw[j][e] = fmaf(rz, v[j][e], dw[j][e]);
                        u[e] = fmaf(v[j][e], back, rz * w[j][e]);
                    }
                    if (mine[j]) {
                        Chunk<T, CH>::store(dx + i * h.y_head + at[j].a, u);
                        Chunk<T, CH>::store(dx + i * h.y_head + at[j].b, u + CH);
                    }
                }
            }
            x += HEADS * h.x_head;
            dy += HEADS * h.dy_head;
            dx += HEADS * h.y_head;
        }
    }
    if (h.dw == nullptr) return;                                 // (the same for the whole block)
    float* row = sums + (threadIdx.x >> wk.log_lanes) * p.dim;
#pragma unroll
    for (int j = 0; j < NCH; ++j)
        if (mine[j])
#pragma unroll
            for (int e = 0; e < 2 * CH; ++e) row[e < CH ? at[j].a + e : at[j].b + e - CH] = dw[j][e];
    __syncthreads();
    float* out = wk.partial + ((int64_t)part * HEAD_NORM_BLOCKS + (int64_t)run * gridDim.x + blockIdx.x) * p.dim;
    for (int c = threadIdx.x; c < p.dim; c += THREADS) {
        float v = 0.f;
        for (int g = 0; g < per_block; ++g) v += sums[g * p.dim + c];
        out[c] = v;
    }
}

// dw (+)= the blocks' shares, in their order: a block per 32 columns of a part, a warp per run of blocks.
constexpr int FOLD_WARPS = 32;
__global__ void __launch_bounds__(32 * FOLD_WARPS) head_norm_fold_kernel(const HeadNormArgs p, const Work wk, int columns) {
    __shared__ float sums[FOLD_WARPS][32];
    grid_dependency_wait();
    const int part = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * 32 + lane;
    void* dw = p.part[part].dw;
    if (dw == nullptr) return;
    const int n = columns * wk.runs[part], b0 = (int)((int64_t)n * warp / FOLD_WARPS), b1 = (int)((int64_t)n * (warp + 1) / FOLD_WARPS);
    float v = 0.f;
    if (c < p.dim) {
        const float* from = wk.partial + (int64_t)part * HEAD_NORM_BLOCKS * p.dim + c;
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

template <typename T, int CH, int NCH, int HEADS, bool NEIGHBOURS>
cudaError_t launch_form(const HeadNormArgs& p, bool grad, float* partial, int num_sms, cudaStream_t s, uint64_t* launches) {
    Work wk = {};
    wk.chunks = (p.dim / 2 + CH - 1) / CH;
    while (((int64_t)NCH << wk.log_lanes) < wk.chunks) ++wk.log_lanes;
    const int per_block = THREADS >> wk.log_lanes;
    const int64_t columns = (p.tokens + per_block - 1) / per_block;
    wk.w_vec = 1;
    for (int i = 0; i < p.count; ++i) wk.w_vec = wk.w_vec && reinterpret_cast<uintptr_t>(p.part[i].w) % (p.w_type == CERAR_TYPE_F32 ? (CH < 4 ? CH * 4 : 16) : CH * 2) == 0;
    // Eight heads a run share a token's weights and rotation; as few as are loaded together where there are not enough runs for two blocks per SM.
    // (Runs are also counted by blockIdx.y, and in the gradient by the blocks whose shares of dw are kept.)
    auto count = [&](int run) {
        wk.run = run;
        for (int i = 0; i < 2; ++i) wk.runs[i] = i < p.count ? (p.part[i].heads + run - 1) / run : 0;
        return wk.runs[0] + wk.runs[1];
    };
    constexpr int ROWS_MAX = 65535;
    int rows = count(HEADS);
    if (columns * rows >= 2 * num_sms || rows > 256) rows = count(8);
    while (rows > (grad ? 256 : ROWS_MAX)) rows = count(2 * wk.run);
    wk.partial = partial;
    int64_t grid = columns;
    if (grad) {
        const int64_t most = (int64_t)num_sms * 6 / (rows > 0 ? rows : 1), kept = HEAD_NORM_BLOCKS / (wk.runs[0] > wk.runs[1] ? wk.runs[0] : wk.runs[1] > 0 ? wk.runs[1] : 1);
        if (grid > most) grid = most < 1 ? 1 : most;
        if (grid > kept) grid = kept;
    }
    cudaError_t e = cudaSuccess;
    if (grid > 0 && rows > 0) {
        const dim3 blocks((unsigned)grid, (unsigned)rows);
        e = grad ? launch_pdl(head_norm_grad_kernel<T, CH, NCH, HEADS, NEIGHBOURS>, blocks, dim3(THREADS), (size_t)per_block * p.dim * 4, s, p, wk)
                 : launch_pdl(head_norm_kernel<T, CH, NCH, HEADS, NEIGHBOURS>, blocks, dim3(THREADS), 0, s, p, wk);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    if (grad && (p.part[0].dw || (p.count > 1 && p.part[1].dw))) {
        e = launch_pdl(head_norm_fold_kernel, dim3((unsigned)((p.dim + 31) / 32), (unsigned)p.count), dim3(32 * FOLD_WARPS), 0, s, p, wk, (int)grid);
        if (e == cudaSuccess) ++*launches;
    }
    return e;
}

template <typename T, int CH, int NCH, int HEADS>
cudaError_t launch_pairs(const HeadNormArgs& p, bool grad, float* partial, int num_sms, cudaStream_t s, uint64_t* launches) {
    return p.neighbours ? launch_form<T, CH, NCH, HEADS, true>(p, grad, partial, num_sms, s, launches)
                        : launch_form<T, CH, NCH, HEADS, false>(p, grad, partial, num_sms, s, launches);
}

// Chunks of 16 bytes go with one or two per thread (half a row is at most 256 values); shorter ones with more, so that a row still fits a warp.
cudaError_t launch(const HeadNormArgs& p, bool grad, float* partial, int num_sms, cudaStream_t s, uint64_t* launches) {
    if (p.type == CERAR_TYPE_F32) {
        switch (chunk_of(p, 4, grad)) {
            case 4: return launch_pairs<float, 4, 2, 2>(p, grad, partial, num_sms, s, launches);
            case 2: return launch_pairs<float, 2, 4, 1>(p, grad, partial, num_sms, s, launches);
            default: return launch_pairs<float, 1, 8, 1>(p, grad, partial, num_sms, s, launches);
        }
    }
    switch (chunk_of(p, 2, grad)) {
        case 8: return grad ? launch_pairs<__nv_bfloat16, 8, 1, 2>(p, grad, partial, num_sms, s, launches) : launch_pairs<__nv_bfloat16, 8, 1, 4>(p, grad, partial, num_sms, s, launches);
        case 4: return launch_pairs<__nv_bfloat16, 4, 2, 2>(p, grad, partial, num_sms, s, launches);
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
