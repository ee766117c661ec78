// Embedding lookup with scaling, and its gradient by sorted tokens (cerar_embed, cerar_embed_grad).
//
//   y[t] = s table[ids[t]]                            memory bound: every row read and written once
//   dtable[v] (+)= s sum_{t: ids[t] = v} dy[t]        the same, and each row of dtable written (read and written) once
//
// The gradient has to add rows whose number is known only from the ids, and it adds them in the order of the tokens whatever
// the GPU does when: the ids are sorted (stably), the sorted list is cut into pieces of equal length, and a block adds up the rows of
// one piece and some columns, token after token, in registers.  Sums of tokens that lie in one piece go straight to dtable;
// those that run over a piece's end leave a binary32 partial row, which the next kernel adds in the order of the pieces.  A token that
// makes up half of a batch so costs no more than others do, and nothing depends on the order of atomics.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "kernels.cuh"
#include "ops.cuh"
#include "ptx.cuh"

namespace cerar {
namespace {

using namespace ptx;

// A token's key: its id; `vocab` for those that take no part (negative: padding; beyond the table: also reported).
__device__ __forceinline__ int64_t id_of(const void* ids, int id_bytes, int64_t t) {
    return id_bytes == 8 ? __ldg(static_cast<const long long*>(ids) + t) : (int64_t)__ldg(static_cast<const int*>(ids) + t);
}
__device__ __forceinline__ uint32_t key_of(int64_t id, int64_t vocab, int* status) {
    if (id >= vocab) atomicCAS(status, 0, STATUS_BEYOND);
    return id < 0 || id >= vocab ? (uint32_t)vocab : (uint32_t)id;
}
__device__ __forceinline__ uint32_t key_of(const void* ids, int id_bytes, int64_t t, int64_t vocab, int* status) { return key_of(id_of(ids, id_bytes, t), vocab, status); }

// CH consecutive elements as binary32
template <typename T, int CH> struct Chunk;
template <int CH> struct Chunk<float, CH> {
    static __device__ __forceinline__ void load(const float* p, float* v) {
        if constexpr (CH == 4) { const float4 q = __ldg(reinterpret_cast<const float4*>(p)); v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w; }
        else v[0] = __ldg(p);
    }
};
template <int CH> struct Chunk<__nv_bfloat16, CH> {
    static __device__ __forceinline__ void two(uint32_t q, float* v) { v[0] = __uint_as_float(q << 16); v[1] = __uint_as_float(q & 0xFFFF0000u); }
    static __device__ __forceinline__ void load(const __nv_bfloat16* p, float* v) {
        if constexpr (CH == 8) {
            const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
            two(q.x, v); two(q.y, v + 2); two(q.z, v + 4); two(q.w, v + 6);
        } else if constexpr (CH == 2) {
            two(__ldg(reinterpret_cast<const uint32_t*>(p)), v);
        } else {
            v[0] = __uint_as_float((uint32_t)__ldg(reinterpret_cast<const unsigned short*>(p)) << 16);
        }
    }
};
__device__ __forceinline__ uint32_t bf16_two(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// CH values to T, one rounding; whole chunks are aligned
template <int CH>
__device__ __forceinline__ void store(float* p, const float* v) {
    if constexpr (CH % 4 == 0) {
#pragma unroll
        for (int i = 0; i < CH; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < CH; ++i) p[i] = v[i];
    }
}
template <int CH>
__device__ __forceinline__ void store(__nv_bfloat16* p, const float* v) {
    if constexpr (CH == 8) *reinterpret_cast<uint4*>(p) = make_uint4(bf16_two(v[0], v[1]), bf16_two(v[2], v[3]), bf16_two(v[4], v[5]), bf16_two(v[6], v[7]));
    else if constexpr (CH == 4) *reinterpret_cast<uint2*>(p) = make_uint2(bf16_two(v[0], v[1]), bf16_two(v[2], v[3]));
    else if constexpr (CH == 2) *reinterpret_cast<uint32_t*>(p) = bf16_two(v[0], v[1]);
    else p[0] = __float2bfloat16_rn(v[0]);
}

// ------------------------------------------------------------------------------------------------ lookup

constexpr int LOOKUP_THREADS = 256, LOOKUP_CHUNKS = 4;

// 2^log_lanes threads per row (a power of two that a row's chunks fill, at most a warp), four chunks each; wider rows take several turns.
template <typename T, typename Y, int CH>
__global__ void __launch_bounds__(LOOKUP_THREADS) embed_kernel(const EmbedArgs a, int log_lanes, int turns) {
    grid_dependency_wait();
    const int lanes = 1 << log_lanes, lane = threadIdx.x & (lanes - 1);
    const int64_t groups = (int64_t)gridDim.x * (LOOKUP_THREADS >> log_lanes), units = a.tokens * turns;
    const int chunks = (int)((a.width + CH - 1) / CH);
    for (int64_t u = (int64_t)blockIdx.x * (LOOKUP_THREADS >> log_lanes) + (threadIdx.x >> log_lanes); u < units; u += groups) {
        const int64_t t = turns == 1 ? u : u / turns;
        const int c0 = (int)(u - t * turns) * (lanes * LOOKUP_CHUNKS) + lane;
        const uint32_t key = key_of(a.ids, a.id_bytes, t, a.vocab, a.status);
        const bool there = key < (uint32_t)a.vocab;
        const T* src = static_cast<const T*>(a.table) + (int64_t)key * a.ld;
        Y* dst = static_cast<Y*>(a.y) + t * a.ldy;
        float v[LOOKUP_CHUNKS][CH];
#pragma unroll
        for (int i = 0; i < LOOKUP_CHUNKS; ++i) {
            const int c = c0 + i * lanes;
#pragma unroll
            for (int e = 0; e < CH; ++e) v[i][e] = 0.f;
            if (there && c < chunks) Chunk<T, CH>::load(src + (int64_t)c * CH, v[i]);
        }
#pragma unroll
        for (int i = 0; i < LOOKUP_CHUNKS; ++i) {
            const int c = c0 + i * lanes;
#pragma unroll
            for (int e = 0; e < CH; ++e) v[i][e] = there ? v[i][e] * a.scale : 0.f;
            if (c < chunks) store<CH>(dst + (int64_t)c * CH, v[i]);
        }
    }
}

// Rows on other boundaries (an odd width in bfloat16): 16 bytes are written at a time from the first boundary inside a row of y on, and read as the
// one or two aligned pieces that they lie in (each holds an element of the row), shifted to their place.  65536 x 1999 of bfloat16 184 us element by
// element.
constexpr int SHIFTED_CHUNKS = 2;
__device__ __forceinline__ uint4 load_shifted(const unsigned char* p) {
    const uint32_t s = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u);
    const uint4* q = reinterpret_cast<const uint4*>(p - s);
    const uint4 a = __ldg(q), b = s ? __ldg(q + 1) : a;
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (s & 4u)
#pragma unroll
        for (int i = 0; i < 7; ++i) w[i] = w[i + 1];
    if (s & 8u)
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    if (s & 2u)
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__global__ void __launch_bounds__(LOOKUP_THREADS) embed_shifted_kernel(const EmbedArgs a, int log_lanes, int turns) {
    constexpr int CH = 16 / sizeof(T);
    grid_dependency_wait();
    const int lanes = 1 << log_lanes, lane = threadIdx.x & (lanes - 1);
    const int64_t groups = (int64_t)gridDim.x * (LOOKUP_THREADS >> log_lanes), units = a.tokens * turns;
    for (int64_t u = (int64_t)blockIdx.x * (LOOKUP_THREADS >> log_lanes) + (threadIdx.x >> log_lanes); u < units; u += groups) {
        const int64_t t = turns == 1 ? u : u / turns;
        const int turn = (int)(u - t * turns);
        const uint32_t key = key_of(a.ids, a.id_bytes, t, a.vocab, a.status);
        const bool there = key < (uint32_t)a.vocab;
        const T* src = static_cast<const T*>(a.table) + (int64_t)key * a.ld;
        T* dst = static_cast<T*>(a.y) + t * a.ldy;
        const int gap = (int)((16u - (uint32_t)(reinterpret_cast<uintptr_t>(dst) & 15u)) & 15u) / (int)sizeof(T);
        const int first = gap < a.width ? gap : (int)a.width, whole = ((int)a.width - first) / CH, end = first + whole * CH;
        auto element = [&](int e) {
            float v;
            if (there) Chunk<T, 1>::load(src + e, &v);
            v = there ? v * a.scale : 0.f;
            store<1>(dst + e, &v);
        };
        if (turn == 0) {                         // the ends
            for (int e = lane; e < first; e += lanes) element(e);
            for (int e = end + lane; e < a.width; e += lanes) element(e);
        }
        uint4 q[SHIFTED_CHUNKS];
#pragma unroll
        for (int i = 0; i < SHIFTED_CHUNKS; ++i) {
            const int c = (turn * SHIFTED_CHUNKS + i) * lanes + lane;
            if (there && c < whole) q[i] = load_shifted(reinterpret_cast<const unsigned char*>(src + first + c * CH));
        }
#pragma unroll
        for (int i = 0; i < SHIFTED_CHUNKS; ++i) {
            const int c = (turn * SHIFTED_CHUNKS + i) * lanes + lane;
            if (c >= whole) continue;
            float v[CH];
            if constexpr (sizeof(T) == 2) {
                Chunk<T, 2>::two(q[i].x, v); Chunk<T, 2>::two(q[i].y, v + 2); Chunk<T, 2>::two(q[i].z, v + 4); Chunk<T, 2>::two(q[i].w, v + 6);
            } else {
                v[0] = __uint_as_float(q[i].x); v[1] = __uint_as_float(q[i].y); v[2] = __uint_as_float(q[i].z); v[3] = __uint_as_float(q[i].w);
            }
#pragma unroll
            for (int e = 0; e < CH; ++e) v[e] = there ? v[e] * a.scale : 0.f;
            store<CH>(dst + first + c * CH, v);
        }
    }
}

template <typename T, typename Y, int CH>
cudaError_t launch_lookup(const EmbedArgs& a, int num_sms, cudaStream_t s) {
    const int64_t chunks = (a.width + CH - 1) / CH;
    int log_lanes = 0;
    while (log_lanes < 5 && ((int64_t)LOOKUP_CHUNKS << log_lanes) < chunks) ++log_lanes;
    const int64_t turns = (chunks + (LOOKUP_CHUNKS << log_lanes) - 1) / (LOOKUP_CHUNKS << log_lanes), per_block = LOOKUP_THREADS >> log_lanes;
    const int64_t blocks = (a.tokens * turns + per_block - 1) / per_block, most = (int64_t)num_sms * 64;
    return launch_pdl(embed_kernel<T, Y, CH>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(LOOKUP_THREADS), 0, s, a, log_lanes, (int)turns);
}
template <typename T, typename Y>
cudaError_t launch_lookup_typed(const EmbedArgs& a, int num_sms, cudaStream_t s) {
    constexpr int WIDE = 16 / sizeof(T);
    auto fits = [&](int ch) {                // whole chunks in a row, all of them aligned on both sides (16 bytes are as much as one access takes)
        const uintptr_t in = ch * sizeof(T), out = ch * sizeof(Y) < 16 ? ch * sizeof(Y) : 16;
        return a.width % ch == 0 && reinterpret_cast<uintptr_t>(a.table) % in == 0 && a.ld * sizeof(T) % in == 0 &&
               reinterpret_cast<uintptr_t>(a.y) % out == 0 && a.ldy * sizeof(Y) % out == 0;
    };
    if (fits(WIDE)) return launch_lookup<T, Y, WIDE>(a, num_sms, s);
    if constexpr (std::is_same<T, Y>::value) {
        if (a.width >= 4 * WIDE) {               // (shorter rows are mostly ends)
            const int64_t chunks = a.width / WIDE;
            int log_lanes = 0;
            while (log_lanes < 5 && ((int64_t)SHIFTED_CHUNKS << log_lanes) < chunks) ++log_lanes;
            const int64_t turns = (chunks + (SHIFTED_CHUNKS << log_lanes) - 1) / (SHIFTED_CHUNKS << log_lanes), per_block = LOOKUP_THREADS >> log_lanes;
            const int64_t blocks = (a.tokens * turns + per_block - 1) / per_block, most = (int64_t)num_sms * 64;
            return launch_pdl(embed_shifted_kernel<T>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(LOOKUP_THREADS), 0, s, a, log_lanes, (int)turns);
        }
    }
    if constexpr (sizeof(T) == 2) if (fits(2)) return launch_lookup<T, Y, 2>(a, num_sms, s);
    return launch_lookup<T, Y, 1>(a, num_sms, s);
}

// ------------------------------------------------------------------------------------------------ sorting
//
// Short lists: a token's place is the number of keys in front of it, counted; eight threads share a token's count.  T^2 comparisons are
// one launch where a radix sort would be four.

constexpr int RANK_THREADS = 256, RANK_SHARE = 8, RANK_MAX = 8192;

__global__ void __launch_bounds__(RANK_THREADS) rank_kernel(const void* ids, int id_bytes, int tokens, int64_t vocab, uint32_t* keys, uint32_t* order, uint32_t* crossing, int* status) {
    __shared__ __align__(16) uint32_t all[RANK_MAX];
    grid_dependency_wait();
    if (blockIdx.x == 0 && threadIdx.x < 2) crossing[threadIdx.x] = 0u;
    const int groups = (tokens + 3) >> 2;
    for (int t0 = threadIdx.x; t0 < 4 * groups; t0 += 8 * RANK_THREADS) {
        int64_t id[8];                         // (their loads together)
#pragma unroll
        for (int i = 0; i < 8; ++i) id[i] = t0 + i * RANK_THREADS < tokens ? id_of(ids, id_bytes, t0 + i * RANK_THREADS) : -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int t = t0 + i * RANK_THREADS;
            if (t < 4 * groups) all[t] = t < tokens ? key_of(id[i], vocab, status) : 0xFFFFFFFFu;
        }
    }
    __syncthreads();
    const int t = blockIdx.x * (RANK_THREADS / RANK_SHARE) + threadIdx.x / RANK_SHARE, share = threadIdx.x % RANK_SHARE;
    const bool mine = t < tokens;
    const uint32_t key = mine ? all[t] : 0u;
    int before = 0;
    const int own = t >> 2;                    // equal keys come before this one in the groups in front of its own ...
#pragma unroll 4
    for (int g = share; g < groups; g += RANK_SHARE) {
        const uint4 q = reinterpret_cast<const uint4*>(all)[g];
        const uint32_t limit = key + (g < own ? 1u : 0u);
        before += (q.x < limit) + (q.y < limit) + (q.z < limit) + (q.w < limit);
    }
    if (mine && own % RANK_SHARE == share)     // ... and, in that one, in front of itself
        for (int j = own * 4; j < t; ++j) before += all[j] == key;
#pragma unroll
    for (int o = RANK_SHARE / 2; o; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
    if (mine && share == 0) {
        keys[before] = key;
        order[before] = (uint32_t)t;
    }
}

// Long lists: least significant digit first, digits of up to 9 bits.  One launch counts the first digit in every tile; one for each digit brings
// every tile's tokens to their places and counts the next digit where they go.  A warp owns a run of its tile; equal digits among its 32
// tokens are ranked by their lanes, so every pass keeps the order.
constexpr int DIGIT_MAX = 9, PASSES_MAX = 4 /* 32 bits */, DIGITS = 1 << DIGIT_MAX, SORT_THREADS = 512, SORT_WARPS = SORT_THREADS / 32;
constexpr int SORT_TILE = 2048, SORT_TILES_MAX = 256, KEYS = SORT_TILE / SORT_THREADS;
constexpr uint32_t NONE = 0xFFFFFFFFu;

struct SortPass {
    const void* ids;                           // first pass: the keys are made from these
    int id_bytes;
    int64_t vocab;
    const uint32_t *keys_in, *order_in;
    uint32_t *keys, *order, *counts;           // counts: [tiles][DIGITS], of this digit
    uint32_t* next_counts;                     // of the next one (null: there is none): cleared by the first kernel, counted while placing
    int passes;
    uint32_t *named, *crossing;                // a bit for every row that some token names (cleared by the first count, set by the first placing)
    int64_t tokens;
    int tile, tiles, shift, next_shift, digits; // digits: a power of two
    int* status;
};
__device__ __forceinline__ uint32_t sort_key(const SortPass& p, int64_t t) {
    return p.ids ? key_of(p.ids, p.id_bytes, t, p.vocab, p.status) : p.keys_in[t];
}

__global__ void __launch_bounds__(SORT_THREADS) count_kernel(const SortPass p) {
    __shared__ uint32_t count[DIGITS];
    count[threadIdx.x] = 0;
    grid_dependency_wait();
    __syncthreads();
    {
        if (blockIdx.x == 0 && threadIdx.x < 2) p.crossing[threadIdx.x] = 0u;
        for (int i = 1; i < p.passes; ++i) p.counts[((int64_t)i * p.tiles + blockIdx.x) * DIGITS + threadIdx.x] = 0u;
        if (p.named)
            for (int64_t w = (int64_t)blockIdx.x * SORT_THREADS + threadIdx.x; w <= p.vocab / 32; w += (int64_t)gridDim.x * SORT_THREADS) p.named[w] = 0u;
    }
    const int64_t t0 = (int64_t)blockIdx.x * p.tile, t1 = t0 + p.tile < p.tokens ? t0 + p.tile : p.tokens;
#pragma unroll 4
    for (int64_t t = t0 + threadIdx.x; t < t1; t += SORT_THREADS) atomicAdd(&count[(sort_key(p, t) >> p.shift) & (p.digits - 1)], 1u);
    __syncthreads();
    p.counts[(int64_t)blockIdx.x * DIGITS + threadIdx.x] = count[threadIdx.x];
}

__global__ void __launch_bounds__(SORT_THREADS) place_kernel(const SortPass p) {
    __shared__ uint32_t at[SORT_WARPS][DIGITS];
    __shared__ uint32_t scan[SORT_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int w = 0; w < SORT_WARPS; ++w) at[w][threadIdx.x] = 0;
    grid_dependency_wait();
    __syncthreads();
    const int64_t t0 = (int64_t)blockIdx.x * p.tile + (int64_t)warp * (p.tile / SORT_WARPS), t1 = t0 + p.tile / SORT_WARPS;
    const uint32_t dmask = p.digits - 1;
    // A run of a tile of the usual size is four keys per lane, which stay in registers (and their loads on their way together).
    uint32_t held[KEYS], number[KEYS];
    auto load = [&](int64_t from) {
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const int64_t t = from + i * 32 + lane;
            const bool there = t < t1 && t < p.tokens;
            held[i] = there ? sort_key(p, t) : NONE;
            number[i] = !p.ids && there ? p.order_in[t] : (uint32_t)t;
        }
    };
    if (t1 - t0 <= 32 * KEYS) load(t0);
    // This digit's (thread's) tokens, and those of the tiles in front.
    uint32_t total = 0, front = 0;
#pragma unroll 16
    for (int i = 0; i < p.tiles; ++i) {
        const uint32_t c = p.counts[(int64_t)i * DIGITS + threadIdx.x];
        total += c;
        if (i < (int)blockIdx.x) front += c;
    }
    for (int64_t from = t0; from < t1 && from < p.tokens; from += 32 * KEYS) {
        if (t1 - t0 > 32 * KEYS) load(from);
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const bool there = held[i] != NONE;
            const uint32_t d = there ? (held[i] >> p.shift) & dmask : NONE;
            const uint32_t same = __match_any_sync(0xffffffffu, d);
            if (there && lane == __ffs(same) - 1) at[warp][d] += __popc(same);
            if (there && p.ids && p.named) atomicOr(p.named + (held[i] >> 5), 1u << (held[i] & 31));
            __syncwarp();
        }
    }
    // The first place: the smaller digits' tokens, the same digit's of the tiles in front.
    uint32_t incl = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    uint32_t place = incl - total + front;
    for (int w = 0; w < warp; ++w) place += scan[w];
    for (int w = 0; w < SORT_WARPS; ++w) {
        const uint32_t c = at[w][threadIdx.x];
        at[w][threadIdx.x] = place;
        place += c;
    }
    __syncthreads();
    for (int64_t from = t0; from < t1 && from < p.tokens; from += 32 * KEYS) {
        if (t1 - t0 > 32 * KEYS) load(from);
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const bool there = held[i] != NONE;
            const uint32_t d = there ? (held[i] >> p.shift) & dmask : NONE;
            const uint32_t same = __match_any_sync(0xffffffffu, d);
            uint32_t to = 0;
            if (there) to = at[warp][d] + __popc(same & ((1u << lane) - 1u));
            __syncwarp();
            if (there) {
                if (lane == __ffs(same) - 1) at[warp][d] += __popc(same);
                p.keys[to] = held[i];
                p.order[to] = number[i];
                if (p.next_counts) atomicAdd(p.next_counts + (int64_t)(to / (uint32_t)p.tile) * DIGITS + ((held[i] >> p.next_shift) & dmask), 1u);
            }
            __syncwarp();
        }
    }
}

// ------------------------------------------------------------------------------------------------ sums

constexpr int SHORT_ROWS = 16;
constexpr int SUM_THREADS = 128, PIECE_MAX = 64, ZERO_ROWS = 32;

// Tokens of a piece.  Short batches need the blocks, long ones the few partial rows.
__host__ int piece_of(int64_t tokens) { return tokens <= 2048 ? 4 : tokens <= 8192 ? 8 : tokens <= 32768 ? 16 : tokens <= 131072 ? 32 : PIECE_MAX; }

struct SumArgs {
    const void* dy;
    int64_t lddy;
    const uint32_t *keys, *order;              // sorted
    const uint32_t* named;                     // a bit for every row that some token names; null: it is looked for in the sorted keys
    uint32_t* crossing;                        // numbers of, and then, the pieces whose last token has up to SHORT_ROWS partial rows; more
    float* partial;                            // [pieces][2][ldp]: of the token that came over the piece's start, of the one that goes over its end
    int64_t ldp;
    int64_t tokens, vocab, width, ld;
    void* dtable;
    float scale;
    int d_type, accumulate;
    int piece, slabs;
    int64_t pieces;
};

template <int CH>
__device__ __forceinline__ void write_row(const SumArgs& a, uint32_t row, int64_t col, const float* acc, bool aligned) {
    const int64_t at = (int64_t)row * a.ld + col;
    float v[CH];
    if (a.d_type == CERAR_TYPE_F32) {
        float* p = static_cast<float*>(a.dtable) + at;
#pragma unroll
        for (int e = 0; e < CH; ++e) v[e] = a.accumulate ? fmaf(a.scale, acc[e], p[e]) : a.scale * acc[e];
        if (aligned) store<CH>(p, v);
        else
#pragma unroll
            for (int e = 0; e < CH; ++e) p[e] = v[e];
    } else {
        __nv_bfloat16* p = static_cast<__nv_bfloat16*>(a.dtable) + at;
#pragma unroll
        for (int e = 0; e < CH; ++e) v[e] = a.accumulate ? fmaf(a.scale, acc[e], __bfloat162float(p[e])) : a.scale * acc[e];
        if (aligned) store<CH>(p, v);
        else
#pragma unroll
            for (int e = 0; e < CH; ++e) p[e] = __float2bfloat16_rn(v[e]);
    }
}

// A chunk of a row as it lies in memory.  The loads are volatile: they are to be issued together, not each where it is used (which is what
// becomes of them behind the branches of the sums: 65536 x 2048 in 269 us).
template <int BYTES> struct Bits;
template <> struct Bits<16> {
    uint4 q;
    __device__ __forceinline__ void load(const void* p) { asm volatile("ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p)); }
    __device__ __forceinline__ void values(const float*, float* v) const {
        v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
    }
    __device__ __forceinline__ void values(const __nv_bfloat16*, float* v) const {
        Chunk<__nv_bfloat16, 2>::two(q.x, v); Chunk<__nv_bfloat16, 2>::two(q.y, v + 2); Chunk<__nv_bfloat16, 2>::two(q.z, v + 4); Chunk<__nv_bfloat16, 2>::two(q.w, v + 6);
    }
};
template <> struct Bits<4> {
    uint32_t q;
    __device__ __forceinline__ void load(const void* p) { asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(q) : "l"(p)); }
    __device__ __forceinline__ void values(const float*, float* v) const { v[0] = __uint_as_float(q); }
    __device__ __forceinline__ void values(const __nv_bfloat16*, float* v) const { Chunk<__nv_bfloat16, 2>::two(q, v); }
};
template <> struct Bits<2> {
    uint16_t q;
    __device__ __forceinline__ void load(const void* p) { asm volatile("ld.global.nc.u16 %0, [%1];" : "=h"(q) : "l"(p)); }
    __device__ __forceinline__ void values(const __nv_bfloat16*, float* v) const { v[0] = __uint_as_float((uint32_t)q << 16); }
};

// pieces * slabs blocks add up pieces; the others (nothing is kept of what dtable held) set the rows of no token to zero, 32 rows each.  They take
// turns, so that reads of the ones and writes of the others go on at the same time.
template <typename T, int CH>
__global__ void __launch_bounds__(SUM_THREADS) sum_kernel(const SumArgs a) {
    __shared__ uint32_t key[PIECE_MAX + 2], row[PIECE_MAX];
    grid_dependency_wait();
    const uint64_t sums = (uint64_t)a.pieces * a.slabs;
    const uint64_t before = sums * blockIdx.x / gridDim.x;                // blocks in front of this one that add up
    if (sums * (blockIdx.x + 1ull) / gridDim.x == before) {
        const int64_t r0 = (int64_t)(blockIdx.x - before) * ZERO_ROWS;
        if (threadIdx.x < ZERO_ROWS) {
            const int64_t r = r0 + threadIdx.x;
            bool skip = r >= a.vocab;
            if (!skip && a.named) {
                skip = a.named[r >> 5] >> (r & 31) & 1u;
            } else if (!skip) {
                int64_t lo = 0, hi = a.tokens;   // the first sorted key that is not below r
                while (lo < hi) {
                    const int64_t mid = (lo + hi) >> 1;
                    if (a.keys[mid] < (uint32_t)r) lo = mid + 1; else hi = mid;
                }
                skip = lo < a.tokens && a.keys[lo] == (uint32_t)r;
            }
            key[threadIdx.x] = skip ? 1u : 0u;
        }
        __syncthreads();
        const int64_t size = a.d_type == CERAR_TYPE_F32 ? 4 : 2;
        for (int i = 0; i < ZERO_ROWS; ++i) {
            if (key[i]) continue;
            // 16 bytes at a time from the first boundary inside the row on
            unsigned char* p = static_cast<unsigned char*>(a.dtable) + (r0 + i) * a.ld * size;
            const int64_t bytes = a.width * size, gap = (int64_t)(-reinterpret_cast<uintptr_t>(p) & 15u), first = gap < bytes ? gap : bytes;
            const int64_t end = first + ((bytes - first) & ~15ll);
            for (int64_t b = first + threadIdx.x * 16; b < end; b += SUM_THREADS * 16) *reinterpret_cast<uint4*>(p + b) = make_uint4(0, 0, 0, 0);
            const int64_t head = 2 * threadIdx.x, tail = end + 2 * threadIdx.x;
            if (head < first) *reinterpret_cast<unsigned short*>(p + head) = 0;
            if (tail < bytes) *reinterpret_cast<unsigned short*>(p + tail) = 0;
        }
        return;
    }
    const int64_t piece = (int64_t)before / a.slabs, e0 = piece * a.piece;
    const int slab = (int)((int64_t)before - piece * a.slabs);
    const int n = (int)(a.tokens - e0 < a.piece ? a.tokens - e0 : a.piece);
    for (int i = threadIdx.x; i < n + 2; i += SUM_THREADS) {
        const int64_t e = e0 + i - 1;
        key[i] = e >= 0 && e < a.tokens ? a.keys[e] : NONE;
        if (i < n) row[i] = a.order[e0 + i];
    }
    __syncthreads();
    const int64_t col = ((int64_t)slab * SUM_THREADS + threadIdx.x) * CH;
    if (col >= a.width) return;
    const T* dy = static_cast<const T*>(a.dy) + col;
    constexpr int AHEAD = 8;                     // rows whose loads are on their way together
    float acc[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) acc[e] = 0.f;
    bool came = key[0] == key[1];                // the sum of this token began in an earlier piece
    for (int i0 = 0; i0 < n; i0 += AHEAD) {
        Bits<CH * sizeof(T)> raw[AHEAD];         // (behind the end: the last row again; of padding: not used)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) raw[i].load(dy + (int64_t)row[i0 + i < n ? i0 + i : n - 1] * a.lddy);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (i0 + i >= n) break;
            const uint32_t k = key[i0 + i + 1], next = key[i0 + i + 2];
            if (k >= (uint32_t)a.vocab) return;  // (the rest takes no part)
            float v[CH];
            raw[i].values(static_cast<const T*>(nullptr), v);
#pragma unroll
            for (int e = 0; e < CH; ++e) acc[e] += v[e];
            if (next == k && i0 + i + 1 < n) continue;
            if (next != k && !came) {
                write_row<CH>(a, k, col, acc, true);
            } else {
                if (!came && col == 0) {         // its sum begins here and goes on: the next kernel puts it together
                    const int64_t after = e0 + (int64_t)SHORT_ROWS * a.piece;
                    const int far = after < a.tokens && a.keys[after] == k;
                    a.crossing[2 + far * a.pieces + atomicAdd(a.crossing + far, 1u)] = (uint32_t)piece;
                }
                float* p = a.partial + (piece * 2 + (came ? 0 : 1)) * a.ldp + col;
#pragma unroll
                for (int e = 0; e < CH; ++e) p[e] = acc[e];
            }
            came = false;
#pragma unroll
            for (int e = 0; e < CH; ++e) acc[e] = 0.f;
        }
    }
}

// Tokens that go over the end of a piece p in which their sum began: partial rows p (second), p + 1 ... (first), in this order.  Up to sixteen rows:
// a warp adds 128 columns.  More: sixteen warps take a run of the rows of 128 columns each, and their sums are added in the order of the
// runs.  (The order of the lists is that of atomics; what is added, and in which order, does not depend on it.)
constexpr int JOIN_WARPS = 16;
__device__ __forceinline__ void write_four(const SumArgs& a, uint32_t k, int64_t col, const float4& v, bool aligned) {
    const float acc[4] = {v.x, v.y, v.z, v.w};
    if (col + 4 <= a.width) {
        write_row<4>(a, k, col, acc, aligned);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < a.width) write_row<1>(a, k, col + e, acc + e, true);
    }
}
__device__ __forceinline__ void add(float4& v, const float4& x) { v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w; }
__global__ void __launch_bounds__(32 * JOIN_WARPS) join_kernel(const SumArgs a, int slabs, int aligned) {
    __shared__ float4 sums[JOIN_WARPS][32];
    grid_dependency_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto partial = [&](int64_t p, int which, int64_t col) { return *reinterpret_cast<const float4*>(a.partial + (p * 2 + which) * a.ldp + col); };
    // whether the sum that began in piece p has a row in piece q > p: true up to its last one
    auto goes_on = [&](uint32_t k, int64_t q) { return q * a.piece < a.tokens && a.keys[q * a.piece] == k; };
    const int64_t few = (int64_t)a.crossing[0] * slabs, many = (int64_t)a.crossing[1] * slabs;
    for (int64_t u = blockIdx.x; u < many; u += gridDim.x) {
        const int64_t p = a.crossing[2 + a.pieces + u / slabs], col = (u % slabs * 32 + lane) * 4;
        const uint32_t k = a.keys[p * a.piece + a.piece - 1];
        int64_t rows = 1;
        for (int n = 32 * JOIN_WARPS; n == 32 * JOIN_WARPS; rows += n) n = __syncthreads_count(goes_on(k, p + rows + threadIdx.x));
        const int64_t r0 = rows * warp / JOIN_WARPS, r1 = rows * (warp + 1) / JOIN_WARPS;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (col < a.ldp) {
#pragma unroll 8
            for (int64_t r = r0; r < r1; ++r) add(v, partial(p + r, r == 0 ? 1 : 0, col));
        }
        sums[warp][lane] = v;
        __syncthreads();
        if (warp == 0 && col < a.width) {
#pragma unroll
            for (int w = 1; w < JOIN_WARPS; ++w) add(v, sums[w][lane]);
            write_four(a, k, col, v, aligned != 0);
        }
        __syncthreads();
    }
    for (int64_t u = (int64_t)blockIdx.x * JOIN_WARPS + warp; u < few; u += (int64_t)gridDim.x * JOIN_WARPS) {
        const int64_t p = a.crossing[2 + u / slabs], col = (u % slabs * 32 + lane) * 4;
        const uint32_t k = a.keys[p * a.piece + a.piece - 1];
        const int rows = 1 + __popc(__ballot_sync(0xffffffffu, lane < SHORT_ROWS && goes_on(k, p + 1 + lane)));
        if (col >= a.width) continue;
        float4 v = partial(p, 1, col);
#pragma unroll 4
        for (int r = 1; r < rows; ++r) add(v, partial(p + r, 0, col));
        write_four(a, k, col, v, aligned != 0);
    }
}

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Layout {
    int64_t keys, order, keys2, order2, counts, named, crossing, partial, bytes;
    int64_t ldp, pieces;
    int piece, tile, tiles;
};
Layout layout_of(int64_t tokens, int64_t vocab, int64_t width) {
    Layout l = {};
    l.piece = piece_of(tokens);
    l.pieces = (tokens + l.piece - 1) / l.piece;
    l.ldp = round_up(width, 4);
    const int64_t list = round_up(4 * tokens, 256);
    int64_t at = 0;
    l.keys = at; at += list;
    l.order = at; at += list;
    if (tokens > RANK_MAX) {
        l.tile = (int)round_up((tokens + SORT_TILES_MAX - 1) / SORT_TILES_MAX, SORT_TILE);
        l.tiles = (int)((tokens + l.tile - 1) / l.tile);
        l.keys2 = at; at += list;
        l.order2 = at; at += list;
        l.counts = at; at += (int64_t)l.tiles * DIGITS * 4 * PASSES_MAX;
        l.named = at; at += round_up(vocab / 8 + 8, 256);
    }
    l.crossing = at; at += round_up(4 * (2 + 2 * l.pieces), 256);
    l.partial = at;
    at += l.pieces * 2 * l.ldp * 4;
    l.bytes = at;
    return l;
}

template <typename T, int CH>
cudaError_t launch_sums(SumArgs s, cudaStream_t st) {
    s.slabs = (int)((s.width + SUM_THREADS * CH - 1) / (SUM_THREADS * CH));
    const int64_t blocks = s.pieces * s.slabs + (s.accumulate ? 0 : (s.vocab + ZERO_ROWS - 1) / ZERO_ROWS);
    if (blocks > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    return launch_pdl(sum_kernel<T, CH>, dim3((unsigned)blocks), dim3(SUM_THREADS), 0, st, s);
}

}  // namespace

cudaError_t launch_embed(const EmbedArgs& a, int num_sms, cudaStream_t s, uint64_t* launches) {
    cudaError_t e;
    if (a.type == CERAR_TYPE_F32) e = a.y_type == CERAR_TYPE_F32 ? launch_lookup_typed<float, float>(a, num_sms, s) : launch_lookup_typed<float, __nv_bfloat16>(a, num_sms, s);
    else e = a.y_type == CERAR_TYPE_F32 ? launch_lookup_typed<__nv_bfloat16, float>(a, num_sms, s) : launch_lookup_typed<__nv_bfloat16, __nv_bfloat16>(a, num_sms, s);
    if (e == cudaSuccess) ++*launches;
    return e;
}

size_t embed_grad_workspace(int64_t tokens, int64_t vocab, int64_t width) { return (size_t)layout_of(tokens, vocab, width).bytes; }

cudaError_t launch_embed_grad(const EmbedGradArgs& a, int num_sms, cudaStream_t st, uint64_t* launches) {
    const Layout l = layout_of(a.tokens, a.vocab, a.width);
    unsigned char* ws = static_cast<unsigned char*>(a.workspace);
    uint32_t* keys = reinterpret_cast<uint32_t*>(ws + l.keys);
    uint32_t* order = reinterpret_cast<uint32_t*>(ws + l.order);
    uint32_t* crossing = reinterpret_cast<uint32_t*>(ws + l.crossing);
    uint32_t* named = !a.accumulate && a.tokens > RANK_MAX ? reinterpret_cast<uint32_t*>(ws + l.named) : nullptr;
    cudaError_t e = cudaSuccess;
    if (a.tokens > 0 && a.tokens <= RANK_MAX) {
        constexpr int PER = RANK_THREADS / RANK_SHARE;
        e = launch_pdl(rank_kernel, dim3((unsigned)((a.tokens + PER - 1) / PER)), dim3(RANK_THREADS), 0, st, a.ids, a.id_bytes, (int)a.tokens, a.vocab, keys, order, crossing, a.status);
        if (e != cudaSuccess) return e;
        ++*launches;
    } else if (a.tokens > 0) {
        int bits = 1;
        while (a.vocab >> bits) ++bits;         // of the largest key, vocab
        const int passes = (bits + DIGIT_MAX - 1) / DIGIT_MAX, digit = (bits + passes - 1) / passes;
        uint32_t *k2 = reinterpret_cast<uint32_t*>(ws + l.keys2), *o2 = reinterpret_cast<uint32_t*>(ws + l.order2);
        SortPass p = {};
        p.id_bytes = a.id_bytes; p.vocab = a.vocab; p.tokens = a.tokens; p.tile = l.tile; p.tiles = l.tiles; p.digits = 1 << digit; p.status = a.status;
        p.named = named; p.crossing = crossing;
        p.counts = reinterpret_cast<uint32_t*>(ws + l.counts);
        p.passes = passes; p.ids = a.ids;
        if ((e = launch_pdl(count_kernel, dim3((unsigned)l.tiles), dim3(SORT_THREADS), 0, st, p)) != cudaSuccess) return e;
        ++*launches;
        for (int i = 0; i < passes; ++i) {
            // the last pass ends in keys and order
            const bool to_first = (passes - 1 - i) % 2 == 0;
            p.ids = i == 0 ? a.ids : nullptr;
            p.keys_in = to_first ? k2 : keys; p.order_in = to_first ? o2 : order;
            p.keys = to_first ? keys : k2; p.order = to_first ? order : o2;
            p.shift = i * digit; p.next_shift = p.shift + digit;
            p.next_counts = i + 1 < passes ? p.counts + (int64_t)l.tiles * DIGITS : nullptr;
            if ((e = launch_pdl(place_kernel, dim3((unsigned)l.tiles), dim3(SORT_THREADS), 0, st, p)) != cudaSuccess) return e;
            ++*launches;
            p.counts += (int64_t)l.tiles * DIGITS;
        }
    }
    SumArgs s = {};
    s.dy = a.dy; s.lddy = a.lddy; s.keys = keys; s.order = order; s.partial = reinterpret_cast<float*>(ws + l.partial); s.ldp = l.ldp;
    s.tokens = a.tokens; s.vocab = a.vocab; s.width = a.width; s.ld = a.ld; s.dtable = a.dtable; s.scale = a.scale; s.d_type = a.d_type;
    s.named = named; s.crossing = crossing; s.accumulate = a.accumulate; s.piece = l.piece; s.pieces = l.pieces;
    const int64_t dsize = a.d_type == CERAR_TYPE_F32 ? 4 : 2;
    const uintptr_t dt = reinterpret_cast<uintptr_t>(a.dtable), dy = reinterpret_cast<uintptr_t>(a.dy);
    auto fits = [&](int ch) {
        const int64_t in = ch * (a.type == CERAR_TYPE_F32 ? 4 : 2), out = ch * dsize < 16 ? ch * dsize : 16;
        return a.width % ch == 0 && dy % in == 0 && a.lddy * (in / ch) % in == 0 && dt % out == 0 && a.ld * dsize % out == 0;
    };
    if (a.type == CERAR_TYPE_F32) e = fits(4) ? launch_sums<float, 4>(s, st) : launch_sums<float, 1>(s, st);
    else e = fits(8) ? launch_sums<__nv_bfloat16, 8>(s, st) : fits(2) ? launch_sums<__nv_bfloat16, 2>(s, st) : launch_sums<__nv_bfloat16, 1>(s, st);
    if (e != cudaSuccess) return e;
    ++*launches;
    if (l.pieces > 1) {
        const int slabs = (int)((l.ldp + 127) / 128);
        const int64_t units = (l.pieces - 1) * slabs, most = (int64_t)num_sms * 4, four = 4 * dsize;
        e = launch_pdl(join_kernel, dim3((unsigned)(units < most ? units : most)), dim3(32 * JOIN_WARPS), 0, st, s, slabs, (int)(dt % four == 0 && a.ld * dsize % four == 0));
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    return e;
}

}  // namespace cerar
