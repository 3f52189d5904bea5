// Attention of one new token per request over a paged cache (amap_cache_attend): s_i = scale q . k_i over the visible tokens,
// out = sum softmax(s)_i v_i, lse = log sum exp s_i, with the running maximum and sum of a softmax in one pass over the cache.
//
// Bound by the cache's bytes: every visible key and value is read once, and 2 heads / kv_heads flop are done with each byte.  So the
// kernel is built around keeping loads in flight.
//   Work: tiles of 32 tokens for each wavefront of a workgroup.  The tiles of all requests and key heads are one line, cut into equal
//     shares, one for each workgroup of a grid that fills the chip once: long requests are split, short ones follow one
//     another, whatever the mix, and only where a cut falls inside a request are results joined (amap_attend_join_kernel).
//   Loads: keys, values and the table's entries go straight into LDS (global_load_lds), a ring of stages per wavefront, waited for by count.
//     No wavefront waits for another before its share of a request is done.  A token that is not visible is read from 16 bytes of
//     zeros, so nothing that lies in the cache behind a request's end comes near the sums.
//   Products: the scores as K Q^T, 32 tokens by 16 columns (the queries that share a key head), by 16 x 16 x 32 matrix instructions.  The tokens
//     are dealt to the rows of the two tiles so that a lane ends up with 8 consecutive ones: just what the next product,
//     V^T P^T, takes from it, so weights never leave their lane.  V comes transposed out of LDS (ds_read_tr).
//   A weight is kept in two 16-bit parts, itself rounded and what that leaves: one part alone would be off by as much as
//     the result's own rounding is.  With up to 8 queries to a key head the second part costs nothing: it takes the columns that are
//     idle.  (A value that is infinite makes its column NaN, as 0 * inf does in the sum itself where a weight has vanished.)
#include "amap_cache.hpp"

using namespace amap_cache_detail;
using namespace amap_detail;
using namespace amap_dev;

namespace {

constexpr uint32_t kUnits = 256;   // compute units of an MI355X
constexpr int kTokens = 32;        // of a wavefront's step
constexpr int kColumns = 16;       // queries of a workgroup at a time (8 where their weights' second parts have the others)
constexpr uint32_t kNoRow = 0xFFFFFFFFu;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

struct AttendArgs {
    const char *k, *v, *q;
    char *out;
    float *lse, *parts;
    const float *k_scale, *v_scale;
    const int32_t *table, *length;
    int64_t table_stride, q_token, q_head, out_token, out_head;
    uint32_t page_step, token_step, head_step;   // of the cache, in 16-byte pieces
    uint32_t n_pages, page, most;                // most: tokens that a row of the table can name
    uint32_t requests, kv_heads, group, dim, pieces;   // pieces: 16-byte ones of a row
    uint32_t heads, columns, segments;           // segments of a request: kv_heads times the column blocks of one
    FastDiv by_page, by_segments, by_blocks;
    uint32_t blocks, least;                      // column blocks of a key head; tiles of a share, at least
    uint32_t window, aligned;                    // aligned: q in whole 16-byte pieces
    float scale;
};

// What a workgroup leaves for the join: of the segment that begins in its share and goes on in the next ones.
struct Split {
    uint32_t request, segment, count, pad;
};

__device__ const u32x4 kZeros = {0u, 0u, 0u, 0u};

constexpr int trailing_zeros(int x) { return x & 1 ? 0 : 1 + trailing_zeros(x >> 1); }
constexpr int at_most(int x, int y) { return x < y ? x : y; }

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x2 __attribute__((ext_vector_type(2)));

template <class T>
struct Of;   // the 16-bit type that products are made in
template <>
struct Of<Bf16> {
    typedef __bf16 one;
    typedef bf16x8 eight;
    static __device__ __forceinline__ f32x4 product(eight a, eight b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ uint32_t two_of_e4m3(uint32_t x, bool high) {
        return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true))
                    : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false));
    }
};
template <>
struct Of<F16> {
    typedef _Float16 one;
    typedef f16x8 eight;
    static __device__ __forceinline__ f32x4 product(eight a, eight b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ uint32_t two_of_e4m3(uint32_t x, bool high) {
        return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, true))
                    : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, false));
    }
};
template <class T>
__device__ __forceinline__ typename Of<T>::eight eight_of_e4m3(u32x2 x) {   // (exact: either type holds all its values)
    const u32x4 y = {Of<T>::two_of_e4m3(x.x, false), Of<T>::two_of_e4m3(x.x, true), Of<T>::two_of_e4m3(x.y, false), Of<T>::two_of_e4m3(x.y, true)};
    return __builtin_bit_cast(typename Of<T>::eight, y);
}

// DP: head_dim rounded up, what the products are made for; ES: bytes of the cache's elements
template <class T_, int ES_, int DP_, bool PAIRED_>
struct Form {
    typedef T_ T;
    static constexpr int ES = ES_, DP = DP_;
    static constexpr bool PAIRED = PAIRED_;                 // the weights' second parts in columns 8 .. 15
    static constexpr int ROW = DP * ES, NC = ROW / 16;      // bytes and 16-byte pieces of a row in LDS
    static constexpr int WAVES = ROW > 256 ? 2 : 4;
    static constexpr int STAGES = ROW <= 64 ? 4 : ROW <= 96 ? 3 : 2;
    static constexpr int SIDE = kTokens * ROW, STAGE = 2 * SIDE;
    static constexpr int LOADS = NC / 2;                    // of a side, 1 KB each
    static constexpr int IDS = STAGES * 256;                // a word per lane and stage
    static constexpr int PER_WAVE = STAGES * STAGE + IDS;
    static constexpr int OUT_ROW = DP + 4;                  // floats; the 4 spread a wavefront's rows over the banks
    static constexpr int LDS = WAVES * PER_WAVE;
    static constexpr int PER_UNIT = at_most(4, 160 * 1024 / LDS);
    static constexpr int TILE = kTokens * WAVES;
    static_assert(kColumns * OUT_ROW * 4 <= STAGES * STAGE && LDS <= 160 * 1024, "a wavefront's result takes the place of its stages");
    static_assert((STAGES - 1) * (2 * LOADS + 1) + LOADS < 64, "vmcnt");
};

// ---- where things lie in a stage: rows of NC pieces, a piece's place XOR-ed with bits of its row, so that what one LDS access serves together (16
// lanes of 16 bytes, 32 of 8) lies in different banks.  What the row's own offset does not spread, `Z` bits of the piece's number do.

// keys: the 16 rows of a tile are tokens 8 (x / 4) + 4 t + x % 4
template <class F>
__host__ __device__ constexpr uint32_t key_swizzle(uint32_t row) {
    constexpr int Z = at_most(4, trailing_zeros(F::NC));
    return ((((row >> 3) & 3u) << 2 | (row & 3u)) >> (4 - Z)) & ((1u << Z) - 1u);
}
// values, 16-bit: four rows of 32 bytes for each group of 16 lanes; 8-bit: eight rows of 16 bytes
template <class F>
__host__ __device__ constexpr uint32_t value_swizzle(uint32_t row) {
    if constexpr (F::ES == 2) {
        constexpr int Z = at_most(3, trailing_zeros(F::NC / 2));
        return ((((row >> 3) & 1u) << 2 | (row & 3u)) >> (3 - Z) & ((1u << Z) - 1u)) << 1;
    } else {
        constexpr int Z = at_most(4, trailing_zeros(F::NC));
        return ((row & 15u) >> (4 - Z)) & ((1u << Z) - 1u);
    }
}

// lane i's 16 (4) bytes at lds + 16 i (4 i); the wait for them is counted (the compiler does not know of these loads)
__device__ __forceinline__ void load16(const char *at, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(at), "s"(lds) : "memory");
}
__device__ __forceinline__ void load4(const void *at, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(at), "s"(lds) : "memory");
}
template <int N>
__device__ __forceinline__ void landed() {
    static_assert(N < 64, "vmcnt");
    asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
}
// all but the newest `later` batches of L loads have landed
template <int L, int R>
__device__ __forceinline__ void landed_but(uint32_t later) {
    if constexpr (R == 0) {
        landed<0>();
    } else {
        if (later >= (uint32_t)R)
            landed<R * L>();
        else
            landed_but<L, R - 1>(later);
    }
}

typedef __attribute__((address_space(3))) char lds_char;
template <class X>
__device__ __forceinline__ X lds_at(uint32_t at) {
    return *reinterpret_cast<__attribute__((address_space(3))) X *>((lds_char *)(uintptr_t)at);
}
template <class X>
__device__ __forceinline__ void lds_put(uint32_t at, X x) {
    *reinterpret_cast<__attribute__((address_space(3))) X *>((lds_char *)(uintptr_t)at) = x;
}

// the visible tokens of a request, and the tiles that hold them
struct Seen {
    uint32_t first, past, tile, tiles;
};
template <int TILE>
__device__ __forceinline__ Seen seen_of(const AttendArgs &a, uint32_t r) {
    Seen s;
    s.past = min((uint32_t)max(a.length[r], 0), a.most);
    s.first = a.window && s.past > a.window ? s.past - a.window : 0u;
    s.tile = s.first / TILE;
    s.tiles = (s.past + TILE - 1) / TILE - s.tile;
    return s;
}

template <class F>
__global__ __launch_bounds__(64 * F::WAVES, F::PER_UNIT) void amap_attend_kernel(const AttendArgs a) {
    typedef typename Of<typename F::T>::eight eight;
    constexpr uint32_t kThreads = 64 * F::WAVES;
    extern __shared__ char smem[];
    __shared__ uint32_t sums[F::WAVES], found[4];
    __shared__ float top[F::WAVES][kColumns], total[F::WAVES][kColumns];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t g = lane >> 4, col = lane & 15u;
    const uint32_t base = (uint32_t)(uintptr_t)(lds_char *)smem + wave * F::PER_WAVE, ids = base + F::STAGES * F::STAGE;

    // ---- the share: tiles of all requests, and of those before each
    uint32_t tiles = 0;
    for (uint32_t r = tid; r < a.requests; r += kThreads) tiles += seen_of<F::TILE>(a, r).tiles;
#pragma unroll
    for (int d = 32; d; d >>= 1) tiles += __shfl_xor(tiles, d);
    if (lane == 0) sums[wave] = tiles;
    __syncthreads();
    uint32_t all = 0;
#pragma unroll
    for (int w = 0; w < F::WAVES; ++w) all += sums[w];
    all *= a.segments;
    const uint32_t share = max(a.least, (all + gridDim.x - 1) / gridDim.x);
    uint32_t u = blockIdx.x * share;
    const uint32_t end = min(u + share, all);
    // rows that see nothing, request by request over the workgroups
    for (uint32_t r = blockIdx.x; r < a.requests; r += gridDim.x) {
        if (seen_of<F::TILE>(a, r).tiles) continue;
        for (uint32_t i = tid; i < a.heads * a.dim; i += kThreads) {
            const uint32_t h = i / a.dim;
            reinterpret_cast<uint16_t *>(a.out)[(int64_t)r * a.out_token + (int64_t)h * a.out_head + (i - h * a.dim)] = 0;
        }
        if (a.lse)
            for (uint32_t h = tid; h < a.heads; h += kThreads) a.lse[(int64_t)r * a.heads + h] = -INFINITY;
    }
    Split *const split = reinterpret_cast<Split *>(a.parts) + blockIdx.x;
    float *const parts = a.parts + gridDim.x * (sizeof(Split) / 4);
    constexpr uint32_t kPart = kColumns * (F::DP + 2);   // maxima, sums, results of one piece of a segment
    if (u >= end) {
        if (a.parts && tid == 0) *split = Split{0, 0, 0, 0};
        return;
    }
    {
        const uint32_t want = fdiv(u, a.by_segments);
        uint32_t before = 0;
        for (uint32_t r0 = 0;; r0 += kThreads) {   // (ends: `want` is under the sum of all)
            const uint32_t r = r0 + tid, n = r < a.requests ? seen_of<F::TILE>(a, r).tiles : 0u;
            uint32_t x = n;
#pragma unroll
            for (uint32_t d = 1; d < 64; d <<= 1) {
                const uint32_t y = __shfl_up(x, d);
                if (lane >= d) x += y;
            }
            __syncthreads();
            if (lane == 63) sums[wave] = x;
            __syncthreads();
            uint32_t to = before;
            for (uint32_t w = 0; w < F::WAVES; ++w) {
                if (w == wave) x += to;
                to += sums[w];
            }
            if (want >= x - n && want < x) found[0] = r, found[1] = x - n;
            before = to;
            if (want < to) break;
        }
        __syncthreads();
    }
    uint32_t r = __builtin_amdgcn_readfirstlane(found[0]);
    uint32_t first_of = __builtin_amdgcn_readfirstlane(found[1]) * a.segments;   // the request's first unit
    Seen seen = seen_of<F::TILE>(a, r);
    uint32_t segment = (u - first_of) / seen.tiles, tile = u - first_of - segment * seen.tiles;
    bool leads_on = false;

    // ---- what does not change from segment to segment
    uint32_t row_of[F::LOADS], k_piece[F::LOADS], v_piece[F::LOADS];   // of the 16 bytes that this lane loads
#pragma unroll
    for (int j = 0; j < F::LOADS; ++j) {
        const uint32_t i = 64u * j + lane, row = i / F::NC, at = i % F::NC;
        row_of[j] = 4u * row;   // (as a byte address of ds_bpermute)
        k_piece[j] = at ^ key_swizzle<F>(row);
        v_piece[j] = at ^ value_swizzle<F>(row);
    }

    while (u < end) {
        const uint32_t n = min(seen.tiles - tile, end - u);   // tiles of this segment's piece
        const uint32_t kv = fdiv(segment, a.by_blocks), block = segment - kv * a.blocks;
        const uint32_t q0 = block * a.columns, rows = min(a.group - q0, a.columns);   // queries of the block
        const uint32_t head0 = kv * a.group + q0;

        // ---- a wavefront's steps: its 32 tokens of every tile that hold a visible one
        const uint32_t t0 = (seen.tile + tile) * F::TILE + wave * kTokens;
        const uint32_t s0 = t0 + kTokens <= seen.first ? 1u : 0u;
        const uint32_t s1 = t0 + (n - 1) * F::TILE >= seen.past ? n - 1 : n;
        const uint32_t steps = s1 > s0 ? s1 - s0 : 0u, begin = t0 + s0 * F::TILE;
        const int32_t *const row = a.table + (int64_t)r * a.table_stride;
        constexpr int L = 2 * F::LOADS + 1;   // loads of a step
        uint32_t mask[F::STAGES];   // of each stage's visible tokens
        auto ask = [&](uint32_t s, uint32_t slot) __attribute__((always_inline)) {   // the pages of step s
            const uint32_t token = min(max(begin + s * F::TILE + (lane & 31u), seen.first), seen.past - 1u);
            load4(row + fdiv(token, a.by_page), ids + slot * 256u);
        };
        auto issue = [&](uint32_t s, uint32_t slot) __attribute__((always_inline)) {   // -> the mask
            const uint32_t token = begin + s * F::TILE + (lane & 31u);
            const uint32_t id = lds_at<uint32_t>(ids + slot * 256u + 4u * (lane & 31u));
            const bool there = token >= seen.first && token < seen.past && id < a.n_pages;
            const uint32_t j = fdiv(token, a.by_page);
            const uint32_t at = there ? id * a.page_step + (token - j * a.page) * a.token_step + kv * a.head_step : kNoRow;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this stage has been read, and its ids
            const uint32_t lds = base + slot * F::STAGE;
            const char *const none = reinterpret_cast<const char *>(&kZeros);
            uint32_t off[F::LOADS];
#pragma unroll
            for (int i = 0; i < F::LOADS; ++i) off[i] = (uint32_t)__builtin_amdgcn_ds_bpermute((int)row_of[i], (int)at);
#pragma unroll
            for (int i = 0; i < F::LOADS; ++i)
                load16(off[i] != kNoRow && k_piece[i] < a.pieces ? a.k + ((uint64_t)(off[i] + k_piece[i]) << 4) : none, lds + 1024u * i);
            if constexpr (F::STAGES * L > 63) landed<63 - (F::LOADS + 1)>();   // no more than the counter holds
#pragma unroll
            for (int i = 0; i < F::LOADS; ++i)
                load16(off[i] != kNoRow && v_piece[i] < a.pieces ? a.v + ((uint64_t)(off[i] + v_piece[i]) << 4) : none, lds + F::SIDE + 1024u * i);
            ask(s + F::STAGES, slot);
            return (uint32_t)__ballot(there);
        };
        if (steps) {
#pragma unroll
            for (int s = 0; s < F::STAGES; ++s) ask(s, s);
        }
        // the queries: column c is query c, or c % 8 where the weights' second parts have columns 8 .. 15
        eight qf[F::DP / 32];
        {
            const uint32_t c = F::PAIRED ? col & 7u : col;
            const char *const q = a.q + 2 * ((int64_t)r * a.q_token + (int64_t)(head0 + (c < rows ? c : 0u)) * a.q_head);
#pragma unroll
            for (int i = 0; i < F::DP / 32; ++i) {
                const uint32_t d = 32u * i + 8u * g;
                u32x4 x = {0u, 0u, 0u, 0u};
                if (c < rows && d < a.dim) {
                    if (a.aligned)
                        x = *reinterpret_cast<const u32x4 *>(q + 2u * d);
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint16_t *const p = reinterpret_cast<const uint16_t *>(q) + d + 2 * e;
                            x[e] = p[0] | (uint32_t)p[1] << 16;
                        }
                }
                qf[i] = __builtin_bit_cast(eight, x);
            }
        }
        const float by = a.scale * kLog2e * (a.k_scale ? a.k_scale[kv] : 1.f);
        // (in registers before the first load that is waited for by count: the compiler would wait for them in the loop, each time)
#pragma unroll
        for (int i = 0; i < F::DP / 32; ++i) asm volatile("" ::"v"(qf[i]));
        asm volatile("" ::"v"(by));
        f32x4 o[F::DP / 16];
#pragma unroll
        for (int i = 0; i < F::DP / 16; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        if (steps) {
            landed<0>();   // the first pages, and the queries
#pragma unroll
            for (int s = 0; s < F::STAGES; ++s) mask[s] = (uint32_t)s < steps ? issue(s, s) : 0u;
        }
        for (uint32_t s = 0, slot = 0; s < steps; ++s) {
            landed_but<L, F::STAGES - 1>(steps - 1u - s);
            const uint32_t k_at = base + slot * F::STAGE, v_at = k_at + F::SIDE, shown = mask[0];
            // ---- scores: this lane's are of column `col` and tokens 8 g .. 8 g + 7
            f32x4 c[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint32_t token = 8u * (col >> 2) + 4u * t + (col & 3u);
#pragma unroll
                for (int i = 0; i < F::DP / 32; ++i) {
                    eight kf;
                    if constexpr (F::ES == 2) {
                        kf = lds_at<eight>(k_at + token * F::ROW + (((4u * i + g) ^ key_swizzle<F>(token)) << 4));
                    } else {
                        kf = eight_of_e4m3<typename F::T>(lds_at<u32x2>(k_at + token * F::ROW + (((2u * i + (g >> 1)) ^ key_swizzle<F>(token)) << 4) + ((g & 1u) << 3)));
                    }
                    c[t] = Of<typename F::T>::product(kf, qf[i], c[t]);
                }
            }
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = c[j >> 2][j & 3] * by;
            if (shown != 0xFFFFFFFFu) {
                const uint32_t mine = shown >> (8u * g);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = mine >> j & 1u ? x[j] : -INFINITY;
            }
            float high = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
            high = fmaxf(high, __shfl_xor(high, 16));
            high = fmaxf(high, __shfl_xor(high, 32));
            high = fmaxf(high, m);
            const float from = high == -INFINITY ? 0.f : high;
            if (__any(high != m)) {
                const float keep = __builtin_amdgcn_exp2f(m - from);
                l *= keep;
#pragma unroll
                for (int i = 0; i < F::DP / 16; ++i) o[i] *= keep;
                m = high;
            }
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(x[j] - from);
            l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
            eight pf, rest;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const typename Of<typename F::T>::one part = (typename Of<typename F::T>::one)p[j];
                pf[j] = part;
                rest[j] = (typename Of<typename F::T>::one)(p[j] - (float)part);
            }
            if constexpr (F::PAIRED) {
                if (col >= 8u) pf = rest;
            }
            // ---- results: 16 elements of V's rows at a time
#pragma unroll
            for (int i = 0; i < F::DP / 16; ++i) {
                eight vf;
                if constexpr (F::ES == 2) {
                    const uint32_t r0 = 8u * g + (col >> 2), in = (col & 3u) << 3;
                    union {
                        i16x4 half[2];
                        eight whole;
                    } y;
#pragma unroll
                    for (int hi = 0; hi < 2; ++hi) {
                        const uint32_t at = v_at + (r0 + 4u * hi) * F::ROW + (((2u * i + (in >> 4)) ^ value_swizzle<F>(r0 + 4u * hi)) << 4) + (in & 8u);
                        y.half[hi] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(lds_char *)(uintptr_t)at);
                    }
                    vf = y.whole;
                } else {
                    const uint32_t r0 = 8u * g + (col >> 1);
                    const uint32_t at = v_at + r0 * F::ROW + (((uint32_t)i ^ value_swizzle<F>(r0)) << 4) + ((col & 1u) << 3);
                    vf = eight_of_e4m3<typename F::T>(__builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2 *)(lds_char *)(uintptr_t)at)));
                }
                o[i] = Of<typename F::T>::product(vf, pf, o[i]);
                if constexpr (!F::PAIRED) o[i] = Of<typename F::T>::product(vf, rest, o[i]);
            }
#pragma unroll
            for (int i = 0; i + 1 < F::STAGES; ++i) mask[i] = mask[i + 1];
            mask[F::STAGES - 1] = s + F::STAGES < steps ? issue(s + F::STAGES, slot) : 0u;
            slot = slot + 1 == F::STAGES ? 0u : slot + 1;
        }
        landed<0>();   // (pages asked for that no step needs)

        // ---- the wavefronts' results side by side, in the place of their stages
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (g == 0) top[wave][col] = m, total[wave][col] = l;
#pragma unroll
        for (int i = 0; i < F::DP / 16; ++i) lds_put<f32x4>(base + 4u * (col * F::OUT_ROW + 16u * i + 4u * g), o[i]);
        __syncthreads();
        const bool whole = tile == 0 && n == seen.tiles;
        const float vs = a.v_scale ? a.v_scale[kv] : 1.f;
        float *const part = parts + (size_t)(2u * blockIdx.x + (tile == 0)) * kPart;   // the first piece of a segment, or a later one
        const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char *)smem;
        for (uint32_t i = tid; i < rows * F::DP; i += kThreads) {
            const uint32_t c = i / F::DP, d = i - c * F::DP;
            float high = top[0][c];
#pragma unroll
            for (int w = 1; w < F::WAVES; ++w) high = fmaxf(high, top[w][c]);
            const float from = high == -INFINITY ? 0.f : high;
            float sum = 0.f, x = 0.f;
#pragma unroll
            for (int w = 0; w < F::WAVES; ++w) {
                const float keep = __builtin_amdgcn_exp2f(top[w][c] - from);
                const uint32_t at = lds0 + w * F::PER_WAVE + 4u * (c * F::OUT_ROW + d);
                float y = lds_at<float>(at);
                if constexpr (F::PAIRED) y += lds_at<float>(at + 4u * 8u * F::OUT_ROW);
                sum += keep * total[w][c];
                x += keep * y;
            }
            if (whole) {
                const bool none = sum == 0.f;   // (scores of -inf only)
                if (d < a.dim) {
                    const float y = none ? 0.f : x * vs / sum;
                    reinterpret_cast<typename Of<typename F::T>::one *>(a.out)[(int64_t)r * a.out_token + (int64_t)(head0 + c) * a.out_head + d] =
                        (typename Of<typename F::T>::one)y;
                }
                if (d == 0 && a.lse) a.lse[(int64_t)r * a.heads + head0 + c] = none ? -INFINITY : (high + __builtin_amdgcn_logf(sum)) * kLn2;
            } else {
                part[2 * kColumns + i] = x;
                if (d == 0) part[c] = high, part[kColumns + c] = sum;
            }
        }
        __syncthreads();
        if (!whole && tile == 0) {
            leads_on = true;
            if (tid == 0) *split = Split{r, segment, (u + seen.tiles - 1) / share - blockIdx.x + 1, 0};
        }
        u += n;
        tile = 0;
        if (++segment == a.segments) {
            segment = 0;
            if (u < end) do
                    seen = seen_of<F::TILE>(a, ++r);
                while (seen.tiles == 0);   // (there is one: units are left)
        }
    }
    if (a.parts && !leads_on && tid == 0) *split = Split{0, 0, 0, 0};
}

// The pieces of a segment that was cut, joined: one workgroup per row of a segment, found at the workgroup in whose share it began.
struct JoinArgs {
    const float *parts;
    char *out;
    float *lse;
    const float *v_scale;
    int64_t out_token, out_head;
    uint32_t groups, columns, group, heads, dim, blocks;
    FastDiv by_columns, by_blocks;
};

template <class T, int DP>
__global__ __launch_bounds__(256) void amap_attend_join_kernel(const JoinArgs a) {
    constexpr uint32_t kPart = kColumns * (DP + 2), kLanes = DP / 4, kAtOnce = 256 / kLanes;
    __shared__ float sums[kAtOnce];
    __shared__ f32x4 results[kAtOnce][kLanes];
    const uint32_t w = fdiv(blockIdx.x, a.by_columns), c = blockIdx.x - w * a.columns;
    const Split s = reinterpret_cast<const Split *>(a.parts)[w];
    const uint32_t kv = fdiv(s.segment, a.by_blocks), block = s.segment - kv * a.blocks;
    if (s.count == 0 || c >= min(a.group - block * a.columns, a.columns)) return;
    const float *const parts = a.parts + a.groups * (sizeof(Split) / 4) + (size_t)(2u * w) * kPart;
    auto at = [&](uint32_t i) { return parts + (size_t)(i ? 2u * i : 1u) * kPart; };
    const uint32_t tid = threadIdx.x, from = tid / kLanes, d = 4u * (tid % kLanes);
    float high = -INFINITY;
    for (uint32_t i = 0; i < s.count; ++i) high = fmaxf(high, at(i)[c]);
    const float base = high == -INFINITY ? 0.f : high;
    float sum = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (from < kAtOnce)
        for (uint32_t i = from; i < s.count; i += kAtOnce) {
            const float *const p = at(i);
            const float keep = __builtin_amdgcn_exp2f(p[c] - base);
            sum += keep * p[kColumns + c];
            x += keep * *reinterpret_cast<const f32x4 *>(p + 2 * kColumns + c * DP + d);
        }
    if (from < kAtOnce) {
        results[from][tid % kLanes] = x;
        if (tid % kLanes == 0) sums[from] = sum;
    }
    __syncthreads();
    if (from) return;
    for (uint32_t i = 1; i < kAtOnce; ++i) {
        sum += sums[i];
        x += results[i][tid];
    }
    const bool none = sum == 0.f;
    const uint32_t h = kv * a.group + block * a.columns + c;
    const float vs = a.v_scale ? a.v_scale[kv] : 1.f;
    typename Of<T>::one *const out = reinterpret_cast<typename Of<T>::one *>(a.out) + (int64_t)s.request * a.out_token + (int64_t)h * a.out_head;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (d + e < a.dim) out[d + e] = (typename Of<T>::one)(none ? 0.f : x[e] * vs / sum);
    if (tid == 0 && a.lse) a.lse[(int64_t)s.request * a.heads + h] = none ? -INFINITY : (high + __builtin_amdgcn_logf(sum)) * kLn2;
}

// How a call is cut: workgroups, columns of a block, and whether a segment may be split between workgroups.
struct Cut {
    uint32_t groups, columns, blocks, segments, tile;
    bool splits;
    int dp;
    int64_t bytes;
};

template <class F>
amap_status attend(AttendArgs a, const Cut &cut, hipStream_t s) {
    static LdsReservation reserved;
    if constexpr (F::LDS > 65536 - 1024) {
        const hipError_t e = reserved.on_current_device({reinterpret_cast<const void *>(amap_attend_kernel<F>)}, F::LDS);
        if (e != hipSuccess) return launched(e, "amap_attend_kernel: cannot reserve its LDS stages");
    }
    hipError_t e = launch_kernel<amap_attend_kernel<F>>(dim3(cut.groups), dim3(64 * F::WAVES), F::LDS, s, a);
    if (e != hipSuccess || !cut.splits) return launched(e, "amap_attend_kernel");
    const JoinArgs j{a.parts, a.out, a.lse, a.v_scale, a.out_token, a.out_head, cut.groups, a.columns, a.group, a.heads, a.dim, a.blocks, make_fastdiv(a.columns), a.by_blocks};
    e = launch_kernel<amap_attend_join_kernel<typename F::T, F::DP>>(dim3(cut.groups * a.columns), dim3(256), 0, s, j);
    return launched(e, "amap_attend_join_kernel");
}

// the kernel form of a call, handed to f as a type
template <class T, int ES, class G>
void with_dim(int dp, bool paired, G f) {
    if (dp == 64) return paired ? f(Form<T, ES, 64, true>()) : f(Form<T, ES, 64, false>());
    if (dp == 96) return paired ? f(Form<T, ES, 96, true>()) : f(Form<T, ES, 96, false>());
    if (dp == 128) return paired ? f(Form<T, ES, 128, true>()) : f(Form<T, ES, 128, false>());
    return paired ? f(Form<T, ES, 256, true>()) : f(Form<T, ES, 256, false>());
}
template <class G>
void with_form(amap_type q, amap_type cache, int dp, bool paired, G f) {
    if (q == AMAP_BF16)
        cache == AMAP_E4M3 ? with_dim<Bf16, 1>(dp, paired, f) : with_dim<Bf16, 2>(dp, paired, f);
    else
        cache == AMAP_E4M3 ? with_dim<F16, 1>(dp, paired, f) : with_dim<F16, 2>(dp, paired, f);
}

amap_status check_attend(const amap_cache *cache, int heads, int64_t requests, int table_width) {
    Box k, v;
    const amap_status st = check_cache(cache, k, v);
    if (st != AMAP_OK) return st;
    if (heads < 1 || requests < 0 || table_width < 0) return AMAP_E_INVALID;
    if (heads % cache->kv_heads || requests > INT32_MAX / heads) return AMAP_E_SHAPE;
    if ((int64_t)table_width * cache->page_size > INT32_MAX) return AMAP_E_SHAPE;   // (lengths are int32)
    const int es = bytes_of(cache->type);
    if (cache->head_dim > 256 || cache->head_dim * es % 16) return refuse("head_dim over 256, or rows of the cache that are no whole 16-byte pieces");
    uint64_t at = reinterpret_cast<uintptr_t>(cache->k) | reinterpret_cast<uintptr_t>(cache->v);
    if (cache->n_pages > 1) at |= (uint64_t)cache->page_stride * es;
    if (cache->page_size > 1) at |= (uint64_t)cache->token_stride * es;
    if (cache->kv_heads > 1) at |= (uint64_t)cache->head_stride * es;
    if (at % 16) return refuse("rows of the cache that are not 16-byte aligned");
    // (offsets are counted in 16-byte pieces, in 32 bits)
    return k.past - k.first > ((uint64_t)1 << 36) - 65536 ? refuse("keys or values of 64 GB and more") : AMAP_OK;
}

amap_status cut_of(const amap_cache &c, int heads, int64_t requests, int table_width, Cut &cut) {
    const uint32_t group = (uint32_t)(heads / c.kv_heads);
    cut.dp = c.head_dim <= 64 ? 64 : c.head_dim <= 96 ? 96 : c.head_dim <= 128 ? 128 : 256;
    cut.columns = group <= 8 ? 8 : kColumns;
    cut.blocks = (group + cut.columns - 1) / cut.columns;
    cut.segments = cut.blocks * (uint32_t)c.kv_heads;
    uint32_t per_unit = 1;
    with_form(AMAP_BF16, c.type, cut.dp, group <= 8, [&](auto form) {
        cut.tile = decltype(form)::TILE;
        per_unit = decltype(form)::PER_UNIT;
    });
    const int64_t tiles = ((int64_t)table_width * c.page_size + cut.tile - 1) / cut.tile;
    int64_t most;
    if (__builtin_mul_overflow(requests * cut.segments, tiles, &most) || most >= ((int64_t)1 << 31)) return refuse("2^31 tiles of tokens or more over all requests and key heads");
    cut.splits = tiles > 1;
    cut.groups = (uint32_t)(most < 1 ? 1 : most < kUnits * per_unit ? most : kUnits * per_unit);
    cut.bytes = cut.splits ? (int64_t)cut.groups * (int64_t)(sizeof(Split) + 2 * 4 * kColumns * (cut.dp + 2)) : 0;
    return AMAP_OK;
}

}  // namespace

extern "C" amap_status amap_cache_attend_workspace(const amap_cache *cache, int heads, int64_t requests, int table_width, int64_t *bytes) {
    if (!bytes) return AMAP_E_INVALID;
    amap_status st = check_attend(cache, heads, requests, table_width);
    if (st != AMAP_OK) return st;
    Cut cut;
    st = cut_of(*cache, heads, requests, table_width, cut);
    if (st == AMAP_OK) *bytes = cut.bytes;
    return st;
}

extern "C" amap_status amap_cache_attend(const amap_cache *cache, const amap_heads *q, int64_t requests, const int32_t *table, int64_t table_stride, int table_width,
                                         const int32_t *length, float scale, int window, const amap_heads *out, float *lse, void *workspace, int64_t workspace_bytes,
                                         void *stream) {
    if (!q || !out) return AMAP_E_INVALID;
    amap_status st = check_attend(cache, q->heads, requests, table_width);
    if (st != AMAP_OK) return st;
    if (window < 0 || workspace_bytes < 0 || !std::isfinite(scale)) return AMAP_E_INVALID;
    if (requests == 0) return AMAP_OK;
    if (!length || (table_width && !table) || !q->data || !out->data) return AMAP_E_INVALID;
    if ((q->type != AMAP_BF16 && q->type != AMAP_F16) || out->type != q->type || (cache->type != q->type && cache->type != AMAP_E4M3)) return AMAP_E_INVALID;
    if (out->heads != q->heads || (requests > 1 && table_stride < table_width) || table_stride > ((int64_t)1 << 40)) return AMAP_E_SHAPE;
    const int dim = cache->head_dim, es = bytes_of(cache->type);
    const Box from = box_of(*q, requests, dim), to = box_of(*out, requests, dim), k = box_of(*cache, cache->k), v = box_of(*cache, cache->v);
    if (!from.fits || !to.fits || !to.apart) return AMAP_E_SHAPE;
    if (meet(to, from) || meet(to, k) || meet(to, v)) return AMAP_E_ALIAS;
    const uintptr_t q_at = reinterpret_cast<uintptr_t>(q->data);
    if ((q_at | reinterpret_cast<uintptr_t>(out->data)) % 2) return refuse("a tensor that does not begin at a whole element");
    Cut cut;
    st = cut_of(*cache, q->heads, requests, table_width, cut);
    if (st != AMAP_OK) return st;
    if (cut.bytes && (!workspace || workspace_bytes < cut.bytes)) return AMAP_E_INVALID;
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return refuse("a workspace that is not 16-byte aligned");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const StreamDevice device(s);
    if (device.status() != hipSuccess) return launched(device.status(), "the stream's device");
    AttendArgs a = {};
    a.k = static_cast<const char *>(cache->k);
    a.v = static_cast<const char *>(cache->v);
    a.q = static_cast<const char *>(q->data);
    a.out = static_cast<char *>(out->data);
    a.lse = lse;
    a.parts = cut.splits ? static_cast<float *>(workspace) : nullptr;
    a.k_scale = cache->k_scale;
    a.v_scale = cache->v_scale;
    a.table = table;
    a.length = length;
    a.table_stride = table_stride;
    a.q_token = q->token_stride;
    a.q_head = q->head_stride;
    a.out_token = out->token_stride;
    a.out_head = out->head_stride;
    // (strides of a dimension of one entry are never multiplied by anything but 0)
    a.page_step = (uint32_t)(cache->n_pages > 1 ? cache->page_stride * es / 16 : 0);
    a.token_step = (uint32_t)(cache->page_size > 1 ? cache->token_stride * es / 16 : 0);
    a.head_step = (uint32_t)(cache->kv_heads > 1 ? cache->head_stride * es / 16 : 0);
    a.n_pages = (uint32_t)cache->n_pages;
    a.page = (uint32_t)cache->page_size;
    a.most = (uint32_t)table_width * a.page;
    a.requests = (uint32_t)requests;
    a.kv_heads = (uint32_t)cache->kv_heads;
    a.heads = (uint32_t)q->heads;
    a.group = a.heads / a.kv_heads;
    a.dim = (uint32_t)dim;
    a.pieces = (uint32_t)(dim * es / 16);
    a.columns = cut.columns;
    a.blocks = cut.blocks;
    a.segments = cut.segments;
    a.by_page = make_fastdiv(a.page);
    a.by_segments = make_fastdiv(a.segments);
    a.by_blocks = make_fastdiv(a.blocks);
    a.least = 1;
    a.window = (uint32_t)window;
    a.aligned = q_at % 16 == 0 && (requests == 1 || q->token_stride % 8 == 0) && (q->heads == 1 || q->head_stride % 8 == 0);
    a.scale = scale;
    with_form(q->type, cache->type, cut.dp, cut.columns == 8, [&](auto form) { st = attend<decltype(form)>(a, cut, s); });
    return st;
}
