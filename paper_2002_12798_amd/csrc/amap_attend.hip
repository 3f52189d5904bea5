// Attention of one new token per request over a paged cache (amap_cache_attend): s_i = scale q . k_i over the visible tokens,
// out = sum softmax(s)_i v_i, lse = log sum exp s_i, with the running maximum and sum of a softmax in one pass over the cache.
//
// Bound by the cache's bytes: every visible key and value is read once, and 2 heads / kv_heads flop are done with each byte.  So the
// kernel is built around keeping loads in flight.
//   Work: tiles of 32 tokens, a workgroup is one wavefront.  The tiles of all requests and key heads are one line, cut into equal
//     shares, one for each workgroup of a grid that fills the chip once: long requests are split, short ones follow one
//     another, whatever the mix, and only where a cut falls inside a request are results joined (amap_attend_join_kernel).  Where no
//     request can be long, a workgroup of a few wavefronts has one request and key head to itself (amap_attend_team_kernel).
//   Loads: keys, values and the table's entries go straight into LDS (global_load_lds), a ring of two stages, waited for by count.
//     No wavefront waits for another; while one begins or ends a request its neighbours on the compute unit keep loading.  A token that is not visible is read from 16 bytes of
//     zeros, so nothing that lies in the cache behind a request's end comes near the sums.
//   Products: the scores as K Q^T, 32 tokens by 16 columns (the queries that share a key head), by 16 x 16 x 32 matrix instructions.  The tokens
//     are dealt to the rows of the two tiles so that a lane ends up with 8 consecutive ones: just what the next product,
//     V^T P^T, takes from it, so weights never leave their lane.  V comes transposed out of LDS (ds_read_tr).
//   A weight is kept in two 16-bit parts, itself rounded and what that leaves: one part alone would be off by as much as
//     the result's own rounding is.  With up to 8 queries to a key head the second part costs nothing: it takes the columns that are
//     idle.
//   An infinite value times a second part of 0 or of the other sign, or times a weight that has vanished in 32 bits, is NaN where the sum itself is infinite.  So a
//     result that is not finite is looked at again: the same tiles with one weight, positive in both parts, for every score but -inf, and what is not finite then (infinite,
//     or NaN of NaN, of both signs, or of an infinite score) takes the place of what was stored.  Whoever has no infinite values pays for the look: a multiply-add to a result.
// Measured, cold: two requests of 131072 tokens, 32 queries to 8 key heads of 128, bf16 (1.07 GB) 181 us, 5.9 TB/s; 64 ragged ones up to 4096 (140 MB) 33.8 us, 28 of
// them over shares and 5 of joining; 128 up to 2048 of an 8-bit cache, 12 heads of 64 (54 MB) 19 us; one of 500, 16 heads of 64, 6.7 us.
#include "amap_cache.hpp"

#include <type_traits>

using namespace amap_cache_detail;
using namespace amap_detail;
using namespace amap_dev;

namespace {

constexpr uint32_t kUnits = 256;   // compute units of an MI355X
constexpr int kTokens = 32;        // of a wavefront's step
constexpr int kColumns = 16;       // queries of a workgroup at a time (8 where their weights' second parts have the others)
constexpr uint32_t kNoRow = 0xFFFFFFFFu;
// What beginning and ending a segment counts for in a share, in tiles (1, 3, 6 or 10: 16 requests of about 1500 tokens 26.2 us by 3 and 27 by 10, 128 ragged ones of an 8-bit
// cache 20.2 and 22.2; 6 level with 3).
constexpr uint32_t kBegin = 3;
constexpr uint32_t kMostJoining = 8192;    // workgroups of a join
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

struct AttendArgs {
    const char *k, *v, *q;
    char *out;
    float *lse, *parts;
    struct Split *splits;
    const float *k_scale, *v_scale;
    const int32_t *table, *length;
    int64_t table_stride, q_token, q_head, out_token, out_head;
    uint32_t page_step, token_step, head_step;   // of the cache, in 16-byte pieces
    uint32_t n_pages, page, most;                // most: tokens that a row of the table can name
    uint32_t requests, kv_heads, group, dim, pieces;   // pieces: 16-byte ones of a row
    uint32_t heads, columns, segments;           // segments of a request: kv_heads times the column blocks of one
    FastDiv by_page, by_segments, by_blocks, by_groups;
    uint32_t blocks, groups;                     // column blocks of a key head; workgroups
    uint32_t window, aligned, halves;            // aligned: q in whole 16-byte pieces; halves: 16 tokens from a multiple of 16 on lie in one page
    float scale;
};

// Of each segment, for the join: the workgroup in whose share it begins and in how many pieces it is (0: in none, the result is there).
struct Split {
    uint32_t group, count;
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
    static constexpr float UP = 0.f;   // weights are kept times 2^UP
    static constexpr float ALIKE = 0x1p-30f * (1.f + 0x1p-10f);   // the one weight of a second look: both parts positive, 2^31 of the largest values no overflow
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
    // 2^15 times a weight (at most 1) is the largest that fits; without it all of a long cache's weights under 2^-25 would vanish beside one key of weight 1,
    // 131072 of them at 2^-26 0.2 % of the sum
    static constexpr float UP = 15.f;
    static constexpr float ALIKE = 1.f + 0x1p-12f;
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
    static constexpr bool INFINITE = ES_ == 2;              // whether a value can be infinite
    static constexpr int ROW = DP * ES, NC = ROW / 16;      // bytes and 16-byte pieces of a row in LDS
    static constexpr int STAGES = 2;
    static constexpr int SIDE = kTokens * ROW, STAGE = 2 * SIDE;
    static constexpr int LOADS = NC / 2;                    // of a side, 1 KB each (of the keys, and one of the table's entries)
    static constexpr int IDS = STAGES * 256;                // a word per lane and stage
    static constexpr int OUT_ROW = DP + 4;                  // floats; the 4 spread a wavefront's rows over the banks
    static constexpr int LDS = STAGES * STAGE + IDS;
    static constexpr int PER_UNIT = at_most(16, 160 * 1024 / LDS);   // workgroups that a compute unit holds at once
    static_assert(kColumns * OUT_ROW * 4 <= STAGES * STAGE && LDS <= 160 * 1024, "the results take the place of the stages");
    static constexpr bool HALVES = NC % 4 == 0;             // whether a load's rows are of one half of the tile
    static_assert(3 * LOADS + 2 < 64, "vmcnt");
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
// N loads of 16 bytes a lane, 1 KB apart in LDS: load i from base + off[i] (off counts 4096 - 1024 (i % 4) on top: the instruction's offset counts on both
// sides, so that one write of M0 serves four; base is 4096 less).  The first half of them from `lo`, the others from `hi`.  Past the caches where no
// other workgroup reads the same (ONCE): 205 -> 183 us over 1.07 GB; with four workgroups to a key head 30 -> 38.
#define AMAP_ROWS_OF_FOUR(HINT)                                                                                                                          \
    asm volatile("s_mov_b32 m0, %8\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %4" HINT "\n\tglobal_load_lds_dwordx4 %1, %5 offset:1024" HINT "\n\t"         \
                 "global_load_lds_dwordx4 %2, %6 offset:2048" HINT "\n\tglobal_load_lds_dwordx4 %3, %7 offset:3072" HINT ::"v"(off[i]),                    \
                 "v"(off[i + 1 < N ? i + 1 : 0]), "v"(off[i + 2 < N ? i + 2 : 0]), "v"(off[i + 3 < N ? i + 3 : 0]), "s"(b0), "s"(b1), "s"(b2), "s"(b3), "s"(at)       \
                 : "memory")
#define AMAP_ROWS_OF_TWO(HINT)                                                                                                                            \
    asm volatile("s_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2" HINT "\n\tglobal_load_lds_dwordx4 %1, %3 offset:1024" HINT ::"v"(off[i]), \
                 "v"(off[i + 1 < N ? i + 1 : 0]), "s"(b0), "s"(b1), "s"(at)                                                                                  \
                 : "memory")
template <bool ONCE, int N>
__device__ __forceinline__ void load_rows(const char *lo, const char *hi, const uint32_t (&off)[N], uint32_t lds) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const uint32_t at = lds + 1024u * i;
        const char *const b0 = 2 * i < N ? lo : hi, *const b1 = 2 * i + 2 < N ? lo : hi, *const b2 = 2 * i + 4 < N ? lo : hi, *const b3 = 2 * i + 6 < N ? lo : hi;
        if constexpr (ONCE) {
            if (i + 4 <= N)
                AMAP_ROWS_OF_FOUR(" nt");
            else
                AMAP_ROWS_OF_TWO(" nt");
        } else {
            if (i + 4 <= N)
                AMAP_ROWS_OF_FOUR("");
            else
                AMAP_ROWS_OF_TWO("");
        }
    }
}
#undef AMAP_ROWS_OF_FOUR
#undef AMAP_ROWS_OF_TWO
// the larger (sum) of what the four lanes of one column hold
__device__ __forceinline__ float top_of_column(float x) {
    const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1]));
    const auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
__device__ __forceinline__ float sum_of_column(float x) {
    const auto u = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(u[0]) + __uint_as_float(u[1]);
    const auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(w[0]) + __uint_as_float(w[1]);
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
    uint32_t first, past, tile, tiles, units;   // units: its tiles and what a segment of them costs besides
};
__device__ __forceinline__ Seen seen_of(const AttendArgs &a, int32_t length) {
    Seen s;
    s.past = min((uint32_t)max(length, 0), a.most);
    s.first = a.window && s.past > a.window ? s.past - a.window : 0u;
    s.tile = s.first / kTokens;
    s.tiles = (s.past + kTokens - 1) / kTokens - s.tile;
    s.units = s.tiles ? s.tiles + kBegin : 0u;
    return s;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t plus_shifted(uint32_t x) {
    return x + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ uint32_t sum_up_to(uint32_t x) {   // over the lanes, this one's included: within rows of 16 lanes, then their last ones' sums
    x = plus_shifted<0x118, 0xF>(plus_shifted<0x114, 0xF>(plus_shifted<0x112, 0xF>(plus_shifted<0x111, 0xF>(x))));
    return plus_shifted<0x143, 0xC>(plus_shifted<0x142, 0xA>(x));
}

// What a lane keeps from segment to segment.
template <class F>
struct Lane {
    uint32_t lane, g, col, base, ids;   // base, ids: of the wavefront's stages in LDS, and of the table's entries behind them
    // of the 16 bytes that it loads, the row (as an address of ds_bpermute), the piece of it, and both as an offset in half a tile of one page
    uint32_t row_of[F::LOADS], k_piece[F::LOADS], v_piece[F::LOADS], k_off[F::LOADS], v_off[F::LOADS];
    uint32_t k_at[2][F::DP / 32], v_at[2][F::DP / 16];   // where its parts of a stage lie
};
template <class F>
__device__ __forceinline__ Lane<F> lane_of(const AttendArgs &a, uint32_t lane, uint32_t base) {
    const uint32_t g = lane >> 4, col = lane & 15u;
    Lane<F> w;
    w.lane = lane, w.g = g, w.col = col, w.base = base, w.ids = base + F::STAGES * F::STAGE;
#pragma unroll
    for (int j = 0; j < F::LOADS; ++j) {
        const uint32_t i = 64u * j + lane, row = i / F::NC, at = i % F::NC;
        w.row_of[j] = 4u * row;
        w.k_piece[j] = at ^ key_swizzle<F>(row);
        w.v_piece[j] = at ^ value_swizzle<F>(row);
        w.k_off[j] = (((row & 15u) * a.token_step + w.k_piece[j]) << 4) + 4096u - 1024u * (j & 3);
        w.v_off[j] = (((row & 15u) * a.token_step + w.v_piece[j]) << 4) + 4096u - 1024u * (j & 3);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const uint32_t token = 8u * (col >> 2) + 4u * t + (col & 3u);
#pragma unroll
        for (int i = 0; i < F::DP / 32; ++i)
            w.k_at[t][i] = base + token * F::ROW +
                         (F::ES == 2 ? ((4u * i + g) ^ key_swizzle<F>(token)) << 4 : (((2u * i + (g >> 1)) ^ key_swizzle<F>(token)) << 4) + ((g & 1u) << 3));
#pragma unroll
        for (int i = 0; i < F::DP / 16; ++i) {
            const uint32_t row = F::ES == 2 ? 8u * g + (col >> 2) + 4u * t : 8u * g + (col >> 1);   // (8-bit: one access, t unused)
            w.v_at[t][i] = base + F::SIDE + row * F::ROW +
                         (F::ES == 2 ? ((2u * i + ((col & 3u) >> 1)) ^ value_swizzle<F>(row)) << 4 : ((uint32_t)i ^ value_swizzle<F>(row)) << 4) + ((col & 1u) << 3);
        }
    }
    return w;
}

// `steps` tiles of a segment from token `begin` on by one wavefront: the results of all its columns, not yet divided (o), a column's largest score less UP
// (m, in powers of two) and this lane's part of the column's sum of weights (l).  AGAIN, the second look: with the weight ALIKE for all scores but -inf, m of no use.
template <class F, bool AGAIN>
__device__ __forceinline__ void attend_tiles(const AttendArgs &a, const Lane<F> &w, uint32_t r, uint32_t kv, uint32_t head0, uint32_t rows, const Seen &seen, uint32_t begin,
                                             uint32_t steps, f32x4 (&o)[F::DP / 16], float &m, float &l) {
    typedef typename Of<typename F::T>::eight eight;
    const uint32_t lane = w.lane, g = w.g, col = w.col, base = w.base, ids = w.ids;
    const int32_t *const row = a.table + (int64_t)r * a.table_stride;
    constexpr int LV = F::LOADS, LK = LV + 1;   // loads of a step's values; of its keys and the pages of the step after next
    auto ask = [&](uint32_t s, uint32_t slot) __attribute__((always_inline)) {   // the pages of step s
        const uint32_t token = min(max(begin + s * kTokens + (lane & 31u), seen.first), seen.past - 1u);
        load4(row + fdiv(token, a.by_page), ids + slot * 256u);
    };
    uint32_t shown[2];    // of each stage, which tokens are visible
    uint32_t places = 0;  // of the step being loaded: where this lane's token lies (kNoRow: nowhere), in 16-byte pieces,
    bool fast = false;    // or, all of them being visible, where either half of them begins
    int64_t lo = 0, hi = 0;
    const char *const zeros = reinterpret_cast<const char *>(&kZeros);
    auto load_side = [&](const char *from, const uint32_t (&off)[F::LOADS], const uint32_t (&piece)[F::LOADS], uint32_t lds) __attribute__((always_inline)) {
        if (fast) {
            if (F::PAIRED || a.blocks == 1)
                load_rows<true>(from + lo, from + hi, off, lds);
            else
                load_rows<false>(from + lo, from + hi, off, lds);
        } else {
            uint32_t x[F::LOADS];
#pragma unroll
            for (int i = 0; i < F::LOADS; ++i) x[i] = (uint32_t)__builtin_amdgcn_ds_bpermute((int)w.row_of[i], (int)places);
#pragma unroll
            for (int i = 0; i < F::LOADS; ++i)
                load16(x[i] != kNoRow && piece[i] < a.pieces ? from + ((uint64_t)(x[i] + piece[i]) << 4) : zeros, lds + 1024u * i);
        }
    };
    auto load_keys = [&](uint32_t s, int slot) __attribute__((always_inline)) {
        const uint32_t t0 = begin + s * kTokens, token = t0 + (lane & 31u);
        const uint32_t id = lds_at<uint32_t>(ids + slot * 256u + 4u * (lane & 31u));
        const bool there = token >= seen.first && token < seen.past && id < a.n_pages;
        shown[slot] = (uint32_t)__ballot(there);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the keys that were here have been read, and the pages
        if constexpr (2 * LV + LK + LK > 63) landed<63 - LK>();   // no more than the counter holds
        fast = !AGAIN && F::HALVES && a.halves && shown[slot] == 0xFFFFFFFFu;   // (a second look is rare: the one form of loads that takes all)
        if (fast) {
            const uint32_t j0 = fdiv(t0, a.by_page), j1 = fdiv(t0 + 16u, a.by_page), id0 = __builtin_amdgcn_readlane(id, 0), id1 = __builtin_amdgcn_readlane(id, 16);
            const uint32_t x0 = id0 * a.page_step + (t0 - j0 * a.page) * a.token_step + kv * a.head_step;
            const uint32_t x1 = id1 * a.page_step + (t0 + 16u - j1 * a.page) * a.token_step + kv * a.head_step;
            lo = ((int64_t)x0 << 4) - 4096;
            hi = ((int64_t)x1 << 4) - 4096;
        } else {
            const uint32_t j = fdiv(token, a.by_page);
            places = there ? id * a.page_step + (token - j * a.page) * a.token_step + kv * a.head_step : kNoRow;
        }
        load_side(a.k, w.k_off, w.k_piece, base + slot * F::STAGE);
        ask(s + 2, slot);
    };
    auto load_values = [&](int slot) __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the values that were here have been read
        if constexpr (LV + LK + LK + LV > 63) landed<63 - LV>();
        load_side(a.v, w.v_off, w.v_piece, base + F::SIDE + slot * F::STAGE);
    };
#pragma unroll
    for (int s = 0; s < 2; ++s) ask(s, s);
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
#pragma unroll
    for (int i = 0; i < F::DP / 16; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = AGAIN ? INFINITY : -INFINITY;   // (INFINITY: never another, nothing is scaled)
    l = 0.f;
    landed<0>();   // the first pages, and the queries
    load_keys(0, 0);
    load_values(0);
    if (steps > 1) {
        load_keys(1, 1);
        load_values(1);
    }
    auto step = [&](uint32_t s, auto stage) __attribute__((always_inline)) {
        constexpr int slot = decltype(stage)::value;
        const bool next = s + 1 < steps, after = s + 2 < steps;
        if (next)
            landed<2 * LV + LK>();
        else
            landed<LV>();
        // ---- scores: this lane's are of column `col` and tokens 8 g .. 8 g + 7
        f32x4 c[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int i = 0; i < F::DP / 32; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                eight kf;
                if constexpr (F::ES == 2)
                    kf = lds_at<eight>(w.k_at[t][i] + slot * F::STAGE);
                else
                    kf = eight_of_e4m3<typename F::T>(lds_at<u32x2>(w.k_at[t][i] + slot * F::STAGE));
                c[t] = Of<typename F::T>::product(kf, qf[i], c[t]);
            }
        const uint32_t visible = shown[slot];
        if (after) load_keys(s + 2, slot);
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = c[j >> 2][j & 3] * by;
        if (visible != 0xFFFFFFFFu) {
            const uint32_t mine = visible >> (8u * g);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = mine >> j & 1u ? x[j] : -INFINITY;
        }
        float high = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        high = fmaxf(top_of_column(high) - Of<typename F::T>::UP, m);
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
        for (int j = 0; j < 8; ++j) {
            if constexpr (AGAIN)
                p[j] = x[j] == -INFINITY ? 0.f : Of<typename F::T>::ALIKE + (x[j] - x[j]);   // (NaN for a score of inf or NaN)
            else
                p[j] = __builtin_amdgcn_exp2f(x[j] - from);
        }
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
        if (after)
            landed<2 * LK + LV>();
        else if (next)
            landed<LK + LV>();
        else
            landed<0>();
#pragma unroll
        for (int i = 0; i < F::DP / 16; ++i) {
            eight vf;
            if constexpr (F::ES == 2) {
                union {
                    i16x4 half[2];
                    eight whole;
                } y;
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    y.half[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(lds_char *)(uintptr_t)(w.v_at[t][i] + slot * F::STAGE));
                vf = y.whole;
            } else {
                vf = eight_of_e4m3<typename F::T>(__builtin_bit_cast(
                    u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2 *)(lds_char *)(uintptr_t)(w.v_at[0][i] + slot * F::STAGE))));
            }
            o[i] = Of<typename F::T>::product(vf, pf, o[i]);
            if constexpr (!F::PAIRED) o[i] = Of<typename F::T>::product(vf, rest, o[i]);
        }
        if (after) load_values(slot);
    };
    for (uint32_t s = 0; s < steps; s += 2) {
        step(s, std::integral_constant<int, 0>{});
        if (s + 1 < steps) step(s + 1, std::integral_constant<int, 1>{});
    }
}

// whether one of a wavefront's results is not finite
template <class F>
__device__ __forceinline__ bool any_infinite(const f32x4 (&o)[F::DP / 16]) {
    if constexpr (!F::INFINITE) return false;
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < F::DP / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) x = __builtin_fmaf(o[i][e], 0.f, x);
    return __any(x != x);
}

// The kernel's arguments once more, for the second look: read there, not kept in scalar registers all the way.  (They are its only ones: offset 0.)
__device__ __forceinline__ const AttendArgs &arguments_again() {
    auto p = (const __attribute__((address_space(4))) AttendArgs *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const AttendArgs *)p;
}

template <class F>
__global__ __launch_bounds__(64, (F::PER_UNIT + 3) / 4) void amap_attend_kernel(const AttendArgs a) {
    extern __shared__ char smem[];
    const uint32_t lane = threadIdx.x, g = lane >> 4, col = lane & 15u;
    const uint32_t base = (uint32_t)(uintptr_t)(lds_char *)smem;

    // (the arguments that come later too: another wait for them costs 0.3 us)
    asm volatile("" ::"s"(a.k), "s"(a.v), "s"(a.q), "s"(a.out), "s"(a.lse), "s"(a.parts), "s"(a.splits), "s"(a.k_scale), "s"(a.table), "s"(a.table_stride), "s"(a.scale), "s"(a.by_page.mul),
                 "s"(a.by_segments.mul), "s"(a.by_blocks.mul), "s"(a.by_groups.mul), "s"(a.groups), "s"(a.window));
    // ---- the share: tiles of all requests, an equal run of them to a lane
    const uint32_t run = (a.requests + 63u) >> 6, r0 = min(lane * run, a.requests), r1 = min(r0 + run, a.requests);
    uint32_t mine = min(blockIdx.x, a.requests - 1u);
    asm volatile("" : "+v"(mine));
    const int32_t own = a.length[mine];   // (asked for here, looked at below: in a scalar register it would be waited for at once)
    uint32_t units = 0;
    int32_t length = 0;
    for (uint32_t r = r0; r < r1; r += 4u) {
        int32_t n[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) n[i] = a.length[min(r + i, r1 - 1u)];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) units += seen_of(a, r + i < r1 ? n[i] : 0).units;
        length = n[0];
    }
    const uint32_t upto = sum_up_to(units), all = __builtin_amdgcn_readlane(upto, 63) * a.segments;
    const uint32_t share = fdiv(max(all, 1u) - 1u, a.by_groups) + 1u;
    uint32_t u = blockIdx.x * share;
    const uint32_t end = min(u + share, all);
    // rows that see nothing, request by request over the workgroups
    for (uint32_t r = blockIdx.x; r < a.requests; r += a.groups) {
        if (__builtin_expect(seen_of(a, r == blockIdx.x ? __builtin_amdgcn_readfirstlane(own) : a.length[r]).tiles != 0u, 1)) continue;
        for (uint32_t i = lane; i < a.heads * a.dim; i += 64u) {
            const uint32_t h = i / a.dim;
            reinterpret_cast<uint16_t *>(a.out)[(int64_t)r * a.out_token + (int64_t)h * a.out_head + (i - h * a.dim)] = 0;
        }
        if (a.lse)
            for (uint32_t h = lane; h < a.heads; h += 64u) a.lse[(int64_t)r * a.heads + h] = -INFINITY;
        if (a.splits)
            for (uint32_t i = lane; i < a.segments; i += 64u) a.splits[r * a.segments + i] = Split{0u, 0u};
    }
    if (u >= end) return;
    constexpr uint32_t kPart = kColumns * (F::DP + 2);   // maxima, sums, results of one piece of a segment
    // the request of the first unit: the lane whose run holds it, then the request in its run
    const uint32_t want = fdiv(u, a.by_segments);
    uint32_t r, first_of;
    {
        const uint32_t at = (uint32_t)__builtin_ctzll(__ballot(want < upto));   // (there is one: `want` is under the sum of all)
        uint32_t before = __builtin_amdgcn_readlane(upto - units, at);
        r = at * run;
        first_of = before * a.segments;   // the request's first unit
        length = __builtin_amdgcn_readlane(length, at);
        for (; run > 1; r += 64u) {
            const uint32_t mine = r + lane;
            const int32_t theirs = a.length[min(mine, a.requests - 1u)];
            const uint32_t n = seen_of(a, mine < a.requests ? theirs : 0).units, x = before + sum_up_to(n);
            const uint64_t in = __ballot(want < x);
            if (in) {
                const uint32_t of = (uint32_t)__builtin_ctzll(in);
                r += of;
                length = __builtin_amdgcn_readlane(theirs, of);
                first_of = __builtin_amdgcn_readlane(x - n, of) * a.segments;
                break;
            }
            before = __builtin_amdgcn_readlane(x, 63);
        }
    }
    Seen seen = seen_of(a, length);
    uint32_t segment = (u - first_of) / seen.units, at = u - first_of - segment * seen.units;   // `at`: of the segment's units

    const Lane<F> w = lane_of<F>(a, lane, base);
    while (u < end) {
        // the piece of this segment in the share: its tiles follow the units of its beginning
        const uint32_t past = min(seen.units, at + (end - u)), tile = at > kBegin ? at - kBegin : 0u, n = past > kBegin ? past - kBegin - tile : 0u;
        if (n == 0) break;   // (the share ends before the segment's first tile)
        const uint32_t kv = fdiv(segment, a.by_blocks), block = segment - kv * a.blocks;
        const uint32_t q0 = block * a.columns, rows = min(a.group - q0, a.columns);   // queries of the block
        const uint32_t head0 = kv * a.group + q0;

        const bool whole = tile == 0 && n == seen.tiles;
        bool look = false;
        const auto attend_piece = [&](const AttendArgs &a, auto second) __attribute__((always_inline)) {
            constexpr bool AGAIN = decltype(second)::value;
            f32x4 o[F::DP / 16];
            float m, l;
            attend_tiles<F, AGAIN>(a, w, r, kv, head0, rows, seen, (seen.tile + tile) * kTokens, n, o, m, l);
            if constexpr (!AGAIN) look = any_infinite<F>(o);

            // ---- the results, through LDS (in the place of the stages) into rows; a piece of a segment into the workspace
            l = sum_of_column(l);
            const bool none = l == 0.f;   // (scores of -inf only)
            float *const part = a.parts + (size_t)(2u * blockIdx.x + (tile == 0)) * kPart;   // the first piece of a segment, or a later one
            const float vs = whole ? (none ? 0.f : (a.v_scale ? a.v_scale[kv] : 1.f) / l) : 1.f;
            if (!AGAIN && lane < rows) {
                if (!whole)
                    part[lane] = m, part[kColumns + lane] = l;
                else if (a.lse)
                    a.lse[(int64_t)r * a.heads + head0 + lane] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
            }
#pragma unroll
            for (int i = 0; i < F::DP / 16; ++i) lds_put<f32x4>(base + 4u * (col * F::OUT_ROW + 16u * i + 4u * g), none ? f32x4{0.f, 0.f, 0.f, 0.f} : o[i] * vs);
            for (uint32_t i = lane; i < rows * (F::DP / 4); i += 64u) {
                const uint32_t c = i / (F::DP / 4), d = 4u * (i % (F::DP / 4)), at = base + 4u * (c * F::OUT_ROW + d);
                f32x4 x = lds_at<f32x4>(at);
                if constexpr (F::PAIRED) x += lds_at<f32x4>(at + 4u * 8u * F::OUT_ROW);
                if (!whole) {
                    if constexpr (!AGAIN)
                        *reinterpret_cast<f32x4 *>(part + 2 * kColumns + 4 * i) = x;
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!__builtin_isfinite(x[e])) part[2 * kColumns + 4 * i + e] = x[e];
                } else {
                    typename Of<typename F::T>::one *const out =
                        reinterpret_cast<typename Of<typename F::T>::one *>(a.out) + (int64_t)r * a.out_token + (int64_t)(head0 + c) * a.out_head + d;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (d + e < a.dim && (!AGAIN || !__builtin_isfinite(x[e]))) out[e] = (typename Of<typename F::T>::one)x[e];
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read, before the next loads land there
        };
        attend_piece(a, std::false_type{});
        if constexpr (F::INFINITE)
            if (__builtin_expect(look, 0)) attend_piece(arguments_again(), std::true_type{});
        if (a.splits && tile == 0 && lane == 0) a.splits[r * a.segments + segment] = Split{blockIdx.x, whole ? 0u : (u - at + seen.units - 1) / share - blockIdx.x + 1};
        u += past - at;
        at = 0;
        if (++segment == a.segments) {
            segment = 0;
            if (u < end) do
                    seen = seen_of(a, a.length[++r]);
                while (seen.tiles == 0);   // (there is one: units are left)
        }
    }
}

// The segments that were cut, their pieces joined: a segment (all its rows at once) or one row of it to a workgroup.
struct JoinArgs {
    const float *parts_at;
    const Split *splits;
    char *out;
    float *lse;
    const float *v_scale;
    int64_t out_token, out_head;
    uint32_t work, at_once, columns, group, heads, dim;   // at_once: rows of a workgroup
    FastDiv by_parts, by_segments, by_blocks;             // parts: workgroups to a segment
    uint32_t parts, segments, blocks;
};

template <class T, int DP, int THREADS>
__global__ __launch_bounds__(THREADS) void amap_attend_join_kernel(const JoinArgs a) {
    constexpr uint32_t kPart = kColumns * (DP + 2), kLanes = DP / 4, kSlots = THREADS / kLanes;   // slots: of a row's lanes
    __shared__ float tops[kSlots], sums[kSlots];
    __shared__ f32x4 results[kSlots][kLanes];
    const uint32_t slot = threadIdx.x / kLanes, lane = threadIdx.x % kLanes, d = 4u * lane;
    for (uint32_t i = blockIdx.x; i < a.work; i += gridDim.x) {
        const uint32_t id = fdiv(i, a.by_parts), c0 = (i - id * a.parts) * a.at_once;
        const Split s = a.splits[id];
        if (s.count == 0) continue;
        const uint32_t r = fdiv(id, a.by_segments), segment = id - r * a.segments;
        const uint32_t kv = fdiv(segment, a.by_blocks), block = segment - kv * a.blocks, rows = min(a.group - block * a.columns, a.columns);
        // a slot has one row of so many, and every so-manieth piece of it
        const uint32_t ways = kSlots / a.at_once, way = slot / a.at_once, c = c0 + slot % a.at_once;
        const float *const first = a.parts_at + (size_t)(2u * s.group) * kPart;
        float high = -INFINITY, sum = 0.f;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        if (way < ways && c < rows) {
#pragma unroll 8
            for (uint32_t p = way; p < s.count; p += ways) {
                const float *const part = first + (size_t)(p ? 2u * p : 1u) * kPart;
                const float m = part[c], l = part[kColumns + c];
                const f32x4 y = *reinterpret_cast<const f32x4 *>(part + 2 * kColumns + c * DP + d);
                const float up = fmaxf(high, m), base = up == -INFINITY ? 0.f : up;
                const float keep = __builtin_amdgcn_exp2f(high - base), take = __builtin_amdgcn_exp2f(m - base);
                sum = sum * keep + l * take;
                x = x * keep + y * take;
                high = up;
            }
        }
        if (slot < kSlots) {
            results[slot][lane] = x;
            if (lane == 0) tops[slot] = high, sums[slot] = sum;
        }
        __syncthreads();
        if (way == 0 && c < rows) {
            for (uint32_t w = 1; w < ways; ++w) {
                const uint32_t other = slot + w * a.at_once;
                const float m = tops[other], up = fmaxf(high, m), base = up == -INFINITY ? 0.f : up;
                const float keep = __builtin_amdgcn_exp2f(high - base), take = __builtin_amdgcn_exp2f(m - base);
                sum = sum * keep + sums[other] * take;
                x = x * keep + results[other][lane] * take;
                high = up;
            }
            const bool none = sum == 0.f;
            const uint32_t h = kv * a.group + block * a.columns + c;
            const float by = none ? 0.f : (a.v_scale ? a.v_scale[kv] : 1.f) / sum;
            typename Of<T>::one *const out = reinterpret_cast<typename Of<T>::one *>(a.out) + (int64_t)r * a.out_token + (int64_t)h * a.out_head;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (d + e < a.dim) out[d + e] = (typename Of<T>::one)(none ? 0.f : x[e] * by);
            // (a factor may be 0: what is infinite or NaN in a piece is that in the result)
            if (__builtin_expect(!__builtin_isfinite((x[0] + x[1]) + (x[2] + x[3])), 0)) {
                f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (uint32_t p = 0; p < s.count; ++p) {
                    const f32x4 z = *reinterpret_cast<const f32x4 *>(first + (size_t)(p ? 2u * p : 1u) * kPart + 2 * kColumns + c * DP + d);
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] += __builtin_isfinite(z[e]) ? 0.f : z[e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (d + e < a.dim && !__builtin_isfinite(y[e])) out[d + e] = (typename Of<T>::one)(none ? 0.f : y[e] * by);
            }
            if (lane == 0 && a.lse) a.lse[(int64_t)r * a.heads + h] = none ? -INFINITY : (high + __builtin_amdgcn_logf(sum)) * kLn2;
        }
        __syncthreads();
    }
}

// One segment to a workgroup, its tiles dealt to the wavefronts, which join what they have through LDS: one launch and no workspace, for calls whose
// segments are all short (team_of says which).
template <class F>
__global__ __launch_bounds__(64 * F::PER_UNIT, (F::PER_UNIT + 3) / 4) void amap_attend_team_kernel(const AttendArgs a) {
    typedef typename Of<typename F::T>::one one;
    extern __shared__ char smem[];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const uint32_t stages = (uint32_t)(uintptr_t)(lds_char *)smem;
    const uint32_t r = fdiv(blockIdx.x, a.by_segments), segment = blockIdx.x - r * a.segments;
    const uint32_t kv = fdiv(segment, a.by_blocks), q0 = (segment - kv * a.blocks) * a.columns, rows = min(a.group - q0, a.columns), head0 = kv * a.group + q0;
    const Seen seen = seen_of(a, a.length[r]);
    const uint32_t each = (seen.tiles + waves - 1) / waves, first = wave * each, n = first < seen.tiles ? min(each, seen.tiles - first) : 0u;
    const uint32_t base = stages + wave * F::LDS, stats = F::STAGES * F::STAGE;   // stats: of a wavefront's LDS, maxima and sums of its columns
    const uint32_t parts = each ? (seen.tiles + each - 1) / each : 0u;   // wavefronts that have something
    const float vs = a.v_scale ? a.v_scale[kv] : 1.f;
    uint32_t look = 0;
    const auto attend_segment = [&](const AttendArgs &a, auto second) __attribute__((always_inline)) {
        constexpr bool AGAIN = decltype(second)::value;
        if (n) {
            const Lane<F> w = lane_of<F>(a, lane, base);
            f32x4 o[F::DP / 16];
            float m, l;
            attend_tiles<F, AGAIN>(a, w, r, kv, head0, rows, seen, (seen.tile + first) * kTokens, n, o, m, l);
            l = sum_of_column(l);
#pragma unroll
            for (int i = 0; i < F::DP / 16; ++i) lds_put<f32x4>(base + 4u * (w.col * F::OUT_ROW + 16u * i + 4u * w.g), o[i]);
            if (lane < kColumns) {
                lds_put<float>(base + stats + 4u * lane, AGAIN ? 0.f : m);
                lds_put<float>(base + stats + 64u + 4u * lane, l);
            }
            if constexpr (F::INFINITE && !AGAIN) lds_put<uint32_t>(base + stats + 128u, any_infinite<F>(o));
        }
        __syncthreads();
        if constexpr (F::INFINITE && !AGAIN)
            for (uint32_t p = 0; p < parts; ++p) look |= lds_at<uint32_t>(stages + p * F::LDS + stats + 128u);
        for (uint32_t i = threadIdx.x; i < rows * (F::DP / 4); i += blockDim.x) {
            const uint32_t c = i / (F::DP / 4), d = 4u * (i % (F::DP / 4));
            float high = -INFINITY, sum = 0.f;
            for (uint32_t p = 0; p < parts; ++p) high = fmaxf(high, lds_at<float>(stages + p * F::LDS + stats + 4u * c));
            const float from = high == -INFINITY ? 0.f : high;
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
            for (uint32_t p = 0; p < parts; ++p) {
                const uint32_t at = stages + p * F::LDS;
                const float take = __builtin_amdgcn_exp2f(lds_at<float>(at + stats + 4u * c) - from);
                sum += take * lds_at<float>(at + stats + 64u + 4u * c);
                f32x4 y = lds_at<f32x4>(at + 4u * (c * F::OUT_ROW + d));
                if constexpr (F::PAIRED) y += lds_at<f32x4>(at + 4u * ((c + 8u) * F::OUT_ROW + d));
                x += y * take;
            }
            const bool none = sum == 0.f;   // (nothing seen, or scores of -inf only)
            const float by = none ? 0.f : vs / sum;
            one *const out = reinterpret_cast<one *>(a.out) + (int64_t)r * a.out_token + (int64_t)(head0 + c) * a.out_head + d;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (d + e < a.dim && (!AGAIN || !__builtin_isfinite(x[e]))) out[e] = (one)(none ? 0.f : x[e] * by);
            if (!AGAIN && d == 0 && a.lse) a.lse[(int64_t)r * a.heads + head0 + c] = none ? -INFINITY : (high + __builtin_amdgcn_logf(sum)) * kLn2;
        }
    };
    attend_segment(a, std::false_type{});
    if constexpr (F::INFINITE)
        if (__builtin_expect(look != 0u, 0)) {
            __syncthreads();   // (the results have been read: the stages are in their place)
            attend_segment(arguments_again(), std::true_type{});
        }
}

// How a call is cut: workgroups, columns of a block, and whether a segment may be split between workgroups.
struct Cut {
    uint32_t groups, columns, blocks, segments;
    bool splits;
    int dp;
    int64_t parts, bytes;   // where the pieces begin in the workspace, and its size
};

template <class F>
amap_status attend(AttendArgs a, const Cut &cut, uint32_t team, hipStream_t s) {
    if (team) {
        if constexpr (F::PER_UNIT * F::LDS > 65536) {
            static LdsReservation reserved;
            const hipError_t e = reserved.on_current_device({reinterpret_cast<const void *>(amap_attend_team_kernel<F>)}, F::PER_UNIT * F::LDS);
            if (e != hipSuccess) return launched(e, "amap_attend_team_kernel: cannot reserve its LDS stages");
        }
        const hipError_t e = launch_kernel<amap_attend_team_kernel<F>>(dim3(a.requests * a.segments), dim3(64u * team), team * F::LDS, s, a);
        return launched(e, "amap_attend_team_kernel");
    }
    if constexpr (F::LDS > 65536) {
        static LdsReservation reserved;
        const hipError_t e = reserved.on_current_device({reinterpret_cast<const void *>(amap_attend_kernel<F>)}, F::LDS);
        if (e != hipSuccess) return launched(e, "amap_attend_kernel: cannot reserve its LDS stages");
    }
    hipError_t e = launch_kernel<amap_attend_kernel<F>>(dim3(cut.groups), dim3(64), F::LDS, s, a);
    if (e != hipSuccess || !cut.splits) return launched(e, "amap_attend_kernel");
    // As many lanes to a row as there are pieces of a segment, if all are split alike; a wavefront at a time where those are few (six pieces of
    // each of 253 segments: 7.3 us by 256 threads, 5.3 by 64).
    const uint32_t segments = a.requests * a.segments, rows = a.columns < a.group ? a.columns : a.group, pieces = 1u + cut.groups / segments;
    const bool few = pieces <= 16;
    uint32_t at_once = (few ? 64u : 256u) / (F::DP / 4) / pieces;
    at_once = at_once < 1 ? 1 : at_once > rows ? rows : at_once;
    const uint32_t parts = (rows + at_once - 1) / at_once, work = segments * parts;
    const JoinArgs j{a.parts, a.splits, a.out, a.lse, a.v_scale, a.out_token, a.out_head, work, at_once, a.columns, a.group, a.heads, a.dim, make_fastdiv(parts), a.by_segments, a.by_blocks,
                     parts, a.segments, a.blocks};
    const dim3 grid(work < kMostJoining ? work : kMostJoining);
    e = few ? launch_kernel<amap_attend_join_kernel<typename F::T, F::DP, 64>>(grid, dim3(64), 0, s, j)
            : launch_kernel<amap_attend_join_kernel<typename F::T, F::DP, 256>>(grid, dim3(256), 0, s, j);
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
        per_unit = decltype(form)::PER_UNIT;
    });
    const int64_t tiles = ((int64_t)table_width * c.page_size + kTokens - 1) / kTokens;
    int64_t most;
    if (__builtin_mul_overflow(requests * cut.segments, tiles + kBegin, &most) || most >= ((int64_t)1 << 31)) return refuse("2^31 tiles of tokens or more over all requests and key heads");
    cut.splits = tiles > 1 && requests > 0;
    cut.groups = (uint32_t)(most < 1 ? 1 : most < kUnits * per_unit ? most : kUnits * per_unit);
    cut.parts = (requests * cut.segments * (int64_t)sizeof(Split) + 15) / 16 * 16;
    cut.bytes = cut.splits ? cut.parts + (int64_t)cut.groups * (2 * 4 * kColumns * (cut.dp + 2)) : 0;
    return AMAP_OK;
}

// Wavefronts of a workgroup that has a segment to itself, or 0 for shares.  A compute unit by itself loads 52 bytes a ns, by four wavefronts as by eight (2000 tokens of 64,
// one, two, four, eight of them: 44, 24.6, 15.1, 15.5 us), and the join of shares costs 4 to 6 us: so segments up to 288 KB (16 requests of 500 tokens, heads of 128, four to
// a key head: 14.0 -> 11.0 us; four of 1000 tokens 12.4 by shares and 15.5), and 512 KB where all compute units have one (a window of 1000, 256 requests, heads of 96: 18.9 -> 13.3, now 13.6).  No more wavefronts
// than the chip holds at once (1600 segments of 500 tokens, one, two, three, four of them: 16.3, 14.7, 15.4, 17.7), and none with less than 32 KB.  A wavefront's
// own part: up to 96 KB and 10 tiles (8 tiles of heads of 256, 32 KB each, by two wavefronts: 14.2 us, by shares 12.7).  (These limits stand between the few points named here, the second
// on the window alone; and the table says what a segment can be, not what it is: one request of 500 tokens, 16 heads of 64, 7.2 us in a table for 528 or 1024 and 9.5 in one for 4096 or 32768.)
template <class F>
uint32_t team_of(const AttendArgs &a) {
    uint32_t tiles = (a.most + kTokens - 1) / kTokens;   // of the longest segment that the table and the window allow: lengths are on the device
    if (a.window) {
        const uint32_t seen = (a.window - 1) / kTokens + 2;   // tiles that a window can touch
        tiles = tiles < seen ? tiles : seen;
    }
    const uint64_t segments = (uint64_t)a.requests * a.segments;
    if (segments > 1u << 22) return 0;   // (a launch counts its threads in 32 bits)
    if (tiles < 2) return 1;
    constexpr uint32_t kSteps = at_most(10, 98304 / F::STAGE);
    const uint64_t bytes = (uint64_t)tiles * F::STAGE;
    if (bytes > (segments < kUnits ? 288u << 10 : 512u << 10)) return 0;
    uint64_t most = (kUnits * F::PER_UNIT + segments - 1) / segments;
    if (most > F::PER_UNIT) most = F::PER_UNIT;
    uint64_t waves = (bytes + 32767) / 32768;
    if (waves > 4) waves = 4;
    if (waves * kSteps < tiles) waves = (tiles + kSteps - 1) / kSteps;
    if (waves > most) waves = most;
    const uint32_t steps = (uint32_t)((tiles + waves - 1) / waves);
    return steps <= kSteps ? (tiles + steps - 1) / steps : 0u;
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
    if (out->heads != q->heads || table_stride < 0 || table_stride > ((int64_t)1 << 40)) return AMAP_E_SHAPE;   // (0: requests of one table row)
    const int dim = cache->head_dim, es = bytes_of(cache->type);
    const Box from = box_of(*q, requests, dim), to = box_of(*out, requests, dim), k = box_of(*cache, cache->k), v = box_of(*cache, cache->v);
    if (!from.fits || !to.fits || !to.apart) return AMAP_E_SHAPE;
    if (share(*out, *q, requests, dim) || meet(to, k) || meet(to, v)) return AMAP_E_ALIAS;
    const int64_t rows_of_table[2] = {requests, table_width}, strides_of_table[2] = {table_stride, 1};
    const Box entries = table_width ? box_of(table, 4, 2, rows_of_table, strides_of_table) : box_of(table, 0);
    if (!entries.fits) return AMAP_E_SHAPE;
    const uintptr_t q_at = reinterpret_cast<uintptr_t>(q->data);
    if ((q_at | reinterpret_cast<uintptr_t>(out->data)) % 2) return refuse("a tensor that does not begin at a whole element");
    Cut cut;
    st = cut_of(*cache, q->heads, requests, table_width, cut);
    if (st != AMAP_OK) return st;
    if (cut.bytes && (!workspace || workspace_bytes < cut.bytes)) return AMAP_E_INVALID;
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return refuse("a workspace that is not 16-byte aligned");
    // what the call writes against one another and against all that it reads: lengths that changed on the way would give workgroups different shares, and pieces that were written over
    // would name places outside the workspace
    const Box sums = box_of(lse, lse ? 4 * requests * q->heads : 0), work = box_of(workspace, cut.bytes);
    const Box read[] = {from, k, v, entries, box_of(length, 4 * requests), box_of(cache->k_scale, cache->k_scale ? 4 * cache->kv_heads : 0),
                        box_of(cache->v_scale, cache->v_scale ? 4 * cache->kv_heads : 0)};
    for (const Box &b : read)
        if (meet(sums, b) || meet(work, b) || (&b != read && meet(to, b))) return AMAP_E_ALIAS;
    if (meet(sums, to) || meet(work, to) || meet(sums, work)) return AMAP_E_ALIAS;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const StreamDevice device(s);
    if (device.status() != hipSuccess) return launched(device.status(), "the stream's device");
    AttendArgs a = {};
    a.k = static_cast<const char *>(cache->k);
    a.v = static_cast<const char *>(cache->v);
    a.q = static_cast<const char *>(q->data);
    a.out = static_cast<char *>(out->data);
    a.lse = lse;
    if (cut.splits) {
        a.splits = static_cast<Split *>(workspace);
        a.parts = reinterpret_cast<float *>(static_cast<char *>(workspace) + cut.parts);
    }
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
    a.groups = cut.groups;
    a.by_groups = make_fastdiv(a.groups);
    a.window = (uint32_t)window;
    a.aligned = q_at % 16 == 0 && (requests == 1 || q->token_stride % 8 == 0) && (q->heads == 1 || q->head_stride % 8 == 0);
    // (16 rows of a page within 32-bit byte offsets; heads of a whole form: no pieces of zeros)
    a.halves = cache->page_size % 16 == 0 && dim == cut.dp && (cache->page_size == 1 || cache->token_stride * es * 16 < ((int64_t)1 << 31));
    a.scale = scale;
    with_form(q->type, cache->type, cut.dp, cut.columns == 8, [&](auto form) { st = attend<decltype(form)>(a, cut, team_of<decltype(form)>(a), s); });
    return st;
}
