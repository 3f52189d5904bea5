// The product of operands in 8 bits with a scale for each block (amap_gemm_scaled):
//     out[m, n] = sum_b a_scale[m, b] w_scale[n / 128, b] sum_{k in b} a[m, k] w[n, k].
//
// A block of 128 k is one matrix instruction (16 x 16 x 128): it gives a block's sums from zero, which go into the running sums times their scales.
// The matrix instructions for 8 bits add eight neighbouring products at a time, and of each no more than what lies above 2^-13 of the largest of the eight (found with
// products of 2^16 and less beside one another; the sums of eight are added in 32 bits).  Over normally distributed operands that is 1.5e-5 of a result (2-norm): far below the rounding
// of a 16-bit one (1.2e-3 in bf16, 1.4e-4 in fp16), but not what one of 32 bits is asked for.  Those are made by the instructions for bf16, which holds every
// number of 8 bits and adds the products in 32 bits (9e-9), at half the rate.
//
// Three kernels, eleven shapes (way_of chooses): few rows of a stream w straight into registers; tiles that wavefronts of their own load into LDS; tiles of 256 rows whose loads are
// spread between the matrix instructions.  Additions to the running sums are four vector instructions to each matrix instruction, half the time of it: they run beside it, two
// instructions behind, but not for nothing (16384 x 8192 x 4096 without them 397 us, with them 448).
#include <algorithm>
#include <atomic>
#include <cstdio>
#include <cstdlib>

#include "amap_rows.hpp"

using namespace amap_rows_detail;
using namespace amap_detail;
using namespace amap_dev;

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct ScaledArgs {
    const char *a, *w;
    const float *a_scale, *w_scale;
    char *out;
    int64_t a_row, w_row, out_row;   // out: elements
    int64_t a_scale_row, a_scale_block, w_scale_row, w_scale_block;
    uint32_t M, N, K, type, tiles_m, tiles_n, tiles;
    FastDiv by_band;   // tiles of a band
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ bf16x8 bf16_of(uint32_t low, uint32_t high) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, 1.f, true),
                 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, 1.f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// a block's sums: 16 rows of w by 16 of a, of each 32 k to a lane (which ones is the same for both)
template <bool EXACT>
__device__ __forceinline__ f32x4 block_sums(const i32x8 &w, const i32x8 &a) {
    f32x4 p = {0.f, 0.f, 0.f, 0.f};
    if constexpr (EXACT) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of(w[i], w[i + 1]), bf16_of(a[i], a[i + 1]), p, 0, 0, 0);
    } else {
        p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, p, 0, 0, 0, 0, 0, 0);
    }
    return p;
}

// ---- tiles

template <class X>
__device__ __forceinline__ X lds_read(uint32_t at) {
    return *reinterpret_cast<__attribute__((address_space(3))) const X *>(at);
}
template <class X>
__device__ __forceinline__ void lds_write(uint32_t at, X x) {
    *reinterpret_cast<__attribute__((address_space(3))) X *>(at) = x;
}

// Loads straight into LDS: lane i's bytes land at `to` + 16 i (or 4 i).  The compiler does not know of them: landed() waits.
__device__ __forceinline__ void load_to_lds(const char *base, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(to) : "memory");
}
__device__ __forceinline__ void load_to_lds4(const float *at, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(at), "s"(to) : "memory");
}
// all but the newest N loads of this wavefront have landed and its reads of LDS are done; then the other wavefronts are met
template <int N>
__device__ __forceinline__ void landed() {
    static_assert(N < 64, "vmcnt");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(N) : "memory");
}

// the tile with an index (a workgroup's): each XCD (workgroups go round them) has a run of tiles of its own, along bands of `kBand` tile rows
constexpr uint32_t kXcds = 8, kBand = 8;
__device__ __forceinline__ void tile_of(const ScaledArgs &g, uint32_t index, uint32_t &tm, uint32_t &tn) {
    const uint32_t q = g.tiles / kXcds, r = g.tiles % kXcds, xcd = index % kXcds;
    const uint32_t t = xcd * q + min(xcd, r) + index / kXcds, in_band = kBand * g.tiles_n, band = fdiv(t, g.by_band), left = t - band * in_band;
    const uint32_t high = min(kBand, g.tiles_m - band * kBand);
    tn = __builtin_amdgcn_readfirstlane(high == kBand ? left / kBand : left / high);
    tm = __builtin_amdgcn_readfirstlane(band * kBand + left - tn * high);
}

// BM x BN of out to a workgroup of WVM x WVN wavefronts that compute and LOAD that only load (0: all load), NST steps of 128 k (a block) in LDS
template <int BM_, int BN_, int WVM_, int WVN_, int LOAD_, int NST_, bool EXACT_>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WVM = WVM_, WVN = WVN_, LOAD = LOAD_, NST = NST_, WAVES = WVM * WVN, LOADING = LOAD ? LOAD : WAVES;
    static constexpr bool EXACT = EXACT_;
    static constexpr int XM = BM / WVM, XN = BN / WVN, TI = XM / 16, TJ = XN / 16;   // a wavefront's part, in matrix instructions
    static constexpr uint32_t A = BM * 128, W = BN * 128, SCALES = (BM + BN + 63) / 64 * 256, STAGE = A + W + SCALES, LDS = NST * STAGE;
    static constexpr int NA = A / (1024 * LOADING), NW = W / (1024 * LOADING), NS = ((int)SCALES / 256 + LOADING - 1) / LOADING, L = NA + NW + NS;   // loads of a wavefront in a step
    static_assert(128 % XN == 0 && A % (1024 * LOADING) == 0 && W % (1024 * LOADING) == 0 && BM % 64 == 0, "");
    static_assert(LDS <= 160 * 1024 && XM * XN * (EXACT ? 4 : 2) * WAVES <= (int)LDS, "");
};

// A wavefront's part of the product through LDS (which everyone is done with by then), so that whole rows of it are stored: a lane holds four consecutive n of one m.
template <class T>
__device__ __forceinline__ void store_tile(const ScaledArgs &g, const f32x4 (&acc)[T::TI][T::TJ], uint32_t m0, uint32_t n0, uint32_t wave, uint32_t lane) {
    constexpr int TI = T::TI, TJ = T::TJ;
    const uint32_t in = lane & 15u, quarter = lane >> 4, wm = wave / T::WVN, wn = wave % T::WVN;
    __syncthreads();
    auto store = [&](auto of, auto to) __attribute__((always_inline)) {
        typedef decltype(of) E;
        constexpr uint32_t kRow = T::XN * E::bytes, kChunks = kRow / 16, kRows = 64 / kChunks, kEach = 16 / E::bytes;
        const uint32_t base = wave * (T::XM * kRow);
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int j = 0; j < TJ; ++j) {
                const uint32_t row = 16u * i + in, byte = (16u * j + 4u * quarter) * E::bytes;
                const uint32_t at = base + row * kRow + (((byte >> 4) ^ (row & (kChunks - 1))) << 4 | (byte & 15u));
                if constexpr (E::bytes == 4)
                    lds_write(at, acc[i][j]);
                else
                    lds_write(at, u32x2{bits<E>(acc[i][j][0]) | bits<E>(acc[i][j][1]) << 16, bits<E>(acc[i][j][2]) | bits<E>(acc[i][j][3]) << 16});
            }
        const uint32_t chunk = lane % kChunks, n = n0 + wn * T::XN + chunk * kEach;
#pragma unroll
        for (uint32_t first = 0; first < (uint32_t)T::XM; first += kRows) {
            const uint32_t row = first + lane / kChunks, m = m0 + wm * T::XM + row;
            const u32x4 x = lds_read<u32x4>(base + row * kRow + ((chunk ^ (row & (kChunks - 1))) << 4));
            if (m < g.M && n < g.N) store_piece<E>(to + ((int64_t)m * g.out_row + n) * E::bytes, 0, g.N - n, x);
        }
    };
    if constexpr (T::EXACT)
        store(F32{}, g.out);
    else if (g.type == AMAP_BF16)
        store(Bf16{}, g.out);
    else
        store(F16{}, g.out);
}

// A load instruction holds its wavefront until the address unit takes it, and the few matrix instructions of a smaller tile's step do not fill that time: loading is left to
// wavefronts of their own, which meet the others once a step.  The others have a step's fragments in registers while they read the next step's.  What is left is the chain of a step: a
// barrier, the latency of the first reads, the matrix instructions.  us a step of 128 k, one tile to a compute unit, operands in L2: 64 x 16 0.16, 64 x 32 0.19, 64 x 64 0.21, 128 x 128 0.37
// (out of memory 0.20, 0.24, 0.31, 0.50: what a unit has on its way).  With operands out of memory 64 x 4096 x 6144 12.1 us, 389 x 2576 x 5003 in 32 bits 28.3, 512 x 4096 x 6144 23.7 (1.1 PFLOP/s);
// out of the last-level cache 9.7, 24.2 and 18.9.
template <class T>
__global__ __launch_bounds__(64 * (T::WAVES + T::LOAD), 2) void amap_gemm_scaled_tile_kernel(const ScaledArgs g) {
    constexpr int TI = T::TI, TJ = T::TJ, NA = T::NA, NW = T::NW, NS = T::NS, NST = T::NST;
    static_assert(T::LOAD > 0 && NST >= 4, "a stage is refilled a step after it is read");
    const uint32_t tid = threadIdx.x, lane = tid & 63u, in = lane & 15u, quarter = lane >> 4;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint32_t tm, tn;
    tile_of(g, blockIdx.x, tm, tn);
    const uint32_t m0 = tm * T::BM, n0 = tn * T::BN;
    const uint32_t steps = (g.K + 127u) / 128u, tail = g.K % 128u;
    if (wave >= (uint32_t)T::WAVES) {
        // A row's 128 bytes of a step lie as eight chunks of 16, XOR-ed with row / 2, so that the rows which an LDS read serves together cover all banks.
        // A load instruction fills eight rows, lane by lane; rows past the last one read that again.
        const uint32_t own = wave - T::WAVES;
        uint32_t a_off[NA], w_off[NW];
        auto row_of = [&](uint32_t block) __attribute__((always_inline)) { return 8u * block + (lane >> 3); };
        auto chunk_of = [&](uint32_t block) __attribute__((always_inline)) { return (lane & 7u) ^ ((block & 1u) << 2 | lane >> 4); };
#pragma unroll
        for (int j = 0; j < NA; ++j) a_off[j] = (min(m0 + row_of(own * NA + j), g.M - 1u) - m0) * (uint32_t)g.a_row + 16u * chunk_of(own * NA + j);
#pragma unroll
        for (int j = 0; j < NW; ++j) w_off[j] = (min(n0 + row_of(own * NW + j), g.N - 1u) - n0) * (uint32_t)g.w_row + 16u * chunk_of(own * NW + j);
        const char *ka = g.a + (int64_t)m0 * g.a_row, *kw = g.w + (int64_t)n0 * g.w_row;
        // the scales of 64 rows or columns to an instruction (some the same ones)
        uint32_t part[NS];
        const float *scale[NS];
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            part[j] = (own * NS + j) % (T::SCALES / 256);
            const uint32_t line = 64u * part[j] + lane;
            scale[j] = part[j] < T::BM / 64 ? g.a_scale + min(m0 + line, g.M - 1u) * g.a_scale_row : g.w_scale + min(n0 + line - T::BM, g.N - 1u) / 128u * g.w_scale_row;
        }
        uint32_t to_load = steps, to = 0;
        auto issue = [&]() __attribute__((always_inline)) {
            const uint32_t a_to = to + own * (NA * 1024u), w_to = to + T::A + own * (NW * 1024u);
            if (to_load > 1 || tail == 0) {
#pragma unroll
                for (int j = 0; j < NA; ++j) load_to_lds(ka, a_off[j], a_to + 1024u * j);
#pragma unroll
                for (int j = 0; j < NW; ++j) load_to_lds(kw, w_off[j], w_to + 1024u * j);
            } else {   // what lies behind the last k is nobody's: zeros
#pragma unroll
                for (int j = 0; j < NA; ++j) {
                    if (16u * chunk_of(own * NA + j) < tail)
                        load_to_lds(ka, a_off[j], a_to + 1024u * j);
                    else
                        lds_write(a_to + 1024u * j + 16u * lane, u32x4{0, 0, 0, 0});
                }
#pragma unroll
                for (int j = 0; j < NW; ++j) {
                    if (16u * chunk_of(own * NW + j) < tail)
                        load_to_lds(kw, w_off[j], w_to + 1024u * j);
                    else
                        lds_write(w_to + 1024u * j + 16u * lane, u32x4{0, 0, 0, 0});
                }
            }
#pragma unroll
            for (int j = 0; j < NS; ++j) {
                load_to_lds4(scale[j], to + T::A + T::W + 256u * part[j]);
                scale[j] += part[j] < T::BM / 64 ? g.a_scale_block : g.w_scale_block;
            }
            ka += 128;
            kw += 128;
            --to_load;
            to = to + T::STAGE == T::LDS ? 0u : to + T::STAGE;
        };
        for (int s = 0; s < NST; ++s)
            if (to_load > 0) issue();
        // (the last step's loads may be fewer than T::L: once they are issued all are waited for)
        if (to_load > 0)
            landed<(NST - 1) * T::L>();
        else
            landed<0>();
        for (uint32_t s = 0; s + 1 < steps; ++s) {   // the next step has landed; the others are done with the last one's stage
            if (to_load > 0)
                landed<(NST - 3) * T::L>();
            else
                landed<0>();
            if (s > 0 && to_load > 0) issue();
        }
        return;
    }

    const uint32_t wm = wave / T::WVN, wn = wave % T::WVN;
    // a lane has 32 bytes of one row, chunks `quarter` and quarter + 4.  Addresses of the stage that is read, and what lies in it at constant offsets
    struct Reads {
        uint32_t a, a_far, w, w_far, sa, sw;
    } r;
    const uint32_t swizzled = (quarter ^ (in >> 1)) << 4;
    const uint32_t a_at = (wm * T::XM + in) * 128u + swizzled, w_at = T::A + (wn * T::XN + in) * 128u + swizzled;
    const uint32_t sa_at = T::A + T::W + 4u * (wm * T::XM + in), sw_at = T::A + T::W + 4u * (T::BM + wn * T::XN);
    auto turn_to = [&](uint32_t stage) __attribute__((always_inline)) {
        r = Reads{stage + a_at, stage + (a_at ^ 64u), stage + w_at, stage + (w_at ^ 64u), stage + sa_at, stage + sw_at};
        // (seen through, every sum with a constant would have a register of its own)
        asm volatile("" : "+v"(r.a), "+v"(r.a_far), "+v"(r.w), "+v"(r.w_far), "+v"(r.sa), "+v"(r.sw));
    };
    auto fragment = [&](uint32_t near, uint32_t far, uint32_t f) __attribute__((always_inline)) {
        const u32x4 x = lds_read<u32x4>(near + 2048u * f), y = lds_read<u32x4>(far + 2048u * f);
        return __builtin_bit_cast(i32x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    f32x4 acc[TI][TJ];
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // Two sets of fragments and scales: one is read while the other feeds the matrix cores.  (Read into each register behind its last use, most of them were asked for at the end of a step and
    // waited for at the beginning of the next: 64 x 64 0.30 us a step.)
    constexpr bool TWO = (TI + TJ) * 16 + TI * TJ * 4 < 128;   // (larger parts have no room for that)
    i32x8 fa[TWO + 1][TI], fw[TWO + 1][TJ];
    float sa[TWO + 1][TI], sw[TWO + 1];
    constexpr int Q = TI * TJ, R = TI + TJ, PER = (R + Q - 1) / Q, D = Q < 3 ? Q : 3;
    auto read = [&](int set, int f) __attribute__((always_inline)) {   // fragment f of a step
        if (f == 0) sw[set] = lds_read<float>(r.sw);
        if (f < TI)
            fa[set][f] = fragment(r.a, r.a_far, f), sa[set][f] = lds_read<float>(r.sa + 64u * f);
        else if (f < R)
            fw[set][f - TI] = fragment(r.w, r.w_far, f - TI);
    };
    asm volatile("s_barrier" ::: "memory");   // the first step has landed
    turn_to(0);
#pragma unroll
    for (int f = 0; f < R; ++f) read(0, f);
    // Block sums wait for D - 1 further matrix instructions before they are added, so that nothing waits for them.
    f32x4 p[D];
    float s[TI];
    auto add = [&](int q) __attribute__((always_inline)) {
        const int i = q / TJ, j = q % TJ;
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(p[q % D][v], s[i], acc[i][j][v]);
        asm volatile("" : "+v"(acc[i][j]));   // (else the additions gather behind the last of the matrix instructions)
    };
    uint32_t next = T::STAGE, left = steps;
    auto step = [&](auto of) __attribute__((always_inline)) {
        constexpr int set = decltype(of)::value;
        if (left > 1) asm volatile("s_barrier" ::: "memory");   // the next step has landed
        turn_to(next);   // (after the last step: a stale stage, read and unused)
#pragma unroll
        for (int i = 0; i < TI; ++i) s[i] = sa[set][i] * sw[set];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if constexpr (TWO) {
#pragma unroll
                for (int f = q * PER; f < (q + 1) * PER; ++f) read(set ^ 1, f);
                __builtin_amdgcn_sched_barrier(0);
            }
            p[q % D] = block_sums<T::EXACT>(fw[set][q % TJ], fa[set][q / TJ]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (!TWO) {
                if (q % TJ == TJ - 1) read(0, q / TJ);
                if (q / TJ == TI - 1) read(0, TI + q % TJ);
            }
            if (q >= D - 1) add(q - (D - 1));
        }
#pragma unroll
        for (int q = Q - (D - 1); q < Q; ++q) add(q);
        next = next + T::STAGE == T::LDS ? 0u : next + T::STAGE;
    };
    for (;;) {
        step(std::integral_constant<int, 0>{});
        if (--left == 0) break;
        if constexpr (!TWO) continue;
        step(std::integral_constant<int, TWO>{});
        if (--left == 0) break;
    }
    store_tile<T>(g, acc, m0, n0, wave, lane);
}

// the first `left` of eight elements of 16 bits
__device__ __forceinline__ void store_left(char *to, uint32_t left, u32x4 x) {
    if (left >= 8) {
        *reinterpret_cast<u32x4_any *>(to) = x;
        return;
    }
#pragma unroll 1
    for (; left > 0; --left, to += 2) {
        *reinterpret_cast<uint16_t *>(to) = (uint16_t)x[0];
        x = u32x4{x[0] >> 16 | x[1] << 16, x[1] >> 16 | x[2] << 16, x[2] >> 16 | x[3] << 16, x[3] >> 16};
    }
}

// The largest tiles: two stages, one workgroup to a compute unit, and the loads spread between the matrix instructions.  (Eight of them at once keep a wavefront from
// issuing anything else until the address unit has taken them.)  A step has two turns, each a barrier: at the second half of A's fragments, when w and the first half of A
// in its stage are read and may be refilled for the step after the next, and at the last fragment, when the second half may be.  So a load has a step and a half to land.
// A workgroup goes from tile to tile: behind a tile's last step the next one's first is loaded, and its products begin while the stores of the last are on their way (a workgroup to each tile:
// 9 us more for each, most of it the stores of all of them at once).  Where no tile is left the last step is loaded again, into a stage that nobody reads, so that what is in flight is
// always the same.
// 16384 x 8192 x 4096 447 us (2.46 PFLOP/s; 439 to 455 by card), the matrix cores busy 63 % of the cycles; a library's product with one scale for each operand, which adds no block sums, 346 on the same
// card (81 % at the same clock).  Without the additions 397, without reads of fragments 442.  With all loads of a step at its end 453, without any 406 (of 439); one turn a step, its loads
// spread over all of it, 446 to 457, and 4096 x 4096 x 4096 out of memory 66 us instead of 60.
template <class T>
struct Large : T {
    static constexpr uint32_t STAGE = T::A + T::W, SLOTS = 4;   // (scales are read until a step's end, and loaded with its first half)
    static constexpr uint32_t OUT = 2 * STAGE + SLOTS * T::SCALES, OUT_WAVE = 16 * T::XN * 2, LDS = OUT + T::WAVES * OUT_WAVE;   // room for 16 rows of each wavefront's products
    static constexpr int STORES = T::XM * T::XN * 2 / 1024;   // of a wavefront, for a tile
    static_assert(T::TI % 4 == 0 && T::NA % 2 == 0 && LDS <= 160 * 1024, "");
};

template <class T>
__global__ __launch_bounds__(64 * T::WAVES, 2) void amap_gemm_scaled_large_kernel(const ScaledArgs g) {
    constexpr int TI = T::TI, TJ = T::TJ, NA = T::NA, NW = T::NW, Q = TI * TJ, D = 3;
    constexpr int FIRST = NW + NA / 2 + 1, SECOND = NA / 2;   // loads of a turn
    const uint32_t tid = threadIdx.x, lane = tid & 63u, in = lane & 15u, quarter = lane >> 4;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / T::WVN, wn = wave % T::WVN;
    // ---- loads, as in the other tiles; a wavefront's first NA / 2 blocks of A are of the halves that the wavefronts read first
    uint32_t a_off[NA], w_off[NW];
    auto a_block = [&](int j) __attribute__((always_inline)) {
        constexpr uint32_t kHalf = T::XM / 16;   // blocks of half a wavefront's rows
        const uint32_t b = wave * (NA / 2) + (uint32_t)j % (NA / 2);
        return b / kHalf * (2 * kHalf) + b % kHalf + (j < NA / 2 ? 0u : kHalf);
    };
    auto row_of = [](uint32_t block, uint32_t lane) __attribute__((always_inline)) { return 8u * block + (lane >> 3); };
    auto chunk_of = [](uint32_t block, uint32_t lane) __attribute__((always_inline)) { return (lane & 7u) ^ ((block & 1u) << 2 | lane >> 4); };
    // (what is worked out once a tile is worked out there, and not kept in registers all along)
    auto once = [](uint32_t x) __attribute__((always_inline)) {
        asm volatile("" : "+v"(x));
        return x;
    };
    const char *ka, *kw;
    const uint32_t part = wave % ((T::BM + T::BN) / 64);
    const bool of_a = part < T::BM / 64;
    const float *scale;
    const int64_t scale_step = of_a ? g.a_scale_block : g.w_scale_block;
    const uint32_t whole = g.K / 128u, tail = g.K % 128u, steps = whole + (tail != 0);
    // What lies behind the last k is nobody's: lanes that would load it load their row's first 16 bytes of the step, and put zeros there once those have landed.
    uint32_t load_index = blockIdx.x, load_step = 0;
    auto fold_tail = [&]() __attribute__((always_inline)) {
        const uint32_t at = once(lane);
#pragma unroll
        for (int j = 0; j < NA; ++j)
            if (16u * chunk_of(a_block(j), at) >= tail) a_off[j] -= 16u * chunk_of(a_block(j), at);
#pragma unroll
        for (int j = 0; j < NW; ++j)
            if (16u * chunk_of(wave * NW + j, at) >= tail) w_off[j] -= 16u * chunk_of(wave * NW + j, at);
    };
    auto begin_tile = [&]() __attribute__((always_inline)) {
        const uint32_t at = once(lane), line = 64u * part + at;
        uint32_t tm, tn;
        tile_of(g, load_index, tm, tn);
        const uint32_t m0 = tm * T::BM, n0 = tn * T::BN;
#pragma unroll
        for (int j = 0; j < NA; ++j) a_off[j] = (min(m0 + row_of(a_block(j), at), g.M - 1u) - m0) * (uint32_t)g.a_row + 16u * chunk_of(a_block(j), at);
#pragma unroll
        for (int j = 0; j < NW; ++j) w_off[j] = (min(n0 + row_of(wave * NW + j, at), g.N - 1u) - n0) * (uint32_t)g.w_row + 16u * chunk_of(wave * NW + j, at);
        ka = g.a + (int64_t)m0 * g.a_row;
        kw = g.w + (int64_t)n0 * g.w_row;
        scale = of_a ? g.a_scale + min(m0 + line, g.M - 1u) * g.a_scale_row : g.w_scale + min(n0 + line - T::BM, g.N - 1u) / 128u * g.w_scale_row;
        load_step = 0;
        if (whole == 0) fold_tail();
    };
    auto next_step = [&]() __attribute__((always_inline)) {
        if (load_step + 1 < steps) {
            ++load_step;
            ka += 128;
            kw += 128;
            scale += scale_step;
            if (load_step == whole) fold_tail();
        } else if (load_index + gridDim.x < g.tiles) {
            load_index += gridDim.x;
            begin_tile();
        }
    };
    const char *from_a, *from_w;   // the step's, in scalar registers
    auto scalar = [](const char *p) __attribute__((always_inline)) {
        const uint64_t x = reinterpret_cast<uint64_t>(p);
        return reinterpret_cast<const char *>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)x));
    };
    auto to_scalar = [&]() __attribute__((always_inline)) {
        from_a = scalar(ka);
        from_w = scalar(kw);
        asm volatile("s_nop 4" : "+s"(from_a), "+s"(from_w));   // (a load reads a scalar register that a vector instruction has written five wait states later; the compiler does not see these loads)
    };
    auto load_a = [&](int j, uint32_t stage) __attribute__((always_inline)) { load_to_lds(from_a, a_off[j], stage + 1024u * a_block(j)); };
    auto load_w = [&](int j, uint32_t stage) __attribute__((always_inline)) { load_to_lds(from_w, w_off[j], stage + T::A + 1024u * (wave * NW + j)); };
    auto load_first = [&](int l, uint32_t stage, uint32_t slot) __attribute__((always_inline)) {
        if (l < NW)
            load_w(l, stage);
        else if (l < NW + NA / 2)
            load_a(l - NW, stage);
        else
            load_to_lds4(scale, 2 * T::STAGE + slot * T::SCALES + 256u * part);
    };
    auto clear = [&](bool second, uint32_t stage) __attribute__((always_inline)) {
        const uint32_t at = once(lane);
#pragma unroll
        for (int j = second ? NA / 2 : 0; j < (second ? NA : NA / 2); ++j)
            if (16u * chunk_of(a_block(j), at) >= tail) lds_write(stage + 1024u * a_block(j) + 16u * at, u32x4{0, 0, 0, 0});
        if (!second) {
#pragma unroll
            for (int j = 0; j < NW; ++j)
                if (16u * chunk_of(wave * NW + j, at) >= tail) lds_write(stage + T::A + 1024u * (wave * NW + j) + 16u * at, u32x4{0, 0, 0, 0});
        }
    };

    struct Reads {
        uint32_t a, a_far, w, w_far, sa, sw;
    } r;
    const uint32_t swizzled = (quarter ^ (in >> 1)) << 4;
    const uint32_t a_at = (wm * T::XM + in) * 128u + swizzled, w_at = T::A + (wn * T::XN + in) * 128u + swizzled;
    const uint32_t sa_at = 2 * T::STAGE + 4u * (wm * T::XM + in), sw_at = 2 * T::STAGE + 4u * (T::BM + wn * T::XN);
    auto turn_to = [&](uint32_t stage, uint32_t slot) __attribute__((always_inline)) {
        r = Reads{stage + a_at, stage + (a_at ^ 64u), stage + w_at, stage + (w_at ^ 64u), slot * T::SCALES + sa_at, slot * T::SCALES + sw_at};
        asm volatile("" : "+v"(r.a), "+v"(r.a_far), "+v"(r.w), "+v"(r.w_far), "+v"(r.sa), "+v"(r.sw));
    };
    auto fragment = [&](uint32_t near, uint32_t far, uint32_t f) __attribute__((always_inline)) {
        const u32x4 x = lds_read<u32x4>(near + 2048u * f), y = lds_read<u32x4>(far + 2048u * f);
        return __builtin_bit_cast(i32x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };

    f32x4 acc[TI][TJ];
#pragma unroll
    for (uint32_t t = 0; t < 2; ++t) {
        if (t == 0)
            begin_tile();
        else
            next_step();
        to_scalar();
#pragma unroll
        for (int l = 0; l < FIRST; ++l) load_first(l, t * T::STAGE, t);
#pragma unroll
        for (int l = 0; l < SECOND; ++l) load_a(NA / 2 + l, t * T::STAGE);
    }
    landed<FIRST + SECOND>();
    if (whole == 0) {
        clear(false, 0);
        clear(true, 0);
        landed<0>();
    }
    turn_to(0, 0);
    i32x8 fa[2], fw[TJ];
#pragma unroll
    for (int j = 0; j < TJ; ++j) fw[j] = fragment(r.w, r.w_far, j);
    fa[0] = fragment(r.a, r.a_far, 0);
    float sa = lds_read<float>(r.sa), sw = lds_read<float>(r.sw), s[2] = {0.f, 0.f};
    f32x4 p[D];
    auto add = [&](int q) __attribute__((always_inline)) {
        const int i = q / TJ, j = q % TJ;
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(p[q % D][v], s[i & 1], acc[i][j][v]);
        asm volatile("" : "+v"(acc[i][j]));   // (else the additions gather behind the last of the matrix instructions, and the registers do not suffice)
    };
    constexpr int Y = TJ * (TI / 2 - 1), X = TJ * (TI - 1);   // the turns
    constexpr int GAP = (X - Y) / FIRST > 0 ? (X - Y) / FIRST : 1;
    static_assert(Y + GAP * (FIRST - 1) < X, "a turn's loads are issued before the next one waits");
    uint32_t cur = 0, slot = 0;
    bool behind = false;   // STORES stores of the last tile were issued behind the loads of this one's first two steps
    for (uint32_t index = blockIdx.x; index < g.tiles; index += gridDim.x) {
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int j = 0; j < TJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (uint32_t step = 0; step < steps; ++step) {
            const uint32_t next = T::STAGE - cur;
            auto wait = [&](bool stores) __attribute__((always_inline)) {
                if (stores)
                    landed<FIRST + SECOND + T::STORES>();
                else
                    landed<FIRST + SECOND>();
            };
            float next_sw = 0.f;
            auto multiply = [&](int q) __attribute__((always_inline)) {
                const int i = q / TJ, j = q % TJ;
                if (j == 0) {
                    s[i & 1] = sa * sw;
                    fa[(i + 1) & 1] = fragment(r.a, r.a_far, (i + 1) % TI);
                    sa = lds_read<float>(r.sa + 64u * ((i + 1) % TI));
                }
                p[q % D] = block_sums<false>(fw[j], fa[i & 1]);
                __builtin_amdgcn_sched_barrier(0);
                if (i == TI - 1) fw[j] = fragment(r.w, r.w_far, j);
                if (q >= Y && (q - Y) % GAP == 0 && (q - Y) / GAP < FIRST) load_first((q - Y) / GAP, cur, (slot + 2) % T::SLOTS);
                if (q >= X && q - X < SECOND) load_a(NA / 2 + q - X, cur);
                if (q >= D - 1) add(q - (D - 1));
                __builtin_amdgcn_sched_barrier(0);
            };
#pragma unroll
            for (int q = 0; q < Y; ++q) multiply(q);
            wait(behind && step < 2);   // the second half of A of this step; the first halves of it and w are read
            if (step == whole) {
                clear(true, cur);
                landed<FIRST + SECOND>();
            }
            next_step();
            to_scalar();
#pragma unroll
            for (int q = Y; q < X; ++q) multiply(q);
            wait(behind && step == 0);   // the next step's w, scales and first half of A; this one's second half is read
            if (tail && (step + 1 < steps ? step + 1 : 0u) == whole) {
                clear(false, next);
                landed<FIRST + SECOND>();
            }
            turn_to(next, (slot + 1) % T::SLOTS);   // (the next tile's first step behind the last one)
            next_sw = lds_read<float>(r.sw);
#pragma unroll
            for (int q = X; q < Q; ++q) multiply(q);
#pragma unroll
            for (int q = Q - (D - 1); q < Q; ++q) add(q);
            sw = next_sw;
            cur = next;
            ++slot;
        }

        // ---- the tile's products, 16 rows at a time through the wavefront's own room (its accesses to LDS are in order): a lane holds four consecutive n of one m
        uint32_t tm, tn;
        tile_of(g, index, tm, tn);
        const uint32_t m0 = tm * T::BM + wm * T::XM, n0 = tn * T::BN + wn * T::XN;
        auto store = [&](auto of, auto whole_tile) __attribute__((always_inline)) {
            typedef decltype(of) E;
            constexpr uint32_t kRow = T::XN * 2, kChunks = kRow / 16, kRows = 64 / kChunks, kLoads = 16 / kRows;
            const uint32_t room = T::OUT + wave * T::OUT_WAVE, at_lane = once(lane), in = at_lane & 15u, quarter = at_lane >> 4, chunk = at_lane % kChunks, row = at_lane / kChunks;
            char *to = g.out + ((int64_t)(m0 + row) * g.out_row + n0 + 8u * chunk) * 2;
            const int64_t down = g.out_row * (kRows * 2);
            const uint32_t left = n0 + 8u * chunk < g.N ? g.N - n0 - 8u * chunk : 0u;
            uint32_t m = m0 + row;
#pragma unroll
            for (int i = 0; i < TI; ++i) {
#pragma unroll
                for (int j = 0; j < TJ; ++j) {
                    const uint32_t byte = (16u * j + 4u * quarter) * 2u;
                    lds_write(room + in * kRow + (((byte >> 4) ^ (in & (kChunks - 1))) << 4 | (byte & 15u)),
                              u32x2{bits<E>(acc[i][j][0]) | bits<E>(acc[i][j][1]) << 16, bits<E>(acc[i][j][2]) | bits<E>(acc[i][j][3]) << 16});
                }
#pragma unroll
                for (uint32_t l = 0; l < kLoads; ++l) {
                    const uint32_t at = row + l * kRows;
                    const u32x4 x = lds_read<u32x4>(room + at * kRow + ((chunk ^ (at & (kChunks - 1))) << 4));
                    // (The next tile's waits count one instruction to each of these; more of them would only wait longer.  Not in inline assembly: the hardware reads a 16-byte store's
                    // registers for two more instructions, in which the compiler then does not know that it must not write there.)
                    if constexpr (decltype(whole_tile)::value)
                        *reinterpret_cast<u32x4_any *>(to) = x;
                    else if (m < g.M)
                        store_left(to, left, x);
                    to += down;
                    m += kRows;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        behind = steps >= 2 && (tm + 1) * T::BM <= g.M && (tn + 1) * T::BN <= g.N;
        if (g.type == AMAP_BF16) {
            if (behind)
                store(Bf16{}, std::true_type{});
            else
                store(Bf16{}, std::false_type{});
        } else {
            if (behind)
                store(F16{}, std::true_type{});
            else
                store(F16{}, std::false_type{});
        }
    }
    landed<0>();   // (nothing lands in LDS that is another workgroup's by then)
}

// of the current device
uint32_t compute_units() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) == hipSuccess && dev >= 0 && dev < 64) n = known[dev].load(std::memory_order_relaxed);
    if (n > 0) return (uint32_t)n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) {
        (void)hipGetLastError();
        return 256;
    }
    if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
    return (uint32_t)n;
}

template <class T, bool LARGE = false>
hipError_t launch_tiles(ScaledArgs &g, hipStream_t s) {
    g.tiles_m = (g.M + T::BM - 1) / T::BM;
    g.tiles_n = (g.N + T::BN - 1) / T::BN;
    g.tiles = g.tiles_m * g.tiles_n;
    g.by_band = make_fastdiv(kBand * g.tiles_n);
    if constexpr (LARGE) {
        static LdsReservation reserved;
        const hipError_t e = reserved.on_current_device({reinterpret_cast<const void *>(amap_gemm_scaled_large_kernel<Large<T>>)}, Large<T>::LDS);
        if (e != hipSuccess) return e;
        const uint32_t units = compute_units();
        return launch_kernel<amap_gemm_scaled_large_kernel<Large<T>>>(dim3(g.tiles < units ? g.tiles : units), dim3(64 * T::WAVES), Large<T>::LDS, s, g);
    }
    if constexpr (!LARGE) {
        if (T::LDS > 65536) {
            static LdsReservation reserved;
            const hipError_t e = reserved.on_current_device({reinterpret_cast<const void *>(amap_gemm_scaled_tile_kernel<T>)}, T::LDS);
            if (e != hipSuccess) return e;
        }
        return launch_kernel<amap_gemm_scaled_tile_kernel<T>>(dim3(g.tiles), dim3(64 * (T::WAVES + T::LOAD)), T::LDS, s, g);
    }
}

// ---- few rows of a: w is streamed once, straight into registers

// TM x TN matrix instructions (16 TM rows of a, 16 TN of w) to a workgroup, whose wavefronts take the blocks of k in turn and join their sums in LDS, in their
// order.  A wavefront has U blocks on their way: as one is used the next is asked for.  Bound by what memory gives, behind a launch and one latency: 1 x 4096 x 4096 6.2 us with weights out of memory (17 MB, 2.7 TB/s; 5.3 out of the last-level cache), 8 x 14336 x 4096
// 15.4 (59 MB, 3.8 TB/s; 13.9); more rows read a's rows again for every 16 or 32 columns, from L2, and tiles take over (64 x 4096 x 6144 26, tiles of 64 x 32 12.5).
template <int TM_, int TN_, int U_, bool EXACT_>
struct Few {
    static constexpr int TM = TM_, TN = TN_, U = U_, MOST = 8;   // MOST: wavefronts
    static constexpr bool EXACT = EXACT_;
};

template <class T>
__global__ __launch_bounds__(64 * T::MOST) void amap_gemm_scaled_few_kernel(const ScaledArgs g) {
    constexpr int TM = T::TM, TN = T::TN, U = T::U;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, in = lane & 15u, quarter = lane >> 4, waves = blockDim.x >> 6;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t tm = fdiv(blockIdx.x, g.by_band), tn = blockIdx.x - tm * g.tiles_n, m0 = tm * (16 * TM), n0 = tn * (16 * TN);   // (a band: a row of tiles)
    // offsets from the first row's, which are scalar; rows past the last one read that again
    const char *const a0 = g.a + (int64_t)m0 * g.a_row, *const w0 = g.w + (int64_t)n0 * g.w_row;
    const float *const s0 = g.a_scale + (int64_t)m0 * g.a_scale_row, *t0[TN];
    uint32_t a_off[TM], w_off[TN], s_off[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const uint32_t m = min(m0 + 16 * i + in, g.M - 1u) - m0;
        a_off[i] = m * (uint32_t)g.a_row + 16 * quarter;
        s_off[i] = m * (uint32_t)g.a_scale_row;
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        w_off[j] = (min(n0 + 16 * j + in, g.N - 1u) - n0) * (uint32_t)g.w_row + 16 * quarter;
        t0[j] = g.w_scale + min(n0 + 16 * j, g.N - 1u) / 128u * g.w_scale_row;
    }
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    struct Block {
        u32x4 a[TM][2], w[TN][2];   // a lane's 32 bytes of a row's block: chunks `quarter` and quarter + 4
        float s[TM], t[TN];
    };
    auto load = [&](Block &x, uint32_t b, auto whole) __attribute__((always_inline)) {
        const char *const w = w0 + 128u * b, *const a = a0 + 128u * b;
        const uint32_t left = g.K - 128u * b;
        auto piece = [&](const char *row, uint32_t off, uint32_t h) __attribute__((always_inline)) {
            if (decltype(whole)::value || 16u * quarter + 64u * h < left) return *reinterpret_cast<const u32x4 *>(row + off + 64u * h);
            return u32x4{0, 0, 0, 0};   // behind the last k
        };
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            x.w[j][0] = piece(w, w_off[j], 0);
            x.w[j][1] = piece(w, w_off[j], 1);
            x.t[j] = t0[j][b * g.w_scale_block];
        }
        const float *const s = s0 + b * g.a_scale_block;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            x.a[i][0] = piece(a, a_off[i], 0);
            x.a[i][1] = piece(a, a_off[i], 1);
            x.s[i] = s[s_off[i]];
        }
    };
    auto fragment = [&](const u32x4 (&x)[2]) __attribute__((always_inline)) {
        return __builtin_bit_cast(i32x8, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto use = [&](const Block &x) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const f32x4 p = block_sums<T::EXACT>(fragment(x.w[j]), fragment(x.a[i]));
                const float by = x.s[i] * x.t[j];
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(p[v], by, acc[i][j][v]);
            }
    };
    const uint32_t blocks = g.K / 128u;   // whole ones
    Block x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (wave + u * waves < blocks) load(x[u], wave + u * waves, std::true_type{});
    for (uint32_t b = wave; b < blocks; b += U * waves) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t at = b + u * waves;
            if (at < blocks) {
                use(x[u]);
                if (at + U * waves < blocks) load(x[u], at + U * waves, std::true_type{});
            }
        }
    }
    if (g.K % 128u && blocks % waves == wave) {
        load(x[0], blocks, std::false_type{});
        use(x[0]);
    }

    // ---- the wavefronts' sums joined: four consecutive n of one m to a thread
    extern __shared__ f32x4 parts[];   // [waves][TM * TN][64]
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) parts[(wave * (TM * TN) + i * TN + j) * 64u + lane] = acc[i][j];
    __syncthreads();
    for (uint32_t at = tid; at < TM * TN * 64u; at += 64u * waves) {
        f32x4 x = parts[at];
        for (uint32_t k = 1; k < waves; ++k) x += parts[k * (TM * TN * 64u) + at];
        const uint32_t tile = at >> 6, m = m0 + tile / TN * 16u + (at & 15u), n = n0 + tile % TN * 16u + (at >> 4 & 3u) * 4u;
        if (m >= g.M || n >= g.N) continue;
        const int64_t to = (int64_t)m * g.out_row + n;
        auto put = [&](auto of) __attribute__((always_inline)) {
            typedef decltype(of) E;
            if constexpr (E::bytes == 4) {
                store_piece<F32>(g.out + to * 4, 0, g.N - n, __builtin_bit_cast(u32x4, x));
            } else {
                const uint32_t low = bits<E>(x[0]) | bits<E>(x[1]) << 16, high = bits<E>(x[2]) | bits<E>(x[3]) << 16;
                char *const out = g.out + to * 2;
                if (n + 4 <= g.N) {
                    *reinterpret_cast<u32x2_any *>(out) = u32x2{low, high};
                } else {
#pragma unroll
                    for (uint32_t e = 0; e < 3; ++e)
                        if (n + e < g.N) reinterpret_cast<uint16_t *>(out)[e] = (uint16_t)((e < 2 ? low : high) >> (e % 2 * 16));
                }
            }
        };
        if (T::EXACT)
            put(F32{});
        else if (g.type == AMAP_BF16)
            put(Bf16{});
        else
            put(F16{});
    }
}

template <class T>
hipError_t launch_few(ScaledArgs &g, hipStream_t s) {
    g.tiles_m = (g.M + 16 * T::TM - 1) / (16 * T::TM);
    g.tiles_n = (g.N + 16 * T::TN - 1) / (16 * T::TN);
    g.by_band = make_fastdiv(g.tiles_n);
    const uint32_t blocks = (g.K + 127u) / 128u, waves = blocks < (uint32_t)T::MOST ? blocks : (uint32_t)T::MOST;
    return launch_kernel<amap_gemm_scaled_few_kernel<T>>(dim3(g.tiles_m * g.tiles_n), dim3(64 * waves), waves * T::TM * T::TN * 1024u, s, g);
}

// The ways to run a product, and what each takes: us, `launch` for the launch, the first loads and the last stores, `tile` for a tile, and for every block of k s1 where
// a unit has one tile and all units have one (s0: the fewer have one the faster each), s2 for two and `more` for each further one; what lies between whole numbers of tiles per
// unit counts for `up` of the next one; `mb` for a megabyte of operands and product.  Fitted by least squares of the logarithm of estimate over time, a product weighted by the square of the
// best way's time over this one's, to products of M = 1 .. 16384, N = 16 .. 20000, K = 32 .. 16384 timed on the
// device with operands from memory (5078 with an out of 16 bits, 2709 of 32), each way where it takes up to twice the best one's time.  What the estimates choose is 0.9 %
// (0.7 %) off the best way in the mean, 7 % (5 %) at the 95th percentile, 38 % (35 %) at the worst.  They count on the 256 units of a whole card; whatever way is taken is right on any number.
// Whoever changes a kernel times it anew against the others at such sizes, and fits its line again.
enum Way { FEW_16x16, FEW_16x32, FEW_32x32, TILE_64x16, TILE_64x32, TILE_64x32_4, TILE_64x64, TILE_64x64_4, TILE_128x128, LARGE_256x128, LARGE_256x256, kWays };
struct Cost {
    float launch, tile, s0, s1, s2, more, up, mb;   // launch 0: not a way for this type
};
struct Shape {
    uint32_t bm, bn;
    const char *name;
    Cost wide, exact;   // out of 16 bits; of 32
};
const Shape kShapes[kWays] = {
    {16, 16, "few rows, 16 x 16", {2.37f, .01f, .088f, .137f, .236f, .106f, .646f, 0.f}, {2.385f, .015f, .096f, .140f, .261f, .115f, .458f, 0.f}},
    {16, 32, "few rows, 16 x 32", {2.483f, .001f, .132f, .201f, .399f, .185f, .736f, .017f}, {2.525f, 0.f, .144f, .204f, .418f, .212f, .722f, .026f}},
    {32, 32, "few rows, 32 x 32", {2.511f, .15f, .161f, .252f, .497f, .255f, .715f, 0.f}, {2.521f, .169f, .177f, .270f, .545f, .294f, .720f, 0.f}},
    {64, 16, "tiles of 64 x 16", {1.325f, 1.656f, .166f, .196f, .371f, .159f, .870f, .027f}, {}},
    {64, 32, "tiles of 64 x 32", {1.088f, 2.061f, .207f, .257f, .465f, .215f, .836f, .010f}, {}},
    {64, 32, "tiles of 64 x 32, four stages", {2.397f, .432f, .213f, .321f, .347f, .202f, .433f, .073f}, {2.207f, .705f, .367f, .421f, .557f, .204f, .589f, .049f}},
    {64, 64, "tiles of 64 x 64", {1.001f, 2.255f, .238f, .378f, .665f, .276f, .772f, .013f}, {}},
    {64, 64, "tiles of 64 x 64, four stages", {2.095f, .852f, .253f, .373f, .564f, .221f, .379f, .082f}, {2.108f, 1.068f, .366f, .408f, .688f, .301f, .662f, .065f}},
    {128, 128, "tiles of 128 x 128", {.779f, 3.031f, .426f, .654f, 1.192f, .492f, .916f, .081f}, {2.496f, 1.526f, .822f, .869f, 1.910f, .898f, 1.f, .192f}},
    {256, 128, "tiles of 256 x 128", {4.048f, 1.152f, .789f, .948f, 1.903f, .927f, .963f, .153f}, {}},
    {256, 256, "tiles of 256 x 256", {6.089f, .356f, 1.275f, 1.373f, 2.820f, 1.464f, .932f, .172f}, {}},
};

// kWays if the product has too many tiles for any of them
Way way_of(uint64_t M, uint64_t N, uint64_t K, bool exact) {
    Way best = kWays;
    float least = 0.f;
    const float steps = (float)((K + 127) / 128), mb = 1e-6f * ((float)(M * K + N * K) + (exact ? 4.f : 2.f) * (float)M * (float)N);
    for (int i = 0; i < kWays; ++i) {
        const Shape &w = kShapes[i];
        const Cost &c = exact ? w.exact : w.wide;
        const uint64_t tiles = ((M + w.bm - 1) / w.bm) * ((N + w.bn - 1) / w.bn);
        if (c.launch == 0.f || tiles >= 1u << 22) continue;   // (threads of a launch: 32 bits)
        const float q = (float)tiles / 256.f, up = (float)((tiles + 255) / 256), e = q > 1.f ? q + c.up * (up - q) : 1.f;
        const float step = c.s0 + (c.s1 - c.s0) * std::min(q, 1.f) + (c.s2 - c.s1) * (std::min(e, 2.f) - 1.f) + c.more * std::max(e - 2.f, 0.f);
        const float t = c.launch + c.tile * e + steps * step + c.mb * mb;
        if (best == kWays || t < least) best = (Way)i, least = t;
    }
    return best;
}

template <bool E>
hipError_t launch_as(Way way, ScaledArgs &g, hipStream_t s) {
    switch (way) {
    case FEW_16x16: return launch_few<Few<1, 1, 4, E>>(g, s);
    case FEW_16x32: return launch_few<Few<1, 2, 4, E>>(g, s);
    case FEW_32x32: return launch_few<Few<2, 2, E ? 3 : 4, E>>(g, s);
    case TILE_64x32_4: return launch_tiles<Tile<64, 32, 2, 1, 2, 4, E>>(g, s);
    case TILE_64x64_4: return launch_tiles<Tile<64, 64, 2, 2, 4, 4, E>>(g, s);
    case TILE_128x128: return launch_tiles<Tile<128, 128, 2, 4, 4, 4, E>>(g, s);
    default: break;
    }
    if constexpr (!E) {
        switch (way) {
        case TILE_64x16: return launch_tiles<Tile<64, 16, 2, 1, 2, 8, E>>(g, s);
        case TILE_64x32: return launch_tiles<Tile<64, 32, 2, 1, 2, 8, E>>(g, s);
        case TILE_64x64: return launch_tiles<Tile<64, 64, 2, 2, 4, 8, E>>(g, s);
        case LARGE_256x128: return launch_tiles<Tile<256, 128, 2, 4, 0, 2, E>, true>(g, s);
        case LARGE_256x256: return launch_tiles<Tile<256, 256, 2, 4, 0, 2, E>, true>(g, s);
        default: break;
        }
    }
    return hipErrorInvalidValue;
}

}  // namespace

extern "C" amap_status amap_gemm_scaled(const amap_rows *a, const amap_scales *a_scale, const amap_rows *w, const amap_scales *w_scale, int64_t M, int64_t N, int64_t K,
                                        const amap_rows *out, void *stream) {
    if (!a || !a_scale || !w || !w_scale || !out || M < 0 || N < 0 || K < 0 || a->type != AMAP_E4M3 || w->type != AMAP_E4M3 || !is_wide(out->type)) return AMAP_E_INVALID;
    if (M > INT32_MAX || N > INT32_MAX || K > INT32_MAX) return AMAP_E_SHAPE;
    if (K == 0) return refuse("a product over no k");
    if (K % 16) return refuse("a K that is no multiple of 16");
    if (M == 0 || N == 0) return AMAP_OK;
    if (!a->data || !w->data || !out->data || !a_scale->data || !w_scale->data) return AMAP_E_INVALID;
    const Runs from = runs_of(*a, M, K), by = runs_of(*w, N, K), to = runs_of(*out, M, N), sa = runs_of(*a_scale, M, blocks_of(K)), sw = runs_of(*w_scale, blocks_of(N), blocks_of(K));
    if (!from.box.fits || !by.box.fits || !sa.box.fits || !sw.box.fits || !to.box.fits || !to.box.apart) return AMAP_E_SHAPE;
    if (share(to, from) || share(to, by) || share(to, sa) || share(to, sw)) return AMAP_E_ALIAS;
    if (reinterpret_cast<uintptr_t>(a->data) % 16 || reinterpret_cast<uintptr_t>(w->data) % 16 || (M > 1 && a->row_stride % 16) || (N > 1 && w->row_stride % 16))
        return refuse("rows that do not begin at multiples of 16 bytes");
    if (reinterpret_cast<uintptr_t>(out->data) % bytes_of(out->type) || reinterpret_cast<uintptr_t>(a_scale->data) % 4 || reinterpret_cast<uintptr_t>(w_scale->data) % 4)
        return refuse("a tensor that does not begin at a whole element");
    ScaledArgs g = {};
    g.a = static_cast<const char *>(a->data), g.a_row = a->row_stride;
    g.w = static_cast<const char *>(w->data), g.w_row = w->row_stride;
    g.a_scale = a_scale->data, g.a_scale_row = a_scale->row_stride, g.a_scale_block = a_scale->block_stride;
    g.w_scale = w_scale->data, g.w_scale_row = w_scale->row_stride, g.w_scale_block = w_scale->block_stride;
    g.out = static_cast<char *>(out->data), g.out_row = out->row_stride;
    g.M = (uint32_t)M, g.N = (uint32_t)N, g.K = (uint32_t)K;
    g.type = out->type;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if ((M > 1 && (uint64_t)a->row_stride >= 1u << 24) || (N > 1 && (uint64_t)w->row_stride >= 1u << 24)) return refuse("rows that begin 16 MB apart or more");
    if (M > 1 && a_scale->row_stride >= 1 << 24) return refuse("scales of rows that begin 64 MB apart or more");
    const StreamDevice device(s);
    if (device.status() != hipSuccess) return launched(device.status(), "the stream's device");
    const Way way = way_of((uint64_t)M, (uint64_t)N, (uint64_t)K, g.type == AMAP_F32);
    if (way == kWays) return refuse("too many tiles for one launch");
    if (const char *tr = std::getenv("AMAP_PLAN_TRACE"); tr && tr[0] != '0')
        std::fprintf(stderr, "amap gemm scaled: %s, %lld x %lld x %lld\n", kShapes[way].name, (long long)M, (long long)N, (long long)K);
    return launched(g.type == AMAP_F32 ? launch_as<true>(way, g, s) : launch_as<false>(way, g, s), "amap_gemm_scaled");
}
