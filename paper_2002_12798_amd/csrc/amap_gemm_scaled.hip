// The product of operands in 8 bits with a scale for each block (amap_gemm_scaled):
//     out[m, n] = sum_b a_scale[m, b] w_scale[n / 128, b] sum_{k in b} a[m, k] w[n, k].
//
// A block of 128 k is one matrix instruction (16 x 16 x 128): it gives a block's sums from zero, which go into the running sums times their scales.
// The matrix instructions for 8 bits add eight neighbouring products at a time, and of each no more than what lies above 2^-13 of the largest of the eight (found with
// products of 2^16 and less beside one another; the sums of eight are added in 32 bits).  Over normally distributed operands that is 1.5e-5 of a result (2-norm): far below the rounding
// of a 16-bit one (1.2e-3 in bf16, 1.4e-4 in fp16), but not what one of 32 bits is asked for.  Those are made by the instructions for bf16, which holds every
// number of 8 bits and adds the products in 32 bits (9e-9), at half the rate.
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
    uint32_t M, N, K, type, tiles_m, tiles_n;
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

// the tile of a workgroup: each XCD (workgroups go round them) has a run of tiles of its own, along bands of `kBand` tile rows
constexpr uint32_t kXcds = 8, kBand = 8;
__device__ __forceinline__ void tile_of(const ScaledArgs &g, uint32_t &tm, uint32_t &tn) {
    const uint32_t q = gridDim.x / kXcds, r = gridDim.x % kXcds, xcd = blockIdx.x % kXcds;
    const uint32_t t = xcd * q + min(xcd, r) + blockIdx.x / kXcds, in_band = kBand * g.tiles_n, band = fdiv(t, g.by_band), left = t - band * in_band;
    const uint32_t high = min(kBand, g.tiles_m - band * kBand);
    tn = high == kBand ? left / kBand : left / high;
    tm = band * kBand + left - tn * high;
}

// BM x BN of out to a workgroup of WVM x WVN wavefronts, NST steps of 128 k (a block) in LDS
template <int BM_, int BN_, int WVM_, int WVN_, int NST_, bool EXACT_>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WVM = WVM_, WVN = WVN_, NST = NST_, WAVES = WVM * WVN;
    static constexpr bool EXACT = EXACT_;
    static constexpr int XM = BM / WVM, XN = BN / WVN, TI = XM / 16, TJ = XN / 16;   // a wavefront's part, in matrix instructions
    static constexpr uint32_t A = BM * 128, W = BN * 128, SCALES = (BM + BN) * 4, STAGE = A + W + SCALES, LDS = NST * STAGE;
    static constexpr int NA = A / (1024 * WAVES), NW = W / (1024 * WAVES), L = NA + NW + 1;   // loads of a wavefront in a step
    static_assert(TI % 2 == 0 && 128 % XN == 0 && A % (1024 * WAVES) == 0 && W % (1024 * WAVES) == 0 && (BM + BN) / 64 <= WAVES, "");
    static_assert(LDS <= 160 * 1024 && XM * XN * (EXACT ? 4 : 2) * WAVES <= LDS, "");
};

template <class T>
__global__ __launch_bounds__(64 * T::WAVES, 2) void amap_gemm_scaled_tile_kernel(const ScaledArgs g) {
    constexpr int TI = T::TI, TJ = T::TJ, NA = T::NA, NW = T::NW, NST = T::NST;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, in = lane & 15u, quarter = lane >> 4;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / T::WVN, wn = wave % T::WVN;
    uint32_t tm, tn;
    tile_of(g, tm, tn);
    const uint32_t m0 = tm * T::BM, n0 = tn * T::BN;

    // ---- loads.  A row's 128 bytes of a step lie as eight chunks of 16, XOR-ed with row / 2, so that the rows which an LDS read serves together cover all banks.
    // A load instruction fills eight rows, lane by lane; rows past the last one read that again.
    uint32_t a_off[NA], w_off[NW];
    auto row_of = [&](uint32_t block) __attribute__((always_inline)) { return 8u * block + (lane >> 3); };
    auto chunk_of = [&](uint32_t block) __attribute__((always_inline)) { return (lane & 7u) ^ ((block & 1u) << 2 | lane >> 4); };
#pragma unroll
    for (int j = 0; j < NA; ++j) a_off[j] = (min(m0 + row_of(wave * NA + j), g.M - 1u) - m0) * (uint32_t)g.a_row + 16u * chunk_of(wave * NA + j);
#pragma unroll
    for (int j = 0; j < NW; ++j) w_off[j] = (min(n0 + row_of(wave * NW + j), g.N - 1u) - n0) * (uint32_t)g.w_row + 16u * chunk_of(wave * NW + j);
    const char *ka = g.a + (int64_t)m0 * g.a_row, *kw = g.w + (int64_t)n0 * g.w_row;
    // a wavefront brings the scales of 64 rows or columns (some the same ones)
    const uint32_t part = wave % ((T::BM + T::BN) / 64), line = 64u * part + lane;
    const bool of_a = part < T::BM / 64;
    const float *scale = of_a ? g.a_scale + min(m0 + line, g.M - 1u) * g.a_scale_row : g.w_scale + min(n0 + line - T::BM, g.N - 1u) / 128u * g.w_scale_row;
    const int64_t scale_step = of_a ? g.a_scale_block : g.w_scale_block;
    const uint32_t steps = (g.K + 127u) / 128u, tail = g.K % 128u;
    uint32_t to_load = steps;
    auto issue = [&](uint32_t stage) __attribute__((always_inline)) {
        const uint32_t a_to = stage + wave * (NA * 1024u), w_to = stage + T::A + wave * (NW * 1024u);
        if (to_load > 1 || tail == 0) {
#pragma unroll
            for (int j = 0; j < NA; ++j) load_to_lds(ka, a_off[j], a_to + 1024u * j);
#pragma unroll
            for (int j = 0; j < NW; ++j) load_to_lds(kw, w_off[j], w_to + 1024u * j);
        } else {   // what lies behind the last k is nobody's: zeros
#pragma unroll
            for (int j = 0; j < NA; ++j) {
                if (16u * chunk_of(wave * NA + j) < tail)
                    load_to_lds(ka, a_off[j], a_to + 1024u * j);
                else
                    lds_write(a_to + 1024u * j + 16u * lane, u32x4{0, 0, 0, 0});
            }
#pragma unroll
            for (int j = 0; j < NW; ++j) {
                if (16u * chunk_of(wave * NW + j) < tail)
                    load_to_lds(kw, w_off[j], w_to + 1024u * j);
                else
                    lds_write(w_to + 1024u * j + 16u * lane, u32x4{0, 0, 0, 0});
            }
        }
        load_to_lds4(scale, stage + T::A + T::W + 256u * part);
        ka += 128;
        kw += 128;
        scale += scale_step;
        --to_load;
    };
    // the next step has landed, and every wavefront is done with what it read of the last stage.  (The last step's loads may be fewer: then all are waited for.)
    auto wait = [&]() __attribute__((always_inline)) {
        if constexpr (NST > 2) {
            if (to_load > 0) {
                landed<(NST - 2) * T::L>();
                return;
            }
        }
        landed<0>();
    };

    // ---- fragments: a lane has 32 bytes of one row, chunks `quarter` and quarter + 4.  Addresses of the stage that is read, and what lies in it at constant offsets
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
#pragma unroll
    for (int s = 0; s < NST; ++s)
        if ((uint32_t)s < steps) issue((uint32_t)s * T::STAGE);
    uint32_t cur = 0;
    landed<0>();
    turn_to(0);
    i32x8 fa[2], fw[TJ];
#pragma unroll
    for (int j = 0; j < TJ; ++j) fw[j] = fragment(r.w, r.w_far, j);
    fa[0] = fragment(r.a, r.a_far, 0);
    float sa = lds_read<float>(r.sa), sw = lds_read<float>(r.sw), s[2] = {0.f, 0.f};
    // Block sums wait for D - 1 further matrix instructions before they are added, so that nothing waits for them.
    constexpr int D = 3, Q = TI * TJ;
    f32x4 p[D];
#pragma unroll
    for (int d = 0; d < D; ++d) p[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto add = [&](int q) __attribute__((always_inline)) {
        const int i = q / TJ, j = q % TJ;
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(p[q % D][v], s[i & 1], acc[i][j][v]);
        asm volatile("" : "+v"(acc[i][j]));   // (else the additions gather behind the last of the matrix instructions, and the registers do not suffice)
    };
    static_assert(Q >= D, "");
    for (uint32_t left = steps; left > 0; --left) {
        const uint32_t next = cur + T::STAGE == T::LDS ? 0u : cur + T::STAGE;
        float next_sw = 0.f;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int i = q / TJ, j = q % TJ;
            if (j == 0) {
                if (i == TI - 1) {   // this stage is read: the step after those in LDS goes there
                    if (left > 1) wait();
                    if (to_load > 0) issue(cur);
                    turn_to(next);
                    next_sw = lds_read<float>(r.sw);   // (after the last step: a stale stage, read and unused)
                }
                s[i & 1] = sa * sw;
                fa[(i + 1) & 1] = fragment(r.a, r.a_far, (i + 1) % TI);
                sa = lds_read<float>(r.sa + 64u * ((i + 1) % TI));
            }
            p[q % D] = block_sums<T::EXACT>(fw[j], fa[i & 1]);
            __builtin_amdgcn_sched_barrier(0);
            if (i == TI - 1) fw[j] = fragment(r.w, r.w_far, j);
            if (q >= D - 1) add(q - (D - 1));
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int q = Q - (D - 1); q < Q; ++q) add(q);
        sw = next_sw;
        cur = next;
    }

    // ---- the wavefront's part through LDS, so that whole rows of it are stored: a lane holds four consecutive n of one m
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

template <class T>
hipError_t launch_tiles(ScaledArgs &g, hipStream_t s, bool &fits) {
    g.tiles_m = (g.M + T::BM - 1) / T::BM;
    g.tiles_n = (g.N + T::BN - 1) / T::BN;
    const uint64_t grid = (uint64_t)g.tiles_m * g.tiles_n, band = (uint64_t)kBand * g.tiles_n;
    fits = grid < 1u << 22 && band < 1u << 31;
    if (!fits) return hipSuccess;
    g.by_band = make_fastdiv((uint32_t)band);
    if (T::LDS > 65536) {
        static LdsReservation reserved;
        const hipError_t e = reserved.on_current_device({reinterpret_cast<const void *>(amap_gemm_scaled_tile_kernel<T>)}, T::LDS);
        if (e != hipSuccess) return e;
    }
    return launch_kernel<amap_gemm_scaled_tile_kernel<T>>(dim3((uint32_t)grid), dim3(64 * T::WAVES), T::LDS, s, g);
}

hipError_t launch_for(ScaledArgs &g, hipStream_t s, bool &fits) {
    const uint64_t large = (uint64_t)((g.M + 255) / 256) * ((g.N + 255) / 256), mid = (uint64_t)((g.M + 127) / 128) * ((g.N + 127) / 128);
    if (g.type == AMAP_F32) return mid >= 192 ? launch_tiles<Tile<128, 128, 2, 4, 2, true>>(g, s, fits) : launch_tiles<Tile<64, 64, 2, 2, 2, true>>(g, s, fits);
    if (large >= 192) return launch_tiles<Tile<256, 256, 2, 4, 2, false>>(g, s, fits);
    return mid >= 192 ? launch_tiles<Tile<128, 128, 2, 4, 2, false>>(g, s, fits) : launch_tiles<Tile<64, 64, 2, 2, 2, false>>(g, s, fits);
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
    const Box from = amap_rows_detail::box_of(*a, M, K), by = amap_rows_detail::box_of(*w, N, K), to = amap_rows_detail::box_of(*out, M, N),
              sa = amap_rows_detail::box_of(*a_scale, M, blocks_of(K)), sw = amap_rows_detail::box_of(*w_scale, blocks_of(N), blocks_of(K));
    if (!from.fits || !by.fits || !sa.fits || !sw.fits || !to.fits || !to.apart) return AMAP_E_SHAPE;
    if (meet(to, from) || meet(to, by) || meet(to, sa) || meet(to, sw)) return AMAP_E_ALIAS;
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
    const StreamDevice device(s);
    if (device.status() != hipSuccess) return launched(device.status(), "the stream's device");
    bool fits = true;
    const hipError_t e = launch_for(g, s, fits);
    return fits ? launched(e, "amap_gemm_scaled_tile_kernel") : refuse("too many tiles for one launch");
}
