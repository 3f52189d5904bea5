// The root mean square norm of rows with the residual's addition and the step to 8 bits (amap_norm), and its gradient (amap_norm_grad).
//
// A row is held in registers by 16, 32 or 64 lanes, or by a workgroup of up to 16 wavefronts, in pieces of 16 bytes: read once, its squares summed over the lanes (and, by way
// of LDS, over the wavefronts), scaled, written once.  Bound by the bytes: bf16 16391 rows of 4096 with the residual into 8 bits 77.6 us (472 MB, 6.1 TB/s; an identity copy reaches
// 6.0), 4111 x 40 heads of 128 inside their projection 15.0 us (84 MB, 5.6), 16 rows of 4096 4.1 us in the kernel, 5.6 a call.
// The gradient takes both of a row's sums (of h^2, and of grad weight h) in one pass.  Its columns' sums stay with the lanes that have the columns, workgroup by workgroup, and a second launch
// adds the workgroups' parts in their order, so that every call gives the same bits: 16384 rows of 4096 with `extra` 91.6 us (537 MB, 5.9 TB/s), 4.5 of them the second launch;
// fp32 1531 rows of 1001 11.6 to 12.2 us (3.5 of them the second launch).
#include <algorithm>

#include "amap_rows.hpp"

using namespace amap_rows_detail;
using namespace amap_detail;
using namespace amap_dev;

namespace {

constexpr int kMaxDim = 32768;
constexpr uint32_t kMaxWaves = 16;
constexpr uint32_t kHeldDim = 16384;   // rows whose gradient is made in registers

struct NormArgs {
    const char *x, *residual, *weight;
    char *total, *out;
    float *scale;
    int64_t x_token, x_head, residual_token, residual_head, total_token, total_head, out_token, out_head;   // bytes
    int64_t scale_row, scale_block;
    uint32_t rows, heads, dim, wide;   // wide: a weight of 32 bits
    FastDiv by_heads;
    float eps, inverse_dim;
};

// the sums of a workgroup's wavefronts, if a row is held by several: `part` has room for N of each
template <int N>
__device__ __forceinline__ void over_waves(float (&x)[N], float (*part)[N]) {
    const uint32_t waves = blockDim.x >> 6, wave = threadIdx.x >> 6;
    if (waves == 1) return;
    if ((threadIdx.x & 63u) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) part[wave][i] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = part[0][i];
    for (uint32_t w = 1; w < waves; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += part[w][i];
}

// LANES: that hold a row (64: a workgroup of whole wavefronts); U: pieces of a lane
template <class T, int LANES, int U, bool EIGHT, int PAST>
__global__ __launch_bounds__(LANES == 64 ? 64 * kMaxWaves : 256) void amap_norm_kernel(const NormArgs a) {
    constexpr int V = kPer<T>;
    __shared__ float part[kMaxWaves][1];
    const uint32_t lanes = LANES == 64 ? blockDim.x : LANES, lane = LANES == 64 ? threadIdx.x : threadIdx.x % LANES;
    uint32_t at_row = LANES == 64 ? blockIdx.x : blockIdx.x * (256u / LANES) + threadIdx.x / LANES;
    // Sixteen rows beside one another to one XCD (workgroups go round all eight): the scales of a column of blocks, which lie beside one another, leave its L2 as whole pieces
    // (16391 rows of 4096: 218 MB written without, 203.5 needed).
    if (EIGHT && LANES == 64 && (at_row | 127u) < a.rows) at_row = (at_row & ~127u) + (at_row & 7u) * 16u + (at_row >> 3 & 15u);
    const bool there = at_row < a.rows;
    const uint32_t row = there ? at_row : a.rows - 1u;   // (a group of lanes past the last row reads that again, and writes nothing)
    const uint32_t token = fdiv(row, a.by_heads), head = row - token * a.heads;
    const char *const x = a.x + token * a.x_token + head * a.x_head;
    u32x4 h[U];
#pragma unroll
    for (int u = 0; u < U; ++u) h[u] = load_piece<T, PAST>(x, (lane + u * lanes) * V, a.dim);
    if (a.residual) {
        const char *const r = a.residual + token * a.residual_token + head * a.residual_head;
        u32x4 more[U];
#pragma unroll
        for (int u = 0; u < U; ++u) more[u] = load_piece<T, PAST>(r, (lane + u * lanes) * V, a.dim);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float sum[V];
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] = element<T>(h[u], e) + element<T>(more[u], e);
            h[u] = piece_of<T>(sum);
        }
    }
    float squares[1] = {0.f};
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) squares[0] = __builtin_fmaf(element<T>(h[u], e), element<T>(h[u], e), squares[0]);
    squares[0] = sum_over<LANES>(squares[0]);
    if constexpr (LANES == 64) over_waves(squares, part);
    if (a.total && there) {
        char *const t = a.total + token * a.total_token + head * a.total_head;
#pragma unroll
        for (int u = 0; u < U; ++u) store_piece<T, PAST>(t, (lane + u * lanes) * V, a.dim, h[u]);
    }
    const float r = 1.f / __builtin_sqrtf(__builtin_fmaf(squares[0], a.inverse_dim, a.eps));
    char *const out = a.out + token * a.out_token + head * a.out_head;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t at = (lane + u * lanes) * V;
        float w[V], y[V];
        load_weight<T>(a.weight, a.wide, at, a.dim, w);
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = element<T>(h[u], e) * r * w[e];
        if constexpr (EIGHT) {
            const float scale = scale_of(most_over<kBlockLanes<T>>(most_of<V>(y)));
            uint32_t word[V / 4];
            eight_bits<V>(y, divisor_of(scale), word);
            if (there) {
                store_eight<V, PAST>(out, at, a.dim, word);
                if (lane % kBlockLanes<T> == 0 && at < a.dim) a.scale[token * a.scale_row + (int64_t)(at / kBlock) * a.scale_block] = scale;
            }
        } else {
            if (there) store_piece<T, PAST>(out, at, a.dim, piece_of<T>(y));
        }
    }
}

// ---- the gradient

struct GradArgs {
    const char *x, *grad, *extra, *weight;
    char *dx;
    float *dw;                 // of workgroup i: dw + i * pitch
    int64_t x_token, x_head, grad_token, grad_head, extra_token, extra_head, dx_token, dx_head;   // bytes
    uint32_t rows, heads, dim, wide, pitch;
    FastDiv by_heads;
    float eps, inverse_dim;
};

// where a row lies
struct Place {
    const char *x, *grad, *extra;
    char *dx;
};
__device__ __forceinline__ Place place_of(const GradArgs &a, uint32_t row) {
    const uint32_t token = fdiv(row, a.by_heads), head = row - token * a.heads;
    return Place{a.x + token * a.x_token + head * a.x_head, a.grad + token * a.grad_token + head * a.grad_head,
                 a.extra ? a.extra + token * a.extra_token + head * a.extra_head : nullptr, a.dx + token * a.dx_token + head * a.dx_head};
}

// A group of LANES takes row after row; what each adds to the weight's gradient stays with the lane that has the column.
template <class T, int LANES, int U, int PAST>
__global__ __launch_bounds__(LANES == 64 ? 64 * kMaxWaves : 256) void amap_norm_grad_kernel(const GradArgs a) {
    constexpr int V = kPer<T>;
    constexpr uint32_t kGroups = LANES == 64 ? 1u : 256u / LANES;
    __shared__ float part[2][kMaxWaves][2];
    extern __shared__ float column[];   // [kGroups][LANES * V], LANES < 64
    const uint32_t lanes = LANES == 64 ? blockDim.x : LANES, lane = LANES == 64 ? threadIdx.x : threadIdx.x % LANES;
    const uint32_t group = LANES == 64 ? 0u : threadIdx.x / LANES;
    float w[U][V], dw[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        load_weight<T>(a.weight, a.wide, (lane + u * lanes) * V, a.dim, w[u]);
#pragma unroll
        for (int e = 0; e < V; ++e) dw[u][e] = 0.f;
    }
    struct Row {
        u32x4 h[U], g[U], more[U];
    };
    auto load = [&](const Place &at) __attribute__((always_inline)) {
        Row x;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x.h[u] = load_piece<T, PAST>(at.x, (lane + u * lanes) * V, a.dim);
            x.g[u] = load_piece<T, PAST>(at.grad, (lane + u * lanes) * V, a.dim);
        }
        if (at.extra) {
#pragma unroll
            for (int u = 0; u < U; ++u) x.more[u] = load_piece<T, PAST>(at.extra, (lane + u * lanes) * V, a.dim);
        }
        return x;
    };
    // where there is room for it the next row is on its way while one is worked on
    constexpr bool AHEAD = U == 1;
    uint32_t turn = 0, first = blockIdx.x * kGroups;   // (every workgroup has rows)
    Place at = place_of(a, min(first + group, a.rows - 1u));
    Row row;
    if constexpr (AHEAD) row = load(at);
    for (; first < a.rows; first += gridDim.x * kGroups, turn ^= 1u) {
        const bool there = first + group < a.rows;
        const uint32_t next = first + gridDim.x * kGroups;
        Row now;
        Place place = at;
        if constexpr (AHEAD) {
            now = row;
            if (next < a.rows) {
                at = place_of(a, min(next + group, a.rows - 1u));
                row = load(at);
            }
        } else {
            now = load(at);
            if (next < a.rows) at = place_of(a, min(next + group, a.rows - 1u));
        }
        const u32x4(&h)[U] = now.h, (&g)[U] = now.g, (&more)[U] = now.more;
        float sums[2] = {0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float f = element<T>(h[u], e);
                sums[0] = __builtin_fmaf(f, f, sums[0]);
                sums[1] = __builtin_fmaf(element<T>(g[u], e) * w[u][e], f, sums[1]);
            }
        sums[0] = sum_over<LANES>(sums[0]);
        sums[1] = sum_over<LANES>(sums[1]);
        if constexpr (LANES == 64) over_waves(sums, part[turn]);   // (two sets: whoever writes this one again has met all who read it at the other's barrier)
        // (r^2 by itself may pass 32 bits: a row of zeros, or nearly, and eps below 3e-39)
        const float r = 1.f / __builtin_sqrtf(__builtin_fmaf(sums[0], a.inverse_dim, a.eps)), along = sums[1] * a.inverse_dim * r * r;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float d[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float f = element<T>(h[u], e), ge = element<T>(g[u], e);
                d[e] = r * __builtin_fmaf(-f, along, ge * w[u][e]);
                if (place.extra) d[e] += element<T>(more[u], e);
                if (there) dw[u][e] = __builtin_fmaf(ge, f * r, dw[u][e]);   // (h r is at most the root of the row's length; grad h has no such bound)
            }
            if (there) store_piece<T, PAST>(place.dx, (lane + u * lanes) * V, a.dim, piece_of<T>(d));
        }
    }
    if constexpr (LANES < 64) {   // the groups' sums in their order
        static_assert(U == 1, "a group's columns");
#pragma unroll
        for (int e = 0; e < V; ++e) column[(group * LANES + lane) * V + e] = dw[0][e];
        __syncthreads();
        if (group != 0) return;
#pragma unroll 1
        for (uint32_t k = 1; k < kGroups; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) dw[0][e] += column[(k * LANES + lane) * V + e];
    }
    float *const to = a.dw + (size_t)blockIdx.x * a.pitch;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const uint32_t c = (lane + u * lanes) * V + e;
            if (c < a.dim) to[c] = dw[u][e];
        }
}

// The same for rows of more than 16 elements to a lane of sixteen wavefronts: a row is read twice (the second time out of the caches), and the columns' sums are
// kept in LDS, each by the lane that has its column.  Bound by one workgroup to a compute unit, which reads, sums and meets before it writes: bf16 3000 rows of 20000 135.5 us (360 MB, 2.7 TB/s),
// of 32768 218 (590 MB, 2.7); fp32 2000 rows of 20000 with `extra` 166 (640 MB, 3.9).
template <class T>
__global__ __launch_bounds__(64 * kMaxWaves) void amap_norm_grad_wide_kernel(const GradArgs a) {
    constexpr int V = kPer<T>;
    __shared__ float part[2][kMaxWaves][2];
    extern __shared__ float column[];   // [whole pieces of a row]
    for (uint32_t c = threadIdx.x * V; c < a.dim; c += blockDim.x * V)
#pragma unroll
        for (int e = 0; e < V; ++e) column[c + e] = 0.f;
    uint32_t turn = 0;
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1u) {
        const Place at = place_of(a, row);
        float sums[2] = {0.f, 0.f};
        for (uint32_t c = threadIdx.x * V; c < a.dim; c += blockDim.x * V) {
            const u32x4 h = load_piece<T>(at.x, c, a.dim), g = load_piece<T>(at.grad, c, a.dim);
            float w[V];
            load_weight<T>(a.weight, a.wide, c, a.dim, w);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float f = element<T>(h, e);
                sums[0] = __builtin_fmaf(f, f, sums[0]);
                sums[1] = __builtin_fmaf(element<T>(g, e) * w[e], f, sums[1]);
            }
        }
        sums[0] = sum_over<64>(sums[0]);
        sums[1] = sum_over<64>(sums[1]);
        over_waves(sums, part[turn]);
        const float r = 1.f / __builtin_sqrtf(__builtin_fmaf(sums[0], a.inverse_dim, a.eps)), along = sums[1] * a.inverse_dim * r * r;
        for (uint32_t c = threadIdx.x * V; c < a.dim; c += blockDim.x * V) {   // (dx may be any of the rows that are read: a lane has read its piece before it writes there)
            const u32x4 h = load_piece<T>(at.x, c, a.dim), g = load_piece<T>(at.grad, c, a.dim);
            u32x4 more = {0, 0, 0, 0};
            if (at.extra) more = load_piece<T>(at.extra, c, a.dim);
            float w[V], d[V];
            load_weight<T>(a.weight, a.wide, c, a.dim, w);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float f = element<T>(h, e), ge = element<T>(g, e);
                d[e] = r * __builtin_fmaf(-f, along, ge * w[e]);
                if (at.extra) d[e] += element<T>(more, e);
                column[c + e] = __builtin_fmaf(ge, f * r, column[c + e]);
            }
            store_piece<T>(at.dx, c, a.dim, piece_of<T>(d));
        }
    }
    float *const to = a.dw + (size_t)blockIdx.x * a.pitch;
    for (uint32_t c = threadIdx.x * V; c < a.dim; c += blockDim.x * V)
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < a.dim) to[c + e] = column[c + e];
}

// dweight = the sum of the workgroups' parts, in their order: four lanes of four columns, 64 sets of parts
__global__ __launch_bounds__(256) void amap_norm_join_kernel(const float *parts, uint32_t count, uint32_t pitch, uint32_t dim, float *dw) {
    __shared__ float sums[64][16];
    const uint32_t lane = threadIdx.x & 3u, set = threadIdx.x >> 2, at = blockIdx.x * 16u + 4u * lane;
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (at < dim) {   // (parts are whole fours of columns wide)
        constexpr uint32_t U = 4;   // on their way at once
        const char *const from = reinterpret_cast<const char *>(parts + at);
        for (uint32_t i = set; i < count; i += 64 * U) {
            f32x4 x[U];
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) x[u] = i + 64 * u < count ? *reinterpret_cast<const f32x4 *>(from + (size_t)(i + 64 * u) * pitch * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (uint32_t u = 0; u < U; ++u) sum += x[u];
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[set][4 * lane + e] = sum[e];
    __syncthreads();
    // 16 lanes to a column, four sets each
    const uint32_t column = threadIdx.x >> 4, first = threadIdx.x & 15u;
    float x = (sums[first][column] + sums[first + 16][column]) + (sums[first + 32][column] + sums[first + 48][column]);
    x = sum_over<16>(x);
    if (first == 0 && blockIdx.x * 16u + column < dim) dw[blockIdx.x * 16u + column] = x;
}

// ---- host

// How a row is held: by so many lanes, in so many pieces each.
struct Held {
    uint32_t lanes, threads, each, grid;   // threads: of a workgroup
};
Held held(uint64_t rows, uint32_t dim, int per, bool eight, uint32_t most_each) {
    const uint32_t pieces = (dim + per - 1) / per, least = eight ? (uint32_t)(kBlock / per) : 16u;
    Held h = {64, 64, 1, 0};
    if (pieces <= 32) {
        h.lanes = pieces <= 16 && least <= 16 ? 16 : 32;
        h.threads = 256;
        h.grid = (uint32_t)((rows * h.lanes + 255) / 256);
        return h;
    }
    // Few rows by as many lanes as there are pieces, many by lanes of several: the norm, us by pieces of a lane, bf16 16391 rows of 4096 with residual into 8 bits 1 83.3, 2 78.4, 4 78.2,
    // 2048 rows 1 13.5, 2 12.6, 4 13.3, 60000 rows of 1000 alone 1 44.5, 2 41.0, 4 44.9; fp32 3000 rows of 4096 1 18.1, 2 16.5, 4 16.3, 8 17.1.
    h.each = most_each;
    while (h.each > 1 && (uint64_t)rows * ((pieces + 64 * h.each - 1) / (64 * h.each)) < 4096) h.each /= 2;
    while ((pieces + 64 * h.each - 1) / (64 * h.each) > kMaxWaves) h.each *= 2;
    h.threads = (pieces + 64 * h.each - 1) / (64 * h.each) * 64;
    h.grid = (uint32_t)rows;
    return h;
}

template <class T, bool EIGHT, int PAST>
hipError_t norm_by(const Held &h, const NormArgs &g, hipStream_t s) {
    const dim3 grid(h.grid), threads(h.threads);
    if constexpr (kBlockLanes<T> == 16 || !EIGHT)
        if (h.lanes == 16) return launch_kernel<amap_norm_kernel<T, 16, 1, EIGHT, PAST>>(grid, threads, 0, s, g);
    if (h.lanes == 32) return launch_kernel<amap_norm_kernel<T, 32, 1, EIGHT, PAST>>(grid, threads, 0, s, g);
    if (h.each == 1) return launch_kernel<amap_norm_kernel<T, 64, 1, EIGHT, PAST>>(grid, threads, 0, s, g);
    if (h.each == 2) return launch_kernel<amap_norm_kernel<T, 64, 2, EIGHT, PAST>>(grid, threads, 0, s, g);
    if constexpr (T::bytes == 4)
        if (h.each == 8) return launch_kernel<amap_norm_kernel<T, 64, 8, EIGHT, PAST>>(grid, threads, 0, s, g);
    return launch_kernel<amap_norm_kernel<T, 64, 4, EIGHT, PAST>>(grid, threads, 0, s, g);
}
template <class T>
hipError_t norm_of(const Held &h, const NormArgs &g, hipStream_t s) {
    const bool eight = g.scale != nullptr;
    const int each = eight ? 1 : T::bytes;
    const uint64_t stored = reinterpret_cast<uintptr_t>(g.out) | (uint64_t)g.out_token | (uint64_t)g.out_head | g.dim * (uint64_t)each |
                            (g.total ? reinterpret_cast<uintptr_t>(g.total) | (uint64_t)g.total_token | (uint64_t)g.total_head : 0u);
    const int past = past_caches((uint64_t)g.rows * g.dim * (T::bytes * (1 + (g.residual != nullptr) + (g.total != nullptr)) + each), stored);
    if (eight) return past == kBoth ? norm_by<T, true, kBoth>(h, g, s) : past == kStores ? norm_by<T, true, kStores>(h, g, s) : norm_by<T, true, kThrough>(h, g, s);
    return past == kBoth ? norm_by<T, false, kBoth>(h, g, s) : past == kStores ? norm_by<T, false, kStores>(h, g, s) : norm_by<T, false, kThrough>(h, g, s);
}
template <class T, int PAST>
hipError_t grad_by(const Held &h, const GradArgs &g, hipStream_t s) {
    const dim3 grid(h.grid), threads(h.threads);
    constexpr uint32_t lds = 256 * kPer<T> * 4;
    if (g.dim > kHeldDim) {
        static LdsReservation reserved;
        const hipError_t e = reserved.on_current_device({reinterpret_cast<const void *>(amap_norm_grad_wide_kernel<T>)}, kMaxDim * 4);
        if (e != hipSuccess) return e;
        return launch_kernel<amap_norm_grad_wide_kernel<T>>(grid, threads, (g.dim + kPer<T> - 1) / kPer<T> * kPer<T> * 4u, s, g);
    }
    if (h.lanes == 16) return launch_kernel<amap_norm_grad_kernel<T, 16, 1, PAST>>(grid, threads, lds, s, g);
    if (h.lanes == 32) return launch_kernel<amap_norm_grad_kernel<T, 32, 1, PAST>>(grid, threads, lds, s, g);
    if (h.each == 1) return launch_kernel<amap_norm_grad_kernel<T, 64, 1, PAST>>(grid, threads, 0, s, g);
    if constexpr (T::bytes == 4)
        if (h.each == 4) return launch_kernel<amap_norm_grad_kernel<T, 64, 4, PAST>>(grid, threads, 0, s, g);
    return launch_kernel<amap_norm_grad_kernel<T, 64, 2, PAST>>(grid, threads, 0, s, g);
}
template <class T>
hipError_t grad_of(const Held &h, const GradArgs &g, hipStream_t s) {
    const uint64_t stored = reinterpret_cast<uintptr_t>(g.dx) | (uint64_t)g.dx_token | (uint64_t)g.dx_head | (uint64_t)g.dim * T::bytes;
    const int past = past_caches((uint64_t)g.rows * g.dim * T::bytes * (g.extra ? 4 : 3), stored);
    return past == kBoth ? grad_by<T, kBoth>(h, g, s) : past == kStores ? grad_by<T, kStores>(h, g, s) : grad_by<T, kThrough>(h, g, s);
}

bool same_rows(const amap_heads &a, const amap_heads &b, int64_t tokens) {
    return a.data == b.data && a.type == b.type && (tokens <= 1 || a.token_stride == b.token_stride) && (a.heads <= 1 || a.head_stride == b.head_stride);
}
// (rows of one head each: of any types)
bool share_any(const amap_heads &a, const amap_heads &b, int64_t tokens, int dim) {
    return a.heads == 1 && b.heads == 1 ? share(runs_of(a, tokens, dim), runs_of(b, tokens, dim)) : share(a, b, tokens, dim);
}
// what is written may be the very rows of what is read, or share nothing with it
bool clash(const amap_heads &written, const amap_heads *read, int64_t tokens, int dim) {
    return read && !same_rows(written, *read, tokens) && share_any(written, *read, tokens, dim);
}
amap_status check_rows(const amap_heads *h, const amap_heads *like, int64_t tokens, int dim, bool written) {
    if (!h->data || h->type != like->type) return AMAP_E_INVALID;
    if (h->heads != like->heads) return AMAP_E_SHAPE;
    const Box b = amap_cache_detail::box_of(*h, tokens, dim);
    return b.fits && (!written || b.apart) ? AMAP_OK : AMAP_E_SHAPE;
}
amap_status check_sizes(const amap_heads *x, int64_t tokens, int dim, const void *weight, amap_type weight_type, float eps) {
    if (!x || tokens < 0 || dim < 1 || x->heads < 1 || !is_wide(x->type) || !weight || (weight_type != x->type && weight_type != AMAP_F32)) return AMAP_E_INVALID;
    if (!(eps > 0.f) || eps > 3.4e38f) return AMAP_E_INVALID;
    if (dim > kMaxDim) return refuse("rows of more than 32768 elements");
    int64_t rows;
    return __builtin_mul_overflow(tokens, (int64_t)x->heads, &rows) || rows > INT32_MAX ? AMAP_E_SHAPE : AMAP_OK;
}
bool whole_elements(const amap_heads *h) { return !h || reinterpret_cast<uintptr_t>(h->data) % bytes_of(h->type) == 0; }
const char *const kBegins = "a tensor that does not begin at a whole element";

// Workgroups of the gradient's first launch, each of which leaves one part of the weight's: three rows (or groups of them) to each, up to eight wavefronts to a compute unit.
// us by workgroups, rows of 4096 in bf16: 512 rows 128 13.4, 256 13.6, 512 17.0   2048 rows 128 28, 256 21.0, 512 22.4   16384 rows 256 97, 512 105, 1024 110;
// 32768 rows of 1024 512 71.6, 768 57.2, 1024 53.7.  Up to four are left to one workgroup, whose part is the whole: no second launch.
uint32_t grad_grid(const Held &h) {
    const uint32_t waves = h.threads / 64, most = std::max(256u, 2048 / waves);
    return h.grid <= 4 ? std::min(h.grid, 1u) : std::min(most, (h.grid + 2) / 3);
}
uint32_t grad_pitch(int dim) { return ((uint32_t)dim + 3u) / 4u * 4u; }
Held grad_held(int heads, int64_t tokens, int dim, amap_type type) {
    // one piece to a lane as long as sixteen wavefronts hold a row so: the next row is on its way then (16384 rows of 4096 97 us, by two pieces 105; 32768 of 1024 53.7 and 62)
    Held h = held((uint64_t)tokens * heads, (uint32_t)dim, 16 / bytes_of(type), false, 1);
    if (dim > (int)kHeldDim) h = Held{64, 64 * kMaxWaves, 1, (uint32_t)(tokens * heads)};
    h.grid = grad_grid(h);
    return h;
}

}  // namespace

extern "C" amap_status amap_norm(const amap_heads *x, const amap_heads *residual, int64_t tokens, int head_dim, const void *weight, amap_type weight_type, float eps,
                                 const amap_heads *total, const amap_heads *out, const amap_scales *scale, void *stream) {
    if (!out || (total && !residual)) return AMAP_E_INVALID;
    amap_status st = check_sizes(x, tokens, head_dim, weight, weight_type, eps);
    if (st != AMAP_OK) return st;
    const bool eight = out->type == AMAP_E4M3;
    if (eight != (scale != nullptr) || (!eight && out->type != x->type)) return AMAP_E_INVALID;
    if (eight && x->heads != 1) return refuse("8 bits of rows of several heads");
    if (tokens == 0) return AMAP_OK;
    if (!x->data || !out->data || (eight && !scale->data)) return AMAP_E_INVALID;
    st = check_rows(x, x, tokens, head_dim, false);
    if (st == AMAP_OK && residual) st = check_rows(residual, x, tokens, head_dim, false);
    if (st == AMAP_OK && total) st = check_rows(total, x, tokens, head_dim, true);
    if (st == AMAP_OK) st = check_rows(out, eight ? out : x, tokens, head_dim, true);
    if (st == AMAP_OK && out->heads != x->heads) st = AMAP_E_SHAPE;
    if (st != AMAP_OK) return st;
    const Box to = amap_cache_detail::box_of(*out, tokens, head_dim), w = amap_cache_detail::box_of(weight, (int64_t)head_dim * bytes_of(weight_type));
    const Box sum = total ? amap_cache_detail::box_of(*total, tokens, head_dim) : Box{};
    if (clash(*out, x, tokens, head_dim) || clash(*out, residual, tokens, head_dim) || meet(to, w) || meet(sum, w)) return AMAP_E_ALIAS;
    if (total && (clash(*total, x, tokens, head_dim) || clash(*total, residual, tokens, head_dim) || share_any(*out, *total, tokens, head_dim))) return AMAP_E_ALIAS;
    if (eight) {
        const Runs s = runs_of(*scale, tokens, blocks_of(head_dim));
        if (!s.box.fits || !s.box.apart) return AMAP_E_SHAPE;
        if (meet(s.box, w) || share(s, runs_of(*out, tokens, head_dim)) || (total && share(s, runs_of(*total, tokens, head_dim))) || share(s, runs_of(*x, tokens, head_dim)) ||
            (residual && share(s, runs_of(*residual, tokens, head_dim))))
            return AMAP_E_ALIAS;
        if (reinterpret_cast<uintptr_t>(scale->data) % 4) return refuse(kBegins);
    }
    if (!whole_elements(x) || !whole_elements(residual) || !whole_elements(total) || !whole_elements(out) || reinterpret_cast<uintptr_t>(weight) % bytes_of(weight_type))
        return refuse(kBegins);
    const int es = bytes_of(x->type);
    NormArgs g = {};
    g.x = static_cast<const char *>(x->data);
    g.x_token = x->token_stride * es, g.x_head = x->head_stride * es;
    if (residual) {
        g.residual = static_cast<const char *>(residual->data);
        g.residual_token = residual->token_stride * es, g.residual_head = residual->head_stride * es;
    }
    if (total) {
        g.total = static_cast<char *>(total->data);
        g.total_token = total->token_stride * es, g.total_head = total->head_stride * es;
    }
    g.out = static_cast<char *>(out->data);
    g.out_token = out->token_stride * (eight ? 1 : es), g.out_head = out->head_stride * (eight ? 1 : es);
    if (eight) g.scale = scale->data, g.scale_row = scale->row_stride, g.scale_block = scale->block_stride;
    g.weight = static_cast<const char *>(weight);
    g.wide = weight_type == AMAP_F32;
    g.rows = (uint32_t)(tokens * x->heads);
    g.heads = (uint32_t)x->heads;
    g.by_heads = make_fastdiv(g.heads);
    g.dim = (uint32_t)head_dim;
    g.eps = eps;
    g.inverse_dim = 1.f / (float)head_dim;
    const Held h = held(g.rows, g.dim, 16 / es, eight, x->type == AMAP_F32 ? 4 : 2);
    if ((uint64_t)h.grid * h.threads >> 32) return refuse("too many rows for one launch");
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const StreamDevice device(s);
    if (device.status() != hipSuccess) return launched(device.status(), "the stream's device");
    const hipError_t e = x->type == AMAP_F32 ? norm_of<F32>(h, g, s) : x->type == AMAP_BF16 ? norm_of<Bf16>(h, g, s) : norm_of<F16>(h, g, s);
    return launched(e, "amap_norm_kernel");
}

extern "C" amap_status amap_norm_grad_workspace(int heads, int64_t tokens, int head_dim, amap_type type, int64_t *bytes) {
    if (!bytes || heads < 1 || tokens < 0 || head_dim < 1 || !is_wide(type)) return AMAP_E_INVALID;
    if (head_dim > kMaxDim) return refuse("rows of more than 32768 elements");
    if (tokens > INT32_MAX / heads) return AMAP_E_SHAPE;
    const uint32_t grid = tokens ? grad_held(heads, tokens, head_dim, type).grid : 0;
    *bytes = grid <= 1 ? 0 : (int64_t)grid * grad_pitch(head_dim) * 4;   // (one workgroup's part is the whole)
    return AMAP_OK;
}

extern "C" amap_status amap_norm_grad(const amap_heads *x, int64_t tokens, int head_dim, const void *weight, amap_type weight_type, float eps, const amap_heads *grad,
                                      const amap_heads *extra, const amap_heads *dx, float *dweight, void *workspace, int64_t workspace_bytes, void *stream) {
    if (!grad || !dx || !dweight) return AMAP_E_INVALID;
    amap_status st = check_sizes(x, tokens, head_dim, weight, weight_type, eps);
    if (st != AMAP_OK) return st;
    const Box dw = amap_cache_detail::box_of(dweight, (int64_t)head_dim * 4), w = amap_cache_detail::box_of(weight, (int64_t)head_dim * bytes_of(weight_type));
    if (reinterpret_cast<uintptr_t>(dweight) % 4 || reinterpret_cast<uintptr_t>(weight) % bytes_of(weight_type)) return refuse(kBegins);
    if (meet(dw, w)) return AMAP_E_ALIAS;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    GradArgs g = {};
    Held h = {};
    g.pitch = grad_pitch(head_dim);
    if (tokens > 0) {
        if (!x->data) return AMAP_E_INVALID;
        st = check_rows(x, x, tokens, head_dim, false);
        if (st == AMAP_OK) st = check_rows(grad, x, tokens, head_dim, false);
        if (st == AMAP_OK && extra) st = check_rows(extra, x, tokens, head_dim, false);
        if (st == AMAP_OK) st = check_rows(dx, x, tokens, head_dim, true);
        if (st != AMAP_OK) return st;
        if (!whole_elements(x) || !whole_elements(grad) || !whole_elements(extra) || !whole_elements(dx)) return refuse(kBegins);
        const Box box[4] = {amap_cache_detail::box_of(*x, tokens, head_dim), amap_cache_detail::box_of(*grad, tokens, head_dim),
                            extra ? amap_cache_detail::box_of(*extra, tokens, head_dim) : Box{}, amap_cache_detail::box_of(*dx, tokens, head_dim)};
        if (clash(*dx, x, tokens, head_dim) || clash(*dx, grad, tokens, head_dim) || clash(*dx, extra, tokens, head_dim) || meet(box[3], w)) return AMAP_E_ALIAS;
        for (const Box &b : box)
            if (meet(dw, b)) return AMAP_E_ALIAS;
        h = grad_held(x->heads, tokens, head_dim, x->type);
        if (h.grid > 1) {
            const int64_t need = (int64_t)h.grid * g.pitch * 4;
            if (!workspace || workspace_bytes < need) return AMAP_E_INVALID;
            if (reinterpret_cast<uintptr_t>(workspace) % 16) return refuse("a workspace that does not begin at a multiple of 16 bytes");
            const Box room = amap_cache_detail::box_of(workspace, need);
            for (const Box &b : box)
                if (meet(room, b)) return AMAP_E_ALIAS;
            if (meet(room, dw) || meet(room, w)) return AMAP_E_ALIAS;
        }
        const int es = bytes_of(x->type);
        g.x = static_cast<const char *>(x->data);
        g.x_token = x->token_stride * es, g.x_head = x->head_stride * es;
        g.grad = static_cast<const char *>(grad->data);
        g.grad_token = grad->token_stride * es, g.grad_head = grad->head_stride * es;
        if (extra) {
            g.extra = static_cast<const char *>(extra->data);
            g.extra_token = extra->token_stride * es, g.extra_head = extra->head_stride * es;
        }
        g.dx = static_cast<char *>(dx->data);
        g.dx_token = dx->token_stride * es, g.dx_head = dx->head_stride * es;
        g.weight = static_cast<const char *>(weight);
        g.wide = weight_type == AMAP_F32;
        g.rows = (uint32_t)(tokens * x->heads);
        g.heads = (uint32_t)x->heads;
        g.by_heads = make_fastdiv(g.heads);
        g.dim = (uint32_t)head_dim;
        g.eps = eps;
        g.inverse_dim = 1.f / (float)head_dim;
        g.dw = h.grid > 1 ? static_cast<float *>(workspace) : dweight;
    }
    const StreamDevice device(s);
    if (device.status() != hipSuccess) return launched(device.status(), "the stream's device");
    if (tokens > 0) {
        const hipError_t e = x->type == AMAP_F32 ? grad_of<F32>(h, g, s) : x->type == AMAP_BF16 ? grad_of<Bf16>(h, g, s) : grad_of<F16>(h, g, s);
        if (e != hipSuccess) return launched(e, "amap_norm_grad_kernel");
        if (h.grid == 1) return AMAP_OK;
    }
    const hipError_t e = launch_kernel<amap_norm_join_kernel>(dim3(((uint32_t)head_dim + 15u) / 16u), dim3(256), 0, s, static_cast<const float *>(workspace), h.grid, g.pitch,
                                                              (uint32_t)head_dim, dweight);
    return launched(e, "amap_norm_join_kernel");
}
