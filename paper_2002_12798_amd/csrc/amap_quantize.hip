// Rows and weights into 8 bits with a scale for each block (amap_quantize): every block is read once, held in registers while the lanes that hold it
// agree on its largest value, and written once.  Bound by the bytes: bf16 8192 x 10240 behind a gate 66 to 67 us (422 MB, 6.3 TB/s; the vector
// units are at work in 95 % of the cycles), 6100 x 4080 by 128 rows 14.4 us (75 MB, 5.2), 64 x 2560 3.2 us in the kernel, 4.6 to 5.2 a call.
#include "amap_rows.hpp"

using namespace amap_rows_detail;
using namespace amap_detail;
using namespace amap_dev;

namespace {

constexpr int kThreads = 256;

struct QuantizeArgs {
    const char *x, *gate;
    char *out;
    float *scale;
    int64_t x_row, gate_row, out_row;   // bytes
    int64_t scale_row, scale_block;
    uint32_t rows, columns, across;     // across: workgroups along a row
    FastDiv by_across;
    bool neighbours;   // blocks beside one another to one XCD
};

// gate / (1 + exp(-gate)) * x.  The exponential's argument, the gate over ln 2, is carried in two parts, so that the power of two has 32 bits whatever the gate.
// In the order x / (1 + exp(-gate)) * gate no step leaves the range of 32 bits that the value does not leave: from gates of -69 on, where the quotient is at least 2^-100 of x.
// (The gate enters the exponential as -69 to 200: below that as below, above it the sum is 1 from 18 on.)
constexpr float kInverseLn2 = 0x1.715476p+0f, kInverseLn2Rest = 0x1.4ae0bf8p-26f, kLn2 = 0x1.62e43p-1f, kLowGate = -69.f;
__device__ __forceinline__ float gated(float gate, float x) {
    const float g = __builtin_amdgcn_fmed3f(gate, kLowGate, 200.f), t = g * -kInverseLn2;
    const float rest = __builtin_fmaf(g, -kInverseLn2Rest, __builtin_fmaf(g, -kInverseLn2, -t));
    float e = __builtin_amdgcn_exp2f(t);
    e = __builtin_fmaf(e, rest * kLn2, e);
    return x * __builtin_amdgcn_rcpf(1.f + e) * gate;
}
// The same for gates below -69, where the sum is the exponential itself: exp(gate) as a power of two times a factor of 0.7 to 1.4, so that it may lie far below what 32 bits hold and the
// value still be an ordinary number.  (Below -400 no x leaves anything.)
__device__ __forceinline__ float low_gated(float gate, float x) {
    const float g = fmaxf(gate, -400.f), n = __builtin_rintf(g * kInverseLn2);
    const float f = __builtin_fmaf(g, kInverseLn2Rest, __builtin_fmaf(g, kInverseLn2, -n));
    return __builtin_ldexpf(x, (int)n) * __builtin_amdgcn_exp2f(f) * gate;
}

// Blocks of one row: a block to as many lanes as it has pieces, U blocks beside one another for each of them; the rows of a workgroup follow one another, so that
// the scales of a column of blocks are written beside one another.
template <class T, bool GATE, int U, int PAST>
__global__ __launch_bounds__(kThreads) void amap_quantize_kernel(const QuantizeArgs a) {
    constexpr int V = kPer<T>, L = kBlockLanes<T>;
    constexpr uint32_t kRows = kThreads / L;
    const uint32_t block = a.neighbours ? xcd_remap(blockIdx.x, gridDim.x) : blockIdx.x;
    const uint32_t down = fdiv(block, a.by_across), across = block - down * a.across;
    const uint32_t lane = threadIdx.x % L, row = down * kRows + threadIdx.x / L;
    if (row >= a.rows) return;   // (whole groups of lanes)
    // (from the workgroup's first column on)
    const uint32_t column = across * (U * kBlock), left = min(a.columns - column, (uint32_t)(U * kBlock)), first = lane * V;
    const char *const x = a.x + row * a.x_row + (size_t)column * T::bytes, *const gate = GATE ? a.gate + row * a.gate_row + (size_t)column * T::bytes : nullptr;
    char *const out = a.out + row * a.out_row + column;
    u32x4 p[U], q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        p[u] = load_piece<T, PAST>(x, first + u * kBlock, left);
        if constexpr (GATE) q[u] = load_piece<T, PAST>(gate, first + u * kBlock, left);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t at = first + u * kBlock;
        float y[V], least = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            y[e] = element<T>(p[u], e);
            if constexpr (GATE) {
                const float gate = element<T>(q[u], e);
                least = fminf(least, gate);
                y[e] = gated(gate, y[e]);
            }
        }
        if (GATE && least < kLowGate) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float gate = element<T>(q[u], e);
                if (gate < kLowGate) y[e] = low_gated(gate, element<T>(p[u], e));
            }
        }
        float most;
        if constexpr (GATE)
            most = most_of<V>(y);
        else
            most = most_of<T, 1>({p[u]});
        const float scale = scale_of(most_over<L>(most));
        uint32_t word[V / 4];
        eight_bits<V>(y, divisor_of(scale), word);
        store_eight<V, PAST>(out, at, left, word);
        if (lane == 0 && at < left) a.scale[row * a.scale_row + (int64_t)(across * U + u) * a.scale_block] = scale;
    }
}

// Blocks of 128 rows: one to a workgroup.
template <class T, int PAST>
__global__ __launch_bounds__(kThreads) void amap_quantize_tall_kernel(const QuantizeArgs a) {
    constexpr int V = kPer<T>, L = kBlockLanes<T>, kRows = kThreads / L, U = kBlock / kRows;
    __shared__ float part[kThreads / 64];
    const uint32_t block = a.neighbours ? xcd_remap(blockIdx.x, gridDim.x) : blockIdx.x;
    const uint32_t down = fdiv(block, a.by_across), across = block - down * a.across;
    const uint32_t column = across * kBlock, left = min(a.columns - column, (uint32_t)kBlock), at = threadIdx.x % L * V, first = down * kBlock + threadIdx.x / L;
    const char *const x = a.x + (size_t)column * T::bytes;
    u32x4 p[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t row = first + u * kRows;
        p[u] = load_piece<T, PAST>(x + row * a.x_row, row < a.rows ? at : left, left);
    }
    float most = most_over<64>(most_of<T>(p));
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) most = fmaxf(most, part[w]);
#pragma unroll
    for (int u = 0; u < U; ++u) asm volatile("" : "+v"(p[u]));   // (else the elements stay in 32 bits: 84 registers of bf16, and five workgroups to a compute unit instead of eight)
    const float scale = scale_of(most);
    const Divisor by = divisor_of(scale);
    if (threadIdx.x == 0) a.scale[down * a.scale_row + across * a.scale_block] = scale;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t row = first + u * kRows;
        float y[V];
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = element<T>(p[u], e);
        uint32_t word[V / 4];
        eight_bits<V>(y, by, word);
        if (row < a.rows) store_eight<V, PAST>(a.out + column + row * a.out_row, at, left, word);
    }
}

template <class T>
hipError_t quantize_of(QuantizeArgs &g, int tall, hipStream_t s, bool &fits) {
    const uint64_t blocks = (uint64_t)blocks_of(g.columns);
    uint64_t each = 1, rows = kBlock;
    if (tall == 1) {
        rows = kThreads / kBlockLanes<T>;
        each = g.gate ? 2 : 4;   // blocks of a lane: as many while that leaves every compute unit four workgroups
        while (each > 1 && ((blocks + each - 1) / each) * ((g.rows + rows - 1) / rows) < 1024) each /= 2;
    }
    g.across = (uint32_t)((blocks + each - 1) / each);
    g.by_across = make_fastdiv(g.across);
    const uint64_t grid = g.across * (((uint64_t)g.rows + rows - 1) / rows);
    fits = grid < (1u << 24);   // (threads of a launch: 32 bits)
    if (!fits) return hipSuccess;
    const dim3 at((uint32_t)grid), threads(kThreads);
    const int past = past_caches((uint64_t)g.rows * g.columns * (T::bytes * (g.gate ? 2 : 1) + 1), reinterpret_cast<uintptr_t>(g.out) | (uint64_t)g.out_row | g.columns);
    // Blocks beside one another share the lines at their edges where rows are no whole lines, and go to one XCD (6100 x 4080 17.8 us, in turn over all eight 21.3; 20000 x 1040 17.6
    // and 19.9), through its L2 (16391 x 10240 with rows 20496 bytes apart 93.4 us, past it 102.9); else in turn (8192 x 8192 38.2 us, beside one another 43.2).
    // Blocks of one row likewise, but not past the caches (4096 x 4080 12.6 and 13.6, 16391 x 10224 100 and 106; 16391 x 10240 with rows 20496 bytes apart 92.7 and 90.6).
    g.neighbours = (tall != 1 || past == kThrough) && (g.x_row % 128 != 0 || reinterpret_cast<uintptr_t>(g.x) % 128 != 0);
    const bool few = each == 1;   // (few rows and blocks: nothing goes past the caches)
    if (tall != 1)
        return past == kBoth && !g.neighbours ? launch_kernel<amap_quantize_tall_kernel<T, kBoth>>(at, threads, 0, s, g)
               : past != kThrough ? launch_kernel<amap_quantize_tall_kernel<T, kStores>>(at, threads, 0, s, g)
                                  : launch_kernel<amap_quantize_tall_kernel<T, kThrough>>(at, threads, 0, s, g);
    if (g.gate) {
        if (few) return launch_kernel<amap_quantize_kernel<T, true, 1, kThrough>>(at, threads, 0, s, g);
        return past == kBoth     ? launch_kernel<amap_quantize_kernel<T, true, 2, kBoth>>(at, threads, 0, s, g)
               : past == kStores ? launch_kernel<amap_quantize_kernel<T, true, 2, kStores>>(at, threads, 0, s, g)
                                 : launch_kernel<amap_quantize_kernel<T, true, 2, kThrough>>(at, threads, 0, s, g);
    }
    if (few) return launch_kernel<amap_quantize_kernel<T, false, 1, kThrough>>(at, threads, 0, s, g);
    if (each == 2) return launch_kernel<amap_quantize_kernel<T, false, 2, kThrough>>(at, threads, 0, s, g);
    return past == kBoth     ? launch_kernel<amap_quantize_kernel<T, false, 4, kBoth>>(at, threads, 0, s, g)
           : past == kStores ? launch_kernel<amap_quantize_kernel<T, false, 4, kStores>>(at, threads, 0, s, g)
                             : launch_kernel<amap_quantize_kernel<T, false, 4, kThrough>>(at, threads, 0, s, g);
}

}  // namespace

extern "C" amap_status amap_quantize(const amap_rows *x, const amap_rows *gate, int64_t rows, int64_t columns, int tall, const amap_rows *out, const amap_scales *scale,
                                     void *stream) {
    if (!x || !out || !scale || rows < 0 || columns < 0 || !is_wide(x->type) || out->type != AMAP_E4M3 || (gate && gate->type != x->type)) return AMAP_E_INVALID;
    if (tall != 1 && tall != kBlock) return refuse("blocks of other than 1 or 128 rows");
    if (gate && tall != 1) return refuse("a gate in front of blocks of 128 rows");
    if (rows > INT32_MAX || columns > INT32_MAX) return AMAP_E_SHAPE;
    if (rows == 0 || columns == 0) return AMAP_OK;
    if (!x->data || !out->data || !scale->data || (gate && !gate->data)) return AMAP_E_INVALID;
    const Runs from = runs_of(*x, rows, columns), by = gate ? runs_of(*gate, rows, columns) : Runs{}, to = runs_of(*out, rows, columns),
               sc = runs_of(*scale, (rows + tall - 1) / tall, blocks_of(columns));
    if (!from.box.fits || (gate && !by.box.fits) || !to.box.fits || !to.box.apart || !sc.box.fits || !sc.box.apart) return AMAP_E_SHAPE;
    if (share(to, from) || share(to, by) || share(sc, from) || share(sc, by) || share(sc, to)) return AMAP_E_ALIAS;
    const int es = bytes_of(x->type);
    if (reinterpret_cast<uintptr_t>(x->data) % es || (gate && reinterpret_cast<uintptr_t>(gate->data) % es) || reinterpret_cast<uintptr_t>(scale->data) % 4)
        return refuse("a tensor that does not begin at a whole element");
    QuantizeArgs g = {};
    g.x = static_cast<const char *>(x->data);
    g.x_row = x->row_stride * es;
    if (gate) g.gate = static_cast<const char *>(gate->data), g.gate_row = gate->row_stride * es;
    g.out = static_cast<char *>(out->data);
    g.out_row = out->row_stride;
    g.scale = scale->data;
    g.scale_row = scale->row_stride, g.scale_block = scale->block_stride;
    g.rows = (uint32_t)rows;
    g.columns = (uint32_t)columns;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const StreamDevice device(s);
    if (device.status() != hipSuccess) return launched(device.status(), "the stream's device");
    bool fits;
    const hipError_t e = x->type == AMAP_F32 ? quantize_of<F32>(g, tall, s, fits) : x->type == AMAP_BF16 ? quantize_of<Bf16>(g, tall, s, fits) : quantize_of<F16>(g, tall, s, fits);
    return fits ? launched(e, "amap_quantize_kernel") : refuse("too many blocks for one launch");
}
