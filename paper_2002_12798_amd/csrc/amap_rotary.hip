// Rotary positions (amap_rotary) and the store of fresh keys and values through a slot map (amap_cache_append): rows of heads
// read once, turned where there is something to turn, rounded once and written once.
//
// A workgroup takes a few tokens.  A lane has one unit of a token's rows, the widest piece that their layout allows (both halves of the
// pairs, or a piece that holds whole pairs, or one that is only carried over), and the same one of up to U tokens: what it
// is and where it lies are worked out once.  Its loads are issued first; while they are on their way the workgroup makes the tokens' angles, one
// pair per lane, in LDS, where every head finds them: the angle is position x frequency in 64 bits, brought into one turn
// there (at position 100 000 a 32-bit product is off by 4e-3 of a radian), its sine and cosine in 32 by two parts of the angle.  Bound by the bytes of the rows: fp32
// [65536, 16, 64] 90.6 us (537 MB, 5.9 TB/s), bf16 [12480, 16, 80] 16.1 us (64 MB; an identity copy 11.6), 16391 tokens of 32 + 2 x 8 heads of 128 with keys and values into 8
// bits 71.8 us (369 MB; 58.8).  Four tokens of a lane: two 84 us, eight 94 us (their registers leave half the wavefronts) in the last case.
#include "amap_cache.hpp"

using namespace amap_cache_detail;
using namespace amap_detail;
using namespace amap_dev;

namespace {

constexpr int kMostThreads = 512, kMaxJobs = 3, kAtOnce = 4;   // tokens of a lane
constexpr uint32_t kMostAngles = 4096;   // 32 KB of them
constexpr int kMaxDim = 2048;

// one tensor's way: where it comes from, where it goes
struct TurnJob {
    const char *src;
    char *dst;
    const float *scale;        // divide by scale[head] first (E4M3)
    int64_t src_token, src_head, dst_token, dst_head, dst_page;   // strides in elements; dst_token: of a cache's rows
    uint32_t units;            // of one token, heads * per_head
    uint32_t per_head;
    FastDiv by_head;
    uint32_t turns, to_cache, out_type;
};
struct TurnArgs {
    TurnJob job[kMaxJobs];
    const float *freq;
    const int32_t *position;
    const int64_t *slot;
    int64_t axis_stride, n_slots;
    uint32_t tokens, pairs, interleaved, n_jobs, inverse, page;
    uint32_t axis_end[AMAP_MAX_AXES];
    uint32_t units;            // of one token, all jobs
    uint32_t width, beside;    // lanes to one token, tokens side by side
    uint32_t each, group;      // tokens of a lane, of a workgroup
    uint32_t rounds, splits;   // rounds of `width` units to all of a token's, dealt to so many workgroups
    FastDiv by_width, by_split, by_pairs;
};

template <int BYTES>
struct Piece;
template <>
struct Piece<16> {
    typedef u32x4 type;
};
template <>
struct Piece<8> {
    typedef u32x2 type;
};
template <>
struct Piece<4> {
    typedef uint32_t type;
};
template <>
struct Piece<2> {
    typedef uint16_t type;
};
template <>
struct Piece<1> {
    typedef uint8_t type;
};

template <class T>
__device__ __forceinline__ float widen(const char *at);
template <>
__device__ __forceinline__ float widen<F32>(const char *at) {
    float x;
    __builtin_memcpy(&x, at, 4);
    return x;
}
template <>
__device__ __forceinline__ float widen<Bf16>(const char *at) {
    uint16_t x;
    __builtin_memcpy(&x, at, 2);
    return __uint_as_float((uint32_t)x << 16);
}
template <>
__device__ __forceinline__ float widen<F16>(const char *at) {
    _Float16 x;
    __builtin_memcpy(&x, at, 2);
    return (float)x;
}

// x / s, by whose reciprocal: rounded as the division is but for some last places (one correction of the product; none where what is
// left is not finite: the quotient is not, or the divisor)
__device__ __forceinline__ float over(float x, float s, float reciprocal) {
    const float q = x * reciprocal, r = __builtin_fmaf(-q, s, x);
    return __builtin_isfinite(r) ? __builtin_fmaf(r, reciprocal, q) : q;
}

template <bool STREAM, class P>
__device__ __forceinline__ void put(char *at, P p) {
    if constexpr (STREAM)
        __builtin_nontemporal_store(p, reinterpret_cast<P *>(at));
    else
        *reinterpret_cast<P *>(at) = p;
}
// V values rounded to nearest even and stored in one access
template <int V, bool STREAM>
__device__ __forceinline__ void store_as(uint32_t type, char *at, const float (&x)[V]) {
    if (type == AMAP_F32) {
        if constexpr (V * 4 <= 16) {
            typename Piece<V * 4>::type p;
            __builtin_memcpy(&p, x, sizeof(p));
            put<STREAM>(at, p);
        }
    } else if (type == AMAP_E4M3) {
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = x[i] != x[i] ? x[i] : fminf(fmaxf(x[i], -448.f), 448.f);
        uint16_t b[V > 1 ? V / 2 : 1];
#pragma unroll
        for (int i = 0; i < (V > 1 ? V / 2 : 1); ++i) b[i] = (uint16_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2 * i], y[V > 1 ? 2 * i + 1 : 0], 0, false);
        typename Piece<V>::type p;
        __builtin_memcpy(&p, b, V);
        put<STREAM>(at, p);
    } else {
        uint16_t h[V];
#pragma unroll
        for (int i = 0; i < V; ++i)
            h[i] = type == AMAP_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)x[i]) : __builtin_bit_cast(uint16_t, (_Float16)x[i]);
        typename Piece<V * 2>::type p;
        __builtin_memcpy(&p, h, sizeof(p));
        put<STREAM>(at, p);
    }
}

// How a pair's elements come to one lane: beside one another in one access (or nothing is turned); in two accesses, one to each half of the pairs; or in
// two neighbouring lanes, one access each, which hand each other half of what they have.  The last covers rows without gaps where a half is no
// whole number of 64-byte pieces (heads of 80, 40 pairs: 20.4 -> 18.2 us over 64 MB when it was made, 16.1 now), and costs the others a little.
enum Pairs { kBeside = 0, kHalves = 1, kLanes = 2 };

// the neighbouring lane's
__device__ __forceinline__ uint32_t of_neighbour(uint32_t x) { return __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, false); }   // quad_perm 1, 0, 3, 2

// `b` where the mask is all ones, else `a` (a choice between elements of an array, written as one, went through memory)
__device__ __forceinline__ uint32_t choose(uint32_t mask, uint32_t a, uint32_t b) { return (a & ~mask) | (b & mask); }
__device__ __forceinline__ float choose(uint32_t mask, float a, float b) { return __uint_as_float(choose(mask, __float_as_uint(a), __float_as_uint(b))); }

// T: the rows' type; BYTES: of one access to them; STREAM: stores past the caches
template <class T, int BYTES, Pairs PAIRS, bool STREAM>
__global__ __launch_bounds__(kMostThreads) void amap_turn_kernel(const TurnArgs a) {
    constexpr int V = BYTES / T::bytes, U = kAtOnce;
    constexpr bool HALVES = PAIRS == kHalves;
    typedef typename Piece<BYTES>::type piece;
    extern __shared__ char lds[];
    int64_t *const place = reinterpret_cast<int64_t *>(lds);                          // [group]: of a token's row in the cache, -1: none
    float2 *const angle = reinterpret_cast<float2 *>(lds + 8u * (a.slot ? a.group : 0u));   // [group][pairs]: cosine, sine
    const uint32_t tid = threadIdx.x, block = fdiv(blockIdx.x, a.by_split), split = blockIdx.x - block * a.splits;
    const uint32_t t0 = block * a.group, count = min(a.group, a.tokens - t0);
    const uint32_t beside = fdiv(tid, a.by_width), in = tid - beside * a.width;
    // the first of this lane's angles: asked for in front of the rows, so that it can be made while they are on their way
    auto axis_of = [&](uint32_t p) __attribute__((always_inline)) {
        uint32_t axis = 0;
#pragma unroll
        for (int k = 0; k + 1 < AMAP_MAX_AXES; ++k) axis += p >= a.axis_end[k];
        return axis;
    };
    const uint32_t angles = count * a.pairs;
    int32_t position = 0;
    float freq = 0.f;
    if (tid < angles) {
        const uint32_t t = fdiv(tid, a.by_pairs), p = tid - t * a.pairs;
        position = a.position[axis_of(p) * a.axis_stride + t0 + t];
        freq = a.freq[p];
    }
    for (uint32_t round = split; round < a.rounds; round += a.splits) {
        // ---- this lane's unit
        uint32_t u = round * a.width + in, j = 0;
        const bool mine = u < a.units && beside < a.beside;
        if (!mine) u = 0;
        // Its tensor, put together from scalars: read by an index that differs from lane to lane, each field would be a load of its own, and those in the
        // last loop would wait for the stores in front of them.
        TurnJob job = a.job[0];
        if (a.n_jobs > 1) {
#pragma unroll
            for (int k = 0; k + 1 < kMaxJobs; ++k) {
                const bool on = (uint32_t)k + 1 < a.n_jobs && j == (uint32_t)k && u >= a.job[k].units;
                const TurnJob &to = a.job[k + 1];
                if (on) {
                    u -= a.job[k].units;
                    j = k + 1;
                    job = to;
                }
            }
        }
        const uint32_t head = fdiv(u, job.by_head);
        u -= head * job.per_head;
        const uint32_t halves = HALVES && job.turns ? a.pairs / V : 0u, second = u & 1u;   // second: (neighbouring lanes) of the pairs' second elements
        const bool turned = HALVES ? u < halves : job.turns && u * V < 2u * a.pairs;
        // its first element: of the first halves, or of what lies behind both
        const uint32_t at = PAIRS == kLanes && turned ? (u >> 1) * V + second * a.pairs : u < halves ? u * V : (u + halves) * V;
        const char *const src = job.src + ((int64_t)(t0 + beside) * job.src_token + (int64_t)head * job.src_head + at) * T::bytes;
        const int64_t step = (int64_t)a.beside * job.src_token * T::bytes;
        piece x[U], y[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (!mine || (uint32_t)k >= a.each || beside + k * a.beside >= count) continue;
            x[k] = *reinterpret_cast<const piece *>(src + k * step);
            if (HALVES && turned) y[k] = *reinterpret_cast<const piece *>(src + k * step + (size_t)a.pairs * T::bytes);
        }
        if (round == split) {
            if (a.slot)
                for (uint32_t i = tid; i < count; i += blockDim.x) {
                    const int64_t slot = a.slot[t0 + i], page = slot / a.page;   // (the caches' strides are the first job's)
                    place[i] = slot >= 0 && slot < a.n_slots ? page * a.job[0].dst_page + (slot - page * a.page) * a.job[0].dst_token : -1;
                }
            for (uint32_t i = tid; i < angles; i += blockDim.x) {
                if (i != tid) {
                    const uint32_t t = fdiv(i, a.by_pairs), p = i - t * a.pairs;
                    position = a.position[axis_of(p) * a.axis_stride + t0 + t];
                    freq = a.freq[p];
                }
                const double turns = (double)position * (double)freq * 0.15915494309189533577, half = 2.0 * (turns - rint(turns));   // 1 / (2 pi)
                float s, c;
                const float most = (float)half, rest = (float)(half - (double)most) * 3.14159265358979323846f;
                sincospif(most, &s, &c);
                // (what rounding the angle left out, up to 9e-8 of a radian: as much as a step of the result, and all that there is of a sine next to a whole half turn)
                const float sine = __builtin_fmaf(c, rest, s), cosine = __builtin_fmaf(-s, rest, c);
                angle[i] = make_float2(cosine, a.inverse ? -sine : sine);
            }
            __syncthreads();
        }
        const uint32_t type = job.out_type, es = type == AMAP_F32 ? 4u : type == AMAP_E4M3 ? 1u : 2u;
        const float scale = job.scale ? job.scale[head] : 1.f, reciprocal = 1.f / scale;
        const int64_t in_token = (int64_t)head * job.dst_head + at;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const uint32_t t = beside + k * a.beside;
            if (!mine || (uint32_t)k >= a.each || t >= count) continue;
            const int64_t to = job.to_cache ? place[t] : (int64_t)(t0 + t) * job.dst_token;
            if (to < 0) continue;
            char *const dst = job.dst + (to + in_token) * es;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = widen<T>(reinterpret_cast<const char *>(&x[k]) + e * T::bytes);
            const float2 *const cs = angle + t * a.pairs;
            if constexpr (HALVES) {
                if (turned) {
                    float w[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float b = widen<T>(reinterpret_cast<const char *>(&y[k]) + e * T::bytes), f = v[e];
                        const float2 c = cs[at + e];
                        v[e] = f * c.x - b * c.y;
                        w[e] = b * c.x + f * c.y;
                    }
                    if (scale != 1.f) {
#pragma unroll
                        for (int e = 0; e < V; ++e) w[e] = over(w[e], scale, reciprocal);
                    }
                    store_as<V, STREAM>(type, dst + a.pairs * es, w);
                }
            } else if constexpr (PAIRS == kLanes) {
                // first elements 0 .. V - 1 here and the second ones next door: this lane takes pairs 0 .. V / 2 - 1, the other one the rest
                if (turned) {
                    constexpr int W = BYTES / 8;   // words of half a piece
                    const uint32_t mask = 0u - second;
                    uint32_t got[W];
#pragma unroll
                    for (int e = 0; e < W; ++e) got[e] = of_neighbour(choose(mask, x[k][W + e], x[k][e]));
                    float f[V / 2], b[V / 2];
                    const uint32_t pair = (u >> 1) * V + second * (V / 2);
#pragma unroll
                    for (int e = 0; e < V / 2; ++e) {
                        const float own = choose(mask, v[e], v[V / 2 + e]), its = widen<T>(reinterpret_cast<const char *>(got) + e * T::bytes);
                        const float first = choose(mask, own, its), other = choose(mask, its, own);
                        const float2 c = cs[pair + e];
                        f[e] = first * c.x - other * c.y;
                        b[e] = other * c.x + first * c.y;
                    }
#pragma unroll
                    for (int e = 0; e < V / 2; ++e) {
                        const float its = __uint_as_float(of_neighbour(__float_as_uint(choose(mask, b[e], f[e]))));
                        v[e] = choose(mask, f[e], its);
                        v[V / 2 + e] = choose(mask, its, b[e]);
                    }
                }
            } else if constexpr (V > 1) {
                if (turned) {
#pragma unroll
                    for (int e = 0; e < V; e += 2)
                        if (at + e < 2u * a.pairs) {
                            const float f = v[e], b = v[e + 1];
                            const float2 c = cs[(at + e) >> 1];
                            v[e] = f * c.x - b * c.y;
                            v[e + 1] = b * c.x + f * c.y;
                        }
                }
            }
            if (scale != 1.f) {
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = over(v[e], scale, reciprocal);
            }
            store_as<V, STREAM>(type, dst, v);
        }
    }
}

bool rope_fits(const amap_rope *r, int dim, amap_status &st) {
    st = AMAP_E_INVALID;
    if (!r->freq || r->pairs < 1 || r->n_axes < 1 || r->n_axes > AMAP_MAX_AXES) return false;
    int64_t sum = 0;
    for (int i = 0; i < r->n_axes; ++i) {
        if (r->axis_pairs[i] < 0) return false;
        sum += r->axis_pairs[i];
    }
    st = AMAP_E_SHAPE;
    return sum == r->pairs && r->pairs <= dim / 2;
}

// The widest access that all rows of the jobs allow, 16 bytes of the rows' type at most, down to one element (two of them where neighbours are
// pairs: whole pairs in a unit).
struct Way {
    const amap_heads *in;
    void *dst;
    amap_type out;
    int64_t token, head, page;   // of dst
    bool turns, to_cache;
    const float *scale;
};

template <class T, int BYTES, Pairs PAIRS, bool STREAM>
hipError_t turn(const TurnArgs &g, uint32_t grid, uint32_t threads, uint32_t lds, hipStream_t s) {
    return launch_kernel<amap_turn_kernel<T, BYTES, PAIRS, STREAM>>(dim3(grid), dim3(threads), lds, s, g);
}
template <class T, int BYTES, bool STREAM>
hipError_t turn_by(Pairs pairs, const TurnArgs &g, uint32_t grid, uint32_t threads, uint32_t lds, hipStream_t s) {
    if constexpr (BYTES == 16)
        if (pairs == kLanes) return turn<T, BYTES, kLanes, STREAM>(g, grid, threads, lds, s);
    return pairs == kHalves ? turn<T, BYTES, kHalves, STREAM>(g, grid, threads, lds, s) : turn<T, BYTES, kBeside, STREAM>(g, grid, threads, lds, s);
}
template <class T>
hipError_t turn_of(int bytes, Pairs pairs, bool stream, const TurnArgs &g, uint32_t grid, uint32_t threads, uint32_t lds, hipStream_t s) {
    if (bytes == 16) return stream ? turn_by<T, 16, true>(pairs, g, grid, threads, lds, s) : turn_by<T, 16, false>(pairs, g, grid, threads, lds, s);
    if (bytes == 8) return turn_by<T, 8, false>(pairs, g, grid, threads, lds, s);
    if (T::bytes == 2 && bytes == 2) return turn_by<T, T::bytes, false>(pairs, g, grid, threads, lds, s);
    return turn_by<T, 4, false>(pairs, g, grid, threads, lds, s);
}

// Threads of a workgroup for rows of so many units: as few lanes as possible without one (64 .. 512 in steps of 64; 256 where others are no better).
uint32_t threads_for(uint64_t units) {
    uint32_t best = 256;
    double most = 0.0;
    if (units > 256 && units <= kMostThreads) return (uint32_t)(units + 63) / 64 * 64;   // all of a token's at once
    for (uint32_t n : {256u, 320u, 384u, 448u, 512u, 192u, 128u}) {
        const double held = units <= n ? (double)(n / units * units) / n : (double)units / (double)((units + n - 1) / n * n);
        if (held > most + 0.03) most = held, best = n;
    }
    return best;
}

amap_status run(const Way *way, int n, int64_t tokens, int dim, const amap_rope *rope, const int32_t *position, int64_t axis_stride, int inverse, const int64_t *slot,
                const amap_cache *cache, hipStream_t s) {
    const amap_type type = way[0].in->type;
    const int es = bytes_of(type);
    // ---- the width: what divides every offset, in elements, and in bytes on both sides
    uint64_t elements = (uint64_t)dim;
    uint64_t most = 16 / es;
    if (rope) elements |= rope->interleaved ? 0u : (uint64_t)rope->pairs;
    for (int i = 0; i < n; ++i) {
        const Way &w = way[i];
        const uint64_t out = (uint64_t)bytes_of(w.out);
        if (tokens > 1) elements |= (uint64_t)w.in->token_stride;
        if (w.in->heads > 1) elements |= (uint64_t)w.in->head_stride | (uint64_t)w.head;
        elements |= w.to_cache ? (uint64_t)w.token | (uint64_t)w.page : tokens > 1 ? (uint64_t)w.token : 0u;
        const uint64_t in_at = reinterpret_cast<uintptr_t>(w.in->data), out_at = reinterpret_cast<uintptr_t>(w.dst);
        if (in_at % es || out_at % out) return refuse("a tensor that does not begin at a whole element");
        elements |= in_at / es | out_at / out;
        most = most < 16 / out ? most : 16 / out;
    }
    uint64_t width = aligned_to(elements, most);
    if (rope && rope->interleaved && width < 2) {   // pairs of two elements in one access, where rows allow no wider one: an odd element
        return refuse("neighbouring pairs need rows that begin at even elements, and an even head_dim");
    }
    TurnArgs g = {};
    g.n_jobs = (uint32_t)n;
    g.tokens = (uint32_t)tokens;
    if (rope) {
        g.freq = rope->freq;
        g.position = position;
        g.axis_stride = axis_stride;
        g.pairs = (uint32_t)rope->pairs;
        g.interleaved = rope->interleaved != 0;
        g.inverse = inverse != 0;
        uint32_t end = 0;
        for (int i = 0; i < AMAP_MAX_AXES; ++i) {
            if (i < rope->n_axes) end += (uint32_t)rope->axis_pairs[i];
            g.axis_end[i] = i + 1 < rope->n_axes ? end : 0xFFFFFFFFu;   // (the last axis has the rest)
        }
    }
    if (cache) {
        g.slot = slot;
        g.n_slots = cache->n_pages * cache->page_size;
        g.page = (uint32_t)cache->page_size;
    }
    const uint32_t per_head = (uint32_t)(dim / (int)width), all_halves = rope && !rope->interleaved ? (uint32_t)rope->pairs / (uint32_t)width : 0u;
    // pairs in neighbouring lanes: the units of one head, and of all in front of it, have to be even in number
    Pairs pairs = all_halves ? kHalves : kBeside;
    // (Whole pieces as well where they are read and written far beyond the caches: 134 MB in and out 51.6 -> 51.2 us, 268 MB 98.6 -> 94.7, heads of 64 52 -> 47;
    // 67 MB 23.4 against 26.4, 8 MB 8.3 against 10.)
    const bool far_beyond = n == 1 && tokens * way[0].in->heads * dim * es >= ((int64_t)128 << 20);
    if (all_halves && (int)width * es == 16 && per_head % 2 == 0 && ((uint64_t)rope->pairs * es % 64 || far_beyond)) pairs = kLanes;
    const uint32_t halves = pairs == kHalves ? all_halves : 0u;
    uint64_t units = 0;
    for (int i = 0; i < n; ++i) {
        const Way &w = way[i];
        TurnJob &j = g.job[i];
        j.src = static_cast<const char *>(w.in->data);
        j.dst = static_cast<char *>(w.dst);
        j.scale = w.scale;
        j.src_token = w.in->token_stride;
        j.src_head = w.in->head_stride;
        j.dst_token = w.token;
        j.dst_head = w.head;
        j.dst_page = w.page;
        j.per_head = w.turns ? per_head - halves : per_head;
        j.units = j.per_head * (uint32_t)w.in->heads;
        j.by_head = make_fastdiv(j.per_head);
        j.turns = w.turns;
        j.to_cache = w.to_cache;
        j.out_type = w.out;
        units += j.units;
    }
    if (units > (1u << 24)) return refuse("more than 2^24 pieces in the rows of one token");
    g.units = (uint32_t)units;
    g.by_pairs = make_fastdiv(g.pairs ? g.pairs : 1u);
    uint32_t threads = threads_for(units);
    g.width = units < threads ? (uint32_t)units : threads;
    g.beside = threads / g.width;
    g.by_width = make_fastdiv(g.width);
    if (g.pairs && g.beside > kMostAngles / g.pairs) g.beside = kMostAngles / g.pairs;   // (pairs <= 1024: at least 4)
    // tokens of a lane: as many as it loads at once, while that leaves every compute unit two workgroups
    g.each = kAtOnce;
    if (g.pairs && g.each * g.beside > kMostAngles / g.pairs) g.each = kMostAngles / g.pairs / g.beside;
    while (g.each > 1 && (uint64_t)tokens < 512ull * g.beside * g.each) g.each /= 2;
    while (g.beside > 1 && (uint64_t)tokens < 512ull * g.beside) g.beside = (g.beside + 1) / 2;
    g.group = g.beside * g.each;
    threads = (g.width * g.beside + 63u) / 64u * 64u;
    g.rounds = (g.units + g.width - 1) / g.width;
    const uint64_t blocks = ((uint64_t)tokens + g.group - 1) / g.group;
    g.splits = blocks >= 2048 ? 1 : g.rounds;
    if (blocks * g.splits >= (1u << 31)) return refuse("too many tokens for one launch");
    g.by_split = make_fastdiv(g.splits);
    const uint32_t lds = g.group * g.pairs * 8u + (slot ? 8u * g.group : 0u), grid = (uint32_t)(blocks * g.splits);
    const StreamDevice device(s);
    if (device.status() != hipSuccess) return launched(device.status(), "the stream's device");
    const int bytes = (int)width * es;
    // Past the caches where every run of a store is whole 64-byte pieces at both ends: [65536,16,128] bf16 106 -> 98 us, [16391,8,128] k and v stored
    // 34 -> 25, but rows of 160 bytes in two halves of 80 20.4 -> 24.
    uint64_t runs = 0;
    for (int i = 0; i < n; ++i) {
        const Way &w = way[i];
        const uint64_t out = (uint64_t)bytes_of(w.out);
        // (heads that follow one another are one run, unless their halves are stored apart)
        const bool apart = pairs == kHalves && w.turns, joined = !apart && w.head == dim;
        runs |= reinterpret_cast<uintptr_t>(w.dst) | out * ((uint64_t)w.token | (uint64_t)w.page);
        runs |= out * (joined ? (uint64_t)dim * (uint64_t)w.in->heads : (uint64_t)w.head | (uint64_t)dim | (apart ? (uint64_t)rope->pairs : 0u));
    }
    const bool past = runs % 64 == 0;
    const hipError_t e = type == AMAP_F32    ? turn_of<F32>(bytes, pairs, past, g, grid, threads, lds, s)
                         : type == AMAP_BF16 ? turn_of<Bf16>(bytes, pairs, past, g, grid, threads, lds, s)
                                             : turn_of<F16>(bytes, pairs, past, g, grid, threads, lds, s);
    return launched(e, "amap_turn_kernel");
}

// a tensor of rows that a call reads or writes
amap_status check_rows(const amap_heads *h, int64_t tokens, int dim, bool written, Box &box) {
    if (!h || !h->data || h->heads < 1 || !is_wide(h->type)) return AMAP_E_INVALID;
    box = box_of(*h, tokens, dim);
    return box.fits && (!written || box.apart) ? AMAP_OK : AMAP_E_SHAPE;
}

bool same_rows(const amap_heads &a, const amap_heads &b) { return a.data == b.data && a.token_stride == b.token_stride && a.head_stride == b.head_stride; }

// (out is x itself, or beside it: in one projection, say)
amap_status check_turn(const amap_heads *x, const amap_heads *out, int64_t tokens, int dim, Box &from, Box &to) {
    amap_status st = check_rows(x, tokens, dim, false, from);
    if (st == AMAP_OK) st = check_rows(out, tokens, dim, true, to);
    if (st != AMAP_OK) return st;
    if (x->type != out->type) return AMAP_E_INVALID;
    if (x->heads != out->heads) return AMAP_E_SHAPE;
    return !same_rows(*x, *out) && share(*x, *out, tokens, dim) ? AMAP_E_ALIAS : AMAP_OK;
}

amap_status check_sizes(int64_t tokens, int dim) {
    if (tokens < 0 || dim < 1) return AMAP_E_INVALID;
    if (tokens > INT32_MAX) return AMAP_E_SHAPE;
    return dim > kMaxDim ? refuse("heads of more than 2048 elements") : AMAP_OK;
}

}  // namespace

extern "C" amap_status amap_rotary(const amap_heads *x, const amap_heads *out, int64_t tokens, int head_dim, const amap_rope *rope, const int32_t *position,
                                   int64_t axis_stride, int inverse, void *stream) {
    if (!x || !out || !rope) return AMAP_E_INVALID;
    amap_status st = check_sizes(tokens, head_dim);
    if (st != AMAP_OK) return st;
    if (!rope_fits(rope, head_dim, st)) return st;
    if (tokens == 0) return AMAP_OK;
    if (!position || axis_stride < 0) return AMAP_E_INVALID;
    Box from, to;
    st = check_turn(x, out, tokens, head_dim, from, to);
    if (st != AMAP_OK) return st;
    const Way way{x, out->data, out->type, out->token_stride, out->head_stride, 0, true, false, nullptr};
    return run(&way, 1, tokens, head_dim, rope, position, axis_stride, inverse, nullptr, nullptr, reinterpret_cast<hipStream_t>(stream));
}

extern "C" amap_status amap_cache_append(const amap_cache *cache, const amap_heads *k, const amap_heads *v, int64_t tokens, const int64_t *slot, const amap_rope *rope,
                                         const int32_t *position, int64_t axis_stride, const amap_heads *q, const amap_heads *q_out, void *stream) {
    Box ck, cv, rows[3], to;
    amap_status st = check_cache(cache, ck, cv);
    if (st != AMAP_OK) return st;
    if (keys_and_values_share(*cache)) return AMAP_E_ALIAS;
    const int dim = cache->head_dim;
    if (!k || !v || (q != nullptr) != (q_out != nullptr) || (q && !rope)) return AMAP_E_INVALID;
    st = check_sizes(tokens, dim);
    if (st != AMAP_OK) return st;
    if (rope && !rope_fits(rope, dim, st)) return st;
    if (tokens == 0) return AMAP_OK;
    if (!slot || (rope && (!position || axis_stride < 0))) return AMAP_E_INVALID;
    st = check_rows(k, tokens, dim, false, rows[0]);
    if (st == AMAP_OK) st = check_rows(v, tokens, dim, false, rows[1]);
    if (st != AMAP_OK) return st;
    if (k->type != v->type || (q && q->type != k->type)) return AMAP_E_INVALID;
    if (k->heads != cache->kv_heads || v->heads != cache->kv_heads) return AMAP_E_SHAPE;
    int n = 2;
    Way way[kMaxJobs] = {{k, cache->k, cache->type, cache->token_stride, cache->head_stride, cache->page_stride, rope != nullptr, true, cache->k_scale},
                         {v, cache->v, cache->type, cache->token_stride, cache->head_stride, cache->page_stride, false, true, cache->v_scale},
                         {}};
    if (q) {
        st = check_turn(q, q_out, tokens, dim, rows[2], to);
        if (st != AMAP_OK) return st;
        if (meet(to, ck) || meet(to, cv)) return AMAP_E_ALIAS;
        // (q may lie beside k and v in one projection, and be turned there in place)
        if (share(*q_out, *k, tokens, dim) || share(*q_out, *v, tokens, dim)) return AMAP_E_ALIAS;
        way[n++] = Way{q, q_out->data, q_out->type, q_out->token_stride, q_out->head_stride, 0, true, false, nullptr};
    }
    for (int i = 0; i < n; ++i)
        if (meet(rows[i], ck) || meet(rows[i], cv)) return AMAP_E_ALIAS;
    return run(way, n, tokens, dim, rope, position, axis_stride, 0, slot, cache, reinterpret_cast<hipStream_t>(stream));
}
