// What the kernels over rows share (norm, its gradient, rows into 8 bits): 16-byte pieces of a row at any address, their elements in 32 bits, sums and
// maxima over the lanes that hold a row or a block of it, and the step to 8 bits.
#pragma once

#include "amap_cache.hpp"

namespace amap_rows_detail {

using namespace amap_cache_detail;

// (a row may begin at any element: the hardware takes a 16-byte access at any byte, and pieces at whole 16 bytes cost nothing more)
typedef u32x4 u32x4_any __attribute__((aligned(1)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));
typedef uint32_t u32_any __attribute__((aligned(1)));

enum Past { kThrough = 0, kStores = 1, kBoth = 2 };   // the caches: see past_caches

template <class T>
constexpr int kPer = 16 / T::bytes;   // elements of a piece
constexpr int kBlock = AMAP_SCALE_BLOCK;
template <class T>
constexpr int kBlockLanes = kBlock / kPer<T>;   // lanes that hold a block, a piece each

// Elements `at` .. of a row of `dim` (2^30 bytes at most): whole pieces in one access, the last one of a row by elements; zeros past it.  PAST: not kept in the caches.
template <class T, int PAST = kThrough>
__device__ __forceinline__ u32x4 load_piece(const char *row, uint32_t at, uint32_t dim) {
    u32x4 p = {0, 0, 0, 0};
    if (at + kPer<T> <= dim) {
        const u32x4_any *const from = reinterpret_cast<const u32x4_any *>(row + at * (uint32_t)T::bytes);
        if constexpr (PAST == kBoth)
            p = __builtin_nontemporal_load(from);
        else
            p = *from;
    } else if (at < dim) {
        const char *const from = row + at * (uint32_t)T::bytes;
        const uint32_t n = dim - at;
#pragma unroll
        for (uint32_t e = 0; e < (uint32_t)kPer<T> - 1; ++e)
            if (e < n) {
                if constexpr (T::bytes == 4)
                    p[e] = *reinterpret_cast<const uint32_t *>(from + 4 * e);
                else
                    p[e / 2] |= (uint32_t)*reinterpret_cast<const uint16_t *>(from + 2 * e) << (e % 2 * 16);
            }
    }
    return p;
}
template <class T, int PAST = kThrough>
__device__ __forceinline__ void store_piece(char *row, uint32_t at, uint32_t dim, u32x4 p) {
    char *const to = row + at * (uint32_t)T::bytes;
    if (at + kPer<T> <= dim) {
        if constexpr (PAST != kThrough)
            __builtin_nontemporal_store(p, reinterpret_cast<u32x4_any *>(to));
        else
            *reinterpret_cast<u32x4_any *>(to) = p;
    } else if (at < dim) {
        const uint32_t n = dim - at;
#pragma unroll
        for (uint32_t e = 0; e < (uint32_t)kPer<T> - 1; ++e)
            if (e < n) {
                if constexpr (T::bytes == 4)
                    *reinterpret_cast<uint32_t *>(to + 4 * e) = p[e];
                else
                    *reinterpret_cast<uint16_t *>(to + 2 * e) = (uint16_t)(p[e / 2] >> (e % 2 * 16));
            }
    }
}

template <class T>
__device__ __forceinline__ float element(const u32x4 &p, int e) {
    if constexpr (T::bytes == 4) {
        return __uint_as_float(p[e]);
    } else if constexpr (std::is_same<T, Bf16>::value) {
        return __uint_as_float(e % 2 ? p[e / 2] & 0xFFFF0000u : p[e / 2] << 16);
    } else {
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(e % 2 ? p[e / 2] >> 16 : p[e / 2]));
    }
}
// rounded to nearest even
template <class T>
__device__ __forceinline__ uint32_t bits(float x) {
    if constexpr (T::bytes == 4)
        return __float_as_uint(x);
    else if constexpr (std::is_same<T, Bf16>::value)
        return __builtin_bit_cast(uint16_t, (__bf16)x);
    else
        return __builtin_bit_cast(uint16_t, (_Float16)x);
}
template <class T>
__device__ __forceinline__ u32x4 piece_of(const float (&x)[kPer<T>]) {
    u32x4 p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (T::bytes == 4)
            p[i] = __float_as_uint(x[i]);
        else
            p[i] = bits<T>(x[2 * i]) | bits<T>(x[2 * i + 1]) << 16;
    }
    return p;
}

// a weight's elements `at` .. (of the rows' type, or 32 bits)
template <class T>
__device__ __forceinline__ void load_weight(const char *weight, bool wide, uint32_t at, uint32_t dim, float (&w)[kPer<T>]) {
    if (T::bytes == 4 || !wide) {
        const u32x4 p = load_piece<T>(weight, at, dim);
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) w[e] = element<T>(p, e);
    } else {
#pragma unroll
        for (int h = 0; h < kPer<T> / 4; ++h) {
            const u32x4 p = load_piece<F32>(weight, at + 4 * h, dim);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[4 * h + e] = __uint_as_float(p[e]);
        }
    }
}

// ---- over lanes: every one of a group of LANES (16, 32 or 64, beside one another) gets the result, the same bits in each

template <int CTRL>
__device__ __forceinline__ float from_lane(float x) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xF, 0xF, false));
}
template <int LANES, class F>
__device__ __forceinline__ float over_lanes(float x, F f) {
    x = f(x, from_lane<0xB1>(x));    // the neighbour's
    x = f(x, from_lane<0x4E>(x));    // the other pair's
    x = f(x, from_lane<0x141>(x));   // the other four's
    x = f(x, from_lane<0x140>(x));   // the other eight's
    if constexpr (LANES >= 32) x = f(x, __shfl_xor(x, 16));
    if constexpr (LANES >= 64) x = f(x, __shfl_xor(x, 32));
    return x;
}
template <int LANES>
__device__ __forceinline__ float sum_over(float x) {
    return over_lanes<LANES>(x, [](float a, float b) { return a + b; });
}
// (of sizes, which are in the order of their bits: maxima of whole numbers take the other lane's in the same instruction)
template <int LANES>
__device__ __forceinline__ float most_over(float x) {
    uint32_t u = __float_as_uint(x);
    auto from = [](uint32_t v, auto lane) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(lane)::value, 0xF, 0xF, false); };
    u = max(u, from(u, std::integral_constant<int, 0xB1>{}));
    u = max(u, from(u, std::integral_constant<int, 0x4E>{}));
    u = max(u, from(u, std::integral_constant<int, 0x141>{}));
    u = max(u, from(u, std::integral_constant<int, 0x140>{}));
    if constexpr (LANES >= 32) u = max(u, (uint32_t)__shfl_xor((int)u, 16));
    if constexpr (LANES >= 64) u = max(u, (uint32_t)__shfl_xor((int)u, 32));
    return __uint_as_float(u);
}

// ---- to 8 bits

// the size of a value that a scale goes by: 0 where it is infinite or NaN
__device__ __forceinline__ float size_of(float x) {
    const float a = __builtin_fabsf(x);
    return a < __builtin_inff() ? a : 0.f;
}
// The largest size of V values that a scale goes by.  (They are looked at one by one only where one of them is infinite: NaN does not enter a maximum.)
template <int V>
__device__ __forceinline__ float most_of(const float (&x)[V]) {
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) most = fmaxf(most, __builtin_fabsf(x[e]));
    if (most == __builtin_inff()) {
        most = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) most = fmaxf(most, size_of(x[e]));
    }
    return most;
}
// The same for pieces as they were loaded: sizes are in the order of their bits, two of 16 to an instruction; infinite ones and NaN come after all others, and are left out one by one.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <class T, int N>
__device__ __forceinline__ float most_of(const u32x4 (&p)[N]) {
    constexpr uint32_t kSize = T::bytes == 4 ? 0x7FFFFFFFu : 0x7FFF7FFFu, kInfinite = T::bytes == 4 ? 0x7F800000u : std::is_same<T, Bf16>::value ? 0x7F80u : 0x7C00u;
    uint32_t top = 0;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t size = p[n][i] & kSize;
            if constexpr (T::bytes == 4)
                top = max(top, size);
            else
                top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, size)));
        }
    if constexpr (T::bytes == 2) top = max(top & 0xFFFFu, top >> 16);
    if (top < kInfinite) return element<T>(u32x4{top, 0, 0, 0}, 0);
    float most = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) most = fmaxf(most, size_of(element<T>(p[n], e)));
    return most;
}
// (most / 448, rounded to 32 bits, from 2^-126 on: the remainder is a whole number of 2^-143)
__device__ __forceinline__ float scale_of(float most) {
    constexpr float kInverse = 1.f / 448.f;
    const float q = most * kInverse;
    return fmaxf(__builtin_fmaf(__builtin_fmaf(-q, 448.f, most), kInverse, q), 0x1p-126f);
}
// A scale to divide by: a division's quotient, rounded to 32 bits, in three instructions instead of eleven.  From the nearest reciprocal, the remainder of value times reciprocal, which a multiply-add has
// exactly, makes that the nearest quotient (Markstein, Computation of elementary functions on the IBM RISC System/6000 processor, 1990).  By the hardware's reciprocal alone ties of 8 bits, which one in 2000 numbers of 16 bits over a
// scale of theirs is, went either way.  Remainders are exact where scales are 2^-64 or more; smaller ones are divided by times 2^64.
struct Divisor {
    float scale, reciprocal;
    bool small;   // the scale is 2^64 of it
};
__device__ __forceinline__ Divisor divisor_of(float scale) {
    Divisor d;
    d.small = scale < 0x1p-64f;
    d.scale = d.small ? scale * 0x1p64f : scale;
    d.reciprocal = 1.f / d.scale;   // (a step of Newton's from the hardware's misses the nearest one for some scales, 0x1.fffffep0 among them)
    return d;
}
// (the remainder with its sign turned: -0 stays -0)
__device__ __forceinline__ float over(float x, const Divisor &d) {
    const float q = x * d.reciprocal;
    return __builtin_fmaf(-__builtin_fmaf(q, d.scale, -x), d.reciprocal, q);
}
// V values over a scale, rounded to nearest even, side by side.  No finite value of the block comes to 464, from where on the conversion would give NaN, as it does for what is infinite.
template <int V>
__device__ __forceinline__ void eight_bits(float (&x)[V], const Divisor &by, uint32_t (&word)[V / 4]) {
    if (by.small) {
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] *= 0x1p64f;
    }
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        const int low = __builtin_amdgcn_cvt_pk_fp8_f32(over(x[4 * i], by), over(x[4 * i + 1], by), 0, false);
        word[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(over(x[4 * i + 2], by), over(x[4 * i + 3], by), low, true);
    }
}
// `at` .. of a row of `dim` bytes
template <int V, int PAST = kThrough>
__device__ __forceinline__ void store_eight(char *row, uint32_t at, uint32_t dim, const uint32_t (&word)[V / 4]) {
    if (at + V <= dim) {
        if constexpr (V == 8 && PAST != kThrough)
            __builtin_nontemporal_store(u32x2{word[0], word[1]}, reinterpret_cast<u32x2_any *>(row + at));
        else if constexpr (V == 8)
            *reinterpret_cast<u32x2_any *>(row + at) = u32x2{word[0], word[1]};
        else if constexpr (PAST != kThrough)
            __builtin_nontemporal_store(word[0], reinterpret_cast<u32_any *>(row + at));
        else
            *reinterpret_cast<u32_any *>(row + at) = word[0];
    } else if (at < dim) {
        const uint32_t n = dim - at;
#pragma unroll
        for (uint32_t e = 0; e < V - 1; ++e)
            if (e < n) row[at + e] = (char)(word[e / 4] >> (e % 4 * 8));
    }
}

// ---- host

// What a call that moves so many bytes stores, and loads as well, past the caches.  us through them / stored past them / loaded past them as well, total MB read and written, outputs in new
// memory:
//   norm with residual into 8 bits   117 24.1/21.0        235 45.6/42.9        345 63.8/60.2/59.5   472 85.0/ - /79.7      norm alone   67 12.5/11.6   134 23.5/20.7   268 46.5/45.7
//   its gradient                     134 31.1/30.5        268 53.1/52.4        393 72.9/ - /70.0    537 96.5/ - /92.6
//   into 8 bits behind a gate        211 38.4/37.2        422 73.3/ - /65.4    844 144/ - /127      without   127 21.5/20.3   254 45.9/44.4   508 88.9/ - /81.1
//   by 128 rows                      125 23.0/19.8        251 48.5/45.7        368 69.5/ - /62.9    503 94.2/ - /85.2
// (Loaded past them below 300 MB, what a call before has left there is read from memory again: norm alone 67 MB 13.3 -> 19.9, 134 MB 22 -> 31.)  Rows that are no whole 64-byte pieces are
// stored through the caches: a piece is stored by two instructions there.  `stored`: the addresses and steps of what is stored, or-ed.
inline int past_caches(uint64_t bytes, uint64_t stored) { return stored % 64 || bytes < (64u << 20) ? kThrough : bytes < 300000000 ? kStores : kBoth; }
inline int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }

}  // namespace amap_rows_detail
