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
template <int LANES>
__device__ __forceinline__ float most_over(float x) {
    return over_lanes<LANES>(x, [](float a, float b) { return fmaxf(a, b); });
}

// ---- to 8 bits

// the size of a value that a scale goes by: 0 where it is infinite or NaN
__device__ __forceinline__ float size_of(float x) {
    const float a = __builtin_fabsf(x);
    return a < __builtin_inff() ? a : 0.f;
}
__device__ __forceinline__ float scale_of(float most) { return fmaxf(most / 448.f, 0x1p-126f); }
// A value over a scale, by the scale's reciprocal: up to 1.5 steps of 2^-24 from the quotient, where the rounding to 8 bits takes 2^-4; no finite value of the block
// comes to 464, from where on the conversion would give NaN, as it does for what is infinite.  (From 2^-126 up, a scale and its reciprocal are normal numbers.)
__device__ __forceinline__ float reciprocal_of(float scale) { return __builtin_amdgcn_rcpf(scale); }
// V values times `by`, rounded, side by side
template <int V>
__device__ __forceinline__ void eight_bits(const float (&x)[V], float by, uint32_t (&word)[V / 4]) {
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        const int low = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * by, x[4 * i + 1] * by, 0, false);
        word[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * by, x[4 * i + 3] * by, low, true);
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

inline Box box_of(const amap_rows &r, int64_t rows, int64_t columns) {
    const int64_t extent[2] = {rows, columns}, stride[2] = {r.row_stride, 1};
    return amap_cache_detail::box_of(r.data, bytes_of(r.type), 2, extent, stride);
}
inline Box box_of(const amap_scales &s, int64_t rows, int64_t blocks) {
    const int64_t extent[2] = {rows, blocks}, stride[2] = {s.row_stride, s.block_stride};
    return amap_cache_detail::box_of(s.data, 4, 2, extent, stride);
}
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
