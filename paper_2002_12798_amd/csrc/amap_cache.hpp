// What the entry points around the paged cache share: the element types on both sides, and the checks of their arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "amap.h"
#include "amap_device.hpp"
#include "amap_index.hpp"
#include "amap_launch.hpp"
#include "amap_plan.hpp"

namespace amap_cache_detail {

using amap_dev::FastDiv;
using amap_dev::make_fastdiv;

// ---- host

inline amap_status refuse(const char *why) {
    amap_detail::set_last_error("unsupported", why);
    return AMAP_E_UNSUPPORTED;
}

inline amap_status launched(hipError_t e, const char *what) {
    if (e == hipSuccess) return AMAP_OK;
    amap_detail::set_last_error(what, hipGetErrorString(e));
    return AMAP_E_HIP;
}

inline int bytes_of(amap_type t) { return t == AMAP_F32 ? 4 : t == AMAP_E4M3 ? 1 : 2; }

// A strided box of elements: `first` to `past` bytes, and whether no two of its elements share a place (as far as one
// dimension holding all of the next inner one says).
struct Box {
    uintptr_t first = 0, past = 0;
    bool fits = false, apart = false;
};
inline Box box_of(const void *data, int64_t es, int n, const int64_t *extent, const int64_t *stride) {
    Box b;
    int64_t last = 0, ext[4], st[4];
    int m = 0;
    for (int i = 0; i < n; ++i) {
        if (extent[i] < 1 || stride[i] < 0) return b;
        if (extent[i] == 1) continue;
        int64_t far;
        if (__builtin_mul_overflow(extent[i] - 1, stride[i], &far) || __builtin_add_overflow(last, far, &last)) return b;
        int at = m++;
        for (; at > 0 && st[at - 1] > stride[i]; --at) st[at] = st[at - 1], ext[at] = ext[at - 1];
        st[at] = stride[i];
        ext[at] = extent[i];
    }
    int64_t bytes;
    if (__builtin_add_overflow(last, 1, &last) || __builtin_mul_overflow(last, es, &bytes) || bytes > ((int64_t)1 << 46)) return b;
    b.first = reinterpret_cast<uintptr_t>(data);
    b.past = b.first + (uintptr_t)bytes;
    b.fits = b.past >= b.first;
    b.apart = true;
    int64_t held = 1;   // elements from the first to the last of the dimensions inside
    for (int i = 0; i < m; ++i) {
        b.apart = b.apart && st[i] >= held;
        held += (ext[i] - 1) * st[i];
    }
    return b;
}
inline bool meet(const Box &a, const Box &b) { return a.first < b.past && b.first < a.past; }

inline Box box_of(const amap_heads &h, int64_t tokens, int dim) {
    const int64_t extent[3] = {tokens, h.heads, dim}, stride[3] = {h.token_stride, h.head_stride, 1};
    return box_of(h.data, bytes_of(h.type), 3, extent, stride);
}
inline Box box_of(const amap_cache &c, const void *data) {
    const int64_t extent[4] = {c.n_pages, c.page_size, c.kv_heads, c.head_dim}, stride[4] = {c.page_stride, c.token_stride, c.head_stride, 1};
    return box_of(data, bytes_of(c.type), 4, extent, stride);
}

// A cache that a call may use: AMAP_OK, and its two boxes.
inline amap_status check_cache(const amap_cache *c, Box &k, Box &v) {
    if (!c || !c->k || !c->v || c->k == c->v || c->n_pages < 1 || c->page_size < 1 || c->kv_heads < 1 || c->head_dim < 1) return AMAP_E_INVALID;
    if (c->type != AMAP_BF16 && c->type != AMAP_F16 && c->type != AMAP_E4M3) return AMAP_E_INVALID;
    if ((c->k_scale || c->v_scale) && c->type != AMAP_E4M3) return AMAP_E_INVALID;
    if (c->n_pages > INT32_MAX) return AMAP_E_SHAPE;   // (a table's entries are int32)
    k = box_of(*c, c->k);
    v = box_of(*c, c->v);
    return k.fits && v.fits && k.apart ? AMAP_OK : AMAP_E_SHAPE;
}

inline bool is_wide(amap_type t) { return t == AMAP_F32 || t == AMAP_BF16 || t == AMAP_F16; }
inline bool known(amap_type t) { return t == AMAP_F32 || t == AMAP_BF16 || t == AMAP_F16 || t == AMAP_E4M3; }

// the largest power of two (up to `most`) that divides all that is or-ed into `bits`
inline uint64_t aligned_to(uint64_t bits, uint64_t most) {
    bits |= most;
    return bits & (~bits + 1);
}

// ---- device

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// element types as the kernels are instantiated for them
struct F32 {
    static constexpr int bytes = 4;
};
struct Bf16 {
    static constexpr int bytes = 2;
};
struct F16 {
    static constexpr int bytes = 2;
};

}  // namespace amap_cache_detail
