// What the entry points around the paged cache share: the element types on both sides, and the checks of their arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "amap.h"
#include "amap_device.hpp"
#include "amap_index.hpp"
#include "amap_launch.hpp"
#include "amap_overlap.hpp"
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
