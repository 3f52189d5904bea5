// Which memory the tensors of a call take up, and whether two of them have an element in common (host only; no GPU runtime is needed).
#pragma once

#include <cstdint>

#include "amap.h"

namespace amap_cache_detail {

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
inline bool meet(const Box &a, const Box &b) { return a.first < a.past && b.first < b.past && a.first < b.past && b.first < a.past; }

// so many bytes (none at all: a box that meets no other)
inline Box box_of(const void *data, int64_t bytes) {
    Box b;
    b.first = reinterpret_cast<uintptr_t>(data);
    b.past = b.first + (uintptr_t)bytes;
    b.fits = b.apart = b.past >= b.first;
    return b;
}
inline Box box_of(const amap_heads &h, int64_t tokens, int dim) {
    const int64_t extent[3] = {tokens, h.heads, dim}, stride[3] = {h.token_stride, h.head_stride, 1};
    return box_of(h.data, bytes_of(h.type), 3, extent, stride);
}
inline Box box_of(const amap_cache &c, const void *data) {
    const int64_t extent[4] = {c.n_pages, c.page_size, c.kv_heads, c.head_dim}, stride[4] = {c.page_stride, c.token_stride, c.head_stride, 1};
    return box_of(data, bytes_of(c.type), 4, extent, stride);
}

// ---- tensors inside one another's box: heads of one projection, keys and values side by side

// The steps that lead from an element of one tensor to an element of the other: `lo` to `hi` strides of each dimension, in bytes, the widest stride first.
struct Steps {
    int n = 0;
    int64_t stride[4], lo[4], hi[4];
    void add(int64_t by, int64_t from, int64_t to) {
        if (by == 0 || (from == 0 && to == 0)) return;
        int at = n++;
        for (; at > 0 && stride[at - 1] < by; --at) stride[at] = stride[at - 1], lo[at] = lo[at - 1], hi[at] = hi[at - 1];
        stride[at] = by, lo[at] = from, hi[at] = to;
    }
};
inline int64_t floor_of(int64_t x, int64_t by) { return x / by - (x % by < 0); }
// Whether some of them bring two rows of `width` bytes, `apart` from one another, to where they have a byte in common.  Strides that hold all of the next
// inner one leave at most three counts of each to try; where there are many it is taken to be so.
inline bool reach(const Steps &s, int at, int64_t apart, int64_t width) {
    if (at == s.n) return -width < apart && apart < width;
    int64_t least = 0, most = 0;   // what the strides inside add
    for (int i = at + 1; i < s.n; ++i) least += s.lo[i] * s.stride[i], most += s.hi[i] * s.stride[i];
    const int64_t by = s.stride[at];
    int64_t from = -floor_of(width - 1 + apart + most, by), to = floor_of(width - 1 - apart - least, by);
    if (from < s.lo[at]) from = s.lo[at];
    if (to > s.hi[at]) to = s.hi[at];
    if (to - from >= 8) return true;
    for (int64_t d = from; d <= to; ++d)
        if (reach(s, at + 1, apart + d * by, width)) return true;
    return false;
}

// Whether two tensors of rows whose boxes fit have a byte in common; taken to be so if their boxes meet and their strides or types differ.
inline bool share(const amap_heads &a, const amap_heads &b, int64_t tokens, int dim) {
    if (!meet(box_of(a, tokens, dim), box_of(b, tokens, dim))) return false;
    if (bytes_of(a.type) != bytes_of(b.type) || (tokens > 1 && a.token_stride != b.token_stride) || (a.heads > 1 && b.heads > 1 && a.head_stride != b.head_stride)) return true;
    const int64_t es = bytes_of(a.type);
    Steps s;
    s.add(es * a.token_stride, 1 - tokens, tokens - 1);
    s.add(es * (a.heads > 1 ? a.head_stride : b.head_stride), 1 - a.heads, b.heads - 1);
    return reach(s, 0, (int64_t)(reinterpret_cast<uintptr_t>(b.data) - reinterpret_cast<uintptr_t>(a.data)), es * dim);
}

// Whether a cache's keys and values, which have the same strides, have a byte in common.
inline bool keys_and_values_share(const amap_cache &c) {
    const int64_t es = bytes_of(c.type);
    Steps s;
    s.add(es * c.page_stride, 1 - c.n_pages, c.n_pages - 1);
    s.add(es * c.token_stride, 1 - c.page_size, c.page_size - 1);
    s.add(es * c.head_stride, 1 - c.kv_heads, c.kv_heads - 1);
    return meet(box_of(c, c.k), box_of(c, c.v)) && reach(s, 0, (int64_t)(reinterpret_cast<uintptr_t>(c.v) - reinterpret_cast<uintptr_t>(c.k)), es * c.head_dim);
}

}  // namespace amap_cache_detail
