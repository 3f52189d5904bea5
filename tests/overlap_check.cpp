// share() of amap_overlap.hpp against every byte of both tensors, over random strides and places.  Prints how many cases shared something and how many
// whose boxes met did not; ends with 1 at the first case that it gets wrong.
#include <cstdio>
#include <random>
#include <set>

#include "amap_overlap.hpp"

using namespace amap_cache_detail;

static std::set<uintptr_t> bytes(const amap_heads &h, int64_t tokens, int dim) {
    std::set<uintptr_t> all;
    for (int64_t t = 0; t < tokens; ++t)
        for (int i = 0; i < h.heads; ++i)
            for (int b = 0; b < dim * bytes_of(h.type); ++b) all.insert(reinterpret_cast<uintptr_t>(h.data) + bytes_of(h.type) * (t * h.token_stride + i * h.head_stride) + b);
    return all;
}

int main() {
    std::mt19937_64 rng(5);
    auto upto = [&](int lo, int hi) { return (int)(lo + rng() % (uint64_t)(hi - lo + 1)); };
    int shared = 0, beside = 0, careful = 0;
    for (int i = 0; i < 60000; ++i) {
        const int64_t tokens = upto(1, 4);
        const int dim = upto(1, 6), all = upto(1, 7);
        const amap_type type = upto(0, 1) ? AMAP_BF16 : AMAP_F32;
        // heads of one projection, tokens or heads outermost, with gaps now and then; one in eight with strides of 0
        const int64_t gap = upto(0, 2) ? 0 : upto(0, 3), inner = dim + gap;
        const bool heads_first = upto(0, 1);
        int64_t token = heads_first ? inner : inner * all + (upto(0, 2) ? 0 : upto(0, 9)), head = heads_first ? inner * tokens : inner;
        amap_heads x{nullptr, type, upto(1, 4), token, head}, y{nullptr, type, upto(1, 4), token, head};
        if (!upto(0, 7)) x.token_stride = y.token_stride = 0;
        if (!upto(0, 7)) y.head_stride = upto(0, 20);
        const uintptr_t at = (uintptr_t)1 << 20;
        x.data = reinterpret_cast<void *>(at + upto(0, 60) * bytes_of(type));
        y.data = reinterpret_cast<void *>(at + upto(0, 60) * bytes_of(type) + (upto(0, 9) ? 0 : 1));
        if (!upto(0, 3)) y.data = reinterpret_cast<void *>(reinterpret_cast<uintptr_t>(x.data) + bytes_of(type) * head * upto(-1, 3));
        const auto a = bytes(x, tokens, dim), b = bytes(y, tokens, dim);
        bool truth = false;
        for (uintptr_t p : a) truth = truth || b.count(p);
        const bool said = share(x, y, tokens, dim), met = meet(box_of(x, tokens, dim), box_of(y, tokens, dim));
        const bool alike = (tokens == 1 || x.token_stride == y.token_stride) && (x.heads == 1 || y.heads == 1 || x.head_stride == y.head_stride);
        if (said != share(y, x, tokens, dim) || (truth && !said) || (said && !truth && (alike || !met))) {
            std::printf("case %d: said %d, is %d (tokens %d dim %d heads %d %d strides %d %d, %d %d, apart %d)\n", i, said, truth, (int)tokens, dim, x.heads, y.heads, (int)x.token_stride, (int)x.head_stride,
                        (int)y.token_stride, (int)y.head_stride, (int)((intptr_t)y.data - (intptr_t)x.data));
            return 1;
        }
        shared += truth;
        beside += met && !said;
        careful += said && !truth;
    }
    std::printf("%d shared, %d beside one another, %d refused for their strides\n", shared, beside, careful);
    return shared > 1000 && beside > 1000 ? 0 : 1;
}
