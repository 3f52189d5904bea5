// share() of runs (amap_overlap.hpp) against every byte of both tensors, over random strides and places.  Prints how many cases shared something and how many
// whose boxes met did not; ends with 1 at the first case that it gets wrong.
#include <algorithm>
#include <cstdio>
#include <random>
#include <set>

#include "amap_overlap.hpp"

using namespace amap_cache_detail;

static void add(std::set<uintptr_t> &all, uintptr_t at, int64_t n) {
    for (int64_t i = 0; i < n; ++i) all.insert(at + i);
}

int main() {
    std::mt19937_64 rng(7);
    auto upto = [&](int lo, int hi) { return (int)(lo + rng() % (uint64_t)(hi - lo + 1)); };
    const amap_type types[] = {AMAP_F32, AMAP_BF16, AMAP_F16, AMAP_E4M3};
    int shared = 0, beside = 0, careful = 0;
    for (int i = 0; i < 120000; ++i) {
        const uintptr_t at = (uintptr_t)1 << 20;
        const int pitch = 4 * upto(0, 9);   // bytes: rows of both within rows of one buffer, mostly
        Runs r[2];
        std::set<uintptr_t> all[2];
        bool dense = true;   // what lies between the scales of a run counts as the run's
        for (int k = 0; k < 2; ++k) {
            const int rows = upto(1, 4), columns = upto(1, 5);
            const uintptr_t first = at + 4 * upto(0, 30);
            const bool other = !upto(0, 5);
            if (upto(0, 1)) {
                const amap_type type = types[upto(0, 3)];
                const int es = bytes_of(type);
                const amap_rows t{reinterpret_cast<void *>(first), type, other ? upto(0, 12) : pitch / es};
                r[k] = upto(0, 1) ? runs_of(t, rows, columns) : runs_of(amap_heads{t.data, t.type, 1, t.row_stride, 7}, rows, columns);
                for (int j = 0; j < rows; ++j) add(all[k], first + es * j * t.row_stride, columns * es);
            } else {
                const amap_scales t{reinterpret_cast<float *>(first), other ? upto(0, 9) : pitch / 4, upto(0, 2) ? 1 : upto(0, 9)};
                const amap_scales u{t.data, t.block_stride, t.row_stride};
                const bool turned = !upto(0, 3);
                const amap_scales &s = turned ? u : t;
                r[k] = runs_of(s, rows, columns);
                for (int j = 0; j < rows; ++j)
                    for (int b = 0; b < columns; ++b) add(all[k], first + 4 * (j * s.row_stride + b * s.block_stride), 4);
                if (rows > 1 && columns > 1) dense = dense && std::min(s.row_stride, s.block_stride) <= 1;
            }
        }
        bool truth = false;
        for (uintptr_t p : all[0]) truth = truth || all[1].count(p);
        const bool said = share(r[0], r[1]), met = meet(r[0].box, r[1].box), alike = r[0].count <= 1 || r[1].count <= 1 || r[0].step == r[1].step;
        if (said != share(r[1], r[0]) || (truth && !said) || (said && !truth && ((alike && dense) || !met))) {
            std::printf("case %d: said %d, is %d (%d runs of %d, %d apart; %d of %d, %d; %d)\n", i, said, truth, (int)r[0].count, (int)r[0].width, (int)r[0].step, (int)r[1].count, (int)r[1].width,
                        (int)r[1].step, (int)((intptr_t)r[1].box.first - (intptr_t)r[0].box.first));
            return 1;
        }
        shared += truth;
        beside += met && !said;
        careful += said && !truth;
    }
    std::printf("%d shared, %d beside one another, %d refused for their strides\n", shared, beside, careful);
    return shared > 1000 && beside > 1000 ? 0 : 1;
}
