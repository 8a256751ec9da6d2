// The measured times that products are cut by (one MI355X, 64 to 1536 tiles of 8 to 128 turns, all operand orders; us):
//   256-wide: 12.5 + 1.29 a turn up to 128 tiles, 1.65 for 256 (one workgroup a compute unit)
//   128-wide: 6 + 0.57 a turn up to 256 tiles, 8 + 1.05 for 512 (two)
//   64-wide:  3 + 0.35 a turn up to 256 tiles, 4 + 0.42 for 512 (two)
#include "mm_cut.hpp"

#include <algorithm>
#include <cmath>

namespace al {

double mm_time(int tile, int64_t tiles, int64_t turns) {
    const double t = (double)turns;
    if (tile == 256) {
        const int64_t whole = tiles / 256, rest = tiles % 256;
        return 2.0 + whole * (10.5 + 1.65 * t) + (rest == 0 ? 0.0 : 10.5 + (rest > 128 ? 1.55 : 1.29) * t);
    }
    const double end1 = tile == 128 ? 4.0 : 1.0, end2 = tile == 128 ? 6.0 : 2.0, one = tile == 128 ? 0.6 : 0.36, two = tile == 128 ? 1.05 : 0.42;
    const int64_t whole = tiles / 512, rest = tiles % 512;
    return 2.0 + whole * (end2 + two * t) + (rest == 0 ? 0.0 : rest <= 256 ? end1 + one * t : end2 + two * t);
}

static int64_t tiles_of(int tile, int64_t m, int64_t n) { return ((m + tile - 1) / tile) * ((n + tile - 1) / tile); }

MmCut mm_cut(int64_t m, int64_t n, int64_t turns) {
    static constexpr int counts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
    MmCut best = {64, 1};
    double least = -1;
    for (const int tile : {64, 128, 256}) {
        const int64_t tiles = tiles_of(tile, m, n);
        for (const int c : counts) {
            if (c > 1 && (4 * c > turns || tiles * c > 1024)) break;
            // splitting: a launch, and the partial sums' way out and back
            const double t = mm_time(tile, tiles * c, (turns + c - 1) / c) + (c > 1 ? 4 + 1.6e-6 * (double)(c * tiles) * tile * tile : 0);
            if (least < 0 || t < least) least = t, best = {tile, c};
        }
    }
    return best;
}

size_t mm_part_bytes(const MmCut& c, int64_t m, int64_t n) {
    return c.splits == 1 ? 0 : (size_t)(tiles_of(c.tile, m, n) * c.splits) * c.tile * c.tile * 4;
}

}  // namespace al
