// The measured times that products are cut by: one MI355X, 64 to 1024 tiles of 8 to 96 turns, means over the operands' orders.
#include "mm_cut.hpp"

#include <algorithm>
#include <cmath>

namespace al {

namespace {

// us of a launch of up to 128, up to 256 and up to 512 tiles (where a compute unit holds two), without the launch's own 2: ends + turn * turns.
struct Times {
    int tile, parts, fit;
    double ends[3], turn[3];
};
constexpr Times kTimes[] = {
    {64, 2, 2, {0.5, 0.5, 1.5}, {0.32, 0.33, 0.41}},    {64, 3, 2, {0, 0, 1}, {0.53, 0.53, 0.58}},       {64, 4, 2, {0, 0, 1.5}, {0.61, 0.63, 0.91}},
    {128, 2, 2, {3, 3, 4.5}, {0.6, 0.65, 1.06}},        {256, 2, 1, {10, 9.5, 0}, {1.33, 1.7, 0}},
};
const Times& times(int tile, int parts) {
    for (const Times& t : kTimes)
        if (t.tile == tile && (t.parts == parts || tile > 64)) return t;
    return kTimes[0];
}
// A turn of up to 128 workgroups, 129 to 256 (between the two measured: the clock falls as more of them work), and more.
double turn_of(const Times& t, int64_t tiles) {
    if (tiles <= 128) return t.turn[0];
    if (tiles > 256 && t.fit > 1) return t.turn[2];
    return t.turn[0] + (t.turn[1] - t.turn[0]) * (double)(std::min<int64_t>(tiles, 256) - 128) / 128;
}
double ends_of(const Times& t, int64_t tiles) { return t.ends[tiles <= 128 ? 0 : tiles <= 256 || t.fit == 1 ? 1 : 2]; }

int64_t tiles_of(int tile, int64_t m, int64_t n) { return ((m + tile - 1) / tile) * ((n + tile - 1) / tile); }

}  // namespace

int mm_segments(int tile, int parts) { return tile == 64 ? 1 : parts - 1; }
int mm_fit(int tile, int parts) { return times(tile, parts).fit; }
double mm_turn(int tile, int64_t slots, int parts) { return turn_of(times(tile, parts), slots); }
double mm_ends(int tile, int64_t slots, int parts) { return ends_of(times(tile, parts), slots); }

double mm_time(int tile, int64_t tiles, int64_t turns, int parts) {
    const Times& t = times(tile, parts);
    const int64_t round = 256 * t.fit, rest = tiles % round;
    const double n = (double)(turns * mm_segments(tile, parts));
    return 2.0 + (double)(tiles / round) * (ends_of(t, round) + turn_of(t, round) * n) + (rest == 0 ? 0.0 : ends_of(t, rest) + turn_of(t, rest) * n);
}

MmCut mm_cut(int64_t m, int64_t n, int64_t turns, int parts) {
    static constexpr int counts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
    MmCut best = {64, 1};
    double least = -1;
    for (const int tile : {64, 128, 256}) {
        const int64_t tiles = tiles_of(tile, m, n);
        for (const int c : counts) {
            if (c > 1 && (4 * c > turns * mm_segments(tile, parts) || tiles * c > 1024)) break;
            // splitting: a launch, and the partial sums' way out and back
            const double t = mm_time(tile, tiles * c, (turns + c - 1) / c, parts) + (c > 1 ? 4 + 1.6e-6 * (double)(c * tiles) * tile * tile : 0);
            if (least < 0 || t < least) least = t, best = {tile, c};
        }
    }
    return best;
}

int64_t mm_threads(const MmCut& c, int64_t m, int64_t n) { return tiles_of(c.tile, m, n) * c.splits * (c.tile == 256 ? 512 : 256); }

size_t mm_part_bytes(const MmCut& c, int64_t m, int64_t n) {
    return c.splits == 1 ? 0 : (size_t)(tiles_of(c.tile, m, n) * c.splits) * c.tile * c.tile * 4;
}

}  // namespace al
