// How the products of mm_device.hpp are cut. Host only.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace al {

// Segments that a tile's turns are taken in; parts: of both operands together (2 to 4).
int mm_segments(int tile, int parts);
// us, measured, of `tiles` tiles of `turns` turns (a segment) each, every tile a workgroup's.
double mm_time(int tile, int64_t tiles, int64_t turns, int parts);
// What a turn takes of a slot's time with `slots` workgroups at work, and what a tile takes besides its turns.
double mm_turn(int tile, int64_t slots, int parts);
double mm_ends(int tile, int64_t slots, int parts);
// Workgroups that a compute unit holds.
int mm_fit(int tile, int parts);

struct MmCut {
    int32_t tile, splits;
};
// One product: tile and splits of k.
MmCut mm_cut(int64_t m, int64_t n, int64_t turns, int parts);
// Threads of the launch of a product cut so. A grid of 2^32 threads and more loses its upper part without an error.
int64_t mm_threads(const MmCut& c, int64_t m, int64_t n);
// Bytes of the partial sums of a product cut so.
size_t mm_part_bytes(const MmCut& c, int64_t m, int64_t n);

}  // namespace al
