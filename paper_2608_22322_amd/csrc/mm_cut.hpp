// How the products of mm_device.hpp are cut. Host only.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace al {

struct MmCut {
    int32_t tile, splits;
};
// One product: tile and splits of k by a measured model.
MmCut mm_cut(int64_t m, int64_t n, int64_t turns);
// Bytes of the partial sums of a product cut so.
size_t mm_part_bytes(const MmCut& c, int64_t m, int64_t n);

// us of `tiles` outputs of `turns` turns each, every tile a workgroup's.
double mm_time(int tile, int64_t tiles, int64_t turns);

}  // namespace al
