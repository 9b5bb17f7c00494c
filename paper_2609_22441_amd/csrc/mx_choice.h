// Which kernel computes a product of 4-bit rows: a rule on its sizes alone. Host code without HIP, so that
// tests can ask it which kernel a call takes.
#pragma once

#include <stdint.h>

namespace ccj {

// Few results: 16 x 16 tiles, fragments straight from memory, k shared out over 8 wavefronts.
constexpr int32_t kMxSkinny = 0;
// Tiles through LDS, (rows x columns, groups that share out k).
constexpr int32_t kMxTile64 = 1;         // 64 x 64, 4
constexpr int32_t kMxTile128x64 = 2;     // 128 x 64, 2
constexpr int32_t kMxTile128Split = 3;   // 128 x 128, 2
constexpr int32_t kMxTile128 = 4;        // 128 x 128, 1
constexpr int32_t kMxTile256 = 5;        // 256 x 256, 1

constexpr int64_t kMxUnits = 256;        // compute units

inline int64_t mx_tiles(int64_t m, int64_t n, int64_t tm, int64_t tn) {
    return ((m + tm - 1) / tm) * ((n + tn - 1) / tn);
}

inline int32_t mx_product_choice(int64_t m, int64_t n, int64_t k) {
    const int64_t t16 = mx_tiles(m, n, 16, 16);
    if (t16 <= 256 || (t16 <= 512 && k <= 4096))
        return kMxSkinny;
    // Larger tiles as soon as smaller ones would give a unit a second one.
    if (mx_tiles(m, n, 64, 64) <= kMxUnits)
        return kMxTile64;
    if (mx_tiles(m, n, 128, 64) <= kMxUnits)
        return kMxTile128x64;
    const int64_t t128 = mx_tiles(m, n, 128, 128), t256 = mx_tiles(m, n, 256, 256);
    if (t128 <= kMxUnits)
        return k >= 2048 ? kMxTile128Split : kMxTile128;
    if (k <= 1024)
        return kMxTile128;
    // A unit has two 128 x 128 tiles at a time or one of 256 x 256.
    const int64_t r128 = (t128 + 2 * kMxUnits - 1) / (2 * kMxUnits), r256 = (t256 + kMxUnits - 1) / kMxUnits;
    return 3 * r256 <= 2 * r128 ? kMxTile256 : kMxTile128;
}

}  // namespace ccj
