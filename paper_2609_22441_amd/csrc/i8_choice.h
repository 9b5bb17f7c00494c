// Which kernel computes an 8-bit product: a rule on its sizes alone. Host code without HIP, so that
// tests can ask it which kernel a call takes.
//
// Times below are in us for m x n x k, bf16 output, weights of two calls in turn; a / b: the kernel in
// question against the next one.
#pragma once

#include <stdint.h>

namespace ccj {

// Few results: 16 x 16 tiles, fragments straight from memory, k shared out over 8 wavefronts.
constexpr int32_t kSkinny = 0;
// Tiles through LDS, (rows x columns, groups that share out k).
constexpr int32_t kTile64 = 1;         // 64 x 64, 4
constexpr int32_t kTile128x64 = 2;     // 128 x 64, 2
constexpr int32_t kTile128Split = 3;   // 128 x 128, 2
constexpr int32_t kTile128 = 4;        // 128 x 128, 1
constexpr int32_t kTile256 = 5;        // 256 x 256, 1
constexpr int32_t kTileShort = 6;      // 128 x 128, 1, all of k at once

constexpr int64_t kUnits = 256;        // compute units

// 16 x 4,096 x 8,192 11.3 / 14.5, 64 x 1,024 x 8,192 9.8 / 13.4, 1 x 4,096 x 2,048 4.2 / 6.2. Twice as
// many tiles: 16 x 8,192 x 2,048 6.2 / 6.7, but 16 x 8,192 x 8,192 19.3 / 14.8.
constexpr int64_t kSkinnyTiles = 256, kSkinnyShortTiles = 512, kSkinnyShortK = 2048;

// Of rows that the skinny kernel quantises itself, one launch less: 1 x 8,192 x 8,192 is 15.4 / 14.7
// before the quantisation's launch.
constexpr int64_t kSkinnyRows = 16, kSkinnyLinearTiles = 1024, kSkinnyLds = 64 << 10;

// 512 x 8,192 x 512: 7.8 without shared k against 8.7 with it; x 2,048 16.4 / 16.0, x 8,192 48.9 / 45.4.
constexpr int64_t kSplitK = 1024;

// Of products this short the output is the work.
constexpr int64_t kShortK = 128, kShortTile = 128;

// Of longer ones up to this a tile's loads and stores still cost as much as its products: two tiles at
// a time on a unit, 50,000 x 2,048 x 512 117 / 133 in 256 x 256 (x 1,024 183 / 180).
constexpr int64_t kMidK = 512;

inline int64_t tiles_of(int64_t m, int64_t n, int64_t tm, int64_t tn) {
    return ((m + tm - 1) / tm) * ((n + tn - 1) / tn);
}

inline int32_t product_choice(int64_t m, int64_t n, int64_t k) {
    const int64_t t16 = tiles_of(m, n, 16, 16);
    if (t16 <= kSkinnyTiles || (t16 <= kSkinnyShortTiles && k <= kSkinnyShortK))
        return kSkinny;
    // Larger tiles as soon as smaller ones would give a unit a second one: 256 x 4,096 x 8,192 takes 19
    // in 64 x 64, 26 in 128 x 64; 512 x 4,096 x 8,192 37 and 28, 40 in 128 x 128; 512 x 8,192 x 8,192
    // 57 in 128 x 64, 45 in 128 x 128.
    if (tiles_of(m, n, 64, 64) <= kUnits)
        return kTile64;
    if (tiles_of(m, n, 128, 64) <= kUnits)
        return kTile128x64;
    const int64_t t128 = tiles_of(m, n, 128, 128), t256 = tiles_of(m, n, 256, 256);
    // Few rows of many outputs take these tiles as well. The weights' bytes are their work, whatever rows a
    // tile lacks: 1 x 32,000 x 4,096 24.2 and 16 x 32,000 x 4,096 24.8 in 128 x 128 with shared k, 1 x 50,000
    // x 2,048 19.6 without, where a large copy's 4.8 TB/s would give 27.3 and 21.3 (a part of the weights is
    // in the caches from call to call).
    if (t128 <= kUnits)
        return k >= kSplitK ? kTile128Split : kTile128;
    if (k <= kShortK)
        return kTileShort;
    if (k <= kMidK)
        return kTile128;
    // A unit has two 128 x 128 tiles at a time (87 for k = 8,192) or one of 256 x 256 (127): 1,024 x
    // 8,192 x 8,192 89 / 89, 2,048 x 8,192 x 8,192 127 in 256 x 256, 171 in 128 x 128.
    const int64_t r128 = (t128 + 2 * kUnits - 1) / (2 * kUnits), r256 = (t256 + kUnits - 1) / kUnits;
    return 3 * r256 <= 2 * r128 ? kTile256 : kTile128;
}

// Whether a linear layer's rows are quantised by the tile kernel: each tile of columns would do so
// again.
inline bool quantize_in_tile(int64_t, int64_t n, int64_t k) { return k <= kShortK && n <= kShortTile; }

// Whether a linear layer's rows are quantised by the skinny kernel.
inline bool quantize_inside(int64_t m, int64_t n, int64_t k) {
    return m <= kSkinnyRows && tiles_of(m, n, 16, 16) <= kSkinnyLinearTiles &&
           m * (k + 16) <= kSkinnyLds;
}

}  // namespace ccj
