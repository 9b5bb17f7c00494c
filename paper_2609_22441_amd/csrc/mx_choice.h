// Which kernel computes a product of 4-bit rows: a rule on its sizes alone. Host code without HIP, so that
// tests can ask it which kernel a call takes.
//
// Times below are in us for m x n x k, bf16 output, weights of two calls in turn; a / b: the kernel in
// question against the next one.
#pragma once

#include <stdint.h>

namespace ccj {

// Few results: 16 x 16 tiles, fragments straight from memory, k shared out over 8 wavefronts.
constexpr int32_t kMxSkinny = 0;
// Tiles through LDS.
constexpr int32_t kMxTile64 = 1;         // 64 x 64, two groups that share out k
constexpr int32_t kMxTile128 = 2;        // 128 x 128
constexpr int32_t kMxTile256 = 3;        // 256 x 256

constexpr int64_t kMxUnits = 256;        // compute units

// 32 x 4,096 x 4,096 6.5 / 6.9, 1 x 8,192 x 16,384 14.2 / 23.3, 16 x 8,192 x 8,192 11.9 / 13.3; of more
// tiles 33 x 4,096 x 4,096 7.9 / 6.9, 16 x 12,288 x 8,192 16.4 / 14.3, 48 x 4,096 x 8,192 15.9 / 13.1.
constexpr int64_t kMxSkinnyTiles = 512;

// A unit has two 64 x 64 tiles at a time: 512 x 4,096 x 16,384 38.8 / 45.8, 1,025 x 1,024 x 8,192 18.9 /
// 24.2. A second round is too many: 512 x 8,192 x 4,096 23.3 / 16.0, 2,049 x 1,024 x 8,192 30.5 / 24.7.
constexpr int64_t kMxTiles64 = 2 * kMxUnits;

// Its wavefronts have a slab of 512 values of k each; of longer k two on their way, which takes registers: 4 x
// 4,096 x 16,384 9.4 / 10.9, 1 x 2,048 x 65,536 23.6 / 27.7, the linear layer 1 x 8,192 x 8,192 9.4 / 12.7, but
// 1 x 16,384 x 4,096, of one slab, 10.9 / 10.0.
constexpr int64_t kMxOneSlab = 4096;

// A linear layer's rows that the skinny kernel puts in 4 bits itself, every tile again: the values that a
// unit's tiles take together. 1 x 4,096 x 4,096 4.2 / 7.0 (the next being a launch for them), 8 x 4,096 x
// 4,096 6.1 / 6.9, 1 x 16,384 x 4,096 10.0 / 11.9, 1 x 8,192 x 8,192 9.4 / 11.1; of more values 16 x 4,096
// x 4,096 8.7 / 7.4, 8 x 8,192 x 8,192 16.6 / 13.0, of more tiles 1 x 32,000 x 2,048 11.7 / 10.6.
constexpr int64_t kMxInsideRows = 16, kMxInsideTiles = 1024, kMxInsideValues = 32768;

// Short products of 256 x 256 tiles have their loads and stores on their own.
constexpr int64_t kMxLongK = 4096;

inline int64_t mx_tiles(int64_t m, int64_t n, int64_t tm, int64_t tn) {
    return ((m + tm - 1) / tm) * ((n + tn - 1) / tn);
}

inline int32_t mx_product_choice(int64_t m, int64_t n, int64_t k) {
    if (mx_tiles(m, n, 16, 16) <= kMxSkinnyTiles)
        return kMxSkinny;
    if (mx_tiles(m, n, 64, 64) <= kMxTiles64)
        return kMxTile64;
    // A unit has two 128 x 128 tiles at a time or one of 256 x 256, which take 1.7 to 1.9 times as long:
    // 4,096 x 4,096 x 1,024 22.2 in 128 x 128, 15.7 in 256 x 256; 4,300 x 4,100 x 8,192 100 / 120 (3 rounds
    // against 2); of 13 rounds against 7 50,000 x 2,048 x 2,048 137 / 145, but x 8,192 575 / 484; 16,384 x
    // 8,192 x 8,192 634 / 533.
    const int64_t t128 = mx_tiles(m, n, 128, 128), t256 = mx_tiles(m, n, 256, 256);
    const int64_t r128 = (t128 + 2 * kMxUnits - 1) / (2 * kMxUnits), r256 = (t256 + kMxUnits - 1) / kMxUnits;
    return (k < kMxLongK ? 2 * r256 <= r128 : 5 * r256 <= 3 * r128) ? kMxTile256 : kMxTile128;
}

// Bytes of LDS that rows in 4 bits take there, with their scales.
inline int64_t mx_quantize_lds(int64_t m, int64_t k) { return m * (k / 2 + 16 + k / 32 + 4); }

// Whether a linear layer's rows are put in 4 bits by the skinny kernel; k a multiple of 128.
inline bool mx_quantize_inside(int64_t m, int64_t n, int64_t k) {
    const int64_t tiles = mx_tiles(m, n, 16, 16);
    return m <= kMxInsideRows && tiles <= kMxInsideTiles &&
           m * k * (tiles < kMxUnits ? kMxUnits : tiles) <= kMxInsideValues * kMxUnits;
}

}  // namespace ccj
