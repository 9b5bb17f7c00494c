// How an embedding gradient is computed and what its workspace holds: a rule on the call's sizes alone.
// Host code without HIP, so that tests can ask it which form a call takes.
#pragma once

#include <algorithm>
#include <stdint.h>

#include "grad_runs.h"

namespace ccj {

constexpr int kGradBlock = 8;           // columns of a lane

// ---- sorted pairs ----

struct Pair {
    uint32_t key, token;
};

constexpr int kSortThreads = 1024;
constexpr int kMaxDigitBits = 9;
constexpr int kMinTile = 2048;          // pairs per workgroup of a digit pass
constexpr int kMaxTiles = 256;          // every workgroup reads the counts of all tiles
constexpr int64_t kMaxChunks = 1 << 18; // chunks times column tiles: the joins' grid stays launchable

struct SortShape {
    int32_t passes, digit_bits;         // digit passes, bits of each
    int32_t tiles;
    int64_t tile;                       // pairs per tile, a multiple of kSortThreads
};

inline SortShape sort_shape(int64_t n, int64_t rows) {
    SortShape s;
    int bits = 1;
    while (rows >> bits)                // keys 0 to rows: the last is every id outside the table
        ++bits;
    s.passes = (bits + kMaxDigitBits - 1) / kMaxDigitBits;
    s.digit_bits = (bits + s.passes - 1) / s.passes;
    const int64_t even = (n + kMaxTiles - 1) / kMaxTiles;
    s.tile = std::max<int64_t>(kMinTile, (even + kSortThreads - 1) / kSortThreads * kSortThreads);
    s.tiles = (int32_t)((n + s.tile - 1) / s.tile);
    return s;
}

// ---- sums of runs ----

constexpr int kJoinThreads = 1024;

// ---- small calls and small tables: pairs in LDS ----

constexpr int kSmallIds = 4096;         // tokens of a workgroup of 1,024: 12 bits
constexpr int kWindowThreads = 256;     // of a small table's windows, of 4 tokens per thread
constexpr int kSmallRows = 64;          // rows of a workgroup, at most
constexpr int kSmallGroups = 1024;      // workgroups of a small call, at most: each reads all ids
constexpr int kSmallTable = 128;        // rows of a small table

struct Window {
    int32_t rows, tiles;         // of the table per workgroup; column tiles
    int32_t tokens, count;       // tokens per window; windows
    float *partial;              // [count][a.rows][width], or null: one window, its sums are final
    int32_t width;
};

// ---- layout of the workspace ----

inline int64_t round16(int64_t x) { return (x + 15) & ~(int64_t)15; }

struct GradPlan {
    SortShape sort;
    Window window;                                       // count 0: the sorted way
    int64_t chunk, chunks;
    int32_t lanes, tiles, width;
    int64_t folds;                                       // 0: none, the chunks are joined
    int64_t counts, found, list, pairs0, pairs1, partial, folded, bytes;  // offsets, the total size
};

inline GradPlan grad_plan(int64_t n, int64_t rows, int32_t cols) {
    GradPlan p = {};
    p.sort = sort_shape(n, rows);
    const int blocks = (cols + kGradBlock - 1) / kGradBlock;
    p.lanes = blocks <= 4 ? 4 : blocks <= 16 ? 16 : 64;
    p.tiles = (blocks + p.lanes - 1) / p.lanes;
    p.width = blocks * kGradBlock;
    p.window.tiles = p.tiles;
    p.window.width = p.width;
    const int64_t ranges = (rows + kSmallRows - 1) / kSmallRows;
    const int window_tokens = kWindowThreads * (kSmallIds / kSortThreads);
    // Windows of 1,024 tokens, shorter ones while there are fewer than 512 workgroups of them, but with
    // twice as many tokens as rows and so as sums. 400,000 x 96 bf16 into 51 rows 39 us, 57 by the sort
    // of the whole call; 4,096 x 64 fp32 into 50 rows 10.8 with windows of 128, 17.5 with 512.
    if (rows <= kSmallTable && n > window_tokens) {
        p.window.rows = (int)std::min<int64_t>(rows, kSmallRows);
        int tokens = window_tokens;
        while (tokens > 128 && tokens > 4 * rows && n / tokens * ranges * p.tiles < 512)
            tokens /= 2;
        p.window.tokens = tokens;
        p.window.count = (int)((n + p.window.tokens - 1) / p.window.tokens);
        p.bytes = (int64_t)p.window.count * rows * p.width * 4;
        return p;
    }
    // One launch: while a lane group of one workgroup, which may have all the tokens, has at most 64.
    // 2,049 x 96 fp32 into 1,000 rows 10.5 us, 26 in the six launches; 4,096 x 1,024 into 2 rows would
    // be 167.
    if (n <= std::min(kSmallIds, 64 * (kSortThreads / p.lanes)) && ranges * p.tiles <= kSmallGroups) {
        p.window.rows = (int)std::max<int64_t>(
            1, std::min<int64_t>(kSmallRows, (rows * p.tiles + 255) / 256));
        p.window.tokens = kSmallIds;
        p.window.count = 1;
        return p;
    }
    // Chunks of 16 tokens where rows are wide, so that the last wavefronts to run are few of many, and 32
    // where more groups share a wavefront; shorter ones while the chip has fewer than 4 wavefronts per
    // SIMD of them. 131,072 x 2,048 bf16, Zipf frequencies: 183 us in the sums with 16, 192 with 32, 207
    // with 64.
    p.chunk = p.lanes == 64 ? 16 : 32;
    while (p.chunk > 8 && n / p.chunk * p.tiles * p.lanes < 4 * 1024 * 64)
        p.chunk /= 2;
    while (n / p.chunk * p.tiles > kMaxChunks)
        p.chunk *= 2;
    p.chunks = (n + p.chunk - 1) / p.chunk;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += round16(bytes);
        return here;
    };
    p.counts = take((int64_t)p.sort.tiles << p.sort.digit_bits << 2);
    p.found = take(rows + 1);               // the last: ids outside the table
    p.list = take(4 * (p.chunks + 1));
    p.pairs0 = take(n * (int64_t)sizeof(Pair));
    p.pairs1 = take(p.sort.passes > 1 ? n * (int64_t)sizeof(Pair) : 0);
    p.partial = take(p.chunks * 2 * p.width * 4);
    // A run's partial sums are added up by the lane groups of one workgroup: folded first where a group
    // could get more than 32 of them.
    p.folds = p.chunks > 32 * (kJoinThreads / p.lanes) ? (p.chunks + kFold - 1) / kFold : 0;
    p.folded = take(p.folds * 2 * p.width * 4);
    p.bytes = at;
    return p;
}

}  // namespace ccj
