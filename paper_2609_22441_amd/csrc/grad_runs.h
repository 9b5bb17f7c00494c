// Which of the sorted pairs a chunk of the embedding gradient adds up, and what becomes of the runs at
// its edges. Code without HIP, so that tests can walk through it on the host.
#pragma once

#include <stdint.h>

namespace ccj {

constexpr int kSumAhead = 4;        // rows on their way while as many are added
constexpr int kFold = 16;        // chunks whose partial sums are added up together

struct ChunkEnds {
    int64_t i0, i1;              // the chunk's own pairs
    bool head, tail;             // its first run began before it, its last one goes on past it: both
                                 // leave partial sums
};

// The chunk of pairs [start, stop) of n sorted ones, `chunk` in whole chunks. began: the pair before it has
// its first key. of_low: how many of its pairs have its first key; of_high: how many of the `chunk` pairs
// after it have its last one, `high`. Keys of `rows` and above are ids outside the table: they come last,
// no row has their run, and the sums stop before them. So it is no tail: the run that the sums stop at, of
// the table's last id, ends in its chunk.
constexpr ChunkEnds chunk_ends(int64_t start, int64_t stop, int64_t n, int64_t chunk, bool began,
                               int64_t of_low, int64_t of_high, uint32_t high, int64_t rows) {
    const int64_t left = n - stop;
    const bool covers = of_low == stop - start, next = of_high == (chunk < left ? chunk : left);
    return ChunkEnds{start + (began && !covers ? of_low : 0), stop + (next ? 0 : of_high),
                     began && covers, of_high && next && (uint64_t)high < (uint64_t)rows};
}

// The end of the pairs that are added 2 * kSumAhead at a time; the rest come one by one.
constexpr int64_t pipelined(const ChunkEnds &e) {
    return e.i0 + (e.i1 - e.i0) / (2 * kSumAhead) * (2 * kSumAhead);
}

}  // namespace ccj
