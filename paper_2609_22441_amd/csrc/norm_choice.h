// How the norms share out their rows: rules on sizes alone. Host code without HIP, so that tests can ask
// which kernel a call takes.
#pragma once

#include <stdint.h>

namespace ccj {

// Lanes of a row, and blocks of 8 columns that each of them holds in registers; none: rows too long for
// that, which go through the caches in pieces. Beyond a wavefront a row has as many as it needs.
struct NormShape {
    int32_t lanes, blocks;
};

inline int32_t whole_wavefronts(int32_t lanes) { return (lanes + 63) / 64 * 64; }

inline NormShape norm_shape(int32_t cols) {
    const int32_t blocks = (cols + 7) / 8;
    if (blocks <= 64)
        return {blocks <= 16 ? 16 : blocks <= 32 ? 32 : 64, 1};
    if (blocks <= 128)
        return {64, 2};
    if (blocks <= 256)
        return {whole_wavefronts(blocks), 1};
    if (blocks <= 2048)
        return {whole_wavefronts((blocks + 1) / 2), 2};
    return {0, 0};
}

// Workgroups of the norm for `rows` rows or groups of rows that a workgroup takes at a time: one each up to
// 2,048 threads a unit (registers let a unit hold 512 to 2,048 of them at a time, the others follow), and of
// more rows one for each four, which keeps the chip full to the end (65,536 x 4,096 bf16 484 us, with 2,048
// threads a unit 558) and still reads the weights once for four rows; a launch may not have any number of
// them.
inline int64_t norm_groups(int64_t rows, int32_t threads) {
    const int64_t held = 256 * (int64_t)(2048 / threads), fours = (rows + 3) / 4, most = 1 << 20;
    return rows < held ? rows : fours < held ? held : fours < most ? fours : most;
}

// The gradient's, which holds five matrices' elements and the sums over rows; wide: the residual stream is in
// 32 bits, which leaves fewer registers. Two blocks a lane where one wavefront then has the row, without
// barriers (100,000 x 1,024 bf16 296 us, 321 in 128 lanes), and where 1,024 lanes would have too few
// registers; else one, which leaves room for more rows (65,536 x 4,096 804, 841 in 256 lanes). With a wide
// stream the lanes are a power of two, known to the kernel: with any number of them it spilled more registers
// (65,536 x 4,096 1,288 us, 1,047 so).
inline NormShape norm_grad_shape(int32_t cols, bool wide) {
    const int32_t blocks = (cols + 7) / 8;
    if (blocks <= 64)
        return {blocks <= 16 ? 16 : blocks <= 32 ? 32 : 64, 1};
    if (blocks > 1024)
        return {0, 0};
    if (wide)
        return blocks <= 512 ? NormShape{blocks <= 128 ? 128 : blocks <= 256 ? 256 : 512, 1} : NormShape{512, 2};
    return blocks <= 128 ? NormShape{64, 2} : NormShape{whole_wavefronts(blocks), 1};
}

// Its workgroups, each of which adds up its rows to a partial result: up to 1,024 threads a unit, of fewer
// rows so many that each has eight, but not fewer than half of that (4,000 x 1,024 30 us with 1,024 threads a
// unit, 20 with half of them; 1,000 x 2,048 24 and 17). A unit holds 1,024 at a time of the kernels with four
// wavefronts to a SIMD (grad_wavefronts in norm_grad_kernels.hip); of those with three or two, which biases,
// 32-bit elements and two blocks a lane have, it holds 768 or 512, and the others follow in a second round.
inline int64_t norm_grad_groups(int64_t rows, int32_t cols, bool wide) {
    const int32_t lanes = norm_grad_shape(cols, wide).lanes, threads = lanes <= 64 ? 256 : lanes;
    const int64_t at_once = threads / lanes, need = (rows + at_once - 1) / at_once;
    const int64_t most = 256 * (int64_t)(1024 / threads);
    const int64_t half = 256 * (int64_t)(threads < 512 ? 512 / threads : 1);
    const int64_t eighth = (need + 7) / 8, some = need < half ? need : half;
    const int64_t groups = eighth > some ? eighth : some;
    return groups < most ? groups : most;
}

// Strips of rows whose sums over columns are partial results of one workgroup each, of the kernels that
// go over rows in pieces: about 3,072 workgroups of 256 blocks of 8 columns, four times what the chip holds.
inline int64_t norm_wide_strips(int64_t rows, int32_t cols) {
    const int64_t pieces = ((int64_t)cols + 2047) / 2048, most = 3072 / pieces;
    const int64_t strips = most < 1 ? 1 : most;
    return strips < rows ? strips : rows;
}

}  // namespace ccj
