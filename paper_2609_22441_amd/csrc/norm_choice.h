// How the norms share out their rows: rules on sizes alone. Host code without HIP, so that tests can ask
// which kernel a call takes.
#pragma once

#include <stdint.h>

namespace ccj {

// Lanes of a row, and blocks of 8 columns that each of them holds in registers; none: rows too long for
// that, which go through the caches in pieces.
struct NormShape {
    int32_t lanes, blocks;
};

inline NormShape norm_shape(int32_t cols) {
    const int32_t blocks = (cols + 7) / 8;
    if (blocks <= 16)
        return {16, 1};
    if (blocks <= 64)
        return {64, 1};
    if (blocks <= 128)
        return {64, 2};
    if (blocks <= 256)
        return {256, 1};
    if (blocks <= 512)
        return {256, 2};
    if (blocks <= 1024)
        return {512, 2};
    if (blocks <= 2048)
        return {1024, 2};
    return {0, 0};
}

// The gradient's, which holds five matrices' elements and the sums over rows: one block a lane.
inline int32_t norm_grad_lanes(int32_t cols) {
    const int32_t blocks = (cols + 7) / 8;
    return blocks <= 16 ? 16 : blocks <= 64 ? 64 : blocks <= 256 ? 256 : blocks <= 512 ? 512
                                                                     : blocks <= 1024 ? 1024 : 0;
}

// Its workgroups, each of which adds up its rows: as many as the chip holds at a time.
inline int64_t norm_grad_groups(int64_t rows, int32_t cols) {
    const int32_t lanes = norm_grad_lanes(cols), threads = lanes < 256 ? 256 : lanes;
    const int64_t rows_at_once = threads / lanes, need = (rows + rows_at_once - 1) / rows_at_once;
    const int64_t most = 256 * (int64_t)(1024 / threads);
    return need < most ? need : most;
}

// Strips of rows whose sums over columns are partial results of one workgroup each, of the kernels that
// go over rows in pieces: about 1,024 workgroups of 256 blocks of 8 columns.
inline int64_t norm_wide_strips(int64_t rows, int32_t cols) {
    const int64_t pieces = ((int64_t)cols + 2047) / 2048, most = 1024 / pieces;
    const int64_t strips = most < 1 ? 1 : most;
    return strips < rows ? strips : rows;
}

}  // namespace ccj
