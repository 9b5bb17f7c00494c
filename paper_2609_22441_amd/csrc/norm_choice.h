// How the norms share out their rows: rules on sizes alone. Host code without HIP, so that tests can ask
// which kernel a call takes.
#pragma once

#include <stdint.h>

namespace ccj {

// Strips of rows whose sums over columns are partial results of one workgroup each, of the kernels that
// go over rows in pieces: about 1,024 workgroups of 256 blocks of 8 columns.
inline int64_t norm_wide_strips(int64_t rows, int32_t cols) {
    const int64_t pieces = ((int64_t)cols + 2047) / 2048, most = 1024 / pieces;
    const int64_t strips = most < 1 ? 1 : most;
    return strips < rows ? strips : rows;
}

}  // namespace ccj
