// Internal interface between the C ABI layer (layers_api.hip) and the kernels of the scoring
// model's input layer (row_kernels.hip, embedding_grad_kernels.hip, i8_kernels.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ccj {

enum Type : int32_t { kF32 = 0, kF16 = 1, kBF16 = 2 };

inline int type_bytes(int32_t t) { return t == kF32 ? 4 : 2; }

// Rows that all start at a multiple of 16 bytes.
inline bool even_rows(const void *p, int64_t stride) { return !(((uintptr_t)p | stride) & 15); }

constexpr int32_t kMaxCols = 1 << 24;          // elements per row: blocks of a row fit 32 bits
constexpr int64_t kMaxK = 131056;              // 8-bit product: 2^14 * k stays below 2^31
constexpr int kThresholdOne = 65536;           // dropout threshold that keeps everything

// Dropout of a call: kept elements' 16 bits lie below `threshold`.
struct Mask {
    uint32_t key0, key1, site;
    int32_t threshold;
    int64_t first_row;
};

// out[t][c] = keep(t, c) ? source row * factor : 0 (+ residual), the source row being
// src[ids[t]] (zeros for an id outside [0, src_rows)) or, without ids, src[t].
struct RowArgs {
    const void *src, *res, *ids;
    void *out;
    int64_t src_stride, res_stride, out_stride;   // bytes
    int64_t src_rows, n;
    int32_t cols, id_bytes;
    int32_t src_type, out_type;
    float factor;
    Mask mask;
};
hipError_t launch_rows(const RowArgs &a, hipStream_t stream);

struct GradArgs {
    const void *ids, *grad;
    void *table, *workspace;
    int64_t grad_stride, table_stride;            // bytes
    int64_t n, rows;
    int32_t cols, id_bytes, grad_type, table_type;
    bool accumulate;
    float factor;
    Mask mask;
};
int64_t grad_workspace_bytes(int64_t n, int64_t rows, int32_t cols);
hipError_t launch_embedding_grad(const GradArgs &a, hipStream_t stream);

struct QuantizeArgs {
    const void *x;
    int8_t *q;
    float *scales;
    int64_t x_stride, q_stride;                   // bytes
    int64_t n;
    int32_t cols, type;
};
hipError_t launch_quantize(const QuantizeArgs &a, hipStream_t stream);

struct ProductArgs {
    const int8_t *a, *b;
    const float *a_scales, *b_scales, *bias;
    void *out;
    int64_t a_stride, b_stride, out_stride;       // bytes
    int64_t m, n, k;
    int32_t out_type;
    bool relu;
};
hipError_t launch_product(const ProductArgs &a, hipStream_t stream);

// The product of rows that are quantised on the way: q, scales: room for their 8-bit form.
struct LinearArgs {
    const void *x;
    int64_t x_stride;                             // bytes
    int32_t cols, type;                           // of x; the product's k is cols rounded up to 16
    int8_t *q;
    float *scales;
};
hipError_t launch_linear(const LinearArgs &x, const ProductArgs &product, hipStream_t stream);

}  // namespace ccj
