// Internal interface between the C ABI layer (layers_api.hip) and the kernels of the scoring
// model's layers (row_kernels.hip, embedding_grad_kernels.hip, i8_kernels.hip, norm_kernels.hip,
// norm_grad_kernels.hip, mx_kernels.hip).
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

enum Norm : int32_t { kNormNone = 0, kNormRms = 1, kNormLayer = 2 };
enum Gate : int32_t { kGateLinear = 0, kGateSigmoid = 1, kGateNone = 2 };

// n = post(f), y = x + scale * g * n, h = pre(y): x, weights, biases and h or NULL.
struct NormArgs {
    const void *x, *f, *gate;
    void *y, *h;
    const float *post_weight, *post_bias, *pre_weight, *pre_bias;
    int64_t x_stride, f_stride, gate_stride, y_stride, h_stride;     // bytes
    int64_t n;
    int32_t cols, type, stream_type, post, pre, gate_kind;
    float post_eps, pre_eps, scale;
};
hipError_t launch_norm(const NormArgs &a, hipStream_t stream);

// Sums over rows, in this order wherever they are numbered.
enum Sum : int { kPostWeight = 0, kPreWeight = 1, kPostBias = 2, kPreBias = 3, kSums = 4 };

// The gradients, of NormArgs without y, h and pre_bias: dy, dh, dx, dgate or sums may be NULL.
struct NormGradArgs {
    NormArgs a;
    const void *dy, *dh;
    void *dx, *df, *dgate;
    int64_t dy_stride, dh_stride, dx_stride, df_stride, dgate_stride;       // bytes
    float *sums[kSums];
    void *workspace;
    bool accumulate;
};
int64_t norm_grad_workspace_bytes(int64_t n, int32_t cols);
hipError_t launch_norm_grad(const NormGradArgs &a, hipStream_t stream);

// Rows in microscaled 4-bit floating point.
inline int64_t mx_padded(int64_t k) { return (k + 127) & ~(int64_t)127; }
inline int64_t mx_scales(int64_t k) { return (k + 511) / 512 * 16; }       // bytes of a row's scales

struct MxRowsArgs {
    const void *x;                                // the rows of the other type; written by dequantise
    uint8_t *q, *scales;
    int64_t x_stride, q_stride, scales_stride;    // bytes
    int64_t n;
    int32_t cols, type;
};
hipError_t launch_mx_quantize(const MxRowsArgs &a, hipStream_t stream);
hipError_t launch_mx_dequantize(const MxRowsArgs &a, hipStream_t stream);

struct MxProductArgs {
    const uint8_t *a, *b, *a_scales, *b_scales;
    const float *bias;
    void *out;
    int64_t a_stride, b_stride, a_scales_stride, b_scales_stride, out_stride;   // bytes
    int64_t m, n, k;
    int32_t out_type;
    bool relu;
};
hipError_t launch_mx_product(const MxProductArgs &a, hipStream_t stream);
// The product of rows that are quantised on the way: product.a, a_scales: room for their 4-bit form.
hipError_t launch_mx_linear(const MxRowsArgs &x, const MxProductArgs &product, hipStream_t stream);

}  // namespace ccj
