// C ABI of the scoring model's input layer: argument validation and the layout of workspaces. The
// kernels live in row_kernels.hip, embedding_grad_kernels.hip and i8_kernels.hip.
#include <math.h>

#include "api_common.h"
#include "cc_layers.h"
#include "layers_internal.h"

using ccj::aligned;
using ccj::device_error;
using ccj::mul_ok;
using ccj::overlaps;

static_assert(CC_F32 == ccj::kF32 && CC_F16 == ccj::kF16 && CC_BF16 == ccj::kBF16,
              "element types of the header and the kernels agree");

namespace {

bool known(int32_t type) { return type == CC_F32 || type == CC_F16 || type == CC_BF16; }

// Rows of `width` bytes each: `bytes` gets what they span. False when pointer, stride or size
// break the rules.
bool rows_ok(const void *p, int64_t rows, int64_t stride, int64_t width, int64_t align,
             int64_t *bytes) {
    *bytes = 0;
    if (rows == 0)
        return true;
    if (!p || !aligned(p, (uintptr_t)align))
        return false;
    if (rows > 1 && (stride < width || stride % align))
        return false;
    if (rows > 1 && !mul_ok(rows - 1, stride, bytes))
        return false;
    return !__builtin_add_overflow(*bytes, width, bytes);
}

bool mask_of(double p, uint64_t seed, uint32_t site, int64_t first_row, int64_t rows,
             ccj::Mask *m) {
    int64_t end;
    if (!(p >= 0.0 && p <= 1.0) || first_row < 0 || __builtin_add_overflow(first_row, rows, &end))
        return false;
    m->key0 = (uint32_t)seed;
    m->key1 = (uint32_t)(seed >> 32);
    m->site = site;
    m->threshold = ccj::kThresholdOne - (int32_t)floor(65536.0 * p + 0.5);
    m->first_row = first_row;
    return true;
}

// What kept elements are multiplied by; where nothing is kept the factor reaches no result.
float factor_of(double scale, const ccj::Mask &m) {
    return m.threshold ? (float)(scale * 65536.0 / m.threshold) : 0.0f;
}

bool cols_ok(int32_t cols) { return cols >= 1 && cols <= ccj::kMaxCols; }

int64_t padded(int64_t k) { return (k + 15) & ~(int64_t)15; }

constexpr int64_t kMaxInt = INT32_MAX;

// The checks of a product's sizes, weights, scales and output.
bool product_ok(const void *b, int64_t b_stride, const float *b_scales, const float *bias,
                int64_t m, int64_t n, int64_t k, const void *out, int64_t out_stride, int32_t type,
                int64_t *b_bytes, int64_t *out_bytes) {
    if (m < 0 || n < 0 || k < 0 || m > kMaxInt || n > kMaxInt || k > ccj::kMaxK || !known(type))
        return false;
    if (m == 0 || n == 0)
        return true;
    const int64_t eb = ccj::type_bytes(type);
    if (!rows_ok(out, m, out_stride, n * eb, eb, out_bytes))
        return false;
    *b_bytes = 0;
    if (k > 0 && !rows_ok(b, n, b_stride, k, 16, b_bytes))
        return false;
    if (!b_scales || !aligned(b_scales, 4) || !aligned(bias, 4))
        return false;
    return !overlaps(out, *out_bytes, b, *b_bytes) && !overlaps(out, *out_bytes, b_scales, 4 * n) &&
           !overlaps(out, *out_bytes, bias, bias ? 4 * n : 0);
}

}  // namespace

extern "C" {

cc_status cc_embedding_lookup(const void *table, int64_t n_rows, int64_t table_stride,
                              int32_t table_type, const void *ids, int32_t id_bytes, int64_t n_ids,
                              int32_t cols, double scale, double p, uint64_t seed, uint32_t site,
                              int64_t first_row, void *out, int64_t out_stride, int32_t out_type,
                              hipStream_t stream) {
    ccj::RowArgs a = {};
    if (n_rows < 0 || n_ids < 0 || !cols_ok(cols) || !known(table_type) || !known(out_type) ||
        (out_type != table_type && table_type != CC_F32) || (id_bytes != 4 && id_bytes != 8))
        return CC_ERR_INVALID_ARGUMENT;
    if (!mask_of(p, seed, site, first_row, n_ids, &a.mask))
        return CC_ERR_INVALID_ARGUMENT;
    if (n_ids == 0)
        return CC_OK;
    const int64_t et = ccj::type_bytes(table_type), eo = ccj::type_bytes(out_type);
    int64_t table_bytes, out_bytes, ids_bytes;
    if (!rows_ok(table, n_rows, table_stride, cols * et, et, &table_bytes) ||
        !rows_ok(out, n_ids, out_stride, cols * eo, eo, &out_bytes) || !ids ||
        !aligned(ids, (uintptr_t)id_bytes) || !mul_ok(n_ids, id_bytes, &ids_bytes))
        return CC_ERR_INVALID_ARGUMENT;
    if (overlaps(out, out_bytes, table, table_bytes) || overlaps(out, out_bytes, ids, ids_bytes))
        return CC_ERR_INVALID_ARGUMENT;
    a.src = table;
    a.src_stride = table_stride;
    a.src_rows = n_rows;
    a.src_type = table_type;
    a.ids = ids;
    a.id_bytes = id_bytes;
    a.n = n_ids;
    a.cols = cols;
    a.out = out;
    a.out_stride = out_stride;
    a.out_type = out_type;
    a.factor = factor_of(scale, a.mask);
    const hipError_t e = ccj::launch_rows(a, stream);
    return e == hipSuccess ? CC_OK : device_error(e);
}

int64_t cc_embedding_grad_workspace_bytes(int64_t n_ids, int64_t n_rows, int32_t cols) {
    if (n_ids < 0 || n_ids > kMaxInt || n_rows < 0 || n_rows >= kMaxInt || !cols_ok(cols))
        return 0;
    return n_rows ? ccj::grad_workspace_bytes(n_ids, n_rows, cols) : 0;
}

cc_status cc_embedding_grad(const void *ids, int32_t id_bytes, int64_t n_ids, const void *grad_out,
                            int64_t grad_out_stride, int32_t grad_type, int32_t cols, double scale,
                            double p, uint64_t seed, uint32_t site, int64_t first_row,
                            int64_t n_rows, void *grad_table, int64_t grad_table_stride,
                            int32_t table_type, int32_t accumulate, void *workspace,
                            int64_t workspace_bytes, hipStream_t stream) {
    ccj::GradArgs a = {};
    if (n_ids < 0 || n_ids > kMaxInt || n_rows < 0 || n_rows >= kMaxInt || !cols_ok(cols) ||
        !known(grad_type) || !known(table_type) ||
        (table_type != grad_type && table_type != CC_F32) || (id_bytes != 4 && id_bytes != 8))
        return CC_ERR_INVALID_ARGUMENT;
    if (!mask_of(p, seed, site, first_row, n_ids, &a.mask))
        return CC_ERR_INVALID_ARGUMENT;
    if (n_rows == 0 || (n_ids == 0 && accumulate))
        return CC_OK;
    const int64_t eg = ccj::type_bytes(grad_type), et = ccj::type_bytes(table_type);
    int64_t grad_bytes, table_bytes;
    if (!rows_ok(grad_out, n_ids, grad_out_stride, cols * eg, eg, &grad_bytes) ||
        !rows_ok(grad_table, n_rows, grad_table_stride, cols * et, et, &table_bytes) ||
        (n_ids > 0 && (!ids || !aligned(ids, (uintptr_t)id_bytes))))
        return CC_ERR_INVALID_ARGUMENT;
    const int64_t need = ccj::grad_workspace_bytes(n_ids, n_rows, cols), ids_bytes = n_ids * id_bytes;
    if (need > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < need))
        return CC_ERR_INVALID_ARGUMENT;
    if (overlaps(grad_table, table_bytes, grad_out, grad_bytes) ||
        overlaps(grad_table, table_bytes, ids, ids_bytes) ||
        overlaps(grad_table, table_bytes, workspace, need) ||
        overlaps(workspace, need, grad_out, grad_bytes) || overlaps(workspace, need, ids, ids_bytes))
        return CC_ERR_INVALID_ARGUMENT;
    a.ids = ids;
    a.id_bytes = id_bytes;
    a.n = n_ids;
    a.grad = grad_out;
    a.grad_stride = grad_out_stride;
    a.grad_type = grad_type;
    a.cols = cols;
    a.rows = n_rows;
    a.table = grad_table;
    a.table_stride = grad_table_stride;
    a.table_type = table_type;
    a.accumulate = accumulate != 0;
    a.workspace = workspace;
    a.factor = factor_of(scale, a.mask);
    const hipError_t e = ccj::launch_embedding_grad(a, stream);
    return e == hipSuccess ? CC_OK : device_error(e);
}

cc_status cc_dropout(const void *x, int64_t x_stride, const void *residual,
                     int64_t residual_stride, int64_t n_rows, int32_t cols, int32_t type, double p,
                     uint64_t seed, uint32_t site, int64_t first_row, void *out,
                     int64_t out_stride, hipStream_t stream) {
    ccj::RowArgs a = {};
    if (n_rows < 0 || !cols_ok(cols) || !known(type) ||
        !mask_of(p, seed, site, first_row, n_rows, &a.mask))
        return CC_ERR_INVALID_ARGUMENT;
    if (n_rows == 0)
        return CC_OK;
    const int64_t e = ccj::type_bytes(type), width = cols * e;
    int64_t x_bytes, res_bytes = 0, out_bytes;
    if (!rows_ok(x, n_rows, x_stride, width, e, &x_bytes) ||
        (residual && !rows_ok(residual, n_rows, residual_stride, width, e, &res_bytes)) ||
        !rows_ok(out, n_rows, out_stride, width, e, &out_bytes))
        return CC_ERR_INVALID_ARGUMENT;
    // In place only element on element.
    const bool on_x = out == x && (n_rows == 1 || out_stride == x_stride);
    const bool on_res = out == residual && (n_rows == 1 || out_stride == residual_stride);
    if ((!on_x && overlaps(out, out_bytes, x, x_bytes)) ||
        (!on_res && overlaps(out, out_bytes, residual, res_bytes)))
        return CC_ERR_INVALID_ARGUMENT;
    a.src = x;
    a.src_stride = x_stride;
    a.src_rows = n_rows;
    a.src_type = type;
    a.res = residual;
    a.res_stride = residual_stride;
    a.n = n_rows;
    a.cols = cols;
    a.out = out;
    a.out_stride = out_stride;
    a.out_type = type;
    a.factor = factor_of(1.0, a.mask);
    const hipError_t err = ccj::launch_rows(a, stream);
    return err == hipSuccess ? CC_OK : device_error(err);
}

cc_status cc_quantize_rows(const void *x, int64_t x_stride, int32_t type, int64_t n_rows,
                           int32_t cols, int8_t *q, int64_t q_stride, float *scales,
                           hipStream_t stream) {
    if (n_rows < 0 || n_rows > kMaxInt || !cols_ok(cols) || !known(type))
        return CC_ERR_INVALID_ARGUMENT;
    if (n_rows == 0)
        return CC_OK;
    const int64_t e = ccj::type_bytes(type);
    int64_t x_bytes, q_bytes;
    if (!rows_ok(x, n_rows, x_stride, cols * e, e, &x_bytes) ||
        !rows_ok(q, n_rows, q_stride, padded(cols), 16, &q_bytes) || !scales || !aligned(scales, 4))
        return CC_ERR_INVALID_ARGUMENT;
    if (overlaps(q, q_bytes, x, x_bytes) || overlaps(scales, 4 * n_rows, x, x_bytes) ||
        overlaps(q, q_bytes, scales, 4 * n_rows))
        return CC_ERR_INVALID_ARGUMENT;
    const ccj::QuantizeArgs a{x, q, scales, x_stride, q_stride, n_rows, cols, type};
    const hipError_t err = ccj::launch_quantize(a, stream);
    return err == hipSuccess ? CC_OK : device_error(err);
}

int64_t cc_matmul_i8_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

cc_status cc_matmul_i8(const int8_t *a, int64_t a_stride, const float *a_scales, const int8_t *b,
                       int64_t b_stride, const float *b_scales, const float *bias, int64_t m,
                       int64_t n, int64_t k, int32_t relu, void *out, int64_t out_stride,
                       int32_t out_type, void *, int64_t, hipStream_t stream) {
    int64_t a_bytes = 0, b_bytes = 0, out_bytes = 0;
    if ((k & 15) || !product_ok(b, b_stride, b_scales, bias, m, n, k, out, out_stride, out_type,
                                &b_bytes, &out_bytes))
        return CC_ERR_INVALID_ARGUMENT;
    if (m == 0 || n == 0)
        return CC_OK;
    if ((k > 0 && !rows_ok(a, m, a_stride, k, 16, &a_bytes)) || !a_scales || !aligned(a_scales, 4) ||
        overlaps(out, out_bytes, a, a_bytes) || overlaps(out, out_bytes, a_scales, 4 * m))
        return CC_ERR_INVALID_ARGUMENT;
    const ccj::ProductArgs args{a, b, a_scales, b_scales, bias, out, a_stride, b_stride, out_stride,
                                m, n, k, out_type, relu != 0};
    const hipError_t e = ccj::launch_product(args, stream);
    return e == hipSuccess ? CC_OK : device_error(e);
}

int64_t cc_linear_i8_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (m <= 0 || n <= 0 || k <= 0 || m > kMaxInt || n > kMaxInt || k > ccj::kMaxK)
        return 0;
    return padded(4 * m) + m * padded(k);
}

cc_status cc_linear_i8(const void *x, int64_t x_stride, int32_t type, const int8_t *w,
                       int64_t w_stride, const float *w_scales, const float *bias, int64_t m,
                       int64_t n, int64_t k, int32_t relu, void *out, int64_t out_stride,
                       void *workspace, int64_t workspace_bytes, hipStream_t stream) {
    int64_t x_bytes = 0, w_bytes = 0, out_bytes = 0;
    if (k < 1 || !product_ok(w, w_stride, w_scales, bias, m, n, padded(k), out, out_stride, type,
                             &w_bytes, &out_bytes))
        return CC_ERR_INVALID_ARGUMENT;
    if (m == 0 || n == 0)
        return CC_OK;
    const int64_t e = ccj::type_bytes(type), need = cc_linear_i8_workspace_bytes(m, n, k);
    if (!rows_ok(x, m, x_stride, k * e, e, &x_bytes) || !workspace || !aligned(workspace, 16) ||
        workspace_bytes < need)
        return CC_ERR_INVALID_ARGUMENT;
    if (overlaps(out, out_bytes, x, x_bytes) || overlaps(out, out_bytes, workspace, need) ||
        overlaps(workspace, need, x, x_bytes) || overlaps(workspace, need, w, w_bytes) ||
        overlaps(workspace, need, w_scales, 4 * n) || overlaps(workspace, need, bias, bias ? 4 * n : 0))
        return CC_ERR_INVALID_ARGUMENT;
    float *scales = static_cast<float *>(workspace);
    int8_t *q = static_cast<int8_t *>(workspace) + padded(4 * m);
    const ccj::LinearArgs la{x, x_stride, (int32_t)k, type, q, scales};
    const ccj::ProductArgs args{q, w, scales, w_scales, bias, out, padded(k), w_stride, out_stride,
                                m, n, padded(k), type, relu != 0};
    const hipError_t err = ccj::launch_linear(la, args, stream);
    return err == hipSuccess ? CC_OK : device_error(err);
}

}  // extern "C"
