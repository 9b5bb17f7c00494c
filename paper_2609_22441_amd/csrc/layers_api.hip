// C ABI of the scoring model's layers: argument validation and the layout of workspaces. The kernels
// live in row_kernels.hip, embedding_grad_kernels.hip, i8_kernels.hip, norm_kernels.hip,
// norm_grad_kernels.hip and mx_kernels.hip.
#include <math.h>

#include <initializer_list>

#include "api_common.h"
#include "cc_layers.h"
#include "layers_internal.h"

using ccj::aligned;
using ccj::device_error;
using ccj::mul_ok;
using ccj::overlaps;

static_assert(CC_F32 == ccj::kF32 && CC_F16 == ccj::kF16 && CC_BF16 == ccj::kBF16,
              "element types of the header and the kernels agree");
static_assert(CC_NORM_NONE == ccj::kNormNone && CC_NORM_RMS == ccj::kNormRms &&
                  CC_NORM_LAYER == ccj::kNormLayer && CC_GATE_LINEAR == ccj::kGateLinear &&
                  CC_GATE_SIGMOID == ccj::kGateSigmoid,
              "norms and gates of the header and the kernels agree");

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

// What one argument spans.
struct Span {
    const void *p;
    int64_t bytes;
};

// An output overlaps none of the others.
bool apart(const Span &out, std::initializer_list<Span> others) {
    for (const Span &s : others)
        if (out.p && s.p && overlaps(out.p, out.bytes, s.p, s.bytes))
            return false;
    return true;
}

bool norm_known(int32_t norm) { return norm >= CC_NORM_NONE && norm <= CC_NORM_LAYER; }

// A norm's eps in 32 bits, whose inverse root the kernels take: not a subnormal number.
bool eps_ok(int32_t norm, double eps, float *to) {
    *to = norm == CC_NORM_NONE ? 1.0f : (float)eps;
    return *to >= 0x1p-126f && *to < INFINITY;
}

// The arguments that the norm and its gradient share, and what x, f and gate span.
bool norm_args(const void *x, int64_t x_stride, int32_t stream_type, const void *f, int64_t f_stride,
               const void *gate, int64_t gate_stride, int32_t gate_kind, int32_t type,
               int32_t post_norm, const float *post_weight, const float *post_bias, double post_eps,
               bool pre, int32_t pre_norm, const float *pre_weight, double pre_eps, double scale,
               int64_t n_rows, int32_t cols, ccj::NormArgs *a, int64_t (&bytes)[3]) {
    if (n_rows < 0 || n_rows > kMaxInt || !cols_ok(cols) || !known(type) || !known(stream_type) ||
        (stream_type != type && stream_type != CC_F32) || !norm_known(post_norm) ||
        (pre && !norm_known(pre_norm)) ||
        (gate && gate_kind != CC_GATE_LINEAR && gate_kind != CC_GATE_SIGMOID) ||
        !eps_ok(post_norm, post_eps, &a->post_eps) ||
        !eps_ok(pre ? pre_norm : CC_NORM_NONE, pre_eps, &a->pre_eps))
        return false;
    a->scale = (float)scale;
    if (!(fabsf(a->scale) < INFINITY) || !aligned(post_weight, 4) || !aligned(post_bias, 4) ||
        (pre && !aligned(pre_weight, 4)))
        return false;
    const int64_t e = ccj::type_bytes(type), es = ccj::type_bytes(stream_type);
    bytes[0] = bytes[1] = bytes[2] = 0;
    if ((x && !rows_ok(x, n_rows, x_stride, cols * es, es, &bytes[0])) ||
        !rows_ok(f, n_rows, f_stride, cols * e, e, &bytes[1]) ||
        (gate && !rows_ok(gate, n_rows, gate_stride, cols * e, e, &bytes[2])))
        return false;
    a->x = x;
    a->f = f;
    a->gate = gate;
    a->x_stride = x_stride;
    a->f_stride = f_stride;
    a->gate_stride = gate_stride;
    a->post_weight = post_weight;
    a->post_bias = post_bias;
    a->pre_weight = pre ? pre_weight : nullptr;
    a->n = n_rows;
    a->cols = cols;
    a->type = type;
    a->stream_type = stream_type;
    a->post = post_norm;
    a->pre = pre ? pre_norm : (int32_t)CC_NORM_NONE;
    a->gate_kind = gate ? gate_kind : (int32_t)ccj::kGateNone;
    return true;
}

// An output on an input of the same rows: element by element.
bool in_place(const void *out, int64_t out_stride, const void *in, int64_t in_stride, int64_t rows) {
    return out == in && (rows <= 1 || out_stride == in_stride);
}

// The checks of a 4-bit product's sizes, weights and output.
bool mx_product_ok(const void *b, int64_t b_stride, const void *b_scales, int64_t b_scales_stride,
                   const float *bias, int64_t m, int64_t n, int64_t k, const void *out,
                   int64_t out_stride, int32_t type, Span (&inputs)[3], int64_t *out_bytes) {
    if (m < 0 || n < 0 || k < 0 || m > kMaxInt || n > kMaxInt || k > ccj::kMaxCols || !known(type))
        return false;
    if (m == 0 || n == 0)
        return true;
    const int64_t eb = ccj::type_bytes(type), padded = ccj::mx_padded(k);
    int64_t b_bytes = 0, scale_bytes = 0;
    if (!rows_ok(out, m, out_stride, n * eb, eb, out_bytes) || !aligned(bias, 4))
        return false;
    if (k > 0 && (!rows_ok(b, n, b_stride, padded / 2, 16, &b_bytes) ||
                  !rows_ok(b_scales, n, b_scales_stride, ccj::mx_scales(k), 16, &scale_bytes)))
        return false;
    inputs[0] = {b, b_bytes};
    inputs[1] = {b_scales, scale_bytes};
    inputs[2] = {bias, bias ? 4 * n : 0};
    return apart({out, *out_bytes}, {inputs[0], inputs[1], inputs[2]});
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

cc_status cc_block_norm(const void *x, int64_t x_stride, int32_t stream_type, const void *f,
                        int64_t f_stride, const void *gate, int64_t gate_stride, int32_t gate_kind,
                        int32_t type, int32_t post_norm, const float *post_weight,
                        const float *post_bias, double post_eps, int32_t pre_norm,
                        const float *pre_weight, const float *pre_bias, double pre_eps,
                        double scale, int64_t n_rows, int32_t cols, void *y, int64_t y_stride,
                        void *h, int64_t h_stride, hipStream_t stream) {
    ccj::NormArgs a = {};
    int64_t bytes[3], y_bytes, h_bytes = 0;
    if (!norm_args(x, x_stride, stream_type, f, f_stride, gate, gate_stride, gate_kind, type,
                   post_norm, post_weight, post_bias, post_eps, h != nullptr, pre_norm, pre_weight,
                   pre_eps, scale, n_rows, cols, &a, bytes) ||
        (h && !aligned(pre_bias, 4)))
        return CC_ERR_INVALID_ARGUMENT;
    if (n_rows == 0)
        return CC_OK;
    const int64_t e = ccj::type_bytes(type), es = ccj::type_bytes(stream_type);
    if (!rows_ok(y, n_rows, y_stride, cols * es, es, &y_bytes) ||
        (h && !rows_ok(h, n_rows, h_stride, cols * e, e, &h_bytes)))
        return CC_ERR_INVALID_ARGUMENT;
    const int64_t vector = (int64_t)4 * cols;
    const Span sx{x, bytes[0]}, sf{f, bytes[1]}, sg{gate, bytes[2]}, sy{y, y_bytes}, sh{h, h_bytes},
        w0{post_weight, vector}, w1{post_bias, vector}, w2{h ? pre_weight : nullptr, vector},
        w3{h ? pre_bias : nullptr, vector};
    const bool on_x = in_place(y, y_stride, x, x_stride, n_rows);
    const bool on_f = in_place(h, h_stride, f, f_stride, n_rows);
    if (!apart(sy, {on_x ? Span{} : sx, sf, sg, sh, w0, w1, w2, w3}) ||
        !apart(sh, {sx, on_f ? Span{} : sf, sg, w0, w1, w2, w3}))
        return CC_ERR_INVALID_ARGUMENT;
    a.y = y;
    a.y_stride = y_stride;
    a.h = h;
    a.h_stride = h_stride;
    a.pre_bias = h ? pre_bias : nullptr;
    const hipError_t err = ccj::launch_norm(a, stream);
    return err == hipSuccess ? CC_OK : device_error(err);
}

int64_t cc_block_norm_grad_workspace_bytes(int64_t n_rows, int32_t cols) {
    if (n_rows <= 0 || n_rows > kMaxInt || !cols_ok(cols))
        return 0;
    return ccj::norm_grad_workspace_bytes(n_rows, cols);
}

cc_status cc_block_norm_grad(
    const void *x, int64_t x_stride, int32_t stream_type, const void *f, int64_t f_stride,
    const void *gate, int64_t gate_stride, int32_t gate_kind, int32_t type, int32_t post_norm,
    const float *post_weight, const float *post_bias, double post_eps, int32_t pre_norm,
    const float *pre_weight, double pre_eps, double scale, int64_t n_rows, int32_t cols,
    const void *dy, int64_t dy_stride, const void *dh, int64_t dh_stride, void *dx,
    int64_t dx_stride, void *df, int64_t df_stride, void *dgate, int64_t dgate_stride,
    float *d_post_weight, float *d_post_bias, float *d_pre_weight, float *d_pre_bias,
    int32_t accumulate, void *workspace, int64_t workspace_bytes, hipStream_t stream) {
    ccj::NormGradArgs g = {};
    int64_t bytes[3], dy_bytes = 0, dh_bytes = 0, dx_bytes = 0, df_bytes, dg_bytes = 0;
    if (!norm_args(dh ? x : nullptr, x_stride, stream_type, f, f_stride, gate, gate_stride,
                   gate_kind, type, post_norm, post_weight, post_bias, post_eps, dh != nullptr,
                   pre_norm, pre_weight, pre_eps, scale, n_rows, cols, &g.a, bytes))
        return CC_ERR_INVALID_ARGUMENT;
    const int64_t e = ccj::type_bytes(type), es = ccj::type_bytes(stream_type);
    const int64_t row = cols * e, row_s = cols * es, vector = (int64_t)4 * cols;
    float *const sums[ccj::kSums] = {d_post_weight, d_pre_weight, d_post_bias, d_pre_bias};
    for (float *s : sums)
        if (!aligned(s, 4))
            return CC_ERR_INVALID_ARGUMENT;
    if (((dgate && !gate) || ((d_pre_weight || d_pre_bias) && !dh)) && n_rows > 0)
        return CC_ERR_INVALID_ARGUMENT;
    if (n_rows > 0 &&
        ((!dy && !dh) || (dy && !rows_ok(dy, n_rows, dy_stride, row_s, es, &dy_bytes)) ||
         (dh && !rows_ok(dh, n_rows, dh_stride, row, e, &dh_bytes)) ||
         (dx && !rows_ok(dx, n_rows, dx_stride, row_s, es, &dx_bytes)) ||
         !rows_ok(df, n_rows, df_stride, row, e, &df_bytes) ||
         (dgate && !rows_ok(dgate, n_rows, dgate_stride, row, e, &dg_bytes))))
        return CC_ERR_INVALID_ARGUMENT;
    if (n_rows == 0)
        dy = dh = dx = df = dgate = nullptr, df_bytes = 0;
    const int64_t need = cc_block_norm_grad_workspace_bytes(n_rows, cols);
    if (need > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < need))
        return CC_ERR_INVALID_ARGUMENT;
    if (need == 0)
        workspace = nullptr;
    const Span in[] = {{g.a.x, bytes[0]}, {f, bytes[1]}, {gate, bytes[2]}, {dy, dy_bytes},
                       {dh, dh_bytes}, {post_weight, vector}, {post_bias, vector},
                       {g.a.pre_weight, vector}};
    const Span out[] = {{dx, dx_bytes}, {df, df_bytes}, {dgate, dg_bytes}, {sums[0], vector},
                        {sums[1], vector}, {sums[2], vector}, {sums[3], vector}, {workspace, need}};
    const bool on_dy = in_place(dx, dx_stride, dy, dy_stride, n_rows);
    const bool on_dh = in_place(df, df_stride, dh, dh_stride, n_rows);
    for (int i = 0; i < 8; ++i) {
        for (int j = 0; j < 8; ++j)
            if (!(i == 0 && j == 3 && on_dy) && !(i == 1 && j == 4 && on_dh) &&
                !apart(out[i], {in[j]}))
                return CC_ERR_INVALID_ARGUMENT;
        for (int j = 0; j < i; ++j)
            if (!apart(out[i], {out[j]}))
                return CC_ERR_INVALID_ARGUMENT;
    }
    g.dy = dy;
    g.dh = dh;
    g.dx = dx;
    g.df = df;
    g.dgate = dgate;
    g.dy_stride = dy_stride;
    g.dh_stride = dh_stride;
    g.dx_stride = dx_stride;
    g.df_stride = df_stride;
    g.dgate_stride = dgate_stride;
    for (int i = 0; i < ccj::kSums; ++i)
        g.sums[i] = sums[i];
    g.workspace = workspace;
    g.accumulate = accumulate != 0;
    const hipError_t err = ccj::launch_norm_grad(g, stream);
    return err == hipSuccess ? CC_OK : device_error(err);
}

cc_status cc_quantize_mxfp4(const void *x, int64_t x_stride, int32_t type, int64_t n_rows,
                            int32_t cols, uint8_t *q, int64_t q_stride, uint8_t *scales,
                            int64_t scales_stride, hipStream_t stream) {
    if (n_rows < 0 || n_rows > kMaxInt || !cols_ok(cols) || !known(type))
        return CC_ERR_INVALID_ARGUMENT;
    if (n_rows == 0)
        return CC_OK;
    const int64_t e = ccj::type_bytes(type);
    int64_t x_bytes, q_bytes, s_bytes;
    if (!rows_ok(x, n_rows, x_stride, cols * e, e, &x_bytes) ||
        !rows_ok(q, n_rows, q_stride, ccj::mx_padded(cols) / 2, 16, &q_bytes) ||
        !rows_ok(scales, n_rows, scales_stride, ccj::mx_scales(cols), 16, &s_bytes))
        return CC_ERR_INVALID_ARGUMENT;
    if (overlaps(q, q_bytes, x, x_bytes) || overlaps(scales, s_bytes, x, x_bytes) ||
        overlaps(q, q_bytes, scales, s_bytes))
        return CC_ERR_INVALID_ARGUMENT;
    const ccj::MxRowsArgs a{x, q, scales, x_stride, q_stride, scales_stride, n_rows, cols, type};
    const hipError_t err = ccj::launch_mx_quantize(a, stream);
    return err == hipSuccess ? CC_OK : device_error(err);
}

cc_status cc_dequantize_mxfp4(const uint8_t *q, int64_t q_stride, const uint8_t *scales,
                              int64_t scales_stride, int64_t n_rows, int32_t cols, void *out,
                              int64_t out_stride, int32_t out_type, hipStream_t stream) {
    if (n_rows < 0 || n_rows > kMaxInt || !cols_ok(cols) || !known(out_type))
        return CC_ERR_INVALID_ARGUMENT;
    if (n_rows == 0)
        return CC_OK;
    const int64_t e = ccj::type_bytes(out_type);
    int64_t out_bytes, q_bytes, s_bytes;
    if (!rows_ok(out, n_rows, out_stride, cols * e, e, &out_bytes) ||
        !rows_ok(q, n_rows, q_stride, ccj::mx_padded(cols) / 2, 16, &q_bytes) ||
        !rows_ok(scales, n_rows, scales_stride, ccj::mx_scales(cols), 16, &s_bytes))
        return CC_ERR_INVALID_ARGUMENT;
    if (overlaps(out, out_bytes, q, q_bytes) || overlaps(out, out_bytes, scales, s_bytes))
        return CC_ERR_INVALID_ARGUMENT;
    const ccj::MxRowsArgs a{out, const_cast<uint8_t *>(q), const_cast<uint8_t *>(scales), out_stride,
                            q_stride, scales_stride, n_rows, cols, out_type};
    const hipError_t err = ccj::launch_mx_dequantize(a, stream);
    return err == hipSuccess ? CC_OK : device_error(err);
}

int64_t cc_matmul_mxfp4_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

cc_status cc_matmul_mxfp4(const uint8_t *a, int64_t a_stride, const uint8_t *a_scales,
                          int64_t a_scales_stride, const uint8_t *b, int64_t b_stride,
                          const uint8_t *b_scales, int64_t b_scales_stride, const float *bias,
                          int64_t m, int64_t n, int64_t k, int32_t relu, void *out,
                          int64_t out_stride, int32_t out_type, void *, int64_t,
                          hipStream_t stream) {
    Span inputs[3];
    int64_t a_bytes = 0, s_bytes = 0, out_bytes = 0;
    if ((k & 127) || !mx_product_ok(b, b_stride, b_scales, b_scales_stride, bias, m, n, k, out,
                                    out_stride, out_type, inputs, &out_bytes))
        return CC_ERR_INVALID_ARGUMENT;
    if (m == 0 || n == 0)
        return CC_OK;
    if (k > 0 && (!rows_ok(a, m, a_stride, k / 2, 16, &a_bytes) ||
                  !rows_ok(a_scales, m, a_scales_stride, ccj::mx_scales(k), 16, &s_bytes)))
        return CC_ERR_INVALID_ARGUMENT;
    if (!apart({out, out_bytes}, {{a, a_bytes}, {a_scales, s_bytes}}))
        return CC_ERR_INVALID_ARGUMENT;
    const ccj::MxProductArgs args{a, b, a_scales, b_scales, bias, out, a_stride, b_stride,
                                  a_scales_stride, b_scales_stride, out_stride, m, n, k, out_type,
                                  relu != 0};
    const hipError_t e = ccj::launch_mx_product(args, stream);
    return e == hipSuccess ? CC_OK : device_error(e);
}

int64_t cc_linear_mxfp4_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (m <= 0 || n <= 0 || k <= 0 || m > kMaxInt || n > kMaxInt || k > ccj::kMaxCols)
        return 0;
    return m * (ccj::mx_scales(k) + ccj::mx_padded(k) / 2);
}

cc_status cc_linear_mxfp4(const void *x, int64_t x_stride, int32_t type, const uint8_t *w,
                          int64_t w_stride, const uint8_t *w_scales, int64_t w_scales_stride,
                          const float *bias, int64_t m, int64_t n, int64_t k, int32_t relu,
                          void *out, int64_t out_stride, void *workspace, int64_t workspace_bytes,
                          hipStream_t stream) {
    Span inputs[3];
    int64_t x_bytes = 0, out_bytes = 0;
    if (k < 1 || !mx_product_ok(w, w_stride, w_scales, w_scales_stride, bias, m, n, k, out,
                                out_stride, type, inputs, &out_bytes))
        return CC_ERR_INVALID_ARGUMENT;
    if (m == 0 || n == 0)
        return CC_OK;
    const int64_t e = ccj::type_bytes(type), need = cc_linear_mxfp4_workspace_bytes(m, n, k);
    if (!rows_ok(x, m, x_stride, k * e, e, &x_bytes) || !workspace || !aligned(workspace, 16) ||
        workspace_bytes < need)
        return CC_ERR_INVALID_ARGUMENT;
    if (!apart({out, out_bytes}, {{x, x_bytes}, {workspace, need}}) ||
        !apart({workspace, need}, {{x, x_bytes}, inputs[0], inputs[1], inputs[2]}))
        return CC_ERR_INVALID_ARGUMENT;
    const int64_t padded = ccj::mx_padded(k), width = ccj::mx_scales(k);
    uint8_t *scales = static_cast<uint8_t *>(workspace), *q = scales + m * width;
    const ccj::MxRowsArgs rows{x, q, scales, x_stride, padded / 2, width, m, (int32_t)k, type};
    const ccj::MxProductArgs args{q, w, scales, w_scales, bias, out, padded / 2, w_stride, width,
                                  w_scales_stride, out_stride, m, n, padded, type, relu != 0};
    const hipError_t err = ccj::launch_mx_linear(rows, args, stream);
    return err == hipSuccess ? CC_OK : device_error(err);
}

}  // extern "C"
