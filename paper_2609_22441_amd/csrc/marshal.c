/*
 * Argument marshalling of the hot entry points in native code: the checks of binding.py on plain
 * torch tensors, then the C call. Each function returns the call's status, or None when an
 * argument is anything but the plain case (another type, dtype, device or layout, too short, a
 * subclass, a raw pointer): nothing was called then, and binding.py's own checks either raise or
 * make the call. Python's attribute protocol is used throughout, so the module depends on no
 * torch header or ABI. An AttributeError, a TypeError or an OverflowError on the way means "not
 * plain"; any other exception (a KeyboardInterrupt, a MemoryError) is the caller's and is raised.
 *
 * A cc_join through binding.py's checks costs the host about 8 us, more than the kernel of a
 * request of 10,000 candidates takes (5.6 us): such requests in a row took 9.1 us each, through
 * this module 6.2.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

typedef struct cc_store cc_store;
typedef int (*info_fn)(const cc_store *, int64_t *, int32_t *);
typedef int (*join_fn)(const cc_store *, const int64_t *, int64_t, const int64_t *, int64_t,
                       const void *, int32_t, const void *, void *, int64_t, int8_t *, void *);
typedef int (*batched_fn)(const cc_store *, int32_t, const int64_t *, const int64_t *, int64_t,
                          const int64_t *, const int64_t *, int64_t, const void *, int32_t,
                          const void *, int32_t, const int64_t *const *, void *, int64_t, int8_t *,
                          void *);
typedef int (*authors_fn)(const cc_store *, int32_t, const int64_t *, const int64_t *,
                          const int64_t *, int64_t, const int64_t *, const int64_t *, int64_t,
                          const void *, int32_t, const void *, int32_t, const int64_t *const *,
                          void *, int64_t, int8_t *, void *);
typedef int (*padded_fn)(const cc_store *, int32_t, const int64_t *, const int64_t *, int64_t,
                         const int64_t *, const int64_t *, int64_t, const void *, int32_t,
                         const void *, int32_t, const int64_t *const *, int64_t, void *, int64_t,
                         int8_t *, int8_t *, void *);
typedef int (*resolve_fn)(const cc_store *, const int64_t *, int64_t, int64_t *, void *);
typedef int (*upsert_fn)(cc_store *, int64_t, const int64_t *, const int64_t *, const void *, void *,
                         int64_t, int64_t *, int64_t *, void *);
typedef int (*sort_fn)(int32_t, int32_t, int32_t, const int64_t *, const int64_t *, const void *,
                       int32_t, int64_t, int64_t, int64_t *, void *, void *, int64_t, void *);

/* include/cc_layers.h */
typedef int (*lookup_fn)(const void *, int64_t, int64_t, int32_t, const void *, int32_t, int64_t,
                         int32_t, double, double, uint64_t, uint32_t, int64_t, void *, int64_t,
                         int32_t, void *);
typedef int64_t (*grad_bytes_fn)(int64_t, int64_t, int32_t);
typedef int (*grad_fn)(const void *, int32_t, int64_t, const void *, int64_t, int32_t, int32_t,
                       double, double, uint64_t, uint32_t, int64_t, int64_t, void *, int64_t,
                       int32_t, int32_t, void *, int64_t, void *);
typedef int (*dropout_fn)(const void *, int64_t, const void *, int64_t, int64_t, int32_t, int32_t,
                          double, uint64_t, uint32_t, int64_t, void *, int64_t, void *);
typedef int (*quantize_fn)(const void *, int64_t, int32_t, int64_t, int32_t, int8_t *, int64_t,
                           float *, void *);
typedef int64_t (*product_bytes_fn)(int64_t, int64_t, int64_t);
typedef int (*matmul_fn)(const int8_t *, int64_t, const float *, const int8_t *, int64_t,
                         const float *, const float *, int64_t, int64_t, int64_t, int32_t, void *,
                         int64_t, int32_t, void *, int64_t, void *);
typedef int (*linear_fn)(const void *, int64_t, int32_t, const int8_t *, int64_t, const float *,
                         const float *, int64_t, int64_t, int64_t, int32_t, void *, int64_t, void *,
                         int64_t, void *);

typedef int (*norm_fn)(const void *, int64_t, int32_t, const void *, int64_t, const void *, int64_t,
                       int32_t, int32_t, int32_t, const float *, const float *, double, int32_t,
                       const float *, const float *, double, double, int64_t, int32_t, void *,
                       int64_t, void *, int64_t, void *);
typedef int64_t (*norm_bytes_fn)(int64_t, int32_t);
typedef int (*norm_grad_fn)(const void *, int64_t, int32_t, const void *, int64_t, const void *,
                            int64_t, int32_t, int32_t, int32_t, const float *, const float *,
                            double, int32_t, const float *, double, double, int64_t, int32_t,
                            const void *, int64_t, const void *, int64_t, void *, int64_t, void *,
                            int64_t, void *, int64_t, float *, float *, float *, float *, int32_t,
                            void *, int64_t, void *);
typedef int (*mx_quantize_fn)(const void *, int64_t, int32_t, int64_t, int32_t, uint8_t *, int64_t,
                              uint8_t *, int64_t, void *);
typedef int (*mx_dequantize_fn)(const uint8_t *, int64_t, const uint8_t *, int64_t, int64_t, int32_t,
                                void *, int64_t, int32_t, void *);
typedef int (*mx_matmul_fn)(const uint8_t *, int64_t, const uint8_t *, int64_t, const uint8_t *,
                            int64_t, const uint8_t *, int64_t, const float *, int64_t, int64_t,
                            int64_t, int32_t, void *, int64_t, int32_t, void *, int64_t, void *);
typedef int (*mx_linear_fn)(const void *, int64_t, int32_t, const uint8_t *, int64_t,
                            const uint8_t *, int64_t, const float *, int64_t, int64_t, int64_t,
                            int32_t, void *, int64_t, void *, int64_t, void *);

static PyObject *t_type, *t_i64, *t_i8;       /* torch.Tensor, torch.int64, torch.int8 */
static PyObject *t_u8;                        /* torch.uint8 */
static PyObject *t_float[3], *t_i32;          /* by type code: torch.float32, float16, bfloat16 */
static PyObject *get_device, *raw_stream;     /* () -> current device; (device) -> its stream */
static PyObject *n_get_device;
static PyObject *current_stream;              /* () -> handle of torch's current stream */
static PyObject *n_dtype, *n_is_cuda, *n_numel, *n_contiguous, *n_data_ptr, *n_shape, *n_stride,
    *n_element_size, *n_cuda_stream;

/* What a check that failed returns: 0, with no exception set if what came up (if anything) means
 * that an argument is not plain. */
static int not_plain(void) {
    if (PyErr_ExceptionMatches(PyExc_AttributeError) || PyErr_ExceptionMatches(PyExc_TypeError) ||
        PyErr_ExceptionMatches(PyExc_OverflowError))
        PyErr_Clear();
    return 0;
}

/* What a function returns after a check that failed. */
static PyObject *no_call(void) {
    if (PyErr_Occurred())
        return NULL;
    Py_RETURN_NONE;
}

/* Arguments of the plain case read as numbers; -1 when x is not that. */
static int64_t call_int(PyObject *x, PyObject *name) {
    PyObject *r = PyObject_CallMethodNoArgs(x, name);
    const int64_t v = r && PyLong_Check(r) ? PyLong_AsLongLong(r) : -1;
    Py_XDECREF(r);
    if (v == -1 && PyErr_Occurred())
        not_plain();
    return v;
}

static int is_true(PyObject *r) {             /* steals r */
    if (!r)
        return not_plain();
    const int t = r == Py_True;
    Py_DECREF(r);
    return t;
}

/* A plain tensor in GPU memory, of `dtype` unless it is NULL. */
static int plain(PyObject *x, PyObject *dtype) {
    if ((PyObject *)Py_TYPE(x) != t_type || !is_true(PyObject_GetAttr(x, n_is_cuda)))
        return 0;
    if (!dtype)
        return 1;
    PyObject *d = PyObject_GetAttr(x, n_dtype);
    if (!d)
        return not_plain();
    const int same = d == dtype;
    Py_DECREF(d);
    return same;
}

static int pointer(PyObject *x, void **p) {
    PyObject *r = PyObject_CallMethodNoArgs(x, n_data_ptr);
    if (!r)
        return not_plain();
    *p = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    return PyErr_Occurred() ? not_plain() : 1;
}

/* Dense array of at least `need` elements; *numel gets the element count. */
static int array_of(PyObject *x, PyObject *dtype, int64_t need, void **p, int64_t *numel) {
    if (!plain(x, dtype) || !is_true(PyObject_CallMethodNoArgs(x, n_contiguous)))
        return 0;
    const int64_t n = call_int(x, n_numel);
    if (n < 0 || n < need)
        return 0;
    if (numel)
        *numel = n;
    return pointer(x, p);
}

/* Sizes a tuple of two integers holds. */
static int pair_of(PyObject *t, int64_t *a, int64_t *b) {     /* steals t */
    if (!t)
        return not_plain();
    const int pair = PyTuple_Check(t) && PyTuple_GET_SIZE(t) == 2;
    if (pair) {
        *a = PyLong_AsLongLong(PyTuple_GET_ITEM(t, 0));
        if (!PyErr_Occurred())
            *b = PyLong_AsLongLong(PyTuple_GET_ITEM(t, 1));
    }
    Py_DECREF(t);
    return PyErr_Occurred() ? not_plain() : pair;
}

/* Dense [>= n, columns] array of rows; *row_bytes gets the bytes per row. */
static int rows_of(PyObject *x, int64_t n, void **p, int64_t *row_bytes) {
    int64_t r, c, e;
    if (!plain(x, NULL) || !pair_of(PyObject_GetAttr(x, n_shape), &r, &c) || r < n ||
        !is_true(PyObject_CallMethodNoArgs(x, n_contiguous)) ||
        (e = call_int(x, n_element_size)) <= 0)
        return 0;
    *row_bytes = c * e;
    return *row_bytes > 0 && *row_bytes <= INT32_MAX && pointer(x, p);
}

/* Output rows [>= n, >= width bytes] with dense rows and any row stride. */
static int out_of(PyObject *x, int64_t n, int64_t width, void **p, int64_t *stride) {
    int64_t r, c, sr, sc, e;
    if (!plain(x, NULL) || !pair_of(PyObject_GetAttr(x, n_shape), &r, &c) || r < n ||
        !pair_of(PyObject_CallMethodNoArgs(x, n_stride), &sr, &sc) || sc != 1 ||
        (e = call_int(x, n_element_size)) <= 0 || c * e < width)
        return 0;
    *stride = sr * e;
    return pointer(x, p);
}

/* NULL for None, else a dense buffer of at least `bytes` bytes. */
static int bytes_of(PyObject *x, int64_t bytes, void **p, int64_t *size) {
    int64_t n, e;
    if (x == Py_None) {
        *p = NULL;
        return size == NULL;
    }
    if (!array_of(x, NULL, 0, p, &n) || (e = call_int(x, n_element_size)) <= 0 || n * e < bytes)
        return 0;
    if (size)
        *size = n * e;
    return 1;
}

static int number(PyObject *x, int64_t *v) {  /* a plain int */
    if (!PyLong_CheckExact(x))
        return 0;
    *v = PyLong_AsLongLong(x);
    return PyErr_Occurred() ? not_plain() : 1;
}

static int address(PyObject *x, void **p) {   /* a store handle or a function: an int */
    if (!PyLong_CheckExact(x))
        return 0;
    *p = PyLong_AsVoidPtr(x);
    return PyErr_Occurred() ? not_plain() : 1;
}

/* The stream argument: None (torch's current one), a handle or a stream object. */
static int stream_of(PyObject *x, void **p) {
    if (PyLong_CheckExact(x))
        return address(x, p);
    PyObject *r = x == Py_None ? PyObject_CallNoArgs(current_stream)
                               : PyObject_GetAttr(x, n_cuda_stream);
    if (!r)
        return not_plain();
    const int ok = address(r, p);
    Py_DECREF(r);
    return ok;
}

/* Reads the store, which the library itself only compares against 0: asked when every argument has
 * passed that needs no row width, so a call that is refused for one of them reads no handle. */
static int doc_row_bytes(PyObject *info, const cc_store *s, int64_t *bytes) {
    void *f;
    int32_t w = 0;
    if (!s || !address(info, &f) || ((info_fn)f)(s, NULL, &w) != 0)
        return 0;
    *bytes = w;
    return 1;
}

#define CALL(...)                  \
    int st;                        \
    Py_BEGIN_ALLOW_THREADS         \
    st = __VA_ARGS__;              \
    Py_END_ALLOW_THREADS           \
    return PyLong_FromLong(st)

/* join(cc_join, cc_store_info, store, cand_idx, keys, feats, out, hit, default_row, stream) */
static PyObject *m_join(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *store, *cand, *keys, *feats, *out, *hit, *def, *stream;
    int64_t n, k, ew, stride, dw;
    if (n_args != 10 || !address(a[0], &fn) || !address(a[2], &store) ||
        !array_of(a[3], t_i64, 0, &cand, &n) || !array_of(a[4], t_i64, 0, &keys, &k) ||
        !rows_of(a[5], k, &feats, &ew) || !array_of(a[7], t_i8, n, &hit, NULL) ||
        !bytes_of(a[8], ew, &def, NULL) || !stream_of(a[9], &stream) ||
        !doc_row_bytes(a[1], store, &dw) || !out_of(a[6], n, dw + ew, &out, &stride))
        return no_call();
    CALL(((join_fn)fn)(store, cand, n, keys, k, feats, (int32_t)ew, def, out, stride, hit, stream));
}

/* Inputs that the batched forms share. */
typedef struct {
    void *store, *co, *cand, *ko, *keys, *feats, *def, *extra[1], *stream;
    int64_t B, tc, tk, ew, L;
} Batch;

/* a: store, cand_offsets, cand_idx, key_offsets, keys, feats, default_row, extra, stream
 * (extra: None, or the second lookup's keys). */
static int batch_of(PyObject *const *a, Batch *b) {
    int64_t nb;
    if (!address(a[0], &b->store) || !array_of(a[1], t_i64, 1, &b->co, &nb) || nb - 1 > INT32_MAX ||
        !array_of(a[2], t_i64, 0, &b->cand, &b->tc) || !array_of(a[3], t_i64, nb, &b->ko, NULL) ||
        !array_of(a[4], t_i64, 0, &b->keys, &b->tk) || !rows_of(a[5], b->tk, &b->feats, &b->ew) ||
        !bytes_of(a[6], b->ew, &b->def, NULL) || !stream_of(a[8], &b->stream))
        return 0;
    b->B = nb - 1;
    b->L = a[7] == Py_None ? 1 : 2;
    return b->L == 1 || array_of(a[7], t_i64, b->tc, &b->extra[0], NULL);
}

/* batched(cc_join_batched, cc_join_batched_authors, cc_store_info, <batch>, out, hit, author_ids) */
static PyObject *m_batched(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    Batch b;
    void *fn, *fn_authors, *out, *hit, *authors = NULL;
    int64_t stride, dw;
    if (n_args != 15 || !address(a[0], &fn) || !address(a[1], &fn_authors) || !batch_of(a + 3, &b) ||
        !array_of(a[13], t_i8, b.tc * b.L, &hit, NULL) ||
        (a[14] != Py_None && !array_of(a[14], t_i64, b.tc, &authors, NULL)) ||
        !doc_row_bytes(a[2], b.store, &dw) || !out_of(a[12], b.tc, dw + b.L * b.ew, &out, &stride))
        return no_call();
    const int64_t *const *ex = b.L == 2 ? (const int64_t *const *)b.extra : NULL;
    if (a[14] != Py_None) {
        CALL(((authors_fn)fn_authors)(b.store, (int32_t)b.B, b.co, b.cand, authors, b.tc, b.ko,
                                      b.keys, b.tk, b.feats, (int32_t)b.ew, b.def, (int32_t)b.L, ex,
                                      out, stride, hit, b.stream));
    }
    CALL(((batched_fn)fn)(b.store, (int32_t)b.B, b.co, b.cand, b.tc, b.ko, b.keys, b.tk, b.feats,
                          (int32_t)b.ew, b.def, (int32_t)b.L, ex, out, stride, hit, b.stream));
}

/* padded(cc_join_batched_padded, cc_store_info, <batch>, n_max, out, hit, valid) */
static PyObject *m_padded(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    Batch b;
    void *fn, *out, *hit, *valid;
    int64_t n_max, stride, dw;
    if (n_args != 15 || !address(a[0], &fn) || !batch_of(a + 2, &b) || !number(a[11], &n_max) ||
        n_max < 1 || n_max > INT32_MAX || !array_of(a[13], t_i8, b.B * n_max * b.L, &hit, NULL) ||
        !array_of(a[14], t_i8, b.B * n_max, &valid, NULL) || !doc_row_bytes(a[1], b.store, &dw) ||
        !out_of(a[12], b.B * n_max, dw + b.L * b.ew, &out, &stride))
        return no_call();
    const int64_t *const *ex = b.L == 2 ? (const int64_t *const *)b.extra : NULL;
    CALL(((padded_fn)fn)(b.store, (int32_t)b.B, b.co, b.cand, b.tc, b.ko, b.keys, b.tk, b.feats,
                         (int32_t)b.ew, b.def, (int32_t)b.L, ex, n_max, out, stride, hit, valid,
                         b.stream));
}

/* resolve(cc_resolve_ids, store, doc_ids, positions, stream) */
static PyObject *m_resolve(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *store, *ids, *pos, *stream;
    int64_t n;
    if (n_args != 5 || !address(a[0], &fn) || !address(a[1], &store) ||
        !array_of(a[2], t_i64, 0, &ids, &n) || !array_of(a[3], t_i64, n, &pos, NULL) ||
        !stream_of(a[4], &stream))
        return no_call();
    CALL(((resolve_fn)fn)(store, ids, n, pos, stream));
}

/* upsert(cc_store_upsert, cc_store_info, store, doc_ids, author_ids, doc_rows, workspace, stream):
 * (status, new ids, rejected records) */
static PyObject *m_upsert(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *store, *ids, *authors, *rows, *ws, *stream;
    int64_t n, dw, rb, ws_bytes, n_new = 0, n_rejected = 0;
    if (n_args != 8 || !address(a[0], &fn) || !address(a[2], &store) ||
        !array_of(a[3], t_i64, 0, &ids, &n) || !array_of(a[4], t_i64, n, &authors, NULL) ||
        !rows_of(a[5], n, &rows, &rb) || a[6] == Py_None || !bytes_of(a[6], 0, &ws, &ws_bytes) ||
        !stream_of(a[7], &stream) || !doc_row_bytes(a[1], store, &dw) || rb != dw)
        return no_call();
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = ((upsert_fn)fn)(store, n, ids, authors, rows, ws, ws_bytes, &n_new, &n_rejected, stream);
    Py_END_ALLOW_THREADS
    return Py_BuildValue("iLL", st, (long long)n_new, (long long)n_rejected);
}

/* sort(cc_sort_affinity_method, method, key_bits, key_offsets, keys_in, rows_in, keys_out, rows_out,
 * workspace, max_keys, stream) */
static PyObject *m_sort(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *ko, *ki, *ri, *k, *r, *ws, *stream;
    int64_t method, bits, nb, tk, rb, rb_out, ws_bytes, max_keys;
    if (n_args != 11 || !address(a[0], &fn) || !number(a[1], &method) || !number(a[2], &bits) ||
        method != (int32_t)method || bits != (int32_t)bits ||
        !array_of(a[3], t_i64, 1, &ko, &nb) || nb - 1 > INT32_MAX ||
        !array_of(a[4], t_i64, 0, &ki, &tk) || !rows_of(a[5], tk, &ri, &rb) ||
        !array_of(a[6], t_i64, tk, &k, NULL) || !rows_of(a[7], tk, &r, &rb_out) || rb_out != rb ||
        a[8] == Py_None || !bytes_of(a[8], 0, &ws, &ws_bytes) || !number(a[9], &max_keys) ||
        !stream_of(a[10], &stream))
        return no_call();
    CALL(((sort_fn)fn)((int32_t)method, (int32_t)bits, (int32_t)(nb - 1), ko, ki, ri, (int32_t)rb, tk,
                       max_keys, k, r, ws, ws_bytes, stream));
}

/* ---- the scoring model's input layer (layers.py) ----
 * As above; beyond it, every tensor is on the current device. */

typedef struct {
    void *p;
    int64_t stride, rows, cols;               /* the row stride in bytes */
    int32_t code;                             /* of the type: 0 to 2, -1 for int8, -2 for uint8 */
} Matrix;

/* A tensor on device *device; the first one asked (*device < 0) says which. */
static int on_device(PyObject *x, int64_t *device) {
    const int64_t d = call_int(x, n_get_device);
    if (d < 0 || (*device >= 0 && d != *device))
        return 0;
    *device = d;
    return 1;
}

/* [rows, cols] with dense rows that do not overlap, of a floating-point type, or of 8 bits: int8 for 1,
 * uint8 for 2. */
static int matrix_of(PyObject *x, int eight_bits, int64_t *device, Matrix *m) {
    static const int64_t size[] = {1, 1, 4, 2, 2};
    int64_t step, inner;
    if (!plain(x, NULL))
        return 0;
    PyObject *d = PyObject_GetAttr(x, n_dtype);
    if (!d)
        return not_plain();
    m->code = d == t_i8 ? -1 : d == t_u8 ? -2 : d == t_float[0] ? 0 : d == t_float[1] ? 1
              : d == t_float[2] ? 2 : 3;
    Py_DECREF(d);
    if (m->code == 3 || (m->code < 0 ? -m->code : 0) != eight_bits ||
        !pair_of(PyObject_GetAttr(x, n_shape), &m->rows, &m->cols) ||
        !pair_of(PyObject_CallMethodNoArgs(x, n_stride), &step, &inner) ||
        (inner != 1 && m->cols > 1) || (m->rows > 1 && step < m->cols) || !on_device(x, device))
        return 0;
    m->stride = (m->rows > 1 ? step : m->cols) * size[m->code + 2];
    return m->cols <= INT32_MAX && pointer(x, &m->p);
}

static int vector_of(PyObject *x, PyObject *dtype, int64_t need, int64_t *device, void **p) {
    return array_of(x, dtype, need, p, NULL) && on_device(x, device);
}

static int ids_of(PyObject *x, int64_t *device, void **p, int32_t *size, int64_t *n) {
    PyObject *d = PyObject_GetAttr(x, n_dtype);
    if (!d)
        return not_plain();
    *size = d == t_i64 ? 8 : d == t_i32 ? 4 : 0;
    Py_DECREF(d);
    return *size && array_of(x, NULL, 0, p, n) && on_device(x, device);
}

static int real(PyObject *x, double *v) {
    if (!PyFloat_CheckExact(x) && !PyLong_CheckExact(x))
        return 0;
    *v = PyFloat_AsDouble(x);
    return PyErr_Occurred() ? not_plain() : 1;
}

typedef struct {
    double p;
    uint64_t seed;
    uint32_t site;
    int64_t first_row;
} Drop;

/* a: p, seed, site, first_row */
static int drop_of(PyObject *const *a, Drop *d) {
    int64_t site;
    if (!real(a[0], &d->p) || !(d->p >= 0 && d->p <= 1) || !PyLong_CheckExact(a[1]) ||
        !number(a[2], &site) || site < 0 || site > UINT32_MAX || !number(a[3], &d->first_row) ||
        d->first_row < 0)
        return 0;
    d->seed = PyLong_AsUnsignedLongLongMask(a[1]);
    d->site = (uint32_t)site;
    return PyErr_Occurred() ? not_plain() : 1;
}

/* The stream argument: None is the current stream of the tensors' device, which is the current one. */
static int device_stream(PyObject *x, int64_t device, void **p) {
    PyObject *r = PyObject_CallNoArgs(get_device);
    if (!r)
        return not_plain();
    const int64_t current = PyLong_Check(r) ? PyLong_AsLongLong(r) : -1;
    int ok = current == device && !PyErr_Occurred();
    if (ok && x == Py_None) {
        PyObject *h = PyObject_CallOneArg(raw_stream, r);
        Py_DECREF(r);
        if (!h)
            return not_plain();
        ok = address(h, p);
        Py_DECREF(h);
        return ok;
    }
    Py_DECREF(r);
    return ok ? stream_of(x, p) : (PyErr_Occurred() ? not_plain() : 0);
}

static int workspace_of(PyObject *x, int64_t need, int64_t *device, void **p, int64_t *size) {
    *p = NULL;
    *size = 0;
    if (x == Py_None)
        return need == 0;
    return bytes_of(x, need, p, size) && on_device(x, device);
}

static int optional_vector(PyObject *x, int64_t need, int64_t *device, void **p) {
    *p = NULL;
    return x == Py_None || vector_of(x, t_float[0], need, device, p);
}

/* lookup(cc_embedding_lookup, table, ids, out, scale, p, seed, site, first_row, stream) */
static PyObject *m_lookup(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *ids, *stream;
    Matrix table, out;
    Drop d;
    double scale;
    int32_t id_bytes;
    int64_t n, device = -1;
    if (n_args != 10 || !address(a[0], &fn) || !matrix_of(a[1], 0, &device, &table) ||
        !ids_of(a[2], &device, &ids, &id_bytes, &n) || !matrix_of(a[3], 0, &device, &out) ||
        out.rows != n || out.cols != table.cols || (out.code != table.code && table.code != 0) ||
        !real(a[4], &scale) || !drop_of(a + 5, &d) || !device_stream(a[9], device, &stream))
        return no_call();
    CALL(((lookup_fn)fn)(table.p, table.rows, table.stride, table.code, ids, id_bytes, n,
                         (int32_t)table.cols, scale, d.p, d.seed, d.site, d.first_row, out.p,
                         out.stride, out.code, stream));
}

/* grad(cc_embedding_grad, cc_embedding_grad_workspace_bytes, ids, grad_out, grad_table, workspace,
 * scale, p, seed, site, first_row, accumulate, stream) */
static PyObject *m_grad(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *size, *ids, *ws, *stream;
    Matrix grad, table;
    Drop d;
    double scale;
    int32_t id_bytes;
    int64_t n, ws_bytes, device = -1;
    if (n_args != 13 || !address(a[0], &fn) || !address(a[1], &size) ||
        !ids_of(a[2], &device, &ids, &id_bytes, &n) || !matrix_of(a[3], 0, &device, &grad) ||
        !matrix_of(a[4], 0, &device, &table) || grad.rows != n || grad.cols != table.cols ||
        (table.code != grad.code && table.code != 0) || !real(a[6], &scale) || !drop_of(a + 7, &d) ||
        (a[11] != Py_True && a[11] != Py_False) ||
        !workspace_of(a[5], ((grad_bytes_fn)size)(n, table.rows, (int32_t)table.cols), &device, &ws,
                      &ws_bytes) ||
        !device_stream(a[12], device, &stream))
        return no_call();
    CALL(((grad_fn)fn)(ids, id_bytes, n, grad.p, grad.stride, grad.code, (int32_t)grad.cols, scale,
                       d.p, d.seed, d.site, d.first_row, table.rows, table.p, table.stride,
                       table.code, a[11] == Py_True, ws, ws_bytes, stream));
}

/* dropout(cc_dropout, x, out, p, seed, site, first_row, residual, stream) */
static PyObject *m_dropout(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *stream;
    Matrix x, out, res = {NULL, 0, 0, 0, 0};
    Drop d;
    int64_t device = -1;
    if (n_args != 9 || !address(a[0], &fn) || !matrix_of(a[1], 0, &device, &x) ||
        !matrix_of(a[2], 0, &device, &out) || out.rows != x.rows || out.cols != x.cols ||
        out.code != x.code || !drop_of(a + 3, &d) ||
        (a[7] != Py_None && (!matrix_of(a[7], 0, &device, &res) || res.rows != x.rows ||
                             res.cols != x.cols || res.code != x.code)) ||
        !device_stream(a[8], device, &stream))
        return no_call();
    CALL(((dropout_fn)fn)(x.p, x.stride, res.p, res.stride, x.rows, (int32_t)x.cols, x.code, d.p,
                          d.seed, d.site, d.first_row, out.p, out.stride, stream));
}

/* quantize(cc_quantize_rows, x, q, scales, stream) */
static PyObject *m_quantize(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *scales, *stream;
    Matrix x, q;
    int64_t device = -1;
    if (n_args != 5 || !address(a[0], &fn) || !matrix_of(a[1], 0, &device, &x) ||
        !matrix_of(a[2], 1, &device, &q) || q.rows != x.rows || q.cols != (x.cols + 15) / 16 * 16 ||
        !vector_of(a[3], t_float[0], x.rows, &device, &scales) ||
        !device_stream(a[4], device, &stream))
        return no_call();
    CALL(((quantize_fn)fn)(x.p, x.stride, x.code, x.rows, (int32_t)x.cols, q.p, q.stride, scales,
                           stream));
}

/* matmul(cc_matmul_i8, cc_matmul_i8_workspace_bytes, a, a_scales, b, b_scales, out, bias, relu,
 * workspace, stream) */
static PyObject *m_matmul(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *size, *sa, *sb, *bias, *ws, *stream;
    Matrix x, w, out;
    int64_t ws_bytes, device = -1;
    if (n_args != 11 || !address(a[0], &fn) || !address(a[1], &size) ||
        !matrix_of(a[2], 1, &device, &x) || !vector_of(a[3], t_float[0], x.rows, &device, &sa) ||
        !matrix_of(a[4], 1, &device, &w) || w.cols != x.cols ||
        !vector_of(a[5], t_float[0], w.rows, &device, &sb) || !matrix_of(a[6], 0, &device, &out) ||
        out.rows != x.rows || out.cols != w.rows ||
        !optional_vector(a[7], w.rows, &device, &bias) || (a[8] != Py_True && a[8] != Py_False) ||
        !workspace_of(a[9], ((product_bytes_fn)size)(x.rows, w.rows, x.cols), &device, &ws,
                      &ws_bytes) ||
        !device_stream(a[10], device, &stream))
        return no_call();
    CALL(((matmul_fn)fn)(x.p, x.stride, sa, w.p, w.stride, sb, bias, x.rows, w.rows, x.cols,
                         a[8] == Py_True, out.p, out.stride, out.code, ws, ws_bytes, stream));
}

/* linear(cc_linear_i8, cc_linear_i8_workspace_bytes, x, w, w_scales, out, bias, relu, workspace,
 * stream) */
static PyObject *m_linear(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *size, *sw, *bias, *ws, *stream;
    Matrix x, w, out;
    int64_t ws_bytes, device = -1;
    if (n_args != 10 || !address(a[0], &fn) || !address(a[1], &size) ||
        !matrix_of(a[2], 0, &device, &x) || !matrix_of(a[3], 1, &device, &w) ||
        w.cols != (x.cols + 15) / 16 * 16 || !vector_of(a[4], t_float[0], w.rows, &device, &sw) ||
        !matrix_of(a[5], 0, &device, &out) || out.rows != x.rows || out.cols != w.rows ||
        out.code != x.code || !optional_vector(a[6], w.rows, &device, &bias) ||
        (a[7] != Py_True && a[7] != Py_False) ||
        !workspace_of(a[8], ((product_bytes_fn)size)(x.rows, w.rows, x.cols), &device, &ws,
                      &ws_bytes) ||
        !device_stream(a[9], device, &stream))
        return no_call();
    CALL(((linear_fn)fn)(x.p, x.stride, x.code, w.p, w.stride, sw, bias, x.rows, w.rows, x.cols,
                         a[7] == Py_True, out.p, out.stride, ws, ws_bytes, stream));
}

static const Matrix no_matrix = {NULL, 0, 0, 0, 0};

/* None, or [rows, cols] of the type of `code`. */
static int optional_matrix(PyObject *x, int64_t rows, int64_t cols, int32_t code, int64_t *device,
                           Matrix *m) {
    *m = no_matrix;
    return x == Py_None || (matrix_of(x, 0, device, m) && m->rows == rows && m->cols == cols &&
                            m->code == code);
}

static int small(PyObject *x, int32_t *v) {
    int64_t n;
    if (!number(x, &n) || n != (int32_t)n)
        return 0;
    *v = (int32_t)n;
    return 1;
}

/* norm(cc_block_norm, f, y, x, gate, gate_kind, post_norm, post_weight, post_bias, post_eps, scale, h,
 * pre_norm, pre_weight, pre_bias, pre_eps, stream) */
static PyObject *m_norm(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *stream, *w, *b, *q, *c;
    Matrix f, y, x, gate, h;
    int32_t kind, post, pre;
    double post_eps, pre_eps, scale;
    int64_t device = -1;
    if (n_args != 17 || !address(a[0], &fn) || !matrix_of(a[1], 0, &device, &f) ||
        !matrix_of(a[2], 0, &device, &y) || y.rows != f.rows || y.cols != f.cols ||
        (y.code != f.code && y.code != 0) ||
        !optional_matrix(a[3], f.rows, f.cols, y.code, &device, &x) ||
        !optional_matrix(a[4], f.rows, f.cols, f.code, &device, &gate) || !small(a[5], &kind) ||
        !small(a[6], &post) || !optional_vector(a[7], f.cols, &device, &w) ||
        !optional_vector(a[8], f.cols, &device, &b) || !real(a[9], &post_eps) ||
        !real(a[10], &scale) || !optional_matrix(a[11], f.rows, f.cols, f.code, &device, &h) ||
        !small(a[12], &pre) || !optional_vector(a[13], f.cols, &device, &q) ||
        !optional_vector(a[14], f.cols, &device, &c) || !real(a[15], &pre_eps) ||
        !device_stream(a[16], device, &stream))
        return no_call();
    CALL(((norm_fn)fn)(x.p, x.stride, y.code, f.p, f.stride, gate.p, gate.stride, kind, f.code, post, w,
                       b, post_eps, pre, q, c, pre_eps, scale, f.rows, (int32_t)f.cols, y.p, y.stride,
                       h.p, h.stride, stream));
}

/* norm_grad(cc_block_norm_grad, cc_block_norm_grad_workspace_bytes, f, df, workspace, x, gate,
 * gate_kind, post_norm, post_weight, post_bias, post_eps, scale, pre_norm, pre_weight, pre_bias,
 * pre_eps, dy, dh, dx, dgate, d_post_weight, d_post_bias, d_pre_weight, d_pre_bias, accumulate,
 * stream) */
static PyObject *m_norm_grad(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *size, *stream, *ws, *w, *b, *q, *c, *sums[4];
    Matrix f, df, x, gate, dy, dh, dx, dgate;
    int32_t kind, post, pre, stream_code;
    double post_eps, pre_eps, scale;
    int64_t device = -1, ws_bytes;
    if (n_args != 27 || !address(a[0], &fn) || !address(a[1], &size) ||
        !matrix_of(a[2], 0, &device, &f))
        return no_call();
    /* The residual stream's type: that of dy, dx or x, whichever is given. */
    PyObject *first = a[17] != Py_None ? a[17] : a[19] != Py_None ? a[19] : a[5];
    stream_code = f.code;
    if (first != Py_None) {
        if (!matrix_of(first, 0, &device, &x) || (x.code != f.code && x.code != 0))
            return no_call();
        stream_code = x.code;
    }
    if ((a[17] == Py_None && a[18] == Py_None) || (a[20] != Py_None && a[6] == Py_None) ||
        (a[18] == Py_None && (a[23] != Py_None || a[24] != Py_None)) || a[3] == Py_None ||
        !optional_matrix(a[3], f.rows, f.cols, f.code, &device, &df) ||
        !optional_matrix(a[5], f.rows, f.cols, stream_code, &device, &x) ||
        !optional_matrix(a[6], f.rows, f.cols, f.code, &device, &gate) || !small(a[7], &kind) ||
        !small(a[8], &post) || !optional_vector(a[9], f.cols, &device, &w) ||
        !optional_vector(a[10], f.cols, &device, &b) || !real(a[11], &post_eps) ||
        !real(a[12], &scale) || !small(a[13], &pre) || !optional_vector(a[14], f.cols, &device, &q) ||
        !optional_vector(a[15], f.cols, &device, &c) || !real(a[16], &pre_eps) ||
        !optional_matrix(a[17], f.rows, f.cols, stream_code, &device, &dy) ||
        !optional_matrix(a[18], f.rows, f.cols, f.code, &device, &dh) ||
        !optional_matrix(a[19], f.rows, f.cols, stream_code, &device, &dx) ||
        !optional_matrix(a[20], f.rows, f.cols, f.code, &device, &dgate))
        return no_call();
    for (int i = 0; i < 4; ++i)
        if (!optional_vector(a[21 + i], f.cols, &device, &sums[i]))
            return no_call();
    if ((a[25] != Py_True && a[25] != Py_False) ||
        !workspace_of(a[4], ((norm_bytes_fn)size)(f.rows, (int32_t)f.cols), &device, &ws, &ws_bytes) ||
        !device_stream(a[26], device, &stream))
        return no_call();
    CALL(((norm_grad_fn)fn)(x.p, x.stride, stream_code, f.p, f.stride, gate.p, gate.stride, kind,
                            f.code, post, w, b, post_eps, pre, q, pre_eps, scale, f.rows,
                            (int32_t)f.cols, dy.p, dy.stride, dh.p, dh.stride, dx.p, dx.stride,
                            df.p, df.stride, dgate.p, dgate.stride, sums[0], sums[1], sums[2],
                            sums[3], a[25] == Py_True, ws, ws_bytes, stream));
}

/* Rows of k values in 4 bits with their scales. */
static int mx_of(PyObject *q, PyObject *scales, int64_t rows, int64_t k, int64_t *device, Matrix *m,
                 Matrix *s) {
    return matrix_of(q, 2, device, m) && matrix_of(scales, 2, device, s) && s->rows == m->rows &&
           (rows < 0 || m->rows == rows) && m->cols == (k + 127) / 128 * 64 &&
           s->cols == (k + 511) / 512 * 16;
}

/* mx_quantize(cc_quantize_mxfp4, x, q, scales, stream) */
static PyObject *m_mx_quantize(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *stream;
    Matrix x, q, s;
    int64_t device = -1;
    if (n_args != 5 || !address(a[0], &fn) || !matrix_of(a[1], 0, &device, &x) ||
        !mx_of(a[2], a[3], x.rows, x.cols, &device, &q, &s) || !device_stream(a[4], device, &stream))
        return no_call();
    CALL(((mx_quantize_fn)fn)(x.p, x.stride, x.code, x.rows, (int32_t)x.cols, q.p, q.stride, s.p,
                              s.stride, stream));
}

/* mx_dequantize(cc_dequantize_mxfp4, q, scales, out, stream) */
static PyObject *m_mx_dequantize(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *stream;
    Matrix out, q, s;
    int64_t device = -1;
    if (n_args != 5 || !address(a[0], &fn) || !matrix_of(a[3], 0, &device, &out) ||
        !mx_of(a[1], a[2], out.rows, out.cols, &device, &q, &s) ||
        !device_stream(a[4], device, &stream))
        return no_call();
    CALL(((mx_dequantize_fn)fn)(q.p, q.stride, s.p, s.stride, out.rows, (int32_t)out.cols, out.p,
                                out.stride, out.code, stream));
}

/* mx_matmul(cc_matmul_mxfp4, cc_matmul_mxfp4_workspace_bytes, a, a_scales, b, b_scales, out, bias, relu,
 * workspace, stream) */
static PyObject *m_mx_matmul(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *size, *bias, *ws, *stream;
    Matrix x, sx, w, sw, out;
    int64_t ws_bytes, device = -1;
    if (n_args != 11 || !address(a[0], &fn) || !address(a[1], &size) ||
        !matrix_of(a[2], 2, &device, &x) || x.cols % 64 ||
        !mx_of(a[2], a[3], -1, x.cols * 2, &device, &x, &sx) ||
        !mx_of(a[4], a[5], -1, x.cols * 2, &device, &w, &sw) || !matrix_of(a[6], 0, &device, &out) ||
        out.rows != x.rows || out.cols != w.rows ||
        !optional_vector(a[7], w.rows, &device, &bias) || (a[8] != Py_True && a[8] != Py_False) ||
        !workspace_of(a[9], ((product_bytes_fn)size)(x.rows, w.rows, x.cols * 2), &device, &ws,
                      &ws_bytes) ||
        !device_stream(a[10], device, &stream))
        return no_call();
    CALL(((mx_matmul_fn)fn)(x.p, x.stride, sx.p, sx.stride, w.p, w.stride, sw.p, sw.stride, bias,
                            x.rows, w.rows, x.cols * 2, a[8] == Py_True, out.p, out.stride, out.code,
                            ws, ws_bytes, stream));
}

/* mx_linear(cc_linear_mxfp4, cc_linear_mxfp4_workspace_bytes, x, w, w_scales, out, bias, relu, workspace,
 * stream) */
static PyObject *m_mx_linear(PyObject *self, PyObject *const *a, Py_ssize_t n_args) {
    (void)self;
    void *fn, *size, *bias, *ws, *stream;
    Matrix x, w, sw, out;
    int64_t ws_bytes, device = -1;
    if (n_args != 10 || !address(a[0], &fn) || !address(a[1], &size) ||
        !matrix_of(a[2], 0, &device, &x) || !mx_of(a[3], a[4], -1, x.cols, &device, &w, &sw) ||
        !matrix_of(a[5], 0, &device, &out) || out.rows != x.rows || out.cols != w.rows ||
        out.code != x.code || !optional_vector(a[6], w.rows, &device, &bias) ||
        (a[7] != Py_True && a[7] != Py_False) ||
        !workspace_of(a[8], ((product_bytes_fn)size)(x.rows, w.rows, x.cols), &device, &ws,
                      &ws_bytes) ||
        !device_stream(a[9], device, &stream))
        return no_call();
    CALL(((mx_linear_fn)fn)(x.p, x.stride, x.code, w.p, w.stride, sw.p, sw.stride, bias, x.rows, w.rows,
                            x.cols, a[7] == Py_True, out.p, out.stride, ws, ws_bytes, stream));
}

/* init_blocks(torch.uint8) */
static PyObject *m_init_blocks(PyObject *self, PyObject *u8) {
    (void)self;
    Py_INCREF(u8);
    Py_XSETREF(t_u8, u8);
    Py_RETURN_NONE;
}

/* init_layers(torch.float32, torch.float16, torch.bfloat16, torch.int32, get_device, raw_stream) */
static PyObject *m_init_layers(PyObject *self, PyObject *args) {
    (void)self;
    PyObject *o[6];
    if (!PyArg_ParseTuple(args, "OOOOOO", o, o + 1, o + 2, o + 3, o + 4, o + 5))
        return NULL;
    PyObject **to[] = {t_float, t_float + 1, t_float + 2, &t_i32, &get_device, &raw_stream};
    for (int i = 0; i < 6; ++i) {
        Py_INCREF(o[i]);
        Py_XSETREF(*to[i], o[i]);
    }
    Py_RETURN_NONE;
}

/* init(torch.Tensor, torch.int64, torch.int8, current_stream) */
static PyObject *m_init(PyObject *self, PyObject *args) {
    (void)self;
    PyObject *t, *i64, *i8, *cs;
    if (!PyArg_ParseTuple(args, "OOOO", &t, &i64, &i8, &cs))
        return NULL;
    Py_INCREF(t);
    Py_INCREF(i64);
    Py_INCREF(i8);
    Py_INCREF(cs);
    Py_XSETREF(current_stream, cs);
    Py_XSETREF(t_type, t);
    Py_XSETREF(t_i64, i64);
    Py_XSETREF(t_i8, i8);
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"init", m_init, METH_VARARGS, "The types the other functions accept, and the query of the current stream."},
    {"join", (PyCFunction)(void (*)(void))m_join, METH_FASTCALL, "cc_join"},
    {"batched", (PyCFunction)(void (*)(void))m_batched, METH_FASTCALL, "cc_join_batched"},
    {"padded", (PyCFunction)(void (*)(void))m_padded, METH_FASTCALL, "cc_join_batched_padded"},
    {"resolve", (PyCFunction)(void (*)(void))m_resolve, METH_FASTCALL, "cc_resolve_ids"},
    {"upsert", (PyCFunction)(void (*)(void))m_upsert, METH_FASTCALL, "cc_store_upsert"},
    {"sort", (PyCFunction)(void (*)(void))m_sort, METH_FASTCALL, "cc_sort_affinity_method"},
    {"init_layers", m_init_layers, METH_VARARGS, "The types and queries that the functions below need too."},
    {"lookup", (PyCFunction)(void (*)(void))m_lookup, METH_FASTCALL, "cc_embedding_lookup"},
    {"grad", (PyCFunction)(void (*)(void))m_grad, METH_FASTCALL, "cc_embedding_grad"},
    {"dropout", (PyCFunction)(void (*)(void))m_dropout, METH_FASTCALL, "cc_dropout"},
    {"quantize", (PyCFunction)(void (*)(void))m_quantize, METH_FASTCALL, "cc_quantize_rows"},
    {"matmul", (PyCFunction)(void (*)(void))m_matmul, METH_FASTCALL, "cc_matmul_i8"},
    {"linear", (PyCFunction)(void (*)(void))m_linear, METH_FASTCALL, "cc_linear_i8"},
    {"init_blocks", m_init_blocks, METH_O, "The type that the functions below need too."},
    {"norm", (PyCFunction)(void (*)(void))m_norm, METH_FASTCALL, "cc_block_norm"},
    {"norm_grad", (PyCFunction)(void (*)(void))m_norm_grad, METH_FASTCALL, "cc_block_norm_grad"},
    {"mx_quantize", (PyCFunction)(void (*)(void))m_mx_quantize, METH_FASTCALL, "cc_quantize_mxfp4"},
    {"mx_dequantize", (PyCFunction)(void (*)(void))m_mx_dequantize, METH_FASTCALL, "cc_dequantize_mxfp4"},
    {"mx_matmul", (PyCFunction)(void (*)(void))m_mx_matmul, METH_FASTCALL, "cc_matmul_mxfp4"},
    {"mx_linear", (PyCFunction)(void (*)(void))m_mx_linear, METH_FASTCALL, "cc_linear_mxfp4"},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal",
                                    "Native argument marshalling of the hot entry points.", -1,
                                    methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
    n_dtype = PyUnicode_InternFromString("dtype");
    n_is_cuda = PyUnicode_InternFromString("is_cuda");
    n_numel = PyUnicode_InternFromString("numel");
    n_contiguous = PyUnicode_InternFromString("is_contiguous");
    n_data_ptr = PyUnicode_InternFromString("data_ptr");
    n_shape = PyUnicode_InternFromString("shape");
    n_stride = PyUnicode_InternFromString("stride");
    n_element_size = PyUnicode_InternFromString("element_size");
    n_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    n_get_device = PyUnicode_InternFromString("get_device");
    if (!n_cuda_stream || !n_get_device || !n_dtype || !n_is_cuda || !n_numel || !n_contiguous || !n_data_ptr || !n_shape ||
        !n_stride || !n_element_size)
        return NULL;
    return PyModule_Create(&module);
}
