/* qmm_layer_py.c -- argument marshalling of the router, the norm, the 8-bit rows and the adapters, as a CPython extension (see qmm_py.c:
 * these calls take microseconds on the GPU, their arguments took longer in Python and ctypes).  Checks and conversions only.     */
#include "qmm_py.h"

static PyObject* dt8[2];                                             /* torch.float8_e4m3fn, torch.int8: the number is the qmm_row_format */

/* Rows of 8 bits and their scales. */
static int get_rows8(PyObject* codes, PyObject* scales, const char* what, rows_t* r, void** s, int64_t* dev)
{
    if (get_matrix(codes, what, r, dev, dt8, 2, "torch.float8_e4m3fn or torch.int8 is wanted")) return -1;
    return get_flat(scales, "scales", dt[2], r->rows, 1, 0, s, dev);
}
/* An optional matrix of a type and shape that is given already; None: a null pointer. */
static int get_like(PyObject* t, const char* what, const rows_t* like, rows_t* r, int64_t* dev)
{
    r->ptr = NULL;
    r->ld = like->cols;
    if (t == Py_None) return 0;
    if (get_rows(t, what, r, dev)) return -1;
    if (r->rows != like->rows || r->cols != like->cols || r->dtype != like->dtype) return fail_assert(what, "another shape or type than the input's");
    return 0;
}
static int get_float(PyObject* v, float* f)
{
    *f = (float)PyFloat_AsDouble(v);
    return PyErr_Occurred() ? -1 : 0;
}

/* (logits, topk, scores, bias, groups, top_groups, group_top, renormalize, scale, idx, weights) */
static PyObject* py_expert_route(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t v[2], g[4], dev = -1;
    rows_t l;
    float scale;
    void *bias, *idx, *w, *stream;
    TRY(arity(n, 11) || get_counts(a + 1, 2, v) || get_counts(a + 4, 4, g) || get_float(a[8], &scale) || get_rows(a[0], "logits", &l, &dev));
    TRY(fits_32(l.rows) || fits_32(l.cols) || get_flat(a[3], "bias", dt[2], l.cols, 1, 1, &bias, &dev) || get_flat(a[9], "idx", dt_i32, l.rows * v[0], 1, 0, &idx, &dev) ||
        get_flat(a[10], "weights", dt[2], l.rows * v[0], 1, 0, &w, &dev) || get_stream(dev, &stream));
    CALL(qmm_expert_route((qmm_dtype)l.dtype, l.ptr, l.ld, (int32_t)l.rows, (int32_t)l.cols, (int32_t)v[0], (qmm_scores)v[1], bias, (int32_t)g[0], (int32_t)g[1], (int32_t)g[2],
                          (int32_t)g[3], scale, idx, w, stream));
}

/* (dweights, logits, idx, topk, scores, renormalize, scale, out) */
static PyObject* py_expert_route_grad(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t v[3], dev = -1;
    rows_t l, o;
    float scale;
    void *idx, *dw, *stream;
    TRY(arity(n, 8) || get_counts(a + 3, 3, v) || get_float(a[6], &scale) || get_rows(a[1], "logits", &l, &dev) || get_like(a[7], "out", &l, &o, &dev));
    UNLESS(o.ptr || l.rows == 0, "out", "a tensor is wanted");
    TRY(fits_32(l.rows) || fits_32(l.cols) || get_flat(a[0], "dweights", dt[2], l.rows * v[0], 1, 0, &dw, &dev) || get_flat(a[2], "idx", dt_i32, l.rows * v[0], 1, 0, &idx, &dev) ||
        get_stream(dev, &stream));
    CALL(qmm_expert_route_grad((qmm_dtype)l.dtype, dw, l.ptr, l.ld, idx, (int32_t)l.rows, (int32_t)l.cols, (int32_t)v[0], (qmm_scores)v[1], (int32_t)v[2], scale, o.ptr, o.ld,
                               stream));
}

/* (x, weight, eps, residual, h, y, codes, scales) */
static PyObject* py_rms_norm(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t dev = -1;
    rows_t x, r, h, y, c = {NULL, 0, 0, 0, 0};
    float eps;
    void *w, *s = NULL, *stream;
    TRY(arity(n, 8) || get_float(a[2], &eps) || get_rows(a[0], "x", &x, &dev) || get_like(a[3], "residual", &x, &r, &dev) || get_like(a[4], "h", &x, &h, &dev) ||
        get_like(a[5], "y", &x, &y, &dev));
    if (a[6] != Py_None) {
        TRY(get_rows8(a[6], a[7], "codes", &c, &s, &dev));
        UNLESS(c.rows == x.rows && c.cols == x.cols, "codes", "another shape than the input's");
    }
    TRY(get_flat(a[1], "weight", dt[x.dtype], x.cols, 1, 1, &w, &dev) || get_stream(dev, &stream));
    CALL(qmm_rms_norm((qmm_dtype)x.dtype, x.ptr, x.ld, r.ptr, r.ld, w, eps, x.rows, x.cols, h.ptr, h.ld, y.ptr, y.ld, (qmm_row_format)c.dtype, c.ptr, c.ld, s, stream));
}

/* (dy, h, weight, eps, dh, dx, dweight, ws) */
static PyObject* py_rms_norm_grad(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t dev = -1;
    rows_t dy, h, dh, dx;
    float eps;
    void *w, *dw, *ws, *stream;
    TRY(arity(n, 8) || get_float(a[3], &eps) || get_rows(a[0], "dy", &dy, &dev) || get_like(a[1], "h", &dy, &h, &dev) || get_like(a[4], "dh", &dy, &dh, &dev) ||
        get_like(a[5], "dx", &dy, &dx, &dev));
    TRY(get_flat(a[2], "weight", dt[dy.dtype], dy.cols, 1, 1, &w, &dev) || get_flat(a[6], "dweight", dt[2], dy.cols, 1, 1, &dw, &dev) ||
        get_flat(a[7], "ws", dt_u8, 0, 0, 1, &ws, &dev) || get_stream(dev, &stream));
    const int64_t ws_bytes = ws ? number(a[7], s_numel) : 0;
    CALL(qmm_rms_norm_grad((qmm_dtype)dy.dtype, dy.ptr, dy.ld, h.ptr, h.ld, w, eps, dy.rows, dy.cols, dh.ptr, dh.ld, dx.ptr, dx.ld, dw, ws, (size_t)ws_bytes, stream));
}

/* (x, codes, scales) */
static PyObject* py_rows_quantize(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t dev = -1;
    rows_t x, c;
    void *s, *stream;
    TRY(arity(n, 3) || get_rows(a[0], "x", &x, &dev) || get_rows8(a[1], a[2], "codes", &c, &s, &dev));
    UNLESS(c.rows == x.rows && c.cols == x.cols, "codes", "another shape than the input's");
    TRY(get_stream(dev, &stream));
    CALL(qmm_rows_quantize((qmm_dtype)x.dtype, x.ptr, x.ld, x.rows, x.cols, (qmm_row_format)c.dtype, c.ptr, c.ld, s, stream));
}

/* (codes, scales, out) */
static PyObject* py_rows_dequantize(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t dev = -1;
    rows_t o, c;
    void *s, *stream;
    TRY(arity(n, 3) || get_rows(a[2], "out", &o, &dev) || get_rows8(a[0], a[1], "codes", &c, &s, &dev));
    UNLESS(c.rows == o.rows && c.cols == o.cols, "out", "another shape than the codes'");
    TRY(get_stream(dev, &stream));
    CALL(qmm_rows_dequantize((qmm_row_format)c.dtype, c.ptr, c.ld, s, o.rows, o.cols, (qmm_dtype)o.dtype, o.ptr, o.ld, stream));
}

/* What both directions of the adapters read: x (or None), x_scale, idx, a [n, r, K], b [n, N, r], scale, and a plan's order, offsets, units (0: none), device */
static int shape3(PyObject* t, const char* what, int64_t* d)
{
    PyObject* s = PyObject_GetAttr(t, s_shape);
    if (!s) return -1;
    int ok = PyTuple_Check(s) && PyTuple_GET_SIZE(s) == 3;
    for (int i = 0; ok && i < 3; ++i) d[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(s, i));
    Py_DECREF(s);
    return ok ? 0 : fail_assert(what, "a 3-D tensor is wanted");
}
static int get_adapters(PyObject* const* v, qmm_lora_args* q, int64_t rows, int dtype, int64_t* dev)
{
    int64_t da[3], db[3], plan[4];
    rows_t x = {NULL, 0, 0, 0, 0};
    void *p, *b;
    if (shape3(v[3], "a", da) || shape3(v[4], "b", db)) return -1;
    if (da[0] != db[0] || da[1] != db[2]) return fail_assert("b", "[n, N, r] beside a [n, r, K] is wanted");
    q->T = (int32_t)rows, q->n = (int32_t)da[0], q->r = (int32_t)da[1], q->K = da[2], q->N = db[1];
    q->dtype = dtype;
    if (fits_32(rows) || fits_32(da[0]) || fits_32(da[1])) return -1;
    if (get_flat(v[3], "a", dt[dtype], da[0] * da[1] * da[2], 1, 0, &p, dev) || get_flat(v[4], "b", dt[dtype], db[0] * db[1] * db[2], 1, 0, &b, dev)) return -1;
    q->A = p, q->B = b;
    if (v[0] != Py_None) {
        if (v[1] != Py_None) {
            if (get_rows8(v[0], v[1], "x", &x, &p, dev)) return -1;
            q->x_scale = p, q->x_format = x.dtype;
        } else {
            if (get_rows(v[0], "x", &x, dev)) return -1;
            if (x.dtype != dtype) return fail_assert("x", "another type than the other rows (or 8 bits without x_scale)");
        }
        if (x.rows != rows || x.cols != da[2]) return fail_assert("x", "[T, K] is wanted");
        q->X = x.ptr, q->ldx = x.ld;
    }
    if (get_flat(v[2], "idx", dt_i32, rows, 1, 0, &p, dev)) return -1;
    q->idx = p;
    if (get_flat(v[5], "scale", dt[2], da[0], 1, 1, &p, dev)) return -1;
    q->scale = p;
    if (get_ints(v + 6, 4, plan)) return -1;
    if (plan[0]) {
        if (on_device(plan[3], "plan", dev)) return -1;
        q->order = (const int32_t*)plan[0], q->offsets = (const int32_t*)plan[1], q->units = (const int32_t*)plan[2];
    }
    return 0;
}
/* An optional fp32 tensor of n elements. */
static int get_f32(PyObject* t, const char* what, int64_t n, float** out, int64_t* dev)
{
    void* p;
    if (get_flat(t, what, dt[2], n, 1, 1, &p, dev)) return -1;
    *out = p;
    return 0;
}

/* (x, x_scale, idx, a, b, scale, order, offsets, units, device, s, y0, y, ws) */
static PyObject* py_lora(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t dev = -1;
    rows_t y, y0;
    qmm_lora_args q = {0};
    void *ws, *stream;
    TRY(arity(n, 14) || get_rows(a[12], "out", &y, &dev) || get_adapters(a, &q, y.rows, y.dtype, &dev) || get_like(a[11], "y0", &y, &y0, &dev));
    UNLESS(y.cols == q.N, "out", "[T, N] is wanted");
    UNLESS(a[0] != Py_None, "x", "a tensor is wanted");
    TRY(get_f32(a[10], "s", y.rows * q.r, &q.S, &dev) || get_flat(a[13], "ws", dt_u8, 0, 0, 1, &ws, &dev) || get_stream(dev, &stream));
    q.Y0 = y0.ptr, q.ldy0 = y0.ld, q.Y = y.ptr, q.ldy = y.ld;
    const int64_t ws_bytes = ws ? number(a[13], s_numel) : 0;
    CALL(qmm_lora(&q, ws, (size_t)ws_bytes, stream));
}

/* (x, x_scale, idx, a, b, scale, order, offsets, units, device, s, dy, dx0, dx, da, db, ws) */
static PyObject* py_lora_grad(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t dev = -1;
    rows_t dy, dx, dx0, like;
    qmm_lora_args q = {0};
    void *ws, *stream;
    TRY(arity(n, 17) || get_rows(a[11], "dy", &dy, &dev) || get_adapters(a, &q, dy.rows, dy.dtype, &dev));
    UNLESS(dy.cols == q.N, "dy", "[T, N] is wanted");
    like = dy;
    like.cols = q.K;
    TRY(get_like(a[12], "dx0", &like, &dx0, &dev) || get_like(a[13], "dx", &like, &dx, &dev));
    TRY(get_f32(a[10], "s", dy.rows * q.r, &q.S, &dev) || get_f32(a[14], "da", (int64_t)q.n * q.r * q.K, &q.dA, &dev) || get_f32(a[15], "db", (int64_t)q.n * q.r * q.N, &q.dB, &dev) ||
        get_flat(a[16], "ws", dt_u8, 0, 0, 1, &ws, &dev) || get_stream(dev, &stream));
    UNLESS(!q.dA || q.X || q.T == 0, "x", "a tensor is wanted for da");
    q.dY = dy.ptr, q.lddy = dy.ld, q.dX0 = dx0.ptr, q.lddx0 = dx0.ld, q.dX = dx.ptr, q.lddx = dx.ld;
    const int64_t ws_bytes = ws ? number(a[16], s_numel) : 0;
    CALL(qmm_lora_grad(&q, ws, (size_t)ws_bytes, stream));
}

static PyMethodDef methods[] = {METHOD(expert_route),    METHOD(expert_route_grad), METHOD(rms_norm), METHOD(rms_norm_grad), METHOD(rows_quantize),
                                METHOD(rows_dequantize), METHOD(lora),              METHOD(lora_grad), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_qmm_layer_py", "Argument marshalling of libqmm's router, norm and adapters.", -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__qmm_layer_py(void)
{
    if (common_init()) return NULL;
    PyObject* torch = PyImport_ImportModule("torch");
    if (!torch) return NULL;
    dt8[0] = PyObject_GetAttrString(torch, "float8_e4m3fn");
    dt8[1] = PyObject_GetAttrString(torch, "int8");
    Py_DECREF(torch);
    if (PyErr_Occurred()) return NULL;
    return PyModule_Create(&module);
}
