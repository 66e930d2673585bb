/* qmm_py.c -- argument marshalling of the short hot-path calls of qmm.py, as a CPython extension.
 *
 * A call of the expert sort or of a microscaled product of few rows keeps the GPU busy for 2 to 7 us; checking and
 * converting its arguments in Python and ctypes took 3 us beside a launch of 2.6.  These wrappers read the tensors' attributes
 * and call the C ABI directly (0.5 us).  They only check and convert: every step of every operator runs in libqmm's kernels.
 * Each returns the qmm_status; wrong tensors raise AssertionError, like the asserts of the other wrappers.
 * A kernel runs on the current device, in its current stream: tensors of another device are refused.                     */
#include "qmm_py.h"

/* Elements of a packed operand (for an unknown format the library's own refusal follows). */
static int64_t packed_need(int64_t fmt, int64_t rows, int64_t K) { return rows > 0 ? (int64_t)qmm_mx_bytes((qmm_mx_format)fmt, rows, K) : 0; }

/* (fmt, x, out, tensor_scale) */
static PyObject* py_mx_quantize(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t fmt, dev = -1;
    rows_t x;
    void *out, *scale, *stream;
    TRY(arity(n, 4) || get_counts(a, 1, &fmt) || get_rows(a[1], "x", &x, &dev));
    TRY(get_flat(a[2], "out", dt_u8, packed_need(fmt, x.rows, x.cols), 0, 0, &out, &dev) || get_flat(a[3], "tensor_scale", dt[2], 1, 1, 1, &scale, &dev) || get_stream(dev, &stream));
    CALL(qmm_mx_quantize((qmm_mx_format)fmt, (qmm_dtype)x.dtype, x.ptr, x.ld, x.rows, x.cols, scale, out, stream));
}

/* (fmt, packed, out, tensor_scale) */
static PyObject* py_mx_dequantize(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t fmt, dev = -1;
    rows_t o;
    void *packed, *scale, *stream;
    TRY(arity(n, 4) || get_counts(a, 1, &fmt) || get_rows(a[2], "out", &o, &dev));
    TRY(get_flat(a[1], "packed", dt_u8, packed_need(fmt, o.rows, o.cols), 0, 0, &packed, &dev) || get_flat(a[3], "tensor_scale", dt[2], 1, 1, 1, &scale, &dev) || get_stream(dev, &stream));
    CALL(qmm_mx_dequantize((qmm_mx_format)fmt, packed, o.rows, o.cols, scale, (qmm_dtype)o.dtype, o.ptr, o.ld, stream));
}

/* (fmt, X, w, N, Y, x_scale, w_scale, ws) */
static PyObject* py_mx_linear(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t fmt, N, dev = -1;
    rows_t x, y;
    void *w, *xs, *wsc, *ws, *stream;
    TRY(arity(n, 8) || get_counts(a, 1, &fmt) || get_ints(a + 3, 1, &N) || get_rows(a[1], "X", &x, &dev) || get_rows(a[4], "Y", &y, &dev));
    UNLESS(y.rows == x.rows && y.cols == N && y.dtype == x.dtype, "Y", "[M, N] of X's type is wanted");
    TRY(get_flat(a[2], "w", dt_u8, packed_need(fmt, N, x.cols), 0, 0, &w, &dev) || get_flat(a[5], "x_scale", dt[2], 1, 1, 1, &xs, &dev) ||
        get_flat(a[6], "w_scale", dt[2], 1, 1, 1, &wsc, &dev) || get_flat(a[7], "ws", dt_u8, 0, 0, 0, &ws, &dev) || get_stream(dev, &stream));
    const int64_t ws_bytes = number(a[7], s_numel);
    CALL(qmm_mx_linear((qmm_mx_format)fmt, (qmm_dtype)x.dtype, x.ptr, x.ld, x.rows, w, N, x.cols, xs, wsc, y.ptr, y.ld, ws, (size_t)ws_bytes, stream));
}

/* (idx, E, order, place, offsets, units, ws, ws_bytes, device): the plan's arrays as addresses, and their device */
static PyObject* py_expert_sort(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t v[8], T, topk, dev = -1;
    void *idx, *stream;
    TRY(arity(n, 9) || get_counts(a + 1, 1, v) || get_ints(a + 2, 7, v + 1) || on_device(v[7], "plan", &dev));
    TRY(get_flat(a[0], "idx", dt_i32, 0, 0, 0, &idx, &dev));
    if (pair(PyObject_GetAttr(a[0], s_shape), &T, &topk)) return fail_assert("idx", "[T, topk] is wanted"), NULL;
    TRY(fits_32(T) || fits_32(topk) || get_stream(dev, &stream));
    CALL(qmm_expert_sort(idx, (int32_t)T, (int32_t)topk, (int32_t)v[0], (int32_t*)v[1], (int32_t*)v[2], (int32_t*)v[3], (int32_t*)v[4], (void*)v[5],
                                           (size_t)v[6], stream));
}

/* (x, T, topk, order, place, device, weights, xs) */
static PyObject* py_expert_gather(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t v[5], dev = -1;
    rows_t x, o;
    void *w, *stream;
    TRY(arity(n, 8) || get_counts(a + 1, 2, v) || get_ints(a + 3, 3, v + 2) || on_device(v[4], "plan", &dev) || get_rows(a[0], "x", &x, &dev) || get_rows(a[7], "out", &o, &dev));
    UNLESS(x.rows == v[0] && o.rows == v[0] * v[1] && o.cols == x.cols && o.dtype == x.dtype, "out", "x [T, H] and out [T * topk, H] of one type are wanted");
    TRY(get_flat(a[6], "weights", dt[2], v[0] * v[1], 1, 1, &w, &dev) || get_stream(dev, &stream));
    CALL(qmm_expert_gather((qmm_dtype)x.dtype, x.ptr, x.ld, (int32_t)v[0], (int32_t)v[1], x.cols, (const int32_t*)v[2], (const int32_t*)v[3], w, o.ptr,
                                             o.ld, stream));
}

/* (ys, T, topk, place, device, weights, y) */
static PyObject* py_expert_combine(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t v[4], dev = -1;
    rows_t y, o;
    void *w, *stream;
    TRY(arity(n, 7) || get_counts(a + 1, 2, v) || get_ints(a + 3, 2, v + 2) || on_device(v[3], "plan", &dev) || get_rows(a[0], "ys", &y, &dev) || get_rows(a[6], "out", &o, &dev));
    UNLESS(y.rows == v[0] * v[1] && o.rows == v[0] && o.cols == y.cols && o.dtype == y.dtype, "out", "ys [T * topk, H] and out [T, H] of one type are wanted");
    TRY(get_flat(a[5], "weights", dt[2], v[0] * v[1], 1, 1, &w, &dev) || get_stream(dev, &stream));
    CALL(qmm_expert_combine((qmm_dtype)y.dtype, y.ptr, y.ld, (int32_t)v[0], (int32_t)v[1], y.cols, (const int32_t*)v[2], w, o.ptr, o.ld, stream));
}

/* (dy, ys, T, topk, order, place, device, weights, dys, dw) */
static PyObject* py_expert_combine_grad(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    int64_t v[5], dev = -1;
    rows_t d, y, o;
    void *w, *dw, *stream;
    TRY(arity(n, 10) || get_counts(a + 2, 2, v) || get_ints(a + 4, 3, v + 2) || on_device(v[4], "plan", &dev) || get_rows(a[0], "dy", &d, &dev) || get_rows(a[1], "ys", &y, &dev) || get_rows(a[8], "dys", &o, &dev));
    UNLESS(d.rows == v[0] && y.rows == v[0] * v[1] && o.rows == y.rows && y.cols == d.cols && o.cols == d.cols && y.dtype == d.dtype && o.dtype == d.dtype, "dys",
           "dy [T, H], ys and dys [T * topk, H] of one type are wanted");
    TRY(get_flat(a[7], "weights", dt[2], v[0] * v[1], 1, 1, &w, &dev) || get_flat(a[9], "dw", dt[2], v[0] * v[1], 1, 0, &dw, &dev) || get_stream(dev, &stream));
    CALL(qmm_expert_combine_grad((qmm_dtype)d.dtype, d.ptr, d.ld, y.ptr, y.ld, (int32_t)v[0], (int32_t)v[1], d.cols, (const int32_t*)v[2],
                                                   (const int32_t*)v[3], w, o.ptr, o.ld, dw, stream));
}

static PyMethodDef methods[] = {METHOD(mx_quantize),   METHOD(mx_dequantize),  METHOD(mx_linear),           METHOD(expert_sort),
                                METHOD(expert_gather), METHOD(expert_combine), METHOD(expert_combine_grad), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_qmm_py", "Argument marshalling of hot-path calls of libqmm.", -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__qmm_py(void)
{
    if (common_init()) return NULL;
    return PyModule_Create(&module);
}
