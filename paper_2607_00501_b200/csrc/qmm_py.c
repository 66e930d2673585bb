/* qmm_py.c -- argument marshalling of the short hot-path calls of qmm.py, as a CPython extension.
 *
 * A call of the expert sort or of a microscaled product of few rows keeps the GPU busy for 2 to 7 us; checking and
 * converting its arguments in Python and ctypes took 3 us beside a launch of 2.6.  These wrappers read the tensors' attributes
 * and call the C ABI directly (0.5 us).  They only check and convert: every step of every operator runs in libqmm's kernels.
 * Each returns the qmm_status; wrong tensors raise AssertionError, like the asserts of the other wrappers.
 * A kernel runs on the current device, in its current stream: tensors of another device are refused.                     */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/qmm.h"

static PyObject *s_shape, *s_stride, *s_dtype, *s_data_ptr, *s_numel, *s_is_contiguous, *s_get_device;
static PyObject *device_count, *current_device, *raw_stream;         /* torch._C._cuda_getDeviceCount, _cuda_getDevice, _cuda_getCurrentRawStream */
static PyObject *dt[3], *dt_u8, *dt_i32;                              /* dtype objects */

static int fail_assert(const char* what, const char* why)
{
    if (!PyErr_Occurred()) PyErr_Format(PyExc_AssertionError, "%s: %s", what, why);
    return -1;
}

static int is_contiguous(PyObject* t)
{
    PyObject* v = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (!v) return 0;
    const int yes = v == Py_True;
    Py_DECREF(v);
    return yes;
}
static int64_t number(PyObject* t, PyObject* name)                   /* method without arguments that returns an integer */
{
    PyObject* v = PyObject_CallMethodNoArgs(t, name);
    if (!v) return -1;
    const int64_t n = (int64_t)PyLong_AsUnsignedLongLongMask(v);
    Py_DECREF(v);
    return n;
}
static int is_dtype(PyObject* t, PyObject* want)
{
    PyObject* v = PyObject_GetAttr(t, s_dtype);
    if (!v) return 0;
    Py_DECREF(v);                                                    /* (dtype objects live as long as torch) */
    return v == want;
}
static int pair(PyObject* tuple, int64_t* a, int64_t* b)              /* a tuple of two integers; steals the reference */
{
    if (!tuple) return -1;
    int ok = PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) == 2;
    if (ok) {
        *a = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, 0));
        *b = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, 1));
    }
    Py_DECREF(tuple);
    return ok ? 0 : -1;
}

/* All tensors (and the plan) of a call are on one device: *dev, -1 before the first. */
static int on_device(int64_t d, const char* what, int64_t* dev)
{
    if (d < 0) return fail_assert(what, "a CUDA tensor is wanted");
    if (*dev < 0) *dev = d;
    return d == *dev ? 0 : fail_assert(what, "on another device than the tensors before it");
}

typedef struct {
    void* ptr;
    int64_t ld, rows, cols;
    int dtype;
} rows_t;

/* A 2-D CUDA tensor with contiguous rows of fp16, bf16 or fp32. */
static int get_rows(PyObject* t, const char* what, rows_t* r, int64_t* dev)
{
    int64_t inner;
    if (on_device(number(t, s_get_device), what, dev)) return -1;    /* (-1: a CPU tensor) */
    if (pair(PyObject_GetAttr(t, s_shape), &r->rows, &r->cols) || pair(PyObject_CallMethodNoArgs(t, s_stride), &r->ld, &inner))
        return fail_assert(what, "a 2-D tensor is wanted");
    if (inner != 1 && r->cols > 1) return fail_assert(what, "rows must be contiguous");
    if (r->rows <= 1 && r->ld < r->cols) r->ld = r->cols;
    PyObject* d = PyObject_GetAttr(t, s_dtype);
    if (!d) return -1;
    Py_DECREF(d);
    for (r->dtype = 0; r->dtype < 3 && dt[r->dtype] != d;) ++r->dtype;
    if (r->dtype == 3) return fail_assert(what, "fp16, bf16 or fp32 is wanted");
    r->ptr = (void*)number(t, s_data_ptr);
    return PyErr_Occurred() ? -1 : 0;
}

/* A contiguous CUDA tensor of type `type` with exactly (exact) or at least n elements; None gives a null pointer where `optional`. */
static int get_flat(PyObject* t, const char* what, PyObject* type, int64_t n, int exact, int optional, void** ptr, int64_t* dev)
{
    *ptr = NULL;
    if (t == Py_None) return optional ? 0 : fail_assert(what, "a tensor is wanted");
    if (on_device(number(t, s_get_device), what, dev)) return -1;
    if (!is_dtype(t, type) || !is_contiguous(t)) return fail_assert(what, "a contiguous CUDA tensor of the right type is wanted");
    const int64_t have = number(t, s_numel);
    if (exact ? have != n : have < n) {
        if (!PyErr_Occurred()) PyErr_Format(PyExc_AssertionError, "%s: %lld elements, %lld needed", what, (long long)have, (long long)n);
        return -1;
    }
    *ptr = (void*)number(t, s_data_ptr);
    return PyErr_Occurred() ? -1 : 0;
}

/* Current stream of device `dev`, which has to be the current device (with one GPU there is no other: asking takes 0.2 us). */
static int get_stream(int64_t dev, void** stream)
{
    static int gpus = 0;
    PyObject* v;
    if (gpus == 0) {
        if (!(v = PyObject_CallNoArgs(device_count))) return -1;
        gpus = (int)PyLong_AsLong(v);
        Py_DECREF(v);
    }
    if (gpus != 1) {
        if (!(v = PyObject_CallNoArgs(current_device))) return -1;
        const long long now = PyLong_AsLongLong(v);
        Py_DECREF(v);
        if (now != dev) {
            if (!PyErr_Occurred()) PyErr_Format(PyExc_AssertionError, "the tensors are on device %lld, the current device is %lld", (long long)dev, now);
            return -1;
        }
    }
    PyObject* d = PyLong_FromLongLong(dev);
    if (!d) return -1;
    v = PyObject_CallOneArg(raw_stream, d);
    Py_DECREF(d);
    if (!v) return -1;
    *stream = (void*)PyLong_AsUnsignedLongLongMask(v);
    Py_DECREF(v);
    return 0;
}

static int get_ints(PyObject* const* a, int n, int64_t* out)
{
    for (int i = 0; i < n; ++i) {
        out[i] = (int64_t)PyLong_AsUnsignedLongLongMask(a[i]);
        if (out[i] == -1 && PyErr_Occurred()) return -1;
    }
    return 0;
}
/* formats and counts, which are 32-bit in the library: refused, not cut */
static int fits_32(int64_t v) { return v == (int32_t)v ? 0 : fail_assert("arguments", "a format or count past 32 bits"); }
static int get_counts(PyObject* const* a, int n, int64_t* out)
{
    for (int i = 0; i < n; ++i) {
        int over;
        out[i] = PyLong_AsLongLongAndOverflow(a[i], &over);
        if (out[i] == -1 && PyErr_Occurred()) return -1;
        if (over || fits_32(out[i])) return fits_32(INT64_MAX);
    }
    return 0;
}
static int arity(Py_ssize_t have, Py_ssize_t want)
{
    if (have == want) return 0;
    PyErr_Format(PyExc_TypeError, "%zd arguments wanted, %zd given", want, have);
    return -1;
}

/* The library's call, its status the result.  Other Python threads run meanwhile: a launch waits where the launch queue is full, and the stream before it may wait
 * for a host function that needs the interpreter. */
#define CALL(expr)                      \
    do {                                \
        qmm_status status_;             \
        Py_BEGIN_ALLOW_THREADS          \
        status_ = expr;                 \
        Py_END_ALLOW_THREADS            \
        return PyLong_FromLong(status_); \
    } while (0)
#define TRY(x) \
    if (x) return NULL
#define UNLESS(cond, what, why) \
    if (!(cond)) return fail_assert(what, why), NULL

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

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(mx_quantize),   METHOD(mx_dequantize),  METHOD(mx_linear),           METHOD(expert_sort),
                                METHOD(expert_gather), METHOD(expert_combine), METHOD(expert_combine_grad), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_qmm_py", "Argument marshalling of hot-path calls of libqmm.", -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__qmm_py(void)
{
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* c = PyImport_ImportModule("torch._C");
    if (!torch || !c) return NULL;
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_numel = PyUnicode_InternFromString("numel");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_get_device = PyUnicode_InternFromString("get_device");
    device_count = PyObject_GetAttrString(c, "_cuda_getDeviceCount");
    current_device = PyObject_GetAttrString(c, "_cuda_getDevice");
    raw_stream = PyObject_GetAttrString(c, "_cuda_getCurrentRawStream");
    dt[0] = PyObject_GetAttrString(torch, "float16");
    dt[1] = PyObject_GetAttrString(torch, "bfloat16");
    dt[2] = PyObject_GetAttrString(torch, "float32");
    dt_u8 = PyObject_GetAttrString(torch, "uint8");
    dt_i32 = PyObject_GetAttrString(torch, "int32");
    Py_DECREF(torch);
    Py_DECREF(c);
    if (PyErr_Occurred()) return NULL;
    return PyModule_Create(&module);
}
