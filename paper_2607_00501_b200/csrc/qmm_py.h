/* qmm_py.h -- what the CPython extensions share: reading the attributes of tensors, the current stream, the call into the library. */
#ifndef QMM_PY_H
#define QMM_PY_H
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/qmm.h"

static PyObject *s_shape, *s_stride, *s_dtype, *s_data_ptr, *s_numel, *s_is_contiguous, *s_get_device;
static PyObject *device_count, *current_device, *raw_stream;         /* torch._C._cuda_getDeviceCount, _cuda_getDevice, _cuda_getCurrentRawStream */
static PyObject *dt[3], *dt_u8, *dt_i32;                              /* dtype objects */

static inline int fail_assert(const char* what, const char* why)
{
    if (!PyErr_Occurred()) PyErr_Format(PyExc_AssertionError, "%s: %s", what, why);
    return -1;
}

static inline int is_contiguous(PyObject* t)
{
    PyObject* v = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (!v) return 0;
    const int yes = v == Py_True;
    Py_DECREF(v);
    return yes;
}
static inline int64_t number(PyObject* t, PyObject* name)                   /* method without arguments that returns an integer */
{
    PyObject* v = PyObject_CallMethodNoArgs(t, name);
    if (!v) return -1;
    const int64_t n = (int64_t)PyLong_AsUnsignedLongLongMask(v);
    Py_DECREF(v);
    return n;
}
static inline int is_dtype(PyObject* t, PyObject* want)
{
    PyObject* v = PyObject_GetAttr(t, s_dtype);
    if (!v) return 0;
    Py_DECREF(v);                                                    /* (dtype objects live as long as torch) */
    return v == want;
}
static inline int pair(PyObject* tuple, int64_t* a, int64_t* b)              /* a tuple of two integers; steals the reference */
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
static inline int on_device(int64_t d, const char* what, int64_t* dev)
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

/* A 2-D CUDA tensor with contiguous rows, of any of the n types in `types` (r->dtype: which). */
static inline int get_matrix(PyObject* t, const char* what, rows_t* r, int64_t* dev, PyObject* const* types, int n, const char* wanted)
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
    for (r->dtype = 0; r->dtype < n && types[r->dtype] != d;) ++r->dtype;
    if (r->dtype == n) return fail_assert(what, wanted);
    r->ptr = (void*)number(t, s_data_ptr);
    return PyErr_Occurred() ? -1 : 0;
}
/* Of fp16, bf16 or fp32. */
static inline int get_rows(PyObject* t, const char* what, rows_t* r, int64_t* dev) { return get_matrix(t, what, r, dev, dt, 3, "fp16, bf16 or fp32 is wanted"); }

/* A contiguous CUDA tensor of type `type` with exactly (exact) or at least n elements; None gives a null pointer where `optional`. */
static inline int get_flat(PyObject* t, const char* what, PyObject* type, int64_t n, int exact, int optional, void** ptr, int64_t* dev)
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
static inline int get_stream(int64_t dev, void** stream)
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

static inline int get_ints(PyObject* const* a, int n, int64_t* out)
{
    for (int i = 0; i < n; ++i) {
        out[i] = (int64_t)PyLong_AsUnsignedLongLongMask(a[i]);
        if (out[i] == -1 && PyErr_Occurred()) return -1;
    }
    return 0;
}
/* formats and counts, which are 32-bit in the library: refused, not cut */
static inline int fits_32(int64_t v) { return v == (int32_t)v ? 0 : fail_assert("arguments", "a format or count past 32 bits"); }
static inline int get_counts(PyObject* const* a, int n, int64_t* out)
{
    for (int i = 0; i < n; ++i) {
        int over;
        out[i] = PyLong_AsLongLongAndOverflow(a[i], &over);
        if (out[i] == -1 && PyErr_Occurred()) return -1;
        if (over || fits_32(out[i])) return fits_32(INT64_MAX);
    }
    return 0;
}
static inline int arity(Py_ssize_t have, Py_ssize_t want)
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

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, NULL}

/* Names and objects of torch that the functions above read; -1 with a Python error set. */
static inline int common_init(void)
{
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* c = PyImport_ImportModule("torch._C");
    if (!torch || !c) return -1;
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
    return PyErr_Occurred() ? -1 : 0;
}

#endif
