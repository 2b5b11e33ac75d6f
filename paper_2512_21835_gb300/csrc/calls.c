/* calls.c -- the windowed-serving entry points as functions of an extension module.
 *
 * The smallest calls of these operators take the GPU two or three microseconds, and ctypes takes
 * one and a half to convert their fifteen to twenty-two arguments.  Here an argument is one C API
 * call.  Arguments and results are those of the ctypes functions, which these take the place of:
 * whole numbers, floats, and addresses as whole numbers, None or whatever ctypes takes for a pointer
 * (but text).  Two things differ: a number past its type is an OverflowError and not cut off, and what is no
 * number is a TypeError where ctypes has an ArgumentError. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <limits.h>
#include <stdint.h>

#include "../../include/loip.h"

/* Each sets *bad where Python has raised an error, and does nothing where it has before. */
static void* ptr(PyObject* o, int* bad) {
    if (*bad || o == Py_None) return NULL;
    void* p = NULL;
    if (PyLong_Check(o)) {
        p = PyLong_AsVoidPtr(o);
    } else if (PyUnicode_Check(o) || PyBytes_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "an address is a number, None or a ctypes pointer");
    } else { /* the address that ctypes would pass */
        PyObject* ctypes = PyImport_ImportModule("ctypes");
        PyObject* type = ctypes ? PyObject_GetAttrString(ctypes, "c_void_p") : NULL;
        PyObject* at = type ? PyObject_CallMethod(ctypes, "cast", "OO", o, type) : NULL;
        PyObject* v = at ? PyObject_GetAttrString(at, "value") : NULL;
        if (v && v != Py_None) p = PyLong_AsVoidPtr(v);
        Py_XDECREF(v);
        Py_XDECREF(at);
        Py_XDECREF(type);
        Py_XDECREF(ctypes);
    }
    if (!p && PyErr_Occurred()) *bad = 1;
    return p;
}
static int32_t i32(PyObject* o, int* bad) {
    if (*bad) return 0;
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        *bad = 1;
    } else if (v < INT32_MIN || v > INT32_MAX) {
        PyErr_SetString(PyExc_OverflowError, "an argument does not fit into 32 bits");
        *bad = 1;
    }
    return (int32_t)v;
}
static int64_t i64(PyObject* o, int* bad) {
    if (*bad) return 0;
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) *bad = 1;
    return v;
}
static uint64_t u64(PyObject* o, int* bad) {
    if (*bad) return 0;
    PyObject* whole = PyNumber_Index(o); /* (unlike the signed conversion, the unsigned one asks for an int) */
    const unsigned long long v = whole ? PyLong_AsUnsignedLongLong(whole) : (unsigned long long)-1;
    if (v == (unsigned long long)-1 && PyErr_Occurred()) *bad = 1;
    Py_XDECREF(whole);
    return v;
}
static float f32(PyObject* o, int* bad) {
    if (*bad) return 0.f;
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) *bad = 1;
    return (float)v;
}

#define P(i) void* const p##i = ptr(a[i], &bad)
#define I(i) const int32_t p##i = i32(a[i], &bad)
#define L(i) const int64_t p##i = i64(a[i], &bad)
#define U(i) const uint64_t p##i = u64(a[i], &bad)
#define F(i) const float p##i = f32(a[i], &bad)

/* A function of `count` arguments, which `types` takes apart into p0, p1, ... */
#define ENTRY(name, count, types, ...)                                                             \
    static PyObject* py_##name(PyObject* self, PyObject* const* a, Py_ssize_t n) {                 \
        (void)self;                                                                                \
        int bad = 0, rc;                                                                           \
        if (n != count) return PyErr_Format(PyExc_TypeError, #name " takes %d arguments", count);  \
        types;                                                                                     \
        if (bad) return NULL;                                                                      \
        Py_BEGIN_ALLOW_THREADS rc = name(__VA_ARGS__);                                             \
        Py_END_ALLOW_THREADS return PyLong_FromLong(rc);                                           \
    }

#define APPEND P(0); I(1); L(2); I(3); I(4); I(5); I(6); P(7); P(8); F(9); F(10); P(11); P(12); I(13); P(14); P(15); \
    P(16); I(17); I(18); I(19); U(20); P(21)
#define ATTENTION P(0); I(1); P(2); P(3); I(4); P(5); I(6); I(7); I(8); I(9); I(10); I(11); U(12); I(13); I(14); \
    I(15); P(16); U(17); P(18); P(19)
#define PREFILL P(0); I(1); P(2); P(3); I(4); P(5); P(6); I(7); I(8); I(9); I(10); I(11); I(12); I(13); U(14); \
    I(15); I(16); I(17); P(18); U(19); P(20); P(21)
#define READ P(0); P(1); I(2); P(3); P(4); I(5); I(6); I(7); I(8); I(9); I(10); U(11); P(12); I(13); P(14)

#define ENTRIES(suffix)                                                                                           \
    ENTRY(loip_k_qk_append##suffix, 22, APPEND, p0, p1, p2, p3, p4, p5, p6, p7, p8, p9, p10, p11, p12, p13, p14, \
          p15, p16, p17, p18, p19, p20, p21)                                                                      \
    ENTRY(loip_k_window_attention##suffix, 20, ATTENTION, p0, p1, p2, p3, p4, p5, p6, p7, p8, p9, p10, p11, p12, \
          p13, p14, p15, p16, p17, p18, p19)                                                                      \
    ENTRY(loip_k_window_prefill##suffix, 22, PREFILL, p0, p1, p2, p3, p4, p5, p6, p7, p8, p9, p10, p11, p12, p13, \
          p14, p15, p16, p17, p18, p19, p20, p21)
ENTRIES()
ENTRIES(_q8)
ENTRY(loip_k_cache_read_q8, 15, READ, p0, p1, p2, p3, p4, p5, p6, p7, p8, p9, p10, p11, p12, p13, p14)

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(loip_k_qk_append),        METHOD(loip_k_qk_append_q8),
                                METHOD(loip_k_window_attention), METHOD(loip_k_window_attention_q8),
                                METHOD(loip_k_window_prefill),   METHOD(loip_k_window_prefill_q8),
                                METHOD(loip_k_cache_read_q8),    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
