/*
 * The Python side of the sub-layer calls (dropout, layer normalisation and their fused form): small passes whose GPU
 * work takes 2 us, as long as generic argument conversion would.  Each function takes the arguments of its C
 * counterpart in include/qfmt.h, in order: for a pointer (the address of a record, the stream) an integer, None for NULL or
 * a tensor, whose data_ptr() is taken; for a size whatever converts to an integer.  It returns the status.  The C
 * functions are those of the library that the binding has loaded; it hands over their addresses with bind().
 */
#define PY_SSIZE_T_CLEAN
#define Py_LIMITED_API 0x030A0000
#include <Python.h>
#include <string.h>

#include "qfmt.h"

#define MOST 18

static struct {
    int (*dropout)(const void*, int64_t, const void*, int64_t, void*, int64_t, int64_t, int64_t, int32_t, const qfmt_dropout_t*, void*);
    int (*layer_norm)(const qfmt_norm_t*, const void*, const float*, const float*, void*, float*, float*, const qfmt_format_t*, qfmt_stats_t*,
                      int, void*);
    int (*layer_norm_backward)(const qfmt_norm_t*, const void*, const void*, const float*, const float*, const float*, void*, float*, float*,
                               const qfmt_format_t*, qfmt_stats_t*, int, void*, size_t, void*);
    int (*dropout_add_layer_norm)(const qfmt_norm_t*, const qfmt_dropout_t*, const void*, const void*, const float*, const float*, void*, void*,
                                  float*, float*, const qfmt_format_t*, qfmt_stats_t*, int, void*);
    int (*dropout_add_layer_norm_backward)(const qfmt_norm_t*, const qfmt_dropout_t*, const void*, const void*, const void*, const float*,
                                           const float*, const float*, void*, void*, float*, float*, const qfmt_format_t*, qfmt_stats_t*, int,
                                           void*, size_t, void*);
} lib;

static PyObject* data_ptr;  /* the method's name */

/* The arguments as 64-bit words; 0 and an exception set if one is not what `kinds` says: p a pointer, i an integer.  (A size is
 * never taken from a tensor's address.) */
static int words(PyObject* const* args, Py_ssize_t n, const char* kinds, uint64_t* v) {
    const Py_ssize_t want = (Py_ssize_t)strlen(kinds);
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
        return 0;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (PyLong_Check(args[i])) {
            v[i] = PyLong_AsUnsignedLongLongMask(args[i]);
        } else if (kinds[i] == 'p' && args[i] == Py_None) {
            v[i] = 0;
        } else {
            PyObject* p = kinds[i] == 'p' ? PyObject_CallMethodObjArgs(args[i], data_ptr, NULL) : PyNumber_Index(args[i]);
            if (p == NULL) {
                if (kinds[i] == 'p') PyErr_Format(PyExc_TypeError, "argument %zd: an address, a tensor or None expected", i);
                return 0;
            }
            v[i] = PyLong_AsUnsignedLongLongMask(p);
            Py_DECREF(p);
        }
        if (PyErr_Occurred()) return 0;
    }
    return 1;
}

#define P(i) ((void*)(uintptr_t)v[i])
#define CALL(function, kinds, ...)                                                                    \
    static PyObject* py_##function(PyObject* self, PyObject* const* args, Py_ssize_t n) {             \
        uint64_t v[MOST];                                                                             \
        int status;                                                                                   \
        (void)self;                                                                                   \
        if (!words(args, n, kinds, v)) return NULL;                                                   \
        if (lib.function == NULL) {                                                                   \
            PyErr_SetString(PyExc_RuntimeError, "the library is not loaded");                         \
            return NULL;                                                                              \
        }                                                                                             \
        Py_BEGIN_ALLOW_THREADS                                                                        \
        status = lib.function(__VA_ARGS__);                                                           \
        Py_END_ALLOW_THREADS                                                                          \
        return PyLong_FromLong(status);                                                               \
    }

CALL(dropout, "pipipiiiipp", P(0), (int64_t)v[1], P(2), (int64_t)v[3], P(4), (int64_t)v[5], (int64_t)v[6], (int64_t)v[7], (int32_t)v[8], P(9),
     P(10))
CALL(layer_norm, "pppppppppip", P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), P(8), (int)v[9], P(10))
CALL(layer_norm_backward, "pppppppppppipip", P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), P(8), P(9), P(10), (int)v[11], P(12), (size_t)v[13],
     P(14))
CALL(dropout_add_layer_norm, "ppppppppppppip", P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), P(8), P(9), P(10), P(11), (int)v[12], P(13))
CALL(dropout_add_layer_norm_backward, "ppppppppppppppipip", P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), P(8), P(9), P(10), P(11), P(12),
     P(13), (int)v[14], P(15), (size_t)v[16], P(17))

static PyObject* py_bind(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    uint64_t v[MOST];
    (void)self;
    if (!words(args, n, "ppppp", v)) return NULL;
    *(void**)&lib.dropout = P(0);
    *(void**)&lib.layer_norm = P(1);
    *(void**)&lib.layer_norm_backward = P(2);
    *(void**)&lib.dropout_add_layer_norm = P(3);
    *(void**)&lib.dropout_add_layer_norm_backward = P(4);
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(dropout), METHOD(layer_norm), METHOD(layer_norm_backward), METHOD(dropout_add_layer_norm),
                                METHOD(dropout_add_layer_norm_backward), METHOD(bind), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void) {
    data_ptr = PyUnicode_InternFromString("data_ptr");
    if (data_ptr == NULL) return NULL;
    return PyModule_Create(&module);
}
