/*
 * The Python side of the sub-layer calls (dropout, layer normalisation and their fused form) and of the calls around a step's last
 * products (products with an epilogue, cross entropy, clipping): small passes whose GPU work takes 2 us, as long as generic argument
 * conversion would.  Each function takes the arguments of its C
 * counterpart in include/qfmt.h, in order: for a pointer (the address of a record, the stream) an integer, None for NULL or
 * a tensor, whose data_ptr() is taken; for a size whatever converts to an integer; for a float a number.  It returns the status.  The C
 * functions are those of the library that the binding has loaded; it hands over their addresses with bind() and bind_step().
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
    int (*linear_act)(const qfmt_matrix16_t*, const qfmt_matrix16_t*, const qfmt_epilogue_t*, void*, int64_t, int32_t, void*, size_t, void*);
    int (*linear_act_backward)(const qfmt_matrix16_t*, const qfmt_matrix16_t*, const qfmt_epilogue_t*, void*, int64_t, float*, int32_t, void*,
                               size_t, void*);
    int (*act_backward)(const void*, int64_t, const void*, int64_t, void*, int64_t, float*, int64_t, int64_t, int32_t, int32_t, void*, size_t,
                        void*);
    int (*linear_cross_entropy)(const qfmt_matrix16_t*, const qfmt_matrix16_t*, const qfmt_cross_entropy_t*, const float*, const int64_t*, float*,
                                float*, float*, void*, size_t, void*);
    int (*linear_cross_entropy_backward)(const qfmt_matrix16_t*, const qfmt_matrix16_t*, const qfmt_cross_entropy_t*, const float*,
                                         const int64_t*, const float*, const float*, const qfmt_dls_t*, void*, int64_t, void*, int64_t, float*,
                                         void*, size_t, void*);
    int (*grad_norm)(const qfmt_tensor_t*, int64_t, int64_t, float, const qfmt_dls_t*, qfmt_grad_norm_t*, qfmt_stats_t*, void*, size_t, void*);
    int (*grad_clip)(const qfmt_tensor_t*, int64_t, int64_t, const qfmt_grad_norm_t*, void*);
} lib;

static PyObject* data_ptr;  /* the method's name */

/* The arguments as 64-bit words; 0 and an exception set if one is not what `kinds` says: p a pointer, i an integer,
 * f a float (its bits).  (A size is never taken from a tensor's address.) */
static int words(PyObject* const* args, Py_ssize_t n, const char* kinds, uint64_t* v) {
    const Py_ssize_t want = (Py_ssize_t)strlen(kinds);
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
        return 0;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (kinds[i] == 'f') {
            const float f = (float)PyFloat_AsDouble(args[i]);
            v[i] = 0;
            memcpy(&v[i], &f, sizeof f);
        } else if (PyLong_Check(args[i])) {
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

static float to_float(const uint64_t* v) {
    float f;
    memcpy(&f, v, sizeof f);
    return f;
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

CALL(linear_act, "ppppiipip", P(0), P(1), P(2), P(3), (int64_t)v[4], (int32_t)v[5], P(6), (size_t)v[7], P(8))
CALL(linear_act_backward, "ppppipipip", P(0), P(1), P(2), P(3), (int64_t)v[4], P(5), (int32_t)v[6], P(7), (size_t)v[8], P(9))
CALL(act_backward, "pipipipiiiipip", P(0), (int64_t)v[1], P(2), (int64_t)v[3], P(4), (int64_t)v[5], P(6), (int64_t)v[7], (int64_t)v[8],
     (int32_t)v[9], (int32_t)v[10], P(11), (size_t)v[12], P(13))
CALL(linear_cross_entropy, "pppppppppip", P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), P(8), (size_t)v[9], P(10))
CALL(linear_cross_entropy_backward, "pppppppppipippip", P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), P(8), (int64_t)v[9], P(10), (int64_t)v[11],
     P(12), P(13), (size_t)v[14], P(15))
CALL(grad_norm, "piifppppip", P(0), (int64_t)v[1], (int64_t)v[2], to_float(&v[3]), P(4), P(5), P(6), P(7), (size_t)v[8], P(9))
CALL(grad_clip, "piipp", P(0), (int64_t)v[1], (int64_t)v[2], P(3), P(4))

static PyObject* py_bind_step(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    uint64_t v[MOST];
    (void)self;
    if (!words(args, n, "ppppppp", v)) return NULL;
    *(void**)&lib.linear_act = P(0);
    *(void**)&lib.linear_act_backward = P(1);
    *(void**)&lib.act_backward = P(2);
    *(void**)&lib.linear_cross_entropy = P(3);
    *(void**)&lib.linear_cross_entropy_backward = P(4);
    *(void**)&lib.grad_norm = P(5);
    *(void**)&lib.grad_clip = P(6);
    Py_RETURN_NONE;
}

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
                                METHOD(dropout_add_layer_norm_backward), METHOD(bind), METHOD(linear_act), METHOD(linear_act_backward),
                                METHOD(act_backward), METHOD(linear_cross_entropy), METHOD(linear_cross_entropy_backward), METHOD(grad_norm),
                                METHOD(grad_clip), METHOD(bind_step), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void) {
    data_ptr = PyUnicode_InternFromString("data_ptr");
    if (data_ptr == NULL) return NULL;
    return PyModule_Create(&module);
}
