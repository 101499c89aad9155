// Calls of the library from Python without ctypes: function(address) returns a callable for a function of harp_apply_ex's
// signature at that address, and so do quantize, linear_i8, grouped_linear_i8, grouped (also the gradient with respect to rows) and
// grad_weights for theirs.  ctypes converts seven arguments in 1.7 us and fifteen in 3 (0.3 and 0.5 us here, argument checks included), a
// fifth of a decode step's call and more.  Plain C beside CPython's headers, of the stable interface since 3.10, so that one build serves every
// later interpreter; it does not link to the library.
#define PY_SSIZE_T_CLEAN
#define Py_LIMITED_API 0x030a0000
#include <Python.h>
#include <stdint.h>

typedef int (*apply_fn)(const void *plan, void *x, int64_t n_rows, int dtype, int transpose, int kernel, void *stream);
typedef int (*quantize_fn)(const void *x, int64_t ld_x, int64_t n_rows, int64_t d, int dtype, void *q, int64_t ld_q, void *scale, void *stream);
typedef int (*linear_fn)(const void *x, int64_t ld_x, const void *x_scale, const void *w, int64_t ld_w, const void *w_scale, int64_t n_rows,
                         int64_t d_in, int64_t d_out, void *y, int64_t ld_y, int y_dtype, void *stream);
typedef int (*grouped_i8_fn)(const void *x, int64_t ld_x, const void *x_scale, const void *w, int64_t ld_w, const void *w_scale,
                             const void *offsets, int32_t n_groups, int64_t n_rows, int64_t d_in, int64_t d_out, void *y, int64_t ld_y,
                             int y_dtype, void *stream);
typedef int (*grouped_fn)(const void *x, int64_t ld_x, const void *w, int64_t ld_w, const void *offsets, int32_t n_groups, int64_t n_rows,
                          int64_t d_in, int64_t d_out, void *y, int64_t ld_y, int y_dtype, void *stream);
typedef int (*grad_weights_fn)(const void *gy, int64_t ld_gy, const void *x, int64_t ld_x, const void *offsets, int32_t n_groups,
                               int64_t n_rows, int64_t d_in, int64_t d_out, void *gw, int64_t ld_gw, int gw_dtype, int accumulate, void *stream);

// integers, None for a null pointer alone; whatever has __index__ counts as an integer, and pointers and codes wrap, as with ctypes
static int to_u64(PyObject *o, int pointer, uint64_t *out) {
    if (pointer && o == Py_None) { *out = 0; return 1; }
    PyObject *i = PyNumber_Index(o);
    if (!i) return 0;
    *out = PyLong_AsUnsignedLongLongMask(i);
    Py_DECREF(i);
    return !(*out == (uint64_t)-1 && PyErr_Occurred());
}

enum { MOST = 15 };
// the arguments of a call; bit k of `pointers`: argument k is one
static int take(PyObject *const *args, Py_ssize_t n, int want, unsigned pointers, uint64_t *a) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", want, n);
        return 0;
    }
    for (int k = 0; k < want; ++k)
        if (!to_u64(args[k], pointers >> k & 1, &a[k])) return 0;
    return 1;
}

#define P(k) ((void *)(uintptr_t)a[k])
#define L(k) ((int64_t)a[k])
#define I(k) ((int)a[k])
#define DEFINE_CALL(name, type, n_args, pointers, ...)                                          \
    static PyObject *name##_call(PyObject *self, PyObject *const *args, Py_ssize_t n) {          \
        uint64_t a[MOST];                                                                        \
        if (!take(args, n, n_args, pointers, a)) return NULL;                                    \
        const type fn = (type)PyLong_AsVoidPtr(self);                                            \
        int st;                                                                                  \
        Py_BEGIN_ALLOW_THREADS                                                                   \
        st = fn(__VA_ARGS__);                                                                    \
        Py_END_ALLOW_THREADS                                                                     \
        return PyLong_FromLong(st);                                                              \
    }                                                                                            \
    static PyMethodDef name##_def = {#name, (PyCFunction)(void (*)(void))name##_call, METH_FASTCALL, "the call -> status"}; \
    static PyObject *name(PyObject *self, PyObject *address) {                                   \
        (void)self;                                                                              \
        return callable(&name##_def, address);                                                   \
    }

static PyObject *callable(PyMethodDef *def, PyObject *address) {
    if (!PyLong_Check(address) || !PyLong_AsVoidPtr(address)) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "the address of a function expected");
        return NULL;
    }
    return PyCFunction_New(def, address);
}

#define BIT(k) (1u << (k))
DEFINE_CALL(function, apply_fn, 7, BIT(0) | BIT(1) | BIT(6), P(0), P(1), L(2), I(3), I(4), I(5), P(6))
DEFINE_CALL(quantize, quantize_fn, 9, BIT(0) | BIT(5) | BIT(7) | BIT(8), P(0), L(1), L(2), L(3), I(4), P(5), L(6), P(7), P(8))
DEFINE_CALL(linear_i8, linear_fn, 13, BIT(0) | BIT(2) | BIT(3) | BIT(5) | BIT(9) | BIT(12), P(0), L(1), P(2), P(3), L(4), P(5), L(6), L(7), L(8),
            P(9), L(10), I(11), P(12))
DEFINE_CALL(grouped_linear_i8, grouped_i8_fn, 15, BIT(0) | BIT(2) | BIT(3) | BIT(5) | BIT(6) | BIT(11) | BIT(14), P(0), L(1), P(2), P(3), L(4), P(5),
            P(6), I(7), L(8), L(9), L(10), P(11), L(12), I(13), P(14))
DEFINE_CALL(grouped, grouped_fn, 13, BIT(0) | BIT(2) | BIT(4) | BIT(9) | BIT(12), P(0), L(1), P(2), L(3), P(4), I(5), L(6), L(7), L(8), P(9), L(10),
            I(11), P(12))
DEFINE_CALL(grad_weights, grad_weights_fn, 14, BIT(0) | BIT(2) | BIT(4) | BIT(9) | BIT(13), P(0), L(1), P(2), L(3), P(4), I(5), L(6), L(7), L(8), P(9),
            L(10), I(11), I(12), P(13))

static PyMethodDef methods[] = {{"function", function, METH_O, "callable for the function at this address"},
                                {"quantize", quantize, METH_O, "... of harp_quantize_rows's signature"},
                                {"linear_i8", linear_i8, METH_O, "... of harp_linear_i8's"},
                                {"grouped_linear_i8", grouped_linear_i8, METH_O, "... of harp_grouped_linear_i8's"},
                                {"grouped", grouped, METH_O, "... of harp_grouped_linear's and harp_grouped_grad_rows's"},
                                {"grad_weights", grad_weights, METH_O, "... of harp_grouped_grad_weights's"},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_harpcall", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__harpcall(void) { return PyModule_Create(&module); }
