/* The layer operators' entry points as Python functions: a call through ctypes spends 0.8 to 1.4 us on its arguments, more than
 * the checks in front of it, where a layer's whole call takes 5 to 7 us of host time.  Same names, same arguments, integers
 * for pointers, None for NULL; the functions come from the library that the binding has loaded (bind). */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/sparsecomm.h"

static struct {
    int (*sc_checkpoint_pack)(sc_ctx*, int, const void*, size_t, size_t, size_t, int8_t*, uint8_t*, void*);
    int (*sc_checkpoint_unpack)(sc_ctx*, int, const int8_t*, const uint8_t*, size_t, size_t, void*, size_t, void*);
    int (*sc_activation_grad)(sc_ctx*, int, int, const void*, size_t, const int8_t*, const uint8_t*, size_t, size_t, void*, size_t, float*, int, void*);
    int (*sc_linear)(sc_ctx*, int, int, const void*, size_t, const void*, size_t, const void*, const void*, size_t, size_t, size_t, size_t, void*, size_t,
                     int8_t*, uint8_t*, void*);
    int (*sc_linear_grad_input)(sc_ctx*, int, int, const void*, size_t, const void*, size_t, const void*, size_t, const int8_t*, const uint8_t*, size_t,
                                size_t, size_t, void*, size_t, void*);
    int (*sc_linear_grad_weight)(sc_ctx*, int, const void*, size_t, const void*, size_t, const int8_t*, const uint8_t*, size_t, size_t, size_t, float*, size_t,
                                 int, void*);
} fn;

static void* P(PyObject* o) { return o == Py_None ? NULL : PyLong_AsVoidPtr(o); }
static size_t U(PyObject* o) { return PyLong_AsSize_t(o); }
static int I(PyObject* o) { return (int)PyLong_AsLong(o); }

/* Converts the arguments, then calls without the interpreter lock: a first call may allocate and wait. */
#define WRAPPER(name, count, ...)                                                                  \
    static PyObject* name##_py(PyObject* self, PyObject* const* a, Py_ssize_t n) {                 \
        int rc;                                                                                    \
        (void)self;                                                                                \
        if (n != count || !fn.name) {                                                              \
            PyErr_SetString(PyExc_TypeError, #name ": wrong number of arguments, or not bound");   \
            return NULL;                                                                           \
        }                                                                                          \
        CONVERT_##name                                                                             \
        if (PyErr_Occurred()) return NULL;                                                         \
        Py_BEGIN_ALLOW_THREADS                                                                     \
        rc = fn.name(__VA_ARGS__);                                                                 \
        Py_END_ALLOW_THREADS                                                                       \
        return PyLong_FromLong(rc);                                                                \
    }

#define CONVERT_sc_checkpoint_pack \
    void *h = P(a[0]), *x = P(a[2]), *q = P(a[6]), *s = P(a[7]), *st = P(a[8]); int t = I(a[1]); size_t ld = U(a[3]), r = U(a[4]), c = U(a[5]);
WRAPPER(sc_checkpoint_pack, 9, (sc_ctx*)h, t, x, ld, r, c, (int8_t*)q, (uint8_t*)s, st)

#define CONVERT_sc_checkpoint_unpack \
    void *h = P(a[0]), *q = P(a[2]), *s = P(a[3]), *o = P(a[6]), *st = P(a[8]); int t = I(a[1]); size_t r = U(a[4]), c = U(a[5]), ld = U(a[7]);
WRAPPER(sc_checkpoint_unpack, 9, (sc_ctx*)h, t, (const int8_t*)q, (const uint8_t*)s, r, c, o, ld, st)

#define CONVERT_sc_activation_grad                                                                                                   \
    void *h = P(a[0]), *dy = P(a[3]), *q = P(a[5]), *s = P(a[6]), *dz = P(a[9]), *db = P(a[11]), *st = P(a[13]);                       \
    int t = I(a[1]), act = I(a[2]), add = I(a[12]); size_t ldy = U(a[4]), r = U(a[7]), c = U(a[8]), ldz = U(a[10]);
WRAPPER(sc_activation_grad, 14, (sc_ctx*)h, t, act, dy, ldy, (const int8_t*)q, (const uint8_t*)s, r, c, dz, ldz, (float*)db, add, st)

#define CONVERT_sc_linear                                                                                                            \
    void *h = P(a[0]), *x = P(a[3]), *w = P(a[5]), *b = P(a[7]), *r = P(a[8]), *y = P(a[13]), *q = P(a[15]), *s = P(a[16]), *st = P(a[17]); \
    int t = I(a[1]), act = I(a[2]);                                                                                                    \
    size_t ldx = U(a[4]), ldw = U(a[6]), ldr = U(a[9]), M = U(a[10]), N = U(a[11]), K = U(a[12]), ldy = U(a[14]);
WRAPPER(sc_linear, 18, (sc_ctx*)h, t, act, x, ldx, w, ldw, b, r, ldr, M, N, K, y, ldy, (int8_t*)q, (uint8_t*)s, st)

#define CONVERT_sc_linear_grad_input                                                                                                 \
    void *h = P(a[0]), *dz = P(a[3]), *w = P(a[5]), *r = P(a[7]), *q = P(a[9]), *s = P(a[10]), *dx = P(a[14]), *st = P(a[16]);           \
    int t = I(a[1]), act = I(a[2]);                                                                                                    \
    size_t lddz = U(a[4]), ldw = U(a[6]), ldr = U(a[8]), M = U(a[11]), N = U(a[12]), K = U(a[13]), lddx = U(a[15]);
WRAPPER(sc_linear_grad_input, 17, (sc_ctx*)h, t, act, dz, lddz, w, ldw, r, ldr, (const int8_t*)q, (const uint8_t*)s, M, N, K, dx, lddx, st)

#define CONVERT_sc_linear_grad_weight                                                                                                \
    void *h = P(a[0]), *dz = P(a[2]), *x = P(a[4]), *q = P(a[6]), *s = P(a[7]), *dw = P(a[11]), *st = P(a[14]); int t = I(a[1]), add = I(a[13]); \
    size_t lddz = U(a[3]), ldx = U(a[5]), M = U(a[8]), N = U(a[9]), K = U(a[10]), lddw = U(a[12]);
WRAPPER(sc_linear_grad_weight, 15, (sc_ctx*)h, t, dz, lddz, x, ldx, (const int8_t*)q, (const uint8_t*)s, M, N, K, (float*)dw, lddw, add, st)

/* bind(pack, unpack, activation_grad, linear, grad_input, grad_weight): the functions' addresses. */
static PyObject* bind(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void* p[6];
    (void)self;
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "bind: six addresses");
        return NULL;
    }
    for (int i = 0; i < 6; ++i) p[i] = P(a[i]);
    if (PyErr_Occurred()) return NULL;
    *(void**)&fn.sc_checkpoint_pack = p[0];
    *(void**)&fn.sc_checkpoint_unpack = p[1];
    *(void**)&fn.sc_activation_grad = p[2];
    *(void**)&fn.sc_linear = p[3];
    *(void**)&fn.sc_linear_grad_input = p[4];
    *(void**)&fn.sc_linear_grad_weight = p[5];
    Py_RETURN_NONE;
}

#define METHOD(name, f) {name, (PyCFunction)(void (*)(void))f, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD("bind", bind),
                                METHOD("sc_checkpoint_pack", sc_checkpoint_pack_py),
                                METHOD("sc_checkpoint_unpack", sc_checkpoint_unpack_py),
                                METHOD("sc_activation_grad", sc_activation_grad_py),
                                METHOD("sc_linear", sc_linear_py),
                                METHOD("sc_linear_grad_input", sc_linear_grad_input_py),
                                METHOD("sc_linear_grad_weight", sc_linear_grad_weight_py),
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sc_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__sc_calls(void) { return PyModule_Create(&module); }
