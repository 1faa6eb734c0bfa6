// The layer operators' entry points as Python functions: a call through ctypes spends 0.8 to 1.4 us on its arguments, more than
// the checks in front of it, where a layer's whole call takes 5 to 7 us of host time.  Same names, same arguments, integers
// for pointers, None for NULL; the functions come from the library that the binding has loaded (bind).
//
// The operators around a layer (norm, dropout, 8-bit rows and their product) have a second form that takes the tensors themselves: Python
// needs 0.4 us to look at a matrix, and a norm has seven.  It checks what the binding checks and calls the library; for any argument
// that it does not take as it is, it returns None, and the binding's own checks say what is wrong.  That form needs torch's headers and is
// built with SC_TENSORS; the rest needs Python's alone.
#ifdef SC_TENSORS
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>
#else
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#endif

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
    int (*sc_quantize)(sc_ctx*, int, const void*, size_t, size_t, size_t, int8_t*, size_t, float*, void*);
    int (*sc_dequantize)(sc_ctx*, int, const int8_t*, size_t, const float*, size_t, size_t, void*, size_t, void*);
    int (*sc_linear_quantized)(sc_ctx*, int, int, const int8_t*, size_t, const float*, const int8_t*, size_t, const float*, const void*, const void*, size_t,
                               size_t, size_t, size_t, void*, size_t, int8_t*, uint8_t*, void*);
    int (*sc_dropout)(sc_ctx*, int, const void*, size_t, const void*, size_t, double, uint64_t, size_t, size_t, void*, size_t, void*);
    int (*sc_rms_norm)(sc_ctx*, int, const void*, size_t, const void*, size_t, const void*, float, double, uint64_t, size_t, size_t, void*, size_t, void*,
                       size_t, int8_t*, size_t, float*, void*);
    int (*sc_rms_norm_grad)(sc_ctx*, int, const void*, size_t, const void*, size_t, const void*, float, const void*, size_t, double, uint64_t, size_t, size_t,
                            void*, size_t, void*, size_t, float*, int, void*);
} fn;

static void* P(PyObject* o) { return o == Py_None ? NULL : PyLong_AsVoidPtr(o); }
static size_t U(PyObject* o) { return PyLong_AsSize_t(o); }
static int I(PyObject* o) { return (int)PyLong_AsLong(o); }
static double D(PyObject* o) { return PyFloat_AsDouble(o); }
static uint64_t S(PyObject* o) { return PyLong_AsUnsignedLongLongMask(o); }

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

#define CONVERT_sc_quantize \
    void *h = P(a[0]), *x = P(a[2]), *q = P(a[6]), *s = P(a[8]), *st = P(a[9]); int t = I(a[1]); size_t ldx = U(a[3]), r = U(a[4]), c = U(a[5]), ldq = U(a[7]);
WRAPPER(sc_quantize, 10, (sc_ctx*)h, t, x, ldx, r, c, (int8_t*)q, ldq, (float*)s, st)

#define CONVERT_sc_dequantize \
    void *h = P(a[0]), *q = P(a[2]), *s = P(a[4]), *o = P(a[7]), *st = P(a[9]); int t = I(a[1]); size_t ldq = U(a[3]), r = U(a[5]), c = U(a[6]), ldo = U(a[8]);
WRAPPER(sc_dequantize, 10, (sc_ctx*)h, t, (const int8_t*)q, ldq, (const float*)s, r, c, o, ldo, st)

#define CONVERT_sc_linear_quantized                                                                                                  \
    void *h = P(a[0]), *x = P(a[3]), *xs = P(a[5]), *w = P(a[6]), *ws = P(a[8]), *b = P(a[9]), *r = P(a[10]), *y = P(a[15]), *q = P(a[17]), \
         *s = P(a[18]), *st = P(a[19]);                                                                                                \
    int t = I(a[1]), act = I(a[2]);                                                                                                    \
    size_t ldx = U(a[4]), ldw = U(a[7]), ldr = U(a[11]), M = U(a[12]), N = U(a[13]), K = U(a[14]), ldy = U(a[16]);
WRAPPER(sc_linear_quantized, 20, (sc_ctx*)h, t, act, (const int8_t*)x, ldx, (const float*)xs, (const int8_t*)w, ldw, (const float*)ws, b, r, ldr, M, N, K, y,
        ldy, (int8_t*)q, (uint8_t*)s, st)

#define CONVERT_sc_dropout                                                                                                           \
    void *h = P(a[0]), *x = P(a[2]), *r = P(a[4]), *y = P(a[10]), *st = P(a[12]); int t = I(a[1]); double p = D(a[6]); uint64_t seed = S(a[7]); \
    size_t ldx = U(a[3]), ldr = U(a[5]), rows = U(a[8]), cols = U(a[9]), ldy = U(a[11]);
WRAPPER(sc_dropout, 13, (sc_ctx*)h, t, x, ldx, r, ldr, p, seed, rows, cols, y, ldy, st)

#define CONVERT_sc_rms_norm                                                                                                          \
    void *h = P(a[0]), *x = P(a[2]), *r = P(a[4]), *g = P(a[6]), *o = P(a[12]), *y = P(a[14]), *q = P(a[16]), *s = P(a[18]), *st = P(a[19]); \
    int t = I(a[1]); double eps = D(a[7]), p = D(a[8]); uint64_t seed = S(a[9]);                                                         \
    size_t ldx = U(a[3]), ldr = U(a[5]), rows = U(a[10]), cols = U(a[11]), ldh = U(a[13]), ldy = U(a[15]), ldq = U(a[17]);
WRAPPER(sc_rms_norm, 20, (sc_ctx*)h, t, x, ldx, r, ldr, g, (float)eps, p, seed, rows, cols, o, ldh, y, ldy, (int8_t*)q, ldq, (float*)s, st)

#define CONVERT_sc_rms_norm_grad                                                                                                     \
    void *h = P(a[0]), *dy = P(a[2]), *o = P(a[4]), *g = P(a[6]), *r = P(a[8]), *dh = P(a[14]), *dx = P(a[16]), *dg = P(a[18]), *st = P(a[20]); \
    int t = I(a[1]), add = I(a[19]); double eps = D(a[7]), p = D(a[10]); uint64_t seed = S(a[11]);                                       \
    size_t ldy = U(a[3]), ldo = U(a[5]), ldr = U(a[9]), rows = U(a[12]), cols = U(a[13]), lddh = U(a[15]), lddx = U(a[17]);
WRAPPER(sc_rms_norm_grad, 21, (sc_ctx*)h, t, dy, ldy, o, ldo, g, (float)eps, r, ldr, p, seed, rows, cols, dh, lddh, dx, lddx, (float*)dg, add, st)

/* bind(addresses): the functions' addresses, in the order of `fn`. */
static PyObject* bind(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void** to[] = {(void**)&fn.sc_checkpoint_pack, (void**)&fn.sc_checkpoint_unpack, (void**)&fn.sc_activation_grad, (void**)&fn.sc_linear,
                   (void**)&fn.sc_linear_grad_input, (void**)&fn.sc_linear_grad_weight, (void**)&fn.sc_quantize, (void**)&fn.sc_dequantize,
                   (void**)&fn.sc_linear_quantized, (void**)&fn.sc_dropout, (void**)&fn.sc_rms_norm, (void**)&fn.sc_rms_norm_grad};
    void* p[sizeof(to) / sizeof(to[0])];
    (void)self;
    if (n != (Py_ssize_t)(sizeof(to) / sizeof(to[0]))) {
        PyErr_SetString(PyExc_TypeError, "bind: an address for each function");
        return NULL;
    }
    for (Py_ssize_t i = 0; i < n; ++i) p[i] = P(a[i]);
    if (PyErr_Occurred()) return NULL;
    for (Py_ssize_t i = 0; i < n; ++i) *to[i] = p[i];
    Py_RETURN_NONE;
}

// -- calls that take tensors ---------------------------------------------------------------------------------
#ifdef SC_TENSORS
namespace {

// What is wrong with an argument is not said here: the first failed check ends the call, whose answer is None.
struct NotTaken {};

struct Call {
    long device;

    static bool given(PyObject* o) { return o != Py_None; }
    const at::Tensor& tensor(PyObject* o) const {
        if (!THPVariable_Check(o)) throw NotTaken();
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.get_device() != device) throw NotTaken();
        return t;
    }
    // Rows of `cols` elements; the distance between them is returned.
    size_t matrix(const at::Tensor& t, int64_t rows, int64_t cols, at::ScalarType type) const {
        if (t.scalar_type() != type || t.dim() != 2) throw NotTaken();
        const auto size = t.sizes(), step = t.strides();
        if (size[0] != rows || size[1] != cols || step[1] != 1 || step[0] < cols) throw NotTaken();
        return (size_t)step[0];
    }
    void* matrix(PyObject* o, int64_t rows, int64_t cols, at::ScalarType type, size_t& ld) const {
        ld = (size_t)cols;
        if (!given(o)) return nullptr;
        const at::Tensor& t = tensor(o);
        ld = matrix(t, rows, cols, type);
        return t.data_ptr();
    }
    void* dense(PyObject* o, int64_t numbers, at::ScalarType type) const {
        if (!given(o)) return nullptr;
        const at::Tensor& t = tensor(o);
        if (t.scalar_type() != type || t.numel() != numbers || !t.is_contiguous()) throw NotTaken();
        return t.data_ptr();
    }
    static int type_of(const at::Tensor& t, bool f32 = false) {
        if (t.dim() != 2) throw NotTaken();
        switch (t.scalar_type()) {
            case at::kBFloat16: return SC_BF16;
            case at::kHalf: return SC_F16;
            case at::kFloat: if (f32) return SC_F32; [[fallthrough]];
            default: throw NotTaken();
        }
    }
};
double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw NotTaken();
    return v;
}
double probability(PyObject* o) {
    const double v = number(o);
    if (!(v >= 0.0 && v <= 1.0)) throw NotTaken();
    return v;
}
uint64_t seed_of(PyObject* o) {
    if (!PyLong_Check(o)) throw NotTaken();
    return PyLong_AsUnsignedLongLongMask(o);
}
int whole(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw NotTaken();
    return (int)v;
}

// Runs body(call, arguments after the handle and the device); its answer is the library's status.
template <typename F>
PyObject* with_tensors(PyObject* const* a, Py_ssize_t n, Py_ssize_t count, F&& body) {
    if (n != count) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    sc_ctx* ctx = (sc_ctx*)P(a[0]);
    const long device = PyLong_AsLong(a[1]);
    void* stream = P(a[n - 1]);
    if (PyErr_Occurred()) return nullptr;
    try {
        return PyLong_FromLong(body(Call{device}, ctx, a + 2, stream));
    } catch (...) {                                    // an argument of another kind, or a tensor without memory of its own
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}
// Calls the library without the interpreter lock.
template <typename F>
int unlocked(F&& call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return rc;
}

// (x, q, scales)
PyObject* quantize(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return with_tensors(args, n, 6, [](const Call& c, sc_ctx* h, PyObject* const* a, void* st) {
        const at::Tensor& x = c.tensor(a[0]);
        const int type = Call::type_of(x, true);
        const int64_t rows = x.size(0), cols = x.size(1);
        size_t ldq;
        const size_t ldx = c.matrix(x, rows, cols, x.scalar_type());
        void *q = c.matrix(a[1], rows, cols, at::kChar, ldq), *s = c.dense(a[2], rows, at::kFloat);
        if (!Call::given(a[1]) || !Call::given(a[2])) throw NotTaken();
        const void* xp = x.data_ptr();
        return unlocked([&] { return fn.sc_quantize(h, type, xp, ldx, rows, cols, (int8_t*)q, ldq, (float*)s, st); });
    });
}

// (q, scales, out)
PyObject* dequantize(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return with_tensors(args, n, 6, [](const Call& c, sc_ctx* h, PyObject* const* a, void* st) {
        const at::Tensor& out = c.tensor(a[2]);
        const int type = Call::type_of(out, true);
        const int64_t rows = out.size(0), cols = out.size(1);
        size_t ldq;
        const size_t ldo = c.matrix(out, rows, cols, out.scalar_type());
        void *q = c.matrix(a[0], rows, cols, at::kChar, ldq), *s = c.dense(a[1], rows, at::kFloat);
        if (!Call::given(a[0]) || !Call::given(a[1])) throw NotTaken();
        void* o = out.data_ptr();
        return unlocked([&] { return fn.sc_dequantize(h, type, (const int8_t*)q, ldq, (const float*)s, rows, cols, o, ldo, st); });
    });
}

// (act, x, x_scales, w, w_scales, y, bias, residual, q, scales)
PyObject* linear_quantized(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return with_tensors(args, n, 13, [](const Call& c, sc_ctx* h, PyObject* const* a, void* st) {
        const int act = whole(a[0]);
        const at::Tensor &x = c.tensor(a[1]), &y = c.tensor(a[5]);
        const int type = Call::type_of(y);
        if (x.dim() != 2 || !Call::given(a[2]) || !Call::given(a[3]) || !Call::given(a[4])) throw NotTaken();
        const int64_t M = y.size(0), N = y.size(1), K = x.size(1), groups = (N + 31) / 32;
        size_t ldw, ldr, ignored;
        const size_t ldy = c.matrix(y, M, N, y.scalar_type()), ldx = c.matrix(x, M, K, at::kChar);
        const void *xs = c.dense(a[2], M, at::kFloat), *w = c.matrix(a[3], N, K, at::kChar, ldw), *ws = c.dense(a[4], N, at::kFloat);
        const void *bias = c.dense(a[6], N, y.scalar_type()), *residual = c.matrix(a[7], M, N, y.scalar_type(), ldr);
        void *q = c.matrix(a[8], M, N, at::kChar, ignored), *scales = c.matrix(a[9], M, groups, at::kByte, ignored);
        if (Call::given(a[8]) != Call::given(a[9])) throw NotTaken();
        c.dense(a[8], M * N, at::kChar);
        c.dense(a[9], M * groups, at::kByte);
        const void* xp = x.data_ptr();
        void* yp = y.data_ptr();
        return unlocked([&] {
            return fn.sc_linear_quantized(h, type, act, (const int8_t*)xp, ldx, (const float*)xs, (const int8_t*)w, ldw, (const float*)ws, bias, residual, ldr, M, N, K,
                                          yp, ldy, (int8_t*)q, (uint8_t*)scales, st);
        });
    });
}

// (x, y, p, seed, residual)
PyObject* dropout(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return with_tensors(args, n, 8, [](const Call& c, sc_ctx* h, PyObject* const* a, void* st) {
        const at::Tensor& x = c.tensor(a[0]);
        const int type = Call::type_of(x);
        const int64_t rows = x.size(0), cols = x.size(1);
        size_t ldy, ldr;
        const size_t ldx = c.matrix(x, rows, cols, x.scalar_type());
        void* y = c.matrix(a[1], rows, cols, x.scalar_type(), ldy);
        if (!Call::given(a[1])) throw NotTaken();
        const double p = probability(a[2]);
        const uint64_t seed = seed_of(a[3]);
        const void *residual = c.matrix(a[4], rows, cols, x.scalar_type(), ldr), *xp = x.data_ptr();
        return unlocked([&] { return fn.sc_dropout(h, type, xp, ldx, residual, ldr, p, seed, rows, cols, y, ldy, st); });
    });
}

// (x, gamma, eps, y, q, scales, residual, h, p, seed)
PyObject* rms_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return with_tensors(args, n, 13, [](const Call& c, sc_ctx* h, PyObject* const* a, void* st) {
        const at::Tensor& x = c.tensor(a[0]);
        const int type = Call::type_of(x);
        const auto t = x.scalar_type();
        const int64_t rows = x.size(0), cols = x.size(1);
        size_t ldy, ldq, ldr, ldh;
        const size_t ldx = c.matrix(x, rows, cols, t);
        if (!Call::given(a[1]) || (!Call::given(a[3]) && !Call::given(a[4])) || Call::given(a[4]) != Call::given(a[5])) throw NotTaken();
        const void* gamma = c.dense(a[1], cols, t);
        const double eps = number(a[2]), p = probability(a[8]);
        const uint64_t seed = seed_of(a[9]);
        void *y = c.matrix(a[3], rows, cols, t, ldy), *q = c.matrix(a[4], rows, cols, at::kChar, ldq), *s = c.dense(a[5], rows, at::kFloat);
        const void* residual = c.matrix(a[6], rows, cols, t, ldr);
        void* out = c.matrix(a[7], rows, cols, t, ldh);
        const void* xp = x.data_ptr();
        return unlocked([&] {
            return fn.sc_rms_norm(h, type, xp, ldx, residual, ldr, gamma, (float)eps, p, seed, rows, cols, out, ldh, y, ldy, (int8_t*)q, ldq, (float*)s, st);
        });
    });
}

// (dy, h, gamma, eps, dh, dgamma, residual, dx, p, seed, accumulate)
PyObject* rms_norm_grad(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return with_tensors(args, n, 14, [](const Call& c, sc_ctx* h, PyObject* const* a, void* st) {
        const at::Tensor& dy = c.tensor(a[0]);
        const int type = Call::type_of(dy);
        const auto t = dy.scalar_type();
        const int64_t rows = dy.size(0), cols = dy.size(1);
        size_t ldh, lddh, ldr, lddx;
        const size_t lddy = c.matrix(dy, rows, cols, t);
        if (!Call::given(a[1]) || !Call::given(a[2]) || (!Call::given(a[4]) && !Call::given(a[5]) && !Call::given(a[7]))) throw NotTaken();
        const void *hp = c.matrix(a[1], rows, cols, t, ldh), *gamma = c.dense(a[2], cols, t), *residual = c.matrix(a[6], rows, cols, t, ldr);
        const double eps = number(a[3]), p = probability(a[8]);
        const uint64_t seed = seed_of(a[9]);
        void *dh = c.matrix(a[4], rows, cols, t, lddh), *dgamma = c.dense(a[5], cols, at::kFloat), *dx = c.matrix(a[7], rows, cols, t, lddx);
        const int add = PyObject_IsTrue(a[10]);
        if (add < 0) throw NotTaken();
        const void* dyp = dy.data_ptr();
        return unlocked([&] {
            return fn.sc_rms_norm_grad(h, type, dyp, lddy, hp, ldh, gamma, (float)eps, residual, ldr, p, seed, rows, cols, dh, lddh, dx, lddx, (float*)dgamma, add, st);
        });
    });
}

}  // namespace
#endif

#define METHOD(name, f) {name, (PyCFunction)(void (*)(void))f, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD("bind", bind),
                                METHOD("sc_checkpoint_pack", sc_checkpoint_pack_py),
                                METHOD("sc_checkpoint_unpack", sc_checkpoint_unpack_py),
                                METHOD("sc_activation_grad", sc_activation_grad_py),
                                METHOD("sc_linear", sc_linear_py),
                                METHOD("sc_linear_grad_input", sc_linear_grad_input_py),
                                METHOD("sc_linear_grad_weight", sc_linear_grad_weight_py),
                                METHOD("sc_quantize", sc_quantize_py),
                                METHOD("sc_dequantize", sc_dequantize_py),
                                METHOD("sc_linear_quantized", sc_linear_quantized_py),
                                METHOD("sc_dropout", sc_dropout_py),
                                METHOD("sc_rms_norm", sc_rms_norm_py),
                                METHOD("sc_rms_norm_grad", sc_rms_norm_grad_py),
#ifdef SC_TENSORS
                                METHOD("quantize", quantize),
                                METHOD("dequantize", dequantize),
                                METHOD("linear_quantized", linear_quantized),
                                METHOD("dropout", dropout),
                                METHOD("rms_norm", rms_norm),
                                METHOD("rms_norm_grad", rms_norm_grad),
#endif
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef definition = {PyModuleDef_HEAD_INIT, "_sc_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__sc_calls(void) {
    PyObject* m = PyModule_Create(&definition);
#ifdef SC_TENSORS
    // the tensors' layout is that of the headers it was built with: the binding compares
    if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) Py_CLEAR(m);
#endif
    return m;
}
