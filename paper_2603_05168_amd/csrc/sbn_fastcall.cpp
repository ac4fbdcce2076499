// The Python side of one call, in C++: shapes, types, pointers and the current stream are read from the tensors without the
// interpreter, and the C ABI is called.  A direct call of the layer costs the host 2.1 us less its launch in Python and 0.6 here (the
// kernel of one token through 2560 x 2560 takes 3.4 us), so without this the host and not the device sets the pace of single calls.
// Marshalling only: whatever is not a plain tensor of the expected kind (an integer address, a subclass, another type or rank, a
// tensor without storage) is answered with None, and the Python code beside it does the call or raises its own error.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>
#include <exception>
#include <new>

namespace {

using linear_fn = int (*)(const void *, int64_t, int64_t, int64_t, int, int, const void *, const float *, const float *, float *, int8_t *, float *,
                          int32_t *, int, void *, size_t, void *);
using grouped_fn = int (*)(int, const void *const *, const int64_t *, const int64_t *, const int64_t *, int, int, const void *const *,
                           const float *const *, float *const *, int, void *, size_t, void *);
linear_fn g_linear = nullptr;
grouped_fn g_grouped = nullptr;

const at::Tensor *plain(PyObject *o)
{
    return Py_TYPE(o) == reinterpret_cast<PyTypeObject *>(THPVariableClass) ? &THPVariable_Unpack(o) : nullptr;
}

// address of a plain tensor, null for None; false for anything else
bool address(PyObject *o, void *&p)
{
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = plain(o);
    if (!t) return false;
    p = t->data_ptr();
    return true;
}

bool small_int(PyObject *o, int &v)
{
    if (!PyLong_CheckExact(o)) return false;
    const long l = PyLong_AsLong(o);
    if ((l == -1 && PyErr_Occurred()) || l < INT32_MIN || l > INT32_MAX) {
        PyErr_Clear();
        return false;
    }
    v = (int)l;
    return true;
}

// The call itself, without the interpreter's lock: -> status, or null with a Python error where it throws (the lock is held again by
// then; the call has begun, so the Python code must not do it once more)
template <class Call> PyObject *released(Call &&call)
{
    struct Unlocked {
        PyThreadState *state = PyEval_SaveThread();
        ~Unlocked() { PyEval_RestoreThread(state); }
    };
    try {
        int status;
        {
            Unlocked unlocked;
            status = call();
        }
        return PyLong_FromLong(status);
    } catch (const std::bad_alloc &) {
        return PyErr_NoMemory();
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "exception of an unknown kind");
    }
    return nullptr;
}

void *current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// (X, packed, gamma, Y, N, M, workspace, bias, xq_out, sx_out, acc_out, path) -> status, or None
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 12 || !g_linear) Py_RETURN_NONE;
    try {
        const at::Tensor *Y = plain(a[3]), *ws = plain(a[6]), *rows = plain(a[0] != Py_None ? a[0] : a[8]);
        if (!Y || !ws || !rows || !Y->is_cuda() || Y->dim() < 2 || rows->dim() != 2 || Y->scalar_type() != at::kFloat) Py_RETURN_NONE;
        if (a[0] != Py_None && rows->scalar_type() != at::kBFloat16) Py_RETURN_NONE;
        void *x, *packed, *gamma, *bias, *xq, *sx, *acc;
        int N, M, path;
        if (!address(a[0], x) || !address(a[1], packed) || !address(a[2], gamma) || !address(a[7], bias) || !address(a[8], xq) || !address(a[9], sx) ||
            !address(a[10], acc) || !small_int(a[4], N) || !small_int(a[5], M) || !small_int(a[11], path))
            Py_RETURN_NONE;
        const int64_t tokens = rows->size(0), d_in = rows->size(1), d_out = Y->size(1);
        void *y = Y->data_ptr(), *w = ws->data_ptr(), *stream = current_stream();
        const size_t bytes = ws->nbytes();
        return released([&] {
            return g_linear(x, tokens, d_in, d_out, N, M, packed, static_cast<const float *>(gamma), static_cast<const float *>(bias), static_cast<float *>(y),
                            static_cast<int8_t *>(xq), static_cast<float *>(sx), static_cast<int32_t *>(acc), path, w, bytes, stream);
        });
    } catch (...) {
        Py_RETURN_NONE;   // a tensor without storage, no device: the Python code raises its own error
    }
}

// A ctypes array of at least `count` pointers or 64-bit integers, held while its address is in use; anything else is not held.
struct Array {
    Py_buffer view{};
    bool held;
    enum Kind { POINTERS, INTEGERS };
    Array(PyObject *o, int count, Kind kind)
    {
        held = PyObject_GetBuffer(o, &view, PyBUF_ND | PyBUF_FORMAT) == 0;
        if (!held) {
            PyErr_Clear();
            return;
        }
        // the formats of ctypes, which names the byte order; a ctypes pointer has no dimension
        const auto is = [&](const char *format) { return !strcmp(view.format, format); };
        if (view.ndim != 1 || view.itemsize != 8 || view.shape[0] < count || !(kind == POINTERS ? is("<P") : is("<q") || is("<l"))) release();
    }
    ~Array() { release(); }
    Array(const Array &) = delete;
    void release()
    {
        if (held) PyBuffer_Release(&view);
        held = false;
    }
    template <class T> T as() const { return reinterpret_cast<T>(view.buf); }
};

// (count, X, tokens, d_in, d_out, N, M, packed, gamma, Y, path, workspace): the arrays as they are at this call -> status, or None
PyObject *grouped(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 12 || !g_grouped) Py_RETURN_NONE;
    try {
        const at::Tensor *ws = plain(a[11]);
        int count, N, M, path;
        if (!ws || !ws->is_cuda() || !small_int(a[0], count) || count < 0 || !small_int(a[5], N) || !small_int(a[6], M) || !small_int(a[10], path))
            Py_RETURN_NONE;
        const Array X(a[1], count, Array::POINTERS), tokens(a[2], count, Array::INTEGERS), d_in(a[3], count, Array::INTEGERS),
            d_out(a[4], count, Array::INTEGERS), packed(a[7], count, Array::POINTERS), gamma(a[8], count, Array::POINTERS), Y(a[9], count, Array::POINTERS);
        if (!X.held || !tokens.held || !d_in.held || !d_out.held || !packed.held || !gamma.held || !Y.held) Py_RETURN_NONE;
        void *w = ws->data_ptr(), *stream = current_stream();
        const size_t bytes = ws->nbytes();
        return released([&] {
            return g_grouped(count, X.as<const void *const *>(), tokens.as<const int64_t *>(), d_in.as<const int64_t *>(), d_out.as<const int64_t *>(), N, M,
                             packed.as<const void *const *>(), gamma.as<const float *const *>(), Y.as<float *const *>(), path, w, bytes, stream);
        });
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// ---- output head and microscaled 4-bit floating point: the checks of the Python code (types, shapes, contiguous), on GPU tensors ----------------
using ce_fn = int (*)(const void *, const void *, const void *, int64_t, int64_t, int64_t, void *, void *, void *, size_t, void *);
using ce_backward_fn = int (*)(const void *, const void *, const void *, const void *, const void *, int64_t, int64_t, int64_t, void *, void *, void *, size_t, void *);
using distill_fn = int (*)(const void *, const void *, const void *, const void *, int, int64_t, float, const void *, int64_t, int64_t, int64_t, void *, void *, void *,
                           void *, size_t, void *);
using distill_backward_fn = int (*)(const void *, const void *, const void *, const void *, int, int64_t, float, const void *, const void *, const void *, const void *,
                                    int64_t, int64_t, int64_t, void *, void *, void *, size_t, void *);
using quantize_fn = int (*)(const void *, int, int64_t, int64_t, void *, void *, void *);
using dequantize_fn = int (*)(const void *, const void *, int64_t, int64_t, void *, int, void *);
using mx_linear_fn = int (*)(const void *, int64_t, int64_t, int64_t, const void *, const void *, const void *, void *, void *, size_t, void *);
using head_bytes_fn = int (*)(int64_t, int64_t, int64_t, int64_t, int, size_t *);
using mx_bytes_fn = int (*)(int64_t, int64_t, size_t *, size_t *);
using mx_workspace_fn = int (*)(int64_t, int64_t, size_t *);
struct HeadCalls {
    ce_fn ce;
    ce_backward_fn ce_backward;
    distill_fn distill;
    distill_backward_fn distill_backward;
    quantize_fn quantize;
    dequantize_fn dequantize;
    mx_linear_fn mx_linear;
    head_bytes_fn head_bytes;
    mx_bytes_fn mx_bytes;
    mx_workspace_fn mx_workspace;
};
HeadCalls g_head{};

// a plain contiguous GPU tensor of this type; dims -1: any.  Null where it is not, or where it is None
const at::Tensor *matrix(PyObject *o, at::ScalarType type, int64_t rows, int64_t cols)
{
    const at::Tensor *t = plain(o);
    return t && t->is_cuda() && t->scalar_type() == type && t->dim() == 2 && (rows < 0 || t->size(0) == rows) && (cols < 0 || t->size(1) == cols) && t->is_contiguous() ? t
                                                                                                                                                                 : nullptr;
}
const at::Tensor *vector(PyObject *o, at::ScalarType type, int64_t n)
{
    const at::Tensor *t = plain(o);
    return t && t->is_cuda() && t->scalar_type() == type && t->dim() == 1 && t->size(0) == n && t->is_contiguous() ? t : nullptr;
}
void *data(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }

// what may be None: false where it is something else than None and the tensor that is expected
bool maybe(PyObject *o, const at::Tensor *t) { return t || o == Py_None; }

struct Head {   // H, W, targets and what they say about sizes
    const at::Tensor *H, *W, *targets;
    int64_t tokens = 0, d = 0, vocab = 0;
    bool good;
    Head(PyObject *h, PyObject *w, PyObject *y, bool optional)
    {
        H = matrix(h, at::kBFloat16, -1, -1);
        if (H) tokens = H->size(0), d = H->size(1);
        W = H ? matrix(w, at::kBFloat16, -1, d) : nullptr;
        if (W) vocab = W->size(0);
        targets = W ? vector(y, at::kLong, tokens) : nullptr;
        good = W && (optional ? maybe(y, targets) : targets != nullptr);
    }
};

// the two gradients, either of which may be None
struct Gradients {
    const at::Tensor *dH, *dW;
    bool good;
    Gradients(const Head &h, PyObject *x, PyObject *w)
    {
        dH = matrix(x, at::kBFloat16, h.tokens, h.d);
        dW = matrix(w, at::kBFloat16, h.vocab, h.d);
        good = maybe(x, dH) && maybe(w, dW);
    }
};

struct Teacher {
    const at::Tensor *idx, *logits = nullptr;
    double tau = 0;
    int type = 0;
    bool good;
    Teacher(const Head &h, PyObject *i, PyObject *l, PyObject *t)
    {
        idx = matrix(i, at::kLong, h.tokens, -1);
        if (idx) logits = matrix(l, at::kFloat, h.tokens, idx->size(1));
        if (idx && !logits) logits = matrix(l, at::kBFloat16, h.tokens, idx->size(1)), type = 1;
        good = logits && PyFloat_CheckExact(t);
        if (good) tau = PyFloat_AS_DOUBLE(t);
    }
};

template <class Call> PyObject *guarded(bool bound, Call &&call)
{
    if (!bound) Py_RETURN_NONE;
    try {
        return call();
    } catch (...) {
        Py_RETURN_NONE;   // as above
    }
}

// (H, W, targets, ce, lse, workspace) -> status, or None
PyObject *head_ce(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n == 6 && g_head.ce, [&]() -> PyObject * {
        const Head h(a[0], a[1], a[2], false);
        const at::Tensor *ce = vector(a[3], at::kFloat, h.tokens), *lse = vector(a[4], at::kFloat, h.tokens), *ws = plain(a[5]);
        if (!h.good || !ce || !lse || !ws || !ws->is_cuda()) Py_RETURN_NONE;
        void *const stream = current_stream();
        return released([&] { return g_head.ce(data(h.H), data(h.W), data(h.targets), h.tokens, h.d, h.vocab, data(ce), data(lse), data(ws), ws->nbytes(), stream); });
    });
}

// (H, W, targets, lse, d_ce, workspace, dH, dW)
PyObject *head_ce_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n == 8 && g_head.ce_backward, [&]() -> PyObject * {
        const Head h(a[0], a[1], a[2], false);
        const at::Tensor *lse = vector(a[3], at::kFloat, h.tokens), *d = vector(a[4], at::kFloat, h.tokens), *ws = plain(a[5]);
        const Gradients g(h, a[6], a[7]);
        if (!h.good || !lse || !d || !ws || !ws->is_cuda() || !g.good) Py_RETURN_NONE;
        void *const stream = current_stream();
        return released([&] {
            return g_head.ce_backward(data(h.H), data(h.W), data(h.targets), data(lse), data(d), h.tokens, h.d, h.vocab, data(g.dH), data(g.dW), data(ws), ws->nbytes(),
                                      stream);
        });
    });
}

// (H, W, top_idx, top_logits, tau, kd, lse, workspace, targets, ce)
PyObject *head_distill(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n == 10 && g_head.distill, [&]() -> PyObject * {
        const Head h(a[0], a[1], a[8], true);
        const Teacher t(h, a[2], a[3], a[4]);
        const at::Tensor *kd = vector(a[5], at::kFloat, h.tokens), *lse = matrix(a[6], at::kFloat, 2, h.tokens), *ws = plain(a[7]), *ce = vector(a[9], at::kFloat, h.tokens);
        if (!h.good || !t.good || !kd || !lse || !ws || !ws->is_cuda() || !maybe(a[9], ce)) Py_RETURN_NONE;
        void *const stream = current_stream();
        return released([&] {
            return g_head.distill(data(h.H), data(h.W), data(t.idx), data(t.logits), t.type, t.idx->size(1), (float)t.tau, data(h.targets), h.tokens, h.d, h.vocab, data(kd),
                                  data(ce), data(lse), data(ws), ws->nbytes(), stream);
        });
    });
}

// (H, W, top_idx, top_logits, tau, lse, d_kd, workspace, targets, d_ce, dH, dW)
PyObject *head_distill_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n == 12 && g_head.distill_backward, [&]() -> PyObject * {
        const Head h(a[0], a[1], a[8], true);
        const Teacher t(h, a[2], a[3], a[4]);
        const at::Tensor *lse = matrix(a[5], at::kFloat, 2, h.tokens), *kd = vector(a[6], at::kFloat, h.tokens), *ws = plain(a[7]), *d = vector(a[9], at::kFloat, h.tokens);
        const Gradients g(h, a[10], a[11]);
        if (!h.good || !t.good || !lse || !kd || !ws || !ws->is_cuda() || !maybe(a[9], d) || !g.good) Py_RETURN_NONE;
        void *const stream = current_stream();
        return released([&] {
            return g_head.distill_backward(data(h.H), data(h.W), data(t.idx), data(t.logits), t.type, t.idx->size(1), (float)t.tau, data(h.targets), data(lse), data(kd),
                                           data(d), h.tokens, h.d, h.vocab, data(g.dH), data(g.dW), data(ws), ws->nbytes(), stream);
        });
    });
}

// codes and scales (uint8, any shape) of a [rows, cols] matrix
struct Mxfp4 {
    const at::Tensor *codes, *scales;
    bool good;
    Mxfp4(PyObject *c, PyObject *s, int64_t rows, int64_t cols) : codes(plain(c)), scales(plain(s))
    {
        const int64_t wide = (cols + 127) / 128 * 128;
        good = codes && scales && bytes(codes, rows * wide / 2) && bytes(scales, rows * wide / 32);
    }
    static bool bytes(const at::Tensor *t, int64_t n) { return t->is_cuda() && t->scalar_type() == at::kByte && t->numel() == n && t->is_contiguous(); }
};

const at::Tensor *floats(PyObject *o, int &type)
{
    const at::Tensor *t = matrix(o, at::kFloat, -1, -1);
    type = t ? 0 : 1;
    return t ? t : matrix(o, at::kBFloat16, -1, -1);
}

// (X, codes, scales)
PyObject *mxfp4_quantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n == 3 && g_head.quantize, [&]() -> PyObject * {
        int type;
        const at::Tensor *X = floats(a[0], type);
        if (!X) Py_RETURN_NONE;
        const Mxfp4 m(a[1], a[2], X->size(0), X->size(1));
        if (!m.good) Py_RETURN_NONE;
        void *const stream = current_stream();
        return released([&] { return g_head.quantize(data(X), type, X->size(0), X->size(1), data(m.codes), data(m.scales), stream); });
    });
}

// (codes, scales, Y)
PyObject *mxfp4_dequantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n == 3 && g_head.dequantize, [&]() -> PyObject * {
        int type;
        const at::Tensor *Y = floats(a[2], type);
        if (!Y) Py_RETURN_NONE;
        const Mxfp4 m(a[0], a[1], Y->size(0), Y->size(1));
        if (!m.good) Py_RETURN_NONE;
        void *const stream = current_stream();
        return released([&] { return g_head.dequantize(data(m.codes), data(m.scales), Y->size(0), Y->size(1), data(Y), type, stream); });
    });
}

// (X, codes, scales, Y, workspace, bias)
PyObject *mxfp4_linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n == 6 && g_head.mx_linear, [&]() -> PyObject * {
        const at::Tensor *X = matrix(a[0], at::kBFloat16, -1, -1), *ws = plain(a[4]);
        const at::Tensor *Y = X ? matrix(a[3], at::kFloat, X->size(0), -1) : nullptr;
        if (!Y || !ws || !ws->is_cuda()) Py_RETURN_NONE;
        const int64_t d_out = Y->size(1);
        const Mxfp4 m(a[1], a[2], d_out, X->size(1));
        const at::Tensor *bias = vector(a[5], at::kFloat, d_out);
        if (!m.good || !maybe(a[5], bias)) Py_RETURN_NONE;
        void *const stream = current_stream();
        return released(
            [&] { return g_head.mx_linear(data(X), X->size(0), X->size(1), d_out, data(m.codes), data(m.scales), data(bias), data(Y), data(ws), ws->nbytes(), stream); });
    });
}

// sizes, as whole numbers -> bytes, or None (the Python code raises the error)
bool whole(PyObject *const *a, Py_ssize_t n, int64_t *v)
{
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (!PyLong_CheckExact(a[i])) return false;
        v[i] = PyLong_AsLongLong(a[i]);
        if (v[i] == -1 && PyErr_Occurred()) {
            PyErr_Clear();
            return false;
        }
    }
    return true;
}
PyObject *head_bytes(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    int64_t v[5];
    size_t bytes;
    if (n != 5 || !g_head.head_bytes || !whole(a, 5, v) || g_head.head_bytes(v[0], v[1], v[2], v[3], v[4] != 0, &bytes) != 0) Py_RETURN_NONE;
    return PyLong_FromSize_t(bytes);
}
PyObject *mxfp4_bytes(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    int64_t v[2];
    size_t codes, scales;
    if (n != 2 || !g_head.mx_bytes || !whole(a, 2, v) || g_head.mx_bytes(v[0], v[1], &codes, &scales) != 0) Py_RETURN_NONE;
    return Py_BuildValue("nn", (Py_ssize_t)codes, (Py_ssize_t)scales);
}
PyObject *mxfp4_workspace_bytes(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    int64_t v[2];
    size_t bytes;
    if (n != 2 || !g_head.mx_workspace || !whole(a, 2, v) || g_head.mx_workspace(v[0], v[1], &bytes) != 0) Py_RETURN_NONE;
    return PyLong_FromSize_t(bytes);
}

// addresses of the C ABI's functions of this part, in the order of HeadCalls
PyObject *bind_head(PyObject *, PyObject *args)
{
    unsigned long long f[10];
    if (!PyArg_ParseTuple(args, "KKKKKKKKKK", f, f + 1, f + 2, f + 3, f + 4, f + 5, f + 6, f + 7, f + 8, f + 9)) return nullptr;
    g_head = HeadCalls{reinterpret_cast<ce_fn>(f[0]),         reinterpret_cast<ce_backward_fn>(f[1]), reinterpret_cast<distill_fn>(f[2]),
                       reinterpret_cast<distill_backward_fn>(f[3]), reinterpret_cast<quantize_fn>(f[4]), reinterpret_cast<dequantize_fn>(f[5]),
                       reinterpret_cast<mx_linear_fn>(f[6]),  reinterpret_cast<head_bytes_fn>(f[7]),  reinterpret_cast<mx_bytes_fn>(f[8]),
                       reinterpret_cast<mx_workspace_fn>(f[9])};
    Py_RETURN_NONE;
}

// (object, count): whether the grouped call takes the object as an array
template <Array::Kind KIND> PyObject *takes_array(PyObject *, PyObject *args)
{
    PyObject *o;
    int count;
    if (!PyArg_ParseTuple(args, "Oi", &o, &count)) return nullptr;
    return PyBool_FromLong(Array(o, count, KIND).held);
}

PyObject *stream(PyObject *, PyObject *) { return PyLong_FromVoidPtr(current_stream()); }

// (address of a C function without arguments): called as the library's functions are
PyObject *call(PyObject *, PyObject *args)
{
    unsigned long long f;
    if (!PyArg_ParseTuple(args, "K", &f)) return nullptr;
    return released(reinterpret_cast<int (*)()>(f));
}

// addresses of the C ABI's functions in the library that the binding has loaded
PyObject *bind(PyObject *, PyObject *args)
{
    unsigned long long l, g;
    if (!PyArg_ParseTuple(args, "KK", &l, &g)) return nullptr;
    g_linear = reinterpret_cast<linear_fn>(l);
    g_grouped = reinterpret_cast<grouped_fn>(g);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear)), METH_FASTCALL, nullptr},
    {"grouped", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(grouped)), METH_FASTCALL, nullptr},
    {"head_ce", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(head_ce)), METH_FASTCALL, nullptr},
    {"head_ce_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(head_ce_backward)), METH_FASTCALL, nullptr},
    {"head_distill", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(head_distill)), METH_FASTCALL, nullptr},
    {"head_distill_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(head_distill_backward)), METH_FASTCALL, nullptr},
    {"mxfp4_quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mxfp4_quantize)), METH_FASTCALL, nullptr},
    {"mxfp4_dequantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mxfp4_dequantize)), METH_FASTCALL, nullptr},
    {"mxfp4_linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mxfp4_linear)), METH_FASTCALL, nullptr},
    {"head_bytes", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(head_bytes)), METH_FASTCALL, nullptr},
    {"mxfp4_bytes", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mxfp4_bytes)), METH_FASTCALL, nullptr},
    {"mxfp4_workspace_bytes", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mxfp4_workspace_bytes)), METH_FASTCALL, nullptr},
    {"bind_head", bind_head, METH_VARARGS, nullptr},
    {"array_of_pointers", takes_array<Array::POINTERS>, METH_VARARGS, nullptr},
    {"array_of_integers", takes_array<Array::INTEGERS>, METH_VARARGS, nullptr},
    {"call", call, METH_VARARGS, nullptr},
    {"stream", stream, METH_NOARGS, nullptr},
    {"bind", bind, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall()
{
    PyObject *m = PyModule_Create(&module);
    // tensors are read by the layout of this version's headers, so the binding compares it with the torch that runs
    if (m && PyModule_AddStringConstant(m, "torch_version", SBN_TORCH_VERSION) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
