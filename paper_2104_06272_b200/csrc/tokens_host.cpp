// Host side of tokens.py: checks of torch tensors, outputs and workspaces from torch's allocator, and the stateless calls of anakin.h on the tensors'
// device and its current torch stream.  In C++ because the smallest of these calls cost the host more than the GPU: from Python, with ctypes, a call
// took 9 us and its kernels 2 to 6; this way 5 us.
//
// Every function takes its arguments by position (tokens.py has the names and the documentation) and refuses by raising the binding's error class,
// handed over once with set_error, before anything is enqueued.  What touches Python objects comes first; allocations and launches run without the
// interpreter's lock (`On`).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cfloat>
#include <cmath>
#include <cstring>
#include <string>

#include "anakin.h"

namespace {

PyObject* g_error = nullptr;

struct Refusal {
    int code;
    std::string why;
};
[[noreturn]] void refuse(const std::string& why, int code = ANAKIN_E_INVALID_ARG) { throw Refusal{code, why}; }
struct PythonError {};  // already set

int dtype_of(at::ScalarType t) {
    return t == at::kFloat ? ANAKIN_DTYPE_F32 : t == at::kBFloat16 ? ANAKIN_DTYPE_BF16 : t == at::kHalf ? ANAKIN_DTYPE_F16 : -1;
}
const char* name_of(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return "float32";
        case at::kBFloat16: return "bfloat16";
        case at::kHalf: return "float16";
        case at::kLong: return "int64";
        case at::kInt: return "int32";
        case at::kBool: return "bool";
        case at::kByte: return "uint8";
        default: return c10::toString(t);
    }
}

// The tensor behind an argument; undefined for None.
at::Tensor tensor(const char* name, PyObject* o) {
    if (o == Py_None) return at::Tensor();
    if (!THPVariable_Check(o)) refuse(std::string(name) + ": a tensor is needed");
    return THPVariable_Unpack(o);
}

struct Matrix {
    at::Tensor t;
    int64_t rows = 0, cols = 0, ld = 0;
    int dtype = 0;
    void* p() const { return t.data_ptr(); }
};
// A matrix of one of the three types whose rows are dense.
Matrix matrix(const char* name, const at::Tensor& t) {
    if (!t.defined() || !t.is_cuda() || t.dim() != 2 || dtype_of(t.scalar_type()) < 0 || t.size(1) < 1)
        refuse(std::string(name) + ": a CUDA matrix of float32, bfloat16 or float16 with at least one column is needed");
    Matrix m{t, t.size(0), t.size(1), t.size(0) > 1 ? t.stride(0) : t.size(1), dtype_of(t.scalar_type())};
    if ((m.cols > 1 && t.stride(1) != 1) || m.ld < m.cols) refuse(std::string(name) + ": columns have to lie side by side, and rows one after the other");
    return m;
}
// The same, of a given shape and type on a given device.
Matrix matrix(const char* name, const at::Tensor& t, int64_t rows, int64_t cols, at::ScalarType type, c10::Device dev) {
    const Matrix m = matrix(name, t);
    if (m.rows != rows || m.cols != cols || t.scalar_type() != type || t.device() != dev)
        refuse(std::string(name) + ": " + name_of(type) + " of shape (" + std::to_string(rows) + ", " + std::to_string(cols) + ") on " + dev.str() + " is needed");
    return m;
}
// Address of a dense vector of n numbers on that device; None: null.
void* vector(const char* name, PyObject* o, int64_t n, c10::Device dev, at::ScalarType a, at::ScalarType b) {
    const at::Tensor t = tensor(name, o);
    if (!t.defined()) return nullptr;
    if ((t.scalar_type() != a && t.scalar_type() != b) || t.dim() != 1 || t.size(0) != n || t.device() != dev || !t.is_contiguous())
        refuse(std::string(name) + ": a dense vector of " + std::to_string(n) + " numbers (" + name_of(a) + (a != b ? std::string(", ") + name_of(b) : "") + ") on " + dev.str() + " is needed");
    return t.data_ptr();
}
const float* vector(const char* name, PyObject* o, int64_t n, c10::Device dev) { return static_cast<const float*>(vector(name, o, n, dev, at::kFloat, at::kFloat)); }
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError{};
    return v != 0;
}
int64_t number(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw PythonError{};
    return v;
}
float real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError{};
    return std::abs(v) <= FLT_MAX ? (float)v : INFINITY;  // (NaN too: refused alike)
}

// (0.5 us; by way of at::empty and its dispatcher 0.7)
at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, c10::Device dev) { return at::detail::empty_cuda(shape, type, dev, std::nullopt); }
at::Tensor floats(int64_t n, c10::Device dev) { return empty({n}, at::kFloat, dev); }
at::Tensor bytes(size_t n, c10::Device dev) { return empty({(int64_t)n}, at::kByte, dev); }
// An output matrix: `out`, checked; without one (no tensor in it yet) it is made by made().
Matrix output(PyObject* out, int64_t rows, int64_t cols, at::ScalarType type, c10::Device dev) {
    const at::Tensor t = tensor("out", out);
    return t.defined() ? matrix("out", t, rows, cols, type, dev) : Matrix{t, rows, cols, cols, dtype_of(type)};
}
Matrix output_like(PyObject* out, const Matrix& l) { return output(out, l.rows, l.cols, l.t.scalar_type(), l.t.device()); }
void made(Matrix& m, at::ScalarType type, c10::Device dev) {
    if (!m.t.defined()) m.t = empty({m.rows, m.cols}, type, dev);
}

// The tensors' device as the current one, its current stream, and the interpreter's lock released.
struct On {
    struct Unlocked {
        PyThreadState* state = PyEval_SaveThread();
        ~Unlocked() { PyEval_RestoreThread(state); }
    } unlocked;
    c10::cuda::CUDAGuard guard;
    void* stream;
    explicit On(c10::Device dev) : guard(dev), stream(c10::cuda::getCurrentCUDAStream(dev.index()).stream()) {}
};

void check(int rc) {
    if (rc != ANAKIN_OK) refuse("", rc);
}

anakin_token_rows token_rows(c10::Device dev, int64_t n, PyObject* tokens, PyObject* mask, PyObject* offsets, const Matrix* logits = nullptr, float scale = 1.0f) {
    anakin_token_rows r = {};
    r.struct_size = sizeof(r);
    r.rows = n;
    r.scale = scale;
    if (logits) {
        r.dtype = logits->dtype;
        r.vocab = logits->cols;
        r.ld = logits->ld;
        r.logits = logits->p();
    }
    if (tokens != Py_None) {
        r.tokens = vector("tokens", tokens, n, dev, at::kLong, at::kInt);
        r.token_bytes = THPVariable_Unpack(tokens).scalar_type() == at::kLong ? 8 : 4;
    }
    r.mask = static_cast<const uint8_t*>(vector("mask", mask, n, dev, at::kBool, at::kByte));
    if (offsets != Py_None) {
        const int64_t count = tensor("offsets", offsets).numel();
        if (count < 1) refuse("offsets: one number more than there are sequences");
        r.offsets = vector("offsets", offsets, count, dev, at::kLong, at::kInt);
        r.offset_bytes = THPVariable_Unpack(offsets).scalar_type() == at::kLong ? 8 : 4;
        r.sequences = count - 1;
    }
    return r;
}
at::Tensor token_workspace(const anakin_token_rows& r, c10::Device dev, size_t* size) {
    check(anakin_token_workspace_bytes(r.rows, r.sequences, size));
    return bytes(*size, dev);
}
template <class T> T objective(PyObject* o) {
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw PythonError{};
    T t = {};
    const bool fits = b.len == (Py_ssize_t)sizeof(T);
    if (fits) memcpy(&t, b.buf, sizeof(T));
    PyBuffer_Release(&b);
    if (!fits) refuse("objective: of another kind");
    return t;
}

PyObject* wrap(const at::Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    PyObject* o = THPVariable_Wrap(t);
    if (!o) throw PythonError{};
    return o;
}
template <class... T> PyObject* tuple(const T&... t) {
    PyObject* r = PyTuple_New(sizeof...(T));
    if (!r) throw PythonError{};
    Py_ssize_t i = 0;
    try {
        (void)std::initializer_list<int>{(PyTuple_SET_ITEM(r, i++, wrap(t)), 0)...};
    } catch (...) {
        Py_DECREF(r);
        throw;
    }
    return r;
}

using Args = PyObject* const*;

// logits, tokens, scale, mask, entropy? -> logp, entropy, norm
PyObject* logp(Args a) {
    const Matrix x = matrix("logits", tensor("logits", a[0]));
    const c10::Device dev = x.t.device();
    if (a[1] == Py_None) refuse("tokens are needed");
    const anakin_token_rows r = token_rows(dev, x.rows, a[1], a[3], Py_None, &x, real(a[2]));
    const bool want = truth(a[4]);
    at::Tensor lp, ent, norm;
    {
        const On on(dev);
        lp = floats(x.rows, dev), norm = empty({x.rows, 2}, at::kFloat, dev);
        if (want) ent = floats(x.rows, dev);
        check(anakin_token_logp(&r, lp.data_ptr<float>(), want ? ent.data_ptr<float>() : nullptr, norm.data_ptr<float>(), on.stream));
    }
    return tuple(lp, ent, norm);
}

// logits, tokens, norm, dlogp, entropy, dentropy, scale, mask, out -> dlogits
PyObject* logp_backward(Args a) {
    const Matrix x = matrix("logits", tensor("logits", a[0]));
    const c10::Device dev = x.t.device();
    if (a[1] == Py_None || a[3] == Py_None || (a[5] != Py_None && a[4] == Py_None)) refuse("tokens, norm and dlogp are needed, and entropy with dentropy");
    const anakin_token_rows r = token_rows(dev, x.rows, a[1], a[7], Py_None, &x, real(a[6]));
    const Matrix norm = matrix("norm", tensor("norm", a[2]), x.rows, 2, at::kFloat, dev);
    if (norm.ld != 2) refuse("norm: its rows lie one behind the other");
    const float* dl = vector("dlogp", a[3], x.rows, dev);
    const float *ent = vector("entropy", a[4], x.rows, dev), *dent = vector("dentropy", a[5], x.rows, dev);
    Matrix out = output_like(a[8], x);
    {
        const On on(dev);
        made(out, x.t.scalar_type(), dev);
        check(anakin_token_logp_backward(&r, static_cast<const float*>(norm.p()), ent, dl, dent, out.p(), out.ld, on.stream));
    }
    return wrap(out.t);
}

// objective, logp, old_logp, adv, ref_logp, entropy, mask, offsets, tokens -> stats, dlogp, dentropy
PyObject* policy_loss(Args a) {
    const at::Tensor lp = tensor("logp", a[1]);
    if (!lp.defined() || !lp.is_cuda() || lp.dim() != 1) refuse("logp: a CUDA vector is needed");
    const auto o = objective<anakin_policy_objective>(a[0]);
    const c10::Device dev = lp.device();
    const int64_t n = lp.size(0);
    auto f = [&](const char* name, int i) { return vector(name, a[i], n, dev); };
    const float *l = f("logp", 1), *old = f("old_logp", 2), *adv = f("adv", 3), *ref = f("ref_logp", 4), *ent = f("entropy", 5);
    if (a[3] == Py_None || (o.kl != ANAKIN_KL_NONE && a[4] == Py_None)) refuse("adv is needed, and ref_logp with a KL term");
    const anakin_token_rows r = token_rows(dev, n, a[8], a[6], a[7]);
    const bool want = a[5] != Py_None;
    at::Tensor stats, dl, dent;
    {
        const On on(dev);
        size_t size = 0;
        const at::Tensor ws = token_workspace(r, dev, &size);
        stats = floats(ANAKIN_POLICY_STATS, dev), dl = floats(n, dev);
        if (want) dent = floats(n, dev);
        check(anakin_token_policy_loss(&r, &o, l, old, adv, ref, ent, stats.data_ptr<float>(), dl.data_ptr<float>(), want ? dent.data_ptr<float>() : nullptr,
                                       ws.data_ptr(), size, on.stream));
    }
    return tuple(stats, dl, dent);
}

// objective, logits, tokens, old_logp, adv, ref_logp, mask, offsets, scale, out -> stats, logp, entropy, dlogits
PyObject* policy_grad(Args a) {
    const Matrix x = matrix("logits", tensor("logits", a[1]));
    const auto o = objective<anakin_policy_objective>(a[0]);
    const c10::Device dev = x.t.device();
    const int64_t n = x.rows;
    auto f = [&](const char* name, int i) { return vector(name, a[i], n, dev); };
    const float *old = f("old_logp", 3), *adv = f("adv", 4), *ref = f("ref_logp", 5);
    if (a[2] == Py_None || a[4] == Py_None || (o.kl != ANAKIN_KL_NONE && a[5] == Py_None)) refuse("tokens and adv are needed, and ref_logp with a KL term");
    const anakin_token_rows r = token_rows(dev, n, a[2], a[6], a[7], &x, real(a[8]));
    Matrix out = output_like(a[9], x);
    at::Tensor stats, lp, ent;
    {
        const On on(dev);
        size_t size = 0;
        const at::Tensor ws = token_workspace(r, dev, &size);
        stats = floats(ANAKIN_POLICY_STATS, dev), lp = floats(n, dev), ent = floats(n, dev);
        made(out, x.t.scalar_type(), dev);
        check(anakin_token_policy_grad(&r, &o, old, adv, ref, stats.data_ptr<float>(), lp.data_ptr<float>(), ent.data_ptr<float>(), out.p(), out.ld, ws.data_ptr(),
                                       size, on.stream));
    }
    return tuple(stats, lp, ent, out.t);
}

// objective, logp, offsets, ref_logp, mask, tokens -> stats, margin, dlogp
PyObject* preference_loss(Args a) {
    const at::Tensor lp = tensor("logp", a[1]), off = tensor("offsets", a[2]);
    if (!lp.defined() || !lp.is_cuda() || lp.dim() != 1) refuse("logp: a CUDA vector is needed");
    if (!off.defined() || off.numel() % 2 == 0) refuse("offsets of an even number of sequences are needed");
    const auto o = objective<anakin_preference_objective>(a[0]);
    const c10::Device dev = lp.device();
    const int64_t n = lp.size(0);
    const float *l = vector("logp", a[1], n, dev), *ref = vector("ref_logp", a[3], n, dev);
    const anakin_token_rows r = token_rows(dev, n, a[5], a[4], a[2]);
    at::Tensor stats, z, dl;
    {
        const On on(dev);
        size_t size = 0;
        const at::Tensor ws = token_workspace(r, dev, &size);
        stats = floats(ANAKIN_PREFERENCE_STATS, dev), z = floats(r.sequences / 2, dev), dl = floats(n, dev);
        check(anakin_token_preference_loss(&r, &o, l, ref, stats.data_ptr<float>(), z.data_ptr<float>(), dl.data_ptr<float>(), ws.data_ptr(), size, on.stream));
    }
    return tuple(stats, z, dl);
}

struct Kept {
    at::Tensor codes, scales;
    int64_t rows, cols;
    const uint8_t* c() const { return codes.data_ptr<uint8_t>(); }
    const uint8_t* s() const { return scales.data_ptr<uint8_t>(); }
};
// A checkpoint: codes, scales, columns.
Kept kept(Args a) {
    Kept k{tensor("codes", a[0]), tensor("scales", a[1]), 0, number(a[2])};
    if (k.cols < 1 || k.cols > INT32_MAX) refuse("a checkpoint has one column at least");
    const int64_t blocks = (k.cols + 31) / 32;
    auto dense = [](const at::Tensor& t) { return t.defined() && t.is_cuda() && t.scalar_type() == at::kByte && t.dim() == 2 && t.is_contiguous(); };
    if (!dense(k.codes) || k.codes.size(1) != blocks * 32) refuse("codes: a dense CUDA matrix of uint8 with " + std::to_string(blocks * 32) + " columns is needed");
    k.rows = k.codes.size(0);
    if (!dense(k.scales) || k.scales.size(0) != k.rows || k.scales.size(1) != blocks || k.scales.device() != k.codes.device())
        refuse("scales: a dense matrix of uint8, " + std::to_string(k.rows) + " x " + std::to_string(blocks) + ", is needed beside the codes");
    return k;
}

// x, act, y?, out -> y, codes, scales
PyObject* ckpt_forward(Args a) {
    const Matrix x = matrix("x", tensor("x", a[0]));
    const c10::Device dev = x.t.device();
    const int64_t blocks = (x.cols + 31) / 32;
    const int act = (int)number(a[1]);
    const bool want = truth(a[2]);
    Matrix y = want ? output_like(a[3], x) : Matrix{};
    at::Tensor codes, scales;
    {
        const On on(dev);
        if (want) made(y, x.t.scalar_type(), dev);
        codes = empty({x.rows, blocks * 32}, at::kByte, dev), scales = empty({x.rows, blocks}, at::kByte, dev);
        check(anakin_ckpt_forward(x.dtype, act, x.rows, x.cols, x.p(), x.ld, want ? y.p() : nullptr, y.ld, codes.data_ptr<uint8_t>(), scales.data_ptr<uint8_t>(),
                                  on.stream));
    }
    return tuple(y.t, codes, scales);
}

// checkpoint (3), type of a new output (ANAKIN_DTYPE_*), out -> x
PyObject* ckpt_unpack(Args a) {
    const Kept k = kept(a);
    const c10::Device dev = k.codes.device();
    const at::Tensor given = tensor("out", a[4]);
    const int64_t want = number(a[3]);
    const at::ScalarType type = given.defined() ? given.scalar_type() : want == ANAKIN_DTYPE_F32 ? at::kFloat : want == ANAKIN_DTYPE_BF16 ? at::kBFloat16 : at::kHalf;
    Matrix out = output(a[4], k.rows, k.cols, type, dev);
    {
        const On on(dev);
        made(out, type, dev);
        check(anakin_ckpt_unpack(out.dtype, k.rows, k.cols, k.c(), k.s(), out.p(), out.ld, on.stream));
    }
    return wrap(out.t);
}

// checkpoint (3), dy, act, out -> dx
PyObject* ckpt_backward(Args a) {
    const Kept k = kept(a);
    const c10::Device dev = k.codes.device();
    const at::Tensor t = tensor("dy", a[3]);
    const Matrix dy = matrix("dy", t, k.rows, k.cols, t.defined() ? t.scalar_type() : at::kFloat, dev);
    const int act = (int)number(a[4]);
    Matrix out = output_like(a[5], dy);
    {
        const On on(dev);
        made(out, t.scalar_type(), dev);
        check(anakin_ckpt_backward(dy.dtype, act, k.rows, k.cols, k.c(), k.s(), dy.p(), dy.ld, out.p(), out.ld, on.stream));
    }
    return wrap(out.t);
}

// checkpoint (3), dy, act, out, accumulate?, status -> dw
PyObject* ckpt_weight_grad(Args a) {
    const Kept k = kept(a);
    const c10::Device dev = k.codes.device();
    const Matrix dy = matrix("dy", tensor("dy", a[3]));
    if (dy.rows != k.rows || dy.t.device() != dev) refuse("dy: " + std::to_string(k.rows) + " rows on " + dev.str() + " are needed");
    const int act = (int)number(a[4]), add = truth(a[6]);
    if (act != ANAKIN_ACT_IDENTITY && act != ANAKIN_ACT_RELU) refuse("act is identity or relu here: checkpoint the activation's output", ANAKIN_E_UNSUPPORTED_CFG);
    if (add && a[5] == Py_None) refuse("accumulate adds to `out`");
    auto* status = static_cast<int32_t*>(vector("status", a[7], 1, dev, at::kInt, at::kInt));
    Matrix dw = output(a[5], k.cols, dy.cols, at::kFloat, dev);
    {
        const On on(dev);
        made(dw, at::kFloat, dev);
        size_t size = 0;
        const bool aligned = (((uintptr_t)dy.p() | (uintptr_t)(dy.ld * dy.t.element_size())) & 15) == 0;
        check(anakin_ckpt_weight_grad_workspace_bytes(dy.dtype, k.rows, k.cols, dy.cols, aligned, &size));
        const at::Tensor ws = bytes(size, dev);
        check(anakin_ckpt_weight_grad(dy.dtype, act, k.rows, k.cols, dy.cols, k.c(), k.s(), dy.p(), dy.ld, static_cast<float*>(dw.p()), dw.ld, add, ws.data_ptr(), size,
                                      status, on.stream));
    }
    return wrap(dw.t);
}

// A call with N arguments; refusals as the error class, torch's own errors (out of memory) as torch raises them.
template <PyObject* (*F)(Args), int N>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    HANDLE_TH_ERRORS
    try {
        return F(args);
    } catch (const Refusal& e) {
        if (!g_error) {
            PyErr_SetString(PyExc_RuntimeError, e.why.c_str());
        } else if (PyObject* exc = PyObject_CallFunction(g_error, "is", e.code, e.why.c_str())) {
            PyErr_SetObject(g_error, exc);
            Py_DECREF(exc);
        }
    } catch (const PythonError&) {
    }
    return nullptr;
    END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* cls) {
    Py_INCREF(cls);
    Py_XDECREF(g_error);
    g_error = cls;
    Py_RETURN_NONE;
}

#define CALL(f, n) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<f, n>)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {
    CALL(logp, 5), CALL(logp_backward, 9), CALL(policy_loss, 9), CALL(policy_grad, 10), CALL(preference_loss, 6),
    CALL(ckpt_forward, 4), CALL(ckpt_unpack, 5), CALL(ckpt_backward, 6), CALL(ckpt_weight_grad, 8),
    {"set_error", set_error, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_tokens_host", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tokens_host(void) { return PyModule_Create(&kModule); }
