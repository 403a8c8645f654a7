// Argument marshalling of binding.py in native code: the checks that the Python functions make, the output tensors, the current
// stream and the call of the C entry point.  In Python these bound what a latency-bound program gets: host time of a call with its
// launches, Python -> here, one query over a ragged corpus 9.2 -> 4.4 us, over a uniform one 8.5 -> 4.2, forward with argmax 10.5 -> 5.1,
// cross-entropy gradient 9.2 -> 5.1, backward 11.9 -> 5.4, a training step of 16 x 16 31.7 -> 15.2.
//
// A function returns the Python function's result, an int (the error code of the C entry point), or None where anything about the
// call is out of the ordinary -- a tensor of another class, kind, type, shape, device or memory layout, an active
// mode that watches torch calls, a value it does not know.  binding.py then does the same work in Python and raises what there is to raise.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/TensorSubclassLikeUtils.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cmath>
#include <vector>

#include "../../include/maxsim.h"

namespace {

struct Entries {
    decltype(&maxsim_forward) forward;
    decltype(&maxsim_forward_ragged) forward_ragged;
    decltype(&maxsim_backward) backward;
    decltype(&maxsim_backward_ragged) backward_ragged;
    decltype(&maxsim_ce_grad) ce_grad;
    decltype(&maxsim_quantize_rows_i8) quantize;
    decltype(&maxsim_forward_i8) forward_i8;
    decltype(&maxsim_forward_i8_ragged) forward_i8_ragged;
    decltype(&maxsim_rope) rope;
    decltype(&maxsim_attention_workspace) attention_workspace;
    decltype(&maxsim_attention) attention;
    decltype(&maxsim_attention_backward_workspace) attention_backward_workspace;
    decltype(&maxsim_attention_backward) attention_backward;
    decltype(&maxsim_clip_workspace) clip_workspace;
    decltype(&maxsim_clip_grad_norm) clip_grad_norm;
} entry;

// One call's arguments.  ok() after everything has been looked at: nothing was out of the ordinary.
class Call {
public:
    explicit Call(PyObject *first) { ok_ = !c10::impl::TorchDispatchModeTLS::any_modes_set() && !at::impl::torch_function_mode_enabled() && plain(first) != nullptr; }

    bool ok() const { return ok_; }
    void require(bool x) { ok_ = ok_ && x; }

    // A contiguous tensor of the call's GPU, which is that of the first one and the current one
    const at::Tensor &tensor(PyObject *o, int dims)
    {
        const at::Tensor *t = ok_ ? plain(o) : nullptr;
        if (!t || t->dim() != dims || !t->is_contiguous()) {
            ok_ = false;
            return none();
        }
        on_device(*t);
        return *t;
    }
    const at::Tensor &tensor(PyObject *o) // of any number of dimensions
    {
        const at::Tensor *t = ok_ ? plain(o) : nullptr;
        return t ? tensor(o, (int)t->dim()) : (ok_ = false, none());
    }
    const at::Tensor &tensor(PyObject *o, at::IntArrayRef shape, at::ScalarType type)
    {
        const at::Tensor &t = tensor(o, (int)shape.size());
        ok_ = ok_ && t.scalar_type() == type && t.sizes() == shape;
        return ok_ ? t : none();
    }
    // A packed tensor [tokens, heads, d], which may be a view with rows of stride 1, and its two strides
    const at::Tensor &rows(PyObject *o, int64_t *strides)
    {
        const at::Tensor *t = ok_ ? plain(o) : nullptr;
        if (!t || t->dim() != 3 || t->numel() == 0 || (t->size(2) > 1 && t->stride(2) != 1)) {
            ok_ = false;
            return none();
        }
        on_device(*t);
        strides[0] = t->size(0) > 1 ? t->stride(0) : t->size(2);
        strides[1] = t->size(1) > 1 ? t->stride(1) : t->size(2);
        return *t;
    }
    const at::Tensor &rows(PyObject *o, int64_t *strides, const at::Tensor &like)
    {
        const at::Tensor &t = rows(o, strides);
        ok_ = ok_ && t.scalar_type() == like.scalar_type() && t.sizes() == like.sizes();
        return ok_ ? t : none();
    }
    at::Tensor output_rows(PyObject *o, int64_t *strides, const at::Tensor &like)
    {
        if (o != Py_None)
            return rows(o, strides, like);
        if (!ok_)
            return at::Tensor();
        strides[0] = like.size(0) > 1 ? like.size(1) * like.size(2) : like.size(2);
        strides[1] = like.size(2);
        return at::empty(like.sizes(), at::TensorOptions().dtype(like.scalar_type()).device(at::kCUDA, device_));
    }
    at::Tensor workspace(PyObject *o, int64_t bytes) // the caller's, of any length, or a new one
    {
        if (o != Py_None) {
            const at::Tensor &t = tensor(o, 1);
            ok_ = ok_ && t.scalar_type() == at::kByte;
            return ok_ ? t : none();
        }
        return ok_ && bytes ? at::empty({bytes}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, device_)) : at::Tensor();
    }
    // The caller's output or, for None, a new one
    at::Tensor output(PyObject *o, at::IntArrayRef shape, at::ScalarType type)
    {
        if (o != Py_None)
            return tensor(o, shape, type);
        return ok_ ? at::empty(shape, at::TensorOptions().dtype(type).device(at::kCUDA, device_)) : at::Tensor();
    }
    int size(int64_t n)
    {
        ok_ = ok_ && n >= 0 && n <= INT_MAX;
        return ok_ ? (int)n : 0;
    }
    maxsim_dtype dtype(const at::Tensor &t)
    {
        switch (ok_ ? t.scalar_type() : at::ScalarType::Undefined) {
        case at::ScalarType::Float: return MAXSIM_F32;
        case at::ScalarType::Half: return MAXSIM_F16;
        case at::ScalarType::BFloat16: return MAXSIM_BF16;
        default: ok_ = false; return MAXSIM_F32;
        }
    }
    void *stream() const { return c10::hip::getCurrentHIPStream((c10::DeviceIndex)device_).stream(); }

private:
    void on_device(const at::Tensor &t)
    {
        if (device_ < 0) {
            device_ = t.get_device();
            ok_ = device_ == c10::hip::current_device();
        }
        ok_ = ok_ && t.get_device() == device_;
    }
    static const at::Tensor &none() // (not looked at: ok() is false)
    {
        static const at::Tensor t;
        return t;
    }
    static const at::Tensor *plain(PyObject *o)
    {
        if (!THPVariable_CheckExact(o))
            return nullptr;
        const at::Tensor &t = THPVariable_Unpack(o);
        return t.defined() && t.is_cuda() && !at::isTensorSubclassLike(t) && t.layout() == at::kStrided && !t.is_neg() && !t.is_conj() ? &t : nullptr;
    }
    bool ok_ = false;
    int device_ = -1;
};

const void *in(const at::Tensor &t) { return t.data_ptr(); }
template <typename T> T *at_ptr(const at::Tensor &t) { return static_cast<T *>(t.data_ptr()); }

PyObject *give(PyObject *given, const at::Tensor &t) // the caller's own object, or the new tensor
{
    if (given == Py_None)
        return THPVariable_Wrap(t);
    Py_INCREF(given);
    return given;
}
PyObject *give2(PyObject *g0, const at::Tensor &t0, PyObject *g1, const at::Tensor &t1)
{
    PyObject *a = give(g0, t0);
    PyObject *b = a ? give(g1, t1) : nullptr;
    PyObject *r = b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    return r;
}

template <typename F> int without_gil(F &&f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

#define ARGUMENTS(N)                                                                                                   \
    if (n != (N)) {                                                                                                    \
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");                                                 \
        return nullptr;                                                                                                \
    }

// (Q, D, scores, argmax, want_argmax)
PyObject *forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(5)
    Call c(a[0]);
    const at::Tensor &Q = c.tensor(a[0], 3), &D = c.tensor(a[1], 3);
    const maxsim_dtype dt = c.dtype(Q);
    c.require(c.ok() && D.scalar_type() == Q.scalar_type() && D.size(2) == Q.size(2));
    if (!c.ok())
        Py_RETURN_NONE;
    const int n_q = c.size(Q.size(0)), l_q = c.size(Q.size(1)), d = c.size(Q.size(2)), l_d = c.size(D.size(1));
    const int64_t b = D.size(0);
    const int want = a[3] != Py_None ? 1 : PyObject_IsTrue(a[4]);
    if (want < 0)
        return nullptr;
    const at::Tensor scores = c.output(a[2], {n_q, b}, at::kFloat);
    const at::Tensor argmax = want ? c.output(a[3], {n_q, b, l_q}, at::kInt) : at::Tensor();
    if (!c.ok())
        Py_RETURN_NONE;
    const int rc = without_gil([&] {
        return entry.forward(in(Q), n_q, l_q, in(D), b, l_d, d, dt, at_ptr<float>(scores), want ? at_ptr<int32_t>(argmax) : nullptr, c.stream());
    });
    if (rc != 0)
        return PyLong_FromLong(rc);
    return want ? give2(a[2], scores, a[3], argmax) : give(a[2], scores);
    END_HANDLE_TH_ERRORS
}

// (Q, D_packed, doc_offsets, scores, argmax, want_argmax): all rows of D_packed
PyObject *forward_ragged(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(6)
    Call c(a[0]);
    const at::Tensor &Q = c.tensor(a[0], 3), &D = c.tensor(a[1], 2), &off = c.tensor(a[2], 1);
    const maxsim_dtype dt = c.dtype(Q);
    c.require(c.ok() && D.scalar_type() == Q.scalar_type() && D.size(1) == Q.size(2) && off.scalar_type() == at::kInt && off.size(0) >= 2);
    if (!c.ok())
        Py_RETURN_NONE;
    const int n_q = c.size(Q.size(0)), l_q = c.size(Q.size(1)), d = c.size(Q.size(2));
    const int64_t b = off.size(0) - 1, tokens = D.size(0);
    const int want = a[4] != Py_None ? 1 : PyObject_IsTrue(a[5]);
    if (want < 0)
        return nullptr;
    const at::Tensor scores = c.output(a[3], {n_q, b}, at::kFloat);
    const at::Tensor argmax = want ? c.output(a[4], {n_q, b, l_q}, at::kInt) : at::Tensor();
    if (!c.ok())
        Py_RETURN_NONE;
    const int rc = without_gil([&] {
        return entry.forward_ragged(in(Q), n_q, l_q, in(D), at_ptr<int32_t>(off), b, tokens, d, dt, at_ptr<float>(scores), want ? at_ptr<int32_t>(argmax) : nullptr, c.stream());
    });
    if (rc != 0)
        return PyLong_FromLong(rc);
    return want ? give2(a[3], scores, a[4], argmax) : give(a[3], scores);
    END_HANDLE_TH_ERRORS
}

// (Q, D, argmax, dscore, dQ, dD)
PyObject *backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(6)
    Call c(a[0]);
    const at::Tensor &Q = c.tensor(a[0], 3), &D = c.tensor(a[1], 3);
    const maxsim_dtype dt = c.dtype(Q);
    c.require(c.ok() && D.scalar_type() == Q.scalar_type() && D.size(2) == Q.size(2));
    if (!c.ok())
        Py_RETURN_NONE;
    const int n_q = c.size(Q.size(0)), l_q = c.size(Q.size(1)), d = c.size(Q.size(2)), l_d = c.size(D.size(1));
    const int64_t b = D.size(0);
    const at::Tensor &A = c.tensor(a[2], {n_q, b, l_q}, at::kInt), &g = c.tensor(a[3], {n_q, b}, at::kFloat);
    const at::Tensor dQ = c.output(a[4], {n_q, l_q, d}, at::kFloat);
    const at::Tensor dD = c.output(a[5], {b, l_d, d}, at::kFloat);
    if (!c.ok())
        Py_RETURN_NONE;
    const int rc = without_gil([&] {
        return entry.backward(in(Q), n_q, l_q, in(D), b, l_d, d, dt, at_ptr<int32_t>(A), at_ptr<float>(g), at_ptr<float>(dQ), at_ptr<float>(dD), c.stream());
    });
    return rc != 0 ? PyLong_FromLong(rc) : give2(a[4], dQ, a[5], dD);
    END_HANDLE_TH_ERRORS
}

// (Q, D_packed, doc_offsets, argmax, dscore, dQ, dD): all rows of D_packed
PyObject *backward_ragged(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(7)
    Call c(a[0]);
    const at::Tensor &Q = c.tensor(a[0], 3), &D = c.tensor(a[1], 2), &off = c.tensor(a[2], 1);
    const maxsim_dtype dt = c.dtype(Q);
    c.require(c.ok() && D.scalar_type() == Q.scalar_type() && D.size(1) == Q.size(2) && off.scalar_type() == at::kInt && off.size(0) >= 2);
    if (!c.ok())
        Py_RETURN_NONE;
    const int n_q = c.size(Q.size(0)), l_q = c.size(Q.size(1)), d = c.size(Q.size(2));
    const int64_t b = off.size(0) - 1, tokens = D.size(0);
    const at::Tensor &A = c.tensor(a[3], {n_q, b, l_q}, at::kInt), &g = c.tensor(a[4], {n_q, b}, at::kFloat);
    const at::Tensor dQ = c.output(a[5], {n_q, l_q, d}, at::kFloat);
    const at::Tensor dD = c.output(a[6], {tokens, d}, at::kFloat);
    if (!c.ok())
        Py_RETURN_NONE;
    const int rc = without_gil([&] {
        return entry.backward_ragged(in(Q), n_q, l_q, in(D), at_ptr<int32_t>(off), b, tokens, d, dt, at_ptr<int32_t>(A), at_ptr<float>(g), at_ptr<float>(dQ), at_ptr<float>(dD),
                                     c.stream());
    });
    return rc != 0 ? PyLong_FromLong(rc) : give2(a[5], dQ, a[6], dD);
    END_HANDLE_TH_ERRORS
}

// (scores, tau, g, loss)
PyObject *ce_grad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(4)
    Call c(a[0]);
    const at::Tensor &s = c.tensor(a[0], 2);
    if (!c.ok() || s.scalar_type() != at::kFloat || !PyFloat_CheckExact(a[1]))
        Py_RETURN_NONE;
    const int rows = c.size(s.size(0)), b = c.size(s.size(1));
    const float tau = (float)PyFloat_AS_DOUBLE(a[1]);
    const at::Tensor g = c.output(a[2], {rows, b}, at::kFloat);
    const at::Tensor loss = c.output(a[3], {1}, at::kFloat);
    if (!c.ok())
        Py_RETURN_NONE;
    const int rc = without_gil([&] { return entry.ce_grad(at_ptr<float>(s), rows, b, tau, at_ptr<float>(g), at_ptr<float>(loss), c.stream()); });
    return rc != 0 ? PyLong_FromLong(rc) : give2(a[2], g, a[3], loss);
    END_HANDLE_TH_ERRORS
}

// (X, X_i8, scale): X of two or three dimensions
PyObject *quantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(3)
    Call c(a[0]);
    if (!c.ok())
        Py_RETURN_NONE;
    const int64_t dims = THPVariable_Unpack(a[0]).dim();
    const at::Tensor &X = c.tensor(a[0], dims == 2 ? 2 : 3);
    const maxsim_dtype dt = c.dtype(X);
    if (!c.ok() || X.numel() == 0)
        Py_RETURN_NONE;
    const int d = c.size(X.size(-1));
    const at::Tensor codes = c.output(a[1], X.sizes(), at::kChar);
    const at::Tensor scale = c.output(a[2], X.sizes().slice(0, dims - 1), at::kFloat);
    if (!c.ok())
        Py_RETURN_NONE;
    const int rc = without_gil([&] { return entry.quantize(in(X), X.numel() / d, d, dt, at_ptr<int8_t>(codes), at_ptr<float>(scale), c.stream()); });
    return rc != 0 ? PyLong_FromLong(rc) : give2(a[1], codes, a[2], scale);
    END_HANDLE_TH_ERRORS
}

// (Q_i8, q_scale, D_i8, d_scale, scores)
PyObject *forward_i8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(5)
    Call c(a[0]);
    const at::Tensor &Q = c.tensor(a[0], 3), &D = c.tensor(a[2], 3);
    c.require(c.ok() && Q.scalar_type() == at::kChar && D.scalar_type() == at::kChar && D.size(2) == Q.size(2));
    if (!c.ok())
        Py_RETURN_NONE;
    const int n_q = c.size(Q.size(0)), l_q = c.size(Q.size(1)), d = c.size(Q.size(2)), l_d = c.size(D.size(1));
    const int64_t b = D.size(0);
    const at::Tensor &qs = c.tensor(a[1], {n_q, l_q}, at::kFloat), &ds = c.tensor(a[3], {b, l_d}, at::kFloat);
    const at::Tensor scores = c.output(a[4], {n_q, b}, at::kFloat);
    if (!c.ok())
        Py_RETURN_NONE;
    const int rc = without_gil([&] {
        return entry.forward_i8(at_ptr<int8_t>(Q), at_ptr<float>(qs), n_q, l_q, at_ptr<int8_t>(D), at_ptr<float>(ds), b, l_d, d, at_ptr<float>(scores), c.stream());
    });
    return rc != 0 ? PyLong_FromLong(rc) : give(a[4], scores);
    END_HANDLE_TH_ERRORS
}

// (Q_i8, q_scale, D_i8_packed, d_scale_packed, doc_offsets, scores): all rows of D_i8_packed
PyObject *forward_i8_ragged(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(6)
    Call c(a[0]);
    const at::Tensor &Q = c.tensor(a[0], 3), &D = c.tensor(a[2], 2), &off = c.tensor(a[4], 1);
    c.require(c.ok() && Q.scalar_type() == at::kChar && D.scalar_type() == at::kChar && D.size(1) == Q.size(2) && off.scalar_type() == at::kInt && off.size(0) >= 2);
    if (!c.ok())
        Py_RETURN_NONE;
    const int n_q = c.size(Q.size(0)), l_q = c.size(Q.size(1)), d = c.size(Q.size(2));
    const int64_t b = off.size(0) - 1, tokens = D.size(0);
    const at::Tensor &qs = c.tensor(a[1], {n_q, l_q}, at::kFloat), &ds = c.tensor(a[3], {tokens}, at::kFloat);
    const at::Tensor scores = c.output(a[5], {n_q, b}, at::kFloat);
    if (!c.ok())
        Py_RETURN_NONE;
    const int rc = without_gil([&] {
        return entry.forward_i8_ragged(at_ptr<int8_t>(Q), at_ptr<float>(qs), n_q, l_q, at_ptr<int8_t>(D), at_ptr<float>(ds), at_ptr<int32_t>(off), b, tokens, d, at_ptr<float>(scores),
                                       c.stream());
    });
    return rc != 0 ? PyLong_FromLong(rc) : give(a[5], scores);
    END_HANDLE_TH_ERRORS
}

// A flag as Python has it
bool flag(PyObject *o, Call &c)
{
    const int x = PyBool_Check(o) ? o == Py_True : -1;
    c.require(x >= 0);
    return x > 0;
}
float real(PyObject *o, Call &c)
{
    c.require(PyFloat_CheckExact(o));
    return c.ok() ? (float)PyFloat_AS_DOUBLE(o) : 0.0f;
}

// (X, freqs, positions, offsets, interleaved, inverse, scale, out)
PyObject *rope(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(8)
    Call c(a[0]);
    int64_t xs[2], ys[2];
    const at::Tensor &X = c.rows(a[0], xs), &freqs = c.tensor(a[1], 1);
    const maxsim_dtype dt = c.dtype(X);
    c.require(c.ok() && freqs.scalar_type() == at::kFloat && freqs.size(0) >= 1 && 2 * freqs.size(0) <= X.size(2));
    const bool neighbours = flag(a[4], c), inverse = flag(a[5], c);
    const float scale = real(a[6], c);
    if (!c.ok())
        Py_RETURN_NONE;
    const int32_t *positions = nullptr, *offsets = nullptr;
    int64_t b = 0;
    if (a[2] != Py_None) {
        const at::Tensor &p = c.tensor(a[2], {X.size(0)}, at::kInt);
        positions = c.ok() ? at_ptr<int32_t>(p) : nullptr;
    } else if (a[3] != Py_None) {
        const at::Tensor &o = c.tensor(a[3], 1);
        c.require(c.ok() && o.scalar_type() == at::kInt && o.size(0) >= 2);
        if (!c.ok())
            Py_RETURN_NONE;
        offsets = at_ptr<int32_t>(o);
        b = o.size(0) - 1;
    }
    const int heads = c.size(X.size(1)), d = c.size(X.size(2));
    const at::Tensor Y = c.output_rows(a[7], ys, X);
    if (!c.ok())
        Py_RETURN_NONE;
    const int rc = without_gil([&] {
        return entry.rope(in(X), X.size(0), heads, d, xs[0], xs[1], dt, at_ptr<float>(freqs), 2 * (int)freqs.size(0), positions, offsets, b, scale, neighbours, inverse,
                          Y.data_ptr(), ys[0], ys[1], c.stream());
    });
    return rc != 0 ? PyLong_FromLong(rc) : give(a[7], Y);
    END_HANDLE_TH_ERRORS
}

// What both directions of attention look at first
struct Attention {
    int64_t strides[16];
    const int32_t *q_off, *k_off;
    int64_t b, tq, tk;
    int hq, hkv, d;
    maxsim_dtype dt;
    float scale;

    void look(Call &c, const at::Tensor &Q, const at::Tensor &K, const at::Tensor &V, PyObject *q_offsets, PyObject *k_offsets, PyObject *scale_)
    {
        dt = c.dtype(Q);
        c.require(c.ok() && dt != MAXSIM_F32 && K.scalar_type() == Q.scalar_type() && V.scalar_type() == Q.scalar_type() && K.sizes() == V.sizes() && K.size(2) == Q.size(2) &&
                  Q.size(1) % K.size(1) == 0);
        if (!c.ok())
            return;
        tq = Q.size(0), tk = K.size(0);
        hq = c.size(Q.size(1)), hkv = c.size(K.size(1)), d = c.size(Q.size(2));
        const at::Tensor &qo = c.tensor(q_offsets, 1);
        c.require(c.ok() && qo.scalar_type() == at::kInt && qo.size(0) >= 2 && ((k_offsets != Py_None && k_offsets != q_offsets) || tq == tk));
        if (!c.ok())
            return;
        q_off = k_off = at_ptr<int32_t>(qo);
        b = qo.size(0) - 1;
        if (k_offsets != Py_None) {
            const at::Tensor &ko = c.tensor(k_offsets, {b + 1}, at::kInt);
            k_off = c.ok() ? at_ptr<int32_t>(ko) : nullptr;
        }
        scale = scale_ == Py_None ? (float)std::pow((double)d, -0.5) : real(scale_, c);
    }
};

// (Q, K, V, q_offsets, k_offsets, causal, scale, out, lse, workspace)
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(10)
    Call c(a[0]);
    Attention x;
    const at::Tensor &Q = c.rows(a[0], x.strides), &K = c.rows(a[1], x.strides + 2), &V = c.rows(a[2], x.strides + 4);
    x.look(c, Q, K, V, a[3], a[4], a[6]);
    const bool causal = flag(a[5], c);
    if (!c.ok())
        Py_RETURN_NONE;
    const at::Tensor O = c.output_rows(a[7], x.strides + 6, Q), lse = c.output(a[8], {x.tq, x.hq}, at::kFloat);
    const at::Tensor ws = c.workspace(a[9], c.ok() ? entry.attention_workspace(x.b, x.tq, x.tk, x.hq, x.hkv, x.d) : 0);
    if (!c.ok())
        Py_RETURN_NONE;
    const int rc = without_gil([&] {
        return entry.attention(in(Q), in(K), in(V), x.strides, x.q_off, x.k_off, x.b, x.tq, x.tk, x.hq, x.hkv, x.d, x.dt, causal, x.scale, O.data_ptr(), at_ptr<float>(lse),
                               ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.numel() : 0, c.stream());
    });
    return rc != 0 ? PyLong_FromLong(rc) : give2(a[7], O, a[8], lse);
    END_HANDLE_TH_ERRORS
}

// (Q, K, V, out, lse, dout, q_offsets, k_offsets, causal, scale, dQ, dK, dV, workspace)
PyObject *attention_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(14)
    Call c(a[0]);
    Attention x;
    const at::Tensor &Q = c.rows(a[0], x.strides), &K = c.rows(a[1], x.strides + 2), &V = c.rows(a[2], x.strides + 4);
    x.look(c, Q, K, V, a[6], a[7], a[9]);
    const bool causal = flag(a[8], c);
    if (!c.ok())
        Py_RETURN_NONE;
    const at::Tensor &O = c.rows(a[3], x.strides + 6, Q), &lse = c.tensor(a[4], {x.tq, x.hq}, at::kFloat), &dO = c.rows(a[5], x.strides + 8, Q);
    const at::Tensor dQ = c.output_rows(a[10], x.strides + 10, Q), dK = c.output_rows(a[11], x.strides + 12, K), dV = c.output_rows(a[12], x.strides + 14, V);
    const at::Tensor ws = c.workspace(a[13], c.ok() ? entry.attention_backward_workspace(x.b, x.tq, x.tk, x.hq, x.hkv, x.d) : 0);
    if (!c.ok())
        Py_RETURN_NONE;
    const int rc = without_gil([&] {
        return entry.attention_backward(in(Q), in(K), in(V), in(O), at_ptr<float>(lse), in(dO), x.strides, x.q_off, x.k_off, x.b, x.tq, x.tk, x.hq, x.hkv, x.d, x.dt, causal,
                                        x.scale, dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.numel() : 0, c.stream());
    });
    if (rc != 0)
        return PyLong_FromLong(rc);
    PyObject *two = give2(a[10], dQ, a[11], dK), *third = two ? give(a[12], dV) : nullptr;
    PyObject *r = third ? PyTuple_Pack(3, PyTuple_GET_ITEM(two, 0), PyTuple_GET_ITEM(two, 1), third) : nullptr;
    Py_XDECREF(two);
    Py_XDECREF(third);
    return r;
    END_HANDLE_TH_ERRORS
}

// (grads, max_norm, out, norm, workspace): grads and out (or None) lists
PyObject *clip_grad_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    ARGUMENTS(5)
    if (!PyList_CheckExact(a[0]) || !(a[2] == Py_None || PyList_CheckExact(a[2])))
        Py_RETURN_NONE;
    const Py_ssize_t count = PyList_GET_SIZE(a[0]);
    if (count < 1 || count > INT_MAX || (a[2] != Py_None && PyList_GET_SIZE(a[2]) != count))
        Py_RETURN_NONE;
    Call c(PyList_GET_ITEM(a[0], 0));
    std::vector<const void *> g(count);
    std::vector<void *> out(count);
    std::vector<int64_t> numel(count);
    std::vector<int32_t> dtype(count);
    for (Py_ssize_t i = 0; i < count; ++i) {
        const at::Tensor &t = c.tensor(PyList_GET_ITEM(a[0], i));
        dtype[i] = c.dtype(t);
        if (!c.ok())
            Py_RETURN_NONE;
        g[i] = out[i] = t.data_ptr();
        numel[i] = t.numel();
        if (a[2] != Py_None) {
            const at::Tensor &o = c.tensor(PyList_GET_ITEM(a[2], i));
            c.require(c.ok() && o.scalar_type() == t.scalar_type() && o.sizes() == t.sizes());
            if (!c.ok())
                Py_RETURN_NONE;
            out[i] = o.data_ptr();
        }
    }
    const float max_norm = real(a[1], c);
    const at::Tensor norm = c.output(a[3], {1}, at::kFloat), ws = c.workspace(a[4], c.ok() ? entry.clip_workspace((int)count) : 0);
    if (!c.ok())
        Py_RETURN_NONE;
    const int rc = without_gil([&] {
        return entry.clip_grad_norm(g.data(), out.data(), numel.data(), dtype.data(), (int)count, max_norm, at_ptr<float>(norm), ws.data_ptr(), ws.numel(), c.stream());
    });
    return rc != 0 ? PyLong_FromLong(rc) : give(a[3], norm);
    END_HANDLE_TH_ERRORS
}

// The addresses of the entry points in the library that binding.py has loaded, in the order of Entries
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    ARGUMENTS(15)
    void *p[15];
    for (int i = 0; i < 15; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred())
            return nullptr;
    }
    int i = 0;
    entry.forward = reinterpret_cast<decltype(entry.forward)>(p[i++]);
    entry.forward_ragged = reinterpret_cast<decltype(entry.forward_ragged)>(p[i++]);
    entry.backward = reinterpret_cast<decltype(entry.backward)>(p[i++]);
    entry.backward_ragged = reinterpret_cast<decltype(entry.backward_ragged)>(p[i++]);
    entry.ce_grad = reinterpret_cast<decltype(entry.ce_grad)>(p[i++]);
    entry.quantize = reinterpret_cast<decltype(entry.quantize)>(p[i++]);
    entry.forward_i8 = reinterpret_cast<decltype(entry.forward_i8)>(p[i++]);
    entry.forward_i8_ragged = reinterpret_cast<decltype(entry.forward_i8_ragged)>(p[i++]);
    entry.rope = reinterpret_cast<decltype(entry.rope)>(p[i++]);
    entry.attention_workspace = reinterpret_cast<decltype(entry.attention_workspace)>(p[i++]);
    entry.attention = reinterpret_cast<decltype(entry.attention)>(p[i++]);
    entry.attention_backward_workspace = reinterpret_cast<decltype(entry.attention_backward_workspace)>(p[i++]);
    entry.attention_backward = reinterpret_cast<decltype(entry.attention_backward)>(p[i++]);
    entry.clip_workspace = reinterpret_cast<decltype(entry.clip_workspace)>(p[i++]);
    entry.clip_grad_norm = reinterpret_cast<decltype(entry.clip_grad_norm)>(p[i++]);
    Py_RETURN_NONE;
}

#define METHOD(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(NAME)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind),     METHOD(forward),    METHOD(forward_ragged),    METHOD(backward), METHOD(backward_ragged), METHOD(ce_grad),
                         METHOD(quantize), METHOD(forward_i8), METHOD(forward_i8_ragged), METHOD(rope), METHOD(attention), METHOD(attention_backward),
                         METHOD(clip_grad_norm), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__marshal()
{
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "BUILT_FOR", MARSHAL_ABI) < 0) { // (binding.py looks at it before anything else)
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
