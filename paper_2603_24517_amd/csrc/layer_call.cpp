// attention_backward(), qk_norm_rope() and qk_norm_rope_backward() of the package as one native call each: checks, results and workspace allocated by
// torch, the C entry on torch's current stream.
//
// Host code only.  In Python the same steps take 20 to 30 us a call, and the kernel of one token of 64 sequences 4.  Each function
// returns its results; a status code of the C entry if it is not 0; or None for whatever it does not take (tensors of another type than torch.Tensor
// itself, torch function modes, a C++ exception of torch's, arguments that are refused): the caller's general form takes or refuses it.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <vector>

#include "../../include/attn_layer.h"

namespace {

decltype(&attn_bwd) bwd = nullptr;
decltype(&attn_bwd_workspace) bwd_workspace = nullptr;
decltype(&attn_qk_norm_rope) rope_fwd = nullptr;
decltype(&attn_qk_norm_rope_bwd) rope_bwd = nullptr;
decltype(&attn_qk_norm_rope_bwd_workspace) rope_workspace = nullptr;

struct General {};      // thrown for what the general form has to take

// The tensor behind an argument; undefined for None.
at::Tensor tensor(PyObject *x)
{
    if (x == Py_None) return at::Tensor();
    if (!THPVariable_CheckExact(x)) throw General();
    return THPVariable_Unpack(x);
}
double number(PyObject *x)
{
    const double v = PyFloat_AsDouble(x);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw General();
    }
    return v;
}
bool truth(PyObject *x)
{
    const int v = PyObject_IsTrue(x);
    if (v < 0) throw python_error();
    return v != 0;
}
void require(bool ok)
{
    if (!ok) throw General();
}
int size(int64_t n)
{
    require(n <= INT_MAX);
    return (int)n;
}
bool on(const at::Tensor &t, const at::Tensor &q) { return !t.defined() || (t.is_cuda() && t.device() == q.device()); }
void *ptr(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

// A fresh contiguous tensor on q's device.  No dispatch mode wants to see it: past torch's dispatcher, which takes longer than the allocation.
at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor &q)
{
    if (c10::impl::TorchDispatchModeTLS::any_modes_set()) return at::empty(sizes, q.options().dtype(type));
    return at::Tensor(at::detail::empty_cuda(sizes, type, q.device(), std::nullopt));
}

// The interpreter's lock given back, and taken again however the block ends.
struct Unlocked {
    PyThreadState *const state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// f(stream, workspace), without the interpreter's lock, with q's device current.  The workspace, if any, comes from torch's allocator, as a tensor's
// memory would: it belongs to the stream, and goes back to it when the call has been enqueued.
template <class F>
int launch(const at::Tensor &q, long long bytes, F &&f)
{
    const auto index = q.get_device();
    int rc;
    auto go = [&]() {
        void *stream = (void *)c10::hip::getCurrentHIPStream(index).stream();
        c10::DataPtr workspace;
        if (bytes > 0) workspace = c10::hip::HIPCachingAllocator::get()->allocate((size_t)bytes);
        const Unlocked unlocked;
        rc = f(stream, workspace.get());
    };
    if (index == c10::hip::current_device()) {
        go();
    } else {
        const c10::DeviceGuard guard(q.device());
        go();
    }
    return rc;
}

PyObject *tuple(const std::vector<at::Tensor> &all)
{
    PyObject *t = PyTuple_New((Py_ssize_t)all.size());
    for (size_t i = 0; t && i < all.size(); ++i) {
        PyObject *x;
        if (all[i].defined()) {
            x = THPVariable_Wrap(all[i]);
        } else {
            x = Py_None;
            Py_INCREF(x);
        }
        if (!x) {
            Py_DECREF(t);
            return nullptr;
        }
        PyTuple_SET_ITEM(t, (Py_ssize_t)i, x);
    }
    return t;
}

template <class F>
PyObject *guarded(Py_ssize_t given, Py_ssize_t wanted, F &&f)
{
    if (given != wanted) {
        PyErr_SetString(PyExc_ValueError, "wrong number of arguments");
        return nullptr;
    }
    try {
        if (bwd != nullptr && !at::impl::torch_function_mode_enabled()) return f();
    } catch (const General &) {
    } catch (python_error &e) {     // of a dispatch mode, for instance: the exception itself
        e.restore();
    } catch (const std::exception &) {
    }
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;         // (the general form meets it again, and raises)
}

// backward(do, q, k, v, o, lse, causal, scale, dlse)
PyObject *backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(n, 9, [&]() -> PyObject * {
        const at::Tensor dout = tensor(args[0]), q = tensor(args[1]), k = tensor(args[2]), v = tensor(args[3]), o = tensor(args[4]),
                         lse = tensor(args[5]), dlse = tensor(args[8]);
        for (const at::Tensor *t : {&dout, &q, &k, &v, &o})
            require(t->defined() && t->is_cuda() && t->scalar_type() == at::kBFloat16 && t->dim() == 4 && t->is_contiguous() && t->device() == q.device());
        const int B = size(q.size(0)), Sq = size(q.size(1)), Hq = size(q.size(2)), D = size(q.size(3)), Skv = size(k.size(1)), Hkv = size(k.size(2));
        require(k.size(0) == B && k.size(3) == D && k.sizes() == v.sizes() && dout.sizes() == q.sizes() && o.sizes() == q.sizes());
        require(lse.defined());
        for (const at::Tensor *t : {&lse, &dlse})
            require(!t->defined() || (on(*t, q) && t->scalar_type() == at::kFloat && t->dim() == 3 && t->is_contiguous() && t->size(0) == B &&
                                      t->size(1) == Hq && t->size(2) == Sq));
        const bool causal = truth(args[6]);
        require(D > 0);
        const float scale = (float)(args[7] == Py_None ? std::pow((double)D, -0.5) : number(args[7]));
        const long long bytes = bwd_workspace(B, Hq, Hkv, Sq, Skv, D, causal);
        if (bytes < 0) return PyLong_FromLongLong(bytes);
        const at::Tensor dq = fresh(q.sizes(), at::kBFloat16, q), dk = fresh(k.sizes(), at::kBFloat16, q), dv = fresh(v.sizes(), at::kBFloat16, q);
        // (addresses with the lock held: torch throws for a tensor without storage, a functorch wrapper say)
        void *const in[] = {ptr(dout), ptr(q), ptr(k), ptr(v), ptr(o)}, *const out[] = {ptr(dq), ptr(dk), ptr(dv)};
        const float *const figures[] = {(const float *)ptr(dlse), (const float *)ptr(lse)};
        const int rc = launch(q, bytes, [&](void *stream, void *workspace) {
            return bwd(in[0], figures[0], in[1], in[2], in[3], in[4], figures[1], out[0], out[1], out[2], workspace, (size_t)bytes, B, Hq, Hkv, Sq, Skv, D,
                       causal, scale, stream);
        });
        return rc != 0 ? PyLong_FromLong(rc) : tuple({dq, dk, dv});
    });
}

// ------------------------------------------------------------------------------------------- norm and rotation
attn_heads heads(const at::Tensor &t)
{
    if (!t.defined()) return {nullptr, 0, 0, 0};
    return {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
}
void check_heads(const at::Tensor &t, const at::Tensor &like)
{
    require(t.defined() && on(t, like) && t.scalar_type() == at::kBFloat16 && t.dim() == 4 && t.sizes() == like.sizes() && (t.size(3) <= 1 || t.stride(3) == 1));
}
// Two elements of an output must not share memory.
void check_output(const at::Tensor &t)
{
    std::vector<std::pair<int64_t, int64_t>> dims;      // stride, size
    for (int64_t i = 0; i < t.dim(); ++i) dims.emplace_back(t.stride(i), t.size(i));
    std::stable_sort(dims.begin(), dims.end(), [](const auto &a, const auto &b) { return a.first < b.first; });
    int64_t need = 1;
    for (const auto &[stride, n] : dims) {
        if (n <= 1) continue;
        require(stride >= need);
        need += stride * (n - 1);
    }
}
// (q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved) from args[0] on
struct Rope {
    at::Tensor q, k, qw, kw, cos, sin, positions;
    attn_rope r;
    explicit Rope(PyObject *const *args)
        : q(tensor(args[0])), k(tensor(args[1])), qw(tensor(args[2])), kw(tensor(args[3])), cos(tensor(args[4])), sin(tensor(args[5])), positions(tensor(args[6]))
    {
        require(q.defined() && q.is_cuda() && q.dim() == 4 && k.defined() && k.dim() == 4 && cos.defined() && sin.defined());
        check_heads(q, q);
        check_heads(k, k);
        require(on(k, q) && k.size(0) == q.size(0) && k.size(1) == q.size(1) && k.size(3) == q.size(3) && qw.defined() == kw.defined());
        r = {};
        r.B = size(q.size(0));
        r.S = size(q.size(1));
        r.Hq = size(q.size(2));
        r.Hkv = size(k.size(2));
        r.D = size(q.size(3));
        if (qw.defined()) {
            const auto type = qw.scalar_type();
            require(type == at::kBFloat16 || type == at::kFloat);
            for (const at::Tensor *w : {&qw, &kw}) require(on(*w, q) && w->scalar_type() == type && w->is_contiguous() && w->dim() == 1 && w->size(0) == r.D);
            r.weight_type = type == at::kFloat ? ATTN_FP32 : ATTN_BF16;
        }
        for (const at::Tensor *t : {&cos, &sin}) require(on(*t, q) && t->scalar_type() == at::kFloat && t->is_contiguous() && t->dim() == 2 && t->sizes() == cos.sizes());
        if (positions.defined()) {
            const auto type = positions.scalar_type();
            require((type == at::kInt || type == at::kLong) && on(positions, q) && positions.is_contiguous() && positions.dim() == 2 && positions.size(0) == r.B &&
                    positions.size(1) == r.S);
            r.position_type = type == at::kLong ? ATTN_INT64 : ATTN_INT32;
        }
        require(cos.size(1) <= INT_MAX / 2);
        r.q_weight = ptr(qw);
        r.k_weight = ptr(kw);
        r.cos = (const float *)ptr(cos);
        r.sin = (const float *)ptr(sin);
        r.places = cos.size(0);
        r.rotated = 2 * (int)cos.size(1);
        r.positions = ptr(positions);
        r.eps = (float)number(args[7]);
        r.pairing = truth(args[8]) ? ATTN_ROPE_ADJACENT : ATTN_ROPE_HALVES;
    }
};
// The results: fresh contiguous tensors, or those of `out`.
std::vector<at::Tensor> results(PyObject *out, const std::vector<at::Tensor> &like)
{
    std::vector<at::Tensor> all;
    if (out == Py_None) {
        for (const at::Tensor &t : like) all.push_back(fresh(t.sizes(), t.scalar_type(), t));
        return all;
    }
    require(PyTuple_CheckExact(out) && PyTuple_GET_SIZE(out) == (Py_ssize_t)like.size());
    for (size_t i = 0; i < like.size(); ++i) {
        all.push_back(tensor(PyTuple_GET_ITEM(out, (Py_ssize_t)i)));
        check_heads(all.back(), like[i]);
        check_output(all.back());
        for (size_t j = 0; j < i; ++j) require(all[j].data_ptr() != all[i].data_ptr());
    }
    return all;
}

// The caller's tensors have been written to: autograd counts that, so that a graph that saved one does not take the new values for the old.
void written(PyObject *out, const std::vector<at::Tensor> &all)
{
    if (out == Py_None) return;
    for (const at::Tensor &t : all)
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, v, out)
PyObject *rope(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(n, 11, [&]() -> PyObject * {
        const Rope x(args);
        std::vector<at::Tensor> in = {x.q, x.k};
        if (const at::Tensor v = tensor(args[9]); v.defined()) {
            check_heads(v, x.k);
            in.push_back(v);
        }
        const std::vector<at::Tensor> out = results(args[10], in);
        attn_heads h[6] = {};
        for (size_t i = 0; i < in.size(); ++i) {
            h[i] = heads(in[i]);
            h[3 + i] = heads(out[i]);
        }
        const int rc = launch(x.q, 0, [&](void *stream, void *) { return rope_fwd(&x.r, h, h + 1, h + 2, h + 3, h + 4, h + 5, stream); });
        if (rc != 0) return PyLong_FromLong(rc);
        written(args[10], out);
        return tuple(out);
    });
}

// rope_backward(dq, dk, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, dv, out)
PyObject *rope_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(n, 13, [&]() -> PyObject * {
        const Rope x(args + 2);
        std::vector<at::Tensor> in = {tensor(args[0]), tensor(args[1])};
        check_heads(in[0], x.q);
        check_heads(in[1], x.k);
        if (const at::Tensor dv = tensor(args[11]); dv.defined()) {
            check_heads(dv, x.k);
            in.push_back(dv);
        }
        std::vector<at::Tensor> out = results(args[12], in);
        at::Tensor dw[2];
        long long bytes = 0;
        if (x.qw.defined()) {
            bytes = rope_workspace(&x.r);
            if (bytes < 0) return PyLong_FromLongLong(bytes);
            for (at::Tensor &w : dw) w = fresh({x.r.D}, at::kFloat, x.q);
        }
        attn_heads h[8] = {};
        for (size_t i = 0; i < in.size(); ++i) {
            h[i] = heads(in[i]);
            h[5 + i] = heads(out[i]);
        }
        h[3] = heads(x.q);
        h[4] = heads(x.k);
        float *const weights[] = {(float *)ptr(dw[0]), (float *)ptr(dw[1])};
        const int rc = launch(x.q, bytes, [&](void *stream, void *workspace) {
            return rope_bwd(&x.r, h, h + 1, h + 2, h + 3, h + 4, h + 5, h + 6, h + 7, weights[0], weights[1], workspace, (size_t)bytes, stream);
        });
        if (rc != 0) return PyLong_FromLong(rc);
        written(args[12], out);
        out.push_back(dw[0]);
        out.push_back(dw[1]);
        return tuple(out);
    });
}

// bind(addresses of the five C entries)
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    void *p[5];
    if (n != 5) {
        PyErr_SetString(PyExc_ValueError, "bind(five addresses)");
        return nullptr;
    }
    for (int i = 0; i < 5; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (p[i] == nullptr && PyErr_Occurred()) return nullptr;
    }
    bwd = (decltype(bwd))p[0];
    bwd_workspace = (decltype(bwd_workspace))p[1];
    rope_fwd = (decltype(rope_fwd))p[2];
    rope_bwd = (decltype(rope_bwd))p[3];
    rope_workspace = (decltype(rope_workspace))p[4];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"backward", (PyCFunction)(void (*)(void))backward, METH_FASTCALL, "attention_backward() on tensors"},
                         {"rope", (PyCFunction)(void (*)(void))rope, METH_FASTCALL, "qk_norm_rope() on tensors"},
                         {"rope_backward", (PyCFunction)(void (*)(void))rope_backward, METH_FASTCALL, "qk_norm_rope_backward() on tensors"},
                         {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, "sets the C entries"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_layer_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layer_call() { return PyModule_Create(&module); }
