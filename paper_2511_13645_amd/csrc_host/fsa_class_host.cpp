// Host path of the class losses: argument checks, allocations, the call into the C ABI and the differentiable loss's
// node in autograd's graph, without the interpreter in between.  A loss over a few labels is bound by its host side.
//
// As fsa_host.cpp, a module by itself: its functions take the arguments that nearly every call has and return None for
// anything else, which the Python code then takes; a failed library call returns its status, an int.
#include "../../include/fsa.h"

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

namespace {

using at::Tensor;

PyObject* raw_stream = nullptr;                            // device index -> current stream's handle

// Addresses of the C ABI's entry points, set by bind(), with the types that fsa.h declares them with.
#define FSA_HOST_ENTRIES(X) X(fsa_class_fwd_workspace_bytes) X(fsa_class_bwd_workspace_bytes) X(fsa_xent_fwd) X(fsa_xent_bwd) \
                            X(fsa_distill_fwd) X(fsa_distill_bwd)
struct {
#define FSA_HOST_MEMBER(name) decltype(&::name) name;
    FSA_HOST_ENTRIES(FSA_HOST_MEMBER)
#undef FSA_HOST_MEMBER
} abi;

// The tensor behind an argument, or nullptr for anything but a plain tensor or parameter.
const Tensor* tensor_of(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

bool plain(const Tensor* t, int64_t dim) { return t && t->is_cuda() && t->dim() == dim && t->is_contiguous(); }
bool plain(const Tensor* t, int64_t dim, at::ScalarType type) { return plain(t, dim) && t->scalar_type() == type; }
bool together(const Tensor& a, const Tensor& b) { return a.get_device() == b.get_device(); }

int float_code(const Tensor& t) {                      // fsa.h's dtype code, -1 for none
    switch (t.scalar_type()) {
        case at::kFloat: return FSA_F32;
        case at::kBFloat16: return FSA_BF16;
        case at::kHalf: return FSA_F16;
        default: return -1;
    }
}

bool observed() { return at::impl::torch_function_mode_enabled() || c10::impl::dispatch_mode_enabled(); }

// Current stream of t's device; false with an error set.
bool stream_of(const Tensor& t, void** stream) {
    PyObject* index = PyLong_FromLong(t.get_device());
    if (!index) return false;
    PyObject* h = PyObject_CallOneArg(raw_stream, index);
    Py_DECREF(index);
    if (!h) return false;
    *stream = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    return !PyErr_Occurred();
}

PyObject* wrap(const Tensor& t) {
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}

template <size_t N> PyObject* tuple_of(const Tensor (&t)[N]) {
    PyObject* r = PyTuple_New(N);
    if (!r) return nullptr;
    for (size_t i = 0; i < N; ++i) {
        PyObject* o = wrap(t[i]);
        if (!o) { Py_DECREF(r); return nullptr; }
        PyTuple_SET_ITEM(r, i, o);
    }
    return r;
}

template <typename T = void> T* data(const Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }

// Allocations (which may wait for the driver) and the C call, with other threads free to run meanwhile.
template <typename F> int without_gil(F f) {
    struct Released {
        PyThreadState* state = PyEval_SaveThread();
        ~Released() { PyEval_RestoreThread(state); }
    } released;
    return f();
}

// What no check here foresees is the Python code's to report.
template <typename F> PyObject* or_none(F f) {
    try {
        return f();
    } catch (const std::exception&) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

struct ClassCall {
    Tensor h, w, ids, logits;                              // logits undefined: cross entropy
    int64_t h_stride, w_stride, T, V, D;
    int code, teacher_code = FSA_F32;
    int32_t K = 1;
    float temperature, scale;
    void* stream;
};

// Rows of a matrix are contiguous and do not overlap; how far they lie apart, 0 if they do not.
int64_t rows_of(const Tensor* t) {
    if (!t || !t->is_cuda() || t->dim() != 2 || t->layout() != at::kStrided) return 0;
    const int64_t D = t->size(1);
    if (D < 1 || (t->stride(1) != 1 && D > 1) || (t->size(0) > 1 && t->stride(0) < D)) return 0;
    return t->size(0) > 1 ? t->stride(0) : D;
}

// (h, w, ids, logits | None, temperature, scale, ...): whether the call is as plain as most; false with an error set, or
// without one where the Python code is to take it.
bool class_call(ClassCall& c, PyObject* const* a) {
    const Tensor *h = tensor_of(a[0]), *w = tensor_of(a[1]), *ids = tensor_of(a[2]);
    const bool distill = a[3] != Py_None;
    const Tensor* logits = distill ? tensor_of(a[3]) : nullptr;
    if (!PyFloat_CheckExact(a[4]) || !PyFloat_CheckExact(a[5]) || observed()) return false;
    c.h_stride = rows_of(h);
    c.w_stride = rows_of(w);
    if (!c.h_stride || !c.w_stride || (c.code = float_code(*h)) < 0 || h->scalar_type() != w->scalar_type()) return false;
    c.T = h->size(0); c.D = h->size(1); c.V = w->size(0);
    if (w->size(1) != c.D || !together(*h, *w) || !plain(ids, distill ? 2 : 1, at::kInt) || ids->size(0) != c.T || !together(*h, *ids)) return false;
    if (distill) {
        if (!plain(logits, 2) || (c.teacher_code = float_code(*logits)) < 0 || logits->sizes() != ids->sizes() || !together(*h, *logits)) return false;
        if (ids->size(1) < 1 || ids->size(1) > FSA_KMAX) return false;
        c.K = (int32_t)ids->size(1);
        c.logits = *logits;
    }
    c.h = *h; c.w = *w; c.ids = *ids;
    c.temperature = (float)PyFloat_AS_DOUBLE(a[4]);
    c.scale = (float)PyFloat_AS_DOUBLE(a[5]);
    return stream_of(*h, &c.stream);
}

// (loss, lse, row_grad or nothing) of a call, or a status.
int class_forward(const ClassCall& c, bool emit_row_grad, Tensor (&o)[3]) {
    const auto f = at::TensorOptions().dtype(at::kFloat).device(c.h.device());
    const int64_t need = abi.fsa_class_fwd_workspace_bytes(c.T, c.V, c.D, c.code, c.K, emit_row_grad);
    o[0] = at::empty({c.T}, f);
    o[1] = at::empty({c.T}, f);
    if (emit_row_grad) o[2] = at::empty({c.T, c.D}, f);
    const Tensor ws = at::empty({need}, f.dtype(at::kByte));       // (may go once the call is queued: same stream)
    if (!c.logits.defined())
        return abi.fsa_xent_fwd(data(c.h), c.h_stride, data(c.w), c.w_stride, c.code, c.T, c.V, c.D, c.scale, data<int32_t>(c.ids),
                                data<float>(o[0]), data<float>(o[1]), data<float>(o[2]), data(ws), need, c.stream);
    return abi.fsa_distill_fwd(data(c.h), c.h_stride, data(c.w), c.w_stride, c.code, c.T, c.V, c.D, c.scale, c.temperature,
                               data<int32_t>(c.ids), data(c.logits), c.teacher_code, c.K,
                               data<float>(o[0]), data<float>(o[1]), data<float>(o[2]), data(ws), need, c.stream);
}

struct Refused : std::exception { int status; explicit Refused(int s) : status(s) {} };

// The differentiable loss.  Its backward runs on the stream of its forward, which is the one that autograd then makes current.
struct ClassLoss : torch::autograd::Function<ClassLoss> {
    static Tensor forward(torch::autograd::AutogradContext* ctx, const Tensor& h, const Tensor& w, const ClassCall& c, bool emit_row_grad) {
        Tensor o[3];
        if (const int rc = class_forward(c, emit_row_grad, o)) throw Refused(rc);
        ctx->save_for_backward({h, w, c.ids, c.logits, o[1], o[2]});
        auto& d = ctx->saved_data;
        d["temperature"] = (double)c.temperature;
        d["scale"] = (double)c.scale;
        d["stream"] = (int64_t)reinterpret_cast<intptr_t>(c.stream);
        return o[0];
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        const auto v = ctx->get_saved_variables();
        const Tensor &h = v[0], &w = v[1], &ids = v[2], &logits = v[3], &lse = v[4], &row_grad = v[5];
        const bool again = c10::GradMode::is_enabled() && grads[0].requires_grad();
        torch::autograd::variable_list out(4);
        {
            at::AutoGradMode off(false);
            const Tensor g = grads[0].contiguous();
            const int64_t T = h.size(0), D = h.size(1), V = w.size(0), hs = rows_of(&h), wst = rows_of(&w);
            const bool want_h = ctx->needs_input_grad(0), want_w = ctx->needs_input_grad(1);
            const int code = float_code(h);
            const int32_t K = logits.defined() ? (int32_t)ids.size(1) : 1;
            const auto rows = at::TensorOptions().dtype(h.dtype()).device(h.device());
            if (want_h) out[0] = at::empty({T, D}, rows);
            if (want_w) out[1] = at::empty({V, D}, rows);
            const int64_t need = abi.fsa_class_bwd_workspace_bytes(T, V, D, code, K, want_h && !row_grad.defined(), want_w);
            const Tensor ws = at::empty({need}, rows.dtype(at::kByte));
            const float temperature = (float)ctx->saved_data["temperature"].toDouble(), scale = (float)ctx->saved_data["scale"].toDouble();
            void* stream = reinterpret_cast<void*>((intptr_t)ctx->saved_data["stream"].toInt());
            const int rc = !logits.defined()
                ? abi.fsa_xent_bwd(data<float>(g), data(h), hs, data(w), wst, code, T, V, D, scale, data<int32_t>(ids),
                                   data<float>(lse), data<float>(row_grad), data(out[0]), data(out[1]), data(ws), need, stream)
                : abi.fsa_distill_bwd(data<float>(g), data(h), hs, data(w), wst, code, T, V, D, scale, temperature, data<int32_t>(ids),
                                      data(logits), float_code(logits), K, data<float>(lse), data<float>(row_grad), data(out[0]), data(out[1]),
                                      data(ws), need, stream);
            TORCH_CHECK(rc == FSA_OK, "the backward of a class loss was refused (status ", rc, ")");
        }
        if (again) {                                       // as torch's once_differentiable: a second derivative raises
            auto node = std::make_shared<torch::autograd::DelayedError>("a class loss is differentiable once", 2);
            auto err = (*node)({out[0], out[1]});
            out[0] = err[0];
            out[1] = err[1];
        }
        return out;
    }
};

// (h, w, ids, logits | None, temperature, scale, emit_row_grad) -> (loss, lse, row_grad | None)
PyObject* class_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7 || !PyBool_Check(a[6])) Py_RETURN_NONE;
    return or_none([&]() -> PyObject* {
        ClassCall c;
        if (!class_call(c, a)) { if (PyErr_Occurred()) return nullptr; Py_RETURN_NONE; }
        Tensor o[3];
        const int rc = without_gil([&] {
            at::AutoGradMode off(false);
            return class_forward(c, a[6] == Py_True, o);
        });
        return rc != FSA_OK ? PyLong_FromLong(rc) : tuple_of(o);
    });
}

// (h, w, ids, logits | None, temperature, scale) -> loss with its gradient
PyObject* class_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 6) Py_RETURN_NONE;
    return or_none([&]() -> PyObject* {
        ClassCall c;
        if (!class_call(c, a)) { if (PyErr_Occurred()) return nullptr; Py_RETURN_NONE; }
        Tensor loss;
        const int rc = without_gil([&] {
            try {
                // (with a gradient of w alone as well: the log-sum-exp that its backward takes is then as exact as both need it)
                loss = ClassLoss::apply(c.h, c.w, c, c10::GradMode::is_enabled() && (c.h.requires_grad() || c.w.requires_grad()));
                return (int)FSA_OK;
            } catch (const Refused& r) {
                return r.status;
            }
        });
        return rc != FSA_OK ? PyLong_FromLong(rc) : wrap(loss);
    });
}

// (raw_stream, {entry point: address})
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 2 || !PyDict_Check(a[1])) { PyErr_SetString(PyExc_TypeError, "a stream function and the entry points' addresses"); return nullptr; }
#define FSA_HOST_BIND(name)                                                                                             \
    {                                                                                                                   \
        PyObject* at = PyDict_GetItemString(a[1], #name);                                                               \
        if (!at) { PyErr_SetString(PyExc_TypeError, "no address for " #name); return nullptr; }                         \
        abi.name = reinterpret_cast<decltype(abi.name)>(PyLong_AsVoidPtr(at));                                          \
        if (PyErr_Occurred()) return nullptr;                                                                           \
    }
    FSA_HOST_ENTRIES(FSA_HOST_BIND)
#undef FSA_HOST_BIND
    Py_INCREF(a[0]);
    Py_XDECREF(raw_stream);
    raw_stream = a[0];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind)), METH_FASTCALL, nullptr},
    {"class_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(class_fwd)), METH_FASTCALL, nullptr},
    {"class_loss", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(class_loss)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fsa_class_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fsa_class_host() { return PyModule_Create(&module); }
