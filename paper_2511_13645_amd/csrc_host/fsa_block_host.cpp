// Host path of the residual norm and the gated feed-forward block: argument checks, allocations, the calls into the C ABI and
// their nodes in autograd's graph, without the interpreter in between.  A block of a small batch is bound by its host side.
//
// As fsa_class_host.cpp, a module by itself: its functions take the arguments that nearly every call has and return None for
// anything else, which the Python code then takes; a failed library call returns its status, an int.
#include "../../include/fsa.h"

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/accumulate_grad.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <optional>

namespace {

using at::Tensor;

PyObject* raw_stream = nullptr;                            // device index -> current stream's handle

// Addresses of the C ABI's entry points, set by bind(), with the types that fsa.h declares them with.
#define FSA_HOST_ENTRIES(X) X(fsa_norm_fwd) X(fsa_norm_bwd) X(fsa_norm_bwd_workspace_bytes) X(fsa_gated_fwd) X(fsa_gated_bwd) \
                            X(fsa_gated_fwd_workspace_bytes) X(fsa_gated_bwd_workspace_bytes) X(fsa_gated_keep_pays) X(fsa_gated_kept_bytes)
struct {
#define FSA_HOST_MEMBER(name) decltype(&::name) name;
    FSA_HOST_ENTRIES(FSA_HOST_MEMBER)
#undef FSA_HOST_MEMBER
} abi;

// The tensor behind an argument, or nullptr for anything but a plain tensor or parameter.
const Tensor* tensor_of(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

bool plain(const Tensor* t, int64_t dim) { return t && t->is_cuda() && t->dim() == dim && t->is_contiguous(); }
bool together(const Tensor& a, const Tensor& b) { return a.get_device() == b.get_device(); }

int float_code(const Tensor& t) {                      // fsa.h's dtype code, -1 for none
    switch (t.scalar_type()) {
        case at::kFloat: return FSA_F32;
        case at::kBFloat16: return FSA_BF16;
        case at::kHalf: return FSA_F16;
        default: return -1;
    }
}

int current_device() { return c10::impl::getDeviceGuardImpl(at::kCUDA)->getDevice().index(); }

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

// Rows of a matrix are contiguous and do not overlap; how far they lie apart, 0 if they do not.
int64_t rows_of(const Tensor* t) {
    if (!t || !t->is_cuda() || t->dim() != 2 || t->layout() != at::kStrided) return 0;
    const int64_t D = t->size(1);
    if (D < 1 || (t->stride(1) != 1 && D > 1) || (t->size(0) > 1 && t->stride(0) < D)) return 0;
    return t->size(0) > 1 ? t->stride(0) : D;
}
// The stream is the current one of the tensors' device, which has to be the current device: allocations and launches belong to it.
bool here(const Tensor& t, void** stream) { return !observed() && t.get_device() == current_device() && stream_of(t, stream); }

struct Refused : std::exception { int status; explicit Refused(int s) : status(s) {} };

// A second derivative raises, as with torch's once_differentiable.
void once(const char* what, bool again, torch::autograd::variable_list& out) {
    if (!again) return;
    for (Tensor& t : out) if (t.defined()) t.requires_grad_(true);         // a node is put behind none but these
    auto node = std::make_shared<torch::autograd::DelayedError>(std::string(what) + " is differentiable once", (int)out.size());
    out = (*node)(std::move(out));
}
// The leaf that a gradient goes to: straight, or through nodes that have one input alone, as casts and views do; nullptr for another way.
torch::autograd::Node* leaf_of(torch::autograd::Node* node) {
    for (int i = 0; node && i < 8; ++i) {
        if (dynamic_cast<torch::autograd::AccumulateGrad*>(node)) return node;
        torch::autograd::Node* next = nullptr;
        for (const auto& e : node->next_edges()) {
            if (!e.function) continue;
            if (next) return nullptr;
            next = e.function.get();
        }
        node = next;
    }
    return nullptr;
}
// A backward that is captured into a graph while a leaf that its gradient goes to has an eager graph alive: autograd would have the
// leaf's stream wait for the captured one, which ends the capture and the process.  Raises instead.
void refuse_capture(const char* what) {
    const auto node = torch::autograd::get_current_node();
    if (!node) return;
    const auto own = node->stream();
    bool other = false;
    for (const auto& e : node->next_edges())
        if (torch::autograd::Node* leaf = leaf_of(e.function.get())) {
            const auto theirs = leaf->stream();
            other = other || (own && theirs && *own != *theirs);
        }
    if (!other) return;
    const PyGILState_STATE gil = PyGILState_Ensure();
    PyObject *torch_c = PyImport_ImportModule("torch._C"), *r = torch_c ? PyObject_CallMethod(torch_c, "_cuda_isCurrentStreamCapturing", nullptr) : nullptr;
    const bool capturing = r == Py_True;
    Py_XDECREF(r);
    Py_XDECREF(torch_c);
    PyErr_Clear();
    PyGILState_Release(gil);
    TORCH_CHECK(!capturing, "the backward of ", what, " cannot be captured while an eager graph of the same parameters is alive "
                "(one made on another stream): drop it, or what holds it, first");
}
// (what): the same for a backward that the Python code makes.
PyObject* refuse_captured(PyObject*, PyObject* what) {
    const char* name = PyUnicode_AsUTF8(what);
    if (!name) return nullptr;
    try {
        refuse_capture(name);
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    Py_RETURN_NONE;
}
bool differentiated(const torch::autograd::variable_list& grads) {
    if (!c10::GradMode::is_enabled()) return false;
    for (const Tensor& g : grads) if (g.defined() && g.requires_grad()) return true;
    return false;
}

// ---------------------------------------------------------------------------------------------------------------
// norm
// ---------------------------------------------------------------------------------------------------------------
struct NormCall {
    Tensor x, weight, residual;                            // residual undefined: none
    int64_t x_stride, residual_stride = 0;
    int code, weight_code;
    float eps;
    void* stream;
};

// (x, weight, residual | None, eps): whether the call is as plain as most; false with an error set, or without one where the Python
// code is to take it.
bool norm_call(NormCall& c, PyObject* const* a) {
    const Tensor *x = tensor_of(a[0]), *w = tensor_of(a[1]), *r = a[2] == Py_None ? nullptr : tensor_of(a[2]);
    if (!PyFloat_CheckExact(a[3]) || (a[2] != Py_None && !r)) return false;
    c.x_stride = rows_of(x);
    if (!c.x_stride || !plain(w, 1) || w->size(0) != x->size(1) || !together(*x, *w)) return false;
    if ((c.code = float_code(*x)) < 0 || (c.weight_code = float_code(*w)) < 0) return false;
    if (r) {
        c.residual_stride = rows_of(r);
        if (!c.residual_stride || r->scalar_type() != x->scalar_type() || r->sizes() != x->sizes() || !together(*x, *r)) return false;
        c.residual = *r;
    }
    c.x = *x; c.weight = *w;
    c.eps = (float)PyFloat_AS_DOUBLE(a[3]);
    return here(*x, &c.stream);
}

// (y, s or nothing) of a call, or a status.
int norm_forward(const NormCall& c, Tensor (&o)[2]) {
    const auto like = at::TensorOptions().dtype(c.x.dtype()).device(c.x.device());
    const int64_t T = c.x.size(0), D = c.x.size(1);
    o[0] = at::empty({T, D}, like);
    if (c.residual.defined()) o[1] = at::empty({T, D}, like);
    return abi.fsa_norm_fwd(data(c.x), c.x_stride, data(c.residual), c.residual_stride, data(c.weight), c.code, c.weight_code, T, D, c.eps,
                            data(o[0]), data(o[1]), c.stream);
}

// Its backward runs on the stream of its forward, which is the one that autograd then makes current.
struct Norm : torch::autograd::Function<Norm> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const Tensor& x, const Tensor& weight,
                                                  const std::optional<Tensor>& residual, const NormCall& c) {
        Tensor o[2];
        if (const int rc = norm_forward(c, o)) throw Refused(rc);
        ctx->save_for_backward({residual ? o[1] : x, weight});
        ctx->set_materialize_grads(false);
        auto& d = ctx->saved_data;
        d["eps"] = (double)c.eps;
        d["stream"] = (int64_t)reinterpret_cast<intptr_t>(c.stream);
        if (residual) return {o[0], o[1]};
        return {o[0]};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        refuse_capture("a norm");
        const auto v = ctx->get_saved_variables();
        const Tensor &s = v[0], &weight = v[1];
        const bool again = differentiated(grads);
        torch::autograd::variable_list out(4);
        {
            at::AutoGradMode off(false);
            const Tensor gy = grads[0].defined() ? grads[0].contiguous() : Tensor(),
                         gs = grads.size() > 1 && grads[1].defined() ? grads[1].contiguous() : Tensor();
            const bool want_x = ctx->needs_input_grad(0), want_r = grads.size() > 1 && ctx->needs_input_grad(2), want_w = ctx->needs_input_grad(1);
            const int64_t T = s.size(0), D = s.size(1);
            const int code = float_code(s), weight_code = float_code(weight);
            const auto like = at::TensorOptions().dtype(s.dtype()).device(s.device());
            Tensor gx, ws;
            if (want_x || want_r) gx = at::empty({T, D}, like);
            if (want_w) out[1] = at::empty({D}, like.dtype(weight.dtype()));
            const int64_t need = want_w ? abi.fsa_norm_bwd_workspace_bytes(T, D, code) : 0;
            if (need) ws = at::empty({need}, like.dtype(at::kByte));
            const int rc = abi.fsa_norm_bwd(data(gy), data(gs), data(s), rows_of(&s), data(weight), code, weight_code, T, D,
                                            (float)ctx->saved_data["eps"].toDouble(), data(gx), data(out[1]), data(ws), need,
                                            reinterpret_cast<void*>((intptr_t)ctx->saved_data["stream"].toInt()));
            TORCH_CHECK(rc == FSA_OK, "the backward of a norm was refused (status ", rc, ")");
            if (want_x) out[0] = gx;
            if (want_r) out[2] = gx;
        }
        once("a norm", again, out);
        return out;
    }
};

// (x, weight, residual | None, eps) -> (y, s | None)
PyObject* norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 4) Py_RETURN_NONE;
    return or_none([&]() -> PyObject* {
        NormCall c;
        if (!norm_call(c, a)) { if (PyErr_Occurred()) return nullptr; Py_RETURN_NONE; }
        Tensor o[2];
        const int rc = without_gil([&] {
            at::AutoGradMode off(false);
            return norm_forward(c, o);
        });
        return rc != FSA_OK ? PyLong_FromLong(rc) : tuple_of(o);
    });
}

// The same with their gradients.
PyObject* norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 4) Py_RETURN_NONE;
    return or_none([&]() -> PyObject* {
        NormCall c;
        if (!norm_call(c, a)) { if (PyErr_Occurred()) return nullptr; Py_RETURN_NONE; }
        Tensor o[2];
        const int rc = without_gil([&] {
            try {
                // (an argument that is an undefined tensor is none that torch's function takes)
                const auto r = Norm::apply(c.x, c.weight, c.residual.defined() ? std::optional<Tensor>(c.residual) : std::nullopt, c);
                o[0] = r[0];
                if (r.size() > 1) o[1] = r[1];
                return (int)FSA_OK;
            } catch (const Refused& r) {
                return r.status;
            }
        });
        return rc != FSA_OK ? PyLong_FromLong(rc) : tuple_of(o);
    });
}

// ---------------------------------------------------------------------------------------------------------------
// gated feed-forward
// ---------------------------------------------------------------------------------------------------------------
struct GatedCall {
    Tensor t[4];                                           // x, w_gate, w_up, w_down
    int64_t stride[4], T, D, H, O;
    int code, activation;                                  // code: of the type, with FSA_GATED_FINE
    bool fine = false;
    enum Keep { kAsPays, kNever, kAlways } keep = kAsPays;    // what a backward would make again
    void* stream;
};

void gated_sizes(GatedCall& c) {
    for (int i = 0; i < 4; ++i) c.stride[i] = rows_of(&c.t[i]);
    c.T = c.t[0].size(0); c.D = c.t[0].size(1); c.H = c.t[1].size(0); c.O = c.t[3].size(0);
    c.code = float_code(c.t[0]);
    if (c.code >= 0 && c.fine) c.code |= FSA_GATED_FINE;
}

// (x, w_gate, w_up, w_down, activation's number[, fine[, keep: None, False or True]])
bool gated_call(GatedCall& c, PyObject* const* a, Py_ssize_t n) {
    if (!PyLong_CheckExact(a[4])) return false;
    c.activation = (int)PyLong_AsLong(a[4]);
    if (n > 5) {
        if (!PyBool_Check(a[5])) return false;
        c.fine = a[5] == Py_True;
    }
    if (n > 6) {
        if (a[6] != Py_None && !PyBool_Check(a[6])) return false;
        c.keep = a[6] == Py_None ? GatedCall::kAsPays : a[6] == Py_True ? GatedCall::kAlways : GatedCall::kNever;
    }
    for (int i = 0; i < 4; ++i) {
        const Tensor* t = tensor_of(a[i]);
        if (!rows_of(t)) return false;
        c.t[i] = *t;
    }
    gated_sizes(c);
    if (c.code < 0 || c.H < 1 || c.O < 1) return false;
    for (int i = 1; i < 4; ++i) if (c.t[i].scalar_type() != c.t[0].scalar_type() || !together(c.t[i], c.t[0])) return false;
    if (c.t[1].size(1) != c.D || c.t[2].size(0) != c.H || c.t[2].size(1) != c.D || c.t[3].size(1) != c.H) return false;
    return here(c.t[0], &c.stream);
}

int gated_forward(const GatedCall& c, bool keep, Tensor& y, Tensor& kept) {
    const auto like = at::TensorOptions().dtype(c.t[0].dtype()).device(c.t[0].device());
    y = at::empty({c.T, c.O}, like);
    if (keep && c.keep != GatedCall::kNever && (c.keep == GatedCall::kAlways || abi.fsa_gated_keep_pays(c.T, c.D, c.H, c.O, c.code))) {
        try {
            kept = at::empty({abi.fsa_gated_kept_bytes(c.T, c.D, c.H, c.O, c.code)}, like.dtype(at::kByte));
        } catch (const c10::OutOfMemoryError&) {           // no room for it: making it again needs none
            if (c.keep == GatedCall::kAlways) throw;
        }
    }
    const int64_t need = abi.fsa_gated_fwd_workspace_bytes(c.T, c.D, c.H, c.O, c.code);
    const Tensor ws = at::empty({need}, like.dtype(at::kByte));            // (may go once the call is queued: same stream)
    return abi.fsa_gated_fwd(data(c.t[0]), c.stride[0], data(c.t[1]), c.stride[1], data(c.t[2]), c.stride[2], data(c.t[3]), c.stride[3],
                             c.code, c.activation, c.T, c.D, c.H, c.O, data(y), data(kept), data(ws), need, c.stream);
}

struct Gated : torch::autograd::Function<Gated> {
    static Tensor forward(torch::autograd::AutogradContext* ctx, const Tensor& x, const Tensor& gate, const Tensor& up, const Tensor& down,
                          const GatedCall& c, bool keep) {
        Tensor y, kept;
        if (const int rc = gated_forward(c, keep, y, kept)) throw Refused(rc);
        ctx->save_for_backward({x, gate, up, down, kept});
        ctx->saved_data["activation"] = (int64_t)c.activation;
        ctx->saved_data["fine"] = c.fine;
        ctx->saved_data["stream"] = (int64_t)reinterpret_cast<intptr_t>(c.stream);
        return y;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads) {
        refuse_capture("a gated block");
        const auto v = ctx->get_saved_variables();
        const bool again = differentiated(grads);
        torch::autograd::variable_list out(6);
        {
            at::AutoGradMode off(false);
            GatedCall c;
            for (int i = 0; i < 4; ++i) c.t[i] = v[i];
            c.fine = ctx->saved_data["fine"].toBool();
            gated_sizes(c);
            const Tensor g = grads[0].contiguous(), &kept = v[4];
            const auto like = at::TensorOptions().dtype(g.dtype()).device(g.device());
            for (int i = 0; i < 4; ++i) if (ctx->needs_input_grad(i)) out[i] = at::empty(c.t[i].sizes(), like);
            const int64_t need = abi.fsa_gated_bwd_workspace_bytes(c.T, c.D, c.H, c.O, c.code);
            const Tensor ws = at::empty({need}, like.dtype(at::kByte));
            const int rc = abi.fsa_gated_bwd(data(g), rows_of(&g), data(c.t[0]), c.stride[0], data(c.t[1]), c.stride[1], data(c.t[2]), c.stride[2],
                                             data(c.t[3]), c.stride[3], c.code, (int)ctx->saved_data["activation"].toInt(), c.T, c.D, c.H, c.O,
                                             data(kept), data(out[0]), data(out[1]), data(out[2]), data(out[3]), data(ws), need,
                                             reinterpret_cast<void*>((intptr_t)ctx->saved_data["stream"].toInt()));
            TORCH_CHECK(rc == FSA_OK, "the backward of a gated block was refused (status ", rc, ")");
        }
        once("a gated block", again, out);
        return out;
    }
};

// (x, w_gate, w_up, w_down, activation's number[, fine]) -> y
PyObject* gated_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5 && n != 6) Py_RETURN_NONE;
    return or_none([&]() -> PyObject* {
        GatedCall c;
        if (!gated_call(c, a, n)) { if (PyErr_Occurred()) return nullptr; Py_RETURN_NONE; }
        Tensor y, kept;
        const int rc = without_gil([&] {
            at::AutoGradMode off(false);
            return gated_forward(c, false, y, kept);
        });
        return rc != FSA_OK ? PyLong_FromLong(rc) : wrap(y);
    });
}

// The same with its gradients (and `keep`).
PyObject* gated(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n < 5 || n > 7) Py_RETURN_NONE;
    return or_none([&]() -> PyObject* {
        GatedCall c;
        if (!gated_call(c, a, n)) { if (PyErr_Occurred()) return nullptr; Py_RETURN_NONE; }
        Tensor y;
        const int rc = without_gil([&] {
            try {
                bool keep = false;
                for (const Tensor& t : c.t) keep = keep || t.requires_grad();
                y = Gated::apply(c.t[0], c.t[1], c.t[2], c.t[3], c, keep && c10::GradMode::is_enabled());
                return (int)FSA_OK;
            } catch (const Refused& r) {
                return r.status;
            }
        });
        return rc != FSA_OK ? PyLong_FromLong(rc) : wrap(y);
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
    {"norm_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(norm_fwd)), METH_FASTCALL, nullptr},
    {"norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(norm)), METH_FASTCALL, nullptr},
    {"gated_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(gated_fwd)), METH_FASTCALL, nullptr},
    {"refuse_capture", refuse_captured, METH_O, nullptr},
    {"gated", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(gated)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fsa_block_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fsa_block_host() { return PyModule_Create(&module); }
