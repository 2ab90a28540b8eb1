// Native side of the Python binding: the common call of every entry point, from tensors to launch.
//
// A call of a small rollout is bound by its host side: argument checks, two output
// allocations and a ctypes call of some sixteen arguments took 8 to 12 us in Python against 2 to
// 5 us on the GPU (GAE 8 x 128: 9.7 us a call; 4096 x 256: 10.3). These functions do the same
// checks, allocate the missing outputs and call the C interface on the current stream.
//
// They only take calls that are plain in every respect (tensors of exactly torch's own type on
// the current GPU, right shapes and types, no active dispatch mode, no function mode but torch's
// default device) and return NotImplemented for any other, having done nothing: the Python function then runs its own checks
// and reports what is wrong, or handles the call. So every error a caller sees about its arguments
// comes from one place. Errors of the C interface are raised here as they are there.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <dlfcn.h>
#include <torch/csrc/PyInterpreter.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <initializer_list>
#include <vector>

#include "rlcs.h"

namespace {

PyObject* g_error = nullptr;   // RlcsError(fn, code)
PyObject* g_device = nullptr;  // torch.utils._device.DeviceContext

// The library's functions, looked up in the handle the package loaded.
struct Library {
    decltype(&rlcs_gae) gae;
    decltype(&rlcs_vtrace) vtrace;
    decltype(&rlcs_retrace) retrace;
    decltype(&rlcs_retrace_full) retrace_full;
    decltype(&rlcs_td_lambda) td_lambda;
    decltype(&rlcs_discounted) discounted;
    decltype(&rlcs_elig_trace) elig_trace;
    decltype(&rlcs_episodic_prefix) episodic_prefix;
    decltype(&rlcs_affine_scan) affine_scan;
    decltype(&rlcs_gae_strided) gae_strided;
    decltype(&rlcs_vtrace_strided) vtrace_strided;
    decltype(&rlcs_retrace_strided) retrace_strided;
    decltype(&rlcs_td_lambda_strided) td_lambda_strided;
    decltype(&rlcs_discounted_strided) discounted_strided;
    decltype(&rlcs_elig_trace_strided) elig_trace_strided;
    decltype(&rlcs_episodic_prefix_strided) episodic_prefix_strided;
    decltype(&rlcs_elig_trace_vec) elig_trace_vec;
    decltype(&rlcs_gae_masked) gae_masked;
    decltype(&rlcs_gae_masked_noalloc) gae_masked_noalloc;
    decltype(&rlcs_token_logp) token_logp;
    decltype(&rlcs_policy_loss) policy_loss;
    decltype(&rlcs_sample) sample;
    decltype(&rlcs_workspace_size_sample) workspace_size_sample;
    decltype(&rlcs_shared_prefix_attn) shared_prefix_attn;
    decltype(&rlcs_workspace_size_attn) workspace_size_attn;
    decltype(&rlcs_paged_attn) paged_attn;
    decltype(&rlcs_workspace_size_paged) workspace_size_paged;
    decltype(&rlcs_paged_write) paged_write;
    decltype(&rlcs_pages_fork) pages_fork;
    decltype(&rlcs_pages_resize) pages_resize;
    decltype(&rlcs_pages_compact) pages_compact;
    decltype(&rlcs_workspace_size_pages) workspace_size_pages;
    decltype(&rlcs_pages_copy) pages_copy;
    decltype(&rlcs_verify_draft) verify_draft;
    decltype(&rlcs_workspace_size_verify) workspace_size_verify;
    decltype(&rlcs_distill_loss) distill_loss;
} g_lib;
bool g_bound = false;

struct NoGil {
    PyThreadState* state = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(state); }
};

// Keys of tensors whose memory is not simply theirs (function transforms, subclasses, lazy
// negation and the like).
const c10::DispatchKeySet kSpecial({c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot,
                                    c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                    c10::DispatchKey::Functionalize, c10::DispatchKey::Conjugate,
                                    c10::DispatchKey::Negative, c10::DispatchKey::ZeroTensor});

// Whether the function modes in force leave the call as it is: none, or torch's default device
// (torch.set_default_device, `with torch.device(...)`), which only gives a device to factory
// functions called without one. Every allocation here names its device.
bool modes_pass() {
    using TLS = at::impl::PythonTorchFunctionTLS;
    for (int64_t i = 0, n = TLS::stack_len(); i < n; ++i)
        if (reinterpret_cast<PyObject*>(Py_TYPE(TLS::get_stack_at(i)->ptr(getPyInterpreter()))) != g_device) return false;
    return true;
}

// One call: its shape, and whether every argument seen so far is a plain one.
struct Call {
    bool ok = true;
    const bool strided;
    int64_t N = 0, T = 0, sn = 0, st = 0;
    int64_t inner = 0;  // last dimension of a 3-D first input, or 0
    at::ScalarType dtype = at::kFloat;
    at::Device device = at::kCPU;

    explicit Call(bool s) : strided(s) {
        ok = g_bound && !c10::impl::TorchDispatchModeTLS::any_modes_set() &&
             modes_pass();
    }

    bool bf16() const { return dtype == at::kBFloat16; }
    rlcs_dtype type() const { return bf16() ? RLCS_BF16 : RLCS_F32; }

    // A plain tensor, or null (None, or not plain: then ok is false).
    const at::Tensor* plain(PyObject* o) {
        if (!ok || o == Py_None) return nullptr;
        if (!THPVariable_CheckExact(o)) {
            ok = false;
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.key_set().has_any(kSpecial) || t.layout() != at::kStrided || !t.has_storage()) {
            ok = false;
            return nullptr;
        }
        return &t;
    }

    // (stride_n, stride_t) of an [N, T] view; a dimension of one step takes the stride that nests
    // the two (it never multiplies an index other than 0).
    void strides(const at::Tensor& t, int64_t& a, int64_t& b) const {
        a = t.stride(0);
        b = t.stride(1);
        if (T == 1) b = std::max<int64_t>(1, N * std::max<int64_t>(a, 1));
        if (N == 1) a = std::max<int64_t>(1, T * std::max<int64_t>(b, 1));
    }

    // The first data input decides shape, type and device.
    void* first(PyObject* o, int dims = 2) {
        const at::Tensor* t = plain(o);
        if (!t) {
            ok = false;
            return nullptr;
        }
        dtype = t->scalar_type();
        device = t->device();
        if (t->dim() != dims || (dtype != at::kFloat && dtype != at::kBFloat16) || !device.is_cuda() ||
            device.index() != c10::hip::current_device()) {
            ok = false;
            return nullptr;
        }
        N = t->size(0);
        T = t->size(1);
        if (dims == 3) inner = t->size(2);
        if (strided) strides(*t, sn, st);
        return same_layout(*t) ? t->data_ptr() : nullptr;
    }

    // Whether a tensor of the call's shape lies as the call says it does.
    bool same_layout(const at::Tensor& t) {
        if (strided) {
            int64_t a, b;
            strides(t, a, b);
            ok = ok && a == sn && b == st;
        } else {
            ok = ok && t.is_contiguous();
        }
        return ok;
    }

    void* checked(PyObject* o, at::ScalarType type, at::IntArrayRef shape, bool of_call) {
        const at::Tensor* t = plain(o);
        if (!t) return nullptr;
        ok = ok && t->scalar_type() == type && t->sizes() == shape && t->device() == device;
        if (!ok) return nullptr;
        if (of_call) same_layout(*t);
        else ok = t->is_contiguous();
        return ok ? t->data_ptr() : nullptr;
    }
    void* data(PyObject* o) { return checked(o, dtype, {N, T}, true); }
    void* actions_axis(PyObject* o, int64_t A) { return checked(o, dtype, {N, T, A}, false); }
    int32_t* actions(PyObject* o) { return static_cast<int32_t*>(checked(o, at::kInt, {N, T}, false)); }
    void* per_row(PyObject* o) { return checked(o, dtype, {N}, false); }
    const uint8_t* flags(PyObject* o) {
        const at::Tensor* t = plain(o);
        if (!t) return nullptr;
        const at::ScalarType s = t->scalar_type();
        ok = ok && (s == at::kByte || s == at::kBool);
        return static_cast<const uint8_t*>(checked(o, s, {N, T}, true));
    }
    void* workspace(PyObject* o, size_t& bytes) {
        bytes = 0;
        const at::Tensor* t = plain(o);
        if (!t) return nullptr;
        ok = ok && t->device() == device && t->is_contiguous();
        if (!ok) return nullptr;
        bytes = t->nbytes();
        return t->data_ptr();
    }
    float number(PyObject* o) {
        if (PyFloat_CheckExact(o)) return float(PyFloat_AS_DOUBLE(o));
        if (PyLong_CheckExact(o)) {
            const double v = PyLong_AsDouble(o);
            if (v != -1.0 || !PyErr_Occurred()) return float(v);
            PyErr_Clear();
        }
        ok = false;
        return 0.f;
    }
    int64_t integer(PyObject* o) {
        if (PyLong_CheckExact(o)) {
            int over = 0;
            const long long v = PyLong_AsLongLongAndOverflow(o, &over);
            if (!over) return v;
        }
        ok = false;
        return 0;
    }
    bool truth(PyObject* o) {
        if (o != Py_True && o != Py_False) ok = false;
        return o == Py_True;
    }
};

// An output: given by the caller, allocated by the call, or not wanted.
struct Out {
    PyObject* given = nullptr;
    bool make = false;
    at::Tensor made;
    float* ptr = nullptr;

    Out(Call& c, PyObject* o, bool want) {
        if (o == Py_None) {
            make = want;
            return;
        }
        given = o;
        if (c.inner) ptr = static_cast<float*>(c.checked(o, at::kFloat, {c.N, c.T, c.inner}, false));
        else ptr = static_cast<float*>(c.checked(o, at::kFloat, {c.N, c.T}, true));
    }
    void allocate(const Call& c) {
        if (!make) return;
        const auto options = at::TensorOptions().dtype(at::kFloat).device(c.device);
        if (c.inner) made = at::empty({c.N, c.T, c.inner}, options);
        else if (c.strided) made = at::empty_strided({c.N, c.T}, {c.sn, c.st}, options);
        else made = at::empty({c.N, c.T}, options);
        ptr = static_cast<float*>(made.data_ptr());
    }
    // A new reference: the tensor, or None.
    PyObject* object() {
        if (make) return THPVariable_Wrap(made);
        PyObject* o = given ? given : Py_None;
        Py_INCREF(o);
        return o;
    }
};

// Allocates, calls `fn(stream)` and returns the outputs: one tensor, or a pair with `second`.
template <class Fn>
PyObject* run(Call& c, const char* name, Out& a, Out* second, Fn&& fn) {
    if (!c.ok) Py_RETURN_NOTIMPLEMENTED;
    int code = 0;
    try {
        NoGil no_gil;
        a.allocate(c);
        if (second) second->allocate(c);
        code = fn(static_cast<rlcs_stream_t>(c10::hip::getCurrentHIPStream(c.device.index()).stream()));
    } catch (...) {  // an allocation that failed: the Python function meets it again and reports it
        Py_RETURN_NOTIMPLEMENTED;
    }
    if (code != RLCS_OK) {
        PyObject* e = PyObject_CallFunction(g_error, "si", name, code);
        if (e) {
            PyErr_SetObject(g_error, e);
            Py_DECREF(e);
        }
        return nullptr;
    }
    PyObject* x = a.object();
    if (!second || !x) return x;
    PyObject* y = second->object();
    if (!y) {
        Py_DECREF(x);
        return nullptr;
    }
    PyObject* pair = PyTuple_New(2);
    if (!pair) {
        Py_DECREF(x);
        Py_DECREF(y);
        return nullptr;
    }
    PyTuple_SET_ITEM(pair, 0, x);
    PyTuple_SET_ITEM(pair, 1, y);
    return pair;
}

typedef PyObject* const* Argv;

// A function of the module: F, or NotImplemented where an accessor of an exotic tensor throws.
template <PyObject* (*F)(Argv, Py_ssize_t)>
PyObject* entry(PyObject*, Argv x, Py_ssize_t nargs) {
    try {
        return F(x, nargs);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NOTIMPLEMENTED;
    }
}

#define RLCS_ARGS(n) \
    if (nargs != (n)) Py_RETURN_NOTIMPLEMENTED

// gae(r, v, term, trunc, bv, boot, adv, ret, gamma, lam, ws, want_ret)
template <bool S>
PyObject* gae(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(12);
    Call c(S);
    void *r = c.first(x[0]), *v = c.data(x[1]);
    const uint8_t *te = c.flags(x[2]), *tr = c.flags(x[3]);
    void *bv = c.data(x[4]), *b = c.per_row(x[5]);
    Out o0(c, x[6], true), o1(c, x[7], c.truth(x[11]));
    const float g = c.number(x[8]), l = c.number(x[9]);
    size_t wb;
    void* ws = c.workspace(x[10], wb);
    return run(c, S ? "rlcs_gae_strided" : "rlcs_gae", o0, &o1, [&](rlcs_stream_t s) {
        if constexpr (S) return g_lib.gae_strided(r, v, te, tr, bv, b, o0.ptr, o1.ptr, c.N, c.T, c.sn, c.st, g, l, c.type(), ws, wb, s);
        else return g_lib.gae(r, v, te, tr, bv, b, o0.ptr, o1.ptr, c.N, c.T, g, l, c.type(), ws, wb, s);
    });
}

// vtrace(r, v, log_rho, term, trunc, bv, boot, vs, pg, gamma, rho_bar, c_bar, ws, want_pg)
template <bool S>
PyObject* vtrace(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(14);
    Call c(S);
    void *r = c.first(x[0]), *v = c.data(x[1]), *lr = c.data(x[2]);
    const uint8_t *te = c.flags(x[3]), *tr = c.flags(x[4]);
    void *bv = c.data(x[5]), *b = c.per_row(x[6]);
    Out o0(c, x[7], true), o1(c, x[8], c.truth(x[13]));
    const float g = c.number(x[9]), rb = c.number(x[10]), cb = c.number(x[11]);
    size_t wb;
    void* ws = c.workspace(x[12], wb);
    return run(c, S ? "rlcs_vtrace_strided" : "rlcs_vtrace", o0, &o1, [&](rlcs_stream_t s) {
        if constexpr (S) return g_lib.vtrace_strided(r, v, lr, te, tr, bv, b, o0.ptr, o1.ptr, c.N, c.T, c.sn, c.st, g, rb, cb, c.type(), ws, wb, s);
        else return g_lib.vtrace(r, v, lr, te, tr, bv, b, o0.ptr, o1.ptr, c.N, c.T, g, rb, cb, c.type(), ws, wb, s);
    });
}

// retrace(r, q, eq, log_rho, term, trunc, bv, boot, delta, q_ret, gamma, lam, c_bar, ws, want_q_ret)
template <bool S>
PyObject* retrace(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(15);
    Call c(S);
    void *r = c.first(x[0]), *q = c.data(x[1]), *eq = c.data(x[2]), *lr = c.data(x[3]);
    const uint8_t *te = c.flags(x[4]), *tr = c.flags(x[5]);
    void *bv = c.data(x[6]), *b = c.per_row(x[7]);
    Out o0(c, x[8], true), o1(c, x[9], c.truth(x[14]));
    const float g = c.number(x[10]), l = c.number(x[11]), cb = c.number(x[12]);
    size_t wb;
    void* ws = c.workspace(x[13], wb);
    return run(c, S ? "rlcs_retrace_strided" : "rlcs_retrace", o0, &o1, [&](rlcs_stream_t s) {
        if constexpr (S) return g_lib.retrace_strided(r, q, eq, lr, te, tr, bv, b, o0.ptr, o1.ptr, c.N, c.T, c.sn, c.st, g, l, cb, c.type(), ws, wb, s);
        else return g_lib.retrace(r, q, eq, lr, te, tr, bv, b, o0.ptr, o1.ptr, c.N, c.T, g, l, cb, c.type(), ws, wb, s);
    });
}

// retrace_full(r, q, pi, actions, mu, term, trunc, bv, boot, delta, q_ret, gamma, lam, c_bar, ws,
// want_q_ret)
PyObject* retrace_full(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(16);
    Call c(false);
    void* r = c.first(x[0]);
    const at::Tensor* qt = c.plain(x[1]);
    if (!qt || qt->dim() != 3 || x[2] == Py_None || x[3] == Py_None) Py_RETURN_NOTIMPLEMENTED;
    const int64_t A = qt->size(2);
    void *q = c.actions_axis(x[1], A), *pi = c.actions_axis(x[2], A);
    int32_t* act = c.actions(x[3]);
    void* mu = c.data(x[4]);
    const uint8_t *te = c.flags(x[5]), *tr = c.flags(x[6]);
    void *bv = c.data(x[7]), *b = c.per_row(x[8]);
    Out o0(c, x[9], true), o1(c, x[10], c.truth(x[15]));
    const float g = c.number(x[11]), l = c.number(x[12]), cb = c.number(x[13]);
    size_t wb;
    void* ws = c.workspace(x[14], wb);
    return run(c, "rlcs_retrace_full", o0, &o1, [&](rlcs_stream_t s) {
        return g_lib.retrace_full(r, q, pi, act, mu, te, tr, bv, b, o0.ptr, o1.ptr, c.N, c.T, A, g, l, cb, c.type(), ws, wb, s);
    });
}

// td_lambda(r, v, term, trunc, bv, boot, ret, gamma, lam, ws)
template <bool S>
PyObject* td_lambda(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(10);
    Call c(S);
    void *r = c.first(x[0]), *v = c.data(x[1]);
    const uint8_t *te = c.flags(x[2]), *tr = c.flags(x[3]);
    void *bv = c.data(x[4]), *b = c.per_row(x[5]);
    Out o(c, x[6], true);
    const float g = c.number(x[7]), l = c.number(x[8]);
    size_t wb;
    void* ws = c.workspace(x[9], wb);
    return run(c, S ? "rlcs_td_lambda_strided" : "rlcs_td_lambda", o, nullptr, [&](rlcs_stream_t s) {
        if constexpr (S) return g_lib.td_lambda_strided(r, v, te, tr, bv, b, o.ptr, c.N, c.T, c.sn, c.st, g, l, c.type(), ws, wb, s);
        else return g_lib.td_lambda(r, v, te, tr, bv, b, o.ptr, c.N, c.T, g, l, c.type(), ws, wb, s);
    });
}

// discounted(r, term, trunc, bv, boot, ret, gamma, ws)
template <bool S>
PyObject* discounted(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(8);
    Call c(S);
    void* r = c.first(x[0]);
    const uint8_t *te = c.flags(x[1]), *tr = c.flags(x[2]);
    void *bv = c.data(x[3]), *b = c.per_row(x[4]);
    Out o(c, x[5], true);
    const float g = c.number(x[6]);
    size_t wb;
    void* ws = c.workspace(x[7], wb);
    return run(c, S ? "rlcs_discounted_strided" : "rlcs_discounted", o, nullptr, [&](rlcs_stream_t s) {
        if constexpr (S) return g_lib.discounted_strided(r, te, tr, bv, b, o.ptr, c.N, c.T, c.sn, c.st, g, c.type(), ws, wb, s);
        else return g_lib.discounted(r, te, tr, bv, b, o.ptr, c.N, c.T, g, c.type(), ws, wb, s);
    });
}

// elig_trace(x, term, trunc, z, gamma, lam, ws)
template <bool S>
PyObject* elig_trace(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(7);
    Call c(S);
    void* in = c.first(x[0]);
    const uint8_t *te = c.flags(x[1]), *tr = c.flags(x[2]);
    Out o(c, x[3], true);
    const float g = c.number(x[4]), l = c.number(x[5]);
    size_t wb;
    void* ws = c.workspace(x[6], wb);
    return run(c, S ? "rlcs_elig_trace_strided" : "rlcs_elig_trace", o, nullptr, [&](rlcs_stream_t s) {
        if constexpr (S) return g_lib.elig_trace_strided(in, te, tr, o.ptr, c.N, c.T, c.sn, c.st, g, l, c.type(), ws, wb, s);
        else return g_lib.elig_trace(in, te, tr, o.ptr, c.N, c.T, g, l, c.type(), ws, wb, s);
    });
}

// episodic_prefix(x, term, trunc, c, starts_at, ws)
template <bool S>
PyObject* episodic_prefix(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(6);
    Call c(S);
    void* in = c.first(x[0]);
    const uint8_t *te = c.flags(x[1]), *tr = c.flags(x[2]);
    Out o(c, x[3], true);
    const rlcs_boundary b = c.truth(x[4]) ? RLCS_STARTS_AT : RLCS_ENDS_AT;
    size_t wb;
    void* ws = c.workspace(x[5], wb);
    return run(c, S ? "rlcs_episodic_prefix_strided" : "rlcs_episodic_prefix", o, nullptr, [&](rlcs_stream_t s) {
        if constexpr (S) return g_lib.episodic_prefix_strided(in, te, tr, o.ptr, c.N, c.T, c.sn, c.st, b, c.type(), ws, wb, s);
        else return g_lib.episodic_prefix(in, te, tr, o.ptr, c.N, c.T, b, c.type(), ws, wb, s);
    });
}

// affine_scan(alpha, beta, carry, out, reverse, ws)
PyObject* affine_scan(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(6);
    Call c(false);
    void *al = c.first(x[0]), *be = c.data(x[1]), *carry = c.per_row(x[2]);
    Out o(c, x[3], true);
    const rlcs_direction d = c.truth(x[4]) ? RLCS_BACKWARD : RLCS_FORWARD;
    size_t wb;
    void* ws = c.workspace(x[5], wb);
    return run(c, "rlcs_affine_scan", o, nullptr, [&](rlcs_stream_t s) {
        return g_lib.affine_scan(al, be, carry, o.ptr, c.N, c.T, d, c.type(), ws, wb, s);
    });
}

// elig_trace_vec(x, term, trunc, z, gamma, lam, ws)
PyObject* elig_trace_vec(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(7);
    Call c(false);
    void* in = c.first(x[0], 3);
    const int64_t F = c.inner;
    if (!c.ok || F == 0) Py_RETURN_NOTIMPLEMENTED;
    const uint8_t *te = c.flags(x[1]), *tr = c.flags(x[2]);
    Out o(c, x[3], true);
    const float g = c.number(x[4]), l = c.number(x[5]);
    size_t wb;
    void* ws = c.workspace(x[6], wb);
    return run(c, "rlcs_elig_trace_vec", o, nullptr, [&](rlcs_stream_t s) {
        return g_lib.elig_trace_vec(in, te, tr, o.ptr, c.N, c.T, F, g, l, c.type(), ws, wb, s);
    });
}

// gae_masked(r, v, mask, term, trunc, bv, boot, adv, ret, gamma, lam, normalize, eps, want_ret[, ws])
PyObject* gae_masked(Argv x, Py_ssize_t nargs) {
    if (nargs != 14 && nargs != 15) Py_RETURN_NOTIMPLEMENTED;
    Call c(false);
    void *r = c.first(x[0]), *v = c.data(x[1]);
    const uint8_t *mk = c.flags(x[2]), *te = c.flags(x[3]), *tr = c.flags(x[4]);
    void *bv = c.data(x[5]), *b = c.per_row(x[6]);
    Out o0(c, x[7], true), o1(c, x[8], c.truth(x[13]));
    const float g = c.number(x[9]), l = c.number(x[10]), eps = c.number(x[12]);
    const int norm = c.truth(x[11]) ? 1 : 0;
    size_t wb = 0;
    void* ws = nargs == 15 ? c.workspace(x[14], wb) : nullptr;
    if (nargs == 14)
        return run(c, "rlcs_gae_masked_noalloc", o0, &o1, [&](rlcs_stream_t s) {
            return g_lib.gae_masked_noalloc(r, v, mk, te, tr, bv, b, o0.ptr, o1.ptr, c.N, c.T, g, l, norm, eps, c.type(), s);
        });
    if (norm && !ws) Py_RETURN_NOTIMPLEMENTED;  // the Python function makes one
    return run(c, "rlcs_gae_masked", o0, &o1, [&](rlcs_stream_t s) {
        return g_lib.gae_masked(r, v, mk, te, tr, bv, b, o0.ptr, o1.ptr, c.N, c.T, g, l, norm, eps, c.type(), ws, wb, s);
    });
}

// ------------------------------------------------------------- rows of logits and attention

// Rows of [..., V] logits (contiguous, or a matrix with its rows any stride apart) and what the calls
// on them share.
struct Rows {
    int64_t M = 1, V = 0, ld = 0;
    std::vector<int64_t> lead;

    // False: not such rows.
    bool of(const at::Tensor& t) {
        const int64_t dims = t.dim();
        if (dims < 2) return false;
        V = t.size(dims - 1);
        lead.assign(t.sizes().begin(), t.sizes().end() - 1);
        for (const int64_t n : lead) M *= n;
        ld = V;
        if (t.is_contiguous()) return true;
        if (dims != 2 || (V > 1 && t.stride(1) != 1)) return false;
        if (M > 1) ld = t.stride(0);
        return ld >= V;
    }
};

// (Rows without logits are left to the Python function.)
void* rows_input(Call& c, PyObject* o, Rows& r) {
    const at::Tensor* t = c.plain(o);
    if (!t) {
        c.ok = false;
        return nullptr;
    }
    c.dtype = t->scalar_type();
    c.device = t->device();
    c.ok = c.ok && (c.dtype == at::kFloat || c.dtype == at::kBFloat16) && c.device.is_cuda() &&
           c.device.index() == c10::hip::current_device() && r.of(*t) && r.V > 0;
    return c.ok ? t->data_ptr() : nullptr;
}

// A matrix of the logits' shape with rows of its own stride.
void* rows_beside(Call& c, PyObject* o, at::ScalarType type, const Rows& r, int64_t& ld) {
    ld = r.V;
    const at::Tensor* t = c.plain(o);
    if (!t) return nullptr;
    Rows own;
    c.ok = c.ok && t->scalar_type() == type && t->device() == c.device && own.of(*t) && own.V == r.V && own.lead == r.lead;
    ld = own.ld;
    return c.ok ? t->data_ptr() : nullptr;
}

// An output of any shape and type: given by the caller, allocated by the call, or not wanted.
struct Result {
    PyObject* given = nullptr;
    bool make = false;
    at::ScalarType type;
    std::vector<int64_t> shape;
    at::Tensor made;
    void* ptr = nullptr;

    Result(Call& c, PyObject* o, bool want, at::ScalarType t, at::IntArrayRef sizes) : type(t), shape(sizes.vec()) {
        if (o == Py_None) {
            make = want;
            return;
        }
        given = o;
        ptr = c.checked(o, type, sizes, false);
    }
    void allocate(const Call& c) {
        if (!make) return;
        made = at::empty(shape, at::TensorOptions().dtype(type).device(c.device));
        ptr = made.data_ptr();
    }
    PyObject* object() {
        if (make) return THPVariable_Wrap(made);
        PyObject* o = given ? given : Py_None;
        Py_INCREF(o);
        return o;
    }
    // Tells autograd that the caller's tensor has new contents: a backward that saved the old ones raises an error.
    void written() const {
        if (!given) return;
        const at::Tensor& t = THPVariable_Unpack(given);
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    }
    float* f32() const { return static_cast<float*>(ptr); }
};

// Allocates the results and `ws_bytes` of workspace, calls `fn(stream, workspace)` and returns the
// results as a tuple.
template <class Fn>
PyObject* run_results(Call& c, const char* name, std::initializer_list<Result*> results, size_t ws_bytes, Fn&& fn) {
    if (!c.ok) Py_RETURN_NOTIMPLEMENTED;
    int code = 0;
    try {
        NoGil no_gil;
        for (Result* r : results) r->allocate(c);
        at::Tensor ws;
        if (ws_bytes) ws = at::empty({int64_t(ws_bytes)}, at::TensorOptions().dtype(at::kByte).device(c.device));
        code = fn(static_cast<rlcs_stream_t>(c10::hip::getCurrentHIPStream(c.device.index()).stream()),
                  ws_bytes ? ws.data_ptr() : nullptr);
    } catch (...) {  // an allocation that failed: the Python function meets it again and reports it
        Py_RETURN_NOTIMPLEMENTED;
    }
    if (code != RLCS_OK) {
        PyObject* e = PyObject_CallFunction(g_error, "si", name, code);
        if (e) {
            PyErr_SetObject(g_error, e);
            Py_DECREF(e);
        }
        return nullptr;
    }
    for (const Result* r : results) r->written();
    PyObject* tuple = PyTuple_New(Py_ssize_t(results.size()));
    Py_ssize_t i = 0;
    for (Result* r : results) {
        PyObject* o = tuple ? r->object() : nullptr;
        if (!o) {
            Py_XDECREF(tuple);
            return nullptr;
        }
        PyTuple_SET_ITEM(tuple, i++, o);
    }
    return tuple;
}

// token_logp(logits, tokens, logp, ent, temperature, want_ent)
PyObject* token_logp(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(6);
    if (x[1] == Py_None) Py_RETURN_NOTIMPLEMENTED;
    Call c(false);
    Rows r;
    void* logits = rows_input(c, x[0], r);
    const int32_t* tokens = static_cast<int32_t*>(c.checked(x[1], at::kInt, r.lead, false));
    Result logp(c, x[2], true, at::kFloat, r.lead), ent(c, x[3], c.truth(x[5]), at::kFloat, r.lead);
    const float temperature = c.number(x[4]);
    return run_results(c, "rlcs_token_logp", {&logp, &ent}, 0, [&](rlcs_stream_t s, void*) {
        return g_lib.token_logp(logits, tokens, logp.f32(), ent.f32(), r.M, r.V, r.ld, temperature, c.type(), s);
    });
}

// policy_loss(logits, tokens, logp_old, adv, weight, loss, dlogits, logp, ent, clip_low, clip_high, ent_coef,
// temperature, want_grad)
PyObject* policy_loss(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(14);
    if (x[1] == Py_None || x[2] == Py_None || x[3] == Py_None) Py_RETURN_NOTIMPLEMENTED;
    Call c(false);
    Rows r;
    void* logits = rows_input(c, x[0], r);
    const int32_t* tokens = static_cast<int32_t*>(c.checked(x[1], at::kInt, r.lead, false));
    auto per_token = [&](PyObject* o) { return static_cast<float*>(c.checked(o, at::kFloat, r.lead, false)); };
    const float *old = per_token(x[2]), *adv = per_token(x[3]), *weight = per_token(x[4]);
    Result loss(c, x[5], true, at::kFloat, r.lead);
    std::vector<int64_t> full = r.lead;
    full.push_back(r.V);
    Result grad(c, Py_None, c.truth(x[13]), c.dtype, full);
    int64_t ld_grad = r.V;
    if (x[6] != Py_None) {  // rows of its own stride
        grad.make = false;
        grad.given = x[6];
        grad.ptr = rows_beside(c, x[6], c.dtype, r, ld_grad);
    }
    Result logp(c, x[7], true, at::kFloat, r.lead), ent(c, x[8], true, at::kFloat, r.lead);
    const float lo = c.number(x[9]), hi = c.number(x[10]), ec = c.number(x[11]), temperature = c.number(x[12]);
    return run_results(c, "rlcs_policy_loss", {&loss, &grad, &logp, &ent}, 0, [&](rlcs_stream_t s, void*) {
        return g_lib.policy_loss(logits, tokens, old, adv, weight, loss.f32(), grad.ptr, logp.f32(), ent.f32(), r.M, r.V, r.ld,
                                 ld_grad, lo, hi, ec, temperature, c.type(), s);
    });
}

// sample(logits, noise, tokens, logp, temperature, top_k, top_p, min_p, want_logp, ws)
PyObject* sample(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(10);
    Call c(false);
    Rows r;
    void* logits = rows_input(c, x[0], r);
    int64_t ld_noise = 0;
    const float* noise = static_cast<float*>(rows_beside(c, x[1], at::kFloat, r, ld_noise));
    Result tokens(c, x[2], true, at::kInt, r.lead), logp(c, x[3], c.truth(x[8]), at::kFloat, r.lead);
    // a setting: a number, or a tensor of each row's own
    float all[3] = {0.f, 0.f, 0.f};
    const float* own[3] = {nullptr, nullptr, nullptr};
    const int at_arg[3] = {4, 6, 7};
    for (int i = 0; i < 3; ++i) {
        PyObject* o = x[at_arg[i]];
        if (THPVariable_CheckExact(o)) own[i] = static_cast<float*>(c.checked(o, at::kFloat, r.lead, false));
        else all[i] = c.number(o);
    }
    const int32_t* own_k = nullptr;
    int32_t all_k = 0;
    if (THPVariable_CheckExact(x[5])) {
        own_k = static_cast<int32_t*>(c.checked(x[5], at::kInt, r.lead, false));
    } else if (PyLong_CheckExact(x[5])) {
        int over = 0;
        const long long k = PyLong_AsLongLongAndOverflow(x[5], &over);
        if (over || k > INT32_MAX || k < -1) Py_RETURN_NOTIMPLEMENTED;
        all_k = int32_t(k);
    } else {
        Py_RETURN_NOTIMPLEMENTED;
    }
    size_t wb = 0;
    void* ws = c.workspace(x[9], wb);
    const size_t make = c.ok && !ws ? g_lib.workspace_size_sample(r.M, r.V) : 0;
    return run_results(c, "rlcs_sample", {&tokens, &logp}, make, [&](rlcs_stream_t s, void* made) {
        return g_lib.sample(logits, noise, own[0], own_k, own[1], own[2], static_cast<int32_t*>(tokens.ptr), logp.f32(), r.M, r.V,
                            r.ld, ld_noise, all[0], all_k, all[1], all[2], c.type(), made ? made : ws, made ? make : wb, s);
    });
}

// shared_prefix_attn(q, kp, vp, ks, vs, prefix_len, suffix_len, o, lse, scale, want_lse, ws)
PyObject* shared_prefix_attn(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(12);
    Call c(false);
    const at::Tensor* q = c.plain(x[0]);
    const at::Tensor *kp = c.plain(x[1]), *vp = c.plain(x[2]), *ks = c.plain(x[3]), *vs = c.plain(x[4]);
    if (!c.ok || !q || !kp || !vp || q->dim() != 4 || kp->dim() != 4 || (ks == nullptr) != (vs == nullptr)) Py_RETURN_NOTIMPLEMENTED;
    c.dtype = q->scalar_type();
    c.device = q->device();
    c.ok = (c.dtype == at::kFloat || c.dtype == at::kBFloat16) && c.device.is_cuda() && c.device.index() == c10::hip::current_device();
    const int64_t N = q->size(0), G = q->size(1), Hq = q->size(2), D = q->size(3), P = kp->size(1), Hkv = kp->size(2);
    const int64_t S = ks && ks->dim() == 5 ? ks->size(2) : 0;
    if (D == 0) Py_RETURN_NOTIMPLEMENTED;
    rlcs_attn_layout at{};
    auto operand = [&](const at::Tensor* t, at::IntArrayRef sizes, int64_t* strides) -> const void* {
        if (!t) return nullptr;
        c.ok = c.ok && t->scalar_type() == c.dtype && t->device() == c.device && t->sizes() == sizes && (D <= 1 || t->stride(-1) == 1);
        if (!c.ok) return nullptr;
        for (size_t i = 0; i + 1 < sizes.size(); ++i) strides[i] = sizes[i] <= 1 ? 0 : t->stride(int64_t(i));
        return t->data_ptr();
    };
    const void *pq = operand(q, {N, G, Hq, D}, at.q), *pkp = operand(kp, {N, P, Hkv, D}, at.kp), *pvp = operand(vp, {N, P, Hkv, D}, at.vp);
    const void *pks = operand(ks, {N, G, S, Hkv, D}, at.ks), *pvs = operand(vs, {N, G, S, Hkv, D}, at.vs);
    const int32_t* pl = static_cast<int32_t*>(c.checked(x[5], at::kInt, {N}, false));
    const int32_t* sl = static_cast<int32_t*>(c.checked(x[6], at::kInt, {N, G}, false));
    Result o(c, x[7], true, c.dtype, {N, G, Hq, D}), lse(c, x[8], c.truth(x[10]), at::kFloat, {N, G, Hq});
    const float scale = x[9] == Py_None ? float(1.0 / std::sqrt(double(D))) : c.number(x[9]);
    size_t wb = 0;
    void* ws = c.workspace(x[11], wb);
    const size_t make = c.ok && !ws ? g_lib.workspace_size_attn(N, G, Hq, Hkv, D, P, S) : 0;
    return run_results(c, "rlcs_shared_prefix_attn", {&o, &lse}, make, [&](rlcs_stream_t s, void* made) {
        return g_lib.shared_prefix_attn(pq, pkp, pvp, pks, pvs, pl, sl, o.ptr, lse.f32(), N, G, Hq, Hkv, D, P, S, &at, scale, c.type(),
                                        made ? made : ws, made ? make : wb, s);
    });
}

// ------------------------------------------------------------- a paged cache, drafted tokens, distillation

// A tensor that is not the call's first input, contiguous in its last dimension; its other strides go to `strides`.
void* rows_of(Call& c, PyObject* o, at::IntArrayRef sizes, int64_t* strides) {
    const at::Tensor* t = c.plain(o);
    c.ok = c.ok && t && t->scalar_type() == c.dtype && t->device() == c.device && t->sizes() == sizes &&
           (sizes.back() <= 1 || t->stride(-1) == 1);
    if (!c.ok) return nullptr;
    for (size_t i = 0; i + 1 < sizes.size(); ++i) strides[i] = sizes[i] <= 1 ? 0 : t->stride(int64_t(i));
    return t->data_ptr();
}
int32_t* ints(Call& c, PyObject* o, at::IntArrayRef sizes) { return static_cast<int32_t*>(c.checked(o, at::kInt, sizes, false)); }

// What a call changes in place.
struct InPlace : Result {
    InPlace(Call& c, PyObject* o, void* p) : Result(c, Py_None, false, c.dtype, {}) {
        given = o;
        ptr = p;
    }
};

// Cache, table and sequences of the calls on a paged cache; `first` is [tokens, heads, D].
struct Paged {
    int64_t n = 0, heads = 0, D = 0, B = 0, W = 0, ld = 0, pages = 0, page = 0, Hkv = 0;
    void *k = nullptr, *v = nullptr;
    const int32_t *table = nullptr, *length = nullptr, *start = nullptr;
    rlcs_paged_layout at{};

    void of(Call& c, PyObject* first, PyObject* k_cache, PyObject* v_cache, PyObject* t, PyObject* len, PyObject* q_start) {
        const at::Tensor *f = c.plain(first), *kc = c.plain(k_cache), *tb = c.plain(t);
        c.ok = c.ok && f && kc && tb && len != Py_None && f->dim() == 3 && kc->dim() == 4 && tb->dim() == 2;
        if (!c.ok) return;
        c.dtype = f->scalar_type();
        c.device = f->device();
        n = f->size(0); heads = f->size(1); D = f->size(2);
        pages = kc->size(0); page = kc->size(1); Hkv = kc->size(2);
        B = tb->size(0); W = tb->size(1);
        ld = B > 1 ? tb->stride(0) : W;
        c.ok = (c.dtype == at::kFloat || c.dtype == at::kBFloat16) && c.device.is_cuda() && c.device.index() == c10::hip::current_device() && D > 0 &&
               B > 0 && tb->scalar_type() == at::kInt && tb->device() == c.device && (W <= 1 || tb->stride(1) == 1) && ld >= W;
        if (!c.ok) return;
        k = rows_of(c, k_cache, {pages, page, Hkv, D}, at.k_cache);
        v = rows_of(c, v_cache, {pages, page, Hkv, D}, at.v_cache);
        table = static_cast<const int32_t*>(tb->data_ptr());
        length = ints(c, len, {B});
        start = ints(c, q_start, {B + 1});
        c.ok = c.ok && (start || n % B == 0);
    }
};

// paged_attn(q, k_cache, v_cache, table, length, q_start, o, lse, scale, max_chunk, want_lse, ws)
PyObject* paged_attn(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(12);
    Call c(false);
    Paged p;
    p.of(c, x[0], x[1], x[2], x[3], x[4], x[5]);
    if (!c.ok) Py_RETURN_NOTIMPLEMENTED;
    const void* q = rows_of(c, x[0], {p.n, p.heads, p.D}, p.at.q);
    Result o(c, x[6], true, c.dtype, {p.n, p.heads, p.D}), lse(c, x[7], c.truth(x[10]), at::kFloat, {p.n, p.heads});
    const float scale = x[8] == Py_None ? float(1.0 / std::sqrt(double(p.D))) : c.number(x[8]);
    const int64_t most = x[9] == Py_None ? 0 : c.integer(x[9]);
    size_t wb = 0;
    void* ws = c.workspace(x[11], wb);
    const size_t make = c.ok && !ws ? g_lib.workspace_size_paged(p.n, p.B, p.heads, p.Hkv, p.D, p.start ? most : p.n / p.B) : 0;
    return run_results(c, "rlcs_paged_attn", {&o, &lse}, make, [&](rlcs_stream_t s, void* made) {
        return g_lib.paged_attn(q, p.k, p.v, p.table, p.length, p.start, o.ptr, lse.f32(), p.n, p.B, p.W, p.ld, p.pages, p.page, p.heads, p.Hkv, p.D, most,
                                &p.at, scale, c.type(), made ? made : ws, made ? make : wb, s);
    });
}

// paged_write(k, v, k_cache, v_cache, table, length, q_start)
PyObject* paged_write(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(7);
    Call c(false);
    Paged p;
    p.of(c, x[0], x[2], x[3], x[4], x[5], x[6]);
    if (!c.ok || p.heads != p.Hkv) Py_RETURN_NOTIMPLEMENTED;
    const void *k = rows_of(c, x[0], {p.n, p.Hkv, p.D}, p.at.k_new), *v = rows_of(c, x[1], {p.n, p.Hkv, p.D}, p.at.v_new);
    InPlace to_k(c, x[2], p.k), to_v(c, x[3], p.v);
    return run_results(c, "rlcs_paged_write", {&to_k, &to_v}, 0, [&](rlcs_stream_t s, void*) {
        return g_lib.paged_write(k, v, p.k, p.v, p.table, p.length, p.start, p.n, p.B, p.W, p.ld, p.pages, p.page, p.Hkv, p.D, &p.at, c.type(), s);
    });
}

// Table and references of the calls on pages.
struct Pages {
    int64_t B = 0, W = 0, pages = 0;
    const int32_t *table = nullptr, *refs = nullptr;

    Pages(Call& c, PyObject* t, PyObject* r) {
        const at::Tensor *tb = c.plain(t), *rf = c.plain(r);
        c.ok = c.ok && tb && rf && tb->dim() == 2 && rf->dim() == 1 && tb->device().is_cuda() && tb->device().index() == c10::hip::current_device();
        if (!c.ok) return;
        c.device = tb->device();
        B = tb->size(0); W = tb->size(1); pages = rf->size(0);
        c.ok = B > 0 && W > 0 && pages > 0;
        table = ints(c, t, {B, W});
        refs = ints(c, r, {pages});
    }
};

// pages_fork(table, length, refs, parent, table_out, length_out, refs_out, page, ws)
PyObject* pages_fork(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(9);
    if (x[1] == Py_None || x[3] == Py_None) Py_RETURN_NOTIMPLEMENTED;
    Call c(false);
    const Pages p(c, x[0], x[2]);
    const int32_t *length = ints(c, x[1], {p.B}), *parent = ints(c, x[3], {p.B});
    Result table(c, x[4], true, at::kInt, {p.B, p.W}), out(c, x[5], true, at::kInt, {p.B}), refs(c, x[6], true, at::kInt, {p.pages});
    const int64_t page = c.integer(x[7]);
    size_t wb = 0;
    void* ws = c.workspace(x[8], wb);
    const size_t make = c.ok && !ws ? g_lib.workspace_size_pages(p.B, p.pages) : 0;
    return run_results(c, "rlcs_pages_fork", {&table, &out, &refs}, make, [&](rlcs_stream_t s, void* made) {
        return g_lib.pages_fork(p.table, length, p.refs, parent, static_cast<int32_t*>(table.ptr), static_cast<int32_t*>(out.ptr),
                                static_cast<int32_t*>(refs.ptr), p.B, p.W, p.pages, page, made ? made : ws, made ? make : wb, s);
    });
}

// pages_resize(table, length, refs, new_length, table_out, length_out, refs_out, moves, page, ws)
PyObject* pages_resize(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(10);
    if (x[1] == Py_None || x[3] == Py_None) Py_RETURN_NOTIMPLEMENTED;
    Call c(false);
    const Pages p(c, x[0], x[2]);
    const int32_t *length = ints(c, x[1], {p.B}), *wanted = ints(c, x[3], {p.B});
    Result table(c, x[4], true, at::kInt, {p.B, p.W}), out(c, x[5], true, at::kInt, {p.B}), refs(c, x[6], true, at::kInt, {p.pages});
    Result moves(c, x[7], true, at::kInt, {p.B, 2});
    const int64_t page = c.integer(x[8]);
    size_t wb = 0;
    void* ws = c.workspace(x[9], wb);
    const size_t make = c.ok && !ws ? g_lib.workspace_size_pages(p.B, p.pages) : 0;
    return run_results(c, "rlcs_pages_resize", {&table, &out, &refs, &moves}, make, [&](rlcs_stream_t s, void* made) {
        return g_lib.pages_resize(p.table, length, p.refs, wanted, static_cast<int32_t*>(table.ptr), static_cast<int32_t*>(out.ptr),
                                  static_cast<int32_t*>(refs.ptr), static_cast<int32_t*>(moves.ptr), p.B, p.W, p.pages, page, made ? made : ws,
                                  made ? make : wb, s);
    });
}

// pages_compact(table, refs, table_out, refs_out, moves, count, ws)
PyObject* pages_compact(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(7);
    Call c(false);
    const Pages p(c, x[0], x[1]);
    Result table(c, x[2], true, at::kInt, {p.B, p.W}), refs(c, x[3], true, at::kInt, {p.pages}), moves(c, x[4], true, at::kInt, {p.pages / 2, 2});
    Result count(c, x[5], true, at::kInt, {1});
    size_t wb = 0;
    void* ws = c.workspace(x[6], wb);
    const size_t make = c.ok && !ws ? g_lib.workspace_size_pages(p.B, p.pages) : 0;
    return run_results(c, "rlcs_pages_compact", {&table, &refs, &moves, &count}, make, [&](rlcs_stream_t s, void* made) {
        return g_lib.pages_compact(p.table, p.refs, static_cast<int32_t*>(table.ptr), static_cast<int32_t*>(refs.ptr), static_cast<int32_t*>(moves.ptr),
                                   static_cast<int32_t*>(count.ptr), p.B, p.W, p.pages, made ? made : ws, made ? make : wb, s);
    });
}

// pages_copy(cache, moves)
PyObject* pages_copy(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(2);
    Call c(false);
    const at::Tensor *t = c.plain(x[0]), *m = c.plain(x[1]);
    if (!c.ok || !t || !m || t->dim() < 3 || m->dim() != 2 || !t->device().is_cuda() || t->device().index() != c10::hip::current_device())
        Py_RETURN_NOTIMPLEMENTED;
    c.device = t->device();
    const int64_t es = t->element_size(), layers = t->size(0), pages = t->size(1), n = m->size(0);
    int64_t size = es;
    for (int64_t i = t->dim() - 1; i >= 2; --i) {  // a page's contents are contiguous
        c.ok = c.ok && (t->size(i) <= 1 || t->stride(i) * es == size);
        size *= t->size(i);
    }
    if (t->numel() == 0) Py_RETURN_NOTIMPLEMENTED;
    const int32_t* moves = ints(c, x[1], {n, 2});
    if (!c.ok) Py_RETURN_NOTIMPLEMENTED;
    InPlace cache(c, x[0], t->data_ptr());
    PyObject* one = run_results(c, "rlcs_pages_copy", {&cache}, 0, [&](rlcs_stream_t s, void*) {
        return g_lib.pages_copy(cache.ptr, moves, n, layers, pages, layers > 1 ? t->stride(0) * es : 0, pages > 1 ? t->stride(1) * es : 0, size, s);
    });
    if (!one || one == Py_NotImplemented) return one;
    PyObject* o = PyTuple_GET_ITEM(one, 0);
    Py_INCREF(o);
    Py_DECREF(one);
    return o;
}

// verify_draft(target, draft, draft_tokens, u, noise, n_draft, tokens, count, logp, temperature, draft_temperature, want_logp, ws)
PyObject* verify_draft(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(13);
    if (x[2] == Py_None || x[3] == Py_None || x[4] == Py_None) Py_RETURN_NOTIMPLEMENTED;
    Call c(false);
    const at::Tensor* t = c.plain(x[0]);
    if (!c.ok || !t || t->dim() != 3 || t->size(1) < 1 || t->size(2) < 1) Py_RETURN_NOTIMPLEMENTED;
    c.dtype = t->scalar_type();
    c.device = t->device();
    c.ok = (c.dtype == at::kFloat || c.dtype == at::kBFloat16) && c.device.is_cuda() && c.device.index() == c10::hip::current_device();
    const int64_t B = t->size(0), K = t->size(1) - 1, V = t->size(2);
    int64_t ts[2] = {}, ds[2] = {}, ns = 0;
    auto operand = [&](PyObject* o, int64_t rows, int64_t* s) -> const void* {
        const at::Tensor* r = c.plain(o);
        if (!r) return nullptr;
        c.ok = c.ok && r->scalar_type() == c.dtype && r->device() == c.device && r->sizes() == at::IntArrayRef({B, rows, V}) && (V <= 1 || r->stride(2) == 1);
        if (!c.ok) return nullptr;
        s[0] = r->stride(0);
        s[1] = r->stride(1);
        return r->data_ptr();
    };
    const void *target = operand(x[0], K + 1, ts), *draft = operand(x[1], K, ds);
    const int32_t* drawn = ints(c, x[2], {B, K});
    const float* u = static_cast<float*>(c.checked(x[3], at::kFloat, {B, K}, false));
    Rows like;
    like.V = V;
    like.lead = {B};
    const float* noise = static_cast<float*>(rows_beside(c, x[4], at::kFloat, like, ns));
    const int32_t* n_draft = ints(c, x[5], {B});
    Result tokens(c, x[6], true, at::kInt, {B, K + 1}), count(c, x[7], true, at::kInt, {B}), logp(c, x[8], c.truth(x[11]), at::kFloat, {B, K + 1});
    float all[2] = {0.f, 0.f};
    const float* own[2] = {nullptr, nullptr};
    for (int i = 0; i < 2; ++i) {
        if (THPVariable_CheckExact(x[9 + i])) own[i] = static_cast<float*>(c.checked(x[9 + i], at::kFloat, {B}, false));
        else all[i] = c.number(x[9 + i]);
    }
    size_t wb = 0;
    void* ws = c.workspace(x[12], wb);
    const size_t make = c.ok && !ws ? g_lib.workspace_size_verify(B, K, V) : 0;
    return run_results(c, "rlcs_verify_draft", {&tokens, &count, &logp}, make, [&](rlcs_stream_t s, void* made) {
        return g_lib.verify_draft(target, draft, drawn, u, noise, n_draft, own[0], own[1], static_cast<int32_t*>(tokens.ptr),
                                  static_cast<int32_t*>(count.ptr), logp.f32(), B, K, V, ts[0], ts[1], ds[0], ds[1], ns, all[0], all[1], c.type(),
                                  made ? made : ws, made ? make : wb, s);
    });
}

// distill_loss(logits, top_ids, top_logp, weight, loss, dlogits, temperature, tail, want_grad)
PyObject* distill_loss(Argv x, Py_ssize_t nargs) {
    RLCS_ARGS(9);
    if (x[1] == Py_None || x[2] == Py_None) Py_RETURN_NOTIMPLEMENTED;
    Call c(false);
    Rows r;
    void* logits = rows_input(c, x[0], r);
    const at::Tensor* t = c.plain(x[1]);
    if (!c.ok || !t || t->dim() != int64_t(r.lead.size()) + 1) Py_RETURN_NOTIMPLEMENTED;
    std::vector<int64_t> listed = r.lead, full = r.lead;
    listed.push_back(t->size(-1));
    full.push_back(r.V);
    const int32_t* ids = ints(c, x[1], listed);
    const float* top = static_cast<float*>(c.checked(x[2], at::kFloat, listed, false));
    const float* weight = static_cast<float*>(c.checked(x[3], at::kFloat, r.lead, false));
    Result loss(c, x[4], true, at::kFloat, r.lead), grad(c, Py_None, c.truth(x[8]), c.dtype, full);
    int64_t ld_grad = r.V;
    if (x[5] != Py_None) {  // rows of its own stride
        grad.make = false;
        grad.given = x[5];
        grad.ptr = rows_beside(c, x[5], c.dtype, r, ld_grad);
    }
    const float temperature = c.number(x[6]);
    const int tail = c.truth(x[7]) ? 1 : 0;
    return run_results(c, "rlcs_distill_loss", {&loss, &grad}, 0, [&](rlcs_stream_t s, void*) {
        return g_lib.distill_loss(logits, ids, top, weight, loss.f32(), grad.ptr, r.M, r.V, listed.back(), r.ld, ld_grad, temperature, tail, c.type(), s);
    });
}

// bind(handle, error, device): the dlopen handle of librlcs.so, the exception class of its status
// codes and the class of torch's default-device mode
PyObject* bind(PyObject*, PyObject* args) {
    unsigned long long handle = 0;
    PyObject *error = nullptr, *device = nullptr;
    if (!PyArg_ParseTuple(args, "KOO", &handle, &error, &device)) return nullptr;
    void* h = reinterpret_cast<void*>(handle);
    bool all = true;
    auto get = [&](auto& fn, const char* name) {
        fn = reinterpret_cast<std::decay_t<decltype(fn)>>(dlsym(h, name));
        all = all && fn;
    };
    get(g_lib.gae, "rlcs_gae");
    get(g_lib.vtrace, "rlcs_vtrace");
    get(g_lib.retrace, "rlcs_retrace");
    get(g_lib.retrace_full, "rlcs_retrace_full");
    get(g_lib.td_lambda, "rlcs_td_lambda");
    get(g_lib.discounted, "rlcs_discounted");
    get(g_lib.elig_trace, "rlcs_elig_trace");
    get(g_lib.episodic_prefix, "rlcs_episodic_prefix");
    get(g_lib.affine_scan, "rlcs_affine_scan");
    get(g_lib.gae_strided, "rlcs_gae_strided");
    get(g_lib.vtrace_strided, "rlcs_vtrace_strided");
    get(g_lib.retrace_strided, "rlcs_retrace_strided");
    get(g_lib.td_lambda_strided, "rlcs_td_lambda_strided");
    get(g_lib.discounted_strided, "rlcs_discounted_strided");
    get(g_lib.elig_trace_strided, "rlcs_elig_trace_strided");
    get(g_lib.episodic_prefix_strided, "rlcs_episodic_prefix_strided");
    get(g_lib.elig_trace_vec, "rlcs_elig_trace_vec");
    get(g_lib.gae_masked, "rlcs_gae_masked");
    get(g_lib.gae_masked_noalloc, "rlcs_gae_masked_noalloc");
    get(g_lib.token_logp, "rlcs_token_logp");
    get(g_lib.policy_loss, "rlcs_policy_loss");
    get(g_lib.sample, "rlcs_sample");
    get(g_lib.workspace_size_sample, "rlcs_workspace_size_sample");
    get(g_lib.shared_prefix_attn, "rlcs_shared_prefix_attn");
    get(g_lib.workspace_size_attn, "rlcs_workspace_size_attn");
    get(g_lib.paged_attn, "rlcs_paged_attn");
    get(g_lib.workspace_size_paged, "rlcs_workspace_size_paged");
    get(g_lib.paged_write, "rlcs_paged_write");
    get(g_lib.pages_fork, "rlcs_pages_fork");
    get(g_lib.pages_resize, "rlcs_pages_resize");
    get(g_lib.pages_compact, "rlcs_pages_compact");
    get(g_lib.workspace_size_pages, "rlcs_workspace_size_pages");
    get(g_lib.pages_copy, "rlcs_pages_copy");
    get(g_lib.verify_draft, "rlcs_verify_draft");
    get(g_lib.workspace_size_verify, "rlcs_workspace_size_verify");
    get(g_lib.distill_loss, "rlcs_distill_loss");
    if (!all) {
        PyErr_SetString(PyExc_RuntimeError, "librlcs.so lacks a function of the binding");
        return nullptr;
    }
    Py_INCREF(error);
    Py_XSETREF(g_error, error);
    Py_INCREF(device);
    Py_XSETREF(g_device, device);
    g_bound = true;
    Py_RETURN_NONE;
}

template <PyObject* (*F)(Argv, Py_ssize_t)>
PyMethodDef fast(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<F>)), METH_FASTCALL, nullptr};
}

PyMethodDef g_methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    fast<gae<false>>("gae"), fast<gae<true>>("gae_strided"),
    fast<vtrace<false>>("vtrace"), fast<vtrace<true>>("vtrace_strided"),
    fast<retrace<false>>("retrace"), fast<retrace<true>>("retrace_strided"),
    fast<retrace_full>("retrace_full"),
    fast<td_lambda<false>>("td_lambda"), fast<td_lambda<true>>("td_lambda_strided"),
    fast<discounted<false>>("discounted"), fast<discounted<true>>("discounted_strided"),
    fast<elig_trace<false>>("elig_trace"), fast<elig_trace<true>>("elig_trace_strided"),
    fast<episodic_prefix<false>>("episodic_prefix"), fast<episodic_prefix<true>>("episodic_prefix_strided"),
    fast<affine_scan>("affine_scan"), fast<elig_trace_vec>("elig_trace_vec"), fast<gae_masked>("gae_masked"),
    fast<token_logp>("token_logp"), fast<policy_loss>("policy_loss"), fast<sample>("sample"),
    fast<shared_prefix_attn>("shared_prefix_attn"), fast<paged_attn>("paged_attn"), fast<paged_write>("paged_write"),
    fast<pages_fork>("pages_fork"), fast<pages_resize>("pages_resize"), fast<pages_compact>("pages_compact"),
    fast<pages_copy>("pages_copy"), fast<verify_draft>("verify_draft"), fast<distill_loss>("distill_loss"),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&g_module); }
