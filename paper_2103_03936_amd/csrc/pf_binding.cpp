// The layers' calls from Python: argument checks, output tensors, workspace and the call into libpufferfish.so, natively.
// A small layer's kernels take 10 to 20 us; marshalling its arguments in Python (ctypes, torch.empty, current_stream)
// took 10 us forward and 15 us backward on top and bounded every small call.  Here a call costs its outputs' allocations and
// the launches.  Nothing is computed here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <map>
#include <mutex>
#include <string>
#include <utility>
#include <vector>

#include "../../include/pufferfish.h"

namespace {

PyObject *g_error = nullptr, *g_no_memory = nullptr; // the package's PfError, torch.OutOfMemoryError

struct Fail { // a Python exception to raise
    PyObject *type;
    std::string what;
};
[[noreturn]] void fail(const std::string &what) { throw Fail{g_error, what}; }

using at::Tensor;
constexpr auto F32 = at::kFloat;
constexpr auto ANY = at::ScalarType::Undefined;

const Tensor &tensor(PyObject *o)
{
    if (!THPVariable_Check(o)) throw Fail{PyExc_TypeError, "expected a tensor"};
    return THPVariable_Unpack(o);
}
void *address(const Tensor &t, at::ScalarType want)
{
    if (!t.is_cuda()) fail("tensors must live on the GPU; there is no CPU path");
    if (!t.is_contiguous()) fail("tensors must be contiguous");
    if (want != ANY && t.scalar_type() != want)
        fail(std::string("expected ") + c10::toString(want) + ", got " + c10::toString(t.scalar_type()));
    return t.data_ptr();
}
void *ptr(PyObject *o, at::ScalarType want = ANY) { return o == Py_None ? nullptr : address(tensor(o), want); }

int dtype_code(const Tensor &t)
{
    if (t.scalar_type() == at::kFloat) return PF_F32;
    if (t.scalar_type() == at::kBFloat16) return PF_BF16;
    fail(std::string("unsupported dtype ") + c10::toString(t.scalar_type()));
}
void dims(const Tensor &t, int n, const char *name)
{
    if (t.dim() != n) throw Fail{PyExc_ValueError, std::string(name) + " must have " + std::to_string(n) + " dimensions"};
}

// An output tensor (owned by Python once given out)
struct Out {
    Tensor t;
    void *p = nullptr;
    Out() {}
    Out(at::IntArrayRef size, at::ScalarType type, const at::Device &dev)
    {
        if (!dev.is_cuda()) fail("tensors must live on the GPU; there is no CPU path");
        t = Tensor(at::detail::empty_cuda(size, type, dev, std::nullopt));
        p = t.data_ptr();
    }
    PyObject *give()
    {
        if (!t.defined()) Py_RETURN_NONE;
        return THPVariable_Wrap(std::move(t));
    }
};
PyObject *tuple(std::initializer_list<PyObject *> items)
{
    PyObject *t = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    for (PyObject *o : items) PyTuple_SET_ITEM(t, i++, o);
    return t;
}
PyObject *borrowed(PyObject *o)
{
    Py_INCREF(o);
    return o;
}
PyObject *give_or(Out &o, PyObject *given) { return given ? borrowed(given) : o.give(); }

void *stream() { return (void *)c10::hip::getCurrentHIPStream().stream(); }

void check(int status, const char *what)
{
    if (status != PF_OK)
        fail(std::string(what) + ": status " + std::to_string(status) + " (" + pf_status_string(status) + "), hip error " +
             std::to_string(pf_last_hip_error()));
}

// A reusable byte buffer per (device, stream): calls enqueued on one stream are ordered, so they may share scratch
// memory; calls on different streams get different buffers.  It grows and never shrinks; one that is outgrown is kept
// alive rather than freed, so that graphs captured through these calls stay valid when a later call needs more.  Every call
// of the package takes it from here, those that Python marshals through lend(), and holds it until its launches are
// enqueued: of two threads' calls on one stream the second's launches follow the first's.
struct Space {
    void *p;
    size_t n;
};
struct Scratch {
    std::recursive_mutex busy; // (recursive: a finalizer may run a call while its thread has the buffer lent)
    Tensor t;
    std::vector<Tensor> retired;
    Space get(size_t bytes, const at::Device &dev)
    {
        if (!t.defined() || (size_t)t.numel() < bytes) {
            if (t.defined()) retired.push_back(t);
            t = Tensor(at::detail::empty_cuda({(int64_t)(bytes < 256 ? 256 : bytes)}, at::kByte, dev, std::nullopt));
        }
        return Space{t.data_ptr(), (size_t)t.numel()};
    }
};
Scratch &scratch(const at::Device &dev)
{
    static std::mutex lock;
    static auto &all = *new std::map<std::pair<int, void *>, Scratch>; // (never destroyed: the allocator may be gone)
    std::lock_guard<std::mutex> hold(lock);
    return all[{dev.index(), (void *)c10::hip::getCurrentHIPStream(dev.index()).stream()}];
}

// The interpreter runs other threads meanwhile
struct NoGil {
    PyThreadState *state = PyEval_SaveThread();
    NoGil() {}
    NoGil(const NoGil &) = delete;
    ~NoGil() { PyEval_RestoreThread(state); }
};
// f(scratch memory): the call into the library, which touches no Python object
template <class F>
void call(const char *what, size_t bytes, const at::Device &dev, F f)
{
    if (!dev.is_cuda()) fail("tensors must live on the GPU; there is no CPU path");
    int status;
    {
        NoGil released;
        Scratch &s = scratch(dev);
        std::lock_guard<std::recursive_mutex> hold(s.busy);
        status = f(s.get(bytes, dev));
    }
    check(status, what);
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Fail{nullptr, ""};
    return v != 0;
}
long integer(PyObject *o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Fail{nullptr, ""};
    return v;
}

// (a number that an int does not hold is refused, not taken modulo 2^32)
int integer32(PyObject *o)
{
    const long v = integer(o);
    if (v != (int)v) throw Fail{PyExc_OverflowError, std::to_string(v) + " does not fit 32 bits"};
    return (int)v;
}

template <PyObject *(*F)(PyObject *const *), int N>
PyObject *entry(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        return F(a);
    } catch (const Fail &f) {
        if (f.type) PyErr_SetString(f.type, f.what.c_str());
    } catch (const c10::OutOfMemoryError &e) {
        PyErr_SetString(g_no_memory, e.what());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// An owned reference
struct Ref {
    PyObject *o;
    explicit Ref(PyObject *owned = nullptr) : o(owned) {}
    Ref(const Ref &) = delete;
    Ref(Ref &&r) : o(r.o) { r.o = nullptr; }
    ~Ref() { Py_XDECREF(o); }
};

// parameter gradients: new tensors, or those of a given sequence of n (accumulated into; None: not wanted)
struct Grads {
    Ref items; // a list or tuple, which keeps them
    PyObject *g[3] = {nullptr, nullptr, nullptr};
    Out o[3];
    void *p[3] = {nullptr, nullptr, nullptr};
    bool given;
    Grads(PyObject *grads, int n) : given(grads != Py_None)
    {
        if (!given) return;
        items.o = PySequence_Fast(grads, "grads must be a sequence");
        if (!items.o) throw Fail{nullptr, ""};
        const Py_ssize_t have = PySequence_Fast_GET_SIZE(items.o);
        if (have != n)
            throw Fail{PyExc_ValueError, "grads must hold " + std::to_string(n) + " entries, not " + std::to_string(have)};
        for (int i = 0; i < n; ++i) {
            g[i] = PySequence_Fast_GET_ITEM(items.o, i);
            p[i] = ptr(g[i], F32);
        }
    }
    void make(int i, at::IntArrayRef size, const at::Device &dev)
    {
        o[i] = Out(size, F32, dev);
        p[i] = o[i].p;
    }
    PyObject *give(int i) { return give_or(o[i], g[i]); }
};

// ------------------------------------------------------------------ linear
pf_linear_desc linear_desc(const Tensor &X, const Tensor &U, bool bias)
{
    dims(X, 2, "X");
    dims(U, 2, "U");
    pf_linear_desc d = {};
    d.M = X.size(0);
    d.in = X.size(1);
    d.out = U.size(0);
    d.r = U.size(1);
    d.dtype = dtype_code(X);
    d.wgrad_dtype = PF_F32;
    d.has_bias = bias;
    return d;
}

// X, V, U, bias, residual, act, save_T, with epilogue
PyObject *linear_fwd(PyObject *const *a)
{
    const Tensor &X = tensor(a[0]), &U = tensor(a[2]);
    const pf_linear_desc d = linear_desc(X, U, a[3] != Py_None);
    const auto dt = X.scalar_type();
    const auto dev = X.device();
    Out Y({d.M, d.out}, dt, dev), T;
    if (truth(a[6])) T = Out({d.M, d.r}, dt, dev);
    void *const p[5] = {ptr(a[0], dt), ptr(a[1], dt), ptr(a[2], dt), ptr(a[3], dt), ptr(a[4], dt)}, *const st = stream();
    const size_t need = pf_lowrank_linear_fwd_workspace_bytes(&d);
    const int act = (int)integer(a[5]);
    if (truth(a[7]))
        call("pf_lowrank_linear_fwd_ep", need, dev, [&](Space ws) {
            return pf_lowrank_linear_fwd_ep(&d, p[0], p[1], p[2], p[3], p[4], act, Y.p, T.p, ws.p, ws.n, st);
        });
    else
        call("pf_lowrank_linear_fwd", need, dev,
             [&](Space ws) { return pf_lowrank_linear_fwd(&d, p[0], p[1], p[2], p[3], Y.p, T.p, ws.p, ws.n, st); });
    return tuple({Y.give(), T.give()});
}

// X, V, U, dY, T_saved, dX_add, x_is_relu, need_dX, has_bias, grads, with epilogue
PyObject *linear_bwd(PyObject *const *a)
{
    const Tensor &X = tensor(a[0]), &U = tensor(a[2]);
    const pf_linear_desc d = linear_desc(X, U, truth(a[8]));
    const auto dt = X.scalar_type();
    const auto dev = X.device();
    Out dX;
    if (truth(a[7])) dX = Out(X.sizes(), dt, dev);
    Grads g(a[9], 3);
    if (!g.given) {
        g.make(0, {d.out, d.r}, dev);
        g.make(1, {d.in, d.r}, dev);
        if (d.has_bias) g.make(2, {d.out}, dev);
    }
    void *const p[6] = {ptr(a[0], dt), ptr(a[1], dt), ptr(a[2], dt), ptr(a[3], dt), ptr(a[4], dt), ptr(a[5], dt)}, *const st = stream();
    const size_t need = pf_lowrank_linear_bwd_workspace_bytes(&d);
    const bool relu = truth(a[6]);
    if (truth(a[10]))
        call("pf_lowrank_linear_bwd_ep", need, dev, [&](Space ws) {
            return pf_lowrank_linear_bwd_ep(&d, p[0], p[1], p[2], p[3], p[4], p[5], relu, dX.p, g.p[0], g.p[1], g.p[2], g.given, ws.p, ws.n, st);
        });
    else
        call("pf_lowrank_linear_bwd", need, dev, [&](Space ws) {
            return pf_lowrank_linear_bwd(&d, p[0], p[1], p[2], p[3], p[4], dX.p, g.p[0], g.p[1], g.p[2], g.given, ws.p, ws.n, st);
        });
    return tuple({dX.give(), g.give(0), g.give(1), g.give(2)});
}

pf_linear_shared_desc shared_desc(const Tensor &X, const Tensor &U, bool bias)
{
    dims(X, 2, "X");
    dims(U, 3, "U");
    pf_linear_shared_desc d = {};
    d.M = X.size(0);
    d.n_in = X.size(1);
    d.groups = (int)U.size(0);
    d.n_out = U.size(1);
    d.r = U.size(2);
    d.dtype = dtype_code(X);
    d.has_bias = bias;
    return d;
}

// X, V, U, bias, save_T
PyObject *shared_fwd(PyObject *const *a)
{
    const Tensor &X = tensor(a[0]), &U = tensor(a[2]);
    const pf_linear_shared_desc d = shared_desc(X, U, a[3] != Py_None);
    const auto dt = X.scalar_type();
    const auto dev = X.device();
    Out Y({d.groups, d.M, d.n_out}, dt, dev), T;
    if (truth(a[4])) T = Out({d.groups, d.M, d.r}, dt, dev);
    void *const p[4] = {ptr(a[0]), ptr(a[1], dt), ptr(a[2], dt), ptr(a[3], dt)}, *const st = stream();
    call("pf_lowrank_linear_shared_fwd", pf_lowrank_linear_shared_fwd_workspace_bytes(&d), dev,
         [&](Space ws) { return pf_lowrank_linear_shared_fwd(&d, p[0], p[1], p[2], p[3], Y.p, T.p, ws.p, ws.n, st); });
    return tuple({Y.give(), T.give()});
}

// X, V, U, dY, T_saved, need_dX, has_bias, grads
PyObject *shared_bwd(PyObject *const *a)
{
    const Tensor &X = tensor(a[0]), &V = tensor(a[1]), &U = tensor(a[2]);
    const pf_linear_shared_desc d = shared_desc(X, U, truth(a[6]));
    const auto dt = X.scalar_type();
    const auto dev = X.device();
    Out dX;
    if (truth(a[5])) dX = Out(X.sizes(), dt, dev);
    Grads g(a[7], 3);
    if (!g.given) {
        g.make(0, U.sizes(), dev);
        g.make(1, V.sizes(), dev);
        if (d.has_bias) g.make(2, {d.groups, d.n_out}, dev);
    }
    void *const p[5] = {ptr(a[0]), ptr(a[1], dt), ptr(a[2], dt), ptr(a[3], dt), ptr(a[4], dt)}, *const st = stream();
    call("pf_lowrank_linear_shared_bwd", pf_lowrank_linear_shared_bwd_workspace_bytes(&d), dev, [&](Space ws) {
        return pf_lowrank_linear_shared_bwd(&d, p[0], p[1], p[2], p[3], p[4], dX.p, g.p[0], g.p[1], g.p[2], g.given, ws.p, ws.n, st);
    });
    return tuple({dX.give(), g.give(0), g.give(1), g.give(2)});
}

// ------------------------------------------------------------------ convolution
pf_conv_desc conv_desc(const Tensor &X, const Tensor &Uk, const Tensor &Vp, long stride, long pad)
{
    dims(X, 4, "X");
    dims(Uk, 4, "Uk");
    pf_conv_desc d = {};
    d.N = X.size(0);
    d.Cin = X.size(1);
    d.H = X.size(2);
    d.W = X.size(3);
    d.Cout = Vp.size(0);
    d.r = Uk.size(0);
    d.k = (int)Uk.size(2);
    d.stride = (int)stride;
    d.pad = (int)pad;
    d.layout = PF_NCHW;
    d.dtype = dtype_code(X);
    d.wgrad_dtype = PF_F32;
    return d;
}

// X, Uk, Vp, scale, shift, residual, act, stride, pad, save_T, save_W, with epilogue
PyObject *conv_fwd(PyObject *const *a)
{
    const Tensor &X = tensor(a[0]), &Uk = tensor(a[1]), &Vp = tensor(a[2]);
    const long stride_ = integer(a[7]), pad = integer(a[8]);
    if (stride_ <= 0) fail("stride must be positive");
    const pf_conv_desc d = conv_desc(X, Uk, Vp, stride_, pad);
    const int64_t Ho = (d.H + 2 * pad - d.k) / d.stride + 1, Wo = (d.W + 2 * pad - d.k) / d.stride + 1;
    const auto dt = X.scalar_type();
    const auto dev = X.device();
    const bool save_W = truth(a[10]);
    Out Y({d.N, d.Cout, Ho, Wo}, dt, dev), T, W;
    if (truth(a[9])) T = Out({d.N, d.r, Ho, Wo}, dt, dev);
    const size_t nW = save_W ? pf_lowrank_conv_saved_weights_bytes(&d) : 0;
    if (nW) W = Out({(int64_t)nW}, at::kByte, dev);
    void *const p[6] = {ptr(a[0], dt), ptr(a[1], dt), ptr(a[2], dt), ptr(a[3], F32), ptr(a[4], F32), ptr(a[5], dt)}, *const st = stream();
    const size_t need = pf_lowrank_conv_fwd_workspace_bytes(&d);
    const int act = (int)integer(a[6]);
    if (truth(a[11]))
        call("pf_lowrank_conv_fwd_ep", need, dev, [&](Space ws) {
            return pf_lowrank_conv_fwd_ep(&d, p[0], p[1], p[2], p[3], p[4], p[5], act, Y.p, T.p, W.p, ws.p, ws.n, st);
        });
    else
        call("pf_lowrank_conv_fwd", need, dev,
             [&](Space ws) { return pf_lowrank_conv_fwd(&d, p[0], p[1], p[2], Y.p, T.p, W.p, ws.p, ws.n, st); });
    return save_W ? tuple({Y.give(), T.give(), W.give()}) : tuple({Y.give(), T.give()});
}

// X, Uk, Vp, scale, dZ, T_saved, stride, pad, dX_add, x_is_relu, need_dX, need_dshift, grads, W_saved, with epilogue
PyObject *conv_bwd(PyObject *const *a)
{
    const Tensor &X = tensor(a[0]), &Uk = tensor(a[1]), &Vp = tensor(a[2]);
    const pf_conv_desc d = conv_desc(X, Uk, Vp, integer(a[6]), integer(a[7]));
    const auto dt = X.scalar_type();
    const auto dev = X.device();
    const bool ep = truth(a[14]);
    Out dX;
    if (truth(a[10])) dX = Out(X.sizes(), dt, dev);
    Grads g(a[12], ep ? 3 : 2);
    if (!g.given) {
        g.make(0, Uk.sizes(), dev);
        g.make(1, Vp.sizes(), dev);
        if (ep && truth(a[11])) g.make(2, {d.Cout}, dev);
    }
    void *const p[6] = {ptr(a[0], dt), ptr(a[1], dt), ptr(a[2], dt), ptr(a[4], dt), ptr(a[5], dt), ptr(a[13])}, *const st = stream();
    if (ep) {
        void *const scale = ptr(a[3], F32), *const add = ptr(a[8], dt);
        const bool relu = truth(a[9]);
        call("pf_lowrank_conv_bwd_ep", pf_lowrank_conv_bwd_ep_workspace_bytes(&d), dev, [&](Space ws) {
            return pf_lowrank_conv_bwd_ep(&d, p[0], p[1], p[2], scale, p[3], p[4], p[5], add, relu, dX.p, g.p[0], g.p[1], g.p[2], g.given,
                                          ws.p, ws.n, st);
        });
        return tuple({dX.give(), g.give(0), g.give(1), g.give(2)});
    }
    call("pf_lowrank_conv_bwd", pf_lowrank_conv_bwd_workspace_bytes(&d), dev, [&](Space ws) {
        return pf_lowrank_conv_bwd(&d, p[0], p[1], p[2], p[3], p[4], p[5], dX.p, g.p[0], g.p[1], g.given, ws.p, ws.n, st);
    });
    return tuple({dX.give(), g.give(0), g.give(1)});
}

// ------------------------------------------------------------------ LSTM
const char *const GRAD_NAMES[5] = {"dVx", "dUx", "dVh", "dUh", "dbias"};

// The five parameter gradients of a layer: a given dict's tensors, or new ones in a new dict
struct LstmGrads {
    Ref dict, items[5];
    void *p[5];
    LstmGrads(PyObject *given, const Tensor &Vx, const Tensor &Ux, const Tensor &Vh, const Tensor &Uh, int64_t h)
    {
        if (given != Py_None) {
            dict.o = borrowed(given);
            for (int i = 0; i < 5; ++i) {
                items[i].o = PyMapping_GetItemString(given, GRAD_NAMES[i]);
                if (!items[i].o) throw Fail{nullptr, ""};
                p[i] = ptr(items[i].o, F32);
            }
            return;
        }
        dict.o = PyDict_New();
        const at::IntArrayRef sizes[4] = {Vx.sizes(), Ux.sizes(), Vh.sizes(), Uh.sizes()};
        for (int i = 0; i < 5; ++i) {
            const int64_t nb[1] = {4 * h};
            Out o(i < 4 ? sizes[i] : at::IntArrayRef(nb), F32, Vx.device());
            p[i] = o.p;
            PyObject *t = o.give();
            PyDict_SetItemString(dict.o, GRAD_NAMES[i], t);
            Py_DECREF(t);
        }
    }
    LstmGrads(LstmGrads &&) = default;
    PyObject *give() { return std::exchange(dict.o, nullptr); }
};

pf_lstm_desc cell_desc(const Tensor &x, const Tensor &h, const Tensor &Ux, long groups, bool bias)
{
    dims(x, 2, "x");
    pf_lstm_desc d = {};
    d.B = x.size(0);
    d.d_in = x.size(1);
    d.h = h.size(1);
    d.r = Ux.size(1);
    d.groups = (int)groups;
    d.dtype = dtype_code(x);
    d.has_bias = bias;
    return d;
}

// x, h_prev, c_prev, Vx, Ux, Vh, Uh, bias, groups
PyObject *cell_fwd(PyObject *const *a)
{
    const Tensor &x = tensor(a[0]);
    const pf_lstm_desc d = cell_desc(x, tensor(a[1]), tensor(a[4]), integer(a[8]), a[7] != Py_None);
    const auto dev = x.device();
    const int64_t gr = d.groups * d.r;
    Out h({d.B, d.h}, F32, dev), c({d.B, d.h}, F32, dev), g({d.B, 4 * d.h}, F32, dev), Tx({d.B, gr}, F32, dev),
        Th({d.B, gr}, F32, dev);
    void *p[8], *const st = stream();
    for (int i = 0; i < 8; ++i) p[i] = ptr(a[i], F32);
    call("pf_lowrank_lstm_cell_fwd", pf_lowrank_lstm_cell_fwd_workspace_bytes(&d), dev, [&](Space ws) {
        return pf_lowrank_lstm_cell_fwd(&d, p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], h.p, c.p, g.p, Tx.p, Th.p, ws.p, ws.n, st);
    });
    return tuple({h.give(), c.give(), g.give(), Tx.give(), Th.give()});
}

// x, h_prev, c_prev, c_out, gates, Tx, Th, Vx, Ux, Vh, Uh, dh, dc_next, groups, need_dx, grads
PyObject *cell_bwd(PyObject *const *a)
{
    const Tensor &x = tensor(a[0]), &hp = tensor(a[1]);
    const pf_lstm_desc d = cell_desc(x, hp, tensor(a[8]), integer(a[13]), true);
    const auto dev = x.device();
    Out dx, dh(hp.sizes(), F32, dev), dc(tensor(a[2]).sizes(), F32, dev);
    if (truth(a[14])) dx = Out(x.sizes(), F32, dev);
    LstmGrads g(a[15], tensor(a[7]), tensor(a[8]), tensor(a[9]), tensor(a[10]), d.h);
    void *p[13], *const st = stream();
    for (int i = 0; i < 13; ++i) p[i] = ptr(a[i], F32);
    const bool given = a[15] != Py_None;
    call("pf_lowrank_lstm_cell_bwd", pf_lowrank_lstm_cell_bwd_workspace_bytes(&d), dev, [&](Space ws) {
        return pf_lowrank_lstm_cell_bwd(&d, p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], p[10], p[11], p[12], dx.p, dh.p,
                                        dc.p, g.p[0], g.p[1], g.p[2], g.p[3], g.p[4], given, ws.p, ws.n, st);
    });
    return tuple({dx.give(), dh.give(), dc.give(), g.give()});
}

// A list with one tensor (or None) per layer and the host array of its pointers
struct Layers {
    PyObject *seq = nullptr;
    std::vector<Tensor> keep; // (another thread may change the list during the call)
    std::vector<void *> p;
    bool present;
    explicit Layers(PyObject *o, at::ScalarType want = F32) : present(o != Py_None)
    {
        if (!present) return;
        seq = PySequence_Fast(o, "expected a list with one tensor per layer");
        if (!seq) throw Fail{nullptr, ""};
        for (Py_ssize_t i = 0; i < size(); ++i) {
            PyObject *t = PySequence_Fast_GET_ITEM(seq, i);
            p.push_back(ptr(t, want));
            if (t != Py_None) keep.push_back(tensor(t));
        }
    }
    Layers(const Layers &) = delete;
    ~Layers() { Py_XDECREF(seq); }
    Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(seq); }
    const Tensor &at(Py_ssize_t i) const { return tensor(PySequence_Fast_GET_ITEM(seq, i)); }
    template <class T>
    T *arr()
    {
        return present ? (T *)p.data() : nullptr;
    }
};
// One new tensor per layer
struct Outs {
    std::vector<Out> o;
    std::vector<void *> p;
    void add(at::IntArrayRef size, const at::Device &dev)
    {
        o.emplace_back(size, F32, dev);
        p.push_back(o.back().p);
    }
    PyObject *give()
    {
        PyObject *l = PyList_New((Py_ssize_t)o.size());
        for (size_t i = 0; i < o.size(); ++i) PyList_SET_ITEM(l, (Py_ssize_t)i, o[i].give());
        return l;
    }
};

pf_lstm_stack_desc stack_desc(const Tensor &x, const Layers &h0, const Layers &Ux, long groups, bool bias)
{
    dims(x, 3, "x");
    pf_lstm_stack_desc d = {};
    if (Ux.size() == 0 || h0.size() < Ux.size()) throw Fail{PyExc_ValueError, "one tensor per layer is wanted"};
    d.T = x.size(0);
    d.B = x.size(1);
    d.d_in = x.size(2);
    d.h = h0.at(0).size(1);
    d.r = Ux.at(0).size(1);
    d.groups = (int)groups;
    d.layers = (int)Ux.size();
    d.dtype = dtype_code(x);
    d.has_bias = bias;
    return d;
}
void per_layer(const pf_lstm_stack_desc &d, std::initializer_list<const Layers *> ls)
{
    for (const Layers *l : ls)
        if (l->present && l->size() < d.layers) throw Fail{PyExc_ValueError, "one tensor per layer is wanted"};
}

// x, h0, c0, Vx, Ux, Vh, Uh, bias, groups
PyObject *stack_fwd(PyObject *const *a)
{
    const Tensor &x = tensor(a[0]);
    Layers h0(a[1]), c0(a[2]), Vx(a[3]), Ux(a[4]), Vh(a[5]), Uh(a[6]), bias(a[7]);
    const pf_lstm_stack_desc d = stack_desc(x, h0, Ux, integer(a[8]), bias.present);
    per_layer(d, {&h0, &c0, &Vx, &Ux, &Vh, &Uh, &bias});
    const auto dev = x.device();
    const int64_t n[5] = {d.h, d.h, 4 * d.h, d.groups * d.r, d.groups * d.r};
    Outs o[5];
    for (int i = 0; i < 5; ++i)
        for (int l = 0; l < d.layers; ++l) o[i].add({d.T, d.B, n[i]}, dev);
    void *const px = ptr(a[0], F32), *const st = stream();
    call("pf_lowrank_lstm_stack_fwd", pf_lowrank_lstm_stack_fwd_workspace_bytes(&d), dev, [&](Space ws) {
        return pf_lowrank_lstm_stack_fwd(&d, px, h0.arr<const void *>(), c0.arr<const void *>(), Vx.arr<const void *>(),
                                         Ux.arr<const void *>(), Vh.arr<const void *>(), Uh.arr<const void *>(),
                                         bias.arr<const void *>(), o[0].p.data(), o[1].p.data(), o[2].p.data(), o[3].p.data(),
                                         o[4].p.data(), ws.p, ws.n, st);
    });
    return tuple({o[0].give(), o[1].give(), o[2].give(), o[3].give(), o[4].give()});
}

// x, h0, c0, h_all, c_all, gates_all, Tx_all, Th_all, Vx, Ux, Vh, Uh, dh_top, dhT, dcT, groups, need_dx, grads
PyObject *stack_bwd(PyObject *const *a)
{
    const Tensor &x = tensor(a[0]);
    Layers h0(a[1]), c0(a[2]), h(a[3]), c(a[4]), g(a[5]), Tx(a[6]), Th(a[7]), Vx(a[8]), Ux(a[9]), Vh(a[10]), Uh(a[11]),
        dhT(a[13]), dcT(a[14]);
    const pf_lstm_stack_desc d = stack_desc(x, h0, Ux, integer(a[15]), true);
    per_layer(d, {&h0, &c0, &h, &c, &g, &Tx, &Th, &Vx, &Ux, &Vh, &Uh, &dhT, &dcT});
    const auto dev = x.device();
    Out dx;
    if (truth(a[16])) dx = Out(x.sizes(), F32, dev);
    Outs dh0, dc0;
    for (int l = 0; l < d.layers; ++l) dh0.add(h0.at(l).sizes(), dev);
    for (int l = 0; l < d.layers; ++l) dc0.add(c0.at(l).sizes(), dev);
    std::vector<LstmGrads> gr;
    gr.reserve(d.layers);
    for (int l = 0; l < d.layers; ++l) {
        Ref given(a[17] != Py_None ? PySequence_GetItem(a[17], l) : borrowed(Py_None));
        if (!given.o) throw Fail{nullptr, ""};
        gr.emplace_back(given.o, Vx.at(l), Ux.at(l), Vh.at(l), Uh.at(l), d.h);
    }
    std::vector<void *> gp[5];
    for (int i = 0; i < 5; ++i)
        for (int l = 0; l < d.layers; ++l) gp[i].push_back(gr[l].p[i]);
    void *const px = ptr(a[0], F32), *const pdh = ptr(a[12], F32), *const st = stream();
    const bool given = a[17] != Py_None;
    call("pf_lowrank_lstm_stack_bwd", pf_lowrank_lstm_stack_bwd_workspace_bytes(&d), dev, [&](Space ws) {
        return pf_lowrank_lstm_stack_bwd(&d, px, h0.arr<const void *>(), c0.arr<const void *>(), h.arr<const void *>(),
                                         c.arr<const void *>(), g.arr<const void *>(), Tx.arr<const void *>(), Th.arr<const void *>(),
                                         Vx.arr<const void *>(), Ux.arr<const void *>(), Vh.arr<const void *>(), Uh.arr<const void *>(),
                                         pdh, dhT.arr<const void *>(), dcT.arr<const void *>(), dx.p, dh0.p.data(), dc0.p.data(),
                                         gp[0].data(), gp[1].data(), gp[2].data(), gp[3].data(), gp[4].data(), given, ws.p, ws.n, st);
    });
    PyObject *grads = a[17];
    if (grads == Py_None) {
        grads = PyList_New(d.layers);
        for (int l = 0; l < d.layers; ++l) PyList_SET_ITEM(grads, l, gr[l].give());
    } else {
        Py_INCREF(grads);
    }
    return tuple({dx.give(), dh0.give(), dc0.give(), grads});
}

// ------------------------------------------------------------------ between the projections
// These calls run on the device of their tensors, on torch's current stream there, whatever device is current, and take
// their workspace from torch's allocator for the call: of two graphs captured on one stream each has memory of its own.
hipStream_t stream_of(const at::Device &dev) { return c10::hip::getCurrentHIPStream(dev.index()).stream(); }

template <class F>
void call_here(const char *what, size_t bytes, const at::Device &dev, F f)
{
    const Out ws = bytes ? Out({(int64_t)bytes}, at::kByte, dev) : Out();
    void *const s = (void *)stream_of(dev);
    int status;
    {
        NoGil released;
        status = f(ws.p, bytes, s);
    }
    check(status, what);
}

void same_device(const Tensor &t, const at::Device &dev)
{
    if (!t.is_cuda()) fail("tensors must live on the GPU; there is no CPU path");
    if (t.device() != dev) fail("tensors must be on one device");
}
void shape_is(const Tensor &t, at::IntArrayRef want, const char *name)
{
    if (t.sizes() != want) {
        std::string w = std::string(name) + " must have the shape (";
        for (int64_t x : want) w += std::to_string(x) + ", ";
        throw Fail{PyExc_ValueError, w + ")"};
    }
}
// A dense tensor of a given shape and type, or none
void *dense(PyObject *o, at::IntArrayRef want, at::ScalarType type, const at::Device &dev, const char *name)
{
    if (o == Py_None) return nullptr;
    const Tensor &t = tensor(o);
    same_device(t, dev);
    shape_is(t, want, name);
    return address(t, type);
}
// [B, L, heads, head_dim] with the values of a head adjacent: its address, and its strides (extents of one: 0, which
// no element depends on)
void *heads(const Tensor &t, at::IntArrayRef want, at::ScalarType type, const at::Device &dev, int64_t (&stride)[3], const char *name, bool written)
{
    same_device(t, dev);
    shape_is(t, want, name);
    if (t.scalar_type() != type) fail(std::string("expected ") + c10::toString(type) + ", got " + c10::toString(t.scalar_type()));
    if (t.is_contiguous()) {
        stride[0] = stride[1] = stride[2] = 0;
        return t.data_ptr();
    }
    if (t.size(3) > 1 && t.stride(3) != 1) fail(std::string(name) + ": the values of a head must be adjacent");
    for (int i = 0; i < 3; ++i) stride[i] = t.size(i) > 1 ? t.stride(i) : 0;
    if (!stride[0] && !stride[1] && !stride[2]) fail(std::string(name) + ": one head cannot stand for all of them");
    if (written) { // each dimension steps over what the smaller ones span
        int order[3] = {0, 1, 2};
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j)
                if (stride[order[j]] > stride[order[j + 1]]) std::swap(order[j], order[j + 1]);
        int64_t span = t.size(3);
        for (int i : order) {
            if (t.size(i) <= 1) continue;
            if (stride[i] < span) fail(std::string(name) + ": elements of an output meet");
            span = stride[i] * (t.size(i) - 1) + span;
        }
    }
    return t.data_ptr();
}

// The tensors of one call: Q (4 dimensions), K or none
struct QkCall {
    pf_qk_norm_desc d = {};
    at::Device dev;
    at::ScalarType dt;
    int64_t sq[4], sk[4] = {0, 0, 0, 0};
    // positions, norm, eps, rot_dim (or None), theta, style from a[0] on
    void *positions;
    QkCall(const Tensor &Q, PyObject *K, PyObject *const *a) : dev(Q.device()), dt(Q.scalar_type())
    {
        dims(Q, 4, "Q");
        same_device(Q, dev);
        for (int i = 0; i < 4; ++i) sq[i] = Q.size(i);
        d.B = sq[0], d.L = sq[1], d.heads_q = (int)sq[2], d.head_dim = (int)sq[3];
        if (K != Py_None) {
            const Tensor &k = tensor(K);
            dims(k, 4, "K");
            sk[0] = sq[0], sk[1] = sq[1], sk[2] = k.size(2), sk[3] = sq[3];
            d.heads_k = (int)sk[2];
        }
        d.dtype = dtype_code(Q);
        d.norm = (int)integer(a[1]);
        d.eps = (float)number(a[2]);
        d.rot_dim = a[3] == Py_None ? d.head_dim : integer32(a[3]);
        d.theta = number(a[4]);
        d.rotation = (int)integer(a[5]);
        positions = dense(a[0], {sq[0], sq[1]}, at::kInt, dev, "positions");
    }
    at::IntArrayRef qshape() const { return at::IntArrayRef(sq, 4); }
    at::IntArrayRef kshape() const { return at::IntArrayRef(sk, 4); }
    static double number(PyObject *o)
    {
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) throw Fail{nullptr, ""};
        return v;
    }
};

// A pair of given tensors, or two new ones
struct Pair {
    Ref items;
    PyObject *given[2] = {nullptr, nullptr};
    Pair(PyObject *o, const char *what)
    {
        if (o == Py_None) return;
        items.o = PySequence_Fast(o, what);
        if (!items.o) throw Fail{nullptr, ""};
        if (PySequence_Fast_GET_SIZE(items.o) != 2) throw Fail{PyExc_ValueError, what};
        for (int i = 0; i < 2; ++i) given[i] = PySequence_Fast_GET_ITEM(items.o, i);
    }
};
// Output i of a call: the given tensor's address and strides, or a new dense tensor
void *output(const Pair &p, int i, Out &o, at::IntArrayRef shape, at::ScalarType dt, const at::Device &dev, int64_t (&stride)[3], const char *name)
{
    if (p.given[i] && p.given[i] != Py_None) return heads(tensor(p.given[i]), shape, dt, dev, stride, name, true);
    o = Out(shape, dt, dev);
    stride[0] = stride[1] = stride[2] = 0;
    return o.p;
}
PyObject *give_output(const Pair &p, int i, Out &o) { return p.given[i] && p.given[i] != Py_None ? borrowed(p.given[i]) : o.give(); }

// Q, K, gamma_q, gamma_k, positions, norm, eps, rot_dim, theta, rotation, out
PyObject *qk_fwd(PyObject *const *a)
{
    const Tensor &Q = tensor(a[0]);
    QkCall c(Q, a[1], a + 4);
    const c10::DeviceGuard on(c.dev);
    const bool keys = a[1] != Py_None;
    void *const q = heads(Q, c.qshape(), c.dt, c.dev, c.d.q_stride, "Q", false);
    void *const k = keys ? heads(tensor(a[1]), c.kshape(), c.dt, c.dev, c.d.k_stride, "K", false) : nullptr;
    void *const gq = dense(a[2], {c.d.head_dim}, F32, c.dev, "gamma_q"), *const gk = dense(a[3], {c.d.head_dim}, F32, c.dev, "gamma_k");
    Pair out(a[10], "out must hold the outputs for Q and K");
    Out oq, ok;
    void *const pq = output(out, 0, oq, c.qshape(), c.dt, c.dev, c.d.qo_stride, "out[0]");
    void *const pk = keys ? output(out, 1, ok, c.kshape(), c.dt, c.dev, c.d.ko_stride, "out[1]") : nullptr;
    call_here("pf_qk_norm_rotate_fwd", 0, c.dev, [&](void *, size_t, void *s) { return pf_qk_norm_rotate_fwd(&c.d, q, k, gq, gk, c.positions, pq, pk, s); });
    return tuple({give_output(out, 0, oq), keys ? give_output(out, 1, ok) : borrowed(Py_None)});
}

// Q, K, dQo, dKo, gamma_q, gamma_k, positions, norm, eps, rot_dim, theta, rotation, grads, out
PyObject *qk_bwd(PyObject *const *a)
{
    const Tensor &Q = tensor(a[0]);
    QkCall c(Q, a[1], a + 6);
    const c10::DeviceGuard on(c.dev);
    const bool keys = a[1] != Py_None;
    int64_t in_q[3], in_k[3] = {0, 0, 0};
    void *const q = heads(Q, c.qshape(), c.dt, c.dev, in_q, "Q", false);
    void *const k = keys ? heads(tensor(a[1]), c.kshape(), c.dt, c.dev, in_k, "K", false) : nullptr;
    void *const gq = dense(a[4], {c.d.head_dim}, F32, c.dev, "gamma_q"), *const gk = dense(a[5], {c.d.head_dim}, F32, c.dev, "gamma_k");
    void *const dqo = heads(tensor(a[2]), c.qshape(), c.dt, c.dev, c.d.qo_stride, "dQo", false);
    void *const dko = keys ? heads(tensor(a[3]), c.kshape(), c.dt, c.dev, c.d.ko_stride, "dKo", false) : nullptr;
    Pair grads(a[12], "grads must hold dgamma_q and dgamma_k"), out(a[13], "out must hold dQ and dK");
    const bool given = a[12] != Py_None;
    Out oq, ok, og[2];
    void *dg[2] = {nullptr, nullptr};
    for (int i = 0; i < 2; ++i) {
        if (given) {
            dg[i] = dense(grads.given[i], {c.d.head_dim}, F32, c.dev, "a gamma gradient");
        } else if (c.d.norm && (i ? keys && gk : gq != nullptr)) {
            og[i] = Out({c.d.head_dim}, F32, c.dev);
            dg[i] = og[i].p;
        }
    }
    int64_t sq[3], sk[3] = {0, 0, 0};
    void *const pq = output(out, 0, oq, c.qshape(), c.dt, c.dev, sq, "out[0]");
    void *const pk = keys ? output(out, 1, ok, c.kshape(), c.dt, c.dev, sk, "out[1]") : nullptr;
    for (int i = 0; i < 3; ++i) {
        c.d.q_stride[i] = in_q[i], c.d.k_stride[i] = in_k[i];
        c.d.dq_stride[i] = sq[i], c.d.dk_stride[i] = sk[i];
    }
    call_here("pf_qk_norm_rotate_bwd", pf_qk_norm_rotate_bwd_workspace_bytes(&c.d), c.dev, [&](void *ws, size_t n, void *s) {
        return pf_qk_norm_rotate_bwd(&c.d, q, k, gq, gk, c.positions, dqo, dko, pq, pk, dg[0], dg[1], given, ws, n, s);
    });
    return tuple({give_output(out, 0, oq), keys ? give_output(out, 1, ok) : borrowed(Py_None), given ? borrowed(grads.given[0]) : og[0].give(),
                  given ? borrowed(grads.given[1]) : og[1].give()});
}

// Q, K, V, table, causal, scale (or None), max_distance, bidirectional, q_start, q_len, kv_len from a[0] on
struct AttnCall {
    pf_attention_desc d = {};
    at::Device dev;
    at::ScalarType dt;
    void *q, *k, *v, *table, *start, *nq, *nk;
    int64_t sq[4], sk[4], stat[3], tab[2];
    explicit AttnCall(PyObject *const *a) : dev(tensor(a[0]).device()), dt(tensor(a[0]).scalar_type())
    {
        const Tensor &Q = tensor(a[0]), &K = tensor(a[1]), &V = tensor(a[2]);
        dims(Q, 4, "Q");
        dims(K, 4, "K");
        for (int i = 0; i < 4; ++i) sq[i] = Q.size(i);
        sk[0] = sq[0], sk[1] = K.size(1), sk[2] = K.size(2), sk[3] = sq[3];
        d.B = sq[0], d.Lq = sq[1], d.Lk = sk[1], d.heads_q = (int)sq[2], d.heads_kv = (int)sk[2], d.head_dim = (int)sq[3];
        d.dtype = dtype_code(Q);
        q = heads(Q, at::IntArrayRef(sq, 4), dt, dev, d.q_stride, "Q", false);
        k = heads(K, at::IntArrayRef(sk, 4), dt, dev, d.k_stride, "K", false);
        v = heads(V, at::IntArrayRef(sk, 4), dt, dev, d.v_stride, "V", false);
        d.causal = truth(a[4]);
        d.scale = (float)(a[5] == Py_None ? 1.0 / std::sqrt((double)std::max<int64_t>(1, sq[3])) : QkCall::number(a[5]));
        table = nullptr;
        tab[0] = 0, tab[1] = sq[2];
        if (a[3] != Py_None) {
            const Tensor &T = tensor(a[3]);
            dims(T, 2, "table");
            tab[0] = T.size(0);
            if (tab[0] == 0) throw Fail{PyExc_ValueError, "table has no bucket"};
            table = dense(a[3], at::IntArrayRef(tab, 2), F32, dev, "table");
            d.buckets = (int)std::min<int64_t>(tab[0], INT32_MAX);
            d.max_distance = integer32(a[6]);
            d.bidirectional = truth(a[7]);
        }
        start = dense(a[8], {sq[0]}, at::kInt, dev, "q_start");
        nq = dense(a[9], {sq[0]}, at::kInt, dev, "q_len");
        nk = dense(a[10], {sq[0]}, at::kInt, dev, "kv_len");
        stat[0] = sq[0], stat[1] = sq[2], stat[2] = sq[1];
    }
};

// Q .. kv_len as above, save_lse
PyObject *attn_fwd(PyObject *const *a)
{
    AttnCall c(a);
    const c10::DeviceGuard on(c.dev);
    Out O(at::IntArrayRef(c.sq, 4), c.dt, c.dev), lse;
    if (truth(a[11])) lse = Out(at::IntArrayRef(c.stat, 3), F32, c.dev);
    call_here("pf_attention_fwd", pf_attention_fwd_workspace_bytes(&c.d), c.dev, [&](void *ws, size_t n, void *s) {
        return pf_attention_fwd(&c.d, c.q, c.k, c.v, c.table, c.start, c.nq, c.nk, O.p, lse.p, ws, n, s);
    });
    return tuple({O.give(), lse.give()});
}

// Q .. kv_len as above, O, lse, dO, need_dtable, grads, out
PyObject *attn_bwd(PyObject *const *a)
{
    AttnCall c(a);
    const c10::DeviceGuard on(c.dev);
    const at::IntArrayRef qs(c.sq, 4), ks(c.sk, 4), ts(c.tab, 2);
    void *const o = dense(a[11], qs, c.dt, c.dev, "O"), *const lse = dense(a[12], at::IntArrayRef(c.stat, 3), F32, c.dev, "lse"),
               *const g = dense(a[13], qs, c.dt, c.dev, "dO");
    const bool given = a[15] != Py_None;
    Out dt, d[3];
    void *pt = given ? dense(a[15], ts, F32, c.dev, "grads") : nullptr, *p[3];
    if (!given && c.table && truth(a[14])) {
        dt = Out(ts, F32, c.dev);
        pt = dt.p;
    }
    Ref items;
    if (a[16] != Py_None) {
        items.o = PySequence_Fast(a[16], "out must hold dQ, dK and dV");
        if (!items.o) throw Fail{nullptr, ""};
        if (PySequence_Fast_GET_SIZE(items.o) != 3) throw Fail{PyExc_ValueError, "out must hold dQ, dK and dV"};
    }
    PyObject *into[3];
    for (int i = 0; i < 3; ++i) {
        into[i] = items.o ? PySequence_Fast_GET_ITEM(items.o, i) : Py_None;
        if (into[i] != Py_None) {
            p[i] = dense(into[i], i ? ks : qs, c.dt, c.dev, "out");
        } else {
            d[i] = Out(i ? ks : qs, c.dt, c.dev);
            p[i] = d[i].p;
        }
    }
    call_here("pf_attention_bwd", pf_attention_bwd_workspace_bytes(&c.d), c.dev, [&](void *ws, size_t n, void *s) {
        return pf_attention_bwd(&c.d, c.q, c.k, c.v, c.table, c.start, c.nq, c.nk, o, lse, g, p[0], p[1], p[2], pt, given, ws, n, s);
    });
    const auto give = [&](int i) { return into[i] != Py_None ? borrowed(into[i]) : d[i].give(); };
    return tuple({give(0), give(1), give(2), given ? borrowed(a[15]) : dt.give()});
}

// tensors, state_bits, beta1, beta2, eps, plan, lr, grad_scale, steps
PyObject *adamw_step(PyObject *const *a)
{
    pf_adamw_desc d = {};
    d.tensors = integer(a[0]);
    d.state_bits = (int)integer(a[1]);
    d.beta1 = QkCall::number(a[2]);
    d.beta2 = QkCall::number(a[3]);
    d.eps = QkCall::number(a[4]);
    const Tensor &plan = tensor(a[5]);
    const auto dev = plan.device();
    same_device(plan, dev);
    const c10::DeviceGuard on(dev);
    void *const p = address(plan, at::kByte), *const lr = dense(a[6], {1}, F32, dev, "lr");
    void *scale = nullptr;
    if (a[7] != Py_None) {
        const Tensor &t = tensor(a[7]);
        same_device(t, dev);
        if (t.numel() != 1) throw Fail{PyExc_ValueError, "grad_scale must have one element"};
        scale = address(t, F32);
    }
    const Tensor &steps = tensor(a[8]);
    same_device(steps, dev);
    if (steps.numel() != 1) throw Fail{PyExc_ValueError, "steps must have one element"};
    void *const st = address(steps, at::kLong);
    const size_t n = (size_t)plan.numel();
    call_here("pf_adamw_step", 0, dev, [&](void *, size_t, void *s) { return pf_adamw_step(&d, p, n, lr, scale, st, s); });
    Py_RETURN_NONE;
}

// bytes, a tensor on the device: the scratch buffer of the current stream, held by this thread until it gives it back
PyObject *lend(PyObject *const *a)
{
    const size_t bytes = (size_t)integer(a[0]);
    const auto dev = tensor(a[1]).device();
    if (!dev.is_cuda()) fail("tensors must live on the GPU; there is no CPU path");
    Scratch *s;
    {
        NoGil released;
        s = &scratch(dev);
        s->busy.lock();
    }
    try {
        s->get(bytes, dev);
    } catch (...) {
        s->busy.unlock();
        throw;
    }
    return tuple({PyLong_FromVoidPtr(s), THPVariable_Wrap(s->t)});
}
PyObject *give_back(PyObject *const *a)
{
    ((Scratch *)PyLong_AsVoidPtr(a[0]))->busy.unlock();
    Py_RETURN_NONE;
}

// The exceptions to raise: PfError, torch.OutOfMemoryError
PyObject *set_errors(PyObject *, PyObject *args)
{
    PyObject *e, *m;
    if (!PyArg_ParseTuple(args, "OO", &e, &m)) return nullptr;
    g_error = borrowed(e);
    g_no_memory = borrowed(m);
    Py_RETURN_NONE;
}

#define CALL(name, n) {#name, (PyCFunction)(void (*)(void))entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(linear_fwd, 8),
                         CALL(linear_bwd, 11),
                         CALL(shared_fwd, 5),
                         CALL(shared_bwd, 8),
                         CALL(conv_fwd, 12),
                         CALL(conv_bwd, 15),
                         CALL(cell_fwd, 9),
                         CALL(cell_bwd, 16),
                         CALL(stack_fwd, 9),
                         CALL(stack_bwd, 18),
                         CALL(qk_fwd, 11),
                         CALL(qk_bwd, 14),
                         CALL(attn_fwd, 12),
                         CALL(attn_bwd, 17),
                         CALL(adamw_step, 9),
                         CALL(lend, 2),
                         CALL(give_back, 1),
                         {"set_errors", set_errors, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
