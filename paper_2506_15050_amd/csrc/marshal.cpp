// Python side of the C ABI (tppo.h), native: turns a call's tensors into pointers, allocates its results, and calls.  The
// smallest passes are bound by what happens here, once a call: through ctypes and torch's Python functions a token filter
// with its plan took 18.8 us of host time, log-probs 10.6, EGAE 5.7 and losses 6.0; here 9.1, 8.7, 3.6 and 3.9.
// What is taken and what is refused is what ctypes and the binding's own assertions take and refuse; sizes, ranges and NULLs are
// the C entry points' own business.
#include <Python.h>
#include <ATen/Context.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/Device.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <exception>
#include <initializer_list>
#include <utility>

#include "tppo.h"

namespace {

struct Raised {};                                                   // a Python exception is set

[[noreturn]] void raise(PyObject* type, const char* text) {
    PyErr_SetString(type, text);
    throw Raised{};
}

// a new reference, or the exception that is there instead
class Held {
  public:
    explicit Held(PyObject* o) : o_(o) {
        if (!o) throw Raised{};
    }
    ~Held() { Py_DECREF(o_); }
    Held(const Held&) = delete;
    PyObject* get() const { return o_; }

  private:
    PyObject* o_;
};

// The arguments of one call, in order.
class Args {
  public:
    Args(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : at_(args) {
        if (n != want) raise(PyExc_TypeError, "wrong number of arguments");
    }
    // a tensor's memory; None: NULL.  Anything but a plain tensor is asked through Python, where a subclass or another
    // library's array has its own say.
    void* any() {
        PyObject* o = *at_++;
        if (o == Py_None) return nullptr;
        if (THPVariable_CheckExact(o)) return THPVariable_Unpack(o).data_ptr();
        const Held p(PyObject_CallMethod(o, "data_ptr", nullptr));
        if (p.get() == Py_None) return nullptr;
        void* v = PyLong_AsVoidPtr(p.get());
        if (PyErr_Occurred()) throw Raised{};
        return v;
    }
    template <typename T>
    T* ptr() { return static_cast<T*>(any()); }
    int32_t* dev_i32() { return static_cast<int32_t*>(checked(at::kInt)); }
    float* dev_f32() { return static_cast<float*>(checked(at::kFloat)); }
    // a buffer and its size in bytes; None: NULL and 0
    void* buffer(size_t& bytes) {
        bytes = 0;
        PyObject* o = *at_;
        if (o == Py_None) return any();
        if (THPVariable_CheckExact(o)) {
            bytes = (size_t)THPVariable_Unpack(o).numel();
        } else {
            const Held n(PyObject_CallMethod(o, "numel", nullptr));
            bytes = (size_t)PyLong_AsUnsignedLongLongMask(n.get());
            if (PyErr_Occurred()) throw Raised{};
        }
        return any();
    }
    int64_t i64() {
        PyObject* o = *at_++;
        const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
        if (v == ~0ull && PyErr_Occurred()) refuse(o);
        return (int64_t)v;
    }
    int32_t i32() { return (int32_t)i64(); }
    float f32() {
        const double v = PyFloat_AsDouble(*at_++);
        if (v == -1.0 && PyErr_Occurred()) throw Raised{};
        return (float)v;
    }
    void* stream() {
        void* s = PyLong_AsVoidPtr(*at_++);
        if (PyErr_Occurred()) throw Raised{};
        return s;
    }

  private:
    // what is no whole number: ctypes' own exception
    [[noreturn]] static void refuse(PyObject* o) {
        PyErr_Clear();
        const Held ctypes(PyImport_ImportModule("ctypes")), error(PyObject_GetAttrString(ctypes.get(), "ArgumentError"));
        PyErr_Format(error.get(), "int expected instead of %.200s instance", Py_TYPE(o)->tp_name);
        throw Raised{};
    }
    void* checked(at::ScalarType type) {
        PyObject* o = *at_;
        if (o == Py_None) raise(PyExc_AssertionError, "a tensor is required");
        bool good;
        if (THPVariable_CheckExact(o)) {
            const at::Tensor& t = THPVariable_Unpack(o);
            good = t.is_cuda() && t.scalar_type() == type && t.is_contiguous();
        } else {
            const Held cuda(PyObject_GetAttrString(o, "is_cuda")), dtype(PyObject_GetAttrString(o, "dtype"));
            const Held dense(PyObject_CallMethod(o, "is_contiguous", nullptr));
            good = truth(PyObject_IsTrue(cuda.get())) && truth(PyObject_IsTrue(dense.get())) &&
                   truth(PyObject_RichCompareBool(dtype.get(), reinterpret_cast<PyObject*>(torch::getTHPDtype(type)), Py_EQ));
        }
        if (!good) raise(PyExc_AssertionError, "a contiguous device tensor of the documented type is required");
        return any();
    }
    static bool truth(int answer) {
        if (answer < 0) throw Raised{};
        return answer != 0;
    }
    PyObject* const* at_;
};

// What torch raises passes as from its own functions: an allocation that fails is torch.OutOfMemoryError, an exception of a
// Python dispatch mode is that exception.
template <class F>
PyObject* guarded(F&& f) {
    try {
        return f();
    } catch (const Raised&) {
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

// other Python threads run while one of these lives
class NoInterpreter {
  public:
    NoInterpreter() : state_(PyEval_SaveThread()) {}
    ~NoInterpreter() { PyEval_RestoreThread(state_); }
    NoInterpreter(const NoInterpreter&) = delete;

  private:
    PyThreadState* state_;
};

// the call itself, with the interpreter free as it is under ctypes
template <class F>
PyObject* status_of(F&& call) {
    int rc;
    {
        NoInterpreter other_threads_run;
        rc = call();
    }
    return PyLong_FromLong(rc);
}

// a call of `want` arguments
template <PyObject* (*call)(Args&), int want>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&] {
        Args x(args, n, want);
        return call(x);
    });
}

PyObject* select(Args& x) {
    auto *cu = x.dev_i32(), *ctx = x.dev_i32(), *done = x.dev_i32(), *ids = x.ptr<int32_t>();
    const int64_t B = x.i64(), n_tok = x.i64();
    const int32_t drop = x.i32();
    auto *resp = x.ptr<int32_t>(), *sel = x.ptr<int32_t>(), *keep = x.ptr<int32_t>(), *rows = x.ptr<int32_t>();
    auto *targets = x.ptr<int32_t>(), *idx = x.ptr<int32_t>();
    const int64_t cap = x.i64();
    auto* counts = x.ptr<int64_t>();
    size_t ws_bytes, plan_bytes;
    void *ws = x.buffer(ws_bytes), *plan = x.buffer(plan_bytes);
    auto* status = x.ptr<int32_t>();
    void* s = x.stream();
    return status_of([&] {
        return tppo_select(cu, ctx, done, ids, B, n_tok, drop, resp, sel, keep, rows, targets, idx, cap, counts, ws, ws_bytes,
                           plan, plan_bytes, status, s);
    });
}

PyObject* token_logprobs(Args& x) {
    const void* hidden = x.any();
    const int64_t n_rows = x.i64(), H = x.i64(), ld_h = x.i64();
    const void* w = x.any();
    const int64_t V = x.i64(), ld_w = x.i64();
    const auto dt = (tppo_dtype)x.i32();
    auto *rows = x.dev_i32(), *targets = x.dev_i32();
    const int64_t M = x.i64();
    auto* m_actual = x.ptr<int64_t>();
    auto* out_index = x.ptr<int32_t>();
    auto *logp = x.ptr<float>(), *lse = x.ptr<float>();
    size_t bytes;
    void* ws = x.buffer(bytes);
    auto* status = x.ptr<int32_t>();
    void* s = x.stream();
    return status_of([&] {
        return tppo_token_logprobs(hidden, n_rows, H, ld_h, w, V, ld_w, dt, rows, targets, M, m_actual, out_index, logp, lse, ws,
                                   bytes, status, s);
    });
}

// tppo_egae, tppo_egae_terminal
template <decltype(tppo_egae)* entry_point>
PyObject* egae(Args& x) {
    auto *rewards = x.dev_f32(), *values = x.dev_f32();
    auto *resp = x.dev_i32(), *done = x.dev_i32();
    auto* boot = x.ptr<float>();
    const int64_t B = x.i64(), n_resp = x.i64();
    const float gamma = x.f32(), lam = x.f32();
    auto *adv = x.ptr<float>(), *ret = x.ptr<float>();
    size_t bytes;
    void *ws = x.buffer(bytes), *plan = x.any();
    auto* status = x.ptr<int32_t>();
    void* s = x.stream();
    return status_of([&] {
        return entry_point(rewards, values, resp, done, boot, B, n_resp, gamma, lam, adv, ret, ws, bytes, plan, status, s);
    });
}

PyObject* ppo_losses(Args& x) {
    const float* in[6];
    for (auto& p : in) p = x.ptr<float>();
    auto *resp = x.dev_i32(), *keep = x.dev_i32(), *done = x.dev_i32();
    const int64_t B = x.i64(), n_resp = x.i64();
    const float el = x.f32(), eh = x.f32(), xl = x.f32(), xh = x.f32();
    auto* out = x.ptr<tppo_loss_out>();
    size_t bytes;
    void *ws = x.buffer(bytes), *plan = x.any();
    auto* status = x.ptr<int32_t>();
    void* s = x.stream();
    return status_of([&] {
        return tppo_ppo_losses(in[0], in[1], in[2], in[3], in[4], in[5], resp, keep, done, B, n_resp, el, eh, xl, xh, out, ws, bytes,
                               plan, status, s);
    });
}

PyObject* ppo_losses_backward(Args& x) {
    const float* in[6];
    for (auto& p : in) p = x.ptr<float>();
    auto *resp = x.dev_i32(), *keep = x.dev_i32(), *done = x.dev_i32();
    const int64_t B = x.i64(), n_resp = x.i64();
    const float el = x.f32(), eh = x.f32(), xl = x.f32(), xh = x.f32(), ps = x.f32(), vs = x.f32();
    const int64_t pd = x.i64(), vd = x.i64();
    auto *g_logp = x.ptr<float>(), *g_v = x.ptr<float>();
    auto* out = x.ptr<tppo_loss_out>();
    auto* stats = x.ptr<tppo_loss_stats>();
    size_t bytes;
    void *ws = x.buffer(bytes), *plan = x.any();
    auto* status = x.ptr<int32_t>();
    void* s = x.stream();
    return status_of([&] {
        return tppo_ppo_losses_backward(in[0], in[1], in[2], in[3], in[4], in[5], resp, keep, done, B, n_resp, el, eh, xl, xh, ps, vs,
                                        pd, vd, g_logp, g_v, out, stats, ws, bytes, plan, status, s);
    });
}

PyObject* value_head(Args& x) {
    const void* hidden = x.any();
    const int64_t n_rows = x.i64(), H = x.i64(), ld = x.i64();
    const void* w = x.any();
    const float bias = x.f32();
    const auto dt = (tppo_dtype)x.i32();
    auto *rows = x.ptr<int32_t>(), *out_index = x.ptr<int32_t>();
    const int64_t M = x.i64();
    auto* m_actual = x.ptr<int64_t>();
    auto* v = x.ptr<float>();
    auto* status = x.ptr<int32_t>();
    void* s = x.stream();
    return status_of([&] { return tppo_value_head(hidden, n_rows, H, ld, w, bias, dt, rows, out_index, M, m_actual, v, status, s); });
}

// sizes of buffers that a caller did not bring
PyObject* select_workspace_bytes(Args& x) {
    const int64_t B = x.i64(), capacity = x.i64();
    return PyLong_FromSize_t(tppo_select_workspace_bytes(B, capacity));
}
PyObject* plan_bytes(Args& x) {
    const int64_t n_resp = x.i64(), B = x.i64();
    return PyLong_FromSize_t(tppo_plan_bytes(n_resp, B));
}

// empties(like, kinds, n0, n1, ...): one-dimensional uninitialised tensors on `like`'s device, kinds[i] in "ilfb" (int32, int64,
// float32, bytes).  The interpreter is free meanwhile, as it is in torch.empty: an allocator that has to ask the driver, or that
// waits for another thread's call into it, must not hold up the other Python threads.
constexpr Py_ssize_t kMostBuffers = 16;

// Each buffer is an allocation of its own, as torch.empty's: a caller may resize it, give it as `out`, save it, keep it, and record a
// stream's use of it without the others.  (Pieces of one allocation are cheaper still and allow none of these: what grows runs into the
// next piece, and storages of their own over one block are none that the device's allocator knows to record a stream for.)  The first
// is at::empty's; the others are made here from its storage's allocator, past the dispatcher, whose way costs more than the allocation
// (a token filter's nine: 7.3 us of host time, so 4.4; pieces of one block 2.15), unless a dispatch mode, a transform, a trace or the
// fill of deterministic runs has its own say about allocations.
const c10::DispatchKeySet kPlainKeys({c10::DispatchKey::CPU, c10::DispatchKey::CUDA, c10::DispatchKey::ADInplaceOrView,
                                      c10::DispatchKey::AutogradCPU, c10::DispatchKey::AutogradCUDA, c10::DispatchKey::AutocastCPU,
                                      c10::DispatchKey::AutocastCUDA});
bool undisturbed() {                                               // nothing beyond the usual takes part in this thread's calls
    return !c10::impl::dispatch_mode_enabled() && c10::default_included_set.has_all(c10::impl::tls_local_dispatch_key_set().included_) &&
           !at::globalContext().deterministicAlgorithms();         // (which fills what is allocated, by type)
}
void allocate(const at::TensorOptions& on, const at::ScalarType* types, const int64_t* sizes, Py_ssize_t count, at::Tensor* made) {
    if (count == 0) return;
    made[0] = at::empty({sizes[0]}, on.dtype(types[0]));
    Py_ssize_t i = 1;
    const auto keys = made[0].key_set();
    if (count > 1 && undisturbed() && kPlainKeys.has_all(keys) && made[0].has_storage() && made[0].storage().allocator()) {
        const c10::DeviceGuard there(made[0].device());
        // (sizes that are none, or too many bytes for a number, are at::empty's to refuse)
        for (; i < count && sizes[i] >= 0 && sizes[i] <= INT64_MAX / 8; ++i) {
            c10::Storage own(c10::Storage::use_byte_size_t(), (size_t)sizes[i] * c10::elementSize(types[i]), made[0].storage().allocator(), true);
            made[i] = at::detail::make_tensor<c10::TensorImpl>(std::move(own), keys, c10::scalarTypeToTypeMeta(types[i]));
            made[i].unsafeGetTensorImpl()->set_sizes_contiguous({sizes[i]});
        }
    }
    for (; i < count; ++i) made[i] = at::empty({sizes[i]}, on.dtype(types[i]));
}
at::Device device_of(PyObject* like) {
    if (THPVariable_CheckExact(like)) return THPVariable_Unpack(like).device();
    const Held device(PyObject_GetAttrString(like, "device"));
    if (!THPDevice_Check(device.get())) raise(PyExc_TypeError, "a torch.device is required");
    return reinterpret_cast<THPDevice*>(device.get())->device;
}
PyObject* empties(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS                                                // (the allocator's warnings are Python's)
    try {
        if (n < 2 || args[0] == Py_None) raise(PyExc_TypeError, "empties(tensor, kinds, sizes...)");
        Py_ssize_t count = 0;
        const char* kinds = PyUnicode_AsUTF8AndSize(args[1], &count);
        if (!kinds) throw Raised{};
        if (count != n - 2) raise(PyExc_TypeError, "a size for each kind");
        const auto on = at::TensorOptions().device(device_of(args[0]));
        int64_t sizes[kMostBuffers];
        at::Tensor made[kMostBuffers];
        if (count > kMostBuffers) raise(PyExc_TypeError, "too many buffers");
        for (Py_ssize_t i = 0; i < count; ++i) {
            sizes[i] = PyLong_AsLongLong(args[2 + i]);
            if (sizes[i] == -1 && PyErr_Occurred()) throw Raised{};
        }
        {
            NoInterpreter other_threads_run;
            at::ScalarType types[kMostBuffers];
            for (Py_ssize_t i = 0; i < count; ++i)
                types[i] = kinds[i] == 'i' ? at::kInt : kinds[i] == 'l' ? at::kLong : kinds[i] == 'f' ? at::kFloat : at::kByte;
            allocate(on, types, sizes, count, made);
        }
        PyObject* out = PyTuple_New(count);
        if (!out) throw Raised{};
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject* t = THPVariable_Wrap(made[i]);
            if (!t) {
                Py_DECREF(out);
                throw Raised{};
            }
            PyTuple_SET_ITEM(out, i, t);
        }
        return out;
    } catch (const Raised&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// ---- layer norm, balance loss, orthogonalisation: a call's tensors looked over, its results made, and the call, in one trip.  (The same
// looking over by Python: 10 to 14 us a call.)

// What a call of one of these has been given.  `name` opens its refusals, which are ValueErrors.
class Taken {
  public:
    Taken(const char* name, PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : name_(name), at_(args) {
        if (n != want) raise(PyExc_TypeError, "wrong number of arguments");
    }
    [[noreturn]] void refuse(const char* why) const {
        PyErr_Format(PyExc_ValueError, "%s: %s", name_, why);
        throw Raised{};
    }
    PyObject* next() { return *at_++; }
    // a device tensor, on the device of those before it; None where that may be: null
    const at::Tensor* tensor(bool optional, const char* what) { return checked(next(), optional, what); }
    const at::Tensor* checked(PyObject* o, bool optional, const char* what) {
        if (o == Py_None && optional) return nullptr;
        if (!THPVariable_Check(o)) refuse(what);
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda()) refuse("device tensors are required");
        if (!on_) on_ = &t;
        else if (t.device() != on_->device()) refuse("all tensors have to be on one device");
        return &t;
    }
    // a dense one of n elements at least (exactly n, if so)
    const at::Tensor* dense(PyObject* o, at::ScalarType type, int64_t n, bool exactly, bool optional, const char* what) {
        const at::Tensor* t = checked(o, optional, what);
        if (t && (t->scalar_type() != type || !t->is_contiguous() || t->numel() < n || (exactly && t->numel() != n))) refuse(what);
        return t;
    }
    int64_t i64(int64_t none) {
        PyObject* o = next();
        if (o == Py_None) return none;
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) throw Raised{};
        return v;
    }
    float f32() {
        const double v = PyFloat_AsDouble(next());
        if (v == -1.0 && PyErr_Occurred()) throw Raised{};
        return (float)v;
    }
    bool flag() {
        const int v = PyObject_IsTrue(next());
        if (v < 0) throw Raised{};
        return v != 0;
    }
    void* stream() {
        void* s = PyLong_AsVoidPtr(next());
        if (PyErr_Occurred()) throw Raised{};
        return s;
    }
    // the entries of a tuple or list of `n`
    PyObject* entry(PyObject* o, Py_ssize_t n, Py_ssize_t i) const {
        if (!(PyTuple_Check(o) || PyList_Check(o)) || PySequence_Fast_GET_SIZE(o) != n) refuse("a tuple of output tensors is required");
        return PySequence_Fast_GET_ITEM(o, i);
    }
    at::TensorOptions like() const { return at::TensorOptions().device(on_->device()); }

  private:
    const char* name_;
    PyObject* const* at_;
    const at::Tensor* on_ = nullptr;
};
void* memory(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
template <class T>
T* memory(const at::Tensor* t) { return static_cast<T*>(memory(t)); }
bool known(const at::Tensor& t) { return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16; }
tppo_dtype type_of(const at::Tensor& t) { return t.scalar_type() == at::kBFloat16 ? TPPO_BF16 : TPPO_F32; }
size_t bytes_of(const at::Tensor* t) { return t ? (size_t)t->numel() * t->element_size() : 0; }

// a matrix, or a stack of them, with rows whole in memory
struct Rows {
    const at::Tensor* t = nullptr;
    int64_t rows = 0, cols = 0, ld = 0, count = 1, each = 0;
    Rows() = default;
    Rows(const Taken& x, const at::Tensor* tensor, const char* what, bool stack = false) : t(tensor) {
        const int64_t dims = t->dim();
        if (dims != 2 && !(stack && dims == 3)) x.refuse(what);
        rows = t->size(dims - 2);
        cols = t->size(dims - 1);
        if (cols > 1 && t->stride(dims - 1) != 1) x.refuse("rows have to be contiguous in memory");
        ld = rows > 1 ? t->stride(dims - 2) : std::max(t->stride(dims - 2), cols);
        if (ld < cols) x.refuse("rows that share memory");
        count = dims == 3 ? t->size(0) : 1;
        each = dims == 3 ? t->stride(0) : rows * ld;
    }
};

// rows, M, m_actual
struct Listed {
    const at::Tensor *rows, *m_actual;
    int64_t M;
    Listed(Taken& x, int64_t n_rows) {
        PyObject* o = x.next();
        rows = x.dense(o, at::kInt, 0, false, true, "rows must be a contiguous int32 device tensor");
        const int64_t there = rows ? rows->numel() : n_rows;
        M = x.i64(there);
        if (M < 0 || M > there) x.refuse("M is negative or more than there are rows");
        m_actual = x.dense(x.next(), at::kLong, 1, false, true, "m_actual must be an int64 device tensor");
    }
};
const at::Tensor* index_of(Taken& x, int64_t M) {
    return x.dense(x.next(), at::kInt, M, false, true, "out_index must be a contiguous int32 device tensor of M entries");
}
const at::Tensor* workspace_of(Taken& x) {
    const at::Tensor* t = x.tensor(true, "workspace must be a device tensor");
    if (t && !t->is_contiguous()) x.refuse("workspace must be contiguous");
    return t;
}
const at::Tensor* status_word(Taken& x) {
    return x.dense(x.next(), at::kInt, 1, false, true, "status must be an int32 device tensor");
}

// the call itself, with the interpreter free; what it returns
template <class F>
int run(F&& call) {
    NoInterpreter other_threads_run;
    return call();
}
PyObject* tuple_of(std::initializer_list<const at::Tensor*> results) {
    const Held out(PyTuple_New((Py_ssize_t)results.size()));
    Py_ssize_t i = 0;
    for (const at::Tensor* t : results) {
        PyObject* o = Py_None;
        if (t) {
            o = THPVariable_Wrap(*t);
            if (!o) throw Raised{};
        } else {
            Py_INCREF(o);
        }
        PyTuple_SET_ITEM(out.get(), i++, o);
    }
    Py_INCREF(out.get());
    return out.get();
}
// each as at::empty makes it, the interpreter free meanwhile (see empties)
at::Tensor made(const at::TensorOptions& on, at::ScalarType type, at::IntArrayRef sizes) {
    NoInterpreter other_threads_run;
    return at::empty(sizes, on.dtype(type));
}
const at::Tensor* scratch(const at::Tensor* given, size_t bytes, const at::TensorOptions& on, at::Tensor& own) {
    if (given) return given;
    own = made(on, at::kByte, {(int64_t)std::max(bytes, (size_t)256)});
    return &own;
}

// (x, weight, bias, eps, rows, M, m_actual, want_stats, status, out, stream)
PyObject* layer_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&] {
        Taken a("tppo_layer_norm", args, n, 11);
        const Rows x(a, a.tensor(false, "x must be a device matrix"), "x must be a device matrix");
        if (!known(*x.t)) a.refuse("x must be fp32 or bf16");
        const at::Tensor* w = a.tensor(false, "weight must be a device tensor");
        if (!known(*w)) a.refuse("weight must be fp32 or bf16");
        a.dense(args[1], w->scalar_type(), x.cols, true, false, "weight must be contiguous, of H elements");
        const at::Tensor* b = a.dense(a.next(), w->scalar_type(), x.cols, true, true, "bias must be as weight");
        const float eps = a.f32();
        const Listed l(a, x.rows);
        const bool want_stats = a.flag();
        const at::Tensor* status = status_word(a);
        PyObject* out = a.next();
        void* s = a.stream();
        at::Tensor own[3];
        const at::Tensor *y, *mean = nullptr, *rstd = nullptr;
        if (out == Py_None) {
            own[0] = made(a.like(), x.t->scalar_type(), {l.M, x.cols});
            y = &own[0];
            if (want_stats) {
                own[1] = made(a.like(), at::kFloat, {l.M});
                own[2] = made(a.like(), at::kFloat, {l.M});
                mean = &own[1];
                rstd = &own[2];
            }
        } else {
            y = a.checked(a.entry(out, 3, 0), false, "y must be a device matrix");
            mean = a.dense(a.entry(out, 3, 1), at::kFloat, l.M, false, true, "mean must be contiguous fp32 of M elements");
            rstd = a.dense(a.entry(out, 3, 2), at::kFloat, l.M, false, true, "rstd must be contiguous fp32 of M elements");
        }
        const Rows to(a, y, "y must be a device matrix");
        if (y->scalar_type() != x.t->scalar_type() || to.rows < l.M || to.cols != x.cols) a.refuse("y must be [M, H] of x's type");
        const int rc = run([&] {
            return tppo_layer_norm(memory(x.t), x.rows, x.cols, x.ld, type_of(*x.t), memory(w), memory(b), type_of(*w), eps,
                                   memory<int32_t>(l.rows), l.M, memory<int64_t>(l.m_actual), memory(y), to.ld, memory<float>(mean),
                                   memory<float>(rstd), memory<int32_t>(status), s);
        });
        return rc ? PyLong_FromLong(rc) : tuple_of({y, mean, rstd});
    });
}

// (grad_y, x, weight, mean, rstd, rows, M, m_actual, out_index, out, grad_type, want_x, want_w, want_bias, grad_w, accumulate_w, status,
// workspace, stream); grad_type: 0 fp32, 1 bf16, None: x's
PyObject* layer_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&] {
        Taken a("tppo_layer_norm_backward", args, n, 19);
        const Rows gy(a, a.tensor(false, "grad_y must be a device matrix"), "grad_y must be a device matrix");
        const Rows x(a, a.tensor(false, "x must be a device matrix"), "x must be a device matrix");
        if (!known(*x.t) || !known(*gy.t)) a.refuse("x and grad_y must be fp32 or bf16");
        const at::Tensor* w = a.tensor(false, "weight must be a device tensor");
        if (!known(*w)) a.refuse("weight must be fp32 or bf16");
        a.dense(args[2], w->scalar_type(), x.cols, true, false, "weight must be contiguous, of H elements");
        PyObject *mean_o = a.next(), *rstd_o = a.next();
        const Listed l(a, x.rows);
        if (gy.rows < l.M || gy.cols != x.cols) a.refuse("grad_y must be [M, H]");
        const at::Tensor* mean = a.dense(mean_o, at::kFloat, l.M, false, false, "mean must be contiguous fp32 of M elements");
        const at::Tensor* rstd = a.dense(rstd_o, at::kFloat, l.M, false, false, "rstd must be contiguous fp32 of M elements");
        const at::Tensor* index = index_of(a, l.M);
        PyObject* out = a.next();
        const int64_t grad_type = a.i64(-1);
        const bool want_x = a.flag(), want_w = a.flag(), want_bias = a.flag();
        PyObject* grad_w = a.next();
        const bool accumulate = a.flag();
        const at::Tensor* status = status_word(a);
        const at::Tensor* ws = workspace_of(a);
        void* s = a.stream();
        at::Tensor own[4];
        const at::Tensor *gx = nullptr, *gw = nullptr, *gb = nullptr;
        Rows to;
        if (want_x) {
            if (out == Py_None) {
                if (index) a.refuse("out_index needs the tensor that it points into (out)");
                own[0] = made(a.like(), grad_type < 0 ? x.t->scalar_type() : grad_type ? at::kBFloat16 : at::kFloat, {l.M, x.cols});
                gx = &own[0];
            } else {
                gx = a.checked(out, false, "out must be a device matrix");
            }
            to = Rows(a, gx, "out must be a device matrix");
            if (!known(*gx) || to.cols != x.cols || (!index && to.rows < l.M)) a.refuse("out must be [M, H], fp32 or bf16");
        }
        if (grad_w != Py_None) {
            gw = a.dense(a.entry(grad_w, 2, 0), at::kFloat, x.cols, true, true, "grad_weight must be contiguous fp32 of H elements");
            gb = a.dense(a.entry(grad_w, 2, 1), at::kFloat, x.cols, true, true, "grad_bias must be contiguous fp32 of H elements");
            if (!want_w) gw = nullptr;
            if (!want_bias) gb = nullptr;
        } else {
            if (accumulate && (want_w || want_bias)) a.refuse("accumulate_w needs the tensors to add to (grad_w)");
            if (want_w) own[1] = made(a.like(), at::kFloat, {x.cols});
            if (want_bias) own[2] = made(a.like(), at::kFloat, {x.cols});
            gw = want_w ? &own[1] : nullptr;
            gb = want_bias ? &own[2] : nullptr;
        }
        if (gw || gb) ws = scratch(ws, tppo_layer_norm_backward_workspace_bytes(l.M, x.cols), a.like(), own[3]);
        const int rc = run([&] {
            return tppo_layer_norm_backward(memory(gy.t), gy.ld, type_of(*gy.t), memory(x.t), x.rows, x.cols, x.ld, type_of(*x.t), memory(w),
                                            type_of(*w), memory<float>(mean), memory<float>(rstd), memory<int32_t>(l.rows), l.M,
                                            memory<int64_t>(l.m_actual), memory(gx), gx ? to.ld : x.cols, type_of(gx ? *gx : *x.t),
                                            memory<int32_t>(index), to.rows, memory<float>(gw), memory<float>(gb), accumulate, memory(ws),
                                            bytes_of(ws), memory<int32_t>(status), s);
        });
        return rc ? PyLong_FromLong(rc) : tuple_of({gx, gw, gb});
    });
}

// (logits, experts, rows, M, m_actual, coefficient, status, workspace, out, stream), and for the derivative (..., out, scale, counts_in,
// token_denominator, out_index, grad, stream)
template <bool BACKWARD>
PyObject* balance(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&] {
        Taken a(BACKWARD ? "tppo_balance_loss_backward" : "tppo_balance_loss", args, n, BACKWARD ? 15 : 10);
        const Rows z(a, a.tensor(false, "logits must be a device matrix"), "logits must be a device matrix");
        if (!known(*z.t)) a.refuse("logits must be fp32 or bf16");
        const Rows ids(a, a.tensor(false, "experts must be a device matrix"), "experts must be a device matrix");
        if (ids.t->scalar_type() != at::kInt || ids.rows != z.rows) a.refuse("experts must be int32 [n_rows, k]");
        const Listed l(a, z.rows);
        const float coefficient = a.f32();
        const at::Tensor* status = status_word(a);
        const at::Tensor* ws = workspace_of(a);
        PyObject* out = a.next();
        at::Tensor own[5];
        const at::Tensor *loss, *counts, *mean;
        if (out == Py_None) {
            own[0] = made(a.like(), at::kFloat, {1});
            own[1] = made(a.like(), at::kLong, {z.cols});
            own[2] = made(a.like(), at::kFloat, {z.cols});
            loss = &own[0];
            counts = &own[1];
            mean = &own[2];
        } else {
            loss = a.dense(a.entry(out, 3, 0), at::kFloat, 1, true, true, "loss must be one fp32 element");
            counts = a.dense(a.entry(out, 3, 1), at::kLong, z.cols, true, true, "counts must be contiguous int64 of E elements");
            mean = a.dense(a.entry(out, 3, 2), at::kFloat, z.cols, true, true, "mean_prob must be contiguous fp32 of E elements");
        }
        ws = scratch(ws, tppo_balance_loss_workspace_bytes(l.M, z.cols), a.like(), own[3]);
        if constexpr (!BACKWARD) {
            void* s = a.stream();
            const int rc = run([&] {
                return tppo_balance_loss(memory(z.t), z.rows, z.cols, z.ld, type_of(*z.t), memory<int32_t>(ids.t), ids.cols, ids.ld,
                                         memory<int32_t>(l.rows), l.M, memory<int64_t>(l.m_actual), coefficient, memory<float>(loss),
                                         memory<int64_t>(counts), memory<float>(mean), memory(ws), bytes_of(ws), memory<int32_t>(status), s);
            });
            return rc ? PyLong_FromLong(rc) : tuple_of({loss, counts, mean});
        } else {
            const float scale = a.f32();
            const at::Tensor* counts_in = a.dense(a.next(), at::kLong, z.cols, true, true, "counts_in must be contiguous int64 of E elements");
            const int64_t denominator = a.i64(0);
            const at::Tensor* index = index_of(a, l.M);
            PyObject* grad = a.next();
            void* s = a.stream();
            const at::Tensor* g = &own[4];
            if (grad == Py_None) {
                if (index) a.refuse("out_index needs the tensor that it points into (grad)");
                own[4] = made(a.like(), z.t->scalar_type(), {l.M, z.cols});
            } else {
                g = a.checked(grad, false, "grad must be a device matrix");
            }
            const Rows to(a, g, "grad must be a device matrix");
            if (g->scalar_type() != z.t->scalar_type() || to.cols != z.cols || (!index && to.rows < l.M))
                a.refuse("grad must be [M, E] of the logits' type");
            const int rc = run([&] {
                return tppo_balance_loss_backward(memory(z.t), z.rows, z.cols, z.ld, type_of(*z.t), memory<int32_t>(ids.t), ids.cols, ids.ld,
                                                  memory<int32_t>(l.rows), l.M, memory<int64_t>(l.m_actual), coefficient, scale,
                                                  memory<int64_t>(counts_in), denominator, memory(g), to.ld, memory<int32_t>(index), to.rows,
                                                  memory<float>(loss), memory<int64_t>(counts), memory<float>(mean), memory(ws), bytes_of(ws),
                                                  memory<int32_t>(status), s);
            });
            return rc ? PyLong_FromLong(rc) : tuple_of({g, loss, counts, mean});
        }
    });
}

// (g, steps, a, b, c, eps, scale, workspace, out, stream)
PyObject* orthogonalize(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&] {
        Taken a("tppo_orthogonalize", args, n, 10);
        const Rows g(a, a.tensor(false, "g must be device matrices"), "g must be device matrices", true);
        if (!known(*g.t)) a.refuse("g must be fp32 or bf16");
        const int64_t steps = a.i64(0);
        float v[5];
        for (float& f : v) f = a.f32();
        const at::Tensor* ws = workspace_of(a);
        PyObject* out = a.next();
        void* s = a.stream();
        at::Tensor own[2];
        const at::Tensor* o = &own[0];
        if (out == Py_None) own[0] = made(a.like(), at::kBFloat16, g.t->sizes());
        else o = a.checked(out, false, "out must be device matrices");
        if (o->scalar_type() != at::kBFloat16 || o->sizes() != g.t->sizes()) a.refuse("out must be bf16 of g's shape");
        const Rows to(a, o, "out must be device matrices", true);
        if (steps < INT32_MIN || steps > INT32_MAX) a.refuse("steps");
        ws = scratch(ws, tppo_orthogonalize_workspace_bytes(g.count, g.rows, g.cols), a.like(), own[1]);
        const int rc = run([&] {
            return tppo_orthogonalize(memory(g.t), g.count, g.rows, g.cols, g.ld, g.each, type_of(*g.t), (int32_t)steps, v[0], v[1], v[2], v[3],
                                      v[4], memory(o), to.ld, to.each, memory(ws), bytes_of(ws), s);
        });
        return rc ? PyLong_FromLong(rc) : tuple_of({o});
    });
}

template <PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method<entry<select, 19>>("select"),
                         method<entry<token_logprobs, 18>>("token_logprobs"),
                         method<entry<egae<tppo_egae>, 15>>("egae"),
                         method<entry<egae<tppo_egae_terminal>, 15>>("egae_terminal"),
                         method<entry<ppo_losses, 20>>("ppo_losses"),
                         method<entry<ppo_losses_backward, 27>>("ppo_losses_backward"),
                         method<entry<value_head, 14>>("value_head"),
                         method<entry<select_workspace_bytes, 2>>("select_workspace_bytes"),
                         method<entry<plan_bytes, 2>>("plan_bytes"),
                         method<empties>("empties"),
                         method<layer_norm>("layer_norm"),
                         method<layer_norm_backward>("layer_norm_backward"),
                         method<balance<false>>("balance_loss"),
                         method<balance<true>>("balance_loss_backward"),
                         method<orthogonalize>("orthogonalize"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
