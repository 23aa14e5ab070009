// Plan.forward for ordinary calls, as one native call: checks of shapes and types, the output's allocation, the current
// stream and smha_forward.  A call with a short kernel lasts as long as its host side: 8 us in Python through ctypes, 4.7 so, of which
// the launch is 3.5 and the output's allocation 0.6 (window 1 x 2 x 128 x 64 8.0 -> 4.9 us a call; a launch of torch's own 4 to 5).
//
// It answers for plain dense tensors only, and leaves every other call, those that are errors among them, to
// binding.smha_forward (by returning None): subclasses, named, functorch-wrapped, tracked by a mode, other layouts, a shape or type
// that does not fit.
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/core/Allocator.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/csrc/autograd/python_variable.h>

#include "smha.h"

namespace {

using Forward = decltype(&smha_forward);

bool plain(PyObject *obj, int64_t dims = 4) {
    if (!THPVariable_CheckExact(obj)) return false;
    const at::Tensor &t = THPVariable_Unpack(obj);
    constexpr c10::DispatchKeySet ordinary({c10::DispatchKey::CUDA, c10::DispatchKey::AutogradCUDA, c10::DispatchKey::ADInplaceOrView,
                                            c10::DispatchKey::AutocastCUDA});
    return t.defined() && (t.key_set() | ordinary) == ordinary && t.is_cuda() && t.dim() == dims && !t.has_names() &&
           !t.unsafeGetTensorImpl()->has_symbolic_sizes_strides();
}

int code_of(at::ScalarType type) {
    return type == at::kHalf ? SMHA_F16 : type == at::kBFloat16 ? SMHA_BF16 : type == at::kFloat ? SMHA_F32 : -1;
}

// the three leading strides, or null where the tensor is packed; ok is cleared where a head's elements do not follow each other
const int64_t *strides_of(const at::Tensor &t, bool &ok) {
    if (t.is_contiguous()) return nullptr;
    ok = ok && t.strides()[3] == 1;
    return t.strides().data();
}

// forward(address of smha_forward, plan handle, S, Sk, Q, K, V, out or None, out_dtype or None, scale, kernel) -> the output, a status that is
// not SMHA_OK, or None
PyObject *forward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 11 || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) Py_RETURN_NONE;
    if (!plain(args[4]) || !plain(args[5]) || !plain(args[6])) Py_RETURN_NONE;
    if (!PyLong_CheckExact(args[1]) || !PyFloat_CheckExact(args[9]) || !PyLong_CheckExact(args[10])) Py_RETURN_NONE;
    const auto entry = reinterpret_cast<Forward>(PyLong_AsVoidPtr(args[0]));
    const auto *plan = static_cast<const smha_plan_t *>(PyLong_AsVoidPtr(args[1]));
    const int64_t S = PyLong_AsLongLong(args[2]), Sk = PyLong_AsLongLong(args[3]);
    const double scale = PyFloat_AS_DOUBLE(args[9]);
    const long kernel = PyLong_AsLong(args[10]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    const at::Tensor &q = THPVariable_Unpack(args[4]), &k = THPVariable_Unpack(args[5]), &v = THPVariable_Unpack(args[6]);
    const at::ScalarType type = q.scalar_type();
    const int in = code_of(type);
    if (in < 0 || in == SMHA_F32 || k.scalar_type() != type || v.scalar_type() != type) Py_RETURN_NONE;
    const at::IntArrayRef qn = q.sizes(), kn = k.sizes();
    if (kn != v.sizes() || qn[0] != kn[0] || qn[1] != kn[1] || qn[3] != kn[3] || qn[2] != S || kn[2] != Sk) Py_RETURN_NONE;
    if (qn[0] > INT32_MAX || qn[1] > INT32_MAX || qn[3] > INT32_MAX) Py_RETURN_NONE;
    at::Tensor o;
    if (args[7] == Py_None) {
        at::ScalarType out_type = type;
        if (args[8] != Py_None) {
            if (!THPDtype_Check(args[8])) Py_RETURN_NONE;
            out_type = reinterpret_cast<THPDtype *>(args[8])->scalar_type;
        }
        if (code_of(out_type) < 0) Py_RETURN_NONE;
        o = at::empty(qn, q.options().dtype(out_type), at::MemoryFormat::Contiguous);
    } else {
        if (!plain(args[7])) Py_RETURN_NONE;
        o = THPVariable_Unpack(args[7]);
        if (o.sizes() != qn) Py_RETURN_NONE;
    }
    const int out = code_of(o.scalar_type());
    bool ok = out >= 0;
    const int64_t *qs = strides_of(q, ok), *ks = strides_of(k, ok), *vs = strides_of(v, ok), *os = strides_of(o, ok);
    if (!ok) Py_RETURN_NONE;
    void *const stream = c10::hip::getCurrentHIPStream(q.device().index()).stream();
    const void *const qp = q.data_ptr(), *const kp = k.data_ptr(), *const vp = v.data_ptr();
    void *const op = o.data_ptr();
    smha_status_t status;
    Py_BEGIN_ALLOW_THREADS
    status = entry(plan, qp, kp, vp, op, (int)qn[0], (int)qn[1], (int)qn[3], (smha_dtype_t)in, (smha_dtype_t)out, qs, ks, vs, os, (float)scale,
                   (smha_kernel_t)kernel, stream);
    Py_END_ALLOW_THREADS
    if (status != SMHA_OK) return PyLong_FromLong((long)status);
    if (args[7] != Py_None) {
        Py_INCREF(args[7]);
        return args[7];
    }
    return THPVariable_Wrap(std::move(o));
    END_HANDLE_TH_ERRORS
}

// ---- attention with sinks, attention on a cache, eviction, a cache held in 4 bits (sink.py, cache.py and packed.py: the same calls, and the errors of those that
// are refused here)

struct Entries {
    decltype(&smha_sink_forward) sink_forward;
    decltype(&smha_sink_backward) sink_backward;
    decltype(&smha_sink_workspace) sink_workspace;
    decltype(&smha_cache_forward) cache_forward;
    decltype(&smha_cache_workspace) cache_workspace;
    decltype(&smha_cache_evict) cache_evict;
    decltype(&smha_cache_evict_workspace) cache_evict_workspace;
    decltype(&smha_packed_write) packed_write;
    decltype(&smha_packed_read) packed_read;
    decltype(&smha_packed_forward) packed_forward;
    decltype(&smha_packed_workspace) packed_workspace;
} entries;
constexpr int kEntries = 11;

// link(the addresses of those, in that order)
PyObject *link(PyObject *, PyObject *const *args, Py_ssize_t n) {
    void *at[kEntries];
    if (n != kEntries) {
        PyErr_SetString(PyExc_TypeError, "eleven addresses");
        return nullptr;
    }
    for (int i = 0; i < kEntries; ++i) at[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
    entries = {reinterpret_cast<decltype(entries.sink_forward)>(at[0]), reinterpret_cast<decltype(entries.sink_backward)>(at[1]),
               reinterpret_cast<decltype(entries.sink_workspace)>(at[2]), reinterpret_cast<decltype(entries.cache_forward)>(at[3]),
               reinterpret_cast<decltype(entries.cache_workspace)>(at[4]), reinterpret_cast<decltype(entries.cache_evict)>(at[5]),
               reinterpret_cast<decltype(entries.cache_evict_workspace)>(at[6]), reinterpret_cast<decltype(entries.packed_write)>(at[7]),
               reinterpret_cast<decltype(entries.packed_read)>(at[8]), reinterpret_cast<decltype(entries.packed_forward)>(at[9]),
               reinterpret_cast<decltype(entries.packed_workspace)>(at[10])};
    Py_RETURN_NONE;
}

// {batch, head, token} strides, null where packed; what a dimension of size 1 has is not looked at.
struct Strides3 {
    int64_t s[3];
    const int64_t *ptr = nullptr;
    bool ok = true;
    explicit Strides3(const at::Tensor &t) {
        if (t.is_contiguous()) return;
        const auto n = t.sizes(), st = t.strides();
        ok = st[3] == 1 || n[3] == 1;
        s[0] = n[0] > 1 ? st[0] : 0;
        s[1] = n[1] > 1 ? st[1] : 0;
        s[2] = n[2] > 1 ? st[2] : n[3];
        ptr = s;
    }
    Strides3(const Strides3 &) = delete;
};

bool int_from(PyObject *o, int &to) {  // 0 .. 2^31 - 1
    if (!PyLong_CheckExact(o)) return false;
    const int64_t v = PyLong_AsLongLong(o);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    to = (int)v;
    return v >= 0 && v <= INT32_MAX;
}

bool small_sizes(const at::Tensor &t) {
    for (const int64_t n : t.sizes())
        if (n > INT32_MAX) return false;
    return true;
}

// int32 [B] on q's GPU, or None
bool per_sequence(PyObject *o, const at::Tensor &q, const int32_t *&to, at::Tensor &held) {
    to = nullptr;
    if (o == Py_None) return true;
    if (!plain(o, 1)) return false;
    held = THPVariable_Unpack(o);
    if (held.scalar_type() != at::kInt || held.size(0) != q.size(0) || held.device() != q.device() || !held.is_contiguous()) return false;
    to = held.data_ptr<int32_t>();
    return true;
}

bool heads_fit(const at::Tensor &q, const at::Tensor &k, const at::Tensor &v) {
    const int type = code_of(q.scalar_type());
    return (type == SMHA_F16 || type == SMHA_BF16) && k.scalar_type() == q.scalar_type() && v.scalar_type() == q.scalar_type() && k.sizes() == v.sizes() &&
           q.size(0) == k.size(0) && q.size(3) == k.size(3) && k.size(1) > 0 && q.size(1) % k.size(1) == 0 && k.device() == q.device() &&
           v.device() == q.device() && small_sizes(q) && small_sizes(k);
}

struct SinkCall {
    int window, n_sink;
    float scale;
};

smha_status_t run_sink_forward(const at::Tensor &q, const at::Tensor &k, const at::Tensor &v, at::Tensor &o, float *lse, void *rest, const int32_t *offsets,
                               const int32_t *lengths, const SinkCall &c) {
    const Strides3 qs(q), ks(k), vs(v);
    return entries.sink_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse, rest, (int)q.size(0), (int)q.size(1), (int)k.size(1),
                                (int)q.size(2), (int)k.size(2), (int)q.size(3), (smha_dtype_t)code_of(q.scalar_type()), qs.ptr, ks.ptr, vs.ptr, nullptr, offsets, lengths,
                                c.window, c.n_sink, c.scale, c10::hip::getCurrentHIPStream(q.device().index()).stream());
}

// Memory for the work that a call enqueues, from torch's allocator for the current stream, on the current device.
c10::DataPtr scratch(size_t bytes) { return c10::GetAllocator(c10::DeviceType::CUDA)->allocate(bytes); }

at::Tensor packed_like(const at::Tensor &t) { return at::empty(t.sizes(), t.options(), at::MemoryFormat::Contiguous); }

int64_t lse_bytes(const at::Tensor &q) { return (q.size(0) * q.size(1) * q.size(2) * 4 + 15) / 16 * 16; }

// Whether smha_sink_backward reads a tensor as it lies: autograd may hand on gradients that are expanded, transposed, or of more than 2 GiB between a
// head's first and last row, and hooks of saved tensors may give those back with other strides.
bool taken(const at::Tensor &g) {
    if (reinterpret_cast<uintptr_t>(g.data_ptr()) % 16) return false;
    const Strides3 s(g);
    if (!s.ptr) return true;
    return s.ok && s.s[0] % 8 == 0 && s.s[1] % 8 == 0 && s.s[2] % 8 == 0 && s.s[2] >= g.size(3) && s.s[2] <= INT32_MAX &&
           ((g.size(2) + 128) * s.s[2] + g.size(3)) * 2 <= INT32_MAX;
}

at::Tensor readable(const at::Tensor &t) { return taken(t) ? t : t.clone(at::MemoryFormat::Contiguous); }

// The backward pass of one call.
struct SinkBackward : torch::autograd::Node {
    torch::autograd::SavedVariable q_, k_, v_, o_, kept_, offsets_, lengths_;  // kept: lse, then what O's rounding left out
    SinkCall call_;

    std::string name() const override { return "SinkAttentionBackward"; }

    void release_variables() override {
        const std::lock_guard<std::mutex> lock(mutex_);
        for (auto *t : {&q_, &k_, &v_, &o_, &kept_, &offsets_, &lengths_}) t->reset_data();
    }

    torch::autograd::variable_list apply(torch::autograd::variable_list &&grads) override {
        const std::lock_guard<std::mutex> lock(mutex_);
        if (!grads[0].defined()) return torch::autograd::variable_list(3);
        at::Tensor q = q_.unpack(), k = k_.unpack(), v = v_.unpack(), o = o_.unpack(shared_from_this()), kept = kept_.unpack(), offsets = offsets_.unpack(),
                   lengths = lengths_.unpack();
        at::Tensor g = grads[0].detach(), dq, dk, dv;
        {
            const at::AutoGradMode off(false);
            for (at::Tensor *t : {&q, &k, &v, &g}) *t = readable(*t);
            for (at::Tensor *t : {&o, &kept, &offsets, &lengths})
                if (t->defined()) *t = t->contiguous();
            dq = packed_like(q);
            dk = packed_like(k);
            dv = packed_like(v);
            const int B = (int)q.size(0), H = (int)q.size(1), Hkv = (int)k.size(1), Sq = (int)q.size(2), Sk = (int)k.size(2), d = (int)q.size(3);
            const c10::DeviceGuard guard(q.device());
            size_t need = 0;
            smha_status_t st = entries.sink_workspace(B, H, Hkv, Sq, Sk, d, call_.window, call_.n_sink, &need);
            const Strides3 qs(q), ks(k), vs(v), ds(g);
            if (st == SMHA_OK) {
                const c10::DataPtr ws = scratch(need);
                st = entries.sink_backward(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), static_cast<char *>(kept.data_ptr()) + lse_bytes(q), static_cast<const float *>(kept.data_ptr()), g.data_ptr(), dq.data_ptr(),
                                           dk.data_ptr(), dv.data_ptr(), B, H, Hkv, Sq, Sk, d, (smha_dtype_t)code_of(q.scalar_type()), qs.ptr, ks.ptr, vs.ptr, nullptr, ds.ptr,
                                           nullptr, nullptr, nullptr, offsets.defined() ? offsets.data_ptr<int32_t>() : nullptr,
                                           lengths.defined() ? lengths.data_ptr<int32_t>() : nullptr, call_.window, call_.n_sink, call_.scale, ws.get(), need,
                                           c10::hip::getCurrentHIPStream(q.device().index()).stream());
            }
            TORCH_CHECK(st == SMHA_OK, "smha_sink_backward: status ", (int)st);
        }
        torch::autograd::variable_list out = {dq, dk, dv};
        if (at::GradMode::is_enabled()) {  // (a graph of the gradients is wanted: they have none of their own)
            for (auto &t : out) t.requires_grad_();
            out = (*std::make_shared<torch::autograd::DelayedError>("sink_attention cannot be differentiated twice", (int64_t)out.size()))(std::move(out));
        }
        for (size_t i = 0; i < 3; ++i)
            if (!task_should_compute_output(i)) out[i] = at::Tensor();
        return out;
    }
};

// The forward of a call whose gradients may be wanted: the output, or a status.
smha_status_t sink_with_graph(const at::Tensor &q, const at::Tensor &k, const at::Tensor &v, const at::Tensor &offsets, const at::Tensor &lengths, const SinkCall &c,
                              at::Tensor &o) {
    using torch::autograd::SavedVariable;
    at::Tensor kept;
    {
        const at::AutoGradMode off(false);
        o = packed_like(q);
        kept = at::empty({lse_bytes(q) + q.numel() * (int64_t)q.element_size()}, q.options().dtype(at::kByte));
        const smha_status_t st = run_sink_forward(q, k, v, o, static_cast<float *>(kept.data_ptr()), static_cast<char *>(kept.data_ptr()) + lse_bytes(q), offsets.defined() ? offsets.data_ptr<int32_t>() : nullptr,
                                                  lengths.defined() ? lengths.data_ptr<int32_t>() : nullptr, c);
        if (st != SMHA_OK) return st;
    }
    const auto node = std::shared_ptr<SinkBackward>(new SinkBackward(), torch::autograd::deleteNode);
    node->set_next_edges(torch::autograd::collect_next_edges(q, k, v));
    node->call_ = c;
    torch::autograd::set_history(o, node);
    node->q_ = SavedVariable(q, false);
    node->k_ = SavedVariable(k, false);
    node->v_ = SavedVariable(v, false);
    node->o_ = SavedVariable(o, true);
    node->kept_ = SavedVariable(kept, false);
    node->offsets_ = SavedVariable(offsets, false);
    node->lengths_ = SavedVariable(lengths, false);
    return SMHA_OK;
}

// Forward mode, which the general way refuses (it goes by itself: neither gradients that are required nor that are switched off say that there is none).
bool has_tangent(const at::Tensor &t) { return t._fw_grad(0).defined(); }

// sink_attention(q, k, v, window, n_sink, offsets, lengths, scale) -> the output, a status, or None
PyObject *sink_attention(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 8 || !entries.sink_forward || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) Py_RETURN_NONE;
    if (!plain(args[0]) || !plain(args[1]) || !plain(args[2]) || !PyFloat_CheckExact(args[7])) Py_RETURN_NONE;
    const at::Tensor &q = THPVariable_Unpack(args[0]), &k = THPVariable_Unpack(args[1]), &v = THPVariable_Unpack(args[2]);
    SinkCall c{0, 0, (float)PyFloat_AS_DOUBLE(args[7])};
    if (!int_from(args[3], c.window) || !int_from(args[4], c.n_sink) || !heads_fit(q, k, v)) Py_RETURN_NONE;
    const int32_t *offsets, *lengths;
    at::Tensor offsets_t, lengths_t;
    if (!per_sequence(args[5], q, offsets, offsets_t) || !per_sequence(args[6], q, lengths, lengths_t)) Py_RETURN_NONE;
    if (!Strides3(q).ok || !Strides3(k).ok || !Strides3(v).ok) Py_RETURN_NONE;
    if (has_tangent(q) || has_tangent(k) || has_tangent(v)) Py_RETURN_NONE;
    const c10::DeviceGuard guard(q.device());
    at::Tensor o;
    if (at::GradMode::is_enabled() && (q.requires_grad() || k.requires_grad() || v.requires_grad())) {
        const smha_status_t st = sink_with_graph(q, k, v, offsets_t, lengths_t, c, o);
        if (st != SMHA_OK) return PyLong_FromLong((long)st);
    } else {
        o = packed_like(q);
        const smha_status_t st = run_sink_forward(q, k, v, o, nullptr, nullptr, offsets, lengths, c);
        if (st != SMHA_OK) return PyLong_FromLong((long)st);
    }
    return THPVariable_Wrap(std::move(o));
    END_HANDLE_TH_ERRORS
}

// A tensor that was written: autograd refuses to go back through what was saved of it.
void written(const at::Tensor &t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// A derivative of it would be lost, or it would be written though it is a leaf.
bool wants_derivative(const at::Tensor &t) { return (at::GradMode::is_enabled() && t.requires_grad()) || has_tangent(t); }

// cache_attention(q, k, v, lengths, window, n_sink, prefix keys or None, prefix values or None, weights or None, scale) -> the output, a status, or None
PyObject *cache_attention(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 10 || !entries.cache_forward || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) Py_RETURN_NONE;
    if (!plain(args[0]) || !plain(args[1]) || !plain(args[2]) || !PyFloat_CheckExact(args[9])) Py_RETURN_NONE;
    const at::Tensor &q = THPVariable_Unpack(args[0]), &k = THPVariable_Unpack(args[1]), &v = THPVariable_Unpack(args[2]);
    if (!heads_fit(q, k, v) || wants_derivative(q) || wants_derivative(k) || wants_derivative(v)) Py_RETURN_NONE;
    const int32_t *lengths;
    at::Tensor lengths_t;
    int window, n_sink;
    if (args[3] == Py_None || !per_sequence(args[3], q, lengths, lengths_t) || !int_from(args[4], window) || !int_from(args[5], n_sink)) Py_RETURN_NONE;
    const int B = (int)q.size(0), H = (int)q.size(1), T = (int)q.size(2), d = (int)q.size(3), Hkv = (int)k.size(1), Sk = (int)k.size(2);
    int P = 0;
    const void *pk = nullptr, *pv = nullptr;
    if (args[6] != Py_None || args[7] != Py_None) {
        if (!plain(args[6], 3) || !plain(args[7], 3)) Py_RETURN_NONE;
        const at::Tensor &a = THPVariable_Unpack(args[6]), &b = THPVariable_Unpack(args[7]);
        if (a.sizes() != b.sizes() || a.size(0) != Hkv || a.size(2) != d || a.size(1) > INT32_MAX || a.scalar_type() != q.scalar_type() ||
            b.scalar_type() != q.scalar_type() || a.device() != q.device() || b.device() != q.device() || !a.is_contiguous() || !b.is_contiguous() || wants_derivative(a) || wants_derivative(b))
            Py_RETURN_NONE;
        P = (int)a.size(1);
        pk = a.data_ptr();
        pv = b.data_ptr();
    }
    float *weights = nullptr;
    at::Tensor weights_t;
    if (args[8] != Py_None) {
        if (!plain(args[8], 3)) Py_RETURN_NONE;
        const at::Tensor &w = THPVariable_Unpack(args[8]);
        if (w.scalar_type() != at::kFloat || w.size(0) != B || w.size(1) != Hkv || w.size(2) != Sk || w.device() != q.device() || !w.is_contiguous() || wants_derivative(w))
            Py_RETURN_NONE;
        weights_t = w;
        weights = w.data_ptr<float>();
    }
    const Strides3 qs(q), ks(k), vs(v);
    if (!qs.ok || !ks.ok || !vs.ok) Py_RETURN_NONE;
    const c10::DeviceGuard guard(q.device());
    size_t need = 0;
    smha_status_t st = entries.cache_workspace(B, H, Hkv, T, Sk, P, d, window, n_sink, weights != nullptr, &need);
    if (st != SMHA_OK) return PyLong_FromLong((long)st);
    const at::AutoGradMode off(false);
    at::Tensor o = packed_like(q);
    const c10::DataPtr ws = need ? scratch(need) : c10::DataPtr();
    st = entries.cache_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), pk, pv, o.data_ptr(), weights, lengths, B, H, Hkv, T, Sk, P, d,
                               (smha_dtype_t)code_of(q.scalar_type()), qs.ptr, ks.ptr, vs.ptr, nullptr, nullptr, nullptr, nullptr, window, n_sink,
                               (float)PyFloat_AS_DOUBLE(args[9]), ws.get(), need, c10::hip::getCurrentHIPStream(q.device().index()).stream());
    if (st != SMHA_OK) return PyLong_FromLong((long)st);
    if (weights) written(weights_t);
    return THPVariable_Wrap(std::move(o));
    END_HANDLE_TH_ERRORS
}

// cache_evict(k, v, weights, positions, lengths, budget, recent) -> (weights, positions, lengths), a status, or None
PyObject *cache_evict(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 7 || !entries.cache_evict || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) Py_RETURN_NONE;
    if (!plain(args[0]) || !plain(args[1]) || !plain(args[2], 3) || !plain(args[3], 3) || !plain(args[4], 1)) Py_RETURN_NONE;
    const at::Tensor &k = THPVariable_Unpack(args[0]), &v = THPVariable_Unpack(args[1]), &w = THPVariable_Unpack(args[2]), &p = THPVariable_Unpack(args[3]),
                     &len = THPVariable_Unpack(args[4]);
    int budget, recent;
    if (!int_from(args[5], budget) || !int_from(args[6], recent)) Py_RETURN_NONE;
    const int type = code_of(k.scalar_type());
    if ((type != SMHA_F16 && type != SMHA_BF16) || v.scalar_type() != k.scalar_type() || k.sizes() != v.sizes() || v.device() != k.device() || !small_sizes(k)) Py_RETURN_NONE;
    if (wants_derivative(k) || wants_derivative(v) || wants_derivative(w)) Py_RETURN_NONE;
    for (const at::Tensor *t : {&w, &p})
        if (t->sizes() != k.sizes().slice(0, 3) || t->device() != k.device() || !t->is_contiguous()) Py_RETURN_NONE;
    if (w.scalar_type() != at::kFloat || p.scalar_type() != at::kInt || len.scalar_type() != at::kInt || len.size(0) != k.size(0) || len.device() != k.device() ||
        !len.is_contiguous())
        Py_RETURN_NONE;
    for (const at::Tensor *t : {&k, &v})
        for (int i = 0; i < 3; ++i)
            if (t->size(i) > 1 && t->stride(i) < t->size(3)) Py_RETURN_NONE;
    const Strides3 ks(k), vs(v);
    if (!ks.ok || !vs.ok) Py_RETURN_NONE;
    const int B = (int)k.size(0), Hkv = (int)k.size(1), Sk = (int)k.size(2), d = (int)k.size(3);
    const c10::DeviceGuard guard(k.device());
    size_t need = 0;
    smha_status_t st = entries.cache_evict_workspace(B, Hkv, Sk, d, budget, recent, &need);
    if (st != SMHA_OK) return PyLong_FromLong((long)st);
    const at::AutoGradMode off(false);
    at::Tensor w2 = packed_like(w), p2 = packed_like(p), len2 = packed_like(len);
    const c10::DataPtr ws = scratch(need);
    st = entries.cache_evict(k.data_ptr(), v.data_ptr(), w.data_ptr<float>(), p.data_ptr<int32_t>(), len.data_ptr<int32_t>(), w2.data_ptr<float>(),
                             p2.data_ptr<int32_t>(), len2.data_ptr<int32_t>(), B, Hkv, Sk, d, budget, recent, ks.ptr, vs.ptr, ws.get(), need,
                             c10::hip::getCurrentHIPStream(k.device().index()).stream());
    if (st != SMHA_OK) return PyLong_FromLong((long)st);
    written(k);
    written(v);
    PyObject *out = PyTuple_New(3);
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(w2)));
    PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(std::move(p2)));
    PyTuple_SET_ITEM(out, 2, THPVariable_Wrap(std::move(len2)));
    return out;
    END_HANDLE_TH_ERRORS
}

// A packed cache: uint8 [B,Hkv,Sk,row], keys and values alike.  The columns of its rows, or 0.
int packed_width(const at::Tensor &k, const at::Tensor &v) {
    if (k.scalar_type() != at::kByte || v.scalar_type() != at::kByte || k.sizes() != v.sizes() || v.device() != k.device() || !small_sizes(k)) return 0;
    const int64_t row = k.size(3);
    for (int d = 8; d <= 128; d += 8)
        if (4 * ((d + 31) / 32) + d / 2 == row) return d;
    return 0;
}

// Rows that are written must not overlap (the entry point looks at all strides together).
bool steps_over_rows(const at::Tensor &t) {
    for (int i = 0; i < 3; ++i)
        if (t.size(i) > 1 && t.stride(i) < t.size(3)) return false;
    return true;
}

// Whether [B][Hkv][T][d] of `size` bytes is of a size that the entry points take: what they would refuse is not allocated first.
bool outputs_fit(const at::Tensor &cache, int64_t T, int64_t d, int64_t size) {
    const __int128 heads = (__int128)cache.size(0) * cache.size(1);
    return heads * T <= SMHA_PACKED_MOST_ROWS && (T + 64) * d * size < (int64_t)1 << 31;
}

PyObject *pair_of(at::Tensor &&a, at::Tensor &&b) {
    PyObject *out = PyTuple_New(2);
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(a)));
    PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(std::move(b)));
    return out;
}

// packed_write(new keys, new values, k, v, lengths, offsets or None, values) -> True, (keys, values), a status, or None
PyObject *packed_write(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 7 || !entries.packed_write || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) Py_RETURN_NONE;
    if (!plain(args[0]) || !plain(args[1]) || !plain(args[2]) || !plain(args[3]) || !PyBool_Check(args[6])) Py_RETURN_NONE;
    const at::Tensor &kn = THPVariable_Unpack(args[0]), &vn = THPVariable_Unpack(args[1]), &k = THPVariable_Unpack(args[2]), &v = THPVariable_Unpack(args[3]);
    const int d = packed_width(k, v), type = code_of(kn.scalar_type());
    if (!d || (type != SMHA_F16 && type != SMHA_BF16) || vn.scalar_type() != kn.scalar_type() || kn.sizes() != vn.sizes() || kn.device() != k.device() || vn.device() != k.device() ||
        kn.size(0) != k.size(0) || kn.size(1) != k.size(1) || kn.size(3) != d || !small_sizes(kn) || wants_derivative(kn) || wants_derivative(vn) || !steps_over_rows(k) || !steps_over_rows(v))
        Py_RETURN_NONE;
    const int32_t *lengths, *offsets;
    at::Tensor lengths_t, offsets_t;
    if (args[4] == Py_None || !per_sequence(args[4], k, lengths, lengths_t) || !per_sequence(args[5], k, offsets, offsets_t)) Py_RETURN_NONE;
    const Strides3 ns(kn), ms(vn), ks(k), vs(v);
    if (!ns.ok || !ms.ok || !ks.ok || !vs.ok) Py_RETURN_NONE;
    const c10::DeviceGuard guard(k.device());
    const at::AutoGradMode off(false);
    at::Tensor keys, values;
    if (args[6] == Py_True) {
        if (!outputs_fit(k, kn.size(2), d, 2)) Py_RETURN_NONE;
        keys = packed_like(kn);
        values = packed_like(vn);
    }
    const smha_status_t st = entries.packed_write(kn.data_ptr(), vn.data_ptr(), k.data_ptr(), v.data_ptr(), keys.defined() ? keys.data_ptr() : nullptr,
                                                  values.defined() ? values.data_ptr() : nullptr, lengths, offsets, (int)k.size(0), (int)k.size(1), (int)kn.size(2), (int)k.size(2), d,
                                                  (smha_dtype_t)type, ns.ptr, ms.ptr, ks.ptr, vs.ptr, c10::hip::getCurrentHIPStream(k.device().index()).stream());
    if (st != SMHA_OK) return PyLong_FromLong((long)st);
    written(k);
    written(v);
    if (!keys.defined()) Py_RETURN_TRUE;
    return pair_of(std::move(keys), std::move(values));
    END_HANDLE_TH_ERRORS
}

// packed_read(k, v, lengths, offsets or None, tokens or None, dtype) -> (keys, values), a status, or None
PyObject *packed_read(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 6 || !entries.packed_read || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) Py_RETURN_NONE;
    if (!plain(args[0]) || !plain(args[1]) || !THPDtype_Check(args[5])) Py_RETURN_NONE;
    const at::Tensor &k = THPVariable_Unpack(args[0]), &v = THPVariable_Unpack(args[1]);
    const at::ScalarType out_type = reinterpret_cast<THPDtype *>(args[5])->scalar_type;
    const int d = packed_width(k, v), type = code_of(out_type);
    if (!d || type < 0) Py_RETURN_NONE;
    const int32_t *lengths, *offsets;
    at::Tensor lengths_t, offsets_t;
    if (args[2] == Py_None || !per_sequence(args[2], k, lengths, lengths_t) || !per_sequence(args[3], k, offsets, offsets_t)) Py_RETURN_NONE;
    int tokens = (int)k.size(2);
    if (args[4] != Py_None && !int_from(args[4], tokens)) Py_RETURN_NONE;
    const Strides3 ks(k), vs(v);
    if (!ks.ok || !vs.ok || !outputs_fit(k, tokens, d, at::elementSize(out_type))) Py_RETURN_NONE;
    const c10::DeviceGuard guard(k.device());
    const at::AutoGradMode off(false);
    const int64_t shape[4] = {k.size(0), k.size(1), tokens, d};
    at::Tensor keys = at::empty(shape, k.options().dtype(out_type)), values = at::empty(shape, k.options().dtype(out_type));
    const smha_status_t st = entries.packed_read(k.data_ptr(), v.data_ptr(), keys.data_ptr(), values.data_ptr(), lengths, offsets, (int)k.size(0), (int)k.size(1), tokens, (int)k.size(2), d,
                                                 (smha_dtype_t)type, ks.ptr, vs.ptr, nullptr, nullptr, c10::hip::getCurrentHIPStream(k.device().index()).stream());
    if (st != SMHA_OK) return PyLong_FromLong((long)st);
    return pair_of(std::move(keys), std::move(values));
    END_HANDLE_TH_ERRORS
}

// packed_attention(q, k, v, lengths, window, n_sink, scale) -> the output, a status, or None
PyObject *packed_attention(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 7 || !entries.packed_forward || at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) Py_RETURN_NONE;
    if (!plain(args[0]) || !plain(args[1]) || !plain(args[2]) || !PyFloat_CheckExact(args[6])) Py_RETURN_NONE;
    const at::Tensor &q = THPVariable_Unpack(args[0]), &k = THPVariable_Unpack(args[1]), &v = THPVariable_Unpack(args[2]);
    const int d = packed_width(k, v), type = code_of(q.scalar_type());
    if (!d || (type != SMHA_F16 && type != SMHA_BF16) || q.size(0) != k.size(0) || q.size(3) != d || k.size(1) < 1 || q.size(1) % k.size(1) || q.device() != k.device() || !small_sizes(q) ||
        wants_derivative(q))
        Py_RETURN_NONE;
    const int32_t *lengths;
    at::Tensor lengths_t;
    int window, n_sink;
    if (args[3] == Py_None || !per_sequence(args[3], q, lengths, lengths_t) || !int_from(args[4], window) || !int_from(args[5], n_sink)) Py_RETURN_NONE;
    const Strides3 qs(q), ks(k), vs(v);
    if (!qs.ok || !ks.ok || !vs.ok) Py_RETURN_NONE;
    const int B = (int)q.size(0), H = (int)q.size(1), T = (int)q.size(2), Hkv = (int)k.size(1), Sk = (int)k.size(2);
    const c10::DeviceGuard guard(q.device());
    size_t need = 0;
    smha_status_t st = entries.packed_workspace(B, H, Hkv, T, Sk, d, window, n_sink, &need);
    if (st != SMHA_OK) return PyLong_FromLong((long)st);
    const at::AutoGradMode off(false);
    at::Tensor o = packed_like(q);
    const c10::DataPtr ws = need ? scratch(need) : c10::DataPtr();
    st = entries.packed_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lengths, B, H, Hkv, T, Sk, d, (smha_dtype_t)type, qs.ptr, ks.ptr, vs.ptr, nullptr, window, n_sink,
                                (float)PyFloat_AS_DOUBLE(args[6]), ws.get(), need, c10::hip::getCurrentHIPStream(q.device().index()).stream());
    if (st != SMHA_OK) return PyLong_FromLong((long)st);
    return THPVariable_Wrap(std::move(o));
    END_HANDLE_TH_ERRORS
}

using Fast = PyObject *(*)(PyObject *, PyObject *const *, Py_ssize_t);
PyCFunction fast(Fast f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {{"link", fast(link), METH_FASTCALL, nullptr}, {"sink_attention", fast(sink_attention), METH_FASTCALL, nullptr},
                         {"cache_attention", fast(cache_attention), METH_FASTCALL, nullptr}, {"cache_evict", fast(cache_evict), METH_FASTCALL, nullptr},
                         {"packed_write", fast(packed_write), METH_FASTCALL, nullptr}, {"packed_read", fast(packed_read), METH_FASTCALL, nullptr},
                         {"packed_attention", fast(packed_attention), METH_FASTCALL, nullptr},
                         {"forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(forward)), METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_smha_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__smha_torch() {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "stamp", SMHA_STAMP) < 0) Py_CLEAR(m);  // what it was built from: build.py looks for it in the file
    return m;
}
