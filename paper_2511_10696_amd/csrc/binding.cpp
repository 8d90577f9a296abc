// binding.cpp -- the argument marshalling of the hot entry points in native
// code: from torch tensors to the C ABI of include/pi_attn.h.
//
// A call that launches one small kernel is bound by its host work: in Python
// the checks, the gate's broadcast view, the stream object and the ctypes
// conversion took 11 of a forward's 14.4 us, the launch itself 3.4; here the
// whole call takes 3.8 us.
//
// Each function takes the arguments of its namesake in __init__.py by
// position and serves the plain call: strided GPU tensors of one device,
// every argument of its documented type and valid.  For anything else --
// another type, another device, a tensor subclass or a wrapped tensor, an
// active torch function or dispatch mode, a given stream, an argument that
// the checks or the library refuse -- it returns None before anything is
// enqueued, and the Python code handles the call (and words the error).  A
// launch that the HIP runtime refuses (PI_ATTN_EHIP) raises PiAttnError here:
// of a call of several launches the first ones may be enqueued by then.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>

#include <algorithm>
#include <array>
#include <cmath>
#include <string>

#include "pi_attn.h"

namespace {

using at::Tensor;

// A plain call's arguments, read in order; `ok` turns false at the first one
// that is not plain, and stays so.
struct Args {
    PyObject *const *a;
    Py_ssize_t i = 0;
    bool ok;
    c10::Device device = c10::Device(c10::kCPU);

    Args(PyObject *const *args, Py_ssize_t n, Py_ssize_t want) : a(args) {
        ok = n == want && !c10::impl::TorchDispatchModeTLS::any_modes_set() && !at::impl::torch_function_mode_enabled();
    }
    // A tensor on the device of the first one; an undefined tensor for None
    // where `optional`.
    Tensor tensor(bool optional = false) {
        PyObject *o = next();
        if (!o || (optional && o == Py_None)) return Tensor();
        if (!THPVariable_CheckExact(o)) return fail();
        const Tensor &t = THPVariable_Unpack(o);
        if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || !t.has_storage()) return fail();
        const auto keys = t.key_set();
        if (keys.has(c10::DispatchKey::Python) || keys.has_any(c10::functorch_transforms_ks)) return fail();
        if (device.is_cpu()) device = t.device();
        if (t.device() != device) return fail();
        return t;
    }
    int32_t integer() {
        PyObject *o = next();
        if (!o || !PyLong_CheckExact(o)) return fail(), 0;
        int overflow = 0;
        const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
        if (overflow || v < INT32_MIN || v > INT32_MAX) return fail(), 0;
        return (int32_t)v;
    }
    bool boolean() {
        PyObject *o = next();
        if (!o || !PyBool_Check(o)) return fail(), false;
        return o == Py_True;
    }
    // a float or an int; `none` for None (NaN: None is not taken)
    float real(float none) {
        PyObject *o = next();
        if (!o) return 0.0f;
        if (o == Py_None && !std::isnan(none)) return none;
        if (PyFloat_CheckExact(o)) return (float)PyFloat_AS_DOUBLE(o);
        if (PyLong_CheckExact(o)) {
            int overflow = 0;
            const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
            if (!overflow) return (float)(double)v;
        }
        return fail(), 0.0f;
    }
    void none() {
        if (next() != Py_None) ok = false;
    }
    // the next argument; null once the call is not plain
    PyObject *next() { return ok ? a[i++] : nullptr; }
    Tensor fail() {
        ok = false;
        return Tensor();
    }
};

bool same_layout(const Tensor &x, const Tensor &y) { return x.sizes() == y.sizes() && x.strides() == y.strides(); }

int32_t dtype_of(const Tensor &t) {
    return t.scalar_type() == at::kFloat ? PI_ATTN_F32 : t.scalar_type() == at::kBFloat16 ? PI_ATTN_BF16 : -1;
}

// q, k, v [B, H, N, D]: one dtype, shape and strides, D contiguous, no empty
// extent.
struct Shape {
    int64_t B, H, N, D;
};

bool sequence_ok(const Tensor &q, const Tensor &k, const Tensor &v, Shape &s) {
    if (q.dim() != 4 || dtype_of(q) < 0 || k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type())
        return false;
    if (!same_layout(q, k) || !same_layout(q, v) || q.stride(3) != 1) return false;
    s = Shape{q.size(0), q.size(1), q.size(2), q.size(3)};
    return q.numel() > 0 && s.B <= INT32_MAX && s.H <= INT32_MAX && s.N <= INT32_MAX && s.D <= INT32_MAX;
}

bool is_f32(const Tensor &t, at::IntArrayRef shape) {
    return t.scalar_type() == at::kFloat && t.sizes() == shape && t.is_contiguous();
}

// A float32 output buffer: the given one, checked, or a new one.
bool f32_out(Tensor &t, at::IntArrayRef shape, const c10::Device &device) {
    if (!t.defined()) {
        t = at::empty(shape, at::TensorOptions().dtype(at::kFloat).device(device));
        return true;
    }
    return is_f32(t, shape);
}

// The output in q's shape and dtype: the given one, checked, or a new one.
bool like_out(Tensor &out, const Tensor &q) {
    if (!out.defined()) {
        out = at::empty(q.sizes(), at::TensorOptions().dtype(q.scalar_type()).device(q.device()));
        return true;
    }
    return out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type() && out.stride(3) == 1;
}

// Element strides of the gate logits: [H], or [B, H, N] (per_query).
bool gate_strides(const Tensor &g, const Shape &s, int64_t (&st)[3], bool &per_query) {
    if (g.scalar_type() != at::kFloat) return false;
    per_query = g.dim() == 3;
    if (g.dim() == 1 && g.size(0) == s.H) {
        st[0] = st[2] = 0;
        st[1] = g.stride(0);
        return true;
    }
    if (!per_query || g.size(0) != s.B || g.size(1) != s.H || g.size(2) != s.N) return false;
    for (int i = 0; i < 3; ++i) st[i] = g.stride(i);
    return true;
}

void *stream_of(const c10::Device &d) { return c10::hip::getCurrentHIPStream(d.index()).stream(); }

template <typename T>
T *ptr(const Tensor &t) {
    return t.defined() ? static_cast<T *>(t.data_ptr()) : nullptr;
}

PyObject *pack(std::initializer_list<Tensor> ts) {
    PyObject *r = PyTuple_New((Py_ssize_t)ts.size());
    Py_ssize_t i = 0;
    for (const Tensor &t : ts) PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(t));
    return r;
}

// The result of a call whose status is not PI_ATTN_OK.
PyObject *refused(PyObject *self, int status, const char *where) {
    if (status != PI_ATTN_EHIP) Py_RETURN_NONE;
    const auto package = pybind11::handle(self).attr("__package__");
    const auto error = pybind11::module_::import(pybind11::str(package).cast<std::string>().c_str()).attr("PiAttnError");
    PyErr_SetObject(error.ptr(), error(status, where).ptr());
    return nullptr;
}

// q, k, v, gate, k_window, pi, scale, logit_clamp, out, return_lse, lse, stream, causal
PyObject *forward(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Args a(args, n, 13);
    const Tensor q = a.tensor(), k = a.tensor(), v = a.tensor(), gate = a.tensor();
    const int32_t kw = a.integer(), pi = a.integer();
    Shape s{};
    if (!a.ok || !sequence_ok(q, k, v, s)) Py_RETURN_NONE;
    const float scale = a.real(pi_attn_default_scale((int32_t)s.D)), clamp = a.real(NAN);
    Tensor out = a.tensor(true);
    const bool want_lse = a.boolean();
    Tensor lse = a.tensor(true);
    a.none();
    const bool causal = a.boolean();
    int64_t gs[3];
    bool per_query;
    if (!a.ok || !gate_strides(gate, s, gs, per_query)) Py_RETURN_NONE;
    const bool with_lse = want_lse || lse.defined();
    int status = PI_ATTN_EINVAL;
    {
        pybind11::gil_scoped_release no_gil;
        if (like_out(out, q) && (!with_lse || f32_out(lse, {s.B, s.H, s.N}, a.device)))
            status = pi_attn_forward(dtype_of(q), s.B, s.H, s.N, s.D, kw, pi, causal, q.data_ptr(), k.data_ptr(),
                                     v.data_ptr(), q.stride(0), q.stride(1), q.stride(2), ptr<float>(gate), gs[0],
                                     gs[1], gs[2], scale, clamp, out.data_ptr(), out.stride(0), out.stride(1),
                                     out.stride(2), ptr<float>(lse), stream_of(a.device));
    }
    if (status != PI_ATTN_OK) return refused(self, status, "pi_attn_forward");
    return with_lse ? pack({out, lse}) : THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// q, k, v, u, w2, b2, k_window, pi, scale, logit_clamp, out, return_lse, lse, gate_out, stream, causal
PyObject *forward_gated(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Args a(args, n, 16);
    const Tensor q = a.tensor(), k = a.tensor(), v = a.tensor(), u = a.tensor(), w2 = a.tensor();
    const Tensor b2 = a.tensor(true);
    const int32_t kw = a.integer(), pi = a.integer();
    Shape s{};
    if (!a.ok || !sequence_ok(q, k, v, s)) Py_RETURN_NONE;
    const float scale = a.real(pi_attn_default_scale((int32_t)s.D)), clamp = a.real(NAN);
    Tensor out = a.tensor(true);
    const bool want_lse = a.boolean();
    Tensor lse = a.tensor(true), gate = a.tensor(true);
    a.none();
    const bool causal = a.boolean();
    if (!a.ok || u.scalar_type() != q.scalar_type() || w2.scalar_type() != q.scalar_type()) Py_RETURN_NONE;
    if (u.dim() != 3 || u.size(0) != s.B || u.size(1) != s.N || u.stride(2) != 1) Py_RETURN_NONE;
    const int64_t dh = u.size(2);
    if (dh > INT32_MAX || w2.sizes() != at::IntArrayRef({s.H, dh}) || !w2.is_contiguous()) Py_RETURN_NONE;
    if (b2.defined() && !is_f32(b2, {s.H})) Py_RETURN_NONE;
    const bool with_lse = want_lse || lse.defined();
    int status = PI_ATTN_EINVAL;
    {
        pybind11::gil_scoped_release no_gil;
        if (like_out(out, q) && f32_out(gate, {s.B, s.H, s.N}, a.device) &&
            (!with_lse || f32_out(lse, {s.B, s.H, s.N}, a.device)))
            status = pi_attn_forward_gated(dtype_of(q), s.B, s.H, s.N, s.D, kw, pi, causal, q.data_ptr(), k.data_ptr(),
                                           v.data_ptr(), q.stride(0), q.stride(1), q.stride(2), u.data_ptr(),
                                           u.stride(0), u.stride(1), dh, w2.data_ptr(), ptr<float>(b2), scale, clamp,
                                           out.data_ptr(), out.stride(0), out.stride(1), out.stride(2), ptr<float>(lse),
                                           ptr<float>(gate), stream_of(a.device));
    }
    if (status != PI_ATTN_OK) return refused(self, status, "pi_attn_forward_gated");
    return with_lse ? pack({out, gate, lse}) : pack({out, gate});
    END_HANDLE_TH_ERRORS
}

// q, k, v, gate, k_window, pi, out, lse, dout, scale, logit_clamp, gate_grad_per_query, stream, causal, dq, dk, dv,
// dgate, rowterm
PyObject *backward(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Args a(args, n, 19);
    const Tensor q = a.tensor(), k = a.tensor(), v = a.tensor(), gate = a.tensor();
    const int32_t kw = a.integer(), pi = a.integer();
    const Tensor out = a.tensor(), lse = a.tensor(), dout = a.tensor();
    Shape s{};
    if (!a.ok || !sequence_ok(q, k, v, s)) Py_RETURN_NONE;
    const float scale = a.real(pi_attn_default_scale((int32_t)s.D)), clamp = a.real(NAN);
    const bool keep_per_query = a.boolean();
    a.none();
    const bool causal = a.boolean();
    Tensor dq = a.tensor(true), dk = a.tensor(true), dv = a.tensor(true), dg = a.tensor(true), rt = a.tensor(true);
    int64_t gs[3];
    bool per_query;
    if (!a.ok || !gate_strides(gate, s, gs, per_query)) Py_RETURN_NONE;
    if (out.scalar_type() != q.scalar_type() || dout.scalar_type() != q.scalar_type() || !same_layout(out, dout) ||
        out.sizes() != q.sizes() || dout.stride(3) != 1 || !is_f32(lse, {s.B, s.H, s.N}))
        Py_RETURN_NONE;
    Tensor per_head;
    int status = PI_ATTN_EINVAL;
    const char *where = "pi_attn_backward";
    {
        pybind11::gil_scoped_release no_gil;
        const std::array<int64_t, 4> full{s.B, s.H, s.N, s.D};
        const std::array<int64_t, 3> rows{s.B, s.H, s.N};
        void *stream = stream_of(a.device);
        if (f32_out(dq, full, a.device) && f32_out(dk, full, a.device) && f32_out(dv, full, a.device) &&
            f32_out(dg, rows, a.device) && f32_out(rt, rows, a.device))
            status = pi_attn_backward(dtype_of(q), s.B, s.H, s.N, s.D, kw, pi, causal, q.data_ptr(), k.data_ptr(),
                                      v.data_ptr(), q.stride(0), q.stride(1), q.stride(2), ptr<float>(gate), gs[0],
                                      gs[1], gs[2], scale, clamp, ptr<float>(lse), out.data_ptr(), dout.data_ptr(),
                                      dout.stride(0), dout.stride(1), dout.stride(2), ptr<float>(dq), ptr<float>(dk),
                                      ptr<float>(dv), ptr<float>(dg), ptr<float>(rt), stream);
        if (status == PI_ATTN_OK && !per_query && !keep_per_query) {
            where = "pi_attn_gate_grad_per_head";   // of valid arguments: refused by the runtime or not at all
            f32_out(per_head, {s.H}, a.device);
            status = pi_attn_gate_grad_per_head(s.B, s.H, s.N, ptr<float>(dg), ptr<float>(per_head), stream);
        }
    }
    if (status != PI_ATTN_OK) return refused(self, status, where);
    return pack({dq, dk, dv, per_head.defined() ? per_head : dg});
    END_HANDLE_TH_ERRORS
}

// len_in, q_new, k_new, v_new, k_cache, v_cache, gate, k, pi, scale, logit_clamp, len_out, out, lse, stream
PyObject *decode_step(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Args a(args, n, 15);
    const Tensor len_in = a.tensor(), q = a.tensor(), k = a.tensor(), v = a.tensor(), kc = a.tensor(),
                 vc = a.tensor(), gate = a.tensor();
    const int32_t kw = a.integer(), pi = a.integer();
    if (!a.ok || kc.dim() != 4 || dtype_of(kc) < 0 || kc.numel() == 0) Py_RETURN_NONE;
    const int64_t S = kc.size(0), H = kc.size(1), cap = kc.size(2), D = kc.size(3);
    if (S > INT32_MAX || H > INT32_MAX || cap > INT32_MAX || D > INT32_MAX) Py_RETURN_NONE;
    const float scale = a.real(pi_attn_default_scale((int32_t)D)), clamp = a.real(NAN);
    const Tensor len_out = a.tensor(true);
    Tensor out = a.tensor(true);
    const Tensor lse = a.tensor(true);
    a.none();
    if (!a.ok) Py_RETURN_NONE;
    const std::array<int64_t, 3> rows{S, H, D};
    const auto cached = [&](const Tensor &t, at::IntArrayRef shape) {
        return t.scalar_type() == kc.scalar_type() && t.sizes() == shape && t.is_contiguous();
    };
    const auto lengths = [&](const Tensor &t) {
        return t.scalar_type() == at::kInt && t.dim() == 1 && t.size(0) == S && t.is_contiguous();
    };
    if (!cached(q, rows) || !cached(k, rows) || !cached(v, rows) || !cached(vc, kc.sizes()) || !kc.is_contiguous())
        Py_RETURN_NONE;
    if (!lengths(len_in) || (len_out.defined() && !lengths(len_out)) || gate.scalar_type() != at::kFloat) Py_RETURN_NONE;
    int64_t gss, gsh;
    if (gate.dim() == 1 && gate.size(0) == H) {
        gss = 0;
        gsh = gate.stride(0);
    } else if (gate.dim() == 2 && gate.size(0) == S && gate.size(1) == H) {
        gss = gate.stride(0);
        gsh = gate.stride(1);
    } else {
        Py_RETURN_NONE;
    }
    if ((out.defined() && !cached(out, rows)) || (lse.defined() && !is_f32(lse, {S, H}))) Py_RETURN_NONE;
    int status;
    {
        pybind11::gil_scoped_release no_gil;
        if (!out.defined()) out = at::empty(rows, at::TensorOptions().dtype(kc.scalar_type()).device(a.device));
        status = pi_attn_decode_step(dtype_of(kc), S, H, D, cap, kw, pi, ptr<int32_t>(len_in), ptr<int32_t>(len_out),
                                     q.data_ptr(), k.data_ptr(), v.data_ptr(), kc.data_ptr(), vc.data_ptr(),
                                     ptr<float>(gate), gss, gsh, scale, clamp, out.data_ptr(), ptr<float>(lse),
                                     stream_of(a.device));
    }
    if (status != PI_ATTN_OK) return refused(self, status, "pi_attn_decode_step");
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// A quantised cache: codes [S, H, cap, D] and bytes [S, H, cap], no empty extent.
struct Cache {
    Tensor k, v, ke, ve;
    int64_t S, H, cap, D;
};

bool bytes_ok(const Tensor &t, at::IntArrayRef shape) {
    return t.scalar_type() == at::kByte && t.sizes() == shape && t.is_contiguous();
}

// The tables' type and layout; `rows`: the type of codes or of plain rows.
bool cache_ok(Cache &c, at::ScalarType rows) {
    if (c.k.dim() != 4 || c.k.scalar_type() != rows || c.v.scalar_type() != rows || c.k.numel() == 0) return false;
    if (c.v.sizes() != c.k.sizes() || !c.k.is_contiguous() || !c.v.is_contiguous()) return false;
    c.S = c.k.size(0), c.H = c.k.size(1), c.cap = c.k.size(2), c.D = c.k.size(3);
    if (c.S > INT32_MAX || c.H > INT32_MAX || c.cap > INT32_MAX || c.D > INT32_MAX) return false;
    const bool quantised = rows == at::kFloat8_e4m3fn;
    if (c.ke.defined() != quantised || c.ve.defined() != quantised) return false;
    const std::array<int64_t, 3> table{c.S, c.H, c.cap};
    return !quantised || (bytes_ok(c.ke, table) && bytes_ok(c.ve, table));
}

bool per_sequence(const Tensor &t, int64_t S) {
    return !t.defined() || (t.scalar_type() == at::kInt && t.dim() == 1 && t.size(0) == S && t.is_contiguous());
}

// k, v [S, H, n, D] of a cache's rows.
bool rows_ok(const Tensor &k, const Tensor &v, const Cache &c) {
    return k.dim() == 4 && dtype_of(k) >= 0 && v.scalar_type() == k.scalar_type() && same_layout(k, v) &&
           k.size(0) == c.S && k.size(1) == c.H && k.size(3) == c.D && k.stride(3) == 1 && k.size(2) <= INT32_MAX;
}

// k, v, k_cache, v_cache, k_exp, v_exp, start, count, stream
PyObject *cache_store(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Args a(args, n, 9);
    Cache c;
    const Tensor k = a.tensor(), v = a.tensor();
    c.k = a.tensor(), c.v = a.tensor(), c.ke = a.tensor(), c.ve = a.tensor();
    const Tensor start = a.tensor(true), count = a.tensor(true);
    a.none();
    if (!a.ok || !cache_ok(c, at::kFloat8_e4m3fn) || !rows_ok(k, v, c) || !per_sequence(start, c.S) ||
        !per_sequence(count, c.S))
        Py_RETURN_NONE;
    int status;
    {
        pybind11::gil_scoped_release no_gil;
        const c10::DeviceGuard on(a.device);
        status = pi_attn_cache_store(dtype_of(k), c.S, c.H, c.D, k.size(2), c.cap, k.data_ptr(), v.data_ptr(),
                                     k.stride(0), k.stride(1), k.stride(2), ptr<int32_t>(start), ptr<int32_t>(count),
                                     c.k.data_ptr(), c.v.data_ptr(), ptr<uint8_t>(c.ke), ptr<uint8_t>(c.ve),
                                     stream_of(a.device));
    }
    if (status != PI_ATTN_OK) return refused(self, status, "pi_attn_cache_store");
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

// k_cache, v_cache, k_exp, v_exp, n, start, count, dtype, k, v, stream
PyObject *cache_load(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Args a(args, n, 11);
    Cache c;
    c.k = a.tensor(), c.v = a.tensor(), c.ke = a.tensor(), c.ve = a.tensor();
    const int32_t rows = a.integer();
    const Tensor start = a.tensor(true), count = a.tensor(true);
    PyObject *dtype = a.next();
    Tensor k = a.tensor(true), v = a.tensor(true);
    a.none();
    if (!a.ok || rows < 1 || !cache_ok(c, at::kFloat8_e4m3fn) || !per_sequence(start, c.S) ||
        !per_sequence(count, c.S) || k.defined() != v.defined())
        Py_RETURN_NONE;
    if (dtype != Py_None && !THPDtype_Check(dtype)) Py_RETURN_NONE;
    const at::ScalarType want = dtype != Py_None ? reinterpret_cast<THPDtype *>(dtype)->scalar_type
                                : k.defined()    ? k.scalar_type()
                                                 : at::kBFloat16;
    if (want != at::kFloat && want != at::kBFloat16) Py_RETURN_NONE;
    if (k.defined() && (k.scalar_type() != want || !rows_ok(k, v, c) || k.size(2) != rows)) Py_RETURN_NONE;
    int status;
    {
        pybind11::gil_scoped_release no_gil;
        const c10::DeviceGuard on(a.device);
        if (!k.defined()) {
            const std::array<int64_t, 4> shape{c.S, c.H, rows, c.D};
            const auto options = at::TensorOptions().dtype(want).device(a.device);
            k = at::empty(shape, options);
            v = at::empty(shape, options);
        }
        status = pi_attn_cache_load(dtype_of(k), c.S, c.H, c.D, rows, c.cap, c.k.data_ptr(), c.v.data_ptr(),
                                    ptr<uint8_t>(c.ke), ptr<uint8_t>(c.ve), ptr<int32_t>(start), ptr<int32_t>(count),
                                    k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2),
                                    stream_of(a.device));
    }
    if (status != PI_ATTN_OK) return refused(self, status, "pi_attn_cache_load");
    return pack({k, v});
    END_HANDLE_TH_ERRORS
}

// The arguments of a decode step but for its caches.
struct Step {
    Tensor len_in, q, k, v, gate, len_out, out, lse, work;
    int64_t gss, gsh;
};

// What both cached steps check of them, for caches of S, H, cap, D; allocates
// the output and the workspace where none is given.
bool step_ok(Step &s, const Cache &c, int64_t plen, int32_t kw, const c10::Device &device) {
    const std::array<int64_t, 3> rows{c.S, c.H, c.D};
    const int32_t dt = dtype_of(s.q);
    const auto fits = [&](const Tensor &t) {
        return t.scalar_type() == s.q.scalar_type() && t.sizes() == at::IntArrayRef(rows) && t.is_contiguous();
    };
    if (dt < 0 || !fits(s.q) || !fits(s.k) || !fits(s.v)) return false;
    if (!per_sequence(s.len_in, c.S) || !per_sequence(s.len_out, c.S) || s.gate.scalar_type() != at::kFloat) return false;
    if (s.gate.dim() == 1 && s.gate.size(0) == c.H) {
        s.gss = 0;
        s.gsh = s.gate.stride(0);
    } else if (s.gate.dim() == 2 && s.gate.size(0) == c.S && s.gate.size(1) == c.H) {
        s.gss = s.gate.stride(0);
        s.gsh = s.gate.stride(1);
    } else {
        return false;
    }
    if ((s.out.defined() && !fits(s.out)) || (s.lse.defined() && !is_f32(s.lse, {c.S, c.H}))) return false;
    const int64_t need = pi_attn_decode_workspace(dt, c.S, c.H, c.D, plen, c.cap, kw);
    if (need < 0) return false;
    if (s.work.defined()) {
        if (s.work.scalar_type() != at::kFloat || !s.work.is_contiguous() || s.work.numel() < need) return false;
    } else if (need > 0) {
        s.work = at::empty({need}, at::TensorOptions().dtype(at::kFloat).device(device));
    }
    if (!s.out.defined()) s.out = at::empty(rows, at::TensorOptions().dtype(s.q.scalar_type()).device(device));
    return true;
}

// len_in, q_new, k_new, v_new, k_cache, v_cache, k_exp, v_exp, gate, k, pi, scale, logit_clamp, len_out, out, lse, work,
// stream
PyObject *decode_step_e4m3(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Args a(args, n, 18);
    Step s;
    Cache c;
    s.len_in = a.tensor(), s.q = a.tensor(), s.k = a.tensor(), s.v = a.tensor();
    c.k = a.tensor(), c.v = a.tensor(), c.ke = a.tensor(), c.ve = a.tensor();
    s.gate = a.tensor();
    const int32_t kw = a.integer(), pi = a.integer();
    if (!a.ok || !cache_ok(c, at::kFloat8_e4m3fn)) Py_RETURN_NONE;
    const float scale = a.real(pi_attn_default_scale((int32_t)c.D)), clamp = a.real(NAN);
    s.len_out = a.tensor(true), s.out = a.tensor(true), s.lse = a.tensor(true), s.work = a.tensor(true);
    a.none();
    if (!a.ok) Py_RETURN_NONE;
    int status = PI_ATTN_EINVAL;
    {
        pybind11::gil_scoped_release no_gil;
        const c10::DeviceGuard on(a.device);
        if (step_ok(s, c, 0, kw, a.device))
            status = pi_attn_decode_step_e4m3(dtype_of(s.q), c.S, c.H, c.D, c.cap, kw, pi, ptr<int32_t>(s.len_in),
                                              ptr<int32_t>(s.len_out), s.q.data_ptr(), s.k.data_ptr(), s.v.data_ptr(),
                                              c.k.data_ptr(), c.v.data_ptr(), ptr<uint8_t>(c.ke), ptr<uint8_t>(c.ve),
                                              ptr<float>(s.gate), s.gss, s.gsh, scale, clamp, s.out.data_ptr(),
                                              ptr<float>(s.lse), ptr<float>(s.work), stream_of(a.device));
    }
    if (status != PI_ATTN_OK) return refused(self, status, "pi_attn_decode_step_e4m3");
    return THPVariable_Wrap(s.out);
    END_HANDLE_TH_ERRORS
}

// len_in, q_new, k_new, v_new, k_prefix, v_prefix, k_cache, v_cache, gate, k, pi, k_prefix_exp, v_prefix_exp, k_exp,
// v_exp, scale, logit_clamp, len_out, out, lse, work, stream
PyObject *decode_step_prefix(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Args a(args, n, 22);
    Step s;
    Cache c;
    s.len_in = a.tensor(), s.q = a.tensor(), s.k = a.tensor(), s.v = a.tensor();
    const Tensor kp = a.tensor(), vp = a.tensor();
    c.k = a.tensor(), c.v = a.tensor();
    s.gate = a.tensor();
    const int32_t kw = a.integer(), pi = a.integer();
    const Tensor kpe = a.tensor(true), vpe = a.tensor(true);
    c.ke = a.tensor(true), c.ve = a.tensor(true);
    if (!a.ok) Py_RETURN_NONE;
    const at::ScalarType rows = c.ke.defined() ? at::kFloat8_e4m3fn : s.q.scalar_type();
    if (!cache_ok(c, rows)) Py_RETURN_NONE;
    const float scale = a.real(pi_attn_default_scale((int32_t)c.D)), clamp = a.real(NAN);
    s.len_out = a.tensor(true), s.out = a.tensor(true), s.lse = a.tensor(true), s.work = a.tensor(true);
    a.none();
    if (!a.ok || kp.dim() != 3 || kp.scalar_type() != rows || vp.scalar_type() != rows || !same_layout(kp, vp))
        Py_RETURN_NONE;
    const int64_t plen = kp.size(1), pcap = c.H > 1 ? kp.stride(0) / c.D : plen;
    if (kp.size(0) != c.H || kp.size(2) != c.D || plen < 1 || kp.stride(2) != 1 || (plen > 1 && kp.stride(1) != c.D) ||
        (c.H > 1 && kp.stride(0) % c.D != 0) || pcap < plen || pcap > INT32_MAX)
        Py_RETURN_NONE;
    if (kpe.defined() != c.ke.defined() || vpe.defined() != c.ke.defined()) Py_RETURN_NONE;
    for (const Tensor &t : {kpe, vpe}) {
        if (t.defined() && (t.scalar_type() != at::kByte || t.dim() != 2 || t.size(0) != c.H || t.size(1) != plen ||
                            (plen > 1 && t.stride(1) != 1) || (c.H > 1 && t.stride(0) != pcap)))
            Py_RETURN_NONE;
    }
    int status = PI_ATTN_EINVAL;
    {
        pybind11::gil_scoped_release no_gil;
        const c10::DeviceGuard on(a.device);
        if (step_ok(s, c, plen, kw, a.device))
            status = pi_attn_decode_step_prefix(
                dtype_of(s.q), c.S, c.H, c.D, plen, pcap, c.cap, kw, pi, ptr<int32_t>(s.len_in),
                ptr<int32_t>(s.len_out), s.q.data_ptr(), s.k.data_ptr(), s.v.data_ptr(), kp.data_ptr(), vp.data_ptr(),
                ptr<uint8_t>(kpe), ptr<uint8_t>(vpe), c.k.data_ptr(), c.v.data_ptr(), ptr<uint8_t>(c.ke),
                ptr<uint8_t>(c.ve), ptr<float>(s.gate), s.gss, s.gsh, scale, clamp, s.out.data_ptr(),
                ptr<float>(s.lse), ptr<float>(s.work), stream_of(a.device));
    }
    if (status != PI_ATTN_OK) return refused(self, status, "pi_attn_decode_step_prefix");
    return THPVariable_Wrap(s.out);
    END_HANDLE_TH_ERRORS
}

// Element strides of the rows of t [.., .., .., D]: 0 where there is one alone.
std::array<int64_t, 3> row_strides(const Tensor &t) {
    std::array<int64_t, 3> st{0, 0, 0};
    for (int i = 0; t.defined() && i < 3; ++i) st[i] = t.size(i) > 1 ? t.stride(i) : 0;
    return st;
}

// The rotation of rows: frequencies, the pairs of each axis, positions.
struct Turn {
    Tensor freq, pos;
    std::array<int32_t, 3> pairs{0, 0, 0};
    std::array<int64_t, 3> ps{0, 0, 0};   // of pos: axis, and the positions' own dimensions
};

// `sections` None or a tuple of whole numbers; positions of `shape`, behind an axis,
// or for one axis alone.
bool turn_ok(Turn &t, PyObject *sections, at::IntArrayRef shape, int64_t D) {
    if (!t.freq.defined()) return !t.pos.defined() && sections == Py_None;
    if (t.freq.scalar_type() != at::kFloat || t.freq.dim() != 1 || !t.freq.is_contiguous()) return false;
    const int64_t total = t.freq.size(0);
    int64_t axes = 1;
    if (total > D / 2) return false;
    if (sections == Py_None) {
        t.pairs[0] = (int32_t)total;
    } else {
        if (!PyTuple_CheckExact(sections)) return false;
        axes = PyTuple_GET_SIZE(sections);
        if (axes < 1 || axes > 3) return false;
        int64_t sum = 0;
        for (int64_t i = 0; i < axes; ++i) {
            PyObject *const o = PyTuple_GET_ITEM(sections, i);
            if (!PyLong_CheckExact(o)) return false;
            int overflow = 0;
            const long long n = PyLong_AsLongLongAndOverflow(o, &overflow);
            if (overflow || n < 0 || n > total) return false;
            t.pairs[i] = (int32_t)n;
            sum += n;
        }
        if (sum != total) return false;
    }
    if (!t.pos.defined()) return true;
    const int64_t dims = (int64_t)shape.size(), at = t.pos.dim();
    if (t.pos.scalar_type() != at::kInt || at < 1 || at > dims + 1) return false;
    if (at == dims + 1 ? t.pos.size(0) != axes : axes != 1) return false;
    const int64_t own = std::min(at, dims);   // trailing dimensions of `shape` that pos has
    for (int64_t i = 0; i < own; ++i)
        if (t.pos.size(at - own + i) != shape[dims - own + i]) return false;
    for (int64_t i = 0; i < at; ++i) t.ps[dims + 1 - at + i] = t.pos.stride(i);
    return true;
}

// q, k, pos, freq, sections, dtype, q_out, k_out, stream, back
PyObject *rotate(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Args a(args, n, 10);
    Turn t;
    const Tensor q = a.tensor(), k = a.tensor(true);
    t.pos = a.tensor(true), t.freq = a.tensor(true);
    PyObject *const sections = a.next(), *const dtype = a.next();
    Tensor qo = a.tensor(true), ko = a.tensor(true);
    a.none();
    const bool back = a.boolean();
    if (!a.ok || q.dim() != 4 || dtype_of(q) < 0 || q.numel() == 0 || q.stride(3) != 1) Py_RETURN_NONE;
    if (dtype != Py_None && !THPDtype_Check(dtype)) Py_RETURN_NONE;
    const int64_t B = q.size(0), H = q.size(1), N = q.size(2), D = q.size(3);
    const int64_t Hk = k.defined() && k.dim() == 4 ? k.size(1) : 0;
    if (B > INT32_MAX || H > INT32_MAX || Hk > INT32_MAX || N > INT32_MAX || D > INT32_MAX) Py_RETURN_NONE;
    if (k.defined() ? k.dim() != 4 || k.size(0) != B || k.size(2) != N || k.size(3) != D || k.stride(3) != 1 ||
                          k.scalar_type() != q.scalar_type()
                    : ko.defined())
        Py_RETURN_NONE;
    const at::ScalarType want = dtype != Py_None ? reinterpret_cast<THPDtype *>(dtype)->scalar_type
                                : qo.defined()   ? qo.scalar_type()
                                : ko.defined()   ? ko.scalar_type()
                                                 : q.scalar_type();
    if (want != at::kFloat && want != at::kBFloat16) Py_RETURN_NONE;
    const auto fits = [&](const Tensor &o, const Tensor &x) {
        return !o.defined() || (o.sizes() == x.sizes() && o.scalar_type() == want && o.stride(3) == 1);
    };
    if (!fits(qo, q) || !fits(ko, k) || !turn_ok(t, sections, {B, N}, D)) Py_RETURN_NONE;
    int status;
    {
        pybind11::gil_scoped_release no_gil;
        const c10::DeviceGuard on(a.device);
        const auto options = at::TensorOptions().dtype(want).device(a.device);
        if (!qo.defined()) qo = at::empty(q.sizes(), options);
        if (k.defined() && !ko.defined()) ko = at::empty(k.sizes(), options);
        const auto qs = row_strides(q), ks = row_strides(k), qos = row_strides(qo), kos = row_strides(ko);
        status = pi_attn_rotate(dtype_of(q), dtype_of(qo), B, H, Hk, N, D, back, q.data_ptr(), qs[0], qs[1], qs[2],
                                ptr<void>(k), ks[0], ks[1], ks[2], ptr<int32_t>(t.pos), t.ps[0], t.ps[1], t.ps[2],
                                ptr<float>(t.freq), t.pairs[0], t.pairs[1], t.pairs[2], qo.data_ptr(), qos[0], qos[1],
                                qos[2], ptr<void>(ko), kos[0], kos[1], kos[2], stream_of(a.device));
    }
    if (status != PI_ATTN_OK) return refused(self, status, back ? "pi_attn_rotate_backward" : "pi_attn_rotate");
    if (ko.defined()) return pack({qo, ko});
    return PyTuple_Pack(2, pybind11::reinterpret_steal<pybind11::object>(THPVariable_Wrap(qo)).ptr(), Py_None);
    END_HANDLE_TH_ERRORS
}

// A paged cache: pages [n, Hk, page, D], bytes [n, Hk, page], table [S, max], no empty extent.
struct Paged {
    Tensor k, v, ke, ve, table;
    int64_t n, Hk, page, D, S, max;
};

bool paged_ok(Paged &g, at::ScalarType rows) {
    if (g.k.dim() != 4 || g.k.numel() == 0 || !g.k.is_contiguous() || !g.v.is_contiguous()) return false;
    const bool quantised = g.k.scalar_type() == at::kFloat8_e4m3fn;
    if (g.v.scalar_type() != g.k.scalar_type() || g.v.sizes() != g.k.sizes()) return false;
    if (!quantised && g.k.scalar_type() != rows) return false;
    if (g.table.scalar_type() != at::kInt || g.table.dim() != 2 || !g.table.is_contiguous() || g.table.numel() == 0)
        return false;
    g.n = g.k.size(0), g.Hk = g.k.size(1), g.page = g.k.size(2), g.D = g.k.size(3);
    g.S = g.table.size(0), g.max = g.table.size(1);
    for (const int64_t x : {g.n, g.Hk, g.page, g.D, g.S, g.max})
        if (x > INT32_MAX) return false;
    if (g.ke.defined() != quantised || g.ve.defined() != quantised) return false;
    const std::array<int64_t, 3> bytes{g.n, g.Hk, g.page};
    return !quantised || (bytes_ok(g.ke, bytes) && bytes_ok(g.ve, bytes));
}

// k, v [S, Hk, n, D] of a paged cache's rows.
bool paged_rows_ok(const Tensor &k, const Tensor &v, const Paged &g) {
    return k.dim() == 4 && dtype_of(k) >= 0 && v.scalar_type() == k.scalar_type() && same_layout(k, v) &&
           k.size(0) == g.S && k.size(1) == g.Hk && k.size(3) == g.D && k.stride(3) == 1 && k.size(2) <= INT32_MAX;
}

// k, v, k_pages, v_pages, table, start, count, k_exp, v_exp, freq, pos, sections, stream
PyObject *paged_store(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Args a(args, n, 13);
    Paged g;
    Turn t;
    const Tensor k = a.tensor(), v = a.tensor();
    g.k = a.tensor(), g.v = a.tensor(), g.table = a.tensor();
    const Tensor start = a.tensor(true), count = a.tensor(true);
    g.ke = a.tensor(true), g.ve = a.tensor(true);
    t.freq = a.tensor(true), t.pos = a.tensor(true);
    PyObject *const sections = a.next();
    a.none();
    if (!a.ok || dtype_of(k) < 0 || !paged_ok(g, k.scalar_type()) || !paged_rows_ok(k, v, g) ||
        !per_sequence(start, g.S) || !per_sequence(count, g.S) || !turn_ok(t, sections, {g.S, k.size(2)}, g.D))
        Py_RETURN_NONE;
    int status;
    {
        pybind11::gil_scoped_release no_gil;
        const c10::DeviceGuard on(a.device);
        const auto ks = row_strides(k);
        status = pi_attn_paged_store(dtype_of(k), g.S, g.Hk, g.D, k.size(2), g.n, g.page, g.max, k.data_ptr(),
                                     v.data_ptr(), ks[0], ks[1], ks[2], ptr<int32_t>(start), ptr<int32_t>(count),
                                     ptr<int32_t>(g.table), g.k.data_ptr(), g.v.data_ptr(), ptr<uint8_t>(g.ke),
                                     ptr<uint8_t>(g.ve), ptr<float>(t.freq), t.pairs[0], t.pairs[1], t.pairs[2],
                                     ptr<int32_t>(t.pos), t.ps[0], t.ps[1], t.ps[2], stream_of(a.device));
    }
    if (status != PI_ATTN_OK) return refused(self, status, "pi_attn_paged_store");
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

// k_pages, v_pages, table, n, start, count, k_exp, v_exp, dtype, k, v, stream
PyObject *paged_load(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Args a(args, n, 12);
    Paged g;
    g.k = a.tensor(), g.v = a.tensor(), g.table = a.tensor();
    const int32_t rows = a.integer();
    const Tensor start = a.tensor(true), count = a.tensor(true);
    g.ke = a.tensor(true), g.ve = a.tensor(true);
    PyObject *const dtype = a.next();
    Tensor k = a.tensor(true), v = a.tensor(true);
    a.none();
    if (!a.ok || rows < 1 || k.defined() != v.defined() || (dtype != Py_None && !THPDtype_Check(dtype))) Py_RETURN_NONE;
    const at::ScalarType want = dtype != Py_None ? reinterpret_cast<THPDtype *>(dtype)->scalar_type
                                : k.defined()    ? k.scalar_type()
                                : g.k.scalar_type() == at::kFloat8_e4m3fn ? at::kBFloat16
                                                                          : g.k.scalar_type();
    if ((want != at::kFloat && want != at::kBFloat16) || !paged_ok(g, want) || !per_sequence(start, g.S) ||
        !per_sequence(count, g.S))
        Py_RETURN_NONE;
    if (k.defined() && (k.scalar_type() != want || !paged_rows_ok(k, v, g) || k.size(2) != rows)) Py_RETURN_NONE;
    int status;
    {
        pybind11::gil_scoped_release no_gil;
        const c10::DeviceGuard on(a.device);
        if (!k.defined()) {
            const std::array<int64_t, 4> shape{g.S, g.Hk, rows, g.D};
            const auto options = at::TensorOptions().dtype(want).device(a.device);
            k = at::empty(shape, options);
            v = at::empty(shape, options);
        }
        const auto ks = row_strides(k);
        status = pi_attn_paged_load(dtype_of(k), g.S, g.Hk, g.D, rows, g.n, g.page, g.max, g.k.data_ptr(),
                                    g.v.data_ptr(), ptr<uint8_t>(g.ke), ptr<uint8_t>(g.ve), ptr<int32_t>(start),
                                    ptr<int32_t>(count), ptr<int32_t>(g.table), k.data_ptr(), v.data_ptr(), ks[0], ks[1],
                                    ks[2], stream_of(a.device));
    }
    if (status != PI_ATTN_OK) return refused(self, status, "pi_attn_paged_load");
    return pack({k, v});
    END_HANDLE_TH_ERRORS
}

// len_in, q_new, k_new, v_new, k_pages, v_pages, table, gate, k, pi, k_exp, v_exp, freq, pos, sections, scale,
// logit_clamp, len_out, out, lse, work, stream
PyObject *decode_step_paged(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Args a(args, n, 22);
    Paged g;
    Turn t;
    const Tensor len_in = a.tensor(), q = a.tensor(), k = a.tensor(), v = a.tensor();
    g.k = a.tensor(), g.v = a.tensor(), g.table = a.tensor();
    const Tensor gate = a.tensor();
    const int32_t kw = a.integer(), pi = a.integer();
    g.ke = a.tensor(true), g.ve = a.tensor(true);
    t.freq = a.tensor(true), t.pos = a.tensor(true);
    PyObject *const sections = a.next();
    if (!a.ok || dtype_of(q) < 0 || !paged_ok(g, q.scalar_type())) Py_RETURN_NONE;
    const float scale = a.real(pi_attn_default_scale((int32_t)g.D)), clamp = a.real(NAN);
    const Tensor len_out = a.tensor(true);
    Tensor out = a.tensor(true);
    const Tensor lse = a.tensor(true);
    Tensor work = a.tensor(true);
    a.none();
    if (!a.ok || q.dim() != 3 || q.size(0) != g.S || q.size(2) != g.D || !q.is_contiguous() || q.numel() == 0 ||
        q.size(1) > INT32_MAX || q.size(1) % g.Hk != 0)
        Py_RETURN_NONE;
    const int64_t H = q.size(1);
    const std::array<int64_t, 3> key_rows{g.S, g.Hk, g.D};
    for (const Tensor &x : {k, v})
        if (x.scalar_type() != q.scalar_type() || x.sizes() != at::IntArrayRef(key_rows) || !x.is_contiguous())
            Py_RETURN_NONE;
    if (!per_sequence(len_in, g.S) || !per_sequence(len_out, g.S) || gate.scalar_type() != at::kFloat ||
        !turn_ok(t, sections, {g.S}, g.D))
        Py_RETURN_NONE;
    int64_t gss, gsh;
    if (gate.dim() == 1 && gate.size(0) == H) {
        gss = 0;
        gsh = gate.stride(0);
    } else if (gate.dim() == 2 && gate.size(0) == g.S && gate.size(1) == H) {
        gss = gate.stride(0);
        gsh = gate.stride(1);
    } else {
        Py_RETURN_NONE;
    }
    if (out.defined() && (out.scalar_type() != q.scalar_type() || out.sizes() != q.sizes() || !out.is_contiguous()))
        Py_RETURN_NONE;
    if (lse.defined() && !is_f32(lse, {g.S, H})) Py_RETURN_NONE;
    const int64_t need = pi_attn_paged_workspace(dtype_of(q), g.S, H, g.Hk, g.D, g.page, g.max, kw);
    if (need < 0) Py_RETURN_NONE;
    if (work.defined() && (work.scalar_type() != at::kFloat || !work.is_contiguous() || work.numel() < need))
        Py_RETURN_NONE;
    int status;
    {
        pybind11::gil_scoped_release no_gil;
        const c10::DeviceGuard on(a.device);
        if (!out.defined()) out = at::empty(q.sizes(), at::TensorOptions().dtype(q.scalar_type()).device(a.device));
        if (!work.defined() && need > 0) work = at::empty({need}, at::TensorOptions().dtype(at::kFloat).device(a.device));
        status = pi_attn_decode_step_paged(
            dtype_of(q), g.S, H, g.Hk, g.D, g.n, g.page, g.max, kw, pi, ptr<int32_t>(len_in), ptr<int32_t>(len_out),
            q.data_ptr(), k.data_ptr(), v.data_ptr(), ptr<int32_t>(g.table), g.k.data_ptr(), g.v.data_ptr(),
            ptr<uint8_t>(g.ke), ptr<uint8_t>(g.ve), ptr<float>(t.freq), t.pairs[0], t.pairs[1], t.pairs[2],
            ptr<int32_t>(t.pos), t.ps[0], t.ps[1], ptr<float>(gate), gss, gsh, scale, clamp, out.data_ptr(),
            ptr<float>(lse), ptr<float>(work), stream_of(a.device));
    }
    if (status != PI_ATTN_OK) return refused(self, status, "pi_attn_decode_step_paged");
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

template <typename F>
PyCFunction fast(F f) {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef methods[] = {{"forward", fast(forward), METH_FASTCALL, nullptr},
                         {"forward_gated", fast(forward_gated), METH_FASTCALL, nullptr},
                         {"backward", fast(backward), METH_FASTCALL, nullptr},
                         {"decode_step", fast(decode_step), METH_FASTCALL, nullptr},
                         {"cache_store", fast(cache_store), METH_FASTCALL, nullptr},
                         {"cache_load", fast(cache_load), METH_FASTCALL, nullptr},
                         {"decode_step_e4m3", fast(decode_step_e4m3), METH_FASTCALL, nullptr},
                         {"decode_step_prefix", fast(decode_step_prefix), METH_FASTCALL, nullptr},
                         {"rotate", fast(rotate), METH_FASTCALL, nullptr},
                         {"paged_store", fast(paged_store), METH_FASTCALL, nullptr},
                         {"paged_load", fast(paged_load), METH_FASTCALL, nullptr},
                         {"decode_step_paged", fast(decode_step_paged), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
