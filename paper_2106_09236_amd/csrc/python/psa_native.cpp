// The Python entry points of the hot calls, in native code: tensors in, checks, allocation of what the caller did not
// bring, the current stream, one call of the C ABI.  For short utterances the GPU is done in 10 us; marshalling the
// same call through ctypes took 8 us of the interpreter's time on top of the launches (B=1 H=4 L=128, output and
// scratch given: 13.0 us per call, here 8.7, of which two launches are 5).
//
// A function returns None where anything is out of the ordinary before the library is called (an argument that is no
// contiguous device tensor, an unknown type, no memory); nothing has been enqueued then, and the caller's ctypes path takes
// over, which reports the error.  A status other than PSA_OK is raised from here: a launch that failed may come after
// stages that have been enqueued, and those are not enqueued again.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../../include/probsparse.h"

namespace {

// A device tensor argument: a contiguous tensor on a GPU, or None where `optional`.
struct Arg {
    const at::Tensor* t = nullptr;
    void* ptr = nullptr;
};
bool take(PyObject* o, Arg& a, bool optional)
{
    if (o == Py_None) return optional;
    if (!THPVariable_Check(o)) return false;
    a.t = &THPVariable_Unpack(o);
    if (!a.t->is_cuda() || !a.t->is_contiguous()) return false;
    a.ptr = a.t->data_ptr();
    return true;
}
bool dtype_of(const at::Tensor& t, int32_t* dtype)
{
    const auto s = t.scalar_type();
    if (s == at::kFloat) { *dtype = PSA_F32; return true; }
    if (s == at::kBFloat16) { *dtype = PSA_BF16; return true; }
    return false;
}
// shape of Q [B, H, L, D]; U is the last dimension of sample_idx, or 1
bool shape_of(const at::Tensor& q, const Arg& idx, psa_shape_t* s)
{
    if (q.dim() != 4 || (idx.t && idx.t->dim() < 1)) return false;
    s->B = (int32_t)q.size(0); s->H = (int32_t)q.size(1); s->L_Q = s->L_K = (int32_t)q.size(2); s->D = (int32_t)q.size(3);
    s->U = idx.t ? (int32_t)idx.t->size(-1) : 1;
    return dtype_of(q, &s->dtype);
}
void* stream() { return c10::hip::getCurrentHIPStream().stream(); }
at::Tensor scratch(const at::Tensor& like, size_t bytes)
{
    return at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
}
PyObject* none() { Py_RETURN_NONE; }
// what raises the binding's exception for a status (set by the binding)
PyObject* raise_status = nullptr;
PyObject* failed(int rc)
{
    PyObject* r = raise_status ? PyObject_CallFunction(raise_status, "i", rc) : nullptr;
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_Format(PyExc_RuntimeError, "libprobsparse: status %d", rc);
    return nullptr;
}
PyObject* on_status(PyObject*, PyObject* callable)
{
    Py_INCREF(callable);
    Py_XSETREF(raise_status, callable);
    Py_RETURN_NONE;
}
// Other Python threads run while a call allocates and enqueues: either may wait (for memory, for room in a queue).
// No Python object is touched inside; the caller holds the arguments.
struct Unlocked {
    PyThreadState* const state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked&) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};
// the caller's output object, or the one made here
PyObject* result(PyObject* given, at::Tensor&& made)
{
    if (given == Py_None) return THPVariable_Wrap(std::move(made));
    Py_INCREF(given);
    return given;
}

// The forward's common part: Q, K, V, lengths, sample_idx, options, out, workspace (the last two may be None).
PyObject* forward(PyObject* const* a, const psa_options_t& opt, PyObject* out_o, PyObject* ws_o)
{
    Arg q, k, v, len, idx, out, ws;
    if (!take(a[0], q, false) || !take(a[1], k, false) || !take(a[2], v, false) || !take(a[3], len, true) ||
        !take(a[4], idx, false) || !take(out_o, out, true) || !take(ws_o, ws, true)) return none();
    psa_shape_t s;
    if (!shape_of(*q.t, idx, &s)) return none();
    at::Tensor made, room;
    const size_t bytes = ws.t ? (size_t)ws.t->numel() : probsparse_attn_workspace_bytes_opt(&s, &opt);
    if (bytes == 0) return none();
    int rc;
    {
        const Unlocked unlocked;
        if (!ws.t) { room = scratch(*q.t, bytes); ws.ptr = room.data_ptr(); }
        if (!out.t) { made = at::empty_like(*q.t); out.ptr = made.data_ptr(); }
        rc = probsparse_attn_fwd_opt(q.ptr, k.ptr, v.ptr, static_cast<const int32_t*>(len.ptr),
                                     static_cast<const int32_t*>(idx.ptr), &opt, out.ptr, &s, ws.ptr, bytes, stream(),
                                     nullptr, nullptr, nullptr);
    }
    return rc == PSA_OK ? result(out_o, std::move(made)) : failed(rc);
}

// attn_fwd(Q, K, V, lengths, sample_idx, c, out, workspace)
PyObject* attn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 8) return none();
    const double c = PyFloat_AsDouble(a[5]);
    if (PyErr_Occurred()) { PyErr_Clear(); return none(); }
    return forward(a, psa_options_t{PSA_U_LOG, PSA_FILL_MEAN, c}, a[6], a[7]);
}

bool option_args(PyObject* rule, PyObject* factor, PyObject* fill, psa_options_t* o)
{
    o->u_rule = (int32_t)PyLong_AsLong(rule);
    o->factor = PyFloat_AsDouble(factor);
    o->fill = (int32_t)PyLong_AsLong(fill);
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}

// attn_fwd_opt(Q, K, V, lengths, sample_idx, u_rule, factor, fill, out, workspace), without taps
PyObject* attn_fwd_opt(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    psa_options_t opt;
    if (n != 10 || !option_args(a[5], a[6], a[7], &opt)) return none();
    return forward(a, opt, a[8], a[9]);
}

// attn_fwd_with_indices(Q, K, V, lengths, sel, u, fill, out, workspace)
PyObject* attn_fwd_with_indices(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Arg q, k, v, len, sel, u, out, ws;
    if (n != 9 || !take(a[0], q, false) || !take(a[1], k, false) || !take(a[2], v, false) || !take(a[3], len, true) ||
        !take(a[4], sel, false) || !take(a[5], u, false) || !take(a[7], out, true) || !take(a[8], ws, true)) return none();
    const int32_t fill = (int32_t)PyLong_AsLong(a[6]);
    if (PyErr_Occurred()) { PyErr_Clear(); return none(); }
    psa_shape_t s;
    if (!shape_of(*q.t, Arg{}, &s) || sel.t->dim() < 1) return none();
    const int32_t stride = (int32_t)sel.t->size(-1);
    at::Tensor made, room;
    const size_t bytes = ws.t ? (size_t)ws.t->numel() : probsparse_attn_with_indices_workspace_bytes(&s, stride);
    if (bytes == 0) return none();
    int rc;
    {
        const Unlocked unlocked;
        if (!ws.t) { room = scratch(*q.t, bytes); ws.ptr = room.data_ptr(); }
        if (!out.t) { made = at::empty_like(*q.t); out.ptr = made.data_ptr(); }
        rc = probsparse_attn_fwd_with_indices(q.ptr, k.ptr, v.ptr, static_cast<const int32_t*>(len.ptr),
                                              static_cast<const int32_t*>(sel.ptr), static_cast<const int32_t*>(u.ptr),
                                              stride, fill, out.ptr, &s, ws.ptr, bytes, stream());
    }
    return rc == PSA_OK ? result(a[7], std::move(made)) : failed(rc);
}

// attn_bwd(Q, K, V, lengths, sel, u, dOut, fill, workspace) -> (dQ, dK, dV)
PyObject* attn_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Arg q, k, v, len, sel, u, g, ws;
    if (n != 9 || !take(a[0], q, false) || !take(a[1], k, false) || !take(a[2], v, false) || !take(a[3], len, true) ||
        !take(a[4], sel, false) || !take(a[5], u, false) || !take(a[6], g, false) || !take(a[8], ws, true)) return none();
    const int32_t fill = (int32_t)PyLong_AsLong(a[7]);
    if (PyErr_Occurred()) { PyErr_Clear(); return none(); }
    psa_shape_t s;
    if (!shape_of(*q.t, Arg{}, &s) || sel.t->dim() < 1) return none();
    const int32_t stride = (int32_t)sel.t->size(-1);
    at::Tensor room, dq, dk, dv;
    const size_t bytes = ws.t ? (size_t)ws.t->numel() : probsparse_attn_bwd_workspace_bytes(&s, stride);
    if (bytes == 0) return none();
    int rc;
    {
        const Unlocked unlocked;
        if (!ws.t) { room = scratch(*q.t, bytes); ws.ptr = room.data_ptr(); }
        dq = at::empty_like(*q.t); dk = at::empty_like(*q.t); dv = at::empty_like(*q.t);
        rc = probsparse_attn_bwd(q.ptr, k.ptr, v.ptr, static_cast<const int32_t*>(len.ptr),
                                 static_cast<const int32_t*>(sel.ptr), static_cast<const int32_t*>(u.ptr), stride, fill,
                                 g.ptr, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), &s, ws.ptr, bytes, stream());
    }
    if (rc != PSA_OK) return failed(rc);
    PyObject* t = PyTuple_New(3);
    if (!t) return nullptr;
    PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(std::move(dq)));
    PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(std::move(dk)));
    PyTuple_SET_ITEM(t, 2, THPVariable_Wrap(std::move(dv)));
    return t;
}

// mhsa_fwd(X, weights, lengths, sample_idx, u_rule, factor, fill, Y, workspace); `weights`: anything whose buffer is a
// psa_mhsa_weights_t (the ctypes structure of the binding)
PyObject* mhsa_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Arg x, len, idx, y, ws;
    psa_options_t opt;
    if (n != 9 || !take(a[0], x, false) || !take(a[2], len, true) || !take(a[3], idx, false) ||
        !option_args(a[4], a[5], a[6], &opt) || !take(a[7], y, true) || !take(a[8], ws, true)) return none();
    if (x.t->dim() != 3 || idx.t->dim() < 1) return none();
    psa_shape_t s;
    s.B = (int32_t)x.t->size(0); s.H = (int32_t)(x.t->size(2) / 64); s.L_Q = s.L_K = (int32_t)x.t->size(1); s.D = 64;
    s.U = (int32_t)idx.t->size(-1);
    if (!dtype_of(*x.t, &s.dtype)) return none();
    Py_buffer view;
    if (PyObject_GetBuffer(a[1], &view, PyBUF_SIMPLE) != 0) { PyErr_Clear(); return none(); }
    psa_mhsa_weights_t w;
    const bool whole = view.len == (Py_ssize_t)sizeof(w);
    if (whole) w = *static_cast<const psa_mhsa_weights_t*>(view.buf);
    PyBuffer_Release(&view);
    if (!whole) return none();
    at::Tensor made, room;
    const size_t bytes = ws.t ? (size_t)ws.t->numel() : probsparse_mhsa_workspace_bytes(&s, &opt);
    if (bytes == 0) return none();
    int rc;
    {
        const Unlocked unlocked;
        if (!ws.t) { room = scratch(*x.t, bytes); ws.ptr = room.data_ptr(); }
        if (!y.t) { made = at::empty_like(*x.t); y.ptr = made.data_ptr(); }
        rc = probsparse_mhsa_fwd(x.ptr, &w, static_cast<const int32_t*>(len.ptr), static_cast<const int32_t*>(idx.ptr),
                                 &opt, y.ptr, &s, ws.ptr, bytes, stream());
    }
    return rc == PSA_OK ? result(a[7], std::move(made)) : failed(rc);
}

// ---- layer norm, rotary positions, dense attention over packed sequences.  Everything has to be on the current device here; the
// caller's path switches to the tensors' own.
bool here(const at::Tensor& t) { return t.is_cuda() && t.device().index() == c10::hip::current_device(); }

bool take_like(PyObject* o, Arg& a, at::IntArrayRef sizes, at::ScalarType type, bool optional)
{
    if (!take(o, a, optional)) return false;
    return !a.t || (here(*a.t) && a.t->scalar_type() == type && a.t->sizes() == sizes);
}
// A tensor of heads [B, H, L, 64] or [H, T, 64] with any strides
struct HeadsArg {
    const at::Tensor* t = nullptr;
    psa_heads_t h{};
    const psa_heads_t* ptr() const { return t ? &h : nullptr; }
    void set(const at::Tensor& x) {
        const int64_t n = x.dim();
        h = psa_heads_t{x.data_ptr(), n == 4 ? x.stride(0) : 0, x.stride(n - 3), x.stride(n - 2)};
    }
};
bool take_heads(PyObject* o, HeadsArg& a, bool optional)
{
    if (o == Py_None) return optional;
    if (!THPVariable_Check(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if ((t.dim() != 3 && t.dim() != 4) || t.size(-1) != 64 || t.stride(-1) != 1 || t.numel() == 0 || !here(t)) return false;
    a.t = &t;
    a.set(t);
    return true;
}
bool take_heads_like(PyObject* o, HeadsArg& a, const at::Tensor& like, bool optional)
{
    return take_heads(o, a, optional) && (!a.t || (a.t->sizes() == like.sizes() && a.t->scalar_type() == like.scalar_type()));
}
void make_heads(HeadsArg& a, at::Tensor& made, const at::Tensor& like)
{
    if (a.t) return;
    made = at::empty_like(like);
    a.set(made);
}
PyObject* tuple(PyObject* const* objects, int n)
{
    PyObject* t = PyTuple_New(n);
    for (int i = 0; i < n; ++i) {
        if (t && objects[i]) PyTuple_SET_ITEM(t, i, objects[i]);
        else Py_XDECREF(objects[i]);
    }
    return t;
}

// layer_norm_fwd(X, gamma, beta, eps, Y, stats) -> Y or (Y, mean, rstd)
PyObject* layer_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Arg x, g, b, y;
    if (n != 6 || !take(a[0], x, false) || !here(*x.t) || x.t->dim() < 1 || x.t->numel() == 0) return none();
    const int64_t cols = x.t->size(-1), rows = x.t->numel() / cols;
    const auto type = x.t->scalar_type();
    int32_t dtype;
    const double eps = PyFloat_AsDouble(a[3]);
    const int stats = PyObject_IsTrue(a[5]);
    if (PyErr_Occurred()) { PyErr_Clear(); return none(); }
    if (cols > INT32_MAX || !dtype_of(*x.t, &dtype) || !take_like(a[1], g, {cols}, type, true) || !take_like(a[2], b, {cols}, type, true) ||
        !take_like(a[4], y, x.t->sizes(), type, true)) return none();
    at::Tensor made, mean, rstd;
    int rc;
    {
        const Unlocked unlocked;
        if (!y.t) { made = at::empty_like(*x.t); y.ptr = made.data_ptr(); }
        if (stats) {
            const auto lead = x.t->sizes().slice(0, x.t->dim() - 1);
            mean = at::empty(lead, x.t->options().dtype(at::kFloat));
            rstd = at::empty(lead, x.t->options().dtype(at::kFloat));
        }
        rc = probsparse_layer_norm_fwd(x.ptr, g.ptr, b.ptr, eps, y.ptr, stats ? mean.data_ptr<float>() : nullptr,
                                       stats ? rstd.data_ptr<float>() : nullptr, rows, (int32_t)cols, dtype, stream());
    }
    if (rc != PSA_OK) return failed(rc);
    PyObject* r = result(a[4], std::move(made));
    if (!stats) return r;
    PyObject* const all[] = {r, THPVariable_Wrap(std::move(mean)), THPVariable_Wrap(std::move(rstd))};
    return tuple(all, 3);
}

// layer_norm_bwd(dY, X, gamma, mean, rstd, workspace) -> (dX, dgamma, dbeta)
PyObject* layer_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Arg dy, x, g, m, r, ws;
    if (n != 6 || !take(a[1], x, false) || !here(*x.t) || x.t->dim() < 1 || x.t->numel() == 0) return none();
    const int64_t cols = x.t->size(-1), rows = x.t->numel() / cols;
    const auto type = x.t->scalar_type();
    const auto lead = x.t->sizes().slice(0, x.t->dim() - 1);
    int32_t dtype;
    if (cols > INT32_MAX || !dtype_of(*x.t, &dtype) || !take_like(a[0], dy, x.t->sizes(), type, false) || !take_like(a[2], g, {cols}, type, true) ||
        !take_like(a[3], m, lead, at::kFloat, false) || !take_like(a[4], r, lead, at::kFloat, false) || !take(a[5], ws, true) ||
        (ws.t && !here(*ws.t))) return none();
    const size_t bytes = ws.t ? ws.t->nbytes() : probsparse_layer_norm_bwd_workspace_bytes(rows, (int32_t)cols, dtype);
    if (bytes == 0) return none();
    at::Tensor room, dx, dg, db;
    int rc;
    {
        const Unlocked unlocked;
        if (!ws.t) { room = scratch(*x.t, bytes); ws.ptr = room.data_ptr(); }
        dx = at::empty_like(*x.t);
        dg = at::empty({cols}, x.t->options().dtype(at::kFloat));
        db = at::empty({cols}, x.t->options().dtype(at::kFloat));
        rc = probsparse_layer_norm_bwd(dy.ptr, x.ptr, g.ptr, static_cast<const float*>(m.ptr), static_cast<const float*>(r.ptr), dx.data_ptr(),
                                       dg.data_ptr<float>(), db.data_ptr<float>(), rows, (int32_t)cols, dtype, ws.ptr, bytes, stream());
    }
    if (rc != PSA_OK) return failed(rc);
    PyObject* const all[] = {THPVariable_Wrap(std::move(dx)), THPVariable_Wrap(std::move(dg)), THPVariable_Wrap(std::move(db))};
    return tuple(all, 3);
}

// rotary(back, Q, K, rotary, positions, first, Q_out, K_out) -> Q_out or (Q_out, K_out)
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HeadsArg q, k, qo, ko;
    Arg pos;
    if (n != 8 || !take_heads(a[1], q, false) || !take_heads(a[2], k, true) || !take(a[4], pos, true) || !take_heads_like(a[6], qo, *q.t, true)) return none();
    const int back = PyObject_IsTrue(a[0]);
    const long first = PyLong_AsLong(a[5]);
    if (PyErr_Occurred()) { PyErr_Clear(); return none(); }
    const int64_t dim = q.t->dim(), B = dim == 4 ? q.t->size(0) : 1, H = q.t->size(dim - 3), L = q.t->size(dim - 2);
    if (first != (int32_t)first || B > INT32_MAX || H > INT32_MAX || L > INT32_MAX) return none();
    psa_shape_t s{(int32_t)B, (int32_t)H, (int32_t)L, (int32_t)L, 64, 1, 0};
    if (!dtype_of(*q.t, &s.dtype)) return none();
    if (k.t) {
        if (k.t->dim() != dim || (dim == 4 && k.t->size(0) != B) || k.t->size(dim - 2) != L || k.t->scalar_type() != q.t->scalar_type() ||
            !take_heads_like(a[7], ko, *k.t, true)) return none();
    } else if (a[7] != Py_None) {
        return none();
    }
    if (pos.t && (!here(*pos.t) || pos.t->scalar_type() != at::kInt || (pos.t->sizes() != at::IntArrayRef({L}) && pos.t->sizes() != at::IntArrayRef({B, L})))) return none();
    Py_buffer view;
    if (PyObject_GetBuffer(a[3], &view, PyBUF_SIMPLE) != 0) { PyErr_Clear(); return none(); }
    psa_rotary_t o;
    const bool whole = view.len == (Py_ssize_t)sizeof(o);
    if (whole) o = *static_cast<const psa_rotary_t*>(view.buf);
    PyBuffer_Release(&view);
    if (!whole) return none();
    at::Tensor q_made, k_made;
    int rc;
    {
        const Unlocked unlocked;
        make_heads(qo, q_made, *q.t);
        if (k.t) make_heads(ko, k_made, *k.t);
        rc = (back ? probsparse_rotary_bwd : probsparse_rotary_fwd)(&q.h, k.ptr(), k.t ? (int32_t)k.t->size(dim - 3) : 0, &o, static_cast<const int32_t*>(pos.ptr),
                                                                    pos.t && pos.t->dim() == 2 ? L : 0, (int32_t)first, &qo.h, k.t ? &ko.h : nullptr, &s, stream());
    }
    if (rc != PSA_OK) return failed(rc);
    PyObject* r = result(a[6], std::move(q_made));
    if (!k.t) return r;
    PyObject* const all[] = {r, result(a[7], std::move(k_made))};
    return tuple(all, 2);
}

// Q, K, V, q_offsets, k_offsets, causal, scale
struct Packed {
    HeadsArg q, k, v;
    Arg qo, ko;
    psa_packed_shape_t s{};
    bool take_all(PyObject* const* a, PyObject* qo_o, PyObject* ko_o, PyObject* causal, PyObject* scale) {
        if (!take_heads(a[0], q, false) || !take_heads(a[1], k, false) || q.t->dim() != 3 || k.t->dim() != 3 || !take_heads_like(a[2], v, *k.t, false) ||
            q.t->scalar_type() != k.t->scalar_type()) return false;
        int64_t B = 1;
        if (qo_o != Py_None) {
            if (ko_o == Py_None && q.t->size(1) != k.t->size(1)) return false;
            if (!take(qo_o, qo, false) || qo.t->dim() != 1 || qo.t->numel() < 2 || qo.t->scalar_type() != at::kInt || !here(*qo.t) ||
                !take_like(ko_o == Py_None ? qo_o : ko_o, ko, qo.t->sizes(), at::kInt, false)) return false;
            B = qo.t->numel() - 1;
        } else if (ko_o != Py_None) {
            return false;
        }
        const int c = PyObject_IsTrue(causal);
        const double f = scale == Py_None ? 0.125 : PyFloat_AsDouble(scale);
        if (PyErr_Occurred()) { PyErr_Clear(); return false; }
        if (B > INT32_MAX || q.t->size(0) % k.t->size(0) != 0 || q.t->size(0) > INT32_MAX || q.t->size(1) > INT32_MAX || k.t->size(1) > INT32_MAX) return false;
        s = psa_packed_shape_t{(int32_t)B, (int32_t)q.t->size(0), (int32_t)k.t->size(0), (int32_t)q.t->size(1), (int32_t)k.t->size(1), 64, 0, c, f};
        return dtype_of(*q.t, &s.dtype);
    }
    const int32_t* q_offsets() const { return static_cast<const int32_t*>(qo.ptr); }
    const int32_t* k_offsets() const { return static_cast<const int32_t*>(ko.ptr); }
};

// packed_fwd(Q, K, V, q_offsets, k_offsets, causal, scale, out, lse, workspace) -> out or (out, lse)
PyObject* packed_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Packed p;
    HeadsArg out;
    Arg ws;
    if (n != 10 || !p.take_all(a, a[3], a[4], a[5], a[6]) || !take_heads_like(a[7], out, *p.q.t, true) || !take(a[9], ws, true) || (ws.t && !here(*ws.t))) return none();
    const int want_lse = PyObject_IsTrue(a[8]);
    if (PyErr_Occurred()) { PyErr_Clear(); return none(); }
    const size_t bytes = ws.t ? ws.t->nbytes() : dense_attn_packed_workspace_bytes(&p.s);
    if (bytes == 0) return none();
    at::Tensor made, lse, room;
    int rc;
    {
        const Unlocked unlocked;
        if (!ws.t) { room = scratch(*p.q.t, bytes); ws.ptr = room.data_ptr(); }
        make_heads(out, made, *p.q.t);
        if (want_lse) lse = at::empty({p.q.t->size(0), p.q.t->size(1)}, p.q.t->options().dtype(at::kFloat));
        rc = dense_attn_packed_fwd(&p.q.h, &p.k.h, &p.v.h, p.q_offsets(), p.k_offsets(), &out.h, want_lse ? lse.data_ptr<float>() : nullptr, &p.s,
                                   ws.ptr, bytes, stream());
    }
    if (rc != PSA_OK) return failed(rc);
    PyObject* r = result(a[7], std::move(made));
    if (!want_lse) return r;
    PyObject* const all[] = {r, THPVariable_Wrap(std::move(lse))};
    return tuple(all, 2);
}

// packed_bwd(Q, K, V, out, lse, dOut, q_offsets, k_offsets, causal, scale, dQ, dK, dV, workspace) -> (dQ, dK, dV)
PyObject* packed_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Packed p;
    HeadsArg out, g, dq, dk, dv;
    Arg lse, ws;
    if (n != 14 || !p.take_all(a, a[6], a[7], a[8], a[9]) || !take_heads_like(a[3], out, *p.q.t, false) ||
        !take_like(a[4], lse, {p.q.t->size(0), p.q.t->size(1)}, at::kFloat, false) || !take_heads_like(a[5], g, *p.q.t, false) ||
        !take_heads_like(a[10], dq, *p.q.t, true) || !take_heads_like(a[11], dk, *p.k.t, true) || !take_heads_like(a[12], dv, *p.k.t, true) ||
        !take(a[13], ws, true) || (ws.t && !here(*ws.t))) return none();
    const size_t bytes = ws.t ? ws.t->nbytes() : dense_attn_packed_bwd_workspace_bytes(&p.s);
    if (bytes == 0) return none();
    at::Tensor room, made[3];
    int rc;
    {
        const Unlocked unlocked;
        if (!ws.t) { room = scratch(*p.q.t, bytes); ws.ptr = room.data_ptr(); }
        make_heads(dq, made[0], *p.q.t);
        make_heads(dk, made[1], *p.k.t);
        make_heads(dv, made[2], *p.v.t);
        rc = dense_attn_packed_bwd(&p.q.h, &p.k.h, &p.v.h, p.q_offsets(), p.k_offsets(), &out.h, static_cast<const float*>(lse.ptr), &g.h, &dq.h, &dk.h,
                                   &dv.h, &p.s, ws.ptr, bytes, stream());
    }
    if (rc != PSA_OK) return failed(rc);
    PyObject* const all[] = {result(a[10], std::move(made[0])), result(a[11], std::move(made[1])), result(a[12], std::move(made[2]))};
    return tuple(all, 3);
}

// ---- a cache in pages
// K_pages, V_pages, table, lengths, offsets, K_scales, V_scales, of new rows `rows`
struct CacheArg {
    HeadsArg k, v;
    Arg table, lengths, offsets;
    psa_cache_t c{};
    int64_t B = 0;
    static bool scales(PyObject* o, const at::Tensor& pages, psa_heads_t& h) {
        if (!THPVariable_Check(o)) return false;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.dim() != 4 || t.scalar_type() != at::kByte || !here(t) || t.stride(3) != 1 || t.size(3) != 2) return false;
        for (int i = 0; i < 3; ++i) if (t.size(i) != pages.size(i)) return false;
        h = psa_heads_t{t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
        return true;
    }
    bool take_all(const at::Tensor& rows, PyObject* k_o, PyObject* v_o, PyObject* table_o, PyObject* lengths_o, PyObject* offsets_o, PyObject* ks_o, PyObject* vs_o) {
        if (!take_heads(k_o, k, false) || k.t->dim() != 4 || !take_heads_like(v_o, v, *k.t, false)) return false;
        const bool mx = k.t->scalar_type() == at::kFloat8_e4m3fn;
        if (!mx && (k.t->scalar_type() != rows.scalar_type() || ks_o != Py_None || vs_o != Py_None)) return false;
        if (mx && (!scales(ks_o, *k.t, c.K_scales) || !scales(vs_o, *k.t, c.V_scales))) return false;
        if (!take(table_o, table, false) || table.t->dim() != 2 || table.t->numel() == 0 || table.t->scalar_type() != at::kInt || !here(*table.t)) return false;
        B = table.t->size(0);
        if (!take_like(lengths_o, lengths, {B}, at::kInt, false) || !take_like(offsets_o, offsets, {B + 1}, at::kInt, true)) return false;
        if (B > INT32_MAX || table.t->size(1) > INT32_MAX || k.t->size(0) > INT32_MAX || k.t->size(1) > INT32_MAX || k.t->size(2) > INT32_MAX ||
            rows.size(1) > INT32_MAX || rows.size(0) > INT32_MAX || (!offsets.t && rows.size(1) % B != 0)) return false;
        c.K = k.h;
        c.V = v.h;
        c.table = static_cast<const int32_t*>(table.ptr);
        c.lengths = static_cast<const int32_t*>(lengths.ptr);
        c.n_pages = (int32_t)k.t->size(0);
        c.page_rows = (int32_t)k.t->size(2);
        c.max_pages = (int32_t)table.t->size(1);
        c.format = mx ? PSA_CACHE_MX : PSA_CACHE_PLAIN;
        return true;
    }
    const int32_t* rows_of() const { return static_cast<const int32_t*>(offsets.ptr); }
};

// cache_append(K, V, K_pages, V_pages, table, lengths, offsets, K_scales, V_scales) -> True
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HeadsArg k, v;
    CacheArg c;
    psa_paged_shape_t s{};
    if (n != 9 || !take_heads(a[0], k, false) || k.t->dim() != 3 || !take_heads_like(a[1], v, *k.t, false) || !dtype_of(*k.t, &s.dtype) ||
        !c.take_all(*k.t, a[2], a[3], a[4], a[5], a[6], a[7], a[8]) || c.k.t->size(1) != k.t->size(0)) return none();
    s.B = (int32_t)c.B; s.H = s.H_kv = (int32_t)k.t->size(0); s.T = (int32_t)k.t->size(1); s.D = 64; s.scale = 0.125;
    int rc;
    {
        const Unlocked unlocked;
        rc = probsparse_cache_append(&k.h, &v.h, c.rows_of(), &c.c, &s, stream());
    }
    if (rc != PSA_OK) return failed(rc);
    Py_RETURN_TRUE;
}

// paged_fwd(Q, K_pages, V_pages, table, lengths, offsets, causal, scale, K_scales, V_scales, out, lse, workspace) -> out or (out, lse)
PyObject* paged_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HeadsArg q, out;
    CacheArg c;
    Arg ws;
    psa_paged_shape_t s{};
    if (n != 13 || !take_heads(a[0], q, false) || q.t->dim() != 3 || !dtype_of(*q.t, &s.dtype) || !c.take_all(*q.t, a[1], a[2], a[3], a[4], a[5], a[8], a[9]) ||
        q.t->size(0) % c.k.t->size(1) != 0 || !take_heads_like(a[10], out, *q.t, true) || !take(a[12], ws, true) || (ws.t && !here(*ws.t))) return none();
    s.causal = PyObject_IsTrue(a[6]);
    s.scale = a[7] == Py_None ? 0.125 : PyFloat_AsDouble(a[7]);
    const int want_lse = PyObject_IsTrue(a[11]);
    if (PyErr_Occurred()) { PyErr_Clear(); return none(); }
    s.B = (int32_t)c.B; s.H = (int32_t)q.t->size(0); s.H_kv = (int32_t)c.k.t->size(1); s.T = (int32_t)q.t->size(1); s.D = 64;
    const size_t bytes = ws.t ? ws.t->nbytes() : dense_attn_paged_workspace_bytes(&c.c, &s);
    if (bytes == 0) return none();
    at::Tensor made, lse, room;
    int rc;
    {
        const Unlocked unlocked;
        if (!ws.t) { room = scratch(*q.t, bytes); ws.ptr = room.data_ptr(); }
        make_heads(out, made, *q.t);
        if (want_lse) lse = at::empty({q.t->size(0), q.t->size(1)}, q.t->options().dtype(at::kFloat));
        rc = dense_attn_paged_fwd(&q.h, c.rows_of(), &c.c, &out.h, want_lse ? lse.data_ptr<float>() : nullptr, &s, ws.ptr, bytes, stream());
    }
    if (rc != PSA_OK) return failed(rc);
    PyObject* r = result(a[10], std::move(made));
    if (!want_lse) return r;
    PyObject* const all[] = {r, THPVariable_Wrap(std::move(lse))};
    return tuple(all, 2);
}

int32_t* ints(const Arg& a) { return static_cast<int32_t*>(a.ptr); }
// The integer outputs that the caller did not bring, as parts of one allocation: each of its own takes 0.7 us of a call whose kernel takes 7
struct Ints { Arg& a; at::Tensor& made; int64_t rows, cols; };     // cols 0: one dimension
void make_ints(std::initializer_list<Ints> all, const at::Tensor& like)
{
    auto size = [](const Ints& x) { return (x.rows * (x.cols ? x.cols : 1) + 3) & ~(int64_t)3; };
    int64_t total = 0, at = 0;
    for (const Ints& x : all) if (!x.a.t) total += size(x);
    if (total == 0) return;
    const at::AutoDispatchBelowADInplaceOrView quick;
    const at::Tensor room = at::empty({total}, like.options());
    for (const Ints& x : all) {
        if (x.a.t) continue;
        x.made = x.cols ? room.as_strided({x.rows, x.cols}, {x.cols, 1}, at) : room.as_strided({x.rows}, {1}, at);
        x.a.ptr = room.data_ptr<int32_t>() + at;
        at += size(x);
    }
}
bool int_arg(PyObject* o, int32_t* x)
{
    const long v = PyLong_AsLong(o);
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    *x = (int32_t)v;
    return v >= INT32_MIN && v <= INT32_MAX;
}

// cache_update(table, lengths, refs, page_rows, parents, grow, table_out, lengths_out, refs_out, pairs, counts, workspace) -> the five outputs
PyObject* cache_update(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Arg table, lengths, refs, parents, grow, out[5], ws;
    int32_t page_rows;
    if (n != 12 || !take(a[0], table, false) || table.t->dim() != 2 || table.t->numel() == 0 || table.t->scalar_type() != at::kInt || !here(*table.t)) return none();
    const int64_t B = table.t->size(0), max_pages = table.t->size(1);
    if (!take_like(a[1], lengths, {B}, at::kInt, false) || !take(a[2], refs, false) || refs.t->dim() != 1 || refs.t->numel() == 0 || refs.t->scalar_type() != at::kInt ||
        !here(*refs.t) || !int_arg(a[3], &page_rows) || !take(a[4], parents, true)) return none();
    const int64_t n_pages = refs.t->numel(), B_out = parents.t ? parents.t->numel() : B;
    if (B_out == 0 || (parents.t && (parents.t->dim() != 1 || parents.t->scalar_type() != at::kInt || !here(*parents.t))) || !take_like(a[5], grow, {B_out}, at::kInt, true) ||
        !take_like(a[6], out[0], {B_out, max_pages}, at::kInt, true) || !take_like(a[7], out[1], {B_out}, at::kInt, true) || !take_like(a[8], out[2], {n_pages}, at::kInt, true) ||
        !take_like(a[9], out[3], {B_out, 2}, at::kInt, true) || !take_like(a[10], out[4], {2}, at::kInt, true) || !take(a[11], ws, true) || (ws.t && !here(*ws.t)) ||
        B > INT32_MAX || B_out > INT32_MAX || n_pages > INT32_MAX || max_pages > INT32_MAX) return none();
    const size_t bytes = ws.t ? ws.t->nbytes() : probsparse_cache_update_workspace_bytes((int32_t)B, (int32_t)B_out, (int32_t)n_pages);
    if (bytes == 0) return none();
    at::Tensor made[5], room;
    int rc;
    {
        const Unlocked unlocked;
        if (!ws.t) { room = at::empty({(int64_t)bytes}, table.t->options().dtype(at::kByte)); ws.ptr = room.data_ptr(); }
        make_ints({{out[0], made[0], B_out, max_pages}, {out[1], made[1], B_out, 0}, {out[2], made[2], n_pages, 0}, {out[3], made[3], B_out, 2}, {out[4], made[4], 2, 0}}, *table.t);
        rc = probsparse_cache_update(ints(table), ints(lengths), ints(refs), (int32_t)B, ints(parents), ints(grow), (int32_t)B_out, (int32_t)n_pages, page_rows, (int32_t)max_pages,
                                     ints(out[0]), ints(out[1]), ints(out[2]), ints(out[3]), ints(out[4]), ws.ptr, bytes, stream());
    }
    if (rc != PSA_OK) return failed(rc);
    PyObject* all[5];
    for (int i = 0; i < 5; ++i) all[i] = result(a[6 + i], std::move(made[i]));
    return tuple(all, 5);
}

// cache_compact(table, refs, table_out, refs_out, pairs, counts, workspace) -> the four outputs
PyObject* cache_compact(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    Arg table, refs, out[4], ws;
    if (n != 7 || !take(a[0], table, false) || table.t->dim() != 2 || table.t->numel() == 0 || table.t->scalar_type() != at::kInt || !here(*table.t) || !take(a[1], refs, false) ||
        refs.t->dim() != 1 || refs.t->numel() == 0 || refs.t->scalar_type() != at::kInt || !here(*refs.t)) return none();
    const int64_t B = table.t->size(0), max_pages = table.t->size(1), n_pages = refs.t->numel();
    if (!take_like(a[2], out[0], {B, max_pages}, at::kInt, true) || !take_like(a[3], out[1], {n_pages}, at::kInt, true) || !take_like(a[4], out[2], {n_pages / 2, 2}, at::kInt, true) ||
        !take_like(a[5], out[3], {2}, at::kInt, true) || !take(a[6], ws, true) || (ws.t && !here(*ws.t)) || B > INT32_MAX || n_pages > INT32_MAX || max_pages > INT32_MAX) return none();
    const size_t bytes = ws.t ? ws.t->nbytes() : probsparse_cache_compact_workspace_bytes((int32_t)n_pages);
    if (bytes == 0) return none();
    at::Tensor made[4], room;
    int rc;
    {
        const Unlocked unlocked;
        if (!ws.t) { room = at::empty({(int64_t)bytes}, table.t->options().dtype(at::kByte)); ws.ptr = room.data_ptr(); }
        make_ints({{out[0], made[0], B, max_pages}, {out[1], made[1], n_pages, 0}, {out[2], made[2], n_pages / 2, 2}, {out[3], made[3], 2, 0}}, *table.t);
        rc = probsparse_cache_compact(ints(table), ints(refs), (int32_t)B, (int32_t)n_pages, (int32_t)max_pages, ints(out[0]), ints(out[1]), ints(out[2]), ints(out[3]), ws.ptr,
                                      bytes, stream());
    }
    if (rc != PSA_OK) return failed(rc);
    PyObject* all[4];
    for (int i = 0; i < 4; ++i) all[i] = result(a[2 + i], std::move(made[i]));
    return tuple(all, 4);
}

// cache_copy(pools, pairs, counts) -> True
PyObject* cache_copy(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    constexpr Py_ssize_t kMost = 64;
    Arg pairs, counts;
    if (n != 3 || !(PyList_Check(a[0]) || PyTuple_Check(a[0])) || !take(a[1], pairs, false) || pairs.t->dim() != 2 || pairs.t->size(1) != 2 ||
        pairs.t->scalar_type() != at::kInt || !here(*pairs.t) || pairs.t->size(0) > INT32_MAX || !take(a[2], counts, true) ||
        (counts.t && (counts.t->scalar_type() != at::kInt || counts.t->numel() == 0 || !here(*counts.t)))) return none();
    const Py_ssize_t n_pools = PySequence_Fast_GET_SIZE(a[0]);
    if (n_pools < 1 || n_pools > kMost) return none();
    psa_pool_t pools[kMost];
    int64_t n_pages = 0;
    for (Py_ssize_t i = 0; i < n_pools; ++i) {
        PyObject* o = PySequence_Fast_GET_ITEM(a[0], i);
        if (!THPVariable_Check(o)) return none();
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.dim() < 2 || t.numel() == 0 || !here(t) || (i > 0 && t.size(0) != n_pages) || t.size(0) > INT32_MAX) return none();
        n_pages = t.size(0);
        int64_t elements = 1;                          // of a page, which is contiguous
        for (int64_t d = t.dim() - 1; d > 0; --d) {
            if (t.size(d) != 1 && t.stride(d) != elements) return none();
            elements *= t.size(d);
        }
        pools[i] = psa_pool_t{t.data_ptr(), t.stride(0) * (int64_t)t.element_size(), elements * (int64_t)t.element_size()};
    }
    int rc;
    {
        const Unlocked unlocked;
        rc = probsparse_cache_copy(pools, (int32_t)n_pools, (int32_t)n_pages, ints(pairs), ints(counts), (int32_t)pairs.t->size(0), stream());
    }
    if (rc != PSA_OK) return failed(rc);
    Py_RETURN_TRUE;
}

// exceptions of the tensor library (no memory, say) must not cross into the interpreter: the caller's path meets them
// again and reports them
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    try {
        return F(self, a, n);
    } catch (const std::exception&) {
        return none();
    }
}
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction entry() { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<F>)); }

PyMethodDef methods[] = {
    {"attn_fwd", entry<attn_fwd>(), METH_FASTCALL, nullptr},
    {"attn_fwd_opt", entry<attn_fwd_opt>(), METH_FASTCALL, nullptr},
    {"attn_fwd_with_indices", entry<attn_fwd_with_indices>(), METH_FASTCALL, nullptr},
    {"attn_bwd", entry<attn_bwd>(), METH_FASTCALL, nullptr},
    {"mhsa_fwd", entry<mhsa_fwd>(), METH_FASTCALL, nullptr},
    {"layer_norm_fwd", entry<layer_norm_fwd>(), METH_FASTCALL, nullptr},
    {"layer_norm_bwd", entry<layer_norm_bwd>(), METH_FASTCALL, nullptr},
    {"rotary", entry<rotary>(), METH_FASTCALL, nullptr},
    {"packed_fwd", entry<packed_fwd>(), METH_FASTCALL, nullptr},
    {"packed_bwd", entry<packed_bwd>(), METH_FASTCALL, nullptr},
    {"cache_append", entry<cache_append>(), METH_FASTCALL, nullptr},
    {"paged_fwd", entry<paged_fwd>(), METH_FASTCALL, nullptr},
    {"cache_update", entry<cache_update>(), METH_FASTCALL, nullptr},
    {"cache_compact", entry<cache_compact>(), METH_FASTCALL, nullptr},
    {"cache_copy", entry<cache_copy>(), METH_FASTCALL, nullptr},
    {"on_status", on_status, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
