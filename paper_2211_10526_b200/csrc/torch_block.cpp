// From torch tensors to the C ABI for the operators around the attention core and its gradients: checks, strides, outputs,
// workspace, device and stream.  No arithmetic here.
#include "torch_call.h"

#include <array>

namespace torch_call {
namespace {

decltype(&castling_attn_rotate) g_rotate = nullptr;
decltype(&castling_attn_norm_forward) g_norm_forward = nullptr;
decltype(&castling_attn_norm_backward) g_norm_backward = nullptr;
decltype(&castling_attn_norm_workspace_bytes) g_norm_bytes = nullptr;
decltype(&castling_attn_backward) g_backward = nullptr;
decltype(&castling_attn_backward_workspace_bytes) g_backward_bytes = nullptr;

// An optional tensor argument; *ok becomes false (and a Python error is set) where it is neither a tensor nor None.
const at::Tensor* optional(PyObject* o, const char* name, bool* ok) {
    if (o == Py_None) return nullptr;
    const at::Tensor* t = tensor(o, name);
    if (!t) *ok = false;
    return t;
}

bool type_error(const char* what) { PyErr_SetString(PyExc_TypeError, what); return false; }
bool bad_value(const char* what) { PyErr_SetString(PyExc_ValueError, what); return false; }

// The element type all tensors share, on one CUDA device.
bool same_kind(const at::Tensor& first, std::initializer_list<const at::Tensor*> rest) {
    if (!first.is_cuda()) return bad_value("expected cuda tensors");
    const at::ScalarType dt = first.scalar_type();
    for (const at::Tensor* t : rest) {
        if (!t) continue;
        if (!t->is_cuda()) return bad_value("expected cuda tensors");
        if (t->device() != first.device()) return bad_value("all tensors must be on one device");
        if (t->scalar_type() != dt) return type_error("all tensors must share one dtype");
    }
    if (dt != at::kFloat && dt != at::kBFloat16) return type_error("unsupported dtype: float32 or bfloat16 expected");
    return true;
}
castling_dtype_t code_of(const at::Tensor& t) { return t.scalar_type() == at::kFloat ? CASTLING_F32 : CASTLING_BF16; }

bool fits_int(int64_t v) { return v >= 0 && v <= INT32_MAX; }

// Strides of a [B, H, N, d] tensor; a dimension of one element gets those of a contiguous tensor, whatever torch says of it.
castling_attn_strides_t strides_of(const at::Tensor* t) {
    if (!t) return {0, 0, 0};
    const int64_t B = t->size(0), H = t->size(1), N = t->size(2), d = t->size(3);
    return {B > 1 ? t->stride(0) : H * N * d, H > 1 ? t->stride(1) : N * d, N > 1 ? t->stride(2) : d};
}
bool heads(const at::Tensor* t, const char* what) {
    return !t || (t->dim() == 4 && (t->stride(3) == 1 || t->size(3) == 1)) || bad_value(what);
}

// Leaves Python while the library runs, with the tensors' device current.
template <typename Call> int without_gil(const at::Tensor& on, Call call) {
    const c10::cuda::CUDAGuard guard(on.device());
    void* stream = c10::cuda::getCurrentCUDAStream(on.get_device()).stream();
    PyThreadState* gil = PyEval_SaveThread();
    const int rc = call(stream);
    PyEval_RestoreThread(gil);
    return rc;
}

PyObject* wrap(at::Tensor t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(t));
}
template <size_t n> PyObject* pack(std::array<PyObject*, n> items) {
    PyObject* r = PyTuple_New(n);
    bool ok = r != nullptr;
    for (PyObject* o : items) ok = ok && o;
    if (!ok) {
        for (PyObject* o : items) Py_XDECREF(o);
        Py_XDECREF(r);
        return nullptr;
    }
    for (size_t i = 0; i < n; ++i) PyTuple_SET_ITEM(r, i, items[i]);
    return r;
}

// Up to three integers of a tuple; their number, or -1.
int small_tuple(PyObject* o, const char* name, int (&to)[3]) {
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) < 1 || PyTuple_GET_SIZE(o) > 3) {
        PyErr_Format(PyExc_ValueError, "%s: one to three sizes expected", name);
        return -1;
    }
    const int n = (int)PyTuple_GET_SIZE(o);
    for (int i = 0; i < n; ++i) {
        const long v = PyLong_AsLong(PyTuple_GET_ITEM(o, i));
        if (v == -1 && PyErr_Occurred()) return -1;
        if (v < 0 || v > INT32_MAX) { PyErr_Format(PyExc_ValueError, "%s: size out of range", name); return -1; }
        to[i] = (int)v;
    }
    return n;
}

const void* at_of(const at::Tensor* t) { return t ? t->const_data_ptr() : nullptr; }
void* out_of(at::Tensor& t) { return t.defined() ? t.mutable_data_ptr() : nullptr; }

// [B, N, D] or [N, D]
struct Stream { int64_t B, N, D; };
bool stream_of(const at::Tensor& x, Stream* s) {
    if (x.dim() != 2 && x.dim() != 3) return bad_value("x: [B, N, D] or [N, D] expected");
    const int o = (int)x.dim() - 2;
    *s = {o ? x.size(0) : 1, x.size(o), x.size(o + 1)};
    if (s->B < 1 || s->N < 1 || s->D < 1) return bad_value("empty tensors are not taken");
    return (fits_int(s->B) && fits_int(s->N) && fits_int(s->D)) || bad_value("size out of range");
}
bool rows_of(const at::Tensor* t, const at::Tensor& x, const Stream& s, const char* what, castling_attn_rows_t* to) {
    *to = {s.N * s.D, s.D};
    if (!t) return true;
    if (t->sizes() != x.sizes()) return bad_value(what);
    const int o = (int)t->dim() - 2;
    if (s.D > 1 && t->stride(o + 1) != 1) return bad_value("the D features of a token must be contiguous (stride 1 in the last dimension)");
    if (s.N > 1) to->token = t->stride(o);
    if (s.B > 1) to->batch = t->stride(0);
    return true;
}

struct NormCall {
    castling_attn_norm_t cfg = {};
    castling_attn_norm_params_t params = {};
    const at::Tensor *x, *branch, *param[6];
    Stream s;
    castling_attn_rows_t x_rows, branch_rows;
};
// a: kind, post, eps, residual_scale, x, branch, weight, bias, post_weight, post_bias, scale, gate
bool norm_call(PyObject* const* a, NormCall* c) {
    c->cfg.norm = (int)PyLong_AsLong(a[0]);
    c->cfg.norm_post = (int)PyLong_AsLong(a[1]);
    c->cfg.eps = PyFloat_AsDouble(a[2]);
    c->cfg.residual_scale = PyFloat_AsDouble(a[3]);
    if (PyErr_Occurred()) return false;
    bool ok = true;
    c->x = tensor(a[4], "x");
    if (!c->x) return false;
    c->branch = optional(a[5], "branch", &ok);
    static const char* names[6] = {"weight", "bias", "post_weight", "post_bias", "scale", "gate"};
    for (int i = 0; i < 6; ++i) c->param[i] = optional(a[6 + i], names[i], &ok);
    if (!ok) return false;
    if (!stream_of(*c->x, &c->s)) return false;
    if (!same_kind(*c->x, {c->branch, c->param[0], c->param[1], c->param[2], c->param[3], c->param[4], c->param[5]})) return false;
    if (!rows_of(c->x, *c->x, c->s, "x", &c->x_rows) || !rows_of(c->branch, *c->x, c->s, "branch must have the shape of x", &c->branch_rows)) return false;
    for (int i = 0; i < 6; ++i) {
        const at::Tensor* p = c->param[i];
        if (!p) continue;
        if (i < 5 ? (p->dim() != 1 || p->size(0) != c->s.D) : (p->dim() != 2 || p->size(0) != c->s.B || p->size(1) != c->s.D))
            return bad_value("parameters: [D] expected, gate: [B, D]");
        if (!p->is_contiguous()) return bad_value("parameters must be contiguous");
    }
    c->cfg.B = (int)c->s.B; c->cfg.N = (int)c->s.N; c->cfg.D = (int)c->s.D;
    c->cfg.dtype = code_of(*c->x);
    c->params = {at_of(c->param[0]), at_of(c->param[1]), at_of(c->param[2]), at_of(c->param[3]), at_of(c->param[4]), at_of(c->param[5])};
    return true;
}

}  // namespace

PyObject* bind_block(PyObject*, PyObject* args) {
    unsigned long long f[6];
    if (!PyArg_ParseTuple(args, "KKKKKK", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5])) return nullptr;
    g_rotate = reinterpret_cast<decltype(g_rotate)>(f[0]);
    g_norm_forward = reinterpret_cast<decltype(g_norm_forward)>(f[1]);
    g_norm_backward = reinterpret_cast<decltype(g_norm_backward)>(f[2]);
    g_norm_bytes = reinterpret_cast<decltype(g_norm_bytes)>(f[3]);
    g_backward = reinterpret_cast<decltype(g_backward)>(f[4]);
    g_backward_bytes = reinterpret_cast<decltype(g_backward_bytes)>(f[5]);
    Py_RETURN_NONE;
}

// rotate(axis_dims, base, interleaved, inverse, q, k | None, grid | None, prefix_tokens, positions | None, in_place)
// -> (q, k | None), or the (non-zero) return code of the C call as an int
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 10 || !g_rotate) { PyErr_SetString(PyExc_TypeError, "rotate: 10 arguments expected, after bind_block()"); return nullptr; }
    castling_attn_rotary_t cfg = {};
    cfg.axes = small_tuple(a[0], "axis_dims", cfg.axis_dims);
    if (cfg.axes < 0) return nullptr;
    cfg.base = PyFloat_AsDouble(a[1]);
    cfg.interleaved = PyObject_IsTrue(a[2]);
    cfg.inverse = PyObject_IsTrue(a[3]);
    const long prefix = PyLong_AsLong(a[7]);
    const bool in_place = PyObject_IsTrue(a[9]) == 1;
    if (PyErr_Occurred()) return nullptr;
    bool ok = true;
    const at::Tensor* q = tensor(a[4], "q");
    if (!q) return nullptr;
    const at::Tensor *k = optional(a[5], "k", &ok), *positions = optional(a[8], "positions", &ok);
    if (!ok || !same_kind(*q, {k})) return nullptr;
    if (!heads(q, "q: [B, H, N, d] with stride 1 in the last dimension expected") || !heads(k, "k: [B, H, N, d] with stride 1 in the last dimension expected")) return nullptr;
    const int64_t B = q->size(0), N = q->size(2), d = q->size(3);
    if (k && (k->size(0) != B || k->size(2) != N || k->size(3) != d)) return value_error("q and k may differ in their numbers of heads only");
    if (!fits_int(B) || !fits_int(q->size(1)) || !fits_int(N) || !fits_int(d) || (k && !fits_int(k->size(1))) || prefix < 0 || prefix > INT32_MAX) return value_error("size out of range");
    if (q->numel() == 0 || (k && k->numel() == 0)) return value_error("empty tensors are not taken");
    cfg.B = (int)B; cfg.H = (int)q->size(1); cfg.H_k = k ? (int)k->size(1) : 0; cfg.N = (int)N; cfg.d = (int)d;
    cfg.dtype = code_of(*q);
    if ((a[6] == Py_None) == (positions == nullptr)) return value_error("exactly one of grid and positions is needed");
    if (positions) {
        if (prefix) return value_error("prefix_tokens goes with grid; given positions are every token's");
        const at::ScalarType pt = positions->scalar_type();
        cfg.positions_type = pt == at::kInt ? CASTLING_POSITIONS_INT32 : pt == at::kLong ? CASTLING_POSITIONS_INT64
                           : pt == at::kFloat ? CASTLING_POSITIONS_FLOAT32 : CASTLING_POSITIONS_GRID;
        if (cfg.positions_type == CASTLING_POSITIONS_GRID) { type_error("positions: int32, int64 or float32 expected"); return nullptr; }
        if (positions->device() != q->device()) return value_error("all tensors must be on one device");
        const int64_t pd = positions->dim();
        if ((pd != 2 && pd != 3) || positions->size(pd - 1) != cfg.axes || positions->size(pd - 2) != N || (pd == 3 && positions->size(0) != B && positions->size(0) != 1))
            return value_error("positions: [B, N, axes], [1, N, axes] or [N, axes] expected");
        if (!positions->is_contiguous()) return value_error("positions must be contiguous");
        cfg.positions_batched = pd == 3 && positions->size(0) == B;
    } else {
        const int axes = small_tuple(a[6], "grid", cfg.grid);
        if (axes < 0) return nullptr;
        if (axes != cfg.axes) return value_error("grid must have a size for every axis");
        cfg.prefix_tokens = (int)prefix;
        int64_t tokens = prefix;
        {
            int64_t m = 1;
            for (int i = 0; i < axes; ++i) { m *= cfg.grid[i]; if (m > INT32_MAX) return value_error("size out of range"); }
            tokens += m;
        }
        if (tokens != N) return value_error("N != prefix_tokens + the grid's tokens");
    }
    at::Tensor qo, ko;
    if (!in_place) {
        qo = at::empty_like(*q);
        if (k) ko = at::empty_like(*k);
        if ((qo.stride(3) != 1 && d > 1) || (k && ko.stride(3) != 1 && d > 1)) return value_error("the d elements of a token must be contiguous (stride 1 in the last dimension)");
    }
    const at::Tensor *to_q = in_place ? q : &qo, *to_k = in_place ? k : (k ? &ko : nullptr);
    cfg.q = strides_of(q); cfg.k = strides_of(k); cfg.q_out = strides_of(to_q); cfg.k_out = strides_of(to_k);
    const void *qp = q->const_data_ptr(), *kp = at_of(k), *pp = at_of(positions);
    void *qop = to_q->mutable_data_ptr(), *kop = to_k ? to_k->mutable_data_ptr() : nullptr;
    const int rc = without_gil(*q, [&](void* stream) { return g_rotate(&cfg, qp, kp, qop, kop, pp, stream); });
    if (rc != CASTLING_OK) return PyLong_FromLong(rc);
    if (in_place) {
        written(*q);
        if (k) written(*k);
        Py_INCREF(a[4]); Py_INCREF(a[5]);
        return pack<2>({a[4], a[5]});
    }
    return pack<2>({wrap(std::move(qo)), wrap(std::move(ko))});
    END_HANDLE_TH_ERRORS
}

// norm_forward(kind, post, eps, residual_scale, x, branch | None, weight, bias, post_weight, post_bias, scale, gate (each | None))
// -> (h, y | None), or a return code
PyObject* norm_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12 || !g_norm_forward) { PyErr_SetString(PyExc_TypeError, "norm_forward: 12 arguments expected, after bind_block()"); return nullptr; }
    NormCall c;
    if (!norm_call(a, &c)) return nullptr;
    const bool is_x = !c.branch && c.cfg.residual_scale == 1.0;   // h is x
    at::Tensor h, y;
    if (!is_x) h = at::empty(c.x->sizes(), c.x->options());
    if (c.cfg.norm != CASTLING_NORM_NONE) y = at::empty(c.x->sizes(), c.x->options());
    const castling_attn_rows_t dense = {c.s.N * c.s.D, c.s.D};
    const void *xp = c.x->const_data_ptr(), *bp = at_of(c.branch);
    void *hp = out_of(h), *yp = out_of(y);
    const int rc = without_gil(*c.x, [&](void* stream) { return g_norm_forward(&c.cfg, &c.params, xp, c.x_rows, bp, c.branch_rows, hp, dense, yp, dense, stream); });
    if (rc != CASTLING_OK) return PyLong_FromLong(rc);
    if (is_x) { Py_INCREF(a[4]); return pack<2>({a[4], wrap(std::move(y))}); }
    return pack<2>({wrap(std::move(h)), wrap(std::move(y))});
    END_HANDLE_TH_ERRORS
}

// norm_backward(the twelve arguments of norm_forward, grad_y | None, grad_h | None)
// -> gradients of x, branch, weight, bias, post_weight, post_bias, scale, gate (None where the call had none), or a return code
PyObject* norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 14 || !g_norm_backward) { PyErr_SetString(PyExc_TypeError, "norm_backward: 14 arguments expected, after bind_block()"); return nullptr; }
    NormCall c;
    if (!norm_call(a, &c)) return nullptr;
    bool ok = true;
    const at::Tensor *dy = optional(a[12], "grad_y", &ok), *dh = optional(a[13], "grad_h", &ok);
    if (!ok || !same_kind(*c.x, {dy, dh})) return nullptr;
    if (!dy && !dh) return value_error("one of grad_y and grad_h is needed");
    castling_attn_rows_t dy_rows, dh_rows;
    if (!rows_of(dy, *c.x, c.s, "grad_y must have the shape of x", &dy_rows) || !rows_of(dh, *c.x, c.s, "grad_h must have the shape of x", &dh_rows)) return nullptr;
    const castling_attn_rows_t dense = {c.s.N * c.s.D, c.s.D};
    at::Tensor dx = at::empty(c.x->sizes(), c.x->options()), db, dp[6];
    if (c.branch) db = at::empty(c.x->sizes(), c.x->options());
    for (int i = 0; i < 6; ++i)
        if (c.param[i]) dp[i] = at::empty(c.param[i]->sizes(), c.x->options());
    const c10::cuda::CUDAGuard guard(c.x->device());   // the workspace's size goes by the device
    const castling_attn_norm_grads_t grads = {out_of(dp[0]), out_of(dp[1]), out_of(dp[2]), out_of(dp[3]), out_of(dp[4]), out_of(dp[5])};
    const size_t bytes = g_norm_bytes(&c.cfg);
    at::Tensor ws = at::empty({(int64_t)(bytes ? bytes : 16)}, c.x->options().dtype(at::kByte));
    const void *xp = c.x->const_data_ptr(), *bp = at_of(c.branch), *dyp = at_of(dy), *dhp = at_of(dh);
    void *dxp = out_of(dx), *dbp = out_of(db), *wp = out_of(ws);
    const int rc = without_gil(*c.x, [&](void* stream) {
        return g_norm_backward(&c.cfg, &c.params, xp, c.x_rows, bp, c.branch_rows, dhp, dh_rows, dyp, dy_rows, dxp, dense, dbp, dense, &grads, wp, bytes, stream);
    });
    if (rc != CASTLING_OK) return PyLong_FromLong(rc);
    return pack<8>({wrap(std::move(dx)), wrap(std::move(db)), wrap(std::move(dp[0])), wrap(std::move(dp[1])), wrap(std::move(dp[2])),
                    wrap(std::move(dp[3])), wrap(std::move(dp[4])), wrap(std::move(dp[5]))});
    END_HANDLE_TH_ERRORS
}

// attention_backward(handle, ksize, prefix_tokens, grad_out, q, k, v, dw_weight, gridH, gridW, bias, (grad_q, grad_k, grad_v) | None)
// -> gradients of q, k, v, dw_weight and (bias) dw_bias, or a return code
PyObject* attention_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12 || !g_backward) { PyErr_SetString(PyExc_TypeError, "attention_backward: 12 arguments expected, after bind_block()"); return nullptr; }
    castling_attn_t* handle = static_cast<castling_attn_t*>(a[0] == Py_None ? nullptr : PyLong_AsVoidPtr(a[0]));
    const long ks = PyLong_AsLong(a[1]), prefix = PyLong_AsLong(a[2]), gridH = PyLong_AsLong(a[8]), gridW = PyLong_AsLong(a[9]);
    const bool bias = PyObject_IsTrue(a[10]) == 1;
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor *g = tensor(a[3], "grad_out"), *q = g ? tensor(a[4], "q") : nullptr, *k = q ? tensor(a[5], "k") : nullptr,
                     *v = k ? tensor(a[6], "v") : nullptr, *w = v ? tensor(a[7], "dw_weight") : nullptr;
    if (!w) return nullptr;
    at::Tensor made[3];
    const at::Tensor* out[3] = {&made[0], &made[1], &made[2]};
    if (q->dim() != 4 || k->sizes() != q->sizes() || v->sizes() != q->sizes() || g->sizes() != q->sizes())
        return value_error("grad_out, q, k, v must share one [B, H, N, d] shape");
    if (a[11] == Py_None) {
        const at::Tensor* like[3] = {q, k, v};
        for (int i = 0; i < 3; ++i) made[i] = at::empty_like(*like[i]);
    } else {
        if (!PyTuple_Check(a[11]) || PyTuple_GET_SIZE(a[11]) != 3) return value_error("out: (grad_q, grad_k, grad_v) expected");
        for (int i = 0; i < 3; ++i)
            if (!(out[i] = tensor(PyTuple_GET_ITEM(a[11], i), "out"))) return nullptr;
    }
    if (!same_kind(*q, {k, v, w, g, out[0], out[1], out[2]})) return nullptr;
    const int64_t B = q->size(0), H = q->size(1), N = q->size(2), d = q->size(3);
    for (const at::Tensor* t : {q, k, v, g, out[0], out[1], out[2]}) {
        if (t->sizes() != q->sizes()) return value_error("out: gradients must have the shapes of q, k and v");
        if (!heads(t, "the d elements of a token must be contiguous (stride 1 in the last dimension)")) return nullptr;
    }
    if (gridH < 0 || gridW < 0 || gridH > INT32_MAX || gridW > INT32_MAX || !fits_int(B) || !fits_int(H) || !fits_int(d)) return value_error("size out of range");
    if (N != prefix + (int64_t)gridH * gridW) return value_error("N != prefix_tokens + gridH * gridW");
    if (w->dim() != 3 || w->size(0) != H * d || w->size(1) != ks || w->size(2) != ks) return value_error("dw_weight must be [H*d, ksize, ksize]");
    if (!w->is_contiguous()) return value_error("dw_weight must be contiguous");
    const c10::cuda::CUDAGuard guard(q->device());     // the workspace's size goes by the device
    at::Tensor dw = at::empty_like(*w), db;
    if (bias) db = at::empty({H * d}, w->options());
    const castling_attn_grad_layout_t layout = {strides_of(q), strides_of(k), strides_of(v), strides_of(g), strides_of(out[0]), strides_of(out[1]), strides_of(out[2])};
    const size_t bytes = g_backward_bytes(handle, (int)B, (int)H, (int)gridH, (int)gridW, (int)d, code_of(*q));
    at::Tensor ws = at::empty({(int64_t)(bytes ? bytes : 16)}, q->options().dtype(at::kByte));
    const void *qp = q->const_data_ptr(), *kp = k->const_data_ptr(), *vp = v->const_data_ptr(), *wp = w->const_data_ptr(), *gp = g->const_data_ptr();
    void *o[3], *dwp = out_of(dw), *dbp = out_of(db), *wsp = out_of(ws);
    for (int i = 0; i < 3; ++i) o[i] = out[i]->mutable_data_ptr();
    const int rc = without_gil(*q, [&](void* stream) {
        return g_backward(handle, qp, kp, vp, wp, gp, o[0], o[1], o[2], dwp, dbp, (int)B, (int)H, (int)gridH, (int)gridW, (int)d, code_of(*q), &layout, wsp, bytes, stream);
    });
    if (rc != CASTLING_OK) return PyLong_FromLong(rc);
    PyObject* items[3];
    for (int i = 0; i < 3; ++i) {
        if (a[11] == Py_None) { items[i] = wrap(std::move(made[i])); continue; }
        written(*out[i]);
        items[i] = PyTuple_GET_ITEM(a[11], i);
        Py_INCREF(items[i]);
    }
    return pack<5>({items[0], items[1], items[2], wrap(std::move(dw)), wrap(std::move(db))});
    END_HANDLE_TH_ERRORS
}

}  // namespace torch_call
