// The per-call part of the operators' Python binding in native code: check the
// tensors of a call, make its results and workspace, and make the C call.  With
// these steps in Python the smallest calls spend three quarters of their time in
// them (one token's norm: 14 us, 6 so).
//
// Each function takes the address of its library function first and the device
// and stream of the call last, and returns the results; an int: the library's
// status, where the call failed; or None without a call when an argument is not
// plainly right (another class, device, layout, type or size): the caller then
// takes the checks in Python, which accept or word the error.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include <math.h>
#include <stdint.h>

#include "ar_ops.h"

namespace {

// Set once the caller has been told that results have no autograd graph; until
// then a tensor that would need one is left to the checks in Python, which tell.
bool graphs_told = false;

// A tensor argument that is plainly right so far, or null.
const at::Tensor *plain(PyObject *o, long device)
{
    // Subclasses may answer for themselves (__torch_function__).
    if (!THPVariable_CheckExact(o) && (PyObject *)Py_TYPE(o) != ParameterClass) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || t.device().index() != device) return nullptr;
    if (!graphs_told && t.requires_grad() && c10::GradMode::is_enabled()) return nullptr;
    return &t;
}

struct Rows {
    const at::Tensor *t = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    void *p() const { return t ? t->data_ptr() : nullptr; }
};

// A matrix with contiguous rows, whose leading dimensions count rows.
bool as_rows(PyObject *o, long device, Rows *r)
{
    const at::Tensor *t = plain(o, device);
    if (!t || t->dim() < 1 || t->numel() == 0) return false;
    r->t = t, r->cols = t->size(-1), r->rows = t->numel() / r->cols;
    if (t->is_contiguous()) r->ld = r->cols;
    else if (t->dim() == 2 && t->stride(1) == 1 && t->stride(0) >= r->cols) r->ld = t->stride(0);
    else return false;
    return true;
}
bool like(PyObject *o, long device, const Rows &m, Rows *r)
{
    return as_rows(o, device, r) && r->rows == m.rows && r->cols == m.cols && r->t->scalar_type() == m.t->scalar_type();
}

int dtype_of(const at::Tensor &t)
{
    return t.scalar_type() == at::kFloat ? AR_FLOAT32 : t.scalar_type() == at::kBFloat16 ? AR_BFLOAT16 : -1;
}

at::Tensor empty_like(const Rows &m) { return at::empty(m.t->sizes(), m.t->options()); }
at::Tensor workspace(size_t bytes, const Rows &m) { return at::empty({(int64_t)bytes}, m.t->options().dtype(at::kByte)); }

PyObject *none()
{
    Py_RETURN_NONE;
}

// Gives a tuple its elements, each a new reference; null if one is missing.
PyObject *tuple(std::initializer_list<PyObject *> items)
{
    PyObject *t = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    bool ok = t != nullptr;
    for (PyObject *o : items) {
        if (!o) ok = false;
        if (t) PyTuple_SET_ITEM(t, i++, o);
        else Py_XDECREF(o);
    }
    if (!ok) Py_CLEAR(t);
    return t;
}
PyObject *wrap_or_none(const at::Tensor &t)
{
    if (t.defined()) return THPVariable_Wrap(t);
    Py_INCREF(Py_None);
    return Py_None;
}

// The parts of a norm call that forward and backward share.
struct Norm {
    ar_norm_desc d{};
    const at::Tensor *post = nullptr, *pre = nullptr, *gate = nullptr;
};
bool norm_params(PyObject *const *a, long device, const Rows &y, Norm *n)
{
    n->d.rows = (size_t)y.rows, n->d.cols = (size_t)y.cols, n->d.ld_y = (size_t)y.ld;
    n->d.dtype = n->d.param_dtype = dtype_of(*y.t);
    n->d.alpha = (float)PyFloat_AsDouble(a[3]), n->d.eps = (float)PyFloat_AsDouble(a[4]), n->d.flags = (int)PyLong_AsLong(a[5]);
    if (PyErr_Occurred() || n->d.dtype < 0) return false;
    const at::Tensor **to[3] = {&n->post, &n->pre, &n->gate};
    bool first = true;
    for (int i = 0; i < 3; ++i) {
        if (a[i] == Py_None) continue;
        const at::Tensor *t = plain(a[i], device);
        if (!t || !t->is_contiguous()) return false;
        const int dt = dtype_of(*t);
        if (dt < 0 || (!first && dt != n->d.param_dtype)) return false;
        n->d.param_dtype = dt, first = false, *to[i] = t;
        if (i < 2 ? t->dim() != 1 : t->dim() != 1 && t->dim() != 2) return false;
        if (t->size(-1) != y.cols) return false;
    }
    if ((n->post && !(n->d.flags & AR_NORM_POST)) || (n->pre && !(n->d.flags & AR_NORM_PRE))) return false;
    if (n->gate) {
        const int64_t k = n->gate->dim() == 1 ? 1 : n->gate->size(0);
        if (k < 1 || y.rows % k) return false;
        n->d.gate_rows = (size_t)k;
    }
    return true;
}
void *ptr(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }
void *ptr(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

// norm(fn, y, residual, post_weight, pre_weight, gate, alpha, eps, flags, device, stream) -> (s, x)
PyObject *norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 11) return PyErr_Format(PyExc_TypeError, "norm takes 11 arguments");
    void *fn = PyLong_AsVoidPtr(a[0]), *stream = PyLong_AsVoidPtr(a[10]);
    const long device = PyLong_AsLong(a[9]);
    if (PyErr_Occurred()) return nullptr;
    try {
        Rows y, r;
        Norm c;
        if (!as_rows(a[1], device, &y) || !like(a[2], device, y, &r) || !norm_params(a + 3, device, y, &c)) {
            PyErr_Clear();
            return none();
        }
        c.d.ld_residual = (size_t)r.ld;
        at::Tensor s = empty_like(y), x;
        if (c.d.flags & AR_NORM_PRE) x = empty_like(y);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = ((decltype(&ar_residual_norm))fn)(&c.d, y.p(), r.p(), ptr(c.post), ptr(c.gate), ptr(c.pre), ptr(s), ptr(x), stream);
        Py_END_ALLOW_THREADS
        return rc ? PyLong_FromLong(rc) : tuple({THPVariable_Wrap(s), wrap_or_none(x)});
    } catch (...) {
        return none();  // the checks in Python raise what there is to raise
    }
}

// norm_backward(fn, workspace_fn, y, s, ds, dx, post_weight, pre_weight, gate, alpha, eps, flags, param_grads, device, stream)
//   -> (dy, dresidual, dpost_weight, dpre_weight, dgate)
PyObject *norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 15) return PyErr_Format(PyExc_TypeError, "norm_backward takes 15 arguments");
    void *fn = PyLong_AsVoidPtr(a[0]), *space = PyLong_AsVoidPtr(a[1]), *stream = PyLong_AsVoidPtr(a[14]);
    const long device = PyLong_AsLong(a[13]);
    const int grads = PyObject_IsTrue(a[12]);
    if (PyErr_Occurred()) return nullptr;
    try {
        Rows y, s, ds, dx;
        Norm c;
        if (!as_rows(a[2], device, &y) || !like(a[3], device, y, &s) || !norm_params(a + 6, device, y, &c) ||
            (a[4] != Py_None && !like(a[4], device, y, &ds)) || (a[5] != Py_None && !like(a[5], device, y, &dx)) ||
            (a[5] != Py_None) != ((c.d.flags & AR_NORM_PRE) != 0)) {
            PyErr_Clear();
            return none();
        }
        c.d.ld_s = (size_t)s.ld, c.d.ld_ds = (size_t)ds.ld, c.d.ld_dx = (size_t)dx.ld;
        at::Tensor dy = empty_like(y), dr = empty_like(y), dpost, dpre, dgate, ws;
        if (grads) {
            if (c.post) dpost = at::empty(c.post->sizes(), c.post->options());
            if (c.pre) dpre = at::empty(c.pre->sizes(), c.pre->options());
            if (c.gate) dgate = at::empty(c.gate->sizes(), c.gate->options());
        }
        size_t bytes = 0;
        if (dpost.defined() || dpre.defined() || dgate.defined()) {
            bytes = ((decltype(&ar_residual_norm_backward_workspace))space)(&c.d);
            ws = workspace(bytes, y);
        }
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = ((decltype(&ar_residual_norm_backward))fn)(&c.d, y.p(), s.p(), ds.p(), dx.p(), ptr(c.post), ptr(c.gate), ptr(c.pre), ptr(dy),
                                                        ptr(dr), ptr(dpost), ptr(dgate), ptr(dpre), ptr(ws), bytes, stream);
        Py_END_ALLOW_THREADS
        if (rc) return PyLong_FromLong(rc);
        return tuple({THPVariable_Wrap(dy), THPVariable_Wrap(dr), wrap_or_none(dpost), wrap_or_none(dpre), wrap_or_none(dgate)});
    } catch (...) {
        return none();
    }
}

bool ffn_desc(const Rows &x, const Rows &g, const Rows &u, long act, ar_ffn_desc *d)
{
    if (dtype_of(*x.t) != AR_BFLOAT16 || g.t->scalar_type() != x.t->scalar_type() || g.t->dim() != 2 || u.t->dim() != 2 || g.cols != x.cols)
        return false;
    d->tokens = (size_t)x.rows, d->dim = (size_t)x.cols, d->hidden = (size_t)g.rows, d->dtype = AR_BFLOAT16, d->act = (int)act;
    d->ld_x = (size_t)x.ld, d->ld_w_gate = (size_t)g.ld, d->ld_w_up = (size_t)u.ld;
    return true;
}

// ffn(fn, workspace_for_fn, x, w_gate, w_up, act, save, device, stream) -> (h, saved or None)
PyObject *ffn(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 9) return PyErr_Format(PyExc_TypeError, "ffn takes 9 arguments");
    void *fn = PyLong_AsVoidPtr(a[0]), *space = PyLong_AsVoidPtr(a[1]), *stream = PyLong_AsVoidPtr(a[8]);
    const long device = PyLong_AsLong(a[7]), act = PyLong_AsLong(a[5]);
    const int save = PyObject_IsTrue(a[6]);
    if (PyErr_Occurred()) return nullptr;
    try {
        Rows x, g, u;
        ar_ffn_desc d{};
        if (!as_rows(a[2], device, &x) || !as_rows(a[3], device, &g) || !like(a[4], device, g, &u) || !ffn_desc(x, g, u, act, &d)) return none();
        auto shape = x.t->sizes().vec();
        shape.back() = g.rows;
        at::Tensor h = at::empty(shape, x.t->options()), saved, ws;
        if (save) saved = at::empty({2, x.rows, g.rows}, x.t->options().dtype(at::kFloat));
        // only operands that have to be laid out, and a dim in several runs, need a workspace
        const size_t bytes = ((decltype(&ar_gated_ffn_workspace_for))space)(&d, x.p(), g.p(), u.p());
        if (bytes) ws = workspace(bytes, x);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = ((decltype(&ar_gated_ffn))fn)(&d, x.p(), g.p(), u.p(), ptr(h), (float *)ptr(saved), ptr(ws), bytes, stream);
        Py_END_ALLOW_THREADS
        return rc ? PyLong_FromLong(rc) : tuple({THPVariable_Wrap(h), wrap_or_none(saved)});
    } catch (...) {
        return none();
    }
}

// ffn_backward(fn, workspace_fn, dh, x, w_gate, w_up, saved, act, need_dx, need_dw, device, stream) -> (dx, dw_gate, dw_up)
PyObject *ffn_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 12) return PyErr_Format(PyExc_TypeError, "ffn_backward takes 12 arguments");
    void *fn = PyLong_AsVoidPtr(a[0]), *space = PyLong_AsVoidPtr(a[1]), *stream = PyLong_AsVoidPtr(a[11]);
    const long device = PyLong_AsLong(a[10]), act = PyLong_AsLong(a[7]);
    const int need_dx = PyObject_IsTrue(a[8]), need_dw = PyObject_IsTrue(a[9]);
    if (PyErr_Occurred()) return nullptr;
    try {
        Rows dh, x, g, u;
        ar_ffn_desc d{};
        if (!as_rows(a[2], device, &dh) || !as_rows(a[3], device, &x) || !as_rows(a[4], device, &g) || !like(a[5], device, g, &u) ||
            !ffn_desc(x, g, u, act, &d))
            return none();
        const at::Tensor *saved = plain(a[6], device);
        if (dh.rows != x.rows || dh.cols != g.rows || dh.t->scalar_type() != x.t->scalar_type() || !saved || !saved->is_contiguous() ||
            saved->scalar_type() != at::kFloat || saved->dim() != 3 || saved->size(0) != 2 || saved->size(1) != x.rows || saved->size(2) != g.rows)
            return none();
        d.ld_h = (size_t)dh.ld;
        at::Tensor dx, dg, du;
        if (need_dx) dx = empty_like(x);
        if (need_dw) dg = empty_like(g), du = empty_like(u);
        const size_t bytes = ((decltype(&ar_gated_ffn_backward_workspace))space)(&d);
        at::Tensor ws = workspace(bytes, x);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = ((decltype(&ar_gated_ffn_backward))fn)(&d, dh.p(), x.p(), g.p(), u.p(), (const float *)ptr(saved), ptr(dx), ptr(dg), ptr(du),
                                                    ptr(ws), bytes, stream);
        Py_END_ALLOW_THREADS
        return rc ? PyLong_FromLong(rc) : tuple({wrap_or_none(dx), wrap_or_none(dg), wrap_or_none(du)});
    } catch (...) {
        return none();
    }
}

// One of attention's tensors: (tokens, heads, dim), the elements of a head contiguous,
// nothing overlapping.
struct HeadsOf {
    const at::Tensor *t = nullptr;
    int64_t tokens = 0, heads = 0, dim = 0, ld = 0, hs = 0;
};
bool as_heads(PyObject *o, long device, HeadsOf *r)
{
    const at::Tensor *t = plain(o, device);
    if (!t || t->dim() != 3 || t->numel() == 0 || t->scalar_type() != at::kBFloat16) return false;
    r->t = t, r->tokens = t->size(0), r->heads = t->size(1), r->dim = t->size(2), r->ld = t->stride(0), r->hs = t->stride(1);
    if (r->dim > 1 && t->stride(2) != 1) return false;
    if (r->heads == 1) r->hs = r->dim;
    if (r->tokens == 1) r->ld = (r->heads - 1) * r->hs + r->dim;
    return r->hs >= r->dim && r->ld >= r->dim && (r->ld >= (r->heads - 1) * r->hs + r->dim || r->hs >= (r->tokens - 1) * r->ld + r->dim);
}
bool as_starts(PyObject *o, long device, const at::Tensor **t)
{
    *t = plain(o, device);
    return *t && (*t)->dim() == 1 && (*t)->is_contiguous() && (*t)->scalar_type() == at::kInt && (*t)->numel() >= 2;
}

// attention(fn, workspace_for_fn, q, k, v, starts_q, starts_k, causal, scale, save, device, stream) -> (o, lse or None)
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 12) return PyErr_Format(PyExc_TypeError, "attention takes 12 arguments");
    void *fn = PyLong_AsVoidPtr(a[0]), *space = PyLong_AsVoidPtr(a[1]), *stream = PyLong_AsVoidPtr(a[11]);
    const long device = PyLong_AsLong(a[10]);
    const int causal = PyObject_IsTrue(a[7]), save = PyObject_IsTrue(a[9]);
    if (PyErr_Occurred()) return nullptr;
    try {
        HeadsOf q, k, v;
        if (!as_heads(a[2], device, &q) || !as_heads(a[3], device, &k) || !as_heads(a[4], device, &v)) return none();
        if (k.tokens != v.tokens || k.heads != v.heads || k.dim != q.dim || v.dim != q.dim || q.heads % k.heads) return none();
        ar_attention_desc d{};
        d.sequences = 1;
        const at::Tensor *sq = nullptr, *sk = nullptr;
        if (a[5] != Py_None) {
            if (!as_starts(a[5], device, &sq) || (a[6] != Py_None && !as_starts(a[6], device, &sk))) return none();
            if (!sk) sk = sq;
            if (sk->numel() != sq->numel()) return none();
            d.sequences = (size_t)sq->numel() - 1;
        } else if (a[6] != Py_None) {
            return none();
        }
        d.tokens_q = (size_t)q.tokens, d.tokens_k = (size_t)k.tokens, d.heads = (size_t)q.heads, d.kv_heads = (size_t)k.heads;
        d.dim = (size_t)q.dim, d.dtype = AR_BFLOAT16, d.flags = (causal ? AR_ATTN_CAUSAL : 0) | AR_ATTN_CLEAR;
        const double scale = a[8] == Py_None ? 1.0 / sqrt((double)q.dim) : PyFloat_AsDouble(a[8]);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            return none();
        }
        d.scale = (float)scale;
        d.ld_q = (size_t)q.ld, d.hs_q = (size_t)q.hs, d.ld_k = (size_t)k.ld, d.hs_k = (size_t)k.hs, d.ld_v = (size_t)v.ld, d.hs_v = (size_t)v.hs;
        at::Tensor o = at::empty(q.t->sizes(), q.t->options()), lse, ws;
        if (save) lse = at::empty({q.heads, q.tokens}, q.t->options().dtype(at::kFloat));
        const size_t bytes = ((decltype(&ar_attention_workspace_for))space)(&d, q.t->data_ptr(), k.t->data_ptr(), v.t->data_ptr());
        if (bytes) ws = at::empty({(int64_t)bytes}, q.t->options().dtype(at::kByte));
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = ((decltype(&ar_attention))fn)(&d, q.t->data_ptr(), k.t->data_ptr(), v.t->data_ptr(), (const int32_t *)ptr(sq), (const int32_t *)ptr(sk),
                                           ptr(o), (float *)ptr(lse), ptr(ws), bytes, stream);
        Py_END_ALLOW_THREADS
        return rc ? PyLong_FromLong(rc) : tuple({THPVariable_Wrap(o), wrap_or_none(lse)});
    } catch (...) {
        return none();
    }
}

// vocab_loss(fn, workspace_fn, x, weight, target, device, stream) -> (loss, lse)
PyObject *vocab_loss(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 7) return PyErr_Format(PyExc_TypeError, "vocab_loss takes 7 arguments");
    void *fn = PyLong_AsVoidPtr(a[0]), *space = PyLong_AsVoidPtr(a[1]), *stream = PyLong_AsVoidPtr(a[6]);
    const long device = PyLong_AsLong(a[5]);
    if (PyErr_Occurred()) return nullptr;
    try {
        Rows x, w;
        const at::Tensor *t = plain(a[4], device);
        if (!as_rows(a[2], device, &x) || !as_rows(a[3], device, &w) || w.t->dim() != 2 || w.cols != x.cols || dtype_of(*x.t) != AR_BFLOAT16 ||
            w.t->scalar_type() != x.t->scalar_type())
            return none();
        if (!t || !t->is_contiguous() || t->numel() != x.rows || (t->scalar_type() != at::kLong && t->scalar_type() != at::kInt)) return none();
        ar_vocab_desc d{};
        d.tokens = (size_t)x.rows, d.dim = (size_t)x.cols, d.rows = d.classes = (size_t)w.rows, d.dtype = AR_BFLOAT16;
        d.target_bytes = t->scalar_type() == at::kLong ? 8 : 4, d.ld_x = (size_t)x.ld, d.ld_w = (size_t)w.ld;
        at::Tensor loss = at::empty(t->sizes(), t->options().dtype(at::kFloat)), lse = at::empty(t->sizes(), loss.options());
        const size_t bytes = ((decltype(&ar_vocab_loss_workspace))space)(&d, x.p(), w.p());
        at::Tensor ws = workspace(bytes, x);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = ((decltype(&ar_vocab_loss))fn)(&d, x.p(), w.p(), ptr(t), (float *)ptr(loss), (float *)ptr(lse), ptr(ws), bytes, stream);
        Py_END_ALLOW_THREADS
        return rc ? PyLong_FromLong(rc) : tuple({THPVariable_Wrap(loss), THPVariable_Wrap(lse)});
    } catch (...) {
        return none();
    }
}

PyObject *tell_graphs(PyObject *, PyObject *told)
{
    const int is = PyObject_IsTrue(told);
    if (is < 0) return nullptr;
    graphs_told = is != 0;
    return none();
}

PyMethodDef methods[] = {
    {"norm", (PyCFunction)(void (*)(void))norm, METH_FASTCALL, "ar_residual_norm on tensors."},
    {"norm_backward", (PyCFunction)(void (*)(void))norm_backward, METH_FASTCALL, "ar_residual_norm_backward on tensors."},
    {"ffn", (PyCFunction)(void (*)(void))ffn, METH_FASTCALL, "ar_gated_ffn on tensors."},
    {"ffn_backward", (PyCFunction)(void (*)(void))ffn_backward, METH_FASTCALL, "ar_gated_ffn_backward on tensors."},
    {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, "ar_attention on tensors."},
    {"vocab_loss", (PyCFunction)(void (*)(void))vocab_loss, METH_FASTCALL, "ar_vocab_loss on tensors."},
    {"tell_graphs", tell_graphs, METH_O, "Whether the caller knows that results have no autograd graph."},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// torch_version: the torch whose headers this was compiled with.  The binding
// uses the module with that one alone.
PyMODINIT_FUNC PyInit__ops_args(void)
{
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", AR_TORCH_VERSION) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
