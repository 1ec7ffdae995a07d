// The calls that every layer of a model makes, for Python: hdt_build_layout, hdt_attn_fwd and hdt_attn_bwd, the relative-bias
// attention, dropout, norms, embeddings and the feed-forward block, on plain torch tensors.  Checks, output tensors, addresses, stream and the call into libhdt in one piece of native code.
//
// A layer of a thousand positions is bound by the host: its kernels take 8 us each, and a call from the interpreter took 8.1 us
// (forward: two outputs 3.0, the launch 3.0, checks 1.0, ctypes 0.7), 11.5 (backward) and 6.7 (deferred build with its
// destruction); from here 5.2, 6.9 and 4.3.  A build that is waited for and a forward, 1000 positions x 12 heads: 25.4 -> 20.1
// us; with the backward, one head of 512 in fp32: 38.7 -> 28.3.
//
// Nothing is decided here that binding.py does not decide: a call whose arguments are not the plain case (a tensor subclass, a
// wrong shape or type, a tensor that has no storage, a torch function mode, ...) returns None before it has done anything, and
// binding.py's own path takes it, errors included.
#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "hdt.h"

namespace {

decltype(&hdt_build_layout) build_layout_fn;
decltype(&hdt_attn_fwd) fwd_fn;
decltype(&hdt_attn_fwd_ws) fwd_ws_fn;
decltype(&hdt_attn_bwd) bwd_fn;
decltype(&hdt_attn_bwd_workspace_bytes) bwd_bytes_fn;
decltype(&hdt_rel_attn_fwd_workspace_bytes) rel_fwd_bytes_fn;
decltype(&hdt_rel_attn_fwd) rel_fwd_fn;
decltype(&hdt_rel_attn_bwd_workspace_bytes) rel_bwd_bytes_fn;
decltype(&hdt_rel_attn_bwd) rel_bwd_fn;
decltype(&hdt_dropout_add) dropout_fn;
decltype(&hdt_add_norm_fwd) norm_fwd_fn;
decltype(&hdt_add_norm_bwd_workspace_bytes) norm_bwd_bytes_fn;
decltype(&hdt_add_norm_bwd) norm_bwd_fn;
decltype(&hdt_embed_fwd) embed_fwd_fn;
decltype(&hdt_embed_bwd_workspace_bytes) embed_bwd_bytes_fn;
decltype(&hdt_embed_bwd) embed_bwd_fn;
decltype(&hdt_ffn_fwd_workspace_bytes) ffn_fwd_bytes_fn;
decltype(&hdt_ffn_fwd) ffn_fwd_fn;
decltype(&hdt_ffn_bwd_workspace_bytes) ffn_bwd_bytes_fn;
decltype(&hdt_ffn_bwd) ffn_bwd_fn;
decltype(&hdt_gate_norm_fwd) gate_norm_fwd_fn;
decltype(&hdt_gate_norm_bwd_workspace_bytes) gate_norm_bwd_bytes_fn;
decltype(&hdt_gate_norm_bwd) gate_norm_bwd_fn;

// What is not plain is refused by return values: a C++ exception takes 1.5 us, and the calls that the general path takes then
// pay for it (us, no native form - refused by an exception - by return values: forward with a numpy scale 9.0 - 10.8 - 9.1, backward
// 13.3 - 15.0 - 13.2, on another stream with a temporary workspace 19.4 - 21.1 - 19.7, deferred build with a numpy number 6.9 - 8.5 - 7.0).

const at::Tensor *plain(PyObject *o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

bool whole(PyObject *o, int64_t *v)
{
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &over);
    return !over;
}

bool whole32(PyObject *o, int32_t *v)
{
    int64_t w;
    if (!whole(o, &w) || w != (int32_t)w) return false;
    *v = (int32_t)w;
    return true;
}

bool address(PyObject *o, void **p)
{
    *p = nullptr;
    if (o == Py_None) return true;
    if (!PyLong_CheckExact(o)) return false;
    *p = PyLong_AsVoidPtr(o);
    if (*p || !PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}

// a raw stream handle, or None: the current stream of the current device
bool stream_of(PyObject *o, hipStream_t *st)
{
    void *p;
    if (!address(o, &p)) return false;
    *st = o == Py_None ? c10::hip::getCurrentHIPStream().stream() : (hipStream_t)p;
    return true;
}

bool dense(const at::Tensor &t) { return t.is_cuda() && t.is_contiguous(); }

bool has_shape(const at::Tensor &t, int64_t b, int64_t h, int64_t n, int64_t d)
{
    const auto s = t.sizes();
    return s.size() == 4 && s[0] == b && s[1] == h && s[2] == n && s[3] == d;
}

// what the arguments of an attention call have in common
struct Call {
    const at::Tensor *q, *k, *v;
    void *layout;
    int64_t batch, n_pos, n_kv, heads, head_dim;
    float scale;
    hdt_dtype_t dtype;

    // a: (layout, batch, n_pos, n_kv, q, k, v, scale, ...)
    bool plain_case(PyObject *const *a)
    {
        if (!PyFloat_CheckExact(a[7])) return false;
        scale = (float)PyFloat_AS_DOUBLE(a[7]);
        if (!(q = plain(a[4])) || !(k = plain(a[5])) || !(v = plain(a[6]))) return false;
        if (!address(a[0], &layout) || !whole(a[1], &batch) || !whole(a[2], &n_pos) || !whole(a[3], &n_kv)) return false;
        if (q->dim() != 4 || q->scalar_type() != k->scalar_type() || q->scalar_type() != v->scalar_type()) return false;
        heads = q->size(1), head_dim = q->size(3);
        if (heads > INT32_MAX || head_dim > INT32_MAX) return false;
        if (q->scalar_type() == at::kBFloat16) dtype = HDT_BF16;
        else if (q->scalar_type() == at::kFloat) dtype = HDT_F32;
        else return false;
        return like_q(*q) && like_k(*k) && like_k(*v);
    }
    bool like_q(const at::Tensor &t) const { return dense(t) && has_shape(t, batch, heads, n_pos, head_dim); }
    bool like_k(const at::Tensor &t) const { return dense(t) && has_shape(t, batch, heads, n_kv, head_dim); }
};

// the caller's tensor (a plain one, or None), or a new one
at::Tensor given_or(PyObject *o, const at::Tensor &like) { return o == Py_None ? at::empty_like(like) : THPVariable_Unpack(o); }

bool plain_or_none(PyObject *o) { return o == Py_None || THPVariable_CheckExact(o); }

// runs f, which returns NULL without a Python error where the general path has to take the call; None then
template <typename F>
PyObject *guarded(F f)
{
    try {
        PyObject *r = at::impl::torch_function_mode_enabled() ? nullptr : f();
        if (r || PyErr_Occurred()) return r;
    } catch (...) {  // (torch's own exceptions: the general path meets them again and reports them)
        PyErr_Clear();
    }
    Py_RETURN_NONE;
}

PyObject *results(hdt_status_t st, std::initializer_list<at::Tensor> ts)
{
    if (st != HDT_OK) return PyLong_FromLong(st);
    PyObject *out = PyTuple_New((Py_ssize_t)ts.size());
    if (!out) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor &t : ts) {
        PyObject *w = THPVariable_Wrap(t);
        if (!w) {
            Py_DECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, i++, w);
    }
    return out;
}

// (layout, batch, n_pos, n_kv, q, k, v, scale, o, lse, workspace, stream) -> (o, lse), a status, or None
PyObject *attn_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 12) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        Call c;
        hipStream_t st;
        if (!c.plain_case(a) || !plain_or_none(a[8]) || !plain_or_none(a[9]) || !plain_or_none(a[10]) || !stream_of(a[11], &st)) return nullptr;
        const at::Tensor &q = *c.q, &k = *c.k, &v = *c.v;
        const void *pq = q.data_ptr(), *pk = k.data_ptr(), *pv = v.data_ptr();
        at::Tensor o = given_or(a[8], q);
        at::Tensor lse = a[9] == Py_None ? at::empty({c.batch, c.heads, c.n_pos}, q.options().dtype(at::kFloat))
                                        : THPVariable_Unpack(a[9]);
        void *po = o.data_ptr();
        float *pl = (float *)lse.data_ptr(), *pw = nullptr;
        size_t bytes = 0;
        if (a[10] != Py_None) {
            const at::Tensor &w = THPVariable_Unpack(a[10]);
            pw = (float *)w.data_ptr();
            bytes = (size_t)w.numel() * w.element_size();
        }
        hdt_status_t r;
        Py_BEGIN_ALLOW_THREADS
        r = a[10] != Py_None ? fwd_ws_fn((const hdt_layout_t *)c.layout, pq, pk, pv, po, pl, (int32_t)c.heads, (int32_t)c.head_dim,
                                         c.dtype, c.scale, pw, bytes, st)
                             : fwd_fn((const hdt_layout_t *)c.layout, pq, pk, pv, po, pl, (int32_t)c.heads, (int32_t)c.head_dim,
                                      c.dtype, c.scale, st);
        Py_END_ALLOW_THREADS
        return results(r, {o, lse});
    });
}

// (layout, batch, n_pos, n_kv, q, k, v, scale, o, lse, d_o, dq, dk, dv, workspace, stream) -> (dq, dk, dv), a status, or None
PyObject *attn_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 16) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        // a temporary workspace comes from the stream the kernels run on: the current one, that is
        if (a[14] == Py_None && a[15] != Py_None) return nullptr;
        Call c;
        hipStream_t st;
        if (!c.plain_case(a) || !plain(a[8]) || !plain(a[9]) || !plain(a[10]) || !stream_of(a[15], &st)) return nullptr;
        for (int i = 11; i <= 14; i++)
            if (!plain_or_none(a[i])) return nullptr;
        const at::Tensor &q = *c.q, &k = *c.k, &v = *c.v, &o = *plain(a[8]), &lse = *plain(a[9]), &d_o = *plain(a[10]);
        if (o.scalar_type() != q.scalar_type() || d_o.scalar_type() != q.scalar_type() || !c.like_q(o) || !c.like_q(d_o)) return nullptr;
        const void *pq = q.data_ptr(), *pk = k.data_ptr(), *pv = v.data_ptr(), *po = o.data_ptr(), *pd = d_o.data_ptr();
        const float *pl = (const float *)lse.data_ptr();
        at::Tensor dq = given_or(a[11], q), dk = given_or(a[12], k), dv = given_or(a[13], k), w;
        if (a[14] == Py_None) {
            size_t need;
            Py_BEGIN_ALLOW_THREADS  // (waits for the report of a cross-attention build)
            need = bwd_bytes_fn((const hdt_layout_t *)c.layout, (int32_t)c.heads, (int32_t)c.head_dim, c.dtype);
            Py_END_ALLOW_THREADS
            w = at::empty({(int64_t)std::max<size_t>(need, 16)}, q.options().dtype(at::kByte));
        } else {
            w = THPVariable_Unpack(a[14]);
        }
        void *pdq = dq.data_ptr(), *pdk = dk.data_ptr(), *pdv = dv.data_ptr(), *pw = w.data_ptr();
        const size_t bytes = (size_t)w.numel() * w.element_size();
        hdt_status_t r;
        Py_BEGIN_ALLOW_THREADS
        r = bwd_fn((const hdt_layout_t *)c.layout, pq, pk, pv, po, pl, pd, pdq, pdk, pdv, (int32_t)c.heads, (int32_t)c.head_dim,
                   c.dtype, c.scale, pw, bytes, st);
        Py_END_ALLOW_THREADS
        return results(r, {dq, dk, dv});
    });
}

// (level, parent, tile_m, tile_n, force_dense, no_sort, windowed, edges, deferred, capacity, stream)
//   -> (handle, batch, n_pos), a status, or None
PyObject *build_layout(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 11) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        hdt_layout_opts_t opts = {};
        hipStream_t st;
        for (int i = 4; i <= 8; i++)
            if (i != 7 && !PyBool_Check(a[i])) return nullptr;
        if (!plain(a[0]) || !plain(a[1]) || !whole32(a[2], &opts.tile_m) || !whole32(a[3], &opts.tile_n) || !whole32(a[7], &opts.edges) ||
            !whole(a[9], &opts.capacity))
            return nullptr;
        opts.force_dense = a[4] == Py_True;
        opts.no_sort = a[5] == Py_True;
        opts.windowed = a[6] == Py_True;
        opts.deferred = a[8] == Py_True;
        const at::Tensor &level = *plain(a[0]), &parent = *plain(a[1]);
        if (level.scalar_type() != at::kInt || parent.scalar_type() != at::kInt || level.dim() != 2 || !dense(level) || !dense(parent) ||
            level.sizes() != parent.sizes())
            return nullptr;
        const int64_t B = level.size(0), N = level.size(1);
        if (B > INT32_MAX || N > INT32_MAX || !stream_of(a[10], &st)) return nullptr;
        const int32_t *pl = B * N ? (const int32_t *)level.data_ptr() : nullptr, *pp = B * N ? (const int32_t *)parent.data_ptr() : nullptr;
        hdt_layout_t *h = nullptr;
        hdt_status_t r;
        Py_BEGIN_ALLOW_THREADS
        r = build_layout_fn(pl, pp, (int32_t)B, (int32_t)N, &opts, st, &h);
        Py_END_ALLOW_THREADS
        if (r != HDT_OK) return PyLong_FromLong(r);
        return Py_BuildValue("(KLL)", (unsigned long long)(uintptr_t)h, (long long)B, (long long)N);
    });
}

// ---- relative-bias attention, dropout, norm: the same rules ----
bool dtype_of(const at::Tensor &t, hdt_dtype_t *d)
{
    if (t.scalar_type() == at::kBFloat16) *d = HDT_BF16;
    else if (t.scalar_type() == at::kFloat) *d = HDT_F32;
    else return false;
    return true;
}
bool number(PyObject *o, double *v)
{
    if (PyFloat_CheckExact(o)) *v = PyFloat_AS_DOUBLE(o);
    else return false;
    return true;
}
// on the device that is current, whose streams the kernels go to
bool here(const at::Tensor &t, int device) { return t.is_cuda() && t.get_device() == device; }
// None, or a plain tensor here
bool optional(PyObject *o, int device, const at::Tensor **t)
{
    *t = nullptr;
    if (o == Py_None) return true;
    return (*t = plain(o)) && here(**t, device);
}
const void *data(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }
bool like(const at::Tensor &t, const at::Tensor &other)
{
    return t.scalar_type() == other.scalar_type() && t.is_contiguous() && t.sizes() == other.sizes();
}
// rows of consecutive values at any distance; a dimension of one element has the distance it would have in a dense tensor
bool strides_of(const at::Tensor &t, at::IntArrayRef shape, at::ScalarType type, hdt_strides_t *s)
{
    if (t.scalar_type() != type || t.sizes() != shape) return false;
    if (t.is_contiguous()) return true;
    const int64_t d = shape[3], n = shape[2], h = shape[1];
    if (t.stride(3) != 1 || (n > 1 && t.stride(2) < d)) return false;  // (one row expanded over all three would be described as dense)
    s->batch = shape[0] > 1 ? t.stride(0) : h * n * d;
    s->head = h > 1 ? t.stride(1) : n * d;
    s->row = n > 1 ? t.stride(2) : d;
    return true;
}

struct RelCall {
    hdt_rel_attn_t c = {};
    const at::Tensor *q, *k, *v, *bias;
    int device;
    // a: (q, k, v, bias, table, scale, causal, lengths, q_start, ...)
    bool plain_case(PyObject *const *a)
    {
        const at::Tensor *table, *lengths, *start;
        double scale;
        device = c10::hip::current_device();
        if (!(q = plain(a[0])) || !(k = plain(a[1])) || !(v = plain(a[2])) || !(bias = plain(a[3])) || !(table = plain(a[4]))) return false;
        if (!number(a[5], &scale) || !PyBool_Check(a[6]) || !optional(a[7], device, &lengths) || !optional(a[8], device, &start)) return false;
        for (const at::Tensor *t : {q, k, v, bias, table})
            if (!here(*t, device)) return false;
        if (q->dim() != 4 || k->dim() != 4 || bias->dim() != 2 || table->dim() != 1 || !dtype_of(*q, &c.dtype) || !dtype_of(*bias, &c.bias_dtype)) return false;
        const auto qs = q->sizes(), ks = k->sizes();
        if (ks[0] != qs[0] || ks[3] != qs[3] || bias->size(1) != qs[1] || !bias->is_contiguous()) return false;
        if (table->scalar_type() != at::kInt || table->numel() % 2 == 0 || !table->is_contiguous()) return false;
        for (const at::Tensor *t : {lengths, start})
            if (t && (t->scalar_type() != at::kInt || t->dim() != 1 || t->size(0) != qs[0] || !t->is_contiguous())) return false;
        for (int64_t n : {qs[0], qs[1], qs[2], qs[3], ks[1], ks[2], bias->size(0), table->numel()})
            if (n > INT32_MAX) return false;
        c.batch = (int32_t)qs[0], c.heads = (int32_t)qs[1], c.n_q = (int32_t)qs[2], c.head_dim = (int32_t)qs[3];
        c.kv_heads = (int32_t)ks[1], c.n_kv = (int32_t)ks[2], c.causal = a[6] == Py_True;
        c.n_buckets = (int32_t)bias->size(0), c.max_distance = (int32_t)(table->numel() / 2), c.softmax_scale = (float)scale;
        c.d_bias = bias->data_ptr(), c.d_table = (const int32_t *)table->data_ptr();
        c.d_lengths = (const int32_t *)data(lengths), c.d_q_start = (const int32_t *)data(start);
        return strides_of(*q, qs, q->scalar_type(), &c.q) && strides_of(*k, ks, q->scalar_type(), &c.k) && strides_of(*v, ks, q->scalar_type(), &c.v);
    }
    bool is_lse(const at::Tensor &t) const
    {
        return here(t, device) && t.scalar_type() == at::kFloat && t.is_contiguous() && t.dim() == 3 && t.size(0) == c.batch && t.size(1) == c.heads && t.size(2) == c.n_q;
    }
};

// the caller's workspace, or a new one of `need` bytes; its address and size
struct Room {
    at::Tensor t;
    void *at_ = nullptr;
    size_t bytes = 0;
    Room(PyObject *given, size_t need, const at::Tensor &like)
    {
        if (given != Py_None) t = THPVariable_Unpack(given);
        else if (need) t = at::empty({(int64_t)need}, like.options().dtype(at::kByte));
        if (t.defined()) at_ = t.data_ptr(), bytes = (size_t)t.numel() * t.element_size();
    }
};
// None or a plain contiguous tensor here; and a temporary workspace comes from the stream the kernels run on: the current one, that is
bool workspace_ok(PyObject *w, PyObject *stream, int device)
{
    const at::Tensor *t;
    return optional(w, device, &t) && (t ? t->is_contiguous() : stream == Py_None);
}

// (q, k, v, bias, table, scale, causal, lengths, q_start, o, lse, workspace, stream) -> (o, lse), a status, or None
PyObject *rel_attn_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 13) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        RelCall r;
        hipStream_t st;
        const at::Tensor *go, *gl;
        if (!r.plain_case(a) || !optional(a[9], r.device, &go) || !optional(a[10], r.device, &gl) || !workspace_ok(a[11], a[12], r.device) || !stream_of(a[12], &st))
            return nullptr;
        if ((go && !strides_of(*go, r.q->sizes(), r.q->scalar_type(), &r.c.o)) || (gl && !r.is_lse(*gl))) return nullptr;
        at::Tensor o = go ? *go : at::empty(r.q->sizes(), r.q->options());
        at::Tensor lse = gl ? *gl : at::empty({r.c.batch, r.c.heads, r.c.n_q}, r.q->options().dtype(at::kFloat));
        const Room w(a[11], rel_fwd_bytes_fn(&r.c), *r.q);
        const void *pq = r.q->data_ptr(), *pk = r.k->data_ptr(), *pv = r.v->data_ptr();
        void *po = o.data_ptr();
        float *pl = (float *)lse.data_ptr();
        hdt_status_t s;
        Py_BEGIN_ALLOW_THREADS
        s = rel_fwd_fn(&r.c, pq, pk, pv, po, pl, w.at_, w.bytes, st);
        Py_END_ALLOW_THREADS
        return results(s, {o, lse});
    });
}

// (q, k, v, bias, table, scale, causal, lengths, q_start, o, lse, d_o, dq, dk, dv, dbias, workspace, stream) -> (dq, dk, dv, dbias), ...
PyObject *rel_attn_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 18) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        RelCall r;
        hipStream_t st;
        const at::Tensor *o, *lse, *d_o, *g[4];
        if (!r.plain_case(a) || !(o = plain(a[9])) || !(lse = plain(a[10])) || !(d_o = plain(a[11])) || !here(*o, r.device) || !here(*d_o, r.device) ||
            !r.is_lse(*lse) || !workspace_ok(a[16], a[17], r.device) || !stream_of(a[17], &st))
            return nullptr;
        for (int i = 0; i < 4; i++)
            if (!optional(a[12 + i], r.device, &g[i])) return nullptr;
        const auto qs = r.q->sizes(), ks = r.k->sizes();
        const auto type = r.q->scalar_type();
        if (!strides_of(*o, qs, type, &r.c.o) || !strides_of(*d_o, qs, type, &r.c.d_o) || (g[0] && !strides_of(*g[0], qs, type, &r.c.dq)) ||
            (g[1] && !strides_of(*g[1], ks, type, &r.c.dk)) || (g[2] && !strides_of(*g[2], ks, type, &r.c.dv)) || (g[3] && !like(*g[3], *r.bias)))
            return nullptr;
        at::Tensor dq = g[0] ? *g[0] : at::empty(qs, r.q->options()), dk = g[1] ? *g[1] : at::empty(ks, r.q->options());
        at::Tensor dv = g[2] ? *g[2] : at::empty(ks, r.q->options()), db = g[3] ? *g[3] : at::empty(r.bias->sizes(), r.bias->options());
        const Room w(a[16], rel_bwd_bytes_fn(&r.c), *r.q);
        const void *pq = r.q->data_ptr(), *pk = r.k->data_ptr(), *pv = r.v->data_ptr(), *po = o->data_ptr(), *pd = d_o->data_ptr();
        const float *pl = (const float *)lse->data_ptr();
        void *p0 = dq.data_ptr(), *p1 = dk.data_ptr(), *p2 = dv.data_ptr(), *p3 = db.data_ptr();
        hdt_status_t s;
        Py_BEGIN_ALLOW_THREADS
        s = rel_bwd_fn(&r.c, pq, pk, pv, po, pl, pd, p0, p1, p2, p3, w.at_, w.bytes, st);
        Py_END_ALLOW_THREADS
        return results(s, {dq, dk, dv, db});
    });
}

// the generator's state: None only where nothing is dropped
bool is_rng(const at::Tensor *t, double p)
{
    return t ? t->scalar_type() == at::kLong && t->dim() == 1 && t->size(0) == 2 && t->is_contiguous() : !(p > 0);
}
bool site_of(PyObject *o, uint32_t *site)
{
    int64_t v;
    if (!whole(o, &v) || v < 0 || v > (int64_t)UINT32_MAX) return false;
    *site = (uint32_t)v;
    return true;
}

// (y, p, rng, site, x, out, stream) -> out, a status, or None
PyObject *dropout_add(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 7) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        const int device = c10::hip::current_device();
        const at::Tensor *y = plain(a[0]), *rng, *x, *given;
        double p;
        uint32_t site;
        hdt_dtype_t dt;
        hipStream_t st;
        if (!y || !here(*y, device) || !y->is_contiguous() || !dtype_of(*y, &dt) || !number(a[1], &p) || !optional(a[2], device, &rng) || !is_rng(rng, p) ||
            !site_of(a[3], &site) || !optional(a[4], device, &x) || !optional(a[5], device, &given) || !stream_of(a[6], &st))
            return nullptr;
        if ((x && !like(*x, *y)) || (given && !like(*given, *y))) return nullptr;
        at::Tensor out = given ? *given : at::empty(y->sizes(), y->options());
        const void *py = y->data_ptr(), *px = data(x);
        const int64_t *pr = (const int64_t *)data(rng);
        void *po = out.data_ptr();
        const int64_t count = y->numel();
        hdt_status_t s;
        Py_BEGIN_ALLOW_THREADS
        s = dropout_fn(py, px, po, count, p, pr, site, dt, st);
        Py_END_ALLOW_THREADS
        return s != HDT_OK ? PyLong_FromLong(s) : THPVariable_Wrap(out);
    });
}

// what norm calls have in common: rows of x (contiguous, here), a weight like its last dimension, perhaps another vector like the weight
struct NormCall {
    const at::Tensor *x, *weight;
    int64_t rows;
    int32_t width;
    hdt_dtype_t dt, wdt;
    int device;
    bool plain_case(PyObject *px, PyObject *pw)
    {
        device = c10::hip::current_device();
        if (!(x = plain(px)) || !(weight = plain(pw)) || !here(*x, device) || !here(*weight, device) || !dtype_of(*x, &dt) || !dtype_of(*weight, &wdt)) return false;
        if (x->dim() < 1 || !x->is_contiguous() || weight->dim() != 1 || !weight->is_contiguous() || weight->size(0) != x->size(-1) || weight->size(0) > INT32_MAX)
            return false;
        width = (int32_t)weight->size(0);
        if (width == 0) return false;
        rows = x->numel() / width;
        return true;
    }
    bool statistic(const at::Tensor &t) const { return here(t, device) && t.scalar_type() == at::kFloat && t.is_contiguous() && t.numel() == rows; }
};

// (x, weight, bias, eps, y, p, rng, site, h, n, mean, rstd, stream) -> (n, h, mean, rstd), a status, or None; y is a tensor
PyObject *add_norm_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 13) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        NormCall c;
        const at::Tensor *bias, *y, *rng, *g[4];
        double eps, p;
        uint32_t site;
        hipStream_t st;
        if (!c.plain_case(a[0], a[1]) || !optional(a[2], c.device, &bias) || !number(a[3], &eps) || !optional(a[4], c.device, &y) || !y || !number(a[5], &p) ||
            !optional(a[6], c.device, &rng) || !is_rng(rng, p) || !site_of(a[7], &site) || !stream_of(a[12], &st))
            return nullptr;
        for (int i = 0; i < 4; i++)
            if (!optional(a[8 + i], c.device, &g[i])) return nullptr;
        if (!like(*y, *c.x) || (bias && !like(*bias, *c.weight)) || (g[0] && !like(*g[0], *c.x)) || (g[1] && !like(*g[1], *c.x)) ||
            (g[2] && !c.statistic(*g[2])) || (g[3] && !c.statistic(*g[3])))
            return nullptr;
        const auto lead = c.x->sizes().slice(0, c.x->dim() - 1);
        at::Tensor h = g[0] ? *g[0] : at::empty(c.x->sizes(), c.x->options()), out = g[1] ? *g[1] : at::empty(c.x->sizes(), c.x->options());
        at::Tensor mean = g[2] ? *g[2] : at::empty(lead, c.x->options().dtype(at::kFloat)), rstd = g[3] ? *g[3] : at::empty(lead, c.x->options().dtype(at::kFloat));
        const void *px = c.x->data_ptr(), *py = y->data_ptr(), *pw = c.weight->data_ptr(), *pb = data(bias);
        const int64_t *pr = (const int64_t *)data(rng);
        void *ph = h.data_ptr(), *pn = out.data_ptr();
        float *pm = (float *)mean.data_ptr(), *ps = (float *)rstd.data_ptr();
        hdt_status_t s;
        Py_BEGIN_ALLOW_THREADS
        s = norm_fwd_fn(px, py, pw, pb, c.rows, c.width, (float)eps, p, pr, site, ph, pn, pm, ps, c.dt, c.wdt, st);
        Py_END_ALLOW_THREADS
        return results(s, {out, h, mean, rstd});
    });
}

// (dn, h, weight, mean, rstd, dh, p, rng, site, bias, dx, dy, dweight, dbias, workspace, stream) -> (dx, dy, dweight, dbias), a status,
// or None; something is dropped
PyObject *add_norm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 16) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        NormCall c;
        const at::Tensor *dn, *mean, *rstd, *dh, *rng, *g[4];
        double p;
        uint32_t site;
        hipStream_t st;
        if (!c.plain_case(a[1], a[2]) || !(dn = plain(a[0])) || !here(*dn, c.device) || !like(*dn, *c.x) || !(mean = plain(a[3])) || !(rstd = plain(a[4])) ||
            !c.statistic(*mean) || !c.statistic(*rstd) || !optional(a[5], c.device, &dh) || (dh && !like(*dh, *c.x)) || !number(a[6], &p) || !(p >= 1. / 65536) ||
            !optional(a[7], c.device, &rng) || !is_rng(rng, p) || !site_of(a[8], &site) || a[9] != Py_True || !workspace_ok(a[14], a[15], c.device) || !stream_of(a[15], &st))
            return nullptr;
        for (int i = 0; i < 4; i++)
            if (!optional(a[10 + i], c.device, &g[i]) || (g[i] && !like(*g[i], i < 2 ? *c.x : *c.weight))) return nullptr;
        at::Tensor dx = g[0] ? *g[0] : at::empty(c.x->sizes(), c.x->options()), dy = g[1] ? *g[1] : at::empty(c.x->sizes(), c.x->options());
        at::Tensor dw = g[2] ? *g[2] : at::empty(c.weight->sizes(), c.weight->options()), db = g[3] ? *g[3] : at::empty(c.weight->sizes(), c.weight->options());
        const Room w(a[14], norm_bwd_bytes_fn(c.rows, c.width), *c.x);
        const void *pn = dn->data_ptr(), *pd = data(dh), *ph = c.x->data_ptr(), *pw = c.weight->data_ptr();
        const float *pm = (const float *)mean->data_ptr(), *ps = (const float *)rstd->data_ptr();
        const int64_t *pr = (const int64_t *)data(rng);
        void *p0 = dx.data_ptr(), *p1 = dy.data_ptr(), *p2 = dw.data_ptr(), *p3 = db.data_ptr();
        hdt_status_t s;
        Py_BEGIN_ALLOW_THREADS
        s = norm_bwd_fn(pn, pd, ph, pw, pm, ps, c.rows, c.width, p, pr, site, p0, p1, p2, p3, c.dt, c.wdt, w.at_, w.bytes, st);
        Py_END_ALLOW_THREADS
        return results(s, {dx, dy, dw, db});
    });
}

// ---- embeddings, feed-forward block, norms around a block: the same rules ----
// None, or a torch dtype
bool dtype_or_none(PyObject *o, bool *given, at::ScalarType *t)
{
    *given = o != Py_None;
    if (!*given) return true;
    if (!THPDtype_Check(o)) return false;
    *t = ((THPDtype *)o)->scalar_type;
    return true;
}
bool is_ids(const at::Tensor *t, int device) { return t && here(*t, device) && t->scalar_type() == at::kInt && t->is_contiguous(); }
// the shape of ids with a last dimension
c10::SmallVector<int64_t, 6> with_last(at::IntArrayRef lead, int64_t width)
{
    c10::SmallVector<int64_t, 6> s(lead.begin(), lead.end());
    s.push_back(width);
    return s;
}

// (ids, table, scale, dtype, out, stream) -> out, a status, or None
PyObject *embed_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 6) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        const int device = c10::hip::current_device();
        const at::Tensor *ids = plain(a[0]), *table = plain(a[1]), *given;
        double scale;
        bool typed;
        at::ScalarType type;
        hdt_dtype_t dt, tdt;
        hipStream_t st;
        if (!is_ids(ids, device) || !table || !here(*table, device) || table->dim() != 2 || !table->is_contiguous() || !dtype_of(*table, &tdt) || !number(a[2], &scale) ||
            !dtype_or_none(a[3], &typed, &type) || !optional(a[4], device, &given) || !stream_of(a[5], &st) || table->size(0) > INT32_MAX || table->size(1) > INT32_MAX)
            return nullptr;
        const auto shape = with_last(ids->sizes(), table->size(1));
        if (given && (given->sizes() != at::IntArrayRef(shape) || !given->is_contiguous() || (typed && given->scalar_type() != type))) return nullptr;
        if (!given && typed && type != at::kBFloat16 && type != at::kFloat) return nullptr;
        at::Tensor out = given ? *given : at::empty(shape, typed ? table->options().dtype(type) : table->options());
        if (!dtype_of(out, &dt)) return nullptr;
        const int32_t *pi = (const int32_t *)ids->data_ptr();
        const void *pt = table->data_ptr();
        void *po = out.data_ptr();
        const int64_t tokens = ids->numel();
        const int32_t vocab = (int32_t)table->size(0), width = (int32_t)table->size(1);
        hdt_status_t s;
        Py_BEGIN_ALLOW_THREADS
        s = embed_fwd_fn(pi, tokens, pt, vocab, width, (float)scale, po, tdt, dt, st);
        Py_END_ALLOW_THREADS
        return s != HDT_OK ? PyLong_FromLong(s) : THPVariable_Wrap(out);
    });
}

// (d_out, ids, vocab, scale, dtype, grad, accumulate, workspace, stream) -> grad, a status, or None
PyObject *embed_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 9) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        const int device = c10::hip::current_device();
        const at::Tensor *d = plain(a[0]), *ids = plain(a[1]), *given;
        double scale;
        int32_t vocab;
        bool typed;
        at::ScalarType type;
        hdt_dtype_t dt, tdt;
        hipStream_t st;
        if (!d || !here(*d, device) || !d->is_contiguous() || !dtype_of(*d, &dt) || !is_ids(ids, device) || !whole32(a[2], &vocab) || vocab < 0 || !number(a[3], &scale) ||
            !dtype_or_none(a[4], &typed, &type) || !optional(a[5], device, &given) || !PyBool_Check(a[6]) || (!given && a[6] == Py_True) ||
            !workspace_ok(a[7], a[8], device) || !stream_of(a[8], &st))
            return nullptr;
        if (d->dim() < 1 || d->size(-1) > INT32_MAX || d->sizes().slice(0, d->dim() - 1) != ids->sizes()) return nullptr;
        const int64_t tokens = ids->numel(), width = d->size(-1);
        if (given && (given->dim() != 2 || given->size(0) != vocab || given->size(1) != width || !given->is_contiguous() || (typed && given->scalar_type() != type)))
            return nullptr;
        if (!given && typed && type != at::kBFloat16 && type != at::kFloat) return nullptr;
        at::Tensor grad = given ? *given : at::empty({vocab, width}, typed ? d->options().dtype(type) : d->options());
        if (!dtype_of(grad, &tdt)) return nullptr;
        const Room w(a[7], embed_bwd_bytes_fn(tokens, (int32_t)width), *d);
        const void *pd = d->data_ptr();
        const int32_t *pi = (const int32_t *)ids->data_ptr();
        void *pg = grad.data_ptr();
        hdt_status_t s;
        Py_BEGIN_ALLOW_THREADS
        s = embed_bwd_fn(pd, pi, tokens, vocab, (int32_t)width, (float)scale, a[6] == Py_True, pg, tdt, dt, w.at_, w.bytes, st);
        Py_END_ALLOW_THREADS
        return s != HDT_OK ? PyLong_FromLong(s) : THPVariable_Wrap(grad);
    });
}

// what feed-forward calls have in common: rows of x, three weights
struct FfnCall {
    const at::Tensor *x, *wg, *wu, *wd;
    int64_t rows;
    int32_t width, inner;
    hdt_act_t act = HDT_SILU;
    hdt_dtype_t dt;
    int device;
    // x, w_gate, w_up, w_down
    bool plain_case(PyObject *const *a)
    {
        device = c10::hip::current_device();
        if (!(x = plain(a[0])) || !(wg = plain(a[1])) || !(wu = plain(a[2])) || !(wd = plain(a[3])) || !dtype_of(*x, &dt)) return false;
        for (const at::Tensor *t : {x, wg, wu, wd})
            if (!here(*t, device) || t->scalar_type() != x->scalar_type() || !t->is_contiguous()) return false;
        if (x->dim() < 1 || wg->dim() != 2 || wd->dim() != 2 || wu->sizes() != wg->sizes()) return false;
        const int64_t f = wg->size(0), d = wg->size(1);
        if (x->size(-1) != d || wd->size(0) != d || wd->size(1) != f || d > INT32_MAX || f > INT32_MAX || d == 0) return false;
        width = (int32_t)d, inner = (int32_t)f, rows = x->numel() / d;
        return true;
    }
    bool activation(PyObject *name)
    {
        if (!PyUnicode_CheckExact(name)) return false;
        if (PyUnicode_CompareWithASCIIString(name, "silu") == 0) act = HDT_SILU;
        else if (PyUnicode_CompareWithASCIIString(name, "gelu") == 0) act = HDT_GELU;
        else if (PyUnicode_CompareWithASCIIString(name, "gelu_tanh") == 0) act = HDT_GELU_TANH;
        else return false;
        return true;
    }
    // None or a tensor of x's type: like x, or [..][inner]
    bool result(PyObject *o, const at::Tensor **t, at::IntArrayRef shape) const
    {
        return optional(o, device, t) && (!*t || ((*t)->scalar_type() == x->scalar_type() && (*t)->is_contiguous() && (*t)->sizes() == shape));
    }
    c10::SmallVector<int64_t, 6> kept() const { return with_last(x->sizes().slice(0, x->dim() - 1), inner); }
};

// (x, w_gate, w_up, w_down, act, train, y, by_gate, by_up, hidden, workspace, stream) -> (y, by_gate, by_up, hidden), (y,) without train, a status, or None
PyObject *ffn_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 12) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        FfnCall c;
        hipStream_t st;
        const at::Tensor *gy, *g[3];
        if (!c.plain_case(a) || !c.activation(a[4]) || !PyBool_Check(a[5]) || !c.result(a[6], &gy, c.x->sizes()) || !workspace_ok(a[10], a[11], c.device) || !stream_of(a[11], &st)) return nullptr;
        const bool train = a[5] == Py_True;
        const auto shape = c.kept();
        for (int i = 0; i < 3; i++)
            if (!c.result(a[7 + i], &g[i], shape) || (g[i] && !train)) return nullptr;
        at::Tensor y = gy ? *gy : at::empty(c.x->sizes(), c.x->options()), k[3];
        void *pk[3] = {};
        if (train)
            for (int i = 0; i < 3; i++) {
                k[i] = g[i] ? *g[i] : at::empty(shape, c.x->options());
                pk[i] = k[i].data_ptr();
            }
        const Room w(a[10], ffn_fwd_bytes_fn(c.rows, c.width, c.inner, train, c.dt), *c.x);
        const void *px = c.x->data_ptr(), *pg = c.wg->data_ptr(), *pu = c.wu->data_ptr(), *pd = c.wd->data_ptr();
        void *py = y.data_ptr();
        hdt_status_t s;
        Py_BEGIN_ALLOW_THREADS
        s = ffn_fwd_fn(px, pg, pu, pd, c.rows, c.width, c.inner, c.act, py, pk[0], pk[1], pk[2], c.dt, w.at_, w.bytes, st);
        Py_END_ALLOW_THREADS
        return train ? results(s, {y, k[0], k[1], k[2]}) : results(s, {y});
    });
}

// (dy, x, w_gate, w_up, w_down, by_gate, by_up, hidden, dx, dw_gate, dw_up, dw_down, workspace, stream) -> (dx, dw_gate, dw_up, dw_down), a
// status, or None
PyObject *ffn_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 14) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        FfnCall c;
        hipStream_t st;
        const at::Tensor *dy, *kept[3], *g[4];
        if (!c.plain_case(a + 1) || !c.result(a[0], &dy, c.x->sizes()) || !dy || !workspace_ok(a[12], a[13], c.device) || !stream_of(a[13], &st)) return nullptr;
        const auto shape = c.kept();
        for (int i = 0; i < 3; i++)
            if (!c.result(a[5 + i], &kept[i], shape) || !kept[i]) return nullptr;
        const at::Tensor *like_[4] = {c.x, c.wg, c.wu, c.wd};
        at::Tensor out[4];
        for (int i = 0; i < 4; i++) {
            if (!c.result(a[8 + i], &g[i], like_[i]->sizes())) return nullptr;
        }
        for (int i = 0; i < 4; i++) out[i] = g[i] ? *g[i] : at::empty(like_[i]->sizes(), c.x->options());
        const Room w(a[12], ffn_bwd_bytes_fn(c.rows, c.width, c.inner, c.dt), *c.x);
        const void *p[8] = {dy->data_ptr(), c.x->data_ptr(), c.wg->data_ptr(), c.wu->data_ptr(), c.wd->data_ptr(), kept[0]->data_ptr(), kept[1]->data_ptr(), kept[2]->data_ptr()};
        void *o[4] = {out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), out[3].data_ptr()};
        hdt_status_t s;
        Py_BEGIN_ALLOW_THREADS
        s = ffn_bwd_fn(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], c.rows, c.width, c.inner, o[0], o[1], o[2], o[3], c.dt, w.at_, w.bytes, st);
        Py_END_ALLOW_THREADS
        return results(s, {out[0], out[1], out[2], out[3]});
    });
}

bool is_stats(const at::Tensor &t, const at::Tensor &x, int device)
{
    return here(t, device) && t.scalar_type() == at::kFloat && t.is_contiguous() && t.dim() == x.dim() && t.size(0) == 4 && t.sizes().slice(1) == x.sizes().slice(0, x.dim() - 1);
}

// (x, y, post_weight, weight, gate, post_bias, bias, scale, eps, rms, h, n, stats, stream) -> (n, h, stats), a status, or None
PyObject *gate_norm_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 14) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        NormCall c;
        const at::Tensor *y = plain(a[1]), *pw = plain(a[2]), *v[3], *g[2], *gs;
        double scale, eps;
        hipStream_t st;
        if (!c.plain_case(a[0], a[3]) || !y || !here(*y, c.device) || !like(*y, *c.x) || !pw || !here(*pw, c.device) || !like(*pw, *c.weight) || !number(a[7], &scale) ||
            !number(a[8], &eps) || !PyBool_Check(a[9]) || !optional(a[12], c.device, &gs) || (gs && !is_stats(*gs, *c.x, c.device)) || !stream_of(a[13], &st))
            return nullptr;
        for (int i = 0; i < 3; i++)
            if (!optional(a[4 + i], c.device, &v[i]) || (v[i] && !like(*v[i], *c.weight))) return nullptr;
        for (int i = 0; i < 2; i++)
            if (!optional(a[10 + i], c.device, &g[i]) || (g[i] && !like(*g[i], *c.x))) return nullptr;
        at::Tensor h = g[0] ? *g[0] : at::empty(c.x->sizes(), c.x->options()), out = g[1] ? *g[1] : at::empty(c.x->sizes(), c.x->options()), stats;
        if (gs) {
            stats = *gs;
        } else {
            c10::SmallVector<int64_t, 6> shape = {4};
            const auto lead = c.x->sizes().slice(0, c.x->dim() - 1);
            shape.append(lead.begin(), lead.end());
            stats = at::empty(shape, c.x->options().dtype(at::kFloat));
        }
        const void *px = c.x->data_ptr(), *py = y->data_ptr(), *pp = pw->data_ptr(), *pw_ = c.weight->data_ptr(), *pg = data(v[0]), *pb = data(v[1]), *pc = data(v[2]);
        void *ph = h.data_ptr(), *pn = out.data_ptr();
        float *ps = (float *)stats.data_ptr();
        hdt_status_t s;
        Py_BEGIN_ALLOW_THREADS
        s = gate_norm_fwd_fn(px, py, pp, pb, pg, pw_, pc, c.rows, c.width, (float)eps, (float)scale, a[9] == Py_True, ph, pn, ps, c.dt, c.wdt, st);
        Py_END_ALLOW_THREADS
        return results(s, {out, h, stats});
    });
}

// (dn, h, y, stats, post_weight, weight, gate, post_bias, bias, dh, scale, rms, dx, dy, dpost_weight, dweight, dgate, dpost_bias, dbias, workspace,
// stream) -> (dx, dy, dpost_weight, dweight, dgate, dpost_bias, dbias), a status, or None
PyObject *gate_norm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 21) Py_RETURN_NONE;
    return guarded([&]() -> PyObject * {
        NormCall c;
        const at::Tensor *dn = plain(a[0]), *y = plain(a[2]), *stats = plain(a[3]), *pw = plain(a[4]), *gate, *pb, *dh, *g[7];
        double scale;
        hipStream_t st;
        if (!c.plain_case(a[1], a[5]) || !dn || !here(*dn, c.device) || !like(*dn, *c.x) || !y || !here(*y, c.device) || !like(*y, *c.x) || !stats || !is_stats(*stats, *c.x, c.device) ||
            !pw || !here(*pw, c.device) || !like(*pw, *c.weight) || !optional(a[6], c.device, &gate) || (gate && !like(*gate, *c.weight)) || !optional(a[7], c.device, &pb) ||
            (pb && !like(*pb, *c.weight)) || !PyBool_Check(a[8]) || !optional(a[9], c.device, &dh) || (dh && !like(*dh, *c.x)) || !number(a[10], &scale) || !PyBool_Check(a[11]) ||
            !workspace_ok(a[19], a[20], c.device) || !stream_of(a[20], &st))
            return nullptr;
        const bool there[7] = {true, true, true, true, gate != nullptr, pb != nullptr, a[8] == Py_True};
        for (int i = 0; i < 7; i++)
            if (!optional(a[12 + i], c.device, &g[i]) || (g[i] && (!there[i] || !like(*g[i], i < 2 ? *c.x : *c.weight)))) return nullptr;
        at::Tensor out[7];
        void *po[7] = {};
        for (int i = 0; i < 7; i++) {
            if (!there[i]) continue;
            const at::Tensor &as = i < 2 ? *c.x : *c.weight;
            out[i] = g[i] ? *g[i] : at::empty(as.sizes(), as.options());
            po[i] = out[i].data_ptr();
        }
        const Room w(a[19], gate_norm_bwd_bytes_fn(c.rows, c.width), *c.x);
        const void *pn = dn->data_ptr(), *pd = data(dh), *ph = c.x->data_ptr(), *py = y->data_ptr(), *pp = pw->data_ptr(), *pq = data(pb), *pg = data(gate), *pw_ = c.weight->data_ptr();
        const float *ps = (const float *)stats->data_ptr();
        hdt_status_t s;
        Py_BEGIN_ALLOW_THREADS
        s = gate_norm_bwd_fn(pn, pd, ph, py, ps, pp, pq, pg, pw_, c.rows, c.width, (float)scale, a[11] == Py_True, po[0], po[1], po[2], po[5], po[4], po[3], po[6], c.dt, c.wdt,
                             w.at_, w.bytes, st);
        Py_END_ALLOW_THREADS
        return results(s, {out[0], out[1], out[2], out[3], out[4], out[5], out[6]});
    });
}

// the addresses of the operators' functions, in the order of their pointers above
PyObject *bind_operators(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 18) {
        PyErr_SetString(PyExc_TypeError, "bind_operators takes eighteen addresses");
        return nullptr;
    }
    void *p[18];
    for (int i = 0; i < 18; i++)
        if (!(p[i] = PyLong_AsVoidPtr(a[i]))) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind_operators: NULL");
            return nullptr;
        }
    rel_fwd_bytes_fn = (decltype(rel_fwd_bytes_fn))p[0];
    rel_fwd_fn = (decltype(rel_fwd_fn))p[1];
    rel_bwd_bytes_fn = (decltype(rel_bwd_bytes_fn))p[2];
    rel_bwd_fn = (decltype(rel_bwd_fn))p[3];
    dropout_fn = (decltype(dropout_fn))p[4];
    norm_fwd_fn = (decltype(norm_fwd_fn))p[5];
    norm_bwd_bytes_fn = (decltype(norm_bwd_bytes_fn))p[6];
    norm_bwd_fn = (decltype(norm_bwd_fn))p[7];
    embed_fwd_fn = (decltype(embed_fwd_fn))p[8];
    embed_bwd_bytes_fn = (decltype(embed_bwd_bytes_fn))p[9];
    embed_bwd_fn = (decltype(embed_bwd_fn))p[10];
    ffn_fwd_bytes_fn = (decltype(ffn_fwd_bytes_fn))p[11];
    ffn_fwd_fn = (decltype(ffn_fwd_fn))p[12];
    ffn_bwd_bytes_fn = (decltype(ffn_bwd_bytes_fn))p[13];
    ffn_bwd_fn = (decltype(ffn_bwd_fn))p[14];
    gate_norm_fwd_fn = (decltype(gate_norm_fwd_fn))p[15];
    gate_norm_bwd_bytes_fn = (decltype(gate_norm_bwd_bytes_fn))p[16];
    gate_norm_bwd_fn = (decltype(gate_norm_bwd_fn))p[17];
    Py_RETURN_NONE;
}

// the addresses of libhdt's functions, in the order of the first pointers above
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "bind takes five addresses");
        return nullptr;
    }
    void *p[5];
    for (int i = 0; i < 5; i++)
        if (!(p[i] = PyLong_AsVoidPtr(a[i]))) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: NULL");
            return nullptr;
        }
    build_layout_fn = (decltype(build_layout_fn))p[0];
    fwd_fn = (decltype(fwd_fn))p[1];
    fwd_ws_fn = (decltype(fwd_ws_fn))p[2];
    bwd_fn = (decltype(bwd_fn))p[3];
    bwd_bytes_fn = (decltype(bwd_bytes_fn))p[4];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
    {"build_layout", (PyCFunction)(void (*)(void))build_layout, METH_FASTCALL, nullptr},
    {"attn_fwd", (PyCFunction)(void (*)(void))attn_fwd, METH_FASTCALL, nullptr},
    {"attn_bwd", (PyCFunction)(void (*)(void))attn_bwd, METH_FASTCALL, nullptr},
    {"bind_operators", (PyCFunction)(void (*)(void))bind_operators, METH_FASTCALL, nullptr},
    {"rel_attn_fwd", (PyCFunction)(void (*)(void))rel_attn_fwd, METH_FASTCALL, nullptr},
    {"rel_attn_bwd", (PyCFunction)(void (*)(void))rel_attn_bwd, METH_FASTCALL, nullptr},
    {"dropout_add", (PyCFunction)(void (*)(void))dropout_add, METH_FASTCALL, nullptr},
    {"add_norm_fwd", (PyCFunction)(void (*)(void))add_norm_fwd, METH_FASTCALL, nullptr},
    {"add_norm_bwd", (PyCFunction)(void (*)(void))add_norm_bwd, METH_FASTCALL, nullptr},
    {"embed_fwd", (PyCFunction)(void (*)(void))embed_fwd, METH_FASTCALL, nullptr},
    {"embed_bwd", (PyCFunction)(void (*)(void))embed_bwd, METH_FASTCALL, nullptr},
    {"ffn_fwd", (PyCFunction)(void (*)(void))ffn_fwd, METH_FASTCALL, nullptr},
    {"ffn_bwd", (PyCFunction)(void (*)(void))ffn_bwd, METH_FASTCALL, nullptr},
    {"gate_norm_fwd", (PyCFunction)(void (*)(void))gate_norm_fwd, METH_FASTCALL, nullptr},
    {"gate_norm_bwd", (PyCFunction)(void (*)(void))gate_norm_bwd, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_hdt_pycall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__hdt_pycall()
{
    PyObject *m = PyModule_Create(&module);
    // (binding.py uses the module under this torch alone: nothing else says that its tensors are laid out as in these headers)
    if (m && PyModule_AddStringConstant(m, "torch_version", HDT_TORCH_VERSION) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
