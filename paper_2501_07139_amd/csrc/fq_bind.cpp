// The way from a Python call to its C entry point for the calls that a served token or a small linear makes: argument checks, device
// addresses and the current stream without a Python call each.  A call of fq_qlinear at 16 x 512 x 512 took 5.7 us through
// ctypes, 3.7 of them the launch itself; through here 4.0.
//
// Every function takes the arguments of its namesake in the package and returns the entry point's code, or None when
// something is not as the plain case has it (an output to allocate, another tensor type, a size that does not fit,
// a wrong type): the caller then goes the long way, which allocates or raises.  Nothing is kept from one call to the next.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "fq.h"

#include <climits>
#include <cstring>
#include <initializer_list>
#include <memory>

namespace {

// entry points of libfq, as the package has loaded it
struct Entries {
    decltype(&fq_qlinear_tile) qlinear;
    decltype(&fq_qlinear_mixed) mixed;
    decltype(&fq_dense_f16) dense;
    decltype(&fq_head_nll) head_nll;
    decltype(&fq_token_nll) token_nll;
    decltype(&fq_logit_l2) logit_l2;
    decltype(&fq_qk_norm_rope) norm_rope;
    decltype(&fq_attn_paged) attn_paged;
    decltype(&fq_cache_evict) evict;
    decltype(&fq_paged_plan) plan;
    decltype(&fq_attn_tree) attn_tree;
    decltype(&fq_tree_commit) commit;
    decltype(&fq_beam_step) beam;
} entry;

PyObject *s_packed, *s_scales, *s_zeros, *s_n, *s_k, *s_bits, *s_struct, *s_positions, *s_slots, *s_q_start, *s_seq_len, *s_table, *s_held, *s_free_pages, *s_free_count,
    *s_lacking, *s_mask;

// A contiguous device tensor of plain type, else nullptr.
const at::Tensor *device_tensor(PyObject *o, at::ScalarType type)
{
    if (!THPVariable_CheckExact(o))
        return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.is_cuda() && t.scalar_type() == type && t.is_contiguous() ? &t : nullptr;
}

const at::Tensor *half_matrix(PyObject *o, int *rows, int *cols)
{
    const at::Tensor *t = device_tensor(o, at::kHalf);
    if (!t || t->dim() != 2 || t->size(0) > INT_MAX || t->size(1) > INT_MAX)
        return nullptr;
    *rows = (int)t->size(0);
    *cols = (int)t->size(1);
    return t;
}

// None: the current stream; a number: that handle.
bool stream_of(PyObject *o, void **stream)
{
    if (o == Py_None) {
        *stream = c10::hip::getCurrentHIPStream().stream();
        return true;
    }
    if (!PyLong_CheckExact(o))
        return false;
    *stream = PyLong_AsVoidPtr(o);
    return !PyErr_Occurred();
}

bool int_of(PyObject *o, int *v)
{
    if (!PyLong_CheckExact(o))
        return false;
    int overflow = 0;
    const long l = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow || l < INT_MIN || l > INT_MAX)
        return false;
    *v = (int)l;
    return true;
}

bool int_attr(PyObject *o, PyObject *name, int *v)
{
    PyObject *a = PyObject_GetAttr(o, name);
    if (!a)
        return false;
    const bool ok = int_of(a, v);
    Py_DECREF(a);
    return ok;
}

// Address of an attribute that is a tensor; the object keeps the tensor alive during the call.
bool tensor_attr(PyObject *o, PyObject *name, const void **v)
{
    PyObject *a = PyObject_GetAttr(o, name);
    if (!a)
        return false;
    const bool ok = THPVariable_CheckExact(a);
    if (ok)
        *v = THPVariable_Unpack(a).data_ptr();
    Py_DECREF(a);
    return ok;
}

bool matrix_of(PyObject *w, fq_segment *m, int *K)
{
    return tensor_attr(w, s_packed, &m->packed) && tensor_attr(w, s_scales, &m->scales) && tensor_attr(w, s_zeros, &m->zeros) &&
           int_attr(w, s_n, &m->N) && int_attr(w, s_k, K) && int_attr(w, s_bits, &m->bits);
}

// f(args) with C++ exceptions (a tensor without storage) and pending Python errors turned into "the long way".
template <class F>
PyObject *guarded(Py_ssize_t have, Py_ssize_t need, F &&f)
{
    int rc = 0;
    bool done = false;
    if (have == need) {
        try {
            done = f(&rc);
        } catch (...) {
            done = false;
        }
    }
    if (done)
        return PyLong_FromLong(rc);
    PyErr_Clear();
    Py_RETURN_NONE;
}

template <class F>
int without_gil(F &&f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = f();
    Py_END_ALLOW_THREADS return rc;
}

PyObject *qlinear(PyObject *, PyObject *const *a, Py_ssize_t n) // x, w, out, stream, group, tile_rows
{
    return guarded(n, 6, [&](int *rc) {
        int M, K, wk, group, tile_rows;
        void *stream;
        fq_segment w;
        const at::Tensor *x = half_matrix(a[0], &M, &K), *out = device_tensor(a[2], at::kHalf);
        if (!x || !out || !matrix_of(a[1], &w, &wk) || wk != K || !stream_of(a[3], &stream) || !int_of(a[4], &group) ||
            !int_of(a[5], &tile_rows))
            return false;
        const void *px = x->data_ptr();
        void *po = out->data_ptr();
        *rc = without_gil([&] { return entry.qlinear(px, M, w.packed, w.scales, w.zeros, w.N, K, w.bits, group, po, tile_rows, stream); });
        return true;
    });
}

PyObject *mixed(PyObject *, PyObject *const *a, Py_ssize_t n) // x, segments (list or tuple), out, stream, group
{
    return guarded(n, 5, [&](int *rc) {
        int M, K, group;
        void *stream;
        fq_segment seg[FQ_MAX_SEGMENTS];
        const at::Tensor *x = half_matrix(a[0], &M, &K), *out = device_tensor(a[2], at::kHalf);
        if (!x || !out || !(PyList_CheckExact(a[1]) || PyTuple_CheckExact(a[1])) || !stream_of(a[3], &stream) || !int_of(a[4], &group))
            return false;
        // its items, held: reading an attribute may run Python code, which may change the list
        const std::unique_ptr<PyObject, void (*)(PyObject *)> items(PySequence_Tuple(a[1]), [](PyObject *o) { Py_DECREF(o); });
        const Py_ssize_t count = items ? PyTuple_GET_SIZE(items.get()) : 0;
        if (count < 1 || count > FQ_MAX_SEGMENTS)
            return false;
        for (Py_ssize_t i = 0; i < count; ++i) {
            int wk;
            if (!matrix_of(PyTuple_GET_ITEM(items.get(), i), &seg[i], &wk) || wk != K)
                return false;
        }
        const void *px = x->data_ptr();
        void *po = out->data_ptr();
        *rc = without_gil([&] { return entry.mixed(px, M, seg, (int)count, K, group, po, stream); });
        return true;
    });
}

PyObject *dense_f16(PyObject *, PyObject *const *a, Py_ssize_t n) // x, W, out, stream
{
    return guarded(n, 4, [&](int *rc) {
        int M, K, N, wk;
        void *stream;
        const at::Tensor *x = half_matrix(a[0], &M, &K), *W = half_matrix(a[1], &N, &wk), *out = device_tensor(a[2], at::kHalf);
        if (!x || !W || !out || wk != K || !stream_of(a[3], &stream))
            return false;
        const void *px = x->data_ptr(), *pw = W->data_ptr();
        void *po = out->data_ptr();
        *rc = without_gil([&] { return entry.dense(px, M, pw, N, K, po, stream); });
        return true;
    });
}

PyObject *head_nll(PyObject *, PyObject *const *a, Py_ssize_t n) // x, W, labels, out, workspace, stream
{
    return guarded(n, 6, [&](int *rc) {
        int M, K, V, wk;
        void *stream;
        const at::Tensor *x = half_matrix(a[0], &M, &K), *W = half_matrix(a[1], &V, &wk), *labels = device_tensor(a[2], at::kInt),
                         *out = device_tensor(a[3], at::kFloat), *ws = device_tensor(a[4], at::kByte);
        if (!x || !W || !labels || !out || !ws || wk != K || labels->numel() != M || !stream_of(a[5], &stream))
            return false;
        const void *px = x->data_ptr(), *pw = W->data_ptr();
        const int32_t *pl = static_cast<const int32_t *>(labels->data_ptr());
        float *po = static_cast<float *>(out->data_ptr());
        void *pws = ws->data_ptr();
        const size_t bytes = (size_t)ws->numel();
        *rc = without_gil([&] { return entry.head_nll(px, M, pw, V, K, pl, po, pws, bytes, stream); });
        return true;
    });
}

PyObject *token_nll(PyObject *, PyObject *const *a, Py_ssize_t n) // logits, labels, out, stream
{
    return guarded(n, 4, [&](int *rc) {
        int M, V;
        void *stream;
        const at::Tensor *l = half_matrix(a[0], &M, &V), *labels = device_tensor(a[1], at::kInt), *out = device_tensor(a[2], at::kFloat);
        if (!l || !labels || !out || !stream_of(a[3], &stream))
            return false;
        const void *pl = l->data_ptr();
        const int32_t *pi = static_cast<const int32_t *>(labels->data_ptr());
        float *po = static_cast<float *>(out->data_ptr());
        *rc = without_gil([&] { return entry.token_nll(pl, pi, M, V, po, stream); });
        return true;
    });
}

PyObject *logit_l2(PyObject *, PyObject *const *a, Py_ssize_t n) // a, b, out, stream
{
    return guarded(n, 4, [&](int *rc) {
        int M, V, mb, vb;
        void *stream;
        const at::Tensor *x = half_matrix(a[0], &M, &V), *y = half_matrix(a[1], &mb, &vb), *out = device_tensor(a[2], at::kFloat);
        if (!x || !y || !out || mb != M || vb != V || !stream_of(a[3], &stream))
            return false;
        const void *px = x->data_ptr(), *py = y->data_ptr();
        float *po = static_cast<float *>(out->data_ptr());
        *rc = without_gil([&] { return entry.logit_l2(px, py, M, V, po, stream); });
        return true;
    });
}

// ---- paged cache: the calls that a step makes once a block
bool float_of(PyObject *o, float *v)
{
    if (!PyFloat_CheckExact(o))
        return false;
    *v = (float)PyFloat_AS_DOUBLE(o);
    return true;
}

// Whether an attribute is an int32 tensor on dev at this address.
bool ints_at(PyObject *o, PyObject *name, c10::Device dev, const int32_t *at)
{
    PyObject *a = PyObject_GetAttr(o, name);
    if (!a)
        return false;
    const at::Tensor *t = device_tensor(a, at::kInt);
    const bool ok = t && t->device() == dev && t->data_ptr() == at;
    Py_DECREF(a);
    return ok;
}

// The C structure of a PagedBatch whose arrays are on dev: the structure itself has bare addresses, which may be the host's or another device's.
bool batch_of(PyObject *o, c10::Device dev, fq_paged_batch *b)
{
    PyObject *a = PyObject_GetAttr(o, s_struct);
    if (!a)
        return false;
    Py_buffer view;
    bool ok = PyObject_GetBuffer(a, &view, PyBUF_SIMPLE) == 0;
    if (ok) {
        ok = view.len == (Py_ssize_t)sizeof(*b);
        if (ok)
            memcpy(b, view.buf, sizeof(*b));
        PyBuffer_Release(&view);
    }
    Py_DECREF(a);
    return ok && ints_at(o, s_q_start, dev, b->q_start) && ints_at(o, s_seq_len, dev, b->seq_len) && ints_at(o, s_table, dev, b->table);
}

// None, or a contiguous device tensor of this type on dev.
bool optional(PyObject *o, at::ScalarType type, c10::Device dev, const void **v)
{
    *v = nullptr;
    if (o == Py_None)
        return true;
    const at::Tensor *t = device_tensor(o, type);
    if (!t || t->device() != dev)
        return false;
    *v = t->data_ptr();
    return true;
}

// An attribute that is an int32 device tensor of an entry a token.
bool token_ints(PyObject *o, PyObject *name, int64_t tokens, c10::Device dev, const void **v)
{
    PyObject *a = PyObject_GetAttr(o, name);
    if (!a)
        return false;
    const at::Tensor *t = device_tensor(a, at::kInt);
    const bool ok = t && t->numel() == tokens && t->device() == dev;
    if (ok)
        *v = t->data_ptr();
    Py_DECREF(a);
    return ok;
}

bool shape_is(const at::Tensor *t, std::initializer_list<int64_t> dims) // -1: any
{
    if (!t || t->dim() != (int64_t)dims.size())
        return false;
    int64_t i = 0;
    for (const int64_t d : dims)
        if (t->size(i++) != d && d >= 0)
            return false;
    return true;
}

// fp16 rows of a matrix that may be columns of a wider one.
const at::Tensor *half_rows(PyObject *o, int64_t rows, int64_t width, int *ld)
{
    if (!THPVariable_CheckExact(o))
        return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != at::kHalf || t.dim() != 2 || t.size(0) != rows || t.size(1) != width || t.stride(1) != 1)
        return nullptr;
    const int64_t step = rows > 1 ? t.stride(0) : (width + 7) / 8 * 8;
    if (step < 0 || step > INT_MAX)
        return nullptr;
    *ld = (int)step;
    return &t;
}

// Both pools of a batch: [pages, heads, page, 128]; the heads, or 0.
int64_t pools_of(PyObject *k, PyObject *v, int64_t pages, int64_t page, c10::Device dev, const void **pk, const void **pv)
{
    const at::Tensor *tk = device_tensor(k, at::kHalf), *tv = device_tensor(v, at::kHalf);
    if (!shape_is(tk, {pages, -1, page, 128}) || !tv || tv->sizes() != tk->sizes() || tk->device() != dev || tv->device() != dev ||
        tk->size(0) > INT_MAX || tk->size(1) > INT_MAX)
        return 0;
    *pk = tk->data_ptr();
    *pv = tv->data_ptr();
    return tk->size(1);
}

PyObject *qk_norm_rope(PyObject *, PyObject *const *a, Py_ssize_t n) // q, k, v, batch, rope, k_pages, v_pages, q_gain, k_gain, eps, out, stream
{
    return guarded(n, 12, [&](int *rc) {
        fq_paged_batch b;
        const at::Tensor *rope = device_tensor(a[4], at::kFloat), *out = device_tensor(a[10], at::kHalf);
        if (!out || out->dim() != 2 || !shape_is(rope, {-1, 64, 2}) || rope->size(0) > INT_MAX || !batch_of(a[3], out->device(), &b) || b.tokens == 0)
            return false;
        const c10::Device dev = out->device();
        const int64_t tokens = b.tokens, width = out->size(1);
        const void *pk, *pv, *qg, *kg, *positions, *slots;
        void *stream;
        float eps;
        int ldq, ldk, ldv;
        const int64_t kv = pools_of(a[5], a[6], b.pages, b.page, dev, &pk, &pv);
        const at::Tensor *q = half_rows(a[0], tokens, width, &ldq), *k = half_rows(a[1], tokens, 128 * kv, &ldk),
                         *v = half_rows(a[2], tokens, 128 * kv, &ldv);
        if (kv == 0 || width % 128 != 0 || width > INT_MAX || out->size(0) != tokens || !q || !k || !v || rope->device() != dev || q->device() != dev ||
            k->device() != dev || v->device() != dev || !optional(a[7], at::kHalf, dev, &qg) || !optional(a[8], at::kHalf, dev, &kg) ||
            (qg && THPVariable_Unpack(a[7]).numel() != 128) || (kg && THPVariable_Unpack(a[8]).numel() != 128) || !float_of(a[9], &eps) ||
            !token_ints(a[3], s_positions, tokens, dev, &positions) || !token_ints(a[3], s_slots, tokens, dev, &slots) || !stream_of(a[11], &stream))
            return false;
        const void *px = q->data_ptr(), *py = k->data_ptr(), *pz = v->data_ptr();
        const float *pr = static_cast<const float *>(rope->data_ptr());
        const int rows = (int)rope->size(0);
        void *po = out->data_ptr();
        *rc = without_gil([&] {
            return entry.norm_rope(px, ldq, py, ldk, pz, ldv, b.tokens, (int)(width / 128), (int)kv, static_cast<const int32_t *>(positions),
                                   static_cast<const int32_t *>(slots), pr, rows, qg, kg, eps, po, const_cast<void *>(pk),
                                   const_cast<void *>(pv), b.page, b.pages, stream);
        });
        return true;
    });
}

PyObject *attn_paged(PyObject *, PyObject *const *a, Py_ssize_t n) // q, batch, k_pages, v_pages, scale, out, lse, weights, weights_out, workspace, stream
{
    return guarded(n, 11, [&](int *rc) {
        fq_paged_batch b;
        const at::Tensor *out = device_tensor(a[5], at::kHalf), *ws = a[9] == Py_None ? nullptr : device_tensor(a[9], at::kByte);
        if (!out || out->dim() != 2 || (!ws && a[9] != Py_None) || !batch_of(a[1], out->device(), &b) || b.tokens == 0)
            return false;
        const c10::Device dev = out->device();
        const int64_t tokens = b.tokens, width = out->size(1);
        const void *pk, *pv, *lse, *win, *wout;
        void *stream;
        float scale;
        int ldq;
        const int64_t kv = pools_of(a[2], a[3], b.pages, b.page, dev, &pk, &pv);
        const at::Tensor *q = half_rows(a[0], tokens, width, &ldq);
        if (kv == 0 || width % 128 != 0 || width > INT_MAX || out->size(0) != tokens || !q || q->device() != dev || (ws && ws->device() != dev) ||
            !float_of(a[4], &scale) || !optional(a[6], at::kFloat, dev, &lse) || !optional(a[7], at::kFloat, dev, &win) ||
            !optional(a[8], at::kFloat, dev, &wout) || (win && !wout) || !stream_of(a[10], &stream))
            return false;
        if (lse && !shape_is(&THPVariable_Unpack(a[6]), {tokens, width / 128}))
            return false;
        int64_t wstride = 0;
        if (wout) {
            const at::Tensor &w = THPVariable_Unpack(a[8]);
            if (!shape_is(&w, {b.seqs, kv, -1}) || w.size(2) > INT_MAX || (win && THPVariable_Unpack(a[7]).sizes() != w.sizes()))
                return false;
            wstride = w.size(2);
        }
        const void *px = q->data_ptr();
        void *po = out->data_ptr(), *pw = ws ? ws->data_ptr() : nullptr;
        const size_t bytes = ws ? (size_t)ws->numel() : 0;
        *rc = without_gil([&] {
            return entry.attn_paged(&b, px, ldq, (int)(width / 128), (int)kv, pk, pv, scale, po, static_cast<float *>(const_cast<void *>(lse)),
                                    static_cast<const float *>(win), static_cast<float *>(const_cast<void *>(wout)), (int)wstride, pw, bytes, stream);
        });
        return !(*rc == FQ_ERR_WORKSPACE && !ws); // none given: the long way makes one
    });
}

// batch, weights, k_pages, v_pages, dst_table, keep, recent, k_out, v_out, kept, new_len, weights_out, stream
PyObject *cache_evict(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 13, [&](int *rc) {
        fq_paged_batch b;
        const at::Tensor *w = device_tensor(a[1], at::kFloat), *dst = device_tensor(a[4], at::kInt), *kept = device_tensor(a[9], at::kInt),
                         *len = device_tensor(a[10], at::kInt);
        int keep, recent;
        void *stream;
        if (!w || !dst || !kept || !len || !batch_of(a[0], w->device(), &b) || !int_of(a[5], &keep) || !int_of(a[6], &recent) || !stream_of(a[12], &stream))
            return false;
        const c10::Device dev = w->device();
        const void *pk, *pv, *ko, *vo, *wout;
        const int64_t kv = pools_of(a[2], a[3], b.pages, b.page, dev, &pk, &pv);
        if (kv == 0 || pools_of(a[7], a[8], -1, b.page, dev, &ko, &vo) != kv || !shape_is(w, {b.seqs, kv, -1}) || w->size(2) > INT_MAX ||
            !shape_is(dst, {b.seqs, -1}) || dst->size(1) > INT_MAX || !shape_is(kept, {b.seqs, kv, keep}) || len->numel() != b.seqs ||
            dst->device() != dev || kept->device() != dev || len->device() != dev || !optional(a[11], at::kFloat, dev, &wout))
            return false;
        int64_t ostride = 0;
        if (wout) {
            const at::Tensor &t = THPVariable_Unpack(a[11]);
            if (!shape_is(&t, {b.seqs, kv, -1}) || t.size(2) > INT_MAX)
                return false;
            ostride = t.size(2);
        }
        const int64_t pages_out = THPVariable_Unpack(a[7]).size(0);
        const float *pw = static_cast<const float *>(w->data_ptr());
        const int32_t *pd = static_cast<const int32_t *>(dst->data_ptr());
        int32_t *pkept = static_cast<int32_t *>(kept->data_ptr()), *plen = static_cast<int32_t *>(len->data_ptr());
        *rc = without_gil([&] {
            return entry.evict(&b, pk, pv, (int)kv, pw, (int)w->size(2), keep, recent, pd, (int)dst->size(1), (int)pages_out, const_cast<void *>(ko),
                               const_cast<void *>(vo), pkept, plen, static_cast<float *>(const_cast<void *>(wout)), (int)ostride, stream);
        });
        return true;
    });
}

// ---- trees of tokens
// The current device: a launch goes there, whatever device the tensors are on.
bool is_current(c10::Device dev) { return dev.index() == c10::hip::getCurrentHIPStream().device_index(); }

// An int32 device tensor of this shape on dev, or None where it need not be there.
bool ints_of(PyObject *o, std::initializer_list<int64_t> dims, c10::Device dev, bool needed, const void **v)
{
    return optional(o, at::kInt, dev, v) && (o == Py_None ? !needed : shape_is(&THPVariable_Unpack(o), dims));
}

// batch, new_tokens, cached, next_position, parents, held_out, free_out, stream
PyObject *paged_plan(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 8, [&](int *rc) {
        fq_paged_batch b;
        const at::Tensor *fresh = device_tensor(a[1], at::kInt);
        void *stream;
        if (!fresh || !is_current(fresh->device()) || !batch_of(a[0], fresh->device(), &b) || !stream_of(a[7], &stream))
            return false;
        const c10::Device dev = fresh->device();
        const void *nw, *cached, *next, *parents, *held, *held_out, *pages, *count, *count_out, *lacking, *positions, *slots;
        if (!ints_of(a[1], {b.seqs}, dev, true, &nw) || !ints_of(a[2], {b.seqs}, dev, true, &cached) || !ints_of(a[3], {b.seqs}, dev, false, &next) ||
            !ints_of(a[4], {b.tokens}, dev, false, &parents) || !ints_of(a[5], {b.seqs}, dev, false, &held_out) ||
            !ints_of(a[6], {1}, dev, false, &count_out) || !token_ints(a[0], s_held, b.seqs, dev, &held) ||
            !token_ints(a[0], s_free_pages, b.pages, dev, &pages) || !token_ints(a[0], s_free_count, 1, dev, &count) ||
            !token_ints(a[0], s_lacking, 1, dev, &lacking) || !token_ints(a[0], s_positions, b.tokens, dev, &positions) ||
            !token_ints(a[0], s_slots, b.tokens, dev, &slots))
            return false;
        void *mask = nullptr;
        int words = 0;
        if (parents && b.tokens > 0) {
            const std::unique_ptr<PyObject, void (*)(PyObject *)> m(PyObject_GetAttr(a[0], s_mask), [](PyObject *o) { Py_XDECREF(o); });
            if (!m)
                return false;
            if (m.get() != Py_None) {
                const at::Tensor *t = device_tensor(m.get(), at::kLong);
                if (!shape_is(t, {b.tokens, -1}) || t->device() != dev || t->size(1) < 1 || t->size(1) > FQ_TREE_WORDS)
                    return false;
                mask = t->data_ptr();
                words = (int)t->size(1);
            }
        }
        const auto in = [](const void *p) { return static_cast<const int32_t *>(p); };
        const auto out = [](const void *p) { return static_cast<int32_t *>(const_cast<void *>(p)); };
        *rc = without_gil([&] {
            return entry.plan(&b, in(nw), in(cached), in(next), in(parents), in(held), out(held_out ? held_out : held), out(pages), in(count),
                              out(count_out ? count_out : count), out(lacking), out(positions), out(slots), static_cast<uint64_t *>(mask), words, stream);
        });
        return true;
    });
}

PyObject *attn_tree(PyObject *, PyObject *const *a, Py_ssize_t n) // q, batch, mask, k_pages, v_pages, tail, scale, out, lse, workspace, stream
{
    return guarded(n, 11, [&](int *rc) {
        fq_paged_batch b;
        const at::Tensor *out = device_tensor(a[7], at::kHalf), *mask = device_tensor(a[2], at::kLong),
                         *ws = a[9] == Py_None ? nullptr : device_tensor(a[9], at::kByte);
        if (!out || out->dim() != 2 || !mask || (!ws && a[9] != Py_None) || !is_current(out->device()) || !batch_of(a[1], out->device(), &b) || b.tokens == 0)
            return false;
        const c10::Device dev = out->device();
        const int64_t tokens = b.tokens, width = out->size(1);
        const void *pk, *pv, *lse, *tail;
        void *stream;
        float scale;
        int ldq;
        const int64_t kv = pools_of(a[3], a[4], b.pages, b.page, dev, &pk, &pv);
        const at::Tensor *q = half_rows(a[0], tokens, width, &ldq);
        if (kv == 0 || width % 128 != 0 || width > INT_MAX || out->size(0) != tokens || !q || q->device() != dev || (ws && ws->device() != dev) ||
            mask->device() != dev || !shape_is(mask, {tokens, -1}) || mask->size(1) < 1 || mask->size(1) > FQ_TREE_WORDS || !float_of(a[6], &scale) ||
            !ints_of(a[5], {b.seqs}, dev, false, &tail) || !optional(a[8], at::kFloat, dev, &lse) || !stream_of(a[10], &stream) ||
            (lse && !shape_is(&THPVariable_Unpack(a[8]), {tokens, width / 128})))
            return false;
        const void *px = q->data_ptr(), *pm = mask->data_ptr();
        const int words = (int)mask->size(1);
        void *po = out->data_ptr(), *pw = ws ? ws->data_ptr() : nullptr;
        const size_t bytes = ws ? (size_t)ws->numel() : 0;
        *rc = without_gil([&] {
            return entry.attn_tree(&b, static_cast<const uint64_t *>(pm), words, static_cast<const int32_t *>(tail), px, ldq, (int)(width / 128), (int)kv, pk, pv,
                                   scale, po, static_cast<float *>(const_cast<void *>(lse)), pw, bytes, stream);
        });
        return !(*rc == FQ_ERR_WORKSPACE && !ws); // none given: the long way makes one
    });
}

// batch, k_pages, v_pages, parents, drafted, following, tail, path, accepted, bonus, new_len, stream
PyObject *tree_commit(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 12, [&](int *rc) {
        fq_paged_batch b;
        const at::Tensor *k = device_tensor(a[1], at::kHalf), *v = device_tensor(a[2], at::kHalf), *path = device_tensor(a[7], at::kInt);
        void *stream;
        if (!k || !v || !path || k->dim() != 5 || v->sizes() != k->sizes() || v->device() != k->device() || path->device() != k->device() ||
            !is_current(k->device()) || !batch_of(a[0], k->device(), &b) || !stream_of(a[11], &stream))
            return false;
        const c10::Device dev = k->device();
        const void *parents, *drafted, *following, *tail, *accepted, *bonus, *len;
        if (!shape_is(k, {-1, b.pages, -1, b.page, 128}) || k->size(0) > INT_MAX || k->size(2) > INT_MAX || !shape_is(path, {b.seqs, -1}) ||
            path->size(1) < 1 || path->size(1) > INT_MAX || !ints_of(a[3], {b.tokens}, dev, false, &parents) ||
            !ints_of(a[4], {b.tokens}, dev, false, &drafted) || !ints_of(a[5], {b.tokens}, dev, false, &following) ||
            !ints_of(a[6], {b.seqs}, dev, false, &tail) || !ints_of(a[8], {b.seqs}, dev, true, &accepted) ||
            !ints_of(a[9], {b.seqs}, dev, a[3] != Py_None, &bonus) || !ints_of(a[10], {b.seqs}, dev, true, &len) ||
            (parents != nullptr) != (drafted != nullptr) || (parents != nullptr) != (following != nullptr) || b.tokens == 0)
            return false;
        const auto in = [](const void *p) { return static_cast<const int32_t *>(p); };
        const auto out = [](const void *p) { return static_cast<int32_t *>(const_cast<void *>(p)); };
        void *pk = k->data_ptr(), *pv = v->data_ptr(), *pp = path->data_ptr();
        *rc = without_gil([&] {
            return entry.commit(&b, in(tail), in(parents), in(drafted), in(following), pk, pv, (int)k->size(0), (int)k->size(2), out(pp),
                                (int)path->size(1), out(accepted), out(bonus), out(len), stream);
        });
        return true;
    });
}

// logits, scores, width, done, eos, mask, tail, parent, token, scores_out, done_out, mask_out, workspace, stream
PyObject *beam_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 14, [&](int *rc) {
        const at::Tensor *scores = device_tensor(a[1], at::kFloat), *out = device_tensor(a[9], at::kFloat), *ws = device_tensor(a[12], at::kByte);
        int width, eos;
        void *stream;
        if (!scores || scores->dim() != 2 || !out || !ws || !is_current(scores->device()) || !int_of(a[2], &width) || !int_of(a[4], &eos) ||
            !stream_of(a[13], &stream) || !THPVariable_CheckExact(a[0]))
            return false;
        const c10::Device dev = scores->device();
        const at::Tensor &x = THPVariable_Unpack(a[0]);
        const int64_t requests = scores->size(0), beams = scores->size(1);
        if (requests < 1 || beams < 1 || requests > INT_MAX || beams > 64 || !x.is_cuda() || x.device() != dev || x.scalar_type() != at::kHalf || x.dim() != 2 ||
            x.size(0) != requests * beams || x.size(1) < 2 || x.size(1) > INT_MAX || x.stride(1) != 1 || x.stride(0) < 0 || out->device() != dev ||
            ws->device() != dev || !shape_is(out, {requests, width}))
            return false;
        const int64_t ld = x.size(0) > 1 ? x.stride(0) : x.size(1);
        const void *done, *tail, *parent, *token, *done_out, *mask, *mask_out;
        if (!ints_of(a[3], {requests, beams}, dev, false, &done) || !ints_of(a[6], {requests}, dev, false, &tail) ||
            !ints_of(a[7], {requests, width}, dev, true, &parent) || !ints_of(a[8], {requests, width}, dev, true, &token) ||
            !ints_of(a[10], {requests, width}, dev, done || eos >= 0, &done_out) || !optional(a[5], at::kLong, dev, &mask) ||
            !optional(a[11], at::kLong, dev, &mask_out) || (mask && !mask_out))
            return false;
        int64_t words = 0;
        if (mask_out) {
            const at::Tensor &m = THPVariable_Unpack(a[11]);
            if (!shape_is(&m, {requests, width, -1}))
                return false;
            words = m.size(2);
            if (words < 1 || words > FQ_TREE_WORDS || (mask && !shape_is(&THPVariable_Unpack(a[5]), {requests, beams, words})))
                return false;
        }
        const auto in = [](const void *p) { return static_cast<const int32_t *>(p); };
        const auto ints = [](const void *p) { return static_cast<int32_t *>(const_cast<void *>(p)); };
        const void *px = x.data_ptr();
        const float *ps = static_cast<const float *>(scores->data_ptr());
        float *po = static_cast<float *>(out->data_ptr());
        void *pw = ws->data_ptr();
        const size_t bytes = (size_t)ws->numel();
        *rc = without_gil([&] {
            return entry.beam(px, ld, ps, in(done), eos, (int)requests, (int)beams, (int)x.size(1), width, ints(parent), ints(token), po, ints(done_out),
                              static_cast<const uint64_t *>(mask), static_cast<uint64_t *>(const_cast<void *>(mask_out)), (int)words, in(tail), pw, bytes,
                              stream);
        });
        return true;
    });
}

// Addresses of the entry points, in the order of Entries: the first nine, and those over trees of tokens.
PyObject *bind(PyObject *, PyObject *args)
{
    unsigned long long p[9];
    if (!PyArg_ParseTuple(args, "KKKKKKKKK", &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &p[6], &p[7], &p[8]))
        return nullptr;
    entry.qlinear = reinterpret_cast<decltype(entry.qlinear)>(p[0]);
    entry.mixed = reinterpret_cast<decltype(entry.mixed)>(p[1]);
    entry.dense = reinterpret_cast<decltype(entry.dense)>(p[2]);
    entry.head_nll = reinterpret_cast<decltype(entry.head_nll)>(p[3]);
    entry.token_nll = reinterpret_cast<decltype(entry.token_nll)>(p[4]);
    entry.logit_l2 = reinterpret_cast<decltype(entry.logit_l2)>(p[5]);
    entry.norm_rope = reinterpret_cast<decltype(entry.norm_rope)>(p[6]);
    entry.attn_paged = reinterpret_cast<decltype(entry.attn_paged)>(p[7]);
    entry.evict = reinterpret_cast<decltype(entry.evict)>(p[8]);
    Py_RETURN_NONE;
}

PyObject *bind_trees(PyObject *, PyObject *args)
{
    unsigned long long p[4];
    if (!PyArg_ParseTuple(args, "KKKK", &p[0], &p[1], &p[2], &p[3]))
        return nullptr;
    entry.plan = reinterpret_cast<decltype(entry.plan)>(p[0]);
    entry.attn_tree = reinterpret_cast<decltype(entry.attn_tree)>(p[1]);
    entry.commit = reinterpret_cast<decltype(entry.commit)>(p[2]);
    entry.beam = reinterpret_cast<decltype(entry.beam)>(p[3]);
    Py_RETURN_NONE;
}

#define FQ_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FQ_FAST(qlinear),   FQ_FAST(mixed),    FQ_FAST(dense_f16), FQ_FAST(head_nll),
                         FQ_FAST(token_nll), FQ_FAST(logit_l2), FQ_FAST(qk_norm_rope), FQ_FAST(attn_paged), FQ_FAST(cache_evict),
                         FQ_FAST(paged_plan), FQ_FAST(attn_tree), FQ_FAST(tree_commit), FQ_FAST(beam_step), {"bind", bind, METH_VARARGS, nullptr},
                         {"bind_trees", bind_trees, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__bind()
{
    s_packed = PyUnicode_InternFromString("packed");
    s_scales = PyUnicode_InternFromString("scales");
    s_zeros = PyUnicode_InternFromString("zeros");
    s_n = PyUnicode_InternFromString("N");
    s_k = PyUnicode_InternFromString("K");
    s_bits = PyUnicode_InternFromString("bits");
    s_struct = PyUnicode_InternFromString("struct");
    s_positions = PyUnicode_InternFromString("positions");
    s_slots = PyUnicode_InternFromString("slots");
    s_q_start = PyUnicode_InternFromString("q_start");
    s_seq_len = PyUnicode_InternFromString("seq_len");
    s_table = PyUnicode_InternFromString("table");
    s_held = PyUnicode_InternFromString("held");
    s_free_pages = PyUnicode_InternFromString("free_pages");
    s_free_count = PyUnicode_InternFromString("free_count");
    s_lacking = PyUnicode_InternFromString("lacking");
    s_mask = PyUnicode_InternFromString("mask");
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", FQ_TORCH_VERSION) != 0) { // tensors are read by this version's layout
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
