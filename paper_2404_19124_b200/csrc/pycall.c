/* The calls of a decoding step, marshalled natively.  Small calls are bound by the host: spec_verify of
 * a small problem took 7.4 us with the tensor checks in Python and a ctypes call of 13 arguments, 4.9 so; in two kernels
 * 9.5 and 6.8.  Each function here
 * looks at its tensors (device, type, contiguity, shape) and calls the library through the address it was given; on
 * anything out of the ordinary it returns None and touches nothing: the caller then goes through its own checks, which know
 * what to say.  The interpreter's lock is released around the call.  The calls around a tree of drafted tokens took 11 (plan,
 * tables) to 20 us (attention) with their checks in Python. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "spec_b200.h"

typedef int (*verify_fn)(const int32_t *, const void *, int, int, int, int, int, int32_t *, int32_t *, int32_t *, void *,
                         size_t, void *);
typedef int (*next_ctx_fn)(const void *, const int32_t *, const int32_t *, int, int, int, int, void *, int32_t *, void *);
typedef int (*draft_fn)(spec_handle_t, const void *, const int32_t *, int, const int32_t *, int, int32_t *, float *, void *,
                        size_t, void *);
static verify_fn f_verify, f_verify_early;
static next_ctx_fn f_next_ctx;
static draft_fn f_draft;
static PyObject *t_i32, *t_bf16, *t_f32;   /* torch dtypes */
static PyObject *get_device, *get_raw_stream;   /* of the current device */
static PyObject *s_cuda_stream, *s_is_cuda, *s_dtype, *s_is_contiguous, *s_shape, *s_data_ptr, *s_numel, *s_get_device;

/* Contiguous CUDA tensor of `dtype` (null: bf16 or fp32, which is told in *bf16): fills `dim` with its nd sizes. */
static int look(PyObject *t, PyObject *dtype, int nd, long long *dim, uintptr_t *ptr, int *bf16) {
    int ok = 0;
    PyObject *o = PyObject_GetAttr(t, s_is_cuda);
    if (!o) return 0;
    ok = o == Py_True;
    Py_DECREF(o);
    if (!ok || !(o = PyObject_GetAttr(t, s_dtype))) return 0;
    ok = dtype ? o == dtype : (o == t_bf16 || o == t_f32);
    if (bf16) *bf16 = o == t_bf16;
    Py_DECREF(o);
    if (!ok || !(o = PyObject_CallMethodNoArgs(t, s_is_contiguous))) return 0;
    ok = o == Py_True;
    Py_DECREF(o);
    if (!ok || !(o = PyObject_GetAttr(t, s_shape))) return 0;
    ok = PyTuple_Check(o) && PyTuple_GET_SIZE(o) == nd;
    for (int i = 0; ok && i < nd; ++i) {
        dim[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
        ok = dim[i] > 0 && dim[i] <= INT32_MAX;
    }
    Py_DECREF(o);
    if (!ok || !(o = PyObject_CallMethodNoArgs(t, s_data_ptr))) return 0;
    *ptr = (uintptr_t)PyLong_AsUnsignedLongLong(o);
    Py_DECREF(o);
    return !PyErr_Occurred();
}

static int number(PyObject *t, PyObject *method, long long *out) {
    PyObject *o = PyObject_CallMethodNoArgs(t, method);
    if (!o) return 0;
    *out = PyLong_AsLongLong(o);
    Py_DECREF(o);
    return !PyErr_Occurred();
}

static int bytes_of(PyObject *t, uintptr_t *ptr, long long *n) {   /* a workspace: its address and elements */
    PyObject *o = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!o) return 0;
    *ptr = (uintptr_t)PyLong_AsUnsignedLongLong(o);
    Py_DECREF(o);
    return !PyErr_Occurred() && number(t, s_numel, n);
}

static int vec_i32(PyObject *t, long long n, uintptr_t *ptr) {
    long long d[1];
    return look(t, t_i32, 1, d, ptr, NULL) && d[0] == n;
}

static int stream_of(PyObject *stream, uintptr_t *st) {   /* a stream object, or None: the current one */
    PyObject *o, *dev;
    if (stream != Py_None) {
        o = PyObject_GetAttr(stream, s_cuda_stream);
    } else {
        if (!(dev = PyObject_CallNoArgs(get_device))) return 0;
        o = PyObject_CallOneArg(get_raw_stream, dev);
        Py_DECREF(dev);
    }
    if (!o) return 0;
    *st = (uintptr_t)PyLong_AsUnsignedLongLong(o);
    Py_DECREF(o);
    return !PyErr_Occurred();
}

static PyObject *unusual(void) {
    PyErr_Clear();
    Py_RETURN_NONE;
}

/* verify(cand_tok, base_logits, accept_len, best_cand, next_tok, workspace, stream, early) -> status or None */
static PyObject *py_verify(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    long long c[3], l[4], wn;
    uintptr_t pc, pl, pa, pb, pn, pw, st;
    int bf16 = 0, status;
    if (n != 8 || !look(a[0], t_i32, 3, c, &pc, NULL) || !look(a[1], NULL, 4, l, &pl, &bf16) || l[0] != c[0] || l[1] != c[1] ||
        l[2] != c[2] + 1 || !vec_i32(a[2], c[0], &pa) || !vec_i32(a[3], c[0], &pb) || !vec_i32(a[4], c[0], &pn) ||
        !bytes_of(a[5], &pw, &wn) || !stream_of(a[6], &st))
        return unusual();
    const int early = PyObject_IsTrue(a[7]);
    if (early < 0) return unusual();
    const verify_fn f = early ? f_verify_early : f_verify;
    Py_BEGIN_ALLOW_THREADS
    status = f((const int32_t *)pc, (const void *)pl, bf16 ? SPEC_BF16 : SPEC_F32, (int)c[0], (int)c[1], (int)c[2], (int)l[3],
               (int32_t *)pa, (int32_t *)pb, (int32_t *)pn, (void *)pw, (size_t)wn, (void *)st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* next_ctx(base_state, best_cand, accept_len, ctx_state, err_workspace, stream) -> status or None */
static PyObject *py_next_ctx(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    long long s[4], x[2], on;
    PyObject *dev;
    uintptr_t ps, pb, pa, px, pe = 0, st;
    int status;
    if (n != 6 || !look(a[0], t_bf16, 4, s, &ps, NULL) || !vec_i32(a[1], s[0], &pb) || !vec_i32(a[2], s[0], &pa) ||
        !look(a[3], t_bf16, 2, x, &px, NULL) || x[0] != s[0] || x[1] != s[3] ||
        !number(a[0], s_get_device, &on) || !(dev = PyObject_CallNoArgs(get_device)))
        return unusual();
    const int here = PyLong_AsLongLong(dev) == on;   /* the tensors' device is current */
    Py_DECREF(dev);
    if (!here || !stream_of(a[5], &st)) return unusual();
    if (a[4] != Py_None) {
        PyObject *o = PyObject_CallMethodNoArgs(a[4], s_data_ptr);
        if (!o) return unusual();
        pe = (uintptr_t)PyLong_AsUnsignedLongLong(o);
        Py_DECREF(o);
        if (PyErr_Occurred()) return unusual();
    }
    Py_BEGIN_ALLOW_THREADS
    status = f_next_ctx((const void *)ps, (const int32_t *)pb, (const int32_t *)pa, (int)s[0], (int)s[1], (int)s[2] - 1,
                        (int)s[3], (void *)px, (int32_t *)pe, (void *)st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* draft(handle, n_heads, d_base, ctx_state, last_tok, topk, K, cand_tok, cand_logp, workspace, stream) -> status or None */
static PyObject *py_draft(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    long long x[2], c[3], p[2], wn;
    uintptr_t h, px, pt, pc, pp, pw, st;
    int32_t topk[SPEC_MAX_HEADS];
    int status;
    if (n != 11 || !PyTuple_CheckExact(a[5])) return unusual();
    h = (uintptr_t)PyLong_AsUnsignedLongLong(a[0]);
    const long long heads = PyLong_AsLongLong(a[1]), d_base = PyLong_AsLongLong(a[2]), K = PyLong_AsLongLong(a[6]);
    if (PyErr_Occurred() || heads < 1 || heads > SPEC_MAX_HEADS || PyTuple_GET_SIZE(a[5]) != heads || K < 1 || K > INT32_MAX ||
        !look(a[3], t_bf16, 2, x, &px, NULL) || x[1] != d_base || !vec_i32(a[4], x[0], &pt) ||
        !look(a[7], t_i32, 3, c, &pc, NULL) || c[0] != x[0] || c[1] != K || c[2] != heads ||
        !look(a[8], t_f32, 2, p, &pp, NULL) || p[0] != x[0] || p[1] != K || !bytes_of(a[9], &pw, &wn))
        return unusual();
    for (int l = 0; l < heads; ++l) {
        const long long k = PyLong_AsLongLong(PyTuple_GET_ITEM(a[5], l));
        if (k < 0 || k > INT32_MAX) return unusual();
        topk[l] = (int32_t)k;
    }
    if (PyErr_Occurred() || !stream_of(a[10], &st)) return unusual();
    Py_BEGIN_ALLOW_THREADS
    status = f_draft((spec_handle_t)h, (const void *)px, (const int32_t *)pt, (int)x[0], topk, (int)K, (int32_t *)pc,
                     (float *)pp, (void *)pw, (size_t)wn, (void *)st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* ---- the base model's forward pass over a tree of drafted tokens ---- */
typedef int (*plan_fn)(const int32_t *, const int32_t *, const int32_t *, int, int, int, int, int32_t *, int32_t *, int32_t *,
                       uint32_t *, int32_t *, int32_t *, void *);
typedef int (*tables_fn)(const int32_t *, const int32_t *, int, int, int, int32_t *, int64_t, int, const int32_t *,
                         const int32_t *, const int32_t *, int, int64_t *, int32_t *, int32_t *, int32_t *, void *);
typedef int (*attention_fn)(const spec_tree_attention_t *, void *, size_t, void *);
typedef int (*tree_verify_fn)(const spec_tree_verify_t *, void *);
typedef int (*commit_fn)(const spec_kv_commit_t *, void *);
static plan_fn f_plan;
static tables_fn f_tables;
static attention_fn f_attention;
static tree_verify_fn f_tree_verify;
static commit_fn f_commit;
static PyObject *t_f16, *t_i64, *s_stride, *s_itemsize;

static int current(long long *dev) {
    PyObject *o = PyObject_CallNoArgs(get_device);
    if (!o) return 0;
    *dev = PyLong_AsLongLong(o);
    Py_DECREF(o);
    return !PyErr_Occurred();
}

/* Contiguous tensor of that type on device `dev` with these sizes; None (if allowed) is a null pointer. */
static int dense(PyObject *t, PyObject *dtype, long long dev, int nd, const long long *want, int none, void *ptr) {
    long long d[5], on;
    uintptr_t p = 0;
    if (t == Py_None) {
        if (!none) return 0;
    } else {
        if (!look(t, dtype, nd, d, &p, NULL) || !number(t, s_get_device, &on) || on != dev) return 0;
        for (int i = 0; i < nd; ++i)
            if (d[i] != want[i]) return 0;
    }
    *(uintptr_t *)ptr = p;
    return 1;
}
static int vector(PyObject *t, PyObject *dtype, long long dev, long long n, int none, void *ptr) {
    return dense(t, dtype, dev, 1, &n, none, ptr);
}

/* Tensor of that type on device `dev`, dense in its last dimension: sizes, and strides of the other dimensions (0 for one entry).
 * `want`: sizes it must have, or null.  A written tensor has no stride of 0 elsewhere. */
static int strided(PyObject *t, PyObject *dtype, long long dev, int nd, const long long *want, int written, long long *dim,
                   int64_t *stride, void *ptr) {
    long long on;
    int ok = 0;
    PyObject *o = PyObject_GetAttr(t, s_is_cuda);
    if (!o) return 0;
    ok = o == Py_True;
    Py_DECREF(o);
    if (!ok || !number(t, s_get_device, &on) || on != dev || !(o = PyObject_GetAttr(t, s_dtype))) return 0;
    ok = o == dtype;
    Py_DECREF(o);
    if (!ok || !(o = PyObject_GetAttr(t, s_shape))) return 0;
    ok = PyTuple_Check(o) && PyTuple_GET_SIZE(o) == nd;
    for (int i = 0; ok && i < nd; ++i) {
        dim[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
        ok = dim[i] > 0 && dim[i] <= INT32_MAX && (!want || dim[i] == want[i]);
    }
    Py_DECREF(o);
    if (!ok || !(o = PyObject_CallMethodNoArgs(t, s_stride))) return 0;
    ok = PyTuple_Check(o) && PyTuple_GET_SIZE(o) == nd;
    for (int i = 0; ok && i < nd; ++i) {
        const long long s = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
        if (i == nd - 1) {
            ok = s == 1 || dim[i] == 1;
        } else {
            stride[i] = dim[i] == 1 ? 0 : s;
            ok = !written || stride[i] != 0 || dim[i] == 1;
        }
    }
    Py_DECREF(o);
    if (!ok || PyErr_Occurred() || !(o = PyObject_CallMethodNoArgs(t, s_data_ptr))) return 0;
    *(uintptr_t *)ptr = (uintptr_t)PyLong_AsUnsignedLongLong(o);
    Py_DECREF(o);
    return !PyErr_Occurred();
}

/* An int32 word on device `dev` in a tensor of any type, or None: a null pointer. */
static int error_word(PyObject *t, long long dev, int32_t **err) {
    uintptr_t p = 0;
    long long n, on, size;
    PyObject *o;
    if (t != Py_None) {
        if (!bytes_of(t, &p, &n) || !number(t, s_get_device, &on) || on != dev || p % 4 || !(o = PyObject_GetAttr(t, s_itemsize))) return 0;
        size = PyLong_AsLongLong(o);
        Py_DECREF(o);
        if (PyErr_Occurred() || n * size < 4) return 0;
    }
    *err = (int32_t *)p;
    return 1;
}

/* the stream object's device is left to the Python checks */
static int own_stream(PyObject *stream, uintptr_t *st) { return stream == Py_None && stream_of(stream, st); }

/* tree_plan(cand_tok, last_tok, seq_len, T, tok, pos, parent, mask, node_of, n_nodes, stream) -> status or None */
static PyObject *py_tree_plan(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    long long c[3], dev, on;
    uintptr_t pc, st;
    int32_t *last, *len, *tok, *pos, *parent, *node_of, *nodes;
    uint32_t *mask;
    int status;
    if (n != 11 || !current(&dev) || !look(a[0], t_i32, 3, c, &pc, NULL) || !number(a[0], s_get_device, &on) || on != dev)
        return unusual();
    const long long T = PyLong_AsLongLong(a[3]);
    if (PyErr_Occurred() || T < 1 || T > SPEC_MAX_TREE_NODES) return unusual();
    const long long bt[2] = {c[0], T}, m[3] = {c[0], T, (T + 31) / 32}, k[3] = {c[0], c[1], c[2] + 1};
    if (!vector(a[1], t_i32, dev, c[0], 0, &last) || !vector(a[2], t_i32, dev, c[0], 0, &len) ||
        !dense(a[4], t_i32, dev, 2, bt, 0, &tok) || !dense(a[5], t_i32, dev, 2, bt, 0, &pos) ||
        !dense(a[6], t_i32, dev, 2, bt, 0, &parent) || !dense(a[7], t_i32, dev, 3, m, 0, &mask) ||
        !dense(a[8], t_i32, dev, 3, k, 0, &node_of) || !vector(a[9], t_i32, dev, c[0], 0, &nodes) || !own_stream(a[10], &st))
        return unusual();
    Py_BEGIN_ALLOW_THREADS
    status = f_plan((const int32_t *)pc, last, len, (int)c[0], (int)c[1], (int)c[2], (int)T, tok, pos, parent, mask, node_of, nodes,
                    (void *)st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* page_tables(seq_len, n_new, block_table, n_pages, free_pages, free_count, page_size, slots, n_pages_out, free_count_out, err_workspace,
 * stream) */
static PyObject *py_page_tables(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    long long b[1], t[2], f[1], s[2], dev, on;
    int64_t stride[1], *ps;
    uintptr_t pl, pslots, pf, st;
    int32_t *fresh, *table, *held, *count, *held_out, *count_out, *err;
    int status;
    if (n != 12 || !current(&dev) || !look(a[0], t_i32, 1, b, &pl, NULL) || !number(a[0], s_get_device, &on) || on != dev ||
        !vector(a[1], t_i32, dev, b[0], 1, &fresh) || !strided(a[2], t_i32, dev, 2, NULL, 1, t, stride, &table) || t[0] != b[0] ||
        !vector(a[3], t_i32, dev, b[0], 0, &held) || !look(a[4], t_i32, 1, f, &pf, NULL) || !number(a[4], s_get_device, &on) ||
        on != dev || !vector(a[5], t_i32, dev, 1, 0, &count) || !look(a[7], t_i64, 2, s, &pslots, NULL) ||
        !number(a[7], s_get_device, &on) || on != dev || s[0] != b[0] || !vector(a[8], t_i32, dev, b[0], 0, &held_out) ||
        !vector(a[9], t_i32, dev, 1, 0, &count_out) || !error_word(a[10], dev, &err) || !own_stream(a[11], &st))
        return unusual();
    const long long page = PyLong_AsLongLong(a[6]);
    if (PyErr_Occurred() || page < 1 || page > INT32_MAX) return unusual();
    ps = (int64_t *)pslots;
    Py_BEGIN_ALLOW_THREADS
    status = f_tables((const int32_t *)pl, fresh, (int)b[0], (int)page, (int)s[1], table, stride[0] ? stride[0] : t[1], (int)t[1],
                      held, (const int32_t *)pf, count, (int)f[0], ps, held_out, count_out, err, (void *)st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* tree_attention(q, k, v, k_cache, v_cache, block_table, seq_len, mask, n_nodes, scale, out, lse, workspace, err_workspace,
 * stream) */
static PyObject *py_tree_attention(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    spec_tree_attention_t x;
    long long q[4], d[4], c[4], t[2], dev, on, wn;
    int64_t ts[1];
    uintptr_t pw, st;
    PyObject *dtype;
    int status;
    memset(&x, 0, sizeof x);
    if (n != 15 || !current(&dev) || !(dtype = PyObject_GetAttr(a[0], s_dtype))) return unusual();
    Py_DECREF(dtype);                                   /* the dtype objects live as long as torch */
    if (dtype != t_bf16 && dtype != t_f16) return unusual();
    x.dtype = dtype == t_bf16 ? SPEC_BF16 : SPEC_F16;
    if (!strided(a[0], dtype, dev, 4, NULL, 0, q, x.q_stride, &x.q) || !strided(a[1], dtype, dev, 4, NULL, 0, d, x.k_stride, &x.k) ||
        d[0] != q[0] || d[1] != q[1] || d[3] != q[3])
        return unusual();
    const long long kv[4] = {d[0], d[1], d[2], d[3]};
    if (!strided(a[2], dtype, dev, 4, kv, 0, d, x.v_stride, &x.v) || !strided(a[3], dtype, dev, 4, NULL, 0, c, x.kc_stride, &x.k_cache) ||
        c[2] != kv[2] || c[3] != kv[3])
        return unusual();
    const long long cache[4] = {c[0], c[1], c[2], c[3]}, m[3] = {q[0], q[1], (q[1] + 31) / 32};
    if (!strided(a[4], dtype, dev, 4, cache, 0, c, x.vc_stride, &x.v_cache) ||
        !strided(a[5], t_i32, dev, 2, NULL, 0, t, ts, &x.block_table) || t[0] != q[0] ||
        !vector(a[6], t_i32, dev, q[0], 0, &x.seq_len) || !dense(a[7], t_i32, dev, 3, m, 1, &x.mask) ||
        !vector(a[8], t_i32, dev, q[0], 1, &x.n_nodes) || !strided(a[10], dtype, dev, 4, q, 1, d, x.out_stride, &x.out) ||
        !dense(a[11], t_f32, dev, 3, q, 1, &x.lse) || !bytes_of(a[12], &pw, &wn) || !number(a[12], s_get_device, &on) || on != dev)
        return unusual();
    PyObject *size = PyObject_GetAttr(a[12], s_itemsize);
    if (!size) return unusual();
    wn *= PyLong_AsLongLong(size);
    Py_DECREF(size);
    x.scale = (float)PyFloat_AsDouble(a[9]);
    if (PyErr_Occurred() || !error_word(a[13], dev, &x.err_word) || !own_stream(a[14], &st)) return unusual();
    x.B = (int)q[0], x.T = (int)q[1], x.Hq = (int)q[2], x.D = (int)q[3], x.Hkv = (int)kv[2];
    x.n_pages = (int)cache[0], x.page_size = (int)cache[1], x.max_pages = (int)t[1];
    x.table_stride = q[0] > 1 ? ts[0] : t[1];
    Py_BEGIN_ALLOW_THREADS
    status = f_attention(&x, (void *)pw, (size_t)wn, (void *)st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* verify_tree(tok, parent, n_nodes, logits, hist_tok, hist_len, prompt_len, repetition, frequency, presence, bias_tok, bias_val,
 * bias_len, allow, accept_len, last_node, next_tok, path, stream) */
static PyObject *py_verify_tree(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    spec_tree_verify_t x;
    long long l[3], d[2], p[2], dev;
    uintptr_t at, st;
    PyObject *dtype;
    int status;
    memset(&x, 0, sizeof x);
    if (n != 19 || !current(&dev) || !(dtype = PyObject_GetAttr(a[3], s_dtype))) return unusual();
    Py_DECREF(dtype);
    if (dtype != t_bf16 && dtype != t_f16 && dtype != t_f32) return unusual();
    x.logits_dtype = dtype == t_bf16 ? SPEC_BF16 : dtype == t_f16 ? SPEC_F16 : SPEC_F32;
    if (!strided(a[3], dtype, dev, 3, NULL, 0, l, x.logits_stride, &x.logits)) return unusual();
    const long long B = l[0], bt[2] = {B, l[1]}, words[3] = {B, l[1], (l[2] + 31) / 32};
    if (!dense(a[0], t_i32, dev, 2, bt, 0, &x.tok) || !dense(a[1], t_i32, dev, 2, bt, 0, &x.parent) ||
        !vector(a[2], t_i32, dev, B, 0, &x.n_nodes) || !look(a[17], t_i32, 2, p, &at, NULL) || p[0] != B)
        return unusual();
    if (a[4] != Py_None) {
        if (!look(a[4], t_i32, 2, d, &at, NULL) || d[0] != B || !dense(a[4], t_i32, dev, 2, d, 0, &x.hist_tok)) return unusual();
        x.max_hist = (int)d[1];
    }
    if (a[10] != Py_None) {
        if (!look(a[10], t_i32, 2, d, &at, NULL) || d[0] != B || !dense(a[10], t_i32, dev, 2, d, 0, &x.bias_tok) ||
            !dense(a[11], t_f32, dev, 2, d, 0, &x.bias_val))
            return unusual();
        x.max_bias = (int)d[1];
    } else if (a[11] != Py_None) {
        return unusual();
    }
    if (!vector(a[5], t_i32, dev, B, 1, &x.hist_len) || !vector(a[6], t_i32, dev, B, 1, &x.prompt_len) ||
        !vector(a[7], t_f32, dev, B, 1, &x.repetition) || !vector(a[8], t_f32, dev, B, 1, &x.frequency) ||
        !vector(a[9], t_f32, dev, B, 1, &x.presence) || !vector(a[12], t_i32, dev, B, 1, &x.bias_len) ||
        !dense(a[13], t_i32, dev, 3, words, 1, &x.allow) || !vector(a[14], t_i32, dev, B, 0, &x.accept_len) ||
        !vector(a[15], t_i32, dev, B, 0, &x.last_node) || !vector(a[16], t_i32, dev, B, 0, &x.next_tok) ||
        !dense(a[17], t_i32, dev, 2, p, 0, &x.path) || !own_stream(a[18], &st))
        return unusual();
    x.B = (int)B, x.T = (int)l[1], x.V = (int)l[2], x.n = (int)p[1] - 1;
    Py_BEGIN_ALLOW_THREADS
    status = f_tree_verify(&x, (void *)st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* kv_commit(k, v, k_cache, v_cache, path, accept_len, slots, seq_len, new_len, err_workspace, stream) */
static PyObject *py_kv_commit(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    spec_kv_commit_t x;
    long long k[5], c[5], d[5], p[2], dev;
    uintptr_t at, st;
    PyObject *dtype;
    int status;
    memset(&x, 0, sizeof x);
    if (n != 11 || !current(&dev) || !(dtype = PyObject_GetAttr(a[0], s_dtype))) return unusual();
    Py_DECREF(dtype);
    if (dtype != t_bf16 && dtype != t_f16) return unusual();
    if (!strided(a[0], dtype, dev, 5, NULL, 0, k, x.k_stride, &x.k) || !strided(a[1], dtype, dev, 5, k, 0, d, x.v_stride, &x.v) ||
        !strided(a[2], dtype, dev, 5, NULL, 1, c, x.kc_stride, &x.k_cache) || c[0] != k[0] || c[3] != k[3] || c[4] != k[4] ||
        !strided(a[3], dtype, dev, 5, c, 1, d, x.vc_stride, &x.v_cache) || !look(a[4], t_i32, 2, p, &at, NULL) || p[0] != k[1] ||
        !dense(a[4], t_i32, dev, 2, p, 0, &x.path) || !vector(a[5], t_i32, dev, k[1], 0, &x.accept_len) ||
        !dense(a[6], t_i64, dev, 2, p, 0, &x.slots) || !vector(a[7], t_i32, dev, k[1], 1, &x.seq_len) ||
        !vector(a[8], t_i32, dev, k[1], 1, &x.new_len) || !error_word(a[9], dev, &x.err_word) || !own_stream(a[10], &st))
        return unusual();
    x.L = (int)k[0], x.B = (int)k[1], x.T = (int)k[2], x.n = (int)p[1] - 1, x.H = (int)k[3], x.D = (int)k[4];
    x.n_pages = (int)c[1], x.page_size = (int)c[2];
    Py_BEGIN_ALLOW_THREADS
    status = f_commit(&x, (void *)st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* bind_tree(spec_tree_plan, spec_page_tables, spec_tree_attention, spec_verify_tree, spec_kv_commit, float16, int64): after bind */
static PyObject *py_bind_tree(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "bind_tree() takes five addresses and two dtypes");
        return NULL;
    }
    f_plan = (plan_fn)(uintptr_t)PyLong_AsUnsignedLongLong(a[0]);
    f_tables = (tables_fn)(uintptr_t)PyLong_AsUnsignedLongLong(a[1]);
    f_attention = (attention_fn)(uintptr_t)PyLong_AsUnsignedLongLong(a[2]);
    f_tree_verify = (tree_verify_fn)(uintptr_t)PyLong_AsUnsignedLongLong(a[3]);
    f_commit = (commit_fn)(uintptr_t)PyLong_AsUnsignedLongLong(a[4]);
    if (PyErr_Occurred()) return NULL;
    Py_XSETREF(t_f16, Py_NewRef(a[5]));
    Py_XSETREF(t_i64, Py_NewRef(a[6]));
    Py_RETURN_NONE;
}

/* bind(spec_verify, spec_verify_early, spec_next_ctx, spec_draft, int32, bfloat16, float32, get_device, get_raw_stream): addresses, dtypes
 * and the callables that tell the current device and its current stream */
static PyObject *py_bind(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) {
        PyErr_SetString(PyExc_TypeError, "bind() takes four addresses, three dtypes and two callables");
        return NULL;
    }
    f_verify = (verify_fn)(uintptr_t)PyLong_AsUnsignedLongLong(a[0]);
    f_verify_early = (verify_fn)(uintptr_t)PyLong_AsUnsignedLongLong(a[1]);
    f_next_ctx = (next_ctx_fn)(uintptr_t)PyLong_AsUnsignedLongLong(a[2]);
    f_draft = (draft_fn)(uintptr_t)PyLong_AsUnsignedLongLong(a[3]);
    if (PyErr_Occurred()) return NULL;
    Py_XSETREF(t_i32, Py_NewRef(a[4]));
    Py_XSETREF(t_bf16, Py_NewRef(a[5]));
    Py_XSETREF(t_f32, Py_NewRef(a[6]));
    Py_XSETREF(get_device, Py_NewRef(a[7]));
    Py_XSETREF(get_raw_stream, Py_NewRef(a[8]));
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"bind", (PyCFunction)(void (*)(void))py_bind, METH_FASTCALL, NULL},
                                {"verify", (PyCFunction)(void (*)(void))py_verify, METH_FASTCALL, NULL},
                                {"next_ctx", (PyCFunction)(void (*)(void))py_next_ctx, METH_FASTCALL, NULL},
                                {"draft", (PyCFunction)(void (*)(void))py_draft, METH_FASTCALL, NULL},
                                {"bind_tree", (PyCFunction)(void (*)(void))py_bind_tree, METH_FASTCALL, NULL},
                                {"tree_plan", (PyCFunction)(void (*)(void))py_tree_plan, METH_FASTCALL, NULL},
                                {"page_tables", (PyCFunction)(void (*)(void))py_page_tables, METH_FASTCALL, NULL},
                                {"tree_attention", (PyCFunction)(void (*)(void))py_tree_attention, METH_FASTCALL, NULL},
                                {"verify_tree", (PyCFunction)(void (*)(void))py_verify_tree, METH_FASTCALL, NULL},
                                {"kv_commit", (PyCFunction)(void (*)(void))py_kv_commit, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pycall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__pycall(void) {
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_is_cuda = PyUnicode_InternFromString("is_cuda");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_shape = PyUnicode_InternFromString("shape");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_numel = PyUnicode_InternFromString("numel");
    s_stride = PyUnicode_InternFromString("stride");
    s_itemsize = PyUnicode_InternFromString("itemsize");
    s_get_device = PyUnicode_InternFromString("get_device");
    return PyModule_Create(&module);
}
