/* The calls of binding.py whose argument marshalling costs more than their launch, in C.
 *
 * Each function takes the arguments of the binding's function of that name, makes the same checks by asking the tensors
 * the same questions, and calls the library with the GIL released, as ctypes does.  What any check would refuse, and
 * anything out of the ordinary (a tensor subclass, an integer that is none, a workspace still to be made), is answered
 * with None before anything is called: the Python code then answers it as it always did.
 *
 * What a call from Python took with the arguments marshalled there, and takes now (us): decode of four short sequences 6.9,
 * 5.5 (the kernel 4.5); kv_linear_view of 100 rows of 4096 x 1024 8.2, 5.9 (the kernel 5.8).
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "flying_kv.h"

typedef int (*decode_fn)(const void*, void*, const void*, int64_t, const int32_t*, int64_t, const int32_t*, int, int,
                         const kv_view*, float, void*, size_t, void*);
typedef int (*prefill_fn)(const void*, void*, const void*, int64_t, const int32_t*, int64_t, const int32_t*, const int32_t*,
                          int, int64_t, int, int, const kv_view*, float, void*, size_t, void*);
typedef size_t (*prefill_bytes_fn)(const kv_view*, int, int64_t, int, int);
typedef int (*linear_fn)(const void*, int64_t, const void*, int64_t, int64_t, const kv_weight_view*, void*, int64_t, int, void*,
                         size_t, void*);
typedef size_t (*linear_bytes_fn)(const kv_weight_view*, int);
typedef int (*append_fn)(void*, int64_t, const kv_view*, const void*, const void*, const int32_t*, int64_t, const int32_t*, int,
                         void*);
typedef int (*repack_fn)(void*, int64_t, const kv_view*, const kv_view*, const int32_t*, int64_t, const int32_t*, int64_t,
                         const int32_t*, int, int, void*);

typedef int (*rope_fn)(void*, int64_t, const kv_view*, const void*, int64_t, const void*, int64_t, const void*, int64_t, void*,
                       const int32_t*, int64_t, int, const float*, int, const int32_t*, int, const int32_t*, int64_t,
                       const int32_t*, const int32_t*, int, int64_t, int32_t*, int64_t, float*, int64_t, void*);
typedef int (*accept_fn)(void*, int64_t, const kv_view*, const int32_t*, int64_t, const int32_t*, const int32_t*, const int32_t*,
                         int64_t, const int32_t*, int, int32_t*, int32_t*, int64_t, float*, int64_t, void*);
typedef int (*tree_fn)(const void*, void*, const void*, int64_t, const int32_t*, int64_t, const int32_t*, const int32_t*,
                       const uint64_t*, int64_t, int, int64_t, int, int, const kv_view*, float, void*, size_t, void*);
typedef int (*weights_fn)(const void*, void*, const void*, int64_t, const int32_t*, int64_t, const int32_t*, int, int,
                          const kv_view*, float, float*, int64_t, void*, size_t, void*);
typedef int (*rope_q8_fn)(void*, float*, int, int64_t, const kv_view*, const void*, int64_t, const void*, int64_t, const void*,
                          int64_t, void*, const int32_t*, int64_t, int, const float*, int, const int32_t*, int, const int32_t*,
                          int64_t, const int32_t*, const int32_t*, int, int64_t, void*);
typedef int (*decode_q8_fn)(const void*, void*, const void*, const float*, int, int64_t, const int32_t*, int64_t, const int32_t*,
                            int, int, const kv_view*, float, void*, size_t, void*);
typedef int (*prefill_q8_fn)(const void*, void*, const void*, const float*, int, int64_t, const int32_t*, int64_t, const int32_t*,
                             const int32_t*, int, int64_t, int, int, const kv_view*, float, void*, size_t, void*);
typedef int (*repack_q8_fn)(void*, float*, int64_t, const kv_view*, const kv_view*, const int32_t*, int64_t, const int32_t*,
                            int64_t, const int32_t*, int, int, void*);

static decode_fn f_decode;
static prefill_fn f_prefill;
static prefill_bytes_fn f_prefill_bytes;
static linear_fn f_linear;
static linear_bytes_fn f_linear_bytes;
static append_fn f_append;
static repack_fn f_repack;

static rope_fn f_rope;
static accept_fn f_accept;
static tree_fn f_tree;
static weights_fn f_weights;

static rope_q8_fn f_rope_q8;
static decode_q8_fn f_decode_q8;
static prefill_q8_fn f_prefill_q8;
static repack_q8_fn f_repack_q8;

static PyObject *tensor_type, *parameter_type, *weight_view_type;   /* exact types only */
static PyObject *bf16_types, *int32_type, *uint8_type;              /* dtypes: a tuple, and two */
static PyObject *float_type, *word_types;                           /* float32; the two of 64-bit masks */
static PyObject* q8_formats;                                        /* dtype of an 8-bit cache -> its format */
static PyObject *get_device, *raw_stream, *is_capturing, *workspaces;   /* of torch._C; the binding's dict */
static PyObject *n_is_cuda, *n_dtype, *n_is_contiguous, *n_data_ptr, *n_shape, *n_stride, *n_numel, *n_element_size,
    *n_get_device, *n_cuda_stream, *n_handle, *n_value, *n_block_bytes, *n_n_q_local, *n_n_kv_local, *n_head_dim, *n_scratch,
    *n_numbers, *n_zero, *n_one;

/* All helpers return 1, or 0 where the Python code is to answer (an exception may be set then: `answer` clears it). */

static int is_tensor(PyObject* t)
{
    return (PyObject*)Py_TYPE(t) == tensor_type || (PyObject*)Py_TYPE(t) == parameter_type;
}

static int true_attr(PyObject* t, PyObject* name)
{
    PyObject* v = PyObject_GetAttr(t, name);
    const int yes = v == Py_True;
    Py_XDECREF(v);
    return yes;
}

static PyObject* ask(PyObject* t, PyObject* name, PyObject* arg)
{
    PyObject* args[3] = {NULL, t, arg};   /* (the first is the callee's to use) */
    return PyObject_VectorcallMethod(name, args + 1, (arg ? 2 : 1) | PY_VECTORCALL_ARGUMENTS_OFFSET, NULL);
}

static int to_int64(PyObject* v, int64_t* out)   /* steals v */
{
    int ok = v && PyLong_CheckExact(v);
    if (ok) {
        *out = PyLong_AsLongLong(v);
        ok = !(*out == -1 && PyErr_Occurred());
    }
    Py_XDECREF(v);
    return ok;
}

static int ask_int(PyObject* t, PyObject* name, PyObject* arg, int64_t* out) { return to_int64(ask(t, name, arg), out); }

static int int_attr(PyObject* o, PyObject* name, int64_t* out) { return to_int64(PyObject_GetAttr(o, name), out); }

static int int_arg(PyObject* v, int64_t* out)   /* that fits a C int */
{
    Py_INCREF(v);
    return to_int64(v, out) && *out >= INT32_MIN && *out <= INT32_MAX;
}

static int float_arg(PyObject* v, float* out)
{
    if (!PyFloat_CheckExact(v) && !PyLong_CheckExact(v)) return 0;
    const double d = PyFloat_AsDouble(v);
    *out = (float)d;
    return !(d == -1.0 && PyErr_Occurred());
}

static int dtype_is(PyObject* t, PyObject* want)
{
    PyObject* d = PyObject_GetAttr(t, n_dtype);
    int yes = d && d == want;
    if (d && PyTuple_CheckExact(want))
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(want); ++i) yes |= PyTuple_GET_ITEM(want, i) == d;
    Py_XDECREF(d);
    return yes;
}

static int address(PyObject* t, void** out)
{
    int64_t p;
    if (!ask_int(t, n_data_ptr, NULL, &p)) return 0;
    *out = (void*)(uintptr_t)p;
    return 1;
}

/* binding._dev */
static int dev(PyObject* t, PyObject* dtype, void** out)
{
    if (!is_tensor(t) || !true_attr(t, n_is_cuda) || !dtype_is(t, dtype)) return 0;
    PyObject* c = ask(t, n_is_contiguous, NULL);
    const int yes = c == Py_True;
    Py_XDECREF(c);
    return yes && address(t, out);
}

/* The sizes of a tensor with exactly n dimensions. */
static int sizes(PyObject* t, int n, int64_t* out)
{
    PyObject* s = is_tensor(t) ? PyObject_GetAttr(t, n_shape) : NULL;
    int ok = s && PyTuple_Check(s) && PyTuple_GET_SIZE(s) == n;
    for (int i = 0; ok && i < n; ++i) {
        PyObject* v = PyTuple_GET_ITEM(s, i);
        Py_INCREF(v);
        ok = to_int64(v, out + i);
    }
    Py_XDECREF(s);
    return ok;
}

/* binding._dev_rows, with the sizes and the row stride */
static int dev_rows(PyObject* t, PyObject* dtype, void** out, int64_t size[2], int64_t* row)
{
    int64_t s1;
    if (!sizes(t, 2, size) || !true_attr(t, n_is_cuda) || !dtype_is(t, dtype)) return 0;
    if (size[1] > 1 && !(ask_int(t, n_stride, n_one, &s1) && s1 == 1)) return 0;
    return ask_int(t, n_stride, n_zero, row) && address(t, out);
}

static int pool_blocks(PyObject* pool, int64_t block_bytes, int whole, int64_t* out)
{
    int64_t n, e;
    if (block_bytes <= 0 || !ask_int(pool, n_numel, NULL, &n) || !ask_int(pool, n_element_size, NULL, &e)) return 0;
    *out = n * e / block_bytes;
    return !whole || n * e % block_bytes == 0;
}

static int view_handle(PyObject* view, const kv_view** out)
{
    int64_t p;
    PyObject* h = PyObject_GetAttr(view, n_handle);
    const int ok = h && int_attr(h, n_value, &p);
    Py_XDECREF(h);
    if (!ok) return 0;
    *out = (const kv_view*)(uintptr_t)p;
    return p != 0;
}

/* The stream's handle: as given, or torch's current one of `device`, a new reference (the current device's: NULL). */
static int stream_handle(PyObject* stream, PyObject* device, int64_t* out)
{
    if (stream != Py_None) return int_attr(stream, n_cuda_stream, out);
    PyObject* d = device ? device : PyObject_CallNoArgs(get_device);
    PyObject* h = d ? PyObject_CallOneArg(raw_stream, d) : NULL;
    if (!device) Py_XDECREF(d);
    return to_int64(h, out);
}

/* The workspace: as given, or the binding's own of that device and stream where it is large enough and no graph is being
 * captured (the Python code keeps what a graph saw).  A new reference. */
static int workspace(PyObject* ws, PyObject* on, PyObject* stream, size_t need, PyObject** keep, void** out, size_t* bytes)
{
    int64_t n;
    *keep = NULL;
    if (ws == Py_None) {
        PyObject *capturing = PyObject_CallNoArgs(is_capturing), *device, *h = NULL, *key = NULL;
        int64_t handle;
        Py_XDECREF(capturing);
        if (capturing != Py_False) return 0;
        device = ask(on, n_get_device, NULL);
        if (device && stream_handle(stream, device, &handle)) h = PyLong_FromLongLong(handle);
        if (h) key = PyTuple_Pack(3, device, h, n_scratch);
        ws = key ? PyDict_GetItemWithError(workspaces, key) : NULL;
        Py_XINCREF(ws);
        Py_XDECREF(key);
        Py_XDECREF(h);
        Py_XDECREF(device);
        *keep = ws;
        if (!ws || !ask_int(ws, n_numel, NULL, &n) || n < 0 || (size_t)n < need) return 0;
    } else {
        Py_INCREF(ws);
        *keep = ws;
        if (!is_tensor(ws) || !ask_int(ws, n_numel, NULL, &n)) return 0;
    }
    *bytes = (size_t)n;
    return dev(ws, uint8_type, out);
}

static PyObject* answer(int made, int rc)
{
    if (made) return PyLong_FromLong(rc);
    PyErr_Clear();
    Py_RETURN_NONE;
}

#define ARGS(n) \
    if (nargs != (n)) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return NULL; }

/* decode(q, kv_pool, block_table, ctx_lens, view, max_ctx_len, out, scale, workspace, stream) */
static PyObject* call_decode(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(10)
    int64_t batch, q[3], table[2], row, hq, d, bb, blocks, max_ctx, ws_n, stream;
    void *pq, *pout, *ppool, *ptable, *pctx, *pws;
    const kv_view* view;
    float scale;
    int rc = 0;
    const int ok = sizes(a[3], 1, &batch) && sizes(a[0], 3, q) && int_attr(a[4], n_n_q_local, &hq) &&
                   int_attr(a[4], n_head_dim, &d) && q[0] == batch && q[1] == hq && q[2] == d && sizes(a[2], 2, table) &&
                   table[0] == batch && int_attr(a[4], n_block_bytes, &bb) && dev(a[0], bf16_types, &pq) &&
                   dev(a[6], bf16_types, &pout) && dev(a[1], bf16_types, &ppool) && pool_blocks(a[1], bb, 1, &blocks) &&
                   dev(a[2], int32_type, &ptable) && ask_int(a[2], n_stride, n_zero, &row) && dev(a[3], int32_type, &pctx) &&
                   int_arg(a[5], &max_ctx) && view_handle(a[4], &view) && float_arg(a[7], &scale) &&
                   dev(a[8], uint8_type, &pws) && ask_int(a[8], n_numel, NULL, &ws_n) && stream_handle(a[9], NULL, &stream) &&
                   batch <= INT32_MAX;
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_decode(pq, pout, ppool, blocks, ptable, row, pctx, (int)batch, (int)max_ctx, view, scale, pws, (size_t)ws_n,
                      (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    return answer(ok, rc);
}

/* prefill(q, kv_pool, block_table, ctx_lens, q_offsets, view, max_ctx_len, max_q_len, out, scale, workspace, stream) */
static PyObject* call_prefill(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(12)
    int64_t batch, q[3], off, table[2], row, hq, d, bb, blocks, max_ctx, max_q, stream;
    void *pq, *pout, *ppool, *ptable, *pctx, *poff, *pws;
    size_t ws_n = 0;
    const kv_view* view;
    PyObject* keep = NULL;
    float scale;
    int rc = 0;
    const int ok = sizes(a[3], 1, &batch) && sizes(a[0], 3, q) && int_attr(a[5], n_n_q_local, &hq) &&
                   int_attr(a[5], n_head_dim, &d) && q[1] == hq && q[2] == d && sizes(a[4], 1, &off) && off == batch + 1 &&
                   sizes(a[2], 2, table) && table[0] == batch && int_attr(a[5], n_block_bytes, &bb) &&
                   dev(a[0], bf16_types, &pq) && dev(a[8], bf16_types, &pout) && dev(a[1], bf16_types, &ppool) &&
                   pool_blocks(a[1], bb, 0, &blocks) && dev(a[2], int32_type, &ptable) &&
                   ask_int(a[2], n_stride, n_zero, &row) && dev(a[3], int32_type, &pctx) && dev(a[4], int32_type, &poff) &&
                   int_arg(a[6], &max_ctx) && int_arg(a[7], &max_q) && view_handle(a[5], &view) && float_arg(a[9], &scale) &&
                   batch <= INT32_MAX && stream_handle(a[11], NULL, &stream) &&
                   workspace(a[10], a[0], a[11],
                             a[10] == Py_None ? f_prefill_bytes(view, (int)batch, q[0], (int)max_ctx, (int)max_q) : 0, &keep,
                             &pws, &ws_n);
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_prefill(pq, pout, ppool, blocks, ptable, row, pctx, poff, (int)batch, q[0], (int)max_ctx, (int)max_q, view, scale,
                       pws, ws_n, (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    Py_XDECREF(keep);
    return answer(ok, rc);
}

/* linear(x, w_full, view, out, workspace, stream) */
static PyObject* call_linear(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(6)
    int64_t x[2], w[2], y[2], ldx, ldw, ldy, stream;
    void *px, *pw, *py, *pws;
    size_t ws_n = 0;
    PyObject* keep = NULL;
    Py_buffer view;
    int rc = 0;
    if ((PyObject*)Py_TYPE(a[2]) != weight_view_type || PyObject_GetBuffer(a[2], &view, PyBUF_SIMPLE) != 0) return answer(0, 0);
    const kv_weight_view* v = (const kv_weight_view*)view.buf;
    const int ok = view.len == (Py_ssize_t)sizeof(kv_weight_view) && dev_rows(a[0], bf16_types, &px, x, &ldx) &&
                   x[1] == v->col_count && dev_rows(a[1], bf16_types, &pw, w, &ldw) && dev_rows(a[3], bf16_types, &py, y, &ldy) &&
                   x[0] <= INT32_MAX && stream_handle(a[5], NULL, &stream) &&
                   workspace(a[4], a[0], a[5], a[4] == Py_None ? f_linear_bytes(v, (int)x[0]) : 0, &keep, &pws, &ws_n);
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_linear(px, ldx, pw, w[0], ldw, v, py, ldy, (int)x[0], pws, ws_n, (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    PyBuffer_Release(&view);
    Py_XDECREF(keep);
    return answer(ok, rc);
}

/* append(kv_pool, view, k_new, v_new, block_table, positions, stream) */
static PyObject* call_append(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(7)
    int64_t n, k[3], v[3], hkv, d, bb, blocks, row, stream;
    void *ppool, *pk, *pv, *ptable, *ppos;
    const kv_view* view;
    int rc = 0;
    const int ok = sizes(a[5], 1, &n) && int_attr(a[1], n_n_kv_local, &hkv) && int_attr(a[1], n_head_dim, &d) &&
                   sizes(a[2], 3, k) && sizes(a[3], 3, v) && k[0] == n && k[1] == hkv && k[2] == d && v[0] == n && v[1] == hkv &&
                   v[2] == d && int_attr(a[1], n_block_bytes, &bb) && dev(a[0], bf16_types, &ppool) &&
                   pool_blocks(a[0], bb, 0, &blocks) && view_handle(a[1], &view) && dev(a[2], bf16_types, &pk) &&
                   dev(a[3], bf16_types, &pv) && dev(a[4], int32_type, &ptable) && ask_int(a[4], n_stride, n_zero, &row) &&
                   dev(a[5], int32_type, &ppos) && n <= INT32_MAX && stream_handle(a[6], NULL, &stream);
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_append(ppool, blocks, view, pk, pv, ptable, row, ppos, (int)n, (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    return answer(ok, rc);
}

/* repack(kv_pool, src_view, dst_view, src_block_table, dst_block_table, n_tokens, max_tokens, stream) */
static PyObject* call_repack(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(8)
    int64_t n, bb, blocks, src_row, dst_row, most, stream;
    void *ppool, *psrc, *pdst, *pn;
    const kv_view *src, *dst;
    int rc = 0;
    const int ok = sizes(a[5], 1, &n) && int_attr(a[1], n_block_bytes, &bb) && dev(a[0], bf16_types, &ppool) &&
                   pool_blocks(a[0], bb, 0, &blocks) && view_handle(a[1], &src) && view_handle(a[2], &dst) &&
                   dev(a[3], int32_type, &psrc) && ask_int(a[3], n_stride, n_zero, &src_row) && dev(a[4], int32_type, &pdst) &&
                   ask_int(a[4], n_stride, n_zero, &dst_row) && dev(a[5], int32_type, &pn) && int_arg(a[6], &most) &&
                   n <= INT32_MAX && stream_handle(a[7], NULL, &stream);
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_repack(ppool, blocks, src, dst, psrc, src_row, pdst, dst_row, pn, (int)n, (int)most, (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    return answer(ok, rc);
}

/* The device that is current, which the calls below want all their tensors on (the Python code sorts the others out). */
static int current(int64_t* out) { return to_int64(PyObject_CallNoArgs(get_device), out); }

/* dev(), on that device (of the GPU: the others have no number), with its sizes as given (sizes of -1 are found out) */
static int shaped(PyObject* t, PyObject* dtype, int64_t device, int n, int64_t* size, void** out)
{
    int64_t found[3], on;
    if (!sizes(t, n, found)) return 0;
    for (int i = 0; i < n; ++i) {
        if (size[i] >= 0 && size[i] != found[i]) return 0;
        size[i] = found[i];
    }
    if (!dtype_is(t, dtype) || !ask_int(t, n_get_device, NULL, &on) || on != device || on < 0) return 0;
    PyObject* c = ask(t, n_is_contiguous, NULL);
    const int yes = c == Py_True;
    Py_XDECREF(c);
    return yes && address(t, out);
}

/* binding._token_rows: [tokens][heads][d], tokens may lie apart; tokens of -1 are found out */
static int token_rows(PyObject* t, int64_t device, int64_t* tokens, int64_t heads, int64_t d, void** out, int64_t* row)
{
    int64_t found[3], stride[3], on;
    if (!sizes(t, 3, found) || (*tokens >= 0 && found[0] != *tokens) || found[1] != heads || found[2] != d ||
        !dtype_is(t, bf16_types) || !ask_int(t, n_get_device, NULL, &on) || on != device || on < 0)
        return 0;
    *tokens = found[0];
    PyObject* all = ask(t, n_stride, NULL);   /* (all three in one call) */
    int ok = all && PyTuple_Check(all) && PyTuple_GET_SIZE(all) == 3;
    for (int i = 0; ok && i < 3; ++i) {
        PyObject* x = PyTuple_GET_ITEM(all, i);
        Py_INCREF(x);
        ok = to_int64(x, stride + i);
    }
    Py_XDECREF(all);
    if (!ok || stride[2] != 1 || (heads > 1 && stride[1] != d)) return 0;
    *row = *tokens > 1 ? stride[0] : heads * d;
    return address(t, out);
}

/* What all of the calls below ask of the pool, its view and its table. */
typedef struct {
    int64_t device, batch, blocks, row, hq, hkv, d, bb, heads;   /* heads: KV heads of all ranks */
    void *pool, *table, *ctx;
    const kv_view* view;
} cache_args;
/* The view's handle and numbers, which it keeps in a tuple for this (one attribute in place of seven: 0.15 us). */
static int view_of(PyObject* view, cache_args* c)
{
    int64_t handle = 0;
    int64_t* const to[] = {&handle, &c->hq, &c->hkv, &c->d, &c->bb, &c->heads};
    PyObject* t = PyObject_GetAttr(view, n_numbers);
    int ok = t && PyTuple_CheckExact(t) && PyTuple_GET_SIZE(t) == 6;
    for (int i = 0; ok && i < 6; ++i) {
        PyObject* x = PyTuple_GET_ITEM(t, i);
        Py_INCREF(x);
        ok = to_int64(x, to[i]);
    }
    Py_XDECREF(t);
    c->view = (const kv_view*)(uintptr_t)handle;
    return ok && handle != 0;
}
static int places_of(PyObject* view, PyObject* table, PyObject* ctx, cache_args* c)   /* all but the pool */
{
    int64_t tab[2];
    c->batch = -1;
    if (!current(&c->device) || !shaped(ctx, int32_type, c->device, 1, &c->batch, &c->ctx) || c->batch > INT32_MAX) return 0;
    tab[0] = c->batch;
    tab[1] = -1;
    return shaped(table, int32_type, c->device, 2, tab, &c->table) && ask_int(table, n_stride, n_zero, &c->row) && view_of(view, c);
}
static int cache_of(PyObject* pool, PyObject* view, PyObject* table, PyObject* ctx, cache_args* c)
{
    int64_t on;
    return places_of(view, table, ctx, c) && dev(pool, bf16_types, &c->pool) && ask_int(pool, n_get_device, NULL, &on) &&
           on == c->device && pool_blocks(pool, c->bb, 1, &c->blocks);
}

/* binding._q8_cache on top of that: codes, their format, scales */
typedef struct {
    cache_args c;
    int format;
    void* scales;
} q8_args;
static int q8_of(PyObject* pool, PyObject* scales, PyObject* view, PyObject* table, PyObject* ctx, q8_args* x)
{
    cache_args* c = &x->c;
    int64_t on, n, format;
    if (!places_of(view, table, ctx, c) || !is_tensor(pool)) return 0;
    PyObject* dtype = PyObject_GetAttr(pool, n_dtype);
    PyObject* f = dtype ? PyDict_GetItemWithError(q8_formats, dtype) : NULL;
    Py_XDECREF(dtype);
    if (!f || !int_arg(f, &format)) return 0;
    x->format = (int)format;
    PyObject* cont = ask(pool, n_is_contiguous, NULL);
    const int dense = cont == Py_True;
    Py_XDECREF(cont);
    if (!dense || !ask_int(pool, n_get_device, NULL, &on) || on != c->device || on < 0 || !address(pool, &c->pool) ||
        !ask_int(pool, n_numel, NULL, &n) || c->bb <= 0 || n % (c->bb / 2))   /* (codes of one byte) */
        return 0;
    c->blocks = n / (c->bb / 2);
    if (!is_tensor(scales) || !dtype_is(scales, float_type) || !ask_int(scales, n_get_device, NULL, &on) || on != c->device ||
        !ask_int(scales, n_numel, NULL, &n) || n != c->blocks * 2 * c->heads)
        return 0;
    cont = ask(scales, n_is_contiguous, NULL);
    const int dense_too = cont == Py_True;
    Py_XDECREF(cont);
    return dense_too && address(scales, &x->scales);
}

/* binding._kept_per_token: [batch][n_kv_local][tokens], or none */
static int kept_per_token(PyObject* t, PyObject* dtype, const cache_args* c, void** out, int64_t* tokens)
{
    int64_t size[3] = {c->batch, c->hkv, -1};
    *out = NULL;
    *tokens = 0;
    if (t == Py_None) return 1;
    if (!shaped(t, dtype, c->device, 3, size, out)) return 0;
    *tokens = size[2];
    return 1;
}

/* Positions, [tokens] or [axes][tokens], and which axis a pair of dims takes. */
enum { kMostPairs = 128 };
static int positions_of(PyObject* t, int64_t device, int64_t tokens, void** out, int* n_axes)
{
    int64_t pos[2] = {tokens, -1};
    *n_axes = 1;
    if (shaped(t, int32_type, device, 1, pos, out)) return 1;
    PyErr_Clear();
    pos[0] = -1;
    pos[1] = tokens;
    if (!shaped(t, int32_type, device, 2, pos, out) || pos[0] < 1 || pos[0] > 4) return 0;
    *n_axes = (int)pos[0];
    return 1;
}
static int axes_of(PyObject* list, int n_axes, int64_t half, int32_t axes[kMostPairs])
{
    if (list == Py_None) return n_axes == 1;
    int ok = (PyList_CheckExact(list) || PyTuple_CheckExact(list)) && PySequence_Fast_GET_SIZE(list) == half;
    for (int64_t i = 0; ok && i < half; ++i) {
        int64_t x;
        ok = int_arg(PySequence_Fast_GET_ITEM(list, i), &x);
        axes[i] = (int32_t)x;
    }
    return ok;
}

/* rope(kv_pool, view, q, k, v, positions, inv_freq, block_table, ctx_lens, q_offsets, axes, pairs, out, token_pos, stream, weights) */
static PyObject* call_rope(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(16)
    int64_t q[1] = {-1}, q_row, k_row, v_row, half = -1, off, out[3], per, w_n, pairs, stream;
    void *pq, *pk, *pv, *pout, *ppos, *pfreq, *poff = NULL, *pper, *pw;
    int32_t axes[kMostPairs];
    cache_args c;
    int rc = 0, n_axes = 1;
    int ok = cache_of(a[0], a[1], a[7], a[8], &c) && token_rows(a[2], c.device, q, c.hq, c.d, &pq, &q_row) &&
             token_rows(a[3], c.device, q, c.hkv, c.d, &pk, &k_row) && token_rows(a[4], c.device, q, c.hkv, c.d, &pv, &v_row);
    if (ok) {
        out[0] = q[0];
        out[1] = c.hq;
        out[2] = c.d;
        ok = positions_of(a[5], c.device, q[0], &ppos, &n_axes) && shaped(a[6], float_type, c.device, 1, &half, &pfreq) &&
             half <= kMostPairs && shaped(a[12], bf16_types, c.device, 3, out, &pout) && int_arg(a[11], &pairs) &&
             stream_handle(a[14], NULL, &stream) && axes_of(a[10], n_axes, half, axes);
    }
    if (ok && a[9] != Py_None) {
        off = c.batch + 1;
        ok = shaped(a[9], int32_type, c.device, 1, &off, &poff);
    }
    ok = ok && kept_per_token(a[13], int32_type, &c, &pper, &per) && kept_per_token(a[15], float_type, &c, &pw, &w_n);
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_rope(c.pool, c.blocks, c.view, pq, q_row, pk, k_row, pv, v_row, pout, ppos, q[0], n_axes, pfreq, (int)(2 * half),
                    a[10] == Py_None ? NULL : axes, (int)pairs, c.table, c.row, c.ctx, poff, (int)c.batch, q[0], pper, per,
                    pw, w_n, (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    return answer(ok, rc);
}

/* accept(kv_pool, view, block_table, ctx_lens, q_offsets, accepted, n_accepted, new_lens, stream, token_pos, weights) */
static PyObject* call_accept(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(11)
    int64_t off, acc[2], n, pos_n, w_n, stream;
    void *poff, *pacc, *pn, *pnew, *ppos, *pw;
    cache_args c;
    int rc = 0, ok = cache_of(a[0], a[1], a[2], a[3], &c);
    if (ok) {
        off = c.batch + 1;
        acc[0] = n = c.batch;
        acc[1] = -1;
        ok = shaped(a[4], int32_type, c.device, 1, &off, &poff) && shaped(a[5], int32_type, c.device, 2, acc, &pacc) &&
             shaped(a[6], int32_type, c.device, 1, &n, &pn) && shaped(a[7], int32_type, c.device, 1, &n, &pnew) &&
             kept_per_token(a[9], int32_type, &c, &ppos, &pos_n) && kept_per_token(a[10], float_type, &c, &pw, &w_n) &&
             stream_handle(a[8], NULL, &stream);
    }
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_accept(c.pool, c.blocks, c.view, c.table, c.row, c.ctx, poff, pacc, acc[1], pn, (int)c.batch, pnew, ppos, pos_n, pw, w_n,
                      (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    return answer(ok, rc);
}

/* tree(q, kv_pool, block_table, ctx_lens, q_offsets, tree_mask, view, max_ctx_len, max_q_len, out, scale, workspace, stream) */
static PyObject* call_tree(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(13)
    int64_t q[3], off, mask[2], max_ctx, max_q, ws = -1, stream;
    void *pq, *pout, *poff, *pmask, *pws;
    cache_args c;
    float scale;
    int rc = 0, ok = cache_of(a[1], a[6], a[2], a[3], &c);
    if (ok) {
        q[0] = mask[1] = -1;
        q[1] = c.hq;
        q[2] = c.d;
        off = c.batch + 1;
        ok = shaped(a[0], bf16_types, c.device, 3, q, &pq) && shaped(a[9], bf16_types, c.device, 3, q, &pout) &&
             shaped(a[4], int32_type, c.device, 1, &off, &poff);
        mask[0] = q[0];
        ok = ok && shaped(a[5], word_types, c.device, 2, mask, &pmask) && int_arg(a[7], &max_ctx) && int_arg(a[8], &max_q) &&
             float_arg(a[10], &scale) && shaped(a[11], uint8_type, c.device, 1, &ws, &pws) && stream_handle(a[12], NULL, &stream);
    }
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_tree(pq, pout, c.pool, c.blocks, c.table, c.row, c.ctx, poff, pmask, mask[1], (int)c.batch, q[0], (int)max_ctx,
                    (int)max_q, c.view, scale, pws, (size_t)ws, (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    return answer(ok, rc);
}

/* weights(q, kv_pool, block_table, ctx_lens, view, max_ctx_len, weights, out, scale, workspace, stream) */
static PyObject* call_weights(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(11)
    int64_t q[3], per[3], max_ctx, ws = -1, stream;
    void *pq, *pout, *pper, *pws;
    cache_args c;
    float scale;
    int rc = 0, ok = cache_of(a[1], a[4], a[2], a[3], &c);
    if (ok) {
        q[0] = per[0] = c.batch;
        q[1] = c.hq;
        per[1] = c.hkv;
        q[2] = c.d;
        per[2] = -1;
        ok = shaped(a[0], bf16_types, c.device, 3, q, &pq) && shaped(a[7], bf16_types, c.device, 3, q, &pout) &&
             shaped(a[6], float_type, c.device, 3, per, &pper) && int_arg(a[5], &max_ctx) && float_arg(a[8], &scale) &&
             shaped(a[9], uint8_type, c.device, 1, &ws, &pws) && stream_handle(a[10], NULL, &stream);
    }
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_weights(pq, pout, c.pool, c.blocks, c.table, c.row, c.ctx, (int)c.batch, (int)max_ctx, c.view, scale, pper, per[2],
                       pws, (size_t)ws, (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    return answer(ok, rc);
}

/* rope_q8(kv_pool, scales, view, q, k, v, positions, inv_freq, block_table, ctx_lens, q_offsets, axes, pairs, out, stream) */
static PyObject* call_rope_q8(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(15)
    int64_t k[1] = {-1}, q_row = 0, k_row, v_row, half = 0, off, out[3], pairs, stream;
    void *pq = NULL, *pk, *pv, *pout = NULL, *ppos = NULL, *pfreq = NULL, *poff = NULL;
    int32_t axes[kMostPairs];
    q8_args x;
    const cache_args* c = &x.c;
    int rc = 0, n_axes = 1;
    int ok = q8_of(a[0], a[1], a[2], a[8], a[9], &x) && token_rows(a[4], c->device, k, c->hkv, c->d, &pk, &k_row) &&
             token_rows(a[5], c->device, k, c->hkv, c->d, &pv, &v_row) && (a[3] == Py_None) == (a[13] == Py_None) &&
             (a[7] == Py_None || a[6] != Py_None);
    if (ok && a[3] != Py_None) {
        out[0] = k[0];
        out[1] = c->hq;
        out[2] = c->d;
        ok = token_rows(a[3], c->device, k, c->hq, c->d, &pq, &q_row) && shaped(a[13], bf16_types, c->device, 3, out, &pout);
    }
    if (ok && a[6] != Py_None) ok = positions_of(a[6], c->device, k[0], &ppos, &n_axes);
    if (ok && a[7] != Py_None) {
        half = -1;
        ok = shaped(a[7], float_type, c->device, 1, &half, &pfreq) && half <= kMostPairs;
    }
    ok = ok && axes_of(a[11], n_axes, half, axes) && int_arg(a[12], &pairs) && stream_handle(a[14], NULL, &stream);
    if (ok && a[10] != Py_None) {
        off = c->batch + 1;
        ok = shaped(a[10], int32_type, c->device, 1, &off, &poff);
    }
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_rope_q8(c->pool, x.scales, x.format, c->blocks, c->view, pq, q_row, pk, k_row, pv, v_row, pout, ppos, k[0], n_axes, pfreq,
                       (int)(2 * half), a[11] == Py_None ? NULL : axes, (int)pairs, c->table, c->row, c->ctx, poff, (int)c->batch, k[0],
                       (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    return answer(ok, rc);
}

/* decode_q8(q, kv_pool, scales, block_table, ctx_lens, view, max_ctx_len, out, scale, workspace, stream) */
static PyObject* call_decode_q8(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(11)
    int64_t q[3], max_ctx, ws = -1, stream;
    void *pq, *pout, *pws;
    q8_args x;
    const cache_args* c = &x.c;
    float scale;
    int rc = 0, ok = q8_of(a[1], a[2], a[5], a[3], a[4], &x);
    if (ok) {
        q[0] = c->batch;
        q[1] = c->hq;
        q[2] = c->d;
        ok = shaped(a[0], bf16_types, c->device, 3, q, &pq) && shaped(a[7], bf16_types, c->device, 3, q, &pout) && int_arg(a[6], &max_ctx) &&
             float_arg(a[8], &scale) && shaped(a[9], uint8_type, c->device, 1, &ws, &pws) && stream_handle(a[10], NULL, &stream);
    }
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_decode_q8(pq, pout, c->pool, x.scales, x.format, c->blocks, c->table, c->row, c->ctx, (int)c->batch, (int)max_ctx, c->view,
                         scale, pws, (size_t)ws, (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    return answer(ok, rc);
}

/* prefill_q8(q, kv_pool, scales, block_table, ctx_lens, q_offsets, view, max_ctx_len, max_q_len, out, scale, workspace, stream) */
static PyObject* call_prefill_q8(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(13)
    int64_t q[3], off, max_ctx, max_q, ws = -1, stream;
    void *pq, *pout, *poff, *pws;
    q8_args x;
    const cache_args* c = &x.c;
    float scale;
    int rc = 0, ok = q8_of(a[1], a[2], a[6], a[3], a[4], &x);
    if (ok) {
        q[0] = -1;
        q[1] = c->hq;
        q[2] = c->d;
        off = c->batch + 1;
        ok = shaped(a[0], bf16_types, c->device, 3, q, &pq) && shaped(a[9], bf16_types, c->device, 3, q, &pout) &&
             shaped(a[5], int32_type, c->device, 1, &off, &poff) && int_arg(a[7], &max_ctx) && int_arg(a[8], &max_q) &&
             float_arg(a[10], &scale) && shaped(a[11], uint8_type, c->device, 1, &ws, &pws) && stream_handle(a[12], NULL, &stream);
    }
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_prefill_q8(pq, pout, c->pool, x.scales, x.format, c->blocks, c->table, c->row, c->ctx, poff, (int)c->batch, q[0], (int)max_ctx,
                          (int)max_q, c->view, scale, pws, (size_t)ws, (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    return answer(ok, rc);
}

/* repack_q8(kv_pool, scales, src_view, dst_view, src_block_table, dst_block_table, n_tokens, max_tokens, stream) */
static PyObject* call_repack_q8(PyObject* self, PyObject* const* a, Py_ssize_t nargs)
{
    ARGS(9)
    int64_t tab[2], dst_row, most, stream;
    void* pdst;
    const kv_view* dst;
    q8_args x;
    const cache_args* c = &x.c;
    int rc = 0, ok = q8_of(a[0], a[1], a[2], a[4], a[6], &x);
    if (ok) {
        tab[0] = c->batch;
        tab[1] = -1;
        ok = view_handle(a[3], &dst) && shaped(a[5], int32_type, c->device, 2, tab, &pdst) && ask_int(a[5], n_stride, n_zero, &dst_row) &&
             int_arg(a[7], &most) && stream_handle(a[8], NULL, &stream);
    }
    if (ok) {
        Py_BEGIN_ALLOW_THREADS
        rc = f_repack_q8(c->pool, x.scales, c->blocks, c->view, dst, c->table, c->row, pdst, dst_row, c->ctx, (int)c->batch, (int)most,
                         (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS
    }
    return answer(ok, rc);
}

/* setup_q8((addresses of rope_q8, decode_q8, prefill_q8, repack_q8), dict of formats by dtype); after setup_operators() */
static PyObject* setup_q8(PyObject* self, PyObject* args)
{
    unsigned long long f[4];
    PyObject* formats;
    if (!PyArg_ParseTuple(args, "(KKKK)O!", f, f + 1, f + 2, f + 3, &PyDict_Type, &formats)) return NULL;
    f_rope_q8 = (rope_q8_fn)(uintptr_t)f[0];
    f_decode_q8 = (decode_q8_fn)(uintptr_t)f[1];
    f_prefill_q8 = (prefill_q8_fn)(uintptr_t)f[2];
    f_repack_q8 = (repack_q8_fn)(uintptr_t)f[3];
    Py_INCREF(formats);
    Py_XSETREF(q8_formats, formats);
    Py_RETURN_NONE;
}

/* setup_operators((addresses of rope, accept, tree, weights), (float32, dtypes of mask words)); after setup() */
static PyObject* setup_operators(PyObject* self, PyObject* args)
{
    unsigned long long f[4];
    PyObject *f32, *words;
    if (!PyArg_ParseTuple(args, "(KKKK)(OO)", f, f + 1, f + 2, f + 3, &f32, &words)) return NULL;
    f_rope = (rope_fn)(uintptr_t)f[0];
    f_accept = (accept_fn)(uintptr_t)f[1];
    f_tree = (tree_fn)(uintptr_t)f[2];
    f_weights = (weights_fn)(uintptr_t)f[3];
    Py_INCREF(f32);
    Py_XSETREF(float_type, f32);
    Py_INCREF(words);
    Py_XSETREF(word_types, words);
    Py_RETURN_NONE;
}

/* setup((addresses of the seven functions), (types), (dtypes), (torch._C functions), dict) */
static PyObject* setup(PyObject* self, PyObject* args)
{
    unsigned long long f[7];
    PyObject *t0, *t1, *t2, *bf, *i32, *u8, *gd, *rs, *ic, *ws;
    if (!PyArg_ParseTuple(args, "(KKKKKKK)(OOO)(OOO)(OOO)O!", f, f + 1, f + 2, f + 3, f + 4, f + 5, f + 6, &t0, &t1, &t2, &bf, &i32,
                          &u8, &gd, &rs, &ic, &PyDict_Type, &ws))
        return NULL;
    f_decode = (decode_fn)(uintptr_t)f[0];
    f_prefill = (prefill_fn)(uintptr_t)f[1];
    f_prefill_bytes = (prefill_bytes_fn)(uintptr_t)f[2];
    f_linear = (linear_fn)(uintptr_t)f[3];
    f_linear_bytes = (linear_bytes_fn)(uintptr_t)f[4];
    f_append = (append_fn)(uintptr_t)f[5];
    f_repack = (repack_fn)(uintptr_t)f[6];
    PyObject** const to[] = {&tensor_type, &parameter_type, &weight_view_type, &bf16_types, &int32_type, &uint8_type,
                             &get_device,  &raw_stream,     &is_capturing,     &workspaces};
    PyObject* const from[] = {t0, t1, t2, bf, i32, u8, gd, rs, ic, ws};
    for (int i = 0; i < 10; ++i) {
        Py_INCREF(from[i]);
        Py_XSETREF(*to[i], from[i]);
    }
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"setup", setup, METH_VARARGS, NULL},
    {"decode", (PyCFunction)(void (*)(void))call_decode, METH_FASTCALL, NULL},
    {"prefill", (PyCFunction)(void (*)(void))call_prefill, METH_FASTCALL, NULL},
    {"linear", (PyCFunction)(void (*)(void))call_linear, METH_FASTCALL, NULL},
    {"append", (PyCFunction)(void (*)(void))call_append, METH_FASTCALL, NULL},
    {"setup_operators", setup_operators, METH_VARARGS, NULL},
    {"rope", (PyCFunction)(void (*)(void))call_rope, METH_FASTCALL, NULL},
    {"accept", (PyCFunction)(void (*)(void))call_accept, METH_FASTCALL, NULL},
    {"tree", (PyCFunction)(void (*)(void))call_tree, METH_FASTCALL, NULL},
    {"weights", (PyCFunction)(void (*)(void))call_weights, METH_FASTCALL, NULL},
    {"setup_q8", setup_q8, METH_VARARGS, NULL},
    {"rope_q8", (PyCFunction)(void (*)(void))call_rope_q8, METH_FASTCALL, NULL},
    {"decode_q8", (PyCFunction)(void (*)(void))call_decode_q8, METH_FASTCALL, NULL},
    {"prefill_q8", (PyCFunction)(void (*)(void))call_prefill_q8, METH_FASTCALL, NULL},
    {"repack_q8", (PyCFunction)(void (*)(void))call_repack_q8, METH_FASTCALL, NULL},
    {"repack", (PyCFunction)(void (*)(void))call_repack, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL},
};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void)
{
    struct {
        PyObject** to;
        const char* text;
    } const names[] = {
        {&n_is_cuda, "is_cuda"}, {&n_dtype, "dtype"}, {&n_is_contiguous, "is_contiguous"}, {&n_data_ptr, "data_ptr"},
        {&n_shape, "shape"}, {&n_stride, "stride"}, {&n_numel, "numel"}, {&n_element_size, "element_size"},
        {&n_get_device, "get_device"}, {&n_cuda_stream, "cuda_stream"}, {&n_handle, "handle"}, {&n_value, "value"},
        {&n_block_bytes, "block_bytes"}, {&n_n_q_local, "n_q_local"}, {&n_n_kv_local, "n_kv_local"},
        {&n_head_dim, "head_dim"}, {&n_scratch, "scratch"},
        {&n_numbers, "_numbers"},
    };
    for (size_t i = 0; i < sizeof(names) / sizeof(names[0]); ++i)
        if (!*names[i].to && !(*names[i].to = PyUnicode_InternFromString(names[i].text))) return NULL;
    if (!(n_zero = PyLong_FromLong(0)) || !(n_one = PyLong_FromLong(1))) return NULL;
    return PyModule_Create(&module);
}
