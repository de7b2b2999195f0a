/* Arguments of the fused call, and of the calls between the products, taken from Python objects and handed to the library without ctypes.
 *
 * Bound by host work: a decode step of a few microseconds is issued as fast as its arguments are marshalled.  One call,
 * arguments to return, without the launch: 4.0 us through ctypes and the binding's own Python lines, 1.2 here (15 arguments, four
 * tensors).  The same attributes and methods of the same objects are asked for as the binding does; nothing is kept from one call for the next.
 * Whatever is not as expected is left to the binding's general path: None is returned and nothing has happened.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "../../include/fgmp.h"

typedef int (*fused_fn)(const void *, int, int64_t, int64_t, int64_t, const float *, float, float, const void *, int64_t, float *,
                        int64_t, void *, size_t, void *);

static PyObject *s_is_cuda, *s_shape, *s_dtype, *s_data_ptr, *s_stride, *s_numel, *s_K, *s_rows, *s_buf, *zero;

static int is_true(PyObject *o, PyObject *name)
{
    PyObject *v = PyObject_GetAttr(o, name);
    const int t = v == Py_True;
    Py_XDECREF(v);
    return t;
}

/* an integer result, which is consumed; *bad is set where it is none */
static int64_t integer(PyObject *v, int *bad)
{
    int64_t r = 0;
    if (v != NULL && PyLong_Check(v)) {
        r = PyLong_AsLongLong(v);
        if (r == -1 && PyErr_Occurred()) *bad = 1;
    } else {
        *bad = 1;
    }
    Py_XDECREF(v);
    return r;
}

/* (from here on: nothing is asked for once something was bad, an exception may be pending) */
static int64_t attribute(PyObject *o, PyObject *name, int *bad)
{
    return *bad ? 0 : integer(PyObject_GetAttr(o, name), bad);
}

static void *pointer(PyObject *tensor, int *bad)
{
    if (*bad) return NULL;
    PyObject *const args[1] = {tensor};
    PyObject *v = PyObject_VectorcallMethod(s_data_ptr, args, 1, NULL);
    void *p = NULL;
    if (v != NULL && PyLong_Check(v)) p = PyLong_AsVoidPtr(v);
    if (v == NULL || !PyLong_Check(v) || PyErr_Occurred()) *bad = 1;
    Py_XDECREF(v);
    return p;
}

static int64_t row_stride(PyObject *tensor, int *bad)
{
    PyObject *const args[2] = {tensor, zero};
    return *bad ? 0 : integer(PyObject_VectorcallMethod(s_stride, args, 2, NULL), bad);
}

static int64_t elements(PyObject *tensor, int *bad)
{
    PyObject *const args[1] = {tensor};
    return *bad ? 0 : integer(PyObject_VectorcallMethod(s_numel, args, 1, NULL), bad);
}

static double number(PyObject *o, int *bad)
{
    if (*bad) return 0.0;
    if (PyFloat_CheckExact(o)) return PyFloat_AS_DOUBLE(o);
    PyObject *v = PyNumber_Float(o);
    const double d = v != NULL ? PyFloat_AS_DOUBLE(v) : 0.0;
    if (v == NULL) *bad = 1;
    Py_XDECREF(v);
    return d;
}

/* quant_gemm_fused(entry point, torch.float32, torch.bfloat16, X, fisher, threshold, scale, packed W, out, workspace, stream)
 * -> status, or None */
static PyObject *quant_gemm_fused(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    if (n != 11) {
        PyErr_SetString(PyExc_TypeError, "eleven arguments expected");
        return NULL;
    }
    PyObject *const X = a[3], *const fisher = a[4], *const pW = a[7], *const out = a[8], *const workspace = a[9];
    int bad = 0;
    int64_t M = 0, K = 0;
    PyObject *v = NULL;

    if (!is_true(X, s_is_cuda) || !is_true(fisher, s_is_cuda)) goto general;
    v = PyObject_GetAttr(X, s_shape);
    if (v == NULL || !PyTuple_Check(v) || PyTuple_GET_SIZE(v) != 2) goto general;
    Py_INCREF(PyTuple_GET_ITEM(v, 0));
    Py_INCREF(PyTuple_GET_ITEM(v, 1));
    M = integer(PyTuple_GET_ITEM(v, 0), &bad);
    K = integer(PyTuple_GET_ITEM(v, 1), &bad);
    Py_CLEAR(v);
    if (bad) goto general;
    v = PyObject_GetAttr(X, s_dtype);
    const int dt = v == a[1] ? 0 : v == a[2] ? 1 : -1;
    Py_CLEAR(v);
    if (dt < 0) goto general;
    if (attribute(pW, s_K, &bad) != K) goto general;
    const int64_t N = attribute(pW, s_rows, &bad);
    if (bad) goto general;
    v = PyObject_GetAttr(pW, s_buf);
    if (v == NULL) goto general;
    const void *const w = pointer(v, &bad);
    Py_CLEAR(v);
    const void *const x = pointer(X, &bad);
    const int64_t ldx = row_stride(X, &bad);
    const float *const f = (const float *)pointer(fisher, &bad);
    float *const y = (float *)pointer(out, &bad);
    const int64_t ldy = row_stride(out, &bad);
    void *const ws = pointer(workspace, &bad);
    const int64_t ws_bytes = elements(workspace, &bad);
    const float T = (float)number(a[5], &bad), S = (float)number(a[6], &bad);
    if (bad) goto general;
    const fused_fn fn = (fused_fn)PyLong_AsVoidPtr(a[0]);
    void *const stream = fn != NULL ? PyLong_AsVoidPtr(a[10]) : NULL;
    if (fn == NULL || PyErr_Occurred()) goto general;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(x, dt, M, K, ldx, f, T, S, w, N, y, ldy, ws, (size_t)ws_bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
general:
    Py_XDECREF(v);
    PyErr_Clear();
    Py_RETURN_NONE;
}

/* ---- between the products ----
 *
 * Tensors are checked against letters, one for each dimension: a letter's first tensor sets its size, all others have to agree.
 * What does not fit is left to the general path (call.bad), which says what is wrong. */
enum { F32, BF16, I32, I64, U8, N_TYPES };
typedef struct {
    int64_t size[26];          /* by letter; -1: not known yet */
    PyObject *const *types;    /* torch.float32, .bfloat16, .int32, .int64, .uint8 */
    int bad;
} call_t;

static int64_t *letter(call_t *c, char x) { return &c->size[x - 'A']; }

static void begin(call_t *c, PyObject *types)
{
    for (int i = 0; i < 26; ++i) c->size[i] = -1;
    c->bad = !PyTuple_Check(types) || PyTuple_GET_SIZE(types) != N_TYPES;
    c->types = c->bad ? NULL : &PyTuple_GET_ITEM(types, 0);
}

/* items of a tuple of integers, which is consumed; their number, or -1 */
static int integers(PyObject *v, int64_t *to, int most)
{
    int n = -1;
    if (v != NULL && PyTuple_Check(v) && PyTuple_GET_SIZE(v) <= most) {
        n = (int)PyTuple_GET_SIZE(v);
        for (int i = 0; i < n; ++i) {
            PyObject *const item = PyTuple_GET_ITEM(v, i);
            to[i] = PyLong_Check(item) ? PyLong_AsLongLong(item) : -1;
            if (to[i] < 0) n = -1;   /* (no size or stride here is below zero) */
        }
    }
    Py_XDECREF(v);
    return n;
}

/* A GPU tensor's address; its dimensions are those of `letters`, its type is one of `types` (a bit each, found in *type).  `strides`: taken,
 * and the last dimension's elements have to lie next to each other; without: the tensor has to be contiguous.  None has the address 0 if
 * `optional`. */
static void *tensor(call_t *c, PyObject *t, const char *letters, int types, int *type, int64_t *strides, int optional)
{
    if (c->bad || (optional && t == Py_None)) return NULL;
    const int n = (int)strlen(letters);
    int64_t size[4], step[4];
    c->bad = 1;
    if (!is_true(t, s_is_cuda)) return NULL;
    PyObject *v = PyObject_GetAttr(t, s_dtype);
    int k = 0;
    while (k < N_TYPES && (!(types >> k & 1) || v != c->types[k])) ++k;
    Py_XDECREF(v);
    if (k == N_TYPES || v == NULL) return NULL;
    if (type != NULL) *type = k;
    if (integers(PyObject_GetAttr(t, s_shape), size, 4) != n) return NULL;
    PyObject *const args[1] = {t};
    if (integers(PyObject_VectorcallMethod(s_stride, args, 1, NULL), step, 4) != n) return NULL;
    int64_t next = 1;
    for (int i = n - 1; i >= 0; --i) {
        int64_t *const known = letter(c, letters[i]);
        if (*known < 0) *known = size[i];
        if (*known != size[i]) return NULL;
        if (size[i] != 1 && step[i] != next && (strides == NULL || i == n - 1)) return NULL;
        next *= size[i];
    }
    if (strides != NULL)
        for (int i = 0; i + 1 < n; ++i) strides[i] = step[i];
    c->bad = 0;
    return pointer(t, &c->bad);
}

static fgmp_heads_t heads(call_t *c, PyObject *t, const char *letters, int types, int *type)
{
    fgmp_heads_t h = {NULL, 0, 0, 0};
    int64_t strides[3] = {0, 0, 0};
    h.data = tensor(c, t, letters, types, type, strides, 0);
    h.batch_stride = strides[0], h.token_stride = strides[1], h.head_stride = strides[2];
    return h;
}

/* A cache's handle: (address of its description, B, G, D, S, dtype): batch, heads, head_dim, slots */
static const fgmp_cache_t *cache_of(call_t *c, PyObject *handle, int *types)
{
    if (c->bad || !PyTuple_Check(handle) || PyTuple_GET_SIZE(handle) != 6) {
        c->bad = 1;
        return NULL;
    }
    for (int i = 0; i < 4; ++i) {
        *letter(c, "BGDS"[i]) = PyLong_AsLongLong(PyTuple_GET_ITEM(handle, i + 1));
    }
    *types = PyTuple_GET_ITEM(handle, 5) == c->types[F32] ? 1 << F32 : 1 << BF16;
    const fgmp_cache_t *const p = PyLong_AsVoidPtr(PyTuple_GET_ITEM(handle, 0));
    if (PyErr_Occurred()) c->bad = 1;
    return p;
}

static void *address(call_t *c, PyObject *o)
{
    if (c->bad) return NULL;
    void *const p = PyLong_Check(o) ? PyLong_AsVoidPtr(o) : NULL;
    if (!PyLong_Check(o) || PyErr_Occurred()) c->bad = 1;
    return p;
}

static int64_t whole(call_t *c, PyObject *o)
{
    Py_INCREF(o);
    if (c->bad) {
        Py_DECREF(o);
        return 0;
    }
    return integer(o, &c->bad);
}

static PyObject *result(call_t *c, int rc)
{
    if (!c->bad) return PyLong_FromLong(rc);
    PyErr_Clear();
    Py_RETURN_NONE;
}

#define ARGUMENTS(count)                                              \
    (void)self;                                                       \
    if (n != (count)) {                                               \
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); \
        return NULL;                                                  \
    }                                                                 \
    call_t c;                                                         \
    int rc = 0;                                                       \
    begin(&c, a[1]);

/* (entry, types, q, k, v, cache, tree, counts, scale, max_length, out, lse, workspace, stream) */
static PyObject *tree_attention(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    ARGUMENTS(14)
    int types = 0;
    const fgmp_cache_t *const cache = cache_of(&c, a[5], &types);
    const fgmp_heads_t q = heads(&c, a[2], "BTHD", types, NULL), out = heads(&c, a[10], "BTHD", types, NULL);
    const int with_new = a[3] != Py_None || a[4] != Py_None;
    fgmp_heads_t k = {NULL, 0, 0, 0}, v = {NULL, 0, 0, 0};
    if (with_new) {
        k = heads(&c, a[3], "BTGD", types, NULL);
        v = heads(&c, a[4], "BTGD", types, NULL);
    }
    *letter(&c, 'W') = (*letter(&c, 'T') + 63) / 64;
    const uint64_t *const tree = tensor(&c, a[6], "BTW", 1 << I64, NULL, NULL, 1);
    const int32_t *const counts = tensor(&c, a[7], "B", 1 << I32, NULL, NULL, 1);
    const float scale = (float)number(a[8], &c.bad);
    const int64_t max_length = whole(&c, a[9]);
    float *const lse = tensor(&c, a[11], "BTH", 1 << F32, NULL, NULL, 0);
    void *const ws = tensor(&c, a[12], "N", 1 << U8, NULL, NULL, 0);
    void *const fn = address(&c, a[0]), *const stream = address(&c, a[13]);
    if (!c.bad) {
        Py_BEGIN_ALLOW_THREADS
        rc = ((__typeof__(&fgmp_tree_attention))fn)(&q, with_new ? &k : NULL, with_new ? &v : NULL, *letter(&c, 'T'), *letter(&c, 'H'), cache, tree, counts,
                                                   scale, max_length, &out, lse, ws, (size_t)*letter(&c, 'N'), stream);
        Py_END_ALLOW_THREADS
    }
    return result(&c, rc);
}

/* (entry, types, q, lse, cache, weights, rows, counts, scale, max_length, out, stream) */
static PyObject *attention_weights(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    ARGUMENTS(12)
    int types = 0;
    const fgmp_cache_t *const cache = cache_of(&c, a[4], &types);
    const fgmp_heads_t q = heads(&c, a[2], "BTHD", types, NULL);
    const float *const lse = tensor(&c, a[3], "BTH", 1 << F32, NULL, NULL, 0);
    const float *const weights = tensor(&c, a[5], "BGL", 1 << F32, NULL, NULL, 0);
    if (a[6] == Py_None) *letter(&c, 'A') = *letter(&c, 'T');
    const int32_t *const rows = tensor(&c, a[6], "BA", 1 << I32, NULL, NULL, 1), *const counts = tensor(&c, a[7], "B", 1 << I32, NULL, NULL, 1);
    const float scale = (float)number(a[8], &c.bad);
    const int64_t max_length = whole(&c, a[9]);
    float *const out = tensor(&c, a[10], "BGL", 1 << F32, NULL, NULL, 0);
    void *const fn = address(&c, a[0]), *const stream = address(&c, a[11]);
    if (!c.bad) {
        Py_BEGIN_ALLOW_THREADS
        rc = ((__typeof__(&fgmp_attention_weights))fn)(&q, lse, *letter(&c, 'T'), *letter(&c, 'H'), cache, rows, *letter(&c, 'A'), counts, scale, max_length,
                                                      weights, out, *letter(&c, 'L'), stream);
        Py_END_ALLOW_THREADS
    }
    return result(&c, rc);
}

/* (entry, types, k, v, cache, rows, counts, positions, slot_positions, slot_weights, lengths_out, stream) */
static PyObject *cache_append(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    ARGUMENTS(12)
    int types = 0, type = 0, other = 0;
    const fgmp_cache_t *const cache = cache_of(&c, a[4], &types);
    const fgmp_heads_t k = heads(&c, a[2], "BTGD", 1 << F32 | 1 << BF16, &type), v = heads(&c, a[3], "BTGD", 1 << F32 | 1 << BF16, &other);
    if (type != other) c.bad = 1;
    if (a[5] == Py_None) *letter(&c, 'A') = *letter(&c, 'T');
    const int32_t *const rows = tensor(&c, a[5], "BA", 1 << I32, NULL, NULL, 1), *const counts = tensor(&c, a[6], "B", 1 << I32, NULL, NULL, 1);
    const int32_t *const positions = tensor(&c, a[7], "BT", 1 << I32, NULL, NULL, 1);
    int32_t *const slot_positions = tensor(&c, a[8], "BGL", 1 << I32, NULL, NULL, 1);
    float *const slot_weights = tensor(&c, a[9], "BGL", 1 << F32, NULL, NULL, 1);
    int32_t *const lengths = tensor(&c, a[10], "B", 1 << I32, NULL, NULL, 0);
    void *const fn = address(&c, a[0]), *const stream = address(&c, a[11]);
    if (!c.bad) {
        Py_BEGIN_ALLOW_THREADS
        rc = ((__typeof__(&fgmp_cache_append))fn)(&k, &v, type == F32 ? FGMP_F32 : FGMP_BF16, *letter(&c, 'T'), cache, rows, *letter(&c, 'A'), counts, positions,
                                                 slot_positions, slot_weights, *letter(&c, 'L') < 0 ? 0 : *letter(&c, 'L'), lengths, stream);
        Py_END_ALLOW_THREADS
    }
    return result(&c, rc);
}

/* (entry, types, cache, weights, positions, seen, budget, sinks, recent, weights_out, positions_out, lengths_out, workspace, stream) */
static PyObject *cache_evict(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    ARGUMENTS(14)
    int types = 0;
    const fgmp_cache_t *const cache = cache_of(&c, a[2], &types);
    const float *const weights = tensor(&c, a[3], "BGL", 1 << F32, NULL, NULL, 0);
    const int32_t *const positions = tensor(&c, a[4], "BGL", 1 << I32, NULL, NULL, 0), *const seen = tensor(&c, a[5], "B", 1 << I32, NULL, NULL, 0);
    const int64_t budget = whole(&c, a[6]), sinks = whole(&c, a[7]), recent = whole(&c, a[8]);
    float *const weights_out = tensor(&c, a[9], "BGL", 1 << F32, NULL, NULL, 0);
    int32_t *const positions_out = tensor(&c, a[10], "BGL", 1 << I32, NULL, NULL, 0), *const lengths = tensor(&c, a[11], "B", 1 << I32, NULL, NULL, 0);
    void *const ws = tensor(&c, a[12], "N", 1 << U8, NULL, NULL, 0);
    void *const fn = address(&c, a[0]), *const stream = address(&c, a[13]);
    if (!c.bad) {
        Py_BEGIN_ALLOW_THREADS
        rc = ((__typeof__(&fgmp_cache_evict))fn)(cache, weights, positions, *letter(&c, 'L'), seen, budget, sinks, recent, weights_out, positions_out, lengths, ws,
                                                (size_t)*letter(&c, 'N'), stream);
        Py_END_ALLOW_THREADS
    }
    return result(&c, rc);
}

/* (entry, types, x, o, gate, gate_rows, gate_act, post_weight, post_bias, pre_weight, pre_bias, kind, eps, residual_scale, branch_scale, y, h,
 * stream); gate with rows, gate_rows > 0 */
static PyObject *block_norm(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    ARGUMENTS(18)
    const int either = 1 << F32 | 1 << BF16;
    int x_type = 0, o_type = 0, h_type = 0;
    int64_t ldx = 0, ldo = 0, ldg = 0, ldy = 0, ldh = 0;
    const void *const x = tensor(&c, a[2], "MK", either, &x_type, &ldx, 0), *const o = tensor(&c, a[3], "MK", either, &o_type, &ldo, 1);
    const void *const gate = tensor(&c, a[4], "RK", 1 << o_type, NULL, &ldg, 1);
    const int64_t gate_rows = whole(&c, a[5]), act = whole(&c, a[6]), kind = whole(&c, a[11]);
    if (gate != NULL && (o == NULL || gate_rows <= 0 || *letter(&c, 'R') < (*letter(&c, 'M') + gate_rows - 1) / gate_rows)) c.bad = 1;
    const float *vectors[4];
    for (int i = 0; i < 4; ++i) vectors[i] = tensor(&c, a[7 + i], "K", 1 << F32, NULL, NULL, 1);
    const float eps = (float)number(a[12], &c.bad), residual = (float)number(a[13], &c.bad), branch = (float)number(a[14], &c.bad);
    void *const y = tensor(&c, a[15], "MK", 1 << x_type, NULL, &ldy, 1), *const h = tensor(&c, a[16], "MK", either, &h_type, &ldh, 1);
    void *const fn = address(&c, a[0]), *const stream = address(&c, a[17]);
    if (!c.bad) {
        Py_BEGIN_ALLOW_THREADS
        rc = ((__typeof__(&fgmp_block_norm))fn)(x, x_type == F32 ? FGMP_F32 : FGMP_BF16, ldx, o, o_type == F32 ? FGMP_F32 : FGMP_BF16, ldo, gate, ldg, gate_rows,
                                               (fgmp_gate_t)act, *letter(&c, 'M'), *letter(&c, 'K'), vectors[0], vectors[1], vectors[2], vectors[3],
                                               (fgmp_norm_t)kind, eps, residual, branch, y, ldy, h, h_type == F32 ? FGMP_F32 : FGMP_BF16, ldh, stream);
        Py_END_ALLOW_THREADS
    }
    return result(&c, rc);
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(quant_gemm_fused), METHOD(tree_attention), METHOD(attention_weights), METHOD(cache_append), METHOD(cache_evict),
                                METHOD(block_norm), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fgmp_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__fgmp_call(void)
{
    struct { PyObject **at; const char *name; } const names[] = {{&s_is_cuda, "is_cuda"}, {&s_shape, "shape"}, {&s_dtype, "dtype"},
        {&s_data_ptr, "data_ptr"}, {&s_stride, "stride"}, {&s_numel, "numel"}, {&s_K, "K"}, {&s_rows, "rows"}, {&s_buf, "buf"}};
    for (size_t i = 0; i < sizeof names / sizeof names[0]; ++i)
        if ((*names[i].at = PyUnicode_InternFromString(names[i].name)) == NULL) return NULL;
    if ((zero = PyLong_FromLong(0)) == NULL) return NULL;
    return PyModule_Create(&module);
}
