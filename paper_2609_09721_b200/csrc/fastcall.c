/* Call path from Python into the C ABI for the entry points that a serving loop calls per step: a CPython extension that
 * takes plain integers (addresses, sizes, a stream) and passes them on.  Marshalling only, like the ctypes binding beside
 * it, which costs 2.3 microseconds for the 17 arguments of a forward (and tens for the prefix sums of a packed batch)
 * where this takes a few tenths.  The library is not linked: the binding hands over the addresses of its functions.
 * As in ctypes, the interpreter lock is released around every call: a launch waits while the stream's queue is full, and the
 * table copy of a packed batch may wait for the stream, and neither may stop the other threads of a server. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <stdlib.h>

#include "efq.h"

typedef efq_status_t (*attention_fn)(const void*, const void*, const void*, float*, int, int, int, int64_t, int64_t, int, int,
                                     float, const efq_params_t*, void*, size_t, const efq_debug_t*, void*);
typedef efq_status_t (*etq_attention_fn)(const void*, const void*, const void*, float*, int, int, int, int64_t, int64_t, int, int,
                                         float, int, void*, size_t, const efq_debug_t*, void*);
typedef efq_status_t (*probgen_fn)(const float*, int64_t, const float*, int64_t, int64_t, float, const efq_params_t*, uint8_t*,
                                   uint8_t*, void*);
typedef efq_status_t (*etq_probgen_fn)(const float*, int64_t, const float*, int64_t, int64_t, float, int, uint8_t*, uint8_t*, void*);
typedef efq_status_t (*varlen_fn)(const void*, const void*, const void*, float*, const int64_t*, const int64_t*, int, int, int, int,
                                  int, float, int, const efq_params_t*, void*, size_t, void*);
typedef size_t (*varlen_bytes_fn)(const int64_t*, const int64_t*, int, int, int, int);

typedef efq_status_t (*rotary_fn)(const efq_rows_t*, const efq_rows_t*, const int32_t*, int64_t, int64_t, int, int64_t, int, int,
                                  const efq_rotary_t*, int, void*);
typedef efq_status_t (*paged_append_fn)(const efq_rows_t*, const efq_rows_t*, const efq_rows_t*, int64_t, const int32_t*, int64_t,
                                        const efq_paged_t*, int, int, const efq_rotary_t*, void*);
typedef efq_status_t (*paged_attention_fn)(const efq_rows_t*, float*, int64_t, int, const efq_paged_t*, int, int, int, float, void*, size_t, void*);

static struct {
    attention_fn attention;
    etq_attention_fn etq_attention;
    probgen_fn probgen;
    etq_probgen_fn etq_probgen;
    varlen_fn varlen;
    varlen_bytes_fn varlen_bytes;
} fn;
static struct {
    rotary_fn rotary;
    paged_append_fn append;
    paged_attention_fn attention;
} paged_fn;

/* The call without the interpreter lock; its arguments are plain C values by then. */
#define UNLOCKED(type, call) type st; Py_BEGIN_ALLOW_THREADS st = call; Py_END_ALLOW_THREADS

/* Arguments are converted first and errors looked at once: a conversion that fails leaves the exception set. */
static void* ptr(PyObject* o) { return o == Py_None ? NULL : (void*)(uintptr_t)PyLong_AsUnsignedLongLong(o); }
static int64_t i64(PyObject* o) { return PyLong_AsLongLong(o); }
static int i32(PyObject* o) { return (int)PyLong_AsLong(o); }
static float f32(PyObject* o) { return (float)PyFloat_AsDouble(o); }

static int want(Py_ssize_t got, Py_ssize_t n)
{
    if (fn.attention == NULL) { PyErr_SetString(PyExc_RuntimeError, "efq_fastcall: the library's functions have not been set"); return 0; }
    if (got != n) { PyErr_Format(PyExc_TypeError, "efq_fastcall: %zd arguments expected, got %zd", n, got); return 0; }
    return 1;
}

static PyObject* set_functions(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    if (n != 6) { PyErr_SetString(PyExc_TypeError, "efq_fastcall.set_functions: six addresses expected"); return NULL; }
    fn.attention = (attention_fn)ptr(a[0]);
    fn.etq_attention = (etq_attention_fn)ptr(a[1]);
    fn.probgen = (probgen_fn)ptr(a[2]);
    fn.etq_probgen = (etq_probgen_fn)ptr(a[3]);
    fn.varlen = (varlen_fn)ptr(a[4]);
    fn.varlen_bytes = (varlen_bytes_fn)ptr(a[5]);
    if (PyErr_Occurred()) return NULL;
    Py_RETURN_NONE;
}

/* q, k, v, o, B, Hq, Hkv, Sq, Sk, d, causal, scale, params or scale mode, workspace, bytes, debug, stream */
static PyObject* attention(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    if (!want(n, 17)) return NULL;
    void *q = ptr(a[0]), *k = ptr(a[1]), *v = ptr(a[2]), *o = ptr(a[3]);
    const int B = i32(a[4]), Hq = i32(a[5]), Hkv = i32(a[6]), d = i32(a[9]), causal = i32(a[10]);
    const int64_t Sq = i64(a[7]), Sk = i64(a[8]), bytes = i64(a[14]);
    const float scale = f32(a[11]);
    void *params = ptr(a[12]), *ws = ptr(a[13]), *debug = ptr(a[15]), *stream = ptr(a[16]);
    if (PyErr_Occurred()) return NULL;
    UNLOCKED(efq_status_t, fn.attention(q, k, v, o, B, Hq, Hkv, Sq, Sk, d, causal, scale, params, ws, (size_t)bytes, debug, stream))
    return PyLong_FromLong(st);
}

static PyObject* etq_attention(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    if (!want(n, 17)) return NULL;
    void *q = ptr(a[0]), *k = ptr(a[1]), *v = ptr(a[2]), *o = ptr(a[3]);
    const int B = i32(a[4]), Hq = i32(a[5]), Hkv = i32(a[6]), d = i32(a[9]), causal = i32(a[10]), mode = i32(a[12]);
    const int64_t Sq = i64(a[7]), Sk = i64(a[8]), bytes = i64(a[14]);
    const float scale = f32(a[11]);
    void *ws = ptr(a[13]), *debug = ptr(a[15]), *stream = ptr(a[16]);
    if (PyErr_Occurred()) return NULL;
    UNLOCKED(efq_status_t, fn.etq_attention(q, k, v, o, B, Hq, Hkv, Sq, Sk, d, causal, scale, mode, ws, (size_t)bytes, debug, stream))
    return PyLong_FromLong(st);
}

/* scores, ld, row_max, rows, cols, scale, params or scale mode, codes, scales, stream */
static PyObject* probgen(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    if (!want(n, 10)) return NULL;
    void *scores = ptr(a[0]), *row_max = ptr(a[2]), *params = ptr(a[6]), *codes = ptr(a[7]), *scales = ptr(a[8]), *stream = ptr(a[9]);
    const int64_t ld = i64(a[1]), rows = i64(a[3]), cols = i64(a[4]);
    const float scale = f32(a[5]);
    if (PyErr_Occurred()) return NULL;
    UNLOCKED(efq_status_t, fn.probgen(scores, ld, row_max, rows, cols, scale, params, codes, scales, stream))
    return PyLong_FromLong(st);
}

static PyObject* etq_probgen(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    if (!want(n, 10)) return NULL;
    void *scores = ptr(a[0]), *row_max = ptr(a[2]), *codes = ptr(a[7]), *scales = ptr(a[8]), *stream = ptr(a[9]);
    const int64_t ld = i64(a[1]), rows = i64(a[3]), cols = i64(a[4]);
    const float scale = f32(a[5]);
    const int mode = i32(a[6]);
    if (PyErr_Occurred()) return NULL;
    UNLOCKED(efq_status_t, fn.etq_probgen(scores, ld, row_max, rows, cols, scale, mode, codes, scales, stream))
    return PyLong_FromLong(st);
}

/* A sequence of integers as a C array; NULL with an exception set on failure. */
static int64_t* to_array(PyObject* o, Py_ssize_t* n)
{
    PyObject* s = PySequence_Fast(o, "prefix sums have to be a sequence of integers");
    if (s == NULL) return NULL;
    *n = PySequence_Fast_GET_SIZE(s);
    int64_t* out = malloc(sizeof(int64_t) * (size_t)(*n > 0 ? *n : 1));
    if (out == NULL) { Py_DECREF(s); PyErr_NoMemory(); return NULL; }
    PyObject** items = PySequence_Fast_ITEMS(s);
    for (Py_ssize_t i = 0; i < *n; ++i) {
        if (PyLong_CheckExact(items[i])) {
            out[i] = PyLong_AsLongLong(items[i]);
        } else {                                     /* numpy and torch integers */
            PyObject* x = PyNumber_Long(items[i]);
            out[i] = x == NULL ? -1 : PyLong_AsLongLong(x);
            Py_XDECREF(x);
        }
        if (out[i] == -1 && PyErr_Occurred()) { free(out); Py_DECREF(s); return NULL; }
    }
    Py_DECREF(s);
    return out;
}

/* cu_q, cu_k, total_q, total_k, Hq, Hkv, d, q, k, v, o, causal, scale, producer, params, workspace, bytes, stream
 * -> status, or -1 if the prefix sums do not fit the tensors.  With q None: the bytes the workspace has to have. */
static PyObject* varlen(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    if (!want(n, 18)) return NULL;
    Py_ssize_t nq = 0, nk = 0;
    int64_t* cq = to_array(a[0], &nq);
    if (cq == NULL) return NULL;
    int64_t* ck = to_array(a[1], &nk);
    if (ck == NULL) { free(cq); return NULL; }
    const int64_t total_q = i64(a[2]), total_k = i64(a[3]), bytes = i64(a[16]);
    const int Hq = i32(a[4]), Hkv = i32(a[5]), d = i32(a[6]), causal = i32(a[11]), producer = i32(a[13]);
    void *q = ptr(a[7]), *k = ptr(a[8]), *v = ptr(a[9]), *o = ptr(a[10]), *params = ptr(a[14]), *ws = ptr(a[15]), *stream = ptr(a[17]);
    const float scale = f32(a[12]);
    PyObject* result = NULL;
    if (!PyErr_Occurred()) {
        if (nq < 1 || nk != nq || cq[nq - 1] != total_q || ck[nk - 1] != total_k) {
            result = PyLong_FromLong(-1);
        } else if (a[7] == Py_None) {
            UNLOCKED(size_t, fn.varlen_bytes(cq, ck, (int)(nq - 1), Hq, Hkv, d))
            result = PyLong_FromSize_t(st);
        } else {
            UNLOCKED(efq_status_t, fn.varlen(q, k, v, o, cq, ck, (int)(nq - 1), Hq, Hkv, d, causal, scale, producer, params, ws, (size_t)bytes, stream))
            result = PyLong_FromLong(st);
        }
    }
    free(cq);
    free(ck);
    return result;
}

static PyObject* set_paged_functions(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    if (n != 3) { PyErr_SetString(PyExc_TypeError, "efq_fastcall.set_paged_functions: three addresses expected"); return NULL; }
    paged_fn.rotary = (rotary_fn)ptr(a[0]);
    paged_fn.append = (paged_append_fn)ptr(a[1]);
    paged_fn.attention = (paged_attention_fn)ptr(a[2]);
    if (PyErr_Occurred()) return NULL;
    Py_RETURN_NONE;
}

static int want_paged(Py_ssize_t got, Py_ssize_t n)
{
    if (paged_fn.rotary == NULL) { PyErr_SetString(PyExc_RuntimeError, "efq_fastcall: the library's functions have not been set"); return 0; }
    if (got != n) { PyErr_Format(PyExc_TypeError, "efq_fastcall: %zd arguments expected, got %zd", n, got); return 0; }
    return 1;
}

/* A tensor's shape or strides as `n` integers. */
static int dims(PyObject* o, int64_t* out, Py_ssize_t n)
{
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != n) { PyErr_Format(PyExc_TypeError, "efq_fastcall: a tuple of %zd integers expected", n); return 0; }
    for (Py_ssize_t i = 0; i < n; ++i) out[i] = i64(PyTuple_GET_ITEM(o, i));
    return !PyErr_Occurred();
}

/* Rows from (src, dst, shape, strides of src, strides of dst); src None: no tensor.  The shapes are [B, H, S, d] or, token-major
 * without a batch, [total, H, d]. */
#define GROUP 5
static int rows4(PyObject* const* a, efq_rows_t* r)
{
    int64_t shape[4], s[4], t[4];
    if (a[0] == Py_None) return 0;
    r->src = ptr(a[0]);
    r->dst = ptr(a[1]);
    if (!dims(a[2], shape, 4) || !dims(a[3], s, 4) || !dims(a[4], t, 4)) return -1;
    r->heads = (int32_t)shape[1];
    r->src_batch = s[0]; r->src_head = s[1]; r->src_token = s[2];
    r->dst_batch = t[0]; r->dst_head = t[1]; r->dst_token = t[2];
    return 1;
}
static int rows3(PyObject* const* a, efq_rows_t* r)
{
    int64_t shape[3], s[3], t[3];
    if (a[0] == Py_None) return 0;
    r->src = ptr(a[0]);
    r->dst = ptr(a[1]);
    if (!dims(a[2], shape, 3) || !dims(a[3], s, 3) || !dims(a[4], t, 3)) return -1;
    r->heads = (int32_t)shape[1];
    r->src_batch = r->dst_batch = 0;
    r->src_head = s[1]; r->src_token = s[0];
    r->dst_head = t[1]; r->dst_token = t[0];
    return 1;
}
/* The cache from (k, v, shape of both, strides of k, of v, page_table, its shape, its strides, cu_seqlens, seq_lens). */
#define CACHE 10
static int cache_of(PyObject* const* a, efq_paged_t* c)
{
    int64_t shape[4], s[4], t[4], table[2], ts[2];
    c->k = ptr(a[0]);
    c->v = ptr(a[1]);
    if (!dims(a[2], shape, 4) || !dims(a[3], s, 4) || !dims(a[4], t, 4) || !dims(a[6], table, 2) || !dims(a[7], ts, 2)) return 0;
    if (shape[0] > INT32_MAX || shape[1] > INT32_MAX || shape[2] > INT32_MAX || table[0] > INT32_MAX || table[1] > INT32_MAX) {
        PyErr_SetString(PyExc_ValueError, "efq_fastcall: the cache has a dimension of more than 32 bits");
        return 0;
    }
    c->n_pages = (int32_t)shape[0]; c->n_heads = (int32_t)shape[1]; c->page_size = (int32_t)shape[2];
    c->k_page = s[0]; c->k_head = s[1]; c->k_token = s[2];
    c->v_page = t[0]; c->v_head = t[1]; c->v_token = t[2];
    c->page_table = ptr(a[5]);
    c->n_seqs = (int32_t)table[0];
    c->max_pages = (int32_t)table[1];
    c->table_stride = ts[0];
    c->cu_seqlens = ptr(a[8]);
    c->seq_lens = ptr(a[9]);
    return !PyErr_Occurred();
}

/* q rows, k rows, positions, strides of axis and batch, B, S, dtype, rotary, inverse, stream */
static PyObject* rotary(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    if (!want_paged(n, 2 * GROUP + 9)) return NULL;
    efq_rows_t q = {0}, k = {0};
    const int has_q = rows4(a, &q), has_k = rows4(a + GROUP, &k);
    if (has_q < 0 || has_k < 0) return NULL;
    a += 2 * GROUP;
    void *positions = ptr(a[0]), *rotation = ptr(a[6]), *stream = ptr(a[8]);
    const int64_t axis = i64(a[1]), batch = i64(a[2]), S = i64(a[4]);
    const int B = i32(a[3]), dtype = i32(a[5]), inverse = i32(a[7]);
    if (PyErr_Occurred()) return NULL;
    UNLOCKED(efq_status_t, paged_fn.rotary(has_q ? &q : NULL, has_k ? &k : NULL, positions, axis, batch, B, S, 128, dtype, rotation, inverse, stream))
    return PyLong_FromLong(st);
}

/* k rows, v rows, q rows, total, positions, stride of axis, cache, dtype, rotary, stream */
static PyObject* paged_append(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    if (!want_paged(n, 3 * GROUP + 3 + CACHE + 3)) return NULL;
    efq_rows_t k = {0}, v = {0}, q = {0};
    efq_paged_t cache = {0};
    const int has_k = rows3(a, &k), has_v = rows3(a + GROUP, &v), has_q = rows3(a + 2 * GROUP, &q);
    if (has_k < 0 || has_v < 0 || has_q < 0) return NULL;
    a += 3 * GROUP;
    const int64_t total = i64(a[0]), axis = i64(a[2]);
    void* positions = ptr(a[1]);
    if (!cache_of(a + 3, &cache)) return NULL;
    a += 3 + CACHE;
    const int dtype = i32(a[0]);
    void *rotation = ptr(a[1]), *stream = ptr(a[2]);
    if (PyErr_Occurred()) return NULL;
    UNLOCKED(efq_status_t, paged_fn.append(has_k ? &k : NULL, has_v ? &v : NULL, has_q ? &q : NULL, total, positions, axis, &cache, 128, dtype, rotation, stream))
    return PyLong_FromLong(st);
}

/* q rows, lse, total, max_seqlen_q, cache, dtype, causal, scale, workspace, bytes, stream */
static PyObject* paged_attention(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    (void)self;
    if (!want_paged(n, GROUP + 3 + CACHE + 6)) return NULL;
    efq_rows_t q = {0};
    efq_paged_t cache = {0};
    const int has_q = rows3(a, &q);
    if (has_q < 0) return NULL;
    a += GROUP;
    void* lse = ptr(a[0]);
    const int64_t total = i64(a[1]);
    const int max_q = i32(a[2]);
    if (!cache_of(a + 3, &cache)) return NULL;
    a += 3 + CACHE;
    const int dtype = i32(a[0]), causal = i32(a[1]);
    const float scale = f32(a[2]);
    void *ws = ptr(a[3]), *stream = ptr(a[5]);
    const int64_t bytes = i64(a[4]);
    if (PyErr_Occurred()) return NULL;
    UNLOCKED(efq_status_t, paged_fn.attention(has_q ? &q : NULL, lse, total, max_q, &cache, 128, dtype, causal, scale, ws, (size_t)bytes, stream))
    return PyLong_FromLong(st);
}

static PyMethodDef methods[] = {
    {"set_functions", (PyCFunction)(void (*)(void))set_functions, METH_FASTCALL, NULL},
    {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, NULL},
    {"etq_attention", (PyCFunction)(void (*)(void))etq_attention, METH_FASTCALL, NULL},
    {"probgen", (PyCFunction)(void (*)(void))probgen, METH_FASTCALL, NULL},
    {"etq_probgen", (PyCFunction)(void (*)(void))etq_probgen, METH_FASTCALL, NULL},
    {"varlen", (PyCFunction)(void (*)(void))varlen, METH_FASTCALL, NULL},
    {"set_paged_functions", (PyCFunction)(void (*)(void))set_paged_functions, METH_FASTCALL, NULL},
    {"rotary", (PyCFunction)(void (*)(void))rotary, METH_FASTCALL, NULL},
    {"paged_append", (PyCFunction)(void (*)(void))paged_append, METH_FASTCALL, NULL},
    {"paged_attention", (PyCFunction)(void (*)(void))paged_attention, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "efq_fastcall", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit_efq_fastcall(void) { return PyModule_Create(&module); }
