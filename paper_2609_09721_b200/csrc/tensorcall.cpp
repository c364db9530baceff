// Call path from Python into the C ABI for the operators around a paged cache: a CPython extension that takes torch tensors.  Their calls
// describe up to eleven tensors by address, shape and strides; asking for those in Python took 9 microseconds a call, several times what
// the smallest of them needs on the GPU.  Marshalling only, like the binding beside it: the tensors are looked at here, what they have to be is an
// AssertionError, and the library's status is returned.  The library is not linked: the binding hands over the addresses of its
// functions.  The interpreter lock is released around every call, since a launch waits while the stream's queue is full.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include "efq.h"

namespace {

decltype(&efq_rotary) rotary_fn;
decltype(&efq_paged_append) append_fn;
decltype(&efq_paged_attention_fwd) attention_fn;

constexpr int64_t kD = 128;

// What the arguments are not: set once, the first of them.
struct Checked {
    const char* wrong = nullptr;
    int64_t device;             // the current one, whose stream the call goes to
    at::ScalarType type = at::kBFloat16;

    bool want(bool holds, const char* otherwise)
    {
        if (!holds && wrong == nullptr) wrong = otherwise;
        return wrong == nullptr;
    }
    // null for None; anything else has to be a tensor on the current device
    const at::Tensor* tensor(PyObject* o, const char* otherwise)
    {
        if (o == Py_None) return nullptr;
        if (!want(THPVariable_Check(o), otherwise)) return nullptr;
        const at::Tensor& t = THPVariable_Unpack(o);
        want(t.is_cuda() && t.get_device() == device, "tensors have to be on the current CUDA device");
        return &t;
    }
    const at::Tensor* needed(PyObject* o, const char* otherwise)
    {
        const at::Tensor* t = tensor(o, otherwise);
        want(t != nullptr, otherwise);
        return t;
    }
    bool channels(const at::Tensor& t, int64_t dims, const char* otherwise)
    {
        return want(t.dim() == dims && t.size(dims - 1) == kD && (t.stride(dims - 1) == 1 || t.numel() == 0) && t.scalar_type() == type, otherwise);
    }
    bool ints(const at::Tensor& t, int64_t dims, const char* otherwise)
    {
        return want(t.dim() == dims && t.scalar_type() == at::kInt && (t.size(dims - 1) <= 1 || t.stride(dims - 1) == 1), otherwise);
    }
    void set_type(const at::Tensor& t)
    {
        type = t.scalar_type();
        want(type == at::kBFloat16 || type == at::kHalf, "elements have to be bfloat16 or float16");
    }
    int dtype() const { return type == at::kHalf ? EFQ_FP16 : EFQ_BF16; }
};

PyObject* refused(const Checked& c)
{
    PyErr_SetString(PyExc_AssertionError, c.wrong);
    return nullptr;
}
bool count(Py_ssize_t got, Py_ssize_t n)
{
    if (attention_fn == nullptr) PyErr_SetString(PyExc_RuntimeError, "efq_tensorcall: the library's functions have not been set");
    else if (got != n) PyErr_Format(PyExc_TypeError, "efq_tensorcall: %zd arguments expected, got %zd", n, got);
    else return true;
    return false;
}
void* address(PyObject* o) { return o == Py_None ? nullptr : reinterpret_cast<void*>(static_cast<uintptr_t>(PyLong_AsUnsignedLongLong(o))); }
int64_t number(PyObject* o) { return PyLong_AsLongLong(o); }

PyObject* set_functions(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "efq_tensorcall.set_functions: three addresses expected");
        return nullptr;
    }
    void* f[3] = {address(a[0]), address(a[1]), address(a[2])};
    if (PyErr_Occurred()) return nullptr;
    rotary_fn = reinterpret_cast<decltype(rotary_fn)>(f[0]);
    append_fn = reinterpret_cast<decltype(append_fn)>(f[1]);
    attention_fn = reinterpret_cast<decltype(attention_fn)>(f[2]);
    Py_RETURN_NONE;
}

// [B, heads, S, 128] and its output; false: no tensor
bool rows4(Checked& c, PyObject* src, PyObject* dst, int64_t B, int64_t S, efq_rows_t& r)
{
    const at::Tensor* x = c.tensor(src, "q and k have to be tensors [B, heads, S, 128]");
    if (x == nullptr || !c.channels(*x, 4, "q and k have to be [B, heads, S, 128], of one type, their channels side by side")) return false;
    const at::Tensor* y = c.needed(dst, "q_out and k_out have to be tensors");
    if (y == nullptr || !c.channels(*y, 4, "q_out and k_out have to be of their input's type, their channels side by side")) return false;
    if (!c.want(x->size(0) == B && x->size(2) == S && x->size(1) <= INT32_MAX, "q and k have to be of the same batch and length")) return false;
    if (!c.want(y->sizes() == x->sizes(), "q_out and k_out have to be of their input's shape")) return false;
    r = {x->const_data_ptr(), y->data_ptr(), static_cast<int32_t>(x->size(1)), x->stride(0), x->stride(1), x->stride(2), y->stride(0), y->stride(1), y->stride(2)};
    return true;
}
// [total, heads, 128]
bool rows3(Checked& c, const at::Tensor& x, int64_t total, const char* otherwise, efq_rows_t& r)
{
    if (!c.channels(x, 3, otherwise) || !c.want(x.size(0) == total && x.size(1) <= INT32_MAX, otherwise)) return false;
    r.src = x.const_data_ptr();
    r.heads = static_cast<int32_t>(x.size(1));
    r.src_head = x.stride(1);
    r.src_token = x.stride(0);
    return true;
}
bool out3(Checked& c, PyObject* o, const at::Tensor& x, const char* otherwise, efq_rows_t& r)
{
    const at::Tensor* y = c.needed(o, otherwise);
    if (y == nullptr || !c.channels(*y, 3, otherwise) || !c.want(y->sizes() == x.sizes(), otherwise)) return false;
    r.dst = y->data_ptr();
    r.dst_head = y->stride(1);
    r.dst_token = y->stride(0);
    return true;
}
// k_cache, v_cache, page_table, cu_seqlens, seq_lens
constexpr Py_ssize_t kCacheArgs = 5;
bool cache_of(Checked& c, PyObject* const* a, efq_paged_t& p)
{
    const char* const what = "k_cache and v_cache have to be [pages, heads, page_size, 128], of one type with the tokens, their channels side by side";
    const char* const tables = "page_table, cu_seqlens and seq_lens have to be int32 tensors [n_seqs, max_pages], [n_seqs + 1] and [n_seqs]";
    const at::Tensor *k = c.needed(a[0], what), *v = c.needed(a[1], what), *table = c.needed(a[2], tables), *cu = c.needed(a[3], tables), *lens = c.needed(a[4], tables);
    if (c.wrong != nullptr) return false;
    if (!c.channels(*k, 4, what) || !c.channels(*v, 4, what) || !c.want(v->sizes() == k->sizes(), what)) return false;
    if (!c.ints(*table, 2, tables) || !c.ints(*cu, 1, tables) || !c.ints(*lens, 1, tables)) return false;
    if (!c.want(cu->size(0) == table->size(0) + 1 && lens->size(0) == table->size(0), tables)) return false;
    for (int i = 0; i < 3; ++i)
        if (!c.want(k->size(i) <= INT32_MAX, what)) return false;
    if (!c.want(table->size(0) <= INT32_MAX && table->size(1) <= INT32_MAX, tables)) return false;
    p.k = k->data_ptr();
    p.v = v->data_ptr();
    p.k_page = k->stride(0); p.k_head = k->stride(1); p.k_token = k->stride(2);
    p.v_page = v->stride(0); p.v_head = v->stride(1); p.v_token = v->stride(2);
    p.n_pages = static_cast<int32_t>(k->size(0));
    p.n_heads = static_cast<int32_t>(k->size(1));
    p.page_size = static_cast<int32_t>(k->size(2));
    p.page_table = static_cast<const int32_t*>(table->const_data_ptr());
    p.table_stride = table->stride(0);
    p.max_pages = static_cast<int32_t>(table->size(1));
    p.cu_seqlens = static_cast<const int32_t*>(cu->const_data_ptr());
    p.seq_lens = static_cast<const int32_t*>(lens->const_data_ptr());
    p.n_seqs = static_cast<int32_t>(table->size(0));
    return true;
}

#define UNLOCKED(call) \
    efq_status_t st; \
    Py_BEGIN_ALLOW_THREADS st = call; \
    Py_END_ALLOW_THREADS

// What a call has written counts as changed in place, so that autograd refuses a backward pass that has kept what stood there before.  Tensors of the
// inference mode have no count.
PyObject* wrote(efq_status_t st, std::initializer_list<PyObject*> outputs)
{
    for (PyObject* o : outputs)
        if (st == EFQ_OK && o != Py_None)
            if (const at::Tensor& t = THPVariable_Unpack(o); !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    return PyLong_FromLong(st);
}

// q, k, positions, rotary, inverse, q_out, k_out, device, stream
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (!count(n, 9)) return nullptr;
    Checked c;
    c.device = number(a[7]);
    const auto* const description = static_cast<const efq_rotary_t*>(address(a[3]));
    const int inverse = static_cast<int>(number(a[4]));
    void* const stream = address(a[8]);
    if (PyErr_Occurred()) return nullptr;
    efq_rows_t q{}, k{};
    const at::Tensor* const x = c.needed(a[0] != Py_None ? a[0] : a[1], "q or k has to be a tensor [B, heads, S, 128]");
    if (!c.want(x != nullptr && x->dim() == 4, "q and k have to be [B, heads, S, 128], of one type, their channels side by side")) return refused(c);
    c.set_type(*x);
    const int64_t B = x->size(0), S = x->size(2);
    const bool has_q = rows4(c, a[0], a[5], B, S, q), has_k = rows4(c, a[1], a[6], B, S, k);
    const char* const places = "positions have to be an int32 tensor [axes, S] or [axes, B, S]";
    const at::Tensor* const p = c.needed(a[2], places);
    if (c.wrong != nullptr) return refused(c);
    const bool batched = p->dim() == 3;
    c.ints(*p, batched ? 3 : 2, places);
    if (c.wrong == nullptr)
        c.want(description != nullptr && p->size(0) == description->n_axes && p->size(batched ? 2 : 1) == S && (!batched || p->size(1) == B), places);
    c.want(B <= INT32_MAX, "too many batch entries");
    if (c.wrong != nullptr) return refused(c);
    const int64_t axis = p->stride(0), batch = batched ? p->stride(1) : 0;
    UNLOCKED(rotary_fn(has_q ? &q : nullptr, has_k ? &k : nullptr, static_cast<const int32_t*>(p->const_data_ptr()), axis, batch, static_cast<int>(B), S, kD, c.dtype(),
                       description, inverse, stream))
    return wrote(st, {has_q ? a[5] : Py_None, has_k ? a[6] : Py_None});
}

// k, v, cache, rotary, positions, q, q_out, device, stream
PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (!count(n, 2 + kCacheArgs + 6)) return nullptr;
    PyObject* const* const b = a + 2 + kCacheArgs;
    Checked c;
    c.device = number(b[4]);
    const auto* const description = static_cast<const efq_rotary_t*>(address(b[0]));
    void* const stream = address(b[5]);
    if (PyErr_Occurred()) return nullptr;
    const char* const what = "k and v have to be [total, heads, 128], of one type, their channels side by side";
    const at::Tensor *const k = c.needed(a[0], what), *const v = c.needed(a[1], what);
    if (c.wrong != nullptr || !c.want(k->dim() == 3, what)) return refused(c);
    c.set_type(*k);
    const int64_t total = k->size(0);
    efq_rows_t kr{}, vr{}, qr{};
    efq_paged_t cache{};
    if (!rows3(c, *k, total, what, kr) || !rows3(c, *v, total, what, vr) || !cache_of(c, a + 2, cache)) return refused(c);
    c.want(kr.heads == cache.n_heads && vr.heads == kr.heads, "k and v have to have the cache's heads");
    const char* const queries = "q and q_out have to be [total, heads, 128], of the keys' type, their channels side by side";
    const at::Tensor* const q = c.tensor(b[2], queries);
    if (q != nullptr && c.wrong == nullptr && rows3(c, *q, total, queries, qr)) out3(c, b[3], *q, queries, qr);
    const char* const places = "positions have to be an int32 tensor [axes, total] of the rotation";
    const at::Tensor* const p = c.tensor(b[1], places);
    if (p != nullptr && c.wrong == nullptr && c.ints(*p, 2, places)) c.want(description != nullptr && p->size(0) == description->n_axes && p->size(1) == total, places);
    if (c.wrong != nullptr) return refused(c);
    UNLOCKED(append_fn(&kr, &vr, q != nullptr ? &qr : nullptr, total, p != nullptr ? static_cast<const int32_t*>(p->const_data_ptr()) : nullptr,
                       p != nullptr ? p->stride(0) : 0, &cache, kD, c.dtype(), description, stream))
    return wrote(st, {a[2], a[3], q != nullptr ? b[3] : Py_None});
}

// q, cache, max_seqlen_q, causal, scale, o, lse, workspace, device, stream
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (!count(n, 1 + kCacheArgs + 8)) return nullptr;
    PyObject* const* const b = a + 1 + kCacheArgs;
    Checked c;
    c.device = number(b[6]);
    const int64_t max_q = number(b[0]), causal = number(b[1]);
    const float scale = static_cast<float>(PyFloat_AsDouble(b[2]));
    void* const stream = address(b[7]);
    if (PyErr_Occurred()) return nullptr;
    const char* const what = "q has to be [total, heads, 128], its channels side by side";
    const at::Tensor* const q = c.needed(a[0], what);
    if (c.wrong != nullptr || !c.want(q->dim() == 3, what)) return refused(c);
    c.set_type(*q);
    c.want(max_q >= 0 && max_q <= INT32_MAX, "max_seqlen_q has to be a number of tokens");
    efq_rows_t qr{};
    efq_paged_t cache{};
    if (!rows3(c, *q, q->size(0), what, qr) || !out3(c, b[3], *q, "o has to be of q's shape and type, its channels side by side", qr) || !cache_of(c, a + 1, cache)) return refused(c);
    const char* const sums = "lse has to be a contiguous float32 tensor [total, heads]";
    const at::Tensor* const lse = c.tensor(b[4], sums);
    if (lse != nullptr && c.wrong == nullptr)
        c.want(lse->scalar_type() == at::kFloat && lse->dim() == 2 && lse->size(0) == q->size(0) && lse->size(1) == q->size(1) && lse->is_contiguous(), sums);
    const at::Tensor* const ws = c.needed(b[5], "workspace has to be a contiguous uint8 tensor");
    if (c.wrong == nullptr) c.want(ws->scalar_type() == at::kByte && ws->is_contiguous(), "workspace has to be a contiguous uint8 tensor");
    if (c.wrong != nullptr) return refused(c);
    UNLOCKED(attention_fn(&qr, lse != nullptr ? static_cast<float*>(lse->data_ptr()) : nullptr, q->size(0), static_cast<int>(max_q), &cache, kD, c.dtype(),
                          causal != 0, scale, ws->data_ptr(), static_cast<size_t>(ws->numel()), stream))
    return wrote(st, {b[3], b[4]});
}

template <PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    try {
        return f(self, a, n);
    } catch (const std::exception& e) {          // torch's own checks
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}
template <PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction method() { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(guarded<f>)); }

PyMethodDef methods[] = {
    {"set_functions", method<set_functions>(), METH_FASTCALL, nullptr},
    {"rotary", method<rotary>(), METH_FASTCALL, nullptr},
    {"paged_append", method<paged_append>(), METH_FASTCALL, nullptr},
    {"paged_attention", method<paged_attention>(), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "efq_tensorcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the torch and Python that it was compiled against, which the binding compares before the first call
PyMODINIT_FUNC PyInit_efq_tensorcall(void)
{
    PyObject* const m = PyModule_Create(&module);
    if (m != nullptr && PyModule_AddStringConstant(m, "built_for", EFQ_BUILT_FOR) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
