// The calls of api.py that a program makes between two launches, without the interpreter: arguments checked as api.py checks them, on the
// tensors themselves, and passed on.  A call whose arguments are not plainly right returns None without having done anything; api.py then makes
// it in its own way and says what is wrong.  What that saves (us a call in a row of them, with the launch, of which 3.4 are the runtime's): kv_fork_blk with
// its eleven tensors 7.6 -> 4.2, minikv_norm_rope of 9 tokens 7.9 -> 4.1.
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/core/Tensor.h>

#include <cstring>

#include "minikv.h"

namespace {

// One call's arguments, taken one after the other; `ok` until one is not right.
struct Args {
    PyObject *const *at;
    Py_ssize_t n, i = 0;
    bool ok = true;
    int64_t home = -1;                                 // the GPU that the call runs on

    PyObject *next()
    {
        if (i >= n) ok = false;
        return i < n ? at[i++] : Py_None;
    }
    int64_t integer()
    {
        PyObject *o = next();
        if (!PyLong_Check(o)) return ok = false, 0;
        int over = 0;
        const long long v = PyLong_AsLongLongAndOverflow(o, &over);
        if (over) ok = false;
        return v;
    }
    int32_t int32()
    {
        const int64_t v = integer();
        if (v != (int32_t)v) ok = false;
        return (int32_t)v;
    }
    float number()
    {
        PyObject *o = next();
        if (PyFloat_CheckExact(o)) return (float)PyFloat_AS_DOUBLE(o);
        ok = false;
        return 0.0f;
    }
    void *address() { return (void *)(uintptr_t)integer(); }           // of a stream or a ctypes structure
    const at::Tensor *tensor(PyObject *o)
    {
        if (!ok || !THPVariable_Check(o)) return ok = false, nullptr;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.defined() || t.layout() != at::kStrided || t.get_device() != home) return ok = false, nullptr;
        return &t;
    }
    // elements of `type` one behind the other, at least `least` of them
    template <typename T = int32_t> T *flat(int64_t least, at::ScalarType type = at::kInt, int64_t *count = nullptr)
    {
        const at::Tensor *t = tensor(next());
        if (!t || t->scalar_type() != type || t->numel() < least || !t->is_contiguous()) return ok = false, nullptr;
        if (count) *count = t->numel();
        return (T *)t->data_ptr();
    }
    template <typename T = int32_t> T *flat_or_none(int64_t least, at::ScalarType type)
    {
        if (i < n && at[i] == Py_None) return ++i, nullptr;
        return flat<T>(least, type);
    }
    // rows [tokens][heads][128], the heads of a token side by side: the elements between tokens in `stride`
    void *rows(int64_t least, int64_t heads, at::ScalarType type, int64_t &stride)
    {
        const at::Tensor *t = tensor(next());
        if (!t || t->scalar_type() != type || t->dim() != 3) return ok = false, nullptr;
        const auto size = t->sizes(), step = t->strides();
        if (size[0] < least || size[1] != heads || size[2] != 128 || step[2] != 1 || (step[1] != 128 && heads > 1)) return ok = false, nullptr;
        stride = size[0] > 1 ? step[0] : heads * 128;  // (one token: any stride will do)
        return t->data_ptr();
    }
    // memory that a call may use, in bytes
    void *space(size_t &bytes)
    {
        const at::Tensor *t = tensor(next());
        if (!t || !t->is_contiguous()) return ok = false, nullptr;
        bytes = t->nbytes();
        return t->data_ptr();
    }
    at::ScalarType peek_type() const
    {
        return i < n && THPVariable_Check(at[i]) ? THPVariable_Unpack(at[i]).scalar_type() : at::kByte;
    }
};

int32_t dtype_of(at::ScalarType t) { return t == at::kHalf ? MINIKV_F16 : t == at::kBFloat16 ? MINIKV_BF16 : -1; }
at::ScalarType type_of(int32_t dtype) { return dtype == MINIKV_F16 ? at::kHalf : dtype == MINIKV_BF16 ? at::kBFloat16 : at::kByte; }

template <int (*CALL)(Args &, void *)> PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a{args, n};
    int rc = 0;
    try {                                              // (home, stream, then the call's own)
        a.home = a.integer();
        void *stream = a.address();
        rc = a.ok ? CALL(a, stream) : 0;
    } catch (...) {
        a.ok = false;
    }
    if (PyErr_Occurred()) PyErr_Clear(), a.ok = false;
    if (!a.ok) Py_RETURN_NONE;
    return PyLong_FromLong(rc);
}
// The library's part, without the interpreter's lock; only if everything was taken and right
template <typename F> int made(Args &a, F f)
{
    if (a.i != a.n) a.ok = false;
    if (!a.ok) return 0;
    PyThreadState *state = PyEval_SaveThread();
    const int rc = f();
    PyEval_RestoreThread(state);
    return rc;
}

int norm_rope(Args &a, void *stream)
{
    const int32_t Hq = a.int32(), Hkv = a.int32(), T = a.int32();
    const at::ScalarType type = a.peek_type();
    int64_t qs = 0, ks = 0, qos = 0, kos = 0;
    const void *q = a.rows(T, Hq, type, qs), *k = a.rows(T, Hkv, type, ks), *wq = a.flat_or_none<void>(128, type), *wk = a.flat_or_none<void>(128, type);
    const float eps = a.number();
    PyObject *freq = a.next();
    const int32_t rot = a.int32();
    const float *inv = nullptr;
    if (rot) {
        const at::Tensor *t = a.tensor(freq);
        if (!t || t->scalar_type() != at::kFloat || t->numel() < rot / 2 || !t->is_contiguous()) return a.ok = false, 0;
        inv = (const float *)t->data_ptr();
    }
    const int truth = PyObject_IsTrue(a.next());
    if (truth < 0) a.ok = false;
    const int32_t *pos = a.flat(T);
    void *qo = a.rows(T, Hq, type, qos), *ko = a.rows(T, Hkv, type, kos);
    if (T == 1) qos = qo == q ? qs : qos, kos = ko == k ? ks : kos;     // (one row has no stride of its own)
    return made(a, [&] { return minikv_norm_rope(Hq, Hkv, T, dtype_of(type), q, qs, k, ks, wq, wk, eps, inv, rot, truth, pos, qo, qos, ko, kos, stream); });
}

// (addresses of structures that the caller holds)
int prompt_attn_blk(Args &a, void *stream)
{
    const auto *s = (const minikv_blk_shape *)a.address();
    const int32_t T = a.int32();
    if (!a.ok || T < 0) return a.ok = false, 0;
    int64_t qs = 0;
    const void *q = a.rows(T, s->Hq, type_of(s->dtype), qs);
    const auto *cache = (const minikv_blk_cache *)a.address();
    a.tensor(a.next());                                // (the cache's keys: where they are)
    const int32_t *table = a.flat((int64_t)s->R * s->max_blocks), *q_len = a.flat(s->R), *cu = a.flat((int64_t)s->R + 1);
    const float sm = a.number();
    void *out = a.flat<void>((int64_t)T * s->Hq * 128, type_of(s->dtype));
    float *lse = a.flat_or_none<float>((int64_t)T * s->Hq, at::kFloat);
    size_t bytes = 0;
    void *ws = a.space(bytes);
    return made(a, [&] { return minikv_prompt_attn_blk(s, T, q, qs, cache, table, q_len, cu, sm, out, lse, ws, bytes, stream); });
}

int fork_blk(Args &a, void *stream)
{
    const auto *s = (const minikv_blk_shape *)a.address();
    if (!a.ok) return 0;
    const int64_t R = s->R, rows = R * s->max_blocks;
    const int32_t *q_len = a.flat(R), *parent = a.flat(R), *n_keep = a.flat(R), *table = a.flat(rows), *ring = a.flat(s->n_blocks), *state = a.flat(2);
    int32_t *q_len_next = a.flat(R), *table_next = a.flat(rows), *state_next = a.flat(2), *src = a.flat(R), *dst = a.flat(R);
    return made(a, [&] { return kv_fork_blk(s, q_len, parent, n_keep, table, ring, state, q_len_next, table_next, state_next, src, dst, stream); });
}

int copy_blk(Args &a, void *stream)
{
    const auto *s = (const minikv_blk_shape *)a.address();
    const int32_t n_caches = a.int32();
    const auto *caches = (const minikv_blk_cache *)a.address();
    a.tensor(a.next());                                // (the first cache's keys: where they are)
    int64_t n = 0, m = 0;
    const int32_t *src = a.flat(0, at::kInt, &n), *dst = a.flat(0, at::kInt, &m);
    if (n != m || n != (int32_t)n) a.ok = false;
    return made(a, [&] { return kv_copy_blk(s, n_caches, caches, (int32_t)n, src, dst, stream); });
}

int free_blk(Args &a, void *stream)
{
    const auto *s = (const minikv_blk_shape *)a.address();
    if (!a.ok) return 0;
    const int32_t *q_len = a.flat(s->R), *table = a.flat((int64_t)s->R * s->max_blocks);
    int32_t *ring = a.flat(s->n_blocks), *state = a.flat(2);
    size_t bytes = 0;
    void *ws = a.space(bytes);
    return made(a, [&] { return kv_free_blk(s, q_len, table, ring, state, ws, bytes, stream); });
}

int compact_blk(Args &a, void *stream)
{
    const auto *s = (const minikv_blk_shape *)a.address();
    if (!a.ok) return 0;
    const int64_t rows = (int64_t)s->R * s->max_blocks;
    const int32_t *q_len = a.flat(s->R), *table = a.flat(rows);
    int32_t *table_next = a.flat(rows), *ring = a.flat(s->n_blocks), *state = a.flat(2);
    int64_t n = 0;
    int32_t *src = a.flat(0, at::kInt, &n), *dst = a.flat(n);
    if (n != (int32_t)n) a.ok = false;
    size_t bytes = 0;
    void *ws = a.space(bytes);
    return made(a, [&] { return kv_compact_blk(s, q_len, table, table_next, ring, state, (int32_t)n, src, dst, ws, bytes, stream); });
}

template <int (*CALL)(Args &, void *)> constexpr PyCFunction entry() { return (PyCFunction)(void *)call<CALL>; }
PyMethodDef methods[] = {
    {"norm_rope", entry<norm_rope>(), METH_FASTCALL, nullptr},     {"prompt_attn_blk", entry<prompt_attn_blk>(), METH_FASTCALL, nullptr},
    {"fork_blk", entry<fork_blk>(), METH_FASTCALL, nullptr},       {"copy_blk", entry<copy_blk>(), METH_FASTCALL, nullptr},
    {"free_blk", entry<free_blk>(), METH_FASTCALL, nullptr},       {"compact_blk", entry<compact_blk>(), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bind", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__bind()
{
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", MINIKV_BUILT_FOR) < 0) Py_CLEAR(m);
    return m;
}
