// Python calls of the entry points of rotary positions and of the 8-bit paged cache on torch tensors (include/dkv.h): dkv.py's look at
// every tensor and the call itself, without ctypes. What bounds the smallest calls is the host: dkv_rope takes it 3.1 us so (7.2 in
// Python), dkv_rope_append 3.9 (13.2), dkv_quant_attn 5.1 or, with two kernels, 7.2 (13.9, 16.5), most of it the launches; 16
// sequences' next tokens' rows, 4.0 us on the GPU, are written in 4.1 us a call for 13.8.
//
// Each function takes the entry point's address and what dkv.py's function of that name has, makes the call where everything
// is as it should be, and returns its status; else it returns None and calls nothing, and dkv.py names what is wrong (or takes what only
// it knows: addresses, empty buffers). Nothing is kept between calls.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include "dkv.h"

namespace {

using at::ScalarType;

// A call's device, and whether all looks so far found what they should.
struct Look {
    int64_t device;
    bool ok = true;

    const at::Tensor* tensor(PyObject* o)
    {
        if (!THPVariable_Check(o)) return ok = false, nullptr;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.defined() || !t.is_cuda() || t.get_device() != device || t.layout() != at::kStrided) return ok = false, nullptr;
        return &t;
    }
    static bool is(ScalarType x, ScalarType a, ScalarType b) { return x == a || x == b; }
    // A contiguous tensor of n elements of type a or b.
    void* buffer(PyObject* o, int64_t n, ScalarType a, ScalarType b)
    {
        const at::Tensor* t = tensor(o);
        if (!t || !is(t->scalar_type(), a, b) || t->numel() != n || !t->is_contiguous()) return ok = false, nullptr;
        return t->data_ptr();
    }
    int32_t* ints(PyObject* o, int64_t n) { return static_cast<int32_t*>(buffer(o, n, ScalarType::Int, ScalarType::Int)); }
    int32_t* status(PyObject* o) { return o == Py_None ? nullptr : ints(o, 1); }
    // [tokens][heads][128] rows of `type` whose tokens may lie apart; their stride in elements.
    void* rows(PyObject* o, ScalarType type, int64_t tokens, int64_t heads, int64_t* stride)
    {
        const at::Tensor* t = tensor(o);
        if (!t || t->scalar_type() != type || t->dim() != 3 || t->size(0) != tokens || t->size(1) != heads || t->size(2) != 128 ||
            t->stride(2) != 1 || (t->stride(1) != 128 && heads != 1))
            return ok = false, nullptr;
        *stride = tokens > 1 ? t->stride(0) : heads * 128;
        return t->data_ptr();
    }
    // The first of a call's rows: its type and tokens.
    bool first(PyObject* o, ScalarType* type, int64_t* tokens)
    {
        const at::Tensor* t = tensor(o);
        if (!t || !is(t->scalar_type(), ScalarType::BFloat16, ScalarType::Half) || t->dim() != 3 || t->size(0) > INT32_MAX) return ok = false;
        *type = t->scalar_type();
        *tokens = t->size(0);
        return true;
    }
    void* codes(PyObject* o, int64_t rows) { return buffer(o, rows * 128, ScalarType::Byte, ScalarType::Float8_e4m3fn); }
    uint8_t* scales(PyObject* o, int64_t rows) { return static_cast<uint8_t*>(buffer(o, rows, ScalarType::Byte, ScalarType::Float8_e8m0fnu)); }
};

int32_t dtype_of(ScalarType t) { return t == ScalarType::Half ? DKV_FP16 : DKV_BF16; }
template <class F>
F entry(PyObject* o) { return reinterpret_cast<F>(PyLong_AsVoidPtr(o)); }
template <class P>
P* host(PyObject* o) { return o == Py_None ? nullptr : static_cast<P*>(PyLong_AsVoidPtr(o)); }
// A 32-bit number (what does not fit is for dkv.py).
int32_t number(PyObject* o, Look& look)
{
    const long x = PyLong_Check(o) ? PyLong_AsLong(o) : INT64_MAX;
    if (x != (int32_t)x) look.ok = false;
    return (int32_t)x;
}

// `body` without a Python or C++ error to the caller: either is None.
template <class F>
PyObject* quietly(F body)
{
    try {
        const int s = body();
        if (s >= 0 && !PyErr_Occurred()) return PyLong_FromLong(s);
    } catch (...) {
    }
    PyErr_Clear();
    Py_RETURN_NONE;
}

template <class F>
int called(const Look& look, F call)
{
    if (!look.ok || PyErr_Occurred()) return -1;
    int s;
    Py_BEGIN_ALLOW_THREADS s = call();
    Py_END_ALLOW_THREADS return s;
}

// (entry, device, stream, rotary, x, positions, out, status)
PyObject* rope(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    if (n != 8) Py_RETURN_NONE;
    return quietly([&] {
        Look look{PyLong_AsLong(o[1])};
        ScalarType type;
        int64_t tokens, xs, os;
        if (!look.first(o[4], &type, &tokens)) return -1;
        const int64_t heads = THPVariable_Unpack(o[4]).size(1);
        const void* x = look.rows(o[4], type, tokens, heads, &xs);
        const int32_t* positions = look.ints(o[5], tokens);
        void* out = look.rows(o[6], type, tokens, heads, &os);
        int32_t* status = look.status(o[7]);
        const auto f = entry<decltype(&dkv_rope)>(o[0]);
        const auto stream = host<CUstream_st>(o[2]);
        const auto r = host<const dkv_rotary>(o[3]);
        if (heads > INT32_MAX) return -1;
        return called(look, [&] { return (int)f(r, dtype_of(type), (int32_t)tokens, (int32_t)heads, x, xs, positions, out, os, status, stream); });
    });
}

// (entry, device, stream, pages, layer, rotary, q, k_new, v_new, positions, cu_tokens, table, len, Kp, Vp, q_out, Ks, Vs, status)
PyObject* rope_append(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    if (n != 19) Py_RETURN_NONE;
    return quietly([&] {
        Look look{PyLong_AsLong(o[1])};
        const dkv_pages* p = host<const dkv_pages>(o[3]);
        const int32_t layer = number(o[4], look);
        const auto r = host<const dkv_rotary>(o[5]);
        ScalarType type;
        int64_t tokens, qs = 0, os = 0, ks = 0, vs = 0;
        const bool q = o[6] != Py_None, kv = o[7] != Py_None, held = o[16] != Py_None;
        if (q != (o[15] != Py_None) || kv != (o[8] != Py_None) || held != (o[17] != Py_None) || !look.first(o[q ? 6 : 7], &type, &tokens)) return -1;
        const void* qp = q ? look.rows(o[6], type, tokens, p->H, &qs) : nullptr;
        void* qo = q ? look.rows(o[15], type, tokens, p->H, &os) : nullptr;
        const void* kp = kv ? look.rows(o[7], type, tokens, p->H_kv, &ks) : nullptr;
        const void* vp = kv ? look.rows(o[8], type, tokens, p->H_kv, &vs) : nullptr;
        const int64_t slabs = (int64_t)p->L * p->B * p->H_kv, pool = (int64_t)p->num_pages * p->page_rows;
        const int32_t *positions = r ? look.ints(o[9], tokens) : nullptr, *cu = look.ints(o[10], p->B + 1),
                      *table = look.ints(o[11], slabs * p->max_pages), *len = look.ints(o[12], slabs);
        void* Kp = held ? look.codes(o[13], pool) : look.buffer(o[13], pool * 128, type, type);
        void* Vp = held ? look.codes(o[14], pool) : look.buffer(o[14], pool * 128, type, type);
        uint8_t* Ks = held ? look.scales(o[16], pool) : nullptr;
        uint8_t* Vs = held ? look.scales(o[17], pool) : nullptr;
        int32_t* status = look.status(o[18]);
        const auto f = entry<decltype(&dkv_rope_append)>(o[0]);
        const auto stream = host<CUstream_st>(o[2]);
        if (ks != vs) return -1;
        return called(look, [&] {
            return (int)f(p, layer, r, dtype_of(type), (int32_t)tokens, positions, qp, qs, qo, os, kp, vp, ks, cu, table, len, Kp, Vp, Ks, Vs, status,
                          stream);
        });
    });
}

// (entry, device, stream, pages, layer, q, cu_tokens, table, len, Kp, Vp, Ks, Vs, out, workspace, causal, scale, max_tokens, status)
PyObject* quant_attn(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    if (n != 19) Py_RETURN_NONE;
    return quietly([&] {
        Look look{PyLong_AsLong(o[1])};
        const dkv_pages* p = host<const dkv_pages>(o[3]);
        const int32_t layer = number(o[4], look), most = number(o[17], look);
        ScalarType type;
        int64_t tokens, qs = 0;
        if (!look.first(o[5], &type, &tokens)) return -1;
        const void* q = look.rows(o[5], type, tokens, p->H, &qs);
        const int64_t slabs = (int64_t)p->L * p->B * p->H_kv, pool = (int64_t)p->num_pages * p->page_rows;
        const int32_t *cu = look.ints(o[6], p->B + 1), *table = look.ints(o[7], slabs * p->max_pages), *len = look.ints(o[8], slabs);
        const void *Kp = look.codes(o[9], pool), *Vp = look.codes(o[10], pool);
        const uint8_t *Ks = look.scales(o[11], pool), *Vs = look.scales(o[12], pool);
        void* out = look.buffer(o[13], tokens * p->H * 128, type, type);
        const at::Tensor* w = look.tensor(o[14]);
        if (!w || !w->is_contiguous()) return -1;
        void* work = w->data_ptr();
        const int64_t bytes = w->numel() * w->element_size();
        const int causal = PyObject_IsTrue(o[15]);
        const double scale = PyFloat_AsDouble(o[16]);
        int32_t* status = look.status(o[18]);
        const auto f = entry<decltype(&dkv_quant_attn)>(o[0]);
        const auto stream = host<CUstream_st>(o[2]);
        return called(look, [&] {
            return (int)f(p, layer, dtype_of(type), (int32_t)tokens, most, q, qs, cu, table, len, Kp, Vp, Ks, Vs, causal, (float)scale, out, work, bytes,
                          status, stream);
        });
    });
}

// (entry, device, stream, pages, plan, seq, the plan's L, B, H_kv, K, V, T_stride, table, len, Kp, Vp, Ks, Vs, status)
PyObject* quant_compact(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    if (n != 19) Py_RETURN_NONE;
    return quietly([&] {
        Look look{PyLong_AsLong(o[1])};
        const dkv_pages* p = host<const dkv_pages>(o[3]);
        const auto plan = host<const dkv_plan>(o[4]);
        const int32_t L = number(o[6], look), B = number(o[7], look), Hkv = number(o[8], look);
        const at::Tensor *K = look.tensor(o[9]), *V = look.tensor(o[10]);
        if (!K || !V || K->dim() < 2 || !Look::is(K->scalar_type(), ScalarType::BFloat16, ScalarType::Half) || V->scalar_type() != K->scalar_type() ||
            !K->is_contiguous() || !V->is_contiguous())
            return -1;
        const int64_t stride = o[11] == Py_None ? K->size(-2) : number(o[11], look), dense = (int64_t)L * B * Hkv * stride * 128;
        if (stride < 1 || K->numel() < dense || V->numel() < dense) return -1;
        const int64_t slabs = (int64_t)p->L * p->B * p->H_kv, pool = (int64_t)p->num_pages * p->page_rows;
        const int32_t *seq = o[5] == Py_None ? nullptr : look.ints(o[5], B), *table = look.ints(o[12], slabs * p->max_pages),
                      *len = look.ints(o[13], slabs);
        void *Kp = look.codes(o[14], pool), *Vp = look.codes(o[15], pool);
        uint8_t *Ks = look.scales(o[16], pool), *Vs = look.scales(o[17], pool);
        int32_t* status = look.status(o[18]);
        const auto f = entry<decltype(&dkv_quant_compact)>(o[0]);
        const auto stream = host<CUstream_st>(o[2]);
        const ScalarType type = K->scalar_type();
        const void *k = K->data_ptr(), *v = V->data_ptr();
        return called(look, [&] { return (int)f(p, plan, seq, dtype_of(type), k, v, stride, table, len, Kp, Vp, Ks, Vs, status, stream); });
    });
}

PyMethodDef methods[] = {{"rope", (PyCFunction)(void*)rope, METH_FASTCALL, nullptr},
                         {"rope_append", (PyCFunction)(void*)rope_append, METH_FASTCALL, nullptr},
                         {"quant_compact", (PyCFunction)(void*)quant_compact, METH_FASTCALL, nullptr},
                         {"quant_attn", (PyCFunction)(void*)quant_attn, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "dkv_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_dkv_torch() { return PyModule_Create(&module); }
