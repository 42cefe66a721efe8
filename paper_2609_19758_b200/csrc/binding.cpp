// Python binding of the attention operators (fpsk_attention.h): reads the tensors, checks what the library cannot see (shapes, types,
// devices, contiguous channels), fills the structs of the header and calls the library.  In C++ because a small call's time is its
// marshalling: in Python it took 7 of the 10 us that the smallest norm and rotation call needs on the host, here well under one.
// The library's functions come by address, from the build of it that the process has loaded.
#include <Python.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/python_variable.h>

#include "fpsk_attention.h"

#include <stdarg.h>
#include <stdio.h>

namespace {

struct Library {
    decltype(&fpsk_qk_norm_rope) norm_rope;
    decltype(&fpsk_qk_norm_rope_backward) norm_rope_backward;
    decltype(&fpsk_paged_append) append;
    decltype(&fpsk_paged_attention) attention;
} lib;

struct Refused {};                       // a Python error is set
[[noreturn]] void refuse(PyObject *kind, const char *format, ...)
{
    va_list args;
    va_start(args, format);
    PyErr_FormatV(kind, format, args);
    va_end(args);
    throw Refused{};
}

const at::Tensor *tensor(PyObject *o, const char *what)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s: a tensor or None expected", what);
    return &THPVariable_Unpack(o);
}
const at::Tensor &needed(PyObject *o, const char *what)
{
    const at::Tensor *t = tensor(o, what);
    if (!t) refuse(PyExc_TypeError, "%s: a tensor expected", what);
    return *t;
}
int elem(const at::Tensor &t, const char *what)
{
    switch (t.scalar_type()) {
    case at::kHalf: return FPSK_ELEM_FP16;
    case at::kBFloat16: return FPSK_ELEM_BF16;
    case at::kFloat: return FPSK_ELEM_FP32;
    default: refuse(PyExc_TypeError, "%s: float16, bfloat16 or float32 expected", what);
    }
}
int device_of(const at::Tensor &t, const char *what)
{
    if (!t.is_cuda()) refuse(PyExc_ValueError, "%s: a CUDA tensor expected", what);
    return t.get_device();
}
// (tokens, heads, channels) with contiguous channels
void check_heads(const at::Tensor &t, int64_t tokens, int64_t heads, int64_t dim, at::ScalarType type, int device, const char *what)
{
    if (t.dim() != 3 || t.size(0) != tokens || t.size(1) != heads || t.size(2) != dim || t.scalar_type() != type || !t.is_cuda() ||
        t.get_device() != device || (dim > 1 && t.stride(2) != 1))
        refuse(PyExc_ValueError, "%s: expected (%lld, %lld, %lld) %s on cuda:%d with contiguous channels", what, (long long)tokens,
               (long long)heads, (long long)dim, c10::toString(type), device);
}
// what is written must not be expanded
void check_written(const at::Tensor &t, const char *what)
{
    for (int d = 0; d < t.dim(); ++d)
        if (t.size(d) > 1 && t.stride(d) == 0) refuse(PyExc_ValueError, "%s: elements of an output share memory (an expanded dimension)", what);
}
const void *weight(const at::Tensor *w, int64_t dim, int device, const char *what, int32_t &type)
{
    if (!w) return nullptr;
    if (w->dim() != 1 || w->size(0) != dim || !w->is_cuda() || w->get_device() != device || !w->is_contiguous())
        refuse(PyExc_ValueError, "%s: contiguous (%lld,) on cuda:%d expected", what, (long long)dim, device);
    type = elem(*w, what);
    return w->data_ptr();
}
const at::Tensor &index(PyObject *o, int dims, int device, const char *what)
{
    const at::Tensor &t = needed(o, what);
    if (t.dim() != dims || t.scalar_type() != at::kInt || !t.is_cuda() || t.get_device() != device || (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1))
        refuse(PyExc_ValueError, "%s: a %d-dimensional int32 tensor on cuda:%d with a contiguous last dimension expected", what, dims, device);
    return t;
}
fpsk_rotary rotary(PyObject *cos_, PyObject *sin_, PyObject *positions_, bool interleaved, int64_t tokens, int device)
{
    fpsk_rotary r = {};
    const at::Tensor *cos = tensor(cos_, "cos"), *sin = tensor(sin_, "sin");
    if (!cos) return r;
    if (cos->dim() != 2) refuse(PyExc_ValueError, "cos: (positions, rot_dim / 2) expected");
    if (cos->size(1) == 0) return r;
    if (!sin || sin->sizes() != cos->sizes() || cos->scalar_type() != at::kFloat || sin->scalar_type() != at::kFloat || !cos->is_contiguous() ||
        !sin->is_contiguous() || !cos->is_cuda() || !sin->is_cuda() || cos->get_device() != device || sin->get_device() != device)
        refuse(PyExc_ValueError, "cos, sin: contiguous FP32 tables (positions, rot_dim / 2) on cuda:%d expected", device);
    if (positions_ != Py_None) {
        const at::Tensor &p = index(positions_, 1, device, "positions");
        if (p.size(0) != tokens) refuse(PyExc_ValueError, "positions: one per token expected");
        r.positions = static_cast<const int32_t *>(p.data_ptr());
    }
    r.cos = static_cast<const float *>(cos->data_ptr());
    r.sin = static_cast<const float *>(sin->data_ptr());
    r.n_pos = cos->size(0);
    r.rot_dim = (int32_t)(2 * cos->size(1));
    r.interleaved = interleaved;
    return r;
}
int32_t *status_ptr(PyObject *o, int device)
{
    const at::Tensor *t = tensor(o, "status");
    if (!t) return nullptr;
    if (t->scalar_type() != at::kInt || t->numel() < 1 || !t->is_cuda() || t->get_device() != device)
        refuse(PyExc_ValueError, "status: an int32 tensor on cuda:%d expected", device);
    return static_cast<int32_t *>(t->data_ptr());
}
void *stream_ptr(PyObject *o)
{
    void *p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Refused{};
    return p;
}
double number(PyObject *o)
{
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw Refused{};
    return x;
}
bool truth(PyObject *o)
{
    const int x = PyObject_IsTrue(o);
    if (x < 0) throw Refused{};
    return x != 0;
}
// A bound or a window: beyond 32 bits it limits as little (or is refused as much) as the widest that they hold.
int32_t clamped(PyObject *o)
{
    int beyond = 0;
    const long long x = PyLong_AsLongLongAndOverflow(o, &beyond);
    if (x == -1 && !beyond && PyErr_Occurred()) throw Refused{};
    if (beyond) return beyond > 0 ? INT32_MAX : INT32_MIN;
    return x > INT32_MAX ? INT32_MAX : x < INT32_MIN ? INT32_MIN : (int32_t)x;
}

// One kind of heads and where they go; with no `out`, only what is read.
fpsk_heads heads(const at::Tensor *x, const at::Tensor *out, const at::Tensor *w, const at::Tensor &like, at::ScalarType out_type, int device,
                 const char *what, bool has_out)
{
    fpsk_heads h = {};
    if (!x) return h;
    if (x->dim() != 3) refuse(PyExc_ValueError, "%s: (tokens, heads, channels) expected", what);
    check_heads(*x, like.size(0), x->size(1), like.size(2), like.scalar_type(), device, what);
    h.in = x->data_ptr();
    h.in_token_stride = x->stride(0);
    h.in_head_stride = x->stride(1);
    h.n_heads = (int32_t)x->size(1);
    if (has_out) {
        if (!out) refuse(PyExc_ValueError, "%s_out is missing", what);
        check_heads(*out, x->size(0), x->size(1), x->size(2), out_type, device, what);
        check_written(*out, what);
        h.out = out->data_ptr();
        h.out_token_stride = out->stride(0);
        h.out_head_stride = out->stride(1);
    }
    h.weight = weight(w, like.size(2), device, what, h.weight_type);
    return h;
}
fpsk_heads_grad heads_grad(const at::Tensor *x, PyObject *dy_, PyObject *dx_, const at::Tensor *w, PyObject *dw_, const at::Tensor &like,
                           at::ScalarType grad_type, int device, const char *what)
{
    fpsk_heads_grad h = {};
    if (!x) return h;
    if (x->dim() != 3) refuse(PyExc_ValueError, "%s: (tokens, heads, channels) expected", what);
    const int64_t n = like.size(0), dim = like.size(2);
    const at::Tensor &dy = needed(dy_, "the gradient of the output"), &dx = needed(dx_, "the gradient of the input");
    check_heads(*x, n, x->size(1), dim, like.scalar_type(), device, what);
    check_heads(dy, n, x->size(1), dim, grad_type, device, what);
    check_heads(dx, n, x->size(1), dim, grad_type, device, what);
    check_written(dx, what);
    h.in = x->data_ptr(); h.dout = dy.data_ptr(); h.din = dx.data_ptr();
    h.in_token_stride = x->stride(0); h.in_head_stride = x->stride(1);
    h.dout_token_stride = dy.stride(0); h.dout_head_stride = dy.stride(1);
    h.din_token_stride = dx.stride(0); h.din_head_stride = dx.stride(1);
    h.n_heads = (int32_t)x->size(1);
    h.weight = weight(w, dim, device, what, h.weight_type);
    if (w) {
        const at::Tensor &dw = needed(dw_, "the gradient of the weight");
        if (dw.dim() != 1 || dw.size(0) != dim || dw.scalar_type() != at::kFloat || !dw.is_contiguous() || !dw.is_cuda() || dw.get_device() != device)
            refuse(PyExc_ValueError, "d%s_weight: contiguous FP32 (%lld,) on cuda:%d expected", what, (long long)dim, device);
        h.dweight = static_cast<float *>(dw.data_ptr());
    }
    return h;
}
struct Cache {
    fpsk_paged_cache c;
    int device;
    at::ScalarType type;
};
Cache cache_of(PyObject *k_, PyObject *v_)
{
    const at::Tensor &k = needed(k_, "k"), &v = needed(v_, "v");
    if (k.dim() != 4 || v.dim() != 4 || k.sizes() != v.sizes() || k.scalar_type() != v.scalar_type() || !k.is_cuda() || !v.is_cuda() ||
        k.get_device() != v.get_device())
        refuse(PyExc_ValueError, "a cache: two alike CUDA tensors (pages, page size, heads, channels) expected");
    if (k.scalar_type() != at::kHalf && k.scalar_type() != at::kBFloat16) refuse(PyExc_ValueError, "a cache is float16 or bfloat16");
    if (k.size(3) > 1 && (k.stride(3) != 1 || v.stride(3) != 1)) refuse(PyExc_ValueError, "a cache's channels must be contiguous");
    Cache x;
    x.device = k.get_device();
    x.type = k.scalar_type();
    x.c = {k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2), v.stride(0), v.stride(1), v.stride(2), k.size(0),
           (int32_t)k.size(1), (int32_t)k.size(2), (int32_t)k.size(3), elem(k, "a cache")};
    return x;
}
fpsk_paged_batch batch(PyObject *cu_, PyObject *kv_, PyObject *table_, int64_t tokens, int device)
{
    const at::Tensor &cu = index(cu_, 1, device, "cu_q"), &kv = index(kv_, 1, device, "kv_len"), &table = index(table_, 2, device, "block_table");
    const int64_t n = kv.size(0);
    if (cu.size(0) != n + 1 || table.size(0) != n) refuse(PyExc_ValueError, "cu_q: (sequences + 1,), block_table: (sequences, pages) expected");
    fpsk_paged_batch b = {};
    b.cu_q = static_cast<const int32_t *>(cu.data_ptr());
    b.kv_len = static_cast<const int32_t *>(kv.data_ptr());
    b.block_table = static_cast<const int32_t *>(table.data_ptr());
    b.table_stride = n > 1 ? table.stride(0) : table.size(1);
    b.n_tokens = tokens;
    b.n_seqs = (int32_t)n;
    b.max_pages = (int32_t)table.size(1);
    return b;
}

// The library launches on the current device and sizes its grids by it: that is the tensors' for the time of a call.
struct OnDevice {
    c10::DeviceGuard guard;
    explicit OnDevice(int device) : guard(c10::Device(c10::kCUDA, (c10::DeviceIndex)device)) {}
};

template <typename F> PyObject *call(Py_ssize_t given, Py_ssize_t wanted, F f)
{
    if (given != wanted) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", wanted, given);
        return nullptr;
    }
    try {
        return PyLong_FromLong((long)f());
    } catch (const Refused &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

PyObject *py_bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return call(n, 4, [&] {
        lib.norm_rope = reinterpret_cast<decltype(lib.norm_rope)>(PyLong_AsVoidPtr(a[0]));
        lib.norm_rope_backward = reinterpret_cast<decltype(lib.norm_rope_backward)>(PyLong_AsVoidPtr(a[1]));
        lib.append = reinterpret_cast<decltype(lib.append)>(PyLong_AsVoidPtr(a[2]));
        lib.attention = reinterpret_cast<decltype(lib.attention)>(PyLong_AsVoidPtr(a[3]));
        return 0;
    });
}
// which device a call's stream is asked for
PyObject *py_device(PyObject *, PyObject *o)
{
    return call(1, 1, [&] { return device_of(needed(o, "the first argument"), "the first argument"); });
}

// q, k, cos, sin, positions, q_out, k_out, q_weight, k_weight, eps, interleaved, status, stream
PyObject *py_norm_rope(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return call(n, 13, [&] {
        const at::Tensor *q = tensor(a[0], "q"), *k = tensor(a[1], "k"), *qo = tensor(a[5], "q_out"), *ko = tensor(a[6], "k_out");
        if (!q && !k) refuse(PyExc_ValueError, "q or k expected");
        const at::Tensor &like = q ? *q : *k;
        const at::Tensor *out = q ? qo : ko;
        if (!out) refuse(PyExc_ValueError, "the output is missing");
        if (like.dim() != 3) refuse(PyExc_ValueError, "(tokens, heads, channels) expected");
        const int device = device_of(like, "q, k"), in_type = elem(like, "q, k"), out_type = elem(*out, "the output");
        const fpsk_heads hq = heads(q, qo, tensor(a[7], "q_weight"), like, out->scalar_type(), device, "q", true);
        const fpsk_heads hk = heads(k, ko, tensor(a[8], "k_weight"), like, out->scalar_type(), device, "k", true);
        const fpsk_rotary r = rotary(a[2], a[3], a[4], truth(a[10]), like.size(0), device);
        const OnDevice on(device);
        return lib.norm_rope(&hq, &hk, like.size(0), (int32_t)like.size(2), (fpsk_elem)in_type, (fpsk_elem)out_type, &r,
                             (float)number(a[9]), status_ptr(a[11], device), stream_ptr(a[12]));
    });
}
// q, k, dq_out, dk_out, cos, sin, positions, dq, dk, dq_weight, dk_weight, ws, q_weight, k_weight, eps, interleaved, status, stream
PyObject *py_norm_rope_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return call(n, 18, [&] {
        const at::Tensor *q = tensor(a[0], "q"), *k = tensor(a[1], "k");
        if (!q && !k) refuse(PyExc_ValueError, "q or k expected");
        const at::Tensor &like = q ? *q : *k, &g = needed(q ? a[2] : a[3], "the gradient of the output"), &ws = needed(a[11], "ws");
        if (like.dim() != 3) refuse(PyExc_ValueError, "(tokens, heads, channels) expected");
        const int device = device_of(like, "q, k"), in_type = elem(like, "q, k"), grad_type = elem(g, "the gradient of the output");
        if (!ws.is_cuda() || ws.get_device() != device || !ws.is_contiguous()) refuse(PyExc_ValueError, "ws: on cuda:%d expected", device);
        const fpsk_heads_grad hq = heads_grad(q, a[2], a[7], tensor(a[12], "q_weight"), a[9], like, g.scalar_type(), device, "q");
        const fpsk_heads_grad hk = heads_grad(k, a[3], a[8], tensor(a[13], "k_weight"), a[10], like, g.scalar_type(), device, "k");
        const fpsk_rotary r = rotary(a[4], a[5], a[6], truth(a[15]), like.size(0), device);
        const OnDevice on(device);
        return lib.norm_rope_backward(&hq, &hk, like.size(0), (int32_t)like.size(2), (fpsk_elem)in_type, (fpsk_elem)grad_type, &r,
                                      (float)number(a[14]), ws.data_ptr(), (size_t)ws.nbytes(), status_ptr(a[16], device), stream_ptr(a[17]));
    });
}
PyObject *py_check_cache(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return call(n, 2, [&] { return cache_of(a[0], a[1]).device; });
}
// cache k, cache v, k, v, cu_q, kv_len, block_table, cos, sin, k_weight, q, q_out, q_weight, positions, eps, interleaved, status, stream
PyObject *py_append(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return call(n, 18, [&] {
        const Cache c = cache_of(a[0], a[1]);
        const at::Tensor &k = needed(a[2], "k"), &v = needed(a[3], "v");
        const at::Tensor *q = tensor(a[10], "q");
        if (k.dim() != 3 || k.size(1) != c.c.n_heads || k.size(2) != c.c.head_dim || v.sizes() != k.sizes())
            refuse(PyExc_ValueError, "k, v: (tokens, %d, %d) expected", c.c.n_heads, c.c.head_dim);
        const int in_type = elem(k, "k");
        const fpsk_heads hk = heads(&k, nullptr, tensor(a[9], "k_weight"), k, c.type, c.device, "k", false);
        const fpsk_heads hv = heads(&v, nullptr, nullptr, k, c.type, c.device, "v", false);
        const fpsk_heads hq = heads(q, tensor(a[11], "q_out"), tensor(a[12], "q_weight"), k, c.type, c.device, "q", true);
        const fpsk_rotary r = rotary(a[7], a[8], a[13], truth(a[15]), k.size(0), c.device);
        const fpsk_paged_batch b = batch(a[4], a[5], a[6], k.size(0), c.device);
        const OnDevice on(c.device);
        return lib.append(&c.c, &b, &hk, &hv, &hq, (fpsk_elem)in_type, &r, (float)number(a[14]), status_ptr(a[16], c.device),
                          stream_ptr(a[17]));
    });
}
// cache k, cache v, q, out, cu_q, kv_len, block_table, ws, max_q_len, max_kv_len, scale, causal, window, lse, status, stream
PyObject *py_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return call(n, 16, [&] {
        const Cache c = cache_of(a[0], a[1]);
        const at::Tensor &q = needed(a[2], "q"), &out = needed(a[3], "out"), &ws = needed(a[7], "ws");
        const at::Tensor *lse = tensor(a[13], "lse");
        if (q.dim() != 3) refuse(PyExc_ValueError, "q: (tokens, heads, channels) expected");
        check_heads(q, q.size(0), q.size(1), c.c.head_dim, c.type, c.device, "q");
        check_heads(out, q.size(0), q.size(1), c.c.head_dim, c.type, c.device, "out");
        check_written(out, "out");
        if (!ws.is_cuda() || ws.get_device() != c.device || !ws.is_contiguous()) refuse(PyExc_ValueError, "ws: on cuda:%d expected", c.device);
        fpsk_attention t = {};
        if (lse) {
            if (lse->dim() != 2 || lse->size(0) != q.size(0) || lse->size(1) != q.size(1) || lse->scalar_type() != at::kFloat || !lse->is_contiguous() ||
                !lse->is_cuda() || lse->get_device() != c.device)
                refuse(PyExc_ValueError, "lse: contiguous FP32 (%lld, %lld) on cuda:%d expected", (long long)q.size(0), (long long)q.size(1), c.device);
            t.lse = static_cast<float *>(lse->data_ptr());
        }
        t.q = q.data_ptr(); t.out = out.data_ptr();
        t.q_token_stride = q.stride(0); t.q_head_stride = q.stride(1);
        t.out_token_stride = out.stride(0); t.out_head_stride = out.stride(1);
        t.n_heads = (int32_t)q.size(1);
        t.causal = truth(a[11]);
        t.window = clamped(a[12]);
        t.max_q_len = clamped(a[8]);
        t.max_kv_len = clamped(a[9]);
        if (a[10] != Py_None) {
            const double scale = number(a[10]);
            if (!(scale > 0) || scale > 3.4e38) refuse(PyExc_ValueError, "scale must be positive and finite");
            t.scale = (float)scale;
        }
        const fpsk_paged_batch b = batch(a[4], a[5], a[6], q.size(0), c.device);
        const OnDevice on(c.device);
        return lib.attention(&c.c, &b, &t, ws.data_ptr(), (size_t)ws.nbytes(), status_ptr(a[14], c.device), stream_ptr(a[15]));
    });
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(py_bind), METH_FASTCALL, nullptr},
    {"device", py_device, METH_O, nullptr},
    {"qk_norm_rope", reinterpret_cast<PyCFunction>(py_norm_rope), METH_FASTCALL, nullptr},
    {"qk_norm_rope_backward", reinterpret_cast<PyCFunction>(py_norm_rope_backward), METH_FASTCALL, nullptr},
    {"check_cache", reinterpret_cast<PyCFunction>(py_check_cache), METH_FASTCALL, nullptr},
    {"paged_append", reinterpret_cast<PyCFunction>(py_append), METH_FASTCALL, nullptr},
    {"paged_attention", reinterpret_cast<PyCFunction>(py_attention), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// (kept in the file: by it a binding made against another torch is told)
PyMODINIT_FUNC PyInit__binding()
{
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "made_for", FPSK_BINDING_MARK) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
