// Python extension module `_call`: the device calls of binding.py without ctypes.  A short call is
// bound by its host time: one image's softmax is a kernel of 2.3 us (in a graph) and cost 5.1 us per call
// through ctypes, 3.7 here; its GELU 4.6 and 3.2.  The launch itself is 2.5 to 3 of those.  So the ordinary
// case is checked and converted here.
//
// Every function takes the arguments of its namesake in binding.py and returns the library's return
// code, or None if any of them is not what this path takes (another type, too few elements, an
// integer that does not fit): nothing has been called then, and the caller goes the long way, which
// raises what it always raised.  It calls the library through the addresses it was given.
#include <Python.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <vector>

#include "../../include/iptq.h"

namespace {

// bound by bind(): entry points of the loaded library and the parameter classes of binding.py
struct Bound {
    decltype(&iptq_requant) requant;
    decltype(&iptq_softmax_i32) softmax_i32;
    decltype(&iptq_softmax_i32_windowed) windowed;
    decltype(&iptq_softmax_i32_windowed_bits) windowed_bits;
    decltype(&iptq_gelu_i8) gelu_i8;
    decltype(&iptq_gelu_i32) gelu_i32;
    decltype(&iptq_softmax_i32_layers) softmax_layers;
    decltype(&iptq_gelu_i8_layers) gelu_layers;
    PyTypeObject *softmax_params, *gelu_params, *dyadic;
} g = {};

// A contiguous tensor of that type on the GPU, of class torch.Tensor itself: its address.
bool tensor(PyObject *o, at::ScalarType type, int64_t least, void **p)
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous() || t.numel() < least) return false;
    *p = t.data_ptr();
    return true;
}

bool integer(PyObject *o, int64_t *v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}
bool integer(PyObject *o, int32_t *v)
{
    int64_t w = 0;
    if (!integer(o, &w) || w < INT32_MIN || w > INT32_MAX) return false;
    *v = (int32_t)w;
    return true;
}

// rows x cols, or -1 where that is no element count (left to the long way)
int64_t elements(int64_t rows, int64_t cols)
{
    int64_t n = 0;
    return rows < 0 || cols < 0 || __builtin_mul_overflow(rows, cols, &n) ? -1 : n;
}

// A copy of a parameter structure of exactly that class.
template <typename T>
bool structure(PyObject *o, PyTypeObject *type, T *out)
{
    if (Py_TYPE(o) != type) return false;
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        return false;
    }
    const bool ok = view.len == (Py_ssize_t)sizeof(T);
    if (ok) memcpy(out, view.buf, sizeof(T));
    PyBuffer_Release(&view);
    return ok;
}
template <typename T>
bool structures(PyObject *o, PyTypeObject *type, int32_t n, std::vector<T> *out)
{
    if (!(PyList_CheckExact(o) || PyTuple_CheckExact(o)) || n < 1 || PySequence_Fast_GET_SIZE(o) != n) return false;
    out->resize(n);
    for (int32_t i = 0; i < n; ++i)
        if (!structure(PySequence_Fast_GET_ITEM(o, i), type, &(*out)[i])) return false;
    return true;
}

// Runs the call on torch's current stream without the interpreter's lock, as ctypes does.
template <typename F>
PyObject *enqueue(F call)
{
    void *const stream = c10::hip::getCurrentHIPStream().stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call(stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// Anything torch throws (a tensor without storage, say) is left to the long way.
template <PyObject *(*F)(PyObject *const *, Py_ssize_t)>
PyObject *guarded(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    try {
        PyObject *r = F(a, n);
        if (r != nullptr) return r;
    } catch (...) {
    }
    PyErr_Clear();
    Py_RETURN_NONE;
}

at::ScalarType byte_type(int is_signed) { return is_signed ? at::kChar : at::kByte; }

PyObject *requant(PyObject *const *a, Py_ssize_t n_args)
{
    void *in, *out;
    int64_t n;
    int32_t is_signed;
    iptq_dyadic_t p;
    if (n_args != 5 || g.requant == nullptr || !integer(a[2], &n) || n < 0 || !integer(a[3], &is_signed) ||
        !tensor(a[0], at::kInt, n, &in) || !tensor(a[1], byte_type(is_signed), n, &out) || !structure(a[4], g.dyadic, &p))
        return nullptr;
    return enqueue([&](void *s) { return g.requant((const int32_t *)in, out, n, is_signed, &p, s); });
}

// scores, bias, period, then `skip` arguments of the mask, out, rows, cols, params
struct SoftmaxArguments {
    void *scores, *bias, *out;
    int64_t period, rows;
    int32_t cols;
    iptq_softmax_params_t p;
    bool take(PyObject *const *a, int skip)
    {
        PyObject *const *b = a + 3 + skip;
        bias = nullptr;
        if (!integer(b[1], &rows) || !integer(b[2], &cols) || !integer(a[2], &period) ||
            !structure(b[3], g.softmax_params, &p))
            return false;
        const int64_t n = elements(rows, cols);
        if (n < 0 || !tensor(a[0], at::kInt, n, &scores) || !tensor(b[0], byte_type(p.out_is_signed), n, &out)) return false;
        if (a[1] == Py_None) return true;
        const int64_t table = elements(period, cols);
        return table >= 0 && tensor(a[1], at::kInt, table, &bias);
    }
};

PyObject *softmax_i32(PyObject *const *a, Py_ssize_t n_args)
{
    SoftmaxArguments s;
    if (n_args != 7 || g.softmax_i32 == nullptr || !s.take(a, 0)) return nullptr;
    return enqueue([&](void *st) {
        return g.softmax_i32((const int32_t *)s.scores, (const int32_t *)s.bias, s.period, s.out, s.rows, s.cols, &s.p, st);
    });
}

template <bool BITS>
PyObject *windowed(PyObject *const *a, Py_ssize_t n_args)
{
    SoftmaxArguments s;
    int32_t windows, heads;
    void *mask = nullptr;
    if (n_args != 10 || g.windowed == nullptr || !integer(a[4], &windows) || !integer(a[5], &heads) || !s.take(a, 3)) return nullptr;
    if (a[3] != Py_None) {
        const int64_t queries = elements(windows, s.cols);
        const int64_t n = queries < 0 ? -1 : elements(queries, BITS ? ((int64_t)s.cols + 63) / 64 : s.cols);
        if (n < 0 || !tensor(a[3], BITS ? at::kLong : at::kInt, n, &mask)) return nullptr;
    }
    return enqueue([&](void *st) {
        if (BITS)
            return g.windowed_bits((const int32_t *)s.scores, (const int32_t *)s.bias, s.period, (const uint64_t *)mask, windows,
                                   heads, s.out, s.rows, s.cols, &s.p, st);
        return g.windowed((const int32_t *)s.scores, (const int32_t *)s.bias, s.period, (const int32_t *)mask, windows, heads,
                          s.out, s.rows, s.cols, &s.p, st);
    });
}

template <bool FROM_I8>
PyObject *gelu(PyObject *const *a, Py_ssize_t n_args)
{
    void *in, *out;
    int64_t n;
    iptq_gelu_params_t p;
    if (n_args != 4 || g.gelu_i8 == nullptr || !integer(a[2], &n) || n < 0 || !tensor(a[0], FROM_I8 ? at::kChar : at::kInt, n, &in) ||
        !tensor(a[1], at::kChar, n, &out) || !structure(a[3], g.gelu_params, &p))
        return nullptr;
    return enqueue([&](void *s) {
        return FROM_I8 ? g.gelu_i8((const int8_t *)in, (int8_t *)out, n, &p, s)
                       : g.gelu_i32((const int32_t *)in, (int8_t *)out, n, &p, s);
    });
}

// (n - 1) stride + size, or -1
int64_t extent(int32_t n, int64_t stride, int64_t size)
{
    int64_t e = 0;
    return stride < 0 || size < 0 || __builtin_mul_overflow((int64_t)(n - 1), stride, &e) || __builtin_add_overflow(e, size, &e) ? -1 : e;
}

PyObject *softmax_layers(PyObject *const *a, Py_ssize_t n_args)
{
    void *in, *out;
    int64_t in_stride, out_stride, rows;
    int32_t cols, n;
    std::vector<iptq_softmax_params_t> p;
    if (n_args != 8 || g.softmax_layers == nullptr || !integer(a[1], &in_stride) || !integer(a[3], &out_stride) ||
        !integer(a[4], &rows) || !integer(a[5], &cols) || !integer(a[6], &n) || !structures(a[7], g.softmax_params, n, &p))
        return nullptr;
    const int64_t size = elements(rows, cols);
    const int64_t read = extent(n, in_stride, size), written = extent(n, out_stride, size);
    if (size < 0 || read < 0 || written < 0 || !tensor(a[0], at::kInt, read, &in) ||
        !tensor(a[2], byte_type(p[0].out_is_signed), written, &out))
        return nullptr;
    return enqueue([&](void *s) {
        return g.softmax_layers((const int32_t *)in, in_stride, out, out_stride, rows, cols, n, p.data(), s);
    });
}

PyObject *gelu_layers(PyObject *const *a, Py_ssize_t n_args)
{
    void *in, *out;
    int64_t in_stride, out_stride, size;
    int32_t n;
    std::vector<iptq_gelu_params_t> p;
    if (n_args != 7 || g.gelu_layers == nullptr || !integer(a[1], &in_stride) || !integer(a[3], &out_stride) ||
        !integer(a[4], &size) || !integer(a[5], &n) || !structures(a[6], g.gelu_params, n, &p))
        return nullptr;
    const int64_t read = extent(n, in_stride, size), written = extent(n, out_stride, size);
    if (read < 0 || written < 0 || !tensor(a[0], at::kChar, read, &in) || !tensor(a[2], at::kChar, written, &out)) return nullptr;
    return enqueue([&](void *s) { return g.gelu_layers((const int8_t *)in, in_stride, (int8_t *)out, out_stride, size, n, p.data(), s); });
}

// bind(addresses of the eight entry points in the order of Bound, SoftmaxParams, GeluParams, Dyadic)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    if (n_args != 11) {
        PyErr_SetString(PyExc_TypeError, "bind takes eight addresses and three classes");
        return nullptr;
    }
    void *at[8];
    for (int i = 0; i < 8; ++i) {
        at[i] = PyLong_AsVoidPtr(a[i]);
        if (at[i] == nullptr) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: an entry point is missing");
            return nullptr;
        }
    }
    for (int i = 8; i < 11; ++i)
        if (!PyType_Check(a[i])) {
            PyErr_SetString(PyExc_TypeError, "bind takes eight addresses and three classes");
            return nullptr;
        }
    g.requant = reinterpret_cast<decltype(g.requant)>(at[0]);
    g.softmax_i32 = reinterpret_cast<decltype(g.softmax_i32)>(at[1]);
    g.windowed = reinterpret_cast<decltype(g.windowed)>(at[2]);
    g.windowed_bits = reinterpret_cast<decltype(g.windowed_bits)>(at[3]);
    g.gelu_i8 = reinterpret_cast<decltype(g.gelu_i8)>(at[4]);
    g.gelu_i32 = reinterpret_cast<decltype(g.gelu_i32)>(at[5]);
    g.softmax_layers = reinterpret_cast<decltype(g.softmax_layers)>(at[6]);
    g.gelu_layers = reinterpret_cast<decltype(g.gelu_layers)>(at[7]);
    PyTypeObject **types[3] = {&g.softmax_params, &g.gelu_params, &g.dyadic};
    for (int i = 0; i < 3; ++i) {
        Py_INCREF(a[8 + i]);                          // kept for the life of the process, as the module is
        *types[i] = reinterpret_cast<PyTypeObject *>(a[8 + i]);
    }
    Py_RETURN_NONE;
}

// ---- the block operators (block.py): bound apart, by bind_block()
struct BoundBlock {
    decltype(&iptq_attention_i8) attention_i8;
    decltype(&iptq_cache_store_i4) cache_store_i4;
    decltype(&iptq_attention_cache_i4) attention_cache_i4;
    decltype(&iptq_rmsnorm_i32) rmsnorm_i32;
    decltype(&iptq_requant_rows) requant_rows;
    PyTypeObject *attention_params, *rmsnorm_params, *cache, *dyadic;
} gb = {};

// As tensor(), and on the current device; None: no pointer.
bool local_tensor(PyObject *o, at::ScalarType type, int64_t least, void **p)
{
    return tensor(o, type, least, p) && THPVariable_Unpack(o).get_device() == c10::hip::current_device();
}
bool optional_tensor(PyObject *o, at::ScalarType type, int64_t least, void **p)
{
    *p = nullptr;
    return o == Py_None || local_tensor(o, type, least, p);
}

// An int8 tensor [tokens, heads, head dimension] whose heads lie side by side in a token.
struct Rows {
    void *p;
    int64_t tokens, heads, dim, stride;
    bool take(PyObject *o)
    {
        if (!THPVariable_CheckExact(o)) return false;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.scalar_type() != at::kChar || t.dim() != 3 || t.get_device() != c10::hip::current_device()) return false;
        tokens = t.size(0); heads = t.size(1); dim = t.size(2);
        if (tokens < 1 || heads < 1 || dim < 2 || heads > 65536 || dim > 65536) return false;
        stride = tokens > 1 ? t.stride(0) : heads * dim;
        if (t.stride(2) != 1 || (heads > 1 && t.stride(1) != dim) || stride < heads * dim) return false;
        p = t.data_ptr();
        return true;
    }
};

PyObject *attention_i8(PyObject *const *a, Py_ssize_t n_args)
{
    Rows q, k, v, o;
    void *qo, *ko;
    int32_t n, max_q;
    iptq_attention_params_t p;
    if (n_args != 9 || gb.attention_i8 == nullptr || !integer(a[5], &n) || n < 0 || !integer(a[6], &max_q) || !q.take(a[0]) || !k.take(a[1]) ||
        !v.take(a[2]) || !o.take(a[7]) || !structure(a[8], gb.attention_params, &p) ||
        !optional_tensor(a[3], at::kInt, (int64_t)n + 1, &qo) || !optional_tensor(a[4], at::kInt, (int64_t)n + 1, &ko))
        return nullptr;
    if (k.tokens != v.tokens || k.heads != v.heads || q.dim != k.dim || q.dim != v.dim || q.tokens != o.tokens || q.heads != o.heads || q.dim != o.dim)
        return nullptr;
    return enqueue([&](void *s) {
        return gb.attention_i8((const int8_t *)q.p, q.stride, (const int8_t *)k.p, k.stride, (const int8_t *)v.p, v.stride, (const int32_t *)qo,
                               (const int32_t *)ko, n, max_q, q.tokens, k.tokens, (int32_t)q.heads, (int32_t)k.heads, (int32_t)q.dim,
                               (int8_t *)o.p, o.stride, &p, s);
    });
}

PyObject *cache_store_i4(PyObject *const *a, Py_ssize_t n_args)
{
    Rows k, v;
    void *slots;
    int64_t n;
    iptq_cache_i4_t c;
    if (n_args != 5 || gb.cache_store_i4 == nullptr || !structure(a[0], gb.cache, &c) || !k.take(a[1]) || !v.take(a[2]) || !integer(a[4], &n) ||
        n < 0 || !local_tensor(a[3], at::kInt, n, &slots))
        return nullptr;
    if (k.tokens < n || v.tokens < n || k.heads != c.kv_heads || v.heads != c.kv_heads || k.dim != c.head_dim || v.dim != c.head_dim) return nullptr;
    return enqueue([&](void *s) {
        return gb.cache_store_i4(&c, (const int8_t *)k.p, k.stride, (const int8_t *)v.p, v.stride, (const int32_t *)slots, n, s);
    });
}

PyObject *attention_cache_i4(PyObject *const *a, Py_ssize_t n_args)
{
    Rows q, o;
    void *pages, *lengths, *work = nullptr;
    int32_t n, t;
    iptq_cache_i4_t c;
    iptq_attention_params_t p;
    if (n_args != 9 || gb.attention_cache_i4 == nullptr || !q.take(a[0]) || !structure(a[1], gb.cache, &c) || !integer(a[4], &n) || n < 0 ||
        !integer(a[5], &t) || t < 0 || !o.take(a[6]) || !structure(a[8], gb.attention_params, &p) || !local_tensor(a[2], at::kInt, 0, &pages) ||
        !local_tensor(a[3], at::kInt, n, &lengths) || !optional_tensor(a[7], at::kByte, 0, &work))
        return nullptr;
    const at::Tensor &table = THPVariable_Unpack(a[2]);
    if (table.dim() != 2 || table.size(0) < n || table.size(1) > INT32_MAX || q.tokens != o.tokens || q.heads != o.heads || q.dim != o.dim ||
        q.dim != c.head_dim || q.tokens < (int64_t)n * t)
        return nullptr;
    const int32_t max_pages = (int32_t)table.size(1);
    const int64_t size = work ? THPVariable_Unpack(a[7]).numel() : 0;
    return enqueue([&](void *s) {
        return gb.attention_cache_i4((const int8_t *)q.p, q.stride, &c, (const int32_t *)pages, max_pages, (const int32_t *)lengths, n, t, (int32_t)q.heads,
                                     (int8_t *)o.p, o.stride, work, size, &p, s);
    });
}

PyObject *rmsnorm_i32(PyObject *const *a, Py_ssize_t n_args)
{
    void *x, *residual, *gain, *stream, *out, *scales;
    int64_t rows;
    int32_t cols;
    iptq_rmsnorm_params_t p;
    if (n_args != 9 || gb.rmsnorm_i32 == nullptr || !integer(a[6], &rows) || !integer(a[7], &cols) || !structure(a[8], gb.rmsnorm_params, &p)) return nullptr;
    const int64_t n = elements(rows, cols);
    if (n < 0 || !optional_tensor(a[0], at::kInt, n, &x) || !optional_tensor(a[1], at::kInt, n, &residual) || !local_tensor(a[2], at::kShort, cols, &gain) ||
        !optional_tensor(a[3], at::kInt, n, &stream) || !local_tensor(a[4], at::kChar, n, &out) || !optional_tensor(a[5], at::kInt, rows, &scales))
        return nullptr;
    return enqueue([&](void *s) {
        return gb.rmsnorm_i32((const int32_t *)x, (const int32_t *)residual, (const int16_t *)gain, (int32_t *)stream, (int8_t *)out, (int32_t *)scales, rows,
                              cols, &p, s);
    });
}

PyObject *requant_rows(PyObject *const *a, Py_ssize_t n_args)
{
    void *in, *scales, *out;
    int64_t rows;
    int32_t cols, shift, is_signed;
    iptq_dyadic_t p;
    if (n_args != 8 || gb.requant_rows == nullptr || !integer(a[3], &rows) || !integer(a[4], &cols) || !integer(a[5], &shift) || !integer(a[6], &is_signed) ||
        !structure(a[7], gb.dyadic, &p))
        return nullptr;
    const int64_t n = elements(rows, cols);
    if (n < 0 || !local_tensor(a[0], at::kInt, n, &in) || !local_tensor(a[1], at::kInt, rows, &scales) || !local_tensor(a[2], byte_type(is_signed), n, &out)) return nullptr;
    return enqueue([&](void *s) { return gb.requant_rows((const int32_t *)in, (const int32_t *)scales, shift, out, rows, cols, is_signed, &p, s); });
}

// bind_block(addresses of the five entry points in the order of BoundBlock, AttentionParams, RmsnormParams, CacheI4, Dyadic)
PyObject *bind_block(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    void *at[5];
    bool right = n_args == 9;
    for (int i = 0; right && i < 5; ++i) right = (at[i] = PyLong_AsVoidPtr(a[i])) != nullptr;
    for (int i = 5; right && i < 9; ++i) right = PyType_Check(a[i]);
    if (!right) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "bind_block takes five addresses and four classes");
        return nullptr;
    }
    gb.attention_i8 = reinterpret_cast<decltype(gb.attention_i8)>(at[0]);
    gb.cache_store_i4 = reinterpret_cast<decltype(gb.cache_store_i4)>(at[1]);
    gb.attention_cache_i4 = reinterpret_cast<decltype(gb.attention_cache_i4)>(at[2]);
    gb.rmsnorm_i32 = reinterpret_cast<decltype(gb.rmsnorm_i32)>(at[3]);
    gb.requant_rows = reinterpret_cast<decltype(gb.requant_rows)>(at[4]);
    PyTypeObject **types[4] = {&gb.attention_params, &gb.rmsnorm_params, &gb.cache, &gb.dyadic};
    for (int i = 0; i < 4; ++i) {
        Py_INCREF(a[5 + i]);                          // kept for the life of the process, as the module is
        *types[i] = reinterpret_cast<PyTypeObject *>(a[5 + i]);
    }
    Py_RETURN_NONE;
}

#define IPTQ_METHOD(NAME, FN) {NAME, (PyCFunction)(void (*)(void))(FN), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    IPTQ_METHOD("bind", bind),
    IPTQ_METHOD("requant", guarded<requant>),
    IPTQ_METHOD("softmax_i32", guarded<softmax_i32>),
    IPTQ_METHOD("softmax_i32_windowed", guarded<windowed<false>>),
    IPTQ_METHOD("softmax_i32_windowed_bits", guarded<windowed<true>>),
    IPTQ_METHOD("gelu_i8", guarded<gelu<true>>),
    IPTQ_METHOD("gelu_i32", guarded<gelu<false>>),
    IPTQ_METHOD("softmax_i32_layers", guarded<softmax_layers>),
    IPTQ_METHOD("gelu_i8_layers", guarded<gelu_layers>),
    IPTQ_METHOD("bind_block", bind_block),
    IPTQ_METHOD("attention_i8", guarded<attention_i8>),
    IPTQ_METHOD("cache_store_i4", guarded<cache_store_i4>),
    IPTQ_METHOD("attention_cache_i4", guarded<attention_cache_i4>),
    IPTQ_METHOD("rmsnorm_i32", guarded<rmsnorm_i32>),
    IPTQ_METHOD("requant_rows", guarded<requant_rows>),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call(void) { return PyModule_Create(&module); }
