// The layer, flatten, retile and token calls as a Python extension module: arguments go from Python objects straight into the call's
// C arguments.  A training step of a small chain is six calls with 27 shard lists between them; through ctypes they took
// 44 us of host time, as long as the GPU needs for half the kernels, and so 12 us.
//
// Every function takes the address of the library's function first (the library itself knows nothing of Python).  What is
// accepted is what the ctypes binding accepts: shard lists are None (a NULL list) or sequences of objects with a data_ptr()
// or of integers; tilings and forms are strings, or whatever binding.tiling() / binding.forms() take.  The interpreter's
// lock is released during a call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <cstring>
#include <type_traits>
#include "tensor_tiling.h"
#include "tensor_tiling_tokens.h"
#if __has_include(<ATen/dlpack.h>)
#include <ATen/dlpack.h>
#endif
#if defined(DLPACK_MAJOR_VERSION) && (DLPACK_MAJOR_VERSION > 1 || DLPACK_MINOR_VERSION >= 3)
#define TT_DLPACK_EXCHANGE
#endif

namespace {

constexpr int kMaxShards = 1 << TT_MAX_K;

PyObject *g_data_ptr, *g_numel, *g_element_size, *g_value, *g_dtype_name, *g_is_contiguous; // method and attribute names
PyObject *g_tiling, *g_forms, *g_dtype;                     // the binding's own converters, for the rarer forms
PyObject *g_error;                                          // its exception: (status, what)
PyObject *g_float32;                                        // torch.float32, once a tensor was seen

// What a dense tensor is to a call
struct Described {
    uint64_t address;
    int64_t entries;
    bool fp32, dense;
};
#ifdef TT_DLPACK_EXCHANGE
// A tensor type's DLPack functions: all of the above in one call (a policy loss with seven arrays takes 8.3 us of host time, 9.1
// by data_ptr(), dtype, numel() and is_contiguous(), and took 8.4 when only the address was asked for).
PyObject *g_exchange_name, *g_exchange_type, *g_exchange_capsule; // of the type that was seen last
const DLPackExchangeAPI *g_exchange;
const DLPackExchangeAPI *exchange_of(PyObject *o)
{
    PyObject *type = reinterpret_cast<PyObject *>(Py_TYPE(o));
    if (type == g_exchange_type) return g_exchange;
    PyObject *capsule = PyObject_GetAttr(type, g_exchange_name);
    auto *api = capsule && PyCapsule_IsValid(capsule, "dlpack_exchange_api")
                    ? static_cast<const DLPackExchangeAPI *>(PyCapsule_GetPointer(capsule, "dlpack_exchange_api")) : nullptr;
    PyErr_Clear();
    if (!api || api->header.version.major != DLPACK_MAJOR_VERSION || api->header.version.minor < 3 || !api->dltensor_from_py_object_no_sync) {
        Py_XDECREF(capsule);
        return nullptr;
    }
    Py_INCREF(type);
    Py_XSETREF(g_exchange_type, type);
    Py_XSETREF(g_exchange_capsule, capsule);
    return g_exchange = api;
}
bool described(PyObject *o, Described *d)
{
    const DLPackExchangeAPI *api = exchange_of(o);
    DLTensor t;
    if (!api) return false;
    if (api->dltensor_from_py_object_no_sync(o, &t) != 0) {
        PyErr_Clear(); // (what has no such form is asked by its methods)
        return false;
    }
    d->address = (uint64_t)(uintptr_t)t.data + t.byte_offset;
    d->fp32 = t.dtype.code == kDLFloat && t.dtype.bits == 32 && t.dtype.lanes == 1;
    d->entries = 1;
    d->dense = true;
    for (int i = t.ndim - 1; i >= 0; --i) {
        if (t.shape[i] != 1 && t.strides && t.strides[i] != d->entries) d->dense = false;
        d->entries *= t.shape[i];
    }
    return true;
}
#else
bool described(PyObject *, Described *) { return false; }
#endif

// Arguments of one call.  The first failure leaves a Python exception set and every later step a no-op.
struct Args {
    PyObject *const *a;
    Py_ssize_t n, i = 0;
    bool ok = true;
    PyObject *held[8]; // objects whose buffers the call reads
    Py_buffer view[8];
    int n_held = 0, n_view = 0;

    Args(PyObject *const *args, Py_ssize_t nargs, Py_ssize_t want) : a(args), n(nargs)
    {
        if (n != want) {
            PyErr_Format(PyExc_TypeError, "%zd arguments expected, not %zd", want, n);
            ok = false;
        }
    }
    ~Args()
    {
        for (int v = 0; v < n_view; ++v) PyBuffer_Release(&view[v]);
        for (int h = 0; h < n_held; ++h) Py_DECREF(held[h]);
    }
    PyObject *next() { return ok ? a[i++] : nullptr; }
    bool fail() { return ok = false; }

    // an integer, wrapped to 64 bits as ctypes does
    uint64_t integer_of(PyObject *o)
    {
        PyObject *x = PyNumber_Index(o);
        if (!x) { fail(); return 0; }
        const uint64_t v = PyLong_AsUnsignedLongLongMask(x);
        Py_DECREF(x);
        if (v == ~0ull && PyErr_Occurred()) fail();
        return v;
    }
    int64_t i64() { PyObject *o = next(); return o ? (int64_t)integer_of(o) : 0; }
    int i32() { return (int)i64(); }
    template <class F> F address() { return reinterpret_cast<F>((uintptr_t)i64()); }
    int flag()
    {
        PyObject *o = next();
        if (!o) return 0;
        const int v = PyObject_IsTrue(o);
        if (v < 0) fail();
        return v > 0;
    }
    float real()
    {
        PyObject *o = next();
        if (!o) return 0.0f;
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) fail();
        return (float)v;
    }
    void refuse(const char *what, const char *why)
    {
        if (PyObject *e = PyObject_CallFunction(g_error, "iN", (int)TT_EINVAL, PyUnicode_FromFormat("%s: %s", what, why))) {
            PyErr_SetObject(g_error, e);
            Py_DECREF(e);
        }
        fail();
    }
    // A per-token array of `count` entries: a dense tensor, an address (anything without a dtype is taken for one), or None (NULL).
    // These are the tensors that come out of slicing: a strided one, one of another type or a short one would be read as if it
    // were not.
    template <typename T = void> T *array(const char *what, int64_t count)
    {
        PyObject *o = next();
        if (!o || o == Py_None) return nullptr;
        Described d{0, count, true, true};
        if (!described(o, &d)) {
            d.address = pointer_of(o);
            if (ok && !PyLong_CheckExact(o)) ask(o, &d);
        }
        if (ok && count > 0) {
            if (std::is_same<typename std::remove_const<T>::type, float>::value && !d.fp32) refuse(what, "fp32 values are expected");
            else if (d.entries < count) refuse(what, "fewer entries than tokens");
            else if (!d.dense) refuse(what, "a dense tensor is expected");
        }
        return reinterpret_cast<T *>((uintptr_t)d.address);
    }
    // by an object's methods; left as it is without a dtype
    void ask(PyObject *o, Described *d)
    {
        PyObject *type = PyObject_GetAttr(o, g_dtype_name);
        if (!type) {
            if (PyErr_ExceptionMatches(PyExc_AttributeError)) PyErr_Clear();
            else fail();
            return;
        }
        d->fp32 = type == g_float32 || is_float32(type);
        Py_DECREF(type);
        if (ok) d->entries = (int64_t)method(o, g_numel);
        if (ok) d->dense = truth(o, g_is_contiguous);
    }
    bool is_float32(PyObject *type)
    {
        if (!g_float32) {
            PyObject *torch = PyImport_ImportModule("torch");
            g_float32 = torch ? PyObject_GetAttrString(torch, "float32") : nullptr;
            Py_XDECREF(torch);
            if (!g_float32) return fail();
        }
        return type == g_float32;
    }
    bool truth(PyObject *o, PyObject *name)
    {
        PyObject *x = PyObject_CallMethodNoArgs(o, name);
        const int v = x ? PyObject_IsTrue(x) : -1;
        Py_XDECREF(x);
        if (v < 0) fail();
        return v > 0;
    }
    // bytes of a ctypes object, valid until the call is over
    const void *bytes_of(PyObject *o, Py_ssize_t least)
    {
        if (n_view == 8 || PyObject_GetBuffer(o, &view[n_view], PyBUF_SIMPLE) != 0) { fail(); return nullptr; }
        const Py_buffer &v = view[n_view++];
        if (v.len < least) {
            PyErr_SetString(PyExc_TypeError, "structure of another type");
            fail();
            return nullptr;
        }
        return v.buf;
    }
    PyObject *converted(PyObject *converter, PyObject *o) // kept until the call is over
    {
        PyObject *x = n_held < 8 ? PyObject_CallOneArg(converter, o) : nullptr;
        if (!x) { fail(); return nullptr; }
        return held[n_held++] = x;
    }
    const tt_layer *layer()
    {
        PyObject *o = next();
        return o ? static_cast<const tt_layer *>(bytes_of(o, sizeof(tt_layer))) : nullptr;
    }
    tt_tiling tiling()
    {
        tt_tiling t;
        std::memset(&t, 0, sizeof(t));
        PyObject *o = next();
        if (!o) return t;
        if (PyUnicode_CheckExact(o) && PyUnicode_GET_LENGTH(o) <= TT_MAX_K) {
            for (Py_ssize_t j = 0; j < PyUnicode_GET_LENGTH(o); ++j) {
                const Py_UCS4 c = PyUnicode_READ_CHAR(o, j);
                t.cut[j] = c == 'R' ? TT_R : c == 'C' ? TT_C : c == 'r' ? TT_REP : 255;
            }
            return t;
        }
        PyObject *x = converted(g_tiling, o);
        if (const void *b = x ? bytes_of(x, sizeof(t)) : nullptr) std::memcpy(&t, b, sizeof(t));
        return t;
    }
    const uint8_t *forms(uint8_t (&buf)[TT_MAX_K])
    {
        PyObject *o = next();
        if (!o || o == Py_None) return nullptr;
        std::memset(buf, 255, sizeof(buf)); // (no form: a sequence shorter than k is refused)
        if (PyUnicode_CheckExact(o) && PyUnicode_GET_LENGTH(o) <= TT_MAX_K) {
            Py_ssize_t j = 0;
            for (; j < PyUnicode_GET_LENGTH(o); ++j) {
                const Py_UCS4 c = PyUnicode_READ_CHAR(o, j);
                if (c < '1' || c > '9') break;
                buf[j] = (uint8_t)(c - '1');
            }
            if (j == PyUnicode_GET_LENGTH(o)) return buf;
        }
        PyObject *x = converted(g_forms, o);
        return x ? static_cast<const uint8_t *>(bytes_of(x, TT_MAX_K)) : nullptr; // (the converter fills up short sequences)
    }
    int dtype()
    {
        PyObject *o = next();
        if (!o) return 0;
        if (PyUnicode_CheckExact(o)) {
            if (PyUnicode_CompareWithASCIIString(o, "bf16") == 0) return TT_BF16;
            if (PyUnicode_CompareWithASCIIString(o, "f32") == 0) return TT_F32;
        }
        PyObject *x = converted(g_dtype, o);
        return x ? (int)integer_of(x) : 0;
    }
    uint64_t pointer_of(PyObject *o)
    {
        PyObject *p = PyObject_CallMethodNoArgs(o, g_data_ptr);
        if (!p) {
            if (!PyErr_ExceptionMatches(PyExc_AttributeError)) { fail(); return 0; }
            PyErr_Clear();
            p = PyNumber_Long(o);
            if (!p) { fail(); return 0; }
        }
        const uint64_t v = integer_of(p);
        Py_DECREF(p);
        return v;
    }
    // a shard list; entries past the last one given are NULL
    void **shards(void *(&buf)[kMaxShards])
    {
        PyObject *o = next();
        if (!o || o == Py_None) return nullptr;
        PyObject *s = PySequence_Fast(o, "a shard list is a sequence");
        if (!s) { fail(); return nullptr; }
        for (Py_ssize_t j = 0; j < kMaxShards; ++j) { // (data_ptr() is Python code: the length is read anew)
            buf[j] = nullptr;
            if (!ok || j >= PySequence_Fast_GET_SIZE(s)) continue;
            PyObject *item = PySequence_Fast_GET_ITEM(s, j);
            Py_INCREF(item);
            buf[j] = reinterpret_cast<void *>((uintptr_t)pointer_of(item));
            Py_DECREF(item);
        }
        Py_DECREF(s);
        return buf;
    }
    uint64_t method(PyObject *o, PyObject *name)
    {
        PyObject *x = PyObject_CallMethodNoArgs(o, name);
        if (!x) { fail(); return 0; }
        const uint64_t v = integer_of(x);
        Py_DECREF(x);
        return v;
    }
    void *workspace(size_t *bytes)
    {
        *bytes = 0;
        PyObject *o = next();
        if (!o || o == Py_None) return nullptr;
        const uint64_t p = method(o, g_data_ptr);
        if (ok) *bytes = (size_t)method(o, g_numel);
        if (ok) *bytes *= (size_t)method(o, g_element_size);
        return reinterpret_cast<void *>((uintptr_t)p);
    }
    // a handle: an integer, None or a ctypes pointer
    void *stream()
    {
        PyObject *o = next();
        if (!o || o == Py_None) return nullptr;
        if (PyLong_CheckExact(o)) return reinterpret_cast<void *>((uintptr_t)integer_of(o));
        PyObject *v = PyObject_GetAttr(o, g_value);
        if (!v) { fail(); return nullptr; }
        void *p = v == Py_None ? nullptr : reinterpret_cast<void *>((uintptr_t)integer_of(v));
        Py_DECREF(v);
        return p;
    }
};

template <class F> PyObject *finish(Args &g, F &&call)
{
    if (!g.ok) return nullptr;
    tt_status st;
    Py_BEGIN_ALLOW_THREADS
    st = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

const void *const *in(void **p) { return const_cast<const void *const *>(p); }

// forward(address, layer, batch, k, dtype, tX, tW, tY, forms, X, W, Y, workspace, stream): tt_fc_forward, tt_conv_forward
PyObject *forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args g(args, n, 14);
    auto fn = g.address<decltype(&tt_fc_forward)>();
    const tt_layer *lay = g.layer();
    const int64_t batch = g.i64();
    const int k = g.i32(), dt = g.dtype();
    const tt_tiling tX = g.tiling(), tW = g.tiling(), tY = g.tiling();
    uint8_t fb[TT_MAX_K];
    void *x[kMaxShards], *w[kMaxShards], *y[kMaxShards];
    const uint8_t *f = g.forms(fb);
    void **X = g.shards(x), **W = g.shards(w), **Y = g.shards(y);
    size_t bytes;
    void *ws = g.workspace(&bytes), *stream = g.stream();
    return finish(g, [&] { return fn(lay, batch, k, dt, tX, tW, tY, f, in(X), in(W), Y, ws, bytes, stream); });
}

// forward_static(address, layer, batch, k, dtype, tX, tW, tY, forms, X, W, Y, stream): tt_fc_forward_static
PyObject *forward_static(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args g(args, n, 13);
    auto fn = g.address<decltype(&tt_fc_forward_static)>();
    const tt_layer *lay = g.layer();
    const int64_t batch = g.i64();
    const int k = g.i32(), dt = g.dtype();
    const tt_tiling tX = g.tiling(), tW = g.tiling(), tY = g.tiling();
    uint8_t fb[TT_MAX_K];
    void *x[kMaxShards], *w[kMaxShards], *y[kMaxShards];
    const uint8_t *f = g.forms(fb);
    void **X = g.shards(x), **W = g.shards(w), **Y = g.shards(y);
    void *stream = g.stream();
    return finish(g, [&] { return fn(lay, batch, k, dt, tX, tW, tY, f, in(X), in(W), Y, stream); });
}

// backward(address, layer, batch, k, dtype, tX, tW, tY, tdY, tdX, forms_dgrad, forms_wgrad, X, W, Y, dY, dX, dW, workspace,
// stream): tt_fc_backward, tt_conv_backward
PyObject *backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args g(args, n, 20);
    auto fn = g.address<decltype(&tt_fc_backward)>();
    const tt_layer *lay = g.layer();
    const int64_t batch = g.i64();
    const int k = g.i32(), dt = g.dtype();
    const tt_tiling tX = g.tiling(), tW = g.tiling(), tY = g.tiling(), tdY = g.tiling(), tdX = g.tiling();
    uint8_t fdb[TT_MAX_K], fwb[TT_MAX_K];
    void *x[kMaxShards], *w[kMaxShards], *y[kMaxShards], *dy[kMaxShards], *dx[kMaxShards], *dw[kMaxShards];
    const uint8_t *fd = g.forms(fdb), *fw = g.forms(fwb);
    void **X = g.shards(x), **W = g.shards(w), **Y = g.shards(y), **dY = g.shards(dy), **dX = g.shards(dx), **dW = g.shards(dw);
    size_t bytes;
    void *ws = g.workspace(&bytes), *stream = g.stream();
    return finish(g, [&] {
        return fn(lay, batch, k, dt, tX, tW, tY, tdY, tdX, fd, fw, in(X), in(W), in(Y), in(dY), dX, dW, ws, bytes, stream);
    });
}

// flatten(address, dst, B, src, A, k, batch, channels, pixels, elem_bytes, to_matrix, stream): tt_flatten
PyObject *flatten(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args g(args, n, 12);
    auto fn = g.address<decltype(&tt_flatten)>();
    void *d[kMaxShards], *s[kMaxShards];
    void **dst = g.shards(d);
    const tt_tiling B = g.tiling();
    void **src = g.shards(s);
    const tt_tiling A = g.tiling();
    const int k = g.i32();
    const int64_t batch = g.i64(), channels = g.i64(), pixels = g.i64();
    const int eb = g.i32(), to_matrix = g.flag();
    void *stream = g.stream();
    return finish(g, [&] { return fn(dst, B, in(src), A, k, batch, channels, pixels, eb, to_matrix, stream); });
}

// retile(address, dst, B, src, A, k, rows, cols, elem_bytes, stream): tt_retile
PyObject *retile(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args g(args, n, 10);
    auto fn = g.address<decltype(&tt_retile)>();
    void *d[kMaxShards], *s[kMaxShards];
    void **dst = g.shards(d);
    const tt_tiling B = g.tiling();
    void **src = g.shards(s);
    const tt_tiling A = g.tiling();
    const int k = g.i32();
    const int64_t rows = g.i64(), cols = g.i64();
    const int eb = g.i32();
    void *stream = g.stream();
    return finish(g, [&] { return fn(dst, B, in(src), A, k, rows, cols, eb, stream); });
}

// embed_forward(address, tokens, vocab, width, k, dtype, tW, tX, id_dtype, ids, scale, W, X, stream): tt_embed_forward
PyObject *embed_forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args g(args, n, 14);
    auto fn = g.address<decltype(&tt_embed_forward)>();
    const int64_t tokens = g.i64(), vocab = g.i64(), width = g.i64();
    const int k = g.i32(), dt = g.dtype();
    const tt_tiling tW = g.tiling(), tX = g.tiling();
    const int idt = g.i32();
    const void *ids = g.array<const void>("ids", tokens);
    const float scale = g.real();
    void *w[kMaxShards], *x[kMaxShards];
    void **W = g.shards(w), **X = g.shards(x);
    void *stream = g.stream();
    return finish(g, [&] { return fn(tokens, vocab, width, k, dt, tW, tX, idt, ids, scale, in(W), X, stream); });
}

// embed_backward(address, tokens, vocab, width, k, dtype, tdX, tdW, id_dtype, ids, scale, dX, dW, workspace, stream): tt_embed_backward
PyObject *embed_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args g(args, n, 15);
    auto fn = g.address<decltype(&tt_embed_backward)>();
    const int64_t tokens = g.i64(), vocab = g.i64(), width = g.i64();
    const int k = g.i32(), dt = g.dtype();
    const tt_tiling tX = g.tiling(), tW = g.tiling();
    const int idt = g.i32();
    const void *ids = g.array<const void>("ids", tokens);
    const float scale = g.real();
    void *dx[kMaxShards], *dw[kMaxShards];
    void **dX = g.shards(dx), **dW = g.shards(dw);
    size_t bytes;
    void *ws = g.workspace(&bytes), *stream = g.stream();
    return finish(g, [&] { return fn(tokens, vocab, width, k, dt, tX, tW, idt, ids, scale, in(dX), dW, ws, bytes, stream); });
}

// policy_loss(address, policy, tokens, vocab, k, dtype, tX, tdX, X, id_dtype, actions, old_logp, ref_logp, advantage, weight, loss,
// logp, dX, workspace, stream): tt_policy_loss
PyObject *policy_loss(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args g(args, n, 20);
    auto fn = g.address<decltype(&tt_policy_loss)>();
    PyObject *o = g.next();
    const tt_policy *policy = o ? static_cast<const tt_policy *>(g.bytes_of(o, sizeof(tt_policy))) : nullptr;
    const int64_t tokens = g.i64(), vocab = g.i64();
    const int k = g.i32(), dt = g.dtype();
    const tt_tiling tX = g.tiling(), tdX = g.tiling();
    void *x[kMaxShards], *dx[kMaxShards];
    void **X = g.shards(x);
    const int idt = g.i32();
    const void *actions = g.array<const void>("actions", tokens);
    const float *old_logp = g.array<const float>("old_logp", tokens);
    const float *ref_logp = g.array<const float>("ref_logp", policy && policy->kl != 0.0f ? tokens : 0); // (not read otherwise)
    const float *advantage = g.array<const float>("advantage", tokens), *weight = g.array<const float>("weight", tokens);
    float *loss = g.array<float>("loss", 1), *logp = g.array<float>("logp", tokens);
    void **dX = g.shards(dx);
    size_t bytes;
    void *ws = g.workspace(&bytes), *stream = g.stream();
    return finish(g, [&] {
        return fn(policy, tokens, vocab, k, dt, tX, tdX, in(X), idt, actions, old_logp, ref_logp, advantage, weight, loss, logp, dX, ws, bytes, stream);
    });
}

// token_logp(address, tokens, vocab, k, dtype, tX, scale, X, id_dtype, ids, logp, workspace, stream): tt_token_logp
PyObject *token_logp(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args g(args, n, 13);
    auto fn = g.address<decltype(&tt_token_logp)>();
    const int64_t tokens = g.i64(), vocab = g.i64();
    const int k = g.i32(), dt = g.dtype();
    const tt_tiling tX = g.tiling();
    const float scale = g.real();
    void *x[kMaxShards];
    void **X = g.shards(x);
    const int idt = g.i32();
    const void *ids = g.array<const void>("ids", tokens);
    float *logp = g.array<float>("logp", tokens);
    size_t bytes;
    void *ws = g.workspace(&bytes), *stream = g.stream();
    return finish(g, [&] { return fn(tokens, vocab, k, dt, tX, scale, in(X), idt, ids, logp, ws, bytes, stream); });
}

// pack8(address, rows, cols, k, dtype, t, a, b, c, stream): tt_pack8 (X, Q, S) and tt_unpack8 (Q, S, X), whose shard lists are
// arrays of pointers alike
PyObject *pack8(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args g(args, n, 10);
    typedef tt_status (*Fn)(int64_t, int64_t, int, int, tt_tiling, void *const *, void *const *, void *const *, void *);
    auto fn = g.address<Fn>();
    const int64_t rows = g.i64(), cols = g.i64();
    const int k = g.i32(), dt = g.dtype();
    const tt_tiling t = g.tiling();
    void *a[kMaxShards], *b[kMaxShards], *c[kMaxShards];
    void **A = g.shards(a), **B = g.shards(b), **C = g.shards(c);
    void *stream = g.stream();
    return finish(g, [&] { return fn(rows, cols, k, dt, t, A, B, C, stream); });
}

// backward_packed(address, layer, batch, k, dtype, tX, tW, tY, tdY, tdX, forms_dgrad, forms_wgrad, XQ, XS, W, YQ, YS, dY, dX, dW,
// workspace, stream): tt_fc_backward_packed
PyObject *backward_packed(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args g(args, n, 22);
    auto fn = g.address<decltype(&tt_fc_backward_packed)>();
    const tt_layer *lay = g.layer();
    const int64_t batch = g.i64();
    const int k = g.i32(), dt = g.dtype();
    const tt_tiling tX = g.tiling(), tW = g.tiling(), tY = g.tiling(), tdY = g.tiling(), tdX = g.tiling();
    uint8_t fdb[TT_MAX_K], fwb[TT_MAX_K];
    void *xq[kMaxShards], *xs[kMaxShards], *w[kMaxShards], *yq[kMaxShards], *ys[kMaxShards], *dy[kMaxShards], *dx[kMaxShards], *dw[kMaxShards];
    const uint8_t *fd = g.forms(fdb), *fw = g.forms(fwb);
    void **XQ = g.shards(xq), **XS = g.shards(xs), **W = g.shards(w), **YQ = g.shards(yq), **YS = g.shards(ys), **dY = g.shards(dy);
    void **dX = g.shards(dx), **dW = g.shards(dw);
    size_t bytes;
    void *ws = g.workspace(&bytes), *stream = g.stream();
    const auto i8 = [](void **p) { return reinterpret_cast<const int8_t *const *>(p); };
    const auto u8 = [](void **p) { return reinterpret_cast<const uint8_t *const *>(p); };
    return finish(g, [&] {
        return fn(lay, batch, k, dt, tX, tW, tY, tdY, tdX, fd, fw, i8(XQ), u8(XS), in(W), i8(YQ), u8(YS), in(dY), dX, dW, ws, bytes, stream);
    });
}

// converters(tiling, forms, dtype, error): what the binding uses for arguments that are no plain strings, and its exception
PyObject *converters(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 4) {
        PyErr_SetString(PyExc_TypeError, "4 arguments expected");
        return nullptr;
    }
    PyObject **const to[4] = {&g_tiling, &g_forms, &g_dtype, &g_error};
    for (int i = 0; i < 4; ++i) {
        Py_INCREF(args[i]);
        Py_XSETREF(*to[i], args[i]);
    }
    Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)> PyMethodDef method_def(const char *name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef g_methods[] = {method_def<forward>("forward"), method_def<forward_static>("forward_static"), method_def<backward>("backward"),
                           method_def<flatten>("flatten"), method_def<retile>("retile"), method_def<embed_forward>("embed_forward"), method_def<embed_backward>("embed_backward"),
                           method_def<policy_loss>("policy_loss"), method_def<token_logp>("token_logp"), method_def<pack8>("pack8"),
                           method_def<backward_packed>("backward_packed"), method_def<converters>("converters"),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__calls()
{
    g_data_ptr = PyUnicode_InternFromString("data_ptr");
    g_numel = PyUnicode_InternFromString("numel");
    g_element_size = PyUnicode_InternFromString("element_size");
    g_value = PyUnicode_InternFromString("value");
    g_dtype_name = PyUnicode_InternFromString("dtype");
    g_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    if (!g_data_ptr || !g_numel || !g_element_size || !g_value || !g_dtype_name || !g_is_contiguous) return nullptr;
#ifdef TT_DLPACK_EXCHANGE
    if (!(g_exchange_name = PyUnicode_InternFromString("__dlpack_c_exchange_api__"))) return nullptr;
#endif
    return PyModule_Create(&g_module);
}
