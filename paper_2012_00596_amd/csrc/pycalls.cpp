// CPython entry points of the run calls a serving loop makes once per layer or stack: argument marshalling only, like the
// rest of the binding.  A call through ctypes costs about a microsecond more than this (a conversion object per argument,
// a Python frame per tensor), a fifth of what a small layer takes from call to call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/npas.h"

namespace {

PyObject *error_class; // NpasError(code, message), set by init()
PyObject *c_void_p;    // ctypes.c_void_p, set by init()
PyObject *s_handle, *s_scales, *s_value, *s_is_contiguous, *s_data_ptr, *s_shape, *s_stride, *s_nbytes, *s_itemsize, *s_dtype;

// The arguments of one call, converted in their order.  Once one does not convert, the later conversions do nothing.
struct Args {
    PyObject *const *a;
    enum { PLAIN, FAILED, OTHER } state = PLAIN; // all plain so far; a Python error is set; one is of a kind that is left to ctypes

    // Device pointer: None, an address, or a contiguous tensor.
    void *pointer(int i)
    {
        PyObject *o = a[i];
        if (state != PLAIN || o == Py_None) return nullptr;
        if (PyLong_Check(o)) return number(PyLong_AsUnsignedLongLongMask(o));
        PyObject *c = PyObject_CallMethodNoArgs(o, s_is_contiguous);
        const int yes = c ? PyObject_IsTrue(c) : -1;
        Py_XDECREF(c);
        if (yes == 0) PyErr_SetString(PyExc_AssertionError, "tensor is not contiguous");
        PyObject *p = yes == 1 ? PyObject_CallMethodNoArgs(o, s_data_ptr) : nullptr;
        if (!p) return fail();
        void *v = PyLong_Check(p) ? number(PyLong_AsUnsignedLongLongMask(p)) : other();
        Py_DECREF(p);
        return v;
    }

    // Address that is not a tensor's, such as a stream: None or an integer; ctypes knows the rest (c_void_p, _as_parameter_).
    void *address(int i)
    {
        PyObject *o = a[i];
        if (state != PLAIN || o == Py_None) return nullptr;
        return PyLong_Check(o) ? number(PyLong_AsUnsignedLongLongMask(o)) : other();
    }

    // Library handle of a Packed / Stack object: its `handle` is a ctypes c_void_p, or None once released.
    void *handle(int i) { return handle(i, s_handle); }
    void *handle(int i, PyObject *name)
    {
        if (state != PLAIN) return nullptr;
        PyObject *h = PyObject_GetAttr(a[i], name);
        if (!h) return fail();
        void *v = nullptr;
        if (PyLong_Check(h)) v = number(PyLong_AsUnsignedLongLongMask(h));
        else if (h != Py_None) {
            PyObject *p = PyObject_IsInstance(h, c_void_p) == 1 ? PyObject_GetAttr(h, s_value) : nullptr;
            if (p && PyLong_Check(p)) v = number(PyLong_AsUnsignedLongLongMask(p));
            else if (p != Py_None) v = PyErr_Occurred() ? fail() : other();
            Py_XDECREF(p);
        }
        Py_DECREF(h);
        return v;
    }

    // As ctypes: anything with __index__, an int reduced to 32 bits; no floats.
    int integer(int i) { return (int)(unsigned int)size(i); }
    size_t size(int i)
    {
        if (state != PLAIN) return 0;
        if (PyFloat_Check(a[i])) {
            PyErr_SetString(PyExc_TypeError, "int expected instead of float");
            fail();
            return 0;
        }
        if (!PyIndex_Check(a[i])) return (size_t)(uintptr_t)other();
        return (size_t)(uintptr_t)number(PyLong_AsUnsignedLongLongMask(a[i]));
    }

    float real(int i)
    {
        if (state != PLAIN) return 0.f;
        if (!PyFloat_Check(a[i]) && !PyLong_Check(a[i])) {
            other();
            return 0.f;
        }
        const double v = PyFloat_AsDouble(a[i]);
        if (v == -1.0 && PyErr_Occurred()) fail();
        return (float)v;
    }

    // The same, where a tensor must hold `count` elements of `size` bytes (size 0: of whatever size; the library refuses the type).
    void *elements(int i, int64_t count, int size)
    {
        void *p = pointer(i);
        if (state == PLAIN && is_tensor(i)) {
            const int64_t bytes = attribute(a[i], s_nbytes);
            if (bytes != count * size) { // (just as long: no further look)
                of_size(i, size);
                if (state == PLAIN && bytes < count * size) refuse("tensor is shorter than the call needs");
            }
        }
        return p;
    }
    // ... of `bytes` bytes, whatever its elements.
    void *buffer(int i, size_t bytes)
    {
        void *p = pointer(i);
        if (state == PLAIN && is_tensor(i) && (size_t)attribute(a[i], s_nbytes) < bytes && state == PLAIN) refuse("tensor is shorter than the call needs");
        return p;
    }
    // ... of a 32-bit type: integers, or fp32.
    void *words(int i, int64_t count, bool fp32)
    {
        void *p = pointer(i);
        if (state == PLAIN && is_tensor(i)) {
            of_kind(i, fp32);
            if (state == PLAIN && attribute(a[i], s_nbytes) < count * 4 && state == PLAIN) refuse("tensor is shorter than the call needs");
        }
        return p;
    }

    // Rows of `width` elements of `size` bytes, at least `least` of them: a tensor whose rows are contiguous, or the address of contiguous rows.
    // count: rows of a tensor, -1 of an address.
    struct Rows {
        void *p;
        int64_t stride, count;
    };
    Rows rows(int i, int64_t width, int64_t least, int size)
    {
        PyObject *o = a[i];
        if (state != PLAIN || o == Py_None) return Rows{nullptr, width, -1};
        if (PyLong_Check(o)) return Rows{number(PyLong_AsUnsignedLongLongMask(o)), width, -1};
        Rows r{nullptr, width, 0};
        PyObject *shape = PyObject_GetAttr(o, s_shape), *stride = shape ? PyObject_CallMethodNoArgs(o, s_stride) : nullptr;
        if (!stride) fail();
        else if (!PyTuple_Check(shape) || !PyTuple_Check(stride) || PyTuple_GET_SIZE(shape) != PyTuple_GET_SIZE(stride) || !PyTuple_GET_SIZE(shape)) other();
        else {
            int64_t inner = 1;
            for (Py_ssize_t d = PyTuple_GET_SIZE(shape) - 1; d > 0 && state == PLAIN; --d) {
                const int64_t n = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, d)), by = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, d));
                if (n != 1 && by != inner) refuse("rows are not contiguous");
                inner *= n;
            }
            if (state == PLAIN && inner != width) refuse("rows of another length than the call's");
            r.count = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 0));
            if (r.count > 1) r.stride = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, 0));
            if (state == PLAIN && PyErr_Occurred()) fail();
            if (state == PLAIN && r.count < least) refuse("tensor has fewer rows than the call");
            of_size(i, size);
        }
        Py_XDECREF(shape);
        Py_XDECREF(stride);
        PyObject *p = state == PLAIN ? PyObject_CallMethodNoArgs(o, s_data_ptr) : nullptr;
        if (state == PLAIN) {
            if (!p) fail();
            else if (PyLong_Check(p)) r.p = number(PyLong_AsUnsignedLongLongMask(p));
            else other();
        }
        Py_XDECREF(p);
        return r;
    }
    // ... that is fp32 where it is a tensor.
    Rows rows_fp32(int i, int64_t width)
    {
        const Rows r = rows(i, width, 0, 0);
        if (state == PLAIN && is_tensor(i)) of_kind(i, true);
        return r;
    }
    void refuse(const char *why)
    {
        PyErr_SetString(PyExc_AssertionError, why);
        fail();
    }

private:
    bool is_tensor(int i) const { return a[i] != Py_None && !PyLong_Check(a[i]); }
    // A number that is an attribute of o; -1 where it is not.
    int64_t attribute(PyObject *o, PyObject *name)
    {
        PyObject *v = PyObject_GetAttr(o, name);
        const int64_t n = v ? PyLong_AsLongLong(v) : -1;
        Py_XDECREF(v);
        if (n == -1 && PyErr_Occurred()) fail();
        return n;
    }
    bool yes(PyObject *o, const char *name)
    {
        PyObject *v = PyObject_GetAttrString(o, name);
        const int is = v ? PyObject_IsTrue(v) : -1;
        Py_XDECREF(v);
        if (is < 0) fail();
        return is > 0;
    }
    void of_size(int i, int size)
    {
        if (state == PLAIN && size && attribute(a[i], s_itemsize) != size && state == PLAIN) refuse("tensor of another element size than the call's");
    }
    // 32-bit integers, or fp32.  A type's object stands for the type: the last one that was right needs no further look.
    void of_kind(int i, bool fp32)
    {
        static PyObject *right[2];
        PyObject *t = PyObject_GetAttr(a[i], s_dtype);
        if (!t) fail();
        else if (t != right[fp32]) {
            of_size(i, 4);
            const bool floating = state == PLAIN && yes(t, "is_floating_point"), complex = state == PLAIN && yes(t, "is_complex");
            if (state == PLAIN && (complex || floating != fp32)) refuse(fp32 ? "tensor is not fp32" : "tensor is not of 32-bit integers");
            if (state == PLAIN) {
                Py_INCREF(t);
                Py_XSETREF(right[fp32], t);
            }
        }
        Py_XDECREF(t);
    }
    void *fail()
    {
        state = FAILED;
        return nullptr;
    }
    void *other()
    {
        state = OTHER;
        return nullptr;
    }
    void *number(unsigned long long v) { return v == (unsigned long long)-1 && PyErr_Occurred() ? fail() : (void *)(uintptr_t)v; }
};

PyObject *result(int rc)
{
    if (rc == NPAS_OK) Py_RETURN_NONE;
    PyObject *e = PyObject_CallFunction(error_class, "is", rc, npas_last_error());
    if (e) {
        PyErr_SetObject(error_class, e);
        Py_DECREF(e);
    }
    return nullptr;
}

// What follows the conversions: the library call without the interpreter lock, or, where an argument is of another kind, the
// same call through ctypes (which accepts or refuses it).
enum Call { CONV2D, FC, DEPTHWISE, STACK, NORM, APPEND, ATTENTION, QUANTIZE, DEQUANTIZE, FC_MXFP4, WRITE, READ, ATTENTION8, CHUNK, CALLS };
PyObject *by_ctypes[CALLS]; // set by init()

template <typename F> PyObject *finish(const Args &g, Call which, Py_ssize_t n, F call)
{
    if (g.state == Args::FAILED) return nullptr;
    if (g.state == Args::OTHER) return PyObject_Vectorcall(by_ctypes[which], g.a, (size_t)n, nullptr);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return result(rc);
}

int size_of(int dtype) { return dtype == NPAS_F32 ? 4 : dtype == NPAS_BF16 || dtype == NPAS_F16 ? 2 : 0; }

bool argc(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, n);
    return false;
}

// conv2d_sparse(packed, x, y, N, H, W, stride, pad, bias, residual, act, stream)
PyObject *conv2d_sparse(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 12)) return nullptr;
    Args g{a};
    npas_packed *p = (npas_packed *)g.handle(0);
    void *x = g.pointer(1), *y = g.pointer(2);
    const int N = g.integer(3), H = g.integer(4), W = g.integer(5), stride = g.integer(6), pad = g.integer(7);
    void *b = g.pointer(8), *r = g.pointer(9);
    const int act = g.integer(10);
    void *st = g.address(11);
    return finish(g, CONV2D, n, [&] { return npas_conv2d_sparse(p, x, y, N, H, W, stride, pad, b, r, (npas_act)act, st); });
}

// fc_sparse(packed, x, y, B, bias, act, stream)
PyObject *fc_sparse(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 7)) return nullptr;
    Args g{a};
    npas_packed *p = (npas_packed *)g.handle(0);
    void *x = g.pointer(1), *y = g.pointer(2);
    const int B = g.integer(3);
    void *b = g.pointer(4);
    const int act = g.integer(5);
    void *st = g.address(6);
    return finish(g, FC, n, [&] { return npas_fc_sparse(p, x, y, B, b, (npas_act)act, st); });
}

// depthwise3x3(packed, x, y, N, H, W, stride, bias, residual, act, stream)
PyObject *depthwise3x3(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 11)) return nullptr;
    Args g{a};
    npas_packed *p = (npas_packed *)g.handle(0);
    void *x = g.pointer(1), *y = g.pointer(2);
    const int N = g.integer(3), H = g.integer(4), W = g.integer(5), stride = g.integer(6);
    void *b = g.pointer(7), *r = g.pointer(8);
    const int act = g.integer(9);
    void *st = g.address(10);
    return finish(g, DEPTHWISE, n, [&] { return npas_depthwise3x3(p, x, y, N, H, W, stride, b, r, (npas_act)act, st); });
}

// run_stack(stack, x, y, N, workspace, workspace_bytes, stream)
PyObject *run_stack(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 7)) return nullptr;
    Args g{a};
    npas_stack *s = (npas_stack *)g.handle(0);
    void *x = g.pointer(1), *y = g.pointer(2);
    const int N = g.integer(3);
    void *w = g.pointer(4);
    const size_t bytes = g.size(5);
    void *st = g.address(6);
    return finish(g, STACK, n, [&] { return npas_run_stack(s, x, y, N, w, bytes, st); });
}

// gated_residual_norm(branch, h, h_out, n_out, T, D, dtype, gate, post_weight, pre_weight, residual_scale, eps, stream)
PyObject *gated_residual_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 13)) return nullptr;
    Args g{a};
    const int T = g.integer(4), D = g.integer(5), dt = g.integer(6), size = size_of(dt);
    const int64_t all = (int64_t)T * D;
    void *branch = g.elements(0, all, size), *h = g.elements(1, all, size), *ho = g.elements(2, all, size), *no = g.elements(3, all, size);
    // one row [D] or [1][D] for all tokens, or a row a token
    int64_t stride = 0;
    void *gate = nullptr;
    if (g.state == Args::PLAIN && a[7] != Py_None) {
        PyObject *shape = PyLong_Check(a[7]) ? nullptr : PyObject_GetAttr(a[7], s_shape);
        const Py_ssize_t dims = shape && PyTuple_Check(shape) ? PyTuple_GET_SIZE(shape) : 0;
        const int64_t first = dims ? PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 0)) : 0, last = dims ? PyLong_AsLongLong(PyTuple_GET_ITEM(shape, dims - 1)) : 0;
        Py_XDECREF(shape);
        if (PyErr_Occurred()) return nullptr;
        if (dims == 1 || (dims == 2 && first == 1)) {
            gate = g.elements(7, D, size);
            if (g.state == Args::PLAIN && last != D) g.refuse("gate is [D], [1][D] or [T][D]");
        } else {
            const Args::Rows r = g.rows(7, D, 1, size);
            gate = r.p;
            stride = r.count == 1 ? 0 : r.stride;
            if (g.state == Args::PLAIN && r.count >= 0 && r.count != 1 && r.count != T) g.refuse("gate is [D], [1][D] or [T][D]");
        }
    }
    void *post = g.words(8, D, true), *pre = g.words(9, D, true);
    const float scale = g.real(10), eps = g.real(11);
    void *st = g.address(12);
    return finish(g, NORM, n, [&] {
        return npas_gated_residual_norm(branch, h, gate, stride, (const float *)post, (const float *)pre, scale, eps, ho, no, T, D, (npas_dtype)dt, st);
    });
}

// kv_append(cache, q, k, v, q_out, T, heads, positions, sequences, cos_sin, rot_dim, kind, stream)
PyObject *kv_append(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 13)) return nullptr;
    Args g{a};
    const npas_kv_cache *c = (const npas_kv_cache *)g.handle(0);
    const int T = g.integer(5), heads = g.integer(6), rot = g.integer(10), kind = g.integer(11);
    const int64_t D = c ? c->head_dim : 0, kv = c ? c->kv_heads : 0;
    const Args::Rows q = g.rows(1, heads * D, T, 2), k = g.rows(2, kv * D, T, 2), v = g.rows(3, kv * D, T, 2);
    void *qo = g.elements(4, (int64_t)T * heads * D, 2), *pos = g.words(7, T, false), *seq = g.words(8, T, false);
    const Args::Rows cs = g.rows_fp32(9, rot);
    if (g.state == Args::PLAIN && cs.stride != rot) g.refuse("cos_sin is not contiguous");
    void *st = g.address(12);
    return finish(g, APPEND, n, [&] {
        return npas_kv_append(c, q.p, q.stride, k.p, k.stride, v.p, v.stride, qo, T, heads, (const int32_t *)seq, (const int32_t *)pos,
                              (const float *)cs.p, (int)(cs.count > 0x7fffffff ? 0x7fffffff : cs.count), rot, (npas_rotation)kind, st);
    });
}

// paged_attention(cache, q, y, heads, lengths, max_length, scale, window, lse, workspace, workspace_bytes, stream)
template <Call CALL> PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 12)) return nullptr;
    Args g{a};
    const npas_kv_cache *c = (const npas_kv_cache *)g.handle(0);
    const npas_kv_scales *scales = CALL == ATTENTION8 ? (const npas_kv_scales *)g.handle(0, s_scales) : nullptr;
    const int heads = g.integer(3), most = g.integer(5), window = g.integer(7);
    const int64_t width = (int64_t)heads * (c ? c->head_dim : 0), sequences = c ? c->sequences : 0;
    const Args::Rows q = g.rows(1, width, sequences, 2);
    void *y = g.elements(2, sequences * width, 2), *len = g.words(4, sequences, false);
    const float scale = g.real(6);
    const size_t bytes = g.size(10);
    void *lse = g.words(8, sequences * heads, true), *w = g.buffer(9, bytes);
    void *st = g.address(11);
    return finish(g, CALL, n, [&] {
        if (CALL == ATTENTION8)
            return npas_paged_attention8(c, scales, q.p, q.stride, y, (float *)lse, heads, (const int32_t *)len, most, window, scale, w, bytes, st);
        return npas_paged_attention(c, q.p, q.stride, y, (float *)lse, heads, (const int32_t *)len, most, window, scale, w, bytes, st);
    });
}

// kv_write(cache, q, k, v, q_out, T, heads, positions, sequences, q_weight, k_weight, eps, cos_sin, rot_dim, kind, stream)
PyObject *kv_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 16)) return nullptr;
    Args g{a};
    const npas_kv_cache *c = (const npas_kv_cache *)g.handle(0);
    const npas_kv_scales *scales = (const npas_kv_scales *)g.handle(0, s_scales);
    const int T = g.integer(5), heads = g.integer(6), rot = g.integer(13), kind = g.integer(14);
    const int64_t D = c ? c->head_dim : 0, kv = c ? c->kv_heads : 0;
    const Args::Rows q = g.rows(1, heads * D, T, 2), k = g.rows(2, kv * D, T, 2), v = g.rows(3, kv * D, T, 2);
    void *qo = g.elements(4, (int64_t)T * heads * D, 2), *pos = g.words(7, T, false), *seq = g.words(8, T, false);
    void *qw = g.words(9, D, true), *kw = g.words(10, D, true);
    const float eps = g.real(11);
    const Args::Rows cs = g.rows_fp32(12, rot);
    if (g.state == Args::PLAIN && cs.stride != rot) g.refuse("cos_sin is not contiguous");
    void *st = g.address(15);
    return finish(g, WRITE, n, [&] {
        return npas_kv_write(c, scales, q.p, q.stride, k.p, k.stride, v.p, v.stride, qo, T, heads, (const int32_t *)seq, (const int32_t *)pos,
                             (const float *)qw, (const float *)kw, eps, (const float *)cs.p, (int)(cs.count > 0x7fffffff ? 0x7fffffff : cs.count), rot,
                             (npas_rotation)kind, st);
    });
}

// kv_read(cache, k, v, T, positions, sequences, stream)
PyObject *kv_read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 7)) return nullptr;
    Args g{a};
    const npas_kv_cache *c = (const npas_kv_cache *)g.handle(0);
    const npas_kv_scales *scales = (const npas_kv_scales *)g.handle(0, s_scales);
    const int T = g.integer(3);
    const int64_t count = (int64_t)T * (c ? (int64_t)c->kv_heads * c->head_dim : 0);
    void *k = g.elements(1, count, 2), *v = g.elements(2, count, 2), *pos = g.words(4, T, false), *seq = g.words(5, T, false), *st = g.address(6);
    return finish(g, READ, n, [&] { return npas_kv_read(c, scales, k, v, T, (const int32_t *)seq, (const int32_t *)pos, st); });
}

// chunk_attention(cache, q, y, T, heads, starts, lengths, max_length, scale, window, lse, workspace, workspace_bytes, stream)
PyObject *chunk_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 14)) return nullptr;
    Args g{a};
    const npas_kv_cache *c = (const npas_kv_cache *)g.handle(0);
    const npas_kv_scales *scales = (const npas_kv_scales *)g.handle(0, s_scales);
    const int T = g.integer(3), heads = g.integer(4), most = g.integer(7), window = g.integer(9);
    const int64_t width = (int64_t)heads * (c ? c->head_dim : 0), sequences = c ? c->sequences : 0;
    const Args::Rows q = g.rows(1, width, T, 2);
    void *y = g.elements(2, T * width, 2), *start = g.words(5, sequences + 1, false), *len = g.words(6, sequences, false);
    const float scale = g.real(8);
    const size_t bytes = g.size(12);
    void *lse = g.words(10, (int64_t)T * heads, true), *w = g.buffer(11, bytes);
    void *st = g.address(13);
    return finish(g, CHUNK, n, [&] {
        return npas_chunk_attention(c, scales, q.p, q.stride, y, (float *)lse, T, heads, (const int32_t *)start, (const int32_t *)len, most, window,
                                    scale, w, bytes, st);
    });
}

// mxfp4_quantize(x, codes, scales, M, K, dtype, stream)
PyObject *mxfp4_quantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 7)) return nullptr;
    Args g{a};
    const int M = g.integer(3), K = g.integer(4), dt = g.integer(5);
    const Args::Rows x = g.rows(0, K, M, size_of(dt));
    const int64_t blocks = M * (((int64_t)K + 31) / 32);
    void *codes = g.elements(1, blocks * 16, 1), *scales = g.elements(2, blocks, 1), *st = g.address(6);
    return finish(g, QUANTIZE, n, [&] { return npas_mxfp4_quantize(x.p, x.stride, codes, scales, M, K, (npas_dtype)dt, st); });
}

// mxfp4_dequantize(codes, scales, y, M, K, dtype, stream)
PyObject *mxfp4_dequantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 7)) return nullptr;
    Args g{a};
    const int M = g.integer(3), K = g.integer(4), dt = g.integer(5);
    const int64_t blocks = M * (((int64_t)K + 31) / 32);
    void *codes = g.elements(0, blocks * 16, 1), *scales = g.elements(1, blocks, 1), *y = g.elements(2, (int64_t)M * K, size_of(dt));
    void *st = g.address(6);
    return finish(g, DEQUANTIZE, n, [&] { return npas_mxfp4_dequantize(codes, scales, y, M, K, (npas_dtype)dt, st); });
}

// fc_mxfp4(packed, x, y, B, bias, act, workspace, workspace_bytes, stream, IN, OUT, dtype)
PyObject *fc_mxfp4(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 12)) return nullptr;
    Args g{a};
    npas_mxfp4 *p = (npas_mxfp4 *)g.handle(0);
    const int B = g.integer(3), IN = g.integer(9), OUT = g.integer(10), size = size_of(g.integer(11));
    const Args::Rows x = g.rows(1, IN, B, size);
    void *y = g.elements(2, (int64_t)B * OUT, size), *b = g.words(4, OUT, true);
    const int act = g.integer(5);
    const size_t bytes = g.size(7);
    void *w = g.buffer(6, bytes);
    void *st = g.address(8);
    return finish(g, FC_MXFP4, n, [&] { return npas_fc_mxfp4(p, x.p, x.stride, y, B, b, (npas_act)act, w, bytes, st); });
}

// init(NpasError, c_void_p, the calls through ctypes in the order of Call)
PyObject *init(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!argc(n, 2 + CALLS)) return nullptr;
    auto keep = [](PyObject *&slot, PyObject *o) {
        Py_INCREF(o);
        Py_XSETREF(slot, o);
    };
    keep(error_class, a[0]);
    keep(c_void_p, a[1]);
    for (int i = 0; i < CALLS; ++i) keep(by_ctypes[i], a[2 + i]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"init", (PyCFunction)(void (*)(void))init, METH_FASTCALL, nullptr},
    {"conv2d_sparse", (PyCFunction)(void (*)(void))conv2d_sparse, METH_FASTCALL, nullptr},
    {"fc_sparse", (PyCFunction)(void (*)(void))fc_sparse, METH_FASTCALL, nullptr},
    {"depthwise3x3", (PyCFunction)(void (*)(void))depthwise3x3, METH_FASTCALL, nullptr},
    {"run_stack", (PyCFunction)(void (*)(void))run_stack, METH_FASTCALL, nullptr},
    {"gated_residual_norm", (PyCFunction)(void (*)(void))gated_residual_norm, METH_FASTCALL, nullptr},
    {"kv_append", (PyCFunction)(void (*)(void))kv_append, METH_FASTCALL, nullptr},
    {"paged_attention", (PyCFunction)(void (*)(void))attention<ATTENTION>, METH_FASTCALL, nullptr},
    {"paged_attention8", (PyCFunction)(void (*)(void))attention<ATTENTION8>, METH_FASTCALL, nullptr},
    {"kv_write", (PyCFunction)(void (*)(void))kv_write, METH_FASTCALL, nullptr},
    {"kv_read", (PyCFunction)(void (*)(void))kv_read, METH_FASTCALL, nullptr},
    {"chunk_attention", (PyCFunction)(void (*)(void))chunk_attention, METH_FASTCALL, nullptr},
    {"mxfp4_quantize", (PyCFunction)(void (*)(void))mxfp4_quantize, METH_FASTCALL, nullptr},
    {"mxfp4_dequantize", (PyCFunction)(void (*)(void))mxfp4_dequantize, METH_FASTCALL, nullptr},
    {"fc_mxfp4", (PyCFunction)(void (*)(void))fc_mxfp4, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pycalls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__pycalls()
{
    s_handle = PyUnicode_InternFromString("handle");
    s_scales = PyUnicode_InternFromString("scales");
    s_value = PyUnicode_InternFromString("value");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    s_itemsize = PyUnicode_InternFromString("itemsize");
    s_dtype = PyUnicode_InternFromString("dtype");
    if (!s_handle || !s_scales || !s_value || !s_is_contiguous || !s_data_ptr || !s_shape || !s_stride || !s_nbytes || !s_itemsize || !s_dtype) return nullptr;
    return PyModule_Create(&module);
}
