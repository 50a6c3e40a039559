// The calls of the operators around the matmuls (norm, 4-bit cache, attention)
// of tilefuse.py in native code, as tf_binding.cpp has the matmul calls: argument
// checks, outputs, workspace and current stream, then the C ABI call, in one entry
// from Python.  Only calls in the common form are taken (plain tensors of the
// documented types and shapes, Python numbers); anything else, and every refusal,
// returns NotImplemented, and the general path in tilefuse.py runs it or raises.
// Measured on MI355X, us a call in a loop, through ctypes -> here: norm of one
// row of 4096 11.6 -> 5.6, attention of one token on 513 15.6 -> 9.2.
#include <ATen/ops/empty.h>
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>

#include "tf_binding_shared.h"
#include "tilefuse.h"

namespace {

using tf_binding::Held;

PyObject* not_here() { return Py_NewRef(Py_NotImplemented); }

// A plain tensor (no subclass) on the GPU, with strides.
const at::Tensor* on_gpu(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.layout() == at::kStrided ? &t : nullptr;
}
// The same, contiguous.
const at::Tensor* plain(PyObject* o) {
    const at::Tensor* t = on_gpu(o);
    return t && t->is_contiguous() ? t : nullptr;
}

struct Ops {
    decltype(&tf_add_rms_norm) norm;
    decltype(&tf_kv4_append) append;
    decltype(&tf_kv4_read) read;
    decltype(&tf_kv4_attention_workspace_bytes) decode_bytes;
    decltype(&tf_kv4_attention) decode;
    decltype(&tf_prompt_attention_workspace_bytes) prompt_bytes;
    decltype(&tf_prompt_attention) prompt;
    tf_binding::CaptureFn capture;
} g_ops;
PyObject *g_ops_stream, *g_decode_ws, *g_prompt_ws, *g_make_ws;
PyObject *g_name_data, *g_name_sizes, *g_name_device;

// bind((addresses in the order of Ops), current stream function, workspace
//          dicts of decode and prompt attention, function that makes a workspace)
PyObject* bind(PyObject*, PyObject* args) {
    PyObject *fns, *stream, *decode_ws, *prompt_ws, *make;
    if (!PyArg_ParseTuple(args, "O!OO!O!O", &PyTuple_Type, &fns, &stream, &PyDict_Type, &decode_ws, &PyDict_Type,
                          &prompt_ws, &make))
        return nullptr;
    unsigned long long at[8];
    if (PyTuple_GET_SIZE(fns) != 8) {
        PyErr_SetString(PyExc_ValueError, "bind needs eight functions");
        return nullptr;
    }
    for (int i = 0; i < 8; ++i) {
        at[i] = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(fns, i));
        if (PyErr_Occurred()) return nullptr;
    }
    g_ops = {reinterpret_cast<decltype(Ops::norm)>(at[0]),         reinterpret_cast<decltype(Ops::append)>(at[1]),
             reinterpret_cast<decltype(Ops::read)>(at[2]),         reinterpret_cast<decltype(Ops::decode_bytes)>(at[3]),
             reinterpret_cast<decltype(Ops::decode)>(at[4]),       reinterpret_cast<decltype(Ops::prompt_bytes)>(at[5]),
             reinterpret_cast<decltype(Ops::prompt)>(at[6]),
             reinterpret_cast<decltype(Ops::capture)>(at[7])};
    Py_XSETREF(g_ops_stream, Py_NewRef(stream));
    Py_XSETREF(g_decode_ws, Py_NewRef(decode_ws));
    Py_XSETREF(g_prompt_ws, Py_NewRef(prompt_ws));
    Py_XSETREF(g_make_ws, Py_NewRef(make));
    Py_RETURN_NONE;
}

int dtype_code(const at::Tensor& t) {
    return t.scalar_type() == at::kHalf ? TF_F16 : t.scalar_type() == at::kBFloat16 ? TF_BF16 : 0;
}
// Contiguous, of that type, device and shape.
bool is(const at::Tensor* t, at::ScalarType type, int dev, at::IntArrayRef shape) {
    return t && t->scalar_type() == type && t->get_device() == dev && t->is_contiguous() && t->sizes() == shape;
}
// [tokens, heads, head_dim] whose tokens may be strided: the stride, or -1.
int64_t heads_stride(const at::Tensor& t) {
    if (t.dim() != 3) return -1;
    const int64_t T = t.size(0), H = t.size(1), D = t.size(2);
    if (T < 1 || H < 1 || t.stride(2) != 1 || (H > 1 && t.stride(1) != D)) return -1;
    return T > 1 ? t.stride(0) : H * D;
}
bool as_float(PyObject* o, float& v) {
    if (PyFloat_CheckExact(o)) v = (float)PyFloat_AS_DOUBLE(o);
    else if (PyLong_CheckExact(o)) v = (float)PyLong_AsDouble(o);
    else return false;
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}
const void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
const int32_t* ints(const at::Tensor* t) { return static_cast<const int32_t*>(t->data_ptr()); }

// A cache object's buffer and sizes, and a page table for it.
struct Cache {
    tf_kv4_cache c{};
    at::ScalarType type = at::kHalf;
    int dev = -1;
    Held data, sizes;
    bool read(PyObject* cache, const at::Tensor* table, int64_t batch) {
        data.o = PyObject_GetAttr(cache, g_name_data);
        sizes.o = data.o ? PyObject_GetAttr(cache, g_name_sizes) : nullptr;
        if (!sizes.o) { PyErr_Clear(); return false; }
        const at::Tensor* d = plain(data.o);
        if (!d || !PyTuple_CheckExact(sizes.o) || PyTuple_GET_SIZE(sizes.o) != 5) return false;
        int64_t v[5];
        for (int i = 0; i < 5; ++i) v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(sizes.o, i));
        if (PyErr_Occurred()) { PyErr_Clear(); return false; }
        dev = d->get_device();
        if (!table || table->scalar_type() != at::kInt || table->dim() != 2 || table->get_device() != dev ||
            table->size(0) != batch || (table->size(1) > 1 && table->stride(1) != 1))
            return false;
        type = v[4] == TF_BF16 ? at::kBFloat16 : at::kHalf;
        c.data = d->data_ptr();
        c.pages = v[0];
        c.page_size = (int32_t)v[1];
        c.kv_heads = (int32_t)v[2];
        c.head_dim = (int32_t)v[3];
        c.dtype = (int32_t)v[4];
        c.table = ints(table);
        c.max_pages = table->size(1);
        c.table_stride = batch > 1 ? table->stride(0) : table->size(1);
        return true;
    }
};

// The workspace of an attention call on `stream`: None the cached one, False none
// (where allowed), or the caller's.
bool workspace_of(PyObject* o, PyObject* cached, PyObject* any, int dev, void* stream, int64_t need, Held& held,
                  void*& ws, size_t& bytes) {
    ws = nullptr;
    bytes = 0;
    if (o == Py_False) return true;
    const at::Tensor* t = nullptr;
    if (o == Py_None) {
        if (need == 0) return true;
        if (!tf_binding::find_workspace(cached, g_ops.capture, dev, stream, held)) return false;
        t = held.o ? plain(held.o) : nullptr;
        if (!t || (int64_t)t->nbytes() < need) {
            const Held device{PyObject_GetAttr(any, g_name_device)};
            if (!device.o) return false;
            Py_XSETREF(held.o, PyObject_CallFunction(g_make_ws, "OOL", cached, device.o, (long long)need));
            if (!held.o) return false;
            t = plain(held.o);
        }
    } else {
        t = plain(o);
    }
    if (!t) return false;
    ws = t->data_ptr();
    bytes = t->nbytes();
    return true;
}

// norm(x, residual, weight, post_weight, gate, scale, offset, eps, out, residual_out)
PyObject* norm_common(PyObject* const* a, Py_ssize_t n) {
    if (n != 10 || !g_ops.norm) return not_here();
    const at::Tensor* x = plain(a[0]);
    float scale, offset, eps;
    if (!x || x->dim() != 2 || x->size(0) < 1 || !dtype_code(*x) || !as_float(a[5], scale) || !as_float(a[6], offset) ||
        !as_float(a[7], eps) || a[2] == Py_None)
        return not_here();
    const int64_t M = x->size(0), N = x->size(1);
    const int dev = x->get_device();
    const auto type = x->scalar_type();
    const at::Tensor* in[5] = {};            // residual, weight, post_weight, out, residual_out
    const int at_arg[5] = {1, 2, 3, 8, 9};
    for (int i = 0; i < 5; ++i) {
        PyObject* o = a[at_arg[i]];
        if (o == Py_None) continue;
        in[i] = plain(o);
        const int64_t vec[1] = {N}, mat[2] = {M, N};
        if (!is(in[i], type, dev, i == 1 || i == 2 ? at::IntArrayRef(vec) : at::IntArrayRef(mat))) return not_here();
    }
    const at::Tensor* gate = nullptr;
    int64_t gate_stride = 0;
    if (a[4] != Py_None) {
        gate = on_gpu(a[4]);
        if (!gate || gate->scalar_type() != type || gate->get_device() != dev || gate->dim() > 2 || gate->dim() < 1 ||
            gate->size(-1) != N || (gate->dim() == 2 && gate->size(0) != M) || (N > 1 && gate->stride(-1) != 1))
            return not_here();
        gate_stride = gate->dim() == 2 && M > 1 ? gate->stride(0) : 0;
    }
    const bool keep = !in[0] && !in[2] && !gate && scale == 1.0f && !in[4];
    void* stream;
    if (!tf_binding::stream_of(g_ops_stream, dev, stream)) return PyErr_Occurred() ? nullptr : not_here();
    at::Tensor y, r;
    if (!in[3]) y = at::empty({M, N}, x->options().requires_grad(false));
    if (!in[4] && !keep) r = at::empty({M, N}, x->options().requires_grad(false));
    void* yp = in[3] ? in[3]->data_ptr() : y.data_ptr();
    void* rp = in[4] ? in[4]->data_ptr() : keep ? nullptr : r.data_ptr();
    int rc;
    const void *xp = ptr(x), *res = ptr(in[0]), *w = ptr(in[1]), *post = ptr(in[2]), *gp = ptr(gate);
    const int code = dtype_code(*x);
    Py_BEGIN_ALLOW_THREADS;
    rc = g_ops.norm(code, xp, res, post, gp, gate_stride, scale, w, offset, eps, M, N, rp, yp, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    const Held yo{in[3] ? Py_NewRef(a[8]) : THPVariable_Wrap(std::move(y))};
    const Held ro{keep ? Py_NewRef(a[0]) : in[4] ? Py_NewRef(a[9]) : THPVariable_Wrap(std::move(r))};
    return yo.o && ro.o ? PyTuple_Pack(2, yo.o, ro.o) : nullptr;
}

// append(cache, table, cu, starts, k, v, cos, sin, q, keys, q_out, k_out)
PyObject* append_common(PyObject* const* a, Py_ssize_t n) {
    if (n != 12 || !g_ops.append) return not_here();
    const at::Tensor *cu = plain(a[2]), *starts = plain(a[3]), *k = on_gpu(a[4]), *v = on_gpu(a[5]);
    if (!cu || !starts || !k || !v || starts->dim() != 1 || starts->size(0) < 1) return not_here();
    const int64_t B = starts->size(0);
    Cache cache;
    if (!cache.read(a[0], on_gpu(a[1]), B)) return not_here();
    const int dev = cache.dev;
    const int64_t k_stride = heads_stride(*k), v_stride = heads_stride(*v);
    if (k_stride < 0 || v_stride < 0) return not_here();
    const int64_t T = k->size(0), H = cache.c.kv_heads, D = cache.c.head_dim;
    const int64_t kv[3] = {T, H, D}, one[1] = {B}, more[1] = {B + 1};
    for (const at::Tensor* t : {k, v})
        if (t->scalar_type() != cache.type || t->get_device() != dev || t->sizes() != at::IntArrayRef(kv))
            return not_here();
    if (!is(cu, at::kInt, dev, more) || !is(starts, at::kInt, dev, one)) return not_here();
    const at::Tensor *cos = nullptr, *sin = nullptr;
    int64_t positions = 0;
    if (a[6] != Py_None || a[7] != Py_None) {
        cos = plain(a[6]);
        sin = plain(a[7]);
        if (!cos || !sin || cos->dim() != 2) return not_here();
        positions = cos->size(0);
        const int64_t table[2] = {positions, D / 2};
        if (!is(cos, at::kFloat, dev, table) || !is(sin, at::kFloat, dev, table)) return not_here();
    }
    const at::Tensor* q = nullptr;
    int64_t q_stride = 0, Hq = 0;
    if (a[8] != Py_None) {
        q = on_gpu(a[8]);
        if (!q || q->scalar_type() != cache.type || q->get_device() != dev) return not_here();
        q_stride = heads_stride(*q);
        if (q_stride < 0 || q->size(0) != T || q->size(2) != D) return not_here();
        Hq = q->size(1);
    } else if (a[10] != Py_None) {
        return not_here();
    }
    const int64_t qs[3] = {T, Hq, D};
    const at::Tensor *q_out = nullptr, *k_out = nullptr;
    if (a[10] != Py_None && !is(q_out = plain(a[10]), cache.type, dev, qs)) return not_here();
    if (a[11] != Py_None && !is(k_out = plain(a[11]), cache.type, dev, kv)) return not_here();
    const int keys = a[9] == Py_True ? 1 : a[9] == Py_False ? 0 : -1;
    if (keys < 0) return not_here();
    void* stream;
    if (!tf_binding::stream_of(g_ops_stream, dev, stream)) return PyErr_Occurred() ? nullptr : not_here();
    at::Tensor made_q, made_k;
    if (q && !q_out) {
        made_q = at::empty(qs, k->options().requires_grad(false));
        q_out = &made_q;
    }
    const bool make_k = keys && !k_out;
    if (make_k) {
        made_k = at::empty(kv, k->options().requires_grad(false));
        k_out = &made_k;
    }
    const void *qp = ptr(q), *kp = ptr(k), *vp = ptr(v);
    void *qo = const_cast<void*>(ptr(q_out)), *ko = const_cast<void*>(ptr(k_out));
    const float *cp = static_cast<const float*>(ptr(cos)), *sp = static_cast<const float*>(ptr(sin));
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = g_ops.append(&cache.c, qp, q_stride, kp, k_stride, vp, v_stride, cp, sp, positions, ints(cu), ints(starts), B,
                      T, (int)Hq, qo, ko, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    const Held q_o{made_q.defined() ? THPVariable_Wrap(std::move(made_q)) : Py_NewRef(a[10])};
    const Held k_o{make_k ? THPVariable_Wrap(std::move(made_k)) : Py_NewRef(a[11])};
    return q_o.o && k_o.o ? PyTuple_Pack(2, q_o.o, k_o.o) : nullptr;
}

// read(cache, table, cu, starts, tokens, k_out, v_out)
PyObject* read_common(PyObject* const* a, Py_ssize_t n) {
    if (n != 7 || !g_ops.read || !PyLong_CheckExact(a[4])) return not_here();
    const at::Tensor *cu = plain(a[2]), *starts = plain(a[3]);
    int over = 0;
    const int64_t T = PyLong_AsLongLongAndOverflow(a[4], &over);
    if (over || T < 1 || T > TF_MAX_M || !cu || !starts || starts->dim() != 1 || starts->size(0) < 1) return not_here();
    const int64_t B = starts->size(0);
    Cache cache;
    if (!cache.read(a[0], on_gpu(a[1]), B)) return not_here();
    const int dev = cache.dev;
    const int64_t one[1] = {B}, more[1] = {B + 1}, kv[3] = {T, cache.c.kv_heads, cache.c.head_dim};
    if (!is(cu, at::kInt, dev, more) || !is(starts, at::kInt, dev, one)) return not_here();
    const at::Tensor* out[2] = {};
    for (int i = 0; i < 2; ++i)
        if (a[5 + i] != Py_None && !is(out[i] = plain(a[5 + i]), cache.type, dev, kv)) return not_here();
    void* stream;
    if (!tf_binding::stream_of(g_ops_stream, dev, stream)) return PyErr_Occurred() ? nullptr : not_here();
    at::Tensor made[2];
    for (int i = 0; i < 2; ++i)
        if (!out[i])
            made[i] = at::empty(kv, at::TensorOptions().dtype(cache.type).device(at::Device(at::kCUDA, (int8_t)dev)));
    void *kp = out[0] ? out[0]->data_ptr() : made[0].data_ptr(), *vp = out[1] ? out[1]->data_ptr() : made[1].data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = g_ops.read(&cache.c, ints(cu), ints(starts), B, T, kp, vp, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    const Held k{out[0] ? Py_NewRef(a[5]) : THPVariable_Wrap(std::move(made[0]))};
    const Held v{out[1] ? Py_NewRef(a[6]) : THPVariable_Wrap(std::move(made[1]))};
    return k.o && v.o ? PyTuple_Pack(2, k.o, v.o) : nullptr;
}

// decode(q, cache, table, lens, scale, out, workspace)
PyObject* decode_common(PyObject* const* a, Py_ssize_t n) {
    if (n != 7 || !g_ops.decode) return not_here();
    const at::Tensor *q = on_gpu(a[0]), *lens = plain(a[3]);
    if (!q || !lens || (q->dim() != 3 && q->dim() != 4) || q->numel() == 0) return not_here();
    const bool many = q->dim() == 4;
    const int64_t B = q->size(0), Q = many ? q->size(1) : 1, H = q->size(-2), D = q->size(-1);
    Cache cache;
    if (!cache.read(a[1], on_gpu(a[2]), B)) return not_here();
    const int dev = cache.dev;
    const int64_t one[1] = {B};
    if (q->scalar_type() != cache.type || q->get_device() != dev || D != cache.c.head_dim || q->stride(-1) != 1 ||
        (H > 1 && q->stride(-2) != D) || !is(lens, at::kInt, dev, one) || Q > TF_KV4_MAX_Q || H > TF_MAX_HEADS)
        return not_here();
    if (Q > 1 && B > 1 && q->stride(0) != Q * q->stride(1)) return not_here();
    const int64_t stride = Q > 1 ? q->stride(1) : B > 1 ? q->stride(0) : H * D;
    float scale = 1.0f / std::sqrt((float)D);
    if (a[4] != Py_None && !as_float(a[4], scale)) return not_here();
    const at::Tensor* out = nullptr;
    if (a[5] != Py_None && !is(out = plain(a[5]), cache.type, dev, q->sizes())) return not_here();
    const int64_t need = g_ops.decode_bytes(B, (int)Q, (int)H, cache.c.kv_heads, (int)D);
    if (need < 0) return not_here();
    Held held;
    void *ws, *stream;
    size_t ws_bytes;
    if (a[6] == Py_False) return not_here();
    if (!tf_binding::stream_of(g_ops_stream, dev, stream)) return PyErr_Occurred() ? nullptr : not_here();
    if (!workspace_of(a[6], g_decode_ws, a[0], dev, stream, need, held, ws, ws_bytes))
        return PyErr_Occurred() ? nullptr : not_here();
    at::Tensor made;
    if (!out) {
        made = at::empty(q->sizes(), q->options().requires_grad(false));
        out = &made;
    }
    const void* qp = q->data_ptr();
    void* op = out->data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = g_ops.decode(&cache.c, qp, stride, ints(lens), B, (int)Q, (int)H, scale, op, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    return a[5] == Py_None ? THPVariable_Wrap(std::move(made)) : Py_NewRef(a[5]);
}

// prompt(q, k, v, cu_q, cu_k, scale, causal, out, workspace)
PyObject* prompt_common(PyObject* const* a, Py_ssize_t n) {
    if (n != 9 || !g_ops.prompt || !PyBool_Check(a[6])) return not_here();
    const at::Tensor *q = on_gpu(a[0]), *k = on_gpu(a[1]), *v = on_gpu(a[2]), *cu_q = plain(a[3]),
                     *cu_k = plain(a[4] == Py_None ? a[3] : a[4]);
    if (!q || !k || !v || !cu_q || !cu_k || !dtype_code(*q) || cu_q->dim() != 1 || cu_q->size(0) < 2) return not_here();
    const int64_t qs = heads_stride(*q), ks = heads_stride(*k), vs = heads_stride(*v);
    if (qs < 0 || ks < 0 || vs < 0) return not_here();
    const int dev = q->get_device();
    const int64_t B = cu_q->size(0) - 1, T = q->size(0), H = q->size(1), D = q->size(2), Tk = k->size(0);
    const int64_t more[1] = {B + 1}, kv[3] = {Tk, k->size(1), D};
    for (const at::Tensor* t : {k, v})
        if (t->scalar_type() != q->scalar_type() || t->get_device() != dev || t->sizes() != at::IntArrayRef(kv))
            return not_here();
    if (!is(cu_q, at::kInt, dev, more) || !is(cu_k, at::kInt, dev, more) || H > TF_MAX_HEADS || kv[1] > TF_MAX_HEADS)
        return not_here();
    float scale = 1.0f / std::sqrt((float)D);
    if (a[5] != Py_None && !as_float(a[5], scale)) return not_here();
    const at::Tensor* out = nullptr;
    if (a[7] != Py_None && !is(out = plain(a[7]), q->scalar_type(), dev, q->sizes())) return not_here();
    const int64_t need = g_ops.prompt_bytes(B, T, Tk, (int)H, (int)kv[1], (int)D);
    if (need < 0) return not_here();
    Held held;
    void *ws, *stream;
    size_t ws_bytes;
    if (!tf_binding::stream_of(g_ops_stream, dev, stream)) return PyErr_Occurred() ? nullptr : not_here();
    if (!workspace_of(a[8], g_prompt_ws, a[0], dev, stream, need, held, ws, ws_bytes))
        return PyErr_Occurred() ? nullptr : not_here();
    at::Tensor made;
    if (!out) {
        made = at::empty({T, H, D}, q->options().requires_grad(false));
        out = &made;
    }
    const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr();
    void* op = out->data_ptr();
    const int code = dtype_code(*q), causal = a[6] == Py_True;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = g_ops.prompt(code, qp, qs, kp, ks, vp, vs, ints(cu_q), ints(cu_k), B, T, Tk, (int)H, (int)kv[1], (int)D, scale,
                      causal, op, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    return a[7] == Py_None ? THPVariable_Wrap(std::move(made)) : Py_NewRef(a[7]);
}

// No exception leaves a C entry (any access to a tensor may throw), and none
// follows the launch but the wrapping of outputs: the general path meets the same
// condition and raises it as torch does.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        return F(a, n);
    } catch (...) {
        return PyErr_Occurred() ? nullptr : not_here();
    }
}
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyCFunction fast() {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<F>));
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, "Hand over the library's functions."},
    {"norm", fast<norm_common>(), METH_FASTCALL, "add_rms_norm, or NotImplemented."},
    {"append", fast<append_common>(), METH_FASTCALL, "kv4_append, or NotImplemented."},
    {"read", fast<read_common>(), METH_FASTCALL, "kv4_read, or NotImplemented."},
    {"decode", fast<decode_common>(), METH_FASTCALL, "kv4_attention, or NotImplemented."},
    {"prompt", fast<prompt_common>(), METH_FASTCALL, "prompt_attention, or NotImplemented."},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tf_binding_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tf_binding_ops() {
    g_name_data = PyUnicode_InternFromString("data");
    g_name_sizes = PyUnicode_InternFromString("_sizes");
    g_name_device = PyUnicode_InternFromString("device");
    if (!g_name_data || !g_name_sizes || !g_name_device) return nullptr;
    return PyModule_Create(&module);
}
