// The calls of the 8-bit linear layers and the layers made of experts of tilefuse.py
// in native code, as tf_binding_ops.cpp has those of the norm, cache and attention:
// only calls in the common form are taken; anything else, and every refusal, returns
// NotImplemented, and the general path in tilefuse.py runs it or raises.
// Measured on MI355X, us in a loop, through ctypes -> here: one token's codes and
// product (two calls, one weight of 4096 x 4096) 19.7 -> 8.5, the choice of experts for
// 64 tokens 18.9 -> 10.1.
#include <ATen/ops/empty.h>
#include <Python.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <initializer_list>

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
bool is(const at::Tensor* t, at::ScalarType type, int dev, at::IntArrayRef shape) {
    return t && t->scalar_type() == type && t->get_device() == dev && t->is_contiguous() && t->sizes() == shape;
}

struct Fns {
    decltype(&tf_quantize_rows) quantize;
    decltype(&tf_w8a8_packed_bytes) packed_bytes;
    decltype(&tf_w8a8_workspace_bytes) workspace_bytes;
    decltype(&tf_w8a8_gemm) gemm;
    decltype(&tf_route_experts) route;
    decltype(&tf_w8a8_expert_gemm) expert_gemm;
    decltype(&tf_combine_experts) combine;
    tf_binding::CaptureFn capture;
} g_fns;
PyObject *g_stream, *g_workspaces, *g_make_workspace, *g_name_device;

// bind((addresses in the order of Fns), current stream function, workspaces of
//          gemm, function (device, bytes) that makes one)
PyObject* bind(PyObject*, PyObject* args) {
    PyObject *fns, *stream, *cached, *make;
    if (!PyArg_ParseTuple(args, "O!OO!O", &PyTuple_Type, &fns, &stream, &PyDict_Type, &cached, &make)) return nullptr;
    unsigned long long at[8];
    if (PyTuple_GET_SIZE(fns) != 8) {
        PyErr_SetString(PyExc_ValueError, "bind needs eight functions");
        return nullptr;
    }
    for (int i = 0; i < 8; ++i) {
        at[i] = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(fns, i));
        if (PyErr_Occurred()) return nullptr;
    }
    g_fns = {reinterpret_cast<decltype(Fns::quantize)>(at[0]),
             reinterpret_cast<decltype(Fns::packed_bytes)>(at[1]),
             reinterpret_cast<decltype(Fns::workspace_bytes)>(at[2]),
             reinterpret_cast<decltype(Fns::gemm)>(at[3]),
             reinterpret_cast<decltype(Fns::route)>(at[4]),
             reinterpret_cast<decltype(Fns::expert_gemm)>(at[5]),
             reinterpret_cast<decltype(Fns::combine)>(at[6]),
             reinterpret_cast<tf_binding::CaptureFn>(at[7])};
    Py_XSETREF(g_stream, Py_NewRef(stream));
    Py_XSETREF(g_workspaces, Py_NewRef(cached));
    Py_XSETREF(g_make_workspace, Py_NewRef(make));
    Py_RETURN_NONE;
}

int code16(at::ScalarType t) { return t == at::kHalf ? TF_F16 : t == at::kBFloat16 ? TF_BF16 : 0; }
// A Python integer within what the calls count in.
bool as_int(PyObject* o, int64_t& v) {
    int over = 0;
    if (!PyLong_CheckExact(o)) return false;
    v = PyLong_AsLongLongAndOverflow(o, &over);
    return !over && v > 0 && v <= INT32_MAX;
}
// The type of a product's output: that of `out`, the one named, or fp16.
bool output_type(PyObject* dtype, const at::Tensor* out, at::ScalarType& type) {
    if (dtype == Py_None) {
        type = out ? out->scalar_type() : at::kHalf;
    } else {
        if (!THPDtype_Check(dtype)) return false;
        type = reinterpret_cast<THPDtype*>(dtype)->scalar_type;
        if (out && out->scalar_type() != type) return false;
    }
    return code16(type) != 0;
}
at::Tensor make(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) {
    return at::empty(shape, like.options().dtype(type).requires_grad(false));
}

// quantize(x, gated, codes, scales)
PyObject* quantize_common(PyObject* const* a, Py_ssize_t n) {
    if (n != 4 || !g_fns.quantize || (a[1] != Py_True && a[1] != Py_False)) return not_here();
    const at::Tensor* x = on_gpu(a[0]);
    const int gated = a[1] == Py_True;
    if (!x || x->dim() != 2 || x->size(0) < 1 || x->size(1) < 2 || x->stride(1) != 1 || !code16(x->scalar_type()) ||
        (gated && x->size(1) % 2 != 0))
        return not_here();
    const int64_t M = x->size(0), N = x->size(1) / (gated ? 2 : 1), mat[2] = {M, N}, vec[1] = {M};
    const int dev = x->get_device();
    const at::Tensor *codes = nullptr, *scales = nullptr;
    if (a[2] != Py_None && !is(codes = plain(a[2]), at::kChar, dev, mat)) return not_here();
    if (a[3] != Py_None && !is(scales = plain(a[3]), at::kFloat, dev, vec)) return not_here();
    void* stream;
    if (!tf_binding::stream_of(g_stream, dev, stream)) return PyErr_Occurred() ? nullptr : not_here();
    at::Tensor made_codes, made_scales;
    if (!codes) made_codes = make(mat, at::kChar, *x);
    if (!scales) made_scales = make(vec, at::kFloat, *x);
    int8_t* cp = static_cast<int8_t*>(codes ? codes->data_ptr() : made_codes.data_ptr());
    float* sp = static_cast<float*>(scales ? scales->data_ptr() : made_scales.data_ptr());
    const void* xp = x->data_ptr();
    const int64_t stride = M > 1 ? x->stride(0) : x->size(1);
    const int code = code16(x->scalar_type());
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = g_fns.quantize(code, xp, stride, M, N, gated, cp, sp, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    const Held c{codes ? Py_NewRef(a[2]) : THPVariable_Wrap(std::move(made_codes))};
    const Held s{scales ? Py_NewRef(a[3]) : THPVariable_Wrap(std::move(made_scales))};
    return c.o && s.o ? PyTuple_Pack(2, c.o, s.o) : nullptr;
}

// The operands that both products have: codes, scales, packed, K, N.
struct Operands {
    const at::Tensor *codes, *scales, *packed;
    int64_t M, K, N;
    int dev;
    bool read(PyObject* const* a, int64_t weights) {
        codes = plain(a[0]);
        scales = plain(a[1]);
        packed = plain(a[2]);
        if (!codes || !scales || !packed || !as_int(a[3], K) || !as_int(a[4], N) || codes->dim() != 2 ||
            codes->scalar_type() != at::kChar || codes->size(1) != K || codes->size(0) < 1)
            return false;
        M = codes->size(0);
        dev = codes->get_device();
        const int64_t vec[1] = {M}, need = g_fns.packed_bytes(K, N);
        return need > 0 && is(scales, at::kFloat, dev, vec) && packed->get_device() == dev &&
               (int64_t)packed->nbytes() / weights >= need;
    }
};

// gemm(codes, scales, packed, K, N, dtype, out, workspace)
PyObject* gemm_common(PyObject* const* a, Py_ssize_t n) {
    Operands op;
    if (n != 8 || !g_fns.gemm || !op.read(a, 1)) return not_here();
    const at::Tensor* out = a[6] == Py_None ? nullptr : plain(a[6]);
    at::ScalarType type;
    if ((a[6] != Py_None && !out) || !output_type(a[5], out, type)) return not_here();
    const int64_t mat[2] = {op.M, op.N};
    if (out && !is(out, type, op.dev, mat)) return not_here();
    void* stream;
    if (!tf_binding::stream_of(g_stream, op.dev, stream)) return PyErr_Occurred() ? nullptr : not_here();
    // the workspace: False none, None the stream's cached one, or the caller's
    Held held;
    const at::Tensor* ws = nullptr;
    if (a[7] == Py_None) {
        const int64_t need = g_fns.workspace_bytes(op.M, op.K, op.N);
        if (need < 0) return not_here();
        if (need > 0) {
            if (!tf_binding::find_workspace(g_workspaces, g_fns.capture, op.dev, stream, held))
                return PyErr_Occurred() ? nullptr : not_here();
            ws = held.o ? plain(held.o) : nullptr;
            if (!ws || (int64_t)ws->nbytes() < need) {
                const Held device{PyObject_GetAttr(a[0], g_name_device)};
                if (!device.o) return nullptr;
                Py_XSETREF(held.o, PyObject_CallFunction(g_make_workspace, "OL", device.o, (long long)need));
                if (!held.o) return nullptr;
                if (!(ws = plain(held.o))) return not_here();
            }
        }
    } else if (a[7] != Py_False) {
        if (!(ws = plain(a[7])) || ws->get_device() != op.dev) return not_here();
    }
    void* wsp = ws ? ws->data_ptr() : nullptr;
    const size_t ws_bytes = ws ? ws->nbytes() : 0;
    at::Tensor made;
    if (!out) made = make(mat, type, *op.codes);
    void* c = out ? out->data_ptr() : made.data_ptr();
    const int8_t* q = static_cast<const int8_t*>(op.codes->data_ptr());
    const float* s = static_cast<const float*>(op.scales->data_ptr());
    const void* w = op.packed->data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = g_fns.gemm(code16(type), q, s, w, c, op.M, op.K, op.N, wsp, ws_bytes, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    return out ? Py_NewRef(a[6]) : THPVariable_Wrap(std::move(made));
}

// expert_gemm(codes, scales, packed, K, N, offsets, rows, dtype, out)
PyObject* expert_gemm_common(PyObject* const* a, Py_ssize_t n) {
    if (n != 9 || !g_fns.expert_gemm) return not_here();
    const at::Tensor* offsets = plain(a[5]);
    if (!offsets || offsets->scalar_type() != at::kInt || offsets->dim() != 1 || offsets->size(0) < 2) return not_here();
    const int64_t E = offsets->size(0) - 1;
    Operands op;
    if (!op.read(a, E) || offsets->get_device() != op.dev) return not_here();
    const at::Tensor* rows = nullptr;
    int64_t slots = op.M;
    if (a[6] != Py_None) {
        rows = plain(a[6]);
        if (!rows || rows->dim() != 1 || rows->size(0) < 1) return not_here();
        slots = rows->size(0);
        const int64_t vec[1] = {slots};
        if (!is(rows, at::kInt, op.dev, vec)) return not_here();
    }
    const at::Tensor* out = a[8] == Py_None ? nullptr : plain(a[8]);
    at::ScalarType type;
    if ((a[8] != Py_None && !out) || !output_type(a[7], out, type)) return not_here();
    const int64_t mat[2] = {slots, op.N};
    if (out && !is(out, type, op.dev, mat)) return not_here();
    void* stream;
    if (!tf_binding::stream_of(g_stream, op.dev, stream)) return PyErr_Occurred() ? nullptr : not_here();
    at::Tensor made;
    if (!out) made = make(mat, type, *op.codes);
    void* c = out ? out->data_ptr() : made.data_ptr();
    const int8_t* q = static_cast<const int8_t*>(op.codes->data_ptr());
    const float* s = static_cast<const float*>(op.scales->data_ptr());
    const void* w = op.packed->data_ptr();
    const int32_t *of = static_cast<const int32_t*>(offsets->data_ptr()),
                  *rp = rows ? static_cast<const int32_t*>(rows->data_ptr()) : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = g_fns.expert_gemm(code16(type), q, s, op.M, w, of, rp, c, slots, op.K, op.N, E, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    return out ? Py_NewRef(a[8]) : THPVariable_Wrap(std::move(made));
}

// route(logits, top_k, bias, scoring, groups, top_groups, group_score, renormalize, scale):
// scoring and group_score as the library's numbers
PyObject* route_common(PyObject* const* a, Py_ssize_t n) {
    if (n != 9 || !g_fns.route) return not_here();
    const at::Tensor* x = on_gpu(a[0]);
    int64_t k, groups, top_groups;
    if (!x || x->dim() != 2 || x->size(0) < 1 || x->size(1) < 1 || !as_int(a[1], k) || !as_int(a[4], groups) ||
        !as_int(a[5], top_groups) || !PyLong_CheckExact(a[3]) || !PyLong_CheckExact(a[6]) || !PyFloat_CheckExact(a[8]) ||
        (a[7] != Py_True && a[7] != Py_False) || k > TF_MAX_TOP_K)
        return not_here();
    const int64_t T = x->size(0), E = x->size(1), vec[1] = {E};
    const int dev = x->get_device();
    const int code = x->scalar_type() == at::kFloat ? TF_F32 : code16(x->scalar_type());
    if (!code || (E > 1 && x->stride(1) != 1) || T > TF_MAX_M || E > TF_MAX_EXPERTS) return not_here();
    const at::Tensor* bias = nullptr;
    if (a[2] != Py_None && !is(bias = plain(a[2]), at::kFloat, dev, vec)) return not_here();
    const int scoring = (int)PyLong_AsLong(a[3]), group_score = (int)PyLong_AsLong(a[6]);
    const float scale = (float)PyFloat_AS_DOUBLE(a[8]);
    void* stream;
    if (!tf_binding::stream_of(g_stream, dev, stream)) return PyErr_Occurred() ? nullptr : not_here();
    const int64_t mat[2] = {T, k}, ends[1] = {E + 1}, slots[1] = {T * k};
    at::Tensor made[5] = {make(mat, at::kFloat, *x), make(mat, at::kInt, *x), make(ends, at::kInt, *x),
                          make(slots, at::kInt, *x), make(mat, at::kInt, *x)};
    const void* xp = x->data_ptr();
    const float* bp = bias ? static_cast<const float*>(bias->data_ptr()) : nullptr;
    float* wp = static_cast<float*>(made[0].data_ptr());
    int32_t* ip[4];
    for (int i = 0; i < 4; ++i) ip[i] = static_cast<int32_t*>(made[i + 1].data_ptr());
    const int64_t stride = T > 1 ? x->stride(0) : E;
    const int renormalize = a[7] == Py_True;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = g_fns.route(code, xp, stride, bp, T, (int)E, (int)k, scoring, (int)groups, (int)top_groups, group_score,
                     renormalize, scale, wp, ip[0], ip[1], ip[2], ip[3], stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    const Held t{PyTuple_New(5)};
    if (!t.o) return nullptr;
    for (int i = 0; i < 5; ++i) {
        PyObject* o = THPVariable_Wrap(std::move(made[i]));
        if (!o) return nullptr;
        PyTuple_SET_ITEM(t.o, i, o);
    }
    return Py_NewRef(t.o);
}

// combine(y, weights, places, add, out)
PyObject* combine_common(PyObject* const* a, Py_ssize_t n) {
    if (n != 5 || !g_fns.combine) return not_here();
    const at::Tensor *y = plain(a[0]), *w = plain(a[1]), *places = plain(a[2]);
    if (!y || !w || !places || y->dim() != 2 || places->dim() != 2 || !code16(y->scalar_type()) || y->size(0) < 1 ||
        places->size(0) < 1 || places->size(1) < 1 || places->size(1) > TF_MAX_TOP_K)
        return not_here();
    const int64_t T = places->size(0), k = places->size(1), N = y->size(1), mat[2] = {T, k}, rows[2] = {T, N};
    const int dev = y->get_device();
    if (!is(places, at::kInt, dev, mat) || !is(w, at::kFloat, dev, mat)) return not_here();
    const at::Tensor *add = nullptr, *out = nullptr;
    if (a[3] != Py_None && !is(add = plain(a[3]), y->scalar_type(), dev, rows)) return not_here();
    if (a[4] != Py_None && !is(out = plain(a[4]), y->scalar_type(), dev, rows)) return not_here();
    void* stream;
    if (!tf_binding::stream_of(g_stream, dev, stream)) return PyErr_Occurred() ? nullptr : not_here();
    at::Tensor made;
    if (!out) made = make(rows, y->scalar_type(), *y);
    void* op = out ? out->data_ptr() : made.data_ptr();
    const void *yp = y->data_ptr(), *ap = add ? add->data_ptr() : nullptr;
    const float* wp = static_cast<const float*>(w->data_ptr());
    const int32_t* pp = static_cast<const int32_t*>(places->data_ptr());
    const int code = code16(y->scalar_type());
    const int64_t slots = y->size(0);
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = g_fns.combine(code, yp, slots, wp, pp, ap, T, (int)k, N, op, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    return out ? Py_NewRef(a[4]) : THPVariable_Wrap(std::move(made));
}

// No exception leaves a C entry: what throws here (memory that is short, say) throws
// again in the general path, as torch raises it.
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
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<F>));
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, "Hand over the library's functions."},
    {"quantize", fast<quantize_common>(), METH_FASTCALL, "quantize_rows, or NotImplemented."},
    {"gemm", fast<gemm_common>(), METH_FASTCALL, "w8a8_gemm, or NotImplemented."},
    {"route", fast<route_common>(), METH_FASTCALL, "route_experts, or NotImplemented."},
    {"expert_gemm", fast<expert_gemm_common>(), METH_FASTCALL, "w8a8_expert_gemm, or NotImplemented."},
    {"combine", fast<combine_common>(), METH_FASTCALL, "combine_experts, or NotImplemented."},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tf_binding_experts", nullptr, -1, methods, nullptr, nullptr, nullptr,
                      nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tf_binding_experts() {
    g_name_device = PyUnicode_InternFromString("device");
    return g_name_device ? PyModule_Create(&module) : nullptr;
}
