// Python module _train: the operators behind the decode (include/pcr.h) on PyTorch tensors.  Checks of arguments, allocation of results
// and the call of the C entry point, for train.py: a call made of ctypes and Python checks takes 15 to 25 us of the host's time, which is three to five
// times what a small call takes the GPU, and 5 to 8 us here.
// Every function takes its arguments by position and works on PyTorch's current stream; a wrong argument raises ValueError, an error of the
// library PcrError (set_up).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include <cmath>
#include <cstdarg>
#include <exception>

#include "../../include/pcr.h"

namespace {

PyObject* g_error = nullptr;                                   // PcrError
PyObject* g_current_stream = nullptr;                          // device index -> the current stream's hipStream_t as an integer

struct Refused {};                                             // a Python exception is set

[[noreturn]] void refuse(const char* format, ...) {
    va_list v;
    va_start(v, format);
    PyErr_FormatV(PyExc_ValueError, format, v);
    va_end(v);
    throw Refused();
}
void need(bool ok, const char* what) {
    if (!ok) refuse("%s", what);
}
void need(bool ok, const char* name, const char* what) {
    if (!ok) refuse("%s: %s", name, what);
}
void check(int rc, const char* what) {
    if (rc == PCR_OK) return;
    PyObject* e = PyObject_CallFunction(g_error, "is", rc, what);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw Refused();
}

const at::Tensor* maybe_tensor(PyObject* o, const char* name) {
    if (o == Py_None) return nullptr;
    need(THPVariable_Check(o), name, "a tensor is wanted");
    const at::Tensor& t = THPVariable_Unpack(o);
    need(!t._fw_grad(0).defined(), name, "has a derivative of forward mode, which would be lost");
    return &t;
}
const at::Tensor& tensor(PyObject* o, const char* name) {
    const at::Tensor* t = maybe_tensor(o, name);
    need(t != nullptr, name, "a tensor is wanted");
    return *t;
}
double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused();
    return v;
}
int64_t integer(PyObject* o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    return v;
}
int small(PyObject* o, const char* name) {
    const int64_t v = integer(o);
    need(v >= INT32_MIN && v <= INT32_MAX, name, "out of range");
    return (int)v;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refused();
    return v != 0;
}

int type_of(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case at::kFloat: return PCR_FLOAT;
        case at::kHalf: return PCR_HALF;
        case at::kBFloat16: return PCR_BFLOAT;
        default: return -1;
    }
}
void on(const at::Tensor& t, const at::Tensor& other, const char* name) { need(t.is_cuda() && t.device() == other.device(), name, "a tensor on the GPU of the others is wanted"); }

// A tensor of the caller's that a call writes: as with PyTorch's operators in place, not a leaf that requires a gradient, which would lose its place in the graph ...
void check_written(const at::Tensor& t, const char* name) {
    if (!t.requires_grad() || !c10::GradMode::is_enabled()) return;
    need(!(t.is_view() ? t._base() : t).is_leaf(), name, "a leaf that requires a gradient is not written over (under torch.no_grad() it is)");
}
// ... and behind the call of a version of its own, so that what was kept of the old one for a gradient is not taken for it.
void written(PyObject* o) {
    if (o == Py_None) return;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// PyTorch's current stream of the tensor's device.
void* stream_of(const at::Tensor& t) {
    PyObject* index = PyLong_FromLong(t.device().index());
    PyObject* s = index ? PyObject_CallOneArg(g_current_stream, index) : nullptr;
    Py_XDECREF(index);
    if (!s) throw Refused();
    void* p = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (!p && PyErr_Occurred()) throw Refused();
    return p;
}
int device_number(const at::Tensor& t) { return t.device().index(); }

PyObject* some(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* none() { Py_RETURN_NONE; }
// (first, second, ...), taking the references.
template <typename... P> PyObject* tuple(P... parts) {
    PyObject* all[] = {parts...};
    PyObject* t = PyTuple_New(sizeof...(parts));
    bool ok = t != nullptr;
    for (size_t i = 0; i < sizeof...(parts); i++) {
        ok = ok && all[i];
        if (t) PyTuple_SET_ITEM(t, i, all[i]);
        else Py_XDECREF(all[i]);
    }
    if (ok) return t;
    Py_XDECREF(t);
    throw Refused();
}

// Runs f (which gives a new reference) with everything that may be thrown turned into a Python exception.
template <typename F> PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, F f) {
    if (given != wanted) {
        PyErr_Format(PyExc_TypeError, "%zd arguments are wanted, %zd given", wanted, given);
        return nullptr;
    }
    if (torch::jit::tracer::isTracing()) {                     // (a trace would hold the results' allocation and not the kernel that fills them)
        PyErr_SetString(PyExc_RuntimeError, "the operators behind the decode cannot be traced");
        return nullptr;
    }
    try {
        return f();
    } catch (const Refused&) {
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// ---- patch rows ----

PyObject* patch_rows(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return guarded(given, 13, [&] {
        const at::Tensor& pixels = tensor(a[0], "pixels");
        need(pixels.is_cuda() && pixels.scalar_type() == at::kByte && pixels.is_contiguous(), "pixels", "a contiguous uint8 CUDA tensor is wanted");
        const at::Tensor &shapes = tensor(a[1], "shapes"), &offsets = tensor(a[2], "offsets"), &first = tensor(a[3], "first_rows");
        on(shapes, pixels, "shapes"); on(offsets, pixels, "offsets"); on(first, pixels, "first_rows");
        need(shapes.scalar_type() == at::kInt && shapes.dim() == 2 && shapes.size(1) == 2 && shapes.is_contiguous(), "shapes", "contiguous int32 [pictures, 2] is wanted");
        const int64_t n = shapes.size(0);
        need(offsets.scalar_type() == at::kLong && offsets.dim() == 1 && offsets.size(0) == n + 1 && offsets.is_contiguous(), "offsets", "contiguous int64 [pictures + 1] is wanted");
        need(first.scalar_type() == at::kLong && first.dim() == 1 && first.size(0) == n + 1 && first.is_contiguous(), "first_rows", "contiguous int64 [pictures + 1] is wanted");
        const int64_t rows = integer(a[4]);
        const int patch = small(a[5], "patch"), merge = small(a[8], "merge"), frames = small(a[9], "frames");
        PyObject *m = a[6], *s = a[7];
        need(PyTuple_Check(m) && PyTuple_Check(s) && PyTuple_GET_SIZE(m) == PyTuple_GET_SIZE(s) && (PyTuple_GET_SIZE(m) == 1 || PyTuple_GET_SIZE(m) == 3), "mean and inv_std",
             "one or three values each");
        const int C = (int)PyTuple_GET_SIZE(m);
        float mean[3], inv_std[3];
        for (int c = 0; c < C; c++) { mean[c] = (float)number(PyTuple_GET_ITEM(m, c)); inv_std[c] = (float)number(PyTuple_GET_ITEM(s, c)); }
        need(rows >= 0 && patch >= 1 && patch <= 4096 && merge >= 1 && frames >= 1, "rows, patch, merge, frames: out of range");
        const int64_t per = (int64_t)C * patch * patch;
        const int dtype = small(a[10], "dtype");
        const at::Tensor *given_out = maybe_tensor(a[11], "out"), *given_positions = maybe_tensor(a[12], "positions");
        need(given_out || (dtype >= 0 && dtype <= 2), "dtype", "float32, float16 or bfloat16 is wanted");
        if (given_out) {
            on(*given_out, pixels, "out");
            check_written(*given_out, "out");
            need(type_of(*given_out) >= 0 && given_out->is_contiguous() && given_out->numel() == rows * per, "out", "contiguous [rows, channels * patch * patch] is wanted");
        }
        if (given_positions) {
            on(*given_positions, pixels, "positions");
            need(given_positions->scalar_type() == at::kInt && given_positions->is_contiguous() && given_positions->dim() == 2 && given_positions->size(0) == 3 &&
                 given_positions->size(1) == rows, "positions", "contiguous int32 [3, rows] is wanted");
        }
        const at::Tensor out = given_out ? *given_out : at::empty({rows, per}, pixels.options().dtype(dtype == PCR_FLOAT ? at::kFloat : dtype == PCR_HALF ? at::kHalf : at::kBFloat16));
        const at::Tensor positions = given_positions ? *given_positions : at::empty({3, rows}, pixels.options().dtype(at::kInt));
        check(pcr_patch_rows(device_number(pixels), (const uint8_t*)pixels.data_ptr(), (size_t)pixels.numel(), (const int32_t*)shapes.data_ptr(), (const int64_t*)offsets.data_ptr(),
                             (const int64_t*)first.data_ptr(), n, rows, patch, merge, frames, C, mean, inv_std, type_of(out), out.data_ptr(), (int32_t*)positions.data_ptr(),
                             stream_of(pixels)), "pcr_patch_rows");
        written(a[11]);
        written(a[12]);
        return tuple(some(out), some(positions));
    });
}

// ---- positions in queries and keys ----

void check_side(const at::Tensor& t, const at::Tensor& x, const char* name) {
    on(t, x, name);
    need(t.scalar_type() == x.scalar_type() && t.sizes() == x.sizes() && (t.size(-1) == 1 || t.stride(-1) == 1), name,
         "the type and shape of its side is wanted, with each head's elements contiguous");
}
void check_into(const at::Tensor& t, const at::Tensor& x, const char* name) {
    check_side(t, x, name);
    check_written(t, name);
    for (int64_t i = 0; i < t.dim(); i++) need(t.stride(i) != 0 || t.size(i) < 2, name, "every element needs a place of its own");
}
void check_weight(const at::Tensor* w, const at::Tensor& x, const char* name) {
    if (!w) return;
    on(*w, x, name);
    need(w->dim() == 1 && w->size(0) == x.size(-1) && w->is_contiguous() && (w->scalar_type() == at::kFloat || w->scalar_type() == x.scalar_type()), name,
         "contiguous [dim] of float32 or the heads' type is wanted");
}

// What the two sides share: q, k (or nothing), the weights and the rotation.
struct Turn {
    const at::Tensor* x[2];
    const at::Tensor* w[2];
    pcr_heads side[2] = {};
    pcr_rotation rotation = {};
    int dtype, weight_dtype;

    Turn(PyObject* q, PyObject* k, PyObject* qw, PyObject* kw, PyObject* at_positions, PyObject* at_frequency, PyObject* at_axis, PyObject* adjacent) {
        const at::Tensor& Q = tensor(q, "q");
        x[0] = &Q; x[1] = maybe_tensor(k, "k");
        dtype = type_of(Q);
        need(Q.is_cuda() && dtype >= 0 && (Q.dim() == 3 || Q.dim() == 4), "q", "float32, float16 or bfloat16 [(batch,) tokens, heads, dim] on the GPU is wanted");
        need(Q.size(-1) == 1 || Q.stride(-1) == 1, "q", "each head's elements contiguous are wanted");
        const bool batched = Q.dim() == 4;
        if (x[1]) {
            const at::Tensor& K = *x[1];
            on(K, Q, "k");
            need(K.scalar_type() == Q.scalar_type() && K.dim() == Q.dim() && K.size(-1) == Q.size(-1) && K.size(0) == Q.size(0) && (!batched || K.size(1) == Q.size(1)), "k",
                 "the type, batch, tokens and dim of q are wanted");
            need(K.size(-1) == 1 || K.stride(-1) == 1, "k", "each head's elements contiguous are wanted");
        }
        w[0] = qw ? maybe_tensor(qw, "q_weight") : nullptr;
        w[1] = kw ? maybe_tensor(kw, "k_weight") : nullptr;
        check_weight(w[0], Q, "q_weight");
        check_weight(w[1], Q, "k_weight");
        need(x[1] || !w[1], "k_weight without k");
        need(!w[0] || !w[1] || w[0]->scalar_type() == w[1]->scalar_type(), "q_weight and k_weight: one type is wanted");
        weight_dtype = w[0] ? type_of(*w[0]) : w[1] ? type_of(*w[1]) : dtype;

        const at::Tensor &p = tensor(at_positions, "positions"), &f = tensor(at_frequency, "frequency"), &ax = tensor(at_axis, "axis");
        on(p, Q, "positions"); on(f, Q, "frequency"); on(ax, Q, "axis");
        pcr_rotation& R = rotation;
        R.batch = batched ? Q.size(0) : 1;
        R.tokens = Q.size(batched ? 1 : 0);
        need(p.scalar_type() == at::kInt || p.scalar_type() == at::kLong, "positions", "int32 or int64 is wanted");
        need(f.scalar_type() == at::kFloat && ax.scalar_type() == at::kInt && f.dim() == 1 && ax.dim() == 1 && f.size(0) == ax.size(0) && f.is_contiguous() && ax.is_contiguous(),
             "frequency and axis: contiguous float32 [pairs] and int32 [pairs] are wanted");
        need(2 * f.size(0) <= Q.size(-1), "frequency", "more pairs than half of a head");
        if (p.dim() == 2) {                                    // the same for every sequence
            need(p.size(1) == R.tokens, "positions", "[axes, tokens] or [axes, batch, tokens] is wanted");
            R.token_stride = p.stride(1);
        } else {
            need(p.dim() == 3 && p.size(1) == R.batch && p.size(2) == R.tokens, "positions", "[axes, tokens] or [axes, batch, tokens] is wanted");
            R.batch_stride = p.stride(1); R.token_stride = p.stride(2);
        }
        need(p.size(0) >= 1 && p.size(0) <= 4, "positions", "one to four axes are wanted");
        need(Q.size(-1) <= INT32_MAX, "q", "out of range");
        R.axis_stride = p.stride(0);
        R.position = p.data_ptr(); R.frequency = (const float*)f.data_ptr(); R.axis = (const int32_t*)ax.data_ptr();
        R.wide = p.scalar_type() == at::kLong; R.axes = (int32_t)p.size(0); R.dim = (int32_t)Q.size(-1); R.pairs = (int32_t)f.size(0); R.adjacent = truth(adjacent);
        for (int z = 0; z < 2; z++) {
            if (!x[z]) continue;
            pcr_heads& S = side[z];
            place(*x[z], S.in, S.in_batch, S.in_token, S.in_head);
            S.heads = x[z]->size(-2);
            if (w[z]) S.weight = w[z]->data_ptr();
        }
    }
    template <typename P> static void place(const at::Tensor& t, P*& p, int64_t& batch, int64_t& token, int64_t& head) {
        p = t.data_ptr();
        const int64_t d = t.dim();
        batch = d == 4 ? t.stride(0) : 0; token = t.stride(d - 3); head = t.stride(d - 2);
    }
    // Where side z's result goes: the tensor given, or a new one.
    at::Tensor into(int z, PyObject* given, const char* name) {
        const at::Tensor* t = maybe_tensor(given, name);
        if (!x[z]) return at::Tensor();
        if (t) check_into(*t, *x[z], name);
        at::Tensor out = t ? *t : at::empty(x[z]->sizes(), x[z]->options());
        pcr_heads& S = side[z];
        place(out, S.out, S.out_batch, S.out_token, S.out_head);
        return out;
    }
};

PyObject* rotate_axes(PyObject*, PyObject* const* a, Py_ssize_t given) {         // q k positions frequency axis adjacent inverse q_out k_out
    return guarded(given, 9, [&] {
        Turn T(a[0], a[1], nullptr, nullptr, a[2], a[3], a[4], a[5]);
        const at::Tensor q = T.into(0, a[7], "q_out"), k = T.into(1, a[8], "k_out");
        check(pcr_rotate_axes(device_number(q), &T.side[0], &T.side[1], &T.rotation, truth(a[6]), T.dtype, stream_of(q)), "pcr_rotate_axes");
        written(a[7]);
        written(a[8]);
        return tuple(some(q), T.x[1] ? some(k) : none());
    });
}

PyObject* norm_rotate(PyObject*, PyObject* const* a, Py_ssize_t given) {         // q k q_weight k_weight positions frequency axis eps adjacent q_out k_out
    return guarded(given, 11, [&] {
        Turn T(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[8]);
        const double eps = number(a[7]);
        need(eps >= 0, "eps", "not below 0");
        const at::Tensor q = T.into(0, a[9], "q_out"), k = T.into(1, a[10], "k_out");
        check(pcr_norm_rotate(device_number(q), &T.side[0], &T.side[1], &T.rotation, (float)eps, T.dtype, T.weight_dtype, stream_of(q)), "pcr_norm_rotate");
        written(a[9]);
        written(a[10]);
        return tuple(some(q), T.x[1] ? some(k) : none());
    });
}

PyObject* norm_rotate_backward(PyObject*, PyObject* const* a, Py_ssize_t given) {   // gq gk q k q_weight k_weight positions frequency axis eps adjacent dq dk
    return guarded(given, 13, [&] {
        Turn T(a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[10]);
        const double eps = number(a[9]);
        need(eps >= 0, "eps", "not below 0");
        const char* names[2] = {"gq", "gk"};
        need((a[1] == Py_None) == !T.x[1], "gk", "one for k");
        for (int z = 0; z < 2; z++) {
            if (!T.x[z]) continue;
            const at::Tensor& g = tensor(a[z], names[z]);
            check_side(g, *T.x[z], names[z]);
            pcr_heads& S = T.side[z];
            Turn::place(g, S.grad, S.grad_batch, S.grad_token, S.grad_head);
        }
        const at::Tensor q = T.into(0, a[11], "dq"), k = T.into(1, a[12], "dk");
        at::Tensor sums[2];
        for (int z = 0; z < 2; z++)
            if (T.w[z]) {
                sums[z] = at::empty({T.rotation.dim}, q.options().dtype(at::kFloat));
                T.side[z].weight_grad = (float*)sums[z].data_ptr();
            }
        at::Tensor work;
        size_t bytes = 0;
        if (T.w[0] || T.w[1]) {
            check(pcr_norm_rotate_workspace(T.rotation.batch * T.rotation.tokens, T.rotation.dim, &bytes), "pcr_norm_rotate_workspace");
            work = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
        }
        check(pcr_norm_rotate_backward(device_number(q), &T.side[0], &T.side[1], &T.rotation, (float)eps, T.dtype, T.weight_dtype, bytes ? work.data_ptr() : nullptr, bytes,
                                       stream_of(q)), "pcr_norm_rotate_backward");
        written(a[11]);
        written(a[12]);
        return tuple(some(q), T.x[1] ? some(k) : none(), T.w[0] ? some(sums[0]) : none(), T.w[1] ? some(sums[1]) : none());
    });
}

// ---- distillation ----

struct Distill {
    const at::Tensor& z;
    pcr_distill d = {};
    Distill(PyObject* logits, PyObject* top_index, PyObject* top_logits, PyObject* labels, PyObject* temperature, PyObject* distill_part, PyObject* label_part)
        : z(tensor(logits, "logits")) {
        need(z.is_cuda() && type_of(z) >= 0 && z.dim() == 2 && (z.size(1) == 1 || z.stride(1) == 1), "logits",
             "float32, float16 or bfloat16 [rows, classes] on the GPU, a row contiguous, is wanted");
        const at::Tensor &index = tensor(top_index, "top_index"), &t = tensor(top_logits, "top_logits");
        on(index, z, "top_index"); on(t, z, "top_logits");
        need(index.dim() == 2 && index.size(0) == z.size(0) && (index.scalar_type() == at::kInt || index.scalar_type() == at::kLong) && index.is_contiguous(), "top_index",
             "contiguous int32 or int64 [rows, top] is wanted");
        need(t.sizes() == index.sizes() && type_of(t) >= 0 && t.is_contiguous(), "top_logits", "contiguous, of top_index's shape, is wanted");
        const at::Tensor* l = maybe_tensor(labels, "labels");
        if (l) {
            on(*l, z, "labels");
            need(l->scalar_type() == at::kLong && l->dim() == 1 && l->size(0) == z.size(0) && l->is_contiguous(), "labels", "contiguous int64 [rows] is wanted");
        }
        const double T = number(temperature);
        need(T > 0 && std::isfinite(T), "temperature", "above 0");
        need(index.size(1) <= INT32_MAX, "top_index", "out of range");
        d.logits = z.data_ptr(); d.row_stride = z.stride(0); d.top_index = index.data_ptr(); d.top_logits = t.data_ptr();
        d.labels = l ? (const int64_t*)l->data_ptr() : nullptr;
        d.rows = z.size(0); d.classes = z.size(1); d.top = (int32_t)index.size(1); d.dtype = type_of(z); d.top_dtype = type_of(t); d.index_wide = index.scalar_type() == at::kLong;
        d.temperature = (float)T; d.distill_part = (float)number(distill_part); d.label_part = (float)number(label_part);
    }
    at::Tensor rows(int64_t columns = 0) const { return columns ? at::empty({d.rows, columns}, z.options().dtype(at::kFloat)) : at::empty({d.rows}, z.options().dtype(at::kFloat)); }
    const float* per_row(PyObject* o, const char* name) const {
        const at::Tensor& t = tensor(o, name);
        on(t, z, name);
        need(t.scalar_type() == at::kFloat && t.dim() == 1 && t.size(0) == d.rows && t.is_contiguous(), name, "contiguous float32 [rows] is wanted");
        return (const float*)t.data_ptr();
    }
    at::Tensor into(PyObject* o) const {
        const at::Tensor* t = maybe_tensor(o, "out");
        if (!t) return at::empty(z.sizes(), z.options());
        on(*t, z, "out");
        need(t->scalar_type() == z.scalar_type() && t->sizes() == z.sizes() && (t->size(1) == 1 || t->stride(1) == 1) && (t->size(0) < 2 || t->stride(0) != 0), "out",
             "type and shape of logits, a row contiguous, is wanted");
        check_written(*t, "out");
        return *t;
    }
    at::Tensor work(size_t& bytes) const {
        check(pcr_distill_workspace(d.rows, d.classes, &bytes), "pcr_distill_workspace");
        return bytes ? at::empty({(int64_t)bytes}, z.options().dtype(at::kByte)) : at::Tensor();
    }
};

PyObject* distill_forward(PyObject*, PyObject* const* a, Py_ssize_t given) {     // logits top_index top_logits labels temperature distill_part label_part
    return guarded(given, 7, [&] {
        Distill D(a[0], a[1], a[2], a[3], a[4], a[5], a[6]);
        const at::Tensor loss = D.rows(), sums = D.rows(2);
        size_t bytes = 0;
        const at::Tensor work = D.work(bytes);
        check(pcr_distill_forward(device_number(D.z), &D.d, (float*)loss.data_ptr(), (float*)sums.data_ptr(), bytes ? work.data_ptr() : nullptr, bytes, stream_of(D.z)),
              "pcr_distill_forward");
        return tuple(some(loss), some(sums));
    });
}

PyObject* distill_backward(PyObject*, PyObject* const* a, Py_ssize_t given) {    // row_grad logits top_index top_logits sums labels temperature distill_part label_part out
    return guarded(given, 10, [&] {
        Distill D(a[1], a[2], a[3], a[5], a[6], a[7], a[8]);
        const float* g = D.per_row(a[0], "row_grad");
        const at::Tensor& sums = tensor(a[4], "sums");
        on(sums, D.z, "sums");
        need(sums.scalar_type() == at::kFloat && sums.dim() == 2 && sums.size(0) == D.d.rows && sums.size(1) == 2 && sums.is_contiguous(), "sums", "contiguous float32 [rows, 2] is wanted");
        const at::Tensor out = D.into(a[9]);
        check(pcr_distill_backward(device_number(D.z), &D.d, (const float*)sums.data_ptr(), g, out.data_ptr(), out.stride(0), stream_of(D.z)), "pcr_distill_backward");
        written(a[9]);
        return some(out);
    });
}

PyObject* distill_step(PyObject*, PyObject* const* a, Py_ssize_t given) {        // logits top_index top_logits row_weight labels temperature distill_part label_part out
    return guarded(given, 9, [&] {
        Distill D(a[0], a[1], a[2], a[4], a[5], a[6], a[7]);
        const float* weight = D.per_row(a[3], "row_weight");
        const at::Tensor out = D.into(a[8]), loss = D.rows();
        size_t bytes = 0;
        const at::Tensor work = D.work(bytes);
        check(pcr_distill_step(device_number(D.z), &D.d, weight, (float*)loss.data_ptr(), out.data_ptr(), out.stride(0), bytes ? work.data_ptr() : nullptr, bytes, stream_of(D.z)),
              "pcr_distill_step");
        written(a[8]);
        return tuple(some(loss), some(out));
    });
}

PyObject* set_up(PyObject*, PyObject* const* a, Py_ssize_t given) {              // PcrError, the function that gives a device's current stream
    return guarded(given, 2, [&] {
        Py_INCREF(a[0]);
        Py_INCREF(a[1]);
        Py_XSETREF(g_error, a[0]);
        Py_XSETREF(g_current_stream, a[1]);
        return none();
    });
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {ENTRY(patch_rows), ENTRY(rotate_axes), ENTRY(norm_rotate), ENTRY(norm_rotate_backward), ENTRY(distill_forward), ENTRY(distill_backward),
                           ENTRY(distill_step), ENTRY(set_up), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_train", "The operators behind the decode on PyTorch tensors.", -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__train() { return PyModule_Create(&g_module); }
