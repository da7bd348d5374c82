// Native fast path of the Python binding (binding.py): the calls a user makes on every step, with the checks of the Python
// wrappers done on the tensors themselves.  A short call on the device takes 2 us; the wrapper's Python and ctypes took 2 to 6.
//
// Every function takes the wrapper's arguments and returns the output tensor, or None when anything is not as the fast path
// expects it (a wrong type, layout, device or size, an argument out of range, a status other than OK): the wrapper then goes
// its own way, which raises the error.  Nothing is decided here that the wrapper would decide differently.
// As under ctypes, the library's calls run without the interpreter lock: a launch blocks while its stream's queue is full, and what
// empties the queue may be a Python callback.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "hikonv.h"

namespace {

decltype(&hikonv_conv1d) g_conv1d = nullptr;
decltype(&hikonv_conv1d_dense) g_conv1d_dense = nullptr;
decltype(&hikonv_conv2d) g_conv2d = nullptr;
decltype(&hikonv_conv2d_dense) g_conv2d_dense = nullptr;
decltype(&hikonv_conv2d_workspace_bytes) g_workspace_bytes = nullptr;
decltype(&hikonv_pack) g_pack = nullptr;
decltype(&hikonv_quantize_rows) g_quantize_rows = nullptr;
decltype(&hikonv_linear) g_linear = nullptr;
decltype(&hikonv_grouped_linear) g_grouped_linear = nullptr;
decltype(&hikonv_linear_workspace_bytes) g_linear_workspace_bytes = nullptr;
decltype(&hikonv_sort_by_expert) g_sort_by_expert = nullptr;
decltype(&hikonv_sort_by_expert_workspace_bytes) g_sort_workspace_bytes = nullptr;
decltype(&hikonv_rows_to_experts) g_rows_to_experts = nullptr;
decltype(&hikonv_rows_from_experts) g_rows_from_experts = nullptr;
decltype(&hikonv_rows_from_experts_grad) g_rows_from_experts_grad = nullptr;
decltype(&hikonv_zero_other_rows) g_zero_other_rows = nullptr;
decltype(&hikonv_quantize_blocks) g_quantize_blocks = nullptr;
decltype(&hikonv_linear_f8) g_linear_f8 = nullptr;
decltype(&hikonv_grouped_linear_f8) g_grouped_linear_f8 = nullptr;

// Reads arguments one after the other; `ok` stays true while all are as expected.
struct Args {
    PyObject *const *a;
    Py_ssize_t n, at = 0;
    bool ok = true;

    PyObject *next() {
        if (at >= n) ok = false;
        return at < n ? a[at++] : Py_None;
    }
    long integer() {
        const long v = PyLong_AsLong(next());
        if (v == -1 && PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        return v;
    }
    int int32() {
        const long v = integer();
        if (v != (int)v) ok = false;
        return (int)v;
    }
    const at::Tensor *tensor() {
        PyObject *o = next();
        if (!THPVariable_Check(o)) {
            ok = false;
            return nullptr;
        }
        return &THPVariable_Unpack(o);
    }
    // a tensor, or null for None
    const at::Tensor *optional_tensor() {
        if (at < n && a[at] == Py_None) {
            ++at;
            return nullptr;
        }
        return tensor();
    }
    // (shift, lo, hi), or false for None
    bool requant(int *shift, int *lo, int *hi) {
        PyObject *o = next();
        *shift = *lo = *hi = 0;
        if (o == Py_None) return false;
        if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 3) {
            ok = false;
            return false;
        }
        Args inner{&PyTuple_GET_ITEM(o, 0), 3};
        *shift = inner.int32();
        *lo = inner.int32();
        *hi = inner.int32();
        ok = ok && inner.ok;
        return true;
    }
    // a tuple or torch.Size of four sizes
    bool shape4(int64_t (&s)[4]) {
        PyObject *o = next();
        if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) return ok = false;
        Args inner{&PyTuple_GET_ITEM(o, 0), 4};
        for (auto &v : s) v = inner.integer();
        return ok = ok && inner.ok;
    }
};

bool plain_cuda(const at::Tensor *t) { return t && t->is_cuda() && t->layout() == at::kStrided && t->is_contiguous(); }
bool codes(const at::Tensor *t) { return plain_cuda(t) && (t->scalar_type() == at::kChar || t->scalar_type() == at::kByte); }
bool fits_int(int64_t v) { return v == (int)v; }
bool output_ok(const at::Tensor &t, int64_t numel, bool bytes, const at::Tensor &like) {
    return plain_cuda(&t) && t.device() == like.device() && t.numel() == numel &&
           (bytes ? t.scalar_type() == at::kChar || t.scalar_type() == at::kByte : t.scalar_type() == at::kInt);
}
at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor &like) {
    return at::empty(sizes, at::TensorOptions().dtype(type).device(like.device()));
}
// The stream a call without one runs on: the current stream of the current device, as in the wrappers.
void *current_stream() { return (void *)c10::cuda::getCurrentCUDAStream().stream(); }

// `out` when it was given, else a new Python object for the tensor that was made.
PyObject *result(PyObject *given, const at::Tensor &made) {
    if (given != Py_None) {
        Py_INCREF(given);
        return given;
    }
    return THPVariable_Wrap(made);
}

// Calls into the library with the interpreter lock released.
template <typename F>
int unlocked(F call) {
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call();
    Py_END_ALLOW_THREADS
    return status;
}

template <typename F>
PyObject *guarded(F f) {
    try {
        if (PyObject *r = f()) return r;
        if (PyErr_Occurred()) return nullptr;
    } catch (const std::exception &) {                   // an allocation that failed, say: the wrapper meets it again
    }
    Py_RETURN_NONE;
}

// conv1d(f, g, p, q, f_signed, g_signed, algo, out)
PyObject *conv1d(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *f = in.tensor(), *g = in.tensor();
        const int p = in.int32(), q = in.int32(), fs = in.int32() != 0, gs = in.int32() != 0, algo = in.int32();
        const at::Tensor *given = in.optional_tensor();
        if (!in.ok || !codes(f) || !codes(g) || !fits_int(g->numel())) return nullptr;
        const int64_t len = f->numel(), n_out = len + g->numel() - 1;
        if (len < 1 || g->numel() < 1) return nullptr;
        at::Tensor made;
        if (!given) made = empty({n_out}, at::kInt, *f);
        const at::Tensor &y = given ? *given : made;
        if (!output_ok(y, n_out, false, *f)) return nullptr;
        const int8_t *f_ptr = (const int8_t *)f->data_ptr(), *g_ptr = (const int8_t *)g->data_ptr();
        const int K = (int)g->numel();
        int32_t *y_ptr = (int32_t *)y.data_ptr();
        void *st = current_stream();
        if (unlocked([&] { return g_conv1d(f_ptr, (size_t)len, g_ptr, K, p, q, fs, gs, y_ptr, algo, nullptr, st); }) != HIKONV_OK) return nullptr;
        return result(a[7], made);
    });
}

// conv1d_dense(f_dense, n, g, p, q, f_signed, g_signed, out)
PyObject *conv1d_dense(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *f = in.tensor();
        const int64_t len = in.integer();
        const at::Tensor *g = in.tensor();
        const int p = in.int32(), q = in.int32(), fs = in.int32() != 0, gs = in.int32() != 0;
        const at::Tensor *given = in.optional_tensor();
        if (!in.ok || !codes(f) || f->scalar_type() != at::kByte || !codes(g) || !fits_int(g->numel())) return nullptr;
        if (len < 1 || g->numel() < 1 || p < 1 || p > 8 || f->numel() * 8 < len * p) return nullptr;
        const int64_t n_out = len + g->numel() - 1;
        at::Tensor made;
        if (!given) made = empty({n_out}, at::kInt, *f);
        const at::Tensor &y = given ? *given : made;
        if (!output_ok(y, n_out, false, *f)) return nullptr;
        const uint8_t *f_ptr = (const uint8_t *)f->data_ptr();
        const int8_t *g_ptr = (const int8_t *)g->data_ptr();
        const int K = (int)g->numel();
        int32_t *y_ptr = (int32_t *)y.data_ptr();
        void *st = current_stream();
        if (unlocked([&] { return g_conv1d_dense(f_ptr, (size_t)len, g_ptr, K, p, q, fs, gs, y_ptr, nullptr, st); }) != HIKONV_OK) return nullptr;
        return result(a[7], made);
    });
}

// pack(in, bits, is_signed, S, N, word_bits)
PyObject *pack(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *x = in.tensor();
        const int bits = in.int32(), is_signed = in.int32() != 0, S = in.int32(), N = in.int32(), word_bits = in.int32();
        if (!in.ok || !codes(x) || N < 1 || (word_bits != 32 && word_bits != 64)) return nullptr;
        const int64_t count = x->numel();
        const at::Tensor words = empty({(count + N - 1) / N}, word_bits == 32 ? at::kInt : at::kLong, *x);
        const int8_t *x_ptr = (const int8_t *)x->data_ptr();
        void *words_ptr = words.data_ptr(), *st = current_stream();
        if (unlocked([&] { return g_pack(x_ptr, (size_t)count, bits, is_signed, S, N, word_bits, words_ptr, st); }) != HIKONV_OK) return nullptr;
        return THPVariable_Wrap(words);
    });
}

// What the 2-D calls share.  B, Ci, H, W and Co, Ci, K, K are known; makes the workspace and the output where none was given.
struct Layer {
    int64_t B, Ci, H, W, Co, K;
    int pad;
    int64_t Ho() const { return H + 2 * pad - K + 1; }
    int64_t Wo() const { return W + 2 * pad - K + 1; }
    bool plausible() const {
        for (int64_t v : {B, Ci, H, W, Co, K})
            if (v < 1 || !fits_int(v)) return false;
        return pad >= 0 && pad < 1 << 20 && Ho() >= 1 && Wo() >= 1;
    }
    bool workspace(const at::Tensor *given, const at::Tensor &like, at::Tensor *made, void **ptr, size_t *bytes) const {
        if (!given) {
            *made = empty({(int64_t)g_workspace_bytes((int)B, (int)Ci, (int)H, (int)W, (int)Co, (int)K, pad)}, at::kByte, like);
            given = made;
        } else if (!plain_cuda(given) || given->device() != like.device()) {
            return false;
        }
        *ptr = given->data_ptr();
        *bytes = (size_t)given->numel() * given->element_size();
        return true;
    }
};

// conv2d(x, w, pad, p, q, x_signed, w_signed, requant, algo, workspace, out, stride)
PyObject *conv2d(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *x = in.tensor(), *w = in.tensor();
        Layer l;
        l.pad = in.int32();
        const int p = in.int32(), q = in.int32(), xs = in.int32() != 0, ws = in.int32() != 0;
        int shift, lo, hi;
        const bool rq = in.requant(&shift, &lo, &hi);
        const int algo = in.int32();
        const at::Tensor *space = in.optional_tensor(), *given = in.optional_tensor();
        const int stride = in.int32();
        if (!in.ok || !codes(x) || !codes(w) || x->dim() != 4 || w->dim() != 4) return nullptr;
        l.B = x->size(0); l.Ci = x->size(1); l.H = x->size(2); l.W = x->size(3);
        l.Co = w->size(0); l.K = w->size(2);
        if (w->size(1) != l.Ci || w->size(3) != l.K || !l.plausible()) return nullptr;
        at::Tensor made_space, made;
        void *space_ptr;
        size_t space_bytes;
        if (!l.workspace(space, *x, &made_space, &space_ptr, &space_bytes)) return nullptr;
        if (!given) made = empty({l.B, l.Co, l.Ho(), l.Wo()}, rq ? at::kChar : at::kInt, *x);
        const at::Tensor &y = given ? *given : made;
        if (!output_ok(y, l.B * l.Co * l.Ho() * l.Wo(), rq, *x)) return nullptr;
        const int8_t *x_ptr = (const int8_t *)x->data_ptr(), *w_ptr = (const int8_t *)w->data_ptr();
        void *y_ptr = y.data_ptr(), *st = current_stream();
        const int status = unlocked([&] {
            return g_conv2d(x_ptr, (int)l.B, (int)l.Ci, (int)l.H, (int)l.W, w_ptr, (int)l.Co, (int)l.K, stride, l.pad, p, q, xs, ws, y_ptr,
                            rq ? 1 : 0, shift, lo, hi, space_ptr, space_bytes, algo, nullptr, st);
        });
        if (status != HIKONV_OK) return nullptr;
        return result(a[10], made);
    });
}

// conv2d_dense(x, x_shape, x_store_bits, w, w_shape, w_store_bits, pad, p, q, x_signed, w_signed, requant, out_store_bits, pool,
//              algo, workspace, out, stride)
PyObject *conv2d_dense(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *x = in.tensor();
        int64_t xsh[4], wsh[4];
        in.shape4(xsh);
        const int x_bits = in.int32();
        const at::Tensor *w = in.tensor();
        in.shape4(wsh);
        const int w_bits = in.int32();
        Layer l;
        l.pad = in.int32();
        const int p = in.int32(), q = in.int32(), xs = in.int32() != 0, ws = in.int32() != 0;
        int shift, lo, hi;
        const bool rq = in.requant(&shift, &lo, &hi);
        const int out_bits = in.int32(), pool = in.int32() != 0, algo = in.int32();
        const at::Tensor *space = in.optional_tensor(), *given = in.optional_tensor();
        const int stride = in.int32();
        if (!in.ok || !codes(x) || !codes(w)) return nullptr;
        l.B = xsh[0]; l.Ci = xsh[1]; l.H = xsh[2]; l.W = xsh[3];
        l.Co = wsh[0]; l.K = wsh[2];
        if (wsh[1] != l.Ci || wsh[3] != l.K || !l.plausible()) return nullptr;
        if (x_bits < 1 || x_bits > 8 || w_bits < 1 || w_bits > 8 || out_bits < 1 || out_bits > 8) return nullptr;
        if (x->numel() * 8 < l.B * l.Ci * l.H * l.W * x_bits || w->numel() * 8 < l.Co * l.Ci * l.K * l.K * w_bits) return nullptr;
        const int64_t Hq = pool ? l.Ho() / 2 : l.Ho(), Wq = pool ? l.Wo() / 2 : l.Wo();
        at::Tensor made_space, made;
        void *space_ptr;
        size_t space_bytes;
        if (!l.workspace(space, *x, &made_space, &space_ptr, &space_bytes)) return nullptr;
        const int64_t n_out = rq ? (l.B * l.Co * Hq * Wq * out_bits + 7) / 8 : l.B * l.Co * l.Ho() * l.Wo();
        if (!given)
            made = !rq ? empty({l.B, l.Co, l.Ho(), l.Wo()}, at::kInt, *x)
                 : out_bits == 8 ? empty({l.B, l.Co, Hq, Wq}, at::kChar, *x) : empty({n_out}, at::kByte, *x);
        const at::Tensor &y = given ? *given : made;
        if (!output_ok(y, n_out, rq, *x)) return nullptr;
        const void *x_ptr = x->data_ptr(), *w_ptr = w->data_ptr();
        void *y_ptr = y.data_ptr(), *st = current_stream();
        const int status = unlocked([&] {
            return g_conv2d_dense(x_ptr, x_bits, (int)l.B, (int)l.Ci, (int)l.H, (int)l.W, w_ptr, w_bits, (int)l.Co, (int)l.K, stride, l.pad, p, q,
                                  xs, ws, y_ptr, rq ? out_bits : 32, rq ? 1 : 0, shift, lo, hi, pool, space_ptr, space_bytes, algo, nullptr, st);
        });
        if (status != HIKONV_OK) return nullptr;
        return result(a[16], made);
    });
}

// What the linear layers share: a matrix on a device whose rows may lie apart, and contiguous scales, biases and offsets.
bool matrix(const at::Tensor *t, int64_t *row) {
    if (!t || !t->is_cuda() || t->layout() != at::kStrided || t->dim() != 2 || (t->size(1) > 1 && t->stride(1) != 1)) return false;
    *row = t->size(0) > 1 ? t->stride(0) : t->size(1);
    return fits_int(t->size(0)) && fits_int(t->size(1));
}
bool out_matrix(const at::Tensor *t, int64_t M, int64_t N, at::ScalarType type, const at::Tensor &like, int64_t *row) {
    return matrix(t, row) && t->scalar_type() == type && t->device() == like.device() && t->size(0) == M && t->size(1) == N;
}
bool vector_ok(const at::Tensor *t, at::ScalarType type, at::IntArrayRef shape, const at::Tensor &like) {
    return !t || (plain_cuda(t) && t->scalar_type() == type && t->device() == like.device() && t->sizes() == shape);
}
const void *address(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }
int float_type(at::ScalarType t) {
    return t == at::kFloat ? HIKONV_OUT_F32 : t == at::kHalf ? HIKONV_OUT_F16 : t == at::kBFloat16 ? HIKONV_OUT_BF16 : -1;
}

// quantize_rows(x, bits, is_signed, codes, scale)
PyObject *quantize_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *x = in.tensor();
        const int bits = in.int32(), is_signed = in.int32() != 0;
        const at::Tensor *codes_given = in.optional_tensor(), *scale_given = in.optional_tensor();
        int64_t x_row;
        if (!in.ok || !matrix(x, &x_row)) return nullptr;
        const int type = float_type(x->scalar_type());
        const int64_t M = x->size(0), K = x->size(1);
        if (type < 0 || K < 1) return nullptr;
        at::Tensor made_codes, made_scale;
        if (!codes_given) made_codes = empty({M, K}, is_signed ? at::kChar : at::kByte, *x);
        if (!scale_given) made_scale = empty({M}, at::kFloat, *x);
        const at::Tensor &c = codes_given ? *codes_given : made_codes, &s = scale_given ? *scale_given : made_scale;
        if (!output_ok(c, M * K, true, *x) || c.dim() != 2 || c.size(0) != M || !vector_ok(&s, at::kFloat, {M}, *x)) return nullptr;
        const c10::cuda::OptionalCUDAGuard guard(x->device());
        const void *x_ptr = x->data_ptr();
        int8_t *c_ptr = (int8_t *)c.data_ptr();
        float *s_ptr = (float *)s.data_ptr();
        void *st = current_stream();
        if (unlocked([&] { return g_quantize_rows(x_ptr, type, x_row, (int)M, (int)K, bits, is_signed, c_ptr, s_ptr, st); }) != HIKONV_OK)
            return nullptr;
        PyObject *pc = result(a[3], made_codes), *ps = result(a[4], made_scale);
        PyObject *both = pc && ps ? PyTuple_Pack(2, pc, ps) : nullptr;
        Py_XDECREF(pc);
        Py_XDECREF(ps);
        return both;
    });
}

// linear(x, w, offsets or None, p, q, x_signed, w_signed, w_store_bits, x_scale, w_scale, bias, activation, residual, requant, out_dtype, out,
//        workspace)
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *x = in.tensor(), *w = in.tensor(), *offsets = in.optional_tensor();
        const int p = in.int32(), q = in.int32(), xs = in.int32() != 0, ws = in.int32() != 0, w_bits = in.int32();
        const at::Tensor *x_scale = in.optional_tensor(), *w_scale = in.optional_tensor(), *bias = in.optional_tensor();
        hikonv_epilogue_t ep{};
        ep.activation = in.int32();
        const at::Tensor *residual = in.optional_tensor();
        const bool rq = in.requant(&ep.shift, &ep.lo, &ep.hi);
        PyObject *dtype = in.next();
        const at::Tensor *given = in.optional_tensor(), *space = in.optional_tensor();
        int64_t x_row, out_row, res_row;
        if (!in.ok || !matrix(x, &x_row) || (x->scalar_type() != at::kChar && x->scalar_type() != at::kByte)) return nullptr;
        if (!codes(w) || w->device() != x->device() || w->dim() != (offsets ? 3 : 2)) return nullptr;
        const int64_t M = x->size(0), K = x->size(1), E = offsets ? w->size(0) : 1, N = w->size(w->dim() - 2);
        if (K < 1 || N < 1 || E < 1 || !fits_int(N) || !fits_int(E) || w_bits < 1 || w_bits > 8 || w->size(w->dim() - 1) * 8 != K * w_bits) return nullptr;
        if (dtype != Py_None && !THPDtype_Check(dtype)) return nullptr;
        // the output's type: what `out_dtype` says, else the given output's, else what the other arguments ask for
        const bool scaled = x_scale || w_scale;
        const at::ScalarType type = dtype != Py_None ? ((THPDtype *)dtype)->scalar_type : given ? given->scalar_type()
                                  : rq ? at::kChar : scaled ? at::kBFloat16 : at::kInt;
        const int real = float_type(type);
        if (rq ? scaled || (type != at::kChar && type != at::kByte) : real < 0 && (scaled || type != at::kInt)) return nullptr;
        ep.out_type = rq ? HIKONV_OUT_CODES : real >= 0 ? real : HIKONV_OUT_SUMS;
        at::Tensor made;
        if (!given) made = empty({M, N}, type, *x);
        const at::Tensor &y = given ? *given : made;
        if (!out_matrix(&y, M, N, type, *x, &out_row)) return nullptr;
        const int64_t per_column[2] = {E, N};
        const at::IntArrayRef columns(per_column + (offsets ? 0 : 1), offsets ? 2 : 1);
        if (!vector_ok(x_scale, at::kFloat, {M}, *x) || !vector_ok(w_scale, at::kFloat, columns, *x) ||
            !vector_ok(bias, rq ? at::kInt : at::kFloat, columns, *x) || !vector_ok(offsets, at::kInt, {E + 1}, *x))
            return nullptr;
        if (residual) {
            if (!out_matrix(residual, M, N, type, *x, &res_row)) return nullptr;
            ep.residual_row_stride = res_row;
        }
        ep.d_x_scale = (const float *)address(x_scale);
        ep.d_w_scale = (const float *)address(w_scale);
        ep.d_bias = address(bias);
        ep.d_residual = address(residual);
        const c10::cuda::OptionalCUDAGuard guard(x->device());
        const void *x_ptr = x->data_ptr(), *w_ptr = w->data_ptr();
        const int32_t *off_ptr = (const int32_t *)address(offsets);
        const size_t need = g_linear_workspace_bytes(x_ptr, x_row, w_ptr, w_bits, offsets ? (int)E : 0, (int)M, (int)N, (int)K);
        at::Tensor made_space;
        if (need && !space) {
            made_space = empty({(int64_t)need}, at::kByte, *x);
            space = &made_space;
        }
        if (space && (!plain_cuda(space) || space->device() != x->device())) return nullptr;
        void *y_ptr = y.data_ptr(), *st = current_stream(), *space_ptr = space ? space->data_ptr() : nullptr;
        const size_t space_bytes = space ? (size_t)space->numel() * space->element_size() : 0;
        const int status = unlocked([&] {
            return offsets ? g_grouped_linear(x_ptr, x_row, w_ptr, w_bits, off_ptr, (int)E, (int)M, (int)N, (int)K, p, q, xs, ws, y_ptr, out_row, &ep,
                                              space_ptr, space_bytes, st)
                           : g_linear(x_ptr, x_row, w_ptr, w_bits, (int)M, (int)N, (int)K, p, q, xs, ws, y_ptr, out_row, &ep, space_ptr, space_bytes, st);
        });
        if (status != HIKONV_OK) return nullptr;
        return result(a[15], made);
    });
}

// What the calls of a mixture of experts share: the places of pairs, and two results.
bool slots_ok(const at::Tensor *t, const at::Tensor &like, int64_t rows) {
    return plain_cuda(t) && t->scalar_type() == at::kInt && t->dim() == 2 && t->device() == like.device() && (rows < 0 || t->size(0) == rows) &&
           fits_int(t->size(0)) && fits_int(t->size(1));
}
PyObject *two(PyObject *a, PyObject *b) {
    PyObject *both = a && b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    return both;
}
int f8_type(at::ScalarType t) { return t == at::kFloat8_e4m3fn ? HIKONV_F8_E4M3 : t == at::kFloat8_e5m2 ? HIKONV_F8_E5M2 : -1; }
// Rows on 16-byte boundaries.
at::Tensor f8_rows(int64_t rows, int64_t K, at::ScalarType type, const at::Tensor &like) {
    const int64_t wide = (K + 15) / 16 * 16;
    const at::Tensor t = empty({rows, wide}, type, like);
    return wide == K ? t : t.narrow(1, 0, K);
}

// sort_by_expert(experts, n_experts, offsets, slots, workspace)
PyObject *sort_by_expert(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *x = in.tensor();
        const int E = in.int32();
        const at::Tensor *offsets = in.optional_tensor(), *slots = in.optional_tensor(), *space = in.optional_tensor();
        int64_t row;
        if (!in.ok || !matrix(x, &row) || (x->scalar_type() != at::kInt && x->scalar_type() != at::kLong) || E < 1) return nullptr;
        const int64_t T = x->size(0), k = x->size(1);
        at::Tensor made_offsets, made_slots, made_space;
        if (!offsets) made_offsets = empty({(int64_t)E + 1}, at::kInt, *x);
        if (!slots) made_slots = empty({T, k}, at::kInt, *x);
        const at::Tensor &o = offsets ? *offsets : made_offsets, &s = slots ? *slots : made_slots;
        if (!vector_ok(&o, at::kInt, {(int64_t)E + 1}, *x) || !vector_ok(&s, at::kInt, {T, k}, *x)) return nullptr;
        const c10::cuda::OptionalCUDAGuard guard(x->device());
        const size_t need = g_sort_workspace_bytes((int)T, (int)k, E);
        if (need && !space) {
            made_space = empty({(int64_t)need}, at::kByte, *x);
            space = &made_space;
        }
        if (space && (!plain_cuda(space) || space->device() != x->device())) return nullptr;
        const void *x_ptr = x->data_ptr();
        const int index_bytes = (int)x->element_size();
        int32_t *o_ptr = (int32_t *)o.data_ptr(), *s_ptr = (int32_t *)s.data_ptr();
        void *space_ptr = space ? space->data_ptr() : nullptr, *st = current_stream();
        const size_t space_bytes = space ? (size_t)space->numel() * space->element_size() : 0;
        if (unlocked([&] { return g_sort_by_expert(x_ptr, index_bytes, row, (int)T, (int)k, E, o_ptr, s_ptr, space_ptr, space_bytes, st); }) != HIKONV_OK)
            return nullptr;
        return two(result(a[2], made_offsets), result(a[3], made_slots));
    });
}

// rows_to_experts(x, slots, out)
PyObject *rows_to_experts(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *x = in.tensor(), *slots = in.tensor(), *given = in.optional_tensor();
        int64_t x_row, out_row;
        if (!in.ok || !matrix(x, &x_row) || x->is_complex() || !slots_ok(slots, *x, x->size(0))) return nullptr;
        const int size = (int)x->element_size();
        if (size != 1 && size != 2 && size != 4) return nullptr;
        const int64_t T = x->size(0), H = x->size(1), k = slots->size(1);
        at::Tensor made;
        if (!given) made = empty({T * k, H}, x->scalar_type(), *x);
        const at::Tensor &y = given ? *given : made;
        if (y.dim() != 2 || !out_matrix(&y, y.size(0), H, x->scalar_type(), *x, &out_row)) return nullptr;
        const c10::cuda::OptionalCUDAGuard guard(x->device());
        const void *x_ptr = x->data_ptr();
        const int32_t *s_ptr = (const int32_t *)slots->data_ptr();
        void *y_ptr = y.data_ptr(), *st = current_stream();
        const int R = (int)y.size(0);
        if (unlocked([&] { return g_rows_to_experts(x_ptr, size, x_row, s_ptr, (int)T, (int)k, (int)H, y_ptr, out_row, R, st); }) != HIKONV_OK) return nullptr;
        return result(a[2], made);
    });
}

// rows_from_experts(y, slots, weights, residual, out)
PyObject *rows_from_experts(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *y = in.tensor(), *slots = in.tensor(), *weights = in.optional_tensor(), *residual = in.optional_tensor(), *given = in.optional_tensor();
        int64_t y_row, out_row, res_row;
        if (!in.ok || !matrix(y, &y_row) || !slots_ok(slots, *y, -1)) return nullptr;
        const int type = float_type(y->scalar_type());
        if (type < 0) return nullptr;
        const int64_t R = y->size(0), H = y->size(1), T = slots->size(0), k = slots->size(1);
        at::Tensor made;
        if (!given) made = empty({T, H}, y->scalar_type(), *y);
        const at::Tensor &o = given ? *given : made;
        res_row = H;
        if (!out_matrix(&o, T, H, y->scalar_type(), *y, &out_row) || !vector_ok(weights, at::kFloat, {T, k}, *y) ||
            (residual && !out_matrix(residual, T, H, y->scalar_type(), *y, &res_row)))
            return nullptr;
        const c10::cuda::OptionalCUDAGuard guard(y->device());
        const void *y_ptr = y->data_ptr(), *r_ptr = address(residual);
        const int32_t *s_ptr = (const int32_t *)slots->data_ptr();
        const float *w_ptr = (const float *)address(weights);
        void *o_ptr = o.data_ptr(), *st = current_stream();
        if (unlocked([&] {
                return g_rows_from_experts(y_ptr, type, y_row, (int)R, s_ptr, w_ptr, (int)T, (int)k, (int)H, r_ptr, res_row, o_ptr, out_row, st);
            }) != HIKONV_OK)
            return nullptr;
        return result(a[4], made);
    });
}

constexpr int64_t kZeroAllBytes = 8 << 20;             // as in binding.py

// rows_from_experts_grad(grad, y, slots, weights, grad_y, grad_weights)
PyObject *rows_from_experts_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *grad = in.tensor(), *y = in.optional_tensor(), *slots = in.tensor(), *weights = in.optional_tensor(),
                         *given_y = in.optional_tensor(), *given_w = in.optional_tensor();
        int64_t grad_row, y_row, grad_y_row;
        if (!in.ok || !matrix(grad, &grad_row) || !slots_ok(slots, *grad, grad->size(0)) || (given_w && !weights) || (weights && !y)) return nullptr;
        const at::ScalarType type = grad->scalar_type();
        if (float_type(type) < 0 || (y && y->dim() != 2)) return nullptr;
        const int64_t T = grad->size(0), H = grad->size(1), k = slots->size(1);
        at::Tensor made_y, made_w, others;
        if (!given_y) {
            // rows that no slot names are zeros: all rows beforehand where that is cheap, else those alone
            const int64_t rows = y ? y->size(0) : T * k;
            const bool small = rows * H * (int64_t)grad->element_size() <= kZeroAllBytes;
            made_y = small ? at::zeros({rows, H}, at::TensorOptions().dtype(type).device(grad->device())) : empty({rows, H}, type, *grad);
            if (!small) others = empty({rows}, at::kByte, *grad);
        }
        if (weights && !given_w) made_w = empty({T, k}, at::kFloat, *grad);
        const at::Tensor &gy = given_y ? *given_y : made_y;
        const at::Tensor *gw = given_w ? given_w : weights ? &made_w : nullptr;
        if (gy.dim() != 2 || !out_matrix(&gy, gy.size(0), H, type, *grad, &grad_y_row)) return nullptr;
        const int64_t R = gy.size(0);
        y_row = H;
        if (weights && !out_matrix(y, R, H, type, *grad, &y_row)) return nullptr;
        if (!vector_ok(weights, at::kFloat, {T, k}, *grad) || !vector_ok(gw, at::kFloat, {T, k}, *grad)) return nullptr;
        const c10::cuda::OptionalCUDAGuard guard(grad->device());
        const void *g_ptr = grad->data_ptr(), *y_ptr = weights ? y->data_ptr() : nullptr;
        const int32_t *s_ptr = (const int32_t *)slots->data_ptr();
        const float *w_ptr = (const float *)address(weights);
        void *gy_ptr = gy.data_ptr(), *st = current_stream();
        float *gw_ptr = (float *)address(gw);
        void *others_ptr = others.defined() ? others.data_ptr() : nullptr;
        const int size = (int)grad->element_size();
        if (unlocked([&] {
                const int rc = others_ptr ? g_zero_other_rows(s_ptr, (int)T, (int)k, gy_ptr, size, grad_y_row, (int)R, (int)H, others_ptr, (size_t)R, st) : HIKONV_OK;
                if (rc != HIKONV_OK) return rc;
                return g_rows_from_experts_grad(g_ptr, float_type(type), grad_row, y_ptr, y_row, (int)R, s_ptr, w_ptr, (int)T, (int)k, (int)H, gy_ptr,
                                                grad_y_row, gw_ptr, st);
            }) != HIKONV_OK)
            return nullptr;
        PyObject *second = nullptr;
        if (gw) {
            second = result(a[5], made_w);
        } else {
            Py_INCREF(Py_None);
            second = Py_None;
        }
        return two(result(a[4], made_y), second);
    });
}

// quantize_blocks(x, dtype, slots, values, scale)
PyObject *quantize_blocks(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *x = in.tensor();
        PyObject *dtype = in.next();
        const at::Tensor *slots = in.optional_tensor(), *given_v = in.optional_tensor(), *given_s = in.optional_tensor();
        int64_t x_row, v_row, s_row;
        if (!in.ok || !matrix(x, &x_row) || !THPDtype_Check(dtype)) return nullptr;
        const int type = float_type(x->scalar_type());
        const at::ScalarType f8 = ((THPDtype *)dtype)->scalar_type;
        if (type < 0 || f8_type(f8) < 0 || (slots && !slots_ok(slots, *x, x->size(0)))) return nullptr;
        const int64_t M = x->size(0), K = x->size(1), k = slots ? slots->size(1) : 0, blocks = (K + 127) / 128;
        if (K < 1 || (given_v && given_v->dim() != 2)) return nullptr;
        const int64_t rows = !slots ? M : given_v ? given_v->size(0) : M * k;
        at::Tensor made_v, made_s;
        if (!given_v) made_v = f8_rows(rows, K, f8, *x);
        if (!given_s) made_s = empty({blocks, rows}, at::kFloat, *x);
        const at::Tensor &v = given_v ? *given_v : made_v, &s = given_s ? *given_s : made_s;
        if (!out_matrix(&v, rows, K, f8, *x, &v_row) || !out_matrix(&s, blocks, rows, at::kFloat, *x, &s_row)) return nullptr;
        const c10::cuda::OptionalCUDAGuard guard(x->device());
        const void *x_ptr = x->data_ptr();
        const int32_t *slots_ptr = (const int32_t *)address(slots);
        uint8_t *v_ptr = (uint8_t *)v.data_ptr();
        float *s_ptr = (float *)s.data_ptr();
        void *st = current_stream();
        if (unlocked([&] {
                return g_quantize_blocks(x_ptr, type, x_row, (int)M, (int)K, f8_type(f8), slots_ptr, (int)k, slots ? (int)rows : 0, v_ptr, v_row, s_ptr, s_row, st);
            }) != HIKONV_OK)
            return nullptr;
        return two(result(a[3], made_v), result(a[4], made_s));
    });
}

// linear_f8(x, w, offsets or None, x_scale, w_scale, bias, activation, residual, out_dtype, out)
PyObject *linear_f8(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        Args in{a, n};
        const at::Tensor *x = in.tensor(), *w = in.tensor(), *offsets = in.optional_tensor(), *x_scale = in.tensor(), *w_scale = in.tensor(),
                         *bias = in.optional_tensor();
        hikonv_epilogue_t ep{};
        ep.activation = in.int32();
        const at::Tensor *residual = in.optional_tensor();
        PyObject *dtype = in.next();
        const at::Tensor *given = in.optional_tensor();
        int64_t x_row, xs_row, out_row, res_row;
        if (!in.ok || !matrix(x, &x_row) || f8_type(x->scalar_type()) < 0 || (dtype != Py_None && !THPDtype_Check(dtype))) return nullptr;
        const int dims = offsets ? 3 : 2;
        if (!w->is_cuda() || w->layout() != at::kStrided || f8_type(w->scalar_type()) < 0 || w->device() != x->device() || w->dim() != dims) return nullptr;
        const int64_t M = x->size(0), K = x->size(1), E = offsets ? w->size(0) : 1, N = w->size(dims - 2), blocks = (K + 127) / 128, n_blocks = (N + 127) / 128;
        if (K < 1 || N < 1 || E < 1 || !fits_int(N) || !fits_int(E) || w->size(dims - 1) != K || (K > 1 && w->stride(dims - 1) != 1)) return nullptr;
        const int64_t w_row = N > 1 ? w->stride(dims - 2) : E > 1 ? w->stride(0) : K;
        if (E > 1 && w->stride(0) != N * w_row) return nullptr;
        const at::ScalarType type = dtype != Py_None ? ((THPDtype *)dtype)->scalar_type : given ? given->scalar_type() : at::kBFloat16;
        ep.out_type = float_type(type);
        if (ep.out_type < 0) return nullptr;
        at::Tensor made;
        if (!given) made = empty({M, N}, type, *x);
        const at::Tensor &y = given ? *given : made;
        if (!out_matrix(&y, M, N, type, *x, &out_row) || !out_matrix(x_scale, blocks, M, at::kFloat, *x, &xs_row)) return nullptr;
        const int64_t per_column[2] = {E, N}, per_tile[3] = {E, n_blocks, blocks};
        if (!vector_ok(w_scale, at::kFloat, at::IntArrayRef(per_tile + (offsets ? 0 : 1), dims), *x) ||
            !vector_ok(bias, at::kFloat, at::IntArrayRef(per_column + (offsets ? 0 : 1), dims - 1), *x) || !vector_ok(offsets, at::kInt, {E + 1}, *x))
            return nullptr;
        if (residual) {
            if (!out_matrix(residual, M, N, type, *x, &res_row)) return nullptr;
            ep.residual_row_stride = res_row;
        }
        ep.d_bias = address(bias);
        ep.d_residual = address(residual);
        const c10::cuda::OptionalCUDAGuard guard(x->device());
        const void *x_ptr = x->data_ptr(), *w_ptr = w->data_ptr();
        const int x_f8 = f8_type(x->scalar_type()), w_f8 = f8_type(w->scalar_type());
        const int32_t *off_ptr = (const int32_t *)address(offsets);
        const float *xs_ptr = (const float *)x_scale->data_ptr(), *ws_ptr = (const float *)w_scale->data_ptr();
        void *y_ptr = y.data_ptr(), *st = current_stream();
        const int status = unlocked([&] {
            return offsets ? g_grouped_linear_f8(x_ptr, x_f8, x_row, w_ptr, w_f8, w_row, off_ptr, (int)E, (int)M, (int)N, (int)K, xs_ptr, xs_row, ws_ptr, y_ptr,
                                                 out_row, &ep, st)
                           : g_linear_f8(x_ptr, x_f8, x_row, w_ptr, w_f8, w_row, (int)M, (int)N, (int)K, xs_ptr, xs_row, ws_ptr, y_ptr, out_row, &ep, st);
        });
        if (status != HIKONV_OK) return nullptr;
        return result(a[9], made);
    });
}

// bind(name, address): the entry points of the library that is loaded.
PyObject *bind(PyObject *, PyObject *args) {
    const char *name;
    unsigned long long address;
    if (!PyArg_ParseTuple(args, "sK", &name, &address)) return nullptr;
    const std::string s(name);
    void *ptr = (void *)(uintptr_t)address;
    if (s == "hikonv_conv1d") g_conv1d = (decltype(g_conv1d))ptr;
    else if (s == "hikonv_conv1d_dense") g_conv1d_dense = (decltype(g_conv1d_dense))ptr;
    else if (s == "hikonv_conv2d") g_conv2d = (decltype(g_conv2d))ptr;
    else if (s == "hikonv_conv2d_dense") g_conv2d_dense = (decltype(g_conv2d_dense))ptr;
    else if (s == "hikonv_conv2d_workspace_bytes") g_workspace_bytes = (decltype(g_workspace_bytes))ptr;
    else if (s == "hikonv_pack") g_pack = (decltype(g_pack))ptr;
    else if (s == "hikonv_quantize_rows") g_quantize_rows = (decltype(g_quantize_rows))ptr;
    else if (s == "hikonv_linear") g_linear = (decltype(g_linear))ptr;
    else if (s == "hikonv_grouped_linear") g_grouped_linear = (decltype(g_grouped_linear))ptr;
    else if (s == "hikonv_linear_workspace_bytes") g_linear_workspace_bytes = (decltype(g_linear_workspace_bytes))ptr;
    else if (s == "hikonv_sort_by_expert") g_sort_by_expert = (decltype(g_sort_by_expert))ptr;
    else if (s == "hikonv_sort_by_expert_workspace_bytes") g_sort_workspace_bytes = (decltype(g_sort_workspace_bytes))ptr;
    else if (s == "hikonv_rows_to_experts") g_rows_to_experts = (decltype(g_rows_to_experts))ptr;
    else if (s == "hikonv_rows_from_experts") g_rows_from_experts = (decltype(g_rows_from_experts))ptr;
    else if (s == "hikonv_rows_from_experts_grad") g_rows_from_experts_grad = (decltype(g_rows_from_experts_grad))ptr;
    else if (s == "hikonv_zero_other_rows") g_zero_other_rows = (decltype(g_zero_other_rows))ptr;
    else if (s == "hikonv_quantize_blocks") g_quantize_blocks = (decltype(g_quantize_blocks))ptr;
    else if (s == "hikonv_linear_f8") g_linear_f8 = (decltype(g_linear_f8))ptr;
    else if (s == "hikonv_grouped_linear_f8") g_grouped_linear_f8 = (decltype(g_grouped_linear_f8))ptr;
    else {
        PyErr_Format(PyExc_ValueError, "no entry point %s", name);
        return nullptr;
    }
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"conv1d", (PyCFunction)(void (*)(void))conv1d, METH_FASTCALL, nullptr},
    {"conv1d_dense", (PyCFunction)(void (*)(void))conv1d_dense, METH_FASTCALL, nullptr},
    {"pack", (PyCFunction)(void (*)(void))pack, METH_FASTCALL, nullptr},
    {"conv2d", (PyCFunction)(void (*)(void))conv2d, METH_FASTCALL, nullptr},
    {"conv2d_dense", (PyCFunction)(void (*)(void))conv2d_dense, METH_FASTCALL, nullptr},
    {"quantize_rows", (PyCFunction)(void (*)(void))quantize_rows, METH_FASTCALL, nullptr},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, nullptr},
    {"sort_by_expert", (PyCFunction)(void (*)(void))sort_by_expert, METH_FASTCALL, nullptr},
    {"rows_to_experts", (PyCFunction)(void (*)(void))rows_to_experts, METH_FASTCALL, nullptr},
    {"rows_from_experts", (PyCFunction)(void (*)(void))rows_from_experts, METH_FASTCALL, nullptr},
    {"rows_from_experts_grad", (PyCFunction)(void (*)(void))rows_from_experts_grad, METH_FASTCALL, nullptr},
    {"quantize_blocks", (PyCFunction)(void (*)(void))quantize_blocks, METH_FASTCALL, nullptr},
    {"linear_f8", (PyCFunction)(void (*)(void))linear_f8, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fast", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fast(void) { return PyModule_Create(&module); }
