// The Python binding's native part: argument marshalling of the calls that are made per layer or per time step, whose kernels take a
// few microseconds.  ctypes and the reading of shapes and strides through Python objects cost 2.7 of the 5.4 us that such a call took on
// the host (the launch itself 2.7); here they cost 0.2.
//
// Every function returns the C entry point's status, or -1 for "not here": the caller then takes the general path in __init__.py, which
// handles whatever this one does not (no output given, other tensor classes, tensors without memory, numbers that are no integers) and
// raises the errors.  Nothing is kept between calls but the entry points' addresses.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include "qnn.h"

namespace {

typedef int (*PackSign)(const float *, int64_t, int64_t, int64_t, uint32_t *, int64_t, void *);
typedef int (*LinearQuant)(const float *, int64_t, int64_t, int64_t, float, int32_t, int32_t, int, uint32_t *, int64_t, int64_t, void *);
typedef int (*BinaryGemm)(const uint32_t *, int64_t, const uint32_t *, int64_t, int32_t *, int64_t, int64_t, int64_t, int64_t, void *);
typedef int (*BinaryGemmSign)(const uint32_t *, int64_t, const uint32_t *, int64_t, const int32_t *, const uint8_t *, uint32_t *, int64_t, int64_t,
                              int64_t, int64_t, int, void *);
typedef int (*BitplaneGemm)(const uint32_t *, int, const int32_t *, int, int64_t, int64_t, const uint32_t *, int, const int32_t *, int, int64_t, int64_t,
                            int32_t *, int64_t, int64_t, int64_t, int64_t, void *);
typedef int (*Conv2d)(const uint32_t *, int, const int32_t *, int, int64_t, int64_t, int64_t, int64_t, int64_t, const uint32_t *, int, const int32_t *,
                      int, int64_t, int64_t, int, int, int, int, int32_t *, void *);
typedef int (*RmsNormQuant)(const void *, int64_t, const void *, int64_t, int, const void *, int, float, int64_t, int64_t, void *, int64_t, int8_t *, int64_t, float *, void *);
typedef int (*RmsNormBackward)(const void *, int64_t, const void *, int64_t, const void *, int64_t, int, const void *, int, float, int64_t, int64_t, void *, int64_t, float *,
                               void *, size_t, void *);
typedef int (*SiluGateQuant)(const void *, int64_t, const void *, int64_t, int, int64_t, int64_t, int8_t *, int64_t, float *, void *);
typedef int (*SiluGateBackward)(const void *, int64_t, const void *, int64_t, const void *, int64_t, int, int64_t, int64_t, void *, int64_t, void *, int64_t, void *);
typedef int (*Int8Gemm)(const int8_t *, int64_t, const float *, const int8_t *, int64_t, const float *, const float *, void *, int64_t, int, int64_t, int64_t, int64_t, void *);
typedef int (*Int8Moe)(const int8_t *, int64_t, const float *, const float *, int64_t, int64_t, int, int, int64_t, int64_t, const int8_t *, int64_t, const float *,
                       const int8_t *, int64_t, const float *, void *, int64_t, int, void *, size_t, void *);
typedef decltype(&qnn_qk_norm_rotate) QkNormRotate;
typedef decltype(&qnn_qk_norm_rotate_backward) QkNormRotateBackward;
typedef decltype(&qnn_cache_append) CacheAppend;
typedef decltype(&qnn_cache_attention) CacheAttention;
typedef decltype(&qnn_rows_quant) RowsQuant;
enum { kPackSign, kLinearQuant, kBinaryGemm, kBinaryGemmSign, kBitplaneGemm, kConv2d, kRmsNormQuant, kRmsNormBackward, kSiluGateQuant, kSiluGateBackward, kInt8Gemm, kInt8Moe, kQkNormRotate, kQkNormRotateBackward,
       kCacheAppend, kCacheAttention, kRowsQuant, kEntries };
void *g_entry[kEntries];

constexpr int kMaxPlanes = 8;  // QNN_MAX_PLANES

PyObject *not_here() {
    PyErr_Clear();
    return PyLong_FromLong(-1);
}

// A plain tensor of this type with memory on a GPU (others have no address, or are not asked for it like this)
const at::Tensor *tensor(PyObject *o, at::ScalarType type, int64_t dims) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || t.scalar_type() != type || (dims >= 0 && t.dim() != dims)) return nullptr;
    return &t;
}
struct Rows {
    void *p;
    int64_t planes, rows, cols, ld, stride;
};
// [rows][cols], or [planes][rows][cols], with contiguous rows
bool rows_of(PyObject *o, at::ScalarType type, int64_t dims, Rows &r) {
    const at::Tensor *t = tensor(o, type, dims);
    if (!t) return false;
    const auto size = t->sizes(), step = t->strides();
    const int64_t at = dims - 2;
    r.planes = dims == 3 ? size[0] : 1, r.rows = size[at], r.cols = size[at + 1];
    if (r.cols > 1 && step[at + 1] != 1) return false;
    r.ld = r.rows > 1 ? step[at] : (r.cols > 1 ? r.cols : 1);
    r.stride = r.planes > 1 ? step[0] : 0;
    r.p = t->data_ptr();
    return true;
}
bool integer(PyObject *o, int64_t &v) {
    if (!PyLong_CheckExact(o)) return false;
    v = PyLong_AsLongLong(o);
    return !(v == -1 && PyErr_Occurred());
}
// The current stream's handle, from the function that __init__.py has for it (after everything else is known to be in order)
bool stream(PyObject *function, int64_t &v) {
    PyObject *const r = PyObject_CallNoArgs(function);
    if (!r) return false;
    const bool ok = integer(r, v);
    Py_DECREF(r);
    return ok;
}
bool integer32(PyObject *o, int32_t &v) {
    int64_t w;
    if (!integer(o, w) || w < INT32_MIN || w > INT32_MAX) return false;
    v = (int32_t)w;
    return true;
}
bool coefficients(PyObject *o, int64_t count, int32_t (&c)[kMaxPlanes]) {
    if (!(PyList_CheckExact(o) || PyTuple_CheckExact(o)) || count > kMaxPlanes || PySequence_Fast_GET_SIZE(o) != count) return false;
    for (int64_t i = 0; i < count; ++i)
        if (!integer32(PySequence_Fast_GET_ITEM(o, i), c[i])) return false;
    return true;
}
// Calls f, which returns a status, without the interpreter's lock
template <typename F>
PyObject *call(F f) {
    int status;
    Py_BEGIN_ALLOW_THREADS status = f();
    Py_END_ALLOW_THREADS return PyLong_FromLong(status);
}
void *stream_of(int64_t v) { return reinterpret_cast<void *>(v); }
template <typename T>
T *as(const Rows &r) {
    return static_cast<T *>(r.p);
}

// qnn_float_type of a type of numbers, -1 for others
int float_type(at::ScalarType t) { return t == at::kFloat ? 0 : t == at::kHalf ? 1 : t == at::kBFloat16 ? 2 : -1; }
// [rows][cols] of any of these types
bool floats_of(PyObject *o, Rows &r, int &type) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::ScalarType t = THPVariable_Unpack(o).scalar_type();
    type = float_type(t);
    return type >= 0 && rows_of(o, t, 2, r);
}
// ... of a given one and shape
bool shaped_like(PyObject *o, int type, int64_t rows, int64_t cols, Rows &r) {
    int t;
    return floats_of(o, r, t) && t == type && r.rows == rows && r.cols == cols;
}
bool codes_like(PyObject *o, int64_t rows, int64_t cols, Rows &r) { return rows_of(o, at::kChar, 2, r) && r.rows == rows && r.cols == cols; }
// dense [n]
bool vector_of(PyObject *o, at::ScalarType type, int64_t n, void *&p) {
    const at::Tensor *const t = tensor(o, type, 1);
    if (!t || t->size(0) != n || (n > 1 && t->stride(0) != 1)) return false;
    p = t->data_ptr();
    return true;
}
bool floats_vector(PyObject *o, int64_t n, void *&p, int &type) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::ScalarType t = THPVariable_Unpack(o).scalar_type();
    type = float_type(t);
    return type >= 0 && vector_of(o, t, n, p);
}

// x, out, stream
PyObject *pack_sign(PyObject *const *a) {
    Rows x, o;
    int64_t s;
    if (!rows_of(a[0], at::kFloat, 2, x) || !rows_of(a[1], at::kInt, 2, o) || !stream(a[2], s)) return not_here();
    return call([&] { return reinterpret_cast<PackSign>(g_entry[kPackSign])(as<float>(x), x.rows, x.cols, x.ld, as<uint32_t>(o), o.ld, stream_of(s)); });
}
// x, step, qmin, qmax, nbits, out, stream
PyObject *linear_quant_planes(PyObject *const *a) {
    Rows x, o;
    int32_t lo, hi, bits;
    int64_t s;
    if (!PyFloat_CheckExact(a[1]) || !rows_of(a[0], at::kFloat, 2, x) || !integer32(a[2], lo) || !integer32(a[3], hi) || !integer32(a[4], bits) ||
        !rows_of(a[5], at::kInt, 3, o) || o.planes != bits || !stream(a[6], s))
        return not_here();
    const float step = (float)PyFloat_AS_DOUBLE(a[1]);
    return call([&] { return reinterpret_cast<LinearQuant>(g_entry[kLinearQuant])(as<float>(x), x.rows, x.cols, x.ld, step, lo, hi, bits, as<uint32_t>(o), o.ld, o.stride, stream_of(s)); });
}
// A, W, K, out, stream
PyObject *binary_gemm(PyObject *const *a) {
    Rows A, W, c;
    int64_t K, s;
    if (!rows_of(a[0], at::kInt, 2, A) || !rows_of(a[1], at::kInt, 2, W) || !integer(a[2], K) || !rows_of(a[3], at::kInt, 2, c) || !stream(a[4], s))
        return not_here();
    return call([&] { return reinterpret_cast<BinaryGemm>(g_entry[kBinaryGemm])(as<uint32_t>(A), A.ld, as<uint32_t>(W), W.ld, as<int32_t>(c), c.ld, A.rows, W.rows, K, stream_of(s)); });
}
// A, W, K, T, flip, out, engine, stream
PyObject *binary_gemm_sign(PyObject *const *a) {
    Rows A, W, o;
    int64_t K, s;
    int32_t engine;
    const at::Tensor *T = tensor(a[3], at::kInt, -1), *flip = a[4] == Py_None ? nullptr : tensor(a[4], at::kByte, -1);
    if (!T || (a[4] != Py_None && !flip) || !rows_of(a[0], at::kInt, 2, A) || !rows_of(a[1], at::kInt, 2, W) || !integer(a[2], K) ||
        !rows_of(a[5], at::kInt, 2, o) || !integer32(a[6], engine) || !stream(a[7], s))
        return not_here();
    const int32_t *const t = static_cast<const int32_t *>(T->data_ptr());
    const uint8_t *const f = flip ? static_cast<const uint8_t *>(flip->data_ptr()) : nullptr;
    return call([&] {
        return reinterpret_cast<BinaryGemmSign>(g_entry[kBinaryGemmSign])(as<uint32_t>(A), A.ld, as<uint32_t>(W), W.ld, t, f, as<uint32_t>(o), o.ld, A.rows, W.rows, K, engine, stream_of(s));
    });
}
// A, coefA, modeA, W, coefW, modeW, K, out, stream
PyObject *bitplane_gemm(PyObject *const *a) {
    Rows A, W, c;
    int32_t ca[kMaxPlanes], cw[kMaxPlanes], ma, mw;
    int64_t K, s;
    if (!rows_of(a[0], at::kInt, 3, A) || !coefficients(a[1], A.planes, ca) || !integer32(a[2], ma) || !rows_of(a[3], at::kInt, 3, W) ||
        !coefficients(a[4], W.planes, cw) || !integer32(a[5], mw) || !integer(a[6], K) || !rows_of(a[7], at::kInt, 2, c) || !stream(a[8], s))
        return not_here();
    return call([&] {
        return reinterpret_cast<BitplaneGemm>(g_entry[kBitplaneGemm])(as<uint32_t>(A), (int)A.planes, ca, ma, A.ld, A.stride, as<uint32_t>(W), (int)W.planes, cw, mw, W.ld, W.stride,
                                                                      as<int32_t>(c), c.ld, A.rows, W.rows, K, stream_of(s));
    });
}
// A, coefA, modeA, Cin, W, coefW, modeW, pad, stride, out, stream
PyObject *bitplane_conv2d(PyObject *const *a) {
    const at::Tensor *A = tensor(a[0], at::kInt, 5), *W = tensor(a[4], at::kInt, 5), *out = tensor(a[9], at::kInt, 4);
    int32_t ca[kMaxPlanes], cw[kMaxPlanes], ma, mw, pad, step;
    int64_t cin, s;
    if (!A || !W || !out || !A->is_contiguous() || !W->is_contiguous() || !out->is_contiguous() || !coefficients(a[1], A->size(0), ca) || !integer32(a[2], ma) ||
        !integer(a[3], cin) || !coefficients(a[5], W->size(0), cw) || !integer32(a[6], mw) || !integer32(a[7], pad) || !integer32(a[8], step))
        return not_here();
    const int64_t B = A->size(1), H = A->size(2), Wd = A->size(3), Cw = A->size(4), N = W->size(1), KH = W->size(2), KW = W->size(3);
    if (cin < 1 || Cw != (cin + 31) / 32 || W->size(4) != Cw || step < 1 || H + 2 * (int64_t)pad < KH || Wd + 2 * (int64_t)pad < KW || KH > INT32_MAX || KW > INT32_MAX)
        return not_here();
    if (out->size(0) != B || out->size(1) != (H + 2 * (int64_t)pad - KH) / step + 1 || out->size(2) != (Wd + 2 * (int64_t)pad - KW) / step + 1 || out->size(3) != N || !stream(a[10], s)) return not_here();
    const int Pa = (int)A->size(0), Pb = (int)W->size(0);
    const int64_t sa = Pa > 1 ? A->stride(0) : 0, sw = Pb > 1 ? W->stride(0) : 0;
    const uint32_t *const pa = static_cast<const uint32_t *>(A->data_ptr()), *const pw = static_cast<const uint32_t *>(W->data_ptr());
    int32_t *const po = static_cast<int32_t *>(out->data_ptr());
    return call([&] {
        return reinterpret_cast<Conv2d>(g_entry[kConv2d])(pa, Pa, ca, ma, sa, B, H, Wd, cin, pw, Pb, cw, mw, sw, N, (int)KH, (int)KW, pad, step, po, stream_of(s));
    });
}

// x, gamma, eps, residual, codes, scale, total, stream
PyObject *rms_norm_quant(PyObject *const *a) {
    Rows x, res = {}, c, total = {};
    void *gamma, *scale;
    int type, gamma_type;
    int64_t s;
    if (!PyFloat_CheckExact(a[2]) || !floats_of(a[0], x, type) || !floats_vector(a[1], x.cols, gamma, gamma_type) ||
        (a[3] != Py_None && !shaped_like(a[3], type, x.rows, x.cols, res)) || !codes_like(a[4], x.rows, x.cols, c) || !vector_of(a[5], at::kFloat, x.rows, scale) ||
        (a[6] != Py_None && !shaped_like(a[6], type, x.rows, x.cols, total)) || !stream(a[7], s))
        return not_here();
    const float eps = (float)PyFloat_AS_DOUBLE(a[2]);
    return call([&] {
        return reinterpret_cast<RmsNormQuant>(g_entry[kRmsNormQuant])(x.p, x.ld, res.p, res.ld, type, gamma, gamma_type, eps, x.rows, x.cols, total.p, total.ld, as<int8_t>(c), c.ld,
                                                                      static_cast<float *>(scale), stream_of(s));
    });
}
// grad, h, gamma, eps, grad_sum, grad_h, grad_gamma, workspace, stream
PyObject *rms_norm_backward(PyObject *const *a) {
    Rows g, h, z = {}, o;
    void *gamma, *grad_gamma;
    int type, gamma_type;
    int64_t s;
    const at::Tensor *const ws = tensor(a[7], at::kByte, 1);
    if (!ws || !ws->is_contiguous() || !PyFloat_CheckExact(a[3]) || !floats_of(a[1], h, type) || !shaped_like(a[0], type, h.rows, h.cols, g) ||
        !floats_vector(a[2], h.cols, gamma, gamma_type) || (a[4] != Py_None && !shaped_like(a[4], type, h.rows, h.cols, z)) ||
        !shaped_like(a[5], type, h.rows, h.cols, o) || !vector_of(a[6], at::kFloat, h.cols, grad_gamma) || !stream(a[8], s))
        return not_here();
    const float eps = (float)PyFloat_AS_DOUBLE(a[3]);
    void *const w = ws->data_ptr();
    const size_t bytes = (size_t)ws->numel();
    return call([&] {
        return reinterpret_cast<RmsNormBackward>(g_entry[kRmsNormBackward])(g.p, g.ld, h.p, h.ld, z.p, z.ld, type, gamma, gamma_type, eps, h.rows, h.cols, o.p, o.ld,
                                                                            static_cast<float *>(grad_gamma), w, bytes, stream_of(s));
    });
}
// gate, up, codes, scale, stream
PyObject *silu_gate_quant(PyObject *const *a) {
    Rows g, u, c;
    void *scale;
    int type;
    int64_t s;
    if (!floats_of(a[0], g, type) || !shaped_like(a[1], type, g.rows, g.cols, u) || !codes_like(a[2], g.rows, g.cols, c) || !vector_of(a[3], at::kFloat, g.rows, scale) ||
        !stream(a[4], s))
        return not_here();
    return call([&] {
        return reinterpret_cast<SiluGateQuant>(g_entry[kSiluGateQuant])(g.p, g.ld, u.p, u.ld, type, g.rows, g.cols, as<int8_t>(c), c.ld, static_cast<float *>(scale), stream_of(s));
    });
}
// grad, gate, up, grad_gate, grad_up, stream
PyObject *silu_gate_backward(PyObject *const *a) {
    Rows d, g, u, dg, du;
    int type;
    int64_t s;
    if (!floats_of(a[1], g, type) || !shaped_like(a[0], type, g.rows, g.cols, d) || !shaped_like(a[2], type, g.rows, g.cols, u) || !shaped_like(a[3], type, g.rows, g.cols, dg) ||
        !shaped_like(a[4], type, g.rows, g.cols, du) || !stream(a[5], s))
        return not_here();
    return call([&] {
        return reinterpret_cast<SiluGateBackward>(g_entry[kSiluGateBackward])(d.p, d.ld, g.p, g.ld, u.p, u.ld, type, g.rows, g.cols, dg.p, dg.ld, du.p, du.ld, stream_of(s));
    });
}
// A, scaleA, W, scaleW, bias, out, stream
PyObject *int8_gemm(PyObject *const *a) {
    Rows A, W, o;
    void *sa, *sw, *bias = nullptr;
    int type;
    int64_t s;
    if (!rows_of(a[0], at::kChar, 2, A) || !rows_of(a[2], at::kChar, 2, W) || A.cols != W.cols || !vector_of(a[1], at::kFloat, A.rows, sa) ||
        !vector_of(a[3], at::kFloat, W.rows, sw) || (a[4] != Py_None && !vector_of(a[4], at::kFloat, W.rows, bias)) || !floats_of(a[5], o, type) || o.rows != A.rows ||
        o.cols != W.rows || !stream(a[6], s))
        return not_here();
    return call([&] {
        return reinterpret_cast<Int8Gemm>(g_entry[kInt8Gemm])(as<int8_t>(A), A.ld, static_cast<float *>(sa), as<int8_t>(W), W.ld, static_cast<float *>(sw),
                                                              static_cast<float *>(bias), o.p, o.ld, type, A.rows, W.rows, A.cols, stream_of(s));
    });
}
// x, scale_x, logits, top, W1, scale1, W2, scale2, out, workspace, stream
PyObject *int8_moe(PyObject *const *a) {
    Rows x, l, o;
    void *sx;
    int32_t top;
    int type, type_l;
    int64_t s;
    const at::Tensor *const W1 = tensor(a[4], at::kChar, 3), *const s1 = tensor(a[5], at::kFloat, 2), *const W2 = tensor(a[6], at::kChar, 3), *const s2 = tensor(a[7], at::kFloat, 2),
                            *const ws = tensor(a[9], at::kByte, 1);
    // (dense weights: others go the general way)
    if (!W1 || !s1 || !W2 || !s2 || !ws || !W1->is_contiguous() || !W2->is_contiguous() || !s1->is_contiguous() || !s2->is_contiguous() || !ws->is_contiguous()) return not_here();
    const int64_t E = W1->size(0), F = W2->size(2);
    if (!rows_of(a[0], at::kChar, 2, x) || !vector_of(a[1], at::kFloat, x.rows, sx) || !floats_of(a[2], l, type_l) || type_l != 0 || l.rows != x.rows || l.cols != E ||
        E > INT32_MAX || !integer32(a[3], top) || W1->size(1) != 2 * F || W1->size(2) != x.cols || W2->size(0) != E || W2->size(1) != x.cols || s1->size(0) != E ||
        s1->size(1) != 2 * F || s2->size(0) != E || s2->size(1) != x.cols || !floats_of(a[8], o, type) || o.rows != x.rows || o.cols != x.cols || !stream(a[10], s))
        return not_here();
    const int8_t *const w1 = static_cast<const int8_t *>(W1->data_ptr()), *const w2 = static_cast<const int8_t *>(W2->data_ptr());
    const float *const f1 = static_cast<const float *>(s1->data_ptr()), *const f2 = static_cast<const float *>(s2->data_ptr());
    void *const w = ws->data_ptr();
    const size_t bytes = (size_t)ws->numel();
    return call([&] {
        return reinterpret_cast<Int8Moe>(g_entry[kInt8Moe])(as<int8_t>(x), x.ld, static_cast<float *>(sx), as<float>(l), l.ld, x.rows, (int)E, top, x.cols, F, w1, x.cols, f1, w2, F, f2,
                                                            o.p, o.ld, type, w, bytes, stream_of(s));
    });
}

// A plain tensor on the device that the call is going to run on
struct Here {
    int64_t device = -1;
    bool set(PyObject *function) { return stream(function, device); }  // (any function without arguments that gives a whole number)
    const at::Tensor *operator()(PyObject *o, at::ScalarType type, int64_t dims) const {
        const at::Tensor *const t = tensor(o, type, dims);
        return t && t->get_device() == device ? t : nullptr;
    }
    bool vector(PyObject *o, at::ScalarType type, int64_t n, void *&p) const {
        const at::Tensor *const t = (*this)(o, type, 1);
        if (!t || t->size(0) != n || (n > 1 && t->stride(0) != 1)) return false;
        p = t->data_ptr();
        return true;
    }
};
// [tokens][heads][D] with contiguous heads
struct Heads {
    void *p = nullptr;
    int64_t tokens = 0, heads = 0, D = 0, ld = 0, step = 0;
};
bool heads_of(const Here &here, PyObject *o, at::ScalarType type, Heads &h) {
    const at::Tensor *const t = here(o, type, 3);
    if (!t) return false;
    const auto size = t->sizes(), step = t->strides();
    h.tokens = size[0], h.heads = size[1], h.D = size[2];
    if (h.D > 1 && step[2] != 1) return false;
    h.step = h.heads > 1 ? step[1] : h.D;
    h.ld = h.tokens > 1 ? step[0] : h.heads * h.step;
    h.p = t->data_ptr();
    return true;
}
bool heads_like(const Here &here, PyObject *o, at::ScalarType type, const Heads &like, Heads &h) {
    return heads_of(here, o, type, h) && h.tokens == like.tokens && h.heads == like.heads && h.D == like.D;
}
bool scalar_type(PyObject *o, at::ScalarType &t) {
    if (!THPVariable_CheckExact(o)) return false;
    t = THPVariable_Unpack(o).scalar_type();
    return float_type(t) >= 0;
}
// gamma_q, gamma_k: none, or of one type
bool gammas_of(const Here &here, PyObject *q, PyObject *k, int64_t D, void *&pq, void *&pk, int &kind) {
    at::ScalarType tq = at::kFloat, tk = at::kFloat;
    pq = pk = nullptr;
    if (q != Py_None && (!scalar_type(q, tq) || !here.vector(q, tq, D, pq))) return false;
    if (k != Py_None && (!scalar_type(k, tk) || !here.vector(k, tk, D, pk))) return false;
    if (q != Py_None && k != Py_None && tq != tk) return false;
    kind = float_type(q != Py_None ? tq : tk);
    return true;
}
// positions, freq, axis, neighbours
bool rotation_of(const Here &here, PyObject *const *a, int64_t tokens, qnn_rotation &r) {
    r = {};
    if (a[1] == Py_None) return true;
    const at::Tensor *p = here(a[0], at::kInt, 2);
    const at::Tensor *const f = here(a[1], at::kDouble, 1);
    if (!p || !f || p->size(1) != tokens || (tokens > 1 && p->stride(1) != 1) || p->size(0) > INT32_MAX || f->size(0) > INT32_MAX ||
        (f->size(0) > 1 && f->stride(0) != 1) || !PyBool_Check(a[3]))
        return false;
    r.positions = static_cast<const int32_t *>(p->data_ptr()), r.freq = static_cast<const double *>(f->data_ptr());
    r.axes = (int32_t)p->size(0), r.pairs = (int32_t)f->size(0), r.neighbours = a[3] == Py_True;
    r.ld_positions = r.axes > 1 ? p->stride(0) : (tokens > 1 ? tokens : 1);
    if (a[2] != Py_None) {
        void *axis;
        if (!here.vector(a[2], at::kInt, f->size(0), axis)) return false;
        r.axis = static_cast<const int32_t *>(axis);
    }
    return true;
}
// cache, table, starts, lengths
bool cache_of(const Here &here, PyObject *const *a, qnn_paged_cache &c) {
    if (!PyTuple_CheckExact(a[0]) || PyTuple_GET_SIZE(a[0]) != 4) return false;
    const at::Tensor *const k = here(PyTuple_GET_ITEM(a[0], 0), at::kChar, 4), *const ks = here(PyTuple_GET_ITEM(a[0], 1), at::kFloat, 3),
                            *const v = here(PyTuple_GET_ITEM(a[0], 2), at::kChar, 4), *const vs = here(PyTuple_GET_ITEM(a[0], 3), at::kFloat, 3),
                            *const t = here(a[1], at::kInt, 2);
    if (!k || !ks || !v || !vs || !t || !k->is_contiguous() || !v->is_contiguous() || !ks->is_contiguous() || !vs->is_contiguous() || v->sizes() != k->sizes() ||
        ks->sizes() != k->sizes().slice(0, 3) || vs->sizes() != ks->sizes() || (t->size(1) > 1 && t->stride(1) != 1))
        return false;
    void *starts, *lengths;
    c.sequences = t->size(0), c.width = t->size(1);
    if (!here.vector(a[2], at::kInt, c.sequences + 1, starts) || !here.vector(a[3], at::kInt, c.sequences, lengths)) return false;
    c.ld_table = c.sequences > 1 ? t->stride(0) : (c.width > 1 ? c.width : 1);
    c.k = static_cast<int8_t *>(k->data_ptr()), c.v = static_cast<int8_t *>(v->data_ptr());
    c.k_scale = static_cast<float *>(ks->data_ptr()), c.v_scale = static_cast<float *>(vs->data_ptr());
    c.pages = k->size(0), c.heads = k->size(1), c.page = k->size(2), c.D = k->size(3);
    c.table = static_cast<const int32_t *>(t->data_ptr()), c.starts = static_cast<const int32_t *>(starts), c.lengths = static_cast<const int32_t *>(lengths);
    return true;
}

// q, k, gamma_q, gamma_k, eps, positions, freq, axis, neighbours, q_out, k_out, device, stream
PyObject *qk_norm_rotate(PyObject *const *a) {
    Here here;
    Heads q, k, qo, ko;
    at::ScalarType t;
    void *gq, *gk;
    int gamma_kind;
    qnn_rotation r;
    int64_t s;
    if (!here.set(a[11]) || !PyFloat_CheckExact(a[4]) || !scalar_type(a[0], t) || !heads_of(here, a[0], t, q) || !heads_of(here, a[1], t, k) || k.tokens != q.tokens ||
        k.D != q.D || !gammas_of(here, a[2], a[3], q.D, gq, gk, gamma_kind) || !rotation_of(here, a + 5, q.tokens, r) || !heads_like(here, a[9], t, q, qo) ||
        !heads_like(here, a[10], t, k, ko) || !stream(a[12], s))
        return not_here();
    const float eps = (float)PyFloat_AS_DOUBLE(a[4]);
    return call([&] {
        return reinterpret_cast<QkNormRotate>(g_entry[kQkNormRotate])(q.p, q.ld, q.step, q.heads, k.p, k.ld, k.step, k.heads, float_type(t), gq, gk, gamma_kind, eps, &r,
                                                                      q.tokens, q.D, qo.p, qo.ld, qo.step, ko.p, ko.ld, ko.step, stream_of(s));
    });
}
// grad_q, grad_k, q, k, gamma_q, gamma_k, eps, positions, freq, axis, neighbours, out_q, out_k, grad_gamma_q, grad_gamma_k, workspace, device, stream
PyObject *qk_norm_rotate_backward(PyObject *const *a) {
    Here here;
    Heads dq, dk, q, k, qo, ko;
    at::ScalarType t;
    void *gq, *gk, *sq = nullptr, *sk = nullptr;
    int gamma_kind;
    qnn_rotation r;
    int64_t s;
    if (!here.set(a[16]) || !PyFloat_CheckExact(a[6]) || !scalar_type(a[2], t) || !heads_of(here, a[2], t, q) || !heads_of(here, a[3], t, k) || k.tokens != q.tokens ||
        k.D != q.D || !heads_like(here, a[0], t, q, dq) || !heads_like(here, a[1], t, k, dk) || !gammas_of(here, a[4], a[5], q.D, gq, gk, gamma_kind) ||
        !rotation_of(here, a + 7, q.tokens, r) || !heads_like(here, a[11], t, q, qo) || !heads_like(here, a[12], t, k, ko))
        return not_here();
    const at::Tensor *const ws = here(a[15], at::kByte, 1);
    if (!ws || !ws->is_contiguous() || (gq && !here.vector(a[13], at::kFloat, q.D, sq)) || (gk && !here.vector(a[14], at::kFloat, q.D, sk)) || !stream(a[17], s)) return not_here();
    const float eps = (float)PyFloat_AS_DOUBLE(a[6]);
    void *const w = ws->data_ptr();
    const size_t bytes = (size_t)ws->numel();
    return call([&] {
        return reinterpret_cast<QkNormRotateBackward>(g_entry[kQkNormRotateBackward])(dq.p, dq.ld, dq.step, dk.p, dk.ld, dk.step, q.p, q.ld, q.step, q.heads, k.p, k.ld, k.step, k.heads,
                                                                                      float_type(t), gq, gk, gamma_kind, eps, &r, q.tokens, q.D, qo.p, qo.ld, qo.step, ko.p, ko.ld,
                                                                                      ko.step, static_cast<float *>(sq), static_cast<float *>(sk), w, bytes, stream_of(s));
    });
}
// cache, table, starts, lengths, k, v, gamma_k, eps, positions, freq, axis, neighbours, q, gamma_q, q_out, device, stream
PyObject *cache_append(PyObject *const *a) {
    Here here;
    qnn_paged_cache c;
    Heads q, k, v, qo;
    at::ScalarType t;
    void *gq, *gk;
    int gamma_kind;
    qnn_rotation r;
    int64_t s;
    if (!here.set(a[15]) || !PyFloat_CheckExact(a[7]) || !cache_of(here, a, c) || !scalar_type(a[4], t) || !heads_of(here, a[4], t, k) || k.heads != c.heads || k.D != c.D ||
        !heads_like(here, a[5], t, k, v) || !gammas_of(here, a[13], a[6], k.D, gq, gk, gamma_kind) || !rotation_of(here, a + 8, k.tokens, r) ||
        (a[12] != Py_None && (!heads_of(here, a[12], t, q) || q.tokens != k.tokens || q.D != k.D || !heads_like(here, a[14], t, q, qo))) || !stream(a[16], s))
        return not_here();
    const float eps = (float)PyFloat_AS_DOUBLE(a[7]);
    return call([&] {
        return reinterpret_cast<CacheAppend>(g_entry[kCacheAppend])(&c, q.p, q.ld, q.step, q.heads, k.p, k.ld, k.step, v.p, v.ld, v.step, float_type(t), gq, gk, gamma_kind, eps, &r,
                                                                    k.tokens, qo.p, qo.ld, qo.step, stream_of(s));
    });
}
// q, cache, table, starts, lengths, scale, cap, slopes, tree, most_new, longest, out, workspace, device, stream
PyObject *cache_attention(PyObject *const *a) {
    Here here;
    qnn_paged_cache c;
    Heads q, o;
    at::ScalarType t;
    void *slopes = nullptr, *tree = nullptr;
    int64_t most_new, longest, s;
    if (!here.set(a[13]) || !PyFloat_CheckExact(a[5]) || !PyFloat_CheckExact(a[6]) || !cache_of(here, a + 1, c) || !scalar_type(a[0], t) || !heads_of(here, a[0], t, q) || q.D != c.D ||
        (a[7] != Py_None && !here.vector(a[7], at::kFloat, q.heads, slopes)) || (a[8] != Py_None && !here.vector(a[8], at::kLong, q.tokens, tree)) || !integer(a[9], most_new) ||
        !integer(a[10], longest) || !heads_like(here, a[11], t, q, o))
        return not_here();
    const at::Tensor *const ws = here(a[12], at::kByte, 1);
    if (!ws || !ws->is_contiguous() || !stream(a[14], s)) return not_here();
    const float scale = (float)PyFloat_AS_DOUBLE(a[5]), cap = (float)PyFloat_AS_DOUBLE(a[6]);
    void *const w = ws->data_ptr();
    const size_t bytes = (size_t)ws->numel();
    return call([&] {
        return reinterpret_cast<CacheAttention>(g_entry[kCacheAttention])(&c, q.p, q.ld, q.step, q.heads, float_type(t), scale, cap, static_cast<const float *>(slopes),
                                                                          static_cast<const uint64_t *>(tree), q.tokens, most_new, longest, o.p, o.ld, o.step, w, bytes, stream_of(s));
    });
}
// x, codes, scale, device, stream
PyObject *rows_quant(PyObject *const *a) {
    Here here;
    Rows x, c;
    void *scale;
    int type;
    int64_t s;
    if (!here.set(a[3]) || !floats_of(a[0], x, type) || THPVariable_Unpack(a[0]).get_device() != here.device || !here(a[1], at::kChar, 2) || !codes_like(a[1], x.rows, x.cols, c) ||
        !here.vector(a[2], at::kFloat, x.rows, scale) || !stream(a[4], s))
        return not_here();
    return call([&] { return reinterpret_cast<RowsQuant>(g_entry[kRowsQuant])(x.p, x.ld, type, x.rows, x.cols, as<int8_t>(c), c.ld, static_cast<float *>(scale), stream_of(s)); });
}

// (C++ errors, of a tensor that has no memory for instance, are the general path's)
template <PyObject *(*kCall)(PyObject *const *), Py_ssize_t kArgs, int kEntry>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != kArgs || !g_entry[kEntry]) return not_here();
    try {
        return kCall(args);
    } catch (...) {
        return not_here();
    }
}
// The addresses of the entry points, in the order of the enumeration above
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n) {
    for (Py_ssize_t i = 0; i < n && i < kEntries; ++i) {
        g_entry[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    Py_RETURN_NONE;
}

template <typename F>
PyCFunction function(F f) {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}
PyMethodDef kMethods[] = {
    {"bind", function(bind), METH_FASTCALL, nullptr},
    {"pack_sign", function(entry<pack_sign, 3, kPackSign>), METH_FASTCALL, nullptr},
    {"linear_quant_planes", function(entry<linear_quant_planes, 7, kLinearQuant>), METH_FASTCALL, nullptr},
    {"binary_gemm", function(entry<binary_gemm, 5, kBinaryGemm>), METH_FASTCALL, nullptr},
    {"binary_gemm_sign", function(entry<binary_gemm_sign, 8, kBinaryGemmSign>), METH_FASTCALL, nullptr},
    {"bitplane_gemm", function(entry<bitplane_gemm, 9, kBitplaneGemm>), METH_FASTCALL, nullptr},
    {"bitplane_conv2d", function(entry<bitplane_conv2d, 11, kConv2d>), METH_FASTCALL, nullptr},
    {"rms_norm_quant", function(entry<rms_norm_quant, 8, kRmsNormQuant>), METH_FASTCALL, nullptr},
    {"rms_norm_backward", function(entry<rms_norm_backward, 9, kRmsNormBackward>), METH_FASTCALL, nullptr},
    {"silu_gate_quant", function(entry<silu_gate_quant, 5, kSiluGateQuant>), METH_FASTCALL, nullptr},
    {"silu_gate_backward", function(entry<silu_gate_backward, 6, kSiluGateBackward>), METH_FASTCALL, nullptr},
    {"int8_gemm", function(entry<int8_gemm, 7, kInt8Gemm>), METH_FASTCALL, nullptr},
    {"int8_moe", function(entry<int8_moe, 11, kInt8Moe>), METH_FASTCALL, nullptr},
    {"qk_norm_rotate", function(entry<qk_norm_rotate, 13, kQkNormRotate>), METH_FASTCALL, nullptr},
    {"qk_norm_rotate_backward", function(entry<qk_norm_rotate_backward, 18, kQkNormRotateBackward>), METH_FASTCALL, nullptr},
    {"cache_append", function(entry<cache_append, 17, kCacheAppend>), METH_FASTCALL, nullptr},
    {"cache_attention", function(entry<cache_attention, 15, kCacheAttention>), METH_FASTCALL, nullptr},
    {"rows_quant", function(entry<rows_quant, 5, kRowsQuant>), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// (BUILT_FOR: the torch and Python whose headers this was compiled with; with others, whose classes may be laid out differently, it is not used)
PyMODINIT_FUNC PyInit__native() {
    PyObject *const m = PyModule_Create(&kModule);
    if (m && PyModule_AddStringConstant(m, "BUILT_FOR", QNN_BUILT_FOR) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
