// The dense operators' calls from Python whose arguments are as the library takes
// them: CUDA tensors on the current device, rows contiguous, types and sizes
// that fit.  Each checks that, makes the outputs and the working memory with
// torch's allocator, and makes the call on the current stream.  For any other
// arguments it returns NotImplemented, and dense.py says what is wrong with
// them or copies what has to be; a status other than MLKV_OK comes back as an int.
//
// Bound by the host: a small call is nothing but this.  (Layer norm of 416 rows of 128: 13.6 us a
// call through the checks of dense.py, 4.6 through these; log probabilities of a row of 131,072: 25, 11.3.)
#include <Python.h>
#include <dlfcn.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <limits>
#include <vector>

#include "mlkv_dense.h"

namespace {

struct Library {
    decltype(&mlkv_layer_norm) layer_norm;
    decltype(&mlkv_layer_norm_backward) layer_norm_backward;
    decltype(&mlkv_layer_norm_backward_workspace) layer_norm_backward_workspace;
    decltype(&mlkv_linear) linear;
    decltype(&mlkv_linear_workspace) linear_workspace;
    decltype(&mlkv_linear_backward) linear_backward;
    decltype(&mlkv_linear_backward_workspace) linear_backward_workspace;
    decltype(&mlkv_token_logprobs) token_logprobs;
    decltype(&mlkv_token_logprobs_workspace) token_logprobs_workspace;
    decltype(&mlkv_token_logprobs_backward) token_logprobs_backward;
    decltype(&mlkv_gated_linear) gated_linear;
    decltype(&mlkv_gated_linear_workspace) gated_linear_workspace;
    decltype(&mlkv_gated_linear_backward) gated_linear_backward;
    decltype(&mlkv_gated_linear_backward_workspace) gated_linear_backward_workspace;
    decltype(&mlkv_linear_cross_entropy) linear_cross_entropy;
    decltype(&mlkv_linear_cross_entropy_workspace) linear_cross_entropy_workspace;
    decltype(&mlkv_linear_cross_entropy_backward) linear_cross_entropy_backward;
    decltype(&mlkv_linear_cross_entropy_backward_workspace) linear_cross_entropy_backward_workspace;
    decltype(&mlkv_adamw) adamw;
} lib = {};

constexpr auto kFloat = at::kFloat;

int type_of(at::ScalarType t) {
    return t == at::kFloat ? MLKV_TYPE_FLOAT : t == at::kBFloat16 ? MLKV_TYPE_BFLOAT : t == at::kHalf ? MLKV_TYPE_HALF : -1;
}
at::ScalarType scalar_of(int type) { return type == MLKV_TYPE_FLOAT ? at::kFloat : type == MLKV_TYPE_BFLOAT ? at::kBFloat16 : at::kHalf; }

struct Mat {
    void* p = nullptr;
    int64_t rows = 0, cols = 0, stride = 0;
    at::ScalarType scalar = at::kFloat;
    int type = -1;
    c10::Device device = c10::Device(c10::kCPU);
    bool read(PyObject* o) {
        if (!THPVariable_Check(o)) return false;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.dim() != 2) return false;
        scalar = t.scalar_type();
        type = type_of(scalar);
        rows = t.size(0);
        cols = t.size(1);
        stride = rows > 1 ? t.stride(0) : cols;
        if (type < 0 || stride < cols || (cols > 1 && t.stride(1) != 1)) return false;
        p = t.data_ptr();
        device = t.device();
        return true;
    }
    bool read(PyObject* o, const Mat& like, int64_t r, int64_t c) { return read(o) && rows == r && cols == c && device == like.device; }
};
bool vector_of(PyObject* o, const Mat& like, int64_t n, at::ScalarType scalar, void** p) {
    if (!THPVariable_Check(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || t.dim() != 1 || t.size(0) != n || t.device() != like.device || t.scalar_type() != scalar ||
        (n > 1 && t.stride(0) != 1))
        return false;
    *p = t.data_ptr();
    return true;
}
// (of any of the operators' types)
bool vector_of(PyObject* o, const Mat& like, int64_t n, void** p, at::ScalarType* scalar) {
    if (!THPVariable_Check(o)) return false;
    *scalar = THPVariable_Unpack(o).scalar_type();
    return type_of(*scalar) >= 0 && vector_of(o, like, n, *scalar, p);
}
bool here(const Mat& m) { return c10::cuda::current_device() == m.device.index(); }
void* stream_of(const Mat& m) { return c10::cuda::getCurrentCUDAStream(m.device.index()).stream(); }
at::Tensor make(const Mat& like, at::IntArrayRef size, at::ScalarType scalar) {
    return at::Tensor(at::detail::empty_cuda(size, scalar, like.device, std::nullopt));
}
struct Workspace {
    at::Tensor t;
    void* p = nullptr;
    Workspace(const Mat& like, int64_t bytes) {
        if (bytes > 0) {
            t = make(like, {bytes}, at::kByte);
            p = t.data_ptr();
        }
    }
};
PyObject* pass() { Py_RETURN_NOTIMPLEMENTED; }
// An error that Python has been told of already.
struct Told {};
bool truth(PyObject* o) {
    if (o == Py_True || o == Py_False) return o == Py_True;
    const int r = PyObject_IsTrue(o);
    if (r < 0) throw Told{};
    return r != 0;
}
PyObject* given(const at::Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
template <int N>
PyObject* tuple_of(const at::Tensor (&t)[N]) {
    PyObject* r = PyTuple_New(N);
    for (int i = 0; r && i < N; ++i) {
        PyObject* o = given(t[i]);
        if (!o) {
            Py_DECREF(r);
            return nullptr;
        }
        PyTuple_SET_ITEM(r, i, o);
    }
    return r;
}
void* at_of(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
// A C++ exception (of torch's allocator: out of memory; of a flag without a truth) as a Python one.
template <class F>
PyObject* guarded(F f) {
    try {
        return f();
    } catch (const c10::OutOfMemoryError&) {
        return pass();  // the call in Python meets the same, and raises torch's error
    } catch (const Told&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// x, weight, bias, eps, out_type (-1: x's), save_stats
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Mat x;
        if (n != 6 || !x.read(a[0]) || !here(x) || !PyFloat_Check(a[3])) return pass();
        const int asked = (int)PyLong_AsLong(a[4]), out = asked == -1 ? x.type : asked;
        if (out < 0 || (out != x.type && x.type != MLKV_TYPE_FLOAT)) return pass();
        void *w = nullptr, *b = nullptr;
        at::ScalarType kind = kFloat;
        if (a[1] != Py_None && !vector_of(a[1], x, x.cols, &w, &kind)) return pass();
        if (a[2] != Py_None && !(a[1] != Py_None ? vector_of(a[2], x, x.cols, kind, &b) : vector_of(a[2], x, x.cols, &b, &kind))) return pass();
        const bool save = truth(a[5]);
        const at::Tensor r[2] = {make(x, {x.rows, x.cols}, scalar_of(out)), save ? make(x, {x.rows, 2}, kFloat) : at::Tensor()};
        const int rc = lib.layer_norm(x.p, x.stride, x.type, x.rows, x.cols, w, b, type_of(kind), (float)PyFloat_AS_DOUBLE(a[3]), r[0].data_ptr(), x.cols,
                                      out, (float*)at_of(r[1]), stream_of(x));
        if (rc != MLKV_OK) return PyLong_FromLong(rc);
        return save ? tuple_of(r) : given(r[0]);
    });
}

// dy, x, weight, stats, bias
PyObject* layer_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Mat x, dy, stats;
        if (n != 5 || !x.read(a[1]) || !here(x) || !dy.read(a[0], x, x.rows, x.cols) || !stats.read(a[3], x, x.rows, 2)) return pass();
        if ((dy.type != x.type && x.type != MLKV_TYPE_FLOAT) || stats.type != MLKV_TYPE_FLOAT || stats.stride != 2) return pass();
        void* w = nullptr;
        at::ScalarType kind = kFloat;
        const bool weight = a[2] != Py_None, bias = truth(a[4]);
        if (weight && !vector_of(a[2], x, x.cols, &w, &kind)) return pass();
        const int64_t bytes = lib.layer_norm_backward_workspace(x.rows, x.cols);
        if (bytes < 0) return pass();
        const at::Tensor r[3] = {make(x, {x.rows, x.cols}, x.scalar), weight ? make(x, {x.cols}, kind) : at::Tensor(),
                                 bias ? make(x, {x.cols}, kind) : at::Tensor()};
        const Workspace ws(x, bytes);
        const int rc = lib.layer_norm_backward(dy.p, dy.stride, dy.type, x.p, x.stride, x.type, x.rows, x.cols, w, type_of(kind), (const float*)stats.p,
                                               r[0].data_ptr(), x.cols, at_of(r[1]), at_of(r[2]), ws.p, bytes, stream_of(x));
        return rc != MLKV_OK ? PyLong_FromLong(rc) : tuple_of(r);
    });
}

// x [m][k] and weight [n][k], both of one 16-bit type
bool operands(PyObject* xo, PyObject* wo, PyObject* act, Mat& x, mlkv_linear_args& g) {
    Mat w;
    if (!x.read(xo) || !here(x) || !w.read(wo) || w.device != x.device || w.type != x.type || x.type == MLKV_TYPE_FLOAT || w.cols != x.cols) return false;
    g = mlkv_linear_args{};
    g.m = x.rows; g.n = w.rows; g.k = x.cols;
    g.d_x = x.p; g.x_stride = x.stride; g.d_weight = w.p; g.weight_stride = w.stride;
    g.type = x.type;
    g.activation = (int32_t)PyLong_AsLong(act);
    return g.activation >= MLKV_ACT_NONE;
}

// x, weight, bias, activation, residual, save_pre
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Mat x, res;
        mlkv_linear_args g;
        if (n != 6 || !operands(a[0], a[1], a[3], x, g)) return pass();
        if (a[2] != Py_None && !vector_of(a[2], x, g.n, x.scalar, const_cast<void**>(&g.d_bias))) return pass();
        if (a[4] != Py_None) {
            if (!res.read(a[4], x, g.m, g.n) || res.type != x.type) return pass();
            g.d_residual = res.p; g.residual_stride = res.stride;
        }
        const bool save = truth(a[5]);
        const at::Tensor r[2] = {make(x, {g.m, g.n}, x.scalar), save && g.activation != MLKV_ACT_NONE ? make(x, {g.m, g.n}, x.scalar) : at::Tensor()};
        g.d_y = r[0].data_ptr(); g.y_stride = g.n;
        g.d_pre = at_of(r[1]); g.pre_stride = g.n;
        g.workspace_bytes = lib.linear_workspace(&g);
        const Workspace ws(x, g.workspace_bytes);
        g.d_workspace = ws.p;
        const int rc = lib.linear(&g, stream_of(x));
        if (rc != MLKV_OK) return PyLong_FromLong(rc);
        return save ? tuple_of(r) : given(r[0]);
    });
}

// dy, x, weight, pre, activation, bias, want_dx, want_dweight
PyObject* linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Mat x, dy, pre;
        mlkv_linear_args g;
        if (n != 8 || !operands(a[1], a[2], a[4], x, g) || !dy.read(a[0], x, g.m, g.n) || dy.type != x.type) return pass();
        g.d_dy = dy.p; g.dy_stride = dy.stride;
        if (g.activation != MLKV_ACT_NONE) {
            if (!pre.read(a[3], x, g.m, g.n) || pre.type != x.type) return pass();
            g.d_pre = pre.p; g.pre_stride = pre.stride;
        }
        const at::Tensor r[3] = {truth(a[6]) ? make(x, {g.m, g.k}, x.scalar) : at::Tensor(), truth(a[7]) ? make(x, {g.n, g.k}, x.scalar) : at::Tensor(),
                                 truth(a[5]) ? make(x, {g.n}, x.scalar) : at::Tensor()};
        g.d_dx = at_of(r[0]); g.dx_stride = g.k;
        g.d_dweight = at_of(r[1]); g.dweight_stride = g.k;
        g.d_dbias = at_of(r[2]);
        g.workspace_bytes = lib.linear_backward_workspace(&g);
        const Workspace ws(x, g.workspace_bytes);
        g.d_workspace = ws.p;
        const int rc = lib.linear_backward(&g, stream_of(x));
        return rc != MLKV_OK ? PyLong_FromLong(rc) : tuple_of(r);
    });
}

bool logits_of(PyObject* o, PyObject* targets, PyObject* scale, Mat& x, void** t) {
    if (!x.read(o) || !here(x) || x.cols < 1 || !PyFloat_Check(scale) || !vector_of(targets, x, x.rows, at::kLong, t)) return false;
    const double s = PyFloat_AS_DOUBLE(scale);
    return s > 0 && s < std::numeric_limits<double>::infinity();
}

// logits, targets, top, scale
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Mat x;
        void* t;
        if (n != 4 || !logits_of(a[0], a[1], a[3], x, &t) || !PyLong_CheckExact(a[2])) return pass();
        const long top = PyLong_AsLong(a[2]);
        if (top < 0 || top > MLKV_MAX_TOP) return PyErr_Clear(), pass();
        const int64_t bytes = lib.token_logprobs_workspace(x.rows, x.cols, x.type, (int32_t)top);
        if (bytes < 0) return pass();
        const at::Tensor r[5] = {make(x, {x.rows}, kFloat), make(x, {x.rows}, kFloat), make(x, {x.rows, 2}, kFloat),
                                 top ? make(x, {x.rows, top}, kFloat) : at::Tensor(), top ? make(x, {x.rows, top}, at::kLong) : at::Tensor()};
        const Workspace ws(x, bytes);
        const int rc = lib.token_logprobs(x.p, x.stride, x.type, x.rows, x.cols, (const int64_t*)t, (float)PyFloat_AS_DOUBLE(a[3]), (int32_t)top,
                                          (float*)r[0].data_ptr(), (float*)r[1].data_ptr(), (float*)r[2].data_ptr(), (float*)at_of(r[3]),
                                          (int64_t*)at_of(r[4]), ws.p, bytes, stream_of(x));
        return rc != MLKV_OK ? PyLong_FromLong(rc) : tuple_of(r);
    });
}

// logits, targets, entropy, stats, dlogprob, dentropy, scale, in_place
PyObject* token_logprobs_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Mat x, stats;
        void *t, *entropy, *g = nullptr, *h = nullptr;
        if (n != 8 || !logits_of(a[0], a[1], a[6], x, &t) || !vector_of(a[2], x, x.rows, kFloat, &entropy) || !stats.read(a[3], x, x.rows, 2) ||
            stats.type != MLKV_TYPE_FLOAT || stats.stride != 2)
            return pass();
        if (a[4] != Py_None && !vector_of(a[4], x, x.rows, kFloat, &g)) return pass();
        if (a[5] != Py_None && !vector_of(a[5], x, x.rows, kFloat, &h)) return pass();
        const bool in_place = truth(a[7]);
        const at::Tensor out = in_place ? at::Tensor() : make(x, {x.rows, x.cols}, x.scalar);
        const int rc = lib.token_logprobs_backward(x.p, x.stride, x.type, x.rows, x.cols, (const int64_t*)t, (float)PyFloat_AS_DOUBLE(a[6]),
                                                   (const float*)entropy, (const float*)stats.p, (const float*)g, (const float*)h,
                                                   in_place ? x.p : out.data_ptr(), in_place ? x.stride : x.cols, stream_of(x));
        if (rc != MLKV_OK) return PyLong_FromLong(rc);
        if (!in_place) return given(out);
        Py_INCREF(a[0]);
        return a[0];
    });
}

// x [m][k], w_gate and w_up [f][k], all of one 16-bit type
bool gated_operands(PyObject* xo, PyObject* go, PyObject* uo, PyObject* act, Mat& x, mlkv_gated_linear_args& g) {
    Mat wg, wu;
    if (!x.read(xo) || !here(x) || x.type == MLKV_TYPE_FLOAT || !wg.read(go) || wg.device != x.device || wg.type != x.type || wg.cols != x.cols ||
        !wu.read(uo, x, wg.rows, x.cols) || wu.type != x.type)
        return false;
    g = mlkv_gated_linear_args{};
    g.m = x.rows; g.f = wg.rows; g.k = x.cols;
    g.d_x = x.p; g.x_stride = x.stride; g.d_w_gate = wg.p; g.w_gate_stride = wg.stride; g.d_w_up = wu.p; g.w_up_stride = wu.stride;
    g.type = x.type;
    g.activation = (int32_t)PyLong_AsLong(act);
    return g.activation >= MLKV_ACT_NONE;
}

// x, w_gate, w_up, activation, save_pre
PyObject* gated_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Mat x;
        mlkv_gated_linear_args g;
        if (n != 5 || !gated_operands(a[0], a[1], a[2], a[3], x, g)) return pass();
        const bool save = truth(a[4]);
        const int64_t wide = (g.f + 7) / 8 * 8;
        auto saved = [&] { return !save ? at::Tensor() : wide == g.f ? make(x, {g.m, g.f}, x.scalar) : make(x, {g.m, wide}, x.scalar).narrow(1, 0, g.f); };
        const at::Tensor r[3] = {make(x, {g.m, g.f}, x.scalar), saved(), saved()};
        g.d_h = r[0].data_ptr(); g.d_gate = at_of(r[1]); g.d_up = at_of(r[2]);
        g.h_stride = g.f; g.gate_stride = g.up_stride = wide;
        g.workspace_bytes = lib.gated_linear_workspace(&g);
        const Workspace ws(x, g.workspace_bytes);
        g.d_workspace = ws.p;
        const int rc = lib.gated_linear(&g, stream_of(x));
        if (rc != MLKV_OK) return PyLong_FromLong(rc);
        return save ? tuple_of(r) : given(r[0]);
    });
}

// dh, x, w_gate, w_up, gate, up, activation, want_dx, want_dweight
PyObject* gated_linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Mat x, dh, gate, up;
        mlkv_gated_linear_args g;
        if (n != 9 || !gated_operands(a[1], a[2], a[3], a[6], x, g) || !dh.read(a[0], x, g.m, g.f) || dh.type != x.type || !gate.read(a[4], x, g.m, g.f) ||
            gate.type != x.type || !up.read(a[5], x, g.m, g.f) || up.type != x.type)
            return pass();
        g.d_dh = dh.p; g.dh_stride = dh.stride; g.d_gate = gate.p; g.gate_stride = gate.stride; g.d_up = up.p; g.up_stride = up.stride;
        const bool dx = truth(a[7]), dw = truth(a[8]);
        const at::Tensor r[3] = {dx ? make(x, {g.m, g.k}, x.scalar) : at::Tensor(), dw ? make(x, {g.f, g.k}, x.scalar) : at::Tensor(),
                                 dw ? make(x, {g.f, g.k}, x.scalar) : at::Tensor()};
        g.d_dx = at_of(r[0]); g.d_dw_gate = at_of(r[1]); g.d_dw_up = at_of(r[2]);
        g.dx_stride = g.dw_gate_stride = g.dw_up_stride = g.k;
        g.workspace_bytes = lib.gated_linear_backward_workspace(&g);
        const Workspace ws(x, g.workspace_bytes);
        g.d_workspace = ws.p;
        const int rc = lib.gated_linear_backward(&g, stream_of(x));
        return rc != MLKV_OK ? PyLong_FromLong(rc) : tuple_of(r);
    });
}

// x [n][k] and weight [vocab][k], of one 16-bit type
bool xent_operands(PyObject* xo, PyObject* wo, PyObject* targets, PyObject* scale, Mat& x, mlkv_linear_cross_entropy_args& g) {
    Mat w;
    void* t;
    if (!x.read(xo) || !here(x) || x.type == MLKV_TYPE_FLOAT || !w.read(wo) || w.device != x.device || w.type != x.type || w.cols != x.cols ||
        w.rows < 1 || x.cols < 1 || !PyFloat_Check(scale) || !vector_of(targets, x, x.rows, at::kLong, &t))
        return false;
    const double s = PyFloat_AS_DOUBLE(scale);
    if (!(s > 0 && s < 0x1p127)) return false;
    g = mlkv_linear_cross_entropy_args{};
    g.n = x.rows; g.k = x.cols; g.vocab = w.rows;
    g.d_x = x.p; g.x_stride = x.stride; g.d_weight = w.p; g.weight_stride = w.stride; g.d_targets = (const int64_t*)t;
    g.scale = (float)s; g.type = x.type;
    return true;
}

// x, weight, targets, scale
PyObject* linear_cross_entropy(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Mat x;
        mlkv_linear_cross_entropy_args g;
        if (n != 4 || !xent_operands(a[0], a[1], a[2], a[3], x, g)) return pass();
        const at::Tensor r[2] = {make(x, {g.n}, kFloat), make(x, {g.n, 2}, kFloat)};
        g.d_loss = (float*)r[0].data_ptr(); g.d_stats = (float*)r[1].data_ptr();
        g.workspace_bytes = lib.linear_cross_entropy_workspace(&g);
        const Workspace ws(x, g.workspace_bytes);
        g.d_workspace = ws.p;
        const int rc = lib.linear_cross_entropy(&g, stream_of(x));
        return rc != MLKV_OK ? PyLong_FromLong(rc) : tuple_of(r);
    });
}

// dloss, x, weight, targets, stats, scale, want_dx, want_dweight
PyObject* linear_cross_entropy_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        Mat x, stats;
        mlkv_linear_cross_entropy_args g;
        void* d;
        if (n != 8 || !xent_operands(a[1], a[2], a[3], a[5], x, g) || !vector_of(a[0], x, g.n, kFloat, &d) || !stats.read(a[4], x, g.n, 2) ||
            stats.type != MLKV_TYPE_FLOAT || stats.stride != 2)
            return pass();
        g.d_dloss = (const float*)d; g.d_stats = (float*)stats.p;
        const at::Tensor r[2] = {truth(a[6]) ? make(x, {g.n, g.k}, x.scalar) : at::Tensor(), truth(a[7]) ? make(x, {g.vocab, g.k}, x.scalar) : at::Tensor()};
        g.d_dx = at_of(r[0]); g.d_dweight = at_of(r[1]);
        g.dx_stride = g.dweight_stride = g.k;
        g.workspace_bytes = lib.linear_cross_entropy_backward_workspace(&g);
        const Workspace ws(x, g.workspace_bytes);
        g.d_workspace = ws.p;
        const int rc = lib.linear_cross_entropy_backward(&g, stream_of(x));
        return rc != MLKV_OK ? PyLong_FromLong(rc) : tuple_of(r);
    });
}

// A list or a tuple of n objects (null: None).
struct Items {
    PyObject* const* at = nullptr;
    bool read(PyObject* o, Py_ssize_t n) {
        if (!(PyList_CheckExact(o) || PyTuple_CheckExact(o)) || PySequence_Fast_GET_SIZE(o) != n) return false;
        at = PySequence_Fast_ITEMS(o);
        return true;
    }
    bool read_or_none(PyObject* o, Py_ssize_t n) { return o == Py_None || read(o, n); }
};
const at::Tensor* contiguous(PyObject* o, c10::Device device) {
    if (!THPVariable_Check(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.defined() && t.layout() == at::kStrided && t.device() == device && t.is_contiguous() ? &t : nullptr;
}
// A value on the device.
template <class T>
bool value_of(PyObject* o, c10::Device device, at::ScalarType scalar, const T** at) {
    const at::Tensor* t = contiguous(o, device);
    if (!t || t->scalar_type() != scalar || t->numel() != 1) return false;
    *at = (const T*)t->data_ptr();
    return true;
}

// params, grads, m, v, scales, copies, lr, beta1, beta2, eps, weight_decay, step, grad_scale, seed
PyObject* adamw(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 14 || !(PyList_CheckExact(a[0]) || PyTuple_CheckExact(a[0]))) return pass();
        const Py_ssize_t count = PySequence_Fast_GET_SIZE(a[0]);
        Items params, grads, m, v, scales, copies;
        if (count < 1 || !params.read(a[0], count) || !grads.read(a[1], count) || !m.read(a[2], count) || !v.read(a[3], count) ||
            !scales.read_or_none(a[4], count) || !copies.read_or_none(a[5], count) || !THPVariable_Check(params.at[0]))
            return pass();
        const at::Tensor& first = THPVariable_Unpack(params.at[0]);
        if (!first.defined() || !first.is_cuda() || c10::cuda::current_device() != first.device().index()) return pass();
        const c10::Device device = first.device();
        const bool small = scales.at != nullptr;
        const at::ScalarType state = small ? at::kFloat8_e4m3fn : kFloat;
        static thread_local std::vector<mlkv_adamw_tensor> table;
        table.assign(count, mlkv_adamw_tensor{});
        for (Py_ssize_t i = 0; i < count; ++i) {
            mlkv_adamw_tensor& t = table[i];
            const at::Tensor *p = contiguous(params.at[i], device), *ms = contiguous(m.at[i], device), *vs = contiguous(v.at[i], device);
            if (!p || !ms || !vs || type_of(p->scalar_type()) < 0 || ms->scalar_type() != state || vs->scalar_type() != state ||
                ms->sizes() != p->sizes() || vs->sizes() != p->sizes())
                return pass();
            t.param_type = type_of(p->scalar_type());
            if (small) {
                const at::Tensor* s = contiguous(scales.at[i], device);
                if (!s || s->scalar_type() != kFloat || s->dim() != 2 || s->size(0) != 2 || s->size(1) != (p->numel() + 255) / 256) return pass();
                t.d_scales = (float*)s->data_ptr();
            }
            if (copies.at && copies.at[i] != Py_None) {
                const at::Tensor* c = contiguous(copies.at[i], device);
                if (!c || t.param_type != MLKV_TYPE_FLOAT || c->sizes() != p->sizes()) return pass();
                t.copy_type = type_of(c->scalar_type());
                if (t.copy_type <= MLKV_TYPE_FLOAT) return pass();
                t.d_copy = c->data_ptr();
            }
            if (grads.at[i] == Py_None) continue;
            const at::Tensor* g = contiguous(grads.at[i], device);
            if (!g || type_of(g->scalar_type()) < 0 || g->sizes() != p->sizes()) return pass();
            t.grad_type = type_of(g->scalar_type());
            t.d_grad = g->data_ptr();
            t.d_param = p->data_ptr();
            t.d_m = ms->data_ptr();
            t.d_v = vs->data_ptr();
            t.n = p->numel();
        }
        mlkv_adamw_args g = {};
        for (int i = 7; i < 11; ++i)
            if (!PyFloat_CheckExact(a[i])) return pass();
        if (!PyLong_CheckExact(a[13])) return pass();
        const long long seed = PyLong_AsLongLong(a[13]);
        if (seed < 0 || seed > 0xFFFFFFFFll) return PyErr_Clear(), pass();
        if (PyFloat_CheckExact(a[6])) g.lr = PyFloat_AS_DOUBLE(a[6]);
        else if (!value_of(a[6], device, kFloat, &g.d_lr)) return pass();
        if (PyLong_CheckExact(a[11])) {
            g.step = PyLong_AsLongLong(a[11]);
            if (g.step < 1) return PyErr_Clear(), pass();
        } else if (!value_of(a[11], device, at::kLong, &g.d_step)) {
            return pass();
        }
        if (a[12] != Py_None && !value_of(a[12], device, kFloat, &g.d_grad_scale)) return pass();
        g.tensors = table.data(); g.count = count;
        g.beta1 = PyFloat_AS_DOUBLE(a[7]); g.beta2 = PyFloat_AS_DOUBLE(a[8]); g.eps = PyFloat_AS_DOUBLE(a[9]); g.weight_decay = PyFloat_AS_DOUBLE(a[10]);
        g.seed = (uint32_t)seed; g.state_bits = small ? 8 : 32;
        const int rc = lib.adamw(&g, c10::cuda::getCurrentCUDAStream(device.index()).stream());
        if (rc != MLKV_OK) return PyLong_FromLong(rc);
        Py_RETURN_NONE;
    });
}

// The library's path: its calls from here on.
PyObject* bind(PyObject*, PyObject* path) {
    const char* p = PyUnicode_AsUTF8(path);
    if (!p) return nullptr;
    void* h = dlopen(p, RTLD_NOW | RTLD_LOCAL);
    Library found = {};
    bool ok = h != nullptr;
    auto get = [&](auto& f, const char* name) {
        f = h ? reinterpret_cast<std::remove_reference_t<decltype(f)>>(dlsym(h, name)) : nullptr;
        ok = ok && f;
    };
    get(found.layer_norm, "mlkv_layer_norm");
    get(found.layer_norm_backward, "mlkv_layer_norm_backward");
    get(found.layer_norm_backward_workspace, "mlkv_layer_norm_backward_workspace");
    get(found.linear, "mlkv_linear");
    get(found.linear_workspace, "mlkv_linear_workspace");
    get(found.linear_backward, "mlkv_linear_backward");
    get(found.linear_backward_workspace, "mlkv_linear_backward_workspace");
    get(found.token_logprobs, "mlkv_token_logprobs");
    get(found.token_logprobs_workspace, "mlkv_token_logprobs_workspace");
    get(found.token_logprobs_backward, "mlkv_token_logprobs_backward");
    get(found.gated_linear, "mlkv_gated_linear");
    get(found.gated_linear_workspace, "mlkv_gated_linear_workspace");
    get(found.gated_linear_backward, "mlkv_gated_linear_backward");
    get(found.gated_linear_backward_workspace, "mlkv_gated_linear_backward_workspace");
    get(found.linear_cross_entropy, "mlkv_linear_cross_entropy");
    get(found.linear_cross_entropy_workspace, "mlkv_linear_cross_entropy_workspace");
    get(found.linear_cross_entropy_backward, "mlkv_linear_cross_entropy_backward");
    get(found.linear_cross_entropy_backward_workspace, "mlkv_linear_cross_entropy_backward_workspace");
    get(found.adamw, "mlkv_adamw");
    if (!ok) return PyErr_Format(PyExc_ImportError, "%s: not the library of these calls", p);
    lib = found;
    Py_RETURN_NONE;
}

#define CALL(f) {#f, (PyCFunction)(void (*)())(f), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(layer_norm), CALL(layer_norm_backward), CALL(linear), CALL(linear_backward), CALL(token_logprobs),
                         CALL(token_logprobs_backward), CALL(gated_linear), CALL(gated_linear_backward), CALL(linear_cross_entropy),
                         CALL(linear_cross_entropy_backward), CALL(adamw), {"bind", bind, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_dense_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dense_calls() { return PyModule_Create(&module); }
