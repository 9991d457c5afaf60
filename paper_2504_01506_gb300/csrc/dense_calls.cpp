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
    if (!ok) return PyErr_Format(PyExc_ImportError, "%s: not the library of these calls", p);
    lib = found;
    Py_RETURN_NONE;
}

#define CALL(f) {#f, (PyCFunction)(void (*)())(f), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(layer_norm), CALL(layer_norm_backward), CALL(linear), CALL(linear_backward), CALL(token_logprobs),
                         CALL(token_logprobs_backward), {"bind", bind, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_dense_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dense_calls() { return PyModule_Create(&module); }
