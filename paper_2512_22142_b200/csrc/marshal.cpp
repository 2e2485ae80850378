// Argument marshalling of the operators' Python binding: torch tensors -> the records of include/cleave.h.  What the
// library cannot see (types, shapes, strides, devices) is checked here; everything else is the library's.  In C++
// because a call lasts a few microseconds and the same checks in Python take twice that.
//
// Each function takes its arguments by position, None for what is absent, the raw stream or None (torch's current
// stream of the tensors' device) last, raises ValueError for arguments that cannot be marshalled and returns the
// library's code.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include "cleave.h"

namespace {

struct Refused {};          // a Python error is set

[[noreturn]] void refuse(const char* name, const char* what) {
    PyErr_Format(PyExc_ValueError, "%s: %s", name, what);
    throw Refused{};
}

constexpr unsigned kBf16 = 1u << CLEAVE_T_BF16, kF32 = 1u << CLEAVE_T_F32, kE4M3 = 1u << CLEAVE_T_E4M3, kFloats = kBf16 | kF32;

uint32_t type_of(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case at::kBFloat16: return CLEAVE_T_BF16;
        case at::kFloat: return CLEAVE_T_F32;
        case at::kFloat8_e4m3fn: return CLEAVE_T_E4M3;
        default: return CLEAVE_T_NONE;
    }
}
const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse(name, "a tensor is wanted");
    return THPVariable_Unpack(o);
}
// `like`: the call's leading operand, on whose device the launch goes
uint32_t checked_type(const at::Tensor& t, const char* name, unsigned types, const at::Tensor& like) {
    const uint32_t kind = type_of(t);
    if (!kind || !(types >> kind & 1u) || !t.is_cuda()) refuse(name, "a GPU tensor of a supported type is wanted");
    if (t.device() != like.device()) refuse(name, "the operands are on different devices");
    return kind;
}

struct Matrix { uint32_t type = 0; void* p = nullptr; uint64_t ld = 0; };
Matrix matrix(PyObject* o, const char* name, const at::Tensor& like, int64_t rows, int64_t cols, unsigned types, bool optional = false) {
    Matrix m;
    if (optional && o == Py_None) return m;
    const at::Tensor& t = tensor(o, name);
    m.type = checked_type(t, name, types, like);
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols) {
        PyErr_Format(PyExc_ValueError, "%s: shape (%lld, %lld) is wanted", name, (long long)rows, (long long)cols);
        throw Refused{};
    }
    if (t.stride(1) != 1 && cols > 1) refuse(name, "rows have to be contiguous");
    int64_t ld = t.stride(0);
    if (rows <= 1) ld = cols;                              // a single row: any stride
    else if (ld < cols) refuse(name, "rows overlap");
    m.p = t.data_ptr();
    m.ld = (uint64_t)ld;
    return m;
}
struct Vector { uint32_t type = 0; void* p = nullptr; };
Vector vector(PyObject* o, const char* name, const at::Tensor& like, int64_t n, unsigned types) {
    Vector v;
    if (o == Py_None) return v;
    const at::Tensor& t = tensor(o, name);
    v.type = checked_type(t, name, types, like);
    if (t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1)) {
        PyErr_Format(PyExc_ValueError, "%s: a contiguous tensor of %lld elements is wanted", name, (long long)n);
        throw Refused{};
    }
    v.p = t.data_ptr();
    return v;
}
const at::Tensor& leading(PyObject* o, const char* name) {
    const at::Tensor& t = tensor(o, name);
    if (t.dim() != 2) refuse(name, "two dimensions are wanted");
    if (t.size(0) > 0xFFFFFFFFll || t.size(1) > 0xFFFFFFFFll) refuse(name, "too large");
    if (!t.is_cuda()) refuse(name, "a GPU tensor of a supported type is wanted");
    return t;
}
void* stream_of(PyObject* o, const at::Tensor& t) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream(t.device().index()).stream();
    void* s = PyLong_AsVoidPtr(o);
    if (!s && PyErr_Occurred()) throw Refused{};
    return s;
}
// The caller's workspace, or one from torch's allocator (on the current stream: the launch's own, see ops.py).
void* workspace(PyObject* o, uint64_t bytes, const at::Tensor& like, at::Tensor& hold) {
    if (o == Py_None) {
        hold = at::empty({(int64_t)(bytes > 16 ? bytes : 16)}, like.options().dtype(at::kByte));
        return hold.data_ptr();
    }
    const at::Tensor& t = tensor(o, "workspace");
    if (!t.is_cuda() || t.device() != like.device() || !t.is_contiguous() || (uint64_t)t.nbytes() < bytes) {
        PyErr_Format(PyExc_ValueError, "workspace: %llu contiguous bytes on the operands' GPU are wanted", (unsigned long long)bytes);
        throw Refused{};
    }
    return t.data_ptr();
}

PyObject* run_rmsnorm(PyObject* const* a) {                // x, weight, y, residual, h, rstd, scale, eps, stream
    const at::Tensor& x = leading(a[0], "x");
    const int64_t rows = x.size(0), cols = x.size(1);
    const Matrix mx = matrix(a[0], "x", x, rows, cols, kFloats), my = matrix(a[2], "y", x, rows, cols, kFloats | kE4M3);
    const Matrix mr = matrix(a[3], "residual", x, rows, cols, kFloats, true), mh = matrix(a[4], "h", x, rows, cols, kFloats, true);
    const Vector w = vector(a[1], "weight", x, cols, kFloats);
    if (mh.p && mr.type && mh.type != mr.type) refuse("h", "the residual's type is wanted");
    cleave_rmsnorm_t d = {};
    d.rows = (uint64_t)rows; d.cols = (uint32_t)cols;
    d.x_type = mx.type; d.r_type = mr.type; d.w_type = w.type; d.y_type = my.type;
    d.eps = (float)PyFloat_AsDouble(a[7]);
    if (PyErr_Occurred()) throw Refused{};
    d.x = mx.p; d.ldx = mx.ld; d.r = mr.p; d.ldr = mr.ld; d.h = mh.p; d.ldh = mh.ld; d.w = w.p; d.y = my.p; d.ldy = my.ld;
    d.rstd = static_cast<float*>(vector(a[5], "rstd", x, rows, kF32).p);
    d.scale = static_cast<float*>(vector(a[6], "scale", x, rows, kF32).p);
    const c10::cuda::CUDAGuard guard(x.device());
    return PyLong_FromLong(cleave_rmsnorm(&d, stream_of(a[8], x)));
}

PyObject* run_rmsnorm_backward(PyObject* const* a) {       // dy, h, weight, rstd, dx, dweight, dres, workspace, stream
    const at::Tensor& h = leading(a[1], "h");
    const int64_t rows = h.size(0), cols = h.size(1);
    const Matrix mh = matrix(a[1], "h", h, rows, cols, kFloats), mdy = matrix(a[0], "dy", h, rows, cols, kFloats);
    const Matrix mdx = matrix(a[4], "dx", h, rows, cols, 1u << mh.type), mr = matrix(a[6], "dres", h, rows, cols, 1u << mh.type, true);
    const Vector w = vector(a[2], "weight", h, cols, kFloats);
    cleave_rmsnorm_backward_t d = {};
    d.rows = (uint64_t)rows; d.cols = (uint32_t)cols;
    d.dy_type = mdy.type; d.h_type = mh.type; d.w_type = w.type;
    d.dy = mdy.p; d.lddy = mdy.ld; d.h = mh.p; d.ldh = mh.ld; d.w = w.p; d.dres = mr.p; d.lddres = mr.ld; d.dx = mdx.p; d.lddx = mdx.ld;
    d.rstd = static_cast<const float*>(vector(a[3], "rstd", h, rows, kF32).p);
    d.dw = static_cast<float*>(vector(a[5], "dweight", h, cols, kF32).p);
    at::Tensor hold;
    void* ws = a[5] != Py_None ? workspace(a[7], cleave_rmsnorm_backward_workspace(d.rows, d.cols), h, hold) : nullptr;
    const c10::cuda::CUDAGuard guard(h.device());
    return PyLong_FromLong(cleave_rmsnorm_backward(&d, ws, stream_of(a[8], h)));
}

PyObject* run_quantize_rows(PyObject* const* a) {          // x, y, scale, stream
    const at::Tensor& x = leading(a[0], "x");
    const int64_t rows = x.size(0), cols = x.size(1);
    const Matrix mx = matrix(a[0], "x", x, rows, cols, kFloats), my = matrix(a[1], "y", x, rows, cols, kE4M3);
    if (a[2] == Py_None) refuse("scale", "a tensor is wanted");
    float* scale = static_cast<float*>(vector(a[2], "scale", x, rows, kF32).p);
    const c10::cuda::CUDAGuard guard(x.device());
    return PyLong_FromLong(cleave_quantize_rows(mx.p, mx.type, (uint64_t)rows, (uint32_t)cols, mx.ld, my.p, my.ld, scale, stream_of(a[3], x)));
}

// A, B, out, transA, transB, scale_a, scale_b, bias, act, z, mul, residual, stream
PyObject* run_linear(PyObject* const* a) {
    const at::Tensor &A = leading(a[0], "A"), &B = leading(a[1], "B");
    const int ta = PyObject_IsTrue(a[3]), tb = PyObject_IsTrue(a[4]);
    if (ta < 0 || tb < 0) throw Refused{};
    const int64_t M = A.size(ta ? 1 : 0), K = A.size(ta ? 0 : 1), N = B.size(tb ? 0 : 1);
    const Matrix ma = matrix(a[0], "A", A, A.size(0), A.size(1), kBf16 | kE4M3), mb = matrix(a[1], "B", A, tb ? N : K, tb ? K : N, 1u << ma.type);
    const Matrix mc = matrix(a[2], "out", A, M, N, kFloats), mz = matrix(a[9], "z", A, M, N, kFloats, true), mm = matrix(a[10], "mul", A, M, N, kFloats, true),
                 mr = matrix(a[11], "residual", A, M, N, kFloats, true);
    const Vector bias = vector(a[7], "bias", A, N, kFloats);
    const uint64_t unit = ma.type == CLEAVE_T_E4M3 ? 16 : 8;
    auto ld = [&](const Matrix& m, const at::Tensor& t) -> uint32_t {
        const uint64_t l = t.size(0) == 1 ? (m.ld + unit - 1) / unit * unit : m.ld;          // a single row has no second one
        if (l > 0xFFFFFFFFull) refuse("A, B", "rows lie too far apart");
        return (uint32_t)l;
    };
    cleave_linear_t d = {};
    d.g.M = (uint32_t)M; d.g.N = (uint32_t)N; d.g.K = (uint32_t)K; d.g.lda = ld(ma, A); d.g.ldb = ld(mb, B);
    d.g.transA = (uint8_t)ta; d.g.transB = (uint8_t)tb;
    d.in_type = ma.type; d.c_type = mc.type; d.bias_type = bias.type; d.z_type = mz.type; d.mul_type = mm.type; d.res_type = mr.type;
    d.act = (uint32_t)PyLong_AsUnsignedLong(a[8]);
    if (PyErr_Occurred()) throw Refused{};
    d.A = ma.p; d.B = mb.p; d.bias = bias.p;
    d.scale_a = static_cast<const float*>(vector(a[5], "scale_a", A, M, kF32).p);
    d.scale_b = static_cast<const float*>(vector(a[6], "scale_b", A, N, kF32).p);
    d.z = mz.p; d.ldz = mz.ld; d.mul = mm.p; d.ldmul = mm.ld; d.res = mr.p; d.ldres = mr.ld; d.C = mc.p; d.ldc = mc.ld;
    const c10::cuda::CUDAGuard guard(A.device());
    return PyLong_FromLong(cleave_linear(&d, stream_of(a[12], A)));
}

// dy, z, dz, act, mul, dmul, dbias, workspace, stream
PyObject* run_act_backward(PyObject* const* a) {
    const at::Tensor& dy = leading(a[0], "dy");
    const int64_t rows = dy.size(0), cols = dy.size(1);
    const Matrix mdy = matrix(a[0], "dy", dy, rows, cols, kFloats), mz = matrix(a[1], "z", dy, rows, cols, kFloats, true), mdz = matrix(a[2], "dz", dy, rows, cols, kFloats, true),
                 mm = matrix(a[4], "mul", dy, rows, cols, kFloats, true), mdm = matrix(a[5], "dmul", dy, rows, cols, kFloats, true);
    cleave_act_backward_t d = {};
    d.rows = (uint64_t)rows; d.cols = (uint32_t)cols;
    d.act = (uint32_t)PyLong_AsUnsignedLong(a[3]);
    if (PyErr_Occurred()) throw Refused{};
    d.dy_type = mdy.type; d.z_type = mz.type; d.mul_type = mm.type; d.dz_type = mdz.type; d.dmul_type = mdm.type;
    d.dy = mdy.p; d.lddy = mdy.ld; d.z = mz.p; d.ldz = mz.ld; d.mul = mm.p; d.ldmul = mm.ld; d.dz = mdz.p; d.lddz = mdz.ld; d.dmul = mdm.p; d.lddmul = mdm.ld;
    d.dbias = static_cast<float*>(vector(a[6], "dbias", dy, cols, kF32).p);
    at::Tensor hold;
    void* ws = a[6] != Py_None ? workspace(a[7], cleave_act_backward_workspace(d.rows, d.cols), dy, hold) : nullptr;
    const c10::cuda::CUDAGuard guard(dy.device());
    return PyLong_FromLong(cleave_act_backward(&d, ws, stream_of(a[8], dy)));
}

// No C++ exception leaves a call: the ones above have set a Python error, torch's become one.
template <PyObject* (*RUN)(PyObject* const*), int N>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N) return PyErr_Format(PyExc_TypeError, "%d arguments are wanted, got %zd", N, n);
    try {
        return RUN(args);
    } catch (const Refused&) {
        return nullptr;
    } catch (const std::exception& e) {
        return PyErr_Format(PyExc_RuntimeError, "%s", e.what());
    }
}

template <PyObject* (*RUN)(PyObject* const*), int N>
PyMethodDef method(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call<RUN, N>)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method<run_rmsnorm, 9>("rmsnorm"), method<run_rmsnorm_backward, 9>("rmsnorm_backward"), method<run_quantize_rows, 4>("quantize_rows"),
                         method<run_linear, 13>("linear"), method<run_act_backward, 9>("act_backward"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of the operators (see ops.py).", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
