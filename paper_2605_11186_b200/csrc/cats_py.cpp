// Argument marshalling of the 8-bit calls for binding.py, as a CPython extension.
//
// A call of these operators runs for 2 to 5 us on the GPU; checking its tensors and filling its arguments through Python
// and ctypes took 13 us, through this file under 1 us.  Every function takes the tensors of the C entry point of the same
// name (include/cats.h), checks what the pointers cannot say -- device, element type, shape, strides -- and raises
// ValueError, else calls the entry point on the current stream and returns its status code.  The entry points' addresses
// come from the library binding.py has loaded (bind), so this file links against torch only.
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/cats.h"

namespace {

decltype(&cats_quantize_i8) f_quantize = nullptr;
decltype(&cats_dequantize_i8) f_dequantize = nullptr;
decltype(&cats_rmsnorm_i8) f_rmsnorm = nullptr;
decltype(&cats_swiglu_i8) f_swiglu = nullptr;
decltype(&cats_linear_i8) f_linear = nullptr;

struct Refused {};      // thrown with a Python error set

[[noreturn]] void refuse(const char* what, const char* name, const char* why) {
    PyErr_Format(PyExc_ValueError, "%s: %s %s", what, name, why);
    throw Refused();
}

const at::Tensor& tensor(PyObject* o, const char* what, const char* name) {
    if (!THPVariable_Check(o)) refuse(what, name, "must be a tensor");
    return THPVariable_Unpack(o);
}

struct Call {
    const char* what;
    int device = -1;        // of the first tensor; the others have to be there too

    void place(const at::Tensor& t, const char* name) {
        if (!t.is_cuda() || t.layout() != c10::kStrided || t.is_neg()) refuse(what, name, "must be a plain CUDA tensor");
        const int d = t.get_device();
        if (device < 0) {
            device = d;
            if (d != (int)c10::cuda::current_device()) refuse(what, name, "is not on the current device");
        } else if (d != device) {
            refuse(what, name, "is on another device");
        }
    }
    void* stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
};

struct Matrix {
    void* p = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    int32_t type = 0;
};

constexpr int64_t kAny = -1;

// A 2-D tensor whose rows are contiguous; rows, cols: what they have to be, or kAny.
Matrix matrix(Call& c, PyObject* o, const char* name, int64_t rows, int64_t cols, bool floats) {
    const at::Tensor& t = tensor(o, c.what, name);
    c.place(t, name);
    if (t.dim() != 2 || (rows != kAny && t.size(0) != rows) || (cols != kAny && t.size(1) != cols)) refuse(c.what, name, "has the wrong shape");
    if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX) refuse(c.what, name, "is too large");
    Matrix m;
    const auto type = t.scalar_type();
    if (floats && type == at::kFloat) m.type = CATS_F32;
    else if (floats && type == at::kBFloat16) m.type = CATS_BF16;
    else if (floats || type != at::kChar) refuse(c.what, name, floats ? "must be float32 or bfloat16" : "must be int8");
    m.rows = t.size(0);
    m.cols = t.size(1);
    if (m.cols > 1 && t.stride(1) != 1) refuse(c.what, name, "must have contiguous rows");
    m.ld = m.rows > 1 ? t.stride(0) : (m.cols + 15) / 16 * 16;      // a single row's stride means nothing
    m.p = t.data_ptr();
    return m;
}

void* vector(Call& c, PyObject* o, const char* name, int64_t n, at::ScalarType type, const char* must) {
    const at::Tensor& t = tensor(o, c.what, name);
    c.place(t, name);
    if (t.dim() != 1 || (n != kAny && t.size(0) != n)) refuse(c.what, name, "has the wrong shape");
    if (t.scalar_type() != type) refuse(c.what, name, must);
    if (t.size(0) > 1 && t.stride(0) != 1) refuse(c.what, name, "must be contiguous");
    return t.data_ptr();
}
float* scales(Call& c, PyObject* o, const char* name, int64_t n) { return (float*)vector(c, o, name, n, at::kFloat, "must be float32"); }

template <typename F> PyObject* guarded(const char* what, Py_ssize_t n, Py_ssize_t want, F body) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%s: %zd arguments, %zd are wanted", what, n, want);
        return nullptr;
    }
    try {
        return PyLong_FromLong(body());
    } catch (const Refused&) {
    } catch (const std::exception& e) {
        PyErr_Format(PyExc_RuntimeError, "%s: %s", what, e.what());
    }
    return nullptr;
}
template <typename F> int without_gil(F f) {        // a launch may block when the stream's queue is full
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

PyObject* py_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("cats_quantize_i8", n, 3, [&] {
        Call c{"cats_quantize_i8"};
        const Matrix x = matrix(c, a[0], "x", kAny, kAny, true), q = matrix(c, a[1], "q", x.rows, x.cols, false);
        float* s = scales(c, a[2], "scale", x.rows);
        void* st = c.stream();
        return without_gil([&] { return f_quantize(x.p, x.type, x.ld, (int32_t)x.rows, (int32_t)x.cols, (int8_t*)q.p, q.ld, s, st); });
    });
}

PyObject* py_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("cats_dequantize_i8", n, 3, [&] {
        Call c{"cats_dequantize_i8"};
        const Matrix q = matrix(c, a[0], "q", kAny, kAny, false);
        const float* s = scales(c, a[1], "scale", q.rows);
        const Matrix o = matrix(c, a[2], "out", q.rows, q.cols, true);
        void* st = c.stream();
        return without_gil([&] { return f_dequantize((const int8_t*)q.p, q.ld, s, (int32_t)q.rows, (int32_t)q.cols, o.p, o.type, o.ld, st); });
    });
}

PyObject* py_rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("cats_rmsnorm_i8", n, 7, [&] {
        Call c{"cats_rmsnorm_i8"};
        const Matrix x = matrix(c, a[0], "resid", kAny, kAny, true);
        Matrix d, o;
        if (a[1] != Py_None) d = matrix(c, a[1], "delta", x.rows, x.cols, true);
        const void* g = vector(c, a[2], "gain", x.cols, at::kBFloat16, "must be bfloat16");
        const double eps = PyFloat_AsDouble(a[3]);
        if (eps == -1.0 && PyErr_Occurred()) throw Refused();
        if (a[4] != Py_None) {
            o = matrix(c, a[4], "resid_out", x.rows, x.cols, true);
            if (o.type != x.type) refuse(c.what, "resid_out", "must have resid's type");
        }
        const Matrix q = matrix(c, a[5], "q", x.rows, x.cols, false);
        float* s = scales(c, a[6], "scale", x.rows);
        void* st = c.stream();
        return without_gil([&] {
            return f_rmsnorm(x.p, x.type, x.ld, d.p, d.type, d.ld, g, (float)eps, (int32_t)x.rows, (int32_t)x.cols, o.p, o.ld, (int8_t*)q.p, q.ld, s, st);
        });
    });
}

PyObject* py_swiglu(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("cats_swiglu_i8", n, 3, [&] {
        Call c{"cats_swiglu_i8"};
        const Matrix x = matrix(c, a[0], "gate_up", kAny, kAny, true), q = matrix(c, a[1], "q", x.rows, kAny, false);
        if (x.cols != 2 * q.cols) refuse(c.what, "gate_up", "must have twice the columns of q");
        float* s = scales(c, a[2], "scale", x.rows);
        void* st = c.stream();
        return without_gil([&] { return f_swiglu(x.p, x.type, x.ld, (int32_t)q.rows, (int32_t)q.cols, (int8_t*)q.p, q.ld, s, st); });
    });
}

PyObject* py_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("cats_linear_i8", n, 6, [&] {
        Call c{"cats_linear_i8"};
        const Matrix x = matrix(c, a[0], "x", kAny, kAny, false);
        const float* sx = scales(c, a[1], "x_scale", x.rows);
        const at::Tensor& sw_t = tensor(a[3], c.what, "w_scale");
        const float* sw = scales(c, a[3], "w_scale", kAny);
        const int64_t outs = sw_t.size(0);
        const void* w = vector(c, a[2], "w_packed", (x.cols + 127) / 128 * ((outs + 7) / 8) * 1024, at::kByte, "must be uint8");
        const Matrix o = matrix(c, a[4], "out", x.rows, outs, true);
        int32_t* status = (int32_t*)vector(c, a[5], "status", 1, at::kInt, "must be int32");
        void* st = c.stream();
        return without_gil([&] {
            return f_linear((const int8_t*)x.p, x.ld, sx, w, sw, (int32_t)x.rows, (int32_t)x.cols, (int32_t)outs, o.p, o.type, o.ld, status, st);
        });
    });
}

// bind(quantize, dequantize, rmsnorm, swiglu, linear): addresses of the loaded library's entry points
PyObject* py_bind(PyObject*, PyObject* args) {
    unsigned long long p[5];
    if (!PyArg_ParseTuple(args, "KKKKK", &p[0], &p[1], &p[2], &p[3], &p[4])) return nullptr;
    f_quantize = (decltype(f_quantize))p[0];
    f_dequantize = (decltype(f_dequantize))p[1];
    f_rmsnorm = (decltype(f_rmsnorm))p[2];
    f_swiglu = (decltype(f_swiglu))p[3];
    f_linear = (decltype(f_linear))p[4];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", py_bind, METH_VARARGS, nullptr},
    {"quantize_i8", (PyCFunction)(void (*)(void))py_quantize, METH_FASTCALL, nullptr},
    {"dequantize_i8", (PyCFunction)(void (*)(void))py_dequantize, METH_FASTCALL, nullptr},
    {"rmsnorm_i8", (PyCFunction)(void (*)(void))py_rmsnorm, METH_FASTCALL, nullptr},
    {"swiglu_i8", (PyCFunction)(void (*)(void))py_swiglu, METH_FASTCALL, nullptr},
    {"linear_i8", (PyCFunction)(void (*)(void))py_linear, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_cats_py", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// What this was built from and for (build.py): looked for in the file before it is loaded.
PyMODINIT_FUNC PyInit__cats_py(void) {
    PyObject* const m = PyModule_Create(&module);
    if (m != nullptr && PyModule_AddStringConstant(m, "stamp", CATS_PY_STAMP) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
