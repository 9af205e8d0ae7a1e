// Argument marshalling of the 8-bit, paged-cache and sampling calls for binding.py, as a CPython extension.
//
// A call of these operators runs for 2 to 5 us on the GPU; checking its tensors and filling its arguments through Python
// and ctypes took 13 us, through this file under 1 us.  Every function takes the tensors of the C entry point of the same
// name (include/cats.h), checks what the pointers cannot say -- device, element type, shape, strides -- and raises
// ValueError, else calls the entry point on the current stream and returns its status code.  The entry points' addresses
// come from the library binding.py has loaded (bind), so this file links against torch only.
#include <Python.h>

#include <cstring>

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
decltype(&cats_paged_append) f_append = nullptr;
decltype(&cats_paged_read) f_read = nullptr;
decltype(&cats_paged_attention) f_attention = nullptr;
decltype(&cats_sample) f_sample = nullptr;

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

// A matrix [rows][cols], or [rows][cols / hd][hd] with the heads of a row together; hd: of the cache.
Matrix heads(Call& c, PyObject* o, const char* name, int64_t rows, int64_t cols, int64_t hd, bool bf16_only) {
    const at::Tensor& t = tensor(o, c.what, name);
    c.place(t, name);
    const bool three = t.dim() == 3;
    if ((!three && t.dim() != 2) || (rows != kAny && t.size(0) != rows) || (three && t.size(2) != hd)) refuse(c.what, name, "has the wrong shape");
    Matrix m;
    m.rows = t.size(0);
    m.cols = three ? t.size(1) * hd : t.size(1);
    if (cols != kAny && m.cols != cols) refuse(c.what, name, "has the wrong shape");
    if (m.rows > INT32_MAX || m.cols > INT32_MAX) refuse(c.what, name, "is too large");
    const auto type = t.scalar_type();
    if (type == at::kFloat && !bf16_only) m.type = CATS_F32;
    else if (type == at::kBFloat16) m.type = CATS_BF16;
    else refuse(c.what, name, bf16_only ? "must be bfloat16" : "must be float32 or bfloat16");
    if (m.cols > 0 && (t.stride(-1) != 1 || (three && t.size(1) > 1 && t.stride(1) != hd))) refuse(c.what, name, "must have contiguous rows");
    m.ld = m.rows > 1 ? t.stride(0) : (m.cols + 7) / 8 * 8;
    m.p = t.data_ptr();
    return m;
}

// The cache (its tensors, None where it has none, and its cats_paged_kv as bytes) and the table of its pages.
struct Paged {
    cats_paged_kv kv;
    const int32_t* table;
    int64_t ld, width, n_seqs;
};
Paged paged(Call& c, PyObject* tensors, PyObject* desc, PyObject* table) {
    Paged p;
    if (!PyTuple_Check(tensors) || PyTuple_GET_SIZE(tensors) != 4 || !PyBytes_Check(desc) || PyBytes_GET_SIZE(desc) != (Py_ssize_t)sizeof p.kv)
        refuse(c.what, "cache", "must be a PagedKV");
    std::memcpy(&p.kv, PyBytes_AS_STRING(desc), sizeof p.kv);
    if (p.kv.n_kv_heads < 1 || p.kv.head_dim < 1) refuse(c.what, "cache", "has no heads");      // shapes are divided by them
    const void* const at[] = {p.kv.k, p.kv.v, p.kv.k_scale, p.kv.v_scale};
    for (int i = 0; i < 4; ++i) {
        PyObject* const o = PyTuple_GET_ITEM(tensors, i);
        const void* now = nullptr;
        if (i < 2 || o != Py_None) {
            const at::Tensor& t = tensor(o, c.what, "cache");
            c.place(t, "cache");
            now = t.data_ptr();
        }
        if (now != at[i]) refuse(c.what, "cache", "has been moved");      // its layout is that of the tensors it was made from
    }
    const at::Tensor& b = tensor(table, c.what, "table");
    c.place(b, "table");
    if (b.dim() != 2 || b.scalar_type() != at::kInt) refuse(c.what, "table", "must be an int32 matrix");
    p.n_seqs = b.size(0);
    p.width = b.size(1);
    if (p.n_seqs > INT32_MAX || p.width > INT32_MAX) refuse(c.what, "table", "is too large");
    if (p.width > 1 && b.stride(1) != 1) refuse(c.what, "table", "must have contiguous rows");
    p.ld = p.n_seqs > 1 ? b.stride(0) : p.width;
    p.table = (const int32_t*)b.data_ptr();
    return p;
}
const int32_t* ints(Call& c, PyObject* o, const char* name, int64_t n, bool optional) {
    return optional && o == Py_None ? nullptr : (const int32_t*)vector(c, o, name, n, at::kInt, "must be int32");
}
float* floats_or_none(Call& c, PyObject* o, const char* name, int64_t n) { return o == Py_None ? nullptr : scales(c, o, name, n); }
double number(PyObject* o) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw Refused();
    return x;
}

// (tensors, desc, table, seq, pos, q, k, v, rope_base, q_out, status)
PyObject* py_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("cats_paged_append", n, 11, [&] {
        Call c{"cats_paged_append"};
        const Paged p = paged(c, a[0], a[1], a[2]);
        const int64_t hd = p.kv.head_dim, cols = p.kv.n_kv_heads * hd;
        const Matrix k = heads(c, a[6], "k", kAny, cols, hd, false), v = heads(c, a[7], "v", k.rows, cols, hd, false);
        const int32_t *seq = ints(c, a[3], "seq", k.rows, true), *pos = ints(c, a[4], "pos", k.rows, false);
        Matrix q, qo;
        if (a[5] != Py_None) {
            q = heads(c, a[5], "q", k.rows, kAny, hd, false);
            qo = heads(c, a[9], "q_out", k.rows, q.cols, hd, true);
            if (q.cols == 0 || q.cols % hd) refuse(c.what, "q", "has the wrong shape");
        }
        if (v.type != k.type || (q.p && q.type != k.type)) refuse(c.what, "q, k and v", "must have one type");
        if (!seq && k.rows > p.n_seqs) refuse(c.what, "k", "has more rows than the table has sequences");
        const double base = number(a[8]);
        int32_t* status = (int32_t*)vector(c, a[10], "status", 1, at::kInt, "must be int32");
        void* st = c.stream();
        return without_gil([&] {
            return f_append(&p.kv, p.table, p.ld, (int32_t)p.width, (int32_t)p.n_seqs, seq, pos, (int32_t)k.rows, q.p, q.ld, (int32_t)(q.cols / hd), k.p, k.ld, v.p,
                            v.ld, k.type, (float)base, qo.p, qo.ld, status, st);
        });
    });
}

// (tensors, desc, table, seq, pos, k_out, v_out, status)
PyObject* py_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("cats_paged_read", n, 8, [&] {
        Call c{"cats_paged_read"};
        const Paged p = paged(c, a[0], a[1], a[2]);
        const int64_t hd = p.kv.head_dim, cols = p.kv.n_kv_heads * hd;
        const Matrix k = heads(c, a[5], "k_out", kAny, cols, hd, false), v = heads(c, a[6], "v_out", k.rows, cols, hd, false);
        const int32_t *seq = ints(c, a[3], "seq", k.rows, true), *pos = ints(c, a[4], "pos", k.rows, false);
        if (v.type != k.type) refuse(c.what, "k_out and v_out", "must have one type");
        if (!seq && k.rows > p.n_seqs) refuse(c.what, "k_out", "has more rows than the table has sequences");
        int32_t* status = (int32_t*)vector(c, a[7], "status", 1, at::kInt, "must be int32");
        void* st = c.stream();
        return without_gil([&] {
            return f_read(&p.kv, p.table, p.ld, (int32_t)p.width, (int32_t)p.n_seqs, seq, pos, (int32_t)k.rows, k.p, k.ld, v.p, v.ld, k.type, status, st);
        });
    });
}

// (tensors, desc, table, lens, q, scale, out, ws, status)
PyObject* py_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("cats_paged_attention", n, 9, [&] {
        Call c{"cats_paged_attention"};
        const Paged p = paged(c, a[0], a[1], a[2]);
        const int64_t hd = p.kv.head_dim;
        const int32_t* len = ints(c, a[3], "lens", p.n_seqs, false);
        const Matrix q = heads(c, a[4], "q", p.n_seqs, kAny, hd, true), o = heads(c, a[6], "out", p.n_seqs, q.cols, hd, true);
        if (q.cols == 0 || q.cols % (hd * p.kv.n_kv_heads)) refuse(c.what, "q", "has the wrong shape");
        const double scale = number(a[5]);
        const at::Tensor& ws = tensor(a[7], c.what, "ws");
        void* const w = vector(c, a[7], "ws", kAny, at::kByte, "must be uint8");
        int32_t* status = (int32_t*)vector(c, a[8], "status", 1, at::kInt, "must be int32");
        const size_t bytes = (size_t)ws.numel();
        void* st = c.stream();
        return without_gil([&] {
            return f_attention(&p.kv, p.table, p.ld, (int32_t)p.width, len, (int32_t)p.n_seqs, q.p, q.ld, (int32_t)(q.cols / hd), (float)scale, o.p, o.ld, w, bytes,
                               status, st);
        });
    });
}

// (logits, row, temperature, top_k, top_p, min_p, u, token, prob, status)
PyObject* py_sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("cats_sample", n, 10, [&] {
        Call c{"cats_sample"};
        const Matrix x = matrix(c, a[0], "logits", kAny, kAny, true);
        const float* u = scales(c, a[6], "u", kAny);
        const int64_t rows = THPVariable_Unpack(a[6]).size(0);
        if (rows > INT32_MAX) refuse(c.what, "u", "is too large");
        const int32_t* row = ints(c, a[1], "row", rows, true);
        if (!row && rows > x.rows) refuse(c.what, "u", "has more draws than there are rows of logits");
        const float *t = floats_or_none(c, a[2], "temperature", rows), *top_p = floats_or_none(c, a[4], "top_p", rows), *min_p = floats_or_none(c, a[5], "min_p", rows);
        const int32_t* top_k = ints(c, a[3], "top_k", rows, true);
        int32_t* token = (int32_t*)vector(c, a[7], "token", rows, at::kInt, "must be int32");
        float* prob = floats_or_none(c, a[8], "prob", rows);
        int32_t* status = (int32_t*)vector(c, a[9], "status", 1, at::kInt, "must be int32");
        void* st = c.stream();
        return without_gil([&] {
            return f_sample(x.p, x.type, x.ld, (int32_t)x.rows, (int32_t)x.cols, row, (int32_t)rows, t, top_k, top_p, min_p, u, token, prob, status, st);
        });
    });
}

// bind(quantize, dequantize, rmsnorm, swiglu, linear, append, read, attention, sample): addresses of the loaded library's entry points
PyObject* py_bind(PyObject*, PyObject* args) {
    unsigned long long p[9];
    if (!PyArg_ParseTuple(args, "KKKKKKKKK", &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &p[6], &p[7], &p[8])) return nullptr;
    f_quantize = (decltype(f_quantize))p[0];
    f_dequantize = (decltype(f_dequantize))p[1];
    f_rmsnorm = (decltype(f_rmsnorm))p[2];
    f_swiglu = (decltype(f_swiglu))p[3];
    f_linear = (decltype(f_linear))p[4];
    f_append = (decltype(f_append))p[5];
    f_read = (decltype(f_read))p[6];
    f_attention = (decltype(f_attention))p[7];
    f_sample = (decltype(f_sample))p[8];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", py_bind, METH_VARARGS, nullptr},
    {"quantize_i8", (PyCFunction)(void (*)(void))py_quantize, METH_FASTCALL, nullptr},
    {"dequantize_i8", (PyCFunction)(void (*)(void))py_dequantize, METH_FASTCALL, nullptr},
    {"rmsnorm_i8", (PyCFunction)(void (*)(void))py_rmsnorm, METH_FASTCALL, nullptr},
    {"swiglu_i8", (PyCFunction)(void (*)(void))py_swiglu, METH_FASTCALL, nullptr},
    {"linear_i8", (PyCFunction)(void (*)(void))py_linear, METH_FASTCALL, nullptr},
    {"paged_append", (PyCFunction)(void (*)(void))py_append, METH_FASTCALL, nullptr},
    {"paged_read", (PyCFunction)(void (*)(void))py_read, METH_FASTCALL, nullptr},
    {"paged_attention", (PyCFunction)(void (*)(void))py_attention, METH_FASTCALL, nullptr},
    {"sample", (PyCFunction)(void (*)(void))py_sample, METH_FASTCALL, nullptr},
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
