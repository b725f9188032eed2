// The way from a Python call to the C ABI, in native code: reads the tensors' device pointers, checks what binding.py
// checks and calls the library on torch's current stream.  A call of a small matrix is over on the GPU in about 4 us;
// reading five tensors, the stream and fifteen ctypes arguments in Python took 8 us of host time per call, which is
// what such calls were bound by (1,024 rows of 10 entries, N = 32: 9.6 us a call, 4 us of it kernel).
//
// Every function returns the library's status, or -1 if an argument is not what the quick way takes (no tensor, not on
// the GPU, another type or length): nothing has been done then, and binding.py's own checks say what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <initializer_list>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/sgap.h"

namespace {

constexpr int kNotTaken = -1;

struct Call {
    PyObject* const* arg;
    bool ok = true;

    int64_t number(int n)
    {
        PyObject* o = arg[n];
        if (!PyLong_CheckExact(o)) return ok = false, 0;
        int overflow = 0;
        const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
        if (overflow) ok = false;
        return v;
    }
    // a C int: what does not fit is not taken (ctypes would cut it off: left to the slow way)
    int small(int n)
    {
        const int64_t v = number(n);
        if (v != (int)v) ok = false;
        return (int)v;
    }
    const at::Tensor* tensor(int n)
    {
        if (!ok || !THPVariable_Check(arg[n])) return ok = false, nullptr;
        return &THPVariable_Unpack(arg[n]);
    }
    // device pointer of a contiguous tensor of `count` elements (null for an empty one)
    void* data(int n, at::ScalarType type, int64_t count)
    {
        const at::Tensor* t = tensor(n);
        if (!t) return nullptr;
        if (!t->is_cuda() || t->scalar_type() != type || t->numel() != count || !t->is_contiguous()) {
            ok = false;
            return nullptr;
        }
        return count ? t->data_ptr() : nullptr;
    }
    int32_t* ints(int n, int64_t count) { return static_cast<int32_t*>(data(n, at::kInt, count)); }
    float* floats(int n, int64_t count) { return static_cast<float*>(data(n, at::kFloat, count)); }
    int64_t length(int n)
    {
        const at::Tensor* t = tensor(n);
        return t ? t->numel() : 0;
    }
    int64_t number_or(int n, int64_t otherwise) { return arg[n] == Py_None ? otherwise : number(n); }
    // a torch stream; None: torch's current stream on the current device
    void* stream(int n)
    {
        if (!ok) return nullptr;
        if (arg[n] == Py_None) return c10::hip::getCurrentHIPStream().stream();
        PyObject* handle = PyObject_GetAttrString(arg[n], "cuda_stream");
        void* s = handle && PyLong_Check(handle) ? PyLong_AsVoidPtr(handle) : nullptr;
        if (!handle || !PyLong_Check(handle) || PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        Py_XDECREF(handle);
        return s;
    }
    // None, or a CUDA uint8 tensor
    void* workspace(int n, int64_t* bytes)
    {
        *bytes = 0;
        if (arg[n] == Py_None) return nullptr;
        const at::Tensor* t = tensor(n);
        if (!t) return nullptr;
        if (!t->is_cuda() || t->scalar_type() != at::kByte) {
            ok = false;
            return nullptr;
        }
        *bytes = t->numel();
        return *bytes ? t->data_ptr() : nullptr;
    }
    // the same, its bytes side by side: a tensor that repeats its elements has less memory than their number says
    void* whole_workspace(int n, int64_t* bytes)
    {
        void* p = workspace(n, bytes);
        if (ok && arg[n] != Py_None && !tensor(n)->is_contiguous()) ok = false;
        return p;
    }
};

struct Matrix {
    int64_t M, K, N, nnz;
    const int32_t *rowptr, *colidx;
    const float *vals, *B;
    float* C;
    // arguments 0 .. 7: M, K, N, rowptr, colidx, vals, B, C
    explicit Matrix(Call& c)
    {
        M = c.number(0); K = c.number(1); N = c.number(2);
        if (!c.ok || M < 0 || K < 0 || N < 0 || M > INT32_MAX || K > INT32_MAX || N > INT32_MAX) {
            c.ok = false;
            return;
        }
        nnz = c.length(4);
        rowptr = c.ints(3, M + 1);
        colidx = c.ints(4, nnz);
        vals = c.floats(5, nnz);
        B = c.floats(6, K * N);
        C = c.floats(7, M * N);
    }
};

struct Rows {
    void* data;
    int64_t ld;
};

// the calls' element types
int element_type(at::ScalarType t)
{
    return t == at::kFloat ? SGAP_F32 : t == at::kHalf ? SGAP_F16 : t == at::kBFloat16 ? SGAP_BF16 : -1;
}

// a matrix of rows x columns whose rows lie side by side at any distance
Rows rows_of(Call& c, int n, at::ScalarType type, int64_t rows, int64_t columns)
{
    const at::Tensor* t = c.tensor(n);
    if (!t) return {nullptr, 0};
    if (!t->is_cuda() || t->scalar_type() != type || t->dim() != 2 || t->size(0) != rows || t->size(1) != columns ||
        (columns > 1 && t->stride(1) != 1) || (rows > 1 && t->stride(0) < columns)) {
        c.ok = false;
        return {nullptr, 0};
    }
    return {t->numel() ? t->data_ptr() : nullptr, rows > 1 ? t->stride(0) : columns};
}

at::ScalarType type_of(Call& c, int n)
{
    const at::Tensor* t = c.tensor(n);
    if (!t) return at::kFloat;
    if (element_type(t->scalar_type()) < 0) c.ok = false;
    return t->scalar_type();
}

PyObject* status(int st) { return PyLong_FromLong(st); }

// the library call itself, without the interpreter's lock: a launch may wait for room in the queue
template <typename F>
PyObject* enqueue(F&& f)
{
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return status(st);
}

// M, K, N, rowptr, colidx, vals, B, C, group_size, strategy, schedule, nnz_hint, stream; sgap_ttm_csf has the same
// arguments with fibers for rows, and forwards to the same code in the library
PyObject* spmm_csr_ex(PyObject*, PyObject* const* arg, Py_ssize_t n)
{
    Call c{arg};
    if (n != 13) return status(kNotTaken);
    const Matrix m(c);
    const int group = c.small(8), strategy = c.small(9), schedule = c.small(10);
    const int64_t hint = c.number_or(11, m.nnz);
    void* stream = c.stream(12);
    if (!c.ok) return status(kNotTaken);
    return enqueue([&] {
        return sgap_spmm_csr_ex(m.M, m.K, m.N, m.rowptr, m.colidx, m.vals, m.B, m.C, group, strategy, schedule, hint,
                                   stream);
    });
}

// M, K, N, rowptr, colidx, vals, B, C, config, nnz_hint, workspace, stream
PyObject* spmm_csr_cfg(PyObject*, PyObject* const* arg, Py_ssize_t n)
{
    Call c{arg};
    if (n != 12) return status(kNotTaken);
    const Matrix m(c);
    const int64_t hint = c.number_or(9, m.nnz);
    int64_t bytes = 0;
    void* ws = c.workspace(10, &bytes);
    void* stream = c.stream(11);
    if (!c.ok) return status(kNotTaken);
    Py_buffer config;  // a ctypes structure lends its memory
    if (PyObject_GetBuffer(arg[8], &config, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        return status(kNotTaken);
    }
    PyObject* st = config.len != (Py_ssize_t)sizeof(sgap_config) ? status(kNotTaken) : enqueue([&] {
        return sgap_spmm_csr_cfg(m.M, m.K, m.N, m.rowptr, m.colidx, m.vals, m.B, m.C,
                                 static_cast<const sgap_config*>(config.buf), hint, ws, bytes, stream);
    });
    PyBuffer_Release(&config);
    return st;
}

struct Sampled {
    int64_t M, K, J, nnz;
    const int32_t *rowptr, *colidx;
    const float *vals, *X1, *X2T;
    float* out;
    // arguments 0 .. 8: M, K, J, rowptr, colidx, vals, X1, X2T, out_vals
    explicit Sampled(Call& c)
    {
        M = c.number(0); K = c.number(1); J = c.number(2);
        if (!c.ok || M < 0 || K < 0 || J < 0 || M > INT32_MAX || K > INT32_MAX || J > INT32_MAX) {
            c.ok = false;
            return;
        }
        nnz = c.length(4);
        rowptr = c.ints(3, M + 1);
        colidx = c.ints(4, nnz);
        vals = c.floats(5, nnz);
        X1 = c.floats(6, M * J);
        X2T = c.floats(7, K * J);
        out = c.floats(8, nnz);
    }
};

// M, K, J, rowptr, colidx, vals, X1, X2T, out_vals, group_size, strategy, nnz_hint, stream
PyObject* sddmm_csr(PyObject*, PyObject* const* arg, Py_ssize_t n)
{
    Call c{arg};
    if (n != 13) return status(kNotTaken);
    const Sampled s(c);
    const int group = c.small(9), strategy = c.small(10);
    const int64_t hint = c.number_or(11, s.nnz);
    void* stream = c.stream(12);
    if (!c.ok) return status(kNotTaken);
    return enqueue([&] {
        return sgap_sddmm_csr(s.M, s.K, s.J, s.rowptr, s.colidx, s.vals, s.X1, s.X2T, s.out, group, strategy, hint,
                                 stream);
    });
}

// ..., group_size, strategy, nnz_hint, long_row_min, window_kb, max_long_rows, workspace, stream
PyObject* sddmm_csr_windows(PyObject*, PyObject* const* arg, Py_ssize_t n)
{
    Call c{arg};
    if (n != 17) return status(kNotTaken);
    const Sampled s(c);
    const int group = c.small(9), strategy = c.small(10);
    const int64_t hint = c.number_or(11, s.nnz);
    const int long_row_min = c.small(12), window_kb = c.small(13), max_long_rows = c.small(14);
    int64_t bytes = 0;
    void* ws = c.workspace(15, &bytes);
    void* stream = c.stream(16);
    if (!c.ok) return status(kNotTaken);
    return enqueue([&] {
        return sgap_sddmm_csr_windows(s.M, s.K, s.J, s.rowptr, s.colidx, s.vals, s.X1, s.X2T, s.out, group, strategy,
                                         hint, long_row_min, window_kb, max_long_rows, ws, bytes, stream);
    });
}

// I, K, L, J, fptr, fidx, eptr, eidx, vals, X1, X2, Y, group_size, strategy, schedule, nnz_hint, stream
PyObject* mttkrp_csf_ex(PyObject*, PyObject* const* arg, Py_ssize_t n)
{
    Call c{arg};
    if (n != 17) return status(kNotTaken);
    const int64_t I = c.number(0), K = c.number(1), L = c.number(2), J = c.number(3);
    if (!c.ok || I < 0 || K < 0 || L < 0 || J < 0 || I > INT32_MAX || K > INT32_MAX || L > INT32_MAX || J > INT32_MAX)
        return status(kNotTaken);
    const int64_t fibers = c.length(5), nnz = c.length(8);
    const int32_t *fptr = c.ints(4, I + 1), *fidx = c.ints(5, fibers), *eptr = c.ints(6, fibers + 1), *eidx = c.ints(7, nnz);
    const float *vals = c.floats(8, nnz), *X1 = c.floats(9, K * J), *X2 = c.floats(10, L * J);
    float* Y = c.floats(11, I * J);
    const int group = c.small(12), strategy = c.small(13), schedule = c.small(14);
    const int64_t hint = c.number_or(15, nnz);
    void* stream = c.stream(16);
    if (!c.ok) return status(kNotTaken);
    return enqueue([&] {
        return sgap_mttkrp_csf_ex(I, K, L, J, fptr, fidx, eptr, eidx, vals, X1, X2, Y, group, strategy, schedule, hint,
                                     stream);
    });
}

bool sizes_ok(Call& c, std::initializer_list<int64_t> sizes)
{
    for (int64_t v : sizes)
        if (v < 0 || v > INT32_MAX) c.ok = false;
    return c.ok;
}

// T, E, k, logits, gates, experts, slot, order, offsets, renormalise, workspace, stream
PyObject* route_topk(PyObject*, PyObject* const* arg, Py_ssize_t n)
{
    Call c{arg};
    if (n != 12) return status(kNotTaken);
    const int64_t T = c.number(0), E = c.number(1), k = c.number(2);
    if (!sizes_ok(c, {T, E, k})) return status(kNotTaken);
    const at::ScalarType type = type_of(c, 3);
    const Rows logits = rows_of(c, 3, type, T, E);
    float* gates = c.floats(4, T * k);
    int32_t *experts = c.ints(5, T * k), *slot = c.ints(6, T * k), *order = c.ints(7, T * k), *offsets = c.ints(8, E + 1);
    const int renormalise = c.small(9);
    int64_t bytes = 0;
    void* ws = c.whole_workspace(10, &bytes);
    void* stream = c.stream(11);
    if (!c.ok) return status(kNotTaken);
    return enqueue([&] {
        return sgap_route_topk(T, E, k, element_type(type), logits.data, logits.ld, renormalise, gates, experts, slot, order,
                               offsets, ws, bytes, stream);
    });
}

// T, E, k, logits, gates, experts, dgates, dlogits, renormalise, stream
PyObject* route_topk_grad(PyObject*, PyObject* const* arg, Py_ssize_t n)
{
    Call c{arg};
    if (n != 10) return status(kNotTaken);
    const int64_t T = c.number(0), E = c.number(1), k = c.number(2);
    if (!sizes_ok(c, {T, E, k})) return status(kNotTaken);
    const at::ScalarType type = type_of(c, 3);
    const Rows logits = rows_of(c, 3, type, T, E), dlogits = rows_of(c, 7, type, T, E);
    const float *gates = c.floats(4, T * k), *dgates = c.floats(6, T * k);
    const int32_t* experts = c.ints(5, T * k);
    const int renormalise = c.small(8);
    void* stream = c.stream(9);
    if (!c.ok) return status(kNotTaken);
    return enqueue([&] {
        return sgap_route_topk_grad(T, E, k, element_type(type), logits.data, logits.ld, renormalise, gates, experts, dgates,
                                    dlogits.data, dlogits.ld, stream);
    });
}

// T, k, D, Z, slot, gates or None, out, stream
PyObject* route_combine(PyObject*, PyObject* const* arg, Py_ssize_t n)
{
    Call c{arg};
    if (n != 8) return status(kNotTaken);
    const int64_t T = c.number(0), k = c.number(1), D = c.number(2);
    if (!sizes_ok(c, {T, k, D})) return status(kNotTaken);
    const at::ScalarType type = type_of(c, 3);
    const void* Z = c.data(3, type, T * k * D);
    const int32_t* slot = c.ints(4, T * k);
    const float* gates = arg[5] == Py_None ? nullptr : c.floats(5, T * k);
    void* out = c.data(6, type, T * D);
    void* stream = c.stream(7);
    if (!c.ok) return status(kNotTaken);
    return enqueue([&] { return sgap_route_combine(T, k, D, element_type(type), Z, slot, gates, out, stream); });
}

// T, k, D, Z, slot, order, gates, dout, dZ, dgates, stream
PyObject* route_combine_grad(PyObject*, PyObject* const* arg, Py_ssize_t n)
{
    Call c{arg};
    if (n != 11) return status(kNotTaken);
    const int64_t T = c.number(0), k = c.number(1), D = c.number(2);
    if (!sizes_ok(c, {T, k, D})) return status(kNotTaken);
    const at::ScalarType type = type_of(c, 3);
    const void *Z = c.data(3, type, T * k * D), *dout = c.data(7, type, T * D);
    const int32_t *slot = c.ints(4, T * k), *order = c.ints(5, T * k);
    const float* gates = c.floats(6, T * k);
    void* dZ = c.data(8, type, T * k * D);
    float* dgates = c.floats(9, T * k);
    void* stream = c.stream(10);
    if (!c.ok) return status(kNotTaken);
    return enqueue([&] {
        return sgap_route_combine_grad(T, k, D, element_type(type), Z, slot, order, gates, dout, dZ, dgates, stream);
    });
}

// the rows that a product over groups takes
struct Grouped {
    int64_t G, R, K, N, x_rows = 0, src_div;
    at::ScalarType type;
    const int32_t *offsets, *src;
    Rows X;
    // arguments 0 .. 3: G, R, K, N; then the places of offsets, X, src and src_div
    Grouped(Call& c, int offsets_at, int x_at, int src_at)
    {
        G = c.number(0); R = c.number(1); K = c.number(2); N = c.number(3);
        if (!sizes_ok(c, {G, R, K, N})) return;
        offsets = c.arg[offsets_at] == Py_None ? nullptr : c.ints(offsets_at, G + 1);
        type = type_of(c, x_at);
        const at::Tensor* x = c.tensor(x_at);
        if (x && x->dim() == 2) x_rows = x->size(0);
        X = rows_of(c, x_at, type, x_rows, K);
        src = c.arg[src_at] == Py_None ? nullptr : c.ints(src_at, R);
        src_div = c.number(src_at + 1);
    }
};

// G, R, K, N, offsets or None, X, W, Y, layout, src or None, src_div, stream
PyObject* grouped_mm(PyObject*, PyObject* const* arg, Py_ssize_t n)
{
    Call c{arg};
    if (n != 12) return status(kNotTaken);
    const Grouped m(c, 4, 5, 9);
    if (!c.ok) return status(kNotTaken);
    const void* W = c.data(6, m.type, m.G * m.K * m.N);
    const Rows Y = rows_of(c, 7, m.type, m.R, m.N);
    const int layout = c.small(8);
    void* stream = c.stream(11);
    if (!c.ok) return status(kNotTaken);
    return enqueue([&] {
        return sgap_grouped_mm(m.G, m.R, m.K, m.N, element_type(m.type), m.offsets, m.X.data, m.X.ld, m.x_rows, m.src, m.src_div,
                               W, layout, Y.data, Y.ld, stream);
    });
}

// G, R, K, N, offsets or None, X, dY, dW, layout, src or None, src_div, stream
PyObject* grouped_mm_wgrad(PyObject*, PyObject* const* arg, Py_ssize_t n)
{
    Call c{arg};
    if (n != 12) return status(kNotTaken);
    const Grouped m(c, 4, 5, 9);
    if (!c.ok) return status(kNotTaken);
    const Rows dY = rows_of(c, 6, m.type, m.R, m.N);
    void* dW = c.data(7, m.type, m.G * m.K * m.N);
    const int layout = c.small(8);
    void* stream = c.stream(11);
    if (!c.ok) return status(kNotTaken);
    return enqueue([&] {
        return sgap_grouped_mm_wgrad(m.G, m.R, m.K, m.N, element_type(m.type), m.offsets, m.X.data, m.X.ld, m.x_rows, m.src,
                                     m.src_div, dY.data, dY.ld, dW, layout, stream);
    });
}

// G, R, K, N, group_k, offsets or None, X, weights, Y, zeros, src or None, src_div, stream
PyObject* grouped_mm_w4(PyObject*, PyObject* const* arg, Py_ssize_t n)
{
    Call c{arg};
    if (n != 13) return status(kNotTaken);
    const Grouped m(c, 5, 6, 10);
    if (!c.ok) return status(kNotTaken);
    const int64_t group_k = c.number(4);
    int64_t bytes = 0;
    const void* weights = c.whole_workspace(7, &bytes);
    const Rows Y = rows_of(c, 8, m.type, m.R, m.N);
    const int zeros = c.small(9);
    void* stream = c.stream(12);
    if (!c.ok || m.type == at::kFloat) return status(kNotTaken);
    return enqueue([&] {
        return sgap_grouped_mm_w4(m.G, m.R, m.K, m.N, element_type(m.type), group_k, zeros, m.offsets, m.X.data, m.X.ld, m.x_rows,
                                  m.src, m.src_div, weights, bytes, Y.data, Y.ld, stream);
    });
}

PyMethodDef kMethods[] = {
    {"spmm_csr_ex", (PyCFunction)(void (*)())spmm_csr_ex, METH_FASTCALL, nullptr},
    {"spmm_csr_cfg", (PyCFunction)(void (*)())spmm_csr_cfg, METH_FASTCALL, nullptr},
    {"sddmm_csr", (PyCFunction)(void (*)())sddmm_csr, METH_FASTCALL, nullptr},
    {"sddmm_csr_windows", (PyCFunction)(void (*)())sddmm_csr_windows, METH_FASTCALL, nullptr},
    {"mttkrp_csf_ex", (PyCFunction)(void (*)())mttkrp_csf_ex, METH_FASTCALL, nullptr},
    {"route_topk", (PyCFunction)(void (*)())route_topk, METH_FASTCALL, nullptr},
    {"route_topk_grad", (PyCFunction)(void (*)())route_topk_grad, METH_FASTCALL, nullptr},
    {"route_combine", (PyCFunction)(void (*)())route_combine, METH_FASTCALL, nullptr},
    {"route_combine_grad", (PyCFunction)(void (*)())route_combine_grad, METH_FASTCALL, nullptr},
    {"grouped_mm", (PyCFunction)(void (*)())grouped_mm, METH_FASTCALL, nullptr},
    {"grouped_mm_wgrad", (PyCFunction)(void (*)())grouped_mm_wgrad, METH_FASTCALL, nullptr},
    {"grouped_mm_w4", (PyCFunction)(void (*)())grouped_mm_w4, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&kModule); }
