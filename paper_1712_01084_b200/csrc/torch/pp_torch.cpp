// Fast entry to the decoder operators for PyTorch tensors: a call's checks, its new output tensors and the call of the C
// interface, in C++.  The operators take a few microseconds on the GPU, and the same steps in Python took longer than that
// (13 us for the 8-bit norm, whose three outputs alone cost 5).  Arguments are marshalled and nothing is computed here;
// the C functions' addresses come from the already loaded library (init).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "pp.h"

namespace {

decltype(&pp_rmsnorm_q8) g_rmsnorm_q8;
decltype(&pp_q4_forward) g_q4_forward;
decltype(&pp_moe_forward) g_moe_forward;

// A Python exception that is already set.
struct Raised {};
[[noreturn]] void raise(PyObject* type, const char* format, ...) {
    va_list va;
    va_start(va, format);
    PyErr_FormatV(type, format, va);
    va_end(va);
    throw Raised{};
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, "%s must be a tensor", name);
    return THPVariable_Unpack(o);
}
int number(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    if (v < INT32_MIN || v > INT32_MAX) raise(PyExc_ValueError, "%ld is out of range", v);
    return (int)v;
}
// An address; a closed handle is None, which the C functions refuse.
void* address(PyObject* o) {
    if (o == Py_None) return nullptr;
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Raised{};
    return p;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised{};
    return v != 0;
}
at::ScalarType dtype(PyObject* o, at::ScalarType none) {
    if (o == Py_None) return none;
    if (!THPDtype_Check(o)) raise(PyExc_TypeError, "out_dtype must be a torch dtype");
    return reinterpret_cast<THPDtype*>(o)->scalar_type;
}

// The library's number of an element type.
pp_dtype_t type_of(at::ScalarType t, const char* name) {
    switch (t) {
        case at::kFloat: return PP_F32;
        case at::kHalf: return PP_F16;
        case at::kBFloat16: return PP_BF16;
        case at::kChar: return PP_I8;
        case at::kFloat8_e4m3fn: return PP_E4M3;
        default: raise(PyExc_TypeError, "%s: %s is no type of the library", name, c10::toString(t));
    }
}

struct Rows { int rows; int64_t ld; };
// A CUDA matrix [rows][cols] whose rows are contiguous, any distance apart; a vector is one row.
Rows rows_of(const at::Tensor& x, int64_t cols, const char* name, int device) {
    const int64_t dims = x.dim();
    if (x.is_cuda() && device >= 0 && x.get_device() == device && (dims == 1 || dims == 2) && x.size(dims - 1) == cols) {
        const int64_t rows = dims == 2 ? x.size(0) : 1;
        if (rows <= INT32_MAX) {
            if (x.is_contiguous()) return {(int)rows, cols};
            if (dims == 2 && (cols == 1 || x.stride(1) == 1)) return {(int)rows, rows > 1 ? x.stride(0) : cols};
        }
    }
    raise(PyExc_ValueError, "%s must be a CUDA tensor [rows][%lld] with contiguous rows, on device %d", name, (long long)cols, device);
}

at::Tensor fresh(at::IntArrayRef shape, at::ScalarType t, int device) {
    return at::Tensor(at::detail::empty_cuda(shape, t, at::Device(at::kCUDA, (c10::DeviceIndex)device), std::nullopt));
}

// The device and the stream of a call, the given one or the current one.  The given one is made current until the call is over:
// a new tensor then comes from its own memory, and is not what an earlier tensor of another stream has just left with work on
// it still to come.
struct Enqueue {
    c10::cuda::CUDAGuard device;
    c10::cuda::OptionalCUDAStreamGuard given;
    void* stream;
    Enqueue(PyObject* o, int d) : device((c10::DeviceIndex)d) {
        if (o != Py_None) given.reset_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(address(o)), (c10::DeviceIndex)d));
        stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)d).stream();
    }
};

// An output tensor: the given one, checked, or a new one.
at::Tensor output(PyObject* out, PyObject* out_dtype, at::ScalarType standard, int64_t rows, int64_t cols, int device) {
    if (out == Py_None) return fresh({rows, cols}, dtype(out_dtype, standard), device);
    const at::Tensor& y = tensor(out, "out");
    if (!y.is_cuda() || y.get_device() != device || !y.is_contiguous() || y.numel() != rows * cols || (y.dim() == 2 && rows > 1 && y.size(0) != rows) ||
        (out_dtype != Py_None && y.scalar_type() != dtype(out_dtype, standard)))
        raise(PyExc_ValueError, "out must be a contiguous CUDA tensor [%lld][%lld] of out_dtype", (long long)rows, (long long)cols);
    return y;
}

template <typename F> PyObject* guarded(Py_ssize_t got, Py_ssize_t want, F body) {
    try {
        if (got != want) raise(PyExc_TypeError, "%zd arguments, %zd expected", got, want);
        return body();
    } catch (const Raised&) {
    } catch (const c10::OutOfMemoryError& e) {
        PyObject* torch = PyImport_ImportModule("torch");
        PyObject* type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
        if (type) PyErr_SetString(type, e.what_without_backtrace());
        Py_XDECREF(type);
        Py_XDECREF(torch);
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

PyObject* keep(PyObject* o) {
    Py_INCREF(o);
    return o;
}

// (x, weight, residual, eps, codes, group, hidden_out, normed, stream) -> (codes, scales, hidden[, normed]), or the status
PyObject* rmsnorm_q8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 9, [&]() -> PyObject* {
        const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "weight");
        const int device = x.is_cuda() ? (int)x.get_device() : -1;
        const int64_t cols = x.dim() ? x.size(-1) : 0;
        const Rows rx = rows_of(x, cols, "x", device);
        if (cols < 1 || cols > INT32_MAX) raise(PyExc_ValueError, "x must have columns");
        const at::ScalarType t = x.scalar_type();
        const pp_dtype_t dt = type_of(t, "x"), wt = type_of(w.scalar_type(), "weight");
        if (!w.is_cuda() || w.get_device() != device || w.dim() != 1 || w.numel() != cols || !w.is_contiguous())
            raise(PyExc_ValueError, "weight must be a contiguous CUDA tensor [%lld] on device %d", (long long)cols, device);
        pp_dtype_t code;
        at::ScalarType code_type;
        if (PyUnicode_Check(a[4]) && PyUnicode_CompareWithASCIIString(a[4], "e4m3") == 0) code = PP_E4M3, code_type = at::kFloat8_e4m3fn;
        else if (PyUnicode_Check(a[4]) && PyUnicode_CompareWithASCIIString(a[4], "int8") == 0) code = PP_I8, code_type = at::kChar;
        else raise(PyExc_ValueError, "codes must be 'e4m3' or 'int8'");
        const double eps = PyFloat_AsDouble(a[3]);
        if (eps == -1.0 && PyErr_Occurred()) throw Raised{};
        const int group = number(a[5]);
        const bool normed = truth(a[7]);
        const Enqueue on(a[8], device);

        const void* r = nullptr;
        Rows rr{0, 0}, rh{0, 0};
        if (a[2] != Py_None) {
            const at::Tensor& res = tensor(a[2], "residual");
            if (res.scalar_type() != t || res.sizes() != x.sizes()) raise(PyExc_TypeError, "residual must have x's shape and type");
            rr = rows_of(res, cols, "residual", device);
            r = res.const_data_ptr();
        }
        at::Tensor hidden;
        if (a[6] != Py_None) {
            hidden = tensor(a[6], "hidden_out");
            if (hidden.scalar_type() != t || hidden.sizes() != x.sizes()) raise(PyExc_TypeError, "hidden_out must have x's shape and type");
            rh = rows_of(hidden, cols, "hidden_out", device);
        } else if (r) {
            hidden = fresh(x.sizes(), t, device);
            rh.ld = cols;
        }
        const at::Tensor q = fresh(x.sizes(), code_type, device);
        const int64_t groups = group > 0 ? (cols + group - 1) / group : 1;
        const at::Tensor scales = x.dim() == 2 ? fresh({rx.rows, groups}, at::kFloat, device) : fresh({groups}, at::kFloat, device);
        const at::Tensor norm = normed ? fresh(x.sizes(), t, device) : at::Tensor();
        const pp_status_t st = g_rmsnorm_q8(x.const_data_ptr(), rx.ld, r, rr.ld, w.const_data_ptr(), dt, wt, rx.rows, (int)cols, (float)eps, code,
                                            group, q.data_ptr(), static_cast<float*>(scales.data_ptr()),
                                            hidden.defined() ? hidden.data_ptr() : nullptr, rh.ld, normed ? norm.data_ptr() : nullptr,
                                            on.stream);
        if (st != PP_OK) return PyLong_FromLong(st);
        PyObject* out = PyTuple_New(normed ? 4 : 3);
        if (!out) return nullptr;
        PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(q));
        PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(scales));
        PyTuple_SET_ITEM(out, 2, a[6] != Py_None ? keep(a[6]) : hidden.defined() ? THPVariable_Wrap(hidden) : keep(Py_None));
        if (normed) PyTuple_SET_ITEM(out, 3, THPVariable_Wrap(norm));
        return out;
    });
}

// (handle, M, N, device, x, act, x_scales, out_dtype, out, stream) -> out, or the status
PyObject* q4_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 10, [&]() -> PyObject* {
        const int64_t M = number(a[1]), N = number(a[2]);
        const int device = number(a[3]);
        const at::Tensor& x = tensor(a[4], "x");
        const Rows rx = rows_of(x, N, "x", device);
        const pp_dtype_t xt = type_of(x.scalar_type(), "x");
        const float* scales = nullptr;
        int x_group = 0;
        if (a[6] != Py_None) {
            const at::Tensor& s = tensor(a[6], "x_scales");
            const int64_t groups = (N + 127) / 128;
            if (s.numel() != rx.rows && s.numel() != rx.rows * groups)
                raise(PyExc_ValueError, "x_scales must hold 1 or %lld values per row of x", (long long)groups);
            if (!s.is_cuda() || s.get_device() != device || !s.is_contiguous() || s.scalar_type() != at::kFloat)
                raise(PyExc_ValueError, "x_scales must be a contiguous float32 CUDA tensor on device %d", device);
            x_group = s.numel() == rx.rows ? 0 : 128;
            if (x_group && rx.rows > 1 && s.dim() == 2 && s.size(0) != rx.rows)
                raise(PyExc_ValueError, "x_scales must be [%d][%lld]", rx.rows, (long long)groups);
            scales = static_cast<const float*>(s.const_data_ptr());
        }
        const Enqueue on(a[9], device);
        const at::Tensor y = output(a[8], a[7], at::kFloat, rx.rows, M, device);
        const pp_status_t st = g_q4_forward(static_cast<pp_q4_t*>(address(a[0])), x.const_data_ptr(), rx.ld, xt, scales, x_group, y.data_ptr(),
                                            type_of(y.scalar_type(), "out"), rx.rows, (pp_act_t)number(a[5]), on.stream);
        if (st != PP_OK) return PyLong_FromLong(st);
        return a[8] != Py_None ? keep(a[8]) : THPVariable_Wrap(y);
    });
}

// (handle, H, top_k, device, x, out_dtype, out, routing, stream) -> out or (out, ids, gates), or the status
PyObject* moe_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 9, [&]() -> PyObject* {
        const int64_t H = number(a[1]), top_k = number(a[2]);
        const int device = number(a[3]);
        const at::Tensor& x = tensor(a[4], "x");
        const Rows rx = rows_of(x, H, "x", device);
        const pp_dtype_t xt = type_of(x.scalar_type(), "x");
        const bool routing = truth(a[7]);
        const Enqueue on(a[8], device);
        const at::Tensor y = output(a[6], a[5], x.scalar_type(), rx.rows, H, device);
        at::Tensor ids, gates;
        if (routing) {
            ids = fresh({rx.rows, top_k}, at::kInt, device);
            gates = fresh({rx.rows, top_k}, at::kFloat, device);
        }
        const pp_status_t st = g_moe_forward(static_cast<pp_moe_t*>(address(a[0])), x.const_data_ptr(), rx.ld, xt, y.data_ptr(),
                                             type_of(y.scalar_type(), "out"), rx.rows, routing ? static_cast<int32_t*>(ids.data_ptr()) : nullptr,
                                             routing ? static_cast<float*>(gates.data_ptr()) : nullptr, on.stream);
        if (st != PP_OK) return PyLong_FromLong(st);
        PyObject* out = a[6] != Py_None ? keep(a[6]) : THPVariable_Wrap(y);
        if (!routing || !out) return out;
        PyObject* all = PyTuple_New(3);
        if (!all) {
            Py_DECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(all, 0, out);
        PyTuple_SET_ITEM(all, 1, THPVariable_Wrap(ids));
        PyTuple_SET_ITEM(all, 2, THPVariable_Wrap(gates));
        return all;
    });
}

// (address of pp_rmsnorm_q8, of pp_q4_forward, of pp_moe_forward)
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 3, [&]() -> PyObject* {
        g_rmsnorm_q8 = reinterpret_cast<decltype(g_rmsnorm_q8)>(address(a[0]));
        g_q4_forward = reinterpret_cast<decltype(g_q4_forward)>(address(a[1]));
        g_moe_forward = reinterpret_cast<decltype(g_moe_forward)>(address(a[2]));
        return keep(Py_None);
    });
}

PyMethodDef methods[] = {
    {"init", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(init)), METH_FASTCALL, nullptr},
    {"rmsnorm_q8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rmsnorm_q8)), METH_FASTCALL, nullptr},
    {"q4_forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(q4_forward)), METH_FASTCALL, nullptr},
    {"moe_forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(moe_forward)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pp_torch", "Decoder operators on PyTorch tensors.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pp_torch() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "made_for", PP_TORCH_VERSION) != 0) Py_CLEAR(m);
    return m;
}
