// Python's way to the calls on rows (geocache_add_rms_norm, geocache_quantize_rows, geocache_linear): checks that the
// tensors are what the C call will read and write, and marshals them.  A call on a few rows takes 2 to 5 us on the GPU;
// reading its tensors' attributes from Python took 4 to 6 us, here it takes 0.2.
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "geocache.h"

namespace {

struct Raised {};   // a Python exception is set

const char* name_of(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return "torch.float32";
        case at::kBFloat16: return "torch.bfloat16";
        case at::kHalf: return "torch.float16";
        case at::kFloat8_e4m3fn: return "torch.float8_e4m3fn";
        default: return c10::toString(t);
    }
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a torch tensor", name);
        throw Raised();
    }
    return THPVariable_Unpack(o);
}

// The kernels run on the current device (asked for once a call), whose memory is all that they can reach.
thread_local c10::DeviceIndex g_device = 0;
bool elsewhere(const at::Tensor& t) { return t.device().index() != g_device; }

// [T, C] rows of one type on the device, whose elements are consecutive
geocache_rows rows(PyObject* o, at::ScalarType type, int64_t T, int64_t C, const char* name) {
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_TypeError, "%s must be %s (got %s)", name, name_of(type), name_of(t.scalar_type()));
    } else if (!t.is_cuda()) {
        PyErr_Format(PyExc_ValueError, "%s must be on a CUDA device", name);
    } else if (elsewhere(t)) {
        PyErr_Format(PyExc_ValueError, "%s must be on the current device", name);
    } else if (t.dim() != 2 || t.size(0) != T || t.size(1) != C) {
        PyErr_Format(PyExc_ValueError, "%s must be [%lld, %lld]", name, (long long)T, (long long)C);
    } else if (t.stride(1) != 1 && C != 1) {
        PyErr_Format(PyExc_ValueError, "the elements of a row of %s must be consecutive", name);
    } else {
        return {t.data_ptr(), t.stride(0)};
    }
    throw Raised();
}

// n consecutive f32 on the device, or None
float* vector(PyObject* o, int64_t n, const char* name) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, name);
    if (!t.is_cuda()) {
        PyErr_Format(PyExc_ValueError, "%s must be on a CUDA device", name);
    } else if (elsewhere(t)) {
        PyErr_Format(PyExc_ValueError, "%s must be on the current device", name);
    } else if (t.scalar_type() != at::kFloat) {
        PyErr_Format(PyExc_TypeError, "%s must be torch.float32 (got %s)", name, name_of(t.scalar_type()));
    } else if (!t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s must be contiguous", name);
    } else if (t.numel() != n) {
        PyErr_Format(PyExc_ValueError, "%s has %lld elements, expected %lld", name, (long long)t.numel(), (long long)n);
    } else {
        return static_cast<float*>(t.data_ptr());
    }
    throw Raised();
}

// a type of the C interface; rows of 8 bits where they are allowed
geocache_dtype dtype(const at::Tensor& t, bool eight, bool f32, const char* name, const char* allowed) {
    switch (t.scalar_type()) {
        case at::kFloat:
            if (f32) return GEOCACHE_F32;
            break;
        case at::kBFloat16: return GEOCACHE_BF16;
        case at::kHalf: return GEOCACHE_F16;
        case at::kFloat8_e4m3fn:
            if (eight) return GEOCACHE_E4M3;
            break;
        default: break;
    }
    PyErr_Format(PyExc_TypeError, "%s must be %s (got %s)", name, allowed, name_of(t.scalar_type()));
    throw Raised();
}

void two_axes(const at::Tensor& t, const char* name) {
    if (t.dim() == 2) return;
    PyErr_Format(PyExc_ValueError, "%s must have two axes (has %lld)", name, (long long)t.dim());
    throw Raised();
}

int size32(int64_t n, const char* name) {
    if (n >= 0 && n <= INT32_MAX) return (int)n;
    PyErr_Format(PyExc_ValueError, "%s=%lld must be a 32-bit integer", name, (long long)n);
    throw Raised();
}

void count(Py_ssize_t n, Py_ssize_t expected) {
    if (n == expected) return;
    PyErr_Format(PyExc_TypeError, "%zd arguments, expected %zd", n, expected);
    throw Raised();
}

int64_t integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}

// a stream's handle, or the current one of the calling thread for None
void* stream_of(PyObject* o) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    return reinterpret_cast<void*>(integer(o));
}

template <typename F>
PyObject* status(F call) {
    try {
        int r;
        if (c10::cuda::GetDevice(&g_device) != cudaSuccess) g_device = -1;   // (without a device no tensor is on one)
        const auto launch = call();
        Py_BEGIN_ALLOW_THREADS
        r = launch();
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(r);
    } catch (const Raised&) {
    } catch (const std::exception& e) {   // (a tensor without memory)
        PyErr_SetString(PyExc_ValueError, e.what());
    }
    return nullptr;
}

const char* kWhole = "float32, bfloat16 or float16";

// (x, residual, weight, eps, out, scale, residual_out, stream)
PyObject* add_rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return status([=] {
        count(n, 8);
        const at::Tensor& x = tensor(a[0], "x");
        const geocache_dtype type = dtype(x, false, true, "x", kWhole);
        two_axes(x, "x");
        const int64_t T = x.size(0);
        const int C = size32(x.size(1), "C");
        const geocache_rows from = rows(a[0], x.scalar_type(), T, C, "x");
        const geocache_rows to = rows(a[4], a[5] == Py_None ? x.scalar_type() : at::kFloat8_e4m3fn, T, C, "out");
        geocache_rows residual{}, residual_out{};
        geocache_dtype residual_type = type;
        const bool has = a[1] != Py_None;
        if (has) {
            const at::Tensor& r = tensor(a[1], "residual");
            if (r.scalar_type() != x.scalar_type() && r.scalar_type() != at::kFloat) {
                PyErr_Format(PyExc_TypeError, "residual must be %s or torch.float32 (got %s)", name_of(x.scalar_type()), name_of(r.scalar_type()));
                throw Raised();
            }
            if (r.scalar_type() == at::kFloat) residual_type = GEOCACHE_F32;
            residual = rows(a[1], r.scalar_type(), T, C, "residual");
            residual_out = rows(a[6], r.scalar_type(), T, C, "residual_out");
        } else if (a[6] != Py_None) {
            PyErr_SetString(PyExc_ValueError, "residual_out without residual");
            throw Raised();
        }
        const float* weight = vector(a[2], C, "weight");
        float* scale = vector(a[5], T, "scale");
        const double eps = PyFloat_AsDouble(a[3]);
        if (eps == -1.0 && PyErr_Occurred()) throw Raised();
        void* stream = stream_of(a[7]);
        return [=] {
            return geocache_add_rms_norm(&from, has ? &residual : nullptr, has ? &residual_out : nullptr, &to, T, C, type, residual_type,
                                         weight, eps, scale, stream);
        };
    });
}

// (x, out, scale, stream)
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return status([=] {
        count(n, 4);
        const at::Tensor& x = tensor(a[0], "x");
        const geocache_dtype type = dtype(x, false, true, "x", kWhole);
        two_axes(x, "x");
        const int64_t T = x.size(0);
        const int C = size32(x.size(1), "C");
        const geocache_rows from = rows(a[0], x.scalar_type(), T, C, "x"), to = rows(a[1], at::kFloat8_e4m3fn, T, C, "out");
        float* scale = vector(a[2], T, "scale");
        void* stream = stream_of(a[3]);
        return [=] { return geocache_quantize_rows(&from, &to, T, C, type, scale, stream); };
    });
}

// (x, weight, bias, activation, gated, residual, x_scale, weight_scale, out, stream)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return status([=] {
        count(n, 10);
        const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "weight"), &out = tensor(a[8], "out");
        two_axes(x, "x");
        two_axes(w, "weight");
        const int64_t T = x.size(0), features = w.size(0);
        const int K = size32(x.size(1), "K"), gated = PyObject_IsTrue(a[4]);
        if (gated < 0) throw Raised();
        if (gated && features % 2) {
            PyErr_Format(PyExc_ValueError, "a gated product has an even number of weight rows (got %lld)", (long long)features);
            throw Raised();
        }
        const geocache_dtype type = dtype(x, true, false, "x", "bfloat16, float16 or float8_e4m3fn");
        const geocache_dtype out_type = dtype(out, false, true, "out", kWhole);
        const int N = size32(gated ? features / 2 : features, "N");
        const geocache_rows from = rows(a[0], x.scalar_type(), T, K, "x"), weight = rows(a[1], x.scalar_type(), features, K, "weight"),
                            to = rows(a[8], out.scalar_type(), T, N, "out");
        const bool has = a[5] != Py_None;
        geocache_rows residual{};
        if (has) residual = rows(a[5], out.scalar_type(), T, N, "residual");
        const float *bias = vector(a[2], features, "bias"), *x_scale = vector(a[6], T, "x_scale"),
                    *weight_scale = vector(a[7], features, "weight_scale");
        const geocache_activation act = (geocache_activation)integer(a[3]);
        void* stream = stream_of(a[9]);
        return [=] {
            return geocache_linear(&from, &weight, has ? &residual : nullptr, &to, T, K, N, type, out_type, act, gated, bias, x_scale,
                                   weight_scale, stream);
        };
    });
}

PyMethodDef methods[] = {
    {"add_rms_norm", reinterpret_cast<PyCFunction>(add_rms_norm), METH_FASTCALL, nullptr},
    {"quantize_rows", reinterpret_cast<PyCFunction>(quantize_rows), METH_FASTCALL, nullptr},
    {"linear", reinterpret_cast<PyCFunction>(linear), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "geocache_rows_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_geocache_rows_binding() { return PyModule_Create(&module); }
