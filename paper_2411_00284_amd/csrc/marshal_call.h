// What the marshallers of the operators share: a call's tensors and their checks,
// its stream, its workspace, and the way back to Python.
#pragma once

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Device.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>

#include "fsdp_block.h"

namespace {

// A Python error is set; unwinds to the entry point.
struct Raised {};

[[noreturn]] void raise(PyObject* type, const char* format, ...) {
    va_list args;
    va_start(args, format);
    PyErr_FormatV(type, format, args);
    va_end(args);
    throw Raised();
}

int code_of(at::ScalarType t) {
    return t == at::kBFloat16 ? FSDP_DTYPE_BF16 : t == at::kFloat ? FSDP_DTYPE_F32 : t == at::kHalf ? FSDP_DTYPE_F16 : -1;
}

const char* name_of(fsdp_dtype t) { return t == FSDP_DTYPE_BF16 ? "bf16" : t == FSDP_DTYPE_F16 ? "f16" : "f32"; }

// One call's tensors: all on one device.
class Call {
public:
    // The tensor of an argument; NULL for None where that is allowed.
    const at::Tensor* tensor(PyObject* o, const char* name, bool needed) {
        if (o == Py_None && !needed) return nullptr;
        if (!THPVariable_Check(o)) raise(PyExc_TypeError, "%s must be a tensor", name);
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda()) {
            // an empty tensor has no memory that could be on the wrong device
            if (t.numel() != 0) raise(PyExc_ValueError, "%s must be a device tensor", name);
            return &t;
        }
        const int device = t.device().index();
        if (device_ < 0) device_ = device;
        if (device != device_)
            raise(PyExc_ValueError, "%s is on device %d where %d is expected: one call's tensors and stream must share one device",
                  name, device, device_);
        return &t;
    }

    fsdp_dtype dtype(const at::Tensor& t, const char* name) {
        const int code = code_of(t.scalar_type());
        if (code < 0) raise(PyExc_TypeError, "%s must be of dtype bfloat16, float16 or float32", name);
        return code;
    }
    void dtype(const at::Tensor& t, const char* name, fsdp_dtype want) {
        if (code_of(t.scalar_type()) != want) raise(PyExc_TypeError, "%s must be of dtype %s", name, name_of(want));
    }

    // A matrix [rows, cols] with contiguous columns: its pointer and row stride.
    void* matrix(const at::Tensor* t, const char* name, int64_t rows, int64_t cols, int64_t* stride) {
        *stride = cols;
        if (!t) return nullptr;
        if (t->dim() != 2 || t->size(0) != rows || t->size(1) != cols)
            raise(PyExc_ValueError, "%s must have the shape (%lld, %lld)", name, (long long)rows, (long long)cols);
        if (rows == 0 || cols == 0) return nullptr;
        if (cols > 1 && t->stride(1) != 1) raise(PyExc_ValueError, "%s must have contiguous columns", name);
        if (rows > 1) *stride = t->stride(0);
        if (*stride < cols) raise(PyExc_ValueError, "%s: its rows overlap", name);
        return t->data_ptr();
    }
    void* vector(const at::Tensor* t, const char* name, int64_t n) {
        if (!t) return nullptr;
        if (t->dim() != 1 || t->size(0) != n) raise(PyExc_ValueError, "%s must have the shape (%lld,)", name, (long long)n);
        if (n > 1 && t->stride(0) != 1) raise(PyExc_ValueError, "%s must be contiguous", name);
        return n == 0 ? nullptr : t->data_ptr();
    }

    // The HIP stream of `o` (torch's current stream of the tensors' device for None).
    hipStream_t stream(PyObject* o) {
        if (o == Py_None) {
            const auto current = c10::hip::getCurrentHIPStream(c10::DeviceIndex(device_ < 0 ? c10::hip::current_device() : device_));
            if (device_ < 0) device_ = current.device_index();
            return current.stream();
        }
        if (PyLong_Check(o)) {
            if (device_ < 0) device_ = c10::hip::current_device();
            void* const handle = PyLong_AsVoidPtr(o);
            if (PyErr_Occurred()) throw Raised();
            return static_cast<hipStream_t>(handle);
        }
        PyObject* handle = PyObject_GetAttrString(o, "cuda_stream");
        PyObject* device = handle ? PyObject_GetAttrString(o, "device") : nullptr;
        const bool fine = device && PyLong_Check(handle) && THPDevice_Check(device);
        void* const s = fine ? PyLong_AsVoidPtr(handle) : nullptr;
        const int index = fine ? reinterpret_cast<THPDevice*>(device)->device.index() : -1;
        Py_XDECREF(handle);
        Py_XDECREF(device);
        if (PyErr_Occurred()) PyErr_Clear();
        if (!fine) raise(PyExc_TypeError, "stream must be a torch stream, a stream handle or None");
        if (device_ < 0) device_ = index;
        if (index != device_)
            raise(PyExc_ValueError, "the stream is on device %d, the tensors are on %d: one call's tensors and stream must share one device",
                  index, device_);
        return static_cast<hipStream_t>(s);
    }

    int device() const { return device_; }

private:
    int device_ = -1;
};

class Workspace {
public:
    Workspace(int64_t bytes, hipStream_t stream) : bytes_(bytes) {
        if (bytes > 0) p_ = c10::hip::HIPCachingAllocator::raw_alloc_with_stream(size_t(bytes), stream);
    }
    ~Workspace() {
        if (p_) c10::hip::HIPCachingAllocator::raw_delete(p_);
    }
    Workspace(const Workspace&) = delete;
    Workspace& operator=(const Workspace&) = delete;
    void* data() const { return p_; }
    int64_t bytes() const { return bytes_; }

private:
    void* p_ = nullptr;
    int64_t bytes_;
};

double number(PyObject* o, const char* name) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        raise(PyExc_TypeError, "%s must be a number", name);
    }
    return v;
}

// Runs `f`, which returns a status, on the device of the call's tensors.
template <typename F>
PyObject* entry(Py_ssize_t n, Py_ssize_t want, F f) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments where %zd are expected", n, want);
        return nullptr;
    }
    try {
        return PyLong_FromLong(f());
    } catch (const Raised&) {
    } catch (const c10::OutOfMemoryError& e) {                   // of the workspace, as torch raises it
        PyObject* const torch = PyImport_ImportModule("torch");
        PyObject* const type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
        if (type) PyErr_SetString(type, e.what_without_backtrace());
        Py_XDECREF(type);
        Py_XDECREF(torch);
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

void two_dims(const at::Tensor& t, const char* name) {
    if (t.dim() != 2) raise(PyExc_ValueError, "%s must have two dimensions", name);
}

fsdp_activation activation_of(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return fsdp_activation(v);
}

#define FSDP_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL

}  // namespace
