// What the modules that call the libraries from PyTorch share: errors, arguments, streams, the interpreter lock.  Included once
// per module; each has its own error type.
#pragma once

#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/Stream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include <cstring>
#include <optional>
#include <string>

#include "../../include/dgsp.h"

namespace {

PyObject* g_error = nullptr;      // DgspError, a strong reference for the life of the process

// A Python exception is set: unwinds to the function's entry.
struct Raised {};

[[noreturn]] void fail(const std::string& what) {
    PyErr_SetString(g_error ? g_error : PyExc_RuntimeError, what.c_str());
    throw Raised{};
}

void check_status(int rc, const char* what) {
    if (rc != DGSP_OK) fail(std::string(what) + ": " + dgsp_status_string(rc) + " (status " + std::to_string(rc) + ")");
}

int64_t as_int(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}

// Entry counts, algos and factors: what int() and float() take.
int64_t to_int(PyObject* o) {
    if (PyLong_CheckExact(o)) return as_int(o);
    PyObject* i = PyNumber_Long(o);
    if (!i) throw Raised{};
    const long long v = PyLong_AsLongLong(i);
    Py_DECREF(i);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}

float to_float(PyObject* o) {
    if (PyFloat_CheckExact(o)) return (float)PyFloat_AS_DOUBLE(o);
    PyObject* f = PyNumber_Float(o);
    if (!f) throw Raised{};
    const double v = PyFloat_AS_DOUBLE(f);
    Py_DECREF(f);
    return (float)v;
}

const at::Tensor& as_tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) {
        fail(std::string(name) + " must be a tensor");
    }
    return THPVariable_Unpack(o);
}

// The stream that a call runs on; `known`: as torch's allocator knows it, none for a stream that is not torch's, which may be gone
// when the allocator asks how far it has come.
struct CallStream {
    void* handle;
    std::optional<c10::hip::HIPStream> known;
};

CallStream call_stream(c10::hip::HIPStream s) {
    void* handle = s.stream();
    const bool foreign = handle != nullptr && s.id() == (int64_t)reinterpret_cast<intptr_t>(handle);      // named by their address
    return {handle, foreign ? std::nullopt : std::make_optional(s)};
}

CallStream current_stream() { return call_stream(c10::hip::getCurrentHIPStream()); }

// the torch stream given, or the current one
CallStream as_stream(PyObject* o) {
    if (o == Py_None) return current_stream();
    PyObject* handle = PyObject_GetAttrString(o, "cuda_stream");
    if (!handle) throw Raised{};
    void* p = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    if (!p && PyErr_Occurred()) throw Raised{};
    if (!THPStream_Check(o)) return {p, std::nullopt};
    const auto* t = reinterpret_cast<THPStream*>(o);
    const c10::Device device(c10::DeviceType::HIP, (c10::DeviceIndex)t->device_index);
    const c10::Stream named(c10::Stream::UNSAFE, device, t->stream_id);
    const CallStream s = call_stream(c10::hip::HIPStream(c10::hip::HIPStream::UNCHECKED, named));
    return s.handle == p ? s : CallStream{p, std::nullopt};
}

void* ptr(const at::Tensor& t) { return t.numel() == 0 ? nullptr : t.data_ptr(); }

bool on_gpu(const at::Tensor& t) { return t.device().is_cuda() && t.layout() == at::kStrided; }

bool is_array(const at::Tensor& t, at::ScalarType type) { return on_gpu(t) && t.scalar_type() == type && t.is_contiguous(); }

// The library call itself, with the interpreter lock released: a full queue can make a launch wait.
template <typename F>
int unlocked(F&& call) {
    PyThreadState* state = PyEval_SaveThread();
    const int rc = call();
    PyEval_RestoreThread(state);
    return rc;
}

void want(Py_ssize_t n, Py_ssize_t expected) {
    if (n != expected) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", expected, n);
        throw Raised{};
    }
}

template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        return F(a, n);
    } catch (const Raised&) {
        return nullptr;
    } catch (...) {                                // out of memory, among others: the exception torch itself would raise
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    }
}

PyObject* set_error_type(PyObject* const* a, Py_ssize_t n) {
    want(n, 1);
    Py_INCREF(a[0]);
    Py_XDECREF(g_error);
    g_error = a[0];
    Py_RETURN_NONE;
}

// Does nothing but reverse mode look at a product of X?  Not so under a tangent on X (forward mode), a function transform
// (vmap, grad, jvp), a trace that is being recorded, or Python code that intercepts operations: a graph node of our own
// would pass by them and return a result without tangent, batch or record.
bool only_reverse_mode(const at::Tensor& X) {
    const auto included = c10::impl::tls_local_dispatch_key_set().included_;
    return !X._fw_grad(/*level=*/0).defined() && !X.unsafeGetTensorImpl()->is_python_dispatch() &&
           !included.has(c10::DispatchKey::FuncTorchDynamicLayerFrontMode) &&
           !included.has(c10::DispatchKey::FuncTorchDynamicLayerBackMode) && !torch::jit::tracer::isTracing() &&
           !c10::impl::TorchDispatchModeTLS::any_modes_set();
}

}  // namespace
