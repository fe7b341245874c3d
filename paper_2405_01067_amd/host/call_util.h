// What the native calls from Python share (layer_call.cpp, adapter_call.cpp): which tensors they take, the stream, the results.
#pragma once

#include <Python.h>

#include <ATen/ops/empty.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/autograd/python_variable.h>

namespace native_call {

inline PyObject *get_device, *get_stream, *check;      // torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, binding._check

// A tensor on the GPU with a memory of its own, contiguous, nobody between it and its data
inline const at::Tensor* plain(PyObject* o, int64_t dim = 2) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    static const c10::DispatchKeySet wrapped({c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot, c10::DispatchKey::FuncTorchBatched,
                                              c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize, c10::DispatchKey::Negative,
                                              c10::DispatchKey::Conjugate, c10::DispatchKey::ZeroTensor, c10::DispatchKey::Batched});
    if (!t.defined() || t.key_set().has_any(wrapped) || t.layout() != at::kStrided || !t.is_cuda() || t.dim() != dim || !t.has_storage() ||
        t.unsafeGetTensorImpl()->has_symbolic_sizes_strides() || !t.is_contiguous())
        return nullptr;
    return &t;
}
inline bool watched() {
    return c10::impl::TorchDispatchModeTLS::any_modes_set() || at::impl::torch_function_mode_enabled() ||
           c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode) ||
           c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::Functionalize) || c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::Tracer);
}
// the current stream of the current device, as the Python code asks for it
inline bool current_stream(void** s) {
    PyObject* dev = PyObject_CallNoArgs(get_device);
    if (!dev) return false;
    PyObject* raw = PyObject_CallOneArg(get_stream, dev);
    Py_DECREF(dev);
    if (!raw) return false;
    *s = reinterpret_cast<void*>(PyLong_AsSsize_t(raw));
    Py_DECREF(raw);
    return !PyErr_Occurred();
}
// The results, or for an error of the library what binding._check raises
inline PyObject* finished(PyObject* results, int code, const char* what) {
    if (code == 0) return results;
    Py_DECREF(results);
    PyObject* r = PyObject_CallFunction(check, "is", code, what);
    Py_XDECREF(r);
    return nullptr;
}
inline PyObject* wrap_or_none(const at::Tensor& t) {
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}

// Everything that can fail comes before the launch: a call that is answered with None has done nothing.  Addresses are asked for with
// data_ptr(), as from Python: what materialises or refuses there does here.

}  // namespace native_call
