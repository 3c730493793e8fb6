// What the native parts of the Python binding share: which tensors and streams they take.
#pragma once
#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

// set once by bind(), under the interpreter's lock
PyObject *tensor_type, *parameter_type;

// wrappers without memory of their own, or whose memory is not theirs to hand out
const c10::DispatchKeySet WRAPPERS({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                    c10::DispatchKey::Functionalize});

const at::Tensor *plain(PyObject *o)
{
    if ((PyObject *)Py_TYPE(o) != tensor_type && (PyObject *)Py_TYPE(o) != parameter_type) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.key_set().has_any(WRAPPERS) || !t.has_storage()) return nullptr;
    return &t;
}

struct DescView {                            // a descriptor's bytes while the call lasts
    Py_buffer view = {};
    ~DescView() { if (view.obj) PyBuffer_Release(&view); }
};

// The hipStream_t of a call's last argument: torch's current stream for None, else its handle where that is a number
enum StreamFound { STREAM_TAKEN, STREAM_OTHER, STREAM_ERROR };
StreamFound stream_of(PyObject *given, void **stream)
{
    if (given == Py_None) {
        *stream = c10::hip::getCurrentHIPStream().stream();
        return STREAM_TAKEN;
    }
    PyObject *handle = PyObject_GetAttrString(given, "cuda_stream");
    if (!handle) return STREAM_ERROR;
    bool taken = PyLong_Check(handle);       // (the foreign call also takes None, a c_void_p and what else stands for a pointer)
    *stream = taken ? PyLong_AsVoidPtr(handle) : nullptr;
    Py_DECREF(handle);
    if (PyErr_Occurred()) { PyErr_Clear(); taken = false; }
    return taken ? STREAM_TAKEN : STREAM_OTHER;
}

}  // namespace
