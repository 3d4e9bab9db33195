// What the native binding modules share: checks of tensors, the call's stream, descriptors, and the wall that no C++ exception passes.
// A decode step makes such calls once per layer with a dozen tensors each, and reading that many tensors' fields from Python
// takes longer than the kernels run; here a call costs the host about as much as its launches.  Nothing is kept between calls.
// Errors of the library go through the Python function given to set_check.
#pragma once
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>

#include "../../include/bd.h"

namespace {

PyObject *g_check = nullptr;

struct Raised {};                                                  // a Python error is already set

[[noreturn]] void refuse(const std::string &text) { throw std::invalid_argument(text); }

const at::Tensor &tensor(PyObject *o, const char *what) {
    if (!THPVariable_Check(o)) refuse(std::string(what) + " must be a tensor");
    return THPVariable_Unpack(o);
}
void here(const at::Tensor &t, const char *what) {
    if (!t.is_cuda() || t.get_device() != c10::cuda::current_device()) refuse(std::string(what) + " must be on the current CUDA device");
}
bool dtype_of(at::ScalarType s, bd_dtype *dt) {
    if (s == at::kFloat) *dt = BD_F32;
    else if (s == at::kBFloat16) *dt = BD_BF16;
    else if (s == at::kHalf) *dt = BD_F16;
    else return false;
    return true;
}
at::ScalarType scalar_of(bd_dtype dt) { return dt == BD_F32 ? at::kFloat : dt == BD_BF16 ? at::kBFloat16 : at::kHalf; }
int64_t integer(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}
double real(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return v;
}
// The call's stream: the current one, or the one given, which then also is the stream of what the call allocates.
struct StreamScope {
    c10::cuda::OptionalCUDAStreamGuard guard;
    void *raw;
    explicit StreamScope(PyObject *o) {
        if (o != Py_None) {
            PyObject *v = PyObject_GetAttrString(o, "cuda_stream");
            if (!v) throw Raised();
            raw = PyLong_AsVoidPtr(v);
            Py_DECREF(v);
            if (PyErr_Occurred()) throw Raised();
            const auto current = c10::cuda::getCurrentCUDAStream();
            if (raw != current.stream()) guard.reset_stream(c10::cuda::getStreamFromExternal((cudaStream_t)raw, current.device_index()));
        } else {
            raw = c10::cuda::getCurrentCUDAStream().stream();
        }
    }
};
void check(bd_status s) {
    if (s == BD_OK) return;
    PyObject *r = PyObject_CallFunction(g_check, "i", (int)s);
    if (r) {
        Py_DECREF(r);
        PyErr_SetString(PyExc_RuntimeError, "the library returned an error");
    }
    throw Raised();
}
// A descriptor as Python keeps it, with the device its buffers are on.
template <typename T>
struct Held {
    T s;
    int64_t device;
};
template <typename T>
PyObject *hold(const T &s) {
    const Held<T> h{s, (int64_t)c10::cuda::current_device()};
    return PyBytes_FromStringAndSize((const char *)&h, sizeof h);
}
template <typename T>
const T &structure(PyObject *o, const char *what = "cache and batch") {
    if (!PyBytes_Check(o) || PyBytes_GET_SIZE(o) != (Py_ssize_t)sizeof(Held<T>)) refuse("not a descriptor of this module");
    const Held<T> &h = *(const Held<T> *)PyBytes_AS_STRING(o);
    if (h.device != c10::cuda::current_device()) refuse(std::string(what) + " must be on the current CUDA device");
    return h.s;
}
void need(Py_ssize_t got, Py_ssize_t want) {
    if (got != want) refuse("wrong number of arguments");
}

PyObject *set_check(PyObject *const *a, Py_ssize_t n) {
    need(n, 1);
    Py_INCREF(a[0]);
    Py_XSETREF(g_check, a[0]);
    Py_RETURN_NONE;
}

// No C++ exception leaves an entry point.
template <PyObject *(*F)(PyObject *const *, Py_ssize_t)>
PyObject *entry(PyObject *, PyObject *const *a, Py_ssize_t n) {
    try {
        return F(a, n);
    } catch (const Raised &) {
    } catch (const std::invalid_argument &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const c10::OutOfMemoryError &e) {
        PyErr_SetString(PyExc_MemoryError, e.what_without_backtrace());
    } catch (const c10::Error &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
#define BD_ENTRY(f) {#f, (PyCFunction)(void (*)(void)) & entry<f>, METH_FASTCALL, nullptr}

}  // namespace
