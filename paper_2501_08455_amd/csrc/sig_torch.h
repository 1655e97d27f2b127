// What the files of the native torch binding share: arguments from Python, errors on their way there.
#ifndef SIG_TORCH_H
#define SIG_TORCH_H

#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>

#include "sig.h"

namespace sig_torch {

extern sig_ctx *default_ctx;   // the binding's default context, set once by set_default_ctx
extern PyMethodDef sequence_methods[];   // of sig_torch_sequence.cpp

// A failed library call on its way to Python, where it becomes binding.SigError(status, where)
struct Failure {
    int status;
    const char *where;
};

// module.type(*args), raised; `args` is taken over
inline void raise_named(const char *module_name, const char *type_name, PyObject *args)
{
    PyObject *module = args ? PyImport_ImportModule(module_name) : nullptr;
    PyObject *type = module ? PyObject_GetAttrString(module, type_name) : nullptr;
    PyObject *error = type ? PyObject_CallObject(type, args) : nullptr;
    if (error) PyErr_SetObject(type, error);
    Py_XDECREF(error);
    Py_XDECREF(type);
    Py_XDECREF(module);
    Py_XDECREF(args);
}

inline PyObject *raise(const Failure &f)
{
    raise_named("paper_2501_08455_amd.binding", "SigError", Py_BuildValue("(is)", f.status, f.where));
    return nullptr;
}

// the same from a thread of the autograd engine: the exception travels as torch's carrier of Python errors
[[noreturn]] inline void rethrow_in_python(const Failure &f)
{
    const PyGILState_STATE gil = PyGILState_Ensure();
    python_error carrier;
    raise(f);
    carrier.persist();
    PyGILState_Release(gil);
    throw carrier;
}

inline void *current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// ---------------------------------------------------------------- Python arguments
inline const at::Tensor *tensor_arg(PyObject *o)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "expected a torch tensor, got %s", Py_TYPE(o)->tp_name);
        return nullptr;
    }
    return &THPVariable_Unpack(o);
}

// what int(o) gives
inline bool int_arg(PyObject *o, int *value)
{
    PyObject *number = PyLong_CheckExact(o) ? Py_NewRef(o) : PyNumber_Long(o);
    if (!number) return false;
    const long v = PyLong_AsLong(number);
    Py_DECREF(number);
    if (v == -1 && PyErr_Occurred()) return false;
    if (v != (long)(int)v) {
        PyErr_SetString(PyExc_OverflowError, "integer argument out of range");
        return false;
    }
    *value = (int)v;
    return true;
}

// a context or a stream: None, an address, or an object that holds one under `attribute`
inline bool address_arg(PyObject *o, const char *attribute, void **address)
{
    *address = nullptr;
    if (o == Py_None) return true;
    PyObject *value = PyLong_Check(o) ? Py_NewRef(o) : PyObject_GetAttrString(o, attribute);
    if (!value) return false;
    if (value != Py_None) *address = PyLong_AsVoidPtr(value);
    Py_DECREF(value);
    return !PyErr_Occurred();
}

inline bool stream_arg(PyObject *o, void **stream)
{
    if (o != Py_None) return address_arg(o, "cuda_stream", stream);
    *stream = current_stream();
    return true;
}

template <typename F>
inline PyObject *guarded(F f)
{
    try {
        return f();
    } catch (const Failure &e) {
        return raise(e);
    } catch (const std::invalid_argument &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (...) {
        // torch's own, and what Python code raised in between (python_error: a saved-tensor hook, a dispatch mode)
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

// runs `f` without the interpreter lock (a launch may wait for room in the queue)
template <typename F>
auto unlocked(F f)
{
    struct Unlock {
        PyThreadState *state = PyEval_SaveThread();
        ~Unlock() { PyEval_RestoreThread(state); }
    } unlock;
    return f();
}

inline bool arity(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return n == want;
}

#define FASTCALL(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL

}  // namespace sig_torch
#endif
