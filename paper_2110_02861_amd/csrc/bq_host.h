// Shared by the two halves of the module _bqhost: bq_host.cpp and bq_host_ops.cpp.
#pragma once

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <exception>
#include <initializer_list>

#include <torch/csrc/autograd/python_variable.h>

namespace bq_host {

// Thrown where the Python code is to run instead (errors and unusual
// arguments included).
struct NotHandled : std::exception {};

inline void need(bool ok)
{
    if (!ok)
        throw NotHandled{};
}

inline PyObject *none()
{
    Py_RETURN_NONE;
}

// Whether every argument is None or of exactly torch's own classes.
inline bool plain(std::initializer_list<PyObject *> tensors)
{
    for (PyObject *o : tensors)
        if (o != Py_None && !THPVariable_CheckExact(o))
            return false;
    return true;
}

// An int, or any other object that stands for one (numpy's).
inline int64_t whole(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);  // by __index__
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw NotHandled{};
    }
    return v;
}

// Runs f, which returns a new reference, and hands anything unusual to Python.
template <class F>
PyObject *handled(F f)
{
    try {
        return f();
    } catch (const NotHandled &) {
    } catch (const std::exception &) {
        // e.g. a tensor without storage: the Python code meets it again and
        // raises its error
    }
    PyErr_Clear();
    return none();
}

}  // namespace bq_host

// The methods of bq_host_ops.cpp, added to the module.
extern PyMethodDef bq_ops_methods[];
