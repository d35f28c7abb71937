// Shared by the translation units of the binding's native half.
#pragma once
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../../include/nuna.h"

namespace nuna_py {

// nuna_py.cpp: each returns false, or null, with a Python exception set.
bool to_address(PyObject* x, void** out);
bool address_of(PyObject* x, bool host, void** out);
bool to_u64(PyObject* x, unsigned long long* out);
bool to_stream(PyObject* x, void** out);
PyObject* finish(int status, const char* what, PyObject* check);

// nuna_py_ops.cpp: adds the operators' functions to the module.
bool add_operators(PyObject* module);

}  // namespace nuna_py
