// The operators' methods of the binding's extension module (args_ops.cpp).
#ifndef WB_ARGS_OPS_HPP
#define WB_ARGS_OPS_HPP

#include <Python.h>

PyObject* wb_py_add_rms_norm(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_route(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_route_backward(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_linear(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_combine(PyObject*, PyObject* const* args, Py_ssize_t n);

#endif
