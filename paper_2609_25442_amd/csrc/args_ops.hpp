// The operators' methods of the binding's extension module (args_ops.cpp, args_train.cpp).
#ifndef WB_ARGS_OPS_HPP
#define WB_ARGS_OPS_HPP

#include <Python.h>

PyObject* wb_py_add_rms_norm(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_route(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_route_backward(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_linear(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_combine(PyObject*, PyObject* const* args, Py_ssize_t n);

PyObject* wb_py_embedding(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_embedding_backward(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_add_layer_norm(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_add_layer_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_dispatch(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_dispatch_backward(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_collect(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_collect_backward(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_activate(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_activate_backward(PyObject*, PyObject* const* args, Py_ssize_t n);
PyObject* wb_py_held_elsewhere(PyObject*, PyObject* const* args, Py_ssize_t n);

#endif
