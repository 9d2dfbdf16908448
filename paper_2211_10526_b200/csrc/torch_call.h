// What the files of the torch-facing module share.
#pragma once

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/Functions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "castling_attn.h"

namespace torch_call {

inline const at::Tensor* tensor(PyObject* o, const char* name) {
    if (THPVariable_Check(o)) return &THPVariable_Unpack(o);
    PyErr_Format(PyExc_TypeError, "%s: expected a torch.Tensor", name);
    return nullptr;
}

// A caller's tensor has been written: autograd has to know that what it may have kept of it is gone.
inline void written(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

inline PyObject* value_error(const char* what) { PyErr_SetString(PyExc_ValueError, what); return nullptr; }

// torch_block.cpp: the operators around the attention core
PyObject* bind_block(PyObject*, PyObject* args);
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* norm_forward(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* attention_backward(PyObject*, PyObject* const* a, Py_ssize_t n);

}  // namespace torch_call
