// What the host sides of the calls share (decode_call.cpp, packed_call.cpp, packed_grad.cpp): reading Python arguments without its own
// machinery.
#pragma once

#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/core/DispatchKeySet.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cstring>

#include "../../include/gformer.h"

namespace gformer_host {

// A strided tensor and nothing else: a wrapper's data pointer is not what the caller means.
inline const at::Tensor* strided(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || t.layout() != at::kStrided || t.is_nested() || !t.has_storage() ||
      t.unsafeGetTensorImpl()->has_symbolic_sizes_strides())
    return nullptr;
  constexpr c10::DispatchKeySet wrapped({
      c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot, c10::DispatchKey::Functionalize,
      c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Conjugate,
      c10::DispatchKey::Negative, c10::DispatchKey::ZeroTensor});
  return t.key_set().has_any(wrapped) ? nullptr : &t;
}
// A dense one.
inline const at::Tensor* plain(PyObject* o) {
  const at::Tensor* t = strided(o);
  return t && t->is_contiguous() ? t : nullptr;
}

inline bool to_long(PyObject* o, int64_t lo, int64_t hi, int64_t& x) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  x = PyLong_AsLongLongAndOverflow(o, &over);
  return over == 0 && x >= lo && x <= hi;
}
inline bool to_float(PyObject* o, float& x) {
  if (!PyFloat_CheckExact(o)) return false;
  x = (float)PyFloat_AS_DOUBLE(o);
  return true;
}

extern PyObject* raw_stream_getter;   // torch._C._cuda_getCurrentRawStream, where torch has it

// The current stream's handle on `device`; false with a Python error set.
inline bool current_stream(int64_t device, int64_t& stream) {
  PyObject* index = PyLong_FromLong((long)device);
  PyObject* handle = index ? PyObject_CallOneArg(raw_stream_getter, index) : nullptr;
  Py_XDECREF(index);
  if (!handle) return false;
  stream = (int64_t)PyLong_AsUnsignedLongLongMask(handle);
  Py_DECREF(handle);
  return true;
}

// packed_call.cpp
PyObject* packed_fwd(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* packed_bwd(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* paged_fill(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* paged_decode(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* pages_copy(PyObject*, PyObject* const* a, Py_ssize_t n);
// packed_grad.cpp
PyObject* packed_attention(PyObject*, PyObject* const* a, Py_ssize_t n);

}  // namespace gformer_host
