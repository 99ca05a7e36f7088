// How the extensions behind the Python calls of the 8-bit operators read their arguments: plain ints, floats, lists and tensors, without a call into Python.
// Tensors are read in place, as the headers of one torch lay them out.  Each reader returns 0, false or null for an argument that is not plain (with no
// error set), and the call is then declined: None, before anything is launched.
#pragma once
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "../../include/dlm.h"

namespace {

constexpr int MAX_SEQS = 32;

int to_i64(PyObject* o, int64_t* out) {
  int overflow;
  if (!PyLong_Check(o)) return 0;
  *out = PyLong_AsLongLongAndOverflow(o, &overflow);
  return !overflow;
}
int to_int(PyObject* o, int* out) {
  int64_t v;
  if (!to_i64(o, &v) || v < INT32_MIN || v > INT32_MAX) return 0;
  *out = (int)v;
  return 1;
}
int to_float(PyObject* o, float* out) {
  if (!PyFloat_CheckExact(o)) return 0;
  const double v = PyFloat_AS_DOUBLE(o);
  *out = (float)v;
  return (*out - *out == 0.f) || v - v != 0.;  // (a finite value that overflows is the other way's error)
}
// the first n entries of an array that has as many (n < 0: all of them); their number, or -1
int to_ints(PyObject* o, int n, int32_t* out) {
  PyObject** item;
  Py_ssize_t len;
  if (PyList_CheckExact(o)) {
    item = ((PyListObject*)o)->ob_item;
    len = PyList_GET_SIZE(o);
  } else if (PyTuple_CheckExact(o)) {
    item = ((PyTupleObject*)o)->ob_item;
    len = PyTuple_GET_SIZE(o);
  } else {
    return -1;
  }
  if (n < 0) n = len <= MAX_SEQS ? (int)len : -1;
  if (n < 0 || len < n) return -1;
  for (int i = 0; i < n; ++i)
    if (!to_int(item[i], out + i)) return -1;
  return n;
}

const at::Tensor* plain(PyObject* o, int dev) {  // of torch's own type, in memory of GPU `dev`
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& x = THPVariable_Unpack(o);
  return x.defined() && x.get_device() == dev && x.layout() == at::kStrided ? &x : nullptr;
}
struct Tensor {
  void* p;
  int dtype, dims;  // dtype: a DLM_ code, 2 for int32, 3 for int8, 4 for uint8
  int64_t shape[3], stride;
};
// a tensor of 1 to 3 dimensions whose rows (everything behind the first) are contiguous
bool to_tensor(PyObject* o, int dev, Tensor* t) {
  const at::Tensor* x = plain(o, dev);
  if (!x) return false;
  const auto type = x->scalar_type();
  t->dtype = type == at::kBFloat16 ? DLM_BF16 : type == at::kFloat ? DLM_F32 : type == at::kInt ? 2 : type == at::kChar ? 3 : type == at::kByte ? 4 : -1;
  const auto shape = x->sizes(), stride = x->strides();
  t->dims = (int)shape.size();
  if (t->dtype < 0 || t->dims < 1 || t->dims > 3 || shape[0] < 1) return false;  // (a tensor without rows has no address)
  int64_t width = 1;
  for (int i = t->dims - 1; i >= 0; --i) {
    t->shape[i] = shape[i];
    if (i == 0) break;
    if (stride[i] != width && shape[i] != 1) return false;
    width *= shape[i];
  }
  t->stride = shape[0] > 1 ? stride[0] : width;
  t->p = x->data_ptr();
  return true;
}
bool is_float(const Tensor& t) { return t.dtype == DLM_F32 || t.dtype == DLM_BF16; }
#define DECLINE_UNLESS(cond) \
  if (!(cond)) Py_RETURN_NONE

// what torch throws (a tensor without memory, say) is the other way's to report
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* quiet(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  try {
    return F(self, a, n_args);
  } catch (...) {
    Py_RETURN_NONE;
  }
}

}  // namespace
