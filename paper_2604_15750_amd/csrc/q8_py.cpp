// Python calls of the 8-bit integer layers' operators (dlm_q8_rows, dlm_add_norm_q8, dlm_q8_gemm of dlm.h) without ctypes, as kv8_py.cpp has them
// for the 8-bit cache and for the same reason.  Only calls with all their outputs given, and that need no refusal, are taken; anything else returns None
// before anything is launched, and the caller goes the way through ctypes.
#include "py_args.h"

namespace {

int (*g_rows)(const void*, int64_t, int, int, int, int8_t*, int64_t, float*, void*);
int (*g_norm)(const void*, int64_t, int, int, int, const void*, int64_t, void*, int64_t, int, const void*, float, int8_t*, int64_t, float*, void*);
int (*g_gemm)(const dlm_q8_weight*, const int8_t*, int64_t, const float*, int, void*, int64_t, int, void*, size_t, void*);

constexpr int INT8 = 3;
int elem_bytes(const Tensor& t) { return t.dtype == DLM_BF16 ? 2 : t.dtype == INT8 ? 1 : 4; }

// a matrix whose rows are contiguous; a single row, which has no stride, gets one that holds it in multiples of 16 bytes
bool to_matrix(PyObject* o, int dev, Tensor* t) {
  if (!to_tensor(o, dev, t) || t->dims != 2 || t->shape[0] > INT32_MAX || t->shape[1] < 1 || t->shape[1] > INT32_MAX) return false;
  if (t->shape[0] == 1) {
    const int64_t step = 16 / elem_bytes(*t);
    t->stride = (t->shape[1] + step - 1) / step * step;
  }
  return true;
}
bool same_shape(const Tensor& a, const Tensor& b) { return a.shape[0] == b.shape[0] && a.shape[1] == b.shape[1]; }
bool to_vector(PyObject* o, int dev, int64_t n, int dtype, Tensor* t) {
  return to_tensor(o, dev, t) && t->dims == 1 && t->shape[0] == n && t->stride == 1 && t->dtype == dtype;
}

// rows(x, codes, scale, device, stream) -> status or None
PyObject* rows(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  int dev;
  Tensor x, codes, scale;
  DECLINE_UNLESS(n_args == 5 && g_rows && to_int(a[3], &dev));
  void* stream = PyLong_AsVoidPtr(a[4]);
  if (PyErr_Occurred()) return nullptr;
  DECLINE_UNLESS(to_matrix(a[0], dev, &x) && is_float(x) && to_matrix(a[1], dev, &codes) && codes.dtype == INT8 && same_shape(x, codes));
  DECLINE_UNLESS(to_vector(a[2], dev, x.shape[0], DLM_F32, &scale));
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_rows(x.p, x.stride, (int)x.shape[0], (int)x.shape[1], x.dtype, (int8_t*)codes.p, codes.stride, (float*)scale.p, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// norm(x, gain, residual, h, eps, codes, scale, device, stream) -> status or None
PyObject* norm(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  int dev;
  float eps;
  Tensor x, gain, residual = {}, h = {}, codes, scale;
  DECLINE_UNLESS(n_args == 9 && g_norm && to_int(a[7], &dev) && to_float(a[4], &eps));
  void* stream = PyLong_AsVoidPtr(a[8]);
  if (PyErr_Occurred()) return nullptr;
  DECLINE_UNLESS(to_matrix(a[0], dev, &x) && is_float(x) && to_vector(a[1], dev, x.shape[1], x.dtype, &gain));
  DECLINE_UNLESS((a[2] == Py_None) == (a[3] == Py_None));
  if (a[2] != Py_None) {
    DECLINE_UNLESS(to_matrix(a[2], dev, &residual) && same_shape(x, residual) && (residual.dtype == DLM_F32 || residual.dtype == x.dtype));
    DECLINE_UNLESS(to_matrix(a[3], dev, &h) && same_shape(x, h) && h.dtype == residual.dtype);
  }
  DECLINE_UNLESS(to_matrix(a[5], dev, &codes) && codes.dtype == INT8 && same_shape(x, codes) && to_vector(a[6], dev, x.shape[0], DLM_F32, &scale));
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_norm(x.p, x.stride, (int)x.shape[0], (int)x.shape[1], x.dtype, residual.p, residual.p ? residual.stride : 0, h.p, h.p ? h.stride : 0, h.p ? h.dtype : 0, gain.p, eps,
              (int8_t*)codes.p, codes.stride, (float*)scale.p, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// gemm(weight, weight memory, x, x_scale, out, workspace, device, stream) -> status or None.  DLM_ECAPACITY without a workspace: it may need one.
PyObject* gemm(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  int dev;
  Tensor x, scale, out;
  DECLINE_UNLESS(n_args == 8 && g_gemm && to_int(a[6], &dev));
  const dlm_q8_weight* w = (const dlm_q8_weight*)PyLong_AsVoidPtr(a[0]);
  void* stream = PyLong_AsVoidPtr(a[7]);
  if (PyErr_Occurred()) return nullptr;
  DECLINE_UNLESS(w && plain(a[1], dev) && to_matrix(a[2], dev, &x) && x.dtype == INT8 && x.shape[1] == w->k && to_vector(a[3], dev, x.shape[0], DLM_F32, &scale));
  if (w->k % 16) {  // the last row's bytes up to a multiple of 16 have to be the tensor's memory
    const at::Tensor& t = *plain(a[2], dev);
    DECLINE_UNLESS((int64_t)t.storage().nbytes() >= t.storage_offset() + (x.shape[0] - 1) * x.stride + (w->k + 15) / 16 * 16);
  }
  DECLINE_UNLESS(to_matrix(a[4], dev, &out) && is_float(out) && out.shape[0] == x.shape[0] && out.shape[1] == (w->gated ? w->n / 2 : w->n));
  void* ws = nullptr;
  size_t ws_bytes = 0;
  if (a[5] != Py_None) {
    const at::Tensor* t = plain(a[5], dev);
    DECLINE_UNLESS(t && t->is_contiguous());
    ws = t->data_ptr();
    ws_bytes = (size_t)t->numel() * t->element_size();
  }
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_gemm(w, (const int8_t*)x.p, x.stride, (const float*)scale.p, (int)x.shape[0], out.p, out.stride, out.dtype, ws, ws_bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// bind(addresses of dlm_q8_rows, dlm_add_norm_q8, dlm_q8_gemm)
PyObject* bind(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  void* f[3];
  if (n_args != 3) {
    PyErr_SetString(PyExc_TypeError, "bind takes three arguments");
    return nullptr;
  }
  for (int i = 0; i < 3; ++i) f[i] = PyLong_AsVoidPtr(a[i]);
  if (PyErr_Occurred()) return nullptr;
  *(void**)&g_rows = f[0];
  *(void**)&g_norm = f[1];
  *(void**)&g_gemm = f[2];
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"rows", (PyCFunction)(void (*)(void))quiet<rows>, METH_FASTCALL, "dlm_q8_rows"},
                         {"norm", (PyCFunction)(void (*)(void))quiet<norm>, METH_FASTCALL, "dlm_add_norm_q8"},
                         {"gemm", (PyCFunction)(void (*)(void))quiet<gemm>, METH_FASTCALL, "dlm_q8_gemm"},
                         {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, "the library's entry points"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_q8", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__q8(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_BUILT_WITH) < 0) Py_CLEAR(m);
  return m;
}
