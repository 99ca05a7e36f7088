// Python calls of the 8-bit cache's operators (dlm_kv8_write, dlm_kv8_read, dlm_kv8_attention, dlm_qk_norm_rope of dlm.h) without ctypes.
// Their kernels take a few microseconds at the row counts of a decode, so a call is bound by what checking and marshalling its
// arguments costs the host: dlm_qk_norm_rope of 8 rows 7.2 us a call through ctypes, 4.0 here, of which the launch has 3 (1.2 more with the
// tensors' properties asked for through Python instead of torch's headers).
// Only calls that need no refusal are taken: tensors on the given GPU, of the types and shapes that the operator reads, with
// contiguous rows; lists or tuples of ints that fit 32 bits, long enough and at most 32 sequences.  Anything else returns None before
// anything is launched, and the caller goes the way through ctypes, which takes every other form and says what it refuses.
// Tensors are read in place, as the headers of one torch lay them out: `torch_version` says which, and with another one nothing here is to be called.
#include "py_args.h"

namespace {

int (*g_span[2])(const dlm_kv8_cache*, void*, void*, int64_t, int, const int32_t*, const int32_t*, const int32_t*, int, void*);
int (*g_attention)(const dlm_kv8_cache*, const void*, int64_t, void*, int, int, const int32_t*, const int32_t*, const int32_t*, int, const uint32_t*, int,
                          void*, size_t, void*);
int (*g_rope)(const void*, int64_t, int, int, int, int, int, const void*, const void*, float, float, const int32_t*, void*, int64_t, void*);
// span(0 write, 1 read, cache, cache memory, k, v, row_offsets, start, slot, device, stream) -> status or None
PyObject* span(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  int32_t off[MAX_SEQS + 1], start[MAX_SEQS], slot[MAX_SEQS];
  int which, dev;
  Tensor k, v;
  DECLINE_UNLESS(n_args == 10 && g_attention && to_int(a[0], &which) && (which == 0 || which == 1) && to_int(a[8], &dev));
  const dlm_kv8_cache* c = (const dlm_kv8_cache*)PyLong_AsVoidPtr(a[1]);
  void* stream = PyLong_AsVoidPtr(a[9]);
  if (PyErr_Occurred()) return nullptr;
  const int n = to_ints(a[6], -1, start);
  DECLINE_UNLESS(n > 0 && to_ints(a[5], n + 1, off) > 0 && (a[7] == Py_None || to_ints(a[7], n, slot) > 0));
  DECLINE_UNLESS(to_tensor(a[3], dev, &k) && to_tensor(a[4], dev, &v) && plain(a[2], dev));
  DECLINE_UNLESS(is_float(k) && v.dtype == k.dtype && k.dims == 3 && v.dims == 3 && k.stride == v.stride && k.shape[0] == v.shape[0] && off[n] <= k.shape[0]);
  for (int i = 1; i < 3; ++i) DECLINE_UNLESS(k.shape[i] == (i == 1 ? c->n_kv : c->head_dim) && v.shape[i] == k.shape[i]);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_span[which](c, k.p, v.p, k.stride, k.dtype, off, start, a[7] == Py_None ? nullptr : slot, n, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// attention(cache, cache memory, q, row_offsets, n_keys, slot, mask, out, workspace, workspace bytes, device, stream) -> status or None.  Declines a
// call without `out`, or one that may need a workspace and has none.
PyObject* attention(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  int32_t off[MAX_SEQS + 1], keys[MAX_SEQS], slot[MAX_SEQS];
  int dev;
  int64_t ws_bytes = 0;
  void* ws = nullptr;
  Tensor q, out, mask = {};
  DECLINE_UNLESS(n_args == 12 && g_attention && to_int(a[10], &dev));
  const dlm_kv8_cache* c = (const dlm_kv8_cache*)PyLong_AsVoidPtr(a[0]);
  void* stream = PyLong_AsVoidPtr(a[11]);
  if (PyErr_Occurred()) return nullptr;
  const int n = to_ints(a[4], -1, keys);
  DECLINE_UNLESS(n > 0 && to_ints(a[3], n + 1, off) > 0 && (a[5] == Py_None || to_ints(a[5], n, slot) > 0));
  DECLINE_UNLESS(to_tensor(a[2], dev, &q) && to_tensor(a[7], dev, &out) && plain(a[1], dev));
  DECLINE_UNLESS(is_float(q) && out.dtype == q.dtype && q.dims == 3 && out.dims == 3 && off[n] <= q.shape[0] && q.shape[1] <= INT32_MAX && q.shape[2] == c->head_dim);
  for (int i = 0; i < 3; ++i) DECLINE_UNLESS(out.shape[i] == q.shape[i]);
  DECLINE_UNLESS(out.stride == q.shape[1] * q.shape[2]);
  if (a[6] != Py_None)
    DECLINE_UNLESS(to_tensor(a[6], dev, &mask) && mask.dtype == 2 && mask.dims == 2 && mask.shape[0] >= off[n] && mask.shape[1] <= INT32_MAX && mask.stride == mask.shape[1]);
  if (a[8] != Py_None) {
    DECLINE_UNLESS(to_i64(a[9], &ws_bytes) && ws_bytes >= 0 && plain(a[8], dev));
    ws = plain(a[8], dev)->data_ptr();
  }
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_attention(c, q.p, q.stride, out.p, q.dtype, (int)q.shape[1], off, keys, a[5] == Py_None ? nullptr : slot, n, (const uint32_t*)mask.p,
                   mask.p ? (int)mask.shape[1] : 0, ws, (size_t)ws_bytes, stream);
  Py_END_ALLOW_THREADS
  DECLINE_UNLESS(rc != DLM_ECAPACITY || a[8] != Py_None);  // (it may need a workspace; nothing has been launched)
  return PyLong_FromLong(rc);
}

// rope(x, positions, n_q, n_kv, head_dim, q_gain, k_gain, eps, theta, out, device, stream) -> status or None.  Declines a call without `out`.
PyObject* rope(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  int n_q, n_kv, hd, dev;
  float eps, theta;
  Tensor x, pos, out, gain[2] = {};
  DECLINE_UNLESS(n_args == 12 && g_rope && to_int(a[2], &n_q) && to_int(a[3], &n_kv) && to_int(a[4], &hd) && to_int(a[10], &dev));
  DECLINE_UNLESS(to_float(a[7], &eps) && to_float(a[8], &theta));
  void* stream = PyLong_AsVoidPtr(a[11]);
  if (PyErr_Occurred()) return nullptr;
  DECLINE_UNLESS(to_tensor(a[0], dev, &x) && to_tensor(a[1], dev, &pos) && is_float(x) && x.dims == 2 && x.shape[0] <= INT32_MAX);
  if (a[9] == a[0]) out = x;
  else DECLINE_UNLESS(to_tensor(a[9], dev, &out));
  if (x.shape[0] == 1 && out.dims == 2) x.stride = out.stride = ((x.shape[1] > out.shape[1] ? x.shape[1] : out.shape[1]) + 7) & ~INT64_C(7);  // (a row has no stride)
  const int64_t width = ((int64_t)n_q + n_kv) * hd;
  DECLINE_UNLESS(out.dtype == x.dtype && out.dims == 2 && out.shape[0] == x.shape[0] && x.shape[1] >= width && out.shape[1] >= width);
  DECLINE_UNLESS(pos.dtype == 2 && pos.dims == 1 && pos.shape[0] == x.shape[0] && pos.stride == 1);
  for (int i = 0; i < 2; ++i)
    if (a[5 + i] != Py_None) DECLINE_UNLESS(to_tensor(a[5 + i], dev, &gain[i]) && gain[i].dtype == x.dtype && gain[i].dims == 1 && gain[i].shape[0] == hd && gain[i].stride == 1);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_rope(x.p, x.stride, (int)x.shape[0], n_q, n_kv, hd, x.dtype, gain[0].p, gain[1].p, eps, theta, (const int32_t*)pos.p, out.p, out.stride, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// bind(addresses of dlm_kv8_write, dlm_kv8_read, dlm_kv8_attention, dlm_qk_norm_rope)
PyObject* bind(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  void* f[4];
  if (n_args != 4) {
    PyErr_SetString(PyExc_TypeError, "bind takes four arguments");
    return nullptr;
  }
  for (int i = 0; i < 4; ++i) f[i] = PyLong_AsVoidPtr(a[i]);
  if (PyErr_Occurred()) return nullptr;
  *(void**)&g_span[0] = f[0];
  *(void**)&g_span[1] = f[1];
  *(void**)&g_attention = f[2];
  *(void**)&g_rope = f[3];
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"span", (PyCFunction)(void (*)(void))quiet<span>, METH_FASTCALL, "dlm_kv8_write and dlm_kv8_read"},
                         {"attention", (PyCFunction)(void (*)(void))quiet<attention>, METH_FASTCALL, "dlm_kv8_attention"},
                         {"rope", (PyCFunction)(void (*)(void))quiet<rope>, METH_FASTCALL, "dlm_qk_norm_rope"},
                         {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, "the library's entry points"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv8", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv8(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_BUILT_WITH) < 0) Py_CLEAR(m);
  return m;
}
