/* Argument marshalling of the per-step calls (CPython extension `_calls`).
 *
 * A decode step takes the GPU a few microseconds, and converting its seventeen arguments in Python and
 * ctypes took the host about as long.  Here a call is one C function: descriptors come as addresses,
 * device memory as anything with a data_ptr() (a torch tensor), as an integer address or None, a plan as a
 * numpy array.  Returns the efim_status as an int; nothing else happens here. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include "efim.h"

static PyObject *s_data_ptr, *s_nbytes;
static PyTypeObject* ndarray; /* numpy.ndarray */

/* address of a numpy array's memory, which the object keeps valid */
static int array_ptr(PyObject* o, void** out) {
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_STRIDES) != 0) return 0;
  *out = b.buf;
  PyBuffer_Release(&b);
  return 1;
}
/* address of a device tensor, an integer address, a numpy array (over memory that the device can address), or
   NULL for None.  Not of any other object with a buffer: a numpy scalar's is a temporary. */
static int as_ptr(PyObject* o, void** out) {
  if (o == Py_None) {
    *out = NULL;
    return 1;
  }
  if (PyLong_Check(o)) {
    *out = PyLong_AsVoidPtr(o);
    return !(*out == NULL && PyErr_Occurred());
  }
  if (PyObject_TypeCheck(o, ndarray)) return array_ptr(o, out);
  PyObject* r = PyObject_CallMethodNoArgs(o, s_data_ptr);
  if (!r) return 0;
  *out = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return !(*out == NULL && PyErr_Occurred());
}
static int as_i32(PyObject* o, int32_t* out) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) return 0;
  *out = (int32_t)v;
  return 1;
}
static int as_i64(PyObject* o, int64_t* out) {
  *out = PyLong_AsLongLong(o);
  return !(*out == -1 && PyErr_Occurred());
}
static int as_float(PyObject* o, float* out) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) return 0;
  *out = (float)v;
  return 1;
}
/* bytes of an object with an `nbytes`, 0 for None */
static int as_bytes(PyObject* o, size_t* out) {
  *out = 0;
  if (o == Py_None) return 1;
  PyObject* r = PyObject_GetAttr(o, s_nbytes);
  if (!r) return 0;
  *out = PyLong_AsSize_t(r);
  Py_DECREF(r);
  return !(*out == (size_t)-1 && PyErr_Occurred());
}
/* a workspace: device memory whose size the object knows */
static int as_workspace(PyObject* o, void** out, size_t* bytes) {
  if (PyObject_TypeCheck(o, ndarray)) {
    PyErr_SetString(PyExc_TypeError, "the workspace is device memory, not a numpy array");
    return 0;
  }
  return as_ptr(o, out) && as_bytes(o, bytes);
}
/* a plan: host memory, a numpy array or None */
static int as_plan(PyObject* o, void** out, size_t* bytes) {
  *out = NULL;
  *bytes = 0;
  if (o == Py_None) return 1;
  if (!PyObject_TypeCheck(o, ndarray)) {
    PyErr_SetString(PyExc_TypeError, "the plan is a numpy array in host memory");
    return 0;
  }
  return array_ptr(o, out) && as_bytes(o, bytes);
}
static int want(Py_ssize_t n, Py_ssize_t expected) {
  if (n == expected) return 1;
  PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", expected, n);
  return 0;
}
#define PTR(i) as_ptr(a[i], &p[i])
/* a launch can wait for room in the stream's queue: other Python threads go on meanwhile */
#define RETURN_STATUS(call)        \
  do {                             \
    efim_status st_;               \
    Py_BEGIN_ALLOW_THREADS         \
    st_ = (call);                  \
    Py_END_ALLOW_THREADS           \
    return PyLong_FromLong(st_);   \
  } while (0)

/* cache, batch, rope, q, k_new, v_new, status, stream */
static PyObject* kv_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p[8];
  if (!want(n, 8)) return NULL;
  for (int i = 0; i < 8; ++i)
    if (!PTR(i)) return NULL;
  RETURN_STATUS(efim_kv_append(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7]));
}

/* cache, batch, q, out, lse, sm_scale, workspace, status, stream, plan or None, lists_resident */
static PyObject* append_prefill_attn(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p[11];
  float scale;
  size_t ws, plan_bytes;
  int32_t resident;
  if (!want(n, 11)) return NULL;
  if (!PTR(0) || !PTR(1) || !PTR(2) || !PTR(3) || !PTR(4) || !as_float(a[5], &scale) ||
      !as_workspace(a[6], &p[6], &ws) || !PTR(7) || !PTR(8) || !as_plan(a[9], &p[9], &plan_bytes) ||
      !as_i32(a[10], &resident))
    return NULL;
  if (a[9] == Py_None)
    RETURN_STATUS(efim_append_prefill_attn(p[0], p[1], p[2], p[3], p[4], scale, p[6], ws, p[7], p[8]));
  RETURN_STATUS(efim_append_prefill_attn_planned(p[0], p[1], p[9], plan_bytes, resident, p[2], p[3], p[4], scale,
                                                          p[6], ws, p[7], p[8]));
}

/* cache, batch, rope, q, k_new, v_new, out, lse, sm_scale, plan or None, lists_resident, workspace, status, stream */
static PyObject* append_prefill_step(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p[14];
  float scale;
  size_t ws, plan_bytes;
  int32_t resident;
  if (!want(n, 14)) return NULL;
  for (int i = 0; i < 8; ++i)
    if (!PTR(i)) return NULL;
  if (!as_float(a[8], &scale) || !as_plan(a[9], &p[9], &plan_bytes) || !as_i32(a[10], &resident) ||
      !as_workspace(a[11], &p[11], &ws) || !PTR(12) || !PTR(13))
    return NULL;
  RETURN_STATUS(efim_append_prefill_step(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], scale, p[9], plan_bytes,
                                                  resident, p[11], ws, p[12], p[13]));
}

/* cache, batch, ctx_len, max_ctx_len, block_table, max_pages, q, out, lse, sm_scale, workspace, status, stream */
static PyObject* decode_attn(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p[13];
  int32_t batch, max_ctx, max_pages;
  float scale;
  size_t ws;
  if (!want(n, 13)) return NULL;
  if (!PTR(0) || !as_i32(a[1], &batch) || !PTR(2) || !as_i32(a[3], &max_ctx) || !PTR(4) || !as_i32(a[5], &max_pages) ||
      !PTR(6) || !PTR(7) || !PTR(8) || !as_float(a[9], &scale) ||
      !as_workspace(a[10], &p[10], &ws) || !PTR(11) || !PTR(12))
    return NULL;
  RETURN_STATUS(efim_decode_attn(p[0], batch, p[2], max_ctx, p[4], max_pages, p[6], p[7], p[8], scale, p[10], ws,
                                          p[11], p[12]));
}

/* cache, batch, ctx_len, max_ctx_len, block_table, max_pages, rope, q, k_new, v_new, out, lse, sm_scale, workspace,
   status, stream */
static PyObject* decode_step(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p[16];
  int32_t batch, max_ctx, max_pages;
  float scale;
  size_t ws;
  if (!want(n, 16)) return NULL;
  if (!PTR(0) || !as_i32(a[1], &batch) || !PTR(2) || !as_i32(a[3], &max_ctx) || !PTR(4) || !as_i32(a[5], &max_pages))
    return NULL;
  for (int i = 6; i < 12; ++i)
    if (!PTR(i)) return NULL;
  if (!as_float(a[12], &scale) || !as_workspace(a[13], &p[13], &ws) || !PTR(14) || !PTR(15)) return NULL;
  RETURN_STATUS(efim_decode_step(p[0], batch, p[2], max_ctx, p[4], max_pages, p[6], p[7], p[8], p[9], p[10], p[11],
                                          scale, p[13], ws, p[14], p[15]));
}

/* cache, batch, norm, rope, q, q_stride, k, k_stride, v, v_stride, q_out, status, stream */
static PyObject* qk_norm_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p[13];
  int64_t q_stride, k_stride, v_stride;
  if (!want(n, 13)) return NULL;
  if (!PTR(0) || !PTR(1) || !PTR(2) || !PTR(3) || !PTR(4) || !as_i64(a[5], &q_stride) || !PTR(6) || !as_i64(a[7], &k_stride) ||
      !PTR(8) || !as_i64(a[9], &v_stride) || !PTR(10) || !PTR(11) || !PTR(12))
    return NULL;
  RETURN_STATUS(efim_qk_norm_append(p[0], p[1], p[2], p[3], p[4], q_stride, p[6], k_stride, p[8], v_stride, p[10], p[11], p[12]));
}

/* batch, history, stride, max_len, len, min_ngram, max_ngram, num_drafts, drafts, draft_len, status, stream */
static PyObject* draft_lookup(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p[12];
  int64_t stride;
  int32_t batch, max_len, lo, hi, num;
  if (!want(n, 12)) return NULL;
  if (!as_i32(a[0], &batch) || !PTR(1) || !as_i64(a[2], &stride) || !as_i32(a[3], &max_len) || !PTR(4) || !as_i32(a[5], &lo) ||
      !as_i32(a[6], &hi) || !as_i32(a[7], &num) || !PTR(8) || !PTR(9) || !PTR(10) || !PTR(11))
    return NULL;
  RETURN_STATUS(efim_draft_lookup(batch, p[1], stride, max_len, p[4], lo, hi, num, p[8], p[9], p[10], p[11]));
}

/* batch, rows, vocab, kind, row_indptr, tokens, target, stride, draft_probs, stride, uniform, noise, stride, temperature, accepted,
   next_token, out_tokens, out_logprobs, out_stride, workspace, status, stream */
static PyObject* verify_drafts(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p[22];
  efim_verify_desc d;
  int32_t out_stride;
  size_t ws;
  if (!want(n, 22)) return NULL;
  if (!as_i32(a[0], &d.batch) || !as_i32(a[1], &d.total_rows) || !as_i32(a[2], &d.vocab) || !as_i32(a[3], &d.target_kind) ||
      !PTR(4) || !PTR(5) || !PTR(6) || !as_i64(a[7], &d.target_stride) || !PTR(8) || !as_i64(a[9], &d.draft_stride) || !PTR(10) ||
      !PTR(11) || !as_i64(a[12], &d.noise_stride) || !PTR(13) || !PTR(14) || !PTR(15) || !PTR(16) || !PTR(17) ||
      !as_i32(a[18], &out_stride) || !as_workspace(a[19], &p[19], &ws) || !PTR(20) || !PTR(21))
    return NULL;
  d.d_row_indptr = p[4];
  d.d_tokens = p[5];
  d.d_target = p[6];
  d.d_draft_probs = p[8];
  d.d_uniform = p[10];
  d.d_noise = p[11];
  d.d_temperature = p[13];
  RETURN_STATUS(efim_verify_drafts(&d, p[14], p[15], p[16], p[17], out_stride, p[19], ws, p[20], p[21]));
}

static PyMethodDef methods[] = {
    {"kv_append", (PyCFunction)(void*)kv_append, METH_FASTCALL, NULL},
    {"append_prefill_attn", (PyCFunction)(void*)append_prefill_attn, METH_FASTCALL, NULL},
    {"append_prefill_step", (PyCFunction)(void*)append_prefill_step, METH_FASTCALL, NULL},
    {"decode_attn", (PyCFunction)(void*)decode_attn, METH_FASTCALL, NULL},
    {"decode_step", (PyCFunction)(void*)decode_step, METH_FASTCALL, NULL},
    {"qk_norm_append", (PyCFunction)(void*)qk_norm_append, METH_FASTCALL, NULL},
    {"draft_lookup", (PyCFunction)(void*)draft_lookup, METH_FASTCALL, NULL},
    {"verify_drafts", (PyCFunction)(void*)verify_drafts, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void) {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_nbytes = PyUnicode_InternFromString("nbytes");
  PyObject* numpy = PyImport_ImportModule("numpy");
  if (!s_data_ptr || !s_nbytes || !numpy) return NULL;
  ndarray = (PyTypeObject*)PyObject_GetAttrString(numpy, "ndarray");
  Py_DECREF(numpy);
  if (!ndarray || !PyType_Check(ndarray)) return NULL;
  return PyModule_Create(&module);
}
