/* Argument marshalling of the per-step calls (CPython extension `_calls`).
 *
 * A decode step takes the GPU a few microseconds, and converting its seventeen arguments in Python and
 * ctypes took the host about as long.  Here a call is one C function: descriptors come as addresses,
 * device memory as anything with a data_ptr() (a torch tensor), as an integer address or None, a plan as a
 * numpy array.  Calls whose tensors may be strided take shapes, types and strides from the tensors and check them.  Returns the
 * efim_status as an int; nothing else happens here. */
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
  if (v < INT32_MIN || v > INT32_MAX) {
    PyErr_Format(PyExc_OverflowError, "%ld does not fit 32 bits", v);
    return 0;
  }
  *out = (int32_t)v;
  return 1;
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

/* ---- calls that take shapes and row strides from the tensors themselves */
static PyObject *s_shape, *s_stride, *s_numel, *s_is_contiguous, *s_dtype, *s_new_empty, *kw_dtype;
static PyObject *bf16, *f32, *i32, *u8; /* torch's types, looked up by the first such call */

static int have_types(void) {
  if (i32) return 1;
  PyObject* torch = PyImport_ImportModule("torch");
  if (!torch) return 0;
  bf16 = PyObject_GetAttrString(torch, "bfloat16");
  f32 = PyObject_GetAttrString(torch, "float32");
  u8 = PyObject_GetAttrString(torch, "uint8");
  i32 = PyObject_GetAttrString(torch, "int32");
  Py_DECREF(torch);
  return bf16 && f32 && u8 && i32;
}
static int is_tensor(PyObject* o) { return o != Py_None && !PyLong_Check(o) && !PyObject_TypeCheck(o, ndarray); }
static int is_type(PyObject* o, PyObject* type) { /* -1: no such attribute */
  PyObject* t = PyObject_GetAttr(o, s_dtype);
  Py_XDECREF(t); /* (the types live on) */
  return t ? t == type : -1;
}
/* address of values of one type; an address without a type is taken at its word */
static int as_typed(PyObject* o, PyObject* type, const char* what, void** out) {
  if (is_tensor(o)) {
    const int ok = is_type(o, type);
    if (ok <= 0) {
      if (!ok) PyErr_Format(PyExc_TypeError, "%s: a tensor of %S is expected", what, type);
      return 0;
    }
  }
  return as_ptr(o, out);
}
/* at least n values of one type, packed */
static int as_vector(PyObject* o, PyObject* type, const char* what, int64_t n, void** out) {
  if (!as_typed(o, type, what, out)) return 0;
  if (!is_tensor(o)) return 1;
  PyObject* count = PyObject_CallMethodNoArgs(o, s_numel);
  PyObject* packed = count ? PyObject_CallMethodNoArgs(o, s_is_contiguous) : NULL;
  const int ok = packed ? packed == Py_True && PyLong_AsLongLong(count) >= n : -1;
  Py_XDECREF(count);
  Py_XDECREF(packed);
  if (ok == 0) PyErr_Format(PyExc_ValueError, "%s: %lld packed values are expected", what, (long long)n);
  return ok > 0;
}
/* Rows of a tensor: their number, values and the distance from one to the next.  None has none.  A row is all dimensions but the first,
   packed, where it is HEADS; where it is a LINE it is the last, and any between are of size 1. */
enum { HEADS, LINE };
static int as_rows(PyObject* o, PyObject* type, const char* what, int form, void** out, int64_t* rows, int64_t* row, int64_t* step) {
  *out = NULL;
  *rows = *row = *step = 0;
  if (o == Py_None) return 1;
  if (!as_typed(o, type, what, out)) return 0;
  PyObject* shape = PyObject_GetAttr(o, s_shape);
  PyObject* stride = shape ? PyObject_CallMethodNoArgs(o, s_stride) : NULL;
  int ok = 0;
  if (stride && PyTuple_Check(shape) && PyTuple_Check(stride) && PyTuple_GET_SIZE(shape) >= 2 &&
      PyTuple_GET_SIZE(shape) == PyTuple_GET_SIZE(stride)) {
    ok = 1;
    *row = 1;
    for (Py_ssize_t d = PyTuple_GET_SIZE(shape) - 1; d >= 0; --d) {
      const int64_t n = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, d)), s = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, d));
      if (d == 0) {
        *rows = n;
        *step = n > 1 ? s : *row; /* a single row may stand anywhere */
      } else {
        if (s != *row && n > 1) ok = 0;
        if (form == LINE && n != 1 && d < PyTuple_GET_SIZE(shape) - 1) ok = 0;
        *row *= n;
      }
    }
  }
  Py_XDECREF(shape);
  Py_XDECREF(stride);
  if (PyErr_Occurred()) return 0;
  if (!ok) PyErr_Format(PyExc_ValueError, "%s: rows of packed values are expected", what);
  if (ok && (*rows > INT32_MAX || *row > INT32_MAX)) {
    PyErr_Format(PyExc_ValueError, "%s: more rows or values of a row than 32 bits count", what);
    ok = 0;
  }
  return ok;
}
static int expect(int64_t got, int64_t wanted, const char* what) {
  if (got == wanted) return 1;
  PyErr_Format(PyExc_ValueError, "%s: %lld expected, got %lld", what, (long long)wanted, (long long)got);
  return 0;
}
/* rows of what is given, of a known shape */
static int as_matrix(PyObject* o, PyObject* type, const char* what, int form, int64_t rows, int64_t row, void** out, int64_t* step) {
  int64_t n, m;
  return as_rows(o, type, what, form, out, &n, &m, step) && (o == Py_None || (expect(n, rows, what) && expect(m, row, what)));
}

/* cache, batch, norm, head_dim of its weights (or 0), rope, q, k, v, q_out, status, stream */
static PyObject* qk_norm_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p[11];
  int32_t weights;
  int64_t qs, ks, vs, os;
  if (!want(n, 11) || !have_types()) return NULL;
  if (!PTR(0) || !PTR(1) || !PTR(2) || !as_i32(a[3], &weights) || !PTR(4) || !as_typed(a[9], i32, "status", &p[9]) || !PTR(10)) return NULL;
  const efim_cache_desc* c = p[0];
  const int64_t rows = ((const efim_batch_desc*)p[1])->total_new_tokens, q = (int64_t)c->num_q_heads * c->head_dim,
                kv = (int64_t)c->num_kv_heads * c->head_dim;
  if ((weights && !expect(weights, c->head_dim, "the norm's weights, values")) || !as_matrix(a[5], bf16, "q", HEADS, rows, q, &p[5], &qs) ||
      !as_matrix(a[6], bf16, "k", HEADS, rows, kv, &p[6], &ks) || !as_matrix(a[7], bf16, "v", HEADS, rows, kv, &p[7], &vs) ||
      !as_matrix(a[8], bf16, "q_out", HEADS, rows, q, &p[8], &os) || (p[8] && !expect(os, q, "q_out, values from one row to the next")))
    return NULL;
  RETURN_STATUS(efim_qk_norm_append(p[0], p[1], p[2], p[4], p[5], qs, p[6], ks, p[7], vs, p[8], p[9], p[10]));
}

/* history, len, min_ngram, max_ngram, drafts, draft_len, status, stream */
static PyObject* draft_lookup(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p[8];
  int64_t batch, max_len, stride, rows, num, step;
  int32_t lo, hi;
  if (!want(n, 8) || !have_types()) return NULL;
  if (!as_rows(a[0], i32, "history", LINE, &p[0], &batch, &max_len, &stride) || !as_vector(a[1], i32, "lengths", batch, &p[1]) ||
      !as_i32(a[2], &lo) || !as_i32(a[3], &hi) || !as_rows(a[4], i32, "drafts", HEADS, &p[4], &rows, &num, &step) ||
      !expect(rows, batch, "drafts, rows") || !expect(step, num, "drafts, values from one row to the next") ||
      !as_vector(a[5], i32, "draft_len", batch, &p[5]) || !as_typed(a[6], i32, "status", &p[6]) || !PTR(7))
    return NULL;
  RETURN_STATUS(efim_draft_lookup((int32_t)batch, p[0], stride, (int32_t)max_len, p[1], lo, hi, (int32_t)num, p[4], p[5], p[6], p[7]));
}

/* batch, target, target_is_probs */
static PyObject* verify_workspace_bytes(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p;
  int32_t batch;
  int64_t rows, vocab, step;
  if (!want(n, 3) || !have_types() || !as_i32(a[0], &batch)) return NULL;
  const int probs = PyObject_IsTrue(a[2]), half = probs ? 0 : is_type(a[1], bf16);
  if (probs < 0 || half < 0 || !as_rows(a[1], half ? bf16 : f32, "target", LINE, &p, &rows, &vocab, &step)) return NULL;
  const int kind = probs ? EFIM_TARGET_PROBS_F32 : half ? EFIM_TARGET_LOGITS_BF16 : EFIM_TARGET_LOGITS_F32;
  return PyLong_FromSize_t(efim_verify_workspace_bytes(batch, (int32_t)rows, (int32_t)vocab, kind));
}

/* `n` bytes beside a tensor, of torch's allocator on torch's current stream */
static PyObject* bytes_beside(PyObject* o, size_t n) {
  PyObject* size = PyLong_FromSize_t(n);
  if (!size) return NULL;
  PyObject* args[3] = {o, size, u8};
  PyObject* r = PyObject_VectorcallMethod(s_new_empty, args, 2 | PY_VECTORCALL_ARGUMENTS_OFFSET, kw_dtype);
  Py_DECREF(size);
  return r;
}

/* batch, row_indptr, tokens, target, target_is_probs, draft_probs, uniform, noise, temperature, accepted, next_token, out_tokens,
   out_logprobs, workspace or None (one is taken beside the target), status, stream */
static PyObject* verify_drafts(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p[16];
  efim_verify_desc d;
  int64_t rows, vocab, out_rows, step, width = 0, logs = 0;
  size_t ws;
  PyObject* own = NULL;
  if (!want(n, 16) || !have_types()) return NULL;
  const int probs = PyObject_IsTrue(a[4]), half = probs ? 0 : is_type(a[3], bf16);
  if (probs < 0 || half < 0) return NULL;
  if (!as_i32(a[0], &d.batch) || !as_vector(a[1], i32, "row_indptr", (int64_t)d.batch + 1, &p[1]) ||
      !as_rows(a[3], half ? bf16 : f32, "target", LINE, &p[3], &rows, &vocab, &d.target_stride) ||
      !as_vector(a[2], i32, "tokens", rows, &p[2]) || !as_matrix(a[5], f32, "draft_probs", LINE, rows, vocab, &p[5], &d.draft_stride) ||
      !as_vector(a[6], f32, "uniform", rows, &p[6]) || !as_matrix(a[7], f32, "noise", LINE, d.batch, vocab, &p[7], &d.noise_stride) ||
      !as_vector(a[8], f32, "temperature", d.batch, &p[8]) || !as_vector(a[9], i32, "accepted", d.batch, &p[9]) ||
      !as_vector(a[10], i32, "next_token", d.batch, &p[10]) ||
      !as_rows(a[11], i32, "out_tokens", HEADS, &p[11], &out_rows, &width, &step) ||
      (p[11] && (!expect(out_rows, d.batch, "out_tokens, rows") || !expect(step, width, "out_tokens, values from one row to the next"))) ||
      !as_rows(a[12], f32, "out_logprobs", HEADS, &p[12], &out_rows, &logs, &step) ||
      (p[12] && (!expect(out_rows, d.batch, "out_logprobs, rows") || !expect(step, logs, "out_logprobs, values from one row to the next"))) ||
      (p[11] && p[12] && !expect(logs, width, "out_logprobs, values of a row")) || !as_workspace(a[13], &p[13], &ws) ||
      !as_typed(a[14], i32, "status", &p[14]) || !PTR(15))
    return NULL;
  d.total_rows = (int32_t)rows;
  d.vocab = (int32_t)vocab;
  d.target_kind = probs ? EFIM_TARGET_PROBS_F32 : half ? EFIM_TARGET_LOGITS_BF16 : EFIM_TARGET_LOGITS_F32;
  d.d_row_indptr = p[1];
  d.d_tokens = p[2];
  d.d_target = p[3];
  d.d_draft_probs = p[5];
  d.d_uniform = p[6];
  d.d_noise = p[7];
  d.d_temperature = p[8];
  if (a[13] == Py_None) {
    ws = efim_verify_workspace_bytes(d.batch, d.total_rows, d.vocab, d.target_kind);
    if (ws > 0 && (!(own = bytes_beside(a[3], ws)) || !as_ptr(own, &p[13]))) {
      Py_XDECREF(own);
      return NULL;
    }
  }
  efim_status st;
  Py_BEGIN_ALLOW_THREADS
  st = efim_verify_drafts(&d, p[9], p[10], p[11], p[12], (int32_t)(p[11] ? width : logs), p[13], ws, p[14], p[15]);
  Py_END_ALLOW_THREADS
  Py_XDECREF(own); /* (whatever takes its place next comes behind the call on the stream) */
  return PyLong_FromLong(st);
}

static PyMethodDef methods[] = {
    {"kv_append", (PyCFunction)(void*)kv_append, METH_FASTCALL, NULL},
    {"append_prefill_attn", (PyCFunction)(void*)append_prefill_attn, METH_FASTCALL, NULL},
    {"append_prefill_step", (PyCFunction)(void*)append_prefill_step, METH_FASTCALL, NULL},
    {"decode_attn", (PyCFunction)(void*)decode_attn, METH_FASTCALL, NULL},
    {"decode_step", (PyCFunction)(void*)decode_step, METH_FASTCALL, NULL},
    {"qk_norm_append", (PyCFunction)(void*)qk_norm_append, METH_FASTCALL, NULL},
    {"draft_lookup", (PyCFunction)(void*)draft_lookup, METH_FASTCALL, NULL},
    {"verify_workspace_bytes", (PyCFunction)(void*)verify_workspace_bytes, METH_FASTCALL, NULL},
    {"verify_drafts", (PyCFunction)(void*)verify_drafts, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void) {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_nbytes = PyUnicode_InternFromString("nbytes");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_numel = PyUnicode_InternFromString("numel");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_new_empty = PyUnicode_InternFromString("new_empty");
  kw_dtype = s_dtype ? PyTuple_Pack(1, s_dtype) : NULL;
  PyObject* numpy = PyImport_ImportModule("numpy");
  if (!s_data_ptr || !s_nbytes || !s_shape || !s_stride || !s_numel || !s_is_contiguous || !s_dtype || !s_new_empty || !kw_dtype || !numpy) return NULL;
  ndarray = (PyTypeObject*)PyObject_GetAttrString(numpy, "ndarray");
  Py_DECREF(numpy);
  if (!ndarray || !PyType_Check(ndarray)) return NULL;
  return PyModule_Create(&module);
}
