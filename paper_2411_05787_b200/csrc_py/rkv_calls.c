/* The 8-bit cache's calls and rkv_rope as a CPython extension: argument checks and marshalling for rkv.Context.
 *
 * A decode loop issues these calls once per layer and token, and one of them runs for 2 to 5 us on the GPU: checked in
 * Python and marshalled by ctypes, a call costs the host 7 to 11 us, of which the library (the launch) needs 2.5.
 * Here the checks are C calls of the tensors' own methods.  Every function takes a context's key
 *   (handle, n_seq, n_q_heads, n_kv_heads, device)
 * first and its stream last (None: the device's current one; an object with a cuda_stream; a number), raises ValueError
 * for tensors that do not fit, and returns the library's status.  The tensors' memory is the caller's, as in the library.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "rkv.h"

static PyObject *s_dtype, *s_shape, *s_stride, *s_numel, *s_get_device, *s_is_contiguous, *s_data_ptr, *s_cuda_stream,
    *s_device, *s_n_seq, *s_freqs, *s_rot_dim, *s_layout, *s_amplitude;
/* set once by setup() */
static PyObject *t_bf16, *t_f32, *t_i32, *c_quant_cache, *c_cache, *c_table, *f_stream;

typedef struct {
  rkv_ctx* ctx;
  long long n_seq, n_q, n_kv;
  long device;
} Key;

/* ------------------------------------------------------------------------------------------------ reading arguments */
static int as_key(PyObject* o, Key* k) {
  if (t_bf16 == NULL || !PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 5) {
    PyErr_SetString(PyExc_TypeError, "a context's key is a tuple of five numbers");
    return -1;
  }
  k->ctx = (rkv_ctx*)PyLong_AsVoidPtr(PyTuple_GET_ITEM(o, 0));
  k->n_seq = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 1));
  k->n_q = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 2));
  k->n_kv = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 3));
  k->device = PyLong_AsLong(PyTuple_GET_ITEM(o, 4));
  return PyErr_Occurred() ? -1 : 0;
}

static int as_i32(PyObject* o, int32_t* out) {
  int overflow = 0;
  const long v = PyLong_AsLongAndOverflow(o, &overflow);
  if (v == -1 && PyErr_Occurred()) return -1;
  if (overflow != 0 || v < INT32_MIN || v > INT32_MAX) {
    PyErr_SetString(PyExc_ValueError, "a number does not fit 32 bits");
    return -1;
  }
  *out = (int32_t)v;
  return 0;
}

static int attr_ll(PyObject* o, PyObject* name, long long* out) {
  PyObject* r = PyObject_GetAttr(o, name);
  if (r == NULL) return -1;
  *out = PyLong_AsLongLong(r);
  Py_DECREF(r);
  return (*out == -1 && PyErr_Occurred()) ? -1 : 0;
}

static int method_ll(PyObject* o, PyObject* name, long long* out) {
  PyObject* r = PyObject_CallMethodNoArgs(o, name);
  if (r == NULL) return -1;
  *out = PyLong_AsLongLong(r);
  Py_DECREF(r);
  return (*out == -1 && PyErr_Occurred()) ? -1 : 0;
}

static int pointer_of(PyObject* t, void** out) {
  PyObject* r = PyObject_CallMethodNoArgs(t, s_data_ptr);
  if (r == NULL) return -1;
  *out = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return (*out == NULL && PyErr_Occurred()) ? -1 : 0;
}

static int has_dtype(PyObject* t, PyObject* want) { /* 1, 0, -1 on error */
  PyObject* d = PyObject_GetAttr(t, s_dtype);
  if (d == NULL) return -1;
  const int same = d == want;
  Py_DECREF(d);
  return same;
}

static int on_device(PyObject* t, long device, const char* what) {
  long long dev;
  if (method_ll(t, s_get_device, &dev) != 0) return -1;
  if (dev != device) {
    PyErr_Format(PyExc_ValueError, "%s is on another device than the context", what);
    return -1;
  }
  return 0;
}

enum { kOptional = 0, kRequired = 1 };

/* Device pointer of a contiguous tensor of the context's device with this type and number of elements. */
static int tensor(PyObject* t, PyObject* dtype, long long numel, long device, int required, const char* what, void** out) {
  *out = NULL;
  if (t == Py_None) {
    if (!required) return 0;
    PyErr_Format(PyExc_ValueError, "%s is missing", what);
    return -1;
  }
  const int same = has_dtype(t, dtype);
  if (same < 0) return -1;
  long long n;
  if (method_ll(t, s_numel, &n) != 0) return -1;
  if (!same || n != numel) {
    PyErr_Format(PyExc_ValueError, "%s: %R with %lld elements expected", what, dtype, numel);
    return -1;
  }
  if (on_device(t, device, what) != 0) return -1;
  PyObject* c = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  if (c == NULL) return -1;
  Py_DECREF(c); /* (True and False are immortal) */
  if (c != Py_True) {
    PyErr_Format(PyExc_ValueError, "%s: librkv takes contiguous tensors", what);
    return -1;
  }
  return pointer_of(t, out);
}

/* q, out, q_last_full */
static int queries(PyObject* t, const Key* k, int required, void** out) {
  return tensor(t, t_bf16, k->n_seq * k->n_q * RKV_HEAD_DIM, k->device, required, "queries and outputs [B, Hq, 128]", out);
}
static int per_seq(PyObject* t, const Key* k, int required, void** out) {
  return tensor(t, t_i32, k->n_seq, k->device, required, "a per-sequence argument [B]", out);
}
static int indices(PyObject* t, const Key* k, int32_t k_max, void** out) {
  return tensor(t, t_i32, k->n_seq * k->n_kv * (long long)k_max, k->device, kRequired, "topk_idx [B, Hkv, k_max]", out);
}
static int dims(PyObject* t, PyObject* name, int call, Py_ssize_t want, long long* out) { /* shape, or stride() */
  PyObject* s = call ? PyObject_CallMethodNoArgs(t, name) : PyObject_GetAttr(t, name);
  if (s == NULL) return -1;
  int ok = PyTuple_Check(s);
  const Py_ssize_t n = ok ? PyTuple_GET_SIZE(s) : 0;
  if (ok && n == want)
    for (Py_ssize_t i = 0; i < n; ++i) out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(s, i));
  Py_DECREF(s);
  if (PyErr_Occurred()) return -1;
  return (int)n;
}
static int score_rows(PyObject* t, const Key* k, void** out, int64_t* stride) {
  *out = NULL;
  *stride = 0;
  if (t == Py_None) return 0;
  long long shape[3];
  const int n = dims(t, s_shape, 0, 3, shape);
  if (n < 0) return -1;
  if (n != 3) {
    PyErr_SetString(PyExc_ValueError, "scores is a float32 tensor [B, Hkv, stride]");
    return -1;
  }
  *stride = shape[2];
  return tensor(t, t_f32, k->n_seq * k->n_kv * shape[2], k->device, kRequired, "scores [B, Hkv, stride]", out);
}

/* The struct inside a ctypes object of exactly this class. */
static int structure(PyObject* o, PyObject* cls, const char* what, void* to, Py_ssize_t size) {
  if ((PyObject*)Py_TYPE(o) != cls) {
    PyErr_Format(PyExc_TypeError, "%s expected, %.100s given", what, Py_TYPE(o)->tp_name);
    return -1;
  }
  Py_buffer view;
  if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) return -1;
  const int fits = view.len == size;
  if (fits) memcpy(to, view.buf, (size_t)size);
  PyBuffer_Release(&view);
  if (!fits) PyErr_Format(PyExc_TypeError, "%s: another size than the library's struct", what);
  return fits ? 0 : -1;
}
static int quant_cache(PyObject* o, const Key* k, rkv_quant_cache* c) {
  if (structure(o, c_quant_cache, "an RkvQuantCache", c, sizeof(*c)) != 0) return -1;
  long long device, n_seq;
  if (attr_ll(o, s_device, &device) != 0 || attr_ll(o, s_n_seq, &n_seq) != 0) return -1;
  if (device != k->device) {
    PyErr_SetString(PyExc_ValueError, "the cache is on another device than the context");
    return -1;
  }
  if (n_seq != k->n_seq) {
    PyErr_SetString(PyExc_ValueError, "the cache holds another number of sequences than the context");
    return -1;
  }
  return 0;
}
/* The small cache's tensors are on the context's device and describe its sequences (the kernel writes where they say). */
static int small_cache_fits(PyObject* o, const Key* k) {
  long long device, n_seq;
  if (attr_ll(o, s_device, &device) != 0 || attr_ll(o, s_n_seq, &n_seq) != 0) {
    if (PyErr_ExceptionMatches(PyExc_AttributeError))
      PyErr_SetString(PyExc_ValueError, "the small cache is one that cache_struct describes");
    return -1;
  }
  if (device != k->device) {
    PyErr_SetString(PyExc_ValueError, "the small cache is on another device than the context");
    return -1;
  }
  if (n_seq < k->n_seq) {
    PyErr_SetString(PyExc_ValueError, "the small cache holds fewer sequences than the context");
    return -1;
  }
  return 0;
}

static int stream_of(PyObject* o, long device, void** out) {
  PyObject* r;
  if (o == Py_None) {
    PyObject* d = PyLong_FromLong(device);
    if (d == NULL) return -1;
    r = PyObject_CallOneArg(f_stream, d);
    Py_DECREF(d);
  } else if (PyLong_Check(o)) {
    r = Py_NewRef(o);
  } else {
    r = PyObject_GetAttr(o, s_cuda_stream);
  }
  if (r == NULL) return -1;
  *out = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return (*out == NULL && PyErr_Occurred()) ? -1 : 0;
}

static int count_args(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return 0;
  PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, n);
  return -1;
}

/* The library is called without the interpreter's lock, as ctypes would: a launch may wait for room in the queue. */
#define CALL(expr)                \
  do {                            \
    rkv_status rc;                \
    Py_BEGIN_ALLOW_THREADS        \
    rc = (expr);                  \
    Py_END_ALLOW_THREADS          \
    return PyLong_FromLong((long)rc); \
  } while (0)

/* ------------------------------------------------------------------------------------------------------------- calls */
static int new_rows(PyObject* x, const Key* k, const char* what, void** at, int64_t* seq, int64_t* tok, long long* n_tok) {
  long long shape[4], stride[4];
  const int same = has_dtype(x, t_bf16), n = dims(x, s_shape, 0, 4, shape);
  if (same < 0 || n < 0) return -1;
  if (!same || n != 4 || shape[0] != k->n_seq || shape[2] != k->n_kv || shape[3] != RKV_HEAD_DIM || shape[1] < 1 ||
      shape[1] > INT32_MAX) {
    PyErr_Format(PyExc_ValueError, "%s is a bfloat16 tensor [B, T, Hkv, 128]", what);
    return -1;
  }
  if (on_device(x, k->device, what) != 0 || dims(x, s_stride, 1, 4, stride) != 4) return -1;
  if (stride[3] != 1 || (stride[2] != RKV_HEAD_DIM && shape[2] > 1)) {
    PyErr_SetString(PyExc_ValueError, "the heads of a new row lie side by side");
    return -1;
  }
  *seq = shape[0] > 1 ? stride[0] : 0; /* (a stride that is never taken may have any value) */
  *tok = shape[1] > 1 ? stride[1] : 0;
  *n_tok = shape[1];
  if (pointer_of(x, at) != 0) return -1;
  if (*seq % 8 != 0 || *tok % 8 != 0 || (uintptr_t)*at % 16 != 0) {
    PyErr_SetString(PyExc_ValueError, "new rows start on 16-byte boundaries");
    return -1;
  }
  return 0;
}

/* quant_store(key, k_new, v_new, full, start, count, stream) */
static PyObject* quant_store(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Key k;
  rkv_quant_cache full;
  void *kn, *vn, *start, *count, *st;
  int64_t ks, kt, vs, vt;
  long long tk, tv;
  if (count_args(n, 7) || as_key(a[0], &k) || quant_cache(a[3], &k, &full) || new_rows(a[1], &k, "k_new", &kn, &ks, &kt, &tk) ||
      new_rows(a[2], &k, "v_new", &vn, &vs, &vt, &tv))
    return NULL;
  if (tk != tv) {
    PyErr_SetString(PyExc_ValueError, "k_new and v_new hold the same number of rows");
    return NULL;
  }
  if (per_seq(a[4], &k, kOptional, &start) || per_seq(a[5], &k, kOptional, &count) || stream_of(a[6], k.device, &st))
    return NULL;
  CALL(rkv_quant_store(k.ctx, kn, ks, kt, vn, vs, vt, (int32_t)tk, start, count, &full, st));
}

/* quant_full_attention(key, q, full, out, active, max_len_hint, keep_logits, stream) */
static PyObject* quant_full_attention(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Key k;
  rkv_quant_cache full;
  void *q, *out, *active, *st;
  int32_t hint;
  int keep;
  if (count_args(n, 8) || as_key(a[0], &k) || quant_cache(a[2], &k, &full) || queries(a[1], &k, kRequired, &q) ||
      queries(a[3], &k, kRequired, &out) || per_seq(a[4], &k, kOptional, &active) || as_i32(a[5], &hint) ||
      (keep = PyObject_IsTrue(a[6])) < 0 || stream_of(a[7], k.device, &st))
    return NULL;
  CALL(rkv_quant_full_attention(k.ctx, q, &full, active, out, keep, hint, st));
}

/* quant_score_keys(key, q, full, k_small, k_max, active, scores, q_last_full, stream) */
static PyObject* quant_score_keys(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Key k;
  rkv_quant_cache full;
  void *q, *k_small, *active, *scores, *last, *st;
  int64_t stride;
  int32_t k_max;
  if (count_args(n, 9) || as_key(a[0], &k) || quant_cache(a[2], &k, &full) || queries(a[1], &k, kOptional, &q) ||
      per_seq(a[3], &k, kRequired, &k_small) || as_i32(a[4], &k_max) || per_seq(a[5], &k, kOptional, &active) ||
      score_rows(a[6], &k, &scores, &stride) || queries(a[7], &k, kOptional, &last) || stream_of(a[8], k.device, &st))
    return NULL;
  CALL(rkv_quant_score_keys(k.ctx, q, &full, k_small, k_max, active, scores, stride, last, st));
}

/* quant_select_topk(key, q, full, k_small, k_max, topk_idx, active, scores, q_last_full, stream) */
static PyObject* quant_select_topk(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Key k;
  rkv_quant_cache full;
  void *q, *k_small, *idx, *active, *scores, *last, *st;
  int64_t stride;
  int32_t k_max;
  if (count_args(n, 10) || as_key(a[0], &k) || quant_cache(a[2], &k, &full) || queries(a[1], &k, kOptional, &q) ||
      per_seq(a[3], &k, kRequired, &k_small) || as_i32(a[4], &k_max) || indices(a[5], &k, k_max, &idx) ||
      per_seq(a[6], &k, kOptional, &active) || score_rows(a[7], &k, &scores, &stride) ||
      queries(a[8], &k, kOptional, &last) || stream_of(a[9], k.device, &st))
    return NULL;
  CALL(rkv_quant_select_topk(k.ctx, q, &full, k_small, k_max, active, scores, stride, idx, last, st));
}

/* quant_full_step(key, q, full, k_small, k_max, out, topk_idx, active, scores, q_last_full, max_len_hint, stream) */
static PyObject* quant_full_step(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Key k;
  rkv_quant_cache full;
  void *q, *k_small, *out, *idx, *active, *scores, *last, *st;
  int64_t stride;
  int32_t k_max, hint;
  if (count_args(n, 12) || as_key(a[0], &k) || quant_cache(a[2], &k, &full) || queries(a[1], &k, kRequired, &q) ||
      per_seq(a[3], &k, kRequired, &k_small) || as_i32(a[4], &k_max) || queries(a[5], &k, kRequired, &out) ||
      indices(a[6], &k, k_max, &idx) || per_seq(a[7], &k, kOptional, &active) || score_rows(a[8], &k, &scores, &stride) ||
      queries(a[9], &k, kOptional, &last) || as_i32(a[10], &hint) || stream_of(a[11], k.device, &st))
    return NULL;
  CALL(rkv_quant_full_step(k.ctx, q, &full, k_small, k_max, active, out, scores, stride, idx, last, hint, st));
}

/* quant_gather_small(key, topk_idx, k_small, k_max, full, small, active, stream) */
static PyObject* quant_gather_small(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Key k;
  rkv_quant_cache full;
  rkv_cache small;
  void *idx, *k_small, *active, *st;
  int32_t k_max;
  if (count_args(n, 8) || as_key(a[0], &k) || quant_cache(a[4], &k, &full) ||
      structure(a[5], c_cache, "an RkvCache", &small, sizeof(small)) || as_i32(a[3], &k_max) || small_cache_fits(a[5], &k) ||
      indices(a[1], &k, k_max, &idx) || per_seq(a[2], &k, kRequired, &k_small) || per_seq(a[6], &k, kOptional, &active) ||
      stream_of(a[7], k.device, &st))
    return NULL;
  CALL(rkv_quant_gather_small(k.ctx, idx, k_small, k_max, &full, &small, active, st));
}

/* rope(key, qkv, pos, table, q, k, v, stream) */
static PyObject* rope(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Key k;
  void *at, *pos, *freqs, *q, *kk, *v, *st;
  long long shape[2], stride[2], qs[3], ks[3], rot, layout;
  if (count_args(n, 8) || as_key(a[0], &k)) return NULL;
  PyObject *qkv = a[1], *table = a[3];
  const int bf16 = has_dtype(qkv, t_bf16), f32 = has_dtype(qkv, t_f32);
  if (bf16 < 0 || f32 < 0) return NULL;
  const int d0 = dims(qkv, s_shape, 0, 2, shape), d1 = dims(a[4], s_shape, 0, 3, qs), d2 = dims(a[5], s_shape, 0, 3, ks);
  if (d0 < 0 || d1 < 0 || d2 < 0) return NULL;
  if (d1 != 3 || d2 != 3) {
    PyErr_SetString(PyExc_ValueError, "q is a tensor [T, Hq, 128], k and v are tensors [T, Hkv, 128]");
    return NULL;
  }
  const long long n_q = qs[1], n_kv = ks[1];
  if (!(bf16 || f32) || d0 != 2 || n_q < 1 || n_kv < 1 || n_q > (1 << 16) || n_kv > (1 << 16) || shape[0] < 1 ||
      shape[0] > INT32_MAX || shape[1] != (n_q + 2 * n_kv) * RKV_HEAD_DIM) {
    PyErr_SetString(PyExc_ValueError, "qkv is a bfloat16 or float32 tensor [T, (Hq + 2 Hkv) * 128]");
    return NULL;
  }
  if (on_device(qkv, k.device, "qkv") || dims(qkv, s_stride, 1, 2, stride) != 2 || pointer_of(qkv, &at)) return NULL;
  const long long n_tok = shape[0], tok = n_tok > 1 ? stride[0] : 0;
  if (stride[1] != 1 || tok % (bf16 ? 8 : 4) != 0 || (uintptr_t)at % 16 != 0) {
    PyErr_SetString(PyExc_ValueError, "the projection's rows are contiguous and start on 16-byte boundaries");
    return NULL;
  }
  if ((PyObject*)Py_TYPE(table) != c_table) {
    PyErr_SetString(PyExc_TypeError, "a RopeTable expected");
    return NULL;
  }
  PyObject* fr = PyObject_GetAttr(table, s_freqs);
  if (fr == NULL) return NULL;
  const int bad = on_device(fr, k.device, "the table") || pointer_of(fr, &freqs);
  Py_DECREF(fr); /* (the table keeps it) */
  if (bad || attr_ll(table, s_rot_dim, &rot) || attr_ll(table, s_layout, &layout)) return NULL;
  PyObject* am = PyObject_GetAttr(table, s_amplitude);
  if (am == NULL) return NULL;
  const double amplitude = PyFloat_AsDouble(am);
  Py_DECREF(am);
  if (amplitude == -1.0 && PyErr_Occurred()) return NULL;
  if (tensor(a[2], t_i32, n_tok, k.device, kRequired, "pos [T]", &pos) ||
      tensor(a[4], t_bf16, n_tok * n_q * RKV_HEAD_DIM, k.device, kRequired, "q [T, Hq, 128]", &q) ||
      tensor(a[5], t_bf16, n_tok * n_kv * RKV_HEAD_DIM, k.device, kRequired, "k [T, Hkv, 128]", &kk) ||
      tensor(a[6], t_bf16, n_tok * n_kv * RKV_HEAD_DIM, k.device, kOptional, "v [T, Hkv, 128]", &v) ||
      stream_of(a[7], k.device, &st))
    return NULL;
  CALL(rkv_rope(k.ctx, at, bf16, tok, pos, (int32_t)n_tok, (int32_t)n_q, (int32_t)n_kv, freqs, (int32_t)rot, (int32_t)layout,
                (float)amplitude, q, kk, v, st));
}

/* setup(bfloat16, float32, int32, RkvQuantCache, RkvCache, RopeTable, raw_stream): what the checks compare with */
static PyObject* setup(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (count_args(n, 7)) return NULL;
  PyObject** to[7] = {&t_bf16, &t_f32, &t_i32, &c_quant_cache, &c_cache, &c_table, &f_stream};
  for (int i = 0; i < 7; ++i) Py_XSETREF(*to[i], Py_NewRef(a[i]));
  Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(setup), METHOD(quant_store), METHOD(quant_full_attention), METHOD(quant_score_keys),
                                METHOD(quant_select_topk), METHOD(quant_full_step), METHOD(quant_gather_small),
                                METHOD(rope), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rkv_calls", "Checked calls of librkv.", -1, methods,
                                    NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__rkv_calls(void) {
  PyObject** names[] = {&s_dtype, &s_shape, &s_stride, &s_numel, &s_get_device, &s_is_contiguous, &s_data_ptr,
                        &s_cuda_stream, &s_device, &s_n_seq, &s_freqs, &s_rot_dim, &s_layout, &s_amplitude};
  const char* text[] = {"dtype", "shape", "stride", "numel", "get_device", "is_contiguous", "data_ptr",
                        "cuda_stream", "device", "n_seq", "freqs", "rot_dim", "layout", "amplitude"};
  for (size_t i = 0; i < sizeof(names) / sizeof(names[0]); ++i)
    if ((*names[i] = PyUnicode_InternFromString(text[i])) == NULL) return NULL;
  return PyModule_Create(&module);
}
