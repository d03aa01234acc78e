/* CPython shim for the calls a program makes per layer and step: takes the tensors themselves, reads what the
 * C entry point wants to know of them and calls it.  Through ctypes the same marshalling (eleven arguments
 * converted one by one, as many attribute look-ups from bytecode) took 3.6 us of a call's 8.5.
 * No arithmetic, no checks of its own: those are the library's. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

static PyObject *s_data_ptr, *s_size, *s_shape, *s_stride, *s_numel, *s_is_contiguous, *s_dtype, *s_get_device, *zero, *one, *float32_type, *bfloat16_type, *int32_type, *int64_type;
static PyTypeObject *tensor_type;

typedef int (*linear_fn)(const void *, const void *, const void *, int64_t, int64_t, void *, int32_t, int64_t, void *, size_t,
                         void *);
typedef int (*quantise_fn)(const void *, const void *, int64_t, int64_t, int64_t, void *, void *, int32_t, void *);

/* A tensor's data pointer, None, or whatever int() takes; bits above 64 are dropped, as ctypes does. */
static int as_pointer(PyObject *o, void **out) {
  if (o == Py_None) { *out = NULL; return 0; }
  PyObject *r = PyLong_Check(o)                        ? Py_NewRef(o)
                : PyObject_TypeCheck(o, tensor_type) ? PyObject_CallMethodNoArgs(o, s_data_ptr)
                                                     : PyNumber_Long(o);
  if (r == NULL) return -1;
  *out = (void *)(uintptr_t)PyLong_AsUnsignedLongLongMask(r);
  Py_DECREF(r);
  return PyErr_Occurred() ? -1 : 0;
}

static int as_int(PyObject *o, PyObject *method, PyObject *arg, int64_t *out) {
  PyObject *r = arg ? PyObject_CallMethodOneArg(o, method, arg) : PyObject_CallMethodNoArgs(o, method);
  if (r == NULL) return -1;
  *out = (int64_t)PyLong_AsLongLong(r);
  Py_DECREF(r);
  return PyErr_Occurred() ? -1 : 0;
}

/* x.shape[i]; of a tensor without the torch.Size. */
static int as_extent(PyObject *o, PyObject *i, int64_t *out) {
  if (PyObject_TypeCheck(o, tensor_type)) return as_int(o, s_size, i, out);
  PyObject *shape = PyObject_GetAttr(o, s_shape);
  if (shape == NULL) return -1;
  PyObject *r = PyObject_GetItem(shape, i);
  Py_DECREF(shape);
  if (r == NULL) return -1;
  *out = (int64_t)PyLong_AsLongLong(r);
  Py_DECREF(r);
  return PyErr_Occurred() ? -1 : 0;
}

/* linear(function, transform, weight, x, y, workspace, stream) -> status */
static PyObject *linear(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  if (n != 7) { PyErr_SetString(PyExc_TypeError, "linear: 7 arguments"); return NULL; }
  void *fn, *t, *w, *x, *y, *ws, *stream;
  int64_t s, ld, ldy, bytes;
  if (as_pointer(a[0], &fn) || as_pointer(a[1], &t) || as_pointer(a[2], &w) || as_extent(a[3], zero, &s) ||
      as_int(a[3], s_stride, zero, &ld) || as_pointer(a[3], &x) || as_pointer(a[4], &y) ||
      as_int(a[4], s_stride, zero, &ldy) || as_pointer(a[5], &ws) || as_int(a[5], s_numel, NULL, &bytes) ||
      as_pointer(a[6], &stream))
    return NULL;
  PyObject *dt = PyObject_GetAttr(a[4], s_dtype);
  if (dt == NULL) return NULL;
  const int32_t y_dtype = dt == float32_type ? 0 : 1;   /* BATQ_F32, BATQ_BF16 */
  Py_DECREF(dt);
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = ((linear_fn)fn)(t, w, x, s, ld, y, y_dtype, ldy, ws, (size_t)bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* quantise(function, transform, x, codes, scales, scale_layout, stream) -> status */
static PyObject *quantise(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  if (n != 7) { PyErr_SetString(PyExc_TypeError, "quantise: 7 arguments"); return NULL; }
  void *fn, *t, *x, *codes, *scales, *stream;
  int64_t s, cols, ld;
  if (as_pointer(a[0], &fn) || as_pointer(a[1], &t) || as_extent(a[2], zero, &s) || as_extent(a[2], one, &cols) ||
      as_int(a[2], s_stride, zero, &ld) || as_pointer(a[2], &x) || as_pointer(a[3], &codes) ||
      as_pointer(a[4], &scales) || as_pointer(a[6], &stream))
    return NULL;
  if (!PyLong_Check(a[5])) { PyErr_SetString(PyExc_TypeError, "quantise: scale_layout is not an int"); return NULL; }
  const unsigned long layout = PyLong_AsUnsignedLongMask(a[5]);
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = ((quantise_fn)fn)(t, x, s, cols, ld, codes, scales, (int32_t)layout, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

typedef int (*append_fn)(const void *, const void *, const void *, const void *, const void *, int64_t, const void *, int64_t,
                         const void *, int64_t, void *, int64_t, int32_t, int64_t, const void *, const void *, const void *,
                         int64_t, int32_t, void *);
typedef int (*attention_fn)(const void *, const void *, int64_t, int32_t, int64_t, const void *, const void *, const void *,
                            int64_t, int32_t, int32_t, int32_t, float, int32_t, void *, int64_t, void *, void *, size_t, void *);

static int as_int32(PyObject *o, int32_t *out) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) return -1;
  if (v < INT32_MIN || v > INT32_MAX) { PyErr_SetString(PyExc_OverflowError, "does not fit 32 bits"); return -1; }
  *out = (int32_t)v;
  return 0;
}

/* The kernels take sizes, types and places on trust: a tensor that is shorter, or of another type, would be read or written
 * past its end, one of the host's or of another GPU's memory is not there for them.  So these two look at what they are
 * given (as binding.py does where this shim is missing); for the devices that is 0.5 us a call. */
static int is_on(PyObject *o, int64_t device, const char *what) {
  int64_t at;
  if (as_int(o, s_get_device, NULL, &at)) return -1;
  if (at != device) { PyErr_Format(PyExc_ValueError, "%s: on device %lld, the cache is on %lld", what, (long long)at, (long long)device); return -1; }
  return 0;
}

static int is_type(PyObject *o, PyObject *want, const char *what) {
  PyObject *dt = PyObject_GetAttr(o, s_dtype);
  if (dt == NULL) return -1;
  Py_DECREF(dt);
  if (dt != want) { PyErr_Format(PyExc_ValueError, "%s: %R is wanted", what, want); return -1; }
  return 0;
}

/* A bf16 matrix of at least `tokens` rows and, unless 0, of `width` columns, which are dense: address, rows, columns, stride. */
static int as_rows(PyObject *o, int64_t device, int64_t tokens, int64_t width, const char *what, void **p, int64_t *n, int64_t *w, int64_t *ld) {
  int64_t step;
  if (is_type(o, bfloat16_type, what) || as_pointer(o, p) || as_extent(o, zero, n) || as_extent(o, one, w) || as_int(o, s_stride, zero, ld) ||
      as_int(o, s_stride, one, &step) || is_on(o, device, what))
    return -1;
  if (*n < tokens || (width != 0 && *w != width) || *w == 0 || (step != 1 && *w > 1)) {
    PyErr_Format(PyExc_ValueError, "%s: %lld dense bf16 rows, %lld wide", what, (long long)tokens, (long long)(width ? width : *w));
    return -1;
  }
  return 0;
}

/* A dense vector of at least n entries, or None. */
static int as_vector(PyObject *o, int64_t device, PyObject *type, int64_t n, const char *what, void **p) {
  if (as_pointer(o, p) || o == Py_None) return PyErr_Occurred() ? -1 : 0;
  int64_t size, step;
  if (is_type(o, type, what) || as_extent(o, zero, &size) || as_int(o, s_stride, zero, &step) || is_on(o, device, what)) return -1;
  if (size < n || (step != 1 && n > 1)) { PyErr_Format(PyExc_ValueError, "%s: a dense vector of %lld entries", what, (long long)n); return -1; }
  return 0;
}

/* kv_append(function, cache, device, kv_heads, head_dim, t_k, t_v, t_q, k, v, q, q_out, slots, positions, rope, stream) -> status */
static PyObject *kv_append(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  if (n != 16) { PyErr_SetString(PyExc_TypeError, "kv_append: 16 arguments"); return NULL; }
  void *fn, *c, *tk, *tv, *tq, *k, *v, *q = NULL, *q_out = NULL, *slots, *positions, *rope, *stream;
  int64_t ldk, ldv, ldq = 0, ldqo = 0, tokens, rows, w, width = 0, rope_rows = 0, rot = 0, step;
  int32_t heads, d, dev;
  if (as_pointer(a[0], &fn) || as_pointer(a[1], &c) || as_int32(a[2], &dev) || as_int32(a[3], &heads) || as_int32(a[4], &d) || as_pointer(a[5], &tk) ||
      as_pointer(a[6], &tv) || as_pointer(a[7], &tq) || as_rows(a[8], dev, 0, (int64_t)heads * d, "k", &k, &tokens, &w, &ldk) ||
      as_rows(a[9], dev, tokens, (int64_t)heads * d, "v", &v, &rows, &w, &ldv) || as_vector(a[12], dev, int64_type, tokens, "slots", &slots) ||
      as_vector(a[13], dev, int32_type, tokens, "positions", &positions) || as_pointer(a[14], &rope) || as_pointer(a[15], &stream))
    return NULL;
  if (a[10] != Py_None && as_rows(a[10], dev, tokens, 0, "q", &q, &rows, &width, &ldq)) return NULL;
  if (width % d != 0) { PyErr_SetString(PyExc_ValueError, "q: whole heads"); return NULL; }
  if (a[11] != Py_None && as_rows(a[11], dev, tokens, width, "q_out", &q_out, &rows, &w, &ldqo)) return NULL;
  if (a[14] != Py_None) {
    if (is_type(a[14], float32_type, "rope") || as_extent(a[14], zero, &rope_rows) || as_extent(a[14], one, &rot) || as_int(a[14], s_stride, zero, &w) ||
        as_int(a[14], s_stride, one, &step) || is_on(a[14], dev, "rope"))
      return NULL;
    if (step != 1 || (w != rot && rope_rows > 1)) { PyErr_SetString(PyExc_ValueError, "rope: a dense float32 table"); return NULL; }
  }
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = ((append_fn)fn)(c, tk, tv, tq, k, ldk, v, ldv, q, ldq, q_out, ldqo, (int32_t)(width / d), tokens, slots, positions, rope,
                       rope_rows, (int32_t)rot, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* attention(function, cache, device, head_dim, q, out, kv_lens, page_table, max_q, max_kv, workspace, q_starts, scale, causal, lse,
 * stream) -> status */
static PyObject *attention(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  if (n != 16) { PyErr_SetString(PyExc_TypeError, "attention: 16 arguments"); return NULL; }
  void *fn, *c, *q, *out, *lens, *table, *ws, *starts, *lse, *stream;
  int64_t ldq, width, tokens, ldo, seqs, table_rows, ld_pages, step, rows, w, bytes = 0, size;
  int32_t max_q, max_kv, causal, d, dev;
  if (as_pointer(a[0], &fn) || as_pointer(a[1], &c) || as_int32(a[2], &dev) || as_int32(a[3], &d) || as_rows(a[4], dev, 0, 0, "q", &q, &tokens, &width, &ldq) ||
      as_rows(a[5], dev, tokens, width, "out", &out, &rows, &w, &ldo) || as_extent(a[6], zero, &seqs) ||
      as_vector(a[6], dev, int32_type, seqs, "kv_lens", &lens) || is_type(a[7], int32_type, "page_table") || is_on(a[7], dev, "page_table") || as_pointer(a[7], &table) ||
      as_extent(a[7], zero, &table_rows) || as_extent(a[7], one, &ld_pages) || as_int(a[7], s_stride, zero, &w) ||
      as_int(a[7], s_stride, one, &step) || as_int32(a[8], &max_q) || as_int32(a[9], &max_kv) || as_pointer(a[10], &ws) ||
      as_vector(a[11], dev, int32_type, seqs + 1, "q_starts", &starts) || as_int32(a[13], &causal) || as_pointer(a[14], &lse) ||
      as_pointer(a[15], &stream))
    return NULL;
  if (table_rows < seqs || (step != 1 && ld_pages > 1) || (w != ld_pages && table_rows > 1)) {
    PyErr_SetString(PyExc_ValueError, "page_table: dense int32, a row per sequence");
    return NULL;
  }
  if (width % d != 0) { PyErr_SetString(PyExc_ValueError, "q: whole heads"); return NULL; }
  if (a[14] != Py_None) {
    PyObject *dense = PyObject_CallMethodNoArgs(a[14], s_is_contiguous);
    if (dense == NULL) return NULL;
    const int yes = PyObject_IsTrue(dense);
    Py_DECREF(dense);
    if (yes < 0 || is_type(a[14], float32_type, "lse") || is_on(a[14], dev, "lse") || as_int(a[14], s_numel, NULL, &size)) return NULL;
    if (!yes || size < tokens * (width / d)) { PyErr_SetString(PyExc_ValueError, "lse: dense float32, [tokens, q_heads]"); return NULL; }
  }
  if (a[10] != Py_None && (as_int(a[10], s_numel, NULL, &bytes) || is_on(a[10], dev, "workspace"))) return NULL;
  const double scale = PyFloat_AsDouble(a[12]);
  if (scale == -1.0 && PyErr_Occurred()) return NULL;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = ((attention_fn)fn)(c, q, ldq, (int32_t)(width / d), tokens, starts, lens, table, ld_pages, (int32_t)seqs, max_q, max_kv,
                          (float)scale, causal, out, ldo, lse, ws, (size_t)bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* setup(torch.float32, torch.Tensor, torch.bfloat16, torch.int32, torch.int64) */
static PyObject *setup(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  if (n != 5 || !PyType_Check(a[1])) { PyErr_SetString(PyExc_TypeError, "setup: a dtype, a type and three dtypes"); return NULL; }
  Py_XSETREF(float32_type, Py_NewRef(a[0]));
  Py_XSETREF(tensor_type, (PyTypeObject *)Py_NewRef(a[1]));
  Py_XSETREF(bfloat16_type, Py_NewRef(a[2]));
  Py_XSETREF(int32_type, Py_NewRef(a[3]));
  Py_XSETREF(int64_type, Py_NewRef(a[4]));
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, NULL},
                                {"quantise", (PyCFunction)(void (*)(void))quantise, METH_FASTCALL, NULL},
                                {"kv_append", (PyCFunction)(void (*)(void))kv_append, METH_FASTCALL, NULL},
                                {"attention", (PyCFunction)(void (*)(void))attention, METH_FASTCALL, NULL},
                                {"setup", (PyCFunction)(void (*)(void))setup, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pycall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__pycall(void) {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_size = PyUnicode_InternFromString("size");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_numel = PyUnicode_InternFromString("numel");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_get_device = PyUnicode_InternFromString("get_device");
  zero = PyLong_FromLong(0);
  one = PyLong_FromLong(1);
  if (!s_data_ptr || !s_size || !s_shape || !s_stride || !s_numel || !s_is_contiguous || !s_dtype || !s_get_device || !zero || !one) return NULL;
  return PyModule_Create(&module);
}
