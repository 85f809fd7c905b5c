/* The calls of the binding that serving makes most often, in C: what ctypes and the interpreter take for the checks and the
 * conversion of 28 arguments (8 of 10 us of a small rotation and append) is several times what the launch takes.  The
 * checks and their errors are those of the package's other calls; statuses are returned for Python to raise. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "sdsat.h"

static sdsat_status (*set_stream)(sdsat_ctx*, void*);
static __typeof__(&sdsat_op_rotary_append) rotary_append;
static __typeof__(&sdsat_op_chunk_attention) chunk_attention;
static __typeof__(&sdsat_op_adjust_logits) adjust_logits;
static PyObject *f32, *bf16, *i32, *current_stream;                                       /* torch's types; a callable */
static PyObject *s_dtype, *s_is_cuda, *s_shape, *s_stride, *s_data_ptr, *s_numel, *s_is_contiguous, *s_value;

static int wrong(const char* what) {
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, what);
  return 0;
}

/* 1: the attribute is `is`, 0: another or an error */
static int attr_is(PyObject* t, PyObject* name, PyObject* is) {
  PyObject* x = PyObject_GetAttr(t, name);
  Py_XDECREF(x);
  return x == is;
}
static int integer(PyObject* x, long long* out) {
  *out = PyLong_AsLongLong(x);
  return !(*out == -1 && PyErr_Occurred());
}
static int small(PyObject* x, int* out) {
  long long v;
  if (!integer(x, &v)) return 0;
  if (v < INT32_MIN || v > INT32_MAX) return wrong("a number outside 32 bits");
  *out = (int)v;
  return 1;
}
static int number(PyObject* t, PyObject* method, long long* out) {
  PyObject* x = PyObject_CallMethodNoArgs(t, method);
  const int ok = x && integer(x, out);
  Py_XDECREF(x);
  return ok;
}
static int address(PyObject* t, void** out) {
  PyObject* x = PyObject_CallMethodNoArgs(t, s_data_ptr);
  if (!x) return 0;
  *out = PyLong_AsVoidPtr(x);
  Py_DECREF(x);
  return !(*out == NULL && PyErr_Occurred());
}
/* a tuple of n integers (taken over) */
static int integers(PyObject* x, Py_ssize_t n, long long* out) {
  int ok = x && PyTuple_Check(x) && PyTuple_GET_SIZE(x) == n;
  for (Py_ssize_t i = 0; ok && i < n; ++i) ok = integer(PyTuple_GET_ITEM(x, i), out + i);
  Py_XDECREF(x);
  return ok;
}
static int handle(PyObject* h, void** out) {   /* a ctypes pointer, or None */
  *out = NULL;
  if (h == Py_None) return 1;
  PyObject* x = PyObject_GetAttr(h, s_value);
  if (!x) return 0;
  if (x != Py_None) *out = PyLong_AsVoidPtr(x);
  Py_DECREF(x);
  return !PyErr_Occurred();
}

typedef struct {
  void* at;
  long long ld, rows, cols;
  int type;
} Rows;
/* a CUDA matrix whose rows are contiguous */
static int get_rows(PyObject* t, Rows* r) {
  long long shape[2], stride[2];
  PyObject* dtype = PyObject_GetAttr(t, s_dtype);
  if (!dtype) return 0;
  r->type = dtype == f32 ? SDSAT_FP32 : dtype == bf16 ? SDSAT_BF16 : -1;
  Py_DECREF(dtype);
  if (r->type < 0 || !attr_is(t, s_is_cuda, Py_True) || !integers(PyObject_GetAttr(t, s_shape), 2, shape))
    return wrong("expected a float32 or bfloat16 CUDA matrix");
  if (!integers(PyObject_CallMethodNoArgs(t, s_stride), 2, stride)) return wrong("expected a float32 or bfloat16 CUDA matrix");
  r->rows = shape[0];
  r->cols = shape[1];
  if (stride[1] != 1 && r->cols > 1) return wrong("expected contiguous rows");
  r->ld = r->rows > 1 ? stride[0] : r->cols;
  return address(t, &r->at);
}
/* a contiguous CUDA tensor of n values or more of a type; NULL of None, an address as it is */
static int get_array(PyObject* t, PyObject* dtype, long long n, void** out) {
  *out = NULL;
  if (t == Py_None) return 1;
  if (PyLong_Check(t)) {
    *out = PyLong_AsVoidPtr(t);
    return !PyErr_Occurred();
  }
  long long has = 0;
  int ok = number(t, s_numel, &has) && has >= n && attr_is(t, s_dtype, dtype) && attr_is(t, s_is_cuda, Py_True);
  if (ok) {
    PyObject* x = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    ok = x == Py_True;
    Py_XDECREF(x);
  }
  if (ok) return address(t, out);
  if (!PyErr_Occurred()) {
    PyObject* has_type = PyObject_GetAttr(t, s_dtype);
    if (has_type) PyErr_Format(PyExc_ValueError, "expected %lld values of %S in a contiguous CUDA tensor, got %lld of %S", n, dtype, has, has_type);
    Py_XDECREF(has_type);
  }
  return 0;
}
static int get_shape(PyObject* t, Py_ssize_t n, long long* out, const char* what) {
  return integers(PyObject_GetAttr(t, s_shape), n, out) ? 1 : wrong(what);
}
/* the pools of pages [n][Hk][SDSAT_PAGE][hd] */
static int get_pages(PyObject* k, PyObject* v, int Hk, int hd, int* n, void** kp, void** vp) {
  long long a[4], b[4];
  if (!get_shape(k, 4, a, "expected pages of [Hk][64][hd]") || !get_shape(v, 4, b, "expected pages of [Hk][64][hd]")) return 0;
  if (a[0] != b[0] || a[0] > INT32_MAX || a[1] != Hk || b[1] != Hk || a[2] != SDSAT_PAGE || b[2] != SDSAT_PAGE || a[3] != hd || b[3] != hd)
    return wrong("expected pages of [Hk][64][hd]");
  *n = (int)a[0];
  return get_array(k, bf16, 0, kp) && get_array(v, bf16, 0, vp);
}
static int bind_stream(sdsat_ctx* c) {
  PyObject* s = PyObject_CallNoArgs(current_stream);
  if (!s) return 0;
  void* stream = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  if (PyErr_Occurred()) return 0;
  set_stream(c, stream);
  return 1;
}
static int ready(Py_ssize_t n, Py_ssize_t want) {
  if (!f32 || !set_stream) return wrong("the binding has not been set up");
  if (n != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return 0;
  }
  return 1;
}

/* ctx, rope, q, k, v, q_out, k_pages, v_pages, table, lens, starts, H, Hk, hd, positions, q_gain, k_gain, eps, refs */
static PyObject* py_rotary_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *ctx, *rope, *kp, *vp, *table, *lens, *starts, *positions, *q_gain, *k_gain, *refs;
  Rows q, k, v, o;
  int H, Hk, hd, pages;
  long long shape[2];
  (void)self;
  if (!ready(n, 19) || !handle(a[0], &ctx) || !handle(a[1], &rope) || !bind_stream(ctx)) return NULL;
  if (!get_rows(a[2], &q) || !get_rows(a[3], &k) || !get_rows(a[4], &v) || !get_rows(a[5], &o) || !small(a[11], &H) || !small(a[12], &Hk) ||
      !small(a[13], &hd))
    return NULL;
  const double eps = PyFloat_AsDouble(a[17]);
  if (eps == -1. && PyErr_Occurred()) return NULL;
  if (q.type != k.type || q.type != v.type || q.type != o.type) return wrong("q, k, v and q_out are of different types"), NULL;
  if (k.rows < q.rows || v.rows < q.rows || o.rows < q.rows) return wrong("k, v or q_out of fewer rows than q"), NULL;
  if (q.cols < (long long)H * hd || o.cols < (long long)H * hd || k.cols < (long long)Hk * hd || v.cols < (long long)Hk * hd)
    return wrong("fewer columns than heads * hd"), NULL;
  if (!get_shape(a[8], 2, shape, "expected a table of pages [b][columns]") || !get_pages(a[6], a[7], Hk, hd, &pages, &kp, &vp)) return NULL;
  if (q.rows > INT32_MAX || shape[0] >= INT32_MAX || shape[1] > INT32_MAX) return wrong("a size outside 32 bits"), NULL;
  if (!get_array(a[10], i32, shape[0] + 1, &starts) || !get_array(a[9], i32, shape[0], &lens) || !get_array(a[14], i32, q.rows, &positions) ||
      !get_array(a[15], bf16, hd, &q_gain) || !get_array(a[16], bf16, hd, &k_gain) || !get_array(a[8], i32, 0, &table) ||
      !get_array(a[18], i32, pages, &refs))
    return NULL;
  sdsat_status s;
  Py_BEGIN_ALLOW_THREADS
  s = rotary_append(ctx, rope, q.at, q.ld, k.at, k.ld, v.at, v.ld, q.type, (int)q.rows, starts, lens, (int)shape[0], positions, q_gain, k_gain,
                    (float)eps, H, Hk, hd, o.at, o.ld, kp, vp, pages, table, (int)shape[1], refs);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(s);
}

/* ctx, q, k_pages, v_pages, table, lens, starts, H, Hk, hd, out */
static PyObject* py_chunk_attention(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *ctx, *kp, *vp, *table, *lens, *starts;
  Rows q, o;
  int H, Hk, hd, pages;
  long long shape[2];
  (void)self;
  if (!ready(n, 11) || !handle(a[0], &ctx) || !bind_stream(ctx)) return NULL;
  if (!get_rows(a[1], &q) || !get_rows(a[10], &o) || !small(a[7], &H) || !small(a[8], &Hk) || !small(a[9], &hd)) return NULL;
  if (q.type != o.type) return wrong("q and out are of different types"), NULL;
  if (o.rows < q.rows) return wrong("out of fewer rows than q"), NULL;
  if (q.cols < (long long)H * hd || o.cols < (long long)H * hd) return wrong("fewer columns than H * hd"), NULL;
  if (!get_shape(a[4], 2, shape, "expected a table of pages [b][columns]") || !get_pages(a[2], a[3], Hk, hd, &pages, &kp, &vp)) return NULL;
  if (q.rows > INT32_MAX || shape[0] >= INT32_MAX || shape[1] > INT32_MAX) return wrong("a size outside 32 bits"), NULL;
  if (!get_array(a[4], i32, 0, &table) || !get_array(a[6], i32, shape[0] + 1, &starts) || !get_array(a[5], i32, shape[0], &lens)) return NULL;
  sdsat_status s;
  Py_BEGIN_ALLOW_THREADS
  s = chunk_attention(ctx, q.at, q.ld, (int)q.rows, kp, vp, pages, table, (int)shape[1], starts, lens, (int)shape[0], H, Hk, hd, o.at, o.ld, q.type);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(s);
}

/* the second size of a matrix, 0 of None */
static int width(PyObject* t, long long* out) {
  long long shape[2];
  *out = 0;
  if (t == Py_None) return 1;
  if (!get_shape(t, 2, shape, "expected a matrix")) return 0;
  *out = shape[1];
  return shape[1] <= INT32_MAX ? 1 : wrong("a size outside 32 bits");
}
/* ctx, logits, out, q, history, history_lens, prompt_lens, tokens, anc, repetition, frequency, presence, bias_ids, bias, allowed */
static PyObject* py_adjust_logits(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *ctx, *history, *history_lens, *prompt_lens, *tokens, *anc, *repetition, *frequency, *presence, *bias_ids, *bias, *allowed;
  Rows x, o;
  int q;
  long long nh, nb, nb2, words;
  (void)self;
  if (!ready(n, 15) || !handle(a[0], &ctx) || !bind_stream(ctx)) return NULL;
  if (!get_rows(a[1], &x) || !get_rows(a[2], &o) || !small(a[3], &q)) return NULL;
  if (x.type != o.type) return wrong("logits and out are of different types"), NULL;
  if (q < 1 || x.rows % q) return wrong("rows are no multiple of q"), NULL;
  if (o.rows < x.rows || o.cols < x.cols) return wrong("out is smaller than logits"), NULL;
  if (x.rows > INT32_MAX || x.cols > INT32_MAX) return wrong("a size outside 32 bits"), NULL;
  const long long b = x.rows / q;
  if (!width(a[4], &nh) || !width(a[12], &nb) || !width(a[13], &nb2) || !width(a[14], &words)) return NULL;
  if ((a[12] == Py_None) != (a[13] == Py_None) || nb != nb2) return wrong("bias_ids and bias are of different widths"), NULL;
  if (a[14] != Py_None && words < (x.cols + 31) / 32) return wrong("allowed is narrower than the vocabulary"), NULL;
  if (!get_array(a[4], i32, b * nh, &history) || !get_array(a[5], i32, b, &history_lens) || !get_array(a[6], i32, b, &prompt_lens) ||
      !get_array(a[7], i32, x.rows, &tokens) || !get_array(a[8], i32, x.rows, &anc) || !get_array(a[9], f32, b, &repetition) ||
      !get_array(a[10], f32, b, &frequency) || !get_array(a[11], f32, b, &presence) || !get_array(a[12], i32, b * nb, &bias_ids) ||
      !get_array(a[13], f32, b * nb, &bias) || !get_array(a[14], i32, x.rows * words, &allowed))
    return NULL;
  sdsat_status s;
  Py_BEGIN_ALLOW_THREADS
  s = adjust_logits(ctx, x.at, x.ld, x.type, (int)b, q, (int)x.cols, history, (int)nh, history_lens, prompt_lens, tokens, anc, repetition, frequency,
                    presence, bias_ids, bias, (int)nb, allowed, (int)words, o.at, o.ld);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(s);
}

/* the library's functions: sdsat_set_stream, sdsat_op_rotary_append, sdsat_op_chunk_attention, sdsat_op_adjust_logits */
static PyObject* py_library(PyObject* self, PyObject* args) {
  unsigned long long f[4];
  (void)self;
  if (!PyArg_ParseTuple(args, "KKKK", f, f + 1, f + 2, f + 3)) return NULL;
  set_stream = (void*)(uintptr_t)f[0];
  rotary_append = (void*)(uintptr_t)f[1];
  chunk_attention = (void*)(uintptr_t)f[2];
  adjust_logits = (void*)(uintptr_t)f[3];
  Py_RETURN_NONE;
}
/* float32, bfloat16, int32, and what returns the current stream as an integer */
static PyObject* py_types(PyObject* self, PyObject* args) {
  PyObject* t[4];
  (void)self;
  if (!PyArg_ParseTuple(args, "OOOO", t, t + 1, t + 2, t + 3)) return NULL;
  PyObject** to[4] = {&f32, &bf16, &i32, &current_stream};
  for (int i = 0; i < 4; ++i) {
    Py_INCREF(t[i]);
    Py_XSETREF(*to[i], t[i]);
  }
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"library", py_library, METH_VARARGS, NULL},
                                {"types", py_types, METH_VARARGS, NULL},
                                {"rotary_append", (PyCFunction)(void*)py_rotary_append, METH_FASTCALL, NULL},
                                {"chunk_attention", (PyCFunction)(void*)py_chunk_attention, METH_FASTCALL, NULL},
                                {"adjust_logits", (PyCFunction)(void*)py_adjust_logits, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__native(void) {
  PyObject** names[] = {&s_dtype, &s_is_cuda, &s_shape, &s_stride, &s_data_ptr, &s_numel, &s_is_contiguous, &s_value};
  const char* texts[] = {"dtype", "is_cuda", "shape", "stride", "data_ptr", "numel", "is_contiguous", "value"};
  for (int i = 0; i < 8; ++i)
    if (!(*names[i] = PyUnicode_InternFromString(texts[i]))) return NULL;
  return PyModule_Create(&module);
}
