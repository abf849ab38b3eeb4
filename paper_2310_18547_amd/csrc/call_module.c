// CPython module with the calls a decode loop makes once per layer and projection.
//
// What bounds it: a decode add-on runs 4-6 us on the GPU, and one call through ctypes cost the
// host 5.3 us, of which 3.4 us are the kernel launch itself -- the loop was bound by its host
// side.  ctypes spends 1.1 us on converting the arguments and Python code another 0.7 us on
// taking the tensors' addresses; here both are done in C from the interpreter's argument vector
// (vectorcall, nothing is packed into tuples or dicts).
//
// Only the usual forms are converted here: addresses as ints, None or objects with data_ptr(), numbers
// as Python converts them, lists or tuples of pointers.  A call with anything else in it (ctypes objects,
// numpy arrays, pointer lists of different lengths, wrong arguments) goes, arguments untouched, to the
// Python function of the same name in binding.py, whose answer or exception it gets.
//
// The module calls the library that binding.py has loaded: it is handed the entry points'
// addresses, so that a tuning build of the library works the same way.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/sgmv.h"

typedef int (*shrink_fn)(const sgmv_problem*, float*, const void*, const void* const*, const int32_t*, int32_t, int32_t,
                         void*);
typedef int (*expand_fn)(const sgmv_problem*, void*, const float*, const void* const*, const int32_t*, int32_t, int32_t,
                         float, void*);
typedef int (*add_lora_fn)(const sgmv_problem*, void*, const void*, const void* const*, const void* const*,
                           const int32_t*, int32_t, int32_t, float, void*);
typedef int (*add_lora_multi_fn)(const sgmv_problem*, int32_t, void* const*, const void* const*,
                                 const void* const* const*, const void* const* const*, const int32_t*, int32_t,
                                 int32_t, float, void*);
typedef int (*rms_norm_fn)(int32_t, void*, int8_t*, float*, void*, const void*, const void*, const void*, float, int32_t,
                           int32_t, void*);
typedef int (*silu_mul_fn)(int32_t, void*, int8_t*, float*, const void*, const void*, int32_t, int32_t, void*);
typedef int (*quantize_fn)(int32_t, int8_t*, float*, const void*, int32_t, int32_t, void*);
typedef int (*dense_fn)(int32_t, int32_t, void* const*, const int8_t*, const float*, const int8_t* const*, const float* const*,
                        int32_t, int32_t, const int32_t*, void*, size_t, void*);

typedef int (*kv_assign_fn)(const sgmv_kv_cache*, const sgmv_kv_batch*, const int32_t*, const int32_t*, int32_t*, const int32_t*, int32_t*,
                            int32_t*, void*);
typedef int (*kv_append_fn)(const sgmv_kv_cache*, const sgmv_kv_batch*, int32_t, void*, const void*, const void*, const void*, int32_t, int64_t,
                            int64_t, int64_t, const sgmv_rope*, void*);
typedef int (*kv_read_fn)(const sgmv_kv_cache*, int32_t, void*, void*, int64_t, const int32_t*, int32_t, void*);
typedef int (*attention_fn)(const sgmv_kv_cache*, const sgmv_kv_batch*, int32_t, void*, float*, const void*, int32_t, int64_t, int64_t, float,
                            int32_t, int32_t, void*, size_t, void*);

static shrink_fn fn_shrink;
static expand_fn fn_expand;
static add_lora_fn fn_add_lora;
static add_lora_fn fn_add_lora_static;
static add_lora_multi_fn fn_add_lora_multi;
static rms_norm_fn fn_rms_norm;
static silu_mul_fn fn_silu_mul;
static quantize_fn fn_quantize;
static dense_fn fn_dense;
static kv_assign_fn fn_kv_assign;
static kv_append_fn fn_kv_append;
static kv_read_fn fn_kv_read;
static attention_fn fn_attention;
enum { PROBLEM, KV_CACHE, KV_BATCH, ROPE, STRUCTS };
static PyObject* struct_types[STRUCTS];  // binding.SgmvProblem, SgmvKvCache, SgmvKvBatch, SgmvRope
static PyObject* error_type;    // binding.SgmvError
enum { SHRINK, EXPAND, ADD_LORA, ADD_LORA_STATIC, ADD_LORA_MULTI, RMS_NORM, SILU_MUL, QUANTIZE, DENSE,
       KV_ASSIGN, KV_APPEND, KV_READ, ATTENTION, CALLS };
static PyObject* general[CALLS];  // the functions in Python, in the order of bind()'s addresses
static PyObject *str_data_ptr, *str_cuda_stream;

// What the conversions below return besides an error (-1, an exception is set): the value is there, or
// the argument is not of a usual form.
enum { DONE = 0, UNUSUAL = 1 };

// After a failed conversion: the general function decides what becomes of the argument.
static int unusual(void) {
  if (!PyErr_ExceptionMatches(PyExc_Exception)) return -1;  // an interrupt stays one
  PyErr_Clear();
  return UNUSUAL;
}

// The address behind a pointer argument: None, an int, or an object with data_ptr() (a tensor).
static int address_of(PyObject* o, void** out) {
  if (o == Py_None) {
    *out = NULL;
    return DONE;
  }
  PyObject* value;
  if (PyLong_Check(o)) {
    value = o;
    Py_INCREF(value);
  } else {
    value = PyObject_CallMethodNoArgs(o, str_data_ptr);
    if (value == NULL) return unusual();
  }
  int rc = UNUSUAL;
  if (PyLong_Check(value)) {
    const unsigned long long a = PyLong_AsUnsignedLongLongMask(value);
    rc = a == (unsigned long long)-1 && PyErr_Occurred() ? unusual() : DONE;
    *out = (void*)(uintptr_t)a;
  }
  Py_DECREF(value);
  return rc;
}

// None, an int, or an object with cuda_stream (a torch stream).
static int stream_of(PyObject* o, void** out) {
  if (o == NULL || o == Py_None || PyLong_Check(o)) return address_of(o == NULL ? Py_None : o, out);
  PyObject* s = PyObject_GetAttr(o, str_cuda_stream);
  if (s == NULL) return unusual();
  const int rc = s == Py_None || PyLong_Check(s) ? address_of(s, out) : UNUSUAL;
  Py_DECREF(s);
  return rc;
}

static int int32_of(PyObject* o, int32_t* out) {
  if (!PyIndex_Check(o)) return UNUSUAL;
  const unsigned long v = PyLong_AsUnsignedLongMask(o);  // wraps like a C cast
  if (v == (unsigned long)-1 && PyErr_Occurred()) return unusual();
  *out = (int32_t)v;
  return DONE;
}

static int float_of(PyObject* o, float* out) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) return unusual();
  *out = (float)v;
  return DONE;
}

// The caller's struct of that type; PyBuffer_Release when done.
static int struct_of(PyObject* o, int which, Py_buffer* view) {
  const int is = PyObject_IsInstance(o, struct_types[which]);
  if (is < 0) return -1;
  if (!is) return UNUSUAL;
  return PyObject_GetBuffer(o, view, PyBUF_SIMPLE);
}
static int problem_of(PyObject* o, Py_buffer* view) { return struct_of(o, PROBLEM, view); }

// Positional and keyword arguments into `got` by name; the first `required` must be there.
static int sort_arguments(const char* const* names, int n, int required, PyObject* const* args, Py_ssize_t nargs,
                          PyObject* kwnames, PyObject** got) {
  if (nargs > n) return UNUSUAL;
  for (int i = 0; i < n; ++i) got[i] = i < nargs ? args[i] : NULL;
  const Py_ssize_t nkw = kwnames == NULL ? 0 : PyTuple_GET_SIZE(kwnames);
  for (Py_ssize_t k = 0; k < nkw; ++k) {
    PyObject* key = PyTuple_GET_ITEM(kwnames, k);
    int i = 0;
    while (i < n && PyUnicode_CompareWithASCIIString(key, names[i]) != 0) ++i;
    if (i == n || got[i] != NULL) return UNUSUAL;
    got[i] = args[nargs + k];
  }
  for (int i = 0; i < required; ++i)
    if (got[i] == NULL) return UNUSUAL;
  return DONE;
}

// The first of several conversions that is not DONE.
#define FIRST(a) do { if (rc == DONE) rc = (a); } while (0)

// The call's status as a Python int, or SgmvError(status, where) when `check` is true (the default).
static PyObject* finish(int rc, PyObject* check, const char* where) {
  if (rc != 0) {
    const int raise = check == NULL ? 1 : PyObject_IsTrue(check);
    if (raise < 0) return NULL;
    if (raise) {
      PyObject* e = PyObject_CallFunction(error_type, "is", rc, where);
      if (e != NULL) {
        PyErr_SetObject(error_type, e);
        Py_DECREF(e);
      }
      return NULL;
    }
  }
  return PyLong_FromLong(rc);
}

static PyObject* call_shrink(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"p", "v", "x", "A_ptrs", "seg_starts", "n_segs", "layer_idx", "stream", "check"};
  PyObject* g[9];
  void *v, *x, *a, *seg, *stream;
  int32_t n_segs, layer;
  Py_buffer p;
  int rc = sort_arguments(names, 9, 7, args, nargs, kwnames, g);
  FIRST(address_of(g[1], &v));
  FIRST(address_of(g[2], &x));
  FIRST(address_of(g[3], &a));
  FIRST(address_of(g[4], &seg));
  FIRST(int32_of(g[5], &n_segs));
  FIRST(int32_of(g[6], &layer));
  FIRST(stream_of(g[7], &stream));
  FIRST(problem_of(g[0], &p));
  if (rc != DONE) return rc < 0 ? NULL : PyObject_Vectorcall(general[SHRINK], args, nargs, kwnames);
  Py_BEGIN_ALLOW_THREADS
  rc = fn_shrink((const sgmv_problem*)p.buf, (float*)v, x, (const void* const*)a, (const int32_t*)seg, n_segs, layer, stream);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&p);
  return finish(rc, g[8], "sgmv_shrink");
}

static PyObject* call_expand(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"p", "y", "v", "B_ptrs", "seg_starts", "n_segs", "layer_idx", "scale", "stream", "check"};
  PyObject* g[10];
  void *y, *v, *b, *seg, *stream;
  int32_t n_segs, layer;
  float scale;
  Py_buffer p;
  int rc = sort_arguments(names, 10, 8, args, nargs, kwnames, g);
  FIRST(address_of(g[1], &y));
  FIRST(address_of(g[2], &v));
  FIRST(address_of(g[3], &b));
  FIRST(address_of(g[4], &seg));
  FIRST(int32_of(g[5], &n_segs));
  FIRST(int32_of(g[6], &layer));
  FIRST(float_of(g[7], &scale));
  FIRST(stream_of(g[8], &stream));
  FIRST(problem_of(g[0], &p));
  if (rc != DONE) return rc < 0 ? NULL : PyObject_Vectorcall(general[EXPAND], args, nargs, kwnames);
  Py_BEGIN_ALLOW_THREADS
  rc = fn_expand((const sgmv_problem*)p.buf, y, (const float*)v, (const void* const*)b, (const int32_t*)seg, n_segs, layer,
                 scale, stream);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&p);
  return finish(rc, g[9], "sgmv_expand");
}

static PyObject* add_lora(add_lora_fn fn, int which, const char* where, PyObject* const* args, Py_ssize_t nargs,
                          PyObject* kwnames) {
  static const char* const names[] = {"p",      "y",         "x",     "A_ptrs", "B_ptrs", "seg_starts",
                                      "n_segs", "layer_idx", "scale", "stream", "check"};
  PyObject* g[11];
  void *y, *x, *a, *b, *seg, *stream;
  int32_t n_segs, layer;
  float scale;
  Py_buffer p;
  int rc = sort_arguments(names, 11, 9, args, nargs, kwnames, g);
  FIRST(address_of(g[1], &y));
  FIRST(address_of(g[2], &x));
  FIRST(address_of(g[3], &a));
  FIRST(address_of(g[4], &b));
  FIRST(address_of(g[5], &seg));
  FIRST(int32_of(g[6], &n_segs));
  FIRST(int32_of(g[7], &layer));
  FIRST(float_of(g[8], &scale));
  FIRST(stream_of(g[9], &stream));
  FIRST(problem_of(g[0], &p));
  if (rc != DONE) return rc < 0 ? NULL : PyObject_Vectorcall(general[which], args, nargs, kwnames);
  Py_BEGIN_ALLOW_THREADS
  rc = fn((const sgmv_problem*)p.buf, y, x, (const void* const*)a, (const void* const*)b, (const int32_t*)seg, n_segs,
          layer, scale, stream);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&p);
  return finish(rc, g[10], where);
}

static PyObject* call_add_lora(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  return add_lora(fn_add_lora, ADD_LORA, "sgmv_add_lora", args, nargs, kwnames);
}

static PyObject* call_add_lora_static(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  return add_lora(fn_add_lora_static, ADD_LORA_STATIC, "sgmv_add_lora_static", args, nargs, kwnames);
}

// The addresses of a list's or tuple's `n` elements.
// An element's data_ptr() is Python code and may change the very list that is read: the size is looked up
// again and the element kept alive around each one, and what is no longer there counts as NULL.
#define MOST_ADD_ONS 8  // that the library takes; more are left for it to refuse
static int addresses_of(PyObject* seq, Py_ssize_t n, void** out) {
  if (!(PyList_Check(seq) || PyTuple_Check(seq)) || PySequence_Fast_GET_SIZE(seq) != n) return UNUSUAL;
  for (Py_ssize_t i = 0; i < n; ++i) {
    out[i] = NULL;
    if (i >= PySequence_Fast_GET_SIZE(seq)) continue;
    PyObject* element = PySequence_Fast_GET_ITEM(seq, i);
    Py_INCREF(element);
    const int rc = address_of(element, &out[i]);
    Py_DECREF(element);
    if (rc != DONE) return rc;
  }
  return DONE;
}

static PyObject* call_add_lora_multi(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"p",      "ys",        "xs",    "A_ptrs", "B_ptrs", "seg_starts",
                                      "n_segs", "layer_idx", "scale", "stream", "check"};
  PyObject* g[11];
  void *ys[MOST_ADD_ONS], *xs[MOST_ADD_ONS], *as[MOST_ADD_ONS], *bs[MOST_ADD_ONS], *seg, *stream;
  Py_ssize_t n = 0;
  int32_t n_segs, layer;
  float scale;
  Py_buffer p;
  int rc = sort_arguments(names, 11, 9, args, nargs, kwnames, g);
  if (rc == DONE) {
    n = PyList_Check(g[1]) || PyTuple_Check(g[1]) ? PySequence_Fast_GET_SIZE(g[1]) : MOST_ADD_ONS + 1;
    if (n > MOST_ADD_ONS) rc = UNUSUAL;
  }
  FIRST(addresses_of(g[1], n, ys));
  FIRST(addresses_of(g[2], n, xs));
  FIRST(addresses_of(g[3], n, as));
  FIRST(addresses_of(g[4], n, bs));
  FIRST(address_of(g[5], &seg));
  FIRST(int32_of(g[6], &n_segs));
  FIRST(int32_of(g[7], &layer));
  FIRST(float_of(g[8], &scale));
  FIRST(stream_of(g[9], &stream));
  FIRST(problem_of(g[0], &p));
  if (rc != DONE) return rc < 0 ? NULL : PyObject_Vectorcall(general[ADD_LORA_MULTI], args, nargs, kwnames);
  Py_BEGIN_ALLOW_THREADS
  rc = fn_add_lora_multi((const sgmv_problem*)p.buf, (int32_t)n, ys, (const void* const*)xs, (const void* const* const*)as,
                         (const void* const* const*)bs, (const int32_t*)seg, n_segs, layer, scale, stream);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&p);
  return finish(rc, g[10], "sgmv_add_lora_multi");
}

static PyObject* call_rms_norm(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"dtype", "out",    "q",   "q_scales", "sum", "x",      "residual",
                                      "weight", "eps", "n_tokens", "h",   "stream", "check"};
  PyObject* g[13];
  void* a[7];  // out .. weight
  void* stream;
  int32_t dtype, n_tokens, h;
  float eps;
  int rc = sort_arguments(names, 13, 11, args, nargs, kwnames, g);
  FIRST(int32_of(g[0], &dtype));
  for (int i = 0; i < 7; ++i) FIRST(address_of(g[1 + i], &a[i]));
  FIRST(float_of(g[8], &eps));
  FIRST(int32_of(g[9], &n_tokens));
  FIRST(int32_of(g[10], &h));
  FIRST(stream_of(g[11], &stream));
  if (rc != DONE) return rc < 0 ? NULL : PyObject_Vectorcall(general[RMS_NORM], args, nargs, kwnames);
  Py_BEGIN_ALLOW_THREADS
  rc = fn_rms_norm(dtype, a[0], (int8_t*)a[1], (float*)a[2], a[3], a[4], a[5], a[6], eps, n_tokens, h, stream);
  Py_END_ALLOW_THREADS
  return finish(rc, g[12], "sgmv_rms_norm_q8");
}

static PyObject* call_silu_mul(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"dtype", "out", "q", "q_scales", "gate", "up", "n_tokens", "h", "stream", "check"};
  PyObject* g[10];
  void* a[5];  // out .. up
  void* stream;
  int32_t dtype, n_tokens, h;
  int rc = sort_arguments(names, 10, 8, args, nargs, kwnames, g);
  FIRST(int32_of(g[0], &dtype));
  for (int i = 0; i < 5; ++i) FIRST(address_of(g[1 + i], &a[i]));
  FIRST(int32_of(g[6], &n_tokens));
  FIRST(int32_of(g[7], &h));
  FIRST(stream_of(g[8], &stream));
  if (rc != DONE) return rc < 0 ? NULL : PyObject_Vectorcall(general[SILU_MUL], args, nargs, kwnames);
  Py_BEGIN_ALLOW_THREADS
  rc = fn_silu_mul(dtype, a[0], (int8_t*)a[1], (float*)a[2], a[3], a[4], n_tokens, h, stream);
  Py_END_ALLOW_THREADS
  return finish(rc, g[9], "sgmv_silu_mul_q8");
}

static PyObject* call_quantize(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"dtype", "q", "q_scales", "x", "n_tokens", "h", "stream", "check"};
  PyObject* g[8];
  void* a[3];  // q .. x
  void* stream;
  int32_t dtype, n_tokens, h;
  int rc = sort_arguments(names, 8, 6, args, nargs, kwnames, g);
  FIRST(int32_of(g[0], &dtype));
  for (int i = 0; i < 3; ++i) FIRST(address_of(g[1 + i], &a[i]));
  FIRST(int32_of(g[4], &n_tokens));
  FIRST(int32_of(g[5], &h));
  FIRST(stream_of(g[6], &stream));
  if (rc != DONE) return rc < 0 ? NULL : PyObject_Vectorcall(general[QUANTIZE], args, nargs, kwnames);
  Py_BEGIN_ALLOW_THREADS
  rc = fn_quantize(dtype, (int8_t*)a[0], (float*)a[1], a[2], n_tokens, h, stream);
  Py_END_ALLOW_THREADS
  return finish(rc, g[7], "sgmv_quantize_q8");
}

// A list's or tuple's `n` whole numbers (an element's __index__ is Python code too).
static int widths_of(PyObject* seq, Py_ssize_t n, int32_t* out) {
  if (!(PyList_Check(seq) || PyTuple_Check(seq)) || PySequence_Fast_GET_SIZE(seq) != n) return UNUSUAL;
  for (Py_ssize_t i = 0; i < n; ++i) {
    out[i] = 0;
    if (i >= PySequence_Fast_GET_SIZE(seq)) continue;
    PyObject* element = PySequence_Fast_GET_ITEM(seq, i);
    Py_INCREF(element);
    const int rc = int32_of(element, &out[i]);
    Py_DECREF(element);
    if (rc != DONE) return rc;
  }
  return DONE;
}

static int size_of(PyObject* o, size_t* out) {
  if (o == NULL) {
    *out = 0;
    return DONE;
  }
  if (!PyLong_Check(o)) return UNUSUAL;
  *out = PyLong_AsSize_t(o);
  return *out == (size_t)-1 && PyErr_Occurred() ? unusual() : DONE;
}

static PyObject* call_dense(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"dtype",    "ys",   "q",      "q_scales",  "ws",              "w_scales",
                                      "n_tokens", "h_in", "h_outs", "workspace", "workspace_bytes", "stream", "check"};
  PyObject* g[13];
  void *ys[MOST_ADD_ONS], *ws[MOST_ADD_ONS], *scales[MOST_ADD_ONS], *q, *q_scales, *workspace, *stream;
  int32_t dtype, n_tokens, h_in, h_outs[MOST_ADD_ONS];
  size_t bytes;
  Py_ssize_t n = 0;
  int rc = sort_arguments(names, 13, 9, args, nargs, kwnames, g);
  if (rc == DONE) {
    n = PyList_Check(g[1]) || PyTuple_Check(g[1]) ? PySequence_Fast_GET_SIZE(g[1]) : MOST_ADD_ONS + 1;
    if (n > MOST_ADD_ONS) rc = UNUSUAL;
  }
  FIRST(int32_of(g[0], &dtype));
  FIRST(addresses_of(g[1], n, ys));
  FIRST(address_of(g[2], &q));
  FIRST(address_of(g[3], &q_scales));
  FIRST(addresses_of(g[4], n, ws));
  FIRST(addresses_of(g[5], n, scales));
  FIRST(int32_of(g[6], &n_tokens));
  FIRST(int32_of(g[7], &h_in));
  FIRST(widths_of(g[8], n, h_outs));
  FIRST(address_of(g[9] == NULL ? Py_None : g[9], &workspace));
  FIRST(size_of(g[10], &bytes));
  FIRST(stream_of(g[11], &stream));
  if (rc != DONE) return rc < 0 ? NULL : PyObject_Vectorcall(general[DENSE], args, nargs, kwnames);
  Py_BEGIN_ALLOW_THREADS
  rc = fn_dense(dtype, (int32_t)n, ys, (const int8_t*)q, (const float*)q_scales, (const int8_t* const*)ws,
                (const float* const*)scales, n_tokens, h_in, h_outs, workspace, bytes, stream);
  Py_END_ALLOW_THREADS
  return finish(rc, g[12], "sgmv_dense_q8");
}

static int int64_of(PyObject* o, int64_t* out) {
  if (!PyLong_Check(o)) return UNUSUAL;
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) return unusual();
  *out = v;
  return DONE;
}

// Up to three structs of a call at once: all of them, or none is held.  An absent last one (None or left out) has no address.
typedef struct {
  Py_buffer views[3];
  int n;
} Structs;
static int structs_of(Structs* s, PyObject* const* objects, const int* types, int n) {
  s->n = 0;
  for (int i = 0; i < n; ++i) {
    s->views[i].buf = NULL;
    s->views[i].obj = NULL;
    if (i == 2 && (objects[i] == NULL || objects[i] == Py_None)) continue;
    const int rc = struct_of(objects[i], types[i], &s->views[i]);
    if (rc != DONE) {
      while (s->n > 0) PyBuffer_Release(&s->views[--s->n]);
      return rc;
    }
    s->n = i + 1;
  }
  return DONE;
}
static void structs_done(Structs* s) {
  while (s->n > 0) PyBuffer_Release(&s->views[--s->n]);
}
static const int kv_types[] = {KV_CACHE, KV_BATCH, ROPE};

static PyObject* call_kv_assign(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"cache", "batch", "new_lens", "old_lens", "free_pages", "free_count", "free_count_out", "status",
                                      "stream", "check"};
  PyObject* g[10];
  void *a[6], *stream;  // new_lens .. status
  Structs s;
  int rc = sort_arguments(names, 10, 8, args, nargs, kwnames, g);
  for (int i = 0; i < 6; ++i) FIRST(address_of(g[2 + i], &a[i]));
  FIRST(stream_of(g[8], &stream));
  FIRST(structs_of(&s, g, kv_types, 2));
  if (rc != DONE) return rc < 0 ? NULL : PyObject_Vectorcall(general[KV_ASSIGN], args, nargs, kwnames);
  Py_BEGIN_ALLOW_THREADS
  rc = fn_kv_assign(s.views[0].buf, s.views[1].buf, a[0], a[1], a[2], a[3], a[4], a[5], stream);
  Py_END_ALLOW_THREADS
  structs_done(&s);
  return finish(rc, g[9], "sgmv_kv_assign");
}

static PyObject* call_kv_append(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"cache", "batch", "layer_idx", "q_out", "q", "k", "v", "n_heads", "q_out_stride", "q_stride",
                                      "kv_stride", "rope", "stream", "check"};
  PyObject* g[14];
  void *a[4], *stream;  // q_out .. v
  int32_t layer, n_heads;
  int64_t strides[3];
  Structs s;
  int rc = sort_arguments(names, 14, 11, args, nargs, kwnames, g);
  FIRST(int32_of(g[2], &layer));
  for (int i = 0; i < 4; ++i) FIRST(address_of(g[3 + i], &a[i]));
  FIRST(int32_of(g[7], &n_heads));
  for (int i = 0; i < 3; ++i) FIRST(int64_of(g[8 + i], &strides[i]));
  FIRST(stream_of(g[12], &stream));
  if (rc == DONE) {
    PyObject* const objects[] = {g[0], g[1], g[11]};
    rc = structs_of(&s, objects, kv_types, 3);
  }
  if (rc != DONE) return rc < 0 ? NULL : PyObject_Vectorcall(general[KV_APPEND], args, nargs, kwnames);
  Py_BEGIN_ALLOW_THREADS
  rc = fn_kv_append(s.views[0].buf, s.views[1].buf, layer, a[0], a[1], a[2], a[3], n_heads, strides[0], strides[1], strides[2],
                    s.views[2].buf, stream);
  Py_END_ALLOW_THREADS
  structs_done(&s);
  return finish(rc, g[13], "sgmv_kv_append_q4");
}

static PyObject* call_kv_read(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"cache", "layer_idx", "k", "v", "kv_stride", "slots", "n_rows", "stream", "check"};
  PyObject* g[9];
  void *k, *v, *slots, *stream;
  int32_t layer, n_rows;
  int64_t stride;
  Structs s;
  int rc = sort_arguments(names, 9, 7, args, nargs, kwnames, g);
  FIRST(int32_of(g[1], &layer));
  FIRST(address_of(g[2], &k));
  FIRST(address_of(g[3], &v));
  FIRST(int64_of(g[4], &stride));
  FIRST(address_of(g[5], &slots));
  FIRST(int32_of(g[6], &n_rows));
  FIRST(stream_of(g[7], &stream));
  FIRST(structs_of(&s, g, kv_types, 1));
  if (rc != DONE) return rc < 0 ? NULL : PyObject_Vectorcall(general[KV_READ], args, nargs, kwnames);
  Py_BEGIN_ALLOW_THREADS
  rc = fn_kv_read(s.views[0].buf, layer, k, v, stride, slots, n_rows, stream);
  Py_END_ALLOW_THREADS
  structs_done(&s);
  return finish(rc, g[8], "sgmv_kv_read_q4");
}

static PyObject* call_attention(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"cache", "batch", "layer_idx", "out", "lse", "q", "n_heads", "out_stride", "q_stride", "scale",
                                      "causal", "window", "workspace", "workspace_bytes", "stream", "check"};
  PyObject* g[16];
  void *out, *lse, *q, *workspace, *stream;
  int32_t layer, n_heads, causal = 1, window = 0;
  int64_t strides[2];
  float scale;
  size_t bytes;
  Structs s;
  int rc = sort_arguments(names, 16, 10, args, nargs, kwnames, g);
  FIRST(int32_of(g[2], &layer));
  FIRST(address_of(g[3], &out));
  FIRST(address_of(g[4], &lse));
  FIRST(address_of(g[5], &q));
  FIRST(int32_of(g[6], &n_heads));
  for (int i = 0; i < 2; ++i) FIRST(int64_of(g[7 + i], &strides[i]));
  FIRST(float_of(g[9], &scale));
  if (rc == DONE && g[10] != NULL) rc = int32_of(g[10], &causal);
  if (rc == DONE && g[11] != NULL) rc = int32_of(g[11], &window);
  FIRST(address_of(g[12] == NULL ? Py_None : g[12], &workspace));
  FIRST(size_of(g[13], &bytes));
  FIRST(stream_of(g[14], &stream));
  FIRST(structs_of(&s, g, kv_types, 2));
  if (rc != DONE) return rc < 0 ? NULL : PyObject_Vectorcall(general[ATTENTION], args, nargs, kwnames);
  Py_BEGIN_ALLOW_THREADS
  rc = fn_attention(s.views[0].buf, s.views[1].buf, layer, out, lse, q, n_heads, strides[0], strides[1], scale, causal, window, workspace,
                    bytes, stream);
  Py_END_ALLOW_THREADS
  structs_done(&s);
  return finish(rc, g[15], "sgmv_attention_q4");
}

// bind(struct types, error type, then of the calls, in the order of the enumeration above, the
// addresses and the functions in Python)
static PyObject* call_bind(PyObject* self, PyObject* args) {
  PyObject *structs, *error, *addresses, *functions;
  if (!PyArg_ParseTuple(args, "O!OO!O!", &PyTuple_Type, &structs, &error, &PyTuple_Type, &addresses, &PyTuple_Type, &functions)) return NULL;
  if (PyTuple_GET_SIZE(structs) != STRUCTS || PyTuple_GET_SIZE(addresses) != CALLS || PyTuple_GET_SIZE(functions) != CALLS) {
    PyErr_SetString(PyExc_ValueError, "a type for every struct, an address and a function for every call");
    return NULL;
  }
  unsigned long long f[CALLS];
  for (int i = 0; i < CALLS; ++i) {
    f[i] = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(addresses, i));
    if (f[i] == (unsigned long long)-1 && PyErr_Occurred()) return NULL;
  }
  for (int i = 0; i < STRUCTS; ++i) {
    PyObject* type = PyTuple_GET_ITEM(structs, i);
    Py_INCREF(type);
    Py_XSETREF(struct_types[i], type);
  }
  Py_INCREF(error);
  Py_XSETREF(error_type, error);
  for (int i = 0; i < CALLS; ++i) {
    PyObject* function = PyTuple_GET_ITEM(functions, i);
    Py_INCREF(function);
    Py_XSETREF(general[i], function);
  }
  fn_shrink = (shrink_fn)(uintptr_t)f[SHRINK];
  fn_expand = (expand_fn)(uintptr_t)f[EXPAND];
  fn_add_lora = (add_lora_fn)(uintptr_t)f[ADD_LORA];
  fn_add_lora_static = (add_lora_fn)(uintptr_t)f[ADD_LORA_STATIC];
  fn_add_lora_multi = (add_lora_multi_fn)(uintptr_t)f[ADD_LORA_MULTI];
  fn_rms_norm = (rms_norm_fn)(uintptr_t)f[RMS_NORM];
  fn_silu_mul = (silu_mul_fn)(uintptr_t)f[SILU_MUL];
  fn_quantize = (quantize_fn)(uintptr_t)f[QUANTIZE];
  fn_dense = (dense_fn)(uintptr_t)f[DENSE];
  fn_kv_assign = (kv_assign_fn)(uintptr_t)f[KV_ASSIGN];
  fn_kv_append = (kv_append_fn)(uintptr_t)f[KV_APPEND];
  fn_kv_read = (kv_read_fn)(uintptr_t)f[KV_READ];
  fn_attention = (attention_fn)(uintptr_t)f[ATTENTION];
  return Py_BuildValue("nnnn", (Py_ssize_t)sizeof(sgmv_problem), (Py_ssize_t)sizeof(sgmv_kv_cache), (Py_ssize_t)sizeof(sgmv_kv_batch),
                       (Py_ssize_t)sizeof(sgmv_rope));
}

#define FAST(name, fn, doc) {name, (PyCFunction)(void (*)(void))fn, METH_FASTCALL | METH_KEYWORDS, doc}
static PyMethodDef methods[] = {
    FAST("sgmv_shrink", call_shrink,
         "sgmv_shrink(p, v, x, A_ptrs, seg_starts, n_segs, layer_idx, stream=None, check=True)\n--\n\n"),
    FAST("sgmv_expand", call_expand,
         "sgmv_expand(p, y, v, B_ptrs, seg_starts, n_segs, layer_idx, scale, stream=None, check=True)\n--\n\n"),
    FAST("sgmv_add_lora", call_add_lora,
         "sgmv_add_lora(p, y, x, A_ptrs, B_ptrs, seg_starts, n_segs, layer_idx, scale, stream=None, check=True)\n--\n\n"),
    FAST("sgmv_add_lora_static", call_add_lora_static,
         "sgmv_add_lora_static(p, y, x, A_ptrs, B_ptrs, seg_starts, n_segs, layer_idx, scale, stream=None, check=True)\n--\n\n"),
    FAST("sgmv_add_lora_multi", call_add_lora_multi,
         "sgmv_add_lora_multi(p, ys, xs, A_ptrs, B_ptrs, seg_starts, n_segs, layer_idx, scale, stream=None, check=True)\n"
         "--\n\nys, xs, A_ptrs, B_ptrs are sequences of equal length (one entry per add-on)."),
    FAST("sgmv_rms_norm_q8", call_rms_norm,
         "sgmv_rms_norm_q8(dtype, out, q, q_scales, sum, x, residual, weight, eps, n_tokens, h, stream=None, check=True)\n--\n\n"),
    FAST("sgmv_silu_mul_q8", call_silu_mul,
         "sgmv_silu_mul_q8(dtype, out, q, q_scales, gate, up, n_tokens, h, stream=None, check=True)\n--\n\n"),
    FAST("sgmv_quantize_q8", call_quantize,
         "sgmv_quantize_q8(dtype, q, q_scales, x, n_tokens, h, stream=None, check=True)\n--\n\n"),
    FAST("sgmv_dense_q8", call_dense,
         "sgmv_dense_q8(dtype, ys, q, q_scales, ws, w_scales, n_tokens, h_in, h_outs, workspace=None, workspace_bytes=0, "
         "stream=None, check=True)\n--\n\nys, ws, w_scales, h_outs are sequences of equal length (one entry per projection)."),
    FAST("sgmv_kv_assign", call_kv_assign,
         "sgmv_kv_assign(cache, batch, new_lens, old_lens, free_pages, free_count, free_count_out, status, stream=None, check=True)\n--\n\n"),
    FAST("sgmv_kv_append_q4", call_kv_append,
         "sgmv_kv_append_q4(cache, batch, layer_idx, q_out, q, k, v, n_heads, q_out_stride, q_stride, kv_stride, rope=None, stream=None, "
         "check=True)\n--\n\n"),
    FAST("sgmv_kv_read_q4", call_kv_read,
         "sgmv_kv_read_q4(cache, layer_idx, k, v, kv_stride, slots, n_rows, stream=None, check=True)\n--\n\n"),
    FAST("sgmv_attention_q4", call_attention,
         "sgmv_attention_q4(cache, batch, layer_idx, out, lse, q, n_heads, out_stride, q_stride, scale, causal=1, window=0, workspace=None, "
         "workspace_bytes=0, stream=None, check=True)\n--\n\n"),
    {"bind", call_bind, METH_VARARGS, "bind(struct_types, error_type, addresses, functions) -> sizes of the C structs"},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sgmv_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__sgmv_call(void) {
  str_data_ptr = PyUnicode_InternFromString("data_ptr");
  str_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  if (!str_data_ptr || !str_cuda_stream) return NULL;
  return PyModule_Create(&module);
}
