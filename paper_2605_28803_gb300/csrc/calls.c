/* The calls of a served step as Python functions: the same names and arguments as in include/qvla.h, tensors by their data_ptr(),
 * streams by their cuda_stream, the GIL released around the library.  Argument marshalling only, like the rest of the binding;
 * what takes ctypes 1.2 to 1.6 us a call takes 0.3 here, of the 3 us that such a call costs with its launch. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <limits.h>
#include <stdint.h>

#include "../../include/qvla.h"

static PyObject *s_data_ptr, *s_cuda_stream, *s_handle, *s_address, *s_dt, *s_width, *s_tokens; /* interned names */
static PyObject *g_check, *g_layer, *g_norm; /* callable(status): raises; the types Fp4Layer and BlockNorm */

/* Positional and keyword arguments into slots; the last `optional` of n may be left out (None). */
static int take(const char* call, const char* const* names, int n, int optional, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames,
                PyObject** slots) {
  Py_ssize_t i, k;
  if (!g_check) {
    PyErr_Format(PyExc_RuntimeError, "%s(): not set up (import the package's qvla)", call);
    return -1;
  }
  if (nargs > n) {
    PyErr_Format(PyExc_TypeError, "%s() takes %d arguments but %zd were given", call, n, nargs);
    return -1;
  }
  for (i = 0; i < n; ++i) slots[i] = i < nargs ? args[i] : NULL;
  for (k = 0; kwnames && k < PyTuple_GET_SIZE(kwnames); ++k) {
    PyObject* const key = PyTuple_GET_ITEM(kwnames, k);
    for (i = 0; i < n; ++i)
      if (PyUnicode_CompareWithASCIIString(key, names[i]) == 0) break;
    if (i == n || slots[i]) {
      PyErr_Format(PyExc_TypeError, i == n ? "%s() has no argument '%U'" : "%s() got two values for argument '%U'", call, key);
      return -1;
    }
    slots[i] = args[nargs + k];
  }
  for (i = 0; i < n; ++i) {
    if (slots[i]) continue;
    if (i < n - optional) {
      PyErr_Format(PyExc_TypeError, "%s() needs the argument '%s'", call, names[i]);
      return -1;
    }
    slots[i] = Py_None;
  }
  return 0;
}

/* Each returns 0, or -1 with an exception set. */
static int get_pointer(PyObject* o, PyObject* attribute, int call, void** out) {
  PyObject* v;
  *out = NULL;
  if (o == Py_None) return 0;
  v = call ? PyObject_CallMethodNoArgs(o, attribute) : PyObject_GetAttr(o, attribute);
  if (!v) return -1;
  if (v != Py_None) *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return *out == NULL && PyErr_Occurred() ? -1 : 0;
}
static int get_tensor(PyObject* o, void** out) { return get_pointer(o, s_data_ptr, 1, out); }
static int get_stream(PyObject* o, void** out) {
  if (PyLong_CheckExact(o)) {
    *out = PyLong_AsVoidPtr(o);
    return *out == NULL && PyErr_Occurred() ? -1 : 0;
  }
  return get_pointer(o, s_cuda_stream, 0, out);
}
static int get_int(PyObject* o, int* out) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) return -1;
  if (v < INT_MIN || v > INT_MAX) {
    PyErr_SetString(PyExc_OverflowError, "an argument does not fit a C int");
    return -1;
  }
  *out = (int)v;
  return 0;
}
static int get_int64(PyObject* o, int64_t* out) {
  *out = PyLong_AsLongLong(o);
  return *out == -1 && PyErr_Occurred() ? -1 : 0;
}
static int get_size(PyObject* o, size_t* out) {
  *out = PyLong_AsSize_t(o);
  return *out == (size_t)-1 && PyErr_Occurred() ? -1 : 0;
}

/* A layer's handle (a handle of another kind would be read as one). */
static int get_layer(PyObject* o, void** out) {
  if (!PyObject_TypeCheck(o, (PyTypeObject*)g_layer)) {
    PyErr_Format(PyExc_TypeError, "an Fp4Layer is needed, not %s", Py_TYPE(o)->tp_name);
    return -1;
  }
  return get_pointer(o, s_handle, 0, out);
}
static int get_attribute_int(PyObject* o, PyObject* name, int* out) {
  PyObject* const v = PyObject_GetAttr(o, name);
  int bad;
  if (!v) return -1;
  bad = get_int(v, out);
  Py_DECREF(v);
  return bad;
}
/* A norm's parameters and type, and whether its vectors and index reach over the call's M rows of K. */
static int get_norm(PyObject* o, PyObject* rows, PyObject* channels, void** out, int* dt, int* M, int* K) {
  int width, tokens;
  if (!PyObject_TypeCheck(o, (PyTypeObject*)g_norm)) {
    PyErr_Format(PyExc_TypeError, "a BlockNorm is needed, not %s", Py_TYPE(o)->tp_name);
    return -1;
  }
  if (get_int(rows, M) || get_int(channels, K) || get_pointer(o, s_address, 0, out) || get_attribute_int(o, s_dt, dt) ||
      get_attribute_int(o, s_width, &width) || get_attribute_int(o, s_tokens, &tokens))
    return -1;
  if (*K > width || *M > tokens) {
    PyErr_Format(PyExc_ValueError, *K > width ? "the norm's vectors have %d channels, the call %d" : "mod_index has %d tokens, the call %d",
                 *K > width ? width : tokens, *K > width ? *K : *M);
    return -1;
  }
  return 0;
}

static PyObject* result(qvla_status s) {
  if (s == QVLA_OK) Py_RETURN_NONE;
  return PyObject_CallFunction(g_check, "i", (int)s);
}

#define TAKE(call, n, optional)                                                                     \
  PyObject* a[n];                                                                                   \
  qvla_status s;                                                                                    \
  if (take(call, names, n, optional, args, nargs, kwnames, a)) return NULL
#define CALL(expression)      \
  Py_BEGIN_ALLOW_THREADS;     \
  s = expression;             \
  Py_END_ALLOW_THREADS;       \
  return result(s)

static PyObject* quantize_rows(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"x", "xdt", "x_stride", "M", "K", "had_block", "fmt", "step_scale", "xq", "xs", "xscale", "stream"};
  void *x, *step, *xq, *xs, *xscale, *stream;
  int xdt, M, K, had, fmt;
  int64_t stride;
  TAKE("qvla_fp4_quantize_rows", 12, 2);
  if (get_tensor(a[0], &x) || get_int(a[1], &xdt) || get_int64(a[2], &stride) || get_int(a[3], &M) || get_int(a[4], &K) || get_int(a[5], &had) ||
      get_int(a[6], &fmt) || get_tensor(a[7], &step) || get_tensor(a[8], &xq) || get_tensor(a[9], &xs) || get_tensor(a[10], &xscale) ||
      get_stream(a[11], &stream))
    return NULL;
  CALL(qvla_fp4_quantize_rows(x, (qvla_dtype)xdt, stride, M, K, had, (qvla_fp4_format)fmt, step, xq, xs, xscale, stream));
}

static PyObject* dequantize_rows(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"xq", "xs", "xscale", "fmt", "M", "K", "out", "odt", "stream"};
  void *xq, *xs, *xscale, *out, *stream;
  int fmt, M, K, odt;
  TAKE("qvla_fp4_dequantize_rows", 9, 1);
  if (get_tensor(a[0], &xq) || get_tensor(a[1], &xs) || get_tensor(a[2], &xscale) || get_int(a[3], &fmt) || get_int(a[4], &M) || get_int(a[5], &K) ||
      get_tensor(a[6], &out) || get_int(a[7], &odt) || get_stream(a[8], &stream))
    return NULL;
  CALL(qvla_fp4_dequantize_rows(xq, xs, xscale, (qvla_fp4_format)fmt, M, K, out, (qvla_dtype)odt, stream));
}

static PyObject* gemm(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"layer", "xq", "xs", "xscale", "M", "y", "stream"};
  void *layer, *xq, *xs, *xscale, *y, *stream;
  int M;
  TAKE("qvla_gemm_fp4", 7, 1);
  if (get_layer(a[0], &layer) || get_tensor(a[1], &xq) || get_tensor(a[2], &xs) || get_tensor(a[3], &xscale) || get_int(a[4], &M) ||
      get_tensor(a[5], &y) || get_stream(a[6], &stream))
    return NULL;
  CALL(qvla_gemm_fp4(layer, xq, xs, xscale, M, y, stream));
}

static PyObject* linear(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"layer", "x", "M", "step_scale", "y", "workspace", "workspace_bytes", "stream"};
  void *layer, *x, *step, *y, *work, *stream;
  int M;
  size_t bytes;
  TAKE("qvla_fp4_linear", 8, 1);
  if (get_layer(a[0], &layer) || get_tensor(a[1], &x) || get_int(a[2], &M) || get_tensor(a[3], &step) || get_tensor(a[4], &y) ||
      get_tensor(a[5], &work) || get_size(a[6], &bytes) || get_stream(a[7], &stream))
    return NULL;
  CALL(qvla_fp4_linear(layer, x, M, step, y, work, bytes, stream));
}

static PyObject* block_norm(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"norm", "r", "rdt", "r_stride", "y", "y_stride", "M", "K", "r_out", "h", "stream"};
  void *norm, *r, *y, *r_out, *h, *stream;
  int dt, rdt, M, K;
  int64_t r_stride, y_stride;
  TAKE("qvla_block_norm", 11, 1);
  if (get_norm(a[0], a[6], a[7], &norm, &dt, &M, &K) || get_tensor(a[1], &r) || get_int(a[2], &rdt) || get_int64(a[3], &r_stride) || get_tensor(a[4], &y) || get_int64(a[5], &y_stride) ||
      get_tensor(a[8], &r_out) || get_tensor(a[9], &h) || get_stream(a[10], &stream))
    return NULL;
  CALL(qvla_block_norm(norm, (qvla_dtype)dt, r, (qvla_dtype)rdt, r_stride, y, y_stride, M, K, r_out, h, stream));
}

static PyObject* block_norm_fp4(PyObject* self, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
  static const char* const names[] = {"norm", "r", "rdt", "r_stride", "y", "y_stride", "M", "K", "r_out", "h", "had_block", "fmt", "step_scale", "hq", "hs",
                                      "hscale", "stream"};
  void *norm, *r, *y, *r_out, *h, *step, *hq, *hs, *hscale, *stream;
  int dt, rdt, M, K, had, fmt;
  int64_t r_stride, y_stride;
  TAKE("qvla_block_norm_fp4", 17, 2);
  if (get_norm(a[0], a[6], a[7], &norm, &dt, &M, &K) || get_tensor(a[1], &r) || get_int(a[2], &rdt) || get_int64(a[3], &r_stride) || get_tensor(a[4], &y) || get_int64(a[5], &y_stride) ||
      get_tensor(a[8], &r_out) || get_tensor(a[9], &h) || get_int(a[10], &had) || get_int(a[11], &fmt) ||
      get_tensor(a[12], &step) || get_tensor(a[13], &hq) || get_tensor(a[14], &hs) || get_tensor(a[15], &hscale) || get_stream(a[16], &stream))
    return NULL;
  CALL(qvla_block_norm_fp4(norm, (qvla_dtype)dt, r, (qvla_dtype)rdt, r_stride, y, y_stride, M, K, r_out, h, had, (qvla_fp4_format)fmt, step, hq, hs, hscale,
                           stream));
}

static PyObject* setup(PyObject* self, PyObject* args) {
  PyObject *check, *layer, *norm;
  if (!PyArg_ParseTuple(args, "OO!O!", &check, &PyType_Type, &layer, &PyType_Type, &norm)) return NULL;
  Py_INCREF(check);
  Py_INCREF(layer);
  Py_INCREF(norm);
  Py_XSETREF(g_check, check);
  Py_XSETREF(g_layer, layer);
  Py_XSETREF(g_norm, norm);
  Py_RETURN_NONE;
}

#define METHOD(name, function, signature, text) \
  {name, (PyCFunction)(void (*)(void))function, METH_FASTCALL | METH_KEYWORDS, name signature "\n--\n\n" text}
static PyMethodDef methods[] = {
    METHOD("qvla_fp4_quantize_rows", quantize_rows, "(x, xdt, x_stride, M, K, had_block, fmt, step_scale, xq, xs, xscale=None, stream=None)",
           "Rotate and quantise rows to E2M1 codes and block scales (NVFP4: and a float32 scale a row)."),
    METHOD("qvla_fp4_dequantize_rows", dequantize_rows, "(xq, xs, xscale, fmt, M, K, out, odt, stream=None)",
           "What the codes stand for, in the rotated basis."),
    METHOD("qvla_gemm_fp4", gemm, "(layer, xq, xs, xscale, M, y, stream=None)", "The product of quantised rows and a layer."),
    METHOD("qvla_fp4_linear", linear, "(layer, x, M, step_scale, y, workspace, workspace_bytes, stream=None)",
           "The layer's rotation and quantiser on x, then the product."),
    METHOD("qvla_block_norm", block_norm, "(norm, r, rdt, r_stride, y, y_stride, M, K, r_out, h, stream=None)",
           "Residual + gated branch, then the norm; y, r_out or h may be None as in include/qvla.h."),
    METHOD("qvla_block_norm_fp4", block_norm_fp4,
           "(norm, r, rdt, r_stride, y, y_stride, M, K, r_out, h, had_block, fmt, step_scale, hq, hs, hscale=None, stream=None)",
           "The same with its output rotated and quantised."),
    {"setup", setup, METH_VARARGS, "The callable that turns a non-zero status into an exception, and the types of layers and norms; ahead of any call."},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "libqvla's calls of a served step.", -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void) {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  s_handle = PyUnicode_InternFromString("handle");
  s_address = PyUnicode_InternFromString("ref");
  s_dt = PyUnicode_InternFromString("dt");
  s_width = PyUnicode_InternFromString("width");
  s_tokens = PyUnicode_InternFromString("tokens");
  if (!s_data_ptr || !s_cuda_stream || !s_handle || !s_address || !s_dt || !s_width || !s_tokens) return NULL;
  return PyModule_Create(&module);
}
