/* The per-token calls of the Python binding without ctypes, whose conversion of nine arguments costs the host more than the
 * checks and the choice of a kernel behind them (a call that fails the first check: 0.42 us, 0.06 so, on one host, 1.25 and 0.12 on
 * another).  A decode call of a small layer is bound by the host: 128 x 205 fp32 4.8 -> 4.1 us, a prompt and 16 tokens of 256 x 1024
 * 137 -> 126. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "coreinfer.h"

static int pointer(PyObject* o, void** out) {
  *out = o == Py_None ? NULL : PyLong_AsVoidPtr(o);
  return *out != NULL || !PyErr_Occurred();
}

static int number(PyObject* o, long long* out) {
  *out = PyLong_AsLongLong(o);
  return *out != -1 || !PyErr_Occurred();
}

/* ffn_decode(x, B, weights, dtype, act, y, ws, ws_bytes, stream) -> status; addresses are integers or None */
static PyObject* ffn_decode(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *x, *w, *y, *ws, *stream;
  long long B, dtype, act, bytes;
  int status;
  (void)self;
  if (n != 9) {
    PyErr_SetString(PyExc_TypeError, "nine arguments");
    return NULL;
  }
  if (!pointer(a[0], &x) || !number(a[1], &B) || !pointer(a[2], &w) || !number(a[3], &dtype) || !number(a[4], &act) ||
      !pointer(a[5], &y) || !pointer(a[6], &ws) || !number(a[7], &bytes) || !pointer(a[8], &stream))
    return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = coreinfer_ffn_decode(x, B, (const ci_ffn_weights*)w, (int)dtype, (int)act, y, ws, (size_t)bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

/* The 4-bit operators' calls: their C arguments in order, three element strides one by one.  kinds, a letter an argument: p an address (an
 * integer, or None for NULL), i an integer, f a float, which is left out of v. */
static int values(const char* name, PyObject* const* a, Py_ssize_t n, const char* kinds, long long* v) {
  Py_ssize_t i;
  if (n != (Py_ssize_t)strlen(kinds)) {
    PyErr_Format(PyExc_TypeError, "%s: %zd arguments", name, (Py_ssize_t)strlen(kinds));
    return 0;
  }
  for (i = 0; i < n; ++i) {
    v[i] = 0;
    if (kinds[i] == 'f' || (kinds[i] == 'p' && a[i] == Py_None)) continue;
    if (!number(a[i], &v[i])) return 0;
  }
  return 1;
}
#define P(i) ((void*)(intptr_t)v[i])
#define I(i) ((int)v[i])

/* x, M, ldx, x_dtype, w, gate, bias, bias_dtype, act, R, C, group, y, ldy, y_dtype, ws, ws_bytes, stream */
static PyObject* w4_matvec(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  long long v[18];
  int status;
  (void)self;
  if (!values("w4_matvec", a, n, "piiipppiiiiipiipip", v)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = coreinfer_w4_matvec(P(0), v[1], v[2], I(3), P(4), P(5), P(6), I(7), I(8), v[9], v[10], I(11), P(12), v[13], I(14), P(15),
                               (size_t)v[16], P(17));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

/* cache, k, v, S, strides b, s, h, dtype, start, lens, next, stream */
static PyObject* kv4_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  long long v[12];
  int64_t stride[3];
  int status;
  (void)self;
  if (!values("kv4_append", a, n, "pppiiiiipppp", v)) return NULL;
  stride[0] = v[4];
  stride[1] = v[5];
  stride[2] = v[6];
  Py_BEGIN_ALLOW_THREADS
  status = coreinfer_kv4_append((const ci_kv4*)P(0), P(1), P(2), v[3], stride, I(7), (const int32_t*)P(8), (const int32_t*)P(9),
                                (const int32_t*)P(10), P(11));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

/* cache, lens, first, count, k, v, dtype, stream */
static PyObject* kv4_read(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  long long v[8];
  int status;
  (void)self;
  if (!values("kv4_read", a, n, "ppiippip", v)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = coreinfer_kv4_read((const ci_kv4*)P(0), (const int32_t*)P(1), v[2], v[3], P(4), P(5), I(6), P(7));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

/* cache, q, S, Hq, strides b, s, h, dtype, scale (a float), lens, max_len, out, lse, weight_out, ws, ws_bytes, stream */
static PyObject* kv4_attend(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  long long v[17];
  int64_t stride[3];
  double scale;
  int status;
  (void)self;
  if (!values("kv4_attend", a, n, "ppiiiiiifpippppip", v)) return NULL;
  scale = PyFloat_AsDouble(a[8]);
  if (scale == -1.0 && PyErr_Occurred()) return NULL;
  stride[0] = v[4];
  stride[1] = v[5];
  stride[2] = v[6];
  Py_BEGIN_ALLOW_THREADS
  status = coreinfer_kv4_attend((const ci_kv4*)P(0), P(1), v[2], v[3], stride, I(7), (float)scale, (const int32_t*)P(9), v[10], P(11),
                                (float*)P(12), (float*)P(13), P(14), (size_t)v[15], P(16));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

/* cache, lens, next, max_len, budget, recent, weight_out, pos_out, lens_out, ws, ws_bytes, stream */
static PyObject* kv4_evict(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  long long v[12];
  int status;
  (void)self;
  if (!values("kv4_evict", a, n, "pppiiippppip", v)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = coreinfer_kv4_evict((const ci_kv4*)P(0), (const int32_t*)P(1), (const int32_t*)P(2), v[3], v[4], v[5], (float*)P(6),
                               (int32_t*)P(7), (int32_t*)P(8), P(9), (size_t)v[10], P(11));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

#define CALL(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {CALL(ffn_decode), CALL(w4_matvec), CALL(kv4_append), CALL(kv4_read), CALL(kv4_attend), CALL(kv4_evict),
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
