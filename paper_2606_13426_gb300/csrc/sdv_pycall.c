/* sdv_pycall.c - the calls a serving loop makes, without ctypes: converting 25 arguments
 * takes ctypes 4-5 us, longer than the launch of a small call; here it takes under 1 us.
 * Integers (modulo their C type's range, as ctypes takes them), floats and None for NULL are
 * taken; any other object is a TypeError, upon which the binding calls through ctypes.  The GIL
 * is released around the call, and the entry points' addresses come from the binding, which
 * has loaded the library. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "specdiff.h"

typedef int (*verify_fn)(const void *, const void *, const void *, const float *, int64_t, int, int, int64_t, int,
                         uint64_t, int, const int32_t *, const void *, const float *, int, float, int32_t *, void *,
                         float *, float *, uint32_t *, float *, void *, size_t, sdv_stream_t);
typedef int (*ratios_fn)(const void *, const void *, const void *, const float *, int64_t, int, int, int64_t, int,
                         const int32_t *, float *, float *, void *, size_t, sdv_stream_t);

/* An argument; errors are left for PyErr_Occurred. */
static unsigned long long u64(PyObject *o) {
  if (PyLong_Check(o)) return PyLong_AsUnsignedLongLongMask(o);
  PyErr_SetString(PyExc_TypeError, "an integer is required");
  return 0;
}
static void *ptr(PyObject *o) { return o == Py_None ? NULL : (void *)(uintptr_t)u64(o); }
static float f32(PyObject *o) {
  if (PyFloat_Check(o) || PyLong_Check(o)) return (float)PyFloat_AsDouble(o);
  PyErr_SetString(PyExc_TypeError, "a number is required");
  return 0;
}

static PyObject *wrong_count(const char *name, int want, Py_ssize_t got) {
  PyErr_Format(PyExc_TypeError, "%s takes %d arguments (%zd given)", name, want, got);
  return NULL;
}

/* verify(address, the 25 arguments of sdv_verify_ex): its return code. */
static PyObject *verify(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  if (n != 26) return wrong_count("verify", 26, n);
  const verify_fn fn = (verify_fn)ptr(a[0]);
  ++a;
  const void *x = ptr(a[0]), *mq = ptr(a[1]), *mp = ptr(a[2]);
  const float *sigma = ptr(a[3]);
  const int64_t stride = (int64_t)u64(a[4]), d = (int64_t)u64(a[7]);
  const int B = (int)u64(a[5]), L = (int)u64(a[6]), dtype = (int)u64(a[8]), mode = (int)u64(a[10]);
  const uint64_t seed = u64(a[9]);
  const int32_t *L_eff = ptr(a[11]);
  const void *mqb = ptr(a[12]);
  const float *sgb = ptr(a[13]);
  const int residual = (int)u64(a[14]);
  const float omega = f32(a[15]);
  int32_t *acc = ptr(a[16]);
  void *y = ptr(a[17]);
  float *lr = ptr(a[18]), *dn = ptr(a[19]);
  uint32_t *st = ptr(a[20]);
  float *aux = ptr(a[21]);
  void *ws = ptr(a[22]);
  const size_t bytes = (size_t)u64(a[23]);
  const sdv_stream_t stream = ptr(a[24]);
  int rc;
  if (PyErr_Occurred()) return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(x, mq, mp, sigma, stride, B, L, d, dtype, seed, mode, L_eff, mqb, sgb, residual, omega, acc, y, lr, dn, st,
          aux, ws, bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* ratios(address, the 15 arguments of sdv_log_ratios): its return code. */
static PyObject *ratios(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  if (n != 16) return wrong_count("ratios", 16, n);
  const ratios_fn fn = (ratios_fn)ptr(a[0]);
  ++a;
  const void *x = ptr(a[0]), *mq = ptr(a[1]), *mp = ptr(a[2]);
  const float *sigma = ptr(a[3]);
  const int64_t stride = (int64_t)u64(a[4]), d = (int64_t)u64(a[7]);
  const int B = (int)u64(a[5]), L = (int)u64(a[6]), dtype = (int)u64(a[8]);
  const int32_t *L_eff = ptr(a[9]);
  float *lr = ptr(a[10]), *dn = ptr(a[11]);
  void *ws = ptr(a[12]);
  const size_t bytes = (size_t)u64(a[13]);
  const sdv_stream_t stream = ptr(a[14]);
  int rc;
  if (PyErr_Occurred()) return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(x, mq, mp, sigma, stride, B, L, d, dtype, L_eff, lr, dn, ws, bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* The token operators: each takes the address and its entry point's arguments, in their order. */
typedef int (*scores_fn)(const void *, int64_t, int, int, int, const int32_t *, float, int, float *, float *, float *,
                         float *, int32_t *, float *, uint32_t *, sdv_stream_t);
static PyObject *scores(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  if (n != 17) return wrong_count("scores", 17, n);
  const scores_fn fn = (scores_fn)ptr(a[0]);
  ++a;
  const void *x = ptr(a[0]);
  const int64_t stride = (int64_t)u64(a[1]);
  const int N = (int)u64(a[2]), V = (int)u64(a[3]), dtype = (int)u64(a[4]), top_k = (int)u64(a[7]);
  const int32_t *tokens = ptr(a[5]);
  const float temperature = f32(a[6]);
  float *lp = ptr(a[8]), *h = ptr(a[9]), *m = ptr(a[10]), *ls = ptr(a[11]), *tlp = ptr(a[13]);
  int32_t *ids = ptr(a[12]);
  uint32_t *st = ptr(a[14]);
  const sdv_stream_t stream = ptr(a[15]);
  int rc;
  if (PyErr_Occurred()) return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(x, stride, N, V, dtype, tokens, temperature, top_k, lp, h, m, ls, ids, tlp, st, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

typedef int (*train_fn)(const void *, int64_t, int, int, int, const int32_t *, float, const float *, const float *, float *,
                        float *, float *, float *, uint32_t *, void *, int64_t, sdv_stream_t);
static PyObject *train(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  if (n != 18) return wrong_count("train", 18, n);
  const train_fn fn = (train_fn)ptr(a[0]);
  ++a;
  const void *x = ptr(a[0]);
  const int64_t stride = (int64_t)u64(a[1]), d_stride = (int64_t)u64(a[15]);
  const int N = (int)u64(a[2]), V = (int)u64(a[3]), dtype = (int)u64(a[4]);
  const int32_t *tokens = ptr(a[5]);
  const float temperature = f32(a[6]);
  const float *gl = ptr(a[7]), *gh = ptr(a[8]);
  float *lp = ptr(a[9]), *h = ptr(a[10]), *m = ptr(a[11]), *ls = ptr(a[12]);
  uint32_t *st = ptr(a[13]);
  void *dx = ptr(a[14]);
  const sdv_stream_t stream = ptr(a[16]);
  int rc;
  if (PyErr_Occurred()) return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(x, stride, N, V, dtype, tokens, temperature, gl, gh, lp, h, m, ls, st, dx, d_stride, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

typedef int (*token_verify_fn)(const void *, int64_t, int64_t, const void *, int64_t, int64_t, const int32_t *, int, int, int,
                               int, float, float, int, const int32_t *, uint64_t, const float *, const float *, int32_t *,
                               int32_t *, float *, uint32_t *, void *, size_t, sdv_stream_t);
static PyObject *token_verify(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  if (n != 26) return wrong_count("token_verify", 26, n);
  const token_verify_fn fn = (token_verify_fn)ptr(a[0]);
  ++a;
  const void *q = ptr(a[0]), *p = ptr(a[3]);
  const int64_t qb = (int64_t)u64(a[1]), qr = (int64_t)u64(a[2]), pb = (int64_t)u64(a[4]), pr = (int64_t)u64(a[5]);
  const int32_t *tokens = ptr(a[6]), *L_eff = ptr(a[14]);
  const int B = (int)u64(a[7]), L = (int)u64(a[8]), V = (int)u64(a[9]), dtype = (int)u64(a[10]), mode = (int)u64(a[13]);
  const float t = f32(a[11]), td = f32(a[12]);
  const uint64_t seed = u64(a[15]);
  const float *coins = ptr(a[16]), *race = ptr(a[17]);
  int32_t *acc = ptr(a[18]), *next = ptr(a[19]);
  float *lr = ptr(a[20]);
  uint32_t *st = ptr(a[21]);
  void *ws = ptr(a[22]);
  const size_t bytes = (size_t)u64(a[23]);
  const sdv_stream_t stream = ptr(a[24]);
  int rc;
  if (PyErr_Occurred()) return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(q, qb, qr, p, pb, pr, tokens, B, L, V, dtype, t, td, mode, L_eff, seed, coins, race, acc, next, lr, st, ws, bytes,
          stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

typedef int (*append_fn)(const void *, const void *, int64_t, int64_t, int64_t, int, int, int, int, int, int, void *, void *,
                         float *, float *, int64_t, const int32_t *, int, const int32_t *, const int32_t *, uint32_t *,
                         sdv_stream_t);
static PyObject *append(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  if (n != 23) return wrong_count("append", 23, n);
  const append_fn fn = (append_fn)ptr(a[0]);
  ++a;
  const void *k = ptr(a[0]), *v = ptr(a[1]);
  const int64_t sb = (int64_t)u64(a[2]), st = (int64_t)u64(a[3]), sh = (int64_t)u64(a[4]), pages = (int64_t)u64(a[15]);
  const int dtype = (int)u64(a[5]), B = (int)u64(a[6]), W = (int)u64(a[7]), H = (int)u64(a[8]), D = (int)u64(a[9]),
            block = (int)u64(a[10]), max_pages = (int)u64(a[17]);
  void *kc = ptr(a[11]), *vc = ptr(a[12]);
  float *ks = ptr(a[13]), *vs = ptr(a[14]);
  const int32_t *table = ptr(a[16]), *lengths = ptr(a[18]), *counts = ptr(a[19]);
  uint32_t *status = ptr(a[20]);
  const sdv_stream_t stream = ptr(a[21]);
  int rc;
  if (PyErr_Occurred()) return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(k, v, sb, st, sh, dtype, B, W, H, D, block, kc, vc, ks, vs, pages, table, max_pages, lengths, counts, status, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

typedef int (*attend_fn)(const void *, int64_t, int64_t, int64_t, int, int, int, int, int, int, int, const void *, const void *,
                         const float *, const float *, int64_t, const int32_t *, int, const int32_t *, const int32_t *, float,
                         int, void *, float *, uint32_t *, void *, size_t, sdv_stream_t);
static PyObject *attend(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  if (n != 29) return wrong_count("attend", 29, n);
  const attend_fn fn = (attend_fn)ptr(a[0]);
  ++a;
  const void *q = ptr(a[0]), *kc = ptr(a[11]), *vc = ptr(a[12]);
  const int64_t sb = (int64_t)u64(a[1]), st = (int64_t)u64(a[2]), sh = (int64_t)u64(a[3]), pages = (int64_t)u64(a[15]);
  const int dtype = (int)u64(a[4]), B = (int)u64(a[5]), W = (int)u64(a[6]), Hq = (int)u64(a[7]), H = (int)u64(a[8]),
            D = (int)u64(a[9]), block = (int)u64(a[10]), max_pages = (int)u64(a[17]), span = (int)u64(a[21]);
  const float *ks = ptr(a[13]), *vs = ptr(a[14]);
  const int32_t *table = ptr(a[16]), *lengths = ptr(a[18]), *counts = ptr(a[19]);
  const float scale = f32(a[20]);
  void *out = ptr(a[22]), *ws = ptr(a[25]);
  float *lse = ptr(a[23]);
  uint32_t *status = ptr(a[24]);
  const size_t bytes = (size_t)u64(a[26]);
  const sdv_stream_t stream = ptr(a[27]);
  int rc;
  if (PyErr_Occurred()) return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(q, sb, st, sh, dtype, B, W, Hq, H, D, block, kc, vc, ks, vs, pages, table, max_pages, lengths, counts, scale, span, out,
          lse, status, ws, bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

static PyMethodDef methods[] = {
    {"verify", (PyCFunction)(void (*)(void))verify, METH_FASTCALL, "verify(address, *arguments of sdv_verify_ex)"},
    {"ratios", (PyCFunction)(void (*)(void))ratios, METH_FASTCALL, "ratios(address, *arguments of sdv_log_ratios)"},
    {"scores", (PyCFunction)(void (*)(void))scores, METH_FASTCALL, "scores(address, *arguments of sdv_token_scores)"},
    {"train", (PyCFunction)(void (*)(void))train, METH_FASTCALL, "train(address, *arguments of sdv_token_scores_train)"},
    {"token_verify", (PyCFunction)(void (*)(void))token_verify, METH_FASTCALL,
     "token_verify(address, *arguments of sdv_token_verify)"},
    {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, "append(address, *arguments of sdv_cache_append)"},
    {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, "attend(address, *arguments of sdv_cache_attend)"},
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sdvcall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__sdvcall(void) { return PyModule_Create(&module); }
