/* kia_host.c -- the calls of around.py that serving and training loops repeat, in C.
 *
 * A call for one token is as long as its host work: checks, allocation and marshalling
 * take 10 to 25 us in Python, this module a third of that. Each function makes the call
 * if every argument is what the kernels take as it is (types, shapes, one device that
 * is the current one, layouts), and returns None otherwise: the caller then goes on in
 * Python, which copies what needs copying and says what is wrong. Of the tensors only
 * attributes and methods are used; the current device and stream come from torch._C
 * (_cuda_getDevice, _cuda_getCurrentRawStream).
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "kia.h"

static PyObject *Tensor, *f32, *bf16, *i32, *f64, *empty_like, *empty, *get_device, *get_stream;
static PyObject *check, *contiguous, *u8;
static PyObject *s_shape, *s_stride, *s_dtype, *s_data_ptr, *s_get_device, *s_device;
static PyObject *kw_like, *kw_empty;

static int (*p_rotary)(const kia_view *, const kia_view *, const kia_view *, const kia_view *,
                       const int32_t *, int64_t, int, const double *, float, int, int, int, int, int,
                       int, int, int, int, void *);
static int (*p_window_fwd)(const kia_view *, const kia_view *, const kia_view *, const kia_view *,
                           float *, const int32_t *, int, int, int, int, int, int, int, int, void *);
static int (*p_window_ws)(int, int, int, int, int, int, int, size_t *);
static int (*p_window_bwd)(const kia_view *, const kia_view *, const kia_view *, const kia_view *,
                           const kia_view *, const float *, const int32_t *, void *, const kia_view *,
                           const kia_view *, const kia_view *, int, int, int, int, int, int, int, int,
                           void *);
static int (*p_write)(const kia_view *, const kia_view *, void *, int, int, const int32_t *, int,
                      const int32_t *, const int32_t *, int, int, int, int, int, void *);
static int (*p_read)(const void *, int, int, const int32_t *, int, const int32_t *, const int32_t *,
                     const kia_view *, const kia_view *, int, int, int, int, int, void *);
static int (*p_attn_ws)(int, int, int, int, int, int, int, int, int, size_t *);
static int (*p_attn)(const kia_view *, const kia_view *, const void *, int, int, const int32_t *, int,
                     const int32_t *, void *, int, int, int, int, int, int, int, float, int, int, int,
                     int, void *);
static int (*p_append)(const kia_view *, const kia_view *, const kia_view *, const kia_view *, void *, void *,
                       int, int, const int32_t *, int, const int32_t *, const int32_t *, const double *, float,
                       int, int, int, int, int, int, int, int, void *);
static int (*p_select_ws)(int, int, int, int, int, int, int, size_t *);
static int (*p_select)(const kia_view *, const void *, int, int, const int32_t *, int, const int32_t *, void *,
                       int32_t *, int, int, int, int, int, int, int, int, int, void *);
static int (*p_pages_ws)(int, int, int, int, int, int, int, int, size_t *);
static int (*p_attn_pages)(const kia_view *, const kia_view *, const void *, int, int, const int32_t *, int,
                           const int32_t *, const int32_t *, int, void *, int, int, int, int, int, int, int, float,
                           int, int, void *);
static int (*p_shared_ws)(int, int, int, int, int, int, int, int, size_t *);
static int (*p_attn_shared)(const kia_view *, const kia_view *, const void *, int, int, const int32_t *, int,
                            const int32_t *, int, void *, int, int, int, int, int, int, int, float, int, int, void *);

/* ---- reading a tensor: 1 as wanted, 0 not (no exception is left) ---------------- */
typedef struct {
  long n[4], s[4];
  int dims, dtype, device; /* dtype: KIA_F32, KIA_BF16, or -1 */
  uintptr_t ptr;
} tensor;

static int longs(PyObject *t, long *out, int most) { /* length, or -1 */
  if (!t || !PyTuple_Check(t)) return -1;
  const Py_ssize_t n = PyTuple_GET_SIZE(t);
  if (n > most) return -1;
  for (Py_ssize_t i = 0; i < n; ++i) {
    out[i] = PyLong_AsLong(PyTuple_GET_ITEM(t, i));
    if (out[i] == -1 && PyErr_Occurred()) return -1;
  }
  return (int)n;
}

static int method_long(PyObject *o, PyObject *name, long long *out) {
  PyObject *r = PyObject_CallMethodNoArgs(o, name);
  if (!r) return 0;
  *out = PyLong_Check(r) ? (long long)PyLong_AsUnsignedLongLongMask(r) : -2;
  Py_DECREF(r);
  return *out != -2;
}

static int read_tensor(PyObject *o, tensor *t) {
  long long v;
  int ok = 0;
  if ((PyObject *)Py_TYPE(o) != Tensor) return 0;
  PyObject *shape = PyObject_GetAttr(o, s_shape);
  PyObject *stride = PyObject_CallMethodNoArgs(o, s_stride);
  PyObject *dtype = PyObject_GetAttr(o, s_dtype);
  if (shape && stride && dtype) {
    t->dims = longs(shape, t->n, 4);
    ok = t->dims >= 0 && longs(stride, t->s, 4) == t->dims;
    t->dtype = dtype == f32 ? KIA_F32 : dtype == bf16 ? KIA_BF16 : -1;
  }
  Py_XDECREF(shape);
  Py_XDECREF(stride);
  Py_XDECREF(dtype);
  if (!ok || !method_long(o, s_get_device, &v) || v < 0) goto no;
  t->device = (int)v;
  if (!method_long(o, s_data_ptr, &v)) goto no;
  t->ptr = (uintptr_t)v;
  return 1;
no:
  PyErr_Clear();
  return 0;
}

/* A [B, H, T, d] tensor of the kernels' types in a layout that they take. */
static int fits(const tensor *t, kia_view *v) {
  if (t->dims != 4 || t->dtype < 0 || t->ptr == 0 || t->ptr % 16 || t->s[3] != 1) return 0;
  const long unit = t->dtype == KIA_F32 ? 4 : 8;
  for (int i = 0; i < 4; ++i)
    if (t->n[i] < 1 || t->n[i] > INT32_MAX) return 0;
  if (t->n[2] > 1 && (t->s[2] < t->n[3] || t->s[2] % unit || t->s[2] > 1 << 22)) return 0;
  if ((t->n[1] > 1 && t->s[1] % unit) || (t->n[0] > 1 && t->s[0] % unit)) return 0;
  v->data = (void *)t->ptr;
  v->sb = t->s[0], v->sh = t->s[1], v->st = t->s[2];
  return 1;
}
static int view_of(PyObject *o, tensor *t, kia_view *v) { return read_tensor(o, t) && fits(t, v); }
/* the same, of q's type, device, batch, tokens and channels */
static int view_like(PyObject *o, const tensor *q, long heads, kia_view *v) {
  tensor t;
  return view_of(o, &t, v) && t.dtype == q->dtype && t.device == q->device && t.n[0] == q->n[0] &&
         t.n[1] == heads && t.n[2] == q->n[2] && t.n[3] == q->n[3];
}

/* A contiguous int32 tensor of up to two dimensions (None: NULL, if `none`). */
static int ints_of(PyObject *o, const tensor *q, int dims, const long *n, int none,
                   const int32_t **out) {
  *out = NULL;
  if (o == Py_None) return none;
  tensor t;
  if (!read_tensor(o, &t) || t.dims != dims || t.device != q->device) return 0;
  long step = 1;
  for (int i = dims - 1; i >= 0; --i) {
    if (t.n[i] != n[i] || (t.n[i] > 1 && t.s[i] != step)) return 0;
    step *= t.n[i];
  }
  PyObject *dtype = PyObject_GetAttr(o, s_dtype);
  const int ok = dtype == i32;
  Py_XDECREF(dtype);
  PyErr_Clear();
  *out = (const int32_t *)t.ptr;
  return ok && t.ptr != 0;
}

static int an_int(PyObject *o, long low, int *out) {
  if (!PyLong_CheckExact(o)) return 0;
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    return 0;
  }
  *out = (int)v;
  return v >= low && v <= INT32_MAX;
}

/* The stream to launch on: the device is the current one. */
static int stream_of(const tensor *q, void **out) {
  PyObject *r = PyObject_CallNoArgs(get_device);
  long dev = r ? PyLong_AsLong(r) : -1;
  Py_XDECREF(r);
  if (dev != q->device) {
    PyErr_Clear();
    return 0;
  }
  PyObject *d = PyLong_FromLong(dev);
  r = d ? PyObject_CallOneArg(get_stream, d) : NULL;
  Py_XDECREF(d);
  if (!r) {
    PyErr_Clear();
    return 0;
  }
  *out = (void *)(uintptr_t)PyLong_AsUnsignedLongLongMask(r);
  Py_DECREF(r);
  return 1;
}

/* A new contiguous tensor of ref's shape and its view (NULL: an exception). */
static PyObject *new_like(PyObject *ref, const tensor *t, kia_view *v) {
  PyObject *args[2] = {ref, contiguous};
  PyObject *o = PyObject_Vectorcall(empty_like, args, 1, kw_like);
  long long ptr;
  if (!o) return NULL;
  if (!method_long(o, s_data_ptr, &ptr)) {
    Py_DECREF(o);
    return NULL;
  }
  v->data = (void *)(uintptr_t)ptr;
  v->st = t->n[3], v->sh = t->n[2] * t->n[3], v->sb = t->n[1] * v->sh;
  return o;
}
/* torch.empty(*n, dtype=, device=ref.device), of up to four dimensions */
static PyObject *new_of(PyObject *ref, const long *n, int dims, PyObject *dtype, uintptr_t *ptr) {
  PyObject *args[6] = {NULL}, *o = NULL;
  long long v;
  int i, ok = 1;
  for (i = 0; i < dims; ++i) ok = (args[i] = PyLong_FromLong(n[i])) != NULL && ok;
  PyObject *dev = PyObject_GetAttr(ref, s_device);
  if (ok && dev) {
    args[dims] = dtype;
    args[dims + 1] = dev;
    o = PyObject_Vectorcall(empty, args, dims, kw_empty);
  }
  for (i = 0; i < dims; ++i) Py_XDECREF(args[i]);
  Py_XDECREF(dev);
  if (o && !method_long(o, s_data_ptr, &v)) Py_CLEAR(o);
  if (o) *ptr = (uintptr_t)v;
  return o;
}

/* What a call returns: `out`, or the exception of a failed call. */
static PyObject *done(int rc, PyObject *out) {
  if (rc == KIA_OK || !out) return out;
  Py_DECREF(out);
  PyObject *r = PyObject_CallFunction(check, "i", rc);
  Py_XDECREF(r);
  if (r) PyErr_SetString(PyExc_RuntimeError, "libkia failed");
  return NULL;
}
#define NONE Py_RETURN_NONE
#define CALL(...)                          \
  do {                                     \
    Py_BEGIN_ALLOW_THREADS rc = __VA_ARGS__; \
    Py_END_ALLOW_THREADS                   \
  } while (0)

/* rotary(q, k or None, freq, positions or None, layout, factor, back) */
static PyObject *rotary(PyObject *self, PyObject *const *a, Py_ssize_t na) {
  tensor q, k, f;
  kia_view vq, vk, vy, vz;
  const int32_t *pos = NULL;
  void *stream;
  int rc = 0, layout, back, first = 0;
  int64_t sb = 0;
  if (na != 7 || !view_of(a[0], &q, &vq)) NONE;
  const int keys = a[1] != Py_None;
  if (keys && (!view_of(a[1], &k, &vk) || !view_like(a[1], &q, k.n[1], &vk))) NONE;
  if (!read_tensor(a[2], &f) || f.dims != 1 || f.device != q.device || f.ptr % 8 || f.n[0] < 1 ||
      (f.n[0] > 1 && f.s[0] != 1) || 2 * f.n[0] > q.n[3])
    NONE;
  PyObject *dtype = PyObject_GetAttr(a[2], s_dtype);
  Py_XDECREF(dtype);
  PyErr_Clear();
  if (dtype != f64) NONE;
  if (PyLong_CheckExact(a[3])) {
    if (!an_int(a[3], INT32_MIN, &first)) NONE;
  } else if (!ints_of(a[3], &q, 1, &q.n[2], 1, &pos)) {
    const long n[2] = {q.n[0], q.n[2]}, one[2] = {1, q.n[2]}; /* [1, T]: for every sequence */
    if (ints_of(a[3], &q, 2, n, 0, &pos)) sb = q.n[2];
    else if (!ints_of(a[3], &q, 2, one, 0, &pos)) NONE;
  }
  const double factor = PyFloat_AsDouble(a[5]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    NONE;
  }
  if (!an_int(a[4], 0, &layout) || !an_int(a[6], 0, &back) || !stream_of(&q, &stream)) NONE;
  PyObject *y = new_like(a[0], &q, &vy), *z = NULL;
  if (y && keys) z = new_like(a[1], &k, &vz);
  if (!y || (keys && !z)) {
    Py_XDECREF(y);
    return NULL;
  }
  CALL(p_rotary(&vq, &vy, keys ? &vk : NULL, keys ? &vz : NULL, pos, sb, first,
                (const double *)f.ptr, (float)factor, layout, back, (int)q.n[0], (int)q.n[1],
                keys ? (int)k.n[1] : 0, (int)q.n[2], (int)q.n[3], (int)(2 * f.n[0]), q.dtype, stream));
  PyObject *out = keys ? PyTuple_Pack(2, y, z) : PyTuple_Pack(2, y, Py_None);
  Py_DECREF(y);
  Py_XDECREF(z);
  return done(rc, out);
}

/* the arguments that both directions of the window share: q, k, v, window, sinks, lengths */
static int window_args(PyObject *const *a, tensor *q, tensor *k, kia_view *v, int *window, int *sinks,
                       const int32_t **lengths, void **stream) {
  return view_of(a[0], q, &v[0]) && view_of(a[1], k, &v[1]) && view_like(a[1], q, k->n[1], &v[1]) &&
         view_like(a[2], q, k->n[1], &v[2]) && an_int(a[3], 1, window) && an_int(a[4], 0, sinks) &&
         ints_of(a[5], q, 1, &q->n[0], 1, lengths) && stream_of(q, stream);
}

/* window_forward(q, k, v, window, sinks, lengths) -> (o, lse) */
static PyObject *window_forward(PyObject *self, PyObject *const *a, Py_ssize_t na) {
  tensor q, k;
  kia_view v[4];
  int window, sinks, rc = 0;
  const int32_t *lengths;
  void *stream;
  uintptr_t lse;
  if (na != 6 || !window_args(a, &q, &k, v, &window, &sinks, &lengths, &stream)) NONE;
  PyObject *o = new_like(a[0], &q, &v[3]);
  PyObject *l = o ? new_of(a[0], q.n, 3, f32, &lse) : NULL;
  if (!l) {
    Py_XDECREF(o);
    return NULL;
  }
  CALL(p_window_fwd(&v[0], &v[1], &v[2], &v[3], (float *)lse, lengths, (int)q.n[0], (int)q.n[1],
                    (int)k.n[1], (int)q.n[2], (int)q.n[3], window, sinks, q.dtype, stream));
  PyObject *out = PyTuple_Pack(2, o, l);
  Py_DECREF(o);
  Py_DECREF(l);
  return done(rc, out);
}

/* window_backward(q, k, v, window, sinks, lengths, o, dO, lse) -> (dq, dk, dv) */
static PyObject *window_backward(PyObject *self, PyObject *const *a, Py_ssize_t na) {
  tensor q, k, l;
  kia_view v[8];
  int window, sinks, rc = 0;
  const int32_t *lengths;
  void *stream;
  if (na != 9 || !window_args(a, &q, &k, v, &window, &sinks, &lengths, &stream) ||
      !view_like(a[6], &q, q.n[1], &v[3]) || !view_like(a[7], &q, q.n[1], &v[4]))
    NONE;
  /* lse: [B, H, T] as the forward leaves it */
  if (!read_tensor(a[8], &l) || l.dtype != KIA_F32 || l.device != q.device || l.dims != 3 ||
      l.ptr % 16 || l.n[0] != q.n[0] || l.n[1] != q.n[1] || l.n[2] != q.n[2])
    NONE;
  if ((l.n[2] > 1 && l.s[2] != 1) || (l.n[1] > 1 && l.s[1] != l.n[2]) ||
      (l.n[0] > 1 && l.s[0] != l.n[1] * l.n[2]))
    NONE;
  size_t need;
  if (p_window_ws((int)q.n[0], (int)q.n[1], (int)k.n[1], (int)q.n[2], (int)q.n[3], window, sinks, &need))
    NONE;
  uintptr_t ws;
  const long bytes = (long)need;
  PyObject *w = new_of(a[0], &bytes, 1, u8, &ws), *g[3] = {NULL};
  if (w) g[0] = new_like(a[0], &q, &v[5]);
  if (g[0]) g[1] = new_like(a[1], &k, &v[6]);
  if (g[1]) g[2] = new_like(a[1], &k, &v[7]);
  PyObject *out = NULL;
  if (g[2]) {
    CALL(p_window_bwd(&v[0], &v[1], &v[2], &v[3], &v[4], (const float *)l.ptr, lengths, (void *)ws,
                      &v[5], &v[6], &v[7], (int)q.n[0], (int)q.n[1], (int)k.n[1], (int)q.n[2],
                      (int)q.n[3], window, sinks, q.dtype, stream));
    out = PyTuple_Pack(3, g[0], g[1], g[2]);
  }
  Py_XDECREF(w);
  for (int i = 0; i < 3; ++i) Py_XDECREF(g[i]);
  return done(rc, out);
}

/* a cache's data [pages, 2, heads, bytes] (checked by Cache4) on q's device, and a table */
static int cache_args(PyObject *data, PyObject *table, const tensor *q, tensor *c, long *width,
                      const int32_t **ptr) {
  tensor t;
  if (!read_tensor(data, c) || c->dims != 4 || c->device != q->device || c->ptr % 16) return 0;
  if (!read_tensor(table, &t) || t.dims != 2) return 0;
  const long n[2] = {q->n[0], t.n[1]};
  *width = t.n[1];
  return t.n[1] >= 1 && t.n[1] <= INT32_MAX && ints_of(table, q, 2, n, 0, ptr);
}

/* cache4_write(k, v, data, page, d, table, starts, counts) -> True */
static PyObject *cache4_write(PyObject *self, PyObject *const *a, Py_ssize_t na) {
  tensor k, c;
  kia_view vk, vv;
  int page, d, rc = 0;
  long width;
  const int32_t *table, *starts, *counts;
  void *stream;
  if (na != 8 || !view_of(a[0], &k, &vk) || !view_like(a[1], &k, k.n[1], &vv) ||
      !an_int(a[3], 1, &page) || !an_int(a[4], 1, &d) ||
      !cache_args(a[2], a[5], &k, &c, &width, &table) || d != k.n[3] || c.n[2] != k.n[1] ||
      !ints_of(a[6], &k, 1, &k.n[0], 0, &starts) || !ints_of(a[7], &k, 1, &k.n[0], 1, &counts) ||
      !stream_of(&k, &stream))
    NONE;
  CALL(p_write(&vk, &vv, (void *)c.ptr, (int)c.n[0], page, table, (int)width, starts, counts,
               (int)k.n[0], (int)k.n[1], (int)k.n[2], d, k.dtype, stream));
  Py_INCREF(Py_True);
  return done(rc, Py_True);
}

/* cache4_read(k, data, page, d, table, starts, counts) -> (k, v); k: a new contiguous tensor */
static PyObject *cache4_read(PyObject *self, PyObject *const *a, Py_ssize_t na) {
  tensor k, c;
  kia_view vk, vv;
  int page, d, rc = 0;
  long width;
  const int32_t *table, *starts, *counts;
  void *stream;
  if (na != 7 || !view_of(a[0], &k, &vk) || !an_int(a[2], 1, &page) || !an_int(a[3], 1, &d) ||
      !cache_args(a[1], a[4], &k, &c, &width, &table) || d != k.n[3] || c.n[2] != k.n[1] ||
      !ints_of(a[5], &k, 1, &k.n[0], 0, &starts) || !ints_of(a[6], &k, 1, &k.n[0], 1, &counts) ||
      !stream_of(&k, &stream))
    NONE;
  PyObject *v = new_like(a[0], &k, &vv);
  if (!v) return NULL;
  CALL(p_read((const void *)c.ptr, (int)c.n[0], page, table, (int)width, starts, counts, &vk, &vv,
              (int)k.n[0], (int)k.n[1], (int)k.n[2], d, k.dtype, stream));
  PyObject *out = PyTuple_Pack(2, a[0], v);
  Py_DECREF(v);
  return done(rc, out);
}

/* cache4_attention(q, data, page, d, table, lengths, K, calib, tau, recon, window, sinks) -> o */
static PyObject *cache4_attention(PyObject *self, PyObject *const *a, Py_ssize_t na) {
  tensor q, c;
  kia_view vq, vo;
  int page, d, K, calib, recon, window, sinks, rc = 0;
  long width;
  const int32_t *table, *lengths;
  void *stream;
  if (na != 12 || !view_of(a[0], &q, &vq) || !an_int(a[2], 1, &page) || !an_int(a[3], 1, &d) ||
      !cache_args(a[1], a[4], &q, &c, &width, &table) || d != q.n[3] ||
      !ints_of(a[5], &q, 1, &q.n[0], 0, &lengths) || !an_int(a[6], INT32_MIN, &K) ||
      !an_int(a[7], INT32_MIN, &calib) || !an_int(a[9], INT32_MIN, &recon) ||
      !an_int(a[10], 0, &window) || !an_int(a[11], 0, &sinks))
    NONE;
  const double tau = PyFloat_AsDouble(a[8]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    NONE;
  }
  if (!stream_of(&q, &stream)) NONE;
  size_t need;
  if (p_attn_ws(page, (int)width, (int)q.n[0], (int)q.n[1], (int)c.n[2], (int)q.n[2], d, window, sinks,
                &need))
    NONE;
  uintptr_t ws;
  const long bytes = (long)need;
  PyObject *o = new_like(a[0], &q, &vo);
  PyObject *w = o ? new_of(a[0], &bytes, 1, u8, &ws) : NULL;
  if (!w) {
    Py_XDECREF(o);
    return NULL;
  }
  CALL(p_attn(&vq, &vo, (const void *)c.ptr, (int)c.n[0], page, table, (int)width, lengths, (void *)ws,
              (int)q.n[0], (int)q.n[1], (int)c.n[2], (int)q.n[2], d, K, calib, (float)tau, recon, window,
              sinks, q.dtype, stream));
  Py_DECREF(w);
  return done(rc, o);
}

/* a cache's bounds [pages, heads, 2, d] in bf16, contiguous, on the cache's device */
static int bounds_of(PyObject *o, const tensor *c, long d, uintptr_t *out) {
  tensor t;
  if (!read_tensor(o, &t) || t.dims != 4 || t.dtype != KIA_BF16 || t.device != c->device || !t.ptr || t.ptr % 16)
    return 0;
  if (t.n[0] != c->n[0] || t.n[1] != c->n[2] || t.n[2] != 2 || t.n[3] != d) return 0;
  if (t.s[3] != 1 || t.s[2] != d || (t.n[1] > 1 && t.s[1] != 2 * d) || (t.n[0] > 1 && t.s[0] != 2 * d * t.n[1]))
    return 0;
  *out = t.ptr;
  return 1;
}

/* cache4_append(q, k, v, data, page, d, table, starts, counts, freq, factor, layout, bounds) -> q turned */
static PyObject *cache4_append(PyObject *self, PyObject *const *a, Py_ssize_t na) {
  tensor q, k, c, f;
  kia_view vq, vo, vk, vv;
  int page, d, layout, rc = 0;
  long width;
  const int32_t *table, *starts, *counts;
  uintptr_t bounds = 0;
  void *stream;
  if (na != 13 || !view_of(a[1], &k, &vk) || !view_of(a[0], &q, &vq) || !view_like(a[0], &k, q.n[1], &vq) ||
      !view_like(a[2], &k, k.n[1], &vv) || !an_int(a[4], 1, &page) || !an_int(a[5], 1, &d) ||
      !cache_args(a[3], a[6], &k, &c, &width, &table) || d != k.n[3] || c.n[2] != k.n[1] ||
      !ints_of(a[7], &k, 1, &k.n[0], 0, &starts) || !ints_of(a[8], &k, 1, &k.n[0], 1, &counts) ||
      !an_int(a[11], 0, &layout) || (a[12] != Py_None && !bounds_of(a[12], &c, d, &bounds)))
    NONE;
  if (!read_tensor(a[9], &f) || f.dims != 1 || f.device != k.device || f.ptr % 8 || f.n[0] < 1 ||
      (f.n[0] > 1 && f.s[0] != 1) || 2 * f.n[0] > d)
    NONE;
  PyObject *dtype = PyObject_GetAttr(a[9], s_dtype);
  Py_XDECREF(dtype);
  const double factor = PyFloat_AsDouble(a[10]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    NONE;
  }
  if (dtype != f64 || !stream_of(&k, &stream)) NONE;
  PyObject *o = new_like(a[0], &q, &vo);
  if (!o) return NULL;
  CALL(p_append(&vq, &vo, &vk, &vv, (void *)c.ptr, (void *)bounds, (int)c.n[0], page, table, (int)width, starts,
                counts, (const double *)f.ptr, (float)factor, layout, (int)k.n[0], (int)q.n[1], (int)k.n[1],
                (int)k.n[2], d, (int)(2 * f.n[0]), k.dtype, stream));
  return done(rc, o);
}

/* what the calls of queries on a cache share: q, data, page, d, table, lengths */
static int served_args(PyObject *const *a, tensor *q, tensor *c, kia_view *vq, int *page, int *d, long *width,
                       const int32_t **table, const int32_t **lengths) {
  return view_of(a[0], q, vq) && an_int(a[2], 1, page) && an_int(a[3], 1, d) &&
         cache_args(a[1], a[4], q, c, width, table) && *d == q->n[3] &&
         ints_of(a[5], q, 1, &q->n[0], 0, lengths);
}

/* cache4_select(q, data, page, d, table, lengths, bounds, count, first, last) -> pages */
static PyObject *cache4_select(PyObject *self, PyObject *const *a, Py_ssize_t na) {
  tensor q, c;
  kia_view vq;
  int page, d, count, first, last, rc = 0;
  long width;
  const int32_t *table, *lengths;
  uintptr_t bounds, ws, list;
  void *stream;
  size_t need;
  if (na != 10 || !served_args(a, &q, &c, &vq, &page, &d, &width, &table, &lengths) ||
      !bounds_of(a[6], &c, d, &bounds) || !an_int(a[7], 1, &count) || !an_int(a[8], 0, &first) ||
      !an_int(a[9], 1, &last) || (long)first + last > count || !stream_of(&q, &stream) ||
      p_select_ws(page, (int)width, (int)q.n[0], (int)q.n[1], (int)c.n[2], (int)q.n[2], d, &need))
    NONE;
  const long n[4] = {q.n[0], c.n[2], q.n[2], count}, bytes = (long)need;
  PyObject *o = new_of(a[0], n, 4, i32, &list);
  PyObject *w = o ? new_of(a[0], &bytes, 1, u8, &ws) : NULL;
  if (!w) {
    Py_XDECREF(o);
    return NULL;
  }
  CALL(p_select(&vq, (const void *)bounds, (int)c.n[0], page, table, (int)width, lengths, (void *)ws, (int32_t *)list,
                count, first, last, (int)q.n[0], (int)q.n[1], (int)c.n[2], (int)q.n[2], d, q.dtype, stream));
  Py_DECREF(w);
  return done(rc, o);
}

/* cache4_served(q, data, page, d, table, lengths, pages or None, shared, K, calib, tau, recon) -> o */
static PyObject *cache4_served(PyObject *self, PyObject *const *a, Py_ssize_t na) {
  tensor q, c, t;
  kia_view vq, vo;
  int page, d, shared, K, calib, recon, rc = 0;
  long width;
  const int32_t *table, *lengths, *list = NULL;
  void *stream;
  if (na != 12 || !served_args(a, &q, &c, &vq, &page, &d, &width, &table, &lengths) ||
      !an_int(a[7], 0, &shared) || !an_int(a[8], INT32_MIN, &K) || !an_int(a[9], INT32_MIN, &calib) ||
      !an_int(a[11], INT32_MIN, &recon))
    NONE;
  const double tau = PyFloat_AsDouble(a[10]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    NONE;
  }
  const int listed = a[6] != Py_None;
  if (listed == (shared != 0)) NONE; /* (one of the two) */
  if (listed) {
    if (!read_tensor(a[6], &t) || t.dims != 4) NONE;
    const long n[4] = {q.n[0], c.n[2], q.n[2], t.n[3]};
    if (!ints_of(a[6], &q, 4, n, 0, &list) || t.n[3] < 1 || t.n[3] > INT32_MAX) NONE;
  }
  size_t need;
  if (!stream_of(&q, &stream) ||
      (listed ? p_pages_ws(page, (int)width, (int)t.n[3], (int)q.n[0], (int)q.n[1], (int)c.n[2], (int)q.n[2], d, &need)
              : p_shared_ws(page, (int)width, shared, (int)q.n[0], (int)q.n[1], (int)c.n[2], (int)q.n[2], d, &need)))
    NONE;
  uintptr_t ws;
  const long bytes = (long)need;
  PyObject *o = new_like(a[0], &q, &vo);
  PyObject *w = o ? new_of(a[0], &bytes, 1, u8, &ws) : NULL;
  if (!w) {
    Py_XDECREF(o);
    return NULL;
  }
  if (listed)
    CALL(p_attn_pages(&vq, &vo, (const void *)c.ptr, (int)c.n[0], page, table, (int)width, lengths, list, (int)t.n[3],
                      (void *)ws, (int)q.n[0], (int)q.n[1], (int)c.n[2], (int)q.n[2], d, K, calib, (float)tau, recon,
                      q.dtype, stream));
  else
    CALL(p_attn_shared(&vq, &vo, (const void *)c.ptr, (int)c.n[0], page, table, (int)width, lengths, shared,
                       (void *)ws, (int)q.n[0], (int)q.n[1], (int)c.n[2], (int)q.n[2], d, K, calib, (float)tau, recon,
                       q.dtype, stream));
  Py_DECREF(w);
  return done(rc, o);
}

/* bind(torch, check, addresses of the entry points by name): before any other call */
static PyObject *bind(PyObject *self, PyObject *args) {
  PyObject *torch, *fns;
  if (!PyArg_ParseTuple(args, "OOO!", &torch, &check, &PyDict_Type, &fns)) return NULL;
  Py_INCREF(check);
  PyObject *C = PyObject_GetAttrString(torch, "_C");
  if (!C) return NULL;
  get_device = PyObject_GetAttrString(C, "_cuda_getDevice");
  get_stream = PyObject_GetAttrString(C, "_cuda_getCurrentRawStream");
  Py_DECREF(C);
  struct { PyObject **to; const char *name; } names[] = {
      {&Tensor, "Tensor"}, {&f32, "float32"}, {&bf16, "bfloat16"}, {&i32, "int32"}, {&f64, "float64"},
      {&u8, "uint8"}, {&empty_like, "empty_like"}, {&empty, "empty"},
      {&contiguous, "contiguous_format"}};
  for (size_t i = 0; i < sizeof names / sizeof *names; ++i)
    if (!(*names[i].to = PyObject_GetAttrString(torch, names[i].name))) return NULL;
  if (!get_device || !get_stream) return NULL;
  struct { void *to; const char *name; } entry[] = {
      {&p_rotary, "kia_rotary"}, {&p_window_fwd, "kia_window_fwd"},
      {&p_window_ws, "kia_window_ws_bytes"}, {&p_window_bwd, "kia_window_bwd"},
      {&p_write, "kia_cache4_write"}, {&p_read, "kia_cache4_read"},
      {&p_attn_ws, "kia_cache4_ws_bytes"}, {&p_attn, "kia_cache4_attn"},
      {&p_append, "kia_cache4_append"}, {&p_select_ws, "kia_cache4_select_ws_bytes"},
      {&p_select, "kia_cache4_select"}, {&p_pages_ws, "kia_cache4_pages_ws_bytes"},
      {&p_attn_pages, "kia_cache4_attn_pages"}, {&p_shared_ws, "kia_cache4_shared_ws_bytes"},
      {&p_attn_shared, "kia_cache4_attn_shared"}};
  for (size_t i = 0; i < sizeof entry / sizeof *entry; ++i) {
    PyObject *x = PyDict_GetItemString(fns, entry[i].name);
    void *p = x ? PyLong_AsVoidPtr(x) : NULL;
    if (!p) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, entry[i].name);
      return NULL;
    }
    *(void **)entry[i].to = p;
  }
  NONE;
}

static PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, NULL},
#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, NULL}
    FAST(rotary), FAST(window_forward), FAST(window_backward), FAST(cache4_write), FAST(cache4_read),
    FAST(cache4_attention), FAST(cache4_append), FAST(cache4_select), FAST(cache4_served),
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", NULL, -1, methods};

PyMODINIT_FUNC PyInit__host(void) {
  struct { PyObject **to; const char *s; } strings[] = {
      {&s_shape, "shape"}, {&s_stride, "stride"}, {&s_dtype, "dtype"}, {&s_data_ptr, "data_ptr"},
      {&s_get_device, "get_device"}, {&s_device, "device"}};
  for (size_t i = 0; i < sizeof strings / sizeof *strings; ++i)
    if (!(*strings[i].to = PyUnicode_InternFromString(strings[i].s))) return NULL;
  kw_like = Py_BuildValue("(s)", "memory_format");
  kw_empty = Py_BuildValue("(ss)", "dtype", "device");
  return kw_like && kw_empty ? PyModule_Create(&module) : NULL;
}
