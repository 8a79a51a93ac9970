/* The binding's calls of the rotary positions and the key-value cache without ctypes: the same checks
 * of the same tensors as the functions of __init__.py, in C.  Each function returns the library's status, or
 * None where an argument is not what it usually is; the caller then goes its own way, which says what is
 * wrong.  Nothing is kept between calls but what bind() is given: the library's entry points and torch's
 * types.  A call of one or two kernels takes the host 3.7 to 6.9 us this way, and 5.4 to 12 through ctypes. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "last.h"

typedef last_status (*rope_fn)(const last_rotary *, int32_t, int32_t, int32_t, const int32_t *, int64_t, const last_heads *,
                               const last_heads *, void *);
typedef last_status (*append_fn)(const last_cache *, int32_t, const last_sequences *, int32_t, const int32_t *, const last_rotary *,
                                 const int32_t *, int64_t, const last_heads *, const last_heads *, const last_heads *, void *,
                                 size_t, void *);
typedef last_status (*attention_fn)(const last_cache *, int32_t, const last_sequences *, int32_t, float, const void *, int64_t,
                                    void *, int64_t, float *, void *, size_t, void *);
typedef last_status (*chunk_fn)(const last_cache *, int32_t, const last_sequences *, int32_t, const int32_t *, int32_t, float, int32_t,
                                int32_t, const void *, int64_t, void *, int64_t, float *, void *, size_t, void *);
typedef last_status (*difference_fn)(const last_cache *, int32_t, const last_sequences *, int32_t, const int32_t *, int32_t, float,
                                     int32_t, int32_t, const last_difference *, const void *, int64_t, void *, int64_t, void *,
                                     size_t, void *);
typedef last_status (*copy_fn)(const last_cache *, int32_t, const int32_t *, const int32_t *, void *, size_t, void *);
typedef last_status (*compact_fn)(const last_cache *, const last_sequences *, const int32_t *, int32_t, int64_t, const int32_t *,
                                  const int32_t *, const int32_t *, const int32_t *, int32_t, int32_t *, void *, size_t, void *);

static rope_fn f_rope[2];
static append_fn f_append;
static attention_fn f_attention;
static chunk_fn f_chunk;
static difference_fn f_difference;
static copy_fn f_copy;
static compact_fn f_compact;
static PyObject *t_f32, *t_bf16, *t_int32, *get_stream, *get_device;
static PyObject *s_shape, *s_stride, *s_is_cuda, *s_dtype, *s_data_ptr, *s_nbytes, *s_is_contiguous, *s_cuda_stream;

typedef struct {
  void *ptr;
  int rank;
  long long shape[5], stride[5];
  PyObject *dtype;   /* compared only */
} tensor;

static int attribute_is_true(PyObject *o, PyObject *name) {
  PyObject *v = PyObject_GetAttr(o, name);
  const int yes = v == Py_True;
  Py_XDECREF(v);
  return yes;
}

static int numbers(PyObject *tuple, long long *to) {   /* consumes the tuple; its length, or -1 */
  int n = -1;
  if (tuple != NULL && PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) <= 5) {
    n = (int)PyTuple_GET_SIZE(tuple);
    for (int i = 0; i < n; ++i) {
      to[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, i));
      if (to[i] == -1 && PyErr_Occurred()) n = -1;
    }
  }
  Py_XDECREF(tuple);
  return n;
}

static int pointer_of(PyObject *o, void **to) {
  PyObject *v = PyObject_CallMethodNoArgs(o, s_data_ptr);
  if (v == NULL) return 0;
  *to = (void *)(uintptr_t)PyLong_AsUnsignedLongLong(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}

/* A device tensor of this type (NULL: any); 0 if it is none. */
static int get(PyObject *o, PyObject *dtype, tensor *t) {
  t->rank = numbers(PyObject_GetAttr(o, s_shape), t->shape);
  if (t->rank < 0 || numbers(PyObject_CallMethodNoArgs(o, s_stride), t->stride) != t->rank) return 0;
  t->dtype = PyObject_GetAttr(o, s_dtype);
  if (t->dtype == NULL) return 0;
  Py_DECREF(t->dtype);
  return (dtype == NULL || t->dtype == dtype) && attribute_is_true(o, s_is_cuda) && pointer_of(o, &t->ptr);
}

/* int32 [n] (n < 0: any length). */
static int get_ints(PyObject *o, long long n, tensor *t) {
  return get(o, t_int32, t) && t->rank == 1 && (n < 0 || t->shape[0] == n) && (t->shape[0] <= 1 || t->stride[0] == 1);
}

static int get_workspace(PyObject *o, void **ptr, size_t *bytes) {
  if (!attribute_is_true(o, s_is_cuda)) return 0;
  PyObject *c = PyObject_CallMethodNoArgs(o, s_is_contiguous), *n;
  const int ok = c == Py_True;
  Py_XDECREF(c);
  if (!ok || (n = PyObject_GetAttr(o, s_nbytes)) == NULL) return 0;
  *bytes = PyLong_AsSize_t(n);
  Py_DECREF(n);
  return !PyErr_Occurred() && pointer_of(o, ptr);
}

static int stream_of(PyObject *o, void **to) {
  PyObject *v;
  if (o == Py_None) {
    PyObject *d = PyObject_CallNoArgs(get_device);
    if (d == NULL) return 0;
    v = PyObject_CallOneArg(get_stream, d);
    Py_DECREF(d);
  } else if (PyLong_Check(o)) {
    v = Py_NewRef(o);
  } else {
    v = PyObject_GetAttr(o, s_cuda_stream);
  }
  if (v == NULL) return 0;
  *to = (void *)(uintptr_t)PyLong_AsUnsignedLongLong(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}

static int get_heads(PyObject *in, PyObject *out, PyObject *dtype, long long dim, long long tokens, last_heads *h) {
  tensor x, y;
  if (!get(in, dtype, &x) || x.rank != 3 || x.shape[0] != tokens || x.shape[2] != dim || (x.stride[2] != 1 && dim > 1) ||
      x.shape[1] > INT32_MAX)
    return 0;
  *h = (last_heads){x.ptr, NULL, (int32_t)x.shape[1], x.stride[0], x.stride[1], 0, 0};
  if (out == Py_None) return 1;
  if (!get(out, dtype, &y) || y.rank != 3 || y.shape[0] != tokens || y.shape[1] != x.shape[1] || y.shape[2] != dim ||
      (y.stride[2] != 1 && dim > 1))
    return 0;
  h->out = y.ptr;
  h->out_token = y.stride[0];
  h->out_head = y.stride[1];
  return 1;
}

static int get_positions(PyObject *o, long long axes, long long tokens, const int32_t **ptr, int64_t *stride) {
  tensor t;
  if (!get(o, t_int32, &t)) return 0;
  if (t.rank == 1 && axes == 1) {
    if (t.shape[0] != tokens || (tokens > 1 && t.stride[0] != 1)) return 0;
    *stride = tokens;
  } else {
    if (t.rank != 2 || t.shape[0] != axes || t.shape[1] != tokens || (tokens > 1 && t.stride[1] != 1)) return 0;
    *stride = axes > 1 ? t.stride[0] : tokens;
  }
  *ptr = t.ptr;
  return 1;
}

static int integer(PyObject *o, long long *to) {
  if (!PyLong_Check(o)) return 0;
  *to = PyLong_AsLongLong(o);
  return !PyErr_Occurred();
}

static int address(PyObject *o, const void **to) {
  long long v;
  if (!integer(o, &v)) return 0;
  *to = (const void *)(uintptr_t)v;
  return 1;
}

static PyObject *other_way(void) {
  PyErr_Clear();
  Py_RETURN_NONE;
}

#define CALL(expression)              \
  do {                                \
    last_status st_;                  \
    Py_BEGIN_ALLOW_THREADS            \
    st_ = (expression);               \
    Py_END_ALLOW_THREADS              \
    return PyLong_FromLong((long)st_);\
  } while (0)

/* rope(backward, rotary, num_axes, positions, q, q_out, k, k_out, stream) */
static PyObject *rope(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  long long back, axes;
  const void *r;
  tensor q;
  last_heads qh, kh;
  const int32_t *pos;
  int64_t stride;
  void *stream;
  if (n != 9 || !integer(a[0], &back) || !address(a[1], &r) || !integer(a[2], &axes) || !get(a[4], NULL, &q) || q.rank != 3 ||
      (q.dtype != t_f32 && q.dtype != t_bf16) || q.shape[0] > INT32_MAX || q.shape[2] > INT32_MAX || a[5] == Py_None ||
      (a[6] == Py_None) != (a[7] == Py_None) || !get_heads(a[4], a[5], q.dtype, q.shape[2], q.shape[0], &qh) ||
      (a[6] != Py_None && !get_heads(a[6], a[7], q.dtype, q.shape[2], q.shape[0], &kh)) ||
      !get_positions(a[3], axes, q.shape[0], &pos, &stride) || !stream_of(a[8], &stream))
    return other_way();
  CALL(f_rope[back != 0](r, q.dtype == t_f32 ? LAST_DTYPE_F32 : LAST_DTYPE_BF16, (int32_t)q.shape[0], (int32_t)q.shape[2], pos,
                         stride, &qh, a[6] == Py_None ? NULL : &kh, stream));
}

/* append(cache, layer, sequences, batch, head_dim, dtype, k, v, ws, cu_new, rotary, num_axes, positions, q, q_out, stream) */
static PyObject *append(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  long long layer, batch, dim, axes = 0;
  const void *c, *s, *r = NULL;
  tensor k, cu;
  last_heads kh, vh, qh;
  const int32_t *pos = NULL;
  int64_t stride = 0;
  void *ws, *stream;
  size_t bytes;
  if (n != 16 || !address(a[0], &c) || !integer(a[1], &layer) || !address(a[2], &s) || !integer(a[3], &batch) || !integer(a[4], &dim) ||
      !get(a[6], a[5], &k) || k.rank != 3 || k.shape[0] > INT32_MAX || layer != (int32_t)layer ||
      (a[13] == Py_None) != (a[14] == Py_None) || !get_heads(a[6], Py_None, a[5], dim, k.shape[0], &kh) ||
      !get_heads(a[7], Py_None, a[5], dim, k.shape[0], &vh) || !get_workspace(a[8], &ws, &bytes) ||
      (a[9] != Py_None && !get_ints(a[9], batch + 1, &cu)) ||
      (a[10] != Py_None && (!address(a[10], &r) || !integer(a[11], &axes) || !get_positions(a[12], axes, k.shape[0], &pos, &stride))) ||
      (a[13] != Py_None && !get_heads(a[13], a[14], a[5], dim, k.shape[0], &qh)) || !stream_of(a[15], &stream))
    return other_way();
  CALL(f_append(c, (int32_t)layer, s, (int32_t)k.shape[0], a[9] == Py_None ? NULL : cu.ptr, r, pos, stride,
                a[13] == Py_None ? NULL : &qh, &kh, &vh, ws, bytes, stream));
}

/* attention(cache, layer, sequences, batch, head_dim, dtype, q, out, ws, lse, scale, stream) */
static PyObject *attention(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  long long layer, batch, dim;
  const void *c, *s;
  tensor q, o, l = {0};
  void *ws, *stream;
  size_t bytes;
  if (n != 12 || !address(a[0], &c) || !integer(a[1], &layer) || !address(a[2], &s) || !integer(a[3], &batch) || !integer(a[4], &dim) ||
      !get(a[6], a[5], &q) || !get(a[7], a[5], &o) || q.rank != 3 || o.rank != 3 || q.shape[0] != batch || q.shape[2] != dim ||
      o.shape[0] != batch || o.shape[1] != q.shape[1] || o.shape[2] != dim || q.stride[2] != 1 || o.stride[2] != 1 ||
      (q.shape[1] > 1 && (q.stride[1] != dim || o.stride[1] != dim)) || q.shape[1] > INT32_MAX || layer != (int32_t)layer)
    return other_way();
  if (a[9] != Py_None &&
      (!get(a[9], t_f32, &l) || l.rank != 2 || l.shape[0] != batch || l.shape[1] != q.shape[1] ||
       (l.shape[1] > 1 && l.stride[1] != 1) || (l.shape[0] > 1 && l.stride[0] != l.shape[1])))
    return other_way();
  const double scale = PyFloat_AsDouble(a[10]);
  if (PyErr_Occurred() || !get_workspace(a[8], &ws, &bytes) || !stream_of(a[11], &stream)) return other_way();
  CALL(f_attention(c, (int32_t)layer, s, (int32_t)q.shape[1], (float)scale, q.ptr, q.stride[0], o.ptr, o.stride[0], l.ptr, ws, bytes,
                   stream));
}

/* fp32, contiguous, [n] or, with m >= 0, [n][m]. */
static int get_floats(PyObject *o, long long n, long long m, tensor *t) {
  return get(o, t_f32, t) && t->rank == (m < 0 ? 1 : 2) && t->shape[0] == n && (m < 0 || t->shape[1] == m) &&
         (t->shape[t->rank - 1] <= 1 || t->stride[t->rank - 1] == 1) && (m < 0 || n <= 1 || t->stride[0] == m);
}

typedef struct {
  long long layer, window, tokens, heads;
  const void *c, *s;
  tensor q, o, cu;
  void *ws, *stream;
  size_t bytes;
  double scale;
  int causal;
} chunk_args;

/* What both kinds of attention of several new tokens take: cache, layer, sequences, batch, head_dim, dtype, q, out, ws, cu_new in a;
 * causal, window, scale, stream in z.  pairs: a value is two heads wide. */
static int get_chunk(PyObject *const *a, PyObject *const *z, int pairs, chunk_args *g) {
  long long batch, dim;
  if (!address(a[0], &g->c) || !integer(a[1], &g->layer) || !address(a[2], &g->s) || !integer(a[3], &batch) || !integer(a[4], &dim) ||
      !get(a[6], a[5], &g->q) || !get(a[7], a[5], &g->o) || g->q.rank != 3 || g->o.rank != 3 || g->q.shape[2] != dim ||
      g->q.shape[0] > INT32_MAX || g->q.shape[1] > INT32_MAX || g->q.shape[1] % (pairs ? 2 : 1) != 0 || g->o.shape[0] != g->q.shape[0] ||
      g->o.shape[1] != (pairs ? g->q.shape[1] / 2 : g->q.shape[1]) || g->o.shape[2] != (pairs ? 2 * dim : dim) ||
      g->q.stride[2] != 1 || g->o.stride[2] != 1 || (g->q.shape[1] > 1 && g->q.stride[1] != dim) ||
      (g->o.shape[1] > 1 && g->o.stride[1] != g->o.shape[2]) || g->layer != (int32_t)g->layer || !get_workspace(a[8], &g->ws, &g->bytes))
    return 0;
  g->cu = (tensor){0};
  if (a[9] != Py_None && !get_ints(a[9], batch + 1, &g->cu)) return 0;
  g->tokens = g->q.shape[0];
  g->heads = g->q.shape[1];
  g->scale = PyFloat_AsDouble(z[2]);
  return (z[0] == Py_True || z[0] == Py_False) && integer(z[1], &g->window) && g->window == (int32_t)g->window && !PyErr_Occurred() &&
         (g->causal = z[0] == Py_True, stream_of(z[3], &g->stream));
}

/* chunk(cache, layer, sequences, batch, head_dim, dtype, q, out, ws, cu_new, lse, causal, window, scale, stream) */
static PyObject *chunk(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  chunk_args g;
  tensor l = {0};
  if (n != 15 || !get_chunk(a, a + 11, 0, &g) || (a[10] != Py_None && !get_floats(a[10], g.tokens, g.heads, &l))) return other_way();
  CALL(f_chunk(g.c, (int32_t)g.layer, g.s, (int32_t)g.tokens, g.cu.ptr, (int32_t)g.heads, (float)g.scale, g.causal, (int32_t)g.window,
               g.q.ptr, g.q.stride[0], g.o.ptr, g.o.stride[0], l.ptr, g.ws, g.bytes, g.stream));
}

/* difference(cache, layer, sequences, batch, head_dim, dtype, q, out, ws, cu_new, lam, norm_weight, norm_eps, out_scale, causal, window,
 * scale, stream) */
static PyObject *difference(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  chunk_args g;
  tensor lam, w = {0};
  if (n != 18 || !get_chunk(a, a + 14, 1, &g) || !get_floats(a[10], g.heads / 2, -1, &lam) ||
      (a[11] != Py_None && !get_floats(a[11], g.o.shape[2], -1, &w)))
    return other_way();
  const double eps = PyFloat_AsDouble(a[12]), scale = PyFloat_AsDouble(a[13]);
  if (PyErr_Occurred()) return other_way();
  const last_difference d = {lam.ptr, w.ptr, (float)eps, (float)scale};
  CALL(f_difference(g.c, (int32_t)g.layer, g.s, (int32_t)g.tokens, g.cu.ptr, (int32_t)g.heads, (float)g.scale, g.causal,
                    (int32_t)g.window, &d, g.q.ptr, g.q.stride[0], g.o.ptr, g.o.stride[0], g.ws, g.bytes, g.stream));
}

/* copy(cache, src, dst, ws, stream) */
static PyObject *copy(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  const void *c;
  tensor x, y;
  void *ws, *stream;
  size_t bytes;
  if (n != 5 || !address(a[0], &c) || !get_ints(a[1], -1, &x) || !get_ints(a[2], x.shape[0], &y) || x.shape[0] > INT32_MAX ||
      !get_workspace(a[3], &ws, &bytes) || !stream_of(a[4], &stream))
    return other_way();
  CALL(f_copy(c, (int32_t)x.shape[0], x.ptr, y.ptr, ws, bytes, stream));
}

/* compact(cache, sequences, batch, dst_table, cu_keep, idx, lens_out, ws, span_begin, span_len, stream) */
static PyObject *compact(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  const void *c, *s;
  long long batch;
  tensor d, keep, idx, out, first = {0}, len = {0};
  void *ws, *stream;
  size_t bytes;
  if (n != 11 || !address(a[0], &c) || !address(a[1], &s) || !integer(a[2], &batch) || !get(a[3], t_int32, &d) || d.rank != 2 ||
      d.shape[0] != batch || (d.shape[1] > 1 && d.stride[1] != 1) || d.shape[1] > INT32_MAX || !get_ints(a[4], batch + 1, &keep) ||
      !get_ints(a[5], -1, &idx) || idx.shape[0] > INT32_MAX || !get_ints(a[6], batch, &out) || !get_workspace(a[7], &ws, &bytes) ||
      (a[8] != Py_None && !get_ints(a[8], batch, &first)) || (a[9] != Py_None && !get_ints(a[9], batch, &len)) ||
      !stream_of(a[10], &stream))
    return other_way();
  CALL(f_compact(c, s, d.ptr, (int32_t)d.shape[1], d.stride[0], first.ptr, len.ptr, keep.ptr, idx.ptr, (int32_t)idx.shape[0], out.ptr,
                 ws, bytes, stream));
}

/* bind(rope, rope_backward, append, attention, copy, compact, chunk, difference, float32, bfloat16, int32, get_stream, get_device):
 * the first eight are addresses. */
static PyObject *bind(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  (void)self;
  const void *f[8];
  if (n != 13) {
    PyErr_SetString(PyExc_TypeError, "bind takes 13 arguments");
    return NULL;
  }
  for (int i = 0; i < 8; ++i)
    if (!address(a[i], &f[i])) {
      PyErr_SetString(PyExc_TypeError, "an address is an int");
      return NULL;
    }
  f_rope[0] = (rope_fn)f[0];
  f_rope[1] = (rope_fn)f[1];
  f_append = (append_fn)f[2];
  f_attention = (attention_fn)f[3];
  f_copy = (copy_fn)f[4];
  f_compact = (compact_fn)f[5];
  f_chunk = (chunk_fn)f[6];
  f_difference = (difference_fn)f[7];
  PyObject **to[5] = {&t_f32, &t_bf16, &t_int32, &get_stream, &get_device};
  for (int i = 0; i < 5; ++i) Py_XSETREF(*to[i], Py_NewRef(a[8 + i]));
  Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(bind), METHOD(rope), METHOD(append), METHOD(attention), METHOD(copy), METHOD(compact),
                                METHOD(chunk), METHOD(difference), {0}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
  PyObject **names[8] = {&s_shape, &s_stride, &s_is_cuda, &s_dtype, &s_data_ptr, &s_nbytes, &s_is_contiguous, &s_cuda_stream};
  const char *text[8] = {"shape", "stride", "is_cuda", "dtype", "data_ptr", "nbytes", "is_contiguous", "cuda_stream"};
  for (int i = 0; i < 8; ++i)
    if ((*names[i] = PyUnicode_InternFromString(text[i])) == NULL) return NULL;
  return PyModule_Create(&module);
}
