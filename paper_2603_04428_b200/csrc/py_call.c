/* Argument marshalling of the per-layer entry points for Python: a CPython module that turns the binding's arguments into one
 * C call.  Bound by interpreter overhead: through ctypes the smallest decode call spent 7.3 us on the host, 1.6 of them on the
 * conversion of its nineteen arguments and 1.4 on the pointers of its nine tensors; the launch itself takes 2.9.  Here 5.1 us,
 * below what the GPU takes (6.5); an append 5.5 -> 4.0.  The other entry points are called rarely and stay with ctypes.
 * The later calls (norm and rotation, shared prefixes, block copies) also refuse tensors of another device than the current one.
 * The entry points' addresses come from the ctypes library (bind), so there is one copy of the library in the process. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/q4kv.h"

static int (*f_append)(const q4kv_spec*, void*, int32_t, int32_t, const q4kv_batch*, const int32_t*, const int32_t*, int32_t,
                       const void*, const void*, int32_t*, void*);
static int (*f_decode)(const q4kv_spec*, const void*, int32_t, int32_t, const q4kv_batch*, const int32_t*, int32_t, int32_t,
                       const void*, float, void*, int32_t, float*, void*, size_t, int32_t*, void*);
static int (*f_append_decode)(const q4kv_spec*, void*, int32_t, int32_t, const q4kv_batch*, const int32_t*, int32_t, int32_t,
                              const void*, const void*, const void*, float, void*, int32_t, float*, void*, size_t, int32_t*,
                              void*);
static int (*f_prefill)(const q4kv_spec*, const void*, int32_t, int32_t, const q4kv_batch*, const int32_t*, const int32_t*,
                        int32_t, int32_t, int32_t, int32_t, const void*, float, void*, int32_t, float*, void*, size_t, int32_t*,
                        void*);
static int (*f_norm_rope)(const q4kv_spec*, const q4kv_norm_rotation*, int32_t, const int32_t*, const int32_t*, int32_t, const void*,
                          int64_t, const void*, int64_t, void*, void*, int32_t*, void*);
static int (*f_copy_blocks)(const q4kv_spec*, const void*, int32_t, void*, int32_t, int32_t, int32_t, const int32_t*, int32_t,
                            int32_t*, void*);
static int (*f_shared_prefix)(const q4kv_spec*, const void*, int32_t, int32_t, const q4kv_batch*, const int32_t*, int32_t, const int32_t*,
                              const int32_t*, int32_t, const void*, float, void*, int32_t, float*, void*, size_t, int32_t*, void*);
static PyObject *s_is_cuda, *s_is_contiguous, *s_data_ptr, *s_nbytes, *s_get_device, *s_stride, *s_dtype, *s_shape;
static PyObject* bfloat16;                                 /* torch.bfloat16 */

static int on_device(PyObject* o, long dev);
/* A device pointer: None, an integer, or a contiguous CUDA tensor.
   dev: the device that a tensor has to lie on (which also says that it is a CUDA tensor), or kAnyDevice */
enum { kAnyDevice = -1 };
static int get_ptr_at(PyObject* o, long dev, void** out) {
  if (o == Py_None) { *out = NULL; return 1; }
  if (PyLong_Check(o)) { *out = PyLong_AsVoidPtr(o); return !(*out == NULL && PyErr_Occurred()); }
  PyObject* r;
  int ok = 1;
  if (dev == kAnyDevice) {
    if (!(r = PyObject_GetAttr(o, s_is_cuda))) return 0;
    ok = PyObject_IsTrue(r);
    Py_DECREF(r);
  } else if (!on_device(o, dev)) {
    return 0;
  }
  if (ok > 0) {
    if (!(r = PyObject_CallMethodNoArgs(o, s_is_contiguous))) return 0;
    ok = PyObject_IsTrue(r);
    Py_DECREF(r);
  }
  if (ok < 0) return 0;
  if (!ok) { PyErr_SetString(PyExc_AssertionError, "device pointers come from contiguous CUDA tensors"); return 0; }
  if (!(r = PyObject_CallMethodNoArgs(o, s_data_ptr))) return 0;
  *out = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return !(*out == NULL && PyErr_Occurred());
}
static int get_ptr(PyObject* o, void** out) { return get_ptr_at(o, kAnyDevice, out); }
static int get_i32(PyObject* o, int32_t* out) {
  const unsigned long v = PyLong_AsUnsignedLongMask(o);
  *out = (int32_t)(uint32_t)v;
  return !(v == (unsigned long)-1 && PyErr_Occurred());
}
static int get_f32(PyObject* o, float* out) {
  const double v = PyFloat_AsDouble(o);
  *out = (float)v;
  return !(v == -1.0 && PyErr_Occurred());
}
static int get_bytes(PyObject* o, size_t* out) {           /* of a tensor */
  PyObject* r = PyObject_GetAttr(o, s_nbytes);
  if (!r) return 0;
  *out = PyLong_AsSize_t(r);
  Py_DECREF(r);
  return !(*out == (size_t)-1 && PyErr_Occurred());
}
/* The bytes of a ctypes structure, copied. */
static int get_struct(PyObject* o, void* out, size_t size) {
  Py_buffer v;
  if (PyObject_GetBuffer(o, &v, PyBUF_SIMPLE) != 0) return 0;
  const int ok = (size_t)v.len == size;
  if (ok) memcpy(out, v.buf, size);
  PyBuffer_Release(&v);
  if (!ok) PyErr_SetString(PyExc_TypeError, "a Spec and a Batch are expected");
  return ok;
}
static int count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return 1;
  PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, n);
  return 0;
}

/* spec, pool, n_blocks, layer, batch: the first five arguments of all four */
typedef struct { q4kv_spec spec; q4kv_batch batch; void* pool; int32_t n_blocks, layer; } Head;
static int get_head(PyObject* const* a, Head* h) {
  return get_struct(a[0], &h->spec, sizeof h->spec) && get_ptr(a[1], &h->pool) && get_i32(a[2], &h->n_blocks) &&
         get_i32(a[3], &h->layer) && get_struct(a[4], &h->batch, sizeof h->batch);
}
/* q, softmax_scale, out, out_dtype, lse, workspace, status_flags, stream: the last eight of the attention calls */
typedef struct { void *q, *out, *lse, *ws, *flags, *stream; float scale; int32_t out_dtype; size_t ws_bytes; } Tail;
static int get_tail(PyObject* const* a, Tail* t) {
  return get_ptr(a[0], &t->q) && get_f32(a[1], &t->scale) && get_ptr(a[2], &t->out) && get_i32(a[3], &t->out_dtype) &&
         get_ptr(a[4], &t->lse) && get_ptr(a[5], &t->ws) && get_bytes(a[5], &t->ws_bytes) && get_ptr(a[6], &t->flags) &&
         get_ptr(a[7], &t->stream);
}

static PyObject* append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Head h;
  void *pos, *offs, *k, *v, *flags, *stream;
  int32_t total;
  int rc;
  if (!count(n, 12) || !get_head(a, &h) || !get_ptr(a[5], &pos) || !get_ptr(a[6], &offs) || !get_i32(a[7], &total) ||
      !get_ptr(a[8], &k) || !get_ptr(a[9], &v) || !get_ptr(a[10], &flags) || !get_ptr(a[11], &stream))
    return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = f_append(&h.spec, h.pool, h.n_blocks, h.layer, &h.batch, pos, offs, total, k, v, flags, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
static PyObject* decode(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Head h;
  Tail t;
  void* lens;
  int32_t max_kv, window;
  int rc;
  if (!count(n, 16) || !get_head(a, &h) || !get_ptr(a[5], &lens) || !get_i32(a[6], &max_kv) || !get_i32(a[7], &window) ||
      !get_tail(a + 8, &t))
    return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = f_decode(&h.spec, h.pool, h.n_blocks, h.layer, &h.batch, lens, max_kv, window, t.q, t.scale, t.out, t.out_dtype, t.lse,
                t.ws, t.ws_bytes, t.flags, t.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
static PyObject* append_decode(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Head h;
  Tail t;
  void *lens, *k, *v;
  int32_t max_kv, window;
  int rc;
  if (!count(n, 18) || !get_head(a, &h) || !get_ptr(a[5], &lens) || !get_i32(a[6], &max_kv) || !get_i32(a[7], &window) ||
      !get_ptr(a[8], &k) || !get_ptr(a[9], &v) || !get_tail(a + 10, &t))
    return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = f_append_decode(&h.spec, h.pool, h.n_blocks, h.layer, &h.batch, lens, max_kv, window, k, v, t.q, t.scale, t.out,
                       t.out_dtype, t.lse, t.ws, t.ws_bytes, t.flags, t.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
static PyObject* prefill(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Head h;
  Tail t;
  void *lens, *offs;
  int32_t total, max_q, max_kv, window;
  int rc;
  if (!count(n, 19) || !get_head(a, &h) || !get_ptr(a[5], &lens) || !get_ptr(a[6], &offs) || !get_i32(a[7], &total) ||
      !get_i32(a[8], &max_q) || !get_i32(a[9], &max_kv) || !get_i32(a[10], &window) || !get_tail(a + 11, &t))
    return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = f_prefill(&h.spec, h.pool, h.n_blocks, h.layer, &h.batch, lens, offs, total, max_q, max_kv, window, t.q, t.scale, t.out,
                 t.out_dtype, t.lse, t.ws, t.ws_bytes, t.flags, t.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
/* Whether a tensor lies on device dev (an integer or None does). */
static int on_device(PyObject* o, long dev) {
  if (o == Py_None || PyLong_Check(o)) return 1;
  PyObject* r = PyObject_CallMethodNoArgs(o, s_get_device);
  if (!r) return 0;
  const long at = PyLong_AsLong(r);
  Py_DECREF(r);
  if (at == -1 && PyErr_Occurred()) return 0;
  if (at != dev) { PyErr_SetString(PyExc_AssertionError, "a tensor lies on another device than the current one"); return 0; }
  return 1;
}
/* The same as get_ptr for a tensor that has to lie on device dev. */
static int get_ptr_on(PyObject* o, int32_t dev, void** out) {
  if (dev < 0) { PyErr_SetString(PyExc_AssertionError, "no such device"); return 0; }
  return get_ptr_at(o, dev, out);
}
static int is_bf16(PyObject* o) {                          /* -1: an error is set */
  PyObject* r = PyObject_GetAttr(o, s_dtype);
  if (!r) return -1;
  const int same = r == bfloat16;
  Py_DECREF(r);
  return same;
}
/* Whether the shape is [at least rows][heads][d] (no len(): it takes a tensor longer than all the rest of these calls). */
static int has_shape(PyObject* o, int64_t rows, int64_t heads, int64_t d) {
  PyObject* r = PyObject_GetAttr(o, s_shape);
  if (!r) { PyErr_Clear(); return 0; }
  int ok = PyTuple_Check(r) && PyTuple_GET_SIZE(r) == 3;
  const int64_t want[3] = {rows, heads, d};
  for (int i = 0; ok && i < 3; ++i) {
    const int64_t n = PyLong_AsLongLong(PyTuple_GET_ITEM(r, i));
    ok = i == 0 ? n >= want[i] : n == want[i];
  }
  Py_DECREF(r);
  return ok;
}
/* Rows [tokens][heads][d] of bfloat16 whose first stride is free: pointer and stride. */
static int get_rows(PyObject* o, long dev, void** out, int64_t heads, int64_t d, int64_t rows, int64_t* stride) {
  int64_t st[3];
  PyObject* r;
  *stride = heads * d;
  if (o == Py_None) { *out = NULL; return 1; }
  if (!on_device(o, dev) || !(r = PyObject_CallMethodNoArgs(o, s_stride))) return 0;
  int ok = PyArg_ParseTuple(r, "LLL", &st[0], &st[1], &st[2]);
  Py_DECREF(r);
  if (!ok) return 0;
  ok = rows <= 0 || (has_shape(o, rows, heads, d) && (st[2] == 1 || d == 1) && (st[1] == d || heads == 1) && is_bf16(o) != 0);
  if (PyErr_Occurred()) return 0;
  if (!ok) {
    PyErr_SetString(PyExc_AssertionError, "rows are bfloat16 [tokens][heads][d] with whole heads next to each other");
    return 0;
  }
  if (rows > 1) *stride = st[0];
  if (!(r = PyObject_CallMethodNoArgs(o, s_data_ptr))) return 0;
  *out = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return !(*out == NULL && PyErr_Occurred());
}
/* Where such rows go: a contiguous bfloat16 tensor with room for them, whatever its shape. */
static int get_rows_out(PyObject* o, int32_t dev, void** out, int64_t heads, int64_t d, int64_t rows) {
  size_t bytes;
  if (!get_ptr_on(o, dev, out)) return 0;
  if (o == Py_None || PyLong_Check(o) || rows <= 0) return 1;
  const int ok = is_bf16(o);
  if (ok < 0 || !get_bytes(o, &bytes)) return 0;
  if (!ok || bytes / 2 / (size_t)rows < (size_t)(heads * d)) {
    PyErr_SetString(PyExc_AssertionError, "an output is bfloat16 with room for every row");
    return 0;
  }
  return 1;
}
/* spec, how, n_agents, pos, new_offs, total_new, q, k, q_out, k_out, status_flags, stream, device */
static PyObject* norm_rope(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  q4kv_spec spec;
  q4kv_norm_rotation how;
  void *pos, *offs, *q, *k, *qo, *ko, *flags, *stream;
  int32_t agents, total, dev;
  int64_t qs, ks;
  int rc;
  if (!count(n, 13) || !get_struct(a[0], &spec, sizeof spec) || !get_struct(a[1], &how, sizeof how) || !get_i32(a[2], &agents) ||
      !get_i32(a[12], &dev) || !get_ptr_on(a[3], dev, &pos) || !get_ptr_on(a[4], dev, &offs) || !get_i32(a[5], &total) ||
      !get_rows(a[6], dev, &q, spec.n_q_heads, spec.d_qk, total, &qs) ||
      !get_rows(a[7], dev, &k, spec.n_kv_heads, spec.d_qk, total, &ks) ||
      !get_rows_out(a[8], dev, &qo, spec.n_q_heads, spec.d_qk, total) ||
      !get_rows_out(a[9], dev, &ko, spec.n_kv_heads, spec.d_qk, total) || !get_ptr_on(a[10], dev, &flags) || !get_ptr(a[11], &stream))
    return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = f_norm_rope(&spec, &how, agents, pos, offs, total, q, qs, k, ks, qo, ko, flags, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
/* spec, src_pool, src_blocks, dst_pool, dst_blocks, layer_begin, layer_count, copies, n_copies, status_flags, stream, device */
static PyObject* copy_blocks(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  q4kv_spec spec;
  void *src, *dst, *copies, *flags, *stream;
  int32_t ns, nd, l0, nl, nc, dev;
  int rc;
  if (!count(n, 12) || !get_struct(a[0], &spec, sizeof spec) || !get_i32(a[11], &dev) || !get_ptr_on(a[1], dev, &src) ||
      !get_i32(a[2], &ns) || !get_ptr_on(a[3], dev, &dst) || !get_i32(a[4], &nd) || !get_i32(a[5], &l0) || !get_i32(a[6], &nl) ||
      !get_ptr_on(a[7], dev, &copies) || !get_i32(a[8], &nc) || !get_ptr_on(a[9], dev, &flags) || !get_ptr(a[10], &stream))
    return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = f_copy_blocks(&spec, src, ns, dst, nd, l0, nl, copies, nc, flags, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
/* spec, pool, n_blocks, layer, batch, kv_lens, max_kv_len, group_offs, prefix_lens, n_groups, q .. stream, device */
static PyObject* shared_prefix(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Head h;
  Tail t;
  void *lens, *offs, *prefix;
  int32_t max_kv, groups, dev;
  int rc;
  if (!count(n, 19) || !get_head(a, &h) || !get_i32(a[18], &dev) || !on_device(a[1], dev) || !get_ptr_on(a[5], dev, &lens) ||
      !get_i32(a[6], &max_kv) || !get_ptr_on(a[7], dev, &offs) || !get_ptr_on(a[8], dev, &prefix) || !get_i32(a[9], &groups) ||
      !get_tail(a + 10, &t))
    return NULL;
  for (int i = 10; i < 17; ++i)                            /* q, out, lse, workspace, status_flags (numbers pass) */
    if (i != 11 && i != 13 && !on_device(a[i], dev)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = f_shared_prefix(&h.spec, h.pool, h.n_blocks, h.layer, &h.batch, lens, max_kv, offs, prefix, groups, t.q, t.scale, t.out,
                       t.out_dtype, t.lse, t.ws, t.ws_bytes, t.flags, t.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
/* bind(append, decode, append_decode, prefill, norm_rope, copy_blocks, shared_prefix): the entry points' addresses */
static PyObject* bind(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* p[7];
  if (!count(n, 7)) return NULL;
  for (int i = 0; i < 7; ++i)
    if (!get_ptr(a[i], &p[i])) return NULL;
  *(void**)&f_append = p[0]; *(void**)&f_decode = p[1]; *(void**)&f_append_decode = p[2]; *(void**)&f_prefill = p[3];
  *(void**)&f_norm_rope = p[4]; *(void**)&f_copy_blocks = p[5]; *(void**)&f_shared_prefix = p[6];
  Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {FAST(append), FAST(decode), FAST(append_decode), FAST(prefill), FAST(norm_rope),
                                FAST(copy_blocks), FAST(shared_prefix), FAST(bind), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__call(void) {
  s_is_cuda = PyUnicode_InternFromString("is_cuda");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_nbytes = PyUnicode_InternFromString("nbytes");
  s_get_device = PyUnicode_InternFromString("get_device");
  s_stride = PyUnicode_InternFromString("stride");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_shape = PyUnicode_InternFromString("shape");
  PyObject* torch = PyImport_ImportModule("torch");
  if (!torch) return NULL;
  bfloat16 = PyObject_GetAttrString(torch, "bfloat16");
  Py_DECREF(torch);
  if (!bfloat16) return NULL;
  return PyModule_Create(&module);
}
