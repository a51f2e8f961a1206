/* Calls of libbitdecode.so from Python without ctypes' conversion of every argument: the cache classes' steps and prefills.
 *
 * A step of a short context is bound by what the host does for it.  On a slow core KVCache.decode_step without the library's
 * own work 7.5 -> 2.7 us, PagedKVCache.quant_pack_kv 4.9 -> 2.7; issued one by one 8 paged prompts of up to 1333 tokens 43.7 ->
 * 39.7 us, a step of 6K tokens 9.3 -> 8.1.  Functions get the address of the library's entry point first (the library stays the one that
 * ctypes has loaded), a bd_cache / bd_paged_cache next (read through the buffer protocol), tensors as they are (their
 * data_ptr(); None is NULL), and return what the entry point returns.  As with ctypes, the interpreter's lock is released
 * during the call and integers are taken modulo 2^32.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "bitdecode.h"

static PyObject *name_data_ptr, *name_shape, *name_stride, *name_dtype, *name_get_device;

/* Address of a tensor's data, NULL for None; -1 with an exception set. */
static int tensor_address(PyObject* t, void** p) {
  *p = NULL;
  if (t == Py_None) return 0;
  PyObject* n = PyObject_CallMethodNoArgs(t, name_data_ptr);
  if (!n) return -1;
  *p = PyLong_AsVoidPtr(n);
  Py_DECREF(n);
  return !*p && PyErr_Occurred() ? -1 : 0;
}
static int address(PyObject* o, void** p) {
  *p = o == Py_None ? NULL : PyLong_AsVoidPtr(o);
  return !*p && PyErr_Occurred() ? -1 : 0;
}
static int int32_of(PyObject* o, int32_t* v) {
  const unsigned long n = PyLong_AsUnsignedLongMask(o);
  *v = (int32_t)(uint32_t)n;
  return n == (unsigned long)-1 && PyErr_Occurred() ? -1 : 0;
}
static int float_of(PyObject* o, float* v) {
  const double x = PyFloat_AsDouble(o);
  *v = (float)x;
  return x == -1.0 && PyErr_Occurred() ? -1 : 0;
}
/* A ctypes structure, which the caller's frame keeps alive. */
static int structure(PyObject* o, Py_buffer* b) { return PyObject_GetBuffer(o, b, PyBUF_SIMPLE); }
static int count_is(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return 1;
  PyErr_Format(PyExc_TypeError, "%zd arguments for %zd", n, want);
  return 0;
}

/* splits(fn, cache, packed_len) -> count   (bd_choose_splits, bd_step_splits) */
static PyObject* splits(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* fn;
  int32_t len, count;
  Py_buffer c;
  (void)self;
  if (!count_is(n, 3) || address(a[0], &fn) || int32_of(a[2], &len) || structure(a[1], &c)) return NULL;
  count = ((int32_t(*)(const void*, int32_t))fn)(c.buf, len);
  PyBuffer_Release(&c);
  return PyLong_FromLong(count);
}

/* step(fn, cache, k_new, v_new, q, packed_len, res_len, scale, num_splits, workspace, out, stream)
 *   -> (status, packed_len, res_len)   (bd_decode_step, bd_decode_step_lazy) */
static PyObject* step(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *fn, *k, *v, *q, *ws, *out, *stream;
  int32_t packed, res, ns;
  float scale;
  int status;
  Py_buffer c;
  (void)self;
  if (!count_is(n, 12) || address(a[0], &fn) || tensor_address(a[2], &k) || tensor_address(a[3], &v) || tensor_address(a[4], &q) ||
      int32_of(a[5], &packed) || int32_of(a[6], &res) || float_of(a[7], &scale) || int32_of(a[8], &ns) ||
      tensor_address(a[9], &ws) || tensor_address(a[10], &out) || address(a[11], &stream) || structure(a[1], &c))
    return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = ((int (*)(const void*, const void*, const void*, const void*, int32_t*, int32_t*, float, int32_t, void*, void*,
                     void*))fn)(c.buf, k, v, q, &packed, &res, scale, ns, ws, out, stream);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&c);
  return Py_BuildValue("(iii)", status, (int)packed, (int)res);
}

/* paged_step(fn, cache, k_new, v_new, q, scale, num_splits, workspace, out, stream) -> status
 *   (bd_paged_decode_step, bd_paged_counted_step and their lazy forms) */
static PyObject* paged_step(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *fn, *k, *v, *q, *ws, *out, *stream;
  int32_t ns;
  float scale;
  int status;
  Py_buffer c;
  (void)self;
  if (!count_is(n, 10) || address(a[0], &fn) || tensor_address(a[2], &k) || tensor_address(a[3], &v) || tensor_address(a[4], &q) ||
      float_of(a[5], &scale) || int32_of(a[6], &ns) || tensor_address(a[7], &ws) || tensor_address(a[8], &out) ||
      address(a[9], &stream) || structure(a[1], &c))
    return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = ((int (*)(const void*, const void*, const void*, const void*, float, int32_t, void*, void*, void*))fn)(
      c.buf, k, v, q, scale, ns, ws, out, stream);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&c);
  return PyLong_FromLong(status);
}

/* paged_quant(fn, cache, seq, k, v, L, stream) -> status   (bd_paged_quant_pack_kv) */
static PyObject* paged_quant(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *fn, *k, *v, *stream;
  int32_t seq, len;
  int status;
  Py_buffer c;
  (void)self;
  if (!count_is(n, 7) || address(a[0], &fn) || int32_of(a[2], &seq) || tensor_address(a[3], &k) || tensor_address(a[4], &v) ||
      int32_of(a[5], &len) || address(a[6], &stream) || structure(a[1], &c))
    return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = ((int (*)(const void*, int32_t, const void*, const void*, int32_t, void*))fn)(c.buf, seq, k, v, len, stream);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&c);
  return PyLong_FromLong(status);
}

/* quant(fn, cache, k, v, L, stream) -> (status, packed_len, res_len)   (bd_quant_pack_kv) */
static PyObject* quant(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *fn, *k, *v, *stream;
  int32_t len, packed = 0, res = 0;
  int status;
  Py_buffer c;
  (void)self;
  if (!count_is(n, 6) || address(a[0], &fn) || tensor_address(a[2], &k) || tensor_address(a[3], &v) || int32_of(a[4], &len) ||
      address(a[5], &stream) || structure(a[1], &c))
    return NULL;
  Py_BEGIN_ALLOW_THREADS
  status = ((int (*)(const void*, const void*, const void*, int32_t, int32_t*, int32_t*, void*))fn)(c.buf, k, v, len, &packed, &res,
                                                                                                    stream);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&c);
  return Py_BuildValue("(iii)", status, (int)packed, (int)res);
}

/* ---- Paged cache in 8 bits.  These check the tensors too: in Python that took longer than all the rest of a call. ---- */

/* PagedKV8Cache._layout: (batch, query heads, KV heads, head_dim, dtype, int32, float32, number of the device, text for the device). */
typedef struct {
  long batch, q_heads, kv_heads, dim, device;
  PyObject *dtype, *int32, *float32, *where;
} layout8;
static int layout_of(PyObject* o, layout8* l) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 9) {
    PyErr_SetString(PyExc_TypeError, "layout");
    return -1;
  }
  l->batch = PyLong_AsLong(PyTuple_GET_ITEM(o, 0));
  l->q_heads = PyLong_AsLong(PyTuple_GET_ITEM(o, 1));
  l->kv_heads = PyLong_AsLong(PyTuple_GET_ITEM(o, 2));
  l->dim = PyLong_AsLong(PyTuple_GET_ITEM(o, 3));
  l->dtype = PyTuple_GET_ITEM(o, 4);
  l->int32 = PyTuple_GET_ITEM(o, 5);
  l->float32 = PyTuple_GET_ITEM(o, 6);
  l->device = PyLong_AsLong(PyTuple_GET_ITEM(o, 7));
  l->where = PyTuple_GET_ITEM(o, 8);
  return PyErr_Occurred() ? -1 : 0;
}
/* Up to 3 sizes and strides of a tensor of `dims` dimensions, of the given type on the given device: 1; 0 if it is another; -1 error. */
static int tensor_is(PyObject* t, int dims, PyObject* dtype, long device, long* size, long* stride) {
  PyObject *shape = NULL, *strides = NULL, *type = NULL, *dev = NULL;
  int ok = -1;
  if (!(shape = PyObject_GetAttr(t, name_shape)) || !(strides = PyObject_CallMethodNoArgs(t, name_stride)) ||
      !(type = PyObject_GetAttr(t, name_dtype)) || !(dev = PyObject_CallMethodNoArgs(t, name_get_device)))
    goto out;
  ok = 0;
  if (!PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) != dims || !PyTuple_Check(strides) || PyTuple_GET_SIZE(strides) != dims || type != dtype ||
      PyLong_AsLong(dev) != device)
    goto out;
  for (int i = 0; i < dims; ++i) {
    size[i] = PyLong_AsLong(PyTuple_GET_ITEM(shape, i));
    stride[i] = PyLong_AsLong(PyTuple_GET_ITEM(strides, i));
  }
  ok = 1;
out:
  Py_XDECREF(shape);
  Py_XDECREF(strides);
  Py_XDECREF(type);
  Py_XDECREF(dev);
  return PyErr_Occurred() ? -1 : ok;
}
/* A step's tensor [rows][heads][channels]; *rows -1: whatever it has. */
static int rows_of(PyObject* t, const layout8* l, long heads, int contiguous, const char* what, bd_rows* r, long* rows) {
  long size[3], stride[3];
  void* p;
  const int ok = tensor_is(t, 3, l->dtype, l->device, size, stride);
  if (ok < 0) return -1;
  if (!ok || size[1] != heads || size[2] != l->dim || stride[2] != 1 || (*rows >= 0 && size[0] != *rows) ||
      (contiguous && ((heads > 1 && stride[1] != l->dim) || (size[0] > 1 && stride[0] != heads * l->dim)))) {
    if (*rows >= 0)
      PyErr_Format(PyExc_ValueError, "%s: a %S tensor [%ld][%ld][%ld] on %S, %s", what, l->dtype, *rows, heads, l->dim, l->where,
                   contiguous ? "contiguous" : "channels adjacent");
    else
      PyErr_Format(PyExc_ValueError, "%s: a %S tensor [rows][%ld][%ld] on %S, channels adjacent", what, l->dtype, heads, l->dim, l->where);
    return -1;
  }
  if (tensor_address(t, &p)) return -1;
  r->data = p;
  r->token_stride = stride[0];
  r->head_stride = stride[1];
  *rows = size[0];
  return 0;
}
/* A list of n numbers, or None. */
static int list_of(PyObject* t, const layout8* l, long n, PyObject* dtype, const char* what, void** p) {
  long size, stride;
  int ok;
  *p = NULL;
  if (t == Py_None) return 0;
  ok = tensor_is(t, 1, dtype, l->device, &size, &stride);
  if (ok < 0) return -1;
  if (!ok || size != n || (n > 1 && stride != 1)) {
    PyErr_Format(PyExc_ValueError, "%s: a contiguous %S tensor [%ld] on %S", what, dtype, n, l->where);
    return -1;
  }
  return tensor_address(t, p);
}

/* append8(fn, cache, layout, k_new, v_new, q, q_out, cu_tokens, max_tokens, rotation, positions, stream) -> status   (bd_paged8_append) */
static PyObject* append8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *fn, *cu, *positions, *stream;
  layout8 l;
  bd_rows k, v, q = {0}, q_out = {0};
  long rows = -1;
  int32_t most;
  int status, has_q;
  Py_buffer c, rot = {0};
  (void)self;
  if (!count_is(n, 12) || address(a[0], &fn) || layout_of(a[2], &l) || rows_of(a[3], &l, l.kv_heads, 0, "k_new", &k, &rows) ||
      rows_of(a[4], &l, l.kv_heads, 0, "v_new", &v, &rows))
    return NULL;
  has_q = a[5] != Py_None;
  if (has_q && a[6] == Py_None) {
    PyErr_SetString(PyExc_ValueError, "q needs q_out");
    return NULL;
  }
  if ((has_q && (rows_of(a[5], &l, l.q_heads, 0, "q", &q, &rows) || rows_of(a[6], &l, l.q_heads, 0, "q_out", &q_out, &rows))) ||
      list_of(a[7], &l, l.batch + 1, l.int32, "cu_tokens", &cu) || int32_of(a[8], &most) || list_of(a[10], &l, rows, l.int32, "positions", &positions) ||
      address(a[11], &stream) || (a[9] != Py_None && structure(a[9], &rot)))
    return NULL;
  if (structure(a[1], &c)) {
    if (rot.buf) PyBuffer_Release(&rot);
    return NULL;
  }
  Py_BEGIN_ALLOW_THREADS
  status = ((int (*)(const void*, const bd_rows*, const bd_rows*, const bd_rows*, const bd_rows*, const void*, int32_t, int32_t, const void*, void*))fn)(
      c.buf, &k, &v, has_q ? &q : NULL, has_q ? &q_out : NULL, cu, (int32_t)rows, most, rot.buf, stream);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&c);
  if (rot.buf) PyBuffer_Release(&rot);
  return PyLong_FromLong(status);
}

/* plan8(choose, bytes, cache, rows, max_tokens, max_len, num_splits) -> (num_splits, workspace bytes)
 *   (bd_paged8_choose_splits where num_splits is 0, bd_paged8_workspace_bytes) */
static PyObject* plan8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *choose, *bytes;
  int32_t rows, most, len, ns;
  size_t need;
  Py_buffer c;
  (void)self;
  if (!count_is(n, 7) || address(a[0], &choose) || address(a[1], &bytes) || int32_of(a[3], &rows) || int32_of(a[4], &most) ||
      int32_of(a[5], &len) || int32_of(a[6], &ns) || structure(a[2], &c))
    return NULL;
  if (!ns) ns = ((int32_t(*)(const void*, int32_t, int32_t))choose)(c.buf, most, len);
  need = ((size_t(*)(const void*, int32_t, int32_t, int32_t))bytes)(c.buf, rows, most, ns);
  PyBuffer_Release(&c);
  return Py_BuildValue("(in)", (int)ns, (Py_ssize_t)need);
}

/* attn8(fn, cache, layout, q, cu_tokens, max_tokens, scale, softcap, slopes, prefix_lens, window, num_splits, workspace, out, stream) -> status
 *   (bd_paged8_attn) */
static PyObject* attn8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *fn, *cu, *slopes, *prefix, *ws, *stream;
  layout8 l;
  bd_rows q, out;
  bd_scores s;
  long rows = -1;
  int32_t most, ns;
  int status;
  Py_buffer c;
  (void)self;
  if (!count_is(n, 15) || address(a[0], &fn) || layout_of(a[2], &l) || rows_of(a[3], &l, l.q_heads, 0, "q", &q, &rows) ||
      rows_of(a[13], &l, l.q_heads, 1, "out", &out, &rows) || list_of(a[4], &l, l.batch + 1, l.int32, "cu_tokens", &cu) || int32_of(a[5], &most) ||
      float_of(a[6], &s.softmax_scale) || float_of(a[7], &s.softcap) || list_of(a[8], &l, l.q_heads, l.float32, "slopes", &slopes) ||
      list_of(a[9], &l, l.batch, l.int32, "prefix_lens", &prefix) || int32_of(a[10], &s.window) || int32_of(a[11], &ns) || tensor_address(a[12], &ws) ||
      address(a[14], &stream) || structure(a[1], &c))
    return NULL;
  s.slopes = slopes;
  s.prefix_lens = prefix;
  Py_BEGIN_ALLOW_THREADS
  status = ((int (*)(const void*, const bd_rows*, const void*, int32_t, int32_t, const bd_scores*, int32_t, void*, void*, void*))fn)(
      c.buf, &q, cu, (int32_t)rows, most, &s, ns, ws, out.data, stream);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&c);
  return PyLong_FromLong(status);
}

static PyMethodDef methods[] = {
    {"splits", (PyCFunction)(void (*)(void))splits, METH_FASTCALL, NULL},
    {"step", (PyCFunction)(void (*)(void))step, METH_FASTCALL, NULL},
    {"paged_step", (PyCFunction)(void (*)(void))paged_step, METH_FASTCALL, NULL},
    {"paged_quant", (PyCFunction)(void (*)(void))paged_quant, METH_FASTCALL, NULL},
    {"quant", (PyCFunction)(void (*)(void))quant, METH_FASTCALL, NULL},
    {"append8", (PyCFunction)(void (*)(void))append8, METH_FASTCALL, NULL},
    {"plan8", (PyCFunction)(void (*)(void))plan8, METH_FASTCALL, NULL},
    {"attn8", (PyCFunction)(void (*)(void))attn8, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bdcall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__bdcall(void) {
  name_data_ptr = PyUnicode_InternFromString("data_ptr");
  name_shape = PyUnicode_InternFromString("shape");
  name_stride = PyUnicode_InternFromString("stride");
  name_dtype = PyUnicode_InternFromString("dtype");
  name_get_device = PyUnicode_InternFromString("get_device");
  return name_data_ptr && name_shape && name_stride && name_dtype && name_get_device ? PyModule_Create(&module) : NULL;
}
