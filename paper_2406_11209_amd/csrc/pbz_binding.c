/* The calls of the Python binding that programs make over and over: tensors in, one C entry point called on torch's current stream.
 *
 * What it spares is the interpreter's share of a small call: with ctypes an operation on a 256 x 256 image took 4.4 (negate) to
 * 7.8 us (decompress) of host time, of which the entry point and its launch are some 3; now 3.7 to 5.1, and eleven of them in a row 51 us
 * instead of 68.  Nothing of torch's or of the library's
 * is linked: a tensor is asked for its address by the methods that Python code would use, and the entry points come as
 * addresses, so that several builds of the library can be loaded.  The interpreter lock is released around the entry point.
 *
 * Every function returns the entry point's status; -1000 never is one.  A tensor that is not a contiguous one on the device is
 * refused with ValueError before anything is called. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "pbz_cache.h"

static PyObject *s_is_cuda, *s_is_contiguous, *s_data_ptr, *s_shape, *s_get_device, *s_device, *s_dtype, *s_stride;
static PyObject *get_device, *get_stream; /* of torch */

static int address_of(PyObject *t, void **out) {
  int cuda, contiguous;
  PyObject *v = PyObject_GetAttr(t, s_is_cuda);
  if (!v) return -1;
  cuda = PyObject_IsTrue(v);
  Py_DECREF(v);
  if (cuda < 0) return -1;
  contiguous = 0;
  if (cuda) {
    v = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (!v) return -1;
    contiguous = PyObject_IsTrue(v);
    Py_DECREF(v);
    if (contiguous < 0) return -1;
  }
  if (!contiguous) {
    PyErr_SetString(PyExc_ValueError, "pbz takes contiguous device tensors");
    return -1;
  }
  v = PyObject_CallMethodNoArgs(t, s_data_ptr);
  if (!v) return -1;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return *out == NULL && PyErr_Occurred() ? -1 : 0;
}

static int optional_address_of(PyObject *t, void **out) {
  *out = NULL;
  return t == Py_None ? 0 : address_of(t, out);
}

/* t.shape[0] */
static int blocks_of(PyObject *t, int64_t *n) {
  PyObject *shape = PyObject_GetAttr(t, s_shape), *first;
  if (!shape) return -1;
  first = PySequence_GetItem(shape, 0);
  Py_DECREF(shape);
  if (!first) return -1;
  *n = PyLong_AsLongLong(first);
  Py_DECREF(first);
  return *n == -1 && PyErr_Occurred() ? -1 : 0;
}

/* torch's current stream on the current device; its number as an object, too, where the caller asks for that */
static int current_stream_object(void **out, PyObject **object) {
  PyObject *device, *stream;
  if (!get_device) {
    PyObject *c = PyImport_ImportModule("torch._C"), *d = NULL, *s = NULL;
    if (!c) return -1;
    d = PyObject_GetAttrString(c, "_cuda_getDevice");
    s = d ? PyObject_GetAttrString(c, "_cuda_getCurrentRawStream") : NULL;
    Py_DECREF(c);
    if (!s) {
      Py_XDECREF(d);
      return -1;
    }
    get_stream = s;
    get_device = d;
  }
  device = PyObject_CallNoArgs(get_device);
  if (!device) return -1;
  stream = PyObject_CallOneArg(get_stream, device);
  Py_DECREF(device);
  if (!stream) return -1;
  *out = PyLong_AsVoidPtr(stream);
  if (*out == NULL && PyErr_Occurred()) {
    Py_DECREF(stream);
    return -1;
  }
  if (object) *object = stream;
  else Py_DECREF(stream);
  return 0;
}

static int current_stream(void **out) { return current_stream_object(out, NULL); }

/* spaces[(device of t, stream)] = (address, bytes): 1, and 0 where there is none yet */
static int space_of(PyObject *spaces, PyObject *t, PyObject *stream, void **ws, size_t *bytes) {
  PyObject *device = PyObject_CallMethodNoArgs(t, s_get_device), *key, *space;
  if (!device) return -1;
  key = PyTuple_Pack(2, device, stream);
  Py_DECREF(device);
  if (!key) return -1;
  space = PyDict_GetItemWithError(spaces, key); /* borrowed; spaces keeps it while the lock is held */
  Py_DECREF(key);
  if (!space) return PyErr_Occurred() ? -1 : 0;
  *ws = PyLong_AsVoidPtr(PyTuple_GET_ITEM(space, 0));
  *bytes = PyLong_AsSize_t(PyTuple_GET_ITEM(space, 1));
  return PyErr_Occurred() ? -1 : 1;
}

static int expect(Py_ssize_t got, Py_ssize_t least, Py_ssize_t most) {
  if (got >= least && got <= most) return 0;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return -1;
}

static int as_pointer(PyObject *v, void **out) {
  *out = PyLong_AsVoidPtr(v);
  return *out == NULL && PyErr_Occurred() ? -1 : 0;
}

#define CALL(expression)                 \
  do {                                   \
    Py_BEGIN_ALLOW_THREADS               \
    status = (expression);               \
    Py_END_ALLOW_THREADS                 \
  } while (0)

enum { kMaxTensors = 6 };

/* blocks(entry, codec, tensor whose first extent is the number of blocks, tensors...):
 * entry(codec, blocks, addresses..., stream) */
static PyObject *blocks(PyObject *self, PyObject *const *args, Py_ssize_t n) {
  void *fn, *codec, *p[kMaxTensors], *s;
  int64_t k;
  int status = -1000;
  const int count = (int)n - 3;
  (void)self;
  if (expect(n, 5, 3 + kMaxTensors) || as_pointer(args[0], &fn) || as_pointer(args[1], &codec) || blocks_of(args[2], &k)) return NULL;
  for (int i = 0; i < count; ++i)
    if (address_of(args[3 + i], p + i)) return NULL;
  if (current_stream(&s)) return NULL;
  switch (count) {
    case 2: CALL(((int (*)(void *, int64_t, void *, void *, void *))fn)(codec, k, p[0], p[1], s)); break;
    case 3: CALL(((int (*)(void *, int64_t, void *, void *, void *, void *))fn)(codec, k, p[0], p[1], p[2], s)); break;
    case 5:
      CALL(((int (*)(void *, int64_t, void *, void *, void *, void *, void *, void *))fn)(codec, k, p[0], p[1], p[2], p[3], p[4], s));
      break;
    case 6:
      CALL(((int (*)(void *, int64_t, void *, void *, void *, void *, void *, void *, void *))fn)(codec, k, p[0], p[1], p[2], p[3], p[4],
                                                                                                  p[5], s));
      break;
    default: PyErr_SetString(PyExc_TypeError, "no entry point takes that many tensors"); return NULL;
  }
  return PyLong_FromLong(status);
}

/* reduce(entry, codec, workspaces by device and stream, tensor whose first extent is the number of blocks, tensors...):
 * entry(codec, blocks, addresses..., workspace, bytes, stream); None where the first tensor's device and the stream have no workspace */
static PyObject *reduce(PyObject *self, PyObject *const *args, Py_ssize_t n) {
  void *fn, *codec, *ws, *p[5], *s;
  PyObject *stream;
  int64_t k;
  size_t bytes;
  int status = -1000, found;
  const int count = (int)n - 4;
  (void)self;
  if (expect(n, 7, 9) || as_pointer(args[0], &fn) || as_pointer(args[1], &codec) || blocks_of(args[3], &k)) return NULL;
  for (int i = 0; i < count; ++i)
    if (address_of(args[4 + i], p + i)) return NULL;
  if (current_stream_object(&s, &stream)) return NULL;
  found = space_of(args[2], args[4], stream, &ws, &bytes);
  Py_DECREF(stream);
  if (found < 0) return NULL;
  if (!found) Py_RETURN_NONE;
  switch (count) {
    case 3:
      CALL(((int (*)(void *, int64_t, void *, void *, void *, void *, size_t, void *))fn)(codec, k, p[0], p[1], p[2], ws, bytes, s));
      break;
    case 5:
      CALL(((int (*)(void *, int64_t, void *, void *, void *, void *, void *, void *, size_t, void *))fn)(codec, k, p[0], p[1], p[2], p[3],
                                                                                                        p[4], ws, bytes, s));
      break;
    default: PyErr_SetString(PyExc_TypeError, "no entry point takes that many tensors"); return NULL;
  }
  return PyLong_FromLong(status);
}

/* scalar(entry, codec, x, N, F, N_out, F_out): entry(codec, blocks of F, N, F, x, N_out, F_out, stream) */
static PyObject *scalar(PyObject *self, PyObject *const *args, Py_ssize_t n) {
  void *fn, *codec, *p[4], *s;
  int64_t k;
  int status = -1000;
  double x;
  (void)self;
  if (expect(n, 7, 7) || as_pointer(args[0], &fn) || as_pointer(args[1], &codec)) return NULL;
  x = PyFloat_AsDouble(args[2]);
  if (x == -1.0 && PyErr_Occurred()) return NULL;
  if (blocks_of(args[4], &k)) return NULL;
  for (int i = 0; i < 4; ++i)
    if (address_of(args[3 + i], p + i)) return NULL;
  if (current_stream(&s)) return NULL;
  CALL(((int (*)(void *, int64_t, void *, void *, double, void *, void *, void *))fn)(codec, k, p[0], p[1], x, p[2], p[3], s));
  return PyLong_FromLong(status);
}

/* compress(entry, codec, x, type of x, buffer of its extents, N, F): entry(codec, x, type, extents, N, F, stream) */
static PyObject *compress(PyObject *self, PyObject *const *args, Py_ssize_t n) {
  void *fn, *codec, *x, *N, *F, *s;
  Py_buffer shape;
  long type;
  int status = -1000;
  (void)self;
  if (expect(n, 7, 7) || as_pointer(args[0], &fn) || as_pointer(args[1], &codec) || address_of(args[2], &x)) return NULL;
  type = PyLong_AsLong(args[3]);
  if (type == -1 && PyErr_Occurred()) return NULL;
  if (address_of(args[5], &N) || address_of(args[6], &F) || current_stream(&s)) return NULL;
  if (PyObject_GetBuffer(args[4], &shape, PyBUF_SIMPLE)) return NULL;
  CALL(((int (*)(void *, void *, int, void *, void *, void *, void *))fn)(codec, x, (int)type, shape.buf, N, F, s));
  PyBuffer_Release(&shape);
  return PyLong_FromLong(status);
}

/* decompress(entry, codec, N, F, buffer of the extents, y, type of y): entry(codec, N, F, extents, y, type, stream) */
static PyObject *decompress(PyObject *self, PyObject *const *args, Py_ssize_t n) {
  void *fn, *codec, *y, *N, *F, *s;
  Py_buffer shape;
  long type;
  int status = -1000;
  (void)self;
  if (expect(n, 7, 7) || as_pointer(args[0], &fn) || as_pointer(args[1], &codec) || address_of(args[2], &N) || address_of(args[3], &F) ||
      address_of(args[5], &y))
    return NULL;
  type = PyLong_AsLong(args[6]);
  if (type == -1 && PyErr_Occurred()) return NULL;
  if (current_stream(&s)) return NULL;
  if (PyObject_GetBuffer(args[4], &shape, PyBUF_SIMPLE)) return NULL;
  CALL(((int (*)(void *, void *, void *, void *, void *, int, void *))fn)(codec, N, F, shape.buf, y, (int)type, s));
  PyBuffer_Release(&shape);
  return PyLong_FromLong(status);
}

/* segmented(entry, codec, workspaces, statistic, segments, blocks per segment, N1, F1, N2 or None, F2 or None, out): as reduce */
static PyObject *segmented(PyObject *self, PyObject *const *args, Py_ssize_t n) {
  void *fn, *codec, *ws, *p[5], *s;
  PyObject *stream;
  long what;
  int64_t segments, per;
  size_t bytes;
  int status = -1000, found;
  (void)self;
  if (expect(n, 11, 11) || as_pointer(args[0], &fn) || as_pointer(args[1], &codec)) return NULL;
  what = PyLong_AsLong(args[3]);
  segments = PyLong_AsLongLong(args[4]);
  per = PyLong_AsLongLong(args[5]);
  if ((what == -1 || segments == -1 || per == -1) && PyErr_Occurred()) return NULL;
  if (address_of(args[6], p) || address_of(args[7], p + 1) || optional_address_of(args[8], p + 2) || optional_address_of(args[9], p + 3) ||
      address_of(args[10], p + 4) || current_stream_object(&s, &stream))
    return NULL;
  found = space_of(args[2], args[6], stream, &ws, &bytes);
  Py_DECREF(stream);
  if (found < 0) return NULL;
  if (!found) Py_RETURN_NONE;
  CALL(((int (*)(void *, int, int64_t, int64_t, void *, void *, void *, void *, void *, void *, size_t, void *))fn)(
      codec, (int)what, segments, per, p[0], p[1], p[2], p[3], p[4], ws, bytes, s));
  return PyLong_FromLong(status);
}

/* ---- the paged compressed cache (paper_2406_11209_amd/cache.py): an append took 6.3 us of host time with ctypes, an attention call of two launches 11.7,
 * a copy of a few pages 5.1; now 4.0, 9.5 and 3.5 ---- */

/* What a cache's tensors are held against: PyTuple (device, int32, int64, float32, heads, head_dim) */
enum { kDevice, kInt32, kInt64, kFloat32, kHeads, kDim, kOfCache };

static int int_of(PyObject *sequence, Py_ssize_t i, int64_t *out) {
  PyObject *v = PySequence_GetItem(sequence, i);
  if (!v) return -1;
  *out = PyLong_AsLongLong(v);
  Py_DECREF(v);
  return *out == -1 && PyErr_Occurred() ? -1 : 0;
}

static int pointer_of(PyObject *t, void **out) {
  PyObject *v = PyObject_CallMethodNoArgs(t, s_data_ptr);
  int status;
  if (!v) return -1;
  status = as_pointer(v, out);
  Py_DECREF(v);
  return status;
}

/* extents of t, at most four; how many, or -1 */
static Py_ssize_t extents_of(PyObject *t, int64_t *out) {
  PyObject *shape = PyObject_GetAttr(t, s_shape);
  Py_ssize_t n, i;
  if (!shape) return -1;
  n = PySequence_Size(shape);
  for (i = 0; i < n && i < 4; ++i)
    if (int_of(shape, i, out + i)) n = -1;
  Py_DECREF(shape);
  return n;
}

static int strides_of(PyObject *t, Py_ssize_t n, int64_t *out) {
  PyObject *strides = PyObject_CallMethodNoArgs(t, s_stride);
  Py_ssize_t i;
  int status = 0;
  if (!strides) return -1;
  for (i = 0; i < n && !status; ++i) status = int_of(strides, i, out + i);
  Py_DECREF(strides);
  return status;
}

static int on_device(PyObject *t, PyObject *of) {
  PyObject *device = PyObject_GetAttr(t, s_device);
  int same;
  if (!device) return -1;
  same = PyObject_RichCompareBool(device, PyTuple_GET_ITEM(of, kDevice), Py_EQ);
  Py_DECREF(device);
  return same;
}

static int has_type(PyObject *t, PyObject *type) {
  PyObject *dtype = PyObject_GetAttr(t, s_dtype);
  if (!dtype) return -1;
  Py_DECREF(dtype); /* a type outlives every tensor of it */
  return dtype == type;
}

static int refuse_shape(PyObject *t, const char *name, int64_t heads, int64_t dim) {
  PyObject *shape = PyObject_GetAttr(t, s_shape), *tuple = shape ? PySequence_Tuple(shape) : NULL;
  Py_XDECREF(shape);
  if (tuple) PyErr_Format(PyExc_ValueError, "%s has to be [tokens, %lld, %lld], not %R", name, (long long)heads, (long long)dim, tuple);
  Py_XDECREF(tuple);
  return -1;
}

/* Lines [tokens, heads, head_dim]: address, tokens, strides of tokens and heads.  *tokens and *heads: as they have to be, or -1. */
static int lines_of(PyObject *t, PyObject *of, const char *name, int64_t *tokens, int64_t *heads, pbz_lines *out) {
  int64_t extents[4] = {0, 0, 0, 0}, strides[3];
  const int64_t dim = PyLong_AsLongLong(PyTuple_GET_ITEM(of, kDim));
  const Py_ssize_t n = extents_of(t, extents);
  void *at;
  int same;
  if (n < 0) return -1;
  if (n != 3 || (*heads >= 0 && extents[1] != *heads) || extents[2] != dim || (*tokens >= 0 && extents[0] != *tokens))
    return refuse_shape(t, name, *heads >= 0 || n != 3 ? *heads : extents[1], dim);
  same = on_device(t, of);
  if (same < 0) return -1;
  if (!same) {
    PyErr_Format(PyExc_ValueError, "%s is not on the cache's device", name);
    return -1;
  }
  if (strides_of(t, 3, strides)) return -1;
  if (strides[2] != 1) {
    PyErr_Format(PyExc_ValueError, "%s's last dimension has to be contiguous", name);
    return -1;
  }
  if (pointer_of(t, &at)) return -1;
  *tokens = extents[0];
  *heads = extents[1];
  out->data = at;
  out->token_stride = strides[0];
  out->head_stride = strides[1];
  return 0;
}

/* A contiguous tensor of a type and of one extent or (second >= 0) two. */
static int indices_of(PyObject *t, PyObject *of, int type, const char *name, int64_t first, int64_t second, void **out) {
  int64_t extents[4] = {0, 0, 0, 0};
  const Py_ssize_t n = extents_of(t, extents);
  int right = has_type(t, PyTuple_GET_ITEM(of, type));
  if (n < 0 || right < 0) return -1;
  right = right && n == (second >= 0 ? 2 : 1) && extents[0] == first && (second < 0 || extents[1] == second);
  if (right) right = on_device(t, of);
  if (right > 0) {
    PyObject *v = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (!v) return -1;
    right = PyObject_IsTrue(v);
    Py_DECREF(v);
  }
  if (right < 0) return -1;
  if (!right) {
    if (second >= 0)
      PyErr_Format(PyExc_ValueError, "%s has to be a contiguous %R tensor of shape (%lld, %lld) on the cache's device", name,
                   PyTuple_GET_ITEM(of, type), (long long)first, (long long)second);
    else
      PyErr_Format(PyExc_ValueError, "%s has to be a contiguous %R tensor of shape (%lld,) on the cache's device", name, PyTuple_GET_ITEM(of, type),
                   (long long)first);
    return -1;
  }
  return pointer_of(t, out);
}

/* cache_append(entry, codec, cache, what its tensors are held against, type of k and v, k, v, slots) */
static PyObject *cache_append(PyObject *self, PyObject *const *args, Py_ssize_t n) {
  void *fn, *codec, *cache, *slots, *s;
  int64_t tokens = -1, heads;
  pbz_lines k, v;
  long type;
  int status = -1000;
  (void)self;
  if (expect(n, 8, 8) || as_pointer(args[0], &fn) || as_pointer(args[1], &codec) || as_pointer(args[2], &cache)) return NULL;
  heads = PyLong_AsLongLong(PyTuple_GET_ITEM(args[3], kHeads));
  type = PyLong_AsLong(args[4]);
  if (PyErr_Occurred() || lines_of(args[5], args[3], "k", &tokens, &heads, &k) || lines_of(args[6], args[3], "v", &tokens, &heads, &v) ||
      indices_of(args[7], args[3], kInt64, "slots", tokens, -1, &slots))
    return NULL;
  if (tokens == 0) return PyLong_FromLong(0);
  if (current_stream(&s)) return NULL;
  CALL(((int (*)(void *, void *, int64_t, const pbz_lines *, const pbz_lines *, int, void *, void *))fn)(codec, cache, tokens, &k, &v, (int)type,
                                                                                                         slots, s));
  return PyLong_FromLong(status);
}

/* cache_copy(entry, codec, cache, buffer of pairs of int32) */
static PyObject *cache_copy(PyObject *self, PyObject *const *args, Py_ssize_t n) {
  void *fn, *codec, *cache, *s;
  Py_buffer pairs;
  int status = -1000;
  (void)self;
  if (expect(n, 4, 4) || as_pointer(args[0], &fn) || as_pointer(args[1], &codec) || as_pointer(args[2], &cache) || current_stream(&s)) return NULL;
  if (PyObject_GetBuffer(args[3], &pairs, PyBUF_SIMPLE)) return NULL;
  CALL(((int (*)(void *, void *, int64_t, void *, void *))fn)(codec, cache, pairs.len / 8, pairs.buf, s));
  PyBuffer_Release(&pairs);
  return PyLong_FromLong(status);
}

/* cache_attention(buffer of a pbz_attention, what a cache's tensors are held against, q, out, lse or None, starts or None, lengths, table): the tensors'
 * part of it. */
static PyObject *cache_attention(PyObject *self, PyObject *const *args, Py_ssize_t n) {
  int64_t tokens = -1, heads = -1, seqs[4] = {0, 0, 0, 0}, extents[4] = {0, 0, 0, 0}, strides[2];
  PyObject *of, *table;
  Py_buffer into;
  pbz_attention a;
  pbz_lines lines;
  void *at;
  Py_ssize_t dims;
  int right;
  (void)self;
  if (expect(n, 8, 8)) return NULL;
  of = args[1];
  table = args[7];
  memset(&a, 0, sizeof a);
  if (lines_of(args[2], of, "q", &tokens, &heads, &lines)) return NULL;
  a.q = lines.data;
  a.q_token_stride = lines.token_stride;
  a.q_head_stride = lines.head_stride;
  a.n_tokens = tokens;
  if (lines_of(args[3], of, "out", &tokens, &heads, &lines)) return NULL;
  a.out = (void *)lines.data;
  a.out_token_stride = lines.token_stride;
  a.out_head_stride = lines.head_stride;
  if (heads > INT32_MAX) {
    PyErr_SetString(PyExc_ValueError, "too many query heads");
    return NULL;
  }
  a.q_heads = (int32_t)heads;
  if (extents_of(args[6], seqs) < 0) return NULL;
  a.n_seqs = seqs[0];
  dims = extents_of(table, extents);
  right = dims < 0 ? -1 : has_type(table, PyTuple_GET_ITEM(of, kInt32));
  if (right > 0) right = dims == 2 && extents[0] == a.n_seqs ? on_device(table, of) : 0;
  if (right > 0) right = strides_of(table, 2, strides) ? -1 : extents[1] < 2 || strides[1] == 1;
  if (right < 0) return NULL;
  if (!right) {
    PyErr_Format(PyExc_ValueError, "table has to be an int32 tensor [%lld, pages] with contiguous rows on the cache's device", (long long)a.n_seqs);
    return NULL;
  }
  if (pointer_of(table, &at)) return NULL;
  a.table = at;
  a.table_stride = strides[0] > extents[1] ? strides[0] : extents[1];
  a.max_pages = extents[1];
  if (indices_of(args[6], of, kInt32, "lengths", a.n_seqs, -1, &at)) return NULL;
  a.lengths = at;
  if (args[5] != Py_None) {
    if (indices_of(args[5], of, kInt32, "starts", a.n_seqs + 1, -1, &at)) return NULL;
    a.starts = at;
  }
  if (args[4] != Py_None) {
    if (indices_of(args[4], of, kFloat32, "lse", tokens, heads, &at)) return NULL;
    a.lse = at;
  }
  if (PyObject_GetBuffer(args[0], &into, PyBUF_WRITABLE)) return NULL;
  if (into.len != (Py_ssize_t)sizeof a) {
    PyBuffer_Release(&into);
    PyErr_SetString(PyExc_TypeError, "not a pbz_attention");
    return NULL;
  }
  memcpy(into.buf, &a, sizeof a);
  PyBuffer_Release(&into);
  Py_RETURN_NONE;
}

/* cache_attend(entry, codec, cache, buffer of a pbz_attention, workspace, its bytes) */
static PyObject *cache_attend(PyObject *self, PyObject *const *args, Py_ssize_t n) {
  void *fn, *codec, *cache, *space, *s;
  size_t bytes;
  Py_buffer call;
  int status = -1000;
  (void)self;
  if (expect(n, 6, 6) || as_pointer(args[0], &fn) || as_pointer(args[1], &codec) || as_pointer(args[2], &cache) || address_of(args[4], &space))
    return NULL;
  bytes = PyLong_AsSize_t(args[5]);
  if (PyErr_Occurred() || current_stream(&s) || PyObject_GetBuffer(args[3], &call, PyBUF_SIMPLE)) return NULL;
  CALL(((int (*)(void *, void *, void *, void *, size_t, void *))fn)(codec, cache, call.buf, space, bytes, s));
  PyBuffer_Release(&call);
  return PyLong_FromLong(status);
}

static PyMethodDef methods[] = {{"blocks", (PyCFunction)(void (*)(void))blocks, METH_FASTCALL, NULL},
                                {"reduce", (PyCFunction)(void (*)(void))reduce, METH_FASTCALL, NULL},
                                {"scalar", (PyCFunction)(void (*)(void))scalar, METH_FASTCALL, NULL},
                                {"compress", (PyCFunction)(void (*)(void))compress, METH_FASTCALL, NULL},
                                {"decompress", (PyCFunction)(void (*)(void))decompress, METH_FASTCALL, NULL},
                                {"segmented", (PyCFunction)(void (*)(void))segmented, METH_FASTCALL, NULL},
                                {"cache_append", (PyCFunction)(void (*)(void))cache_append, METH_FASTCALL, NULL},
                                {"cache_copy", (PyCFunction)(void (*)(void))cache_copy, METH_FASTCALL, NULL},
                                {"cache_attention", (PyCFunction)(void (*)(void))cache_attention, METH_FASTCALL, NULL},
                                {"cache_attend", (PyCFunction)(void (*)(void))cache_attend, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__binding(void) {
  s_is_cuda = PyUnicode_InternFromString("is_cuda");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_shape = PyUnicode_InternFromString("shape");
  s_get_device = PyUnicode_InternFromString("get_device");
  s_device = PyUnicode_InternFromString("device");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_stride = PyUnicode_InternFromString("stride");
  if (!s_device || !s_dtype || !s_stride || !s_is_cuda || !s_is_contiguous || !s_data_ptr || !s_shape || !s_get_device) return NULL;
  return PyModule_Create(&module);
}
