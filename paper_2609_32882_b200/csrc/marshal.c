/* Argument marshalling of the calls between hidden states and attention, and of those of the residual stream, as a CPython module: tensors to the structs of vsa2.h and the library's function called,
 * nothing else.  A toy grid's calls wait for the host, and a view of a tensor costs the interpreter 0.6 us (norms and rotation: six of them), ctypes another
 * 0.7 us a call.  Tensors are used through their Python attributes, so the module needs no header of torch's.
 *
 * Every function returns the library's code; what cannot be marshalled raises ValueError. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <string.h>

#include "vsa2.h"

/* names, torch's types (bind), the library's functions (bind) */
static PyObject *n_shape, *n_stride, *n_dtype, *n_is_cuda, *n_data_ptr, *n_is_contiguous, *n_numel, *n_nbytes, *n_values, *n_scales, *n_get_device;
static PyObject *t_bf16, *t_f32, *t_i32, *t_e4m3, *t_u8, *t_i8, *t_i64, *stream_of, *device_of, *raw_stream;
static int (*f_rope_apply)(const vsa2_rope*, const vsa2_place*, const vsa2_heads*, const vsa2_heads*, int32_t, void*);
static int (*f_qkv_fwd)(const vsa2_rope*, const vsa2_place*, const vsa2_qk_norm*, const vsa2_heads*, const vsa2_heads*, void*);
static int (*f_qkv_bwd)(const vsa2_rope*, const vsa2_place*, const vsa2_qk_norm*, const vsa2_heads*, const vsa2_heads*, const vsa2_heads*, float*, float*, void*,
                        size_t, void*);
static int (*f_quantize)(const void*, int32_t, int32_t, int32_t, int64_t, int32_t, const vsa2_fp8*, const vsa2_fp8*, void*);
static int (*f_matmul)(int32_t, int32_t, int32_t, const vsa2_fp8*, const vsa2_fp8*, void*, int32_t, int64_t, void*, size_t, void*);
static int (*f_norm_fwd)(int32_t, int32_t, const vsa2_rows*, const vsa2_rows*, const vsa2_drop*, const float*, float, const vsa2_rows*, const vsa2_rows*,
                         const vsa2_fp8*, const vsa2_int8*, void*);
static int (*f_norm_bwd)(int32_t, int32_t, const vsa2_rows*, const vsa2_rows*, const vsa2_rows*, const vsa2_drop*, const float*, float, const vsa2_rows*,
                         const vsa2_rows*, float*, void*, size_t, void*);
static int (*f_dropout)(int32_t, int32_t, const vsa2_rows*, const vsa2_rows*, const vsa2_drop*, const vsa2_rows*, void*);
static int (*f_int8_quantize)(int32_t, int32_t, const vsa2_rows*, const vsa2_int8*, void*);
static int (*f_int8_matmul)(int32_t, int32_t, int32_t, const vsa2_int8*, const vsa2_int8*, const float*, void*, int32_t, int64_t, void*, size_t, void*);

static int refuse(const char* what) {
  PyErr_SetString(PyExc_ValueError, what);
  return -1;
}

/* ---- attributes of a tensor; each returns 0, or -1 with an exception */
static int integers(PyObject* tuple, int64_t* out, int most) { /* a tuple of at most `most` integers (stolen); their number */
  Py_ssize_t n;
  if (tuple == NULL) return -1;
  if (!PyTuple_Check(tuple) || (n = PyTuple_GET_SIZE(tuple)) > most) {
    Py_DECREF(tuple);
    return refuse("a tensor of fewer dimensions is expected");
  }
  for (Py_ssize_t i = 0; i < n; ++i) {
    out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, i));
    if (out[i] == -1 && PyErr_Occurred()) {
      Py_DECREF(tuple);
      return -1;
    }
  }
  Py_DECREF(tuple);
  return (int)n;
}
static int truth(PyObject* v) { /* of a new reference */
  int r;
  if (v == NULL) return -1;
  r = PyObject_IsTrue(v);
  Py_DECREF(v);
  return r;
}
static int number(PyObject* v, int64_t* out) {
  if (v == NULL) return -1;
  *out = PyLong_AsLongLong(v);
  Py_DECREF(v);
  return *out == -1 && PyErr_Occurred() ? -1 : 0;
}
static int address(PyObject* t, void** out) {
  PyObject* v = PyObject_CallMethodNoArgs(t, n_data_ptr);
  if (v == NULL) return -1;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return *out == NULL && PyErr_Occurred() ? -1 : 0;
}
static int is_type(PyObject* t, PyObject* type) {
  PyObject* v = PyObject_GetAttr(t, n_dtype);
  if (v == NULL) return -1;
  Py_DECREF(v); /* (torch's types live as long as torch) */
  return v == type;
}
static int on_gpu(PyObject* t, const char* otherwise) {
  const int r = truth(PyObject_GetAttr(t, n_is_cuda));
  return r < 0 ? -1 : r ? 0 : refuse(otherwise);
}
static int float_type(PyObject* t, int32_t* out) {
  PyObject* v = PyObject_GetAttr(t, n_dtype);
  if (v == NULL) return -1;
  Py_DECREF(v);
  if (v != t_bf16 && v != t_f32) return refuse("a tensor in bf16 or fp32 is expected");
  *out = v == t_f32 ? VSA2_F32 : VSA2_BF16;
  return 0;
}
static int fits_int(const int64_t* v, int n) {
  for (int i = 0; i < n; ++i)
    if (v[i] < 0 || v[i] > INT32_MAX) return refuse("a tensor's dimension does not fit 32 bits");
  return 0;
}

/* [batch, heads, tokens, channels], any strides but 1 for the channels */
static int get_view(PyObject* t, vsa2_heads* v) {
  int64_t shape[4], stride[4];
  const int n = integers(PyObject_GetAttr(t, n_shape), shape, 4);
  if (n < 0) return -1;
  if (n != 4) return refuse("expected a CUDA tensor [batch, heads, tokens, channels]");
  if (on_gpu(t, "expected a CUDA tensor [batch, heads, tokens, channels]") || integers(PyObject_CallMethodNoArgs(t, n_stride), stride, 4) != 4) return -1;
  if (stride[3] != 1) return refuse("the channels of a row must be contiguous");
  if (fits_int(shape, 4) || address(t, &v->data) || float_type(t, &v->dtype)) return -1;
  v->batch_stride = stride[0]; v->head_stride = stride[1]; v->token_stride = stride[2];
  v->batch = (int32_t)shape[0]; v->heads = (int32_t)shape[1]; v->tokens = (int32_t)shape[2]; v->channels = (int32_t)shape[3];
  v->reserved = 0;
  return 0;
}
/* the first n members of a sequence; a None among them is a view without heads, of the others' shape (of `otherwise`'s where all are None; may be null) */
static int get_views(PyObject* sequence, vsa2_heads* v, int n, const vsa2_heads* otherwise) {
  int given = 0, result = -1;
  vsa2_heads like;
  PyObject* fast = PySequence_Fast(sequence, "a sequence of tensors is expected");
  if (fast == NULL) return -1;
  if (PySequence_Fast_GET_SIZE(fast) < n) {
    refuse("a sequence of (q, k, v) is expected");
    goto out;
  }
  for (int i = 0; i < n; ++i) {
    PyObject* t = PySequence_Fast_GET_ITEM(fast, i);
    if (t == Py_None) continue;
    if (get_view(t, &v[i])) goto out;
    if (!given) like = v[i];
    given = 1;
  }
  if (!given) {
    if (otherwise == NULL) {
      refuse("no tensor is given");
      goto out;
    }
    like = *otherwise;
  }
  for (int i = 0; i < n; ++i) {
    if (PySequence_Fast_GET_ITEM(fast, i) != Py_None) continue;
    memset(&v[i], 0, sizeof v[i]);
    v[i].batch = like.batch; v[i].tokens = like.tokens; v[i].channels = like.channels; v[i].dtype = like.dtype;
  }
  result = 0;
out:
  Py_DECREF(fast);
  return result;
}
/* a contiguous CUDA tensor's address, None: null; `bytes`: its size (may be null) */
static int get_memory(PyObject* t, void** out, size_t* bytes) {
  *out = NULL;
  if (bytes != NULL) *bytes = 0;
  if (t == Py_None) return 0;
  if (on_gpu(t, "expected a CUDA tensor")) return -1;
  const int whole = truth(PyObject_CallMethodNoArgs(t, n_is_contiguous));
  if (whole < 0) return -1;
  if (!whole) return refuse("tensors must be contiguous");
  if (bytes != NULL) {
    int64_t n;
    if (number(PyObject_GetAttr(t, n_nbytes), &n)) return -1;
    *bytes = (size_t)n;
  }
  return address(t, out);
}
static int get_weight(PyObject* t, int channels, void** out) {
  *out = NULL;
  if (t == Py_None) return 0;
  int64_t n;
  const int f32 = is_type(t, t_f32);
  if (f32 < 0 || number(PyObject_CallMethodNoArgs(t, n_numel), &n)) return -1;
  if (!f32 || n != channels) return refuse("a norm's weight, or its gradient, must be fp32 with one element a channel");
  return get_memory(t, out, NULL);
}
static int get_place(PyObject* grid, PyObject* first, PyObject* positions, const vsa2_heads* like, vsa2_place* p) {
  memset(p, 0, sizeof *p);
  int64_t v[4];
  if (number(Py_NewRef(first), &v[0])) return -1;
  if (v[0] < INT32_MIN || v[0] > INT32_MAX) return refuse("first does not fit 32 bits");
  p->first = (int32_t)v[0];
  if (positions != Py_None) {
    const int i32 = is_type(positions, t_i32);
    if (i32 < 0) return -1;
    if (!i32) return refuse("positions must be a contiguous CUDA int32 tensor [batch, tokens, 3] or [tokens, 3]");
    void* at;
    if (get_memory(positions, &at, NULL)) return -1;
    const int n = integers(PyObject_GetAttr(positions, n_shape), v, 3);
    if (n < 0) return -1;
    const int batches = n == 3 && (v[0] == like->batch || v[0] == 1);
    if (!(n == 2 && v[0] == like->tokens && v[1] == 3) && !(batches && v[1] == like->tokens && v[2] == 3))
      return refuse("positions do not fit the tokens: [batch, tokens, 3], [1, tokens, 3] or [tokens, 3] is expected");
    p->positions = (const int32_t*)at;
    p->positions_batch_stride = n == 3 && v[0] > 1 ? 3 * (int64_t)like->tokens : 0;
    return 0;
  }
  if (grid != Py_None) {
    int32_t* to[3] = {&p->grid_t, &p->grid_h, &p->grid_w};
    PyObject* fast = PySequence_Fast(grid, "grid is (t, h, w)");
    if (fast == NULL) return -1;
    int bad = PySequence_Fast_GET_SIZE(fast) != 3 ? refuse("grid is (t, h, w)") : 0;
    for (int i = 0; i < 3 && !bad; ++i) {
      bad = number(Py_NewRef(PySequence_Fast_GET_ITEM(fast, i)), &v[i]);
      if (!bad && (v[i] < INT32_MIN || v[i] > INT32_MAX)) bad = refuse("grid does not fit 32 bits");
      if (!bad) *to[i] = (int32_t)v[i];
    }
    Py_DECREF(fast);
    return bad;
  }
  return 0;
}
static int get_rope(PyObject* o, vsa2_rope* r, const vsa2_rope** out) { /* vsa2_rope as any object with its bytes; None: none */
  *out = NULL;
  if (o == Py_None) return 0;
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE)) return -1;
  const int fits = b.len == (Py_ssize_t)sizeof *r;
  if (fits) memcpy(r, b.buf, sizeof *r);
  PyBuffer_Release(&b);
  if (!fits) return refuse("rope is what vsa2_rope_plan returns");
  *out = r;
  return 0;
}
static int get_norm(PyObject* on, PyObject* eps, PyObject* qw, PyObject* kw, int channels, vsa2_qk_norm* norm, const vsa2_qk_norm** out) {
  void *q, *k;
  const int wanted = PyObject_IsTrue(on);
  *out = NULL;
  if (wanted < 0) return -1;
  if (!wanted) return 0;
  const double e = PyFloat_AsDouble(eps);
  if ((e == -1.0 && PyErr_Occurred()) || get_weight(qw, channels, &q) || get_weight(kw, channels, &k)) return -1;
  norm->q_weight = (const float*)q; norm->k_weight = (const float*)k;
  norm->eps = (float)e;
  norm->reserved = 0;
  *out = norm;
  return 0;
}
/* values and scales of a matrix in 8-bit form, on any device: its shape and strides */
static int fp8_form(PyObject* values, PyObject* scales, int64_t* shape, int64_t* stride) {
  int64_t of[3];
  int rank, typed = is_type(values, t_e4m3);
  if (typed < 0 || (rank = integers(PyObject_GetAttr(values, n_shape), shape, 2)) < 0) return -1;
  if (rank == 2 && integers(PyObject_CallMethodNoArgs(values, n_stride), stride, 2) != 2) return -1;
  if (!typed || rank != 2 || (shape[1] > 1 && stride[1] != 1)) return refuse("values must be float8_e4m3fn [rows, cols] with contiguous rows");
  typed = is_type(scales, t_u8);
  if (typed < 0 || (rank = integers(PyObject_GetAttr(scales, n_shape), of, 3)) < 0) return -1;
  if (!typed || rank != 3 || of[0] != (shape[1] + 511) / 512 || of[1] != shape[0] || of[2] != 4)
    return refuse("scales must be uint8 [ceil(cols / 512), rows, 4]");
  return 0;
}
/* an Fp8 object; its shape.  (Its members may have been assigned, or resized, since it was made: they are looked at again at every call, 0.1 us.) */
static int get_fp8(PyObject* o, vsa2_fp8* v, int64_t* shape) {
  int bad = -1;
  int64_t stride[2];
  void* scales;
  PyObject *values = PyObject_GetAttr(o, n_values), *s = values != NULL ? PyObject_GetAttr(o, n_scales) : NULL;
  if (s == NULL || on_gpu(values, "expected a CUDA tensor") || fp8_form(values, s, shape, stride) || fits_int(shape, 2) || address(values, &v->values) ||
      get_memory(s, &scales, NULL))
    goto out;
  v->scales = (uint8_t*)scales;
  v->ld = shape[0] > 1 ? stride[0] : (shape[1] + 15) / 16 * 16;
  bad = 0;
out:
  Py_XDECREF(values);
  Py_XDECREF(s);
  return bad;
}
/* a CUDA matrix with contiguous rows */
static int get_matrix(PyObject* t, int64_t* shape, int64_t* ld, int32_t* type, void** data) {
  static const char* const what = "expected a CUDA matrix with contiguous rows";
  int64_t stride[2];
  const int n = integers(PyObject_GetAttr(t, n_shape), shape, 2);
  if (n < 0) return -1;
  if (n != 2) return refuse(what);
  if (on_gpu(t, what) || integers(PyObject_CallMethodNoArgs(t, n_stride), stride, 2) != 2) return -1;
  if (shape[1] > 1 && stride[1] != 1) return refuse(what);
  *ld = shape[0] > 1 ? stride[0] : shape[1];
  return fits_int(shape, 2) || float_type(t, type) || address(t, data) ? -1 : 0;
}
static int get_stream(PyObject* s, void** out) { /* None, a handle, or a stream object: as the binding's own function says */
  PyObject* v = PyObject_CallOneArg(stream_of, s);
  if (v == NULL) return -1;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return *out == NULL && PyErr_Occurred() ? -1 : 0;
}
/* The library's answer, called without the interpreter's lock as ctypes does it: a launch can wait (full queue, first load of a kernel), and a host function on that
 * stream that needs the lock would then never run.  (The caller holds the arguments.) */
#define CALLED(call)                                        \
  do {                                                      \
    int code_;                                              \
    Py_BEGIN_ALLOW_THREADS code_ = (call);                  \
    Py_END_ALLOW_THREADS return PyLong_FromLong(code_);     \
  } while (0)
static int arguments(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return 0;
  PyErr_Format(PyExc_TypeError, "%zd arguments are expected, not %zd", want, n);
  return -1;
}

/* ---- the calls */
/* (rope, x, y, grid, first, positions, inverse, stream) */
static PyObject* rope_apply(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  vsa2_rope store;
  const vsa2_rope* rope;
  vsa2_heads x, y;
  vsa2_place place;
  void* stream;
  int inverse;
  if (arguments(n, 8) || get_rope(a[0], &store, &rope) || get_view(a[1], &x) || get_view(a[2], &y) || get_place(a[3], a[4], a[5], &x, &place) ||
      (inverse = PyObject_IsTrue(a[6])) < 0 || get_stream(a[7], &stream))
    return NULL;
  CALLED(f_rope_apply(rope, &place, &x, &y, inverse, stream));
}
/* (rope, x, y, q_weight, k_weight, eps, norm, grid, first, positions, stream) */
static PyObject* qkv_fwd(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  vsa2_rope store;
  const vsa2_rope* rope;
  vsa2_heads x[3], y[3];
  vsa2_place place;
  vsa2_qk_norm norm;
  const vsa2_qk_norm* with;
  void* stream;
  if (arguments(n, 11) || get_rope(a[0], &store, &rope) || get_views(a[1], x, 3, NULL) || get_views(a[2], y, 3, NULL) ||
      get_norm(a[6], a[5], a[3], a[4], x[0].channels, &norm, &with) || get_place(a[7], a[8], a[9], &x[0], &place) || get_stream(a[10], &stream))
    return NULL;
  CALLED(f_qkv_fwd(rope, &place, with, x, y, stream));
}
/* (rope, x, dy, dx, q_weight, k_weight, d_q_weight, d_k_weight, workspace, eps, norm, grid, first, positions, stream) */
static PyObject* qkv_bwd(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  vsa2_rope store;
  const vsa2_rope* rope;
  vsa2_heads x[2], dy[3], dx[3];
  vsa2_place place;
  vsa2_qk_norm norm;
  const vsa2_qk_norm* with;
  void *stream, *dq, *dk, *workspace;
  size_t bytes;
  if (arguments(n, 15) || get_rope(a[0], &store, &rope) || get_views(a[2], dy, 3, NULL) || get_views(a[3], dx, 3, NULL) ||
      get_norm(a[10], a[9], a[4], a[5], dy[0].channels, &norm, &with) || (with != NULL && get_views(a[1], x, 2, &dy[0])) ||
      get_weight(a[6], dy[0].channels, &dq) || get_weight(a[7], dy[0].channels, &dk) || get_memory(a[8], &workspace, &bytes) ||
      get_place(a[11], a[12], a[13], &dy[0], &place) || get_stream(a[14], &stream))
    return NULL;
  CALLED(f_qkv_bwd(rope, &place, with, with != NULL ? x : NULL, dy, dx, (float*)dq, (float*)dk, workspace, bytes, stream));
}
/* (x, out, out_t, squares, stream) */
static PyObject* quantize(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t shape[2], ld, of[2], of_t[2];
  int32_t type;
  void *x, *stream;
  vsa2_fp8 out, out_t;
  int squares;
  if (arguments(n, 5) || get_matrix(a[0], shape, &ld, &type, &x) || (a[1] != Py_None && get_fp8(a[1], &out, of)) ||
      (a[2] != Py_None && get_fp8(a[2], &out_t, of_t)) || (squares = PyObject_IsTrue(a[3])) < 0 || get_stream(a[4], &stream))
    return NULL;
  if ((a[1] != Py_None && (of[0] != shape[0] || of[1] != shape[1])) || (a[2] != Py_None && (of_t[0] != shape[1] || of_t[1] != shape[0]))) {
    refuse("outputs do not have the shape of x and of its transpose");
    return NULL;
  }
  CALLED(f_quantize(x, type, (int32_t)shape[0], (int32_t)shape[1], ld, squares, a[1] != Py_None ? &out : NULL,
                                    a[2] != Py_None ? &out_t : NULL, stream));
}
/* (a, b, c, workspace, stream) */
static PyObject* matmul(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t of_a[2], of_b[2], of_c[2], ld;
  int32_t type;
  void *c, *workspace, *stream;
  size_t bytes;
  vsa2_fp8 va, vb;
  if (arguments(n, 5) || get_fp8(a[0], &va, of_a) || get_fp8(a[1], &vb, of_b) || get_matrix(a[2], of_c, &ld, &type, &c) ||
      get_memory(a[3], &workspace, &bytes) || get_stream(a[4], &stream))
    return NULL;
  if (of_a[1] != of_b[1] || of_c[0] != of_a[0] || of_c[1] != of_b[0]) {
    refuse("the shapes of a, b and c do not fit");
    return NULL;
  }
  CALLED(f_matmul((int32_t)of_a[0], (int32_t)of_b[0], (int32_t)of_a[1], &va, &vb, c, type, ld, workspace, bytes, stream));
}
/* (values, scales): whether they are a matrix in 8-bit form */
static PyObject* check_fp8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t shape[2], stride[2];
  if (arguments(n, 2) || fp8_form(a[0], a[1], shape, stride)) return NULL;
  Py_RETURN_NONE;
}

/* ---- the residual stream.  Its calls look at every tensor's device: the library runs on the current one, where another's addresses mean nothing */
static int here(PyObject* t, int64_t* device) { /* *device: the current one, -1 before it was asked for */
  int64_t of; /* -1: not a CUDA tensor's */
  if (number(PyObject_CallMethodNoArgs(t, n_get_device), &of)) return -1;
  if (of < 0) return refuse("expected a CUDA tensor");
  if (*device < 0 && number(PyObject_CallNoArgs(device_of), device)) return -1;
  return of == *device ? 0 : refuse("tensors must be on the current CUDA device");
}
/* the stream of a call whose tensors were looked at: None is the device's current one, without the detour through the binding's function (0.7 us) */
static int stream_here(PyObject* s, int64_t device, void** out) {
  if (s != Py_None || raw_stream == Py_None || device < 0) return get_stream(s, out);
  PyObject *d = PyLong_FromLongLong(device), *v = d != NULL ? PyObject_CallOneArg(raw_stream, d) : NULL;
  Py_XDECREF(d);
  if (v == NULL) return -1;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return *out == NULL && PyErr_Occurred() ? -1 : 0;
}
/* a matrix of the call's shape (the first sets it: rows < 0), None: absent */
static int get_rows(PyObject* t, int64_t* device, int64_t* shape, vsa2_rows* r, const vsa2_rows** out) {
  static const char* const what = "expected a CUDA matrix with contiguous rows";
  int64_t of[2], stride[2];
  *out = NULL;
  if (t == Py_None) return 0;
  const int n = integers(PyObject_GetAttr(t, n_shape), of, 2);
  if (n < 0) return -1;
  if (n != 2) return refuse(what);
  if (here(t, device) || integers(PyObject_CallMethodNoArgs(t, n_stride), stride, 2) != 2) return -1;
  if (of[1] > 1 && stride[1] != 1) return refuse(what);
  if (shape[0] >= 0 && (of[0] != shape[0] || of[1] != shape[1])) return refuse("the matrices of a call must have one shape");
  if (fits_int(of, 2) || float_type(t, &r->dtype) || address(t, &r->data)) return -1;
  r->ld = of[0] > 1 ? stride[0] : of[1];
  r->reserved = 0;
  shape[0] = of[0]; shape[1] = of[1];
  *out = r;
  return 0;
}
/* rng: int64 [2] on the device, or None */
static int get_drop(PyObject* p, PyObject* rng, int64_t* device, vsa2_drop* d, const vsa2_drop** out) {
  void* at = NULL;
  d->p = PyFloat_AsDouble(p);
  if (d->p == -1.0 && PyErr_Occurred()) return -1;
  if (rng != Py_None) {
    int64_t n;
    const int typed = is_type(rng, t_i64);
    if (typed < 0 || number(PyObject_CallMethodNoArgs(rng, n_numel), &n)) return -1;
    if (!typed || n != 2) return refuse("rng must be a contiguous CUDA int64 tensor of two elements: seed and offset");
    if (get_memory(rng, &at, NULL) || here(rng, device)) return -1;
  }
  d->rng = (const uint64_t*)at;
  *out = d;
  return 0;
}
static int get_weights(PyObject* t, int64_t* device, int64_t cols, float** out) { /* fp32 [cols], None: null */
  void* at;
  if (get_weight(t, (int)cols, &at) || (t != Py_None && here(t, device))) return -1;
  *out = (float*)at;
  return 0;
}
/* values and scales of a matrix in int8 form, on any device */
static int int8_form(PyObject* values, PyObject* scales, int64_t* shape, int64_t* stride) {
  int64_t of[1];
  int rank, typed = is_type(values, t_i8);
  if (typed < 0 || (rank = integers(PyObject_GetAttr(values, n_shape), shape, 2)) < 0) return -1;
  if (rank == 2 && integers(PyObject_CallMethodNoArgs(values, n_stride), stride, 2) != 2) return -1;
  if (!typed || rank != 2 || (shape[1] > 1 && stride[1] != 1)) return refuse("values must be int8 [rows, cols] with contiguous rows");
  typed = is_type(scales, t_f32);
  if (typed < 0 || (rank = integers(PyObject_GetAttr(scales, n_shape), of, 1)) < 0) return -1;
  if (!typed || rank != 1 || of[0] != shape[0]) return refuse("scales must be fp32 [rows]");
  return 0;
}
static int get_int8(PyObject* o, int64_t* device, vsa2_int8* v, int64_t* shape) { /* an Int8 object; its shape */
  int bad = -1;
  int64_t stride[2];
  void* scales;
  PyObject *values = PyObject_GetAttr(o, n_values), *s = values != NULL ? PyObject_GetAttr(o, n_scales) : NULL;
  if (s == NULL || here(values, device) || here(s, device) || int8_form(values, s, shape, stride) || fits_int(shape, 2) || address(values, &v->values) ||
      get_memory(s, &scales, NULL))
    goto out;
  v->scales = (float*)scales;
  v->ld = shape[0] > 1 ? stride[0] : (shape[1] + 15) / 16 * 16;
  bad = 0;
out:
  Py_XDECREF(values);
  Py_XDECREF(s);
  return bad;
}
static int fp8_here(PyObject* o, int64_t* device) {
  PyObject *values = PyObject_GetAttr(o, n_values), *s = values != NULL ? PyObject_GetAttr(o, n_scales) : NULL;
  const int bad = s == NULL || here(values, device) || here(s, device);
  Py_XDECREF(values);
  Py_XDECREF(s);
  return bad ? -1 : 0;
}
static int one_shape(const int64_t* a, const int64_t* b) {
  return a[0] == b[0] && a[1] == b[1] ? 0 : refuse("the matrices of a call must have one shape");
}
/* (x, residual, weight, eps, h, y, y_fp8, y_int8, p, rng, stream) */
static PyObject* norm_fwd(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t shape[2] = {-1, -1}, of[2], device = -1;
  vsa2_rows m[4];
  const vsa2_rows *x, *r, *h, *y;
  vsa2_fp8 fp8;
  vsa2_int8 int8;
  vsa2_drop store;
  const vsa2_drop* drop;
  float* w;
  void* stream;
  if (arguments(n, 11) || get_rows(a[0], &device, shape, &m[0], &x) || get_rows(a[1], &device, shape, &m[1], &r) ||
      get_rows(a[4], &device, shape, &m[2], &h) || get_rows(a[5], &device, shape, &m[3], &y))
    return NULL;
  if (x == NULL) {
    refuse("x is missing");
    return NULL;
  }
  if ((a[6] != Py_None && (get_fp8(a[6], &fp8, of) || fp8_here(a[6], &device) || one_shape(of, shape))) ||
      (a[7] != Py_None && (get_int8(a[7], &device, &int8, of) || one_shape(of, shape))) || get_weights(a[2], &device, shape[1], &w) ||
      get_drop(a[8], a[9], &device, &store, &drop))
    return NULL;
  const double eps = PyFloat_AsDouble(a[3]);
  if ((eps == -1.0 && PyErr_Occurred()) || stream_here(a[10], device, &stream)) return NULL;
  CALLED(f_norm_fwd((int32_t)shape[0], (int32_t)shape[1], x, r, drop, w, (float)eps, h, y, a[6] != Py_None ? &fp8 : NULL, a[7] != Py_None ? &int8 : NULL,
                    stream));
}
/* (h, dy, dh, weight, eps, d_residual, dx, d_weight, workspace, p, rng, stream) */
static PyObject* norm_bwd(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t shape[2] = {-1, -1}, device = -1;
  vsa2_rows m[5];
  const vsa2_rows *h, *dy, *dh, *dr, *dx;
  vsa2_drop store;
  const vsa2_drop* drop;
  float *w, *dw;
  void *workspace, *stream;
  size_t bytes;
  if (arguments(n, 12) || get_rows(a[0], &device, shape, &m[0], &h) || get_rows(a[1], &device, shape, &m[1], &dy) ||
      get_rows(a[2], &device, shape, &m[2], &dh) || get_rows(a[5], &device, shape, &m[3], &dr) || get_rows(a[6], &device, shape, &m[4], &dx))
    return NULL;
  if (h == NULL || dy == NULL) {
    refuse("h or dy is missing");
    return NULL;
  }
  if (get_weights(a[3], &device, shape[1], &w) || get_weights(a[7], &device, shape[1], &dw) || get_memory(a[8], &workspace, &bytes) ||
      (a[8] != Py_None && here(a[8], &device)) || get_drop(a[9], a[10], &device, &store, &drop))
    return NULL;
  const double eps = PyFloat_AsDouble(a[4]);
  if ((eps == -1.0 && PyErr_Occurred()) || stream_here(a[11], device, &stream)) return NULL;
  CALLED(f_norm_bwd((int32_t)shape[0], (int32_t)shape[1], h, dy, dh, drop, w, (float)eps, dr, dx, dw, workspace, bytes, stream));
}
/* (x, y, p, rng, residual, stream) */
static PyObject* dropout(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t shape[2] = {-1, -1}, device = -1;
  vsa2_rows m[3];
  const vsa2_rows *x, *y, *r;
  vsa2_drop store;
  const vsa2_drop* drop;
  void* stream;
  if (arguments(n, 6) || get_rows(a[0], &device, shape, &m[0], &x) || get_rows(a[1], &device, shape, &m[1], &y) ||
      get_rows(a[4], &device, shape, &m[2], &r) || get_drop(a[2], a[3], &device, &store, &drop) || stream_here(a[5], device, &stream))
    return NULL;
  CALLED(f_dropout((int32_t)shape[0], (int32_t)shape[1], x, r, drop, y, stream));
}
/* (x, out, stream) */
static PyObject* int8_quantize(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t shape[2] = {-1, -1}, of[2], device = -1;
  vsa2_rows m;
  const vsa2_rows* x;
  vsa2_int8 out;
  void* stream;
  if (arguments(n, 3) || get_rows(a[0], &device, shape, &m, &x) || get_int8(a[1], &device, &out, of) || one_shape(of, shape) ||
      stream_here(a[2], device, &stream))
    return NULL;
  CALLED(f_int8_quantize((int32_t)shape[0], (int32_t)shape[1], x, &out, stream));
}
/* (a, b, c, workspace, bias, stream) */
static PyObject* int8_matmul(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t of_a[2], of_b[2], of_c[2], ld, device = -1;
  int32_t type;
  void *c, *workspace, *stream;
  size_t bytes;
  vsa2_int8 va, vb;
  float* bias;
  if (arguments(n, 6) || get_int8(a[0], &device, &va, of_a) || get_int8(a[1], &device, &vb, of_b) ||
      get_matrix(a[2], of_c, &ld, &type, &c) || here(a[2], &device) || get_memory(a[3], &workspace, &bytes) || (a[3] != Py_None && here(a[3], &device)))
    return NULL;
  if (of_a[1] != of_b[1] || of_c[0] != of_a[0] || of_c[1] != of_b[0]) {
    refuse("the shapes of a, b and c do not fit");
    return NULL;
  }
  if (get_weights(a[4], &device, of_b[0], &bias) || stream_here(a[5], device, &stream)) return NULL;
  CALLED(f_int8_matmul((int32_t)of_a[0], (int32_t)of_b[0], (int32_t)of_a[1], &va, &vb, bias, c, type, ld, workspace, bytes, stream));
}
/* (values, scales): whether they are a matrix in int8 form */
static PyObject* check_int8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t shape[2], stride[2];
  if (arguments(n, 2) || int8_form(a[0], a[1], shape, stride)) return NULL;
  Py_RETURN_NONE;
}

/* n objects of a tuple, borrowed, and n addresses of another */
static int bound(PyObject* types, PyObject* calls, int n_types, int n_calls, void** f) {
  if (!PyTuple_Check(types) || !PyTuple_Check(calls) || PyTuple_GET_SIZE(types) != n_types || PyTuple_GET_SIZE(calls) != n_calls)
    return refuse("a tuple of types and a tuple of addresses are expected");
  for (int i = 0; i < n_calls; ++i) {
    f[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(calls, i));
    if (f[i] == NULL) return PyErr_Occurred() ? -1 : refuse("a function's address is missing");
  }
  return 0;
}
/* ((bf16, fp32, int32, e4m3, uint8), (addresses of the five functions between hidden states and attention), function that gives a stream's handle) */
static PyObject* bind(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  PyObject** const types[5] = {&t_bf16, &t_f32, &t_i32, &t_e4m3, &t_u8};
  void* f[5];
  if (arguments(n, 3) || bound(a[0], a[1], 5, 5, f)) return NULL;
  for (int i = 0; i < 5; ++i) Py_XSETREF(*types[i], Py_NewRef(PyTuple_GET_ITEM(a[0], i)));
  Py_XSETREF(stream_of, Py_NewRef(a[2]));
  memcpy(&f_rope_apply, &f[0], sizeof f[0]);
  memcpy(&f_qkv_fwd, &f[1], sizeof f[0]);
  memcpy(&f_qkv_bwd, &f[2], sizeof f[0]);
  memcpy(&f_quantize, &f[3], sizeof f[0]);
  memcpy(&f_matmul, &f[4], sizeof f[0]);
  Py_RETURN_NONE;
}
/* ((int8, int64), (addresses of the five functions of the residual stream), function that gives the current device, one that gives a device's current stream or None); behind bind */
static PyObject* bind_rows(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void* f[5];
  if (arguments(n, 4) || bound(a[0], a[1], 2, 5, f)) return NULL;
  Py_XSETREF(t_i8, Py_NewRef(PyTuple_GET_ITEM(a[0], 0)));
  Py_XSETREF(t_i64, Py_NewRef(PyTuple_GET_ITEM(a[0], 1)));
  Py_XSETREF(device_of, Py_NewRef(a[2]));
  Py_XSETREF(raw_stream, Py_NewRef(a[3]));
  memcpy(&f_norm_fwd, &f[0], sizeof f[0]);
  memcpy(&f_norm_bwd, &f[1], sizeof f[0]);
  memcpy(&f_dropout, &f[2], sizeof f[0]);
  memcpy(&f_int8_quantize, &f[3], sizeof f[0]);
  memcpy(&f_int8_matmul, &f[4], sizeof f[0]);
  Py_RETURN_NONE;
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {ENTRY(bind), ENTRY(bind_rows), ENTRY(check_fp8), ENTRY(rope_apply), ENTRY(qkv_fwd), ENTRY(qkv_bwd), ENTRY(quantize), ENTRY(matmul),
                                ENTRY(check_int8), ENTRY(norm_fwd), ENTRY(norm_bwd), ENTRY(dropout), ENTRY(int8_quantize), ENTRY(int8_matmul), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, .m_name = "_marshal", .m_size = -1, .m_methods = methods};

PyMODINIT_FUNC PyInit__marshal(void) {
  static const struct { PyObject** at; const char* name; } names[] = {
      {&n_shape, "shape"}, {&n_stride, "stride"}, {&n_dtype, "dtype"}, {&n_is_cuda, "is_cuda"}, {&n_data_ptr, "data_ptr"},
      {&n_is_contiguous, "is_contiguous"}, {&n_numel, "numel"}, {&n_nbytes, "nbytes"}, {&n_values, "values"}, {&n_scales, "scales"},
      {&n_get_device, "get_device"}};
  for (size_t i = 0; i < sizeof names / sizeof names[0]; ++i)
    if ((*names[i].at = PyUnicode_InternFromString(names[i].name)) == NULL) return NULL;
  return PyModule_Create(&module);
}
