/* CPython entry to the device calls of libdasc that sit on a serving engine's path: argument marshalling only, like
 * binding.py, which uses it for these calls.  A ctypes call with ten to twenty-six arguments costs 4 to 8 us of interpreter
 * time on the host of a B200, more than the GPU needs for the smallest calls; here it is under 1 us.
 *
 * Tensors are taken as they are: None is a null pointer, an int an address, anything with a data_ptr() that; what an address
 * is for other objects binding.py says.  `stream` is None (torch's current stream) or has a cuda_stream attribute.  Every function
 * returns the dasc_status_t. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "dasc.h"

static PyObject *s_data_ptr, *s_numel, *s_element_size, *s_cuda_stream, *s_dtype, *s_is_contiguous, *s_get_device;
static PyObject *g_raw_stream, *g_device, *g_bf16, *g_address, *g_fp32, *g_int32; /* set by init() */

static int as_ptr(PyObject *o, void **out) {
  if (o == Py_None) {
    *out = NULL;
    return 0;
  }
  PyObject *v;
  if (PyLong_Check(o)) {
    v = Py_NewRef(o);
  } else {
    v = PyObject_CallMethodNoArgs(o, s_data_ptr);
    if (!v && PyErr_ExceptionMatches(PyExc_AttributeError)) {
      PyErr_Clear();
      v = PyObject_CallOneArg(g_address, o);
    }
    if (!v) return -1;
  }
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return *out == NULL && PyErr_Occurred() ? -1 : 0;
}

/* A stride, a layer, an enumerator: whole numbers only, a float is an error and not cut off. */
static int as_index(PyObject *o, int64_t *out) {
  if (PyLong_Check(o)) {
    *out = PyLong_AsLongLong(o);
  } else {
    PyObject *v = PyNumber_Index(o);
    if (!v) return -1;
    *out = PyLong_AsLongLong(v);
    Py_DECREF(v);
  }
  return *out == -1 && PyErr_Occurred() ? -1 : 0;
}

/* A token count: whatever int() takes. */
static int as_count(PyObject *o, int64_t *out) {
  if (PyLong_Check(o)) {
    *out = PyLong_AsLongLong(o);
  } else {
    PyObject *v = PyNumber_Long(o);
    if (!v) return -1;
    *out = PyLong_AsLongLong(v);
    Py_DECREF(v);
  }
  return *out == -1 && PyErr_Occurred() ? -1 : 0;
}

static int method_i64(PyObject *o, PyObject *name, int64_t *out) {
  PyObject *v = PyObject_CallMethodNoArgs(o, name);
  if (!v) return -1;
  const int r = as_index(v, out);
  Py_DECREF(v);
  return r;
}

static int as_stream(PyObject *o, void **out) {
  PyObject *v;
  if (o == Py_None) {
    PyObject *dev = PyObject_CallNoArgs(g_device);
    if (!dev) return -1;
    v = PyObject_CallOneArg(g_raw_stream, dev);
    Py_DECREF(dev);
  } else {
    v = PyObject_GetAttr(o, s_cuda_stream);
  }
  if (!v) return -1;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return *out == NULL && PyErr_Occurred() ? -1 : 0;
}

/* DASC_IO_BF16 or DASC_IO_FP32 */
static int as_io(PyObject *o, int32_t *out) {
  *out = DASC_IO_FP32;
  if (o == Py_None) return 0;
  PyObject *v = PyObject_GetAttr(o, s_dtype);
  if (!v) return -1;
  if (v == g_bf16) *out = DASC_IO_BF16;
  Py_DECREF(v);
  return 0;
}

static int nbytes(PyObject *o, size_t *out) {
  *out = 0;
  if (o == Py_None) return 0;
  int64_t n, e;
  if (method_i64(o, s_numel, &n) || method_i64(o, s_element_size, &e)) return -1;
  *out = (size_t)(n * e);
  return 0;
}

static int arg_count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return 0;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  return -1;
}

/* raw_stream(device) -> cudaStream_t of torch's current stream, device() -> current device, torch.bfloat16, address(object),
 * torch.float32, torch.int32 */
static PyObject *py_init(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  if (arg_count(n, 6)) return NULL;
  Py_XSETREF(g_raw_stream, Py_NewRef(a[0]));
  Py_XSETREF(g_device, Py_NewRef(a[1]));
  Py_XSETREF(g_bf16, Py_NewRef(a[2]));
  Py_XSETREF(g_address, Py_NewRef(a[3]));
  Py_XSETREF(g_fp32, Py_NewRef(a[4]));
  Py_XSETREF(g_int32, Py_NewRef(a[5]));
  Py_RETURN_NONE;
}

/* plan, state, layer_stride, req_stride, src_req, pool, pool_arg, dst_slot, stream; pool_arg: slot stride or slot count */
typedef dasc_status_t (*store_fn)(const dasc_plan_t *, const float *, int64_t, int64_t, const int32_t *, void *, int64_t,
                                  const int32_t *, int32_t, void *);
static PyObject *store_call(store_fn fn, PyObject *const *a, Py_ssize_t n) {
  void *plan, *state, *src, *pool, *dst, *stream;
  int64_t ls, rs, arg, pairs;
  if (arg_count(n, 9) || as_ptr(a[0], &plan) || as_ptr(a[1], &state) || as_index(a[2], &ls) || as_index(a[3], &rs) ||
      as_ptr(a[4], &src) || as_ptr(a[5], &pool) || as_index(a[6], &arg) || as_ptr(a[7], &dst) ||
      method_i64(a[4], s_numel, &pairs) || as_stream(a[8], &stream))
    return NULL;
  dasc_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = fn(plan, state, ls, rs, src, pool, arg, dst, (int32_t)pairs, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* plan, pool, pool_arg, src_slot, state, layer_stride, req_stride, dst_req, stream */
typedef dasc_status_t (*load_fn)(const dasc_plan_t *, const void *, int64_t, const int32_t *, float *, int64_t, int64_t,
                                 const int32_t *, int32_t, void *);
static PyObject *load_call(load_fn fn, PyObject *const *a, Py_ssize_t n) {
  void *plan, *state, *src, *pool, *dst, *stream;
  int64_t ls, rs, arg, pairs;
  if (arg_count(n, 9) || as_ptr(a[0], &plan) || as_ptr(a[1], &pool) || as_index(a[2], &arg) || as_ptr(a[3], &src) ||
      as_ptr(a[4], &state) || as_index(a[5], &ls) || as_index(a[6], &rs) || as_ptr(a[7], &dst) ||
      method_i64(a[3], s_numel, &pairs) || as_stream(a[8], &stream))
    return NULL;
  dasc_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = fn(plan, pool, arg, src, state, ls, rs, dst, (int32_t)pairs, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

#define COPY_CALL(name, kind, fn) \
  static PyObject *name(PyObject *self, PyObject *const *a, Py_ssize_t n) { return kind##_call((kind##_fn)fn, a, n); }
COPY_CALL(py_pack, store, dasc_pack)
COPY_CALL(py_pack_padded, store, dasc_pack_padded)
COPY_CALL(py_pack_int8, store, dasc_pack_int8)
COPY_CALL(py_restore, load, dasc_restore)
COPY_CALL(py_restore_padded, load, dasc_restore_padded)
COPY_CALL(py_restore_int8, load, dasc_restore_int8)

/* What the two refresh calls share: plan, state, layer_stride, req_stride, req_idx, q, k, v, g, beta, cu_seqlens, total_tokens,
 * bound (longest request or window), layer_begin, layer_end, q_scale, o, algo, workspace, stream */
struct refresh_args {
  void *plan, *state, *req, *q, *k, *v, *g, *beta, *cu, *o, *ws, *stream;
  int64_t ls, rs, total, bound, lb, le, algo, n_cu;
  int32_t io, o_io;
  float q_scale;
  size_t ws_bytes;
};
static int refresh_parse(struct refresh_args *r, PyObject *const *a, PyObject *io_from) {
  if (as_ptr(a[0], &r->plan) || as_ptr(a[1], &r->state) || as_index(a[2], &r->ls) || as_index(a[3], &r->rs) ||
      as_ptr(a[4], &r->req) || as_ptr(a[5], &r->q) || as_ptr(a[6], &r->k) || as_ptr(a[7], &r->v) || as_ptr(a[8], &r->g) ||
      as_ptr(a[9], &r->beta) || as_ptr(a[10], &r->cu) || method_i64(a[10], s_numel, &r->n_cu) || as_count(a[11], &r->total) ||
      as_count(a[12], &r->bound) || as_index(a[13], &r->lb) || as_index(a[14], &r->le) || as_ptr(a[16], &r->o) ||
      as_index(a[17], &r->algo) || as_ptr(a[18], &r->ws) || nbytes(a[18], &r->ws_bytes) || as_stream(a[19], &r->stream) ||
      as_io(io_from, &r->io) || as_io(a[16], &r->o_io))
    return -1;
  PyObject *s = PyNumber_Float(a[15]);
  if (!s) return -1;
  r->q_scale = (float)PyFloat_AS_DOUBLE(s);
  Py_DECREF(s);
  return 0;
}

/* the arguments above, then mode */
static PyObject *py_refresh(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  struct refresh_args r;
  int64_t mode;
  if (arg_count(n, 21) || refresh_parse(&r, a, a[5]) || as_index(a[20], &mode)) return NULL;
  dasc_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = dasc_refresh(r.plan, r.state, r.ls, r.rs, r.req, r.q, r.k, r.v, r.io, r.g, r.beta, r.cu, (int32_t)(r.n_cu - 1), r.total,
                    (int32_t)r.bound, (int32_t)r.lb, (int32_t)r.le, r.q_scale, r.o, r.o_io, (int32_t)mode, (int32_t)r.algo, r.ws,
                    r.ws_bytes, r.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* the arguments above, then window_begin */
static PyObject *py_refresh_window(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  struct refresh_args r;
  void *wb;
  if (arg_count(n, 21) || refresh_parse(&r, a, a[6]) || as_ptr(a[20], &wb)) return NULL;
  dasc_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = dasc_refresh_window(r.plan, r.state, r.ls, r.rs, r.req, r.q, r.k, r.v, r.io, r.g, r.beta, r.cu, (int32_t)(r.n_cu - 1),
                           r.total, r.bound, (int32_t)r.lb, (int32_t)r.le, r.q_scale, r.o, r.o_io, (int32_t)r.algo, wb, r.ws,
                           r.ws_bytes, r.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* ---- decayed linear attention, draft verification: their tensors are looked at before their addresses are used ---- */

static int current_device(int64_t *out) {
  PyObject *v = PyObject_CallNoArgs(g_device);
  if (!v) return -1;
  const int r = as_index(v, out);
  Py_DECREF(v);
  return r;
}

/* Is the tensor on device `dev`, and contiguous (unless `any_layout`)? */
static int is_placed(PyObject *o, const char *name, int64_t dev, int any_layout) {
  int64_t x;
  if (method_i64(o, s_get_device, &x)) return -1;
  if (x != dev) {
    PyErr_Format(PyExc_ValueError, "%s is not on the current CUDA device", name);
    return -1;
  }
  if (any_layout) return 0;
  PyObject *v = PyObject_CallMethodNoArgs(o, s_is_contiguous);
  if (!v) return -1;
  const int yes = PyObject_IsTrue(v);
  Py_DECREF(v);
  if (yes < 0) return -1;
  if (!yes) {
    PyErr_Format(PyExc_ValueError, "%s is not contiguous", name);
    return -1;
  }
  return 0;
}

/* A tensor's address (None: NULL; an int is an address and taken as it is where there is one type it can be of).  It has to be on device
 * `dev`, of type `dtype` (NULL: bf16 or fp32, which *io says), contiguous unless `any_layout`, and to hold at least `need` values. */
static int as_tensor(PyObject *o, const char *name, int64_t dev, PyObject *dtype, int any_layout, double need, int32_t *io, void **out) {
  if (!dtype && PyLong_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s has to be a tensor: an address does not say whether its values are bf16 or fp32", name);
    return -1;
  }
  if (o == Py_None || PyLong_Check(o)) return as_ptr(o, out);
  int64_t x;
  PyObject *v = PyObject_GetAttr(o, s_dtype);
  if (!v) return -1;
  const int bf16 = v == g_bf16, ok = dtype ? v == dtype : bf16 || v == g_fp32;
  if (!ok) PyErr_Format(PyExc_TypeError, "%s has type %S", name, v);
  Py_DECREF(v);
  if (!ok) return -1;
  if (io) *io = bf16 ? DASC_IO_BF16 : DASC_IO_FP32;
  if (is_placed(o, name, dev, any_layout)) return -1;
  if (need > 0) {
    if (method_i64(o, s_numel, &x)) return -1;
    if ((double)x < need) {
      PyErr_Format(PyExc_ValueError, "%s holds %lld values, the call needs %lld", name, (long long)x, (long long)need);
      return -1;
    }
  }
  return as_ptr(o, out);
}

static int as_float(PyObject *o, float *out) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) return -1;
  *out = (float)x;
  return 0;
}

static int as_i32(int64_t x, const char *name, int32_t *out) {
  if (x < INT32_MIN || x > INT32_MAX) {
    PyErr_Format(PyExc_ValueError, "%s does not fit 32 bits", name);
    return -1;
  }
  *out = (int32_t)x;
  return 0;
}

/* plan, state, layer_stride, req_stride, req_idx, q, k, v, g, decay, layer_begin, layer_end, q_scale, o */
struct decay_args {
  void *plan, *state, *req, *q, *k, *v, *g, *o;
  int64_t dev, ls, rs, n_req;
  int32_t decay, lb, le, n_req32, io, o_io;
  float q_scale;
};
static int decay_parse(struct decay_args *r, PyObject *const *a, int64_t tokens /* < 0: one per request */) {
  dasc_plan_info_t info;
  int64_t decay, lb, le;
  int32_t io_q = -1, io_k = -1, io_v = -1;
  r->o_io = DASC_IO_FP32;
  if (as_ptr(a[0], &r->plan) || current_device(&r->dev) || as_index(a[2], &r->ls) || as_index(a[3], &r->rs) || as_index(a[9], &decay) ||
      as_index(a[10], &lb) || as_index(a[11], &le) || as_float(a[12], &r->q_scale) || as_i32(decay, "decay", &r->decay) ||
      as_i32(lb, "layer_begin", &r->lb) || as_i32(le, "layer_end", &r->le))
    return -1;
  if (dasc_plan_info(r->plan, &info) != DASC_OK) {
    PyErr_SetString(PyExc_ValueError, "no plan");
    return -1;
  }
  if (PyLong_Check(a[4]) || a[4] == Py_None) {
    PyErr_SetString(PyExc_TypeError, "req_idx has to be a tensor");
    return -1;
  }
  if (method_i64(a[4], s_numel, &r->n_req) || as_i32(r->n_req, "n_req", &r->n_req32)) return -1;
  const double layers = (double)le - (double)lb, rows = layers * (double)(tokens < 0 ? r->n_req : tokens);
  const double qk = rows * info.n_k_heads * info.d_k, vo = rows * info.n_v_heads * info.d_v;
  const double g = (r->decay == DASC_DECAY_PER_HEAD ? layers : rows) * info.n_v_heads;
  if (as_tensor(a[1], "state", r->dev, g_fp32, 1, 0, NULL, &r->state) || as_tensor(a[4], "req_idx", r->dev, g_int32, 0, 0, NULL, &r->req) ||
      as_tensor(a[5], "q", r->dev, NULL, 0, qk, &io_q, &r->q) || as_tensor(a[6], "k", r->dev, NULL, 0, qk, &io_k, &r->k) ||
      as_tensor(a[7], "v", r->dev, NULL, 0, vo, &io_v, &r->v) || as_tensor(a[8], "g", r->dev, g_fp32, 0, g, NULL, &r->g))
    return -1;
  r->io = io_k == -1 ? DASC_IO_FP32 : io_k;
  if ((io_q != -1 && io_q != r->io) || (io_v != -1 && io_v != r->io)) {
    PyErr_SetString(PyExc_TypeError, "q, k and v have to be of one type");
    return -1;
  }
  return as_tensor(a[13], "o", r->dev, NULL, 0, vo, &r->o_io, &r->o);
}

/* the arguments above, then cu_seqlens, total_tokens, max_seqlen, seq_used, from_zero, mode, algo, workspace, stream */
static PyObject *py_decay_attn(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  struct decay_args r;
  void *cu, *used, *zero, *ws, *stream;
  int64_t total, longest, mode, algo, n_cu;
  int32_t most, mode32, algo32;
  size_t ws_bytes;
  if (arg_count(n, 23) || as_count(a[15], &total) || as_count(a[16], &longest) || as_index(a[19], &mode) || as_index(a[20], &algo) ||
      as_i32(longest, "max_seqlen", &most) || as_i32(mode, "mode", &mode32) || as_i32(algo, "algo", &algo32))
    return NULL;
  if (decay_parse(&r, a, total < 0 ? 0 : total) || as_tensor(a[14], "cu_seqlens", r.dev, g_int32, 0, 1, NULL, &cu) || method_i64(a[14], s_numel, &n_cu))
    return NULL;
  if (n_cu != r.n_req + 1) {
    PyErr_Format(PyExc_ValueError, "cu_seqlens holds %lld values for %lld requests", (long long)n_cu, (long long)r.n_req);
    return NULL;
  }
  if (as_tensor(a[17], "seq_used", r.dev, g_int32, 0, (double)r.n_req, NULL, &used) ||
      as_tensor(a[18], "from_zero", r.dev, g_int32, 0, (double)r.n_req, NULL, &zero) || (a[21] != Py_None && is_placed(a[21], "workspace", r.dev, 0)) ||
      as_ptr(a[21], &ws) || nbytes(a[21], &ws_bytes) || as_stream(a[22], &stream))
    return NULL;
  dasc_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = dasc_decay_attn(r.plan, r.state, r.ls, r.rs, r.req, r.q, r.k, r.v, r.io, r.g, r.decay, cu, used, zero, r.n_req32, total, most, r.lb, r.le,
                       r.q_scale, r.o, r.o_io, mode32, algo32, ws, ws_bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* the arguments above, then stream */
static PyObject *py_decay_step(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  struct decay_args r;
  void *stream;
  if (arg_count(n, 15) || decay_parse(&r, a, -1) || as_stream(a[14], &stream)) return NULL;
  dasc_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = dasc_decay_step(r.plan, r.state, r.ls, r.rs, r.req, r.q, r.k, r.v, r.io, r.g, r.decay, r.n_req32, r.lb, r.le, r.q_scale, r.o, r.o_io, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* target, target_stride, draft, draft_stride, vocab, tokens, cu_drafts, u_accept, u_next, max_drafts, out, out_stride, n_kept, stream;
 * rows of target, draft and out may be further apart than they are long, so the caller has looked at their shapes */
static PyObject *py_verify_draft(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  void *target, *draft, *tokens, *cu, *ua, *un, *out, *kept, *stream;
  int64_t dev, ts, ds, vocab, most, os, n_cu, n_drafts;
  int32_t io = DASC_IO_FP32, io_d = -1, n_req, most32, vocab32;
  if (arg_count(n, 14) || current_device(&dev) || as_index(a[1], &ts) || as_index(a[3], &ds) || as_index(a[4], &vocab) || as_index(a[9], &most) ||
      as_index(a[11], &os) || as_tensor(a[0], "target", dev, NULL, 1, 0, &io, &target) || as_tensor(a[2], "draft", dev, NULL, 1, 0, &io_d, &draft) ||
      as_tensor(a[5], "tokens", dev, g_int32, 0, 0, NULL, &tokens) || method_i64(a[5], s_numel, &n_drafts) ||
      as_tensor(a[6], "cu_drafts", dev, g_int32, 0, 1, NULL, &cu) || method_i64(a[6], s_numel, &n_cu) ||
      as_tensor(a[7], "u_accept", dev, g_fp32, 0, (double)n_drafts, NULL, &ua) ||
      as_tensor(a[8], "u_next", dev, g_fp32, 0, (double)(n_cu - 1), NULL, &un) || as_tensor(a[10], "out", dev, g_int32, 1, 0, NULL, &out) ||
      as_tensor(a[12], "n_kept", dev, g_int32, 0, (double)(n_cu - 1), NULL, &kept) || as_stream(a[13], &stream) ||
      as_i32(n_cu - 1, "n_req", &n_req) || as_i32(most, "max_drafts", &most32) || as_i32(vocab, "vocab", &vocab32))
    return NULL;
  if (io_d != -1 && io_d != io) {
    PyErr_SetString(PyExc_TypeError, "target and draft have to be of one type");
    return NULL;
  }
  if (n_drafts == 0) tokens = ua = NULL;
  dasc_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = dasc_verify_draft(target, ts, draft, ds, io, vocab32, tokens, cu, ua, un, n_req, most32, out, os, kept, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* ---- the gated delta rule for single and drafted tokens, beam search ---- */

/* plan, state, layer_stride, req_stride, req_idx, q, k, v, g, beta, layer_begin, layer_end, q_scale, o */
struct delta_args {
  void *plan, *state, *req, *q, *k, *v, *g, *beta, *o;
  int64_t dev, ls, rs, n_req;
  int32_t lb, le, n_req32, io, o_io;
  float q_scale;
};
static int delta_parse(struct delta_args *r, PyObject *const *a, int64_t tokens /* < 0: one per request */) {
  dasc_plan_info_t info;
  int64_t lb, le;
  int32_t io_q = -1, io_k = -1, io_v = -1;
  r->o_io = DASC_IO_FP32;
  if (as_ptr(a[0], &r->plan) || current_device(&r->dev) || as_index(a[2], &r->ls) || as_index(a[3], &r->rs) || as_index(a[10], &lb) ||
      as_index(a[11], &le) || as_float(a[12], &r->q_scale) || as_i32(lb, "layer_begin", &r->lb) || as_i32(le, "layer_end", &r->le))
    return -1;
  if (dasc_plan_info(r->plan, &info) != DASC_OK) {
    PyErr_SetString(PyExc_ValueError, "no plan");
    return -1;
  }
  if (PyLong_Check(a[4]) || a[4] == Py_None) {
    PyErr_SetString(PyExc_TypeError, "req_idx has to be a tensor");
    return -1;
  }
  if (method_i64(a[4], s_numel, &r->n_req) || as_i32(r->n_req, "n_req", &r->n_req32)) return -1;
  const double rows = ((double)le - (double)lb) * (double)(tokens < 0 ? r->n_req : tokens);
  const double qk = rows * info.n_k_heads * info.d_k, vo = rows * info.n_v_heads * info.d_v, heads = rows * info.n_v_heads;
  if (as_tensor(a[1], "state", r->dev, g_fp32, 1, 0, NULL, &r->state) || as_tensor(a[4], "req_idx", r->dev, g_int32, 0, 0, NULL, &r->req) ||
      as_tensor(a[5], "q", r->dev, NULL, 0, qk, &io_q, &r->q) || as_tensor(a[6], "k", r->dev, NULL, 0, qk, &io_k, &r->k) ||
      as_tensor(a[7], "v", r->dev, NULL, 0, vo, &io_v, &r->v) ||
      as_tensor(a[8], "g", r->dev, g_fp32, 0, info.kind == DASC_KDA ? heads * info.d_k : heads, NULL, &r->g) ||
      as_tensor(a[9], "beta", r->dev, g_fp32, 0, heads, NULL, &r->beta))
    return -1;
  r->io = io_k == -1 ? DASC_IO_FP32 : io_k;
  if ((io_q != -1 && io_q != r->io) || (io_v != -1 && io_v != r->io)) {
    PyErr_SetString(PyExc_TypeError, "q, k and v have to be of one type");
    return -1;
  }
  return as_tensor(a[13], "o", r->dev, NULL, 0, vo, &r->o_io, &r->o);
}

/* delta_parse's arguments, then src_idx, beam_width, stream */
static PyObject *py_delta_step(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  struct delta_args r;
  void *src, *stream;
  int64_t width;
  int32_t width32;
  if (arg_count(n, 17) || delta_parse(&r, a, -1) || as_tensor(a[14], "src_idx", r.dev, g_int32, 0, (double)r.n_req, NULL, &src) ||
      as_index(a[15], &width) || as_i32(width, "beam_width", &width32) || as_stream(a[16], &stream))
    return NULL;
  dasc_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = dasc_delta_step(r.plan, r.state, r.ls, r.rs, r.req, src, width32, r.q, r.k, r.v, r.io, r.g, r.beta, r.n_req32, r.lb, r.le, r.q_scale, r.o, r.o_io,
                       stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* delta_parse's arguments, then cu_seqlens, total_tokens, max_seqlen, seq_used, from_zero, mode, stream */
static PyObject *py_delta_draft(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  struct delta_args r;
  void *cu, *used, *zero, *stream;
  int64_t total, longest, mode, n_cu;
  int32_t most, mode32;
  if (arg_count(n, 21) || as_count(a[15], &total) || as_count(a[16], &longest) || as_index(a[19], &mode) || as_i32(longest, "max_seqlen", &most) ||
      as_i32(mode, "mode", &mode32))
    return NULL;
  if (delta_parse(&r, a, total < 0 ? 0 : total) || as_tensor(a[14], "cu_seqlens", r.dev, g_int32, 0, 1, NULL, &cu) || method_i64(a[14], s_numel, &n_cu))
    return NULL;
  if (n_cu != r.n_req + 1) {
    PyErr_Format(PyExc_ValueError, "cu_seqlens holds %lld values for %lld requests", (long long)n_cu, (long long)r.n_req);
    return NULL;
  }
  if (as_tensor(a[17], "seq_used", r.dev, g_int32, 0, (double)r.n_req, NULL, &used) ||
      as_tensor(a[18], "from_zero", r.dev, g_int32, 0, (double)r.n_req, NULL, &zero) || as_stream(a[20], &stream))
    return NULL;
  dasc_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = dasc_delta_draft(r.plan, r.state, r.ls, r.rs, r.req, r.q, r.k, r.v, r.io, r.g, r.beta, cu, used, zero, r.n_req32, total, most, r.lb, r.le, r.q_scale,
                        r.o, r.o_io, mode32, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* logits, logits_stride, vocab, scores, ended, end_token, n_req, width, n_out, out_scores, out_parent, out_token, out_ended, stream; rows of logits may be
 * further apart than they are long, so the caller has looked at their shape */
static PyObject *py_beam_select(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  void *logits, *scores, *ended, *os, *op, *ot, *oe, *stream;
  int64_t dev, stride, x[5];
  int32_t io = DASC_IO_FP32, i[5];
  static const char *const names[5] = {"vocab", "end_token", "n_req", "width", "n_out"};
  static const int at[5] = {2, 5, 6, 7, 8};
  if (arg_count(n, 14) || current_device(&dev) || as_index(a[1], &stride)) return NULL;
  for (int j = 0; j < 5; ++j)
    if (as_index(a[at[j]], &x[j]) || as_i32(x[j], names[j], &i[j])) return NULL;
  const double beams = (double)i[2] * i[3], outs = (double)i[2] * i[4];
  if (as_tensor(a[0], "logits", dev, NULL, 1, 0, &io, &logits) || as_tensor(a[3], "scores", dev, g_fp32, 0, beams, NULL, &scores) ||
      as_tensor(a[4], "ended", dev, g_int32, 0, beams, NULL, &ended) || as_tensor(a[9], "out_scores", dev, g_fp32, 0, outs, NULL, &os) ||
      as_tensor(a[10], "out_parent", dev, g_int32, 0, outs, NULL, &op) || as_tensor(a[11], "out_token", dev, g_int32, 0, outs, NULL, &ot) ||
      as_tensor(a[12], "out_ended", dev, g_int32, 0, outs, NULL, &oe) || as_stream(a[13], &stream))
    return NULL;
  dasc_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = dasc_beam_select(logits, stride, io, i[0], scores, ended, i[1], i[2], i[3], i[4], os, op, ot, oe, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

/* plan, state, layer_stride, req_stride, conv, conv_stride_bytes, conv_bytes, req_idx, parent, n_req, width, layer_begin, layer_end, new_idx, src_idx,
 * stream */
static PyObject *py_beam_reorder(PyObject *self, PyObject *const *a, Py_ssize_t n) {
  void *plan, *state, *conv, *req, *parent, *to, *src, *stream;
  int64_t dev, ls, rs, cs, cb, x[4];
  int32_t i[4];
  static const char *const names[4] = {"n_req", "width", "layer_begin", "layer_end"};
  if (arg_count(n, 16) || as_ptr(a[0], &plan) || current_device(&dev) || as_index(a[2], &ls) || as_index(a[3], &rs) || as_index(a[5], &cs) ||
      as_index(a[6], &cb))
    return NULL;
  for (int j = 0; j < 4; ++j)
    if (as_index(a[9 + j], &x[j]) || as_i32(x[j], names[j], &i[j])) return NULL;
  const double beams = (double)i[0] * i[1];
  if (as_tensor(a[1], "state", dev, g_fp32, 1, 0, NULL, &state) || (a[4] != Py_None && !PyLong_Check(a[4]) && is_placed(a[4], "conv", dev, 1)) ||
      as_ptr(a[4], &conv) || as_tensor(a[7], "req_idx", dev, g_int32, 0, beams, NULL, &req) ||
      as_tensor(a[8], "parent", dev, g_int32, 0, beams, NULL, &parent) || as_tensor(a[13], "new_idx", dev, g_int32, 0, beams, NULL, &to) ||
      as_tensor(a[14], "src_idx", dev, g_int32, 0, beams, NULL, &src) || as_stream(a[15], &stream))
    return NULL;
  dasc_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = dasc_beam_reorder(plan, state, ls, rs, conv, cs, cb, req, parent, i[0], i[1], i[2], i[3], to, src, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

#define M(name, fn) {name, (PyCFunction)(void (*)(void))fn, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {
    M("init", py_init), M("pack", py_pack), M("pack_padded", py_pack_padded), M("pack_int8", py_pack_int8),
    M("restore", py_restore), M("restore_padded", py_restore_padded), M("restore_int8", py_restore_int8),
    M("refresh", py_refresh), M("refresh_window", py_refresh_window),
    M("decay_attn", py_decay_attn), M("decay_step", py_decay_step), M("verify_draft", py_verify_draft),
    M("delta_step", py_delta_step), M("delta_draft", py_delta_draft), M("beam_select", py_beam_select), M("beam_reorder", py_beam_reorder), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_dasccall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__dasccall(void) {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_numel = PyUnicode_InternFromString("numel");
  s_element_size = PyUnicode_InternFromString("element_size");
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_get_device = PyUnicode_InternFromString("get_device");
  if (!s_data_ptr || !s_numel || !s_element_size || !s_cuda_stream || !s_dtype || !s_is_contiguous || !s_get_device) return NULL;
  return PyModule_Create(&module);
}
