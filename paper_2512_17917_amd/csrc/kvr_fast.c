/* The calls of a decode step (the compressed cache's two, and those that put a token into an uncompressed cache and attend
 * over it) without the interpreter between the checks: the same checks of every tensor that
 * binding._ptr makes (that it is one, type, place, contiguity, size), made through the tensor's own attributes, and the call itself.  A
 * check that fails, or an argument of an unexpected kind, returns None: the caller then takes the Python path, which
 * says what is wrong.  Nothing is kept between calls but the names, the types and the five entry points. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/kvr.h"

typedef int32_t (*step_fn)(const kvr_desc*, const void*, const void*, const int32_t*, void*, void*, int32_t*, int32_t,
                           const float*, int64_t, int32_t, int32_t, int32_t*, int32_t*, int32_t*, int32_t, int32_t*,
                           int32_t*, int32_t, void*, void*, void*);
typedef int32_t (*attend_fn)(const kvr_desc*, const void*, const void*, const void*, const int32_t*, int32_t,
                             const void*, const void*, const int32_t*, const int32_t*, int32_t, float*, float*, int64_t,
                             void*, size_t, const kvr_attend_opts*, void*);

typedef int32_t (*rotate_fn)(const kvr_desc*, const kvr_rotation*, const void*, int64_t, const void*, int64_t, const void*, int64_t,
                             int32_t, const int32_t*, const int32_t*, void*, void*, const kvr_pages*, void*);
typedef int32_t (*paged_fn)(const kvr_desc*, const void*, const int32_t*, const kvr_pages*, int32_t, int32_t, void*, float*,
                            int64_t, void*, size_t, void*);

typedef int32_t (*prompt_fn)(const kvr_desc*, const void*, int32_t, const int32_t*, const int32_t*, const kvr_pages*, int32_t, int32_t,
                             void*, float*, int64_t, void*, size_t, void*);

typedef int32_t (*rotate_axes_fn)(const kvr_desc*, const kvr_rotation*, const kvr_axes*, const int32_t*, int64_t, const void*, int64_t,
                                  const void*, int64_t, const void*, int64_t, int32_t, const int32_t*, const int32_t*, void*, void*,
                                  const kvr_pages*, void*);

typedef int32_t (*shared_fn)(const kvr_desc*, const void*, int32_t, const int32_t*, const int32_t*, const kvr_pages*, const kvr_groups*,
                             int32_t, int32_t, void*, float*, int64_t, void*, size_t, void*);

static prompt_fn f_prompt;
static shared_fn f_shared;
static rotate_axes_fn f_rotate_axes;
static PyObject *n_get_device, *n_shape, *n_stride;
static rotate_fn f_rotate;
static paged_fn f_paged;
static PyObject *n_dtype, *n_is_cuda, *n_is_contiguous, *n_numel, *n_data_ptr;
static PyObject *t_f32, *t_bf16, *t_i32, *t_u8, *t_tensor;
static step_fn f_step;
static attend_fn f_attend;

static int integer(PyObject* o, int64_t* v) {
  if (!PyLong_CheckExact(o)) return 0;
  *v = PyLong_AsLongLong(o);
  return !(*v == -1 && PyErr_Occurred());
}

static int asked(PyObject* t, PyObject* name, int64_t* v) {          /* an integer method without arguments */
  PyObject* r = PyObject_CallMethodNoArgs(t, name);
  const int ok = r && integer(r, v);
  Py_XDECREF(r);
  return ok;
}

static int truth(PyObject* r) {
  const int yes = r == Py_True;
  Py_XDECREF(r);
  return yes;
}

/* device address of a contiguous tensor of that type with at least `need` elements; numel may be null */
static int tensor(PyObject* t, PyObject* dtype, int64_t need, int none_ok, void** p, int64_t* numel) {
  int64_t n, a;
  *p = NULL;
  if (t == Py_None) return none_ok;
  if (PyObject_IsInstance(t, t_tensor) != 1) return 0;
  PyObject* dt = PyObject_GetAttr(t, n_dtype);
  const int same = dt == dtype;
  Py_XDECREF(dt);
  if (!same || !truth(PyObject_GetAttr(t, n_is_cuda)) || !truth(PyObject_CallMethodNoArgs(t, n_is_contiguous))) return 0;
  if (!asked(t, n_numel, &n) || n < need || !asked(t, n_data_ptr, &a)) return 0;
  *p = (void*)(uintptr_t)a;
  if (numel) *numel = n;
  return 1;
}

/* The products of sizes that the checks form stay within 64 bits: the descriptor's are what the library takes at most, every
 * count fits 32 bits.  Others go to the Python checks, whose integers have no end. */
static int sizes_fit(const kvr_desc* d, const int64_t* count, int n) {
  const int64_t U = (int64_t)d->batch * d->n_kv_heads, H = (int64_t)d->batch * d->n_q_heads;
  if (U > 65535 || H > 8 * 65535 || d->head_dim != KVR_HEAD_DIM || d->r > KVR_MAX_ROWS || d->w > 65536) return 0;
  for (int i = 0; i < n; ++i)
    if (count[i] != (int32_t)count[i]) return 0;
  return 1;
}

static PyObject* refuse(void) {
  PyErr_Clear();
  Py_RETURN_NONE;
}

static PyObject* setup(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t s, t;
  if (n != 7 || !integer(a[0], &s) || !integer(a[1], &t)) return PyErr_Format(PyExc_TypeError, "setup");
  f_step = (step_fn)(uintptr_t)s;
  f_attend = (attend_fn)(uintptr_t)t;
  for (int i = 2; i < 7; ++i) Py_INCREF(a[i]);
  t_f32 = a[2]; t_bf16 = a[3]; t_i32 = a[4]; t_u8 = a[5]; t_tensor = a[6];
  Py_RETURN_NONE;
}

/* desc address, stream, then the arguments of binding.kvr_step_update behind desc */
static PyObject* step_update(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t da, st, ret_cap, n_cap, n_recent, k_cand, evict_cap, vague_cap;
  void *kn, *vn, *nc, *kr, *vr, *rp, *sc, *es, *ep, *ne, *vp, *nv, *sk, *sv;
  if (n != 22 || !f_step || !integer(a[0], &da) || !integer(a[1], &st) || !integer(a[8], &ret_cap) || !integer(a[10], &n_cap) ||
      !integer(a[11], &n_recent) || !integer(a[12], &k_cand) || !integer(a[16], &evict_cap) || !integer(a[19], &vague_cap))
    return refuse();
  const kvr_desc* d = (const kvr_desc*)(uintptr_t)da;
  if (!sizes_fit(d, (int64_t[]){ret_cap, n_cap, n_recent, k_cand, evict_cap, vague_cap}, 6)) return refuse();
  PyObject* dt = d->dtype == KVR_F32 ? t_f32 : t_bf16;
  const int64_t U = (int64_t)d->batch * d->n_kv_heads, D = d->head_dim, S = (int64_t)d->r * d->w * D;
  if (!tensor(a[2], dt, U * D, 0, &kn, 0) || !tensor(a[3], dt, U * D, 0, &vn, 0) || !tensor(a[4], t_i32, d->batch, 0, &nc, 0) ||
      !tensor(a[5], dt, U * ret_cap * D, 0, &kr, 0) || !tensor(a[6], dt, U * ret_cap * D, 0, &vr, 0) ||
      !tensor(a[7], t_i32, U * ret_cap, 0, &rp, 0) || !tensor(a[9], t_f32, U * n_cap, 0, &sc, 0) ||
      !tensor(a[13], t_i32, U * evict_cap, 0, &es, 0) || !tensor(a[14], t_i32, U * evict_cap, 0, &ep, 0) ||
      !tensor(a[15], t_i32, U, 0, &ne, 0) || !tensor(a[17], t_i32, U * vague_cap, 1, &vp, 0) || !tensor(a[18], t_i32, U, 1, &nv, 0) ||
      !tensor(a[20], dt, U * S, 0, &sk, 0) || !tensor(a[21], dt, U * S, 0, &sv, 0))
    return refuse();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f_step(d, kn, vn, nc, kr, vr, rp, (int32_t)ret_cap, sc, n_cap, (int32_t)n_recent, (int32_t)k_cand, es, ep, ne,
              (int32_t)evict_cap, vp, nv, (int32_t)vague_cap, sk, sv, (void*)(uintptr_t)st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* desc address, stream, address of the options (0: none), then the arguments of binding.kvr_attend_decode from q to ws */
static PyObject* attend_decode(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t da, st, op, ret_cap, n_cap, vague_cap, wb = 0;
  void *q, *kr, *vr, *rp, *sk, *sv, *vp, *nv, *out, *sc, *ws;
  if (n != 17 || !f_attend || !integer(a[0], &da) || !integer(a[1], &st) || !integer(a[2], &op) || !integer(a[7], &ret_cap) ||
      !integer(a[12], &vague_cap) || !integer(a[15], &n_cap))
    return refuse();
  const kvr_desc* d = (const kvr_desc*)(uintptr_t)da;
  if (!sizes_fit(d, (int64_t[]){ret_cap, vague_cap, n_cap}, 3)) return refuse();
  PyObject* dt = d->dtype == KVR_F32 ? t_f32 : t_bf16;
  const int64_t U = (int64_t)d->batch * d->n_kv_heads, D = d->head_dim, S = (int64_t)d->r * d->w * D, H = (int64_t)d->batch * d->n_q_heads;
  if (!tensor(a[3], dt, H * D, 0, &q, 0) || !tensor(a[4], dt, U * ret_cap * D, 0, &kr, 0) ||
      !tensor(a[5], dt, U * ret_cap * D, 0, &vr, 0) || !tensor(a[6], t_i32, U * ret_cap, 1, &rp, 0) ||
      !tensor(a[8], dt, U * S, 1, &sk, 0) || !tensor(a[9], dt, U * S, 1, &sv, 0) || !tensor(a[10], t_i32, U * vague_cap, 1, &vp, 0) ||
      !tensor(a[11], t_i32, U, 1, &nv, 0) || !tensor(a[13], t_f32, H * D, 0, &out, 0) || !tensor(a[14], t_f32, U * n_cap, 1, &sc, 0) ||
      !tensor(a[16], t_u8, 0, 0, &ws, &wb))
    return refuse();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f_attend(d, q, kr, vr, rp, (int32_t)ret_cap, sk, sv, vp, nv, (int32_t)vague_cap, out, sc, n_cap, ws, (size_t)wb,
                (const kvr_attend_opts*)(uintptr_t)op, (void*)(uintptr_t)st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* as binding._here: the tensor lives on the current device */
static int here(PyObject* t, int64_t dev) {
  int64_t at;
  return t == Py_None || (asked(t, n_get_device, &at) && at == dev);
}

static int item(PyObject* seq, Py_ssize_t i, int64_t* v) {
  return PyTuple_Check(seq) && PyTuple_GET_SIZE(seq) == 3 && integer(PyTuple_GET_ITEM(seq, i), v);
}

/* as binding._rows: device address and row stride of [n_rows or more, heads, D] with dense heads */
static int rows(PyObject* t, PyObject* dtype, int64_t n_rows, int64_t heads, int64_t D, int64_t dev, void** p, int64_t* stride) {
  int64_t n0, n1, n2, s0, s1, s2, a;
  *p = NULL;
  *stride = 0;
  if (t == Py_None) return 1;
  if (PyObject_IsInstance(t, t_tensor) != 1) return 0;
  PyObject* dt = PyObject_GetAttr(t, n_dtype);
  const int same = dt == dtype;
  Py_XDECREF(dt);
  if (!same || !truth(PyObject_GetAttr(t, n_is_cuda)) || !here(t, dev)) return 0;
  PyObject* shape = PyObject_GetAttr(t, n_shape);
  int ok = shape && item(shape, 0, &n0) && item(shape, 1, &n1) && item(shape, 2, &n2);
  Py_XDECREF(shape);
  if (!ok || n0 < n_rows || n1 != heads || n2 != D) return 0;
  PyObject* strides = PyObject_CallMethodNoArgs(t, n_stride);
  ok = strides && item(strides, 0, &s0) && item(strides, 1, &s1) && item(strides, 2, &s2);
  Py_XDECREF(strides);
  if (!ok || s2 != 1 || (heads > 1 && s1 != D) || !asked(t, n_data_ptr, &a)) return 0;
  *p = (void*)(uintptr_t)a;
  *stride = n_rows > 1 ? s0 : heads * D;
  return 1;
}

static PyObject* setup_cache(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t r, p, m;
  if (n != 3 || !integer(a[0], &r) || !integer(a[1], &p) || !integer(a[2], &m)) return PyErr_Format(PyExc_TypeError, "setup_cache");
  f_rotate = (rotate_fn)(uintptr_t)r;
  f_paged = (paged_fn)(uintptr_t)p;
  f_prompt = (prompt_fn)(uintptr_t)m;
  Py_RETURN_NONE;
}

static PyObject* setup_more(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t r, t;
  if (n != 2 || !integer(a[0], &r) || !integer(a[1], &t)) return PyErr_Format(PyExc_TypeError, "setup_more");
  f_rotate_axes = (rotate_axes_fn)(uintptr_t)r;
  f_shared = (shared_fn)(uintptr_t)t;
  Py_RETURN_NONE;
}

/* device address and stride of positions [n_axes or more, n_rows or more] with dense rows; none where no pair is turned */
static int positions(PyObject* t, int64_t n_axes, int64_t n_rows, int64_t dev, int none_ok, void** p, int64_t* stride) {
  int64_t n0, n1, s0, s1, a;
  *p = NULL;
  *stride = 0;
  if (t == Py_None) return none_ok;
  if (PyObject_IsInstance(t, t_tensor) != 1) return 0;
  PyObject* dt = PyObject_GetAttr(t, n_dtype);
  const int same = dt == t_i32;
  Py_XDECREF(dt);
  if (!same || !truth(PyObject_GetAttr(t, n_is_cuda)) || !here(t, dev)) return 0;
  PyObject* shape = PyObject_GetAttr(t, n_shape);
  int ok = shape && PyTuple_Check(shape) && PyTuple_GET_SIZE(shape) == 2 && integer(PyTuple_GET_ITEM(shape, 0), &n0) &&
           integer(PyTuple_GET_ITEM(shape, 1), &n1);
  Py_XDECREF(shape);
  if (!ok || n0 < n_axes || n1 < n_rows) return 0;
  PyObject* strides = PyObject_CallMethodNoArgs(t, n_stride);
  ok = strides && PyTuple_Check(strides) && PyTuple_GET_SIZE(strides) == 2 && integer(PyTuple_GET_ITEM(strides, 0), &s0) &&
       integer(PyTuple_GET_ITEM(strides, 1), &s1);
  Py_XDECREF(strides);
  if (!ok || (s1 != 1 && n1 > 1) || !asked(t, n_data_ptr, &a)) return 0;
  *p = (void*)(uintptr_t)a;
  *stride = s0;
  return 1;
}

/* addresses of desc, rotation and pages (0: none), current device, stream, then binding.kvr_rotate's arguments from q to k_out; for
 * kvr_rotate_axes the address of the axes and the positions behind them */
static PyObject* rotate_any(PyObject* const* a, Py_ssize_t n, int with_axes) {
  int64_t da, ra, pa, dev, st, n_rows, qs, ks, vs, xa = 0, xs = 0;
  void *q, *k, *v, *start, *nc, *qo, *ko, *pos = NULL;
  if (n != (with_axes ? 15 : 13) || !(with_axes ? f_rotate_axes != NULL : f_rotate != NULL) || !integer(a[0], &da) ||
      !integer(a[1], &ra) || !integer(a[2], &pa) || !integer(a[3], &dev) || !integer(a[4], &st) || !integer(a[8], &n_rows) ||
      (with_axes && !integer(a[13], &xa)))
    return refuse();
  const kvr_desc* d = (const kvr_desc*)(uintptr_t)da;
  const kvr_rotation* rot = (const kvr_rotation*)(uintptr_t)ra;
  const kvr_axes* axes = (const kvr_axes*)(uintptr_t)xa;
  if (!sizes_fit(d, (int64_t[]){n_rows}, 1) || n_rows < 0) return refuse();
  PyObject* dt = d->dtype == KVR_F32 ? t_f32 : t_bf16;
  const int64_t D = d->head_dim, Hq = d->n_q_heads, Hkv = d->n_kv_heads;
  if (!rows(a[5], dt, n_rows, Hq, D, dev, &q, &qs) || !rows(a[6], dt, n_rows, Hkv, D, dev, &k, &ks) ||
      !rows(a[7], dt, n_rows, Hkv, D, dev, &v, &vs) || !tensor(a[9], t_i32, d->batch + 1, 1, &start, 0) ||
      !tensor(a[10], t_i32, d->batch, with_axes && pa == 0, &nc, 0) || !tensor(a[11], dt, n_rows * Hq * D, 1, &qo, 0) ||
      !tensor(a[12], dt, n_rows * Hkv * D, 1, &ko, 0) || !here(a[9], dev) || !here(a[10], dev) || !here(a[11], dev) || !here(a[12], dev) ||
      (with_axes && !positions(a[14], axes->n_axes, n_rows, dev, rot->rot_dim == 0, &pos, &xs)))
    return refuse();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  if (with_axes)
    rc = f_rotate_axes(d, rot, axes, pos, xs, q, qs, k, ks, v, vs, (int32_t)n_rows, start, nc, qo, ko, (const kvr_pages*)(uintptr_t)pa,
                       (void*)(uintptr_t)st);
  else
    rc = f_rotate(d, rot, q, qs, k, ks, v, vs, (int32_t)n_rows, start, nc, qo, ko, (const kvr_pages*)(uintptr_t)pa, (void*)(uintptr_t)st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
static PyObject* rotate(PyObject* self, PyObject* const* a, Py_ssize_t n) { return rotate_any(a, n, 0); }
static PyObject* rotate_axes(PyObject* self, PyObject* const* a, Py_ssize_t n) { return rotate_any(a, n, 1); }

/* addresses of desc and pages, current device, stream, then binding.kvr_attend_paged's arguments without pages */
static PyObject* attend_paged(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  int64_t da, pa, dev, st, window, n_sink, n_cap, wb = 0;
  void *q, *nc, *out, *sc, *ws;
  if (n != 12 || !f_paged || !integer(a[0], &da) || !integer(a[1], &pa) || !integer(a[2], &dev) || !integer(a[3], &st) ||
      !integer(a[6], &window) || !integer(a[7], &n_sink) || !integer(a[10], &n_cap))
    return refuse();
  const kvr_desc* d = (const kvr_desc*)(uintptr_t)da;
  if (!sizes_fit(d, (int64_t[]){window, n_sink, n_cap}, 3)) return refuse();
  PyObject* dt = d->dtype == KVR_F32 ? t_f32 : t_bf16;
  const int64_t U = (int64_t)d->batch * d->n_kv_heads, H = (int64_t)d->batch * d->n_q_heads, D = d->head_dim;
  if (!tensor(a[4], dt, H * D, 0, &q, 0) || !tensor(a[5], t_i32, d->batch, 0, &nc, 0) || !tensor(a[8], dt, H * D, 0, &out, 0) ||
      !tensor(a[9], t_f32, U * n_cap, 1, &sc, 0) || !tensor(a[11], t_u8, 0, 1, &ws, &wb) || !here(a[4], dev) || !here(a[5], dev) ||
      !here(a[8], dev) || !here(a[9], dev) || !here(a[11], dev))
    return refuse();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f_paged(d, q, nc, (const kvr_pages*)(uintptr_t)pa, (int32_t)window, (int32_t)n_sink, out, sc, n_cap, ws, (size_t)wb,
               (void*)(uintptr_t)st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* addresses of desc and pages, current device, stream, then binding.kvr_attend_prompt's arguments without pages; for kvr_attend_shared
 * the address of the groups (0: none) behind them */
static PyObject* attend_rows(PyObject* const* a, Py_ssize_t n, int shared) {
  int64_t da, pa, dev, st, n_rows, window, n_sink, n_cap, ga = 0, wb = 0;
  void *q, *start, *nc, *out, *sc, *ws;
  if (n != (shared ? 15 : 14) || !(shared ? f_shared != NULL : f_prompt != NULL) || !integer(a[0], &da) || !integer(a[1], &pa) ||
      !integer(a[2], &dev) || !integer(a[3], &st) || !integer(a[5], &n_rows) || !integer(a[8], &window) || !integer(a[9], &n_sink) ||
      !integer(a[12], &n_cap) || (shared && !integer(a[14], &ga)))
    return refuse();
  const kvr_desc* d = (const kvr_desc*)(uintptr_t)da;
  if (!sizes_fit(d, (int64_t[]){n_rows, window, n_sink, n_cap}, 4) || n_rows < 0) return refuse();
  PyObject* dt = d->dtype == KVR_F32 ? t_f32 : t_bf16;
  const int64_t U = (int64_t)d->batch * d->n_kv_heads, H = n_rows * d->n_q_heads, D = d->head_dim;
  if (!tensor(a[4], dt, H * D, 0, &q, 0) || !tensor(a[6], t_i32, d->batch + 1, 1, &start, 0) || !tensor(a[7], t_i32, d->batch, 0, &nc, 0) ||
      !tensor(a[10], dt, H * D, 0, &out, 0) || !tensor(a[11], t_f32, U * n_cap, 1, &sc, 0) || !tensor(a[13], t_u8, 0, 1, &ws, &wb) ||
      !here(a[4], dev) || !here(a[6], dev) || !here(a[7], dev) || !here(a[10], dev) || !here(a[11], dev) || !here(a[13], dev))
    return refuse();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  if (shared)
    rc = f_shared(d, q, (int32_t)n_rows, start, nc, (const kvr_pages*)(uintptr_t)pa, (const kvr_groups*)(uintptr_t)ga, (int32_t)window,
                  (int32_t)n_sink, out, sc, n_cap, ws, (size_t)wb, (void*)(uintptr_t)st);
  else
    rc = f_prompt(d, q, (int32_t)n_rows, start, nc, (const kvr_pages*)(uintptr_t)pa, (int32_t)window, (int32_t)n_sink, out, sc, n_cap, ws,
                  (size_t)wb, (void*)(uintptr_t)st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
static PyObject* attend_prompt(PyObject* self, PyObject* const* a, Py_ssize_t n) { return attend_rows(a, n, 0); }
static PyObject* attend_shared(PyObject* self, PyObject* const* a, Py_ssize_t n) { return attend_rows(a, n, 1); }

static PyMethodDef methods[] = {{"setup", (PyCFunction)(void*)setup, METH_FASTCALL, 0},
                                {"step_update", (PyCFunction)(void*)step_update, METH_FASTCALL, 0},
                                {"attend_decode", (PyCFunction)(void*)attend_decode, METH_FASTCALL, 0},
                                {"setup_cache", (PyCFunction)(void*)setup_cache, METH_FASTCALL, 0},
                                {"setup_more", (PyCFunction)(void*)setup_more, METH_FASTCALL, 0},
                                {"rotate_axes", (PyCFunction)(void*)rotate_axes, METH_FASTCALL, 0},
                                {"rotate", (PyCFunction)(void*)rotate, METH_FASTCALL, 0},
                                {"attend_paged", (PyCFunction)(void*)attend_paged, METH_FASTCALL, 0},
                                {"attend_shared", (PyCFunction)(void*)attend_shared, METH_FASTCALL, 0},
                                {"attend_prompt", (PyCFunction)(void*)attend_prompt, METH_FASTCALL, 0},
                                {0, 0, 0, 0}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kvr_fast", 0, -1, methods, 0, 0, 0, 0};

PyMODINIT_FUNC PyInit__kvr_fast(void) {
  n_dtype = PyUnicode_InternFromString("dtype");
  n_is_cuda = PyUnicode_InternFromString("is_cuda");
  n_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  n_numel = PyUnicode_InternFromString("numel");
  n_data_ptr = PyUnicode_InternFromString("data_ptr");
  n_get_device = PyUnicode_InternFromString("get_device");
  n_shape = PyUnicode_InternFromString("shape");
  n_stride = PyUnicode_InternFromString("stride");
  return PyModule_Create(&module);
}
