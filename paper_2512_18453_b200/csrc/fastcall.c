/* The binding's hot calls as a CPython extension: tensor checks, pointers, sizes and the current stream are
 * collected here instead of attribute by attribute in Python and through ctypes.  A three-kernel layer call spends
 * 7 us in its launches; the Python and ctypes work around it took 3.1 us, this takes 0.9 (a 16 x 16 layer in one
 * kernel: 5.9 -> 3.9 us per call).  The library's functions arrive as addresses, so that there is one copy of libnova. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "nova.h"

static struct {
  __typeof__(&nova_conv2d_fwd) conv2d;
  __typeof__(&nova_filter_transform) filter;
  __typeof__(&nova_conv2d_fwd_int8) int8;
  __typeof__(&nova_causal_conv1d) causal;
  __typeof__(&nova_selective_scan) scan;
  __typeof__(&nova_linear_int4) linear;
} fn;
static PyObject *get_device, *get_stream;                 /* torch's accessors of the current device and stream */
static PyObject *t_types[3], *t_int32, *t_uint8, *t_bool; /* torch's types: float32, float16, bfloat16, .. */
static PyObject* empty_strided;   /* torch's (size, stride, type) -> tensor on the current device, or None; 0.8 us where new_empty takes 1.9 */
static PyObject *s_get_device, *s_stride, *s_new_empty;
static PyObject *s_is_cuda, *s_is_contiguous, *s_dtype, *s_shape, *s_data_ptr, *s_numel;

/* 1 if `t` is a contiguous CUDA tensor of `dtype`; 0 with AssertionError set, or -1 with another error */
static int check(PyObject* t, PyObject* dtype) {
  PyObject* v = PyObject_GetAttr(t, s_is_cuda);
  if (!v) return -1;
  int ok = v == Py_True;
  Py_DECREF(v);
  if (ok) {
    if (!(v = PyObject_CallMethodNoArgs(t, s_is_contiguous))) return -1;
    ok = v == Py_True;
    Py_DECREF(v);
  }
  if (ok) {
    if (!(v = PyObject_GetAttr(t, s_dtype))) return -1;
    ok = v == dtype;
    Py_DECREF(v);
  }
  if (!ok) PyErr_SetString(PyExc_AssertionError, "a contiguous CUDA tensor of the plan's storage type is needed");
  return ok;
}
/* the first `count` sizes of a tensor; `exact`: it has no more dimensions */
static int shape(PyObject* t, long long* out, Py_ssize_t count, int exact) {
  PyObject* s = PyObject_GetAttr(t, s_shape);
  if (!s) return 0;
  int ok = PyTuple_Check(s) && (exact ? PyTuple_GET_SIZE(s) == count : PyTuple_GET_SIZE(s) >= count);
  for (Py_ssize_t i = 0; ok && i < count; ++i) {
    out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(s, i));
    if (out[i] < 0 || out[i] > INT32_MAX) ok = 0;
  }
  Py_DECREF(s);
  if (!ok && !PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "a tensor of %zd dimensions is needed", count);
  return ok;
}
static int integer(PyObject* t, PyObject* method, unsigned long long* out) {
  PyObject* v = PyObject_CallMethodNoArgs(t, method);
  if (!v) return 0;
  *out = PyLong_AsUnsignedLongLong(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}
static int pointer(PyObject* t, void** out) {
  unsigned long long v;
  if (!integer(t, s_data_ptr, &v)) return 0;
  *out = (void*)(uintptr_t)v;
  return 1;
}
static int stream(nova_stream* out) {
  PyObject* dev = PyObject_CallNoArgs(get_device);
  if (!dev) return 0;
  PyObject* s = PyObject_CallOneArg(get_stream, dev);
  Py_DECREF(dev);
  if (!s) return 0;
  *out = (nova_stream)(uintptr_t)PyLong_AsUnsignedLongLong(s);
  Py_DECREF(s);
  return !PyErr_Occurred();
}

/* conv2d(plan, dtype, x, U, y, workspace, flags) -> status */
static PyObject* conv2d(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  long long d[4], u[2];
  void *x, *U, *y, *ws;
  unsigned long long bytes;
  nova_stream st;
  if (n != 7) return PyErr_Format(PyExc_TypeError, "seven arguments are needed");
  const nova_plan* plan = (const nova_plan*)PyLong_AsVoidPtr(a[0]);
  if (PyErr_Occurred()) return NULL;
  if (check(a[2], a[1]) != 1 || !shape(a[2], d, 4, 1) || !shape(a[3], u, 2, 0) || !pointer(a[2], &x) || !pointer(a[3], &U) ||
      !pointer(a[4], &y) || !pointer(a[5], &ws) || !integer(a[5], s_numel, &bytes))
    return NULL;
  const long flags = PyLong_AsLong(a[6]);
  if (PyErr_Occurred() || !stream(&st)) return NULL;
  int r;
  Py_BEGIN_ALLOW_THREADS
  r = fn.conv2d(plan, x, U, y, (int)d[0], (int)d[1], (int)d[2], (int)d[3], (int)u[1], ws, (size_t)bytes, (int)flags, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(r);
}

/* filter_transform(plan, g, K, C, U) -> status */
static PyObject* filter_transform(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *g, *U;
  nova_stream st;
  if (n != 5) return PyErr_Format(PyExc_TypeError, "five arguments are needed");
  const nova_plan* plan = (const nova_plan*)PyLong_AsVoidPtr(a[0]);
  const long K = PyLong_AsLong(a[2]), C = PyLong_AsLong(a[3]);
  if (PyErr_Occurred() || !pointer(a[1], &g) || !pointer(a[4], &U) || !stream(&st)) return NULL;
  int r;
  Py_BEGIN_ALLOW_THREADS
  r = fn.filter(plan, g, (int)K, (int)C, U, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(r);
}

/* conv2d_int8(plan, x, Uq, scale_U, scale_V, y, workspace, N, H, W, C, K, flags) -> status */
static PyObject* conv2d_int8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  void *x, *U, *y, *ws, *sU;
  unsigned long long bytes;
  nova_stream st;
  long v[6];
  if (n != 13) return PyErr_Format(PyExc_TypeError, "thirteen arguments are needed");
  const nova_plan* plan = (const nova_plan*)PyLong_AsVoidPtr(a[0]);
  const double sV = PyFloat_AsDouble(a[4]);
  for (int i = 0; i < 6; ++i) v[i] = PyLong_AsLong(a[7 + i]);
  if (PyErr_Occurred() || !pointer(a[1], &x) || !pointer(a[2], &U) || !pointer(a[3], &sU) || !pointer(a[5], &y) ||
      !pointer(a[6], &ws) || !integer(a[6], s_numel, &bytes) || !stream(&st))
    return NULL;
  int r;
  Py_BEGIN_ALLOW_THREADS
  r = fn.int8(plan, x, U, (const float*)sU, (float)sV, y, (int)v[0], (int)v[1], (int)v[2], (int)v[3], (int)v[4], ws,
              (size_t)bytes, (int)v[5], st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(r);
}

/* ---- token mixers.  What these take is what the Python functions of the same names accept; for anything else, and so for every
 * mistake, they return None, and the Python functions check argument by argument and say what is wrong.  A status other than 0
 * is returned as a number. */
typedef struct {
  void* p;
  int dims;
  long long size[4], stride[4];
} Tensor;
static int tuple_of(PyObject* o, long long* out, int most) {
  if (!o || !PyTuple_Check(o)) return -1;
  const Py_ssize_t n = PyTuple_GET_SIZE(o);
  if (n > most) return -1;
  for (Py_ssize_t i = 0; i < n; ++i) out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
  return (int)n;
}
/* a tensor of `dtype` on device `dev` whose columns are contiguous; `whole`: all of it is, and the strides are not asked for */
static int tensor(PyObject* o, PyObject* dtype, long dev, int whole, Tensor* t) {
  PyObject* v = PyObject_CallMethodNoArgs(o, s_get_device);
  if (!v) return 0;
  const long d = PyLong_AsLong(v);
  Py_DECREF(v);
  if (d != dev || d < 0 || !(v = PyObject_GetAttr(o, s_dtype))) return 0;
  const int same = v == dtype;
  Py_DECREF(v);
  if (!same) return 0;
  v = PyObject_GetAttr(o, s_shape);
  t->dims = tuple_of(v, t->size, 4);
  Py_XDECREF(v);
  if (t->dims < 1) return 0;
  v = PyObject_CallMethodNoArgs(o, whole ? s_is_contiguous : s_stride);
  const int n = whole ? t->dims : tuple_of(v, t->stride, 4), ok = !whole || v == Py_True;
  Py_XDECREF(v);
  if (!ok || n != t->dims || PyErr_Occurred() || !pointer(o, &t->p)) return 0;
  return whole || t->size[n - 1] <= 1 || t->stride[n - 1] == 1;
}
static int vector(PyObject* o, PyObject* dtype, long dev, long long n, const void** p) {
  Tensor t;
  if (o == Py_None) return *p = NULL, 1;
  if (!tensor(o, dtype, dev, 1, &t) || t.dims != 1 || t.size[0] != n) return 0;
  *p = t.p;
  return 1;
}
/* the type of a tensor, its place in t_types, or -1 */
static int type_of(PyObject* o) {
  PyObject* v = PyObject_GetAttr(o, s_dtype);
  int r = -1;
  for (int i = 0; v && i < 3; ++i)
    if (v == t_types[i]) r = i;
  Py_XDECREF(v);
  return r;
}
typedef struct {
  int lead, step;                 /* leading dimensions of a token tensor; single tokens */
  long long n[2], channels;
  long dev;
  nova_sequences q;
} Call;
static int token_rows(PyObject* o, PyObject* dtype, const Call* c, int inner, const long long* cols, nova_rows* r, int64_t* group) {
  Tensor t;
  if (!tensor(o, dtype, c->dev, 0, &t) || t.dims != c->lead + inner) return 0;
  for (int i = 0; i < c->lead; ++i)
    if (t.size[i] != c->n[i]) return 0;
  for (int i = 0; i < inner; ++i)
    if (t.size[c->lead + i] != cols[i]) return 0;
  r->data_dev = t.p;
  r->row_stride = c->step ? 0 : t.stride[c->lead - 1];
  r->seq_stride = c->step || c->lead == 2 ? t.stride[0] : 0;
  if (group) *group = inner == 2 ? t.stride[c->lead] : 0;
  return 1;
}
/* sequences, x's leading sizes and the state's slots; state [slots, a, b] of state_dtype is checked by the caller for a and b */
static int sequences(Call* c, PyObject* x, PyObject* dtype, PyObject* state, PyObject* state_dtype, Tensor* st, PyObject* cu, PyObject* slots,
                     PyObject* resume, int step, nova_rows* xr) {
  Tensor t;
  PyObject* d = PyObject_CallNoArgs(get_device);
  if (!d) return 0;
  c->dev = PyLong_AsLong(d);
  Py_DECREF(d);
  c->step = step;
  c->lead = step || cu != Py_None ? 1 : 2;
  if (!tensor(x, dtype, c->dev, 0, &t) || t.dims != c->lead + 1) return 0;
  c->n[0] = t.size[0];
  c->n[1] = t.size[1];
  c->channels = t.size[c->lead];
  memset(&c->q, 0, sizeof c->q);
  long long count = t.size[0], tokens = step ? 1 : c->lead == 2 ? t.size[1] : t.size[0];
  if (cu != Py_None) {
    Tensor b;
    if (!tensor(cu, t_int32, c->dev, 1, &b) || b.dims != 1 || b.size[0] < 1) return 0;
    c->q.cu_seqlens_dev = (const int32_t*)b.p;
    count = b.size[0] - 1;
  }
  if (count > INT32_MAX || c->channels > INT32_MAX) return 0;
  c->q.sequences = (int32_t)count;
  c->q.tokens = tokens;
  if (state == Py_None) {
    if (slots != Py_None || resume != Py_None) return 0;
  } else {
    const void* p;
    if (!tensor(state, state_dtype, c->dev, 1, st) || st->dims != 3) return 0;
    c->q.slots = st->size[0];
    if (slots == Py_None && c->q.slots < count) return 0;
    if (!vector(slots, t_int32, c->dev, count, &p)) return 0;
    c->q.slots_dev = (const int32_t*)p;
    if (!vector(resume, t_bool, c->dev, count, &p)) return 0;
    c->q.resume_dev = (const uint8_t*)p;
  }
  xr->data_dev = t.p;
  xr->row_stride = step ? 0 : t.stride[c->lead - 1];
  xr->seq_stride = c->lead == 2 || step ? t.stride[0] : 0;
  return 1;
}
/* a new reference to `out`, or to a new tensor like x of these sizes; rows that overlap are left to Python */
static PyObject* output(PyObject* out, PyObject* x, const long long* n, int lead, long long cols, PyObject* dtype, long dev, Tensor* t) {
  if (out != Py_None) {
    Py_INCREF(out);
  } else {
    PyObject *size = PyTuple_New(lead + 1), *step = PyTuple_New(lead + 1);
    long long apart = 1;
    for (int i = lead; size && step && i >= 0; --i) {
      const long long v = i < lead ? n[i] : cols;
      PyTuple_SET_ITEM(size, i, PyLong_FromLongLong(v));
      PyTuple_SET_ITEM(step, i, PyLong_FromLongLong(apart));
      apart *= v > 1 ? v : 1;
    }
    PyObject* args[3] = {size, step, dtype};
    out = !size || !step || PyErr_Occurred() ? NULL
          : empty_strided != Py_None ? PyObject_Vectorcall(empty_strided, args, 3, NULL) : PyObject_CallMethodOneArg(x, s_new_empty, size);
    Py_XDECREF(size);
    Py_XDECREF(step);
    if (!out) return NULL;
  }
  int ok = tensor(out, dtype, dev, 0, t) && t->dims == lead + 1 && t->size[lead] == cols;
  for (int i = 0; ok && i < lead; ++i) ok = t->size[i] == n[i];
  const int near = lead == 2 && (n[0] <= 1 || (n[1] > 1 && t->stride[1] <= t->stride[0]));      /* the dimension of the smaller stride */
  long long wide = cols;                                                                        /* of what the other one repeats */
  for (int k = 0, i = near; ok && k < lead; ++k, i = !near)
    if (n[i] > 1) {
      ok = t->stride[i] >= wide;
      wide += (n[i] - 1) * t->stride[i];
    }
  if (!ok) Py_CLEAR(out);
  return out;
}
static PyObject* not_here(void) {
  PyErr_Clear();
  Py_RETURN_NONE;
}
static PyObject* outcome(int r, PyObject* y) {
  if (!r) return y;
  Py_DECREF(y);
  return PyLong_FromLong(r);
}

/* causal_conv1d(x, state, weight, bias, cu_seqlens, slots, resume, flags, out, step) */
static PyObject* causal_conv1d(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Call c;
  Tensor st, w, y;
  nova_rows xr, yr;
  const void* bias;
  nova_stream s;
  if (n != 10) return PyErr_Format(PyExc_TypeError, "ten arguments are needed");
  const int type = type_of(a[0]), step = a[9] == Py_True;
  const long flags = PyLong_AsLong(a[7]);
  if (type < 0 || PyErr_Occurred()) return not_here();
  PyObject* dtype = t_types[type];
  if (!sequences(&c, a[0], dtype, a[1], dtype, &st, a[4], a[5], a[6], step, &xr) || !tensor(a[2], dtype, c.dev, 1, &w) || w.dims != 2 ||
      w.size[0] != c.channels || w.size[1] > 64 || !vector(a[3], dtype, c.dev, c.channels, &bias) || !stream(&s))
    return not_here();
  if (a[1] != Py_None && (st.size[1] != w.size[1] - 1 || st.size[2] != c.channels)) return not_here();
  PyObject* out = output(a[8], a[0], c.n, c.lead, c.channels, dtype, c.dev, &y);
  if (!out) return not_here();
  yr = (nova_rows){y.p, step ? 0 : y.stride[c.lead - 1], c.lead == 2 || step ? y.stride[0] : 0};
  int r;
  Py_BEGIN_ALLOW_THREADS
  r = fn.causal(&c.q, type, &xr, w.p, bias, (int)c.channels, (int)w.size[1], a[1] == Py_None ? NULL : st.p, &yr, (int)flags, s);
  Py_END_ALLOW_THREADS
  return outcome(r, out);
}

/* selective_scan(u, state, delta, A, B, C, D, z, delta_bias, cu_seqlens, slots, resume, flags, out, step) */
static PyObject* selective_scan(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Call c;
  Tensor st, A, B, y;
  nova_scan q;
  const void* p;
  nova_stream s;
  if (n != 15) return PyErr_Format(PyExc_TypeError, "fifteen arguments are needed");
  const int type = type_of(a[0]), step = a[14] == Py_True;
  memset(&q, 0, sizeof q);
  q.flags = (int)PyLong_AsLong(a[12]);
  if (type < 0 || PyErr_Occurred()) return not_here();
  PyObject *dtype = t_types[type], *f32 = t_types[0];
  if (!sequences(&c, a[0], dtype, a[1], f32, &st, a[9], a[10], a[11], step, &q.u) || !tensor(a[3], f32, c.dev, 1, &A) || A.dims != 2 ||
      A.size[0] != c.channels || A.size[1] > 64 || !tensor(a[4], dtype, c.dev, 0, &B) || !stream(&s))
    return not_here();
  if (a[1] != Py_None && (st.size[1] != c.channels || st.size[2] != A.size[1])) return not_here();
  const int inner = B.dims - c.lead;
  if (inner != 1 && inner != 2) return not_here();
  const long long groups = inner == 2 ? B.size[c.lead] : 1, cols[2] = {inner == 2 ? groups : A.size[1], A.size[1]};
  if (groups > INT32_MAX || !token_rows(a[4], dtype, &c, inner, cols, &q.B, &q.B_group) ||
      !token_rows(a[5], dtype, &c, inner, cols, &q.C, &q.C_group) || !token_rows(a[2], dtype, &c, 1, &c.channels, &q.delta, NULL) ||
      (a[7] != Py_None && !token_rows(a[7], dtype, &c, 1, &c.channels, &q.z, NULL)))
    return not_here();
  if (!vector(a[6], f32, c.dev, c.channels, &p)) return not_here();
  q.D_dev = (const float*)p;
  if (!vector(a[8], f32, c.dev, c.channels, &p)) return not_here();
  q.delta_bias_dev = (const float*)p;
  q.A_dev = (const float*)A.p;
  q.state_dev = a[1] == Py_None ? NULL : (float*)st.p;
  q.channels = (int32_t)c.channels;
  q.states = (int32_t)A.size[1];
  q.groups = (int32_t)groups;
  PyObject* out = output(a[13], a[0], c.n, c.lead, c.channels, dtype, c.dev, &y);
  if (!out) return not_here();
  q.y = (nova_rows){y.p, step ? 0 : y.stride[c.lead - 1], c.lead == 2 || step ? y.stride[0] : 0};
  int r;
  Py_BEGIN_ALLOW_THREADS
  r = fn.scan(&c.q, type, &q, s);
  Py_END_ALLOW_THREADS
  return outcome(r, out);
}

/* linear_int4(x, codes, scales, zeros, bias, out) */
static PyObject* linear_int4(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  Tensor x, codes, scales, zeros, y;
  const void* bias;
  nova_stream s;
  if (n != 6) return PyErr_Format(PyExc_TypeError, "six arguments are needed");
  const int type = type_of(a[0]);
  PyObject* d = type < 1 ? NULL : PyObject_CallNoArgs(get_device);
  if (!d) return not_here();
  const long dev = PyLong_AsLong(d);
  Py_DECREF(d);
  PyObject* dtype = t_types[type];
  if (!tensor(a[0], dtype, dev, 0, &x) || x.dims != 2 || !tensor(a[1], t_uint8, dev, 1, &codes) || codes.dims != 2 ||
      !tensor(a[2], dtype, dev, 1, &scales) || scales.dims != 2)
    return not_here();
  const long long M = x.size[0], K = x.size[1], N = scales.size[0], groups = scales.size[1];
  if (M > INT32_MAX || K > INT32_MAX || N > INT32_MAX || groups < 1 || K % groups || codes.size[0] != N || codes.size[1] != K / 2 ||
      !vector(a[4], dtype, dev, N, &bias) || !stream(&s))
    return not_here();
  if (a[3] != Py_None && (!tensor(a[3], t_uint8, dev, 1, &zeros) || zeros.dims != 2 || zeros.size[0] != N || zeros.size[1] != groups))
    return not_here();
  PyObject* out = output(a[5], a[0], &M, 1, N, dtype, dev, &y);
  if (!out) return not_here();
  int r;
  Py_BEGIN_ALLOW_THREADS
  r = fn.linear(type, x.p, x.stride[0], (int)M, (int)K, codes.p, scales.p, a[3] == Py_None ? NULL : zeros.p, (int)(K / groups), bias,
                (int)N, y.p, y.stride[0], s);
  Py_END_ALLOW_THREADS
  return outcome(r, out);
}

/* bind_mixer(addresses of nova_causal_conv1d, nova_selective_scan, nova_linear_int4, torch's float32, float16, bfloat16, int32,
 * uint8, bool, empty_strided or None); after bind */
static PyObject* bind_mixer(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 10) return PyErr_Format(PyExc_TypeError, "ten arguments are needed");
  *(void**)&fn.causal = PyLong_AsVoidPtr(a[0]);
  *(void**)&fn.scan = PyLong_AsVoidPtr(a[1]);
  *(void**)&fn.linear = PyLong_AsVoidPtr(a[2]);
  if (PyErr_Occurred()) return NULL;
  PyObject** to[7] = {&t_types[0], &t_types[1], &t_types[2], &t_int32, &t_uint8, &t_bool, &empty_strided};
  for (int i = 0; i < 7; ++i) {
    Py_INCREF(a[3 + i]);
    Py_XSETREF(*to[i], a[3 + i]);
  }
  Py_RETURN_NONE;
}

/* bind(address of nova_conv2d_fwd, of nova_filter_transform, of nova_conv2d_fwd_int8, get_device, get_stream) */
static PyObject* bind(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 5) return PyErr_Format(PyExc_TypeError, "five arguments are needed");
  *(void**)&fn.conv2d = PyLong_AsVoidPtr(a[0]);
  *(void**)&fn.filter = PyLong_AsVoidPtr(a[1]);
  *(void**)&fn.int8 = PyLong_AsVoidPtr(a[2]);
  if (PyErr_Occurred()) return NULL;
  Py_INCREF(a[3]);
  Py_INCREF(a[4]);
  Py_XSETREF(get_device, a[3]);
  Py_XSETREF(get_stream, a[4]);
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, NULL},
    {"conv2d", (PyCFunction)(void (*)(void))conv2d, METH_FASTCALL, NULL},
    {"filter_transform", (PyCFunction)(void (*)(void))filter_transform, METH_FASTCALL, NULL},
    {"conv2d_int8", (PyCFunction)(void (*)(void))conv2d_int8, METH_FASTCALL, NULL},
    {"bind_mixer", (PyCFunction)(void (*)(void))bind_mixer, METH_FASTCALL, NULL},
    {"causal_conv1d", (PyCFunction)(void (*)(void))causal_conv1d, METH_FASTCALL, NULL},
    {"selective_scan", (PyCFunction)(void (*)(void))selective_scan, METH_FASTCALL, NULL},
    {"linear_int4", (PyCFunction)(void (*)(void))linear_int4, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__fastcall(void) {
  s_get_device = PyUnicode_InternFromString("get_device");
  s_stride = PyUnicode_InternFromString("stride");
  s_new_empty = PyUnicode_InternFromString("new_empty");
  s_is_cuda = PyUnicode_InternFromString("is_cuda");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_shape = PyUnicode_InternFromString("shape");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_numel = PyUnicode_InternFromString("numel");
  return PyModule_Create(&module);
}
