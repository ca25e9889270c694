// Argument marshalling of the Python binding: fills mt_tensor descriptors from
// torch tensors and calls the C entry points. In native code because a call of
// the smallest layer is bound by it: with ctypes and descriptors built in Python
// a call took 11 us, more than its kernels. Nothing is kept between calls.
//
// Plain tensors are read through torch's DLPack exchange functions (0.08 us a
// tensor), anything else by its Python attributes (0.5 us); all of them where torch
// or its header has no such functions.
//
// init(handle, float32, bfloat16, int32, describe, current_stream, stream_of,
// tensor, parameter, device): the library's dlopen handle, torch's dtypes, binding.desc
// (called to raise its error for a tensor that is refused), how a stream is found
// (none given / given), torch's two plain tensor types and how the current device
// is found. Every other function returns the entry point's status.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>
#if __has_include(<ATen/dlpack.h>)
#include <ATen/dlpack.h>
#endif

#include "../../include/minitensor_hip.h"

namespace {

PyObject *g_f32, *g_bf16, *g_i32, *g_describe, *g_current, *g_stream_of, *g_tensor, *g_parameter, *g_device;
PyObject *s_is_cuda, *s_dtype, *s_shape, *s_stride, *s_data_ptr, *s_numel, *s_element_size, *s_get_device;

struct Lib {
  decltype(&mt_linear_fwd) linear_fwd;
  decltype(&mt_linear_act_fwd) linear_act_fwd;
  decltype(&mt_linear_bwd) linear_bwd;
  decltype(&mt_matmul) matmul;
  decltype(&mt_reduce_broadcast_grad) reduce_broadcast_grad;
  decltype(&mt_act_bwd) act_bwd;
  decltype(&mt_mse_loss) mse_loss;
  decltype(&mt_sgd_step) sgd_step;
  decltype(&mt_adam_step) adam_step;
  decltype(&mt_rmsprop_step) rmsprop_step;
  decltype(&mt_conv2d_fwd) conv2d_fwd;
  decltype(&mt_conv2d_bwd) conv2d_bwd;
  decltype(&mt_attention_fwd) attention_fwd;
  decltype(&mt_attention_bwd) attention_bwd;
  decltype(&mt_qk_norm_rope_fwd) qk_norm_rope_fwd;
  decltype(&mt_qk_norm_rope_bwd) qk_norm_rope_bwd;
  decltype(&mt_dropout_fwd) dropout_fwd;
  decltype(&mt_dropout_bwd) dropout_bwd;
  decltype(&mt_embedding_fwd) embedding_fwd;
  decltype(&mt_embedding_bwd) embedding_bwd;
  decltype(&mt_layer_norm_fwd) layer_norm_fwd;
  decltype(&mt_layer_norm_bwd) layer_norm_bwd;
  decltype(&mt_cross_entropy) cross_entropy;
  decltype(&mt_clip_grad_norm) clip_grad_norm;
} L;

bool as_i64(PyObject* o, int64_t* v) {
  if (PyLong_Check(o)) {
    *v = PyLong_AsLongLong(o);
  } else {
    PyObject* i = PyNumber_Long(o);
    if (!i) return false;
    *v = PyLong_AsLongLong(i);
    Py_DECREF(i);
  }
  return *v != -1 || !PyErr_Occurred();
}

bool as_address(PyObject* o, void** p) {  // consumes o
  if (!o) return false;
  const unsigned long long v = PyLong_AsUnsignedLongLong(o);
  Py_DECREF(o);
  *p = (void*)(uintptr_t)v;
  return v != (unsigned long long)-1 || !PyErr_Occurred();
}

bool ints(PyObject* tuple, int64_t* out, Py_ssize_t* n) {  // consumes tuple
  if (!tuple) return false;
  bool ok = PyTuple_Check(tuple);
  if (!ok) PyErr_SetString(PyExc_TypeError, "expected a tuple of sizes");
  *n = ok ? PyTuple_GET_SIZE(tuple) : 0;
  for (Py_ssize_t i = 0; ok && i < *n && i < MT_MAX_DIMS; ++i) ok = as_i64(PyTuple_GET_ITEM(tuple, i), &out[i]);
  Py_DECREF(tuple);
  return ok;
}

bool refuse(PyObject* t, bool index) {
  // raises what is wrong with it
  PyObject* r = PyObject_CallFunctionObjArgs(g_describe, t, index ? Py_True : Py_False, nullptr);
  if (r) {
    Py_DECREF(r);
    PyErr_SetString(PyExc_RuntimeError, "tensor cannot be described");
  }
  return false;
}

// The device of a tensor that is read by its attributes; -1: it names none.
bool device_of(PyObject* t, int* device) {
  *device = -1;
  PyObject* v = PyObject_CallMethodNoArgs(t, s_get_device);
  if (v) {
    *device = (int)PyLong_AsLong(v);
    Py_DECREF(v);
  } else if (PyErr_ExceptionMatches(PyExc_AttributeError)) {
    PyErr_Clear();
  }
  return !PyErr_Occurred();
}

// What a plain tensor holds.
struct Plain {
  void* data;
  const int64_t *shape, *stride;
  int ndim, device, dtype;  // the GPU, -1: the host's; MT_F32 .., -1: another type
  size_t bytes;             // of an element
};
#if defined(DLPACK_MAJOR_VERSION) && defined(DLPACK_MINOR_VERSION)
#if DLPACK_MAJOR_VERSION == 1 && DLPACK_MINOR_VERSION >= 3  // with the exchange functions
#define MT_EXCHANGE
#endif
#endif
#ifdef MT_EXCHANGE
const DLPackExchangeAPI* g_exchange;  // torch's; NULL: none
void find_exchange() {  // the functions live as long as torch
  PyObject* c = PyObject_GetAttrString(g_tensor, "__dlpack_c_exchange_api__");
  g_exchange = c && PyCapsule_IsValid(c, "dlpack_exchange_api")
                   ? (const DLPackExchangeAPI*)PyCapsule_GetPointer(c, "dlpack_exchange_api") : nullptr;
  if (g_exchange && (g_exchange->header.version.major != DLPACK_MAJOR_VERSION || !g_exchange->dltensor_from_py_object_no_sync))
    g_exchange = nullptr;
  Py_XDECREF(c);
  PyErr_Clear();
}
// Without taking hold of it; false: by its attributes.
bool view_of(PyObject* t, Plain* v) {
  if (!g_exchange || ((PyObject*)Py_TYPE(t) != g_tensor && (PyObject*)Py_TYPE(t) != g_parameter)) return false;
  DLTensor x;
  if (g_exchange->dltensor_from_py_object_no_sync(t, &x) != 0 || (!x.strides && x.ndim > 0)) {
    PyErr_Clear();
    return false;
  }
  const bool gpu = x.device.device_type == kDLROCM || x.device.device_type == kDLCUDA, one = x.dtype.lanes == 1;
  *v = Plain{(char*)x.data + x.byte_offset, x.shape, x.strides, x.ndim, gpu ? x.device.device_id : -1, -1,
             ((size_t)x.dtype.bits * x.dtype.lanes + 7) / 8};
  if (one && x.dtype.code == kDLInt && x.dtype.bits == 32) v->dtype = MT_I32;
  if (one && x.dtype.code == kDLFloat && x.dtype.bits == 32) v->dtype = MT_F32;
  if (one && x.dtype.code == kDLBfloat && x.dtype.bits == 16) v->dtype = MT_BF16;
  return true;
}
#else
void find_exchange() {}
bool view_of(PyObject*, Plain*) { return false; }
#endif

// index: a tensor of int32 lengths, positions, tokens or classes, else one of the two dtypes.
// device: receives a plain tensor's.
bool describe(PyObject* t, mt_tensor* d, bool index = false, int* device = nullptr) {
  Plain x;
  if (view_of(t, &x)) {
    if (x.device < 0 || x.dtype < 0 || (x.dtype == MT_I32) != index || x.ndim > MT_MAX_DIMS) return refuse(t, index);
    if (device) *device = x.device;
    d->dtype = x.dtype;
    d->data = x.data;
    d->ndim = x.ndim;
    for (int i = 0; i < x.ndim; ++i) {
      d->shape[i] = x.shape[i];
      d->stride[i] = x.stride[i];
    }
    return true;
  }
  PyObject* v = PyObject_GetAttr(t, s_is_cuda);
  if (!v) return false;
  Py_DECREF(v);
  if (v != Py_True) return refuse(t, index);
  if (!(v = PyObject_GetAttr(t, s_dtype))) return false;
  Py_DECREF(v);
  if (index && v == g_i32) d->dtype = MT_I32;
  else if (!index && v == g_f32) d->dtype = MT_F32;
  else if (!index && v == g_bf16) d->dtype = MT_BF16;
  else return refuse(t, index);
  Py_ssize_t n, m;
  if (!ints(PyObject_GetAttr(t, s_shape), d->shape, &n)) return false;
  if (n > MT_MAX_DIMS) return refuse(t, index);
  if (!ints(PyObject_CallMethodNoArgs(t, s_stride), d->stride, &m)) return false;
  if (m != n) return refuse(t, index);
  d->ndim = (int32_t)n;
  return as_address(PyObject_CallMethodNoArgs(t, s_data_ptr), &d->data);
}

// A call's arguments, converted in the order they are asked for; `ok` turns
// false with a Python error set, and later conversions do nothing.
struct Args {
  PyObject* const* a;
  bool ok = true;
  mt_tensor d[12];
  int used = 0;
  int device = -1;  // of the tensors so far
  bool mixed = false;
  PyObject* unseen[13];  // tensors (12) and a workspace whose device is asked for where it matters (one_device)
  int n_unseen = 0;
  Args(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : a(args) {
    if (n != want) {
      PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
      ok = false;
    }
  }
  const mt_tensor* tensor(int i, bool index = false) {
    if (!ok || a[i] == Py_None) return nullptr;
    mt_tensor* t = &d[used++];
    int dev = -1;
    ok = describe(a[i], t, index, &dev);
    if (dev < 0) unseen[n_unseen++] = a[i];
    met(dev);
    return t;
  }
  void met(int dev) {
    if (dev < 0) return;
    mixed = mixed || (device >= 0 && device != dev);
    device = dev;
  }
  // The tensors lie on one device, where none is given for the stream the current one.
  bool one_device(int stream) {
    for (int i = 0; ok && i < n_unseen; ++i) {
      int dev = -1;
      ok = device_of(unseen[i], &dev);
      met(dev);
    }
    if (!ok) return false;
    if (mixed) {
      PyErr_SetString(PyExc_ValueError, "the tensors lie on different devices");
      return ok = false;
    }
    if (device < 0 || a[stream] != Py_None) return true;
    PyObject* now = PyObject_CallNoArgs(g_device);
    const long n = now ? PyLong_AsLong(now) : -1;
    Py_XDECREF(now);
    if (PyErr_Occurred()) return ok = false;
    if (n != device) PyErr_Format(PyExc_ValueError, "the tensors lie on device %d, the current one is %ld", device, n);
    return ok = n == device;
  }
  uint64_t u64(int i) {
    if (!ok) return 0;
    const unsigned long long v = PyLong_AsUnsignedLongLong(a[i]);
    ok = v != (unsigned long long)-1 || !PyErr_Occurred();
    return v;
  }
  int64_t i64(int i) {
    int64_t v = 0;
    if (ok) ok = as_i64(a[i], &v);
    return v;
  }
  double f64(int i) {
    if (!ok) return 0.0;
    const double v = PyFloat_AsDouble(a[i]);
    ok = v != -1.0 || !PyErr_Occurred();
    return v;
  }
  float f32(int i) { return (float)f64(i); }
  struct Ws {
    void* p = nullptr;
    size_t n = 0;
  };
  Ws ws(int i) {
    Ws w;
    if (!ok || a[i] == Py_None) return w;
    Plain x;
    if (view_of(a[i], &x) && x.device >= 0) {
      met(x.device);
      w.p = x.data;
      w.n = x.bytes;
      for (int d = 0; d < x.ndim; ++d) w.n *= (size_t)x.shape[d];
      return w;
    }
    unseen[n_unseen++] = a[i];
    PyObject* c = PyObject_GetAttr(a[i], s_is_cuda);
    ok = c != nullptr;
    if (c) Py_DECREF(c);
    if (ok && c != Py_True) {
      PyErr_SetString(PyExc_AssertionError, "the workspace is a device tensor");
      ok = false;
    }
    void *count = nullptr, *size = nullptr;
    ok = ok && as_address(PyObject_CallMethodNoArgs(a[i], s_data_ptr), &w.p) &&
         as_address(PyObject_CallMethodNoArgs(a[i], s_numel), &count) &&
         as_address(PyObject_CallMethodNoArgs(a[i], s_element_size), &size);
    w.n = (size_t)(uintptr_t)count * (size_t)(uintptr_t)size;
    return w;
  }
  void* stream(int i) {
    void* s = nullptr;
    if (ok)
      ok = as_address(a[i] == Py_None ? PyObject_CallNoArgs(g_current) : PyObject_CallOneArg(g_stream_of, a[i]), &s);
    return s;
  }
};

template <typename F>
PyObject* call(bool ok, F f) {
  if (!ok) return nullptr;
  mt_status s;
  Py_BEGIN_ALLOW_THREADS
  s = f();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)s);
}

#define FN(name) PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n)

FN(linear_fwd) {  // x, w, b, y, stream
  Args g(a, n, 5);
  const mt_tensor *x = g.tensor(0), *w = g.tensor(1), *b = g.tensor(2), *y = g.tensor(3);
  void* st = g.stream(4);
  return call(g.ok, [&] { return L.linear_fwd(x, w, b, y, st); });
}
FN(linear_act_fwd) {  // x, w, b, act, z, y, stream
  Args g(a, n, 7);
  const mt_tensor *x = g.tensor(0), *w = g.tensor(1), *b = g.tensor(2);
  const int32_t act = (int32_t)g.i64(3);
  const mt_tensor *z = g.tensor(4), *y = g.tensor(5);
  void* st = g.stream(6);
  return call(g.ok, [&] { return L.linear_act_fwd(x, w, b, act, z, y, st); });
}
FN(linear_bwd) {  // x, w, dy, dx, dw, db, flags, ws, stream
  Args g(a, n, 9);
  const mt_tensor *x = g.tensor(0), *w = g.tensor(1), *dy = g.tensor(2), *dx = g.tensor(3), *dw = g.tensor(4),
                  *db = g.tensor(5);
  const uint32_t flags = (uint32_t)g.i64(6);
  const Args::Ws ws = g.ws(7);
  void* st = g.stream(8);
  return call(g.ok, [&] { return L.linear_bwd(x, w, dy, dx, dw, db, flags, ws.p, ws.n, st); });
}
FN(matmul) {  // a, b, c, flags, ws, stream
  Args g(a, n, 6);
  const mt_tensor *x = g.tensor(0), *y = g.tensor(1), *c = g.tensor(2);
  const uint32_t flags = (uint32_t)g.i64(3);
  const Args::Ws ws = g.ws(4);
  void* st = g.stream(5);
  return call(g.ok, [&] { return L.matmul(x, y, c, flags, ws.p, ws.n, st); });
}
FN(reduce_broadcast_grad) {  // grad_out, grad_in, flags, ws, stream
  Args g(a, n, 5);
  const mt_tensor *o = g.tensor(0), *i = g.tensor(1);
  const uint32_t flags = (uint32_t)g.i64(2);
  const Args::Ws ws = g.ws(3);
  void* st = g.stream(4);
  return call(g.ok, [&] { return L.reduce_broadcast_grad(o, i, flags, ws.p, ws.n, st); });
}
FN(act_bwd) {  // act, z, dy, dz, db, flags, ws, stream
  Args g(a, n, 8);
  const int32_t act = (int32_t)g.i64(0);
  const mt_tensor *z = g.tensor(1), *dy = g.tensor(2), *dz = g.tensor(3), *db = g.tensor(4);
  const uint32_t flags = (uint32_t)g.i64(5);
  const Args::Ws ws = g.ws(6);
  void* st = g.stream(7);
  return call(g.ok, [&] { return L.act_bwd(act, z, dy, dz, db, flags, ws.p, ws.n, st); });
}
FN(mse_loss) {  // pred, target, loss, dpred, ws, stream
  Args g(a, n, 6);
  const mt_tensor *p = g.tensor(0), *t = g.tensor(1), *l = g.tensor(2), *d = g.tensor(3);
  const Args::Ws ws = g.ws(4);
  void* st = g.stream(5);
  return call(g.ok, [&] { return L.mse_loss(p, t, l, d, ws.p, ws.n, st); });
}
FN(conv2d_fwd) {  // x, w, b, y, sh, sw, ph, pw, ws, stream
  Args g(a, n, 10);
  const mt_tensor *x = g.tensor(0), *w = g.tensor(1), *b = g.tensor(2), *y = g.tensor(3);
  int32_t v[4];
  for (int i = 0; i < 4; ++i) v[i] = (int32_t)g.i64(4 + i);
  const Args::Ws ws = g.ws(8);
  void* st = g.stream(9);
  return call(g.ok, [&] { return L.conv2d_fwd(x, w, b, y, v[0], v[1], v[2], v[3], ws.p, ws.n, st); });
}
FN(conv2d_bwd) {  // x, w, dy, dx, dw, db, sh, sw, ph, pw, flags, ws, stream
  Args g(a, n, 13);
  const mt_tensor *x = g.tensor(0), *w = g.tensor(1), *dy = g.tensor(2), *dx = g.tensor(3), *dw = g.tensor(4),
                  *db = g.tensor(5);
  int32_t v[4];
  for (int i = 0; i < 4; ++i) v[i] = (int32_t)g.i64(6 + i);
  const uint32_t flags = (uint32_t)g.i64(10);
  const Args::Ws ws = g.ws(11);
  void* st = g.stream(12);
  return call(g.ok, [&] { return L.conv2d_bwd(x, w, dy, dx, dw, db, v[0], v[1], v[2], v[3], flags, ws.p, ws.n, st); });
}

FN(attention_fwd) {  // q, k, v, kv_len, q_start, o, lse, scale, flags, ws, stream
  Args g(a, n, 11);
  const mt_tensor *q = g.tensor(0), *k = g.tensor(1), *v = g.tensor(2), *len = g.tensor(3, true),
                  *start = g.tensor(4, true), *o = g.tensor(5), *lse = g.tensor(6);
  const float scale = g.f32(7);
  const uint32_t flags = (uint32_t)g.i64(8);
  const Args::Ws ws = g.ws(9);
  void* st = g.stream(10);
  return call(g.ok, [&] { return L.attention_fwd(q, k, v, len, start, o, lse, scale, flags, ws.p, ws.n, st); });
}
FN(attention_bwd) {  // q, k, v, kv_len, q_start, o, lse, dout, dq, dk, dv, scale, flags, ws, stream
  Args g(a, n, 15);
  const mt_tensor *q = g.tensor(0), *k = g.tensor(1), *v = g.tensor(2), *len = g.tensor(3, true),
                  *start = g.tensor(4, true), *o = g.tensor(5), *lse = g.tensor(6), *dout = g.tensor(7),
                  *dq = g.tensor(8), *dk = g.tensor(9), *dv = g.tensor(10);
  const float scale = g.f32(11);
  const uint32_t flags = (uint32_t)g.i64(12);
  const Args::Ws ws = g.ws(13);
  void* st = g.stream(14);
  return call(g.ok, [&] {
    return L.attention_bwd(q, k, v, len, start, o, lse, dout, dq, dk, dv, scale, flags, ws.p, ws.n, st);
  });
}
FN(qk_norm_rope_fwd) {  // q, k, wq, wk, cos, sin, yq, yk, eps, flags, stream
  Args g(a, n, 11);
  const mt_tensor* t[8];
  for (int i = 0; i < 8; ++i) t[i] = g.tensor(i);
  const float eps = g.f32(8);
  const uint32_t flags = (uint32_t)g.i64(9);
  void* st = g.stream(10);
  return call(g.ok, [&] { return L.qk_norm_rope_fwd(t[0], t[1], t[2], t[3], t[4], t[5], t[6], t[7], eps, flags, st); });
}
FN(qk_norm_rope_bwd) {  // q, k, wq, wk, cos, sin, dyq, dyk, dq, dk, dwq, dwk, eps, flags, ws, stream
  Args g(a, n, 16);
  const mt_tensor* t[12];
  for (int i = 0; i < 12; ++i) t[i] = g.tensor(i);
  const float eps = g.f32(12);
  const uint32_t flags = (uint32_t)g.i64(13);
  const Args::Ws ws = g.ws(14);
  void* st = g.stream(15);
  return call(g.ok, [&] {
    return L.qk_norm_rope_bwd(t[0], t[1], t[2], t[3], t[4], t[5], t[6], t[7], t[8], t[9], t[10], t[11], eps, flags,
                              ws.p, ws.n, st);
  });
}
FN(dropout_fwd) {  // x, residual, p, seed, offset, y, stream
  Args g(a, n, 7);
  const mt_tensor *x = g.tensor(0), *r = g.tensor(1);
  const float p = g.f32(2);
  const uint64_t seed = g.u64(3), offset = g.u64(4);
  const mt_tensor* y = g.tensor(5);
  void* st = g.stream(6);
  return call(g.ok, [&] { return L.dropout_fwd(x, r, p, seed, offset, y, st); });
}
FN(dropout_bwd) {  // dy, p, seed, offset, dx, flags, stream
  Args g(a, n, 7);
  const mt_tensor* dy = g.tensor(0);
  const float p = g.f32(1);
  const uint64_t seed = g.u64(2), offset = g.u64(3);
  const mt_tensor* dx = g.tensor(4);
  const uint32_t flags = (uint32_t)g.i64(5);
  void* st = g.stream(6);
  return call(g.ok, [&] { return L.dropout_bwd(dy, p, seed, offset, dx, flags, st); });
}
FN(embedding_fwd) {  // ids, table, scale, y, stream
  Args g(a, n, 5);
  const mt_tensor *ids = g.tensor(0, true), *t = g.tensor(1);
  const float scale = g.f32(2);
  const mt_tensor* y = g.tensor(3);
  void* st = g.stream(4);
  return call(g.one_device(4), [&] { return L.embedding_fwd(ids, t, scale, y, st); });
}
FN(embedding_bwd) {  // ids, dy, scale, dtable, flags, ws, stream
  Args g(a, n, 7);
  const mt_tensor *ids = g.tensor(0, true), *dy = g.tensor(1);
  const float scale = g.f32(2);
  const mt_tensor* d = g.tensor(3);
  const uint32_t flags = (uint32_t)g.i64(4);
  const Args::Ws ws = g.ws(5);
  void* st = g.stream(6);
  return call(g.one_device(6), [&] { return L.embedding_bwd(ids, dy, scale, d, flags, ws.p, ws.n, st); });
}
FN(layer_norm_fwd) {  // x, w, b, eps, y, stream
  Args g(a, n, 6);
  const mt_tensor *x = g.tensor(0), *w = g.tensor(1), *b = g.tensor(2);
  const float eps = g.f32(3);
  const mt_tensor* y = g.tensor(4);
  void* st = g.stream(5);
  return call(g.one_device(5), [&] { return L.layer_norm_fwd(x, w, b, eps, y, st); });
}
FN(layer_norm_bwd) {  // x, w, dy, eps, dx, dw, db, flags, ws, stream
  Args g(a, n, 10);
  const mt_tensor *x = g.tensor(0), *w = g.tensor(1), *dy = g.tensor(2);
  const float eps = g.f32(3);
  const mt_tensor *dx = g.tensor(4), *dw = g.tensor(5), *db = g.tensor(6);
  const uint32_t flags = (uint32_t)g.i64(7);
  const Args::Ws ws = g.ws(8);
  void* st = g.stream(9);
  return call(g.one_device(9), [&] { return L.layer_norm_bwd(x, w, dy, eps, dx, dw, db, flags, ws.p, ws.n, st); });
}
FN(cross_entropy) {  // logits, targets, loss, losses, dlogits, ws, stream
  Args g(a, n, 7);
  const mt_tensor *z = g.tensor(0), *t = g.tensor(1, true), *l = g.tensor(2), *ls = g.tensor(3), *d = g.tensor(4);
  const Args::Ws ws = g.ws(5);
  void* st = g.stream(6);
  return call(g.one_device(6), [&] { return L.cross_entropy(z, t, l, ls, d, ws.p, ws.n, st); });
}

// Descriptors of up to four lists of n tensors each, one list after another.
// The lists' tensors are held until the call has returned: it runs without
// the interpreter's lock, while another thread may change a list, and an
// iterable may make its tensors as it is read. What has no length is refused.
struct Lists {
  PyObject* held[4] = {};
  mt_tensor* d = nullptr;
  Py_ssize_t n = 0;
  bool ok = true;
  Lists(PyObject* const* a, int lists, Args* args = nullptr) {
    for (int l = 0; ok && l < lists; ++l) ok = PyObject_Size(a[l]) >= 0 && (held[l] = PySequence_Tuple(a[l])) != nullptr;
    if (!ok) return;
    n = PyTuple_GET_SIZE(held[0]);
    for (int l = 1; l < lists; ++l) {
      if (PyTuple_GET_SIZE(held[l]) == n) continue;
      PyErr_SetString(PyExc_AssertionError, "the lists of tensors have different lengths");
      ok = false;
      return;
    }
    d = (mt_tensor*)PyMem_Malloc(sizeof(mt_tensor) * (size_t)(lists * (n > 0 ? n : 1)));
    if (!d) {
      PyErr_NoMemory();
      ok = false;
    }
    for (int l = 0; ok && l < lists; ++l)
      for (Py_ssize_t i = 0; ok && i < n; ++i) {
        int dev = -1;
        ok = describe(PyTuple_GET_ITEM(held[l], i), &d[l * n + i], false, &dev);
        if (!ok || !args) continue;
        if (dev < 0) ok = device_of(PyTuple_GET_ITEM(held[l], i), &dev);
        args->met(dev);
      }
  }
  ~Lists() {
    PyMem_Free(d);
    for (PyObject* h : held) Py_XDECREF(h);
  }
  const mt_tensor* operator[](int l) const { return d + l * n; }
};

FN(sgd_step) {  // params, grads, velocity, lr, momentum, weight_decay, stream
  Args g(a, n, 7);
  if (!g.ok) return nullptr;
  const Lists t(a, 3);
  if (!t.ok) return nullptr;
  const float lr = g.f32(3), mu = g.f32(4), wd = g.f32(5);
  void* st = g.stream(6);
  return call(g.ok, [&] { return L.sgd_step((int32_t)t.n, t[0], t[1], t[2], lr, mu, wd, st); });
}
FN(adam_step) {  // params, grads, exp_avg, exp_avg_sq, lr, beta1, beta2, eps, step, stream
  Args g(a, n, 10);
  if (!g.ok) return nullptr;
  const Lists t(a, 4);
  if (!t.ok) return nullptr;
  const float lr = g.f32(4), b1 = g.f32(5), b2 = g.f32(6), eps = g.f32(7);
  const int64_t step = g.i64(8);
  void* st = g.stream(9);
  return call(g.ok, [&] { return L.adam_step((int32_t)t.n, t[0], t[1], t[2], t[3], lr, b1, b2, eps, step, st); });
}
FN(rmsprop_step) {  // params, grads, sq_avg, lr, alpha, eps, stream
  Args g(a, n, 7);
  if (!g.ok) return nullptr;
  const Lists t(a, 3);
  if (!t.ok) return nullptr;
  const float lr = g.f32(3), alpha = g.f32(4), eps = g.f32(5);
  void* st = g.stream(6);
  return call(g.ok, [&] { return L.rmsprop_step((int32_t)t.n, t[0], t[1], t[2], lr, alpha, eps, st); });
}
FN(clip_grad_norm) {  // grads, out, max_norm, norm, ws, stream
  Args g(a, n, 6);
  if (!g.ok) return nullptr;
  const bool in_place = a[1] == Py_None;
  const Lists t(a, in_place ? 1 : 2, &g);
  if (!t.ok) return nullptr;
  const double most = g.f64(2);
  const mt_tensor* norm = g.tensor(3);
  const Args::Ws ws = g.ws(4);
  void* st = g.stream(5);
  return call(g.one_device(5), [&] {
    return L.clip_grad_norm((int32_t)t.n, t[0], most, in_place ? nullptr : t[1], norm, ws.p, ws.n, st);
  });
}

FN(init) {
  if (n != 10) {
    PyErr_SetString(PyExc_TypeError, "init(handle, float32, bfloat16, int32, describe, current_stream, stream_of, tensor, parameter, device)");
    return nullptr;
  }
  void* h = PyLong_AsVoidPtr(a[0]);
  if (!h) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null library handle");
    return nullptr;
  }
#define SYM(f)                                              \
  if (!(L.f = (decltype(L.f))dlsym(h, "mt_" #f))) {         \
    PyErr_SetString(PyExc_ImportError, "no symbol mt_" #f); \
    return nullptr;                                         \
  }
  SYM(linear_fwd) SYM(linear_act_fwd) SYM(linear_bwd) SYM(matmul) SYM(reduce_broadcast_grad) SYM(act_bwd)
  SYM(mse_loss) SYM(sgd_step) SYM(adam_step) SYM(rmsprop_step) SYM(conv2d_fwd) SYM(conv2d_bwd)
  SYM(attention_fwd) SYM(attention_bwd) SYM(qk_norm_rope_fwd) SYM(qk_norm_rope_bwd) SYM(dropout_fwd)
  SYM(dropout_bwd) SYM(embedding_fwd) SYM(embedding_bwd) SYM(layer_norm_fwd) SYM(layer_norm_bwd) SYM(cross_entropy)
  SYM(clip_grad_norm)
#undef SYM
  PyObject** to[] = {&g_f32, &g_bf16, &g_i32, &g_describe, &g_current, &g_stream_of, &g_tensor, &g_parameter, &g_device};
  for (int i = 0; i < 9; ++i) {
    Py_INCREF(a[i + 1]);
    Py_XSETREF(*to[i], a[i + 1]);
  }
  find_exchange();
  Py_RETURN_NONE;
}

#define METHOD(f) {#f, (PyCFunction)(void (*)())f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(init), METHOD(linear_fwd), METHOD(linear_act_fwd), METHOD(linear_bwd), METHOD(matmul),
                         METHOD(reduce_broadcast_grad), METHOD(act_bwd), METHOD(mse_loss), METHOD(sgd_step),
                         METHOD(adam_step), METHOD(rmsprop_step), METHOD(conv2d_fwd), METHOD(conv2d_bwd),
                         METHOD(attention_fwd), METHOD(attention_bwd), METHOD(qk_norm_rope_fwd),
                         METHOD(qk_norm_rope_bwd), METHOD(dropout_fwd), METHOD(dropout_bwd),
                         METHOD(embedding_fwd), METHOD(embedding_bwd), METHOD(layer_norm_fwd), METHOD(layer_norm_bwd),
                         METHOD(cross_entropy), METHOD(clip_grad_norm),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "argument marshalling of the binding", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
  struct {
    PyObject** to;
    const char* name;
  } names[] = {{&s_is_cuda, "is_cuda"}, {&s_dtype, "dtype"},       {&s_shape, "shape"},
               {&s_stride, "stride"},   {&s_data_ptr, "data_ptr"}, {&s_numel, "numel"},
               {&s_element_size, "element_size"}, {&s_get_device, "get_device"}};
  for (auto& e : names)
    if (!(*e.to = PyUnicode_InternFromString(e.name))) return nullptr;
  return PyModule_Create(&module);
}
