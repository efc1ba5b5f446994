// layer_norm_forward, layer_norm_backward, rotary_forward, rotary_backward and a step of
// AdamW of the binding: argument checks and marshalling of torch tensors, as attn_call.cpp does
// for the attention operators, but from torch's C++ objects: these kernels take a few us, and by
// attribute a tensor costs 0.35 us to look at and 1.1 to 1.6 to make (32 tokens turned 5.6 -> 3.5 to 4.3
// us a call, layer norm of 8 x 1024 7.9 -> 5.7, a step of 231 x 765 15.7 -> 10.0 to 10.9).
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <cmath>
#include <cstring>

#include "../../../include/adamw.h"
#include "../../../include/norm.h"
#include "../../../include/rotary.h"
#include "call.h"

namespace {

// Set by setup().
decltype(&layer_norm_workspace) norm_workspace_fn;
decltype(&layer_norm_forward) norm_forward_fn;
decltype(&layer_norm_backward) norm_backward_fn;
decltype(&layer_norm_last_error) norm_error_fn;
decltype(&rotary_forward) rotary_forward_fn;
decltype(&rotary_backward) rotary_backward_fn;
decltype(&rotary_last_error) rotary_error_fn;
decltype(&adamw_step) adamw_step_fn;
decltype(&adamw_last_error) adamw_error_fn;

bool wants(const char* name, Py_ssize_t n, Py_ssize_t takes) {
  if (n == takes && norm_forward_fn) return true;
  PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, after setup", name, takes);
  return false;
}

bool load(const char* name, PyObject* obj, Tensor* o, int most) {
  if (!THPVariable_Check(obj)) {
    PyErr_Format(PyExc_TypeError, "%s is not a tensor", name);
    return false;
  }
  try {
    const at::Tensor& t = THPVariable_Unpack(obj);
    const auto size = t.sizes(), stride = t.strides();
    if ((int)size.size() > most)
      return refuse("%s has more than %s dimensions", name, most == 4 ? "four" : "eight");
    o->nd = (int)size.size();
    for (int i = 0; i < o->nd; ++i) o->size[i] = size[i], o->stride[i] = stride[i];
    const at::ScalarType type = t.scalar_type();
    o->dtype = type == at::kBFloat16 ? bf16 : type == at::kFloat ? f32 : type == at::kInt ? i32
               : type == at::kByte   ? u8
                                     : nullptr;
    o->dev = t.is_cuda() ? (int)t.get_device() : -1;
    o->p = t.mutable_data_ptr();
    return true;
  } catch (const std::exception& e) {  // (no strides, no memory)
    return refuse("%s: %.200s", name, e.what());
  }
}
// An uninitialised tensor, and what there is to know of it.
PyObject* fresh(const int64_t* size, int nd, PyObject* dtype, int dev, Tensor* made) {
  HANDLE_TH_ERRORS
  const auto type = dtype == bf16 ? at::kBFloat16 : dtype == f32 ? at::kFloat : at::kByte;
  at::Tensor t = at::empty(at::IntArrayRef(size, nd), at::TensorOptions().dtype(type).device(at::kCUDA, dev));
  made->nd = nd;
  for (int i = 0; i < nd; ++i) made->size[i] = size[i], made->stride[i] = t.stride(i);
  made->dtype = dtype;
  made->dev = dev;
  made->p = t.mutable_data_ptr();
  return THPVariable_Wrap(std::move(t));
  END_HANDLE_TH_ERRORS
}
PyObject* new_bytes(size_t n, int dev, void** p) {
  const int64_t size = (int64_t)n;
  Tensor made;
  PyObject* t = fresh(&size, 1, u8, dev, &made);
  *p = made.p;
  return t;
}

// ---------------------------------------------------------------------------
// Layer norm
// ---------------------------------------------------------------------------
// Rows of a tensor: all dimensions but the last one, as [batch, seq].  Up to three dimensions as
// they are, more as one where they follow each other in memory.
struct Rows {
  Tensor like;  // sizes and type
  int64_t batch = 1, seq = 1, width = 0;
};
bool rows_of(const char* name, PyObject* x, Rows* r) {
  if (!load(name, x, &r->like, MAX_DIMS)) return false;
  const Tensor& t = r->like;
  if (t.dtype != bf16 && t.dtype != f32) return refuse("%s must be bfloat16 or float32", name);
  if (t.nd < 1 || t.dev < 0) return refuse("%s must be [..., width] on a GPU", name);
  r->width = t.size[t.nd - 1];
  if (t.nd == 3) r->batch = t.size[0], r->seq = t.size[1];
  else
    for (int i = 0; i < t.nd - 1; ++i) r->seq *= t.size[i];
  if (r->batch > INT_MAX || r->seq > INT_MAX || r->width > INT_MAX) return refuse("sizes beyond 31 bits");
  return true;
}
// A tensor of the same sizes and type: its pointer, and its strides of batch and position.
bool like_rows(const char* name, const Tensor& t, const Rows& r, void** p, int64_t* st) {
  if (!same(t, r.like.nd, r.like.size, r.like.dtype, r.like.dev))
    return refuse("%s must be %s, on cuda:%d, with the sizes of the other tensors of the call", name,
                  name_of(r.like.dtype), r.like.dev);
  const int nd = t.nd;
  if (r.width > 1 && t.stride[nd - 1] != 1) return refuse("the values of a row of %s must lie side by side", name);
  st[0] = st[1] = 0;
  if (nd == 3) st[0] = t.stride[0], st[1] = t.stride[1];
  else {
    int64_t step = 0;  // (of the dimensions after i that hold more than one row)
    for (int i = nd - 2; i >= 0; --i) {
      if (t.size[i] == 1) continue;
      if (step == 0) st[1] = t.stride[i];
      else if (t.stride[i] != step && r.seq > 0)
        return refuse("the rows of %s, of more than three dimensions, must be evenly spaced", name);
      step = t.stride[i] * t.size[i];
      if (t.stride[i] == 0 && r.seq > 0 && nd > 2) {
        // (broadcast: the dimensions before it would have to be so too)
        for (int j = 0; j < i; ++j)
          if (t.size[j] > 1 && t.stride[j] != 0)
            return refuse("the rows of %s, of more than three dimensions, must be evenly spaced", name);
        break;
      }
    }
  }
  *p = t.p;
  return true;
}
bool like_rows(const char* name, PyObject* x, const Rows& r, void** p, int64_t* st) {
  Tensor t;
  return load(name, x, &t, MAX_DIMS) && like_rows(name, t, r, p, st);
}
// The one given, or, where that is None, a new one.
bool rows_output(const char* name, PyObject* given, const Rows& r, Ref* out, void** p, int64_t* st) {
  if (given != Py_None) {
    Py_INCREF(given);
    out->set(given);
    return like_rows(name, given, r, p, st);
  }
  Tensor t;
  out->set(fresh(r.like.size, r.like.nd, r.like.dtype, r.like.dev, &t));
  return out->p && like_rows(name, t, r, p, st);
}
// fp32 [width], or None.
bool weight(const char* name, PyObject* x, const Rows& r, void** p) {
  *p = nullptr;
  return x == Py_None || plain(name, x, 1, r.width, 1, 1, f32, r.like.dev, p);
}
// fp32, contiguous, of the rows' sizes.
bool stat(const char* name, PyObject* x, const Rows& r, void** p) {
  Tensor t;
  if (!load(name, x, &t, MAX_DIMS)) return false;
  bool ok = same(t, r.like.nd - 1, r.like.size, f32, r.like.dev);
  int64_t step = 1;
  for (int i = t.nd - 1; ok && i >= 0; --i) {
    if (r.batch * r.seq > 0 && t.size[i] > 1) ok = t.stride[i] == step;
    step *= t.size[i];
  }
  if (!ok) return refuse("%s must be contiguous float32 of the rows' sizes on cuda:%d", name, r.like.dev);
  *p = t.p;
  return true;
}
bool stat_output(const char* name, PyObject* given, const Rows& r, Ref* out, void** p) {
  if (given != Py_None) {
    Py_INCREF(given);
    out->set(given);
    return stat(name, given, r, p);
  }
  Tensor t;
  out->set(fresh(r.like.size, r.like.nd - 1, f32, r.like.dev, &t));
  *p = t.p;
  return out->p;
}
bool norm_done(stage_status st) { return st == STAGE_OK || raise((int)st, norm_error_fn()); }

layer_norm_shape norm_shape(const Rows& r, float eps) {
  layer_norm_shape s = {};
  s.dtype = r.like.dtype == bf16 ? STAGE_BF16 : STAGE_F32;
  s.batch = (int)r.batch;
  s.seq = (int)r.seq;
  s.width = (int)r.width;
  s.eps = eps;
  return s;
}

// norm_forward(x, gamma, beta, residual, eps, out, total, mean, rstd): (out, total, mean, rstd), or
// the tensors' device where that is not the current one (nothing is launched).
PyObject* norm_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!wants("norm_forward", n, 9)) return nullptr;
  Rows r;
  if (!rows_of("x", a[0], &r)) return nullptr;
  const double eps = PyFloat_AsDouble(a[4]);
  if (eps == -1.0 && PyErr_Occurred()) return nullptr;
  layer_norm_shape s = norm_shape(r, (float)eps);
  void *x, *res = nullptr, *gamma, *beta, *out, *total = nullptr, *mean, *rstd;
  if (!like_rows("x", r.like, r, &x, s.x) || !weight("gamma", a[1], r, &gamma) ||
      !weight("beta", a[2], r, &beta))
    return nullptr;
  const bool add = a[3] != Py_None;
  if (add && !like_rows("residual", a[3], r, &res, s.residual)) return nullptr;
  if (!add && a[6] != Py_None) return refuse("total without a residual"), nullptr;
  const int here = on_device(r.like.dev);
  if (here <= 0) return here < 0 ? nullptr : PyLong_FromLong(r.like.dev);
  Ref o, tot, m, rs;
  if (!rows_output("out", a[5], r, &o, &out, s.out)) return nullptr;
  if (!add) {
    Py_INCREF(a[0]);
    tot.set(a[0]);
  } else if (!rows_output("total", a[6], r, &tot, &total, s.total)) {
    return nullptr;
  }
  if (!stat_output("mean", a[7], r, &m, &mean) || !stat_output("rstd", a[8], r, &rs, &rstd)) return nullptr;
  Room room;
  if (!take_room(r.like.dev, 0, &room)) return nullptr;
  stage_status st;
  Py_BEGIN_ALLOW_THREADS
  st = norm_forward_fn(&s, x, res, (const float*)gamma, (const float*)beta, total, out, (float*)mean,
                       (float*)rstd, room.stream);
  Py_END_ALLOW_THREADS
  if (!norm_done(st)) return nullptr;
  return PyTuple_Pack(4, o.p, tot.p, m.p, rs.p);
}

// norm_backward(dy, total, gamma, mean, rstd, dtotal, dx, dgamma, dbeta): (dx, dgamma, dbeta), or
// the device as above.  dx, dgamma or dbeta False: it is not made, None in its place.
PyObject* norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!wants("norm_backward", n, 9)) return nullptr;
  Rows r;
  if (!rows_of("dy", a[0], &r)) return nullptr;
  layer_norm_shape s = norm_shape(r, 0.0f);
  void *dy, *total, *gamma, *mean, *rstd, *dtotal = nullptr, *dx = nullptr, *dgamma = nullptr,
                                          *dbeta = nullptr;
  if (!like_rows("dy", r.like, r, &dy, s.dy) || !like_rows("total", a[1], r, &total, s.total) ||
      !weight("gamma", a[2], r, &gamma) || !stat("mean", a[3], r, &mean) ||
      !stat("rstd", a[4], r, &rstd) ||
      (a[5] != Py_None && !like_rows("dtotal", a[5], r, &dtotal, s.dtotal)))
    return nullptr;
  const int here = on_device(r.like.dev);
  if (here <= 0) return here < 0 ? nullptr : PyLong_FromLong(r.like.dev);
  Ref x, g, b;
  if (a[6] == Py_False) {
    Py_INCREF(Py_None);
    x.set(Py_None);
  } else if (!rows_output("dx", a[6], r, &x, &dx, s.dx)) {
    return nullptr;
  }
  Ref* const to[2] = {&g, &b};
  void** const p[2] = {&dgamma, &dbeta};
  for (int i = 0; i < 2; ++i) {
    const bool none = a[7 + i] == Py_False;
    if (none || a[7 + i] != Py_None) {
      PyObject* given = none ? Py_None : a[7 + i];
      Py_INCREF(given);
      to[i]->set(given);
      if (!weight(i ? "dbeta" : "dgamma", given, r, p[i])) return nullptr;
    } else {
      Tensor made;
      to[i]->set(fresh(&r.width, 1, f32, r.like.dev, &made));
      if (!to[i]->p) return nullptr;
      *p[i] = made.p;
    }
  }
  size_t bytes = 0;
  if ((dgamma || dbeta) && !norm_done(norm_workspace_fn(&s, &bytes))) return nullptr;
  Room room;
  if (!take_room(r.like.dev, bytes, &room)) return nullptr;
  stage_status st;
  Py_BEGIN_ALLOW_THREADS
  st = norm_backward_fn(&s, dy, total, (const float*)gamma, (const float*)mean, (const float*)rstd,
                        dtotal, dx, (float*)dgamma, (float*)dbeta, room.p, room.bytes, room.stream);
  Py_END_ALLOW_THREADS
  if (!norm_done(st)) return nullptr;
  return PyTuple_Pack(3, x.p, g.p, b.p);
}

// ---------------------------------------------------------------------------
// Rotary positions
// ---------------------------------------------------------------------------
bool heads(const char* name, const Tensor* like, Tensor* t, int64_t* st) {
  if (t->nd != 4 || t->size[3] != 64 || t->dev < 0 || (t->dtype != bf16 && t->dtype != f32))
    return refuse("%s must be bfloat16 or float32 [batch, length, heads, 64] on a GPU", name);
  for (int i = 0; i < 3; ++i)
    if (t->size[i] > INT_MAX) return refuse("lengths beyond 31 bits");
  if (like && (t->dtype != like->dtype || t->dev != like->dev || t->size[0] != like->size[0] ||
               t->size[1] != like->size[1]))
    return refuse("%s must have the type, device, batch and length of q", name);
  if (t->stride[3] != 1) return refuse("the 64 values of a head of %s must lie side by side", name);
  for (int i = 0; i < 3; ++i) st[i] = t->stride[i];
  return true;
}
bool heads(const char* name, PyObject* x, const Tensor* like, Tensor* t, int64_t* st) {
  return load(name, x, t) && heads(name, like, t, st);
}
// The one given, or, where that is None, a new one of the sizes of `of`.
bool heads_output(const char* name, PyObject* given, const Tensor& of, const Tensor* like, Ref* out, Tensor* t,
                  int64_t* st) {
  if (given != Py_None) {
    Py_INCREF(given);
    out->set(given);
    return heads(name, given, like, t, st);
  }
  out->set(fresh(of.size, 4, of.dtype, of.dev, t));
  return out->p && heads(name, like, t, st);
}

// rotary(backward, freqs, q, k, pos, q_out, k_out): (q_out, k_out), or the device as above.
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!wants("rotary", n, 7)) return nullptr;
  const int backward = PyObject_IsTrue(a[0]);
  if (backward < 0) return nullptr;
  Ref addr(PyObject_GetAttr(a[1], n_addr));
  if (!addr.p) return nullptr;
  const rotary_freqs* f = (const rotary_freqs*)PyLong_AsVoidPtr(addr.p);
  if (!f) return PyErr_Occurred() ? nullptr : (refuse("rotary holds no frequencies"), nullptr);
  rotary_shape s = {};
  Tensor q, k, qo, ko;
  const bool both = a[3] != Py_None;
  if (!heads("q", a[2], nullptr, &q, s.q) || (both && !heads("k", a[3], &q, &k, s.k))) return nullptr;
  if (!both && a[6] != Py_None) return refuse("k_out without k"), nullptr;
  s.dtype = q.dtype == bf16 ? STAGE_BF16 : STAGE_F32;
  s.batch = (int)q.size[0];
  s.seq = (int)q.size[1];
  s.heads = (int)q.size[2];
  s.kv_heads = both ? (int)k.size[2] : 0;
  if (both && s.kv_heads == 0) return refuse("k has no heads"), nullptr;
  void* pos = nullptr;
  if (a[4] != Py_None) {
    Tensor p;
    if (!load("pos", a[4], &p)) return nullptr;
    s.pos_each = p.nd == 2;
    if (p.nd < 1 || p.nd > 2 || p.dtype != i32 || p.dev != q.dev || p.size[0] != q.size[0] ||
        (p.nd == 2 && p.size[1] != q.size[1]))
      return refuse("pos must be int32 [%d] or [%d, %d] on cuda:%d", s.batch, s.batch, s.seq, q.dev), nullptr;
    s.pos[0] = p.stride[0];
    s.pos[1] = p.nd == 2 ? p.stride[1] : 0;
    pos = p.p;
  }
  const int here = on_device(q.dev);
  if (here <= 0) return here < 0 ? nullptr : PyLong_FromLong(q.dev);
  Ref q_out, k_out;
  if (!heads_output("q_out", a[5], q, &q, &q_out, &qo, s.q_out)) return nullptr;
  if (!both) {
    Py_INCREF(Py_None);
    k_out.set(Py_None);
  } else if (!heads_output("k_out", a[6], k, &q, &k_out, &ko, s.k_out)) {
    return nullptr;
  }
  if (qo.size[2] != q.size[2] || (both && ko.size[2] != k.size[2]))
    return refuse("q_out and k_out must have the heads of q and k"), nullptr;
  Room room;
  if (!take_room(q.dev, 0, &room)) return nullptr;
  stage_status st;
  Py_BEGIN_ALLOW_THREADS
  st = (backward ? rotary_backward_fn : rotary_forward_fn)(&s, f, q.p, both ? k.p : nullptr,
                                                           (const int32_t*)pos, qo.p,
                                                           both ? ko.p : nullptr, room.stream);
  Py_END_ALLOW_THREADS
  if (st != STAGE_OK) return raise((int)st, rotary_error_fn()), nullptr;
  return PyTuple_Pack(2, q_out.p, k_out.p);
}

// ---------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------
// Where a tensor is: the memory of its storage and its offset there.
struct Place {
  uint64_t memory, offset;
};
Place place_of(const at::Tensor& t) {
  const c10::TensorImpl* const of = t.unsafeGetTensorImpl();
  const c10::StorageImpl* const memory = of->unsafe_storage().unsafeGetStorageImpl();
  return {memory ? (uint64_t)(uintptr_t)memory->data_ptr().get() : 0, (uint64_t)of->storage_offset()};
}

// hold(tensors, a tuple): (aliases of them, as a list, which keep their memory; their places, as bytes).
PyObject* hold(PyObject*, PyObject* tensors) {
  HANDLE_TH_ERRORS
  if (!PyTuple_Check(tensors)) return PyErr_SetString(PyExc_TypeError, "not a tuple"), nullptr;
  const Py_ssize_t n = PyTuple_GET_SIZE(tensors);
  Ref held(PyList_New(n)), places(PyBytes_FromStringAndSize(nullptr, n * sizeof(Place)));
  if (!held.p || !places.p) return nullptr;
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* const x = PyTuple_GET_ITEM(tensors, i);
    if (!THPVariable_Check(x)) return PyErr_SetString(PyExc_TypeError, "not a tensor"), nullptr;
    const at::Tensor& t = THPVariable_Unpack(x);
    const Place p = place_of(t);
    memcpy(PyBytes_AS_STRING(places.p) + sizeof(p) * i, &p, sizeof(p));
    PyObject* const alias = THPVariable_Wrap(t.variable_data());
    if (!alias) return nullptr;
    PyList_SET_ITEM(held.p, i, alias);
  }
  return PyTuple_Pack(2, held.p, places.p);
  END_HANDLE_TH_ERRORS
}

// The first of the tensors `given` that is no longer at its place (-1: none, -2: an error): .data of a
// tensor can be set, its storage can be given up or made anew.  Straight from the objects, 3 ns a
// tensor: 24 weights with their gradients and states 0.3 us, 640 of them 8 us.
Py_ssize_t moved(PyObject* given, PyObject* places) {
  if (!PyTuple_Check(given) || !PyBytes_Check(places) ||
      PyBytes_GET_SIZE(places) != (Py_ssize_t)sizeof(Place) * PyTuple_GET_SIZE(given)) {
    PyErr_SetString(PyExc_TypeError, "the tensors and their places are not as many");
    return -2;
  }
  for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(given); ++i) {
    PyObject* const t = PyTuple_GET_ITEM(given, i);
    Place was;
    memcpy(&was, PyBytes_AS_STRING(places) + sizeof(was) * i, sizeof(was));
    try {
      if (!THPVariable_Check(t)) {
        PyErr_SetString(PyExc_TypeError, "not a tensor");
        return -2;
      }
      const Place now = place_of(THPVariable_Unpack(t));
      if (now.memory != was.memory || now.offset != was.offset) return i;
    } catch (const std::exception&) {  // (memory that is not to be had)
      return PyErr_Occurred() ? -2 : i;
    }
  }
  return -1;
}

// adamw(handle, device, lr, beta1, beta2, eps, max_norm, norm, given, places): None, or the device as above,
// or (i,), with nothing launched, where tensor i of `given` has moved.  lr: a number, or fp32 of one
// element on the device; max_norm None: no clipping (norm is then not written).
PyObject* adamw_call(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!wants("adamw", n, 10)) return nullptr;
  adamw_t* h = (adamw_t*)PyLong_AsVoidPtr(a[0]);
  if (!h) return PyErr_Occurred() ? nullptr : (refuse("the optimizer is closed"), nullptr);
  const Py_ssize_t i = moved(a[8], a[9]);
  if (i != -1) return i < 0 ? nullptr : Py_BuildValue("(n)", i);
  const int dev = (int)PyLong_AsLong(a[1]);
  if (dev == -1 && PyErr_Occurred()) return nullptr;
  adamw_args g = {};
  if (PyFloat_Check(a[2]) || PyLong_Check(a[2])) {
    g.lr = (float)PyFloat_AsDouble(a[2]);
  } else {
    Tensor t;
    if (!load("lr", a[2], &t)) return nullptr;
    bool one = t.dtype == f32 && t.dev == dev;
    for (int i = 0; i < t.nd; ++i) one = one && t.size[i] == 1;
    if (!one) return refuse("lr must be a number or one float32 on cuda:%d", dev), nullptr;
    g.lr_ptr = (const float*)t.p;
  }
  double v[3];
  for (int i = 0; i < 3; ++i) v[i] = PyFloat_AsDouble(a[3 + i]);
  g.beta1 = v[0];
  g.beta2 = v[1];
  g.eps = (float)v[2];
  if (a[6] != Py_None) {
    const double most = PyFloat_AsDouble(a[6]);
    if (PyErr_Occurred()) return nullptr;
    g.max_norm = (float)most;
    if (!(g.max_norm > 0.0f)) return refuse("max_norm must be positive"), nullptr;
    void* p = nullptr;
    if (!plain("norm", a[7], 1, 1, 1, 1, f32, dev, &p)) return nullptr;
    g.norm = (float*)p;
  }
  if (PyErr_Occurred()) return nullptr;
  const int here = on_device(dev);
  if (here <= 0) return here < 0 ? nullptr : PyLong_FromLong(dev);
  Room room;
  if (!take_room(dev, 0, &room)) return nullptr;
  stage_status st;
  Py_BEGIN_ALLOW_THREADS
  st = adamw_step_fn(h, &g, room.stream);
  Py_END_ALLOW_THREADS
  if (st != STAGE_OK) return raise((int)st, adamw_error_fn()), nullptr;
  Py_RETURN_NONE;
}

// setup(addresses of the nine functions above, in their order; then as set_common())
PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 17) {
    PyErr_SetString(PyExc_TypeError, "setup takes 17 arguments");
    return nullptr;
  }
  void* f[9];
  if (!addresses(a, 9, f)) return nullptr;
  set_common(a + 9);
  norm_workspace_fn = (decltype(norm_workspace_fn))f[0];
  norm_forward_fn = (decltype(norm_forward_fn))f[1];
  norm_backward_fn = (decltype(norm_backward_fn))f[2];
  norm_error_fn = (decltype(norm_error_fn))f[3];
  rotary_forward_fn = (decltype(rotary_forward_fn))f[4];
  rotary_backward_fn = (decltype(rotary_backward_fn))f[5];
  rotary_error_fn = (decltype(rotary_error_fn))f[6];
  adamw_step_fn = (decltype(adamw_step_fn))f[7];
  adamw_error_fn = (decltype(adamw_error_fn))f[8];
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"setup", (PyCFunction)(void*)setup, METH_FASTCALL, nullptr},
                         {"norm_forward", (PyCFunction)(void*)norm_forward, METH_FASTCALL, nullptr},
                         {"norm_backward", (PyCFunction)(void*)norm_backward, METH_FASTCALL, nullptr},
                         {"rotary", (PyCFunction)(void*)rotary, METH_FASTCALL, nullptr},
                         {"hold", hold, METH_O, nullptr},
                         {"adamw", (PyCFunction)(void*)adamw_call, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops_call", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops_call(void) {
  return intern_names() ? PyModule_Create(&module) : nullptr;
}
