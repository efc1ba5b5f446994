// layer_norm_forward, layer_norm_backward, rotary_forward, rotary_backward and a step of
// AdamW of the binding: argument checks and marshalling of torch tensors, as attn_call.cpp does
// for the attention operators.
#include <cmath>

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
bool like_rows(const char* name, PyObject* x, const Rows& r, void** p, int64_t* st, Tensor* out = nullptr) {
  Tensor t;
  if (!load(name, x, &t, MAX_DIMS)) return false;
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
  if (out) *out = t;
  return true;
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
PyObject* new_stat(PyObject* like, const Rows& r) {
  Ref shape(PyTuple_New(r.like.nd - 1));
  if (!shape.p) return nullptr;
  for (int i = 0; i < r.like.nd - 1; ++i) {
    PyObject* n = PyLong_FromLongLong(r.like.size[i]);
    if (!n) return nullptr;
    PyTuple_SET_ITEM(shape.p, i, n);
  }
  PyObject* args[3] = {like, shape.p, f32};
  return PyObject_VectorcallMethod(n_new_empty, args, 2, kw_dtype);
}
PyObject* stat_output(PyObject* given, PyObject* like, const Rows& r) {
  if (given == Py_None) return new_stat(like, r);
  Py_INCREF(given);
  return given;
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
  if (!like_rows("x", a[0], r, &x, s.x) || !weight("gamma", a[1], r, &gamma) ||
      !weight("beta", a[2], r, &beta))
    return nullptr;
  const bool add = a[3] != Py_None;
  if (add && !like_rows("residual", a[3], r, &res, s.residual)) return nullptr;
  if (!add && a[6] != Py_None) return refuse("total without a residual"), nullptr;
  const int here = on_device(r.like.dev);
  if (here <= 0) return here < 0 ? nullptr : PyLong_FromLong(r.like.dev);
  Ref o(output(a[5], a[0])), tot(!o.p ? nullptr : add ? output(a[6], a[0]) : (Py_INCREF(a[0]), a[0]));
  if (!tot.p) return nullptr;
  Ref m(stat_output(a[7], a[0], r)), rs(m.p ? stat_output(a[8], a[0], r) : nullptr);
  if (!rs.p) return nullptr;
  if (!like_rows("out", o.p, r, &out, s.out) ||
      (add && !like_rows("total", tot.p, r, &total, s.total)) || !stat("mean", m.p, r, &mean) ||
      !stat("rstd", rs.p, r, &rstd))
    return nullptr;
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
  if (!like_rows("dy", a[0], r, &dy, s.dy) || !like_rows("total", a[1], r, &total, s.total) ||
      !weight("gamma", a[2], r, &gamma) || !stat("mean", a[3], r, &mean) ||
      !stat("rstd", a[4], r, &rstd) ||
      (a[5] != Py_None && !like_rows("dtotal", a[5], r, &dtotal, s.dtotal)))
    return nullptr;
  const int here = on_device(r.like.dev);
  if (here <= 0) return here < 0 ? nullptr : PyLong_FromLong(r.like.dev);
  Ref x, g, b;
  const bool makes[3] = {a[6] != Py_False, a[7] != Py_False, a[8] != Py_False};
  Ref* const to[3] = {&x, &g, &b};
  for (int i = 0; i < 3; ++i) {
    if (!makes[i]) {
      Py_INCREF(Py_None);
      to[i]->set(Py_None);
    } else if (i == 0 || a[6 + i] != Py_None) {
      to[i]->set(output(a[6 + i], a[0]));
    } else {
      Ref shape(Py_BuildValue("(L)", (long long)r.width));
      if (!shape.p) return nullptr;
      PyObject* args[3] = {a[0], shape.p, f32};
      to[i]->set(PyObject_VectorcallMethod(n_new_empty, args, 2, kw_dtype));
    }
    if (!to[i]->p) return nullptr;
  }
  if ((makes[0] && !like_rows("dx", x.p, r, &dx, s.dx)) || !weight("dgamma", g.p, r, &dgamma) ||
      !weight("dbeta", b.p, r, &dbeta))
    return nullptr;
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
bool heads(const char* name, PyObject* x, const Tensor* like, Tensor* t, int64_t* st) {
  if (!load(name, x, t)) return false;
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
  Ref q_out(output(a[5], a[2])), k_out;
  if (!q_out.p) return nullptr;
  if (both) {
    k_out.set(output(a[6], a[3]));
  } else {
    Py_INCREF(Py_None);
    k_out.set(Py_None);
  }
  if (!k_out.p || !heads("q_out", q_out.p, &q, &qo, s.q_out) ||
      (both && !heads("k_out", k_out.p, &q, &ko, s.k_out)))
    return nullptr;
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
// adamw(handle, device, lr, beta1, beta2, eps, max_norm, norm): None, or the device as above.  lr: a
// number, or fp32 of one element on the device; max_norm None: no clipping (norm is then not
// written).
PyObject* adamw_call(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!wants("adamw", n, 8)) return nullptr;
  adamw_t* h = (adamw_t*)PyLong_AsVoidPtr(a[0]);
  if (!h) return PyErr_Occurred() ? nullptr : (refuse("the optimizer is closed"), nullptr);
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
                         {"adamw", (PyCFunction)(void*)adamw_call, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops_call", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops_call(void) {
  return intern_names() ? PyModule_Create(&module) : nullptr;
}
