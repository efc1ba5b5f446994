// attn_forward and attn_backward of the binding: argument checks and marshalling of
// torch tensors, by attribute, for calls whose kernels take less time than the
// interpreter would (one token: 9.2 us a call with these checks in Python, 5.9 here, of
// which the launch takes about 3.5).
// The library's functions come as addresses, so this module links to neither it nor torch.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <climits>
#include <cstdarg>
#include <cstdio>

#include "../../../include/attn.h"

namespace {

typedef decltype(&attn_workspace) WorkspaceFn;
typedef decltype(&attn_forward) ForwardFn;
typedef decltype(&attn_backward) BackwardFn;
typedef decltype(&attn_last_error) ErrorFn;

WorkspaceFn workspace_fn;
ForwardFn forward_fn;
BackwardFn backward_fn;
ErrorFn error_fn;

// Set by setup(): what is taken from torch and the binding.
PyObject *stage_error, *bf16, *f32, *u8, *i32, *current_device, *current_stream, *new_workspace;
// Names of attributes
PyObject *n_shape, *n_stride, *n_dtype, *n_get_device, *n_data_ptr, *n_new_empty, *n_addr;
PyObject* kw_dtype;

// Owns a reference.
struct Ref {
  PyObject* p;
  explicit Ref(PyObject* p_ = nullptr) : p(p_) {}
  ~Ref() { Py_XDECREF(p); }
  Ref(const Ref&) = delete;
  Ref& operator=(const Ref&) = delete;
  void set(PyObject* q) {
    Py_XDECREF(p);
    p = q;
  }
  PyObject* release() {
    PyObject* q = p;
    p = nullptr;
    return q;
  }
};

bool raise(int status, const char* msg) {
  Ref e(PyObject_CallFunction(stage_error, "is", status, msg));
  if (e.p) PyErr_SetObject(stage_error, e.p);
  return false;
}
bool refuse(const char* fmt, ...) {
  char msg[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof(msg), fmt, ap);
  va_end(ap);
  return raise(STAGE_EINVAL, msg);
}
// The library's status as an exception.
bool done(stage_status st) { return st == STAGE_OK || raise((int)st, error_fn()); }

// What a call needs to know of a tensor.
struct Tensor {
  int nd = 0, dev = -1;
  int64_t size[4], stride[4];
  PyObject* dtype = nullptr;  // (borrowed: compared only)
  void* p = nullptr;
};

bool ints(PyObject* t, int n, int64_t* out) {
  for (int i = 0; i < n; ++i) {
    out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
    if (out[i] == -1 && PyErr_Occurred()) return false;
  }
  return true;
}

bool load(const char* name, PyObject* t, Tensor* o) {
  Ref shape(PyObject_GetAttr(t, n_shape));
  if (!shape.p) return false;
  Ref stride(PyObject_CallMethodNoArgs(t, n_stride));
  if (!stride.p) return false;
  if (!PyTuple_Check(shape.p) || !PyTuple_Check(stride.p) ||
      PyTuple_GET_SIZE(shape.p) != PyTuple_GET_SIZE(stride.p))
    return refuse("%s is not a tensor", name);
  if (PyTuple_GET_SIZE(shape.p) > 4) return refuse("%s has more than four dimensions", name);
  o->nd = (int)PyTuple_GET_SIZE(shape.p);
  if (!ints(shape.p, o->nd, o->size) || !ints(stride.p, o->nd, o->stride)) return false;
  Ref dtype(PyObject_GetAttr(t, n_dtype));
  if (!dtype.p) return false;
  o->dtype = dtype.p;
  Ref dev(PyObject_CallMethodNoArgs(t, n_get_device));
  if (!dev.p) return false;
  o->dev = (int)PyLong_AsLong(dev.p);
  if (o->dev == -1 && PyErr_Occurred()) return false;
  Ref p(PyObject_CallMethodNoArgs(t, n_data_ptr));
  if (!p.p) return false;
  o->p = PyLong_AsVoidPtr(p.p);
  return o->p || !PyErr_Occurred();
}

const char* name_of(PyObject* dtype) {
  return dtype == bf16 ? "bfloat16" : dtype == f32 ? "float32" : dtype == u8 ? "uint8" : "int32";
}

bool same(const Tensor& t, int nd, const int64_t* size, PyObject* dtype, int dev) {
  if (t.nd != nd || t.dtype != dtype || t.dev != dev) return false;
  for (int i = 0; i < nd; ++i)
    if (t.size[i] != size[i]) return false;
  return true;
}

// Whether a tensor is an operand [batch, length, heads, 64] of this shape and type; its
// strides into st.
bool fits(const char* name, const Tensor& t, const int64_t* size, PyObject* dtype, int dev, int64_t* st) {
  if (!same(t, 4, size, dtype, dev))
    return refuse("%s must be %s [%lld, %lld, %lld, %lld] on cuda:%d", name, name_of(dtype),
                  (long long)size[0], (long long)size[1], (long long)size[2], (long long)size[3], dev);
  if (t.stride[3] != 1) return refuse("the 64 values of a head of %s must lie side by side", name);
  for (int i = 0; i < 3; ++i) st[i] = t.stride[i];
  return true;
}
bool operand(const char* name, PyObject* obj, const int64_t* size, PyObject* dtype, int dev, Tensor* t,
             int64_t* st) {
  return load(name, obj, t) && fits(name, *t, size, dtype, dev, st);
}

// A contiguous tensor of nd dimensions; None leaves *p alone where it may.
bool plain(const char* name, PyObject* obj, int nd, int64_t a, int64_t b, int64_t c, PyObject* dtype,
           int dev, void** p) {
  const int64_t size[3] = {a, b, c};
  Tensor t;
  if (!load(name, obj, &t)) return false;
  bool ok = same(t, nd, size, dtype, dev);
  int64_t step = 1;
  const bool empty = a == 0 || (nd > 1 && b == 0) || (nd > 2 && c == 0);
  for (int i = nd - 1; ok && i >= 0; --i) {
    if (!empty && size[i] > 1) ok = t.stride[i] == step;
    step *= size[i];
  }
  if (!ok)
    return refuse("%s must be contiguous %s, %d dimensions of %lld, %lld, %lld, on cuda:%d", name,
                  name_of(dtype), nd, (long long)a, (long long)(nd > 1 ? b : 1),
                  (long long)(nd > 2 ? c : 1), dev);
  *p = t.p;
  return true;
}

// What both calls take.
struct Inputs {
  Tensor q, k, v;
  int64_t q_size[4], kv_size[4];
  int dev = -1;
  PyObject* dtype = nullptr;
  const attn_relpos* rp = nullptr;
  void *table = nullptr, *mask = nullptr, *pos = nullptr;
  int64_t buckets = 0;
  attn_shape s = {};
};

bool inputs(PyObject* q, PyObject* k, PyObject* v, PyObject* key_mask, PyObject* scale,
            PyObject* causal, PyObject* q_pos, PyObject* relpos, PyObject* table, Inputs* in) {
  if (!load("q", q, &in->q)) return false;
  const Tensor& t = in->q;
  in->dtype = t.dtype;
  in->dev = t.dev;
  if (t.dtype != bf16 && t.dtype != f32) return refuse("q must be bfloat16 or float32");
  if (!load("k", k, &in->k)) return false;
  if (t.nd != 4 || t.size[3] != 64 || in->k.nd != 4 || t.dev < 0)
    return refuse("q, k, v must be [batch, length, heads, 64] on a GPU");
  attn_shape& s = in->s;
  const int64_t kv[4] = {t.size[0], in->k.size[1], in->k.size[2], 64};
  for (int i = 0; i < 4; ++i) {
    in->q_size[i] = t.size[i];
    in->kv_size[i] = kv[i];
    if (t.size[i] > INT_MAX || kv[i] > INT_MAX) return refuse("lengths beyond 31 bits");
  }
  if (!fits("q", t, in->q_size, t.dtype, t.dev, s.q) || !fits("k", in->k, kv, t.dtype, t.dev, s.k) ||
      !operand("v", v, kv, t.dtype, t.dev, &in->v, s.v))
    return false;
  s.dtype = t.dtype == bf16 ? STAGE_BF16 : STAGE_F32;
  s.batch = (int)t.size[0];
  s.seq_q = (int)t.size[1];
  s.heads = (int)t.size[2];
  s.seq_k = (int)in->kv_size[1];
  s.kv_heads = (int)in->kv_size[2];
  double f = 0.125;
  if (scale != Py_None) {
    f = PyFloat_AsDouble(scale);
    if (f == -1.0 && PyErr_Occurred()) return false;
    if (!(f > 0.0 && f < 3e38)) return refuse("scale must be finite and positive");
  }
  s.scale = (float)f;
  s.causal = PyObject_IsTrue(causal);
  if (s.causal < 0) return false;
  if ((relpos == Py_None) != (table == Py_None)) return refuse("relpos and table go together");
  if (relpos != Py_None) {
    Ref addr(PyObject_GetAttr(relpos, n_addr));
    if (!addr.p) return false;
    in->rp = (const attn_relpos*)PyLong_AsVoidPtr(addr.p);
    if (!in->rp) return PyErr_Occurred() ? false : refuse("relpos holds no buckets");
    in->buckets = in->rp->num_buckets;
    if (!plain("table", table, 2, in->buckets, t.size[2], 1, f32, t.dev, &in->table)) return false;
  }
  if (key_mask != Py_None &&
      !plain("key_mask", key_mask, 2, t.size[0], in->kv_size[1], 1, u8, t.dev, &in->mask))
    return false;
  return q_pos == Py_None || plain("q_pos", q_pos, 1, t.size[0], 1, 1, i32, t.dev, &in->pos);
}

// The current device as 1 where it is dev, 0 where not, -1 for an error.
int on_device(int dev) {
  Ref now(PyObject_CallNoArgs(current_device));
  if (!now.p) return -1;
  const long d = PyLong_AsLong(now.p);
  return d == -1 && PyErr_Occurred() ? -1 : d == dev;
}

// A call's stream and workspace.  The workspace comes from torch's allocator, which gives
// no memory of a stream (or of a captured graph) away while work on it may still use it.
struct Room {
  Ref ws;
  void* p = nullptr;
  size_t bytes = 0;
  void* stream = nullptr;
};
bool room(const Inputs& in, int backward, Room* r) {
  if (!done(workspace_fn(&in.s, in.rp, backward, &r->bytes))) return false;
  Ref dev(PyLong_FromLong(in.dev));
  if (!dev.p) return false;
  if (r->bytes) {
    Ref n(PyLong_FromSize_t(r->bytes));
    if (!n.p) return false;
    r->ws.set(PyObject_CallFunctionObjArgs(new_workspace, n.p, dev.p, nullptr));
    if (!r->ws.p) return false;
    Ref p(PyObject_CallMethodNoArgs(r->ws.p, n_data_ptr));
    if (!p.p) return false;
    r->p = PyLong_AsVoidPtr(p.p);
  }
  Ref st(PyObject_CallOneArg(current_stream, dev.p));
  if (!st.p) return false;
  r->stream = PyLong_AsVoidPtr(st.p);
  return !PyErr_Occurred();
}

// given, or an uninitialised tensor shaped like `like` if it is None.
PyObject* output(PyObject* given, PyObject* like) {
  if (given != Py_None) {
    Py_INCREF(given);
    return given;
  }
  Ref shape(PyObject_GetAttr(like, n_shape));
  return shape.p ? PyObject_CallMethodOneArg(like, n_new_empty, shape.p) : nullptr;
}

// forward(q, k, v, key_mask, scale, causal, q_pos, relpos, table, out, lse): (out, lse), or the
// operands' device where that is not the current one (nothing is launched).
PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 11 || !workspace_fn) {
    PyErr_SetString(PyExc_TypeError, "forward takes 11 arguments, after setup");
    return nullptr;
  }
  Inputs in;
  if (!inputs(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], &in)) return nullptr;
  const int here = on_device(in.dev);
  if (here <= 0) return here < 0 ? nullptr : PyLong_FromLong(in.dev);
  Ref out(output(a[9], a[0])), lse;
  if (!out.p) return nullptr;
  if (a[10] != Py_None) {
    Py_INCREF(a[10]);
    lse.set(a[10]);
  } else {
    Ref shape(Py_BuildValue("(LLL)", (long long)in.q_size[0], (long long)in.q_size[2],
                            (long long)in.q_size[1]));
    if (!shape.p) return nullptr;
    PyObject* args[3] = {a[0], shape.p, f32};
    lse.set(PyObject_VectorcallMethod(n_new_empty, args, 2, kw_dtype));
    if (!lse.p) return nullptr;
  }
  Tensor o;
  void* l = nullptr;
  if (!operand("out", out.p, in.q_size, in.dtype, in.dev, &o, in.s.out) ||
      !plain("lse", lse.p, 3, in.q_size[0], in.q_size[2], in.q_size[1], f32, in.dev, &l))
    return nullptr;
  Room r;
  if (!room(in, 0, &r)) return nullptr;
  stage_status st;
  Py_BEGIN_ALLOW_THREADS
  st = forward_fn(&in.s, in.rp, (const float*)in.table, in.q.p, in.k.p, in.v.p,
                  (const uint8_t*)in.mask, (const int32_t*)in.pos, o.p, (float*)l, r.p, r.bytes,
                  r.stream);
  Py_END_ALLOW_THREADS
  if (!done(st)) return nullptr;
  return PyTuple_Pack(2, out.p, lse.p);
}

// backward(q, k, v, out, lse, dout, key_mask, scale, causal, q_pos, relpos, table, dq, dk, dv,
// dtable): (dq, dk, dv, dtable), or the device as above.  dtable False: none is made.
PyObject* backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 16 || !workspace_fn) {
    PyErr_SetString(PyExc_TypeError, "backward takes 16 arguments, after setup");
    return nullptr;
  }
  Inputs in;
  if (!inputs(a[0], a[1], a[2], a[6], a[7], a[8], a[9], a[10], a[11], &in)) return nullptr;
  const bool table_grad = a[11] != Py_None && a[15] != Py_False;
  if (a[11] == Py_None && a[15] != Py_None && a[15] != Py_False) {
    refuse("dtable without a table");
    return nullptr;
  }
  const int here = on_device(in.dev);
  if (here <= 0) return here < 0 ? nullptr : PyLong_FromLong(in.dev);
  Tensor out, dout, tq, tk, tv;
  void *lse = nullptr, *dt = nullptr;
  if (!operand("out", a[3], in.q_size, in.dtype, in.dev, &out, in.s.out) ||
      !plain("lse", a[4], 3, in.q_size[0], in.q_size[2], in.q_size[1], f32, in.dev, &lse) ||
      !operand("dout", a[5], in.q_size, in.dtype, in.dev, &dout, in.s.dout))
    return nullptr;
  Ref dq(output(a[12], a[0])), dk(dq.p ? output(a[13], a[1]) : nullptr),
      dv(dk.p ? output(a[14], a[2]) : nullptr);
  if (!dv.p) return nullptr;
  Ref dtable;
  if (table_grad) {
    dtable.set(output(a[15], a[11]));
    if (!dtable.p || !plain("dtable", dtable.p, 2, in.buckets, in.q_size[2], 1, f32, in.dev, &dt))
      return nullptr;
  } else {
    Py_INCREF(Py_None);
    dtable.set(Py_None);
  }
  if (!operand("dq", dq.p, in.q_size, in.dtype, in.dev, &tq, in.s.dq) ||
      !operand("dk", dk.p, in.kv_size, in.dtype, in.dev, &tk, in.s.dk) ||
      !operand("dv", dv.p, in.kv_size, in.dtype, in.dev, &tv, in.s.dv))
    return nullptr;
  Room r;
  if (!room(in, 1, &r)) return nullptr;
  stage_status st;
  Py_BEGIN_ALLOW_THREADS
  st = backward_fn(&in.s, in.rp, (const float*)in.table, in.q.p, in.k.p, in.v.p,
                   (const uint8_t*)in.mask, (const int32_t*)in.pos, out.p, (const float*)lse, dout.p,
                   tq.p, tk.p, tv.p, (float*)dt, r.p, r.bytes, r.stream);
  Py_END_ALLOW_THREADS
  if (!done(st)) return nullptr;
  return PyTuple_Pack(4, dq.p, dk.p, dv.p, dtable.p);
}

// setup(addresses of attn_workspace, attn_forward, attn_backward, attn_last_error; StageError;
// torch.bfloat16, float32, uint8, int32; current_device(), current_stream(device),
// new_workspace(bytes, device))
PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 12) {
    PyErr_SetString(PyExc_TypeError, "setup takes 12 arguments");
    return nullptr;
  }
  void* f[4];
  for (int i = 0; i < 4; ++i) {
    f[i] = PyLong_AsVoidPtr(a[i]);
    if (!f[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a null address");
      return nullptr;
    }
  }
  PyObject** const to[8] = {&stage_error, &bf16, &f32, &u8, &i32, &current_device, &current_stream,
                            &new_workspace};
  for (int i = 0; i < 8; ++i) {
    Py_INCREF(a[4 + i]);
    Py_XDECREF(*to[i]);
    *to[i] = a[4 + i];
  }
  forward_fn = (ForwardFn)f[1];
  backward_fn = (BackwardFn)f[2];
  error_fn = (ErrorFn)f[3];
  workspace_fn = (WorkspaceFn)f[0];
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"setup", (PyCFunction)(void*)setup, METH_FASTCALL, nullptr},
    {"forward", (PyCFunction)(void*)forward, METH_FASTCALL, nullptr},
    {"backward", (PyCFunction)(void*)backward, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_attn_call", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__attn_call(void) {
  struct {
    PyObject** to;
    const char* name;
  } const names[] = {{&n_shape, "shape"},         {&n_stride, "stride"},
                     {&n_dtype, "dtype"},         {&n_get_device, "get_device"},
                     {&n_data_ptr, "data_ptr"},   {&n_new_empty, "new_empty"},
                     {&n_addr, "addr"}};
  for (const auto& e : names)
    if (!(*e.to = PyUnicode_InternFromString(e.name))) return nullptr;
  if (!(kw_dtype = PyTuple_Pack(1, n_dtype))) return nullptr;
  return PyModule_Create(&module);
}
