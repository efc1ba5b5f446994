// What the modules of operators' calls share: references, errors, and checks of what a call
// needs to know of a tensor.  Each module has its own copy.
#pragma once
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <climits>
#include <cstdarg>
#include <cstdio>

#include "../../../include/stage.h"

namespace {

// Set by set_common(): what is taken from torch and the binding.
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

// What a call needs to know of a tensor.
constexpr int MAX_DIMS = 8;
struct Tensor {
  int nd = 0, dev = -1;
  int64_t size[MAX_DIMS], stride[MAX_DIMS];
  PyObject* dtype = nullptr;  // (borrowed: compared only)
  void* p = nullptr;
};

// By each module in its own way: what there is to know of an object that has to be a tensor of at
// most so many dimensions; an uninitialised tensor of n bytes.
bool load(const char* name, PyObject* t, Tensor* o, int most = 4);
PyObject* new_bytes(size_t n, int dev, void** p);

const char* name_of(PyObject* dtype) {
  return dtype == bf16 ? "bfloat16" : dtype == f32 ? "float32" : dtype == u8 ? "uint8" : "int32";
}

bool same(const Tensor& t, int nd, const int64_t* size, PyObject* dtype, int dev) {
  if (t.nd != nd || t.dtype != dtype || t.dev != dev) return false;
  for (int i = 0; i < nd; ++i)
    if (t.size[i] != size[i]) return false;
  return true;
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
bool take_room(int device, size_t bytes, Room* r) {
  Ref dev(PyLong_FromLong(device));
  if (!dev.p) return false;
  r->bytes = bytes;
  if (bytes) {
    r->ws.set(new_bytes(bytes, device, &r->p));
    if (!r->ws.p) return false;
  }
  Ref st(PyObject_CallOneArg(current_stream, dev.p));
  if (!st.p) return false;
  r->stream = PyLong_AsVoidPtr(st.p);
  return !PyErr_Occurred();
}

// The objects a[0 .. 7]: StageError; torch.bfloat16, float32, uint8, int32; current_device(),
// current_stream(device), new_workspace(bytes, device).
void set_common(PyObject* const* a) {
  PyObject** const to[8] = {&stage_error, &bf16, &f32, &u8, &i32, &current_device, &current_stream,
                            &new_workspace};
  for (int i = 0; i < 8; ++i) {
    Py_INCREF(a[i]);
    Py_XDECREF(*to[i]);
    *to[i] = a[i];
  }
}

// n addresses (of the library's functions).
bool addresses(PyObject* const* a, int n, void** f) {
  for (int i = 0; i < n; ++i) {
    f[i] = PyLong_AsVoidPtr(a[i]);
    if (!f[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a null address");
      return false;
    }
  }
  return true;
}

bool intern_names() {
  struct {
    PyObject** to;
    const char* name;
  } const names[] = {{&n_shape, "shape"},         {&n_stride, "stride"},
                     {&n_dtype, "dtype"},         {&n_get_device, "get_device"},
                     {&n_data_ptr, "data_ptr"},   {&n_new_empty, "new_empty"},
                     {&n_addr, "addr"}};
  for (const auto& e : names)
    if (!(*e.to = PyUnicode_InternFromString(e.name))) return false;
  return (kw_dtype = PyTuple_Pack(1, n_dtype)) != nullptr;
}

}  // namespace
