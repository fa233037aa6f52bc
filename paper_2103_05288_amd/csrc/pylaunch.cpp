// Python's way into disc_launch, disc_graph_launch and the operators of decoder.py and step.py: turns the argument lists of a call (dims,
// tensors, workspace) into the C arrays of the ABI.  Marshalling only, like the ctypes binding whose
// per-call part it is: with ctypes arrays a call spent 5 us here, more than a small kernel takes
// (37 x 768 fp32: 9.3 us a call, 4.4 us of them the kernel).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstddef>
#include <cstdint>

#include "disc.h"

namespace {

PyObject *s_data_ptr, *s_numel, *s_element_size, *s_dtype, *s_get_device, *s_shape, *s_stride, *s_is_contiguous;

// int(x) of any Python number, modulo 2^64
bool as_u64(PyObject* x, uint64_t* out) {
  if (PyLong_CheckExact(x)) {
    *out = PyLong_AsUnsignedLongLongMask(x);
    return !(*out == (uint64_t)-1 && PyErr_Occurred());
  }
  PyObject* n = PyNumber_Long(x);
  if (!n) return false;
  *out = PyLong_AsUnsignedLongLongMask(n);
  Py_DECREF(n);
  return !(*out == (uint64_t)-1 && PyErr_Occurred());
}

bool call_u64(PyObject* x, PyObject* method, uint64_t* out) {
  PyObject* r = PyObject_CallMethodNoArgs(x, method);
  if (!r) return false;
  const bool ok = as_u64(r, out);
  Py_DECREF(r);
  return ok;
}

// after a failed call_u64: the object has no such method (the error is cleared), or the method failed
bool lacks(PyObject* x, PyObject* method) {
  if (!PyErr_ExceptionMatches(PyExc_AttributeError)) return false;
  PyObject *type, *value, *trace;
  PyErr_Fetch(&type, &value, &trace);
  if (PyObject_HasAttr(x, method)) {
    PyErr_Restore(type, value, trace);
    return false;
  }
  Py_XDECREF(type);
  Py_XDECREF(value);
  Py_XDECREF(trace);
  return true;
}

// the device address of a tensor (anything with data_ptr()), or a raw address
bool as_address(PyObject* x, uint64_t* out) {
  if (PyLong_CheckExact(x)) return as_u64(x, out);
  if (call_u64(x, s_data_ptr, out)) return true;
  return lacks(x, s_data_ptr) && as_u64(x, out);
}

// A Python sequence as an array of 8-byte words; up to kInline of them need no allocation.
struct Words {
  static constexpr Py_ssize_t kInline = 24;
  uint64_t inl[kInline];
  uint64_t* p = inl;
  Py_ssize_t n = 0;
  ~Words() {
    if (p != inl) PyMem_Free(p);
  }
  bool fill(PyObject* seq, bool addresses) {
    PyObject* f = PySequence_Fast(seq, "expected a sequence");
    if (!f) return false;
    n = PySequence_Fast_GET_SIZE(f);
    if (n > kInline) p = (uint64_t*)PyMem_Malloc((size_t)n * sizeof(uint64_t));
    bool ok = p != nullptr;
    if (!ok) {
      p = inl;
      PyErr_NoMemory();
    }
    for (Py_ssize_t i = 0; ok && i < n; ++i) {
      // (the item is held: a data_ptr() written in Python could change the sequence)
      PyObject* x = PySequence_Fast_GET_ITEM(f, i);
      Py_INCREF(x);
      ok = addresses ? as_address(x, p + i) : as_u64(x, p + i);
      Py_DECREF(x);
      if (ok && PySequence_Fast_GET_SIZE(f) != n) {
        PyErr_SetString(PyExc_RuntimeError, "sequence changed size during the call");
        ok = false;
      }
    }
    Py_DECREF(f);
    return ok;
  }
};

typedef int (*launch_fn)(void*, int32_t, const int64_t*, int, const void* const*, int, void* const*, int, void*, size_t, void*);

// launch(function address, ctx address, id, dims, inputs, outputs, workspace or None, workspace
// bytes (0 or None: the size of the workspace tensor), stream) -> status.  The GIL is released during the call.
PyObject* launch(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 9) {
    PyErr_SetString(PyExc_TypeError, "launch takes 9 arguments");
    return nullptr;
  }
  uint64_t fn, ctx, id, ws = 0, bytes = 0, stream;
  bool no_bytes = a[7] == Py_None;
  Words dims, ins, outs;
  if (!as_u64(a[0], &fn) || !as_u64(a[1], &ctx) || !as_u64(a[2], &id) || !dims.fill(a[3], false) || !ins.fill(a[4], true) ||
      !outs.fill(a[5], true) || (!no_bytes && !as_u64(a[7], &bytes)) || !as_u64(a[8], &stream))
    return nullptr;
  if (a[6] != Py_None) {
    if (!as_address(a[6], &ws)) return nullptr;
    if (bytes == 0 && !PyLong_CheckExact(a[6])) {
      uint64_t n = 0, size = 0;
      if (call_u64(a[6], s_numel, &n)) {
        if (!call_u64(a[6], s_element_size, &size)) return nullptr;
        bytes = n * size;
        no_bytes = false;
      } else if (!lacks(a[6], s_numel)) {
        return nullptr;
      }
    }
  }
  if (no_bytes) {
    PyErr_SetString(PyExc_TypeError, "workspace_bytes=None needs a workspace tensor to take the size from");
    return nullptr;
  }
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<launch_fn>(fn)(reinterpret_cast<void*>(ctx), (int32_t)id, reinterpret_cast<const int64_t*>(dims.p), (int)dims.n,
                                       reinterpret_cast<const void* const*>(ins.p), (int)ins.n, reinterpret_cast<void* const*>(outs.p),
                                       (int)outs.n, reinterpret_cast<void*>(ws), (size_t)bytes, reinterpret_cast<void*>(stream));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// ---- the operators of decoder.py -------------------------------------------------------------------
// What decoder.py's handles check of their tensors and pass on, for calls that fit: the same in Python costs 5 us a
// call.  Whatever does not fit here returns None, and the handle goes through its own checks, which say why.

// get()'s result as a number, and whether that worked; no error is left behind
bool number(PyObject* r, int64_t* out) {
  if (!r) return false;
  *out = PyLong_AsLongLong(r);
  Py_DECREF(r);
  return !(*out == -1 && PyErr_Occurred());
}
bool on(PyObject* t, PyObject* dtype, int64_t device, uint64_t* address) {
  PyObject* x = PyObject_GetAttr(t, s_dtype);
  Py_XDECREF(x);
  if (x != dtype) return false;
  int64_t d;
  return number(PyObject_CallMethodNoArgs(t, s_get_device), &d) && d == device && call_u64(t, s_data_ptr, address);
}
// a tuple of n numbers
bool numbers(PyObject* r, Py_ssize_t n, int64_t* out) {
  bool ok = r && PyTuple_Check(r) && PyTuple_GET_SIZE(r) == n;
  for (Py_ssize_t i = 0; ok && i < n; ++i) {
    out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(r, i));
    ok = !(out[i] == -1 && PyErr_Occurred());
  }
  Py_XDECREF(r);
  return ok;
}
// [rows, heads, head_dim], the last axis dense
struct Rows {
  uint64_t address;
  int64_t shape[3], stride[3];
  bool take(PyObject* t, PyObject* dtype, int64_t device, int64_t head_dim) {
    return on(t, dtype, device, &address) && numbers(PyObject_GetAttr(t, s_shape), 3, shape) && shape[2] == head_dim &&
           numbers(PyObject_CallMethodNoArgs(t, s_stride), 3, stride) && stride[2] == 1;
  }
};
// dense, n axes
bool dense(PyObject* t, PyObject* dtype, int64_t device, Py_ssize_t n, int64_t* shape, uint64_t* address) {
  if (!on(t, dtype, device, address) || !numbers(PyObject_GetAttr(t, s_shape), n, shape)) return false;
  PyObject* r = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  Py_XDECREF(r);
  return r == Py_True;
}
// the pages of a cache: their shape, and two or four addresses
bool cache_pages(PyObject* seq, bool scaled, PyObject* stored, PyObject* f32, int64_t device, int64_t head_dim, int64_t* shape, uint64_t* address) {
  if ((!PyTuple_Check(seq) && !PyList_Check(seq)) || PySequence_Fast_GET_SIZE(seq) != (scaled ? 4 : 2)) return false;
  for (int i = 0; i < (scaled ? 4 : 2); ++i) {
    int64_t s[4];
    PyObject* t = PySequence_Fast_GET_ITEM(seq, i);
    Py_INCREF(t);
    const bool ok = dense(t, i < 2 ? stored : f32, device, i < 2 ? 4 : 3, i ? s : shape, address + i);
    Py_DECREF(t);
    if (!ok || PySequence_Fast_GET_SIZE(seq) != (scaled ? 4 : 2)) return false;
    for (int k = 0; i && k < (i < 2 ? 4 : 3); ++k)
      if (s[k] != shape[k]) return false;
  }
  return shape[3] == head_dim;
}
bool rows_of(PyObject* seq, Py_ssize_t n, Rows* r, PyObject* dtype, int64_t device, int64_t head_dim) {
  if ((!PyTuple_Check(seq) && !PyList_Check(seq)) || PySequence_Fast_GET_SIZE(seq) != n) return false;
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* t = PySequence_Fast_GET_ITEM(seq, i);
    Py_INCREF(t);
    const bool ok = r[i].take(t, dtype, device, head_dim);
    Py_DECREF(t);
    if (!ok || PySequence_Fast_GET_SIZE(seq) != n) return false;
  }
  return true;
}

// the first six arguments of each: function address, ctx address, id, dtype, device, head_dim
struct Call {
  uint64_t fn, ctx, id;
  int64_t device, head_dim;
  PyObject* dtype;
  bool take(PyObject* const* a) {
    uint64_t d, h;
    if (!as_u64(a[0], &fn) || !as_u64(a[1], &ctx) || !as_u64(a[2], &id) || !as_u64(a[4], &d) || !as_u64(a[5], &h)) return false;
    dtype = a[3];
    device = (int64_t)d;
    head_dim = (int64_t)h;
    return true;
  }
  PyObject* run(const int64_t* dims, int n_dims, const uint64_t* ins, int n_in, const uint64_t* outs, int n_out, uint64_t ws, uint64_t bytes,
                uint64_t stream) const {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = reinterpret_cast<launch_fn>(fn)(reinterpret_cast<void*>(ctx), (int32_t)id, dims, n_dims, reinterpret_cast<const void* const*>(ins), n_in,
                                         reinterpret_cast<void* const*>(const_cast<uint64_t*>(outs)), n_out, reinterpret_cast<void*>(ws), (size_t)bytes,
                                         reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  }
};
PyObject* does_not_fit() {
  PyErr_Clear();
  Py_RETURN_NONE;
}

// rotary(fn, ctx, id, dtype, device, head_dim, int32, int64, positions, inputs, outputs, backward, stream)
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  Call c;
  uint64_t stream;
  if (n_args != 13 || !c.take(a) || !as_u64(a[12], &stream)) return does_not_fit();
  const Py_ssize_t n = PyTuple_Check(a[9]) || PyList_Check(a[9]) ? PySequence_Fast_GET_SIZE(a[9]) : 0;
  Rows x[4], y[4];
  int64_t tokens, dims[3 + 5 * 4];
  uint64_t in[5], out[4];
  if (n < 1 || n > 4 || !rows_of(a[9], n, x, c.dtype, c.device, c.head_dim) || !rows_of(a[10], n, y, c.dtype, c.device, c.head_dim)) return does_not_fit();
  bool wide = false;
  if (!dense(a[8], a[6], c.device, 1, &tokens, in)) {
    PyErr_Clear();
    wide = true;
    if (!dense(a[8], a[7], c.device, 1, &tokens, in)) return does_not_fit();
  }
  const int backward = PyObject_IsTrue(a[11]);
  if (backward < 0) return does_not_fit();
  dims[0] = tokens;
  dims[1] = wide ? 8 : 4;
  dims[2] = backward;
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (x[i].shape[0] != tokens || y[i].shape[0] != tokens || x[i].shape[1] != y[i].shape[1]) return does_not_fit();
    int64_t* d = dims + 3 + 5 * i;
    d[0] = x[i].shape[1];
    d[1] = x[i].stride[0];
    d[2] = x[i].stride[1];
    d[3] = y[i].stride[0];
    d[4] = y[i].stride[1];
    in[1 + i] = x[i].address;
    out[i] = y[i].address;
  }
  return c.run(dims, 3 + 5 * (int)n, in, 1 + (int)n, out, (int)n, 0, 0, stream);
}

// cache_rows(fn, ctx, id, dtype, device, head_dim, scaled, stored type, int64, fp32, store, slots, rows, pages, stream)
PyObject* cache_rows(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  Call c;
  uint64_t stream;
  if (n_args != 15 || !c.take(a) || !as_u64(a[14], &stream)) return does_not_fit();
  const bool scaled = a[6] == Py_True, store = a[10] == Py_True;
  const int n = scaled ? 4 : 2;
  int64_t tokens, shape[4];
  uint64_t slots, pages[4];
  Rows r[2];
  if (!cache_pages(a[13], scaled, a[7], a[9], c.device, c.head_dim, shape, pages) || !rows_of(a[12], 2, r, c.dtype, c.device, c.head_dim) ||
      !dense(a[11], a[8], c.device, 1, &tokens, &slots) || r[0].shape[0] != tokens || r[1].shape[0] != tokens || r[0].shape[1] != shape[1] ||
      r[1].shape[1] != shape[1])
    return does_not_fit();
  const int64_t dims[8] = {tokens, shape[1], shape[0], shape[2], r[0].stride[0], r[0].stride[1], r[1].stride[0], r[1].stride[1]};
  const uint64_t rows[2] = {r[0].address, r[1].address};
  if (store) {
    const uint64_t in[3] = {slots, rows[0], rows[1]};
    return c.run(dims, 8, in, 3, pages, n, 0, 0, stream);
  }
  const uint64_t in[5] = {slots, pages[0], pages[1], scaled ? pages[2] : 0, scaled ? pages[3] : 0};
  return c.run(dims, 8, in, 1 + n, rows, 2, 0, 0, stream);
}

// cache_attend(fn, ctx, id, dtype, device, head_dim, scaled, stored type, int32, fp32, q, lengths, table, pages, out,
//              workspace, prefix table, prefix length, stream)
PyObject* cache_attend(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  Call c;
  uint64_t stream, prefix;
  if (n_args != 19 || !c.take(a) || !as_u64(a[18], &stream) || !PyLong_CheckExact(a[17]) || !as_u64(a[17], &prefix)) return does_not_fit();
  const bool scaled = a[6] == Py_True;
  const int n = scaled ? 4 : 2;
  int64_t batch, shape[4], table[2], prefix_width = 0;
  uint64_t in[8], pages[4], ws = 0, bytes = 0;
  Rows q, out;
  if (!cache_pages(a[13], scaled, a[7], a[9], c.device, c.head_dim, shape, pages) || !q.take(a[10], c.dtype, c.device, c.head_dim) ||
      !out.take(a[14], c.dtype, c.device, c.head_dim) || !dense(a[11], a[8], c.device, 1, &batch, in + 1) || !dense(a[12], a[8], c.device, 2, table, in + 2) ||
      q.shape[0] != batch || out.shape[0] != batch || table[0] != batch || q.shape[1] != out.shape[1])
    return does_not_fit();
  in[0] = q.address;
  for (int i = 0; i < n; ++i) in[3 + i] = pages[i];
  if (prefix && !dense(a[16], a[8], c.device, 1, &prefix_width, in + 3 + n)) return does_not_fit();
  if (a[15] != Py_None) {
    int64_t d;
    uint64_t count, size;
    PyObject* whole = PyObject_CallMethodNoArgs(a[15], s_is_contiguous);     // (elements may share memory otherwise)
    Py_XDECREF(whole);
    if (whole != Py_True || !number(PyObject_CallMethodNoArgs(a[15], s_get_device), &d) || d != c.device || !call_u64(a[15], s_data_ptr, &ws) ||
        !call_u64(a[15], s_numel, &count) || !call_u64(a[15], s_element_size, &size))
      return does_not_fit();
    bytes = count * size;
  }
  const int64_t dims[12] = {batch,           q.shape[1],  shape[1],    shape[0],    shape[2],      table[1],
                            (int64_t)prefix, prefix_width, q.stride[0], q.stride[1], out.stride[0], out.stride[1]};
  return c.run(dims, 12, in, 3 + n + (prefix ? 1 : 0), &out.address, 1, ws, bytes, stream);
}

// ---- the operators of step.py ----------------------------------------------------------------------

// [rows, width], the last axis dense
struct Matrix {
  uint64_t address;
  int64_t shape[2], stride[2];
  bool take(PyObject* t, PyObject* dtype, int64_t device) {
    return on(t, dtype, device, &address) && numbers(PyObject_GetAttr(t, s_shape), 2, shape) && numbers(PyObject_CallMethodNoArgs(t, s_stride), 2, stride) &&
           (stride[1] == 1 || shape[1] == 1);
  }
  bool take(PyObject* t, PyObject* dtype, int64_t device, int64_t rows, int64_t width) { return take(t, dtype, device) && shape[0] == rows && shape[1] == width; }
};
bool vector(PyObject* t, PyObject* dtype, int64_t device, int64_t n, uint64_t* address) {
  int64_t m;
  return dense(t, dtype, device, 1, &m, address) && m == n;
}
bool table(PyObject* t, PyObject* dtype, int64_t device, int64_t rows, int64_t width, uint64_t* address) {
  int64_t s[2];
  return dense(t, dtype, device, 2, s, address) && s[0] == rows && s[1] == width;
}
// a dense workspace, or None
bool scratch(PyObject* t, int64_t device, uint64_t* address, uint64_t* bytes) {
  *address = *bytes = 0;
  if (t == Py_None) return true;
  int64_t d;
  uint64_t count, size;
  PyObject* whole = PyObject_CallMethodNoArgs(t, s_is_contiguous);
  Py_XDECREF(whole);
  if (whole != Py_True || !number(PyObject_CallMethodNoArgs(t, s_get_device), &d) || d != device || !call_u64(t, s_data_ptr, address) || !call_u64(t, s_numel, &count) ||
      !call_u64(t, s_element_size, &size))
    return false;
  *bytes = count * size;
  return true;
}

// norm(fn, ctx, id, dtype, device, 0, stored type, fp32, x, weight, codes, scales, residual, total, stream)
PyObject* norm(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  Call c;
  uint64_t stream, in[3], out[3];
  Matrix x, codes, residual, total;
  if (n_args != 15 || !c.take(a) || !as_u64(a[14], &stream) || !x.take(a[8], c.dtype, c.device)) return does_not_fit();
  const int64_t rows = x.shape[0], width = x.shape[1];
  if (!vector(a[9], c.dtype, c.device, width, in + 1) || !codes.take(a[10], a[6], c.device, rows, width) || !vector(a[11], a[7], c.device, rows, out + 1) ||
      (a[12] == Py_None) != (a[13] == Py_None))
    return does_not_fit();
  const bool adds = a[12] != Py_None;
  if (adds && (!residual.take(a[12], c.dtype, c.device, rows, width) || !total.take(a[13], c.dtype, c.device, rows, width))) return does_not_fit();
  in[0] = x.address;
  in[2] = adds ? residual.address : 0;
  out[0] = codes.address;
  out[2] = adds ? total.address : 0;
  const int64_t dims[6] = {rows, width, x.stride[0], adds ? residual.stride[0] : 0, adds ? total.stride[0] : 0, codes.stride[0]};
  return c.run(dims, 6, in, adds ? 3 : 2, out, adds ? 3 : 2, 0, 0, stream);
}

// norm_backward(fn, ctx, id, dtype, device, 0, fp32, total, weight, dy, dx, dweight, dtotal, workspace, stream)
PyObject* norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  Call c;
  uint64_t stream, in[4], out[2], ws, bytes;
  Matrix total, dy, dx, dtotal;
  if (n_args != 15 || !c.take(a) || !as_u64(a[14], &stream) || !total.take(a[7], c.dtype, c.device)) return does_not_fit();
  const int64_t rows = total.shape[0], width = total.shape[1];
  const bool adds = a[12] != Py_None;
  if (!vector(a[8], c.dtype, c.device, width, in + 1) || !dy.take(a[9], c.dtype, c.device, rows, width) || !dx.take(a[10], c.dtype, c.device, rows, width) ||
      !vector(a[11], a[6], c.device, width, out + 1) || (adds && !dtotal.take(a[12], c.dtype, c.device, rows, width)) || !scratch(a[13], c.device, &ws, &bytes))
    return does_not_fit();
  in[0] = total.address;
  in[2] = dy.address;
  in[3] = adds ? dtotal.address : 0;
  out[0] = dx.address;
  const int64_t dims[6] = {rows, width, total.stride[0], dy.stride[0], adds ? dtotal.stride[0] : 0, dx.stride[0]};
  return c.run(dims, 6, in, adds ? 4 : 3, out, 2, ws, bytes, stream);
}

// linear4(fn, ctx, id, dtype, device, group, type of x, fp32, uint8, scaled, with zeros, x, weights, scales, out, row_scales, zeros, bias, stream)
PyObject* linear4(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  Call c;
  uint64_t stream, in[6];
  Matrix x, out;
  int64_t w[2];
  if (n_args != 19 || !c.take(a) || !as_u64(a[18], &stream) || !x.take(a[11], a[6], c.device) || !dense(a[12], a[8], c.device, 2, w, in + 1)) return does_not_fit();
  const int64_t rows = x.shape[0], k = x.shape[1], n = w[0], group = c.head_dim;
  const bool scaled = a[9] == Py_True, zeros = a[10] == Py_True;
  if (group < 1 || k % group || w[1] != k / 2 || !table(a[13], c.dtype, c.device, n, k / group, in + 2) || !out.take(a[14], c.dtype, c.device, rows, n) ||
      scaled != (a[15] != Py_None) || zeros != (a[16] != Py_None))
    return does_not_fit();
  int m = 3;
  if (scaled && !vector(a[15], a[7], c.device, rows, in + m++)) return does_not_fit();
  if (zeros && !table(a[16], a[8], c.device, n, k / group, in + m++)) return does_not_fit();
  if (a[17] != Py_None && !vector(a[17], c.dtype, c.device, n, in + m++)) return does_not_fit();
  in[0] = x.address;
  const int64_t dims[5] = {rows, n, k, x.stride[0], out.stride[0]};
  return c.run(dims, 5, in, m, &out.address, 1, 0, 0, stream);
}

// [batch, places, vocabulary], the last axis dense
bool probabilities(PyObject* t, PyObject* dtype, int64_t device, int64_t* shape, int64_t* stride, uint64_t* address) {
  return on(t, dtype, device, address) && numbers(PyObject_GetAttr(t, s_shape), 3, shape) && numbers(PyObject_CallMethodNoArgs(t, s_stride), 3, stride) &&
         (stride[2] == 1 || shape[2] == 1);
}
// verify(fn, ctx, id, dtype, device, 0, fp32, int32, target, drafted, uniforms, tokens, accepted, draft, lengths, workspace, stream)
PyObject* verify(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  Call c;
  uint64_t stream, in[5], out[2], ws, bytes;
  int64_t t[3], ts[3], d[3] = {0, 0, 0}, ds[3] = {0, 0, 0};
  if (n_args != 17 || !c.take(a) || !as_u64(a[16], &stream) || !probabilities(a[8], c.dtype, c.device, t, ts, in)) return does_not_fit();
  const int64_t batch = t[0], drafts = t[1] - 1, vocabulary = t[2];
  int m = 3;
  if (drafts < 0 || !table(a[9], a[7], c.device, batch, drafts, in + 1) || !table(a[10], a[6], c.device, batch, drafts + 1, in + 2) ||
      !table(a[11], a[7], c.device, batch, drafts + 1, out) || !vector(a[12], a[7], c.device, batch, out + 1))
    return does_not_fit();
  const bool drafted = a[13] != Py_None, ragged = a[14] != Py_None;
  if (drafted && (!probabilities(a[13], c.dtype, c.device, d, ds, in + m++) || d[0] != batch || d[1] != drafts || d[2] != vocabulary)) return does_not_fit();
  if (ragged && !vector(a[14], a[7], c.device, batch, in + m++)) return does_not_fit();
  if (!scratch(a[15], c.device, &ws, &bytes)) return does_not_fit();
  const int64_t dims[9] = {batch, drafts, vocabulary, ts[0], ts[1], ds[0], ds[1], drafted, ragged};
  return c.run(dims, 9, in, m, out, 2, ws, bytes, stream);
}

PyMethodDef methods[] = {{"launch", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(launch)), METH_FASTCALL,
                          "launch(fn, ctx, id, dims, inputs, outputs, workspace, workspace_bytes, stream) -> status"},
                         {"rotary", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rotary)), METH_FASTCALL, "status, or None"},
                         {"cache_rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_rows)), METH_FASTCALL, "status, or None"},
                         {"cache_attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_attend)), METH_FASTCALL, "status, or None"},
                         {"norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(norm)), METH_FASTCALL, "status, or None"},
                         {"norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(norm_backward)), METH_FASTCALL, "status, or None"},
                         {"linear4", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear4)), METH_FASTCALL, "status, or None"},
                         {"verify", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(verify)), METH_FASTCALL, "status, or None"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pylaunch", "argument marshalling of disc_launch", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pylaunch() {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_numel = PyUnicode_InternFromString("numel");
  s_element_size = PyUnicode_InternFromString("element_size");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_get_device = PyUnicode_InternFromString("get_device");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  if (!s_data_ptr || !s_numel || !s_element_size || !s_dtype || !s_get_device || !s_shape || !s_stride || !s_is_contiguous) return nullptr;
  return PyModule_Create(&module);
}
