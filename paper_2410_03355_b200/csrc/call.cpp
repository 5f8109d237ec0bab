// Marshalling of the arguments of verify() and of the cache operators from torch tensors to the library, natively.  The binding does the
// same through ctypes, where a call cost 13 to 16 us of host time, more than the GPU needs for a small one; here it only recognises
// calls that need nothing but their pointers taken (all outputs and the workspace given, tensors of the right types on the current
// device) and answers None to everything else, which the binding then handles itself, errors included.
#include <torch/csrc/autograd/python_variable.h>
#include <c10/cuda/CUDAStream.h>

#include <cmath>

#include "lantern.h"

namespace {

using VerifyFn = decltype(&lantern_verify_ex);
VerifyFn g_verify = nullptr;

// bind(address of lantern_verify_ex)
PyObject* bind(PyObject*, PyObject* address) {
  void* p = PyLong_AsVoidPtr(address);
  if (!p && PyErr_Occurred()) return nullptr;
  g_verify = reinterpret_cast<VerifyFn>(p);
  Py_RETURN_NONE;
}

// The pointer of an optional tensor; false if it is anything but a contiguous one of that type on that device.
bool pointer(PyObject* o, at::ScalarType type, int device, void** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  if (!THPVariable_CheckExact(o)) return false;   // (a subclass may have no memory of its own)
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type || !t.is_contiguous()) return false;
  *out = t.data_ptr();
  return true;
}
bool attribute(PyObject* o, PyObject* name, at::ScalarType type, int device, void** out) {
  PyObject* v = PyObject_GetAttr(o, name);
  if (!v) {
    PyErr_Clear();
    return false;
  }
  const bool ok = pointer(v, type, device, out);   // (the attribute keeps the tensor alive)
  Py_DECREF(v);
  return ok;
}

// names of VerifyOutputs' fields
enum { LEN, TOKEN, PATH, STATUS, QA, PX, M, FIELDS };
PyObject* g_names[FIELDS];

// verify(target, draft, cfg_scale, T, tokens, parents, neighbors, delta, uniforms, out, workspace, divergence, top_k) -> status or None
PyObject* call_verify(PyObject* const* a, Py_ssize_t n) {
  if (n != 13 || !g_verify) Py_RETURN_NONE;
  if (!THPVariable_CheckExact(a[0]) || !THPVariable_CheckExact(a[6]) || !THPVariable_CheckExact(a[10]) || !PyLong_CheckExact(a[11]) || !PyLong_CheckExact(a[12]))
    Py_RETURN_NONE;
  double scalar[3];
  const int at_scalar[3] = {2, 3, 7};
  for (int i = 0; i < 3; ++i) {
    PyObject* v = a[at_scalar[i]];
    if (PyFloat_CheckExact(v)) scalar[i] = PyFloat_AS_DOUBLE(v);
    else if (PyLong_CheckExact(v)) scalar[i] = PyLong_AsDouble(v);
    else Py_RETURN_NONE;
  }
  const long divergence = PyLong_AsLong(a[11]), top_k = PyLong_AsLong(a[12]);
  if (PyErr_Occurred() || top_k != static_cast<int>(top_k)) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  const at::Tensor& target = THPVariable_Unpack(a[0]);
  const at::Tensor& neighbors = THPVariable_Unpack(a[6]);
  const at::Tensor& workspace = THPVariable_Unpack(a[10]);
  if (!target.is_cuda() || target.dim() != 4 || neighbors.dim() != 2) Py_RETURN_NONE;
  const int device = target.get_device();
  const at::ScalarType type = target.scalar_type();
  const int64_t C = target.size(0), B = target.size(1), R = target.size(2), V = target.size(3), k = neighbors.size(1);
  if ((type != at::kBFloat16 && type != at::kFloat) || (C != 1 && C != 2) || R < 1 || neighbors.size(0) != V || B > INT32_MAX || V > INT32_MAX ||
      R > INT32_MAX || device != c10::cuda::current_device())
    Py_RETURN_NONE;
  const bool sampling = scalar[1] != 0.0;
  if (sampling && (a[8] == Py_None || (a[1] == Py_None && R > 1))) Py_RETURN_NONE;
  void *p_target, *p_draft, *p_tokens, *p_parents, *p_neighbors, *p_uniforms, *p_out[FIELDS], *p_workspace;
  if (!pointer(a[0], type, device, &p_target) || !pointer(a[1], type, device, &p_draft) || !pointer(a[4], at::kInt, device, &p_tokens) ||
      !pointer(a[5], at::kInt, device, &p_parents) || !pointer(a[6], at::kInt, device, &p_neighbors) ||
      !pointer(a[8], at::kFloat, device, &p_uniforms) || !pointer(a[10], at::kByte, device, &p_workspace))
    Py_RETURN_NONE;
  for (int f = 0; f < FIELDS; ++f)
    if (!attribute(a[9], g_names[f], f == QA || f == PX ? at::kFloat : at::kInt, device, &p_out[f])) Py_RETURN_NONE;
  const size_t workspace_bytes = static_cast<size_t>(workspace.numel());
  lantern_status rc;
  cudaStream_t stream = c10::cuda::getCurrentCUDAStream(device).stream();
  Py_BEGIN_ALLOW_THREADS
  rc = g_verify(p_target, p_draft, type == at::kBFloat16 ? LANTERN_BF16 : LANTERN_F32, static_cast<float>(scalar[0]), C == 2,
                static_cast<float>(scalar[1]), static_cast<const int32_t*>(p_tokens), static_cast<const int32_t*>(p_parents),
                static_cast<const int32_t*>(p_neighbors), static_cast<int>(k), static_cast<float>(scalar[2]), static_cast<int>(divergence),
                static_cast<int>(top_k), static_cast<const float*>(p_uniforms), static_cast<int>(B), static_cast<int>(R - 1), static_cast<int>(V),
                static_cast<int32_t*>(p_out[LEN]), static_cast<int32_t*>(p_out[TOKEN]), static_cast<int32_t*>(p_out[PATH]),
                static_cast<int32_t*>(p_out[STATUS]), static_cast<float*>(p_out[QA]), static_cast<float*>(p_out[PX]),
                static_cast<int32_t*>(p_out[M]), p_workspace, workspace_bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

PyObject* verify(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    return call_verify(a, n);
  } catch (...) {   // (a tensor without memory that can be read, say: the binding finds out)
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// ---- the cache operators ------------------------------------------------------------------------------------------------

decltype(&lantern_rotary) g_rotary = nullptr;
decltype(&lantern_cache_append) g_append = nullptr;
decltype(&lantern_cache_attention) g_attention = nullptr;
decltype(&lantern_cache_keep) g_keep = nullptr;
decltype(&lantern_cache_read) g_read = nullptr;

// bind_cache(addresses of rotary, append, attention, keep, read)
PyObject* bind_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* p[5];
  if (n != 5) Py_RETURN_NONE;
  for (int i = 0; i < 5; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i] && PyErr_Occurred()) return nullptr;
  }
  g_rotary = reinterpret_cast<decltype(g_rotary)>(p[0]);
  g_append = reinterpret_cast<decltype(g_append)>(p[1]);
  g_attention = reinterpret_cast<decltype(g_attention)>(p[2]);
  g_keep = reinterpret_cast<decltype(g_keep)>(p[3]);
  g_read = reinterpret_cast<decltype(g_read)>(p[4]);
  Py_RETURN_NONE;
}

// A row tensor [B, R, heads, D] whose components lie side by side.
struct Rows {
  void* data;
  at::ScalarType type;
  int B, R, H, D;
  int64_t stride[3];
};
bool rows(PyObject* o, int device, Rows* r) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.get_device() != device || t.dim() != 4 || t.numel() == 0) return false;
  r->type = t.scalar_type();
  if (r->type != at::kBFloat16 && r->type != at::kFloat) return false;
  for (int i = 0; i < 4; ++i)
    if (t.size(i) > INT32_MAX) return false;
  if (t.stride(3) != 1 && t.size(3) > 1) return false;
  r->B = static_cast<int>(t.size(0)), r->R = static_cast<int>(t.size(1)), r->H = static_cast<int>(t.size(2)), r->D = static_cast<int>(t.size(3));
  for (int i = 0; i < 3; ++i) r->stride[i] = t.stride(i);
  r->data = t.data_ptr();
  return true;
}
bool same_shape(const Rows& x, const Rows& y) { return x.type == y.type && x.B == y.B && x.R == y.R && x.H == y.H && x.D == y.D; }
// An int32 tensor [d0], [d0, d1] or [d0, d1, d2] (unused sizes are -1); None is allowed where `optional`.
bool index(PyObject* o, int device, int64_t d0, int64_t d1, int64_t d2, bool optional, const int32_t** out) {
  *out = nullptr;
  if (o == Py_None) return optional;
  void* p;
  if (!pointer(o, at::kInt, device, &p)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  const int64_t d[3] = {d0, d1, d2};
  const int dims = d1 < 0 ? 1 : d2 < 0 ? 2 : 3;
  if (t.dim() != dims) return false;
  for (int i = 0; i < dims; ++i)
    if (t.size(i) != d[i]) return false;
  *out = static_cast<const int32_t*>(p);
  return true;
}
bool table_of(PyObject* o, int device, int64_t B, const int32_t** out, int* width) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.dim() != 2 || t.size(1) > INT32_MAX) return false;
  *width = static_cast<int>(t.size(1));
  return index(o, device, B, t.size(1), -1, false, out);
}
// The caller's structure behind an address, and the device that its tensors are on, which has to be the current one.
template <class T>
bool handle(PyObject* address, PyObject* device, T** out, int* dev) {
  if (!PyLong_CheckExact(address) || !PyLong_CheckExact(device)) return false;
  *out = static_cast<T*>(PyLong_AsVoidPtr(address));
  *dev = static_cast<int>(PyLong_AsLong(device));
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return *out && *dev == c10::cuda::current_device();
}
bool rotated(PyObject* address, PyObject* device, PyObject* positions, int B, int R, int dev, lantern_rotation* out) {
  lantern_rotation* r;
  int at;
  if (!handle(address, device, &r, &at) || at != dev) return false;
  *out = *r;
  return index(positions, dev, out->axes, B, R, false, &out->positions);
}
int dtype_of(at::ScalarType t) { return t == at::kBFloat16 ? LANTERN_BF16 : LANTERN_F32; }
void* stream_of(int device) { return c10::cuda::getCurrentCUDAStream(device).stream(); }

template <class F>
PyObject* without_lock(F f) {
  lantern_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// rotary(x, positions, rotation address, rotation device, inverse, out)
PyObject* call_rotary(PyObject* const* a, Py_ssize_t n) {
  if (n != 6 || !g_rotary) Py_RETURN_NONE;
  const int dev = c10::cuda::current_device();
  Rows x, out;
  lantern_rotation rot;
  if (!rows(a[0], dev, &x) || !rows(a[5], dev, &out) || !same_shape(x, out) || !rotated(a[2], a[3], a[1], x.B, x.R, dev, &rot)) Py_RETURN_NONE;
  if (x.data == out.data)
    for (int i = 0; i < 3; ++i)
      if (x.stride[i] != out.stride[i]) Py_RETURN_NONE;
  const int inverse = PyObject_IsTrue(a[4]) == 1;
  void* stream = stream_of(dev);
  return without_lock([&] { return g_rotary(x.data, out.data, dtype_of(x.type), x.B, x.R, x.H, x.D, x.stride, out.stride, &rot, inverse, stream); });
}

// append(k, v, cache address, cache device, table, lengths, counts, positions, rotation address or None, rotation device, status)
PyObject* call_append(PyObject* const* a, Py_ssize_t n) {
  if (n != 11 || !g_append) Py_RETURN_NONE;
  lantern_cache* c;
  int dev, width;
  Rows k, v;
  const int32_t *table, *lengths, *counts, *status;
  if (!handle(a[2], a[3], &c, &dev) || !rows(a[0], dev, &k) || !rows(a[1], dev, &v) || !same_shape(k, v) || k.H != c->heads || k.D != c->head_dim ||
      !table_of(a[4], dev, k.B, &table, &width) || !index(a[5], dev, k.B, -1, -1, false, &lengths) || !index(a[6], dev, k.B, -1, -1, true, &counts) ||
      !index(a[10], dev, k.B, -1, -1, true, &status))
    Py_RETURN_NONE;
  lantern_rotation rot;
  const bool turns = a[8] != Py_None;
  if (turns ? !rotated(a[8], a[9], a[7], k.B, k.R, dev, &rot) : a[7] != Py_None) Py_RETURN_NONE;
  void* stream = stream_of(dev);
  return without_lock([&] {
    return g_append(k.data, v.data, dtype_of(k.type), k.B, k.R, k.stride, v.stride, c, table, width, lengths, counts, turns ? &rot : nullptr,
                    const_cast<int32_t*>(status), stream);
  });
}

// attention(q, cache address, cache device, table, lengths, counts, starts, parents, scale or None, out, workspace or None, status)
PyObject* call_attention(PyObject* const* a, Py_ssize_t n) {
  if (n != 12 || !g_attention) Py_RETURN_NONE;
  lantern_cache* c;
  int dev, width;
  Rows q;
  const int32_t *table, *lengths, *counts, *starts, *parents, *status;
  void *out, *workspace;
  if (!handle(a[1], a[2], &c, &dev) || !rows(a[0], dev, &q) || q.D != c->head_dim || q.H % c->heads || a[9] == Py_None || !pointer(a[9], q.type, dev, &out) ||
      !table_of(a[3], dev, q.B, &table, &width) || !index(a[4], dev, q.B, -1, -1, false, &lengths) || !index(a[5], dev, q.B, -1, -1, true, &counts) ||
      !index(a[6], dev, q.B, -1, -1, true, &starts) || !index(a[7], dev, q.B, q.R - 1, -1, true, &parents) || !pointer(a[10], at::kByte, dev, &workspace) ||
      !index(a[11], dev, q.B, -1, -1, true, &status))
    Py_RETURN_NONE;
  const at::Tensor& o = THPVariable_Unpack(a[9]);
  if (o.dim() != 4 || o.size(0) != q.B || o.size(1) != q.R || o.size(2) != q.H || o.size(3) != q.D) Py_RETURN_NONE;
  float scale;
  if (a[8] == Py_None) {
    scale = static_cast<float>(1.0 / std::sqrt(static_cast<double>(q.D)));
  } else if (PyFloat_CheckExact(a[8])) {
    scale = static_cast<float>(PyFloat_AS_DOUBLE(a[8]));
  } else {
    Py_RETURN_NONE;
  }
  size_t bytes = 0;
  if (a[10] != Py_None) bytes = static_cast<size_t>(THPVariable_Unpack(a[10]).numel());
  void* stream = stream_of(dev);
  return without_lock([&] {
    return g_attention(q.data, out, dtype_of(q.type), q.B, q.R, q.H, q.stride, c, table, width, lengths, counts, starts, parents, scale,
                       const_cast<int32_t*>(status), workspace, bytes, stream);
  });
}

// keep(cache address, cache device, table, lengths, accept_len, accept_path, out_lengths, status)
PyObject* call_keep(PyObject* const* a, Py_ssize_t n) {
  if (n != 8 || !g_keep) Py_RETURN_NONE;
  lantern_cache* c;
  int dev, width;
  const int32_t *table, *lengths, *accept, *path, *out, *status;
  if (!handle(a[0], a[1], &c, &dev) || !THPVariable_CheckExact(a[5])) Py_RETURN_NONE;
  const at::Tensor& p = THPVariable_Unpack(a[5]);
  if (p.dim() != 2 || p.size(0) > INT32_MAX || p.size(1) > INT32_MAX) Py_RETURN_NONE;
  const int64_t B = p.size(0), N = p.size(1);
  if (!index(a[5], dev, B, N, -1, false, &path) || !table_of(a[2], dev, B, &table, &width) || !index(a[3], dev, B, -1, -1, false, &lengths) ||
      !index(a[4], dev, B, -1, -1, false, &accept) || !index(a[6], dev, B, -1, -1, false, &out) || !index(a[7], dev, B, -1, -1, true, &status))
    Py_RETURN_NONE;
  void* stream = stream_of(dev);
  return without_lock([&] {
    return g_keep(c, table, width, lengths, accept, path, static_cast<int>(B), static_cast<int>(N), const_cast<int32_t*>(out),
                  const_cast<int32_t*>(status), stream);
  });
}

// read(cache address, cache device, table, first, rows, counts, out_k, out_v, status)
PyObject* call_read(PyObject* const* a, Py_ssize_t n) {
  if (n != 9 || !g_read || !PyLong_CheckExact(a[4])) Py_RETURN_NONE;
  const long R = PyLong_AsLong(a[4]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  lantern_cache* c;
  int dev, width;
  Rows k, v;
  const int32_t *table, *first, *counts, *status;
  if (!handle(a[0], a[1], &c, &dev) || !rows(a[6], dev, &k) || !rows(a[7], dev, &v) || !same_shape(k, v) || k.R != R || k.H != c->heads || k.D != c->head_dim ||
      !THPVariable_Unpack(a[6]).is_contiguous() || !THPVariable_Unpack(a[7]).is_contiguous() || !table_of(a[2], dev, k.B, &table, &width) ||
      !index(a[3], dev, k.B, -1, -1, false, &first) || !index(a[5], dev, k.B, -1, -1, true, &counts) || !index(a[8], dev, k.B, -1, -1, true, &status))
    Py_RETURN_NONE;
  void* stream = stream_of(dev);
  return without_lock([&] {
    return g_read(c, table, width, first, counts, k.B, k.R, dtype_of(k.type), k.data, v.data, const_cast<int32_t*>(status), stream);
  });
}

template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    return F(a, n);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

PyMethodDef kMethods[] = {
    {"bind", bind, METH_O, nullptr},
    {"verify", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(verify)), METH_FASTCALL, nullptr},
    {"bind_cache", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind_cache)), METH_FASTCALL, nullptr},
    {"rotary", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<call_rotary>)), METH_FASTCALL, nullptr},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<call_append>)), METH_FASTCALL, nullptr},
    {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<call_attention>)), METH_FASTCALL, nullptr},
    {"keep", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<call_keep>)), METH_FASTCALL, nullptr},
    {"read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<call_read>)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call() {
  const char* names[FIELDS] = {"accept_len", "next_token", "accept_path", "status", "node_qa", "node_px", "node_m"};
  for (int f = 0; f < FIELDS; ++f) {
    g_names[f] = PyUnicode_InternFromString(names[f]);
    if (!g_names[f]) return nullptr;
  }
  return PyModule_Create(&kModule);
}
