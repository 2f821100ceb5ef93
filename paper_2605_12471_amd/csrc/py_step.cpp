// The Python binding's step, and the calls that stand beside it, in native code: what KvFoldCache.step() does for a call in its ordinary form, from the
// tensors' own fields instead of a dozen Python attributes.  A step was queued from Python in 9.3 us (two launches; 7.1 with one), of which the library and the HIP runtime
// take 5.9 (3.9), and the kernels of a decoding step less than the whole: one token on 1000 keys 7.1 us.
//
// Each answers None for whatever is not in that form -- other types, shapes, devices, layouts, tensors without storage, conflicting
// options, numbers out of range -- and the caller then goes the way of plain Python, which raises what it always has.
#include <Python.h>

#include <c10/core/ScalarType.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <cstdint>
#include <new>

#include "../../include/kvfold.h"

namespace {

struct Cache {
  decltype(&kvfold_step_ex) step_ex;
  decltype(&kvfold_step_noalloc) step_noalloc;
  decltype(&kvfold_step_rope) step_rope;
  decltype(&kvfold_step_window) step_window;
  kvfold_cache_t* handle;
  int64_t device, n_q_heads, n_kv_heads, head_dim;
  c10::ScalarType dtype;
};

// The tensor's memory if it is a plain one of this shape on the device, nullptr if not.
void* plain(PyObject* obj, int64_t device, c10::ScalarType dtype, c10::IntArrayRef shape) {
  if (!THPVariable_CheckExact(obj)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(obj);
  if (!t.defined() || !t.has_storage() || t.layout() != c10::kStrided || !t.is_cuda() || t.get_device() != device || t.scalar_type() != dtype ||
      t.sizes() != shape || !t.is_contiguous())
    return nullptr;
  return t.data_ptr();
}
void* plain(PyObject* obj, const Cache& c, c10::ScalarType dtype, c10::IntArrayRef shape) { return plain(obj, c.device, dtype, shape); }

bool whole_number(PyObject* obj, int64_t lo, int64_t hi, int64_t* out) {
  if (!PyLong_CheckExact(obj)) return false;
  int overflow = 0;
  const long long v = PyLong_AsLongLongAndOverflow(obj, &overflow);
  if (overflow || v < lo || v > hi) return false;
  *out = v;
  return true;
}

void free_cache(PyObject* capsule) { delete static_cast<Cache*>(PyCapsule_GetPointer(capsule, "kvfold")); }

// bind(step_ex, step_noalloc, step_rope, step_window, handle, device, n_q_heads, n_kv_heads, head_dim, bf16): the addresses as integers
PyObject* bind(PyObject*, PyObject* args) {
  unsigned long long f[4], handle;
  long long device, hq, hkv, d;
  int bf16;
  if (!PyArg_ParseTuple(args, "KKKKKLLLLp", &f[0], &f[1], &f[2], &f[3], &handle, &device, &hq, &hkv, &d, &bf16)) return nullptr;
  Cache* c = new (std::nothrow) Cache;
  if (!c) return PyErr_NoMemory();
  c->step_ex = reinterpret_cast<decltype(c->step_ex)>(f[0]);
  c->step_noalloc = reinterpret_cast<decltype(c->step_noalloc)>(f[1]);
  c->step_rope = reinterpret_cast<decltype(c->step_rope)>(f[2]);
  c->step_window = reinterpret_cast<decltype(c->step_window)>(f[3]);
  c->handle = reinterpret_cast<kvfold_cache_t*>(handle);
  c->device = device;
  c->n_q_heads = hq;
  c->n_kv_heads = hkv;
  c->head_dim = d;
  c->dtype = bf16 ? c10::ScalarType::BFloat16 : c10::ScalarType::Float;
  PyObject* capsule = PyCapsule_New(c, "kvfold", free_cache);
  if (!capsule) delete c;
  return capsule;
}

// step(cache, layer, q, k_new, v_new, out, pos, lse, stream, rope, window, noalloc): the library's status, or None
PyObject* step(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 12) {
    PyErr_SetString(PyExc_TypeError, "step: 12 arguments");
    return nullptr;
  }
  Cache* c = static_cast<Cache*>(PyCapsule_GetPointer(a[0], "kvfold"));
  if (!c) return nullptr;
  try {
    int64_t layer, pos, n_sink = 0, window = 0;
    if (!whole_number(a[1], INT32_MIN, INT32_MAX, &layer) || !whole_number(a[6], INT64_MIN, INT64_MAX, &pos)) Py_RETURN_NONE;
    if (!THPVariable_CheckExact(a[2])) Py_RETURN_NONE;
    const at::Tensor& qt = THPVariable_Unpack(a[2]);
    if (!qt.defined() || qt.dim() != 3) Py_RETURN_NONE;
    const int64_t n = qt.size(0);
    if (n > INT32_MAX) Py_RETURN_NONE;
    const int64_t wide[3] = {n, c->n_q_heads, c->head_dim}, narrow[3] = {n, c->n_kv_heads, c->head_dim}, per_head[2] = {c->n_q_heads, n}, angles[2] = {n, c->head_dim / 2};
    // (An empty tensor has no memory; the library's answer to it comes by the other way.)
    void *q = plain(a[2], *c, c->dtype, wide), *k = plain(a[3], *c, c->dtype, narrow), *v = plain(a[4], *c, c->dtype, narrow), *out = plain(a[5], *c, c->dtype, wide);
    if (!q || !k || !v || !out) Py_RETURN_NONE;
    float* lse = nullptr;
    if (a[7] != Py_None && !(lse = static_cast<float*>(plain(a[7], *c, c10::ScalarType::Float, per_head)))) Py_RETURN_NONE;
    void* stream;
    if (a[8] == Py_None) {
      stream = c10::hip::getCurrentHIPStream((c10::DeviceIndex)c->device).stream();
    } else {
      int64_t s;
      if (!whole_number(a[8], 0, INT64_MAX, &s)) Py_RETURN_NONE;
      stream = reinterpret_cast<void*>(s);
    }
    const bool rope = a[9] != Py_None, win = a[10] != Py_None, noalloc = a[11] == Py_True;
    if (!noalloc && a[11] != Py_False) Py_RETURN_NONE;
    if ((int)rope + (int)win + (int)noalloc > 1) Py_RETURN_NONE;
    const float *cos = nullptr, *sin = nullptr;
    if (rope) {
      if (!PyTuple_CheckExact(a[9]) || PyTuple_GET_SIZE(a[9]) != 2) Py_RETURN_NONE;
      cos = static_cast<const float*>(plain(PyTuple_GET_ITEM(a[9], 0), *c, c10::ScalarType::Float, angles));
      sin = static_cast<const float*>(plain(PyTuple_GET_ITEM(a[9], 1), *c, c10::ScalarType::Float, angles));
      if (!cos || !sin) Py_RETURN_NONE;
    }
    if (win) {
      if (!PyTuple_CheckExact(a[10]) || PyTuple_GET_SIZE(a[10]) != 2 || !whole_number(PyTuple_GET_ITEM(a[10], 0), INT32_MIN, INT32_MAX, &n_sink) ||
          !whole_number(PyTuple_GET_ITEM(a[10], 1), INT64_MIN, INT64_MAX, &window))
        Py_RETURN_NONE;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    if (win)
      rc = c->step_window(c->handle, (int)layer, q, k, v, (int32_t)n, pos, (int32_t)n_sink, window, out, lse, stream);
    else if (rope)
      rc = c->step_rope(c->handle, (int)layer, q, k, v, (int32_t)n, pos, cos, sin, out, lse, stream);
    else
      rc = (noalloc ? c->step_noalloc : c->step_ex)(c->handle, (int)layer, q, k, v, (int32_t)n, pos, out, lse, stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
  } catch (...) {
    Py_RETURN_NONE;  // (before anything was queued: the library throws nothing)
  }
}

// ---- the calls beside the step --------------------------------------------------------------------------------------------
// The tensor's memory, or nothing where there is none (*ok: it is one or the other).
void* plain_or_none(PyObject* obj, int64_t device, c10::ScalarType dtype, c10::IntArrayRef shape, bool* ok) {
  if (obj == Py_None) return nullptr;
  void* p = plain(obj, device, dtype, shape);
  *ok = *ok && p;
  return p;
}

// The rows of a tensor with three dimensions, -1 for anything else.
int64_t rows_of(PyObject* obj) {
  if (!THPVariable_CheckExact(obj)) return -1;
  const at::Tensor& t = THPVariable_Unpack(obj);
  return t.defined() && t.dim() == 3 && t.size(0) <= INT32_MAX ? t.size(0) : -1;
}

bool stream_of(PyObject* obj, int64_t device, void** out) {
  int64_t s = 0;
  if (obj != Py_None && !whole_number(obj, 0, INT64_MAX, &s)) return false;
  *out = obj == Py_None ? (void*)c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream() : reinterpret_cast<void*>(s);
  return true;
}

bool angles_of(PyObject* obj, int64_t device, int64_t n, int64_t head_dim, const float** cos, const float** sin) {
  *cos = *sin = nullptr;
  if (obj == Py_None) return true;
  if (!PyTuple_CheckExact(obj) || PyTuple_GET_SIZE(obj) != 2) return false;
  const int64_t shape[2] = {n, head_dim / 2};
  *cos = static_cast<const float*>(plain(PyTuple_GET_ITEM(obj, 0), device, c10::ScalarType::Float, shape));
  *sin = static_cast<const float*>(plain(PyTuple_GET_ITEM(obj, 1), device, c10::ScalarType::Float, shape));
  return *cos && *sin;
}

struct Quant {
  decltype(&kvfold_qcache_step) step;
  decltype(&kvfold_qcache_read) read;
  kvfold_qcache_t* handle;
  int64_t device, n_q_heads, n_kv_heads, head_dim;
};
struct Weights {
  decltype(&kvfold_cache_weigh) weigh;
  decltype(&kvfold_cache_evict) evict;
  kvfold_cache_t* handle;
  int64_t device, n_q_heads, n_kv_heads, head_dim, capacity;
  c10::ScalarType dtype;
};
template <class T>
void free_bound(PyObject* capsule) {
  delete static_cast<T*>(PyCapsule_GetPointer(capsule, PyCapsule_GetName(capsule)));
}
template <class T>
PyObject* capsule_of(const T& bound, const char* name) {
  T* c = new (std::nothrow) T(bound);
  if (!c) return PyErr_NoMemory();
  PyObject* capsule = PyCapsule_New(c, name, free_bound<T>);
  if (!capsule) delete c;
  return capsule;
}

// bind_quant(step, read, handle, device, n_q_heads, n_kv_heads, head_dim): the addresses as integers
PyObject* bind_quant(PyObject*, PyObject* args) {
  unsigned long long f[2], handle;
  long long device, hq, hkv, d;
  if (!PyArg_ParseTuple(args, "KKKLLLL", &f[0], &f[1], &handle, &device, &hq, &hkv, &d)) return nullptr;
  return capsule_of(Quant{reinterpret_cast<decltype(&kvfold_qcache_step)>(f[0]), reinterpret_cast<decltype(&kvfold_qcache_read)>(f[1]),
                          reinterpret_cast<kvfold_qcache_t*>(handle), device, hq, hkv, d},
                    "kvfold_quant");
}

// quant_step(cache, layer, q, k_new, v_new, out, pos, lse, stream, rope)
PyObject* quant_step(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 10) {
    PyErr_SetString(PyExc_TypeError, "quant_step: 10 arguments");
    return nullptr;
  }
  const Quant* c = static_cast<Quant*>(PyCapsule_GetPointer(a[0], "kvfold_quant"));
  if (!c) return nullptr;
  try {
    int64_t layer, pos;
    const int64_t n = rows_of(a[2]);
    if (n < 0 || !whole_number(a[1], INT32_MIN, INT32_MAX, &layer) || !whole_number(a[6], INT64_MIN, INT64_MAX, &pos)) Py_RETURN_NONE;
    const int64_t wide[3] = {n, c->n_q_heads, c->head_dim}, narrow[3] = {n, c->n_kv_heads, c->head_dim}, per_head[2] = {c->n_q_heads, n};
    constexpr auto type = c10::ScalarType::BFloat16;
    void *q = plain(a[2], c->device, type, wide), *k = plain(a[3], c->device, type, narrow), *v = plain(a[4], c->device, type, narrow),
         *out = plain(a[5], c->device, type, wide), *stream;
    bool ok = q && k && v && out;
    float* lse = static_cast<float*>(plain_or_none(a[7], c->device, c10::ScalarType::Float, per_head, &ok));
    const float *cos, *sin;
    if (!ok || !stream_of(a[8], c->device, &stream) || !angles_of(a[9], c->device, n, c->head_dim, &cos, &sin)) Py_RETURN_NONE;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = c->step(c->handle, (int)layer, q, k, v, (int32_t)n, pos, cos, sin, out, lse, stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// quant_read(cache, layer, first, k_out, v_out, stream)
PyObject* quant_read(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 6) {
    PyErr_SetString(PyExc_TypeError, "quant_read: 6 arguments");
    return nullptr;
  }
  const Quant* c = static_cast<Quant*>(PyCapsule_GetPointer(a[0], "kvfold_quant"));
  if (!c) return nullptr;
  try {
    int64_t layer, first;
    const int64_t n = rows_of(a[3] == Py_None ? a[4] : a[3]), shape[3] = {n, c->n_kv_heads, c->head_dim};
    if (n < 0 || !whole_number(a[1], INT32_MIN, INT32_MAX, &layer) || !whole_number(a[2], INT64_MIN, INT64_MAX, &first)) Py_RETURN_NONE;
    bool ok = true;
    float* k = static_cast<float*>(plain_or_none(a[3], c->device, c10::ScalarType::Float, shape, &ok));
    float* v = static_cast<float*>(plain_or_none(a[4], c->device, c10::ScalarType::Float, shape, &ok));
    void* stream;
    if (!ok || !stream_of(a[5], c->device, &stream)) Py_RETURN_NONE;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = c->read(c->handle, (int)layer, first, n, k, v, stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// bind_weights(weigh, evict, handle, device, n_q_heads, n_kv_heads, head_dim, capacity, bf16): the addresses as integers
PyObject* bind_weights(PyObject*, PyObject* args) {
  unsigned long long f[2], handle;
  long long device, hq, hkv, d, capacity;
  int bf16;
  if (!PyArg_ParseTuple(args, "KKKLLLLLp", &f[0], &f[1], &handle, &device, &hq, &hkv, &d, &capacity, &bf16)) return nullptr;
  return capsule_of(Weights{reinterpret_cast<decltype(&kvfold_cache_weigh)>(f[0]), reinterpret_cast<decltype(&kvfold_cache_evict)>(f[1]),
                            reinterpret_cast<kvfold_cache_t*>(handle), device, hq, hkv, d, capacity, bf16 ? c10::ScalarType::BFloat16 : c10::ScalarType::Float},
                    "kvfold_weights");
}

// weigh(cache, layer, q, lse, weights, add, rope, stream)
PyObject* weigh(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 8) {
    PyErr_SetString(PyExc_TypeError, "weigh: 8 arguments");
    return nullptr;
  }
  const Weights* c = static_cast<Weights*>(PyCapsule_GetPointer(a[0], "kvfold_weights"));
  if (!c) return nullptr;
  try {
    int64_t layer;
    const int64_t n = rows_of(a[2]);
    if (n < 0 || !whole_number(a[1], INT32_MIN, INT32_MAX, &layer) || (a[5] != Py_True && a[5] != Py_False)) Py_RETURN_NONE;
    const int64_t wide[3] = {n, c->n_q_heads, c->head_dim}, per_head[2] = {c->n_q_heads, n}, all[2] = {c->n_kv_heads, c->capacity};
    constexpr auto f32 = c10::ScalarType::Float;
    void *q = plain(a[2], c->device, c->dtype, wide), *lse = plain(a[3], c->device, f32, per_head), *weights = plain(a[4], c->device, f32, all), *stream;
    const float *cos, *sin;
    if (!q || !lse || !weights || !angles_of(a[6], c->device, n, c->head_dim, &cos, &sin) || !stream_of(a[7], c->device, &stream)) Py_RETURN_NONE;
    const int add = a[5] == Py_True;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = c->weigh(c->handle, (int)layer, q, (int32_t)n, cos, sin, static_cast<float*>(lse), static_cast<float*>(weights), add, stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// evict(cache, layer, weights, n_keep, n_sink, n_recent, target or None, to_layer, to_weights or None, kept, workspace, stream); target: what bind_weights made of it
PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 12) {
    PyErr_SetString(PyExc_TypeError, "evict: 12 arguments");
    return nullptr;
  }
  const Weights* c = static_cast<Weights*>(PyCapsule_GetPointer(a[0], "kvfold_weights"));
  if (!c) return nullptr;
  const Weights* to = a[6] == Py_None ? c : static_cast<Weights*>(PyCapsule_GetPointer(a[6], "kvfold_weights"));
  if (!to) return nullptr;
  try {
    int64_t layer, keep, sink, recent, to_layer;
    if (!whole_number(a[1], INT32_MIN, INT32_MAX, &layer) || !whole_number(a[3], 1, INT64_MAX, &keep) || !whole_number(a[4], INT64_MIN, INT64_MAX, &sink) ||
        !whole_number(a[5], INT64_MIN, INT64_MAX, &recent) || !whole_number(a[7], INT32_MIN, INT32_MAX, &to_layer) || !THPVariable_CheckExact(a[10]))
      Py_RETURN_NONE;
    const int64_t all[2] = {c->n_kv_heads, c->capacity}, target[2] = {c->n_kv_heads, to->capacity}, rows[2] = {c->n_kv_heads, keep};
    const int64_t bytes[1] = {THPVariable_Unpack(a[10]).numel()};
    void *weights = plain(a[2], c->device, c10::ScalarType::Float, all), *kept = plain(a[9], c->device, c10::ScalarType::Int, rows),
         *space = plain(a[10], c->device, c10::ScalarType::Byte, bytes), *stream;
    bool ok = weights && kept && space;
    float* to_weights = static_cast<float*>(plain_or_none(a[8], c->device, c10::ScalarType::Float, target, &ok));
    if (!ok || !stream_of(a[11], c->device, &stream)) Py_RETURN_NONE;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = c->evict(c->handle, (int)layer, static_cast<float*>(weights), keep, sink, recent, a[6] == Py_None ? nullptr : to->handle, (int)to_layer, to_weights,
                  static_cast<int32_t*>(kept), space, (size_t)bytes[0], stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
  } catch (...) {
    Py_RETURN_NONE;
  }
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef fast(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"step", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(step)), METH_FASTCALL, nullptr},
    {"bind_quant", bind_quant, METH_VARARGS, nullptr},
    fast<quant_step>("quant_step"),
    fast<quant_read>("quant_read"),
    {"bind_weights", bind_weights, METH_VARARGS, nullptr},
    fast<weigh>("weigh"),
    fast<evict>("evict"),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "kvfold_py_step", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_kvfold_py_step() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
