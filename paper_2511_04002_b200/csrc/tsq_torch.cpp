// The per-step calls of the binding, tsq_encode, tsq_decode and those of the paged caches on torch tensors, as a CPython extension: argument
// checks, pointers, sizes and the current stream are read from the tensors in C++ and the C ABI (include/tsq.h) is called
// directly.  A decode step is a few microseconds of GPU work, so what the interpreter spends around the call counts: through
// ctypes, with the stream object that torch.cuda.current_stream() builds, a 64 x 4096 decode took 9.1 us of host time per
// call, of which the stream lookup 3.5 us and the argument conversions about 1.5 us.  The interpreter lock is released around the
// call, as ctypes does: a launch can wait for room in the stream's queue.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <type_traits>

#include "tsq.h"

namespace {

// NULL with a Python error set when `o` is no tensor.
const at::Tensor* tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
    return nullptr;
  }
  return &THPVariable_Unpack(o);
}

// None: the current stream of the current device; else an object with a cuda_stream attribute, or the handle as a number.
bool stream_of(PyObject* o, void** out) {
  if (o == Py_None) {
    *out = c10::cuda::getCurrentCUDAStream().stream();
    return true;
  }
  PyObject* handle = PyObject_HasAttrString(o, "cuda_stream") ? PyObject_GetAttrString(o, "cuda_stream") : Py_NewRef(o);
  if (!handle) return false;
  *out = PyLong_AsVoidPtr(handle);
  Py_DECREF(handle);
  return !(*out == nullptr && PyErr_Occurred());
}

// A contiguous [tokens x hidden] CUDA tensor of the plan's type (tokens < 0: any number of rows).
bool check_rows(const at::Tensor& t, long dtype, long hidden, int64_t tokens, const char* name) {
  const at::ScalarType want = dtype == TSQ_BF16 ? at::kBFloat16 : at::kHalf;
  if (t.is_cuda() && t.is_contiguous() && t.scalar_type() == want && t.dim() == 2 && t.size(1) == hidden &&
      (tokens < 0 || t.size(0) == tokens))
    return true;
  PyErr_Format(PyExc_AssertionError, "%s must be a contiguous CUDA tensor [tokens, %ld] of the plan's dtype", name, hidden);
  return false;
}

// encode(plan, dtype, hidden, x, blob, ws, stream) -> status
PyObject* encode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7) return PyErr_Format(PyExc_TypeError, "encode takes 7 arguments");
  const auto* plan = static_cast<const tsq_plan_t*>(PyLong_AsVoidPtr(a[0]));
  const long dtype = PyLong_AsLong(a[1]), hidden = PyLong_AsLong(a[2]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor *x = tensor(a[3], "x"), *blob = x ? tensor(a[4], "blob") : nullptr, *ws = blob ? tensor(a[5], "ws") : nullptr;
  void* stream = nullptr;
  if (!ws || !check_rows(*x, dtype, hidden, -1, "x") || !stream_of(a[6], &stream)) return nullptr;
  const void* xp = x->data_ptr();
  void *bp = blob->data_ptr(), *wp = ws->data_ptr();
  const int64_t tokens = x->size(0);
  const size_t blob_bytes = static_cast<size_t>(blob->numel()), ws_bytes = static_cast<size_t>(ws->numel());
  tsq_status_t st;
  Py_BEGIN_ALLOW_THREADS;
  st = tsq_encode(plan, xp, tokens, bp, blob_bytes, wp, ws_bytes, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(st);
}

// decode(plan, dtype, hidden, blob, tokens, y, ws, stream) -> status
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 8) return PyErr_Format(PyExc_TypeError, "decode takes 8 arguments");
  const auto* plan = static_cast<const tsq_plan_t*>(PyLong_AsVoidPtr(a[0]));
  const long dtype = PyLong_AsLong(a[1]), hidden = PyLong_AsLong(a[2]);
  const long long tokens = PyLong_AsLongLong(a[4]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor *blob = tensor(a[3], "blob"), *y = blob ? tensor(a[5], "y") : nullptr, *ws = y ? tensor(a[6], "ws") : nullptr;
  void* stream = nullptr;
  if (!ws || !check_rows(*y, dtype, hidden, tokens, "y") || !stream_of(a[7], &stream)) return nullptr;
  const void* bp = blob->data_ptr();
  void *yp = y->data_ptr(), *wp = ws->data_ptr();
  const size_t blob_bytes = static_cast<size_t>(blob->numel()), ws_bytes = static_cast<size_t>(ws->numel());
  tsq_status_t st;
  Py_BEGIN_ALLOW_THREADS;
  st = tsq_decode(plan, bp, blob_bytes, tokens, yp, wp, ws_bytes, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(st);
}

// ---- the paged cache ----

// A contiguous int32 tensor of `dims` dimensions on `device`; the first and the second have the given sizes (< 0: any).
bool check_ints(const at::Tensor* t, int device, int64_t dims, int64_t first, int64_t second, const char* name) {
  if (!t) return false;
  if (t->is_cuda() && t->get_device() == device && t->scalar_type() == at::kInt && t->is_contiguous() && t->dim() == dims && (first < 0 || t->size(0) == first) &&
      (dims < 2 || second < 0 || t->size(1) == second))
    return true;
  PyErr_Format(PyExc_AssertionError, "%s must be a contiguous int32 CUDA tensor with %ld dimension(s) on the call's device, of a size that fits the others", name,
               static_cast<long>(dims));
  return false;
}

// Rows [tokens][heads][dim] of the cache's type on its device, the heads of a token contiguous (tokens, heads < 0: any).
bool check_heads(const at::Tensor* t, long dtype, int device, int64_t tokens, int64_t heads, int64_t dim, const char* name) {
  if (!t) return false;
  const at::ScalarType want = dtype == TSQ_BF16 ? at::kBFloat16 : at::kHalf;
  if (t->is_cuda() && t->get_device() == device && t->scalar_type() == want && t->dim() == 3 && (tokens < 0 || t->size(0) == tokens) &&
      (heads < 0 || t->size(1) == heads) && t->size(2) == dim && t->stride(2) == 1 && (t->size(1) == 1 || t->stride(1) == dim))
    return true;
  PyErr_Format(PyExc_AssertionError, "%s must be a CUDA tensor [tokens, heads, %ld] of the cache's dtype on its device, the heads of a token contiguous", name,
               static_cast<long>(dim));
  return false;
}

// Elements between a tensor's tokens; of one token or none, the least that is taken.
int64_t token_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1) * t.size(2); }

// The device that a call is made on, current for as long as it lasts, and its stream.
struct OnDevice {
  c10::cuda::CUDAGuard guard;
  void* stream = nullptr;
  bool ok;
  OnDevice(int device, PyObject* stream_arg) : guard(static_cast<c10::DeviceIndex>(device)), ok(stream_of(stream_arg, &stream)) {}
};

// What a function of this part does, with C++ exceptions (a tensor without storage, a device that is not there) turned into Python's.
template <typename F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// CacheT: tsq_cache_t or tsq_cache4_t.
template <typename CacheT>
const CacheT* cache_of(PyObject* address, PyObject* device, int* out) {
  const auto* cache = static_cast<const CacheT*>(PyLong_AsVoidPtr(address));
  *out = static_cast<int>(PyLong_AsLong(device));
  if (PyErr_Occurred()) return nullptr;
  if (!cache) PyErr_SetString(PyExc_ValueError, "no cache");
  return cache;
}

// cache_slots(page_tokens, held, added, free_pages, query_start, lengths, block_table, slots, taken, stream) -> status
PyObject* cache_slots(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 10) return PyErr_Format(PyExc_TypeError, "cache_slots takes 10 arguments");
  return guarded([&]() -> PyObject* {
    const long page_tokens = PyLong_AsLong(a[0]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor* t[8];
    static const char* const names[8] = {"held", "added", "free_pages", "query_start", "lengths", "block_table", "slots", "taken"};
    for (int i = 0; i < 8; ++i) {
      if (!(t[i] = tensor(a[1 + i], names[i]))) return nullptr;
    }
    if (!t[0]->is_cuda()) return PyErr_Format(PyExc_AssertionError, "held must be a CUDA tensor");
    const int device = t[0]->get_device();
    if (!check_ints(t[0], device, 1, -1, -1, names[0])) return nullptr;
    const int64_t requests = t[0]->size(0);
    if (!check_ints(t[1], device, 1, requests, -1, names[1]) || !check_ints(t[2], device, 1, -1, -1, names[2]) ||
        !check_ints(t[3], device, 1, requests + 1, -1, names[3]) || !check_ints(t[4], device, 1, requests, -1, names[4]) ||
        !check_ints(t[5], device, 2, requests, -1, names[5]) || !check_ints(t[6], device, 1, -1, -1, names[6]) || !check_ints(t[7], device, 1, 1, -1, names[7]))
      return nullptr;
    OnDevice on(device, a[9]);
    if (!on.ok) return nullptr;
    const int64_t most = 0x7fffffff;
    if (page_tokens < 0 || page_tokens > most || requests > most || t[2]->size(0) > most || t[5]->size(1) > most) return PyLong_FromLong(TSQ_ERR_INVALID_ARG);
    const auto in = [&](int i) { return static_cast<const int32_t*>(t[i]->data_ptr()); };
    const auto out = [&](int i) { return static_cast<int32_t*>(t[i]->data_ptr()); };
    tsq_status_t st;
    Py_BEGIN_ALLOW_THREADS;
    st = tsq_cache_slots(static_cast<int32_t>(page_tokens), in(0), in(1), static_cast<int32_t>(requests), in(2), static_cast<int32_t>(t[2]->size(0)), out(3), out(4),
                         out(5), static_cast<int32_t>(t[5]->size(1)), out(6), t[6]->size(0), out(7), on.stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(st);
  });
}

tsq_status_t store_rows(const tsq_cache_t* c, const void* k, int64_t ks, const void* v, int64_t vs, int64_t tokens, const int32_t* slots, void* stream) {
  return tsq_cache_store(c, k, ks, v, vs, tokens, slots, stream);
}
tsq_status_t store_rows(const tsq_cache4_t* c, const void* k, int64_t ks, const void* v, int64_t vs, int64_t tokens, const int32_t* slots, void* stream) {
  return tsq_cache4_store(c, k, ks, v, vs, tokens, slots, stream);
}
tsq_status_t load_rows(const tsq_cache_t* c, const int32_t* slots, int64_t tokens, void* k, int64_t ks, void* v, int64_t vs, void* stream) {
  return tsq_cache_load(c, slots, tokens, k, ks, v, vs, stream);
}
tsq_status_t load_rows(const tsq_cache4_t* c, const int32_t* slots, int64_t tokens, void* k, int64_t ks, void* v, int64_t vs, void* stream) {
  return tsq_cache4_load(c, slots, tokens, k, ks, v, vs, stream);
}

// cache_store(cache, device, k, v, slots, stream) -> status; cache_load(cache, device, slots, k, v, stream) -> status; cache4_store, cache4_load the same
template <typename CacheT>
PyObject* move_rows(PyObject* const* a, bool store) {
  return guarded([&]() -> PyObject* {
    int device = 0;
    const CacheT* const cache = cache_of<CacheT>(a[0], a[1], &device);
    if (!cache) return nullptr;
    const at::Tensor *k = tensor(a[store ? 2 : 3], "k"), *v = k ? tensor(a[store ? 3 : 4], "v") : nullptr, *slots = v ? tensor(a[store ? 4 : 2], "slots") : nullptr;
    if (!check_ints(slots, device, 1, -1, -1, "slots")) return nullptr;
    const int64_t tokens = slots->size(0);
    if (!check_heads(k, cache->dtype, device, tokens, cache->kv_heads, cache->head_dim, "k") ||
        !check_heads(v, cache->dtype, device, tokens, cache->kv_heads, cache->head_dim, "v"))
      return nullptr;
    OnDevice on(device, a[5]);
    if (!on.ok) return nullptr;
    void *kp = k->data_ptr(), *vp = v->data_ptr();
    const auto* sp = static_cast<const int32_t*>(slots->data_ptr());
    const int64_t ks = token_stride(*k), vs = token_stride(*v);
    tsq_status_t st;
    Py_BEGIN_ALLOW_THREADS;
    st = store ? store_rows(cache, kp, ks, vp, vs, tokens, sp, on.stream) : load_rows(cache, sp, tokens, kp, ks, vp, vs, on.stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(st);
  });
}
template <typename CacheT, bool STORE>
PyObject* move_call(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return n == 6 ? move_rows<CacheT>(a, STORE) : PyErr_Format(PyExc_TypeError, "a call that moves rows takes 6 arguments");
}

tsq_status_t attend(const tsq_cache_t* c, const void* q, int64_t qs, int32_t heads, int64_t tokens, const int32_t* start, const int32_t* lengths, int32_t requests, int32_t most,
                    const int32_t* table, int32_t width, float scale, int32_t, void* out, int64_t os, void* ws, size_t ws_bytes, void* stream) {
  return tsq_cache_attention(c, q, qs, heads, tokens, start, lengths, requests, most, table, width, scale, out, os, ws, ws_bytes, stream);
}
tsq_status_t attend(const tsq_cache4_t* c, const void* q, int64_t qs, int32_t heads, int64_t tokens, const int32_t* start, const int32_t* lengths, int32_t requests, int32_t most,
                    const int32_t* table, int32_t width, float scale, int32_t causal, void* out, int64_t os, void* ws, size_t ws_bytes, void* stream) {
  return tsq_cache4_attention(c, q, qs, heads, tokens, start, lengths, requests, most, table, width, scale, causal, out, os, ws, ws_bytes, stream);
}

// cache_attention(cache, device, q, query_start, lengths, block_table, out, ws, max_query, scale, stream) -> status; cache4_attention the same with `causal` in front of the stream
template <typename CacheT>
PyObject* attention_call(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr bool kMayBeWhole = std::is_same<CacheT, tsq_cache4_t>::value;
  constexpr Py_ssize_t kArguments = kMayBeWhole ? 12 : 11;
  if (n != kArguments) return PyErr_Format(PyExc_TypeError, "this call of attention takes %zd arguments", kArguments);
  return guarded([&]() -> PyObject* {
    int device = 0;
    const CacheT* const cache = cache_of<CacheT>(a[0], a[1], &device);
    if (!cache) return nullptr;
    const at::Tensor* t[6];
    static const char* const names[6] = {"q", "query_start", "lengths", "block_table", "out", "ws"};
    for (int i = 0; i < 6; ++i) {
      if (!(t[i] = tensor(a[2 + i], names[i]))) return nullptr;
    }
    const long long max_query = PyLong_AsLongLong(a[8]);
    const double scale = PyFloat_AsDouble(a[9]);
    const int causal = kMayBeWhole ? PyObject_IsTrue(a[10]) : 1;
    if (PyErr_Occurred()) return nullptr;
    if (!check_ints(t[2], device, 1, -1, -1, names[2])) return nullptr;
    const int64_t requests = t[2]->size(0);
    if (!check_ints(t[1], device, 1, requests + 1, -1, names[1]) || !check_ints(t[3], device, 2, requests, -1, names[3]) ||
        !check_heads(t[0], cache->dtype, device, -1, -1, cache->head_dim, names[0]) ||
        !check_heads(t[4], cache->dtype, device, t[0]->size(0), t[0]->size(1), cache->head_dim, names[4]))
      return nullptr;
    if (!t[5]->is_cuda() || t[5]->get_device() != device || t[5]->scalar_type() != at::kByte || !t[5]->is_contiguous())
      return PyErr_Format(PyExc_AssertionError, "ws must be a contiguous uint8 CUDA tensor on the cache's device");
    OnDevice on(device, a[kArguments - 1]);
    if (!on.ok) return nullptr;
    const int64_t most = 0x7fffffff;
    if (max_query < 1 || max_query > most || t[0]->size(1) > most || requests > most || t[3]->size(1) > most) return PyLong_FromLong(TSQ_ERR_INVALID_ARG);
    const auto ints = [&](int i) { return static_cast<const int32_t*>(t[i]->data_ptr()); };
    const void* const qp = t[0]->data_ptr();
    void *const op = t[4]->data_ptr(), *const wp = t[5]->data_ptr();
    tsq_status_t st;
    Py_BEGIN_ALLOW_THREADS;
    st = attend(cache, qp, token_stride(*t[0]), static_cast<int32_t>(t[0]->size(1)), t[0]->size(0), ints(1), ints(2), static_cast<int32_t>(requests),
                static_cast<int32_t>(max_query), ints(3), static_cast<int32_t>(t[3]->size(1)), static_cast<float>(scale), causal, op, token_stride(*t[4]), wp,
                static_cast<size_t>(t[5]->numel()), on.stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(st);
  });
}

// current_stream() -> handle of the current device's current stream
PyObject* current_stream(PyObject*, PyObject*) { return PyLong_FromVoidPtr(c10::cuda::getCurrentCUDAStream().stream()); }

PyMethodDef methods[] = {
    {"encode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(encode)), METH_FASTCALL, nullptr},
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(decode)), METH_FASTCALL, nullptr},
    {"cache_slots", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(cache_slots)), METH_FASTCALL, nullptr},
    {"cache_store", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(move_call<tsq_cache_t, true>)), METH_FASTCALL, nullptr},
    {"cache_load", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(move_call<tsq_cache_t, false>)), METH_FASTCALL, nullptr},
    {"cache_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(attention_call<tsq_cache_t>)), METH_FASTCALL, nullptr},
    {"cache4_store", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(move_call<tsq_cache4_t, true>)), METH_FASTCALL, nullptr},
    {"cache4_load", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(move_call<tsq_cache4_t, false>)), METH_FASTCALL, nullptr},
    {"cache4_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(attention_call<tsq_cache4_t>)), METH_FASTCALL, nullptr},
    {"current_stream", current_stream, METH_NOARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tsq_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tsq_torch(void) { return PyModule_Create(&module); }
