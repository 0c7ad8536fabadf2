// CPython side of the calls that decode one token at a time: as marshal.c, and every tensor is held against the type, the
// number of elements, the contiguity and the device that the call needs before its pointer is taken.  Asking a tensor for
// these through its Python methods takes 0.3 us each, 3 to 4 us a call of a step that runs for 2 to 8 us on the GPU, so this module
// is built against torch's headers and looks into the tensor itself (a call's marshalling 4.1 -> 0.4 us).  The entry points
// come by address (bind), as there.  FB_TORCH_VERSION: torch.__version__ of those headers, whole, since the version in the headers
// leaves out what tells one pre-release from the next.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include "../../include/flowblock.h"

namespace {

PyObject* s_cache[5];
const char* const k_cache[5] = {"kv_len", "tok_pos", "kv_pos", "kv_weight", "page_table"};

// entry points, in the order of `_TOKEN` in binding.py
enum { F_APPEND, F_APPEND8, F_TOKEN, F_TOKEN8, F_EVICT, F_COUNT };
void* fn[F_COUNT];

PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != F_COUNT) { PyErr_SetString(PyExc_TypeError, "bind: one address per entry point"); return nullptr; }
  void* got[F_COUNT];
  for (int i = 0; i < F_COUNT; ++i) {
    got[i] = PyLong_AsVoidPtr(args[i]);
    if (!got[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: null address");
      return nullptr;
    }
  }
  for (int i = 0; i < F_COUNT; ++i) fn[i] = got[i];
  Py_RETURN_NONE;
}

// `sizes` of a context, in elements (binding.Context): requests, records, page table, a K or V row a request, a q row a
// request, a pool, KV heads, bytes of workspace of the attention without and with weights and of the eviction, whether the
// pools hold 8 bits
enum { Z_REQ, Z_REC, Z_PT, Z_KV, Z_Q, Z_POOL, Z_HEADS, Z_WS, Z_WS_WEIGHTS, Z_WS_EVICT, Z_FP8, Z_COUNT };

// One call being put together: the first failure sets the Python error and `ok`, and what comes after does nothing.
struct Call {
  const char* name;
  void* ctx = nullptr;
  long long z[Z_COUNT] = {};
  long device = -1;
  fb_cache kv{};
  bool ok = true;

  // handle, sizes, device, cache, ...
  Call(const char* name_, PyObject* const* a, Py_ssize_t n, Py_ssize_t count) : name(name_) {
    if (n != count) { fail(PyExc_TypeError, "wrong number of arguments"); return; }
    if (!fn[0]) { fail(PyExc_RuntimeError, "the library is not bound"); return; }
    ctx = pointer(a[0]);
    if (!PyTuple_Check(a[1]) || PyTuple_GET_SIZE(a[1]) != Z_COUNT) { fail(PyExc_TypeError, "sizes"); return; }
    for (int i = 0; i < Z_COUNT; ++i)
      if ((z[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(a[1], i))) == -1 && PyErr_Occurred()) { ok = false; return; }
    device = PyLong_AsLong(a[2]);
    if (device == -1 && PyErr_Occurred()) { ok = false; return; }
    static const c10::ScalarType type[5] = {c10::kInt, c10::kInt, c10::kInt, c10::kFloat, c10::kInt};
    static const int size[5] = {Z_REQ, Z_REQ, Z_REC, Z_REC, Z_PT};
    void* got[5] = {};
    for (int i = 0; i < 5 && ok; ++i) {
      PyObject* t = PyObject_GetAttr(a[3], s_cache[i]);
      if (!t) { ok = false; return; }
      got[i] = tensor(t, k_cache[i], type[i], z[size[i]]);
      Py_DECREF(t);                               // (the cache holds it)
    }
    kv.kv_len = static_cast<int32_t*>(got[0]); kv.tok_pos = static_cast<int32_t*>(got[1]);
    kv.kv_pos = static_cast<int32_t*>(got[2]); kv.kv_weight = static_cast<float*>(got[3]);
    kv.page_table = static_cast<int32_t*>(got[4]);
  }
  void fail(PyObject* kind, const char* what) {
    PyErr_Format(kind, "%s: %s", name, what);
    ok = false;
  }
  // None -> null, an int -> itself
  void* pointer(PyObject* o) {
    if (!ok || o == Py_None) return nullptr;
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) ok = false;
    return p;
  }
  int32_t integer(PyObject* o) {
    if (!ok) return 0;
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) ok = false;
    else if (v < INT32_MIN || v > INT32_MAX) fail(PyExc_OverflowError, "value does not fit in 32 bits");
    return (int32_t)v;
  }
  float real(PyObject* o) {
    if (!ok) return 0.f;
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) ok = false;
    return (float)v;
  }
  // a tensor's data (`more`: at least that many elements: pools and workspaces); None and raw pointers pass as they are
  void* tensor(PyObject* o, const char* what, c10::ScalarType type, long long numel, bool more = false) {
    if (!ok) return nullptr;
    if (o == Py_None || PyLong_Check(o)) return pointer(o);
    if (!THPVariable_Check(o)) {
      PyErr_Format(PyExc_TypeError, "%s: %s must be a tensor", name, what);
      ok = false;
      return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    const long long n = t.numel();
    if (t.layout() != c10::kStrided || t.scalar_type() != type || !t.is_contiguous() || (more ? n < numel : n != numel) ||
        (t.is_cuda() ? (long)t.get_device() : -1l) != device) {
      PyErr_Format(PyExc_ValueError, "%s: %s must be a contiguous %s tensor of %s%lld elements on device %ld (the current one)", name,
                   what, c10::toString(type), more ? "at least " : "", numel, device);
      ok = false;
      return nullptr;
    }
    return t.data_ptr();
  }
  c10::ScalarType pool() const { return z[Z_FP8] ? c10::kByte : c10::kBFloat16; }
};

// (nothing that throws a C++ exception may leave a function that Python calls)
template <typename Make>
PyObject* guarded(Make make) {
  try {
    return make();
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}
template <typename Enter>
PyObject* enter(const Call& c, Enter go) {
  if (!c.ok) return nullptr;
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = go();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}
template <typename F>
F entry(int i, F) { return reinterpret_cast<F>(fn[i]); }
#define FN(index, f) entry(index, &f)

// handle, sizes, device, cache, k_new, v_new, k_pool, v_pool, rope_base, status, stream[, k_scale, v_scale]
template <bool F8>
PyObject* m_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Call c(F8 ? "fb_append_kv_fp8" : "fb_append_kv", a, n, F8 ? 13 : 11);
    if (!c.ok) return nullptr;
    const c10::ScalarType pool = F8 ? c10::kByte : c10::kBFloat16;
    void *k = c.tensor(a[4], "k_new", c10::kBFloat16, c.z[Z_KV]), *v = c.tensor(a[5], "v_new", c10::kBFloat16, c.z[Z_KV]);
    void *kp = c.tensor(a[6], "k_pool", pool, c.z[Z_POOL], true), *vp = c.tensor(a[7], "v_pool", pool, c.z[Z_POOL], true);
    const float base = c.real(a[8]);
    int32_t* status = (int32_t*)c.tensor(a[9], "status", c10::kInt, 1, true);
    void* stream = c.pointer(a[10]);
    if constexpr (F8) {
      const float* ks = (const float*)c.tensor(a[11], "k_scale", c10::kFloat, c.z[Z_HEADS]);
      const float* vs = (const float*)c.tensor(a[12], "v_scale", c10::kFloat, c.z[Z_HEADS]);
      return enter(c, [&] { return FN(F_APPEND8, fb_append_kv_fp8)((fb_ctx*)c.ctx, &c.kv, k, v, kp, vp, ks, vs, base, status, stream); });
    } else {
      return enter(c, [&] { return FN(F_APPEND, fb_append_kv)((fb_ctx*)c.ctx, &c.kv, k, v, kp, vp, base, status, stream); });
    }
  });
}

// handle, sizes, device, cache, q, k_pool, v_pool, out, accumulate, ws, status, stream[, k_scale, v_scale]
template <bool F8>
PyObject* m_token(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Call c(F8 ? "fb_token_attn_fp8" : "fb_token_attn", a, n, F8 ? 14 : 12);
    if (!c.ok) return nullptr;
    const c10::ScalarType pool = F8 ? c10::kByte : c10::kBFloat16;
    const int32_t accumulate = c.integer(a[8]);
    void *q = c.tensor(a[4], "q", c10::kBFloat16, c.z[Z_Q]), *out = c.tensor(a[7], "out", c10::kBFloat16, c.z[Z_Q]);
    void *kp = c.tensor(a[5], "k_pool", pool, c.z[Z_POOL], true), *vp = c.tensor(a[6], "v_pool", pool, c.z[Z_POOL], true);
    void* ws = c.tensor(a[9], "ws", c10::kByte, c.z[accumulate ? Z_WS_WEIGHTS : Z_WS], true);
    int32_t* status = (int32_t*)c.tensor(a[10], "status", c10::kInt, 1, true);
    void* stream = c.pointer(a[11]);
    if constexpr (F8) {
      const float* ks = (const float*)c.tensor(a[12], "k_scale", c10::kFloat, c.z[Z_HEADS]);
      const float* vs = (const float*)c.tensor(a[13], "v_scale", c10::kFloat, c.z[Z_HEADS]);
      return enter(c, [&] { return FN(F_TOKEN8, fb_token_attn_fp8)((fb_ctx*)c.ctx, &c.kv, q, kp, vp, ks, vs, out, accumulate, ws, status, stream); });
    } else {
      return enter(c, [&] { return FN(F_TOKEN, fb_token_attn)((fb_ctx*)c.ctx, &c.kv, q, kp, vp, out, accumulate, ws, status, stream); });
    }
  });
}

// handle, sizes, device, cache, keep, recent, sinks, k_pool, v_pool, ws, status, stream
PyObject* m_evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Call c("fb_evict_kv", a, n, 12);
    if (!c.ok) return nullptr;
    const int32_t* keep = (const int32_t*)c.tensor(a[4], "keep", c10::kInt, c.z[Z_REQ]);
    const int32_t recent = c.integer(a[5]), sinks = c.integer(a[6]);
    void *kp = c.tensor(a[7], "k_pool", c.pool(), c.z[Z_POOL], true), *vp = c.tensor(a[8], "v_pool", c.pool(), c.z[Z_POOL], true);
    void* ws = c.tensor(a[9], "ws", c10::kByte, c.z[Z_WS_EVICT], true);
    int32_t* status = (int32_t*)c.tensor(a[10], "status", c10::kInt, 1, true);
    void* stream = c.pointer(a[11]);
    return enter(c, [&] { return FN(F_EVICT, fb_evict_kv)((fb_ctx*)c.ctx, &c.kv, keep, recent, sinks, kp, vp, ws, status, stream); });
  });
}

#define M(name, f) {name, (PyCFunction)(void (*)(void))(PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {M("bind", bind), M("append", m_append<false>), M("append_fp8", m_append<true>), M("token_attn", m_token<false>),
                         M("token_attn_fp8", m_token<true>), M("evict", m_evict), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal_token", "argument marshalling of the token-by-token calls", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal_token(void) {
  for (int i = 0; i < 5; ++i) if (!(s_cache[i] = PyUnicode_InternFromString(k_cache[i]))) return nullptr;
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", FB_TORCH_VERSION) < 0) { Py_DECREF(m); return nullptr; }
  return m;
}
