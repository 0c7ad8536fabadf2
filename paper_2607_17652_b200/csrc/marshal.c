/* CPython side of the binding: tensors -> raw device pointers -> one C call.
 *
 * Each function takes the context handle (an int), the Python objects of the
 * call in the order of the C entry point and the stream (an int), reads
 * `data_ptr()` of every tensor anew (nothing is kept from one call for the
 * next), fills fb_state / fb_pack on the stack, releases the GIL around the C
 * call and returns its error code.  What it is for: a decode step of a single
 * request is bound by the host, and marshalling through ctypes structures took
 * about 10 us a call (step of one small request: 55.6 us, now 32.2 us; the
 * marshalling part of a call is now about 2 us).
 *
 * The entry points come from libflowblock.so by address (bind), so this module
 * links against nothing. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/flowblock.h"

static PyObject *s_data_ptr;
static PyObject *s_state[7], *s_pack[9];
static PyObject *s_cache[5], *s_dtype, *s_contiguous, *s_numel, *s_device;
static const char* const k_cache[5] = {"kv_len", "tok_pos", "kv_pos", "kv_weight", "page_table"};
static const char* const k_state[7] = {"active", "prefix_len", "L", "R", "tokens", "pe_done", "page_table"};
static const char* const k_pack[9] = {"n_live", "slot_req", "slot_s", "slot_pos0", "slot_kv_len", "slot_flags",
                                      "req_slot_begin", "qtok", "pos"};

/* entry points, in the order of `names` in bind() */
enum { F_PACK, F_ATTN, F_T2T, F_GATE, F_SCATTER, F_SCATTER8, F_ATTN8, F_EMBED, F_HEAD, F_STATIC,
       F_APPEND, F_APPEND8, F_TOKEN, F_TOKEN8, F_EVICT, F_COUNT };
static void* fn[F_COUNT];

static PyObject* bind(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  if (n != F_COUNT) { PyErr_SetString(PyExc_TypeError, "bind: one address per entry point"); return NULL; }
  void* got[F_COUNT];
  for (int i = 0; i < F_COUNT; ++i) {
    got[i] = PyLong_AsVoidPtr(args[i]);
    if (!got[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: null address");
      return NULL;
    }
  }
  for (int i = 0; i < F_COUNT; ++i) fn[i] = got[i];
  Py_RETURN_NONE;
}

/* dtypes(int32, float32, bfloat16, uint8): the torch types that tensors are held against */
enum { T_I32, T_F32, T_BF16, T_U8, T_COUNT };
static PyObject* k_dtype[T_COUNT];
static const char* const k_dtype_name[T_COUNT] = {"int32", "float32", "bfloat16", "uint8"};
static PyObject* dtypes(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  (void)self;
  if (n != T_COUNT) { PyErr_SetString(PyExc_TypeError, "dtypes: one object per type"); return NULL; }
  for (int i = 0; i < T_COUNT; ++i) { Py_INCREF(args[i]); Py_XSETREF(k_dtype[i], args[i]); }
  Py_RETURN_NONE;
}

/* None -> NULL, an int -> itself, anything else -> its data_ptr() */
static int as_ptr(PyObject* o, void** out) {
  if (o == Py_None) { *out = NULL; return 0; }
  if (PyLong_Check(o)) {
    *out = PyLong_AsVoidPtr(o);
    return *out == NULL && PyErr_Occurred() ? -1 : 0;
  }
  PyObject* v = PyObject_CallMethodNoArgs(o, s_data_ptr);
  if (!v) return -1;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return *out == NULL && PyErr_Occurred() ? -1 : 0;
}

static int fill(PyObject* o, PyObject* const* names, int n, void** out) {
  for (int i = 0; i < n; ++i) {
    PyObject* t = PyObject_GetAttr(o, names[i]);
    if (!t) return -1;
    const int e = as_ptr(t, &out[i]);
    Py_DECREF(t);
    if (e) return -1;
  }
  return 0;
}
_Static_assert(sizeof(fb_state) == 7 * sizeof(void*) && sizeof(fb_pack) == 9 * sizeof(void*), "plain pointer structures");

static int as_int(PyObject* o, int32_t* out) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) return -1;
  if (v < INT32_MIN || v > INT32_MAX) { PyErr_SetString(PyExc_OverflowError, "value does not fit in 32 bits"); return -1; }
  *out = (int32_t)v;
  return 0;
}

/* A tensor of the calls that decode one token at a time: its type, that it is contiguous, how many elements it has (at
 * least that many where `more` is set: pools and workspaces) and on which device it is; None and raw pointers pass as
 * they are.  About 0.2 us a tensor. */
static int number(PyObject* o, PyObject* method, long long* out) {
  PyObject* v = PyObject_CallMethodNoArgs(o, method);
  if (!v) return -1;
  *out = PyLong_AsLongLong(v);
  Py_DECREF(v);
  return *out == -1 && PyErr_Occurred() ? -1 : 0;
}
static int as_tensor(PyObject* o, const char* call, const char* name, int type, long long numel, int more, long device, void** out) {
  if (o == Py_None || PyLong_Check(o)) return as_ptr(o, out);
  PyObject* dt = PyObject_GetAttr(o, s_dtype);
  if (!dt) return -1;
  const int same = dt == k_dtype[type];
  Py_DECREF(dt);
  long long n, dev;
  if (number(o, s_numel, &n) || number(o, s_device, &dev)) return -1;
  PyObject* c = PyObject_CallMethodNoArgs(o, s_contiguous);
  if (!c) return -1;
  const int contiguous = c == Py_True;
  Py_DECREF(c);
  if (!same || !contiguous || (more ? n < numel : n != numel) || dev != device) {
    PyErr_Format(PyExc_ValueError, "%s: %s must be a contiguous %s tensor of %s%lld elements on device %ld (the current one)", call,
                 name, k_dtype_name[type], more ? "at least " : "", numel, device);
    return -1;
  }
  return as_ptr(o, out);
}

#define ARGS(count, name)                                                                        \
  (void)self;                                                                                    \
  if (n != (count)) { PyErr_SetString(PyExc_TypeError, name ": wrong number of arguments"); return NULL; } \
  if (!fn[F_PACK]) { PyErr_SetString(PyExc_RuntimeError, "the library is not bound"); return NULL; } \
  void* ctx;                                                                                     \
  if (as_ptr(a[0], &ctx)) return NULL;
#define STATE(i, st) fb_state st; if (fill(a[i], s_state, 7, (void**)&st)) return NULL;
#define PACK(i, pk) fb_pack pk; if (fill(a[i], s_pack, 9, (void**)&pk)) return NULL;
#define PTRS(first, count) void* q[count]; for (int i = 0; i < (count); ++i) if (as_ptr(a[(first) + i], &q[i])) return NULL;
#define CALL(expr) int rc; Py_BEGIN_ALLOW_THREADS rc = (expr); Py_END_ALLOW_THREADS return PyLong_FromLong(rc);
#define FN(index, f) ((__typeof__(&f))fn[index])

/* handle, st, pk, ws, status, stream */
static PyObject* m_pack(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  ARGS(6, "pack") STATE(1, st) PACK(2, pk) PTRS(3, 3)
  CALL(FN(F_PACK, fb_pack_wavefronts)(ctx, &st, &pk, q[0], q[1], q[2]))
}
/* handle, pk, q, k_win, v_win, k_pool, v_pool, page_table, out, ws, status, stream */
static PyObject* m_attn(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  ARGS(12, "attn") PACK(1, pk) PTRS(2, 10)
  CALL(FN(F_ATTN, fb_wavefront_attn)(ctx, &pk, q[0], q[1], q[2], q[3], q[4], q[5], q[6], q[7], q[8], q[9]))
}
/* handle, pk, q, k_pool8, v_pool8, k_scale, v_scale, page_table, out, ws, status, stream */
static PyObject* m_attn8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  ARGS(12, "attn_fp8") PACK(1, pk) PTRS(2, 10)
  CALL(FN(F_ATTN8, fb_wavefront_attn_fp8)(ctx, &pk, q[0], q[1], q[2], q[3], q[4], q[5], q[6], q[7], q[8], q[9]))
}
/* handle, pk, logits, st, argmax, conf, action, slot_stats, status, stream */
static PyObject* m_t2t(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  ARGS(10, "t2t") PACK(1, pk) STATE(3, st) PTRS(4, 6)
  void* logits;
  if (as_ptr(a[2], &logits)) return NULL;
  CALL(FN(F_T2T, fb_t2t_step)(ctx, &pk, logits, &st, q[0], q[1], q[2], q[3], q[4], q[5]))
}
/* handle, pk, slot_stats, st, k_win, v_win, k_pool, v_pool, n_committed, spawned, step_counters, status, stream */
static PyObject* m_gate(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  ARGS(13, "gate") PACK(1, pk) STATE(3, st) PTRS(4, 9)
  void* stats;
  if (as_ptr(a[2], &stats)) return NULL;
  CALL(FN(F_GATE, fb_gate_commit)(ctx, &pk, stats, &st, q[0], q[1], q[2], q[3], q[4], q[5], q[6], q[7], q[8]))
}
/* handle, pk, page_table, k_new, v_new, k_pool, v_pool, rope_base, status, stream */
static PyObject* m_scatter(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  ARGS(10, "scatter") PACK(1, pk) PTRS(2, 5)
  void *status, *stream;
  const double base = PyFloat_AsDouble(a[7]);
  if (base == -1.0 && PyErr_Occurred()) return NULL;
  if (as_ptr(a[8], &status) || as_ptr(a[9], &stream)) return NULL;
  CALL(FN(F_SCATTER, fb_scatter_window_kv)(ctx, &pk, q[0], q[1], q[2], q[3], q[4], (float)base, status, stream))
}
/* handle, pk, page_table, k_new, v_new, k_pool8, v_pool8, k_scale, v_scale, rope_base, status, stream */
static PyObject* m_scatter8(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  ARGS(12, "scatter_fp8") PACK(1, pk) PTRS(2, 7)
  void *status, *stream;
  const double base = PyFloat_AsDouble(a[9]);
  if (base == -1.0 && PyErr_Occurred()) return NULL;
  if (as_ptr(a[10], &status) || as_ptr(a[11], &stream)) return NULL;
  CALL(FN(F_SCATTER8, fb_scatter_window_kv_fp8)(ctx, &pk, q[0], q[1], q[2], q[3], q[4], q[5], q[6], (float)base, status,
                                                stream))
}
/* handle, pk, table, table_rows, hidden, x, status, stream */
static PyObject* m_embed(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  ARGS(8, "embed") PACK(1, pk) PTRS(5, 3)
  void* table;
  int32_t rows, hidden;
  if (as_ptr(a[2], &table) || as_int(a[3], &rows) || as_int(a[4], &hidden)) return NULL;
  CALL(FN(F_EMBED, fb_embed_gather)(ctx, &pk, table, rows, hidden, q[0], q[1], q[2]))
}
/* handle, pk, x, w, hidden, st, argmax, conf, action, slot_stats, ws, status, stream */
static PyObject* m_head(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  ARGS(13, "lm_head") PACK(1, pk) STATE(5, st) PTRS(6, 7)
  void *x, *w;
  int32_t hidden;
  if (as_ptr(a[2], &x) || as_ptr(a[3], &w) || as_int(a[4], &hidden)) return NULL;
  CALL(FN(F_HEAD, fb_lm_head_t2t)(ctx, &pk, x, w, hidden, &st, q[0], q[1], q[2], q[3], q[4], q[5], q[6]))
}
/* handle, st, pk, q, k_win, v_win, k_pool, v_pool, out, status, stream */
static PyObject* m_static(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  ARGS(11, "attn_static") STATE(1, st) PACK(2, pk) PTRS(3, 8)
  CALL(FN(F_STATIC, fb_wavefront_attn_static)(ctx, &st, &pk, q[0], q[1], q[2], q[3], q[4], q[5], q[6], q[7]))
}

/* `sizes` of a context, in elements (binding.Context): requests, records, page table, a K or V row a request, a q row a
 * request, a pool, KV heads, bytes of workspace of the attention without and with weights and of the
 * eviction, whether the pools hold 8 bits */
enum { Z_REQ, Z_REC, Z_PT, Z_KV, Z_Q, Z_POOL, Z_HEADS, Z_WS, Z_WS_WEIGHTS, Z_WS_EVICT, Z_FP8, Z_COUNT };
static int as_sizes(PyObject* o, long long* z) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != Z_COUNT) { PyErr_SetString(PyExc_TypeError, "sizes"); return -1; }
  for (int i = 0; i < Z_COUNT; ++i)
    if ((z[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i))) == -1 && PyErr_Occurred()) return -1;
  return 0;
}
static int as_cache(PyObject* o, const char* call, const long long* z, long device, fb_cache* kv) {
  static const int type[5] = {T_I32, T_I32, T_I32, T_F32, T_I32}, size[5] = {Z_REQ, Z_REQ, Z_REC, Z_REC, Z_PT};
  for (int i = 0; i < 5; ++i) {
    PyObject* t = PyObject_GetAttr(o, s_cache[i]);
    if (!t) return -1;
    const int e = as_tensor(t, call, k_cache[i], type[i], z[size[i]], 0, device, (void**)kv + i);
    Py_DECREF(t);
    if (e) return -1;
  }
  return 0;
}
_Static_assert(sizeof(fb_cache) == 5 * sizeof(void*), "plain pointer structure");
#define CACHE(name)                                                                    \
  long long z[Z_COUNT];                                                                \
  fb_cache kv;                                                                         \
  const long dev = PyLong_AsLong(a[2]);                                                \
  if ((dev == -1 && PyErr_Occurred()) || as_sizes(a[1], z) || as_cache(a[3], name, z, dev, &kv)) return NULL;
#define TENSOR(var, i, call, name, type, numel, more) \
  void* var;                                          \
  if (as_tensor(a[i], call, name, type, numel, more, dev, &var)) return NULL;

/* handle, sizes, device, cache, k_new, v_new, k_pool, v_pool, rope_base, status, stream[, k_scale, v_scale] */
static PyObject* append(PyObject* self, PyObject* const* a, Py_ssize_t n, int fp8) {
  ARGS(fp8 ? 13 : 11, "append") CACHE("fb_append_kv")
  TENSOR(k, 4, "fb_append_kv", "k_new", T_BF16, z[Z_KV], 0) TENSOR(v, 5, "fb_append_kv", "v_new", T_BF16, z[Z_KV], 0)
  TENSOR(kp, 6, "fb_append_kv", "k_pool", fp8 ? T_U8 : T_BF16, z[Z_POOL], 1)
  TENSOR(vp, 7, "fb_append_kv", "v_pool", fp8 ? T_U8 : T_BF16, z[Z_POOL], 1)
  TENSOR(status, 9, "fb_append_kv", "status", T_I32, 1, 1)
  void *ks = NULL, *vs = NULL, *stream;
  if (fp8 && (as_tensor(a[11], "fb_append_kv", "k_scale", T_F32, z[Z_HEADS], 0, dev, &ks) ||
              as_tensor(a[12], "fb_append_kv", "v_scale", T_F32, z[Z_HEADS], 0, dev, &vs))) return NULL;
  const double base = PyFloat_AsDouble(a[8]);
  if (base == -1.0 && PyErr_Occurred()) return NULL;
  if (as_ptr(a[10], &stream)) return NULL;
  if (fp8) { CALL(FN(F_APPEND8, fb_append_kv_fp8)(ctx, &kv, k, v, kp, vp, ks, vs, (float)base, status, stream)) }
  CALL(FN(F_APPEND, fb_append_kv)(ctx, &kv, k, v, kp, vp, (float)base, status, stream))
}
static PyObject* m_append(PyObject* self, PyObject* const* a, Py_ssize_t n) { return append(self, a, n, 0); }
static PyObject* m_append8(PyObject* self, PyObject* const* a, Py_ssize_t n) { return append(self, a, n, 1); }

/* handle, sizes, device, cache, q, k_pool, v_pool, out, accumulate, ws, status, stream[, k_scale, v_scale] */
static PyObject* token(PyObject* self, PyObject* const* a, Py_ssize_t n, int fp8) {
  ARGS(fp8 ? 14 : 12, "token_attn") CACHE("fb_token_attn")
  int32_t accumulate;
  if (as_int(a[8], &accumulate)) return NULL;
  TENSOR(q, 4, "fb_token_attn", "q", T_BF16, z[Z_Q], 0)
  TENSOR(kp, 5, "fb_token_attn", "k_pool", fp8 ? T_U8 : T_BF16, z[Z_POOL], 1)
  TENSOR(vp, 6, "fb_token_attn", "v_pool", fp8 ? T_U8 : T_BF16, z[Z_POOL], 1)
  TENSOR(out, 7, "fb_token_attn", "out", T_BF16, z[Z_Q], 0)
  TENSOR(ws, 9, "fb_token_attn", "ws", T_U8, z[accumulate ? Z_WS_WEIGHTS : Z_WS], 1)
  TENSOR(status, 10, "fb_token_attn", "status", T_I32, 1, 1)
  void *ks = NULL, *vs = NULL, *stream;
  if (fp8 && (as_tensor(a[12], "fb_token_attn", "k_scale", T_F32, z[Z_HEADS], 0, dev, &ks) ||
              as_tensor(a[13], "fb_token_attn", "v_scale", T_F32, z[Z_HEADS], 0, dev, &vs))) return NULL;
  if (as_ptr(a[11], &stream)) return NULL;
  if (fp8) { CALL(FN(F_TOKEN8, fb_token_attn_fp8)(ctx, &kv, q, kp, vp, ks, vs, out, accumulate, ws, status, stream)) }
  CALL(FN(F_TOKEN, fb_token_attn)(ctx, &kv, q, kp, vp, out, accumulate, ws, status, stream))
}
static PyObject* m_token(PyObject* self, PyObject* const* a, Py_ssize_t n) { return token(self, a, n, 0); }
static PyObject* m_token8(PyObject* self, PyObject* const* a, Py_ssize_t n) { return token(self, a, n, 1); }

/* handle, sizes, device, cache, keep, recent, sinks, k_pool, v_pool, ws, status, stream */
static PyObject* m_evict(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  ARGS(12, "evict") CACHE("fb_evict_kv")
  int32_t recent, sinks;
  void* stream;
  if (as_int(a[5], &recent) || as_int(a[6], &sinks) || as_ptr(a[11], &stream)) return NULL;
  TENSOR(keep, 4, "fb_evict_kv", "keep", T_I32, z[Z_REQ], 0)
  TENSOR(kp, 7, "fb_evict_kv", "k_pool", z[Z_FP8] ? T_U8 : T_BF16, z[Z_POOL], 1)
  TENSOR(vp, 8, "fb_evict_kv", "v_pool", z[Z_FP8] ? T_U8 : T_BF16, z[Z_POOL], 1)
  TENSOR(ws, 9, "fb_evict_kv", "ws", T_U8, z[Z_WS_EVICT], 1)
  TENSOR(status, 10, "fb_evict_kv", "status", T_I32, 1, 1)
  CALL(FN(F_EVICT, fb_evict_kv)(ctx, &kv, keep, recent, sinks, kp, vp, ws, status, stream))
}

#define M(name, f) {name, (PyCFunction)(void (*)(void))f, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {
    M("bind", bind), M("pack", m_pack), M("attn", m_attn), M("attn_fp8", m_attn8), M("t2t", m_t2t), M("gate", m_gate),
    M("scatter", m_scatter), M("scatter_fp8", m_scatter8), M("embed", m_embed), M("lm_head", m_head),
    M("attn_static", m_static), M("dtypes", dtypes), M("append", m_append), M("append_fp8", m_append8),
    M("token_attn", m_token), M("token_attn_fp8", m_token8), M("evict", m_evict), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "argument marshalling of the binding", -1, methods,
                                    NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
  if (!(s_data_ptr = PyUnicode_InternFromString("data_ptr"))) return NULL;
  if (!(s_dtype = PyUnicode_InternFromString("dtype")) || !(s_contiguous = PyUnicode_InternFromString("is_contiguous")) ||
      !(s_numel = PyUnicode_InternFromString("numel")) || !(s_device = PyUnicode_InternFromString("get_device"))) return NULL;
  for (int i = 0; i < 5; ++i) if (!(s_cache[i] = PyUnicode_InternFromString(k_cache[i]))) return NULL;
  for (int i = 0; i < 7; ++i) if (!(s_state[i] = PyUnicode_InternFromString(k_state[i]))) return NULL;
  for (int i = 0; i < 9; ++i) if (!(s_pack[i] = PyUnicode_InternFromString(k_pack[i]))) return NULL;
  return PyModule_Create(&module);
}
