// The argument marshalling of binding.py's hot calls, in C.
//
// A hot call takes a handful of tensors, turns each into a pointer, one or two into strides, finds the current stream
// and calls the C interface.  Through ctypes that was 7 us of a decode call's 11.6 (a stream object built to be asked
// for its handle 3.4, the pointer and stride objects 2.3, the conversion of eleven arguments 0.9): more than the kernel of
// a short cache takes.  With this module the whole call takes 4.6.  Nothing is computed or kept: every call
// reads its arguments anew (any object with data_ptr(), integers with __index__, ctypes.ArgumentError for what is none).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <initializer_list>

#include "sagekv.h"

namespace {

typedef int (*ScoreFn)(sagekv_ctx *, const void *, const void *, sagekv_strides, int64_t, int32_t, int32_t, float *, int64_t, void *);
typedef int (*SelectFn)(sagekv_ctx *, const float *, int64_t, const void *, const void *, sagekv_strides, int64_t, int32_t, int32_t,
                        int32_t, int32_t *, void *, void *, sagekv_strides, sagekv_cache_state *, void *);
typedef int (*DecodeFn)(sagekv_ctx *, const void *, const void *, const void *, void *, void *, sagekv_strides,
                        const sagekv_cache_state *, void *, float *, void *);
typedef int (*PoolFn)(sagekv_ctx *, const float *, int64_t, int64_t, int32_t, int32_t, float *, int64_t, void *);
typedef int (*BoundsFn)(sagekv_ctx *, const void *, const void *, const void *, int64_t, float *, int64_t, void *);
typedef int (*TopkFn)(sagekv_ctx *, const float *, int64_t, int64_t, int32_t, int32_t *, void *);
typedef int (*RopeFn)(sagekv_ctx *, const sagekv_rope_plan *, const void *, sagekv_rows, int64_t, int32_t, const int32_t *, void *, sagekv_rows, void *);
typedef int (*AppendFn)(sagekv_ctx *, const sagekv_paged_cache *, const void *, const void *, sagekv_rows, int64_t, const int32_t *,
                        const int32_t *, const sagekv_rope_plan *, const void *, sagekv_rows, void *, sagekv_rows, void *);
typedef int (*PagedAttnFn)(sagekv_ctx *, const void *, int64_t, const sagekv_paged_cache *, void *, float *, void *);
typedef int (*PagedScoreFn)(sagekv_ctx *, const void *, const sagekv_paged_cache *, int64_t, int32_t, int32_t, float *, int64_t, void *);
typedef int (*PagedCompactFn)(sagekv_ctx *, const int32_t *, const sagekv_paged_cache *, int64_t, int32_t, int32_t, int32_t, void *, void *,
                              sagekv_strides, sagekv_cache_state *, void *);

ScoreFn g_score;
SelectFn g_select;
DecodeFn g_decode;
PoolFn g_pool;
BoundsFn g_bounds;
TopkFn g_topk;
RopeFn g_rope;
AppendFn g_append;
PagedAttnFn g_paged_attn;
PagedScoreFn g_paged_score;
PagedCompactFn g_paged_compact;
PyObject *g_stream_of;   // callable: handle of the current stream of the current device, as an integer
PyObject *g_arg_error;   // ctypes.ArgumentError
PyObject *g_data_ptr, *g_stride, *g_dtype, *g_shape, *g_get_device, *g_numel, *g_is_contiguous;

// All of these return false with a Python exception set.
bool pointer(PyObject *t, void **out) {
  *out = nullptr;
  if (t == Py_None) return true;
  PyObject *v = PyObject_CallMethodNoArgs(t, g_data_ptr);
  if (v == nullptr) return false;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return PyErr_Occurred() == nullptr;
}

bool integer(PyObject *o, int64_t *out) {
  *out = (int64_t)PyLong_AsUnsignedLongLongMask(o);   // as ctypes: no range check
  if (*out == -1 && PyErr_Occurred() != nullptr) {
    PyErr_Clear();
    PyErr_Format(g_arg_error, "'%.100s' object cannot be interpreted as an integer", Py_TYPE(o)->tp_name);
    return false;
  }
  return true;
}
bool integer(PyObject *o, int32_t *out) {
  int64_t v;
  if (!integer(o, &v)) return false;
  *out = (int32_t)(uint32_t)(uint64_t)v;
  return true;
}

// strides of a [B, H_kv, tokens, 128] tensor whose last dimension is contiguous
bool strides(PyObject *t, sagekv_strides *out) {
  PyObject *v = PyObject_CallMethodNoArgs(t, g_stride);
  if (v == nullptr) return false;
  int64_t s[4] = {0, 0, 0, 0};
  const bool four = PyTuple_Check(v) && PyTuple_GET_SIZE(v) == 4;
  for (int i = 0; four && i < 4; ++i) s[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(v, i));
  Py_DECREF(v);
  if (PyErr_Occurred() != nullptr) return false;
  if (!four || s[3] != 1) {
    PyErr_SetString(PyExc_ValueError, "expected a [B, H_kv, tokens, head_dim] tensor with contiguous head_dim");
    return false;
  }
  out->batch_stride = s[0]; out->head_stride = s[1]; out->token_stride = s[2];
  return true;
}

// strides of a [tokens, heads, 128] tensor whose last dimension is contiguous; None: zeros
bool rows(PyObject *t, sagekv_rows *out) {
  *out = {0, 0};
  if (t == Py_None) return true;
  PyObject *v = PyObject_CallMethodNoArgs(t, g_stride);
  if (v == nullptr) return false;
  int64_t s[3] = {0, 0, 0};
  const bool three = PyTuple_Check(v) && PyTuple_GET_SIZE(v) == 3;
  for (int i = 0; three && i < 3; ++i) s[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(v, i));
  Py_DECREF(v);
  if (PyErr_Occurred() != nullptr) return false;
  if (!three || s[2] != 1) {
    PyErr_SetString(PyExc_ValueError, "expected a [tokens, heads, head_dim] tensor with contiguous head_dim");
    return false;
  }
  out->token_stride = s[0]; out->head_stride = s[1];
  return true;
}

// what a method without arguments returns: an integer (or a truth value)
bool number(PyObject *t, PyObject *method, int64_t *out) {
  PyObject *v = PyObject_CallMethodNoArgs(t, method);
  if (v == nullptr) return false;
  *out = PyLong_AsLongLong(v);
  Py_DECREF(v);
  return PyErr_Occurred() == nullptr;
}

// is t of this type (types are single objects), on this device?
bool of_kind(PyObject *t, PyObject *dtype, int64_t device, bool *yes) {
  PyObject *v = PyObject_GetAttr(t, g_dtype);
  if (v == nullptr) return false;
  *yes = v == dtype;
  Py_DECREF(v);
  if (!*yes) return true;
  int64_t on;
  if (!number(t, g_get_device, &on)) return false;
  *yes = on == device;
  return true;
}

// the context handle: a ctypes c_void_p, an integer or None
bool context(PyObject *o, sagekv_ctx **out) {
  *out = nullptr;
  if (o == Py_None) return true;
  if (PyLong_Check(o)) {
    *out = static_cast<sagekv_ctx *>(PyLong_AsVoidPtr(o));
    return PyErr_Occurred() == nullptr;
  }
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return false;
  const bool ok = b.len == (Py_ssize_t)sizeof(*out);
  if (ok) *out = *static_cast<sagekv_ctx **>(b.buf);
  PyBuffer_Release(&b);
  if (!ok) PyErr_SetString(g_arg_error, "not a context handle");
  return ok;
}

// the ctypes structure CacheState, held for the call
struct State {
  Py_buffer b{};
  sagekv_cache_state *p = nullptr;
  bool get(PyObject *o) {
    if (PyObject_GetBuffer(o, &b, PyBUF_WRITABLE) != 0) return false;
    if (b.len != (Py_ssize_t)sizeof(*p)) {
      PyErr_SetString(PyExc_TypeError, "expected a CacheState");
      return false;
    }
    p = static_cast<sagekv_cache_state *>(b.buf);
    return true;
  }
  ~State() { if (b.obj != nullptr) PyBuffer_Release(&b); }
};

// a ctypes structure that is read during the call; None: null
template <typename T>
struct Given {
  Py_buffer b{};
  const T *p = nullptr;
  bool get(PyObject *o, const char *what) {
    if (o == Py_None) return true;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return false;
    if (b.len != (Py_ssize_t)sizeof(T)) {
      PyErr_Format(PyExc_TypeError, "expected a %s", what);
      return false;
    }
    p = static_cast<const T *>(b.buf);
    return true;
  }
  ~Given() { if (b.obj != nullptr) PyBuffer_Release(&b); }
};
typedef Given<sagekv_paged_cache> Cache;
typedef Given<sagekv_rope_plan> Plan;

bool current_stream(void **out) {
  PyObject *v = PyObject_CallNoArgs(g_stream_of);
  if (v == nullptr) return false;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return PyErr_Occurred() == nullptr;
}

bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  return n == want;
}

template <typename Call>
PyObject *answer(Call call) {
  int code;
  Py_BEGIN_ALLOW_THREADS
  code = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(code);
}

// ctx, q_last, K, n_ctx, n_init, n_recent, scores, scores_row_stride
PyObject *score(PyObject *, PyObject *const *a, Py_ssize_t n) {
  sagekv_ctx *ctx; void *q, *K, *scores, *stream; sagekv_strides ks; int64_t n_ctx, stride; int32_t n_init, n_recent;
  if (!count(n, 8) || !context(a[0], &ctx) || !pointer(a[1], &q) || !pointer(a[2], &K) || !strides(a[2], &ks) ||
      !integer(a[3], &n_ctx) || !integer(a[4], &n_init) || !integer(a[5], &n_recent) || !pointer(a[6], &scores) ||
      !integer(a[7], &stride) || !current_stream(&stream))
    return nullptr;
  return answer([&] { return g_score(ctx, q, K, ks, n_ctx, n_init, n_recent, static_cast<float *>(scores), stride, stream); });
}

// ctx, scores, scores_row_stride, K, V, n_ctx, n_init, n_recent, k, idx, Kc, Vc, state
PyObject *select_compact(PyObject *, PyObject *const *a, Py_ssize_t n) {
  sagekv_ctx *ctx; void *scores, *K, *V, *idx, *Kc, *Vc, *stream; sagekv_strides ks, cs;
  int64_t stride, n_ctx; int32_t n_init, n_recent, k; State st;
  if (!count(n, 13) || !context(a[0], &ctx) || !pointer(a[1], &scores) || !integer(a[2], &stride) || !pointer(a[3], &K) ||
      !pointer(a[4], &V) || !strides(a[3], &ks) || !integer(a[5], &n_ctx) || !integer(a[6], &n_init) ||
      !integer(a[7], &n_recent) || !integer(a[8], &k) || !pointer(a[9], &idx) || !pointer(a[10], &Kc) || !pointer(a[11], &Vc) ||
      !strides(a[10], &cs) || !st.get(a[12]) || !current_stream(&stream))
    return nullptr;
  return answer([&] {
    return g_select(ctx, static_cast<float *>(scores), stride, K, V, ks, n_ctx, n_init, n_recent, k, static_cast<int32_t *>(idx), Kc, Vc,
                    cs, st.p, stream);
  });
}

// ctx, q, k_new, v_new, Kc, Vc, state, out, lse
PyObject *decode_attn(PyObject *, PyObject *const *a, Py_ssize_t n) {
  sagekv_ctx *ctx; void *q, *kn, *vn, *Kc, *Vc, *out, *lse, *stream; sagekv_strides cs; State st;
  if (!count(n, 9) || !context(a[0], &ctx) || !pointer(a[1], &q) || !pointer(a[2], &kn) || !pointer(a[3], &vn) ||
      !pointer(a[4], &Kc) || !pointer(a[5], &Vc) || !strides(a[4], &cs) || !st.get(a[6]) || !pointer(a[7], &out) ||
      !pointer(a[8], &lse) || !current_stream(&stream))
    return nullptr;
  return answer([&] { return g_decode(ctx, q, kn, vn, Kc, Vc, cs, st.p, out, static_cast<float *>(lse), stream); });
}

// ctx, scores, scores_row_stride, n_ctx, n_init, n_recent, pooled, pooled_row_stride
PyObject *pool_scores(PyObject *, PyObject *const *a, Py_ssize_t n) {
  sagekv_ctx *ctx; void *scores, *pooled, *stream; int64_t stride, n_ctx, pooled_stride; int32_t n_init, n_recent;
  if (!count(n, 8) || !context(a[0], &ctx) || !pointer(a[1], &scores) || !integer(a[2], &stride) || !integer(a[3], &n_ctx) ||
      !integer(a[4], &n_init) || !integer(a[5], &n_recent) || !pointer(a[6], &pooled) || !integer(a[7], &pooled_stride) ||
      !current_stream(&stream))
    return nullptr;
  return answer([&] {
    return g_pool(ctx, static_cast<float *>(scores), stride, n_ctx, n_init, n_recent, static_cast<float *>(pooled), pooled_stride, stream);
  });
}

// ctx, q, kmin, kmax, n_blocks, bounds, bounds_row_stride
PyObject *quest_bounds(PyObject *, PyObject *const *a, Py_ssize_t n) {
  sagekv_ctx *ctx; void *q, *kmin, *kmax, *bounds, *stream; int64_t n_blocks, stride;
  if (!count(n, 7) || !context(a[0], &ctx) || !pointer(a[1], &q) || !pointer(a[2], &kmin) || !pointer(a[3], &kmax) ||
      !integer(a[4], &n_blocks) || !pointer(a[5], &bounds) || !integer(a[6], &stride) || !current_stream(&stream))
    return nullptr;
  return answer([&] { return g_bounds(ctx, q, kmin, kmax, n_blocks, static_cast<float *>(bounds), stride, stream); });
}

// ctx, scores, scores_row_stride, n, k_q, idx
PyObject *select_topk(PyObject *, PyObject *const *a, Py_ssize_t n) {
  sagekv_ctx *ctx; void *scores, *idx, *stream; int64_t stride, len; int32_t k_q;
  if (!count(n, 6) || !context(a[0], &ctx) || !pointer(a[1], &scores) || !integer(a[2], &stride) || !integer(a[3], &len) ||
      !integer(a[4], &k_q) || !pointer(a[5], &idx) || !current_stream(&stream))
    return nullptr;
  return answer([&] { return g_topk(ctx, static_cast<float *>(scores), stride, len, k_q, static_cast<int32_t *>(idx), stream); });
}

// ctx, plan, x, n_tokens, n_heads, positions, out
PyObject *rope(PyObject *, PyObject *const *a, Py_ssize_t n) {
  sagekv_ctx *ctx; void *x, *pos, *out, *stream; sagekv_rows xs, os; int64_t tokens; int32_t heads; Plan plan;
  if (!count(n, 7) || !context(a[0], &ctx) || !plan.get(a[1], "RopePlan") || !pointer(a[2], &x) || !rows(a[2], &xs) || !integer(a[3], &tokens) ||
      !integer(a[4], &heads) || !pointer(a[5], &pos) || !pointer(a[6], &out) || !rows(a[6], &os) || !current_stream(&stream))
    return nullptr;
  return answer([&] { return g_rope(ctx, plan.p, x, xs, tokens, heads, static_cast<int32_t *>(pos), out, os, stream); });
}

// ctx, cache, k, v, n_tokens, positions, seqs, plan, q, q_out
PyObject *paged_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  sagekv_ctx *ctx; void *k, *v, *pos, *seqs, *q, *q_out, *stream; sagekv_rows ks, vs, qs, qos; int64_t tokens; Cache cache; Plan plan;
  if (!count(n, 10) || !context(a[0], &ctx) || !cache.get(a[1], "PagedCache") || !pointer(a[2], &k) || !rows(a[2], &ks) || !pointer(a[3], &v) ||
      !rows(a[3], &vs) || !integer(a[4], &tokens) || !pointer(a[5], &pos) || !pointer(a[6], &seqs) || !plan.get(a[7], "RopePlan") ||
      !pointer(a[8], &q) || !rows(a[8], &qs) || !pointer(a[9], &q_out) || !rows(a[9], &qos) || !current_stream(&stream))
    return nullptr;
  if ((tokens > 1 && ks.token_stride != vs.token_stride) || ks.head_stride != vs.head_stride) {
    PyErr_SetString(PyExc_ValueError, "expected k and v with the same strides");
    return nullptr;
  }
  return answer([&] {
    return g_append(ctx, cache.p, k, v, ks, tokens, static_cast<int32_t *>(pos), static_cast<int32_t *>(seqs), plan.p, q, qs, q_out, qos, stream);
  });
}

// ctx, q, cache, out, lse
PyObject *paged_attn(PyObject *, PyObject *const *a, Py_ssize_t n) {
  sagekv_ctx *ctx; void *q, *out, *lse, *stream; sagekv_rows qs; Cache cache;
  if (!count(n, 5) || !context(a[0], &ctx) || !pointer(a[1], &q) || !rows(a[1], &qs) || !cache.get(a[2], "PagedCache") || !pointer(a[3], &out) ||
      !pointer(a[4], &lse) || !current_stream(&stream))
    return nullptr;
  if (q != nullptr && qs.head_stride != 128) {
    PyErr_SetString(PyExc_ValueError, "expected queries whose heads lie side by side");
    return nullptr;
  }
  return answer([&] { return g_paged_attn(ctx, q, qs.token_stride, cache.p, out, static_cast<float *>(lse), stream); });
}

// ctx, q_last, cache, n_ctx, n_init, n_recent, scores, scores_row_stride
PyObject *paged_score(PyObject *, PyObject *const *a, Py_ssize_t n) {
  sagekv_ctx *ctx; void *q, *scores, *stream; int64_t n_ctx, stride; int32_t n_init, n_recent; Cache cache;
  if (!count(n, 8) || !context(a[0], &ctx) || !pointer(a[1], &q) || !cache.get(a[2], "PagedCache") || !integer(a[3], &n_ctx) ||
      !integer(a[4], &n_init) || !integer(a[5], &n_recent) || !pointer(a[6], &scores) || !integer(a[7], &stride) || !current_stream(&stream))
    return nullptr;
  return answer([&] { return g_paged_score(ctx, q, cache.p, n_ctx, n_init, n_recent, static_cast<float *>(scores), stride, stream); });
}

// ctx, idx, cache, n_ctx, n_init, n_recent, k, Kc, Vc, state
PyObject *paged_compact(PyObject *, PyObject *const *a, Py_ssize_t n) {
  sagekv_ctx *ctx; void *idx, *Kc, *Vc, *stream; sagekv_strides cs; int64_t n_ctx; int32_t n_init, n_recent, k; Cache cache; State st;
  if (!count(n, 10) || !context(a[0], &ctx) || !pointer(a[1], &idx) || !cache.get(a[2], "PagedCache") || !integer(a[3], &n_ctx) ||
      !integer(a[4], &n_init) || !integer(a[5], &n_recent) || !integer(a[6], &k) || !pointer(a[7], &Kc) || !strides(a[7], &cs) ||
      !pointer(a[8], &Vc) || !st.get(a[9]) || !current_stream(&stream))
    return nullptr;
  return answer([&] {
    return g_paged_compact(ctx, static_cast<int32_t *>(idx), cache.p, n_ctx, n_init, n_recent, k, Kc, Vc, cs, st.p, stream);
  });
}

// dtype, device, tensors: is each (None: passed over) of that type, on that device?
PyObject *placed(PyObject *, PyObject *const *a, Py_ssize_t n) {
  int64_t device;
  if (n < 2) return PyErr_Format(PyExc_TypeError, "expected a type and a device");
  if (!integer(a[1], &device)) return nullptr;
  bool yes = true;
  for (Py_ssize_t i = 2; yes && i < n; ++i)
    if (a[i] != Py_None && !of_kind(a[i], a[0], device, &yes)) return nullptr;
  return PyBool_FromLong(yes);
}

// dtype, device, n, more, tensors: is each (None: passed over) of that type, on that device, and n elements (or, if `more`, at least n) one
// behind the other?
PyObject *placed_row(PyObject *, PyObject *const *a, Py_ssize_t n) {
  int64_t device, want, elements, contiguous;
  if (n < 4) return PyErr_Format(PyExc_TypeError, "expected a type, a device, a number of elements and a truth value");
  if (!integer(a[1], &device) || !integer(a[2], &want)) return nullptr;
  bool yes = true;
  for (Py_ssize_t i = 4; yes && i < n; ++i) {
    if (a[i] == Py_None) continue;
    if (!of_kind(a[i], a[0], device, &yes) || !number(a[i], g_numel, &elements) || !number(a[i], g_is_contiguous, &contiguous)) return nullptr;
    yes = yes && contiguous != 0 && (elements == want || (elements > want && a[3] == Py_True));
  }
  return PyBool_FromLong(yes);
}

// Kc, Vc, batch, heads, rows: are both [batch, heads, at least so many rows, 128], with the same shape and strides?
PyObject *holds_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
  int64_t want[3];
  if (!count(n, 5) || !integer(a[2], &want[0]) || !integer(a[3], &want[1]) || !integer(a[4], &want[2])) return nullptr;
  PyObject *shape = PyObject_GetAttr(a[0], g_shape), *shape_v = shape != nullptr ? PyObject_GetAttr(a[1], g_shape) : nullptr;
  PyObject *strides = shape_v != nullptr ? PyObject_CallMethodNoArgs(a[0], g_stride) : nullptr;
  PyObject *strides_v = strides != nullptr ? PyObject_CallMethodNoArgs(a[1], g_stride) : nullptr;
  int yes = -1;
  if (strides_v != nullptr) {
    yes = PyTuple_Check(shape) && PyTuple_GET_SIZE(shape) == 4;
    for (int i = 0; yes == 1 && i < 4; ++i) {
      const int64_t size = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i));
      yes = i == 2 ? size >= want[2] : size == (i == 3 ? 128 : want[i]);
    }
    if (PyErr_Occurred() != nullptr) yes = -1;
    if (yes == 1) yes = PyObject_RichCompareBool(shape, shape_v, Py_EQ);
    if (yes == 1) yes = PyObject_RichCompareBool(strides, strides_v, Py_EQ);
  }
  Py_XDECREF(shape);
  Py_XDECREF(shape_v);
  Py_XDECREF(strides);
  Py_XDECREF(strides_v);
  return yes < 0 ? nullptr : PyBool_FromLong(yes);
}

// addresses of the paged cache's entry points (rope, paged_append, paged_attn, paged_score, paged_compact)
PyObject *bind_paged(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!count(n, 5)) return nullptr;
  void *f[5];
  for (int i = 0; i < 5; ++i) {
    f[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred() != nullptr) return nullptr;
  }
  g_rope = reinterpret_cast<RopeFn>(f[0]);
  g_append = reinterpret_cast<AppendFn>(f[1]);
  g_paged_attn = reinterpret_cast<PagedAttnFn>(f[2]);
  g_paged_score = reinterpret_cast<PagedScoreFn>(f[3]);
  g_paged_compact = reinterpret_cast<PagedCompactFn>(f[4]);
  Py_RETURN_NONE;
}

// addresses of the six entry points (score, select_compact, decode_attn, pool_scores, quest_bounds, select_topk), the
// callable that tells the current stream, ctypes.ArgumentError
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!count(n, 8)) return nullptr;
  void *f[6];
  for (int i = 0; i < 6; ++i) {
    f[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred() != nullptr) return nullptr;
  }
  g_score = reinterpret_cast<ScoreFn>(f[0]);
  g_select = reinterpret_cast<SelectFn>(f[1]);
  g_decode = reinterpret_cast<DecodeFn>(f[2]);
  g_pool = reinterpret_cast<PoolFn>(f[3]);
  g_bounds = reinterpret_cast<BoundsFn>(f[4]);
  g_topk = reinterpret_cast<TopkFn>(f[5]);
  Py_XSETREF(g_stream_of, Py_NewRef(a[6]));
  Py_XSETREF(g_arg_error, Py_NewRef(a[7]));
  Py_RETURN_NONE;
}

PyCFunction fast(PyObject *(*f)(PyObject *, PyObject *const *, Py_ssize_t)) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef g_methods[] = {
    {"bind", fast(bind), METH_FASTCALL, nullptr},
    {"bind_paged", fast(bind_paged), METH_FASTCALL, nullptr},
    {"placed", fast(placed), METH_FASTCALL, nullptr},
    {"holds_rows", fast(holds_rows), METH_FASTCALL, nullptr},
    {"placed_row", fast(placed_row), METH_FASTCALL, nullptr},
    {"rope", fast(rope), METH_FASTCALL, nullptr},
    {"paged_append", fast(paged_append), METH_FASTCALL, nullptr},
    {"paged_attn", fast(paged_attn), METH_FASTCALL, nullptr},
    {"paged_score", fast(paged_score), METH_FASTCALL, nullptr},
    {"paged_compact", fast(paged_compact), METH_FASTCALL, nullptr},
    {"score", fast(score), METH_FASTCALL, nullptr},
    {"select_compact", fast(select_compact), METH_FASTCALL, nullptr},
    {"decode_attn", fast(decode_attn), METH_FASTCALL, nullptr},
    {"pool_scores", fast(pool_scores), METH_FASTCALL, nullptr},
    {"quest_bounds", fast(quest_bounds), METH_FASTCALL, nullptr},
    {"select_topk", fast(select_topk), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
  g_data_ptr = PyUnicode_InternFromString("data_ptr");
  g_stride = PyUnicode_InternFromString("stride");
  g_dtype = PyUnicode_InternFromString("dtype");
  g_shape = PyUnicode_InternFromString("shape");
  g_get_device = PyUnicode_InternFromString("get_device");
  g_numel = PyUnicode_InternFromString("numel");
  g_is_contiguous = PyUnicode_InternFromString("is_contiguous");
  for (PyObject *name : {g_data_ptr, g_stride, g_dtype, g_shape, g_get_device, g_numel, g_is_contiguous})
    if (name == nullptr) return nullptr;
  return PyModule_Create(&g_module);
}
