// The compute calls of binding.py as a CPython extension: tensors become pointers, sizes and strides here instead of in ctypes
// structures.  The smallest calls of this library are shorter than what the interpreter needed to make them (a
// decode step of one short sequence 4.6 us on the GPU, 9.3 through ctypes structures, of which 3.0 to ask torch for its stream object).
//
// A tensor is whatever has torch's methods (data_ptr, stride, shape, is_contiguous, numel, element_size, and for the calls over a cache of any format
// dtype): nothing of torch is compiled in, nothing is kept from one call to the next, and what the assertions of the ctypes form refused is refused here in its order.
// The functions return the status of the C entry point; binding.py turns it into an exception.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>

#include "../../include/s2attn.h"

namespace {

// Entry points, in the order bind() is given their addresses (_MARSHALLED in binding.py, which compares it with `entry_points`): those of
// the library that ctypes has loaded, so that there is one copy of it in the process.
#define S2_ENTRY_POINTS(X) \
  X(s2_attn_fwd, fwd) X(s2_attn_fwd_rows, fwd_rows) X(s2_attn_fwd_varlen, fwd_varlen) X(s2_attn_bwd_stages, bwd_stages) \
  X(s2_attn_bwd_varlen, bwd_varlen) X(s2_dense_causal_fwd, dense_fwd) X(s2_dense_causal_bwd, dense_bwd) X(s2_attn_decode, decode) \
  X(s2_attn_decode_static, decode_static) X(s2_attn_decode_layout, decode_layout) X(s2_attn_decode_paged, decode_paged) \
  X(s2_attn_decode_paged_layout, decode_paged_layout)
struct Api {
#define X(entry, name) decltype(&entry) name;
  S2_ENTRY_POINTS(X)
#undef X
};
union {
  Api f;
  void* at[sizeof(Api) / sizeof(void*)];
} api;
constexpr Py_ssize_t kEntryPoints = sizeof(Api) / sizeof(void*);

// The entry points of the cache in several formats, in the order bind_cache() is given their addresses (_CACHE_CALLS in binding.py).
#define S2_CACHE_ENTRY_POINTS(X) \
  X(s2_kv_append_paged, append) X(s2_kv_read_paged, read) X(s2_attn_decode_paged_cache, decode) X(s2_attn_decode_paged_cache_layout, decode_layout) \
  X(s2_attn_tree_paged, tree) X(s2_attn_tree_paged_layout, tree_layout)
struct CacheApi {
#define X(entry, name) decltype(&entry) name;
  S2_CACHE_ENTRY_POINTS(X)
#undef X
};
union {
  CacheApi f;
  void* at[sizeof(CacheApi) / sizeof(void*)];
} cache_api;
constexpr Py_ssize_t kCacheEntryPoints = sizeof(CacheApi) / sizeof(void*);

// The entry points of what surrounds attention in a step, in the order bind_step() is given their addresses (_STEP_CALLS in binding.py).
#define S2_STEP_ENTRY_POINTS(X) \
  X(s2_attn_chunk_paged, chunk) X(s2_attn_chunk_paged_layout, chunk_layout) X(s2_kv_plan_paged, plan) X(s2_kv_plan_paged_layout, plan_layout) \
  X(s2_qk_norm_rope_fwd, rope_fwd) X(s2_qk_norm_rope_bwd, rope_bwd)
struct StepApi {
#define X(entry, name) decltype(&entry) name;
  S2_STEP_ENTRY_POINTS(X)
#undef X
};
union {
  StepApi f;
  void* at[sizeof(StepApi) / sizeof(void*)];
} step_api;
constexpr Py_ssize_t kStepEntryPoints = sizeof(StepApi) / sizeof(void*);

struct Names {
  PyObject *data_ptr, *stride, *shape, *is_contiguous, *numel, *element_size, *value, *dtype;
} names;
// torch's objects for the types of elements, for as long as the process lives (set by bind_cache() and bind_step())
struct Types {
  PyObject *bf16, *i32, *f32;
} types;

// An owned reference.
struct Ref {
  PyObject* o;
  explicit Ref(PyObject* x) : o(x) {}
  ~Ref() { Py_XDECREF(o); }
  Ref(const Ref&) = delete;
  Ref& operator=(const Ref&) = delete;
};

// All of these return false with an exception set.
bool fail_assert() {
  PyErr_SetNone(PyExc_AssertionError);
  return false;
}
bool as_i64(PyObject* o, int64_t& out) {
  out = PyLong_AsLongLong(o);
  return out != -1 || !PyErr_Occurred();
}
// as a C int argument of ctypes: an integer, its low 32 bits
bool as_i32(PyObject* o, int32_t& out) {
  const Ref i(PyNumber_Index(o));
  if (!i.o) return false;
  out = (int32_t)(uint32_t)PyLong_AsUnsignedLongMask(i.o);
  return !PyErr_Occurred();
}
bool as_float(PyObject* o, float& out) {
  const double x = PyFloat_AsDouble(o);
  out = (float)x;
  return x != -1.0 || !PyErr_Occurred();
}
// a handle or stream: an integer, a ctypes pointer (its `value`) or None
bool as_address(PyObject* o, void*& out) {
  out = nullptr;
  if (o == Py_None) return true;
  if (PyLong_Check(o)) {
    out = PyLong_AsVoidPtr(o);
    return out || !PyErr_Occurred();
  }
  const Ref v(PyObject_GetAttr(o, names.value));
  if (!v.o) return false;
  if (v.o == Py_None) return true;
  out = PyLong_AsVoidPtr(v.o);
  return out || !PyErr_Occurred();
}
template <class T>
bool data_of(PyObject* t, T*& out) {
  out = nullptr;
  if (t == Py_None) return true;
  const Ref p(PyObject_CallMethodNoArgs(t, names.data_ptr));
  if (!p.o) return false;
  out = static_cast<T*>(PyLong_AsVoidPtr(p.o));
  return out || !PyErr_Occurred();
}
bool contiguous(PyObject* t) {
  const Ref c(PyObject_CallMethodNoArgs(t, names.is_contiguous));
  if (!c.o) return false;
  const int yes = PyObject_IsTrue(c.o);
  return yes < 0 ? false : yes ? true : fail_assert();
}
PyObject* strides_of(PyObject* t) {
  PyObject* s = PyObject_CallMethodNoArgs(t, names.stride);
  if (s && !PyTuple_Check(s)) {
    Py_DECREF(s);
    PyErr_SetString(PyExc_TypeError, "stride() gives a tuple");
    return nullptr;
  }
  return s;
}
// the shape, which has to be of `n` sizes (any number: n < 0)
bool sizes_of(PyObject* t, int n, int64_t* out, Py_ssize_t at_least = 0) {
  const Ref s(PyObject_GetAttr(t, names.shape));
  if (!s.o) return false;
  if (!PyTuple_Check(s.o)) {
    PyErr_SetString(PyExc_TypeError, "shape is a tuple");
    return false;
  }
  const Py_ssize_t have = PyTuple_GET_SIZE(s.o);
  if (n >= 0 && have != n) {
    PyErr_Format(PyExc_ValueError, "expected %d sizes, got %zd", n, have);
    return false;
  }
  if (have < at_least) {
    PyErr_SetString(PyExc_IndexError, "tuple index out of range");
    return false;
  }
  for (Py_ssize_t i = 0; i < (n >= 0 ? n : at_least); ++i)
    if (!as_i64(PyTuple_GET_ITEM(s.o, i), out[i])) return false;
  return true;
}
// stride i of a tuple of strides
bool stride_at(PyObject* strides, int i, int64_t& out) {
  if (i >= PyTuple_GET_SIZE(strides)) {
    PyErr_SetString(PyExc_IndexError, "Dimension out of range");
    return false;
  }
  return as_i64(PyTuple_GET_ITEM(strides, i), out);
}
bool unit_stride(PyObject* strides, int i) {
  int64_t s;
  return stride_at(strides, i, s) && (s == 1 || fail_assert());
}
bool same(PyObject* a, PyObject* b) {
  const int eq = PyObject_RichCompareBool(a, b, Py_EQ);
  return eq < 0 ? false : eq ? true : fail_assert();
}

// q, k, v, o, lse and (n == 9) d_o, dq, dk, dv
bool tensors_of(PyObject* const* a, int n, s2_tensors& t) {
  int64_t size[4];
  if (!sizes_of(a[0], 4, size)) return false;
  const Ref qs(strides_of(a[0])), ks(qs.o ? strides_of(a[1]) : nullptr), vs(ks.o ? strides_of(a[2]) : nullptr), os(vs.o ? strides_of(a[3]) : nullptr);
  if (!os.o) return false;
  if (!unit_stride(qs.o, 3) || !unit_stride(ks.o, 3) || !unit_stride(vs.o, 3) || !unit_stride(os.o, 3)) return false;
  if (!same(ks.o, vs.o) || !same(qs.o, os.o)) return false;
  for (int i = 5; i < n; ++i) {
    if (a[i] == Py_None) continue;
    const Ref gs(strides_of(a[i]));
    if (!gs.o || !same(gs.o, i < 7 ? qs.o : ks.o)) return false;
  }
  if (!contiguous(a[4])) return false;
  if (!data_of(a[0], t.q) || !data_of(a[1], t.k) || !data_of(a[2], t.v) || !data_of(a[3], t.o) || !data_of(a[4], t.lse)) return false;
  t.d_o = t.dq = t.dk = t.dv = nullptr;
  if (n == 9 && (!data_of(a[5], t.d_o) || !data_of(a[6], t.dq) || !data_of(a[7], t.dk) || !data_of(a[8], t.dv))) return false;
  t.batch = (int32_t)size[0];
  t.heads = (int32_t)size[1];
  t.seqlen = (int32_t)size[2];
  t.head_dim = (int32_t)size[3];
  return stride_at(qs.o, 0, t.q_stride_b) && stride_at(qs.o, 1, t.q_stride_h) && stride_at(qs.o, 2, t.q_stride_t) &&
         stride_at(ks.o, 0, t.kv_stride_b) && stride_at(ks.o, 1, t.kv_stride_h) && stride_at(ks.o, 2, t.kv_stride_t);
}

bool workspace_of(PyObject* ws, void*& at, size_t& bytes) {
  if (!data_of(ws, at)) return false;
  const Ref n(PyObject_CallMethodNoArgs(ws, names.numel)), e(n.o ? PyObject_CallMethodNoArgs(ws, names.element_size) : nullptr);
  int64_t count, size;
  if (!e.o || !as_i64(n.o, count) || !as_i64(e.o, size)) return false;
  bytes = (size_t)count * (size_t)size;
  return true;
}

// the row offsets of a packed batch: contiguous, n + 1 of them
bool offsets_of(PyObject* cu, PyObject* q, const int32_t*& at, int32_t& num_seqs) {
  int64_t batch;
  if (!sizes_of(q, -1, &batch, 1)) return false;
  if (batch != 1) return fail_assert();
  if (!contiguous(cu)) return false;
  const Ref n(PyObject_CallMethodNoArgs(cu, names.numel));
  int64_t count;
  if (!n.o || !as_i64(n.o, count)) return false;
  if (count < 2) return fail_assert();
  num_seqs = (int32_t)(count - 1);
  return data_of(cu, at);
}

bool count_is(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  return false;
}

// The call itself, with the interpreter's lock given up (a full queue makes a launch wait).
template <class F>
PyObject* status_of(F&& call) {
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// ------------------------------------------------------------------------------------ calls
// (each: the arguments of the function of the same name in binding.py, the handle or parameters and the stream as addresses)

PyObject* fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {  // layout, q k v o lse, scale, stream
  s2_tensors t;
  float scale;
  void *layout, *stream;
  if (!count_is(n, 8) || !tensors_of(a + 1, 5, t) || !as_address(a[0], layout) || !as_float(a[6], scale) || !as_address(a[7], stream)) return nullptr;
  return status_of([&] { return api.f.fwd(static_cast<s2_layout*>(layout), &t, scale, stream); });
}

PyObject* fwd_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {  // layout, q k v o lse, q_row_start, scale, stream
  s2_tensors t;
  float scale;
  void *layout, *stream;
  int32_t row0;
  int64_t ksize[3];
  if (!count_is(n, 9) || !tensors_of(a + 1, 5, t) || !sizes_of(a[2], -1, ksize, 3) || !as_address(a[0], layout) || !as_i32(a[6], row0) ||
      !as_float(a[7], scale) || !as_address(a[8], stream))
    return nullptr;
  const int32_t rows = t.seqlen;
  t.seqlen = (int32_t)ksize[2];
  return status_of([&] { return api.f.fwd_rows(static_cast<s2_layout*>(layout), &t, row0, rows, scale, stream); });
}

PyObject* fwd_varlen(PyObject*, PyObject* const* a, Py_ssize_t n) {  // layout, q k v o lse, cu_seqlens, max_seqlen, scale, stream
  s2_tensors t;
  float scale;
  void *layout, *stream;
  const int32_t* cu;
  int32_t seqs, longest;
  if (!count_is(n, 10) || !tensors_of(a + 1, 5, t) || !offsets_of(a[6], a[1], cu, seqs) || !as_address(a[0], layout) || !as_i32(a[7], longest) ||
      !as_float(a[8], scale) || !as_address(a[9], stream))
    return nullptr;
  return status_of([&] { return api.f.fwd_varlen(static_cast<s2_layout*>(layout), &t, cu, seqs, longest, scale, stream); });
}

PyObject* bwd_stages(PyObject*, PyObject* const* a, Py_ssize_t n) {  // layout, nine tensors, scale, workspace, stages, stream
  s2_tensors t;
  float scale;
  void *layout, *stream, *ws;
  size_t bytes;
  int32_t stages;
  if (!count_is(n, 14) || !tensors_of(a + 1, 9, t) || !as_address(a[0], layout) || !as_float(a[10], scale) || !workspace_of(a[11], ws, bytes) ||
      !as_i32(a[12], stages) || !as_address(a[13], stream))
    return nullptr;
  return status_of([&] { return api.f.bwd_stages(static_cast<s2_layout*>(layout), &t, scale, ws, bytes, stages, stream); });
}

PyObject* bwd_varlen(PyObject*, PyObject* const* a, Py_ssize_t n) {  // layout, nine tensors, cu_seqlens, max_seqlen, scale, workspace, stream
  s2_tensors t;
  float scale;
  void *layout, *stream, *ws;
  size_t bytes;
  const int32_t* cu;
  int32_t seqs, longest;
  if (!count_is(n, 15) || !tensors_of(a + 1, 9, t) || !offsets_of(a[10], a[1], cu, seqs) || !as_address(a[0], layout) || !as_i32(a[11], longest) ||
      !as_float(a[12], scale) || !workspace_of(a[13], ws, bytes) || !as_address(a[14], stream))
    return nullptr;
  return status_of([&] { return api.f.bwd_varlen(static_cast<s2_layout*>(layout), &t, cu, seqs, longest, scale, ws, bytes, stream); });
}

PyObject* dense_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {  // q k v o lse, scale, stream
  s2_tensors t;
  float scale;
  void* stream;
  if (!count_is(n, 7) || !tensors_of(a, 5, t) || !as_float(a[5], scale) || !as_address(a[6], stream)) return nullptr;
  return status_of([&] { return api.f.dense_fwd(&t, scale, stream); });
}

PyObject* dense_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {  // nine tensors, scale, workspace, stream
  s2_tensors t;
  float scale;
  void *stream, *ws;
  size_t bytes;
  if (!count_is(n, 12) || !tensors_of(a, 9, t) || !as_float(a[9], scale) || !workspace_of(a[10], ws, bytes) || !as_address(a[11], stream)) return nullptr;
  return status_of([&] { return api.f.dense_bwd(&t, scale, ws, bytes, stream); });
}

// q, caches, seq_lens, o, lse, max_len, num_splits
bool decode_of(PyObject* const* a, PyObject* max_len, PyObject* splits, s2_decode_args& d) {
  int64_t size[3];
  if (!sizes_of(a[0], 3, size) || !contiguous(a[0]) || !contiguous(a[4])) return false;
  const Ref ks(strides_of(a[1])), vs(ks.o ? strides_of(a[2]) : nullptr);
  if (!vs.o || !same(ks.o, vs.o) || !unit_stride(ks.o, 3)) return false;
  if (!data_of(a[0], d.q) || !data_of(a[1], d.k_cache) || !data_of(a[2], d.v_cache) || !data_of(a[3], d.seq_lens) || !data_of(a[4], d.o) ||
      !data_of(a[5], d.lse))
    return false;
  d.nseq = (int32_t)size[0];
  d.heads = (int32_t)size[1];
  d.head_dim = (int32_t)size[2];
  return as_i32(max_len, d.max_len) && as_i32(splits, d.num_splits) && stride_at(ks.o, 0, d.kv_stride_seq) && stride_at(ks.o, 1, d.kv_stride_head) &&
         stride_at(ks.o, 2, d.kv_stride_tok);
}

// params or layout, q k v seq_lens o lse, scale, workspace, max_len, num_splits, stream
template <bool LAYOUT>
PyObject* decode_workspace(PyObject* const* a, Py_ssize_t n) {
  s2_decode_args d;
  float scale;
  void *pattern, *stream, *ws;
  size_t bytes;
  if (!count_is(n, 12) || !decode_of(a + 1, a[9], a[10], d) || !as_address(a[0], pattern) || !as_float(a[7], scale) || !workspace_of(a[8], ws, bytes) ||
      !as_address(a[11], stream))
    return nullptr;
  return status_of([&] {
    if constexpr (LAYOUT)
      return api.f.decode_layout(static_cast<s2_layout*>(pattern), &d, scale, ws, bytes, stream);
    else
      return api.f.decode(static_cast<s2_layout_params*>(pattern), &d, scale, ws, bytes, stream);
  });
}
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) { return decode_workspace<false>(a, n); }
PyObject* decode_layout(PyObject*, PyObject* const* a, Py_ssize_t n) { return decode_workspace<true>(a, n); }

PyObject* decode_static(PyObject*, PyObject* const* a, Py_ssize_t n) {  // params, q k v seq_lens o lse, scale, max_len, num_splits, stream
  s2_decode_args d;
  float scale;
  void *params, *stream;
  if (!count_is(n, 11) || !decode_of(a + 1, a[8], a[9], d) || !as_address(a[0], params) || !as_float(a[7], scale) || !as_address(a[10], stream)) return nullptr;
  return status_of([&] { return api.f.decode_static(static_cast<s2_layout_params*>(params), &d, scale, stream); });
}

// params or layout, q k v block_table seq_lens o lse, scale, workspace, missing, num_splits, stream
template <bool LAYOUT>
PyObject* paged(PyObject* const* a, Py_ssize_t n) {
  s2_paged_decode_args d;
  float scale;
  void *pattern, *stream, *ws;
  size_t bytes;
  int64_t size[3], table[3], pages;
  if (!count_is(n, 13) || !sizes_of(a[1], 3, size) || !contiguous(a[1]) || !contiguous(a[6]) || !contiguous(a[4])) return nullptr;
  const Ref ks(strides_of(a[2])), vs(ks.o ? strides_of(a[3]) : nullptr);
  if (!vs.o || !same(ks.o, vs.o) || !unit_stride(ks.o, 2)) return nullptr;
  if (!sizes_of(a[4], -1, table, 2)) {
    // (a table of fewer than two sizes is not [nseq, heads, ...])
    if (PyErr_ExceptionMatches(PyExc_IndexError)) PyErr_SetNone(PyExc_AssertionError);
    return nullptr;
  }
  if (table[0] != size[0] || table[1] != size[1]) {
    fail_assert();
    return nullptr;
  }
  if (!sizes_of(a[4], -1, table, 3) || !sizes_of(a[2], -1, &pages, 1)) return nullptr;
  if (!data_of(a[1], d.q) || !data_of(a[2], d.k_pages) || !data_of(a[3], d.v_pages) || !data_of(a[4], d.block_table) || !data_of(a[5], d.seq_lens) ||
      !data_of(a[6], d.o) || !data_of(a[7], d.lse) || !data_of(a[10], d.missing))
    return nullptr;
  d.nseq = (int32_t)size[0];
  d.heads = (int32_t)size[1];
  d.head_dim = (int32_t)size[2];
  d.max_blocks = (int32_t)table[2];
  d.num_pages = (int32_t)pages;
  if (!as_i32(a[11], d.num_splits) || !stride_at(ks.o, 0, d.page_stride) || !stride_at(ks.o, 1, d.tok_stride)) return nullptr;
  if (!as_address(a[0], pattern) || !as_float(a[8], scale) || !workspace_of(a[9], ws, bytes) || !as_address(a[12], stream)) return nullptr;
  return status_of([&] {
    if constexpr (LAYOUT)
      return api.f.decode_paged_layout(static_cast<s2_layout*>(pattern), &d, scale, ws, bytes, stream);
    else
      return api.f.decode_paged(static_cast<s2_layout_params*>(pattern), &d, scale, ws, bytes, stream);
  });
}
PyObject* decode_paged(PyObject*, PyObject* const* a, Py_ssize_t n) { return paged<false>(a, n); }
PyObject* decode_paged_layout(PyObject*, PyObject* const* a, Py_ssize_t n) { return paged<true>(a, n); }

// ------------------------------------------------------------------------------------ a cache of any format

// an integer of 32 bits; any other is no limit, format or number of splits
bool as_int(PyObject* o, int32_t& out) {
  const Ref i(PyNumber_Index(o));
  int64_t x;
  if (!i.o || !as_i64(i.o, x)) return false;
  out = (int32_t)x;
  if (out == x) return true;
  PyErr_Format(PyExc_OverflowError, "%lld does not fit 32 bits", (long long)x);
  return false;
}
// a tensor whose elements are of this type, or (nullptr) of any of one byte
bool is_of(PyObject* t, PyObject* type) {
  if (type) {
    const Ref have(PyObject_GetAttr(t, names.dtype));
    return have.o && (have.o == type || fail_assert());
  }
  const Ref e(PyObject_CallMethodNoArgs(t, names.element_size));
  int64_t have;
  return e.o && as_i64(e.o, have) && (have == 1 || fail_assert());
}
// the same, of n sizes
bool sizes_and_type(PyObject* t, int n, PyObject* type, int64_t* out) { return sizes_of(t, n, out) && is_of(t, type); }
// elements side by side, `count` of them (any number: count < 0)
template <class T>
bool row_of(PyObject* t, PyObject* type, int64_t count, T*& at) {
  const Ref n(PyObject_CallMethodNoArgs(t, names.numel));
  int64_t have;
  if (!n.o || !as_i64(n.o, have) || !is_of(t, type)) return false;
  if (count >= 0 && have != count) return fail_assert();
  return contiguous(t) && data_of(t, at);
}
bool ints_of(PyObject* t, int64_t count, const int32_t*& at) { return row_of(t, types.i32, count, at); }
bool counter_of(PyObject* t, int32_t*& at) {
  at = nullptr;
  return t == Py_None || row_of(t, types.i32, 1, at);
}

// the strides of two tensors of the same n sizes, which are the same, features side by side; of a size of 1 any is (it is given as 0)
bool strides_of_both(PyObject* a, PyObject* b, int n, const int64_t* size, int64_t* stride) {
  const Ref as(strides_of(a)), bs(as.o ? strides_of(b) : nullptr);
  if (!bs.o || !unit_stride(as.o, n - 1) || !unit_stride(bs.o, n - 1)) return false;
  for (int i = 0; i < n - 1; ++i) {
    int64_t other;
    if (!stride_at(as.o, i, stride[i]) || !stride_at(bs.o, i, other)) return false;
    if (size[i] == 1) stride[i] = 0;
    else if (stride[i] != other) return fail_assert();
  }
  return true;
}

// format, block_size, k_pages, v_pages, block_table, k_scales, v_scales -> the bytes of an s2_paged_cache
PyObject* paged_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  s2_paged_cache c{};
  if (!count_is(n, 7) || !as_int(a[0], c.format) || !as_int(a[1], c.block_size)) return nullptr;
  const bool scaled = c.format != S2_KV_BF16;
  int64_t k[3], v[3], table[3];
  PyObject* const type = scaled ? nullptr : types.bf16;
  if (!sizes_and_type(a[2], 3, type, k) || !sizes_and_type(a[3], 3, type, v) || !sizes_and_type(a[4], 3, types.i32, table)) return nullptr;
  int64_t stride[2];
  if (!strides_of_both(a[2], a[3], 3, k, stride) || !contiguous(a[4])) return nullptr;
  const int64_t D = c.format == S2_KV_MXFP4 ? 2 * k[2] : k[2];
  if (k[0] != v[0] || k[1] != v[1] || k[2] != v[2] || k[1] != c.block_size || k[0] > INT32_MAX || table[0] > INT32_MAX || table[1] > INT32_MAX ||
      table[2] > INT32_MAX || D > INT32_MAX) {
    fail_assert();
    return nullptr;
  }
  c.page_stride = stride[0];
  c.tok_stride = stride[1];
  if (scaled) {
    int64_t sk[3], sv[3];
    if (!sizes_and_type(a[5], 3, nullptr, sk) || !sizes_and_type(a[6], 3, nullptr, sv)) return nullptr;
    for (int i = 0; i < 3; ++i)
      if (sk[i] != sv[i] || sk[i] != (i < 2 ? k[i] : D / 32)) {
        fail_assert();
        return nullptr;
      }
    if (!strides_of_both(a[5], a[6], 3, sk, stride) || !data_of(a[5], c.k_scales) || !data_of(a[6], c.v_scales)) return nullptr;
    c.scale_page_stride = stride[0];
    c.scale_tok_stride = stride[1];
  } else if (a[5] != Py_None || a[6] != Py_None) {
    fail_assert();
    return nullptr;
  }
  if (!data_of(a[2], c.k_pages) || !data_of(a[3], c.v_pages) || !data_of(a[4], c.block_table)) return nullptr;
  c.nseq = (int32_t)table[0];
  c.heads = (int32_t)table[1];
  c.head_dim = (int32_t)D;
  c.max_blocks = (int32_t)table[2];
  c.num_pages = (int32_t)k[0];
  return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&c), sizeof c);
}
bool cache_of(PyObject* o, s2_paged_cache& c) {
  if (!PyBytes_Check(o) || PyBytes_GET_SIZE(o) != (Py_ssize_t)sizeof c) {
    PyErr_SetString(PyExc_TypeError, "expected a paged cache");
    return false;
  }
  __builtin_memcpy(&c, PyBytes_AS_STRING(o), sizeof c);
  return true;
}

// two bf16 tensors of the same strides, of `n` sizes, the last of them features side by side; their sizes and strides
bool pair_of(PyObject* a, PyObject* b, int n, int64_t* size, int64_t* stride) {
  int64_t other[4];
  if (!sizes_and_type(a, n, types.bf16, size) || !sizes_and_type(b, n, types.bf16, other)) return false;
  for (int i = 0; i < n; ++i)
    if (size[i] != other[i]) return fail_assert();
  return strides_of_both(a, b, n, size, stride);
}

PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {  // cache, k v cu_new start, max_new, rows, skipped, stream
  s2_paged_cache c;
  s2_kv_append_args d{};
  void* stream;
  int64_t size[3], stride[2];
  if (!count_is(n, 9) || !cache_of(a[0], c) || !pair_of(a[1], a[2], 3, size, stride)) return nullptr;
  if (size[1] != c.heads || size[2] != c.head_dim || size[0] > INT32_MAX) {
    fail_assert();
    return nullptr;
  }
  if (!ints_of(a[3], (int64_t)c.nseq + 1, d.cu_new) || !ints_of(a[4], c.nseq, d.start) || !as_int(a[5], d.max_new) || !counter_of(a[7], d.skipped)) return nullptr;
  if (a[6] != Py_None) {
    const Ref count(PyObject_CallMethodNoArgs(a[6], names.numel));
    int64_t items;
    if (!count.o || !as_i64(count.o, items) || !ints_of(a[6], -1, d.rows)) return nullptr;
    // (no rows at all: an empty tensor has no address, and is not "as they come")
    if (items == 0 || items > INT32_MAX) {
      fail_assert();
      return nullptr;
    }
    d.num_items = (int32_t)items;
  }
  if (!data_of(a[1], d.k) || !data_of(a[2], d.v) || !as_address(a[8], stream)) return nullptr;
  d.num_rows = (int32_t)size[0];
  d.stride_row = stride[0];
  d.stride_head = stride[1];
  return status_of([&] { return cache_api.f.append(&c, &d, stream); });
}

PyObject* kv_read(PyObject*, PyObject* const* a, Py_ssize_t n) {  // cache, k v (head, row, feature) cu_rows start, max_rows, stream
  s2_paged_cache c;
  s2_kv_read_args d{};
  void* stream;
  int64_t size[3], stride[2];
  if (!count_is(n, 7) || !cache_of(a[0], c) || !pair_of(a[1], a[2], 3, size, stride)) return nullptr;
  if (size[0] != c.heads || size[2] != c.head_dim || size[1] > INT32_MAX) {
    fail_assert();
    return nullptr;
  }
  if (!ints_of(a[3], (int64_t)c.nseq + 1, d.cu_rows) || !ints_of(a[4], c.nseq, d.start) || !as_int(a[5], d.max_rows) || !data_of(a[1], d.k) ||
      !data_of(a[2], d.v) || !as_address(a[6], stream))
    return nullptr;
  d.num_rows = (int32_t)size[1];
  d.stride_head = stride[0];
  d.stride_row = stride[1];
  return status_of([&] { return cache_api.f.read(&c, &d, stream); });
}

// fp32 [nseq, heads, ...] side by side, `count` of them, or None
bool lse_of(PyObject* t, int64_t count, float*& at) {
  at = nullptr;
  return t == Py_None || row_of(t, types.f32, count, at);
}

// params or layout, cache, q seq_lens o lse, scale, workspace, missing, num_splits, stream
template <bool LAYOUT>
PyObject* over_cache(PyObject* const* a, Py_ssize_t n) {
  s2_paged_cache c;
  s2_cache_decode_args d{};
  float scale;
  void *pattern, *stream, *ws;
  size_t bytes;
  int64_t size[3], stride[2];
  if (!count_is(n, 11) || !cache_of(a[1], c) || !pair_of(a[2], a[4], 3, size, stride)) return nullptr;
  if (size[0] != c.nseq || size[1] != c.heads || size[2] != c.head_dim) {
    fail_assert();
    return nullptr;
  }
  if (!ints_of(a[3], c.nseq, d.seq_lens) || !lse_of(a[5], (int64_t)c.nseq * c.heads, d.lse) || !counter_of(a[8], d.missing) || !data_of(a[2], d.q) ||
      !data_of(a[4], d.o) || !as_int(a[9], d.num_splits) || !as_address(a[0], pattern) || !as_float(a[6], scale) || !workspace_of(a[7], ws, bytes) ||
      !as_address(a[10], stream))
    return nullptr;
  d.q_stride_seq = stride[0];
  d.q_stride_head = stride[1];
  return status_of([&] {
    if constexpr (LAYOUT)
      return cache_api.f.decode_layout(static_cast<s2_layout*>(pattern), &c, &d, scale, ws, bytes, stream);
    else
      return cache_api.f.decode(static_cast<s2_layout_params*>(pattern), &c, &d, scale, ws, bytes, stream);
  });
}
PyObject* decode_cache(PyObject*, PyObject* const* a, Py_ssize_t n) { return over_cache<false>(a, n); }
PyObject* decode_cache_layout(PyObject*, PyObject* const* a, Py_ssize_t n) { return over_cache<true>(a, n); }

// params or layout, cache, q k v parents seq_lens o lse, scale, workspace, missing, num_splits, stream
template <bool LAYOUT>
PyObject* drafts(PyObject* const* a, Py_ssize_t n) {
  s2_paged_cache c;
  s2_tree_args d{};
  float scale;
  void *pattern, *stream, *ws;
  size_t bytes;
  int64_t size[4], stride[3], kv_size[4], kv_stride[3];
  if (!count_is(n, 14) || !cache_of(a[1], c) || !pair_of(a[2], a[7], 4, size, stride) || !pair_of(a[3], a[4], 4, kv_size, kv_stride)) return nullptr;
  for (int i = 0; i < 4; ++i)
    if (size[i] != kv_size[i]) {
      fail_assert();
      return nullptr;
    }
  if (size[0] != c.nseq || size[1] != c.heads || size[3] != c.head_dim || size[2] > INT32_MAX) {
    fail_assert();
    return nullptr;
  }
  if (!ints_of(a[5], c.nseq * size[2], d.parents) || !ints_of(a[6], c.nseq, d.seq_lens) ||
      !lse_of(a[8], (int64_t)c.nseq * c.heads * size[2], d.lse) || !counter_of(a[11], d.missing) || !data_of(a[2], d.q) || !data_of(a[3], d.k) ||
      !data_of(a[4], d.v) || !data_of(a[7], d.o) || !as_int(a[12], d.num_splits) || !as_address(a[0], pattern) || !as_float(a[9], scale) ||
      !workspace_of(a[10], ws, bytes) || !as_address(a[13], stream))
    return nullptr;
  d.nodes = (int32_t)size[2];
  d.q_stride_seq = stride[0];
  d.q_stride_head = stride[1];
  d.q_stride_node = stride[2];
  d.kv_stride_seq = kv_stride[0];
  d.kv_stride_head = kv_stride[1];
  d.kv_stride_node = kv_stride[2];
  return status_of([&] {
    if constexpr (LAYOUT)
      return cache_api.f.tree_layout(static_cast<s2_layout*>(pattern), &c, &d, scale, ws, bytes, stream);
    else
      return cache_api.f.tree(static_cast<s2_layout_params*>(pattern), &c, &d, scale, ws, bytes, stream);
  });
}
PyObject* tree(PyObject*, PyObject* const* a, Py_ssize_t n) { return drafts<false>(a, n); }
PyObject* tree_layout(PyObject*, PyObject* const* a, Py_ssize_t n) { return drafts<true>(a, n); }

// params or layout, cache, q cu_new start o lse, scale, workspace, max_new, missing, num_splits, stream
template <bool LAYOUT>
PyObject* chunk_call(PyObject* const* a, Py_ssize_t n) {
  s2_paged_cache c;
  s2_chunk_args d{};
  float scale;
  void *pattern, *stream, *ws = nullptr;
  size_t bytes = 0;
  int64_t size[3], stride[2];
  if (!count_is(n, 13) || !cache_of(a[1], c) || !pair_of(a[2], a[5], 3, size, stride)) return nullptr;
  if (size[1] != c.heads || size[2] != c.head_dim || size[0] > INT32_MAX) {
    fail_assert();
    return nullptr;
  }
  if (!ints_of(a[3], (int64_t)c.nseq + 1, d.cu_new) || !ints_of(a[4], c.nseq, d.start) || !lse_of(a[6], (int64_t)c.heads * size[0], d.lse) ||
      !counter_of(a[10], d.missing) || !data_of(a[2], d.q) || !data_of(a[5], d.o) || !as_int(a[9], d.max_new) || !as_int(a[11], d.num_splits) ||
      !as_address(a[0], pattern) || !as_float(a[7], scale) || (a[8] != Py_None && !workspace_of(a[8], ws, bytes)) || !as_address(a[12], stream))
    return nullptr;
  d.num_rows = (int32_t)size[0];
  d.q_stride_row = stride[0];
  d.q_stride_head = stride[1];
  return status_of([&] {
    if constexpr (LAYOUT)
      return step_api.f.chunk_layout(static_cast<s2_layout*>(pattern), &c, &d, scale, ws, bytes, stream);
    else
      return step_api.f.chunk(static_cast<s2_layout_params*>(pattern), &c, &d, scale, ws, bytes, stream);
  });
}
PyObject* chunk(PyObject*, PyObject* const* a, Py_ssize_t n) { return chunk_call<false>(a, n); }
PyObject* chunk_layout(PyObject*, PyObject* const* a, Py_ssize_t n) { return chunk_call<true>(a, n); }

// int32, side by side, `count` of them, or None
bool ints_or_none(PyObject* t, int64_t count, const int32_t*& at) {
  at = nullptr;
  return t == Py_None || ints_of(t, count, at);
}
bool out_ints(PyObject* t, int64_t count, int32_t*& at) { return row_of(t, types.i32, count, at); }
bool out_ints_or_none(PyObject* t, int64_t count, int32_t*& at) {
  at = nullptr;
  return t == Py_None || out_ints(t, count, at);
}

// params or layout, block_table lens new_lens free_pages free_state new_table new_free_pages new_free_state, workspace, cu_new positions seq_lens query_from short_of,
// stream
template <bool LAYOUT>
PyObject* plan_call(PyObject* const* a, Py_ssize_t n) {
  s2_kv_plan_args d{};
  void *pattern, *stream, *ws;
  size_t bytes;
  int64_t table[3], other[3], pages[1], rows = 0;
  if (!count_is(n, 16) || !sizes_and_type(a[1], 3, types.i32, table) || !sizes_and_type(a[6], 3, types.i32, other) || !sizes_and_type(a[4], 1, types.i32, pages))
    return nullptr;
  for (int i = 0; i < 3; ++i)
    if (table[i] != other[i] || table[i] > INT32_MAX) {
      fail_assert();
      return nullptr;
    }
  if (pages[0] > INT32_MAX) {
    fail_assert();
    return nullptr;
  }
  if (a[11] != Py_None) {
    const Ref count(PyObject_CallMethodNoArgs(a[11], names.numel));
    if (!count.o || !as_i64(count.o, rows)) return nullptr;
    if (rows > INT32_MAX) {
      fail_assert();
      return nullptr;
    }
  }
  // (sizes and types of the tables and of the ring are known)
  if (!contiguous(a[1]) || !data_of(a[1], d.block_table) || !contiguous(a[4]) || !data_of(a[4], d.free_pages) || !contiguous(a[6]) || !data_of(a[6], d.new_table) ||
      !ints_of(a[2], table[0], d.lens) || !ints_of(a[3], table[0], d.new_lens) ||
      !ints_of(a[5], 2, d.free_state) ||
      !out_ints(a[7], pages[0], d.new_free_pages) || !out_ints(a[8], 2, d.new_free_state) || !workspace_of(a[9], ws, bytes) ||
      !out_ints_or_none(a[10], table[0] + 1, d.cu_new) || !out_ints_or_none(a[11], rows, d.positions) || !out_ints_or_none(a[12], table[0], d.seq_lens) ||
      !ints_or_none(a[13], table[0], d.query_from) || !counter_of(a[14], d.short_of) || !as_address(a[0], pattern) || !as_address(a[15], stream))
    return nullptr;
  d.nseq = (int32_t)table[0];
  d.heads = (int32_t)table[1];
  d.max_blocks = (int32_t)table[2];
  d.num_pages = (int32_t)pages[0];
  d.num_rows = (int32_t)rows;
  return status_of([&] {
    if constexpr (LAYOUT)
      return step_api.f.plan_layout(static_cast<s2_layout*>(pattern), &d, ws, bytes, stream);
    else
      return step_api.f.plan(static_cast<s2_layout_params*>(pattern), &d, ws, bytes, stream);
  });
}
PyObject* plan(PyObject*, PyObject* const* a, Py_ssize_t n) { return plan_call<false>(a, n); }
PyObject* plan_layout(PyObject*, PyObject* const* a, Py_ssize_t n) { return plan_call<true>(a, n); }

// Tensors [batch, heads, seqlen, head_dim] of one call that have the same sizes, and in a family (q and k as they go in, or as they come out) the same strides; None
// where there is none.
struct Family {
  bool any = false;
  int64_t stride[3] = {0, 0, 0};  // (of a size of 1: 0)
};
alignas(16) char nothing[16];  // where a tensor without elements lies (which has no address of its own): nothing is read or written there
bool member_of(PyObject* t, Family& f, int64_t* size, bool& sized, void*& at) {
  at = nullptr;
  if (t == Py_None) return true;
  int64_t mine[4], stride[3];
  if (!sizes_and_type(t, 4, types.bf16, mine)) return false;
  for (int i = 0; i < 4; ++i) {
    if ((sized && mine[i] != size[i]) || mine[i] > INT32_MAX) return fail_assert();
    size[i] = mine[i];
  }
  sized = true;
  const Ref strides(strides_of(t));
  if (!strides.o || !unit_stride(strides.o, 3)) return false;
  for (int i = 0; i < 3; ++i) {
    if (!stride_at(strides.o, i, stride[i])) return false;
    if (mine[i] == 1) stride[i] = 0;
    if (f.any && f.stride[i] != stride[i]) return fail_assert();
    f.stride[i] = stride[i];
  }
  f.any = true;
  if (!data_of(t, at)) return false;
  if (!at && mine[0] * mine[2] == 0) at = nothing;
  return true;
}
bool weight_of(PyObject* t, int64_t count, float*& at) {
  at = nullptr;
  return t == Py_None || row_of(t, types.f32, count, at);
}

// q k, (backward: d_q_out d_k_out dq dk, else q_out k_out), q_weight k_weight, (backward: dq_weight dk_weight), inv_freq, eps, (backward: workspace), positions,
// interleaved, stream
template <bool BWD>
PyObject* rope_call(PyObject* const* a, Py_ssize_t n) {
  s2_qk_norm_rope_args d{};
  constexpr int W = BWD ? 6 : 4, F = BWD ? 10 : 6, P = BWD ? 13 : 8;
  if (!count_is(n, P + 3)) return nullptr;
  Family in, out;
  int64_t size[4] = {0, 0, 0, 0};
  bool sized = false;
  void *q, *k, *to[4] = {nullptr, nullptr, nullptr, nullptr}, *ws = nullptr, *stream;
  size_t bytes = 0;
  if (!member_of(a[0], in, size, sized, q) || !member_of(a[1], in, size, sized, k)) return nullptr;
  for (int i = 2; i < W; ++i)
    if (!member_of(a[i], BWD && i >= 4 ? in : out, size, sized, to[i - 2])) return nullptr;
  float *weight[2], *d_weight[2] = {nullptr, nullptr};
  for (int i = 0; i < 2; ++i)
    if (!weight_of(a[W + i], size[3], weight[i]) || (BWD && !weight_of(a[W + 2 + i], size[3], d_weight[i]))) return nullptr;
  float* freq = nullptr;
  int64_t pairs = 0;
  if (a[F] != Py_None) {
    const Ref count(PyObject_CallMethodNoArgs(a[F], names.numel));
    if (!count.o || !as_i64(count.o, pairs) || !row_of(a[F], types.f32, pairs, freq)) return nullptr;
    if (pairs > INT32_MAX / 2) {
      fail_assert();
      return nullptr;
    }
  }
  const int at_eps = F + 1;
  if (!as_float(a[at_eps], d.eps) || (BWD && a[at_eps + 1] != Py_None && !workspace_of(a[at_eps + 1], ws, bytes))) return nullptr;
  if (!ints_or_none(a[P], size[0] * size[2], d.positions)) return nullptr;
  const int interleaved = PyObject_IsTrue(a[P + 1]);
  if (interleaved < 0 || !as_address(a[P + 2], stream)) return nullptr;
  d.q = q;
  d.k = k;
  if (BWD) {
    d.d_q_out = to[0];
    d.d_k_out = to[1];
    d.dq = to[2];
    d.dk = to[3];
  } else {
    d.q_out = to[0];
    d.k_out = to[1];
  }
  d.q_weight = weight[0];
  d.k_weight = weight[1];
  d.dq_weight = d_weight[0];
  d.dk_weight = d_weight[1];
  d.inv_freq = freq;
  d.batch = (int32_t)size[0];
  d.heads = (int32_t)size[1];
  d.seqlen = (int32_t)size[2];
  d.head_dim = (int32_t)size[3];
  d.rotary_dim = (int32_t)(2 * pairs);
  d.interleaved = interleaved;
  d.in_stride_b = in.stride[0];
  d.in_stride_h = in.stride[1];
  d.in_stride_t = in.stride[2];
  d.out_stride_b = out.stride[0];
  d.out_stride_h = out.stride[1];
  d.out_stride_t = out.stride[2];
  return status_of([&] {
    if constexpr (BWD)
      return step_api.f.rope_bwd(&d, ws, bytes, stream);
    else
      return step_api.f.rope_fwd(&d, stream);
  });
}
PyObject* rope_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) { return rope_call<false>(a, n); }
PyObject* rope_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) { return rope_call<true>(a, n); }

PyObject* bind_to(void** to, Py_ssize_t count, PyObject* const* a, Py_ssize_t n) {
  if (!count_is(n, count)) return nullptr;
  for (Py_ssize_t i = 0; i < n; ++i)
    if (!PyLong_AsVoidPtr(a[i])) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no address");
      return nullptr;
    }
  for (Py_ssize_t i = 0; i < n; ++i) to[i] = PyLong_AsVoidPtr(a[i]);
  Py_RETURN_NONE;
}
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) { return bind_to(api.at, kEntryPoints, a, n); }
bool find_types() {
  const Ref torch(PyImport_ImportModule("torch"));
  if (!torch.o) return false;
  const struct {
    PyObject** at;
    const char* name;
  } all[] = {{&types.bf16, "bfloat16"}, {&types.i32, "int32"}, {&types.f32, "float32"}};
  for (const auto& t : all)
    if (!*t.at && !(*t.at = PyObject_GetAttrString(torch.o, t.name))) return false;
  return true;
}
PyObject* bind_cache(PyObject*, PyObject* const* a, Py_ssize_t n) { return find_types() ? bind_to(cache_api.at, kCacheEntryPoints, a, n) : nullptr; }
PyObject* bind_step(PyObject*, PyObject* const* a, Py_ssize_t n) { return find_types() ? bind_to(step_api.at, kStepEntryPoints, a, n) : nullptr; }

#define S2_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {S2_METHOD(bind),          S2_METHOD(fwd),          S2_METHOD(fwd_rows),      S2_METHOD(fwd_varlen),
                         S2_METHOD(bwd_stages),    S2_METHOD(bwd_varlen),   S2_METHOD(dense_fwd),     S2_METHOD(dense_bwd),
                         S2_METHOD(decode),        S2_METHOD(decode_static), S2_METHOD(decode_layout), S2_METHOD(decode_paged),
                         S2_METHOD(decode_paged_layout), S2_METHOD(bind_cache), S2_METHOD(paged_cache), S2_METHOD(kv_append),
                         S2_METHOD(kv_read),       S2_METHOD(decode_cache), S2_METHOD(decode_cache_layout), S2_METHOD(tree),
                         S2_METHOD(tree_layout),   S2_METHOD(bind_step),    S2_METHOD(chunk),         S2_METHOD(chunk_layout),
                         S2_METHOD(plan),          S2_METHOD(plan_layout),  S2_METHOD(rope_fwd),      S2_METHOD(rope_bwd),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
  struct {
    PyObject** at;
    const char* text;
  } const all[] = {{&names.data_ptr, "data_ptr"}, {&names.stride, "stride"},   {&names.shape, "shape"}, {&names.is_contiguous, "is_contiguous"},
                   {&names.numel, "numel"},       {&names.element_size, "element_size"}, {&names.value, "value"},
                   {&names.dtype, "dtype"}};
  for (const auto& n : all)
    if (!(*n.at = PyUnicode_InternFromString(n.text))) return nullptr;
  const Ref m(PyModule_Create(&module));
  if (!m.o) return nullptr;
#define X(entry, name) #entry,
  const char* const entries[] = {S2_ENTRY_POINTS(X)};
  const char* const cache_entries[] = {S2_CACHE_ENTRY_POINTS(X)};
  const char* const step_entries[] = {S2_STEP_ENTRY_POINTS(X)};
#undef X
  const struct {
    const char* attribute;
    const char* const* entry;
    Py_ssize_t count;
  } orders[] = {{"entry_points", entries, kEntryPoints}, {"cache_entry_points", cache_entries, kCacheEntryPoints}, {"step_entry_points", step_entries, kStepEntryPoints}};
  for (const auto& of : orders) {
    const Ref order(PyTuple_New(of.count));
    if (!order.o) return nullptr;
    for (Py_ssize_t i = 0; i < of.count; ++i) {
      PyObject* const name = PyUnicode_FromString(of.entry[i]);
      if (!name) return nullptr;
      PyTuple_SET_ITEM(order.o, i, name);
    }
    if (PyObject_SetAttrString(m.o, of.attribute, order.o)) return nullptr;
  }
  Py_INCREF(m.o);
  return m.o;
}
