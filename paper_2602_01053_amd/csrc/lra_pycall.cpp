// CPython side of the entry points that a program calls once per layer and token: tensors and descriptors to plain
// pointers, then the C ABI.  A small call lasts as long on the host as on the GPU, and of its 9.63 us there (a decode of two
// launches, issued one after the other) ctypes and the interpreter took 4: thirteen argument conversions, three references,
// seven address look-ups and a struct, each an object of its own.  So it takes 6.86, of which the launches are 4.8.  No arithmetic, no state but the handles that bind()
// leaves; addresses are asked of the tensors at every call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "lra_attn.h"
#include "lra_attn8.h"

namespace {

decltype(&lra_attn_decode) g_decode;
decltype(&lra_attn_prefill) g_prefill;
decltype(&lra_cache_append) g_append;
const lra_tuning* g_tuning;
PyTypeObject *g_shape_type, *g_cache_type;
PyObject *g_get_device, *g_get_stream, *g_is_initialized;  // torch's current device and its stream's handle; whether the GPU is in use
PyObject *s_data_ptr, *s_size, *s_nbytes, *s_cuda_stream, *s_zero, *s_one;

// The address of a tensor's first element (None: no address).
bool address(PyObject* t, void** p) {
  *p = nullptr;
  if (t == Py_None) return true;
  PyObject* v = PyObject_CallMethodNoArgs(t, s_data_ptr);
  if (!v) return false;
  *p = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !(*p == nullptr && PyErr_Occurred());
}

// What a 32-bit field takes from a Python number: int(x), its low bits.
bool int32(PyObject* o, int32_t* x) {
  PyObject* v = PyLong_CheckExact(o) ? Py_NewRef(o) : PyNumber_Long(o);
  if (!v) return false;
  *x = static_cast<int32_t>(PyLong_AsUnsignedLongMask(v));
  Py_DECREF(v);
  return !PyErr_Occurred();
}

bool size(PyObject* t, PyObject* dim, int32_t* x) {
  PyObject* v = PyObject_CallMethodOneArg(t, s_size, dim);
  if (!v) return false;
  const bool ok = int32(v, x);
  Py_DECREF(v);
  return ok;
}

bool workspace(PyObject* t, void** p, size_t* bytes) {
  *p = nullptr;
  *bytes = 0;
  if (t == Py_None) return true;
  if (!address(t, p)) return false;
  PyObject* v = PyObject_GetAttr(t, s_nbytes);
  if (!v) return false;
  *bytes = PyLong_AsSize_t(v);
  Py_DECREF(v);
  return !PyErr_Occurred();
}

// The handle of the given stream, or of the current one (the null stream is NULL either way).
bool stream_handle(PyObject* stream, void** p) {
  PyObject* v;
  if (stream != Py_None) {
    v = PyObject_GetAttr(stream, s_cuda_stream);
  } else {
    // (the GPU not in use yet, or not usable in this process: torch starts it, or says why not)
    PyObject* up = PyObject_CallNoArgs(g_is_initialized);
    if (!up) return false;
    const int yes = PyObject_IsTrue(up);
    Py_DECREF(up);
    if (yes < 0) return false;
    if (!yes) {
      PyObject* cuda = PyImport_ImportModule("torch.cuda");
      PyObject* cur = cuda ? PyObject_CallMethod(cuda, "current_stream", nullptr) : nullptr;
      v = cur ? PyObject_GetAttr(cur, s_cuda_stream) : nullptr;
      Py_XDECREF(cur);
      Py_XDECREF(cuda);
    } else {
      PyObject* dev = PyObject_CallNoArgs(g_get_device);
      v = dev ? PyObject_CallOneArg(g_get_stream, dev) : nullptr;
      Py_XDECREF(dev);
    }
  }
  if (!v) return false;
  *p = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return !(*p == nullptr && PyErr_Occurred());
}

// A ctypes struct's memory, held while the call runs.
struct Struct {
  Py_buffer view{};
  bool held = false;
  bool open(PyObject* o, PyTypeObject* type) {
    if (!PyObject_TypeCheck(o, type)) {
      PyErr_Format(PyExc_TypeError, "expected %s, not %s", type->tp_name, Py_TYPE(o)->tp_name);
      return false;
    }
    held = PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) == 0;
    return held;
  }
  template <typename T> const T* as() const { return static_cast<const T*>(view.buf); }
  ~Struct() {
    if (held) PyBuffer_Release(&view);
  }
};

bool arity(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, not %zd", want, n);
  return false;
}

// decode(shape, cache, b_k, b_v, n_adapters, q, query_adapter, seq_query_start, max_queries_per_seq, out, workspace, stream)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Struct sh, c;
  lra_adapters ad{};
  void *b_k, *b_v, *q, *qa, *sqs, *out, *ws, *st;
  size_t ws_bytes;
  int32_t n_queries, mq;
  if (!arity(n, 12) || !sh.open(a[0], g_shape_type) || !c.open(a[1], g_cache_type) || !address(a[2], &b_k) || !address(a[3], &b_v) ||
      !int32(a[4], &ad.n_adapters) || !workspace(a[10], &ws, &ws_bytes) || !address(a[5], &q) || !address(a[6], &qa) ||
      !address(a[7], &sqs) || !size(a[5], s_zero, &n_queries) || !int32(a[8], &mq) || !address(a[9], &out) || !stream_handle(a[11], &st))
    return nullptr;
  ad.b_k = b_k;
  ad.b_v = b_v;
  lra_status status;
  Py_BEGIN_ALLOW_THREADS
  status = g_decode(sh.as<lra_shape>(), c.as<lra_cache>(), &ad, q, static_cast<const int32_t*>(qa), static_cast<const int32_t*>(sqs),
                    n_queries, mq, out, ws, ws_bytes, g_tuning, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// prefill(shape, cache, b_k, b_v, n_adapters, q, seq_index, adapter_index, out, workspace, stream)
PyObject* prefill(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Struct sh, c;
  lra_adapters ad{};
  void *b_k, *b_v, *q, *out, *ws, *st;
  size_t ws_bytes;
  int32_t n_new, seq, adapter;
  if (!arity(n, 11) || !sh.open(a[0], g_shape_type) || !c.open(a[1], g_cache_type) || !address(a[2], &b_k) || !address(a[3], &b_v) ||
      !int32(a[4], &ad.n_adapters) || !workspace(a[9], &ws, &ws_bytes) || !address(a[5], &q) || !int32(a[6], &seq) || !int32(a[7], &adapter) ||
      !size(a[5], s_zero, &n_new) || !address(a[8], &out) || !stream_handle(a[10], &st))
    return nullptr;
  ad.b_k = b_k;
  ad.b_v = b_v;
  lra_status status;
  Py_BEGIN_ALLOW_THREADS
  status = g_prefill(sh.as<lra_shape>(), c.as<lra_cache>(), &ad, q, seq, adapter, n_new, out, ws, ws_bytes, g_tuning, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// append(shape, cache, w, rope_theta, x, seq_index, workspace, stream); x and w dense, of one width (the caller has checked)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Struct sh, c;
  lra_projection proj{};
  void *w, *x, *ws, *st;
  size_t ws_bytes;
  int32_t n_new, seq;
  if (!arity(n, 8) || !address(a[2], &w) || !size(a[2], s_one, &proj.d_model)) return nullptr;
  const double theta = PyFloat_AsDouble(a[3]);
  if ((theta == -1.0 && PyErr_Occurred()) || !workspace(a[6], &ws, &ws_bytes) || !sh.open(a[0], g_shape_type) ||
      !c.open(a[1], g_cache_type) || !address(a[4], &x) || !int32(a[5], &seq) || !size(a[4], s_zero, &n_new) || !stream_handle(a[7], &st))
    return nullptr;
  proj.w = w;
  proj.rope_theta = static_cast<float>(theta);
  lra_status status;
  Py_BEGIN_ALLOW_THREADS
  status = g_append(sh.as<lra_shape>(), c.as<lra_cache>(), &proj, x, seq, n_new, ws, ws_bytes, g_tuning, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// bind(decode, prefill, append, tuning: addresses; LraShape, LraCache; current device, its raw stream, is_initialized: callables)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 9)) return nullptr;
  void* p[4];
  for (int i = 0; i < 4; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no address");
      return nullptr;
    }
  }
  if (!PyType_Check(a[4]) || !PyType_Check(a[5])) {
    PyErr_SetString(PyExc_TypeError, "expected the two struct types");
    return nullptr;
  }
  g_decode = reinterpret_cast<decltype(g_decode)>(p[0]);
  g_prefill = reinterpret_cast<decltype(g_prefill)>(p[1]);
  g_append = reinterpret_cast<decltype(g_append)>(p[2]);
  g_tuning = static_cast<const lra_tuning*>(p[3]);
  g_shape_type = reinterpret_cast<PyTypeObject*>(Py_NewRef(a[4]));  // (held for good, like the library)
  g_cache_type = reinterpret_cast<PyTypeObject*>(Py_NewRef(a[5]));
  g_get_device = Py_NewRef(a[6]);
  g_get_stream = Py_NewRef(a[7]);
  g_is_initialized = Py_NewRef(a[8]);
  Py_RETURN_NONE;
}

// ---- the 8-bit calls (lra_attn8.h): the tensors' shapes, strides and types are checked here too; -1 is "not as documented", which the
// binding's own checks then put into words.  (A decode step's append and read of 64 caches: 18.8 us by ctypes, of which the GPU worked 12.)
decltype(&lra_quantize_rows) g_quantize;
decltype(&lra_matmul_i8) g_matmul;
decltype(&lra_cache8_append) g_append8;
decltype(&lra_cache8_gather) g_gather8;
decltype(&lra_attn_batch8) g_attend8;
PyTypeObject *g_cache8_type, *g_batch_type;
PyObject* g_dtypes[4];  // bfloat16, float32, int8, int32
PyObject *s_shape, *s_stride, *s_dtype, *s_sizes, *s_n_seqs;
enum { kBf16, kF32, kI8, kI32, kOther };

bool ints(PyObject* tuple, int64_t (&x)[4], int& n) {
  if (!PyTuple_Check(tuple)) {
    PyErr_SetString(PyExc_TypeError, "expected a tuple of sizes");
    return false;
  }
  n = static_cast<int>(PyTuple_GET_SIZE(tuple));
  for (int i = 0; i < n && i < 4; ++i) {
    x[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, i));
    if (x[i] == -1 && PyErr_Occurred()) return false;
  }
  return true;
}

// What a call looks at of a tensor.
struct View {
  void* data = nullptr;
  int64_t size[4], stride[4];
  int dims = 0, type = kOther;
  bool open(PyObject* t) {
    PyObject* v = PyObject_GetAttr(t, s_shape);
    if (!v) return false;
    bool ok = ints(v, size, dims);
    Py_DECREF(v);
    if (!ok || !(v = PyObject_CallMethodNoArgs(t, s_stride))) return false;
    int n;
    ok = ints(v, stride, n);
    Py_DECREF(v);
    if (!ok || !(v = PyObject_GetAttr(t, s_dtype))) return false;
    for (int i = 0; i < kOther; ++i)
      if (v == g_dtypes[i]) type = i;
    Py_DECREF(v);
    return address(t, &data);
  }
  bool matrix(int want, int64_t rows, int64_t cols) const { return dims == 2 && type == want && size[0] == rows && size[1] == cols && (cols <= 1 || stride[1] == 1); }
  bool vector(int want, int64_t n) const { return dims == 1 && type == want && size[0] == n && (n <= 1 || stride[0] == 1); }
  // [n][a][b] with dense rows, tokens at any stride; `dense`: those too
  bool rows(int want, int64_t n, int64_t a, int64_t b, bool dense) const {
    return dims == 3 && type == want && size[0] == n && size[1] == a && size[2] == b && stride[2] == 1 && (a == 1 || stride[1] == b) && (!dense || n <= 1 || stride[0] == a * b);
  }
  // `elements` or more, one after the other
  bool dense(int want, int64_t elements) const {
    if (type != want || dims > 4) return false;
    int64_t n = 1;
    for (int i = dims - 1; i >= 0; --i) {
      if (size[i] > 1 && stride[i] != n) return false;
      n *= size[i];
    }
    return n >= elements;
  }
  int64_t row_stride(int64_t row) const { return size[0] > 1 ? stride[0] : row; }
};

PyObject* not_as_documented() { return PyLong_FromLong(-1); }

// Whether the cache's kv heads, head dimension, rank and type of l (which make_cache8 left beside it) are the shape's.  A cache that is
// written (`dst`, of make_cache) may have room for a larger rank, and one that its caller has described by hand is taken as it is.
bool fits(PyObject* cache, const lra_shape* sh, bool& yes, bool dst = false) {
  PyObject* v = PyObject_GetAttr(cache, s_sizes);
  if (!v) return false;
  int64_t x[4];
  int n;
  const bool any = dst && v == Py_None, ok = any || ints(v, x, n);
  Py_DECREF(v);
  yes = any || (ok && n == 4 && x[0] == sh->n_kv_heads && x[1] == sh->head_dim && (dst ? x[2] >= sh->rank : x[2] == sh->rank) && x[3] == sh->dtype);
  return ok;
}

// Whether the batch's seq_query_start (whose length make_batch left beside it) is that of n_seqs sequences.
bool same_sequences(PyObject* batch, int32_t n_seqs, bool& yes) {
  PyObject* v = PyObject_GetAttr(batch, s_n_seqs);
  if (!v) return false;
  yes = v == Py_None || PyLong_AsLongLong(v) == n_seqs;
  Py_DECREF(v);
  return !PyErr_Occurred();
}

// quantize(x, codes, scales, stream)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  View x, c, s;
  void* st;
  if (!arity(n, 4) || !x.open(a[0]) || !c.open(a[1]) || !s.open(a[2])) return nullptr;
  if (x.dims != 2 || x.type > kF32 || !x.matrix(x.type, x.size[0], x.size[1]) || !c.matrix(kI8, x.size[0], x.size[1]) || !s.vector(kF32, x.size[0]) ||
      x.size[0] > INT32_MAX || x.size[1] > INT32_MAX)
    return not_as_documented();
  if (!stream_handle(a[3], &st)) return nullptr;
  lra_status status;
  Py_BEGIN_ALLOW_THREADS
  status = g_quantize(x.data, x.type, x.row_stride(x.size[1]), static_cast<int32_t>(x.size[0]), static_cast<int32_t>(x.size[1]), static_cast<int8_t*>(c.data),
                      c.row_stride(x.size[1]), static_cast<float*>(s.data), st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// matmul(x, x_scale, w, w_scale, y, workspace, stream)
PyObject* matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
  View x, xs, w, ws, y;
  void *room, *st;
  size_t bytes;
  if (!arity(n, 7) || !x.open(a[0]) || !xs.open(a[1]) || !w.open(a[2]) || !ws.open(a[3]) || !y.open(a[4]) || !workspace(a[5], &room, &bytes))
    return nullptr;
  if (x.dims != 2 || w.dims != 2 || y.type > kF32) return not_as_documented();
  const int64_t m = x.size[0], nn = w.size[0], k = x.size[1];
  if (!x.matrix(kI8, m, k) || !w.matrix(kI8, nn, k) || !xs.vector(kF32, m) || !ws.vector(kF32, nn) || !y.matrix(y.type, m, nn) || m > INT32_MAX || nn > INT32_MAX ||
      k > INT32_MAX)
    return not_as_documented();
  const lra_i8_operands ops = {static_cast<const int8_t*>(x.data), static_cast<const int8_t*>(w.data), static_cast<const float*>(xs.data), static_cast<const float*>(ws.data),
                               x.row_stride(k), w.row_stride(k), static_cast<int32_t>(m), static_cast<int32_t>(nn), static_cast<int32_t>(k)};
  if (!stream_handle(a[6], &st)) return nullptr;
  lra_status status;
  Py_BEGIN_ALLOW_THREADS
  status = g_matmul(&ops, y.data, y.type, y.row_stride(nn), room, bytes, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// append8(shape, cache, seq_start, max_new_per_seq, k, v, l, rope_theta, positions, stream)
PyObject* append8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Struct sh, c;
  View start, k, v, l, pos;
  lra_new_rows rows{};
  void* st;
  bool yes;
  if (!arity(n, 10) || !sh.open(a[0], g_shape_type) || !c.open(a[1], g_cache8_type) || !start.open(a[2]) || !int32(a[3], &rows.max_new_per_seq) || !k.open(a[4]) ||
      !v.open(a[5]) || (a[6] != Py_None && !l.open(a[6])))
    return nullptr;
  const double theta = PyFloat_AsDouble(a[7]);
  if ((theta == -1.0 && PyErr_Occurred()) || (a[8] != Py_None && !pos.open(a[8])) || !fits(a[1], sh.as<lra_shape>(), yes)) return nullptr;
  const lra_shape* s = sh.as<lra_shape>();
  const int64_t new_rows = k.dims > 0 ? k.size[0] : 0;
  if (!yes || !k.rows(s->dtype, new_rows, s->n_kv_heads, s->head_dim, false) || !v.rows(s->dtype, new_rows, s->n_kv_heads, s->head_dim, false) ||
      (a[6] != Py_None && !l.matrix(s->dtype, new_rows, s->rank)) || !start.vector(kI32, static_cast<int64_t>(c.as<lra_cache8>()->n_seqs) + 1) ||
      (a[8] != Py_None && !pos.vector(kI32, new_rows)) || new_rows > INT32_MAX)
    return not_as_documented();
  const int64_t row = static_cast<int64_t>(s->n_kv_heads) * s->head_dim;
  rows.k = k.data;
  rows.v = v.data;
  rows.l = l.data;
  rows.k_token_stride = k.row_stride(row);
  rows.v_token_stride = v.row_stride(row);
  rows.l_token_stride = a[6] != Py_None ? l.row_stride(s->rank) : 0;
  rows.seq_start = static_cast<const int32_t*>(start.data);
  rows.positions = static_cast<const int32_t*>(pos.data);
  rows.n_new = static_cast<int32_t>(new_rows);
  rows.rope_theta = static_cast<float>(theta);
  if (!stream_handle(a[9], &st)) return nullptr;
  lra_status status;
  Py_BEGIN_ALLOW_THREADS
  status = g_append8(s, c.as<lra_cache8>(), &rows, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// gather8(shape, cache, dst, kept, stream)
PyObject* gather8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Struct sh, c, d;
  View kept;
  void* st;
  bool yes, room;
  if (!arity(n, 5) || !sh.open(a[0], g_shape_type) || !c.open(a[1], g_cache8_type) || !d.open(a[2], g_cache_type) || (a[3] != Py_None && !kept.open(a[3])) ||
      !fits(a[1], sh.as<lra_shape>(), yes) || !fits(a[2], sh.as<lra_shape>(), room, true))
    return nullptr;
  const lra_cache* dst = d.as<lra_cache>();
  if (!yes || !room || (a[3] != Py_None && (kept.dims != 2 || !kept.matrix(kI32, dst->n_seqs, kept.size[1]) || kept.size[1] < dst->max_seq_len))) return not_as_documented();
  if (!stream_handle(a[4], &st)) return nullptr;
  lra_status status;
  Py_BEGIN_ALLOW_THREADS
  status = g_gather8(sh.as<lra_shape>(), c.as<lra_cache8>(), static_cast<const int32_t*>(kept.data), a[3] != Py_None ? kept.row_stride(kept.size[1]) : 0, dst, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// attend8(shape, cache, b_k, b_v, n_adapters, batch, q, out, workspace, stream)
PyObject* attend8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Struct sh, c, b;
  lra_adapters ad{};
  View q, out, b_k, b_v;
  void *ws, *st;
  size_t bytes;
  bool yes, same;
  if (!arity(n, 10) || !sh.open(a[0], g_shape_type) || !c.open(a[1], g_cache8_type) || (a[2] != Py_None && !b_k.open(a[2])) || (a[3] != Py_None && !b_v.open(a[3])) ||
      !int32(a[4], &ad.n_adapters) || !b.open(a[5], g_batch_type) || !q.open(a[6]) || !out.open(a[7]) || !workspace(a[8], &ws, &bytes) ||
      !fits(a[1], sh.as<lra_shape>(), yes) || !same_sequences(a[5], c.as<lra_cache8>()->n_seqs, same))
    return nullptr;
  const lra_shape* s = sh.as<lra_shape>();
  const int64_t queries = b.as<lra_batch>()->n_queries, table = static_cast<int64_t>(ad.n_adapters) * s->rank * s->n_kv_heads * s->head_dim;
  if ((a[2] != Py_None && !b_k.dense(s->dtype, table)) || (a[3] != Py_None && !b_v.dense(s->dtype, table))) return not_as_documented();
  if (!yes || !same || !q.rows(s->dtype, queries, s->n_q_heads, s->head_dim, true) || !out.rows(s->dtype, queries, s->n_q_heads, s->head_dim, true)) return not_as_documented();
  ad.b_k = b_k.data;
  ad.b_v = b_v.data;
  if (!stream_handle(a[9], &st)) return nullptr;
  lra_status status;
  Py_BEGIN_ALLOW_THREADS
  status = g_attend8(s, c.as<lra_cache8>(), &ad, b.as<lra_batch>(), q.data, out.data, ws, bytes, g_tuning, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// bind8(quantize, matmul, append, gather, attend: addresses; LraCache8, LraBatch; bfloat16, float32, int8, int32), behind bind()
PyObject* bind8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 11)) return nullptr;
  void* p[5];
  for (int i = 0; i < 5; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no address");
      return nullptr;
    }
  }
  if (!PyType_Check(a[5]) || !PyType_Check(a[6])) {
    PyErr_SetString(PyExc_TypeError, "expected the two struct types");
    return nullptr;
  }
  g_quantize = reinterpret_cast<decltype(g_quantize)>(p[0]);
  g_matmul = reinterpret_cast<decltype(g_matmul)>(p[1]);
  g_append8 = reinterpret_cast<decltype(g_append8)>(p[2]);
  g_gather8 = reinterpret_cast<decltype(g_gather8)>(p[3]);
  g_attend8 = reinterpret_cast<decltype(g_attend8)>(p[4]);
  g_cache8_type = reinterpret_cast<PyTypeObject*>(Py_NewRef(a[5]));
  g_batch_type = reinterpret_cast<PyTypeObject*>(Py_NewRef(a[6]));
  for (int i = 0; i < 4; ++i) g_dtypes[i] = Py_NewRef(a[7 + i]);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind8)), METH_FASTCALL, nullptr},
    {"quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(quantize)), METH_FASTCALL, nullptr},
    {"matmul", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(matmul)), METH_FASTCALL, nullptr},
    {"append8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append8)), METH_FASTCALL, nullptr},
    {"gather8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gather8)), METH_FASTCALL, nullptr},
    {"attend8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attend8)), METH_FASTCALL, nullptr},
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind)), METH_FASTCALL, nullptr},
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode)), METH_FASTCALL, nullptr},
    {"prefill", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(prefill)), METH_FASTCALL, nullptr},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lra_pycall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lra_pycall() {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_size = PyUnicode_InternFromString("size");
  s_nbytes = PyUnicode_InternFromString("nbytes");
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  s_zero = PyLong_FromLong(0);
  s_one = PyLong_FromLong(1);
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_sizes = PyUnicode_InternFromString("_sizes");
  s_n_seqs = PyUnicode_InternFromString("_n_seqs");
  if (!s_data_ptr || !s_size || !s_nbytes || !s_cuda_stream || !s_zero || !s_one || !s_shape || !s_stride || !s_dtype || !s_sizes || !s_n_seqs) return nullptr;
  return PyModule_Create(&module);
}
