// Argument marshalling of the launch entry points for torch tensors, as a CPython extension: reads the addresses of the
// tensors of a call, looks up the current stream and calls the C ABI of libsfmp.so.
//
// A decode launch takes 4 to 12 us on the GPU.  Marshalled in Python (ctypes, four tensor methods per argument) an
// sfmp_gemm call took 12.1 us of host time and a launch of three projections 16.2, so that a program waited for the host;
// marshalled here 3.8 and 3.9, most of it the launch itself (back to back, 512 -> 512: 11.6 -> 4.2 us a call, a decoder
// layer of an 8B model in four calls 46 -> 29 us).
//
// Only plain calls are taken: torch.Tensor or Parameter objects themselves (no subclass, which may have methods of its
// own), None, an SfmpLayout.  For anything else a function returns None, nothing having been launched, and the general
// path in binding.py decides, with its own errors.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include "../../include/sfmp.h"

namespace {

struct Api {
  decltype(&sfmp_gemm) gemm = nullptr;
  decltype(&sfmp_gemm_static) gemm_static = nullptr;
  decltype(&sfmp_gemv_batched) gemv_batched = nullptr;
  decltype(&sfmp_gemm_batched) gemm_batched = nullptr;
};

// set by bind()
Api api;
PyObject* layout_type = nullptr;
PyObject* get_device = nullptr;      // torch._C._cuda_getDevice
PyObject* get_raw_stream = nullptr;  // torch._C._cuda_getCurrentRawStream
PyObject* names[9];                  // attributes of a DevicePacked, then "cuda_stream"
const char* const kNames[9] = {"layout", "s2", "s3", "s4", "index", "scales", "zeros", "bitmap", "cuda_stream"};

// What became of reading an argument: taken, not a plain one (the general path decides), or a Python error is set
enum Read { kTaken, kOther, kError };

// Address of a tensor (null for None and for an empty one).  device: the tensor has to be a contiguous one on the GPU.
Read tensor_address(PyObject* o, bool device, const void** out) {
  *out = nullptr;
  if (o == Py_None) return kTaken;
  if (!THPVariable_CheckExact(o)) return kOther;
  try {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.numel() == 0) return kTaken;
    if (device && (!t.is_cuda() || !t.is_contiguous())) return kOther;
    *out = t.data_ptr();
    return kTaken;
  } catch (const std::exception&) {  // a tensor without memory of its own: the general path raises its error
    return kOther;
  }
}

Read tensor_rows(PyObject* o, int64_t* rows, int64_t* numel, int64_t* bytes) {
  if (!THPVariable_CheckExact(o)) return kOther;
  try {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (rows) {
      if (t.dim() < 1 || t.size(0) > INT32_MAX) return kOther;
      *rows = t.size(0);
    }
    if (numel) *numel = t.numel();
    if (bytes) *bytes = t.numel() * (int64_t)t.element_size();
    return kTaken;
  } catch (const std::exception&) {
    return kOther;
  }
}

// Address of the C struct of an SfmpLayout (the caller holds a reference through the call)
Read layout_address(PyObject* o, const sfmp_layout_t** out) {
  if ((PyObject*)Py_TYPE(o) != layout_type) return kOther;
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return kError;
  *out = b.len == (Py_ssize_t)sizeof(sfmp_layout_t) ? (const sfmp_layout_t*)b.buf : nullptr;
  PyBuffer_Release(&b);
  return *out ? kTaken : kOther;
}

Read stream_handle(PyObject* stream, void** out) {
  PyObject* h;
  if (stream == Py_None) {
    PyObject* dev = PyObject_CallNoArgs(get_device);
    h = dev ? PyObject_CallOneArg(get_raw_stream, dev) : nullptr;
    Py_XDECREF(dev);
    if (!h) {  // no usable GPU: the general path initialises torch's side, or raises its error
      PyErr_Clear();
      return kOther;
    }
  } else {
    h = PyObject_GetAttr(stream, names[8]);
  }
  if (!h) return kError;
  *out = PyLong_AsVoidPtr(h);
  Py_DECREF(h);
  return PyErr_Occurred() ? kError : kTaken;
}

#define SFMP_READ(expr)                        \
  do {                                         \
    const Read r_ = (expr);                    \
    if (r_ == kError) return nullptr;          \
    if (r_ == kOther) Py_RETURN_NONE;          \
  } while (0)

// gemm(X, col_perm, layout, s2, s3, s4, index, scales, zeros, bitmap, row_perm, Y, workspace or missing, stream)
template <bool STATIC>
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr Py_ssize_t kArgs = STATIC ? 13 : 14;
  if (n != kArgs) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  int64_t M = 0, nbytes = 0;
  const sfmp_layout_t* layout = nullptr;
  const void* p[13] = {};
  if constexpr (!STATIC) SFMP_READ(tensor_rows(a[12], nullptr, nullptr, &nbytes));
  SFMP_READ(tensor_rows(a[0], &M, nullptr, nullptr));
  SFMP_READ(layout_address(a[2], &layout));
  for (int i = 0; i < kArgs - 1; ++i)
    if (i != 2) SFMP_READ(tensor_address(a[i], true, &p[i]));
  void* stream = nullptr;
  SFMP_READ(stream_handle(a[kArgs - 1], &stream));
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  if constexpr (STATIC)
    rc = api.gemm_static(p[0], (int32_t)M, (const int32_t*)p[1], layout, p[3], p[4], p[5], (const int32_t*)p[6], p[7],
                         p[8], (const int8_t*)p[9], (const int32_t*)p[10], (void*)p[11], stream);
  else
    rc = api.gemm(p[0], (int32_t)M, (const int32_t*)p[1], layout, p[3], p[4], p[5], (const int32_t*)p[6], p[7], p[8],
                  (const int8_t*)p[9], (const int32_t*)p[10], (void*)p[11], (void*)p[12], nbytes, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(rc);
}

constexpr Py_ssize_t kMaxBatch = 8;  // more are refused by the library: left to the general path

// References to everything whose address has been read, dropped when the call returns (with the GIL held).  The tensors
// and layouts of a batch hang on a list and on attributes that other Python code - an attribute lookup of this call, a
// stream object's property, another thread while the library runs without the GIL - may change or clear meanwhile.
struct Held {
  PyObject* ref[1 + 8 * kMaxBatch];
  int count = 0;
  void take(PyObject* owned) { ref[count++] = owned; }
  Held() = default;
  Held(const Held&) = delete;
  Held& operator=(const Held&) = delete;
  ~Held() {
    while (count > 0) Py_DECREF(ref[--count]);
  }
};

// problems: list or tuple of (X, col_perm, DevicePacked, row_perm, Y)
Read read_problems(PyObject* problems, sfmp_gemv_problem_t* out, int32_t* count, Held* held) {
  if (!PyList_CheckExact(problems) && !PyTuple_CheckExact(problems)) return kOther;
  PyObject* all = PySequence_Tuple(problems);  // (its items, and theirs, stay as they are through the call)
  if (!all) return kError;
  held->take(all);
  const Py_ssize_t n = PyTuple_GET_SIZE(all);
  if (n > kMaxBatch) return kOther;
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* q = PyTuple_GET_ITEM(all, i);
    if (!PyTuple_CheckExact(q) || PyTuple_GET_SIZE(q) != 5) return kOther;
    PyObject* dp = PyTuple_GET_ITEM(q, 2);
    const void* v[12] = {};
    if (Read r = tensor_address(PyTuple_GET_ITEM(q, 0), false, &v[0])) return r;
    if (Read r = tensor_address(PyTuple_GET_ITEM(q, 1), false, &v[1])) return r;
    for (int k = 0; k < 8; ++k) {
      PyObject* o = PyObject_GetAttr(dp, names[k]);
      if (!o) return kError;
      held->take(o);
      const Read r = k == 0 ? layout_address(o, (const sfmp_layout_t**)&v[2]) : tensor_address(o, false, &v[2 + k]);
      if (r != kTaken) return r;
    }
    if (Read r = tensor_address(PyTuple_GET_ITEM(q, 3), false, &v[10])) return r;
    if (Read r = tensor_address(PyTuple_GET_ITEM(q, 4), false, &v[11])) return r;
    out[i] = sfmp_gemv_problem_t{v[0], (const int32_t*)v[1], (const sfmp_layout_t*)v[2], v[3], v[4], v[5],
                                 (const int32_t*)v[6], v[7], v[8], (const int8_t*)v[9], (const int32_t*)v[10],
                                 (void*)v[11]};
  }
  *count = (int32_t)n;
  return kTaken;
}

// gemv_batched(problems, stream)
PyObject* gemv_batched(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 2) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  Held held;
  sfmp_gemv_problem_t q[kMaxBatch];
  int32_t count = 0;
  void* stream = nullptr;
  SFMP_READ(read_problems(a[0], q, &count, &held));
  SFMP_READ(stream_handle(a[1], &stream));
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = api.gemv_batched(q, count, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(rc);
}

// gemm_batched(problems, M, workspace, stream)
PyObject* gemm_batched(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  Held held;
  sfmp_gemv_problem_t q[kMaxBatch];
  int32_t count = 0;
  void* stream = nullptr;
  const void* ws = nullptr;
  int64_t numel = 0;
  if (!PyLong_CheckExact(a[1])) Py_RETURN_NONE;
  int overflow = 0;
  const long M = PyLong_AsLongAndOverflow(a[1], &overflow);
  if (overflow || M < INT32_MIN || M > INT32_MAX) Py_RETURN_NONE;
  SFMP_READ(read_problems(a[0], q, &count, &held));
  if (a[2] == Py_None) Py_RETURN_NONE;
  SFMP_READ(tensor_rows(a[2], nullptr, &numel, nullptr));
  if (numel == 0) Py_RETURN_NONE;
  SFMP_READ(tensor_address(a[2], false, &ws));
  SFMP_READ(stream_handle(a[3], &stream));
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = api.gemm_batched(q, count, (int32_t)M, (void*)ws, numel, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(rc);
}

// ---- cache and sampling calls ---------------------------------------------------------------------------------------

struct KvApi {
  decltype(&sfmp_kv_append) append = nullptr;
  decltype(&sfmp_kv_gather) gather = nullptr;
  decltype(&sfmp_kv_attention) attention = nullptr;
  decltype(&sfmp_kv_reserve) reserve = nullptr;
  decltype(&sfmp_kv_fork) fork = nullptr;
  decltype(&sfmp_kv_free) free_pages = nullptr;
  decltype(&sfmp_kv_compact) compact = nullptr;
  decltype(&sfmp_sample) sample = nullptr;
};

// set by bind_kv()
KvApi kv;
PyObject* kv_layout_type = nullptr;
PyObject* kv_names[6];
const char* const kKvNames[6] = {"layout", "codes", "scales", "page_table", "lengths", "refs"};

// A contiguous GPU tensor of this type and these extents (-1: any); null for None and for an empty one.
Read checked(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> shape, const void** out) {
  *out = nullptr;
  if (o == Py_None) return kTaken;
  if (!THPVariable_CheckExact(o)) return kOther;
  try {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != type || t.dim() != (int64_t)shape.size()) return kOther;
    int64_t d = 0;
    for (const int64_t n : shape) {
      if (n >= 0 && t.size(d) != n) return kOther;
      ++d;
    }
    if (!t.is_contiguous()) return kOther;
    if (t.numel()) *out = t.data_ptr();
    return kTaken;
  } catch (const std::exception&) {
    return kOther;
  }
}

// [rows, heads, dim] (heads -1: any), rows contiguous inside
struct RowsArg {
  const void* at = nullptr;
  int32_t type = 0, rows = 0, heads = 0;
  int64_t stride = 0;
};
Read rows_of(PyObject* o, bool fp32, int64_t heads, int64_t dim, RowsArg* out) {
  if (!THPVariable_CheckExact(o)) return kOther;
  try {
    const at::Tensor& t = THPVariable_Unpack(o);
    const at::ScalarType s = t.scalar_type();
    if (!t.is_cuda() || t.dim() != 3 || t.size(2) != dim || (heads >= 0 && t.size(1) != heads) || t.size(0) > INT32_MAX ||
        t.size(1) > INT32_MAX || t.stride(2) != 1 || (t.size(1) > 1 && t.stride(1) != dim))
      return kOther;
    if (s == at::kHalf)
      out->type = SFMP_TYPE_FP16;
    else if (s == at::kBFloat16)
      out->type = SFMP_TYPE_BF16;
    else if (s == at::kFloat && fp32)
      out->type = SFMP_TYPE_FP32;
    else
      return kOther;
    out->at = t.numel() ? t.data_ptr() : nullptr;
    out->rows = (int32_t)t.size(0);
    out->heads = (int32_t)t.size(1);
    out->stride = t.size(0) > 1 ? t.stride(0) : (t.size(1) * dim + 7) / 8 * 8;
    return kTaken;
  } catch (const std::exception&) {
    return kOther;
  }
}

Read length_of(PyObject* o, int32_t* n) {  // of a vector
  if (!THPVariable_CheckExact(o)) return kOther;
  try {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.dim() != 1 || t.size(0) > INT32_MAX) return kOther;
    *n = (int32_t)t.size(0);
    return kTaken;
  } catch (const std::exception&) {
    return kOther;
  }
}

Read int_of(PyObject* o, int32_t* out) {
  if (!PyLong_CheckExact(o)) return kOther;
  int overflow = 0;
  const long x = PyLong_AsLongAndOverflow(o, &overflow);
  if (overflow || x < INT32_MIN || x > INT32_MAX) return kOther;
  *out = (int32_t)x;
  return kTaken;
}

Read workspace_of(PyObject* o, const void** at, int64_t* bytes) {
  *bytes = 0;
  if (Read r = tensor_address(o, true, at)) return r;
  return o == Py_None ? kTaken : tensor_rows(o, nullptr, nullptr, bytes);
}

// DeviceKvCache and DeviceKvTables
struct CacheArg {
  sfmp_kv_layout_t layout;  // (a copy: the struct may be changed by other Python code meanwhile)
  const void* codes = nullptr;
  const void* scales = nullptr;
  sfmp_kv_tables_t tables{};
};
Read attribute(PyObject* o, int name, Held* held, PyObject** out) {
  *out = PyObject_GetAttr(o, kv_names[name]);
  if (!*out) return kError;
  held->take(*out);
  return kTaken;
}
Read read_cache(PyObject* cache, PyObject* tables, Held* held, CacheArg* c) {
  PyObject* o;
  if (Read r = attribute(cache, 0, held, &o)) return r;
  if ((PyObject*)Py_TYPE(o) != kv_layout_type) return kOther;
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return kError;
  const bool whole = b.len == (Py_ssize_t)sizeof(c->layout);
  if (whole) c->layout = *(const sfmp_kv_layout_t*)b.buf;
  PyBuffer_Release(&b);
  if (!whole) return kOther;
  const sfmp_kv_layout_t& L = c->layout;
  if (Read r = attribute(cache, 1, held, &o)) return r;
  if (Read r = checked(o, at::kByte, {L.layers, L.pages, L.kv_heads, 2, (int64_t)SFMP_KV_PAGE * L.head_dim}, &c->codes)) return r;
  if (Read r = attribute(cache, 2, held, &o)) return r;
  if (Read r = checked(o, at::kFloat, {L.layers, L.pages, L.kv_heads, 2}, &c->scales)) return r;
  const void *table, *lengths, *refs;
  if (Read r = attribute(tables, 3, held, &o)) return r;
  if (Read r = checked(o, at::kInt, {-1, -1}, &table)) return r;
  if (o == Py_None) return kOther;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX) return kOther;
  c->tables.sequences = (int32_t)t.size(0);
  c->tables.table_pages = (int32_t)t.size(1);
  if (Read r = attribute(tables, 4, held, &o)) return r;
  if (Read r = checked(o, at::kInt, {c->tables.sequences}, &lengths)) return r;
  if (Read r = attribute(tables, 5, held, &o)) return r;
  if (Read r = checked(o, at::kInt, {L.pages}, &refs)) return r;
  c->tables.page_table_dev = (int32_t*)table;
  c->tables.lengths_dev = (int32_t*)lengths;
  c->tables.refs_dev = (int32_t*)refs;
  return kTaken;
}

Read read_batch(PyObject* slots, PyObject* row_start, int32_t rows, PyObject* max_rows, sfmp_kv_batch_t* b) {
  const void *s, *r0;
  b->rows = b->batch = rows;
  b->reserved = 0;
  if (slots != Py_None) {
    if (Read r = length_of(slots, &b->batch)) return r;
  } else if (row_start != Py_None) {
    if (Read r = length_of(row_start, &b->batch)) return r;
    if (b->batch < 1) return kOther;
    --b->batch;
  }
  if (Read r = checked(slots, at::kInt, {-1}, &s)) return r;
  if (Read r = checked(row_start, at::kInt, {(int64_t)b->batch + 1}, &r0)) return r;
  b->slots_dev = (const int32_t*)s;
  b->row_start_dev = (const int32_t*)r0;
  return int_of(max_rows, &b->max_rows);
}

bool wrong_count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return false;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return true;
}

template <typename F>
PyObject* call(F f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = f();
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(rc);
}

// kv_append(cache, layer, tables, slots, row_start, K, V, max_rows, stream)
// kv_gather(cache, layer, tables, slots, first, row_start, K, V, max_rows, stream)
template <bool GATHER>
PyObject* kv_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr int G = GATHER ? 1 : 0;
  if (wrong_count(n, 9 + G)) return nullptr;
  Held held;
  CacheArg c;
  RowsArg k, v;
  sfmp_kv_batch_t b;
  int32_t layer;
  const void* first = nullptr;
  void* stream = nullptr;
  SFMP_READ(read_cache(a[0], a[2], &held, &c));
  SFMP_READ(int_of(a[1], &layer));
  SFMP_READ(rows_of(a[5 + G], GATHER, c.layout.kv_heads, c.layout.head_dim, &k));
  SFMP_READ(rows_of(a[6 + G], GATHER, c.layout.kv_heads, c.layout.head_dim, &v));
  if (k.rows != v.rows || k.type != v.type) Py_RETURN_NONE;
  SFMP_READ(read_batch(a[3], a[4 + G], k.rows, a[7 + G], &b));
  if constexpr (GATHER) SFMP_READ(checked(a[4], at::kInt, {b.batch}, &first));
  SFMP_READ(stream_handle(a[8 + G], &stream));
  return call([&] {
    if constexpr (GATHER)
      return kv.gather(&c.layout, layer, c.codes, (const float*)c.scales, &c.tables, &b, (const int32_t*)first, (void*)k.at,
                       (void*)v.at, k.type, k.stride, v.stride, stream);
    else
      return kv.append(&c.layout, layer, (void*)c.codes, (float*)c.scales, &c.tables, &b, k.at, v.at, k.type, k.stride, v.stride,
                       stream);
  });
}

// kv_attention(cache, layer, tables, slots, row_start, Q, O, max_rows, max_tokens, scale, workspace, window, lse, stream)
PyObject* kv_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (wrong_count(n, 14)) return nullptr;
  Held held;
  CacheArg c;
  RowsArg q, o;
  sfmp_kv_batch_t b;
  int32_t layer, max_tokens, window;
  int64_t bytes = 0;
  const void *workspace = nullptr, *lse = nullptr;
  void* stream = nullptr;
  SFMP_READ(read_cache(a[0], a[2], &held, &c));
  SFMP_READ(int_of(a[1], &layer));
  SFMP_READ(rows_of(a[5], false, -1, c.layout.head_dim, &q));
  SFMP_READ(rows_of(a[6], false, q.heads, c.layout.head_dim, &o));
  if (q.rows != o.rows || q.type != o.type) Py_RETURN_NONE;
  SFMP_READ(read_batch(a[3], a[4], q.rows, a[7], &b));
  SFMP_READ(int_of(a[8], &max_tokens));
  if (!PyFloat_CheckExact(a[9])) Py_RETURN_NONE;
  const float scale = (float)PyFloat_AS_DOUBLE(a[9]);
  SFMP_READ(workspace_of(a[10], &workspace, &bytes));
  SFMP_READ(int_of(a[11], &window));
  SFMP_READ(checked(a[12], at::kFloat, {q.rows, q.heads}, &lse));
  SFMP_READ(stream_handle(a[13], &stream));
  return call([&] {
    return kv.attention(&c.layout, layer, c.codes, (const float*)c.scales, &c.tables, &b, q.at, q.heads, q.type, q.stride,
                        max_tokens, window, scale, (void*)o.at, o.stride, (float*)lse, (void*)workspace, bytes, stream);
  });
}

// kv_reserve(cache, tables, slots, counts, status, workspace, stream)
PyObject* kv_reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (wrong_count(n, 7)) return nullptr;
  Held held;
  CacheArg c;
  int32_t m = 0;
  int64_t bytes = 0;
  const void *slots = nullptr, *counts = nullptr, *status = nullptr, *workspace = nullptr;
  void* stream = nullptr;
  SFMP_READ(read_cache(a[0], a[1], &held, &c));
  SFMP_READ(length_of(a[2], &m));
  SFMP_READ(checked(a[2], at::kInt, {m}, &slots));
  SFMP_READ(checked(a[3], at::kInt, {m}, &counts));
  SFMP_READ(checked(a[4], at::kInt, {1}, &status));
  SFMP_READ(workspace_of(a[5], &workspace, &bytes));
  SFMP_READ(stream_handle(a[6], &stream));
  return call([&] {
    return kv.reserve(&c.layout, (void*)c.codes, (float*)c.scales, &c.tables, (const int32_t*)slots, (const int32_t*)counts, m,
                      (int32_t*)status, (void*)workspace, bytes, stream);
  });
}

// kv_fork(cache, tables, parents, children, stream); kv_free(cache, tables, slots, keep, stream)
template <bool FORK>
PyObject* kv_tables(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (wrong_count(n, 5)) return nullptr;
  Held held;
  CacheArg c;
  int32_t m = 0;
  const void *x = nullptr, *y = nullptr;
  void* stream = nullptr;
  SFMP_READ(read_cache(a[0], a[1], &held, &c));
  SFMP_READ(length_of(a[2], &m));
  SFMP_READ(checked(a[2], at::kInt, {m}, &x));
  SFMP_READ(checked(a[3], at::kInt, {m}, &y));
  SFMP_READ(stream_handle(a[4], &stream));
  return call([&] {
    return (FORK ? kv.fork : kv.free_pages)(&c.layout, &c.tables, (const int32_t*)x, (const int32_t*)y, m, stream);
  });
}

// kv_compact(cache, tables, status, workspace, stream)
PyObject* kv_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (wrong_count(n, 5)) return nullptr;
  Held held;
  CacheArg c;
  int64_t bytes = 0;
  const void *status = nullptr, *workspace = nullptr;
  void* stream = nullptr;
  SFMP_READ(read_cache(a[0], a[1], &held, &c));
  SFMP_READ(checked(a[2], at::kInt, {1}, &status));
  SFMP_READ(workspace_of(a[3], &workspace, &bytes));
  SFMP_READ(stream_handle(a[4], &stream));
  return call([&] {
    return kv.compact(&c.layout, (void*)c.codes, (float*)c.scales, &c.tables, (int32_t*)status, (void*)workspace, bytes, stream);
  });
}

// sample(logits, temperature, top_k, top_p, min_p, uniform, tokens, logprobs, workspace, stream)
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (wrong_count(n, 10)) return nullptr;
  if (!THPVariable_CheckExact(a[0])) Py_RETURN_NONE;
  int32_t type, rows, vocab;
  int64_t stride, bytes = 0;
  const void *logits, *p[7] = {}, *workspace = nullptr;
  void* stream = nullptr;
  try {
    const at::Tensor& t = THPVariable_Unpack(a[0]);
    const at::ScalarType s = t.scalar_type();
    if (!t.is_cuda() || t.dim() != 2 || t.size(0) > INT32_MAX || t.size(1) > INT32_MAX || (t.size(1) > 1 && t.stride(1) != 1) ||
        (s != at::kHalf && s != at::kBFloat16 && s != at::kFloat))
      Py_RETURN_NONE;
    type = s == at::kHalf ? SFMP_TYPE_FP16 : s == at::kBFloat16 ? SFMP_TYPE_BF16 : SFMP_TYPE_FP32;
    rows = (int32_t)t.size(0);
    vocab = (int32_t)t.size(1);
    stride = rows > 1 ? t.stride(0) : vocab;
    logits = t.numel() ? t.data_ptr() : nullptr;
  } catch (const std::exception&) {
    Py_RETURN_NONE;
  }
  for (int i = 0; i < 7; ++i) SFMP_READ(checked(a[1 + i], i == 1 || i == 5 ? at::kInt : at::kFloat, {rows}, &p[i]));
  SFMP_READ(workspace_of(a[8], &workspace, &bytes));
  SFMP_READ(stream_handle(a[9], &stream));
  return call([&] {
    return kv.sample(logits, type, rows, vocab, stride, (const float*)p[0], (const int32_t*)p[1], (const float*)p[2],
                     (const float*)p[3], (const float*)p[4], (int32_t*)p[5], (float*)p[6], (void*)workspace, bytes, stream);
  });
}

// bind_kv(SfmpKvLayout, addresses of the eight C functions); after bind()
PyObject* bind_kv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (wrong_count(n, 9)) return nullptr;
  void* f[8];
  for (int i = 0; i < 8; ++i) {
    f[i] = PyLong_AsVoidPtr(a[1 + i]);
    if (!f[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null function");
      return nullptr;
    }
  }
  Py_INCREF(a[0]);
  Py_XSETREF(kv_layout_type, a[0]);
  kv.append = (decltype(kv.append))f[0];
  kv.gather = (decltype(kv.gather))f[1];
  kv.attention = (decltype(kv.attention))f[2];
  kv.reserve = (decltype(kv.reserve))f[3];
  kv.fork = (decltype(kv.fork))f[4];
  kv.free_pages = (decltype(kv.free_pages))f[5];
  kv.compact = (decltype(kv.compact))f[6];
  kv.sample = (decltype(kv.sample))f[7];
  Py_RETURN_NONE;
}

// bind(SfmpLayout, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, addresses of the four C functions)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  void* f[4];
  for (int i = 0; i < 4; ++i) {
    f[i] = PyLong_AsVoidPtr(a[3 + i]);
    if (!f[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null function");
      return nullptr;
    }
  }
  PyObject** const slot[3] = {&layout_type, &get_device, &get_raw_stream};
  for (int i = 0; i < 3; ++i) {
    Py_INCREF(a[i]);
    Py_XSETREF(*slot[i], a[i]);
  }
  api.gemm = (decltype(api.gemm))f[0];
  api.gemm_static = (decltype(api.gemm_static))f[1];
  api.gemv_batched = (decltype(api.gemv_batched))f[2];
  api.gemm_batched = (decltype(api.gemm_batched))f[3];
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
    {"gemm", (PyCFunction)(void (*)(void))gemm<false>, METH_FASTCALL, nullptr},
    {"gemm_static", (PyCFunction)(void (*)(void))gemm<true>, METH_FASTCALL, nullptr},
    {"gemv_batched", (PyCFunction)(void (*)(void))gemv_batched, METH_FASTCALL, nullptr},
    {"gemm_batched", (PyCFunction)(void (*)(void))gemm_batched, METH_FASTCALL, nullptr},
    {"bind_kv", (PyCFunction)(void (*)(void))bind_kv, METH_FASTCALL, nullptr},
    {"kv_append", (PyCFunction)(void (*)(void))kv_rows<false>, METH_FASTCALL, nullptr},
    {"kv_gather", (PyCFunction)(void (*)(void))kv_rows<true>, METH_FASTCALL, nullptr},
    {"kv_attention", (PyCFunction)(void (*)(void))kv_attention, METH_FASTCALL, nullptr},
    {"kv_reserve", (PyCFunction)(void (*)(void))kv_reserve, METH_FASTCALL, nullptr},
    {"kv_fork", (PyCFunction)(void (*)(void))kv_tables<true>, METH_FASTCALL, nullptr},
    {"kv_free", (PyCFunction)(void (*)(void))kv_tables<false>, METH_FASTCALL, nullptr},
    {"kv_compact", (PyCFunction)(void (*)(void))kv_compact, METH_FASTCALL, nullptr},
    {"sample", (PyCFunction)(void (*)(void))sample, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sfmp_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__sfmp_torch(void) {
  for (int i = 0; i < 9; ++i)
    if (!(names[i] = PyUnicode_InternFromString(kNames[i]))) return nullptr;
  for (int i = 0; i < 6; ++i)
    if (!(kv_names[i] = PyUnicode_InternFromString(kKvNames[i]))) return nullptr;
  PyObject* m = PyModule_Create(&module);
  // (checked by binding.py before anything else of the module is used)
  if (m && PyModule_AddStringConstant(m, "built_for", SFMP_BUILT_FOR) != 0) Py_CLEAR(m);
  return m;
}
