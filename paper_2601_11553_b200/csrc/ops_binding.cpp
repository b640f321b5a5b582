// Python side of the cache operators' entry points: looks at the tensors, refuses what the C interface cannot take, calls it.
//
// Tensors are looked at through their Python attributes (dtype, shape, strides, device, address), so nothing here depends on
// a version of torch.  It is compiled because a small call's time is the host's: the same checks written in Python, with the
// call through ctypes, made calls on one prompt the host's work: a decode step over 512 slots 16.1 -> 10.6 us a call (its kernel: 10.5),
// moving 1024 slots 14.5 -> 9.5 us, choosing 1024 of 2112 for 28 layers 11.4 -> 8.8 us.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cmath>
#include <cstdio>
#include <cstdint>

#include "../../include/percache.h"

namespace {

// ---------------------------------------------------------------------------------------------------- set once by bind()
decltype(&percache_tree_attention) f_tree;
decltype(&percache_attention_weights) f_weights;
decltype(&percache_select_slots) f_select;
decltype(&percache_compact_slots) f_compact;
decltype(&percache_append_rows) f_append;
decltype(&percache_append_rows_8bit) f_append8;
decltype(&percache_tree_attention_8bit) f_tree8;
decltype(&percache_fork_pages) f_fork;
enum Type { I32 = 1, F32 = 2, U8 = 4, BOOL = 8, I64 = 16, U64 = 32, BF16 = 64, F16 = 128, F8 = 256 };
constexpr int N_TYPES = 9;
PyObject* types[N_TYPES];                       // torch's type objects, in the order of Type
PyObject* current_stream;                       // device -> torch's current stream there
PyObject* to_dlpack;                            // tensor -> its DLPack capsule, or NULL
PyObject *n_dtype, *n_shape, *n_get_device, *n_stride, *n_data_ptr, *n_element_size;

struct Ref {                                    // owns a reference
  PyObject* p;
  explicit Ref(PyObject* x) : p(x) {}
  ~Ref() { Py_XDECREF(p); }
  Ref(const Ref&) = delete;
  Ref& operator=(const Ref&) = delete;
};
struct Error {};                                // a Python exception is set

[[noreturn]] void refuse(const char* name, const char* what) {
  PyErr_Format(PyExc_ValueError, "%s: expected %s", name, what);
  throw Error{};
}
int64_t integer(PyObject* x) {
  const long long v = PyLong_AsLongLong(x);
  if (v == -1 && PyErr_Occurred()) throw Error{};
  return v;
}
int32_t int32(PyObject* x, const char* name) {
  const int64_t v = integer(x);
  if (v < INT32_MIN || v > INT32_MAX) refuse(name, "a 32-bit number");
  return static_cast<int32_t>(v);
}
float number(PyObject* x) {
  const double v = PyFloat_AsDouble(x);
  if (v == -1.0 && PyErr_Occurred()) throw Error{};
  return static_cast<float>(v);
}
void* address(PyObject* x) {                    // of a number, e.g. a stream
  void* p = PyLong_AsVoidPtr(x);
  if (!p && PyErr_Occurred()) throw Error{};
  return p;
}
// The caller's stream, or torch's current one: that is what the tensors' other work is ordered on.
void* stream_of(PyObject* x, int device) {
  if (x != Py_None) return address(x);
  const Ref d(PyLong_FromLong(device));
  if (!d.p) throw Error{};
  const Ref r(PyObject_CallOneArg(current_stream, d.p));
  if (!r.p) throw Error{};
  return address(r.p);
}
int64_t ask(PyObject* x, PyObject* method) {
  const Ref r(PyObject_CallMethodNoArgs(x, method));
  if (!r.p) throw Error{};
  return integer(r.p);
}
void* data_of(PyObject* x) {
  const Ref r(PyObject_CallMethodNoArgs(x, n_data_ptr));
  if (!r.p) throw Error{};
  return address(r.p);
}
int type_of(PyObject* x) {                      // 0: none of ours
  const Ref r(PyObject_GetAttr(x, n_dtype));
  if (!r.p) throw Error{};
  for (int i = 0; i < N_TYPES; ++i)
    if (r.p == types[i]) return 1 << i;
  return 0;
}
// The first N sizes or strides of a tensor; returns how many it has.
template <int N>
int numbers(PyObject* tuple, int64_t (&out)[N]) {
  if (!tuple) throw Error{};
  if (!PyTuple_Check(tuple)) refuse("argument", "a tensor");
  const Py_ssize_t n = PyTuple_GET_SIZE(tuple);
  for (Py_ssize_t i = 0; i < n && i < N; ++i) out[i] = integer(PyTuple_GET_ITEM(tuple, i));
  return static_cast<int>(n);
}
template <int N>
int shape_of(PyObject* x, int64_t (&out)[N]) {
  const Ref r(PyObject_GetAttr(x, n_shape));
  return numbers(r.p, out);
}
template <int N>
int strides_of(PyObject* x, int64_t (&out)[N]) {
  const Ref r(PyObject_CallMethodNoArgs(x, n_stride));
  return numbers(r.p, out);
}
// What a tensor is.  DLPack's description (a public, stable layout: the parts of it used here are restated) comes in one call where torch gives one
// and its type and device are among those told apart here; its Python attributes take five: a fork of one prompt to four samples, 17 tensors, is the
// host's 13 us that way.
constexpr int MOST = 8;                         // sizes
struct Info {
  int type, device, dims;                       // type 0: none of ours; device -1: the host
  int64_t item;                                 // bytes of an element
  int64_t shape[MOST], stride[MOST];
  void* p;
};
struct DlTensor {
  void* data;
  struct { int32_t type, id; } device;
  int32_t ndim;
  struct { uint8_t code, bits; uint16_t lanes; } dtype;
  int64_t *shape, *strides;
  uint64_t byte_offset;
};
int dl_type(const DlTensor& t) {
  if (t.dtype.lanes != 1) return 0;
  switch (t.dtype.code << 8 | t.dtype.bits) {
    case 0 << 8 | 32: return I32;
    case 0 << 8 | 64: return I64;
    case 1 << 8 | 8: return U8;
    case 1 << 8 | 64: return U64;
    case 2 << 8 | 32: return F32;
    case 2 << 8 | 16: return F16;
    case 4 << 8 | 16: return BF16;
    case 6 << 8 | 8: return BOOL;
    case 10 << 8 | 8: return F8;               // 4 exponent bits, 3 mantissa bits, no infinities
    default: return 0;
  }
}
bool described(PyObject* x, Info& out) {
  if (!to_dlpack) return false;
  const Ref capsule(PyObject_CallOneArg(to_dlpack, x));
  const DlTensor* t = capsule.p && PyCapsule_IsValid(capsule.p, "dltensor") ? static_cast<DlTensor*>(PyCapsule_GetPointer(capsule.p, "dltensor")) : nullptr;
  if (!t) {
    PyErr_Clear();
    return false;
  }
  out.type = dl_type(*t);
  // 1: host, 2: CUDA; the types that are told apart here only (others ask the attribute)
  if (out.type == 0 || t->ndim > MOST || (t->device.type != 1 && t->device.type != 2) || (!t->strides && t->ndim > 0)) return false;
  out.device = t->device.type == 2 ? t->device.id : -1;
  out.dims = t->ndim;
  out.item = t->dtype.bits / 8;
  for (int i = 0; i < t->ndim; ++i) { out.shape[i] = t->shape[i]; out.stride[i] = t->strides[i]; }
  out.p = static_cast<char*>(t->data) + t->byte_offset;
  return true;
}
Info look(PyObject* x) {
  Info t = {};
  if (described(x, t)) return t;
  t.type = type_of(x);
  t.device = static_cast<int>(ask(x, n_get_device));
  t.dims = shape_of(x, t.shape);
  strides_of(x, t.stride);
  t.item = ask(x, n_element_size);
  t.p = data_of(x);
  return t;
}
// Dense in the order of its sizes, from size `from` on.
bool dense(const Info& t, int from = 0) {
  int64_t n = 1;
  for (int i = 0; i < t.dims && i < MOST; ++i)
    if (t.shape[i] == 0) return true;
  for (int i = (t.dims < MOST ? t.dims : MOST) - 1; i >= from; --i) {
    if (t.shape[i] != 1 && t.stride[i] != n) return false;
    n *= t.shape[i];
  }
  return t.dims <= MOST;
}

// Address of a contiguous tensor of one of the types on the device with these sizes (a size below 0: any).
template <int DIMS>
void* flat(PyObject* x, const char* name, int allowed, int device, const int64_t (&want)[DIMS], int64_t* last = nullptr, int64_t* first = nullptr) {
  const Info t = look(x);
  bool ok = (t.type & allowed) != 0 && t.device == device && t.dims == DIMS && dense(t);
  for (int i = 0; i < DIMS; ++i) ok = ok && (want[i] < 0 || t.shape[i] == want[i]);
  if (!ok) {
    const Ref shape(PyObject_GetAttr(x, n_shape)), type(PyObject_GetAttr(x, n_dtype));
    if (!shape.p || !type.p) throw Error{};
    char sizes[96] = "";
    for (int i = 0, at = 0; i < DIMS; ++i)
      at += want[i] < 0 ? std::snprintf(sizes + at, sizeof(sizes) - at, "%sany", i ? ", " : "")
                        : std::snprintf(sizes + at, sizeof(sizes) - at, "%s%lld", i ? ", " : "", static_cast<long long>(want[i]));
    const char* kind = allowed == I32 ? "int32" : allowed == F32 ? "float32" : allowed == U8 ? "uint8" : allowed == (U8 | BOOL) ? "uint8 or bool" : "int64 or uint64";
    PyErr_Format(PyExc_ValueError, "%s: expected a contiguous %s tensor of shape (%s) on cuda:%d, got %S %S on device %lld", name, kind, sizes,
                 device, type.p, shape.p, static_cast<long long>(ask(x, n_get_device)));
    throw Error{};
  }
  if (last) *last = t.shape[DIMS - 1];
  if (first) *first = t.shape[0];
  return t.p;
}
void* optional(PyObject* x, const char* name, int allowed, int device, int64_t n) {
  return x == Py_None ? nullptr : flat<1>(x, name, allowed, device, {n});
}

// A [rows, heads, head_dim] tensor whose heads and elements lie one behind the other.
struct Strided {
  int type, device;
  int64_t rows, heads, dim, stride;
  void* p;
};
Strided strided(PyObject* x, const char* name) {
  const Info f = look(x);
  const int64_t *s = f.shape, *st = f.stride;
  Strided t;
  t.type = f.type;
  t.device = f.device;
  if (!(t.type & (BF16 | F16)) || t.device < 0) refuse(name, "a bfloat16 or float16 tensor on a CUDA device");
  if (f.dims != 3) refuse(name, "[rows, heads, head_dim]");
  if ((s[2] > 1 && st[2] != 1) || (s[1] > 1 && st[1] != s[2])) refuse(name, "[rows, heads, head_dim] with dense heads");
  t.rows = s[0]; t.heads = s[1]; t.dim = s[2];
  t.stride = s[0] > 1 ? st[0] : s[1] * s[2];
  t.p = f.p;
  return t;
}
void same_kind(const Strided& t, const Strided& k, const char* name, const char* what) {
  if (t.type != k.type || t.device != k.device || t.dim != k.dim) refuse(name, what);
}

// The pools.  v: NULL where only K is read.
percache_kv_t pools(const Strided& k, PyObject* v, PyObject* page_table, PyObject* ctx_start, int64_t n_seqs) {
  percache_kv_t kv = {};
  if (k.heads > INT32_MAX || k.dim > INT32_MAX) refuse("k", "[slots, kv_heads, head_dim]");
  kv.k = k.p; kv.k_slot_stride = k.stride; kv.n_slots = k.rows;
  kv.n_kv_heads = static_cast<int32_t>(k.heads); kv.head_dim = static_cast<int32_t>(k.dim);
  kv.dtype = k.type == BF16 ? PERCACHE_BF16 : PERCACHE_F16;
  if (v) {
    const Strided t = strided(v, "v");
    same_kind(t, k, "v", "k's type, device and shape");
    if (t.rows != k.rows || t.heads != k.heads) refuse("v", "k's type, device and shape");
    kv.v = t.p; kv.v_slot_stride = t.stride;
  }
  if ((page_table == Py_None) == (ctx_start == Py_None)) {
    PyErr_SetString(PyExc_ValueError, "give either page_table or ctx_start");
    throw Error{};
  }
  if (page_table != Py_None) {
    int64_t width = 0;
    kv.page_table = static_cast<int32_t*>(flat<2>(page_table, "page_table", I32, k.device, {n_seqs, -1}, &width));
    if (width > INT32_MAX) refuse("page_table", "fewer entries a prompt");
    kv.page_table_stride = static_cast<int32_t>(width);
  } else {
    kv.ctx_start = static_cast<int32_t*>(flat<1>(ctx_start, "ctx_start", I32, k.device, {n_seqs}));
  }
  return kv;
}
int64_t length_of(PyObject* x, const char* name) {
  int64_t s[3];
  if (shape_of(x, s) != 1 || s[0] > INT32_MAX - 1) refuse(name, "one number a prompt");
  return s[0];
}
percache_rows_t batch(const Strided& q, const Strided& k, PyObject* ctx_len, PyObject* row_start, PyObject* mask, PyObject* max_nodes,
                      PyObject* max_len, int64_t n_seqs) {
  percache_rows_t r = {};
  same_kind(q, k, "q", "[rows, q_heads, head_dim] of k's type on k's device");
  if (q.rows > INT32_MAX || q.heads > INT32_MAX) refuse("q", "fewer rows or heads");
  r.n_seqs = static_cast<int32_t>(n_seqs); r.n_rows = static_cast<int32_t>(q.rows);
  r.max_nodes = int32(max_nodes, "max_nodes"); r.max_len = int32(max_len, "max_len");
  r.ctx_len = static_cast<int32_t*>(flat<1>(ctx_len, "ctx_len", I32, k.device, {n_seqs}));
  r.row_start = static_cast<int32_t*>(flat<1>(row_start, "row_start", I32, k.device, {n_seqs + 1}));
  if (mask != Py_None) {
    int64_t words = 0;
    r.mask = static_cast<uint64_t*>(flat<2>(mask, "mask", I64 | U64, k.device, {q.rows, -1}, &words));
    if (words > INT32_MAX) refuse("mask", "fewer words a row");
    r.mask_words = static_cast<int32_t>(words);
  }
  return r;
}
float scale_of(PyObject* scale, int64_t dim) { return scale == Py_None ? static_cast<float>(1.0 / std::sqrt(static_cast<double>(dim))) : number(scale); }
struct Space { void* p; int64_t bytes; };
Space workspace_of(PyObject* x, int device) {
  int64_t n = 0;
  void* p = flat<1>(x, "workspace", U8, device, {-1}, &n);
  return {p, n};
}

template <typename Fn>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, Fn fn) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return nullptr;
  }
  if (!f_tree) {
    PyErr_SetString(PyExc_RuntimeError, "bind() first");
    return nullptr;
  }
  try {
    return PyLong_FromLong(fn());
  } catch (const Error&) {
    return nullptr;
  }
}
template <typename Fn>
int released(Fn fn) {                           // other Python threads may run during the call
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = fn();
  Py_END_ALLOW_THREADS
  return rc;
}

// q k v out lse ctx_len row_start max_nodes max_len workspace mask page_table ctx_start scale stream
PyObject* tree_attention(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 15, [&] {
    const Strided q = strided(x[0], "q"), k = strided(x[1], "k"), out = strided(x[3], "out");
    const int64_t n_seqs = length_of(x[5], "ctx_len");
    const percache_kv_t kv = pools(k, x[2], x[11], x[12], n_seqs);
    const percache_rows_t rows = batch(q, k, x[5], x[6], x[10], x[7], x[8], n_seqs);
    same_kind(out, q, "out", "q's type, device and shape");
    if (out.rows != q.rows || out.heads != q.heads) refuse("out", "q's type, device and shape");
    float* lse = x[4] == Py_None ? nullptr : static_cast<float*>(flat<2>(x[4], "lse", F32, k.device, {q.rows, q.heads}));
    const Space ws = workspace_of(x[9], k.device);
    const float scale = scale_of(x[13], q.dim);
    void* stream = stream_of(x[14], k.device);
    return released([&] {
      return f_tree(k.device, stream, &kv, &rows, q.p, q.stride, static_cast<int32_t>(q.heads), scale, out.p, out.stride, lse, ws.p, ws.bytes);
    });
  });
}

// q k lse weights weights_out ctx_len row_start max_nodes max_len workspace mask use page_table ctx_start scale decay stream
PyObject* attention_weights(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 17, [&] {
    const Strided q = strided(x[0], "q"), k = strided(x[1], "k");
    const int64_t n_seqs = length_of(x[5], "ctx_len");
    const percache_kv_t kv = pools(k, nullptr, x[12], x[13], n_seqs);
    const percache_rows_t rows = batch(q, k, x[5], x[6], x[10], x[7], x[8], n_seqs);
    const float* lse = static_cast<float*>(flat<2>(x[2], "lse", F32, k.device, {q.rows, q.heads}));
    const uint8_t* use = static_cast<uint8_t*>(optional(x[11], "use", U8 | BOOL, k.device, q.rows));
    int64_t width = 0;
    float* w_out = static_cast<float*>(flat<3>(x[4], "weights_out", F32, k.device, {n_seqs, k.heads, -1}, &width));
    const float* w_in = x[3] == Py_None ? nullptr : static_cast<float*>(flat<3>(x[3], "weights", F32, k.device, {n_seqs, k.heads, width}));
    const Space ws = workspace_of(x[9], k.device);
    const float scale = scale_of(x[14], q.dim), decay = number(x[15]);
    void* stream = stream_of(x[16], k.device);
    return released([&] {
      return f_weights(k.device, stream, &kv, &rows, q.p, q.stride, static_cast<int32_t>(q.heads), scale, lse, use, decay, w_in, w_out, width,
                       ws.p, ws.bytes);
    });
  });
}

// weights length keep count sink recent max_len stream
PyObject* select_slots(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 8, [&] {
    const int device = static_cast<int>(ask(x[0], n_get_device));
    if (device < 0) refuse("weights", "a tensor on a CUDA device");
    int64_t s[3], budget = 0;
    if (shape_of(x[0], s) != 3 || s[0] > INT32_MAX || s[1] > INT32_MAX || s[2] > INT32_MAX) refuse("weights", "[prompts, heads, slots]");
    const float* w = static_cast<float*>(flat<3>(x[0], "weights", F32, device, {s[0], s[1], s[2]}));
    const int32_t* length = static_cast<int32_t*>(flat<1>(x[1], "length", I32, device, {s[0]}));
    int32_t* keep = static_cast<int32_t*>(flat<3>(x[2], "keep", I32, device, {s[0], s[1], -1}, &budget));
    int32_t* count = static_cast<int32_t*>(flat<1>(x[3], "count", I32, device, {s[0]}));
    if (budget > INT32_MAX) refuse("keep", "a smaller budget");
    const int32_t sink = int32(x[4], "sink"), recent = int32(x[5], "recent");
    const int32_t max_len = x[6] == Py_None ? static_cast<int32_t>(s[2]) : int32(x[6], "max_len");
    void* stream = stream_of(x[7], device);
    return released([&] {
      return f_select(device, stream, w, s[2], length, static_cast<int32_t>(s[0]), static_cast<int32_t>(s[1]), max_len,
                      static_cast<int32_t>(budget), sink, recent, keep, count);
    });
  });
}

// k v keep count max_len weights weights_out first page_table ctx_start dst_page_table dst_start stream
PyObject* compact_slots(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 13, [&] {
    if (x[5] == Py_None && x[6] != Py_None) refuse("weights_out", "weights beside it");
    const Strided k = strided(x[0], "k");
    const int64_t n_seqs = length_of(x[3], "count");
    const percache_kv_t kv = pools(k, x[1], x[8], x[9], n_seqs);
    int64_t s[3], width = 0, dst_width = 0;
    if (shape_of(x[2], s) != 3 || s[1] > INT32_MAX || s[2] > INT32_MAX) refuse("keep", "[prompts, heads or 1, budget]");
    const int32_t* keep = static_cast<int32_t*>(flat<3>(x[2], "keep", I32, k.device, {n_seqs, s[1], s[2]}));
    const int32_t* count = static_cast<int32_t*>(flat<1>(x[3], "count", I32, k.device, {n_seqs}));
    const int32_t max_len = int32(x[4], "max_len");
    const float* w_in = nullptr;
    float* w_out = nullptr;
    if (x[5] != Py_None) {
      w_in = static_cast<float*>(flat<3>(x[5], "weights", F32, k.device, {n_seqs, k.heads, -1}, &width));
      w_out = static_cast<float*>(flat<3>(x[6], "weights_out", F32, k.device, {n_seqs, k.heads, width}));
    }
    const int32_t* first = static_cast<int32_t*>(optional(x[7], "first", I32, k.device, n_seqs));
    const int32_t* table = x[10] == Py_None ? nullptr : static_cast<int32_t*>(flat<2>(x[10], "dst_page_table", I32, k.device, {n_seqs, -1}, &dst_width));
    if (dst_width > INT32_MAX) refuse("dst_page_table", "fewer entries a prompt");
    const int32_t* start = static_cast<int32_t*>(optional(x[11], "dst_start", I32, k.device, n_seqs));
    void* stream = stream_of(x[12], k.device);
    return released([&] {
      return f_compact(k.device, stream, &kv, static_cast<int32_t>(n_seqs), max_len, table, static_cast<int32_t>(dst_width), start, first, keep,
                       static_cast<int32_t>(s[1]), static_cast<int32_t>(s[2]), count, w_in, w_out, width);
    });
  });
}

// ---------------------------------------------------------------------------------------------------- pages
// 8-bit pages [pages, kv_heads, 2, 16, head_dim] with dense inner sizes, and their scales [pages, kv_heads, 2].
percache_kv8_t pages8(PyObject* pages, PyObject* scales, PyObject* page_table, int64_t n_seqs, int type, int device) {
  percache_kv8_t kv = {};
  const Info f = look(pages);
  const int64_t *s = f.shape, *st = f.stride;
  int64_t width = 0;
  if (!(f.type & (F8 | U8)) || f.device != device) refuse("pages", "a float8_e4m3fn or uint8 tensor on the rows' device");
  if (f.dims != 5 || s[2] != 2 || s[3] != 16 || s[1] > INT32_MAX || s[4] > INT32_MAX) refuse("pages", "[pages, kv_heads, 2, 16, head_dim]");
  if (st[4] != 1 || st[3] != s[4] || st[2] != 16 * s[4] || (s[1] > 1 && st[1] != 32 * s[4])) refuse("pages", "[pages, kv_heads, 2, 16, head_dim] with dense pages");
  kv.scales = static_cast<float*>(flat<3>(scales, "scales", F32, device, {s[0], s[1], 2}));
  kv.pages = f.p;
  kv.page_stride = s[0] > 1 ? st[0] : 32 * s[1] * s[4];
  kv.n_pages = s[0]; kv.n_kv_heads = static_cast<int32_t>(s[1]); kv.head_dim = static_cast<int32_t>(s[4]);
  kv.dtype = type == BF16 ? PERCACHE_BF16 : PERCACHE_F16;
  kv.page_table = static_cast<int32_t*>(flat<2>(page_table, "page_table", I32, device, {n_seqs, -1}, &width));
  if (width > INT32_MAX) refuse("page_table", "fewer entries a prompt");
  kv.page_table_stride = static_cast<int32_t>(width);
  return kv;
}

// q k v q_out ctx_len row_start max_len k_pool v_pool pages scales page_table ctx_start q_gain k_gain eps rope position stream
PyObject* append_rows(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 19, [&] {
    const Strided k = strided(x[1], "k"), v = strided(x[2], "v");
    same_kind(v, k, "v", "k's type, device and shape");
    if (v.rows != k.rows || v.heads != k.heads) refuse("v", "k's type, device and shape");
    if (k.rows > INT32_MAX || k.heads > INT32_MAX || k.dim > INT32_MAX) refuse("k", "fewer rows or heads");
    const int64_t n_seqs = length_of(x[4], "ctx_len");
    percache_new_rows_t r = {};
    r.n_seqs = static_cast<int32_t>(n_seqs); r.n_rows = static_cast<int32_t>(k.rows); r.max_len = int32(x[6], "max_len");
    r.ctx_len = static_cast<int32_t*>(flat<1>(x[4], "ctx_len", I32, k.device, {n_seqs}));
    r.row_start = static_cast<int32_t*>(flat<1>(x[5], "row_start", I32, k.device, {n_seqs + 1}));
    r.k = k.p; r.v = v.p; r.k_row_stride = k.stride; r.v_row_stride = v.stride;
    if ((x[0] == Py_None) != (x[3] == Py_None)) refuse("q_out", "q and q_out, or neither");
    if (x[0] != Py_None) {
      const Strided q = strided(x[0], "q"), o = strided(x[3], "q_out");
      same_kind(q, k, "q", "[rows, q_heads, head_dim] of k's type on k's device");
      same_kind(o, q, "q_out", "q's type, device and shape");
      if (q.rows != k.rows || q.heads > INT32_MAX) refuse("q", "as many rows as k");
      if (o.rows != q.rows || o.heads != q.heads) refuse("q_out", "q's type, device and shape");
      r.q = q.p; r.q_out = o.p; r.q_row_stride = q.stride; r.q_out_row_stride = o.stride; r.n_q_heads = static_cast<int32_t>(q.heads);
    }
    if (x[13] != Py_None) r.q_gain = static_cast<float*>(flat<1>(x[13], "q_gain", F32, k.device, {k.dim}));
    if (x[14] != Py_None) r.k_gain = static_cast<float*>(flat<1>(x[14], "k_gain", F32, k.device, {k.dim}));
    r.eps = number(x[15]);
    if (x[16] != Py_None) {
      int64_t positions = 0;
      r.rope = static_cast<float*>(flat<3>(x[16], "rope", F32, k.device, {-1, k.dim / 2, 2}, nullptr, &positions));
      if (positions > INT32_MAX) refuse("rope", "fewer positions");
      r.n_positions = static_cast<int32_t>(positions);
    }
    r.position = static_cast<int32_t*>(optional(x[17], "position", I32, k.device, k.rows));
    if ((x[7] == Py_None) == (x[9] == Py_None) || (x[7] == Py_None) != (x[8] == Py_None) || (x[9] == Py_None) != (x[10] == Py_None))
      refuse("pools", "either k_pool and v_pool or pages and scales");
    if (x[9] != Py_None) {
      if (x[12] != Py_None) refuse("ctx_start", "a page_table with 8-bit pages");
      const percache_kv8_t kv = pages8(x[9], x[10], x[11], n_seqs, k.type, k.device);
      if (kv.n_kv_heads != k.heads || kv.head_dim != k.dim) refuse("pages", "k's heads");
      void* stream = stream_of(x[18], k.device);
      return released([&] { return f_append8(k.device, stream, &kv, &r); });
    }
    const Strided pool = strided(x[7], "k_pool");
    same_kind(pool, k, "k_pool", "k's type, device and heads");
    if (pool.heads != k.heads) refuse("k_pool", "k's type, device and heads");
    const percache_kv_t kv = pools(pool, x[8], x[11], x[12], n_seqs);
    void* stream = stream_of(x[18], k.device);
    return released([&] { return f_append(k.device, stream, &kv, &r); });
  });
}

// q pages scales out lse ctx_len row_start max_nodes max_len workspace mask page_table scale stream
PyObject* tree_attention_8bit(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 14, [&] {
    const Strided q = strided(x[0], "q"), out = strided(x[3], "out");
    const int64_t n_seqs = length_of(x[5], "ctx_len");
    const percache_kv8_t kv = pages8(x[1], x[2], x[11], n_seqs, q.type, q.device);
    if (kv.head_dim != q.dim) refuse("q", "[rows, q_heads, head_dim] with the pages' head_dim");
    const percache_rows_t rows = batch(q, q, x[5], x[6], x[10], x[7], x[8], n_seqs);
    same_kind(out, q, "out", "q's type, device and shape");
    if (out.rows != q.rows || out.heads != q.heads) refuse("out", "q's type, device and shape");
    float* lse = x[4] == Py_None ? nullptr : static_cast<float*>(flat<2>(x[4], "lse", F32, q.device, {q.rows, q.heads}));
    const Space ws = workspace_of(x[9], q.device);
    const float scale = scale_of(x[12], q.dim);
    void* stream = stream_of(x[13], q.device);
    return released([&] {
      return f_tree8(q.device, stream, &kv, &rows, q.p, q.stride, static_cast<int32_t>(q.heads), scale, out.p, out.stride, lse, ws.p, ws.bytes);
    });
  });
}

// A pool [layers, pages, ...] whose pages are dense.
percache_pool_t pool_of(PyObject* x, int device, int64_t n_pages) {
  const Info f = look(x);
  const int64_t *s = f.shape, *st = f.stride;
  percache_pool_t p = {};
  if (f.device != device) refuse("pools", "tensors on the tables' device");
  if (f.dims < 2 || f.dims > MOST || s[1] != n_pages || s[0] < 1 || s[0] > INT32_MAX) refuse("pools", "[layers, pages, ...] with as many pages as refs");
  if (!dense(f, 2)) refuse("pools", "dense pages");
  int64_t page = 1;
  for (int i = 2; i < f.dims; ++i) page *= s[i];
  if ((s[0] > 1 && st[0] <= 0) || (s[1] > 1 && st[1] < page)) refuse("pools", "layers and pages that do not overlap");
  p.base = f.p;
  p.page_bytes = page * f.item;
  p.page_stride = s[1] > 1 ? st[1] * f.item : p.page_bytes;
  p.layer_stride = s[0] > 1 ? st[0] * f.item : 0;
  p.n_layers = static_cast<int32_t>(s[0]);
  return p;
}

// page_table held length parent table_out held_out length_out refs free_list free_count missing pools room refs_out free_list_out
// free_count_out workspace stream
PyObject* fork_pages(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 18, [&] {
    const int device = static_cast<int>(ask(x[0], n_get_device));
    if (device < 0) refuse("page_table", "a tensor on a CUDA device");
    percache_fork_t f = {};
    const int64_t n_seqs = length_of(x[1], "held"), n_children = length_of(x[3], "parent");
    int64_t width = 0, width_out = 0, n_pages = length_of(x[7], "refs");
    auto ints = [&](int i, const char* name, int64_t size) { return static_cast<int32_t*>(flat<1>(x[i], name, I32, device, {size})); };
    f.n_seqs = static_cast<int32_t>(n_seqs); f.n_children = static_cast<int32_t>(n_children);
    f.page_table = static_cast<int32_t*>(flat<2>(x[0], "page_table", I32, device, {n_seqs, -1}, &width));
    f.held = ints(1, "held", n_seqs); f.length = ints(2, "length", n_seqs); f.parent = ints(3, "parent", n_children);
    f.table_out = static_cast<int32_t*>(flat<2>(x[4], "table_out", I32, device, {n_children, -1}, &width_out));
    f.held_out = ints(5, "held_out", n_children); f.length_out = ints(6, "length_out", n_children);
    if (width > INT32_MAX || width_out > INT32_MAX) refuse("page_table", "fewer entries a sequence");
    f.page_table_stride = static_cast<int32_t>(width); f.table_out_stride = static_cast<int32_t>(width_out);
    f.n_pages = n_pages;
    f.refs = ints(7, "refs", n_pages); f.free_list = ints(8, "free_list", n_pages); f.free_count = ints(9, "free_count", 1);
    f.missing = ints(10, "missing", 1);
    f.refs_out = ints(13, "refs_out", n_pages); f.free_list_out = ints(14, "free_list_out", n_pages);
    f.free_count_out = ints(15, "free_count_out", 1);
    f.room = int32(x[12], "room");
    const Ref list(PySequence_Fast(x[11], "pools: expected a sequence of tensors"));
    if (!list.p) throw Error{};
    const Py_ssize_t n_pools = PySequence_Fast_GET_SIZE(list.p);
    if (n_pools > PERCACHE_MAX_POOLS) refuse("pools", "at most eight tensors");
    percache_pool_t pool[PERCACHE_MAX_POOLS];
    for (Py_ssize_t i = 0; i < n_pools; ++i) pool[i] = pool_of(PySequence_Fast_GET_ITEM(list.p, i), device, n_pages);
    f.pools = pool; f.n_pools = static_cast<int32_t>(n_pools);
    const Space ws = workspace_of(x[16], device);
    void* stream = stream_of(x[17], device);
    return released([&] { return f_fork(device, stream, &f, ws.p, ws.bytes); });
  });
}

// bind((addresses of the eight entry points), (torch's int32, float32, uint8, bool, int64, uint64, bfloat16, float16,
// float8_e4m3fn), device -> stream, tensor -> DLPack capsule or None)
PyObject* bind(PyObject*, PyObject* args) {
  unsigned long long f[8];
  PyObject *t[N_TYPES], *stream, *dlpack;
  if (!PyArg_ParseTuple(args, "(KKKKKKKK)(OOOOOOOOO)OO", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &f[6], &f[7], &t[0], &t[1], &t[2], &t[3],
                        &t[4], &t[5], &t[6], &t[7], &t[8], &stream, &dlpack))
    return nullptr;
  for (int i = 0; i < N_TYPES; ++i) {
    Py_INCREF(t[i]);
    Py_XSETREF(types[i], t[i]);
  }
  Py_INCREF(stream);
  Py_XSETREF(current_stream, stream);
  Py_XINCREF(dlpack == Py_None ? nullptr : dlpack);
  Py_XSETREF(to_dlpack, dlpack == Py_None ? nullptr : dlpack);
  f_tree = reinterpret_cast<decltype(f_tree)>(f[0]);
  f_weights = reinterpret_cast<decltype(f_weights)>(f[1]);
  f_select = reinterpret_cast<decltype(f_select)>(f[2]);
  f_compact = reinterpret_cast<decltype(f_compact)>(f[3]);
  f_append = reinterpret_cast<decltype(f_append)>(f[4]);
  f_append8 = reinterpret_cast<decltype(f_append8)>(f[5]);
  f_tree8 = reinterpret_cast<decltype(f_tree8)>(f[6]);
  f_fork = reinterpret_cast<decltype(f_fork)>(f[7]);
  Py_RETURN_NONE;
}

template <typename F>
PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }
PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         {"tree_attention", fast(tree_attention), METH_FASTCALL, nullptr},
                         {"attention_weights", fast(attention_weights), METH_FASTCALL, nullptr},
                         {"select_slots", fast(select_slots), METH_FASTCALL, nullptr},
                         {"compact_slots", fast(compact_slots), METH_FASTCALL, nullptr},
                         {"append_rows", fast(append_rows), METH_FASTCALL, nullptr},
                         {"tree_attention_8bit", fast(tree_attention_8bit), METH_FASTCALL, nullptr},
                         {"fork_pages", fast(fork_pages), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops_binding", "Checked calls of the cache operators.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops_binding() {
  n_dtype = PyUnicode_InternFromString("dtype");
  n_shape = PyUnicode_InternFromString("shape");
  n_get_device = PyUnicode_InternFromString("get_device");
  n_stride = PyUnicode_InternFromString("stride");
  n_data_ptr = PyUnicode_InternFromString("data_ptr");
  n_element_size = PyUnicode_InternFromString("element_size");
  if (!n_element_size || !n_dtype || !n_shape || !n_get_device || !n_stride || !n_data_ptr) return nullptr;
  return PyModule_Create(&module);
}
