// Python binding of the entry points that a training loop calls every step (include/qsgd.h): argument
// marshalling only. A call hands over up to two dozen tensors; taking their addresses, the current
// stream and the scalars here instead of through ctypes is what keeps the host ahead of the GPU on
// small gradients (one fixed-width encode of 4096 coordinates: 10.7 us of host time through ctypes,
// of which the launch itself is about 3; sixteen-message decode: 18.5 us).
//
// Every function takes positional arguments in the order of the C call, with tensors for pointers and a
// stream object or None last, and returns the C call's status. Arguments that must be contiguous CUDA
// tensors and are not raise the package's own exception, handed over once by set_error.
#include <Python.h>

#include <cmath>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/qsgd.h"

namespace {

PyObject* g_error = nullptr;      // QsgdError

struct Fail {};                   // a Python exception is set

const at::Tensor& cuda_tensor(PyObject* o, const char* name) {
  if (THPVariable_Check(o)) {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.is_cuda() && t.is_contiguous()) return t;
  }
  PyErr_Format(g_error ? g_error : PyExc_RuntimeError, "%s must be a contiguous CUDA tensor", name);
  throw Fail{};
}

PyObject* g_ctypes_number = nullptr;   // ctypes' c_uint64, c_float and the like

// A number, also one of ctypes' own.
struct Number {
  PyObject* o;
  explicit Number(PyObject* v) : o(Py_NewRef(v)) {
    if (PyIndex_Check(v) || PyFloat_Check(v)) return;
    const int mine = g_ctypes_number ? PyObject_IsInstance(v, g_ctypes_number) : 0;
    if (mine) Py_SETREF(o, mine > 0 ? PyObject_GetAttrString(v, "value") : nullptr);
    if (!o) throw Fail{};
  }
  Number(const Number&) = delete;
  ~Number() { Py_XDECREF(o); }
};

uint64_t u64(PyObject* v) {
  const Number n(v);
  const unsigned long long u = PyLong_AsUnsignedLongLongMask(n.o);
  if (u == ~0ull && PyErr_Occurred()) throw Fail{};
  return u;
}
uint32_t u32(PyObject* o) { return static_cast<uint32_t>(u64(o)); }
int i32(PyObject* o) { return static_cast<int>(u64(o)); }

float f32(PyObject* o) {
  const Number n(o);
  const double v = PyFloat_AsDouble(n.o);
  if (v == -1.0 && PyErr_Occurred()) throw Fail{};
  return static_cast<float>(v);
}

// Where a tensor, or whatever else has a data_ptr(), lies.
void* data_of(PyObject* o) {
  if (THPVariable_Check(o)) return THPVariable_Unpack(o).data_ptr();
  PyObject* p = PyObject_CallMethod(o, "data_ptr", nullptr);
  if (!p) throw Fail{};
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(p);
  Py_DECREF(p);
  if (v == ~0ull && PyErr_Occurred()) throw Fail{};
  return reinterpret_cast<void*>(v);
}
void* data_or_null(PyObject* o) { return o == Py_None ? nullptr : data_of(o); }

// The same, or a raw device address given as an integer.
void* address(PyObject* o) {
  return !THPVariable_Check(o) && PyIndex_Check(o) ? reinterpret_cast<void*>(u64(o)) : data_of(o);
}

qsgd_stream_t stream_of(PyObject* o) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
  PyObject* v = PyObject_GetAttrString(o, "cuda_stream");
  if (!v) throw Fail{};
  if (v == Py_None) { Py_DECREF(v); return nullptr; }
  const unsigned long long s = PyLong_AsUnsignedLongLongMask(v);
  Py_DECREF(v);
  if (s == ~0ull && PyErr_Occurred()) throw Fail{};
  return reinterpret_cast<qsgd_stream_t>(s);
}

// The K addresses of a sequence. More than the library takes are counted but not stored: the C call
// refuses them by their number before it looks at any.
struct Peers {
  void* p[QSGD_MAX_PEERS] = {};
  uint32_t K = 0;
  bool given = false;
  template <typename T> const T* const* as() const { return given ? reinterpret_cast<const T* const*>(p) : nullptr; }
};

struct Sequence {                 // borrowed items of a list or tuple (or of a copy of any other sequence)
  PyObject* fast = nullptr;
  explicit Sequence(PyObject* o) {
    // what has no length (a generator) could be gone through only once
    if (PyObject_Size(o) >= 0) fast = PySequence_Fast(o, "a sequence is required");
    if (!fast) throw Fail{};
  }
  ~Sequence() { Py_DECREF(fast); }
  uint32_t size() const { return static_cast<uint32_t>(PySequence_Fast_GET_SIZE(fast)); }
  PyObject* operator[](uint32_t i) const { return PySequence_Fast_GET_ITEM(fast, i); }
};

void peers(PyObject* o, Peers* out) {
  if (o == Py_None) return;                       // the library says where that is allowed
  const Sequence s(o);
  out->given = true;
  out->K = s.size();
  for (uint32_t k = 0; k < out->K && k < QSGD_MAX_PEERS; ++k) out->p[k] = address(s[k]);
}

// Fewer tables or byte counts than messages: what is missing would read as "none given", and the payload's bound
// would be gone. (Fixed-width messages have neither: nothing is looked at.)
void at_least(uint32_t have, const Peers& msgs, int code, const char* name) {
  if (have >= msgs.K || (code != QSGD_CODE_ELIAS && code != QSGD_CODE_ELIAS_DENSE)) return;
  PyErr_Format(g_error ? g_error : PyExc_RuntimeError, "%u %s given for %u messages", have, name, msgs.K);
  throw Fail{};
}

// Byte counts of the messages: the given list, or (sizes_of_msgs) the sizes of the message tensors.
const uint64_t* byte_counts(PyObject* o, PyObject* msgs, const Peers& read, int code, bool sizes_of_msgs, uint64_t* out) {
  if (o == Py_None && !sizes_of_msgs) return nullptr;
  const Sequence s(o == Py_None ? msgs : o);
  at_least(s.size(), read, code, "byte counts");
  for (uint32_t k = 0; k < s.size() && k < QSGD_MAX_PEERS; ++k) {
    if (o != Py_None) {
      PyObject* v = PyNumber_Long(s[k]);
      if (!v) throw Fail{};
      out[k] = PyLong_AsUnsignedLongLongMask(v);
      Py_DECREF(v);
    } else if (THPVariable_Check(s[k])) {
      out[k] = THPVariable_Unpack(s[k]).nbytes();
    } else {
      PyErr_SetString(g_error ? g_error : PyExc_RuntimeError, "msg_bytes is required for messages given by address");
      throw Fail{};
    }
  }
  return out;
}

// Runs a C call with the interpreter lock released: a launch may block when the stream's queue is full.
template <typename F>
PyObject* unlocked(F&& call) {
  PyThreadState* save = PyEval_SaveThread();
  const int st = call();
  PyEval_RestoreThread(save);
  return PyLong_FromLong(st);
}

#define QSGD_ARGS(count)                                                                     \
  if (nargs != (count)) {                                                                    \
    PyErr_Format(PyExc_TypeError, "%s takes %d arguments, %zd given", __func__, (count), nargs); \
    return nullptr;                                                                          \
  }
#define QSGD_TRY try {
#define QSGD_CATCH                                                            \
  } catch (const Fail&) {                                                     \
    return nullptr;                                                           \
  } catch (const std::exception& e) {                                         \
    PyErr_SetString(PyExc_RuntimeError, e.what());                            \
    return nullptr;                                                           \
  }

// encode(g, n or None, bucket, s, norm, code, seed, step, worker, out, out_bits, workspace, status, stream)
PyObject* encode(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  QSGD_ARGS(14)
  QSGD_TRY
  void* ws = data_or_null(a[11]);
  const at::Tensor& g = cuda_tensor(a[0], "g");
  const at::Tensor& out = cuda_tensor(a[9], "out");
  const at::Tensor& info = cuda_tensor(a[10], "out_bits");
  const at::Tensor& status = cuda_tensor(a[12], "status_dev");
  const uint64_t n = a[1] == Py_None ? static_cast<uint64_t>(g.numel()) : u64(a[1]);
  const uint32_t bucket = u32(a[2]), s = u32(a[3]), step = u32(a[7]), worker = u32(a[8]);
  const int norm = i32(a[4]), code = i32(a[5]);
  const uint64_t seed = u64(a[6]);
  const qsgd_stream_t stream = stream_of(a[13]);
  return unlocked([&] {
    return qsgd_encode(static_cast<const float*>(g.data_ptr()), n, bucket, s, norm, code, seed, step, worker,
                       out.data_ptr(), out.nbytes(), static_cast<uint64_t*>(info.data_ptr()), ws,
                       static_cast<uint32_t*>(status.data_ptr()), stream);
  });
  QSGD_CATCH
}

// encode_static(g, bucket, s, norm, code, seed, step, worker, out, out_bits, status, stream)
PyObject* encode_static(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  QSGD_ARGS(12)
  QSGD_TRY
  const at::Tensor& g = cuda_tensor(a[0], "g");
  const at::Tensor& out = cuda_tensor(a[8], "out");
  const at::Tensor& info = cuda_tensor(a[9], "out_bits");
  const at::Tensor& status = cuda_tensor(a[10], "status_dev");
  const uint32_t bucket = u32(a[1]), s = u32(a[2]), step = u32(a[6]), worker = u32(a[7]);
  const int norm = i32(a[3]), code = i32(a[4]);
  const uint64_t seed = u64(a[5]);
  const qsgd_stream_t stream = stream_of(a[11]);
  return unlocked([&] {
    return qsgd_encode_elias_static(static_cast<const float*>(g.data_ptr()), static_cast<uint64_t>(g.numel()), bucket,
                                    s, norm, code, seed, step, worker, out.data_ptr(), out.nbytes(),
                                    static_cast<uint64_t*>(info.data_ptr()),
                                    static_cast<uint32_t*>(status.data_ptr()), stream);
  });
  QSGD_CATCH
}

// policy_encode(g, address of a qsgd_policy, bucket, s, norm, code, seed, step, worker, out, out_bits,
//               workspace, status, stream)
PyObject* policy_encode(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  QSGD_ARGS(14)
  QSGD_TRY
  void* ws = data_or_null(a[11]);
  const at::Tensor& g = cuda_tensor(a[0], "g");
  const at::Tensor& out = cuda_tensor(a[9], "out");
  const at::Tensor& info = cuda_tensor(a[10], "out_bits");
  const at::Tensor& status = cuda_tensor(a[12], "status_dev");
  const qsgd_policy* plan = static_cast<const qsgd_policy*>(address(a[1]));
  const uint32_t bucket = u32(a[2]), s = u32(a[3]), step = u32(a[7]), worker = u32(a[8]);
  const int norm = i32(a[4]), code = i32(a[5]);
  const uint64_t seed = u64(a[6]);
  const qsgd_stream_t stream = stream_of(a[13]);
  return unlocked([&] {
    return qsgd_policy_encode(static_cast<const float*>(g.data_ptr()), plan, bucket, s, norm, code, seed, step, worker,
                              out.data_ptr(), out.nbytes(), static_cast<uint64_t*>(info.data_ptr()), ws,
                              static_cast<uint32_t*>(status.data_ptr()), stream);
  });
  QSGD_CATCH
}

// decode(packed, msgs, tables or infos, bytes, n, bucket, s, code, out, eta or None, status, stream):
// eta None: the sum into `out`; else the step on `out`
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  QSGD_ARGS(12)
  QSGD_TRY
  const bool packed = a[0] == Py_True, fused = a[9] != Py_None;
  uint32_t* status = static_cast<uint32_t*>(data_of(a[10]));
  Peers msgs, tables;
  uint64_t count[QSGD_MAX_PEERS] = {};
  peers(a[1], &msgs);
  peers(a[2], &tables);
  const int code = i32(a[7]);
  if (tables.given) at_least(tables.K, msgs, code, packed ? "info words" : "tables");
  const uint64_t* bytes = byte_counts(a[3], a[1], msgs, code, packed, count);
  const uint64_t n = u64(a[4]);
  const uint32_t bucket = u32(a[5]), s = u32(a[6]);
  const float eta = fused ? f32(a[9]) : 0.f;
  float* out = static_cast<float*>(cuda_tensor(a[8], fused ? "x" : "acc").data_ptr());
  const qsgd_stream_t stream = stream_of(a[11]);
  const void* const* mp = msgs.as<void>();
  const uint64_t* const* tp = tables.as<uint64_t>();
  return unlocked([&] {
    if (fused)
      return (packed ? qsgd_decode_sgd_step_packed : qsgd_decode_sgd_step)(mp, tp, bytes, msgs.K, n, bucket, s, code,
                                                                             out, eta, status, stream);
    return (packed ? qsgd_decode_accumulate_packed : qsgd_decode_accumulate)(mp, tp, bytes, msgs.K, n, bucket, s, code,
                                                                               out, status, stream);
  });
  QSGD_CATCH
}

// policy_decode(msgs, tables, bytes, address of a qsgd_policy, bucket, s, code, out, eta or None, status, stream)
PyObject* policy_decode(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  QSGD_ARGS(11)
  QSGD_TRY
  const bool fused = a[8] != Py_None;
  uint32_t* status = static_cast<uint32_t*>(data_of(a[9]));
  Peers msgs, tables;
  uint64_t count[QSGD_MAX_PEERS] = {};
  peers(a[0], &msgs);
  peers(a[1], &tables);
  const qsgd_policy* plan = static_cast<const qsgd_policy*>(address(a[3]));
  const uint32_t bucket = u32(a[4]), s = u32(a[5]);
  const int code = i32(a[6]), lists = plan && !plan->n_buckets ? QSGD_CODE_FIXED : code;      // raw tensors alone: no tables
  if (tables.given) at_least(tables.K, msgs, lists, "tables");
  const uint64_t* bytes = byte_counts(a[2], a[0], msgs, lists, false, count);
  const float eta = fused ? f32(a[8]) : 0.f;
  float* out = static_cast<float*>(cuda_tensor(a[7], fused ? "x" : "acc").data_ptr());
  const qsgd_stream_t stream = stream_of(a[10]);
  const void* const* mp = msgs.as<void>();
  const uint64_t* const* tp = tables.as<uint64_t>();
  return unlocked([&] {
    return fused ? qsgd_policy_decode_sgd_step(mp, tp, bytes, msgs.K, plan, bucket, s, code, out, eta, status, stream)
                 : qsgd_policy_decode_accumulate(mp, tp, bytes, msgs.K, plan, bucket, s, code, out, status, stream);
  });
  QSGD_CATCH
}

// sgd_step(x, acc, eta, K, stream)
PyObject* sgd_step(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  QSGD_ARGS(5)
  QSGD_TRY
  const at::Tensor& x = cuda_tensor(a[0], "x");
  const at::Tensor& acc = cuda_tensor(a[1], "acc");
  const float eta = f32(a[2]);
  const uint32_t K = u32(a[3]);
  const qsgd_stream_t stream = stream_of(a[4]);
  return unlocked([&] {
    return qsgd_sgd_step(static_cast<float*>(x.data_ptr()), static_cast<const float*>(acc.data_ptr()), eta, K,
                         static_cast<uint64_t>(x.numel()), stream);
  });
  QSGD_CATCH
}

// ---- few-bit values outside the gradient exchange ---------------------------------------------------
// These calls take strided tensors, several to a call, so what each must be is checked here by one rule.

[[noreturn]] void refuse(const char* format, const char* name, long long a = 0, long long b = 0) {
  PyErr_Format(g_error ? g_error : PyExc_RuntimeError, format, name, a, b);
  throw Fail{};
}

// A CUDA tensor of a type and number of dimensions, on the device of the others; the last dimension contiguous.
const at::Tensor& strided(PyObject* o, const char* name, c10::ScalarType type, int64_t dims, c10::Device device) {
  if (!THPVariable_Check(o)) refuse("%s must be a CUDA tensor", name);
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) refuse("%s must be a CUDA tensor", name);
  if (t.device() != device) refuse("%s is on another device than the call's first tensor", name);
  if (t.scalar_type() != type) refuse("%s has another element type than the call takes", name);
  if (t.dim() != dims) refuse("%s must have %lld dimensions", name, dims);
  if (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1) refuse("%s must be contiguous along its last dimension", name);
  return t;
}
const at::Tensor& whole(PyObject* o, const char* name, c10::ScalarType type, int64_t dims, c10::Device device) {
  const at::Tensor& t = strided(o, name, type, dims, device);
  if (!t.is_contiguous()) refuse("%s must be contiguous", name);
  return t;
}
void sized(const at::Tensor& t, const char* name, int64_t dim, int64_t size) {
  if (t.size(dim) != size) refuse("%s must have the size %lld in dimension %lld", name, size, dim);
}
uint64_t stride_of(const at::Tensor& t, int64_t dim) { return t.size(dim) > 1 ? static_cast<uint64_t>(t.stride(dim)) : 0u; }

c10::Device device_of(PyObject* o, const char* name) {
  if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda()) refuse("%s must be a CUDA tensor", name);
  return THPVariable_Unpack(o).device();
}

// The given stream, or the current one of the tensors' device.
qsgd_stream_t stream_on(PyObject* o, c10::Device device) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream(device.index()).stream();
  PyObject* index = PyObject_GetAttrString(o, "device_index");
  if (index) {
    const long long at = PyLong_AsLongLong(index);
    Py_DECREF(index);
    if (at == -1 && PyErr_Occurred()) throw Fail{};
    if (at != device.index()) refuse("%s is on another device than the tensors", "stream");
  } else {
    PyErr_Clear();                                    // a bare holder of a cuda_stream
  }
  return stream_of(o);
}

int type_code(c10::ScalarType t, const char* name) {
  switch (t) {
    case at::kFloat: return QSGD_TYPE_F32;
    case at::kHalf: return QSGD_TYPE_F16;
    case at::kBFloat16: return QSGD_TYPE_BF16;
    default: refuse("%s must hold float32, float16 or bfloat16", name);
  }
}

// What the calls on a cache share: (address of a qsgd_cache, its data, table, lengths, starts or None).
struct CacheCall {
  const qsgd_cache* cache;
  qsgd_cache_rows rows{};
  c10::Device device;
  c10::ScalarType type;
  CacheCall(PyObject* const* a) : cache(static_cast<const qsgd_cache*>(address(a[0]))), device(device_of(a[1], "the cache's data")) {
    type = cache->type == QSGD_TYPE_F16 ? at::kHalf : at::kBFloat16;
    const at::Tensor& table = strided(a[2], "table", at::kInt, 2, device);
    const at::Tensor& lengths = whole(a[3], "lengths", at::kInt, 1, device);
    sized(table, "table", 0, lengths.size(0));
    rows.table = table.const_data_ptr<int32_t>();
    rows.table_stride = stride_of(table, 0);
    if (table.size(1) > 0x7fffffff || lengths.size(0) > 0x7fffffff) refuse("%s is too large", "table");
    rows.table_pages = static_cast<uint32_t>(table.size(1));
    rows.sequences = static_cast<uint32_t>(lengths.size(0));
    rows.lengths = lengths.const_data_ptr<int32_t>();
    if (a[4] != Py_None) {
      const at::Tensor& starts = whole(a[4], "starts", at::kInt, 1, device);
      sized(starts, "starts", 0, lengths.size(0) + 1);
      rows.starts = starts.const_data_ptr<int32_t>();
    }
  }
  const at::Tensor& dense(PyObject* o, const char* name, int64_t heads, bool first) {
    const at::Tensor& t = strided(o, name, type, 3, device);
    if (first) rows.rows = static_cast<uint64_t>(t.size(0));
    sized(t, name, 0, static_cast<int64_t>(rows.rows));
    if (heads) sized(t, name, 1, heads);
    sized(t, name, 2, cache->head_dim);
    return t;
  }
  uint32_t* status(PyObject* o) const { return static_cast<uint32_t*>(whole(o, "status_dev", at::kInt, 1, device).data_ptr()); }
};

// cache_store(write, cache, data, table, lengths, starts or None, k, v, status, stream)
PyObject* cache_store(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  QSGD_ARGS(10)
  QSGD_TRY
  CacheCall c(a + 1);
  const at::Tensor& k = c.dense(a[6], "k", c.cache->heads, true);
  const at::Tensor& v = c.dense(a[7], "v", c.cache->heads, false);
  uint32_t* status = c.status(a[8]);
  const qsgd_stream_t stream = stream_on(a[9], c.device);
  const bool write = a[0] == Py_True;
  const c10::cuda::CUDAGuard guard(c.device);
  return unlocked([&] {
    return write ? qsgd_cache_write(c.cache, &c.rows, k.const_data_ptr(), stride_of(k, 0), stride_of(k, 1), v.const_data_ptr(),
                                    stride_of(v, 0), stride_of(v, 1), status, stream)
                 : qsgd_cache_read(c.cache, &c.rows, k.data_ptr(), stride_of(k, 0), stride_of(k, 1), v.data_ptr(), stride_of(v, 0),
                                   stride_of(v, 1), status, stream);
  });
  QSGD_CATCH
}

// cache_attend(cache, data, table, lengths, starts or None, q, out, workspace, status, scale or None, lse or None, stream)
PyObject* cache_attend(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  QSGD_ARGS(12)
  QSGD_TRY
  CacheCall c(a);
  const at::Tensor& q = c.dense(a[5], "q", 0, true);
  const int64_t heads = q.size(1);
  const size_t need = heads > 0 && heads <= 0x7fffffff ? qsgd_cache_attend_workspace_bytes(c.cache, static_cast<uint32_t>(heads)) : 0;
  if (need == 0) refuse("%s must have a multiple of the cache's %lld heads", "q", c.cache->heads);
  const at::Tensor& out = c.dense(a[6], "out", heads, false);
  const at::Tensor& ws = whole(a[7], "workspace", at::kByte, 1, c.device);
  if (ws.nbytes() < need) refuse("%s must have %lld bytes", "workspace", static_cast<long long>(need));
  float* lse = nullptr;
  if (a[10] != Py_None) {
    const at::Tensor& t = whole(a[10], "lse", at::kFloat, 2, c.device);
    sized(t, "lse", 0, q.size(0));
    sized(t, "lse", 1, heads);
    lse = t.data_ptr<float>();
  }
  const float scale = a[9] == Py_None ? 1.0f / std::sqrt(static_cast<float>(c.cache->head_dim)) : f32(a[9]);
  uint32_t* status = c.status(a[8]);
  const qsgd_stream_t stream = stream_on(a[11], c.device);
  const c10::cuda::CUDAGuard guard(c.device);
  return unlocked([&] {
    return qsgd_cache_attend(c.cache, &c.rows, q.const_data_ptr(), stride_of(q, 0), stride_of(q, 1), static_cast<uint32_t>(heads), scale,
                             out.data_ptr(), stride_of(out, 0), stride_of(out, 1), lse, ws.data_ptr(), status, stream);
  });
  QSGD_CATCH
}

// quantize_rows(x, codes, scale, stream)
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  QSGD_ARGS(4)
  QSGD_TRY
  const c10::Device device = device_of(a[0], "x");
  const c10::ScalarType kind = THPVariable_Unpack(a[0]).scalar_type();
  const int type = type_code(kind, "x");
  const at::Tensor& x = strided(a[0], "x", kind, 2, device);
  const at::Tensor& codes = strided(a[1], "codes", at::kChar, 2, device);
  const at::Tensor& scale = whole(a[2], "scale", at::kFloat, 1, device);
  sized(codes, "codes", 0, x.size(0));
  sized(codes, "codes", 1, x.size(1));
  sized(scale, "scale", 0, x.size(0));
  if (x.size(1) > 0x7fffffff) refuse("%s has too many columns", "x");
  const qsgd_stream_t stream = stream_on(a[3], device);
  const c10::cuda::CUDAGuard guard(device);
  return unlocked([&] {
    return qsgd_quantize_rows(x.const_data_ptr(), static_cast<uint64_t>(x.size(0)), static_cast<uint32_t>(x.size(1)), stride_of(x, 0), type,
                              codes.data_ptr<int8_t>(), stride_of(codes, 0), scale.data_ptr<float>(), stream);
  });
  QSGD_CATCH
}

// What the two products share: b, its scales, bias, and the output of m rows.
struct ProductCall {
  const at::Tensor& b;
  const at::Tensor& scale;
  const at::Tensor& out;
  const float* bias = nullptr;
  int type;
  ProductCall(PyObject* ob, PyObject* os, PyObject* oo, PyObject* obias, const at::Tensor& a, const char* name, const char* scale_name,
              c10::Device device)
      : b(strided(ob, name, at::kChar, 2, device)), scale(whole(os, scale_name, at::kFloat, 1, device)),
        out(strided(oo, "out", THPVariable_Check(oo) ? THPVariable_Unpack(oo).scalar_type() : at::kFloat, 2, device)),
        type(type_code(out.scalar_type(), "out")) {
    sized(b, name, 1, a.size(1));
    sized(scale, scale_name, 0, b.size(0));
    sized(out, "out", 0, a.size(0));
    sized(out, "out", 1, b.size(0));
    if (obias != Py_None) {
      const at::Tensor& t = whole(obias, "bias", at::kFloat, 1, device);
      sized(t, "bias", 0, b.size(0));
      bias = t.const_data_ptr<float>();
    }
    if (a.size(1) > 0x7fffffff) refuse("%s has too many columns", name);
  }
};

// matmul_i8(a, a_scale, b, b_scale, out, bias or None, status or None, stream)
PyObject* matmul_i8(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  QSGD_ARGS(8)
  QSGD_TRY
  const c10::Device device = device_of(a[0], "a");
  const at::Tensor& x = strided(a[0], "a", at::kChar, 2, device);
  const at::Tensor& x_scale = whole(a[1], "a_scale", at::kFloat, 1, device);
  sized(x_scale, "a_scale", 0, x.size(0));
  const ProductCall c(a[2], a[3], a[4], a[5], x, "b", "b_scale", device);
  uint32_t* status = a[6] == Py_None ? nullptr : static_cast<uint32_t*>(whole(a[6], "status_dev", at::kInt, 1, device).data_ptr());
  const qsgd_stream_t stream = stream_on(a[7], device);
  const c10::cuda::CUDAGuard guard(device);
  return unlocked([&] {
    return qsgd_matmul_i8(x.const_data_ptr<int8_t>(), stride_of(x, 0), x_scale.const_data_ptr<float>(), c.b.const_data_ptr<int8_t>(),
                          stride_of(c.b, 0), c.scale.const_data_ptr<float>(), c.bias, static_cast<uint64_t>(x.size(0)),
                          static_cast<uint64_t>(c.b.size(0)), static_cast<uint32_t>(x.size(1)), c.out.data_ptr(), stride_of(c.out, 0), c.type,
                          status, stream);
  });
  QSGD_CATCH
}

// linear_i8(x, w, w_scale, out, workspace, bias or None, status or None, stream)
PyObject* linear_i8(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  QSGD_ARGS(8)
  QSGD_TRY
  const c10::Device device = device_of(a[0], "x");
  const c10::ScalarType kind = THPVariable_Unpack(a[0]).scalar_type();
  const int x_type = type_code(kind, "x");
  const at::Tensor& x = strided(a[0], "x", kind, 2, device);
  const ProductCall c(a[1], a[2], a[3], a[5], x, "w", "w_scale", device);
  const at::Tensor& ws = whole(a[4], "workspace", at::kByte, 1, device);
  const size_t need = qsgd_linear_i8_workspace_bytes(static_cast<uint64_t>(x.size(0)), static_cast<uint32_t>(x.size(1)));
  if (ws.nbytes() < need) refuse("%s must have %lld bytes", "workspace", static_cast<long long>(need));
  uint32_t* status = a[6] == Py_None ? nullptr : static_cast<uint32_t*>(whole(a[6], "status_dev", at::kInt, 1, device).data_ptr());
  const qsgd_stream_t stream = stream_on(a[7], device);
  const c10::cuda::CUDAGuard guard(device);
  return unlocked([&] {
    return qsgd_linear_i8(x.const_data_ptr(), stride_of(x, 0), x_type, c.b.const_data_ptr<int8_t>(), stride_of(c.b, 0),
                          c.scale.const_data_ptr<float>(), c.bias, static_cast<uint64_t>(x.size(0)), static_cast<uint64_t>(c.b.size(0)),
                          static_cast<uint32_t>(x.size(1)), c.out.data_ptr(), stride_of(c.out, 0), c.type, ws.data_ptr(), status,
                          stream);
  });
  QSGD_CATCH
}

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_XINCREF(cls);
  Py_XSETREF(g_error, cls);
  Py_RETURN_NONE;
}

#define QSGD_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {QSGD_FAST(encode),        QSGD_FAST(encode_static), QSGD_FAST(policy_encode),
                          QSGD_FAST(decode),        QSGD_FAST(policy_decode), QSGD_FAST(sgd_step),
                          QSGD_FAST(cache_store),   QSGD_FAST(cache_attend),  QSGD_FAST(quantize_rows),
                          QSGD_FAST(matmul_i8),     QSGD_FAST(linear_i8),
                          {"set_error", set_error, METH_O, nullptr},          {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_qsgd_native", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__qsgd_native(void) {
  PyObject* ctypes = PyImport_ImportModule("_ctypes");
  if (!ctypes) return nullptr;
  g_ctypes_number = PyObject_GetAttrString(ctypes, "_SimpleCData");
  Py_DECREF(ctypes);
  return g_ctypes_number ? PyModule_Create(&kModule) : nullptr;
}
