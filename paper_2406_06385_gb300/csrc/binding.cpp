// The short way from Python into the library, for the calls of a serving step: a function here looks at the arguments of
// the binding's function of the same name (lrqat.py) and, where it finds every one of them in order and on the current
// device, makes the call.  For anything else it returns None, and the binding goes through its own checks, which say what
// is wrong; so nothing is accepted here that is not accepted there.  What the interpreter takes to look at a dozen tensors'
// types, devices and strides was most of the host's share: a call for two samples behind a prefix, with its cache and batch
// structures, two outputs and the sizes, 29.4 -> 16.8 us, of which 3.9 are the call and its two launches and the most
// allocations; a head rotation of 48 tokens 17.6 -> 12.5, blocks for 48 tokens 30.7 -> 23.4 (both sides on one machine; on
// others 17 to 22, 12 to 14 and 23 to 25 us).
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "lrqat.h"

namespace {

// Thrown where a call is not for the short way.
struct NotHere {};
inline void need(bool ok) {
  if (!ok) throw NotHere{};
}

PyObject* g_device = nullptr;   // "device"

// The binding's ctypes class of a C structure (see `structures`).
template <typename T>
PyTypeObject* g_class = nullptr;

// The C structure behind one of the binding's ctypes structures; other bytes of its size are not one.
template <typename T>
class Struct {
 public:
  explicit Struct(PyObject* o) {
    need(g_class<T> && PyObject_TypeCheck(o, g_class<T>));
    if (PyObject_GetBuffer(o, &b_, PyBUF_SIMPLE) != 0) {
      PyErr_Clear();
      throw NotHere{};
    }
    if (b_.len != static_cast<Py_ssize_t>(sizeof(T))) {
      PyBuffer_Release(&b_);
      throw NotHere{};
    }
  }
  ~Struct() { PyBuffer_Release(&b_); }
  Struct(const Struct&) = delete;
  Struct& operator=(const Struct&) = delete;
  T* operator->() const { return static_cast<T*>(b_.buf); }
  T* get() const { return static_cast<T*>(b_.buf); }

 private:
  Py_buffer b_;
};

int64_t whole(PyObject* o) {
  need(PyLong_CheckExact(o) || PyBool_Check(o));
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    throw NotHere{};
  }
  return v;
}
int32_t whole32(PyObject* o) {
  const int64_t v = whole(o);
  need(v >= INT32_MIN && v <= INT32_MAX);
  return static_cast<int32_t>(v);
}
float number(PyObject* o) {
  need(PyFloat_CheckExact(o));
  return static_cast<float>(PyFloat_AS_DOUBLE(o));
}
const at::Tensor& tensor(PyObject* o) {
  need(THPVariable_CheckExact(o));
  return THPVariable_Unpack(o);
}
// The device of a tensor; the first one's has to be the current one.
void on(const at::Tensor& t, int& device) {
  need(t.is_cuda() && t.layout() == at::kStrided);
  const int at = t.get_device();
  if (device < 0) {
    need(at == c10::cuda::current_device());
    device = at;
  }
  need(at == device);
}
// The device that a structure's tensors lie on, -1 where the binding has not seen them.
int device_seen(PyObject* o) {
  PyObject* d = PyObject_GetAttr(o, g_device);
  if (!d) {
    PyErr_Clear();
    throw NotHere{};
  }
  const bool none = d == Py_None, known = none || PyLong_CheckExact(d);
  int too_long = 0;                          // no error of the interpreter is left behind
  const long at = none || !known ? -1 : PyLong_AsLongAndOverflow(d, &too_long);
  Py_DECREF(d);
  need(known && !too_long && (none || (at >= 0 && at <= INT32_MAX)));
  return static_cast<int>(at);
}
// The same of a structure whose tensors have been seen, on the current device.
int device_of(PyObject* o) {
  const int at = device_seen(o);
  need(at >= 0 && at == c10::cuda::current_device());
  return at;
}
// The turns of a rotation, where they have been seen, lie on `device`.
void turns_on(PyObject* o, int device) {
  const int at = device_seen(o);
  need(at < 0 || at == device);
}

bool row_type(const at::Tensor& t) {
  const auto type = t.scalar_type();
  return type == at::kBFloat16 || type == at::kShort || type == at::kUInt16;
}
// bf16 rows [n, heads, d], dense within a row.
struct Rows {
  uint16_t* p = nullptr;
  int64_t ld = 0, n = 0;
};
Rows rows_of(PyObject* o, int64_t heads, int64_t d, int& device) {
  const at::Tensor& t = tensor(o);
  on(t, device);
  need(row_type(t) && t.dim() == 3 && t.size(1) == heads && t.size(2) == d && t.stride(2) == 1 && (heads <= 1 || t.stride(1) == d));
  return {static_cast<uint16_t*>(t.data_ptr()), t.size(0) > 1 ? t.stride(0) : heads * d, t.size(0)};
}
// The same of exactly `rows` rows (below 0: any number, which it then is); no heads: no array.
Rows head_rows(PyObject* o, int64_t heads, int64_t d, int64_t& rows, int& device) {
  if (heads == 0) return {};
  const Rows r = rows_of(o, heads, d, device);
  need(rows < 0 || r.n == rows);
  rows = r.n;
  return r;
}
template <typename T>
T* vector(PyObject* o, at::ScalarType type, int64_t n, int& device) {
  const at::Tensor& t = tensor(o);
  on(t, device);
  need(t.scalar_type() == type && t.numel() >= n && t.is_contiguous());
  return static_cast<T*>(t.data_ptr());
}
template <typename T>
T* vector_or_none(PyObject* o, at::ScalarType type, int64_t n, int& device) {
  return o == Py_None ? nullptr : vector<T>(o, type, n, device);
}
uint16_t* gamma_of(PyObject* o, int64_t d, int& device) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  on(t, device);
  need(row_type(t) && t.numel() >= d && t.is_contiguous());
  return static_cast<uint16_t*>(t.data_ptr());
}
struct Room {
  void* p = nullptr;
  size_t bytes = 0;
};
Room room_of(PyObject* o, int& device) {
  if (o == Py_None) return {};
  const at::Tensor& t = tensor(o);
  on(t, device);
  need(t.is_contiguous());                   // or fewer bytes than its elements' are there
  return {t.data_ptr(), static_cast<size_t>(t.numel()) * t.element_size()};
}
cudaStream_t stream_of(int device) { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream(); }

// Runs `call` without the interpreter's lock.
template <typename F>
PyObject* status_of(F call) {
  int status;
  PyThreadState* const state = PyEval_SaveThread();
  try {
    status = call();
  } catch (...) {
    PyEval_RestoreThread(state);
    throw;
  }
  PyEval_RestoreThread(state);
  return PyLong_FromLong(status);
}
// A function of kArgs arguments; whatever it throws means that the call is not for the short way.
template <int kArgs, PyObject* (*kBody)(PyObject* const*)>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != kArgs) Py_RETURN_NONE;
  try {
    return kBody(a);
  } catch (...) {
    Py_RETURN_NONE;
  }
}

PyObject* qk_rope_fwd(PyObject* const* a) {
  const Struct<lrqat_qk_rope> r(a[0]);
  const int64_t hq = r->n_heads, hk = r->n_kv_heads, d = r->head_dim;
  int64_t rows = -1;
  int device = -1;
  const Rows q = head_rows(a[2], hq, d, rows, device), k = head_rows(a[3], hk, d, rows, device);
  const Rows qo = head_rows(a[6], hq, d, rows, device), ko = head_rows(a[7], hk, d, rows, device);
  need(device >= 0);
  turns_on(a[0], device);
  const int32_t* pos = vector_or_none<int32_t>(a[1], at::kInt, rows, device);
  const uint16_t *gq = gamma_of(a[4], d, device), *gk = gamma_of(a[5], d, device);
  const cudaStream_t s = stream_of(device);
  return status_of([&] { return lrqat_qk_rope_fwd(r.get(), rows, pos, q.p, q.ld, k.p, k.ld, gq, gk, qo.p, qo.ld, ko.p, ko.ld, s); });
}

PyObject* qk_rope_bwd(PyObject* const* a) {
  const Struct<lrqat_qk_rope> r(a[0]);
  const int64_t hq = r->n_heads, hk = r->n_kv_heads, d = r->head_dim;
  int64_t rows = -1;
  int device = -1;
  const Rows gq = head_rows(a[2], hq, d, rows, device), gk = head_rows(a[3], hk, d, rows, device);
  need(device >= 0);
  turns_on(a[0], device);
  // the inputs of heads without a norm are not read
  const Rows q = head_rows(a[4], a[6] == Py_None ? 0 : hq, d, rows, device);
  const Rows k = head_rows(a[5], a[7] == Py_None ? 0 : hk, d, rows, device);
  const uint16_t *wq = gamma_of(a[6], d, device), *wk = gamma_of(a[7], d, device);
  const Rows dq = head_rows(a[8], hq, d, rows, device), dk = head_rows(a[9], hk, d, rows, device);
  float *dwq = vector_or_none<float>(a[10], at::kFloat, d, device), *dwk = vector_or_none<float>(a[11], at::kFloat, d, device);
  need(PyBool_Check(a[12]));
  const int accumulate = a[12] == Py_True;
  const Room ws = room_of(a[13], device);
  const int32_t* pos = vector_or_none<int32_t>(a[1], at::kInt, rows, device);
  const cudaStream_t s = stream_of(device);
  return status_of([&] {
    return lrqat_qk_rope_bwd(r.get(), rows, pos, gq.p, gq.ld, gk.p, gk.ld, q.p, q.ld, k.p, k.ld, wq, wk, dq.p, dq.ld, dk.p, dk.ld,
                             dwq, dwk, accumulate, ws.p, ws.bytes, s);
  });
}

PyObject* kv_extend(PyObject* const* a) {
  const Struct<lrqat_kv_blocks> b(a[0]);
  int device = device_of(a[0]);
  const int64_t n = b->n_seqs, rows = tensor(a[8]).numel();
  auto ints = [&](int i, int64_t least) { return vector<int32_t>(a[i], at::kInt, least, device); };
  const int32_t *len = ints(1, n), *add = ints(2, n), *free_count = ints(3, 1);
  int32_t *len_out = ints(4, n), *free_out = ints(5, 1), *batch_len = ints(6, n), *row_start = ints(7, n + 1), *pos = ints(8, rows);
  int64_t* slot = vector_or_none<int64_t>(a[9], at::kLong, rows, device);
  const Room ws = room_of(a[10], device);
  const cudaStream_t s = stream_of(device);
  return status_of([&] {
    return lrqat_kv_extend(b.get(), len, add, free_count, rows, len_out, free_out, batch_len, row_start, pos, slot, ws.p, ws.bytes, s);
  });
}

PyObject* kv_truncate(PyObject* const* a) {
  const Struct<lrqat_kv_blocks> b(a[0]);
  int device = device_of(a[0]);
  const int64_t n = b->n_seqs;
  auto ints = [&](int i, int64_t least) { return vector<int32_t>(a[i], at::kInt, least, device); };
  const int32_t *len = ints(1, n), *keep = ints(2, n), *free_count = ints(3, 1);
  int32_t *len_out = ints(4, n), *free_out = ints(5, 1);
  const Room ws = room_of(a[6], device);
  const cudaStream_t s = stream_of(device);
  return status_of([&] { return lrqat_kv_truncate(b.get(), len, keep, free_count, len_out, free_out, ws.p, ws.bytes, s); });
}

// Cache, batch, rows of Q and O and workspace of an attention call.
struct Attn {
  Struct<lrqat_kv_cache> cache;
  Struct<lrqat_kv_batch> batch;
  int device;
  int32_t heads;
  Rows q, o;
  Room ws;
  cudaStream_t stream;
  Attn(PyObject* c, PyObject* b, PyObject* Q, PyObject* O, PyObject* w) : cache(c), batch(b), device(device_of(c)) {
    need(device_of(b) == device);
    const at::Tensor& t = tensor(Q);
    need(t.dim() == 3 && t.size(1) <= INT32_MAX);
    heads = static_cast<int32_t>(t.size(1));
    q = rows_of(Q, heads, cache->head_dim, device);
    o = rows_of(O, heads, cache->head_dim, device);
    need(q.n >= batch->rows && o.n >= batch->rows);
    ws = room_of(w, device);
    stream = stream_of(device);
  }
};

PyObject* kv_attn_sinks(PyObject* const* a) {
  const Attn t(a[0], a[1], a[2], a[6], a[7]);
  const float scale = number(a[3]);
  const int32_t window = whole32(a[4]), sinks = whole32(a[5]);
  return status_of([&] {
    return lrqat_kv_attn_sinks(t.cache.get(), t.batch.get(), t.heads, scale, window, sinks, t.q.p, t.q.ld, t.o.p, t.o.ld, t.ws.p,
                               t.ws.bytes, t.stream);
  });
}

PyObject* kv_attn_shared(PyObject* const* a) {
  const Attn t(a[0], a[1], a[4], a[6], a[7]);
  const int32_t prefix = whole32(a[3]);
  const float scale = number(a[5]);
  int device = t.device;
  need(prefix >= 0 && t.cache->block > 0);
  const int64_t columns = (static_cast<int64_t>(prefix) + t.cache->block - 1) / t.cache->block;
  need(columns == 0 || a[2] != Py_None);
  const int32_t* table = vector_or_none<int32_t>(a[2], at::kInt, columns, device);
  return status_of([&] {
    return lrqat_kv_attn_shared(t.cache.get(), t.batch.get(), table, prefix, t.heads, scale, t.q.p, t.q.ld, t.o.p, t.o.ld, t.ws.p,
                                t.ws.bytes, t.stream);
  });
}

PyObject* kv_attn_sinks_workspace_bytes(PyObject* const* a) {
  const Struct<lrqat_kv_cache> c(a[0]);
  const Struct<lrqat_kv_batch> b(a[1]);
  return PyLong_FromSize_t(lrqat_kv_attn_sinks_workspace_bytes(c.get(), b.get(), whole32(a[2]), whole32(a[3]), whole32(a[4])));
}
PyObject* kv_attn_shared_workspace_bytes(PyObject* const* a) {
  const Struct<lrqat_kv_cache> c(a[0]);
  const Struct<lrqat_kv_batch> b(a[1]);
  return PyLong_FromSize_t(lrqat_kv_attn_shared_workspace_bytes(c.get(), b.get(), whole32(a[2]), whole32(a[3])));
}
PyObject* kv_blocks_workspace_bytes(PyObject* const* a) {
  const Struct<lrqat_kv_blocks> b(a[0]);
  return PyLong_FromSize_t(lrqat_kv_blocks_workspace_bytes(b.get()));
}
PyObject* qk_rope_bwd_workspace_bytes(PyObject* const* a) {
  const Struct<lrqat_qk_rope> r(a[0]);
  return PyLong_FromSize_t(lrqat_qk_rope_bwd_workspace_bytes(r.get(), whole(a[1])));
}

// Dense tensors of one CUDA device (which need not be the current one), for the structures.
const at::Tensor& dense(PyObject* o, at::ScalarType type, int64_t dim, int& device) {
  const at::Tensor& t = tensor(o);
  need(t.is_cuda() && t.layout() == at::kStrided && t.scalar_type() == type && t.dim() == dim && t.is_contiguous());
  const int at = t.get_device();
  need(device < 0 || at == device);
  device = at;
  for (int64_t i = 0; i < dim; ++i) need(t.size(i) <= INT32_MAX);
  return t;
}
PyObject* fill_cache(PyObject* const* a) {
  const Struct<lrqat_kv_cache> c(a[0]);
  int device = -1;
  const at::Tensor &k = dense(a[1], at::kChar, 4, device), &v = dense(a[2], at::kChar, 4, device);
  const at::Tensor &ks = dense(a[3], at::kFloat, 2, device), &vs = dense(a[4], at::kFloat, 2, device);
  need(v.sizes() == k.sizes() && ks.size(0) == k.size(0) && ks.size(1) == k.size(1) && vs.sizes() == ks.sizes());
  *c.get() = {k.size(0), static_cast<int32_t>(k.size(1)), static_cast<int32_t>(k.size(3)), static_cast<int32_t>(k.size(2)),
              static_cast<int8_t*>(k.data_ptr()), static_cast<int8_t*>(v.data_ptr()), static_cast<float*>(ks.data_ptr()),
              static_cast<float*>(vs.data_ptr())};
  return PyLong_FromLong(device);
}
PyObject* fill_batch(PyObject* const* a) {
  const Struct<lrqat_kv_batch> b(a[0]);
  int device = -1;
  const at::Tensor &len = dense(a[1], at::kInt, 1, device), &start = dense(a[2], at::kInt, 1, device);
  const at::Tensor& table = dense(a[3], at::kInt, 2, device);
  const int64_t n = table.size(0), rows = whole(a[4]);
  const int32_t max_rows = whole32(a[5]), max_len = whole32(a[6]);
  need(len.size(0) == n && start.size(0) == n + 1);
  *b.get() = {static_cast<int32_t>(n), static_cast<int32_t>(table.size(1)), static_cast<int32_t*>(len.data_ptr()),
              static_cast<int32_t*>(start.data_ptr()), static_cast<int32_t*>(table.data_ptr()), rows, max_rows, max_len};
  return PyLong_FromLong(device);
}
PyObject* fill_blocks(PyObject* const* a) {
  const Struct<lrqat_kv_blocks> b(a[0]);
  int device = -1;
  const at::Tensor &table = dense(a[1], at::kInt, 2, device), &ids = dense(a[2], at::kInt, 1, device);
  *b.get() = {static_cast<int32_t>(table.size(0)), static_cast<int32_t>(table.size(1)), whole32(a[3]), whole32(a[4]), ids.size(0),
              static_cast<int32_t*>(table.data_ptr()), static_cast<int32_t*>(ids.data_ptr())};
  return PyLong_FromLong(device);
}

// Takes the binding's classes, once, before anything else.
template <typename T>
void set_class(PyObject* o) {
  Py_INCREF(o);
  g_class<T> = reinterpret_cast<PyTypeObject*>(o);
}
PyObject* structures(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4) return PyErr_Format(PyExc_TypeError, "four classes expected");
  for (Py_ssize_t i = 0; i < n; ++i)
    if (!PyType_Check(a[i])) return PyErr_Format(PyExc_TypeError, "four classes expected");
  set_class<lrqat_qk_rope>(a[0]);
  set_class<lrqat_kv_cache>(a[1]);
  set_class<lrqat_kv_batch>(a[2]);
  set_class<lrqat_kv_blocks>(a[3]);
  Py_RETURN_NONE;
}

#define ENTRY(name, args) \
  { #name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<args, name>)), METH_FASTCALL, nullptr }
PyMethodDef g_methods[] = {{"structures", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&structures)), METH_FASTCALL, nullptr},
                           ENTRY(qk_rope_fwd, 8),
                           ENTRY(qk_rope_bwd, 14),
                           ENTRY(kv_extend, 11),
                           ENTRY(kv_truncate, 7),
                           ENTRY(kv_attn_sinks, 8),
                           ENTRY(kv_attn_shared, 8),
                           ENTRY(kv_attn_sinks_workspace_bytes, 5),
                           ENTRY(kv_attn_shared_workspace_bytes, 4),
                           ENTRY(kv_blocks_workspace_bytes, 1),
                           ENTRY(qk_rope_bwd_workspace_bytes, 2),
                           ENTRY(fill_cache, 5),
                           ENTRY(fill_batch, 7),
                           ENTRY(fill_blocks, 5),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "lrqat_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_lrqat_binding() {
  g_device = PyUnicode_InternFromString("device");
  return g_device ? PyModule_Create(&g_module) : nullptr;
}
