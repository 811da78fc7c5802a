// The calls of a decoding step (eora_serve.h) for Python: arguments are checked and marshalled here instead of through ctypes.
// One of these calls runs for 3 to 6 us on the GPU at small batches; checking up to eight tensors in Python and calling through ctypes took
// 10 to 13 us of the host, this takes 3 (4 where the result is made), the launch itself among them.  No arithmetic; every step is in the library's kernels.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/Stream.h>
#include <torch/csrc/autograd/python_variable.h>
#include "../../include/eora_serve.h"

namespace {

PyObject* g_error = nullptr;            // EoraError(status, where)

struct Refused {};                      // the Python error is set

[[noreturn]] void refuse(int status, const std::string& where) {
  if (!g_error) {
    PyErr_SetString(PyExc_RuntimeError, where.c_str());
  } else if (PyObject* e = PyObject_CallFunction(g_error, "is", status, where.c_str())) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw Refused();
}

at::ScalarType type_of(int code) { return code == 0 ? at::kHalf : code == 1 ? at::kBFloat16 : at::kFloat; }

const at::Tensor* tensor(PyObject* o, const char* what) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse(EORA_ERR_UNSUPPORTED, std::string(what) + ": not a tensor");
  return &THPVariable_Unpack(o);
}
const at::Tensor& needed(PyObject* o, const char* what) {
  const at::Tensor* t = tensor(o, what);
  if (!t) refuse(EORA_ERR_NULL_ARG, std::string(what) + ": missing");
  return *t;
}
std::string shape_text(const at::Tensor& t) {
  std::string s = "shape (";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  s += ") strides (";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.stride(i));
  return s + ")";
}
void check_place(const at::Tensor& t, at::ScalarType type, int device, const char* what) {
  if (t.scalar_type() != type) refuse(EORA_ERR_UNSUPPORTED, std::string(what) + ": type " + c10::toString(t.scalar_type()) + ", not " + c10::toString(type));
  if (!t.is_cuda() || t.device().index() != device) refuse(EORA_ERR_UNSUPPORTED, std::string(what) + ": on " + t.device().str() + ", not on cuda:" + std::to_string(device));
}
// Row stride of a tensor [m][width] (or [m][heads][head_dim]) whose rows are contiguous; m < 0: any.
int64_t rows(const at::Tensor& t, int64_t m, int64_t width, at::ScalarType type, int device, const char* what) {
  check_place(t, type, device, what);
  const bool flat = t.dim() == 2 && t.size(1) == width && t.stride(1) == 1;
  const bool heads = t.dim() == 3 && t.size(1) * t.size(2) == width && t.stride(2) == 1 && (t.stride(1) == t.size(2) || t.size(1) == 1);
  if (!flat && !heads) refuse(EORA_ERR_BAD_SHAPE, std::string(what) + ": " + shape_text(t) + ", not rows of " + std::to_string(width));
  if (m >= 0 && t.size(0) != m) refuse(EORA_ERR_BAD_SHAPE, std::string(what) + ": " + std::to_string(t.size(0)) + " rows, not " + std::to_string(m));
  return t.size(0) > 1 ? t.stride(0) : width;
}
const int32_t* ints(const at::Tensor& t, int64_t n, int device, const char* what) {
  check_place(t, at::kInt, device, what);
  if (t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1)) refuse(EORA_ERR_BAD_SHAPE, std::string(what) + ": " + shape_text(t) + ", not (" + std::to_string(n) + ",)");
  return static_cast<const int32_t*>(t.const_data_ptr());
}
void on_current(int device, const char* where) {
  const int now = c10::cuda::current_device();
  if (now != device) refuse(EORA_ERR_UNSUPPORTED, std::string(where) + ": the tensors are on cuda:" + std::to_string(device) + ", the current device is " + std::to_string(now));
}
// The stream of a call: the current one, a stream object's or a handle's.  What a call makes (results that are not given) is made on it, as memory of
// another stream's pool may still be in use there, or may be given away there while this call runs.
c10::cuda::CUDAStream stream_of(PyObject* o, int device) {
  const auto index = static_cast<c10::DeviceIndex>(device);
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream(index);
  if (THPStream_Check(o)) {
    const auto* t = reinterpret_cast<const THPStream*>(o);
    if (t->device_type != static_cast<int64_t>(c10::DeviceType::CUDA) || t->device_index != device)
      refuse(EORA_ERR_UNSUPPORTED, "stream: of device " + std::to_string(t->device_index) + ", not of cuda:" + std::to_string(device));
    return c10::cuda::CUDAStream::unpack3(t->stream_id, index, c10::DeviceType::CUDA);
  }
  PyObject* v = PyLong_Check(o) ? Py_NewRef(o) : PyObject_GetAttrString(o, "cuda_stream");
  if (!v) throw Refused();
  void* s = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  if (PyErr_Occurred()) throw Refused();
  if (s == cudaStreamLegacy) s = nullptr;                 // (two names of one stream; torch has it as the default one)
  return c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(s), index);
}
// A stream that was made outside of torch, or came as a handle: it may be gone when torch's allocator would ask it for the end of a use.
bool foreign(const c10::cuda::CUDAStream& s) { return s.id() != 0 && !(s.id() & 1); }
template <class T> const T* at_address(PyObject* o) {
  void* p = PyLong_AsVoidPtr(o);
  if (!p) {
    if (!PyErr_Occurred()) refuse(EORA_ERR_NULL_ARG, "a closed or empty object");
    throw Refused();
  }
  return static_cast<const T*>(p);
}
int device_of(PyObject* o) {
  const long d = PyLong_AsLong(o);
  if (d == -1 && PyErr_Occurred()) throw Refused();
  return (int)d;
}
const at::Tensor& or_new(const at::Tensor* t, at::Tensor& own, int64_t m, int64_t width, at::ScalarType type, int device, const c10::cuda::CUDAStream& stream) {
  if (t) return *t;
  c10::cuda::OptionalCUDAStreamGuard on;
  if (stream != c10::cuda::getCurrentCUDAStream(stream.device_index())) on.reset_stream(stream);
  own = at::empty({m, width}, at::TensorOptions().dtype(type).device(at::Device(at::kCUDA, static_cast<c10::DeviceIndex>(device))));
  return own;
}
bool count_is(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", n, want);
  return n == want;
}

// (config, weights, device, x, ids, base, y, stream) -> y
PyObject* adapters(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_is(n, 8)) return nullptr;
  try {
    const auto* cfg = at_address<eora_adapters_config>(a[0]);
    const auto* w = at_address<eora_adapters_weights>(a[1]);
    const int device = device_of(a[2]);
    const at::Tensor& x = needed(a[3], "x");
    const at::Tensor* base = tensor(a[5], "base");
    const at::ScalarType yt = type_of(cfg->y_dtype);
    const int64_t xs = rows(x, -1, cfg->d_in, type_of(cfg->x_dtype), device, "x"), m = x.size(0);
    const int32_t* ids = ints(needed(a[4], "ids"), m, device, "ids");
    const int64_t bs = base ? rows(*base, m, cfg->d_out, yt, device, "base") : 0;
    on_current(device, "adapters");
    const c10::cuda::CUDAStream stream = stream_of(a[7], device);
    at::Tensor own;
    const at::Tensor& y = or_new(tensor(a[6], "y"), own, m, cfg->d_out, yt, device, stream);
    const int64_t ys = rows(y, m, cfg->d_out, yt, device, "y");
    if (m > (1 << 20)) refuse(EORA_ERR_BAD_SHAPE, "adapters: more than 2^20 tokens");
    const int st = eora_adapters_forward(cfg, w, x.const_data_ptr(), xs, (int32_t)m, ids, base ? base->const_data_ptr() : nullptr, bs, y.data_ptr(), ys, stream.stream());
    if (st != EORA_OK) refuse(st, "eora_adapters_forward");
    return THPVariable_Wrap(y);
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (config, device or -1, q, k, v, positions, slots, cache, cache's device, q_out, k_out, stream) -> (q_out, k_out)
PyObject* norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_is(n, 12)) return nullptr;
  try {
    const auto* cfg = at_address<eora_qk_config>(a[0]);
    const at::Tensor& q = needed(a[2], "q");
    const at::Tensor& k = needed(a[3], "k");
    const at::Tensor* v = tensor(a[4], "v");
    const at::Tensor* slots = tensor(a[6], "slots");
    const eora_kv_cache* cache = a[7] == Py_None ? nullptr : at_address<eora_kv_cache>(a[7]);
    int device = device_of(a[1]);
    if (device < 0) device = q.is_cuda() ? q.device().index() : 0;
    const at::ScalarType type = type_of(cfg->dtype);
    const int64_t qw = (int64_t)cfg->n_heads * cfg->head_dim, kw = (int64_t)cfg->n_kv_heads * cfg->head_dim;
    const int64_t qs = rows(q, -1, qw, type, device, "q"), m = q.size(0), ks = rows(k, m, kw, type, device, "k"), vs = v ? rows(*v, m, kw, type, device, "v") : 0;
    const int32_t* pos = ints(needed(a[5], "positions"), m, device, "positions");
    const int32_t* sl = slots ? ints(*slots, m, device, "slots") : nullptr;
    if (cache && device_of(a[8]) != device) refuse(EORA_ERR_UNSUPPORTED, "the cache is on another device");
    on_current(device, "norm and rotation");
    const c10::cuda::CUDAStream stream = stream_of(a[11], device);
    at::Tensor own_q, own_k;
    const at::Tensor& qo = or_new(tensor(a[9], "q_out"), own_q, m, qw, type, device, stream);
    const int64_t qos = rows(qo, m, qw, type, device, "q_out");
    const at::Tensor* ko = tensor(a[10], "k_out");
    if (!ko && !cache) ko = &or_new(nullptr, own_k, m, kw, type, device, stream);
    const int64_t kos = ko ? rows(*ko, m, kw, type, device, "k_out") : 0;
    if (m > (1 << 20)) refuse(EORA_ERR_BAD_SHAPE, "norm and rotation: more than 2^20 tokens");
    const int st = eora_qk_norm_rope(cfg, q.const_data_ptr(), qs, k.const_data_ptr(), ks, v ? v->const_data_ptr() : nullptr, vs, pos, (int32_t)m, qo.data_ptr(), qos,
                                     ko ? ko->data_ptr() : nullptr, kos, sl, cache, stream.stream());
    if (st != EORA_OK) refuse(st, "eora_qk_norm_rope");
    PyObject* po = THPVariable_Wrap(qo);
    PyObject* pk = ko ? THPVariable_Wrap(*ko) : Py_NewRef(Py_None);
    PyObject* both = po && pk ? PyTuple_Pack(2, po, pk) : nullptr;
    Py_XDECREF(po);
    Py_XDECREF(pk);
    return both;
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (config, device, workspace, address of an int, q, cache, cache's device, page_table, lengths, out, lse, stream) -> out.  The int is set to 1 if the
// workspace is in use on a stream that its allocator does not know of.
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_is(n, 12)) return nullptr;
  try {
    const auto* cfg = at_address<eora_attention_config>(a[0]);
    const int device = device_of(a[1]);
    const at::Tensor& ws = needed(a[2], "workspace");
    int* in_use = const_cast<int*>(at_address<int>(a[3]));
    const at::Tensor& q = needed(a[4], "q");
    const auto* cache = at_address<eora_kv_cache>(a[5]);
    const at::Tensor& table = needed(a[7], "page_table");
    const at::Tensor* lse = tensor(a[10], "lse");
    const at::ScalarType type = type_of(cfg->dtype);
    const int64_t width = (int64_t)cfg->n_heads * cfg->head_dim;
    const int64_t qs = rows(q, -1, width, type, device, "q"), batch = q.size(0);
    if (device_of(a[6]) != device) refuse(EORA_ERR_UNSUPPORTED, "the cache is on another device");
    check_place(table, at::kInt, device, "page_table");
    if (table.dim() != 2 || table.size(0) != batch || table.size(1) < cfg->max_pages || (table.stride(1) != 1 && table.size(1) > 1))
      refuse(EORA_ERR_BAD_SHAPE, "page_table: " + shape_text(table) + " for " + std::to_string(batch) + " sequences of " + std::to_string(cfg->max_pages) + " pages");
    const int32_t* lengths = ints(needed(a[8], "lengths"), batch, device, "lengths");
    if (lse) {
      check_place(*lse, at::kFloat, device, "lse");
      if (lse->dim() != 2 || lse->size(0) != batch || lse->size(1) != cfg->n_heads || !lse->is_contiguous()) refuse(EORA_ERR_BAD_SHAPE, "lse: " + shape_text(*lse));
    }
    on_current(device, "attention");
    const c10::cuda::CUDAStream stream = stream_of(a[11], device);
    at::Tensor own;
    const at::Tensor& out = or_new(tensor(a[9], "out"), own, batch, width, type, device, stream);
    const int64_t os = rows(out, batch, width, type, device, "out");
    if (batch > cfg->max_batch) refuse(EORA_ERR_M_TOO_LARGE, "attention: " + std::to_string(batch) + " sequences, at most " + std::to_string(cfg->max_batch));
    if (foreign(stream)) *in_use = 1;
    else c10::cuda::CUDACachingAllocator::recordStream(ws.storage().data_ptr(), stream);
    const int st = eora_attention_forward(cfg, q.const_data_ptr(), qs, cache, static_cast<const int32_t*>(table.const_data_ptr()), batch > 1 ? table.stride(0) : table.size(1), lengths,
                                          (int32_t)batch, out.data_ptr(), os, lse ? static_cast<float*>(lse->data_ptr()) : nullptr, ws.data_ptr(), ws.nbytes(), stream.stream());
    if (st != EORA_OK) refuse(st, "eora_attention_forward");
    return THPVariable_Wrap(out);
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (rows, width, type, device, stream) -> a tensor that is made on the stream
PyObject* empty(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_is(n, 5)) return nullptr;
  try {
    const long long m = PyLong_AsLongLong(a[0]), width = PyLong_AsLongLong(a[1]);
    const int type = (int)PyLong_AsLong(a[2]), device = device_of(a[3]);
    if (PyErr_Occurred()) throw Refused();
    at::Tensor own;
    return THPVariable_Wrap(or_new(nullptr, own, m, width, type_of(type), device, stream_of(a[4], device)));
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* type) {
  Py_XSETREF(g_error, Py_NewRef(type));
  Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)> PyCFunction fast() { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)); }
PyMethodDef g_methods[] = {{"adapters", fast<adapters>(), METH_FASTCALL, nullptr},
                           {"norm_rope", fast<norm_rope>(), METH_FASTCALL, nullptr},
                           {"attention", fast<attention>(), METH_FASTCALL, nullptr},
                           {"empty", fast<empty>(), METH_FASTCALL, nullptr},
                           {"set_error", set_error, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", "The serving calls, for " EORA_BUILT_FOR, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&g_module); }
