// The way from torch tensors to the operators for many requests (amph_project_adapters, amph_paged_write, amph_paged_attention): argument
// checks, output and scratch, one call of the library.  A call through ctypes costs 6-8 us of host time beyond the library's own, as much as
// a small batch's kernels; here it is about 1.
//
// Every entry returns the output tensor (or None), the library's status as an int where a call failed, or NotImplemented where the
// arguments are not what the entry takes: binding.py then says what is wrong with them.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <limits>
#include <map>
#include <optional>
#include <unordered_map>
#include <utility>

#include "amph.h"

namespace {

struct Library {
  decltype(&amph_project_adapters_bytes) project_adapters_bytes;
  decltype(&amph_project_adapters) project_adapters;
  decltype(&amph_paged_write) paged_write;
  decltype(&amph_paged_attention) paged_attention;
} lib;

struct Adapters {
  amph_adapters c;
  int n_seg, out, in, dtype, device;
  std::unordered_map<int, size_t> bytes;      // scratch by rows
};
struct Cache {
  amph_paged_cache c;
  int device;
};

at::ScalarType scalar(int dtype) { return dtype == AMPH_DTYPE_F32 ? at::kFloat : at::kBFloat16; }
int amph_dtype(at::ScalarType t) { return t == at::kFloat ? AMPH_DTYPE_F32 : t == at::kBFloat16 ? AMPH_DTYPE_BF16 : -1; }

// The tensor of an argument, nullptr if it is none.
const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }
bool on(const at::Tensor* t, int device, at::ScalarType type) {
  return t && t->is_cuda() && t->get_device() == device && t->scalar_type() == type && t->layout() == at::kStrided;
}
bool whole(const at::Tensor* t, int device, at::ScalarType type, at::IntArrayRef shape) {
  return on(t, device, type) && t->is_contiguous() && t->sizes() == shape;
}
at::Tensor make(at::IntArrayRef shape, at::ScalarType type, int device) {
  return at::detail::empty_cuda(shape, type, at::Device(at::kCUDA, (c10::DeviceIndex)device), std::nullopt);
}

PyObject* not_these() { Py_RETURN_NOTIMPLEMENTED; }
PyObject* give(const std::optional<at::Tensor>& t, int rc) {
  if (rc != AMPH_OK) return PyLong_FromLong(rc);
  if (!t) Py_RETURN_NONE;
  return THPVariable_Wrap(*t);
}
template <typename T>
T* held(PyObject* o, const char* name) {
  return (T*)PyCapsule_GetPointer(o, name);
}

// Scratch of an attention call on a stream, kept there since its counters are zero between calls (`clean`: only these calls have used it, all
// of them succeeded), 5 MB.  Calls on one stream follow one another, so a stream has one piece; a stream that was destroyed and another that got
// its handle are told apart by their ids.  Calls of one capture share a piece per stream, from the graph's memory: graphs may be replayed
// beside one another and beside anything else, and what a replay finds is what its own first call sets.  It is given back once a call that is not
// of that capture is made; a capture that still goes on then makes another.  (The other operators' scratch holds nothing between calls: an
// ordinary temporary of the allocator's.)
struct Scratch {
  at::Tensor t;
  unsigned long long stream_id = 0;
  bool clean = false;
};
Scratch& attention_scratch(int device, cudaStream_t stream) {
  typedef std::map<std::pair<int, cudaStream_t>, Scratch> Pieces;
  static auto& eager = *new Pieces;                      // never destroyed: the device may be gone by then
  static auto& captured = *new Pieces;
  static unsigned long long capture = 0;                 // that `captured` belongs to
  cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
  unsigned long long id = 0, stream_id = 0;
  C10_CUDA_CHECK(cudaStreamGetCaptureInfo(stream, &status, &id));
  const bool capturing = status != cudaStreamCaptureStatusNone;
  if (!captured.empty() && (!capturing || id != capture)) captured.clear();
  if (capturing) capture = id;
  else C10_CUDA_CHECK(cudaStreamGetId(stream, &stream_id));       // (not while it is captured)
  Scratch& s = (capturing ? captured : eager)[{device, stream}];
  if (!s.t.defined() || s.stream_id != stream_id) {
    s.clean = false;
    s.t = make({AMPH_PAGED_WS_BYTES}, at::kByte, device);         // (before the old one is given back: it may still be in use)
    s.stream_id = stream_id;
  }
  return s;
}

// load(handle of the library)
PyObject* load(PyObject*, PyObject* handle) {
  void* h = PyLong_AsVoidPtr(handle);
  if (PyErr_Occurred()) return nullptr;
  lib.project_adapters_bytes = (decltype(lib.project_adapters_bytes))dlsym(h, "amph_project_adapters_bytes");
  lib.project_adapters = (decltype(lib.project_adapters))dlsym(h, "amph_project_adapters");
  lib.paged_write = (decltype(lib.paged_write))dlsym(h, "amph_paged_write");
  lib.paged_attention = (decltype(lib.paged_attention))dlsym(h, "amph_paged_attention");
  if (!lib.project_adapters_bytes || !lib.project_adapters || !lib.paged_write || !lib.paged_attention) {
    PyErr_SetString(PyExc_RuntimeError, "libamph.so lacks an operator");
    return nullptr;
  }
  Py_RETURN_NONE;
}

// adapters(address of an amph_adapters, n_seg, out, in, dtype, device)
PyObject* adapters(PyObject*, PyObject* args) {
  unsigned long long at;
  auto a = new Adapters;
  if (!PyArg_ParseTuple(args, "Kiiiii", &at, &a->n_seg, &a->out, &a->in, &a->dtype, &a->device)) {
    delete a;
    return nullptr;
  }
  a->c = *(const amph_adapters*)at;
  return PyCapsule_New(a, "adapters", [](PyObject* o) { delete held<Adapters>(o, "adapters"); });
}

// cache(address of an amph_paged_cache, device)
PyObject* cache(PyObject*, PyObject* args) {
  unsigned long long at;
  auto c = new Cache;
  if (!PyArg_ParseTuple(args, "Ki", &at, &c->device)) {
    delete c;
    return nullptr;
  }
  c->c = *(const amph_paged_cache*)at;
  return PyCapsule_New(c, "cache", [](PyObject* o) { delete held<Cache>(o, "cache"); });
}

// project_adapters(adapters, x, ws, rows, use_tensor_core, row_adapter, y, y_dtype, status)
PyObject* project_adapters(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 9) return not_these();
  Adapters* ad = held<Adapters>(a[0], "adapters");
  if (!ad) return nullptr;
  const at::ScalarType type = scalar(ad->dtype);
  const at::Tensor *x = tensor(a[1]), *at_ = tensor(a[5]), *y_in = tensor(a[6]), *status = tensor(a[8]);
  if (!PyLong_Check(a[3])) return not_these();
  const long long rows = PyLong_AsLongLong(a[3]);
  const int tc = PyObject_IsTrue(a[4]);
  if (tc < 0 || (rows == -1 && PyErr_Occurred())) return nullptr;
  if (!on(x, ad->device, type) || x->dim() != 2 || !x->is_contiguous() || x->size(1) != ad->in || rows < 0 || rows > 0x7fffffff ||
      x->size(0) > 0x7fffffff || !whole(at_, ad->device, at::kInt, {(int64_t)rows}))
    return not_these();
  const void* w[8];
  if (!PyList_Check(a[2]) && !PyTuple_Check(a[2])) return not_these();
  if (PySequence_Fast_GET_SIZE(a[2]) != ad->n_seg || ad->n_seg > 8) return not_these();
  for (int s = 0; s < ad->n_seg; ++s) {
    const at::Tensor* t = tensor(PySequence_Fast_GET_ITEM(a[2], s));
    if (!whole(t, ad->device, type, {ad->out, ad->in})) return not_these();
    w[s] = t->data_ptr();
  }
  at::ScalarType y_type = type;
  if (a[7] != Py_None) {
    if (!THPDtype_Check(a[7])) return not_these();
    y_type = ((THPDtype*)a[7])->scalar_type;
    if (amph_dtype(y_type) < 0) return not_these();
  } else if (y_in) {
    y_type = y_in->scalar_type();
    if (amph_dtype(y_type) < 0) return not_these();
  }
  const int64_t ld = (int64_t)ad->n_seg * ad->out;
  if ((a[6] != Py_None && !whole(y_in, ad->device, y_type, {(int64_t)rows, ld})) ||
      (a[8] != Py_None && (!on(status, ad->device, at::kInt) || !status->is_contiguous() || status->numel() < 1)))
    return not_these();
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)ad->device);
  if (rows == 0) return give(y_in ? *y_in : make({0, ld}, y_type, ad->device), AMPH_OK);
  size_t need = 0;
  if (const auto known = ad->bytes.find((int)rows); known != ad->bytes.end()) {
    need = known->second;
  } else {
    const int rc = lib.project_adapters_bytes(ad->n_seg, ad->out, (int)rows, ad->c.rank, &need);
    if (rc != AMPH_OK) return PyLong_FromLong(rc);
    ad->bytes[(int)rows] = need;
  }
  const at::Tensor y = y_in ? *y_in : make({(int64_t)rows, ld}, y_type, ad->device);
  const cudaStream_t stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)ad->device).stream();
  const at::Tensor ws = make({(int64_t)need}, at::kByte, ad->device);
  return give(y, lib.project_adapters(x->data_ptr(), (int)x->size(0), w, ad->n_seg, ad->out, ad->in, (int)rows, ad->dtype, tc, &ad->c,
                                      (const int32_t*)at_->data_ptr(), y.data_ptr(), amph_dtype(y_type), ws.data_ptr(), need,
                                      status ? (int32_t*)status->data_ptr() : nullptr, stream));
  END_HANDLE_TH_ERRORS
}

// Row stride (elements) of [rows][heads * dh] or [rows][heads][dh] whose rows are contiguous, -1 if it is not that.
int64_t row_stride(const at::Tensor& t, int64_t rows, int64_t heads, int64_t dh) {
  const bool flat = t.dim() == 2 && t.size(0) == rows && t.size(1) == heads * dh && t.stride(1) == 1;
  const bool split = t.dim() == 3 && t.size(0) == rows && t.size(1) == heads && t.size(2) == dh && t.stride(2) == 1 && (t.stride(1) == dh || heads == 1);
  return !flat && !split ? -1 : rows > 1 ? t.stride(0) : heads * dh;
}

// paged_write(cache, q, k, v, row_seq, row_pos, table, theta, q_out, status)
PyObject* paged_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 10) return not_these();
  const Cache* c = held<Cache>(a[0], "cache");
  if (!c) return nullptr;
  const int dev = c->device;
  const int64_t dh = c->c.head_dim, kv = c->c.n_kv_heads;
  const at::Tensor *q = tensor(a[1]), *k = tensor(a[2]), *v = tensor(a[3]), *seq = tensor(a[4]), *pos = tensor(a[5]), *table = tensor(a[6]),
                   *q_in = tensor(a[8]), *status = tensor(a[9]);
  const double theta = PyFloat_AsDouble(a[7]);
  if (theta == -1.0 && PyErr_Occurred()) return nullptr;
  if (!k || k->dim() < 2 || amph_dtype(k->scalar_type()) < 0) return not_these();
  const at::ScalarType type = k->scalar_type();
  const int64_t rows = k->size(0);
  if (!on(k, dev, type) || !on(v, dev, type) || rows > 0x7fffffff || !whole(seq, dev, at::kInt, {rows}) || !whole(pos, dev, at::kInt, {rows}) ||
      !on(table, dev, at::kInt) || table->dim() != 2 || !table->is_contiguous() || table->size(0) > 0x7fffffff || table->size(1) > 0x7fffffff ||
      (a[1] != Py_None && (!on(q, dev, type) || q->dim() < 2)) || (a[8] != Py_None && (!q || !q_in)) ||
      (a[9] != Py_None && (!on(status, dev, at::kInt) || !status->is_contiguous() || status->numel() < 1)))
    return not_these();
  const int64_t ks = row_stride(*k, rows, kv, dh), vs = row_stride(*v, rows, kv, dh);
  if (ks < 0 || vs < 0) return not_these();
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)dev);
  int64_t heads = 0, qs = 0;
  std::optional<at::Tensor> q_out;
  if (q) {
    heads = (q->dim() == 3 ? q->size(1) * q->size(2) : q->size(1)) / dh;
    qs = row_stride(*q, rows, heads, dh);
    if (qs < 0 || heads > 0x7fffffff || (q_in && !whole(q_in, dev, scalar(c->c.dtype), {rows, heads, dh}))) return not_these();
    q_out = q_in ? *q_in : make({rows, heads, dh}, scalar(c->c.dtype), dev);
  }
  if (rows == 0) return give(q_out, AMPH_OK);            // (an empty tensor has no address)
  const cudaStream_t stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
  return give(q_out, lib.paged_write(&c->c, q ? q->data_ptr() : nullptr, qs, k->data_ptr(), ks, v->data_ptr(), vs, amph_dtype(type), (int)heads, (int)rows,
                                     (const int32_t*)seq->data_ptr(), (const int32_t*)pos->data_ptr(), (const int32_t*)table->data_ptr(),
                                     (int)table->size(0), (int)table->size(1), (float)theta, q ? q_out->data_ptr() : nullptr,
                                     status ? (int32_t*)status->data_ptr() : nullptr, stream));
  END_HANDLE_TH_ERRORS
}

// paged_attention(cache, q, table, lens, scale, out, lse, status)
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 8) return not_these();
  const Cache* c = held<Cache>(a[0], "cache");
  if (!c) return nullptr;
  const int dev = c->device;
  const at::ScalarType type = scalar(c->c.dtype);
  const at::Tensor *q = tensor(a[1]), *table = tensor(a[2]), *lens = tensor(a[3]), *out_in = tensor(a[5]), *lse = tensor(a[6]), *status = tensor(a[7]);
  const double scale = PyFloat_AsDouble(a[4]);
  if (scale == -1.0 && PyErr_Occurred()) return nullptr;
  float scale_f = (float)scale;                          // 0 means 1 / sqrt(head_dim): not what a scale too small for fp32 asks for
  if (scale_f == 0.f && scale != 0.0) scale_f = std::numeric_limits<float>::denorm_min();
  if (!on(q, dev, type) || q->dim() != 3 || !q->is_contiguous() || q->size(2) != c->c.head_dim || q->size(0) > 0x7fffffff || q->size(1) > 0x7fffffff)
    return not_these();
  const int64_t seqs = q->size(0), heads = q->size(1);
  if (!on(table, dev, at::kInt) || table->dim() != 2 || !table->is_contiguous() || table->size(0) != seqs || table->size(1) > 0x7fffffff ||
      !whole(lens, dev, at::kInt, {seqs}) || (a[5] != Py_None && !whole(out_in, dev, type, q->sizes())) ||
      (a[6] != Py_None && !whole(lse, dev, at::kFloat, {seqs, heads})) ||
      (a[7] != Py_None && (!on(status, dev, at::kInt) || !status->is_contiguous() || status->numel() < 1)))
    return not_these();
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)dev);
  const at::Tensor out = out_in ? *out_in : make(q->sizes(), type, dev);
  if (seqs == 0) return give(out, AMPH_OK);              // (an empty tensor has no address)
  const cudaStream_t stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
  Scratch& ws = attention_scratch(dev, stream);
  const int rc = lib.paged_attention(&c->c, q->data_ptr(), (int)heads, (const int32_t*)lens->data_ptr(), (const int32_t*)table->data_ptr(), (int)seqs,
                                     (int)table->size(1), scale_f, out.data_ptr(), lse ? (float*)lse->data_ptr() : nullptr, ws.t.data_ptr(),
                                     AMPH_PAGED_WS_BYTES, ws.clean, status ? (int32_t*)status->data_ptr() : nullptr, stream);
  ws.clean = rc == AMPH_OK;
  return give(out, rc);
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"load", load, METH_O, nullptr},
    {"adapters", adapters, METH_VARARGS, nullptr},
    {"cache", cache, METH_VARARGS, nullptr},
    {"project_adapters", (PyCFunction)(void (*)())project_adapters, METH_FASTCALL, nullptr},
    {"paged_write", (PyCFunction)(void (*)())paged_write, METH_FASTCALL, nullptr},
    {"paged_attention", (PyCFunction)(void (*)())paged_attention, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "torch_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_torch_ops() { return PyModule_Create(&module); }
