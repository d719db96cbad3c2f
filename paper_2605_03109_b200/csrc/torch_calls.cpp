// The calls that a program makes once per token, as functions of a Python extension module: check the
// tensors, allocate the outputs, call the C ABI.  Marshalling only.
//
// What it is for: with the kernel of a one-token call at 5 us, the caller's side was what a call
// took: three allocations through Python 4.8 us, the ctypes call 3.5, the rest 1.8.
//
// The functions take the entry points' addresses (bind), so that this module needs no link to the
// CUDA library; they return (status, outputs...) and leave the exception to the Python side.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <climits>
#include <memory>

#include <ATen/ATen.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "gsi.h"

namespace {

decltype(&gsi_forward_n) forward_n = nullptr;
decltype(&gsi_extend_basis) extend_basis = nullptr;
decltype(&gsi_forward_static) forward_static = nullptr;
decltype(&gsi_kv_plan) kv_plan = nullptr;
decltype(&gsi_kv_release) kv_release = nullptr;
decltype(&gsi_kv_append) kv_append = nullptr;
decltype(&gsi_kv_read) kv_read = nullptr;
decltype(&gsi_kv_attend) kv_attend = nullptr;
decltype(&gsi_kv_attend_all) kv_attend_all = nullptr;

struct NoGil {
  PyThreadState* state = PyEval_SaveThread();
  ~NoGil() { PyEval_RestoreThread(state); }
};

// The handle of a stream argument that is not None: an int or an object with cuda_stream.
bool stream_of(PyObject* o, bool* given, void** out) {
  *given = o != Py_None;
  *out = nullptr;
  if (!*given) return true;
  PyObject* number = PyObject_GetAttrString(o, "cuda_stream");
  if (!number) {
    if (!PyErr_ExceptionMatches(PyExc_AttributeError)) return false;
    PyErr_Clear();
    number = Py_NewRef(o);
  }
  PyObject* value = PyNumber_Long(number);
  Py_DECREF(number);
  if (!value) return false;
  *out = PyLong_AsVoidPtr(value);
  Py_DECREF(value);
  return !PyErr_Occurred();
}

const at::Tensor* tensor_of(PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_SetString(PyExc_TypeError, "a tensor is expected");
    return nullptr;
  }
  return &THPVariable_Unpack(o);
}
// The input of a call.
const at::Tensor* input_of(PyObject* o) {
  const at::Tensor* x = tensor_of(o);
  if (x && !(x->is_cuda() && x->scalar_type() == at::kFloat && x->is_contiguous())) {
    PyErr_SetString(PyExc_AssertionError, "x must be a contiguous float32 tensor on a CUDA device");
    return nullptr;
  }
  return x;
}
// An output that the caller gave, or one that is allocated here.
bool output_of(PyObject* o, at::Tensor* t) {
  if (o == Py_None) return true;
  const at::Tensor* given = tensor_of(o);
  if (given) *t = *given;
  return given != nullptr;
}
bool enough(Py_ssize_t given, Py_ssize_t wanted) {
  if (given == wanted) return true;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return false;
}

// A tensor that the kernels of a stream write (`given`: one that is not torch's current one, perhaps).  It is of that stream's
// memory, as what is free to the current stream may still be in use there, and is not handed out again before the current stream,
// whose tensor it is from here on, is done with it.
at::Tensor made_on(bool given, void* stream, at::IntArrayRef size, const at::TensorOptions& options) {
  const c10::DeviceIndex device = options.device().index();
  const auto current = c10::cuda::getCurrentCUDAStream(device);
  if (stream == (void*)cudaStreamLegacy) stream = nullptr;
  if (!given || stream == (void*)current.stream()) return at::empty(size, options);
  const c10::cuda::CUDAStreamGuard guard(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), device));
  at::Tensor t = at::empty(size, options);
  if (t.numel()) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), current);
  return t;
}

void allocate(bool given, void* stream, const at::Tensor& x, int64_t n, int64_t O, at::Tensor* y, at::Tensor* gate, at::Tensor* rho) {
  if (!y->defined()) *y = made_on(given, stream, {n, O}, x.options());
  if (!gate->defined()) *gate = made_on(given, stream, {n}, x.options().dtype(at::kByte));
  if (!rho->defined()) *rho = made_on(given, stream, {n}, x.options());
}

// forward(handle, O, x, y, gate, rho, stream) -> (status, y, gate, rho)
PyObject* py_forward(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!enough(n_args, 7)) return nullptr;
  auto handle = static_cast<gsi_handle_t>(PyLong_AsVoidPtr(args[0]));
  const int64_t O = PyLong_AsLongLong(args[1]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor* x = input_of(args[2]);
  at::Tensor y, gate, rho;
  bool given;
  void* stream;
  if (!x || !output_of(args[3], &y) || !output_of(args[4], &gate) || !output_of(args[5], &rho) ||
      !stream_of(args[6], &given, &stream))
    return nullptr;
  int status;
  {
    NoGil no_gil;
    const int64_t n = x->size(0);
    allocate(given, stream, *x, n, O, &y, &gate, &rho);
    if (!given) stream = c10::cuda::getCurrentCUDAStream().stream();
    status = forward_n(handle, static_cast<const float*>(x->data_ptr()), (int)n, static_cast<float*>(y.data_ptr()),
                       static_cast<unsigned char*>(gate.data_ptr()), static_cast<float*>(rho.data_ptr()),
                       static_cast<gsi_stream_t>(stream));
  }
  return Py_BuildValue("iNNN", status, THPVariable_Wrap(y), THPVariable_Wrap(gate), THPVariable_Wrap(rho));
  END_HANDLE_TH_ERRORS
}

// extend(handle, x, tau, k_active, stream) -> (status, appended, rho)
PyObject* py_extend(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!enough(n_args, 5)) return nullptr;
  auto handle = static_cast<gsi_handle_t>(PyLong_AsVoidPtr(args[0]));
  const double tau = PyFloat_AsDouble(args[2]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor* x = input_of(args[1]);
  const at::Tensor* k_active = x ? tensor_of(args[3]) : nullptr;
  bool given;
  void* stream;
  if (!k_active || !stream_of(args[4], &given, &stream)) return nullptr;
  if (!(k_active->is_cuda() && k_active->scalar_type() == at::kInt && k_active->numel() == 1)) {
    PyErr_SetString(PyExc_AssertionError, "k_active must be one int32 on a CUDA device");
    return nullptr;
  }
  at::Tensor appended, rho;
  int status;
  {
    NoGil no_gil;
    appended = made_on(given, stream, {1}, x->options().dtype(at::kInt));
    rho = made_on(given, stream, {1}, x->options());
    if (!given) stream = c10::cuda::getCurrentCUDAStream().stream();
    status = extend_basis(handle, static_cast<const float*>(x->data_ptr()), (float)tau,
                          static_cast<int*>(k_active->data_ptr()), static_cast<int*>(appended.data_ptr()),
                          static_cast<float*>(rho.data_ptr()), static_cast<gsi_stream_t>(stream));
  }
  return Py_BuildValue("iNN", status, THPVariable_Wrap(appended), THPVariable_Wrap(rho));
  END_HANDLE_TH_ERRORS
}

// forward_static(Ws (a list), P, p_dtype, W_P, eps, x, y, gate, rho, stream) -> (status, y, gate, rho)
PyObject* py_forward_static(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!enough(n_args, 10)) return nullptr;
  if (!PyList_Check(args[0])) {
    PyErr_SetString(PyExc_TypeError, "a list of tensors is expected");
    return nullptr;
  }
  const Py_ssize_t maps = PyList_GET_SIZE(args[0]);
  std::vector<const void*> W(maps);
  std::vector<int> d_out(maps);
  int64_t O = 0;
  for (Py_ssize_t j = 0; j < maps; ++j) {
    const at::Tensor* w = tensor_of(PyList_GET_ITEM(args[0], j));
    if (!w) return nullptr;
    W[j] = w->data_ptr();
    d_out[j] = (int)w->size(0);
    O += d_out[j];
  }
  const at::Tensor *P = tensor_of(args[1]), *W_P = P ? tensor_of(args[3]) : nullptr, *x = W_P ? tensor_of(args[5]) : nullptr;
  if (!x) return nullptr;
  const long p_dtype = PyLong_AsLong(args[2]);
  const double eps = PyFloat_AsDouble(args[4]);
  if (PyErr_Occurred()) return nullptr;
  at::Tensor y, gate, rho;
  bool given;
  void* stream;
  if (!output_of(args[6], &y) || !output_of(args[7], &gate) || !output_of(args[8], &rho) ||
      !stream_of(args[9], &given, &stream))
    return nullptr;
  int status;
  {
    NoGil no_gil;
    const int64_t n = x->size(0);
    allocate(given, stream, *x, n, O, &y, &gate, &rho);
    if (!given) stream = c10::cuda::getCurrentCUDAStream().stream();
    status = forward_static(W.data(), d_out.data(), (int)maps, P->data_ptr(), (gsi_dtype_t)p_dtype, W_P->data_ptr(),
                            (int)P->size(0), (int)P->size(1), (float)eps, static_cast<const float*>(x->data_ptr()), (int)n,
                            static_cast<float*>(y.data_ptr()), static_cast<unsigned char*>(gate.data_ptr()),
                            static_cast<float*>(rho.data_ptr()), static_cast<gsi_stream_t>(stream));
  }
  return Py_BuildValue("iNNN", status, THPVariable_Wrap(y), THPVariable_Wrap(gate), THPVariable_Wrap(rho));
  END_HANDLE_TH_ERRORS
}

// bind(address of gsi_forward_n, of gsi_extend_basis, of gsi_forward_static)
PyObject* py_bind(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (!enough(n_args, 3)) return nullptr;
  forward_n = reinterpret_cast<decltype(forward_n)>(PyLong_AsVoidPtr(args[0]));
  extend_basis = reinterpret_cast<decltype(extend_basis)>(PyLong_AsVoidPtr(args[1]));
  forward_static = reinterpret_cast<decltype(forward_static)>(PyLong_AsVoidPtr(args[2]));
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

// ---- the cache of keys and values: a handle and the tensors of its state, in a capsule
struct Cache {
  gsi_kv_t handle = nullptr;
  int64_t n_heads = 0, head_dim = 0, max_seqs = 0, layers = 0;
  at::Tensor pages, table, lens, free, n_free, q_start, kv_len, slots, positions, counts;
  c10::Device device = c10::Device(c10::kCPU);
};
constexpr const char* kCacheName = "_torch_calls.cache";
Cache* cache_of(PyObject* o) { return static_cast<Cache*>(PyCapsule_GetPointer(o, kCacheName)); }
template <typename T>
T* ptr(const at::Tensor& t) {
  return static_cast<T*>(t.data_ptr());
}
bool refuse(const char* why) {
  PyErr_SetString(PyExc_AssertionError, why);
  return false;
}
bool type_of(const at::Tensor& t, gsi_dtype_t* out) {
  switch (t.scalar_type()) {
    case at::kFloat: *out = GSI_F32; return true;
    case at::kBFloat16: *out = GSI_BF16; return true;
    case at::kHalf: *out = GSI_F16; return true;
    default: return refuse("float32, bfloat16 or float16 is expected");
  }
}
// [n][heads][head_dim] on the cache's device, channels adjacent.
bool rows_of(const Cache& c, const at::Tensor& t, int64_t heads, const char* what) {
  if (t.device() == c.device && t.dim() == 3 && t.size(2) == c.head_dim && (heads == 0 || t.size(1) == heads) &&
      (t.stride(2) == 1 || c.head_dim == 1) && t.size(0) <= INT_MAX)
    return true;
  return refuse(what);
}
bool ints_of(const Cache& c, const at::Tensor& t, at::ScalarType type) {
  if (t.device() == c.device && t.scalar_type() == type && t.dim() == 1 && t.is_contiguous() && t.size(0) <= INT_MAX) return true;
  return refuse(type == at::kInt ? "a contiguous vector of int32 on the cache's device is expected"
                                 : "a contiguous vector of bool or uint8 on the cache's device is expected");
}
bool layer_of(const Cache& c, PyObject* o, void** pages) {
  const int64_t layer = PyLong_AsLongLong(o);
  if (PyErr_Occurred()) return false;
  if (layer < 0 || layer >= c.layers) return refuse("no such layer");
  *pages = ptr<char>(c.pages) + layer * (c.pages.numel() / c.layers);
  return true;
}
gsi_stream_t stream_on(const Cache& c, bool given, void* stream) {
  return static_cast<gsi_stream_t>(given ? stream : (void*)c10::cuda::getCurrentCUDAStream(c.device.index()).stream());
}

// kv_state(handle, n_heads, head_dim, layers, pages, table, lens, free, n_free, q_start, kv_len, slots, positions, counts) -> capsule
PyObject* py_kv_state(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!enough(n_args, 14)) return nullptr;
  auto c = std::make_unique<Cache>();
  c->handle = static_cast<gsi_kv_t>(PyLong_AsVoidPtr(args[0]));
  c->n_heads = PyLong_AsLongLong(args[1]);
  c->head_dim = PyLong_AsLongLong(args[2]);
  c->layers = PyLong_AsLongLong(args[3]);
  if (PyErr_Occurred()) return nullptr;
  at::Tensor* to[] = {&c->pages, &c->table, &c->lens, &c->free, &c->n_free, &c->q_start, &c->kv_len, &c->slots, &c->positions, &c->counts};
  for (int i = 0; i < 10; ++i) {
    const at::Tensor* t = tensor_of(args[4 + i]);
    if (!t) return nullptr;
    *to[i] = *t;
  }
  c->device = c->pages.device();
  c->max_seqs = c->lens.numel();
  return PyCapsule_New(c.release(), kCacheName, [](PyObject* o) { delete static_cast<Cache*>(PyCapsule_GetPointer(o, kCacheName)); });
  END_HANDLE_TH_ERRORS
}
// kv_close(capsule): its handle is gone
PyObject* py_kv_close(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (!enough(n_args, 1)) return nullptr;
  Cache* c = cache_of(args[0]);
  if (!c) return nullptr;
  c->handle = nullptr;
  Py_RETURN_NONE;
}
// kv_plan(capsule, n_new, commit, stream) -> status
PyObject* py_kv_plan(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!enough(n_args, 4)) return nullptr;
  Cache* c = cache_of(args[0]);
  const at::Tensor* n_new = c ? tensor_of(args[1]) : nullptr;
  const int commit = n_new ? PyObject_IsTrue(args[2]) : -1;
  bool given;
  void* stream;
  if (commit < 0 || !ints_of(*c, *n_new, at::kInt) || !stream_of(args[3], &given, &stream)) return nullptr;
  int status;
  {
    NoGil no_gil;
    const c10::cuda::CUDAGuard guard(c->device);
    // (for all requests: what comes after goes by the tensors alone, whichever plan a replayed graph has run)
    status = kv_plan(c->handle, ptr<int>(*n_new), (int)n_new->numel(), GSI_KV_ALL_SEQS | (commit ? GSI_KV_COMMIT : 0), ptr<int>(c->lens), ptr<int>(c->n_free), ptr<int>(c->free),
                     ptr<int>(c->table), ptr<int>(c->q_start), ptr<int>(c->kv_len), ptr<int>(c->slots), ptr<int>(c->positions),
                     ptr<int>(c->counts), stream_on(*c, given, stream));
  }
  return PyLong_FromLong(status);
  END_HANDLE_TH_ERRORS
}
// kv_release(capsule, done, stream) -> status
PyObject* py_kv_release(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!enough(n_args, 3)) return nullptr;
  Cache* c = cache_of(args[0]);
  const at::Tensor* done = c ? tensor_of(args[1]) : nullptr;
  bool given;
  void* stream;
  if (!done || !ints_of(*c, *done, done->scalar_type() == at::kBool ? at::kBool : at::kByte) || !stream_of(args[2], &given, &stream)) return nullptr;
  int status;
  {
    NoGil no_gil;
    const c10::cuda::CUDAGuard guard(c->device);
    status = kv_release(c->handle, ptr<unsigned char>(*done), (int)done->numel(), ptr<int>(c->lens), ptr<int>(c->n_free), ptr<int>(c->free),
                        ptr<int>(c->table), stream_on(*c, given, stream));
  }
  return PyLong_FromLong(status);
  END_HANDLE_TH_ERRORS
}
// kv_append(capsule, k, v, layer, slots or None, stream) -> status
PyObject* py_kv_append(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!enough(n_args, 6)) return nullptr;
  Cache* c = cache_of(args[0]);
  const at::Tensor *k = c ? tensor_of(args[1]) : nullptr, *v = k ? tensor_of(args[2]) : nullptr;
  const at::Tensor* slots = v ? (args[4] == Py_None ? &c->slots : tensor_of(args[4])) : nullptr;
  bool given;
  void *stream, *pages;
  gsi_dtype_t type;
  if (!slots || !rows_of(*c, *k, c->n_heads, "k must be [n][n_heads][head_dim] on the cache's device, channels adjacent") ||
      !rows_of(*c, *v, c->n_heads, "v must be [n][n_heads][head_dim] on the cache's device, channels adjacent") || !type_of(*k, &type) ||
      !ints_of(*c, *slots, at::kInt) || !layer_of(*c, args[3], &pages) || !stream_of(args[5], &given, &stream))
    return nullptr;
  if (k->scalar_type() != v->scalar_type() || k->size(0) != v->size(0)) return refuse("k and v differ in type or rows"), nullptr;
  if (args[4] == Py_None ? slots->numel() < k->size(0) : slots->numel() != k->size(0)) return refuse("a slot for each row is expected"), nullptr;
  int status;
  {
    NoGil no_gil;
    const c10::cuda::CUDAGuard guard(c->device);
    status = kv_append(c->handle, k->data_ptr(), v->data_ptr(), type, k->stride(0), k->stride(1), v->stride(0), v->stride(1), ptr<int>(*slots),
                       (int)k->size(0), pages, stream_on(*c, given, stream));
  }
  return PyLong_FromLong(status);
  END_HANDLE_TH_ERRORS
}
// kv_read(capsule, slots, layer, like (a tensor of the type that is wanted), stream) -> (status, k, v)
PyObject* py_kv_read(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!enough(n_args, 5)) return nullptr;
  Cache* c = cache_of(args[0]);
  const at::Tensor *slots = c ? tensor_of(args[1]) : nullptr, *like = slots ? tensor_of(args[3]) : nullptr;
  bool given;
  void *stream, *pages;
  gsi_dtype_t type;
  if (!like || !type_of(*like, &type) || !ints_of(*c, *slots, at::kInt) || !layer_of(*c, args[2], &pages) || !stream_of(args[4], &given, &stream))
    return nullptr;
  at::Tensor k, v;
  int status;
  {
    NoGil no_gil;
    const c10::cuda::CUDAGuard guard(c->device);
    const auto options = slots->options().dtype(like->scalar_type());
    k = made_on(given, stream, {slots->numel(), c->n_heads, c->head_dim}, options);
    v = made_on(given, stream, {slots->numel(), c->n_heads, c->head_dim}, options);
    status = kv_read(c->handle, pages, ptr<int>(*slots), (int)slots->numel(), type, k.data_ptr(), v.data_ptr(), stream_on(*c, given, stream));
  }
  return Py_BuildValue("iNN", status, THPVariable_Wrap(k), THPVariable_Wrap(v));
  END_HANDLE_TH_ERRORS
}
// kv_attend(capsule, q, layer, scale, out or None, stream) -> (status, out)
PyObject* py_kv_attend(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!enough(n_args, 6)) return nullptr;
  Cache* c = cache_of(args[0]);
  const at::Tensor* q = c ? tensor_of(args[1]) : nullptr;
  const double scale = q ? PyFloat_AsDouble(args[3]) : 0.0;
  if (PyErr_Occurred()) return nullptr;
  bool given;
  void *stream, *pages;
  gsi_dtype_t type;
  at::Tensor out;
  if (!q || !rows_of(*c, *q, 0, "q must be [n][heads][head_dim] on the cache's device, channels adjacent") || !type_of(*q, &type) ||
      !layer_of(*c, args[2], &pages) || !output_of(args[4], &out) || !stream_of(args[5], &given, &stream))
    return nullptr;
  if (q->size(1) < 1 || q->size(1) > INT_MAX || q->size(1) % c->n_heads) return refuse("the heads of q must be a multiple of the cache's"), nullptr;
  if (out.defined()) {
    if (!rows_of(*c, out, q->size(1), "out must be of q's shape, on its device, channels adjacent")) return nullptr;
    if (out.size(0) != q->size(0) || out.scalar_type() != q->scalar_type()) return refuse("out must be of q's shape and type"), nullptr;
  }
  int status;
  {
    NoGil no_gil;
    const c10::cuda::CUDAGuard guard(c->device);
    const bool made = !out.defined();   // (whose rows behind the last request's are written, too)
    if (made) out = made_on(given, stream, {q->size(0), q->size(1), q->size(2)}, q->options());
    status = (made ? kv_attend_all : kv_attend)(c->handle, q->data_ptr(), type, q->stride(0), q->stride(1), (int)q->size(0), (int)q->size(1), (float)scale,
                       ptr<int>(c->q_start), ptr<int>(c->kv_len), ptr<int>(c->table), (int)c->max_seqs, pages, out.data_ptr(), out.stride(0),
                       out.stride(1), stream_on(*c, given, stream));
  }
  return Py_BuildValue("iN", status, THPVariable_Wrap(out));
  END_HANDLE_TH_ERRORS
}
// bind_kv(addresses of gsi_kv_plan, _release, _append, _read, _attend, _attend_all)
PyObject* py_bind_kv(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (!enough(n_args, 6)) return nullptr;
  kv_plan = reinterpret_cast<decltype(kv_plan)>(PyLong_AsVoidPtr(args[0]));
  kv_release = reinterpret_cast<decltype(kv_release)>(PyLong_AsVoidPtr(args[1]));
  kv_append = reinterpret_cast<decltype(kv_append)>(PyLong_AsVoidPtr(args[2]));
  kv_read = reinterpret_cast<decltype(kv_read)>(PyLong_AsVoidPtr(args[3]));
  kv_attend = reinterpret_cast<decltype(kv_attend)>(PyLong_AsVoidPtr(args[4]));
  kv_attend_all = reinterpret_cast<decltype(kv_attend_all)>(PyLong_AsVoidPtr(args[5]));
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(forward), METHOD(extend), METHOD(forward_static), METHOD(bind),
                         METHOD(kv_state), METHOD(kv_close), METHOD(kv_plan), METHOD(kv_release), METHOD(kv_append), METHOD(kv_read),
                         METHOD(kv_attend), METHOD(bind_kv), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls() { return PyModule_Create(&module); }
