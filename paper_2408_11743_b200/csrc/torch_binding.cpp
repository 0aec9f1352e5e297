// The per-call part of the Python binding, natively: argument checks, the output tensor, the current stream and the one
// call into libmarlin_b200.  A decode call on a small layer takes 5 us on the GPU; the same steps in Python took 12 us
// (torch.cuda.current_stream() 3.3 us, torch.empty 2.4 us, the ctypes call 1.1 us beside the 2.5 us of the launch
// itself), so that a loop over such layers waited for the host.
//
// A plain CPython extension module: tensors are unpacked with torch's own C++ API, outputs come from its caching
// allocator.  It links to nothing of this library; bind() hands it the addresses of the entry points that the ctypes
// binding has loaded, and what to call to raise MarlinError.
#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cmath>
#include <cstdint>
#include <optional>

#include "marlin_b200.h"

namespace {

typedef int (*GemmFn)(const void*, const void*, const void*, void*, int, int, int, int, void*, size_t, void*);
typedef int (*GemmExtraFn)(const void*, const void*, const void*, const void*, void*, int, int, int, int, void*, size_t,
                           void*);
typedef int (*MlpFn)(const void*, const void*, const void*, const void*, const void*, void*, void*, int, int, int, int,
                     int, void*, size_t, void*);
typedef size_t (*SizeFn)(int, int, int);
typedef size_t (*SizeFn2)(int, int);

// the kinds of product, in the order of kNames
enum Kind { kDense, kSparse, kZero, kW8, kSwiglu, kKinds };
const char* const kNames[kKinds] = {"marlin_gemm", "marlin_gemm_sparse24", "marlin_gemm_zp", "marlin_gemm_w8",
                                    "marlin_gemm_swiglu"};
void* g_fn[kKinds];
MlpFn g_mlp;
decltype(&marlin_kv_append) g_append;
decltype(&marlin_attention_decode) g_attention;
decltype(&marlin_attention_block) g_block;
decltype(&marlin_kv_append_scaled) g_append_scaled;
decltype(&marlin_attention_sinks) g_attention_sinks;
decltype(&marlin_attention_block_sinks) g_block_sinks;
decltype(&marlin_kv_reserve) g_reserve;
SizeFn g_weight_bytes, g_scale_bytes;
SizeFn2 g_meta_bytes, g_weight_bytes_w8;
PyObject* g_raise;  // raise(status, what)

// an argument as the int that the library takes; false with a Python error set (a size beyond it is no other size)
bool integer(PyObject* o, const char* name, int* out) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) return false;
  if (v < INT_MIN || v > INT_MAX) {
    PyErr_Format(PyExc_ValueError, "%s is out of range", name);
    return false;
  }
  *out = (int)v;
  return true;
}

// nullptr with a Python error set, or the tensor
const at::Tensor* tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a CUDA tensor", name);
    return nullptr;
  }
  return &THPVariable_Unpack(o);
}
const at::Tensor* device_tensor(PyObject* o, at::ScalarType type, const char* name) {
  const at::Tensor* t = tensor(o, name);
  if (!t) return nullptr;
  if (!t->is_cuda()) {
    PyErr_Format(PyExc_TypeError, "%s must be a CUDA tensor", name);
    return nullptr;
  }
  if (t->scalar_type() != type) {
    PyErr_Format(PyExc_TypeError, "%s must have dtype %s", name, type == at::kHalf ? "torch.float16" : "torch.uint8");
    return nullptr;
  }
  if (!t->is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "%s must be contiguous", name);
    return nullptr;
  }
  return t;
}
const at::Tensor* activations(PyObject* o, int64_t K) {
  const at::Tensor* t = device_tensor(o, at::kHalf, "A");
  if (t && (t->dim() != 2 || t->size(1) != K)) {
    PyErr_SetString(PyExc_ValueError, "A must be [M, K]");
    return nullptr;
  }
  return t;
}
// `given` (or None: a new tensor from torch's allocator) as fp16 [M][N]; false with a Python error set
bool output(PyObject* given, int64_t M, int64_t N, const at::Device& device, const char* name, at::Tensor* out) {
  if (given == Py_None) {
    *out = at::detail::empty_cuda({M, N}, at::kHalf, device, std::nullopt);
    return true;
  }
  const at::Tensor* t = device_tensor(given, at::kHalf, name);
  if (!t) return false;
  if (t->dim() != 2 || t->size(0) != M || t->size(1) != N) {
    PyErr_Format(PyExc_ValueError, "%s must be [%lld, %lld]", name, (long long)M, (long long)N);
    return false;
  }
  *out = *t;
  return true;
}
// the handle of `stream` (an object with cuda_stream), of the current stream where it is None
bool stream_handle(PyObject* stream, void** handle) {
  if (stream == Py_None) {
    *handle = c10::cuda::getCurrentCUDAStream().stream();
    return true;
  }
  PyObject* h = PyObject_GetAttrString(stream, "cuda_stream");
  if (!h) return false;
  *handle = PyLong_AsVoidPtr(h);
  Py_DECREF(h);
  return !PyErr_Occurred();
}
PyObject* finish(int status, const char* what, PyObject* given, at::Tensor&& out) {
  if (status != 0) {
    PyObject* r = PyObject_CallFunction(g_raise, "is", status, what);
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, what);
    return nullptr;
  }
  if (given != Py_None) {
    Py_INCREF(given);
    return given;
  }
  return THPVariable_Wrap(std::move(out));
}

int launch(int kind, const void* A, const void* w, const void* s, const void* x, void* C, int M, int K, int N, int G,
           void* ws, size_t ws_bytes, void* stream) {
  int st;
  Py_BEGIN_ALLOW_THREADS
  if (kind == kSparse)
    st = reinterpret_cast<GemmExtraFn>(g_fn[kind])(A, w, x, s, C, M, K, N, G, ws, ws_bytes, stream);
  else if (kind == kZero)
    st = reinterpret_cast<GemmExtraFn>(g_fn[kind])(A, w, s, x, C, M, K, N, G, ws, ws_bytes, stream);
  else
    st = reinterpret_cast<GemmFn>(g_fn[kind])(A, w, s, C, M, K, N, G, ws, ws_bytes, stream);
  Py_END_ALLOW_THREADS
  return st;
}

bool count_is(Py_ssize_t nargs, Py_ssize_t want) {
  if (nargs == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, nargs);
  return false;
}

// C++ exceptions of torch (out of memory, a bad device) become Python errors
#define TRY try {
#define CATCH                                      \
  }                                                \
  catch (const std::exception& e) {                \
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what()); \
    return nullptr;                                \
  }

// ---- one packed layer whose buffers were checked when it was built --------------------------------------------
struct LayerCall {
  PyObject_HEAD
  vectorcallfunc vectorcall;
  int kind, K, N, G, device;
  void *w, *s, *x, *ws;
  size_t ws_bytes;
};

PyObject* layer_call(PyObject* self, PyObject* const* args, size_t nargsf, PyObject* kwnames) {
  TRY
  const LayerCall* L = reinterpret_cast<LayerCall*>(self);
  if (kwnames && PyTuple_GET_SIZE(kwnames) != 0) {
    PyErr_SetString(PyExc_TypeError, "positional arguments only");
    return nullptr;
  }
  if (!count_is(PyVectorcall_NARGS(nargsf), 3)) return nullptr;
  const at::Tensor* A = tensor(args[0], "A");
  if (!A) return nullptr;
  if (A->scalar_type() != at::kHalf || !A->is_cuda() || !A->is_contiguous() || A->dim() != 2 || A->size(1) != L->K) {
    PyErr_SetString(PyExc_ValueError, "A must be a contiguous fp16 CUDA tensor [M, K]");
    return nullptr;
  }
  const int64_t M = A->size(0);
  at::Tensor out;
  if (args[1] == Py_None) {
    out = at::detail::empty_cuda({M, L->N}, at::kHalf, at::Device(at::kCUDA, (c10::DeviceIndex)L->device), std::nullopt);
  } else {
    const at::Tensor* o = tensor(args[1], "out");
    if (!o) return nullptr;
    if (o->scalar_type() != at::kHalf || !o->is_cuda() || !o->is_contiguous() || o->dim() != 2 || o->size(0) != M ||
        o->size(1) != L->N) {
      PyErr_SetString(PyExc_ValueError, "out must be a contiguous fp16 CUDA tensor [M, N]");
      return nullptr;
    }
    out = *o;
  }
  void* stream;
  if (!stream_handle(args[2], &stream)) return nullptr;
  const int st = launch(L->kind, A->data_ptr(), L->w, L->s, L->x, out.data_ptr(), (int)M, L->K, L->N, L->G, L->ws,
                        L->ws_bytes, stream);
  return finish(st, kNames[L->kind], args[1], std::move(out));
  CATCH
}

PyTypeObject LayerCallType = {PyVarObject_HEAD_INIT(nullptr, 0)};

// layer_call(kind, K, N, G, w, s, x, ws, ws_bytes, device): pointers as integers; the caller keeps the tensors alive
PyObject* make_layer_call(PyObject*, PyObject* args) {
  int kind, K, N, G, device;
  unsigned long long w, s, x, ws, ws_bytes;
  if (!PyArg_ParseTuple(args, "iiiiKKKKKi", &kind, &K, &N, &G, &w, &s, &x, &ws, &ws_bytes, &device)) return nullptr;
  if (kind < 0 || kind >= kKinds) {
    PyErr_SetString(PyExc_ValueError, "kind");
    return nullptr;
  }
  LayerCall* L = PyObject_New(LayerCall, &LayerCallType);
  if (!L) return nullptr;
  L->vectorcall = layer_call;
  L->kind = kind; L->K = K; L->N = N; L->G = G; L->device = device;
  L->w = reinterpret_cast<void*>(w); L->s = reinterpret_cast<void*>(s); L->x = reinterpret_cast<void*>(x);
  L->ws = reinterpret_cast<void*>(ws); L->ws_bytes = (size_t)ws_bytes;
  return reinterpret_cast<PyObject*>(L);
}

// ---- the module-level functions ---------------------------------------------------------------------------------
// gemm(kind, A, w_packed, s_packed, metadata, zero points or None, K, N, G, workspace, out or None, stream or None)
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  TRY
  if (!count_is(nargs, 11)) return nullptr;
  int kind, K, N, G;
  if (!integer(a[0], "kind", &kind) || !integer(a[5], "K", &K) || !integer(a[6], "N", &N) || !integer(a[7], "group_size", &G))
    return nullptr;
  const at::Tensor* A = activations(a[1], K);
  if (!A) return nullptr;
  const at::Tensor* w = device_tensor(a[2], at::kByte, "w_packed");
  if (!w) return nullptr;
  const at::Tensor* s = device_tensor(a[3], at::kByte, "s_packed");
  if (!s) return nullptr;
  const at::Tensor* x = nullptr;
  if ((kind == kSparse || kind == kZero) && !(x = device_tensor(a[4], at::kByte, kind == kSparse ? "meta_packed" : "z_packed")))
    return nullptr;
  const at::Tensor* ws = device_tensor(a[8], at::kByte, "workspace");
  if (!ws) return nullptr;
  const size_t wb = kind == kW8 ? g_weight_bytes_w8(K, N) : g_weight_bytes(K, N, kind == kSparse ? 1 : 0);
  const size_t sb = g_scale_bytes(K, N, G);
  const size_t xb = kind == kSparse ? g_meta_bytes(K, N) : sb;
  if ((size_t)w->numel() != wb || (size_t)s->numel() != sb || (x && (size_t)x->numel() != xb)) {
    PyErr_SetString(PyExc_ValueError, "packed buffer sizes do not match K, N, group_size");
    return nullptr;
  }
  const int64_t M = A->size(0);
  at::Tensor out;
  if (!output(a[9], M, kind == kSwiglu ? N / 2 : N, A->device(), "out", &out)) return nullptr;
  void* stream;
  if (!stream_handle(a[10], &stream)) return nullptr;
  const int st = launch(kind, A->data_ptr(), w->data_ptr(), s->data_ptr(), x ? x->data_ptr() : nullptr, out.data_ptr(),
                        (int)M, K, N, G, ws->data_ptr(), (size_t)ws->numel(), stream);
  return finish(st, kNames[kind], a[9], std::move(out));
  CATCH
}

// mlp(A, w_gate_up, s_gate_up, w_down, s_down, K, I, N, G, workspace, H or None, out or None, stream or None)
PyObject* mlp(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  TRY
  if (!count_is(nargs, 13)) return nullptr;
  int K, I, N, G;
  if (!integer(a[5], "K", &K) || !integer(a[6], "I", &I) || !integer(a[7], "N", &N) || !integer(a[8], "group_size", &G))
    return nullptr;
  const at::Tensor* A = activations(a[0], K);
  if (!A) return nullptr;
  const at::Tensor* ws = device_tensor(a[9], at::kByte, "workspace");
  if (!ws) return nullptr;
  static const char* const names[4] = {"w_gate_up", "s_gate_up", "w_down", "s_down"};
  const at::Tensor* t[4];
  for (int i = 0; i < 4; ++i)
    if (!(t[i] = device_tensor(a[1 + i], at::kByte, names[i]))) return nullptr;
  if ((size_t)t[0]->numel() != g_weight_bytes(K, 2 * I, 0) || (size_t)t[1]->numel() != g_scale_bytes(K, 2 * I, G) ||
      (size_t)t[2]->numel() != g_weight_bytes(I, N, 0) || (size_t)t[3]->numel() != g_scale_bytes(I, N, G)) {
    PyErr_SetString(PyExc_ValueError, "packed buffer sizes do not match K, I, N, group_size");
    return nullptr;
  }
  const int64_t M = A->size(0);
  at::Tensor H, out;
  if (!output(a[10], M, I, A->device(), "H", &H) || !output(a[11], M, N, A->device(), "out", &out)) return nullptr;
  void* stream;
  if (!stream_handle(a[12], &stream)) return nullptr;
  int st;
  const void *pa = A->data_ptr(), *p0 = t[0]->data_ptr(), *p1 = t[1]->data_ptr(), *p2 = t[2]->data_ptr(), *p3 = t[3]->data_ptr();
  void *ph = H.data_ptr(), *po = out.data_ptr(), *pw = ws->data_ptr();
  const size_t wsb = (size_t)ws->numel();
  Py_BEGIN_ALLOW_THREADS
  st = g_mlp(pa, p0, p1, p2, p3, ph, po, (int)M, K, I, N, G, pw, wsb, stream);
  Py_END_ALLOW_THREADS
  return finish(st, "marlin_mlp_swiglu", a[11], std::move(out));
  CATCH
}

// ---- the paged key-value cache ------------------------------------------------------------------------------------
const char* type_name(at::ScalarType type) {
  return type == at::kHalf ? "torch.float16" : type == at::kInt ? "torch.int32" : type == at::kLong ? "torch.int64" : type == at::kFloat ? "torch.float32" : "torch.uint8";
}
// `o` as a tensor of this type and these sizes (-1: any) on `device`, its elements side by side in the last dimension (and in
// all where `dense`); nullptr with a Python error set
const at::Tensor* argument(PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> sizes,
                           const at::Device& device, bool dense) {
  const at::Tensor* t = tensor(o, name);
  if (!t) return nullptr;
  if (!t->is_cuda()) {
    PyErr_Format(PyExc_TypeError, "%s must be a CUDA tensor", name);
    return nullptr;
  }
  if (t->scalar_type() != type) {
    PyErr_Format(PyExc_TypeError, "%s must have dtype %s", name, type_name(type));
    return nullptr;
  }
  if (t->device() != device) {
    PyErr_Format(PyExc_ValueError, "%s is on another device than the cache", name);
    return nullptr;
  }
  bool fits = t->dim() == (int64_t)sizes.size();
  for (size_t i = 0; fits && i < sizes.size(); ++i) fits = sizes.begin()[i] < 0 || t->size(i) == sizes.begin()[i];
  if (!fits) {
    PyErr_Format(PyExc_ValueError, "%s has the wrong shape", name);
    return nullptr;
  }
  if (dense ? !t->is_contiguous() : t->dim() > 0 && t->size(-1) > 1 && t->stride(-1) != 1) {
    PyErr_Format(PyExc_ValueError, "%s must be contiguous%s", name, dense ? "" : " in its last dimension");
    return nullptr;
  }
  return t;
}
// a row stride: of a single row it means nothing
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : 0; }

// The stream of a call: the one that is given, or the current one of the device of its tensors, which becomes the current device.
bool on_stream_of(PyObject* given, c10::DeviceIndex index, void** stream, std::optional<c10::cuda::CUDAGuard>* on_device,
                  std::optional<c10::cuda::CUDAStreamGuard>* on_stream) {
  if (given == Py_None) {
    if (c10::cuda::current_device() != index) on_device->emplace(index);
    *stream = c10::cuda::getCurrentCUDAStream(index).stream();
  } else {
    if (!stream_handle(given, stream)) return false;
    on_stream->emplace(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(*stream), index));
  }
  return true;
}

// the arguments that all calls on a cache have: (k_cache, v_cache, pages, lengths, workspace, starts, k_scale, v_scale, stream)
struct CacheCall {
  marlin_kv_cache c{};
  marlin_kv_scales by_block{};  // of an 8-bit cache with scales by block
  const marlin_kv_scales* scales = nullptr;  // that, or none
  const int32_t* starts = nullptr;
  void* workspace;
  size_t workspace_bytes;
  void* stream;
  at::Device device{at::kCUDA, 0};
  std::optional<c10::cuda::CUDAGuard> on_device;         // the library works on the current device
  std::optional<c10::cuda::CUDAStreamGuard> on_stream;   // outputs are taken from the pool of the stream that writes them
};
bool cache_arguments(PyObject* const* a, CacheCall* out) {
  const at::Tensor* k = tensor(a[0], "k_cache");
  if (!k) return false;
  const at::Tensor* v = tensor(a[1], "v_cache");
  if (!v) return false;
  marlin_kv_cache& c = out->c;
  if (!k->is_cuda() || !v->is_cuda()) {
    PyErr_SetString(PyExc_TypeError, "k_cache and v_cache must be CUDA tensors");
    return false;
  }
  if (k->scalar_type() == at::kHalf) {
    c.format = MARLIN_KV_FP16;
  } else if (k->scalar_type() == at::kFloat8_e4m3fn) {
    c.format = MARLIN_KV_E4M3;
  } else if (k->scalar_type() == at::kChar) {
    c.format = MARLIN_KV_INT8;
  } else {
    PyErr_SetString(PyExc_TypeError, "k_cache must have dtype torch.float16, torch.float8_e4m3fn or torch.int8");
    return false;
  }
  if (v->scalar_type() != k->scalar_type() || v->device() != k->device() || k->dim() != 4 || k->sizes() != v->sizes() ||
      k->strides() != v->strides() || k->numel() == 0 || (k->size(3) > 1 && k->stride(3) != 1)) {
    PyErr_SetString(PyExc_ValueError, "k_cache and v_cache must be [pages, heads, page_size, head_dim] alike, with elements side by side");
    return false;
  }
  out->device = k->device();
  for (int i = 0; i < 4; ++i)
    if (k->size(i) > INT_MAX) {
      PyErr_SetString(PyExc_ValueError, "k_cache is out of range");
      return false;
    }
  for (int i = 0; i < 3; ++i) {
    if (k->size(i) > 1 && k->stride(i) < k->size(3)) {
      PyErr_SetString(PyExc_ValueError, "k_cache: tokens overlap");
      return false;
    }
    c.stride[i] = k->size(i) > 1 ? k->stride(i) : 0;
  }
  c.k = k->data_ptr();
  c.v = v->data_ptr();
  c.pages = (int)k->size(0);
  c.kv_heads = (int)k->size(1);
  c.page_size = (int)k->size(2);
  c.head_dim = (int)k->size(3);
  const at::Tensor* lengths = argument(a[3], "lengths", at::kInt, {-1}, out->device, true);
  if (!lengths) return false;
  const at::Tensor* pages = argument(a[2], "pages", at::kInt, {lengths->size(0), -1}, out->device, false);
  if (!pages) return false;
  const at::Tensor* ws = argument(a[4], "workspace", at::kByte, {-1}, out->device, true);
  if (!ws) return false;
  if (lengths->size(0) > INT_MAX - 1 || pages->size(1) > INT_MAX) {
    PyErr_SetString(PyExc_ValueError, "pages is out of range");
    return false;
  }
  c.table = static_cast<const int32_t*>(pages->data_ptr());
  c.max_pages = (int)pages->size(1);
  c.table_stride = pages->size(0) > 1 ? pages->stride(0) : pages->size(1);
  c.lengths = static_cast<const int32_t*>(lengths->data_ptr());
  c.sequences = (int)lengths->size(0);
  out->workspace = ws->data_ptr();
  out->workspace_bytes = (size_t)ws->numel();
  if (a[5] != Py_None) {
    const at::Tensor* t = argument(a[5], "starts", at::kInt, {lengths->size(0) + 1}, out->device, true);
    if (!t) return false;
    out->starts = static_cast<const int32_t*>(t->data_ptr());
  }
  static const char* const names[2] = {"k_scale", "v_scale"};
  // scales by block, [pages, kv_heads, blocks of a page], of keys and values alike; or one per key head
  const bool three[2] = {a[6] != Py_None && THPVariable_Check(a[6]) && THPVariable_Unpack(a[6]).dim() == 3,
                         a[7] != Py_None && THPVariable_Check(a[7]) && THPVariable_Unpack(a[7]).dim() == 3};
  const bool by_block = three[0] || three[1] || c.format == MARLIN_KV_INT8;
  const at::Tensor* by[2] = {};
  for (int i = 0; i < 2; ++i) {
    if (a[6 + i] == Py_None) continue;
    if (c.format == MARLIN_KV_FP16) {
      PyErr_Format(PyExc_ValueError, "%s is for 8-bit caches", names[i]);
      return false;
    }
    if (by_block) {
      by[i] = argument(a[6 + i], names[i], at::kFloat, {k->size(0), k->size(1), -1}, out->device, false);
      if (!by[i]) return false;
      continue;
    }
    const at::Tensor* t = argument(a[6 + i], names[i], at::kFloat, {k->size(1)}, out->device, true);
    if (!t) return false;
    (i ? c.v_scale : c.k_scale) = static_cast<const float*>(t->data_ptr());
  }
  if (by_block) {
    if (!by[0] || !by[1]) {
      PyErr_SetString(PyExc_ValueError, "k_scale and v_scale must both be [pages, kv_heads, page_size / block]");
      return false;
    }
    const int64_t blocks = by[0]->size(2);
    if (by[0]->sizes() != by[1]->sizes() || by[0]->strides() != by[1]->strides() || blocks < 1 || k->size(2) % blocks) {
      PyErr_SetString(PyExc_ValueError, "k_scale and v_scale must be [pages, kv_heads, page_size / block] alike");
      return false;
    }
    marlin_kv_scales& s = out->by_block;
    for (int i = 0; i < 3; ++i) {
      s.stride[i] = by[0]->size(i) > 1 ? by[0]->stride(i) : 0;
      if (by[0]->size(i) > 1 && by[0]->stride(i) < 1) {
        PyErr_SetString(PyExc_ValueError, "k_scale: scales overlap");
        return false;
      }
    }
    s.k = static_cast<float*>(by[0]->data_ptr());
    s.v = static_cast<float*>(by[1]->data_ptr());
    s.block_size = (int)(k->size(2) / blocks);
    out->scales = &s;
  }
  return on_stream_of(a[8], out->device.index(), &out->stream, &out->on_device, &out->on_stream);
}
// rows of heads, [T, heads * head_dim]; `o` may be a range of columns of a wider tensor
const at::Tensor* rows_of_heads(PyObject* o, const char* name, const CacheCall& call, int* tokens, int64_t* heads) {
  const at::Tensor* t = argument(o, name, at::kHalf, {-1, -1}, call.device, false);
  if (!t) return nullptr;
  if (t->size(0) > INT_MAX || t->size(1) > INT_MAX || t->size(1) % call.c.head_dim || (t->size(0) > 1 && t->stride(0) < t->size(1))) {
    PyErr_Format(PyExc_ValueError, "%s must be [tokens, heads * head_dim]", name);
    return nullptr;
  }
  *tokens = (int)t->size(0);
  *heads = t->size(1) / call.c.head_dim;
  return t;
}
bool same_device(PyObject* given, const CacheCall& call, const char* name) {
  if (given == Py_None || !THPVariable_Check(given) || THPVariable_Unpack(given).device() == call.device) return true;
  PyErr_Format(PyExc_ValueError, "%s is on another device than the cache", name);
  return false;
}
// the frequencies of a rotation, or nullptr in *out where it is None; false with a Python error set
bool frequencies(PyObject* o, const CacheCall& call, const float** out, int* rotary_dim) {
  *out = nullptr;
  *rotary_dim = 0;
  if (o == Py_None) return true;
  const at::Tensor* t = argument(o, "inv_freq", at::kFloat, {-1}, call.device, true);
  if (!t) return false;
  if (t->numel() < 1 || 2 * t->numel() > call.c.head_dim) {
    PyErr_SetString(PyExc_ValueError, "inv_freq must be [rotary_dim / 2]");
    return false;
  }
  *out = static_cast<const float*>(t->data_ptr());
  *rotary_dim = (int)(2 * t->numel());
  return true;
}

// kv_append(qkv, k_cache, v_cache, pages, lengths, workspace, starts, k_scale, v_scale, stream, inv_freq, interleaved, out)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  TRY
  if (!count_is(nargs, 13)) return nullptr;
  CacheCall call;
  if (!cache_arguments(a + 1, &call)) return nullptr;
  int tokens, rotary_dim;
  int64_t heads;
  const at::Tensor* qkv = rows_of_heads(a[0], "qkv", call, &tokens, &heads);
  if (!qkv) return nullptr;
  const int64_t D = call.c.head_dim, kv = call.c.kv_heads, q_heads = heads - 2 * kv;
  const float* inv_freq;
  if (!frequencies(a[10], call, &inv_freq, &rotary_dim)) return nullptr;
  const int interleaved = PyObject_IsTrue(a[11]);
  if (interleaved < 0) return nullptr;
  if (q_heads < 0) {
    PyErr_SetString(PyExc_ValueError, "qkv must be [tokens, (q_heads + 2 * kv_heads) * head_dim]");
    return nullptr;
  }
  if (!inv_freq && a[12] != Py_None) {
    PyErr_SetString(PyExc_ValueError, "out: without inv_freq the queries stay where they are");
    return nullptr;
  }
  at::Tensor out;
  if (inv_freq) {
    if (!same_device(a[12], call, "out") || !output(a[12], tokens, q_heads * D, call.device, "out", &out)) return nullptr;
  } else {
    out = qkv->narrow(1, 0, q_heads * D);
  }
  const bool turn = inv_freq && q_heads > 0;
  const uint16_t* p = static_cast<const uint16_t*>(qkv->data_ptr());
  const int64_t stride = row_stride(*qkv);
  void* to = turn ? out.data_ptr() : nullptr;
  int st;
  Py_BEGIN_ALLOW_THREADS
  if (call.scales)
    st = g_append_scaled(turn ? p : nullptr, stride, p + q_heads * D, stride, p + (q_heads + kv) * D, stride, to, &call.c, call.scales,
                         call.starts, tokens, turn ? (int)q_heads : 0, inv_freq, rotary_dim, interleaved, call.workspace,
                         call.workspace_bytes, call.stream);
  else
    st = g_append(turn ? p : nullptr, stride, p + q_heads * D, stride, p + (q_heads + kv) * D, stride, to, &call.c, call.starts, tokens,
                  turn ? (int)q_heads : 0, inv_freq, rotary_dim, interleaved, call.workspace, call.workspace_bytes, call.stream);
  Py_END_ALLOW_THREADS
  return finish(st, call.scales ? "marlin_kv_append_scaled" : "marlin_kv_append", a[12], std::move(out));
  CATCH
}

// scale or None (1 / sqrt(head_dim)), window; false with a Python error set
bool softmax_arguments(PyObject* scale_o, PyObject* window_o, int head_dim, float* scale, int* window) {
  *scale = 1.f / std::sqrt((float)head_dim);
  if (scale_o != Py_None) {
    const double x = PyFloat_AsDouble(scale_o);
    if (x == -1.0 && PyErr_Occurred()) return false;
    *scale = (float)x;
  }
  return integer(window_o, "window", window);
}

// attention_decode(q, k_cache, v_cache, pages, lengths, workspace, starts, k_scale, v_scale, stream, scale, window, out, sinks)
PyObject* attention_decode(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  TRY
  if (!count_is(nargs, 14)) return nullptr;
  CacheCall call;
  if (!cache_arguments(a + 1, &call)) return nullptr;
  int tokens, window, sinks;
  int64_t heads;
  float scale;
  const at::Tensor* q = rows_of_heads(a[0], "q", call, &tokens, &heads);
  if (!q || !softmax_arguments(a[10], a[11], call.c.head_dim, &scale, &window) || !integer(a[13], "sinks", &sinks)) return nullptr;
  at::Tensor out;
  if (!same_device(a[12], call, "out") || !output(a[12], tokens, heads * call.c.head_dim, call.device, "out", &out)) return nullptr;
  const void* p = q->data_ptr();
  void* to = out.data_ptr();
  const int64_t stride = row_stride(*q);
  const bool more = call.scales || sinks != 0;
  int st;
  Py_BEGIN_ALLOW_THREADS
  if (more)
    st = g_attention_sinks(p, stride, &call.c, call.scales, call.starts, tokens, (int)heads, scale, window, sinks, to, call.workspace,
                           call.workspace_bytes, call.stream);
  else
    st = g_attention(p, stride, &call.c, call.starts, tokens, (int)heads, scale, window, to, call.workspace, call.workspace_bytes,
                     call.stream);
  Py_END_ALLOW_THREADS
  return finish(st, more ? "marlin_attention_sinks" : "marlin_attention_decode", a[12], std::move(out));
  CATCH
}

// attention_block(A, k_cache, v_cache, pages, lengths, workspace, starts, k_scale, v_scale, stream, inv_freq, interleaved, scale,
//                 window, w_qkv, s_qkv, w_o, s_o, K, q_heads, N, G, QKV, Q, O, out, sinks)
PyObject* attention_block(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  TRY
  if (!count_is(nargs, 27)) return nullptr;
  CacheCall call;
  if (!cache_arguments(a + 1, &call)) return nullptr;
  int K, q_heads, N, G, window, sinks, rotary_dim;
  float scale;
  const float* inv_freq;
  if (!frequencies(a[10], call, &inv_freq, &rotary_dim) || !softmax_arguments(a[12], a[13], call.c.head_dim, &scale, &window) ||
      !integer(a[18], "K", &K) || !integer(a[19], "q_heads", &q_heads) || !integer(a[20], "N", &N) || !integer(a[21], "group_size", &G) ||
      !integer(a[26], "sinks", &sinks))
    return nullptr;
  const int interleaved = PyObject_IsTrue(a[11]);
  if (interleaved < 0) return nullptr;
  const at::Tensor* A = argument(a[0], "A", at::kHalf, {-1, K}, call.device, true);
  if (!A) return nullptr;
  const int64_t M = A->size(0), q_cols = (int64_t)q_heads * call.c.head_dim;
  const int64_t columns = q_cols + 2 * (int64_t)call.c.kv_heads * call.c.head_dim;
  if (M > INT_MAX || q_heads < 1 || columns > INT_MAX || N < 1) {
    PyErr_SetString(PyExc_ValueError, "q_heads, N or the rows of A are out of range");
    return nullptr;
  }
  static const char* const names[4] = {"w_qkv", "s_qkv", "w_o", "s_o"};
  const at::Tensor* t[4];
  for (int i = 0; i < 4; ++i)
    if (!(t[i] = argument(a[14 + i], names[i], at::kByte, {-1}, call.device, true))) return nullptr;
  if ((size_t)t[0]->numel() != g_weight_bytes(K, (int)columns, 0) || (size_t)t[1]->numel() != g_scale_bytes(K, (int)columns, G) ||
      (size_t)t[2]->numel() != g_weight_bytes((int)q_cols, N, 0) || (size_t)t[3]->numel() != g_scale_bytes((int)q_cols, N, G)) {
    PyErr_SetString(PyExc_ValueError, "packed buffer sizes do not match K, q_heads, N, group_size");
    return nullptr;
  }
  at::Tensor QKV, Q, O, out;
  static const char* const scratch[4] = {"QKV", "Q", "O", "out"};
  for (int i = 0; i < 4; ++i)
    if (!same_device(a[22 + i], call, scratch[i])) return nullptr;
  if (!output(a[22], M, columns, call.device, "QKV", &QKV) || (inv_freq && !output(a[23], M, q_cols, call.device, "Q", &Q)) ||
      !output(a[24], M, q_cols, call.device, "O", &O) || !output(a[25], M, N, call.device, "out", &out))
    return nullptr;
  const void *pa = A->data_ptr(), *p[4];
  for (int i = 0; i < 4; ++i) p[i] = t[i]->data_ptr();
  void *pqkv = QKV.data_ptr(), *pq = inv_freq ? Q.data_ptr() : nullptr, *po = O.data_ptr(), *pc = out.data_ptr();
  const bool more = call.scales || sinks != 0;
  int st;
  Py_BEGIN_ALLOW_THREADS
  if (more)
    st = g_block_sinks(pa, p[0], p[1], p[2], p[3], pqkv, pq, po, pc, &call.c, call.scales, call.starts, (int)M, K, q_heads, N, G, inv_freq,
                       rotary_dim, interleaved, scale, window, sinks, call.workspace, call.workspace_bytes, call.stream);
  else
    st = g_block(pa, p[0], p[1], p[2], p[3], pqkv, pq, po, pc, &call.c, call.starts, (int)M, K, q_heads, N, G, inv_freq, rotary_dim,
                 interleaved, scale, window, call.workspace, call.workspace_bytes, call.stream);
  Py_END_ALLOW_THREADS
  return finish(st, more ? "marlin_attention_block_sinks" : "marlin_attention_block", a[25], std::move(out));
  CATCH
}

// an output of a call, in one dimension: `given`, or a new one
bool vector_output(PyObject* given, int64_t n, at::ScalarType type, const at::Device& device, const char* name, at::Tensor* out) {
  if (given == Py_None) {
    *out = at::Tensor(at::detail::empty_cuda({n}, type, device, std::nullopt));
    return true;
  }
  const at::Tensor* t = argument(given, name, type, {n}, device, true);
  if (t) *out = *t;
  return t != nullptr;
}

// kv_reserve(lengths, pages, free_pages, free_count, workspace, page_size, tokens, counts, keep, starts, slots, positions, stream)
PyObject* kv_reserve(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  TRY
  if (!count_is(nargs, 13)) return nullptr;
  const at::Tensor* lengths = tensor(a[0], "lengths");
  if (!lengths) return nullptr;
  const at::Device device = lengths->device();
  if (!(lengths = argument(a[0], "lengths", at::kInt, {-1}, device, true))) return nullptr;
  const int64_t sequences = lengths->size(0);
  const at::Tensor* table = argument(a[1], "pages", at::kInt, {sequences, -1}, device, false);
  if (!table) return nullptr;
  const at::Tensor* free_pages = argument(a[2], "free_pages", at::kInt, {-1}, device, true);
  if (!free_pages) return nullptr;
  const at::Tensor* free_count = argument(a[3], "free_count", at::kInt, {1}, device, true);
  if (!free_count) return nullptr;
  const at::Tensor* ws = argument(a[4], "workspace", at::kByte, {-1}, device, true);
  if (!ws) return nullptr;
  int page_size, tokens;
  if (!integer(a[5], "page_size", &page_size) || !integer(a[6], "tokens", &tokens)) return nullptr;
  if (sequences < 1 || sequences > INT_MAX - 1 || table->size(1) > INT_MAX || free_pages->numel() > INT_MAX || tokens < 0 ||
      (sequences > 1 && table->stride(0) < table->size(1))) {
    PyErr_SetString(PyExc_ValueError, "lengths, pages, free_pages or tokens is out of range");
    return nullptr;
  }
  const int32_t* of[2] = {};
  static const char* const names[2] = {"counts", "keep"};
  for (int i = 0; i < 2; ++i) {
    if (a[7 + i] == Py_None) continue;
    const at::Tensor* t = argument(a[7 + i], names[i], at::kInt, {sequences}, device, true);
    if (!t) return nullptr;
    of[i] = static_cast<const int32_t*>(t->data_ptr());
  }
  std::optional<c10::cuda::CUDAGuard> on_device;
  std::optional<c10::cuda::CUDAStreamGuard> on_stream;
  void* stream;
  if (!on_stream_of(a[12], device.index(), &stream, &on_device, &on_stream)) return nullptr;
  at::Tensor starts, slots, positions;
  if (!vector_output(a[9], sequences + 1, at::kInt, device, "starts", &starts) ||
      !vector_output(a[10], tokens, at::kLong, device, "slots", &slots) ||
      !vector_output(a[11], tokens, at::kInt, device, "positions", &positions))
    return nullptr;
  marlin_kv_pages c{};
  c.table = static_cast<int32_t*>(table->data_ptr());
  c.table_stride = sequences > 1 ? table->stride(0) : table->size(1);
  c.lengths = static_cast<int32_t*>(lengths->data_ptr());
  c.free_pages = static_cast<int32_t*>(free_pages->data_ptr());
  c.free_count = static_cast<int32_t*>(free_count->data_ptr());
  c.capacity = (int)free_pages->numel();
  c.max_pages = (int)table->size(1);
  c.sequences = (int)sequences;
  c.page_size = page_size;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = g_reserve(&c, of[0], of[1], tokens, static_cast<int32_t*>(starts.data_ptr()),
                 tokens ? static_cast<int64_t*>(slots.data_ptr()) : nullptr, tokens ? static_cast<int32_t*>(positions.data_ptr()) : nullptr,
                 ws->data_ptr(), (size_t)ws->numel(), stream);
  Py_END_ALLOW_THREADS
  if (st != 0) return finish(st, "marlin_kv_reserve", Py_None, at::Tensor());
  return Py_BuildValue("(NNN)", THPVariable_Wrap(std::move(starts)), THPVariable_Wrap(std::move(slots)), THPVariable_Wrap(std::move(positions)));
  CATCH
}

// bind(addresses, raise): addresses of the library's entry points by name
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *table, *raise;
  if (!PyArg_ParseTuple(args, "O!O", &PyDict_Type, &table, &raise)) return nullptr;
  bool ok = true;
  auto address = [&](const char* name) -> void* {
    PyObject* v = PyDict_GetItemString(table, name);
    void* p = v ? PyLong_AsVoidPtr(v) : nullptr;
    if (!p) ok = false;
    return p;
  };
  for (int k = 0; k < kKinds; ++k) g_fn[k] = address(kNames[k]);
  g_mlp = reinterpret_cast<MlpFn>(address("marlin_mlp_swiglu"));
  g_append = reinterpret_cast<decltype(g_append)>(address("marlin_kv_append"));
  g_attention = reinterpret_cast<decltype(g_attention)>(address("marlin_attention_decode"));
  g_block = reinterpret_cast<decltype(g_block)>(address("marlin_attention_block"));
  g_append_scaled = reinterpret_cast<decltype(g_append_scaled)>(address("marlin_kv_append_scaled"));
  g_attention_sinks = reinterpret_cast<decltype(g_attention_sinks)>(address("marlin_attention_sinks"));
  g_block_sinks = reinterpret_cast<decltype(g_block_sinks)>(address("marlin_attention_block_sinks"));
  g_reserve = reinterpret_cast<decltype(g_reserve)>(address("marlin_kv_reserve"));
  g_weight_bytes = reinterpret_cast<SizeFn>(address("marlin_packed_weight_bytes"));
  g_scale_bytes = reinterpret_cast<SizeFn>(address("marlin_packed_scale_bytes"));
  g_meta_bytes = reinterpret_cast<SizeFn2>(address("marlin_packed_meta_bytes"));
  g_weight_bytes_w8 = reinterpret_cast<SizeFn2>(address("marlin_packed_weight_bytes_w8"));
  if (!ok) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, "an entry point is missing");
    return nullptr;
  }
  Py_INCREF(raise);
  Py_XDECREF(g_raise);
  g_raise = raise;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"layer_call", make_layer_call, METH_VARARGS, nullptr},
    {"gemm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(gemm)), METH_FASTCALL, nullptr},
    {"mlp", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(mlp)), METH_FASTCALL, nullptr},
    {"kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(kv_append)), METH_FASTCALL, nullptr},
    {"attention_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(attention_decode)), METH_FASTCALL, nullptr},
    {"attention_block", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(attention_block)), METH_FASTCALL, nullptr},
    {"kv_reserve", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(kv_reserve)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_binding", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__torch_binding(void) {
  LayerCallType.tp_name = "_torch_binding.LayerCall";
  LayerCallType.tp_basicsize = sizeof(LayerCall);
  LayerCallType.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_VECTORCALL;
  LayerCallType.tp_vectorcall_offset = offsetof(LayerCall, vectorcall);
  LayerCallType.tp_call = PyVectorcall_Call;
  if (PyType_Ready(&LayerCallType) < 0) return nullptr;
  return PyModule_Create(&module);
}
