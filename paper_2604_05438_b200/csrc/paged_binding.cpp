// CPython module of the paged calls: checks the tensors of a call, fills the C descriptors and calls libtkphi.
// Single-token calls are shorter on the GPU than the same checks written in Python (5 us of 8 for an append), which is
// why these calls do not go through ctypes as the others do.  Marshalling only.
#include <torch/csrc/autograd/python_variable.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <cstring>
#include <limits>
#include <memory>
#include <vector>

#include "../../include/tkphi.h"

namespace {

// What a PagedKVCache object stands for: the C descriptor and the shapes that a call's tensors must have; and the tensors
// that the object made itself (lengths, status), which a call on another stream than theirs has to wait for and to mark as
// used there, because the caller does not know them.
struct Handle {
  tkphi_paged_desc desc;
  at::ScalarType type;
  int device;
  int64_t total_q;
  std::vector<at::Tensor> made;
  cudaStream_t made_on = nullptr;
  cudaEvent_t ready = nullptr;             // behind their making, where that is not complete yet
  ~Handle() {
    if (ready) cudaEventDestroy(ready);
  }
};
const char* kCapsule = "paged cache";

Handle* handle_of(PyObject* o) { return static_cast<Handle*>(PyCapsule_GetPointer(o, kCapsule)); }
void free_handle(PyObject* o) { delete handle_of(o); }

// handle(address of the ctypes descriptor, device index, tuple of the tensors made, whether their making may be pending)
PyObject* make_handle(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 4 || !PyTuple_Check(args[2])) { PyErr_SetString(PyExc_TypeError, "handle(descriptor, device, tensors, pending)"); return nullptr; }
  const void* src = PyLong_AsVoidPtr(args[0]);
  const long dev = PyLong_AsLong(args[1]);
  const int pending = PyObject_IsTrue(args[3]);
  if (PyErr_Occurred()) return nullptr;
  try {
    std::unique_ptr<Handle> h(new Handle);
    std::memcpy(&h->desc, src, sizeof(h->desc));
    h->type = h->desc.dtype == TKPHI_DTYPE_BF16 ? at::kBFloat16 : at::kHalf;
    h->device = (int)dev;
    h->total_q = h->desc.cu_q_host[h->desc.batch];
    if (dev >= 0) {
      const c10::cuda::CUDAGuard guard((c10::DeviceIndex)dev);
      for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(args[2]); ++i) h->made.push_back(THPVariable_Unpack(PyTuple_GET_ITEM(args[2], i)));
      h->made_on = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
      cudaStreamCaptureStatus captured = cudaStreamCaptureStatusNone;
      // (made within a capture, the tensors belong to its graph, whose calls are ordered by it)
      if (pending && cudaStreamIsCapturing(h->made_on, &captured) == cudaSuccess && captured == cudaStreamCaptureStatusNone)
        if (cudaEventCreateWithFlags(&h->ready, cudaEventDisableTiming) != cudaSuccess || cudaEventRecord(h->ready, h->made_on) != cudaSuccess) {
          PyErr_SetString(PyExc_RuntimeError, "no event for the cache's stream");
          return nullptr;
        }
    }
    return PyCapsule_New(h.release(), kCapsule, free_handle);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

struct Refused {};

[[noreturn]] void refuse(const char* what, const char* why) {
  PyErr_Format(PyExc_ValueError, "%s %s", what, why);
  throw Refused{};
}

// A tensor argument on the cache's device with the given type and sizes; the last dim contiguous, all of it where asked.
void* take(const Handle* h, PyObject* o, const char* what, at::ScalarType type, std::initializer_list<int64_t> sizes,
           bool contiguous, int64_t* stride_0 = nullptr, int64_t* stride_1 = nullptr) {
  if (!THPVariable_Check(o)) refuse(what, "must be a tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.scalar_type() != type) refuse(what, "has another type than the call takes");
  if (!t.is_cuda() || t.get_device() != h->device) refuse(what, "is not on the cache's device");
  if (t.sizes() != at::IntArrayRef(sizes)) refuse(what, "has another shape than the call takes");
  if (contiguous ? !t.is_contiguous() : t.stride(t.dim() - 1) != 1 && t.numel() != 0)
    refuse(what, contiguous ? "must be contiguous" : "must be contiguous in its last dim");
  if (stride_0) { *stride_0 = t.stride(0); *stride_1 = t.stride(1); }
  return t.data_ptr();
}

void* take_heads(const Handle* h, PyObject* o, const char* what, int64_t heads, bool contiguous, int64_t* s0 = nullptr,
                 int64_t* s1 = nullptr) {
  return take(h, o, what, h->type, {h->total_q, heads, h->desc.head_dim}, contiguous, s0, s1);
}

float* take_lse(const Handle* h, PyObject* o) {
  return o == Py_None ? nullptr : static_cast<float*>(take(h, o, "lse_out", at::kFloat, {h->total_q, h->desc.n_q_heads}, true));
}

void* take_workspace(const Handle* h, PyObject* o, size_t* bytes) {
  if (!THPVariable_Check(o)) refuse("workspace", "must be a tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.get_device() != h->device || !t.is_contiguous()) refuse("workspace", "must be contiguous on the cache's device");
  *bytes = t.nbytes();
  return t.data_ptr();
}

float take_scale(PyObject* o) {
  if (o == Py_None) return 0.f;
  const double s = PyFloat_AsDouble(o);
  if (PyErr_Occurred()) throw Refused{};
  // (in 32 bits, as the library takes it: there 0 stands for 1 / sqrt(head_dim))
  if (!((float)s > 0.f && (float)s <= std::numeric_limits<float>::max())) refuse("scale", "must be positive and finite in 32 bits");
  return (float)s;
}

uint32_t take_flags(PyObject* o) {
  const unsigned long f = PyLong_AsUnsignedLong(o);
  if (PyErr_Occurred()) throw Refused{};
  if (f > 0xffffffffu) refuse("flags", "has unknown bits");
  return (uint32_t)f;
}

// The stream argument (None: the current one of the cache's device).
void* take_stream(const Handle* h, PyObject* o) {
  cudaStream_t s = nullptr;
  if (o == Py_None) {
    s = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)h->device).stream();
  } else {
    PyObject* raw = PyObject_GetAttrString(o, "cuda_stream");
    if (!raw) throw Refused{};
    s = static_cast<cudaStream_t>(PyLong_AsVoidPtr(raw));
    Py_DECREF(raw);
    if (PyErr_Occurred()) throw Refused{};
  }
  if (s != h->made_on && !h->made.empty()) {
    cudaStreamCaptureStatus captured = cudaStreamCaptureStatusNone;
    // (a captured call cannot wait for what was enqueued before the capture; the capture itself begins behind it)
    if (h->ready && cudaStreamIsCapturing(s, &captured) == cudaSuccess && captured == cudaStreamCaptureStatusNone &&
        cudaStreamWaitEvent(s, h->ready, 0) != cudaSuccess) {
      PyErr_SetString(PyExc_RuntimeError, "the call's stream cannot wait for the cache's");
      throw Refused{};
    }
    const c10::cuda::CUDAStream used = c10::cuda::getStreamFromExternal(s, (c10::DeviceIndex)h->device);
    for (const at::Tensor& t : h->made) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), used);
  }
  return s;
}

// Runs a call's body with the cache's device current; its status is the result.
template <typename F>
PyObject* run(PyObject* const* args, Py_ssize_t n, Py_ssize_t want, F body) {
  try {
    if (n != want) { PyErr_Format(PyExc_TypeError, "%zd arguments, expected %zd", n, want); return nullptr; }
    const Handle* h = handle_of(args[0]);
    if (!h) return nullptr;
    const c10::cuda::OptionalCUDAGuard guard(h->device >= 0 ? std::optional<c10::DeviceIndex>(h->device) : std::nullopt);
    return PyLong_FromLong(body(h));
  } catch (const Refused&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// append(handle, k_new, v_new, inv_freq, pairs, q, q_out, positions, stream)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(a, n, 9, [&](const Handle* h) {
    tkphi_append_desc d{};
    const int64_t hkv = h->desc.n_kv_heads, hq = h->desc.n_q_heads;
    d.pairs = PyObject_IsTrue(a[4]);
    if (d.pairs < 0) throw Refused{};                  // (something without a truth value)
    d.k_new = take_heads(h, a[1], "k_new", hkv, false, &d.k_stride_token, &d.k_stride_head);
    d.v_new = take_heads(h, a[2], "v_new", hkv, false, &d.v_stride_token, &d.v_stride_head);
    if (a[3] != Py_None) {
      if (!THPVariable_Check(a[3])) refuse("inv_freq", "must be a tensor");
      const int64_t half = THPVariable_Unpack(a[3]).numel();
      d.inv_freq = static_cast<const float*>(take(h, a[3], "inv_freq", at::kFloat, {half}, true));
      d.rot_dim = half > 1 << 20 ? -1 : (int32_t)(2 * half);
    }
    if (a[5] != Py_None) d.q = take_heads(h, a[5], "q", hq, false, &d.q_stride_token, &d.q_stride_head);
    if (a[6] != Py_None) d.q_out = take_heads(h, a[6], "q_out", hq, false, &d.o_stride_token, &d.o_stride_head);
    if (a[7] != Py_None) d.positions = static_cast<const int64_t*>(take(h, a[7], "positions", at::kLong, {h->total_q}, true));
    return tkphi_paged_append(&h->desc, &d, take_stream(h, a[8]));
  });
}

// attention(handle, q, y_out, lse_out, scale, flags, workspace, stream)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(a, n, 8, [&](const Handle* h) {
    const float scale = take_scale(a[4]);
    const uint32_t flags = take_flags(a[5]);
    const void* q = take_heads(h, a[1], "q", h->desc.n_q_heads, true);
    void* y = take_heads(h, a[2], "y_out", h->desc.n_q_heads, true);
    float* lse = take_lse(h, a[3]);
    size_t bytes = 0;
    void* ws = take_workspace(h, a[6], &bytes);
    return tkphi_paged_attention(&h->desc, q, y, lse, scale, flags, ws, bytes, take_stream(h, a[7]));
  });
}

// block_attention(handle, n_sink, n_tail, topk, q, y_out, lse_out, page_idx_out, scale, workspace, stream)
PyObject* block_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(a, n, 11, [&](const Handle* h) {
    int32_t v[3];
    for (int i = 0; i < 3; ++i) {
      const long x = PyLong_AsLong(a[1 + i]);
      if (PyErr_Occurred()) throw Refused{};
      if (x < -1 || x > 1 << 24) refuse("selection", "has a page count out of range");
      v[i] = (int32_t)x;
    }
    const tkphi_page_selection sel{v[0], v[1], v[2]};
    const float scale = take_scale(a[8]);
    const void* q = take_heads(h, a[4], "q", h->desc.n_q_heads, true);
    void* y = take_heads(h, a[5], "y_out", h->desc.n_q_heads, true);
    float* lse = take_lse(h, a[6]);
    int32_t* idx = nullptr;
    if (a[7] != Py_None)
      idx = static_cast<int32_t*>(take(h, a[7], "page_idx_out", at::kInt, {h->total_q, h->desc.n_kv_heads, (int64_t)v[0] + v[1] + v[2]}, true));
    size_t bytes = 0;
    void* ws = take_workspace(h, a[9], &bytes);
    return tkphi_paged_block_attention(&h->desc, &sel, q, y, lse, idx, scale, ws, bytes, take_stream(h, a[10]));
  });
}

// (a fast call has another signature than the table's)
PyCFunction fast(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef methods[] = {
    {"handle", fast(make_handle), METH_FASTCALL, nullptr},
    {"append", fast(append), METH_FASTCALL, nullptr},
    {"attention", fast(attention), METH_FASTCALL, nullptr},
    {"block_attention", fast(block_attention), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged_binding(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", TKPHI_TORCH_VERSION) < 0) { Py_DECREF(m); return nullptr; }
  return m;
}
