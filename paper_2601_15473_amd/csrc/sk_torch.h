// What the native functions of the PyTorch surface share: scratch buffers, errors, and which calls they take.
#pragma once
#include <Python.h>

#include <dlfcn.h>
#include <stdlib.h>

#include <list>
#include <mutex>
#include <string>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#define __HIP_PLATFORM_AMD__ 1
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>

#include "../../include/sk.h"

namespace sk_torch {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

// One scratch buffer per (device, stream), grown to the largest request up to MAX_KEPT; the least recently used of more
// than MAX_STREAMS goes back to the allocator, which keeps it until the work queued on it is done.
// Calls queue their kernels under the lock: two threads that share a stream share its buffer.
// A call that is being recorded into a graph gets a buffer of its own, out of the graph's memory: every replay writes there,
// long after a stream's buffer may have been replaced or given back.
struct Workspaces {
  static constexpr size_t MAX_STREAMS = 8;
  // Most that a pass keeps here beside its workspace: an allocation a pass is 1 us of host, 1 to 2 % of a small two-sided layer's step, and the sums
  // of a large one (4096 -> 11008, 2048 columns: 107 MB) would stay on every stream.
  static constexpr size_t MAX_SUMS = 4 << 20;
  // Most that a stream keeps: a call that needs more (attention's parts can be 130 MB) has its own, which the allocator hands on when the call is queued.
  // It does not notice the allocation.
  static constexpr size_t MAX_KEPT = 64 << 20;
  struct Entry {
    c10::DeviceIndex device;
    void* stream;
    Tensor buffer;
  };
  std::mutex mutex;
  std::list<Entry> entries;   // most recently used first

  static Tensor made(const at::Device& device, size_t bytes) {
    return at::empty({(int64_t)(bytes < 256 ? 256 : bytes)}, at::TensorOptions().dtype(at::kByte).device(device));
  }
  static bool recording(void* stream) {
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(static_cast<hipStream_t>(stream), &status) != hipSuccess) {   // (the null stream's answer while another one is recorded)
      (void)hipGetLastError();
      return false;
    }
    return status != hipStreamCaptureStatusNone;
  }

  // For calls that are queued before the tensor and the lock go (the lock is held).
  Tensor get(const at::Device& device, void* stream, size_t bytes) {
    if (bytes > MAX_KEPT || recording(stream)) return made(device, bytes);
    auto it = entries.begin();
    while (it != entries.end() && !(it->device == device.index() && it->stream == stream)) ++it;
    if (it == entries.end()) entries.push_front(Entry{device.index(), stream, Tensor()});
    else if (it != entries.begin()) entries.splice(entries.begin(), entries, it);
    Entry& e = entries.front();
    if (!e.buffer.defined() || (size_t)e.buffer.numel() < bytes) e.buffer = made(device, bytes);
    if (entries.size() > MAX_STREAMS) entries.pop_back();
    return e.buffer;
  }
};
// (never destroyed: the allocator may be gone before this library's own destructors run)
inline Workspaces& workspaces() {
  static Workspaces* w = new Workspaces;
  return *w;
}

inline sk_dtype dtype_of(const Tensor& t) { return t.scalar_type() == at::kFloat ? SK_F32 : SK_BF16; }

inline void* stream_of(const at::Device& device) {
  return static_cast<hipStream_t>(c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(device.index()).stream());
}

inline PyObject* g_error = nullptr;   // libsk.SkError, which nn.py hands over

// As libsk.check: raises SkError with its status.  (Not under the workspaces' lock: it takes the GIL and runs Python.)
inline void check(sk_status s) {
  if (s == SK_OK) return;
  pybind11::gil_scoped_acquire gil;
  PyObject* const e = g_error != nullptr ? PyObject_CallFunction(g_error, "i", (int)s) : nullptr;
  if (e != nullptr) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_RuntimeError, sk_status_string(s));
  }
  python_error error;
  error.persist();   // (a backward pass is on another thread than its caller)
  throw error;
}

inline PyTypeObject* g_parameter = nullptr;   // torch.nn.Parameter

// A plain tensor or parameter on `device` (any, if null) with the given type and dense rows
inline const Tensor* plain(PyObject* o) {
  PyTypeObject* const type = Py_TYPE(o);
  if (type != reinterpret_cast<PyTypeObject*>(THPVariableClass) && type != g_parameter) return nullptr;
  const Tensor& t = THPVariable_Unpack(o);
  return t.defined() && t.is_cuda() && t.layout() == at::kStrided && !t.is_conj() && !t.is_neg() ? &t : nullptr;
}

// Nothing is watching that the native functions would pass by.
inline bool unwatched() {
  using at::DispatchKey;
  for (DispatchKey k : {DispatchKey::FuncTorchDynamicLayerFrontMode, DispatchKey::FuncTorchDynamicLayerBackMode, DispatchKey::Tracer, DispatchKey::Functionalize})
    if (c10::impl::tls_is_dispatch_key_included(k)) return false;
  return !c10::impl::TorchDispatchModeTLS::any_modes_set() && !at::impl::torch_function_mode_enabled();
}
inline bool no_tangent(const Tensor& t) { return !t._fw_grad(0).defined(); }

inline bool aligned(const Tensor& t) { return (reinterpret_cast<uintptr_t>(t.data_ptr()) & 15) == 0; }

}  // namespace sk_torch
