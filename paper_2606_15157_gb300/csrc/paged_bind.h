// paged_bind.h -- what the extension modules of the paged calls (paged_bind.cpp, paged_q8_bind.cpp) share:
// arguments from Python, their checks, and the call's device and stream.
#pragma once
#include <Python.h>
#include <climits>
#include <stdexcept>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <cuda_runtime_api.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/kvev.h"

namespace {

struct Refused {};

[[noreturn]] inline void refuse(const char* name, const char* what) {
  PyErr_Format(PyExc_ValueError, "%s: %s", name, what);
  throw Refused();
}

inline const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(name, "a tensor");
  return THPVariable_Unpack(o);
}

inline long long number(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  return v;
}

inline int small(PyObject* o, const char* name) {
  const long long v = number(o);
  if (v < INT_MIN || v > INT_MAX) refuse(name, "out of range");
  return static_cast<int>(v);
}

inline void* address(PyObject* o) { return reinterpret_cast<void*>(static_cast<uintptr_t>(number(o))); }

inline void on_device(const at::Tensor& t, int device, const char* name) {
  if (!t.is_cuda() || t.get_device() != device) refuse(name, "on the cache's GPU");
}

// A contiguous int32 tensor of n elements (n < 0: any number).
inline int32_t* ints(PyObject* o, int64_t n, int device, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != at::kInt || !t.is_contiguous() || (n >= 0 && t.numel() != n))
    refuse(name, "a contiguous int32 tensor with an element per request, token or count");
  on_device(t, device, name);
  return static_cast<int32_t*>(t.data_ptr());
}

inline int64_t count(PyObject* o, const char* name) { return tensor(o, name).numel(); }

// Makes the GPU current for the call.  (The guard by itself also asks at its end which one is: 0.1 us of an
// attention call's 2.9, on the host.)
struct OnDevice {
  c10::cuda::OptionalCUDAGuard guard;
  explicit OnDevice(int device) {
    c10::DeviceIndex at = -1;
    const cudaError_t e = c10::cuda::GetDevice(&at);
    if (e != cudaSuccess) throw std::runtime_error(cudaGetErrorString(e));
    if (at != device) guard.set_index(static_cast<c10::DeviceIndex>(device));
  }
};

// The stream's number, or the device's current stream for None.
inline void* stream_of(PyObject* o, int device) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
  return address(o);
}

inline at::ScalarType type_of(int dtype) { return dtype == KVEV_FP16 ? at::kHalf : at::kBFloat16; }

// [tokens][heads][d] rows of the cache's type, d contiguous.  The stride of a dimension of one
// element means nothing: it is taken as if contiguous.
struct Rows {
  void* at;
  int64_t tokens, heads, token_stride, head_stride;
};
inline Rows rows(PyObject* o, int d, int dtype, int device, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != 3 || t.size(2) != d || t.scalar_type() != type_of(dtype))
    refuse(name, "[tokens][heads][d] of the cache's type");
  if (t.stride(2) != 1) refuse(name, "the last dimension is contiguous");
  on_device(t, device, name);
  Rows r = {t.data_ptr(), t.size(0), t.size(1), t.stride(0), t.stride(1)};
  if (r.heads == 1) r.head_stride = d;
  if (r.tokens == 1) r.token_stride = r.heads * r.head_stride;
  if (r.tokens > INT_MAX || r.heads > INT_MAX) refuse(name, "out of range");
  return r;
}

// The rows' log-sum-exp, None: not wanted.
inline float* lse_of(PyObject* o, const Rows& q, int device) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, "lse");
  if (t.scalar_type() != at::kFloat || t.dim() != 2 || t.size(0) != q.tokens || t.size(1) != q.heads || !t.is_contiguous())
    refuse("lse", "contiguous float32 [tokens][heads]");
  on_device(t, device, "lse");
  return static_cast<float*>(t.data_ptr());
}

inline int requests(int64_t B, PyObject* most) {
  if (B > number(most)) refuse("requests", "more than the block table has rows");
  return static_cast<int>(B);
}

template <class F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t want, F f) {
  try {
    if (got != want) {
      PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, got);
      throw Refused();
    }
    return PyLong_FromLong(f());
  } catch (const Refused&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}

}  // namespace
