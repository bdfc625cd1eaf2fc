// paged_bind.cpp -- the calls of paged.py on torch tensors: their checks and the call of the
// C entry point in one function each.  These calls take 2 to 4 us on the device and are made
// for every layer of every token; through Python's own attribute reads and ctypes the
// host's share was larger (a tables call 6.1 us, a write 4.4, an attention 8.1; here 2.2, 1.9
// and 2.9).
//
// Each function returns the entry point's status code and raises ValueError where a tensor has
// the wrong type, shape or place.  The entry points launch on the current device: each call makes
// the tensors' GPU current for its time.
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

[[noreturn]] void refuse(const char* name, const char* what) {
  PyErr_Format(PyExc_ValueError, "%s: %s", name, what);
  throw Refused();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(name, "a tensor");
  return THPVariable_Unpack(o);
}

long long number(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  return v;
}

int small(PyObject* o, const char* name) {
  const long long v = number(o);
  if (v < INT_MIN || v > INT_MAX) refuse(name, "out of range");
  return static_cast<int>(v);
}

void* address(PyObject* o) { return reinterpret_cast<void*>(static_cast<uintptr_t>(number(o))); }

void on_device(const at::Tensor& t, int device, const char* name) {
  if (!t.is_cuda() || t.get_device() != device) refuse(name, "on the cache's GPU");
}

// A contiguous int32 tensor of n elements (n < 0: any number).
int32_t* ints(PyObject* o, int64_t n, int device, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != at::kInt || !t.is_contiguous() || (n >= 0 && t.numel() != n))
    refuse(name, "a contiguous int32 tensor with an element per request, token or count");
  on_device(t, device, name);
  return static_cast<int32_t*>(t.data_ptr());
}

int64_t count(PyObject* o, const char* name) { return tensor(o, name).numel(); }

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
void* stream_of(PyObject* o, int device) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
  return address(o);
}

// [tokens][heads][d] rows of the cache's type, d contiguous.  The stride of a dimension of one
// element means nothing: it is taken as if contiguous.
struct Rows {
  void* at;
  int64_t tokens, heads, token_stride, head_stride;
};
Rows rows(PyObject* o, const kvev_paged_cache& c, int device, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != 3 || t.size(2) != c.d || t.scalar_type() != (c.dtype == KVEV_FP16 ? at::kHalf : at::kBFloat16))
    refuse(name, "[tokens][heads][d] of the cache's type");
  if (t.stride(2) != 1) refuse(name, "the last dimension is contiguous");
  on_device(t, device, name);
  Rows r = {t.data_ptr(), t.size(0), t.size(1), t.stride(0), t.stride(1)};
  if (r.heads == 1) r.head_stride = c.d;
  if (r.tokens == 1) r.token_stride = r.heads * r.head_stride;
  if (r.tokens > INT_MAX || r.heads > INT_MAX) refuse(name, "out of range");
  return r;
}

const kvev_paged_cache& cache(PyObject* o) { return *static_cast<const kvev_paged_cache*>(address(o)); }

int requests(int64_t B, PyObject* most) {
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

// (pool: page_size, num_pages, free, block_table, max_requests, max_pages, device_status, device), stream, ...
PyObject* tables(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 19, [&] {
    const int dev = small(a[7], "device");
    const OnDevice on(dev);
    const int B = requests(count(a[9], "lens"), a[4]), T = small(a[11], "T");
    return kvev_paged_tables(ints(a[9], B, dev, "lens"), ints(a[10], B, dev, "new_lens"), B, small(a[0], "page_size"),
                             small(a[1], "num_pages"), static_cast<int32_t*>(address(a[2])), ints(a[17], 1, dev, "free_count"),
                             static_cast<int32_t*>(address(a[3])), small(a[5], "max_pages"), T, ints(a[12], B, dev, "kv_lens"),
                             ints(a[13], B + 1, dev, "cu"), ints(a[14], T, dev, "slots"), ints(a[15], T, dev, "positions"),
                             ints(a[16], B, dev, "granted"), ints(a[18], 1, dev, "free_count_out"),
                             static_cast<int32_t*>(address(a[6])), stream_of(a[8], dev));
  });
}

PyObject* release(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 14, [&] {
    const int dev = small(a[7], "device");
    const OnDevice on(dev);
    const int B = requests(count(a[9], "lens"), a[4]);
    return kvev_paged_release(ints(a[9], B, dev, "lens"), ints(a[10], B, dev, "done"), B, small(a[0], "page_size"),
                              small(a[1], "num_pages"), static_cast<int32_t*>(address(a[3])), small(a[5], "max_pages"),
                              static_cast<int32_t*>(address(a[2])), ints(a[12], 1, dev, "free_count"),
                              ints(a[11], B, dev, "lens_out"), ints(a[13], 1, dev, "free_count_out"),
                              static_cast<int32_t*>(address(a[6])), stream_of(a[8], dev));
  });
}

// (cache: descriptor, block_table, max_requests, max_pages, device_status, device), stream, ...
PyObject* write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    const kvev_paged_cache& c = cache(a[0]);
    const int dev = small(a[5], "device");
    const OnDevice on(dev);
    const Rows k = rows(a[7], c, dev, "k"), v = rows(a[8], c, dev, "v");
    if (k.heads != c.H_kv || v.heads != k.heads || v.tokens != k.tokens || v.token_stride != k.token_stride ||
        v.head_stride != k.head_stride)
      refuse("k, v", "[tokens][H_kv][d] of equal shapes and strides");
    return kvev_paged_write(&c, k.at, v.at, k.token_stride, k.head_stride, ints(a[9], k.tokens, dev, "slots"),
                            static_cast<int>(k.tokens), static_cast<int32_t*>(address(a[4])), stream_of(a[6], dev));
  });
}

PyObject* gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    const kvev_paged_cache& c = cache(a[0]);
    const int dev = small(a[5], "device");
    const OnDevice on(dev);
    const int B = requests(count(a[7], "lens"), a[2]);
    const at::Tensor &K = tensor(a[8], "out_K"), &V = tensor(a[9], "out_V");
    for (const at::Tensor* t : {&K, &V}) {
      if (t->dim() != 4 || t->size(0) != B || t->size(1) != c.H_kv || t->size(2) != K.size(2) || t->size(3) != c.d ||
          !t->is_contiguous() || t->scalar_type() != (c.dtype == KVEV_FP16 ? at::kHalf : at::kBFloat16) || t->size(2) > INT_MAX)
        refuse("out_K, out_V", "contiguous [requests][H_kv][S_cap][d] of the cache's type");
      on_device(*t, dev, "out_K, out_V");
    }
    return kvev_paged_gather(&c, static_cast<int32_t*>(address(a[1])), small(a[3], "max_pages"), ints(a[7], B, dev, "lens"), B,
                             static_cast<int>(K.size(2)), K.data_ptr(), V.data_ptr(), static_cast<int32_t*>(address(a[4])),
                             stream_of(a[6], dev));
  });
}

PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 16, [&] {
    const kvev_paged_cache& c = cache(a[0]);
    const int dev = small(a[5], "device");
    const OnDevice on(dev);
    const Rows q = rows(a[7], c, dev, "q"), out = rows(a[10], c, dev, "out");
    const int B = requests(count(a[9], "kv_lens"), a[2]);
    if (out.tokens != q.tokens || out.heads != q.heads) refuse("out", "q's shape");
    float* lse = nullptr;
    if (a[11] != Py_None) {
      const at::Tensor& t = tensor(a[11], "lse");
      if (t.scalar_type() != at::kFloat || t.dim() != 2 || t.size(0) != q.tokens || t.size(1) != q.heads || !t.is_contiguous())
        refuse("lse", "contiguous float32 [tokens][heads]");
      on_device(t, dev, "lse");
      lse = static_cast<float*>(t.data_ptr());
    }
    const double scale = PyFloat_AsDouble(a[12]);
    if (scale == -1.0 && PyErr_Occurred()) throw Refused();
    return kvev_paged_attention(&c, q.at, q.token_stride, q.head_stride, ints(a[8], B + 1, dev, "cu"), ints(a[9], B, dev, "kv_lens"),
                                static_cast<int32_t*>(address(a[1])), small(a[3], "max_pages"), B, static_cast<int>(q.tokens),
                                static_cast<int>(q.heads), static_cast<float>(scale), small(a[13], "window"), out.at, out.token_stride,
                                out.head_stride, lse, address(a[14]), static_cast<size_t>(number(a[15])),
                                static_cast<int32_t*>(address(a[4])), stream_of(a[6], dev));
  });
}

// (device, stream): the stream's number (the current one's for None), and the id of the capture that it is part of, 0 if
// none.  (0.2 us of an attention call.)
PyObject* stream(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    if (n != 2) throw Refused();
    const int dev = small(a[0], "device");
    const OnDevice on(dev);
    const cudaStream_t s = static_cast<cudaStream_t>(stream_of(a[1], dev));
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    unsigned long long id = 0;
    const cudaError_t e = cudaStreamGetCaptureInfo(s, &status, &id);
    if (e != cudaSuccess) {
      cudaGetLastError();
      PyErr_SetString(PyExc_RuntimeError, cudaGetErrorString(e));
      throw Refused();
    }
    return Py_BuildValue("KK", static_cast<unsigned long long>(reinterpret_cast<uintptr_t>(s)),
                         status == cudaStreamCaptureStatusNone ? 0ull : id);
  } catch (const Refused&) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "stream(device, stream)");
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(tables), FAST(release), FAST(write), FAST(gather), FAST(attention), FAST(stream),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "kvev_paged_bind", "kvev_paged_* on torch tensors", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit_kvev_paged_bind() { return PyModule_Create(&module); }
