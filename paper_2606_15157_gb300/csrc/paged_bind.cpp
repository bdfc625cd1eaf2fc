// paged_bind.cpp -- the calls of paged.py on torch tensors: their checks and the call of the
// C entry point in one function each.  These calls take 2 to 4 us on the device and are made
// for every layer of every token; through Python's own attribute reads and ctypes the
// host's share was larger (a tables call 6.1 us, a write 4.4, an attention 8.1; here 2.2, 1.9
// and 2.9).
//
// Each function returns the entry point's status code and raises ValueError where a tensor has
// the wrong type, shape or place.  The entry points launch on the current device: each call makes
// the tensors' GPU current for its time.
#include "paged_bind.h"

namespace {

const kvev_paged_cache& cache(PyObject* o) { return *static_cast<const kvev_paged_cache*>(address(o)); }

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
    const Rows k = rows(a[7], c.d, c.dtype, dev, "k"), v = rows(a[8], c.d, c.dtype, dev, "v");
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
          !t->is_contiguous() || t->scalar_type() != type_of(c.dtype) || t->size(2) > INT_MAX)
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
    const Rows q = rows(a[7], c.d, c.dtype, dev, "q"), out = rows(a[10], c.d, c.dtype, dev, "out");
    const int B = requests(count(a[9], "kv_lens"), a[2]);
    if (out.tokens != q.tokens || out.heads != q.heads) refuse("out", "q's shape");
    float* lse = lse_of(a[11], q, dev);
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

PyMethodDef methods[] = {FAST(tables), FAST(release), FAST(write), FAST(gather), FAST(attention), FAST(stream),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "kvev_paged_bind", "kvev_paged_* on torch tensors", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit_kvev_paged_bind() { return PyModule_Create(&module); }
