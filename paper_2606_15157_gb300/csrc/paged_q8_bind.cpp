// paged_q8_bind.cpp -- the calls of paged.py on caches of 8 bits, and those for requests that share a prefix:
// their checks and the call of the C entry point, as in paged_bind.cpp.
#include "paged_bind.h"

namespace {

const kvev_paged_q8_cache& q8_cache(PyObject* o) { return *static_cast<const kvev_paged_q8_cache*>(address(o)); }

// (cache: descriptor, block_table, max_requests, max_pages, device_status, device), stream, ...
PyObject* write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    const kvev_paged_q8_cache& c = q8_cache(a[0]);
    const int dev = small(a[5], "device");
    const OnDevice on(dev);
    const Rows k = rows(a[7], c.d, c.dtype, dev, "k"), v = rows(a[8], c.d, c.dtype, dev, "v");
    if (k.heads != c.H_kv || v.heads != k.heads || v.tokens != k.tokens || v.token_stride != k.token_stride ||
        v.head_stride != k.head_stride)
      refuse("k, v", "[tokens][H_kv][d] of equal shapes and strides");
    return kvev_paged_q8_write(&c, k.at, v.at, k.token_stride, k.head_stride, ints(a[9], k.tokens, dev, "slots"),
                               static_cast<int>(k.tokens), static_cast<int32_t*>(address(a[4])), stream_of(a[6], dev));
  });
}

PyObject* gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    const kvev_paged_q8_cache& c = q8_cache(a[0]);
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
    return kvev_paged_q8_gather(&c, static_cast<int32_t*>(address(a[1])), small(a[3], "max_pages"), ints(a[7], B, dev, "lens"), B,
                                static_cast<int>(K.size(2)), K.data_ptr(), V.data_ptr(), static_cast<int32_t*>(address(a[4])),
                                stream_of(a[6], dev));
  });
}

PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 16, [&] {
    const kvev_paged_q8_cache& c = q8_cache(a[0]);
    const int dev = small(a[5], "device");
    const OnDevice on(dev);
    const Rows q = rows(a[7], c.d, c.dtype, dev, "q"), out = rows(a[10], c.d, c.dtype, dev, "out");
    const int B = requests(count(a[9], "kv_lens"), a[2]);
    if (out.tokens != q.tokens || out.heads != q.heads) refuse("out", "q's shape");
    float* lse = lse_of(a[11], q, dev);
    const double scale = PyFloat_AsDouble(a[12]);
    if (scale == -1.0 && PyErr_Occurred()) throw Refused();
    return kvev_paged_q8_attention(&c, q.at, q.token_stride, q.head_stride, ints(a[8], B + 1, dev, "cu"), ints(a[9], B, dev, "kv_lens"),
                                   static_cast<int32_t*>(address(a[1])), small(a[3], "max_pages"), B, static_cast<int>(q.tokens),
                                   static_cast<int>(q.heads), static_cast<float>(scale), small(a[13], "window"), out.at,
                                   out.token_stride, out.head_stride, lse, address(a[14]), static_cast<size_t>(number(a[15])),
                                   static_cast<int32_t*>(address(a[4])), stream_of(a[6], dev));
  });
}

// The same of a 16-bit cache, then q, cu, kv_lens, groups, shared_lens, out, lse, scale, workspace, bytes.
PyObject* attention_shared(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 17, [&] {
    const kvev_paged_cache& c = *static_cast<const kvev_paged_cache*>(address(a[0]));
    const int dev = small(a[5], "device");
    const OnDevice on(dev);
    const Rows q = rows(a[7], c.d, c.dtype, dev, "q"), out = rows(a[12], c.d, c.dtype, dev, "out");
    const int B = requests(count(a[9], "kv_lens"), a[2]);
    if (out.tokens != q.tokens || out.heads != q.heads) refuse("out", "q's shape");
    const int64_t N = count(a[11], "shared_lens");
    if (N > INT_MAX) refuse("shared_lens", "out of range");
    float* lse = lse_of(a[13], q, dev);
    const double scale = PyFloat_AsDouble(a[14]);
    if (scale == -1.0 && PyErr_Occurred()) throw Refused();
    return kvev_paged_attention_shared(&c, q.at, q.token_stride, q.head_stride, ints(a[8], B + 1, dev, "cu"), ints(a[9], B, dev, "kv_lens"),
                                       static_cast<int32_t*>(address(a[1])), small(a[3], "max_pages"), B, static_cast<int>(q.tokens),
                                       static_cast<int>(q.heads), static_cast<float>(scale), ints(a[10], N + 1, dev, "groups"),
                                       ints(a[11], N, dev, "shared_lens"), static_cast<int>(N), out.at, out.token_stride,
                                       out.head_stride, lse, address(a[15]), static_cast<size_t>(number(a[16])),
                                       static_cast<int32_t*>(address(a[4])), stream_of(a[6], dev));
  });
}

PyMethodDef methods[] = {FAST(write), FAST(gather), FAST(attention), FAST(attention_shared), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "kvev_paged_q8_bind", "kvev_paged_q8_* and kvev_paged_attention_shared on torch tensors", -1,
                      methods};

}  // namespace

PyMODINIT_FUNC PyInit_kvev_paged_q8_bind() { return PyModule_Create(&module); }
