// Stands in for the library and for CUDA's current device, so that the calls of paged_q8_bind.cpp can be
// followed on a machine without a GPU.
#include <c10/cuda/CUDAFunctions.h>

#include "kvev.h"

extern "C" {
__attribute__((visibility("default"))) int stub_device = 0, stub_seen = -1, stub_calls = 0;

static int noted() {
  stub_seen = stub_device;
  ++stub_calls;
  return KVEV_OK;
}
KVEV_API int kvev_paged_q8_write(const kvev_paged_q8_cache*, const void*, const void*, int64_t, int64_t, const int32_t*, int, int32_t*,
                                 void*) { return noted(); }
KVEV_API int kvev_paged_q8_gather(const kvev_paged_q8_cache*, const int32_t*, int, const int32_t*, int, int, void*, void*, int32_t*,
                                  void*) { return noted(); }
KVEV_API int kvev_paged_q8_attention(const kvev_paged_q8_cache*, const void*, int64_t, int64_t, const int32_t*, const int32_t*,
                                     const int32_t*, int, int, int, int, float, int, void*, int64_t, int64_t, float*, void*, size_t,
                                     int32_t*, void*) { return noted(); }
KVEV_API int kvev_paged_attention_shared(const kvev_paged_cache*, const void*, int64_t, int64_t, const int32_t*, const int32_t*,
                                         const int32_t*, int, int, int, int, float, const int32_t*, const int32_t*, int, void*, int64_t,
                                         int64_t, float*, void*, size_t, int32_t*, void*) { return noted(); }
}

namespace c10::cuda {
__attribute__((visibility("default"))) DeviceIndex ExchangeDevice(DeviceIndex d) {
  const int was = stub_device;
  stub_device = d;
  return static_cast<DeviceIndex>(was);
}
__attribute__((visibility("default"))) cudaError_t SetDevice(DeviceIndex d, const bool) {
  stub_device = d;
  return cudaSuccess;
}
__attribute__((visibility("default"))) cudaError_t MaybeSetDevice(DeviceIndex d) {
  stub_device = d;
  return cudaSuccess;
}
__attribute__((visibility("default"))) cudaError_t GetDevice(DeviceIndex* d) {
  *d = static_cast<DeviceIndex>(stub_device);
  return cudaSuccess;
}
}  // namespace c10::cuda
