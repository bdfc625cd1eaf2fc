// paged_attn.cu -- causal attention of new tokens over paged caches.
#include <climits>
#include <cmath>

#include "paged.cuh"

namespace kvev {
namespace {

struct PagedAttnParams {
  PagedView c;
  const uint4* q;
  uint4* out;
  float* lse;
  long long q_token, q_head, out_token, out_head;  // strides in vectors
  const int *cu, *kv_lens, *table;
  int B, T, H_q, G, max_pages, window;
  float scale_log2;
  int* status;
};

__device__ __forceinline__ float2 unpack2(uint32_t u, int fp16) {
  if (fp16) {
    float2 f;
    asm("{.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;}" : "=f"(f.x), "=f"(f.y) : "r"(u));
    return f;
  }
  return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}

// One warp per (token, query head): lane i holds 2 * D / 64 elements of the row.
template <int D, int kFp16>
__global__ void __launch_bounds__(256) attn_kernel(const __grid_constant__ PagedAttnParams p) {
  const long long w = (static_cast<long long>(blockIdx.x) * 256 + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  const int t = static_cast<int>(w / p.H_q), j = static_cast<int>(w % p.H_q);
  if (t >= p.T || t >= p.cu[p.B]) return;
  int lo = 0, n = p.B;
  while (n > 1) {
    const int h = n >> 1;
    if (p.cu[lo + h] <= t) lo += h;
    n -= h;
  }
  const int s = lo, c0 = p.cu[s], q_len = p.cu[s + 1] - c0, len = p.kv_lens[s];
  if (q_len <= 0 || c0 < 0 || c0 + q_len > p.T || len < 0 || len > (p.max_pages << p.c.page_shift)) {
    if (lane == 0) atomicOr(p.status, kStatusDevice);
    return;
  }
  const int pos = len - q_len + t - c0, h = j / p.G;
  const int k0 = p.window > 0 ? max(0, pos + 1 - p.window) : 0;
  constexpr int E = D / 64;
  float2 q[E], o[E];
  const uint32_t* qr = reinterpret_cast<const uint32_t*>(p.q + t * p.q_token + j * p.q_head);
  for (int e = 0; e < E; ++e) { q[e] = unpack2(qr[lane * E + e], kFp16); o[e] = make_float2(0.f, 0.f); }
  float m = -INFINITY, z = 0.f;
  for (int k = k0; k <= pos; ++k) {
    const int page = p.table[static_cast<long long>(s) * p.max_pages + (k >> p.c.page_shift)];
    const bool there = static_cast<unsigned>(page) < static_cast<unsigned>(p.c.num_pages);
    if (!there && lane == 0) atomicOr(p.status, kStatusDevice);
    const long long at = page * p.c.page_stride + (k & ((1 << p.c.page_shift) - 1)) * p.c.token_stride + h * p.c.head_stride;
    const uint32_t* kr = reinterpret_cast<const uint32_t*>(p.c.K + at);
    const uint32_t* vr = reinterpret_cast<const uint32_t*>(p.c.V + at);
    float x = 0.f;
    for (int e = 0; e < E; ++e) {
      const float2 f = there ? unpack2(kr[lane * E + e], kFp16) : make_float2(0.f, 0.f);
      x = fmaf(q[e].x, f.x, fmaf(q[e].y, f.y, x));
    }
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    x *= p.scale_log2;
    const float mn = fmaxf(m, x), a = exp2f(m - mn), b = exp2f(x - mn);
    z = z * a + b;
    for (int e = 0; e < E; ++e) {
      const float2 f = there ? unpack2(vr[lane * E + e], kFp16) : make_float2(0.f, 0.f);
      o[e].x = o[e].x * a + b * f.x;
      o[e].y = o[e].y * a + b * f.y;
    }
    m = mn;
  }
  const float inv = z > 0.f ? 1.f / z : 0.f;
  uint32_t* orow = reinterpret_cast<uint32_t*>(p.out + t * p.out_token + j * p.out_head);
  for (int e = 0; e < E; ++e) {
    uint32_t u;
    if (kFp16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(o[e].y * inv), "f"(o[e].x * inv));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(o[e].y * inv), "f"(o[e].x * inv));
    orow[lane * E + e] = u;
  }
  if (p.lse && lane == 0) p.lse[static_cast<long long>(t) * p.H_q + j] = z > 0.f ? (m + log2f(z)) * 0.6931471805599453f : -INFINITY;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
}  // namespace kvev

using namespace kvev;

extern "C" int kvev_paged_attention_workspace(int H_q, int H_kv, int d, size_t* bytes) {
  if (!bytes || H_kv < 1 || H_q < 1 || H_q % H_kv) return KVEV_EINVAL;
  if ((d != 64 && d != 128) || H_q / H_kv > 128) return KVEV_ENOTSUP;
  *bytes = KVEV_PAGED_SYNC_BYTES;
  return KVEV_OK;
}

extern "C" int kvev_paged_attention(const kvev_paged_cache* cache, const void* q, int64_t q_token_stride,
                                    int64_t q_head_stride, const int32_t* cu_new, const int32_t* kv_lens,
                                    const int32_t* block_table, int max_pages, int B, int T, int H_q, float scale,
                                    int window, void* out, int64_t out_token_stride, int64_t out_head_stride,
                                    float* lse, void* workspace, size_t workspace_bytes, int32_t* device_status,
                                    void* stream) {
  PagedAttnParams p = {};
  int rc = paged_view(cache, &p.c);
  if (rc != KVEV_OK) return rc;
  size_t need = 0;
  rc = kvev_paged_attention_workspace(H_q, cache->H_kv, cache->d, &need);
  if (rc != KVEV_OK) return rc;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || !device_status) return KVEV_EINVAL;
  for (int64_t st : {q_token_stride, q_head_stride, out_token_stride, out_head_stride})
    if (st <= 0 || (st & 7)) return KVEV_EINVAL;
  if (B < 0 || T < 0 || max_pages < 1 || static_cast<int64_t>(max_pages) * cache->page_size > INT_MAX || window < 0 ||
      !(scale >= 0.f) || !std::isfinite(scale))
    return KVEV_EINVAL;
  if (B > KVEV_PAGED_MAX_REQUESTS) return KVEV_ENOTSUP;
  if (workspace_bytes < need) return KVEV_ENOMEM;
  if (B == 0 || T == 0) return KVEV_OK;
  if (!q || !out || !aligned16(q) || !aligned16(out) || !cu_new || !kv_lens || !block_table ||
      (reinterpret_cast<uintptr_t>(lse) & 3u))
    return KVEV_EINVAL;
  p.q = static_cast<const uint4*>(q);
  p.out = static_cast<uint4*>(out);
  p.lse = lse;
  p.q_token = q_token_stride / 8;
  p.q_head = q_head_stride / 8;
  p.out_token = out_token_stride / 8;
  p.out_head = out_head_stride / 8;
  p.cu = cu_new;
  p.kv_lens = kv_lens;
  p.table = block_table;
  p.B = B;
  p.T = T;
  p.H_q = H_q;
  p.G = H_q / cache->H_kv;
  p.max_pages = max_pages;
  p.window = window;
  p.scale_log2 = (scale > 0.f ? scale : 1.f / std::sqrt(static_cast<float>(cache->d))) * 1.4426950408889634f;
  p.status = device_status;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(T) * H_q + 7) / 8);
  const bool h = cache->dtype == KVEV_FP16;
  if (cache->d == 64) {
    if (h) attn_kernel<64, 1><<<grid, 256, 0, st>>>(p); else attn_kernel<64, 0><<<grid, 256, 0, st>>>(p);
  } else {
    if (h) attn_kernel<128, 1><<<grid, 256, 0, st>>>(p); else attn_kernel<128, 0><<<grid, 256, 0, st>>>(p);
  }
  return cudaGetLastError() == cudaSuccess ? KVEV_OK : KVEV_ECUDA;
}
