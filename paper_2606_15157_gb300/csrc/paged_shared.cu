// paged_shared.cu -- attention over paged caches for groups of requests that share a prefix.
//
// With a group's common keys C and a request's own keys R, a row needs
//   o = (e^a o_C + e^b o_R) / (e^a + e^b),  lse = ln(e^a + e^b),
// a, b and o_C, o_R the log-sum-exp and the normalised outputs over C and over R.  The rows of all requests of a
// group lie one after another in q, so over C they are one request whose rows see every key: units of up to
// 2 P tokens of the group (kernel: paged_attn.cuh) read C once, beside the requests' units over R in the same
// launch and the same equal shares.  Either leaves its part of a row in the workspace, and the kernel below
// puts them together.
#include "paged_attn.cuh"

namespace kvev {
namespace {

constexpr int kJoinThreads = 256;

// A CTA takes a token at a time: its request by search, then its heads' vectors.
template <int D, bool kFp16>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ PagedAttnParams p) {
  const int lane = threadIdx.x & 31;
  pdl_wait();
  pdl_trigger();
  bool ordered = true;
  for (int g = threadIdx.x; g < p.N; g += kJoinThreads) ordered &= group_in_order(p, g);
  ordered = __syncthreads_and(ordered);
  if (!ordered) return;
  for (int t = blockIdx.x; t < p.T; t += gridDim.x) {
    int s = 0, n = p.B;  // the last request with cu[s] <= t
    while (n > 1) {
      const int step = (n + 31) / 32, i = lane * step;
      const uint32_t upto = __ballot_sync(0xffffffffu, i < n && p.cu[s + min(i, n - 1)] <= t);
      const int j = upto ? 31 - __clz(upto) : 0;
      s += j * step;
      n = min(step, n - j * step);
    }
    bool bad = false;
    const Request r = own_request(p, s, &bad);
    if (t < r.c0 || t >= r.c0 + r.q || shared_of_request(p, s, r, &bad) == 0) continue;
    constexpr int kVec = D / 4;
    for (int i = threadIdx.x; i < p.H_q * kVec; i += kJoinThreads) {
      const int head = i / kVec, c = i % kVec;
      const long long at = static_cast<long long>(t) * p.H_q + head, other = at + static_cast<long long>(p.T) * p.H_q;
      const float a = p.part_lse[at], b = p.part_lse[other];
      const float4 x = reinterpret_cast<const float4*>(p.part_o)[at * kVec + c], y = reinterpret_cast<const float4*>(p.part_o)[other * kVec + c];
      const float m = finite_or_0(fmaxf(a, b));
      float wa = ex2_approx(a - m), wb = ex2_approx(b - m);
      const float sum = wa + wb, inv = sum == 0.f ? 0.f : 1.f / sum;
      wa *= inv;
      wb *= inv;
      uint2 w;
      w.x = pack2<kFp16>(fmaf(x.x, wa, y.x * wb), fmaf(x.y, wa, y.y * wb));
      w.y = pack2<kFp16>(fmaf(x.z, wa, y.z * wb), fmaf(x.w, wa, y.w * wb));
      *reinterpret_cast<uint2*>(p.out + static_cast<long long>(t) * p.out_token + static_cast<long long>(head) * p.out_head + c * 8) = w;
      if (p.lse && c == 0) p.lse[at] = lse_of(m, sum);
    }
  }
}

size_t part_lse_bytes(int T, int H_q) { return (static_cast<size_t>(2) * T * H_q * sizeof(float) + 255) & ~static_cast<size_t>(255); }
size_t shared_bytes(int H_q, int d, int T) {
  return attn_workspace_bytes(d) + part_lse_bytes(T, H_q) + static_cast<size_t>(2) * T * H_q * d * sizeof(float);
}

}  // namespace
}  // namespace kvev

using namespace kvev;

extern "C" int kvev_paged_attention_shared_workspace(int H_q, int H_kv, int d, int T, size_t* bytes) {
  if (!bytes || H_kv < 1 || H_q < 1 || H_q % H_kv || T < 0 || T > kMaxTokens) return KVEV_EINVAL;
  if ((d != 64 && d != 128) || H_q / H_kv > 128) return KVEV_ENOTSUP;
  *bytes = shared_bytes(H_q, d, T);
  return KVEV_OK;
}

extern "C" int kvev_paged_attention_shared(const kvev_paged_cache* cache, const void* q, int64_t q_token_stride,
                                           int64_t q_head_stride, const int32_t* cu_new, const int32_t* kv_lens,
                                           const int32_t* block_table, int max_pages, int B, int T, int H_q, float scale,
                                           const int32_t* groups, const int32_t* shared_lens, int N, void* out,
                                           int64_t out_token_stride, int64_t out_head_stride, float* lse, void* workspace,
                                           size_t workspace_bytes, int32_t* device_status, void* stream) {
  if (N == 0)
    return kvev_paged_attention(cache, q, q_token_stride, q_head_stride, cu_new, kv_lens, block_table, max_pages, B, T, H_q, scale,
                                0, out, out_token_stride, out_head_stride, lse, workspace, workspace_bytes, device_status, stream);
  PagedView view = {};
  int rc = paged_view(cache, &view);
  if (rc != KVEV_OK) return rc;
  if (N < 0 || !groups || !shared_lens) return KVEV_EINVAL;
  const AttnCall a = {q, q_token_stride, q_head_stride, cu_new, kv_lens, block_table, max_pages, B, T, H_q, scale, 0,
                      out, out_token_stride, out_head_stride, lse, workspace, device_status, static_cast<cudaStream_t>(stream)};
  const int d = cache->d;
  const size_t need = T >= 0 && H_q > 0 ? shared_bytes(H_q, d, T) : 0;
  bool nothing = false;
  rc = attn_check(a, cache->H_kv, d, cache->page_size, workspace_bytes, need, &nothing);
  if (rc != KVEV_OK) return rc;
  if (N > KVEV_PAGED_MAX_REQUESTS - B) return KVEV_ENOTSUP;
  if (nothing) return KVEV_OK;
  PagedAttnParams p = {};
  const bool fp16 = cache->dtype == KVEV_FP16;
  rc = attn_params(a, cache->H_kv, d, fp16, cache->page_size, cache->num_pages, &p);
  if (rc != KVEV_OK) return rc;
  if (!attn_page_maps(cache, &p)) return KVEV_ECUDA;
  p.groups = groups;
  p.shared = shared_lens;
  p.N = N;
  p.segs = B + N;
  p.part_lse = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + attn_workspace_bytes(d));
  p.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + attn_workspace_bytes(d) + part_lse_bytes(T, H_q));
  rc = attn_launch<kShared>(p, d, fp16, a.stream);
  if (rc != KVEV_OK) return rc;
  const AttnFn fn = d == 64 ? (fp16 ? join_kernel<64, true> : join_kernel<64, false>) : (fp16 ? join_kernel<128, true> : join_kernel<128, false>);
  const int grid = T < 8 * kMaxCtas ? T : 8 * kMaxCtas;
  return launch_overlapped(fn, p, grid, kJoinThreads, 0, a.stream) == cudaSuccess ? KVEV_OK : KVEV_ECUDA;
}
