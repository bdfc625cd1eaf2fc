// paged_shared.cu -- attention over paged caches for groups of requests that share a prefix.
//
// With a group's common keys C and a request's own keys R, a row needs
//   o = (e^a o_C + e^b o_R) / (e^a + e^b),  lse = ln(e^a + e^b),
// a, b and o_C, o_R the log-sum-exp and the normalised outputs over C and over R.  The rows of all requests of a
// group lie one after another in q, so over C they are one request whose rows see every key: units of up to
// 2 P tokens of the group (kernel: paged_attn.cuh) read C once, beside the requests' units over R in the same
// launch and the same equal shares.  Either leaves its part of a row in the workspace, and the join kernel puts them
// together.  64 generations behind 8K, own tokens to 1,500, 32 query and 8 KV heads of 128: 59 us, 39 of them for the
// own parts alone (HBM 33), kvev_paged_attention on the same batch 202; 12 requests' 3,000 new rows behind 16K 0.62-0.66 ms, 1,400 TFLOP/s
// (0.61: chunks are bound by the products, which stay the same).
//
// The common part and the join come on top of a pass of their own length: a group gains from about 16 single tokens behind 2,048 common ones or 8 behind
// 4,096 on, smaller ones lose up to 10 us (4 behind 2,000 19 us for 12).  Nothing here looks at that; the caller does.
#include "paged_attn.cuh"

namespace kvev {
namespace {

// ---- the plan -------------------------------------------------------------------------------
// The groups over their common keys, then the requests (first row, rows, keys, first key; row of the block table, whether a group,
// the group's first row and the one after its last), 32 bytes each: what the attention's CTAs would all read through the
// groups' and the requests' lengths in turn (made there, a call of 64 generations behind a single page took 70 us, the same
// without a group 39).
// Batches of up to 32 are planned by every CTA's dealing warp, a lane each, and the first CTA's leaves the plan to the join.
constexpr int kPlanThreads = 128;

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const __grid_constant__ PagedAttnParams p) {
  pdl_wait();
  pdl_trigger();
  bool in_order = true;
  for (int g = threadIdx.x; g < p.N; g += kPlanThreads) in_order &= group_in_order(p, g);
  const int s = blockIdx.x * kPlanThreads + threadIdx.x;
  in_order = __syncthreads_and(in_order);
  bool bad = !in_order;
  if (s < p.segs) keep_plan(p, s, plan_of(p, s, in_order, &bad));
  if (bad) atomicOr(p.status, kStatusDevice);
}

// ---- the rows' two parts together ---------------------------------------------------------------
constexpr int kJoinThreads = 256;

struct JoinParams {
  PagedAttnParams p;  // the attention's
  int each;
};

// CTAs (request, one in `each`; part of the heads): every each-th row of the request, its heads' vectors dealt over the
// threads.  A row's part over the common keys is whole, or in the pieces of its unit as the attention left them.
template <int D, bool kFp16>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ JoinParams j) {
  const PagedAttnParams& p = j.p;
  constexpr float kUp = kFp16 ? 7.f : 0.f;  // (of the attention's weights)
  constexpr int kVec = D / 4, kU = 4;
  pdl_wait();
  pdl_trigger();
  const int s = blockIdx.x / j.each;
  const Request r = planned(p, p.N + s);
  if (r.lo == 0) return;
  const int g0 = r.g0, g1 = r.g1;
  for (int i = blockIdx.x - s * j.each; i < r.q; i += j.each) {
    const int t = r.c0 + i, m = (t - g0) / (2 * p.P), tok0 = g0 + 2 * p.P * m, n = min(2 * p.P, g1 - tok0);
    const int kind = n > p.P ? kFull : n * p.G > kFewRows ? kPaired : kFew;
    for (int k = blockIdx.y * kJoinThreads + threadIdx.x; k < p.H_q * kVec; k += gridDim.y * kJoinThreads) {
      // (a KV head's rows of a vector lie next to one another in a record)
      const int h = k / (p.G * kVec), in = k - h * (p.G * kVec), c = in / p.G, head = h * p.G + in - c * p.G, row = (t - tok0) * p.G + in - c * p.G;
      const int2 unit = p.units[static_cast<long long>(h) * p.T + tok0];
      if (unit.x < 0 || unit.y < 1 || unit.x > kMaxCtas - unit.y) continue;  // (a wait of the attention ran out: nothing was left there)
      const long long at = static_cast<long long>(t) * p.H_q + head, own = at + static_cast<long long>(p.T) * p.H_q;
      float top = p.part_lse[own], sum = 1.f;
      float4 o = reinterpret_cast<const float4*>(p.part_o)[own * kVec + c];
      auto add = [&](float a, float l, const float4& x) {
        const float mn = fmaxf(top, a), base = finite_or_0(mn), f = ex2_approx(top - base), w = ex2_approx(a - base);
        sum = fmaf(sum, f, l * w);
        o = make_float4(fmaf(o.x, f, x.x * w), fmaf(o.y, f, x.y * w), fmaf(o.z, f, x.z * w), fmaf(o.w, f, x.w * w));
        top = mn;
      };
      if (unit.y == 1) {
        add(p.part_lse[at], 1.f, reinterpret_cast<const float4*>(p.part_o)[at * kVec + c]);
      } else {
        // side, row and vector of the record
        const int x = kind == kFull ? row >= p.P * p.G : kind == kPaired ? c >= kVec / 2 : row & 1;
        const int rr = kind == kFull ? row - x * p.P * p.G : row, cc = kind == kPaired ? c - x * (kVec / 2) : c;
        const int vec = kind == kFew ? rr * kVec + cc : cc * kRows + rr;
#pragma unroll 1
        for (int q0 = 0; q0 < unit.y; q0 += kU) {
          float2 z[kU];
          float4 v[kU];
#pragma unroll
          for (int q = 0; q < kU; ++q) {  // (past the last piece: the last one again, with no weight)
            const int piece = min(q0 + q, unit.y - 1);
            const Records<D> rec = records<D>(p, unit.x + piece, piece == 0, x);
            z[q] = __ldcg(rec.ml() + rr);
            v[q] = __ldcg(reinterpret_cast<const float4*>(rec.at) + vec);
          }
#pragma unroll
          for (int q = 0; q < kU; ++q)
            if (q0 + q >= unit.y) z[q] = make_float2(-INFINITY, 0.f);
#pragma unroll
          for (int q = 0; q < kU; ++q) add(z[q].x - kUp, z[q].y, v[q]);
        }
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      uint2 w;
      w.x = pack2<kFp16>(o.x * inv, o.y * inv);
      w.y = pack2<kFp16>(o.z * inv, o.w * inv);
      *reinterpret_cast<uint2*>(p.out + static_cast<long long>(t) * p.out_token + static_cast<long long>(head) * p.out_head + c * 8) = w;
      if (p.lse && c == 0) p.lse[at] = lse_of(top, sum);
    }
  }
}

// Behind the attention's own scratch: the plan, where units are, the parts' log-sum-exp, the parts.
constexpr size_t kPlanBytes = static_cast<size_t>(KVEV_PAGED_MAX_REQUESTS) * 2 * sizeof(int4);
size_t part_lse_bytes(int T, int H_q) { return (static_cast<size_t>(2) * T * H_q * sizeof(float) + 255) & ~static_cast<size_t>(255); }
size_t units_bytes(int T, int H_kv) { return (static_cast<size_t>(T) * H_kv * sizeof(int2) + 255) & ~static_cast<size_t>(255); }
size_t shared_bytes(int H_q, int H_kv, int d, int T) {
  return attn_workspace_bytes(d) + kPlanBytes + units_bytes(T, H_kv) + part_lse_bytes(T, H_q) + static_cast<size_t>(2) * T * H_q * d * sizeof(float);
}

}  // namespace
}  // namespace kvev

using namespace kvev;

extern "C" int kvev_paged_attention_shared_workspace(int H_q, int H_kv, int d, int T, size_t* bytes) {
  if (!bytes || H_kv < 1 || H_q < 1 || H_q % H_kv || T < 0 || T > kMaxTokens) return KVEV_EINVAL;
  if ((d != 64 && d != 128) || H_q / H_kv > 128) return KVEV_ENOTSUP;
  *bytes = shared_bytes(H_q, H_kv, d, T);
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
  const size_t need = T >= 0 && H_q > 0 ? shared_bytes(H_q, cache->H_kv, d, T) : 0;
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
  uint8_t* const after = static_cast<uint8_t*>(workspace) + attn_workspace_bytes(d);
  p.plan = reinterpret_cast<int4*>(after);
  p.groups = groups;
  p.shared = shared_lens;
  p.N = N;
  p.segs = B + N;
  uint8_t* const parts = after + kPlanBytes + units_bytes(T, cache->H_kv);
  p.units = reinterpret_cast<int2*>(after + kPlanBytes);
  p.part_lse = reinterpret_cast<float*>(parts);
  p.part_o = reinterpret_cast<float*>(parts + part_lse_bytes(T, H_q));
  if (p.segs > kPlannedByWarp &&
      launch_overlapped(plan_kernel, p, (B + N + kPlanThreads - 1) / kPlanThreads, kPlanThreads, 0, a.stream) != cudaSuccess)
    return KVEV_ECUDA;
  rc = attn_launch<kShared>(p, d, fp16, a.stream);
  if (rc != KVEV_OK) return rc;
  // as many CTAs to a request as it has rows, as far as the host can tell, and enough of them for the GPU in all
  const int rows = (T + B - 1) / B, most = (8 * kMaxCtas + B - 1) / B;
  const JoinParams jp = {p, rows < most ? rows : most};
  const int vectors = H_q * (d / 4), split = (vectors + kJoinThreads - 1) / kJoinThreads, room = 8 * kMaxCtas / (B * jp.each);
  const auto fn = d == 64 ? (fp16 ? join_kernel<64, true> : join_kernel<64, false>) : (fp16 ? join_kernel<128, true> : join_kernel<128, false>);
  return launch_overlapped(fn, jp, dim3(B * jp.each, room < 1 ? 1 : split < room ? split : room), kJoinThreads, 0, a.stream) == cudaSuccess
             ? KVEV_OK
             : KVEV_ECUDA;
}
