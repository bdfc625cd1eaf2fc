// paged_q8_attn.cu -- attention over paged caches of 8-bit codes: a kernel for the requests of few rows, which is bound
// by the cache's bytes (paged_q8_few.cuh), and one for the others, bound by the products (paged_attn.cuh).  Which
// request is which only the device knows; the host leaves the second out where the numbers of rows and requests say, or suggest, that
// it has none.
#include "paged_q8_few.cuh"

using namespace kvev;

extern "C" int kvev_paged_q8_attention(const kvev_paged_q8_cache* cache, const void* q, int64_t q_token_stride,
                                       int64_t q_head_stride, const int32_t* cu_new, const int32_t* kv_lens,
                                       const int32_t* block_table, int max_pages, int B, int T, int H_q, float scale,
                                       int window, void* out, int64_t out_token_stride, int64_t out_head_stride,
                                       float* lse, void* workspace, size_t workspace_bytes, int32_t* device_status,
                                       void* stream) {
  PagedQ8View view = {};
  int rc = paged_q8_view(cache, &view);
  if (rc != KVEV_OK) return rc;
  const AttnCall a = {q, q_token_stride, q_head_stride, cu_new, kv_lens, block_table, max_pages, B, T, H_q, scale, window,
                      out, out_token_stride, out_head_stride, lse, workspace, device_status, static_cast<cudaStream_t>(stream)};
  bool nothing = false;
  rc = attn_check(a, cache->H_kv, cache->d, cache->page_size, workspace_bytes, attn_workspace_bytes(cache->d), &nothing);
  if (rc != KVEV_OK || nothing) return rc;
  PagedAttnParams p = {};
  rc = attn_params(a, cache->H_kv, cache->d, view.fp16, cache->page_size, cache->num_pages, &p);
  if (rc != KVEV_OK) return rc;
  p.K = view.K;
  p.V = view.V;
  p.K_scale = view.K_scale;
  p.V_scale = view.V_scale;
  p.page_stride = view.page_stride;
  p.token_stride = view.token_stride;
  p.head_stride = view.head_stride;
  p.scale_page = view.scale_page;
  const int rows = few_rows_of(p.G, B, T);
  p.few = rows / p.G;
  // Which kernel takes a request goes by its own rows.  The second is left out where it has nothing to do: where all rows together are
  // few, and where there are as many rows as requests, which is taken for a batch of single tokens (it would cost each such call
  // 5 us: 16 at 16K 94 us for 89, 64 ragged ones 64 for 57).  Then the first takes whatever there is and says what is out of range; a longer
  // request is cut into units of few rows, each of which reads its whole context.  (Left out also where there are fewer rows than requests,
  // as among idle ones, 48 new tokens at 32K took 242 us instead of 68-76, 500 took 2.4 ms instead of 0.26.)
  const bool alone = p.G <= kFewRows && (T <= kFewRows / p.G || T == B);
  p.most = alone ? T : kFewRows / p.G;
  p.look = !alone && T > B;
  if (p.most > 0) rc = few_launch(p, cache, rows, a.stream);
  if (rc == KVEV_OK && !alone) {
    if (!q8_page_maps(cache, CU_TENSOR_MAP_SWIZZLE_NONE, &p)) return KVEV_ECUDA;
    rc = attn_launch<kQ8>(p, cache->d, view.fp16, a.stream);
  }
  return rc;
}
