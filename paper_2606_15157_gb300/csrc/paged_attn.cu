// paged_attn.cu -- attention over paged caches of 16 bits (kernel: paged_attn.cuh).
#include "paged_attn.cuh"

using namespace kvev;

extern "C" int kvev_paged_attention_workspace(int H_q, int H_kv, int d, size_t* bytes) {
  if (!bytes || H_kv < 1 || H_q < 1 || H_q % H_kv) return KVEV_EINVAL;
  if ((d != 64 && d != 128) || H_q / H_kv > 128) return KVEV_ENOTSUP;
  static_assert(2 * kMaxCtas * sizeof(int) <= KVEV_PAGED_SYNC_BYTES, "arrival counts");
  *bytes = attn_workspace_bytes(d);
  return KVEV_OK;
}

extern "C" int kvev_paged_attention(const kvev_paged_cache* cache, const void* q, int64_t q_token_stride,
                                    int64_t q_head_stride, const int32_t* cu_new, const int32_t* kv_lens,
                                    const int32_t* block_table, int max_pages, int B, int T, int H_q, float scale,
                                    int window, void* out, int64_t out_token_stride, int64_t out_head_stride,
                                    float* lse, void* workspace, size_t workspace_bytes, int32_t* device_status,
                                    void* stream) {
  PagedView view = {};
  int rc = paged_view(cache, &view);
  if (rc != KVEV_OK) return rc;
  const AttnCall a = {q, q_token_stride, q_head_stride, cu_new, kv_lens, block_table, max_pages, B, T, H_q, scale, window,
                      out, out_token_stride, out_head_stride, lse, workspace, device_status, static_cast<cudaStream_t>(stream)};
  bool nothing = false;
  rc = attn_check(a, cache->H_kv, cache->d, cache->page_size, workspace_bytes, attn_workspace_bytes(cache->d), &nothing);
  if (rc != KVEV_OK || nothing) return rc;
  PagedAttnParams p = {};
  const bool fp16 = cache->dtype == KVEV_FP16;
  rc = attn_params(a, cache->H_kv, cache->d, fp16, cache->page_size, cache->num_pages, &p);
  if (rc != KVEV_OK) return rc;
  if (!attn_page_maps(cache, &p)) return KVEV_ECUDA;
  return attn_launch<kPlain>(p, cache->d, fp16, a.stream);
}
