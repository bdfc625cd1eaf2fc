// paged.cuh -- what the kernels over paged caches share.
#pragma once
#include "kvev_internal.cuh"

namespace kvev {

// A layer's pages as the kernels address them (16-byte vectors of 8 elements).
struct PagedView {
  const uint4* K;
  const uint4* V;
  long long page_stride, token_stride, head_stride;  // in vectors
  int num_pages, page_shift, H_kv, dv;               // dv: vectors of a row (d / 8)
};

// Whether the cache's sizes, strides and pointers are in range; its view.
int paged_view(const kvev_paged_cache* c, PagedView* v);
bool paged_page_size(int page_size);
constexpr int kMaxTokens = 1 << 30;  // of a request, or rows of a call: positions and their differences are ints
inline int log2_of(int x) { return 31 - __builtin_clz(static_cast<unsigned>(x)); }

}  // namespace kvev
