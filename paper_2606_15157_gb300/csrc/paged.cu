// paged.cu -- the paged cache in front of the eviction: block tables and slots
// built on the GPU, rows written to their slots, and whole prompts gathered
// into the contiguous caches that the prefill eviction reads.
#include <algorithm>
#include <climits>

#include "paged.cuh"

namespace kvev {
namespace {

// ---------------------------------------------------------------------------
// Block tables.  Everything a step needs follows from two prefix sums over the
// requests, of new tokens and of new pages, which one CTA forms in shared memory;
// then tokens and pages are dealt over its threads, each finding its request by
// bisection.  Whatever is written may be an input's own memory (lengths, the
// count): it is written after all of it has been read.
// ---------------------------------------------------------------------------
constexpr int kTableThreads = 1024;

struct TableParams {
  const int *lens, *new_lens, *free_pages, *free_count;
  int* table;
  int *kv_lens, *cu, *slots, *positions, *granted, *count_out, *status;
  int B, page_shift, num_pages, max_pages, T;
};

struct ReleaseParams {
  const int *lens, *done, *table, *free_count;
  int *free_pages, *lens_out, *count_out, *status;
  int B, page_shift, num_pages, max_pages;
};

// Inclusive sums of (a, b) over the CTA's threads; ws holds 32 pairs.
__device__ __forceinline__ longlong2 block_scan(long long a, long long b, longlong2* ws) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
    if (lane >= o) { a += x; b += y; }
  }
  __syncthreads();
  if (lane == 31) ws[warp] = make_longlong2(a, b);
  __syncthreads();
  for (int w = 0; w < warp; ++w) { a += ws[w].x; b += ws[w].y; }
  return make_longlong2(a, b);
}

// The last s in [0, B) with start[s] <= x (start ascending, start[0] <= x).
__device__ __forceinline__ int find_request(const int* start, int B, int x) {
  int lo = 0, n = B;
  while (n > 1) {
    const int h = n >> 1;
    if (start[lo + h] <= x) lo += h;
    n -= h;
  }
  return lo;
}

__device__ __forceinline__ int pages_of(int n, int shift) {
  return static_cast<int>((static_cast<long long>(n) + (1 << shift) - 1) >> shift);
}

__global__ void __launch_bounds__(kTableThreads) tables_kernel(const __grid_constant__ TableParams p) {
  extern __shared__ int sm[];
  int* const cu = sm;             // [B] first token
  int* const first = sm + p.B;    // [B] new pages of the requests before
  int* const len = sm + 2 * p.B;  // [B] tokens held
  int* const need = sm + 3 * p.B; // [B] new pages, -1 = refused
  __shared__ longlong2 ws[32];
  __shared__ long long carry[2];
  __shared__ int given;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  if (tid == 0) { carry[0] = carry[1] = 0; given = 0; }
  const int count = min(max(*p.free_count, 0), p.num_pages);
  bool bad = *p.free_count != count;
  __syncthreads();
  for (int s0 = 0; s0 < p.B; s0 += kTableThreads) {
    const int s = s0 + tid;
    int n = 0, q = 0, k = 0;
    bool fits = true;
    if (s < p.B) {
      n = p.lens[s];
      q = p.new_lens[s];
      bad |= n < 0 || q < 0;
      n = max(n, 0);
      q = max(q, 0);
      const long long after = (static_cast<long long>(n) + q + (1 << p.page_shift) - 1) >> p.page_shift;
      fits = after <= p.max_pages;
      bad |= !fits;
      k = fits ? static_cast<int>(after) - pages_of(n, p.page_shift) : 0;
    }
    const longlong2 upto = block_scan(q, k, ws);
    const long long c0 = carry[0], c1 = carry[1];
    __syncthreads();
    if (tid == kTableThreads - 1) { carry[0] = c0 + upto.x; carry[1] = c1 + upto.y; }
    if (s < p.B) {
      const bool ok = fits && (k == 0 || c1 + upto.y <= count);
      cu[s] = static_cast<int>(min(c0 + upto.x - q, static_cast<long long>(INT_MAX)));
      first[s] = static_cast<int>(min(c1 + upto.y - k, static_cast<long long>(INT_MAX)));
      len[s] = n;
      need[s] = ok ? k : -1;
      if (ok && k > 0) atomicMax(&given, static_cast<int>(c1 + upto.y));
      p.cu[s] = cu[s];
      p.granted[s] = ok;
      p.kv_lens[s] = ok ? n + q : n;
    }
    __syncthreads();
  }
  const int total = static_cast<int>(min(carry[0], static_cast<long long>(INT_MAX)));
  if (tid == 0) {
    p.cu[p.B] = total;
    *p.count_out = count - given;
    bad |= total > p.T;
  }
  // pages given out, the k-th of them to the request whose range holds k
  for (int k = tid; k < given; k += kTableThreads) {
    const int s = find_request(first, p.B, k);
    p.table[static_cast<long long>(s) * p.max_pages + pages_of(len[s], p.page_shift) + k - first[s]] =
        p.free_pages[count - 1 - k];
  }
  for (int t = tid; t < p.T; t += kTableThreads) {
    int slot = -1, pos = -1;
    if (t < total) {
      const int s = find_request(cu, p.B, t);
      if (need[s] >= 0) {
        pos = len[s] + t - cu[s];
        const int j = pos >> p.page_shift, held = pages_of(len[s], p.page_shift);
        const int page = j < held ? p.table[static_cast<long long>(s) * p.max_pages + j]
                                  : p.free_pages[count - 1 - (first[s] + j - held)];
        if (static_cast<unsigned>(page) < static_cast<unsigned>(p.num_pages))
          slot = (page << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
        else
          bad = true;
      }
    }
    p.slots[t] = slot;
    p.positions[t] = pos;
  }
  if (bad) atomicOr(p.status, kStatusDevice);
}

__global__ void __launch_bounds__(kTableThreads) release_kernel(const __grid_constant__ ReleaseParams p) {
  extern __shared__ int sm[];
  int* const first = sm;  // [B] pages released by the requests before
  __shared__ longlong2 ws[32];
  __shared__ long long carry;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  if (tid == 0) carry = 0;
  const int count = min(max(*p.free_count, 0), p.num_pages);
  bool bad = *p.free_count != count;
  __syncthreads();
  for (int s0 = 0; s0 < p.B; s0 += kTableThreads) {
    const int s = s0 + tid;
    int k = 0;
    if (s < p.B) {
      const int n = p.lens[s];
      const bool done = p.done[s] != 0;
      bad |= n < 0;
      k = done ? pages_of(max(n, 0), p.page_shift) : 0;
      bad |= k > p.max_pages;
      k = min(k, p.max_pages);
      p.lens_out[s] = done ? 0 : n;
    }
    const longlong2 upto = block_scan(k, 0, ws);
    const long long c = carry;
    __syncthreads();
    if (tid == kTableThreads - 1) carry = c + upto.x;
    if (s < p.B) first[s] = static_cast<int>(min(c + upto.x - k, static_cast<long long>(INT_MAX)));
    __syncthreads();
  }
  bad |= carry > p.num_pages - count;
  const int total = static_cast<int>(min(carry, static_cast<long long>(p.num_pages - count)));
  if (tid == 0) *p.count_out = count + total;
  for (int k = tid; k < total; k += kTableThreads) {
    const int s = find_request(first, p.B, k);
    const int page = p.table[static_cast<long long>(s) * p.max_pages + k - first[s]];
    bad |= static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages);
    p.free_pages[count + k] = page;
  }
  if (bad) atomicOr(p.status, kStatusDevice);
}

// ---------------------------------------------------------------------------
// Rows.
// ---------------------------------------------------------------------------
struct WriteParams {
  PagedView c;
  const uint4 *k, *v;
  long long token_stride, head_stride;  // in vectors
  const int* slots;
  int T;
  int* status;
};

constexpr int kRowThreads = 256;

// A thread carries vectors of 16 bytes, K's and V's of the same place together.
__global__ void __launch_bounds__(kRowThreads) write_kernel(const __grid_constant__ WriteParams p) {
  pdl_wait();
  pdl_trigger();
  const int nv = p.c.H_kv * p.c.dv;
  const long long n = static_cast<long long>(p.T) * nv;
  for (long long i = static_cast<long long>(blockIdx.x) * kRowThreads + threadIdx.x; i < n;
       i += static_cast<long long>(gridDim.x) * kRowThreads) {
    const int t = static_cast<int>(i / nv), r = static_cast<int>(i - static_cast<long long>(t) * nv);
    const int h = r / p.c.dv, x = r - h * p.c.dv;
    const int slot = p.slots[t];
    if (slot < 0) continue;
    const int page = slot >> p.c.page_shift;
    if (page >= p.c.num_pages) {
      atomicOr(p.status, kStatusDevice);
      continue;
    }
    const long long src = t * p.token_stride + h * p.head_stride + x;
    const long long dst = page * p.c.page_stride + (slot & ((1 << p.c.page_shift) - 1)) * p.c.token_stride +
                          h * p.c.head_stride + x;
    const_cast<uint4*>(p.c.K)[dst] = p.k[src];
    const_cast<uint4*>(p.c.V)[dst] = p.v[src];
  }
}

struct PageGatherParams {
  PagedView c;
  const int *table, *lens;
  int B, max_pages, S_cap;
  uint4 *out_K, *out_V;
  int* status;
};

constexpr int kGatherRows = 32;  // positions of a CTA

__global__ void __launch_bounds__(kRowThreads) page_gather_kernel(const __grid_constant__ PageGatherParams p) {
  pdl_wait();
  pdl_trigger();
  const int s = blockIdx.y;
  const int k0 = blockIdx.x * kGatherRows;
  const int len = p.lens[s];
  const int n = min(max(len, 0), min(p.S_cap, p.max_pages << p.c.page_shift));
  if (n != len && threadIdx.x == 0 && blockIdx.x == 0) atomicOr(p.status, kStatusDevice);
  const int rows = min(kGatherRows, n - k0);
  if (rows <= 0) return;
  const int nv = p.c.H_kv * p.c.dv;
  for (int i = threadIdx.x; i < rows * nv; i += kRowThreads) {
    const int k = k0 + i / nv, r = i % nv;
    const int h = r / p.c.dv, x = r - h * p.c.dv;
    const int page = p.table[static_cast<long long>(s) * p.max_pages + (k >> p.c.page_shift)];
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.c.num_pages)) {
      atomicOr(p.status, kStatusDevice);
      continue;
    }
    const long long src = page * p.c.page_stride + (k & ((1 << p.c.page_shift) - 1)) * p.c.token_stride +
                          h * p.c.head_stride + x;
    const long long dst = ((static_cast<long long>(s) * p.c.H_kv + h) * p.S_cap + k) * p.c.dv + x;
    p.out_K[dst] = p.c.K[src];
    p.out_V[dst] = p.c.V[src];
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int launched(cudaError_t e) { return e == cudaSuccess ? KVEV_OK : KVEV_ECUDA; }

bool tables_sizes(int B, int page_size, int num_pages, int max_pages) {
  return B >= 0 && paged_page_size(page_size) && num_pages >= 1 && max_pages >= 1 &&
         static_cast<int64_t>(num_pages) * page_size <= INT_MAX && static_cast<int64_t>(max_pages) * page_size <= INT_MAX;
}

}  // namespace

bool paged_page_size(int page_size) { return page_size >= 8 && page_size <= 256 && (page_size & (page_size - 1)) == 0; }

int paged_view(const kvev_paged_cache* c, PagedView* v) {
  if (!c || !c->K || !c->V || !aligned16(c->K) || !aligned16(c->V)) return KVEV_EINVAL;
  if (c->num_pages < 1 || !paged_page_size(c->page_size) || c->H_kv < 1 ||
      static_cast<int64_t>(c->num_pages) * c->page_size > INT_MAX)
    return KVEV_EINVAL;
  if (c->dtype != KVEV_BF16 && c->dtype != KVEV_FP16) return KVEV_EINVAL;
  for (int64_t st : {c->page_stride, c->token_stride, c->head_stride})
    if (st <= 0 || (st & 7)) return KVEV_EINVAL;
  if (c->d != 64 && c->d != 128) return KVEV_ENOTSUP;
  v->K = static_cast<const uint4*>(c->K);
  v->V = static_cast<const uint4*>(c->V);
  v->page_stride = c->page_stride / 8;
  v->token_stride = c->token_stride / 8;
  v->head_stride = c->head_stride / 8;
  v->num_pages = c->num_pages;
  v->page_shift = log2_of(c->page_size);
  v->H_kv = c->H_kv;
  v->dv = c->d / 8;
  return KVEV_OK;
}

}  // namespace kvev

using namespace kvev;

extern "C" int kvev_paged_tables(const int32_t* lens, const int32_t* new_lens, int B, int page_size, int num_pages,
                                 const int32_t* free_pages, const int32_t* free_count, int32_t* block_table,
                                 int max_pages, int T, int32_t* kv_lens, int32_t* cu_new, int32_t* slots,
                                 int32_t* positions, int32_t* granted, int32_t* free_count_out,
                                 int32_t* device_status, void* stream) {
  if (!free_pages || !free_count || !cu_new || !free_count_out || !device_status || T < 0 ||
      !tables_sizes(B, page_size, num_pages, max_pages) || (T > 0 && (!slots || !positions)) ||
      (B > 0 && (!lens || !new_lens || !block_table || !kv_lens || !granted)))
    return KVEV_EINVAL;
  if (B > KVEV_PAGED_MAX_REQUESTS) return KVEV_ENOTSUP;
  constexpr int kPerRequest = 4 * sizeof(int);
  if (B * kPerRequest > 48 * 1024 &&
      cudaFuncSetAttribute(tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           KVEV_PAGED_MAX_REQUESTS * kPerRequest) != cudaSuccess)
    return KVEV_ECUDA;
  TableParams p = {lens, new_lens, free_pages, free_count, block_table, kv_lens, cu_new, slots, positions, granted,
                   free_count_out, device_status, B, log2_of(page_size), num_pages, max_pages, T};
  return launched(launch_overlapped(tables_kernel, p, 1, kTableThreads, kPerRequest * B,
                                    static_cast<cudaStream_t>(stream)));
}

extern "C" int kvev_paged_release(const int32_t* lens, const int32_t* done, int B, int page_size, int num_pages,
                                  const int32_t* block_table, int max_pages, int32_t* free_pages,
                                  const int32_t* free_count, int32_t* lens_out, int32_t* free_count_out,
                                  int32_t* device_status, void* stream) {
  if (!free_pages || !free_count || !free_count_out || !device_status ||
      !tables_sizes(B, page_size, num_pages, max_pages) || (B > 0 && (!lens || !done || !block_table || !lens_out)))
    return KVEV_EINVAL;
  if (B > KVEV_PAGED_MAX_REQUESTS) return KVEV_ENOTSUP;
  ReleaseParams p = {lens, done, block_table, free_count, free_pages, lens_out, free_count_out, device_status,
                     B, log2_of(page_size), num_pages, max_pages};
  return launched(launch_overlapped(release_kernel, p, 1, kTableThreads, sizeof(int) * B,
                                    static_cast<cudaStream_t>(stream)));
}

extern "C" int kvev_paged_write(const kvev_paged_cache* cache, const void* k, const void* v, int64_t token_stride,
                                int64_t head_stride, const int32_t* slots, int T, int32_t* device_status,
                                void* stream) {
  WriteParams p = {};
  const int rc = paged_view(cache, &p.c);
  if (rc != KVEV_OK) return rc;
  if (!device_status || T < 0 || token_stride <= 0 || head_stride <= 0 || (token_stride & 7) || (head_stride & 7))
    return KVEV_EINVAL;
  if (T == 0) return KVEV_OK;
  if (!k || !v || !aligned16(k) || !aligned16(v) || !slots) return KVEV_EINVAL;
  p.k = static_cast<const uint4*>(k);
  p.v = static_cast<const uint4*>(v);
  p.token_stride = token_stride / 8;
  p.head_stride = head_stride / 8;
  p.slots = slots;
  p.T = T;
  p.status = device_status;
  const int64_t n = static_cast<int64_t>(T) * p.c.H_kv * p.c.dv;
  const int grid = static_cast<int>(std::min<int64_t>((n + kRowThreads - 1) / kRowThreads, 152 * 8));
  return launched(launch_overlapped(write_kernel, p, grid, kRowThreads, 0, static_cast<cudaStream_t>(stream)));
}

extern "C" int kvev_paged_gather(const kvev_paged_cache* cache, const int32_t* block_table, int max_pages,
                                 const int32_t* lens, int B, int S_cap, void* out_K, void* out_V,
                                 int32_t* device_status, void* stream) {
  PageGatherParams p = {};
  const int rc = paged_view(cache, &p.c);
  if (rc != KVEV_OK) return rc;
  if (!device_status || S_cap < 1 || !tables_sizes(B, cache->page_size, cache->num_pages, max_pages))
    return KVEV_EINVAL;
  if (B > KVEV_PAGED_MAX_REQUESTS) return KVEV_ENOTSUP;
  if (B == 0) return KVEV_OK;
  if (!block_table || !lens || !out_K || !out_V || !aligned16(out_K) || !aligned16(out_V)) return KVEV_EINVAL;
  p.table = block_table;
  p.lens = lens;
  p.B = B;
  p.max_pages = max_pages;
  p.S_cap = S_cap;
  p.out_K = static_cast<uint4*>(out_K);
  p.out_V = static_cast<uint4*>(out_V);
  p.status = device_status;
  page_gather_kernel<<<dim3((S_cap + kGatherRows - 1) / kGatherRows, B), kRowThreads, 0,
                       static_cast<cudaStream_t>(stream)>>>(p);
  return launched(cudaGetLastError());
}
