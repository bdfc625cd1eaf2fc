// paged.cu -- the paged cache in front of the eviction: block tables and slots
// built on the GPU, rows written to their slots, and whole prompts gathered
// into the contiguous caches that the prefill eviction reads.
#include <climits>

#include "paged.cuh"

namespace kvev {
namespace {

// ---------------------------------------------------------------------------
// Block tables.  Everything a step needs follows from two prefix sums over the
// requests, of new tokens and of new pages, which every CTA forms in its own shared
// memory; then tokens and pages are dealt over all threads, each finding its request by
// bisection.  Whatever is written may be an input's own memory (lengths, the
// count): nothing is written before every CTA has read all of it, so the CTAs are one
// cluster, of eight when there may be more than a thread's worth.  Bound by its round trips to L2
// (lengths; table or stack), 2 us, and the launch.
// ---------------------------------------------------------------------------
constexpr int kTableThreads = 1024;  // most of a CTA; no more than requests, tokens or pages
constexpr int kTableCluster = 8;  // most CTAs of a cluster that every device takes

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

// Every CTA of the cluster is here, and what their threads read before has been read.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}
__device__ __forceinline__ int cluster_size() {
  int n;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
  return n;
}

// Sets the flag at this place of every CTA's shared memory (all of them are running).
__device__ __forceinline__ void cluster_raise(int* flag) {
  const uint32_t at = smem_u32(flag);
  for (int r = 0; r < cluster_size(); ++r)
    asm volatile(
        "{\n\t.reg .b32 a;\n\t"
        "mapa.shared::cluster.u32 a, %0, %1;\n\t"
        "st.shared::cluster.u32 [a], %2;\n\t}" ::"r"(at), "r"(r), "r"(1)
        : "memory");
}

__global__ void __launch_bounds__(kTableThreads) tables_kernel(const __grid_constant__ TableParams p) {
  extern __shared__ int sm[];
  int* const cu = sm;                     // [B + 1] first token
  int* const first = sm + p.B + 1;        // [B] new pages of the requests before
  int* const len = sm + 2 * p.B + 1;      // [B] tokens held
  int* const grant = sm + 3 * p.B + 1;    // [B] new tokens, -1: refused
  __shared__ longlong2 ws[32];
  __shared__ long long carry[2];
  __shared__ int given;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  if (tid == 0) { carry[0] = carry[1] = 0; given = 0; }
  const int top = *p.free_count, count = min(max(top, 0), p.num_pages);
  bool bad = top != count;
  __syncthreads();
  for (int s0 = 0; s0 < p.B; s0 += blockDim.x) {
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
    if (tid == blockDim.x - 1) { carry[0] = c0 + upto.x; carry[1] = c1 + upto.y; }
    if (s < p.B) {
      const bool ok = fits && (k == 0 || c1 + upto.y <= count);
      cu[s] = static_cast<int>(min(c0 + upto.x - q, static_cast<long long>(INT_MAX)));
      first[s] = static_cast<int>(min(c1 + upto.y - k, static_cast<long long>(INT_MAX)));
      len[s] = n;
      grant[s] = ok ? q : -1;
      if (ok && k > 0) atomicMax(&given, static_cast<int>(c1 + upto.y));
    }
    __syncthreads();
  }
  if (tid == 0) cu[p.B] = static_cast<int>(min(carry[0], static_cast<long long>(INT_MAX)));
  cluster_sync();
  const int total = cu[p.B];
  const int t0 = blockIdx.x * blockDim.x + tid, step = cluster_size() * blockDim.x;
  if (t0 == 0) {
    *p.count_out = count - given;
    bad |= total > p.T;
  }
  for (int s = t0; s <= p.B; s += step) {
    p.cu[s] = cu[s];
    if (s < p.B) {
      p.granted[s] = grant[s] >= 0;
      p.kv_lens[s] = len[s] + max(grant[s], 0);  // (not from cu, which is cut off at INT_MAX)
    }
  }
  // pages given out, the k-th of them to the request whose range holds k
  for (int k = t0; k < given; k += step) {
    const int s = find_request(first, p.B, k);
    p.table[static_cast<long long>(s) * p.max_pages + pages_of(len[s], p.page_shift) + k - first[s]] =
        p.free_pages[count - 1 - k];
  }
  for (int t = t0; t < p.T; t += step) {
    int slot = -1, pos = -1;
    if (t < total) {
      const int s = find_request(cu, p.B, t);
      if (grant[s] >= 0) {
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
  int* const first = sm;        // [B] pages released by the requests before
  int* const len = sm + p.B;    // [B] what is left of the lengths
  __shared__ longlong2 ws[32];
  __shared__ long long carry;
  __shared__ int any_odd;  // an entry outside the pool comes back
  const int tid = threadIdx.x;
  if (tid == 0) { carry = 0; any_odd = 0; }
  __syncwarp();
  cluster_arrive();  // (from where it is waited for on, other CTAs may set any_odd)
  pdl_wait();
  pdl_trigger();
  const int top = *p.free_count, count = min(max(top, 0), p.num_pages);
  bool bad = top != count;
  __syncthreads();
  for (int s0 = 0; s0 < p.B; s0 += blockDim.x) {
    const int s = s0 + tid;
    int k = 0;
    if (s < p.B) {
      const int n = p.lens[s];
      const bool done = p.done[s] != 0;
      bad |= n < 0;
      k = done ? pages_of(max(n, 0), p.page_shift) : 0;
      bad |= k > p.max_pages;
      k = min(k, p.max_pages);
      len[s] = done ? 0 : n;
    }
    const longlong2 upto = block_scan(k, 0, ws);
    const long long c = carry;
    __syncthreads();
    if (tid == blockDim.x - 1) carry = c + upto.x;
    if (s < p.B) first[s] = static_cast<int>(min(c + upto.x - k, static_cast<long long>(INT_MAX)));
    __syncthreads();
  }
  const int room = p.num_pages - count;
  const int all = static_cast<int>(min(carry, static_cast<long long>(INT_MAX)));
  const bool cut = carry > all;
  const int total = min(all, room);
  const int t0 = blockIdx.x * blockDim.x + tid, step = cluster_size() * blockDim.x;
  auto entry = [&](int k) {  // the k-th entry that comes back
    const int s = find_request(first, p.B, k);
    return p.table[static_cast<long long>(s) * p.max_pages + k - first[s]];
  };
  auto outside = [&](int page) { return static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_pages); };
  // Entries outside the pool must not reach the stack: every entry is looked at before the first is put there, and
  // each CTA is told whether there was one, by the barrier after which outputs may be written.  A thread keeps its
  // first four, in flight together.  Those for pages that others keep are outside too, and in order.
  int page[4];
  bool odd = false;
  auto look = [&](int page) {
    odd |= outside(page);
    bad |= outside(page) && page != KVEV_PAGED_KEPT_PAGE;
  };
#pragma unroll
  for (int q = 0; q < 4; ++q) page[q] = t0 + q * step < all ? entry(t0 + q * step) : 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) look(page[q]);
  for (long long k = t0 + 4 * step; k < all; k += step) look(entry(static_cast<int>(k)));
  __syncwarp();
  cluster_wait();
  if (odd) cluster_raise(&any_odd);
  __syncwarp();
  cluster_sync();
  for (int s = t0; s < p.B; s += step) p.lens_out[s] = len[s];
  if (any_odd == 0) {
    bad |= carry > room;
    if (t0 == 0) *p.count_out = count + total;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (t0 + q * step < total) p.free_pages[count + t0 + q * step] = page[q];
    for (int k = t0 + 4 * step; k < total; k += step) p.free_pages[count + k] = entry(k);
  } else if (blockIdx.x == 0) {  // one CTA puts the others there, in order
    long long kept = 0;
    for (long long k0 = 0; k0 < all; k0 += blockDim.x) {
      const int x = k0 + tid < all ? entry(static_cast<int>(k0 + tid)) : -1;
      const long long upto = kept + block_scan(outside(x) ? 0 : 1, 0, ws).x;
      if (!outside(x) && upto <= room) p.free_pages[count + upto - 1] = x;
      __syncthreads();
      if (tid == blockDim.x - 1) carry = upto;
      __syncthreads();
      kept = carry;
    }
    bad |= kept > room || cut;
    if (tid == 0) *p.count_out = count + static_cast<int>(min(kept, static_cast<long long>(room)));
  }
  if (bad) atomicOr(p.status, kStatusDevice);
}

// ---------------------------------------------------------------------------
// Rows.  A CTA moves the rows of 2^row_shift tokens, of every head, K and V: its
// vectors of 16 bytes are numbered head by head, token by token, and a thread has the
// loads of kBatch of them in flight, K's and V's, before the first store.  Plain loads, not
// __ldg, here and in the attention: the launches overlap the kernels before them, which may write
// what is read, so it is constant only from pdl_wait on and not for as long as the grid exists.
// ---------------------------------------------------------------------------
struct WriteParams {
  PagedView c;
  const uint4 *k, *v;
  long long token_stride, head_stride;  // in vectors
  const int* slots;
  int T, row_shift, dv_shift;
  int* status;
};

constexpr int kRowThreads = 256;
constexpr int kBatch = 4;
constexpr int kMaxRowShift = 3;  // 16K tokens' rows 21.4 us; with 2 21.5, 4 22.1, 5 24.9

__global__ void __launch_bounds__(kRowThreads) write_kernel(const __grid_constant__ WriteParams p) {
  __shared__ long long to[1 << kMaxRowShift];  // a token's row in the pool, -1: none
  pdl_wait();
  pdl_trigger();
  const int t0 = blockIdx.x << p.row_shift;
  if (threadIdx.x < (1 << p.row_shift)) {
    const int t = t0 + threadIdx.x;
    const int slot = t < p.T ? p.slots[t] : -1, page = slot >> p.c.page_shift;
    long long at = -1;
    if (slot >= 0) {
      if (page < p.c.num_pages) at = page * p.c.page_stride + (slot & ((1 << p.c.page_shift) - 1)) * p.c.token_stride;
      else atomicOr(p.status, kStatusDevice);
    }
    to[threadIdx.x] = at;
  }
  __syncthreads();
  const int n = p.c.H_kv << (p.row_shift + p.dv_shift);
  for (int i0 = threadIdx.x; i0 < n; i0 += kBatch * kRowThreads) {
    uint4 a[kBatch], b[kBatch];
    long long at[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int i = i0 + q * kRowThreads;
      const int x = i & ((1 << p.dv_shift) - 1), k = (i >> p.dv_shift) & ((1 << p.row_shift) - 1), h = i >> (p.dv_shift + p.row_shift);
      at[q] = i < n ? to[k] : -1;
      if (at[q] < 0) continue;
      at[q] += h * p.c.head_stride + x;
      const long long from = (t0 + k) * p.token_stride + h * p.head_stride + x;
      a[q] = p.k[from];
      b[q] = p.v[from];
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (at[q] >= 0) {
        const_cast<uint4*>(p.c.K)[at[q]] = a[q];
        const_cast<uint4*>(p.c.V)[at[q]] = b[q];
      }
  }
}

struct PageGatherParams {
  PagedView c;
  const int *table, *lens;
  int B, max_pages, S_cap, dv_shift, blocks;  // blocks: CTAs per request
  uint4 *out_K, *out_V;
  int* status;
};

constexpr int kGatherShift = 4;  // 16 positions of a CTA

__global__ void __launch_bounds__(kRowThreads) page_gather_kernel(const __grid_constant__ PageGatherParams p) {
  __shared__ long long from[1 << kGatherShift];  // a position's row in the pool, -1: none
  pdl_wait();
  pdl_trigger();
  const int s = blockIdx.x / p.blocks, k0 = (blockIdx.x - s * p.blocks) << kGatherShift;
  const int len = p.lens[s], n = min(max(len, 0), min(p.S_cap, p.max_pages << p.c.page_shift));
  if (n != len && threadIdx.x == 0 && k0 == 0) atomicOr(p.status, kStatusDevice);
  if (k0 >= n) return;
  if (threadIdx.x < (1 << kGatherShift)) {
    const int k = k0 + threadIdx.x;
    long long at = -1;
    if (k < n) {
      const int page = p.table[static_cast<long long>(s) * p.max_pages + (k >> p.c.page_shift)];
      if (static_cast<unsigned>(page) < static_cast<unsigned>(p.c.num_pages))
        at = page * p.c.page_stride + (k & ((1 << p.c.page_shift) - 1)) * p.c.token_stride;
      else
        atomicOr(p.status, kStatusDevice);
    }
    from[threadIdx.x] = at;
  }
  __syncthreads();
  const int total = p.c.H_kv << (kGatherShift + p.dv_shift);
  const long long out0 = static_cast<long long>(s) * p.c.H_kv * p.S_cap + k0;
  for (int i0 = threadIdx.x; i0 < total; i0 += kBatch * kRowThreads) {
    uint4 a[kBatch], b[kBatch];
    long long at[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int i = i0 + q * kRowThreads;
      const int x = i & ((1 << p.dv_shift) - 1), k = (i >> p.dv_shift) & ((1 << kGatherShift) - 1), h = i >> (p.dv_shift + kGatherShift);
      const long long row = i < total ? from[k] : -1;
      at[q] = -1;
      if (row < 0) continue;
      at[q] = ((out0 + static_cast<long long>(h) * p.S_cap + k) << p.dv_shift) + x;
      a[q] = p.c.K[row + h * p.c.head_stride + x];
      b[q] = p.c.V[row + h * p.c.head_stride + x];
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (at[q] >= 0) {
        p.out_K[at[q]] = a[q];
        p.out_V[at[q]] = b[q];
      }
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int launched(cudaError_t e) { return e == cudaSuccess ? KVEV_OK : KVEV_ECUDA; }

int table_threads(int64_t work) { return work >= kTableThreads ? kTableThreads : work <= 32 ? 32 : static_cast<int>((work + 31) & ~31); }

bool tables_sizes(int B, int page_size, int num_pages, int max_pages) {
  return B >= 0 && paged_page_size(page_size) && num_pages >= 1 && max_pages >= 1 &&
         static_cast<int64_t>(num_pages) * page_size <= INT_MAX && static_cast<int64_t>(max_pages) * page_size <= kMaxTokens;
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
  if (!free_pages || !free_count || !cu_new || !free_count_out || !device_status || T < 0 || T > kMaxTokens ||
      !tables_sizes(B, page_size, num_pages, max_pages) || (T > 0 && (!slots || !positions)) ||
      (B > 0 && (!lens || !new_lens || !block_table || !kv_lens || !granted)))
    return KVEV_EINVAL;
  if (B > KVEV_PAGED_MAX_REQUESTS) return KVEV_ENOTSUP;
  constexpr int kPerRequest = 4 * sizeof(int);
  if (B * kPerRequest > 47 * 1024 &&
      cudaFuncSetAttribute(tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           KVEV_PAGED_MAX_REQUESTS * kPerRequest + sizeof(int)) != cudaSuccess)
    return KVEV_ECUDA;
  TableParams p = {lens, new_lens, free_pages, free_count, block_table, kv_lens, cu_new, slots, positions, granted,
                   free_count_out, device_status, B, log2_of(page_size), num_pages, max_pages, T};
  const int ctas = T > kTableThreads ? kTableCluster : 1;
  return launched(launch_overlapped(tables_kernel, p, ctas, table_threads(B > T ? B : T), kPerRequest * B + sizeof(int),
                                    static_cast<cudaStream_t>(stream), ctas));
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
  constexpr int kPerRequest = 2 * sizeof(int);
  if (B * kPerRequest > 47 * 1024 &&
      cudaFuncSetAttribute(release_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           KVEV_PAGED_MAX_REQUESTS * kPerRequest) != cudaSuccess)
    return KVEV_ECUDA;
  // how many pages come back only the device knows: more than a CTA's threads, as far as the table's size tells
  const int64_t pages = static_cast<int64_t>(B) * max_pages;
  const int ctas = pages > kTableThreads ? kTableCluster : 1;
  return launched(launch_overlapped(release_kernel, p, ctas, table_threads(pages), kPerRequest * B,
                                    static_cast<cudaStream_t>(stream), ctas));
}

extern "C" int kvev_paged_write(const kvev_paged_cache* cache, const void* k, const void* v, int64_t token_stride,
                                int64_t head_stride, const int32_t* slots, int T, int32_t* device_status,
                                void* stream) {
  WriteParams p = {};
  const int rc = paged_view(cache, &p.c);
  if (rc != KVEV_OK) return rc;
  if (!device_status || T < 0 || T > kMaxTokens || token_stride <= 0 || head_stride <= 0 || (token_stride & 7) || (head_stride & 7))
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
  p.dv_shift = log2_of(p.c.dv);
  // few tokens: a CTA each; many: as many as keep a batch of every thread full
  p.row_shift = T < 2048 ? 0 : kMaxRowShift;
  const int grid = static_cast<int>((static_cast<int64_t>(T) + (1 << p.row_shift) - 1) >> p.row_shift);
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
  p.dv_shift = log2_of(p.c.dv);
  p.blocks = ((S_cap - 1) >> kGatherShift) + 1;
  if (static_cast<int64_t>(p.blocks) * B > INT_MAX) return KVEV_ENOTSUP;  // CTAs of a launch
  return launched(launch_overlapped(page_gather_kernel, p, p.blocks * B, kRowThreads, 0, static_cast<cudaStream_t>(stream)));
}
