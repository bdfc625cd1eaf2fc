// paged_q8.cu -- paged caches of 8-bit codes: rows quantised as they are written, and whole prompts read back.
//
// A row x of d elements is held as e4m3 codes of x 2^-e and the byte e + 127, e the smallest whole number with
// max|x| <= 448 2^e: with max|x| = m 2^k, 1 <= m < 2, that is k - 8 for m <= 1.75 and k - 7 above.  The scale is a
// power of two, not max|x| / 448: the codes are floating-point, so what lies between two powers buys them no
// precision, x 2^-e is exact, each element is rounded once, and c 2^e is a value of the 16-bit type (for a row's
// codes span 2^-9 .. 448, so that e - 9 is at or above the type's least exponent, and where e is the largest the
// code 256, whose value would be past the type, is cut to 240).
#include <climits>

#include <cuda_fp16.h>

#include "paged.cuh"

namespace kvev {
namespace {

constexpr int kRowThreads = 256;
// Vectors of K and of V that a thread has in flight: with one, an 8K prompt is read back in 11.5 us, with two 10.6; with four
// 16K tokens are written in 38 us.
constexpr int kBatch = 2;
constexpr int kTokenShift = 3;   // most tokens of a CTA (write)
constexpr int kGatherShift = 4;  // positions of a CTA (gather)

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int launched(cudaError_t e) { return e == cudaSuccess ? KVEV_OK : KVEV_ECUDA; }

template <bool kFp16>
__device__ __forceinline__ float2 floats2(uint32_t u) {
  if (kFp16) return __half22float2(*reinterpret_cast<__half2*>(&u));
  return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
template <bool kFp16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  uint32_t u;
  if (kFp16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(b), "f"(a));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(b), "f"(a));
  return u;
}
// 32 bytes, in one store where they start at a 32-byte boundary.
__device__ __forceinline__ void store32(uint4* at, const uint4 (&v)[2], bool wide) {
  if (!wide) {
    at[0] = v[0];
    at[1] = v[1];
    return;
  }
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(v[0].x), "r"(v[0].y), "r"(v[0].z), "r"(v[0].w),
               "r"(v[1].x), "r"(v[1].y), "r"(v[1].z), "r"(v[1].w)
               : "memory");
}
// Codes of a (low byte) and b.
__device__ __forceinline__ uint32_t codes2(float a, float b) {
  uint16_t u;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(u) : "f"(b), "f"(a));
  return u;
}

// ---------------------------------------------------------------------------
// Write.  A thread holds 16 elements of a row, K's and V's, and the d / 16 threads of a row find its largest
// magnitude by shuffles.  One pass: 2 (2 d + d + 1) bytes a row, nothing else of note.
// ---------------------------------------------------------------------------
struct Q8WriteParams {
  PagedQ8View c;
  const uint4 *k, *v;
  long long token_stride, head_stride;  // in vectors of 8 elements
  const int* slots;
  int T, token_shift;
  int* status;
};

template <bool kFp16>
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {  // of two 16-bit values each; NaN if one of them is
  uint32_t r;
  if (kFp16) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// The exponent of a row whose largest magnitude is a.  (bits + 0x1fffff: the binary exponent goes up where the mantissa is past 0.75)
template <bool kFp16>
__device__ __forceinline__ int exponent_of(float a) {
  constexpr int kLo = kFp16 ? -15 : -120, kHi = kFp16 ? 8 : 120;
  return min(max(static_cast<int>((__float_as_uint(a) + 0x1fffffu) >> 23) - 127 - 8, kLo), kHi);
}

// 16 elements of a row as codes, with the row's exponent byte, for any row; the LANES threads of the row call it together.
template <bool kFp16, int LANES>
__device__ __noinline__ uint4 quantise_any(const uint4 x0, const uint4 x1, int* byte) {
  float f[16];
  const uint32_t u[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 z = floats2<kFp16>(u[i]);
    f[2 * i] = z.x;
    f[2 * i + 1] = z.y;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float m = fabsf(f[i]);
    if (m < INFINITY) a = fmaxf(a, m);
  }
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
  const int e = exponent_of<kFp16>(a);
  const float s = __uint_as_float(static_cast<uint32_t>(127 - e) << 23), top = e == (kFp16 ? 8 : 120) ? 240.f : 448.f;
  *byte = e + 127;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float z = f[4 * i + j];
      y[j] = fabsf(z) < INFINITY ? fminf(fmaxf(z * s, -top), top) : __uint_as_float(0x7fffffffu);
    }
    w[i] = codes2(y[0], y[1]) | codes2(y[2], y[3]) << 16;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The same; rows of finite elements, below the largest exponent, need no look at each element: their maximum comes from pairs of 16-bit
// values and nothing is past 448 (16K tokens 23.7 us with quantise_any for all rows, which the instructions bound).
template <bool kFp16, int LANES>
__device__ __forceinline__ uint4 quantise(const uint4 (&x)[2], int* byte) {
  const uint32_t u[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
  uint32_t m = u[0] & 0x7fff7fffu;
#pragma unroll
  for (int i = 1; i < 8; ++i) m = max2<kFp16>(m, u[i] & 0x7fff7fffu);
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) m = max2<kFp16>(m, __shfl_xor_sync(0xffffffffu, m, o));
  m = max2<kFp16>(m, m >> 16 | m << 16);
  const float a = floats2<kFp16>(m).x;
  const int e = exponent_of<kFp16>(a);
  if (!__all_sync(0xffffffffu, a < INFINITY && e < (kFp16 ? 8 : 120))) return quantise_any<kFp16, LANES>(x[0], x[1], byte);
  const float s = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
  *byte = e + 127;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 y = floats2<kFp16>(u[2 * i]), z = floats2<kFp16>(u[2 * i + 1]);
    w[i] = codes2(y.x * s, y.y * s) | codes2(z.x * s, z.y * s) << 16;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int D, bool kFp16>
__global__ void __launch_bounds__(kRowThreads) q8_write_kernel(const __grid_constant__ Q8WriteParams p) {
  constexpr int kLanes = D / 16;
  __shared__ int slot_of[1 << kTokenShift];  // a token's slot, -1: none
  pdl_wait();
  pdl_trigger();
  const int t0 = blockIdx.x << p.token_shift;
  if (threadIdx.x < (1 << p.token_shift)) {
    const int t = t0 + threadIdx.x;
    int slot = t < p.T ? p.slots[t] : -1;
    if (slot >= 0 && (slot >> p.c.page_shift) >= p.c.num_pages) {
      atomicOr(p.status, kStatusDevice);
      slot = -1;
    }
    slot_of[threadIdx.x] = slot;
  }
  __syncthreads();
  const int n = (p.c.H_kv << p.token_shift) * kLanes;
  for (int i0 = 0; i0 < n; i0 += kBatch * kRowThreads) {
    uint4 a[kBatch][2], b[kBatch][2];
    int slot[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int i = i0 + q * kRowThreads + threadIdx.x, c = i % kLanes, k = (i / kLanes) & ((1 << p.token_shift) - 1);
      const int h = (i / kLanes) >> p.token_shift;
      slot[q] = i < n ? slot_of[k] : -1;
      a[q][0] = a[q][1] = b[q][0] = b[q][1] = make_uint4(0, 0, 0, 0);
      if (slot[q] >= 0) {
        const long long from = (t0 + k) * p.token_stride + h * p.head_stride + 2 * c;
        a[q][0] = p.k[from];
        a[q][1] = p.k[from + 1];
        b[q][0] = p.v[from];
        b[q][1] = p.v[from + 1];
      }
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int i = i0 + q * kRowThreads + threadIdx.x, c = i % kLanes, h = (i / kLanes) >> p.token_shift;
      int ea, eb;
      const uint4 ca = quantise<kFp16, kLanes>(a[q], &ea), cb = quantise<kFp16, kLanes>(b[q], &eb);
      if (slot[q] >= 0) {
        const int page = slot[q] >> p.c.page_shift, r = slot[q] & ((1 << p.c.page_shift) - 1);
        const long long at = page * p.c.page_stride + r * p.c.token_stride + h * p.c.head_stride + c * 16;
        *reinterpret_cast<uint4*>(p.c.K + at) = ca;
        *reinterpret_cast<uint4*>(p.c.V + at) = cb;
        if (c == 0) {
          const long long es = page * p.c.scale_page + (h << p.c.page_shift) + r;
          p.c.K_scale[es] = static_cast<uint8_t>(ea);
          p.c.V_scale[es] = static_cast<uint8_t>(eb);
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Gather: the values of a prompt's rows as 16-bit rows; 16 codes, 32 bytes, a thread.
// ---------------------------------------------------------------------------
struct Q8GatherParams {
  PagedQ8View c;
  const int *table, *lens;
  int B, max_pages, S_cap, blocks;  // blocks: CTAs per request
  uint4 *out_K, *out_V;
  bool wide;  // both at 32-byte boundaries
  int* status;
};

template <bool kFp16>
__device__ __forceinline__ void values16(uint4 codes, uint32_t byte, uint4 (&out)[2]) {
  const float s = __uint_as_float(byte << 23);
  const uint32_t u[4] = {codes.x, codes.y, codes.z, codes.w};
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint2 h;
    asm("{\n\t.reg .b16 a, b;\n\t"
        "mov.b32 {a, b}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(h.x), "=r"(h.y) : "r"(u[i]));
    const float2 a = floats2<true>(h.x), b = floats2<true>(h.y);
    w[2 * i] = pack2<kFp16>(a.x * s, a.y * s);
    w[2 * i + 1] = pack2<kFp16>(b.x * s, b.y * s);
  }
  out[0] = make_uint4(w[0], w[1], w[2], w[3]);
  out[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

template <int D, bool kFp16>
__global__ void __launch_bounds__(kRowThreads) q8_gather_kernel(const __grid_constant__ Q8GatherParams p) {
  constexpr int kLanes = D / 16;
  __shared__ int slot_of[1 << kGatherShift];  // a position's slot, -1: none
  pdl_wait();
  pdl_trigger();
  const int s = blockIdx.x / p.blocks, k0 = (blockIdx.x - s * p.blocks) << kGatherShift;
  const int len = p.lens[s], n = min(max(len, 0), min(p.S_cap, p.max_pages << p.c.page_shift));
  if (n != len && threadIdx.x == 0 && k0 == 0) atomicOr(p.status, kStatusDevice);
  if (k0 >= n) return;
  if (threadIdx.x < (1 << kGatherShift)) {
    const int k = k0 + threadIdx.x;
    int slot = -1;
    if (k < n) {
      const int page = p.table[static_cast<long long>(s) * p.max_pages + (k >> p.c.page_shift)];
      if (static_cast<unsigned>(page) < static_cast<unsigned>(p.c.num_pages))
        slot = (page << p.c.page_shift) + (k & ((1 << p.c.page_shift) - 1));
      else
        atomicOr(p.status, kStatusDevice);
    }
    slot_of[threadIdx.x] = slot;
  }
  __syncthreads();
  const int total = (p.c.H_kv << kGatherShift) * kLanes;
  const long long out0 = static_cast<long long>(s) * p.c.H_kv * p.S_cap + k0;
  for (int i0 = threadIdx.x; i0 < total; i0 += kBatch * kRowThreads) {
    uint4 a[kBatch], b[kBatch];
    uint32_t ea[kBatch], eb[kBatch];
    long long at[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int i = i0 + q * kRowThreads, c = i % kLanes, k = (i / kLanes) & ((1 << kGatherShift) - 1), h = (i / kLanes) >> kGatherShift;
      const int slot = i < total ? slot_of[k] : -1;
      at[q] = -1;
      if (slot < 0) continue;
      const int page = slot >> p.c.page_shift, r = slot & ((1 << p.c.page_shift) - 1);
      const long long from = page * p.c.page_stride + r * p.c.token_stride + h * p.c.head_stride + c * 16;
      const long long es = page * p.c.scale_page + (h << p.c.page_shift) + r;
      at[q] = ((out0 + static_cast<long long>(h) * p.S_cap + k) * kLanes + c) * 2;
      a[q] = *reinterpret_cast<const uint4*>(p.c.K + from);
      b[q] = *reinterpret_cast<const uint4*>(p.c.V + from);
      ea[q] = p.c.K_scale[es];
      eb[q] = p.c.V_scale[es];
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      if (at[q] < 0) continue;
      uint4 o[2];
      values16<kFp16>(a[q], ea[q], o);
      store32(p.out_K + at[q], o, p.wide);
      values16<kFp16>(b[q], eb[q], o);
      store32(p.out_V + at[q], o, p.wide);
    }
  }
}

}  // namespace

int paged_q8_view(const kvev_paged_q8_cache* c, PagedQ8View* v) {
  if (!c || !c->K || !c->V || !aligned16(c->K) || !aligned16(c->V) || !c->K_scale || !c->V_scale) return KVEV_EINVAL;
  if (c->num_pages < 1 || !paged_page_size(c->page_size) || c->H_kv < 1 ||
      static_cast<int64_t>(c->num_pages) * c->page_size > INT_MAX)
    return KVEV_EINVAL;
  if (c->dtype != KVEV_BF16 && c->dtype != KVEV_FP16) return KVEV_EINVAL;
  for (int64_t st : {c->page_stride, c->token_stride, c->head_stride})
    if (st <= 0 || (st & 15)) return KVEV_EINVAL;
  if (c->scale_page_stride < static_cast<int64_t>(c->H_kv) * c->page_size) return KVEV_EINVAL;
  if (c->d != 64 && c->d != 128) return KVEV_ENOTSUP;
  v->K = static_cast<uint8_t*>(c->K);
  v->V = static_cast<uint8_t*>(c->V);
  v->K_scale = c->K_scale;
  v->V_scale = c->V_scale;
  v->page_stride = c->page_stride;
  v->token_stride = c->token_stride;
  v->head_stride = c->head_stride;
  v->scale_page = c->scale_page_stride;
  v->num_pages = c->num_pages;
  v->page_shift = log2_of(c->page_size);
  v->H_kv = c->H_kv;
  v->d = c->d;
  v->fp16 = c->dtype == KVEV_FP16;
  return KVEV_OK;
}

}  // namespace kvev

using namespace kvev;

extern "C" int kvev_paged_q8_write(const kvev_paged_q8_cache* cache, const void* k, const void* v, int64_t token_stride,
                                   int64_t head_stride, const int32_t* slots, int T, int32_t* device_status,
                                   void* stream) {
  Q8WriteParams p = {};
  const int rc = paged_q8_view(cache, &p.c);
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
  // few tokens: a CTA each; more: as many as leave every SM one or two (2,000 tokens 9.2 us with a CTA each, 4.1 with eight to a CTA)
  p.token_shift = T < 256 ? 0 : T < 512 ? 1 : T < 1024 ? 2 : kTokenShift;
  const int grid = static_cast<int>((static_cast<int64_t>(T) + (1 << p.token_shift) - 1) >> p.token_shift);
  const auto fn = p.c.d == 64 ? (p.c.fp16 ? q8_write_kernel<64, true> : q8_write_kernel<64, false>)
                              : (p.c.fp16 ? q8_write_kernel<128, true> : q8_write_kernel<128, false>);
  return launched(launch_overlapped(fn, p, grid, kRowThreads, 0, static_cast<cudaStream_t>(stream)));
}

extern "C" int kvev_paged_q8_gather(const kvev_paged_q8_cache* cache, const int32_t* block_table, int max_pages,
                                    const int32_t* lens, int B, int S_cap, void* out_K, void* out_V,
                                    int32_t* device_status, void* stream) {
  Q8GatherParams p = {};
  const int rc = paged_q8_view(cache, &p.c);
  if (rc != KVEV_OK) return rc;
  if (!device_status || S_cap < 1 || B < 0 || max_pages < 1 || static_cast<int64_t>(max_pages) * cache->page_size > kMaxTokens)
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
  p.wide = ((reinterpret_cast<uintptr_t>(out_K) | reinterpret_cast<uintptr_t>(out_V)) & 31u) == 0;
  p.status = device_status;
  p.blocks = ((S_cap - 1) >> kGatherShift) + 1;
  if (static_cast<int64_t>(p.blocks) * B > INT_MAX) return KVEV_ENOTSUP;  // CTAs of a launch
  const auto fn = p.c.d == 64 ? (p.c.fp16 ? q8_gather_kernel<64, true> : q8_gather_kernel<64, false>)
                              : (p.c.fp16 ? q8_gather_kernel<128, true> : q8_gather_kernel<128, false>);
  return launched(launch_overlapped(fn, p, p.blocks * B, kRowThreads, 0, static_cast<cudaStream_t>(stream)));
}
