// paged_q8_few.cuh -- attention of a few rows (single tokens of up to 16 heads to a KV head) over paged caches of
// 8-bit codes, which the tensor core takes as they are.
//
// A key k holds codes and powers of two, K[k] = 2^a_k A[k], V[k] = 2^b_k B[k], A and B e4m3.  A row needs
//   y_k = log2(e) scale 2^a_k (q . A[k]),  l = sum_k 2^(y_k - m),  o = sum_k 2^(y_k + b_k) B[k] / (2^m l).
// Both products have one operand in e4m3 already, and the tensor core wants the other in it too.  With 16 columns the
// least it takes and a few rows to a KV head there is room for it: q and the weights are split into four e4m3
// parts each, x = x0 + 2^-5 x1 + 2^-10 x2 + 2^-15 x3, a part the rounded rest times 2^5, and each part is a
// column.  (Below 2^8 a rest is at most 2^3: it fits.)  An x in [2^-1, 2^8) is held to 16 bits of its own and more;
// below, to 2^-25: rows of q scaled to [2^7, 2^8) lose under 2^-32 of their largest element, and weights at most 2^-30
// of the largest, where the 16-bit kernel's lose 2^-9 of their own size.
// The weights that go to the second product are 2^(y_k + b_k) with a running maximum of their own: a key of little
// weight may hold values that outweigh all others'.
//
// Layout as in paged_attn.cuh: keys on the lanes, S^T = A q^T (K-major codes as loaded), a thread per key forms
// its key's weights, O^T += B^T w^T with the codes of V as the operand whose key index runs slowest.  Two sides take
// the key tiles in turn; the schedule, its pieces and their merge are the same.
#pragma once
#include "paged_attn.cuh"

namespace kvev {
namespace {

constexpr int kFewMode = kQ8 | kFewOnly;
constexpr int kFewThreads = Split<kFewMode>::kThreads;
constexpr int kQParts = 4;       // e4m3 parts of a row of q or of weights
constexpr float kRest = 32.f;    // what a rest is multiplied by
constexpr float kFewRaise = 3.f; // a maximum is raised when a tile's is this much above it,
constexpr float kFewUp = 5.f;    // and the weights are 2^kFewUp larger: up to 2^8
constexpr int kRowGroup = 4;     // rows that a thread works on at once:
constexpr int kGroupCols = kQParts * kRowGroup;  // columns [part][row] of such a group
constexpr int kFewCols = kQParts * kFewRows;     // columns of a side's scores, and of its output: group after group
constexpr int kFewCtas = 2;      // CTAs of an SM

template <int D>
struct Q8Smem {
  // rows of 64 or 128 bytes: as for 16-bit rows of 64 elements
  static constexpr bool kHeadsOuter = true;
  static constexpr int kTileBytes = kRows * D;
  static constexpr int kStages = D == 128 ? 5 : 10;
  uint8_t kv[kStages][kTileBytes];
  uint8_t p[2][kFewCols * kRows];  // the sides' weights [column][128 keys]
  uint8_t q[kFewCols * D];         // [column][D]
  float qscale[2][kFewRows];       // of an entry's rows: log2(e) scale over their power of two
  float m[2][kFewRows], mz[2][kFewRows], l[2][kFewRows];  // the sides' maxima, the weights' maxima, sums
  Entry ring[kEntries];
  uint64_t qfull[2], qempty, full[kStages], empty[kStages];  // (qfull: of every other entry)
  uint64_t sfull[2], pfull[2], ofull[2];
  uint64_t efull[kEntries], eempty[kEntries];
  uint64_t xfull, xfree, done;
  long long carry, start;
  union {
    float red[2][2][4][kFewRows];  // a side's warps' maxima, or sums, of the rows
    long long scan[16];
  };
  int last[2];
  int abort_flag;
  uint32_t tmem_slot;
};
// (1 KB of an SM's 228 goes to each CTA beside what it asks for)
static_assert(kFewCtas * (sizeof(Q8Smem<64>) + 1024) <= 228 * 1024 && kFewCtas * (sizeof(Q8Smem<128>) + 1024) <= 228 * 1024,
              "shared memory of an SM");

// D(tmem) (+)= A B, e4m3 operands in shared memory, fp32 sums.  From a whole converged warp.
__device__ __forceinline__ void umma8_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// e4m3 operands, fp32 D; A K-major, or with its M index contiguous.
template <bool kAm>
__host__ __device__ constexpr uint32_t idesc8(int M, int N) {
  return (1u << 4) | (kAm ? 1u << 15 : 0u) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
// Descriptor of rows of W bytes (64 or 128) under the swizzle of that width, groups of 8 rows 8 W bytes apart: rows along M or N with
// K contiguous, or rows along K with M contiguous.  (Rows of 64 bytes as the latter give 64 of the 128 lanes: the others read the
// same again, `between` 0, and nothing reads them.)
template <int W>
__device__ __forceinline__ uint64_t rows_desc(uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>((8 * W) >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(W == 128 ? 2 : 4) << 61;
  return d;
}
// Where the 16-byte chunk c of row r lies.
template <int W>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
  return r * W + ((W == 128 ? c ^ (r & 7) : c ^ ((r >> 1) & 3)) << 4);
}

__device__ __forceinline__ uint32_t codes2(float a, float b) {  // of a (low byte) and b
  uint16_t u;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(u) : "f"(b), "f"(a));
  return u;
}
__device__ __forceinline__ float2 floats_of_codes2(uint32_t c) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(c)));
  return __half22float2(*reinterpret_cast<__half2*>(&h));
}
// The parts of two values: codes of a (low byte) and b.
__device__ __forceinline__ void parts2(float a, float b, uint32_t (&c)[kQParts]) {
#pragma unroll
  for (int q = 0; q < kQParts; ++q) {
    c[q] = codes2(a, b);
    if (q + 1 < kQParts) {
      const float2 f = floats_of_codes2(c[q]);
      a = (a - f.x) * kRest;
      b = (b - f.y) * kRest;
    }
  }
}

// Rows in whole groups: 4, 8 or 16.
__device__ __forceinline__ int rows_held(int rows) { return rows <= 4 ? 4 : rows <= 8 ? 8 : 16; }
// The column of part q of row r.
__device__ __forceinline__ int column_of(int q, int r) { return r / kRowGroup * kGroupCols + q * kRowGroup + r % kRowGroup; }

// ---- warp 3: the rows of q in parts --------------------------------------------------------

template <int D, bool kFp16>
__device__ __forceinline__ void split_queries(const PagedAttnParams& p, Q8Smem<D>& sm) {
  constexpr int kLanes = D / 16;
  const int lane = threadIdx.x & 31, c = lane % kLanes;
  uint32_t qn = 0;
  for (uint32_t e = 0;; ++e, ++qn) {
    const Entry en = take(p, sm, e);
    if (uniform(en.n) == 0) return;
    const int rows = uniform(en.n) * p.G, R = rows_held(rows);
    uint4 x[2];
    auto fetch = [&](int r) {
      x[0] = x[1] = make_uint4(0, 0, 0, 0);
      if (r < rows) {
        const int i = r / p.G, head = en.h * p.G + r - i * p.G;
        const uint8_t* at = p.q + static_cast<long long>(en.tok0 + i) * p.q_token + static_cast<long long>(head) * p.q_head + c * 32;
        x[0] = *reinterpret_cast<const uint4*>(at);
        x[1] = *reinterpret_cast<const uint4*>(at + 16);
      }
    };
    fetch(lane / kLanes);
    if (!attn_wait_warp(sm, &sm.qempty, (qn & 1) ^ 1, p.status)) return;
    for (int r0 = 0; r0 < R; r0 += 32 / kLanes) {
      const int r = r0 + lane / kLanes;
      const uint32_t u[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
      float f[16], a = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float2 z;
        if (kFp16) z = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
        else z = make_float2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
        f[2 * i] = z.x;
        f[2 * i + 1] = z.y;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (!(fabsf(f[i]) < INFINITY)) f[i] = __uint_as_float(0x7fffffffu);  // (an infinity gives NaN rows, as its products do)
        a = fmaxf(a, fabsf(f[i]));
      }
#pragma unroll
      for (int o = kLanes / 2; o; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
      // 2^s a in [2^7, 2^8)
      const int s = min(max(7 - (static_cast<int>(__float_as_uint(a) >> 23) - 127), -120), 120);
      const float up = __uint_as_float(static_cast<uint32_t>(s + 127) << 23);
      uint32_t w[kQParts][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t lo[kQParts], hi[kQParts];
        parts2(f[4 * i] * up, f[4 * i + 1] * up, lo);
        parts2(f[4 * i + 2] * up, f[4 * i + 3] * up, hi);
#pragma unroll
        for (int q = 0; q < kQParts; ++q) w[q][i] = lo[q] | hi[q] << 16;
      }
      if (r < R) {
#pragma unroll
        for (int q = 0; q < kQParts; ++q)
          *reinterpret_cast<uint4*>(sm.q + chunk_at<D>(column_of(q, r), c)) = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
      }
      if (c == 0 && r < R) sm.qscale[qn & 1][r] = p.scale_log2 * __uint_as_float(static_cast<uint32_t>(127 - s) << 23);
      fetch(r + 32 / kLanes);
    }
    fence_proxy_async();
    __syncwarp();
    mbar_arrive_elect(&sm.qfull[qn & 1]);
  }
}

// ---- warp 0: pages -----------------------------------------------------------------------
// Tiles in the order K t, K t + 1, V t, K t + 2, V t + 1, ...
template <int D>
__device__ __forceinline__ void few_load_warp(const PagedAttnParams& p, Q8Smem<D>& sm) {
  using S = Q8Smem<D>;
  const int lane = threadIdx.x & 31;
  const int box_shift = min(p.page_shift, 7);
  const int boxes = kRows >> box_shift;
  uint32_t st = 0, ph = 0, issued = 0;
  bool ok = true;
  for (uint32_t e = 0; ok; ++e) {
    const Entry en = take(p, sm, e);
    if (uniform(en.n) == 0) break;
    const int h = uniform(en.h), t0 = uniform(en.t0), t1 = uniform(en.t1), klo = uniform(en.klo), khi = uniform(en.khi);
    const int* row = p.table + static_cast<long long>(uniform(en.s)) * p.max_pages;
    // lane i holds the page of the tile's box i: its entry of the table, read three tiles ahead and checked when used
    auto page_of = [&](int t) {
      const int k = t * kRows + (lane << box_shift);
      return load_int_if(row + (k >> p.page_shift), t < t1 && lane < boxes && k < khi && k + (1 << box_shift) > klo, INT_MAX);
    };
    auto checked = [&](int id) {  // num_pages (loads zeros) for no page or one outside the pool
      if (static_cast<unsigned>(id) < static_cast<unsigned>(p.num_pages)) return id;
      if (id != INT_MAX) atomicOr(p.status, kStatusDevice);
      return p.num_pages;
    };
    auto load = [&](const CUtensorMap* map, int t, int page) {
      ok = ok && attn_wait_warp(sm, &sm.empty[st], ph ^ 1, p.status);
      if (!ok) return;
      const uint32_t dst = smem_u32(sm.kv[st]), bar = smem_u32(&sm.full[st]);
      mbar_expect_elect(&sm.full[st], S::kTileBytes);
      const int y = (t * kRows) & ((1 << p.page_shift) - 1);  // a page is whole boxes, or a box whole pages
      if (boxes == 1) {
        tma_load_4d_elect(dst, map, 0, y, h, uniform(page), bar);
      } else {
        for (int i = 0; i < boxes; i += 2) {
          const int pa = __shfl_sync(0xffffffffu, page, i), pb = __shfl_sync(0xffffffffu, page, i + 1);
          tma_load_4d_elect(dst + (i << box_shift) * D, map, 0, y, h, pa, bar);
          tma_load_4d_elect(dst + ((i + 1) << box_shift) * D, map, 0, y, h, pb, bar);
        }
      }
      ++issued;
      if (++st == S::kStages) { st = 0; ph ^= 1; }
    };
    int r0 = page_of(t0), r1 = page_of(t0 + 1), r2 = page_of(t0 + 2);
    int p0 = checked(r0), p1 = checked(r1);
    for (int a = 0; a < 2 && t0 + a < t1; ++a) load(&p.kmap, t0 + a, a == 0 ? p0 : p1);
    for (int t = t0; ok && t < t1; ++t) {
      const int r3 = page_of(t + 3);
      const int p2 = checked(r2);
      load(&p.vmap, t, p0);
      if (t + 2 < t1) load(&p.kmap, t + 2, p2);
      p0 = p1;
      p1 = p2;
      r2 = r3;
    }
  }
  // After an abort, wait (bounded) for the copies still landing before the CTA retires.
  if (!ok || ld_volatile(&sm.abort_flag)) {
    for (uint32_t b = 0; b < S::kStages && b < issued; ++b) {
      const uint32_t n = issued - 1 - b;
      attn_drain(&sm.full[n % S::kStages], (n / S::kStages) & 1);
    }
  }
}

// ---- warp 1: MMAs ------------------------------------------------------------------------

__device__ __forceinline__ uint32_t few_s_col(int side) { return side * kFewCols; }
__device__ __forceinline__ uint32_t few_o_col(int side) { return (2 + side) * kFewCols; }

template <int D>
__device__ __forceinline__ void few_mma_warp(const PagedAttnParams& p, Q8Smem<D>& sm, uint32_t tmem) {
  using S = Q8Smem<D>;
  uint32_t st = 0, ph = 0, qn = 0, pph[2] = {0, 0};
  bool ok = true;
  auto advance = [&] { if (++st == S::kStages) { st = 0; ph ^= 1; } };
  auto tile = [&] { ok = ok && attn_wait_warp(sm, &sm.full[st], ph, p.status); };
  for (uint32_t e = 0; ok; ++e, ++qn) {
    const Entry en = take(p, sm, e);
    if (uniform(en.n) == 0) break;
    const int n = uniform(en.t1 - en.t0), N = kQParts * rows_held(uniform(en.n) * p.G);
    ok = attn_wait_warp(sm, &sm.qfull[qn & 1], (qn >> 1) & 1, p.status);
    const uint64_t qdesc = rows_desc<D>(smem_u32(sm.q));
    const uint32_t idesc_kq = idesc8<false>(128, 0) | static_cast<uint32_t>(N >> 3) << 17;
    const uint32_t idesc_vp = idesc8<true>(128, 0) | static_cast<uint32_t>(N >> 3) << 17;
    auto kq = [&](int x) {
      tile();
      if (!ok) return;
      tc_fence_after();
      const uint64_t kdesc = rows_desc<D>(smem_u32(sm.kv[st]));
#pragma unroll
      for (int k = 0; k < D / 32; ++k) umma8_ss(tmem + few_s_col(x), kdesc + 2 * k, qdesc + 2 * k, idesc_kq, k > 0);
      umma_commit_elect(&sm.sfull[x]);
      umma_commit_elect(&sm.empty[st]);
      advance();
    };
    for (int j = 0; j < 2 && j < n; ++j) kq(j);
    for (int j = 0; ok && j < n; ++j) {
      const int x = j & 1;
      tile();
      ok = ok && attn_wait_warp(sm, &sm.pfull[x], pph[x], p.status);
      if (!ok) break;
      pph[x] ^= 1;
      tc_fence_after();
      const uint64_t vdesc = rows_desc<D>(smem_u32(sm.kv[st])), pdesc = rows_desc<128>(smem_u32(sm.p[x]));
#pragma unroll
      for (int k = 0; k < kRows / 32; ++k)
        umma8_ss(tmem + few_o_col(x), vdesc + k * (32 * D / 16), pdesc + 2 * k, idesc_vp, j >= 2 || k > 0);
      umma_commit_elect(&sm.empty[st]);
      if (j + 2 >= n) umma_commit_elect(&sm.ofull[x]);
      advance();
      if (j + 2 < n) {
        kq(x);
        if (j + 3 == n) umma_commit_elect(&sm.qempty);
      }
    }
    if (n <= 2) umma_commit_elect(&sm.qempty);
  }
  umma_commit_elect(&sm.done);
  attn_drain(&sm.done, 0);
}

// ---- softmax: a thread per key -------------------------------------------------------------

// As mend_v: zeroes the rows of the V tile that hold no key of the unit but lie in a page box that does.
template <int D>
__device__ __forceinline__ void few_mend_v(const PagedAttnParams& p, Q8Smem<D>& sm, const Entry& en, int j, SideState& st) {
  const int k0 = j * kRows, a = max(en.klo - k0, 0), b = min(en.khi - k0, kRows);
  if (a == 0 && b == kRows) return;
  const int n = en.t1 - en.t0, i = j - en.t0;
  const uint32_t at = st.tiles + min(2 * i + 2, 2 * n - 1);  // the V tile's place in the ring's order
  const uint32_t stage = at % Q8Smem<D>::kStages;
  st.ok = st.ok && attn_wait_warp(sm, &sm.full[stage], (at / Q8Smem<D>::kStages) & 1, p.status);
  const int box = 1 << min(p.page_shift, 7);
  auto zero = [&](int r0, int r1) {
    for (int q = r0 * (D / 16) + static_cast<int>(threadIdx.x & 127); q < r1 * (D / 16); q += 128)
      *reinterpret_cast<uint4*>(sm.kv[stage] + q * 16) = make_uint4(0, 0, 0, 0);
  };
  zero(a & ~(box - 1), a);
  if (b > 0) zero(b, min(kRows, (b + box - 1) & ~(box - 1)));
}

// 16 columns of a thread's lane, the parts of a group's rows, as the rows' sums.
__device__ __forceinline__ void load_rows(uint32_t taddr, float (&v)[kRowGroup]) {
  uint32_t u[kGroupCols];
  tmem_ld_cols<kGroupCols>(taddr, u);
#pragma unroll
  for (int r = 0; r < kRowGroup; ++r) {
    const float a = fmaf(__uint_as_float(u[kRowGroup + r]), 1.f / kRest, __uint_as_float(u[r]));
    const float b = fmaf(__uint_as_float(u[3 * kRowGroup + r]), 1.f / kRest, __uint_as_float(u[2 * kRowGroup + r]));
    v[r] = fmaf(b, 1.f / (kRest * kRest), a);
  }
}

// A cut unit's piece, side x: its rows' outputs [row][D], then their (m, l).
template <int D>
__device__ __forceinline__ Records<D> few_records(const PagedAttnParams& p, long long cta, bool first, int x) {
  constexpr size_t kBytes = kFewRows * (D * sizeof(float) + sizeof(float2));
  static_assert(kFewCtas * kBytes <= kRows * (D * sizeof(float) + sizeof(float2)), "within the workspace");
  return {p.parts + ((2 * cta + (first ? 1 : 0)) * 2 + x) * kBytes};
}
template <int D>
__device__ __forceinline__ float2* few_ml(const Records<D>& r) { return reinterpret_cast<float2*>(r.at + kFewRows * D * sizeof(float)); }

__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

// kGroups groups of rows.
template <int D, bool kFp16, int kGroups>
__device__ __forceinline__ void q8_few_rows(const PagedAttnParams& p, Q8Smem<D>& sm, uint32_t tmem, int x, const Entry& en,
                                            SideState& st) {
  constexpr int R = kGroups * kRowGroup;
  const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31, key = warp * 32 + lane;
  const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
  const uint32_t ts = tmem + lanes + few_s_col(x), to = tmem + lanes + few_o_col(x);
  const int rows = en.n * p.G;
  const int f1 = rows < R ? 0 : (en.pos0 + 1) >> 7;  // [f0, f1): every row sees every key
  const int f0 = p.window > 0 ? (max(0, en.pos0 + en.n - p.window) + 127) >> 7 : 0;
  float l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) l[r] = 0.f;
  if (key < R) sm.m[x][key] = sm.mz[x][key] = -INFINITY;
  // the key's exponents, one tile of the side ahead, and its page, two
  const int* row = p.table + static_cast<long long>(en.s) * p.max_pages;
  auto page_at = [&](int j) {
    const int k = j * kRows + key;
    return load_int_if(row + (k >> p.page_shift), j < en.t1 && k >= en.klo && k < en.khi, -1);
  };
  auto exponents_at = [&](int j, int page) {  // (K's, V's; of a zero row where there is none)
    const bool there = static_cast<unsigned>(page) < static_cast<unsigned>(p.num_pages);
    const long long at = page * p.scale_page + (en.h << p.page_shift) + ((j * kRows + key) & ((1 << p.page_shift) - 1));
    return make_uint2(load_byte_if(p.K_scale + at, there, 127u), load_byte_if(p.V_scale + at, there, 127u));
  };
  const int first = en.t0 + x;
  uint2 ex = exponents_at(first, page_at(first));
  int page = page_at(first + 2);
  // (The rows of the next entry but one come after this side has left this one: its phase cannot be missed.  A side without a
  // tile needs none.)
  if (first < en.t1) st.ok = st.ok && attn_wait_warp(sm, &sm.qfull[st.qn & 1], (st.qn >> 1) & 1, p.status);
  const float* const qscale = sm.qscale[st.qn & 1];
  group_sync(x);  // (the maxima are set)
  for (int j = first; j < en.t1; j += 2) {
    const uint2 next = exponents_at(j + 2, page);
    page = page_at(j + 4);
    st.ok = st.ok && attn_wait_warp(sm, &sm.sfull[x], st.sph, p.status);
    st.sph ^= 1;
    tc_fence_after();
    const float k2 = __uint_as_float(ex.x << 23), b = static_cast<float>(static_cast<int>(ex.y) - 127);
    const bool edge = j < f0 || j >= f1;
    // the logits of group g
    auto logits = [&](int g, float (&y)[kRowGroup]) {
      load_rows(ts + g * kGroupCols, y);
#pragma unroll
      for (int r = 0; r < kRowGroup; ++r) y[r] *= qscale[g * kRowGroup + r] * k2;
      if (edge) {
        const int k = j * kRows + key;
#pragma unroll
        for (int r = 0; r < kRowGroup; ++r) {
          const int t = en.pos0 + (g * kRowGroup + r) / p.G;
          if (g * kRowGroup + r >= rows || k > t || (p.window > 0 && k <= t - p.window)) y[r] = -INFINITY;
        }
      }
    };
    float y[kRowGroup];  // (of more groups: formed again where they are used)
    bool up = false;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      logits(g, y);
#pragma unroll
      for (int r = 0; r < kRowGroup; ++r)
        up |= y[r] > sm.m[x][g * kRowGroup + r] + kFewRaise || y[r] + b > sm.mz[x][g * kRowGroup + r] + kFewRaise;
    }
    if (group_any(x, up)) {
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        if (kGroups > 1) logits(g, y);
#pragma unroll
        for (int r = 0; r < kRowGroup; ++r) {
          const float a = warp_max(y[r]), z = warp_max(y[r] + b);
          if (lane == 0) {
            sm.red[x][0][warp][g * kRowGroup + r] = a;
            sm.red[x][1][warp][g * kRowGroup + r] = z;
          }
        }
      }
      group_sync(x);
      auto raised = [&](int i, int r) {
        const float* top = &sm.red[x][i][0][r];
        return fmaxf(fmaxf(fmaxf(top[0], top[kFewRows]), fmaxf(top[2 * kFewRows], top[3 * kFewRows])), i ? sm.mz[x][r] : sm.m[x][r]);
      };
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        float f[kRowGroup];
#pragma unroll
        for (int r = 0; r < kRowGroup; ++r) {
          const int q = g * kRowGroup + r;
          l[q] *= ex2_approx(sm.m[x][q] - finite_or_0(raised(0, q)));
          f[r] = ex2_approx(sm.mz[x][q] - finite_or_0(raised(1, q)));
        }
        if (j != first) {
          // S of this tile is complete, so is O of the side's tile before it, and the next waits for us
          uint32_t o[kGroupCols];
          tmem_ld_cols<kGroupCols>(to + g * kGroupCols, o);
#pragma unroll
          for (int c = 0; c < kGroupCols; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f[c % kRowGroup]);
          tmem_st_cols<kGroupCols>(to + g * kGroupCols, o);
        }
      }
      if (j != first) tmem_wait_st();
      float mn = 0.f, zn = 0.f;
      if (key < R) {
        mn = raised(0, key);
        zn = raised(1, key);
      }
      group_sync(x);  // (everyone has read the old ones)
      if (key < R) {
        sm.m[x][key] = mn;
        sm.mz[x][key] = zn;
      }
      group_sync(x);
    }
    // this key's byte of a column is in the column's 128
    uint8_t* const pw = sm.p[x] + (key & 15);
    const int chunk = key >> 4;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      if (kGroups > 1) logits(g, y);
#pragma unroll
      for (int r = 0; r < kRowGroup; r += 2) {
        float w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int q = g * kRowGroup + r + i;
          l[q] += ex2_approx(y[r + i] - finite_or_0(sm.m[x][q]));
          w[i] = ex2_approx(y[r + i] + b - (finite_or_0(sm.mz[x][q]) - kFewUp));
        }
        uint32_t c[kQParts];
        parts2(w[0], w[1], c);
#pragma unroll
        for (int q = 0; q < kQParts; ++q) {
          pw[chunk_at<128>(column_of(q, g * kRowGroup + r), chunk)] = static_cast<uint8_t>(c[q]);
          pw[chunk_at<128>(column_of(q, g * kRowGroup + r + 1), chunk)] = static_cast<uint8_t>(c[q] >> 8);
        }
      }
    }
    few_mend_v<D>(p, sm, en, j, st);
    fence_proxy_async();
    tc_fence_before();
    __syncwarp();
    mbar_arrive_elect(&sm.pfull[x]);
    ex = next;
  }
  // ---- the rows' output: sums over the keys, then both sides' accumulators ----
  group_sync(x);  // (the maxima's readers are done)
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float v = l[r];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0) sm.red[x][0][warp][r] = v;
  }
  group_sync(x);
  if (key < R) sm.l[x][key] = (sm.red[x][0][0][key] + sm.red[x][0][1][key]) + (sm.red[x][0][2][key] + sm.red[x][0][3][key]);
  if (first < en.t1) {  // (side 1 of a single tile has no accumulator)
    st.ok = st.ok && attn_wait_warp(sm, &sm.ofull[x], st.oph, p.status);
    st.oph ^= 1;
  }
  tc_fence_before();
  __syncwarp();
  mbar_arrive_elect(&sm.xfull);
  st.ok = st.ok && attn_wait_warp(sm, &sm.xfull, st.xph, p.status);
  tc_fence_after();
  const bool both = en.t0 + 1 < en.t1, whole = en.pieces == 1;
  // side x writes the rows r with r mod 2 = x; the thread's element is d = key
  auto emit = [&](int r, float o, float mm, float ll) {
    const int i = r / p.G, head = en.h * p.G + r - i * p.G;
    if (key < D)
      *reinterpret_cast<uint16_t*>(p.out + static_cast<long long>(en.tok0 + i) * p.out_token +
                                   static_cast<long long>(head) * p.out_head + key * 2) = static_cast<uint16_t>(pack2<kFp16>(o, 0.f));
    if (p.lse && key == r) p.lse[static_cast<long long>(en.tok0 + i) * p.H_q + head] = lse_of(mm, ll);
  };
  const Records<D> mine = few_records<D>(p, blockIdx.x, en.first == static_cast<int>(blockIdx.x), x);
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    float a[kRowGroup], c[kRowGroup];
    load_rows(tmem + lanes + few_o_col(0) + g * kGroupCols, a);
    if (both) load_rows(tmem + lanes + few_o_col(1) + g * kGroupCols, c);
#pragma unroll
    for (int r = 0; r < kRowGroup; ++r) {
      const int q = g * kRowGroup + r;
      if ((q & 1) != x || q >= rows) continue;
      const float ma = sm.m[0][q], mb = both ? sm.m[1][q] : -INFINITY, mm = fmaxf(ma, mb), base = finite_or_0(mm);
      const float ll = fmaf(sm.l[0][q], ex2_approx(ma - base), both ? sm.l[1][q] * ex2_approx(mb - base) : 0.f);
      // the accumulators are 2^kFewUp sum 2^(y + b - mz) B
      float v = 0.f;
      if (ll != 0.f) {
        v = a[r] * ex2_approx(sm.mz[0][q] - kFewUp - base);
        if (both) v = fmaf(c[r], ex2_approx(sm.mz[1][q] - kFewUp - base), v);
      }
      if (whole) {
        emit(q, v * (ll == 0.f ? 0.f : 1.f / ll), mm, ll);
      } else {
        if (key < D) __stcg(reinterpret_cast<float*>(mine.at) + q * D + key, v);
        if (key == q) __stcg(few_ml(mine) + q, make_float2(mm, ll));
      }
    }
  }
  tc_fence_before();
  __syncwarp();
  mbar_arrive_elect(&sm.xfree);
  if (!whole && arrived_last(p, sm, en, x, st.ok)) {
    // row by row, kU records in flight
    constexpr int kU = 16;
#pragma unroll 1
    for (int q = x; q < rows; q += 2) {
      float mm = -INFINITY, ll = 0.f, oo = 0.f;
#pragma unroll 1
      for (int q0 = 0; q0 < en.pieces; q0 += kU) {
        float2 z[kU];
        float o[kU];
#pragma unroll
        for (int i = 0; i < kU; ++i) {
          z[i] = make_float2(-INFINITY, 0.f);
          o[i] = 0.f;
          if (q0 + i < en.pieces) {
            const Records<D> rec = few_records<D>(p, en.first + q0 + i, q0 + i == 0, x);
            z[i] = __ldcg(few_ml(rec) + q);
            if (key < D) o[i] = __ldcg(reinterpret_cast<const float*>(rec.at) + q * D + key);
          }
        }
        float mn = mm;
#pragma unroll
        for (int i = 0; i < kU; ++i) mn = fmaxf(mn, z[i].x);
        const float bs = finite_or_0(mn), f0 = ex2_approx(mm - bs);
        ll *= f0;
        oo *= f0;
#pragma unroll
        for (int i = 0; i < kU; ++i) {
          const float f = ex2_approx(z[i].x - bs);
          ll = fmaf(z[i].y, f, ll);
          oo = fmaf(o[i], f, oo);
        }
        mm = mn;
      }
      emit(q, ll == 0.f ? 0.f : oo * (1.f / ll), mm, ll);
    }
  }
  // both sides have read both accumulators and their maxima and sums before either goes on
  st.ok = st.ok && attn_wait_warp(sm, &sm.xfree, st.xph, p.status);
  st.xph ^= 1;
  tc_fence_after();
  ++st.qn;
}

template <int D, bool kFp16>
__global__ void __launch_bounds__(kFewThreads, kFewCtas) q8_few_kernel(const __grid_constant__ PagedAttnParams p) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  using S = Q8Smem<D>;
  if (smem_u32(smem_raw) & 1023u) {  // the swizzles need 1024-byte aligned buffers
    if (threadIdx.x == 0) atomicOr(p.status, kStatusDevice);
    return;
  }
  S& sm = *reinterpret_cast<S*>(smem_raw);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.sfull[i], 1);
      mbar_init(&sm.pfull[i], 4);
      mbar_init(&sm.ofull[i], 1);
    }
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], 1);
    }
    for (int i = 0; i < kEntries; ++i) {
      mbar_init(&sm.efull[i], 1);
      mbar_init(&sm.eempty[i], 11);  // the load, MMA and query warps and eight softmax warps
    }
    for (int i = 0; i < 2; ++i) mbar_init(&sm.qfull[i], 1);
    mbar_init(&sm.qempty, 1);
    mbar_init(&sm.xfull, 8);
    mbar_init(&sm.xfree, 8);
    mbar_init(&sm.done, 1);
    sm.abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async();
  }
  if (threadIdx.x == 64) {
    for (const CUtensorMap* m : {&p.kmap, &p.vmap})
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_slot, 4 * kFewCols);
    tmem_relinquish();
  }
  pdl_wait();
  pdl_trigger();
  Share sh = {};
  if (p.segs > 32) sh = share_of<kFewMode>(p, sm, true);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_slot;
  if (warp == 0) few_load_warp<D>(p, sm);
  if (warp == 1) few_mma_warp<D>(p, sm, tmem);
  if (warp == 2) deal<kFewMode>(p, sm, sh, true);
  if (warp == 3) split_queries<D, kFp16>(p, sm);
  if (warp >= 4) {
    const int x = (warp - 4) >> 2;
    SideState st;
    for (uint32_t e = 0;; ++e) {
      const Entry en = take(p, sm, e);
      if (group_any(x, en.n == 0)) break;  // no more, or a warp's wait for the entry ran out
      const int rows = en.n * p.G;
      if (rows <= 4) q8_few_rows<D, kFp16, 1>(p, sm, tmem, x, en, st);
      else if (rows <= 8) q8_few_rows<D, kFp16, 2>(p, sm, tmem, x, en, st);
      else q8_few_rows<D, kFp16, 4>(p, sm, tmem, x, en, st);
      st.tiles += 2 * (en.t1 - en.t0);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 4 * kFewCols);
  }
}

AttnFn few_fn(int d, bool fp16) {
  if (d == 64) return fp16 ? q8_few_kernel<64, true> : q8_few_kernel<64, false>;
  return fp16 ? q8_few_kernel<128, true> : q8_few_kernel<128, false>;
}

// The maps of a cache's pages of codes.
bool q8_page_maps(const kvev_paged_q8_cache* cache, CUtensorMapSwizzle swizzle, PagedAttnParams* p) {
  auto encode = encode_fn();
  if (!encode) return false;
  const cuuint64_t dims[4] = {static_cast<cuuint64_t>(cache->d), static_cast<cuuint64_t>(cache->page_size),
                              static_cast<cuuint64_t>(cache->H_kv), static_cast<cuuint64_t>(cache->num_pages)};
  const cuuint64_t strides[3] = {static_cast<cuuint64_t>(cache->token_stride), static_cast<cuuint64_t>(cache->head_stride),
                                 static_cast<cuuint64_t>(cache->page_stride)};
  const cuuint32_t box[4] = {static_cast<cuuint32_t>(cache->d), static_cast<cuuint32_t>(cache->page_size < kRows ? cache->page_size : kRows), 1, 1};
  const cuuint32_t ones[4] = {1, 1, 1, 1};
  for (int i = 0; i < 2; ++i)
    if (encode(i ? &p->vmap : &p->kmap, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, i ? cache->V : cache->K, dims, strides, box, ones,
               CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return false;
  return true;
}

// The requests of few rows; p but for the maps of the pages.
int few_launch(PagedAttnParams p, const kvev_paged_q8_cache* cache, cudaStream_t stream) {
  const int d = cache->d;
  const bool fp16 = cache->dtype == KVEV_FP16;
  const size_t smem = d == 64 ? sizeof(Q8Smem<64>) : sizeof(Q8Smem<128>);
  int grid = 0;
  const AttnFn fn = few_fn(d, fp16);
  static AttnReady ready[4];
  const int rc = ready_kernel(ready[(d == 64 ? 0 : 2) + (fp16 ? 1 : 0)], fn, smem, kFewThreads, 0, &grid);
  if (rc != KVEV_OK) return rc;
  if (!q8_page_maps(cache, d == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, &p)) return KVEV_ECUDA;
  static_assert(2 * kFewCtas * kMaxCtas * sizeof(int) <= KVEV_PAGED_SYNC_BYTES, "arrival counts");
  return launch_overlapped(fn, p, kFewCtas * grid, kFewThreads, smem, stream) == cudaSuccess ? KVEV_OK : KVEV_ECUDA;
}

}  // namespace
}  // namespace kvev
