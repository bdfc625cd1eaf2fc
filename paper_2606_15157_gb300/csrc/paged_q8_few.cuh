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
// its key's weights, O^T += B^T w^T with the codes of V as the operand whose key index runs slowest; the schedule is the
// same, and so are pieces and their merge.  A CTA has one softmax warpgroup and takes its units one after another; what hides a
// tile's chain of latencies (scores, weights, products) and a unit's start and end is the other CTAs of the SM.
//
// Bounds and measurements (one GB300, 32 query and 8 KV heads of 128, pages of 16, tokens first): HBM, and each unit's start
// and end.  16 generations at 16K (pages of 64) 88 us, 6.1 TB/s of codes; 64 at 4K 93 us, 5.8 TB/s; 64 ragged ones to 8K of 64-element
// heads 57 us, 4.7 TB/s; each further 4K of 64 generations at HBM's rate.  One at 4K 13.4 us: schedule and first loads 4, two
// tiles of a CTA 2, records and merge 3, the launch 2.  16 heads to a KV head: 64 at 4K 135 us, the threads' 64 codes a tile.
// Measured on the way (16 at 16K and 64 ragged): two sides of a CTA, each with every other tile, as the 16-bit kernel has them
// 95 and 97 us; scores of a side's next tile formed early 97 and 102; two such CTAs an SM 100 and 80; one side a CTA and three CTAs
// 95 and 64 (100 and 107 before the KV heads were in step); without the other kernel's launch 88 and 57.
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
// CTAs of an SM, by the most rows of a unit (4, 8 or 16): what shared memory and registers allow.
constexpr int few_ctas(int M) { return M <= 8 ? 3 : 2; }

template <int D, int M>
struct Q8Smem {
  // rows of 64 or 128 bytes: as for 16-bit rows of 64 elements
  static constexpr bool kHeadsOuter = true;
  static constexpr int kTileBytes = kRows * D, kCols = kQParts * M;
  static constexpr int kStages = (M <= 4 ? 4 : M == 8 ? 3 : 5) * (D == 128 ? 1 : 2);
  uint8_t kv[kStages][kTileBytes];
  uint8_t p[2][kCols * kRows];  // weights of every other tile [column][128 keys]
  uint8_t q[kCols * D];         // [column][D]
  float qscale[2][M];           // of an entry's rows: log2(e) scale over their power of two
  float m[M], mz[M];            // the rows' maxima, the weights' maxima
  Entry ring[kEntries];
  uint64_t qfull[2], qempty, full[kStages], empty[kStages];  // (qfull: of every other entry)
  uint64_t sfull, pfull;
  // the output holds another tile, its last.  (Told apart: whoever waits for a tile to be in knows that the one before it
  // is, as a phase's parity tells no more; of the last two nobody waits for the first.)
  uint64_t odone, ofull;
  uint64_t efull[kEntries], eempty[kEntries], done;
  long long carry, start;
  union {
    float red[2][4][M];  // the warps' maxima, or sums, of the rows
    long long scan[Split<kQ8 | kFewOnly>::kThreads / 32];
    float2 ml[128];      // (m, l) of pieces
  };
  int last[1];
  int abort_flag;
  uint32_t tmem_slot;
};
// (1 KB of an SM's 228 goes to each CTA beside what it asks for)
template <int M>
constexpr bool fits() {
  return few_ctas(M) * (sizeof(Q8Smem<64, M>) + 1024) <= 228 * 1024 && few_ctas(M) * (sizeof(Q8Smem<128, M>) + 1024) <= 228 * 1024;
}
static_assert(fits<4>() && fits<8>() && fits<16>(), "shared memory of an SM");

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
// K contiguous, or rows along K with M contiguous.  (Rows of 64 bytes as the latter are 64 of the 128 lanes; the next 64 would start
// a leading-dimension offset further on, which is 0: they are the same again, and nothing reads them.)
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
__host__ __device__ inline int rows_held(int rows) { return rows <= 4 ? 4 : rows <= 8 ? 8 : 16; }
// The column of part q of row r.
__device__ __forceinline__ int column_of(int q, int r) { return r / kRowGroup * kGroupCols + q * kRowGroup + r % kRowGroup; }

// ---- warp 3: the rows of q in parts --------------------------------------------------------

template <int D, bool kFp16, int M>
__device__ __forceinline__ void split_queries(const PagedAttnParams& p, Q8Smem<D, M>& sm) {
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
template <int D, int M>
__device__ __forceinline__ void few_load_warp(const PagedAttnParams& p, Q8Smem<D, M>& sm) {
  using S = Q8Smem<D, M>;
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

// Tensor memory: scores, then the output.
template <int D, int M>
__device__ __forceinline__ void few_mma_warp(const PagedAttnParams& p, Q8Smem<D, M>& sm, uint32_t tmem) {
  using S = Q8Smem<D, M>;
  uint32_t st = 0, ph = 0, qn = 0, pph = 0;
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
    auto kq = [&](int j) {
      tile();
      if (!ok) return;
      tc_fence_after();
      const uint64_t kdesc = rows_desc<D>(smem_u32(sm.kv[st]));
#pragma unroll
      for (int k = 0; k < D / 32; ++k) umma8_ss(tmem, kdesc + 2 * k, qdesc + 2 * k, idesc_kq, k > 0);
      umma_commit_elect(&sm.sfull);
      umma_commit_elect(&sm.empty[st]);
      if (j == n - 1) umma_commit_elect(&sm.qempty);
      advance();
    };
    kq(0);
    for (int j = 0; ok && j < n; ++j) {
      // the next tile's scores go first: the softmax waits for them, and for the output only to raise a maximum
      ok = ok && attn_wait_warp(sm, &sm.pfull, pph, p.status);
      if (!ok) break;
      pph ^= 1;
      if (j + 1 < n) kq(j + 1);
      tile();
      if (!ok) break;
      tc_fence_after();
      const uint64_t vdesc = rows_desc<D>(smem_u32(sm.kv[st])), pdesc = rows_desc<128>(smem_u32(sm.p[j & 1]));
#pragma unroll
      for (int k = 0; k < kRows / 32; ++k)
        umma8_ss(tmem + S::kCols, vdesc + k * (32 * D / 16), pdesc + 2 * k, idesc_vp, j > 0 || k > 0);
      umma_commit_elect(&sm.empty[st]);
      umma_commit_elect(j + 1 < n ? &sm.odone : &sm.ofull);
      advance();
    }
  }
  umma_commit_elect(&sm.done);
  attn_drain(&sm.done, 0);
}

// ---- softmax: a thread per key -------------------------------------------------------------

// As mend_v: zeroes the rows of the V tile that hold no key of the unit but lie in a page box that does.
template <int D, int M>
__device__ __forceinline__ void few_mend_v(const PagedAttnParams& p, Q8Smem<D, M>& sm, const Entry& en, int j, SideState& st) {
  using S = Q8Smem<D, M>;
  const int k0 = j * kRows, a = max(en.klo - k0, 0), b = min(en.khi - k0, kRows);
  if (a == 0 && b == kRows) return;
  const int n = en.t1 - en.t0, i = j - en.t0;
  const uint32_t at = st.tiles + min(2 * i + 2, 2 * n - 1);  // the V tile's place in the ring's order
  const uint32_t stage = at % S::kStages;
  st.ok = st.ok && attn_wait_warp(sm, &sm.full[stage], (at / S::kStages) & 1, p.status);
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

// A cut unit's piece: its rows' outputs [row][D], then their (m, l).
template <int D>
__device__ __forceinline__ Records<D> few_record(const PagedAttnParams& p, long long cta, bool first) {
  constexpr size_t kBytes = kFewRows * (D * sizeof(float) + sizeof(float2));
  static_assert(2 * 3 * kBytes <= 4 * kRows * (D * sizeof(float) + sizeof(float2)), "within the workspace");
  return {p.parts + (2 * cta + (first ? 1 : 0)) * kBytes};
}
template <int D>
__device__ __forceinline__ float2* few_ml(const Records<D>& r) { return reinterpret_cast<float2*>(r.at + kFewRows * D * sizeof(float)); }

__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

// kGroups groups of rows.
template <int D, bool kFp16, int M, int kGroups>
__device__ __forceinline__ void q8_few_rows(const PagedAttnParams& p, Q8Smem<D, M>& sm, uint32_t tmem, const Entry& en, SideState& st,
                                            uint32_t& done) {
  constexpr int R = kGroups * kRowGroup;
  const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31, key = warp * 32 + lane;
  const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
  const uint32_t ts = tmem + lanes, to = ts + Q8Smem<D, M>::kCols;
  const int rows = en.n * p.G;
  const int f1 = rows < R ? 0 : (en.pos0 + 1) >> 7;  // [f0, f1): every row sees every key
  const int f0 = p.window > 0 ? (max(0, en.pos0 + en.n - p.window) + 127) >> 7 : 0;
  float l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) l[r] = 0.f;
  if (key < R) sm.m[key] = sm.mz[key] = -INFINITY;
  // the key's exponents, one tile ahead, and its page, two
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
  const int first = en.t0;
  uint2 ex = exponents_at(first, page_at(first));
  int page = page_at(first + 1);
  // (The rows of the next entry but one come after this one's are done with: a phase cannot be missed.)
  st.ok = st.ok && attn_wait_warp(sm, &sm.qfull[st.qn & 1], (st.qn >> 1) & 1, p.status);
  const float* const qscale = sm.qscale[st.qn & 1];
  group_sync(0);  // (the maxima are set)
  for (int j = first; j < en.t1; ++j) {
    const uint2 next = exponents_at(j + 1, page);
    page = page_at(j + 2);
    st.ok = st.ok && attn_wait_warp(sm, &sm.sfull, st.sph, p.status);
    st.sph ^= 1;
    tc_fence_after();
    const float k2 = __uint_as_float(ex.x << 23), b = static_cast<float>(static_cast<int>(ex.y) - 127);
    const bool edge = j < f0 || j >= f1;
    float y[R];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      float v[kRowGroup];
      load_rows(ts + g * kGroupCols, v);
#pragma unroll
      for (int r = 0; r < kRowGroup; ++r) y[g * kRowGroup + r] = v[r] * (qscale[g * kRowGroup + r] * k2);
    }
    if (edge) {
      const int k = j * kRows + key;
      int t = en.pos0, i = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r >= rows || k > t || (p.window > 0 && k <= t - p.window)) y[r] = -INFINITY;
        if (++i == p.G) { i = 0; ++t; }
      }
    }
    bool up = false;
#pragma unroll
    for (int r = 0; r < R; ++r) up |= y[r] > sm.m[r] + kFewRaise || y[r] + b > sm.mz[r] + kFewRaise;
    if (group_any(0, up)) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float a = warp_max(y[r]), z = warp_max(y[r] + b);
        if (lane == 0) {
          sm.red[0][warp][r] = a;
          sm.red[1][warp][r] = z;
        }
      }
      group_sync(0);
      auto raised = [&](int i, int r) {
        const float* top = &sm.red[i][0][r];
        return fmaxf(fmaxf(fmaxf(top[0], top[M]), fmaxf(top[2 * M], top[3 * M])), i ? sm.mz[r] : sm.m[r]);
      };
      if (j != first) {  // the output holds the tile before this one (the one before that since this one's scores were formed)
        st.ok = st.ok && attn_wait_warp(sm, &sm.odone, (done + 1) & 1, p.status);
        tc_fence_after();
      }
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        float f[kRowGroup];
#pragma unroll
        for (int r = 0; r < kRowGroup; ++r) {
          const int q = g * kRowGroup + r;
          l[q] *= ex2_approx(sm.m[q] - finite_or_0(raised(0, q)));
          f[r] = ex2_approx(sm.mz[q] - finite_or_0(raised(1, q)));
        }
        if (j != first) {
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
      group_sync(0);  // (everyone has read the old ones)
      if (key < R) {
        sm.m[key] = mn;
        sm.mz[key] = zn;
      }
      group_sync(0);
    }
    // this key's byte of a column is in the column's 128
    uint8_t* const pw = sm.p[(j - first) & 1] + (key & 15);
    const int chunk = key >> 4;
#pragma unroll
    for (int r = 0; r < R; r += 2) {
      float w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        l[r + i] += ex2_approx(y[r + i] - finite_or_0(sm.m[r + i]));
        w[i] = ex2_approx(y[r + i] + b - (finite_or_0(sm.mz[r + i]) - kFewUp));
      }
      uint32_t c[kQParts];
      parts2(w[0], w[1], c);
#pragma unroll
      for (int q = 0; q < kQParts; ++q) {
        pw[chunk_at<128>(column_of(q, r), chunk)] = static_cast<uint8_t>(c[q]);
        pw[chunk_at<128>(column_of(q, r + 1), chunk)] = static_cast<uint8_t>(c[q] >> 8);
      }
    }
    few_mend_v(p, sm, en, j, st);
    fence_proxy_async();
    tc_fence_before();
    __syncwarp();
    mbar_arrive_elect(&sm.pfull);
    if (j + 1 < en.t1) ++done;
    ex = next;
  }
  // ---- the rows' output ----
  group_sync(0);  // (the maxima's readers are done)
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float v = l[r];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0) sm.red[0][warp][r] = v;
  }
  st.ok = st.ok && attn_wait_warp(sm, &sm.ofull, st.oph, p.status);
  st.oph ^= 1;
  group_sync(0);
  tc_fence_after();
  const bool whole = en.pieces == 1;
  const int i0 = en.h * p.G;
  // row r's element d = key
  auto emit = [&](int r, float o, float mm, float ll) {
    const int i = r < p.G ? 0 : r / p.G;
    const long long tok = en.tok0 + i, head = i0 + r - i * p.G;
    if (key < D) *reinterpret_cast<uint16_t*>(p.out + tok * p.out_token + head * p.out_head + key * 2) = static_cast<uint16_t>(pack2<kFp16>(o, 0.f));
    if (p.lse && key == r) p.lse[tok * p.H_q + head] = lse_of(mm, ll);
  };
  const Records<D> mine = few_record<D>(p, blockIdx.x, en.first == static_cast<int>(blockIdx.x));
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    float a[kRowGroup];
    load_rows(to + g * kGroupCols, a);
#pragma unroll 1
    for (int r = 0; r < kRowGroup; ++r) {
      const int q = g * kRowGroup + r;
      if (q >= rows) break;
      const float* s = &sm.red[0][0][q];
      const float mm = sm.m[q], ll = (s[0] + s[M]) + (s[2 * M] + s[3 * M]);
      // the accumulators are 2^kFewUp sum 2^(y + b - mz) B
      const float v = ll == 0.f ? 0.f : (r == 0 ? a[0] : r == 1 ? a[1] : r == 2 ? a[2] : a[3]) * ex2_approx(sm.mz[q] - kFewUp - finite_or_0(mm));
      if (whole) {
        emit(q, v * (ll == 0.f ? 0.f : 1.f / ll), mm, ll);
      } else {
        if (key < D) __stcg(reinterpret_cast<float*>(mine.at) + q * D + key, v);
        if (key == q) __stcg(few_ml(mine) + q, make_float2(mm, ll));
      }
    }
  }
  tc_fence_before();
  if (!whole && arrived_last(p, sm, en, 0, st.ok)) {
    // a group's pieces in rounds of 32: their maxima and sums by a thread each, then the outputs, kU pieces of all rows in flight
    constexpr int kRound = 32, kU = 8;
#pragma unroll 1
    for (int g = 0; g < rows; g += kRowGroup) {
      float mm[kRowGroup], ll[kRowGroup], oo[kRowGroup];
#pragma unroll
      for (int r = 0; r < kRowGroup; ++r) { mm[r] = -INFINITY; ll[r] = oo[r] = 0.f; }
#pragma unroll 1
      for (int c = 0; c < en.pieces; c += kRound) {
        const int n = min(kRound, en.pieces - c);
        float o[kU][kRowGroup];
        auto fetch = [&](int k) {
#pragma unroll
          for (int i = 0; i < kU; ++i) {
            const float* at = reinterpret_cast<const float*>(few_record<D>(p, en.first + c + k + i, c + k + i == 0).at) + g * D + key;
#pragma unroll
            for (int r = 0; r < kRowGroup; ++r) o[i][r] = k + i < n && g + r < rows && key < D ? __ldcg(at + r * D) : 0.f;
          }
        };
        fetch(0);
        const int pr = key / kRowGroup, q = g + key % kRowGroup;
        const float2 mine2 = pr < n && q < rows ? __ldcg(few_ml(few_record<D>(p, en.first + c + pr, c + pr == 0)) + q) : make_float2(-INFINITY, 0.f);
        group_sync(0);  // (the last round's readers are done)
        sm.ml[key] = mine2;
        group_sync(0);
        float bs[kRowGroup];
#pragma unroll
        for (int r = 0; r < kRowGroup; ++r) {
          float mn = mm[r];
#pragma unroll 8
          for (int i = 0; i < n; ++i) mn = fmaxf(mn, sm.ml[i * kRowGroup + r].x);
          bs[r] = finite_or_0(mn);
          const float f = ex2_approx(mm[r] - bs[r]);
          ll[r] *= f;
          oo[r] *= f;
          mm[r] = mn;
        }
#pragma unroll 1
        for (int k = 0; k < n; k += kU) {
#pragma unroll
          for (int i = 0; i < kU; ++i) {
            if (k + i >= n) break;
#pragma unroll
            for (int r = 0; r < kRowGroup; ++r) {
              const float2 z = sm.ml[(k + i) * kRowGroup + r];
              const float f = ex2_approx(z.x - bs[r]);
              ll[r] = fmaf(z.y, f, ll[r]);
              oo[r] = fmaf(o[i][r], f, oo[r]);
            }
          }
          if (k + kU < n) fetch(k + kU);
        }
      }
#pragma unroll
      for (int r = 0; r < kRowGroup; ++r)
        if (g + r < rows) emit(g + r, ll[r] == 0.f ? 0.f : oo[r] * (1.f / ll[r]), mm[r], ll[r]);
    }
  }
  group_sync(0);  // (maxima and sums have been read)
  ++st.qn;
}

template <int D, bool kFp16, int M>
__global__ void __launch_bounds__(kFewThreads, few_ctas(M)) q8_few_kernel(const __grid_constant__ PagedAttnParams p) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  using S = Q8Smem<D, M>;
  constexpr int kTmem = 2 * S::kCols < 32 ? 32 : 2 * S::kCols;
  if (smem_u32(smem_raw) & 1023u) {  // the swizzles need 1024-byte aligned buffers
    if (threadIdx.x == 0) atomicOr(p.status, kStatusDevice);
    return;
  }
  S& sm = *reinterpret_cast<S*>(smem_raw);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
  if (p.look) {  // (chunks alone leave nothing to do here; what is out of range is said by the other kernel, which is then launched too)
    pdl_wait();
    bool some = false;
    for (int s = threadIdx.x; s < p.B; s += kFewThreads) {
      const int n = p.cu[s + 1] - p.cu[s];
      some |= n > 0 && n <= p.most;
    }
    if (!__syncthreads_or(some)) return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], 1);
    }
    for (int i = 0; i < kEntries; ++i) {
      mbar_init(&sm.efull[i], 1);
      mbar_init(&sm.eempty[i], 7);  // the load, MMA and query warps and four softmax warps
    }
    for (int i = 0; i < 2; ++i) mbar_init(&sm.qfull[i], 1);
    mbar_init(&sm.qempty, 1);
    mbar_init(&sm.sfull, 1);
    mbar_init(&sm.pfull, 4);
    mbar_init(&sm.odone, 1);
    mbar_init(&sm.ofull, 1);
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
    tmem_alloc(&sm.tmem_slot, kTmem);
    tmem_relinquish();
  }
  pdl_wait();
  pdl_trigger();
  Share sh = {};
  if (p.segs > kPlannedByWarp) sh = share_of<kFewMode>(p, sm);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_slot;
  if (warp == 0) few_load_warp(p, sm);
  if (warp == 1) few_mma_warp(p, sm, tmem);
  if (warp == 2) deal<kFewMode>(p, sm, sh);
  if (warp == 3) split_queries<D, kFp16>(p, sm);
  if (warp >= 4) {
    SideState st;
    uint32_t done = 0;  // tiles but the last ones that have been handed over
    for (uint32_t e = 0;; ++e) {
      const Entry en = take(p, sm, e);
      if (group_any(0, en.n == 0)) break;  // no more, or a warp's wait for the entry ran out
      const int rows = en.n * p.G;
      if (M == 4 || rows <= 4) q8_few_rows<D, kFp16, M, 1>(p, sm, tmem, en, st, done);
      else if (M == 8 || rows <= 8) q8_few_rows<D, kFp16, M, M >= 8 ? 2 : 1>(p, sm, tmem, en, st, done);
      else q8_few_rows<D, kFp16, M, M / kRowGroup>(p, sm, tmem, en, st, done);
      st.tiles += 2 * (en.t1 - en.t0);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmem);
  }
}

struct FewKernel {
  AttnFn fn;
  size_t smem;
  AttnReady* ready;
};
template <int D, bool kFp16, int M>
FewKernel few_kernel() {
  static AttnReady ready;
  return {q8_few_kernel<D, kFp16, M>, sizeof(Q8Smem<D, M>), &ready};
}
template <int M>
FewKernel few_kernel(int d, bool fp16) {
  if (d == 64) return fp16 ? few_kernel<64, true, M>() : few_kernel<64, false, M>();
  return fp16 ? few_kernel<128, true, M>() : few_kernel<128, false, M>();
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

// Most rows of a unit: those of as many tokens as the batch has to a request, up to 16, as three CTAs of up to 8
// rows fit an SM and two of 16.  (16 requests of two tokens at 8K 66 us, in units of 16 rows 90.  A request of few rows that has more
// than others of its batch is cut into up to four units.)
int few_rows_of(int G, int B, int T) {
  const int tokens = (T - 1) / B + 1;
  return G > kFewRows || tokens > kFewRows / G ? kFewRows : rows_held(G * tokens);
}

// The requests of few rows; p but for the maps of the pages.
int few_launch(PagedAttnParams p, const kvev_paged_q8_cache* cache, int M, cudaStream_t stream) {
  const int d = cache->d;
  const bool fp16 = cache->dtype == KVEV_FP16;
  const FewKernel k = M == 4 ? few_kernel<4>(d, fp16) : M == 8 ? few_kernel<8>(d, fp16) : few_kernel<16>(d, fp16);
  int grid = 0;
  const int rc = ready_kernel(*k.ready, k.fn, k.smem, kFewThreads, 0, &grid);
  if (rc != KVEV_OK) return rc;
  if (!q8_page_maps(cache, d == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, &p)) return KVEV_ECUDA;
  static_assert(2 * few_ctas(4) * kMaxCtas * sizeof(int) <= KVEV_PAGED_SYNC_BYTES, "arrival counts");
  return launch_overlapped(k.fn, p, few_ctas(M) * grid, kFewThreads, k.smem, stream) == cudaSuccess ? KVEV_OK : KVEV_ECUDA;
}

}  // namespace
}  // namespace kvev
