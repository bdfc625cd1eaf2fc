// paged_attn.cu -- causal attention of new tokens over paged caches.
//
// A row r (one query head of one new token, at position t) needs
//   m = max_k x_k,  l = sum_k exp2(x_k - m),  o = sum_k exp2(x_k - m) V[k] / l,
// x_k = log2(e) scale q.K[k] over its keys k, and lse = ln 2 (m + log2 l).  All
// of it comes from one pass over the keys in tiles of 128, with the row's m and
// l kept in registers and o in tensor memory.
//
// Work.  The G query heads of a KV head and neighbouring tokens share K and V, so
// their rows make up the 128 rows of a tensor-core tile: P = 128 / G tokens x G
// heads.  A unit is up to two such tiles (2 P tokens of a request and KV head)
// against its key tiles; a CTA runs two "sides", each with its own scores, output
// accumulator and softmax warpgroup, so that one side's softmax runs while the tensor
// core works for the other:
//   - full unit (more than P tokens): side x holds the x-th tile of rows, and
//     both take every key tile;
//   - paired unit (17 rows to P tokens): both sides hold the same rows and
//     take the key tiles in turn, and are merged;
//   - few rows (up to 16: single tokens): the same with the products transposed, keys on the
//     lanes, so that a thread per key forms the weights of all rows.  (In rows of
//     lanes, 4 lanes of 128 had work, one after another: 64 generations at 4K
//     167 us with pages of 64, and 163 so.)
// All units' key tiles are laid end to end and cut into equal shares, one per CTA, so that
// any mix of lengths keeps every SM busy to the end and a long context is split
// where there are few rows.  The pieces of a unit that was cut leave (m, l, o) records in the
// workspace; the piece that arrives last merges them in order, so the result does
// not depend on which that is.
//
// Roles (384 threads): warp 0 loads Q tiles and page boxes by TMA, warp 1 issues the
// MMAs, warp 2 deals the entries (pieces of units) to the others through a ring, warps 4-7
// and 8-11 are the sides' softmax warpgroups.  S = Q K^T is read from tensor memory
// into registers, and the weights go back into the same columns as the A operand of
// O += P V (few rows: to shared memory as the B operand of O^T += V^T P^T).
//
// Bounds and measurements (one GB300, 32 query and 8 KV heads of 128, pages of 16):
//   - generations: HBM.  64 at 4K 160 us, 6.7 TB/s; 16 at 16K 158 us, 6.8 TB/s.  One at 4K
//     10.3 us: the dependent steps of one pass (schedule 2 us, first tiles 1.5, products
//     and softmax 2, records and merge 2), the launch 2.
//   - chunks: a side's softmax and the two products after it, which wait for one another
//     (1,640 and 1,220 cycles a tile, the tensor core's own work 1,024 of the sides' 2,860);
//     tensor pipe active 70 %.  Four chunks of 1,200 tokens over 9,000 408 us, 1,620
//     TFLOP/s; the last 4K of a 32K prompt 1.20 ms, 1,722 (1.40 ms under the power cap, the
//     clock at 1.64 of 2.07 GHz).  An 8K prompt 350-385 us: 1,024 units whose start
//     and end cost 3 tiles.
// Measured against it: MMAs issued by a thread per side, whose products interleave, 664 us
// for 541; by one thread for both 586; four softmax warpgroups of 64 columns each (96
// registers a thread) 488 us for 441.
#include <atomic>
#include <climits>
#include <cmath>

#include "paged.cuh"

namespace kvev {
namespace {

constexpr int kAttnThreads = 384;
constexpr int kRegsAttnControl = 56, kRegsAttnSoftmax = 224;
constexpr int kRegsAttnNeeded = 128 * kRegsAttnControl + 256 * kRegsAttnSoftmax;
constexpr int kMaxCtas = 152;
constexpr int kEntries = 4;         // ring of dealt entries
enum Kind : int { kFew = 0, kPaired = 1, kFull = 2 };
constexpr int kFewRows = 16;
// What the shares are cut by: the cost of a key tile, and of a unit's start and end.  Beside
// chunks a generation's tile takes 0.5 to 0.9 of a chunk's, by how many others load.  Us of
// 28 generations and 4 chunks with a window, without one, 60 and 2, an 8K prompt, with
// tiles of full and other units and their ends at
//   5, 3; 16, 8     285  690  207  358        5, 3; 20, 10    285  692  206  384
//   5, 2.5; 16, 5   283  745  190  365        5, 2; 16, 4     343  885  196  359
__host__ __device__ constexpr int tile_cost(int kind) { return kind == kFull ? 5 : 3; }
__host__ __device__ constexpr int unit_cost(int kind) { return kind == kFull ? 16 : 8; }
// Least cost of a share (a tile's or more: no piece of a cut unit is empty).  Records of
// more than a few rows are up to 64 KB a side and piece, and one CTA merges them: a
// chunk of 32 tokens over 4K 25.4 us with shares from 5 on, 21.9 from 20, 29 from 48.
// (Batches of over 32 requests have larger shares anyway.)
constexpr int kMinShare = 5, kMinShareRows = 20;
constexpr int kRows = 128;          // rows of a side
constexpr int kParts = 2;           // halves of a tile's weights, which the second product takes as they come
                                    // (whole: 457 us for 449, four chunks of 1,200 over 9,000)
constexpr float kRaise = 8.f;       // a row's maximum is raised when a tile's is this much (log2) above it
constexpr uint64_t kAttnWaitNs = 2000000000ull;

struct PagedAttnParams {
  CUtensorMap qmap;   // {d, H_q, T}, box {64, G, P}
  CUtensorMap qmap1;  // the same, box {64, G, 1}
  CUtensorMap kmap;   // {d, page rows, H_kv, pages}, box {64, min(page, 128), 1, 1}
  CUtensorMap vmap;
  uint8_t* out;
  float* lse;
  long long out_token, out_head;  // strides in bytes
  const int *cu, *kv_lens, *table;
  int B, T, H_q, H_kv, G, P, page_shift, num_pages, max_pages, window;
  float scale_log2;
  int* status;
  int* sync;       // [2 kMaxCtas] pieces arrived of the unit whose first piece is the CTA's, per side
  uint8_t* parts;  // [2 kMaxCtas][2] records
};

// One piece of a unit.
struct Entry {
  int tok0, n, pos0, h;            // first token, tokens (0: no more entries), the first token's position, KV head
  int s, t0, t1, klo;              // request, key tiles [t0, t1), first key any row sees
  int khi, kind, pieces, first;    // end of the keys, kind of unit, pieces of the unit and the first one's CTA
};

template <int D>
struct AttnSmem {
  static constexpr int kTileBytes = kRows * D * 2;
  // Units lie request by request, head by head; with 64-element heads head by head, request by request: the
  // heads of the same tokens, 128 bytes each next to one another in tokens-first pages, of which L2 fetches
  // 256, are then read by different CTAs at about the same time.  Pages with heads first and chunks gain nothing
  // by it and lose nothing, so the head's size alone decides.  Us in the first order and in the other, 32 query
  // and 8 KV heads of 64, pages of 16:
  //                             tokens first     heads first
  //   64 generations at 4K       150.1  105.9     90.3   90.2
  //   16 at 16K                  133.6  108.7     90.6   89.4
  //   4 chunks of 1,200/9,000    318.6  317.5    318.2  317.2
  //   an 8K prompt               278.9  278.3    278.9  278.2
  // 128-element heads stay in the first: generations the same within 1 %, four chunks of 1,200 over 9,000
  // 409 us, 421 in the other.
  static constexpr bool kHeadsOuter = D == 64;
  static constexpr int kStages = D == 128 ? 5 : 10;
  // (with 64-element rows the transposed products also read the tile's size of
  // bytes after a V tile, for lanes that nothing reads: the Q tiles, after the last)
  uint8_t kv[kStages][kTileBytes];
  uint8_t q[2][kTileBytes];
  float2 ml[2][kRows];   // the sides' (m, l) of the rows they share
  Entry ring[kEntries];
  uint64_t qfull[2], qempty[2], full[kStages], empty[kStages];
  uint64_t sfull[2], pfull[2][kParts], ofull[2];
  uint64_t efull[kEntries], eempty[kEntries];
  uint64_t xfull, xfree;             // rows that both sides share: their (m, l) are there; their O is done with
  uint64_t done;
  long long carry, start;
  union {
    float red[2][4][kFewRows];  // a side's warps' maxima or sums of a few rows
    long long scan[kAttnThreads / 32];  // the schedule's sums, at the start
  };
  int last[2];
  int abort_flag;
  uint32_t tmem_slot;
};
static_assert(sizeof(AttnSmem<64>) <= 227 * 1024 && sizeof(AttnSmem<128>) <= 227 * 1024, "shared memory of a CTA");

// ---- waits, bounded -------------------------------------------------------------

template <class S>
__device__ __forceinline__ bool attn_wait(S& sm, uint64_t* bar, uint32_t parity, int* status) {
  const uint64_t t0 = globaltimer_ns();
  while (!mbar_try_wait_sleep(bar, parity, 20000)) {
    if (ld_volatile(&sm.abort_flag)) return false;
    if (globaltimer_ns() - t0 > kAttnWaitNs) {
      atomicExch(&sm.abort_flag, 1);
      atomicOr(status, kStatusTimeout);
      return false;
    }
  }
  return true;
}

// By every lane of a warp; the warp agrees on the outcome.
template <class S>
__device__ __forceinline__ bool attn_wait_warp(S& sm, uint64_t* bar, uint32_t parity, int* status) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, attn_wait(sm, bar, parity, status));
}

__device__ __forceinline__ void attn_drain(uint64_t* bar, uint32_t parity) {
  const uint64_t t0 = globaltimer_ns();
  while (!mbar_try_wait_sleep(bar, parity, 20000))
    if (globaltimer_ns() - t0 > 1000000000ull) return;
}

// ---- PTX ------------------------------------------------------------------------

// From a whole converged warp; the operands are the same in every lane.
__device__ __forceinline__ void mbar_expect_elect(uint64_t* bar, uint32_t bytes) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "@e mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(smem_u32(bar)), "r"(bytes)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d_elect(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "@e cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];\n\t}" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_4d_elect(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w,
                                                  uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "@e cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
      : "memory");
}

// D(tmem) (+)= A * B, 16-bit operands, fp32 sums; A in shared memory (ss) or tensor memory
// (ts), B in shared memory.  From a whole converged warp, the operands the same in every lane.
__device__ __forceinline__ void umma_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
      "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
      "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
// R consecutive columns (4, 8 or 16) of this thread's lane.
template <int R>
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[R]) {
  if constexpr (R == 4)
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr) : "memory");
  else if constexpr (R == 8)
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr) : "memory");
  else
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}
template <int R>
__device__ __forceinline__ void tmem_st_cols(uint32_t taddr, const uint32_t (&r)[R]) {
  if constexpr (R == 4)
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3])
                 : "memory");
  else if constexpr (R == 8)
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
  else
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <bool kFp16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  uint32_t u;
  if (kFp16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(b), "f"(a));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(b), "f"(a));
  return u;
}

// Instruction descriptor: kind::f16, A and B of one 16-bit type, fp32 D; A and B
// K-major, or with their M (kAm) or N (kBn) index contiguous.
template <bool kFp16, bool kAm, bool kBn>
__host__ __device__ constexpr uint32_t attn_idesc(int M, int N) {
  return (1u << 4) | (kFp16 ? 0u : (1u << 7) | (1u << 10)) | (kAm ? 1u << 15 : 0u) | (kBn ? 1u << 16 : 0u) |
         (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// Descriptor of a V tile as an operand whose K index is the key: [D / 64][128 keys][64
// elements], 128-byte swizzle, the other index (the element) contiguous: 64-element blocks `block` bytes apart, groups
// of 8 keys 1024 bytes apart.
__device__ __forceinline__ uint64_t sw128_v_desc(uint32_t saddr, uint32_t block) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(block >> 4) << 16;
  d |= static_cast<uint64_t>(1024u >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}

// ---- the schedule ------------------------------------------------------------------

// A request's rows and lengths; q = 0 if it has none or they are out of range.
struct Request {
  int c0, q, kv;
};
__device__ __forceinline__ Request request(const PagedAttnParams& p, int s, bool* bad) {
  Request r;
  r.c0 = p.cu[s];
  const int c1 = p.cu[s + 1];
  r.kv = p.kv_lens[s];
  const bool ok = r.c0 >= 0 && c1 >= r.c0 && c1 <= p.T && r.kv >= 0 && r.kv <= (p.max_pages << p.page_shift);
  r.q = ok ? c1 - r.c0 : 0;
  if (!ok) *bad = true;
  return r;
}

// Unit m of a request: tokens [2 P m, 2 P m + n), keys [lo, hi), key tiles [t0, t0 + tiles).
struct Unit {
  int n, lo, hi, t0, tiles, kind;
};
__device__ __forceinline__ Unit unit_of(const PagedAttnParams& p, const Request& r, int m) {
  Unit u;
  const int i0 = 2 * p.P * m;
  u.n = min(2 * p.P, r.q - i0);
  const int pos0 = r.kv - r.q + i0;
  u.hi = max(0, pos0 + u.n);
  u.lo = p.window > 0 ? max(0, pos0 - p.window + 1) : 0;
  u.t0 = u.lo >> 7;
  u.tiles = max(1, ((u.hi + 127) >> 7) - u.t0);
  u.kind = u.n > p.P ? kFull : u.n * p.G > kFewRows ? kPaired : kFew;
  return u;
}
__device__ __forceinline__ long long cost_of(const Unit& u) {
  return static_cast<long long>(tile_cost(u.kind)) * u.tiles + unit_cost(u.kind);
}
__device__ __forceinline__ int units_of(const PagedAttnParams& p, int q) { return (q + 2 * p.P - 1) / (2 * p.P); }

// a / b for 0 <= a, 0 < b (a 64-bit division costs hundreds of cycles).
__device__ __forceinline__ long long divide(long long a, long long b) {
  if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
  return a / b;
}

// Cost of a request's units for one KV head.
__device__ __forceinline__ long long head_cost(const PagedAttnParams& p, const Request& r) {
  long long c = 0;
  const int M = units_of(p, r.q);
  for (int m = 0; m < M; ++m) {
    const Unit u = unit_of(p, r, m);
    c += cost_of(u);
  }
  return c;
}

// Sum of v over the block's threads before this one (total: over all).
template <class S>
__device__ __forceinline__ long long block_prefix(S& sm, long long v, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long a = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, a, o);
    if (lane >= o) a += x;
  }
  __syncthreads();
  if (lane == 31) sm.scan[warp] = a;
  __syncthreads();
  long long before = 0, all = 0;
  for (int w = 0; w < kAttnThreads / 32; ++w) {
    if (w < warp) before += sm.scan[w];
    all += sm.scan[w];
  }
  *total = all;
  return before + a - v;
}

// The CTA's share [x0, x1) of the total cost, and the request that holds x0 with the
// cost before it (all threads; the block's result).
struct Share {
  long long x0, x1, before, share;
  int s, h;  // (h: kHeadsOuter)
};
// The CTA's share of `outer` rounds of cost `round`; before: the cost of the rounds before its own.
__device__ __forceinline__ Share share_at(long long round, int outer, int least) {
  Share r;
  const long long total = round * outer;
  r.share = max(static_cast<long long>(least), divide(total + gridDim.x - 1, gridDim.x));
  r.x0 = min(total, r.share * blockIdx.x);
  r.x1 = min(total, r.x0 + r.share);
  r.h = outer > 1 && round > 0 ? static_cast<int>(divide(r.x0, round)) : 0;
  r.before = r.h * round;
  return r;
}

template <class S>
__device__ __forceinline__ Share share_of(const PagedAttnParams& p, S& sm) {
  const int tid = threadIdx.x;
  bool bad = false;
  long long total = 0, mine = 0, first_before = 0;
  const int per = S::kHeadsOuter ? 1 : p.H_kv, outer = S::kHeadsOuter ? p.H_kv : 1;
  for (int s0 = 0; s0 < p.B; s0 += kAttnThreads) {
    mine = 0;
    if (s0 + tid < p.B) mine = head_cost(p, request(p, s0 + tid, &bad)) * per;
    long long all;
    const long long before = block_prefix(sm, mine, &all);
    if (s0 == 0) first_before = before;
    total += all;
  }
  if (bad && blockIdx.x == 0) atomicOr(p.status, kStatusDevice);
  Share r = share_at(total, outer, kMinShare);
  const long long x = r.x0 - r.before;
  // the thread whose request holds x0 says so
  if (p.B <= kAttnThreads) {
    if (mine > 0 && first_before <= x && x < first_before + mine) {
      sm.start = tid;
      sm.carry = first_before;
    }
  } else {
    long long sum = 0;
    for (int s0 = 0; s0 < p.B; s0 += kAttnThreads) {
      bool b = false;
      const long long c = s0 + tid < p.B ? head_cost(p, request(p, s0 + tid, &b)) * per : 0;
      long long all;
      const long long before = sum + block_prefix(sm, c, &all);
      if (c > 0 && before <= x && x < before + c) {
        sm.start = s0 + tid;
        sm.carry = before;
      }
      sum += all;
      if (sum > x) break;
    }
  }
  __syncthreads();
  r.s = static_cast<int>(sm.start);
  r.before += sm.carry;
  return r;
}

// The same by one warp for up to 32 requests, with no barrier for the block (one generation
// at a 4K context 13.1 us with the block's, 11.3 so).  Lane s keeps request s and its cost
// for one KV head.
template <class S>
__device__ __forceinline__ Share share_of_warp(const PagedAttnParams& p, Request& held, long long& held_cost) {
  const int lane = threadIdx.x & 31;
  bool bad = false;
  held = {};
  if (lane < p.B) held = request(p, lane, &bad);
  held_cost = head_cost(p, held);
  const long long mine = S::kHeadsOuter ? held_cost : held_cost * p.H_kv;
  if (bad && blockIdx.x == 0) atomicOr(p.status, kStatusDevice);
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  const bool rows = __any_sync(0xffffffffu, held.q * p.G > kFewRows);
  Share r = share_at(__shfl_sync(0xffffffffu, upto, 31), S::kHeadsOuter ? p.H_kv : 1, rows ? kMinShareRows : kMinShare);
  const long long x = r.x0 - r.before;
  const uint32_t here = __ballot_sync(0xffffffffu, mine > 0 && upto - mine <= x && x < upto);
  r.s = here ? __ffs(here) - 1 : 0;  // (none: the share is empty)
  r.before += __shfl_sync(0xffffffffu, upto - mine, r.s);
  return r;
}

// Warp 2: the CTA's entries in order.
template <class S>
__device__ __forceinline__ void deal(const PagedAttnParams& p, S& sm, Share sh) {
  uint32_t e = 0;
  const int lane = threadIdx.x & 31;
  const bool short_batch = p.B <= 32;
  Request held;
  long long held_cost;
  if (short_batch) sh = share_of_warp<S>(p, held, held_cost);
  auto get = [&](int s) {
    if (short_batch)
      return Request{__shfl_sync(0xffffffffu, held.c0, s), __shfl_sync(0xffffffffu, held.q, s), __shfl_sync(0xffffffffu, held.kv, s)};
    bool bad = false;  // (said by the schedule's first pass)
    return request(p, s, &bad);
  };
  auto put = [&](const Entry& en) {
    if (!attn_wait_warp(sm, &sm.eempty[e % kEntries], ((e / kEntries) & 1) ^ 1, p.status)) return false;
    if (lane == 0) {
      sm.ring[e % kEntries] = en;
      mbar_arrive(&sm.efull[e % kEntries]);
    }
    __syncwarp();
    ++e;
    return true;
  };
  if (sh.x0 < sh.x1) {
    int s = sh.s;
    Request r = get(s);
    long long a = sh.before;  // cost before the unit
    int h = sh.h, m = 0;
    if (!S::kHeadsOuter) {
      const long long hc = short_batch ? __shfl_sync(0xffffffffu, held_cost, s) : head_cost(p, r);
      h = static_cast<int>(divide(sh.x0 - a, hc));
      a += h * hc;
    }
    Unit u = unit_of(p, r, m);
    while (a + cost_of(u) <= sh.x0) {
      a += cost_of(u);
      u = unit_of(p, r, ++m);
    }
    while (a < sh.x1) {
      // boundary x cuts a unit before tile ceil((x - a) / cost of a tile)
      const int w = tile_cost(u.kind);
      auto cut = [&](long long x) {
        const long long o = x - a;
        return o <= 0 ? 0 : static_cast<int>(min(static_cast<long long>(u.tiles), (o + w - 1) / w));
      };
      const int c0 = cut(sh.x0), c1 = cut(sh.x1);
      if (c0 < c1) {
        Entry en;
        en.tok0 = r.c0 + 2 * p.P * m;
        en.n = u.n;
        en.pos0 = r.kv - r.q + 2 * p.P * m;
        en.h = h;
        en.s = s;
        en.t0 = u.t0 + c0;
        en.t1 = u.t0 + c1;
        en.klo = u.lo;
        en.khi = u.hi;
        en.kind = u.kind;
        en.first = static_cast<int>(divide(a, sh.share));
        en.pieces = static_cast<int>(divide(a + static_cast<long long>(w) * (u.tiles - 1), sh.share)) - en.first + 1;
        if (!put(en)) return;
      }
      a += cost_of(u);
      if (a >= sh.x1) break;
      if (2 * p.P * ++m >= r.q) {
        m = 0;
        if (S::kHeadsOuter) {
          do {
            if (++s == p.B) {
              s = 0;
              ++h;
            }
            r = get(s);
          } while (r.q == 0);
        } else if (++h == p.H_kv) {
          h = 0;
          do r = get(++s);
          while (r.q == 0);
        }
      }
      u = unit_of(p, r, m);
    }
  }
  Entry end = {};
  put(end);
}

// The next entry; every warp that takes entries calls it in order.  n = 0: no more.
template <class S>
__device__ __forceinline__ Entry take(const PagedAttnParams& p, S& sm, uint32_t e) {
  Entry en = {};
  if (attn_wait_warp(sm, &sm.efull[e % kEntries], (e / kEntries) & 1, p.status)) {
    en = sm.ring[e % kEntries];
    __syncwarp();
    mbar_arrive_elect(&sm.eempty[e % kEntries]);
  }
  return en;
}

// A value that is the same in every lane, broadcast, so that the compiler knows it to be: what
// depends on it is one path for the warp, with operands in uniform registers.
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

// ---- warp 0: loads -------------------------------------------------------------------
// Order of an entry's tiles in the ring: A K tiles ahead of V (A = 1 for a full unit;
// 2 for the others, whose sides work on two tiles at once).
template <int D>
__device__ __forceinline__ void load_warp(const PagedAttnParams& p, AttnSmem<D>& sm) {
  using S = AttnSmem<D>;
  const int lane = threadIdx.x & 31;
  const int box_shift = min(p.page_shift, 7);  // rows of a page box
  const int boxes = kRows >> box_shift;        // page boxes of a tile
  uint32_t st = 0, ph = 0, qn = 0, issued = 0;
  bool ok = true;
  for (uint32_t e = 0; ok; ++e) {
    const Entry en = take(p, sm, e);
    if (uniform(en.n) == 0) break;
    const int kind = uniform(en.kind), h = uniform(en.h), t0 = uniform(en.t0), t1 = uniform(en.t1);
    const int tok0 = uniform(en.tok0), klo = uniform(en.klo), khi = uniform(en.khi);
    const bool one = uniform(en.n) == 1;
    // ---- pages ----
    // lane i holds the page of the tile's box i: its entry of the table, read three tiles ahead and checked when used
    const int* row = p.table + static_cast<long long>(uniform(en.s)) * p.max_pages;
    auto page_of = [&](int t) {
      const int k = t * kRows + (lane << box_shift);
      return t < t1 && lane < boxes && k < khi && k + (1 << box_shift) > klo ? row[k >> p.page_shift] : INT_MAX;
    };
    int r0 = page_of(t0), r1 = page_of(t0 + 1), r2 = page_of(t0 + 2);
    // ---- Q tiles ----
    const int sides = kind == kFull ? 2 : 1;
    for (int x = 0; ok && x < sides; ++x) {
      const uint32_t qs = qn & 1;
      ok = attn_wait_warp(sm, &sm.qempty[qs], ((qn >> 1) & 1) ^ 1, p.status);
      if (!ok) break;
      mbar_expect_elect(&sm.qfull[qs], static_cast<uint32_t>(p.G) * (one ? 1 : p.P) * D * 2);
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
        tma_load_3d_elect(smem_u32(sm.q[qs]) + c * (kRows * 128), one ? &p.qmap1 : &p.qmap, c * 64, h * p.G, tok0 + x * p.P,
                          smem_u32(&sm.qfull[qs]));
      ++qn;
    }
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
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
          tma_load_4d_elect(dst + c * (kRows * 128), map, c * 64, y, h, uniform(page), bar);
      } else {
        for (int i = 0; i < boxes; i += 2) {  // an even number of them
          const int pa = __shfl_sync(0xffffffffu, page, i), pb = __shfl_sync(0xffffffffu, page, i + 1);
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            const uint32_t at = dst + c * (kRows * 128) + (i << (box_shift + 7));
            tma_load_4d_elect(at, map, c * 64, y, h, pa, bar);
            tma_load_4d_elect(at + (1 << (box_shift + 7)), map, c * 64, y, h, pb, bar);
          }
        }
      }
      ++issued;
      if (++st == S::kStages) { st = 0; ph ^= 1; }
    };
    const int A = kind == kFull ? 1 : 2;
    int p0 = checked(r0), p1 = checked(r1);  // pages of tiles t, t + 1
    for (int a = 0; a < A && t0 + a < t1; ++a) load(&p.kmap, t0 + a, a == 0 ? p0 : p1);
    for (int t = t0; ok && t < t1; ++t) {
      const int r3 = page_of(t + 3);
      const int p2 = checked(r2);
      load(&p.vmap, t, p0);
      if (t + A < t1) load(&p.kmap, t + A, A == 1 ? p1 : p2);
      p0 = p1;
      p1 = p2;
      r2 = r3;
    }
  }
  // After an abort, wait (bounded) for the copies still landing before the CTA retires.
  if (!ok || ld_volatile(&sm.abort_flag)) {
    for (uint32_t b = 0; b < 2 && b < qn; ++b) attn_drain(&sm.qfull[(qn - 1 - b) & 1], ((qn - 1 - b) >> 1) & 1);
    for (uint32_t b = 0; b < S::kStages && b < issued; ++b) {
      const uint32_t n = issued - 1 - b;
      attn_drain(&sm.full[n % S::kStages], (n / S::kStages) & 1);
    }
  }
}

// ---- warp 1: MMAs --------------------------------------------------------------------

// The weights of a side's few rows, [2][16 rows][64 keys] with the 128-byte swizzle, lie in
// the rows' Q tile from its row 32 on.
__device__ __forceinline__ uint32_t few_p_offset(int side) { return 4096 + side * 4096; }

// Tensor memory columns of a side's scores (then weights) and of its output.
__device__ __forceinline__ uint32_t s_col(int side) { return side * 128; }
__device__ __forceinline__ uint32_t o_col(int side) { return 256 + side * 128; }

// One warp issues every MMA: the sides' products run in turn, whole (issued by a thread
// for each side they interleave, and either side waits twice as long for its own).  What
// steers it is broadcast from lane 0, so that the compiler sees one path for the warp and
// keeps the MMAs' operands in uniform registers.
template <int D, bool kFp16>
__device__ __forceinline__ void mma_warp(const PagedAttnParams& p, AttnSmem<D>& sm, uint32_t tmem) {
  using S = AttnSmem<D>;
  constexpr uint32_t kBlock = kRows * 128;  // bytes of a 64-element column block
  constexpr uint32_t kIdescQK = attn_idesc<kFp16, false, false>(128, 128);
  constexpr uint32_t kIdescPV = attn_idesc<kFp16, false, true>(128, D);
  constexpr uint32_t kIdescKQ = attn_idesc<kFp16, false, false>(128, kFewRows);
  constexpr uint32_t kIdescVP = attn_idesc<kFp16, true, false>(128, kFewRows);
  uint32_t st = 0, ph = 0, qn = 0, pph[2] = {0, 0};
  bool ok = true;
  auto advance = [&] { if (++st == S::kStages) { st = 0; ph ^= 1; } };
  auto tile = [&] {  // the next tile of the ring has landed
    ok = ok && attn_wait_warp(sm, &sm.full[st], ph, p.status);
  };
  for (uint32_t e = 0; ok; ++e) {
    const Entry en = take(p, sm, e);
    if (uniform(en.n) == 0) break;
    const int n = uniform(en.t1 - en.t0), kind = uniform(en.kind);
    const uint32_t q0 = qn & 1;
    if (kind == kFew) {
      // transposed products: S^T = K Q^T (lanes are keys), O^T += V^T P^T (lanes are elements)
      ok = attn_wait_warp(sm, &sm.qfull[q0], (qn >> 1) & 1, p.status);
      ++qn;
      const uint64_t qdesc = sw128_desc(smem_u32(sm.q[q0]));
      auto kq = [&](int x) {
        tile();
        if (!ok) return;
        tc_fence_after();
        const uint64_t kdesc = sw128_desc(smem_u32(sm.kv[st]));
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = (k >> 2) * (kBlock / 16) + (k & 3) * 2;
          umma_ss(tmem + s_col(x), kdesc + off, qdesc + off, kIdescKQ, k > 0);
        }
        umma_commit_elect(&sm.sfull[x]);
        umma_commit_elect(&sm.empty[st]);
        advance();
      };
      for (int j = 0; j < 2 && j < n; ++j) kq(j);
      for (int j = 0; ok && j < n; ++j) {
        const int x = j & 1;
        tile();
        ok = ok && attn_wait_warp(sm, &sm.pfull[x][kParts - 1], pph[x], p.status);
        if (!ok) break;
        pph[x] ^= 1;
        tc_fence_after();
        const uint64_t vdesc = sw128_v_desc(smem_u32(sm.kv[st]), kBlock);
        const uint64_t pdesc = sw128_desc(smem_u32(sm.q[q0]) + few_p_offset(x));
#pragma unroll
        for (int k = 0; k < kRows / 16; ++k)
          umma_ss(tmem + o_col(x), vdesc + k * (16 * 128 / 16), pdesc + (k >> 2) * (kFewRows * 128 / 16) + (k & 3) * 2,
                  kIdescVP, j >= 2 || k > 0);
        umma_commit_elect(&sm.empty[st]);
        if (j + 2 >= n) umma_commit_elect(&sm.ofull[x]);
        advance();
        if (j + 2 < n) kq(x);
      }
      umma_commit_elect(&sm.qempty[q0]);  // (the weights lie in the Q tile)
    } else {
      const bool full = kind == kFull;
      const int sides = full ? 2 : 1, A = full ? 1 : 2;
      for (int i = 0; ok && i < sides; ++i, ++qn) ok = attn_wait_warp(sm, &sm.qfull[qn & 1], (qn >> 1) & 1, p.status);
      auto qk = [&](int x, uint32_t q, uint32_t stage) {
        const uint64_t qdesc = sw128_desc(smem_u32(sm.q[q])), kdesc = sw128_desc(smem_u32(sm.kv[stage]));
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = (k >> 2) * (kBlock / 16) + (k & 3) * 2;
          umma_ss(tmem + s_col(x), qdesc + off, kdesc + off, kIdescQK, k > 0);
        }
        umma_commit_elect(&sm.sfull[x]);
      };
      // the K tile is done with, and after the last one the rows' Q tiles
      auto k_done = [&](int j, uint32_t stage) {
        umma_commit_elect(&sm.empty[stage]);
        if (j == n - 1)
          for (int i = 0; i < sides; ++i) umma_commit_elect(&sm.qempty[q0 ^ i]);
      };
      for (int j = 0; ok && j < A && j < n; ++j) {
        tile();
        if (!ok) break;
        tc_fence_after();
        qk(j, q0, st);
        if (full) qk(1, q0 ^ 1, st);
        k_done(j, st);
        advance();
      }
      for (int j = 0; ok && j < n; ++j) {
        // the V tile and the next K tile are there before the first weights are waited for
        const uint32_t vs = st;
        tile();
        advance();
        const bool more = j + A < n;
        const uint32_t ks = st;
        if (more) {
          tile();
          advance();
        }
        for (int i = 0; ok && i < sides; ++i) {
          const int x = full ? i : j & 1;
          const uint64_t vdesc = sw128_v_desc(smem_u32(sm.kv[vs]), kBlock);
          const bool first = j < A;
#pragma unroll
          for (int part = 0; part < kParts; ++part) {
            ok = ok && attn_wait_warp(sm, &sm.pfull[x][part], pph[x], p.status);
            tc_fence_after();
            if (ok) {
#pragma unroll
              for (int k = part * 8 / kParts; k < (part + 1) * 8 / kParts; ++k)
                umma_ts(tmem + o_col(x), tmem + s_col(x) + k * 8, vdesc + k * (16 * 128 / 16), kIdescPV, !first || k > 0);
            }
          }
          if (!ok) break;
          pph[x] ^= 1;
          if (more) {
            qk(x, full ? q0 ^ i : q0, ks);
          } else {
            umma_commit_elect(&sm.ofull[x]);
          }
          if (i == sides - 1) {
            umma_commit_elect(&sm.empty[vs]);
            if (more) k_done(j + A, ks);
          }
        }
      }
    }
  }
  umma_commit_elect(&sm.done);
  attn_drain(&sm.done, 0);
}

// ---- softmax warpgroups ------------------------------------------------------------------
// A group's four warps run in step: they agree on every entry, and a wait that ran out
// (ok = false) lets them run on with whatever is there, so that each reaches the same
// barriers; the waits of an aborted CTA return at once.

template <int D>
__device__ __forceinline__ size_t part_bytes() { return kRows * D * 4 + kRows * sizeof(float2); }

__device__ __forceinline__ void group_sync(int x) { named_bar_sync(1 + x, 128); }
__device__ __forceinline__ bool group_any(int x, bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred a, b;\n\t"
      "setp.ne.u32 a, %1, 0;\n\t"
      "barrier.cta.red.or.pred b, %2, 128, a;\n\t"
      "selp.u32 %0, 1, 0, b;\n\t}"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(v)), "r"(1 + x)
      : "memory");
  return r != 0;
}

// What a softmax warp keeps from entry to entry.
struct SideState {
  uint32_t sph = 0, oph = 0, xph = 0, qn = 0;  // phases of its barriers, Q tiles before this entry
  uint32_t tiles = 0;                          // K and V tiles before this entry
  bool ok = true;
};

// Before a side's weights of tile j (the a-th of the entry) are handed over: zeroes the
// rows of the V tile that hold no key of the unit, of which anything may be in the pool
// (0 weight times NaN is NaN).  Only the rows of a page box that also holds keys need it,
// the others were loaded as zeros.  In a full unit both sides write the same zeros.
template <int D>
__device__ __forceinline__ void mend_v(const PagedAttnParams& p, AttnSmem<D>& sm, const Entry& en, int j, SideState& st) {
  const int k0 = j * kRows, a = max(en.klo - k0, 0), b = min(en.khi - k0, kRows);
  if (a == 0 && b == kRows) return;
  const int n = en.t1 - en.t0, i = j - en.t0;
  // the V tile's place in the ring's order (K tiles run 1 or 2 ahead)
  const uint32_t at = st.tiles + (en.kind == kFull ? 2 * i + 1 : min(2 * i + 2, 2 * n - 1));
  const uint32_t stage = at % AttnSmem<D>::kStages;
  st.ok = st.ok && attn_wait_warp(sm, &sm.full[stage], (at / AttnSmem<D>::kStages) & 1, p.status);
  const int box = 1 << min(p.page_shift, 7);
  auto zero = [&](int r0, int r1) {
    for (int q = r0 * (D / 8) + static_cast<int>(threadIdx.x & 127); q < r1 * (D / 8); q += 128) {
      const int r = q / (D / 8), c = q % (D / 8);
      *reinterpret_cast<uint4*>(sm.kv[stage] + (c >> 3) * (kRows * 128) + r * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
    }
  };
  zero(a & ~(box - 1), a);
  if (b > 0) zero(b, min(kRows, (b + box - 1) & ~(box - 1)));
  fence_proxy_async();
}

template <int D>
struct Records {  // of a cut unit's piece, side x: the rows' unnormalised output, then their (m, l)
  uint8_t* at;
  __device__ float2* ml() const { return reinterpret_cast<float2*>(at + kRows * D * 4); }
};
template <int D>
__device__ __forceinline__ Records<D> records(const PagedAttnParams& p, long long cta, bool first, int x) {
  return {p.parts + ((2 * cta + (first ? 1 : 0)) * 2 + x) * part_bytes<D>()};
}

// After the group's records of a piece are written: whether it is the last of the unit's pieces.
template <int D>
__device__ __forceinline__ bool arrived_last(const PagedAttnParams& p, AttnSmem<D>& sm, const Entry& en, int x, bool ok) {
  group_sync(x);
  if ((threadIdx.x & 127) == 0) {
    int last = 0;
    if (ok) {
      // releases the whole group's records (the barrier orders them before it), acquires the others'
      int* cnt = p.sync + 2 * en.first + x;
      int n;
      asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(n) : "l"(cnt) : "memory");
      last = n == en.pieces - 1;
      if (last) *cnt = 0;
    }
    sm.last[x] = last;
  }
  group_sync(x);
  return sm.last[x] != 0;
}

__device__ __forceinline__ float lse_of(float m, float l) {  // natural log; m and l of weights 2^up larger
  return l > 0.f ? (m + lg2_approx(l)) * 0.6931471805599453f : (l == 0.f ? -INFINITY : l);
}
__device__ __forceinline__ float finite_or_0(float m) { return m == -INFINITY ? 0.f : m; }

// ---- up to 16 rows: a thread per key ----
// S^T has the tile's keys on the lanes and the rows in the columns, so a thread forms
// its key's weights of R rows; they go to shared memory as the B operand of
// O^T += V^T P^T.  All threads hold the rows' maxima; each sums its own keys' weights.
template <int D, bool kFp16, int R>
__device__ __forceinline__ void few_rows(const PagedAttnParams& p, AttnSmem<D>& sm, uint32_t tmem, int x, const Entry& en,
                                         SideState& st) {
  const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31, key = warp * 32 + lane;
  const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
  const uint32_t ts = tmem + lanes + s_col(x);
  const float c = p.scale_log2;
  constexpr float kUp = kFp16 ? 7.f : 0.f;
  // this key's 2 bytes of row r are at r * 128 + ((chunk ^ r) & 7) * 16 from here
  uint8_t* const pw = sm.q[st.qn & 1] + few_p_offset(x) + (key >> 6) * (kFewRows * 128) + (key & 7) * 2;
  const int chunk = (key & 63) >> 3;
  const int rows = en.n * p.G;
  const int f1 = rows < R ? 0 : (en.pos0 + 1) >> 7;  // [f0, f1): every row sees every key
  const int f0 = p.window > 0 ? (max(0, en.pos0 + en.n - p.window) + 127) >> 7 : 0;
  float m[R], l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) { m[r] = -INFINITY; l[r] = 0.f; }
  const int first = en.t0 + x;
  for (int j = first; j < en.t1; j += 2) {
    st.ok = st.ok && attn_wait_warp(sm, &sm.sfull[x], st.sph, p.status);
    st.sph ^= 1;
    tc_fence_after();
    uint32_t u[R];
    tmem_ld_cols<R>(ts, u);
    float y[R];
#pragma unroll
    for (int r = 0; r < R; ++r) y[r] = __uint_as_float(u[r]) * c;
    if (j < f0 || j >= f1) {
      const int k = j * kRows + key;
      int t = en.pos0, g = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r >= rows || k > t || (p.window > 0 && k <= t - p.window)) y[r] = -INFINITY;
        if (++g == p.G) { g = 0; ++t; }
      }
    }
    bool up = false;
#pragma unroll
    for (int r = 0; r < R; ++r) up |= y[r] > m[r] + kRaise;
    if (group_any(x, up)) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float v = y[r];
#pragma unroll
        for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
        if (lane == 0) sm.red[x][warp][r] = v;
      }
      group_sync(x);
      float f[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float top = fmaxf(fmaxf(sm.red[x][0][r], sm.red[x][1][r]), fmaxf(sm.red[x][2][r], sm.red[x][3][r]));
        const float mn = fmaxf(m[r], top);
        f[r] = ex2_approx(m[r] - finite_or_0(mn));
        m[r] = mn;
        l[r] *= f[r];
      }
      if (j != first) {
        // S of this tile is complete, so is O of the side's tile before it, and the next waits for us
        uint32_t o[R];
        tmem_ld_cols<R>(tmem + lanes + o_col(x), o);
#pragma unroll
        for (int r = 0; r < R; ++r) o[r] = __float_as_uint(__uint_as_float(o[r]) * f[r]);
        tmem_st_cols<R>(tmem + lanes + o_col(x), o);
        tmem_wait_st();
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float w = ex2_approx(y[r] - (finite_or_0(m[r]) - kUp));
      l[r] += w;
      *reinterpret_cast<uint16_t*>(pw + r * 128 + ((chunk ^ r) & 7) * 16) = static_cast<uint16_t>(pack2<kFp16>(w, 0.f));
    }
    mend_v<D>(p, sm, en, j, st);
    fence_proxy_async();
    tc_fence_before();
    __syncwarp();
#pragma unroll
    for (int part = 0; part < kParts; ++part) mbar_arrive_elect(&sm.pfull[x][part]);
  }
  // ---- the rows' output: sums over the keys, then both sides' accumulators ----
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float v = l[r];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    l[r] = v;
  }
  group_sync(x);  // (the maxima's readers are done)
  if (lane < R) {
    float v = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) v = r == lane ? l[r] : v;
    sm.red[x][warp][lane] = v;
  }
  group_sync(x);
  if (warp == 0 && lane < R) {
    float v = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) v = r == lane ? m[r] : v;
    sm.ml[x][lane] = make_float2(v, (sm.red[x][0][lane] + sm.red[x][1][lane]) + (sm.red[x][2][lane] + sm.red[x][3][lane]));
  }
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
  float v[R];
  {
    uint32_t o[R];
    tmem_ld_cols<R>(tmem + lanes + o_col(0), o);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float2 a = sm.ml[0][r], b = both ? sm.ml[1][r] : make_float2(-INFINITY, 0.f);
      m[r] = fmaxf(a.x, b.x);
      const float f = ex2_approx(a.x - finite_or_0(m[r]));
      l[r] = fmaf(a.y, f, b.y * ex2_approx(b.x - finite_or_0(m[r])));
      v[r] = l[r] == 0.f ? 0.f : __uint_as_float(o[r]) * f;
    }
    if (both) {
      tmem_ld_cols<R>(tmem + lanes + o_col(1), o);
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (l[r] != 0.f) v[r] = fmaf(__uint_as_float(o[r]), ex2_approx(sm.ml[1][r].x - finite_or_0(m[r])), v[r]);
    }
  }
  tc_fence_before();
  __syncwarp();
  mbar_arrive_elect(&sm.xfree);
  // side x writes the rows r with r mod 2 = x; the thread's element is d = key
  auto emit = [&](int r, float o, float mm, float ll) {
    const int i = r / p.G, head = en.h * p.G + r - i * p.G;
    if (key < D)
      *reinterpret_cast<uint16_t*>(p.out + static_cast<long long>(en.tok0 + i) * p.out_token +
                                   static_cast<long long>(head) * p.out_head + key * 2) = static_cast<uint16_t>(pack2<kFp16>(o, 0.f));
    if (p.lse && key == r) p.lse[static_cast<long long>(en.tok0 + i) * p.H_q + head] = lse_of(mm - kUp, ll);
  };
  if (whole) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if ((r & 1) == x && r < rows) emit(r, v[r] * (l[r] == 0.f ? 0.f : 1.f / l[r]), m[r], l[r]);
  } else {
    const Records<D> mine = records<D>(p, blockIdx.x, en.first == static_cast<int>(blockIdx.x), x);
#pragma unroll
    for (int r = 0; r < R; ++r)
      if ((r & 1) == x && r < rows) {
        if (key < D) __stcg(reinterpret_cast<float*>(mine.at) + r * D + key, v[r]);
        if (key == r) __stcg(mine.ml() + r, make_float2(m[r], l[r]));
      }
    if (arrived_last(p, sm, en, x, st.ok)) {
      // the side's rows together, 32 records in flight
      constexpr int kR = R / 2, kU = 32 / kR;
      float mm[kR], ll[kR], oo[kR];
#pragma unroll
      for (int r = 0; r < kR; ++r) { mm[r] = -INFINITY; ll[r] = oo[r] = 0.f; }
      for (int q0 = 0; q0 < en.pieces; q0 += kU) {
        float2 z[kR][kU];
        float o[kR][kU];
#pragma unroll
        for (int q = 0; q < kU; ++q) {
          const Records<D> rec = records<D>(p, en.first + q0 + q, q0 + q == 0, x);
#pragma unroll
          for (int r = 0; r < kR; ++r) {
            z[r][q] = make_float2(-INFINITY, 0.f);
            o[r][q] = 0.f;
            if (q0 + q < en.pieces && 2 * r + x < rows) {
              z[r][q] = __ldcg(rec.ml() + 2 * r + x);
              if (key < D) o[r][q] = __ldcg(reinterpret_cast<const float*>(rec.at) + (2 * r + x) * D + key);
            }
          }
        }
#pragma unroll
        for (int r = 0; r < kR; ++r) {
          float mn = mm[r];
#pragma unroll
          for (int q = 0; q < kU; ++q) mn = fmaxf(mn, z[r][q].x);
          const float bs = finite_or_0(mn), f0 = ex2_approx(mm[r] - bs);
          ll[r] *= f0;
          oo[r] *= f0;
#pragma unroll
          for (int q = 0; q < kU; ++q) {
            const float f = ex2_approx(z[r][q].x - bs);
            ll[r] = fmaf(z[r][q].y, f, ll[r]);
            oo[r] = fmaf(o[r][q], f, oo[r]);
          }
          mm[r] = mn;
        }
      }
#pragma unroll
      for (int r = 0; r < kR; ++r)
        if (2 * r + x < rows) emit(2 * r + x, ll[r] == 0.f ? 0.f : oo[r] * (1.f / ll[r]), mm[r], ll[r]);
    }
  }
  // both sides have read both accumulators and (m, l) before either goes on
  st.ok = st.ok && attn_wait_warp(sm, &sm.xfree, st.xph, p.status);
  st.xph ^= 1;
  tc_fence_after();
  ++st.qn;
}

// ---- whole tiles of rows: a thread per row ----

// Keys [a, b] of 32 stay, the others' logits become -inf.
__device__ __forceinline__ void mask_keys(uint32_t (&u)[32], int a, int b) {
  const uint32_t from = a <= 0 ? ~0u : a > 31 ? 0u : ~0u << a;
  const uint32_t to = b < 0 ? 0u : b >= 31 ? ~0u : (2u << b) - 1;
  const uint32_t keep = from & to;
#pragma unroll
  for (int q = 0; q < 32; ++q)
    if (!(keep & (1u << q))) u[q] = 0xff800000u;
}

// Four lanes' four values each, transposed: lane q gets the q-th value of lane k as w[k].
__device__ __forceinline__ void transpose4(uint4 (&w)[4], int q) {
  auto swap = [&](uint4& a, uint4& b, bool up, int d) {  // lanes with `up` give a and take it back as theirs, the others b
    uint4 s = up ? a : b;
    s.x = __shfl_xor_sync(0xffffffffu, s.x, d);
    s.y = __shfl_xor_sync(0xffffffffu, s.y, d);
    s.z = __shfl_xor_sync(0xffffffffu, s.z, d);
    s.w = __shfl_xor_sync(0xffffffffu, s.w, d);
    (up ? a : b) = s;
  };
  swap(w[0], w[1], q & 1, 1);
  swap(w[2], w[3], q & 1, 1);
  swap(w[0], w[2], q & 2, 2);
  swap(w[1], w[3], q & 2, 2);
}

// Weights exp2(c u + nb) of 32 keys as 16-bit pairs, and their sums before rounding.
template <bool kFp16, int N>
__device__ __forceinline__ void weights(const uint32_t (&u)[32], float c, float nb, uint32_t (&w)[N], int o, float2 (&acc)[4]) {
  const float2 cc = make_float2(c, c), bb = make_float2(nb, nb);
#pragma unroll
  for (int q = 0; q < 16; ++q) {
    const float2 y = ffma2(make_float2(__uint_as_float(u[2 * q]), __uint_as_float(u[2 * q + 1])), cc, bb);
    const float2 z = make_float2(ex2_approx(y.x), ex2_approx(y.y));
    acc[q & 3] = fadd2(acc[q & 3], z);
    w[o + q] = pack2<kFp16>(z.x, z.y);
  }
}

__device__ __forceinline__ float max32u(const uint32_t (&u)[32]) {
  float v[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    v[q] = fmax3(__uint_as_float(u[8 * q]), __uint_as_float(u[8 * q + 1]), __uint_as_float(u[8 * q + 2]));
    v[q] = fmax3(v[q], __uint_as_float(u[8 * q + 3]), __uint_as_float(u[8 * q + 4]));
    v[q] = fmax3(v[q], __uint_as_float(u[8 * q + 5]), __uint_as_float(u[8 * q + 6]));
    v[q] = fmaxf(v[q], __uint_as_float(u[8 * q + 7]));
  }
  return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
}

template <int D, bool kFp16>
__device__ __forceinline__ void row_tiles(const PagedAttnParams& p, AttnSmem<D>& sm, uint32_t tmem, int x, const Entry& en,
                                          SideState& st, int i0) {
  const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31;
  const int r = warp * 32 + lane;  // row of the side = TMEM lane
  const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
  const uint32_t ts = tmem + lanes + s_col(x);
  const float c = p.scale_log2;
  // half precision: the weights are kept 2^7 larger, clear of its subnormals (a lagging maximum adds 2^kRaise)
  constexpr float kUp = kFp16 ? 7.f : 0.f;
  const bool paired = en.kind == kPaired;
  const int base = paired ? 0 : x * p.P * p.G;  // first row of the side in the unit
  const int rows = min(en.n * p.G - base, p.P * p.G);
  const bool valid = r < rows;
  const bool work = warp * 32 < rows;  // the warp has rows
  const int side0 = paired ? 0 : x * p.P;  // the side's first token, and its last
  const int side1 = side0 + min(en.n - side0, p.P) - 1;
  const int i = side0 + i0;  // token of the row
  const int t = en.pos0 + i;
  const int lo = p.window > 0 ? t - p.window + 1 : 0;
  // tiles [f0, f1) need no mask: every row of the side sees all of their keys
  const int f1 = (en.pos0 + side0 + 1) >> 7;
  const int f0 = p.window > 0 ? (max(0, en.pos0 + side1 - p.window + 1) + 127) >> 7 : 0;
  float m = -INFINITY, l = 0.f;
  const int step = paired ? 2 : 1;
  const int first = en.t0 + (paired ? x : 0);
  for (int j = first; j < en.t1; j += step) {
    st.ok = st.ok && attn_wait_warp(sm, &sm.sfull[x], st.sph, p.status);
    st.sph ^= 1;
    tc_fence_after();
    // weights stored: half h of the tile's is complete
    auto hand_over = [&](int h) {
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      mbar_arrive_elect(&sm.pfull[x][h]);
    };
    if (work) {
      const bool edge = j < f0 || j >= f1;
      bool slow = edge;
      if (!slow) {
        // the first half's weights by the maximum so far, while the tile's own is being formed
        uint32_t u[4][32], w[32];
        float2 acc[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        tmem_ld32_async(ts, u[0]);
        tmem_wait32(u[0]);
        if (j == first) m = max32u(u[0]) * c;  // (nothing summed yet: any start will do that the others are not far above)
        const float nb = kUp - finite_or_0(m);
        tmem_ld32_async(ts + 32, u[1]);
        weights<kFp16>(u[0], c, nb, w, 0, acc);
        float top = max32u(u[0]);
        tmem_wait32(u[1]);
        tmem_ld32_async(ts + 64, u[2]);
        weights<kFp16>(u[1], c, nb, w, 16, acc);
        top = fmaxf(top, max32u(u[1]));
        tmem_wait32(u[2]);
        tmem_ld32_async(ts + 96, u[3]);
        top = fmaxf(top, max32u(u[2]));
        tmem_wait32(u[3]);
        top = fmaxf(top, max32u(u[3])) * c;
        slow = __any_sync(0xffffffffu, valid && top > m + kRaise);
        if (!slow) {
          tmem_st32(ts, w);
          hand_over(0);
          weights<kFp16>(u[2], c, nb, w, 0, acc);
          weights<kFp16>(u[3], c, nb, w, 16, acc);
          tmem_st32(ts + 32, w);
          const float2 sum = fadd2(fadd2(acc[0], acc[1]), fadd2(acc[2], acc[3]));
          l += sum.x + sum.y;
          hand_over(1);
        }
      }
      if (slow) {
        // an edge of the rows' keys or a maximum to raise: in 32-key pieces
        // and two passes, which keep the code short (the instruction cache is the limit of short units)
        float top = -INFINITY;
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          uint32_t u[32];
          tmem_ld32_async(ts + 32 * q, u);
          tmem_wait32(u);
          if (edge) mask_keys(u, lo - j * kRows - 32 * q, t - j * kRows - 32 * q);
          top = fmaxf(top, max32u(u));
        }
        top *= c;
        const bool raise = valid && (j == first || top > m + kRaise);
        if (__any_sync(0xffffffffu, raise)) {
          const float f = raise ? ex2_approx(m - finite_or_0(top)) : 1.f;
          if (raise) { m = top; l *= f; }
          if (j != first) {
            // S of this tile is complete, so is O += P V of the side's tile before it, and the next waits for us
#pragma unroll 1
            for (int q = 0; q < D; q += 16) {
              uint32_t o[16];
              tmem_ld_cols<16>(tmem + lanes + o_col(x) + q, o);
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
              tmem_st_cols<16>(tmem + lanes + o_col(x) + q, o);
            }
          }
        }
        mend_v<D>(p, sm, en, j, st);
        float2 acc[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          uint32_t u[32], w[16];
          tmem_ld32_async(ts + 32 * q, u);
          tmem_wait32(u);
          if (edge) mask_keys(u, lo - j * kRows - 32 * q, t - j * kRows - 32 * q);
          weights<kFp16>(u, c, kUp - finite_or_0(m), w, 0, acc);
          tmem_st_cols<16>(ts + 16 * q, w);
          if (q & 1) hand_over(q >> 1);
        }
        const float2 sum = fadd2(fadd2(acc[0], acc[1]), fadd2(acc[2], acc[3]));
        l += sum.x + sum.y;
      }
    } else {
      mend_v<D>(p, sm, en, j, st);
      hand_over(0);
      hand_over(1);
    }
  }
  // ---- the rows' output ----
  if (first < en.t1) {  // (side 1 of a paired unit's single tile has no accumulator)
    st.ok = st.ok && attn_wait_warp(sm, &sm.ofull[x], st.oph, p.status);
    st.oph ^= 1;
    tc_fence_after();
  }
  // factors of the accumulators, and the columns that this side writes
  float fa = 1.f, fb = 0.f;
  int col0 = 0, cols = D;
  uint32_t oa = o_col(x);
  bool both = false;
  if (paired) {
    sm.ml[x][r] = make_float2(m, l);
    tc_fence_before();
    __syncwarp();
    mbar_arrive_elect(&sm.xfull);
    st.ok = st.ok && attn_wait_warp(sm, &sm.xfull, st.xph, p.status);
    tc_fence_after();
    both = en.t0 + 1 < en.t1;
    const float2 a = sm.ml[0][r], b = both ? sm.ml[1][r] : make_float2(-INFINITY, 0.f);
    m = fmaxf(a.x, b.x);
    fa = ex2_approx(a.x - finite_or_0(m));
    fb = ex2_approx(b.x - finite_or_0(m));
    l = fmaf(a.y, fa, b.y * fb);
    oa = o_col(0);
    cols = D / 2;
    col0 = x * cols;
  }
  const bool whole = en.pieces == 1;
  const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
  fa *= inv;
  fb *= inv;
  const Records<D> mine = records<D>(p, blockIdx.x, en.first == static_cast<int>(blockIdx.x), x);
  const int head = en.h * p.G + base + r - i * p.G;
  if (work) {
    // a warp's stores go row by row in groups of four lanes: lane q of a group writes the q-th 16 bytes of
    // 64 of each of its four rows in turn
    const int q4 = lane & 3;
    long long at[4];  // of the group's rows; -1: no row
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const long long mine4 = valid ? static_cast<long long>(en.tok0 + i) * p.out_token + static_cast<long long>(head) * p.out_head : -1;
      at[k] = __shfl_sync(0xffffffffu, mine4, (lane & 28) + k);
    }
#pragma unroll 1
    for (int q = col0; q < col0 + cols; q += 32) {
      uint32_t o[32];
      float v[32];
      tmem_ld32_async(tmem + lanes + oa + q, o);
      tmem_wait32(o);
#pragma unroll
      for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(o[k]) * fa;
      if (both) {
        tmem_ld32_async(tmem + lanes + o_col(1) + q, o);
        tmem_wait32(o);
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = fmaf(__uint_as_float(o[k]), fb, v[k]);
      }
      if (__any_sync(0xffffffffu, l == 0.f)) {  // no key (or none with a weight): nothing to weigh
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = l == 0.f ? 0.f : v[k];
      }
      if (whole) {
        uint4 w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          w[k].x = pack2<kFp16>(v[8 * k], v[8 * k + 1]);
          w[k].y = pack2<kFp16>(v[8 * k + 2], v[8 * k + 3]);
          w[k].z = pack2<kFp16>(v[8 * k + 4], v[8 * k + 5]);
          w[k].w = pack2<kFp16>(v[8 * k + 6], v[8 * k + 7]);
        }
        transpose4(w, q4);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (at[k] >= 0) *reinterpret_cast<uint4*>(p.out + at[k] + (q + 8 * q4) * 2) = w[k];
      } else if (valid) {
#pragma unroll
        for (int k = 0; k < 32; k += 4)
          __stcg(reinterpret_cast<float4*>(mine.at) + ((q - col0 + k) / 4) * kRows + r, make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]));
      }
    }
  }
  if (paired) {
    tc_fence_before();
    __syncwarp();
    mbar_arrive_elect(&sm.xfree);
  }
  if (whole) {
    if (p.lse && valid && (!paired || x == 0)) p.lse[static_cast<long long>(en.tok0 + i) * p.H_q + head] = lse_of(m - kUp, l);
  } else {
    if (valid) __stcg(mine.ml() + r, make_float2(m, l));
    if (arrived_last(p, sm, en, x, st.ok)) {
      // merge the unit's records in order: the row's maximum and sum, then 32 columns at a time
      if (valid) {
        float mm = -INFINITY, ll = 0.f;
        for (int q = 0; q < en.pieces; ++q) mm = fmaxf(mm, __ldcg(records<D>(p, en.first + q, q == 0, x).ml() + r).x);
        const float bs = finite_or_0(mm);
        for (int q = 0; q < en.pieces; ++q) {
          const float2 z = __ldcg(records<D>(p, en.first + q, q == 0, x).ml() + r);
          ll = fmaf(z.y, ex2_approx(z.x - bs), ll);
        }
        const float iv = ll == 0.f ? 0.f : 1.f / ll;
        uint8_t* const orow = p.out + static_cast<long long>(en.tok0 + i) * p.out_token + static_cast<long long>(head) * p.out_head;
#pragma unroll 1
        for (int c4 = 0; c4 < cols / 4; c4 += 8) {
          float4 oo[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) oo[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
          for (int q = 0; q < en.pieces; ++q) {
            const Records<D> rec = records<D>(p, en.first + q, q == 0, x);
            const float f = ex2_approx(__ldcg(rec.ml() + r).x - bs);
            float4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __ldcg(reinterpret_cast<const float4*>(rec.at) + (c4 + k) * kRows + r);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              oo[k].x = fmaf(v[k].x, f, oo[k].x);
              oo[k].y = fmaf(v[k].y, f, oo[k].y);
              oo[k].z = fmaf(v[k].z, f, oo[k].z);
              oo[k].w = fmaf(v[k].w, f, oo[k].w);
            }
          }
#pragma unroll
          for (int k = 0; k < 8; k += 2) {
            uint4 w;
            w.x = pack2<kFp16>(oo[k].x * iv, oo[k].y * iv);
            w.y = pack2<kFp16>(oo[k].z * iv, oo[k].w * iv);
            w.z = pack2<kFp16>(oo[k + 1].x * iv, oo[k + 1].y * iv);
            w.w = pack2<kFp16>(oo[k + 1].z * iv, oo[k + 1].w * iv);
            *reinterpret_cast<uint4*>(orow + (col0 + (c4 + k) * 4) * 2) = w;
          }
        }
        if (p.lse && (!paired || x == 0)) p.lse[static_cast<long long>(en.tok0 + i) * p.H_q + head] = lse_of(mm - kUp, ll);
      }
    }
  }
  if (paired) {  // both sides have read both accumulators and (m, l) before either goes on
    st.ok = st.ok && attn_wait_warp(sm, &sm.xfree, st.xph, p.status);
    st.xph ^= 1;
    tc_fence_after();
  }
  st.qn += paired ? 1 : 2;
}

template <int D, bool kFp16>
__device__ __forceinline__ void softmax_group(const PagedAttnParams& p, AttnSmem<D>& sm, uint32_t tmem, int x) {
  SideState st;
  const int i0 = static_cast<int>(threadIdx.x & 127) / p.G;  // the thread's row: its token in the side
  for (uint32_t e = 0;; ++e) {
    const Entry en = take(p, sm, e);
    if (group_any(x, en.n == 0)) break;  // no more, or a warp's wait for the entry ran out
    if (en.kind != kFew) row_tiles<D, kFp16>(p, sm, tmem, x, en, st, i0);
    else if (en.n * p.G <= 4) few_rows<D, kFp16, 4>(p, sm, tmem, x, en, st);
    else if (en.n * p.G <= 8) few_rows<D, kFp16, 8>(p, sm, tmem, x, en, st);
    else few_rows<D, kFp16, 16>(p, sm, tmem, x, en, st);
    st.tiles += 2 * (en.t1 - en.t0);
  }
}

template <int D, bool kFp16>
__global__ void __launch_bounds__(kAttnThreads, 1) paged_attn_kernel(const __grid_constant__ PagedAttnParams p) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  using S = AttnSmem<D>;
  if (smem_u32(smem_raw) & 1023u) {  // the 128-byte swizzle needs 1024-byte aligned buffers
    if (threadIdx.x == 0) atomicOr(p.status, kStatusDevice);
    return;
  }
  S& sm = *reinterpret_cast<S*>(smem_raw);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.qfull[i], 1);
      mbar_init(&sm.qempty[i], 1);
      mbar_init(&sm.sfull[i], 1);
      for (int j = 0; j < kParts; ++j) mbar_init(&sm.pfull[i][j], 4);
      mbar_init(&sm.ofull[i], 1);
    }
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], 1);
    }
    for (int i = 0; i < kEntries; ++i) {
      mbar_init(&sm.efull[i], 1);
      mbar_init(&sm.eempty[i], 10);  // the load and MMA warps and eight softmax warps
    }
    mbar_init(&sm.xfull, 8);
    mbar_init(&sm.xfree, 8);
    mbar_init(&sm.done, 1);
    sm.abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async();
  }
  if (threadIdx.x == 64) {
    for (const CUtensorMap* m : {&p.qmap1, &p.kmap, &p.vmap, &p.qmap})
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_slot, 512);
    tmem_relinquish();
  }
  pdl_wait();
  pdl_trigger();
  Share sh = {};
  if (p.B > 32) sh = share_of(p, sm);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_slot;
  if (warp < 4) {
    regs_dealloc<kRegsAttnControl>();
    if (warp == 0) load_warp<D>(p, sm);
    if (warp == 1) mma_warp<D, kFp16>(p, sm, tmem);
    if (warp == 2) deal(p, sm, sh);
    __syncwarp();
  } else {
    regs_alloc<kRegsAttnSoftmax>();
    softmax_group<D, kFp16>(p, sm, tmem, (warp - 4) >> 2);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

using AttnFn = void (*)(const PagedAttnParams);
AttnFn attn_fn(int d, bool fp16) {
  if (d == 64) return fp16 ? paged_attn_kernel<64, true> : paged_attn_kernel<64, false>;
  return fp16 ? paged_attn_kernel<128, true> : paged_attn_kernel<128, false>;
}
size_t attn_smem(int d) { return d == 64 ? sizeof(AttnSmem<64>) : sizeof(AttnSmem<128>); }

// Readies a kernel for the current device, once: its registers have to cover the
// warpgroups' split (an increase that the launch's registers cannot cover would never
// complete), its shared memory limit is raised.  grid: CTAs to launch.
int attn_ready(int d, bool fp16, int* grid) {
  constexpr int kDevices = 64;
  static std::atomic<int> ctas[4][kDevices];  // 0: not yet
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev >= kDevices) return KVEV_ECUDA;
  std::atomic<int>& ready = ctas[(d == 64 ? 0 : 2) + (fp16 ? 1 : 0)][dev];
  *grid = ready.load(std::memory_order_relaxed);
  if (*grid > 0) return KVEV_OK;
  int sms = 0;
  cudaFuncAttributes a = {};
  const AttnFn fn = attn_fn(d, fp16);
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
      cudaFuncGetAttributes(&a, fn) != cudaSuccess)
    return KVEV_ECUDA;
  if (a.numRegs * kAttnThreads < kRegsAttnNeeded) return KVEV_ENOTSUP;
  if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(attn_smem(d))) != cudaSuccess)
    return KVEV_ECUDA;
  *grid = sms < kMaxCtas ? sms : kMaxCtas;
  ready.store(*grid, std::memory_order_relaxed);  // (two threads at once: the same values)
  return KVEV_OK;
}

bool encode16(CUtensorMap* m, bool fp16, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides,
              const cuuint32_t* box) {
  auto fn = encode_fn();
  if (!fn) return false;
  const cuuint32_t ones[4] = {1, 1, 1, 1};
  return fn(m, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims,
            strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t attn_part_bytes(int d) { return kRows * d * 4 + kRows * sizeof(float2); }

}  // namespace
}  // namespace kvev

using namespace kvev;

extern "C" int kvev_paged_attention_workspace(int H_q, int H_kv, int d, size_t* bytes) {
  if (!bytes || H_kv < 1 || H_q < 1 || H_q % H_kv) return KVEV_EINVAL;
  if ((d != 64 && d != 128) || H_q / H_kv > 128) return KVEV_ENOTSUP;
  static_assert(2 * kMaxCtas * sizeof(int) <= KVEV_PAGED_SYNC_BYTES, "arrival counts");
  *bytes = KVEV_PAGED_SYNC_BYTES + 4 * kMaxCtas * attn_part_bytes(d);
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
  size_t need = 0;
  rc = kvev_paged_attention_workspace(H_q, cache->H_kv, cache->d, &need);
  if (rc != KVEV_OK) return rc;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || !device_status) return KVEV_EINVAL;
  for (int64_t st : {q_token_stride, q_head_stride, out_token_stride, out_head_stride})
    if (st <= 0 || (st & 7)) return KVEV_EINVAL;
  if (B < 0 || T < 0 || T > kMaxTokens || max_pages < 1 || static_cast<int64_t>(max_pages) * cache->page_size > kMaxTokens ||
      window < 0 || !(scale >= 0.f) || !std::isfinite(scale))
    return KVEV_EINVAL;
  if (B > KVEV_PAGED_MAX_REQUESTS) return KVEV_ENOTSUP;
  if (workspace_bytes < need) return KVEV_ENOMEM;
  if (B == 0 || T == 0) return KVEV_OK;
  if (!q || !out || !aligned16(q) || !aligned16(out) || !cu_new || !kv_lens || !block_table ||
      (reinterpret_cast<uintptr_t>(lse) & 3u))
    return KVEV_EINVAL;

  const int d = cache->d;
  const bool fp16 = cache->dtype == KVEV_FP16;
  int grid = 0;
  rc = attn_ready(d, fp16, &grid);
  if (rc != KVEV_OK) return rc;
  PagedAttnParams p = {};
  p.G = H_q / cache->H_kv;
  p.P = kRows / p.G;
  const cuuint64_t du = d;
  {
    const cuuint64_t dims[3] = {du, static_cast<cuuint64_t>(H_q), static_cast<cuuint64_t>(T)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(q_head_stride) * 2, static_cast<cuuint64_t>(q_token_stride) * 2};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(p.G), static_cast<cuuint32_t>(p.P)};
    const cuuint32_t box1[3] = {64, static_cast<cuuint32_t>(p.G), 1};
    if (!encode16(&p.qmap, fp16, q, 3, dims, strides, box) || !encode16(&p.qmap1, fp16, q, 3, dims, strides, box1))
      return KVEV_ECUDA;
  }
  {
    const cuuint64_t dims[4] = {du, static_cast<cuuint64_t>(cache->page_size), static_cast<cuuint64_t>(cache->H_kv),
                                static_cast<cuuint64_t>(cache->num_pages)};
    const cuuint64_t strides[3] = {static_cast<cuuint64_t>(cache->token_stride) * 2, static_cast<cuuint64_t>(cache->head_stride) * 2,
                                   static_cast<cuuint64_t>(cache->page_stride) * 2};
    const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(cache->page_size < kRows ? cache->page_size : kRows), 1, 1};
    if (!encode16(&p.kmap, fp16, cache->K, 4, dims, strides, box) || !encode16(&p.vmap, fp16, cache->V, 4, dims, strides, box))
      return KVEV_ECUDA;
  }
  p.out = static_cast<uint8_t*>(out);
  p.lse = lse;
  p.out_token = out_token_stride * 2;
  p.out_head = out_head_stride * 2;
  p.cu = cu_new;
  p.kv_lens = kv_lens;
  p.table = block_table;
  p.B = B;
  p.T = T;
  p.H_q = H_q;
  p.H_kv = cache->H_kv;
  p.page_shift = view.page_shift;
  p.num_pages = view.num_pages;
  p.max_pages = max_pages;
  p.window = window < static_cast<int64_t>(max_pages) * cache->page_size ? window : 0;  // (a window as long as any sequence is none)
  p.scale_log2 = (scale > 0.f ? scale : 1.f / std::sqrt(static_cast<float>(d))) * 1.4426950408889634f;
  p.status = device_status;
  p.sync = static_cast<int*>(workspace);
  p.parts = static_cast<uint8_t*>(workspace) + KVEV_PAGED_SYNC_BYTES;
  return launch_overlapped(attn_fn(d, fp16), p, grid, kAttnThreads, attn_smem(d), static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? KVEV_OK
             : KVEV_ECUDA;
}
