// Block-causal attention of sequences that share their leading pages.
//
// Row j of sequence s attends to the committed slots [0, len[s]) and to block rows 0..j (or its
// ancestors in a tree block), slots len[s] .. len[s] + j, all on pages of KV_PAGE slots named by the
// page table.  G = H / Hk query heads read the same cache head, so a sequence has q G rows for each
// cache head, and the batch R = b q G.
//
// Softmax is associative: with partial results (m, l, o) of disjoint sets of slots -- row maximum,
// sum of exponentials and weighted sum of values relative to it -- a row's output is
// sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i.  The whole committed pages that all sequences share are
// one set, read once with all R rows against them; the rest of a sequence's slots is another, read
// with its q G rows.  What bounds it are those bytes (K and V once each).
//
// Work: items are (cache head, tile of up to PX_ROWS rows) of the shared pages and (sequence, cache
// head, tile) of the others; units are 128 slots of an item.  The units, items in order, are divided
// among the CTAs (one on an SM) by what they cost; an item's partial results from the CTAs that share it
// are merged by a second kernel, a warp for each row and head.
//
// Per unit, on tcgen05 in the form that puts the slots on the 128 lanes (the rows, often few, are
// the N of the products, so they do not pad to 128):
//   S^T = K Q^T     A = the K tile, B = Q (shared memory, K-major)            128 slots x N rows
//   P^T = exp2(c S^T - m)  one thread for a slot (four groups of 128 threads share the rows)
//   O^T += V^T P^T  A = the V tile read MN-major, B = P (shared memory, MN-major)   hd x N rows
// K and V are the cache's bf16 values.  fp32 queries and the probabilities enter as three bf16 parts
// (24 bits: nothing is lost against fp32 products; one part for bf16 queries, whose probabilities
// have two, 2^-17: the result is rounded to bf16, and 0.2 % of them round to the neighbour of the
// nearest one, as 0.01 to 0.1 % do with fp32 products), one product each into the same fp32 accumulator.
//
// The reference m of a row is its maximum over the first unit; later units only check that no score
// passes it by more than 2^PX_LAZY, which is rare, and then rescale: a maximum over lanes for each
// row and unit would cost more than the exponentials.  Sums of exponentials stay in each thread (a
// slot's) until the end.
//
// The tensor cores cut off what an addition to their fp32 accumulator cannot hold, so that an error of
// half a unit in the last place grows with every 16 slots added.  After PX_RUN units O is therefore
// added, rounded, to a total in TMEM and begun anew (16x4 rows of 7B heads after 16500 slots: an error of
// 0.9e-6; 1.4e-6 and 2 % less time with 8 units, 2.4e-6 and 4 % with 16, 5.9e-6 without; fp32 products
// in a row 2.5e-6).
//
// The three parts are side by side in B (N = three times the rows) and their products in columns of
// their own, added up when they are read: 8 MMAs a tile of K or V instead of 24.  An MMA takes N / 2
// cycles from N = 96 on and 50 below.
//
// Warps: 0 TMA (pages by the table), 1 and 3 MMA issue (a whole warp, one lane's instructions; one warp
// took 1500 cycles for a unit's scores and 1950 for its values beside the busy ones, and bounded all),
// 2 the segments, ahead of their use, 4-19 softmax, 20-23 queries and results, so that a segment's
// queries are in place before the one ahead of it ends and its results leave while the next one runs.
//
// What bounds it: a unit of an SM takes 1.6 us with up to 32 rows when all SMs stream (1.47 at its share of
// the copy rate), 1.9 with 64 (the softmax: 47 % of the issue slots, the rest its chain of loads, votes
// and waits; two halves of the rows in turn, with twice the MMAs to issue, took 2.2).  Beside them the
// starts: 5 us from the launch to the first scores, 0.9 us an item, 2.5 us for the merge.  Measured: 8x6
// rows after 2048 slots of 7B heads 24 us, 16x4 after 16500 91 us (4.4 TB/s).  Registers are what the
// softmax has least of: 44 spilled bytes fewer were worth 4 % to 7 %.
// Shared memory: a ring of K and V tiles, P and Q in three parts; TMEM: S and two O.
#include "common.cuh"
#include "internal.h"
#include "prefix_scratch.h"

namespace sdsat {
namespace {

constexpr int PX_UNIT = 128;      // slots of a unit: two pages
constexpr int PX_PARTS = 3;       // bf16 parts of fp32 queries and of their probabilities
constexpr int PX_GROUPS = 4;      // softmax groups of 128 threads
constexpr int PX_SOFTMAX = 128 * PX_GROUPS;
constexpr int PX_SOFTMAX_WARPS = PX_SOFTMAX / 32;
constexpr int PX_THREADS = 128 + PX_SOFTMAX + 128;
constexpr int PX_MINE = PX_ROWS / 8 / PX_GROUPS;   // pieces of eight rows of a thread
constexpr int PX_SEGS = 4;        // segments described ahead
constexpr int PX_O = PX_PARTS * PX_ROWS;   // TMEM column of O (S from 0 on)
constexpr int PX_O_STEP = 160;    // to the second O, for segments of at most PX_TWICE rows
constexpr int PX_TWICE = 32;      // rows of segments whose queries, and whose O, fit twice
constexpr int PX_TOTAL = 448;     // TMEM column of the total that O is added to
constexpr int PX_RUN = 4;         // units that O takes before it is added to the total
static_assert(PX_O + PX_O_STEP + PX_PARTS * PX_TWICE <= PX_TOTAL && PX_O + PX_PARTS * PX_ROWS <= PX_TOTAL, "columns");
constexpr int PX_MAX_B = 64;
constexpr float PX_LAZY = 8.0f;   // log2 of the growth of a row maximum that is left unscaled
constexpr float PX_UNSET = -1e30f;   // reference of a row that has seen no slot
static_assert(PX_UNIT == 2 * KV_PAGE, "a unit is two pages");

template <int HD>
struct PxCfg {
  static constexpr int HALVES = HD / 64;
  static constexpr int BOX = KV_PAGE * 128;                 // one TMA box: a page's slots x 64 dims
  static constexpr int HALF = PX_UNIT * 128;                // 128 slots x 64 dims, 128-byte swizzle
  static constexpr int TILE = HALVES * HALF;                // K or V of a unit
  static constexpr int SLOTS = HD == 128 ? 4 : 8;           // of the ring
  static constexpr int P_PART = PX_UNIT * 128;              // 128 slots x 64 rows
  static constexpr int Q_HALF = PX_PARTS * PX_ROWS * 128;   // 3 x 64 rows x 64 dims
  static constexpr int Q_SECOND = PX_PARTS * PX_TWICE * 128;   // where a second segment's queries start
  static constexpr size_t OFF_P = (size_t)SLOTS * TILE;     // (MN-major reads of 64-dim tiles run into it)
  static constexpr size_t OFF_Q = OFF_P + PX_PARTS * P_PART;
  static constexpr size_t OFF_MISC = OFF_Q + HALVES * Q_HALF;
};

// What the CTAs, and the merge after them, agree on.  Shares are counted in places: those of an item are
// some for its start and then some for each of its units, which belongs to the CTA that has its first one.
struct PxCost {
  int start, unit;
};
struct PxSched {
  int shared;              // pages that all sequences share, whole and committed
  int q, r;                // places of a CTA's share; the first r CTAs have one more
  int tp;                  // places of the items of the shared pages
  int units;               // units of one of them
  PxCost cost[2];          // of the items of the shared pages, of the others
  int cum[PX_MAX_B + 1];   // places of the items of the sequences before
  __device__ int begin(int c) const { return c * q + min(c, r); }
  __device__ int places(int k, int units) const { return units > 0 ? cost[k].start + units * cost[k].unit : 0; }
};
// What an item of that many rows costs, a unit of up to 32 rows being 4 (1.2 us): units of more rows 2 us
// (1.65 of 16 bits); starts 0.9 us, with more rows, whose queries and O have no second place, 4.5 us beside
// the stream of K and V (3). By the ends of the CTAs of four cases and the times of sets of these numbers;
// with shares of as many units each they are up to 20 % longer, with starts of 8 up to 8 %.  All four have
// heads of 128: those of 64, whose units are half the bytes, take the same numbers and were not measured.
__device__ __forceinline__ PxCost px_cost(int rows, bool bf16) {
  return rows > 32 ? PxCost{bf16 ? 10 : 14, bf16 ? 5 : 6} : PxCost{3, 4};
}
// n / d for n d < 2^32 (rows and heads by a cache head's query heads: checked by the caller), inv = px_inv(d)
__device__ __forceinline__ int px_div(int n, uint32_t inv) { return inv ? (int)__umulhi((uint32_t)n, inv) : n; }
// n / d for 0 <= n < 1.9e9, quotients below 2^30 (the first one is off by 2^-21 of itself at most, the
// second one's operand is exact): a third of the instructions, which are fetched cold here
__device__ __forceinline__ int px_quot(int n, int d) {
  const float inv = __fdividef(1.0f, (float)d);
  int q = __float2int_rz((float)n * inv), r = n - q * d;
  const int more = __float2int_rd((float)r * inv);
  q += more;
  r -= more * d;
  return q + (r >= d) - (r < 0);
}
__device__ __forceinline__ int px_owner(int g, int q, int r) {   // the CTA that has place g
  const int x = g - (q + 1) * r;
  return x < 0 ? px_quot(g, q + 1) : r + px_quot(x, q);
}
// ... from the lengths, by a warp; `end`: the places up to the sequences 2 lane and 2 lane + 1 and theirs,
// `len` their lengths
struct PxPlan {
  int shared, q, r, tp, units, end[2], len[2];
  PxCost cost[2];
};
// units of a sequence of n committed slots beyond the shared pages
__device__ __forceinline__ int px_units(const PrefixAttnParams& p, int n, int shared) {
  return max(0, (min(n + p.nq, p.ld * KV_PAGE) - shared * KV_PAGE + PX_UNIT - 1) / PX_UNIT);
}
__device__ PxPlan px_plan(const PrefixAttnParams& p, int ctas, int lane) {
  PxPlan a;
  const int s0 = 2 * lane, s1 = s0 + 1;
  a.len[0] = s0 < p.b ? max(0, __ldcg(p.len + s0)) : 0;
  a.len[1] = s1 < p.b ? max(0, __ldcg(p.len + s1)) : 0;
  a.shared = 0;
  if (p.common && p.b > 1) {
    a.shared = p.ld;
    if (s0 < p.b) a.shared = min(a.shared, min(__ldcg(p.common + s0), a.len[0] / KV_PAGE));
    if (s1 < p.b) a.shared = min(a.shared, min(__ldcg(p.common + s1), a.len[1] / KV_PAGE));
    a.shared = max(0, __reduce_min_sync(0xffffffffu, a.shared));
  }
  const int per = p.Hk * p.tiles[1].n, first = p.Hk * p.tiles[0].n;
  auto units = [&](int n) { return px_units(p, n, a.shared); };
  a.units = (a.shared + 1) / 2;
  const int units0 = s0 < p.b ? units(a.len[0]) : 0, units1 = s1 < p.b ? units(a.len[1]) : 0;
  const int all = first * a.units + per * (int)__reduce_add_sync(0xffffffffu, (unsigned)(units0 + units1));
  // With few units they are the places (a CTA's share has to hold the places of any unit, or some CTA
  // within an item would have none of its units), and with very many, for the places' range.
  const bool weighed = all > 2 * ctas && all < 1 << 26;
#pragma unroll
  for (int k = 0; k < 2; ++k) a.cost[k] = weighed ? px_cost(p.tiles[k].rows, p.bf16) : PxCost{0, 1};
  auto places = [&](int k, int units) { return units > 0 ? a.cost[k].start + units * a.cost[k].unit : 0; };
  const int u1 = per * places(1, units1);
  int x = per * places(1, units0) + u1;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  a.end[0] = x - u1;
  a.end[1] = x;
  a.tp = first * places(0, a.units);
  const int total = a.tp + __shfl_sync(0xffffffffu, x, 31);
  a.q = px_quot(total, ctas);
  a.r = total - a.q * ctas;
  return a;
}
// a CTA's units of one item
struct PxSeg {
  int s;                   // sequence, or -1: the shared pages
  int hk, row0, rows;      // cache head, rows [row0, row0 + rows) of its R
  int u0, u1;              // units; none: the share has ended
  int slot0, end, len;     // unit u: slots slot0 + 128 u .., those below `end`; committed below len
  int q_at;                // 0 or 1: which half of the queries' space
  int whole;               // it takes the whole space of queries and O, or the segment before does
  __device__ int cols() const { return (rows + 15) / 16 * 16; }
};
struct PxMisc {
  PxSched sched;
  int len[PX_MAX_B];
  uint32_t top[3][PX_ROWS];   // a row's maximum over the unit, as px_order
  __align__(16) float minus_m[PX_ROWS];   // the rows' references, negative
  float by[PX_ROWS];       // the rescaling of what is there
  __align__(16) uint16_t seen[PX_SEGS][PX_ROWS];     // the block rows that a row sees
  PxSeg seg[PX_SEGS];
  uint64_t full[8], empty[8];
  uint64_t seg_full[PX_SEGS], seg_empty[PX_SEGS];
  // [2]: by segment parity.  A phase of a barrier is waited for before the one after it can
  // end: with one barrier for every segment the queries of two segments ahead would end two phases.
  uint64_t q_full[2], q_empty[2], o_full[2], o_empty[2], s_full, s_empty, p_full, p_empty, drain[2];
  uint32_t tmem;
  volatile int abort;
  uint32_t pages_ok[8];    // by unit: its pages are in the pool (bits 0, 1)
};

// the segment that starts at place g and ends at the item's end or at gend, where g goes (it may have no
// units); `near`: no later sequence than its own
__device__ PxSeg px_segment(const PrefixAttnParams& p, const PxSched& sc, const int* len, int& g, int gend, int& near) {
  const int k = g < sc.tp ? 0 : 1;
  const PxTiles& t = p.tiles[k];
  PxSeg e{};
  int x = g, places = sc.places(0, sc.units), units = sc.units;
  if (k) {
    x -= sc.tp;
#pragma unroll 1
    while (sc.cum[near + 1] <= x) ++near;
    x -= sc.cum[near];
    units = px_units(p, len[near], sc.shared);
    places = sc.places(1, units);
  }
  const int item = px_quot(x, places), at = x - item * places, n = min(places - at, gend - g);
  e.hk = px_quot(item, t.n);
  const int rt = item - e.hk * t.n;
  if (k) {
    e.s = near;
    e.row0 = near * p.nq * p.G + rt * t.rows;
    e.rows = min(t.rows, p.nq * p.G - rt * t.rows);
    e.slot0 = sc.shared * KV_PAGE;
    e.len = len[near];
    e.end = min(e.len + p.nq, p.ld * KV_PAGE);
  } else {
    e.s = -1;
    e.row0 = rt * t.rows;
    e.rows = min(t.rows, p.b * p.nq * p.G - e.row0);
    e.end = e.len = sc.shared * KV_PAGE;
  }
  const PxCost c = sc.cost[k];
  auto unit = [&](int place) { return min(units, px_quot(max(0, place - c.start) + c.unit - 1, c.unit)); };   // the first one from there on
  e.u0 = unit(at);
  e.u1 = unit(at + n);
  g += n;
  return e;
}

__device__ __forceinline__ void px_ld8(uint32_t taddr, float* v) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void px_ld4(uint32_t taddr, float* v) {
  uint32_t r[4];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(taddr)
               : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void px_st4(uint32_t taddr, const float* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(__float_as_uint(v[0])),
               "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3]))
               : "memory");
}
__device__ __forceinline__ void px_st8(uint32_t taddr, const float* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
               "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])),
               "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])),
               "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7]))
               : "memory");
}
// MN-major operand in the 128-byte swizzle layout: atoms of 64 elements (128 bytes) x 8 lines of K;
// `lead` bytes to the next 64 elements, 1024 to the next 8 lines
__device__ __forceinline__ uint64_t px_desc_mn(uint32_t saddr, uint32_t lead) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(lead >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}
// one lane's MMA in a converged warp (mine: 1 in that lane)
__device__ __forceinline__ void px_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t mine) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(mine)
      : "memory");
}
__device__ __forceinline__ uint32_t px_elect() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r));
  return r;
}
__device__ __forceinline__ float px_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// two values as packed bf16; what is left of them stays in v
__device__ __forceinline__ uint32_t px_part(uint64_t& v) {
  float a, b;
  f2_unpack(v, a, b);
  uint32_t h;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(b), "f"(a));
  v = f2_sub(v, f2_pack(__uint_as_float(h << 16), __uint_as_float(h & 0xFFFF0000u)));
  return h;
}
__device__ __forceinline__ bool px_bar_or(int id, bool pred) {   // over a group's 128 threads
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %1, 0;\n\t"
      "barrier.cta.red.or.pred p, %2, 128, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)pred), "r"(id)
      : "memory");
  return r != 0;
}
// Waits for the phase of `bar` with this parity: WAIT_LIMIT_NS at most, after which it raises
// ERR_TIMEOUT and sets *abort, which ends every other wait of the CTA.  (A few instructions: the kernel
// has some thirty waits, and its code has to stay near the instruction caches' 32 KB.)
__device__ __noinline__ void px_wait_on(uint64_t* bar, uint32_t parity, volatile int* abort, uint32_t* err) {
  const uint64_t t0 = globaltimer_ns();
#pragma unroll 1
  while (!mbar_try_wait(bar, parity)) {
    if (*abort || globaltimer_ns() - t0 > WAIT_LIMIT_NS) {
      *abort = 1;
      set_error(err, ERR_TIMEOUT);
      return;
    }
  }
}
__device__ __forceinline__ void px_wait(uint64_t* bar, uint32_t parity, volatile int* abort, uint32_t* err) {
  if (!mbar_try_wait(bar, parity)) px_wait_on(bar, parity, abort, err);
}
// floats as whole numbers of the same order, all of them above 0
__device__ __forceinline__ uint32_t px_order(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float px_unorder(uint32_t u) {
  return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ float px_warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// Eight columns of a value a lane each -> in every lane, column (lane & 7) over the warp's 32 lanes
template <typename F>
__device__ __forceinline__ float px_across(const float* v, int lane, F&& f) {
  float a[4], b[2], c;
  const bool h4 = lane & 4, h2 = lane & 2, h1 = lane & 1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float keep = h4 ? v[i + 4] : v[i], give = h4 ? v[i] : v[i + 4];
    a[i] = f(keep, __shfl_xor_sync(0xffffffffu, give, 4));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float keep = h2 ? a[i + 2] : a[i], give = h2 ? a[i] : a[i + 2];
    b[i] = f(keep, __shfl_xor_sync(0xffffffffu, give, 2));
  }
  c = f(h1 ? b[1] : b[0], __shfl_xor_sync(0xffffffffu, h1 ? b[0] : b[1], 1));
  c = f(c, __shfl_xor_sync(0xffffffffu, c, 8));
  return f(c, __shfl_xor_sync(0xffffffffu, c, 16));
}

// where partial results are: of an item's rows from the CTA that holds its first unit, and, for each
// CTA, from the item that it continues
struct PxScratch {
  float* o;        // [2 * row heads + PX_ROWS * CTAs][hd]
  float* m;        // the same rows' references
  float4* l;       // and sums, in four parts
  __device__ PxScratch(const PrefixAttnParams& p) {
    const size_t n = px_scratch_rows((size_t)p.b * p.nq * p.H, p.ctas);
    l = reinterpret_cast<float4*>(p.part);
    m = p.part + 4 * n;
    o = m + n;
  }
};

// a segment's queries (thread i of n) into shared memory, rows past its own as zeros; the loads of
// two pieces of eight dimensions are in flight together
template <int HD>
__device__ __noinline__ void px_queries(const PrefixAttnParams& p, PxMisc& sm, uint8_t* Qs, const PxSeg& x, int seg, int i0, int n) {
  using C = PxCfg<HD>;
  const int G = p.G, cols = x.cols(), total = cols * (HD / 8);
  if (i0 < cols && x.s >= 0) {
    const int tr = px_div(x.row0 + i0, p.inv_g);   // token row
    sm.seen[seg % PX_SEGS][i0] = (uint16_t)(i0 >= x.rows ? 0u : p.anc ? __ldcg(p.anc + tr) : (2u << (tr - px_div(tr, p.inv_nq) * p.nq)) - 1u);
  }
  uint8_t* base = Qs + x.q_at * C::Q_SECOND;
#pragma unroll 1
  for (int i = i0; i < total; i += 2 * n) {
    uint4 w[2], w1[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int r = (i + z * n) / (HD / 8), d = (i + z * n) % (HD / 8);
      w[z] = w1[z] = make_uint4(0, 0, 0, 0);
      if (r < x.rows) {
        const int rr = x.row0 + r, tr = px_div(rr, p.inv_g);
        const long long at = (long long)tr * p.q_ld + (long long)(x.hk * G + (rr - tr * G)) * HD + d * 8;
        if (p.bf16) {
          w[z] = __ldcg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + at));
        } else {
          const uint4* src = reinterpret_cast<const uint4*>(static_cast<const float*>(p.q) + at);
          w[z] = __ldcg(src);
          w1[z] = __ldcg(src + 1);
        }
      }
    }
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int r = (i + z * n) / (HD / 8), d = (i + z * n) % (HD / 8);
      if (i + z * n >= total) break;
      uint8_t* dst = base + (d >> 3) * C::Q_HALF + r * 128 + (((d & 7) ^ (r & 7)) << 4);
      if (p.bf16) {
        *reinterpret_cast<uint4*>(dst) = w[z];
        continue;
      }
      uint64_t v[4] = {(uint64_t)w[z].y << 32 | w[z].x, (uint64_t)w[z].w << 32 | w[z].z, (uint64_t)w1[z].y << 32 | w1[z].x,
                       (uint64_t)w1[z].w << 32 | w1[z].z};
#pragma unroll
      for (int part = 0; part < PX_PARTS; ++part) {
        uint4 o;
        o.x = px_part(v[0]);
        o.y = px_part(v[1]);
        o.z = px_part(v[2]);
        o.w = px_part(v[3]);
        *reinterpret_cast<uint4*>(dst + part * cols * 128) = o;
      }
    }
  }
}
template <int HD>
__global__ void __launch_bounds__(PX_THREADS, 1) prefix_attention_kernel(const __grid_constant__ PrefixAttnParams p) {
  using C = PxCfg<HD>;
  constexpr int NS = C::SLOTS;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* Ps = smem + C::OFF_P;
  uint8_t* Qs = smem + C::OFF_Q;
  PxMisc& sm = *reinterpret_cast<PxMisc*>(smem + C::OFF_MISC);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int R = p.b * p.nq * p.G;
  if (tid == 0) {
#pragma unroll 1
    for (int i = 0; i < NS; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], 1);
    }
#pragma unroll 1
    for (int i = 0; i < PX_SEGS; ++i) {
      mbar_init(&sm.seg_full[i], 1);
      mbar_init(&sm.seg_empty[i], 3 + PX_SOFTMAX_WARPS + 4);   // TMA, MMA, softmax, queries and results
    }
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.q_full[i], 4);
      mbar_init(&sm.q_empty[i], 1);
      mbar_init(&sm.o_full[i], 1);
      mbar_init(&sm.o_empty[i], 4);
    }
    mbar_init(&sm.s_full, 1);
    mbar_init(&sm.s_empty, PX_SOFTMAX_WARPS);
    mbar_init(&sm.p_full, PX_SOFTMAX_WARPS);
    mbar_init(&sm.p_empty, 1);
    mbar_init(&sm.drain[0], 1);
    mbar_init(&sm.drain[1], 1);
    sm.abort = 0;
    fence_mbar_init();
    tma_prefetch_desc(&p.kmap);
    tma_prefetch_desc(&p.vmap);
  }
  if (warp == 1) tmem_alloc(&sm.tmem, 512);
  if (tid < PX_ROWS) sm.top[0][tid] = 0;
  pdl_wait();   // q, lengths, tables and rows come from the kernels before
  pdl_trigger();
  if (warp >= 4) {
    // All queries on their way to L2, a line a thread, before they are loaded: from memory that takes
    // 0.8 us, and 2 us beside the stream of K and V.
    const int lines = p.H * HD * (p.bf16 ? 2 : 4) / 128, z = (tid - 128) * gridDim.x + blockIdx.x, r = px_quot(z, lines);
    if (r < p.b * p.nq) {
      const char* at = static_cast<const char*>(p.q) + r * p.q_ld * (p.bf16 ? 2 : 4) + (z - r * lines) * 128;
      asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
    }
  }
  if (warp == 2) {
    const PxPlan a = px_plan(p, gridDim.x, lane);
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      sm.len[2 * lane + z] = a.len[z];
      sm.sched.cum[2 * lane + z + 1] = a.end[z];
    }
    if (lane == 0) {
      sm.sched.cum[0] = 0;
      sm.sched.shared = a.shared;
      sm.sched.units = a.units;
      sm.sched.tp = a.tp;
      sm.sched.q = a.q;
      sm.sched.r = a.r;
      sm.sched.cost[0] = a.cost[0];
      sm.sched.cost[1] = a.cost[1];
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  const int q_parts = p.bf16 ? 1 : PX_PARTS, p_parts = p.bf16 ? 2 : PX_PARTS;
  // Every role goes through every segment, unit, wait and barrier of the share, whatever the waits
  // return: one that ran out has set the error bit, and the results are invalid.
  auto wait = [&](uint64_t* bar, uint32_t parity) { px_wait(bar, parity, &sm.abort, p.err); };
  // the i-th segment's description (in place until each role has arrived at seg_empty, all lanes of its warps
  // having read it: `arrive`)
  auto segment = [&](int i) -> const PxSeg& {
    wait(&sm.seg_full[i % PX_SEGS], (i / PX_SEGS) & 1);
    return sm.seg[i % PX_SEGS];
  };

  // where a segment's results go: the rows of an item from its first unit on, or those of the CTA's
  // first segment, which continues one
  auto scratch_row = [&](const PxSeg& x) {
    return x.u0 > 0 ? (size_t)2 * p.b * p.nq * p.H + (size_t)PX_ROWS * blockIdx.x
                    : (size_t)(x.s < 0 ? 0 : p.b * p.nq * p.H) + (size_t)x.hk * R + x.row0;
  };

  // a warp's arrival, after what its lanes did before
  auto arrive = [&](uint64_t* bar) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
  };
  // the first segment's, which everything waits for: by warps 4 to 23
  auto first_queries = [&](int i) {
    const PxSeg& x = segment(0);
    if (x.u0 == x.u1) return;
    px_queries<HD>(p, sm, Qs, x, 0, i, PX_SOFTMAX + 128);
    fence_proxy_async_smem();
    named_bar_sync(1 + PX_GROUPS, PX_SOFTMAX + 128);
  };

  if (warp >= 4) first_queries(tid - 128);

  if (warp == 2) {
    // ---- the segments
    if (lane == 0) {
      const int g1 = sm.sched.begin(blockIdx.x + 1);
      int near = 0, rows = 0, q_at = 1;
#pragma unroll 1
      for (int i = 0, g = sm.sched.begin(blockIdx.x);; ++i) {
        PxSeg e{};
        while (g < g1 && e.u0 == e.u1) e = px_segment(p, sm.sched, sm.len, g, g1, near);
        e.q_at = q_at = e.rows <= PX_TWICE ? q_at ^ 1 : 0;
        e.whole = max(rows, e.rows) > PX_TWICE;
        rows = e.rows;
        wait(&sm.seg_empty[i % PX_SEGS], ((i / PX_SEGS) & 1) ^ 1);
        sm.seg[i % PX_SEGS] = e;
        mbar_arrive(&sm.seg_full[i % PX_SEGS]);
        if (e.u0 == e.u1) break;
      }
    }
  } else if (warp == 0) {
    // ---- K and V tiles: K of unit 0, V of unit 0, K of unit 1, ...
    const uint64_t pol = l2_policy_evict_normal();
    int it = 0;
#pragma unroll 1
    for (int seg = 0;; ++seg) {
      const PxSeg e = segment(seg);
      arrive(&sm.seg_empty[seg % PX_SEGS]);
      if (e.u0 == e.u1) break;
      const int* row = p.table + (size_t)max(e.s, 0) * p.ld;
      const int j0 = e.slot0 / KV_PAGE + 2 * e.u0, j1 = min((e.end + KV_PAGE - 1) / KV_PAGE, e.slot0 / KV_PAGE + 2 * e.u1);
      int entry = 0;
#pragma unroll 1
      for (int u = e.u0; u < e.u1; ++u) {
        const int at = 2 * (u - e.u0), j = j0 + at;
        if ((at & 31) == 0) entry = j + lane < j1 ? __ldcg(row + j + lane) : 0;
        const int page[2] = {__shfl_sync(0xffffffffu, entry, at & 31), __shfl_sync(0xffffffffu, entry, (at & 31) + 1)};
        uint32_t ok = 0;
        for (int i = 0; i < 2; ++i)
          if (j + i < j1) {
            if (page[i] >= 0 && page[i] < p.n_pages) ok |= 1u << i;
            else if (lane == 0) set_error(p.err, ERR_PAGE);
          }
        if (lane == 0 && !sm.abort) {
#pragma unroll 1
          for (int kv = 0; kv < 2; ++kv, ++it) {
            const int s = it % NS;
            wait(&sm.empty[s], ((it / NS) & 1) ^ 1);
            if (sm.abort) break;
            // (read until the unit's V slot is free again, 2 or 4 units on)
            sm.pages_ok[(it >> 1) & 7] = ok;
            mbar_arrive_expect_tx(&sm.full[s], __popc(ok) * C::HALVES * C::BOX);
#pragma unroll 1
            for (int i = 0; i < 2; ++i) {
              if (!((ok >> i) & 1)) continue;
              const int r = p.row0 + (page[i] * p.Hk + e.hk) * KV_PAGE;
#pragma unroll 1
              for (int hh = 0; hh < C::HALVES; ++hh)
                tma_load_2d(smem + (size_t)s * C::TILE + hh * C::HALF + i * C::BOX, kv ? &p.vmap : &p.kmap, &sm.full[s], hh * 64,
                            r, pol);
            }
          }
        }
        __syncwarp();
      }
    }
    if (lane == 0 && sm.abort) {   // let the copies in flight land before the CTA exits
#pragma unroll 1
      for (int i = max(0, it - NS); i < it; ++i) {
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait(&sm.full[i % NS], (i / NS) & 1))
          if (globaltimer_ns() - t0 > WAIT_LIMIT_NS) break;
      }
    }
  } else if (warp == 1 || warp == 3) {
    // ---- products: scores on one warp, values on the other; nothing is issued any more once a wait
    // has run out
    const uint32_t mine = px_elect();
    auto ready = [&](uint64_t* bar, uint32_t parity) {
      wait(bar, parity);
      __syncwarp();
      tc_fence_after();
    };
    auto commit = [&](uint64_t* bar) {
      if (mine) umma_commit(bar);
      __syncwarp();
    };
    int k = 0;   // unit of the share
    if (warp == 1) {
      const uint64_t kd = sdesc_sw128(smem_u32(smem)), qd = sdesc_sw128(smem_u32(Qs));
#pragma unroll 1
      for (int seg = 0;; ++seg) {
        const PxSeg& e = segment(seg);
        if (e.u0 == e.u1) break;
        const uint32_t idesc = idesc_bf16_f32(128, q_parts * e.cols());
        const uint64_t b0 = qd + (uint64_t)(e.q_at * (C::Q_SECOND >> 4));
        ready(&sm.q_full[seg & 1], (seg >> 1) & 1);
#pragma unroll 1
        for (int u = e.u0; u < e.u1; ++u, ++k) {
          const int slot = (2 * k) % NS;
          wait(&sm.full[slot], ((2 * k) / NS) & 1);
          if (k > 0) wait(&sm.s_empty, (k - 1) & 1);
          __syncwarp();
          tc_fence_after();
          const uint64_t a0 = kd + (uint64_t)(slot * (C::TILE >> 4));
          if (!sm.abort) {
#pragma unroll 1
            for (int kk = 0; kk < HD / 16; ++kk)
              px_mma(tmem, a0 + ((kk >> 2) * (C::HALF >> 4) + (kk & 3) * 2), b0 + ((kk >> 2) * (C::Q_HALF >> 4) + (kk & 3) * 2), idesc,
                     kk ? 1u : 0u, mine);
          }
          commit(&sm.s_full);
          commit(&sm.empty[slot]);
        }
        commit(&sm.q_empty[seg & 1]);
        arrive(&sm.seg_empty[seg % PX_SEGS]);
      }
    } else {
      const uint64_t vd = px_desc_mn(smem_u32(smem), C::HALF), pd = px_desc_mn(smem_u32(Ps), C::P_PART);
      int run = 0;
#pragma unroll 1
      for (int seg = 0;; ++seg) {
        const PxSeg& e = segment(seg);
        if (e.u0 == e.u1) break;
        const uint32_t idesc = idesc_bf16_f32(128, p_parts * e.cols()) | (1u << 15) | (1u << 16);   // both MN-major
        uint32_t o = 0;
#pragma unroll 1
        for (int u = e.u0; u < e.u1; ++u, ++k) {
          const int in_run = (u - e.u0) % PX_RUN;
          if (in_run == 0) {   // O: the last or the last but one run has been read
            o = tmem + PX_O + (e.rows <= PX_TWICE ? PX_O_STEP * (run & 1) : 0);
            const int before = run - (e.rows > PX_TWICE || (u == e.u0 && e.whole) ? 1 : 2);
            if (before >= 0) ready(&sm.o_empty[before & 1], (before >> 1) & 1);
          }
          const int slot = (2 * k + 1) % NS, steps = (min(PX_UNIT, e.end - e.slot0 - u * PX_UNIT) + 15) / 16;   // 16 slots each
          const uint64_t a0 = vd + (uint64_t)(slot * (C::TILE >> 4));
          wait(&sm.full[slot], ((2 * k + 1) / NS) & 1);
          ready(&sm.p_full, k & 1);
          if (!sm.abort) {
#pragma unroll 1
            for (int kk = 0; kk < steps; ++kk) px_mma(o, a0 + kk * 128, pd + kk * 128, idesc, in_run || kk ? 1u : 0u, mine);
          }
          commit(&sm.p_empty);
          commit(&sm.empty[slot]);
          if (in_run == PX_RUN - 1 || u + 1 == e.u1) {
            commit(&sm.o_full[run & 1]);
            ++run;
          }
        }
        arrive(&sm.seg_empty[seg % PX_SEGS]);
      }
    }
    if (sm.abort) {   // wait for issued MMAs before shared memory goes away
      uint64_t* const drain = &sm.drain[warp >> 1];
      commit(drain);
      if (lane == 0) {
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait(drain, 0))
          if (globaltimer_ns() - t0 > WAIT_LIMIT_NS) break;
      }
    }
  } else if (warp >= 4 + PX_SOFTMAX_WARPS) {
    // ---- queries in and results out.  A segment's queries come when the scores of the one before the
    // last are done, which frees their space, or, where they need all of it, of the last one.
    const int st = tid - 128 - PX_SOFTMAX;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    auto queries = [&](int j) {   // of segment j, once those of segment j - (whole ? 1 : 2) are done with
      const PxSeg& y = sm.seg[j % PX_SEGS];
      const int before = j - (y.whole ? 1 : 2);
      if (before >= 0) wait(&sm.q_empty[before & 1], (before >> 1) & 1);
      px_queries<HD>(p, sm, Qs, y, j, st, 128);
      fence_proxy_async_smem();
      arrive(&sm.q_full[j & 1]);
    };
    if (sm.seg[0].u0 < sm.seg[0].u1) arrive(&sm.q_full[0]);   // (in place: first_queries)
    int run = 0;
#pragma unroll 1
    for (int seg = 0, j = 1; segment(seg).u0 < segment(seg).u1; ++seg) {
      const PxSeg& x = sm.seg[seg % PX_SEGS];
      const int cols = x.cols();
      const size_t row = scratch_row(x);
#pragma unroll 1
      for (int u = x.u0; u < x.u1; u += PX_RUN, ++run) {
        const bool more = u + PX_RUN < x.u1;
        if (!more) {   // (the scores of the segment's last units need what its runs before have left)
#pragma unroll 1
          for (; j <= seg + 2; ++j) {
            const PxSeg& y = segment(j);
            if (y.u0 == y.u1 || (j == seg + 2 && y.whole)) break;
            queries(j);
          }
        }
        wait(&sm.o_full[run & 1], (run >> 1) & 1);
        __syncwarp();
        tc_fence_after();
#pragma unroll 1
        for (int r = 0; r < x.rows; r += 8) {
          float o[8], o1[8], o2[8];
          const uint32_t at = tmem + lanes + PX_O + (x.rows <= PX_TWICE ? PX_O_STEP * (run & 1) : 0) + r, total = tmem + lanes + PX_TOTAL + r;
          px_ld8(at, o);
          px_ld8(at + cols, o1);
          if (p_parts > 2) px_ld8(at + 2 * cols, o2);
          tmem_wait_ld();
#pragma unroll
          for (int z = 0; z < 8; ++z) {
            o[z] += o1[z];
            if (p_parts > 2) o[z] += o2[z];
          }
          if (u > x.u0) {
            px_ld8(total, o1);
            tmem_wait_ld();
#pragma unroll
            for (int z = 0; z < 8; ++z) o[z] += o1[z];
          }
          if (more) {
            px_st8(total, o);
            continue;
          }
          float* dst = PxScratch(p).o + (row + r) * HD + st;
#pragma unroll
          for (int z = 0; z < 8; ++z)
            if (r + z < x.rows && st < HD) dst[z * HD] = o[z];
        }
        if (more) asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        arrive(&sm.o_empty[run & 1]);
      }
      arrive(&sm.seg_empty[seg % PX_SEGS]);
    }
  } else {
    const int wg = (warp >> 2) - 1, e = tid & 127;   // softmax thread, group, slot of the unit
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    constexpr float c = (HD == 64 ? 0.125f : 0.08838834764831845f) * 1.4426950408889634f;
    const uint64_t c2 = f2_pack(c, c);
    auto ready = [&](uint64_t* bar, uint32_t parity) {
      wait(bar, parity);
      __syncwarp();
      tc_fence_after();
    };
    int k = 0, moves = 0, run0 = 0;   // units, new references, runs of the segments before
    float m_mine = 0.f;     // the reference of the lane's row
    float l[8 * PX_MINE];   // the rows' sums of this thread's slots
#pragma unroll 1
    for (int seg = 0;; ++seg) {
      const PxSeg& x = segment(seg);
      if (x.u0 == x.u1) break;
      // this group's pieces of eight rows: wg and wg + 4 of them, as far as there are rows
      const int cols = x.cols(), mine = (cols / 8 - wg + PX_GROUPS - 1) / PX_GROUPS;
      auto first_row = [&](int i) { return 8 * (wg + PX_GROUPS * i); };
      const uint16_t* seen = sm.seen[seg % PX_SEGS];
#pragma unroll
      for (int i = 0; i < 8 * PX_MINE; ++i) l[i] = 0.f;
      // the row that the lane looks after in its warp: 8 of the first piece, 8 of the second
      const int my_row = lane < 8 * mine ? first_row(lane >> 3) + (lane & 7) : 0;
#pragma unroll 1
      for (int u = x.u0; u < x.u1; ++u, ++k) {
        const int slot = x.slot0 + u * PX_UNIT + e;
        ready(&sm.s_full, k & 1);   // (the queries, and what the rows see, were there before)
        float s[8 * PX_MINE];
#pragma unroll
        for (int i = 0; i < PX_MINE; ++i)
          if (i < mine) {
            const uint32_t at = tmem + lanes + first_row(i);
            float a[8];   // the second and third parts' products
            px_ld8(at, s + 8 * i);
            if (q_parts > 1) px_ld8(at + cols, a);
            tmem_wait_ld();
            if (q_parts > 1) {
#pragma unroll
              for (int z = 0; z < 8; z += 2)
                f2_unpack(f2_add(f2_pack(s[8 * i + z], s[8 * i + z + 1]), f2_pack(a[z], a[z + 1])), s[8 * i + z], s[8 * i + z + 1]);
              px_ld8(at + 2 * cols, a);
              tmem_wait_ld();
#pragma unroll
              for (int z = 0; z < 8; z += 2)
                f2_unpack(f2_add(f2_pack(s[8 * i + z], s[8 * i + z + 1]), f2_pack(a[z], a[z + 1])), s[8 * i + z], s[8 * i + z + 1]);
            }
          }
        tc_fence_before();
        arrive(&sm.s_empty);
        // the slot is seen by every row (committed), by some (a block row's) or by none
        const uint32_t ok = sm.pages_ok[k & 7];
        const bool here = slot < x.end && ((ok >> (e >> 6)) & 1);
        if (x.slot0 + (u + 1) * PX_UNIT > x.len || ok != 3u) {
          const int i0 = slot - x.len;
          const uint32_t all = here && i0 < 0 ? 0xFFFFu : 0u, bit = here && i0 >= 0 ? 1u << i0 : 0u;
#pragma unroll
          for (int i = 0; i < PX_MINE; ++i)
            if (i < mine) {
              const uint4 w = *reinterpret_cast<const uint4*>(seen + first_row(i));   // eight rows'
#pragma unroll
              for (int z = 0; z < 8; ++z) {
                const uint32_t bits = ((&w.x)[z >> 1] >> (16 * (z & 1))) & bit;
                if (!(bits | all)) s[8 * i + z] = -INFINITY;
              }
            }
        }
        // the rows' references: the first unit's maxima, and new ones where a score passes them by far
        const bool first = u == x.u0;
        bool move = first;
        if (!first) {
          float top = -INFINITY;
#pragma unroll
          for (int i = 0; i < 8 * PX_MINE; i += 4)
            if (i < 8 * mine) {
              const ulonglong2 m = *reinterpret_cast<const ulonglong2*>(&sm.minus_m[first_row(i >> 3) + (i & 4)]);
              float a, b;
              f2_unpack(f2_fma(f2_pack(s[i], s[i + 1]), c2, m.x), a, b);
              top = fmaxf(fmaxf(top, a), b);
              f2_unpack(f2_fma(f2_pack(s[i + 2], s[i + 3]), c2, m.y), a, b);
              top = fmaxf(fmaxf(top, a), b);
            }
          move = px_bar_or(1 + wg, top > PX_LAZY);
        }
        if (move) {
          // three places in turn: all have read one before any comes to its next use
          const int now_at = moves, next_at = moves == 2 ? 0 : moves + 1;
          moves = next_at;
          float top = -INFINITY;
#pragma unroll
          for (int i = 0; i < PX_MINE; ++i)
            if (i < mine) {
#pragma unroll
              for (int z = 0; z < 8; ++z) {
                const float r = px_warp_max(s[8 * i + z]);
                if (lane == 8 * i + z) top = r;
              }
            }
          if (lane < 8 * mine) {
            atomicMax(&sm.top[now_at][my_row], px_order(top));
          }
          if (lane < 8 * PX_MINE) sm.top[next_at][first_row(lane >> 3) + (lane & 7)] = 0;
          named_bar_sync(1 + wg, 128);
          // (every warp of the group finds, and writes, the same)
          if (lane < 8 * mine) {
            top = px_unorder(sm.top[now_at][my_row]) * c;
            const float old = first ? PX_UNSET : m_mine;
            m_mine = top == -INFINITY ? old : fmaxf(old, top);
            sm.minus_m[my_row] = -m_mine;
            sm.by[my_row] = px_ex2(old - m_mine);
          }
          __syncwarp();
          if (!first) {
            // O holds the run's units before, the total the runs before
            const int runs = (u - x.u0) / PX_RUN, now = run0 + runs, total = runs > 0;
            if (total) ready(&sm.o_empty[(now - 1) & 1], ((now - 1) >> 1) & 1);
            ready(&sm.p_empty, (k - 1) & 1);
#pragma unroll 1
            for (int part = (u - x.u0) % PX_RUN ? 0 : p_parts; part < p_parts + total; ++part)
#pragma unroll 1
              for (int i = 0; i < 2 * mine; ++i) {   // four rows
                const int r = first_row(i >> 1) + 4 * (i & 1);
                const uint32_t at = tmem + lanes + r +
                                    (part < p_parts ? PX_O + (x.rows <= PX_TWICE ? PX_O_STEP * (now & 1) : 0) + part * cols : PX_TOTAL);
                float o[4];
                px_ld4(at, o);
                tmem_wait_ld();
#pragma unroll
                for (int z = 0; z < 4; ++z) o[z] *= sm.by[r + z];
                px_st4(at, o);
              }
#pragma unroll
            for (int i = 0; i < 8 * PX_MINE; ++i)
              if (i < 8 * mine) l[i] *= sm.by[first_row(i >> 3) + (i & 7)];
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          }
        }
        if (k > 0) ready(&sm.p_empty, (k - 1) & 1);   // P of the unit before has been read
#pragma unroll
        for (int i = 0; i < PX_MINE; ++i)
          if (i < mine) {
            uint64_t v[4];
#pragma unroll
            for (int z = 0; z < 4; z += 2) {
              const ulonglong2 m = *reinterpret_cast<const ulonglong2*>(&sm.minus_m[first_row(i) + 2 * z]);
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const int at = 8 * i + 2 * (z + y);
                float a, b;
                f2_unpack(f2_fma(f2_pack(s[at], s[at + 1]), c2, y ? m.y : m.x), a, b);
                v[z + y] = f2_pack(px_ex2(a), px_ex2(b));
                f2_unpack(f2_add(f2_pack(l[at], l[at + 1]), v[z + y]), l[at], l[at + 1]);
              }
            }
#pragma unroll
            for (int part = 0; part < PX_PARTS; ++part) {
              if (part < p_parts) {   // B's columns: the parts side by side
                const int ch = part * cols / 8 + wg + PX_GROUPS * i;
                uint4 o;
                o.x = px_part(v[0]);
                o.y = px_part(v[1]);
                o.z = px_part(v[2]);
                o.w = px_part(v[3]);
                *reinterpret_cast<uint4*>(Ps + (ch >> 3) * C::P_PART + e * 128 + (((ch & 7) ^ (e & 7)) << 4)) = o;
              }
            }
          }
        // a slot that no row sees may hold anything: its values as zeros (0 times anything finite), as
        // far as the product reads (steps of 16 slots)
        const int there = x.end - x.slot0 - u * PX_UNIT;   // slots of the unit
        if (wg == PX_GROUPS - 1 && (there < PX_UNIT || ok != 3u)) {
          constexpr int CHUNKS = 8 * C::HALVES;   // of a slot
          const int vs = (2 * k + 1) % NS, z1 = min(PX_UNIT, (there + 15) / 16 * 16) * CHUNKS;
          wait(&sm.full[vs], ((2 * k + 1) / NS) & 1);
#pragma unroll 1
          for (int z = (ok == 3u ? there * CHUNKS : 0) + e; z < z1; z += 128) {
            const int at = z / CHUNKS, i = z % CHUNKS;
            if (at >= there || !((ok >> (at >> 6)) & 1))
              *reinterpret_cast<uint4*>(smem + (size_t)vs * C::TILE + at * 128 + (i >> 3) * C::HALF + (((i & 7) ^ (at & 7)) << 4)) =
                  make_uint4(0, 0, 0, 0);
          }
        }
        fence_proxy_async_smem();
        tc_fence_before();
        arrive(&sm.p_full);
      }
      // ---- the rows' references and sums (a warp's part of them) for the results
      const size_t row = scratch_row(x);
      const PxScratch scratch(p);
#pragma unroll
      for (int i = 0; i < PX_MINE; ++i)
        if (i < mine) {
          const float sum = px_across(l + 8 * i, lane, [](float a, float b) { return a + b; });
          const int r = first_row(i) + lane;
          if (lane < 8 && r < x.rows) reinterpret_cast<float*>(scratch.l + row + r)[warp & 3] = sum;
        }
      if ((warp & 3) == 0 && lane < 8 * mine && my_row < x.rows) scratch.m[row + my_row] = m_mine;
      run0 += (x.u1 - x.u0 + PX_RUN - 1) / PX_RUN;
      arrive(&sm.seg_empty[seg % PX_SEGS]);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// A warp for each row and head: its partial results by weight, the loads of PX_JOIN of them in flight.
// Where they are is worked out before the wait for them (the lengths are those that the kernel before has
// waited for); small CTAs, as one wave has to hold them all.  (48 rows of 32 heads: 3.3 us less for both.)
constexpr int PX_JOIN = 8, PX_MERGE = 128;
template <int HD>
__global__ void __launch_bounds__(PX_MERGE) prefix_merge_kernel(const __grid_constant__ PrefixAttnParams p) {
  constexpr int E = HD / 32;
  pdl_trigger();
  const int lane = threadIdx.x & 31, w = blockIdx.x * (PX_MERGE / 32) + (threadIdx.x >> 5);
  if (w >= p.b * p.nq * p.H) return;
  const PxScratch scratch(p);
  const int r = px_quot(w, p.H), h = w - r * p.H, s = px_div(r, p.inv_nq), hk = px_div(h, p.inv_g);
  const PxPlan a = px_plan(p, p.ctas, lane);
  const int q = a.q, rest = a.r, tp = a.tp, units = a.units;
  const PxCost* cost = a.cost;
  const int e0 = __shfl_sync(0xffffffffu, a.end[0], s >> 1),
            e_was = __shfl_sync(0xffffffffu, a.end[1], max(0, (s >> 1) - 1));
  const int c_s = s & 1 ? e0 : s ? e_was : 0, own = px_units(p, __shfl_sync(0xffffffffu, s & 1 ? a.len[1] : a.len[0], s >> 1), a.shared);
  const int R = p.b * p.nq * p.G, rr = r * p.G + h - hk * p.G;
  // of the shared pages, of the others: parts, the first one's row of the scratch (an item's own), and
  // how far the second one's (a CTA's) is from 0, the later ones PX_ROWS on each
  const int all = p.b * p.nq * p.H, mine = hk * R + rr;
  int n[2] = {0, 0}, next[2] = {0, 0};
  auto item = [&](int k, int base, int units, int at) {   // its first place, units, and the row of the tile
    const int first = base + cost[k].start, c0 = px_owner(first, q, rest);
    n[k] = px_owner(first + (units - 1) * cost[k].unit, q, rest) - c0 + 1;
    next[k] = 2 * all + PX_ROWS * c0 + at;
  };
  if (units > 0) {
    const int t = px_quot(rr, p.tiles[0].rows);
    item(0, (hk * p.tiles[0].n + t) * (cost[0].start + units * cost[0].unit), units, rr - t * p.tiles[0].rows);
  }
  if (own > 0) {
    const int x = rr - s * p.nq * p.G, t = px_quot(x, p.tiles[1].rows);
    item(1, tp + c_s + (hk * p.tiles[1].n + t) * (cost[1].start + own * cost[1].unit), own, x - t * p.tiles[1].rows);
  }
  const int parts = n[0] + n[1];
  pdl_wait();
  float M = PX_UNSET, L = 0.f, o[E];
#pragma unroll
  for (int i = 0; i < E; ++i) o[i] = 0.f;
#pragma unroll 1
  for (int i0 = 0; i0 < parts; i0 += PX_JOIN) {
    float v[PX_JOIN][E], m[PX_JOIN];
    float4 l[PX_JOIN];
#pragma unroll
    for (int i = 0; i < PX_JOIN; ++i) {
      const int k = i0 + i >= n[0], c = i0 + i - (k ? n[0] : 0), at = c == 0 ? k * all + mine : next[k] + c * PX_ROWS;
      m[i] = PX_UNSET;
      l[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i0 + i < parts) {
        const float* src = scratch.o + (size_t)at * HD + E * lane;
        m[i] = __ldcg(scratch.m + at);
        l[i] = __ldcg(scratch.l + at);
        if constexpr (E == 4) *reinterpret_cast<float4*>(v[i]) = __ldcg(reinterpret_cast<const float4*>(src));
        else *reinterpret_cast<float2*>(v[i]) = __ldcg(reinterpret_cast<const float2*>(src));
      }
    }
    float now = M;
#pragma unroll
    for (int i = 0; i < PX_JOIN; ++i) now = fmaxf(now, m[i]);
    const float f = px_ex2(M - now);
    M = now;
    L *= f;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] *= f;
#pragma unroll
    for (int i = 0; i < PX_JOIN; ++i) {
      const float sum = (l[i].x + l[i].y) + (l[i].z + l[i].w), wt = px_ex2(m[i] - now);
      if (sum == 0.f) continue;   // (none, or of a row that has seen no slot)
      L += wt * sum;
#pragma unroll
      for (int z = 0; z < E; ++z) o[z] += wt * v[i][z];
    }
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;   // (a row that sees no slot: 0)
#pragma unroll
  for (int i = 0; i < E; ++i) o[i] *= inv;
  const long long out = r * p.out_ld + (long long)h * HD + E * lane;
  const size_t op = (size_t)r * p.H * HD + (size_t)h * HD + E * lane;
#pragma unroll
  for (int i = 0; i < E; i += 2) {
    uint64_t v = f2_pack(o[i], o[i + 1]);
    const uint32_t hi = px_part(v);
    if (p.bf16) *reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(p.out) + out + i) = hi;
    else *reinterpret_cast<float2*>(static_cast<float*>(p.out) + out + i) = make_float2(o[i], o[i + 1]);
    if (p.out_hi) {
      *reinterpret_cast<uint32_t*>(p.out_hi + op + i) = hi;
      *reinterpret_cast<uint32_t*>(p.out_lo + op + i) = px_part(v);
    }
  }
}

template <int HD>
constexpr size_t px_smem() {
  static_assert(PxCfg<HD>::OFF_MISC + sizeof(PxMisc) <= 232448, "shared memory of one CTA");
  return PxCfg<HD>::OFF_MISC + sizeof(PxMisc);
}

template <int HD>
cudaError_t px_launch(const PrefixAttnParams& p, cudaStream_t st, bool pdl) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.ctas);
  cfg.blockDim = dim3(PX_THREADS);
  cfg.dynamicSmemBytes = px_smem<HD>();
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, prefix_attention_kernel<HD>, p);
  if (e != cudaSuccess) return e;
  cfg.gridDim = dim3((p.b * p.nq * p.H + PX_MERGE / 32 - 1) / (PX_MERGE / 32));
  cfg.blockDim = dim3(PX_MERGE);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, prefix_merge_kernel<HD>, p);
}

}  // namespace

// tiles of nearly the same number of rows, a multiple of 16
static PxTiles px_tiles(int all) {
  PxTiles t;
  t.n = (all + PX_ROWS - 1) / PX_ROWS;
  t.rows = ((all + t.n - 1) / t.n + 15) / 16 * 16;
  t.n = (all + t.rows - 1) / t.rows;
  return t;
}

// for px_div: n (inv d - 2^32) < n d < 2^32
static uint32_t px_inv(int d) { return d == 1 ? 0u : (uint32_t)(((1ull << 32) + d - 1) / d); }

cudaError_t prefix_attention_prepare() {
  const cudaFuncAttribute a = cudaFuncAttributeMaxDynamicSharedMemorySize;
  cudaError_t e = cudaFuncSetAttribute(prefix_attention_kernel<64>, a, (int)px_smem<64>());
  if (e == cudaSuccess) e = cudaFuncSetAttribute(prefix_attention_kernel<128>, a, (int)px_smem<128>());
  if (e == cudaSuccess) e = prefer_shared(prefix_attention_kernel<64>);
  if (e == cudaSuccess) e = prefer_shared(prefix_attention_kernel<128>);
  if (e == cudaSuccess) e = prefer_shared(prefix_merge_kernel<64>);
  if (e == cudaSuccess) e = prefer_shared(prefix_merge_kernel<128>);
  return e;
}

cudaError_t launch_prefix_attention(const PrefixAttnParams& p0, int num_sms, cudaStream_t st, bool pdl) {
  PrefixAttnParams p = p0;
  p.ctas = num_sms;
  p.G = p.H / p.Hk;
  p.inv_g = px_inv(p.G);
  p.inv_nq = px_inv(p.nq);
  p.tiles[0] = px_tiles(p.b * p.nq * (p.H / p.Hk));
  p.tiles[1] = px_tiles(p.nq * (p.H / p.Hk));
  return p.hd == 64 ? px_launch<64>(p, st, pdl) : px_launch<128>(p, st, pdl);
}

}  // namespace sdsat
