// Causal attention of the new rows of a ragged batch over pages: flash attention on tcgen05.
//
//   out = sum_t p_t v_t / sum_t p_t,  p_t = exp2(c s_t - m),  s = q K^T,  c = log2(e) / sqrt(hd)
//
// A tile is 128 rows: PT = 128 / G positions of the G query heads that share a cache head, so that K and V are
// loaded once for all of them.  An item is TILES tiles of a sequence and cache head, its work the steps of 64 keys (a
// page) that its rows see.  The items stand in a line, weighed by their keys and a start's cost, and every CTA (one on an
// SM) takes an equal stretch of it, wherever that begins: few rows of long sequences are split along their keys, and
// causal tiles of unequal length leave no SM idle.  Of an item that several CTAs share each writes its partial results
// (m, sum, O), and the one that comes last joins them, always in the same order (a second kernel for that took 15 us
// behind a prompt of 4095 positions on 32 heads, 126 in all).  Sequences, lengths and pages are device values, so the
// plan is made on the device, by one warp of each CTA (a scan over the sequences), which then hands items to the others.
//
// Scores have two places in TMEM, by the step's parity: S of step i + 2 is issued behind P V of step i, so that the
// softmax (a thread for each row, no shuffles) always has the next step's scores.  The entries of the ring go by
// what is issued together: entry e of an item is V of step e - 2 and K of step e.
// bf16 (PARTS = 1, TILES = 2): P lies over its S; a warp for each tile issues its products.  What bounds it: the tensor
// cores' 8 x 48 (N = 64: A is read at the shared memory's rate) and 4 x 64 cycles a step and tile, 1280 of the 1600 to 1700
// that a step of both tiles takes; the softmax takes 1150 beside them.
// P is one bf16 part, as the values that it weighs are (2^-9 of each probability, at random: 2.2e-3 of the result against 64
// bits, where the rounding of the result itself is 1.7e-3); two parts leave only that, but take 16 to 30 % longer (7B prompt
// 137 us, 64 single tokens after 8200 slots 235 for 201): not kept.
// fp32 (PARTS = 3, TILES = 1): queries and probabilities as three bf16 parts (24 bits), smallest first; P beside S, so S
// and P V are issued by a warp each.  The tensor cores' accumulator truncates, so O holds one step, and 4 more warps add
// it to a rounded total in registers.  1920 tensor cycles of 2200 a step.
// Waits and products cost the warps that issue them (a wait that is over 100 cycles and more, an MMA 44, 90 from a branch
// of one lane), which is why a tile's step has one wait for both of its barriers and whole warps issue.
//
// Measured, us: 32 heads x 128, 4095 positions bf16 118 (1.16 PFLOP/s; prefill attention, which has fp32 queries in two
// parts, 257); 32 / 8 heads, 8 sequences of 330 to 1100 rows after 800 to 16500 slots 730 (1.33 PFLOP/s; 804 in a long run
// at the power cap), one of 4096 rows after 16384 780 (1.57); 48 sequences of up to 8200 slots, 46 of them with one row,
// 154 to 161 (5.5 TB/s); 40 heads, 777 rows after 2048 slots in fp32 111, 2 x 6 rows after 70 slots 7.2.
//
// A row's reference m is moved only when its maximum has grown by more than 2^8 since the last time (exact: it cancels
// in the division by the row's sum), so that O (the total) is seldom rescaled.
//
// Values that no row may see (behind the last key, up to the 16 keys of a product's step; pages that are not there) take
// part with P = 0 and may hold NaN: they are made zeros in the ring before the product, by the warp that loads.
//
// Warps: 0 loads (TMA), 1 and 3 issue the products of tile 0 and 1, 2 plans; 4-7 softmax and output of tile 0, 8-11 of
// tile 1; with one tile 4-7 bring the queries, too, and 8-11 keep the total and write the output.
#include <algorithm>

#include "chunk_plan.h"
#include "common.cuh"
#include "internal.h"

namespace sdsat {

static_assert(KV_PAGE == CH_STEP, "a page is one box of keys");
constexpr int CH_THREADS = 384;
constexpr int CH_DESC = 4;            // items handed out ahead
constexpr int CH_FLAGS = 16;          // entries whose pages' presence is kept
// Barriers of a tile's scores, taken in turn by its entries.  An item's first two entries wait for no P, so they may be
// complete while the softmax has yet to look at the last two of the item before: four entries that it has not seen.  With two
// barriers one of these would be two phases behind, where its parity reads as incomplete.
constexpr int CH_SBARS = 4;
static_assert((CH_SBARS & (CH_SBARS - 1)) == 0, "an entry's barrier and parity are bits of its number");
constexpr float CH_LAZY = 8.0f;       // log2 of the growth of a row maximum that is left unscaled
constexpr float CH_UNSET = -1e30f;    // reference of a row that has seen no key

struct ChHead {
  int row0, npos, pos0, hk;           // first row, positions, slot of the first; cache head (-1: no more items)
  int seq, kb0, kb1, part;            // steps; of an item in parts, which one this is, else -1
  int head, parts, unused[2];         // the CTA of its first part, their number
};
struct ChItem : ChHead {
  int pages[32];                      // of its first steps
};

template <int HD, int PARTS>
struct ChCfg {
  static constexpr int TILES = PARTS == 1 ? 2 : 1;
  static constexpr int HALVES = HD / 64;
  static constexpr int HALF = CH_ROWS * 128;                // Q: 128 rows x 64 dims, 128-byte swizzle
  static constexpr int TILE = HALVES * HALF;
  static constexpr int BOX = CH_STEP * 128;                 // K or V: 64 keys x 64 dims, a TMA box
  static constexpr int SLOT = HALVES * BOX;                 // a step's K or V
  static constexpr int SLOTS = HD == 128 ? 4 : 8;           // entries of the ring: V, K
  static_assert(CH_FLAGS >= SLOTS + 2, "flags outlast the loads ahead");
  static constexpr size_t OFF_RING = (size_t)TILES * PARTS * TILE;
  static constexpr size_t OFF_BAR = OFF_RING + (size_t)SLOTS * 2 * SLOT;
  static constexpr int NBAR = 2 * SLOTS + 20 + 2 * CH_SBARS + 2 * CH_DESC;
  static constexpr size_t OFF_ITEMS = OFF_BAR + (NBAR + 1) / 2 * 16;
  static constexpr size_t SMEM = 1024 + OFF_ITEMS + CH_DESC * sizeof(ChItem) + CH_FLAGS * 4 + 16;
  static_assert(SMEM <= 232448, "shared memory of one CTA");
  static_assert(OFF_RING + SLOTS * 2 * SLOT >= (CHUNK_MAX_BATCH + 2) * (8 + sizeof(ChSeq)), "the plan lies over the queries and the ring");
  // TMEM columns: S and P of step i, by its parity
  static constexpr int S_COL(int t) { return 128 * t; }
  static constexpr int P_COL(int t) { return PARTS == 1 ? 128 * t : 128; }
  static constexpr int P_STEP = PARTS == 1 ? 64 : 96;
  static constexpr int O_COL(int t) { return PARTS == 1 ? 256 + 128 * t : 320; }
  // one tile: what the softmax tells those who keep the total; the total's factor of a step (four of them: one is read before
  // the P V of the step after it, which the softmax waits for two steps on), and by item's parity the sum and the reference
  static constexpr int F_COL(uint32_t step) { return 448 + (step & 3); }
  static constexpr int L_COL = 452, M_COL = 454;
};

// Two places for partial results a CTA (an item that goes on in the next one, an item that began before), and a counter
// of an item's parts that have come, zero between launches
size_t chunk_attention_counters(int num_sms) { return (size_t)num_sms * 4 * sizeof(int); }
size_t chunk_attention_scratch(int num_sms) { return (size_t)2 * num_sms * (2 + 2 * CH_ROWS * (2 + 128)); }

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* v) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_st1(uint32_t taddr, float v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "r"(__float_as_uint(v)) : "memory");
}
__device__ __forceinline__ float tmem_ld1(uint32_t taddr) {
  uint32_t r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(taddr) : "memory");
  return __uint_as_float(r);
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// The products are issued by a whole warp, in step, of which one lane's instruction counts (`mine`): issued from a
// branch that one lane took, each MMA cost some 90 cycles.
__device__ __forceinline__ uint32_t ch_elect() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r));
  return r;
}
// D[tmem] (+)= A[smem] * B[smem]^T
__device__ __forceinline__ void ch_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t mine) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(mine)
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]: A's rows on the lanes, two bf16 of K per column
__device__ __forceinline__ void ch_mma_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t mine) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(mine)
      : "memory");
}
__device__ __forceinline__ void ch_commit(uint32_t bar, uint32_t mine) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "setp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"(mine)
      : "memory");
}
// whether the phases of two barriers are both complete: one round trip for both
__device__ __forceinline__ bool ch_try_both(uint32_t a, uint32_t pa, uint32_t b, uint32_t pb) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 q, [%3], %4;\n\t"
      "and.pred p, p, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(a), "r"(pa), "r"(b), "r"(pb)
      : "memory");
  return ok != 0;
}
__device__ __noinline__ bool ch_wait_slow(uint64_t* bar, uint32_t parity, volatile int* abort, uint32_t* err) {
  return mbar_wait_bounded(bar, parity, abort, err);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// MN-major operand in the 128-byte swizzle layout: atoms of 64 dims (128 bytes) x 8 keys;
// `lead` bytes to the next 64 dims, 1024 to the next 8 keys
__device__ __forceinline__ uint64_t sdesc_sw128_mn(uint32_t saddr, uint32_t lead) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(lead >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}
__device__ __forceinline__ void tma_load_3d(void* dst, const void* map, uint64_t* bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
          smem_u32(dst)),
      "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// a, b rounded to packed bf16 (a in the low half), and what the rounding left of them
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ uint32_t take_bf16(float& a, float& b) {
  const uint32_t r = pack_bf16(a, b);
  a -= __uint_as_float(r << 16);
  b -= __uint_as_float(r & 0xFFFF0000u);
  return r;
}

template <int HD, int PARTS>
__global__ void __launch_bounds__(CH_THREADS, 1) chunk_attention_kernel(const __grid_constant__ ChunkAttnParams p) {
  using C = ChCfg<HD, PARTS>;
  constexpr int SLOTS = C::SLOTS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = smem + C::OFF_RING;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);   // [SLOTS] an entry landed
  uint64_t* empty = full + SLOTS;         // [SLOTS] its products are done
  uint64_t* z_full = empty + SLOTS;       // an entry landed in which values have to be made zeros
  uint64_t* q_full = z_full + 1;          // [2] per tile: Q is there
  uint64_t* q_empty = q_full + 2;         // [2] two tiles: the item's last S is complete
  uint64_t* s_full = q_empty + 2;         // [2][CH_SBARS] per tile and entry: S of its step, and P V of the one before the last, are complete
  uint64_t* p_full = s_full + 2 * CH_SBARS;   // [2][2] P is in TMEM, O is rescaled (128 threads)
  uint64_t* pv_done = p_full + 4;         // [2] one tile, by step's parity: its P V is complete
  uint64_t* o_free = pv_done + 2;         // one tile: O of a step has been read (128 threads)
  uint64_t* part_full = o_free + 1;       // partial results are written (by all who write)
  uint64_t* part_go = part_full + 1;      // ... and whether they are to be joined here is known
  uint64_t* l_full = part_go + 1;          // [2] one tile, by item's parity: the rows' sums are there (128 threads)
  uint64_t* l_free = l_full + 2;          // [2] ... and have been read
  uint64_t* drain = l_free + 2;           // [2]
  uint64_t* d_full = drain + 2;           // [CH_DESC] an item's description is there
  uint64_t* d_empty = d_full + CH_DESC;   // [CH_DESC] all have read it
  ChItem* items = reinterpret_cast<ChItem*>(smem + C::OFF_ITEMS);
  uint32_t* flags = reinterpret_cast<uint32_t*>(items + CH_DESC);   // [CH_FLAGS] by entry: whether there is the page of its K
  uint32_t* tmem_slot = flags + CH_FLAGS;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* joins = abort_flag + 1;   // this CTA's part was the item's last
  long long* plan = reinterpret_cast<long long*>(smem);             // [b + 1] cost before each sequence
  ChSeq* plan_seq = reinterpret_cast<ChSeq*>(plan + CHUNK_MAX_BATCH + 2);   // [b]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = p.H / p.Hk, pt1 = CH_ROWS / G, pt = C::TILES * pt1, cap = p.ld * KV_PAGE;
  if (threadIdx.x == 0) {
    for (int s = 0; s < SLOTS; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 2);
    }
    mbar_init(z_full, 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&q_full[t], PARTS == 1 ? 1 : 128);
      mbar_init(&q_empty[t], 1);
      for (int b = 0; b < CH_SBARS; ++b) mbar_init(&s_full[CH_SBARS * t + b], 1);
      for (int b = 0; b < 2; ++b) mbar_init(&p_full[2 * t + b], 128);
      mbar_init(&l_full[t], 128);
      mbar_init(&l_free[t], 128);
    }
    mbar_init(&pv_done[0], 1);
    mbar_init(&pv_done[1], 1);
    mbar_init(o_free, 128);
    mbar_init(part_full, C::TILES * 128);
    mbar_init(part_go, 1);
    mbar_init(drain, 1);
    mbar_init(drain + 1, 1);
    for (int i = 0; i < CH_DESC; ++i) {
      mbar_init(&d_full[i], 1);
      mbar_init(&d_empty[i], 11);
    }
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&p.kmap);
    tma_prefetch_desc(&p.vmap);
    if (PARTS == 1) tma_prefetch_desc(&p.qmap);
  }
  if (warp == 1) tmem_alloc(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_trigger();
  pdl_wait();

  int* arrived = reinterpret_cast<int*>(p.part);                              // [4 ctas]
  float2* part_ml = reinterpret_cast<float2*>(arrived + 4 * gridDim.x);       // [2 ctas][256]
  float4* part_o = reinterpret_cast<float4*>(part_ml + 2 * gridDim.x * 2 * CH_ROWS);   // [2 ctas][HD / 4][256]: a thread for each row
  // where part k of the item whose first part is CTA a's leaves its results
  auto part_at = [&](int a, int k) { return (size_t)(k ? 2 * (a + k) : 2 * a + 1); };
  auto ml_of = [&](size_t at, int rr) { return part_ml + at * 2 * CH_ROWS + rr; };
  auto o_of = [&](size_t at, int rr, int x) { return part_o + (at * (HD / 4) + x / 4) * 2 * CH_ROWS + rr; };

  // an item's geometry
  auto item_keys = [&](const ChHead& it, int t) { return (int)min((long long)cap, (long long)it.pos0 + min(it.npos, (t + 1) * pt1)); };
  auto item_tiles = [&](const ChHead& it) { return C::TILES == 2 && it.npos > pt1 ? 2 : 1; };
  // the step up to which this part of tile t goes
  auto item_end = [&](const ChHead& it, int t) { return min(it.kb1, (item_keys(it, t) + CH_STEP - 1) / CH_STEP); };
  // the last tile's step j has values behind its last key in 16 of a product
  auto item_tail = [&](const ChHead& it, int j) {
    const int k = item_keys(it, item_tiles(it) - 1);
    return k % 16 != 0 && j == k / CH_STEP;
  };
  uint32_t d_phase = 0;   // items read
  auto next_item = [&](ChHead& it, int* page = nullptr) {   // by a warp (page: of the item's step `lane`)
    const int d = d_phase % CH_DESC;
    const bool ok = __all_sync(0xffffffffu, mbar_wait_bounded(&d_full[d], (d_phase / CH_DESC) & 1, abort_flag, p.err));
    if (!ok) return false;
    it = items[d];
    if (page) *page = items[d].pages[lane];
    __syncwarp();
    if (lane == 0) mbar_arrive(&d_empty[d]);
    ++d_phase;
    return it.hk >= 0;
  };

  // Partial results have been written by warps w0 .. w0 + W - 1, all of which call this: the one whose part is the item's
  // last joins the parts.  False: a wait ran out.
  uint32_t part_phase = 0;
  auto join = [&](const ChHead& it, int w0) {
    constexpr int W = 4 * C::TILES, E = HD / 32;   // warps; values of a lane
    auto wait = [&](uint64_t* bar) { return (bool)__all_sync(0xffffffffu, mbar_wait_bounded(bar, part_phase & 1, abort_flag, p.err)); };
    __threadfence();
    mbar_arrive(part_full);
    if (warp == w0) {
      if (!wait(part_full)) return false;
      if (lane == 0) {
        const bool last = atomic_add_acq_rel_gpu(arrived + it.head, 1) == it.parts - 1;
        if (last) arrived[it.head] = 0;
        *joins = last;
        mbar_arrive(part_go);
      }
      __syncwarp();
    }
    if (!wait(part_go)) return false;
    ++part_phase;
    if (!*joins) return true;
    auto position = [&](int rr) {   // of a row in the item, -1: no row of it
      const int gi = rr % CH_ROWS / G, i = rr / CH_ROWS * pt1 + gi;
      return gi < pt1 && i < it.npos ? i : -1;
    };
    if (it.npos * G > W * 8) {   // a thread for each row
      const int rr = (int)threadIdx.x - w0 * 32, i = position(rr);
      if (i < 0) return true;
      float m = CH_UNSET, l = 0.f;
#pragma unroll 2
      for (int k = 0; k < it.parts; ++k) {   // (a part that saw no key of the row has a sum of 0, and maybe nothing was written)
        const float2 ml = __ldcg(ml_of(part_at(it.head, k), rr));
        const bool seen = ml.y != 0.f;       // (a sum that is NaN counts, too: the row's result is NaN)
        const float now = seen ? fmaxf(m, ml.x) : m;
        l = l * ex2(m - now) + (seen ? ml.y * ex2(ml.x - now) : 0.f);
        m = now;
      }
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      const long long to = (long long)(it.row0 + i) * p.out_ld + (it.hk * G + rr % CH_ROWS % G) * HD;
#pragma unroll 1
      for (int x = 0; x < HD; x += 32) {
        float acc[32];
#pragma unroll
        for (int y = 0; y < 32; ++y) acc[y] = 0.f;
#pragma unroll 2
        for (int k = 0; k < it.parts; ++k) {
          const size_t at = part_at(it.head, k);
          const float2 ml = __ldcg(ml_of(at, rr));
          float4 v[8];
#pragma unroll
          for (int y = 0; y < 8; ++y) v[y] = __ldcg(o_of(at, rr, x + 4 * y));
          const float w = ex2(ml.x - m);
          if (ml.y != 0.f)
#pragma unroll
            for (int y = 0; y < 8; ++y) {
              acc[4 * y] = fmaf(v[y].x, w, acc[4 * y]);
              acc[4 * y + 1] = fmaf(v[y].y, w, acc[4 * y + 1]);
              acc[4 * y + 2] = fmaf(v[y].z, w, acc[4 * y + 2]);
              acc[4 * y + 3] = fmaf(v[y].w, w, acc[4 * y + 3]);
            }
        }
#pragma unroll
        for (int y = 0; y < 32; y += 8) {
          if (PARTS == 1)
            *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + to + x + y) =
                make_uint4(pack_bf16(acc[y] * inv, acc[y + 1] * inv), pack_bf16(acc[y + 2] * inv, acc[y + 3] * inv),
                           pack_bf16(acc[y + 4] * inv, acc[y + 5] * inv), pack_bf16(acc[y + 6] * inv, acc[y + 7] * inv));
          else
#pragma unroll
            for (int z = y; z < y + 8; z += 4)
              *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to + x + z) = make_float4(acc[z] * inv, acc[z + 1] * inv, acc[z + 2] * inv, acc[z + 3] * inv);
        }
      }
      return true;
    }
    // few rows, often in many parts: a warp for each
#pragma unroll 1
    for (int q = warp - w0; q < it.npos * G; q += W) {
      const int rr = q / (pt1 * G) * CH_ROWS + q % (pt1 * G), i = position(rr);
      float m = CH_UNSET, l = 0.f, acc[E];
#pragma unroll
      for (int y = 0; y < E; ++y) acc[y] = 0.f;
#pragma unroll 8
      for (int k = 0; k < it.parts; ++k) {
        const size_t at = part_at(it.head, k);
        const float2 ml = __ldcg(ml_of(at, rr));
        const float* v = reinterpret_cast<const float*>(o_of(at, rr, lane * E)) + lane * E % 4;
        float u[E];
#pragma unroll
        for (int y = 0; y < E; ++y) u[y] = __ldcg(v + y);
        const bool seen = ml.y != 0.f;
        const float now = seen ? fmaxf(m, ml.x) : m, f = ex2(m - now), w = seen ? ex2(ml.x - now) : 0.f;
        m = now;
        l = fmaf(l, f, ml.y * w);
#pragma unroll
        for (int y = 0; y < E; ++y) acc[y] = fmaf(acc[y], f, seen ? u[y] * w : 0.f);
      }
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      const long long to = (long long)(it.row0 + i) * p.out_ld + (it.hk * G + rr % CH_ROWS % G) * HD + lane * E;
#pragma unroll
      for (int y = 0; y < E; y += 2) {
        if (PARTS == 1) *reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(p.out) + to + y) = pack_bf16(acc[y] * inv, acc[y + 1] * inv);
        else *reinterpret_cast<float2*>(static_cast<float*>(p.out) + to + y) = make_float2(acc[y] * inv, acc[y + 1] * inv);
      }
    }
    return true;
  };

  if (warp == 2) {
    // ---- the plan
    long long total = 0;
    int n_items = 0;
    bool bad = false, past = false;
    for (int s0 = 0; s0 < p.b; s0 += 32) {
      const int s = s0 + lane;
      long long cost = 0;
      int items_here = 0;
      if (s < p.b) {
        const int a = __ldcg(p.start + s), z = __ldcg(p.start + s + 1), len = __ldcg(p.len + s);
        bad |= a < 0 || z < a || z > p.rows;
        past |= z > a && (long long)max(len, 0) + (z - a) > cap;
        const ChSeq q = ch_sequence(a, z, len, pt1, C::TILES, cap);
        if (z >= a) cost = ch_cost(q, pt, cap) * p.Hk, items_here = ch_items(q, pt, p.Hk);
        plan_seq[s] = q;
      }
      long long sum = cost;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += x;
      }
      if (s < p.b) plan[s] = total + sum - cost;
      total += __shfl_sync(0xffffffffu, sum, 31);
      n_items = min(1 << 20, n_items + (int)__reduce_add_sync(0xffffffffu, (unsigned)items_here));
    }
    bad = __any_sync(0xffffffffu, bad);
    past = __any_sync(0xffffffffu, past);
    if (lane == 0) {
      plan[p.b] = total;
      if (bad) set_error(p.err, ERR_CAPACITY);
      else if (past) set_error(p.err, ERR_PAGE);
    }
    __syncwarp();
    const int ctas = ch_ctas(gridDim.x, n_items, total), cta = blockIdx.x;
    const ChPlan line = {plan, plan_seq, p.b, p.Hk, pt, cap, ctas, total};
    // the first sequence from s on that has rows (b: none); the plan is gone once items are handed out (out)
    bool out = false;
    auto with_rows = [&](int s) {
      for (; s < p.b; s += 32) {
        const unsigned some = __ballot_sync(0xffffffffu, s + lane < p.b && (out ? __ldcg(p.start + min(s + lane, p.b - 1)) < __ldcg(p.start + min(s + lane, p.b - 1) + 1)
                                                                                 : plan_seq[min(s + lane, p.b - 1)].n > 0));
        if (some) return s + __ffs(some) - 1;
      }
      return p.b;
    };
    ChPlace a = {p.b, 0, 0, 0, 0}, z = a;
    if (!bad && cta < ctas && lane < 2) a = line.border(cta + lane);
    __syncwarp();
    z.s = __shfl_sync(0xffffffffu, a.s, 1), a.s = __shfl_sync(0xffffffffu, a.s, 0);
    z.hk = __shfl_sync(0xffffffffu, a.hk, 1), a.hk = __shfl_sync(0xffffffffu, a.hk, 0);
    z.t = __shfl_sync(0xffffffffu, a.t, 1), a.t = __shfl_sync(0xffffffffu, a.t, 0);
    z.kb = __shfl_sync(0xffffffffu, a.kb, 1), a.kb = __shfl_sync(0xffffffffu, a.kb, 0);
    a.cost = __shfl_sync(0xffffffffu, a.cost, 0);
    uint32_t n = 0;
    ChPlace end = z;
    ChSeq q = {0, 0, 0, 4};
    int it_seq = -1;
    bool ok = true;
    while (ok) {
      const bool more = a.s < p.b && !(a.s == end.s && a.hk == end.hk && a.t == end.t && a.kb >= end.kb);
      ChHead it = {0, 0, 0, -1, 0, 0, 0, -1, 0, 0, {0, 0}};
      int page = -1;
      bool stop = true;
      if (more) {
        if (!out) q = plan_seq[a.s];
        else if (a.s != it_seq) q = ch_sequence(__ldcg(p.start + a.s), __ldcg(p.start + a.s + 1), __ldcg(p.len + a.s), pt1, C::TILES, cap);
        it_seq = a.s;
        const int steps = ch_steps(q, pt, cap, a.t);
        it.row0 = q.first + a.t * pt;
        it.npos = min(pt, q.n - a.t * pt);
        it.pos0 = q.len + a.t * pt;
        it.hk = a.hk;
        it.seq = a.s;
        it.kb0 = a.kb;
        if (a.kb + lane < p.ld) page = __ldcg(p.table + (size_t)a.s * p.ld + a.kb + lane);
        stop = a.s == end.s && a.hk == end.hk && a.t == end.t;
        it.kb1 = stop ? end.kb : steps;
        if (it.kb0 > 0 || it.kb1 < steps) {
          line.parts(a, q, it.head, it.parts);
          it.part = cta - it.head;
        }
      }
      const int d = n % CH_DESC;
      ok = __all_sync(0xffffffffu, mbar_wait_bounded(&d_empty[d], ((n / CH_DESC) & 1) ^ 1, abort_flag, p.err));
      if (!ok) break;
      if (!out) fence_proxy_async_smem();   // (the plan's place: read before, written by TMA after)
      out = true;
      __syncwarp();
      items[d].pages[lane] = page;
      if (lane == 0) static_cast<ChHead&>(items[d]) = it;
      __syncwarp();
      if (lane == 0) mbar_arrive(&d_full[d]);
      ++n;
      if (!more) break;
      if (stop) a = z = end = ChPlace{p.b, 0, 0, 0, 0};
      else a = line.after(a, q, with_rows);
    }
  } else if (warp == 0) {
    // ---- loads
    const uint64_t pol = l2_policy_evict_normal();
    uint32_t n = 0, qn[2] = {0, 0}, zn = 0;   // entries, Q tiles loaded, entries with zeros
    bool ok = true;
    // the entry whose values wait to be made zeros, keys z_from .. z_to - 1 of its V
    int z_slot = -1, z_from = 0, z_to = 0;
    auto make_zeros = [&]() {
      if (z_slot < 0) return;
      if (mbar_wait_bounded(z_full, zn & 1, abort_flag, p.err)) {
        constexpr int CHUNKS = HD / 8;   // of 16 bytes, of a key
        for (int z = z_from * CHUNKS + lane; z < z_to * CHUNKS; z += 32) {
          const int at = z / CHUNKS, i = z % CHUNKS;
          *reinterpret_cast<uint4*>(ring + (size_t)z_slot * 2 * C::SLOT + (i >> 3) * C::BOX + at * 128 + (((i & 7) ^ (at & 7)) << 4)) =
              make_uint4(0u, 0u, 0u, 0u);
        }
        fence_proxy_async_smem();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&full[z_slot]);
      ++zn;
      z_slot = -1;
    };
    // the queries of an item wait for the last scores of the one before, its keys and values do not
    uint32_t q_wanted = 0;   // tiles (bits)
    ChHead it;
    auto get_queries = [&](bool wait) {
      for (int t = 0; PARTS == 1 && t < 2; ++t) {
        if (!((q_wanted >> t) & 1u)) continue;
        const uint32_t parity = (qn[t] & 1) ^ 1;
        if (!__all_sync(0xffffffffu, mbar_try_wait(&q_empty[t], parity))) {
          if (!wait) continue;
          make_zeros();
          ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(&q_empty[t], parity, abort_flag, p.err));
          if (!ok) return;
        }
        ++qn[t];
        q_wanted &= ~(1u << t);
        if (lane == 0) {
          mbar_arrive_expect_tx(&q_full[t], C::HALVES * 128 * G * pt1);
          for (int hh = 0; hh < C::HALVES; ++hh)
            tma_load_3d(smem + (size_t)t * C::TILE + hh * C::HALF, &p.qmap, &q_full[t], hh * 64, it.hk * G, it.row0 + t * pt1);
        }
        __syncwarp();
      }
    };
    // (what a product waits for is brought and made zeros before anything waits for that product)
    auto acquire = [&](uint64_t* bar, uint32_t parity) {
      if (!__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) {
        make_zeros();
        get_queries(true);
        ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abort_flag, p.err));
      }
      return ok;
    };
    while (ok) {
      if (z_slot >= 0 && !__all_sync(0xffffffffu, mbar_try_wait(&d_full[d_phase % CH_DESC], (d_phase / CH_DESC) & 1))) make_zeros();
      get_queries(true);
      int now = -1;
      if (!ok || !next_item(it, &now)) break;
      const int nt = item_tiles(it), keys = item_keys(it, nt - 1);
      for (int t = 0; t < nt; ++t)
        if (item_end(it, t) > it.kb0) q_wanted |= 1u << t;
      get_queries(false);
      // 32 pages at a time, the next ones asked for ahead
      const int* row = p.table + (size_t)it.seq * p.ld;
      auto pages = [&](int j) { return j + lane < p.ld ? __ldcg(row + j + lane) : -1; };
      int next = it.kb1 > it.kb0 + 32 ? pages(it.kb0 + 32) : -1, base = it.kb0;
      int before[2] = {0, 0};   // the pages of the last two steps
      for (int j = it.kb0; j < it.kb1 + 2 && ok; ++j, ++n) {   // K of step j, V of step j - 2
        if (j == base + 32) base = j, now = next, next = pages(j + 32);
        const int page = __shfl_sync(0xffffffffu, now, j - base), v_page = before[0];
        const bool has_k = j < it.kb1, has_v = j >= it.kb0 + 2;
        const bool k_there = has_k && page >= 0 && page < p.n_pages, v_there = has_v && v_page >= 0 && v_page < p.n_pages;
        before[0] = before[1];
        before[1] = page;
        const int s = n % SLOTS;
        if (!acquire(&empty[s], ((n / SLOTS) & 1) ^ 1)) break;
        const bool zeros = has_v && (!v_there || item_tail(it, j - 2));
        if (zeros) {
          make_zeros();   // (one at a time)
          const int seen = min(CH_STEP, keys - (j - 2) * CH_STEP);
          z_slot = s;
          z_from = v_there ? seen : 0;
          z_to = (seen + 15) / 16 * 16;
        }
        if (lane == 0) {
          uint64_t* bar = zeros ? z_full : &full[s];
          flags[n % CH_FLAGS] = k_there;
          if (has_k && !k_there) set_error(p.err, ERR_PAGE);
          mbar_arrive_expect_tx(bar, (k_there ? C::SLOT : 0) + (v_there ? C::SLOT : 0));
          uint8_t* at = ring + (size_t)s * 2 * C::SLOT;
#pragma unroll
          for (int hh = 0; hh < C::HALVES; ++hh) {
            if (v_there) tma_load_2d(at + hh * C::BOX, &p.vmap, bar, hh * 64, (v_page * p.Hk + it.hk) * KV_PAGE, pol);
            if (k_there) tma_load_2d(at + C::SLOT + hh * C::BOX, &p.kmap, bar, hh * 64, (page * p.Hk + it.hk) * KV_PAGE, pol);
          }
        }
        __syncwarp();
        get_queries(false);
      }
    }
    make_zeros();
    if (*abort_flag && lane == 0) {   // let the copies in flight land before the CTA exits
      auto land = [&](uint64_t* bar, uint32_t parity) {
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait(bar, parity))
          if (globaltimer_ns() - t0 > WAIT_LIMIT_NS) break;
      };
      if (PARTS == 1)
        for (int t = 0; t < 2; ++t)
          if (qn[t]) land(&q_full[t], (qn[t] - 1) & 1);
      if (zn) land(z_full, (zn - 1) & 1);
      for (uint32_t i = n > SLOTS ? n - SLOTS : 0; i < n; ++i) land(&full[i % SLOTS], (i / SLOTS) & 1);
    }
  } else if (warp == 1 || warp == 3) {
    // ---- products: a tile's or, with one tile, S on one warp and P V on the other
    const int t = PARTS == 1 ? warp >> 1 : 0;
    constexpr uint32_t idesc_s = idesc_bf16_f32(128, CH_STEP);
    constexpr uint32_t idesc_o = idesc_bf16_f32(128, HD) | (1u << 16);   // B is MN-major
    const uint32_t mine = ch_elect();
    const uint64_t q_desc = sdesc_sw128(smem_u32(smem)) + (uint64_t)(PARTS * t) * (C::TILE >> 4);
    const uint64_t v_desc = sdesc_sw128_mn(smem_u32(ring), C::BOX), k_desc = sdesc_sw128(smem_u32(ring) + C::SLOT);
    const uint32_t ts = tmem + C::S_COL(t), tp = tmem + C::P_COL(t), to = tmem + C::O_COL(t);
    bool ok = true;
    uint32_t n = 0, x = 0, qn = 0, pn = 0;   // entries of the ring and of the tile, Q tiles, P's
    const uint32_t full_at = smem_u32(full), empty_at = smem_u32(empty), s_at = smem_u32(s_full + CH_SBARS * t), p_at = smem_u32(p_full + 2 * t),
                   qe_at = smem_u32(q_empty + t), pv_at = smem_u32(pv_done);
    const bool does_s = PARTS == 1 || warp == 1, does_pv = PARTS == 1 || warp == 3;
    auto wait = [&](uint64_t* bar, uint32_t parity) {   // (the lanes agree before the products)
      ok = ok && mbar_wait_bounded(bar, parity, abort_flag, p.err);
    };
    auto agree = [&]() {
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      return ok;
    };
    ChHead it;
    while (ok && next_item(it)) {
      const int nt = item_tiles(it), keys = item_keys(it, t) - it.kb0 * CH_STEP, all = it.kb1 - it.kb0 + 2;
      const int steps = t < nt ? max(0, item_end(it, t) - it.kb0) : 0, mine_too = steps ? steps + 2 : 0;
      if (steps && does_s) wait(&q_full[t], qn++ & 1);
      // entry e: P V of step e - 2, then S of step e over the scores that it has used (one tile: once they have been read)
#pragma unroll 1
      for (int e = 0; e < mine_too; ++e, ++n, ++x) {
        const bool has_pv = e >= 2, has_s = e < steps;
        const uint32_t s = n % SLOTS, full_parity = (n / SLOTS) & 1;
        // one tile: x counts this warp's steps; S waits for P of the step before the last, P V for its own P
        if (PARTS != 1 && !(does_s ? has_s : has_pv)) --x;
        const uint32_t b = x & 1;
        uint32_t pw = pn;              // the P that is waited for
        bool wait_p = has_pv;
        if (PARTS != 1) {
          wait_p = does_s ? has_s && x >= 2 : has_pv;
          pw = does_s ? x - 2 : x;
        }
        bool ready;
        if (wait_p) {
          ready = ch_try_both(full_at + 8 * s, full_parity, p_at + 8 * (pw & 1), (pw >> 1) & 1);
          if (PARTS != 1 && does_pv && x > 0) ready = ready && mbar_try_wait(o_free, (x - 1) & 1);
        } else {
          ready = mbar_try_wait(&full[s], full_parity);
        }
        if (!__all_sync(0xffffffffu, ready && ok)) {
          ok = ok && ch_wait_slow(&full[s], full_parity, abort_flag, p.err);
          if (wait_p) {
            if (PARTS != 1 && does_pv && x > 0) ok = ok && ch_wait_slow(o_free, (x - 1) & 1, abort_flag, p.err);
            ok = ok && ch_wait_slow(&p_full[2 * t + (pw & 1)], (pw >> 1) & 1, abort_flag, p.err);
          }
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
        }
        tc_fence_after();
        if (has_pv && does_pv) {
          ++pn;
          const uint64_t v = v_desc + s * (2 * C::SLOT >> 4);
          const int sixteens = min(4, (keys - (e - 2) * CH_STEP + 15) / 16);
          if (sixteens == 4) {
#pragma unroll
            for (int part = PARTS - 1; part >= 0; --part)
#pragma unroll
              for (int kk = 0; kk < 4; ++kk)   // (the first over O's old values where they are another item's or, with one tile, step's)
                ch_mma_ta(to, tp + C::P_STEP * b + part * 32 + kk * 8, v + kk * 128, idesc_o, kk || part < PARTS - 1 ? 1u : PARTS == 1 && e > 2, mine);
          } else {
#pragma unroll 1
            for (int part = PARTS - 1; part >= 0; --part)
#pragma unroll 1
              for (int kk = 0; kk < sixteens; ++kk)
                ch_mma_ta(to, tp + C::P_STEP * b + part * 32 + kk * 8, v + kk * 128, idesc_o, kk || part < PARTS - 1 ? 1u : PARTS == 1 && e > 2, mine);
          }
          if (PARTS != 1) ch_commit(pv_at + 8 * b, mine);
        }
        if (has_s && does_s) {
          const uint64_t k = k_desc + s * (2 * C::SLOT >> 4);
#pragma unroll
          for (int part = PARTS - 1; part >= 0; --part)   // (small ones first: the sums round less)
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk)
              ch_mma(ts + CH_STEP * b, q_desc + part * (C::TILE >> 4) + (kk >> 2) * (C::HALF >> 4) + (kk & 3) * 2,
                     k + (kk >> 2) * (C::BOX >> 4) + (kk & 3) * 2, idesc_s, part < PARTS - 1 || kk ? 1u : 0u, mine);
        }
        if (PARTS == 1 || (has_s && does_s)) ch_commit(s_at + 8 * (x % CH_SBARS), mine);
        ch_commit(empty_at + 8 * s, mine);
        if (PARTS == 1 && e == steps - 1) ch_commit(qe_at, mine);
      }
      // the entries that only the other tile uses
#pragma unroll 1
      for (int e = mine_too; e < all && ok; ++e, ++n) {
        wait(&full[n % SLOTS], (n / SLOTS) & 1);
        if (!agree()) break;
        if (lane == 0) mbar_arrive(&empty[n % SLOTS]);
      }
    }
    if (*abort_flag) {   // wait for issued MMAs before shared memory goes away
      if (mine) umma_commit(&drain[t]);
      __syncwarp();
      if (lane == 0) {
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait(&drain[t], 0))
          if (globaltimer_ns() - t0 > WAIT_LIMIT_NS) break;
      }
    }
    __syncwarp();
  } else if (warp >= 4 && (warp >> 2) - 1 < C::TILES) {
    // ---- softmax (and output, or queries): a thread for each row
    const int t = (warp >> 2) - 1, e = warp & 3, rr = e * 32 + lane, gi = rr / G, g = rr % G;
    const uint32_t tl = tmem + ((uint32_t)(e * 32) << 16), ts = tl + C::S_COL(t), tp = tl + C::P_COL(t), to = tl + C::O_COL(t);
    const float c = rsqrtf((float)HD) * 1.4426950408889634f;
    const uint64_t c2 = f2_pack(c, c);
    uint32_t bn = 0, x = 0, pn = 0, in = 0;   // entries of the ring and of the tile, P's, items
    float m = CH_UNSET, l = 0.f;       // reference exponent (log2) and the row's sum relative to it
    // largest of 64 scores, as an exponent
    auto top = [&](const float (&s)[64]) {
      float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
      for (int x = 4; x < 60; x += 8)
#pragma unroll
        for (int y = 0; y < 4; ++y) mx[y] = max3(mx[y], s[x + 2 * y], s[x + 2 * y + 1]);
      return fmaxf(max3(max3(mx[0], s[60], s[61]), max3(mx[1], s[62], s[63]), fmaxf(mx[2], mx[3])) * c, CH_UNSET);
    };
    // keys that the row does not see; last: of the 64
    auto hide = [&](float (&s)[64], int last) {
#pragma unroll
      for (int x = 0; x < 64; ++x)
        if (x >= last) s[x] = -INFINITY;
    };
    // P of a step, and its share of the sum
    auto probabilities = [&](const float (&s)[64], uint32_t at) {
      uint64_t sum[2] = {0, 0};
      const uint64_t m2 = f2_pack(-m, -m);
      constexpr int STEP = PARTS == 1 ? 32 : 16;
#pragma unroll
      for (int x = 0; x < 64; x += STEP) {
        uint32_t u[PARTS][STEP / 2];
#pragma unroll
        for (int y = 0; y < STEP / 2; ++y) {
          float a, b;
          f2_unpack(f2_fma(f2_pack(s[x + 2 * y], s[x + 2 * y + 1]), c2, m2), a, b);
          a = ex2(a);
          b = ex2(b);
          sum[y & 1] = f2_add(sum[y & 1], f2_pack(a, b));
#pragma unroll
          for (int q = 0; q < PARTS; ++q) u[q][y] = q + 1 < PARTS ? take_bf16(a, b) : pack_bf16(a, b);
        }
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
          if constexpr (PARTS == 1) tmem_st16(at + x / 2, u[q]);
          else tmem_st8(at + 32 * q + x / 2, u[q]);
        }
      }
      float l0, l1;
      f2_unpack(f2_add(sum[0], sum[1]), l0, l1);
      l += l0 + l1;
    };
    auto rescale = [&](float f) {
#pragma unroll 1
      for (int x = 0; x < HD; x += 16) {
        float o[16];
        uint32_t u[16];
        tmem_ld16(to + x, o);
        tmem_wait_ld();
#pragma unroll
        for (int y = 0; y < 16; ++y) u[y] = __float_as_uint(o[y] * f);
        tmem_st16(to + x, u);
      }
    };
    ChHead it;
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abort_flag, p.err));
      tc_fence_after();
      return ok;
    };
    auto wait_s = [&](uint32_t x) { return wait(&s_full[CH_SBARS * t + x % CH_SBARS], (x / CH_SBARS) & 1); };   // the tile's entry x
    while (ok && next_item(it)) {
      const int i = t * pt1 + gi;                              // this row's position in the item
      const bool mine = gi < pt1 && i < it.npos;
      const int lim = mine ? (int)min((long long)cap, (long long)it.pos0 + i + 1) : 0x7FFFFFFF;   // keys that it sees
      const int least = __reduce_min_sync(0xffffffffu, lim);
      const int end = item_tiles(it) > t ? item_end(it, t) : 0;
      if (PARTS != 1) {   // the warp's queries, whole rows at a time (the last item's S have all been read here)
        constexpr int LANES = HD / 4, AT_ONCE = 32 / LANES, N = 32 / AT_ONCE;   // lanes of a row, rows of a load, loads (all in flight)
        const long long mine_at = mine ? (long long)(it.row0 + gi) * p.q_ld + (it.hk * G + g) * HD : -1;
        const int dim = lane % LANES * 4;
        float4 f[N];
#pragma unroll
        for (int y = 0; y < N; ++y) {
          const long long at = __shfl_sync(0xffffffffu, mine_at, y * AT_ONCE + lane / LANES);
          f[y] = at >= 0 ? __ldcg(reinterpret_cast<const float4*>(static_cast<const float*>(p.q) + at + dim)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int y = 0; y < N; ++y) {
          const int r = e * 32 + y * AT_ONCE + lane / LANES;
          uint8_t* to = smem + (dim >> 6) * C::HALF + r * 128 + ((((dim >> 3) & 7) ^ (r & 7)) << 4) + (dim & 4) * 2;
#pragma unroll
          for (int q = 0; q < PARTS; ++q) *reinterpret_cast<uint2*>(to + (size_t)q * C::TILE) = make_uint2(take_bf16(f[y].x, f[y].y), take_bf16(f[y].z, f[y].w));
        }
        fence_proxy_async_smem();
        mbar_arrive(q_full);
      }
      m = CH_UNSET, l = 0.f;
#pragma unroll 1
      for (int j = it.kb0; j < end; ++j, ++x, ++pn) {
        if (!wait_s(x)) break;
        const bool there = flags[(bn + (j - it.kb0)) % CH_FLAGS];   // (keys without a page are not attended to)
        float s[CH_STEP];
        tmem_ld32(ts + CH_STEP * (x & 1), s);
        tmem_ld32(ts + CH_STEP * (x & 1) + 32, s + 32);
        tmem_wait_ld();
        if ((j + 1) * CH_STEP > least || !there) hide(s, there ? lim - j * CH_STEP : 0);
        const float mb = top(s);
        const bool grow = mb > m + CH_LAZY;
        float f = 1.f;
        if (__any_sync(0xffffffffu, grow)) {
          if (grow) f = ex2(m - mb), m = mb;
          l *= f;
          if (PARTS == 1 && j > it.kb0) {   // O of the steps before: the last P V came with the next entry
            if (!wait_s(x + 1)) break;
            rescale(f);
          }
        }
        if (PARTS != 1 && pn >= 2 && !wait(&pv_done[pn & 1], ((pn - 2) >> 1) & 1)) break;   // P's place
        if (PARTS != 1) tmem_st1(tl + C::F_COL(pn), f);   // what the total is multiplied by first
        probabilities(s, tp + C::P_STEP * (x & 1));
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&p_full[2 * t + (pn & 1)]);
      }
      if (PARTS == 1 && end > it.kb0) {   // the last two P V's
        for (int y = 0; y < 2; ++y, ++x) wait_s(x);
      }
      bn += it.kb1 - it.kb0 + 2;
      if (!ok) break;
      if constexpr (PARTS != 1) {   // the sums and the reference, to those who write
        const int b = in & 1;
        if (!wait(&l_free[b], ((in >> 1) & 1) ^ 1)) break;
        tmem_st1(tl + C::L_COL + b, l);
        tmem_st1(tl + C::M_COL + b, m);
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&l_full[b]);
        ++in;
      } else {
        const float inv = l == 0.f ? 0.f : 1.0f / l;   // (0: no key of the row has a page)
        const long long at = (long long)(it.row0 + i) * p.out_ld + (it.hk * G + g) * HD;
        const size_t part = it.part >= 0 ? part_at(it.head, it.part) : 0;
        const int pr = t * CH_ROWS + rr;
        if (it.part >= 0 && mine) *ml_of(part, pr) = make_float2(m, l);
        if (end > it.kb0) {
#pragma unroll 1
          for (int x = 0; x < HD; x += 16) {
            float o[16];
            tmem_ld16(to + x, o);
            tmem_wait_ld();
            if (mine && it.part >= 0) {
#pragma unroll
              for (int y = 0; y < 16; y += 4)
                *o_of(part, pr, x + y) = make_float4(o[y], o[y + 1], o[y + 2], o[y + 3]);
            } else if (mine) {
              uint32_t u[8];
#pragma unroll
              for (int y = 0; y < 8; ++y) u[y] = pack_bf16(o[2 * y] * inv, o[2 * y + 1] * inv);
              uint4* d = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + at + x);
              d[0] = make_uint4(u[0], u[1], u[2], u[3]);
              d[1] = make_uint4(u[4], u[5], u[6], u[7]);
            }
          }
        }
        if (it.part >= 0 && !join(it, 4)) break;
        tc_fence_before();   // (O is read: the next item's products may overwrite it once its P has come)
      }
    }
  } else if (PARTS != 1 && warp >= 8) {
    // ---- one tile: the total of O and the output, a thread for each row
    const int e = warp & 3, rr = e * 32 + lane, gi = rr / G, g = rr % G;
    const uint32_t tl = tmem + ((uint32_t)(e * 32) << 16), to = tl + C::O_COL(0);
    uint32_t pn = 0, in = 0;   // steps, items
    ChHead it;
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abort_flag, p.err));
      tc_fence_after();
      return ok;
    };
    while (ok && next_item(it)) {
      const bool mine = gi < pt1 && gi < it.npos;
      float total[HD];
#pragma unroll
      for (int x = 0; x < HD; ++x) total[x] = 0.f;
#pragma unroll 1
      for (int j = it.kb0; j < it.kb1; ++j, ++pn) {
        if (!wait(&pv_done[pn & 1], (pn >> 1) & 1)) break;
        const float f = tmem_ld1(tl + C::F_COL(pn));
#pragma unroll
        for (int x = 0; x < HD; x += 16) {
          float o[16];
          tmem_ld16(to + x, o);
          tmem_wait_ld();
#pragma unroll
          for (int y = 0; y < 16; ++y) total[x + y] = fmaf(total[x + y], f, o[y]);
        }
        tc_fence_before();
        mbar_arrive(o_free);
      }
      const int b = in & 1;
      if (!ok || !wait(&l_full[b], (in >> 1) & 1)) break;
      const float l = tmem_ld1(tl + C::L_COL + b), m = tmem_ld1(tl + C::M_COL + b);
      tmem_wait_ld();
      tc_fence_before();
      mbar_arrive(&l_free[b]);
      ++in;
      if (mine && it.part >= 0) {
        const size_t part = part_at(it.head, it.part);
        *ml_of(part, rr) = make_float2(m, l);
#pragma unroll
        for (int x = 0; x < HD; x += 4) *o_of(part, rr, x) = make_float4(total[x], total[x + 1], total[x + 2], total[x + 3]);
      } else if (mine) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;   // (0: no key of the row has a page)
        float* out = static_cast<float*>(p.out) + (long long)(it.row0 + gi) * p.out_ld + (it.hk * G + g) * HD;
#pragma unroll
        for (int x = 0; x < HD; x += 4) *reinterpret_cast<float4*>(out + x) = make_float4(total[x] * inv, total[x + 1] * inv, total[x + 2] * inv, total[x + 3] * inv);
      }
      if (it.part >= 0 && !join(it, 8)) break;
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int HD, int PARTS>
static cudaError_t ch_prepare() {
  const auto kernel = chunk_attention_kernel<HD, PARTS>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ChCfg<HD, PARTS>::SMEM);
  return e == cudaSuccess ? prefer_shared(kernel) : e;
}
cudaError_t chunk_attention_prepare() {
  cudaError_t e = ch_prepare<64, 1>();
  if (e == cudaSuccess) e = ch_prepare<128, 1>();
  if (e == cudaSuccess) e = ch_prepare<64, 3>();
  if (e == cudaSuccess) e = ch_prepare<128, 3>();
  return e;
}

template <int HD, int PARTS>
static cudaError_t ch_launch(const ChunkAttnParams& p, int num_sms, cudaStream_t st, bool pdl) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(num_sms);
  cfg.blockDim = dim3(CH_THREADS);
  cfg.dynamicSmemBytes = ChCfg<HD, PARTS>::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, chunk_attention_kernel<HD, PARTS>, p);
}
cudaError_t launch_chunk_attention(const ChunkAttnParams& p, int num_sms, cudaStream_t st, bool pdl) {
  if (p.bf16) return p.hd == 64 ? ch_launch<64, 1>(p, num_sms, st, pdl) : ch_launch<128, 1>(p, num_sms, st, pdl);
  return p.hd == 64 ? ch_launch<64, 3>(p, num_sms, st, pdl) : ch_launch<128, 3>(p, num_sms, st, pdl);
}

}  // namespace sdsat
