// Causal attention of the new rows of a ragged batch over pages: flash attention on tcgen05.
//
//   out = sum_t p_t v_t / sum_t p_t,  p_t = exp2(c s_t - m),  s = q K^T,  c = log2(e) / sqrt(hd)
//
// A tile is 128 rows: PT = 128 / G positions of the G query heads that share a cache head, so that K and V are
// loaded once for all of them.  An item is TILES tiles of a sequence and cache head, its work the blocks of 128 keys that its
// rows see.  The items stand in a line, weighed by their keys and a start's cost, and every CTA (one on an SM) takes an
// equal stretch of it, wherever that begins: few rows of long sequences are split along their keys, and causal tiles of
// unequal length leave no SM idle.  An item that several CTAs share leaves partial results (m, sum, O), which a second
// kernel joins in order.  Sequences, lengths and pages are device values, so the plan is made on the device, by one
// warp of each CTA (a scan over the sequences), which then hands items to the others.
//
// bf16 (PARTS = 1, TILES = 2): S, O of both tiles fill TMEM, P lies over its S.  While one tile's 128 threads (a row
// each, no shuffles) work on its scores, the tensor cores run the other tile's products.
// fp32 (PARTS = 3, TILES = 1): queries and probabilities as three bf16 parts (24 bits); P beside S, so that the next
// block's S is computed while this one's P is made.
//
// O is rescaled only when a row's maximum has grown by more than 2^8 since the last time (exact: the reference value
// cancels in the division by the row's sum).
//
// Values that no row may see (behind the last key, up to the 16 keys of a product's step; pages that are not there) take
// part with P = 0 and may hold NaN: they are made zeros in the ring before the product, by the warp that loads.
//
// Warps: 0 loads (TMA), 1 issues the products, 2 plans, 4-7 softmax and output of tile 0, 8-11 of tile 1, or, with one
// tile, the next item's queries.
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace sdsat {

static_assert(KV_PAGE == 64, "a page is one box of keys");
constexpr int CH_BLK = 128;           // keys of a block, rows of a tile
constexpr int CH_THREADS = 384;
constexpr int CH_DESC = 4;            // items handed out ahead
constexpr int CH_FLAGS = 8;           // blocks whose pages' presence is kept
constexpr int CH_START = 192;         // what an item's start costs, in keys
constexpr int CH_LEAST = 384;         // keys (and starts) for which a CTA is worth its while
constexpr float CH_LAZY = 8.0f;       // log2 of the growth of a row maximum that is left unscaled
constexpr float CH_UNSET = -1e30f;    // reference of a row that has seen no key

// partial results of a CTA: slot 0 an item that began in another, slot 1 one that goes on in the next
struct ChRec {
  int row0, npos, hk, last;           // npos 0: none; last: the item ends here
};
struct ChItem {
  int row0, npos, pos0, hk;           // first row, positions, slot of the first; cache head (-1: no more items)
  int seq, kb0, kb1, slot;            // blocks; partial results' place or -1
};

template <int HD, int PARTS>
struct ChCfg {
  static constexpr int TILES = PARTS == 1 ? 2 : 1;
  static constexpr int HALVES = HD / 64;
  static constexpr int BOX = 64 * 128;                      // one TMA box of K or V: 64 keys x 64 dims
  static constexpr int HALF = CH_BLK * 128;                 // 128 rows x 64 dims, 128-byte swizzle
  static constexpr int TILE = HALVES * HALF;
  static constexpr int SLOTS = HD == 128 ? 4 : 8;
  static constexpr size_t OFF_RING = (size_t)TILES * PARTS * TILE;
  static constexpr size_t OFF_BAR = OFF_RING + (size_t)SLOTS * TILE;
  static constexpr int NBAR = 3 * SLOTS + 5 * 2 + 2 + 2 * CH_DESC;
  static constexpr size_t OFF_ITEMS = OFF_BAR + (NBAR + 1) / 2 * 16;
  static constexpr size_t SMEM = 1024 + OFF_ITEMS + CH_DESC * sizeof(ChItem) + CH_FLAGS * 4 + 16;
  static_assert(SMEM <= 232448, "shared memory of one CTA");
  static_assert(OFF_RING >= (CHUNK_MAX_BATCH + 1) * 8, "the plan lies over the queries");
  // TMEM columns
  static constexpr int S_COL(int t) { return 128 * t; }
  static constexpr int P_COL(int t) { return PARTS == 1 ? 128 * t : 128; }
  static constexpr int O_COL(int t) { return PARTS == 1 ? 256 + 128 * t : 320; }
};

size_t chunk_attention_scratch(int num_sms) {
  return (size_t)2 * num_sms * (sizeof(ChRec) / 4 + 2 * CH_BLK * (2 + 128));
}

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

// ---- the plan: sequences of n new positions after `len` slots, items of pt positions -----------
struct ChSeq {
  int first, n, len;
};
__device__ __forceinline__ ChSeq ch_sequence(const ChunkAttnParams& p, int s) {
  ChSeq q;
  q.first = __ldcg(p.start + s);
  q.n = __ldcg(p.start + s + 1) - q.first;
  q.len = min(max(__ldcg(p.len + s), 0), p.ld * KV_PAGE);
  return q;
}
// cost of a head's items before item t, and of all of them
__device__ __forceinline__ long long ch_before(const ChSeq& q, int pt, int t) {
  return (long long)t * (q.len + CH_START) + (long long)pt * ((long long)t * (t + 1) / 2);
}
__device__ __forceinline__ long long ch_cost(const ChSeq& q, int pt) {
  if (q.n <= 0) return 0;
  const int t = (q.n + pt - 1) / pt;
  return ch_before(q, pt, t - 1) + q.len + CH_START + q.n;
}
__device__ __forceinline__ int ch_keys(const ChSeq& q, int pt, int cap, int t) { return min((long long)cap, (long long)q.len + min((long long)q.n, (long long)(t + 1) * pt)); }

struct ChPlace {
  int s, hk, t, kb;   // s = b: behind the last item
};

template <int HD, int PARTS>
__global__ void __launch_bounds__(CH_THREADS, 1) chunk_attention_kernel(const __grid_constant__ ChunkAttnParams p) {
  using C = ChCfg<HD, PARTS>;
  constexpr int SLOTS = C::SLOTS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = smem + C::OFF_RING;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);   // [SLOTS] K or V block landed
  uint64_t* empty = full + SLOTS;         // [SLOTS] its products are done
  uint64_t* z_done = empty + SLOTS;       // [SLOTS] values that no row may see are zeros (of blocks that have some)
  uint64_t* q_full = z_done + SLOTS;      // [2] per tile: Q is there
  uint64_t* q_empty = q_full + 2;         // [2] the item's last S is complete
  uint64_t* s_full = q_empty + 2;         // [2] S of a block is complete (and everything issued before it)
  uint64_t* p_full = s_full + 2;          // [2] P is in TMEM, O is rescaled (128 threads)
  uint64_t* o_full = p_full + 2;          // [2] two tiles: the item's last product is complete
  uint64_t* pv_done = o_full + 2;         // one tile: a block's P V is complete
  uint64_t* drain = pv_done + 1;
  uint64_t* d_full = drain + 1;           // [CH_DESC] an item's description is there
  uint64_t* d_empty = d_full + CH_DESC;   // [CH_DESC] all have read it
  ChItem* items = reinterpret_cast<ChItem*>(smem + C::OFF_ITEMS);
  uint32_t* flags = reinterpret_cast<uint32_t*>(items + CH_DESC);   // [CH_FLAGS] by block: which of its two pages there are
  uint32_t* tmem_slot = flags + CH_FLAGS;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  long long* plan = reinterpret_cast<long long*>(smem);             // [b + 1] cost before each sequence

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = p.H / p.Hk, pt1 = CH_BLK / G, pt = C::TILES * pt1, cap = p.ld * KV_PAGE;
  if (threadIdx.x == 0) {
    for (int s = 0; s < SLOTS; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
      mbar_init(&z_done[s], 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(&q_full[t], PARTS == 1 ? 1 : 128);
      mbar_init(&q_empty[t], 1);
      mbar_init(&s_full[t], 1);
      mbar_init(&p_full[t], 128);
      mbar_init(&o_full[t], 1);
    }
    mbar_init(pv_done, 1);
    mbar_init(drain, 1);
    for (int i = 0; i < CH_DESC; ++i) {
      mbar_init(&d_full[i], 1);
      mbar_init(&d_empty[i], 10);
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

  ChRec* recs = reinterpret_cast<ChRec*>(p.part);                             // [2 ctas]
  float2* part_ml = reinterpret_cast<float2*>(recs + 2 * gridDim.x);          // [2 ctas][256]
  float* part_o = reinterpret_cast<float*>(part_ml + 2 * gridDim.x * 2 * CH_BLK);   // [2 ctas][256][HD]

  // an item's geometry
  auto item_keys = [&](const ChItem& it, int t) { return (int)min((long long)cap, (long long)it.pos0 + min(it.npos, (t + 1) * pt1)); };
  auto item_tiles = [&](const ChItem& it) { return C::TILES == 2 && it.npos > pt1 ? 2 : 1; };
  // blocks of tile t up to which this part goes
  auto item_end = [&](const ChItem& it, int t) { return min(it.kb1, (item_keys(it, t) + CH_BLK - 1) / CH_BLK); };
  // the last tile's block has values behind its last key in a step of 16
  auto item_tail = [&](const ChItem& it, int j) {
    const int k = item_keys(it, item_tiles(it) - 1);
    return k % 16 != 0 && j == k / CH_BLK;
  };
  uint32_t d_phase = 0;   // items read
  auto next_item = [&](ChItem& it) {   // by a warp
    const int d = d_phase % CH_DESC;
    const bool ok = __all_sync(0xffffffffu, mbar_wait_bounded(&d_full[d], (d_phase / CH_DESC) & 1, abort_flag, p.err));
    if (!ok) return false;
    it = items[d];
    __syncwarp();
    if (lane == 0) mbar_arrive(&d_empty[d]);
    ++d_phase;
    return it.hk >= 0;
  };

  if (warp == 2) {
    // ---- the plan
    long long total = 0;
    bool bad = false, past = false;
    for (int s0 = 0; s0 < p.b; s0 += 32) {
      const int s = s0 + lane;
      long long cost = 0;
      if (s < p.b) {
        const int a = __ldcg(p.start + s), z = __ldcg(p.start + s + 1), len = __ldcg(p.len + s);
        bad |= a < 0 || z < a || z > p.rows;
        past |= z > a && (long long)max(len, 0) + (z - a) > cap;
        ChSeq q = {a, z - a, min(max(len, 0), cap)};
        if (z >= a) cost = ch_cost(q, pt) * p.Hk;
      }
      long long sum = cost;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += x;
      }
      if (s < p.b) plan[s] = total + sum - cost;
      total += __shfl_sync(0xffffffffu, sum, 31);
    }
    bad = __any_sync(0xffffffffu, bad);
    past = __any_sync(0xffffffffu, past);
    if (lane == 0) {
      plan[p.b] = total;
      if (bad) set_error(p.err, ERR_CAPACITY);
      else if (past) set_error(p.err, ERR_PAGE);
    }
    __syncwarp();
    const int ctas = (int)max(1ll, min((long long)gridDim.x, total / CH_LEAST)), cta = blockIdx.x;
    // the first sequence from s on that has rows (b: none); the plan is gone once items are handed out
    auto with_rows = [&](int s) {
      for (; s < p.b; s += 32) {
        const unsigned some = __ballot_sync(0xffffffffu, s + lane < p.b && __ldcg(p.start + min(s + lane, p.b - 1)) < __ldcg(p.start + min(s + lane, p.b - 1) + 1));
        if (some) return s + __ffs(some) - 1;
      }
      return p.b;
    };
    auto after = [&](ChPlace a, const ChSeq& q) {   // the item that follows
      a.kb = 0;
      if (++a.t * pt >= q.n) {
        a.t = 0;
        if (++a.hk == p.Hk) a.hk = 0, a.s = with_rows(a.s + 1);
      }
      return a;
    };
    // the c-th of the borders between the CTAs' stretches
    auto border = [&](int c) {
      ChPlace a = {p.b, 0, 0, 0};
      if (c >= ctas || total == 0) return a;
      const long long x = total / ctas * c + total % ctas * c / ctas;
      int lo = 0, hi = p.b;   // the last sequence whose cost before it is at most x
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (plan[mid] <= x) lo = mid;
        else hi = mid;
      }
      a.s = lo;
      const ChSeq q = ch_sequence(p, lo);
      const long long of_head = ch_cost(q, pt);
      long long rem = x - plan[lo];
      a.hk = (int)(rem / of_head);
      rem -= a.hk * of_head;
      lo = 0, hi = (q.n + pt - 1) / pt;
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (ch_before(q, pt, mid) <= rem) lo = mid;
        else hi = mid;
      }
      a.t = lo;
      // parts of at least two blocks
      const int blocks = (ch_keys(q, pt, cap, a.t) + CH_BLK - 1) / CH_BLK;
      const long long kb = (rem - ch_before(q, pt, a.t) - CH_START + CH_BLK / 2) / CH_BLK;
      a.kb = kb < 2 ? 0 : (int)kb;
      if (a.kb > blocks - 2 && a.kb > 0) a = after(a, q);
      return a;
    };
    const ChRec none = {0, 0, 0, 0};
    ChRec left = none, right = none;
    ChPlace a = {p.b, 0, 0, 0}, z = a;
    if (!bad && cta < ctas) {
      a = border(cta);
      z = border(cta + 1);
    }
    fence_proxy_async_smem();   // the plan's place is the queries': read before, written by TMA after
    uint32_t n = 0;
    ChPlace end = z;
    bool ok = true;
    while (ok) {
      const bool more = a.s < p.b && !(a.s == end.s && a.hk == end.hk && a.t == end.t && a.kb >= end.kb);
      ChItem it = {0, 0, 0, -1, 0, 0, 0, -1};
      ChSeq q = {0, 0, 0};
      bool stop = true;
      if (more) {
        q = ch_sequence(p, a.s);
        const int blocks = (ch_keys(q, pt, cap, a.t) + CH_BLK - 1) / CH_BLK;
        it.row0 = q.first + a.t * pt;
        it.npos = min(pt, q.n - a.t * pt);
        it.pos0 = q.len + a.t * pt;
        it.hk = a.hk;
        it.seq = a.s;
        it.kb0 = a.kb;
        stop = a.s == end.s && a.hk == end.hk && a.t == end.t;
        it.kb1 = stop ? end.kb : blocks;
        if (it.kb0 > 0) {
          it.slot = 2 * cta;
          left = ChRec{it.row0, it.npos, it.hk, it.kb1 == blocks};
        } else if (it.kb1 < blocks) {
          it.slot = 2 * cta + 1;
          right = ChRec{it.row0, it.npos, it.hk, 0};
        }
      }
      const int d = n % CH_DESC;
      ok = __all_sync(0xffffffffu, mbar_wait_bounded(&d_empty[d], ((n / CH_DESC) & 1) ^ 1, abort_flag, p.err));
      if (!ok) break;
      if (lane == 0) {
        items[d] = it;
        mbar_arrive(&d_full[d]);
      }
      ++n;
      if (!more) break;
      if (stop) a = z = end = ChPlace{p.b, 0, 0, 0};
      else a = after(a, q);
    }
    if (lane == 0) {
      recs[2 * cta] = left;
      recs[2 * cta + 1] = right;
    }
  } else if (warp == 0) {
    // ---- loads
    const uint64_t pol = l2_policy_evict_normal();
    uint32_t n = 0, qn[2] = {0, 0};   // ring entries used, Q tiles loaded
    bool ok = true;
    // a block whose values wait to be made zeros
    int z_slot = -1, z_there = 0;
    uint32_t z_parity = 0, z_pages = 3;
    auto make_zeros = [&]() {
      if (z_slot < 0) return;
      if (mbar_wait_bounded(&full[z_slot], z_parity, abort_flag, p.err)) {
        constexpr int CHUNKS = HD / 8;   // of 16 bytes, of a key
        for (int z = lane; z < (z_there + 15) / 16 * 16 * CHUNKS; z += 32) {
          const int at = z / CHUNKS, i = z % CHUNKS;
          if (at >= z_there || !((z_pages >> (at / KV_PAGE)) & 1u))
            *reinterpret_cast<uint4*>(ring + (size_t)z_slot * C::TILE + (i >> 3) * C::HALF + at * 128 + (((i & 7) ^ (at & 7)) << 4)) =
                make_uint4(0u, 0u, 0u, 0u);
        }
        fence_proxy_async_smem();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&z_done[z_slot]);
      z_slot = -1;
    };
    // (values that a product waits for are made zeros before anything waits for that product)
    auto acquire = [&](uint64_t* bar, uint32_t parity) {
      if (!__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) {
        make_zeros();
        ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abort_flag, p.err));
      }
      return ok;
    };
    ChItem it;
    while (ok) {
      if (z_slot >= 0 && !__all_sync(0xffffffffu, mbar_try_wait(&d_full[d_phase % CH_DESC], (d_phase / CH_DESC) & 1))) make_zeros();
      if (!next_item(it)) break;
      const int nt = item_tiles(it), keys = item_keys(it, nt - 1);
      if (PARTS == 1) {
        for (int t = 0; t < nt && ok; ++t) {
          if (item_end(it, t) <= it.kb0) continue;
          if (!acquire(&q_empty[t], (qn[t] & 1) ^ 1)) break;
          ++qn[t];
          if (lane == 0) {
            mbar_arrive_expect_tx(&q_full[t], C::HALVES * 128 * G * pt1);
            for (int hh = 0; hh < C::HALVES; ++hh)
              tma_load_3d(smem + (size_t)t * C::TILE + hh * C::HALF, &p.qmap, &q_full[t], hh * 64, it.hk * G, it.row0 + t * pt1);
          }
        }
      }
      // the pages of 16 blocks at a time, the next ones asked for ahead
      const int* row = p.table + (size_t)it.seq * p.ld;
      auto pages = [&](int j) { return 2 * j + lane < p.ld ? __ldcg(row + 2 * j + lane) : -1; };
      int now = pages(it.kb0), next = pages(it.kb0 + 16), base = it.kb0;
      for (int j = it.kb0; j < it.kb1 && ok; ++j) {
        if (j == base + 16) base = j, now = next, next = pages(j + 16);
        int page[2];
        uint32_t there = 0, load = 0;
        for (int b = 0; b < 2; ++b) {
          page[b] = __shfl_sync(0xffffffffu, now, 2 * (j - base) + b);
          const bool wanted = j * CH_BLK + b * KV_PAGE < keys, in = page[b] >= 0 && page[b] < p.n_pages;
          if (wanted && in) load |= 1u << b;
          if (!wanted || in) there |= 1u << b;
          else if (lane == 0) set_error(p.err, ERR_PAGE);
        }
        const uint32_t bytes = __popc(load) * C::HALVES * C::BOX;
        for (int which = 0; which < 2; ++which, ++n) {
          const int s = n % SLOTS;
          if (!acquire(&empty[s], ((n / SLOTS) & 1) ^ 1)) break;
          if (lane == 0) {
            if (which == 0) flags[(n / 2) % CH_FLAGS] = there;
            mbar_arrive_expect_tx(&full[s], bytes);
            for (int b = 0; b < 2; ++b)
              if ((load >> b) & 1u)
                for (int hh = 0; hh < C::HALVES; ++hh)
                  tma_load_2d(ring + (size_t)s * C::TILE + hh * C::HALF + b * C::BOX, which ? &p.vmap : &p.kmap, &full[s], hh * 64,
                              (page[b] * p.Hk + it.hk) * KV_PAGE, pol);
          }
          __syncwarp();
        }
        if (!ok) break;
        if (there != 3u || item_tail(it, j)) {
          make_zeros();   // (one at a time)
          z_slot = (n - 1) % SLOTS;
          z_parity = ((n - 1) / SLOTS) & 1;
          z_there = min(CH_BLK, keys - j * CH_BLK);
          z_pages = there;
        }
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
      for (uint32_t i = n > SLOTS ? n - SLOTS : 0; i < n; ++i) land(&full[i % SLOTS], (i / SLOTS) & 1);
    }
  } else if (warp == 1) {
    // ---- products
    constexpr uint32_t idesc_s = idesc_bf16_f32(128, CH_BLK);
    constexpr uint32_t idesc_o = idesc_bf16_f32(128, HD) | (1u << 16);   // B is MN-major
    const uint32_t mine = ch_elect();
    const uint64_t q_desc = sdesc_sw128(smem_u32(smem)), k_desc = sdesc_sw128(smem_u32(ring)), v_desc = sdesc_sw128_mn(smem_u32(ring), C::HALF);
    bool ok = true;
    uint32_t n = 0, qn[2] = {0, 0}, pn[2] = {0, 0}, zn = 0;   // blocks; per tile: Q tiles, P's; z_done phases (bits)
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abort_flag, p.err));
      tc_fence_after();
      return ok;
    };
    auto commit = [&](uint64_t* bar) {
      if (mine) umma_commit(bar);
      __syncwarp();
    };
    auto qk = [&](int t, uint32_t blk) {
      const uint64_t k = k_desc + (uint64_t)((2 * blk) % SLOTS) * (C::TILE >> 4), q = q_desc + (uint64_t)(PARTS * t) * (C::TILE >> 4);
#pragma unroll 1
      for (int part = PARTS - 1; part >= 0; --part)   // (small ones first: the sums round less)
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
          const uint32_t o = (kk >> 2) * (C::HALF >> 4) + (kk & 3) * 2;
          ch_mma(tmem + C::S_COL(t), q + part * (C::TILE >> 4) + o, k + o, idesc_s, part < PARTS - 1 || kk ? 1u : 0u, mine);
        }
      commit(&s_full[t]);
    };
    auto pv = [&](int t, uint32_t blk, int steps, bool first) {
      const uint64_t v = v_desc + (uint64_t)((2 * blk + 1) % SLOTS) * (C::TILE >> 4);
#pragma unroll 1
      for (int part = PARTS - 1; part >= 0; --part) {
        const uint32_t a = tmem + C::P_COL(t) + part * 64;
        const uint32_t acc = !first || part < PARTS - 1 ? 1u : 0u;
        if (steps == CH_BLK / 16) {
#pragma unroll
          for (int kk = 0; kk < CH_BLK / 16; ++kk) ch_mma_ta(tmem + C::O_COL(t), a + kk * 8, v + kk * 128, idesc_o, kk ? 1u : acc, mine);
        } else {
#pragma unroll 1
          for (int kk = 0; kk < steps; ++kk) ch_mma_ta(tmem + C::O_COL(t), a + kk * 8, v + kk * 128, idesc_o, kk ? 1u : acc, mine);
        }
      }
    };
    ChItem it;
    while (ok && next_item(it)) {
      const int nt = item_tiles(it);
      const int end[2] = {item_end(it, 0), item_end(it, nt - 1)};
#pragma unroll
      for (int t = 0; t < C::TILES; ++t)
        if (t < nt && end[t] > it.kb0) wait(&q_full[t], qn[t]++ & 1);
      const uint32_t n0 = n;   // block kb0 is the ring's n0-th
      auto has_zeros = [&](uint32_t blk, int j) { return flags[blk % CH_FLAGS] != 3u || item_tail(it, j); };
      // step j: per tile, block j - 1's P V and then block j's S over the P that it has read (one tile: block j's S, into a
      // place of its own, and then block j - 1's P V); the last tile has every block, so its products release V of block
      // j - 1 and K of block j
#pragma unroll 1
      for (int j = it.kb0; j <= it.kb1 && ok; ++j) {
        const uint32_t blk = n0 + (j - it.kb0);
#pragma unroll
        for (int t = 0; t < C::TILES; ++t) {
          if (t >= nt) break;
          const bool has_pv = j > it.kb0 && j <= end[t], has_qk = j < end[t];
          auto do_pv = [&]() {
            const int vs = (2 * blk - 1) % SLOTS;
            if (!wait(&full[vs], ((2 * blk - 1) / SLOTS) & 1)) return;
            const bool zeros = has_zeros(blk - 1, j - 1);
            if (zeros && !wait(&z_done[vs], (zn >> vs) & 1)) return;
            if (PARTS == 1 && !wait(&p_full[t], pn[t]++ & 1)) return;
            pv(t, blk - 1, min(CH_BLK / 16, (item_keys(it, t) - (j - 1) * CH_BLK + 15) / 16), j - 1 == it.kb0);
            if (PARTS != 1) commit(pv_done);
            else if (j == end[t]) commit(&o_full[t]);
            if (t == nt - 1) {
              if (zeros) zn ^= 1u << vs;
              commit(&empty[vs]);
            }
          };
          auto do_qk = [&]() {
            const int ks = (2 * blk) % SLOTS;
            if (!wait(&full[ks], (2 * blk / SLOTS) & 1)) return;
            qk(t, blk);
            if (j == end[t] - 1) commit(&q_empty[t]);
            if (t == nt - 1) commit(&empty[ks]);
          };
          if (PARTS == 1) {
            if (has_pv) do_pv();
            if (has_qk && ok) do_qk();
          } else {
            if (has_pv) wait(&p_full[t], pn[t]++ & 1);   // (S has been read, too)
            if (has_qk && ok) do_qk();
            if (has_pv && ok) do_pv();
          }
        }
      }
      n = n0 + (it.kb1 - it.kb0);
    }
    if (*abort_flag) {   // wait for issued MMAs before shared memory goes away
      commit(drain);
      if (lane == 0) {
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait(drain, 0))
          if (globaltimer_ns() - t0 > WAIT_LIMIT_NS) break;
      }
    }
    __syncwarp();
  } else if (warp >= 4 && (warp >> 2) - 1 < C::TILES) {
    // ---- softmax and output: a thread for each row
    const int t = (warp >> 2) - 1, e = warp & 3, rr = e * 32 + lane, gi = rr / G, g = rr % G;
    const uint32_t lane_off = (uint32_t)(e * 32) << 16;
    const uint32_t ts = tmem + lane_off + C::S_COL(t), tp = tmem + lane_off + C::P_COL(t), to = tmem + lane_off + C::O_COL(t);
    const float c = rsqrtf((float)HD) * 1.4426950408889634f;
    uint32_t sn = 0, on = 0, vn = 0;   // S's read, items done, P V's waited for
    uint32_t bn = 0;                   // blocks of the items before (for flags)
    ChItem it;
    bool ok = true;
    while (ok && next_item(it)) {
      const int i = t * pt1 + gi;                              // this row's position in the item
      const bool mine = gi < pt1 && i < it.npos;
      const int lim = mine ? (int)min((long long)cap, (long long)it.pos0 + i + 1) : 0x7FFFFFFF;   // keys that it sees
      const int least = __reduce_min_sync(0xffffffffu, lim);
      const int end = item_tiles(it) > t ? item_end(it, t) : 0;
      float m = CH_UNSET, l = 0.f;   // reference exponent (log2) and the row's sum relative to it
      for (int j = it.kb0; j < end; ++j) {
        ok = __all_sync(0xffffffffu, mbar_wait_bounded(&s_full[t], sn++ & 1, abort_flag, p.err));
        if (!ok) break;
        tc_fence_after();
        float s[CH_BLK];
#pragma unroll
        for (int x = 0; x < 4; ++x) tmem_ld32(ts + 32 * x, s + 32 * x);
        tmem_wait_ld();
        if ((j + 1) * CH_BLK > least) {
          const int last = lim - j * CH_BLK;
#pragma unroll
          for (int x = 0; x < CH_BLK; ++x)
            if (x >= last) s[x] = -INFINITY;
        }
        const uint32_t there = flags[(bn + (j - it.kb0)) % CH_FLAGS];
        if (there != 3u) {   // keys without a page are not attended to
#pragma unroll
          for (int x = 0; x < CH_BLK; ++x)
            if (!((there >> (x / KV_PAGE)) & 1u)) s[x] = -INFINITY;
        }
        float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int x = 4; x < CH_BLK - 4; x += 8)
#pragma unroll
          for (int y = 0; y < 4; ++y) mx[y] = max3(mx[y], s[x + 2 * y], s[x + 2 * y + 1]);
        const float mb = fmaxf(max3(max3(mx[0], s[CH_BLK - 4], s[CH_BLK - 3]), max3(mx[1], s[CH_BLK - 2], s[CH_BLK - 1]), fmaxf(mx[2], mx[3])) * c, CH_UNSET);
        // two tiles: the S that is ready was issued after block j - 1's P V; one tile: that is waited for
        if (PARTS != 1 && j > it.kb0) {
          ok = __all_sync(0xffffffffu, mbar_wait_bounded(pv_done, vn++ & 1, abort_flag, p.err));
          if (!ok) break;
          tc_fence_after();
        }
        if (j == it.kb0) {
          m = mb;
        } else {
          const bool grow = mb > m + CH_LAZY;
          if (__any_sync(0xffffffffu, grow)) {
            const float f = grow ? ex2(m - mb) : 1.f;
            l *= f;
            if (grow) m = mb;
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
          }
        }
        uint64_t sum[2] = {0, 0};
        const uint64_t c2 = f2_pack(c, c), m2 = f2_pack(-m, -m);
#pragma unroll
        for (int x = 0; x < CH_BLK; x += 32) {
          uint32_t u[PARTS][16];
#pragma unroll
          for (int y = 0; y < 16; ++y) {
            float a, b;
            f2_unpack(f2_fma(f2_pack(s[x + 2 * y], s[x + 2 * y + 1]), c2, m2), a, b);
            a = ex2(a);
            b = ex2(b);
            sum[y & 1] = f2_add(sum[y & 1], f2_pack(a, b));
#pragma unroll
            for (int q = 0; q < PARTS; ++q) u[q][y] = q + 1 < PARTS ? take_bf16(a, b) : pack_bf16(a, b);
          }
#pragma unroll
          for (int q = 0; q < PARTS; ++q) tmem_st16(tp + 64 * q + x / 2, u[q]);
        }
        float l0, l1;
        f2_unpack(f2_add(sum[0], sum[1]), l0, l1);
        l += l0 + l1;
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&p_full[t]);
      }
      bn += it.kb1 - it.kb0;
      if (!ok) break;
      if (end > it.kb0) {
        ok = __all_sync(0xffffffffu, PARTS == 1 ? mbar_wait_bounded(&o_full[t], on++ & 1, abort_flag, p.err)
                                                : mbar_wait_bounded(pv_done, vn++ & 1, abort_flag, p.err));
        if (!ok) break;
        tc_fence_after();
      }
      if (it.slot >= 0) {
        const size_t at = (size_t)it.slot * 2 * CH_BLK + t * CH_BLK + rr;
        if (mine) part_ml[at] = make_float2(m, l);
        if (end > it.kb0) {
#pragma unroll 1
          for (int x = 0; x < HD; x += 16) {
            float o[16];
            tmem_ld16(to + x, o);
            tmem_wait_ld();
            if (mine)
#pragma unroll
              for (int y = 0; y < 16; y += 4) *reinterpret_cast<float4*>(part_o + at * HD + x + y) = make_float4(o[y], o[y + 1], o[y + 2], o[y + 3]);
          }
        }
      } else if (end > it.kb0) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;   // (0: no key of the row has a page)
        const long long at = (long long)(it.row0 + i) * p.out_ld + (it.hk * G + g) * HD;
#pragma unroll 1
        for (int x = 0; x < HD; x += 16) {
          float o[16];
          tmem_ld16(to + x, o);
          tmem_wait_ld();
          if (mine) {
            if (PARTS == 1) {
              uint32_t u[8];
#pragma unroll
              for (int y = 0; y < 8; ++y) u[y] = pack_bf16(o[2 * y] * inv, o[2 * y + 1] * inv);
              uint4* d = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + at + x);
              d[0] = make_uint4(u[0], u[1], u[2], u[3]);
              d[1] = make_uint4(u[4], u[5], u[6], u[7]);
            } else {
#pragma unroll
              for (int y = 0; y < 16; y += 4)
                *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at + x + y) =
                    make_float4(o[y] * inv, o[y + 1] * inv, o[y + 2] * inv, o[y + 3] * inv);
            }
          }
        }
      }
      tc_fence_before();   // (O is read: the next item's products may overwrite it once its P has come)
    }
  } else if (PARTS != 1 && warp >= 8) {
    // ---- queries in three parts: a thread for each row
    const int rr = (int)threadIdx.x - 256, gi = rr / G, g = rr % G;
    uint32_t qn = 0;
    ChItem it;
    while (next_item(it)) {
      const bool mine = gi < pt1 && gi < it.npos;
      const float* src = static_cast<const float*>(p.q) + (long long)(it.row0 + gi) * p.q_ld + (it.hk * G + g) * HD;
      if (!__all_sync(0xffffffffu, mbar_wait_bounded(q_empty, (qn & 1) ^ 1, abort_flag, p.err))) break;
      ++qn;
#pragma unroll 2
      for (int x = 0; x < HD; x += 8) {
        float4 f[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
        if (mine) {
          f[0] = __ldcg(reinterpret_cast<const float4*>(src + x));
          f[1] = __ldcg(reinterpret_cast<const float4*>(src + x + 4));
        }
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
          const uint4 u = make_uint4(take_bf16(f[0].x, f[0].y), take_bf16(f[0].z, f[0].w), take_bf16(f[1].x, f[1].y), take_bf16(f[1].z, f[1].w));
          *reinterpret_cast<uint4*>(smem + (size_t)q * C::TILE + (x >> 6) * C::HALF + rr * 128 + ((((x >> 3) & 7) ^ (rr & 7)) << 4)) = u;
        }
      }
      fence_proxy_async_smem();
      mbar_arrive(q_full);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// Joins the parts of the items that several CTAs shared: item a is the one that goes on behind CTA a's stretch, its parts
// those of a (slot 1) and of the CTAs that follow (slot 0) up to the one that ends it.  A warp takes CM_ROWS rows, whose
// loads are in flight together; the parts' references and sums are on its lanes.
constexpr int CM_WARPS = 8, CM_ROWS = 4;
template <int HD, bool BF16>
__global__ void __launch_bounds__(CM_WARPS * 32) chunk_merge_kernel(const __grid_constant__ ChunkAttnParams p, int ctas, int tiles) {
  constexpr int E = HD / 32;
  const int lane = threadIdx.x & 31;
  const int groups = tiles * CH_BLK / (CM_WARPS * CM_ROWS), a = blockIdx.x / groups;
  const int rr0 = (blockIdx.x % groups * CM_WARPS + (threadIdx.x >> 5)) * CM_ROWS;
  const int G = p.H / p.Hk, pt1 = CH_BLK / G;
  pdl_trigger();
  pdl_wait();
  const ChRec* recs = reinterpret_cast<const ChRec*>(p.part);
  const float2* part_ml = reinterpret_cast<const float2*>(recs + 2 * ctas);
  const float* part_o = reinterpret_cast<const float*>(part_ml + 2 * ctas * 2 * CH_BLK);
  const int4 r = __ldcg(reinterpret_cast<const int4*>(recs + 2 * a + 1));   // row0, npos, hk
  int i[CM_ROWS];   // positions in the item, -1: no row of it
  bool some = false;
#pragma unroll
  for (int y = 0; y < CM_ROWS; ++y) {
    const int rr = rr0 + y, gi = rr % CH_BLK / G;
    i[y] = gi < pt1 && rr / CH_BLK * pt1 + gi < r.y ? rr / CH_BLK * pt1 + gi : -1;
    some |= i[y] >= 0;
  }
  if (!some) return;
  // the last of the parts' CTAs
  int last = a;
  for (int c0 = a + 1; last == a && c0 < ctas; c0 += 32) {
    const int c = c0 + lane;
    const unsigned ends = __ballot_sync(0xffffffffu, c < ctas && __ldcg(reinterpret_cast<const int4*>(recs + 2 * min(c, ctas - 1))).w);
    if (ends) last = c0 + __ffs(ends) - 1;
  }
  const int n = 1 + last - a;
  auto place = [&](int k) { return (size_t)(k ? 2 * (a + k) : 2 * a + 1) * 2 * CH_BLK + rr0; };
  float m[CM_ROWS], l[CM_ROWS], acc[CM_ROWS][E];
#pragma unroll
  for (int y = 0; y < CM_ROWS; ++y) {
    m[y] = CH_UNSET;
    l[y] = 0.f;
#pragma unroll
    for (int x = 0; x < E; ++x) acc[y][x] = 0.f;
  }
  for (int k0 = 0; k0 < n; k0 += 32) {
    const int here = min(32, n - k0);
    float w[CM_ROWS];
#pragma unroll
    for (int y = 0; y < CM_ROWS; ++y) {
      const float2 ml = lane < here && i[y] >= 0 ? __ldcg(part_ml + place(k0 + lane) + y) : make_float2(CH_UNSET, 0.f);
      float top = ml.y > 0.f ? fmaxf(ml.x, m[y]) : m[y];   // (a part that saw no key of the row has a sum of 0)
#pragma unroll
      for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      w[y] = ml.y > 0.f ? ex2(ml.x - top) : 0.f;
      float sum = ml.y * w[y];
#pragma unroll
      for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      const float f = ex2(m[y] - top);
      l[y] = fmaf(l[y], f, sum);
      m[y] = top;
#pragma unroll
      for (int x = 0; x < E; ++x) acc[y][x] *= f;
    }
#pragma unroll 4
    for (int k = 0; k < here; ++k)
#pragma unroll
      for (int y = 0; y < CM_ROWS; ++y) {
        const float f = __shfl_sync(0xffffffffu, w[y], k);
        if (f == 0.f) continue;   // (and maybe nothing was written)
        const float* o = part_o + (place(k0 + k) + y) * HD + lane * E;
        float v[E];
        if (E == 4) {
          const float4 q = __ldcg(reinterpret_cast<const float4*>(o));
          v[0] = q.x, v[1] = q.y, v[E - 2] = q.z, v[E - 1] = q.w;
        } else {
          const float2 q = __ldcg(reinterpret_cast<const float2*>(o));
          v[0] = q.x, v[1] = q.y;
        }
#pragma unroll
        for (int x = 0; x < E; ++x) acc[y][x] = fmaf(v[x], f, acc[y][x]);
      }
  }
#pragma unroll
  for (int y = 0; y < CM_ROWS; ++y) {
    if (i[y] < 0) continue;
    const float inv = l[y] == 0.f ? 0.f : 1.0f / l[y];
    const long long at = (long long)(r.x + i[y]) * p.out_ld + (r.z * G + (rr0 + y) % CH_BLK % G) * HD + lane * E;
#pragma unroll
    for (int x = 0; x < E; x += 2) {
      if (BF16) *reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(p.out) + at + x) = pack_bf16(acc[y][x] * inv, acc[y][x + 1] * inv);
      else *reinterpret_cast<float2*>(static_cast<float*>(p.out) + at + x) = make_float2(acc[y][x] * inv, acc[y][x + 1] * inv);
    }
  }
}

template <int HD, int PARTS>
static cudaError_t ch_prepare() {
  const auto kernel = chunk_attention_kernel<HD, PARTS>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ChCfg<HD, PARTS>::SMEM);
  if (e == cudaSuccess) e = prefer_shared(kernel);
  return e == cudaSuccess ? prefer_shared(chunk_merge_kernel<HD, PARTS == 1>) : e;
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
  const cudaError_t e = cudaLaunchKernelEx(&cfg, chunk_attention_kernel<HD, PARTS>, p);
  // (an item of fewer than four blocks is not split)
  if (e != cudaSuccess || ((long long)p.ld * KV_PAGE + CH_BLK - 1) / CH_BLK < 4) return e;
  constexpr int TILES = ChCfg<HD, PARTS>::TILES;
  cfg.gridDim = dim3(num_sms * (TILES * CH_BLK / (CM_WARPS * CM_ROWS)));
  cfg.blockDim = dim3(CM_WARPS * 32);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, chunk_merge_kernel<HD, PARTS == 1>, p, num_sms, TILES);
}
cudaError_t launch_chunk_attention(const ChunkAttnParams& p, int num_sms, cudaStream_t st, bool pdl) {
  if (p.bf16) return p.hd == 64 ? ch_launch<64, 1>(p, num_sms, st, pdl) : ch_launch<128, 1>(p, num_sms, st, pdl);
  return p.hd == 64 ? ch_launch<64, 3>(p, num_sms, st, pdl) : ch_launch<128, 3>(p, num_sms, st, pdl);
}

}  // namespace sdsat
