// Log probabilities of given tokens, their ranks, the entropy and the best alternatives of rows of
// logits.
//
// With m the row's maximum, d_i = (l_i - m) / T and S = sum_i e^{d_i}:
//   log p_t = d_t - log S        entropy = log S - (sum_i e^{d_i} d_i) / S
//   rank_t  = 1 + |{i : l_i > l_t, or l_i = l_t and i < t}|
// and the n_top ids of largest logit, the lower id first among equal ones.  Sums are fp32.  A NaN
// logit counts as -inf and sets ERR_NAN_LOGITS; where l_i = m the difference is 0, so a row whose
// maximum is +inf shares its mass among those ids; a row of -inf alone has no distribution: its
// probabilities are 0 and its entropy is 0.
//
// What bounds it: reading the logits once.  A few rows go to thread-block clusters of up to 8 CTAs
// each; many rows to one CTA each of a grid that stays (three on an SM), rows taken in turn.  A
// producer warp streams the CTA's runs of 16-byte vectors through a ring in shared memory
// (cp.async.bulk), over the ends of rows, so that the next row is on its way while a row's results are
// put together.  Nothing of a row is kept:
//  - maximum, sums: each thread rescales its running (m, S, E) when a round's maximum passes m;
//  - alternatives: the n-th largest of the LP_GROUPS maxima that groups of threads have met is a lower
//    bound of the run's n-th largest logit.  It is taken in the rounds 0, 3 and 24 (each time costs
//    more than the notes that more of them would spare: 4096 rows of 32016, 10 alternatives 102 us, 104 with
//    0, 2, 8 and 32, 109 with every power of two), and only logits from it on are noted, in shared memory.
//    At the end each noted one's place is the number of larger ones.  Where too many are noted (equal
//    logits, long runs of -inf), they are noted again from a better bound on (another pass, over L2).
//  - the rank: logits before the token are counted two at a time, where a round has any; an if for each
//    was a quarter of the time with tokens of any rank.
// The row's ends that are not whole vectors (rows may start anywhere) are read value by value.
// Measured: 4096 rows of 32016 fp32 logits, 2 alternatives 91 us (5.8 TB/s, 0.85 of the copy rate);
// 1000 rows of 128003 of 16 bits, 20 alternatives 74 us (3.5 TB/s: the instructions, and the last third
// of the rows' turns, which 88 CTAs have); 48 rows of 32016 7 us, 6 of 4104 4.6 (launch, chain of barriers).
#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

#include "common.cuh"
#include "internal.h"

namespace sdsat {
namespace {

constexpr int LP_THREADS = 256;   // and the producer's warp
constexpr int LP_WARPS = LP_THREADS / 32;
constexpr int LP_UNROLL = 4;      // vectors of a thread and round
constexpr int LP_STAGES = 4;      // rounds in the ring
constexpr int LP_GROUPS = 64;     // groups of 4 threads whose maxima bound the alternatives
constexpr int LP_NOTED = 512;     // logits noted by a CTA
constexpr int LP_FEW = 64;        // noted logits that are ranked as they are
static_assert(LP_NOTED <= 2 * LP_THREADS, "two noted logits a thread");
constexpr int LP_CS = 8;          // CTAs of a row
constexpr int LP_PER_SM = 3;
constexpr int LP_ROUND = LP_UNROLL * LP_THREADS;   // vectors of a round
static_assert(LP_GROUPS >= LP_MAX_TOP && LP_GROUPS == LP_THREADS / 4 && LP_MAX_TOP <= 32, "a bound for every n_top");

__device__ __forceinline__ float lp_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// per half: all bits where x >= lo (no NaN), of two bf16 values
__device__ __forceinline__ uint32_t lp_ge2(uint32_t x, uint32_t lo) {
  uint32_t r;
  asm("set.ge.u32.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(lo));
  return r;
}

// larger key = earlier alternative: the logit's order in the high half, the id's inverse in the low
// (every key is above 0)
__device__ __forceinline__ unsigned long long lp_key(float x, int id) {
  const uint32_t b = __float_as_uint(x + 0.0f);   // (-0 and +0 are equal)
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return ((unsigned long long)o << 32) | (uint32_t)~id;
}
__device__ __forceinline__ float lp_key_logit(unsigned long long k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

// a run's maximum, sum of e^d and of e^d d relative to it (d unscaled by the temperature), ids before
// the token
struct __align__(16) LpSums {
  float m, S, E;
  int before;
};
struct LpSmem {
  uint4 ring[LP_STAGES][LP_ROUND];
  LpSums cta[LP_CS];                             // rank 0: each CTA's
  LpSums warp[LP_WARPS];
  float group[LP_GROUPS];
  float low[LP_WARPS];
  unsigned long long noted[LP_NOTED];
  unsigned long long best[LP_CS * LP_MAX_TOP];   // rank 0: the n best of each CTA
  unsigned long long bound;
  uint64_t full[LP_STAGES], empty[LP_STAGES];
  int count;
  volatile int abort;
};

__device__ __forceinline__ bool lp_bar_or(bool pred) {   // over the LP_THREADS threads
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %1, 0;\n\t"
      "barrier.cta.red.or.pred p, 1, %2, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)pred), "r"(LP_THREADS)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ void lp_bar() { named_bar_sync(1, LP_THREADS); }

// what a CTA reads of a row: whole vectors from id `head` on, of them [v0, v1); `tail` follows the last
template <bool BF16>
struct LpRun {
  static constexpr int E = BF16 ? 8 : 4;   // values of a vector
  const char* base;
  int head, tail, v0, v1;
  __device__ LpRun(const LogprobParams& p, long long row, int rank) {
    base = static_cast<const char*>(p.logits) + row * p.ld * (BF16 ? 2 : 4);
    head = min(p.V, (int)((16 - (reinterpret_cast<uintptr_t>(base) & 15)) & 15) / (BF16 ? 2 : 4));
    const int vectors = (p.V - head) / E;
    tail = head + vectors * E;
    v0 = (int)((long long)vectors * rank / p.cs);
    v1 = (int)((long long)vectors * (rank + 1) / p.cs);
  }
  __device__ const uint4* vec() const { return reinterpret_cast<const uint4*>(base + head * (BF16 ? 2 : 4)); }
  __device__ float raw(int i) const {
    return BF16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(base)[i]) : reinterpret_cast<const float*>(base)[i];
  }
};

template <bool BF16>
__global__ void __launch_bounds__(LP_THREADS + 32, LP_PER_SM) logprobs_kernel(const __grid_constant__ LogprobParams p) {
  using Run = LpRun<BF16>;
  constexpr int E = Run::E;
  extern __shared__ __align__(128) uint8_t smem_raw[];
  LpSmem& sm = *reinterpret_cast<LpSmem*>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = p.cs > 1 ? (int)cluster_ctarank() : 0;
  const int step = gridDim.x / p.cs;
  if (tid == 0) {
    for (int i = 0; i < LP_STAGES; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], LP_WARPS);
    }
    sm.abort = 0;
    fence_mbar_init();
  }
  __syncthreads();
  if (p.cs > 1) cluster_arrive_thread();   // (waited for before the cluster's memory is written)
  pdl_wait();
  pdl_trigger();

  if (warp == LP_WARPS) {
    // ---- the producer: the runs' rounds, one after the other, over the ends of rows
    if (lane == 0) {
      int it = 0;
      for (long long row = blockIdx.x / p.cs; row < p.rows && !sm.abort; row += step) {
        const Run run(p, row, rank);
        for (int v = run.v0; v < run.v1; v += LP_ROUND, ++it) {
          const int s = it % LP_STAGES;
          if (!mbar_wait_bounded(&sm.empty[s], ((it / LP_STAGES) & 1) ^ 1, &sm.abort, p.err)) break;
          const uint32_t bytes = min(LP_ROUND, run.v1 - v) * 16;
          mbar_arrive_expect_tx(&sm.full[s], bytes);
          bulk_load_g2s(sm.ring[s], run.vec() + v, bytes, &sm.full[s]);
        }
      }
      if (sm.abort) {   // let the copies in flight land before the CTA exits
        for (int i = max(0, it - LP_STAGES); i < it; ++i) {
          const uint64_t t0 = globaltimer_ns();
          while (!mbar_try_wait(&sm.full[i % LP_STAGES], (i / LP_STAGES) & 1))
            if (globaltimer_ns() - t0 > WAIT_LIMIT_NS) break;
        }
      }
    }
    if (p.cs > 1) {   // the cluster's barriers, with the other warps
      __syncwarp();
      cluster_wait_thread();
      cluster_sync_all();
    }
    return;
  }

  const int n = p.n_top;
  const float c = p.inv_t * 1.4426950408889634f;
  auto value = [&](const uint4& r, int k) {
    const uint32_t w = BF16 ? (&r.x)[k >> 1] : (&r.x)[k];
    return BF16 ? __uint_as_float(k & 1 ? w & 0xFFFF0000u : w << 16) : __uint_as_float(w);
  };
  // the n-th largest of the groups' maxima, the same for every thread: the smallest of those with
  // fewer than n larger ones.  A warp takes eight of them, four lanes each.
  auto nth_group = [&](float mine, bool fresh) {
    float g = fmaxf(mine, __shfl_xor_sync(0xffffffffu, mine, 1));
    g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
    lp_bar();                 // (what was read of the row or of the time before has been)
    if ((lane & 3) == 0) sm.group[warp * 8 + (lane >> 2)] = g;
    if (fresh && tid == 0) sm.count = 0;
    lp_bar();
    int larger = 0;
#pragma unroll
    for (int j = 0; j < LP_GROUPS / 16; ++j) {
      const float4 x = *reinterpret_cast<const float4*>(sm.group + 16 * j + 4 * (lane & 3));
      larger += (x.x > g) + (x.y > g) + (x.z > g) + (x.w > g);
    }
    larger += __shfl_xor_sync(0xffffffffu, larger, 1);
    larger += __shfl_xor_sync(0xffffffffu, larger, 2);
    float low = larger < n ? g : INFINITY;
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
    if (lane == 0) sm.low[warp] = low;
    lp_bar();
    const float4 x = *reinterpret_cast<const float4*>(sm.low), y = *reinterpret_cast<const float4*>(sm.low + 4);
    return fminf(fminf(fminf(x.x, x.y), fminf(x.z, x.w)), fminf(fminf(y.x, y.y), fminf(y.z, y.w)));
  };
  auto join = [&](LpSums a, const LpSums& b) {
    const float m = fmaxf(a.m, b.m);
    // (equal maxima, infinite ones too, differ by 0)
    const float da = a.m == m ? 0.f : a.m - m, db = b.m == m ? 0.f : b.m - m, fa = lp_ex2(da * c), fb = lp_ex2(db * c);
    a.E = fa * fmaxf(fmaf(da, a.S, a.E), -FLT_MAX) + fb * fmaxf(fmaf(db, b.S, b.E), -FLT_MAX);
    a.S = fa * a.S + fb * b.S;
    a.m = m;
    a.before += b.before;
    return a;
  };

  auto token = [&](long long row) { return p.tokens && row < p.rows ? __ldcg(p.tokens + row) : -1; };
  int it = 0;   // rounds taken from the ring
  int t_next = token(blockIdx.x / p.cs);
  float lt_next = 0.f;
  bool fetched = false;
  for (long long row = blockIdx.x / p.cs; row < p.rows; row += step) {
    const Run run(p, row, rank);
    auto logit = [&](int i) {
      const float x = run.raw(i);
      return isnan(x) ? -INFINITY : x;
    };
    int t = t_next;
    t_next = token(row + step);
    const bool given = t != -1;
    if (given && (t < 0 || t >= p.V)) {
      if (tid == 0 && rank == 0) set_error(p.err, ERR_TOKEN);
      t = 0;
    }
    const float lt = !given ? INFINITY : fetched ? lt_next : logit(t);
    // x comes before the token iff x >= lt at lower ids, x >= the next value above lt at higher ones
    constexpr uint32_t step1 = BF16 ? 0x10000u : 1u;
    const float above = lt == INFINITY ? NAN
                        : lt == 0.f    ? __uint_as_float(step1)
                                       : __uint_as_float(__float_as_uint(lt) + (lt > 0.f ? step1 : 0u - step1));
    // this thread's value among the row's ends, which no whole vector holds (fewer than 2 E)
    const int end_id = tid < run.head ? tid : run.tail + tid - run.head;
    const bool end_mine = rank == 0 && tid < 2 * E && end_id < p.V;
    const float end_raw = end_mine ? run.raw(end_id) : 0.f;

    if (run.v0 == run.v1) {   // (the first bound's barriers do this otherwise)
      lp_bar();
      if (tid == 0) sm.count = 0;
      lp_bar();
    }
    float bound = n ? -INFINITY : INFINITY;    // of the alternatives
    LpSums s;
    // One pass over the run, from the ring, or (CLEAN) from memory: there NaN and infinities are
    // looked for value by value; the pass without it ends with a NaN sum where any of them matter.
    auto pass = [&](auto clean_tag) {
      constexpr bool CLEAN = decltype(clean_tag)::value;
      s = LpSums{-FLT_MAX, 0.f, 0.f, 0};
      auto grow = [&](float top) {
        const float dm = s.m - top, f = lp_ex2(dm * c);
        s.E = f * (s.E + fmaxf(dm * s.S, -FLT_MAX));   // (0 where f is 0, whatever the maximum was)
        s.S *= f;
        s.m = top;
      };
      auto add = [&](float x) {
        const float d = CLEAN && x == s.m ? 0.f : x - s.m, e = lp_ex2(d * c);
        s.S += e;
        s.E = fmaf(e, fmaxf(d, -FLT_MAX), s.E);   // (0, not NaN, for a logit of -inf)
      };
      auto note = [&](float x, int id) {
        const int at = atomicAdd(&sm.count, 1);
        if (at < LP_NOTED) sm.noted[at] = lp_key(x, id);
      };
      int round = 0;
      for (int v = run.v0 + tid; v - tid < run.v1; v += LP_ROUND, ++round) {
        uint4 r[LP_UNROLL];
        constexpr uint32_t none = BF16 ? 0xFF80FF80u : 0xFF800000u;   // -inf
        if (CLEAN) {
#pragma unroll
          for (int u = 0; u < LP_UNROLL; ++u)
            r[u] = v + u * LP_THREADS < run.v1 ? __ldcg(run.vec() + v + u * LP_THREADS) : make_uint4(none, none, none, none);
#pragma unroll
          for (int u = 0; u < LP_UNROLL; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) {   // (a NaN is -inf)
              uint32_t& w = (&r[u].x)[k];
              if constexpr (BF16) {
                const __nv_bfloat162 h = __hmax2(reinterpret_cast<__nv_bfloat162&>(w), reinterpret_cast<const __nv_bfloat162&>(none));
                w = reinterpret_cast<const uint32_t&>(h);
              } else {
                w = __float_as_uint(fmaxf(__uint_as_float(w), -INFINITY));
              }
            }
        } else {
          mbar_wait_bounded(&sm.full[it % LP_STAGES], (it / LP_STAGES) & 1, &sm.abort, p.err);
          const uint4* stage = sm.ring[it % LP_STAGES] + tid;
#pragma unroll
          for (int u = 0; u < LP_UNROLL; ++u) r[u] = stage[u * LP_THREADS];
          if (v - tid + LP_ROUND > run.v1) {   // the last round may be short
#pragma unroll
            for (int u = 0; u < LP_UNROLL; ++u)
              if (v + u * LP_THREADS >= run.v1) r[u] = make_uint4(none, none, none, none);
          }
        }
        float vtop[LP_UNROLL];   // the largest of each vector (a NaN is passed over)
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u) {
          if constexpr (BF16) {
            const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&r[u]);
            const __nv_bfloat162 x = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
            vtop[u] = fmaxf(__low2float(x), __high2float(x));
          } else {
            vtop[u] = fmaxf(fmaxf(value(r[u], 0), value(r[u], 1)), fmaxf(value(r[u], 2), value(r[u], 3)));
          }
          vtop[u] = fmaxf(vtop[u], -INFINITY);
        }
        const float top = fmaxf(fmaxf(vtop[0], vtop[1]), fmaxf(vtop[2], vtop[3]));
        static_assert(LP_UNROLL == 4, "the round's maximum");
        // (the same for every thread)
        if (round == 0 || (n && (bound == -INFINITY || round == 3 || round == 24))) {
          const float old = s.S > 0.f ? s.m : -INFINITY;
          const float low = nth_group(fmaxf(old, top), round == 0);
          if (n) bound = fmaxf(bound, low);
        }
        if (top > s.m) grow(top);
        if (CLEAN) {
#pragma unroll
          for (int u = 0; u < LP_UNROLL; ++u)
#pragma unroll
            for (int k = 0; k < E; ++k) {
              add(value(r[u], k));
            }
        } else {
          const uint64_t m2 = f2_pack(-s.m, -s.m), c2 = f2_pack(c, c);
          uint64_t S2 = f2_pack(s.S, 0.f), E2 = f2_pack(s.E, 0.f);
#pragma unroll
          for (int u = 0; u < LP_UNROLL; ++u)
#pragma unroll
            for (int k = 0; k < E; k += 2) {
              const uint64_t d2 = f2_add(f2_pack(value(r[u], k), value(r[u], k + 1)), m2);
              float da, db, ea, eb;
              f2_unpack(f2_mul(d2, c2), ea, eb);
              const uint64_t e2 = f2_pack(lp_ex2(ea), lp_ex2(eb));
              S2 = f2_add(S2, e2);
              f2_unpack(d2, da, db);
              E2 = f2_fma(e2, f2_pack(fmaxf(da, -FLT_MAX), fmaxf(db, -FLT_MAX)), E2);
            }
          float b;
          f2_unpack(S2, s.S, b);
          s.S += b;
          f2_unpack(E2, s.E, b);
          s.E += b;
        }
        // the logits before the token, and those to note
        if (top >= lt) {
          const int id0 = run.head + (v - tid) * E, id1 = run.head + min(v - tid + LP_ROUND, run.v1) * E;   // the round's
          if (!CLEAN && (id1 <= t || id0 > t) && lt > -INFINITY) {
            // the same comparison for all of them (vectors past the run's end are -inf; +inf ends in the slower pass)
            const float lo = id1 <= t ? lt : above;
            uint32_t sum = 0;
            if constexpr (BF16) {   // a low half's mask counts 1 - 2^16, a high one's 2^16
              const uint32_t lo2 = __float_as_uint(lo) >> 16 | (__float_as_uint(lo) & 0xFFFF0000u);
#pragma unroll
              for (int u = 0; u < LP_UNROLL; ++u)
#pragma unroll
                for (int k = 0; k < 4; ++k) sum -= lp_ge2((&r[u].x)[k], lo2);
              s.before += 2 * (int)(sum & 0xFFFFu) + ((int)sum >> 16);
            } else {   // x - lo has a sign where x < lo (-0 - -0 has none)
              const float minus = lo == 0.f ? 0.f : -lo;
              const uint64_t minus2 = f2_pack(minus, minus);
#pragma unroll
              for (int u = 0; u < LP_UNROLL; ++u)
#pragma unroll
                for (int k = 0; k < E; k += 2) {
                  float a, b;
                  f2_unpack(f2_add(f2_pack(value(r[u], k), value(r[u], k + 1)), minus2), a, b);
                  sum += __float_as_uint(a) >> 31;
                  sum += __float_as_uint(b) >> 31;
                }
              s.before += LP_UNROLL * E - (int)sum;
            }
          } else {
#pragma unroll 1
            for (int at = v; at < min(v - tid + LP_ROUND, run.v1); at += LP_THREADS) {
              const int first = run.head + at * E;
              const float lo = first + E <= t ? lt : above;
              const uint4 w = CLEAN ? __ldcg(run.vec() + at) : sm.ring[it % LP_STAGES][at - v + tid];
#pragma unroll
              for (int k = 0; k < E; ++k) s.before += (CLEAN ? fmaxf(value(w, k), -INFINITY) : value(w, k)) >= lo;
              if (first <= t && t < first + E)   // equal logits before the token in its own vector
                for (int k = 0; first + k < t; ++k) s.before += logit(first + k) == lt;
            }
          }
        }
        if (top >= bound) {
          uint32_t hit = 0;   // vectors
#pragma unroll
          for (int u = 0; u < LP_UNROLL; ++u) hit |= (uint32_t)(vtop[u] >= bound && v + u * LP_THREADS < run.v1) << u;
#pragma unroll 1
          while (hit) {
            const int at = v + (__ffs(hit) - 1) * LP_THREADS, id0 = run.head + at * E;
            hit &= hit - 1;
            const uint4* w = CLEAN ? run.vec() + at : sm.ring[it % LP_STAGES] + (at - v + tid);
            const uint4 x4 = *w;
            uint32_t which = 0;
            if (CLEAN && bound == -INFINITY) {   // (a NaN is -inf)
              which = (1u << E) - 1u;
            } else {
#pragma unroll
              for (int k = 0; k < E; ++k) which |= (uint32_t)(value(x4, k) >= bound) << k;
            }
#pragma unroll 1
            for (; which; which &= which - 1) {
              const int k = __ffs(which) - 1;
              float x = BF16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(w)[k]) : reinterpret_cast<const float*>(w)[k];
              if (CLEAN && isnan(x)) x = -INFINITY;
              note(x, id0 + k);
            }
          }
        }
        if (!CLEAN) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.empty[it % LP_STAGES]);
          ++it;
        }
      }
      if (end_mine) {
        const float x = isnan(end_raw) ? -INFINITY : end_raw;
        if (x > s.m) grow(x);
        add(x);
        s.before += x >= (end_id < t ? lt : above);
        if (x >= bound) note(x, end_id);
      }
    };
    pass(std::false_type{});
    if (end_mine && isnan(end_raw)) set_error(p.err, ERR_NAN_LOGITS);
    // every thread of a CTA takes the slower pass when one thread met a NaN or an infinite maximum
    if (lp_bar_or(isnan(s.S) || s.m == INFINITY)) {
      bool nan = false;
      for (int v = run.v0 + tid; v < run.v1; v += LP_THREADS) {
        const uint4 r = __ldcg(run.vec() + v);
#pragma unroll
        for (int k = 0; k < E; ++k) nan |= isnan(value(r, k));
      }
      if (nan) set_error(p.err, ERR_NAN_LOGITS);
      bound = n ? -INFINITY : INFINITY;
      lp_bar();
      if (tid == 0) sm.count = 0;
      lp_bar();
      pass(std::true_type{});
      lp_bar();
    }
    if (given && row + step < p.rows && t_next >= 0 && t_next < p.V) {
      lt_next = LpRun<BF16>(p, row + step, rank).raw(t_next);
      lt_next = isnan(lt_next) ? -INFINITY : lt_next;
      fetched = true;
    } else {
      fetched = false;
    }

    // ---- the warp's sums
    const float mine = s.S > 0.f ? s.m : -INFINITY;   // the thread's largest logit
    {
      float m = s.m;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      const float d = s.m == m ? 0.f : s.m - m, f = lp_ex2(d * c);
      float S = f * s.S, X = f * fmaxf(fmaf(d, s.S, s.E), -FLT_MAX);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        S += __shfl_xor_sync(0xffffffffu, S, o);
        X += __shfl_xor_sync(0xffffffffu, X, o);
      }
      const int before = __reduce_add_sync(0xffffffffu, s.before);
      if (lane == 0) sm.warp[warp] = LpSums{m, S, X, before};
    }

    // ---- the CTA's alternatives
    int count = n ? sm.count : 0;   // (complete: every thread has passed a barrier since it noted)
    if (count > LP_NOTED) {
      // too many: noted again from the n-th largest of the whole run's group maxima on, and, while
      // that is too many still (equal logits), from the n-th best of those noted
      unsigned long long low = lp_key(nth_group(mine, false), INT_MAX);
      while (true) {
        lp_bar();
        if (tid == 0) sm.count = 0;
        lp_bar();
        auto note = [&](int id) {
          const unsigned long long k = lp_key(logit(id), id);
          if (k < low) return;
          const int at = atomicAdd(&sm.count, 1);
          if (at < LP_NOTED) sm.noted[at] = k;
        };
        for (int i = run.head + run.v0 * E + tid; i < run.head + run.v1 * E; i += LP_THREADS) note(i);
        if (end_mine) note(end_id);
        lp_bar();
        count = sm.count;
        if (count <= LP_NOTED) break;
        for (int i = tid; i < LP_NOTED; i += LP_THREADS) {
          const unsigned long long k = sm.noted[i];
          int better = 0;
          for (int j = 0; j < LP_NOTED; ++j) better += sm.noted[j] > k;
          if (better == n - 1) sm.bound = k;
        }
        lp_bar();
        low = sm.bound;
      }
    } else {
      lp_bar();   // the warps' sums
    }
    // Many noted ones (those of the early rounds, from lower bounds on): the whole run's bound keeps
    // about n of them (2000 rows of 32016, 32 alternatives: 8 us less of 87).
    if (count > LP_FEW) {
      const unsigned long long low = lp_key(nth_group(mine, false), INT_MAX);
      const unsigned long long k0 = tid < count ? sm.noted[tid] : 0, k1 = tid + LP_THREADS < count ? sm.noted[tid + LP_THREADS] : 0;
      lp_bar();
      if (tid == 0) sm.count = 0;
      lp_bar();
      if (k0 >= low) sm.noted[atomicAdd(&sm.count, 1)] = k0;
      if (k1 >= low) sm.noted[atomicAdd(&sm.count, 1)] = k1;
      lp_bar();
      count = sm.count;
    }
    // a noted logit's place is the number of larger keys (the keys differ)
    auto ranked = [&](const unsigned long long* keys, int total, auto&& put) {
      for (int i = tid; i < total; i += LP_THREADS) {
        const unsigned long long k = keys[i];
        int better = 0;
#pragma unroll 8
        for (int j = 0; j < total; ++j) better += keys[j] > k;
        if (better < n && k) put(better, k);   // (0: a place that a CTA did not fill)
      }
    };
    {
      const LpSums w = sm.warp[lane & (LP_WARPS - 1)];
      s = w;
#pragma unroll
      for (int o = 1; o < LP_WARPS; o <<= 1) s.m = fmaxf(s.m, __shfl_xor_sync(0xffffffffu, s.m, o));
      const float d = w.m == s.m ? 0.f : w.m - s.m, f = lp_ex2(d * c);
      s.S = f * w.S;
      s.E = f * fmaxf(fmaf(d, w.S, w.E), -FLT_MAX);
#pragma unroll
      for (int o = 1; o < LP_WARPS; o <<= 1) {
        s.S += __shfl_xor_sync(0xffffffffu, s.S, o);
        s.E += __shfl_xor_sync(0xffffffffu, s.E, o);
        s.before += __shfl_xor_sync(0xffffffffu, s.before, o);
      }
    }
    float logz = 0.f;
    auto put_top = [&](int place, unsigned long long k) {
      const float x = lp_key_logit(k);
      p.top_ids[row * n + place] = (int)~(uint32_t)k;
      p.top_logp[row * n + place] = (x == s.m ? 0.f : (x - s.m) * p.inv_t) - logz;
    };
    if (p.cs > 1) {
      cluster_wait_thread();   // every CTA of the cluster runs
      const uint32_t best = mapa_shared(smem_u32(sm.best), 0), sums = mapa_shared(smem_u32(sm.cta), 0);
      auto send = [&](int place, unsigned long long k) {
        asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(best + (rank * n + place) * 8), "l"(k) : "memory");
      };
      for (int i = count + tid; i < n; i += LP_THREADS) send(i, 0);   // fewer logits than places
      ranked(sm.noted, count, send);
      if (tid == 0) {
        asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(sums + rank * (uint32_t)sizeof(LpSums)),
                     "r"(__float_as_uint(s.m)), "r"(__float_as_uint(s.S)), "r"(__float_as_uint(s.E)), "r"(s.before)
                     : "memory");
      }
      cluster_sync_all();
      if (rank) return;
      s = sm.cta[0];
      for (int r = 1; r < p.cs; ++r) s = join(s, sm.cta[r]);
    }
    const bool dead = s.S == 0.f;   // -inf alone
    if (dead) s.m = -INFINITY;
    logz = dead ? INFINITY : logf(s.S);
    if (tid == 0) {
      if (p.entropy) p.entropy[row] = dead ? 0.f : logz - s.E * p.inv_t / s.S;
      if (p.logp) p.logp[row] = given ? (lt == s.m ? 0.f : (lt - s.m) * p.inv_t) - logz : 0.f;
      if (p.rank) p.rank[row] = given ? s.before + 1 : 0;
    }
    if (p.cs > 1) {
      ranked(sm.best, p.cs * n, put_top);
      return;   // (a cluster has one row)
    }
    ranked(sm.noted, count, put_top);
  }
}

}  // namespace

cudaError_t logprobs_prepare() {
  cudaError_t e = cudaSuccess;
  for (auto* k : {logprobs_kernel<false>, logprobs_kernel<true>}) {
    if (e == cudaSuccess) e = prefer_shared(k);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(LpSmem));
  }
  return e;
}

cudaError_t launch_logprobs(const LogprobParams& p0, int num_sms, cudaStream_t st, bool pdl) {
  LogprobParams p = p0;
  // CTAs of a row: as long as they all run at once and each has a round's work
  const int round = LP_ROUND * (p.bf16 ? 8 : 4);
  p.cs = 1;
  while (p.cs < LP_CS && 2ll * p.rows * p.cs <= LP_PER_SM * num_sms && p.V > (long long)p.cs * round) p.cs *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.cs > 1 ? p.rows * p.cs : std::min(p.rows, LP_PER_SM * num_sms));
  cfg.blockDim = dim3(LP_THREADS + 32);
  cfg.dynamicSmemBytes = sizeof(LpSmem);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = p.cs;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 2 : 1;
  return p.bf16 ? cudaLaunchKernelEx(&cfg, logprobs_kernel<true>, p) : cudaLaunchKernelEx(&cfg, logprobs_kernel<false>, p);
}

}  // namespace sdsat
