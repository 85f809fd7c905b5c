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
// What bounds it: reading the logits once (fewer than 8 instructions and one exp a value).  A row is
// read by a thread-block cluster of 1 to 8 CTAs, each a run of its 16-byte vectors, in rounds of
// LP_UNROLL vectors a thread; nothing of it is kept:
//  - maximum, sums: each thread rescales its running (m, S, E) when a round's maximum passes m;
//  - alternatives: the n-th largest of the first round's LP_GROUPS group maxima is a lower bound of
//    the run's n-th largest logit, so only logits from it on are noted (about n for every round:
//    2 n rounds / LP_GROUPS ... of random logits), in shared memory, and ranked at the end by counting
//    the larger ones.  Where too many are noted (ties, ascending rows, long runs of -inf), the n-th
//    best of the noted ones is the bound of another pass over the run, which rereads it through L2.
// The row's ends that are not whole vectors (rows may start anywhere) are read value by value.
#include <cfloat>
#include <climits>
#include <type_traits>

#include "common.cuh"
#include "internal.h"

namespace sdsat {
namespace {

constexpr int LP_THREADS = 256;
constexpr int LP_WARPS = LP_THREADS / 32;
constexpr int LP_UNROLL = 4;      // vectors of a thread and round
constexpr int LP_GROUPS = 64;     // groups of 4 threads whose maxima bound the alternatives
constexpr int LP_NOTED = 1024;    // logits noted by a CTA
constexpr int LP_CS = 8;          // CTAs of a row
constexpr int LP_ROUNDS = 8;      // rounds of a CTA, from which on a row is split over more of them
static_assert(LP_GROUPS >= LP_MAX_TOP && LP_GROUPS == LP_THREADS / 4 && LP_MAX_TOP <= 32, "a bound for every n_top");

__device__ __forceinline__ float lp_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
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
  unsigned long long noted[LP_NOTED];
  unsigned long long best[LP_CS * LP_MAX_TOP];   // rank 0: the best of each CTA
  LpSums cta[LP_CS];                             // rank 0
  LpSums warp[LP_WARPS];
  __align__(16) float group[LP_GROUPS];
  unsigned long long bound;
  int count;
};

template <bool BF16>
__global__ void __launch_bounds__(LP_THREADS) logprobs_kernel(const __grid_constant__ LogprobParams p) {
  constexpr int E = BF16 ? 8 : 4;   // values of a vector
  __shared__ LpSmem sm;
  if (p.cs > 1) cluster_arrive_thread();   // (waited for before the cluster's memory is written)
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = (int)cluster_ctarank();
  const long long row = blockIdx.x / p.cs;
  const int n = p.n_top;
  const char* base = static_cast<const char*>(p.logits) + row * p.ld * (BF16 ? 2 : 4);
  auto logit = [&](int i) {
    const float x = BF16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(base)[i]) : reinterpret_cast<const float*>(base)[i];
    return isnan(x) ? -INFINITY : x;
  };
  // the row's whole vectors start at id `head`; this CTA's are [v0, v1)
  const int head = min(p.V, (int)((16 - (reinterpret_cast<uintptr_t>(base) & 15)) & 15) / (BF16 ? 2 : 4));
  const int vectors = (p.V - head) / E, tail = head + vectors * E;
  const int v0 = (int)((long long)vectors * rank / p.cs), v1 = (int)((long long)vectors * (rank + 1) / p.cs);
  const uint4* vec = reinterpret_cast<const uint4*>(base + head * (BF16 ? 2 : 4));

  int t = p.tokens ? __ldcg(p.tokens + row) : -1;
  const bool given = t != -1;
  if (given && (t < 0 || t >= p.V)) {
    if (tid == 0 && rank == 0) set_error(p.err, ERR_TOKEN);
    t = 0;
  }
  const float lt = given ? logit(t) : INFINITY;
  // x comes before the token iff x >= lt at lower ids, x >= the next value above lt at higher ones
  const float above = lt == INFINITY ? NAN
                      : lt == 0.f    ? __uint_as_float(1u)
                                     : __uint_as_float(__float_as_uint(lt) + (lt > 0.f ? 1u : 0xFFFFFFFFu));
  const float c = p.inv_t * 1.4426950408889634f;

  auto value = [&](const uint4& r, int k) {
    const uint32_t w = BF16 ? (&r.x)[k >> 1] : (&r.x)[k];
    return BF16 ? __uint_as_float(k & 1 ? w & 0xFFFF0000u : w << 16) : __uint_as_float(w);
  };
  // the n-th largest of the groups' maxima, the same for every thread
  auto nth_group = [&](float mine) {
    float g = fmaxf(mine, __shfl_xor_sync(0xffffffffu, mine, 1));
    g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
    __syncthreads();          // (the maxima of the time before have been read)
    if ((lane & 3) == 0) sm.group[warp * 8 + (lane >> 2)] = g;
    __syncthreads();
    const float a = sm.group[lane], b = sm.group[lane + 32];
    int na = 0, nb = 0;       // larger ones
#pragma unroll 4
    for (int j = 0; j < LP_GROUPS; j += 4) {
      const float4 x = *reinterpret_cast<const float4*>(sm.group + j);
      na += (x.x > a) + (x.y > a) + (x.z > a) + (x.w > a);
      nb += (x.x > b) + (x.y > b) + (x.z > b) + (x.w > b);
    }
    float low = fminf(na < n ? a : INFINITY, nb < n ? b : INFINITY);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
    return low;
  };
  if (tid == 0) sm.count = 0;
  float bound = n ? -INFINITY : INFINITY;    // of the alternatives
  LpSums s;
  // One pass over the run.  CLEAN: NaN and infinities are looked for value by value; the pass
  // without it gives a NaN sum where there are any that matter.
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
    for (int v = v0 + tid; v - tid < v1; v += LP_UNROLL * LP_THREADS) {
      uint4 r[LP_UNROLL];
      constexpr uint32_t none = BF16 ? 0xFF80FF80u : 0xFF800000u;   // -inf
#pragma unroll
      for (int u = 0; u < LP_UNROLL; ++u) {
        r[u] = make_uint4(none, none, none, none);
        if (v + u * LP_THREADS < v1) r[u] = __ldcs(vec + v + u * LP_THREADS);
      }
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < LP_UNROLL; ++u)
#pragma unroll
        for (int k = 0; k < E; ++k) top = fmaxf(top, value(r[u], k));   // (a NaN is passed over)
      if (bound == -INFINITY) bound = nth_group(top);   // (the same for every thread)
      if (top > s.m) grow(top);
#pragma unroll
      for (int u = 0; u < LP_UNROLL; ++u) {
        const int id0 = head + (v + u * LP_THREADS) * E;
        const float lo = v + u * LP_THREADS >= v1 ? NAN : id0 + E <= t ? lt : above;
#pragma unroll
        for (int k = 0; k < E; ++k) {
          float x = value(r[u], k);
          if (CLEAN && isnan(x)) x = -INFINITY;
          add(x);
          s.before += x >= lo;
        }
        if (id0 <= t && t < id0 + E && v + u * LP_THREADS < v1)   // equal logits before the token in its own vector
          for (int k = 0; id0 + k < t; ++k) s.before += logit(id0 + k) == lt;
      }
      if (top >= bound || CLEAN) {
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u)
#pragma unroll
          for (int k = 0; k < E; ++k) {
            float x = value(r[u], k);
            if (CLEAN && isnan(x)) x = -INFINITY;
            if (x >= bound && v + u * LP_THREADS < v1) note(x, head + (v + u * LP_THREADS) * E + k);
          }
      }
    }
    // the ids that no whole vector holds: fewer than 2 E
    const int id = tid < head ? tid : tail + tid - head;
    if (rank == 0 && id < p.V && (tid < head || id >= tail)) {
      const float x = logit(id);
      if (x > s.m) grow(x);
      add(x);
      s.before += x >= (id < t ? lt : above);
      if (x >= bound) note(x, id);
    }
  };
  pass(std::false_type{});
  // every thread of a CTA takes the slower pass when one thread met a NaN or an infinite maximum
  if (__syncthreads_or(isnan(s.S) || s.m == INFINITY)) {
    bool nan = false;
    for (int v = v0 + tid; v < v1; v += LP_THREADS) {
      const uint4 r = __ldcs(vec + v);
#pragma unroll
      for (int k = 0; k < E; ++k) nan |= isnan(value(r, k));
    }
    if (nan) set_error(p.err, ERR_NAN_LOGITS);
    if (tid == 0) sm.count = 0;
    bound = n ? -INFINITY : INFINITY;
    __syncthreads();
    pass(std::true_type{});
  }
  if (rank == 0 && tid < 2 * E) {   // NaN in the ends
    const int id = tid < head ? tid : tail + tid - head;
    if (id < p.V && (tid < head || id >= tail) &&
        isnan(BF16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(base)[id]) : reinterpret_cast<const float*>(base)[id]))
      set_error(p.err, ERR_NAN_LOGITS);
  }

  const float mine = s.S > 0.f ? s.m : -INFINITY;   // the thread's largest logit
  // ---- the CTA's sums: warps by shuffles, then rank 0 of the cluster
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
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    LpSums b;
    b.m = __shfl_xor_sync(0xffffffffu, s.m, o);
    b.S = __shfl_xor_sync(0xffffffffu, s.S, o);
    b.E = __shfl_xor_sync(0xffffffffu, s.E, o);
    b.before = __shfl_xor_sync(0xffffffffu, s.before, o);
    s = join(s, b);
  }
  if (lane == 0) sm.warp[warp] = s;
  __syncthreads();
  s = sm.warp[0];
#pragma unroll
  for (int w = 1; w < LP_WARPS; ++w) s = join(s, sm.warp[w]);

  // ---- the CTA's alternatives
  int count = n ? sm.count : 0;
  if (count > LP_NOTED) {
    // too many: noted again from the n-th largest of the whole run's group maxima on, and, while
    // that is too many still (equal logits), from the n-th best of those noted
    unsigned long long low = lp_key(nth_group(mine), INT_MAX);
    while (true) {
      if (tid == 0) sm.count = 0;
      __syncthreads();
      auto note = [&](int id) {
        const unsigned long long k = lp_key(logit(id), id);
        if (k < low) return;
        const int at = atomicAdd(&sm.count, 1);
        if (at < LP_NOTED) sm.noted[at] = k;
      };
      for (int i = head + v0 * E + tid; i < head + v1 * E; i += LP_THREADS) note(i);
      const int id = tid < head ? tid : tail + tid - head;
      if (rank == 0 && id < p.V && (tid < head || id >= tail)) note(id);
      __syncthreads();
      count = sm.count;
      if (count <= LP_NOTED) break;
      for (int i = tid; i < LP_NOTED; i += LP_THREADS) {
        const unsigned long long k = sm.noted[i];
        int better = 0;
        for (int j = 0; j < LP_NOTED; ++j) better += sm.noted[j] > k;
        if (better == n - 1) sm.bound = k;
      }
      __syncthreads();
      low = sm.bound;
    }
  }
  // (the keys differ: each noted logit has a place of its own)
  auto ranked = [&](const unsigned long long* keys, int total, auto&& put) {
    for (int i = tid; i < total; i += LP_THREADS) {
      const unsigned long long k = keys[i];
      int better = 0;
      for (int j = 0; j < total; ++j) better += keys[j] > k;
      if (better < n && k) put(better, k);
    }
  };
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
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(best + (rank * LP_MAX_TOP + place) * 8), "l"(k) : "memory");
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
    // (a place that a CTA did not fill, and the places past n, hold 0)
    for (int i = tid; i < p.cs * LP_MAX_TOP; i += LP_THREADS) {
      if (i % LP_MAX_TOP >= n) sm.best[i] = 0;
    }
    __syncthreads();
  }
  const bool dead = s.S == 0.f;   // -inf alone
  if (dead) s.m = -INFINITY;
  logz = dead ? INFINITY : logf(s.S);
  if (tid == 0) {
    if (p.entropy) p.entropy[row] = dead ? 0.f : logz - s.E * p.inv_t / s.S;
    if (p.logp) p.logp[row] = given ? (lt == s.m ? 0.f : (lt - s.m) * p.inv_t) - logz : 0.f;
    if (p.rank) p.rank[row] = given ? s.before + 1 : 0;
  }
  if (p.cs > 1) ranked(sm.best, p.cs * LP_MAX_TOP, put_top);
  else ranked(sm.noted, count, put_top);
}

}  // namespace

cudaError_t logprobs_prepare() {
  cudaError_t e = prefer_shared(logprobs_kernel<false>);
  if (e == cudaSuccess) e = prefer_shared(logprobs_kernel<true>);
  return e;
}

cudaError_t launch_logprobs(const LogprobParams& p0, int num_sms, cudaStream_t st, bool pdl) {
  LogprobParams p = p0;
  const int round = LP_UNROLL * LP_THREADS * (p.bf16 ? 8 : 4);   // logits of a CTA's round
  p.cs = 1;
  while (p.cs < LP_CS && p.V > (long long)p.cs * round * LP_ROUNDS) p.cs *= 2;
  while (p.cs < LP_CS && 2ll * p.rows * p.cs <= 4 * num_sms && p.V > (long long)p.cs * round) p.cs *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.rows * p.cs);
  cfg.blockDim = dim3(LP_THREADS);
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
