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
#include "common.cuh"
#include "internal.h"

namespace sdsat {
namespace {

constexpr int LP_THREADS = 512;

__device__ __forceinline__ float lp_load(const LogprobParams& p, long long row, int i) {
  return p.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.logits)[row * p.ld + i])
                : static_cast<const float*>(p.logits)[row * p.ld + i];
}

// larger key = earlier alternative: the logit's order in the high half, the id's inverse in the low
__device__ __forceinline__ unsigned long long lp_key(float x, int id) {
  const uint32_t b = __float_as_uint(x + 0.0f);   // (-0 and +0 are equal)
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return ((unsigned long long)o << 32) | (uint32_t)~id;
}

template <typename T, typename F>
__device__ T lp_reduce(T v, T* slots, F&& f) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
  __syncthreads();
  v = slots[0];
  for (int w = 1; w < LP_THREADS / 32; ++w) v = f(v, slots[w]);
  return v;
}

__global__ void __launch_bounds__(LP_THREADS) logprobs_kernel(const __grid_constant__ LogprobParams p) {
  __shared__ float fslots[LP_THREADS / 32];
  __shared__ int islots[LP_THREADS / 32];
  __shared__ unsigned long long kslots[LP_THREADS / 32];
  pdl_wait();
  pdl_trigger();
  const auto fadd = [](float a, float b) { return a + b; };
  const auto fmx = [](float a, float b) { return fmaxf(a, b); };
  const auto iadd = [](int a, int b) { return a + b; };
  const auto kmx = [](unsigned long long a, unsigned long long b) { return a > b ? a : b; };
  for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
    auto logit = [&](int i) {
      const float x = lp_load(p, row, i);
      return isnan(x) ? -INFINITY : x;
    };
    float m = -INFINITY;
    bool nan = false;
    for (int i = threadIdx.x; i < p.V; i += LP_THREADS) {
      nan |= isnan(lp_load(p, row, i));
      m = fmaxf(m, logit(i));
    }
    if (nan) set_error(p.err, ERR_NAN_LOGITS);
    m = lp_reduce(m, fslots, fmx);
    int t = p.tokens ? __ldcg(p.tokens + row) : -1;
    const bool given = t != -1;
    if (given && (t < 0 || t >= p.V)) {
      if (threadIdx.x == 0) set_error(p.err, ERR_TOKEN);
      t = 0;
    }
    const float lt = given ? logit(t) : 0.f;
    auto diff = [&](float x) { return x == m ? 0.f : (x - m) * p.inv_t; };
    float S = 0.f, E = 0.f;
    int before = 0;
    if (m > -INFINITY) {
      for (int i = threadIdx.x; i < p.V; i += LP_THREADS) {
        const float d = diff(logit(i)), e = expf(d);
        S += e;
        E += e > 0.f ? e * d : 0.f;
      }
    }
    for (int i = threadIdx.x; given && i < p.V; i += LP_THREADS) {
      const float x = logit(i);
      before += x > lt || (x == lt && i < t);
    }
    S = lp_reduce(S, fslots, fadd);
    E = lp_reduce(E, fslots, fadd);
    before = lp_reduce(before, islots, iadd);
    const float logz = m > -INFINITY ? logf(S) : INFINITY;
    if (threadIdx.x == 0) {
      if (p.entropy) p.entropy[row] = m > -INFINITY ? logz - E / S : 0.f;
      if (p.logp) p.logp[row] = given ? diff(lt) - logz : 0.f;
      if (p.rank) p.rank[row] = given ? before + 1 : 0;
    }
    unsigned long long last = ~0ull;
    for (int n = 0; n < p.n_top; ++n) {
      unsigned long long best = 0;
      for (int i = threadIdx.x; i < p.V; i += LP_THREADS) {
        const unsigned long long k = lp_key(logit(i), i);
        if (k < last) best = kmx(best, k);
      }
      last = lp_reduce(best, kslots, kmx);
      if (threadIdx.x == 0) {
        const int id = (int)~(uint32_t)last;
        p.top_ids[row * p.n_top + n] = id;
        p.top_logp[row * p.n_top + n] = diff(logit(id)) - logz;
      }
    }
    __syncthreads();
  }
}

}  // namespace

cudaError_t logprobs_prepare() { return prefer_shared(logprobs_kernel); }

cudaError_t launch_logprobs(const LogprobParams& p, int num_sms, cudaStream_t st, bool pdl) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.rows < 4 * num_sms ? p.rows : 4 * num_sms);
  cfg.blockDim = dim3(LP_THREADS);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, logprobs_kernel, p);
}

}  // namespace sdsat
