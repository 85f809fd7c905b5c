// Block-causal attention of sequences that share their leading pages.
//
// Row j of sequence s attends to the committed slots [0, len[s]) and to block rows 0..j (or its
// ancestors in a tree block), slots len[s] .. len[s] + j, all on pages of KV_PAGE slots named by the
// page table.  G = H / Hk query heads read the same cache head.
//
// A CTA per (row, head): a warp takes every fourth key with the head's dimensions over its lanes, a
// running maximum and sum, and the four warps' results are merged at the end.
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace sdsat {
namespace {

template <int HD>
__global__ void __launch_bounds__(128) prefix_attention_kernel(const __grid_constant__ PrefixAttnParams p,
                                                               const __nv_bfloat16* kc, const __nv_bfloat16* vc) {
  constexpr int E = HD / 32;
  __shared__ float o_s[4][HD], m_s[4], l_s[4];
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = blockIdx.x / p.H, h = blockIdx.x % p.H, s = r / p.nq, j = r % p.nq, hk = h / (p.H / p.Hk);
  const int len = __ldcg(p.len + s), end = min(len + p.nq, p.ld * KV_PAGE);
  const uint32_t own = p.anc ? __ldcg(p.anc + r) : (2u << j) - 1u;
  float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const long long at = r * p.q_ld + (long long)h * HD + lane + 32 * e;
    q[e] = (p.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.q)[at]) : static_cast<const float*>(p.q)[at]) *
           rsqrtf((float)HD);
    o[e] = 0.f;
  }
  for (int t = warp; t < end; t += 4) {
    if (t >= len && !((own >> (t - len)) & 1u)) continue;
    const int page = __ldcg(p.table + (size_t)s * p.ld + t / KV_PAGE);
    if (page < 0 || page >= p.n_pages) {
      if (lane == 0) set_error(p.err, ERR_PAGE);
      continue;
    }
    const long long row = (p.row0 + ((long long)page * p.Hk + hk) * KV_PAGE + t % KV_PAGE) * HD;
    float x = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) x += q[e] * __bfloat162float(kc[row + lane + 32 * e]);
#pragma unroll
    for (int a = 16; a > 0; a >>= 1) x += __shfl_xor_sync(0xffffffffu, x, a);
    const float mn = fmaxf(m, x), f = m == -INFINITY ? 0.f : expf(m - mn), w = expf(x - mn);
    l = l * f + w;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + w * __bfloat162float(vc[row + lane + 32 * e]);
    m = mn;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) o_s[warp][lane + 32 * e] = o[e];
  if (lane == 0) m_s[warp] = m, l_s[warp] = l;
  __syncthreads();
  if (threadIdx.x >= HD) return;
  float M = fmaxf(fmaxf(m_s[0], m_s[1]), fmaxf(m_s[2], m_s[3])), L = 0.f, a = 0.f;
  for (int w = 0; w < 4; ++w) {
    const float f = m_s[w] == -INFINITY ? 0.f : expf(m_s[w] - M);
    L += f * l_s[w];
    a += f * o_s[w][threadIdx.x];
  }
  a = L == 0.f ? 0.f : a / L;   // (a row that sees no slot: 0)
  const long long at = r * p.out_ld + (long long)h * HD + threadIdx.x;
  if (p.bf16) static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(a);
  else static_cast<float*>(p.out)[at] = a;
  if (p.out_hi) {
    const size_t x = (size_t)r * p.H * HD + h * HD + threadIdx.x;
    const __nv_bfloat16 hi = __float2bfloat16_rn(a);
    p.out_hi[x] = hi;
    p.out_lo[x] = __float2bfloat16_rn(a - __bfloat162float(hi));
  }
}

}  // namespace

size_t prefix_attention_scratch(int, int, int) { return 1; }

cudaError_t prefix_attention_prepare() {
  cudaError_t e = prefer_shared(prefix_attention_kernel<64>);
  if (e == cudaSuccess) e = prefer_shared(prefix_attention_kernel<128>);
  return e;
}

cudaError_t launch_prefix_attention(const PrefixAttnParams& p, int, cudaStream_t st, bool pdl) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.b * p.nq * p.H);
  cfg.blockDim = dim3(128);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  const __nv_bfloat16 *k = static_cast<const __nv_bfloat16*>(p.k), *v = static_cast<const __nv_bfloat16*>(p.v);
  return p.hd == 64 ? cudaLaunchKernelEx(&cfg, prefix_attention_kernel<64>, p, k, v)
                    : cudaLaunchKernelEx(&cfg, prefix_attention_kernel<128>, p, k, v);
}

}  // namespace sdsat
