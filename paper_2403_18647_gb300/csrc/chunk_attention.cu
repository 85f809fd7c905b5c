// Causal attention of the new rows of a ragged batch over pages.
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace sdsat {

size_t chunk_attention_scratch(int) { return 4; }
cudaError_t chunk_attention_prepare() { return cudaSuccess; }

// A warp for each (row, head), a key at a time: running maximum and sum.
template <bool BF16, int HD>
__global__ void __launch_bounds__(128) chunk_attention_kernel(const __grid_constant__ ChunkAttnParams p) {
  constexpr int E = HD / 32;
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int r = (int)(w / p.H), h = (int)(w % p.H);
  pdl_trigger();
  pdl_wait();
  if (r >= p.rows) return;
  int s = -1, first = 0, last = 0, before = 0;
  bool bad = false;
  for (int i = 0; i <= p.b; ++i) {
    const int at = __ldcg(p.start + i);
    bad |= at < before || at > p.rows;
    if (i < p.b && at <= r && r < __ldcg(p.start + i + 1)) s = i, first = at;
    before = at;
  }
  if (bad && lane == 0) set_error(p.err, ERR_CAPACITY);
  if (bad || s < 0) return;
  last = max(__ldcg(p.len + s), 0);
  const long long see = (long long)last + (r - first) + 1;
  const int n = (int)min(see, (long long)p.ld * KV_PAGE);
  if (see > n && lane == 0) set_error(p.err, ERR_PAGE);
  float q[E], o[E], m = -INFINITY, l = 0.f;
  for (int e = 0; e < E; ++e) {
    const long long at = r * p.q_ld + h * HD + lane * E + e;
    q[e] = BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.q)[at]) : static_cast<const float*>(p.q)[at];
    o[e] = 0.f;
  }
  for (int t = 0; t < n; ++t) {
    const int page = __ldcg(p.table + (size_t)s * p.ld + t / KV_PAGE);
    if (page < 0 || page >= p.n_pages) {
      if (lane == 0) set_error(p.err, ERR_PAGE);
      continue;
    }
    const size_t at = (((size_t)page * p.Hk + h / (p.H / p.Hk)) * KV_PAGE + t % KV_PAGE) * HD + lane * E;
    float d = 0.f;
    for (int e = 0; e < E; ++e) d = fmaf(q[e], __bfloat162float(p.k[at + e]), d);
    for (int x = 16; x; x >>= 1) d += __shfl_xor_sync(0xffffffffu, d, x);
    d *= rsqrtf((float)HD);
    const float now = fmaxf(m, d), f = __expf(m - now), a = __expf(d - now);
    m = now;
    l = l * f + a;
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + a * __bfloat162float(p.v[at + e]);
  }
  for (int e = 0; e < E; ++e) {
    const long long at = r * p.out_ld + h * HD + lane * E + e;
    const float y = l > 0.f ? o[e] / l : 0.f;
    if (BF16) static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(y);
    else static_cast<float*>(p.out)[at] = y;
  }
}

cudaError_t launch_chunk_attention(const ChunkAttnParams& p, int, cudaStream_t st, bool pdl) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(((long long)p.rows * p.H + 3) / 4));
  cfg.blockDim = dim3(128);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  if (p.bf16)
    return p.hd == 64 ? cudaLaunchKernelEx(&cfg, chunk_attention_kernel<true, 64>, p)
                      : cudaLaunchKernelEx(&cfg, chunk_attention_kernel<true, 128>, p);
  return p.hd == 64 ? cudaLaunchKernelEx(&cfg, chunk_attention_kernel<false, 64>, p)
                    : cudaLaunchKernelEx(&cfg, chunk_attention_kernel<false, 128>, p);
}

}  // namespace sdsat
