// Head norms, position rotation and append to pages for the rows of a ragged batch.
//
//   x' = x rsqrt(mean x^2 + eps) g;  (a, z) -> (a cos - z sin, a sin + z cos) for the pairs of the first `dims`
//   dimensions;  queries -> q_out, keys and values -> bf16 rows of the sequence's pages
//
// Written as y = x c + partner s with s negated in a pair's first place, one expression serves both layouts.  What
// bounds it is memory: every row is read and written once.  A warp takes RT_U x (128 / HD) heads of one row, four
// values a lane, all of them loaded before the row's sequence, slot and page are looked up, so that those
// dependent loads run beside the wide ones.  Norm and rotation stay in registers (shuffles); sums are fp32, the
// table's angles are reduced in double (an fp32 angle of position 30000 is off by 1e-3).
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace sdsat {

constexpr int RT_WARPS = 4;
constexpr int RT_U = 4;

__global__ void rope_table_kernel(const RopeBuild f, float2* turn, int n, int pairs) {
  const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= (long long)n * pairs) return;
  double s, c;
  sincos((double)(i / pairs) * f.f[i % pairs], &s, &c);
  turn[i] = make_float2((float)(c * f.magnitude), (float)(s * f.magnitude));
}
cudaError_t launch_rope_table(const RopeBuild& f, float2* turn, int n, int pairs, cudaStream_t st) {
  const long long all = (long long)n * pairs;
  rope_table_kernel<<<(unsigned)((all + 255) / 256), 256, 0, st>>>(f, turn, n, pairs);
  return cudaGetLastError();
}

// The sequence that row r belongs to (-1: none), by the whole warp: 32 places of the ascending starts at a time.
// Whatever the starts hold, the answer is a sequence with start[s] <= r < start[s+1], or -1.
__device__ __forceinline__ int sequence_of(const int* start, int b, int r, int lane, int& first) {
  int lo = 0, n = b + 1;
  while (n > 32) {
    const int step = (n + 31) / 32;
    const int at = lo + lane * step;
    const unsigned below = __ballot_sync(0xffffffffu, lane * step < n && __ldcg(start + at) <= r);
    if (!below) return -1;
    const int i = 31 - __clz(below);
    n = min(step, n - i * step);
    lo += i * step;
  }
  const int mine = lane < n ? __ldcg(start + lo + lane) : 0;
  const unsigned below = __ballot_sync(0xffffffffu, lane < n && mine <= r);
  if (!below) return -1;
  const int i = 31 - __clz(below), s = lo + i;
  first = __shfl_sync(0xffffffffu, mine, i);
  if (s >= b || r >= __ldcg(start + s + 1)) return -1;
  return s;
}

__device__ __forceinline__ float one_of(const float (&v)[4], int i) {
  const float a = i & 1 ? v[1] : v[0], z = i & 1 ? v[3] : v[2];
  return i & 2 ? z : a;
}

template <bool BF16, int HD>
__global__ void __launch_bounds__(RT_WARPS * 32) rotary_append_kernel(const __grid_constant__ RotaryParams p, int groups) {
  constexpr int HPW = 128 / HD, LANES = 32 / HPW;   // heads side by side in a warp, lanes of one
  const int lane = threadIdx.x & 31, sub = lane / LANES, e0 = lane % LANES * 4;
  const long long w = (long long)blockIdx.x * RT_WARPS + (threadIdx.x >> 5);
  const int r = (int)(w / groups), g = (int)(w % groups);
  pdl_trigger();
  pdl_wait();
  if (r >= p.rows) return;
  const int NH = p.H + 2 * p.Hk;
  float x[RT_U][4];
#pragma unroll
  for (int u = 0; u < RT_U; ++u) {
    const int h = (g * RT_U + u) * HPW + sub;
    const void* src = p.q;
    long long at = r * p.q_ld + h * HD + e0;
    if (h >= p.H + p.Hk) src = p.v, at = r * p.v_ld + (h - p.H - p.Hk) * HD + e0;
    else if (h >= p.H) src = p.k, at = r * p.k_ld + (h - p.H) * HD + e0;
    if (h < NH) {
      if (BF16) {
        const uint2 b = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(src) + at);
        x[u][0] = __uint_as_float(b.x << 16);
        x[u][1] = __uint_as_float(b.x & 0xFFFF0000u);
        x[u][2] = __uint_as_float(b.y << 16);
        x[u][3] = __uint_as_float(b.y & 0xFFFF0000u);
      } else {
        const float4 f = *reinterpret_cast<const float4*>(static_cast<const float*>(src) + at);
        x[u][0] = f.x, x[u][1] = f.y, x[u][2] = f.z, x[u][3] = f.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[u][i] = 0.f;
    }
  }

  int first = 0;
  const int s = sequence_of(p.start, p.b, r, lane, first);
  if (s < 0) return;
  const long long slot = (long long)__ldcg(p.len + s) + (r - first);
  // the row of the sequence's page, -1: not written
  long long row = -1;
  if ((g + 1) * RT_U * HPW > p.H) {
    if (slot >= 0 && slot < (long long)p.pages.ld * KV_PAGE) {
      const int page = __ldcg(p.pages.table + (size_t)s * p.pages.ld + slot / KV_PAGE);
      if (page >= 0 && page < p.pages.n && (!p.pages.refs || __ldcg(p.pages.refs + page) == 1))
        row = (long long)page * p.Hk * KV_PAGE + slot % KV_PAGE;
    }
    if (row < 0 && lane == 0) set_error(p.err, ERR_CAPACITY);
  }
  long long pos = p.positions ? __ldcg(p.positions + r) : slot;
  if (pos < 0 || pos >= p.rope.n) {
    if (lane == 0) set_error(p.err, ERR_POSITION);
    pos = pos < 0 ? 0 : p.rope.n - 1;
  }
  // this lane's four places: y = x c + partner s
  const int dims = p.rope.dims, half = dims / 2, d = half & 3;
  float c[4], t[4];
  bool turned[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = e0 + i;
    turned[i] = e < dims;
    const bool head = p.rope.interleaved ? !(e & 1) : e < half;
    const int pair = p.rope.interleaved ? e >> 1 : head ? e : e - half;
    const float2 cs = turned[i] ? __ldg(p.rope.turn + pos * half + pair) : make_float2(1.f, 0.f);
    c[i] = cs.x;
    t[i] = head ? -cs.y : cs.y;
  }
#pragma unroll
  for (int u = 0; u < RT_U; ++u) {
    const int h = (g * RT_U + u) * HPW + sub;
    const bool is_q = h < p.H, is_v = h >= p.H + p.Hk;
    float y[4] = {x[u][0], x[u][1], x[u][2], x[u][3]};
    const __nv_bfloat16* gain = is_q ? p.q_gain : is_v ? nullptr : p.k_gain;
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) sq = fmaf(y[i], y[i], sq);
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
    if (gain) {
      const float f = rsqrtf(sq * (1.0f / HD) + p.eps);
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = y[i] * f * __bfloat162float(gain[e0 + i]);
    }
    float z[4];
    if (p.rope.interleaved) {
#pragma unroll
      for (int i = 0; i < 4; ++i) z[i] = y[i ^ 1];
    } else {
      // the partner of place e is e + half or e - half: (half >> 2) lanes on or back, and d places
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float on = __shfl_sync(0xffffffffu, one_of(y, (i + d) & 3), lane + (half >> 2) + ((i + d) >> 2));
        const float back = __shfl_sync(0xffffffffu, one_of(y, (i - d) & 3), lane - (half >> 2) - (i < d ? 1 : 0));
        z[i] = e0 + i < half ? on : back;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (turned[i] && !is_v) y[i] = fmaf(y[i], c[i], z[i] * t[i]);
    __nv_bfloat162 lo = __floats2bfloat162_rn(y[0], y[1]), hi = __floats2bfloat162_rn(y[2], y[3]);
    const uint2 packed = make_uint2(*reinterpret_cast<uint32_t*>(&lo), *reinterpret_cast<uint32_t*>(&hi));
    if (is_q) {
      const long long at = r * p.out_ld + h * HD + e0;
      if (BF16) *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.q_out) + at) = packed;
      else *reinterpret_cast<float4*>(static_cast<float*>(p.q_out) + at) = make_float4(y[0], y[1], y[2], y[3]);
    } else if (h < NH && row >= 0) {
      const int hk = is_v ? h - p.H - p.Hk : h - p.H;
      *reinterpret_cast<uint2*>((is_v ? p.v_pages : p.k_pages) + (row + (long long)hk * KV_PAGE) * HD + e0) = packed;
    }
  }
}

cudaError_t rotary_prepare() {
  cudaError_t e = prefer_shared(rotary_append_kernel<false, 64>);
  if (e == cudaSuccess) e = prefer_shared(rotary_append_kernel<false, 128>);
  if (e == cudaSuccess) e = prefer_shared(rotary_append_kernel<true, 64>);
  if (e == cudaSuccess) e = prefer_shared(rotary_append_kernel<true, 128>);
  return e;
}

cudaError_t launch_rotary_append(const RotaryParams& p, int, cudaStream_t st, bool pdl) {
  const int per = RT_U * (128 / p.hd), groups = (p.H + 2 * p.Hk + per - 1) / per;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(((long long)p.rows * groups + RT_WARPS - 1) / RT_WARPS));
  cfg.blockDim = dim3(RT_WARPS * 32);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  if (p.bf16)
    return p.hd == 64 ? cudaLaunchKernelEx(&cfg, rotary_append_kernel<true, 64>, p, groups)
                      : cudaLaunchKernelEx(&cfg, rotary_append_kernel<true, 128>, p, groups);
  return p.hd == 64 ? cudaLaunchKernelEx(&cfg, rotary_append_kernel<false, 64>, p, groups)
                    : cudaLaunchKernelEx(&cfg, rotary_append_kernel<false, 128>, p, groups);
}

}  // namespace sdsat
