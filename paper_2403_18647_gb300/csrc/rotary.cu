// Head norms, position rotation and append to pages for the rows of a ragged batch.
//
//   x' = x rsqrt(mean x^2 + eps) g;  (a, z) -> (a cos - z sin, a sin + z cos) for the pairs of the first `dims`
//   dimensions;  queries -> q_out, keys and values -> bf16 rows of the sequence's pages
//
// Written as y = x c + partner s with s negated in a pair's first place, one expression serves both layouts.  What
// bounds it is memory, then instructions: rows are read and written once, 16 bytes a lane.  A warp takes heads of one
// row, RT_U of them on each of its parts at a time, the next ones asked for before these are worked on; the first are
// asked for before the row's sequence, slot and page are looked up, so that those dependent loads run beside the wide
// ones.  Norm and rotation stay in registers (shuffles); pairs that lanes do not hold alike go through shared memory (by
// shuffles and selections of the values 2645 rows of 32 / 8 bf16 heads took 60 us for 14).  Sums are fp32, the table's
// angles are reduced in double (an fp32 angle of position 30000 is off by 1e-3).
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace sdsat {

constexpr int RT_WARPS = 4;
// (12 sequences of up to 1100 rows of 32 / 8 bf16 heads: 45 us, 4.9 TB/s; 62 with one, 60 with four, of more registers)
constexpr int RT_U = 2;

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

enum RotaryLayout : int {
  ROT_INTERLEAVED = 0,   // the partner of place e is e ^ 1
  ROT_LANES = 1,         // e + half or e - half, whole lanes away
  ROT_ANY = 2,           // ... at any place of another lane
};

// heads: how many of a row a warp takes, a multiple of RT_U times its parts
template <bool BF16, int HD, int LAYOUT, bool NORM>
__global__ void __launch_bounds__(RT_WARPS * 32) rotary_append_kernel(const __grid_constant__ RotaryParams p, int groups, int heads) {
  constexpr int E = BF16 ? 8 : 4;                        // values of a lane
  constexpr int LANES = HD / E, PARTS = 32 / LANES;      // lanes of a head, heads side by side in a warp
  using Raw = uint4;
  __shared__ __align__(16) float stage[LAYOUT == ROT_ANY ? RT_WARPS : 1][LAYOUT == ROT_ANY ? PARTS * HD : 4];
  const int lane = threadIdx.x & 31, part = lane / LANES, e0 = lane % LANES * E;
  const long long w = (long long)blockIdx.x * RT_WARPS + (threadIdx.x >> 5);
  const int r = (int)(w / groups), h0 = (int)(w % groups) * heads + part;
  pdl_trigger();
  pdl_wait();
  if (r >= p.rows) return;
  const int Hqk = p.H + p.Hk, NH = min(Hqk + p.Hk, h0 - part + heads);
  constexpr int size = BF16 ? 2 : 4;
  // where head h of queries, keys or values stands: base + h HD values
  const char* q_row = static_cast<const char*>(p.q) + (r * p.q_ld + e0) * size;
  const char* k_row = static_cast<const char*>(p.k) + (r * p.k_ld - (long long)p.H * HD + e0) * size;
  const char* v_row = static_cast<const char*>(p.v) + (r * p.v_ld - (long long)Hqk * HD + e0) * size;
  auto load = [&](int h) { return h < NH ? *reinterpret_cast<const Raw*>((h < p.H ? q_row : h < Hqk ? k_row : v_row) + (long long)h * (HD * size)) : make_uint4(0u, 0u, 0u, 0u); };
  Raw raw[RT_U];
#pragma unroll
  for (int u = 0; u < RT_U; ++u) raw[u] = load(h0 + u * PARTS);

  int first = 0;
  const int s = sequence_of(p.start, p.b, r, lane, first);
  if (s < 0) return;
  const long long slot = (long long)__ldcg(p.len + s) + (r - first);
  // the row of the sequence's page, -1: not written
  long long row = -1;
  if (h0 - part + heads > p.H) {
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
  char* out_row = static_cast<char*>(p.q_out) + (r * p.out_ld + e0) * size;
  __nv_bfloat16* k_slot = p.k_pages + (row - (long long)p.H * KV_PAGE) * HD + e0;
  __nv_bfloat16* v_slot = p.v_pages + (row - (long long)Hqk * KV_PAGE) * HD + e0;

  // this lane's places: y = x c + partner t
  const int dims = p.rope.dims, half = dims / 2;
  const float2* turn = p.rope.turn + pos * half;
  const int e_pair = LAYOUT == ROT_INTERLEAVED ? e0 >> 1 : e0 < half ? e0 : e0 - half;   // (ROT_LANES: of the first place)
  float c[E], t[E];
  const bool turned = e0 < dims;   // (ROT_ANY: some of the places)
  if (LAYOUT == ROT_ANY) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int e = e0 + i;
      const float2 cs = e < dims ? __ldg(turn + (e < half ? e : e - half)) : make_float2(1.f, 0.f);
      c[i] = cs.x;
      t[i] = e < half ? -cs.y : cs.y;
    }
  } else if (LAYOUT == ROT_LANES) {
#pragma unroll
    for (int i = 0; i < E; i += 2) {   // (half is even: rows of the table are 16-byte aligned)
      const float4 cs = turned ? __ldg(reinterpret_cast<const float4*>(turn + e_pair + i)) : make_float4(1.f, 0.f, 1.f, 0.f);
      c[i] = cs.x, c[i + 1] = cs.z;
      t[i] = e0 < half ? -cs.y : cs.y, t[i + 1] = e0 < half ? -cs.w : cs.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      const float2 cs = e0 + i < dims ? __ldg(turn + e_pair + i / 2) : make_float2(1.f, 0.f);
      c[i] = c[i + 1] = cs.x;
      t[i] = -cs.y, t[i + 1] = cs.y;
    }
  }
  uint32_t gain[2][E / 2];   // of queries and keys
  if (NORM)
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const uint16_t* from = reinterpret_cast<const uint16_t*>(g ? p.k_gain : p.q_gain);
#pragma unroll
      for (int i = 0; i < E / 2; ++i) gain[g][i] = from ? (uint32_t)from[e0 + 2 * i] | (uint32_t)from[e0 + 2 * i + 1] << 16 : 0u;
    }
  const int on = lane + (e0 < half ? half / E : -(half / E));   // ROT_LANES: the partner's lane

  for (int h_at = h0; h_at - part < NH; h_at += RT_U * PARTS) {
    Raw now[RT_U];
#pragma unroll
    for (int u = 0; u < RT_U; ++u) {
      now[u] = raw[u];
      raw[u] = load(h_at + (RT_U + u) * PARTS);
    }
#pragma unroll
    for (int u = 0; u < RT_U; ++u) {
      const int h = h_at + u * PARTS;
      const bool is_v = h >= Hqk, is_q = h < p.H;
      float y[E];
      const uint32_t word[4] = {now[u].x, now[u].y, now[u].z, now[u].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (BF16) {
          y[(2 * i) % E] = __uint_as_float(word[i] << 16);
          y[(2 * i + 1) % E] = __uint_as_float(word[i] & 0xFFFF0000u);
        } else {
          y[i] = __uint_as_float(word[i]);
        }
      }
      if (NORM) {
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) sq = fmaf(y[i], y[i], sq);
#pragma unroll
        for (int o = LANES / 2; o; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
        if (!is_v && (is_q ? p.q_gain : p.k_gain)) {
          const float f = rsqrtf(sq * (1.0f / HD) + p.eps);
#pragma unroll
          for (int i = 0; i < E; i += 2) {
            const uint32_t g = is_q ? gain[0][i / 2] : gain[1][i / 2];
            y[i] = y[i] * f * __uint_as_float(g << 16);
            y[i + 1] = y[i + 1] * f * __uint_as_float(g & 0xFFFF0000u);
          }
        }
      }
      float z[E];
      if (LAYOUT == ROT_INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < E; ++i) z[i] = y[i ^ 1];
      } else if (LAYOUT == ROT_LANES) {
#pragma unroll
        for (int i = 0; i < E; ++i) z[i] = __shfl_sync(0xffffffffu, y[i], on);
      } else {
        // partners stand at any places of other lanes: through shared memory
        float* head = stage[LAYOUT == ROT_ANY ? threadIdx.x >> 5 : 0] + part * HD;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < E; i += 4)
          if (e0 + i < dims) *reinterpret_cast<float4*>(head + e0 + i) = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const int e = e0 + i;
          z[i] = e < dims ? head[e < half ? e + half : e - half] : 0.f;
        }
      }
      if (!is_v) {
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (LAYOUT == ROT_LANES ? turned : e0 + i < dims) y[i] = fmaf(y[i], c[i], z[i] * t[i]);
      }
      if (h >= NH) continue;
      uint32_t packed[E / 2];
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        const __nv_bfloat162 two = __floats2bfloat162_rn(y[i], y[i + 1]);
        packed[i / 2] = *reinterpret_cast<const uint32_t*>(&two);
      }
      if (is_q && !BF16) {
        *reinterpret_cast<float4*>(out_row + (long long)h * (HD * size)) = make_float4(y[0], y[1], y[2], y[3]);
      } else if (is_q || row >= 0) {
        char* to = is_q ? out_row + (long long)h * (HD * size) : reinterpret_cast<char*>((is_v ? v_slot : k_slot) + (long long)h * (KV_PAGE * HD));
        if constexpr (BF16) *reinterpret_cast<uint4*>(to) = make_uint4(packed[0], packed[1], packed[2], packed[3]);
        else *reinterpret_cast<uint2*>(to) = make_uint2(packed[0], packed[1]);
      }
    }
  }
}

template <bool BF16, int HD, int LAYOUT, bool NORM>
static int rt_resident = 0;   // warps on an SM

template <bool BF16, int HD, int LAYOUT, bool NORM>
static cudaError_t rt_prepare() {
  const auto kernel = rotary_append_kernel<BF16, HD, LAYOUT, NORM>;
  cudaError_t e = prefer_shared(kernel);
  int ctas = 0;
  if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&ctas, kernel, RT_WARPS * 32, 0);
  rt_resident<BF16, HD, LAYOUT, NORM> = std::max(1, ctas) * RT_WARPS;
  return e;
}
template <bool BF16, int HD, int LAYOUT>
static cudaError_t rt_prepare() {
  const cudaError_t e = rt_prepare<BF16, HD, LAYOUT, false>();
  return e == cudaSuccess ? rt_prepare<BF16, HD, LAYOUT, true>() : e;
}
template <bool BF16, int HD>
static cudaError_t rt_prepare() {
  cudaError_t e = rt_prepare<BF16, HD, ROT_INTERLEAVED>();
  if (e == cudaSuccess) e = rt_prepare<BF16, HD, ROT_LANES>();
  return e == cudaSuccess ? rt_prepare<BF16, HD, ROT_ANY>() : e;
}
cudaError_t rotary_prepare() {
  cudaError_t e = rt_prepare<false, 64>();
  if (e == cudaSuccess) e = rt_prepare<false, 128>();
  if (e == cudaSuccess) e = rt_prepare<true, 64>();
  return e == cudaSuccess ? rt_prepare<true, 128>() : e;
}

// Among how many warps a row's `steps` are divided.  A warp costs its steps and its start, all that are resident run beside
// one another, and what is more than those takes its share and a tail; fp32, close to the copy rate, has its tail in one
// round too, bf16 is bound by what a warp issues.  Within 2 % of the best division that was measured at 27 sizes of each type
// (us, bf16 / fp32 of 32 and 8 heads: 400 rows 5.9 / 6.3, a step to each warp 7.2 / 8.2; 800 7.5 / 8.4, 8.8 / 13.0;
// 4095 fp32 rows of 40 and 40 heads 75, a row to each warp 87).
static int rt_groups(bool bf16, long long rows, int steps, long long resident) {
  const double start = bf16 ? 2.5 : 1.5, tail = 0.3;
  const long long first = std::max(1ll, std::min((long long)steps, resident / rows)), last = std::min((long long)steps, 4 * resident / rows + 1);
  long long groups = first;
  double least = 1e30;
  for (long long g = first; g <= std::max(first, last); ++g) {
    const long long per = (steps + g - 1) / g;
    const double rounds = (double)(rows * g) / (double)resident;
    const double cost = (start + per) * (rounds > 1. ? rounds + tail : bf16 ? 1. : 1. + tail);
    if (cost < least) least = cost, groups = g;
  }
  return (int)groups;
}
template <bool BF16, int HD, int LAYOUT, bool NORM>
static cudaError_t rt_launch(const RotaryParams& p, int num_sms, cudaStream_t st, bool pdl) {
  constexpr int step = RT_U * (32 * (BF16 ? 8 : 4) / HD);   // heads of a warp at a time
  const int steps = (p.H + 2 * p.Hk + step - 1) / step;
  int groups = rt_groups(BF16, p.rows, steps, (long long)rt_resident<BF16, HD, LAYOUT, NORM> * num_sms);
  const int per = (steps + groups - 1) / groups;
  groups = (steps + per - 1) / per;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(((long long)p.rows * groups + RT_WARPS - 1) / RT_WARPS));
  cfg.blockDim = dim3(RT_WARPS * 32);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, rotary_append_kernel<BF16, HD, LAYOUT, NORM>, p, groups, per * step);
}
template <bool BF16, int HD, int LAYOUT>
static cudaError_t rt_launch(const RotaryParams& p, int num_sms, cudaStream_t st, bool pdl) {
  return p.q_gain || p.k_gain ? rt_launch<BF16, HD, LAYOUT, true>(p, num_sms, st, pdl) : rt_launch<BF16, HD, LAYOUT, false>(p, num_sms, st, pdl);
}
template <bool BF16, int HD>
static cudaError_t rt_launch(const RotaryParams& p, int num_sms, cudaStream_t st, bool pdl) {
  if (p.rope.interleaved) return rt_launch<BF16, HD, ROT_INTERLEAVED>(p, num_sms, st, pdl);
  return p.rope.dims / 2 % (BF16 ? 8 : 4) ? rt_launch<BF16, HD, ROT_ANY>(p, num_sms, st, pdl) : rt_launch<BF16, HD, ROT_LANES>(p, num_sms, st, pdl);
}
cudaError_t launch_rotary_append(const RotaryParams& p, int num_sms, cudaStream_t st, bool pdl) {
  if (p.bf16) return p.hd == 64 ? rt_launch<true, 64>(p, num_sms, st, pdl) : rt_launch<true, 128>(p, num_sms, st, pdl);
  return p.hd == 64 ? rt_launch<false, 64>(p, num_sms, st, pdl) : rt_launch<false, 128>(p, num_sms, st, pdl);
}

}  // namespace sdsat
