// Rules on logits before a token is selected: penalties of tokens that were used, biases, a mask of allowed tokens.
//
//   l <- seen ? (l > 0 ? l / rep : l rep) : l;   l <- l - freq c - (c > 0 ? pres : 0);   l <- l + bias;   l <- allowed ? l : -inf
//
// What bounds it is memory: logits are read and written once.  A CTA takes a stretch of the vocabulary for some rows of
// one sequence.  It first builds a word for each id of the stretch (seen in the prompt, the bias's place, times generated)
// from the history, and one bit an id that says whether the word holds anything: most of them do not, and a vector of
// logits whose bits are all clear is passed on without a look at the words.  Counts are whole numbers, added in any
// order; of two biases of an id the first is taken by a maximum, so results do not depend on the order of atomics.
//
// Output vectors of 16 bytes are aligned; a row of the input that lies at another offset is read in aligned vectors
// too, and shifted in registers (the next lane's vector by a shuffle).
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace sdsat {

constexpr int ADJ_THREADS = 256;
constexpr uint32_t ADJ_PROMPT = 1u << 31;
constexpr int ADJ_BIAS_SHIFT = 20;                            // 11 bits: ADJ_MAX_BIAS - place, 0: none
constexpr uint32_t ADJ_COUNT = (1u << ADJ_BIAS_SHIFT) - 1;   // a history and a block's tokens stay below it
static_assert(ADJ_MAX_HISTORY + SDSAT_ATT_MAXQ <= (int)ADJ_COUNT && ADJ_MAX_BIAS < 2048, "fields of a word");

struct AdjRow {
  float rep, freq, pres;
  const float* bias;
};

__device__ __forceinline__ float adjust_one(float l, uint32_t word, const AdjRow& a) {
  const uint32_t c = word & ADJ_COUNT, b = (word >> ADJ_BIAS_SHIFT) & 2047u;
  if (word & (ADJ_PROMPT | ADJ_COUNT)) l = l > 0.f ? __fdiv_rn(l, a.rep) : __fmul_rn(l, a.rep);
  if (c) l = __fsub_rn(__fsub_rn(l, __fmul_rn(a.freq, (float)c)), a.pres);
  if (b) l = __fadd_rn(l, __ldg(a.bias + (ADJ_MAX_BIAS - b)));
  return l;
}

// 32 bits of a bitmap from bit `at` on
__device__ __forceinline__ uint32_t bits_from(uint32_t lo, uint32_t hi, int at) { return __funnelshift_r(lo, hi, at & 31); }

// rp: rows of a sequence that one CTA takes; ch: ids of a stretch (a multiple of 32)
template <bool BF16>
__global__ void __launch_bounds__(ADJ_THREADS) adjust_kernel(const __grid_constant__ AdjustParams p, int rp, int ch, int parts, int chunks) {
  extern __shared__ uint32_t words[];       // [ch], then the bitmap [ch / 32 + 1]
  uint32_t* map = words + ch;
  constexpr int VEC = BF16 ? 8 : 4;         // values of 16 bytes
  const int tid = threadIdx.x, lane = tid & 31;
  const int chunk = blockIdx.x % chunks, part = blockIdx.x / chunks % parts, s = blockIdx.x / chunks / parts;
  const int v0 = chunk * ch, nv = min(ch, p.V - v0);
  const int j0 = part * rp, j1 = min(p.q, j0 + rp);
  for (int i = tid; i <= ch / 32; i += ADJ_THREADS) map[i] = 0;
  for (int i = tid; i < ch; i += ADJ_THREADS) words[i] = 0;
  __syncthreads();
  pdl_trigger();
  pdl_wait();
  bool wrong = false;
  auto note = [&](int id) {
    atomicOr(&map[id >> 5], 1u << (id & 31));
  };
  if (p.n_bias) {
    for (int i = tid; i < p.n_bias; i += ADJ_THREADS) {
      const int id = __ldg(p.bias_id + (size_t)s * p.n_bias + i);
      wrong |= id >= p.V;
      if (id >= v0 && id < v0 + nv) {
        atomicMax(&words[id - v0], (uint32_t)(ADJ_MAX_BIAS - i) << ADJ_BIAS_SHIFT);
        note(id - v0);
      }
    }
    __syncthreads();
  }
  if (p.history) {
    const int n = min(max(__ldg(p.history_len + s), 0), p.history_ld), np = p.prompt_len ? __ldg(p.prompt_len + s) : 0;
    const int* text = p.history + (size_t)s * p.history_ld;
#pragma unroll 4
    for (int i = tid; i < n; i += ADJ_THREADS) {
      const int id = __ldg(text + i);
      wrong |= id >= p.V;
      if (id >= v0 && id < v0 + nv) {
        if (i < np) atomicOr(&words[id - v0], ADJ_PROMPT);
        else atomicAdd(&words[id - v0], 1u);
        note(id - v0);
      }
    }
  }
  // the block's tokens of rows before j0 (a chain: row j comes after tokens 0 .. j)
  auto add = [&](int j, uint32_t n) {
    const int id = __ldg(p.tokens + s * p.q + j);
    wrong |= id >= p.V;
    if (id >= v0 && id < v0 + nv) {
      atomicAdd(&words[id - v0], n);
      note(id - v0);
    }
  };
  if (p.tokens && !p.anc && tid < j0) add(tid, 1u);
  AdjRow a;
  a.rep = p.repetition ? __ldg(p.repetition + s) : 1.f;
  a.freq = p.frequency ? __ldg(p.frequency + s) : 0.f;
  a.pres = p.presence ? __ldg(p.presence + s) : 0.f;
  a.bias = p.bias + (size_t)s * p.n_bias;

  for (int j = j0; j < j1; ++j) {
    const int r = s * p.q + j;
    const uint32_t mine = p.anc ? __ldg(p.anc + r) : 1u << j;
    if (p.tokens && tid < p.q && (mine >> tid & 1u)) add(tid, 1u);
    __syncthreads();
    // the stretch of this row in vectors that are aligned in the output: vector k holds ids first + k VEC ..
    const int size = BF16 ? 2 : 4;
    const uint8_t* in = static_cast<const uint8_t*>(p.in) + (r * p.in_ld + v0) * size;
    uint8_t* out = static_cast<uint8_t*>(p.out) + (r * p.out_ld + v0) * size;
    const int lead = (int)(reinterpret_cast<uintptr_t>(out) & 15u) / size, first = -lead;   // (values before the stretch)
    const int nvec = (nv + lead + VEC - 1) / VEC;
    const uintptr_t src = reinterpret_cast<uintptr_t>(in) - lead * size;      // of vector 0
    const int shift = (int)(src & 15u);
    const uint4* vin = reinterpret_cast<const uint4*>(src - shift);
    const uintptr_t lo = reinterpret_cast<uintptr_t>(in) & ~uintptr_t(15), hi = reinterpret_cast<uintptr_t>(in) + (size_t)nv * size;
    const uint32_t* allowed = p.allowed ? p.allowed + (size_t)r * p.allowed_ld : nullptr;
    // (a vector is loaded if it holds some of the stretch's values)
    auto load = [&](int k) {
      const uintptr_t at = reinterpret_cast<uintptr_t>(vin + k);
      return at >= lo && at < hi ? *(vin + k) : make_uint4(0u, 0u, 0u, 0u);
    };
    for (int k0 = tid - lane; k0 < nvec; k0 += ADJ_THREADS) {
      const int k = k0 + lane;
      uint4 x = load(k);
      if (shift) {
        uint4 y;
        y.x = __shfl_down_sync(0xffffffffu, x.x, 1);
        y.y = __shfl_down_sync(0xffffffffu, x.y, 1);
        y.z = __shfl_down_sync(0xffffffffu, x.z, 1);
        y.w = __shfl_down_sync(0xffffffffu, x.w, 1);
        if (lane == 31) y = load(k + 1);
        uint32_t t[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        if (shift & 8) {
#pragma unroll
          for (int i = 0; i < 6; ++i) t[i] = t[i + 2];
        }
        if (shift & 4) {
#pragma unroll
          for (int i = 0; i < 5; ++i) t[i] = t[i + 1];
        }
        if (BF16 && (shift & 2)) {
#pragma unroll
          for (int i = 0; i < 4; ++i) t[i] = __funnelshift_r(t[i], t[i + 1], 16);
        }
        x = make_uint4(t[0], t[1], t[2], t[3]);
      }
      if (k >= nvec) continue;
      const int e = first + k * VEC;        // id - v0 of the vector's first value
      // bits of ids e .. e + VEC - 1: touched, allowed
      const int w = max(e, 0) >> 5;
      uint32_t touched = bits_from(map[w], map[min(w + 1, ch / 32)], max(e, 0));
      uint32_t ok = 0xFFFFFFFFu;
      if (allowed) {
        const int wa = w + (v0 >> 5);
        const uint32_t a0 = __ldg(allowed + wa), a1 = wa + 1 < (p.V + 31) / 32 ? __ldg(allowed + wa + 1) : 0u;
        ok = bits_from(a0, a1, max(e, 0));
      }
      if (e < 0) touched <<= -e, ok <<= -e;
      touched &= (1u << VEC) - 1u;
      uint32_t v[4] = {x.x, x.y, x.z, x.w};
      if (touched) {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if ((touched >> i) & 1u) {
            const uint32_t word = words[e + i];
            if (BF16) {
              const uint32_t old = v[i / 2];
              const float l = __uint_as_float(i & 1 ? old & 0xFFFF0000u : old << 16);
              const uint32_t now = __bfloat16_as_ushort(__float2bfloat16_rn(adjust_one(l, word, a)));
              v[i / 2] = i & 1 ? (old & 0xFFFFu) | now << 16 : (old & 0xFFFF0000u) | now;
            } else {
              v[i / (BF16 ? 2 : 1)] = __float_as_uint(adjust_one(__uint_as_float(v[i / (BF16 ? 2 : 1)]), word, a));
            }
          }
      }
      if (allowed) {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (!((ok >> i) & 1u)) {
            if (BF16) v[i / 2] = i & 1 ? (v[i / 2] & 0xFFFFu) | 0xFF800000u : (v[i / 2] & 0xFFFF0000u) | 0xFF80u;
            else v[i / (BF16 ? 2 : 1)] = 0xFF800000u;
          }
      }
      uint8_t* at = out + (long long)e * size;
      if (e >= 0 && e + VEC <= nv) {
        *reinterpret_cast<uint4*>(at) = make_uint4(v[0], v[1], v[2], v[3]);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (e + i >= 0 && e + i < nv) {
            if (BF16) *reinterpret_cast<uint16_t*>(at + 2 * i) = (uint16_t)(v[i / 2] >> (i & 1 ? 16 : 0));
            else *reinterpret_cast<uint32_t*>(at + 4 * i) = v[i / (BF16 ? 2 : 1)];
          }
      }
    }
    if (j + 1 < j1) {
      __syncthreads();
      if (p.tokens && p.anc && tid < p.q && (mine >> tid & 1u)) add(tid, 0xFFFFFFFFu);   // (taken back: another branch follows)
    }
  }
  if (wrong) set_error(p.err, ERR_TOKEN);
}

cudaError_t adjust_prepare() {
  const int most = (16384 + 16384 / 32 + 1) * 4;
  cudaError_t e = cudaFuncSetAttribute(adjust_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(adjust_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  if (e == cudaSuccess) e = prefer_shared(adjust_kernel<false>);
  if (e == cudaSuccess) e = prefer_shared(adjust_kernel<true>);
  return e;
}

cudaError_t launch_adjust(const AdjustParams& p, int num_sms, cudaStream_t st, bool pdl) {
  // Long stretches and all rows of a sequence in one CTA read the history least often; shorter ones and a CTA for each
  // row where that leaves SMs without one.
  int ch = 16384, rp = p.q;
  auto ctas = [&](int c, int r) { return (long long)p.b * ((p.q + r - 1) / r) * ((p.V + c - 1) / c); };
  if (ctas(ch, rp) < 2 * num_sms) rp = 1;
  while (ch > 2048 && ctas(ch, rp) < 2 * num_sms) ch /= 2;
  const int parts = (p.q + rp - 1) / rp, chunks = (p.V + ch - 1) / ch;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.b * parts * chunks));
  cfg.blockDim = dim3(ADJ_THREADS);
  cfg.dynamicSmemBytes = (ch + ch / 32 + 1) * 4;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  return p.bf16 ? cudaLaunchKernelEx(&cfg, adjust_kernel<true>, p, rp, ch, parts, chunks)
                : cudaLaunchKernelEx(&cfg, adjust_kernel<false>, p, rp, ch, parts, chunks);
}

}  // namespace sdsat
