// Rules on logits before a token is selected: penalties of tokens that were used, biases, a mask of allowed tokens.
//
//   l <- seen ? (l > 0 ? l / rep : l rep) : l;   l <- l - freq c - (c > 0 ? pres : 0);   l <- l + bias;   l <- allowed ? l : -inf
//
// Logits are read and written once, but what bounds it is instructions.  A CTA takes a stretch of the vocabulary for some
// rows of one sequence: it asks for the first vectors of a row, meanwhile counts the history into a word for each id of
// the stretch (seen in the prompt, the bias's place, times generated) and lists the ids whose word holds anything, writes
// the row with nothing but the mask applied, and computes the listed ids again from their logits.  256 rows of 128003 bf16
// after up to 9000 tokens take 72 us (1.98 TB/s), of which loads, masks and stores alone 37, counting 20, the listed ids 14.
// (Counts by atomics of each thread and a scan of the words for the list 83; a stretch of 32640 ids on 1024 threads 78;
// a cluster of CTAs that share the counts 126; counts in a kernel of its own 109.)
//
// Counts are whole numbers, added in any order, of two biases of an id the first is taken by a maximum, and an id is
// listed once, so results do not depend on the order of atomics.
//
// Output vectors of 16 bytes are aligned; a row of the input that lies at another offset is read in aligned vectors
// too, and shifted in registers (the next lane's vector by a shuffle).
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace sdsat {

// Vectors of a thread in flight; a long stretch takes its threads two turns (us, 256 rows of 128003 bf16: 72; four and one turn
// 76, with registers spilled; one and four turns 75).
constexpr int ADJ_U = 2;
constexpr int ADJ_STRETCH = 16384;                            // ids of a stretch at most
constexpr uint32_t ADJ_PROMPT = 1u << 31;
constexpr int ADJ_BIAS_SHIFT = 20;                            // 11 bits: ADJ_MAX_BIAS - place, 0: none
constexpr uint32_t ADJ_COUNT = (1u << ADJ_BIAS_SHIFT) - 1;   // a history and a block's tokens stay below it
static_assert(ADJ_MAX_HISTORY + SDSAT_ATT_MAXQ <= (int)ADJ_COUNT && ADJ_MAX_BIAS < 2048, "fields of a word");
constexpr size_t adj_smem(int ch) { return (size_t)ch * 6 + 16; }   // words, list, its length (and its length without tokens)

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

// 16 bytes from byte 4 W + 2 half of two vectors on
template <int W>
__device__ __forceinline__ uint4 adj_shift(const uint4& x, const uint4& y, bool half) {
  const uint32_t t[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
  if (!half) return make_uint4(t[W], t[W + 1], t[W + 2], t[W + 3]);
  return make_uint4(__funnelshift_r(t[W], t[W + 1], 16), __funnelshift_r(t[W + 1], t[W + 2], 16), __funnelshift_r(t[W + 2], t[W + 3], 16),
                    __funnelshift_r(t[W + 3], t[W + 4], 16));
}
// the sign of a byte of x in all bits of the byte at each place (selectors 8 + byte)
template <uint32_t SELECT>
__device__ __forceinline__ uint32_t adj_signs(uint32_t x) {
  uint32_t r;
  asm("prmt.b32 %0, %1, %1, %2;" : "=r"(r) : "r"(x), "n"(SELECT));
  return r;
}
// the values of a vector whose bits are clear become -inf
template <bool BF16>
__device__ __forceinline__ void adj_mask(uint4& x, uint32_t ok) {
  if (BF16) {
    // four bits to the tops of four bytes, each top to two bytes
    const uint32_t lo = ((ok & 15u) * 0x10204080u) & 0x80808080u, hi = (((ok >> 4) & 15u) * 0x10204080u) & 0x80808080u;
    const uint32_t k[4] = {adj_signs<0x9988>(lo), adj_signs<0xBBAA>(lo), adj_signs<0x9988>(hi), adj_signs<0xBBAA>(hi)};
    x.x = (x.x & k[0]) | (0xFF80FF80u & ~k[0]);
    x.y = (x.y & k[1]) | (0xFF80FF80u & ~k[1]);
    x.z = (x.z & k[2]) | (0xFF80FF80u & ~k[2]);
    x.w = (x.w & k[3]) | (0xFF80FF80u & ~k[3]);
  } else {
    if (!(ok & 1u)) x.x = 0xFF800000u;
    if (!(ok & 2u)) x.y = 0xFF800000u;
    if (!(ok & 4u)) x.z = 0xFF800000u;
    if (!(ok & 8u)) x.w = 0xFF800000u;
  }
}

// rp: rows of a sequence that one CTA takes; ch: ids of a stretch (a multiple of 128, ADJ_STRETCH at most)
template <bool BF16, int ADJ_THREADS>
__global__ void __launch_bounds__(ADJ_THREADS, 1024 / ADJ_THREADS) adjust_kernel(const __grid_constant__ AdjustParams p, int rp, int ch, int parts, int chunks) {
  extern __shared__ uint4 adj_mem[];
  uint32_t* words = reinterpret_cast<uint32_t*>(adj_mem);            // [ch]
  uint16_t* list = reinterpret_cast<uint16_t*>(words + ch);          // [ch], each id once
  int* listed = reinterpret_cast<int*>(list + ch);
  __shared__ uint16_t queue[ADJ_THREADS / 32][64];           // of a warp: tokens of the stretch, bit 15: of the prompt
  constexpr int VEC = BF16 ? 8 : 4;         // values of 16 bytes
  constexpr int size = BF16 ? 2 : 4;
  const int tid = threadIdx.x, lane = tid & 31;
  const int chunk = blockIdx.x % chunks, part = blockIdx.x / chunks % parts, s = blockIdx.x / chunks / parts;
  const int v0 = chunk * ch, nv = min(ch, p.V - v0);
  const int j0 = part * rp, j1 = min(p.q, j0 + rp);
  for (int i = tid; i < ch / 4; i += ADJ_THREADS) adj_mem[i] = make_uint4(0u, 0u, 0u, 0u);
  if (tid == 0) *listed = 0;
  pdl_trigger();
  pdl_wait();
  const int n_history = p.history ? __ldg(p.history_len + s) : 0, n_prompt = p.history && p.prompt_len ? __ldg(p.prompt_len + s) : 0;
  int largest = -1;   // of the ids
  auto here = [&](int id) { return (uint32_t)id - (uint32_t)v0 < (uint32_t)nv; };
  auto list_it = [&](uint32_t before, int id) {
    if (before == 0) list[atomicAdd(listed, 1)] = (uint16_t)(id - v0);
  };
  auto token = [&](int id, bool prompt) {
    largest = max(largest, id);
    if (here(id)) list_it(prompt ? atomicOr(&words[id - v0], ADJ_PROMPT) : atomicAdd(&words[id - v0], 1u), id);
  };
  AdjRow a;
  a.rep = p.repetition ? __ldg(p.repetition + s) : 1.f;
  a.freq = p.frequency ? __ldg(p.frequency + s) : 0.f;
  a.pres = p.presence ? __ldg(p.presence + s) : 0.f;
  a.bias = p.bias + (size_t)s * p.n_bias;
  const bool branches = p.tokens && p.anc && j1 - j0 > 1;   // rows with other tokens each

  for (int j = j0; j < j1; ++j) {
    const int r = s * p.q + j;
    const uint32_t mine = p.anc ? __ldg(p.anc + r) : 1u << j;
    // the stretch of this row in vectors that are aligned in the output: vector k holds ids k VEC - lead ..
    const uint8_t* in = static_cast<const uint8_t*>(p.in) + (r * p.in_ld + v0) * size;
    uint8_t* out = static_cast<uint8_t*>(p.out) + (r * p.out_ld + v0) * size;
    const int lead = (int)(reinterpret_cast<uintptr_t>(out) & 15u) / size;    // (values before the stretch)
    const int nvec = (nv + lead + VEC - 1) / VEC;
    const uintptr_t src = reinterpret_cast<uintptr_t>(in) - lead * size;      // of vector 0
    const int shift = (int)(src & 15u);
    const uint4* vin = reinterpret_cast<const uint4*>(src - shift);
    uint4* vout = reinterpret_cast<uint4*>(out - lead * size);
    // the input's vectors that hold some of the stretch's values
    const int v_first = (lead * size + shift) / 16, v_last = (lead * size + shift + nv * size - 1) / 16;
    const uint32_t* allowed = p.allowed ? p.allowed + (size_t)r * p.allowed_ld + (v0 >> 5) : nullptr;
    const int mask_words = (p.V + 31) / 32 - (v0 >> 5);
    uint4 x[ADJ_U];
    uint32_t mask[ADJ_U][2];   // the words that a vector's bits begin in and may go on in
    auto load = [&](int k) { return k >= v_first && k <= v_last ? vin[k] : make_uint4(0u, 0u, 0u, 0u); };
    auto ask = [&](int k0) {
#pragma unroll
      for (int u = 0; u < ADJ_U; ++u) {
        const int k = k0 + u * ADJ_THREADS, e = k * VEC - lead;   // id - v0 of the vector's first value
        x[u] = load(k);
        if (allowed && k < nvec) {
          const int w = max(e, 0) >> 5;
          mask[u][0] = __ldg(allowed + w);
          mask[u][1] = __ldg(allowed + min(w + 1, mask_words - 1));
        }
      }
    };
    auto pass_on = [&](int k0) {
#pragma unroll
      for (int u = 0; u < ADJ_U; ++u) {
        const int k = k0 + u * ADJ_THREADS;
        if (shift) {
          uint4 y;
          y.x = __shfl_down_sync(0xffffffffu, x[u].x, 1);
          y.y = __shfl_down_sync(0xffffffffu, x[u].y, 1);
          y.z = __shfl_down_sync(0xffffffffu, x[u].z, 1);
          y.w = __shfl_down_sync(0xffffffffu, x[u].w, 1);
          if (lane == 31) y = load(k + 1);
          const bool half = BF16 && (shift & 2);
          x[u] = shift < 4 ? adj_shift<0>(x[u], y, half) : shift < 8 ? adj_shift<1>(x[u], y, half) : shift < 12 ? adj_shift<2>(x[u], y, half)
                                                                                                      : adj_shift<3>(x[u], y, half);
        }
        if (allowed) {
          const int e = k * VEC - lead;
          adj_mask<BF16>(x[u], e < 0 ? mask[u][0] << -e : __funnelshift_r(mask[u][0], mask[u][1], e));
        }
        if (k > 0 && k < nvec - 1) {
          vout[k] = x[u];
        } else if (k < nvec) {   // (perhaps not whole)
          const uint32_t v[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
          const int e = k * VEC - lead;
#pragma unroll
          for (int i = 0; i < VEC; ++i)
            if (e + i >= 0 && e + i < nv) {
              if (BF16) *(reinterpret_cast<uint16_t*>(vout + k) + i) = (uint16_t)(v[i / 2] >> (i & 1 ? 16 : 0));
              else *(reinterpret_cast<uint32_t*>(vout + k) + i) = v[i / (BF16 ? 2 : 1)];
            }
        }
      }
    };
    ask(tid);
    if (j == j0) {   // the sequence's words, while the first vectors are on their way
      __syncthreads();
      if (p.n_bias) {
        for (int i = tid; i < p.n_bias; i += ADJ_THREADS) {
          const int id = __ldg(p.bias_id + (size_t)s * p.n_bias + i);
          largest = max(largest, id);
          if (here(id)) list_it(atomicMax(&words[id - v0], (uint32_t)(ADJ_MAX_BIAS - i) << ADJ_BIAS_SHIFT), id);
        }
        __syncthreads();
      }
      if (p.history) {
        // Few of a history's tokens are in the stretch, but some of a warp's 32 nearly always: they are queued, and
        // counted when there is one for each lane.
        const int n = min(max(n_history, 0), p.history_ld);
        const int* text = p.history + (size_t)s * p.history_ld;
        uint16_t* q = queue[tid >> 5];
        int held = 0;
        auto count = [&](uint16_t t) {
          const int id = v0 + (t & 0x7FFF);
          list_it(t & 0x8000 ? atomicOr(&words[id - v0], ADJ_PROMPT) : atomicAdd(&words[id - v0], 1u), id);
        };
        auto offer = [&](int id, int i) {
          largest = max(largest, id);
          const bool mine_too = here(id);
          const unsigned some = __ballot_sync(0xffffffffu, mine_too);
          if (!some) return;
          if (mine_too) q[held + __popc(some & ((1u << lane) - 1u))] = (uint16_t)((id - v0) | (i < n_prompt ? 0x8000 : 0));
          held += __popc(some);
          __syncwarp();
          if (held < 32) return;
          count(q[lane]);
          __syncwarp();
          const uint16_t rest = q[32 + lane];
          __syncwarp();
          q[lane] = rest;
          held -= 32;
          __syncwarp();
        };
        int i0 = 0;
        if ((reinterpret_cast<uintptr_t>(text) & 15u) == 0) {   // four at a time
          constexpr int N = 2;
#pragma unroll 1
          for (; i0 + 4 * ADJ_THREADS * (N - 1) < n; i0 += 4 * ADJ_THREADS * N) {
            int4 id[N];
#pragma unroll
            for (int u = 0; u < N; ++u) {
              const int i = i0 + 4 * (u * ADJ_THREADS + tid);
              id[u] = i + 3 < n ? __ldg(reinterpret_cast<const int4*>(text + i)) : make_int4(-1, -1, -1, -1);
              if (i < n && i + 3 >= n) {
                id[u].x = __ldg(text + i);
                if (i + 1 < n) id[u].y = __ldg(text + i + 1);
                if (i + 2 < n) id[u].z = __ldg(text + i + 2);
              }
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
              const int i = i0 + 4 * (u * ADJ_THREADS + tid);
              offer(id[u].x, i);
              offer(id[u].y, i + 1);
              offer(id[u].z, i + 2);
              offer(id[u].w, i + 3);
            }
          }
        }
#pragma unroll 4
        for (; i0 < n; i0 += ADJ_THREADS) {
          const int i = i0 + tid;
          offer(i < n ? __ldg(text + i) : -1, i);
        }
        if (lane < held) count(q[lane]);
      }
      if (branches) {
        __syncthreads();
        if (tid == 0) listed[1] = *listed;   // ids that are listed for all of them
        __syncwarp();                        // (the tokens are brought by this warp)
      }
      if (p.tokens && !p.anc && tid < j0) token(__ldg(p.tokens + s * p.q + tid), false);   // (a chain: row j comes after tokens 0 .. j)
    }
    if (p.tokens && tid < p.q && (mine >> tid & 1u)) token(__ldg(p.tokens + s * p.q + tid), false);
    pass_on(tid);
    for (int k0 = tid + ADJ_U * ADJ_THREADS; k0 - lane < nvec; k0 += ADJ_U * ADJ_THREADS) {
      ask(k0);
      pass_on(k0);
    }
    __syncthreads();   // the words, and the row but for the listed ids (in place, allowed logits are still what they were)
    const int n = *listed;
#pragma unroll 2
    for (int i = tid; i < n; i += ADJ_THREADS) {
      const int id = list[i];
      if (allowed && !(__ldg(allowed + (id >> 5)) >> (id & 31) & 1u)) continue;
      if (BF16) {
        const float l = __uint_as_float((uint32_t) * (reinterpret_cast<const uint16_t*>(in) + id) << 16);
        reinterpret_cast<__nv_bfloat16*>(out)[id] = __float2bfloat16_rn(adjust_one(l, words[id], a));
      } else {
        reinterpret_cast<float*>(out)[id] = adjust_one(reinterpret_cast<const float*>(in)[id], words[id], a);
      }
    }
    if (j + 1 < j1) {
      __syncthreads();
      if (branches && tid < 32) {   // another branch follows: this one's tokens are taken back (all in the warp that brings them)
        if (tid < p.q && (mine >> tid & 1u)) {
          const int id = __ldg(p.tokens + s * p.q + tid);
          if (here(id)) atomicAdd(&words[id - v0], 0xFFFFFFFFu);
        }
        if (tid == 0) *listed = listed[1];
        __syncwarp();
      }
    }
  }
  if (largest >= p.V) set_error(p.err, ERR_TOKEN);
}

template <bool BF16>
static cudaError_t adj_prepare() {
  cudaError_t e = cudaFuncSetAttribute(adjust_kernel<BF16, 256>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)adj_smem(ADJ_STRETCH));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(adjust_kernel<BF16, 512>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)adj_smem(ADJ_STRETCH));
  if (e == cudaSuccess) e = prefer_shared(adjust_kernel<BF16, 256>);
  return e == cudaSuccess ? prefer_shared(adjust_kernel<BF16, 512>) : e;
}
cudaError_t adjust_prepare() {
  const cudaError_t e = adj_prepare<false>();
  return e == cudaSuccess ? adj_prepare<true>() : e;
}

cudaError_t launch_adjust(const AdjustParams& p, int num_sms, cudaStream_t st, bool pdl) {
  // Threads of a CTA, ids of its stretch and whether it takes one row or all of a sequence: whichever a model of a CTA's time
  // makes least (us: its start, a row's waits, the ids and the history by thread; what does not fit in a round takes its
  // share and a tail).  Long histories go to wide CTAs that read them less often, many rows of a sequence to one CTA once
  // others fill the SMs.  Against the longest stretches that leave no SM empty (us): 3 rows of 5010 after 8665 tokens 6.6
  // for 11.3, 13 x 16 rows of 20414 7.8 for 9.5, 197 rows of 16646 4.4 for 7.0, 48 rows of 32016 7.3 for 7.3; 256 of 128003
  // take 72 in stretches of 16000 on 512 threads, 83 in 8064 on 256.
  int ch = 0, rp = 1, threads = 0;
  double least = 1e30;
  for (int n = 256; n <= 512; n *= 2)
    for (int r = 1;; r = p.q) {
      const int most = 2 * n * ADJ_U * (p.bf16 ? 8 : 4) - 128;   // (with the vector more that a misaligned row has, whole turns)
      for (int chunks = (p.V + most - 1) / most;; chunks *= 2) {
        const int c = std::min(most, (p.V + chunks * 128 - 1) / (chunks * 128) * 128);
        const double ctas = (double)p.b * ((p.q + r - 1) / r) * ((p.V + c - 1) / c), rounds = ctas * n / (1024. * num_sms);
        const double one = 1.2 + r * (1.3 + c * (p.bf16 ? 0.128 : 0.2) / n) + (p.history ? 0.28 * p.history_ld / n : 0.);
        const double cost = one * (rounds > 1. ? rounds + 0.5 : 1.);
        if (cost < least) least = cost, ch = c, rp = r, threads = n;
        if (c <= 512) break;
      }
      if (r == p.q) break;
    }
  const int parts = (p.q + rp - 1) / rp, chunks = (p.V + ch - 1) / ch;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.b * parts * chunks));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = adj_smem(ch);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  if (threads == 512)
    return p.bf16 ? cudaLaunchKernelEx(&cfg, adjust_kernel<true, 512>, p, rp, ch, parts, chunks)
                  : cudaLaunchKernelEx(&cfg, adjust_kernel<false, 512>, p, rp, ch, parts, chunks);
  return p.bf16 ? cudaLaunchKernelEx(&cfg, adjust_kernel<true, 256>, p, rp, ch, parts, chunks)
                : cudaLaunchKernelEx(&cfg, adjust_kernel<false, 256>, p, rp, ch, parts, chunks);
}

}  // namespace sdsat
