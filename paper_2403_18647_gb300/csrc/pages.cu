// The paged KV cache: a pool of pages of KV_PAGE slots (every layer and head of them), one row of
// page ids per sequence, and a count of the sequences that hold each page.
//
//   fork      sequence s takes the pages and the length of sequence src[s]: ids and counts only
//   reserve   pages of its own for the slots that a sequence's next rows go to: the lowest free ids,
//             sequences in order; a page that others hold too is replaced by a copy of its committed
//             slots (copy on write), its last holder keeps it
//   compact   the pages in use move to the front of the pool: the i-th one past the front's end to
//             the i-th free one inside it
//
// The tables are small (one CTA works on them, a few microseconds of dependent steps); what costs
// is the copying, a page being 2 L H KV_PAGE hd values (33.5 MB of a 7B-shaped cache).  So the table
// kernels write a list of (source, destination, slots) and a second kernel on every SM copies.
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace sdsat {
namespace {

constexpr int PG_THREADS = 1024;
constexpr int PG_WARPS = PG_THREADS / 32;

// exclusive prefix sum over the CTA (every thread calls it); total in *sum
__device__ int block_scan(int v, int* warp_sums, int* sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();   // (the sums of the call before have been read)
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int w = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += y;
    }
    warp_sums[lane] = w;
  }
  __syncthreads();
  *sum = warp_sums[PG_WARPS - 1];
  return x - v + (warp ? warp_sums[warp - 1] : 0);
}
static_assert(PG_WARPS == 32, "one warp adds the warps up");

// common[s] = leading pages that sequence s holds together with sequence 0 (a warp per sequence)
__device__ void common_pages(const PagesParams& p) {
  const int lane = threadIdx.x & 31;
  for (int s = threadIdx.x >> 5; s < p.batch; s += PG_WARPS) {
    int n = p.ld;
    for (int j0 = 0; j0 < p.ld; j0 += 32) {
      const int j = j0 + lane;
      bool same = false;
      if (j < p.ld) {
        const int a = __ldcg(p.table + j);
        same = a >= 0 && a == __ldcg(p.table + (size_t)s * p.ld + j);
      }
      const unsigned differ = __ballot_sync(0xffffffffu, !same);
      if (differ) {
        n = min(p.ld, j0 + __ffs(differ) - 1);
        break;
      }
    }
    if (lane == 0) p.common[s] = n;
  }
}

// ---- fork and free -------------------------------------------------------------------------
// A round of columns: every sequence's entries are read before any of them is written, so the
// table can be permuted in place.
__global__ void __launch_bounds__(PG_THREADS) pages_fork_kernel(const __grid_constant__ PagesParams p) {
  __shared__ int src_s[PAGES_MAX_BATCH];
  __shared__ int len_s[PAGES_MAX_BATCH];
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, nb = p.src ? p.nb : 1;
  for (int s = tid; s < nb; s += PG_THREADS) {
    int a = p.src ? __ldcg(p.src + s) : -1;
    if (a >= p.batch) {   // there is no such sequence: s stays as it is
      set_error(p.err, ERR_PAGE);
      a = p.seq0 + s;
    }
    src_s[s] = a;
    len_s[s] = a < 0 ? 0 : __ldcg(p.len + a);
  }
  __syncthreads();
  for (int s = tid; s < nb; s += PG_THREADS) p.len[p.seq0 + s] = len_s[s];
  const int cols = PG_THREADS / nb;   // (nb <= PAGES_MAX_BATCH: a thread has one entry a round)
  for (int c0 = 0; c0 < p.ld; c0 += cols) {
    const int s = tid / cols, j = c0 + tid % cols;
    const bool mine = s < nb && j < p.ld;
    int was = -1, now = -1;
    int* entry = nullptr;
    if (mine) {
      entry = p.table + (size_t)(p.seq0 + s) * p.ld + j;
      was = __ldcg(entry);
      const int a = src_s[s];
      now = a < 0 ? -1 : __ldcg(p.table + (size_t)a * p.ld + j);
    }
    __syncthreads();
    if (mine && was != now) {
      __stcg(entry, now);
      if (was >= 0) atomicSub(p.refs + was, 1);
      if (now >= 0) atomicAdd(p.refs + now, 1);
    }
  }
  __syncthreads();
  common_pages(p);
}

// ---- reserve -----------------------------------------------------------------------------------
enum : int { KEEP = 0, FRESH = 1, COPY = 2 };

__global__ void __launch_bounds__(PG_THREADS) pages_reserve_kernel(const __grid_constant__ PagesParams p) {
  __shared__ int first_s[PAGES_MAX_BATCH], end_s[PAGES_MAX_BATCH], at_s[PAGES_MAX_BATCH];
  __shared__ int sums[PG_WARPS], s_copies;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int s = tid; s < p.nb; s += PG_THREADS) {
    const int len = __ldcg(p.len + p.seq0 + s);
    long long end = (long long)len + p.n;
    if (end > p.cap) {   // the slots past the capacity get no page
      set_error(p.err, ERR_CAPACITY);
      end = p.cap;
    }
    first_s[s] = len / KV_PAGE;
    end_s[s] = max(len / KV_PAGE, (int)((end + KV_PAGE - 1) / KV_PAGE));
  }
  if (tid == 0) s_copies = 0;
  __syncthreads();
  // what each wanted page needs
  for (int s = warp; s < p.nb; s += PG_WARPS) {
    int need = 0;
    for (int j0 = first_s[s]; j0 < end_s[s]; j0 += 32) {
      const int j = j0 + lane;
      int kind = KEEP;
      if (j < end_s[s]) {
        const int page = __ldcg(p.table + (size_t)(p.seq0 + s) * p.ld + j);
        if (page < 0) {
          kind = FRESH;
        } else {
          int others = __ldcg(p.refs + page) - 1;
          // earlier sequences of this call give their hold on it up
          for (int t = 0; t < s && others > 0; ++t)
            if (j >= first_s[t] && j < end_s[t] && __ldcg(p.table + (size_t)(p.seq0 + t) * p.ld + j) == page) --others;
          if (others > 0) kind = COPY;
        }
        p.kinds[(size_t)s * p.ld + j] = kind;
      }
      need += __popc(__ballot_sync(0xffffffffu, kind != KEEP));
    }
    if (lane == 0) at_s[s] = need;
  }
  __syncthreads();
  int need = 0;
  {
    const int mine = tid < p.nb ? at_s[tid] : 0;
    const int before = block_scan(mine, sums, &need);
    if (tid < p.nb) at_s[tid] = before;
  }
  // the lowest free pages
  int found = 0;
  for (int c0 = 0; c0 < p.n_pages && found < need; c0 += PG_THREADS) {
    const int page = c0 + tid;
    const bool idle = page < p.n_pages && __ldcg(p.refs + page) == 0;
    int got;
    const int at = found + block_scan(idle, sums, &got);
    if (idle && at < need) p.ids[at] = page;
    found += got;
  }
  __syncthreads();
  if (found < need) {   // not enough of them: nothing changes
    if (tid == 0) {
      set_error(p.err, ERR_CAPACITY);
      p.copies[0] = 0;
    }
    return;
  }
  for (int s = warp; s < p.nb; s += PG_WARPS) {
    int at = at_s[s];
    const int len = __ldcg(p.len + p.seq0 + s);
    for (int j0 = first_s[s]; j0 < end_s[s]; j0 += 32) {
      const int j = j0 + lane;
      const int kind = j < end_s[s] ? p.kinds[(size_t)s * p.ld + j] : KEEP;
      const unsigned who = __ballot_sync(0xffffffffu, kind != KEEP);
      if (kind != KEEP) {
        int* entry = p.table + (size_t)(p.seq0 + s) * p.ld + j;
        const int page = __ldcg(p.ids + at + __popc(who & ((1u << lane) - 1u)));
        if (kind == COPY) {
          const int old = __ldcg(entry), rows = min(KV_PAGE, len - j * KV_PAGE);
          atomicSub(p.refs + old, 1);
          if (rows > 0) {
            int* c = p.copies + 4 + 3 * atomicAdd(&s_copies, 1);
            c[0] = old;
            c[1] = page;
            c[2] = rows;
          }
        }
        __stcg(entry, page);
        __stcg(p.refs + page, 1);
      }
      at += __popc(who);
    }
  }
  __syncthreads();
  if (tid == 0) p.copies[0] = s_copies;
  common_pages(p);
}

// ---- compact -----------------------------------------------------------------------------------
__global__ void __launch_bounds__(PG_THREADS) pages_compact_kernel(const __grid_constant__ PagesParams p) {
  __shared__ int sums[PG_WARPS];
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  int used = 0;
  for (int c0 = 0; c0 < p.n_pages; c0 += PG_THREADS) {
    const int page = c0 + tid;
    int got;
    block_scan(page < p.n_pages && __ldcg(p.refs + page) > 0, sums, &got);
    used += got;
    if (page < p.n_pages) {
      p.kinds[page] = 0;   // slots of the page that some sequence has committed
    }
  }
  // free pages inside the front, ascending
  int holes = 0;
  for (int c0 = 0; c0 < used; c0 += PG_THREADS) {
    const int page = c0 + tid;
    const bool hole = page < used && __ldcg(p.refs + page) == 0;
    int got;
    const int at = holes + block_scan(hole, sums, &got);
    if (hole) p.ids[at] = page;
    holes += got;
  }
  __syncthreads();
  if (p.used && tid == 0) *p.used = used;
  // the committed slots of the pages past the front
  const long long entries = (long long)p.batch * p.ld;
  for (long long i = tid; i < entries && holes; i += PG_THREADS) {
    const int page = __ldcg(p.table + i);
    if (page >= used) {
      const int s = (int)(i / p.ld), rows = min(KV_PAGE, __ldcg(p.len + s) - (int)(i - (long long)s * p.ld) * KV_PAGE);
      if (rows > 0) atomicMax(p.kinds + page, rows);
    }
  }
  __syncthreads();
  // the i-th used page past the front goes to the i-th hole
  int moved = 0, copies = 0;
  for (int c0 = used; c0 < p.n_pages && moved < holes; c0 += PG_THREADS) {
    const int page = c0 + tid;
    const int held = page < p.n_pages ? __ldcg(p.refs + page) : 0;
    const int rows = held > 0 ? __ldcg(p.kinds + page) : 0;
    int got, listed;
    const int at = moved + block_scan(held > 0, sums, &got);
    const int c = copies + block_scan(rows > 0, sums, &listed);
    if (held > 0) {
      const int to = __ldcg(p.ids + at);
      if (rows > 0) {
        int* e = p.copies + 4 + 3 * c;
        e[0] = page;
        e[1] = to;
        e[2] = rows;
      }
      __stcg(p.refs + to, held);
      __stcg(p.refs + page, 0);
      __stcg(p.kinds + page, to);
    }
    moved += got;
    copies += listed;
  }
  __syncthreads();
  for (long long i = tid; i < entries && holes; i += PG_THREADS) {
    const int page = __ldcg(p.table + i);
    if (page >= used) __stcg(p.table + i, __ldcg(p.kinds + page));
  }
  if (tid == 0) p.copies[0] = copies;
}

// ---- copying -------------------------------------------------------------------------------------
// A warp copies the listed slots of one (page, layer, head) of K or of V: hd * 2 bytes a slot, in one
// piece.
__global__ void __launch_bounds__(256) pages_copy_kernel(const __grid_constant__ PagesParams p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int count = __ldcg(p.copies);
  const long long blocks = 2ll * p.L * p.H, total = blocks * count;
  const long long step = (long long)gridDim.x * 8;
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < total; w += step) {
    const int e = (int)(w % count);
    const long long b = w / count;
    const int h = (int)(b % p.H), l = (int)(b / p.H) >> 1;
    const bool v = (b / p.H) & 1;
    const int src = __ldcg(p.copies + 4 + 3 * e), dst = __ldcg(p.copies + 5 + 3 * e), rows = __ldcg(p.copies + 6 + 3 * e);
    const long long page = (long long)KV_PAGE * p.hd;   // elements of one page and head
    __nv_bfloat16* base = (v ? p.v : p.k) + ((long long)l * p.n_pages * p.H + h) * page;
    const uint4* a = reinterpret_cast<const uint4*>(base + (long long)src * p.H * page);
    uint4* z = reinterpret_cast<uint4*>(base + (long long)dst * p.H * page);
    const int n = rows * p.hd / 8;
    for (int i = lane; i < n; i += 32) __stcg(z + i, __ldcg(a + i));
  }
}

// ---- rows in and out -----------------------------------------------------------------------------
// src / dst [H][n][hd] <-> slots slot0 .. of one (layer, sequence); one 16-byte piece a thread
__global__ void __launch_bounds__(256) pages_rows_kernel(const __grid_constant__ PagesParams p, int layer, int slot0,
                                                         uint4* kx, uint4* vx, int write) {
  pdl_wait();
  pdl_trigger();
  const int chunks = p.hd / 8;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, total = 2ll * p.H * p.n * chunks;
  if (i >= total) return;
  const int c = (int)(i % chunks);
  const long long r = i / chunks;
  const int x = (int)(r % p.n), slot = slot0 + x;
  const int h = (int)(r / p.n % p.H);
  const bool v = r / p.n >= p.H;
  const int page = __ldcg(p.table + (size_t)p.seq0 * p.ld + slot / KV_PAGE);
  uint4* buf = (v ? vx : kx) + ((long long)h * p.n + x) * chunks + c;
  // no page, or (to write) one that others hold too
  const bool ok = page >= 0 && page < p.n_pages && (!write || __ldcg(p.refs + page) == 1);
  if (!ok) {
    if (c == 0 && h == 0 && !v) set_error(p.err, ERR_CAPACITY);
    if (!write) *buf = make_uint4(0u, 0u, 0u, 0u);
    return;
  }
  uint4* row = reinterpret_cast<uint4*>((v ? p.v : p.k) + ((((long long)layer * p.n_pages + page) * p.H + h) * KV_PAGE + slot % KV_PAGE) * p.hd) + c;
  if (write) *row = __ldcg(buf);
  else *buf = __ldcg(row);
}

template <typename... A>
cudaError_t launch_pages(void (*kernel)(A...), dim3 grid, int threads, cudaStream_t st, bool pdl,
                         std::common_type_t<A>... args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
}  // namespace

cudaError_t pages_prepare() {
  cudaError_t e = prefer_shared(pages_fork_kernel);
  if (e == cudaSuccess) e = prefer_shared(pages_reserve_kernel);
  if (e == cudaSuccess) e = prefer_shared(pages_compact_kernel);
  if (e == cudaSuccess) e = prefer_shared(pages_copy_kernel);
  if (e == cudaSuccess) e = prefer_shared(pages_rows_kernel);
  return e;
}

cudaError_t launch_pages_fork(const PagesParams& p, cudaStream_t st, bool pdl) {
  return launch_pages(pages_fork_kernel, dim3(1), PG_THREADS, st, pdl, p);
}
cudaError_t launch_pages_reserve(const PagesParams& p, cudaStream_t st, bool pdl) {
  return launch_pages(pages_reserve_kernel, dim3(1), PG_THREADS, st, pdl, p);
}
cudaError_t launch_pages_compact(const PagesParams& p, cudaStream_t st, bool pdl) {
  return launch_pages(pages_compact_kernel, dim3(1), PG_THREADS, st, pdl, p);
}
cudaError_t launch_pages_copy(const PagesParams& p, int num_sms, cudaStream_t st, bool pdl) {
  return launch_pages(pages_copy_kernel, dim3(4 * num_sms), 256, st, pdl, p);
}
cudaError_t launch_pages_rows(const PagesParams& p, int layer, int slot0, void* k, void* v, bool write, cudaStream_t st,
                              bool pdl) {
  const long long pieces = 2ll * p.H * p.n * (p.hd / 8);
  return launch_pages(pages_rows_kernel, dim3((unsigned)((pieces + 255) / 256)), 256, st, pdl, p, layer, slot0,
                      static_cast<uint4*>(k), static_cast<uint4*>(v), write ? 1 : 0);
}

}  // namespace sdsat
