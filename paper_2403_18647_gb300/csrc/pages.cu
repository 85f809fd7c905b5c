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
// kernels list what to copy, a source page with all of its destinations, and a second kernel on every SM
// copies: a source is read once.
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

// a table entry as a page of the pool, or -1 for none (the table can be written from outside: a number that is
// neither is reported and counts as none)
__device__ __forceinline__ int pool_page(const PagesParams& p, int entry) {
  if (entry >= -1 && entry < p.n_pages) return entry;
  set_error(p.err, ERR_PAGE);
  return -1;
}

// common[s] = leading pages that sequence s holds together with sequence 0 (a warp per sequence, the
// loads of 128 columns in flight)
__device__ void common_pages(const PagesParams& p) {
  constexpr int N = 4;
  const int lane = threadIdx.x & 31;
  for (int s = threadIdx.x >> 5; s < p.batch; s += PG_WARPS) {
    int n = p.ld;
    for (int j0 = 0; j0 < p.ld && n == p.ld; j0 += 32 * N) {
      int a[N], z[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int j = j0 + 32 * i + lane;
        a[i] = j < p.ld ? __ldcg(p.table + j) : -1;
        z[i] = j < p.ld ? __ldcg(p.table + (size_t)s * p.ld + j) : -1;
      }
#pragma unroll
      for (int i = N - 1; i >= 0; --i) {   // (the first one that differs is what stays)
        const unsigned differ = __ballot_sync(0xffffffffu, a[i] < 0 || a[i] != z[i]);
        if (differ) n = min(p.ld, j0 + 32 * i + __ffs(differ) - 1);
      }
    }
    if (lane == 0) p.common[s] = n;
  }
}

// ---- fork and free -------------------------------------------------------------------------
// A round of columns: every sequence's entries are read before any of them is written, so the
// table can be permuted in place.
__global__ void __launch_bounds__(PG_THREADS) pages_fork_kernel(const __grid_constant__ PagesParams p) {
  __shared__ int src_s[PAGES_MAX_BATCH], len_all[PAGES_MAX_BATCH];
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, nb = p.src ? p.nb : 1;
  for (int s = tid; s < p.batch; s += PG_THREADS) len_all[s] = __ldcg(p.len + s);
  for (int s = tid; s < nb; s += PG_THREADS) {
    int a = p.src ? __ldcg(p.src + s) : -1;
    if (a < -1 || a >= p.batch) {   // there is no such sequence: s stays as it is
      set_error(p.err, ERR_PAGE);
      a = p.seq0 + s;
    }
    src_s[s] = a;
  }
  __syncthreads();
  for (int s = tid; s < nb; s += PG_THREADS) p.len[p.seq0 + s] = src_s[s] < 0 ? 0 : len_all[src_s[s]];
  const int cols = PG_THREADS / nb;   // (nb <= PAGES_MAX_BATCH: a thread has one entry a round)
  for (int c0 = 0; c0 < p.ld; c0 += cols) {
    const int s = tid / cols, j = c0 + tid % cols;
    const bool mine = s < nb && j < p.ld;
    int there = -1, now = -1;
    int* entry = nullptr;
    if (mine) {
      entry = p.table + (size_t)(p.seq0 + s) * p.ld + j;
      there = __ldcg(entry);
      const int a = src_s[s];
      now = a < 0 ? -1 : pool_page(p, __ldcg(p.table + (size_t)a * p.ld + j));
    }
    __syncthreads();
    if (mine && there != now) {
      const int was = pool_page(p, there);
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
  __shared__ int first_s[PAGES_MAX_BATCH], end_s[PAGES_MAX_BATCH], at_s[PAGES_MAX_BATCH], part_s[PAGES_MAX_BATCH];
  __shared__ int sums[PG_WARPS], s_copies, s_runs, s_ids[PG_THREADS];
  __shared__ int old_s[PAGES_MAX_BATCH], new_s[PAGES_MAX_BATCH], rows_s[PAGES_MAX_BATCH];   // a sequence's copy
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int refs_mine = tid < p.n_pages ? __ldcg(p.refs + tid) : 1;   // (needed later; on its way now)
  for (int s = tid; s < p.nb; s += PG_THREADS) {
    const int was = __ldcg(p.len + p.seq0 + s), len = min(max(was, 0), p.cap);
    long long end = (long long)len + p.n;
    if (end > p.cap || len != was) {   // the slots past the capacity get no page
      set_error(p.err, ERR_CAPACITY);
      end = min(end, (long long)p.cap);
    }
    first_s[s] = len / KV_PAGE;
    part_s[s] = len % KV_PAGE;
    end_s[s] = max(len / KV_PAGE, (int)((end + KV_PAGE - 1) / KV_PAGE));
  }
  if (tid == 0) s_copies = s_runs = 0;
  for (int s = tid; s < p.nb; s += PG_THREADS) rows_s[s] = 0;
  __syncthreads();
  // what each wanted page needs; of a warp's first 32 it is kept, with the page that is there
  int kind0 = KEEP, page0 = -1;
  for (int s = warp; s < p.nb; s += PG_WARPS) {
    int need = 0;
    for (int j0 = first_s[s]; j0 < end_s[s]; j0 += 32) {
      const int j = j0 + lane;
      int kind = KEEP, page = -1;
      if (j < end_s[s]) {
        page = pool_page(p, __ldcg(p.table + (size_t)(p.seq0 + s) * p.ld + j));
        if (page < 0) {
          kind = FRESH;
        } else {
          int others = __ldcg(p.refs + page) - 1;
          if (others > 0) {
            // earlier sequences of this call give their hold on it up (eight loads in flight)
#pragma unroll 8
            for (int t = 0; t < s; ++t)
              if (j >= first_s[t] && j < end_s[t] && __ldcg(p.table + (size_t)(p.seq0 + t) * p.ld + j) == page) --others;
          }
          if (others > 0) kind = COPY;
        }
        p.kinds[(size_t)s * p.ld + j] = kind;
      }
      if (s == warp && j0 == first_s[s]) {
        kind0 = kind;
        page0 = page;
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
    const bool idle = page < p.n_pages && (c0 == 0 ? refs_mine : __ldcg(p.refs + page)) == 0;
    int got;
    const int at = found + block_scan(idle, sums, &got);
    if (idle && at < need) {
      if (at < PG_THREADS) s_ids[at] = page;
      else p.ids[at] = page;
    }
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
    for (int j0 = first_s[s]; j0 < end_s[s]; j0 += 32) {
      const int j = j0 + lane;
      const bool kept = s == warp && j0 == first_s[s];
      const int kind = kept ? kind0 : j < end_s[s] ? p.kinds[(size_t)s * p.ld + j] : KEEP;
      const unsigned who = __ballot_sync(0xffffffffu, kind != KEEP);
      if (kind != KEEP) {
        int* entry = p.table + (size_t)(p.seq0 + s) * p.ld + j;
        const int i = at + __popc(who & ((1u << lane) - 1u)), page = i < PG_THREADS ? s_ids[i] : __ldcg(p.ids + i);
        if (kind == COPY) {
          const int old = kept ? page0 : __ldcg(entry), rows = j == first_s[s] ? part_s[s] : 0;   // committed ones
          atomicSub(p.refs + old, 1);
          if (rows > 0) {
            old_s[s] = old;
            new_s[s] = page;
            rows_s[s] = rows;
          }
        }
        __stcg(entry, page);
        __stcg(p.refs + page, 1);
      }
      at += __popc(who);
    }
  }
  __syncthreads();
  // the copies of one source side by side: a run for each first one of them
  if (tid < p.nb && rows_s[tid] > 0) {
    int same = 0, earlier = 0;
    for (int t = 0; t < p.nb; ++t)
      if (rows_s[t] == rows_s[tid] && old_s[t] == old_s[tid]) {
        ++same;
        earlier += t < tid;
      }
    if (earlier == 0) {
      int at = atomicAdd(&s_copies, same);
      int* run = p.copies + 4 + 4 * atomicAdd(&s_runs, 1);
      run[0] = old_s[tid];
      run[1] = rows_s[tid];
      run[2] = at;
      run[3] = same;
      for (int t = tid; t < p.nb; ++t)
        if (rows_s[t] == rows_s[tid] && old_s[t] == old_s[tid]) p.copies[4 + 4 * p.n_pages + at++] = new_s[t];
    }
  }
  __syncthreads();
  if (tid == 0) p.copies[0] = s_runs;
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
    const int page = pool_page(p, __ldcg(p.table + i));
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
        int* run = p.copies + 4 + 4 * c;
        run[0] = page;
        run[1] = rows;
        run[2] = c;
        run[3] = 1;
        p.copies[4 + 4 * p.n_pages + c] = to;
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
    if (page >= used && page < p.n_pages) __stcg(p.table + i, __ldcg(p.kinds + page));
  }
  if (tid == 0) p.copies[0] = copies;
}

// ---- copying -------------------------------------------------------------------------------------
// Blocks of the committed slots of one (page, layer, head) of K or of V, at most KV_PAGE hd 2 = 16 KB in
// one piece, go through a ring in shared memory by bulk copies: one in, one out for each destination.
// One thread on an SM drives them, loads PC_AHEAD blocks ahead; the warp's lanes have the next 32
// blocks' places.  A branch of a 7B-shaped cache into eight, 288 MB to move at the least: 61 us
// in all, 103 with warps that copied through registers, 32 on an SM; a round of ten samples on a
// 13B-shaped one, 693 MB: 112 and 208 replayed as a graph (calls in a row take 114 to 146).
constexpr int PC_SLOTS = 12, PC_AHEAD = 6;
__device__ __forceinline__ void bulk_store_s2g(void* dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_u32(src)), "r"(bytes) : "memory");
}
__global__ void __launch_bounds__(32) pages_copy_kernel(const __grid_constant__ PagesParams p) {
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ uint64_t full[PC_SLOTS];
  __shared__ volatile int abort;
  const int lane = threadIdx.x;
  if (lane == 0) {
    for (int i = 0; i < PC_SLOTS; ++i) mbar_init(&full[i], 1);
    abort = 0;
    fence_mbar_init();
  }
  __syncwarp();
  pdl_wait();
  pdl_trigger();
  const int runs = __ldcg(p.copies);
  const long long total = 2ll * p.L * p.H * runs;
  const int mine = (int)((total - blockIdx.x + gridDim.x - 1) / gridDim.x);   // blocks of this CTA
  const long long page = (long long)KV_PAGE * p.hd;   // elements of one page and head
  const int* to = p.copies + 4 + 4 * p.n_pages;
  __nv_bfloat16* my_base = nullptr;   // of block (this group of 32) + lane: page 0 of its layer and head
  int4 my_run = make_int4(0, 0, 0, 0);
  int my_to = 0;
  // block i: its base, run and first destination, from the lane that has them
  auto places = [&](int group) {
    const long long u = blockIdx.x + (long long)(32 * group + lane) * gridDim.x;
    if (u < total) {
      const long long b = u / runs;
      const int h = (int)(b % p.H), l = (int)(b / p.H) >> 1;
      my_base = (((b / p.H) & 1) ? p.v : p.k) + ((long long)l * p.n_pages * p.H + h) * page;
      my_run = __ldcg(reinterpret_cast<const int4*>(p.copies + 4) + u % runs);
      my_to = __ldcg(to + my_run.z);
    }
  };
  auto at = [&](const __nv_bfloat16* base, int id) { return const_cast<__nv_bfloat16*>(base) + (long long)id * p.H * page; };
  int loaded = 0, done = 0;
  // loads and stores of a group of 32 blocks: the loads run ahead inside of it
  for (int g = 0; 32 * g < mine; ++g) {
    places(g);
    const int end = min(mine, 32 * g + 32);
    for (; done < end && !abort; ++done) {
      for (; loaded < min(end, done + PC_AHEAD); ++loaded) {
        const int from = loaded & 31;
        const __nv_bfloat16* base = reinterpret_cast<const __nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(my_base), from));
        const int src = __shfl_sync(0xffffffffu, my_run.x, from), rows = __shfl_sync(0xffffffffu, my_run.y, from);
        if (lane == 0) {
          const int slot = loaded % PC_SLOTS;
          // what was stored from the slot has been read: at most PC_SLOTS - PC_AHEAD blocks since
          asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PC_SLOTS - PC_AHEAD) : "memory");
          const uint32_t bytes = rows * p.hd * 2;
          mbar_arrive_expect_tx(&full[slot], bytes);
          bulk_load_g2s(ring + (size_t)slot * page * 2, at(base, src), bytes, &full[slot]);
        }
      }
      const int from = done & 31;
      const __nv_bfloat16* base = reinterpret_cast<const __nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(my_base), from));
      const int rows = __shfl_sync(0xffffffffu, my_run.y, from), first = __shfl_sync(0xffffffffu, my_run.z, from),
                n = __shfl_sync(0xffffffffu, my_run.w, from), dst = __shfl_sync(0xffffffffu, my_to, from);
      if (lane == 0) {
        const int slot = done % PC_SLOTS;
        if (mbar_wait_bounded(&full[slot], (done / PC_SLOTS) & 1, &abort, p.err)) {
          for (int i = 0; i < n; ++i)
            bulk_store_s2g(at(base, i == 0 ? dst : __ldcg(to + first + i)), ring + (size_t)slot * page * 2, rows * p.hd * 2);
        }
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
      }
      __syncwarp();
    }
  }
  if (lane == 0) {
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    if (abort) {   // let the copies in flight land before the CTA exits
      for (done = max(0, done - 1); done < loaded; ++done) {
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait(&full[done % PC_SLOTS], (done / PC_SLOTS) & 1))
          if (globaltimer_ns() - t0 > WAIT_LIMIT_NS) break;
      }
    }
  }
}

// ---- rows in and out -----------------------------------------------------------------------------
// src / dst [H][n][hd] <-> slots slot0 .. of one (layer, sequence); one piece a thread, of 16 bytes where the
// buffers allow it, or of one value
template <typename T>
__global__ void __launch_bounds__(256) pages_rows_kernel(const __grid_constant__ PagesParams p, int layer, int slot0,
                                                         T* kx, T* vx, int write) {
  pdl_wait();
  pdl_trigger();
  const int chunks = p.hd * 2 / (int)sizeof(T);
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, total = 2ll * p.H * p.n * chunks;
  if (i >= total) return;
  const int c = (int)(i % chunks);
  const long long r = i / chunks;
  const int x = (int)(r % p.n), slot = slot0 + x;
  const int h = (int)(r / p.n % p.H);
  const bool v = r / p.n >= p.H;
  const int page = __ldcg(p.table + (size_t)p.seq0 * p.ld + slot / KV_PAGE);
  T* buf = (v ? vx : kx) + ((long long)h * p.n + x) * chunks + c;
  // no page, or (to write) one that others hold too
  const bool ok = page >= 0 && page < p.n_pages && (!write || __ldcg(p.refs + page) == 1);
  if (!ok) {
    if (c == 0 && h == 0 && !v) set_error(p.err, ERR_CAPACITY);
    if (!write) *buf = T{};
    return;
  }
  T* row = reinterpret_cast<T*>((v ? p.v : p.k) + ((((long long)layer * p.n_pages + page) * p.H + h) * KV_PAGE + slot % KV_PAGE) * p.hd) + c;
  if (write) *row = __ldcg(buf);
  else *buf = __ldcg(row);
}

template <typename... A>
cudaError_t launch_pages(void (*kernel)(A...), dim3 grid, int threads, size_t smem, cudaStream_t st, bool pdl,
                         std::common_type_t<A>... args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
size_t pages_copy_smem(int hd) { return (size_t)PC_SLOTS * KV_PAGE * hd * 2; }
}  // namespace

cudaError_t pages_prepare() {
  cudaError_t e = prefer_shared(pages_fork_kernel);
  if (e == cudaSuccess) e = prefer_shared(pages_reserve_kernel);
  if (e == cudaSuccess) e = prefer_shared(pages_compact_kernel);
  if (e == cudaSuccess) e = prefer_shared(pages_copy_kernel);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(pages_copy_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)pages_copy_smem(128));
  if (e == cudaSuccess) e = prefer_shared(pages_rows_kernel<uint4>);
  if (e == cudaSuccess) e = prefer_shared(pages_rows_kernel<unsigned short>);
  return e;
}

cudaError_t launch_pages_fork(const PagesParams& p, cudaStream_t st, bool pdl) {
  return launch_pages(pages_fork_kernel, dim3(1), PG_THREADS, 0, st, pdl, p);
}
cudaError_t launch_pages_reserve(const PagesParams& p, cudaStream_t st, bool pdl) {
  return launch_pages(pages_reserve_kernel, dim3(1), PG_THREADS, 0, st, pdl, p);
}
cudaError_t launch_pages_compact(const PagesParams& p, cudaStream_t st, bool pdl) {
  return launch_pages(pages_compact_kernel, dim3(1), PG_THREADS, 0, st, pdl, p);
}
cudaError_t launch_pages_copy(const PagesParams& p, int num_sms, cudaStream_t st, bool pdl) {
  return launch_pages(pages_copy_kernel, dim3(num_sms), 32, pages_copy_smem(p.hd), st, pdl, p);
}
cudaError_t launch_pages_rows(const PagesParams& p, int layer, int slot0, void* k, void* v, bool write, cudaStream_t st,
                              bool pdl) {
  const bool whole = ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15) == 0;
  const long long pieces = 2ll * p.H * p.n * (p.hd / (whole ? 8 : 1));
  const dim3 grid((unsigned)((pieces + 255) / 256));
  return whole ? launch_pages(pages_rows_kernel<uint4>, grid, 256, 0, st, pdl, p, layer, slot0, static_cast<uint4*>(k),
                              static_cast<uint4*>(v), write ? 1 : 0)
               : launch_pages(pages_rows_kernel<unsigned short>, grid, 256, 0, st, pdl, p, layer, slot0,
                              static_cast<unsigned short*>(k), static_cast<unsigned short*>(v), write ? 1 : 0);
}

}  // namespace sdsat
