// Sequences that go on as others: page tables, counters, the free list, and copies of the pages that two of them would write.
//
// Three things depend on each other: how many pages every child takes (a prefix sum over the children), the counters (a page is free when the last
// holder lets go), and the free list (freed pages in ascending order).  fork_small_kernel: few sequences, table entries and pages, outputs in arrays of their own; every block
// works the children out for itself, the first one has the counters (in shared memory) and the list, the others tables and copies, and nobody
// waits for anybody (one prompt to 4 samples 7.5 us, two kernels 8.6).  Else two.  fork_plan_kernel: one block works the children out, while the
// others clear the marks of freed pages and, where the outputs are arrays of their own, copy the counters and the list.  fork_kernel: tables,
// counters and copies by all blocks; the block that is last with its tables and counters lists the freed pages, while the others copy on.
// Bound by HBM where pages are copied (each read once, written once): 64 beams of a 28-layer cache, 143 MB, 23.5 us; else by latency.
#include <algorithm>

#include "slot_row.cuh"

namespace pc {
namespace {

struct Child { int32_t parent, have, got, full; int64_t start; };      // `have` pages of the parent's, `got` of the list's from place `start` on
struct PlanHead { int32_t count, taken, done, pad; };
// The workspace's first 256 bytes belong to the calls that report in them.
constexpr size_t WS_HEAD = 256, WS_CHILD = 512, WS_COPY = WS_CHILD + sizeof(Child) * MAX_FORK_SEQS, WS_KIDS = WS_COPY + sizeof(int2) * MAX_FORK_SEQS,
                 WS_MARKS = WS_KIDS + sizeof(int32_t) * MAX_FORK_SEQS;
constexpr int64_t MAX_PAGES = INT64_C(1) << 26;
static_assert(WS_MARKS + MAX_PAGES / 8 <= (24u << 20), "PERCACHE_OPS_WORKSPACE_BYTES");

struct Plan {
  PlanHead* head;
  Child* child;
  int2* copy;                    // page to page
  int32_t* kids;                 // children of a sequence
  uint32_t* marks;               // a bit per page: freed by this call
};
__host__ __device__ inline Plan plan_of(void* ws) {
  char* w = static_cast<char*>(ws);
  return Plan{reinterpret_cast<PlanHead*>(w + WS_HEAD), reinterpret_cast<Child*>(w + WS_CHILD), reinterpret_cast<int2*>(w + WS_COPY),
              reinterpret_cast<int32_t*>(w + WS_KIDS), reinterpret_cast<uint32_t*>(w + WS_MARKS)};
}

struct Seq { int held, length; };
__device__ __forceinline__ Seq seq_of(const Fork& f, int s) {
  Seq q;
  q.held = min(max(ld_dep_s32(f.held + s), 0), f.width);
  q.length = min(max(ld_dep_s32(f.length + s), 0), q.held * PAGE_TOKENS);
  return q;
}

// Inclusive sum over the block's threads (up to 1024); `total`: of all.
__device__ __forceinline__ int64_t block_sum(int64_t x, int64_t* warp_sums, int64_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  int64_t all = 0;
#pragma unroll 1
  for (int w = 0; w < warps; ++w) {
    const int64_t y = warp_sums[w];
    if (w < warp) x += y;
    all += y;
  }
  __syncthreads();
  *total = all;
  return x;
}

// Pages of a word of marks into the list, from place `to` on.
__device__ __forceinline__ void return_freed(const Fork& f, uint32_t marks, int page0, int64_t to) {
  for (uint32_t x = marks; x; x &= x - 1, ++to)
    if (to < f.n_pages) f.free_list_out[to] = page0 + __ffs(x) - 1;
}
// What child i takes over (first: every sequence's first child), and how many pages it lacks.
struct Wants {
  Child c;
  int fresh, length;
  bool part;                     // a partly filled page to copy
};
__device__ __forceinline__ Wants wants_of(const Fork& f, int i, const int32_t* first) {
  Wants w{Child{-1, 0, 0, 0, 0}, 0, 0, false};
  if (i >= f.n_children) return w;
  const int p = ld_dep_s32(f.parent + i);
  if (p < 0 || p >= f.n_seqs) return w;
  const Seq q = seq_of(f, p);
  const bool heir = first[p] == i;
  w.c.parent = p;
  w.c.full = q.length / PAGE_TOKENS;
  w.c.have = min(heir ? q.held : w.c.full, f.width_out);
  w.length = q.length;
  w.part = !heir && q.length % PAGE_TOKENS != 0 && w.c.full < f.width_out;
  const int want = static_cast<int>(min((static_cast<int64_t>(q.length) + f.room + PAGE_TOKENS - 1) / PAGE_TOKENS, static_cast<int64_t>(f.width_out)));
  w.fresh = max(want - w.c.have, 0);
  return w;
}
// What the list has for it; start: how many pages the children before it lack.
__device__ __forceinline__ void give(Wants& w, int64_t start, int count) {
  w.c.start = start;
  w.c.got = static_cast<int>(min(max(static_cast<int64_t>(count) - start, static_cast<int64_t>(0)), static_cast<int64_t>(w.fresh)));
}
// Page to page, or -1.
__device__ __forceinline__ int2 copy_of(const Fork& f, const Wants& w, int count) {
  if (!w.part || w.c.got == 0) return make_int2(-1, -1);
  return make_int2(ld_dep_s32(f.table + static_cast<size_t>(w.c.parent) * f.width + w.c.full), ld_dep_s32(f.free_list + count - 1 - w.c.start));
}
__device__ __forceinline__ bool copies(const Fork& f, int2 c) { return c.x >= 0 && c.x < f.n_pages && c.y >= 0 && c.y < f.n_pages && c.x != c.y; }
__device__ __forceinline__ int length_of(const Wants& w) {
  return static_cast<int>(min(static_cast<int64_t>(w.length), static_cast<int64_t>(w.c.have + w.c.got) * PAGE_TOKENS));
}
__device__ __forceinline__ int count_of(const Fork& f) { return static_cast<int>(min(static_cast<int64_t>(max(ld_dep_s32(f.free_count), 0)), f.n_pages)); }
// Entry j of a child's row of table_out.
__device__ __forceinline__ int entry_of(const Fork& f, const Child& c, int count, int j) {
  if (j < c.have) return ld_dep_s32(f.table + static_cast<size_t>(c.parent) * f.width + j);
  return j < c.have + c.got ? ld_dep_s32(f.free_list + count - 1 - c.start - (j - c.have)) : -1;
}

constexpr int COPY_BYTES = 16384;                 // of a page that a block takes at a time
// Stretch `chunk` of a page (over pools, their layers and the page's stretches) by the block.
template <int THREADS>
__device__ __forceinline__ void copy_chunk(const Fork& f, int2 pair, int chunk) {
  int k = 0;
#pragma unroll 1
  for (;; ++k) {                                  // which pool
    const int per = static_cast<int>((f.pools[k].page_bytes + COPY_BYTES - 1) / COPY_BYTES) * f.pools[k].n_layers;
    if (chunk < per || k + 1 == f.n_pools) break;
    chunk -= per;
  }
  const Pool& pool = f.pools[k];
  const int pieces = static_cast<int>((pool.page_bytes + COPY_BYTES - 1) / COPY_BYTES);
  const int64_t off = static_cast<int64_t>(chunk % pieces) * COPY_BYTES, len = min(pool.page_bytes - off, static_cast<int64_t>(COPY_BYTES));
  char* base = pool.base + (chunk / pieces) * pool.layer_stride + off;
  const char* src = base + pair.x * pool.page_stride;
  char* dst = base + pair.y * pool.page_stride;
  const int tid = threadIdx.x;
  if (pool.vec == 16) {
    uint4 v[COPY_BYTES / 16 / THREADS];
#pragma unroll
    for (int e = 0; e < COPY_BYTES / 16 / THREADS; ++e) {
      const int at = (e * THREADS + tid) * 16;
      if (at < len) v[e] = ld_dep_v4(src + at);
    }
#pragma unroll
    for (int e = 0; e < COPY_BYTES / 16 / THREADS; ++e) {
      const int at = (e * THREADS + tid) * 16;
      if (at < len) *reinterpret_cast<uint4*>(dst + at) = v[e];
    }
  } else {
    for (int at = tid * 4; at < len; at += THREADS * 4) *reinterpret_cast<int*>(dst + at) = ld_dep_s32(src + at);
  }
}

// ---------------------------------------------------------------------------------------------------- one kernel
// Where it is the faster one: the first block walks all counters, the list, and the pages of sequences that end or go on as several, which grows with the
// pages and with the tables' entries; the two kernels' time hardly does.  Device us, one kernel / two, without copies (every sequence goes on, or a
// quarter of them does): 4096 pages, one prompt of 127 pages to 4 samples 7.5 / 8.6, to 500 10.3 / 12.0; 16 beams of 127 pages 7.9 / 11.0 or 8.6 / 12.4, 64
// beams of 127 10.4 / 11.6 or 12.4 / 14.7; past the limits 128 beams of 127 pages 12.9 / 12.2 or 17.1 / 15.6, 256 of 34 11.7 / 11.9 or 16.3 / 15.0, 500 of 65
// 18.4 / 14.2 or 31.9 / 18.3, and on 8192 pages the sample 9.5 / 8.6, 64 beams of 127 12.5 / 11.5 or 14.5 / 15.0.
constexpr int SMALL_SEQS = 128, SMALL_CHILDREN = 512, SMALL_PAGES = 4096, SMALL_ENTRIES = 10240, SMALL_THREADS = SMALL_CHILDREN;
struct SmallPlan {
  int32_t first[SMALL_SEQS], kids[SMALL_SEQS];
  Child child[SMALL_CHILDREN];
  int2 copy[SMALL_CHILDREN];
};
__global__ void __launch_bounds__(SMALL_THREADS) fork_small_kernel(const __grid_constant__ Fork f, int chunks) {
  __shared__ SmallPlan plan;
  __shared__ int64_t warp_sums[SMALL_THREADS / 32];
  __shared__ uint32_t marks[SMALL_PAGES / 32];
  extern __shared__ int32_t refs[];               // [n_pages], the first block's
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, n_pages = static_cast<int>(f.n_pages);
  const bool counts = blockIdx.x == 0;
  const int count = count_of(f);
  if (counts) {
    for (int i = tid; i < n_pages; i += SMALL_THREADS) refs[i] = ld_dep_s32(f.refs + i);
    for (int i = tid; i < (n_pages + 31) / 32; i += SMALL_THREADS) marks[i] = 0u;
    for (int i = tid; i < n_pages; i += SMALL_THREADS) f.free_list_out[i] = ld_dep_s32(f.free_list + i);
  }
  if (tid < SMALL_SEQS) {
    plan.first[tid] = INT32_MAX;
    plan.kids[tid] = 0;
  }
  __syncthreads();
  if (tid < f.n_children) {
    const int p = ld_dep_s32(f.parent + tid);
    if (p >= 0 && p < f.n_seqs) {
      atomicMin(plan.first + p, tid);
      atomicAdd(plan.kids + p, 1);
    }
  }
  __syncthreads();
  Wants w = wants_of(f, tid, plan.first);
  int64_t lacking, n_copies;
  give(w, block_sum(w.fresh, warp_sums, &lacking) - w.fresh, count);
  const int2 c = copy_of(f, w, count);
  const bool mine = copies(f, c);
  const int64_t place = block_sum(mine ? 1 : 0, warp_sums, &n_copies);
  if (mine) plan.copy[place - 1] = c;
  plan.child[tid] = w.c;
  const int taken = static_cast<int>(min(lacking, static_cast<int64_t>(count)));
  __syncthreads();
  if (counts) {
    if (tid < f.n_children) {
      f.held_out[tid] = w.c.have + w.c.got;
      f.length_out[tid] = length_of(w);
    }
    if (tid == 0) f.missing[0] = static_cast<int>(min(lacking - taken, static_cast<int64_t>(INT32_MAX)));
    // a warp a sequence: its full pages have its children for holders, without any all its pages one holder less
    for (int s = tid >> 5; s < f.n_seqs; s += SMALL_THREADS / 32) {
      const int kids = plan.kids[s];
      if (kids == 1) continue;
      const Seq q = seq_of(f, s);
      const int n = kids == 0 ? q.held : q.length / PAGE_TOKENS;
      for (int j = tid & 31; j < n; j += 32) {
        const int page = ld_dep_s32(f.table + static_cast<size_t>(s) * f.width + j);
        if (page < 0 || page >= n_pages) continue;
        const int before = atomicAdd(refs + page, kids - 1);
        if (kids == 0 && before == 1) atomicOr(marks + (page >> 5), 1u << (page & 31));
      }
    }
    __syncthreads();
    for (int k = tid; k < taken; k += SMALL_THREADS) {            // the list's last pages
      const int page = ld_dep_s32(f.free_list + count - 1 - k);
      if (page >= 0 && page < n_pages) refs[page] = 1;
    }
    __syncthreads();
    for (int i = tid; i < n_pages; i += SMALL_THREADS) f.refs_out[i] = refs[i];
    int64_t n_freed;
    const uint32_t m = tid < (n_pages + 31) / 32 ? marks[tid] : 0u;
    int64_t to = count - taken + block_sum(__popc(m), warp_sums, &n_freed) - __popc(m);
    return_freed(f, m, tid * 32, to);
    if (tid == 0) f.free_count_out[0] = static_cast<int>(min(count - taken + n_freed, f.n_pages));
    return;
  }
  const int64_t others = gridDim.x - 1, me = blockIdx.x - 1;
  for (int64_t i = me; i < f.n_children; i += others) {
    const Child ch = plan.child[i];
    for (int j = tid; j < f.width_out; j += SMALL_THREADS) f.table_out[static_cast<size_t>(i) * f.width_out + j] = entry_of(f, ch, count, j);
  }
  for (int64_t u = me; u < n_copies * chunks; u += others) copy_chunk<SMALL_THREADS>(f, plan.copy[u / chunks], static_cast<int>(u % chunks));
}

// ---------------------------------------------------------------------------------------------------- two kernels
constexpr int PLAN_THREADS = 1024;
__global__ void __launch_bounds__(PLAN_THREADS) fork_plan_kernel(const __grid_constant__ Fork f) {
  extern __shared__ int32_t by_seq[];             // [n_seqs] first child, [n_seqs] number of children
  __shared__ int64_t warp_sums[PLAN_THREADS / 32];
  pdl_launch_dependents();
  pdl_wait();
  const Plan plan = plan_of(f.workspace);
  const int tid = threadIdx.x;
  if (blockIdx.x > 0) {
    const int64_t step = static_cast<int64_t>(gridDim.x - 1) * PLAN_THREADS, at = static_cast<int64_t>(blockIdx.x - 1) * PLAN_THREADS + tid;
    for (int64_t i = at; i < (f.n_pages + 31) / 32; i += step) plan.marks[i] = 0u;
    if (f.refs_out != f.refs)
      for (int64_t i = at; i < f.n_pages; i += step) {
        const int a = ld_dep_s32(f.refs + i), b = ld_dep_s32(f.free_list + i);
        f.refs_out[i] = a;
        f.free_list_out[i] = b;
      }
    return;
  }
  int32_t *first = by_seq, *kids = by_seq + f.n_seqs;
  for (int s = tid; s < f.n_seqs; s += PLAN_THREADS) { first[s] = INT32_MAX; kids[s] = 0; }
  const int count = count_of(f);
  __syncthreads();
  for (int i = tid; i < f.n_children; i += PLAN_THREADS) {
    const int p = ld_dep_s32(f.parent + i);
    if (p >= 0 && p < f.n_seqs) {
      atomicMin(first + p, i);
      atomicAdd(kids + p, 1);
    }
  }
  __syncthreads();
  for (int s = tid; s < f.n_seqs; s += PLAN_THREADS) plan.kids[s] = kids[s];
  int64_t before = 0;
  for (int i0 = 0; i0 < f.n_children; i0 += PLAN_THREADS) {
    const int i = i0 + tid;
    Wants w = wants_of(f, i, first);
    int64_t all;
    give(w, before + block_sum(w.fresh, warp_sums, &all) - w.fresh, count);
    before += all;
    if (i < f.n_children) {
      plan.child[i] = w.c;
      f.held_out[i] = w.c.have + w.c.got;
      f.length_out[i] = length_of(w);
      plan.copy[i] = copy_of(f, w, count);
    }
  }
  if (tid == 0) {
    const int64_t taken = min(before, static_cast<int64_t>(count));
    f.missing[0] = static_cast<int>(min(before - taken, static_cast<int64_t>(INT32_MAX)));
    *plan.head = PlanHead{count, static_cast<int>(taken), 0, 0};
  }
}

constexpr int FORK_THREADS = 256;

__device__ __forceinline__ int volatile_s32(const int32_t* p) { return *reinterpret_cast<const volatile int32_t*>(p); }

__global__ void __launch_bounds__(FORK_THREADS) fork_kernel(const __grid_constant__ Fork f, int chunks) {
  __shared__ int64_t warp_sums[FORK_THREADS / 32];
  __shared__ int last;
  __shared__ int2 list[FORK_THREADS];
  pdl_launch_dependents();
  pdl_wait();
  const Plan plan = plan_of(f.workspace);
  const int tid = threadIdx.x;
  const int count = volatile_s32(&plan.head->count);

  // ---- tables, and the counters of pages that were taken
  for (int i = blockIdx.x; i < f.n_children; i += gridDim.x) {
    const volatile Child* at = plan.child + i;
    const Child c{at->parent, at->have, at->got, at->full, at->start};
    for (int j = tid; j < f.width_out; j += FORK_THREADS) {
      const int page = entry_of(f, c, count, j);
      if (j >= c.have && page >= 0 && page < f.n_pages) f.refs_out[page] = 1;
      f.table_out[static_cast<size_t>(i) * f.width_out + j] = page;
    }
  }
  // ---- counters: from the other end of the grid
  for (int s = gridDim.x - 1 - blockIdx.x; s < f.n_seqs; s += gridDim.x) {
    const int kids = volatile_s32(plan.kids + s);
    if (kids == 1) continue;
    const Seq q = seq_of(f, s);
    const int n = kids == 0 ? q.held : q.length / PAGE_TOKENS;
    for (int j = tid; j < n; j += FORK_THREADS) {
      const int page = ld_dep_s32(f.table + static_cast<size_t>(s) * f.width + j);
      if (page < 0 || page >= f.n_pages) continue;
      const int before = atomicAdd(f.refs_out + page, kids - 1);
      if (kids == 0 && before == 1) atomicOr(plan.marks + (page >> 5), 1u << (page & 31));
    }
  }
  __threadfence();
  __syncthreads();
  if (tid == 0) last = atomicAdd(&plan.head->done, 1) == static_cast<int>(gridDim.x) - 1;
  __syncthreads();
  if (last) {
    __threadfence();
    // ---- the freed pages behind the list's rest, in ascending order
    const int words = static_cast<int>((f.n_pages + 31) / 32);
    int64_t at = count - volatile_s32(&plan.head->taken);
    for (int w0 = 0; w0 < words; w0 += FORK_THREADS * 4) {
      uint32_t m[4];
      int n = 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int w = w0 + tid * 4 + u;
        m[u] = w < words ? *reinterpret_cast<const volatile uint32_t*>(plan.marks + w) : 0u;
        n += __popc(m[u]);
      }
      int64_t all;
      int64_t to = at + block_sum(n, warp_sums, &all) - n;
      at += all;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        return_freed(f, m[u], (w0 + tid * 4 + u) * 32, to);
        to += __popc(m[u]);
      }
    }
    if (tid == 0) f.free_count_out[0] = static_cast<int>(min(at, f.n_pages));
  }

  // ---- copies
  if (chunks == 0) return;
  for (int i0 = 0; i0 < f.n_children; i0 += FORK_THREADS) {
    // this window's copies, one behind the other
    int2 c = make_int2(-1, -1);
    if (i0 + tid < f.n_children) {
      const volatile int2* p = plan.copy + i0 + tid;
      c = make_int2(p->x, p->y);
    }
    const bool mine = copies(f, c);
    int64_t n;
    const int64_t place = block_sum(mine ? 1 : 0, warp_sums, &n);
    if (mine) list[place - 1] = c;
    __syncthreads();
#pragma unroll 1
    for (int64_t u = blockIdx.x; u < n * chunks; u += gridDim.x) {
      copy_chunk<FORK_THREADS>(f, list[u / chunks], static_cast<int>(u % chunks));
    }
    __syncthreads();
  }
}

}  // namespace

int launch_fork(const Fork& f, int n_sms, cudaStream_t s) {
  static bool set[MAX_DEVICES] = {};
  const int dev = current_device_slot();
  if (!set[dev]) {
    if (cudaFuncSetAttribute(fork_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_FORK_SEQS * 8) != cudaSuccess ||
        cudaFuncSetAttribute(fork_small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMALL_PAGES * 4) != cudaSuccess)
      return -1;
    set[dev] = true;
  }
  int64_t chunks = 0;
  for (int k = 0; k < f.n_pools; ++k) chunks += (f.pools[k].page_bytes + COPY_BYTES - 1) / COPY_BYTES * f.pools[k].n_layers;
  if (chunks > INT32_MAX) return -2;
  // as many blocks as there is work at most: rows of tables, and the copies if every child but one makes one
  const int64_t work = std::max<int64_t>(f.n_children, chunks * std::max(f.n_children - 1, 0));
  // (in place the first block would change what blocks that start later still have to read)
  if (f.refs_out != f.refs && f.n_seqs <= SMALL_SEQS && f.n_children <= SMALL_CHILDREN && f.n_pages <= SMALL_PAGES && static_cast<int64_t>(f.n_seqs) * f.width <= SMALL_ENTRIES) {
    const int others = static_cast<int>(std::max<int64_t>(std::min<int64_t>(work, static_cast<int64_t>(n_sms) * 4 - 1), 1));
    return launch_pdl(fork_small_kernel, dim3(1 + others), dim3(SMALL_THREADS), static_cast<size_t>(f.n_pages) * 4, s, f, static_cast<int>(chunks)) == cudaSuccess ? 0 : -1;
  }
  const int64_t lists = f.refs_out != f.refs ? f.n_pages : (f.n_pages + 31) / 32;
  const int list_blocks = static_cast<int>(std::min<int64_t>((lists + PLAN_THREADS - 1) / PLAN_THREADS, n_sms));
  if (launch_pdl(fork_plan_kernel, dim3(1 + std::max(list_blocks, 1)), dim3(PLAN_THREADS), static_cast<size_t>(f.n_seqs) * 8, s, f) != cudaSuccess) return -1;
  const int blocks = static_cast<int>(std::max<int64_t>(std::min<int64_t>(std::max<int64_t>(work, f.n_seqs), static_cast<int64_t>(n_sms) * 6), 1));
  return launch_pdl(fork_kernel, dim3(blocks), dim3(FORK_THREADS), 0, s, f, static_cast<int>(chunks)) == cudaSuccess ? 0 : -1;
}

}  // namespace pc
