// Which slots of a context to keep, and moving the kept ones together.
#include <algorithm>

#include "slot_row.cuh"

namespace pc {
namespace {

// ---------------------------------------------------------------------------------------------------- choice
// One block per (prompt, head).  What is always kept (the first `sink`, the last `recent`) is written outright; of the slots
// between, the heaviest `need` are found by radix selection: a histogram of the top 11 bits of their keys and the bin in which
// `need` runs out, then of the next 11 bits of the keys in that bin, then of the last 10.  Every warp has a stretch of slots of
// its own, so that it can count what it keeps and then write it, in slot order, without talking to the others: all above the key
// found, and of the equal ones as many as are left, lowest slot first.
// Bounds: the weights are a few bytes a thread; what counts is the number of instructions per weight and pass (11 bins of 43
// were key arithmetic before the always-kept slots were taken out and NaN and -0 were folded into two operations) and the latency of
// the dependent passes.  Weights stay in registers when a warp's stretch is at most 32 x SEL_UNROLL slots.  Longer lists are read
// three times: for the first histogram, to put the keys of the bin found into a list in shared memory (the other passes work on
// that), and to write; where the bin holds more than the list (many equal weights), every pass reads all again.  224 lists of 33024:
// 34 us at 71 % of the issue slots (41.6 without the list); 224 of 2112: 6.8 us.
constexpr int SEL_BITS = 11, SEL_BINS = 1 << SEL_BITS;
constexpr int SEL_UNROLL = 8;

// Order-preserving map of a weight to 32 bits: NaN as -infinity (maximum drops it), -0 as 0 (adding 0 does).
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(fmaxf(w, -INFINITY) + 0.f);
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}

// Block sizes: lists of up to 512 * SEL_UNROLL weights are always held in registers, so only the larger block has the list.
constexpr int SEL_SHORT = 512, SEL_LONG = 1024;
constexpr int SEL_LIST = 4096;
template <int THREADS>
struct SelectShared {
  int hist[SEL_BINS];
  int warp_sum[THREADS / 32], warp_gt[THREADS / 32], warp_eq[THREADS / 32];
  int bin, need, listed;
  uint2 list[THREADS == SEL_LONG ? SEL_LIST : 1];       // key and slot of the first bin's weights
};

// lo .. hi - 1: this warp's stretch (of `stretch` slots) of the middle, whose first slot is `first`; out: where the middle's list starts.
template <int THREADS, bool IN_REGS>
__device__ __forceinline__ void select_middle(SelectShared<THREADS>& sh, const float* w, int first, int stretch, int lo, int hi, int need, int32_t* out) {
  constexpr int BINS_EACH = SEL_BINS / THREADS;
  static_assert(SEL_BINS % THREADS == 0, "");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t key[SEL_UNROLL];
  auto fetch = [&](int s0) {
    float x[SEL_UNROLL];
#pragma unroll
    for (int u = 0; u < SEL_UNROLL; ++u) x[u] = s0 + u * 32 < hi ? __ldg(w + s0 + u * 32) : 0.f;
#pragma unroll
    for (int u = 0; u < SEL_UNROLL; ++u) key[u] = weight_key(x[u]);
  };
  // fn(slot, key, inside) for every slot of the stretch, 32 consecutive ones a step
  auto each = [&](auto fn) {
    if constexpr (IN_REGS) {
#pragma unroll
      for (int u = 0; u < SEL_UNROLL; ++u) fn(lo + lane + u * 32, key[u], lo + lane + u * 32 < hi);
    } else {
      int s0 = lo;
#pragma unroll 1
      for (; s0 + 32 * SEL_UNROLL <= hi; s0 += 32 * SEL_UNROLL) {
        float x[SEL_UNROLL];
#pragma unroll
        for (int u = 0; u < SEL_UNROLL; ++u) x[u] = __ldg(w + s0 + lane + u * 32);
#pragma unroll
        for (int u = 0; u < SEL_UNROLL; ++u) fn(s0 + lane + u * 32, weight_key(x[u]), true);
      }
#pragma unroll 1
      for (; s0 < hi; s0 += 32) fn(s0 + lane, weight_key(s0 + lane < hi ? __ldg(w + s0 + lane) : 0.f), s0 + lane < hi);
    }
  };
  if constexpr (IN_REGS) fetch(lo + lane);
  uint32_t prefix = 0, known = 0;          // the key's bits found so far, and which bits those are
  bool listed = false;                     // the keys that share the prefix are all in sh.list
  int gt = 0, eq = 0;
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t digit = pass == 2 ? 1023u : 2047u;
    for (int i = tid; i < SEL_BINS; i += THREADS) sh.hist[i] = 0;
    __syncthreads();
    auto add = [&](uint32_t k) {
      if ((k & known) == prefix) atomicAdd(&sh.hist[(k >> shift) & digit], 1);
    };
    if (listed) {
      for (int i = tid; i < sh.listed; i += THREADS) add(sh.list[i].x);
    } else {
      each([&](int, uint32_t k, bool inside) {
        if (inside) add(k);
      });
    }
    __syncthreads();
    // thread t has the bins SEL_BINS - 1 - t * BINS_EACH downwards: which of them is it in which the running count reaches `need`
    int c[BINS_EACH], mine = 0;
#pragma unroll
    for (int i = 0; i < BINS_EACH; ++i) { c[i] = sh.hist[SEL_BINS - 1 - tid * BINS_EACH - i]; mine += c[i]; }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    if (lane == 31) sh.warp_sum[warp] = incl;
    __syncthreads();
    int others = lane < warp ? sh.warp_sum[lane] : 0;       // at most 32 warps
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) others += __shfl_xor_sync(0xffffffffu, others, o);
    int before = others + incl - mine;
    if (before < need && before + mine >= need) {
#pragma unroll
      for (int i = 0; i < BINS_EACH; ++i) {
        if (before < need && before + c[i] >= need) { sh.bin = SEL_BINS - 1 - tid * BINS_EACH - i; sh.need = need - before; }
        before += c[i];
      }
    }
    __syncthreads();
    prefix |= static_cast<uint32_t>(sh.bin) << shift;
    known |= digit << shift;
    need = sh.need;
    if constexpr (!IN_REGS) {
      if (pass == 0) {
        if (tid == 0) sh.listed = 0;
        __syncthreads();
        each([&](int s, uint32_t k, bool inside) {
          const uint32_t top = k & known;
          gt += inside && top > prefix;
          const bool mine = inside && top == prefix;
          const uint32_t all = __ballot_sync(0xffffffffu, mine);
          if (all != 0) {
            int at = 0;
            if (lane == 0) at = atomicAdd(&sh.listed, __popc(all));
            at = __shfl_sync(0xffffffffu, at, 0) + __popc(all & ((1u << lane) - 1));
            if (mine && at < SEL_LIST) sh.list[at] = make_uint2(k, static_cast<uint32_t>(s));
          }
        });
        __syncthreads();
        listed = sh.listed <= SEL_LIST;
      }
    }
  }
  // what every warp keeps of its stretch
  if (listed) {
    gt = __reduce_add_sync(0xffffffffu, gt);
    if (lane == 0) { sh.warp_gt[warp] = gt; sh.warp_eq[warp] = 0; }
    __syncthreads();
    for (int i = tid; i < sh.listed; i += THREADS) {
      const uint2 e = sh.list[i];
      if (e.x >= prefix) atomicAdd(e.x > prefix ? &sh.warp_gt[e.y / stretch] : &sh.warp_eq[e.y / stretch], 1);
    }
  } else {
    gt = 0;
    each([&](int, uint32_t k, bool inside) {
      gt += inside && k > prefix;
      eq += inside && k == prefix;
    });
    gt = __reduce_add_sync(0xffffffffu, gt);
    eq = __reduce_add_sync(0xffffffffu, eq);
    if (lane == 0) { sh.warp_gt[warp] = gt; sh.warp_eq[warp] = eq; }
  }
  __syncthreads();
  const bool any_eq = sh.warp_eq[warp] != 0;
  int gt_before = __reduce_add_sync(0xffffffffu, lane < warp ? sh.warp_gt[lane] : 0);
  int eq_before = __reduce_add_sync(0xffffffffu, lane < warp ? sh.warp_eq[lane] : 0);
  const uint32_t below = (1u << lane) - 1;
  each([&](int s, uint32_t k, bool inside) {
    const bool is_gt = inside && k > prefix, is_eq = inside && k == prefix;
    const uint32_t bg = __ballot_sync(0xffffffffu, is_gt);
    if (!any_eq) {                                        // most stretches
      if (is_gt) out[gt_before + __popc(bg & below) + min(eq_before, need)] = first + s;
    } else {
      const uint32_t be = __ballot_sync(0xffffffffu, is_eq);
      const int e = eq_before + __popc(be & below);
      if (is_gt || (is_eq && e < need)) out[gt_before + __popc(bg & below) + min(e, need)] = first + s;
      eq_before += __popc(be);
    }
    gt_before += __popc(bg);
  });
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS)
select_slots_kernel(const float* __restrict__ weights, int64_t w_stride, const int32_t* __restrict__ length, int n_heads,
                    int max_len, int budget, int sink, int recent, int32_t* __restrict__ keep, int32_t* __restrict__ count) {
  __shared__ SelectShared<THREADS> sh;
  const int b = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, warp = tid >> 5;
  const int len = min(max(__ldg(length + b), 0), max_len);
  int32_t* out = keep + (static_cast<size_t>(b) * n_heads + h) * budget;
  if (h == 0 && tid == 0) count[b] = min(len, budget);
  if (len <= budget) {
    for (int j = tid; j < budget; j += THREADS) out[j] = j < len ? j : -1;
    return;
  }
  for (int j = tid; j < sink + recent; j += THREADS) {
    if (j < sink) out[j] = j;
    else out[budget - recent + j - sink] = len - recent + j - sink;
  }
  const int need = budget - sink - recent, n = len - sink - recent;       // 0 <= need < n
  if (need == 0) return;
  const float* w = weights + (static_cast<size_t>(b) * n_heads + h) * w_stride + sink;
  const int stretch = (n + THREADS - 1) / THREADS * 32;                    // whole steps of 32 for each warp
  const int lo = min(warp * stretch, n), hi = min(lo + stretch, n);
  if constexpr (THREADS == SEL_LONG) {
    if (stretch > 32 * SEL_UNROLL) {
      select_middle<THREADS, false>(sh, w, sink, stretch, lo, hi, need, out + sink);
      return;
    }
  }
  select_middle<THREADS, true>(sh, w, sink, stretch, lo, hi, need, out + sink);
}

// ---------------------------------------------------------------------------------------------------- moving
constexpr int MOVE_THREADS = 256;

struct Move { int32_t src, dst; };       // pool rows, or dst = -1: nothing moves
__device__ __forceinline__ Move move_of(const CompactSlots& a, int b, int j, int n, int first, const int32_t* keep) {
  Move m{0, -1};
  if (j >= n) return m;
  const int s = __ldg(keep + j), t = first + j;
  if (s < 0 || s >= a.max_len || t < 0 || t >= a.max_len) return m;
  const int32_t* pt = a.dst_page_table ? a.dst_page_table : a.kv.page_table;
  const int stride = a.dst_page_table ? a.dst_pt_stride : a.kv.pt_stride;
  if (pt && t / PAGE_TOKENS >= stride) return m;
  const int64_t src = slot_row(a.kv.page_table, a.kv.pt_stride, a.kv.ctx_start, a.kv.n_slots, b, s);
  const int64_t dst = slot_row(pt, stride, a.dst_start ? a.dst_start : a.kv.ctx_start, a.kv.n_slots, b, t);
  if (src < 0 || dst < 0) return m;
  m.src = static_cast<int32_t>(src);        // pools have at most 2^31 - 1 rows
  m.dst = static_cast<int32_t>(dst);
  return m;
}

// To another place: nothing that is read is written, so every (prompt, KV head, stretch of the list) is a block of its own.
// 16 lanes (8 for head size 64) take a row of K and of V; a thread has MOVE_ROWS rows of both in flight.  Bound by HBM:
// 2 x 4 D bytes a kept slot and head.  7 x 8 lists of 8192: 81.6 us (475 MB, 5.8 TB/s), 8 lists of 1024: 3.7 us; with one row a
// thread and four blocks an SM 97.7 and 4.3 us.
constexpr int MOVE_ROWS = 2;
template <int D>
__global__ void __launch_bounds__(MOVE_THREADS, 6) copy_slots_kernel(CompactSlots a) {
  constexpr int VECS = D / 8, ROWS = MOVE_THREADS / VECS;
  const int b = blockIdx.z, g = blockIdx.y;
  const int n = min(min(max(__ldg(a.count + b), 0), a.budget), a.max_len);
  const int j0 = blockIdx.x * ROWS * MOVE_ROWS + threadIdx.x / VECS;
  if (static_cast<int>(blockIdx.x) * ROWS * MOVE_ROWS >= n) return;
  const int c = threadIdx.x % VECS;
  const int first = a.first ? __ldg(a.first + b) : 0;
  const int32_t* keep = a.keep + (static_cast<size_t>(b) * a.keep_heads + (a.keep_heads == 1 ? 0 : g)) * a.budget;
  const uint4* k = static_cast<const uint4*>(a.kv.k) + g * VECS + c;
  const uint4* v = static_cast<const uint4*>(a.kv.v) + g * VECS + c;
  const int64_t ks = a.kv.k_stride / 8, vs = a.kv.v_stride / 8;
  Move m[MOVE_ROWS];
  uint4 rk[MOVE_ROWS], rv[MOVE_ROWS];
#pragma unroll
  for (int u = 0; u < MOVE_ROWS; ++u) m[u] = move_of(a, b, j0 + u * ROWS, n, first, keep);
#pragma unroll
  for (int u = 0; u < MOVE_ROWS; ++u) {
    if (m[u].dst < 0) continue;
    rk[u] = k[m[u].src * ks];
    rv[u] = v[m[u].src * vs];
  }
#pragma unroll
  for (int u = 0; u < MOVE_ROWS; ++u) {
    if (m[u].dst < 0) continue;
    const_cast<uint4*>(k)[m[u].dst * ks] = rk[u];
    const_cast<uint4*>(v)[m[u].dst * vs] = rv[u];
  }
  if (a.w_in && a.w_in != a.w_out && c == 0) {
    const size_t row = (static_cast<size_t>(b) * a.kv.n_kv_heads + g) * a.w_stride;
#pragma unroll
    for (int u = 0; u < MOVE_ROWS; ++u) {
      const int j = j0 + u * ROWS, s = j < n ? __ldg(keep + j) : -1;
      if (s >= 0 && s < a.max_len && first + j >= 0 && first + j < a.max_len) a.w_out[row + first + j] = __ldg(a.w_in + row + s);
    }
  }
}

// In place.  A block owns a slice (some 16-byte vectors of K or of V, or the weights) of one (prompt, KV head) and takes the
// list's chunks in order, each read whole before any of it is written: its sources lie at or behind the chunk's own first
// slot, because keep[j] >= first + j and the list ascends, so no chunk reads what an earlier one has written.  Slices, not
// chunks, are what runs in parallel; the host makes them as narrow as it takes to fill the SMs four times (7 x 8 lists of 8192:
// 198 - 215 us in several runs, floor 74; twice: 236 us.  64 x 8 lists of 512: 78 - 81 us either way, floor 42).  What bounds it: a
// chunk's loads, a barrier and its stores follow each other, and 32 bytes of a 256-byte row are a thin slice.
constexpr int SHIFT_UNROLL = 8;
__global__ void __launch_bounds__(MOVE_THREADS) shift_slots_kernel(CompactSlots a, int slices, int vecs, int first_slice) {
  const int b = blockIdx.z, g = blockIdx.y, slice = blockIdx.x + first_slice;
  const int n = min(min(max(__ldg(a.count + b), 0), a.budget), a.max_len);
  const int first = a.first ? __ldg(a.first + b) : 0;
  const int32_t* keep = a.keep + (static_cast<size_t>(b) * a.keep_heads + (a.keep_heads == 1 ? 0 : g)) * a.budget;
  if (slice == 2 * slices) {
    const size_t row = (static_cast<size_t>(b) * a.kv.n_kv_heads + g) * a.w_stride;
    for (int j0 = 0; j0 < n; j0 += MOVE_THREADS * SHIFT_UNROLL) {
      float w[SHIFT_UNROLL];
      bool ok[SHIFT_UNROLL];
#pragma unroll
      for (int u = 0; u < SHIFT_UNROLL; ++u) {
        const int j = j0 + u * MOVE_THREADS + threadIdx.x;
        const int s = j < n ? __ldg(keep + j) : -1;
        ok[u] = s >= 0 && s < a.max_len && first + j >= 0 && first + j < a.max_len;
        if (ok[u]) w[u] = a.w_in[row + s];
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < SHIFT_UNROLL; ++u)
        if (ok[u]) a.w_out[row + first + j0 + u * MOVE_THREADS + threadIdx.x] = w[u];
    }
    return;
  }
  const bool is_k = slice < slices;
  const int64_t stride = (is_k ? a.kv.k_stride : a.kv.v_stride) / 8;
  uint4* pool = static_cast<uint4*>(const_cast<void*>(is_k ? a.kv.k : a.kv.v)) + g * (a.kv.head_dim / 8) +
                (is_k ? slice : slice - slices) * vecs + threadIdx.x % vecs;
  const int rows = MOVE_THREADS / vecs;
  for (int j0 = 0; j0 < n; j0 += rows * SHIFT_UNROLL) {
    uint4 r[SHIFT_UNROLL];
    int64_t to[SHIFT_UNROLL];
#pragma unroll
    for (int u = 0; u < SHIFT_UNROLL; ++u) {
      const Move m = move_of(a, b, j0 + u * rows + threadIdx.x / vecs, n, first, keep);
      to[u] = m.dst == m.src ? -1 : m.dst;
      if (to[u] >= 0) r[u] = pool[m.src * stride];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < SHIFT_UNROLL; ++u)
      if (to[u] >= 0) pool[to[u] * stride] = r[u];
  }
}

__global__ void __launch_bounds__(MOVE_THREADS) clear_weights_kernel(float* weights, int64_t w_stride, int n_prompts, const int32_t* __restrict__ from,
                                                                     const int32_t* __restrict__ to) {
  const int b = blockIdx.x % n_prompts;                  // a list is a layer and a prompt: more than a grid's other dimensions hold
  float* w = weights + (static_cast<size_t>(blockIdx.x) * gridDim.y + blockIdx.y) * w_stride;
  for (int s = __ldg(from + b) + threadIdx.x; s < __ldg(to + b); s += MOVE_THREADS) w[s] = 0.f;
}

// <<<>>> with the launch's own status: the thread's last error may be an earlier call's.
template <typename... KArgs, typename... Args>
cudaError_t launch(void (*kernel)(KArgs...), dim3 grid, int threads, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

}  // namespace

int launch_clear_weights(float* weights, int64_t w_stride, int n_lists, int n_heads, int n_prompts, const int32_t* from, const int32_t* to,
                         cudaStream_t s) {
  return launch(clear_weights_kernel, dim3(n_lists, n_heads), MOVE_THREADS, s, weights, w_stride, n_prompts, from, to) == cudaSuccess ? 0 : -1;
}

int launch_select_slots(const float* weights, int64_t w_stride, const int32_t* length, int n_seqs, int n_heads, int max_len,
                        int budget, int sink, int recent, int32_t* keep, int32_t* count, cudaStream_t s) {
  const dim3 grid(n_heads, n_seqs);
  // 512 threads hold up to 4096 weights of a list in registers, 1024 hold 8192 (and share the reading of longer ones).  8 lists of 2112:
  // 4.9 us with 512, 6.2 with 1024; 512 lists of 2500: 10.7 and 18.5; 224 lists of 8192: 13.0 and 11.8; 8 lists of 33024: 28.3 and 19.8.
  const bool large = max_len > SEL_SHORT * SEL_UNROLL;
  return launch(large ? select_slots_kernel<SEL_LONG> : select_slots_kernel<SEL_SHORT>, grid, large ? SEL_LONG : SEL_SHORT, s, weights, w_stride, length, n_heads,
                max_len, budget, sink, recent, keep, count) == cudaSuccess ? 0 : -1;
}

int launch_compact_slots(const CompactSlots& a, int n_sms, cudaStream_t s) {
  const int n = std::min(a.budget, a.max_len), vecs = a.kv.head_dim / 8;
  const bool in_place = !a.dst_page_table && !a.dst_start;
  const bool shift_weights = a.w_in && (in_place || a.w_in == a.w_out);
  if (!in_place) {
    const int rows = MOVE_THREADS / vecs * MOVE_ROWS;
    const dim3 grid((n + rows - 1) / rows, a.kv.n_kv_heads, a.n_seqs);
    if (launch(a.kv.head_dim == 128 ? copy_slots_kernel<128> : copy_slots_kernel<64>, grid, MOVE_THREADS, s, a) != cudaSuccess) return -1;
  }
  if (in_place || shift_weights) {
    int slices = 1;
    while (slices < vecs / 2 && static_cast<int64_t>(a.n_seqs) * a.kv.n_kv_heads * 2 * slices < 4 * static_cast<int64_t>(n_sms)) slices *= 2;
    const int first_slice = in_place ? 0 : 2 * slices, last = 2 * slices + (shift_weights ? 1 : 0);
    const dim3 grid(last - first_slice, a.kv.n_kv_heads, a.n_seqs);
    if (launch(shift_slots_kernel, grid, MOVE_THREADS, s, a, slices, vecs / slices, first_slice) != cudaSuccess) return -1;
  }
  return 0;
}

}  // namespace pc
