// Which slots of a context to keep, and moving the kept ones together.
#include "kernels.h"
#include "ptx.cuh"

namespace pc {
namespace {

// ---------------------------------------------------------------------------------------------------- choice
constexpr int SEL_THREADS = 1024;
constexpr int SEL_WARPS = SEL_THREADS / 32;

// Order-preserving map of a weight to 32 bits (NaN as -infinity, -0 as 0); slots that are always kept come first.
__device__ __forceinline__ uint32_t weight_key(float w, int slot, int len, int sink, int recent) {
  if (slot < sink || slot >= len - recent) return 0xffffffffu;
  if (isnan(w)) w = -INFINITY;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// One block per (prompt, head): the budget-th largest key by radix selection, eight bits at a time from the top, then
// one ordered pass that writes the slots above it and as many of the equal ones as are left, lowest slot first.
__global__ void __launch_bounds__(SEL_THREADS)
select_slots_kernel(const float* __restrict__ weights, int64_t w_stride, const int32_t* __restrict__ length, int n_heads,
                    int max_len, int budget, int sink, int recent, int32_t* __restrict__ keep, int32_t* __restrict__ count) {
  __shared__ int hist[256];
  __shared__ uint32_t sh_prefix;
  __shared__ int sh_need;
  __shared__ int warp_gt[SEL_WARPS], warp_eq[SEL_WARPS];
  const int b = blockIdx.y, h = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int len = min(max(__ldg(length + b), 0), max_len);
  const float* w = weights + (static_cast<size_t>(b) * n_heads + h) * w_stride;
  int32_t* out = keep + (static_cast<size_t>(b) * n_heads + h) * budget;
  if (h == 0 && tid == 0) count[b] = min(len, budget);
  for (int j = min(len, budget) + tid; j < budget; j += SEL_THREADS) out[j] = -1;
  if (len <= budget) {
    for (int j = tid; j < len; j += SEL_THREADS) out[j] = j;
    return;
  }
  uint32_t prefix = 0;
  int need = budget;                       // how many of the keys that share the prefix are kept
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += SEL_THREADS) hist[i] = 0;
    __syncthreads();
    for (int s = tid; s < len; s += SEL_THREADS) {
      const uint32_t k = weight_key(w[s], s, len, sink, recent);
      if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int left = need, d = 255;
      while (hist[d] < left) left -= hist[d--];
      sh_prefix = prefix | (static_cast<uint32_t>(d) << shift);
      sh_need = left;
    }
    __syncthreads();
    prefix = sh_prefix;
    need = sh_need;
  }
  int base = 0, eq_base = 0;               // slots written so far; equal ones seen so far
  for (int s0 = 0; s0 < len; s0 += SEL_THREADS) {
    const int s = s0 + tid;
    const uint32_t k = s < len ? weight_key(w[s], s, len, sink, recent) : 0u;
    const bool gt = s < len && k > prefix, eq = s < len && k == prefix;
    const uint32_t bg = __ballot_sync(0xffffffffu, gt), be = __ballot_sync(0xffffffffu, eq);
    if (lane == 0) { warp_gt[warp] = __popc(bg); warp_eq[warp] = __popc(be); }
    __syncthreads();
    int g0 = 0, e0 = 0, g_all = 0, e_all = 0;
    for (int i = 0; i < SEL_WARPS; ++i) {
      if (i < warp) { g0 += warp_gt[i]; e0 += warp_eq[i]; }
      g_all += warp_gt[i]; e_all += warp_eq[i];
    }
    const int eq_before = eq_base + e0 + __popc(be & ((1u << lane) - 1));
    const int gt_before = g0 + __popc(bg & ((1u << lane) - 1));
    if (gt || (eq && eq_before < need)) out[base + gt_before + min(eq_before, need) - min(eq_base, need)] = s;
    base += g_all + min(eq_base + e_all, need) - min(eq_base, need);
    eq_base += e_all;
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------------- moving
constexpr int MOVE_THREADS = 512;
constexpr int MOVE_UNROLL = 4;

// A block moves one slice of (prompt, KV head): all vectors of K, all of V, or the weights.  In place the list's chunks
// go in order, each read whole before it is written: its sources lie at or behind the chunk's own start, because
// keep[j] >= first + j and the list ascends, so no later chunk reads what an earlier one has written.
__global__ void __launch_bounds__(MOVE_THREADS) compact_slots_kernel(CompactSlots a) {
  const int b = blockIdx.z, g = blockIdx.y, slice = blockIdx.x;
  const int n = min(min(max(__ldg(a.count + b), 0), a.budget), a.max_len);
  const int first = a.first ? __ldg(a.first + b) : 0;
  const int32_t* keep = a.keep + (static_cast<size_t>(b) * a.keep_heads + (a.keep_heads == 1 ? 0 : g)) * a.budget;
  const int32_t* dpt = a.dst_page_table ? a.dst_page_table : a.kv.page_table;
  const int dpt_stride = a.dst_page_table ? a.dst_pt_stride : a.kv.pt_stride;
  const int32_t* dst0 = a.dst_start ? a.dst_start : a.kv.ctx_start;
  if (first < 0) return;
  if (slice == 2) {
    if (!a.w_in) return;
    const size_t row = (static_cast<size_t>(b) * a.kv.n_kv_heads + g) * a.w_stride;
    for (int j0 = 0; j0 < n; j0 += MOVE_THREADS) {
      const int j = j0 + threadIdx.x;
      const int s = j < n ? keep[j] : -1;
      const bool ok = s >= 0 && s < a.max_len && first + j < a.max_len;
      const float w = ok ? a.w_in[row + s] : 0.f;
      __syncthreads();
      if (ok) a.w_out[row + first + j] = w;
    }
    return;
  }
  const int vecs = a.kv.head_dim / 8;                 // 16-byte vectors of a head's row
  const int64_t stride = slice == 0 ? a.kv.k_stride : a.kv.v_stride;
  uint4* pool = reinterpret_cast<uint4*>(const_cast<void*>(slice == 0 ? a.kv.k : a.kv.v));
  const int total = n * vecs;
  for (int e0 = 0; e0 < total; e0 += MOVE_THREADS * MOVE_UNROLL) {
    uint4 r[MOVE_UNROLL];
    int64_t to[MOVE_UNROLL];
#pragma unroll
    for (int u = 0; u < MOVE_UNROLL; ++u) {
      const int e = e0 + u * MOVE_THREADS + threadIdx.x;
      to[u] = -1;
      if (e >= total) continue;
      const int j = e / vecs, c = e % vecs;
      const int s = keep[j], t = first + j;
      if (s < 0 || s >= a.max_len || t >= a.max_len) continue;
      if (dpt && t / PAGE_TOKENS >= dpt_stride) continue;
      const int64_t src = slot_row(a.kv.page_table, a.kv.pt_stride, a.kv.ctx_start, a.kv.n_slots, b, s);
      const int64_t dst = slot_row(dpt, dpt_stride, dst0, a.kv.n_slots, b, t);
      if (src < 0 || dst < 0) continue;
      r[u] = pool[(src * stride + g * a.kv.head_dim) / 8 + c];
      to[u] = (dst * stride + g * a.kv.head_dim) / 8 + c;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < MOVE_UNROLL; ++u)
      if (to[u] >= 0) pool[to[u]] = r[u];
  }
}

}  // namespace

int launch_select_slots(const float* weights, int64_t w_stride, const int32_t* length, int n_seqs, int n_heads, int max_len,
                        int budget, int sink, int recent, int32_t* keep, int32_t* count, int, cudaStream_t s) {
  select_slots_kernel<<<dim3(n_heads, n_seqs), SEL_THREADS, 0, s>>>(weights, w_stride, length, n_heads, max_len, budget,
                                                                    sink, recent, keep, count);
  return cudaPeekAtLastError() == cudaSuccess ? 0 : -1;
}

int launch_compact_slots(const CompactSlots& a, int, cudaStream_t s) {
  compact_slots_kernel<<<dim3(3, a.kv.n_kv_heads, a.n_seqs), MOVE_THREADS, 0, s>>>(a);
  return cudaPeekAtLastError() == cudaSuccess ? 0 : -1;
}

}  // namespace pc
