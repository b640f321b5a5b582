// What the kernels on a decoding batch's cache share: the device-side schedule, masks, workspace layout, small arithmetic.
#pragma once
#include "slot_row.cuh"

namespace pc {
namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr int BLK = 128;                        // context slots per block, rows per tile
constexpr int TREE_THREADS = 384;

// Workspace: the error word, one merge record per CTA, partial results (two slots per CTA).
constexpr int WS_MERGE = 256, WS_ML = 16384;
constexpr int MAX_CTAS = 160;
constexpr size_t WS_O = WS_ML + sizeof(float) * 2 * BLK * 2 * MAX_CTAS;
static_assert(WS_MERGE + sizeof(int) * 8 * MAX_CTAS <= WS_ML, "");
static_assert(WS_O + sizeof(float) * 2 * MAX_CTAS * BLK * HEAD_DIM <= (24u << 20), "PERCACHE_OPS_WORKSPACE_BYTES");

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Bounded wait for kernels with many wait sites.  A wait site in line is a dozen instructions; the timed loop of mbar_wait (with its
// error word) is one function of the kernel, entered by waits that take long.  Instruction fetches are what a small call's time
// goes into: with everything in line these kernels had 100 KB of code, most of it run once.
__device__ __noinline__ bool bar_wait_slow(uint64_t* bar, uint32_t parity, int* err_word, int code) {
  return mbar_wait(bar, parity, err_word, code);
}
__device__ __forceinline__ bool bar_wait(uint64_t* bar, uint32_t parity, int* err_word, int code) {
#pragma unroll 1
  for (int i = 0; i < 4096; ++i)
    if (mbar_try_wait(bar, parity)) return true;
  return bar_wait_slow(bar, parity, err_word, code);
}

// ---------------------------------------------------------------------------------------------------- schedule
// What a prompt's work looks like to the schedule: units of n_blk blocks, each block costing blk_cost, each unit `over` more (its Q, the
// rows' end).
struct Shape { int units, n_blk, blk_cost, over; };
// A prompt's part of a batch, from the device-side arrays, clamped to the bounds the host knows.
struct SeqPart { int row0, n_nodes, ctx_len; };
__device__ __forceinline__ SeqPart seq_part(const TreeRows& r, int b) {
  const int first = ld_dep_s32(r.row_start + b), last = ld_dep_s32(r.row_start + b + 1), ctx = ld_dep_s32(r.ctx_len + b);
  SeqPart p;
  p.row0 = min(max(first, 0), r.n_rows);
  p.n_nodes = min(min(min(max(last, p.row0), r.n_rows) - p.row0, r.max_nodes), r.max_len);
  p.ctx_len = min(max(ctx, 0), r.max_len - p.n_nodes);
  return p;
}
// A CTA's stretch of the batch's cost, and the prompt it starts in.
struct Span {
  int64_t begin, end, total, seq_start;
  int n_ctas, seq;
  SeqPart part;
};
struct Piece {                   // blocks [blk_begin, blk_end) of one unit
  int seq, unit, blk_begin, blk_end, n_blk;
  SeqPart part;
  int unit_end;                  // cost position behind the unit, from the span's begin on
};

// Fits 32 bits, as does a CTA's share of the batch: the host refuses sizes for which it might not (units_fit).
__device__ __forceinline__ int shape_cost(const Shape& s) { return (s.n_blk * s.blk_cost + s.over) * s.units; }
inline bool units_fit(int64_t n_seqs, int64_t units, int64_t max_len, int64_t blk_cost, int64_t over) {
  const int64_t cost = ((max_len + BLK - 1) / BLK * blk_cost + over) * units;
  return cost <= INT32_MAX / 4 && cost * n_seqs <= INT64_C(1) << 35;       // over 148 CTAs: a span below 2^28 + a unit
}

// Batches the whole of whose cost times the CTA count stays in 32 bits, and of few prompts, are dealt by every warp for itself.
constexpr int SMALL_BATCH = 256;
inline bool small_batch(int n_seqs, int64_t units, int64_t max_len, int64_t blk_cost, int64_t over) {
  return n_seqs <= SMALL_BATCH && ((max_len + BLK - 1) / BLK * blk_cost + over) * units * n_seqs <= INT32_MAX / MAX_CTAS;
}

// shape(part): a prompt's Shape.  Small batches: every warp forms the prefix sums over the prompts for itself, 32 bits, no barrier
// (these steps are ahead of everything a call does: one barrier and one 64-bit division less is 0.5 us of a small call).  Others:
// block-wide, every thread takes a run of prompts; `shared` and `warp_sums` are the block's scratch.
template <typename ShapeFn>
__device__ __forceinline__ Span make_span(const TreeRows& rows, int min_span, bool small, Span* shared, int64_t* warp_sums, ShapeFn shape) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  Span sp;
  if (small) {
    const int per = (rows.n_seqs + 31) >> 5;
    const int b0 = min(lane * per, rows.n_seqs), b1 = min(b0 + per, rows.n_seqs);
    SeqPart p{0, 0, 0};
    int mine = 0;
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
      p = seq_part(rows, b);
      mine += shape_cost(shape(p));
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    const uint32_t total = __shfl_sync(0xffffffffu, incl, 31);
    const uint32_t n = min(gridDim.x, max(total / static_cast<uint32_t>(min_span), 1u));
    const uint32_t border = total * min(blockIdx.x + (lane & 1), n) / n;
    const int begin = __shfl_sync(0xffffffffu, border, 0), end = __shfl_sync(0xffffffffu, border, 1);
    int at = incl - mine, seq = b0;
    const uint32_t owner = __ballot_sync(0xffffffffu, begin >= at && begin < at + mine);
    if (per > 1 && (owner >> lane & 1u)) {
#pragma unroll 1
      for (;; ++seq) {
        p = seq_part(rows, seq);
        const int cost = shape_cost(shape(p));
        if (begin < at + cost) break;
        at += cost;
      }
    }
    __syncwarp();
    const int from = owner ? __ffs(owner) - 1 : 0;
    sp.begin = begin; sp.end = end; sp.total = total; sp.n_ctas = n;
    sp.seq = owner ? __shfl_sync(0xffffffffu, seq, from) : rows.n_seqs;
    sp.seq_start = __shfl_sync(0xffffffffu, at, from);
    sp.part.row0 = __shfl_sync(0xffffffffu, p.row0, from);
    sp.part.n_nodes = __shfl_sync(0xffffffffu, p.n_nodes, from);
    sp.part.ctx_len = __shfl_sync(0xffffffffu, p.ctx_len, from);
    return sp;
  }
  const int per = (rows.n_seqs + TREE_THREADS - 1) / TREE_THREADS;
  const int b0 = min(tid * per, rows.n_seqs), b1 = min(b0 + per, rows.n_seqs);
  int64_t mine = 0;
#pragma unroll 1
  for (int b = b0; b < b1; ++b) mine += shape_cost(shape(seq_part(rows, b)));
  int64_t incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  int64_t at = incl - mine, total = 0;
#pragma unroll 1
  for (int w = 0; w < TREE_THREADS / 32; ++w) {
    const int64_t x = warp_sums[w];
    if (w < warp) at += x;
    total += x;
  }
  const int n = static_cast<int>(min(static_cast<int64_t>(gridDim.x), max(total / static_cast<uint32_t>(min_span), static_cast<int64_t>(1))));
  const int c = min(static_cast<int>(blockIdx.x) + (lane & 1), n);
  const int64_t border = static_cast<int64_t>(static_cast<uint64_t>(total) * c / static_cast<uint32_t>(n));
  sp.begin = __shfl_sync(0xffffffffu, border, 0);
  sp.end = __shfl_sync(0xffffffffu, border, 1);
  sp.total = sp.seq_start = total; sp.n_ctas = n; sp.seq = rows.n_seqs; sp.part = SeqPart{0, 0, 0};
  if (tid == 0) *shared = sp;
  __syncthreads();
  if (mine > 0 && sp.begin >= at && sp.begin < at + mine) {         // one thread at most
    int b = b0;
#pragma unroll 1
    for (;; ++b) {
      sp.part = seq_part(rows, b);
      const int cost = shape_cost(shape(sp.part));
      if (sp.begin < at + cost) break;
      at += cost;
    }
    sp.seq = b;
    sp.seq_start = at;
    *shared = sp;
  }
  __syncthreads();
  return *shared;
}

// The first prompt from `seq` on that costs something, or n_seqs; the whole warp calls, with the same values.
template <typename ShapeFn>
__device__ __forceinline__ int past_idle(const TreeRows& rows, ShapeFn shape, int seq) {
  for (;;) {
    const int b = seq + (threadIdx.x & 31);
    const bool idle = b < rows.n_seqs && shape_cost(shape(seq_part(rows, b))) == 0;
    const uint32_t work = ~__ballot_sync(0xffffffffu, idle);
    if (work != 0) return seq + __ffs(work) - 1;
    seq += 32;
  }
}
// Walks a span, a warp at a time.  Cost positions count from the span's begin: 32 bits (the host refuses batches whose span might not fit).
struct Cursor {
  int pos, end, seq_start;
  int seq;
  SeqPart part;                  // of prompt `seq`
  Cursor() = default;
  __device__ __forceinline__ explicit Cursor(const Span& s)
      : pos(0), end(static_cast<int>(s.end - s.begin)), seq_start(static_cast<int>(s.seq_start - s.begin)), seq(s.seq), part(s.part) {}
  // SKIP: prompts without work are looked at 32 together (8-bit pages, 64 x 2500 slots, one token each: with 250 idle ones between 131 -> 63 us, with none
  // 61.7 -> 62.0).  Kernels without registers to spare leave it (8-bit pages, trees of 26: 121 -> 125 us with none idle).
  template <bool SKIP = false, typename ShapeFn>
  __device__ __forceinline__ bool next(const TreeRows& rows, ShapeFn shape, Piece* pc) {
#pragma unroll 1
    while (pos < end && seq < rows.n_seqs) {
      const Shape sh = shape(part);
      const int whole = shape_cost(sh);
      if (pos - seq_start >= whole) {
        seq_start += whole;
        ++seq;
        if (SKIP && whole == 0) seq = past_idle(rows, shape, seq);
        if (seq < rows.n_seqs) part = seq_part(rows, seq);
        continue;
      }
      const int cost = sh.n_blk * sh.blk_cost + sh.over;
      const int unit = (pos - seq_start) / cost;
      const int unit_start = seq_start + unit * cost, unit_end = unit_start + cost;
      const int stop = min(end, unit_end);
      // a unit's own cost lies ahead of its blocks: a border inside it leaves the whole unit to the later span; a border
      // inside a block leaves the block to the later span
      int bb = max(pos - unit_start - sh.over, 0), be = max(stop - unit_start - sh.over, 0);
      if (sh.blk_cost > 1) { bb /= sh.blk_cost; be /= sh.blk_cost; }
      pos = stop;
      if (be <= bb) continue;
      pc->seq = seq; pc->unit = unit; pc->part = part;
      pc->blk_begin = bb; pc->blk_end = be; pc->n_blk = sh.n_blk; pc->unit_end = unit_end;
      return true;
    }
    return false;
  }
};

// Per-column reduction over the warp's 32 lanes, transposing as it goes: every step exchanges half of the columns that are left
// with the lane across and combines the other half, so NC columns cost about NC shuffles.  Lane l returns column l % NC.
template <int NC, typename Op>
__device__ __forceinline__ float column_reduce(const float (&in)[NC], Op op) {
  const int lane = threadIdx.x & 31;
  float v[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) v[c] = in[c];
#pragma unroll
  for (int h = NC / 2; h >= 1; h >>= 1) {
    const bool hi = (lane & h) != 0;
#pragma unroll
    for (int e = 0; e < h; ++e) {
      const float other = __shfl_xor_sync(0xffffffffu, hi ? v[e] : v[e + h], h);
      v[e] = op(hi ? v[e + h] : v[e], other);
    }
  }
  float x = v[0];
#pragma unroll
  for (int h = NC; h < 32; h <<= 1) x = op(x, __shfl_xor_sync(0xffffffffu, x, h));
  return x;
}
// OR of a predicate over the 128 threads of a block parity.
__device__ __forceinline__ bool parity_any(int i, bool x) {
  uint32_t y;
  if (i == 0)
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, 1, 128, p;\n selp.u32 %0, 1, 0, q;\n}\n" : "=r"(y) : "r"(static_cast<uint32_t>(x)) : "memory");
  else
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, 2, 128, p;\n selp.u32 %0, 1, 0, q;\n}\n" : "=r"(y) : "r"(static_cast<uint32_t>(x)) : "memory");
  return y != 0;
}
// Two values in the pools' type.  A finite value past fp16's range (an average of values at its limit, rounded up) becomes the
// largest finite one; infinity stays infinity.
template <bool BF16>
__device__ __forceinline__ uint32_t pack_out(float a, float b) {
  if constexpr (BF16) {
    __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&v);
  } else {
    if (isinf(a) || isinf(b)) {
      const uint32_t lo = __half_as_ushort(isinf(a) ? __float2half_rn(a) : to_half_sat(a));
      const uint32_t hi = __half_as_ushort(isinf(b) ? __float2half_rn(b) : to_half_sat(b));
      return lo | (hi << 16);
    }
    return pack_half2(a, b);
  }
}

// Bits of the nodes j0 .. j0 + 31 (j0 may be negative) that a node sees.
__device__ __forceinline__ uint32_t node_bits(const TreeRows& r, int row, int node, int n_nodes, int j0) {
  if (j0 <= -32 || j0 >= n_nodes) return 0u;
  const int lo = max(j0, 0);
  uint64_t w = 0;
  if (r.mask != nullptr) {
    const uint64_t* m = r.mask + static_cast<size_t>(row) * r.mask_words;
    w = ld_dep_u64(m + (lo >> 6)) >> (lo & 63);
    if ((lo & 63) != 0 && (lo >> 6) + 1 < r.mask_words) w |= ld_dep_u64(m + (lo >> 6) + 1) << (64 - (lo & 63));
  } else if (node >= lo) {
    w = node - lo >= 63 ? ~0ull : (1ull << (node - lo + 1)) - 1;
  }
  if (n_nodes - lo < 64) w &= (1ull << (n_nodes - lo)) - 1;
  return static_cast<uint32_t>(w << (lo - j0));
}
// A 128-slot tile of K or V (D columns of one KV head) in shared memory, 128-byte swizzle.  From a contiguous context: 64-column
// halves of 128 rows, one copy each.  From pages: one copy per page, of both halves; a box of (64 columns, 8 rows, halves, 2
// row groups) lands as [row group][half][8 rows][128 bytes], so that row groups are one stride apart over all pages.  (With one copy
// per page and half the copies' issue was the limit: 115 clocks each, 32 a block.)
template <int D>
struct TileLayout {
  int half, group, mn_lbo;               // bytes: second 64 columns; next 8 rows; column-block distance of an MN-major operand
  __device__ __forceinline__ explicit TileLayout(bool paged)
      : half(paged ? 1024 : BLK * 128), group(paged ? D / 64 * 1024 : 1024), mn_lbo(D == 128 ? half : 0) {}
  __device__ __forceinline__ int row(int r, int h) const { return (r >> 3) * group + h * half + (r & 7) * 128; }
};
// Called by a whole warp.  With pages, `where` of lanes 0-7 is a page id each, else the pool row of the prompt's slot 0.  One lane issues
// all eight copies: a copy's operands are per-warp registers, so eight lanes with one each take turns anyway, and slower (48-node
// trees on 64 x 2500 slots 157 -> 140 us, weights of 64 tokens 67.8 -> 62.6 us).
template <int D>
__device__ __forceinline__ void load_tile(uint8_t* dst, const CUtensorMap* tm, uint64_t* bar, bool paged, int where, int head, int blk) {
  if (paged) {
    int page[BLK / PAGE_TOKENS];
#pragma unroll
    for (int p = 0; p < BLK / PAGE_TOKENS; ++p) page[p] = __shfl_sync(0xffffffffu, where, p);
    if (elect_one()) {
#pragma unroll
      for (int p = 0; p < BLK / PAGE_TOKENS; ++p) tma_load_4d(dst + p * (PAGE_TOKENS * D * 2), tm, bar, 0, 0, head * (D / 64), page[p] * 2);
    }
  } else if (elect_one()) {
#pragma unroll
    for (int h = 0; h < D / 64; ++h) tma_load_2d(dst + h * (BLK * 128), tm, bar, head * D + h * 64, where + blk * BLK);
  }
}
// `where` of load_tile: pages behind the prompt's last slot repeat its last page (masked either way).
__device__ __forceinline__ int tile_place(const KvView& kv, const SeqPart& p, int seq, int blk, int lane) {
  if (!kv.page_table) return ld_dep_s32(kv.ctx_start + seq);
  const int last = (p.ctx_len + max(p.n_nodes, 1) - 1) / PAGE_TOKENS;
  const int page = ld_dep_s32(kv.page_table + static_cast<size_t>(seq) * kv.pt_stride + min(blk * (BLK / PAGE_TOKENS) + (lane & 7), last));
  return static_cast<int>(min(static_cast<uint32_t>(page), 0x3fffffffu));       // twice that is outside any pool, and does not wrap
}

// K or V for load_tile.
inline int pool_map(CUtensorMap* out, const void* base, const KvView& kv, int64_t stride) {
  const uint64_t row = static_cast<uint64_t>(stride) * 2, cols = static_cast<uint64_t>(kv.n_kv_heads) * kv.head_dim;
  if (kv.page_table) {
    const uint64_t dims[4] = {64, 8, cols / 64, static_cast<uint64_t>(kv.n_slots) / 8};
    const uint64_t str[3] = {row, 128, 8 * row};
    const uint32_t box[4] = {64, 8, static_cast<uint32_t>(kv.head_dim / 64), 2};
    return encode_f16_map(out, base, 4, dims, str, box);
  }
  const uint64_t dims[2] = {cols, static_cast<uint64_t>(kv.n_slots)};
  const uint32_t box[2] = {64, static_cast<uint32_t>(BLK)};
  return encode_f16_map(out, base, 2, dims, &row, box);
}

// Rows of q as a 3-D map: one box is the query heads of a KV head for a tile of nodes.
inline int q_map(CUtensorMap* out, const void* q, const KvView& kv, int64_t stride, int n_q_heads, int n_rows, int tile_nodes) {
  const uint64_t dims[3] = {static_cast<uint64_t>(kv.head_dim), static_cast<uint64_t>(n_q_heads), static_cast<uint64_t>(n_rows)};
  const uint64_t str[2] = {static_cast<uint64_t>(kv.head_dim) * 2, static_cast<uint64_t>(stride) * 2};
  const uint32_t box[3] = {64u, static_cast<uint32_t>(n_q_heads / kv.n_kv_heads), static_cast<uint32_t>(tile_nodes)};
  return encode_f16_map(out, q, 3, dims, str, box);
}

// Does a node see any node at all.
__device__ __noinline__ bool sees_a_node(const TreeRows& r, int row, int node, int n_nodes) {
  bool any = false;
#pragma unroll 1
  for (int w = 0; w < n_nodes && !any; w += 32) any = node_bits(r, row, node, n_nodes, w) != 0;
  return any;
}
// One 64-bit word of what a node sees (bits of nodes past the prompt's last are whatever the caller wrote).
__device__ __forceinline__ uint64_t node_word(const TreeRows& r, int row, int node, int w) {
  if (r.mask) return ld_dep_u64(r.mask + static_cast<size_t>(row) * r.mask_words + w);
  return node < 64 * w ? 0ull : node - 64 * w >= 63 ? ~0ull : (1ull << (node - 64 * w + 1)) - 1;
}

}  // namespace
}  // namespace pc
