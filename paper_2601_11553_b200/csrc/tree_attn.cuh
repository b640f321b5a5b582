// What the two forms of the tree attention share (attn_tree.cu: up to 128 rows a tile; attn_narrow.cu: up to 16).
#pragma once
#include "tree_common.cuh"

namespace pc {

struct MergeRecord {             // written by the CTA that has a cut unit's first part
  int32_t n_parts;               // 0: none
  int32_t row0, n_rows;          // first global row of the tile, valid tile rows
  int32_t head0;
  int32_t pad[4];
};

struct TreeParams {
  KvView kv;
  TreeRows rows;
  int32_t n_q_heads, group, tile_nodes, small, over, whole;
  float scale_log2;
  void* out;
  int64_t out_stride;
  float* lse;
  int* err_word;
  MergeRecord* merges;
  float *partial_ml, *partial_o;
};

// Workspace places of a TreeParams; launches one of the two forms, then (attn_tree.cu) the merge.
int launch_narrow_attention(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const TreeParams& p, int n_ctas,
                            cudaStream_t s);
constexpr int NARROW_ROWS = 16;

namespace {

__device__ __forceinline__ Shape tree_shape(const TreeParams& a, const SeqPart& p) {
  if (p.n_nodes == 0) return Shape{0, 0, 1, 0};
  const int units = (p.n_nodes + a.tile_nodes - 1) / a.tile_nodes * a.kv.n_kv_heads, n_blk = (p.ctx_len + p.n_nodes + BLK - 1) / BLK;
  // units that are not to be cut look like one block that costs as much
  return a.whole ? Shape{units, 1, n_blk, a.over} : Shape{units, n_blk, 1, a.over};
}
struct Item {
  int seq, ctx_len, n_nodes;     // the prompt: its context slots and nodes
  int row0, node0, n_rows;       // the tile: first global row, first node, valid tile rows
  int g, blk_begin, blk_end, n_blk;
  int unit_end;
};
// The last CTA with a part of a unit: where its last cost position lies.
__device__ __forceinline__ int last_cta(const Span& s, int unit_end) {
  return static_cast<int>(static_cast<uint64_t>((s.begin + unit_end) * s.n_ctas - 1) / static_cast<uint64_t>(s.total));
}
__device__ __forceinline__ bool next_item(Cursor& cur, const TreeParams& a, Item* it) {
  Piece pc;
  if (!cur.next(a.rows, [&](const SeqPart& p) { return tree_shape(a, p); }, &pc)) return false;
  // the tiles of one KV head follow each other: they share K and V in L2
  const int tiles = (pc.part.n_nodes + a.tile_nodes - 1) / a.tile_nodes, tile = pc.unit % tiles;
  it->seq = pc.seq; it->ctx_len = pc.part.ctx_len; it->n_nodes = pc.part.n_nodes;
  it->node0 = tile * a.tile_nodes;
  it->row0 = pc.part.row0 + it->node0;
  it->n_rows = min(a.tile_nodes, pc.part.n_nodes - it->node0) * a.group;
  it->g = pc.unit / tiles;
  it->blk_begin = pc.blk_begin; it->blk_end = pc.blk_end; it->n_blk = pc.n_blk; it->unit_end = pc.unit_end;
  if (a.whole) it->blk_end = it->n_blk = (it->ctx_len + it->n_nodes + BLK - 1) / BLK;
  return true;
}
// Bits of the 32 slots from slot0 on that a node sees.
__device__ __forceinline__ uint32_t slot_bits(const TreeRows& r, const Item& it, int row, int node, int slot0) {
  const int in_ctx = it.ctx_len - slot0;
  if (in_ctx >= 32) return 0xffffffffu;
  return (in_ctx > 0 ? (1u << in_ctx) - 1 : 0u) | node_bits(r, row, node, it.n_nodes, -in_ctx);
}

template <bool BF16>
__device__ __forceinline__ float elem(uint32_t bits16) {
  if constexpr (BF16) return __uint_as_float(bits16 << 16);
  else return __half2float(__ushort_as_half(static_cast<unsigned short>(bits16)));
}

// ---------------------------------------------------------------------------------------------------- attention: shared roles
// The running reference lies P_HEADROOM (base 2) below the largest score that set it and is raised when a block exceeds that score by
// RESCALE_THRESHOLD: the largest weight P of a row is between 2^P_HEADROOM and 2^(P_HEADROOM + RESCALE_THRESHOLD).  A 16-bit P has to hold the
// small weights of a long context, which together may be all of the result (a few heavy slots with values near 0): fp16 rounds what is
// below 2^-14 to multiples of 2^-24, so with the largest at 2^7 or more a weight is off by at most 2^-32 of it (without the headroom 2^-25: of
// 2500 slots under two of a score 17.5 higher nothing was left), and at 2^15 it still fits.  bf16 has fp32's exponents.
constexpr float RESCALE_THRESHOLD = 8.0f;
template <bool BF16> constexpr float P_HEADROOM = BF16 ? 0.f : 7.f;
// Least cost of an attention span (in blocks; a unit's own cost counts).  4 -> 2: 26-node trees on one prompt of 2112 slots 14.4 -> 12.7 us,
// one token on 1000 slots 10.9 -> 9.6; 1: 13.2 and 9.5.
constexpr int MIN_SPAN = 2;
constexpr int MAX_STAGES = 8;
constexpr int FLAGS = 8;                        // items a `bad V` flag lives for: more than the roles can be apart
constexpr int MASK_WORDS = 4;                   // 256 nodes

// Shared-memory places and barriers of the K/V ring and the Q slots.
struct Pipe {
  uint8_t* q_smem;
  int q_slot_bytes, q_half_bytes;
  uint8_t* ring;
  uint64_t *q_full, *q_empty, *full, *empty, *raw;
  int* bad_v;                                   // [FLAGS][2]
  uint64_t* node_mask;                          // [Q slot][node][MASK_WORDS] or nullptr
};

// CALLS: the wait's slow path is a function, which keeps the code small; the 128-row form has no registers left for calls.
template <bool CALLS>
__device__ __forceinline__ bool role_wait(uint64_t* bar, uint32_t parity, int* err_word, int code) {
  if constexpr (CALLS) return bar_wait(bar, parity, err_word, code);
  else return mbar_wait(bar, parity, err_word, code);
}

// Copies (one warp): Q tiles, and K and V tiles in the order the MMAs take them, K0 K1 V0 K2 V1 K3 ...
template <int D, int STAGES, int QSLOTS, bool CALLS>
__device__ __forceinline__ void copy_role(const TreeParams& a, const Pipe& pipe, Cursor& cur, const Span& span, const CUtensorMap* tmQ,
                                          const CUtensorMap* tmK, const CUtensorMap* tmV, int* cta_failed) {
  constexpr int HALVES = D / 64, TILE_BYTES = HALVES * BLK * 128;
  const int lane = threadIdx.x & 31;
  uint32_t n_item = 0, st = 0, st_phase = 0, n_raw = 0;
  MergeRecord rec{};
  bool ok = true;
  Item it{};
  while (ok && next_item(cur, a, &it)) {
    const int nb = it.blk_end - it.blk_begin, qs = n_item % QSLOTS;
    ok = __all_sync(0xffffffffu, role_wait<CALLS>(&pipe.q_empty[qs], ((n_item / QSLOTS) & 1u) ^ 1u, a.err_word, DEV_ERR_ATTN_PRODUCER));
    if (!ok) break;
    if (elect_one()) {
      mbar_arrive_expect_tx(&pipe.q_full[qs], HALVES * a.tile_nodes * a.group * 128);
      for (int h = 0; h < HALVES; ++h)
        tma_load_3d(pipe.q_smem + qs * pipe.q_slot_bytes + h * pipe.q_half_bytes, tmQ, &pipe.q_full[qs], h * 64, it.g * a.group, it.row0);
    }
    __syncwarp();
    const SeqPart part{it.row0, it.n_nodes, it.ctx_len};
    auto load = [&](bool is_k, int j, int where) {
      ok = __all_sync(0xffffffffu, role_wait<CALLS>(&pipe.empty[st], st_phase ^ 1u, a.err_word, DEV_ERR_ATTN_PRODUCER));
      if (!ok) return;
      const int blk = it.blk_begin + j;
      // a tile that has to be cleaned lands on a barrier of the cleaning warps; they then complete `full` in its place
      const bool clean = !is_k && (blk + 1) * BLK > it.ctx_len;
      uint64_t* bar = clean ? &pipe.raw[n_raw++ % STAGES] : &pipe.full[st];
      if (elect_one()) {
        mbar_arrive_expect_tx(bar, TILE_BYTES);
        if (!clean) mbar_arrive(bar);
      }
      __syncwarp();
      load_tile<D>(pipe.ring + st * TILE_BYTES, is_k ? tmK : tmV, bar, a.kv.page_table != nullptr, where, it.g, blk);
      if (++st == STAGES) { st = 0; st_phase ^= 1u; }
    };
    // where[n]: the places of block j + n.  Page ids are asked for a block ahead, once for K and V.
    int where[4] = {0, 0, tile_place(a.kv, part, it.seq, it.blk_begin, lane), 0};
#pragma unroll 1
    for (int j = -2; j < nb && ok; ++j) {
      where[3] = where[2];
      if (a.kv.page_table && j + 3 < nb) where[3] = tile_place(a.kv, part, it.seq, it.blk_begin + j + 3, lane);
      if (j >= 0) load(false, j, where[0]);
      if (ok && j + 2 < nb) load(true, j + 2, where[2]);
      where[0] = where[1]; where[1] = where[2]; where[2] = where[3];
    }
    if (it.blk_begin == 0 && it.blk_end < it.n_blk) {              // the rest of this unit is other CTAs' work
      rec.n_parts = last_cta(span, it.unit_end) - static_cast<int>(blockIdx.x) + 1;
      rec.row0 = it.row0; rec.n_rows = it.n_rows; rec.head0 = it.g * a.group;
    }
    ++n_item;
  }
  if (!ok) *cta_failed = 1;
  if (lane == 0) a.merges[blockIdx.x] = rec;
}

// Warps 10-11: V tiles that hold drafted or no slots.  Zeros behind the prompt's last slot, and where a drafted V is not finite (with
// the flag raised).  MASKS: they also put the nodes' masks beside a Q tile whose piece has drafted slots, and then arrive on q_full.
template <int D, int STAGES, bool BF16, bool MASKS, bool CALLS>
__device__ __forceinline__ void clean_role(const TreeParams& a, const Pipe& pipe, Cursor& cur, int* cta_failed) {
  constexpr int HALVES = D / 64, TILE_BYTES = BLK * D * 2;
  const TileLayout<D> tl(a.kv.page_table != nullptr);
  const int tid = threadIdx.x - 320, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t n_item = 0, n_tile = 0, n_raw = 0;
  bool ok = true;
  Item it{};
  while (ok && next_item(cur, a, &it)) {
    const int nb = it.blk_end - it.blk_begin;
    int* flag = pipe.bad_v + (n_item % FLAGS) * 2 + warp - 10;       // read at the end of the item that set it, long before its next use
    if (lane == 0) *flag = 0;
    __syncwarp();
    if constexpr (MASKS) {
      const int qs = n_item & 1;
      ok = __all_sync(0xffffffffu, role_wait<CALLS>(&pipe.q_empty[qs], ((n_item >> 1) & 1u) ^ 1u, a.err_word, DEV_ERR_ATTN_CORR));
      if (!ok) break;
      if (it.blk_end * BLK > it.ctx_len) {
        const int nodes = it.n_rows / a.group, words = (it.n_nodes + 63) / 64;
#pragma unroll 1
        for (int e = tid; e < nodes * words; e += 64)
          pipe.node_mask[(qs * NARROW_ROWS + e / words) * MASK_WORDS + e % words] = node_word(a.rows, it.row0 + e / words, it.node0 + e / words, e % words);
      }
      __syncwarp();
      if (elect_one()) mbar_arrive(&pipe.q_full[qs]);
    }
    // the tiles' order in the ring: K0 [K1] V0 [K2] V1 ...
    uint32_t tile = n_tile + (nb > 1 ? 2 : 1);
#pragma unroll 1
    for (int j = 0; j < nb; ++j) {
      const int blk = it.blk_begin + j;
      if ((blk + 1) * BLK > it.ctx_len) {
        const int st = tile % STAGES;
        ok = __all_sync(0xffffffffu, role_wait<CALLS>(&pipe.raw[n_raw % STAGES], (n_raw / STAGES) & 1u, a.err_word, DEV_ERR_ATTN_CORR));
        if (!ok) break;
        ++n_raw;
        uint8_t* v = pipe.ring + st * TILE_BYTES;
        const int r0 = max(it.ctx_len - blk * BLK, 0), r_end = it.ctx_len + it.n_nodes - blk * BLK;
        bool bad = false;
        // thread t takes 16-byte vector t % 8 (as stored; the swizzle only permutes a row's vectors) of rows t / 8, t / 8 + 8 ...
#pragma unroll 1
        for (int r = r0 + (tid >> 3); r < BLK; r += 8) {
#pragma unroll
          for (int h = 0; h < HALVES; ++h) {
            uint4* p = reinterpret_cast<uint4*>(v + tl.row(r, h) + (tid & 7) * 16);
            if (r >= r_end) {
              *p = make_uint4(0, 0, 0, 0);
            } else {
              const uint4 x = *p;
              uint32_t w[4] = {x.x, x.y, x.z, x.w};
              constexpr uint32_t E = BF16 ? 0x7f80u : 0x7c00u;             // all exponent bits set: infinity or NaN
              bool any = false;
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                if ((w[q] & E) == E) { w[q] &= 0xffff0000u; any = true; }
                if (((w[q] >> 16) & E) == E) { w[q] &= 0x0000ffffu; any = true; }
              }
              if (any) { *p = make_uint4(w[0], w[1], w[2], w[3]); bad = true; }
            }
          }
        }
        if (bad) *reinterpret_cast<volatile int*>(flag) = 1;
        fence_proxy_async_smem();                        // the MMA reads the tile through the async proxy
        __syncwarp();
        if (elect_one()) mbar_arrive(&pipe.full[st]);
      }
      tile += j + 2 < nb ? 2 : 1;
    }
    n_tile += 2 * nb;
    ++n_item;
  }
  if (!ok) *cta_failed = 1;
}

}  // namespace
}  // namespace pc
