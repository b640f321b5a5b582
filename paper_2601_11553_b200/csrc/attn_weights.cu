// Running attention weights of a cache's slots: w' = decay * w + the sum over rows and heads of exp(scale * q . k - lse), on tcgen05.
//
// The scores are formed transposed, S^T = K Q^T: a block of 128 slots is the MMA's M side and the rows (node, query head of
// one KV head, packed as in the attention) its N side, so a slot is a TMEM lane, i.e. a thread, and the sum over the rows
// is that thread's own: nothing is exchanged between threads, a slot's weight is written by exactly one, the order of its sum
// never changes and no atomic is needed.  Only as many columns as there are rows (rounded up to 16) are computed.
//
// Bounds.  A block costs 32 KB of K (head size 128, 0.75 us of an SM's share of the HBM), at most 4.2 MFLOP (0.37 us) and
// 16 K exponentials (0.55 us): bound by reading K once, so as in the attention the copies are what is kept running.  Measured: one
// token on each of 64 x 2500 slots in pages 62.8 us (floor 52.4), the accepted half of 33 nodes on 2 x 33024 slots 31.2 us (21.7: some
// 9 us are the call's start and the blocks of the longest share), one token on 2112 slots 7.4 us.
//
// Schedule as in the attention (spans of the batch's blocks), but a block belongs to one CTA: nothing is merged.
// One CTA per SM, 384 threads: warp 8 copies (K ring, Q ring of two tiles), warp 9 issues the MMAs, warps 10-11 put the rows'
// lse beside each Q tile (and, where a mask says which rows count, fetch those rows alone: of a drafted tree few are accepted),
// warps 0-3 sum the even blocks and warps 4-7 the odd ones, each from two TMEM buffers in turn.
// One tile of rows stays in shared memory for the whole piece; of several, each is copied again for every block (L2).
#include <algorithm>

#include "tree_common.cuh"

namespace pc {
namespace {

constexpr int K_RING = 96 * 1024;              // 128 KB: 64 tokens x 2500 slots 62.9 -> 64.2 us, 33 nodes x 33024 31.2 -> 30.7; 64 KB: 71.8 and 35.4
constexpr int Q_TILE = 32 * 1024;
constexpr int WEIGHTS_SMEM = K_RING + 2 * Q_TILE + 1024;
constexpr int MAX_STAGES = 8;
constexpr int MASK_WORDS = 4;                    // 256 nodes
constexpr int UNIT_COST = 2;                     // of a unit beside its blocks, in blocks
constexpr int MIN_SPAN = UNIT_COST + 1;

struct WeightParams {
  KvView kv;
  TreeRows rows;
  int32_t n_q_heads, group, tile_nodes, small;
  float scale, decay;
  const void* q;
  int64_t q_stride;
  const float* lse;
  const uint8_t* use;
  const float* w_in;
  float* w_out;
  int64_t w_stride;
  int* err_word;
};

// Which of 32 nodes of a prompt count (a whole warp asks).
__device__ __forceinline__ uint32_t used_word(const WeightParams& a, const SeqPart& p, int n0) {
  const int lane = threadIdx.x & 31;
  return __ballot_sync(0xffffffffu, n0 + lane < p.n_nodes && ld_dep_u8(a.use + p.row0 + n0 + lane) != 0);
}
// How many nodes of a prompt count, and which of the first 64.  Those flags are asked for together: a call's first tile waits for
// this, and every round trip is half a microsecond.
__device__ __forceinline__ int used_nodes(const WeightParams& a, const SeqPart& p, uint32_t (&bits)[2]) {
  if (!a.use) return p.n_nodes;
  const int lane = threadIdx.x & 31;
  const uint8_t* flags = a.use + p.row0 + lane;
  const uint32_t lo = lane < p.n_nodes ? ld_dep_u8(flags) : 0u, hi = lane + 32 < p.n_nodes ? ld_dep_u8(flags + 32) : 0u;
  bits[0] = __ballot_sync(0xffffffffu, lo != 0);
  bits[1] = __ballot_sync(0xffffffffu, hi != 0);
  int n = __popc(bits[0]) + __popc(bits[1]);
#pragma unroll 1
  for (int n0 = 64; n0 < p.n_nodes; n0 += 32) n += __popc(used_word(a, p, n0));
  return n;
}
__device__ __forceinline__ int used_nodes(const WeightParams& a, const SeqPart& p) {
  uint32_t bits[2];
  return used_nodes(a, p, bits);
}
__device__ __forceinline__ int n_tiles(const WeightParams& a, int nodes) { return (nodes + a.tile_nodes - 1) / a.tile_nodes; }
__device__ __forceinline__ Shape weight_shape(const WeightParams& a, const SeqPart& p) {
  const int len = p.ctx_len + p.n_nodes;
  if (len == 0) return Shape{0, 0, 1, 0};
  return Shape{a.kv.n_kv_heads, (len + BLK - 1) / BLK, max(n_tiles(a, p.n_nodes), 1), UNIT_COST};
}
__device__ __forceinline__ bool next_piece(Cursor& cur, const WeightParams& a, Piece* pc) {
  return cur.next(a.rows, [&](const SeqPart& p) { return weight_shape(a, p); }, pc);
}

template <int D, bool BF16>
__global__ void __launch_bounds__(TREE_THREADS, 1)
attention_weights_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                         const __grid_constant__ WeightParams a) {
  constexpr int HALVES = D / 64;
  constexpr int HALF_BYTES = BLK * 128;
  constexpr int TILE_BYTES = HALVES * HALF_BYTES;
  constexpr int STAGES = K_RING / TILE_BYTES;
  static_assert(STAGES <= MAX_STAGES, "");
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t q_full[2], q_empty[2], full[MAX_STAGES], empty[MAX_STAGES], s_full[2][2], s_empty[2][2];
  __shared__ __align__(16) float row_lse[2][BLK];          // per Q tile: the rows' lse (0 where a row does not count)
  __shared__ uint32_t row_ok[2][4];                        // which rows count
  __shared__ uint8_t node_list[2][BLK];                    // the tile's nodes
  __shared__ uint64_t node_mask[2][BLK][MASK_WORDS];       // and, where a piece has drafted slots, what the tile's nodes see of them
  __shared__ Span shared_span;
  __shared__ int64_t warp_sums[TREE_THREADS / 32];
  __shared__ uint32_t tmem_slot;
  __shared__ int cta_failed;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* q_smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = q_smem + 2 * Q_TILE;

  if (threadIdx.x == 0) {
    cta_failed = 0;
    for (int i = 0; i < STAGES; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 3);          // the copy and the two warps that fill row_lse
      mbar_init(&q_empty[i], 9);         // the MMAs and the eight summing warps
      for (int j = 0; j < 2; ++j) { mbar_init(&s_full[i][j], 1); mbar_init(&s_empty[i][j], 4); }
    }
    fence_mbar_init();
  }
  if (warp == 9) {
    tmem_alloc<512>(&tmem_slot);
    tmem_relinquish();
  }
  if (warp == 8 && lane == 0) { prefetch_tmap(&tmQ); prefetch_tmap(&tmK); }
  pdl_launch_dependents();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  pdl_wait();                          // lengths, tables, Q, K and V may come from the kernel before
  const Span span = make_span(a.rows, MIN_SPAN, a.small, &shared_span, warp_sums, [&](const SeqPart& p) { return weight_shape(a, p); });
  const uint32_t tmem = tmem_slot;
  Cursor cur(span);
  Piece pc{};
  bool ok = true;
  uint32_t n_q = 0;                      // Q tiles so far: tile n is in slot n & 1

  if (warp == 8) {
    // ------------------------------------------------------------ copies
    uint32_t n_tile = 0;
    while (ok && next_piece(cur, a, &pc)) {
      const int nodes = used_nodes(a, pc.part), tiles = n_tiles(a, nodes);
      if (tiles == 0) continue;          // no rows: the weights only decay
      auto load_q = [&](int t) {
        const int qs = n_q & 1;
        ok = __all_sync(0xffffffffu, bar_wait(&q_empty[qs], ((n_q >> 1) & 1u) ^ 1u, a.err_word, DEV_ERR_ATTN_PRODUCER));
        if (!ok) return;
        ++n_q;
        if (a.use) {                     // the lse warps fetch the rows that count
          if (elect_one()) mbar_arrive(&q_full[qs]);
        } else if (elect_one()) {
          mbar_arrive_expect_tx(&q_full[qs], HALVES * a.tile_nodes * a.group * 128);
          for (int h = 0; h < HALVES; ++h)
            tma_load_3d(q_smem + qs * Q_TILE + h * HALF_BYTES, &tmQ, &q_full[qs], h * 64, pc.unit * a.group, pc.part.row0 + t * a.tile_nodes);
        }
        __syncwarp();
      };
      int next = tile_place(a.kv, pc.part, pc.seq, pc.blk_begin, lane);          // page ids are asked for a tile ahead
      if (tiles == 1) load_q(0);
      for (int blk = pc.blk_begin; blk < pc.blk_end && ok; ++blk) {
        const int st = n_tile % STAGES;
        const int where = next;
        if (a.kv.page_table && blk + 1 < pc.blk_end) next = tile_place(a.kv, pc.part, pc.seq, blk + 1, lane);
        ok = __all_sync(0xffffffffu, bar_wait(&empty[st], ((n_tile / STAGES) & 1u) ^ 1u, a.err_word, DEV_ERR_ATTN_PRODUCER));
        if (!ok) break;
        ++n_tile;
        if (elect_one()) mbar_arrive_expect_tx(&full[st], TILE_BYTES);
        __syncwarp();
        load_tile<D>(ring + st * TILE_BYTES, &tmK, &full[st], a.kv.page_table != nullptr, where, pc.unit, blk);
        for (int t = 0; t < tiles && tiles > 1 && ok; ++t) load_q(t);
      }
    }
  } else if (warp == 9) {
    // ------------------------------------------------------------ MMA issuer
    // the whole warp walks; one lane issues
    const TileLayout<D> tl(a.kv.page_table != nullptr);
    uint32_t st = 0, st_phase = 0, n_s0 = 0, n_s1 = 0;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (ok) ok = __all_sync(0xffffffffu, bar_wait(bar, parity, a.err_word, DEV_ERR_ATTN_MMA));
    };
    while (ok && next_piece(cur, a, &pc)) {
      const int nodes = used_nodes(a, pc.part), tiles = n_tiles(a, nodes);
      if (tiles == 0) continue;
      if (tiles == 1) wait(&q_full[n_q & 1], (n_q >> 1) & 1u);
      for (int blk = pc.blk_begin; blk < pc.blk_end && ok; ++blk) {
        const int i = (blk - pc.blk_begin) & 1;
        wait(&full[st], st_phase);
        const uint64_t k_desc = make_smem_desc_sw128(smem_u32(ring + st * TILE_BYTES), 16, tl.group);
        for (int t = 0; t < tiles && ok; ++t) {
          const int qs = n_q & 1;
          if (tiles > 1) wait(&q_full[qs], (n_q >> 1) & 1u);
          const uint32_t n = i == 0 ? n_s0++ : n_s1++;
          const int buf = n & 1;
          wait(&s_empty[i][buf], ((n >> 1) & 1u) ^ 1u);
          if (!ok) break;
          tc_fence_after_sync();
          const int cols = (min(a.tile_nodes, nodes - t * a.tile_nodes) * a.group + 15) & ~15;
          const uint32_t idesc = make_idesc_f16(BLK, cols, BF16 ? 1 : 0, 0, 0);
          const uint64_t q_desc = make_smem_desc_sw128(smem_u32(q_smem + qs * Q_TILE), 16, 1024);
          const bool q_done = tiles > 1 || blk + 1 == pc.blk_end;
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              umma_ss(tmem + (i * 2 + buf) * BLK, k_desc + (((kk >> 2) * tl.half + (kk & 3) * 32) >> 4),
                      q_desc + (((kk >> 2) * HALF_BYTES + (kk & 3) * 32) >> 4), idesc, kk != 0);
            umma_commit(&s_full[i][buf]);
            if (q_done) umma_commit(&q_empty[qs]);
            if (t + 1 == tiles) umma_commit(&empty[st]);
          }
          __syncwarp();
          if (q_done) ++n_q;
        }
        if (++st == STAGES) { st = 0; st_phase ^= 1u; }
      }
    }
  } else if (warp >= 10) {
    // ------------------------------------------------------------ the rows' lse
    const int tid = threadIdx.x - 320;
    while (ok && next_piece(cur, a, &pc)) {
      uint32_t used[2];
      const int nodes = used_nodes(a, pc.part, used), tiles = n_tiles(a, nodes);
      const int loads = tiles == 1 ? 1 : tiles * (pc.blk_end - pc.blk_begin);
      for (int x = 0; x < loads && ok; ++x) {
        const int t = tiles == 1 ? 0 : x % tiles;
        const int qs = n_q & 1;
        ok = __all_sync(0xffffffffu, bar_wait(&q_empty[qs], ((n_q >> 1) & 1u) ^ 1u, a.err_word, DEV_ERR_ATTN_CORR));
        if (!ok) break;
        ++n_q;
        const int tile_n = min(a.tile_nodes, nodes - t * a.tile_nodes), n_rows = tile_n * a.group;
        // the tile's nodes: those that count, in order (both warps write the same)
        if (a.use) {
          int before = -t * a.tile_nodes;
#pragma unroll 1
          for (int n0 = 0; n0 < pc.part.n_nodes; n0 += 32) {
            const uint32_t all = n0 == 0 ? used[0] : n0 == 32 ? used[1] : used_word(a, pc.part, n0);
            const int at = before + __popc(all & ((1u << lane) - 1));
            if ((all >> lane & 1u) && at >= 0 && at < tile_n) node_list[qs][at] = static_cast<uint8_t>(n0 + lane);
            before += __popc(all);
          }
        } else {
#pragma unroll 1
          for (int e = lane; e < tile_n; e += 32) node_list[qs][e] = static_cast<uint8_t>(t * a.tile_nodes + e);
        }
        __syncwarp();
        float z[2];                                        // on their way while the rows are fetched
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int r = k * 64 + tid;
          z[k] = -INFINITY;
          if (r < n_rows) z[k] = ld_dep_f32(a.lse + static_cast<size_t>(pc.part.row0 + node_list[qs][r / a.group]) * a.n_q_heads + pc.unit * a.group + r % a.group);
        }
        const int words = (pc.part.n_nodes + 63) / 64, n_mask = pc.blk_end * BLK > pc.part.ctx_len ? tile_n * words : 0;
        auto mask_word = [&](int e) {
          const int node = node_list[qs][e / words];
          return node_word(a.rows, pc.part.row0 + node, node, e % words);
        };
        const uint64_t first_mask = tid < n_mask ? mask_word(tid) : 0;
        if (a.use) {                                       // the rows, in the layout a copy would give them
          constexpr int VECS = D / 8, BATCH = 8;
          uint8_t* dst = q_smem + qs * Q_TILE;
          const int total = n_rows * VECS;
#pragma unroll 1
          for (int e0 = tid; e0 < total; e0 += 64 * BATCH) {
            uint4 row[BATCH];
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
              const int e = e0 + u * 64, r = e / VECS;
              if (e >= total) break;
              const int64_t at = static_cast<int64_t>(pc.part.row0 + node_list[qs][r / a.group]) * a.q_stride + (pc.unit * a.group + r % a.group) * D + e % VECS * 8;
              row[u] = ld_dep_v4(static_cast<const unsigned short*>(a.q) + at);
            }
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
              const int e = e0 + u * 64, r = e / VECS, v = e % VECS;
              if (e >= total) break;
              *reinterpret_cast<uint4*>(dst + (v >> 3) * HALF_BYTES + r * 128 + (((v & 7) ^ (r & 7)) << 4)) = row[u];
            }
          }
          fence_proxy_async_smem();
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t counts = __ballot_sync(0xffffffffu, z[k] != -INFINITY);
          row_lse[qs][k * 64 + tid] = z[k] != -INFINITY ? z[k] : 0.f;
          if (lane == 0) row_ok[qs][k * 2 + warp - 10] = counts;
        }
        if (tid < n_mask) node_mask[qs][tid / words][tid % words] = first_mask;
        for (int e = tid + 64; e < n_mask; e += 64) node_mask[qs][e / words][e % words] = mask_word(e);
        __syncwarp();
        if (elect_one()) mbar_arrive(&q_full[qs]);
      }
    }
  } else {
    // ------------------------------------------------------------ sums (warps 0-7): thread = slot of the block
    const int i = warp >> 2, quarter = warp & 3;
    const int r = quarter * 32 + lane;
    const uint32_t t_s = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + i * 2 * BLK;
    uint32_t n_s = 0;
    while (ok && next_piece(cur, a, &pc)) {
      const int nodes = used_nodes(a, pc.part), tiles = n_tiles(a, nodes), len = pc.part.ctx_len + pc.part.n_nodes;
      float* w_row = a.w_out + (static_cast<size_t>(pc.seq) * a.kv.n_kv_heads + pc.unit) * a.w_stride;
      const float* in_row = a.w_in ? a.w_in + (static_cast<size_t>(pc.seq) * a.kv.n_kv_heads + pc.unit) * a.w_stride : nullptr;
      for (int blk = pc.blk_begin; blk < pc.blk_end && ok; ++blk) {
        const bool mine = ((blk - pc.blk_begin) & 1) == i;
        const int slot = blk * BLK + r;
        float before = 0.f, sum0 = 0.f, sum1 = 0.f;
        if (mine && in_row && slot < len) before = ld_dep_f32(in_row + slot);
        for (int t = 0; t < tiles; ++t) {
          const int qs = n_q & 1;
          if (tiles > 1 || blk == pc.blk_begin) {
            ok = __all_sync(0xffffffffu, bar_wait(&q_full[qs], (n_q >> 1) & 1u, a.err_word, DEV_ERR_ATTN_SOFTMAX));
            if (!ok) break;
          }
          if (mine) {
            const int buf = n_s & 1;
            ok = __all_sync(0xffffffffu, bar_wait(&s_full[i][buf], (n_s >> 1) & 1u, a.err_word, DEV_ERR_ATTN_SOFTMAX));
            if (!ok) break;
            ++n_s;
            tc_fence_after_sync();
            const int n_rows = min(a.tile_nodes, nodes - t * a.tile_nodes) * a.group;
            const int n_ch = (n_rows + 15) / 16;
            // 16 columns at a time without a branch among them (a branch per four columns ran at half the speed: every group then waits
            // out its own latencies); the next 16 are on their way from TMEM meanwhile
            auto add = [&](const uint32_t (&s)[16], int ch) {
              uint32_t bits = row_ok[qs][ch >> 1] >> (ch & 1) * 16;
              if (slot >= pc.part.ctx_len) {           // a drafted slot: which of the rows see it
                const int node = slot - pc.part.ctx_len;
                uint32_t seen = 0;
                if (slot < len) {
                  const uint64_t* m = &node_mask[qs][0][node >> 6];
#pragma unroll 4
                  for (int c = 0; c < min(16, n_rows - ch * 16); ++c)
                    seen |= static_cast<uint32_t>((m[(ch * 16 + c) / a.group * MASK_WORDS] >> (node & 63)) & 1u) << c;
                }
                bits &= seen;
              }
              __syncwarp();
#pragma unroll
              for (int c = 0; c < 16; c += 4) {
                const float4 z = *reinterpret_cast<const float4*>(&row_lse[qs][ch * 16 + c]);
                // scale * s - lse in one rounding, then to base 2
                const float e0 = fast_exp2(fmaf(__uint_as_float(s[c]), a.scale, -z.x) * LOG2E);
                const float e1 = fast_exp2(fmaf(__uint_as_float(s[c + 1]), a.scale, -z.y) * LOG2E);
                const float e2 = fast_exp2(fmaf(__uint_as_float(s[c + 2]), a.scale, -z.z) * LOG2E);
                const float e3 = fast_exp2(fmaf(__uint_as_float(s[c + 3]), a.scale, -z.w) * LOG2E);
                sum0 += bits & (1u << c) ? e0 : 0.f;
                sum1 += bits & (2u << c) ? e1 : 0.f;
                sum0 += bits & (4u << c) ? e2 : 0.f;
                sum1 += bits & (8u << c) ? e3 : 0.f;
              }
            };
            uint32_t sa[16], sb[16];
            tmem_ld_32x16(t_s + buf * BLK, sa);
#pragma unroll 1
            for (int ch = 0; ch < n_ch; ch += 2) {
              tmem_wait_ld();
              if (ch + 1 < n_ch) tmem_ld_32x16(t_s + buf * BLK + ch * 16 + 16, sb);
              add(sa, ch);
              if (ch + 1 >= n_ch) break;
              tmem_wait_ld();
              if (ch + 2 < n_ch) tmem_ld_32x16(t_s + buf * BLK + ch * 16 + 32, sa);
              add(sb, ch + 1);
            }
            tc_fence_before_sync();
            __syncwarp();
            if (elect_one()) mbar_arrive(&s_empty[i][buf]);
          }
          if (tiles > 1 || blk + 1 == pc.blk_end) {
            __syncwarp();
            if (elect_one()) mbar_arrive(&q_empty[qs]);
            ++n_q;
          }
        }
        if (ok && mine && slot < len) w_row[slot] = in_row ? fmaf(a.decay, before, sum0 + sum1) : sum0 + sum1;
      }
    }
  }
  if (!ok) cta_failed = 1;

  // ---------------------------------------------------------------- teardown
  tc_fence_before_sync();
  __syncthreads();
  if (cta_failed) {             // let this CTA's bulk copies land before its shared memory is released
    if (threadIdx.x == 0) {
      const unsigned long long t0 = globaltimer_ns();
      while (globaltimer_ns() - t0 < DRAIN_LIMIT_NS) { }
    }
    __syncthreads();
  }
  if (warp == 9) {
    tc_fence_after_sync();
    tmem_dealloc<512>(tmem);
  }
}

template <int D, bool BF16>
int launch_weights(const CUtensorMap& q, const CUtensorMap& k, const WeightParams& p, int n_ctas, cudaStream_t s) {
  static bool set[MAX_DEVICES] = {};
  const int dev = current_device_slot();
  if (!set[dev]) {
    if (cudaFuncSetAttribute(attention_weights_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, WEIGHTS_SMEM) != cudaSuccess) return -1;
    set[dev] = true;
  }
  return launch_pdl(attention_weights_kernel<D, BF16>, dim3(n_ctas), dim3(TREE_THREADS), WEIGHTS_SMEM, s, q, k, p) == cudaSuccess ? 0 : -1;
}

int most_tiles(const AttentionWeights& t) {
  const int tile_nodes = std::min(BLK / (t.n_q_heads / t.kv.n_kv_heads), t.rows.max_nodes);
  return (t.rows.max_nodes + tile_nodes - 1) / tile_nodes;
}

}  // namespace

bool attention_weights_fit(const AttentionWeights& t) { return units_fit(t.rows.n_seqs, t.kv.n_kv_heads, t.rows.max_len, most_tiles(t), UNIT_COST); }

int launch_attention_weights(const AttentionWeights& t, int n_sms, cudaStream_t s) {
  if (!attention_weights_fit(t)) return -2;
  WeightParams p{};
  p.kv = t.kv; p.rows = t.rows;
  p.n_q_heads = t.n_q_heads;
  p.group = t.n_q_heads / t.kv.n_kv_heads;
  p.tile_nodes = std::min(BLK / p.group, t.rows.max_nodes);
  p.q = t.q; p.q_stride = t.q_stride;
  p.scale = t.scale; p.decay = t.decay; p.lse = t.lse; p.use = t.use;
  p.w_in = t.w_in; p.w_out = t.w_out; p.w_stride = t.w_stride;
  p.err_word = static_cast<int*>(t.workspace);
  CUtensorMap q, k;
  if (pool_map(&k, t.kv.k, t.kv, t.kv.k_stride) != 0) return -1;
  q = k;                       // a batch without rows copies none, but the kernel prefetches the map
  if (t.rows.n_rows > 0 && q_map(&q, t.q, t.kv, t.q_stride, t.n_q_heads, t.rows.n_rows, p.tile_nodes) != 0) return -1;
  p.small = small_batch(p.rows.n_seqs, p.kv.n_kv_heads, p.rows.max_len, most_tiles(t), UNIT_COST) ? 1 : 0;
  const int n_ctas = std::min(n_sms, MAX_CTAS);
  if (t.kv.head_dim == 128)
    return t.kv.bf16 ? launch_weights<128, true>(q, k, p, n_ctas, s) : launch_weights<128, false>(q, k, p, n_ctas, s);
  return t.kv.bf16 ? launch_weights<64, true>(q, k, p, n_ctas, s) : launch_weights<64, false>(q, k, p, n_ctas, s);
}

}  // namespace pc
