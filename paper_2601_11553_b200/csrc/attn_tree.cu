// Attention of drafted tokens over a cached context, on tcgen05 (tiles of 17 to 128 rows; fewer rows: attn_narrow.cu).
//
//   out[r] = sum_s exp(scale q_r . k_s - lse_r) v_s,   lse_r = log sum_s exp(scale q_r . k_s),   s over the slots r sees
//
// Rows.  The nodes of a prompt and the query heads of one KV head are packed into the 128 rows of one MMA tile (row =
// node * group + head): all of them read the same K and V, so a K or V byte that reaches shared memory serves every
// row.  A unit of work is (prompt, tile of nodes, KV head); its context is cut into blocks of 128 slots.
//
// Bounds.  A block costs 64 KB of K and V (head size 128, 1.5 us of one SM's share of the HBM) and at most 8.4 MFLOP of
// tensor work (0.75 us) and 16 K exponentials (0.55 us): with the tile at most 128 rows high the operator is bound by
// reading K and V once, whatever the number of rows, and everything below serves to keep the copies running.  Measured,
// 96 rows: 1.50 us a block (6.5 TB/s over 148 SMs), 1.06 us when all K and V are in L2, and 10 - 15 us of a call for its start,
// the ends of its pieces and the merge: 48-node trees on 64 x 2500 slots in pages (floor 105 us) 120 - 123 us a call in a graph of
// back-to-back calls, where one call's start hides behind the last one's end, and 136 - 143 us as one call among others;
// 26-node trees on one prompt of 2112 slots 12.7 us.
//
// Schedule.  Lengths live on the device, so the work is dealt there: every unit costs its blocks and a little more, the
// batch's total cost is cut into one contiguous span per CTA, and a unit that a span border cuts is finished in parts
// whose unnormalised results a second kernel merges (in L2; some 5 us of the batch of trees.  Merging in the CTA that arrives last
// took 4 us more).  Every CTA forms the same prefix sums, so nothing is exchanged.
//
// One CTA per SM, 384 threads:
//   warp 8       copies: Q tile, then K and V tiles in the order the MMAs take them (K0 K1 V0 K2 V1 ...) into one ring
//   warp 9       MMA issuer: S = Q K^T of block j into the score buffer of j's parity, O += P V
//   warps 0-3    softmax of the even blocks, warps 4-7 of the odd ones (thread = row), each parity with an O of its own:
//                two blocks are always under way, so the chain S -> softmax -> PV of one hides behind the other's
//   warps 10-11  clean the V tiles that hold drafted or no slots (see below)
// TMEM (512 columns): O_0 [0,128) O_1 [128,256) S_0 [256,384) S_1 [384,512), P over the first half of its S.
//
// What a row does not see.  Scores are replaced (not added to) where a slot is invisible, so a K of NaN does no harm;
// but 0 * V is NaN where V is infinite or NaN.  The only slots some rows see and others do not are the drafted ones: in
// the V tiles that hold them warps 10-11 put zeros behind the prompt's last slot, and wherever a drafted V is not finite;
// the latter raises a flag, and the rows that do see such a value get it added when they are written.
#include <algorithm>

#include "tree_attn.cuh"

namespace pc {
namespace {

// Four tiles of head size 128 and one Q tile: 48-node trees on 64 x 2500 slots 131 us; with five tiles or two Q tiles 135 - 142 us, 26-node
// trees 15.9 -> 16.0 us.
constexpr int RING_BYTES = 128 * 1024;
constexpr int Q_BYTES = 32 * 1024;
constexpr int TREE_SMEM = RING_BYTES + Q_BYTES + 1024;
constexpr uint32_t TMEM_S = 256;
constexpr int WHOLE_BLOCKS = 6;                 // contexts of up to so many blocks: a unit is one CTA's

// ---------------------------------------------------------------------------------------------------- attention
template <int D, bool BF16>
__global__ void __launch_bounds__(TREE_THREADS, 1)
tree_attention_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                      const __grid_constant__ CUtensorMap tmV, const __grid_constant__ TreeParams a) {
  constexpr int HALVES = D / 64;                         // 64-column halves of a tile, 16 KB each
  constexpr int HALF_BYTES = BLK * 128;
  constexpr int TILE_BYTES = HALVES * HALF_BYTES;
  constexpr int STAGES = RING_BYTES / TILE_BYTES;
  static_assert(STAGES <= MAX_STAGES, "");
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t q_full, q_empty, full[MAX_STAGES], empty[MAX_STAGES], raw[MAX_STAGES], s_full[2], p_full[2], o_full, o_free, ml_full;
  __shared__ float ml[2][2][BLK][2];                     // [item parity][block parity][row]: reference, sum
  __shared__ int bad_v[FLAGS][2];
  __shared__ Span shared_span;
  __shared__ Cursor walks[8];
  __shared__ int64_t warp_sums[TREE_THREADS / 32];
  __shared__ uint32_t tmem_slot;
  __shared__ int cta_failed;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* q_smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = q_smem + Q_BYTES;

  if (threadIdx.x == 0) {
    cta_failed = 0;
    mbar_init(&q_full, 1); mbar_init(&q_empty, 1);
    for (int i = 0; i < STAGES; ++i) { mbar_init(&full[i], 2); mbar_init(&empty[i], 1); mbar_init(&raw[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&p_full[i], 4); }
    mbar_init(&o_full, 1); mbar_init(&o_free, 8); mbar_init(&ml_full, 8);
    fence_mbar_init();
  }
  if (warp == 9) {
    tmem_alloc<512>(&tmem_slot);
    tmem_relinquish();
  }
  if (warp == 8 && lane == 0) { prefetch_tmap(&tmQ); prefetch_tmap(&tmK); prefetch_tmap(&tmV); }
  pdl_launch_dependents();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  pdl_wait();                          // lengths, tables, Q, K and V may come from the kernel before
  const Span span = make_span(a.rows, MIN_SPAN, a.small, &shared_span, warp_sums, [&](const SeqPart& p) { return tree_shape(a, p); });
  const uint32_t tmem = tmem_slot;
  const Pipe pipe{q_smem, Q_BYTES, HALF_BYTES, ring, &q_full, &q_empty, full, empty, raw, &bad_v[0][0], nullptr};
  // 384 threads start with 168 registers each (64 512); the softmax holds a whole row of scores and wants more, the other
  // warpgroup needs few: 256 x 216 + 128 x 72 = 64 512
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    Cursor cur(span);
    Item it{};
    if (warp == 8) {
      copy_role<D, STAGES, 1, false>(a, pipe, cur, span, &tmQ, &tmK, &tmV, &cta_failed);
    } else if (warp == 9) {
      // ------------------------------------------------------------ MMA issuer
      // the whole warp walks; one lane issues
      constexpr uint32_t idesc_qk = make_idesc_f16(BLK, BLK, BF16 ? 1 : 0, 0, 0);
      constexpr uint32_t idesc_pv = make_idesc_f16(BLK, D, BF16 ? 1 : 0, 0, 1);
      uint32_t n_item = 0, st = 0, st_phase = 0, p_phase = 0;        // p_phase: bit i, the parity to wait for on p_full[i]
      bool ok = true;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bar, parity, a.err_word, DEV_ERR_ATTN_MMA));
      };
      auto advance = [&] {
        if (++st == STAGES) { st = 0; st_phase ^= 1u; }
      };
      const uint64_t q_desc = make_smem_desc_sw128(smem_u32(q_smem), 16, 1024);
      const TileLayout<D> tl(a.kv.page_table != nullptr);
      while (ok && next_item(cur, a, &it)) {
        const int nb = it.blk_end - it.blk_begin;
        wait(&q_full, n_item & 1u);
#pragma unroll 1
        for (int j = -2; j < nb && ok; ++j) {                // K0 K1 V0 K2 V1 ...
          const int i = j & 1;
          if (j >= 0) {
            wait(&p_full[i], (p_phase >> i) & 1u);
            p_phase ^= 1u << i;
            if (j == 0) wait(&o_free, (n_item & 1u) ^ 1u);
            wait(&full[st], st_phase);
            if (!ok) break;
            tc_fence_after_sync();
            if (elect_one()) {
              const uint64_t v_desc = make_smem_desc_sw128(smem_u32(ring + st * TILE_BYTES), tl.mn_lbo, tl.group);
#pragma unroll
              for (int kk = 0; kk < BLK / 16; ++kk)
                umma_ts(tmem + i * HEAD_DIM, tmem + TMEM_S + i * BLK + kk * 8, v_desc + (kk * 2 * tl.group >> 4), idesc_pv, j > 1 || kk != 0);
              umma_commit(&empty[st]);
              if (j + 1 == nb) umma_commit(&o_full);
            }
            __syncwarp();
            advance();
          }
          if (j + 2 < nb) {
            wait(&full[st], st_phase);
            if (!ok) break;
            tc_fence_after_sync();
            if (elect_one()) {
              const uint64_t k_desc = make_smem_desc_sw128(smem_u32(ring + st * TILE_BYTES), 16, tl.group);
#pragma unroll
              for (int kk = 0; kk < D / 16; ++kk)
                umma_ss(tmem + TMEM_S + i * BLK, q_desc + (((kk >> 2) * HALF_BYTES + (kk & 3) * 32) >> 4),
                        k_desc + (((kk >> 2) * tl.half + (kk & 3) * 32) >> 4), idesc_qk, kk != 0);
              umma_commit(&s_full[i]);
              umma_commit(&empty[st]);
              if (j + 3 == nb) umma_commit(&q_empty);
            }
            __syncwarp();
            advance();
          }
        }
        ++n_item;
      }
      if (!ok) cta_failed = 1;
    } else {
      clean_role<D, STAGES, BF16, false, false>(a, pipe, cur, &cta_failed);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // where the walk stands waits in shared memory between pieces: the rows' scores want every register
    if (lane == 0) walks[warp] = Cursor(span);
    __syncwarp();
    auto next = [&](Item* item) {
      Cursor cur = walks[warp];
      const bool more = next_item(cur, a, item);
      __syncwarp();
      if (lane == 0) walks[warp] = cur;
      __syncwarp();
      return more;
    };
    Item it{};
    // ------------------------------------------------------------ softmax (warps 0-7)
    const int i = warp >> 2, quarter = warp & 3;
    const int r = quarter * 32 + lane;
    const uint32_t lane_base = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t t_s = tmem + lane_base + TMEM_S + i * BLK, t_o = tmem + lane_base;
    uint32_t n_item = 0, n_s = 0;
    bool ok = true;
    const uint64_t scale2 = pack_f32x2(a.scale_log2, a.scale_log2);
    while (ok && next(&it)) {
      const int nb = it.blk_end - it.blk_begin;
      const bool live = quarter * 32 < it.n_rows;          // warps without rows only keep the barriers' count
      const bool valid = r < it.n_rows;
      const int node_in_tile = min(r, it.n_rows - 1) / a.group;
      const int row = it.row0 + node_in_tile, node = it.node0 + node_in_tile;
      float m = -INFINITY, l = 0.f;
      for (int j = i; j < nb; j += 2) {
        // what the row sees of a block with drafted slots is looked up before its scores take the registers
        const int slot0 = (it.blk_begin + j) * BLK;
        const bool tail = slot0 + BLK > it.ctx_len;
        uint32_t bits[4] = {~0u, ~0u, ~0u, ~0u};
        if (tail) {
#pragma unroll
          for (int c = 0; c < 4; ++c) bits[c] = slot_bits(a.rows, it, row, node, slot0 + c * 32);
          __syncwarp();
        }
        ok = __all_sync(0xffffffffu, mbar_wait(&s_full[i], n_s & 1u, a.err_word, DEV_ERR_ATTN_SOFTMAX));
        if (!ok) break;
        ++n_s;
        tc_fence_after_sync();
        if (live) {
          uint32_t s[128];
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_ld_32x32(t_s + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&s[c * 32]));
          tmem_wait_ld();
          if (tail) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (!((bits[c] >> e) & 1u)) s[c * 32 + e] = 0xff800000u;       // -inf
            }
          }
          float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
          for (int c = 0; c < 128; c += 8) {
            mx0 = fmax3(mx0, __uint_as_float(s[c]), __uint_as_float(s[c + 1]));
            mx1 = fmax3(mx1, __uint_as_float(s[c + 2]), __uint_as_float(s[c + 3]));
            mx2 = fmax3(mx2, __uint_as_float(s[c + 4]), __uint_as_float(s[c + 5]));
            mx3 = fmax3(mx3, __uint_as_float(s[c + 6]), __uint_as_float(s[c + 7]));
          }
          const float m_blk = fmaf(fmax3(fmaxf(mx0, mx1), mx2, mx3), a.scale_log2, -P_HEADROOM<BF16>);       // the block's own reference
          if (j < 2) {
            m = m_blk;
          } else {
            // also the first block that shows anything: the reference was -inf, the sum and O are zero
            const bool need = m_blk > m + RESCALE_THRESHOLD;
            if (__any_sync(0xffffffffu, need)) {           // s_full came behind this parity's last PV: O is complete
              float alpha = 1.0f;
              if (need) { alpha = fast_exp2(m - m_blk); m = m_blk; l *= alpha; }
#pragma unroll 1
              for (int c = 0; c < D / 16; ++c) {
                uint32_t o[16];
                tmem_ld_32x16(t_o + i * HEAD_DIM + c * 16, o);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                tmem_st_32x16(t_o + i * HEAD_DIM + c * 16, o);
              }
              tmem_wait_st();
            }
          }
          const float neg = m == -INFINITY ? 0.f : -m;      // nothing seen yet: every term is exp2(-inf)
          const uint64_t neg2 = pack_f32x2(neg, neg);
          uint64_t sum_a = pack_f32x2(0.f, 0.f), sum_b = sum_a;
#pragma unroll
          for (int h = 0; h < 4; ++h) {                     // 32 columns at a time: the packed words leave before the next are formed
            uint32_t p[16];
#pragma unroll
            for (int c = 0; c < 16; ++c) {
              float x0, x1;
              unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(s[h * 32 + 2 * c]), __uint_as_float(s[h * 32 + 2 * c + 1])), scale2, neg2), x0, x1);
              const float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
              if (c & 1) sum_b = add_f32x2(sum_b, pack_f32x2(p0, p1));
              else sum_a = add_f32x2(sum_a, pack_f32x2(p0, p1));
              if constexpr (BF16) {           // an MMA's operands have one type: P takes V's; the row sum stays unrounded
                __nv_bfloat162 v = __floats2bfloat162_rn(p0, p1);
                p[c] = *reinterpret_cast<uint32_t*>(&v);
              } else {
                __half2 v = __floats2half2_rn(p0, p1);
                p[c] = *reinterpret_cast<uint32_t*>(&v);
              }
            }
            tmem_st_32x16(t_s + h * 16, p);
          }
          float s0, s1;
          unpack_f32x2(add_f32x2(sum_a, sum_b), s0, s1);
          l += s0 + s1;
          tmem_wait_st();
        }
        tc_fence_before_sync();
        __syncwarp();
        if (elect_one()) mbar_arrive(&p_full[i]);
      }
      if (!ok) break;
      // ---- the row's end: both parities' (reference, sum) are exchanged, each warp then writes half of the columns
      const int par = n_item & 1;
      ml[par][i][r][0] = m;
      ml[par][i][r][1] = l;
      __syncwarp();
      if (elect_one()) mbar_arrive(&ml_full);
      ok = __all_sync(0xffffffffu, mbar_wait(&ml_full, par, a.err_word, DEV_ERR_ATTN_CORR));
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&o_full, par, a.err_word, DEV_ERR_ATTN_CORR));
      if (!ok) break;
      tc_fence_after_sync();
      if (live) {
        const float m0 = ml[par][0][r][0], m1 = ml[par][1][r][0];
        const float M = fmaxf(m0, m1), ref = M == -INFINITY ? 0.f : M;
        const float a0 = fast_exp2(m0 - ref), a1 = fast_exp2(m1 - ref);
        const float L = a0 * ml[par][0][r][1] + a1 * ml[par][1][r][1];
        const bool whole = it.blk_begin == 0 && it.blk_end == it.n_blk;
        // a row that sees no slot at all (not: one whose scores are all -inf)
        bool any = it.ctx_len > 0;
#pragma unroll 1
        for (int w = 0; w < it.n_nodes && !any; w += 32) any = node_bits(a.rows, row, node, it.n_nodes, w) != 0;
        __syncwarp();
        const float inv = whole ? 1.0f / L : 1.0f;
        const int head = it.g * a.group + min(r, it.n_rows - 1) % a.group;
        const size_t part = static_cast<size_t>(2 * blockIdx.x + (it.blk_begin == 0 ? 1 : 0)) * BLK + r;
        const bool bad = (*reinterpret_cast<volatile int*>(&bad_v[n_item % FLAGS][0]) | *reinterpret_cast<volatile int*>(&bad_v[n_item % FLAGS][1])) != 0;
        char* dst = static_cast<char*>(a.out) + (static_cast<int64_t>(row) * a.out_stride + head * D) * 2;
#pragma unroll 1
        for (int c = i * (D / 64); c < (i + 1) * (D / 64); ++c) {
          uint32_t o0[32], o1[32];
          tmem_ld_32x32(t_o + c * 32, o0);
          if (nb > 1) tmem_ld_32x32(t_o + HEAD_DIM + c * 32, o1);
          tmem_wait_ld();
          float o[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            o[e] = __uint_as_float(o0[e]) * a0;
            if (nb > 1) o[e] = fmaf(__uint_as_float(o1[e]), a1, o[e]);
          }
          if (bad) {
            // a drafted V that is not finite was taken out of the product: the rows that see it get it here
#pragma unroll 1
            for (int s = max(it.ctx_len, it.blk_begin * BLK); s < min(it.ctx_len + it.n_nodes, it.blk_end * BLK); ++s) {
              if (!(node_bits(a.rows, row, node, it.n_nodes, s - it.ctx_len) & 1u)) continue;
              const int64_t vr = slot_row(a.kv.page_table, a.kv.pt_stride, a.kv.ctx_start, a.kv.n_slots, it.seq, s);
              if (vr < 0) continue;
              const unsigned short* vp = static_cast<const unsigned short*>(a.kv.v) + vr * a.kv.v_stride + it.g * D + c * 32;
#pragma unroll
              for (int e = 0; e < 32; ++e) {
                const float x = elem<BF16>(vp[e]);
                if (!isfinite(x)) o[e] += x;
              }
            }
            __syncwarp();
          }
          if (valid && whole) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t pk[4];
#pragma unroll
              for (int q = 0; q < 4; ++q) pk[q] = any ? pack_out<BF16>(o[8 * e + 2 * q] * inv, o[8 * e + 2 * q + 1] * inv) : 0u;
              *reinterpret_cast<uint4*>(dst + c * 64 + e * 16) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
            }
          } else if (valid) {
            float4* po = reinterpret_cast<float4*>(a.partial_o + part * HEAD_DIM + c * 32);
#pragma unroll
            for (int e = 0; e < 8; ++e) po[e] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          }
        }
        if (valid && i == 0) {
          if (!whole) *reinterpret_cast<float2*>(a.partial_ml + part * 2) = make_float2(M, any ? L : -1.f);
          else if (a.lse) a.lse[static_cast<size_t>(row) * a.n_q_heads + head] = any ? (M + log2f(L)) * LN2 : -INFINITY;
        }
      }
      tc_fence_before_sync();
      __syncwarp();
      if (elect_one()) mbar_arrive(&o_free);
      ++n_item;
    }
    if (!ok) cta_failed = 1;
  }

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

// The parts of a cut unit: out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s, one warp per row.
constexpr int MERGE_WARPS = 8;
template <int D, bool BF16>
__global__ void __launch_bounds__(MERGE_WARPS * 32) tree_merge_kernel(TreeParams a) {
  constexpr int E = D / 32;                             // columns per lane
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int r = blockIdx.y * MERGE_WARPS + (threadIdx.x >> 5);
  const MergeRecord* mr = a.merges + blockIdx.x;
  const int n_parts = *reinterpret_cast<const volatile int*>(&mr->n_parts);
  const int n_rows = *reinterpret_cast<const volatile int*>(&mr->n_rows);
  if (n_parts <= 1 || r >= n_rows) return;
  const int row = *reinterpret_cast<const volatile int*>(&mr->row0) + r / a.group;
  const int head = *reinterpret_cast<const volatile int*>(&mr->head0) + r % a.group;
  // part 0 is the record's CTA's last item, part s > 0 the first item of the s-th CTA behind it
  auto slot = [&](int s) { return static_cast<size_t>(2 * (blockIdx.x + s) + (s == 0 ? 1 : 0)) * BLK + r; };
  // four parts at a time, with a running reference: their sums and results are asked for together
  bool any = true;
  float acc[E], M = -INFINITY, L = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  for (int s0 = 0; s0 < n_parts; s0 += 4) {
    float2 v[4];
    float o[4][E];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      v[u] = make_float2(-INFINITY, 0.f);
      if (s0 + u >= n_parts) continue;
      const size_t at = slot(s0 + u);
      v[u] = ld_dep_f32x2(a.partial_ml + at * 2);
      if constexpr (E == 4) *reinterpret_cast<float4*>(o[u]) = ld_dep_f32x4(a.partial_o + at * HEAD_DIM + lane * 4);
      else *reinterpret_cast<float2*>(o[u]) = ld_dep_f32x2(a.partial_o + at * HEAD_DIM + lane * 2);
    }
    const float top = fmaxf(fmax3(v[0].x, v[1].x, v[2].x), v[3].x), now = fmaxf(M, top), ref = now == -INFINITY ? 0.f : now;
    const float before = fast_exp2(M - ref);
    M = now;
    L *= before;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] *= before;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (s0 + u >= n_parts) break;
      if (v[u].y < 0.f) any = false;
      const float w = fast_exp2(v[u].x - ref);
      L = fmaf(w, v[u].y, L);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(w, o[u][e], acc[e]);
    }
  }
  const float inv = 1.0f / L;
  uint32_t pk[E / 2];
#pragma unroll
  for (int e = 0; e < E; e += 2) pk[e / 2] = any ? pack_out<BF16>(acc[e] * inv, acc[e + 1] * inv) : 0u;
  char* dst = static_cast<char*>(a.out) + (static_cast<int64_t>(row) * a.out_stride + head * D + lane * E) * 2;
  if constexpr (E == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(pk[0], pk[1]);
  else *reinterpret_cast<uint32_t*>(dst) = pk[0];
  if (lane == 0 && a.lse) a.lse[static_cast<size_t>(row) * a.n_q_heads + head] = any ? (M + log2f(L)) * LN2 : -INFINITY;
}

template <int D, bool BF16>
int launch_tree(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const TreeParams& p, int n_ctas, cudaStream_t s) {
  static bool set[MAX_DEVICES] = {};
  const int dev = current_device_slot();
  if (!set[dev]) {
    if (cudaFuncSetAttribute(tree_attention_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, TREE_SMEM) != cudaSuccess) return -1;
    set[dev] = true;
  }
  // Up to 16 rows a tile: the transposed form.  64 x 2500 slots, 2 rows: 107 us against 124 us for the 128-row form; 16 rows: 111 against
  // 115; 32 rows (with twice the columns): 124 against 118; two prompts of 33024 slots, 32 rows: 57 against 55.
  if (p.tile_nodes * p.group <= NARROW_ROWS) {
    if (launch_narrow_attention(q, k, v, p, n_ctas, s) != 0) return -1;
  } else if (launch_pdl(tree_attention_kernel<D, BF16>, dim3(n_ctas), dim3(TREE_THREADS), TREE_SMEM, s, q, k, v, p) != cudaSuccess) {
    return -1;
  }
  if (p.whole) return 0;                          // nothing is ever cut
  const int rows = std::min(p.tile_nodes, p.rows.max_nodes) * p.group;
  return launch_pdl(tree_merge_kernel<D, BF16>, dim3(n_ctas, (rows + MERGE_WARPS - 1) / MERGE_WARPS), dim3(MERGE_WARPS * 32), 0, s, p) == cudaSuccess ? 0 : -1;
}

// What the host decides from a call's sizes; returns the most units a prompt can have.
int64_t set_sizes(TreeParams& p, const TreeAttention& t) {
  p.kv = t.kv; p.rows = t.rows;
  p.n_q_heads = t.n_q_heads;
  p.group = t.n_q_heads / t.kv.n_kv_heads;
  p.tile_nodes = std::min(BLK / p.group, t.rows.max_nodes);
  // A unit's cost beside its blocks grows with its rows (the end of every row is written out while no block is worked on).  2 -> 4: 26-node
  // trees on 2112 slots 16.3 -> 15.8 us; 64 x 2500 single tokens 108.4 -> 110.4 us.
  p.over = p.tile_nodes * p.group <= 16 ? 2 : 4;
  return static_cast<int64_t>((t.rows.max_nodes + p.tile_nodes - 1) / p.tile_nodes) * t.kv.n_kv_heads;
}

}  // namespace

bool tree_attention_fits(const TreeAttention& t) {
  TreeParams p{};
  const int64_t units = set_sizes(p, t);
  return units_fit(t.rows.n_seqs, units, t.rows.max_len, 1, p.over);
}

int launch_tree_attention(const TreeAttention& t, int n_sms, cudaStream_t s) {
  TreeParams p{};
  const int64_t units = set_sizes(p, t);
  if (!units_fit(p.rows.n_seqs, units, p.rows.max_len, 1, p.over)) return -2;
  p.scale_log2 = t.scale * LOG2E;
  p.out = t.out; p.out_stride = t.out_stride; p.lse = t.lse;
  char* ws = static_cast<char*>(t.workspace);
  p.err_word = reinterpret_cast<int*>(ws);
  p.merges = reinterpret_cast<MergeRecord*>(ws + WS_MERGE);
  p.partial_ml = reinterpret_cast<float*>(ws + WS_ML);
  p.partial_o = reinterpret_cast<float*>(ws + WS_O);
  CUtensorMap q, k, v;
  if (q_map(&q, t.q, t.kv, t.q_stride, t.n_q_heads, t.rows.n_rows, p.tile_nodes) != 0 || pool_map(&k, t.kv.k, t.kv, t.kv.k_stride) != 0 ||
      pool_map(&v, t.kv.v, t.kv, t.kv.v_stride) != 0)
    return -1;
  // Short contexts: a unit is one CTA's, and there is no second kernel.  On the device, whole against cut: 64 prompts of 700 slots 43 against
  // 44 us for single tokens and 54 against 57 for trees of 26, ten such prompts 12.5 against 13.7 and 15.3 against 18.3, one prompt of
  // 300 slots 8.7 against 9.0.  Few units of more slots lose by it: one prompt of 512 slots 10.6 against 9.5 us, of 700 11.1 against 9.3,
  // with 26 nodes 13.7 against 11.0.  The rule leaves them whole for single calls, which the host bounds (a second launch is 2 us of its
  // time); in a captured graph the cut form would be the faster one there.
  p.whole = p.rows.max_len <= WHOLE_BLOCKS * BLK ? 1 : 0;
  const int n_ctas = std::min(n_sms, MAX_CTAS);
  p.small = small_batch(p.rows.n_seqs, units, p.rows.max_len, 1, p.over) ? 1 : 0;
  if (t.kv.head_dim == 128)
    return t.kv.bf16 ? launch_tree<128, true>(q, k, v, p, n_ctas, s) : launch_tree<128, false>(q, k, v, p, n_ctas, s);
  return t.kv.bf16 ? launch_tree<64, true>(q, k, v, p, n_ctas, s) : launch_tree<64, false>(q, k, v, p, n_ctas, s);
}

}  // namespace pc
