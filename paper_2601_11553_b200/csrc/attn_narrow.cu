// Tree attention of tiles with at most 16 rows (one token a prompt, short chains): both products formed transposed.
//
// With a handful of rows the 128-row tile of attn_tree.cu leaves its softmax to one warp per block, 128 scores a thread: a
// chain of 1.2 us a block and 2 us at a piece's end, which the copies cannot always hide.  Here a block's slots are the
// MMA's M side: S^T = K Q^T has one TMEM lane, i.e. one thread, per slot and a column per row, so a thread forms as
// many exponentials as there are rows; O^T = V^T P^T has a lane per element of the head and a column per row.  Three things
// cross threads: whether a row's block maximum passes its reference (one barrier with an OR), its sum (only at the piece's end), and
// P, which goes through shared memory (K-major, 128-byte swizzle) because the second product reads it as its B operand.
//
// Roles, ring, schedule, masks and the cleaning of V are those of attn_tree.cu.  The even blocks' four warps and the odd ones'
// each keep a running reference, sum and O of their own, merged at the piece's end; O has two buffers per parity, so the next
// piece's products do not wait for that.  Q has two slots for the same reason.
//
// Measured: one token on each of 64 ragged prompts around 2500 slots, two heads a KV head: 105 - 107 us (655 MB, 6.1 TB/s; a plain copy
// reaches 6.45), 107 - 108 us in pages; the 128-row form takes 124 us.  One token on 512 slots: 10.6 us, one kernel.
#include <algorithm>

#include "tree_attn.cuh"

namespace pc {
namespace {

constexpr int NC = NARROW_ROWS;                  // columns of the products
// Four tiles of head size 128.  64 tokens on 2500 slots with 3 / 4 / 5 / 6 tiles: 111.6 / 107.4 / 107.2 / 113 us contiguous; in pages with
// 4 / 5 / 6: 108.3 / 110.7 / 115.5.  (What is asked for too early comes in the way of what the other SMs wait for.)
constexpr int RING_BYTES = 128 * 1024;

// Per-column reduction over the warp's 32 lanes, transposing as it goes: every step exchanges half of the columns that are left
// with the lane across and combines the other half, so NC columns cost about NC shuffles.  Lane l returns column l % NC.
template <typename Op>
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
  return op(v[0], __shfl_xor_sync(0xffffffffu, v[0], 16));
}
// What the drafted V elements that are not finite (slots s .. end - 1) add to an output element of a row: they were taken out
// of the product.
template <bool BF16>
__device__ __noinline__ float bad_v_sum(const TreeParams& a, int seq, int ctx_len, int n_nodes, int s, int end, int row, int node, int col) {
  float o = 0.f;
#pragma unroll 1
  for (; s < end; ++s) {
    if (!(node_bits(a.rows, row, node, n_nodes, s - ctx_len) & 1u)) continue;
    const int64_t vr = slot_row(a.kv.page_table, a.kv.pt_stride, a.kv.ctx_start, a.kv.n_slots, seq, s);
    if (vr < 0) continue;
    const float x = elem<BF16>(static_cast<const unsigned short*>(a.kv.v)[vr * a.kv.v_stride + col]);
    if (!isfinite(x)) o += x;
  }
  return o;
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
template <int D>
constexpr int narrow_smem() { return 1024 + RING_BYTES + 2 * NC * D * 2 + 2 * NC * BLK * 2; }

template <int D, bool BF16>
__global__ void __launch_bounds__(TREE_THREADS, 1)
narrow_attention_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                        const __grid_constant__ CUtensorMap tmV, const __grid_constant__ TreeParams a) {
  constexpr int HALVES = D / 64;
  constexpr int HALF_BYTES = BLK * 128;
  constexpr int TILE_BYTES = HALVES * HALF_BYTES;
  constexpr int STAGES = RING_BYTES / TILE_BYTES;
  constexpr int Q_HALF = NC * 128, Q_SLOT = HALVES * Q_HALF;
  constexpr int P_HALF = NC * 128, P_BYTES = 2 * P_HALF;
  constexpr int TMEM_COLS = 128;                               // S_0 S_1, then O of (item parity, block parity): six times NC
  constexpr uint32_t TMEM_O = 2 * NC;
  static_assert(STAGES <= MAX_STAGES, "");
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t q_full[2], q_empty[2], full[MAX_STAGES], empty[MAX_STAGES], raw[MAX_STAGES], s_full[2], p_full[2],
      o_full[2], o_free[2], ml_full;
  __shared__ __align__(16) float block_max[2][2][NC][4];       // [block parity][use][row][warp]
  __shared__ __align__(16) float fin_l[2][2][NC][4];            // [item parity][block parity][row][warp]: a warp's share of the sum
  __shared__ float fin_m[2][2][NC];
  __shared__ uint64_t node_mask[2 * NARROW_ROWS * MASK_WORDS];
  __shared__ int bad_v[FLAGS][2];
  __shared__ Span shared_span;
  __shared__ int64_t warp_sums[TREE_THREADS / 32];
  __shared__ uint32_t tmem_slot;
  __shared__ int cta_failed;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* q_smem = ring + RING_BYTES;
  uint8_t* p_smem = q_smem + 2 * Q_SLOT;

  if (threadIdx.x == 0) {
    cta_failed = 0;
    for (int i = 0; i < STAGES; ++i) { mbar_init(&full[i], 2); mbar_init(&empty[i], 1); mbar_init(&raw[i], 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 3);          // the copy and the two warps with the masks
      mbar_init(&q_empty[i], 9);         // the MMAs and the eight softmax warps
      mbar_init(&s_full[i], 1); mbar_init(&p_full[i], 4);
      mbar_init(&o_full[i], 1); mbar_init(&o_free[i], 8);
    }
    mbar_init(&ml_full, 8);
    fence_mbar_init();
  }
  if (warp == 9) {
    tmem_alloc<TMEM_COLS>(&tmem_slot);
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
  const Pipe pipe{q_smem, Q_SLOT, Q_HALF, ring, q_full, q_empty, full, empty, raw, &bad_v[0][0], node_mask};
  Cursor cur(span);
  Item it{};

  if (warp == 8) {
    copy_role<D, STAGES, 2, true>(a, pipe, cur, span, &tmQ, &tmK, &tmV, &cta_failed);
  } else if (warp >= 10) {
    clean_role<D, STAGES, BF16, true, true>(a, pipe, cur, &cta_failed);
  } else if (warp == 9) {
    // ------------------------------------------------------------ MMA issuer
    // the whole warp walks; one lane issues
    constexpr uint32_t idesc_s = make_idesc_f16(BLK, NC, BF16 ? 1 : 0, 0, 0);
    constexpr uint32_t idesc_o = make_idesc_f16(BLK, NC, BF16 ? 1 : 0, 1, 0);       // A = V^T: V's rows are the K index
    const TileLayout<D> tl(a.kv.page_table != nullptr);
    uint32_t n_item = 0, st = 0, st_phase = 0, p_phase = 0;        // p_phase: bit i, the parity to wait for on p_full[i]
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (ok) ok = __all_sync(0xffffffffu, bar_wait(bar, parity, a.err_word, DEV_ERR_ATTN_MMA));
    };
    auto advance = [&] {
      if (++st == STAGES) { st = 0; st_phase ^= 1u; }
    };
    while (ok && next_item(cur, a, &it)) {
      const int nb = it.blk_end - it.blk_begin, par = n_item & 1;
      const uint64_t q_desc = make_smem_desc_sw128(smem_u32(q_smem + par * Q_SLOT), 16, 1024);
      wait(&q_full[par], (n_item >> 1) & 1u);
#pragma unroll 1
      for (int j = -2; j < nb && ok; ++j) {                // K0 K1 V0 K2 V1 ...
        const int i = j & 1;
        if (j >= 0) {
          wait(&p_full[i], (p_phase >> i) & 1u);
          p_phase ^= 1u << i;
          if (j == 0) wait(&o_free[par], ((n_item >> 1) & 1u) ^ 1u);
          wait(&full[st], st_phase);
          if (!ok) break;
          tc_fence_after_sync();
          if (elect_one()) {
            // head size 64 has one 64-element column block: the second 64 TMEM lanes repeat the first (distance 0) and are not read
            const uint64_t v_desc = make_smem_desc_sw128(smem_u32(ring + st * TILE_BYTES), tl.mn_lbo, tl.group);
            const uint64_t p_desc = make_smem_desc_sw128(smem_u32(p_smem + i * P_BYTES), 16, 1024);
#pragma unroll
            for (int kk = 0; kk < BLK / 16; ++kk)
              umma_ss(tmem + TMEM_O + (par * 2 + i) * NC, v_desc + (kk * 2 * tl.group >> 4),
                      p_desc + (((kk >> 2) * P_HALF + (kk & 3) * 32) >> 4), idesc_o, j > 1 || kk != 0);
            umma_commit(&empty[st]);
            if (j + 1 == nb) umma_commit(&o_full[par]);
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
              umma_ss(tmem + i * NC, k_desc + (((kk >> 2) * tl.half + (kk & 3) * 32) >> 4),
                      q_desc + (((kk >> 2) * Q_HALF + (kk & 3) * 32) >> 4), idesc_s, kk != 0);
            umma_commit(&s_full[i]);
            umma_commit(&empty[st]);
            if (j + 3 == nb) umma_commit(&q_empty[par]);
          }
          __syncwarp();
          advance();
        }
      }
      ++n_item;
    }
    if (!ok) cta_failed = 1;
  } else {
    // ------------------------------------------------------------ softmax (warps 0-7).  The four warps of a parity meet at a hardware
    // barrier in every block, so a warp whose wait ran out keeps walking the blocks, without waiting or computing, to the end.
    const int i = warp >> 2, quarter = warp & 3;
    const int r = quarter * 32 + lane;                     // slot of the block; element of the head
    const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    uint8_t* p_row = p_smem + i * P_BYTES + (r >> 6) * P_HALF + (r & 7) * 2;
    const int p_vec = (r & 63) >> 3;
    uint32_t n_item = 0, n_s = 0, n_raise = 0;
    bool ok = true;
    while (next_item(cur, a, &it)) {
      const int nb = it.blk_end - it.blk_begin, par = n_item & 1;
      float neg[NC], l[NC];                                // -reference (the same in all threads); sum over this thread's slots only
      uint32_t unset = (1u << it.n_rows) - 1;       // rows that have seen nothing yet: reference 0, sum and O zero
#pragma unroll
      for (int c = 0; c < NC; ++c) { neg[c] = 0.f; l[c] = 0.f; }
      for (int j = i; j < nb; j += 2) {
        if (ok) ok = __all_sync(0xffffffffu, bar_wait(&s_full[i], n_s & 1u, a.err_word, DEV_ERR_ATTN_SOFTMAX));
        ++n_s;
        uint32_t s[NC];
        bool raise = j == i;                               // does any row's block maximum pass what its reference allows
        if (ok) {
          tc_fence_after_sync();
          tmem_ld_32x16(lanes + i * NC, s);
          tmem_wait_ld();
          const int slot = (it.blk_begin + j) * BLK + r;
          if ((it.blk_begin + j + 1) * BLK > it.ctx_len) {
            ok = __all_sync(0xffffffffu, bar_wait(&q_full[par], (n_item >> 1) & 1u, a.err_word, DEV_ERR_ATTN_SOFTMAX));   // the masks
            if (slot >= it.ctx_len) {
              const int node = slot - it.ctx_len;
              uint32_t seen = 0;
              if (node < it.n_nodes) {
                const uint64_t* w = node_mask + par * NARROW_ROWS * MASK_WORDS + (node >> 6);
                int at = 0, h = 0;
#pragma unroll 1
                for (int c = 0; c < it.n_rows; ++c) {
                  seen |= static_cast<uint32_t>((w[at] >> (node & 63)) & 1u) << c;
                  if (++h == a.group) { h = 0; at += MASK_WORDS; }
                }
              }
#pragma unroll
              for (int c = 0; c < NC; ++c)
                if (!((seen >> c) & 1u)) s[c] = 0xff800000u;          // -inf
            }
            __syncwarp();
          }
#pragma unroll
          for (int c0 = 0; c0 < NC; c0 += 4) {
            if (c0 >= it.n_rows) break;
#pragma unroll
            for (int c = c0; c < c0 + 4; ++c) {
              if (c >= it.n_rows) s[c] = 0xff800000u;                // columns behind the last row hold anything
              raise |= fmaf(__uint_as_float(s[c]), a.scale_log2, neg[c]) > P_HEADROOM<BF16> + RESCALE_THRESHOLD;
            }
          }
          if (unset != 0) {
#pragma unroll
            for (int c = 0; c < NC; ++c) raise |= ((unset >> c) & 1u) && __uint_as_float(s[c]) > -INFINITY;
          }
        }
        if (j != i) raise = parity_any(i, raise);
        if (raise) {
          // The rows' exact block maxima: a warp's by a transposing reduction, the block's from four words a row; lane c then works
          // out row c's new reference and every thread fetches it by shuffles.  Two buffers: between two uses of one lies the
          // other's barrier.
          float(*maxima)[4] = block_max[i][n_raise++ & 1];
          float top[NC];
#pragma unroll
          for (int c = 0; c < NC; ++c) top[c] = c < it.n_rows ? __uint_as_float(s[c]) : -INFINITY;
          const float mine = column_reduce(top, [](float x, float y) { return fmaxf(x, y); });
          if (lane < NC) maxima[lane][quarter] = mine;
          parity_any(i, false);
          const float4 x = *reinterpret_cast<const float4*>(maxima[lane % NC]);
          const float now = fmaf(fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w)), a.scale_log2, -P_HEADROOM<BF16>);    // the block's own reference
          float old = 0.f;
#pragma unroll
          for (int c = 0; c < NC; ++c) old = lane == c ? neg[c] : old;
          const bool fresh = (unset >> (lane & 31)) & 1u;
          const bool up = now > -INFINITY && (fresh || now + old > RESCALE_THRESHOLD);
          const float alpha = !up ? 1.f : fresh ? 0.f : fast_exp2(-old - now);
          const float next = up ? -now : old;
          unset &= ~(__ballot_sync(0xffffffffu, up));
#pragma unroll
          for (int c = 0; c < NC; ++c) neg[c] = __shfl_sync(0xffffffffu, next, c);
          if (j != i && ok) {                              // s_full came behind this parity's last product: O is complete
            const uint32_t t_o = lanes + TMEM_O + (par * 2 + i) * NC;
            uint32_t o[NC];
            tmem_ld_32x16(t_o, o);
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              const float f = __shfl_sync(0xffffffffu, alpha, c);
              l[c] *= f;
              o[c] = __float_as_uint(__uint_as_float(o[c]) * f);
            }
            tmem_st_32x16(t_o, o);
            tmem_wait_st();
          }
        }
        if (ok) {
#pragma unroll
          for (int c0 = 0; c0 < NC; c0 += 4) {
            if (c0 >= it.n_rows) break;
#pragma unroll
            for (int c = c0; c < c0 + 4; ++c) {
              const float p = fast_exp2(fmaf(__uint_as_float(s[c]), a.scale_log2, neg[c]));
              l[c] += p;
              unsigned short bits;                         // an MMA's operands have one type: P takes V's; the row sum stays unrounded
              if constexpr (BF16) bits = __bfloat16_as_ushort(__float2bfloat16_rn(p));
              else bits = __half_as_ushort(__float2half_rn(p));
              *reinterpret_cast<unsigned short*>(p_row + c * 128 + ((p_vec ^ (c & 7)) << 4)) = bits;
            }
          }
          fence_proxy_async_smem();                        // the MMA reads P through the async proxy
          tc_fence_before_sync();
          __syncwarp();
          if (elect_one()) mbar_arrive(&p_full[i]);
        }
      }
      // ---- the piece's end: sums and references of both parities are exchanged; parity i writes rows i, i + 2, ...
      if (ok) {
        const float sum = column_reduce(l, [](float x, float y) { return x + y; });
        if (lane < NC) fin_l[par][i][lane][quarter] = sum;
        float mine = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) mine = lane == c ? -neg[c] : mine;
        if (quarter == 0 && lane < NC) fin_m[par][i][lane] = ((unset >> lane) & 1u) || nb <= i ? -INFINITY : mine;
        __syncwarp();
        if (elect_one()) { mbar_arrive(&ml_full); mbar_arrive(&q_empty[par]); }
        ok = __all_sync(0xffffffffu, bar_wait(&ml_full, par, a.err_word, DEV_ERR_ATTN_CORR));
      }
      if (ok) ok = __all_sync(0xffffffffu, bar_wait(&o_full[par], (n_item >> 1) & 1u, a.err_word, DEV_ERR_ATTN_CORR));
      if (ok) {
        tc_fence_after_sync();
        const bool whole = it.blk_begin == 0 && it.blk_end == it.n_blk;
        const size_t part0 = static_cast<size_t>(2 * blockIdx.x + (it.blk_begin == 0 ? 1 : 0)) * BLK;
        const bool bad = (*reinterpret_cast<volatile int*>(&bad_v[n_item % FLAGS][0]) | *reinterpret_cast<volatile int*>(&bad_v[n_item % FLAGS][1])) != 0;
        // Lane c works out row c's two factors; the loop over rows then only scales and stores.  It is rolled because it runs once
        // a piece: straight-line code for every row cost more in instruction fetches than all the rest (2400 clocks a row).
        float f0 = 0.f, f1 = 0.f;
        if (lane < it.n_rows) {
          const float m0 = fin_m[par][0][lane], m1 = fin_m[par][1][lane];
          const float4 l0 = *reinterpret_cast<const float4*>(fin_l[par][0][lane]), l1 = *reinterpret_cast<const float4*>(fin_l[par][1][lane]);
          const float M = fmaxf(m0, m1), ref = M == -INFINITY ? 0.f : M;
          f0 = fast_exp2(m0 - ref);
          f1 = nb > 1 ? fast_exp2(m1 - ref) : 0.f;
          float L = f0 * ((l0.x + l0.y) + (l0.z + l0.w));
          if (nb > 1) L = fmaf(f1, (l1.x + l1.y) + (l1.z + l1.w), L);
          const int node = lane / a.group, row = it.row0 + node;
          bool any = it.ctx_len > 0;                       // does the row see a slot at all (not: are its scores all -inf)
          if (!any) any = sees_a_node(a.rows, row, it.node0 + node, it.n_nodes);
          if (whole) {
            const float inv = any ? 1.0f / L : 0.f;        // a row that sees nothing has an O of zeros
            f0 *= inv;
            f1 *= inv;
            if (warp == 0 && a.lse)
              a.lse[static_cast<size_t>(row) * a.n_q_heads + it.g * a.group + lane % a.group] = any ? (M + log2f(L)) * LN2 : -INFINITY;
          } else if (warp == 0) {
            *reinterpret_cast<float2*>(a.partial_ml + (part0 + lane) * 2) = make_float2(M, any ? L : -1.f);
          }
        }
        __syncwarp();
        int node = 0, h = i * 4;
#pragma unroll 1
        while (h >= a.group) { h -= a.group; ++node; }
#pragma unroll 1
        for (int c0 = i * 4; c0 < it.n_rows; c0 += 8) {    // four rows at a time, the parities in turn
          uint32_t o0[4], o1[4];
          tmem_ld_32x4(lanes + TMEM_O + par * 2 * NC + c0, o0);
          tmem_ld_32x4(lanes + TMEM_O + (par * 2 + 1) * NC + c0, o1);         // not used when there is one block
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int c = c0 + e;
            float o = __uint_as_float(o0[e]) * __shfl_sync(0xffffffffu, f0, c & 31);
            const float w1 = __shfl_sync(0xffffffffu, f1, c & 31);
            if (nb > 1) o = fmaf(__uint_as_float(o1[e]), w1, o);
            if (r < D && c < it.n_rows) {
              const int row = it.row0 + node;
              if (bad)
                o += bad_v_sum<BF16>(a, it.seq, it.ctx_len, it.n_nodes, max(it.ctx_len, it.blk_begin * BLK),
                                     min(it.ctx_len + it.n_nodes, it.blk_end * BLK), row, it.node0 + node, it.g * D + r);
              if (whole) {
                static_cast<unsigned short*>(a.out)[static_cast<int64_t>(row) * a.out_stride + (it.g * a.group + h) * D + r] =
                    static_cast<unsigned short>(pack_out<BF16>(o, 0.f));
              } else {
                a.partial_o[(part0 + c) * HEAD_DIM + r] = o;
              }
            }
            if (++h == a.group) { h = 0; ++node; }
          }
          __syncwarp();
#pragma unroll 1
          for (h += 4; h >= a.group; ++node) h -= a.group; // the other parity's four rows
        }
        tc_fence_before_sync();
        __syncwarp();
        if (elect_one()) mbar_arrive(&o_free[par]);
      }
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
    tmem_dealloc<TMEM_COLS>(tmem);
  }
}

template <int D, bool BF16>
int launch(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const TreeParams& p, int n_ctas, cudaStream_t s) {
  static bool set[MAX_DEVICES] = {};
  const int dev = current_device_slot();
  if (!set[dev]) {
    if (cudaFuncSetAttribute(narrow_attention_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, narrow_smem<D>()) != cudaSuccess) return -1;
    set[dev] = true;
  }
  return launch_pdl(narrow_attention_kernel<D, BF16>, dim3(n_ctas), dim3(TREE_THREADS), narrow_smem<D>(), s, q, k, v, p) == cudaSuccess ? 0 : -1;
}

}  // namespace

int launch_narrow_attention(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const TreeParams& p, int n_ctas,
                            cudaStream_t s) {
  if (p.kv.head_dim == 128) return p.kv.bf16 ? launch<128, true>(q, k, v, p, n_ctas, s) : launch<128, false>(q, k, v, p, n_ctas, s);
  return p.kv.bf16 ? launch<64, true>(q, k, v, p, n_ctas, s) : launch<64, false>(q, k, v, p, n_ctas, s);
}

}  // namespace pc
