// Tree attention over 8-bit pages: both products transposed, formed by the tensor cores on the 8-bit values as they are stored.
//
// With s_K, s_V a page's scales, x = scale * s_K (q . k8), and out = sum 2^x' s_V v8 / sum 2^x' (x' in base 2, less a reference).  A block's 128 slots are
// the MMAs' M side: S^T = K Q^T has a TMEM lane, i.e. a thread, per slot and columns per row (query head of a node), so a page's
// scales are a thread's own numbers; O^T = V^T P^T has a lane per element of the head.  An 8-bit MMA wants both operands in 8 bits, so q and
// the weights P = 2^x' s_V are split into sums of 8-bit numbers, each some powers of two below the one before, with columns of their own.
// Nothing is unpacked: shared memory sees every byte of the cache twice (copy in, MMA), where forming 16-bit tiles would take seven times.
//   q: 2 parts (bf16, exact: 8 bits of mantissa are 4 + 4) or 3 (fp16), 2^4 apart, of q * 2^-e with the row's largest in (224, 448].
//   P: 3 parts (bf16) or 4 (fp16), 2^4 apart, of 5 exponent bits and 2 mantissa bits (the MMA takes them beside V's e4m3): a rounding to 3 bits
//   leaves 2^-4 of a power of two at most, so weights are kept to 2^-11 or 2^-15 of themselves.  A row's largest lies in 2^7 .. 2^15 and a
//   part's last bit is worth 2^-16, so that holds down to 2^-21 of the largest, and below each is off by at most 2^-32 (bf16) or 2^-36 (fp16) of it.
//   (e4m3 parts have 4 bits but 2^15 less range.  With two or three of them and one far below for small weights, those below 2^-13 or 2^-17 of the
//   largest were off by up to 2^-4 of themselves: all that a long context under one heavy slot, or under a page of a larger scale, adds up to.)
// The accumulation is fp32's (measured: off by at most 2^-21 of the sum of magnitudes).
//
// Bound by HBM: 2 D bytes a slot and KV head.  Measured (bf16, the chains fp16; head size 128, 8 KV heads): one token on each of 64 prompts around 2500 slots 62 us (329 MB,
// 5.3 TB/s; the blocks run at the HBM's rate, the rest is the start, uneven ends and the merge), chains of 7 with four heads a KV head on 2 x 33024
// slots 37.8 us (136 MB; with fp16's weights off by 2^-12 37.0), trees of 26 with two heads a KV head 121 us, fp16 155 (339 MB; every prompt has one or two tiles of up to 32 rows, whose softmax
// takes 0.53 - 0.78 us a block), one token on 512 slots 7.6 us (latency).  One copy per page fetches keys and values of a head: a box of [row group][K, V][8 rows][D
// bytes], so that the row groups of K, and those of V, are one stride apart over all pages of a block.
// Warps 0-7: softmax (even and odd blocks), 8: copies, 9: S products, 10: O products, 11: splits Q, fetches masks, cleans V.  With one warp for
// both products its waits and issues, one behind the other, took 1800 clocks a block (64 x 2500 slots 76 us); a block's bytes take 1490.
#include <algorithm>
#include <type_traits>

#include "tree_common.cuh"

namespace pc {
namespace {

// Six tiles of head size 128 (five beside the larger Q and P): an item's end, where nothing is taken from the ring for 7000 clocks, is as long as
// five tiles take to come in.
__host__ __device__ constexpr int ring_bytes(int nc) { return (nc == 16 ? 192 : 160) * 1024; }
constexpr int CLEAN_BARS = 8;                   // more than the tiles between a product with K and the one with V
constexpr int FLAGS = 8;                        // items a `bad V` flag lives for: more than the roles can be apart
constexpr int MAX_NODES = 256;             // of a prompt, at most
// The running reference lies HEADROOM (base 2) below the largest score that set it and is raised when a score exceeds that by RESCALE_THRESHOLD.
constexpr float HEADROOM = 7.f, RESCALE_THRESHOLD = 8.f;
template <int NC> constexpr int MIN_SPAN = NC == 16 ? 2 : 24;      // a CTA's least share: two blocks, so that none that a unit reaches is without one
constexpr int WHOLE_BLOCKS = 6;
constexpr int PAGES = BLK / PAGE_TOKENS;
constexpr int AHEAD = 32 / PAGES;               // blocks whose pages are asked for together

struct MergeRecord8 {            // written by the CTA that has a cut unit's first part
  int32_t n_parts;               // 0: none
  int32_t row0, flat0, n_rows;   // the prompt's first row; first of the tile's rows (node x head of the KV head), their number
  int32_t head0;
  int32_t pad[3];
};
static_assert(sizeof(MergeRecord8) == 32, "WS_MERGE");

struct Tree8Params {
  Kv8View kv;
  TreeRows rows;
  int32_t n_q_heads, group, small, over, whole, heads_a_page;
  uint32_t group_inverse;        // 2^32 / group, rounded up; 0: group is 1
  float scale_log2;
  const void* q;
  int64_t q_stride;
  void* out;
  int64_t out_stride;
  float* lse;
  int* err_word;
  MergeRecord8* merges;
  float *partial_ml, *partial_o;
};

// A wait that is mostly over when it is asked for: test_wait answers in 120 clocks, try_wait, which can suspend, in 190 (chains of 7 on 2 x 33024 slots
// 38.1 -> 37.2 us; in the products' warps, one token on 512 slots 7.75 -> 7.57, but trees of 26 on 64 x 2500 slots 122.0 -> 123.1, so with 16 columns only).
__device__ __forceinline__ bool ready_wait(uint64_t* bar, uint32_t parity, int* err_word, int code) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
  return ok != 0 || bar_wait(bar, parity, err_word, code);
}

template <int V> using Const = std::integral_constant<int, V>;
template <int NC, bool BF16> struct Parts {
  static constexpr int Q = BF16 ? 2 : 3, P = BF16 ? 3 : 4;
  // Columns: rows c and c + 1 (c even) have c * Q + 2 * part and the one behind it of S, c * P + 2 * part and the one behind it of O
  static constexpr int NS = NC * Q, NO = NC * P;
  static constexpr int P_ROW = NO <= 64 ? 64 : 128;            // bytes of a slot's row of P in shared memory
  // O of (item parity, block parity); one item's at a time where tensor memory does not hold two
  static constexpr int O_ITEMS = 2 * NS + 4 * NO <= 512 ? 2 : 1;
  static constexpr int USED = 2 * NS + 2 * O_ITEMS * NO;
  static constexpr int TMEM = USED <= 256 ? 256 : 512;
  static_assert(USED <= 512 && NS % 16 == 0 && NO % 16 == 0 && NO <= P_ROW, "");
  __host__ __device__ static constexpr float worth(int part) { return 1.0f / static_cast<float>(1 << 4 * part); }    // of a part of P
};

__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<const __half2*>(&x); }
// A number of 5 exponent bits and 2 mantissa bits is a half's upper byte.  Two halves rounded to such numbers, to nearest, ties away from zero.  (NaN becomes
// zero here; the row sum has it, by which all of the row is divided.)  By conversions, fp16 trees of 26 on 64 x 2500 slots take 163 us, so 158.
__device__ __forceinline__ uint32_t upper_bytes(uint32_t h) { return (h + 0x00800080u) & 0xff00ff00u; }
__device__ __forceinline__ uint32_t bits_of(__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); }
// The parts of two weights (at most 2^15), two halves each whose upper bytes count.  What a part leaves is at most 2^11 and exact in a half, also as 16
// times as much: a multiple of the last bit.  bf16 takes the weight as a half, whose own rounding (2^-12 of the next power of two) is less than the parts'; fp16's
// four keep more, so what its first part leaves is taken from the weight itself.
template <typename X, bool BF16>
__device__ __forceinline__ void split_weights(float w0, float w1, uint32_t (&out)[X::P]) {
  const __half2 sixteen = __float2half2_rn(16.f);
  __half2 r = __floats2half2_rn(w0, w1);
  out[0] = upper_bytes(bits_of(r));
  if constexpr (BF16) {
    r = __hmul2(__hsub2(r, as_half2(out[0])), sixteen);
  } else {
    float r0, r1;
    unpack_f32x2(mul_f32x2(pack_f32x2(w0, w1), pack_f32x2(16.f, 16.f)), r0, r1);
    // less 16 times (0xcc00 is -16) the part, fp32 from halves
    asm("{\n .reg .b16 lo, hi, m;\n mov.b32 {lo, hi}, %2;\n mov.b16 m, 0xcc00;\n fma.rn.f32.f16 %0, lo, m, %0;\n fma.rn.f32.f16 %1, hi, m, %1;\n}\n"
        : "+f"(r0), "+f"(r1) : "r"(out[0]));
    r = __floats2half2_rn(r0, r1);
  }
#pragma unroll
  for (int part = 1; part < X::P; ++part) {
    out[part] = upper_bytes(bits_of(r));
    if (part + 1 < X::P) r = __hmul2(__hsub2(r, as_half2(out[part])), sixteen);
  }
}

// N consecutive columns of the warp's 32 lanes, N a multiple of 4.
template <int N>
__device__ __forceinline__ void tmem_columns(uint32_t at, uint32_t* x) {
  if constexpr (N >= 16) {
    tmem_ld_32x16(at, *reinterpret_cast<uint32_t(*)[16]>(x));
    if constexpr (N > 16) tmem_columns<N - 16>(at + 16, x + 16);
  } else {
    tmem_ld_32x4(at, *reinterpret_cast<uint32_t(*)[4]>(x));
    if constexpr (N > 4) tmem_columns<N - 4>(at + 4, x + 4);
  }
}

// With 16 columns a block's time is its copy's, whatever its rows; with 32 it is the softmax's and goes with them (0.53 us with 4 rows,
// 0.78 with 32, so 4 + rows / 4, of a prompt's tiles on average): trees of 26 on 64 x 2500 slots 123.7 us, every block alike 129.3; rows / 3 124.5.
constexpr int max_blk_cost(int columns) { return columns == 16 ? 1 : 12; }
template <int NC>
__device__ __forceinline__ Shape shape8(const Tree8Params& a, const SeqPart& p) {
  if (p.n_nodes == 0) return Shape{0, 0, 1, 0};
  const int rows = p.n_nodes * a.group, tiles = (rows + NC - 1) / NC, units = tiles * a.kv.n_kv_heads, n_blk = (p.ctx_len + p.n_nodes + BLK - 1) / BLK;
  const int c = NC == 16 ? 1 : 4 + (tiles == 1 ? rows >> 2 : tiles == 2 ? rows >> 3 : 7);
  return a.whole ? Shape{units, 1, n_blk * c, a.over} : Shape{units, n_blk, c, a.over};
}
// Row / group: exact below 2^32 / group.
__device__ __forceinline__ int node_of(const Tree8Params& a, int flat) { return a.group_inverse ? static_cast<int>(__umulhi(static_cast<uint32_t>(flat), a.group_inverse)) : flat; }
struct Item {
  int seq, ctx_len, n_nodes, row0;   // the prompt: its context slots, nodes, first row
  int flat0, n_rows;                 // the tile: rows flat0 .. flat0 + n_rows - 1 of the KV head's node x head rows
  int g, blk_begin, blk_end, n_blk;
  int unit_end;
};
template <int NC>
__device__ __forceinline__ bool next_item(Cursor& cur, const Tree8Params& a, Item* it) {
  Piece pc;
  if (!cur.next<NC == 16>(a.rows, [&](const SeqPart& p) { return shape8<NC>(a, p); }, &pc)) return false;
  // the tiles of one KV head follow each other: they share K and V in L2
  const int flat = pc.part.n_nodes * a.group, tiles = (flat + NC - 1) / NC, tile = pc.unit % tiles;
  it->seq = pc.seq; it->ctx_len = pc.part.ctx_len; it->n_nodes = pc.part.n_nodes; it->row0 = pc.part.row0;
  it->flat0 = tile * NC;
  it->n_rows = min(NC, flat - it->flat0);
  it->g = pc.unit / tiles;
  it->blk_begin = pc.blk_begin; it->blk_end = pc.blk_end; it->n_blk = pc.n_blk; it->unit_end = pc.unit_end;
  if (a.whole) it->blk_end = it->n_blk = (it->ctx_len + it->n_nodes + BLK - 1) / BLK;
  return true;
}

// A sum or maximum of every column by the warp, where the first four columns may be all that counts.
template <int NC, typename Op>
__device__ __forceinline__ float column_reduce(const float (&in)[NC], int n_rows, Op op) {
  if (n_rows > 4) return column_reduce<NC>(in, op);
  const float few[4] = {in[0], in[1], in[2], in[3]};
  return column_reduce<4>(few, op);
}
// The warp's largest x (NaN passed over).
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
// NaN if a drafted V element (slots s .. end - 1) that a row sees is NaN: it was taken out of the product.
template <int D>
__device__ __noinline__ float bad_v(const Tree8Params& a, int seq, int ctx_len, int n_nodes, int s, int end, int row, int node, int g, int col) {
#pragma unroll 1
  for (; s < end; ++s) {
    if (!(node_bits(a.rows, row, node, n_nodes, s - ctx_len) & 1u)) continue;
    const int page = ld_dep_s32(a.kv.page_table + static_cast<size_t>(seq) * a.kv.pt_stride + s / PAGE_TOKENS);
    if (page < 0 || page >= a.kv.n_pages) continue;
    const uint8_t* v = static_cast<const uint8_t*>(a.kv.pages) + page * a.kv.page_stride + (static_cast<size_t>(g) * 2 + 1) * (PAGE_TOKENS * D);
    if ((v[(s % PAGE_TOKENS) * D + col] & 0x7f) == 0x7f) return __uint_as_float(0x7fffffffu);
  }
  return 0.f;
}

// Byte b of row n of an operand with rows of W bytes (64 or 128) in the swizzle of that width.
template <int W>
__device__ __forceinline__ int swizzled(int n, int b) {
  const int off = n * W + b;
  return off ^ (W == 128 ? ((off >> 7) & 7) << 4 : ((off >> 7) & 3) << 4);
}

// Rows c0, c0 + step, .. (a warp takes 512 / D of them at a time) of a tile's q as sums of e4m3 numbers, and what those count.  A lane has 16 elements of
// a row.  Rows behind the last one, up to four or sixteen (what the softmax takes at a time), become zeros.
template <int D, int NC, bool BF16>
__device__ __noinline__ void split_q(const Tree8Params& a, int row0, int flat0, int n_rows, int g, uint8_t* q_smem, float* q_scale, int c0, int step) {
  using X = Parts<NC, BF16>;
  constexpr int LANES = D / 16;
  const int lane = threadIdx.x & 31, l = lane % LANES;
  const int last = n_rows & 15, n_zero = last == 0 ? n_rows : n_rows - last + (last <= 4 ? 4 : 16);
#pragma unroll 2
  for (; c0 < n_zero; c0 += step) {
    const int c = c0 + lane / LANES;
    uint4 raw[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (c < n_rows) {
      const int flat = flat0 + c, node = node_of(a, flat);
      const unsigned short* src = static_cast<const unsigned short*>(a.q) + (row0 + node) * a.q_stride + (g * a.group + flat - node * a.group) * D + l * 16;
      raw[0] = ld_dep_v4(src);
      raw[1] = ld_dep_v4(src + 8);
    }
    float x[16], amax = 0.f;
    const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const uint32_t bits = (w[e >> 1] >> (16 * (e & 1))) & 0xffffu;
      if constexpr (BF16) x[e] = __uint_as_float(bits << 16);
      else x[e] = __half2float(__ushort_as_half(static_cast<unsigned short>(bits)));
      const float m = fabsf(x[e]);
      if (m < INFINITY) amax = fmaxf(amax, m);
      else x[e] = __uint_as_float(0x7fffffffu);                // infinity times anything ends as NaN
    }
#pragma unroll
    for (int o = LANES / 2; o >= 1; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    const uint32_t b = __float_as_uint(amax);
    const int ex = min(max(static_cast<int>(b >> 23) - 135 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0), -100), 120);
    const float down = __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
    if (c < n_zero) {
      if (l == 0) q_scale[c] = __uint_as_float(static_cast<uint32_t>(127 + ex) << 23) * a.scale_log2;
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] *= down;
#pragma unroll
      for (int part = 0; part < X::Q; ++part) {
        uint32_t out[4];
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const uint32_t lo = pack_e4m3x2(x[e], x[e + 1]), hi = pack_e4m3x2(x[e + 2], x[e + 3]);
          out[e >> 2] = lo | hi << 16;
          const float2 y = unpack_e4m3x2(lo), z = unpack_e4m3x2(hi);
          x[e] = (x[e] - y.x) * 16.f; x[e + 1] = (x[e + 1] - y.y) * 16.f;
          x[e + 2] = (x[e + 2] - z.x) * 16.f; x[e + 3] = (x[e + 3] - z.y) * 16.f;
        }
        *reinterpret_cast<uint4*>(q_smem + swizzled<D>((c & ~1) * X::Q + part * 2 + (c & 1), l * 16)) = make_uint4(out[0], out[1], out[2], out[3]);
      }
    }
  }
  fence_proxy_async_smem();                                    // the MMA reads Q through the async proxy
}

template <int D, int NC, bool BF16>
constexpr int smem8() { return 1024 + ring_bytes(NC) + 2 * Parts<NC, BF16>::NS * D + 2 * Parts<NC, BF16>::P_ROW * BLK; }

template <int D, int NC, bool BF16>
__global__ void __launch_bounds__(TREE_THREADS, 1)
attention_8bit_kernel(const __grid_constant__ CUtensorMap tm, const __grid_constant__ Tree8Params a) {
  using X = Parts<NC, BF16>;
  constexpr int GROUP_BYTES = 8 * D;                           // eight rows of K or V
  constexpr int SBO = 2 * GROUP_BYTES;                         // K and V take turns
  constexpr int STAGE_BYTES = BLK * 2 * D;
  constexpr int STAGES = ring_bytes(NC) / STAGE_BYTES;
  constexpr int Q_BYTES = X::NS * D, P_BYTES = X::P_ROW * BLK;
  constexpr uint32_t TMEM_O = 2 * X::NS;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t q_full[2], q_empty[2], landed[STAGES], empty[STAGES], dirty[CLEAN_BARS], cleaned[CLEAN_BARS], s_full[2], s_free[2], p_full[2], p_free[2],
      o_full[2], o_free[2], ml_full, q_first;
  __shared__ __align__(16) float4 page_scale[STAGES][PAGES];   // s_K, log2 s_V, 1 / s_V
  __shared__ __align__(16) float q_scale[2][NC];
  __shared__ __align__(16) float block_max[2][2][NC][4];       // [block parity][use][row][warp]
  __shared__ __align__(16) float fin_l[2][2][NC][4];           // [item parity][block parity][row][warp]: a warp's share of the sum
  __shared__ float fin_m[2][2][NC];
  __shared__ __align__(16) float neg_ref[8][NC];                // - reference, a copy per softmax warp; at a piece's end the rows' first factor
  __shared__ __align__(16) float other_factor[8][NC];
  using RowBits = std::conditional_t<NC == 16, uint16_t, uint32_t>;
  __shared__ RowBits seen_by[2][MAX_NODES];               // the tile's rows that see a node
  __shared__ int bad_flag[FLAGS];
  __shared__ Span shared_span;
  __shared__ int64_t warp_sums[TREE_THREADS / 32];
  __shared__ uint32_t tmem_slot;
  __shared__ int cta_failed;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* q_smem = ring + ring_bytes(NC);
  uint8_t* p_smem = q_smem + 2 * Q_BYTES;

  if (threadIdx.x == 0) {
    cta_failed = 0;
    for (int i = 0; i < STAGES; ++i) { mbar_init(&landed[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < CLEAN_BARS; ++i) { mbar_init(&dirty[i], 1); mbar_init(&cleaned[i], 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 1);
      mbar_init(&q_empty[i], 9);         // the MMAs and the eight softmax warps
      mbar_init(&s_full[i], 2); mbar_init(&s_free[i], 4); mbar_init(&p_full[i], 4); mbar_init(&p_free[i], 1);
      mbar_init(&o_full[i], 1); mbar_init(&o_free[i], 8);
    }
    mbar_init(&ml_full, 8); mbar_init(&q_first, 8);
    fence_mbar_init();
  }
  if (warp == 9) {
    tmem_alloc<X::TMEM>(&tmem_slot);
    tmem_relinquish();
  }
  if (warp == 8 && lane == 0) prefetch_tmap(&tm);
  pdl_launch_dependents();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  pdl_wait();                          // lengths, tables, pages and q may come from the kernel before
  const Span span = make_span(a.rows, MIN_SPAN<NC>, a.small, &shared_span, warp_sums, [&](const SeqPart& p) { return shape8<NC>(a, p); });
  const uint32_t tmem = tmem_slot;
  Cursor cur(span);
  Item it{};

  if (warp == 8) {
    // ------------------------------------------------------------ copies
    uint32_t st = 0, phase = 0;
    MergeRecord8 rec{};
    bool ok = true;
    while (ok && next_item<NC>(cur, a, &it)) {
      const int last_page = (it.ctx_len + it.n_nodes - 1) / PAGE_TOKENS;
      const int32_t* table = a.kv.page_table + static_cast<size_t>(it.seq) * a.kv.pt_stride;
      // A lane has a page, of four blocks at a time: its id, asked for four blocks ahead, and scales.
      // Pages behind the prompt's last slot repeat its last page (masked either way); ids outside the pool become one that copies zeros.
      auto page_at = [&](int blk) {
        const int page = ld_dep_s32(table + min(blk * PAGES + lane, last_page));
        return static_cast<int>(min(static_cast<uint32_t>(page), static_cast<uint32_t>(a.kv.n_pages)));
      };
      int page = page_at(it.blk_begin);
#pragma unroll 1
      for (int blk0 = it.blk_begin; blk0 < it.blk_end && ok; blk0 += AHEAD) {
        const int next_page = page_at(blk0 + AHEAD);
        float4 sc = make_float4(0.f, 0.f, 0.f, 0.f);
        const int n = min(AHEAD, it.blk_end - blk0);
#pragma unroll 1
        for (int u = 0; u < n; ++u) {
          ok = __all_sync(0xffffffffu, bar_wait(&empty[st], phase ^ 1u, a.err_word, DEV_ERR_ATTN_PRODUCER));
          if (!ok) break;
          int id[PAGES];
#pragma unroll
          for (int p = 0; p < PAGES; ++p) id[p] = __shfl_sync(0xffffffffu, page, u * PAGES + p);
          if (elect_one()) {
#pragma unroll
            for (int p = 0; p < PAGES; ++p)
              tma_load_5d(ring + st * STAGE_BYTES + p * (PAGE_TOKENS * 2 * D), &tm, &landed[st], 0, 0, 0, 0, id[p] * a.heads_a_page + it.g);
          }
          __syncwarp();
          if (u == 0) {                                              // while the tile is on its way
            float2 x = make_float2(1.f, 1.f);
            if (page < a.kv.n_pages) x = ld_dep_f32x2(a.kv.scales + (static_cast<size_t>(page) * a.kv.n_kv_heads + it.g) * 2);
            const float v = fminf(fmaxf(x.y, 0x1p-32f), 0x1p32f);
            sc = make_float4(fminf(fmaxf(x.x, 0x1p-32f), 0x1p32f), __log2f(v), 1.0f / v, 0.f);
          }
          if (lane / PAGES == u) page_scale[st][lane % PAGES] = sc;
          __syncwarp();
          if (elect_one()) mbar_arrive_expect_tx(&landed[st], STAGE_BYTES);     // the scales are out, too
          __syncwarp();
          if (++st == STAGES) { st = 0; phase ^= 1u; }
        }
        page = next_page;
      }
      if (it.blk_begin == 0 && it.blk_end < it.n_blk) {              // the rest of this unit is other CTAs' work
        rec.n_parts = static_cast<int>(static_cast<uint64_t>((span.begin + it.unit_end) * span.n_ctas - 1) / static_cast<uint64_t>(span.total)) -
                      static_cast<int>(blockIdx.x) + 1;
        rec.row0 = it.row0; rec.flat0 = it.flat0; rec.n_rows = it.n_rows; rec.head0 = it.g * a.group;
      }
    }
    if (!ok) cta_failed = 1;
    if (lane == 0) a.merges[blockIdx.x] = rec;
  } else if (warp == 11) {
    // ------------------------------------------------------------ Q into parts, masks, V without what does not count
    constexpr int LANES = D / 16;                                  // a lane has 16 elements of a row
    uint32_t n_q = 0, n_item = 0, n_tile = 0, n_clean = 0;
    bool ok = true;
    auto prepare_q = [&](const Item& it) {
      const int qs = n_q & 1, node0 = node_of(a, it.flat0);
      int* flag = &bad_flag[n_q % FLAGS];                          // read at the end of its item, long before its next use
      if (lane == 0) *flag = 0;
      ok = __all_sync(0xffffffffu, bar_wait(&q_empty[qs], ((n_q >> 1) & 1u) ^ 1u, a.err_word, DEV_ERR_ATTN_CORR));
      if (!ok) return;
      if (n_q > 0) split_q<D, NC, BF16>(a, it.row0, it.flat0, it.n_rows, it.g, q_smem + qs * Q_BYTES, q_scale[qs], 0, 512 / D);
      if (it.blk_end * BLK > it.ctx_len) {
#pragma unroll 1
        for (int node = lane; node < it.n_nodes; node += 32) {
          uint32_t seen = 0;
          int h = it.flat0 - node0 * a.group, k = node0;           // the tile may begin and end inside a node's heads
#pragma unroll 1
          for (int c = 0; c < it.n_rows; ++k) {
            const int n = min(a.group - h, it.n_rows - c);
            if ((node_word(a.rows, it.row0 + k, k, node >> 6) >> (node & 63)) & 1u) seen |= (0xffffffffu >> (32 - n)) << c;
            c += n;
            h = 0;
          }
          seen_by[qs][node] = static_cast<RowBits>(seen);
        }
        __syncwarp();
      }
      // the first item's Q is the softmax warps' work, who have nothing else to do yet (by one warp: 32 rows 20000 clocks)
      if (n_q == 0) ok = __all_sync(0xffffffffu, bar_wait(&q_first, 0, a.err_word, DEV_ERR_ATTN_CORR));
      if (!ok) return;
      __syncwarp();
      if (elect_one()) mbar_arrive(&q_full[qs]);
      __syncwarp();
      ++n_q;
    };
    // an item's Q is there before the item ahead of it ends (whose V is cleaned last)
    bool more = next_item<NC>(cur, a, &it);
    if (more) prepare_q(it);
    while (ok && more) {
      Item next{};
      more = next_item<NC>(cur, a, &next);
      if (more) prepare_q(next);
      int* flag = &bad_flag[n_item % FLAGS];
      // V: zeros behind the prompt's last slot, and where a drafted V is NaN (with the flag raised)
#pragma unroll 1
      for (int blk = max(it.blk_begin, it.ctx_len / BLK); ok && blk < it.blk_end; ++blk) {
        const uint32_t t = n_tile + blk - it.blk_begin;
        // not on `landed`: this warp passes over most tiles, and a parity says nothing about a phase that is not the next one
        ok = __all_sync(0xffffffffu, bar_wait(&dirty[n_clean % CLEAN_BARS], (n_clean / CLEAN_BARS) & 1u, a.err_word, DEV_ERR_ATTN_CORR));
        if (!ok) break;
        uint8_t* v = ring + (t % STAGES) * STAGE_BYTES + GROUP_BYTES;
        const int r0 = max(it.ctx_len - blk * BLK, 0), r_end = it.ctx_len + it.n_nodes - blk * BLK;
        bool bad = false;
        // a lane takes a 16-byte vector (as stored; the swizzle only permutes a row group's vectors) of rows 32 / LANES apart
        auto vector = [&](int r) { return reinterpret_cast<uint4*>(v + (r >> 3) * SBO + swizzled<D>(r & 7, (lane % LANES) * 16)); };
#pragma unroll 4
        for (int r = max(r_end, 0) + lane / LANES; r < BLK; r += 32 / LANES) *vector(r) = make_uint4(0, 0, 0, 0);
#pragma unroll 4
        for (int r = r0 + lane / LANES; r < min(r_end, BLK); r += 32 / LANES) {
          const uint4 x = *vector(r);
          uint32_t w[4] = {x.x, x.y, x.z, x.w}, any = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t nan = ((w[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
            any |= nan;
            w[e] &= ~((nan >> 7) * 0xffu);
          }
          if (any) { *vector(r) = make_uint4(w[0], w[1], w[2], w[3]); bad = true; }
        }
        if (bad) *reinterpret_cast<volatile int*>(flag) = 1;
        fence_proxy_async_smem();
        __syncwarp();
        if (elect_one()) mbar_arrive(&cleaned[n_clean % CLEAN_BARS]);
        __syncwarp();
        ++n_clean;
      }
      n_tile += it.blk_end - it.blk_begin;
      ++n_item;
      it = next;
    }
    if (!ok) cta_failed = 1;
  } else if (warp == 9 || warp == 10) {
    // ------------------------------------------------------------ MMAs: the whole warp walks, one lane issues
    auto desc = [](uint32_t addr, uint32_t sbo) { return D == 128 ? make_smem_desc_sw128(addr, 0, sbo) : make_smem_desc_sw64(addr, 0, sbo); };
    uint32_t n_item = 0, n_tile = 0, n_dirty = 0, phases = 0;     // phases: bit i, the parity to wait for on the barrier of block parity i
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (ok) ok = __all_sync(0xffffffffu, NC == 16 ? ready_wait(bar, parity, a.err_word, DEV_ERR_ATTN_MMA) : bar_wait(bar, parity, a.err_word, DEV_ERR_ATTN_MMA));
    };
    while (ok && next_item<NC>(cur, a, &it)) {
      const int nb = it.blk_end - it.blk_begin, par = n_item & 1;
      if (warp == 9) {
        const uint32_t idesc = make_idesc_8bit(BLK, (((it.n_rows + 1) & ~1) * X::Q + 15) & ~15, E4M3, E4M3, 0, 0);
        const uint64_t q_desc = desc(smem_u32(q_smem + par * Q_BYTES), GROUP_BYTES);
        wait(&q_full[par], (n_item >> 1) & 1u);
#pragma unroll 1
        for (int j = 0; j < nb && ok; ++j) {
          const uint32_t t = n_tile + j;
          const int i = j & 1;
          wait(&s_free[i], ((phases >> i) & 1u) ^ 1u);
          phases ^= 1u << i;
          wait(&landed[t % STAGES], (t / STAGES) & 1u);
          if (!ok) break;
          tc_fence_after_sync();
          if (elect_one()) {
            const uint64_t k_desc = desc(smem_u32(ring + (t % STAGES) * STAGE_BYTES), SBO);
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk)
              umma_ss_8bit(tmem + i * X::NS, k_desc + (kk * 32 >> 4), q_desc + (kk * 32 >> 4), idesc, kk != 0);
            umma_commit(&s_full[i]);
            mbar_arrive(&s_full[i]);           // and what this warp has seen to arrive: the pages' scales
            if (j + 1 == nb) umma_commit(&q_empty[par]);
            if ((it.blk_begin + j + 1) * BLK > it.ctx_len) mbar_arrive(&dirty[n_dirty % CLEAN_BARS]);
          }
          __syncwarp();
          if ((it.blk_begin + j + 1) * BLK > it.ctx_len) ++n_dirty;
        }
      } else {
        const int ob = X::O_ITEMS == 2 ? par : 0;
        const uint32_t o_uses = X::O_ITEMS == 2 ? n_item >> 1 : n_item;
        const uint32_t idesc = make_idesc_8bit(BLK, (((it.n_rows + 1) & ~1) * X::P + 15) & ~15, E4M3, E5M2, 1, 1);     // A = V^T, B = P^T: the K index is the slot
        wait(&o_free[ob], (o_uses & 1u) ^ 1u);
#pragma unroll 1
        for (int j = 0; j < nb && ok; ++j) {
          const uint32_t t = n_tile + j;
          const int i = j & 1;
          wait(&p_full[i], (phases >> i) & 1u);
          phases ^= 1u << i;
          if ((it.blk_begin + j + 1) * BLK > it.ctx_len) {
            wait(&cleaned[n_dirty % CLEAN_BARS], (n_dirty / CLEAN_BARS) & 1u);
            ++n_dirty;
          }
          if (!ok) break;
          tc_fence_after_sync();
          if (elect_one()) {
            // head size 64 has 64 elements of M in a row: the second 64 TMEM lanes repeat the first (distance 0) and are not read
            const uint64_t v_desc = desc(smem_u32(ring + (t % STAGES) * STAGE_BYTES + GROUP_BYTES), SBO);
            const uint32_t p_at = smem_u32(p_smem + i * P_BYTES);
            const uint64_t p_desc = X::P_ROW == 128 ? make_smem_desc_sw128(p_at, 0, 1024) : make_smem_desc_sw64(p_at, 0, 512);
#pragma unroll
            for (int kk = 0; kk < BLK / 32; ++kk)
              umma_ss_8bit(tmem + TMEM_O + (ob * 2 + i) * X::NO, v_desc + (kk * 4 * SBO >> 4), p_desc + (kk * 32 * X::P_ROW >> 4), idesc, j > 1 || kk != 0);
            umma_commit(&empty[t % STAGES]);
            umma_commit(&p_free[i]);
            if (j + 1 == nb) umma_commit(&o_full[ob]);
          }
          __syncwarp();
        }
      }
      n_tile += nb;
      ++n_item;
    }
    if (!ok) cta_failed = 1;
  } else {
    // ------------------------------------------------------------ softmax (warps 0-7).  The four warps of a parity meet at a hardware
    // barrier in every block, so a warp whose wait ran out keeps walking the blocks, without waiting or computing, to the end.
    const int i = warp >> 2, quarter = warp & 3;
    const int r = quarter * 32 + lane;                     // slot of the block; element of the head
    const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    uint8_t* p_row = p_smem + i * P_BYTES;
    uint32_t n_item = 0, n_tile = 0, n_s = 0, n_raise = 0;
    bool ok = true;
    while (next_item<NC>(cur, a, &it)) {
      const int nb = it.blk_end - it.blk_begin, par = n_item & 1, ob = X::O_ITEMS == 2 ? par : 0;
      const uint32_t o_uses = X::O_ITEMS == 2 ? n_item >> 1 : n_item;
      uint64_t l[NC / 2];                                  // two rows' sums over this thread's slots only
      float* neg = neg_ref[warp];                          // - reference: the same in all threads
      uint32_t unset = 0xffffffffu >> (32 - it.n_rows);    // rows that have seen nothing yet: reference 0, sum and O zero
#pragma unroll
      for (int c = 0; c < NC / 2; ++c) l[c] = 0u;
      if (lane < NC) neg[lane] = lane < it.n_rows ? 0.f : -INFINITY;         // columns behind the last row get no weights
      __syncwarp();
      if (n_item == 0) {
        split_q<D, NC, BF16>(a, it.row0, it.flat0, it.n_rows, it.g, q_smem, q_scale[0], warp * (512 / D), 8 * (512 / D));
        __syncwarp();
        if (elect_one()) mbar_arrive(&q_first);
        __syncwarp();
      }
      if (ok) ok = __all_sync(0xffffffffu, bar_wait(&q_full[par], (n_item >> 1) & 1u, a.err_word, DEV_ERR_ATTN_SOFTMAX));     // scales, masks
      for (int j = i; j < nb; j += 2) {
        if (ok) ok = __all_sync(0xffffffffu, ready_wait(&s_full[i], n_s & 1u, a.err_word, DEV_ERR_ATTN_SOFTMAX));
        float t[NC];                                       // scores in base 2, the page's log2 s_V added, less the reference
        float inv_v = 0.f;
        bool raise = j == i;                               // does any row's block maximum pass what its reference allows
        if (ok) {
          tc_fence_after_sync();
          const float4 sc = page_scale[(n_tile + j) % STAGES][r / PAGE_TOKENS];
          inv_v = sc.z;
          const uint64_t sc_k = pack_f32x2(sc.x, sc.x), sc_v = pack_f32x2(sc.y, sc.y), sixteenth = pack_f32x2(0.0625f, 0.0625f);
          // sixteen rows at a time, or four where there are no more: straight code, so that their latencies overlap
          auto scores = [&](auto rows, int c0) {
            constexpr int R = decltype(rows)::value;
            uint32_t x[R * X::Q];
            tmem_columns<R * X::Q>(lanes + i * X::NS + c0 * X::Q, x);
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < R; c += 4) {
              const float4 q4 = *reinterpret_cast<const float4*>(&q_scale[par][c0 + c]), n4 = *reinterpret_cast<const float4*>(neg + c0 + c);
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                auto column = [&](int part) {
                  const int at = (c + 2 * u) * X::Q + part * 2;
                  return pack_f32x2(__uint_as_float(x[at]), __uint_as_float(x[at + 1]));
                };
                uint64_t y = column(X::Q - 1);
#pragma unroll
                for (int part = X::Q - 2; part >= 0; --part) y = fma_f32x2(y, sixteenth, column(part));
                const uint64_t by = mul_f32x2(sc_k, u ? pack_f32x2(q4.z, q4.w) : pack_f32x2(q4.x, q4.y));
                const uint64_t plus = add_f32x2(sc_v, u ? pack_f32x2(n4.z, n4.w) : pack_f32x2(n4.x, n4.y));
                unpack_f32x2(fma_f32x2(y, by, plus), t[c0 + c + 2 * u], t[c0 + c + 2 * u + 1]);
              }
            }
          };
#pragma unroll
          for (int c0 = 0; c0 < NC; c0 += 16) {
            if (it.n_rows > c0 + 4) {
              scores(Const<16>{}, c0);
            } else {
#pragma unroll
              for (int c = c0; c < c0 + 16; ++c) t[c] = -INFINITY;
              if (it.n_rows > c0) scores(Const<4>{}, c0);
            }
          }
          tc_fence_before_sync();
          __syncwarp();
          if (elect_one()) mbar_arrive(&s_free[i]);
          __syncwarp();
          const int slot = (it.blk_begin + j) * BLK + r;
          if (slot >= it.ctx_len) {
            const int node = slot - it.ctx_len;
            const uint32_t seen = node < it.n_nodes ? seen_by[par][node] : 0u;
#pragma unroll
            for (int c = 0; c < NC; ++c)
              if (!((seen >> c) & 1u)) t[c] = -INFINITY;
          }
          __syncwarp();
          if (j != i) {                                    // (the first block always sets the references)
            float top = -INFINITY;
#pragma unroll
            for (int c0 = 0; c0 < NC; c0 += 16) {
              if (it.n_rows > c0) {
                top = fmax3(top, t[c0], t[c0 + 1]);
                top = fmax3(top, t[c0 + 2], t[c0 + 3]);
              }
              if (it.n_rows > c0 + 4) {
#pragma unroll
                for (int c = 4; c < 16; c += 2) top = fmax3(top, t[c0 + c], t[c0 + c + 1]);
              }
            }
            raise = top > HEADROOM + RESCALE_THRESHOLD;
            if (unset != 0) {
#pragma unroll
              for (int c = 0; c < NC; ++c) raise |= ((unset >> c) & 1u) && t[c] > -INFINITY;
            }
          }
        }
        if (j != i) raise = parity_any(i, raise);
        if (raise) {
          // The rows' exact block maxima: a warp's by one instruction a row, the block's from four words a row; lane c then works
          // out row c's new reference, every thread reads it from shared memory, and what the present scores lose comes by shuffles.  Two
          // buffers: between two uses of one lies the other's barrier.
          float(*maxima)[4] = block_max[i][n_raise++ & 1];
          float mine = -INFINITY;                          // lane c: row c's
#pragma unroll
          for (int c0 = 0; c0 < NC; c0 += 4) {
            if (c0 >= it.n_rows) break;
#pragma unroll
            for (int c = c0; c < c0 + 4; ++c) {
              const float m = warp_max(t[c]);
              mine = lane == c ? m : mine;
            }
          }
          if (lane < NC) maxima[lane][quarter] = mine;
          parity_any(i, false);
          const float4 x = *reinterpret_cast<const float4*>(maxima[lane % NC]);
          const float old = lane < NC ? neg[lane] : 0.f;
          const float over = fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w)) - HEADROOM;             // the block's own reference, less the present one
          const bool fresh = (unset >> lane) & 1u;
          const bool up = lane < it.n_rows && over > -INFINITY && (fresh || over > RESCALE_THRESHOLD);
          const float alpha = !up ? 1.f : fresh ? 0.f : fast_exp2(-over);
          const float less = up ? over : 0.f;
          __syncwarp();
          if (up) neg[lane] = old - over;
          unset &= ~(__ballot_sync(0xffffffffu, up));
          __syncwarp();
#pragma unroll
          for (int c = 0; c < NC; ++c) t[c] -= __shfl_sync(0xffffffffu, less, c);
          if (j != i) {
            if (ok) ok = __all_sync(0xffffffffu, ready_wait(&p_free[i], (n_s & 1u) ^ 1u, a.err_word, DEV_ERR_ATTN_SOFTMAX));    // O is complete
            if (ok) {
              tc_fence_after_sync();
#pragma unroll 1
              for (int c0 = 0; c0 < NC; c0 += 4) {
                if (c0 >= it.n_rows) break;
                const uint32_t t_o = lanes + TMEM_O + (ob * 2 + i) * X::NO + c0 * X::P;
                float f[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = __shfl_sync(0xffffffffu, alpha, c0 + e);
                uint32_t o[4 * X::P];
                tmem_columns<4 * X::P>(t_o, o);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 4 * X::P; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f[e / (2 * X::P) * 2 + (e & 1)]);
#pragma unroll
                for (int e = 0; e < 4 * X::P; e += 4) tmem_st_32x4(t_o + e, *reinterpret_cast<uint32_t(*)[4]>(o + e));
              }
              tmem_wait_st();
#pragma unroll
              for (int c = 0; c < NC; c += 2) l[c / 2] = mul_f32x2(l[c / 2], pack_f32x2(__shfl_sync(0xffffffffu, alpha, c), __shfl_sync(0xffffffffu, alpha, c + 1)));
            }
          }
        }
        if (ok) ok = __all_sync(0xffffffffu, ready_wait(&p_free[i], (n_s & 1u) ^ 1u, a.err_word, DEV_ERR_ATTN_SOFTMAX));     // the product before has read P
        ++n_s;
        if (ok) {
          const uint64_t inv_v2 = pack_f32x2(inv_v, inv_v);
          auto weights = [&](auto rows, int c0) {          // of rows c0 ..: the slot's row of P, two rows' parts a half word
            constexpr int R = decltype(rows)::value, WORDS = (R * X::P + 15) / 16 * 4;
            uint32_t w[WORDS];
#pragma unroll
            for (int e = 0; e < WORDS; ++e) w[e] = 0u;
#pragma unroll
            for (int c = 0; c < R; c += 4) {
              uint32_t two[2][X::P];
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const int k = c0 + c + 2 * u;
                const float w0 = fast_exp2(t[k]), w1 = fast_exp2(t[k + 1]);
                l[k / 2] = fma_f32x2(pack_f32x2(w0, w1), inv_v2, l[k / 2]);   // the row sum has the weights without s_V, and before they are split
                split_weights<X, BF16>(w0, w1, two[u]);
              }
#pragma unroll
              for (int e = 0; e < X::P; ++e) {
                const int lo = 2 * e, hi = 2 * e + 1;
                w[c * X::P / 4 + e] = __byte_perm(two[lo / X::P][lo % X::P], two[hi / X::P][hi % X::P], 0x7531);
              }
            }
#pragma unroll
            for (int q = 0; q < WORDS / 4; ++q)
              *reinterpret_cast<uint4*>(p_row + swizzled<X::P_ROW>(r, c0 * X::P + q * 16)) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
          };
#pragma unroll
          for (int c0 = 0; c0 < NC; c0 += 16) {
            if (it.n_rows > c0 + 4) weights(Const<16>{}, c0);
            else if (it.n_rows > c0) weights(Const<4>{}, c0);
          }
          fence_proxy_async_smem();                        // the MMA reads P through the async proxy
          tc_fence_before_sync();
          __syncwarp();
          if (elect_one()) mbar_arrive(&p_full[i]);
        }
      }
      n_tile += nb;
      // ---- the piece's end: sums and references of both parities are exchanged; parity i writes rows i * 4 .. i * 4 + 3, i * 4 + 8 ...
      if (ok) {
        float ll[NC];
#pragma unroll
        for (int c = 0; c < NC; c += 2) unpack_f32x2(l[c / 2], ll[c], ll[c + 1]);
        const float sum = column_reduce<NC>(ll, it.n_rows, [](float x, float y) { return x + y; });
        if (lane < NC) fin_l[par][i][lane][quarter] = sum;
        const float mine = lane < NC ? -neg[lane] : 0.f;
        if (quarter == 0 && lane < NC) fin_m[par][i][lane] = ((unset >> lane) & 1u) || nb <= i ? -INFINITY : mine;
        __syncwarp();
        if (elect_one()) { mbar_arrive(&ml_full); mbar_arrive(&q_empty[par]); }
        __syncwarp();
        ok = __all_sync(0xffffffffu, bar_wait(&ml_full, par, a.err_word, DEV_ERR_ATTN_CORR));
      }
      const bool whole = it.blk_begin == 0 && it.blk_end == it.n_blk;
      const size_t part0 = static_cast<size_t>(2 * blockIdx.x + (it.blk_begin == 0 ? 1 : 0)) * BLK;
      float f0 = 0.f, f1 = 0.f;
      if (ok) {
        // Lane c works out row c's two factors; the loop over rows then only scales and stores.
        if (lane < it.n_rows) {
          const float m0 = fin_m[par][0][lane], m1 = fin_m[par][1][lane];
          const float4 l0 = *reinterpret_cast<const float4*>(fin_l[par][0][lane]), l1 = *reinterpret_cast<const float4*>(fin_l[par][1][lane]);
          const float M = fmaxf(m0, m1), ref = M == -INFINITY ? 0.f : M;
          f0 = fast_exp2(m0 - ref);
          f1 = nb > 1 ? fast_exp2(m1 - ref) : 0.f;
          float L = f0 * ((l0.x + l0.y) + (l0.z + l0.w));
          if (nb > 1) L = fmaf(f1, (l1.x + l1.y) + (l1.z + l1.w), L);
          const int flat = it.flat0 + lane, node = node_of(a, flat), row = it.row0 + node;
          bool any = it.ctx_len > 0;                       // does the row see a slot at all (not: are its scores all -inf)
          if (!any) any = sees_a_node(a.rows, row, node, it.n_nodes);
          if (whole) {
            const float inv = any ? 1.0f / L : 0.f;        // a row that sees nothing has an O of zeros
            f0 *= inv;
            f1 *= inv;
            if (warp == 0 && a.lse)
              a.lse[static_cast<size_t>(row) * a.n_q_heads + it.g * a.group + flat - node * a.group] = any ? (M + log2f(L)) * LN2 : -INFINITY;
          } else if (warp == 0) {
            *reinterpret_cast<float2*>(a.partial_ml + (part0 + lane) * 2) = make_float2(M, any ? L : -1.f);
          }
        }
      }
      __syncwarp();
      if (lane < NC) { neg[lane] = f0; other_factor[warp][lane] = f1; }      // (the reference is done with)
      __syncwarp();
      if (ok) ok = __all_sync(0xffffffffu, bar_wait(&o_full[ob], o_uses & 1u, a.err_word, DEV_ERR_ATTN_CORR));
      if (ok) {
        tc_fence_after_sync();
        const bool bad = *reinterpret_cast<volatile int*>(&bad_flag[n_item % FLAGS]) != 0;
        __syncwarp();
        int node = node_of(a, it.flat0 + i * 4), h = it.flat0 + i * 4 - node * a.group;
        unsigned short* out = static_cast<unsigned short*>(a.out) + static_cast<int64_t>(it.row0 + node) * a.out_stride + (it.g * a.group + h) * D + r;
        const int64_t next_node = a.out_stride - a.group * D;
        float* partial = a.partial_o + (part0 + i * 4) * HEAD_DIM + r;
#pragma unroll 1
        for (int c0 = i * 4; c0 < it.n_rows; c0 += 8) {    // four rows at a time, the parities in turn
          float o0[4] = {0.f, 0.f, 0.f, 0.f}, o1[4] = {0.f, 0.f, 0.f, 0.f};
          uint32_t x0[4 * X::P], x1[4 * X::P];
          tmem_columns<4 * X::P>(lanes + TMEM_O + ob * 2 * X::NO + c0 * X::P, x0);
          tmem_columns<4 * X::P>(lanes + TMEM_O + (ob * 2 + 1) * X::NO + c0 * X::P, x1);         // not used when there is one block
          const float4 g0 = *reinterpret_cast<const float4*>(neg + c0), g1 = *reinterpret_cast<const float4*>(other_factor[warp] + c0);
          const float f[4] = {g0.x, g0.y, g0.z, g0.w}, w1[4] = {g1.x, g1.y, g1.z, g1.w};
          tmem_wait_ld();
#pragma unroll
          for (int part = X::P - 1; part >= 0; --part) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int at = (e >> 1) * 2 * X::P + part * 2 + (e & 1);
              o0[e] = fmaf(__uint_as_float(x0[at]), X::worth(part), o0[e]);
              o1[e] = fmaf(__uint_as_float(x1[at]), X::worth(part), o1[e]);
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float o = o0[e] * f[e];
            if (nb > 1) o = fmaf(o1[e], w1[e], o);
            if (r < D && c0 + e < it.n_rows) {
              if (bad)
                o += bad_v<D>(a, it.seq, it.ctx_len, it.n_nodes, max(it.ctx_len, it.blk_begin * BLK), min(it.ctx_len + it.n_nodes, it.blk_end * BLK),
                              it.row0 + node, node, it.g, r);
              if (whole) *out = static_cast<unsigned short>(pack_out<BF16>(o, 0.f));
              else partial[e * HEAD_DIM] = o;
            }
            out += D;
            if (++h == a.group) { h = 0; ++node; out += next_node; }
          }
          // the other parity's four rows
          partial += 8 * HEAD_DIM;
          out += 4 * D;
#pragma unroll 1
          for (h += 4; h >= a.group; ++node, out += next_node) h -= a.group;
        }
        tc_fence_before_sync();
        __syncwarp();
        if (elect_one()) mbar_arrive(&o_free[ob]);
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
    tmem_dealloc<X::TMEM>(tmem);
  }
}

// The parts of a cut unit: out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s, one warp per row.
constexpr int MERGE_WARPS = 8;
template <int D, bool BF16>
__global__ void __launch_bounds__(MERGE_WARPS * 32) merge_8bit_kernel(Tree8Params a) {
  constexpr int E = D / 32;                             // columns per lane
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int r = blockIdx.y * MERGE_WARPS + (threadIdx.x >> 5);
  const volatile MergeRecord8* mr = a.merges + blockIdx.x;
  const int n_parts = mr->n_parts, n_rows = mr->n_rows;
  if (n_parts <= 1 || r >= n_rows) return;
  const int flat = mr->flat0 + r, node = node_of(a, flat), row = mr->row0 + node, head = mr->head0 + flat - node * a.group;
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

template <int D, int NC, bool BF16>
int launch(const CUtensorMap& tm, const Tree8Params& p, int n_ctas, cudaStream_t s) {
  static bool set[MAX_DEVICES] = {};
  const int dev = current_device_slot();
  constexpr int smem = smem8<D, NC, BF16>();
  if (!set[dev]) {
    if (cudaFuncSetAttribute(attention_8bit_kernel<D, NC, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return -1;
    set[dev] = true;
  }
  if (launch_pdl(attention_8bit_kernel<D, NC, BF16>, dim3(n_ctas), dim3(TREE_THREADS), smem, s, tm, p) != cudaSuccess) return -1;
  if (p.whole) return 0;                          // nothing is ever cut
  const int rows = std::min(NC, p.rows.max_nodes * p.group);
  return launch_pdl(merge_8bit_kernel<D, BF16>, dim3(n_ctas, (rows + MERGE_WARPS - 1) / MERGE_WARPS), dim3(MERGE_WARPS * 32), 0, s, p) == cudaSuccess ? 0 : -1;
}

// What the host decides from a call's sizes; returns the most units a prompt can have.
int64_t set_sizes(Tree8Params& p, const TreeAttention8& t, int* columns) {
  p.kv = t.kv; p.rows = t.rows;
  p.n_q_heads = t.n_q_heads;
  p.group = t.n_q_heads / t.kv.n_kv_heads;
  p.group_inverse = p.group == 1 ? 0u : static_cast<uint32_t>((UINT64_C(1) << 32) / p.group + ((UINT64_C(1) << 32) % p.group != 0));
  const int64_t rows = static_cast<int64_t>(t.rows.max_nodes) * p.group;
  *columns = rows <= 16 ? 16 : 32;
  // A unit's own cost (its Q, its rows' end), on the scale of its blocks'.  64 x 2500 slots with 1 / 2 / 3 / 4 / 6 blocks: 62.6 / 62.5 / 62.3 /
  // 62.5 / 64.5 us; trees of 26 with about 2 / 4 / 8 / 11: 148 / 137 / 136 / 135 (of an earlier form), chains of 7 on 2 x 33024 slots 41.4 /
  // 39.5 / 37.4 / 37.7.  (Tiles of a prompt made equally large: no change.)
  p.over = *columns == 16 ? 3 : 90;
  return (rows + *columns - 1) / *columns * t.kv.n_kv_heads;
}

}  // namespace

bool tree_attention_8bit_fits(const TreeAttention8& t) {
  Tree8Params p{};
  int columns;
  const int64_t units = set_sizes(p, t, &columns);
  return units_fit(t.rows.n_seqs, units, t.rows.max_len, max_blk_cost(columns), p.over);
}

int launch_tree_attention_8bit(const TreeAttention8& t, int n_sms, cudaStream_t s) {
  Tree8Params p{};
  int columns;
  const int64_t units = set_sizes(p, t, &columns);
  if (!units_fit(p.rows.n_seqs, units, p.rows.max_len, max_blk_cost(columns), p.over)) return -2;
  p.scale_log2 = t.scale * LOG2E;
  p.q = t.q; p.q_stride = t.q_stride;
  p.out = t.out; p.out_stride = t.out_stride; p.lse = t.lse;
  char* ws = static_cast<char*>(t.workspace);
  p.err_word = reinterpret_cast<int*>(ws);
  p.merges = reinterpret_cast<MergeRecord8*>(ws + WS_MERGE);
  p.partial_ml = reinterpret_cast<float*>(ws + WS_ML);
  p.partial_o = reinterpret_cast<float*>(ws + WS_O);
  const uint64_t d = t.kv.head_dim, head_bytes = 2 * PAGE_TOKENS * d;
  p.heads_a_page = static_cast<int32_t>(t.kv.page_stride / static_cast<int64_t>(head_bytes));
  // a box: [row group][K, V][8 rows][D bytes] of one page and KV head
  const uint64_t dims[5] = {d, 8, 2, 2, static_cast<uint64_t>(t.kv.n_pages - 1) * p.heads_a_page + t.kv.n_kv_heads};
  const uint64_t strides[4] = {d, PAGE_TOKENS * d, 8 * d, head_bytes};
  const uint32_t box[5] = {static_cast<uint32_t>(d), 8, 2, 2, 1};
  CUtensorMap tm;
  if (encode_u8_map(&tm, t.kv.pages, 5, dims, strides, box) != 0) return -1;
  p.whole = p.rows.max_len <= WHOLE_BLOCKS * BLK ? 1 : 0;
  const int n_ctas = std::min(n_sms, MAX_CTAS);
  p.small = small_batch(p.rows.n_seqs, units, p.rows.max_len, max_blk_cost(columns), p.over) ? 1 : 0;
  auto run = [&](auto dim, auto nc) {
    constexpr int D = decltype(dim)::value, NC = decltype(nc)::value;
    return t.kv.bf16 ? launch<D, NC, true>(tm, p, n_ctas, s) : launch<D, NC, false>(tm, p, n_ctas, s);
  };
  if (d == 128) return columns == 16 ? run(Const<128>{}, Const<16>{}) : run(Const<128>{}, Const<32>{});
  return columns == 16 ? run(Const<64>{}, Const<16>{}) : run(Const<64>{}, Const<32>{});
}

}  // namespace pc
