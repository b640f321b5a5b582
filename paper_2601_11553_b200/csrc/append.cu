// New rows of a batch on their way into the cache: norms of queries and keys head by head, the position rotation, K and V to their slots.
//
// x' = R(p) (x / sqrt(mean x^2 + eps) * gain).  A row of one head lies in D / 16 lanes, each with eight elements of the lower half and the
// eight that they are turned with: the norm is a sum over those lanes, the rotation needs no exchange, and all accesses are 16 bytes.
// Bound by HBM: every element is read once and written once.
//
// append_rows_kernel: a warp is one row's run of heads (queries, keys, values in turn), four or eight heads side by side; the row's
// cosines and sines stay in registers over the run.  append_pages_kernel: a warp is the keys or the values of one KV head in one 8-bit page (the
// scale is one number for all of the page's new rows), its 16 slots in registers between the maximum and the rounding.
#include <algorithm>

#include "slot_row.cuh"

namespace pc {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;

// The prompt that owns a row: the last one whose row_start is not above it (-1 or n_seqs: none).  A whole warp asks for 128 entries at
// a time, so that up to 127 prompts cost one round trip.
__device__ __forceinline__ int owner_of(const int32_t* row_start, int n_seqs, int row) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = n_seqs + 1;                     // candidates [lo, lo + n)
#pragma unroll 1
  for (;;) {
    const int step = (n + 127) >> 7;
    int below = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = (u * 32 + lane) * step;
      const bool in = at < n && ld_dep_s32(row_start + lo + at) <= row;
      below += __popc(__ballot_sync(0xffffffffu, in));
    }
    if (below == 0) return lo - 1;                // only at the top
    lo += (below - 1) * step;
    n = min(step, n - (below - 1) * step);
    if (step == 1) return lo;
  }
}
struct RowPlace { int seq, first, n, ctx; };      // a prompt, its first row, its new rows, its slots in use
__device__ __forceinline__ RowPlace place_of(const NewRows& r, int seq) {
  RowPlace p{seq, 0, 0, 0};
  if (seq < 0 || seq >= r.n_seqs) return p;
  const int first = ld_dep_s32(r.row_start + seq), last = ld_dep_s32(r.row_start + seq + 1), ctx = ld_dep_s32(r.ctx_len + seq);
  p.first = min(max(first, 0), r.n_rows);
  p.n = min(min(max(last, p.first), r.n_rows) - p.first, r.max_len);
  p.ctx = min(max(ctx, 0), r.max_len - p.n);
  return p;
}

template <bool BF16>
__device__ __forceinline__ void unpack8(const uint4& w, float* x) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    // finite values past fp16's range become the largest, infinity and NaN stay
    if (!(fabsf(a) <= 65504.f) && fabsf(a) < INFINITY) a = copysignf(65504.f, a);
    if (!(fabsf(b) <= 65504.f) && fabsf(b) < INFINITY) b = copysignf(65504.f, b);
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
}
template <bool BF16>
__device__ __forceinline__ uint4 pack8(const float* x) {
  return make_uint4(pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3]), pack2<BF16>(x[4], x[5]), pack2<BF16>(x[6], x[7]));
}

// Eight consecutive floats.
__device__ __forceinline__ void load8(const float* p, float* x) {
  *reinterpret_cast<float4*>(x) = ld_dep_f32x4(p);
  *reinterpret_cast<float4*>(x + 4) = ld_dep_f32x4(p + 4);
}
// x[0..7]: elements 8 l .. of the lower half, x[8..15]: those of the upper half; l: lane within the row's D / 16.  Only that row's lanes meet.
template <int D>
__device__ __forceinline__ void normalise(float (&x)[16], const float* gain, float eps, int l) {
  constexpr int LANES = D / 16;
  const uint32_t row = ((1u << LANES) - 1) << (threadIdx.x & 31 & ~(LANES - 1));
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
  for (int o = LANES / 2; o >= 1; o >>= 1) sum += __shfl_xor_sync(row, sum, o);
  const float f = rsqrtf(fmaf(sum, 1.0f / D, eps));
  float g[16];
  load8(gain + l * 8, g);
  load8(gain + D / 2 + l * 8, g + 8);
#pragma unroll
  for (int e = 0; e < 16; ++e) x[e] = x[e] * f * g[e];
}
struct Turn { float c[8], s[8]; };
template <int D>
__device__ __forceinline__ Turn turn_of(const float* rope, int position, int l) {
  Turn t;
  const float* p = rope + (static_cast<size_t>(position) * (D / 2) + l * 8) * 2;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float4 v = ld_dep_f32x4(p + e * 2);
    t.c[e] = v.x; t.s[e] = v.y; t.c[e + 1] = v.z; t.s[e + 1] = v.w;
  }
  return t;
}
__device__ __forceinline__ void rotate(float (&x)[16], const Turn& t) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float a = x[e], b = x[e + 8];
    x[e] = a * t.c[e] - b * t.s[e];
    x[e + 8] = fmaf(b, t.c[e], a * t.s[e]);
  }
}
__device__ __forceinline__ int position_of(const NewRows& r, int row, int slot) {
  const int p = r.position ? ld_dep_s32(r.position + row) : slot;
  return min(max(p, 0), r.n_positions - 1);
}

// ---------------------------------------------------------------------------------------------------- 16 bits
// One row's heads [h0, h1) by one warp: queries first, then (POOLS) keys and values.  At most four a group of lanes: they are asked for before the
// row's place is looked up (three round trips: its prompt, the prompt's numbers, table entries).
template <int D, bool BF16, bool POOLS>
__device__ __forceinline__ void row_heads(const KvView& kv, const NewRows& r, int row, int h0, int h1) {
  constexpr int LANES = D / 16, GROUPS = 32 / LANES, UNROLL = 4;
  const int lane = threadIdx.x & 31, l = lane % LANES, g = lane / LANES;
  const int hq = r.q ? r.n_q_heads : 0, hkv = kv.n_kv_heads;
  using E = unsigned short;
  uint4 lo[UNROLL], hi[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const int h = h0 + u * GROUPS + g;
    lo[u] = hi[u] = make_uint4(0, 0, 0, 0);
    if (h < h1) {
      const E* src = !POOLS || h < hq ? static_cast<const E*>(r.q) + row * r.q_stride + h * D
                     : h < hq + hkv   ? static_cast<const E*>(r.k) + row * r.k_stride + (h - hq) * D
                                      : static_cast<const E*>(r.v) + row * r.v_stride + (h - hq - hkv) * D;
      lo[u] = ld_dep_v4(src + l * 8);
      hi[u] = ld_dep_v4(src + D / 2 + l * 8);
    }
  }
  const RowPlace p = place_of(r, owner_of(r.row_start, r.n_seqs, row));
  if (row - p.first >= p.n) return;                // no prompt's row
  const int slot = p.ctx + row - p.first;
  Turn t;
  if (r.rope) t = turn_of<D>(r.rope, position_of(r, row, slot), l);
  int64_t at = -1;
  if constexpr (POOLS) at = slot_row(kv.page_table, kv.pt_stride, kv.ctx_start, kv.n_slots, p.seq, slot);
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    if (h0 + u * GROUPS >= h1) break;
    const int h = h0 + u * GROUPS + g;
    const bool is_q = !POOLS || h < hq, is_k = !is_q && h < hq + hkv;
    const float* gain = is_q ? r.q_gain : is_k ? r.k_gain : nullptr;
    if (is_q || is_k) {
      float x[16];
      unpack8<BF16>(lo[u], x);
      unpack8<BF16>(hi[u], x + 8);
      if (gain) normalise<D>(x, gain, r.eps, l);
      if (r.rope) rotate(x, t);
      lo[u] = pack8<BF16>(x);
      hi[u] = pack8<BF16>(x + 8);
    }
    E* dst;
    if (h >= h1) continue;
    if (is_q) dst = static_cast<E*>(r.q_out) + row * r.q_out_stride + h * D;
    else if (at < 0) continue;
    else if (is_k) dst = static_cast<E*>(const_cast<void*>(kv.k)) + at * kv.k_stride + (h - hq) * D;
    else dst = static_cast<E*>(const_cast<void*>(kv.v)) + at * kv.v_stride + (h - hq - hkv) * D;
    *reinterpret_cast<uint4*>(dst + l * 8) = lo[u];
    *reinterpret_cast<uint4*>(dst + D / 2 + l * 8) = hi[u];
  }
}

template <int D, bool BF16>
__global__ void __launch_bounds__(THREADS, 3) append_rows_kernel(const __grid_constant__ KvView kv, const __grid_constant__ NewRows r, int heads, int run) {
  pdl_launch_dependents();
  pdl_wait();
  const int runs = (heads + run - 1) / run;
  const int64_t task = static_cast<int64_t>(blockIdx.x) * WARPS + (threadIdx.x >> 5);
  const int row = static_cast<int>(task / runs), h0 = static_cast<int>(task % runs) * run;
  if (row < r.n_rows) row_heads<D, BF16, true>(kv, r, row, h0, min(h0 + run, heads));
}

// ---------------------------------------------------------------------------------------------------- 8 bits
// Exponent of the least power of two with amax <= 448 * 2^e, within -32 .. 32.
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = static_cast<int>(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);       // 448 = 1.75 * 2^8
  return min(max(e, -32), 32);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// Page j of a prompt: slots [lo, hi) are new.  The keys (even) and values (odd) of KV heads in turn, kinds [kind0, kind1) by one warp: the next kind's rows
// are asked for before this one's are worked on.
template <int D, bool BF16>
__device__ __forceinline__ void fill_page(const Kv8View& kv, const NewRows& r, const RowPlace& p, int j, int lo, int hi, int kind0, int kind1) {
  constexpr int LANES = D / 16, GROUPS = 32 / LANES, PER = 16 / GROUPS;
  const int lane = threadIdx.x & 31, l = lane % LANES, g = lane / LANES;
  using E = unsigned short;
  const int page = ld_dep_s32(kv.page_table + static_cast<size_t>(p.seq) * kv.pt_stride + j);
  const int64_t row0 = p.first + j * PAGE_TOKENS - p.ctx;          // of the page's slot 0
  uint4 raw[PER][2];
  auto fetch = [&](int kind) {
    const E* src = (kind & 1 ? static_cast<const E*>(r.v) : static_cast<const E*>(r.k)) + (kind >> 1) * D + l * 8;
    const int64_t stride = kind & 1 ? r.v_stride : r.k_stride;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int s = g + GROUPS * u;
      raw[u][0] = raw[u][1] = make_uint4(0, 0, 0, 0);
      if (s >= lo && s < hi) {
        const E* row = src + (row0 + s) * stride;
        raw[u][0] = ld_dep_v4(row);
        raw[u][1] = ld_dep_v4(row + D / 2);
      }
    }
  };
  fetch(kind0);
  int position[PER];
  if (r.rope) {
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int s = g + GROUPS * u;
      position[u] = s >= lo && s < hi ? position_of(r, static_cast<int>(row0) + s, j * PAGE_TOKENS + s) : 0;
    }
  }
  if (static_cast<uint32_t>(page) >= static_cast<uint64_t>(kv.n_pages)) return;
  uint8_t* dst0 = static_cast<uint8_t*>(const_cast<void*>(kv.pages)) + page * kv.page_stride;
  float* scales = const_cast<float*>(kv.scales) + static_cast<size_t>(page) * kv.n_kv_heads * 2;
#pragma unroll 1
  for (int kind = kind0; kind < kind1; ++kind) {
    const bool is_k = !(kind & 1);
    const float before = lo > 0 ? fminf(fmaxf(ld_dep_f32(scales + kind), 0x1p-32f), 0x1p32f) : 0.f;
    float x[PER][16];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      unpack8<BF16>(raw[u][0], x[u]);
      unpack8<BF16>(raw[u][1], x[u] + 8);
    }
    if (kind + 1 < kind1) fetch(kind + 1);
    float amax = 0.f;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int s = g + GROUPS * u;
      if (s >= lo && s < hi) {
        if (is_k && r.k_gain) normalise<D>(x[u], r.k_gain, r.eps, l);
        if (is_k && r.rope) rotate(x[u], turn_of<D>(r.rope, position[u], l));
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float a = fabsf(x[u][e]);
          if (a < INFINITY) amax = fmaxf(amax, a);
        }
      }
    }
    __syncwarp();
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    float scale = power_of_two(scale_exponent(amax));
    const bool keep = before >= scale;
    if (keep) scale = before;
    const float inv = 1.0f / scale, again = before * inv;
    uint8_t* dst = dst0 + static_cast<size_t>(kind) * (PAGE_TOKENS * D) + l * 8;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int s = g + GROUPS * u;
      uint2* to = reinterpret_cast<uint2*>(dst + s * D);
      uint2* to_hi = reinterpret_cast<uint2*>(dst + s * D + D / 2);
      if (s >= lo && s < hi) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_e4m3x2(x[u][4 * e] * inv, x[u][4 * e + 1] * inv) | pack_e4m3x2(x[u][4 * e + 2] * inv, x[u][4 * e + 3] * inv) << 16;
        *to = make_uint2(w[0], w[1]);
        *to_hi = make_uint2(w[2], w[3]);
      } else if (s < lo && !keep) {
        const uint2 a = *to, b = *to_hi;
        uint32_t w[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 y = unpack_e4m3x2(w[e] & 0xffffu), z = unpack_e4m3x2(w[e] >> 16);
          w[e] = pack_e4m3x2(y.x * again, y.y * again) | pack_e4m3x2(z.x * again, z.y * again) << 16;
        }
        *to = make_uint2(w[0], w[1]);
        *to_hi = make_uint2(w[2], w[3]);
      }
    }
    if (lane == 0) scales[kind] = scale;
  }
}

// The first `page_blocks` blocks store K and V, a warp per (rows [c * chunk, c * chunk + chunk), run of `kinds` keys and values of KV heads): it takes
// the pages whose first new row is among those rows.  The others write the queries.
template <int D, bool BF16>
__global__ void __launch_bounds__(THREADS, 2) append_pages_kernel(const __grid_constant__ Kv8View kv, const __grid_constant__ NewRows r, int chunk, int kinds, int page_blocks, int run) {
  pdl_launch_dependents();
  pdl_wait();
  const int warp = threadIdx.x >> 5;
  if (static_cast<int>(blockIdx.x) >= page_blocks) {
    const int runs = (r.n_q_heads + run - 1) / run;
    const int64_t task = static_cast<int64_t>(blockIdx.x - page_blocks) * WARPS + warp;
    const int row = static_cast<int>(task / runs), h0 = static_cast<int>(task % runs) * run;
    KvView none{};
    if (row < r.n_rows) row_heads<D, BF16, false>(none, r, row, h0, min(h0 + run, r.n_q_heads));
    return;
  }
  const int all = 2 * kv.n_kv_heads, runs = (all + kinds - 1) / kinds;
  const int64_t task = static_cast<int64_t>(blockIdx.x) * WARPS + warp;
  const int64_t c = task / runs;
  const int kind0 = static_cast<int>(task % runs) * kinds, kind1 = min(kind0 + kinds, all);
  if (c * chunk >= r.n_rows) return;
  const int begin = static_cast<int>(c) * chunk, end = min(begin + chunk, r.n_rows);
  RowPlace p = place_of(r, owner_of(r.row_start, r.n_seqs, begin));
  if (p.seq < 0) p = place_of(r, 0);               // rows ahead of the first prompt's
  int row = begin;
#pragma unroll 1
  while (p.seq < r.n_seqs) {
    row = max(row, p.first);
    if (row >= end) break;
    const int i = row - p.first, in_page = (p.ctx + i) % PAGE_TOKENS;
    if (i >= p.n) {
      p = place_of(r, p.seq + 1);
      continue;
    }
    if (i == 0 || in_page == 0)
      fill_page<D, BF16>(kv, r, p, (p.ctx + i) / PAGE_TOKENS, in_page, min(PAGE_TOKENS, in_page + p.n - i), kind0, kind1);
    row = p.first + min(i + PAGE_TOKENS - in_page, p.n);       // the next page's first new row, or the next prompt's
  }
}

// Heads a warp takes: as many as it can hold at once when that leaves enough warps for every SM, else one a group.
template <int D>
int run_of(int64_t rows, int heads, int n_sms) {
  constexpr int GROUPS = 32 / (D / 16);
  return rows * ((heads + 4 * GROUPS - 1) / (4 * GROUPS)) >= static_cast<int64_t>(n_sms) * WARPS * 2 ? 4 * GROUPS : GROUPS;
}

template <int D, bool BF16>
int append(const KvView& kv, const NewRows& r, int n_sms, cudaStream_t s) {
  const int heads = (r.q ? r.n_q_heads : 0) + 2 * kv.n_kv_heads, run = run_of<D>(r.n_rows, heads, n_sms);
  const int64_t blocks = (static_cast<int64_t>(r.n_rows) * ((heads + run - 1) / run) + WARPS - 1) / WARPS;
  if (blocks > INT32_MAX) return -2;
  return launch_pdl(append_rows_kernel<D, BF16>, dim3(static_cast<unsigned>(blocks)), dim3(THREADS), 0, s, kv, r, heads, run) == cudaSuccess ? 0 : -1;
}
template <int D, bool BF16>
int append8(const Kv8View& kv, const NewRows& r, int n_sms, cudaStream_t s) {
  // Rows of a warp: about as many as a prompt has, so that batches of single tokens spread over the warps and long prompts have a page each.
  const int per = r.n_rows / std::max(r.n_seqs, 1);
  const int chunk = per >= 16 ? 16 : per >= 8 ? 8 : per >= 4 ? 4 : per >= 2 ? 2 : 1;
  const int64_t chunks = (static_cast<int64_t>(r.n_rows) + chunk - 1) / chunk;
  // Keys and values of a warp, one behind the other: four where that leaves enough warps.
  const int all = 2 * kv.n_kv_heads, kinds = chunks * ((all + 3) / 4) >= static_cast<int64_t>(n_sms) * WARPS ? 4 : 1;
  const int64_t page_blocks = (chunks * ((all + kinds - 1) / kinds) + WARPS - 1) / WARPS;
  const int hq = r.q ? r.n_q_heads : 0, run = run_of<D>(r.n_rows, hq, n_sms);
  const int64_t q_blocks = hq ? (static_cast<int64_t>(r.n_rows) * ((hq + run - 1) / run) + WARPS - 1) / WARPS : 0;
  if (page_blocks + q_blocks > INT32_MAX) return -2;
  return launch_pdl(append_pages_kernel<D, BF16>, dim3(static_cast<unsigned>(page_blocks + q_blocks)), dim3(THREADS), 0, s, kv, r, chunk, kinds, static_cast<int>(page_blocks), run) == cudaSuccess ? 0 : -1;
}

}  // namespace

int launch_append(const KvView& kv, const NewRows& r, int n_sms, cudaStream_t s) {
  if (kv.head_dim == 128) return kv.bf16 ? append<128, true>(kv, r, n_sms, s) : append<128, false>(kv, r, n_sms, s);
  return kv.bf16 ? append<64, true>(kv, r, n_sms, s) : append<64, false>(kv, r, n_sms, s);
}
int launch_append_8bit(const Kv8View& kv, const NewRows& r, int n_sms, cudaStream_t s) {
  if (kv.head_dim == 128) return kv.bf16 ? append8<128, true>(kv, r, n_sms, s) : append8<128, false>(kv, r, n_sms, s);
  return kv.bf16 ? append8<64, true>(kv, r, n_sms, s) : append8<64, false>(kv, r, n_sms, s);
}

}  // namespace pc
