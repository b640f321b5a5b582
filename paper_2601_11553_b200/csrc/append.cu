// New rows of a batch on their way into the cache: norms of queries and keys head by head, the position rotation, K and V to their slots.
//
// x' = R(p) (x / sqrt(mean x^2 + eps) * gain).  A row of one head lies in D / 16 lanes, each with eight elements of the lower half and the
// eight that they are turned with: the norm is a sum over those lanes, the rotation needs no exchange, and all accesses are 16 bytes.
// Bound by HBM: every element is read once and written once.
//
// Three kernels.  append_rows_kernel (16-bit pools, few rows): a warp is one row's run of heads, queries, keys and values in turn, four or eight
// heads side by side; the row's cosines and sines stay in registers over the run.  append_pages_kernel (8-bit pages, few rows): a warp is
// keys or values of one KV head in one page (the scale is one number for all of the page's new rows), its 16 slots in registers between
// the maximum and the rounding; other blocks write the queries.  append_units_kernel (many rows of long prompts, either cache): a warp has eight
// rows, and takes their heads one after the other through a ring of asynchronous copies.
// Measured, 16 query and 8 KV heads of 128 elements: one row 2.6 us, 64 single rows into 8-bit pages 4.6 us (latency); 33024 rows into a 16-bit
// context 90 us (6.2 TB/s), 11.6 thousand rows of 8 prompts into 8-bit pages 44.6 us (3.6 TB/s: 430 instructions a warp for eight rows of a
// head, of which 40 for the page's maximum, at half the issue rate: four warps a scheduler wait for their own results, loads and shuffles).
#include <algorithm>

#include "slot_row.cuh"

namespace pc {
namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;


struct RowPlace { int seq, first, n, ctx; };      // a prompt, its first row, its new rows, its slots in use
__device__ __forceinline__ RowPlace place_from(const NewRows& r, int seq, int first, int last, int ctx) {
  RowPlace p;
  p.seq = seq;
  p.first = min(max(first, 0), r.n_rows);
  p.n = min(min(max(last, p.first), r.n_rows) - p.first, r.max_len);
  p.ctx = min(max(ctx, 0), r.max_len - p.n);
  return p;
}
__device__ __forceinline__ RowPlace place_of(const NewRows& r, int seq) {
  if (seq < 0 || seq >= r.n_seqs) return RowPlace{seq, 0, 0, 0};
  return place_from(r, seq, ld_dep_s32(r.row_start + seq), ld_dep_s32(r.row_start + seq + 1), ld_dep_s32(r.ctx_len + seq));
}
// The prompt that owns a row: the last one whose row_start is not above it (seq -1 or n_seqs: none).  A whole warp asks for 128 entries at
// a time: up to 127 prompts cost one round trip, which brings their slots in use along.
__device__ __forceinline__ RowPlace owner_of(const NewRows& r, int row) {
  const int lane = threadIdx.x & 31;
  if (r.n_seqs < 128) {
    int start[4], ctx[4], below = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = u * 32 + lane;
      start[u] = at <= r.n_seqs ? ld_dep_s32(r.row_start + at) : INT32_MAX;
      ctx[u] = at < r.n_seqs ? ld_dep_s32(r.ctx_len + at) : 0;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) below += __popc(__ballot_sync(0xffffffffu, start[u] <= row));
    auto pick = [&](const int (&x)[4], int i) {
      int y = __shfl_sync(0xffffffffu, x[0], i & 31);
#pragma unroll
      for (int u = 1; u < 4; ++u) {
        const int z = __shfl_sync(0xffffffffu, x[u], i & 31);
        if (i >> 5 == u) y = z;
      }
      return y;
    };
    const int seq = below - 1;
    if (seq < 0 || seq >= r.n_seqs) return RowPlace{seq, 0, 0, 0};
    return place_from(r, seq, pick(start, seq), pick(start, seq + 1), pick(ctx, seq));
  }
  int lo = 0, n = r.n_seqs + 1;                   // candidates [lo, lo + n)
#pragma unroll 1
  for (;;) {
    const int step = (n + 127) >> 7;
    int below = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = (u * 32 + lane) * step;
      const bool in = at < n && ld_dep_s32(r.row_start + lo + at) <= row;
      below += __popc(__ballot_sync(0xffffffffu, in));
    }
    if (below == 0) return place_of(r, lo - 1);   // only at the top
    lo += (below - 1) * step;
    n = min(step, n - (below - 1) * step);
    if (step == 1) return place_of(r, lo);
  }
}

// Two floats, for the packed instructions.
struct Two { uint64_t v; };
__device__ __forceinline__ Two two(float a, float b) { return Two{pack_f32x2(a, b)}; }
__device__ __forceinline__ float2 floats(Two x) {
  float2 r;
  unpack_f32x2(x.v, r.x, r.y);
  return r;
}
__device__ __forceinline__ Two operator*(Two a, Two b) { return Two{mul_f32x2(a.v, b.v)}; }
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) { return Two{fma_f32x2(a.v, b.v, c.v)}; }

// A lane's part of a row of one head: eight elements from 8 l on, and the eight behind the half that they are turned with; l: lane within the
// row's D / 16.
struct Part { Two lo[4], hi[4]; };
template <bool BF16>
__device__ __forceinline__ Two unpack2(uint32_t w) {
  if constexpr (BF16) return two(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
  return two(f.x, f.y);
}
template <bool BF16>
__device__ __forceinline__ Part unpack(const uint4& lo, const uint4& hi) {
  return Part{{unpack2<BF16>(lo.x), unpack2<BF16>(lo.y), unpack2<BF16>(lo.z), unpack2<BF16>(lo.w)},
              {unpack2<BF16>(hi.x), unpack2<BF16>(hi.y), unpack2<BF16>(hi.z), unpack2<BF16>(hi.w)}};
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(Two x) {
  const float2 f = floats(x);
  if constexpr (BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    const __half2 v = __floats2half2_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
}
// Halves that became infinite though the value was not: the largest finite one instead (infinity and NaN stay).
__device__ __noinline__ uint32_t largest_half2(uint32_t h, float2 f) {
  if ((h & 0x7fffu) == 0x7c00u && fabsf(f.x) < INFINITY) h -= 1u;
  if ((h & 0x7fff0000u) == 0x7c000000u && fabsf(f.y) < INFINITY) h -= 0x10000u;
  return h;
}
template <bool BF16>
__device__ __forceinline__ uint4 pack4(const Two (&x)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack2<BF16>(x[e]);
  if constexpr (!BF16) {
    const __half2 a = __hmax2(__habs2(*reinterpret_cast<__half2*>(&w[0])), __habs2(*reinterpret_cast<__half2*>(&w[1])));
    const __half2 b = __hmax2(__habs2(*reinterpret_cast<__half2*>(&w[2])), __habs2(*reinterpret_cast<__half2*>(&w[3])));
    const __half2 m = __hmax2(a, b);
    const uint32_t bits = *reinterpret_cast<const uint32_t*>(&m);
    if ((bits & 0xffffu) == 0x7c00u || (bits >> 16) == 0x7c00u) {            // (the maximum passes NaN over)
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = largest_half2(w[e], floats(x[e]));
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// 1 / sqrt(mean x^2 + eps) of the row, which LANES lanes have; the whole warp calls.
template <int LANES, int D, int N>
__device__ __forceinline__ float norm_factor(const Part (&x)[N], float eps) {
  Two a = x[0].lo[0] * x[0].lo[0], b = x[0].hi[0] * x[0].hi[0];
#pragma unroll
  for (int e = 1; e < 4 * N; ++e) { a = fma2(x[e / 4].lo[e % 4], x[e / 4].lo[e % 4], a); b = fma2(x[e / 4].hi[e % 4], x[e / 4].hi[e % 4], b); }
  const float2 fa = floats(a), fb = floats(b);
  float sum = (fa.x + fa.y) + (fb.x + fb.y);
#pragma unroll
  for (int o = LANES / 2; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  return rsqrtf(fmaf(sum, 1.0f / D, eps));
}
template <int D>
__device__ __forceinline__ float norm_factor(const Part& x, float eps) { return norm_factor<D / 16, D, 1>(reinterpret_cast<const Part(&)[1]>(x), eps); }
// x times f and the gain, of which load(q) gives the lane's q-th four.
template <typename Load>
__device__ __forceinline__ void scale_by(Part& x, float f, Load load) {
  const Two ff = two(f, f);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float4 g = load(q);                     // elements 4 q .. of the lane's sixteen
    Two* y = (q < 2 ? x.lo : x.hi) + (q & 1) * 2;
    y[0] = y[0] * ff * two(g.x, g.y);
    y[1] = y[1] * ff * two(g.z, g.w);
  }
}
template <int D>
__device__ __forceinline__ float4 gain_part(const float* gain, int l, int q) { return ld_dep_f32x4(gain + (q >> 1) * (D / 2) + l * 8 + (q & 1) * 4); }
struct Turn { Two c[4], s[4]; };
__device__ __forceinline__ Turn turn_at(const float* p) {         // eight pairs
  Turn t;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float4 v = ld_dep_f32x4(p + e * 4);
    t.c[e] = two(v.x, v.z);
    t.s[e] = two(v.y, v.w);
  }
  return t;
}
template <int D>
__device__ __forceinline__ Turn turn_of(const float* rope, int position, int l) { return turn_at(rope + (static_cast<size_t>(position) * (D / 2) + l * 8) * 2); }
__device__ __forceinline__ void rotate(Part& x, const Turn& t) {
  const Two minus = two(-1.f, -1.f);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const Two a = x.lo[e], b = x.hi[e];
    x.lo[e] = fma2(b * t.s[e], minus, a * t.c[e]);
    x.hi[e] = fma2(b, t.c[e], a * t.s[e]);
  }
}
__device__ __forceinline__ int position_of(const NewRows& r, int row, int slot) {
  const int p = r.position ? ld_dep_s32(r.position + row) : slot;
  return min(max(p, 0), r.n_positions - 1);
}

// ---------------------------------------------------------------------------------------------------- 16 bits
// One row's heads [h0, h1) by one warp: queries first, then (POOLS) keys and values.  At most four a group of lanes: they are asked for before the
// row's place is looked up (two round trips: its prompt, then table entries and the rotation).
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
  const RowPlace p = owner_of(r, row);
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
    // heads of different kinds may be side by side: all lanes work theirs out, values are then stored as they came
    const float* gain = is_q ? r.q_gain : r.k_gain;
    Part x = unpack<BF16>(lo[u], hi[u]);
    const float f = norm_factor<D>(x, r.eps);
    if (gain) scale_by(x, f, [&](int q) { return gain_part<D>(gain, l, q); });
    if (r.rope) rotate(x, t);
    if (is_q || is_k) {
      lo[u] = pack4<BF16>(x.lo);
      hi[u] = pack4<BF16>(x.hi);
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
__global__ void __launch_bounds__(THREADS, 2) append_rows_kernel(const __grid_constant__ KvView kv, const __grid_constant__ NewRows r, int heads, int run) {
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

__device__ __forceinline__ float largest(const Part& x) {                      // finite magnitude
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 a = floats(x.lo[e]), b = floats(x.hi[e]);
    m = fmax3(fmax3(m, fabsf(a.x), fabsf(a.y)), fabsf(b.x), fabsf(b.y));
  }
  if (m < INFINITY) return m;                     // (the maximum passes NaN over)
  m = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 a = floats(x.lo[e]), b = floats(x.hi[e]);
    const float v[4] = {fabsf(a.x), fabsf(a.y), fabsf(b.x), fabsf(b.y)};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (v[i] < INFINITY) m = fmaxf(m, v[i]);
  }
  return m;
}
__device__ __forceinline__ bool is_power_of_two(float x) { return (__float_as_uint(x) & 0x7fffffu) == 0u; }       // of scales: normal numbers
// The scale of a page's keys or values with new values up to amax; before: what it has, which counts if slots are in use.  It need not be a power of
// two (somebody else may have written the page): quotients and products by one that is not are rounded, and a second rounding, to 8 bits, could
// take a value for the border of two bytes that it only lies next to.  So the first one is towards zero with a last bit that says that it left something.
struct PageScale {
  float scale, inv, again;       // inv: exact, or 0: divide; again: what it was over what it is, or 1: bytes in use stay
};
__device__ __forceinline__ float over_scale(float x, float scale) {
  const float q = __fdiv_rz(x, scale);
  return fabsf(q) < INFINITY && fmaf(-q, scale, x) != 0.f ? __uint_as_float(__float_as_uint(q) | 1u) : q;
}
__device__ __forceinline__ float times_again(float x, float again) {
  const float y = __fmul_rz(x, again);
  return fmaf(x, again, -y) != 0.f ? __uint_as_float(__float_as_uint(y) | 1u) : y;
}
__device__ __forceinline__ PageScale page_scale(bool in_use, float before, float amax) {
  const float want = power_of_two(scale_exponent(amax)), have = in_use ? fminf(fmaxf(before, 0x1p-32f), 0x1p32f) : 0.f, scale = fmaxf(have, want);
  const float inv = is_power_of_two(scale) ? 1.0f / scale : 0.f;
  return PageScale{scale, inv, have >= want ? 1.f : have * inv};          // (a scale that grows is a power of two)
}
// A row's values as bytes, from element 8 l of its lower half on.
template <int D>
__device__ __forceinline__ void store_row(uint8_t* to, Part x, const PageScale& ps) {
  Two by = two(ps.inv, ps.inv);
  if (ps.inv == 0.f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 a = floats(x.lo[e]), b = floats(x.hi[e]);
      x.lo[e] = two(over_scale(a.x, ps.scale), over_scale(a.y, ps.scale));
      x.hi[e] = two(over_scale(b.x, ps.scale), over_scale(b.y, ps.scale));
    }
    by = two(1.f, 1.f);
  }
  auto bytes = [&](Two a, Two b) {
    const float2 x = floats(a * by), y = floats(b * by);
    return pack_e4m3x2(x.x, x.y) | pack_e4m3x2(y.x, y.y) << 16;
  };
  *reinterpret_cast<uint2*>(to) = make_uint2(bytes(x.lo[0], x.lo[1]), bytes(x.lo[2], x.lo[3]));
  *reinterpret_cast<uint2*>(to + D / 2) = make_uint2(bytes(x.hi[0], x.hi[1]), bytes(x.hi[2], x.hi[3]));
}
template <int D>
__device__ __forceinline__ void round_again(uint8_t* to, const PageScale& ps) {
  if (ps.again == 1.f) return;
  const uint2 a = *reinterpret_cast<uint2*>(to), b = *reinterpret_cast<uint2*>(to + D / 2);
  uint32_t w[4] = {a.x, a.y, b.x, b.y};
  const bool exact = is_power_of_two(ps.again);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 y = unpack_e4m3x2(w[e] & 0xffffu), z = unpack_e4m3x2(w[e] >> 16);
    if (exact) w[e] = pack_e4m3x2(y.x * ps.again, y.y * ps.again) | pack_e4m3x2(z.x * ps.again, z.y * ps.again) << 16;
    else w[e] = pack_e4m3x2(times_again(y.x, ps.again), times_again(y.y, ps.again)) | pack_e4m3x2(times_again(z.x, ps.again), times_again(z.y, ps.again)) << 16;
  }
  *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
  *reinterpret_cast<uint2*>(to + D / 2) = make_uint2(w[2], w[3]);
}

// The next prompt after p, which has rows or is the last look-up's: past prompts without rows in one search (one after the other 250 of them between two prompts
// took 45 us).  row: the next one to be dealt with.
__device__ __noinline__ RowPlace place_behind(const NewRows& r, int seq, int row) {
  const RowPlace next = place_of(r, seq + 1);
  if (next.n > 0 || next.seq >= r.n_seqs) return next;
  const RowPlace owner = owner_of(r, row);
  return owner.seq > next.seq ? owner : next;
}
// The units (UNIT slots of a prompt, aligned to that) whose first new row is among rows [begin, end): fn(prompt, unit of the prompt, first and behind
// the last new slot in it).
template <int UNIT, typename Fn>
__device__ __forceinline__ void each_unit(const NewRows& r, int begin, int end, Fn fn) {
  RowPlace p = owner_of(r, begin);
  if (p.seq < 0) p = place_of(r, 0);               // rows ahead of the first prompt's
  int row = begin;
#pragma unroll 1
  while (p.seq < r.n_seqs) {
    row = max(row, p.first);
    if (row >= end) break;
    const int i = row - p.first, in_unit = (p.ctx + i) % UNIT;
    if (i >= p.n) {
      p = place_behind(r, p.seq, row);
      continue;
    }
    if (i == 0 || in_unit == 0) fn(p, (p.ctx + i) / UNIT, in_unit, min(UNIT, in_unit + p.n - i));
    row = p.first + min(i + UNIT - in_unit, p.n);       // the next unit's first new row, or the next prompt's
  }
}

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
#pragma unroll 1
  for (int kind = kind0; kind < kind1; ++kind) {
    const bool is_k = !(kind & 1);
    Part x[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) x[u] = unpack<BF16>(raw[u][0], raw[u][1]);
    if (kind + 1 < kind1) fetch(kind + 1);
    float amax = 0.f;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      if (hi <= GROUPS * u || lo >= GROUPS * (u + 1)) continue;      // no lane's row is new
      if (is_k && r.k_gain) scale_by(x[u], norm_factor<D>(x[u], r.eps), [&](int q) { return gain_part<D>(r.k_gain, l, q); });
      if (is_k && r.rope) rotate(x[u], turn_of<D>(r.rope, position[u], l));
      const int s = g + GROUPS * u;
      amax = fmaxf(amax, s >= lo && s < hi ? largest(x[u]) : 0.f);
    }
    __syncwarp();
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    float* scale_at = const_cast<float*>(kv.scales) + static_cast<size_t>(page) * kv.n_kv_heads * 2 + kind;
    const PageScale ps = page_scale(lo > 0, lo > 0 ? ld_dep_f32(scale_at) : 0.f, amax);
    __syncwarp();
    if (lane == 0) *scale_at = ps.scale;
    uint8_t* dst = static_cast<uint8_t*>(const_cast<void*>(kv.pages)) + page * kv.page_stride + static_cast<size_t>(kind) * (PAGE_TOKENS * D) + l * 8;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int s = g + GROUPS * u;
      if (s >= lo && s < hi) store_row<D>(dst + s * D, x[u], ps);
      else if (s < lo) round_again<D>(dst + s * D, ps);
    }
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
  each_unit<PAGE_TOKENS>(r, begin, end, [&](const RowPlace& p, int j, int lo, int hi) { fill_page<D, BF16>(kv, r, p, j, lo, hi, kind0, kind1); });
}

// ---------------------------------------------------------------------------------------------------- long prompts
// Eight rows (those of eight slots of a prompt, aligned to eight), their queries', keys' and values' heads in turn, all by asynchronous copies into the
// warp's own shared memory: a lane copies what it reads itself, so that nothing is waited for but its own copies, and the look-ups are shared by
// eight rows and all heads.  (With a row a warp and loads into registers, a warp's time went into look-ups: 33024 rows 113 us.)
constexpr int DEPTH = 3;                          // heads on their way
// Four warps a block, four blocks an SM, so that nothing is kept in memory for want of registers (to fetch it takes as long as the copies ahead
// of it: 8 prompts into 8-bit pages with 4 / 5 / 6 blocks 44.8 / 47.2 / 57.0 us).
constexpr int UNIT_WARPS = 4, UNIT_BLOCKS = 4, PARTS = 4;
__device__ __forceinline__ void copy_async_16(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// Eight rows a warp: with sixteen, their cosines and sines leave registers for two thirds of the warps (33024 rows 107 -> 98 us).  An 8-bit page's two
// halves are two warps' that tell each other their largest values.
constexpr int UNIT = PAGE_TOKENS / 2;
struct Pair {                    // of warps
  int half, barrier;             // which half of the page is this warp's; a hardware barrier of the two
  float (*amax)[2];              // [turn & 1][half] in shared memory; turns count on from page to page
  int turn;
};
// Four lanes have a row: lane l the chunks of eight elements l, l + 4, .. of the lower half and of the upper one.
template <int D, bool BF16, bool EIGHT>
__device__ __forceinline__ void unit_kinds(const KvView& kv, const Kv8View& kv8, const NewRows& r, const RowPlace& p, int j, int lo, int hi, int first_kind, int kinds,
                                           int step, uint4* mine, const float* gains, Pair& pair) {
  constexpr int LANES = 32 / UNIT, CHUNKS = D / 16 / LANES;
  const int lane = threadIdx.x & 31, l = lane % LANES, s = lane / LANES;     // s: the lane's slot of the unit
  using E = unsigned short;
  const int hq = r.q ? r.n_q_heads : 0, hkv = EIGHT ? kv8.n_kv_heads : kv.n_kv_heads;
  // this warp's slots: from slot0 on, [lo, hi) of them new (in a page, those below lo are in use)
  const bool in_use = lo > 0;
  const int slot0 = EIGHT ? j * PAGE_TOKENS + pair.half * UNIT : j * UNIT;
  if constexpr (EIGHT) {
    lo -= pair.half * UNIT;
    hi -= pair.half * UNIT;
  }
  const bool is_new = s >= lo && s < hi;
  const int64_t row = p.first + slot0 + s - p.ctx;
  // kinds: queries' heads, keys' heads, values' heads
  auto fetch = [&](int kind, int n) {
    if (kind < kinds && is_new) {
      const bool is_q = kind < hq, is_k = !is_q && kind < hq + hkv;
      const E* src = (is_q ? static_cast<const E*>(r.q) + row * r.q_stride + kind * D
                      : is_k ? static_cast<const E*>(r.k) + row * r.k_stride + (kind - hq) * D
                             : static_cast<const E*>(r.v) + row * r.v_stride + (kind - hq - hkv) * D) + l * 8;
      uint4* to = mine + (n % DEPTH) * (CHUNKS * 2 * 32) + lane;
#pragma unroll
      for (int c = 0; c < 2 * CHUNKS; ++c) copy_async_16(to + c * 32, src + c * (LANES * 8));
    }
    copies_commit();                                               // a group per step, empty ones too
  };
#pragma unroll
  for (int n = 0; n < DEPTH - 1; ++n) fetch(first_kind + n * step, n);
  // where they go
  int64_t at = -1;                                                 // 16 bits: row of the pools
  int page = 0;
  if constexpr (EIGHT) page = ld_dep_s32(kv8.page_table + static_cast<size_t>(p.seq) * kv8.pt_stride + j);
  else if (is_new) at = slot_row(kv.page_table, kv.pt_stride, kv.ctx_start, kv.n_slots, p.seq, slot0 + s);
  Turn turn[CHUNKS] = {};                                          // the row's cosines and sines, for all kinds
  if (r.rope && is_new) {
    const float* rope = r.rope + static_cast<size_t>(position_of(r, static_cast<int>(row), slot0 + s)) * D;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) turn[c] = turn_at(rope + (l + c * LANES) * 16);
  }
  const bool there = static_cast<uint32_t>(page) < static_cast<uint64_t>(kv8.n_pages);
  int n = 0;
#pragma unroll 1
  for (int kind = first_kind; kind < kinds; kind += step, ++n) {
    fetch(kind + (DEPTH - 1) * step, n + DEPTH - 1);
    copies_wait<DEPTH - 1>();
    const bool is_q = kind < hq, is_k = !is_q && kind < hq + hkv;
    const float* gain = is_q ? (r.q_gain ? gains : nullptr) : is_k && r.k_gain ? gains + D : nullptr;
    const uint4* from = mine + (n % DEPTH) * (CHUNKS * 2 * 32) + lane;
    uint4 raw[2 * CHUNKS];                                         // lower half's chunks, upper half's chunks
#pragma unroll
    for (int c = 0; c < 2 * CHUNKS; ++c) raw[c] = from[c * 32];
    // Rows that are not new are worked on too (whatever is there), so that lanes keep together; nothing of them is stored.
    Part x[CHUNKS];
    if (EIGHT || is_q || is_k) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) x[c] = unpack<BF16>(raw[c], raw[CHUNKS + c]);
      if (gain) {
        const float f = norm_factor<LANES, D>(x, r.eps);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) scale_by(x[c], f, [&](int q) { return *reinterpret_cast<const float4*>(gain + ((c * 4 + q) * LANES + l) * 4); });
      }
      if (r.rope && (is_q || is_k)) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) rotate(x[c], turn[c]);
      }
    }
    if (!EIGHT || is_q) {
      if (is_q || is_k) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) { raw[c] = pack4<BF16>(x[c].lo); raw[CHUNKS + c] = pack4<BF16>(x[c].hi); }
      }
      bool put = is_new;
      E* dst;
      if (EIGHT || is_q) {
        dst = static_cast<E*>(r.q_out) + row * r.q_out_stride + kind * D;
      } else {
        put = at >= 0;
        dst = is_k ? static_cast<E*>(const_cast<void*>(kv.k)) + at * kv.k_stride + (kind - hq) * D
                   : static_cast<E*>(const_cast<void*>(kv.v)) + at * kv.v_stride + (kind - hq - hkv) * D;
      }
      if (put) {
#pragma unroll
        for (int c = 0; c < 2 * CHUNKS; ++c) *reinterpret_cast<uint4*>(dst + l * 8 + c * (LANES * 8)) = raw[c];
      }
    } else if constexpr (EIGHT) {
      const int page_kind = (is_k ? kind - hq : kind - hq - hkv) * 2 + (is_k ? 0 : 1);
      float* scale_at = const_cast<float*>(kv8.scales) + static_cast<size_t>(there ? page : 0) * kv8.n_kv_heads * 2 + page_kind;
      const float before = in_use && there ? ld_dep_f32(scale_at) : 0.f;
      float amax = 0.f;
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) amax = fmaxf(amax, largest(x[c]));
      if (!is_new) amax = 0.f;
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      if (lane == 0) pair.amax[pair.turn & 1][pair.half] = amax;
      asm volatile("barrier.cta.sync %0, 64;" ::"r"(pair.barrier) : "memory");
      const PageScale ps = page_scale(in_use, before, fmaxf(amax, pair.amax[pair.turn & 1][pair.half ^ 1]));
      ++pair.turn;
      if (there) {
        if (lane == 0 && pair.half == 0) *scale_at = ps.scale;
        uint8_t* dst = static_cast<uint8_t*>(const_cast<void*>(kv8.pages)) + page * kv8.page_stride + static_cast<size_t>(page_kind) * (PAGE_TOKENS * D) + (pair.half * UNIT + s) * D + l * 8;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          if (is_new) store_row<D>(dst + c * (LANES * 8), x[c], ps);
          else if (s < lo) round_again<D>(dst + c * (LANES * 8), ps);
        }
      }
    }
    __syncwarp();
  }
  copies_wait<0>();
}

template <int D, bool BF16, bool EIGHT>
__global__ void __launch_bounds__(UNIT_WARPS * 32, UNIT_BLOCKS) append_units_kernel(const __grid_constant__ KvView kv, const __grid_constant__ Kv8View kv8, const __grid_constant__ NewRows r, int kinds, int parts) {
  constexpr int LANES = 32 / UNIT, CHUNKS = D / 16 / LANES, ROWS = EIGHT ? PAGE_TOKENS : UNIT, SHARE = EIGHT ? 2 : 1;
  extern __shared__ uint4 ring[];
  __shared__ __align__(16) float gains[2 * D];
  __shared__ float amax[UNIT_WARPS / 2][2][2];
  pdl_launch_dependents();
  pdl_wait();
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const float* gain = which ? r.k_gain : r.q_gain;
    const int e = threadIdx.x;
    // a chunk's sixteen (eight of either half) in four parts, the lanes' parts one behind the other: no bank is asked twice
    const int half = e / (D / 2), in = e % (D / 2), chunk = in / 8, part = half * 2 + (in % 8) / 4;
    if (gain && e < D) gains[which * D + (((chunk / LANES) * 4 + part) * LANES + chunk % LANES) * 4 + in % 4] = ld_dep_f32(gain + e);
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5;
  const int64_t task = static_cast<int64_t>(blockIdx.x) * (UNIT_WARPS / SHARE) + warp / SHARE;
  const int64_t c = task / parts;
  if (c * ROWS >= r.n_rows) return;
  const int part = static_cast<int>(task % parts), begin = static_cast<int>(c) * ROWS, end = min(begin + ROWS, r.n_rows);
  Pair pair{warp & 1, 1 + warp / 2, amax[warp / 2], 0};
  each_unit<ROWS>(r, begin, end, [&](const RowPlace& p, int j, int lo, int hi) {
    unit_kinds<D, BF16, EIGHT>(kv, kv8, r, p, j, lo, hi, part, kinds, parts, ring + warp * (DEPTH * CHUNKS * 2 * 32), gains, pair);
  });
}

// Heads a warp takes: as many as it can hold at once when that leaves enough warps for every SM, else one a group.
template <int D>
int run_of(int64_t rows, int heads, int n_sms) {
  constexpr int GROUPS = 32 / (D / 16);
  return rows * ((heads + 4 * GROUPS - 1) / (4 * GROUPS)) >= static_cast<int64_t>(n_sms) * WARPS * 2 ? 4 * GROUPS : GROUPS;
}

// Whether units of rows are the faster form: from enough heads of rows on that a warp's eight or so in turn do not leave the GPU half empty, and if
// units are full on average.  With 16 + 2 x 8 heads of 128, rows or pages against units: into 8-bit pages 2048 rows of one prompt 13.0 / 14.2 us, 4096
// 18.7 / 15.3, 6000 21.9 / 22.7, 8192 31.8 / 27.6, 64 prompts of 100 rows 24.5 / 31.3, of 128 30.9 / 26.6, 500 of 32 58.2 / 49.3, of 64 111.8 / 93.9; into
// 16-bit pages 1024 9.2 / 8.8, 2048 8.9 / 11.0, 4096 15.4 / 11.9, 6000 25.8 / 19.3, 8192 36.0 / 26.0, 64 prompts of 64 15.3 / 12.0, 500 of 8 16.6 / 12.3, of 16
// 34.6 / 25.9; 8192 rows of heads of 64 into 8-bit pages 15.3 / 17.9, 16-bit 14.9 / 13.7.
bool units_pay(const NewRows& r, int kinds, bool eight) {
  return static_cast<int64_t>(r.n_rows) * kinds >= (eight ? 1 << 18 : 1 << 17) && r.n_rows / r.n_seqs >= (eight ? 64 : 16);
}
template <int D, bool BF16, bool EIGHT>
int append_units(const KvView& kv, const Kv8View& kv8, const NewRows& r, cudaStream_t s) {
  static bool set[MAX_DEVICES] = {};
  const int dev = current_device_slot();
  constexpr int ROWS = EIGHT ? PAGE_TOKENS : UNIT, AT_ONCE = EIGHT ? UNIT_WARPS / 2 : UNIT_WARPS, smem = UNIT_WARPS * DEPTH * UNIT * D * 2;
  if (!set[dev]) {
    if (cudaFuncSetAttribute(append_units_kernel<D, BF16, EIGHT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return -1;
    set[dev] = true;
  }
  const int kinds = (r.q ? r.n_q_heads : 0) + 2 * (EIGHT ? kv8.n_kv_heads : kv.n_kv_heads), parts = std::min(kinds, PARTS);
  const int64_t blocks = ((static_cast<int64_t>(r.n_rows) + ROWS - 1) / ROWS * parts + AT_ONCE - 1) / AT_ONCE;
  if (blocks > INT32_MAX) return -2;
  return launch_pdl(append_units_kernel<D, BF16, EIGHT>, dim3(static_cast<unsigned>(blocks)), dim3(UNIT_WARPS * 32), smem, s, kv, kv8, r, kinds, parts) == cudaSuccess ? 0 : -1;
}

template <int D, bool BF16>
int append(const KvView& kv, const NewRows& r, int n_sms, cudaStream_t s) {
  const int heads = (r.q ? r.n_q_heads : 0) + 2 * kv.n_kv_heads;
  if (units_pay(r, heads, false)) return append_units<D, BF16, false>(kv, Kv8View{}, r, s);
  const int run = run_of<D>(r.n_rows, heads, n_sms);
  const int64_t blocks = (static_cast<int64_t>(r.n_rows) * ((heads + run - 1) / run) + WARPS - 1) / WARPS;
  if (blocks > INT32_MAX) return -2;
  return launch_pdl(append_rows_kernel<D, BF16>, dim3(static_cast<unsigned>(blocks)), dim3(THREADS), 0, s, kv, r, heads, run) == cudaSuccess ? 0 : -1;
}
template <int D, bool BF16>
int append8(const Kv8View& kv, const NewRows& r, int n_sms, cudaStream_t s) {
  if (units_pay(r, (r.q ? r.n_q_heads : 0) + 2 * kv.n_kv_heads, true)) return append_units<D, BF16, true>(KvView{}, kv, r, s);
  // Rows of a warp: about as many as a prompt has, so that batches of single tokens spread over the warps and long prompts have a page each (with
  // eight rows half of the warps own none: 500 prompts of 32 rows 68.5 -> 58.2 us, 20000 rows of one KV head 23.7 -> 20.8).
  const int per = r.n_rows / r.n_seqs;
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
