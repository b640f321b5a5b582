// Attention of drafted tokens over a cached context, and the running attention weights of its slots.
#include "kernels.h"
#include "ptx.cuh"

namespace pc {
namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int TREE_WARPS = 4;

template <bool BF16>
__device__ __forceinline__ float2 load2(const void* p, int64_t i) {
  if constexpr (BF16) {
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(static_cast<const __nv_bfloat16*>(p) + i));
  } else {
    return __half22float2(*reinterpret_cast<const __half2*>(static_cast<const __half*>(p) + i));
  }
}
// A finite value past the type's range (a rounded-up average of values at its limit) becomes the largest finite one; infinity stays.
template <bool BF16>
__device__ __forceinline__ void store1(void* p, int64_t i, float x) {
  if constexpr (BF16) {
    static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(x);
  } else {
    static_cast<__half*>(p)[i] = isinf(x) ? __float2half_rn(x) : to_half_sat(x);
  }
}

__device__ __forceinline__ bool node_sees(const TreeRows& r, int row, int i, int j) {
  if (r.mask == nullptr) return j <= i;
  return (r.mask[static_cast<size_t>(row) * r.mask_words + (j >> 6)] >> (j & 63)) & 1;
}

// The prompt a row belongs to, or -1 (rows behind the last prompt, and rows past a prompt's bound).
__device__ __forceinline__ int seq_of_row(const TreeRows& r, int row) {
  for (int b = 0; b < r.n_seqs; ++b) {
    const SeqPart p = seq_part(r, b);
    if (row >= p.row0 && row < p.row0 + p.n_nodes) return b;
  }
  return -1;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(TREE_WARPS * 32) tree_attention_kernel(TreeAttention a) {
  __shared__ float sm_o[TREE_WARPS][D], sm_m[TREE_WARPS], sm_l[TREE_WARPS];
  const int row = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int b = seq_of_row(a.rows, row);
  if (b < 0) return;
  const SeqPart p = seq_part(a.rows, b);
  const int i = row - p.row0;
  const int g = head / (a.n_q_heads / a.kv.n_kv_heads);
  const float scale_log2 = a.scale * LOG2E;
  float q[D / 32], o[D / 32];
#pragma unroll
  for (int e = 0; e < D / 32; e += 2) {
    const float2 f = load2<BF16>(a.q, static_cast<int64_t>(row) * a.q_stride + head * D + e * 32 + lane * 2);
    q[e] = f.x; q[e + 1] = f.y; o[e] = o[e + 1] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  bool any = false;
  for (int s = warp; s < p.ctx_len + p.n_nodes; s += TREE_WARPS) {
    if (s >= p.ctx_len && !node_sees(a.rows, row, i, s - p.ctx_len)) continue;
    any = true;
    const int64_t r = slot_row(a.kv.page_table, a.kv.pt_stride, a.kv.ctx_start, a.kv.n_slots, b, s);
    float x = 0.f, v[D / 32];
#pragma unroll
    for (int e = 0; e < D / 32; e += 2) {
      float2 kf = make_float2(0.f, 0.f), vf = kf;
      if (r >= 0) {
        kf = load2<BF16>(a.kv.k, r * a.kv.k_stride + g * D + e * 32 + lane * 2);
        vf = load2<BF16>(a.kv.v, r * a.kv.v_stride + g * D + e * 32 + lane * 2);
      }
      x = fmaf(q[e], kf.x, fmaf(q[e + 1], kf.y, x));
      v[e] = vf.x; v[e + 1] = vf.y;
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
    x *= scale_log2;
    const float m_new = fmaxf(m, x), ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = exp2f(m - ref), pr = exp2f(x - ref);
    l = l * alpha + pr;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) o[e] = o[e] * alpha + pr * v[e];
    m = m_new;
  }
  if (lane == 0) { sm_m[warp] = m; sm_l[warp] = any ? l : -1.f; }
#pragma unroll
  for (int e = 0; e < D / 32; e += 2) { sm_o[warp][e * 32 + lane * 2] = o[e]; sm_o[warp][e * 32 + lane * 2 + 1] = o[e + 1]; }
  __syncthreads();
  float M = -INFINITY, L = 0.f, acc = 0.f;
  bool seen = false;
  for (int w = 0; w < TREE_WARPS; ++w) if (sm_l[w] >= 0.f || isnan(sm_l[w])) { M = fmaxf(M, sm_m[w]); seen = true; }
  const float ref = M == -INFINITY ? 0.f : M;
  const int d = threadIdx.x;
  for (int w = 0; w < TREE_WARPS; ++w) {
    if (!(sm_l[w] >= 0.f || isnan(sm_l[w]))) continue;
    const float f = exp2f(sm_m[w] - ref);
    L += f * sm_l[w];
    if (d < D) acc += f * sm_o[w][d];
  }
  if (d < D) store1<BF16>(a.out, static_cast<int64_t>(row) * a.out_stride + head * D + d, seen ? acc / L : 0.f);
  if (d == 0 && a.lse) a.lse[static_cast<size_t>(row) * a.n_q_heads + head] = seen ? (M + log2f(L)) / LOG2E : -INFINITY;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(TREE_WARPS * 32) attention_weights_kernel(AttentionWeights a) {
  const int b = blockIdx.z, g = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const SeqPart p = seq_part(a.rows, b);
  const int group = a.n_q_heads / a.kv.n_kv_heads;
  for (int s = blockIdx.x * TREE_WARPS + warp; s < p.ctx_len + p.n_nodes; s += gridDim.x * TREE_WARPS) {
    const int64_t r = slot_row(a.kv.page_table, a.kv.pt_stride, a.kv.ctx_start, a.kv.n_slots, b, s);
    float k[D / 32];
#pragma unroll
    for (int e = 0; e < D / 32; e += 2) {
      float2 f = make_float2(0.f, 0.f);
      if (r >= 0) f = load2<BF16>(a.kv.k, r * a.kv.k_stride + g * D + e * 32 + lane * 2);
      k[e] = f.x; k[e + 1] = f.y;
    }
    float sum = 0.f;
    for (int i = 0; i < p.n_nodes; ++i) {
      const int row = p.row0 + i;
      if ((a.use && !a.use[row]) || (s >= p.ctx_len && !node_sees(a.rows, row, i, s - p.ctx_len))) continue;
      for (int h = g * group; h < (g + 1) * group; ++h) {
        const float z = a.lse[static_cast<size_t>(row) * a.n_q_heads + h];
        if (z == -INFINITY) continue;
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < D / 32; e += 2) {
          const float2 f = load2<BF16>(a.q, static_cast<int64_t>(row) * a.q_stride + h * D + e * 32 + lane * 2);
          x = fmaf(f.x, k[e], fmaf(f.y, k[e + 1], x));
        }
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
        sum += exp2f((x * a.scale - z) * LOG2E);
      }
    }
    if (lane == 0) {
      const size_t at = (static_cast<size_t>(b) * a.kv.n_kv_heads + g) * a.w_stride + s;
      a.w_out[at] = a.w_in ? fmaf(a.decay, a.w_in[at], sum) : sum;
    }
  }
}

}  // namespace

int launch_tree_attention(const TreeAttention& a, int, cudaStream_t s) {
  const dim3 grid(a.rows.n_rows, a.n_q_heads);
  if (a.kv.head_dim == 128) {
    if (a.kv.bf16) tree_attention_kernel<128, true><<<grid, TREE_WARPS * 32, 0, s>>>(a);
    else tree_attention_kernel<128, false><<<grid, TREE_WARPS * 32, 0, s>>>(a);
  } else {
    if (a.kv.bf16) tree_attention_kernel<64, true><<<grid, TREE_WARPS * 32, 0, s>>>(a);
    else tree_attention_kernel<64, false><<<grid, TREE_WARPS * 32, 0, s>>>(a);
  }
  return cudaPeekAtLastError() == cudaSuccess ? 0 : -1;
}

int launch_attention_weights(const AttentionWeights& a, int, cudaStream_t s) {
  const dim3 grid((a.rows.max_len + 63) / 64, a.kv.n_kv_heads, a.rows.n_seqs);
  if (a.kv.head_dim == 128) {
    if (a.kv.bf16) attention_weights_kernel<128, true><<<grid, TREE_WARPS * 32, 0, s>>>(a);
    else attention_weights_kernel<128, false><<<grid, TREE_WARPS * 32, 0, s>>>(a);
  } else {
    if (a.kv.bf16) attention_weights_kernel<64, true><<<grid, TREE_WARPS * 32, 0, s>>>(a);
    else attention_weights_kernel<64, false><<<grid, TREE_WARPS * 32, 0, s>>>(a);
  }
  return cudaPeekAtLastError() == cudaSuccess ? 0 : -1;
}

}  // namespace pc
