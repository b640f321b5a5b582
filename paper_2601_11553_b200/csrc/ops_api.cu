// Entry points of the operators on a decoding batch's cache: argument checks and launches.  Nothing here
// synchronises, allocates or keeps state (percache_ops_status, which exists to wait, apart).
#include <cmath>

#include "../../include/percache.h"
#include "kernels.h"

namespace pc {
namespace {

constexpr int32_t MAX_CONTEXT = 1 << 26;       // slots of a prompt: index arithmetic inside a prompt stays in 32 bits

// Makes `device` current for the call and restores the caller's device afterwards.
struct DeviceGuard {
  int before = -1;
  bool ok = false;
  explicit DeviceGuard(int device) {
    static int n = 0;                          // of the machine: asked for until there is an answer
    if ((n == 0 && cudaGetDeviceCount(&n) != cudaSuccess) || device < 0 || device >= n || cudaGetDevice(&before) != cudaSuccess) {
      cudaGetLastError();
      before = -1;
      return;
    }
    ok = before == device || cudaSetDevice(device) == cudaSuccess;
    if (before == device) before = -1;         // nothing to restore
  }
  ~DeviceGuard() {
    if (before >= 0) cudaSetDevice(before);
  }
};

int sm_count(int device) {
  static int cached[MAX_DEVICES] = {};         // a property of the device, asked for once
  if (device >= 0 && device < MAX_DEVICES && cached[device] > 0) return cached[device];
  int n = 148;
  cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device);
  if (device >= 0 && device < MAX_DEVICES) cached[device] = n;
  return n;
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bool kv_ok(const percache_kv_t* kv, int32_t max_len, bool need_v) {
  if (!kv || !kv->k || (need_v && !kv->v) || kv->n_slots <= 0 || kv->n_slots > INT32_MAX || kv->n_kv_heads <= 0 ||
      (kv->head_dim != 64 && kv->head_dim != 128) || (kv->dtype != PERCACHE_BF16 && kv->dtype != PERCACHE_F16))
    return false;
  const int64_t width = static_cast<int64_t>(kv->n_kv_heads) * kv->head_dim;
  if (!aligned(kv->k, 16) || kv->k_slot_stride < width || kv->k_slot_stride % 8 != 0 || kv->k_slot_stride > (INT64_C(1) << 35))
    return false;
  if (need_v && (!aligned(kv->v, 16) || kv->v_slot_stride < width || kv->v_slot_stride % 8 != 0 ||
                 kv->v_slot_stride > (INT64_C(1) << 35)))
    return false;
  if (kv->page_table) {
    // whole pages only: a page that hangs over the pool's end would be read in part
    if (kv->n_slots % PAGE_TOKENS != 0 || kv->page_table_stride < (max_len + PAGE_TOKENS - 1) / PAGE_TOKENS) return false;
  } else if (!kv->ctx_start) {
    return false;
  }
  return true;
}

bool rows_ok(const percache_rows_t* r) {
  return r && r->n_seqs >= 0 && r->n_seqs <= 65535 && r->n_rows >= 0 && r->max_nodes >= 1 &&
         r->max_nodes <= PERCACHE_MAX_TREE_NODES && r->max_len >= 1 && r->max_len <= MAX_CONTEXT &&
         (r->n_seqs == 0 || (r->ctx_len && r->row_start)) && (!r->mask || r->mask_words >= (r->max_nodes + 63) / 64);
}

bool heads_ok(const percache_kv_t* kv, int32_t n_q_heads) {
  return n_q_heads > 0 && n_q_heads % kv->n_kv_heads == 0 && n_q_heads / kv->n_kv_heads <= 128;
}

bool q_ok(const percache_kv_t* kv, const void* q, int64_t stride, int32_t n_q_heads, float scale) {
  return q && aligned(q, 16) && heads_ok(kv, n_q_heads) &&
         stride >= static_cast<int64_t>(n_q_heads) * kv->head_dim && stride % 8 == 0 && stride <= (INT64_C(1) << 35) &&
         scale > 0.f && std::isfinite(scale);
}

bool workspace_ok(const void* p, int64_t bytes) {
  return p && aligned(p, 256) && bytes >= static_cast<int64_t>(PERCACHE_OPS_WORKSPACE_BYTES);
}

KvView kv_view(const percache_kv_t& kv) {
  KvView v{};
  v.k = kv.k; v.v = kv.v; v.k_stride = kv.k_slot_stride; v.v_stride = kv.v_slot_stride; v.n_slots = kv.n_slots;
  v.page_table = kv.page_table; v.ctx_start = kv.page_table ? nullptr : kv.ctx_start; v.pt_stride = kv.page_table_stride;
  v.n_kv_heads = kv.n_kv_heads; v.head_dim = kv.head_dim; v.bf16 = kv.dtype == PERCACHE_BF16 ? 1 : 0;
  return v;
}

TreeRows tree_rows(const percache_rows_t& r) {
  TreeRows t{};
  t.n_seqs = r.n_seqs; t.n_rows = r.n_rows; t.max_nodes = r.max_nodes; t.max_len = r.max_len;
  t.ctx_len = r.ctx_len; t.row_start = r.row_start; t.mask = r.mask; t.mask_words = r.mask_words;
  return t;
}

int launched(int rc) {
  if (rc == 0) return PERCACHE_OK;
  if (rc == -2) return PERCACHE_E_CAPACITY;
  cudaGetLastError();
  return PERCACHE_E_CUDA;
}

}  // namespace
}  // namespace pc

using namespace pc;

extern "C" {

int percache_tree_attention(int32_t device, void* stream, const percache_kv_t* kv, const percache_rows_t* rows,
                            const void* q, int64_t q_row_stride, int32_t n_q_heads, float scale, void* out,
                            int64_t out_row_stride, float* lse, void* workspace, int64_t workspace_bytes) {
  if (!rows_ok(rows)) return PERCACHE_E_INVAL;
  if (rows->n_seqs == 0 || rows->n_rows == 0) return PERCACHE_OK;
  if (!kv_ok(kv, rows->max_len, true) || !q_ok(kv, q, q_row_stride, n_q_heads, scale) || !out ||
      !aligned(out, 16) || out_row_stride % 8 != 0 || out_row_stride < static_cast<int64_t>(n_q_heads) * kv->head_dim)
    return PERCACHE_E_INVAL;
  if (!workspace_ok(workspace, workspace_bytes)) return workspace && aligned(workspace, 256) ? PERCACHE_E_CAPACITY : PERCACHE_E_INVAL;
  TreeAttention a{};
  a.kv = kv_view(*kv);
  a.rows = tree_rows(*rows);
  a.q = q; a.q_stride = q_row_stride; a.n_q_heads = n_q_heads; a.scale = scale;
  a.out = out; a.out_stride = out_row_stride; a.lse = lse; a.workspace = workspace;
  if (!tree_attention_fits(a)) return PERCACHE_E_CAPACITY;
  const DeviceGuard dev(device);
  if (!dev.ok) return PERCACHE_E_CUDA;
  return launched(launch_tree_attention(a, sm_count(device), static_cast<cudaStream_t>(stream)));
}

int percache_attention_weights(int32_t device, void* stream, const percache_kv_t* kv, const percache_rows_t* rows,
                               const void* q, int64_t q_row_stride, int32_t n_q_heads, float scale, const float* lse,
                               const uint8_t* use, float decay, const float* weights_in, float* weights_out,
                               int64_t weights_stride, void* workspace, int64_t workspace_bytes) {
  if (!rows_ok(rows)) return PERCACHE_E_INVAL;
  if (rows->n_seqs == 0) return PERCACHE_OK;
  if (!kv_ok(kv, rows->max_len, false) || (rows->n_rows > 0 && (!q_ok(kv, q, q_row_stride, n_q_heads, scale) || !lse)) ||
      !heads_ok(kv, n_q_heads) || !weights_out || !(decay >= 0.f) || !std::isfinite(decay) || (decay != 0.f && !weights_in) ||
      weights_stride < rows->max_len)
    return PERCACHE_E_INVAL;
  if (!workspace_ok(workspace, workspace_bytes)) return workspace && aligned(workspace, 256) ? PERCACHE_E_CAPACITY : PERCACHE_E_INVAL;
  AttentionWeights a{};
  a.kv = kv_view(*kv);
  a.rows = tree_rows(*rows);
  a.q = q; a.q_stride = q_row_stride; a.n_q_heads = n_q_heads; a.scale = scale; a.lse = lse; a.use = use;
  a.decay = decay; a.w_in = decay != 0.f ? weights_in : nullptr; a.w_out = weights_out; a.w_stride = weights_stride;
  a.workspace = workspace;
  if (!attention_weights_fit(a)) return PERCACHE_E_CAPACITY;
  const DeviceGuard dev(device);
  if (!dev.ok) return PERCACHE_E_CUDA;
  return launched(launch_attention_weights(a, sm_count(device), static_cast<cudaStream_t>(stream)));
}

int percache_select_slots(int32_t device, void* stream, const float* weights, int64_t weights_stride,
                          const int32_t* length, int32_t n_seqs, int32_t n_heads, int32_t max_len, int32_t budget,
                          int32_t sink, int32_t recent, int32_t* keep, int32_t* count) {
  if (n_seqs == 0) return PERCACHE_OK;
  if (!weights || !length || !keep || !count || n_seqs < 0 || n_seqs > 65535 || n_heads <= 0 || n_heads > 65535 || max_len < 1 ||
      max_len > MAX_CONTEXT || weights_stride < max_len || budget < 1 || budget > MAX_CONTEXT || sink < 0 || recent < 0 ||
      static_cast<int64_t>(sink) + recent > budget)
    return PERCACHE_E_INVAL;
  const DeviceGuard dev(device);
  if (!dev.ok) return PERCACHE_E_CUDA;
  return launched(launch_select_slots(weights, weights_stride, length, n_seqs, n_heads, max_len, budget, sink, recent, keep,
                                      count, static_cast<cudaStream_t>(stream)));
}

int percache_compact_slots(int32_t device, void* stream, const percache_kv_t* kv, int32_t n_seqs, int32_t max_len,
                           const int32_t* dst_page_table, int32_t dst_page_table_stride, const int32_t* dst_start,
                           const int32_t* first, const int32_t* keep, int32_t keep_heads, int32_t budget,
                           const int32_t* count, const float* weights_in, float* weights_out, int64_t weights_stride) {
  if (n_seqs == 0) return PERCACHE_OK;
  if (max_len < 1 || max_len > MAX_CONTEXT || !kv_ok(kv, max_len, true) || n_seqs < 0 || n_seqs > 65535 || !keep || !count ||
      kv->n_kv_heads > 65535 || budget < 1 || (keep_heads != 1 && keep_heads != kv->n_kv_heads) || (dst_page_table && dst_start) ||
      (kv->page_table ? dst_start != nullptr : dst_page_table != nullptr) ||
      ((weights_in == nullptr) != (weights_out == nullptr)) || (weights_in && weights_stride < max_len) ||
      // destination slots are first + j <= max_len - 1, but a table only has to cover those that are written
      (dst_page_table && dst_page_table_stride < 1))
    return PERCACHE_E_INVAL;
  const DeviceGuard dev(device);
  if (!dev.ok) return PERCACHE_E_CUDA;
  CompactSlots a{};
  a.kv = kv_view(*kv);
  a.n_seqs = n_seqs; a.max_len = max_len;
  a.dst_page_table = dst_page_table; a.dst_pt_stride = dst_page_table_stride; a.dst_start = dst_start;
  a.first = first; a.keep = keep; a.keep_heads = keep_heads; a.budget = budget; a.count = count;
  a.w_in = weights_in; a.w_out = weights_out; a.w_stride = weights_stride;
  return launched(launch_compact_slots(a, sm_count(device), static_cast<cudaStream_t>(stream)));
}

int percache_ops_status(int32_t device, void* stream, const void* workspace) {
  if (!workspace) return PERCACHE_E_INVAL;
  const DeviceGuard dev(device);
  if (!dev.ok) return PERCACHE_E_CUDA;
  int word = 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (cudaMemcpyAsync(&word, workspace, sizeof(word), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess) {
    cudaGetLastError();
    return PERCACHE_E_CUDA;
  }
  return word != 0 ? PERCACHE_E_DEVICE_TIMEOUT : PERCACHE_OK;
}

}  // extern "C"
