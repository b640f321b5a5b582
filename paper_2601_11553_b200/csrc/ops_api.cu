// Entry points of the operators on a decoding batch's cache: argument checks and launches.  Nothing here
// synchronises, allocates or keeps state (percache_ops_status, which exists to wait, apart).
#include <cmath>

#include "../../include/percache.h"
#include "kernels.h"

namespace pc {
namespace {

static_assert(PERCACHE_MAX_POOLS == MAX_POOLS && PERCACHE_MAX_FORK_SEQS == MAX_FORK_SEQS, "");
constexpr int32_t MAX_HEADS = 4096;            // of the operators on pages: heads x rows and heads x pages stay in 64 bits
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

bool kv8_ok(const percache_kv8_t* kv, int32_t max_len) {
  return kv && kv->pages && kv->scales && kv->page_table && aligned(kv->pages, 16) && aligned(kv->scales, 8) && kv->n_pages > 0 &&
         kv->n_pages <= (INT64_C(1) << 26) && kv->n_kv_heads > 0 && kv->n_kv_heads <= MAX_HEADS && (kv->head_dim == 64 || kv->head_dim == 128) &&
         (kv->dtype == PERCACHE_BF16 || kv->dtype == PERCACHE_F16) && kv->page_stride <= (INT64_C(1) << 36) && kv->page_stride % (2 * PAGE_TOKENS * kv->head_dim) == 0 &&
         kv->page_stride >= static_cast<int64_t>(kv->n_kv_heads) * 2 * PAGE_TOKENS * kv->head_dim &&
         kv->n_pages < INT32_MAX / (kv->page_stride / (2 * PAGE_TOKENS * kv->head_dim)) &&
         kv->page_table_stride >= (max_len + PAGE_TOKENS - 1) / PAGE_TOKENS;
}

Kv8View kv8_view(const percache_kv8_t& kv) {
  Kv8View v{};
  v.pages = kv.pages; v.scales = kv.scales; v.page_stride = kv.page_stride; v.n_pages = kv.n_pages;
  v.page_table = kv.page_table; v.pt_stride = kv.page_table_stride;
  v.n_kv_heads = kv.n_kv_heads; v.head_dim = kv.head_dim; v.bf16 = kv.dtype == PERCACHE_BF16 ? 1 : 0;
  return v;
}

// Rows [n_rows][heads][dim] of 16-bit elements.
bool rows16_ok(const void* p, int64_t stride, int32_t heads, int32_t dim) {
  return p && aligned(p, 16) && stride % 8 == 0 && stride >= static_cast<int64_t>(heads) * dim && stride <= (INT64_C(1) << 35);
}

// Whether two sets of rows of 16-bit elements, of `a_dim` and `b_dim` elements each, share none.  Rows side by side have one stride.
bool rows_apart(const void* a, int64_t a_stride, int64_t a_dim, const void* b, int64_t b_stride, int64_t b_dim, int64_t n) {
  using Wide = __int128;                        // strides are bounded, but not by any real memory
  const Wide x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b), as = a_stride * 2, bs = b_stride * 2, aw = a_dim * 2, bw = b_dim * 2;
  if (x + (n - 1) * as + aw <= y || y + (n - 1) * bs + bw <= x) return true;
  if (as != bs) return false;
  const Wide d = ((y - x) % as + as) % as;
  return d >= aw && d + bw <= as;
}

// What does not depend on whether there are rows, then what does.
bool new_rows_ok(const percache_new_rows_t* r) {
  return r && r->n_seqs >= 0 && r->n_seqs <= 65535 && r->n_rows >= 0 && r->max_len >= 1 && r->max_len <= MAX_CONTEXT;
}
bool new_rows_ok(const percache_new_rows_t* r, int32_t n_kv_heads, int32_t dim) {
  return r->ctx_len && r->row_start && n_kv_heads <= MAX_HEADS && rows16_ok(r->k, r->k_row_stride, n_kv_heads, dim) &&
         rows16_ok(r->v, r->v_row_stride, n_kv_heads, dim) &&
         (!r->q || (r->n_q_heads > 0 && r->n_q_heads <= MAX_HEADS && rows16_ok(r->q, r->q_row_stride, r->n_q_heads, dim) &&
                    rows16_ok(r->q_out, r->q_out_row_stride, r->n_q_heads, dim) &&
                    ((r->q_out == r->q && r->q_out_row_stride == r->q_row_stride) ||
                     rows_apart(r->q_out, r->q_out_row_stride, r->n_q_heads * dim, r->q, r->q_row_stride, r->n_q_heads * dim, r->n_rows)) &&
                    rows_apart(r->q_out, r->q_out_row_stride, r->n_q_heads * dim, r->k, r->k_row_stride, n_kv_heads * dim, r->n_rows) &&
                    rows_apart(r->q_out, r->q_out_row_stride, r->n_q_heads * dim, r->v, r->v_row_stride, n_kv_heads * dim, r->n_rows))) &&
         aligned(r->q_gain, 16) && aligned(r->k_gain, 16) && aligned(r->rope, 16) && (!r->rope || r->n_positions > 0) &&
         r->eps >= 0.f && std::isfinite(r->eps);
}

NewRows new_rows(const percache_new_rows_t& r) {
  NewRows n{};
  n.n_seqs = r.n_seqs; n.n_rows = r.n_rows; n.max_len = r.max_len; n.n_q_heads = r.n_q_heads;
  n.ctx_len = r.ctx_len; n.row_start = r.row_start; n.position = r.position;
  n.q = r.q; n.q_out = r.q_out; n.k = r.k; n.v = r.v;
  n.q_stride = r.q_row_stride; n.q_out_stride = r.q_out_row_stride; n.k_stride = r.k_row_stride; n.v_stride = r.v_row_stride;
  n.q_gain = r.q ? r.q_gain : nullptr; n.k_gain = r.k_gain; n.rope = r.rope; n.n_positions = r.n_positions; n.eps = r.eps;
  return n;
}

// Arrays of a fork: blocks write one while others read, or write, another.
struct Array {
  const void* p;
  int64_t n;                                    // int32 numbers
};
bool apart(const Array& a, const Array& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.n == 0 || b.n == 0 || x + static_cast<uint64_t>(a.n) * 4 <= y || y + static_cast<uint64_t>(b.n) * 4 <= x;
}
bool fork_arrays_apart(const percache_fork_t& f, const void* workspace) {
  const Array in[] = {{f.refs, f.n_pages}, {f.free_list, f.n_pages}, {f.free_count, 1}, {f.page_table, static_cast<int64_t>(f.n_seqs) * f.page_table_stride},
                      {f.held, f.n_seqs}, {f.length, f.n_seqs}, {f.parent, f.n_children}};
  const Array out[] = {{f.refs_out, f.n_pages}, {f.free_list_out, f.n_pages}, {f.free_count_out, 1}, {f.table_out, static_cast<int64_t>(f.n_children) * f.table_out_stride},
                       {f.held_out, f.n_children}, {f.length_out, f.n_children}, {f.missing, 1}, {workspace, PERCACHE_OPS_WORKSPACE_BYTES / 4}};
  for (int o = 0; o < 8; ++o) {
    for (int i = 0; i < 7; ++i)
      if (!apart(out[o], in[i]) && !(o == i && o < 3 && out[o].p == in[i].p)) return false;      // the first three: in place
    for (int i = 0; i < o; ++i)
      if (!apart(out[o], out[i])) return false;
  }
  return true;
}

bool pool_ok(const percache_pool_t& p) {
  return p.base && aligned(p.base, 4) && p.page_bytes > 0 && p.page_bytes % 4 == 0 && p.page_bytes <= (INT64_C(1) << 32) && p.page_stride % 4 == 0 &&
         p.page_stride >= p.page_bytes && p.page_stride <= (INT64_C(1) << 36) && p.layer_stride % 4 == 0 && p.layer_stride >= 0 &&
         p.layer_stride <= (INT64_C(1) << 44) && p.n_layers >= 1 && p.n_layers <= 65535;
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

int percache_append_rows(int32_t device, void* stream, const percache_kv_t* kv, const percache_new_rows_t* rows) {
  if (!new_rows_ok(rows)) return PERCACHE_E_INVAL;
  if (rows->n_seqs == 0 || rows->n_rows == 0) return PERCACHE_OK;
  if (!kv_ok(kv, rows->max_len, true) || !new_rows_ok(rows, kv->n_kv_heads, kv->head_dim)) return PERCACHE_E_INVAL;
  const DeviceGuard dev(device);
  if (!dev.ok) return PERCACHE_E_CUDA;
  return launched(launch_append(kv_view(*kv), new_rows(*rows), sm_count(device), static_cast<cudaStream_t>(stream)));
}

int percache_append_rows_8bit(int32_t device, void* stream, const percache_kv8_t* kv, const percache_new_rows_t* rows) {
  if (!new_rows_ok(rows)) return PERCACHE_E_INVAL;
  if (rows->n_seqs == 0 || rows->n_rows == 0) return PERCACHE_OK;
  if (!kv8_ok(kv, rows->max_len) || !new_rows_ok(rows, kv->n_kv_heads, kv->head_dim)) return PERCACHE_E_INVAL;
  const DeviceGuard dev(device);
  if (!dev.ok) return PERCACHE_E_CUDA;
  return launched(launch_append_8bit(kv8_view(*kv), new_rows(*rows), sm_count(device), static_cast<cudaStream_t>(stream)));
}

int percache_tree_attention_8bit(int32_t device, void* stream, const percache_kv8_t* kv, const percache_rows_t* rows, const void* q,
                                 int64_t q_row_stride, int32_t n_q_heads, float scale, void* out, int64_t out_row_stride, float* lse,
                                 void* workspace, int64_t workspace_bytes) {
  if (!rows_ok(rows)) return PERCACHE_E_INVAL;
  if (rows->n_seqs == 0 || rows->n_rows == 0) return PERCACHE_OK;
  if (!kv8_ok(kv, rows->max_len) || n_q_heads <= 0 || n_q_heads % kv->n_kv_heads != 0 || n_q_heads / kv->n_kv_heads > 128 ||
      !rows16_ok(q, q_row_stride, n_q_heads, kv->head_dim) || !rows16_ok(out, out_row_stride, n_q_heads, kv->head_dim) || !(scale > 0.f) ||
      !std::isfinite(scale))
    return PERCACHE_E_INVAL;
  if (!workspace_ok(workspace, workspace_bytes)) return workspace && aligned(workspace, 256) ? PERCACHE_E_CAPACITY : PERCACHE_E_INVAL;
  TreeAttention8 a{};
  a.kv = kv8_view(*kv);
  a.rows = tree_rows(*rows);
  a.q = q; a.q_stride = q_row_stride; a.n_q_heads = n_q_heads; a.scale = scale;
  a.out = out; a.out_stride = out_row_stride; a.lse = lse; a.workspace = workspace;
  if (!tree_attention_8bit_fits(a)) return PERCACHE_E_CAPACITY;
  const DeviceGuard dev(device);
  if (!dev.ok) return PERCACHE_E_CUDA;
  return launched(launch_tree_attention_8bit(a, sm_count(device), static_cast<cudaStream_t>(stream)));
}

int percache_fork_pages(int32_t device, void* stream, const percache_fork_t* f, void* workspace, int64_t workspace_bytes) {
  if (!f || f->n_seqs < 0 || f->n_children < 0 || f->n_seqs > MAX_FORK_SEQS || f->n_children > MAX_FORK_SEQS) return PERCACHE_E_INVAL;
  const bool in_place = f->refs_out == f->refs;
  if ((f->n_seqs > 0 && (!f->page_table || !f->held || !f->length || f->page_table_stride < 1 || f->page_table_stride > (1 << 22))) ||
      (f->n_children > 0 && (!f->parent || !f->table_out || !f->held_out || !f->length_out || f->table_out_stride < 1 || f->table_out_stride > (1 << 22))) ||
      f->n_pages <= 0 || f->n_pages > (INT64_C(1) << 26) || !f->refs || !f->free_list || !f->free_count || !f->refs_out || !f->free_list_out ||
      !f->free_count_out || !f->missing || (f->free_list_out == f->free_list) != in_place || (f->free_count_out == f->free_count) != in_place ||
      f->room < 0 || f->room > MAX_CONTEXT || f->n_pools < 0 || f->n_pools > PERCACHE_MAX_POOLS || (f->n_pools > 0 && !f->pools))
    return PERCACHE_E_INVAL;
  Fork k{};
  for (int i = 0; i < f->n_pools; ++i) {
    const percache_pool_t& p = f->pools[i];
    if (!pool_ok(p)) return PERCACHE_E_INVAL;
    const bool wide = aligned(p.base, 16) && p.page_bytes % 16 == 0 && p.page_stride % 16 == 0 && p.layer_stride % 16 == 0;
    k.pools[i] = Pool{static_cast<char*>(p.base), p.page_bytes, p.page_stride, p.layer_stride, p.n_layers, wide ? 16 : 4};
  }
  if (!workspace_ok(workspace, workspace_bytes)) return workspace && aligned(workspace, 256) ? PERCACHE_E_CAPACITY : PERCACHE_E_INVAL;
  if (!fork_arrays_apart(*f, workspace)) return PERCACHE_E_INVAL;
  k.n_seqs = f->n_seqs; k.n_children = f->n_children; k.width = f->page_table_stride; k.width_out = f->table_out_stride;
  k.room = f->room; k.n_pools = f->n_pools; k.table = f->page_table; k.held = f->held; k.length = f->length; k.parent = f->parent;
  k.table_out = f->table_out; k.held_out = f->held_out; k.length_out = f->length_out; k.n_pages = f->n_pages;
  k.refs = f->refs; k.free_list = f->free_list; k.free_count = f->free_count;
  k.refs_out = f->refs_out; k.free_list_out = f->free_list_out; k.free_count_out = f->free_count_out; k.missing = f->missing;
  k.workspace = workspace;
  const DeviceGuard dev(device);
  if (!dev.ok) return PERCACHE_E_CUDA;
  return launched(launch_fork(k, sm_count(device), static_cast<cudaStream_t>(stream)));
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
