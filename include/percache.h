/*
 * percache.h — C ABI of the reuse-prefill library (one model, one GPU per handle).
 *
 * The operation is the one PerCache's QKV-cache tier performs at query time
 * (paper Section 3.2.2 "QKV Cache Reuse", Appendix B.1 "Inference implementation
 * details"): a prompt is an ordered list of knowledge chunks followed by the
 * user's query tokens; tensors of chunks already in the cache are loaded and
 * concatenated in order, the rows they cover are dropped from every block's
 * attention input, projection and position encoding run on the remaining rows
 * only (each at its true position in the full sequence), the computed tensors are
 * concatenated with the loaded ones and the rest of the block proceeds normally.
 * Tensors computed for chunks that were not cached are sliced per chunk and kept
 * (Section 3.2.1, cache slicer).
 *
 * Deliberate differences from the paper's prototype, all documented in the design
 * notes: only K and V are cached (bf16, 16-token pages, K stored before rotation
 * and rotated to its slot's position when gathered); a chunk may hit at any place
 * of the list, not only as part of a prefix; only the new rows (missed chunks and
 * query tokens) continue through the blocks and are returned.
 *
 * General rules
 *  - Every function returns 0 (PERCACHE_OK) or a negative PERCACHE_E_* code; nothing
 *    throws or aborts across this boundary.  percache_strerror() names a code.
 *  - A handle is not thread-safe.  All device work of a handle runs on the stream
 *    given at creation; calls return after that work has finished.
 *  - A call that is refused before its device work starts (every argument, capacity and space check) leaves the
 *    store exactly as it was, also when eviction is on: victims are chosen first but dropped only when the kernels
 *    are about to write.  A call whose device work fails (PERCACHE_E_CUDA, PERCACHE_E_DEVICE_TIMEOUT) stores
 *    nothing and leaves the store consistent, but chunks it evicted to make room stay evicted, and the assembled
 *    context of the previous call is forgotten (percache_decode then returns PERCACHE_E_INVAL).
 *  - Number formats: the store is bf16, the residual stream fp32, every operand of a projection or of the attention
 *    is fp16 with fp32 accumulation.  fp16 carries magnitudes up to 65504; every conversion to fp16 inside the
 *    library saturates (a larger value becomes +-65504, never infinity), so out-of-range weights, cached values or
 *    activations (a SwiGLU product, a rotated key) are clipped and the call stays finite.  Results are only
 *    meaningful while normed activations, projections and SwiGLU products stay within that range; bf16 values below
 *    2^-24 in magnitude flush to zero as operands.
 *  - The library never frees or keeps caller memory: every caller buffer may be
 *    released as soon as the call returns.
 *  - There is no CPU fallback: without a CUDA device every call that needs one fails
 *    with PERCACHE_E_CUDA.
 */
#ifndef PERCACHE_H_
#define PERCACHE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define PERCACHE_API __attribute__((visibility("default")))
#else
#define PERCACHE_API
#endif

#define PERCACHE_OK                 0
#define PERCACHE_E_INVAL           -1   /* bad argument (NULL, negative size, unsupported shape)        */
#define PERCACHE_E_NOMEM           -2   /* host or device allocation failed                            */
#define PERCACHE_E_NOSPACE         -3   /* the paged store has too few free pages                      */
#define PERCACHE_E_EXISTS          -4   /* chunk id already stored                                     */
#define PERCACHE_E_LEN_MISMATCH    -5   /* chunk id stored with a different token count                */
#define PERCACHE_E_MISS_NO_INPUT   -6   /* chunk is not stored and no hidden states were given for it  */
#define PERCACHE_E_CAPACITY        -7   /* prompt / batch exceeds a limit fixed at creation            */
#define PERCACHE_E_DEVICE_TIMEOUT  -8   /* a bounded wait inside a kernel ran out; results are invalid */
#define PERCACHE_E_CUDA            -9   /* a CUDA runtime / driver call failed                         */
#define PERCACHE_E_NOTFOUND        -10  /* chunk id not stored (has / drop)                            */

#define PERCACHE_PAGE_TOKENS 16

/* percache_config_t.flags */
#define PERCACHE_FLAG_REFERENCE_KERNELS  1u  /* debugging aid: run every GEMM and the attention with the plain
                                                one-thread-per-output CUDA kernels instead of the tcgen05 ones */
#define PERCACHE_FLAG_PHASE_TIMING       2u  /* record CUDA events around every kernel class (see stats)       */
#define PERCACHE_FLAG_REFERENCE_ATTENTION 4u /* debugging aid: plain attention kernel, tcgen05 GEMMs            */
#define PERCACHE_FLAG_SINGLE_CTA_GEMM   16u  /* debugging aid: never run a GEMM on CTA pairs (256 x 256 tiles)     */
#define PERCACHE_FLAG_NO_SMALL_ROW_KERNELS 32u /* debugging aid: calls with at most 8 rows (decode) use the tcgen05
                                                GEMMs like any other instead of the weight-streaming kernels     */
#define PERCACHE_FLAG_EVICT_LFU          8u  /* when the store is full, evict least-frequently-used chunks instead
                                                of failing with PERCACHE_E_NOSPACE (see percache_set_store_limit)  */

#define PERCACHE_FLAG_GATHER_FREE       128u  /* take the gather-free form of percache_prefill whenever it is possible
                                                (see percache_prefill), not only when the cached part dominates   */
#define PERCACHE_FLAG_ALWAYS_GATHER     256u  /* never take it: always assemble the contiguous context              */
#define PERCACHE_FLAG_TRACK_WEIGHTS     512u  /* decode steps add their attention weights to running sums per layer, KV head
                                                and context slot (see percache_evict_context)                     */
#define PERCACHE_FLAG_PAPER_MODE         64u  /* creation only: the handle works exactly as the paper states the scheme
                                                (see "Paper-faithful mode" below)                                 */

typedef struct percache percache_t;   /* opaque */

typedef struct {
  int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn;
  float   rope_theta, rms_eps;
  int32_t page_tokens;              /* must be PERCACHE_PAGE_TOKENS                                         */
  int64_t pool_pages;               /* capacity of the paged store, in pages (each page: 16 tokens, all
                                       layers, K and V)                                                    */
  int32_t max_prompt_tokens;        /* longest prompt (chunks + query); also the largest RoPE position + 1  */
  int32_t max_batch_prompts;        /* most prompts in one percache_prefill call                            */
  int64_t max_batch_ctx_tokens;     /* most context tokens (sum of prompt lengths) in one call              */
  int64_t max_batch_new_rows;       /* most new rows (missed-chunk tokens + query tokens) in one call       */
  int32_t device;                   /* CUDA device ordinal                                                  */
  void*   stream;                   /* cudaStream_t of the caller, or NULL for the default stream           */
  uint32_t flags;                   /* PERCACHE_FLAG_*                                                      */
} percache_config_t;

/* One layer's parameters: bf16, row-major [out_features][in_features] (norm gains: [d_model]).
 * Host or device pointers (see weights_on_device); copied during percache_create. */
typedef struct {
  const void *attn_norm, *wq, *wk, *wv, *wo, *ffn_norm, *w_gate, *w_up, *w_down;
} percache_layer_weights_t;

/* Create a handle: allocates the paged store, work buffers and a private copy of the weights on
 * cfg->device.  Supported shapes: head_dim 128; d_model, d_ffn multiples of 64; n_q_heads an even multiple
 * of n_kv_heads (the attention kernel pairs the query heads of a KV head).  Device allocation failure -> PERCACHE_E_NOMEM; the handle is not created. */
PERCACHE_API int percache_create(const percache_config_t* cfg, const percache_layer_weights_t* layers /*[n_layers]*/,
                    int32_t weights_on_device, percache_t** out);

/* Free everything the handle owns.  NULL is accepted. */
PERCACHE_API int percache_destroy(percache_t* h);

/* Insert a chunk's unrotated K and V for all layers (what a prefill of that chunk collected; paper
 * Section 3.2.1).  k, v: bf16 [n_layers][n_tokens][n_kv_heads][head_dim], host or device memory as
 * ptr_is_device says.  Copied into ceil(n_tokens/16) pages before return.  An id that is already stored
 * is not overwritten: PERCACHE_E_EXISTS. */
PERCACHE_API int percache_put_chunk_kv(percache_t* h, uint64_t chunk_id, int32_t n_tokens,
                          const void* k, const void* v, int32_t ptr_is_device);

/* How the chunks of a prompt are matched against the store.
 *  PERCACHE_MATCH_CHUNK_ID     a chunk hits when its id is stored, at whatever place of the list it appears (the
 *                              K/V of layers > 0 were then computed in some other context).
 *  PERCACHE_MATCH_PREFIX_PATH  the paper's rule (Section 3.2.2): entries are nodes of a tree whose paths are chunk
 *                              lists; the first chunk is looked up, then the second as its child, and so on until
 *                              the first mismatch; every later chunk is computed.  The store key of a node is
 *                              percache_path_key() of the ids from the first chunk to that node, and the chunks a
 *                              call computes are stored under their path keys.  Reuse then equals full prefill.
 * Path keys and plain chunk ids share the handle's one 64-bit key space (two keys collide with probability 2^-64);
 * percache_has_chunk / _drop_chunk / _chunk_info / _get_chunk_kv take whichever key an entry was stored under. */
#define PERCACHE_MATCH_CHUNK_ID    0
#define PERCACHE_MATCH_PREFIX_PATH 1

/* Key of the tree node reached by the path chunk_ids[0..n-1] (n = 0: the root's seed). */
PERCACHE_API uint64_t percache_path_key(const uint64_t* chunk_ids, int32_t n);

/* A prompt: ordered chunk list plus query tokens (paper Section 3, system overview). */
typedef struct {
  int32_t n_chunks;
  const uint64_t* chunk_ids;            /* host [n_chunks]                                                 */
  const int32_t*  chunk_len;            /* host [n_chunks], tokens per chunk (> 0)                          */
  const void* const* chunk_hidden;      /* host [n_chunks] of pointers to bf16 [len][d_model] layer-0 input;
                                           an entry (or the whole array) may be NULL for a chunk expected to
                                           hit; NULL for a chunk that misses -> PERCACHE_E_MISS_NO_INPUT    */
  int32_t n_query;                      /* >= 0                                                             */
  const void* query_hidden;             /* bf16 [n_query][d_model]                                          */
  int32_t hidden_on_device;             /* 1: chunk_hidden[i] and query_hidden point to device memory       */
  int32_t match_mode;                   /* PERCACHE_MATCH_*                                                 */
  int32_t reuse_tail_drop;              /* PERCACHE_MATCH_PREFIX_PATH only, else must be 0 (paper Appendix B,
                                           tokenisation paragraph): the tensors of the last reuse_tail_drop tokens
                                           of the final matched chunk are not reused; those tokens are computed
                                           from chunk_hidden (which must then be given for that chunk) and are not
                                           stored again.  0 <= drop <= that chunk's length                      */
} percache_prompt_t;

typedef struct {
  float*   out_hidden;         /* caller-allocated fp32 [out_capacity_rows][d_model]: final residual stream of
                                  the new rows, in prompt order (no final norm)                             */
  int64_t  out_capacity_rows;  /* fewer than n_new -> PERCACHE_E_CAPACITY                                   */
  int32_t  out_on_device;      /* 1: out_hidden is device memory                                            */
  uint8_t* hit_mask;           /* caller-allocated host [n_chunks] or NULL; 1 = served from the store       */
  int32_t  n_new, n_total;     /* written by the call: new rows and total context tokens of this prompt     */
} percache_result_t;

/* Reuse-prefill of a batch of independent prompts (paper Section 3.2.2, Appendix B.1).
 * Hits are decided against the store as it is when the call starts: a chunk hits when its id is stored
 * with the same length (different length -> PERCACHE_E_LEN_MISMATCH).  On success every missed chunk is
 * stored (its K/V as computed inside its prompt; if two prompts of the batch miss the same id, the
 * first prompt's is kept) and query tokens are not.  Too few free pages -> PERCACHE_E_NOSPACE.
 * Synchronous: returns after the stream has drained.
 * Two forms compute the same result.  The default one copies every cached token's K and V into a contiguous context
 * (K rotated to its position there) and lets the attention read that.  The gather-free one leaves them in their
 * pages: the attention walks the prompt's page table, rotates K as it loads it and reads V where it is, so the fetch
 * and its traffic disappear; there P and V enter the second attention product as bf16 (the store's format) instead
 * of fp16.  It is taken when the batch has at least 8 cached tokens per new row and no prompt more than 256 new rows
 * (or PERCACHE_FLAG_GATHER_FREE is set), every chunk length and reuse_tail_drop is a multiple of 16 and
 * PERCACHE_FLAG_ALWAYS_GATHER is not set; rows that are not stored (query tokens) then occupy pages of the store for
 * the duration of the call (they count against the store limit).  After a gather-free call there is no assembled
 * context and percache_debug_read_ctx returns PERCACHE_E_INVAL.  If a decode reserve is set, those pages (and page
 * slots for the tokens to be decoded) stay occupied after the call and the first percache_decode step runs the
 * skipped fetch over all slots, which builds the context and gives the pages back; with PERCACHE_FLAG_GATHER_FREE
 * set at that time the decode steps instead read the pages themselves (K rotated on load; each step's attention is
 * about 40 % slower, no context is ever built, the pages stay occupied).  Any later percache_prefill call, successful
 * or not, gives the pages back and ends that batch's decode steps.  Without a decode reserve percache_decode after a
 * gather-free call returns PERCACHE_E_INVAL. */
PERCACHE_API int percache_prefill(percache_t* h, const percache_prompt_t* prompts, int32_t n_prompts,
                     percache_result_t* results /*[n_prompts]*/);

/* Paper-faithful mode (a handle created with PERCACHE_FLAG_PAPER_MODE).  percache_prefill then computes what the
 * paper describes, without the three departures listed at the top of this file:
 *  - matching is the prefix-tree walk (every prompt must use PERCACHE_MATCH_PREFIX_PATH, Section 3.2.2);
 *  - a node holds the chunk's Q, K and V of every block (Sections 3.2.1 and 5.3: all three projections are skipped
 *    for cached rows), bf16, Q and K after position encoding at the positions the node has on its path;
 *  - all L_total rows of the prompt run through every block; the L_pre rows of the matched chain skip only the
 *    projections and the position encoding, for the others the position counter starts at L_pre (Appendix B.1);
 *    reuse_tail_drop shortens L_pre by the tail of the chain's last node (Appendix B, tokenisation paragraph);
 *  - out_hidden receives ALL n_total rows (out_capacity_rows >= n_total); n_new still counts the computed rows.
 * Q, K (both rotated) and V of every row are rounded to bf16 before the attention uses them, loaded or computed
 * alike, because that is what the store holds.  The attention reads Q, K and V of all rows straight from the pages
 * through a per-prompt page table (nothing is gathered or rotated at query time).  Restrictions of this mode: hidden
 * states must be given for every chunk (the whole prompt is embedded); chunk lengths and reuse_tail_drop must be
 * multiples of 16 (pages are copied whole; the query may have any length); max_batch_new_rows bounds the rows of a
 * batch, i.e. the sum of n_total; percache_put_chunk_kv, _put_chunk_synthetic and percache_decode return
 * PERCACHE_E_INVAL; the debugging flags that select the plain kernels are refused.  percache_get_chunk_kv returns the
 * node's K (rotated) and V, percache_get_chunk_q its Q: bf16 [n_layers][n_tokens][n_q_heads][head_dim], host. */
PERCACHE_API int percache_get_chunk_q(percache_t* h, uint64_t chunk_id, void* q_host);

/* Decode step after a prefill (paper Section 2.1: inference is a prefill over the prompt followed by a decode
 * stage that produces one token at a time, attending to the keys and values of everything before it).
 * One token per prompt of the LAST percache_prefill call: hidden is bf16 [n_prompts][d_model] (row b continues
 * prompt b; host or device memory per hidden_on_device), n_prompts must equal that call's.  Row b is at position
 * n_total_b + (tokens decoded so far); it runs through every block like a new row of the prefill and attends to
 * the prompt's assembled context plus itself; its rotated K and its V are appended to that context (they are
 * not chunk content: nothing is stored).  out_hidden: caller-allocated fp32 [n_prompts][d_model], final residual
 * stream (no final norm).  The context keeps percache_set_decode_reserve() free slots behind every prompt; a
 * prompt that has used them all, or would pass max_prompt_tokens, -> PERCACHE_E_CAPACITY and nothing changes.
 * Any later percache_prefill starts a new batch and discards the decoded tokens.  Synchronous. */
PERCACHE_API int percache_decode(percache_t* h, int32_t n_prompts, const void* hidden, int32_t hidden_on_device,
                    float* out_hidden, int32_t out_on_device);

/* A decode step over drafted tokens: prompt b gets n_nodes[b] of them at once (0 .. PERCACHE_MAX_TREE_NODES, not all
 * zero) as a tree.  parents [sum n_nodes], prompt after prompt: parents[i] < i is the index, inside its prompt, of the
 * token that node i follows, -1 for one that follows the prompt's last token (so a chain is -1, 0, 1, ...).  hidden:
 * bf16 [sum n_nodes][d_model]; out_hidden: fp32 [sum n_nodes][d_model].  Node i is at the position of its depth behind
 * the prompt's tokens so far and attends to the prompt's context, its ancestors and itself, exactly as if the path to it
 * had been decoded token by token.  The nodes' K and V lie behind the context, one slot each (the decode reserve has to
 * hold them: PERCACHE_E_CAPACITY), until percache_accept keeps a path of them; any other decode or prefill call drops
 * them.  Synchronous; same errors as percache_decode; at most 65535 prompts (PERCACHE_E_CAPACITY), as for a
 * percache_decode with PERCACHE_FLAG_TRACK_WEIGHTS.  After a gather-free prefill the first such call assembles the
 * context, whatever the flags. */
PERCACHE_API int percache_decode_tree(percache_t* h, int32_t n_prompts, const int32_t* n_nodes, const int32_t* parents,
                                      const void* hidden, int32_t hidden_on_device, float* out_hidden,
                                      int32_t out_on_device);

/* Keep a path of the last percache_decode_tree call's nodes: for prompt b n_accept[b] of them (0 .. n_nodes[b]),
 * nodes [sum n_accept] prompt after prompt, each prompt's first with parent -1 and every other the child of the one
 * before (PERCACHE_E_INVAL otherwise, and nothing changes).  Their K and V become the prompt's next context slots, the
 * other nodes are dropped.  With PERCACHE_FLAG_TRACK_WEIGHTS set in that call, every prompt's running weights decay once and
 * the accepted nodes' attention weights are added.  Synchronous. */
PERCACHE_API int percache_accept(percache_t* h, int32_t n_prompts, const int32_t* n_accept, const int32_t* nodes);

/* Cut every prompt's context to at most `budget` slots per layer and KV head: the first `sink`, the last `recent`
 * (sink + recent <= budget) and the ones with the most running attention weight, equal weights going to the lower slot.
 * The weights are those that percache_decode and percache_accept have added while PERCACHE_FLAG_TRACK_WEIGHTS was set,
 * since the prefill (every step first multiplies the sums by the decay of percache_set_weight_decay, 1 at creation);
 * without any such step, or while a tree's nodes wait for percache_accept, PERCACHE_E_INVAL.  A tracked step or a
 * percache_accept that returns PERCACHE_E_CUDA or PERCACHE_E_DEVICE_TIMEOUT ends the sums (some layers may have been added to
 * and others not; the context stays as it was, nodes to be accepted are dropped): the next tracked step starts them
 * from zero.  An eviction that returns PERCACHE_E_CUDA ends the batch.  Positions are not touched: later tokens continue at
 * theirs, and the freed slots are free for them (they count towards the decode reserve).  percache_debug_read_ctx and
 * read_weights then see the slots that are left.  Synchronous. */
PERCACHE_API int percache_evict_context(percache_t* h, int32_t budget, int32_t sink, int32_t recent);
PERCACHE_API int percache_set_weight_decay(percache_t* h, float decay);

/* Running weights of one prompt and layer: fp32 [n_kv_heads][slots of the prompt's context], copied to a host buffer of
 * capacity_floats floats (PERCACHE_E_CAPACITY if short).  Returns the number of slots, or a negative code. */
PERCACHE_API int64_t percache_debug_read_weights(percache_t* h, int32_t prompt, int32_t layer, float* out,
                                                 int64_t capacity_floats);

/* Context slots kept free behind every prompt of later percache_prefill calls, so that percache_decode can
 * append tokens (default 0: no decode).  A batch needs sum(n_total) + n_prompts * tokens_per_prompt <=
 * max_batch_ctx_tokens, else percache_prefill returns PERCACHE_E_CAPACITY. */
PERCACHE_API int percache_set_decode_reserve(percache_t* h, int32_t tokens_per_prompt);

/* *n_tokens = stored length, or PERCACHE_E_NOTFOUND. n_tokens may be NULL. */
PERCACHE_API int percache_has_chunk(percache_t* h, uint64_t chunk_id, int32_t* n_tokens);

/* Remove a chunk and free its pages (used to restore the cache state between timed runs). */
PERCACHE_API int percache_drop_chunk(percache_t* h, uint64_t chunk_id);

/* Capacity management (paper Section 3.2.1: a retrieval counter per cached entry, least-frequently-used
 * eviction under a configurable storage limit).  Every stored chunk counts the prompts that used it: 1 when a
 * prompt first stores it (or percache_put_chunk_* inserts it), +1 for every later prompt occurrence that hits it.
 * With PERCACHE_FLAG_EVICT_LFU, a call that needs more pages than the limit leaves free evicts chunks in order
 * of (count ascending, insertion order ascending), never one the calling batch itself hits, until the new pages
 * fit; if they cannot fit the call fails with PERCACHE_E_NOSPACE and nothing is evicted.  Eviction is applied
 * after every host-side check of the call has passed.
 * percache_set_store_limit: limit in pages, 1..pool_pages (default pool_pages).  Lowering it below the current
 * use evicts at once (LFU order) when the flag is set, else fails with PERCACHE_E_NOSPACE. */
PERCACHE_API int percache_set_store_limit(percache_t* h, int64_t pages);

/* *n_tokens = stored length, *retrievals = the chunk's counter; either pointer may be NULL. */
PERCACHE_API int percache_chunk_info(percache_t* h, uint64_t chunk_id, int32_t* n_tokens, int64_t* retrievals);

/* Read a stored chunk back: k, v host buffers bf16 [n_layers][n_tokens][n_kv_heads][head_dim]. */
PERCACHE_API int percache_get_chunk_kv(percache_t* h, uint64_t chunk_id, void* k_host, void* v_host);

/* Fill a new chunk with the synthetic integer pool values of the batched-serving workload:
 * element e of (chunk, which in {K=0,V=1}, layer) takes the 64-bit counter
 *   ((((seed << 20) + chunk_id) * 2 + which) * 64 + layer) << 24) + e
 * through the SplitMix64 output function, and the value (b0 + b1 + b2 + b3 - 126) / 64 with b_i the four
 * lowest 6-bit fields of the result (exact in bf16).  Same errors as percache_put_chunk_kv. */
PERCACHE_API int percache_put_chunk_synthetic(percache_t* h, uint64_t chunk_id, int32_t n_tokens, uint64_t seed);

/* Kernel classes for phase timing. */
enum {
  PERCACHE_PH_GATHER = 0,   /* gather + re-RoPE of hit tokens, all layers                */
  PERCACHE_PH_NORM,         /* both RMSNorms                                              */
  PERCACHE_PH_QKV,          /* QKV projection + RoPE + scatter                           */
  PERCACHE_PH_ATTN,         /* causal GQA attention of the new rows                      */
  PERCACHE_PH_OPROJ,        /* output projection + residual                              */
  PERCACHE_PH_GATEUP,       /* gate/up projection + SwiGLU                               */
  PERCACHE_PH_DOWN,         /* down projection + residual                                */
  PERCACHE_PH_IO,           /* input staging and output copies                           */
  PERCACHE_PH_COUNT
};

typedef struct {
  /* last percache_prefill call */
  int32_t n_prompts, chunks_hit, chunks_missed;
  int64_t ctx_tokens, hit_tokens, new_rows;
  int64_t pages_used, pages_free;
  double  host_plan_us;                        /* lookup + page allocation + index assembly       */
  double  device_us;                           /* first kernel start to last kernel end (events)  */
  double  phase_us[PERCACHE_PH_COUNT];         /* filled when PERCACHE_FLAG_PHASE_TIMING is set   */
  int32_t phase_launches[PERCACHE_PH_COUNT];   /* kernels launched per class (always filled)      */
  int64_t attn_visible_pairs;                  /* sum over new rows of (position + 1)             */
  int64_t evictions;                           /* chunks evicted by the last prefill / put call   */
  int32_t gather_free;                         /* 1: the last prefill took the gather-free form   */
  int32_t reserved0;
} percache_stats_t;

PERCACHE_API int percache_get_stats(percache_t* h, percache_stats_t* out);

/* Replace the handle's flags (any PERCACHE_FLAG_* bits) after creation. */
PERCACHE_API int percache_set_flags(percache_t* h, uint32_t flags);

/* Integer plan of the last successful percache_prefill (host int32 arrays, caller-allocated).
 * which: 0 cu_ctx [n_prompts+1]; 1 cu_new [n_prompts+1]; 2 slot_chunk [ctx_tokens] (index into the prompt's
 * chunk list, n_chunks for query tokens); 3 slot_offset [ctx_tokens]; 4 slot_is_new [ctx_tokens];
 * 5 row_slot [new_rows] (slot of every new row inside its prompt = its position).
 * Returns the number of elements written, or a negative code (PERCACHE_E_CAPACITY if capacity is short). */
PERCACHE_API int64_t percache_debug_read_plan(percache_t* h, int32_t which, int32_t* out, int64_t capacity);

/* Host-only: the attention kernel's work schedule for tiles of given lengths, without a device (the part of
 * percache_prefill's index assembly that cuts every tile's units into items and deals them to the persistent
 * CTAs; the kernel itself is the causal GQA attention of the new rows over the assembled context, paper
 * Appendix B.1).  n_blocks [n_tiles]: context blocks (128 slots) each tile sees; units_per_tile: KV heads x
 * query-head pairs; n_ctas: CTAs available (one per SM); max_partial_slots: parts that may write partial results.
 * items_out: caller-allocated [items_capacity][6] int32 rows (tile, unit, blk_begin, blk_end, partial_slot or -1,
 * cta), in execution order.  counts_out [4]: items, CTAs used, split units, estimated makespan in quarter blocks.
 * Returns PERCACHE_OK, PERCACHE_E_INVAL, or PERCACHE_E_CAPACITY when items_capacity is short. */
PERCACHE_API int percache_debug_attn_plan(const int32_t* n_blocks, int32_t n_tiles, int32_t units_per_tile, int32_t n_ctas,
                             int32_t max_partial_slots, int32_t* items_out, int64_t items_capacity,
                             int64_t* counts_out);

/* Debugging aid for parity checks at full size and depth: while host_buf is set, every percache_prefill (and
 * percache_decode) call also copies the fp32 residual stream of its rows as it enters each decoder block, and once
 * more after the last block, to host_buf laid out [n_layers + 1][rows of the call][d_model] (entry l = input of
 * block l, entry n_layers = the call's output).  A checker can then feed block l's input to a reference
 * implementation and compare single blocks, which keeps the check affordable where a whole reference run is not.
 * host_buf: caller-owned host memory of capacity_floats floats that must stay valid until it is unset with NULL; a
 * prefill that needs more than the capacity fails with PERCACHE_E_CAPACITY before anything runs.  The copies
 * serialise the call's kernels: never leave this on while timing. */
PERCACHE_API int percache_debug_capture_layers(percache_t* h, float* host_buf, int64_t capacity_floats);

/* Test aid: the next decode step through the tree attention, percache_accept or percache_evict_context that gets to decoder
 * block `layer` (-1: none, the default) treats the launch of its cache operators there as failed, on the host: it
 * launches none of them from that block on and returns PERCACHE_E_CUDA. */
PERCACHE_API int percache_debug_fail_layer(percache_t* h, int32_t layer);

/* Assembled context of the last call: rotated K and V of one prompt and layer as fp16
 * [n_total + tokens decoded since][n_kv_heads][head_dim], copied to host buffers that hold capacity_tokens tokens
 * each (fewer than needed -> PERCACHE_E_CAPACITY, nothing is written).  PERCACHE_E_INVAL when the last call left no
 * assembled context (gather-free form, paper-faithful mode). */
PERCACHE_API int percache_debug_read_ctx(percache_t* h, int32_t prompt, int32_t layer, void* k_host, void* v_host,
                                         int64_t capacity_tokens);

/* Failure-path check that is safe to run: one tiny kernel waits, through the very wait function every tcgen05
 * kernel of this library uses, on a shared-memory barrier nobody arrives at.  The first waiter's limit is limit_us
 * (1..2000): its wait runs out and it records a code in the error word; a second waiter with a 1000 times longer
 * limit must leave as soon as it sees that code.  Nothing is in flight (no bulk copy, no tensor memory), the kernel
 * returns normally and the device stays usable.  Returns PERCACHE_E_DEVICE_TIMEOUT when the wait ran out as
 * designed (the mapping percache_prefill applies to a non-zero error word), PERCACHE_OK if the error word stayed
 * zero.  code_out: the recorded code (901 = the probe); waited_ns [2]: how long the two waiters waited.  Either
 * pointer may be NULL. */
PERCACHE_API int percache_debug_wait_probe(int32_t device, uint32_t limit_us, int32_t* code_out, uint64_t* waited_ns);

/* C[M][N] (fp32, host) = A[M][K] * B[N][K]^T with fp16 inputs (host), through the tcgen05 GEMM
 * (use_reference = 0), the plain kernel (1), or the tcgen05 GEMM on CTA pairs with 256 x 256 tiles (2; needs
 * N % 256 == 0).  Test hook for the GEMM core. */
PERCACHE_API int percache_debug_gemm(int32_t device, int32_t M, int32_t N, int32_t K, const void* a_f16, const void* b_f16,
                        float* c, int32_t use_reference);

/* The same GEMM as percache_debug_gemm(use_reference = 0) for callers that cannot allocate device memory.
 * The paper has no counterpart; this exists for two kinds of caller: one whose process has already given
 * all device memory to another allocator (so a raw cudaMalloc would fail), and one inside a serving loop
 * that must avoid the device-wide synchronisation of cudaMalloc / cudaFree.  The device copies of A, B, C
 * and the kernel's error word live in a fixed PERCACHE_NOALLOC_SCRATCH_BYTES array inside the library image
 * (every GPU that loads the library holds that much until the process exits).  The call itself performs no
 * cudaMalloc, cudaFree or other allocating routine.
 *  - Sizes: 256 + pad128(M)*K*2 + N*K*2 + M*N*4 bytes (each term rounded up to 256) must fit in the array,
 *    otherwise PERCACHE_E_CAPACITY and nothing runs.  K % 64 == 0, N % 128 == 0 as for percache_debug_gemm.
 *  - a_f16, b_f16, c are host buffers owned by the caller; the call returns after the result is in c.
 *  - The first call on a device looks up the array's device address; make that call before starting any
 *    stream capture on that device.
 *  - All calls share the one array and it keeps the previous call's bytes; the call clears what must start
 *    at zero.  Two calls whose GPU work overlaps (for instance from two host threads using the same device)
 *    race on it: serialise them. */
#define PERCACHE_NOALLOC_SCRATCH_BYTES (16u << 20)
PERCACHE_API int percache_debug_gemm_noalloc(int32_t device, int32_t M, int32_t N, int32_t K, const void* a_f16,
                                const void* b_f16, float* c);

/* QA-bank lookup (paper Section 3.4.1 "Similar Query Reuse"): cosine similarity of each query embedding with
 * every stored query embedding, the most similar entry, and whether its similarity exceeds tau_query (then the
 * cached answer of that entry can be returned without running the model).
 * bank: device fp32 [n_entries][dim] (dim a multiple of 4, rows 16-byte aligned); queries: device fp32
 * [n_queries][dim], n_queries <= 8 (PERCACHE_E_CAPACITY beyond).  Outputs are host arrays [n_queries]:
 * best_index (lowest index among equal maxima), best_score (cosine, fp32 arithmetic), hit (score > tau_query).
 * kernel_us: optional (may be NULL); receives the kernel's duration from CUDA events on the stream.
 * Runs on `stream` (a cudaStream_t or NULL) and returns after it has finished.  One lookup at a time per
 * device and process (the running maxima live in one device-side array of the library). */
PERCACHE_API int percache_qa_top1(int32_t device, void* stream, const float* bank, int32_t n_entries, int32_t dim,
                     const float* queries, int32_t n_queries, float tau_query, int32_t* best_index,
                     float* best_score, uint8_t* hit, float* kernel_us);

/* ------------------------------------------------------------------------------------------------------------------
 * Operators on the cache of a decoding batch.  The paper's decode stage (Section 2.1) produces one token at a time
 * against the keys and values of everything before it; these are the steps a server adds to it: verifying drafted
 * tokens several at a time, and keeping a prompt's context within a budget of slots.  They work on caller-owned device
 * memory, without a handle; percache_decode_tree, percache_accept and percache_evict_context run them on a handle's
 * own context.
 *
 * Rules of this group
 *  - The calls only enqueue work on `stream` (a cudaStream_t or NULL) of `device` and return: they do not synchronise,
 *    allocate or copy to the host, keep nothing between calls, leave the calling thread's current device as it was, and
 *    may be captured into a CUDA graph.  All array arguments are device memory of `device`, and must stay valid until
 *    the work has run.  Everything that differs from step to step (lengths, page tables, masks) is read on the device,
 *    so a captured call may be replayed after those arrays were rewritten in place.
 *  - NULL is the legacy default stream, which other streams do not wait for unless they were created to.
 *  - Sizes the host has to know are given as upper bounds (max_len, max_nodes).  Device-side values beyond them, or
 *    negative ones, are clamped; a page id or slot outside the pools reads as zeros and is never written.
 *  - Refused calls (PERCACHE_E_INVAL, PERCACHE_E_CAPACITY) enqueue nothing.  PERCACHE_E_CAPACITY: a workspace that is too
 *    small, or bounds that give tree_attention or attention_weights more work than they count: about
 *    ceil(max_len / 128) x KV heads x tiles (128 / (query heads a KV head) nodes each) of 2^29 a prompt, or of 2^35 a batch.
 *  - A prompt without rows, or a batch without prompts or rows, is allowed; outputs of rows at or behind
 *    row_start[n_seqs], and of slots behind a prompt's last one, are left as they were.
 *  - Bounded waits: where a kernel of this group gives up a wait (PERCACHE_E_DEVICE_TIMEOUT elsewhere), it says so in
 *    the workspace's first word, which percache_ops_status() reads. */
#define PERCACHE_BF16 0
#define PERCACHE_F16  1
#define PERCACHE_MAX_TREE_NODES 256
#define PERCACHE_OPS_WORKSPACE_BYTES (24u << 20)

/* K and V of a batch.  A slot of a prompt is a row of the pools: row page_table[b][slot / 16] * 16 + slot % 16 when
 * page_table is given, else row ctx_start[b] + slot.  In a row the heads lie one behind the other (head_dim elements
 * each).  K is as the attention uses it (after position encoding). */
typedef struct {
  void*   k;                       /* 16-byte aligned                                                             */
  void*   v;                       /* likewise; unused (may be NULL) by percache_attention_weights                */
  int64_t k_slot_stride;           /* elements from one row to the next, a multiple of 8, at least
                                      n_kv_heads * head_dim                                                       */
  int64_t v_slot_stride;
  int64_t n_slots;                 /* rows of each pool, at most 2^31 - 1                                         */
  const int32_t* page_table;       /* [n_seqs][page_table_stride] page ids, or NULL                               */
  const int32_t* ctx_start;        /* [n_seqs], used when page_table is NULL                                      */
  int32_t page_table_stride;       /* entries a prompt, at least ceil(max_len / 16)                               */
  int32_t n_kv_heads;
  int32_t head_dim;                /* 64 or 128                                                                   */
  int32_t dtype;                   /* PERCACHE_BF16 or PERCACHE_F16: of k, v, q and out                           */
} percache_kv_t;

/* The rows (drafted tokens, "nodes") of a batch.  Prompt b has ctx_len[b] context slots and
 * n = row_start[b + 1] - row_start[b] nodes; node i is row row_start[b] + i, and its K and V are in slot
 * ctx_len[b] + i.  It sees every context slot and the nodes j < n whose bit (j % 64 of word j / 64) is set in its row
 * of `mask`, itself included only if its own bit is set; without a mask it sees nodes 0 .. i. */
typedef struct {
  int32_t n_seqs;                  /* at most 65535                                                               */
  int32_t n_rows;                  /* rows of q, out, lse (and of mask and use)                                   */
  int32_t max_nodes;               /* most nodes of a prompt, 1 .. PERCACHE_MAX_TREE_NODES                        */
  int32_t max_len;                 /* most slots of a prompt, its nodes included; at most 2^26                    */
  const int32_t*  ctx_len;         /* [n_seqs]                                                                    */
  const int32_t*  row_start;       /* [n_seqs + 1], ascending                                                     */
  const uint64_t* mask;            /* [n_rows][mask_words] or NULL                                                */
  int32_t mask_words;              /* at least ceil(max_nodes / 64)                                               */
  int32_t reserved0;
} percache_rows_t;

/* Attention of every node over the slots it sees: out[row][head] = softmax(scale * q . K) V in fp32, rounded once
 * to the pools' type on the way out (the softmax weights are rounded to that type before they multiply V, their sum is
 * not; with fp16 a weight below 2^-21 of the largest is off by up to 2^-32 of that instead), and lse[row][head] = log of the sum of exp(scale * q . k) over those slots (fp32; may be NULL).  A row that
 * sees nothing gets zeros and -inf.  q, out: [n_rows][n_q_heads][head_dim] with q_row_stride / out_row_stride elements
 * from row to row (multiples of 8, 16-byte aligned); n_q_heads a multiple of n_kv_heads with at most 128 query heads
 * per KV head.  scale > 0.  Slots a row does not see may hold anything, infinities and NaN included.
 * workspace: PERCACHE_OPS_WORKSPACE_BYTES, 256-byte aligned, zeroed once before its first use; calls that may run at
 * the same time need a workspace each. */
PERCACHE_API int percache_tree_attention(int32_t device, void* stream, const percache_kv_t* kv,
                                         const percache_rows_t* rows, const void* q, int64_t q_row_stride,
                                         int32_t n_q_heads, float scale, void* out, int64_t out_row_stride, float* lse,
                                         void* workspace, int64_t workspace_bytes);

/* Running attention weights (what eviction by accumulated weight goes by): for every prompt b, KV head g and slot s
 *   weights_out[b][g][s] = decay * weights_in[b][g][s] + sum of exp(scale * q[r][h] . k[s][g] - lse[r][h])
 * over the rows r of the prompt with use[r] != 0 (use NULL: all) that see s and the query heads h of g.  lse as
 * percache_tree_attention wrote it (fp32 [n_rows][n_q_heads]); a row whose lse is -inf counts nothing.  Sums are kept
 * in fp32 and in a fixed order.  weights_in, weights_out: fp32 [n_seqs][n_kv_heads][weights_stride], weights_stride >=
 * max_len; they may be the same array.  decay 1 accumulates, a smaller one (>= 0) forgets; with decay 0 weights_in is
 * not read and may be NULL. */
PERCACHE_API int percache_attention_weights(int32_t device, void* stream, const percache_kv_t* kv,
                                            const percache_rows_t* rows, const void* q, int64_t q_row_stride,
                                            int32_t n_q_heads, float scale, const float* lse, const uint8_t* use,
                                            float decay, const float* weights_in, float* weights_out,
                                            int64_t weights_stride, void* workspace, int64_t workspace_bytes);

/* The slots to keep: of the length[b] slots of prompt b and every head, all when there are at most `budget`, else
 * `budget` of them: the first `sink`, the last `recent` (sink + recent <= budget), and the heaviest of the rest, equal
 * weights going to the lower slot (NaN counts as -infinity).  weights: fp32 [n_seqs][n_heads][weights_stride],
 * weights_stride >= max_len, at most 65535 heads.  keep: int32 [n_seqs][n_heads][budget], ascending, -1 behind the last one;
 * count[b] = min(length[b], budget).  budget: at most 2^26. */
PERCACHE_API int percache_select_slots(int32_t device, void* stream, const float* weights, int64_t weights_stride,
                                       const int32_t* length, int32_t n_seqs, int32_t n_heads, int32_t max_len,
                                       int32_t budget, int32_t sink, int32_t recent, int32_t* keep, int32_t* count);

/* Move kept slots together: for every prompt b, KV head g and j < count[b], slot first[b] + j of the destination gets
 * the K and V of slot keep[b][g][j] (first NULL: 0), and weights_out[b][g][first[b] + j] = weights_in[b][g][keep[b][g][j]]
 * (weights NULL: none).  keep: int32 [n_seqs][keep_heads][budget] with keep_heads = n_kv_heads, or 1 for a list that all
 * heads share.  An index outside 0 .. max_len - 1, or a destination slot at or past max_len, moves nothing.
 * dst_page_table / dst_start (as page_table / ctx_start of kv) NULL: in place; a list must then be strictly ascending
 * with keep[j] >= first + j, and no two prompts may share rows.  Else the destination's rows must not be rows that are
 * read, nor each other's.  weights_in and weights_out
 * may be the same array under the same rule as in place, with weights_stride >= max_len.  At most 65535 KV heads. */
PERCACHE_API int percache_compact_slots(int32_t device, void* stream, const percache_kv_t* kv, int32_t n_seqs,
                                        int32_t max_len, const int32_t* dst_page_table,
                                        int32_t dst_page_table_stride, const int32_t* dst_start, const int32_t* first,
                                        const int32_t* keep, int32_t keep_heads, int32_t budget, const int32_t* count,
                                        const float* weights_in, float* weights_out, int64_t weights_stride);

/* Waits for `stream` and reads the workspace's first word: PERCACHE_E_DEVICE_TIMEOUT if a wait of a call that used
 * this workspace ran out since it was last zeroed (outputs of calls since then are invalid), PERCACHE_E_CUDA if the
 * stream reports an error. */
PERCACHE_API int percache_ops_status(int32_t device, void* stream, const void* workspace);

PERCACHE_API const char* percache_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* PERCACHE_H_ */
