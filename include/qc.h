/*
 * qc.h -- C ABI of the Lazy Attention / Q Cache decode library (sm_100a).
 *
 * The library implements the decode-step attention of an MLLM decoder stack whose layers
 * are either ordinary ("full") or lazy, as defined in the paper's section "Method":
 *   - Eq. 2   decode attention of an ordinary layer over its KV cache plus the new token;
 *   - section "Lazy Attention": a lazy block is one ordinary layer l_c followed by lazy
 *     layers; the Q Cache holds the query of l_c;
 *   - Eq. 6   GLA decode: Q = Q Cache, K = K cache of l_c, V = the lazy layer's own;
 *   - Eq. 8   VLA decode: K = [own text K, visual K of l_c, own new k], V = own;
 *   - section "Efficiency Analysis": what each layer stores (all V; ordinary layers all K;
 *     VLA lazy layers text K only; GLA lazy layers no K) and the closed-form saving.
 *
 * Conventions common to every call
 *   - Every function returns an int32 status (QC_OK == 0).  Nothing throws, aborts or prints.
 *     On an error status the cache is unchanged and no output is written, with two exceptions:
 *     QC_ERR_CUDA (a CUDA call failed part-way: free the cache) and the device error word.  A
 *     kernel that gives up (a bounded wait that ran out, a page id or work range outside its
 *     limits) ends normally, leaves its part of the output unwritten and records a code in the
 *     device error word, mirrored into mapped host memory: qc_get_stats reports it, and every later
 *     qc_decode_step / qc_decode_step_host on that cache returns it instead of running.
 *   - "dev" pointers are CUDA device pointers on the context's device; "host" pointers are
 *     ordinary host memory.  All device memory is owned by the caller: the pool and the
 *     workspace are handed in at qc_alloc_cache and must outlive the cache.  The library
 *     allocates no device memory.  It owns the qc_ctx / qc_cache host objects and, per
 *     cache and from qc_alloc_cache on, 2 MiB of pinned host memory for what prompt calls upload
 *     and eight copies of a step's descriptors (32 bytes per sequence, 16 per layer and sequence).
 *   - Kernels are launched asynchronously on the stream given to qc_init.  Device pointers
 *     passed to a call must stay valid until that stream has executed the call.  Host arrays
 *     (seq_ids, n_tokens, kind) are consumed before the call returns.
 *   - bf16 tensors are dense, row-major in the index order written in brackets.
 *   - A sequence id is an integer in [0, max_seqs).  The token axis of a sequence is kept as
 *     two ordered streams, text and visual (the paper's "concatenation" simplification after
 *     Eq. 8); generated tokens are text.
 */
#ifndef QC_H_
#define QC_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct qc_ctx qc_ctx;     /* device, stream, SM count */
typedef struct qc_cache qc_cache; /* page tables, stream lengths, free list, Q Cache, plans */

enum {
  QC_OK = 0,
  QC_ERR_INVALID_ARG = 1, /* null pointer, out-of-range id or size, misaligned pointer */
  QC_ERR_UNSUPPORTED = 2, /* shape the kernels do not cover */
  QC_ERR_OOM_PAGES = 3,   /* the pool has too few free pages for this call */
  QC_ERR_STATE = 4,       /* lazy layer 0, decode on an unknown sequence, duplicate id, ... */
  QC_ERR_CUDA = 5,        /* a CUDA runtime call failed */
  QC_ERR_TIMEOUT = 6,     /* a bounded wait inside a kernel ran out (device error word) */
  QC_ERR_BAD_PAGE = 7,    /* a kernel met a page id outside the pool and did not follow it (device error word) */
  QC_ERR_PLAN = 8         /* a kernel met a work range outside the limits it was planned for (device error word) */
};

enum { QC_LAYER_FULL = 0, QC_LAYER_LAZY = 1 };

/* Which query scores which keys in a lazy layer (one mode per cache; the paper's overview
 * states that a model is optimised for a single mode).
 *   QC_MODE_VLA_QC  : text keys = own text K scored by the own q; visual keys = leader's
 *                     visual K scored by the Q Cache (the leader's q of the same token).
 *   QC_MODE_VLA_EQ8 : Eq. 8 as printed: the own q scores own text K and leader's visual K.
 *   QC_MODE_GLA     : Eq. 6: the Q Cache scores all of the leader's K.
 * V is always the lazy layer's own. */
enum { QC_MODE_VLA_QC = 0, QC_MODE_VLA_EQ8 = 1, QC_MODE_GLA = 2 };

/* Streams of one (layer, sequence), in allocation order. */
enum { QC_STREAM_K_TEXT = 0, QC_STREAM_K_VISUAL = 1, QC_STREAM_V_TEXT = 2, QC_STREAM_V_VISUAL = 3 };

enum { QC_KIND_TEXT = 0, QC_KIND_VISUAL = 1 };

typedef struct qc_config {
  int32_t n_layers;            /* 1..127 */
  int32_t n_q_heads;           /* multiple of n_kv_heads; query head h reads KV head h / group */
  int32_t n_kv_heads;
  int32_t head_dim;            /* 64 or 128 */
  int32_t page_size;           /* 16 = paged; 0 = contiguous: every stream owns a fixed extent of
                                  the pool (no allocator, no OOM), index
                                  ((layer*4 + stream)*max_seqs + seq) */
  int32_t max_seqs;            /* 1..4096 */
  int32_t max_tokens_per_seq;  /* bound on text tokens and on visual tokens of one sequence */
  int64_t n_pages;             /* pool capacity in pages (paged mode); ignored when contiguous */
  float softmax_scale;         /* 0 => 1/sqrt(head_dim) (Eq. 2) */
  int32_t lazy_mode;           /* QC_MODE_* */
  int32_t split_tokens;        /* keys per split-KV work item, a multiple of 16 in 16..512.  Every
                                  stream is cut into ceil(len/split_tokens) chunks whose partial
                                  results are merged by log-sum-exp.  0 => chosen per step among
                                  64, 128, 256 and 512 from the amount of work (workspace sized for 64). */
  const uint8_t* layer_kind;   /* host, [n_layers], QC_LAYER_*; layer 0 must be FULL; copied */
} qc_config;

typedef struct qc_stats {
  int64_t pages_total;            /* pool capacity in pages */
  int64_t pages_in_use;
  int64_t page_bytes;             /* bytes of one page: n_kv_heads * 16 * head_dim * 2 */
  int64_t kv_bytes_stored;        /* token-exact bytes of K and V rows held */
  int64_t kv_bytes_all_full;      /* token-exact bytes if every layer were ordinary */
  int64_t kv_bytes_stored_paged;  /* pages_in_use * page_bytes */
  int64_t kv_bytes_all_full_paged;/* page-rounded bytes if every layer were ordinary */
  int64_t qcache_bytes;           /* bytes of the Q Cache buffer */
  int64_t decode_steps;           /* qc_decode_step calls completed (enqueued) */
  int64_t attend_launches;        /* launches of the attention kernel so far */
  int32_t device_error;           /* 0, or the QC_ERR_* code the device error word holds */
  int32_t n_active_seqs;
  int64_t kernel_launches;        /* kernels of this library launched for the cache so far */
  int64_t kv_bytes_swept;         /* algorithmic K/V bytes of the decode steps so far: every stored row of the
                                     listed sequences once per step */
} qc_stats;

/* Per-step kernel timing (CUDA events on the library's stream), for roofline accounting. */
typedef struct qc_profile {
  int64_t steps;              /* decode steps covered */
  double attend_ms;           /* summed duration of the attention (split-KV partial) kernel; when a
                                 step runs as several launches, from the start of its first
                                 attention launch to the end of its last (merges between them
                                 included) */
  double step_ms;             /* summed duration of whole steps (setup+append+attend+merge) */
  int64_t kv_bytes_read;      /* algorithmic K/V bytes those steps had to read: every stored
                                 row of the listed sequences once, per step */
  int64_t items;              /* split-KV work items executed */
  int64_t prefill_calls;      /* qc_prefill_attend calls covered */
  double prefill_attend_ms;   /* summed duration of the prefill attention kernel */
  double prefill_flops;       /* its executed arithmetic: per (query, visible key) pair and query head,
                                 2 * head_dim flops for every score pass (one per layer, or one per
                                 run of layers that share their scores) and 2 * head_dim for every
                                 layer's value product */
  double attend_kernel_ms;    /* option "profile" = 2: summed durations of the attention launches alone,
                                 each between events of its own (events between launches end the
                                 overlap of a launch's start with its predecessor's end: this mode is
                                 for the kernel's time, not for the step's) */
  int64_t attend_kernel_launches;
} qc_profile;

/* Create a context on `device` that launches on `cuda_stream` (a cudaStream_t; NULL is the
 * legacy default stream).  Host object only. */
int32_t qc_init(int32_t device, void* cuda_stream, qc_ctx** out);

/* Bytes the caller must provide for a cache of this configuration.  pool_bytes covers the
 * K/V pages, workspace_bytes the page tables, Q Cache, split-KV partials, logit cache, plans and
 * staging. */
int32_t qc_cache_bytes_required(const qc_config* cfg, size_t* pool_bytes, size_t* workspace_bytes);

/* Build a cache over caller-owned device memory (both 256-byte aligned).  Page layout: one
 * page holds 16 tokens of ONE tensor (K or V) for all KV heads, [n_kv_heads][16][head_dim] bf16.
 * A lazy layer gets no visual-K pages (and in GLA no K pages at all): its reads go to the
 * leader's pages.  The pool contents are not initialised. */
int32_t qc_alloc_cache(qc_ctx* ctx, const qc_config* cfg, void* pool_dev, size_t pool_bytes,
                       void* workspace_dev, size_t workspace_bytes, qc_cache** out);

/* Append prompt tokens (Eq. 1: K and V of the prompt go to the KV cache).  Sequence seq_ids[i]
 * receives n_tokens[i] tokens; `kind` (host, QC_KIND_*, concatenated per sequence in call
 * order) routes each token to the text or the visual stream.  k_dev, v_dev:
 * bf16 [n_layers][sum n_tokens][n_kv_heads][head_dim].  K rows that the mode does not store
 * are ignored.  New sequences become active.  No attention is computed.  The call returns
 * after the copies have been enqueued and the host arrays consumed. */
int32_t qc_prefill_append(qc_cache* cache, int32_t n_seqs, const int32_t* seq_ids,
                          const int32_t* n_tokens, const uint8_t* kind, const void* k_dev,
                          const void* v_dev);

/* Prefill attention of one sequence's whole prompt, all layers, followed by what
 * qc_prefill_append does with the same k/v (section "Q Cache", prefilling forms):
 *   ordinary layer  Eq. 1: causal softmax((Q K^T + M)/sqrt(D)) V over the prompt;
 *   GLA lazy layer  Eq. 5: Q = Q Cache (the queries of the block's first layer for every prompt
 *                   token), K = that layer's K, V own;
 *   VLA lazy layer  Eq. 7 (both VLA modes): query rows and key rows of VISUAL tokens come from
 *                   the block's first layer, those of text tokens are the layer's own; V own.
 * Token t of the prompt sees tokens 0..t in the order given (kind[t] tags it text or visual).
 *   q_dev   bf16 [n_layers][n_tokens][n_q_heads][head_dim]   (the Q Cache of a block is its first
 *           layer's slice of this tensor; nothing prompt-sized is kept afterwards)
 *   k_dev, v_dev bf16 [n_layers][n_tokens][n_kv_heads][head_dim]
 *   out_dev bf16 [n_layers][n_tokens][n_q_heads][head_dim]
 * If the sequence already holds tokens (an earlier prompt chunk, generated tokens: a later turn of
 * a conversation), they precede the new ones: every new token also sees all of them, read from
 * the cache with the cache's own sharing (a lazy layer's visual keys -- in GLA all its keys -- are
 * its leader's), which is what Eq. 5 / Eq. 7 select for those tokens.
 * Errors of qc_prefill_append apply; on an error nothing is stored or written. */
int32_t qc_prefill_attend(qc_cache* cache, int32_t seq_id, int32_t n_tokens, const uint8_t* kind,
                          const void* q_dev, const void* k_dev, const void* v_dev, void* out_dev);

/* Calibration by-product (section "Lazy Attention", Eq. 3).  For a cache whose layers are ALL
 * ordinary (the analysis runs on the unmodified stack; otherwise QC_ERR_STATE) and one query
 * token per listed sequence -- normally the prompt's last token, whose K/V are already cached --
 * computes per layer the attention distribution of that query over every cached token, averaged
 * over the query heads, and the Jensen-Shannon divergence (natural log, 0..ln 2) between the
 * distributions of adjacent layers, averaged over the listed sequences:
 *   similarity_host[l] = mean_i JS(a_i^l, a_i^{l+1}),  l = 0 .. n_layers - 2   (host, written on return)
 *   q_dev     bf16 [n_layers][n_seqs][n_q_heads][head_dim]
 *   rows_dev  fp32 [n_layers][n_seqs][max_len], caller-owned scratch and by-product: the
 *             distributions, text tokens first then visual tokens, zero past a sequence's length
 * max_len >= every listed sequence's token count and <= 12288 (else QC_ERR_UNSUPPORTED).  The
 * cache is not changed.  Synchronises the stream. */
int32_t qc_layer_similarity(qc_cache* cache, int32_t n_seqs, const int32_t* seq_ids, const void* q_dev,
                            float* rows_dev, int32_t max_len, float* similarity_host);

/* Eq. 4 (host only): layer l+1 joins the lazy block of layer l when similarity[l] < eps
 * (0 < eps <= 1) and, if max_block > 0, the block has fewer than max_block layers.  Writes
 * layer_kind[n_layers] for qc_config: the first layer of every block stays ordinary. */
int32_t qc_lazy_blocks(const float* similarity, int32_t n_layers, float eps, int32_t max_block,
                       uint8_t* layer_kind);

/* One generated (text) token for each listed sequence through all layers (Eq. 2, 6, 8):
 * appends k/v, refreshes the Q Cache from every ordinary layer's q, computes split-KV partial
 * attention and merges the partials by log-sum-exp.
 *   q_dev   bf16 [n_layers][n_seqs][n_q_heads][head_dim]
 *   k_dev   bf16 [n_layers][n_seqs][n_kv_heads][head_dim]  (rows of GLA lazy layers ignored)
 *   v_dev   bf16 [n_layers][n_seqs][n_kv_heads][head_dim]
 *   out_dev bf16 [n_layers][n_seqs][n_q_heads][head_dim]
 *   lse_out_dev  optional fp32 [n_layers][n_seqs][n_q_heads], natural-log sum of exp; may be NULL
 * seq_ids (host) must be distinct active sequences.  The call is asynchronous. */
int32_t qc_decode_step(qc_cache* cache, int32_t n_seqs, const int32_t* seq_ids, const void* q_dev,
                       const void* k_dev, const void* v_dev, void* out_dev, float* lse_out_dev);

/* The same step issued layer by layer, for a caller whose layer l+1 inputs only exist after layer l's
 * output (a model that computes layer after layer).  qc_decode_begin does the step's page planning
 * for the listed sequences (distinct, active) and plans every layer's launch; then exactly n_layers
 * calls of qc_decode_layer follow, for layer 0, 1, ... in order, each with that layer's slices
 *   q_dev bf16 [n_seqs][n_q_heads][head_dim], k_dev / v_dev bf16 [n_seqs][n_kv_heads][head_dim],
 *   out_dev bf16 [n_seqs][n_q_heads][head_dim], lse_out_dev optional fp32 [n_seqs][n_q_heads].
 * A call appends the layer's k/v (and refreshes the Q Cache from an ordinary layer's q) and runs the
 * layer's attention launch and its merge, asynchronously (the append is part of the attention
 * launch: no launch of its own); out_dev is complete when the stream
 * has executed the call.  The launches are those of the in-order schedule ("in_order_launches"):
 * a leader's call also weights its followers' cached V rows, so a follower's call is short (VLA_QC:
 * its text sweep; GLA: the merge with the new token as one more key; k_dev of a GLA follower is
 * ignored).  Results equal qc_decode_step's.  While a step is open (begun, layers left), every call
 * that would change the cache returns QC_ERR_STATE; a step cannot be abandoned: the sequences'
 * lengths and pages were committed by qc_decode_begin.  Errors: as qc_decode_step; a layer out of
 * order or without an open step is QC_ERR_STATE. */
int32_t qc_decode_begin(qc_cache* cache, int32_t n_seqs, const int32_t* seq_ids);
int32_t qc_decode_layer(qc_cache* cache, int32_t layer, const void* q_dev, const void* k_dev, const void* v_dev,
                        void* out_dev, float* lse_out_dev);

/* Same step with HOST buffers of the same layouts.  The step runs as up to four launch groups of
 * consecutive lazy blocks; on two internal copy streams the inputs of a group are copied to
 * staging in the workspace while the previous group computes, and its outputs are copied back
 * while the next one computes.  Returns when everything has been copied back.  Pinned host
 * buffers make the copies asynchronous; pageable ones also work (without the overlap). */
int32_t qc_decode_step_host(qc_cache* cache, int32_t n_seqs, const int32_t* seq_ids,
                            const void* q_host, const void* k_host, const void* v_host,
                            void* out_host, float* lse_out_host);

/* Release a sequence: its pages return to the free list in reverse order of allocation. */
int32_t qc_free_seq(qc_cache* cache, int32_t seq_id);

/* Destroy a cache and/or a context (either may be NULL).  Waits for the stream first.
 * Caller-owned device memory is not touched. */
int32_t qc_free(qc_ctx* ctx, qc_cache* cache);

/* Accounting for the "KV bytes saved" metric (section "Efficiency Analysis").  Also reads the
 * device error word (this synchronises the stream). */
int32_t qc_get_stats(qc_cache* cache, qc_stats* out);

/* Page table of one stream, from the host mirror.  Writes up to `cap` page ids, the page
 * count, the stream length in tokens and the layer that owns the pages: `layer` itself, the
 * leader if the stream is an alias, -1 (and zero pages) if the sequence is not active. */
int32_t qc_debug_page_table(const qc_cache* cache, int32_t layer, int32_t stream, int32_t seq_id,
                            int32_t* page_ids, int32_t cap, int32_t* n_pages, int32_t* n_tokens,
                            int32_t* owner_layer);

/* Copy the Q Cache entry a lazy layer reads (its leader's latest queries) to the host:
 * bf16 [max_seqs][n_q_heads][head_dim].  Synchronises the stream. */
int32_t qc_debug_read_qcache(qc_cache* cache, int32_t layer, void* host_bf16);

/* Copy one stored row (bf16 [head_dim]) of a stream to the host; aliases resolve to the
 * leader's pages.  Synchronises the stream.  For tests of the append path. */
int32_t qc_debug_read_row(qc_cache* cache, int32_t layer, int32_t stream, int32_t seq_id,
                          int32_t token, int32_t kv_head, void* host_bf16);

/* Tuning knobs (all optional).  key: "split_tokens" (as in qc_config, never below the value
 * the cache was created with; 0 = per-step choice), "layers_per_launch"
 * (0 = one attention launch for the whole step; k>0 = one launch per k consecutive lazy
 * blocks, in layer order), "per_layer_logit_cache" (1 = one attention + merge launch per layer,
 * in layer order: the schedule of a model in which a layer's q/k/v only exist after the previous
 * layer has run.  A leader with followers then also stores its scaled scores -- of the visual keys
 * in VLA_QC, of all keys in GLA -- in a logit cache inside the workspace, 4 bytes per key and
 * query head, and a follower weights its own V rows with them instead of reading the leader's K
 * again; by Eq. 6 / the Q Cache rule the follower's scores are the leader's, so the result is the
 * one of the fused schedule.  VLA_EQ8 followers score with their own query and re-read the
 * leader's visual K.  0 = back to one launch per step.  qc_decode_step only),
 * "prefill_tcgen05" (0 = use the mma.sync prefill kernel), "prefill_shared_scores" (GLA only: by
 * Eq. 5 the layers of a lazy block attend with the same Q and K, so qc_prefill_attend computes and
 * normalises their scores once per run of up to three layers and applies them to each layer's V,
 * bit-identically to one pass per layer; 0 = never, 1 = for prompts of 1536 tokens or more (the
 * default: below that the pass's lower occupancy costs more than it saves), 2 = always),
 * "prefill_pair_min_tokens" (n > 0: prompts of n tokens or more that start a sequence run on the
 * prefill kernel with two query tiles per CTA and 128-key tiles; 0, the default: never),
 * "profile" (1 = record CUDA events per step; 2 = also around every attention launch), "in_order_launches"
 * (1 = one launch per layer in layer order, each using nothing of later layers; what a follower
 * shares with its leader are scores over rows cached before the step, so a leader's launch also
 * weights its followers' cached V rows and leaves their partial rows behind; a VLA_QC follower's
 * launch is its text sweep, a GLA follower's is the merge with the step's new token as one more
 * key, Eq. 6; VLA_EQ8 followers sweep the leader's visual K with their own query), "static_partition"
 * (-1 = a step of several launches cuts each launch's work into equal ranges of K/V tiles, one or a
 * few per worker, instead of handing out chunk items; 0 = never; 1 = always), "static_min_tiles",
 * "static_row_cost" (tuning of those ranges: shortest range, and what one more output row counts
 * for, in 4 KiB tiles), "plan_ahead" (0 = workers locate their ranges themselves instead of reading
 * starting points that one kernel per step works out for every launch), "fused_merge" (1, the default = an
 * attention launch of one layer without query groups merges its output rows itself where the step's launches
 * are planned ahead and n_seqs * n_q_heads is at most four per SM; 0 = always by a merge launch),
 * "row_cluster" (in-order schedule and qc_decode_layer, with the options above as they come: CTAs that each
 * output row gets in launches that finish their rows themselves, without plan, partials or merge launch;
 * -1, the default = chosen from the numbers of rows and pages, among 1, 2, 4 and 8 or tile ranges; 0 = never;
 * 1 to 8 = that many, where no lazy block has more than four layers and no launch of the step has more than 60
 * pages of its lightest sweep for every worker; larger steps claim chunk items), "row_warps" (the same with one CTA
 * of 1, 2, 3, 4 or 6 warps per row, without query groups; 0, the default = chosen),
 * "fold_append" (in-order schedule and qc_decode_layer; 1, the default = a layer's new k/v rows and an
 * ordinary layer's q are taken from the inputs and stored by that layer's own launch; 0 = by an
 * append when the step begins, resp. an append launch per layer call),
 * "debug_drop_tile" (test hook for the error path: 1 = every worker of an attention launch leaves
 * out the copy of its first tile and waits for it with a short limit; nothing is in flight for that
 * wait, so it runs out, the worker records QC_ERR_TIMEOUT and returns, and the kernel ends normally
 * with its rows unwritten). */
int32_t qc_set_option(qc_cache* cache, const char* key, int64_t value);

/* Sum the recorded kernel times since the last call (synchronises), then reset them. */
int32_t qc_get_profile(qc_cache* cache, qc_profile* out);

/* ---- A call for callers that cannot allocate ------------------------------------------------
 *
 * The paper has no counterpart to this call; it exists for deployment reasons.  Everything
 * above works on memory the caller allocates and hands over.  Some callers cannot do even
 * that at the moment they need attention computed: a serving process whose device memory
 * was partitioned at start-up and whose allocator is frozen afterwards, or code running
 * inside another framework's callback where device allocation is forbidden.  For them
 * qc_attend_static computes plain decode attention (Eq. 2) using only the tensors passed in
 * plus a fixed scratch array that is part of the library image.
 *
 *   q_dev   bf16 [n_seqs][n_q_heads][head_dim]              one query token per sequence
 *   k_dev   bf16 [n_seqs][n_tokens][n_kv_heads][head_dim]   keys, the new token's included
 *   v_dev   bf16 [n_seqs][n_tokens][n_kv_heads][head_dim]
 *   out_dev bf16 [n_seqs][n_q_heads][head_dim]
 *   softmax_scale 0 => 1/sqrt(head_dim)
 *
 * The key axis is cut into QC_STATIC_SPLITS ranges whose partial softmax results are kept in
 * the scratch array and merged by log-sum-exp.  The array holds QC_STATIC_MAX_ROWS *
 * QC_STATIC_SPLITS * 130 floats (about 2 MiB) on every GPU that loads the library, for the
 * life of the process.  Limits: n_seqs * n_q_heads <= QC_STATIC_MAX_ROWS, n_tokens <=
 * QC_STATIC_MAX_TOKENS, head_dim 64 or 128; anything larger returns QC_ERR_INVALID_ARG and
 * launches nothing.
 *
 * The call performs no device or pinned-host allocation and frees nothing.  Its first call
 * on a device looks up the scratch array's device address (once per device).  That look-up, or
 * the first launch, may be the moment the CUDA runtime loads the library's device code onto the
 * GPU, scratch array included -- the one thing here that does take device memory -- so make one
 * call per device at start-up, while memory may still be taken, and outside any stream capture.
 * The calling thread's current device is the same after the call as before.  All calls share the one array, and it keeps whatever
 * the previous call left there: each call overwrites every entry it later reads, so nothing
 * needs clearing, but two calls whose kernels overlap on the GPU (different streams, or
 * different host threads) race on it.  Serialise them on one stream.  Asynchronous on
 * `cuda_stream`; pointers must be 16-byte aligned. */
#define QC_STATIC_MAX_ROWS 512
#define QC_STATIC_SPLITS 8
#define QC_STATIC_MAX_TOKENS 65536
int32_t qc_attend_static(int32_t device, void* cuda_stream, const void* q_dev, const void* k_dev,
                         const void* v_dev, void* out_dev, int32_t n_seqs, int32_t n_tokens,
                         int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float softmax_scale);

/* ---- A cache in 4 bits ------------------------------------------------------------------------
 *
 * The paper has no counterpart to these calls; they make the same use of a cache possible in 27 % of the
 * memory.  Each is complete in itself: device memory is the caller's, nothing is kept between calls, every
 * number that changes from step to step (lengths, page ids, slots) is read on the device, so a step may be
 * captured into a graph once and replayed while its sequences grow.  All calls are asynchronous on
 * `cuda_stream`; the calling thread's current device is the same afterwards.
 *
 * A token axis is a stream, as everywhere here: a stack with lazy layers has a text and a visual one.  One page
 * table serves all layers of a stream.  A layer has a pool for K and one for V per stream, both of n_pages pages
 * addressed by the table's page ids; a lazy layer has no pool for visual K (in GLA for no K): it names its
 * leader's.
 *
 * Device data that does not fit (an id out of range, too few pages) is met on the device: nothing outside the
 * given memory is touched, and a QC_ERR_* code is left in a status word that the caller may read when it likes
 * (the largest code stays; it is never cleared by the calls).  What a call writes overlaps nothing else that it is given, but
 * where it says so. */
#define QC_TABLE_MAX_BATCH 4096   /* sequences listed in one call */
#define QC_TABLE_MAX_SEQS 65536   /* rows of a page table */
#define QC_QUANT_MAX_HEADS 1024
#define QC_QUANT_MAX_SEQS 2048    /* sequences in one qc_quant_attend */
#define QC_QUANT_MAX_QUERIES 16   /* query tokens of one sequence in one qc_quant_attend */
#define QC_QUANT_MAX_TOKENS (1 << 30)   /* tokens of one qc_quant_append or qc_quant_read, slots of one qc_table_extend */

/* Page table of one stream, all arrays int32 on the device. */
typedef struct qc_table {
  int32_t max_seqs;     /* rows */
  int32_t max_pages;    /* pages a row has room for */
  int32_t page_size;    /* tokens of a page: 16, 32 or 64 */
  int32_t n_pages;      /* pages there are; n_pages * page_size < 2^31 */
  int32_t* pages_dev;   /* [max_seqs][max_pages], -1 where a sequence has no page */
  int32_t* lens_dev;    /* [max_seqs] tokens */
  int32_t* free_dev;    /* [n_pages] the free pages, as a stack: the next one taken is free[state[0] - 1] */
  int32_t* state_dev;   /* [4]: number of free pages, status word, two reserved */
} qc_table;

/* Empty table: no tokens, all pages free (0 is taken first), status QC_OK. */
int32_t qc_table_reset(int32_t device, void* cuda_stream, const qc_table* table);

/* n_new_dev[i] (null: 1) more tokens for row seq_ids_dev[i] (null: i) of the table, i < n_seqs.  Pages are
 * taken in the order of the list, then of the tokens.  The counts may be the table's lengths, here and in qc_table_trim: they
 * are read before any of it is written.
 *   starts_dev [n_seqs + 1]  the new tokens are numbered through the list: sequence i's are starts[i] .. starts[i + 1] - 1
 *   slots_dev  [max_slots]   where token t goes: page id * page_size + place in the page; -1 behind the last token
 * All or nothing: on an id out of range or a negative count (QC_ERR_INVALID_ARG), an id listed twice or lengths
 * and free pages that cannot be (QC_ERR_STATE), too few free pages or a row without room (QC_ERR_OOM_PAGES), or
 * more than max_slots tokens (QC_ERR_INVALID_ARG), the status word is set, the table stays as it was, starts are 0
 * and slots -1. */
int32_t qc_table_extend(int32_t device, void* cuda_stream, const qc_table* table, int32_t n_seqs, const int32_t* seq_ids_dev,
                        const int32_t* n_new_dev, int32_t max_slots, int32_t* starts_dev, int32_t* slots_dev);

/* Row seq_ids_dev[i] keeps its first n_keep_dev[i] tokens (null: 0, the sequence is released; more than it has: all).
 * Pages that become empty are free again, in an order that the same qc_table_extend takes them back in.  All or
 * nothing as above. */
int32_t qc_table_trim(int32_t device, void* cuda_stream, const qc_table* table, int32_t n_seqs, const int32_t* seq_ids_dev,
                      const int32_t* n_keep_dev);

/* Shape of a pool: one tensor (K or V) of one layer and stream. */
typedef struct qc_quant_shape {
  int32_t n_kv_heads;   /* 1..QC_QUANT_MAX_HEADS */
  int32_t head_dim;     /* 64 or 128 */
  int32_t page_size;    /* 16, 32 or 64 */
  int32_t n_pages;      /* n_pages * page_size < 2^31 */
} qc_quant_shape;

/* n_pages * n_kv_heads * page_size * (head_dim / 2 + 4).  A row (token, head) is held as lo = its smallest element,
 * r = bf16(15 / (largest - lo)) and codes rint((x - lo) * r) in 4 bits, and stands for lo + code / r.  A row whose
 * range is below 2^-100 stands for lo throughout (r = 0); one with an element that is infinite or no number, or with
 * a range that is not finite, stands for NaN throughout.
 * A page is the codes [n_kv_heads][page_size / 16][8 * head_dim bytes], then [n_kv_heads][page_size] words of lo as
 * bf16 (low half) and r as bf16.  Inside a block of 16 tokens, in bytes of two elements, the even one low:
 *   K, 128 wide  [token % 2][token / 2][d / 32][d / 2 % 16]      V, 128 wide  [d / 8 % 2][d / 16][token / 4][d / 2 % 4][token % 4]
 *   K,  64 wide  [token / 2][d / 16][token % 2][d / 2 % 8]       V,  64 wide  [d / 8][token / 4][d / 2 % 4][token % 4] */
int32_t qc_quant_pool_bytes(const qc_quant_shape* shape, size_t* bytes);

/* Quantise rows and store them: row t of k_dev / v_dev (bf16 [n_tokens][n_kv_heads][head_dim], tokens k_stride /
 * v_stride elements apart, heads dense) at slots_dev[t].  A slot that is negative or not in the pool is left out.
 * Either pair (k_dev, k_pool_dev), (v_dev, v_pool_dev) may be null.  Pointers 16-byte aligned, strides multiples of 8.
 * Slots are distinct; of rows with the same slot, what that row holds afterwards is not specified. */
int32_t qc_quant_append(int32_t device, void* cuda_stream, const qc_quant_shape* shape, int32_t n_tokens,
                        const int32_t* slots_dev, const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride,
                        void* k_pool_dev, void* v_pool_dev);

/* What the rows at slots_dev stand for, as bf16 [n_tokens][n_kv_heads][head_dim] (dense): what the attention of a
 * later prompt chunk is computed on.  Rows of slots that are negative or not in the pool are left as they are. */
int32_t qc_quant_read(int32_t device, void* cuda_stream, const qc_quant_shape* shape, int32_t n_tokens,
                      const int32_t* slots_dev, const void* k_pool_dev, const void* v_pool_dev, void* k_out_dev,
                      void* v_out_dev);

/* One stream as qc_quant_attend reads it. */
typedef struct qc_quant_stream {
  const void* q_dev;           /* bf16 [n_tokens][n_q_heads][head_dim], tokens q_stride elements apart (0: one row for all) */
  int64_t q_stride;
  const void* k_pool_dev;
  const void* v_pool_dev;
  const int32_t* pages_dev;    /* of the stream's table */
  const int32_t* lens_dev;
  int32_t max_pages, n_pages;
} qc_quant_stream;

typedef struct qc_quant_attend_args {
  int32_t n_q_heads, n_kv_heads, head_dim, page_size;
  int32_t n_seqs, max_seqs;      /* sequences of the call; rows of the tables */
  int32_t n_tokens;              /* query tokens: rows of q and out */
  int32_t max_queries;           /* most query tokens of one sequence, 1..QC_QUANT_MAX_QUERIES */
  int32_t causal;                /* 1: the queries' own tokens are the last of the text stream, and a query sees none behind its own */
  float softmax_scale;           /* 0 => 1/sqrt(head_dim) */
  const int32_t* seq_ids_dev;    /* [n_seqs] table row of each sequence; null: i */
  const int32_t* starts_dev;     /* [n_seqs + 1] query tokens of each sequence, as qc_table_extend numbers them; null: one each */
  qc_quant_stream text;
  qc_quant_stream visual;        /* all null: one stream */
  void* out_dev;                 /* bf16 [n_tokens][n_q_heads][head_dim]; over a q_dev only with each row at the place of its query
                                    (anything else that overlaps: QC_ERR_INVALID_ARG), over no other argument */
  float* lse_out_dev;            /* optional fp32 [n_tokens][n_q_heads], natural-log sum of exp */
  void* workspace_dev;           /* qc_quant_workspace_bytes; need not be cleared; one call at a time */
  size_t workspace_bytes;
  int32_t* status_dev;           /* optional status word */
} qc_quant_attend_args;

int32_t qc_quant_workspace_bytes(const qc_quant_attend_args* args, size_t* bytes);

/* Attention of each sequence's query tokens over its cached rows: one softmax over the visual stream's keys scored by
 * visual.q_dev and the text stream's keys scored by text.q_dev (an ordinary layer, VLA_EQ8: the same queries twice;
 * VLA_QC: the Q Cache on the leader's visual K; GLA: the Q Cache on both of the leader's).  V is what the pools hold.
 * A query that sees no key gets 0 and lse minus infinity.  Rows of out that belong to no listed sequence are left as
 * they are, and so are those of a sequence whose row or query numbers are out of range (QC_ERR_INVALID_ARG in the status
 * word).  A page id that is not in the pool is not followed: its keys count as absent (QC_ERR_BAD_PAGE).  A length
 * beyond the table's room is cut to it (QC_ERR_PLAN).  Lengths that another stream changes while a call runs make that call's
 * rows wrong, and no later call's: a captured call is right again in its next replay.  A batch that is too much for one call (over 2^32 rows of K, counted
 * once per KV head and per 2, 4, 8 or 16 query rows, or a sequence with more than 2^28 of them) is not computed at all
 * (QC_ERR_PLAN): out stays as it was.
 * Query elements are kept to 2^-35 of the largest element of their row (token, head; a stream's); a row with an element of 2^101
 * or more in size, infinite or no number gets NaN, and no other row is different for it. */
int32_t qc_quant_attend(int32_t device, void* cuda_stream, const qc_quant_attend_args* args);

/* ---- Positions, and a cache in bf16 pages ------------------------------------------------------
 *
 * The paper has no counterpart to these calls.  Everything above takes rotated queries and keys; qc_rotate makes them
 * (per-head norm and rotation by positions of one or several axes), qc_paged_append does the same on a key's way into a
 * cache, and qc_paged_attend attends over that cache where sequences share a prefix (many questions about one image).
 * The cache is bf16 pages behind the page tables above (qc_table_*): a pool holds one tensor (K or V) of one layer and
 * stream as bf16 [n_pages][n_kv_heads][page_size][head_dim], and a token is at its slot, page id * page_size + place.  As above
 * each call is complete in itself, asynchronous on `cuda_stream`, may be captured and replayed, and reads what changes from
 * step to step on the device. */
#define QC_ROTATE_MAX_AXES 4
#define QC_PAGED_MAX_HEADS 1024
#define QC_PAGED_MAX_SEQS 2048     /* sequences in one qc_paged_attend */
#define QC_PAGED_MAX_QUERIES 128   /* query tokens of one sequence in one qc_paged_attend */
#define QC_PAGED_MAX_TOKENS (1 << 24)   /* tokens of one qc_rotate, qc_paged_append or qc_paged_attend */

/* A row x of one token and head becomes y = x / sqrt(mean x^2 + eps) * w where its norm weights are given, and then each pair i of
 * its first rotary_dim elements is turned by the angle positions[axes[i]][token] * freqs[i]:
 *   (a, b) -> (a cos - b sin, b cos + a sin),  elements (i, i + rotary_dim / 2), or (2 i, 2 i + 1) where `adjacent`.
 * In fp32 throughout, rounded once; an angle is off by a rounding to fp32, 2^-26 turns at most, at every position (for frequencies
 * below 2^32 in size).  Squares are summed in fp32: elements are below 2^60 in size, and where eps
 * is 0 each row has one above 2^-60.  A pair whose axis is none of the n_axes, or whose frequency is not finite, becomes NaN.
 * Rows are bf16 [n_tokens][heads][head_dim], heads dense, tokens `stride` elements apart (multiples of 8, pointers 16-byte
 * aligned).  An output lies over its own input (same pointer and stride) or over nothing
 * that the call reads or writes besides (QC_ERR_INVALID_ARG). */
typedef struct qc_rotate_args {
  int32_t n_tokens, n_q_heads, n_kv_heads;
  int32_t head_dim;              /* 64 or 128 */
  int32_t rotary_dim;            /* elements that turn: a multiple of 16, at most head_dim; 0: none */
  int32_t adjacent;              /* 0: pairs (i, i + rotary_dim / 2); 1: pairs (2 i, 2 i + 1) */
  int32_t n_axes;                /* 1..QC_ROTATE_MAX_AXES */
  int32_t norm_f32;              /* norm weights are fp32 (1) or bf16 (0) */
  const float* freqs_dev;        /* [rotary_dim / 2] radians per position */
  const int32_t* axes_dev;       /* [rotary_dim / 2] the axis of each pair; null: 0 */
  const int32_t* positions_dev;  /* [n_axes][n_tokens], axes position_stride elements apart */
  int64_t position_stride;
  const void* q_norm_dev;        /* [head_dim] weights; null: no norm */
  const void* k_norm_dev;
  float eps;                     /* of both norms */
  const void* q_dev;             /* either of q and k may be null */
  int64_t q_stride;
  void* q_out_dev;
  int64_t q_out_stride;
  const void* k_dev;
  int64_t k_stride;
  void* k_out_dev;               /* qc_paged_append: null, K goes to its pool */
  int64_t k_out_stride;
} qc_rotate_args;

int32_t qc_rotate(int32_t device, void* cuda_stream, const qc_rotate_args* args);

typedef struct qc_paged_append_args {
  qc_rotate_args rows;           /* q optional; k null where the layer stores none */
  const void* v_dev;             /* bf16 [n_tokens][n_kv_heads][head_dim], stored as it is; null: none */
  int64_t v_stride;
  const int32_t* slots_dev;      /* [n_tokens] */
  int32_t page_size, n_pages;    /* 16, 32 or 64; n_pages * page_size < 2^31 */
  void* k_pool_dev;
  void* v_pool_dev;
} qc_paged_append_args;

/* The same, K and V stored at their slots.  A slot that is negative or not in the pool is left out (its query is still made).
 * Slots are distinct; of rows with the same slot, what that row holds afterwards is not specified. */
int32_t qc_paged_append(int32_t device, void* cuda_stream, const qc_paged_append_args* args);

/* One stream as qc_paged_attend reads it. */
typedef struct qc_paged_stream {
  const void* q_dev;             /* bf16 [n_tokens][n_q_heads][head_dim], tokens q_stride elements apart (0: one row for all) */
  int64_t q_stride;
  const void* k_pool_dev;
  const void* v_pool_dev;
  const int32_t* pages_dev;      /* [rows][max_pages] of the stream's table */
  const int32_t* lens_dev;       /* [rows] */
  int32_t max_pages, n_pages, rows;
} qc_paged_stream;

typedef struct qc_paged_attend_args {
  int32_t n_q_heads, n_kv_heads, head_dim, page_size;
  int32_t n_seqs;                /* sequences of the call */
  int32_t n_tokens;              /* query tokens: rows of q and out */
  int32_t max_queries;           /* most query tokens of one sequence, 1..QC_PAGED_MAX_QUERIES */
  int32_t causal;                /* 1: the queries' own tokens are the last of the own stream, and a query sees none behind its own */
  float softmax_scale;           /* 0 => 1/sqrt(head_dim) */
  int32_t n_groups;              /* 0 without a shared stream */
  const int32_t* seq_ids_dev;    /* [n_seqs] row of the own table of each sequence; null: i */
  const int32_t* starts_dev;     /* [n_seqs + 1] query tokens of each sequence, as qc_table_extend numbers them; null: one each */
  const int32_t* groups_dev;     /* [n_groups + 1] sequences groups[g] .. groups[g + 1] - 1 of the call share a prefix; null: one
                                    group of all sequences */
  const int32_t* shared_ids_dev; /* [n_groups] its row of the shared table; null: g */
  qc_paged_stream own;
  qc_paged_stream shared;        /* all null: no sequence has a prefix */
  void* out_dev;                 /* bf16 [n_tokens][n_q_heads][head_dim], over no other argument */
  float* lse_out_dev;            /* optional fp32 [n_tokens][n_q_heads], natural-log sum of exp */
  void* workspace_dev;           /* qc_paged_workspace_bytes of these sizes and lists, 256-byte aligned; need not be cleared; one call at a
                                    time; over no other argument (this is not checked) */
  size_t workspace_bytes;
  int32_t* status_dev;           /* optional status word */
} qc_paged_attend_args;

int32_t qc_paged_workspace_bytes(const qc_paged_attend_args* args, size_t* bytes);

/* Attention of each sequence's query tokens over its prefix, if it is in a group, and its own cached tokens: one softmax over the
 * prefix's keys scored by shared.q_dev and its own keys scored by own.q_dev (an ordinary layer: the same queries twice; a
 * lazy layer whose prefix is the image: the Q Cache on the leader's visual K).  A prefix is read once for all query rows of its
 * group (once per 128 rows of a KV head), whose sequences are adjacent in the list; sequences before the first group and behind the
 * last have none.  All tokens of a prefix are seen by every query.  A query that sees no key gets 0 and lse minus infinity, and so
 * does one whose scores are all minus infinity.  What the pools hold where no token is counts for nothing, whatever it is.
 * The work is divided by sizes alone, so a call gives the same bits each time.  Weights are rounded to bf16 for their products with
 * values, their sums are not; scores and sums are fp32, with weights up to 2^9: where the |q k| of a query and a key, scaled or not, add
 * up to 2^126, or the |values| of a query's keys to 2^118, its row may become infinite or no number.
 * All or nothing: rows out of range, starts or groups that do not ascend or reach outside, more queries than max_queries
 * (QC_ERR_INVALID_ARG in the status word) and batches of too much work (QC_ERR_PLAN) leave out as it was.  Too much is a sum above 2^30
 * (some seconds) over the prefixes and sequences that have keys and more than 16 query rows a KV head, of KV heads * ceil(rows / 128) *
 * (ceil(keys / 64) + 2), or over those of 1 to 16 rows, of KV heads * (ceil(keys / 16) + 6).  A page id that is not in the pool is not
 * followed: its keys count as absent (QC_ERR_BAD_PAGE).  A length beyond the table's room is cut to it, a negative one counts as 0
 * (QC_ERR_PLAN).  Rows of out that belong to no sequence are left as they are. */
int32_t qc_paged_attend(int32_t device, void* cuda_stream, const qc_paged_attend_args* args);

const char* qc_status_string(int32_t status);

#ifdef __cplusplus
}
#endif
#endif /* QC_H_ */
