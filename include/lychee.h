/*
 * lychee.h — C ABI of the MI355X (gfx950) decode-step hybrid-head sparse attention.
 *
 * One decode step of LycheeDecode's attention (Sec. 3.1; Alg. 1, the per-head loop of
 * App. B): in every layer the few *retrieval heads* attend over the whole KV cache
 * (Eq. 1) and pick the k highest-scoring positions (Eq. 2); the *sparse heads* attend
 * only over the k rows named by the set inherited from the previous layer (Eq. 3) and
 * hand that set on unchanged.  Under grouped-query attention there is one set per KV
 * head, ranked by the mean logit of the group's retrieval heads (App. F).  Head types
 * are an input (the trained HardKuma assignment of Sec. 3.2, thresholded).
 *
 * Conventions shared by every call
 *   - Pointers are DEVICE pointers unless a parameter says HOST.  The caller owns every
 *     buffer; the library neither frees nor keeps them after the call's stream-ordered
 *     work has finished.  Nothing is allocated inside a call (a context allocates, once, in
 *     lychee_create: a 4 MiB device arena with its pinned mirror, and about 14 MiB of flags and
 *     counters through which the workgroups of a layer launch hand results to one another).
 *   - Calls only enqueue work on `hip_stream` (a hipStream_t; NULL = the default stream) and
 *     never read device memory from the host.  The layer calls (lychee_decode_attn,
 *     lychee_decode_attn_static, lychee_decode_attn_deferred, lychee_select_flush,
 *     lychee_dense_decode_attn) and the layer-after-layer steps enqueue kernel launches only,
 *     one per layer (two for a layer call under a probability rule with more sets to select than a
 *     quarter of the launch's workgroups: the second selects where the sequences are short or of
 *     very unequal lengths, and else does nothing), and never wait.  The phased steps and the cache
 *     append keep their layer descriptors in the arena: they enqueue one small asynchronous
 *     host-to-device copy when the call's pointers differ from those of earlier calls, and once
 *     the arena has seen about 4 MiB of distinct tables such a call waits for the stream once and starts the arena over
 *     - unless a stream capture has seen the arena: a captured graph keeps pointing into it, so
 *     its tables are never recycled and the call returns LYCHEE_EARENA instead.
 *   - bf16 means the upper 16 bits of an IEEE fp32.  Scores and accumulation are fp32;
 *     `out` is rounded to nearest-even bf16.
 *   - KV-cache element (b, g, t, i), g a KV head, t a position, i < 128, lives at
 *         base + b*kv_stride_batch + g*kv_stride_head + t*kv_stride_tok + i   (elements).
 *     K and V use the same strides.  The preferred layout is [B][H_kv][L_cap][128] with
 *     256-byte aligned rows: each (b, g) is then one contiguous stream of 256-byte rows
 *     (two 128-byte lines), which is what the streaming kernel is tuned for.
 *   - Index sets are int32 [B][H_kv][k]: positions in [0, L_b), distinct, valid entries
 *     first, -1 padding after (when k > L_b).  Sets written by the library are ascending
 *     by position; ties in the score go to the lower position.  Entries of `idx_in` that
 *     are negative or >= L_b are ignored (never dereferenced).
 *   - Return value: 0, or a negative LYCHEE_E* code; on an error nothing was enqueued.
 *   - Results are deterministic: the same inputs give bit-identical outputs.
 *   - Two calls that share a workspace must be ordered on one stream.
 */
#ifndef LYCHEE_H
#define LYCHEE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LYCHEE_OK            0
#define LYCHEE_EINVAL       (-1)  /* a NULL / misaligned pointer or an inconsistent value       */
#define LYCHEE_EUNSUPPORTED (-2)  /* a valid request this build does not serve                 */
#define LYCHEE_EWORKSPACE   (-3)  /* workspace NULL, misaligned or smaller than required       */
#define LYCHEE_EHIP         (-4)  /* a HIP runtime call failed (no device, launch error, ...)  */
#define LYCHEE_EARENA       (-5)  /* the context's descriptor arena is full and cannot be recycled
                                     because a captured graph uses it: create another context   */

#define LYCHEE_HEAD_DIM      128  /* the only head dimension served                            */
#define LYCHEE_MAX_KV_HEADS   64
#define LYCHEE_MAX_GROUP       4  /* query heads per KV head served (1..4)                     */
#define LYCHEE_MAX_BATCH     256

typedef struct lychee_ctx lychee_ctx; /* opaque; holds the device id, tuning, a small device
                                         arena for descriptor tables and the hand-off flags of
                                         the layer launches; use one context per stream, and do
                                         not let two calls on one context overlap.  The attention
                                         calls only enqueue kernels (and at most one
                                         host-to-device copy of a descriptor table from the
                                         context's pinned memory), so a stream that is being
                                         captured into a HIP graph can take them, and the graph can be
                                         replayed while the context lives and timing is off. */

/* Problem shape of one layer call (the inputs of Alg. 1 that are not tensors). */
typedef struct lychee_shape {
    int32_t batch;       /* B in [1, LYCHEE_MAX_BATCH]                                       */
    int32_t n_q_heads;   /* H_q, a multiple of n_kv_heads with H_q / H_kv <= LYCHEE_MAX_GROUP */
    int32_t n_kv_heads;  /* H_kv in [1, LYCHEE_MAX_KV_HEADS]                                 */
    int32_t head_dim;    /* must be LYCHEE_HEAD_DIM                                          */
    int32_t max_len;     /* host-known upper bound of lengths[]; sizes grids and workspace,
                            so that no call has to read lengths[] on the host              */
    int32_t k;           /* token budget of Eq. 2 / Eq. 3, >= 1; the capacity of every set      */
    int64_t kv_stride_batch, kv_stride_head, kv_stride_tok; /* elements; each a multiple of 8
                            (16-byte vector loads), kv_stride_tok >= 128                    */
    int32_t keep_ppm;    /* 0: Eq. 2 selects min(k, L_b) positions.  1 .. 1000000: the Ratio rule
                            of Sec. 4.4.1, a budget proportional to the sequence length:
                            min(k, ceil(L_b * keep_ppm / 10^6)) positions, at least 1.  (The
                            paper's theta is the share of tokens dropped, App. E.2: theta = 70 %
                            is keep_ppm = 300000.)  Sparse heads attend over whatever valid
                            entries the inherited set holds, under either rule.               */
    int32_t block_size;  /* 0 or 1: sets name positions (Sec. 3.1).  64: the block-granular variant of
                            App. C / Sec. 4.3.2: a set entry e names the positions [64e, 64e+63]
                            below L_b, a block is ranked by the best pooled score inside it, and k,
                            idx_in / idx_out and the Ratio rule all count blocks.               */
    int32_t prob_rule;   /* 0: none.  LYCHEE_RULE_THRESHOLD (1), LYCHEE_RULE_TOP_P (2): the rules of
                            Sec. 4.4.1 on attention probabilities, here the softmax over the whole
                            sequence of the pooled selection logits (App. F's pooled query).
                            Threshold keeps the positions whose probability exceeds prob_param;
                            Top-p keeps the shortest prefix of the descending order whose
                            probabilities sum to at least prob_param.  Both keep at least the best
                            position and at most min(k, L_b) - the best ones, if the rule wants
                            more -, break ties like Eq. 2, and pad the set with -1.  Positions
                            only (block_size <= 1), and not together with keep_ppm.  Decisions are
                            taken in fp32: a position whose probability (cumulative probability)
                            lies within rounding of the parameter may fall on either side.     */
    float prob_param;    /* tau or p, in (0, 1]                                                  */
} lychee_shape;
#define LYCHEE_RULE_THRESHOLD 1
#define LYCHEE_RULE_TOP_P     2

/* Create / destroy a context bound to HIP device `device`.  Needs a GPU. */
int lychee_create(lychee_ctx **ctx, int device);
int lychee_destroy(lychee_ctx *ctx);

/* Pure host functions (no GPU needed).
 * lychee_check_shape: validates `shape`; if `head_type_mask` (HOST, [H_q]) is given it also
 *   checks that sparse heads come with an inherited set (`has_idx_in` != 0).
 * lychee_workspace_bytes: bytes of scratch any call below needs for `shape` (selection
 *   candidates and scores, split partials); 0 if the shape is invalid.  lychee_decode_step
 *   needs lychee_step_workspace_bytes (the same per layer).
 *   The workspace must be 256-byte aligned; its contents are don't-care on entry. */
int    lychee_check_shape(const lychee_shape *shape, const uint8_t *head_type_mask, int has_idx_in);
size_t lychee_workspace_bytes(const lychee_shape *shape);
size_t lychee_step_workspace_bytes(const lychee_shape *shape, int32_t n_layers); /* for lychee_decode_step */

/*
 * One layer of Alg. 1's per-head loop (retrieval branch: Eq. 1, Eq. 2, o = A V; sparse
 * branch: Eq. 3), for all sequences of a batch.
 *   q               bf16 [B][H_q][128], 16-byte aligned
 *   k_cache,v_cache bf16, strided as in `shape`, 16-byte aligned, read-only
 *   head_type_mask  HOST uint8 [H_q]: 1 = retrieval head, 0 = sparse head
 *   idx_in          int32 [B][H_kv][k], the sets inherited from the previous layer; may be
 *                   NULL only if every head is a retrieval head (the first layer)
 *   out             bf16 [B][H_q][128], 16-byte aligned
 *   idx_out         int32 [B][H_kv][k]: for a KV head whose group holds a retrieval head,
 *                   the min(k, L_b) positions with the highest mean retrieval logit; for any
 *                   other KV head a verbatim copy of idx_in.  Must not alias idx_in.
 *   lengths         int32 [B], 1 <= L_b <= max_len, the current token included (values
 *                   outside that range are clamped into it)
 * Errors: EINVAL (NULL / misaligned pointer, bad shape, sparse heads without idx_in,
 * idx_out == idx_in), EUNSUPPORTED (head_dim, group size; more than 2^31 blocks of 16 cache rows in
 * one launch, far beyond what fits a GPU), EWORKSPACE, EHIP.
 */
int lychee_decode_attn(lychee_ctx *ctx, const lychee_shape *shape, const void *q,
                       const void *k_cache, const void *v_cache, const uint8_t *head_type_mask,
                       const int32_t *idx_in, void *out, int32_t *idx_out, const int32_t *lengths,
                       void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * The same layer (Alg. 1's per-head loop), for a caller that runs layer after layer: in Alg. 1
 * the set S a retrieval head updates is read again only by the next layer's sparse heads, so
 * `out` does not have to wait for it.  This call enqueues everything that `out` needs and
 * leaves the selection (Eq. 2) of its layer PENDING; the next lychee_decode_attn_deferred call
 * on the same context runs the pending selection in its first launch, beside its own
 * preparations and before its sparse heads read their sets, and lychee_select_flush runs it
 * alone.  Arguments and errors as for lychee_decode_attn, except:
 *   workspace   lychee_step_workspace_bytes(shape, 2) bytes: the pending layer's selection
 *               candidates live in one half while the next layer fills the other
 *   idx_out     complete (in stream order) only after the call that runs the pending
 *               selection; nothing else may write it in between
 *   q           may be reused as soon as this call's work is done (the library keeps a copy of
 *               what a selection can still need)
 *   idx_in, k_cache, lengths (pointer AND contents), the workspace: unchanged until the
 *               pending selection has run.  In particular flush before the lengths grow for
 *               the next token, and before the workspace serves any other call.
 * While a selection is pending, the next deferred call must pass the same shape, lengths
 * pointer and workspace (else EINVAL: flush first), and every other call that is given that
 * workspace returns EINVAL.
 * Each such call is ONE kernel launch.  Inside it the pending selection runs on a few workgroups
 * of its own, the layer's sparse heads wait (with a bounded wait) until it has published the set
 * they read, and the workgroup that finishes a head's last piece merges the head's partials.
 * lychee_select_flush: enqueues a pending selection, if there is one (one small launch); EINVAL
 * for a NULL ctx.  A model that overlaps work on a second stream can flush there, off its
 * critical path, as long as the flush is ordered before the next layer's call.
 */
int lychee_decode_attn_deferred(lychee_ctx *ctx, const lychee_shape *shape, const void *q,
                                const void *k_cache, const void *v_cache, const uint8_t *head_type_mask,
                                const int32_t *idx_in, void *out, int32_t *idx_out, const int32_t *lengths,
                                void *workspace, size_t workspace_bytes, void *hip_stream);
int lychee_select_flush(lychee_ctx *ctx, void *hip_stream);

/*
 * lychee_decode_attn for callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): the same layer call without a workspace
 * argument.  Its scratch is an array of LYCHEE_STATIC_SCRATCH_BYTES bytes that is part of the
 * library's device code, so every GPU the library runs on holds it until the process ends; the
 * call allocates nothing, on the device or on the host.  Arguments, results and errors as for
 * lychee_decode_attn, and:
 *   EWORKSPACE    lychee_workspace_bytes(shape) exceeds LYCHEE_STATIC_SCRATCH_BYTES (the Qwen3-8B-shaped
 *                 128K layer at batch 1 needs about 22 MiB); nothing is enqueued
 *   EUNSUPPORTED  per-launch timing is enabled on the context (it creates events)
 * All calls on one GPU share the one array, whatever their context or stream, and it keeps the last
 * call's contents (which no call depends on): calls that overlap on a GPU race, so order them on one
 * stream or with events.
 */
#define LYCHEE_STATIC_SCRATCH_BYTES (32u << 20)
int lychee_decode_attn_static(lychee_ctx *ctx, const lychee_shape *shape, const void *q,
                              const void *k_cache, const void *v_cache, const uint8_t *head_type_mask,
                              const int32_t *idx_in, void *out, int32_t *idx_out, const int32_t *lengths,
                              void *hip_stream);

/* Dense decode attention on the same buffers: every head runs Eq. 1 and o = A V, nothing
 * is selected.  The in-run speed baseline; `shape->k` is ignored (any value >= 1). */
int lychee_dense_decode_attn(lychee_ctx *ctx, const lychee_shape *shape, const void *q,
                             const void *k_cache, const void *v_cache, void *out,
                             const int32_t *lengths, void *workspace, size_t workspace_bytes,
                             void *hip_stream);

/*
 * The attention of a whole decode step (Alg. 1, the layer loop restricted to its per-head
 * loop): layers 0 .. n_layers-1 in order, the sets written by layer l feeding layer l+1
 * (Sec. 3.1: the set is propagated to the next layer).  All layers share `shape` and
 * `lengths`.
 *   q, k_cache, v_cache, out   HOST arrays of n_layers device pointers
 *   head_type_masks            HOST uint8 [n_layers][H_q]
 *   idx_in                     sets entering layer 0, or NULL when layer 0 is all-retrieval
 *                              (Sec. 3.1: every head of the first layer is a retrieval head)
 *   idx_out                    the sets leaving the last layer; may be NULL
 *   workspace                  at least lychee_step_workspace_bytes(shape, n_layers) bytes
 * Because every layer's query is an input of the call, only the sparse heads of layer l+1
 * depend on layer l (through its sets).  STEP_MODE chooses how that is used:
 *   LYCHEE_STEP_PHASED (default)  five launches for the whole step: the selection
 *     thresholds of all layers, the retrieval streaming of all layers pooled in one launch,
 *     the selects, the sparse gathers of all layers, and the combines.  out[l] of every layer is complete only
 *     when the call's work has finished.
 *   LYCHEE_STEP_LAYERWISE  layer after layer, ONE launch per layer, each as
 *     lychee_decode_attn_deferred (layer l's selection runs inside layer l+1's launch, the last
 *     one alone); out[l] is complete before layer l+1 starts, as a model that computes q[l+1]
 *     from out[l] needs.
 * Fewer than 128 layers; PHASED falls back to LAYERWISE when n_layers * batch > 2048, and a
 * single layer always runs as lychee_decode_attn does.
 */
int lychee_decode_step(lychee_ctx *ctx, const lychee_shape *shape, int32_t n_layers,
                       const void *const *q, const void *const *k_cache,
                       const void *const *v_cache, const uint8_t *head_type_masks,
                       const int32_t *idx_in, void *const *out, int32_t *idx_out,
                       const int32_t *lengths, void *workspace, size_t workspace_bytes,
                       void *hip_stream);

/* Alg. 1, "C.append(k, v)": the decoded token's key and value rows
 *   k_new, v_new   bf16 [B][H_kv][128], 16-byte aligned
 * become row lengths[b] - 1 of every KV head of k_cache / v_cache (strided as in `shape`; lengths
 * count the token being decoded).  One small launch on the stream; needs no workspace. */
int lychee_append_kv(lychee_ctx *ctx, const lychee_shape *shape, const void *k_new,
                     const void *v_new, void *k_cache, void *v_cache, const int32_t *lengths,
                     void *hip_stream);

/* lychee_decode_step with each layer's cache append inside the call (Alg. 1: append, then
 * attend): k_new[l], v_new[l] (HOST arrays of n_layers device pointers, each bf16 [B][H_kv][128])
 * are written to row lengths[b] - 1 of layer l's caches before any of the step's attention
 * reads them.  In the phased step the appends ride in the first launch (the selection
 * thresholds, whose sample never touches the newest row), so they cost no launch of their own
 * (with block-granular sets, which need no thresholds, they are one small launch); layer after
 * layer, all layers' appends are one small launch in front of the first layer. */
int lychee_decode_step_append(lychee_ctx *ctx, const lychee_shape *shape, int32_t n_layers,
                              const void *const *q, const void *const *k_new,
                              const void *const *v_new, void *const *k_cache, void *const *v_cache,
                              const uint8_t *head_type_masks, const int32_t *idx_in,
                              void *const *out, int32_t *idx_out, const int32_t *lengths,
                              void *workspace, size_t workspace_bytes, void *hip_stream);

/* Dense attention for all layers of a step (Eq. 1 and o = A V for every head, no selection), in
 * the order STEP_MODE names: PHASED = all layers' streaming pooled in one launch, then the
 * combines; LAYERWISE = layer after layer as lychee_dense_decode_attn.  The in-run baseline of
 * lychee_decode_step; arguments as there, workspace of lychee_step_workspace_bytes. */
int lychee_dense_decode_step(lychee_ctx *ctx, const lychee_shape *shape, int32_t n_layers,
                             const void *const *q, const void *const *k_cache,
                             const void *const *v_cache, void *const *out, const int32_t *lengths,
                             void *workspace, size_t workspace_bytes, void *hip_stream);

/* ==========================================================================================
 * The paged 4-bit cache: a layer's keys and values in pages of a pool shared by all requests, 4 bits
 * a value, and the hybrid-head decode layer that runs on it (Eq. 1 to 3 of Alg. 1's per-head loop).  A
 * serving step is: lychee_release_pages (finished requests), lychee_plan_pages (pages and slots of
 * the step's new tokens), and per layer lychee_q4_append, lychee_q4_decode_attn and, where retrieval
 * heads choose sets for the next layer, lychee_select_scores.
 *
 *   - A page holds page_size tokens (16, 32, 64, 128 or 256) of every KV head, in tiles of 16 tokens
 *     of one head: tile i of head g of page p is number p*page_tiles + g*(page_size/16) + i, at
 *     cache + number*LYCHEE_Q4_TILE_BYTES.  page_tiles, the tiles from one page to the next, is at
 *     least n_kv_heads*page_size/16 (more where the pages of several layers lie interleaved).
 *   - A tile is 16 rows of 128 bytes, then 128 bytes of scales.  A row is a token's key (64 bytes)
 *     and value (64 bytes): dimension 2j in the low, 2j+1 in the high half of byte j.  The scales are
 *     [8][16] bytes: dimensions 0-31, 32-63, 64-95, 96-127 of the key, then of the value; 16 tokens.
 *   - 4 bits are a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (the e2m1 format that gfx950 converts);
 *     the value is that times 2^(scale byte - 127), and NaN under a scale byte of 255.
 *   - Writing a group of 32 values takes the smallest e in [-125, 125] with max |x| <= 6 * 2^e and
 *     rounds x / 2^e to the nearest of these values, ties to the even code (what lies beyond 6 * 2^125
 *     becomes 6 * 2^125); a group that holds a NaN or an infinity gets the scale byte 255.
 *   - A slot names a token's place in a layer's cache: page * page_size + place in the page.
 *   - block_table is int32 [batch][table_stride]: entry t / page_size of a request's row is the page
 *     of its token t.  Entries outside [0, n_pages) are never followed: tokens there are not
 *     written, and attention leaves them out.  Several requests may share a page that none writes.
 *   - lengths is int32 [batch], tokens a request holds: values outside [0, max_pages * page_size] are
 *     clamped into it, except by lychee_plan_pages, which refuses them.  A request of length 0 is
 *     legal everywhere: its outputs are zero.
 *   - bf16 operands need 16-byte alignment, int32 and float ones 4-byte, the cache 128-byte.
 *   - Each call enqueues one kernel launch (none where there is nothing to do), may be captured, and
 *     leaves the caller's current device as it was.  Launches of these calls are not timed by
 *     lychee_timing_enable.  What else the conventions above say holds here too.
 * ========================================================================================== */
#define LYCHEE_Q4_TILE_BYTES 2176
#define LYCHEE_Q4_MAX_GROUP    16  /* query heads per KV head served by lychee_q4_decode_attn (1..16) */

typedef struct lychee_paged {
    int32_t batch;        /* requests, in [1, LYCHEE_MAX_BATCH]                                   */
    int32_t n_q_heads;    /* a multiple of n_kv_heads                                            */
    int32_t n_kv_heads;   /* in [1, LYCHEE_MAX_KV_HEADS]                                         */
    int32_t head_dim;     /* must be LYCHEE_HEAD_DIM                                             */
    int32_t n_pages;      /* pages of the pool; n_pages * page_size < 2^31                       */
    int32_t page_size;    /* 16, 32, 64, 128 or 256                                              */
    int32_t max_pages;    /* pages a request can hold; max_pages * page_size <= 2^24             */
    int32_t table_stride; /* entries from one row of the block table to the next, >= max_pages   */
    int32_t page_tiles;   /* tiles from one page to the next, >= n_kv_heads * page_size / 16     */
    int32_t k;            /* entries of an index set, >= 1                                       */
} lychee_paged;

/* Pure host functions.  lychee_check_paged: validates `paged` and, if `head_type_mask` (HOST, [H_q]) is
 * given, that sparse heads come with a set.  lychee_paged_workspace_bytes: scratch of
 * lychee_q4_decode_attn (256-byte aligned, contents don't care); 0 if `paged` is invalid. */
int    lychee_check_paged(const lychee_paged *paged, const uint8_t *head_type_mask, int has_idx_in);
size_t lychee_paged_workspace_bytes(const lychee_paged *paged);

/* Gives the pages of finished requests back to the pool.  The free pages are a stack: entries
 * free_pages[0 .. *free_count-1], taken and given at its end.
 *   done           uint8 [B]: not 0 = the request's pages go back, in order of the request and of its
 *                  table, and its length becomes 0.  The table's entries go back as they are, whoever
 *                  else holds them: a page shared with another request is the caller's to take out of the
 *                  table (an entry outside [0, n_pages) that comes back into a table is no page there)
 *   lengths, lengths_out         int32 [B]; may be one array
 *   free_pages     int32 [n_pages]; pages that do not fit any more (given back twice) are dropped
 *   free_count, free_count_out   int32 [1]; may be one word
 * The block table is only read. */
int lychee_release_pages(lychee_ctx *ctx, const lychee_paged *paged, const uint8_t *done, const int32_t *lengths,
                         const int32_t *block_table, int32_t *free_pages, const int32_t *free_count,
                         int32_t *lengths_out, int32_t *free_count_out, void *hip_stream);

/* Block table, slots and lengths of a step in which request b gets new_tokens[b] >= 0 more tokens (free_pages and free_count:
 * the stack of lychee_release_pages).
 *   block_table    entries of the pages taken are written: requests in order take pages off the end of
 *                  free_pages; other entries are left as they are
 *   lengths_out    lengths[b] + new_tokens[b]; may be `lengths`.  free_count_out may be `free_count`
 *   slots          int32 [n_slots]: the slots of the new tokens, request after request, then -1
 *                  (-1 also for a token whose table entry is no page)
 *   token_start    int32 [B + 1]: where each request's tokens begin in `slots`; the last is their number
 *   status         int32 [1]: 0, or why nothing was planned: the number of pages missing; -1: a length or
 *                  count is negative or makes a request longer than max_pages hold, or *free_count is
 *                  not in [0, n_pages]; -2: more new tokens than n_slots.  Then lengths_out and
 *                  free_count_out repeat the inputs, the table is unchanged, `slots` is all -1 and
 *                  `token_start` all 0. */
int lychee_plan_pages(lychee_ctx *ctx, const lychee_paged *paged, const int32_t *lengths, const int32_t *new_tokens,
                      int32_t *block_table, const int32_t *free_pages, const int32_t *free_count,
                      int32_t *lengths_out, int32_t *free_count_out, int32_t *slots, int32_t n_slots,
                      int32_t *token_start, int32_t *status, void *hip_stream);

/* Writes tokens into a layer's cache.
 *   k_new, v_new   bf16, element (i, g, d) of token i at base + i*stride_tok + g*stride_head + d; the
 *                  strides are in elements, multiples of 8, both operands share them
 *   slots          int32 [n_tokens]; a token whose slot is outside [0, n_pages * page_size) is not
 *                  written.  No slot may occur twice in a call
 * EUNSUPPORTED for more than about 2^28 tokens times KV heads in a call. */
int lychee_q4_append(lychee_ctx *ctx, const lychee_paged *paged, const void *k_new, const void *v_new,
                     int64_t stride_tok, int64_t stride_head, const int32_t *slots, int32_t n_tokens, void *cache,
                     void *hip_stream);

/* Reads tokens back as bf16 rows (exactly the values the cache stands for), for example into a cache of the
 * calls above: token t of request b, first[b] <= t < last[b], becomes row t - first[b].
 *   first          int32 [B], or NULL for 0; last int32 [B]; clamped like lengths
 *   k_out, v_out   bf16, element (b, g, row, d) at base + b*stride_batch + g*stride_head + row*stride_tok + d
 *                  (elements, multiples of 8, stride_tok >= 128); rows beyond n_rows and behind a request's
 *                  last token are left as they were, a row whose token has no page is zero */
int lychee_q4_read(lychee_ctx *ctx, const lychee_paged *paged, const void *cache, const int32_t *block_table,
                   const int32_t *first, const int32_t *last, void *k_out, void *v_out, int64_t stride_batch,
                   int64_t stride_head, int64_t stride_tok, int32_t n_rows, void *hip_stream);

/* One layer of Alg. 1's per-head loop on the 4-bit cache, one query token a request.
 *   q, out          bf16 [B][H_q][128]
 *   head_type_mask  HOST uint8 [H_q]: 1 = retrieval head (Eq. 1 over t < L_b), 0 = sparse head (Eq. 3 over its KV
 *                   head's set); NULL: every head is a retrieval head
 *   idx_in          int32 [B][H_kv][k], sets as in the conventions; may be NULL if there is no sparse head.  Of a
 *                   set the first min(k, L_b) entries are read; those negative or >= L_b are ignored
 *   scores          NULL, or float, row (b, g) at scores + (b*H_kv + g)*score_stride: the mean logit of the
 *                   group's retrieval heads at every t < L_b (-infinity where the token has no page).  Rows of
 *                   KV heads without a retrieval head, and what lies behind L_b, are left as they were.
 *                   score_stride >= max_pages * page_size
 * A head with nothing to attend to (L_b = 0, an empty set, no page) gives zeros.  Scores and sums are
 * fp32; the softmax weights multiply V as the sum of two bf16 numbers (about 2^-17 of a weight).
 * Errors: EUNSUPPORTED for a group of more than LYCHEE_Q4_MAX_GROUP, or more than 2^30 blocks of work. */
int lychee_q4_decode_attn(lychee_ctx *ctx, const lychee_paged *paged, const void *q, const void *cache,
                          const int32_t *block_table, const int32_t *lengths, const uint8_t *head_type_mask,
                          const int32_t *idx_in, void *out, float *scores, int64_t score_stride, void *workspace,
                          size_t workspace_bytes, void *hip_stream);

/* Eq. 2 on rows of scores: idx_out [B][H_kv][k] gets, for a KV head whose group holds a retrieval head, the
 * min(k, L_b) positions t < L_b with the highest scores[(b*H_kv + g)*score_stride + t], ties to the lower
 * position, ascending, -1 behind them; for any other KV head a verbatim copy of idx_in.  NaN ranks like
 * -infinity, -0 like 0.  head_type_mask as above (NULL: every KV head selects; then idx_in may be NULL); idx_out
 * must not be idx_in; score_stride >= max_pages * page_size. */
int lychee_select_scores(lychee_ctx *ctx, const lychee_paged *paged, const float *scores, int64_t score_stride,
                         const int32_t *lengths, const uint8_t *head_type_mask, const int32_t *idx_in,
                         int32_t *idx_out, void *hip_stream);

/* ==========================================================================================
 * Attention over whole prompts: several query tokens a request, each attending to the positions up to its own
 * (Eq. 1 with a causal mask, every head dense: what fills the caches that the decode calls read, rewrites the last
 * tokens of a long generation, and, with its gradient, trains head types on full attention).
 *
 *   - Query tokens are packed: those of request b are rows token_start[b] .. token_start[b+1]-1 of q and out, as
 *     lychee_plan_pages numbers them.  token_start is int32 [batch + 1], in ascending order; values are clamped to
 *     [0, n_tokens].  A request may have no tokens.  Rows that belong to no request are left as they were.
 *   - Its keys are L_b in number, and its n_b query tokens are the last n_b of them: query i sits at position
 *     p = L_b - n_b + i and attends to the positions 0 .. p.  A query with p < 0 (or, in pages, no page to attend to) has
 *     nothing to attend to: its output is zero, its lse -infinity.  One whose scores are all -infinity has output NaN,
 *     lse -infinity.
 *   - Query head h uses KV head h / (n_q_heads / n_kv_heads), up to LYCHEE_PROMPT_MAX_GROUP query heads a KV head.
 *   - What a query does not see has no influence on its results, infinities and NaN included.
 *     An infinite value or NaN that it does see reaches its output whatever its weight, one that rounds to zero included: the
 *     output is infinite there, or NaN where it sees a NaN or infinities of both signs.
 *   - Softmax statistics and sums are fp32; weights, and dS in the backward pass, are rounded to bf16 for the matrix units, and
 *     the backward pass has out as it was rounded.  out and dv are 0.0017 to 0.0024 of their norm off, dq and dk 0.0024 to
 *     0.0031 (most where sequences are short), where their own rounding makes 0.0017.  (lychee_q4_decode_attn keeps weights to
 *     2^-17: a single token has the more exact output there.)
 *   - A forward call enqueues one or two kernel launches, a backward call two to four (none for n_tokens = 0).  Calls may be
 *     captured and leave the caller's current device as it was; their launches are not timed by lychee_timing_enable.
 *     Results do not depend on the order in which workgroups run: the same call gives the same bits.
 *   - What a call writes must not overlap what it reads, nor the rest of what it writes (views that share rows of a fused
 *     projection do not overlap).  The same address for an output and another argument is refused: EINVAL.
 *   - The workspace is scratch (256-byte aligned, contents don't care).  One that is large enough for a call is large enough
 *     for every call with the same heads and no more requests, tokens and max_len.  Calls that run at the same time need one each.
 * ========================================================================================== */
#define LYCHEE_PROMPT_MAX_GROUP 16

typedef struct lychee_prompt {
    int32_t batch;        /* requests, in [1, LYCHEE_MAX_BATCH]                                   */
    int32_t n_q_heads;    /* a multiple of n_kv_heads                                            */
    int32_t n_kv_heads;   /* in [1, LYCHEE_MAX_KV_HEADS]                                         */
    int32_t head_dim;     /* must be LYCHEE_HEAD_DIM                                             */
    int32_t n_tokens;     /* packed rows; n_tokens * n_q_heads / n_kv_heads < 2^28                */
    int32_t max_len;      /* upper bound of lengths[] (keys in a cache), <= 2^24; lengths are clamped to it */
    int64_t q_stride_tok, q_stride_head; /* of q and dq: element (i, h, d) at base + i*stride_tok + h*stride_head + d */
    int64_t kv_stride_batch, kv_stride_head, kv_stride_tok; /* of k, v, dk and dv; elements, multiples of 8 as those
                             of q; those of tokens in [128, 2^24], of query heads <= 2^24.  kv_stride_batch counts where
                             `lengths` are given                                                    */
} lychee_prompt;

/* Pure host functions.  lychee_prompt_workspace_bytes serves both calls below; 0 if `prompt` is invalid. */
int    lychee_check_prompt(const lychee_prompt *prompt);
size_t lychee_prompt_workspace_bytes(const lychee_prompt *prompt);

/* out = softmax(q K^T / sqrt(128)) V under the causal mask.
 *   q              bf16, strided, 16-byte aligned (as k, v and out)
 *   k, v           lengths NULL: packed like q, (i, g, d) at base + i*kv_stride_tok + g*kv_stride_head + d, L_b = n_b.
 *                  Else a cache as the decode calls have it, (b, g, t, d) at base + b*kv_stride_batch +
 *                  g*kv_stride_head + t*kv_stride_tok + d, that holds the new tokens' rows already
 *   lengths        NULL, or int32 [B]: L_b, clamped to [0, max_len]
 *   out            bf16 [n_tokens][H_q][128]
 *   lse            NULL, or float [H_q][n_tokens]: log of the sum of exp of a row's scores */
int lychee_prompt_attn(lychee_ctx *ctx, const lychee_prompt *prompt, const void *q, const void *k, const void *v,
                       const int32_t *token_start, const int32_t *lengths, void *out, float *lse, void *workspace,
                       size_t workspace_bytes, void *hip_stream);

/* Its gradient for packed sequences: d_out and out bf16 [n_tokens][H_q][128], out and lse as the call above wrote them; dq
 * strided like q, dk and dv like k and v, summed over the query heads of a KV head.  No two rows (of a token and a head)
 * may have an element in common: EINVAL.  Gradients are written, not added to; rows of no request are left as they were. */
int lychee_prompt_attn_backward(lychee_ctx *ctx, const lychee_prompt *prompt, const void *d_out, const void *q,
                                const void *k, const void *v, const void *out, const float *lse,
                                const int32_t *token_start, void *dq, void *dk, void *dv, void *workspace,
                                size_t workspace_bytes, void *hip_stream);

/* The same attention over the paged 4-bit cache, for the pieces of prompts (and single tokens) that lychee_plan_pages
 * gave slots to and lychee_q4_append has written: lengths as after the step (lengths_out), token_start as planned.
 * Tokens whose table entry is no page are left out.  q strided like above, out bf16 [n_tokens][H_q][128].
 * lychee_q4_prompt_workspace_bytes is 0 for sizes that the call refuses. */
size_t lychee_q4_prompt_workspace_bytes(const lychee_paged *paged, int32_t n_tokens);
int lychee_q4_prompt_attn(lychee_ctx *ctx, const lychee_paged *paged, const void *q, int64_t q_stride_tok,
                          int64_t q_stride_head, int32_t n_tokens, const void *cache, const int32_t *block_table,
                          const int32_t *lengths, const int32_t *token_start, void *out, void *workspace,
                          size_t workspace_bytes, void *hip_stream);

const char *lychee_strerror(int code);

/* ==========================================================================================
 * Tuning and diagnostics.  Nothing below is needed to run the path; results never depend on any
 * of it beyond the fp32 rounding order of the split merge (index sets do not depend on it at all),
 * except on WAIT_POLLS in calls with a pending selection (see there).
 * ========================================================================================== */

/* Options of a context.
 *   DEFAULTS      puts every option back to its default (value ignored)
 *   WG_PER_CU     workgroups per compute unit in every launch (1..3, default 2)
 *   N_WG          workgroups per launch, overriding WG_PER_CU (0 = CUs x WG_PER_CU; at most 768)
 *   STEP_MODE     how lychee_decode_step orders its work (see there)
 *   TAIL_PERMILLE permille of a phased launch's streaming / gather rows that workgroups claim
 *                 dynamically, in small chunks, after their fixed share (0..1000, default 250;
 *                 launches too short to hold several chunks per workgroup use none); it levels out
 *                 compute units that stream at different speeds
 *   GATHER_BLOCK  set entries whose gather is balanced against 64 streamed rows (a multiple
 *                 of 16 in [16, 128]; the default is 64, and 48 for deferred calls and
 *                 layer-after-layer steps of long sequences or many rows in all)
 *   SELECT_MARGIN tenths of a standard deviation by which the sampled selection threshold is
 *                 lowered below its estimate of the k-th score (-10000..100000, default 60).
 *                 A larger margin makes more rows candidates of the exact select; a margin so
 *                 small that fewer than k rows pass, or so large that the candidate list
 *                 overflows, costs time (the row is then ranked from all of its scores) but
 *                 never changes a result
 *   SELECT_LEAD   layer launches: blocks of 64 rows the device streams while a pending select
 *                 runs (default 3000); the gathers that wait for that select get workgroups for
 *                 the work that is left by then
 *   WAIT_POLLS    polls of a flag after which a wait inside a layer launch gives up (0 .. 1048576, the
 *                 default: seconds).  Fewer are for tests of what a launch does then (see
 *                 lychee_wait_timeouts) */
#define LYCHEE_OPT_DEFAULTS     0
#define LYCHEE_OPT_WG_PER_CU    1
#define LYCHEE_OPT_STEP_MODE    2
#define LYCHEE_OPT_GATHER_BLOCK 6
#define LYCHEE_OPT_N_WG         7
#define LYCHEE_OPT_TAIL_PERMILLE 8
#define LYCHEE_OPT_SELECT_MARGIN 9
#define LYCHEE_OPT_SELECT_LEAD  10
#define LYCHEE_OPT_WAIT_POLLS   11
#define LYCHEE_STEP_PHASED      1
#define LYCHEE_STEP_LAYERWISE   0
int lychee_set_option(lychee_ctx *ctx, int32_t option, int32_t value);

/* Debug helper (synchronous): counts entries of idx [B][H_kv][k] that break the index
 * conventions (out of [0, L_b), duplicated, or valid after a -1) into *n_bad (HOST).  The one call
 * of the library that allocates (and frees) device memory, 8 bytes: not for a captured stream. */
int lychee_validate_idx(lychee_ctx *ctx, const lychee_shape *shape, const int32_t *idx,
                        const int32_t *lengths, int64_t *n_bad, void *hip_stream);

/* Debug helper (synchronous): how many score rows, since the context was created, the select had
 * to rank from all of their scores because the sampled threshold let fewer than the budget
 * through (*too_few) or more than the candidate list holds (*too_many).  Both cost time, never
 * correctness; on smooth score distributions both stay 0. */
int lychee_select_stats(lychee_ctx *ctx, int64_t *too_few, int64_t *too_many, void *hip_stream);

/* Debug helper (synchronous): how many bounded waits inside layer launches have given up since the
 * context was created (a piece waiting for its row's threshold, a gather waiting for its set, a
 * workgroup at the end of the grid waiting for the row it selects).
 * It stays 0 unless the device cannot keep a launch's workgroups resident together.  A piece that
 * gives up on a threshold costs time only (its row is ranked whole, and counted as too_many above),
 * and so does a workgroup that gives up on its row (the piece that completes the row selects it); a
 * gather that gives up on a set reads the set as it is. */
int lychee_wait_timeouts(lychee_ctx *ctx, int64_t *timeouts, void *hip_stream);

/* Per-launch timing with HIP events on the caller's stream.  While enabled, every launch of
 * the library's kernels but those of the paged 4-bit cache is bracketed by an event pair.  lychee_timing_read waits for the
 * recorded events, adds up the milliseconds and launches per launch class since the last
 * read and clears the record (arrays of LYCHEE_N_KERNEL_CLASSES entries). */
#define LYCHEE_KERNEL_STREAM  0   /* retrieval streaming of a phased step; a layer launch       */
#define LYCHEE_KERNEL_GATHER  1   /* sparse gather only                                     */
#define LYCHEE_KERNEL_THRESHOLD 2 /* selection thresholds                                   */
#define LYCHEE_KERNEL_SELECT  3   /* select / set copies only                               */
#define LYCHEE_KERNEL_COMBINE 4   /* combine (alone, with select or with set copies)        */
#define LYCHEE_N_KERNEL_CLASSES 5
int lychee_timing_enable(lychee_ctx *ctx, int on);
int lychee_timing_read(lychee_ctx *ctx, float *ms_per_class, int32_t *launches_per_class);

/* Plain streaming kernels used to calibrate the measurements: a read of `bytes` bytes
 * (sum folded into *sink, 4 bytes) and a copy of `bytes` bytes.  16-byte aligned, bytes a
 * multiple of 16. */
int lychee_probe_read(lychee_ctx *ctx, const void *src, size_t bytes, void *sink, void *hip_stream);
int lychee_probe_copy(lychee_ctx *ctx, void *dst, const void *src, size_t bytes, void *hip_stream);



#ifdef __cplusplus
}
#endif
#endif /* LYCHEE_H */
