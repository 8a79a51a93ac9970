/*
 * liblast: GB300 (sm_103a) kernels for LAST's edge-side token selection
 * ("The Last Query Token Guides Visual Token Pruning ...", Sec. 3.2-3.4).
 *
 * The path, per request b of a ragged batch:
 *   1. last_scores  Eq. 6-8: the attention row of the last query position
 *                   p* = P_b - 1 (a full softmax over all P_b keys, visual and
 *                   text, including p* itself) is summed over every layer and
 *                   q-head at the visual positions and normalised over the
 *                   visual span: w~_i = s_i / sum_j s_j.
 *   2. last_select  Eq. 9-11: importance-weighted greedy k-center selection
 *                   under cosine distance on the encoder features X, budget k_b.
 *   3. last_gather  Eq. 12: the kept rows of X in ascending index order.
 *   last_prune runs 1-3 back to back on one stream.
 *
 * Variants the paper evaluates beside the method:
 *   last_select_topk  Table 5: keep the k_b highest scores (no diversity term).
 *   last_scores_rows  Table 4: scores from the attention rows of several query
 *                     positions (First, Middle, All Mean) instead of p* alone.
 * The key-value cache of the models around the path (last section of this file; the
 * paper has no counterpart): last_rope rotates q and K by positions on several axes,
 * as last_scores wants them; last_cache_append also writes K and V into a paged
 * cache; last_cache_compact cuts a cache to the kept tokens; last_cache_attention
 * decodes over it; last_cache_copy and last_pages_* part and free its pages.
 * Deployment aids without a counterpart in the paper: last_prune_host (the
 * whole path on host buffers, copies included), last_scores_noalloc (scoring
 * without a caller workspace) and last_check_bounded_wait (exercises the
 * reporting of an expired device wait).
 *
 * Conventions shared by every entry point
 *   - All tensors are DEVICE pointers (caller-allocated, e.g. torch tensors),
 *     except those of last_prune_host; the library allocates no device memory.  Scratch
 *     lives in a caller workspace (256-byte aligned), sized by last_workspace_size().
 *   - The offset arrays in last_problem are HOST arrays; each call validates
 *     them and copies a small plan into the workspace on `stream`.
 *   - Calls are asynchronous on `stream` (a cudaStream_t; NULL = legacy
 *     default stream).  Successive calls on one stream may reuse one
 *     workspace; concurrent calls need distinct workspaces.
 *   - No entry point but those of the key-value cache may be captured into a
 *     CUDA graph: each call copies its plan from pageable host memory that it owns and releases on return, so
 *     a captured copy would replay freed memory.  Launch-bound callers batch
 *     requests into one call instead (one launch per kernel for the batch).
 *   - Argument errors are detected on the host before any launch; the call
 *     returns a status and touches no output.  Device-side checks set a flag in
 *     the workspace that last_poll() reports: an out-of-range caller index
 *     (last_gather) or an expired bounded wait (every device wait has an
 *     iteration limit, so no call can hang the GPU).
 *   - The selection is deterministic and, given the same w~, bit-identical to
 *     the canonical fp32 arithmetic below on every run:
 *       dot(a,b): lane l in 0..31 owns coordinate groups g = l, l+32, l+64, ...
 *                 of 8 consecutive coordinates; it accumulates them in
 *                 increasing coordinate order with one fp32 fma each; the 32
 *                 lane sums are combined by an xor butterfly (offsets 16..1).
 *       r_i = dot(x_i,x_i) > 0 ? 1/sqrt(dot(x_i,x_i)) : 0  (IEEE div, sqrt)
 *       delta_i = min(delta_i, 1 - (dot(x_i,x_j) * r_i) * r_j),  p_i = w~_i * delta_i
 *       argmax ties go to the lowest index; selected tokens are excluded.
 *
 * Layouts (row-major, no padding)
 *   q      [batch][num_layers][num_q_heads][head_dim]      query of p* per layer
 *   k      [num_layers][cu_seqlens[batch]][num_kv_heads][head_dim]   packed keys
 *   x      [cu_vis[batch]][feat_dim]                       encoder features
 *   w      [cu_vis[batch]] fp32                            w~ (Eq. 8)
 *   idx    [cu_keep[batch]] int32, request-local, ascending per request
 *   x_out  [cu_keep[batch]][feat_dim], same dtype as x
 *   q-head h reads kv-head h / (num_q_heads / num_kv_heads).
 *
 * Limits (LAST_ERR_UNSUPPORTED beyond them; last_error_message() says which):
 *   scoring   G = num_q_heads / num_kv_heads in 1..8; head_dim * elem_bytes a
 *             multiple of 16; num_q_heads * head_dim fp32 values of q plus one
 *             chunk of logits within 100 KB of shared memory (e.g. up to 128
 *             q-heads of 128); num_layers * num_q_heads <= 6144.
 *   selection feat_dim a multiple of 8, at most 2048; the greedy selection
 *             (last_select, last_prune) keeps per-token state of a request in
 *             the shared memory of up to 16 clustered CTAs: about 120K tokens
 *             at feat_dim 64, 72K at bf16 feat_dim 2048, 13K at fp32 feat_dim
 *             2048.  A call of at most 4 requests past that bound runs them on
 *             every SM of the GPU instead (per-token state spread over all
 *             CTAs: millions of tokens); a call of more requests returns
 *             LAST_ERR_UNSUPPORTED for them.  Top-k and the gather have no
 *             such bound.
 */
#ifndef LAST_H_
#define LAST_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  LAST_OK = 0,
  LAST_ERR_INVALID_ARG = 1,          /* shape/offset/pointer check failed (host) */
  LAST_ERR_UNSUPPORTED = 2,          /* valid but outside the compiled limits */
  LAST_ERR_WORKSPACE_TOO_SMALL = 3,  /* ws_bytes below what the call needs at least */
  LAST_ERR_CUDA = 4,                 /* a CUDA runtime call failed */
  LAST_ERR_DEVICE_INDEX = 5,         /* last_poll: a caller index was out of range */
  LAST_ERR_TIMEOUT = 6,              /* last_poll: a bounded device wait expired; outputs invalid */
  LAST_ERR_NO_PAGES = 7              /* last_pages_take: fewer pages are free than asked for */
} last_status;

typedef enum { LAST_DTYPE_F32 = 0, LAST_DTYPE_BF16 = 1 } last_dtype;

/* Problem description (Eq. 2, Eq. 5-7).  Request b has P_b = cu_seqlens[b+1] -
 * cu_seqlens[b] positions whose last one is the query token p*; its N_b =
 * cu_vis[b+1] - cu_vis[b] visual tokens occupy positions vis_start[b] ..
 * vis_start[b] + N_b - 1 (which must end before p*); it keeps
 * k_b = cu_keep[b+1] - cu_keep[b] tokens, 0 <= k_b <= N_b (Eq. 2; see
 * last_budget).  All four arrays are host memory, read during the call only. */
typedef struct {
  int32_t batch;
  int32_t num_layers;      /* L: layers whose rows are summed (Eq. 7) */
  int32_t num_q_heads;     /* H in Eq. 7 */
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t feat_dim;        /* d_v in Eq. 1 */
  int32_t dtype;           /* last_dtype of q, k and x */
  float softmax_scale;     /* <= 0 selects 1/sqrt(head_dim) */
  const int32_t *cu_seqlens; /* [batch+1], cu_seqlens[0] == 0, non-decreasing */
  const int32_t *vis_start;  /* [batch] */
  const int32_t *cu_vis;     /* [batch+1] */
  const int32_t *cu_keep;    /* [batch+1] */
} last_problem;

/* Bytes of device workspace with which the entry points below run `p` fastest, except
 * last_scores_rows and last_prune_host, which are sized by
 * last_scores_rows_workspace_size and last_host_workspace_size.
 * Returns LAST_ERR_INVALID_ARG / LAST_ERR_UNSUPPORTED for a bad problem.
 *
 * Most of it may be room for the selection's Gram matrices: 4 N_b^2 bytes per request
 * with 1 < k_b < N_b, up to 12 GiB a call (8 requests of 16384 tokens: 8.6 GB), where
 * a matrix makes the selection faster.  last_select, last_prune and
 * last_prune_host also take less: without room for the matrices they read the
 * features in every round, with the same results, three to four times slower
 * on such batches.  What a call needs at least grows with its problem, and the size
 * reported for the same problem with cu_keep = cu_vis (no token to choose, so no
 * matrix) is always enough, whatever the budgets; so is that of a problem with
 * more requests, tokens or keys for one with fewer (see last_scores and
 * last_select_topk for callers that do not select).  LAST_ERR_WORKSPACE_TOO_SMALL
 * names the least size in last_error_message(). */
last_status last_workspace_size(const last_problem *p, size_t *bytes);

/* Eq. 6-8.  w_out [cu_vis[batch]] fp32 receives w~ (sums to 1 per request).  The size
 * reported with cu_keep all zero is enough (the budgets are not used). */
last_status last_scores(const last_problem *p, const void *q, const void *k, float *w_out,
                        void *ws, size_t ws_bytes, void *stream);

/* Eq. 9-12.  w [cu_vis[batch]] fp32, not negative (e.g. from last_scores); idx_out
 * [cu_keep[batch]] receives sort(S_K) per request, request-local.  When x_out
 * is not NULL the kept rows are also written there (the fused form of
 * last_gather). */
last_status last_select(const last_problem *p, const float *w, const void *x,
                        int32_t *idx_out, void *x_out, void *ws, size_t ws_bytes,
                        void *stream);

/* Table 5, "LAST (Top-k)": the selection variant without the diversity term.
 * idx_out [cu_keep[batch]] receives, per request and in ascending order, the
 * k_b indices of highest w~ (ties between equal scores go to the lower index;
 * -0 equals +0).  When x_out is not NULL the kept rows of x are also written
 * there (x is then required; feat_dim a positive multiple of 8); x may be NULL
 * otherwise.  The problem's layer/head fields are not used.  Uses no matrix: like for
 * last_gather, the size reported with cu_keep = cu_vis is enough.  Same ownership,
 * stream and error rules as last_select.  w must hold no NaN: the kept set is
 * then unspecified (but still k_b distinct valid indices). */
last_status last_select_topk(const last_problem *p, const float *w, const void *x,
                             int32_t *idx_out, void *x_out, void *ws, size_t ws_bytes,
                             void *stream);

/* Table 4 (attention sources: First, Middle, All Mean): Eq. 6-8 with the
 * attention rows of several query positions per request instead of p* alone.
 * Request b's query rows are cu_rows[b] .. cu_rows[b+1]-1 (HOST array, length
 * batch+1, cu_rows[0] = 0, at least one row per request); row r sits at the
 * request-local position row_pos[r] (HOST array), which must lie after the visual
 * span: vis_start[b] + N_b <= row_pos[r] <= P_b - 1; row r's softmax runs over the
 * keys 0 .. row_pos[r] (causal).  q_rows [cu_rows[batch]][num_layers][num_q_heads]
 * [head_dim] holds one query vector per row, layer and q-head; k as for
 * last_scores.  w_out [cu_vis[batch]] receives the visual probabilities summed
 * over rows, layers and q-heads and normalised per request (a mean over the rows
 * gives the same w~).  With one row per request (First, Middle, Last) the row
 * at position pos is the last-row computation on keys 0 .. pos, and the call
 * runs last_scores' kernels on the requests cut there (when G <= 8).
 * Limits: bf16 only; head_dim 64, 128, 192 or 256; rows x
 * (num_q_heads / num_kv_heads) <= 256 and rows x layers x q-heads <= 6144 per
 * request.  The workspace is sized by last_scores_rows_workspace_size. */
last_status last_scores_rows_workspace_size(const last_problem *p, const int32_t *cu_rows,
                                            const int32_t *row_pos, size_t *bytes);
last_status last_scores_rows(const last_problem *p, const int32_t *cu_rows,
                             const int32_t *row_pos, const void *q_rows, const void *k,
                             float *w_out, void *ws, size_t ws_bytes, void *stream);

/* Eq. 12.  x_out[r] = x[cu_vis[b] + idx[r]] for r in request b's output range.
 * An index outside [0, N_b) leaves its row unwritten and makes last_poll
 * return LAST_ERR_DEVICE_INDEX.  Any feat_dim that is a positive multiple of 8
 * is accepted (the selection's own feat_dim <= 2048 limit does not apply); the
 * workspace carries the plan and the device error word. */
last_status last_gather(const last_problem *p, const void *x, const int32_t *idx,
                        void *x_out, void *ws, size_t ws_bytes, void *stream);

/* The whole path: scores, selection, ordered gather.  w_out may be NULL (w~
 * is then kept in the workspace); x_out may be NULL (indices only). */
last_status last_prune(const last_problem *p, const void *q, const void *k, const void *x,
                       float *w_out, int32_t *idx_out, void *x_out,
                       void *ws, size_t ws_bytes, void *stream);

/* last_prune on HOST buffers: q, k and x are read from host memory and idx_out,
 * x_out (may be NULL) and w_out (may be NULL) are written to host memory, with
 * the layouts above.  The call enqueues on `stream` the host-to-device copies of
 * q, K and X into the device workspace, the whole path, and the device-to-host
 * copies of the results, and returns; the host buffers must stay valid and
 * unchanged until the stream has passed the call.  Pinned (page-locked) host
 * memory keeps every copy asynchronous, so a caller alternating two workspaces
 * on two streams overlaps one call's copies with another's kernels; pageable
 * memory works but the copies then block the host.  The device workspace holds
 * the plan and device copies of q, K, X, w~, the indices and the kept rows:
 * last_host_workspace_size() bytes, 256-byte aligned, or less when that holds Gram
 * matrices (see last_workspace_size). */
last_status last_host_workspace_size(const last_problem *p, size_t *bytes);
last_status last_prune_host(const last_problem *p, const void *q_host, const void *k_host,
                            const void *x_host, float *w_out_host, int32_t *idx_out_host,
                            void *x_out_host, void *ws, size_t ws_bytes, void *stream);

/* last_scores without a caller workspace (the paper has no counterpart: this is
 * a deployment aid).  For callers that cannot allocate device memory at run time
 * -- e.g. an edge service that reserves all of its device memory at start-up and
 * treats later allocations as failures, or a program without a device allocator
 * of its own.  Same inputs, outputs and results as last_scores; the scratch lives
 * in a fixed 16 MiB array inside the library, held on every GPU that loads the
 * library until the process exits.  Each call looks up that array's device
 * address (cudaGetSymbolAddress, cached per device after the first call) with
 * the device current; like every entry point it cannot be captured into a CUDA
 * graph (the plan is copied from host memory the call releases).  All calls share
 * the array and it keeps the last call's contents: calls whose executions
 * overlap on the GPU race on it.  A problem needing more than 16 MiB of scratch
 * (last_workspace_size with cu_keep all zero) returns LAST_ERR_UNSUPPORTED.
 * Allocates nothing. */
last_status last_scores_noalloc(const last_problem *p, const void *q, const void *k,
                                float *w_out, void *stream);

/* Diagnostic (no counterpart in the paper): runs one device-side bounded wait that
 * nothing completes, with a short iteration limit, so that the next last_poll on
 * `ws` (at least 256 bytes) returns LAST_ERR_TIMEOUT.  It exercises the path every
 * device wait of the library takes when a wait expires, without hanging or
 * faulting the GPU. */
last_status last_check_bounded_wait(void *ws, void *stream);

/* ---- rotary positions and the key-value cache ----
 *
 * What a model around the path needs beside it: rotary positions before last_scores,
 * and a paged cache of K and V after it.  These calls read lengths, page tables and
 * positions on the DEVICE and copy nothing from host memory, so that they may be
 * captured into a CUDA graph and replayed while lengths and tables change in place.
 * dtype (last_dtype) is that of q, K, V and the outputs; sums and rotations are
 * formed in fp32 and rounded once.  What cannot be checked on the host (a page, an
 * index or a length out of range) is checked on the device: it is skipped, and
 * last_poll on the call's workspace returns LAST_ERR_DEVICE_INDEX.  What a call writes
 * may overlap nothing else that it reads or writes unless its comment says so. */

/* Rotary positions on several axes (time, height, width; one axis for text): token t's
 * pair i < rot_dim / 2 turns by positions[axis[i]][t] * inv_freq[i].  Elements past
 * rot_dim are copied.  The arrays are HOST memory, read during the call only. */
typedef enum {
  LAST_ROPE_HALF = 0,        /* pair i: elements i and i + rot_dim / 2 */
  LAST_ROPE_ADJACENT = 1     /* pair i: elements 2i and 2i + 1 */
} last_rope_pairs;
typedef struct {
  int32_t rot_dim;           /* even, 2 .. head_dim */
  int32_t num_axes;          /* 1 .. 4 */
  int32_t pairs;             /* last_rope_pairs */
  const float *inv_freq;     /* [rot_dim / 2], 0 <= f <= 65536 */
  const int32_t *axis;       /* [rot_dim / 2], each in 0 .. num_axes - 1; NULL: all on axis 0 */
} last_rotary;

/* Heads of a token tensor [num_tokens][heads][head_dim]: strides in elements, head_dim
 * contiguous.  out may be in, with the same strides; else it may overlap nothing that the call
 * reads or writes.  Heads of `in` may overlap (one token for all, say), heads of `out` may not. */
typedef struct {
  const void *in;
  void *out;
  int32_t heads;
  int64_t in_token, in_head;
  int64_t out_token, out_head;
} last_heads;

/* Rotates q and, unless NULL, k.  positions: int32 [num_axes][axis_stride >= num_tokens],
 * any value (angles are formed modulo one turn in 64-bit integers, so that long
 * positions lose nothing).  Any strides and alignment of whole elements; head_dim 2 .. 256, num_tokens
 * at most 2^30.
 * last_rope_backward turns by the opposite angles: with the gradient with respect to the
 * rotated heads as `in`, `out` receives the gradient with respect to the heads. */
last_status last_rope(const last_rotary *r, int32_t dtype, int32_t num_tokens, int32_t head_dim,
                      const int32_t *positions, int64_t axis_stride, const last_heads *q,
                      const last_heads *k, void *stream);
last_status last_rope_backward(const last_rotary *r, int32_t dtype, int32_t num_tokens,
                               int32_t head_dim, const int32_t *positions, int64_t axis_stride,
                               const last_heads *q, const last_heads *k, void *stream);

/* A paged cache: K and V of num_layers layers in num_pages pages of page_size tokens.
 * Element (layer, page, head, token, c) of either lies at layer * layer_stride +
 * page * page_stride + head * head_stride + token * token_stride + c (strides in elements,
 * each a multiple of 16 bytes; k and v 16-byte aligned).  page_size a multiple of 8, at most
 * 2^20; head_dim * elem_bytes a multiple of 16, head_dim <= 256; at most 4096 layers and
 * kv-heads, and a page of one layer and a token's K of all layers below 2^31 bytes each.  In a
 * cache that a call writes no two elements may share an address, whether of K or V; only layers
 * may be one (layer_stride 0). */
typedef struct {
  void *k, *v;
  int32_t num_layers, num_pages, page_size, num_kv_heads, head_dim;
  int32_t dtype;
  int64_t layer_stride, page_stride, head_stride, token_stride;
} last_cache;

/* Sequences of a cache, all DEVICE int32: token i of sequence b lies in page
 * page_table[b * table_stride + i / page_size], slot i % page_size; lens[b] tokens are held. */
typedef struct {
  int32_t batch;
  int32_t max_pages;         /* entries of a page table row */
  int64_t table_stride;
  const int32_t *page_table;
  const int32_t *lens;
  const int32_t *key_begin;  /* first key that last_cache_attention reads; NULL: 0 */
} last_sequences;

/* Bytes of device workspace (256-byte aligned) for the calls below with up to `batch`
 * sequences and num_q_heads query heads.  Its contents need no initialisation. */
last_status last_cache_workspace_size(const last_cache *c, int32_t batch, int32_t num_q_heads,
                                      size_t *bytes);

/* Writes new tokens behind the sequences' cached ones, in one layer.  Sequence b's new tokens are
 * cu_new[b] .. cu_new[b+1]-1 (DEVICE int32 [batch+1], cu_new[batch] = num_tokens; NULL: one
 * token per sequence) and s->lens[b] counts them already: the last one goes to slot
 * lens[b] - 1.  With r, the tokens' K (and q, unless NULL) are rotated on the way as in
 * last_rope and q's heads written to q->out; without r, K is copied and q must be NULL.
 * The out fields of k and v are not used. */
last_status last_cache_append(const last_cache *c, int32_t layer, const last_sequences *s,
                              int32_t num_tokens, const int32_t *cu_new, const last_rotary *r,
                              const int32_t *positions, int64_t axis_stride, const last_heads *q,
                              const last_heads *k, const last_heads *v, void *ws,
                              size_t ws_bytes, void *stream);

/* Attention of one new token per sequence over its cached keys key_begin[b] .. lens[b]-1, in
 * one layer: out = sum_p softmax_p(scale q.k_p) v_p for every q-head, lse (may be NULL) [batch]
 * [num_q_heads] fp32 = log sum_p exp(scale q.k_p).  A sequence without such a key gets out = 0
 * and lse = -inf, and so does one whose logits are all -inf; a key of logit -inf has weight 0.
 * Slots outside the range are never used, whatever they hold, and pages wholly outside it are
 * not read (their table entries may be anything).  Keys of a page out of range are left out, as
 * if they were not cached; a sequence is taken for one without a key where lens[b] is negative or
 * more than its table row has room for, or key_begin[b] is negative.  q-head h reads kv-head h / (num_q_heads / num_kv_heads).  q and out:
 * [batch][num_q_heads][head_dim], sequences q_stride and out_stride elements apart, both multiples
 * of 16 bytes, 16-byte aligned.  scale <= 0 selects 1/sqrt(head_dim).  Results do not depend on
 * other calls or on timing: repeated calls give the same bits.  batch * num_q_heads *
 * (max_pages * page_size / 32 + 1) must stay below 2^31 (LAST_ERR_UNSUPPORTED). */
last_status last_cache_attention(const last_cache *c, int32_t layer, const last_sequences *s,
                                 int32_t num_q_heads, float scale, const void *q, int64_t q_stride,
                                 void *out, int64_t out_stride, float *lse, void *ws,
                                 size_t ws_bytes, void *stream);

/* Copies page src[i] to page dst[i], i < num_copies (DEVICE int32), in every layer, K and V.  No
 * page may be written twice, nor written and read, by one call; src[i] == dst[i] does nothing. */
last_status last_cache_copy(const last_cache *c, int32_t num_copies, const int32_t *src,
                            const int32_t *dst, void *ws, size_t ws_bytes, void *stream);

/* The pruning applied to a cache (Eq. 12 on K and V): sequence b keeps its tokens before
 * span_begin[b], of the span_len[b] tokens after that the span-local ones idx[cu_keep[b]] ..
 * idx[cu_keep[b+1]-1] (as last_select writes them), and all tokens behind the span; they are
 * copied, in that order and in every layer, to the front of the pages that row b of dst_table
 * ([batch][dst_max_pages], rows dst_stride apart) names, and lens_out[b] receives their number.
 * All arrays are DEVICE int32; span_begin and span_len NULL: the whole sequence is the span.
 * num_idx is the length of idx.  Pages that are written may not be read for another token in the
 * same call, but a page may stand in both tables where its tokens keep their slots (those before
 * the first dropped one): a token that would be copied onto itself is left alone.  A
 * sequence whose span, cu_keep or dst_table cannot hold is skipped, lens_out[b] included;
 * so is a single token whose idx or page is out of range.  lens_out may not overlap any array that
 * the call reads. */
last_status last_cache_compact(const last_cache *c, const last_sequences *s,
                               const int32_t *dst_table, int32_t dst_max_pages,
                               int64_t dst_stride, const int32_t *span_begin,
                               const int32_t *span_len, const int32_t *cu_keep,
                               const int32_t *idx, int32_t num_idx, int32_t *lens_out, void *ws,
                               size_t ws_bytes, void *stream);

/* Who holds which page, on the HOST: holders [num_pages] counts the sequences that hold a page (0: free)
 * and free_pages [num_pages] is a stack of the num_free free ones; both arrays belong to the caller.
 * last_pages_init frees every page.  last_pages_take hands out n free pages (one holder each) or,
 * with fewer free, none: LAST_ERR_NO_PAGES.  last_pages_share adds a holder to each page of a list
 * (a fork), last_pages_release takes one away and frees what nobody holds.  A page that is out of
 * range or free makes either return LAST_ERR_INVALID_ARG, with nothing changed. */
typedef struct {
  int32_t num_pages;
  int32_t num_free;
  int32_t *holders;
  int32_t *free_pages;
} last_page_pool;
last_status last_pages_init(last_page_pool *p);
last_status last_pages_take(last_page_pool *p, int32_t n, int32_t *pages);
last_status last_pages_share(last_page_pool *p, int32_t n, const int32_t *pages);
last_status last_pages_release(last_page_pool *p, int32_t n, const int32_t *pages);

/* Synchronises `stream`, then reports the device-side flags of the last call
 * that used `ws`: LAST_OK, LAST_ERR_DEVICE_INDEX, or LAST_ERR_TIMEOUT (a wait
 * on an asynchronous copy gave up after its iteration limit instead of hanging;
 * the outputs of that call are then invalid). */
last_status last_poll(const void *ws, void *stream);

/* Eq. 2: k = ceil(num * n_vis / den) in exact integer arithmetic
 * (rho = num/den); -1 for n_vis < 0, num < 0 or den <= 0. */
int32_t last_budget(int32_t n_vis, int32_t num, int32_t den);

const char *last_status_string(last_status s);

/* Human-readable detail of the last non-OK status returned on this thread. */
const char *last_error_message(void);

#ifdef __cplusplus
}
#endif

#endif /* LAST_H_ */
