/*
 * pillar.h -- C ABI of the PillarAttn hot path on MI355X (gfx950).
 *
 * One round of PillarAttn (paper Section 4.1) for one transformer layer:
 *
 *   pillar_verify_attn    full attention of the k+1 speculative query
 *                         positions over each request's whole paged KV-Cache,
 *                         which also emits the per-token attention-score
 *                         statistic of the verification step;
 *   pillar_select_topk    Top-K of that statistic per (request, KV head): the
 *                         critical tokens of the next k draft steps;
 *   pillar_sparse_decode  draft attention that loads only the selected rows
 *                         (paged attention at page size 1, Section 4.2).
 * and beside it, for the same cache: trees of drafted tokens, a cache that holds
 * no more than a budget, and new tokens (rotary positions, the write into the
 * cache, attention of prompts, what the logits say).
 *
 * Conventions shared by every entry point
 *   - Every pointer inside pillar_kv_t and every tensor argument is a DEVICE
 *     pointer owned by the caller; the pillar_kv_t struct itself lives on the
 *     host.  The library never allocates, frees or synchronises: all work is
 *     enqueued on `hip_stream` (a hipStream_t, NULL = the default stream) and
 *     the call returns at once.  Scratch memory comes in through `workspace`
 *     (device, 256-byte aligned, at least pillar_workspace_bytes() bytes); its
 *     contents are meaningless between calls and calls sharing one workspace
 *     must be ordered on one stream.  Calls can be captured into a HIP graph;
 *     make one ordinary call with the same shapes first (the first launch of
 *     a kernel may set a function attribute, which is not a stream operation).
 *   - Return value: PILLAR_OK or a negative pillar_status.  Argument errors
 *     are detected on the host before anything is launched, so a failed call
 *     has no effect on the device.  Page ids and token indices stored in
 *     device memory cannot be checked on the host: values outside their
 *     documented ranges are undefined behaviour.
 *   - Outputs are bit-identical from run to run for identical inputs.
 *   - Tensors are dense C-order arrays unless a stride argument is given.
 *   - bf16 is the upper half of an IEEE float32; fp8 is OCP e4m3 (bias 7,
 *     largest finite 448, no infinities), dequantised as code * scale with
 *     one fp32 scale per (page, KV head) for K and one for V.
 *
 * Supported shapes: head_dim 64 or 128; num_q_heads a multiple of
 * num_kv_heads with group size G <= 16; page_size a power of two in 1..256;
 * 0 <= spec_len_k <= 15 and (spec_len_k+1)*G <= 64.  Anything else returns
 * PILLAR_EUNSUPPORTED.
 */
#ifndef PILLAR_H_
#define PILLAR_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  PILLAR_OK = 0,
  PILLAR_EINVAL = -1,        /* NULL pointer, non-positive size, inconsistent shapes */
  PILLAR_EUNSUPPORTED = -2,  /* well-formed but outside the supported shapes/dtypes */
  PILLAR_EWORKSPACE = -3,    /* workspace NULL, misaligned or too small */
  PILLAR_EHIP = -4,          /* the HIP runtime refused a launch */
  PILLAR_ETOOLARGE = -5      /* pillar_sparse_decode_static only: needs more than its fixed scratch */
} pillar_status;

typedef enum { PILLAR_F32 = 0, PILLAR_BF16 = 1, PILLAR_FP8_E4M3 = 2 } pillar_dtype;

/* The paged KV-Cache of one layer and the requests that read it.
 * Token t of request b is row  block_table[b*block_table_stride + t/page_size]
 * (a page id), slot t % page_size; its K vector for KV head g starts at element
 *   page*stride_page + g*stride_head + slot*stride_slot
 * of k_pool (same for v_pool) and is head_dim contiguous elements.
 * seq_lens[b] counts every token whose K/V is already in the pool, including
 * the k+1 speculative tokens of a verification step. */
typedef struct {
  int32_t batch;               /* B  >= 1 */
  int32_t num_q_heads;         /* Hq */
  int32_t num_kv_heads;        /* Hkv, divides Hq */
  int32_t head_dim;            /* D  */
  int32_t page_size;           /* P  */
  int32_t q_dtype;             /* PILLAR_F32 | PILLAR_BF16: type of q and of out */
  int32_t kv_dtype;            /* PILLAR_F32 | PILLAR_BF16 | PILLAR_FP8_E4M3 */
  float   sm_scale;            /* logit scale, normally 1/sqrt(D) */
  const void* k_pool;          /* device */
  const void* v_pool;          /* device */
  int64_t stride_page;         /* element strides; stride_slot >= head_dim */
  int64_t stride_head;
  int64_t stride_slot;
  const float* k_scale;        /* device [num_pages][Hkv], fp8 only, else NULL */
  const float* v_scale;
  int32_t num_pages;
  int32_t block_table_stride;  /* row length of block_table, in entries */
  const int32_t* block_table;  /* device [B][block_table_stride] */
  const int32_t* seq_lens;     /* device [B], 1 <= seq_lens[b] <= max_seq_len */
  int32_t max_seq_len;         /* host-known bound, <= block_table_stride*page_size.
                                * Kernels and grids are chosen by it (and by
                                * max_budget below), lengths being known on the
                                * device only: any bound is correct, a close one
                                * is faster */
  int32_t flags;               /* 0 or an OR of pillar_flag values; unknown bits: PILLAR_EINVAL */
} pillar_kv_t;

/* Per-call choices, carried in pillar_kv_t.flags.
 *   PILLAR_FLAG_EXACT_SCORES     the verification reads K twice (once for the
 *       log-sum-exp of every row, once more with V) and builds the score
 *       statistic from fp32 probabilities, instead of reading K once and
 *       rebuilding the statistic from 16-bit stashed exponentials.  Slower
 *       (about 1.15x); scores then carry fp32 rounding only.
 *   PILLAR_FLAG_GENERIC_KERNELS  every stage runs its plain vector-ALU kernel
 *       even where a matrix-core kernel exists: a second implementation to
 *       cross-check the fast one against.  Much slower. */
typedef enum { PILLAR_FLAG_EXACT_SCORES = 1, PILLAR_FLAG_GENERIC_KERNELS = 2 } pillar_flag;

/* Library version, major*10000 + minor*100 + patch. */
int pillar_version(void);

/* Static, NUL-terminated description of a status code. */
const char* pillar_status_string(int status);

/* Bytes of workspace that any of the three stage calls below may need for
 * this cache description, speculative length and largest budget.  Returns 0
 * when the description is invalid.  Host-only arithmetic. */
size_t pillar_workspace_bytes(const pillar_kv_t* kv, int32_t spec_len_k, int32_t max_budget);

/* Verification attention (Section 4.1, "Overhead-free identification").
 *   q      [B][k+1][Hq][D] q_dtype; row i is the query at position
 *          seq_lens[b]-(k+1)+i and attends to tokens 0..that position.
 *   out    [B][k+1][Hq][D] q_dtype: softmax(sm_scale * q K^T) V.
 *   lse    [B][k+1][Hq] fp32 natural-log-sum-exp of the logits, or NULL.
 *   scores [B][Hkv][score_stride] fp32, or NULL to skip the statistic:
 *          scores[b][g][t] = mean over the (k+1)*G rows of KV head g of the
 *          softmax probability that row assigns to token t (0 where the
 *          causal mask hides t).  Entries t >= seq_lens[b] are not written.
 *          score_stride >= max_seq_len.  Accuracy on the matrix-core path
 *          (bf16 queries): |error| <= 4.9e-4 * score + 2^-62, because every
 *          row's exponential is kept to 11 significant bits and a probability
 *          below 2^-62 (2.2e-19) counts as 0 or as
 *          something below 2^-62; with PILLAR_FLAG_EXACT_SCORES
 *          the error is that of fp32 arithmetic.
 *   Every request must hold its own speculative tokens: seq_lens[b] >= k+1.
 *   A query row that sees no token at all (seq_lens[b] < k+1, down to 0) gets
 *   out = 0 and lse = -inf and adds nothing to the statistic. */
int pillar_verify_attn(const pillar_kv_t* kv, const void* q, int32_t spec_len_k,
                       void* out, float* lse, float* scores, int64_t score_stride,
                       void* workspace, size_t workspace_bytes, void* hip_stream);

/* pillar_verify_attn and pillar_select_topk in one call: the critical tokens
 * are selected from the score statistic while it is still on the chip, so it
 * makes no round trip through memory between two launches.  Arguments as in
 * the two calls; `scores` may be NULL when the caller does not want the
 * statistic itself.  Results are identical to the two calls made in turn.
 * The workspace needs pillar_workspace_bytes() bytes as for every call. */
int pillar_verify_select(const pillar_kv_t* kv, const void* q, int32_t spec_len_k,
                         void* out, float* lse, float* scores, int64_t score_stride,
                         const int32_t* budgets, int32_t max_budget,
                         int32_t* indices, int32_t* counts,
                         void* workspace, size_t workspace_bytes, void* hip_stream);

/* Verification of requests that speculate different numbers of tokens
 * (Section 5.4: heterogeneous request configurations).  spec_lens: device [B],
 * 0 <= spec_lens[b] <= spec_len_max.  Request b has spec_lens[b]+1 queries, the
 * first of its spec_len_max+1 slots in q / out / lse, query i at position
 * seq_lens[b]-(spec_lens[b]+1)+i; its statistic is the mean over
 * (spec_lens[b]+1)*G rows; out and lse of the unused slots are not written.
 * With budgets / indices / counts non-NULL the critical tokens are selected as
 * by pillar_verify_select (all three NULL and max_budget 0: no selection).
 * Served by the matrix-core kernels only: bf16 queries, bf16 or fp8 KV,
 * head_dim 128, pages of >= 16 tokens, slots less than 2^32 / 3 (bf16) or
 * 2^32 / 7 (fp8) bytes apart, neither flag set; anything else returns
 * PILLAR_EUNSUPPORTED.  seq_lens[b] >= spec_lens[b]+1 as above. */
int pillar_verify_hetero(const pillar_kv_t* kv, const void* q, int32_t spec_len_max,
                         const int32_t* spec_lens, void* out, float* lse, float* scores,
                         int64_t score_stride, const int32_t* budgets, int32_t max_budget,
                         int32_t* indices, int32_t* counts,
                         void* workspace, size_t workspace_bytes, void* hip_stream);

/* Critical-token selection (Section 4.1: Top-K on the averaged scores).
 *   scores   as written by pillar_verify_attn (all >= 0).
 *   budgets  device [B]: sparsity budget K of each request (>= 0).
 *   indices  device [B][Hkv][max_budget] int32: for each (b, g) the
 *            K' = min(budgets[b], seq_lens[b], max_budget) positions of
 *            largest score among 0..seq_lens[b]-1, equal scores resolved
 *            towards the lower position, stored in ascending position order
 *            and padded with -1.
 *   counts   device [B] int32: K' of each request. */
int pillar_select_topk(const float* scores, int64_t score_stride, const int32_t* seq_lens,
                       const int32_t* budgets, int32_t batch, int32_t num_kv_heads,
                       int32_t max_seq_len, int32_t max_budget,
                       int32_t* indices, int32_t* counts,
                       void* workspace, size_t workspace_bytes, void* hip_stream);

/* Sparse draft attention (Sections 1 and 4.2): one query row per request
 * attends to the listed rows only, no mask.
 *   q        [B][Hq][D] q_dtype.
 *   indices  device [B][Hkv][max_budget] int32 token positions in
 *            0..seq_lens[b]-1, any order; counts device [B], the first
 *            counts[b] entries of every head's list are used
 *            (0 <= counts[b] <= max_budget).
 *   out      [B][Hq][D] q_dtype (zeros where counts[b] == 0).
 *   lse      [B][Hq] fp32 or NULL (-inf where counts[b] == 0). */
int pillar_sparse_decode(const pillar_kv_t* kv, const void* q, const int32_t* indices,
                         const int32_t* counts, int32_t max_budget, void* out, float* lse,
                         void* workspace, size_t workspace_bytes, void* hip_stream);

/* One iteration of a unified batch (Section 4.2: "Unified Batch Scheduler" and
 * "Fused Sparse and Full Attention"): in the same iteration the requests listed
 * in verify_ids are in their verification phase and those in draft_ids in a
 * draft phase.  Per request the results are those of pillar_verify_select
 * (verify_ids) or pillar_sparse_decode (draft_ids) for that request alone:
 *   verify_ids  device [n_verify], draft_ids device [n_draft]: request indices
 *               in 0..batch-1, no request in both, none twice; the counts are
 *               host values (the scheduler that forms the batch knows them).
 *   q_verify / out_verify / lse_verify / scores, q_draft / out_draft / lse_draft,
 *   budgets / indices / counts: the full-batch tensors of the two calls, indexed
 *               by request id.  Only the rows of listed requests are read or
 *               written: a verifying request gets new out / lse / scores rows
 *               and a new index list and count; a drafting request reads its
 *               current list and gets out_draft / lse_draft rows.
 * Both phases run in ONE grid: the workgroups of the streaming verification
 * pass and those of the draft step are dispatched to their code path on the
 * chip.  (A draft sum may be grouped differently than by pillar_sparse_decode:
 * the results agree to rounding, not necessarily bit for bit, when a KV head
 * has more than 32 query rows.)  Either list may be empty.  Matrix-core shapes only (bf16 queries, bf16 or fp8 KV, head_dim
 * 128, pages of >= 16 tokens, slots as close as pillar_verify_hetero takes them,
 * rows of up to 32768 tokens, flags 0); anything
 * else returns PILLAR_EUNSUPPORTED.  Workspace: pillar_workspace_bytes(). */
int pillar_mixed_step(const pillar_kv_t* kv, const int32_t* verify_ids, int32_t n_verify,
                      const int32_t* draft_ids, int32_t n_draft,
                      const void* q_verify, int32_t spec_len_k, void* out_verify, float* lse_verify,
                      float* scores, int64_t score_stride,
                      const int32_t* budgets, int32_t max_budget, int32_t* indices, int32_t* counts,
                      const void* q_draft, void* out_draft, float* lse_draft,
                      void* workspace, size_t workspace_bytes, void* hip_stream);

/* pillar_sparse_decode for callers that can hand over no workspace and must
 * not cause an allocation: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same arguments, same kernels and the same
 * result bits as pillar_sparse_decode, but the partial results of index lists
 * longer than one workgroup's span of 512 rows go to a 32 MiB array inside the
 * library (one copy per GPU, held until the process ends) instead of a
 * workspace.  A shape whose pillar_sparse_decode would need more than those
 * 32 MiB (batch * Hkv * ceil(max_budget / 512) spans of G rows of 128 floats;
 * about 15000 spans at G = 4; lists of up to 512 rows need none) returns
 * PILLAR_ETOOLARGE and launches nothing.
 * Calls no allocator.  All calls on one GPU share the one array: two such
 * calls that overlap in time on the same GPU (different streams) race; order
 * them.  The first call on a device looks the array's address up; make it
 * outside any stream capture. */
int pillar_sparse_decode_static(const pillar_kv_t* kv, const void* q, const int32_t* indices,
                                const int32_t* counts, int32_t max_budget, void* out, float* lse,
                                void* hip_stream);

/* The write that precedes a verification: the K/V rows of the n_new newest
 * tokens of every request go into their pages (append, then attend:
 * seq_lens already counts them).  k_new, v_new: device [B][n_new][Hkv][D] in
 * kv_dtype; row i of request b is written at position seq_lens[b]-n_new+i
 * (rows whose position would be negative are skipped).  WRITES into the pools
 * that pillar_kv_t describes.  bf16 and fp32 pools only: an fp8 pool returns
 * PILLAR_EUNSUPPORTED (its page scales would have to be recomputed). */
int pillar_append_kv(const pillar_kv_t* kv, const void* k_new, const void* v_new,
                     int32_t n_new, void* hip_stream);

/* Index lists from other sources for pillar_sparse_decode (Section 4.2: at
 * page size 1 any token set is a list).
 *
 * pillar_window_indices: the static "attention sinks + recent window" pattern
 * of the sliding-window drafts the paper compares against (Sections 1, 3.3
 * and 5.2).  For
 * request b, K' = min(budgets[b], seq_lens[b], max_budget); every head's list
 * holds the first min(sink_tokens, K') positions and the last K' minus that
 * many, ascending, padded with -1; counts[b] = K'.  All arrays on the device,
 * layouts as in pillar_select_topk.
 *
 * pillar_extend_indices: tokens generated since the last verification have no
 * score yet but must be visible to a draft step: appends the positions
 * first_new[b] .. first_new[b]+n_new[b]-1 to every head's list of request b
 * (as many as fit below max_budget) and adds that number to counts[b]. */
int pillar_window_indices(const int32_t* seq_lens, const int32_t* budgets, int32_t batch,
                          int32_t num_kv_heads, int32_t sink_tokens, int32_t max_budget,
                          int32_t* indices, int32_t* counts, void* hip_stream);
int pillar_extend_indices(int32_t* indices, int32_t* counts, const int32_t* first_new,
                          const int32_t* n_new, int32_t batch, int32_t num_kv_heads,
                          int32_t max_budget, void* hip_stream);

/* ---- Trees of drafted tokens ------------------------------------------
 *
 * A draft that branches proposes a tree: several continuations are verified at
 * once and the longest accepted path is kept.  The nodes are the last
 * tree_sizes[b] tokens of a request (append, then attend: seq_lens[b] counts
 * them, node i is token seq_lens[b] - tree_sizes[b] + i).
 *
 * pillar_verify_tree: attention of every node.
 *   max_nodes  N, 1..64: slots per request in q, visible, out and lse.
 *   tree_sizes device [B], 0 <= tree_sizes[b] <= N, or NULL: N each.
 *   q          [B][N][Hq][D] q_dtype; node i is the i-th slot.
 *   visible    device [B][N] uint64: bit j of visible[b][i] says whether node i
 *              attends to node j (normally its ancestors and itself; any set of
 *              nodes will do, and bits from tree_sizes[b] on are ignored).  Every
 *              node attends to all tokens before the tree.  A chain is
 *              visible[b][i] = 2^(i+1) - 1, plain decoding N = 1 and a word of 1.
 *              (With the statistic, K is read twice here: chains of up to about 40 rows
 *              per KV head, and single tokens, are faster through pillar_verify_attn,
 *              whose scores have 11 bits.)
 *   out, lse, scores, score_stride: as in pillar_verify_attn, the statistic being
 *              the mean over the tree_sizes[b]*G rows; no part of out may be q
 *              (PILLAR_EINVAL).  Slots from tree_sizes[b] on and scores from
 *              seq_lens[b] on are not written, nor is anything of a request without
 *              nodes.  A node that sees no token gets out = 0 and lse = -inf and adds
 *              nothing to the statistic.  What a node does not see has no influence
 *              on it, whatever the cache holds there (infinities and NaN included).
 * Every shape that pillar_kv_t can describe, page sizes of 1 on, group sizes up
 * to 16, with up to 1024 rows per KV head.  bf16 queries with a bf16 or fp8 cache
 * run on bf16 matrix instructions (P is rounded to bf16), if q, out, the pools and
 * their strides are multiples of 16 bytes; everything else, and with
 * PILLAR_FLAG_GENERIC_KERNELS everything, on fp32 ones.  lse and scores carry
 * fp32 rounding only.  fp8 scales of what is seen are finite and not negative; on bf16
 * instructions a v_scale below 2^-80 counts as that, and what lse lacks, if anything,
 * are probabilities below 2^-46 times the largest v_scale that the row sees.
 * PILLAR_FLAG_EXACT_SCORES changes nothing here.
 * workspace: pillar_tree_workspace_bytes() (0: invalid arguments), enough for any
 * smaller batch, max_seq_len and N too.
 *
 * pillar_tree_commit: the accepted path becomes the end of the context.
 *   path       device [B][max_path] int32 (max_path 1..64), path_lens device [B]:
 *              with first = seq_lens[b] - tree_sizes[b], the K and V rows of tokens
 *              first + path[b][i], i < path_lens[b], move to tokens first + i, all
 *              read before any is written: nodes may be named in any order, and
 *              more than once.  A path ends at the first entry outside
 *              0..tree_sizes[b]-1; a request whose tree is not all in the cache
 *              (first < 0) commits nothing.
 *   scores     the statistic of the verification, or NULL: its entries move along.
 *   new_lens   device [B] int32, receives first + the length of the path; no part of
 *              it may be kv->seq_lens, tree_sizes, path or path_lens (PILLAR_EINVAL).
 * WRITES into the pools and, for fp8, into k_scale and v_scale: a page that
 * receives rows gets the largest scale that any of its rows up to the new length
 * had, and those rows are rounded anew to codes of that scale (at most half a
 * step of e4m3; where the scales are equal the bytes stay).  No page that holds a
 * node may belong to two requests.  Pools and strides in multiples of 16 bytes, else
 * PILLAR_EUNSUPPORTED. */
size_t pillar_tree_workspace_bytes(const pillar_kv_t* kv, int32_t max_nodes);
int pillar_verify_tree(const pillar_kv_t* kv, const void* q, int32_t max_nodes,
                       const int32_t* tree_sizes, const uint64_t* visible,
                       void* out, float* lse, float* scores, int64_t score_stride,
                       void* workspace, size_t workspace_bytes, void* hip_stream);
int pillar_tree_commit(const pillar_kv_t* kv, const int32_t* tree_sizes, int32_t max_nodes,
                       const int32_t* path, const int32_t* path_lens, int32_t max_path,
                       int32_t* new_lens, float* scores, int64_t score_stride, void* hip_stream);

/* ---- A cache that holds no more than a budget --------------------------
 *
 * pillar_evict_kv accumulates the statistic of every verification into a weight
 * per (request, KV head, cached token) and evicts the tokens that the budget does
 * not hold; each KV head keeps a set of its own.  For request b, with
 * L = seq_lens[b] and o = old_lens[b] (tokens the last call left, 0 at first;
 * those from o on are new):
 *   weights    device [B][Hkv][state_stride] fp32, in and out:
 *              w[t] <- decay * w[t] + scores[t] for t < o, scores[t] for o <= t < L.
 *              scores NULL: the weights of old tokens stay, new ones get 0.
 *              (A verification leaves the scores of a request without nodes as
 *              they were: clear them where there may be one.)
 *   positions  device [B][Hkv][state_stride] int32, in and out: the place of each
 *              cached token in the text.  New tokens are numbered on from the
 *              largest number that the head still holds (from 0 where there is
 *              none), which is their place as long as the newest token has never
 *              been evicted: recent_tokens >= 1 and budgets of sink_tokens +
 *              recent_tokens or more see to that.  Where it may go, numbers would
 *              be given twice; there the caller writes the positions of the new
 *              tokens itself, and weights of 0 (which become their scores), and
 *              passes old_lens = kv->seq_lens.
 *   budgets    device [B]: K' = min(budgets[b], L) tokens of each head stay:
 *              first the protected ones, with a position below sink_tokens or
 *              less than recent_tokens below the largest (a window of numbers: it
 *              has fewer tokens where some of them went before), then those of
 *              largest weight; whatever is equal is resolved towards the lower
 *              slot.  (Weights are >= 0; one that is negative or NaN counts as 0.)
 *   new_lens   device [B] int32, receives K'.  May be kv->seq_lens, old_lens or
 *              budgets itself, but must not overlap them in part (PILLAR_EINVAL).
 * Attention does not depend on the order of the rows, so the tokens that stay are
 * not closed up: those in slots below K' stay where they are and those beyond move
 * into the freed slots below K', the i-th into the i-th, K, V, weight and position
 * together.  Pages from ceil(K'/page_size) on are free afterwards; weights and
 * positions from K' on are left as they were.
 * WRITES into the pools and, for fp8, into k_scale and v_scale as
 * pillar_tree_commit does.  No page may belong to two requests.
 * state_stride >= max_seq_len; 0 <= decay < 1e30; pools and strides in multiples
 * of 16 bytes, else PILLAR_EUNSUPPORTED.  (Rows leave their order: queries of
 * a later verification must follow the cached tokens, as they do when appended.
 * The index calls go by slots: pillar_window_indices names the first and last slots,
 * which after an eviction are not the first and last tokens of the text.  A list of
 * those is to be made from `positions`, for each KV head.  Top-K lists, and
 * pillar_extend_indices for tokens appended since, name slots as ever.)
 * workspace: pillar_evict_workspace_bytes() (0: invalid description). */
size_t pillar_evict_workspace_bytes(const pillar_kv_t* kv);
int pillar_evict_kv(const pillar_kv_t* kv, const float* scores, int64_t score_stride, float decay,
                    const int32_t* old_lens, const int32_t* budgets, int32_t sink_tokens,
                    int32_t recent_tokens, float* weights, int32_t* positions, int64_t state_stride,
                    int32_t* new_lens, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- Rotary positions, and new tokens into the cache ---------------------
 *
 * A rotation turns pair i (of rotary_dim / 2) of a head by the angle position * frequencies[i], and multiplies it by `amplitude`:
 *   y1 = amplitude * (x1 cos - x2 sin),  y2 = amplitude * (x2 cos + x1 sin)
 * The pair is (dim i, dim i + rotary_dim/2), or with PILLAR_ROPE_INTERLEAVED (dim 2i, dim 2i + 1).  Dims from rotary_dim on stay as they are.
 * Angles are worked out in 64 bits (positions of any size keep their precision), the rest in fp32, with one rounding to the output's type.
 * Positions may be negative: the rotation by -position undoes one by position (and its amplitude, if the second one has 1 / amplitude).
 * frequencies: device [rotary_dim / 2] double, 8-byte aligned; rotary_dim even, 2..head_dim. */
typedef enum { PILLAR_ROPE_HALVES = 0, PILLAR_ROPE_INTERLEAVED = 1 } pillar_rope_layout;
typedef struct {
  int32_t rotary_dim;
  int32_t layout;              /* pillar_rope_layout */
  float   amplitude;           /* finite; 1 unless the scaling says otherwise */
  int32_t reserved;            /* 0 */
  const double* frequencies;   /* device */
} pillar_rope_t;

/* Frequencies of a model, host arithmetic: frequencies[i] = base^(-2 i / rotary_dim), changed for contexts that are `factor` times the
 * original_len positions that it was trained on:
 *   NONE    as they are (factor, original_len, fast and slow are not looked at)
 *   LINEAR  all divided by factor
 *   BASE    base * factor^(r / (r - 2)) instead of base (r = rotary_dim; r = 2 counts as r / 1): the lowest frequency is divided by about factor
 *   RAMP    pairs of more than `fast` turns over original_len stay, those of fewer than `slow` are divided by factor, linear in i between; amplitude
 *           0.1 ln(factor) + 1.  The two ends are i = r ln(original_len / (2 pi turns)) / (2 ln base), rounded down and up.
 *   BANDS   the same two ends, linear in the number of turns between; amplitude 1
 * frequencies: HOST [rotary_dim / 2], to be copied to the device once; amplitude: host, receives the factor for pillar_rope_t. */
typedef enum { PILLAR_ROPE_NONE = 0, PILLAR_ROPE_LINEAR = 1, PILLAR_ROPE_BASE = 2, PILLAR_ROPE_RAMP = 3, PILLAR_ROPE_BANDS = 4 } pillar_rope_scaling;
int pillar_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, int32_t original_len,
                            double fast, double slow, double* frequencies, float* amplitude);

/* Rows of heads by themselves (queries apart from their keys, keys that get other positions).
 *   x    device [tokens][num_heads][head_dim] of `dtype` (PILLAR_F32 | PILLAR_BF16), token t at element t * x_stride (x_stride >= num_heads *
 *        head_dim: rows of a fused projection will do), heads dense within; out likewise.
 *   positions  device [tokens] int32.
 * out may be x itself with the same stride; else the two spans must not overlap, nor may out's hold positions or frequencies, which the other tokens' workgroups
 * still read (PILLAR_EINVAL).  head_dim 2..512, even; at most 2^24 - 1 tokens. */
int pillar_rotate(const void* x, int64_t x_stride, int32_t tokens, int32_t num_heads, int32_t head_dim, int32_t dtype,
                  const int32_t* positions, const pillar_rope_t* rope, void* out, int64_t out_stride, void* hip_stream);

/* The newest tokens of every request: queries and keys are rotated, keys and values go into their pages (append, then attend: seq_lens
 * already counts them).  Rows are packed: request b has rows starts[b] .. starts[b+1]-1, and row i of its n is token seq_lens[b] - n + i.
 *   starts      device [B+1] int32, ascending, 0 <= starts[b] <= total_rows, at most max_new rows to a request; NULL: max_new rows each
 *               (total_rows = B * max_new).  A request may have none.  Rows from starts[B] on are neither read nor written.
 *   rope        NULL: nothing is rotated (q is copied).
 *   positions   device [total_rows] int32 for the rotation, or NULL: the number of the token in the cache, seq_lens[b] - n + i.  (After an
 *               eviction, and for the nodes of a tree, that is not the place in the text.)
 *   q, q_out    [total_rows][Hq][D] q_dtype, q_out dense, row t of q at element t * q_stride; both NULL: no queries.  q_out may be q itself
 *               if that is dense too, and must not overlap q, k_new or v_new otherwise, nor starts, positions, frequencies, or seq_lens, block_table
 *               and scales of the cache (PILLAR_EINVAL).
 *   k_new, v_new  [total_rows][Hkv][D] q_dtype, row t at element t * k_stride, v_stride.
 * The cache may have any of its types: values are rounded once, to nearest even, from the fp32 result.  WRITES into the pools and, for fp8,
 * into k_scale and v_scale: a page gets the largest scale of its older tokens' (those before the new ones; their codes are rounded anew where it
 * grew, as by pillar_tree_commit) and what the new ones need, max |finite new value| / 448, or 0 where that maximum is below 2^-90; codes are
 * those nearest to value * (1 / scale), infinities becoming the largest code, NaN staying NaN; in a page whose scale is 0, or stays below 2^-90 / 448 (that of
 * older tokens next to nothing, beside new ones that are no more), they are zeros, and NaN for what is not finite.  A page without older tokens takes the
 * new ones' scale alone.
 * Tokens whose number would be negative are skipped (their queries are rotated all the same).  No page that receives rows may belong to
 * two requests.  Bases and strides of pools, q, k_new, v_new and q_out in multiples of 16 bytes, and at most 2^24 - 1 rows (for fp8: rows of
 * queries and pages with new rows times KV heads), else PILLAR_EUNSUPPORTED. */
int pillar_append_rotated(const pillar_kv_t* kv, const pillar_rope_t* rope, const int32_t* starts, int32_t total_rows, int32_t max_new,
                          const int32_t* positions, const void* q, int64_t q_stride, void* q_out,
                          const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride, void* hip_stream);

/* ---- Attention of new tokens -------------------------------------------
 *
 * Causal attention of any number of new tokens per request over its whole context: prompts, chunks of them, and single tokens beside
 * them.  Rows are packed as in pillar_append_rotated, whose tokens they are: row i of request b's n attends to tokens 0 .. seq_lens[b]-n+i.
 *   q, out  [total_rows][Hq][D] q_dtype, dense; no part of out or lse may be q, starts, seq_lens, block_table or scales of the cache, nor the
 *           other one of the two (PILLAR_EINVAL).
 *   lse     [total_rows][Hq] fp32 natural-log-sum-exp of the logits, or NULL.
 * A row that sees no token (its number is negative, or the request has no token) gets out = 0 and lse = -inf.  What a row does not see has no
 * influence on it, whatever the cache holds there.  Every shape that pillar_kv_t can describe, group sizes up to 16.  bf16 queries with a bf16
 * or fp8 cache run on bf16 matrix instructions (P is rounded to bf16), if q, out, the pools and their strides are multiples of 16 bytes;
 * everything else, and with PILLAR_FLAG_GENERIC_KERNELS everything, on fp32 ones.  fp8 scales of what is seen are not negative, 448 times each
 * is finite, and a v_scale below 2^-80 counts as in pillar_verify_tree.  PILLAR_FLAG_EXACT_SCORES changes nothing here.  (A few tokens per request that
 * also want the statistic: pillar_verify_attn; trees: pillar_verify_tree.)
 * workspace: pillar_prompt_workspace_bytes() (0: invalid arguments), enough for any smaller batch, total_rows, max_new and max_seq_len too. */
size_t pillar_prompt_workspace_bytes(const pillar_kv_t* kv, int32_t total_rows, int32_t max_new);
int pillar_prompt_attn(const pillar_kv_t* kv, const void* q, const int32_t* starts, int32_t total_rows, int32_t max_new,
                       void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- What the logits say about given tokens ------------------------------
 *
 * Rows of logits x, one per verified position or node: with z = scale * x,
 *   lse[r]            = log sum_v exp(z[v])
 *   logprobs[r][j]    = z[tokens[r][j]] - lse[r]
 *   entropy[r]        = -sum_v p[v] log p[v],  p = exp(z - lse)                      (natural units throughout)
 *   top_ids[r][j], top_logprobs[r][j], j < top: the tokens of largest logit, in descending order, equal ones by ascending id, and their log
 *                       probabilities; where vocab < top the rest is -1 and -inf.
 *   logits     device [rows][vocab] of `dtype` (PILLAR_F32 | PILLAR_BF16), row r at element r * row_stride (>= vocab); any alignment.
 *   scale      one over the temperature; 0 < scale < 1e30.
 *   tokens     device [rows][num_tokens] int32, or NULL with num_tokens 0; an entry outside 0..vocab-1 (a missing child, say) gets -inf.
 *   lse, entropy: device [rows] fp32, each may be NULL.  top 0..64; top_ids and top_logprobs NULL exactly if top is 0.
 * Logits of -inf (masked tokens) have probability 0 and add nothing to the entropy.  A row of nothing else: lse = -inf, all log probabilities
 * -inf, entropy 0.  NaN makes the row's lse, log probabilities and entropy NaN, but it is nobody's alternative before all numbers, -inf among
 * them, are; +inf gives lse = +inf, -inf for finite tokens and NaN for itself.  Sums are fp32, of shares relative to one of the largest logits, whose own share is
 * kept apart: the log probability of a nearly certain token, and the entropy beside it, are exact to 10^-5 of themselves
 * (at the worst 2^-24 more for every 2048 logits beyond ten thousand).
 * No output may overlap logits or tokens, which others of a row's threads still read, or another output (PILLAR_EINVAL).
 * At most 2^24 - 1 rows, 2^30 logits and 2^30 given tokens in each (PILLAR_EUNSUPPORTED).
 * workspace: pillar_logprobs_workspace_bytes() (0: invalid arguments), enough for fewer rows, smaller vocabularies and fewer alternatives too. */
size_t pillar_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t top);
int pillar_token_logprobs(const void* logits, int32_t dtype, int32_t rows, int32_t vocab, int64_t row_stride, float scale,
                          const int32_t* tokens, int32_t num_tokens, float* logprobs, float* lse, float* entropy,
                          int32_t top, int32_t* top_ids, float* top_logprobs,
                          void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PILLAR_H_ */
