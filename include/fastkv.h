/*
 * fastkv.h -- C ABI of the B200 (sm_100a) FastKV token-saliency selection path.
 *
 * One layer's work is four calls on one CUDA stream:
 *
 *   fastkv_score       window-query saliency scores          (Eq. 1, Eq. 2, Sec. 4.2)
 *   fastkv_select_kv   per-KV-group top-k   (KVCompress)      (App. B.1, Alg. 1)
 *   fastkv_select_tsp  layer-level top-k    (HiddenCompress)  (App. B.1, Sec. 4.2)
 *   fastkv_compact     gather of the kept K/V rows, hidden states and position ids
 *                                                             (Alg. 1: C <- update(K, V); x)
 *
 * Conventions
 *   - Every function returns a fastkv_status; nothing throws or aborts.
 *   - Unless a parameter says HOST, every data pointer is DEVICE memory owned by the
 *     caller.  The library allocates no device memory, keeps no pointer after the
 *     enqueued work has run, and does not synchronise (fastkv_device_status and
 *     fastkv_layer_host excepted).  Work is ordered on `stream` (a cudaStream_t
 *     passed as void*; NULL is the legacy default stream).
 *   - bf16 tensors are passed as void*; the innermost dimension is contiguous and
 *     strides are counted in elements.
 *   - Sequences of a batch are packed along the token axis: sequence b owns rows
 *     cu_seqlens[b] .. cu_seqlens[b+1]-1, L_b = cu_seqlens[b+1]-cu_seqlens[b].
 *     Token indices produced and consumed by the library are sequence-local.
 *   - Inputs must be finite.  With NaN/Inf inputs the index sets are unspecified
 *     (but in range).
 */
#ifndef FASTKV_H_
#define FASTKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum fastkv_status {
  FASTKV_OK = 0,
  FASTKV_ERR_INVALID_ARG = 1,   /* NULL where a pointer is required, bad sizes, k out of range ...  */
  FASTKV_ERR_UNSUPPORTED = 2,   /* valid but not built: head_dim, G*w, alignment, device generation */
  FASTKV_ERR_WORKSPACE = 3,     /* workspace NULL, misaligned or smaller than fastkv_workspace_bytes */
  FASTKV_ERR_CUDA = 4,          /* a CUDA call failed; fastkv_last_error() has the text             */
  FASTKV_ERR_DEVICE_TIMEOUT = 5,/* a bounded device-side wait gave up (fastkv_device_status only)   */
  FASTKV_ERR_DEVICE_INDEX = 6   /* an index handed to fastkv_compact was out of range; row skipped  */
} fastkv_status;

enum { FASTKV_POOL_AVG = 0, FASTKV_POOL_MAX = 1 };
enum { FASTKV_GROUP_THEN_POOL = 0, FASTKV_POOL_THEN_GROUP = 1 };
enum { FASTKV_Q_FULL = 0, FASTKV_Q_WINDOW = 1 };

/*
 * Problem statement of one layer (Sec. 4.2, App. B.1): N_I = L_b prompt tokens per
 * sequence, N_obs = window, H = n_q_heads, key/value groups of G = H / n_kv_heads heads
 * (query head h reads KV head h / G).
 */
typedef struct fastkv_shape {
  int32_t batch;            /* B >= 1                                                         */
  int32_t total_len;        /* sum of L_b: rows of the packed k / v / hidden / pos tensors   */
  int32_t max_len;          /* max L_b (HOST knowledge used for grid sizing)                  */
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;         /* 64 or 128                                                      */
  int32_t hidden_dim;       /* multiple of 8; only used by fastkv_compact                     */
  int32_t window;           /* w = N_obs (paper: 8); fastkv_score needs G*w <= 64             */
  int32_t pool_kernel;      /* odd, 1..63 (paper: 7)                                          */
  int32_t pool_mode;        /* FASTKV_POOL_AVG | FASTKV_POOL_MAX                              */
  int32_t agg_order;        /* FASTKV_GROUP_THEN_POOL: pool the group-summed score;
                               FASTKV_POOL_THEN_GROUP: pool per query head (Eq. 1), then sum
                               within the group (App. B.1).  Identical for AVG up to rounding */
  int32_t force_window;     /* 1: the last w positions are always kept and are not ranked
                               (Sec. 4.2); 0: plain top-k over all positions                  */
  int32_t q_layout;         /* FASTKV_Q_FULL: q has total_len rows, the library reads rows
                               cu_seqlens[b+1]-w .. cu_seqlens[b+1]-1;
                               FASTKV_Q_WINDOW: q has batch*w rows, sequence b at rows b*w..  */
  float softmax_scale;      /* 0 => 1/sqrt(head_dim)                                          */
  const int32_t* cu_seqlens;/* DEVICE int32[B+1], or NULL when B == 1 (then L = total_len)    */
  int64_t q_stride_tok, q_stride_head;   /* elements; multiples of 8                          */
  int64_t k_stride_tok, k_stride_head;
  int64_t v_stride_tok, v_stride_head;
  int64_t hidden_stride_tok;
} fastkv_shape;

/*
 * How many positions each sequence keeps.  Either the same k for every sequence
 * (k > 0, cu_k == NULL; sequence b writes outputs at offset b*k, total = B*k), or a
 * DEVICE int32[B+1] array of output offsets (k_b = cu_k[b+1]-cu_k[b]) whose last entry
 * the caller repeats on the host in `total`.  With force_window, w <= k_b <= L_b;
 * otherwise 1 <= k_b <= L_b.  The uniform form is validated on the host against
 * max_len only when B == 1; per-sequence violations clamp on the device and raise
 * FASTKV_ERR_DEVICE_INDEX in the status word.
 */
typedef struct fastkv_budget {
  int32_t k;
  int32_t total;
  const int32_t* cu_k;
} fastkv_budget;

/*
 * Bytes of workspace the calls below need for this shape (a multiple of 256): what the scoring
 * kernel that fastkv_score will pick for the shape uses -- per-phase counters, per-CTA softmax
 * statistics and one un-pooled fp32 score row per KV head (per query head with
 * FASTKV_POOL_THEN_GROUP), about 4.5 MB at 131072 tokens of the Llama-3.1-8B head shape -- plus the
 * 256-byte header with the device status word.  The other calls only use the header.
 */
int fastkv_workspace_bytes(const fastkv_shape* shape, size_t* bytes);

/*
 * Saliency scores (Eq. 1 and Eq. 2; Sec. 4.2).  For each sequence, query head h and window
 * row j (query position t_j = L-w+j) the causal softmax attention row over keys 0..t_j is
 * formed, summed over the window, aggregated over each KV group and pooled along the
 * sequence (kernel `pool_kernel`, stride 1, same length; AVG zero-pads and divides by the
 * kernel size, MAX ignores out-of-range positions):
 *   scores_kv [n_kv_heads, total_len] fp32   group-wise score used by KVCompress
 *   scores_tsp[total_len] fp32 or NULL       sum over all heads (Eq. 2 up to the factor 1/H)
 * Sums replace the paper's means; rankings are unchanged.
 * q, k: bf16.  workspace: >= fastkv_workspace_bytes, 256-byte aligned; it also holds the
 * device status word, so pass the same workspace to the other calls of the layer.
 */
int fastkv_score(const fastkv_shape* shape, const void* q, const void* k, float* scores_kv,
                 float* scores_tsp, void* workspace, size_t workspace_bytes, void* stream);

/*
 * KVCompress selection (App. B.1): for every sequence and KV head, the k_b positions with the
 * largest scores_kv, ties to the lower index; with force_window the last w positions are
 * always kept and only the prefix is ranked.  idx_kv is int32 [n_kv_heads, budget.total],
 * sequence-local, strictly ascending within each (head, sequence) segment.
 */
int fastkv_select_kv(const fastkv_shape* shape, const float* scores_kv, const fastkv_budget* budget,
                     int32_t* idx_kv, void* workspace, size_t workspace_bytes, void* stream);

/*
 * HiddenCompress selection (App. B.1, Sec. 4.2): the same rule applied once per sequence to
 * the layer-level score.  idx_tsp is int32 [budget.total].
 */
int fastkv_select_tsp(const fastkv_shape* shape, const float* scores_tsp, const fastkv_budget* budget,
                      int32_t* idx_tsp, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Both selections of a TSP layer in one launch (KVCompress and HiddenCompress, App. B.1): exactly
 * what fastkv_select_kv followed by fastkv_select_tsp produce, but the nine problems of a layer
 * (one per KV head plus the layer-level one) run side by side instead of one call after the other.
 */
int fastkv_select(const fastkv_shape* shape, const float* scores_kv, const fastkv_budget* kv, int32_t* idx_kv,
                  const float* scores_tsp, const fastkv_budget* tsp, int32_t* idx_tsp, void* workspace,
                  size_t workspace_bytes, void* stream);

/*
 * Compaction (Alg. 1: C <- update(K, V); reduced hidden states x).  Byte copies:
 *   k_out[g, j, :]   = k[cu_seqlens[b] + idx_kv[g, j], g, :]     [n_kv_heads, kv.total, head_dim]
 *   v_out likewise                                               (v, v_out may both be NULL)
 *   hidden_out[j, :] = hidden[cu_seqlens[b] + idx_tsp[j], :]     [tsp.total, hidden_dim]
 *   pos_out[j]       = pos_ids[cu_seqlens[b] + idx_tsp[j]]       [tsp.total] int32
 * where b is the sequence that owns output slot j.  Pass idx_tsp == NULL on layers without
 * Token-Selective Propagation; hidden/hidden_out and pos_ids/pos_out may each be NULL.
 * An index outside [0, L_b) is skipped and reported through the status word.
 */
int fastkv_compact(const fastkv_shape* shape, const int32_t* idx_kv, const fastkv_budget* kv,
                   const int32_t* idx_tsp, const fastkv_budget* tsp, const void* k, const void* v,
                   const void* hidden, const int32_t* pos_ids, void* k_out, void* v_out,
                   void* hidden_out, int32_t* pos_out, void* workspace, size_t workspace_bytes,
                   void* stream);

/*
 * Decoding over the compressed cache (what the retained KV of Alg. 1 is kept for; Sec. 3, Sec. 5.3): one new
 * query token per sequence attends to the kept entries of its KV group,
 *   out[b, h, :] = sum_j softmax_j(scale * <q[b, h], K[h / G, j]>) * V[h / G, j, :],  j over sequence b's kept entries.
 * q: bf16 [B, n_q_heads, head_dim]; k_cache, v_cache: bf16 [n_kv_heads, kv.total, head_dim], the k_out / v_out
 * layout of fastkv_compact; out: fp32 [B, n_q_heads, head_dim]; lse (optional): fp32 [B, n_q_heads], natural-log
 * sum of exponentials of each head's logits.  workspace: >= fastkv_decode_attn_workspace_bytes, 256-byte aligned
 * (the status word is not cleared by this call).  head_dim 64 or 128, at most 8 query heads per KV head.
 */
int fastkv_decode_attn_workspace_bytes(const fastkv_shape* shape, size_t* bytes);
int fastkv_decode_attn(const fastkv_shape* shape, const void* q, const void* k_cache, const void* v_cache,
                       const fastkv_budget* kv, float* out, float* lse, void* workspace, size_t workspace_bytes,
                       void* stream);

/*
 * The layer's own causal attention with the saliency scores as a by-product (Alg. 1: the scores are read off
 * Att_l, the attention matrix of the layer that is being computed anyway; App. D.4 times the separate
 * "token importance estimation" pass this call makes unnecessary).  For every sequence b and query head h
 *   out[t, h, :] = sum_{i <= t} softmax_i(scale * <q[t, h], k[i, h / G]>) * v[i, h / G, :]        t = 0 .. L_b - 1
 * and, from the rows t = L_b - w .. L_b - 1 of the same attention matrix, the scores fastkv_score defines:
 *   scores_kv [n_kv_heads, total_len] fp32 (may be NULL: attention only), scores_tsp [total_len] fp32 or NULL.
 * q: bf16, the FULL packed queries [total_len, n_q_heads, head_dim] (shape->q_layout must be FASTKV_Q_FULL);
 * k, v: bf16 [total_len, n_kv_heads, head_dim]; strides as in the shape (multiples of 8 elements);
 * out: bf16, dense [total_len, n_q_heads, head_dim], 16-byte aligned.  Probabilities are rounded to bf16 before
 * they are multiplied with v (fp32 accumulation), the scores are formed from the fp32 logits.
 * workspace: >= fastkv_prefill_workspace_bytes, 256-byte aligned: the header with the status word (cleared by this
 * call), the window rows' logits (n_q_heads x window x total_len fp32) and one un-pooled score row per KV head.
 */
int fastkv_prefill_workspace_bytes(const fastkv_shape* shape, size_t* bytes);
int fastkv_prefill_attention(const fastkv_shape* shape, const void* q, const void* k, const void* v, void* out,
                             float* scores_kv, float* scores_tsp, void* workspace, size_t workspace_bytes,
                             void* stream);

/*
 * Paged cache: where the kept entries of Alg. 1 go when decoding continues behind them.  Entry t of sequence b is row
 * t % page_size of page block_table[b][t / page_size]; K and V pools are [n_pages, n_kv_heads, page_size, head_dim], dense,
 * 16-byte aligned.  FASTKV_CACHE_BF16: bf16 values.  FASTKV_CACHE_E4M3: 8-bit floating-point codes (4 exponent bits, 3
 * mantissa bits, largest value 448) that stand for code * scale, with one scale for each page and KV head in
 * k_scales / v_scales, fp32 [n_pages, n_kv_heads]; scales are powers of two from 2^-64 to 2^120, written by
 * fastkv_paged_append.  Pages may be shared between sequences for reading; a page that a call appends to belongs to one
 * sequence.  All pointers are DEVICE memory of the device that is current at the call.
 */
enum { FASTKV_CACHE_BF16 = 0, FASTKV_CACHE_E4M3 = 1 };
enum { FASTKV_ROT_HALVES = 0, FASTKV_ROT_ADJACENT = 1 };

typedef struct fastkv_paged_cache {
  int32_t batch;             /* B >= 1: rows of block_table                                          */
  int32_t max_pages;         /* pages a row of block_table has room for                              */
  int32_t n_pages;           /* pages in the pools                                                   */
  int32_t page_size;         /* 16, 32, 64 or 128 entries                                            */
  int32_t n_kv_heads;
  int32_t head_dim;          /* 64 or 128                                                            */
  int32_t format;            /* FASTKV_CACHE_BF16 | FASTKV_CACHE_E4M3                                */
  int32_t reserved;          /* 0                                                                    */
  void* k_pages;
  void* v_pages;
  float* k_scales;           /* FASTKV_CACHE_E4M3 only, else NULL                                    */
  float* v_scales;
  const int32_t* block_table;/* DEVICE int32 [batch, max_pages]                                      */
} fastkv_paged_cache;

/*
 * The rows one fastkv_paged_append call brings.  Sequence b owns rows cu_new[b] .. cu_new[b+1]-1 of the call's
 * [total] rows (cu_new == NULL: max_new rows each, total == batch * max_new); they become its entries lens[b],
 * lens[b] + 1, ...  Rows that no sequence owns (a padded batch, cu_new[batch] < total) go into no page; their queries are rotated
 * like the others.
 *   Source, new tokens (total_src == 0): k, v [total, n_kv_heads, head_dim] and, with n_q_heads > 0, q
 *     [total, n_q_heads, head_dim], bf16, strides in elements.
 *   Source, kept rows (total_src > 0): row r of KV head g is row cu_src[b] + idx[g, r] of k and v
 *     [total_src, n_kv_heads, head_dim], idx int32 [n_kv_heads, total] sequence-local as fastkv_select_kv writes it
 *     (cu_src == NULL when batch == 1): what fastkv_compact would copy, straight into pages.  No rotation then (the keys
 *     were rotated before they were scored) and no queries.
 *   Rotation (rot_dim > 0): the first rot_dim elements of every query and key head, at position pos[r] of its row; pairs
 *     (i, i + rot_dim / 2) for FASTKV_ROT_HALVES, (2 i, 2 i + 1) for FASTKV_ROT_ADJACENT, angle pos * inv_freq[i]
 *     (formed in 64 bits).  Positions are independent of slots: the cache holds fewer entries than the prompt had tokens.
 */
typedef struct fastkv_new_rows {
  int32_t total;             /* >= 1                                                                 */
  int32_t max_new;           /* HOST: most rows any sequence brings (grid sizing, validation)        */
  int32_t n_q_heads;         /* 0: no queries; else a multiple of n_kv_heads                         */
  int32_t rot_dim;           /* 0: no rotation; else a multiple of 16, <= head_dim                   */
  int32_t rot_pairs;         /* FASTKV_ROT_HALVES | FASTKV_ROT_ADJACENT                              */
  int32_t total_src;         /* 0, or the rows of k / v that idx points into                         */
  const int32_t* cu_new;     /* DEVICE int32 [batch + 1] or NULL                                     */
  const int32_t* cu_src;     /* DEVICE int32 [batch + 1] or NULL                                     */
  int64_t q_stride_tok, q_stride_head;   /* elements; multiples of 8                                 */
  int64_t k_stride_tok, k_stride_head;
  int64_t v_stride_tok, v_stride_head;
} fastkv_new_rows;

/*
 * Appends `rows` behind the lens[b] entries of every sequence, in one launch.  lens: DEVICE int32 [batch], read only;
 * new_lens (may be NULL, must not overlap lens): DEVICE int32 [batch], receives lens[b] plus the rows that there is room for.
 * q_out: bf16, dense [total, n_q_heads, head_dim], the rotated queries; may be q itself when q is dense.
 * Bf16 pages and q_out: rotated in fp32, rounded once.  8-bit pages: a page that had entries keeps its scale unless a new
 * row needs a larger one (the smallest 2^e with 448 * 2^e >= the largest absolute value), in which case the entries that
 * were there are re-encoded, code * old / new, rounded to nearest even; a page without entries takes the scale its new rows
 * need.  Codes are rounded once, from fp32, to nearest even.  Entries behind the new length and pages that no row falls in
 * are left as they were.
 * Reported in the status word (FASTKV_ERR_DEVICE_INDEX), never dereferenced: a page id outside the pool, an index outside
 * its sequence, rows beyond max_new, total or the block table's room; those rows are not written.  A row that is refused for its
 * page id or index keeps its slot, and new_lens counts it: read entries by new_lens only behind a status of 0.  After a wait that
 * ran out (FASTKV_ERR_DEVICE_TIMEOUT) a KV head of a page, K or V, is either as it was or has all of the call's rows.
 * workspace: 256 bytes (the header), 256-byte aligned.  The status word in it is not cleared by this call: zero a new workspace's
 * first 256 bytes once (or use one that fastkv_score has seen).  Calls that write the same sequences must be ordered.
 */
int fastkv_paged_append(const fastkv_paged_cache* cache, const fastkv_new_rows* rows, const int32_t* lens, const void* q,
                        const void* k, const void* v, const int32_t* pos, const float* inv_freq, const int32_t* idx,
                        void* q_out, int32_t* new_lens, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Attention of q_len new query tokens per sequence over the paged cache (Sec. 3, Sec. 5.3: decoding over the kept entries
 * and those appended since).  lens: DEVICE int32 [batch], the entries of each sequence, those of the new tokens included;
 * query token i of sequence b sees entries 0 .. lens[b] - (q_len - 1 - i) - 1:
 *   out[b, i, h, :] = sum_t softmax_t(scale * <q[b, i, h], K[t, h / G]>) * V[t, h / G, :]
 * q: bf16, dense [batch, q_len, n_q_heads, head_dim], 16-byte aligned; out: fp32, the same shape; lse (optional): fp32
 * [batch, q_len, n_q_heads], natural log.  A query that sees no entry gives out 0 and lse -infinity.
 * What a query token does not see never reaches it, NaN and infinities included; a NaN that it sees makes the outputs that
 * depend on it NaN, an infinity in V makes them NaN or infinite.  An entry whose logit is -infinity weighs nothing, a logit
 * of +infinity makes its row NaN, and a query whose logits are all -infinity counts as one that sees no entry.
 * Accuracy: products, maxima and sums in fp32.  8-bit pages: a query's elements below 2^-28 of its largest are rounded to
 * multiples of 2^-38 of that; the weights of 32 neighbouring entries (16 for pages of 16) carry 22 bits, or 2^-39 of their largest.
 * max_len and total_len are what the HOST knows of lens (their maximum and sum, or bounds); they size the launch, and
 * results do not depend on them beyond rounding.  A length beyond the block table's room is cut to it, a page id outside the
 * pool reads page 0 instead; both are reported in the status word (FASTKV_ERR_DEVICE_INDEX), which this call does not clear
 * (zero a new workspace's first 256 bytes once).
 * workspace: >= fastkv_paged_attn_workspace_bytes for this cache and query, 256-byte aligned; not shared by calls that
 * may overlap.  The size may rise and fall with max_len and total_len; 5 MiB are enough for all of them.
 */
typedef struct fastkv_query {
  int32_t n_q_heads;         /* a multiple of the cache's n_kv_heads                                 */
  int32_t q_len;             /* query tokens per sequence, >= 1                                      */
  int32_t max_len;           /* HOST: longest length, >= 1                                           */
  float softmax_scale;       /* 0 => 1/sqrt(head_dim)                                                */
  int64_t total_len;         /* HOST: sum of lengths; 0 => batch * max_len                           */
} fastkv_query;
int fastkv_paged_attn_workspace_bytes(const fastkv_paged_cache* cache, const fastkv_query* query, size_t* bytes);
int fastkv_paged_attn(const fastkv_paged_cache* cache, const fastkv_query* query, const int32_t* lens, const void* q,
                      float* out, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The same attention for sequences that share a long prefix (one document or system prompt behind a batch of requests; several answers
 * to one prompt): the prefix's entries are in pages of their own, in the cache's pools, and are attended once for all sequences that
 * share them.  `cache` and `lens` describe the sequences' own entries, behind the prefix: query token i of sequence b sees all entries
 * of b's prefix and its own entries 0 .. lens[b] - (q_len - 1 - i) - 1, and the softmax runs over both together.
 * Sequences cu_seqs[p] .. cu_seqs[p + 1] - 1 share prefix p; cu_seqs ascends (equal values: a prefix that nobody uses); sequences before
 * the first and behind the last have no prefix.  cu_seqs == NULL: one prefix that all share.  prefix->lens may be 0.
 * q: bf16, dense [batch, q_len, n_q_heads, head_dim], 16-byte aligned; out: bf16, the same shape, 16-byte aligned; lse (optional): fp32
 * [batch, q_len, n_q_heads], natural log, over prefix and own entries (what fastkv_paged_weights wants for the own entries).
 * A query that sees no entry gives out 0 and lse -infinity.  NaN and infinities as in fastkv_paged_attn, but that an infinite element of
 * a query counts as NaN over 8-bit pages; what lies behind a prefix's last entry in its page never reaches an output.
 * Accuracy: the softmax's weights of prefix entries are rounded to bf16 (and the output is divided by the sum of what they were rounded to),
 * all products, sums and the merge are fp32, lse takes the weights unrounded, with one rounding to bf16 at the end; own entries as in fastkv_paged_attn.  8-bit entries of a prefix meet the query as the sum of two e4m3 terms: elements
 * below 2^-9 of the largest of a query and head are rounded to multiples of 2^-16 of that, or finer.
 * Sums of weighted values are divided at the end: they stay finite for values up to 2^113, and to the end of bf16's range as long as
 * all entries of a prefix weigh no more than 2^14 times the heaviest.
 * max_len of `prefix` and of `query` and total_len size the launch only.  A length beyond the table's room is cut to it, a page id
 * outside the pool reads page 0 instead, a cu_seqs that descends or leaves 0 .. batch leaves the outputs of prefixed sequences
 * unspecified; all are reported in the status word (FASTKV_ERR_DEVICE_INDEX), which this call does not clear.
 * At most 1024 prefixes, 2^30 entries a row of their table and 128 query heads per KV head.
 * workspace: >= fastkv_prefix_attn_workspace_bytes, 256-byte aligned; not shared by calls that may overlap.
 */
typedef struct fastkv_prefix {
  int32_t n_prefixes;        /* >= 1: rows of table                                                  */
  int32_t max_pages;         /* pages a row of table has room for                                    */
  int32_t max_len;           /* HOST: longest prefix, >= 1                                           */
  int32_t reserved;          /* 0                                                                    */
  const int32_t* table;      /* DEVICE int32 [n_prefixes, max_pages]: pages of the cache's pools     */
  const int32_t* lens;       /* DEVICE int32 [n_prefixes]                                            */
  const int32_t* cu_seqs;    /* DEVICE int32 [n_prefixes + 1], or NULL with one prefix               */
} fastkv_prefix;
int fastkv_prefix_attn_workspace_bytes(const fastkv_paged_cache* cache, const fastkv_prefix* prefix, const fastkv_query* query,
                                       size_t* bytes);
int fastkv_prefix_attn(const fastkv_paged_cache* cache, const fastkv_prefix* prefix, const fastkv_query* query, const int32_t* lens,
                       const void* q, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The attention weight that every cached entry draws, accumulated over steps (the fused attention of decoding never forms the
 * attention matrix; an eviction needs its column sums).  For the query tokens that fastkv_paged_attn (or fastkv_prefix_attn) was
 * called for, with the lse it wrote:
 *   weights[b, g, t] = decay * weights[b, g, t] + sum over i and over heads h of group g, where i sees t, of
 *                      exp(scale * <q[b, i, h], K[t, g]> - lse[b, i, h])
 * for entries t of sequence b; what query token i sees is as in fastkv_paged_attn.  The last q_len entries are the query tokens' own:
 * their weight starts here, what was in the array is not read.  weights: fp32 [batch, n_kv_heads, weights_stride]; what lies behind
 * a sequence's length is neither read nor written.  q as in fastkv_paged_attn; lse: fp32 [batch, q_len, n_q_heads], natural log; a
 * row whose lse is -infinity (a query that saw nothing) draws nothing.  decay: finite, >= 0.  What a query does not see never reaches
 * a weight, NaN and infinities included.  Products, exponentials and sums in fp32, in a fixed order.
 * max_len and total_len size the launch, as in fastkv_paged_attn.  A length beyond the block table's room or weights_stride is cut
 * to it, a page id outside the pool reads page 0 instead; both are reported in the status word (FASTKV_ERR_DEVICE_INDEX), which
 * this call does not clear.  weights_stride at most 2^30, batch * n_kv_heads at most 65535.  workspace: 256 bytes (the header),
 * 256-byte aligned.
 */
int fastkv_paged_weights(const fastkv_paged_cache* cache, const fastkv_query* query, const int32_t* lens, const void* q,
                         const float* lse, float decay, float* weights, int64_t weights_stride, void* workspace,
                         size_t workspace_bytes, void* stream);

/*
 * Eviction by accumulated weight, in place: KVCompress (App. B.1: per KV head the entries of largest score, the window always) for a
 * cache that has grown while decoding.  A sequence with lens[b] > limit keeps, for each KV head, its last `window` entries and the
 * m = keep - window others of largest weight (ties to the lower slot; -0 counts as 0, NaN as the lowest); the others are untouched.
 * Entries move within the sequence's pages:
 *   a kept entry in a slot below m, the window's aside, stays; the r-th free slot below m (ascending) takes the r-th other kept one
 *   (ascending); window entry lens[b] - window + i goes to slot m + i.
 * Slots behind the new length are left as they were; pages that lie there altogether may be given to other sequences.  8-bit pages: a
 * page that receives entries takes the largest scale of the pages that its entries come from, its own among them if an entry stays;
 * codes are encoded again, code * old / new, rounded to nearest even.
 *   weights, ids: fp32 and int32 [batch, n_kv_heads, stride] (ids may be NULL; what the caller knows the entries by, positions say);
 *   new_weights, new_ids: the same shape, receive those of the entries by their new slots (copies, for sequences that are not cut);
 *   may not overlap weights and ids; new_ids goes with ids.  new_lens (may be NULL, must not overlap lens): int32 [batch].
 * All pages a sequence of the call holds belong to it alone if it is cut.  A length below 0 or beyond max_len, stride or the block
 * table's room leaves the sequence as it is, new_lens[b] = lens[b] and nothing written to new_weights and new_ids; a page id
 * outside the pool is never dereferenced, rows that would be read from or written to it are not moved.  Both are reported in the
 * status word (FASTKV_ERR_DEVICE_INDEX), which this call does not clear.  stride at most 2^30, batch * n_kv_heads at most 65535.
 * workspace: >= fastkv_paged_evict_workspace_bytes, 256-byte aligned; not shared by calls that may overlap.
 */
typedef struct fastkv_eviction {
  int32_t keep;              /* entries that a sequence is cut to, >= 1                              */
  int32_t limit;             /* sequences with more entries are cut; >= keep                         */
  int32_t window;            /* last entries that are always kept, 0 .. keep                         */
  int32_t max_len;           /* HOST: longest length                                                 */
} fastkv_eviction;
int fastkv_paged_evict_workspace_bytes(const fastkv_paged_cache* cache, const fastkv_eviction* eviction, size_t* bytes);
int fastkv_paged_evict(const fastkv_paged_cache* cache, const fastkv_eviction* eviction, const int32_t* lens, const float* weights,
                       const int32_t* ids, int64_t stride, float* new_weights, int32_t* new_ids, int32_t* new_lens,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * Synchronises `stream`, then copies the device status word of `workspace` to the HOST
 * integers *status (a fastkv_status) and *site (which wait or check raised it; 0 if none).
 */
int fastkv_device_status(const void* workspace, void* stream, int32_t* status, int32_t* site);

/*
 * One whole layer step from HOST buffers (the end-to-end path of the bench): copies q, k, v,
 * hidden, pos_ids (HOST, pinned for full speed) into `arena` (DEVICE, caller-owned, at least
 * fastkv_layer_host_arena_bytes), runs score -> select_kv -> select_tsp -> compact on `stream`,
 * copies idx_kv, idx_tsp, k_out, v_out, hidden_out, pos_out back to the HOST outputs and
 * synchronises.  B == 1 or uniform budgets only (budget.cu_k must be NULL); shape->cu_seqlens,
 * if given, is a HOST array here.  k_tsp == 0 skips the TSP part.
 */
int fastkv_layer_host_arena_bytes(const fastkv_shape* shape, int32_t k_kv, int32_t k_tsp,
                                  size_t* bytes);
int fastkv_layer_host(const fastkv_shape* shape, int32_t k_kv, int32_t k_tsp, const void* q,
                      const void* k, const void* v, const void* hidden, const int32_t* pos_ids,
                      int32_t* idx_kv, int32_t* idx_tsp, void* k_out, void* v_out,
                      void* hidden_out, int32_t* pos_out, void* arena, size_t arena_bytes,
                      void* stream);

/*
 * fastkv_score for callers that cannot allocate device memory (no counterpart in the paper:
 * this is a deployment variant, not a step of the method).  Some callers have no workspace to
 * give: a plug-in inside a serving process whose device allocator belongs to the host
 * framework, code that runs where cudaMalloc is not permitted, a minimal C client without an
 * allocator.  This entry point computes exactly what fastkv_score computes, with the scratch
 * memory of the scoring kernels held in a fixed 16 MiB device array inside the library (so
 * every GPU that loads the library carries those 16 MiB until the process exits).  It calls no
 * cudaMalloc, cudaFree or other allocating routine.
 *   - Limit: fastkv_workspace_bytes(shape) must be <= 16 MiB (Llama-3.1-8B head shape: about
 *     500 000 tokens per call); larger shapes return FASTKV_ERR_WORKSPACE and launch nothing.
 *   - The first call on each device looks up the array's device address (the device must be
 *     current); make that first call before starting any stream capture.
 *   - All calls on a device share the one array, which keeps the previous call's contents; the
 *     words that must start at zero are cleared on `stream` by every call.  Two calls whose
 *     GPU work overlaps (different streams, no ordering) race on it: serialise them.
 *   - The device status word lives inside the array; fastkv_score_static_status reads it.
 *     Waits on the device stay bounded as in fastkv_score.
 * q, k, scores_kv, scores_tsp, stream: as for fastkv_score.
 */
int fastkv_score_static(const fastkv_shape* shape, const void* q, const void* k, float* scores_kv,
                        float* scores_tsp, void* stream);
/*
 * fastkv_device_status for the built-in array of the current device (no counterpart in the paper):
 * synchronises `stream`, then copies the status word and site left by the last fastkv_score_static
 * call on this device to the HOST integers.  Allocates nothing.  FASTKV_ERR_INVALID_ARG if
 * fastkv_score_static has not run on this device yet.
 */
int fastkv_score_static_status(void* stream, int32_t* status, int32_t* site);

/*
 * Test and tuning hooks (no counterpart in the paper).  Process-wide, not thread-safe; the
 * defaults (all 0) are what production code wants.  Keys:
 *   "score_path"          0 the library picks the scoring kernel by shape; 1 two kernels with
 *                         fp32 logits buffered in the workspace; 2 persistent kernel that reads K
 *                         a second time from L2; 3 persistent kernel that parks the logits in
 *                         tensor memory (FASTKV_ERR_UNSUPPORTED from the scoring calls when a
 *                         sequence is too long for it).  fastkv_workspace_bytes follows the choice.
 *   "score_partition"     path 3: several (sequence, head) phases side by side, each on its share of
 *                         the CTAs: 0 by shape (batches, and single sequences of middling length);
 *                         1 never; 2 whenever the shape allows it
 *   "fused_heads"         path 2: KV heads scored side by side in one phase (0: by size)
 *   "fused_lead"          path 2: phases the first read may lead the second (0: by size)
 *   "wait_limit_cycles"   clock cycles a device-side wait of the scoring, prefill and paged kernels polls before it
 *                         gives up and raises FASTKV_ERR_DEVICE_TIMEOUT (0: about a second)
 *   "extra_publications"  the scoring kernels' second pass waits for this many publications of
 *                         softmax statistics beyond those that will arrive; with a short wait limit
 *                         this makes a bounded wait run out without any fault (timeout test)
 *   "prefill_skip_commit" n > 0: the prefill attention's issuer withholds the signal that S of key tile
 *                         n - 1 is ready (first query tile of every CTA); with a short wait limit the
 *                         softmax warps' bounded wait runs out without any fault (timeout test); 0: off
 *   "paged_skip_copy"     n > 0: the paged attention withholds the copies of the first pair of warps' n-th chunk of every
 *                         segment, the paged append (new tokens into 8-bit pages, more than 8 rows per sequence) those of
 *                         every block's n-th head; with a short wait limit the wait for them runs out without any fault
 *                         (timeout test); 0: off
 *   "prefix_skip_commit"  n > 0: the prefix attention withholds the signal that S of the n-th chunk of every CTA's share is ready
 *                         (first row tile); with a short wait limit the waits for it run out without any fault (timeout test); 0: off
 *   "paged_two_maps"      1: the paged attention copies K and V pages through a tensor map each, as it does for pools
 *                         that lie 2^40 bytes or more apart (test); 0: through one map where it can
 *   "time_kernels"        1: record a pair of CUDA events around every kernel the library launches
 *                         (this creates events, and an event between two kernels keeps the second
 *                         from starting under the first one's tail); read with
 *                         fastkv_debug_kernel_time
 * Unknown keys return FASTKV_ERR_INVALID_ARG.
 */
int fastkv_debug_set(const char* key, int64_t value);
/*
 * Sum of the device durations (HOST double, milliseconds) and number of launches recorded for one
 * kernel class since the last query (0 scoring kernel, 1 pooling kernel, 2 selection, 3 compaction,
 * 4 decode attention, 5 prefill attention, 6 window scores, 7 paged append, 8 paged attention, 9 accumulated weights, 10 eviction,
 * 11 prefix attention and its merge); waits for the recorded launches and forgets them.  *name receives a static
 * string.  Any of the three outputs may be NULL.  No counterpart in the paper (measurement aid).
 */
int fastkv_debug_kernel_time(int32_t kernel, double* total_ms, int64_t* launches, const char** name);

/* Text for a fastkv_status; static storage. */
const char* fastkv_status_string(int status);
/* Text of the last FASTKV_ERR_CUDA / argument failure on the calling thread; static storage. */
const char* fastkv_last_error(void);
/* Number of kernels the library has launched from this process (for launch accounting). */
int64_t fastkv_kernel_launches(void);

#ifdef __cplusplus
}
#endif
#endif /* FASTKV_H_ */
