/*
 * dopr.h -- C ABI of the DoPR online-scoring hot path on MI355X (gfx950).
 *
 * DoPR (Reusable Compressed Document Prefixes for Efficient LLM Reranking)
 * scores a (query, document) pair by running only the query tokens and one
 * scoring token through the reranker, while every layer's attention also sees
 * the document's compressed prefix key/value states, computed offline and
 * injected as a pre-filled cache (Sec. 3.1, Eq. 3; Sec. 3.3; Sec. 3.4).  This
 * library implements one decoder layer's share of that online step:
 *
 *   dopr_store_*       the HBM-resident prefix store of per-document K/V
 *                      states (Sec. 3.3: query-independent, reused across
 *                      queries; bf16 per Table 7, or 4 bits a value).
 *   dopr_prefix_attn   batched GQA attention in which each pair's online
 *                      tokens attend to [that document's prefix ; their own
 *                      causal keys] (Sec. 3.4; the query/score tokens see the
 *                      document only through its prefix states, Sec. 3.2.2).
 *   dopr_score_logits  the relevance score read off the score token's state
 *                      (Sec. 3.2.3, Eq. for s(q,d)), as a yes/no logit pair.
 *   dopr_prefix_attn_score
 *                      the last layer's share: only the score token's rows,
 *                      with the score head fused into the attention epilogue.
 *   dopr_decoder_layer the whole decoder layer around that attention.
 *   dopr_salience      offline: which document positions become prefix
 *                      slots (Sec. 3.2.1 salience, top-K selection).
 *   dopr_quantize_rows, dopr_quant_matmul, dopr_norm_residual, dopr_rotary
 *                      the operators of a layer around its attention, with
 *                      8-bit integer products and for other layer families.
 *
 * Conventions shared by every call
 *   - All device buffers are allocated by the caller and passed as raw device
 *     pointers; the library never calls hipMalloc/hipFree.  Buffers must stay
 *     alive until the stream has passed the call.  (The one exception is
 *     dopr_prefix_attn_noalloc, whose plan lives in a fixed scratch array
 *     that the library's code object holds on each device.)
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *     Every call is asynchronous on that stream unless stated otherwise.
 *   - bf16 means IEEE bfloat16 bit patterns (uint16); fp32 means IEEE float.
 *   - head_dim D is 128 (Qwen3, Llama 3) or 64 (Llama 3.2 1B, the model of
 *     the cross-family check in the Appendix); the decoder layer and the
 *     salience selection take D = 128 only.  n_q_heads must be a multiple
 *     of n_kv_heads; q head h reads kv head h / (n_q_heads / n_kv_heads).
 *   - Every call returns a dopr_status_t.  Host-checkable argument errors are
 *     returned before anything is launched.  Errors found on the device (a
 *     doc id that is out of range or not resident, malformed cu_seqlens) are
 *     deferred: the affected outputs are written as zeros, nothing is read
 *     out of bounds, and dopr_check_status() reports the error.
 *   - No C++ exception crosses this ABI and the library never aborts.
 *   - Calls that share a store and overlap on different streams may race on
 *     the store's deferred status word only (never on data).
 */
#ifndef DOPR_H
#define DOPR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DOPR_OK = 0,
  DOPR_ERR_INVALID_ARG = -1, /* null pointer, bad size, bad shape          */
  DOPR_ERR_UNSUPPORTED = -2, /* valid but not implemented (e.g. D = 96)    */
  DOPR_ERR_DOC_RANGE = -3,   /* doc id outside [0,n_docs) or not resident  */
  DOPR_ERR_WORKSPACE = -4,   /* workspace or pool smaller than required    */
  DOPR_ERR_HIP = -5,         /* a HIP runtime call failed                  */
  DOPR_ERR_SEQLEN = -6       /* cu_seqlens not monotone, T_p < 1,
                                T_p > max_tokens or cu[P] != total_tokens  */
} dopr_status_t;

/* Opaque store handle.  The library owns only this small host struct; the
 * store's index and payload live in the caller's device pool. */
typedef struct dopr_store *dopr_store_t;

/* ------------------------------------------------------------------------ */
/* Prefix store (Sec. 3.1 Eq. 3 and Sec. 3.3: per document d, the multi-layer
 * K/V states C~_d of its K_infer selected prefix slots, stored offline).      */

typedef struct {
  int32_t n_layers;       /* decoder layers held per document (>= 1)        */
  int32_t n_kv_heads;     /* Hkv (>= 1)                                     */
  int32_t head_dim;       /* D; 128 or 64 (UNSUPPORTED otherwise)           */
  int64_t n_docs;         /* size of the doc-id space [0, n_docs)           */
  const int32_t *doc_len; /* HOST [n_docs]: prefix slots L_d of doc d.
                             0 is allowed (no prefix); -1 = not resident
                             (pairs naming it fail with DOC_RANGE).         */
} dopr_store_desc_t;

/* Sizes of a store.  *pool_bytes (required) is what dopr_store_create needs
 * in the caller's pool: a small header, the index (12 B per doc id) and the
 * payload in the library's internal layout (V rows padded to 8 slots).
 * *payload_bytes (optional, may be NULL) is the canonical K/V size
 * sum_d L_d * n_layers * Hkv * D * 2 (K and V) * 2 bytes, the document-side
 * memory the paper reports per pair (Tables 3 and 9).  Pure host arithmetic. */
dopr_status_t dopr_store_bytes(const dopr_store_desc_t *desc,
                               size_t *pool_bytes, size_t *payload_bytes);

/* Lay out a store in `pool` (device, >= pool_bytes, 256-byte aligned) and
 * write its index (stream-ordered copy from host).  The payload is left
 * uninitialised until dopr_store_put fills it.  *out receives a handle that
 * must be released with dopr_store_destroy (which does not free the pool). */
dopr_status_t dopr_store_create(const dopr_store_desc_t *desc, void *pool,
                                size_t pool_bytes, void *stream,
                                dopr_store_t *out);

/* Copy the prefix K/V states of `n` documents for one layer into the store.
 *   doc_ids      dev int32 [n]   documents to fill (resident ones)
 *   src_cu_slots dev int64 [n+1] slot ranges of each document in k_src/v_src;
 *                must satisfy src_cu_slots[i+1]-src_cu_slots[i] == L_d
 *   k_src, v_src dev bf16 [src_cu_slots[n], Hkv, D] (canonical layout: the
 *                final keys/values of each prefix slot, already normed and
 *                rotated at positions 0..L_d-1 as in any pre-filled cache)
 * A doc id that is out of range, not resident, or whose slot count differs
 * from L_d is skipped and reported by dopr_check_status as DOC_RANGE.      */
dopr_status_t dopr_store_put(dopr_store_t st, int32_t layer, int64_t n,
                             const int32_t *doc_ids,
                             const int64_t *src_cu_slots, const void *k_src,
                             const void *v_src, void *stream);

dopr_status_t dopr_store_destroy(dopr_store_t st);

/* Stores of 4 bits a value.  A store has a format, and every call that takes a
 * store takes one of either (dopr_store_put and dopr_gather_prefix included,
 * whose k and v stay bf16; dopr_store_copy_docs wants both of one format).
 *   DOPR_STORE_BF16  the states as they are put (dopr_store_create)
 *   DOPR_STORE_FP4   17 bytes for 32 values, about a quarter of the bytes: a
 *                    block of 32 values holds a power of two, the smallest 2^e
 *                    with 7 * 2^e >= the block's largest magnitude (e in
 *                    -125 .. 125), and for each value a 4-bit float c (0, 0.5,
 *                    1, 1.5, 2, 3, 4, 6 and their negatives), the nearest to
 *                    value / 2^e, ties to the even code, at most 6.
 *                    A key's block is the 32 dims 64 j + 16 i + 8 h + e of one
 *                    (j, h), i < 4, e < 8, of one slot; a value's block is one
 *                    dim of 32 slots (32 s .. 32 s + 31 of the document, fewer
 *                    at its end).  No value is off by more than 2^e (beyond
 *                    7 * 2^125, by more).  A block with a value that is not
 *                    finite reads as NaN.  A dopr_store_put names a document
 *                    once.
 * What is held are bf16 values, and a call on a 4-bit store computes what it
 * computes on a bf16 store that holds those values: the same bits wherever the
 * same kernels run (not the pairs of one token, see dopr_prefix_attn).  */
typedef enum { DOPR_STORE_BF16 = 0, DOPR_STORE_FP4 = 1 } dopr_store_format_t;

/* dopr_store_bytes and dopr_store_create for a format.  *payload_bytes of a
 * 4-bit store: codes and exponents of the documents' slots; its pool holds
 * whole chunks of 32 slots, and a document has at most 2^31 - 64.          */
dopr_status_t dopr_store_bytes_as(const dopr_store_desc_t *desc,
                                  int32_t format, size_t *pool_bytes,
                                  size_t *payload_bytes);
dopr_status_t dopr_store_create_as(const dopr_store_desc_t *desc,
                                   int32_t format, void *pool,
                                   size_t pool_bytes, void *stream,
                                   dopr_store_t *out);

/* dopr_store_put of keys as a projection leaves them: for slot j of document
 * doc_ids[i], source row r = src_cu_slots[i] + j,
 *   k' = RoPE_pos(RMSNorm(k[r]) * k_norm_w)     (no norm without k_norm_w)
 *   pos = positions[r], or j when positions is NULL
 * the rotation being dopr_rotary's (rotary_dim, interleaved, inv_freq,
 * attention_factor).  k' is formed in 64 bits and rounded to fp32 and from there
 * to bf16, v is rounded to bf16, and both go into the store, of either format,
 * as dopr_store_put would put them.  Rows and heads lie any distance apart (k
 * and v may be parts of one buffer).  A document whose rows do not lie in
 * [0, rows), whose slot count differs from L_d, or that is out of range or not
 * resident, is skipped and reported by dopr_check_status as DOC_RANGE.  Where
 * rows is 0 (documents without slots), k and v may be NULL.  A call names a
 * document once.                                                           */
typedef struct {
  int32_t layer;
  int32_t dtype;            /* of k, v and k_norm_w (dopr_dtype_t: bf16, fp16
                               or fp32)                                     */
  int64_t n;                /* documents, >= 0                              */
  int64_t rows;             /* of k, v and positions                        */
  const int32_t *doc_ids;   /* dev int32 [n]                                */
  const int64_t *src_cu_slots; /* dev int64 [n+1]                           */
  const void *k;            /* dev [rows, Hkv, D]                           */
  int64_t k_row_stride, k_head_stride; /* elements, >= 0                    */
  const void *v;            /* dev [rows, Hkv, D]                           */
  int64_t v_row_stride, v_head_stride;
  const void *k_norm_w;     /* dev [D] or NULL                              */
  const int32_t *positions; /* dev int32 [rows] or NULL                     */
  const float *inv_freq;    /* dev fp32 [rotary_dim / 2]                    */
  int32_t rotary_dim;       /* even, 2 .. D                                 */
  int32_t interleaved;      /* 0 or 1                                       */
  float attention_factor;   /* finite                                       */
  float rms_eps;            /* finite, >= 0                                 */
} dopr_put_rotary_args_t;

dopr_status_t dopr_store_put_rotary(dopr_store_t st,
                                    const dopr_put_rotary_args_t *args,
                                    void *stream);

/* Carry documents over from one store to another (store maintenance: the
 * prefix states are built once per document offline and kept for reuse,
 * Sec. 3.3-3.4, so a collection that grows or shrinks is served by a new
 * store holding the kept documents).  For every document id resident in
 * both stores with the same slot count, dst receives src's states for all
 * layers and kv heads (and their key-norm bounds); ids resident only in dst
 * keep their contents (fill them with dopr_store_put), ids resident only in
 * src are dropped.  So a store with more resident ids appends documents,
 * and one with fewer repacks the kept ones densely.  Both stores must have
 * the same n_docs (id space), n_layers and n_kv_heads and distinct,
 * non-overlapping pools (INVALID_ARG otherwise).  A document resident in
 * both with different slot counts is skipped and reported as a deferred
 * DOC_RANGE on dst.  Asynchronous on `stream`.                             */
dopr_status_t dopr_store_copy_docs(dopr_store_t dst, dopr_store_t src,
                                   void *stream);

/* ------------------------------------------------------------------------ */
/* Online prefix attention (Sec. 3.4): for every pair p with document
 * d = doc_ids[p] and online tokens j = 0..T_p-1 (query tokens, then the
 * score token last), q head h, kv head g = h / n_rep:
 *   q^ = RoPE_{L_d + j}(RMSNorm(q[j,h]) * q_norm_w)
 *   k^ = RoPE_{L_d + j}(RMSNorm(k[j,g]) * k_norm_w)        (own keys)
 *   keys   = [ K_d[g, 0..L_d-1] ; k^[0..j, g] ]
 *   values = [ V_d[g, 0..L_d-1] ;  v[0..j, g] ]
 *   out[j,h] = softmax(softmax_scale * q^ . keys) . values
 * RoPE is the rotate-half form: the pair (x_i, x_{i+D/2}) turns by
 * position * omega_i with omega_i = rope_theta^(-2i/D), or rope_inv_freq[i]
 * when given.  RMSNorm is per head over D with epsilon rms_eps; with both
 * norm gains NULL there is no RMSNorm (q^ = RoPE(q), k^ = RoPE(k), as in
 * attention families without QK-norm such as Llama).  Online positions
 * continue after the prefix.                                               */
typedef struct {
  int32_t n_pairs;          /* P >= 0                                       */
  int32_t n_q_heads;        /* Hq, multiple of the store's Hkv              */
  int32_t max_tokens;       /* upper bound on every T_p (>= 1)              */
  int32_t kernel_variant;   /* 0 = automatic: 8, except at D = 64 for at most
                               128 stacked rows (tokens * Hq / Hkv) with a
                               prefix of more than 256 slots, which run 2;
                               1, 2, 3, 6, 8 select a
                               kernel (identical results, except that a
                               unit over the logit bound with a row out of
                               range is recomputed whole by the exact pass,
                               to bf16 rounding, and units differ; for
                               tuning sweeps): 1 = 4 waves x 64 rows, 2 = 8 waves
                               x 32 rows, 3 = 4 waves x 32 rows (each one
                               block per CU, 256 prefix slots resident;
                               512 at D = 64), 6 = 4 waves x 32 rows, two
                               blocks per CU, 96 slots resident (256 at
                               D = 64); 8 = the pass kernel: 4-wave blocks
                               (two per CU at D = 128, three at D = 64) take
                               (work item, kv head) units of up to 128 rows,
                               stream their keys through LDS and read the
                               own keys from a k^ buffer in the workspace
                               (2 Hkv D bytes per online token) filled by a
                               separate normalise-and-rotate kernel (block
                               kernels run in its place from 2^15 q heads
                               per kv head, prefixes of 2^31 / D slots or
                               Hkv D = 2^25 on);
                               4 = exact running-max softmax for every row
                               (slower; the reference for the fast path);
                               5 = self-check: the fast pass queues every
                               work unit for the exact pass (tests only).
                               Over a 4-bit store 0 runs kernels that need
                               no plan (see dopr_prefix_attn), and 1, 2 and
                               3 run shape 6                               */
  int64_t total_tokens;     /* Ntok = cu_seqlens[P]                         */
  const int32_t *doc_ids;   /* dev int32 [P]                                */
  const int32_t *cu_seqlens;/* dev int32 [P+1], cu[0] = 0, T_p >= 1         */
  const void *q;            /* dev bf16 [Ntok, Hq, D]   raw (pre-norm)      */
  const void *k;            /* dev bf16 [Ntok, Hkv, D]  raw (pre-norm)      */
  const void *v;            /* dev bf16 [Ntok, Hkv, D]                      */
  const void *q_norm_w;     /* dev bf16 [D], or NULL with k_norm_w NULL:
                               no per-head RMSNorm                          */
  const void *k_norm_w;     /* dev bf16 [D], or NULL (see q_norm_w)         */
  float rms_eps;            /* e.g. 1e-6                                    */
  float rope_theta;         /* e.g. 1e6                                     */
  float softmax_scale;      /* e.g. 1/sqrt(D); finite and > 0               */
  void *out;                /* dev bf16 [Ntok, Hq, D]                       */
  float *lse;               /* dev fp32 [Ntok, Hq] natural-log sum-exp of
                               the scaled logits, or NULL                   */
  void *workspace;          /* dev scratch, >= dopr_prefix_attn_workspace() */
  size_t workspace_bytes;
  void *timing_begin;       /* optional hipEvent_t recorded on the stream
                               right before the attention kernel, or NULL.
                               With the pass kernel (8) the interval holds
                               the launch that forms k^; for up to 8,192
                               pairs that launch also fills the plan's
                               tables and zeroes the outputs of pairs
                               without a document.                          */
  void *timing_end;         /* optional hipEvent_t recorded right after it,
                               or NULL (profiling of the dominant kernel)   */
  const float *rope_inv_freq; /* dev fp32 [D/2] rotation frequencies
                               omega_i (e.g. a family's rescaled ones), or
                               NULL for rope_theta^(-2i/D); 4-byte aligned */
  int32_t rows_per_item;    /* 0 = automatic.  Else the size, in stacked
                               rows (token x q head of one kv head), of the
                               work items a document's rows are cut into:
                               a multiple of 32 in [64, 2^20] (the pass
                               kernel's items hold at most 128).  Outputs do
                               not depend on it, but for the rounding of
                               units recomputed whole (see kernel_variant;
                               a tuning and test knob).
                               Full-row calls only: must be 0 for
                               dopr_prefix_attn_score (INVALID_ARG).        */
  int32_t queue_order;      /* order in which each of the 8 work queues
                               (one per XCD) hands out its (item, kv head)
                               units.  0 = automatic: longest-first while
                               the CUs average at most 128 units each,
                               else natural; 1 = natural (item order);
                               2 = longest-first (costliest document group
                               first, item order within a cost class) up to
                               32768 units, natural beyond.  Outputs do not
                               depend on it (a tuning and test knob); other
                               values are INVALID_ARG.                      */
} dopr_attn_args_t;

/* Workspace bytes needed by dopr_prefix_attn for these arguments (host).
 * Never fewer than a plan for them takes, also where none is made.         */
dopr_status_t dopr_prefix_attn_workspace(dopr_store_t st,
                                         const dopr_attn_args_t *args,
                                         size_t *bytes);

/* Run the online attention of one layer for a batch of pairs.  Pairs that
 * share a document are grouped on the device so that the document's prefix
 * is read from HBM once per group and reused from LDS.  Pairs with a bad doc
 * id get zero outputs (lse = -inf) and a deferred DOC_RANGE status.
 *
 * Over a 4-bit store the automatic choice makes no plan and groups nothing.
 * Pairs of several tokens: every 32 stacked rows of a (pair, kv head) stream
 * the document's codes by themselves.  Where such units are many, each is one
 * wave's, and its rows are bit for bit those of the planned kernels; where they
 * are few, waves and blocks share a unit's keys and add their sums, so that a
 * row's last bits go by how many units a call has.  Pairs of one token each
 * (max_tokens 1 and total_tokens = n_pairs): a unit is a (pair, kv head), and
 * q^ and k^ stay in 32 bits (q^ enters the products as two bf16 parts), so the
 * outputs are nearer to the definition than the planned kernels', and not their
 * bits.  Many short pairs that share few documents run faster by a plan, whose
 * items hold rows of several pairs: kernel_variant 8 (4,096 single tokens on 64
 * documents of 512 slots 187 us, and 275; 1,024 pairs of 4 tokens on 16 of
 * 4,096 330 us, and 541).  A value v that is not finite makes its dim NaN in
 * the rows of the tokens before it too, whose weight of zero it meets in the same
 * 32 keys; other pairs' rows stay as they are.  (The planned kernels, over a
 * store of either format, pass it on to the rows of other pairs of the document
 * that share its work unit as well.)                                       */
dopr_status_t dopr_prefix_attn(dopr_store_t st, int32_t layer,
                               const dopr_attn_args_t *args, void *stream);

/* dopr_prefix_attn for callers that cannot allocate device memory (code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc).  Same arguments, results and errors as dopr_prefix_attn,
 * except:
 *   - args->workspace must be NULL and args->workspace_bytes 0: the plan is
 *     laid out in a scratch array that the library holds, one copy per
 *     device, from the first use on that device until the process ends;
 *   - the scratch holds at most 64 MiB (DOPR_NOALLOC_SCRATCH_BYTES).  A call
 *     whose plan needs more returns DOPR_ERR_WORKSPACE and launches nothing;
 *     dopr_prefix_attn_workspace gives the size, except that here the
 *     automatic choice (kernel_variant 0) and the self-check variant 5 never
 *     take the pass kernel (8), whose plan grows with every token; variant 8
 *     is run only when asked for and its plan fits (its work items counted
 *     with up to 2048 rows and 32 bytes each per kv head; when only the
 *     128-row items it is run with do not fit, the block kernels run, with
 *     the same outputs).  Over a 4-bit store the automatic choice is
 *     dopr_prefix_attn's while its keys fit (2 Hkv D + 4 D bytes a token), else
 *     the block kernels;
 *   - the call allocates nothing: no hipMalloc, hipFree or allocating
 *     library routine.
 * Every call on one device shares that device's scratch: calls that overlap
 * on one device (other streams, other threads) race and must be ordered by
 * the caller.  The plan's kernels clear what must start at zero.  Outputs
 * are bitwise identical to dopr_prefix_attn's for the same inputs.  (Over a
 * 4-bit store, past those bytes: to kernel_variant 6's, and to the automatic
 * choice's where its units are one wave's.)                                */
#define DOPR_NOALLOC_SCRATCH_BYTES ((size_t)64 << 20)
dopr_status_t dopr_prefix_attn_noalloc(dopr_store_t st, int32_t layer,
                                       const dopr_attn_args_t *args,
                                       void *stream);

/* ------------------------------------------------------------------------ */
/* Score head (Sec. 3.2.3): s(q,d) from the score token's hidden state h.
 * Read as RMSNorm followed by a two-row linear head (yes, no):
 *   h^ = RMSNorm(h) * norm_w;  l_yes = w_yes . h^;  l_no = w_no . h^;
 *   s  = l_yes - l_no   (log-odds of "relevant"; what RankNet consumes).   */
typedef struct {
  int32_t n_pairs;           /* P >= 0                                      */
  int32_t width;             /* W, multiple of 8, >= 8                      */
  const void *h;             /* dev bf16; row r starts at h + r*h_row_stride */
  int64_t h_row_stride;      /* elements between rows, >= width, mult. of 8 */
  const int32_t *row_index;  /* dev int32 [P]: h row of pair p, or NULL    */
  const int32_t *cu_seqlens; /* dev int32 [P+1]: used when row_index is
                                NULL: row = cu_seqlens[p+1]-1 (the score
                                token is each pair's last online token).
                                Both NULL: row = p.                         */
  const void *norm_w;        /* dev bf16 [W]                                */
  const void *w_head;        /* dev bf16 [2, W]: row 0 = yes, row 1 = no    */
  float rms_eps;
  float *logits;             /* dev fp32 [P, 2] (l_yes, l_no), or NULL      */
  float *score;              /* dev fp32 [P]                                */
} dopr_score_args_t;

dopr_status_t dopr_score_logits(const dopr_score_args_t *args, void *stream);

/* ------------------------------------------------------------------------ */
/* Last-layer scoring (Sec. 3.2.3 with Sec. 3.4).  The score head reads only
 * the score token's hidden state, so in the last layer only the final row
 * j = T_p - 1 of every pair needs an attention output.  This call computes
 * exactly the rows dopr_prefix_attn computes for those tokens (same keys:
 * all L_d prefix slots and all T_p own keys, so every own key and value is
 * still read and every own key is normed and rotated), and feeds them to
 * the score head of dopr_score_logits with width W = n_q_heads * D:
 *   h = out[p] viewed as [W] (bf16-rounded attention output),
 *   h^ = RMSNorm(h) * norm_w;  l_yes = w_yes . h^;  l_no = w_no . h^;
 *   s = l_yes - l_no.
 * The head is fused into the attention epilogue: each (pair, q head) row
 * contributes its partial sums of h^2, norm_w*w_yes*h and norm_w*w_no*h;
 * a small kernel adds the n_q_heads partials of a pair in head order.
 * Arguments are those of dopr_prefix_attn with two differences:
 *   out  dev bf16 [P, Hq, D]: the score rows, or NULL (not written);
 *   lse  dev fp32 [P, Hq], or NULL;
 * and the workspace comes from dopr_prefix_attn_score_workspace.
 * kernel_variant 0 (automatic) runs one wave per work unit of at most 32
 * score rows while every resident prefix is at most 512 slots (one 4-wave
 * block per 4 units, no block barrier), else shape 6; 1 and 3 select
 * shape 6 here (2 and 6 as above; identical results in every case).  A
 * pair with a bad doc id gets zero rows, lse -inf, logits and score 0, and
 * a deferred DOC_RANGE status.  All buffers are caller-owned.              */
typedef struct {
  const void *norm_w;       /* dev bf16 [W], W = n_q_heads * D              */
  const void *w_head;       /* dev bf16 [2, W]: row 0 = yes, row 1 = no    */
  float rms_eps;            /* >= 0, finite                                 */
  float *logits;            /* dev fp32 [P, 2] (l_yes, l_no), or NULL      */
  float *score;             /* dev fp32 [P]                                 */
} dopr_score_head_t;

dopr_status_t dopr_prefix_attn_score_workspace(dopr_store_t st,
                                               const dopr_attn_args_t *args,
                                               size_t *bytes);

dopr_status_t dopr_prefix_attn_score(dopr_store_t st, int32_t layer,
                                     const dopr_attn_args_t *args,
                                     const dopr_score_head_t *head,
                                     void *stream);

/* ------------------------------------------------------------------------ */
/* One decoder layer of the online pass (Sec. 3.4: only [q; t_score] runs
 * through the reranker, every layer's attention also seeing the stored
 * prefix states).  The layer is the Qwen3 decoder layer, in the stored-weight
 * convention y = x W^T with W [out, in]:
 *   h  = RMSNorm(x) * attn_norm_w
 *   q, k, v = h w_q^T, h w_k^T, h w_v^T          (then as dopr_prefix_attn)
 *   x2 = x + attention(q, k, v) w_o^T
 *   h2 = RMSNorm(x2) * mlp_norm_w
 *   y  = x2 + (SiLU(h2 w_gate^T) * (h2 w_up^T)) w_down^T
 * RMSNorm is over the hidden width with epsilon rms_eps of the batch args.
 * Projections accumulate in fp32 and every activation between steps is
 * stored as bf16.  The batch is described by a dopr_attn_args_t whose q, k,
 * v and out must be NULL (the layer forms them in its workspace); lse may be
 * given ([Ntok, Hq]); workspace and workspace_bytes come from
 * dopr_decoder_layer_workspace.  x and y may be the same buffer.           */
typedef struct {
  int32_t hidden;            /* W, multiple of 8                            */
  int32_t intermediate;      /* I, multiple of 8                            */
  const void *attn_norm_w;   /* dev bf16 [W]                                */
  const void *w_q;           /* dev bf16 [Hq*D, W]                          */
  const void *w_k;           /* dev bf16 [Hkv*D, W]                         */
  const void *w_v;           /* dev bf16 [Hkv*D, W]                         */
  const void *w_o;           /* dev bf16 [W, Hq*D]                          */
  const void *mlp_norm_w;    /* dev bf16 [W]                                */
  const void *w_gate;        /* dev bf16 [I, W]                             */
  const void *w_up;          /* dev bf16 [I, W]                             */
  const void *w_down;        /* dev bf16 [W, I]                             */
  const void *x;             /* dev bf16 [Ntok, W] entering the layer       */
  void *y;                   /* dev bf16 [Ntok, W] leaving it               */
} dopr_layer_args_t;

dopr_status_t dopr_decoder_layer_workspace(dopr_store_t st,
                                           const dopr_attn_args_t *batch,
                                           const dopr_layer_args_t *lw,
                                           size_t *bytes);

dopr_status_t dopr_decoder_layer(dopr_store_t st, int32_t layer,
                                 const dopr_attn_args_t *batch,
                                 const dopr_layer_args_t *lw, void *stream);

/* ------------------------------------------------------------------------ */
/* ------------------------------------------------------------------------ */
/* Offline salience selection (Sec. 3.2.1, applied offline in Sec. 3.3): for
 * each document, independently encoded at positions 0..n_d-1, with the final
 * layer's queries q^ and keys k^ as they enter the attention product (after
 * any norm and rotary embedding), q head h reading kv head h / n_rep:
 *   A_h[j, i] = softmax over i <= j of softmax_scale * q^_h[j] . k^_g[i]
 *   Abar      = mean of A_h over the Hq query heads (row j attends,
 *               column i is attended; zero above the diagonal)
 *   u_i       = mean of the m = min(p, n_d - i) largest Abar[j, i] over the
 *               visible rows j >= i (the paper's |T_p| = min(p, n - i + 1)
 *               with 1-based i)
 *   selected  = the K_d positions with the largest u, ties to the lower
 *               position, written in ascending position order.
 * The GPU computes logits in fp32 from the bf16 operands, probabilities
 * with exp2 against each row's log-sum-exp, Abar and u in fp32.           */
#define DOPR_SALIENCE_MAX_LEN 4096
#define DOPR_SALIENCE_MAX_P 64

typedef struct {
  int32_t n_docs;            /* documents in the batch (>= 0)              */
  int32_t max_doclen;        /* M: bound on every n_d, 1..4096             */
  int32_t n_q_heads;         /* Hq, multiple of n_kv_heads                 */
  int32_t n_kv_heads;        /* Hkv >= 1                                   */
  int32_t top_p;             /* p, 1..64                                   */
  float softmax_scale;       /* e.g. 1/sqrt(D); finite and > 0             */
  int64_t total_tokens;      /* Ntok = cu_doclens[n_docs]                  */
  int64_t total_select;      /* cu_select[n_docs] (ignored if selected is
                                NULL)                                      */
  const int32_t *cu_doclens; /* dev int32 [n_docs+1]: document d owns token
                                rows cu[d] .. cu[d+1]-1, 1 <= n_d <= M    */
  const int32_t *cu_select;  /* dev int32 [n_docs+1]: K_d = cs[d+1]-cs[d],
                                0 <= K_d <= n_d; or NULL with selected    */
  const void *q;             /* dev bf16 [Ntok, Hq, D]                     */
  const void *k;             /* dev bf16 [Ntok, Hkv, D]                    */
  float *u;                  /* dev fp32 [Ntok]: salience of every token
                                (output of dopr_salience, input of
                                dopr_select_top_k)                         */
  int32_t *selected;         /* dev int32 [total_select]: doc d's chosen
                                positions (0-based within the document) at
                                cs[d] .., ascending; or NULL (u only)     */
  float *attn_mean;          /* optional dev fp32 [n_docs, M, M]: Abar of
                                doc d at d*M*M + j*M + i; only i <= j < n_d
                                is written.  NULL: kept in the workspace  */
  int32_t *status;           /* optional dev int32, zeroed by the caller:
                                receives DOPR_ERR_SEQLEN when cu_doclens or
                                cu_select is malformed (the affected
                                documents are skipped), else untouched    */
  void *workspace;           /* dev scratch >= dopr_salience_workspace()   */
  size_t workspace_bytes;
} dopr_salience_args_t;

/* Workspace bytes for these arguments (host): the row log-sum-exp of every
 * (token, q head), eight partial maxima of the key norms of every
 * (document, kv head) and,
 * unless attn_mean is given, Abar for as many documents at a time as fit
 * in 1 GiB (at least one).  dopr_salience accepts any workspace that holds
 * the row statistics and key norms plus one document's Abar (4 M^2 bytes)
 * and processes as many documents per pass as fit. */
dopr_status_t dopr_salience_workspace(const dopr_salience_args_t *args,
                                      size_t *bytes);

/* Salience u of every token and, if selected is not NULL, the top-K_d
 * positions of every document.  Asynchronous on `stream`. */
dopr_status_t dopr_salience(const dopr_salience_args_t *args, void *stream);

/* The selection step alone, on u given by the caller: uses n_docs,
 * max_doclen, total_tokens, total_select, cu_doclens, cu_select, u,
 * selected and status; values order as IEEE-754 totalOrder (-0 < +0),
 * ties to the lower position.  No workspace. */
dopr_status_t dopr_select_top_k(const dopr_salience_args_t *args,
                                void *stream);

/* ------------------------------------------------------------------------ */
/* Operators of a decoder layer around its attention: rows in 8-bit integers,
 * products of 8-bit integer matrices, the norms around a gated residual, and
 * rotary positions.  They make up a layer with 8-bit products (the weights
 * take half the bytes of bf16 and the matrix cores run at twice the rate),
 * layers of other families than the one dopr_decoder_layer runs, and the
 * prefix keys that dopr_store_put takes (Sec. 3.3: the selected states are
 * forwarded as prefix inputs and their keys and values kept).
 *
 * Activations are bf16, fp16 or fp32 (`dtype`); sums, norms and scales are
 * held in fp32 or wider, and what comes out is rounded to its type, to nearest
 * even, behind that arithmetic.  Strides are in elements; rows may start at
 * any element-aligned address and lie any distance of at least their length
 * apart.  Everything is asynchronous on `stream`, and outputs do not vary
 * from run to run.                                                         */
typedef enum { DOPR_BF16 = 0, DOPR_F16 = 1, DOPR_F32 = 2 } dopr_dtype_t;

/* Rows in 8-bit integers: v = x, or SiLU(x) * up when `up` is given; with
 * a = max(max_k |v[k]|, 127 * 2^-126) of a row,
 *   scale = a / 127,  q[k] = round-to-nearest-even(v[k] * (127 / a)),
 * each operation in fp32, so |q| <= 127 and v ~ q * scale.  A row of zeros
 * has q = 0.  A row with a value that is not finite has q = 0 and scale NaN,
 * so that every product with it is NaN.  Weights [out, in] are quantised per
 * output channel by the same call.                                         */
typedef struct {
  int32_t dtype;            /* of x and up                                  */
  int64_t rows;             /* >= 0                                         */
  int64_t width;            /* 8 .. 65536                                   */
  const void *x;            /* dev [rows, width]                            */
  int64_t x_row_stride;
  const void *up;           /* dev [rows, width] or NULL                    */
  int64_t up_row_stride;
  int8_t *q;                /* dev [rows, width]                            */
  int64_t q_row_stride;
  float *scale;             /* dev fp32 [rows]                              */
} dopr_quantize_args_t;

dopr_status_t dopr_quantize_rows(const dopr_quantize_args_t *args,
                                 void *stream);

/* Product of 8-bit integer matrices with a scale per row and per column, in
 * the stored-weight convention (w is [out, in]):
 *   y[m, n] = (sum_k x[m, k] w[n, k]) * x_scale[m] * w_scale[n]
 *             + bias[n] + residual[m, n]
 * The integer sum is exact (32 bits); it goes to fp32, where the two scales,
 * bias and residual follow in this order.  y may be the residual (same address
 * and stride).  The bytes between a row's end and its stride are never
 * read.  Rows on 16-byte addresses (x, w and both strides multiples of 16,
 * the strides under 2^22) are multiplied where they lie; others are first
 * laid out again in the workspace, if there is one, else multiplied by a
 * slower kernel (the results are the same).                                */
typedef struct {
  int32_t dtype;            /* of bias, residual and y                      */
  int64_t rows;             /* M >= 0                                       */
  int64_t cols;             /* N >= 0                                       */
  int64_t depth;            /* K, 0 .. 131071                               */
  const int8_t *x;          /* dev [M, K]                                   */
  int64_t x_row_stride;
  const float *x_scale;     /* dev fp32 [M]                                 */
  const int8_t *w;          /* dev [N, K]                                   */
  int64_t w_row_stride;
  const float *w_scale;     /* dev fp32 [N]                                 */
  const void *bias;         /* dev [N] or NULL                              */
  const void *residual;     /* dev [M, N] or NULL                           */
  int64_t residual_row_stride;
  void *y;                  /* dev [M, N]                                   */
  int64_t y_row_stride;
  void *workspace;          /* dev scratch, 256-byte aligned, or NULL: used
                               for rows off 16-byte addresses when it holds
                               (rows + cols) * (depth rounded up to 128)
                               bytes                                        */
  size_t workspace_bytes;
} dopr_quant_matmul_args_t;

/* Workspace bytes worth giving a product (host arithmetic): 0 up to 16 rows,
 * and where the rows lie on 16-byte addresses.  It goes by rows, cols and
 * depth, and by x, w and their strides where they are set: a stride of 0
 * stands for rows back to back, a NULL x or w for an aligned one.  Strides of
 * 2^22 bytes and more count as off 16-byte addresses.                      */
dopr_status_t dopr_quant_matmul_workspace(const dopr_quant_matmul_args_t *args,
                                          size_t *bytes);

dopr_status_t dopr_quant_matmul(const dopr_quant_matmul_args_t *args,
                                void *stream);

/* The norms on either side of a block, fused with its gate and residual:
 *   n = RMSNorm(x) * post_norm_w       (x itself when post_norm_w is NULL)
 *   h = residual_scale * residual + gate * n   (either factor left out when
 *                                               its pointer is NULL)
 *   z = RMSNorm(h) * pre_norm_w        (h itself when pre_norm_w is NULL)
 * x is a block's output, h the residual stream behind it and z the next
 * block's input.  RMSNorm is over the row with epsilon rms_eps.  Outputs: h,
 * and z as dtype (`z`) and / or in 8 bits (`q`, `q_scale`, as
 * dopr_quantize_rows makes them from the unrounded z); at least one.  The
 * second norm reads h before its rounding to residual_dtype.  h may be the
 * residual or x (same address, stride and type), z may be x.               */
typedef struct {
  int32_t dtype;            /* of x, post_norm_w, gate, pre_norm_w and z    */
  int32_t residual_dtype;   /* of residual and h: dtype or DOPR_F32         */
  int64_t rows;             /* >= 0                                         */
  int64_t width;            /* 8 .. 65536                                   */
  const void *x;            /* dev [rows, width]                            */
  int64_t x_row_stride;
  const void *post_norm_w;  /* dev [width] or NULL                          */
  const void *gate;         /* dev [rows, width], or [width] with
                               gate_row_stride 0 (one for all rows), or
                               NULL                                         */
  int64_t gate_row_stride;
  const void *residual;     /* dev [rows, width] or NULL                    */
  int64_t residual_row_stride;
  const void *pre_norm_w;   /* dev [width] or NULL                          */
  float residual_scale;     /* finite                                       */
  float rms_eps;            /* finite, >= 0                                 */
  void *h;                  /* dev [rows, width] or NULL                    */
  int64_t h_row_stride;
  void *z;                  /* dev [rows, width] or NULL                    */
  int64_t z_row_stride;
  int8_t *q;                /* dev [rows, width] or NULL                    */
  int64_t q_row_stride;
  float *q_scale;           /* dev fp32 [rows], with q                      */
} dopr_norm_residual_args_t;

dopr_status_t dopr_norm_residual(const dopr_norm_residual_args_t *args,
                                 void *stream);

/* Rotary positions of query and key heads.  With R = rotary_dim and
 * t = positions[row] * inv_freq[i], pair i < R/2 of a head, (a, b) =
 * (x[i], x[i + R/2]), or (x[2i], x[2i + 1]) when `interleaved`, becomes
 *   attention_factor * (a cos t - b sin t, b cos t + a sin t)
 * (`inverse`: t -> -t); x[R ..] passes through.  With a norm gain, the
 * head's RMSNorm over all of head_dim, times the gain, comes first
 * (dopr_prefix_attn's order).  A prefix attention of heads that are already
 * normed and rotated takes both gains NULL and rope_inv_freq all zero.
 * Outputs may be the inputs (same addresses and strides); other overlaps
 * are not allowed.  Heads lie head_stride apart, so a head-major layout or
 * the q and k parts of one projection's rows are read as they are.         */
typedef struct {
  int32_t dtype;
  int32_t n_q_heads;        /* >= 0                                         */
  int32_t n_kv_heads;       /* >= 0                                         */
  int32_t head_dim;         /* D, 2 .. 512                                  */
  int32_t rotary_dim;       /* R, even, 2 .. D                              */
  int32_t interleaved;      /* 0 or 1                                       */
  int32_t inverse;          /* 0 or 1; 1 takes no norm gains                */
  float attention_factor;   /* finite                                       */
  float rms_eps;            /* finite, >= 0                                 */
  int64_t rows;             /* tokens >= 0                                  */
  const int32_t *positions; /* dev int32 [rows]                             */
  const float *inv_freq;    /* dev fp32 [R/2]                               */
  const void *q;            /* dev [rows, n_q_heads, D]; NULL with 0 heads  */
  int64_t q_row_stride, q_head_stride;
  void *q_out;
  int64_t q_out_row_stride, q_out_head_stride;
  const void *k;            /* dev [rows, n_kv_heads, D]                    */
  int64_t k_row_stride, k_head_stride;
  void *k_out;
  int64_t k_out_row_stride, k_out_head_stride;
  const void *q_norm_w;     /* dev [D] or NULL                              */
  const void *k_norm_w;     /* dev [D] or NULL                              */
} dopr_rotary_args_t;

dopr_status_t dopr_rotary(const dopr_rotary_args_t *args, void *stream);

/* Rotation frequencies for contexts longer than the trained one.  With
 * w_i = theta^(-2i/R), i < R/2, and s = factor:
 *   DOPR_ROPE_PLAIN   w_i
 *   DOPR_ROPE_LINEAR  w_i / s
 *   DOPR_ROPE_BASE    (theta * s^(R/(R-2)))^(-2i/R): the base is stretched so
 *                     that the slowest pair turns s times slower (R > 2)
 *   DOPR_ROPE_RAMP    w_i (g_i + (1 - g_i) / s), g_i = 1 for pairs that turn
 *                     at least turns_high times within original_len, 0 for
 *                     at most turns_low, linear in the pair's index between
 *                     the two (real-valued) indices where the turns are met.
 *                     Implementations that round these two outward to whole
 *                     indices have other frequencies in between: a model that
 *                     was trained with such ones brings its own inv_freq
 *   DOPR_ROPE_BANDS   the same with g_i linear in the number of turns
 * *attention_factor receives 0.1 ln s + 1 for RAMP with s > 1, else 1.
 * Host arithmetic in 64 bits; inv_freq is a HOST array of R/2 floats.      */
typedef enum {
  DOPR_ROPE_PLAIN = 0,
  DOPR_ROPE_LINEAR = 1,
  DOPR_ROPE_BASE = 2,
  DOPR_ROPE_RAMP = 3,
  DOPR_ROPE_BANDS = 4
} dopr_rope_scaling_t;

dopr_status_t dopr_rotary_frequencies(int32_t rotary_dim, double theta,
                                      dopr_rope_scaling_t scaling,
                                      double factor, double original_len,
                                      double turns_low, double turns_high,
                                      float *inv_freq,
                                      float *attention_factor);

/* ------------------------------------------------------------------------ */
/* Exports used by the bit-exact tests of the integer steps.               */

/* Doc-id grouping (Sec. 3.4 with Sec. 4.5.2: the pairs that retrieve the
 * same document share its stored prefix, so they are batched by document)
 * in canonical form: valid pairs (doc id in range and
 * resident) sorted by (doc id, pair index).  group_doc[G] ascending doc ids,
 * group_ptr[G+1] offsets into pair_order[], pair_order[n_valid] pair indices.
 * Capacities: group_doc and pair_order >= n_pairs, group_ptr >= n_pairs+1.
 * `workspace` must hold dopr_prefix_attn_workspace() bytes for the same
 * pairs.  Synchronises `stream` to return *n_groups and *n_valid on the host. */
dopr_status_t dopr_group_pairs(dopr_store_t st, int32_t n_pairs,
                               const int32_t *doc_ids, void *workspace,
                               size_t workspace_bytes, int32_t *n_groups,
                               int32_t *n_valid, int32_t *group_doc,
                               int32_t *group_ptr, int32_t *pair_order,
                               void *stream);

/* Gather the prefix K/V states of doc_ids[i] for one layer out of the store
 * (Sec. 3.4: a candidate's stored prefix states are fetched by its id)
 * into canonical layout: k_out/v_out dev bf16 [out_cu_slots[n], Hkv, D],
 * pair i's slots at rows out_cu_slots[i] .. out_cu_slots[i+1]-1.  A bad doc
 * id, or a slot range that differs from L_d, leaves its rows untouched and
 * raises a deferred DOC_RANGE.                                             */
dopr_status_t dopr_gather_prefix(dopr_store_t st, int32_t layer, int32_t n,
                                 const int32_t *doc_ids,
                                 const int64_t *out_cu_slots, void *k_out,
                                 void *v_out, void *stream);

/* ------------------------------------------------------------------------ */
/* Status (library plumbing; no passage of the paper defines it).          */

/* Synchronise `stream`, then return (and clear) the first deferred device
 * error raised by calls on this store since the last check, else DOPR_OK.  */
dopr_status_t dopr_check_status(dopr_store_t st, void *stream);

/* Human-readable name of a status code (static string). */
const char *dopr_status_str(dopr_status_t s);

/* Thread-local text describing the last non-OK status returned on this
 * thread ("" if none). */
const char *dopr_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* DOPR_H */
