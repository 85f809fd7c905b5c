/*
 * libsdsat -- the SDSAT block decode step on one GB300 (sm_103a).
 *
 * SDSAT ("Speculative Decoding with Semantic Adaptive Tokens", arXiv
 * 2403.18647) decodes with an unmodified Llama-architecture model in loops of
 * "two-step-draft-then-verify" (Sec. 2.1):
 *
 *   draft step 1 (Eq. 1)  block [last token, a_1 .. a_k]  -> y_{n+1} and k drafts
 *   draft step 2 (Eq. 2)  block [y_{n+1}, d_1 .. d_k]     -> targets t_0 .. t_k
 *   verification (Eq. 3)  accept t_0 .. t_m, m = leading matches d_i == t_{i-1}
 *
 * Each step is one pass of q = k + 1 positions through every layer
 * (sdsat_block_forward), then target selection, verification and KV commit
 * (sdsat_accept_greedy / sdsat_accept_nucleus).  The loop emits 2 + m tokens
 * for two passes (Sec. 2.1.1).
 *
 * Conventions for every entry point
 * ---------------------------------
 *  - Pointers named *_dev are CUDA device pointers owned by the caller; they
 *    must stay valid until the work queued on the context stream has run.
 *  - All compute calls are asynchronous on the context stream
 *    (sdsat_set_stream); only sdsat_create, sdsat_kv_create, sdsat_*_destroy
 *    and sdsat_get_error synchronise.  No compute call allocates memory, so
 *    compute calls may be captured into a CUDA graph.
 *  - The calls of a context share its workspaces (partial results, operands, the
 *    error word): calls queued on two streams must not overlap.  Order the streams
 *    by an event, or use a context for each.
 *  - Argument errors are detected on the host and returned synchronously
 *    (nothing is queued).  Errors only the device can see (a NaN logit, a
 *    row past the KV capacity, a timed-out wait) set bits in a device flag
 *    word read by sdsat_get_error.
 *  - Weights are bf16, row-major [out_features, in_features] (the layout of
 *    nn.Linear.weight), 16-byte aligned, in_features a multiple of 8.
 *  - Activations and logits are fp32; token ids int32.
 */
#ifndef SDSAT_H
#define SDSAT_H

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define SDSAT_API __attribute__((visibility("default")))
#else
#define SDSAT_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SDSAT_OK = 0,
  SDSAT_EINVAL = 1,        /* bad argument: null/misaligned pointer, size out of range */
  SDSAT_ENOMEM = 2,        /* device allocation failed (create calls only) */
  SDSAT_ECAPACITY = 3,     /* batch, q, position or KV capacity limit exceeded */
  SDSAT_ECUDA = 4,         /* a CUDA runtime or driver call failed */
  SDSAT_EDEVICE = 5,       /* device-detected error bits were set (sdsat_get_error) */
  SDSAT_EUNSUPPORTED = 6   /* a configuration this library does not implement */
} sdsat_status;

/* device error bits reported by sdsat_get_error */
#define SDSAT_DEV_NAN_LOGITS 0x1u  /* NaN logit seen; it counted as -inf */
#define SDSAT_DEV_TIMEOUT 0x2u     /* a bounded in-kernel wait expired; results invalid */
#define SDSAT_DEV_CAPACITY 0x4u    /* a row fell past the KV capacity, or has no page of its own; not written */
#define SDSAT_DEV_TOKEN 0x8u       /* a token id outside [0, vocab); id 0 used instead */
#define SDSAT_DEV_POSITION 0x10u   /* a RoPE position outside [0, max_position); clamped */
#define SDSAT_DEV_TREE 0x20u       /* a tree parent that is not an earlier row; read as the root */
#define SDSAT_DEV_PAGE 0x40u       /* a slot to attend to without a page, a page number outside the pool or a
                                      sequence to fork from outside the batch; skipped */

#define SDSAT_MAX_Q 16           /* block rows per sequence (k <= 15 adaptive tokens) */
#define SDSAT_MAX_ROWS 64        /* batch * q rows per block forward */
#define SDSAT_MAX_ADAPTIVE 16
#define SDSAT_PAGE 64            /* slots of a page of a paged cache */

/* element types of the kernels that take more than one */
#define SDSAT_FP32 0
#define SDSAT_BF16 1

typedef struct sdsat_ctx sdsat_ctx;
typedef struct sdsat_kv sdsat_kv;

/* Model and decoding configuration (Llama architecture; Sec. 3 uses CodeLlama). */
typedef struct {
  int32_t n_layers;
  int32_t d_model;
  int32_t n_heads;
  int32_t n_kv_heads;      /* must equal n_heads (this library has no grouped-query attention) */
  int32_t head_dim;        /* 64 or 128 */
  int32_t ffn_dim;         /* SwiGLU hidden size */
  int32_t vocab;           /* including the semantic adaptive tokens (Sec. 3.2: ordinary ids) */
  float rms_eps;
  float rope_theta;        /* RoPE base; rotate-half pairing (i, i + head_dim/2) */
  int32_t max_position;    /* RoPE table length: every position must be < max_position */
  int32_t n_adaptive;      /* 1: adaptive_ids[0] repeated k times (recommended, App. B);
                              >1: k distinct ids a_1..a_k (SDSAT-D, App. B) */
  int32_t adaptive_ids[SDSAT_MAX_ADAPTIVE];
} sdsat_config;

/* Per-layer weights (device pointers, borrowed: the caller keeps them alive). */
typedef struct {
  const void* attn_norm;   /* bf16 [d] */
  const void* wq;          /* bf16 [H*hd, d] */
  const void* wk;          /* bf16 [H*hd, d] */
  const void* wv;          /* bf16 [H*hd, d] */
  const void* wo;          /* bf16 [d, H*hd] */
  const void* ffn_norm;    /* bf16 [d] */
  const void* w_gate;      /* bf16 [F, d] */
  const void* w_up;        /* bf16 [F, d] */
  const void* w_down;      /* bf16 [d, F] */
} sdsat_layer_weights;

typedef struct {
  const void* embed;                    /* bf16 [V, d] */
  const void* final_norm;               /* bf16 [d] */
  const void* lm_head;                  /* bf16 [V, d] (untied) */
  const sdsat_layer_weights* layers;    /* host array of n_layers entries (copied) */
} sdsat_weights;

/* ---- lifetime ----------------------------------------------------------------- */

/* Validate `cfg`, record the weight pointers, build the TMA descriptors and the
 * RoPE table, allocate the library-owned workspaces.  The model is the unmodified
 * decoder the method runs (Abstract, Sec. 1: no structural change; Sec. 3.2: the
 * adaptive tokens are ordinary vocabulary ids), so the configuration is a plain
 * Llama configuration plus the adaptive ids; the paper prescribes no interface for
 * it.  `stream` is a cudaStream_t (NULL = legacy default stream).  Synchronous.  Errors: EINVAL (bad config or
 * pointer), EUNSUPPORTED (head_dim, GQA), ENOMEM, ECUDA.
 * Environment: SDSAT_NO_PDL=1 (read at each create) launches this context's kernels
 * without programmatic dependent launch, for tools that cannot follow it;
 * SDSAT_ATT_CLUSTER_MAX=n (read at the first create of the process) caps the
 * attention's thread-block cluster size at n in 1..16 for tuning sweeps (default
 * 16; the size itself is chosen per launch). */
SDSAT_API sdsat_status sdsat_create(const sdsat_config* cfg, const sdsat_weights* w, void* stream,
                          sdsat_ctx** out);
SDSAT_API void sdsat_destroy(sdsat_ctx* ctx);

/* Stream for all later compute calls on ctx (a cudaStream_t). */
SDSAT_API sdsat_status sdsat_set_stream(sdsat_ctx* ctx, void* stream);

/* Library-owned KV cache for `batch` sequences of up to `max_len` slots (the cache
 * that Eq. 1 and Eq. 2 extend by q positions per pass and that Sec. 2.1.1's
 * verification truncates to the accepted prefix; the paper states no layout):
 * K and V bf16 [n_layers][batch][n_heads][max_len][head_dim], and the committed
 * length len[batch] (int32, device, starts at 0).  Synchronous.
 * Errors: EINVAL, ENOMEM, ECAPACITY (max_len > max_position or > 32768). */
SDSAT_API sdsat_status sdsat_kv_create(sdsat_ctx* ctx, int batch, int max_len, sdsat_kv** out);
SDSAT_API void sdsat_kv_destroy(sdsat_kv* kv);

/* A paged KV cache, for many samples of one prompt: `n_pages` pages of SDSAT_PAGE slots
 * (every layer and head of them), K and V bf16
 * [n_layers][n_pages][n_heads][SDSAT_PAGE][head_dim], handed out to `batch` sequences of up
 * to `max_len` slots each, which may share pages.  Every call that takes a cache takes a
 * paged one, with two differences: the slots that a call writes (block rows, a prompt,
 * sdsat_kv_write) need pages that their sequence alone holds (sdsat_kv_reserve), and a row
 * without one is not written and sets device bit CAPACITY (sdsat_prefill, and an accept call
 * with commit, leave the length as it was where a row that they would commit has none;
 * sdsat_kv_commit sets any length); and block forwards read the whole, committed leading
 * pages that all their sequences hold together with sequence 0 once for all of them.  One
 * sequence of the batch with another prompt, or without pages, and none are: several
 * prompts' samples share most in a call for each.
 * Synchronous.  Errors: EINVAL (batch > 256), ENOMEM, ECAPACITY (as sdsat_kv_create),
 * EUNSUPPORTED (n_layers * n_pages * n_heads * SDSAT_PAGE >= 2^31). */
SDSAT_API sdsat_status sdsat_kv_create_paged(sdsat_ctx* ctx, int batch, int max_len, int n_pages, sdsat_kv** out);

/* Device addresses and geometry of a paged cache: table int32 [batch][table_ld], entry j of
 * a sequence the page of its slots 64 j .. 64 j + 63 (-1: none), and refs int32 [n_pages],
 * the sequences that hold each page (0: free).  Any output pointer may be NULL.
 * Fork, free and reserve count the pages that sequences share, and block forwards go by that
 * count: after writing to the table (and refs, which has to agree with it) call one of them.
 * Errors: EINVAL (a contiguous cache). */
SDSAT_API sdsat_status sdsat_kv_pages(const sdsat_kv* kv, int32_t** table_dev, int32_t** refs_dev, int* n_pages,
                                      int* table_ld);

/* Sequence s < b takes the pages and the length that sequence src_dev[s] (any sequence of the
 * cache, its own included) had before the call; -1 leaves it empty.  Pages are shared, not
 * copied; a page that no sequence holds any more is free.  src_dev int32 [b].  The emitted
 * counters stay.  Errors: EINVAL; device bit PAGE where src_dev[s] is neither -1 nor in the
 * batch (s keeps its pages), and where a table entry is no page of the pool (dropped). */
SDSAT_API sdsat_status sdsat_kv_fork(sdsat_ctx* ctx, sdsat_kv* kv, const int32_t* src_dev, int b);

/* Sequence seq gives its pages up (length 0).  Errors: EINVAL. */
SDSAT_API sdsat_status sdsat_kv_free(sdsat_ctx* ctx, sdsat_kv* kv, int seq);

/* Give sequences seq .. seq+b-1 pages of their own for the slots len .. len + n - 1, the next
 * rows they write: a missing page is the lowest free one, sequences and then slots in order; a
 * page that other sequences hold too is replaced by the lowest free one, into which its
 * committed slots are copied (of several sequences that hold it the last one keeps it).
 * Errors: EINVAL; device bit CAPACITY where a sequence would pass max_len (it gets the pages up
 * to it) or the pool has too few free pages (nothing changes); PAGE where a table entry is no
 * page of the pool (replaced). */
SDSAT_API sdsat_status sdsat_kv_reserve(sdsat_ctx* ctx, sdsat_kv* kv, int seq, int b, int n);

/* Move the pages in use to the ids 0 .. u-1 of the pool: the i-th used page with an id >= u
 * goes to the i-th free one below u, with the slots that any sequence has committed in it.
 * *used_dev = u (int32, may be NULL).  Errors: EINVAL. */
SDSAT_API sdsat_status sdsat_kv_compact(sdsat_ctx* ctx, sdsat_kv* kv, int32_t* used_dev);

/* Rotary position embedding of a model that the context's own table does not describe: part of a head, pairs side by
 * side, frequencies scaled for long contexts. */
#define SDSAT_ROPE_PLAIN 0
#define SDSAT_ROPE_LINEAR 1      /* f_i / factor (position interpolation) */
#define SDSAT_ROPE_PARTS 2       /* f_i (g_i + (1 - g_i) / factor), g_i = clamp((r_i - low) / (high - low), 0, 1) with
                                    r_i = original f_i / 2 pi, the turns of pair i in the original context */
typedef struct {
  int32_t dims;            /* rotated dimensions of a head, the first ones: even, 2 .. 128; the rest pass through */
  int32_t interleaved;     /* pairs (2 i, 2 i + 1), else (i, i + dims/2), i < dims/2 */
  int32_t max_position;    /* positions 0 .. max_position - 1, at most 2^24 */
  int32_t scaling;         /* SDSAT_ROPE_* */
  int32_t original;        /* PARTS: positions of the context that the model was trained on */
  int32_t reserved;        /* 0, else EINVAL */
  double theta;            /* f_i = theta^(-2 i / dims) radians a position */
  double factor;           /* LINEAR, PARTS */
  double low, high;        /* PARTS: turns up to which a pair is interpolated, and from which on it stays */
  double magnitude;        /* cosines and sines are multiplied by it (1: none) */
} sdsat_rope_config;
typedef struct sdsat_rope sdsat_rope;

/* The cosines and sines of every position and pair, fp32, from angles in double: max_position * dims * 4 bytes.
 * Synchronous.  The calls of its context take it; it may be destroyed before or after that.
 * Errors: EINVAL (a field out of its range), ENOMEM, ECUDA. */
SDSAT_API sdsat_status sdsat_rope_create(sdsat_ctx* ctx, const sdsat_rope_config* cfg, sdsat_rope** out);
SDSAT_API void sdsat_rope_destroy(sdsat_rope* rope);

/* Device addresses and geometry of a KV cache (for tests and benches that fill
 * or inspect it).  Any output pointer may be NULL. */
SDSAT_API sdsat_status sdsat_kv_info(const sdsat_kv* kv, void** k_dev, void** v_dev, int32_t** len_dev,
                           int* batch, int* max_len);

/* Copy n rows into / out of the cache of one (layer, sequence), all heads:
 * src / dst are bf16 [n_heads][n][head_dim] device buffers; rows land at slots
 * slot0 .. slot0+n-1.  Asynchronous on the context stream.  Used to load a
 * snapshot (or synthetic contents) and to inspect what a block forward wrote.
 * On a paged cache a slot without a page reads as zeros and sets device bit CAPACITY.
 * Errors: EINVAL (null pointer, layer/seq/slot range, buffers not aligned to their values). */
SDSAT_API sdsat_status sdsat_kv_write(sdsat_ctx* ctx, sdsat_kv* kv, int layer, int seq, int slot0, int n,
                                      const void* k_src_dev, const void* v_src_dev);
SDSAT_API sdsat_status sdsat_kv_read(sdsat_ctx* ctx, const sdsat_kv* kv, int layer, int seq, int slot0, int n,
                                     void* k_dst_dev, void* v_dst_dev);

/* ---- the block decode step ------------------------------------------------------- */

/* One pass of q new positions for sequences 0 .. b-1 through every layer
 * (Eq. 1 and Eq. 2 evaluate P_theta at all q positions of a block at once).
 *
 * tokens_dev     int32 [b*q], row j of sequence s at s*q + j.
 * positions_dev  int32 [b*q] RoPE positions, or NULL for len[s] + j.
 * logits_dev     fp32 [b*q][vocab], written.
 * Block rows are written to KV slots len[s] .. len[s]+q-1 (len is NOT advanced;
 * see the accept calls and sdsat_kv_commit).  Row j attends to slots [0, len[s])
 * and to block rows 0..j.
 * Errors: EINVAL (null pointer, b < 1, b > kv batch, q < 1, q > SDSAT_MAX_Q,
 * b*q > SDSAT_MAX_ROWS); device bit CAPACITY if len[s] + q > max_len. */
SDSAT_API sdsat_status sdsat_block_forward(sdsat_ctx* ctx, sdsat_kv* kv, const int32_t* tokens_dev,
                                 const int32_t* positions_dev, int b, int q, float* logits_dev);

/* Greedy target selection, Eq. 3 verification and KV commit (Sec. 2.1.1).
 *
 * logits_dev        fp32 [b*q][vocab] from sdsat_block_forward.
 * drafts_dev        int32 [b*q]: the block's input tokens; entry s*q + i (1 <= i < q)
 *                   is draft d_i.  Entry s*q is not read.
 * n_verify          number of drafts to verify (0 <= n_verify < q).  0 is draft
 *                   step 1: only t_0 is emitted and rows 1..q-1 return the drafts.
 * out_tokens_dev    int32 [b*q]: t_j = argmax of row j (lowest id on ties; NaN
 *                   counts as -inf and sets device bit NAN_LOGITS), for every j.
 * accepted_len_dev  int32 [b]: 1 + m, the number of emitted tokens t_0 .. t_m,
 *                   m = max{i <= n_verify : d_i' == t_{i'-1} for all i' <= i}.
 * commit            non-zero: len[s] += 1 + m on the device (rejected rows and
 *                   the adaptive positions are rolled back by not committing them).
 * Errors: EINVAL. */
SDSAT_API sdsat_status sdsat_accept_greedy(sdsat_ctx* ctx, sdsat_kv* kv, const float* logits_dev,
                                 const int32_t* drafts_dev, int b, int q, int n_verify,
                                 int32_t* accepted_len_dev, int32_t* out_tokens_dev, int commit);

/* Nucleus (top-p) variant (Sec. 2.1.2, chain form: the accepted branch is the
 * longest verified prefix).  Each row's target is a sample defined exactly so
 * that any two implementations agree bit for bit:
 *   s_i = (l_i - max l) / temperature (fp32), w_i = exp(s_i) (fp32, Cody-Waite
 *   reduction + degree-7 polynomial, every step one rounded operation),
 *   W_i = floor(w_i * 2^24) (exact in 32 bits: the top weight is 2^24, and a
 *   token below 2^-24 of it gets 0);  candidates = the top_k heaviest by
 *   (W desc, id asc) (top_k = 0: all);  kept = the shortest prefix of the
 *   candidates in that order with C * 2^24 >= round(top_p * 2^24) * S;
 *   r = Philox4x32-10(key = rng_seed, counter = (position of the produced
 *   token, s, 0, 0)), 64-bit from its first two words;  tau = (r * S_kept) >> 64;
 *   the sample is the first kept id, ascending, whose inclusive cumulative
 *   weight exceeds tau.
 * The produced token of row j has position len[s] + j + 1.  temperature <= 0
 * selects greedy (Fig. 1: greedy is the special case).  Requires vocab <= 32768.
 * Other arguments as sdsat_accept_greedy.  Errors: EINVAL, EUNSUPPORTED. */
SDSAT_API sdsat_status sdsat_accept_nucleus(sdsat_ctx* ctx, sdsat_kv* kv, const float* logits_dev,
                                  const int32_t* drafts_dev, int b, int q, int n_verify,
                                  float top_p, float temperature, uint64_t rng_seed, int top_k,
                                  int32_t* accepted_len_dev, int32_t* out_tokens_dev, int commit);

/* Explicit commit / rollback (implied by Sec. 2.1.1: after Eq. 3 only the accepted
 * prefix stays in the context; the adaptive positions of draft step 1 and the rejected
 * drafts are dropped): len[s] = new_len_dev[s] for s < b (device values,
 * 0 <= new_len <= max_len; out-of-range values are clamped and set CAPACITY).  On a paged
 * cache committed slots without a page are not attended to (device bit PAGE).
 * Errors: EINVAL (b > the cache's batch). */
SDSAT_API sdsat_status sdsat_kv_commit(sdsat_ctx* ctx, sdsat_kv* kv, const int32_t* new_len_dev, int b);

/* Copy the committed lengths len[0 .. b-1] into lens_dev (int32 [b], device),
 * asynchronously.  Errors: EINVAL. */
SDSAT_API sdsat_status sdsat_kv_lengths(sdsat_ctx* ctx, const sdsat_kv* kv, int32_t* lens_dev, int b);

/* Tokens emitted so far per sequence: every accept call with commit != 0 adds
 * 1 + m to emitted[s] on the device.  Copies emitted[0 .. b-1] into
 * emitted_dev (int64 [b]) and, when reset != 0, zeroes the counters after the
 * copy.  Asynchronous.  Errors: EINVAL. */
SDSAT_API sdsat_status sdsat_kv_emitted(sdsat_ctx* ctx, sdsat_kv* kv, int64_t* emitted_dev, int b, int reset);

/* Build the next block input on the device (the block inputs of Eq. 1 and Eq. 2),
 * so that a whole loop runs without the host:
 *   mode 1 (draft step 1): row 0 = prev_out[s*q + prev_acc[s] - 1] (the newest
 *     emitted token), rows 1..q-1 = the adaptive ids a_1 .. a_{q-1};
 *   mode 2 (draft step 2): row 0 = prev_out[s*q] (y_{n+1}), rows 1..q-1 = the drafts:
 *     prev_out[s*q + j] (the drafts draft step 1 produced), or, when
 *     draft_table_dev is given, draft_table_dev[s*table_stride + len[s] + j]
 *     (a per-position draft source, e.g. a test stub).
 * prev_out_dev / prev_acc_dev are the out_tokens / accepted_len of the previous
 * accept call; tokens_out_dev int32 [b*q] is written.  Errors: EINVAL. */
SDSAT_API sdsat_status sdsat_build_block(sdsat_ctx* ctx, sdsat_kv* kv, int mode, const int32_t* prev_out_dev,
                               const int32_t* prev_acc_dev, const int32_t* draft_table_dev,
                               int table_stride, int b, int q, int32_t* tokens_out_dev);

/* ---- tree-structured draft step 2 (Sec. 2.1.2) ----------------------------------- */
/* A tree block holds q rows per sequence: the nodes of a draft tree in
 * topological order.  parent_dev int32 [b*q]: entry s*q + j is the parent row of
 * row j of sequence s; row 0 is the root (parent -1, the token y_{n+1} of draft
 * step 1) and every other row's parent is an earlier row (parent[j] < j).
 * Anything else sets device bit TREE and the row is read as a child of the root.
 * Row j has depth(j) = number of edges to the root, occupies KV slot len[s] + j
 * and sits at position len[s] + depth(j).  A chain (parent[j] = j - 1) is the
 * ordinary block of sdsat_block_forward / sdsat_accept_*. */

/* Tree block forward: as sdsat_block_forward, with RoPE positions
 * len[s] + depth(j) and the tree attention mask -- row j attends to the committed
 * slots [0, len[s]) and to the slots of its ancestors and itself only.
 * tokens_dev int32 [b*q]; logits_dev fp32 [b*q][vocab], written.  len is not
 * advanced.  Errors: EINVAL (null pointer, b < 1, b > kv batch, q < 1,
 * q > SDSAT_MAX_Q, b*q > SDSAT_MAX_ROWS); device bits TREE, CAPACITY. */
SDSAT_API sdsat_status sdsat_block_forward_tree(sdsat_ctx* ctx, sdsat_kv* kv, const int32_t* tokens_dev,
                                                const int32_t* parent_dev, int b, int q, float* logits_dev);

/* Tree verification and commit (Sec. 2.1.2: the longest branch of the tree that
 * is verified and accepted is the loop's result).
 *   targets  t_j = the selection of sdsat_accept_nucleus (temperature > 0) or
 *            argmax (temperature == 0) of row j's logits, the produced token at
 *            position len[s] + depth(j) + 1;
 *   accepted row 0 always; row j > 0 iff its parent p is accepted and
 *            tokens[s*q + j] == t_p (the chain test of Eq. 3 along each branch);
 *   path     n_0 = 0, n_1, ..., n_m: the root path of the deepest accepted row
 *            (the lowest row index among equally deep ones).
 * out_tokens_dev   int32 [b*q]: t_{n_0} .. t_{n_m}, then -1.
 * accepted_len_dev int32 [b]: 1 + m.
 * path_dev         int32 [b*q]: n_0 .. n_m, then -1; may be NULL.
 * The K and V rows of the path always move to slots len[s] + 1 .. len[s] + m
 * (slot len[s] + i receives row n_i's rows, which were rotated at position
 * len[s] + i already), so the cache holds the accepted branch contiguously;
 * commit != 0 then advances len[s] by 1 + m (with commit == 0, an explicit
 * sdsat_kv_commit of len[s] + 1 + m commits it later).
 * Other arguments as sdsat_accept_nucleus.  Errors: EINVAL (null parent_dev,
 * temperature < 0 or NaN, the sdsat_accept_nucleus conditions), EUNSUPPORTED
 * (temperature > 0 and vocab > 32768); device bit TREE. */
SDSAT_API sdsat_status sdsat_accept_tree(sdsat_ctx* ctx, sdsat_kv* kv, const float* logits_dev,
                                         const int32_t* tokens_dev, const int32_t* parent_dev, int b, int q,
                                         float temperature, float top_p, uint64_t rng_seed, int top_k,
                                         int32_t* accepted_len_dev, int32_t* out_tokens_dev, int32_t* path_dev,
                                         int commit);

/* Block building for tree loops, where consecutive blocks differ in size:
 *   mode 1 (draft step 1): q = k + 1 rows; row 0 = prev_out[s*prev_q + prev_acc[s] - 1],
 *     rows 1..k = the adaptive ids;
 *   mode 2 (draft step 2): the tree of `width` chains of k drafts below the root,
 *     q = 1 + width*k rows (parent of row 1 + w*k is 0, of row 1 + w*k + i is
 *     row w*k + i); row 0 = prev_out[s*prev_q]; row 1 + w*k + i - 1 (1 <= i <= k)
 *     = draft_tables_dev[(w*B + s)*table_stride + len[s] + i] with B the KV batch
 *     (branch w's draft for position len[s] + i).  Without tables (width 1 only)
 *     row i = prev_out[s*prev_q + i] (k < prev_q).
 * tokens_out_dev int32 [b*q].  Errors: EINVAL (q > SDSAT_MAX_Q, b*q > SDSAT_MAX_ROWS,
 * table_stride < max_len + SDSAT_MAX_Q, the sdsat_build_block conditions). */
SDSAT_API sdsat_status sdsat_build_tree_block(sdsat_ctx* ctx, sdsat_kv* kv, int mode, const int32_t* prev_out_dev,
                                              int prev_q, const int32_t* prev_acc_dev,
                                              const int32_t* draft_tables_dev, int width, int table_stride, int b,
                                              int k, int32_t* tokens_out_dev);

/* ---- pipelined variant (not a step of the paper) ---------------------------------- */
/* The verification block also carries the k adaptive tokens, so that a loop whose
 * drafts are all accepted needs no separate draft step 1.  Every block has
 * q = 2k + 1 rows [x_0, r_1 .. r_k, a_1 .. a_k] at slots len[s] .. len[s] + 2k:
 *   mode A (drafts known): r_i = the drafts for positions len[s] + i; Eq. 3 verifies
 *     them; if all k are accepted, the adaptive rows' targets are the next block's
 *     drafts and the next block is mode A again, otherwise it is mode S;
 *   mode S: r_i = a_i (the block is draft step 1 with k extra adaptive rows), nothing
 *     is verified, t_0 is emitted and t_1 .. t_k are the next block's drafts (mode A).
 * The emitted tokens are those of the two-step loop (and of plain decoding under greedy
 * selection or the position-keyed sampler). */

/* Build the next pipelined block on the device from the previous one's accept outputs:
 *   prev_out_dev int32 [b*(2k+1)], prev_acc_dev int32 [b]: the previous accept call's
 *     out_tokens and accepted_len (before the first block: out[s*(2k+1)] = the newest
 *     prompt token, acc = 1, mode = 1);
 *   mode_dev int32 [b], in: the previous block's mode (0 S, 1 A), out: this block's;
 *   n_verify_dev int32 [b], out: k for mode A, 0 for mode S (for sdsat_accept_pipelined);
 *   draft_table_dev: optional per-position drafts, [s*table_stride + len[s] + i] for
 *     row i of a mode-A block (the harness's stub); otherwise the previous targets.
 * x_0 = prev_out[s*(2k+1) + acc - 1]; mode A's drafts without a table are
 * prev_out[s*(2k+1) + acc .. + acc + k - 1].  tokens_out_dev int32 [b*(2k+1)].
 * Errors: EINVAL (null pointer, 2k + 1 > SDSAT_MAX_Q, b*(2k+1) > SDSAT_MAX_ROWS,
 * table_stride < max_len + SDSAT_MAX_Q). */
SDSAT_API sdsat_status sdsat_build_pipelined_block(sdsat_ctx* ctx, sdsat_kv* kv, const int32_t* prev_out_dev,
                                                   const int32_t* prev_acc_dev, int32_t* mode_dev,
                                                   int32_t* n_verify_dev, const int32_t* draft_table_dev,
                                                   int table_stride, int b, int k, int32_t* tokens_out_dev);

/* Target selection (argmax for temperature == 0, else the sampler of
 * sdsat_accept_nucleus), Eq. 3 verification of n_verify_dev[s] drafts per sequence
 * (device values, clamped to [0, q-1]) and the KV commit, as sdsat_accept_nucleus.
 * Errors: EINVAL (null n_verify_dev, temperature < 0 or NaN, q < 2, the
 * sdsat_accept_nucleus conditions), EUNSUPPORTED. */
SDSAT_API sdsat_status sdsat_accept_pipelined(sdsat_ctx* ctx, sdsat_kv* kv, const float* logits_dev,
                                              const int32_t* tokens_dev, const int32_t* n_verify_dev, int b, int q,
                                              float temperature, float top_p, uint64_t rng_seed, int top_k,
                                              int32_t* accepted_len_dev, int32_t* out_tokens_dev, int commit);

/* Run n prompt tokens of sequence `seq` through the model and commit them
 * (len[seq] += n): the step before the decode loop (Sec. 2.1.1 starts from a prompt
 * y_1 .. y_n already in the context; the paper gives the prefill no further detail).  Equal chunks of
 * at most 4096 positions (at most max_position rounded up to 128) go through the layers one
 * after the other (the weights stream once per chunk), position i attending to every earlier
 * position.  No logits are produced.  The workspaces of the largest chunk belong to the context
 * (sdsat_create allocates them with the weights): per position 8 d_model + 8 R + 4 ffn_dim bytes
 * and 4 bytes per 128 of d_model, R = n_heads * head_dim; 449 MB for a 7B context, 563 MB at 13B,
 * of max_position 4096 or more.
 * Errors: EINVAL (null pointer, seq outside the KV batch, n < 0), ECAPACITY
 * (n > max_len); device bit CAPACITY if len[seq] + n > max_len. */
SDSAT_API sdsat_status sdsat_prefill(sdsat_ctx* ctx, sdsat_kv* kv, int seq, const int32_t* tokens_dev, int n);

/* Synchronise the context stream, return the accumulated device error bits in
 * *flags (SDSAT_DEV_*) and clear them.  Returns EDEVICE if any bit was set,
 * ECUDA if the stream reported a CUDA error. */
SDSAT_API sdsat_status sdsat_get_error(sdsat_ctx* ctx, uint32_t* flags);

/* A static, NUL-terminated English name of a status code ("ok", "invalid argument", ...;
 * unknown codes give "unknown status").  Host only, never fails.  The paper has no
 * counterpart: it is the error reporting of this library's boundary. */
SDSAT_API const char* sdsat_status_string(sdsat_status s);

/* ---- single kernels (unit parity tests and kernel sweeps) ------------------------- */

/* y[m][n] = sum_k x[m][k] * W[n][k] for m < M, n < N.  M <= 32 runs the weight-streaming
 * skinny GEMM of the block forward, 32 < M <= 512 (and 24 < M <= 32 for narrow W of more than 512
 * columns and wide W of more than 1024) the tiled GEMM of wider blocks and of the prefill path (256 weight rows x 64 or 128 positions per
 * tile of a CTA pair).  x fp32
 * [M][K] (row stride K), W bf16 [N][K], y fp32 [M][N]; x and W 16-byte aligned,
 * K a multiple of 8, K <= 32768.  Errors: EINVAL. */
SDSAT_API sdsat_status sdsat_op_gemm(sdsat_ctx* ctx, const float* x_dev, int M, int K, const void* w_dev, int N,
                           float* y_dev);

/* Block-causal attention of q query rows per sequence against a bf16 cache:
 * out[s*q+j][h*hd+d] = sum_t softmax_t(q_j . k_t / sqrt(hd)) v_t[d] over slots
 * t < len[s] + j + 1.  q_dev fp32 [b*q][H*hd]; k_dev, v_dev bf16
 * [b][H][cap][hd]; len_dev int32 [b] (device); out_dev fp32 [b*q][H*hd].
 * hd must be 64 or 128; k_dev, v_dev and out_dev 16-byte aligned.  Errors: EINVAL. */
SDSAT_API sdsat_status sdsat_op_attention(sdsat_ctx* ctx, const float* q_dev, const void* k_dev, const void* v_dev,
                                const int32_t* len_dev, int b, int q, int H, int hd, int cap,
                                float* out_dev);

/* Block-causal attention over pages, for sequences that share their leading ones:
 * out[s*q+j][h*hd+d] = sum_t softmax_t(q_j . k_t / sqrt(hd)) v_t[d] over slots t < len[s] + j + 1,
 * or, with anc_dev, over the committed slots t < len[s] and the slots len[s] + i with bit i of
 * anc_dev[s*q+j] set (a row that sees no slot is 0).
 *   q_dev      [b*q] rows of H*hd values, q_ld values apart; out_dev the same with out_ld; both of
 *              `type` SDSAT_FP32 or SDSAT_BF16, sums fp32
 *   k_dev, v_dev  bf16 [n_pages][Hk][SDSAT_PAGE][hd]; query head h reads cache head h / (H/Hk)
 *   table_dev  int32 [b][table_ld]: the page of slots 64 j .. of each sequence
 *   shared_dev int32 [b]: the leading table columns in which the sequence's pages are sequence
 *              0's; NULL: none.  The whole pages of committed slots among those that all
 *              sequences share are read once for all of them, through sequence 0's row
 *   len_dev    int32 [b] committed lengths
 * A slot on a page outside [0, n_pages) is not attended to and sets device bit PAGE.  What a page
 * holds in slots that no row of a sequence sees does not matter; a block slot that some of its
 * rows see counts 0 times its value in the others, so a NaN or an infinity there reaches them.
 * Partial results go through the context's workspace (see the conventions on streams).  hd 64 or
 * 128, H a multiple of Hk, b*q <= SDSAT_MAX_ROWS, b*q*H*hd <= SDSAT_MAX_ROWS rows of the
 * context's heads, b*q*H*table_ld <= 2^30, max(b*q*G, H)*G < 2^32 for G = H/Hk; pointers
 * 16-byte aligned, rows a multiple of 16 bytes apart.  Errors: EINVAL. */
SDSAT_API sdsat_status sdsat_op_prefix_attention(sdsat_ctx* ctx, const void* q_dev, int64_t q_ld, const void* k_dev,
                                                 const void* v_dev, int n_pages, const int32_t* table_dev,
                                                 int table_ld, const int32_t* shared_dev, const int32_t* len_dev,
                                                 const uint32_t* anc_dev, int b, int q, int H, int Hk, int hd,
                                                 void* out_dev, int64_t out_ld, int type);

/* ---- ragged batches on pages: sequences with new rows of a number of their own --------------- */
/* The rows of a ragged batch stand one after the other: rows start[s] .. start[s+1]-1 are the new ones of sequence s,
 * row start[s] + i at slot len[s] + i.  start_dev int32 [b+1] ascends within [0, rows]; rows before start[0] and from
 * start[b] on belong to no sequence and are left as they are.  len_dev int32 [b]: the committed slots, which the calls do
 * not advance.  table_dev int32 [b][table_ld] and the pages as in sdsat_op_prefix_attention. */

/* Head norms, rotation and append.  For every new row of every sequence, with x one of its heads of queries or keys:
 *   x' = x rsqrt(mean x^2 + eps) g                        (with gains; else x' = x)
 *   (a, z) -> (a cos - z sin, a sin + z cos)              for the pairs of `rope` at the row's position
 * The queries go to q_out_dev, keys and the values (as they are) as bf16 to the slot's row of the sequence's page.
 *   q_dev, k_dev, v_dev  [rows] of H*hd, Hk*hd and Hk*hd values of `type` (SDSAT_FP32, SDSAT_BF16), q_ld, k_ld and v_ld
 *                        values apart: also parts of one matrix.  q_out_dev: the same type, q_out_ld apart; may be q_dev
 *                        with its q_ld, else no memory that the call reads
 *   q_gain_dev, k_gain_dev  bf16 [hd], or NULL: no norm of those heads
 *   position_dev         int32 [rows], or NULL: the slots.  A position outside the table counts as its nearest (device
 *                        bit POSITION)
 *   k_pages_dev, v_pages_dev  bf16 [n_pages][Hk][SDSAT_PAGE][hd]
 *   refs_dev             int32 [n_pages], or NULL: a row whose page is not held once is not written
 * A row past the table's slots or without a page (of its own, with refs) is not written to the cache and sets device
 * bit CAPACITY; its query is rotated all the same.  Two sequences that write to one page need refs.
 * hd 64 or 128, dims <= hd, H a multiple of Hk, b <= 65536; q, k, v and q_out 16-byte aligned with rows a multiple of 16
 * bytes apart, pages 16-byte aligned, gains aligned to their values.  Errors: EINVAL. */
SDSAT_API sdsat_status sdsat_op_rotary_append(sdsat_ctx* ctx, const sdsat_rope* rope, const void* q_dev, int64_t q_ld,
                                              const void* k_dev, int64_t k_ld, const void* v_dev, int64_t v_ld, int type,
                                              int rows, const int32_t* start_dev, const int32_t* len_dev, int b,
                                              const int32_t* position_dev, const void* q_gain_dev, const void* k_gain_dev,
                                              float eps, int H, int Hk, int hd, void* q_out_dev, int64_t q_out_ld,
                                              void* k_pages_dev, void* v_pages_dev, int n_pages, const int32_t* table_dev,
                                              int table_ld, const int32_t* refs_dev);

/* Causal attention of a ragged batch over pages (its new rows' keys and values among them):
 * out[start[s]+i][h*hd+d] = sum_t softmax_t(q . k_t / sqrt(hd)) v_t[d] over slots t <= len[s] + i.
 *   q_dev, out_dev  [rows] of H*hd values of `type` (SDSAT_FP32, SDSAT_BF16), q_ld and out_ld values apart; sums fp32;
 *                   query head h reads cache head h / (H/Hk).  out_dev may be q_dev with its q_ld, else no memory
 *                   that the call reads
 * fp32 queries and probabilities enter the products in three bf16 parts (24 bits), bf16 queries as they are and their
 * probabilities rounded to bf16.  A slot past the table or on a page outside [0, n_pages) is not attended to and sets
 * device bit PAGE (a row that sees no slot is 0); what a page holds in slots that no row of the sequence sees does not
 * matter; a row's invisible slots that a later row sees count 0 times their value.  A NaN that a row sees makes its result NaN, and
 * so does a score of inf (fp32: any infinite key, whose products with the parts are infinities of both signs); a row whose scores
 * are all -inf is 0.  A start_dev that does not ascend within [0, rows] leaves out_dev as it is and sets device bit CAPACITY;
 * negative lengths count as 0.  Partial results go through the context's workspace (see the conventions on streams).
 * hd 64 or 128, H a multiple of Hk, H/Hk <= 128, b <= 1024, n_pages * Hk * SDSAT_PAGE < 2^31; pointers 16-byte
 * aligned, rows a multiple of 16 bytes apart.  Errors: EINVAL, EUNSUPPORTED (H/Hk or b above that). */
SDSAT_API sdsat_status sdsat_op_chunk_attention(sdsat_ctx* ctx, const void* q_dev, int64_t q_ld, int rows,
                                                const void* k_pages_dev, const void* v_pages_dev, int n_pages,
                                                const int32_t* table_dev, int table_ld, const int32_t* start_dev,
                                                const int32_t* len_dev, int b, int H, int Hk, int hd, void* out_dev,
                                                int64_t out_ld, int type);

/* Log probabilities of rows of logits at a temperature T: with m the row's maximum,
 * d_i = (l_i - m) / T and S = sum_i exp(d_i),
 *   logp[r]    = d_t - log S of the row's token t = tokens_dev[r]
 *   rank[r]    = 1 + the ids of larger logit, or of the same and lower id (1: the argmax)
 *   entropy[r] = log S - sum_i exp(d_i) d_i / S
 *   top_ids, top_logp [rows][n_top]: the n_top largest logits, the lower id first on ties
 * logits_dev: rows of `vocab` values of `type`, ld values apart (any alignment).  tokens_dev
 * int32 [rows]; -1: no token (logp 0, rank 0); NULL: none in any row, logp_dev and rank_dev
 * NULL.  Any output but the two of n_top > 0 may be NULL.  A NaN logit counts as -inf (device
 * bit NAN_LOGITS), a token outside the vocabulary as id 0 (TOKEN); a logit of +inf shares the
 * mass with the others of +inf; a row of -inf alone has probabilities 0 and entropy 0.
 * Errors: EINVAL (temperature <= 0, infinite or below 4.3e-39, n_top > 32 or > vocab, rows >
 * 2^27), EUNSUPPORTED (vocab > 262144). */
SDSAT_API sdsat_status sdsat_op_logprobs(sdsat_ctx* ctx, const void* logits_dev, int64_t ld, int type, int rows,
                                         int vocab, const int32_t* tokens_dev, float temperature, int n_top,
                                         float* logp_dev, float* entropy_dev, int32_t* rank_dev,
                                         int32_t* top_ids_dev, float* top_logp_dev);

/* Rules on the logits of b*q block rows (row j of sequence s at s*q + j) before a token is selected.  With
 * c(t) the number of times that t was generated and seen(t) whether it was, or is in the prompt:
 *   l <- seen(t) ? (l > 0 ? l / repetition[s] : l * repetition[s]) : l
 *   l <- l - frequency[s] c(t) - (c(t) > 0 ? presence[s] : 0)
 *   l <- l + the bias of t
 *   l <- allowed(t) ? l : -inf
 * in fp32, rounded once.  in_dev, out_dev: rows of `vocab` values of `type`, in_ld and out_ld values apart (any
 * alignment of their values); the same rows (in_ld = out_ld), or none in common.
 *   history_dev       int32 [b][history_ld]: the tokens before the block; history_len_dev int32 [b] of them (clamped to
 *                     [0, history_ld]), the first prompt_len_dev int32 [b] the prompt (NULL: none); NULL: no history
 *   tokens_dev        int32 [b*q]: the block's tokens.  Row j comes after tokens 0 .. j of its sequence, or, with anc_dev,
 *                     after those of the bits of anc_dev[s*q+j]; they count as generated.  NULL: none
 *   repetition_dev, frequency_dev, presence_dev  fp32 [b]; NULL: 1, 0, 0
 *   bias_id_dev, bias_dev  int32 and fp32 [b][n_bias]; of an id that is there twice the first counts
 *   allowed_dev       uint32 [b*q][allowed_ld]: bit t % 32 of word t / 32; NULL: all
 * Negative ids in history, tokens and biases are places that hold none; ids from vocab on count as none too and set
 * device bit TOKEN.  NaN logits stay NaN where they are allowed.  q <= SDSAT_MAX_Q, b*q <= 2^20, n_bias <= 1024,
 * history_ld < 2^19.  Errors: EINVAL, EUNSUPPORTED (history_ld, n_bias or vocab > 2^20). */
SDSAT_API sdsat_status sdsat_op_adjust_logits(sdsat_ctx* ctx, const void* in_dev, int64_t in_ld, int type, int b, int q,
                                              int vocab, const int32_t* history_dev, int history_ld,
                                              const int32_t* history_len_dev, const int32_t* prompt_len_dev,
                                              const int32_t* tokens_dev, const uint32_t* anc_dev,
                                              const float* repetition_dev, const float* frequency_dev,
                                              const float* presence_dev, const int32_t* bias_id_dev, const float* bias_dev,
                                              int n_bias, const uint32_t* allowed_dev, int allowed_ld, void* out_dev,
                                              int64_t out_ld);

/* Copy a context workspace of the last block forward into dst_dev (fp32,
 * rows x cols row-major, rows = b*q of that forward): which = 0 the residual
 * stream h [rows][d], 1 the RoPE'd queries [rows][H*hd], 2 the attention
 * output [rows][H*hd], 3 the SwiGLU activations [rows][F] -- of the last
 * layer.  For tests that check a forward stage by stage.  Errors: EINVAL. */
SDSAT_API sdsat_status sdsat_debug_workspace(sdsat_ctx* ctx, int which, int rows, float* dst_dev);

/* The attention grid sdsat_block_forward and sdsat_op_attention launch for `pairs`
 * (sequence, head) pairs (host only, no GPU): one thread-block cluster of *cs CTAs per
 * pair, *nclusters = pairs, for the largest cs <= min(cs_cap, 16) with
 * max_clusters[cs] >= pairs and cs * (pairs + 8) <= max_clusters[1] (the CTAs resident
 * at once, else 2 * num_sms), or, where that cs is above 2 and fewer than a tenth more
 * clusters of it than pairs fit, the next smaller such cs; otherwise *cs = 1 and
 * *nclusters = min(pairs, resident), each CTA taking several pairs.  max_clusters[c]
 * (c = 1..16, host array of 17 entries, [0] unused) = the most clusters of c CTAs the
 * device holds at once, as cudaOccupancyMaxActiveClusters reports it for the attention
 * kernel.  The launches' cs_cap is the number of 64-slot units of the cache.  Errors: EINVAL. */
SDSAT_API sdsat_status sdsat_attention_grid(int pairs, const int32_t* max_clusters, int cs_cap, int num_sms,
                                            int* cs, int* nclusters);

/* Test hook for failure detection: one kernel waits on a barrier that nothing
 * completes, through the bounded wait every kernel of the library uses.  After its
 * limit (2 s) it sets device bit TIMEOUT and returns; nothing faults and the
 * context stays usable.  Asynchronous (read the bit with sdsat_get_error).
 * Errors: EINVAL (null ctx), ECUDA. */
SDSAT_API sdsat_status sdsat_debug_wait_timeout(sdsat_ctx* ctx);

/* out[i] = the nucleus sampler's exp (see sdsat_accept_nucleus) of in[i] <= 0. */
SDSAT_API sdsat_status sdsat_op_exp(sdsat_ctx* ctx, const float* in_dev, float* out_dev, int n);

/* y[m][n] = sum_k x[m][k] * W[n][k] like sdsat_op_gemm, for callers that cannot
 * allocate device memory: no context, no cudaMalloc or other allocating call.
 * This entry point has no counterpart in the paper; it exists because a caller
 * may be capturing a CUDA graph (where allocation is not allowed), may run inside
 * a framework that owns all device memory through its own allocator, or may have
 * a fixed memory budget.  Its scratch -- the operand split, the split-K partial
 * sums and the tile counters -- is one fixed array in device memory (3 MiB +
 * 2 KiB, held by every GPU that loads the library until the process exits).
 *   x_dev fp32 [M][K] (16-byte aligned), W bf16 [N][K] (16-byte aligned),
 *   y_dev fp32 [M][N]; stream is a cudaStream_t (NULL = legacy default stream).
 *   Limits: 1 <= M <= 16, 8 <= K <= 16384 with K % 8 == 0, 1 <= N <= 65536;
 *   sizes past the limits return ECAPACITY, malformed arguments EINVAL.
 *   err_dev: optional caller-owned device word (NULL: not reported); a bounded
 *   in-kernel wait that runs out (2 s) ORs SDSAT_DEV_TIMEOUT into it and leaves
 *   y_dev incomplete.  The call never clears it.
 * The first call on a device (with that device current) looks up the array's
 * device address and prepares the kernels; make that first call before any
 * stream capture.  The set-up is redone when the device's context changes (after
 * cudaDeviceReset, for instance).  Every call shares the one array: calls whose
 * work overlaps on the GPU (different streams, or concurrent host threads) race
 * and must be serialised by the caller.  The call clears the tile counters it
 * uses; the other scratch contents are overwritten before they are read.
 * Asynchronous on `stream`. */
SDSAT_API sdsat_status sdsat_gemm_static(const float* x_dev, int M, int K, const void* w_dev, int N, float* y_dev,
                                         void* stream, uint32_t* err_dev);

/* ---- measurement ------------------------------------------------------------------ */

/* Per-kernel timing: between sdsat_profile_begin and sdsat_profile_end every
 * kernel the library launches on ctx is bracketed by CUDA events recorded on
 * the context stream (which serialises the launches: no overlap between
 * consecutive kernels while profiling).  begin creates a pool of events for
 * up to max_launches launches (call it outside any graph capture); launches
 * past the pool are not timed.  end synchronises and returns one record per
 * kernel class that ran: its name, launch count and summed duration. */
typedef struct {
  char name[32];
  int64_t launches;
  double total_ms;
} sdsat_kernel_stat;

SDSAT_API sdsat_status sdsat_profile_begin(sdsat_ctx* ctx, int max_launches);
SDSAT_API sdsat_status sdsat_profile_end(sdsat_ctx* ctx, sdsat_kernel_stat* out, int max_out, int* n_out);

/* Device timeline trace (does not serialise launches): between sdsat_trace_begin and
 * sdsat_trace_end, thread 0 of every CTA of the block forward's GEMM and attention kernels
 * (and of the prefill's GEMM) appends one record of SDSAT_TRACE_WORDS uint64:
 *   [0] tag << 32 | block index, tag = kernel class << 24 | launch sequence number
 *       (sdsat_kernel_class_name names a class);
 *   [1] flags << 32 | SM id;
 *   [2] %globaltimer (ns) at kernel entry, [3] after the wait for the preceding kernel,
 *   [4], [5], [6] kernel-specific marks (0 = not reached), [7] at exit.
 * GEMM: marks = first MMA issued, accumulator of the CTA's last tile ready, that tile
 * reduced (or handed to another CTA); flags = 1 if this CTA reduced it | contributors << 8.
 * Attention: marks = first K/V tile usable, the CTA's partial of its last (sequence, head)
 * pair written, that pair's share of the merged output stored; flags = pairs taken |
 * units of 64 slots << 8.
 * begin allocates room for max_records records (call it outside any graph capture); end
 * synchronises, copies up to max_records records to host memory and frees the buffer. */
#define SDSAT_TRACE_WORDS 8
SDSAT_API sdsat_status sdsat_trace_begin(sdsat_ctx* ctx, int max_records);
SDSAT_API sdsat_status sdsat_trace_end(sdsat_ctx* ctx, uint64_t* records_host, int max_records, int* n_records);
SDSAT_API const char* sdsat_kernel_class_name(int kernel_class);

#ifdef __cplusplus
}
#endif
#endif /* SDSAT_H */
