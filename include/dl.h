/*
 * dl.h -- C ABI of the Dynamic-LLaVA sparsified-inference hot path for NVIDIA B200 (sm_100a).
 *
 * The calls follow the method's statement in the paper (arXiv 2412.00876):
 *   prefill  (Eq. 5, Eq. 11): a predictor scores every vision token, the k best are kept,
 *            the kept rows plus all text rows form the reduced set S^{P*}, and every later
 *            layer attends over that reduced set only (Eq. 1 on S^{P*});
 *   decoding with KV cache (Eq. 6): the current token always takes part in its own attention,
 *            and its K/V are appended to the cache only if the predictor's decision is 1;
 *            the decision is taken once per token and shared by all later layers (Sec. 3.3.1).
 *
 * Conventions
 *   - Plain C.  Every call returns an int32_t status: DL_OK (0) or a negative DL_ERR_*.
 *   - "dev" pointers are device memory owned by the caller; "host" pointers are host memory.
 *     The library allocates no device memory: scratch comes from the caller (dl_set_workspace).
 *   - Calls are asynchronous on `stream` (a cudaStream_t passed as void*; NULL = default stream)
 *     unless stated otherwise.  One context serves one stream at a time.
 *   - Tensors are dense, innermost dimension contiguous, every tensor pointer 16-byte aligned.
 *     Element type `dtype` (DL_F32 or DL_BF16) applies to activations, Q/K/V, caches, outputs
 *     and W1; scores, logits, b1, w2 are always float32.
 *   - Cache layout (what compaction is judged on, bit for bit): per layer, K and V are separate
 *     tensors [B][H][cap][D], D contiguous.  Rows [0, cache_len[b]) of sequence b are valid;
 *     rows beyond are unspecified.
 *   - Errors found on the device (capacity overflow, NaN score) are recorded in a status word
 *     inside the workspace; dl_device_status reads it back.  Nothing traps.
 */
#ifndef DL_SPARSE_H_
#define DL_SPARSE_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct dl_ctx dl_ctx;

enum { DL_F32 = 0, DL_BF16 = 1 };

enum {
  DL_OK = 0,
  DL_ERR_INVALID_ARG = -1,   /* NULL pointer, negative size, k out of range, ... */
  DL_ERR_ALIGNMENT = -2,     /* a tensor pointer is not 16-byte aligned */
  DL_ERR_UNSUPPORTED = -3,   /* dtype / head_dim / size combination not built */
  DL_ERR_WORKSPACE = -4,     /* workspace missing or too small for this call */
  DL_ERR_CUDA = -5,          /* a CUDA runtime call failed (see dl_last_cuda_error) */
  DL_ERR_CAPACITY = -6,      /* device status: kept rows did not fit into the cache */
  DL_ERR_TIMEOUT = -7,       /* device status: a bounded wait ran out */
  DL_ERR_BOUNDS = -8,        /* device status (checked build only): an index fell outside its buffer; the access was skipped */
  DL_WARN_NAN = 1            /* device status: a NaN score was ranked as -inf / dropped */
};

/* Implementation selectors for dl_set_option. */
enum {
  DL_OPT_PREDICTOR_IMPL = 1,    /* 0 auto, 1 CUDA-core kernel, 2 tcgen05 tensor-core kernel (bf16) */
  DL_OPT_PREFILL_ATTN_IMPL = 2, /* 0 auto, 1 CUDA-core kernel, 2 tcgen05 tensor-core kernel (bf16, D=128) */
  DL_OPT_DECODE_CHUNK = 3,      /* cache rows per decode work item (0 = chosen by the library) */
  DL_OPT_DECODE_IMPL = 4,       /* 0 auto, 1 CUDA-core kernel, 2 tensor-core (mma.sync) kernel (bf16, D=128) */
  DL_OPT_COMPACT_IMPL = 5       /* 0 auto, 1 register-staged copy kernel, 2 bulk-copy (TMA) kernel over even ranges of kept
                                 * rows with one tensor store per row (auto: 2 for up to 2048 sequences, else 1) */
};

typedef struct {
  int32_t hidden;      /* d: width of the hidden rows fed to the predictors */
  int32_t n_heads;     /* H (multi-head attention: as many K/V heads as query heads) */
  int32_t head_dim;    /* D: 64 or 128 */
  int32_t pred_hidden; /* width of the predictor's hidden layer */
  int32_t dtype;       /* DL_F32 or DL_BF16 */
} dl_model_desc;

/* One token predictor in per-token MLP form: score = w2 . GELU(W1 x + b1) + b2, GELU in its
 * exact erf form.  With a single output the score is at once the ranking value of Eq. 11 and
 * the folded two-way decision of Eq. 5 (keep iff score > 0). */
typedef struct {
  const void* w1;   /* dev [pred_hidden][hidden], dtype */
  const float* b1;  /* dev [pred_hidden] */
  const float* w2;  /* dev [pred_hidden] */
  float b2;
} dl_predictor;

/* ---- context ------------------------------------------------------------------------- */

/* Creates a context for `device` and `desc` (copied).  Host call; may initialise the CUDA
 * context.  DL_ERR_UNSUPPORTED for head_dim not in {64,128}, hidden % 8 != 0 or unknown dtype. */
int32_t dl_create(dl_ctx** out, int32_t device, const dl_model_desc* desc);
int32_t dl_destroy(dl_ctx* ctx);

/* Bytes of scratch the calls below need for up to `max_batch` sequences, `max_rows` predictor
 * rows per call (B * n_vis_max in prefill) and caches of `cap` rows.  Negative on bad args.
 * For bf16 models this includes, whatever the sizes, a part that dl_kv4_attn_decode, dl_kv16_attn_tree
 * (the parts of split sequences) and dl_kv16_append (its list of kept rows) use in turn: on 148
 * multiprocessors 39.4 MB with D = 128; with D = 64 20 MB, up to 32 MB with many heads. */
int64_t dl_workspace_bytes(const dl_ctx* ctx, int32_t max_batch, int32_t max_rows, int32_t cap);

/* Hands the context its scratch (dev, 256-byte aligned, caller keeps ownership) and clears the
 * part that must start at zero (asynchronously on `stream`).  The sizes are the ones that were
 * given to dl_workspace_bytes. */
int32_t dl_set_workspace(dl_ctx* ctx, void* dev_ptr, int64_t bytes, int32_t max_batch,
                         int32_t max_rows, int32_t cap, void* stream);

int32_t dl_set_option(dl_ctx* ctx, int32_t option, int32_t value);

/* Synchronises `stream`, copies the device status word back and clears it.  code_out gets
 * DL_OK, DL_ERR_CAPACITY, DL_ERR_TIMEOUT or DL_WARN_NAN; detail_out the sequence index or row. */
int32_t dl_device_status(dl_ctx* ctx, void* stream, int32_t* code_out, int64_t* detail_out);

const char* dl_status_str(int32_t status);
/* Text of the last CUDA error seen by this context (host string owned by the library). */
const char* dl_last_cuda_error(const dl_ctx* ctx);

/* ---- prefill: Eq. 5 / Eq. 11 --------------------------------------------------------- */

/* Predictor alone (first line of Eq. 5 / Eq. 11): score_out[r] for `rows` hidden rows.
 * x dev [rows][hidden] dtype; score_out dev [rows] float32. */
int32_t dl_predictor_scores(dl_ctx* ctx, const dl_predictor* p, const void* x, int32_t rows,
                            float* score_out, void* stream);

/* TopkArgmax_k of Eq. 11 on given scores.  For each sequence b the k[b] largest of its first
 * n_vis[b] scores are kept; between equal scores the lower index wins; -0 equals +0; NaN ranks
 * as -inf (and sets DL_WARN_NAN).
 *   score dev [B][n_vis_max]; n_vis dev [B] or NULL (= n_vis_max); k dev [B], 0 <= k[b] <= n_vis[b]
 *   (a larger k[b] is clamped to n_vis[b]); kept_idx_out dev [B][k_max] ascending, unused slots -1
 *   (may be NULL); keep_out dev [B][n_vis_max] 0/1 (padding slots 0).  n_vis_max <= 16384.
 *   k_max must cover every k[b]: where it does not, the index list holds the first k_max kept indices only
 *   (the mask is complete) and DL_ERR_INVALID_ARG is recorded in the status word with the sequence index. */
int32_t dl_topk_from_scores(dl_ctx* ctx, const float* score, const int32_t* n_vis, const int32_t* k,
                            int32_t B, int32_t n_vis_max, int32_t* kept_idx_out, int32_t k_max,
                            uint8_t* keep_out, void* stream);

/* Eq. 11 end to end: scores of all vision rows, then the selection above.
 *   x_vis dev [B][n_vis_max][hidden]; score_out dev [B][n_vis_max]; others as above. */
int32_t dl_prefill_select(dl_ctx* ctx, const dl_predictor* p_img, const void* x_vis,
                          const int32_t* n_vis, const int32_t* k, int32_t B, int32_t n_vis_max,
                          float* score_out, int32_t* kept_idx_out, int32_t k_max, uint8_t* keep_out,
                          void* stream);

/* ---- compaction: set builder of Eq. 5, reduced set of Eq. 11, append of Eq. 6 --------- */

/* Appends to each sequence's cache, in token order, the source rows whose keep flag is 1,
 * starting at row cache_len[b]; if `commit` != 0, cache_len[b] += number appended.
 *   k_src, v_src dev [B][t_src_max][H][D] (v_src and v_cache may both be NULL: one tensor only);
 *   keep dev [B][keep_cols] or NULL (= keep all): the flags of the first keep_cols source rows;
 *   source rows t >= keep_cols are always kept.  In prefill keep_cols is the number of vision
 *   slots, so that the mask is M^I followed by ones for the text rows (S^{I*} u S^T of Eq. 11);
 *   t_src dev [B] valid source rows or NULL (= t_src_max);
 *   k_cache, v_cache dev [B][H][cap][D]; cache_len dev [B], read, and written when commit != 0.
 * Rows are copied bit for bit.  A sequence whose kept rows do not fit (cache_len + count > cap)
 * is left untouched, its length unchanged, and DL_ERR_CAPACITY is recorded with its index.
 * Several layers that share one decision pass commit = 0 for all but the last layer's call.
 * Needs the workspace. */
int32_t dl_compact_kv(dl_ctx* ctx, const void* k_src, const void* v_src, const uint8_t* keep,
                      int32_t keep_cols, const int32_t* t_src, int32_t B, int32_t t_src_max, void* k_cache,
                      void* v_cache, int32_t cap, int32_t* cache_len, int32_t commit, void* stream);

/* The same for n_tensors tensors that share ONE decision (Sec. 3.3.1: the mask is made once and used by every
 * later layer): K, V (and Q or hidden rows) of all layers in one call.  One plan (count, capacity check, length
 * commit) and a run of copy launches that overlap one another's start-up and tail; everything queued after the
 * call still finds all copies complete.  Same result, bit for bit, as n_tensors single-tensor calls of
 * dl_compact_kv with commit = 0 followed by the length commit.
 *   srcs, caches HOST arrays of n_tensors device pointers: srcs[i] [B][t_src_max][H][D] -> caches[i] [B][H][cap][D],
 *   every tensor appended at row cache_len[b]; the other arguments as for dl_compact_kv.  Needs the workspace. */
int32_t dl_compact_kv_layers(dl_ctx* ctx, int32_t n_tensors, const void* const* srcs, void* const* caches,
                             const uint8_t* keep, int32_t keep_cols, const int32_t* t_src, int32_t B, int32_t t_src_max,
                             int32_t cap, int32_t* cache_len, int32_t commit, void* stream);

/* dl_compact_kv with the SOURCE rows in pinned host memory (Eq. 5 / Eq. 11: only the kept rows enter the
 * reduced set, so only they need to reach the GPU).  The copy kernel reads the kept rows straight from host
 * memory over the bus; dropped rows never cross it, and no staging copy of the whole source is made.
 *   k_src_host, v_src_host HOST, pinned and reachable from the device (cudaHostAlloc / cudaHostRegister,
 *   e.g. torch's pin_memory()), [B][t_src_max][H][D]; every other argument as for dl_compact_kv (device).
 * The host buffers must stay valid and unchanged until the stream has passed this call.
 * DL_ERR_INVALID_ARG if a source is not such host memory. */
int32_t dl_compact_kv_host(dl_ctx* ctx, const void* k_src_host, const void* v_src_host, const uint8_t* keep,
                           int32_t keep_cols, const int32_t* t_src, int32_t B, int32_t t_src_max, void* k_cache,
                           void* v_cache, int32_t cap, int32_t* cache_len, int32_t commit, void* stream);

/* ---- attention over the reduced set --------------------------------------------------- */

/* Prefill (Eq. 1 on S^{P*}): causal scaled-dot-product attention of the compact rows against
 * themselves, per sequence and head: row i attends rows 0..i of the same cache.
 *   q dev [B][H][cap][D] compact queries in the cache layout (built by dl_compact_kv);
 *   k_cache, v_cache dev [B][H][cap][D]; cache_len dev [B]; n_max >= every cache_len[b], <= cap;
 *   out dev [B][n_max][H][D] (rows >= cache_len[b] are not written); scale > 0, usually 1/sqrt(D). */
int32_t dl_sparse_attn_prefill(dl_ctx* ctx, const void* q, const void* k_cache, const void* v_cache,
                               const int32_t* cache_len, int32_t B, int32_t cap, int32_t n_max,
                               float scale, void* out, void* stream);

/* Decoding with KV cache (Eq. 6, second line): Attention(Q, S^K u K, S^V u V) for one new token
 * per sequence: the query attends cache rows [0, cache_len[b]) plus the token's own (k_t, v_t).
 *   q_t, k_t, v_t dev [B][H][D]; out dev [B][H][D].
 * If `keep` (dev [B], may be NULL) is given, the call also performs Eq. 6's conditional append
 * for this layer: where keep[b] != 0, (k_t, v_t) are written to row cache_len[b] of the caches
 * (cache_len itself is not changed: call dl_commit_len once after the last layer).  A full
 * cache (cache_len[b] == cap) records DL_ERR_CAPACITY and skips the write.  Needs the workspace. */
int32_t dl_sparse_attn_decode(dl_ctx* ctx, const void* q_t, const void* k_t, const void* v_t,
                              void* k_cache, void* v_cache, const int32_t* cache_len,
                              const uint8_t* keep, int32_t B, int32_t cap, float scale, void* out,
                              void* stream);

/* The same for a stack of L layers that share cache_len and keep (Eq. 6 applied per layer with the
 * one decision of Sec. 3.3.1): q_t, k_t, v_t, out dev [L][B][H][D]; k_caches, v_caches HOST arrays of
 * L device pointers, each [B][H][cap][D] and all distinct.  Equivalent to L calls of
 * dl_sparse_attn_decode in layer order, except that a layer's kernel may begin while the previous
 * layer's is still draining (they touch different caches and outputs); everything launched after
 * this call still sees all L layers complete. */
int32_t dl_sparse_attn_decode_layers(dl_ctx* ctx, int32_t L, const void* q_t, const void* k_t, const void* v_t,
                                     void* const* k_caches, void* const* v_caches, const int32_t* cache_len,
                                     const uint8_t* keep, int32_t B, int32_t cap, float scale, void* out,
                                     void* stream);

/* ---- decode decision: Eq. 5 applied to the current token (Eq. 6) ----------------------- */

/* logit[b] = P^{OT}(x_t[b]);  keep[b] = logit[b] > threshold (strict; NaN -> 0).
 *   x_t dev [B][hidden] or NULL: with NULL the logits already in logit_inout are used as given.
 *   logit_inout dev [B]; keep_out dev [B]. */
int32_t dl_decode_keep(dl_ctx* ctx, const dl_predictor* p_txt, const void* x_t, int32_t B,
                       float threshold, float* logit_inout, uint8_t* keep_out, void* stream);

/* Decoding WITHOUT KV cache (Eq. 12 and the sentence above Eq. 6): the decisions for ALL generated
 * tokens of every sequence at once; the last generated token of a sequence is always kept, since it
 * produces the next token.  keep[b][i] = i < n_gen[b] and (logit[b][i] > threshold or i == n_gen[b]-1).
 *   x_gen dev [B][n_gen_max][hidden] or NULL (then logit_inout is used as given); n_gen dev [B] or NULL
 *   (= n_gen_max); logit_inout dev [B][n_gen_max] float32; keep_out dev [B][n_gen_max] (padding 0).
 * The reduced set S^{P*} u S^{OT*} is then built with dl_compact_kv (this mask, keep_cols = n_gen_max,
 * t_src = n_gen, appended behind the compact prefill rows) and attended with dl_sparse_attn_prefill. */
int32_t dl_decode_nocache_select(dl_ctx* ctx, const dl_predictor* p_txt, const void* x_gen, const int32_t* n_gen,
                                 int32_t B, int32_t n_gen_max, float threshold, float* logit_inout,
                                 uint8_t* keep_out, void* stream);

/* cache_len[b] += (keep[b] != 0) where cache_len[b] < cap: closes a decode step after every
 * layer has appended with the shared decision (Sec. 3.3.2). */
int32_t dl_commit_len(dl_ctx* ctx, const uint8_t* keep, int32_t B, int32_t cap, int32_t* cache_len,
                      void* stream);

/* One whole decode step over a stack of L layers that share the decision: dl_decode_keep, then
 * per layer dl_sparse_attn_decode with the fused append, then dl_commit_len.  Same results as those calls; the
 * library folds the decision into the predictor's launch and the length commit into the last layer's (1 + L
 * launches per step for bf16 models).
 *   q_t, k_t, v_t, out: dev [L][B][H][D]; k_caches, v_caches: HOST arrays of L device pointers,
 *   each [B][H][cap][D].  Other arguments as in the single calls. */
int32_t dl_decode_step(dl_ctx* ctx, const dl_predictor* p_txt, const void* x_t, int32_t B,
                       float threshold, float* logit_inout, uint8_t* keep_out, int32_t L,
                       const void* q_t, const void* k_t, const void* v_t, void* const* k_caches,
                       void* const* v_caches, int32_t cap, int32_t* cache_len, float scale,
                       void* out, void* stream);

/* A decoder's layer stack with the decision taken after its l-th layer (Sec. 3.3.1): the first l_dense layers run
 * before the decision exists and keep every token, the remaining L - l_dense share the decision.
 *   k_caches, v_caches: HOST arrays of L dev pointers; entries below l_dense are [B][H][cap_dense][D] caches whose
 *   lengths are len_dense (dev [B], +1 per step while below cap_dense), the others [B][H][cap][D] caches whose
 *   lengths are cache_len (dev [B], += keep per step).  The workspace must cover max(cap_dense, cap).
 *   len_dense may be NULL when l_dense == 0, cache_len when l_dense == L. */
typedef struct {
  int32_t L, l_dense;
  void* const* k_caches; void* const* v_caches;
  int32_t cap_dense, cap;
  int32_t* len_dense; int32_t* cache_len;
} dl_layer_stack;

/* dl_decode_step over such a stack (Eq. 6 with the layer placement of Sec. 3.3.1; with l_dense = 2 and one count of
 * image tokens this is the layer split Eq. 13's totals in Tab. 1 are made of): the decision, then one attention
 * launch per layer, dense layers first; the last dense launch advances len_dense, the last launch cache_len.
 *   q_t, k_t, v_t, out dev [L][B][H][D]. */
int32_t dl_decode_step_stack(dl_ctx* ctx, const dl_predictor* p_txt, const void* x_t, int32_t B, float threshold,
                             float* logit_inout, uint8_t* keep_out, const dl_layer_stack* stack, const void* q_t,
                             const void* k_t, const void* v_t, float scale, void* out, void* stream);

/* The same step fed from HOST buffers (pinned for full copy speed): copies x_t, q_t, k_t, v_t
 * into the caller's device staging buffers, runs dl_decode_step, copies `out` and `keep` back to
 * the host, all on `stream`; returns after the stream has been synchronised.
 *   *_host: host counterparts of the dl_decode_step tensors; stage_* : dev buffers of the same
 *   sizes (x [B][hidden]; q, k, v, out [L][B][H][D]); logit_dev [B], keep_dev [B] dev. */
int32_t dl_decode_step_host(dl_ctx* ctx, const dl_predictor* p_txt, const void* x_host, int32_t B,
                            float threshold, int32_t L, const void* q_host, const void* k_host,
                            const void* v_host, void* out_host, uint8_t* keep_host, void* stage_x,
                            void* stage_q, void* stage_k, void* stage_v, void* stage_out,
                            float* logit_dev, uint8_t* keep_dev, void* const* k_caches,
                            void* const* v_caches, int32_t cap, int32_t* cache_len, float scale,
                            void* stream);

/* n_steps decode steps fed from HOST buffers as a pipeline (Eq. 6, once per step): while step t
 * computes, the inputs of step t+1 are copied in and the results of step t-1 are copied out, on
 * two copy streams the context owns (created at the first call, with the events that order them;
 * no device memory is allocated).  Same results as n_steps calls of dl_decode_step_host.
 *   x_host, q_host, k_host, v_host, out_host, keep_host: HOST arrays of n_steps host pointers (the
 *   buffers pinned for full copy speed; keep_host or its entries may be NULL); stage_x dev
 *   [2][B][hidden]; stage_q, stage_k, stage_v, stage_out dev [2][L][B][H][D]; logit_dev dev [2][B];
 *   keep_dev dev [2][B]: two staging sets, used in turn.  The compute runs on `stream`, behind what the
 *   caller queued there; returns after all three streams have been synchronised.  A failed step ends
 *   the sequence: its status is returned once the queued work has drained. */
int32_t dl_decode_steps_host(dl_ctx* ctx, const dl_predictor* p_txt, int32_t n_steps, int32_t B,
                             float threshold, int32_t L, const void* const* x_host,
                             const void* const* q_host, const void* const* k_host,
                             const void* const* v_host, void* const* out_host,
                             uint8_t* const* keep_host, void* stage_x, void* stage_q, void* stage_k,
                             void* stage_v, void* stage_out, float* logit_dev, uint8_t* keep_dev,
                             void* const* k_caches, void* const* v_caches, int32_t cap,
                             int32_t* cache_len, float scale, void* stream);

/* ---- the paper's own predictors (App. "Details of Predictor Architecture") -------------------------------- */

#define DL_PRED2_WIDTH 512      /* width after the input projection; 8 heads of 64; MLP hidden 2048; head 256, 128, 2 */

typedef struct { const void* w; const float* b; } dl_linear;     /* w dev [out][in] bf16, in contiguous; b dev [out] f32 */

/* One pre-norm transformer block over the image tokens of a sequence:
 *   x = x + proj(MHA(LN1(x)));  x = x + fc2(GELU(fc1(LN2(x))))      LayerNorm eps 1e-6, exact-erf GELU,
 * bidirectional scaled-dot-product attention, 8 heads of 64.  ln*_g, ln*_b dev [512] f32; qkv [1536][512] (query,
 * key, value projections stacked, head h owning 64 consecutive outputs of each); proj [512][512]; fc1 [2048][512];
 * fc2 [512][2048]. */
typedef struct {
  const float* ln1_g; const float* ln1_b; dl_linear qkv, proj;
  const float* ln2_g; const float* ln2_b; dl_linear fc1, fc2;
} dl_vit_block;

/* A predictor in the paper's architecture: in [512][hidden]; n_blocks transformer blocks (2 for the image predictor,
 * 0 for the output-text predictor, whose decision depends on the current token alone); head h1 [256][512],
 * h2 [128][256] (GELU after each), w3 dev [2][128] f32, b3 dev [2] f32.  `blocks` is a HOST array. */
typedef struct {
  dl_linear in;
  int32_t n_blocks;
  const dl_vit_block* blocks;
  dl_linear h1, h2;
  const float* w3; const float* b3;
} dl_predictor2;

/* Bytes of scratch dl_predictor2_values needs for `rows` rows (B * n_max).  Negative on bad arguments. */
int64_t dl_predictor2_scratch_bytes(const dl_ctx* ctx, int64_t rows);

/* Decision values of Eq. 5 for every row: D = P(x) in R^{rows x 2}.
 *   x dev [B][n_max][hidden] bf16; n_vis dev [B] or NULL (= n_max): only the first n_vis[b] rows of sequence b are
 *   tokens (they alone attend to one another; padding rows give D = 0, score = -inf, keep = 0);
 *   scratch dev, 256-byte aligned, at least dl_predictor2_scratch_bytes(B * n_max) bytes, caller-owned;
 *   d_out dev [B * n_max][2] f32 or NULL; score_out dev [B * n_max] f32 or NULL: the raw second value D[:,2], the
 *   ranking score of Eq. 11; keep_out dev [B * n_max] or NULL: the argmax of Eq. 5, 1 iff D[:,2] > D[:,1]
 *   (strictly; a NaN drops and records DL_WARN_NAN).  bf16 models only (DL_ERR_UNSUPPORTED otherwise). */
int32_t dl_predictor2_values(dl_ctx* ctx, const dl_predictor2* p, const void* x, const int32_t* n_vis, int32_t B, int32_t n_max,
                      void* scratch, int64_t scratch_bytes, float* d_out, float* score_out, uint8_t* keep_out, void* stream);

/* Eq. 11 with the paper's image predictor: D = P^I(x_vis), then the k[b] tokens with the largest D[:,2] per sequence
 * (ties to the lower index), exactly as dl_prefill_select does with its one-logit predictor. */
int32_t dl_prefill_select2(dl_ctx* ctx, const dl_predictor2* p_img, const void* x_vis, const int32_t* n_vis,
                           const int32_t* k, int32_t B, int32_t n_vis_max, void* scratch, int64_t scratch_bytes,
                           float* d_out, float* score_out, int32_t* kept_idx_out, int32_t k_max, uint8_t* keep_out,
                           void* stream);

/* Eq. 6's decision with the paper's output-text predictor (n_blocks must be 0): keep[b] = D[b][2] > D[b][1].
 *   x_t dev [B][hidden]; d_out dev [B][2] or NULL; keep_out dev [B]. */
int32_t dl_decode_keep2(dl_ctx* ctx, const dl_predictor2* p_txt, const void* x_t, int32_t B, void* scratch,
                        int64_t scratch_bytes, float* d_out, uint8_t* keep_out, void* stream);

/* ---- diagnostics ----------------------------------------------------------------------- */

/* Self-test of the bounded waits (no counterpart in the paper): launches one small kernel that waits, with
 * the library's own wait routine and a bound of `polls` polls (1 .. 65536), on a barrier that can never
 * complete.  The wait gives up, the kernel records DL_ERR_TIMEOUT (detail 0x5e1f) in the status word and
 * returns; nothing traps and the context stays usable.  Asynchronous on `stream`; needs the workspace.
 * dl_device_status then reports the code. */
int32_t dl_selftest_wait_timeout(dl_ctx* ctx, int32_t polls, void* stream);

/* ---- extension, NOT in the paper: K/V cache in 8-bit floating point ---------------------- */

/* Decode attention (Eq. 6) is bound by the bytes of the cache it streams; these two calls store the cache rows as
 * 8-bit floating point in the OCP E4M3 format (1 sign, 4 exponent bits with bias 7, 3 mantissa bits; largest value
 * 448; no infinities) with one fp32 scale per head and tensor:  value = decode(byte) * scale[h].
 * bf16 models with head_dim 128 only (DL_ERR_UNSUPPORTED otherwise). */

/* Rows [0, cache_len[b]) of a bf16 cache as bytes: byte = encode(x / scale[h]), the quotient in fp32, round to
 * nearest with ties to the even code, magnitudes above 448 clamped to 448.  Rows at and past cache_len[b] are not
 * written.
 *   src dev [B][H][cap][128] bf16; scale dev [H] fp32 (> 0); dst dev [B][H][cap][128] uint8 (caller's). */
int32_t dl_quantize_kv_fp8(dl_ctx* ctx, const void* src, const int32_t* cache_len, const float* scale, int32_t B,
                           int32_t cap, void* dst, void* stream);

/* dl_sparse_attn_decode over such caches: the cached rows are read as decode(byte) * scale[h]; the current token is
 * attended with its own bf16 k_t, v_t (kept or not) and, where keep[b] != 0 and the cache has room, appended as
 * bytes at row cache_len[b] (lengths are NOT advanced: dl_commit_len closes the step).
 *   q_t, k_t, v_t, out dev [B][H][128] bf16; k_cache, v_cache dev [B][H][cap][128] uint8, read and (row cache_len[b])
 *   written; k_scale, v_scale dev [H] fp32; keep dev [B] or NULL.  Needs the workspace (split sequences). */
int32_t dl_sparse_attn_decode_fp8(dl_ctx* ctx, const void* q_t, const void* k_t, const void* v_t, void* k_cache,
                                  void* v_cache, const float* k_scale, const float* v_scale,
                                  const int32_t* cache_len, const uint8_t* keep, int32_t B, int32_t cap, float scale,
                                  void* out, void* stream);

/* The layer stack of a decode step over 8-bit caches (the counterpart of dl_sparse_attn_decode_layers): L launches
 * that overlap on the GPU; with commit != 0 the lengths advance once behind the last layer (cache_len[b] += keep[b]).
 *   q_t, k_t, v_t, out dev [L][B][H][128] bf16; k_caches, v_caches HOST arrays of L dev byte caches [B][H][cap][128];
 *   k_scales, v_scales dev [L][H] fp32; cache_len dev [B], read by every layer, written only with commit. */
int32_t dl_sparse_attn_decode_fp8_layers(dl_ctx* ctx, int32_t L, const void* q_t, const void* k_t, const void* v_t,
                                         void* const* k_caches, void* const* v_caches, const float* k_scales,
                                         const float* v_scales, int32_t* cache_len, const uint8_t* keep, int32_t B,
                                         int32_t cap, float scale, void* out, int32_t commit, void* stream);

/* ---- extension, NOT in the paper: whole prompts, packed ----------------------------------- */

/* Causal attention over whole prompts of different lengths, packed one behind the other, with grouped heads: what the
 * layers in front of the token selection compute (Eq. 1 on every token), before any cache exists.
 *   Row i of sequence b (packed row starts[b] + i) attends rows 0..i of the same sequence; query head h reads K/V head
 *   h / (n_heads / n_kv_heads).
 *   q [total][n_heads][D], k, v [total][n_kv_heads][D] dev bf16; q_stride, kv_stride: elements from one token's row to the
 *   next (0: dense), multiples of 8, so that q, k and v may be parts of one projection's output;
 *   starts dev [B + 1]: starts[b] <= starts[b + 1] <= total; equal ones make an empty sequence;
 *   max_rows HOST: no sequence is longer (rows behind it are not computed);
 *   out dev [total][n_heads][D] dense; rows of no sequence are left as they were.
 * A list of starts that breaks these rules records DL_ERR_INVALID_ARG with the sequence (if there is a workspace); nothing
 * is read or written outside the tensors.  A NaN or an infinity in v of a token may reach every row of its sequence that
 * shares a block of 128 keys with it, earlier ones too (0 * NaN in a matrix product).
 * bf16 models only (DL_ERR_UNSUPPORTED otherwise).  No workspace needed. */
int32_t dl_attn_prefill_packed(dl_ctx* ctx, const void* q, const void* k, const void* v, int64_t q_stride,
                               int64_t kv_stride, const int32_t* starts, int32_t B, int32_t n_kv_heads, int32_t total,
                               int32_t max_rows, float scale, void* out, void* stream);

/* ---- extension, NOT in the paper: caches in pages ------------------------------------------- */

/* The books of a paged cache.  All pointers dev, caller-owned.  Sequence b's rows [i * page_rows, (i + 1) * page_rows) are
 * in page table[b][i] of every pool (one pool per layer, say) that goes by these books. */
typedef struct {
  int32_t B;           /* sequences (slots), up to 2048 */
  int32_t n_pages;     /* pages of a pool */
  int32_t max_pages;   /* columns of the table */
  int32_t page_rows;   /* 16, 32, 64 or 128 */
  int32_t* table;      /* [B][max_pages] page numbers; -1 behind a sequence's last page, and nowhere else */
  int32_t* refs;       /* [n_pages] table entries that name the page; 0: free */
  int32_t* len;        /* [B] rows held */
} dl_pages;

/* Bytes of scratch for dl_pages_fork and dl_pages_compact.  Negative on bad arguments. */
int64_t dl_pages_scratch_bytes(const dl_ctx* ctx, const dl_pages* pages);

/* Gives every sequence the pages that len[b] + need[b] rows take (need dev [B]; negative counts as 0): the free pages with
 * the lowest numbers, handed out in order of b.  All or nothing: if the free pages or a row of the table do not suffice
 * nothing changes and DL_ERR_CAPACITY is recorded (detail: the sequence whose table row is too short, else -1). */
int32_t dl_pages_reserve(dl_ctx* ctx, const dl_pages* pages, const int32_t* need, void* stream);

/* Gives back all pages of the sequences with gone[b] != 0 (gone dev [B]) and sets their lengths to 0; a page that another
 * sequence shares stays in use. */
int32_t dl_pages_free(dl_ctx* ctx, const dl_pages* pages, const uint8_t* gone, void* stream);

/* Every sequence b becomes what sequence parent[b] was before the call (parent dev [B]; parent[b] == b: stays as it is, with
 * the pages reserved for it; -1: empty).  What b held is given back.  Full pages are shared; a partly filled last page
 * stays with one holder (the parent if it stays, else its lowest child) and is copied, in all pools, for each other child,
 * into the lowest free pages in order of b (pages given back by this call among them).  All or nothing as above (detail -1);
 * a parent out of range records DL_ERR_INVALID_ARG with b, and b stays as it is.
 *   pools HOST array of n_pools dev pointers, each [n_pages][page_bytes]; page_bytes a multiple of 16;
 *   scratch dev, 256-byte aligned, caller-owned. */
int32_t dl_pages_fork(dl_ctx* ctx, const dl_pages* pages, const int32_t* parent, int32_t n_pools, void* const* pools,
                      int64_t page_bytes, void* scratch, int64_t scratch_bytes, void* stream);

/* Moves the pages in use to the front: afterwards they are pages 0 .. n - 1, n = the number in use, which goes to
 * *n_live (dev, may be NULL).  A used page with number >= n moves to a free one below, both taken in ascending order;
 * the others stay.  Arguments as above. */
int32_t dl_pages_compact(dl_ctx* ctx, const dl_pages* pages, int32_t n_pools, void* const* pools, int64_t page_bytes,
                         int32_t* n_live, void* scratch, int64_t scratch_bytes, void* stream);

/* ---- extension, NOT in the paper: K/V cache in 4 bits, in pages, with grouped heads --------- */

/* K and V rows in 4 bits under one scale and one lowest value for every 64 dims:  value = s * code + z,  z = min,
 * s = bf16((max - min) / 15), code = nearest((x - z) * (1 / s)) (ties to even), clipped to 0..15; each operation in fp32.
 * Where s < 2^-126 all codes are 0.  64 dims with a NaN or an infinity among them (or a range beyond fp32) hold NaN.
 * K and V share a pool; how a page is laid out inside is the library's business (dl_kv4_read gives the values).
 * bf16 models, n_heads / n_kv_heads up to 16 (DL_ERR_UNSUPPORTED otherwise).  These calls need the workspace. */

/* Bytes of one page of a pool: n_kv_heads * page_rows * 9 D / 8.  Negative on bad arguments. */
int64_t dl_kv4_page_bytes(const dl_ctx* ctx, int32_t n_kv_heads, int32_t page_rows);

/* dl_compact_kv for such a cache: appends to every sequence, from row len[b] on and in order, its packed rows
 * [starts[b], starts[b + 1]) whose keep flag is not 0; with commit, len[b] += their number.  Layers that share a decision
 * pass commit = 0 but for the last.
 *   k, v dev bf16 [total][n_kv_heads][D], kv_stride elements from row to row (0: dense; a multiple of 8); starts dev
 *   [B + 1], ascending; keep dev [total] or NULL (all); pool dev [n_pages][page bytes].
 * The pages must be reserved: a sequence that lacks one is left untouched and records DL_ERR_CAPACITY with its index.
 * Pages that other sequences share must not be written: a fork leaves every partly filled page to one sequence. */
int32_t dl_kv4_append(dl_ctx* ctx, const dl_pages* pages, int32_t n_kv_heads, void* pool, const void* k, const void* v,
                      int64_t kv_stride, const int32_t* starts, const uint8_t* keep, int32_t total, int32_t commit,
                      void* stream);

/* The values of rows row0[b], row0[b] + 1, ... of every sequence, rounded to bf16, packed: starts[b + 1] - starts[b] rows of
 * sequence b from packed row starts[b] on.  row0 dev [B]; k_out, v_out dev [total][n_kv_heads][D].  A row without a page
 * reads as zero and records DL_ERR_INVALID_ARG with b. */
int32_t dl_kv4_read(dl_ctx* ctx, const dl_pages* pages, int32_t n_kv_heads, const void* pool, const int32_t* row0,
                    const int32_t* starts, int32_t total, void* k_out, void* v_out, void* stream);

/* dl_sparse_attn_decode (Eq. 6) over such a cache: one new token per sequence attends the values of rows [0, len[b]) and
 * its own bf16 k_t, v_t; where keep[b] != 0 its row is appended in 4 bits at row len[b] (the page must be reserved, else
 * DL_ERR_CAPACITY and no write).  Lengths are not advanced: dl_commit_len (cap = max_pages * page_rows) closes the step.
 *   q_t, out dev bf16 [B][n_heads][D]; k_t, v_t dev bf16 [B][n_kv_heads][D]; keep dev [B] or NULL.
 * Rows below len[b] without a page are left out and record DL_ERR_INVALID_ARG with b. */
int32_t dl_kv4_attn_decode(dl_ctx* ctx, const dl_pages* pages, int32_t n_kv_heads, void* pool, const void* q_t,
                           const void* k_t, const void* v_t, const uint8_t* keep, float scale, void* out, void* stream);

/* ---- extension, NOT in the paper: drafted tokens over a paged cache in 16 bits --------------- */

/* A cache in pages (dl_pages above) that holds K and V rows as they are:  page = [K, V][n_kv_heads][page_rows][D] bf16, so
 * a pool is [n_pages][2][n_kv_heads][page_rows][D].  A step with drafts is: dl_pages_reserve for the nodes, dl_tree_plan,
 * then in every layer dl_kv16_append (commit = 0: the nodes' rows lie behind the rows held) and dl_kv16_attn_tree, then
 * dl_tree_verify, and one dl_kv16_commit for all layers.  A prompt (or a chunk of one) is appended with commit = 1 in
 * its last layer; without drafts a sequence has one node.  dl_pages_fork, dl_pages_free and dl_pages_compact take these pools, too.
 * bf16 models, n_heads / n_kv_heads up to 128 (DL_ERR_UNSUPPORTED otherwise); these calls need the workspace unless noted. */

/* Rotary positions: the first rot_dim dims of a head are rot_dim / 2 pairs, (i, i + rot_dim / 2), or (2 i, 2 i + 1) if
 * interleaved; pair i of a row at position p turns by p * freqs[i] radians and is multiplied by `amplitude`.  Angles are taken
 * in 64 bits (as fractions of a turn), so that far positions lose nothing; the rotation itself is in fp32, rounded once. */
typedef struct {
  int32_t rot_dim;       /* a multiple of 16, 0 <= rot_dim <= D */
  int32_t interleaved;   /* 0: half layout */
  const double* freqs;   /* dev [rot_dim / 2] */
  float amplitude;
} dl_rope;

enum { DL_ROPE_PLAIN = 0, DL_ROPE_LINEAR = 1, DL_ROPE_NTK = 2, DL_ROPE_PARTS = 3 };

/* Host helper: freqs[i] = base^(-2 i / rot_dim), scaled for contexts `factor` times as long as the `orig_len` positions a model
 * was trained on:  LINEAR: divided by factor;  NTK: base * factor^(rot_dim / (rot_dim - 2)) instead of base;  PARTS: pairs
 * that turn more than 32 times in orig_len positions stay, those that turn less than once are divided by factor, linear in the
 * number of turns between, and amplitude = 0.1 ln(factor) + 1 (1 in the other forms).
 * freqs_out HOST [rot_dim / 2], amplitude_out HOST [1].  rot_dim even, base > 1, factor >= 1, orig_len >= 1 (PARTS). */
int32_t dl_rope_freqs(int32_t rot_dim, double base, int32_t scaling, double factor, int32_t orig_len, double* freqs_out,
                      double* amplitude_out);

/* What a step needs to know of its trees.  Sequence b's nodes are the packed rows [starts[b], starts[b + 1]); parent[row] is
 * the node's parent, counted within the sequence, -1 for a root (node 0 always is one: the last token that is certain), and lower
 * than the node's own number.  mask_out[row] gets the bits of the node itself and its ancestors (bit j % 32 of word j / 32),
 * pos_out[row] = pos0[b] + the node's depth.
 *   parent dev [total]; starts dev [B + 1]; pos0 dev [B] or NULL (0); mask_out dev [total][words], words 1..64, up to 32 * words
 *   nodes a sequence; pos_out dev [total] or NULL.  Rows of no sequence are left as they were.
 * A parent that breaks the rule records DL_ERR_INVALID_ARG with the sequence and counts as -1; a sequence with more nodes, too, and
 * its nodes behind 32 * words are left out.  No workspace needed. */
int32_t dl_tree_plan(dl_ctx* ctx, const int32_t* parent, const int32_t* starts, const int32_t* pos0, int32_t B, int32_t total,
                     int32_t words, int32_t* mask_out, int32_t* pos_out, void* stream);

/* Bytes of one page of a pool: 4 * n_kv_heads * page_rows * D.  Negative on bad arguments. */
int64_t dl_kv16_page_bytes(const dl_ctx* ctx, int32_t n_kv_heads, int32_t page_rows);

/* Rotates q and k to their positions and appends k (rotated) and v to a cache of 16-bit pages, in one pass.
 * Cache: from row len[b] on and in order, sequence b's packed rows [starts[b], starts[b + 1]) whose keep flag is not 0; with
 * commit, len[b] += their number.  q_out and k_out get the rotated rows of all sequences, dropped ones among them.
 *   pages, pool, v: NULL for the rotation alone (of all `total` rows; starts, keep and commit are not looked at then);
 *   q [total][n_heads][D] with q_out, or both NULL; k, v [total][n_kv_heads][D]; k_out [total][n_kv_heads][D] or NULL; all dev bf16;
 *   *_stride: elements from one token's row to the next (0: dense), multiples of 8; q_out and k_out may be q and k themselves
 *   (with the same strides), but not lie over anything else; pos dev [total] (may be NULL without rotation); rope HOST
 *   struct or NULL (no rotation); starts dev [B + 1], ascending; keep dev [total] or NULL (all).
 * The rows of q (if any), k and v (with a cache) of one token hold less than 2^19 values together (DL_ERR_UNSUPPORTED).
 * The pages must be reserved: a sequence that lacks one is left as it was and records DL_ERR_CAPACITY with its index (q_out and
 * k_out are written).  A call with `keep` lists its rows in the workspace: up to 33,000 rows a multiprocessor with D = 64, twice as
 * many with 128 (DL_ERR_WORKSPACE).  Pages that other sequences share must not be written: a fork leaves every partly filled page to one.
 * Rows of no sequence are left as they were, in q_out and k_out, too. */
int32_t dl_kv16_append(dl_ctx* ctx, const dl_pages* pages, int32_t n_kv_heads, void* pool, const void* q, int64_t q_stride,
                       const void* k, const void* v, int64_t kv_stride, const int32_t* pos, const dl_rope* rope,
                       const int32_t* starts, const uint8_t* keep, int32_t total, void* q_out, int64_t q_out_stride, void* k_out,
                       int64_t k_out_stride, int32_t commit, void* stream);

/* Attention of new rows over such a cache: node i of sequence b (packed row starts[b] + i) attends the cache's rows [0, len[b])
 * and, of the n = starts[b + 1] - starts[b] rows behind them, which hold the nodes' K and V, those that its mask names: row
 * len[b] + j where bit j % 32 of word j / 32 is set (bits from n on are not looked at).  Query head h reads K/V head
 * h / (n_heads / n_kv_heads).  A row that sees nothing gives 0.
 *   q dev bf16 [total][n_heads][D], rotated; q_stride as above; starts dev [B + 1]; mask dev [total][words] or NULL: node i sees
 *   nodes 0..i (a chain, the next chunk of a prompt, or the single token of a step without drafts);
 *   max_rows HOST: no sequence has more nodes (nodes behind it are not computed, and DL_ERR_INVALID_ARG is recorded), nor more
 *   than 32 * words with a mask; out dev bf16 [total][n_heads][D] dense, not over q; rows of no sequence are left as they were.
 * Rows without a page are left out and record DL_ERR_INVALID_ARG with b.  A row whose scores hold a NaN or +infinity among
 * what it sees is NaN.  NaN and infinities in rows that nobody may see do not matter; in v of a node, they may reach every row of
 * its tree (0 * NaN in a matrix product). */
int32_t dl_kv16_attn_tree(dl_ctx* ctx, const dl_pages* pages, int32_t n_kv_heads, const void* pool, const void* q,
                          int64_t q_stride, const int32_t* starts, int32_t total, int32_t max_rows, const int32_t* mask,
                          int32_t words, float scale, void* out, void* stream);

enum {
  DL_VERIFY_GREEDY = 0,      /* a node is accepted iff its token is the first largest of `target`'s row; draft, u not read */
  DL_VERIFY_SAMPLE = 1,      /* a node's children were drawn from its row of `draft` one after the other, without replacement */
  DL_VERIFY_REPLACED = 2,    /* ... with replacement */
  DL_VERIFY_POINT = 3        /* children were chosen without randomness; draft not read */
};

/* Verifies drafted trees against the target's distributions so that what is kept is distributed as the target's own samples.
 * Nodes as in dl_tree_plan; target[row] (and draft[row]) is the distribution behind that node.  In the order of their
 * numbers, nodes whose parent is the node reached so far (at first the root, node 0) are tested; an accepted one is the node
 * reached.  With p, q the rows of the node reached, and s = 0, R = 1, a = 1 when it is reached, token c of a child with number u
 *   is accepted iff  a > 0 and (u q(c)) R < r(c) a,  r(v) = p(v) - s q(v) held to [0, 1];   if not, and a > 0:  s += R / a,
 *   R = sum of r under the new s, a -= q(c) (REPLACED: a stays 1).
 *   POINT: accepted iff u R < p(c); if not, R -= p(c), and p(c) counts as 0 from then on.
 * At the end a token is drawn from r as it is there, or from p (held to [0, 1]) if all of r is 0, with the root's number u: the first
 * v at which the running sum exceeds u times the whole.  These steps are defined bit for bit: fp64 operations in the order
 * written, sums over r of trunc(r * 2^44), the drawn token's bound (trunc(u * 2^31) * sum) >> 31; no result depends on timing.
 * GREEDY compares values (NaN counts as -infinity; -0 equals +0) and draws the first largest.
 *   target dev [total][vocab] fp32 probabilities, or with GREEDY fp32 or bf16 (`dtype`), probabilities or logits alike;
 *   draft dev [total][vocab] fp32 or NULL; row strides in elements (0: vocab); u dev [total] in [0, 1) (outside: held
 *   to it, below and NaN as 0, from 1 on as the last fp32 number below 1, the root's as 1 - 2^-31);
 *   tokens, parent dev [total] (the root's are not read);
 *   keep_out dev [total]: 1 for the root and the accepted nodes, else 0; count_out dev [B]: their number; next_out dev [B]: the
 *   token drawn; a sequence without nodes gets 0 and -1.  vocab up to 262144, up to 2048 nodes a sequence (those
 *   behind are not reached, and DL_ERR_INVALID_ARG is recorded with the sequence).
 * A token outside the vocabulary is rejected without further effect, a parent as in dl_tree_plan is never reached; both record
 * DL_ERR_INVALID_ARG with the sequence, as a row without any positive entry does (next -1). */
int32_t dl_tree_verify(dl_ctx* ctx, const void* target, int32_t dtype, int64_t target_stride, const float* draft,
                       int64_t draft_stride, const float* u, const int32_t* tokens, const int32_t* parent,
                       const int32_t* starts, int32_t B, int32_t total, int32_t vocab, int32_t mode, uint8_t* keep_out,
                       int32_t* count_out, int32_t* next_out, void* stream);

/* Keeps, of every sequence's rows behind len[b] (the nodes [starts[b], starts[b + 1]) appended there), those whose keep flag is not
 * 0: they move up to row len[b] and on, in order, in all pools, and len[b] += their number.  Rows behind them stay as they are.
 *   pools HOST array of n_pools dev pointers, none of them twice; starts dev [B + 1]; keep dev [total].
 * A sequence that lacks a page of these rows is left as it was and records DL_ERR_CAPACITY with its index. */
int32_t dl_kv16_commit(dl_ctx* ctx, const dl_pages* pages, int32_t n_kv_heads, int32_t n_pools, void* const* pools,
                       const int32_t* starts, const uint8_t* keep, int32_t total, void* stream);

/* ---- checked build ---------------------------------------------------------------------- */

/* The library can be built with -DDL_BOUNDS=1 (libdl_sparse_checked.so): every store a kernel makes through an
 * index it computed (cache rows, outputs, partial sums, masks, index lists) is then compared with the extent of its
 * buffer first; an index outside it is NOT used: the store is skipped and DL_ERR_BOUNDS is recorded in the status
 * word with detail = (kernel id << 48) | index.  Nothing traps.  Copies made by the TMA unit are clipped by their
 * tensor maps in either build.  Results are the same as the normal build's; it is slower. */

/* 1 in the checked build, 0 otherwise. */
int32_t dl_build_is_checked(void);

/* Makes one checked store with an index one past the end of a small buffer inside the workspace.  Checked build:
 * the store is skipped, the buffer unchanged, DL_ERR_BOUNDS recorded (kernel id 0x7e, index 64); normal build:
 * DL_ERR_UNSUPPORTED, nothing launched.  Asynchronous on `stream`; needs the workspace. */
int32_t dl_selftest_bounds(dl_ctx* ctx, void* stream);

/* ---- decode attention without any allocation ------------------------------------------- */

/* Size of the library's built-in scratch array (bytes). */
#define DL_STATIC_SCRATCH_BYTES (8u << 20)

/* The paper has no counterpart to this call; it exists for integration reasons only.
 *
 * Same computation, arguments and results as dl_sparse_attn_decode, for callers that must not
 * allocate device memory: code running inside another framework's memory pool or under a fixed
 * memory budget, plugins that are handed their buffers and nothing else, or processes that are
 * already close to the device's capacity and cannot afford a failing cudaMalloc.  Such callers
 * have no workspace to give to dl_set_workspace; here the split partials and arrival tickets
 * live in a fixed array of DL_STATIC_SCRATCH_BYTES that is part of the library image (each GPU
 * that loads the library holds it until the process exits).  The context needs no workspace;
 * without one, device-side conditions (a full cache on append) are skipped silently instead
 * of being recorded.
 *
 *   - Needs  B*H*4 (rounded up to 256) + B*H*(c + 1)*(D+2)*4  bytes of that array, where c is
 *     the largest number of pieces one sequence may be split into: min(cap/64, max(1, W/(B*H)))
 *     with W = 8 warps per SM of the device (16 for fp32 or head_dim 64), or ceil(cap/chunk)
 *     when DL_OPT_DECODE_CHUNK is set.  Large batches are not split (c = 1).  A larger problem
 *     is refused with DL_ERR_WORKSPACE and nothing is launched.
 *   - The first call on a device looks the array's device address up (cudaGetSymbolAddress, with
 *     that device current); make that first call outside any stream capture.
 *   - The call issues one asynchronous memset (the tickets must start at zero; the array keeps
 *     the previous call's contents) and one kernel on `stream`.  It calls no cudaMalloc/cudaFree.
 *   - All calls on a device share the one array: two calls that may overlap on the GPU (different
 *     streams, or different contexts) race on it.  Serialise them on one stream. */
int32_t dl_sparse_attn_decode_static(dl_ctx* ctx, const void* q_t, const void* k_t, const void* v_t,
                                     void* k_cache, void* v_cache, const int32_t* cache_len,
                                     const uint8_t* keep, int32_t B, int32_t cap, float scale, void* out,
                                     void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DL_SPARSE_H_ */
