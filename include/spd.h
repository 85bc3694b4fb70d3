/*
 * spd.h -- C ABI of the MI355X (gfx950) speculative-decoding hot path.
 *
 * The library implements the data-parallel part of speculative decoding (SPD)
 * for a LLaVA-style multimodal LLM, after "On Speculative Decoding for
 * Multimodal Large Language Models" (arXiv 2404.08856):
 *
 *   - the target verification step: ONE forward pass of a LLaMA-architecture
 *     decoder over the gamma+1 tokens [t, d_1..d_gamma] against a KV cache that
 *     already holds the image-embedding prefix V_1..V_m and the text prefix
 *     X_1..X_n (Section 2.1; Section 2.2, Eq. 1; Section 3);
 *   - the draft model's autoregressive steps (Section 2.1; text-only draft,
 *     Section 3) -- the same kernels at a smaller shape;
 *   - the accept/reject rule min{1, T/D} and the residual resample from
 *     max(0, T - D) (Section 2.1), plus the bonus token on full acceptance
 *     (implied by the maximum block efficiency gamma+1, Section 4 Metrics).
 *
 * Notation: T(x) = target probability, D(x) = draft probability (the paper
 * writes q and p; other texts swap the letters).
 *
 * Conventions
 *   - Every function returns an int32 status (SPD_OK = 0, negative = error) and
 *     never throws.  spd_last_error() returns a static description of the last
 *     error of the calling thread.
 *   - Pointers are DEVICE pointers unless the name starts with h_ (host).
 *   - All device work is enqueued on the caller's hipStream_t, passed as void*
 *     (NULL = the default stream).  No call synchronises the device, except the few
 *     whose comment says so (spd_kv_lens_to_device / _from_device, spd_device_status,
 *     spd_trace_read).
 *   - The library allocates no device memory: weights (packed), KV cache and
 *     workspace live in caller-owned buffers whose sizes spd_model_bytes()
 *     reports.  The model borrows them until spd_model_destroy().
 *   - Shapes: d_model % 32 == 0, head_dim in {64, 128}, (n_heads*head_dim) % 32
 *     == 0, d_ffn % 8 == 0, vocab % 16 == 0, max_seqs <= 64, rows per call
 *     (n_seqs * M) <= 64, M <= 8.  Violations return SPD_ERR_SHAPE before anything is launched.
 */
#ifndef SPD_H
#define SPD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPD_OK               0
#define SPD_ERR_INVALID_ARG (-1)
#define SPD_ERR_SHAPE       (-2)
#define SPD_ERR_CAPACITY    (-3)   /* KV cache / workspace / row limit exceeded */
#define SPD_ERR_HIP         (-4)   /* a HIP runtime call failed; see spd_last_error() */

#define SPD_MAX_ROWS         64    /* rows (n_seqs * M) per forward call          */
#define SPD_MAX_M             8    /* new tokens per sequence per forward call    */

#define SPD_MAX_TOP          32    /* alternatives per row of spd_token_logprobs      */
#define SPD_MAX_LOGPROB_VOCAB (1 << 24)  /* entries per row of spd_token_logprobs       */
#define SPD_MAX_LOGPROB_ROWS  ((1 << 22) - 1)  /* its rows, times vocab / 32768 rounded up    */
#define SPD_Q4_MAX_K          (1 << 24)  /* in_features of a matrix in 4 bits; out_features times in_features / 512 rounded up: 2^26 - 4 at most */

/* flags of spd_speculative_accept */
#define SPD_TARGET_IS_PROBS  1u    /* target rows are probabilities, not logits   */
#define SPD_DRAFT_IS_PROBS   2u    /* draft rows are probabilities, not logits    */

/* flags of spd_token_logprobs, spd_q4_quantize / spd_q4_dequantize, spd_q4_matmul, spd_rope_apply, spd_paged_append, spd_paged_attention */
#define SPD_ROWS_ARE_PROBS   1u    /* rows are probabilities, not logits          */
#define SPD_W_IS_BF16        1u    /* weights bfloat16, else float32              */
#define SPD_X_IS_BF16        1u    /* activations bfloat16, else float32          */
#define SPD_ROPE_INVERSE     2u    /* spd_rope_apply: by the negative angles      */

#define SPD_MAX_HEAD_DIM     256   /* spd_rope_apply; the paged calls: head_dim 64 or 128 */
#define SPD_MAX_PAGED_SEQS   4096  /* sequences per paged call                    */
#define SPD_MAX_PAGED_ROWS   (1 << 20)  /* rows per paged call, and of spd_rope_apply  */
#define SPD_MAX_PAGED_HEADS  1024  /* heads of a row                              */
#define SPD_MAX_PAGED_POSITIONS (1 << 30)  /* positions a row of a page table reaches */
#define SPD_MAX_PAGED_ROW_HEADS (1 << 27)  /* spd_paged_append: rows times heads of q, k and v together */

typedef struct spd_model spd_model;

/* Shape of a LLaMA-architecture decoder (Appendix A.1, Table 1) + capacities. */
typedef struct {
    int32_t n_layers, d_model, n_heads, head_dim, d_ffn, vocab;
    float   rms_eps;           /* RMSNorm epsilon (inside the square root)        */
    float   rope_theta;        /* RoPE base; pair (i, i+head_dim/2), freq theta^(-2i/head_dim) */
    int32_t tied_embeddings;   /* 1: LM head = embedding table                    */
    int32_t max_seqs;          /* sequences the KV cache holds                    */
    int32_t max_positions;     /* positions per sequence the KV cache holds       */
} spd_model_config;

/* Unpacked weights, device memory, row-major [out_features, in_features],
 * bfloat16 matrices and float32 norm gains.  The per-layer members are HOST
 * arrays of n_layers device pointers.  Only read during spd_model_create (and
 * the work it enqueues): once that work has finished the caller may free them. */
typedef struct {
    const void  *embed;              /* bf16 [vocab, d_model]                      */
    const void  *lm_head;            /* bf16 [vocab, d_model]; NULL if tied        */
    const float *final_norm;         /* f32  [d_model]                             */
    const float *const *attn_norm;   /* f32  [d_model] per layer                   */
    const void  *const *wq;          /* bf16 [n_heads*head_dim, d_model]           */
    const void  *const *wk;
    const void  *const *wv;
    const void  *const *wo;          /* bf16 [d_model, n_heads*head_dim]           */
    const float *const *mlp_norm;    /* f32  [d_model]                             */
    const void  *const *w_gate;      /* bf16 [d_ffn, d_model]                      */
    const void  *const *w_up;        /* bf16 [d_ffn, d_model]                      */
    const void  *const *w_down;      /* bf16 [d_model, d_ffn]                      */
} spd_weights;

/* A matrix [out_features N, in_features K] in 4 bits: W[n][k] = scale[n][k / group] * q[n][k].
 *   q       uint8 [N, ceil(K / 2)]: integers -8..7 in two's complement, even columns in the low half of their byte
 *   scales  bfloat16 [N, ceil(K / group)]; group is 32, 64 or 128, the last group of a row may be shorter
 * Both device memory.  spd_q4_quantize makes them; any other quantiser's in this form will do. */
typedef struct {
    const void *q, *scales;
} spd_q4_matrix;

/* Weights of a model whose matrices are in 4 bits (shapes as in spd_weights; embedding table bfloat16, gains float32).
 * lm_head is always given, also with tied embeddings. */
typedef struct {
    int32_t       group;
    const void   *embed;
    spd_q4_matrix lm_head;
    const float  *final_norm;
    const float *const *attn_norm;                    /* per layer, as in spd_weights */
    const spd_q4_matrix *wq, *wk, *wv, *wo;
    const float *const *mlp_norm;
    const spd_q4_matrix *w_gate, *w_up, *w_down;
} spd_weights_q4;

/* Description of the last error on this thread ("" if none).  Host pointer,
 * valid until the next failing call on the same thread. */
const char *spd_last_error(void);

/* Sizes (bytes) of the three caller-owned device buffers of a model:
 * packed weights (matrices re-tiled for the matrix cores + gains + embedding
 * table), KV cache (bf16, K after RoPE and V, all layers) and workspace. */
int32_t spd_model_bytes(const spd_model_config *h_cfg, size_t *h_packed_bytes,
                        size_t *h_kv_bytes, size_t *h_workspace_bytes);

/* Builds a model (target or draft) over caller-owned buffers: enqueues the
 * re-tiling of every matrix of *h_weights into `packed`, the RoPE table and the
 * clearing of the workspace on `stream`.  All KV lengths start at 0.
 * Errors: SPD_ERR_SHAPE (unsupported shape), SPD_ERR_CAPACITY (a buffer is
 * smaller than spd_model_bytes says), SPD_ERR_INVALID_ARG (NULL/misaligned;
 * buffers must be 256-byte aligned), SPD_ERR_HIP. */
int32_t spd_model_create(const spd_model_config *h_cfg, const spd_weights *h_weights,
                         void *packed, size_t packed_bytes, void *kv_cache, size_t kv_bytes,
                         void *workspace, size_t workspace_bytes, void *stream,
                         spd_model **h_out);

/* The same for a model whose matrices stay in 4 bits (spd_weights_q4): 3.8 times fewer bytes per step at groups of 128.  All
 * calls on such a model are those of any other.  Its products have float32 activations and sums as the bf16 model's have, and in
 * prompts of many rows their exactness.  In the other calls an activation counts as in spd_q4_matmul, to 2^-29 of the largest one of its
 * row, where the bf16 model keeps 24 bits of each: the model differs from a bf16 model of the dequantised weights by float32 rounding, and,
 * where some activations of a row are more than about 1000 times the rest, by up to 2^-29 of those in each of the rest.  A row of activations with a
 * value that is not finite gives NaN.  Of spd_tuning only the attention's fields, batch_kernel (prompts in passes of 64 or 40 rows) and
 * wait_spin_limit have an effect.  The workspace also holds one matrix at 16 bits, for prompts.  Errors as spd_model_create, SPD_ERR_SHAPE for another group. */
int32_t spd_model_bytes_q4(const spd_model_config *h_cfg, int32_t group, size_t *h_packed_bytes,
                           size_t *h_kv_bytes, size_t *h_workspace_bytes);
int32_t spd_model_create_q4(const spd_model_config *h_cfg, const spd_weights_q4 *h_weights,
                            void *packed, size_t packed_bytes, void *kv_cache, size_t kv_bytes,
                            void *workspace, size_t workspace_bytes, void *stream,
                            spd_model **h_out);

int32_t spd_model_destroy(spd_model *model);

/* Kernel-selection knobs of a model, for tests and sweeps (not part of the method; production
 * code never needs this call: spd_model_create picks the measured defaults).  Zero-initialise the
 * struct for "all defaults".  Takes effect from the next forward; host-side only.  All fields but wait_spin_limit choose
 * among the kernels of single projections: while one of them is set, the layers of a small model, by default one
 * launch for calls of up to 5 rows where that is faster, run kernel by kernel.  (That launch takes nearly the whole GPU until
 * it ends: work on other streams that used to run beside a draft's short kernels waits for up to a whole step.  All of
 * it together is done sooner; a program to which the other stream's latency matters more sets separate_qkv_attention.)
 * Projections are indexed qkv, o, gate_up, down, lm_head. */
#define SPD_N_PROJECTIONS 5
typedef struct {
    int32_t  separate_qkv_attention; /* 1: QKV projection and attention always as two kernels;
                                        0 = default: one kernel where the shape allows */
    int32_t  attention_slices;       /* workgroups per head of the stand-alone attention kernel at head_dim 128:
                                        1, 2, 4 or 8; 0 = chosen by batch size and length of the caches */
    int32_t  gemm_waves[SPD_N_PROJECTIONS];          /* waves per workgroup: 4, 8 or 16; 0 = default */
    int32_t  gemm_grid_cap[SPD_N_PROJECTIONS];       /* upper bound of the grid; 0 = default         */
    int32_t  gemm_general_kernel[SPD_N_PROJECTIONS]; /* 1: never the register-resident variant       */
    int32_t  gemm_ring[SPD_N_PROJECTIONS];           /* general kernel: weight blocks a wave keeps in flight, 8 or 16; 0 = default */
    int32_t  batch_kernel;           /* calls of more than 5 rows, where no register-resident kernel fits: 0 = the library
                                        chooses per projection between the tile-splitting batched kernel (one pass over
                                        the weights for up to 64 rows) and the K-splitting kernels (passes of 40 rows);
                                        1 = the former, 2 = the latter, also where the library would not.  (At 6 to 10 rows a
                                        matrix of fewer than 256 tiles of 16 columns takes the general kernel at any setting,
                                        and one of more than 262144 columns the K-splitting kernels.)  1 and 2 also keep
                                        prompts on the batched verify path */
    uint32_t wait_spin_limit;        /* polls before a wait between workgroups gives up and raises the flag that
                                        spd_device_status reports (0 = default, 2^22); a tiny value lets a test
                                        drive that error path from the host while every kernel still exits */
} spd_tuning;
int32_t spd_model_set_tuning(spd_model *model, const spd_tuning *h_tuning);

/* Sets the number of valid KV positions of sequences 0..n_seqs-1 (rollback
 * after a rejection, reset to 0, ...).  Host-side bookkeeping only: positions
 * >= the new length are simply overwritten by later calls.
 * Errors: SPD_ERR_CAPACITY if a length exceeds max_positions or n_seqs exceeds
 * max_seqs, SPD_ERR_INVALID_ARG on negative values. */
int32_t spd_kv_set_len(spd_model *model, const int32_t *h_len_per_seq, int32_t n_seqs);
int32_t spd_kv_get_len(const spd_model *model, int32_t *h_len_per_seq, int32_t n_seqs);

/* Inspection (tests, baselines; not part of the method): the cached keys (after RoPE) and values of
 * positions pos0 .. pos0+n-1 of one layer and sequence as float32 [n, n_heads, head_dim] each (the cache
 * itself is bfloat16 in layouts of the library's own).  Positions need not be below the current KV
 * length: whatever the cache holds there is returned.  Errors: SPD_ERR_INVALID_ARG, SPD_ERR_CAPACITY
 * (positions outside max_positions). */
int32_t spd_kv_export(spd_model *model, int32_t layer, int32_t seq, int32_t pos0, int32_t n,
                      float *k_out, float *v_out, void *stream);

/* Not hot: feeds n_rows input-embedding rows (float32 [n_rows, d_model],
 * e.g. [V_1..V_m ; E[X_1..X_n]] for the target, Section 2.2 Eq. 1) to sequence
 * `seq` starting at its current KV length, appending their K, V.  If
 * last_logits != NULL it receives the float32 logits [vocab] of the last row.
 * Long runs go through kernels of their own, up to 2048 rows per pass over the weights (the workspace
 * holds the activations of one such pass, or of max_positions rows if that is less); short ones run as
 * passes of a batched verify step. */
int32_t spd_prefill(spd_model *model, int32_t seq, const float *embeds, int32_t n_rows,
                    float *last_logits, void *stream);

/* Same, from token ids (int32 [n_rows]); the text-only draft's prefill (Section 3). */
int32_t spd_prefill_tokens(spd_model *model, int32_t seq, const int32_t *tokens, int32_t n_rows,
                           float *last_logits, void *stream);

/* HOT.  One decoder forward over M new tokens for each of sequences
 * 0..n_seqs-1, starting at each sequence's current KV length: the single
 * target call that yields T_1..T_{gamma+1} when tokens = [t, d_1..d_gamma] and
 * M = gamma+1 (Section 2.1, Section 3); M = 1 is plain autoregressive decoding.
 * tokens: int32 [n_seqs, M].  logits_out: float32 [n_seqs, M, vocab]; row j is
 * the distribution of the token after input j.  Appends the M keys/values of
 * every sequence and advances its KV length by M (roll back with
 * spd_kv_set_len).  Errors: SPD_ERR_SHAPE (M > 8 or n_seqs*M > 64),
 * SPD_ERR_CAPACITY (KV overflow; nothing is launched). */
int32_t spd_verify_forward(spd_model *target, const int32_t *tokens, int32_t n_seqs, int32_t M,
                           float *logits_out, void *stream);

/* HOT.  One draft decode step (Section 2.1: d_j ~ D(. | X_1:n, d_1..d_{j-1});
 * Section 3: text-only conditioning): feeds n_in (1 or 2) tokens per sequence
 * -- 2 after a fully accepted block, when the draft has not yet consumed
 * d_gamma -- and from the logits of the last one writes
 *   D_row_out  float32 [n_seqs, vocab]  softmax(logits / temperature)
 *   token_out  int32   [n_seqs]         drawn from D_row with the fixed-point
 *                                        inverse-CDF sampler and u_draft[n_seqs];
 * temperature 0: D_row is one-hot at the argmax (lowest index on ties).
 * tokens_in: int32 [n_seqs, n_in].  Advances the draft's KV lengths by n_in. */
int32_t spd_draft_step(spd_model *draft, const int32_t *tokens_in, int32_t n_seqs, int32_t n_in,
                       float temperature, const float *u_draft, float *D_row_out,
                       int32_t *token_out, void *stream);

/* HOT.  Speculative sampling for n_seqs sequences x gamma drafted tokens
 * (Section 2.1; Section 3 for the multimodal conditioning of T).
 *   target        float32 [n_seqs, gamma+1, vocab]  logits, or probabilities with SPD_TARGET_IS_PROBS
 *   draft         float32 [n_seqs, gamma, vocab]    logits, or probabilities with SPD_DRAFT_IS_PROBS
 *   draft_tokens  int32   [n_seqs, gamma]
 *   u             float32 [n_seqs, gamma+1] on the grid j/2^24: u[:, :gamma] drive the
 *                 accept tests, u[:, gamma] the replacement / bonus draw
 * Per sequence: k = number of leading j with u_j * D_j(d_j) < T_j(d_j) (float32
 * multiply and compare: accept probability min{1, T/D}); then the next token y
 * is drawn from max(0, T_{k+1} - D_{k+1}) normalised if k < gamma, else from
 * T_{gamma+1}, with the fixed-point inverse-CDF sampler: w(x) = floor(r(x) 2^32),
 * threshold = floor(u 2^24 * sum w / 2^24), y = first x whose running sum
 * exceeds it (if the residual has no representable mass: same draw from T_{k+1}).
 * temperature scales logits (softmax(l / temperature)); temperature 0 = greedy
 * (one-hot rows, lowest index on ties); it is ignored for probability inputs.
 *   n_accepted_out  int32 [n_seqs]      k
 *   next_token_out  int32 [n_seqs]      y
 *   accept_prob_out float32 [n_seqs, gamma] or NULL: min{1, T_j(d_j)/D_j(d_j)}
 *   workspace       float32 scratch, >= spd_accept_workspace_bytes(...) bytes; it may hold anything before the call,
 *                   and nothing in it has to survive between calls.  Calls that share one must not overlap; the results of
 *                   calls that do are undefined, those of later calls are not, with one exception: a call captured in a
 *                   graph that overlapped with another needs the workspace cleared before its next replay
 * Errors: SPD_ERR_INVALID_ARG (NULL, gamma < 1, temperature < 0),
 * SPD_ERR_CAPACITY (workspace too small). */
int32_t spd_accept_workspace_bytes(int32_t n_seqs, int32_t gamma, int32_t vocab, size_t *h_bytes);
int32_t spd_speculative_accept(const float *target, const float *draft, const int32_t *draft_tokens,
                               const float *u, int32_t n_seqs, int32_t gamma, int32_t vocab,
                               float temperature, uint32_t flags, int32_t *n_accepted_out,
                               int32_t *next_token_out, float *accept_prob_out,
                               void *workspace, size_t workspace_bytes, void *stream);

/* For callers that cannot allocate device memory or pass a workspace (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): spd_speculative_accept with its scratch memory in
 * a fixed 64 KiB array inside the library (one copy per GPU, held until the process ends).  Same
 * arguments, results and errors as spd_speculative_accept, minus the workspace; calls nothing that
 * allocates.  Limit: n_seqs * (2 gamma + 1) <= SPD_STATIC_ACCEPT_MAX_ROWS, else SPD_ERR_CAPACITY and
 * nothing is launched.  All calls on one GPU share that GPU's array: calls that may overlap (different
 * streams, different threads) race on it -- order them, or use spd_speculative_accept with one
 * workspace per stream (a captured call that did overlap has to be captured again).  Nothing in the array has to
 * survive between calls. */
#define SPD_STATIC_ACCEPT_MAX_ROWS 4096
int32_t spd_speculative_accept_static(const float *target, const float *draft, const int32_t *draft_tokens,
                                      const float *u, int32_t n_seqs, int32_t gamma, int32_t vocab,
                                      float temperature, uint32_t flags, int32_t *n_accepted_out,
                                      int32_t *next_token_out, float *accept_prob_out, void *stream);

/* Log probabilities of given tokens, entropy and the most likely alternatives of rows: what a serving program returns
 * with a token, and how sure a draft is.  Rows may be those of spd_verify_forward, or (SPD_ROWS_ARE_PROBS) of spd_draft_step.
 *   rows    float32 [n_rows, vocab], row_stride elements apart: logits, or probabilities
 *   tokens  int32 [n_rows]; NULL if neither logprob_out nor rank_out is wanted
 *   logprob_out       float32 [n_rows] or NULL: lp(x) = z_x - log(sum exp z) of z = logits / temperature, or log(row[x])
 *   entropy_out       float32 [n_rows] or NULL: -sum p lp, in nats (given probabilities below 2^-126 count as 0 here)
 *   rank_out          int32 [n_rows] or NULL: entries before the token in descending order, equal ones by index (0: the first)
 *   top_tokens_out    int32, top_logprobs_out float32 [n_rows, n_top]: the first n_top entries in that order (0 <= n_top <= SPD_MAX_TOP)
 *   workspace         scratch of spd_logprobs_workspace_bytes bytes (which may be 0; then it may be NULL), 16-byte aligned; it may hold
 *                     anything before the call and nothing in it has to survive it.  Calls that share one must not overlap.
 * temperature >= 4.3e-39, finite (temperature 0 leaves no log probabilities: ask for those at 1); ignored for probabilities.
 * Entries at -infinity (probability 0) weigh nothing and are no alternatives: places they leave hold token -1 and -infinity.  A
 * row of nothing else: log probability -infinity, entropy 0.  Finite entries more than 3.4e38 below the largest weigh nothing either (but are alternatives).  A token outside 0..vocab-1: -infinity, rank vocab.  A row with a NaN or
 * +infinity (probabilities: a negative or infinite one or a NaN) has no distribution: NaN, rank and alternatives -1.
 * Errors: SPD_ERR_INVALID_ARG, SPD_ERR_SHAPE (vocab > SPD_MAX_LOGPROB_VOCAB, too many rows), SPD_ERR_CAPACITY (workspace too small). */
int32_t spd_logprobs_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t n_top, size_t *h_bytes);
int32_t spd_token_logprobs(const float *rows, size_t row_stride, const int32_t *tokens, int32_t n_rows, int32_t vocab,
                           float temperature, uint32_t flags, float *logprob_out, float *entropy_out, int32_t *rank_out,
                           int32_t n_top, int32_t *top_tokens_out, float *top_logprobs_out,
                           void *workspace, size_t workspace_bytes, void *stream);

/* ---- weights in 4 bits (format: spd_q4_matrix) -----------------------------------------------------
 * spd_q4_quantize: a = the largest magnitude of a group, scale = a * (float32)(1 / 7) rounded to bfloat16, q = w / scale (float32) rounded to the nearest
 * integer (even on ties), limited to -8..7; 0 where the scale is 0.  A group with a value that is not finite: scale NaN, q 0.
 * w: float32, or bfloat16 with SPD_W_IS_BF16, [N, K] with w_stride elements between rows.
 * spd_q4_dequantize: the values that q and scales stand for (rounded once if bfloat16).
 * spd_q4_pack: re-tiles a matrix for the matrix cores into `packed` (spd_q4_bytes bytes, 256-byte aligned), which spd_q4_matmul reads.
 * Errors: SPD_ERR_INVALID_ARG, SPD_ERR_SHAPE (N or K < 1, another group, too large), SPD_ERR_CAPACITY. */
int32_t spd_q4_bytes(int32_t N, int32_t K, int32_t group, size_t *h_packed_bytes);
int32_t spd_q4_quantize(const void *w, size_t w_stride, uint32_t flags, int32_t N, int32_t K, int32_t group,
                        void *q_out, void *scales_out, void *stream);
int32_t spd_q4_dequantize(const void *q, const void *scales, int32_t N, int32_t K, int32_t group,
                          void *w_out, size_t w_stride, uint32_t flags, void *stream);
int32_t spd_q4_pack(const void *q, const void *scales, int32_t N, int32_t K, int32_t group,
                    void *packed, size_t packed_bytes, void *stream);

/* y[r][n] = sum over k of x[r][k] W[n][k] for rows <= SPD_MAX_ROWS rows: x float32, or bfloat16 with SPD_X_IS_BF16, x_stride
 * elements between rows, y float32, y_stride between rows.  Exact products, float32 sums; an entry of x counts to 2^-29 of the
 * largest magnitude of its row, to 2^-23 of itself or to 2^-120, whichever is most; scales of
 * magnitudes between 2^-100 and 2^100, 0 and NaN (in whose rows of W y is NaN).  A row of x with a value that is not finite gives NaN.  y must not overlap x.
 * workspace: spd_q4_matmul_workspace_bytes bytes (which may be 0; then it may be NULL), 256-byte aligned; it may hold anything before the
 * call and nothing in it has to survive it.  Calls that share one must not overlap.
 * Errors: SPD_ERR_INVALID_ARG, SPD_ERR_SHAPE, SPD_ERR_CAPACITY (workspace too small). */
int32_t spd_q4_matmul_workspace_bytes(int32_t rows, int32_t N, int32_t K, size_t *h_bytes);
int32_t spd_q4_matmul(const void *packed, int32_t N, int32_t K, int32_t group, const void *x, size_t x_stride,
                      uint32_t flags, int32_t rows, float *y, size_t y_stride,
                      void *workspace, size_t workspace_bytes, void *stream);

/* ---- rotary positions -------------------------------------------------------------------------------
 * Pair i < rotary_dim / 2 of a head is turned by the angle position * f_i:  (a, b) -> m (a cos - b sin, a sin + b cos), its elements
 * i and i + rotary_dim / 2, or (interleaved) 2 i and 2 i + 1; elements from rotary_dim on stay as they are.
 *   f_i = theta^(-2 i / rotary_dim) / h_factors[i] (h_factors NULL: 1), then by `scaling`, with t_i = original_positions f_i / (2 pi), the
 *   pair's turns over the context that the model was trained on:
 *     SPD_ROPE_NONE      f_i
 *     SPD_ROPE_LINEAR    f_i / factor
 *     SPD_ROPE_RAMP      f_i (r + (1 - r) / factor),  r = (t_i - low) / (high - low) limited to 0..1
 *     SPD_ROPE_LOG_RAMP  the same with r = (ln t_i - ln low) / (ln high - ln low)
 *   m = magnitude (1 if the model states none).
 * Positions are any int32, negative ones too: a frequency is held as a 64-bit fraction of a turn, so that the angle's place within its
 * turn is exact to 2^-32 turns however far the position (of frequencies of up to a turn a position, 2 pi; one of 2^n turns loses n of its 64 bits).
 * SPD_ROPE_LOG_RAMP is linear in the pair's index i between the indices where t_i is high and low.  Models that round those two to whole indices get the same by
 * the low and high that belong to the whole ones: t_i = original_positions theta^(-2 i / rotary_dim) / (2 pi).
 * spd_rope_table makes the frequencies' table (spd_rope_table_bytes bytes, 16-byte aligned) once; spd_rope names it in the calls. */
#define SPD_ROPE_NONE     0
#define SPD_ROPE_LINEAR   1
#define SPD_ROPE_RAMP     2
#define SPD_ROPE_LOG_RAMP 3
typedef struct {
    int32_t      rotary_dim;          /* even, 2..SPD_MAX_HEAD_DIM                  */
    int32_t      scaling;
    float        theta;               /* > 0                                        */
    float        factor, low, high;   /* factor > 0; ramps: high > low (log: low > 0) */
    float        original_positions;  /* ramps: > 0                                 */
    float        magnitude;
    const float *h_factors;           /* host, [rotary_dim / 2], > 0; or NULL       */
} spd_rope_config;
typedef struct {
    const void *table;
    int32_t     rotary_dim, interleaved;
} spd_rope;

/* Rows of heads: head h of row r starts row_stride r + head_stride h elements behind `data`, its elements are neighbours. */
typedef struct {
    void  *data;
    size_t row_stride, head_stride;
} spd_heads;

/* out = x turned, head_dim elements of each of n_heads heads of n_rows rows; float32, or bfloat16 with SPD_X_IS_BF16 (rounded once).
 * positions: int32 [n_rows].  out may be x itself (the same data and strides); otherwise the two must not overlap.
 * SPD_ROPE_INVERSE turns by the negative angles: the gradient of x from that of out, or, with magnitude 1, the turn taken back.
 * Errors: SPD_ERR_INVALID_ARG (NULL, strides, unknown flags, a config's values), SPD_ERR_SHAPE (rotary_dim odd or above head_dim,
 * head_dim above SPD_MAX_HEAD_DIM, rows or heads out of range), SPD_ERR_CAPACITY (table too small). */
int32_t spd_rope_table_bytes(int32_t rotary_dim, size_t *h_bytes);
int32_t spd_rope_table(const spd_rope_config *h_cfg, void *table, size_t table_bytes, void *stream);
int32_t spd_rope_apply(const spd_rope *h_rope, const spd_heads *h_x, const spd_heads *h_out, const int32_t *positions, int32_t n_rows,
                       int32_t n_heads, int32_t head_dim, uint32_t flags, void *stream);

/* ---- a paged cache of keys and values, and attention over it -------------------------------------------------------
 * The cache of one layer: n_pages pages of page_size positions (16, 32, 64, 128 or 256) of n_kv_heads heads of head_dim elements (64 or
 * 128), in granules of 16 bytes, G elements (bfloat16: 8; e4m3: 16), laid out as the matrix cores read them:
 *   k  [n_pages][n_kv_heads][head_dim / G][page_size][G]       element d of slot p: granule d / G, row p
 *   v  [n_pages][n_kv_heads][page_size / G][head_dim][G]       slot p of element d: granule p / G, row d
 * e4m3 (OCP: largest 448, no infinities): an element stands for itself times the scale of its head, k_scale / v_scale
 * float32 [n_kv_heads], positive, device memory.  A page may be anyone's: several sequences' rows of the table may name it. */
typedef struct {
    void        *k, *v;                        /* 16-byte aligned */
    const float *k_scale, *v_scale;            /* e4m3; else NULL */
    int32_t      n_pages, page_size, n_kv_heads, head_dim, e4m3;
} spd_paged_cache;

/* The new rows of a call: those of sequence s are row_start[s] .. row_start[s + 1] - 1 (row_start int32 [n_seqs + 1], ascending; NULL: n_rows / n_seqs
 * rows each), and row i of them has position lens[s] + i, lens int32 [n_seqs] the positions cached before.  Position p lies in slot
 * p % page_size of page page_table[s * table_stride + p / page_size], p < max_pages * page_size.  All device memory.
 * Rows behind row_start[n_seqs] belong to nobody: nothing is written for them.  A position beyond the table, or whose entry is not in
 * 0..n_pages-1, is no place: nothing is appended there and nobody sees it (entries of pages that were given up may be -1).
 * A length below 0 counts as 0, one beyond the table as its end. */
typedef struct {
    int32_t        n_seqs, n_rows, max_pages;
    size_t         table_stride;
    const int32_t *page_table, *lens, *row_start;
} spd_paged_batch;

/* Appends the rows' keys and values (n_kv_heads heads of head_dim; rounded once to bfloat16, or the float32 quotient x / scale to the nearest e4m3,
 * ties to even, limited to +-448; NaN stays NaN).  h_rope not NULL: keys are turned first, by positions[r] (int32 [n_rows]) or, if that is NULL, by the rows' own.
 * h_q not NULL: n_heads heads of queries are turned in the same launch into h_q_out (which may be h_q itself).
 * Rows float32, or bfloat16 with SPD_X_IS_BF16.  Places that two rows share (a page that two sequences append to) hold either's.
 * Errors: SPD_ERR_INVALID_ARG, SPD_ERR_SHAPE; nothing is launched then. */
int32_t spd_paged_append(const spd_paged_cache *h_cache, const spd_paged_batch *h_batch, const spd_heads *h_k, const spd_heads *h_v,
                         const spd_heads *h_q, const spd_heads *h_q_out, int32_t n_heads, const spd_rope *h_rope, const int32_t *positions,
                         uint32_t flags, void *stream);

/* Attention of the new rows, whose keys and values are in their places by then, over their sequences' positions:
 *   out[r][h] = sum_p softmax_p(scale q[r][h] . k[p]) v[p]      head h reads key head h / (n_heads / n_kv_heads)
 * A row at position x sees p <= x; with window > 0 only p > x - window; with `seen` (uint64 [n_rows]; window 0) the cached
 * positions p < lens[s], and of the sequence's new rows those whose bit is set (bit j: row j; at most 64 rows of a sequence
 * can be seen): a tree of drafted tokens, whose rows have the bits of the tokens that they continue, and their own.
 * Positions that a row does not see weigh nothing, whatever they hold; so do scores of -infinity.  A row that sees nothing: out 0.
 * A key that is not finite and seen may leave its head's row NaN, such a value its element not finite.  A scale of 0 weighs all keys that are seen alike, whatever q holds.
 * lse_out: float32 [n_rows][n_heads] or NULL, log sum exp of the scores (-infinity for a row that sees nothing): with it, parts of
 * a softmax over several caches can be joined.
 * q, out: float32, or bfloat16 with SPD_X_IS_BF16; out must not overlap q.  Sums and statistics are float32.  Products of float32 rows are exact to float32's roundings; with
 * bfloat16 rows the softmax's weights are taken to 16 bits for the product with v, or, where sequences have many rows (a mean of more than 32 rows times n_heads / n_kv_heads,
 * or more than 256 in one), to bfloat16's 8, and divided by the sum of what they were rounded to: out is off by at most 2^-8 of sum_p softmax_p |v[p] - out| before its own rounding.
 * workspace: spd_paged_attention_workspace_bytes bytes, 256-byte aligned; it may hold anything before the call, and nothing in it has to survive
 * it.  Calls that share one must not overlap; the results of calls that do are undefined, those of later calls are not, with one exception: a call captured
 * in a graph that overlapped with another needs the workspace cleared before its next replay.
 * Errors: SPD_ERR_INVALID_ARG, SPD_ERR_SHAPE, SPD_ERR_CAPACITY (workspace too small); nothing is launched then. */
int32_t spd_paged_attention_workspace_bytes(const spd_paged_cache *h_cache, const spd_paged_batch *h_batch, int32_t n_heads, size_t *h_bytes);
int32_t spd_paged_attention(const spd_paged_cache *h_cache, const spd_paged_batch *h_batch, const spd_heads *h_q, const spd_heads *h_out,
                            int32_t n_heads, float scale, int32_t window, const uint64_t *seen, float *lse_out, uint32_t flags,
                            void *workspace, size_t workspace_bytes, void *stream);

/* spd_verify_forward over pages instead of the model's own cache: one forward of the new rows of a batch (ragged ones too, up to SPD_MAX_ROWS
 * together), whose keys and values go into layers[l] of layer l (host array of n_layers; heads and head size those of the model, pages alike in
 * all layers) and whose attention reads them, causal or, with `seen`, over a tree of drafted tokens (then with `positions`, and refused without: what a token's place in
 * its branch says).  tokens: int32 [n_rows].  logits_out: float32 [n_rows, vocab]; those of rows behind the last sequence say nothing.  rope: the
 * model's positions (rotary_dim head_dim, its theta) or others, e.g. stretched for contexts beyond the model's; max_positions bounds nothing here.
 * The model's own cache and lengths stay as they are, the lengths of the batch are the caller's to advance: by the rows that are kept, as long as they are the first ones
 * (everyone sees the positions below a length).  Of an accepted branch of a tree that is not so, the length takes the tokens up to the first gap, and the others go again as the
 * first rows of the next call, which puts their keys and values where they belong.  Prompts go in pieces of up to SPD_MAX_ROWS rows.
 * Works for models in 4 bits too.  Errors as spd_paged_append and spd_paged_attention; SPD_ERR_SHAPE for other heads or more rows. */
int32_t spd_verify_paged_workspace_bytes(const spd_model *model, const spd_paged_cache *h_layers, const spd_paged_batch *h_batch, size_t *h_bytes);
int32_t spd_verify_forward_paged(spd_model *model, const int32_t *tokens, const spd_paged_cache *h_layers, const spd_paged_batch *h_batch,
                                 const spd_rope *h_rope, const int32_t *positions, const uint64_t *seen, float *logits_out,
                                 void *workspace, size_t workspace_bytes, void *stream);

/* ---- the block loop without the host (Section 2.1, one block = gamma draft steps, one
 * target call, accept / resample, commit) ---------------------------------------------
 *
 * With the calls above the host reads k after every block to roll both KV caches back.
 * The calls below keep the KV lengths in device memory, so that a whole block is a fixed
 * sequence of launches with fixed arguments: it can be enqueued back to back, or captured
 * once in a HIP graph and replayed, without a host round trip per block.
 *
 * spd_kv_lens_to_device copies the model's current KV lengths into its workspace and
 * switches the model to device lengths: from then on every forward reads them there and
 * advances them there.  The host copy becomes an upper bound, so KV overflow can no longer
 * be refused before the launch: a forward whose device length leaves no room for its rows
 * works on a clamped length (every access stays in bounds, the results are meaningless) and
 * raises a flag that spd_kv_lens_from_device reports as SPD_ERR_CAPACITY.  Both calls wait
 * for `stream` (they are the only ones besides spd_trace_* that block).  spd_kv_set_len is
 * refused while the lengths live on the device. */
int32_t spd_kv_lens_to_device(spd_model *model, void *stream);
int32_t spd_kv_lens_from_device(spd_model *model, void *stream);

/* spd_draft_step with explicit strides (in elements between consecutive sequences), so that
 * a draft step can read its input from, and write its token and its D row into, the buffers
 * the target call and the accept step use: sequence s reads tokens_in[s * in_stride + i]
 * (i < n_in) and u_draft[s * u_stride], writes D_row_out[s * D_stride + x] (x < vocab) and
 * token_out[s * token_stride]. */
int32_t spd_draft_step_strided(spd_model *draft, const int32_t *tokens_in, int32_t in_stride, int32_t n_seqs,
                               int32_t n_in, float temperature, const float *u_draft, int32_t u_stride,
                               float *D_row_out, size_t D_stride, int32_t *token_out, int32_t token_stride,
                               void *stream);

/* Accept / resample and commit of one block, all on the device.  Both models must be in
 * device-length mode.  Inputs: target_logits float32 [n_seqs, gamma+1, vocab] of the target
 * call over verify_tokens = [t, d_1..d_gamma] (int32 [n_seqs, gamma+1]); draft_probs float32
 * [n_seqs, gamma, vocab], the D rows of the draft steps; u as in spd_speculative_accept.
 * Computes k and y exactly as spd_speculative_accept (target logits, draft probabilities),
 * then per sequence:
 *   - appends d_1..d_k, y to out_tokens[s, n_out[s]..] (int32 [n_seqs, out_capacity], may be
 *     NULL) and adds k+1 to n_out[s] (tokens beyond out_capacity are dropped);
 *   - verify_tokens[s, 0] = y (the next block's t);
 *   - draft_in_out[s] = [token before y, y] (int32 [n_seqs, 2]): the next block's first
 *     draft step takes these two tokens, whether or not the block was fully accepted;
 *   - both models' KV lengths -= gamma - k.
 * Convention of the loop: at the start of a block the target's KV cache holds everything
 * before t and the draft's cache everything before the token that precedes t (so the
 * draft re-computes that one position each block, which makes every block the same shape);
 * the first draft step has n_in = 2, the other gamma-1 steps n_in = 1. */
int32_t spd_block_finish(spd_model *target, spd_model *draft, const float *target_logits, const float *draft_probs,
                         int32_t *verify_tokens, const float *u, int32_t n_seqs, int32_t gamma, float temperature,
                         int32_t *n_accepted_out, int32_t *next_token_out, int32_t *draft_in_out,
                         int32_t *out_tokens, int32_t out_capacity, int32_t *n_out,
                         void *workspace, size_t workspace_bytes, void *stream);

/* Waits for `stream` and reports conditions that kernels can only flag on the device:
 * SPD_ERR_HIP if a bounded wait between workgroups (fused QKV + attention kernel, launch of all layers of a small model) ever ran
 * into its spin limit -- never in a healthy run; results since then are
 * invalid --, SPD_ERR_CAPACITY if a forward in device-length mode found no room for its rows,
 * else SPD_OK. */
int32_t spd_device_status(spd_model *model, void *stream);

/* Tracing aid (not part of the method).  While enabled, every kernel launch group of
 * this model's forward passes is timed with a pair of HIP events (host-side event
 * objects only: no device memory): a group that is a single kernel gets them as the
 * launch's own start / stop events (the kernel's execution time, as a profiler
 * reports it), a group of several launches is bracketed by events recorded on the
 * caller's stream.  Where QKV projection and attention run as one kernel, kind 0
 * covers both and kind 5 stays empty.  The layers of a small model, otherwise one launch for up to 5 rows, run kernel by kernel
 * while tracing is enabled (other kernels than without, and sums in another order).  spd_trace_read WAITS for
 * the recorded events (the one call here that blocks the host), adds the elapsed
 * milliseconds and launch counts per kind into h_ms_sum[n_kinds] / h_count[n_kinds] and
 * forgets them.  Kinds: 0 QKV projection, 1 O projection, 2 gate|up projection + SwiGLU,
 * 3 down projection, 4 LM head, 5 RoPE + KV append + attention, 6 input rows (embedding
 * gather).  The events perturb the stream slightly: time whole steps with tracing off. */
#define SPD_TRACE_KINDS 7
int32_t spd_trace_enable(spd_model *model, int32_t enable);
int32_t spd_trace_read(spd_model *model, int32_t n_kinds, double *h_ms_sum, int32_t *h_count);

/* Measurement aid (not part of the method): launches n_stages plain streaming-read kernels back to back on
 * `stream`, stage i reading h_stage_bytes[i] bytes (multiples of 1024) of `buffer` (any readable device memory
 * of buffer_bytes >= the sum; consecutive repetitions read different windows of it), `reps` times, and reports
 * in microseconds each kernel's own execution time (mean over the repetitions) and the wall time of one chain
 * (events around all repetitions).  This is what a chain of kernels of the projections' sizes costs on the
 * device when the kernels do nothing but read.  `sink`: 4 KiB of device memory the kernels may write.  The chain
 * runs untimed for 0.3 s first (steady clocks), synchronising the stream as it goes, so that every call takes at
 * least that long and blocks the host.  Errors: SPD_ERR_INVALID_ARG, SPD_ERR_CAPACITY (buffer too small / misaligned), SPD_ERR_HIP. */
int32_t spd_probe_read_chain(const void *buffer, size_t buffer_bytes, const size_t *h_stage_bytes, int32_t n_stages,
                             int32_t reps, void *sink, double *h_kernel_us, double *h_chain_us_per_rep, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SPD_H */
