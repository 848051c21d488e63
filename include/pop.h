/*
 * pop.h -- C ABI of the POP (Partition-guided Online Pruning) pruned-FFN library for MI355X (gfx950).
 *
 * One layer = one SwiGLU FFN  y = W_down (silu(W_gate x) * (W_up x))  with hidden size d and
 * intermediate size m.  "Channel" always means one of the m intermediate channels: row j of W_gate and
 * W_up, column j of W_down (Sec. 3.1: an output channel of the first projections is one dimension of the
 * intermediate representation, shared by the consecutive linear maps).
 *
 * Importance (Sec. 3.1 Eq. 1-2, Sec. 3.4 Eq. 3), read on the down projection and its input activations:
 *     I_j = || W_down[:, j] ||_2 * sqrt( sum over tokens t of H[t][j]^2 ),   H = silu(X W_gate^T) * (X W_up^T).
 * The same formula is used at prefill (all prompt tokens) and at a decode step (one token).
 *
 * Conventions for every entry point
 *   - returns a status code (POP_OK == 0, negative on error); never throws, never exits.
 *   - pointers marked "dev" are device (HBM) pointers, "host" are host pointers.  The caller owns every
 *     buffer it passes; the library never frees or keeps them beyond the call, except that
 *     pop_layer_create reads the three weight matrices once and keeps its own repacked copy
 *     (device memory cost: one extra copy of the weights plus scratch: about a hundred rows of m floats, up to 4096 rows
 *     of d floats, and a row of m floats per 16 (float32) or 64 (bf16) tokens of max_tokens).
 *   - argument errors are found on the host before anything is launched.  Device work is enqueued on
 *     the given HIP stream (a hipStream_t passed as void*, NULL = the null stream) and is NOT
 *     synchronised: the caller synchronises the stream before reading outputs.
 *   - a layer handle may be used from one stream at a time.  Calls on one handle that overlap in time race.
 *   - index lists are int32, ascending by channel; regions are one byte per channel.
 *   - dtype of x, weights: the layer's wdtype (float32, or bf16 stored as 16-bit patterns).
 *     bf16 layers need d % 8 == 0, float32 layers d % 4 == 0 (128-bit loads), else POP_EUNSUPPORTED.
 *   - device pointers to activations (x, x_t), weights and outputs y must be 16-byte aligned (the kernels use
 *     128-bit accesses); a misaligned one is rejected with POP_EINVAL.
 *   - inputs must be finite; with non-finite inputs results are deterministic but unspecified.
 */
#ifndef POP_H
#define POP_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pop_layer pop_layer_t; /* opaque, owned by the library */

typedef enum { POP_F32 = 0, POP_BF16 = 1 } pop_dtype_t;

enum {
    POP_OK = 0,
    POP_EINVAL = -1,       /* NULL pointer, negative size, bad enum */
    POP_ESHAPE = -2,       /* sizes inconsistent with the layer or with each other */
    POP_ENOMEM = -3,       /* device allocation failed */
    POP_EHIP = -4,         /* a HIP call failed; text via pop_last_hip_error() */
    POP_ESTATE = -5,       /* call order violated (e.g. decode before prefill) */
    POP_EUNSUPPORTED = -6, /* valid request this build does not implement */
    POP_EDEVICE = -7       /* a kernel gave up a bounded wait; results of that step are invalid */
};

enum { POP_REGION_RETAINED = 0, POP_REGION_CANDIDATE = 1, POP_REGION_PRUNED = 2 };

#define POP_MAX_BATCH 8 /* largest B of pop_decode_mask / largest token chunk processed per pass */

int pop_version(void);
const char *pop_strerror(int status);      /* static storage */
const char *pop_last_hip_error(void);      /* text of the last failing HIP call on this thread */

/* Host only.  Region sizes from fractions (Sec. 3.3: thresholds at quantile levels r-delta and r+delta,
 * realised as exact rank counts):  n_ret = floor(f_ret*m + 1/2),  n_ret + n_cand = floor((f_ret+f_cand)*m + 1/2),
 * n_prn = m - n_ret - n_cand.  With the paper's (r, delta): f_ret = 1-r-delta, f_cand = 2*delta. */
int pop_region_counts(int m, double f_ret, double f_cand, int *n_ret, int *n_cand, int *n_prn);

/* Host only.  Number of candidates to select per token so that the active channel count is
 * floor((1-r)*m + 1/2) (Sec. 3.3 "Decoding Stage"), clamped to [0, n_cand]. */
int pop_k_for_ratio(int m, double r, int n_ret, int n_cand, int *k);

/* Host only.  Region sizes and per-token k of the decode strategies compared in the paper's ablation (Sec. 5,
 * trade-off table), all with floor((1-r)*m + 1/2) active channels per token:
 *   POP_STRATEGY_POP          the method: candidate band of gamma*m channels centred on the sparsity quantile
 *                             (f_ret = 1-r-gamma/2, f_cand = gamma; counts and k as in the two functions above);
 *   POP_STRATEGY_STATIC_MASK  Variant (1): the prefill mask is reused at every step (n_cand = 0, all active
 *                             channels retained): no re-scoring, no selection, no overhead;
 *   POP_STRATEGY_RESCORE_ALL  Variant (2): every channel is a candidate at every step (n_ret = 0, n_cand = m).
 * The counts go to pop_prefill_partition / pop_decode_mask unchanged.  gamma is ignored by the two variants.
 * Errors: a band that leaves [0, 1] or an unknown strategy -> POP_EINVAL. */
enum { POP_STRATEGY_POP = 0, POP_STRATEGY_STATIC_MASK = 1, POP_STRATEGY_RESCORE_ALL = 2 };
int pop_strategy_counts(int strategy, int m, double r, double gamma, int *n_ret, int *n_cand, int *k);
/* Value for n_ret, n_cand (both), k0 and - as a NULL pointer - k in the calls below: "what the layer's strategy says"
 * (pop_layer_set_strategy). */
enum { POP_FROM_STRATEGY = -1 };

/* Create a layer.  w_gate, w_up: dev [m][d]; w_down: dev [d][m]; all of dtype wdtype, read once, on `stream`,
 * and repacked channel-major (one contiguous gate+up row pair and one contiguous down column per channel).
 * Also computes the data-free weight factor n_j = ||W_down[:,j]||_2 of Eq. 3.
 * max_tokens: largest T of pop_prefill_partition; max_batch: largest B (1..POP_MAX_BATCH).
 * The stream is synchronised before returning (the caller may free the source weights afterwards). */
int pop_layer_create(pop_layer_t **out, int d, int m, pop_dtype_t wdtype,
                     const void *w_gate, const void *w_up, const void *w_down,
                     int max_tokens, int max_batch, void *stream);
int pop_layer_destroy(pop_layer_t *layer);

/* Prefill (Sec. 3.3 "Prefilling Stage"): H for all m channels and all T prompt tokens (x: dev [T][d]),
 * I_j over the T tokens, then the three regions by rank in the order (score descending, channel ascending):
 * the best n_ret channels are retained, the next n_cand are candidates, the rest are pruned.
 * Outputs (dev, any may be NULL): scores [m] float32; region [m] (POP_REGION_*); ret_idx [n_ret];
 * cand_idx [n_cand].  The partition is also kept inside the layer for the decode calls.
 * T == 0 is allowed (x may then be NULL): with no tokens every importance is zero and the regions follow the
 * channel order (an expert of a mixture that no prompt token was routed to).
 * Errors: T < 0 or T > max_tokens, n_ret/n_cand < 0 or n_ret + n_cand > m -> POP_ESHAPE. */
int pop_prefill_partition(pop_layer_t *layer, const void *x, int T, int n_ret, int n_cand,
                          float *scores, unsigned char *region, int *ret_idx, int *cand_idx, void *stream);

/* Prefilling stage with its output (Sec. 3.3 "Prefilling Stage", Sec. 3.4: the prompt's forward pass runs under the
 * pruning structure the prompt itself determines).  Everything pop_prefill_partition does, with the same outputs
 * and errors, and then the pruned FFN of the T prompt tokens, y: dev [T][d] of dtype ydtype, under the prefill mask:
 * the retained channels plus the best k0 candidates by prefill score (same order as above), i.e. the n_ret + k0
 * channels of highest prefill importance.  mask: dev [m], 1 = active (may be NULL).
 * On bf16 layers with T >= 32 the hidden activations of the contraction are kept (rounded to bf16), the active
 * columns are gathered, and the down projection runs as one matrix-core GEMM.  Shorter prompts (bf16 layers with
 * d % 64 == 0: T < 32, float32 layers: T <= 64) keep them in float32 and need no second pass over the gate and up rows.
 * Otherwise, and under the input-side reading, the call is pop_prefill_partition followed by pop_pruned_ffn(mask).
 * Scratch of the T >= 32 path (H: 2 x T x m x 2 bytes, m rounded up to 64; partial outputs: n x T x d x 4 bytes where
 * the contraction is split n = 2 .. 8 ways to fill the chip) is allocated at the first call and when T grows, which
 * synchronises the device; it stays with the layer.
 * Errors: as pop_prefill_partition; k0 < 0 or k0 > n_cand -> POP_ESHAPE; y == NULL or bad ydtype -> POP_EINVAL. */
int pop_prefill_forward(pop_layer_t *layer, const void *x, int T, int n_ret, int n_cand, int k0,
                        void *y, pop_dtype_t ydtype, float *scores, unsigned char *region, int *ret_idx,
                        int *cand_idx, unsigned char *mask, void *stream);

/* Decode step, mask part (Sec. 3.3 "Decoding Stage", Sec. 3.4 two-step decoding).  x_t: dev [B][d].
 * Pass 1 evaluates h_j = silu(g_j) * u_j for every retained and candidate channel, for each of the B
 * sequences; candidates are re-scored, I_j(t) = n_j * |h_j|, and for sequence b the best k[b] (host array [B],
 * 0 <= k[b] <= n_cand) are selected with the same tie rule as above.
 * Outputs (dev, any may be NULL): cand_scores [B][n_cand] float32 in cand_idx order; mask [B][m], 1 = active
 * (retained or selected); active_idx [B][n_ret + n_cand], row b holds the retained channels ascending followed
 * by the selected ones ascending, n_active[b] = n_ret + k[b] entries valid; n_active [B].
 * h and the masks stay cached in the layer for pop_pruned_ffn(mask = NULL).
 * Errors: no partition yet -> POP_ESTATE; B < 1 or B > max_batch, k[b] out of range -> POP_ESHAPE. */
int pop_decode_mask(pop_layer_t *layer, const void *x_t, int B, const int *k,
                    float *cand_scores, unsigned char *mask, int *active_idx, int *n_active, void *stream);

/* Pruned FFN output (Sec. 3.3: only retained and selected channels form the step's computation;
 * Sec. 3.4 final computation).  y: dev [T][d] of dtype ydtype.
 *   mask == NULL: finish the decode step started by the immediately preceding pop_decode_mask on this layer
 *       (T must equal its B; x is not read again):  y_b = sum over active j of h_bj * W_down[:, j].
 *   mask != NULL: stand-alone pruned FFN of x (dev [T][d]) under the given masks, dev [mask_rows][m],
 *       mask_rows == 1 (shared by all tokens) or == T (one per token); any T >= 1.  Does not need a
 *       partition.  An all-ones mask gives the dense FFN.  bf16 layers with T >= 32 run this on the matrix
 *       cores: gate/up over the channels active in any row, H rounded to bf16, then one GEMM over those channels
 *       (scratch is allocated at the first such call and when T grows, which synchronises the device); smaller
 *       T and float32 layers keep H in float32 (a few tokens on a layer of few channels, and bf16 layers with d % 64 != 0:
 *       the decode kernels, up to eight tokens at a time; otherwise bf16 layers all tokens in one pass over the weights,
 *       float32 layers 64 at a time).
 * Errors: mask == NULL without a preceding decode step -> POP_ESTATE; T mismatch, bad mask_rows -> POP_ESHAPE. */
int pop_pruned_ffn(pop_layer_t *layer, const void *x, int T, const unsigned char *mask, int mask_rows,
                   void *y, pop_dtype_t ydtype, void *stream);

/* Whole decode step in one call (Sec. 3.3 "Decoding Stage", Sec. 3.4: pass 1 over retained and candidate
 * channels, candidate re-scoring, per-token selection, then the output over retained and selected channels):
 * the same results, bit for bit, as pop_decode_mask followed by pop_pruned_ffn(mask = NULL), with y: dev [B][d] of
 * dtype ydtype and the other outputs as in pop_decode_mask (each may be NULL).
 * It issues those two calls' launches, except that the selection results the caller takes are copied by the last of
 * them, where pop_decode_mask needs a launch for that.  A B == 1 step on a shape the fused single-sequence kernel
 * takes is two launches: that kernel, whose workgroups hand each other the candidates' h and the selection inside the launch,
 * and a small kernel that sums their partial outputs.  Neither keeps host-side state per launch, so captured
 * launches can be replayed.  The waits inside the fused launch, and inside the first launch of a B > 1 step (its
 * selecting workgroups wait for the candidates' scores), are bounded (pop_layer_set_wait_limit): if one gives
 * up, the step's results are invalid, pop_layer_sync_status reports POP_EDEVICE, every kernel still exits and the
 * next step is unaffected.
 * Errors: as pop_decode_mask; y == NULL or bad ydtype -> POP_EINVAL. */
int pop_decode_step(pop_layer_t *layer, const void *x_t, int B, const int *k, void *y, pop_dtype_t ydtype,
                    float *cand_scores, unsigned char *mask, int *active_idx, int *n_active, void *stream);

/* ---- pieces of the path exposed on their own (selection parity is defined on caller-supplied scores) ---- */

/* Three regions from given scores (dev [m] float32), as in pop_prefill_partition.  Needs no layer. */
int pop_partition_from_scores(const float *scores, int m, int n_ret, int n_cand,
                              unsigned char *region, int *ret_idx, int *cand_idx, void *stream);

/* The same, and in the same launch the n_top best channels of that order, 0 <= n_top <= m: the mask a prompt's own
 * forward pass runs under (Sec. 3.4; pop_prefill_forward uses n_top = n_ret + k0: the retained channels plus the best
 * k0 candidates by prefill score are the n_ret + k0 best channels overall).  Outputs (dev): top_mask [m] (1 = among
 * the n_top best; may be NULL), top_list [n_top] ascending channel numbers (required).
 * Errors: as pop_partition_from_scores; top_list == NULL -> POP_EINVAL; n_top out of range -> POP_ESHAPE. */
int pop_partition_top_from_scores(const float *scores, int m, int n_ret, int n_cand, int n_top,
                                  unsigned char *region, int *ret_idx, int *cand_idx,
                                  unsigned char *top_mask, int *top_list, void *stream);

/* Step selection from given candidate scores (Sec. 3.3 "Decoding Stage": of the candidate region the k channels of
 * highest step score stay active next to the retained region; equal scores by lower channel number):
 * cand_scores dev [n_cand] in cand_idx order, cand_idx dev [n_cand] ascending, region dev [m], 0 <= k <= n_cand.
 * Outputs (dev, may be NULL): mask [m] (retained + selected), sel_idx [k] ascending.
 * Errors: NULL inputs -> POP_EINVAL; sizes out of range -> POP_ESHAPE. */
int pop_topk_from_scores(const float *cand_scores, const int *cand_idx, int n_cand, int k,
                         const unsigned char *region, int m, unsigned char *mask, int *sel_idx, void *stream);

/* Column-wise importance reduction alone (Eq. 3): h dev [T][m] (float32 or bf16), nrm dev [m] float32,
 * scores[j] = nrm[j] * sqrt(sum_t h[t][j]^2).  Long prompts of few channels are summed in chunks, whose partial sums
 * (at most 32 x m doubles) live in scratch that this call allocates and frees on `stream` (hipMallocAsync).
 * Errors: NULL pointers, bad dtype -> POP_EINVAL; T < 1 or m < 1 -> POP_ESHAPE; no memory -> POP_ENOMEM. */
int pop_importance_reduce(const void *h, pop_dtype_t hdtype, int T, int m, const float *nrm,
                          float *scores, void *stream);

/* Allocates, now, the scratch that pop_prefill_forward and pop_pruned_ffn(mask) need for prompts of up to T tokens
 * (they otherwise allocate it at their first call and when T grows, which synchronises the device), so that those
 * calls only enqueue work afterwards.  New buffers are cleared on `stream`.  Sec. 3.4 (the prompt's forward pass).
 * Errors: T < 1 or T > max_tokens -> POP_ESHAPE; allocation failure -> POP_ENOMEM. */
int pop_layer_reserve_prompt(pop_layer_t *layer, int T, void *stream);

/* pop_importance_reduce for callers that cannot allocate (code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc): the same kernels, arguments, results (bit for bit) and errors, but the per-chunk partial
 * sums live in a static device array of 8 MiB that every GPU the library runs on holds until the process ends; the
 * call allocates and frees nothing.  Limit: m <= 32768 channels, else POP_EUNSUPPORTED (use pop_importance_reduce).
 * All calls on one GPU share that array: calls that overlap in time on one GPU (different streams) race; calls on one
 * stream are ordered and safe.  A failing HIP call gives POP_EHIP (no text is recorded for pop_last_hip_error). */
int pop_importance_reduce_static(const void *h, pop_dtype_t hdtype, int T, int m, const float *nrm,
                                 float *scores, void *stream);

/* Read-only views of layer state, for tests and callers that build on the partition.
 * Copies are enqueued on `stream`; outputs dev, any may be NULL: nrm [m] float32 (n_j of Eq. 3),
 * h [B][m] float32 of the last decode step (0 for pruned channels is NOT guaranteed: only retained and
 * candidate entries are defined). */
int pop_layer_get_norms(pop_layer_t *layer, float *nrm, void *stream);
/* Synchronises `stream`, then reports whether any decode step on this layer since the last report (or the last
 * prefill) hit the bound of an in-kernel wait: POP_OK, or POP_EDEVICE (the results of such a step are invalid; repeat
 * it).  The record is cleared by the report.  Every kernel exits either way; this call is how a caller finds out. */
int pop_layer_sync_status(pop_layer_t *layer, void *stream);
int pop_layer_get_hidden(pop_layer_t *layer, float *h, int B, void *stream);
/* Host only.  Makes one of the ablation's decode strategies (Sec. 5, trade-off table; see pop_strategy_counts) the
 * layer's mode at sparsity r (and band gamma for POP_STRATEGY_POP): pop_prefill_partition and pop_prefill_forward
 * called with n_ret = n_cand = POP_FROM_STRATEGY (and k0 = POP_FROM_STRATEGY) then take the strategy's region sizes
 * (and its k), and pop_decode_mask / pop_decode_step called with k == NULL select the strategy's k for every
 * sequence.  Explicit counts keep working next to it.  Does not touch an existing partition.
 * Errors: as pop_strategy_counts; without a strategy the sentinels give POP_ESTATE (prefill) / POP_EINVAL (k). */
int pop_layer_set_strategy(pop_layer_t *layer, int strategy, double r, double gamma);
/* Host only.  How many times a bounded in-kernel wait of a decode step looks for what it waits for before it gives
 * up (default 65536: a fraction of a second).  Two kernels wait: the fused single-sequence step (Sec. 3.4: its
 * workgroups hand each other the candidates' h and the selection) and the batched step's first launch, whose
 * selecting workgroups wait for the candidates' scores.  A wait that gives up flags the step (pop_layer_sync_status:
 * POP_EDEVICE) and leaves its results invalid; every kernel still exits, and the next step is unaffected.  0 makes
 * every wait give up at once unless the data is already there: a testing knob.
 * Errors: NULL layer or looks < 0 -> POP_EINVAL. */
int pop_layer_set_wait_limit(pop_layer_t *layer, int looks);
/* Host only.  Which reading of Sec. 3.1 defines channel importance on this layer (the paper's equations admit two):
 *   POP_IMPORTANCE_OUTPUT_SIDE (default)  the down projection and the intermediate activations, as at the top of
 *       this file; the decode step scores candidates from h (Sec. 3.4's two-step decoding).
 *   POP_IMPORTANCE_INPUT_SIDE             Eq. 1-2 literally on the first projections and the FFN input:
 *       I_j = || [W_gate[j,:], W_up[j,:]] * s ||_2,  s_k = sqrt(sum over tokens of x[t][k]^2)  (a channel is removed
 *       from both matrices, so its weights are both rows); at a decode step s_k = |x_k|, per sequence.  Prefill
 *       then needs no contraction (one pass over the gate and up rows).  A single-sequence decode step runs in the
 *       fused kernel, which forms a candidate's score from the same two rows it reads for h; a step with B > 1
 *       selects first and runs the forward pass over retained and selected channels only, as separate launches: h
 *       of an unselected candidate is then not computed, so pop_layer_get_hidden is defined on active channels
 *       only under this reading.  With the shared batch mask s_k runs over the step's B rows.
 * Changing the reading discards the layer's partition (prefill again).  Errors: unknown value -> POP_EINVAL. */
enum { POP_IMPORTANCE_OUTPUT_SIDE = 0, POP_IMPORTANCE_INPUT_SIDE = 1 };
int pop_layer_set_importance(pop_layer_t *layer, int reading);
/* Host only.  How a decode step with B > 1 scores its candidates.  off (default): every sequence by its own
 * activation, I_j = n_j |h_bj|, its own top-k and mask.  on: the activation norm of Eq. 3 runs over the step's B
 * sequences ("tokens and samples", Sec. 3.1), I_j = n_j sqrt(sum_b h_bj^2), and one selection serves the whole
 * batch: all k[b] must be equal (else POP_ESHAPE), every row of cand_scores, mask and active_idx comes out the
 * same.  B == 1 is unaffected.  Invalidates a cached decode step. */
int pop_layer_set_shared_batch_mask(pop_layer_t *layer, int on);
/* Host only.  Which implementation the last successful decode step on this layer used: 0 = none yet,
 * 1 = the fused single-sequence kernel, 2 = the batch-general kernels.  If workgroups != NULL it
 * receives the fused kernel's grid size for the current partition (0 when the fused kernel does not apply). */
int pop_layer_step_kind(pop_layer_t *layer, int *workgroups);

/* ---- measurement aids: bare reads of device memory (they compute nothing of the method) ----
 * The decode step (Sec. 3.3 "Decoding Stage", Sec. 3.4) is bound by the bytes it must stream; these two calls request
 * such bytes and nothing else, so that timing them (events on `stream`) gives the time the memory system itself needs:
 * the yardstick next to the published peak bandwidth.  They load as a decode step of a layer that size does.  sink: dev, one unsigned int the kernels may OR a bit into.
 *   pop_probe_read       contiguous read of `bytes` (rounded down to 16) of buf (dev, 16-byte aligned).
 *   pop_probe_step_read  the weight rows one decode step of the layer's current partition reads: gate and up rows of
 *                        all retained and candidate channels, down rows of the retained channels and of the first k
 *                        candidates (standing in for the selected ones).
 * workgroups: grid size (512 threads each).  Errors: NULL / misaligned pointers -> POP_EINVAL; no partition ->
 * POP_ESTATE; sizes out of range -> POP_ESHAPE. */
int pop_probe_read(const void *buf, size_t bytes, int workgroups, unsigned int *sink, void *stream);
int pop_probe_step_read(pop_layer_t *layer, int k, int workgroups, unsigned int *sink, void *stream);

/* ---- around the FFN: what a decoder needs that serves several beams of a prompt ----
 *
 * The beams of one prompt are the natural batch of the decode calls above: they share the partition that the prompt
 * determined.  The calls below give them a cache of keys and values, attention over it, beam search's selection and the
 * reordering of the cached states after it.  None of them needs a layer or keeps state: the caller owns all buffers.
 *
 * The cache (one decoder layer's keys and values) is held in 4 bits: e2m1 codes (0 .5 1 1.5 2 3 4 6 and a sign) and one
 * scale byte for 32 channels, value = code * 2^(byte - 127) (the OCP microscaling format MXFP4), 17/16 byte for the key and
 * the value of a channel together.  It is [n_pages][n_kv_heads][page_tokens / 16] tiles of 16 (D + D/16) bytes, D = head_dim:
 *     K codes [16 tokens][D/2], V codes [4 groups of 4 tokens][16][4 tokens][D/32] (the 16 are D/16 channels each),
 *     K scales [16 tokens][D/32], V scales [4 groups][D/32][4 tokens];  the lower channel of a byte is its low nibble.
 * A token's *slot* is page * page_tokens + its place in the page.  A row of `block_table` (dev [n_seq][table_stride]) names
 * the pages of a sequence in order; entries outside [0, n_pages) are no page.  All layers of a model can share the tables.
 * head_dim is 64, 128 or 256, page_tokens 16, 32, 64, 128 or 256, n_kv_heads at most 65535, else POP_EUNSUPPORTED; n_pages * page_tokens
 * stays below 2^31 and table_stride * page_tokens does not pass 2^30, else POP_EUNSUPPORTED.  cache, q, k, v, y, logits, workspaces: 16-byte aligned.
 *
 * Free pages stand in a ring: `ring` (dev [n_pages]) and `pool` (dev, two ints): the place of the first free page, and how many
 * are free.  Pages are taken at the front and given back at the end, so a call's inputs stay as they are and its outputs
 * (pool_out, and the new lengths and tables) are buffers of their own: a caller keeps two of each and takes turns.
 * Status words (dev, one int, read it when you next synchronise): 0, or a sum of */
enum {
    POP_PLAN_PAGES = 1,   /* more pages needed than are free */
    POP_PLAN_TOKENS = 2,  /* more new tokens than max_tokens */
    POP_PLAN_INVALID = 4  /* a negative length, a table row that is too short, a pool that is none */
};
/* With a status other than 0 the call changed nothing: its outputs say that every sequence is as it was. */

#define POP_MAX_BEAMS 16 /* rows of one request in pop_beam_select and pop_cache_reorder */

/* Host only.  Bytes of one layer's cache.  Errors: sizes < 1 -> POP_ESHAPE; NULL -> POP_EINVAL. */
int pop_cache_bytes(int n_kv_heads, int head_dim, int page_tokens, int n_pages, size_t *bytes);

/* Pages and slots of a step from request lengths, in one launch.  cached_len, new_len: dev [n_seq], tokens that each sequence
 * has in the cache and tokens that this step adds.  Every sequence keeps its pages and gets as many of the ring's as
 * its new tokens call for, in sequence order.  Outputs (dev): block_table's entries for the new blocks; context_len [n_seq] =
 * cached + new; q_start [n_seq + 1], the exclusive sums of new_len; and for the new tokens, sequence by sequence,
 * slots [max_tokens] and positions [max_tokens] (may be NULL), -1 behind the last; pool_out; status.
 * Errors: NULL pointers, outputs that are their inputs -> POP_EINVAL; negative sizes -> POP_ESHAPE. */
int pop_cache_plan(const int *cached_len, const int *new_len, int n_seq, int page_tokens, int *block_table,
                   int table_stride, const int *ring, int n_pages, const int *pool, int *pool_out, int max_tokens,
                   int *context_len, int *q_start, int *slots, int *positions, int *status, void *stream);

/* Stores tokens.  k, v: dev, one row of [n_kv_heads][head_dim] for each of n_tokens, k_stride and v_stride elements apart (so
 * both may be parts of one projection's rows; multiples of 8 for bf16, of 4 for float32).  Tokens whose slot is negative or
 * beyond the cache are left out.  A block's scale is 2^(e - 2), e the exponent of its largest magnitude, and twice that from a
 * significand of 1.75 on; values go to the nearest code, halves to the even one, magnitudes above 6 to 6.  An infinity is stored
 * as the largest float32, a NaN as zero: nothing that the format holds is infinite or no number.
 * Errors: NULL or misaligned pointers, bad dtype -> POP_EINVAL; sizes, strides -> POP_ESHAPE; n_tokens * n_kv_heads * head_dim of 2^34 or
 * more -> POP_EUNSUPPORTED. */
int pop_cache_write(void *cache, int n_kv_heads, int head_dim, int page_tokens, int n_pages, const void *k,
                    const void *v, pop_dtype_t dtype, long long k_stride, long long v_stride, const int *slots,
                    int n_tokens, void *stream);

/* The values stored at n_tokens slots, k and v: dev [n_tokens][n_kv_heads][head_dim] (exact in bf16 as in float32); zeros
 * where a slot is negative or beyond the cache.  Errors: as pop_cache_write. */
int pop_cache_read(const void *cache, int n_kv_heads, int head_dim, int page_tokens, int n_pages, const int *slots,
                   int n_tokens, void *k, void *v, pop_dtype_t dtype, void *stream);

/* y = softmax(scale * q k^T) v.  q: dev [n_tokens][n_heads][head_dim] of dtype; the new tokens of sequence s are rows q_start[s] ..
 * q_start[s + 1] - 1 and the last of them is at position context_len[s] - 1; all of them
 * have been written.  A token sees the positions up to its own, with window > 0 only the last `window` of them; query head h reads kv
 * head h / (n_heads / n_kv_heads).  A token that sees nothing (pages that are none, a context shorter than the new tokens)
 * gives zeros.  Scores (scale * q k) stay within +-2.3e38, and the values that a token sees add up to less than 1e26 a channel; beyond that
 * sums overflow.  y: dev [n_tokens][n_heads][head_dim] of ydtype; rows of no sequence are not written.  A sequence whose rows leave
 * [0, n_tokens) is left out and its rows are undefined.
 * max_new, max_context: the longest that the caller expects; longer ones are right too, but may be slow.  float32 q is
 * taken in full (three bf16 terms).  The softmax weights are rounded to bf16 where q and y are both bf16, else taken in full too; their
 * sum is of the unrounded ones, in float32.
 * workspace: dev, of pop_cache_attention_workspace bytes for the same sizes, or for larger n_tokens, n_seq, max_new or max_context; any
 * content, for this call alone.
 * Errors: NULL or misaligned pointers, bad dtype, a scale that is not finite -> POP_EINVAL; sizes, n_heads no multiple of
 * n_kv_heads, a workspace that is too small -> POP_ESHAPE; n_seq * n_kv_heads > 65535, n_tokens * n_heads >= 2^30, or more rounds than
 * 32 bits count, (n_tokens * n_heads / n_kv_heads / 16 + n_seq) * n_kv_heads * (table_stride * page_tokens / 128 + 1) >= 2^31 (of the
 * table's width, whatever the contexts are) -> POP_EUNSUPPORTED. */
int pop_cache_attention(const void *q, pop_dtype_t dtype, int n_tokens, const void *cache, int n_kv_heads,
                        int head_dim, int page_tokens, int n_pages, const int *block_table, int table_stride,
                        const int *q_start, const int *context_len, int n_seq, int n_heads, int max_new,
                        int max_context, float scale, int window, void *y, pop_dtype_t ydtype, void *workspace,
                        size_t workspace_bytes, void *stream);
/* Host only. */
int pop_cache_attention_workspace(int n_tokens, int n_seq, int n_heads, int n_kv_heads, int head_dim, int max_new,
                                  int max_context, size_t *bytes);
/* Host only.  Which implementation a call of these sizes runs: 0 = none (nothing to do), 1 = units of 16 columns (new tokens x query heads
 * of a kv head), 2 = blocks of 128.  If parts != NULL it receives the parts that a block's tokens may be split into (0 for 0 and 1).
 * Errors: as pop_cache_attention. */
int pop_cache_attention_kind(pop_dtype_t dtype, pop_dtype_t ydtype, int n_tokens, int n_seq, int n_heads, int n_kv_heads,
                             int head_dim, int max_new, int max_context, int window, int *parts);

/* The same with first tokens that stay visible: with window > 0 a token at position p sees token t <= p if p - t < window or t < sinks.  Without a
 * window, or with sinks = 0, it is pop_cache_attention.  Pages that no token sees may be none (given back to the pool).
 * workspace, the rounding of the softmax weights: as for pop_cache_attention.  Errors: as pop_cache_attention; sinks < 0 -> POP_ESHAPE. */
int pop_cache_attention_sinks(const void *q, pop_dtype_t dtype, int n_tokens, const void *cache, int n_kv_heads,
                              int head_dim, int page_tokens, int n_pages, const int *block_table, int table_stride,
                              const int *q_start, const int *context_len, int n_seq, int n_heads, int max_new,
                              int max_context, float scale, int window, int sinks, void *y, pop_dtype_t ydtype,
                              void *workspace, size_t workspace_bytes, void *stream);
/* Host only.  As pop_cache_attention_kind, which knows of no first tokens (they add to what a window sees). */
int pop_cache_attention_sinks_kind(pop_dtype_t dtype, pop_dtype_t ydtype, int n_tokens, int n_seq, int n_heads, int n_kv_heads,
                                   int head_dim, int max_new, int max_context, int window, int sinks, int *parts);

/* pop_cache_attention (without a window) for sequences that share a prefix: n_seq rows in groups of `group` sequences (beams of a prompt, or questions
 * about one document), whose first prefix_len[g] tokens (dev [n_seq / group]) are the same in all rows of group g.  The caller sees to that: up to
 * the shorter of prefix_len and its context, each row's table names pages that hold the same keys and values there, the same pages or copies, as
 * pop_cache_reorder leaves them.  Tokens of the prefix are read from any of the rows that have new tokens, once for all of them; rows may be
 * shorter than the prefix, and new tokens may stand in it.  prefix_len that is negative or 0 shares nothing.
 * Where that does not pay (pop_cache_attention_shared_kind; prefixes of less than 1024 tokens) each row reads its own pages.
 * Rows, types, the rounding of the softmax weights, limits and errors otherwise as pop_cache_attention (of the rounds: < 2^30); group < 1 or n_seq no multiple of it -> POP_ESHAPE.
 * workspace: dev, of pop_cache_attention_shared_workspace bytes for the same sizes, or for larger n_tokens, n_seq, max_new or max_context; any content,
 * for this call alone. */
int pop_cache_attention_shared(const void *q, pop_dtype_t dtype, int n_tokens, const void *cache, int n_kv_heads,
                               int head_dim, int page_tokens, int n_pages, const int *block_table, int table_stride,
                               const int *q_start, const int *context_len, int n_seq, int group, const int *prefix_len,
                               int n_heads, int max_new, int max_context, float scale, void *y, pop_dtype_t ydtype,
                               void *workspace, size_t workspace_bytes, void *stream);
/* Host only. */
int pop_cache_attention_shared_workspace(int n_tokens, int n_seq, int group, int n_heads, int n_kv_heads, int head_dim,
                                         int max_new, int max_context, size_t *bytes);
/* Host only.  Bytes of that which a call of just these types and sizes uses, from the workspace's beginning on. */
int pop_cache_attention_shared_used(pop_dtype_t dtype, pop_dtype_t ydtype, int n_tokens, int n_seq, int group, int n_heads, int n_kv_heads,
                                    int head_dim, int max_new, int max_context, size_t *bytes);
/* Host only.  Which implementation a call of these sizes runs: 0 = none (nothing to do), 1 = that of pop_cache_attention, each row for itself (chunks that
 * are bound by their products, and calls too small to gain by sharing were all of max_context shared), 2 = prefixes by blocks of 16 or 32 columns (new
 * tokens x query heads of a kv head, of up to 64 rows of a group), 3 = by blocks of 128.  Errors: as pop_cache_attention_shared. */
int pop_cache_attention_shared_kind(pop_dtype_t dtype, pop_dtype_t ydtype, int n_tokens, int n_seq, int group, int n_heads, int n_kv_heads,
                                    int head_dim, int max_new, int max_context);

/* Beam search's selection.  logits: dev [n_requests * n_beams][vocab] (float32 or bf16), scores: dev [n_requests * n_beams]
 * float32, the beams' sums of log-probabilities (-inf: not alive), done: dev, a byte for each beam (may be NULL).
 * A beam proposes scores + logit - logsumexp(logits) for every token; one that is done proposes pad_token at its own score
 * and nothing else.  Per request the k best: scores, tokens and the beams they come from (dev [n_requests][k]), best first, equal
 * scores by lower beam, then lower token.  (Tokens of one beam are first ranked by their logits, equal ones by lower token.)
 * What is proposed at -inf fills up a list that is short.  n_beams <= POP_MAX_BEAMS, k <= 64 and <= n_beams * vocab.
 * NaN logits count as -inf; with +inf ones results are unspecified.
 * workspace: dev, of pop_beam_workspace bytes for the same sizes, any content.
 * Errors: NULL or misaligned pointers, bad dtype -> POP_EINVAL; sizes, pad_token outside the vocabulary, a workspace that is
 * too small -> POP_ESHAPE; beyond the limits above, vocab > 2^24, 2^24 rows or more -> POP_EUNSUPPORTED. */
int pop_beam_select(const void *logits, pop_dtype_t dtype, const float *scores, const unsigned char *done,
                    int n_requests, int n_beams, int vocab, int k, int pad_token, float *out_scores, int *out_tokens,
                    int *out_parents, void *workspace, size_t workspace_bytes, void *stream);
/* Host only. */
int pop_beam_workspace(int n_requests, int n_beams, int vocab, int k, size_t *bytes);

/* The cached states after a selection: n_seq rows in groups of n_beams, and row c of a group becomes what row parents[c]
 * (0 .. n_beams - 1, within the group; anything else ends the row) of it was.  Rows share the full pages they have in common.
 * A last page that is partly filled goes on with the parent's first child; each further child gets a page of the ring and
 * copies = {the parent's page, its own} (dev [n_seq][2], {-1, -1} for none), for pop_cache_copy_pages on every layer.  Pages
 * that no row of the group holds any more go to the end of the ring, by group, block and row.  n_beams = 1 and parents of -1
 * release sequences.  Rows of a group may share pages only at the same block, and groups none, as these calls leave them.
 * Outputs (dev): new_table [n_seq][table_stride] (-1 behind a row's last page), new_len [n_seq], copies, pool_out, status, and
 * the ring's free places.  workspace: dev, of pop_cache_reorder_workspace bytes, any content.
 * Errors: NULL pointers, outputs that are their inputs -> POP_EINVAL; sizes, n_seq no multiple of n_beams, a workspace
 * that is too small -> POP_ESHAPE; n_beams > POP_MAX_BEAMS, 2^24 groups or more -> POP_EUNSUPPORTED. */
int pop_cache_reorder(const int *block_table, const int *len, const int *parents, int n_seq, int n_beams,
                      int page_tokens, int table_stride, int *new_table, int *new_len, int *copies, int *ring,
                      int n_pages, const int *pool, int *pool_out, void *workspace, size_t workspace_bytes, int *status,
                      void *stream);
/* Host only. */
int pop_cache_reorder_workspace(int n_seq, int n_beams, int table_stride, size_t *bytes);

/* Page copies {from, to} of one layer's cache: copies dev [n_copies][2]; pairs with a number that is no page do nothing.  No page
 * may be copied to twice, or from and to.  Errors: NULL or misaligned pointers -> POP_EINVAL; sizes -> POP_ESHAPE; 2^24 copies or
 * more -> POP_EUNSUPPORTED. */
int pop_cache_copy_pages(void *cache, int n_kv_heads, int head_dim, int page_tokens, int n_pages, const int *copies,
                         int n_copies, void *stream);

/* ---- between a layer's blocks ----
 *
 * Residual sums with the norms around a block, and rotary positions, on rows of any length and alignment (of their elements).  Calls are faster where all
 * widths (d, head_dim) and strides are multiples of 8 elements and all addresses of 16 bytes.  Strides are in elements, from row to row. */

/* The residual stream after a block, and the next block's input, in one pass:
 *     u' = u r(u) (w_post + weight_offset)  if post_norm, else u;       r(v) = 1 / sqrt(sum of squares of v / d + eps)
 *     x' = x_scale x + u_scale gate u';
 *     z  = x' r(x') (w_pre + weight_offset).
 * x: dev, n_tokens rows of d of xdtype.  u: dev, rows of dtype, NULL for none (x' = x_scale x; no gate, no post_norm then).  gate: dev, gate_rows
 * = 1 (for all tokens) or n_tokens rows of d of dtype, NULL (and 0) for none.  w_post, w_pre: dev [d] of dtype, NULL for a factor of 1 (without
 * the offset).  Outputs (dev): x_out of xdtype, z of dtype; either may be NULL.  z is formed from x' before that is rounded to xdtype.
 * An output may be x or u itself where type and stride are the same; otherwise outputs lie apart from inputs and from each other.
 * Sums of squares are float32.
 * Errors: NULL x, no output, outputs that are inputs in another way, misaligned pointers, bad dtype, eps not above 0, numbers that are not
 * finite -> POP_EINVAL; sizes, strides below d, other gate_rows -> POP_ESHAPE; d > 65536, 2^22 tokens or more -> POP_EUNSUPPORTED. */
int pop_block_norm(const void *x, pop_dtype_t xdtype, long long x_stride, const void *u, pop_dtype_t dtype, long long u_stride, const void *gate,
                   int gate_rows, long long gate_stride, int n_tokens, int d, const void *w_post, const void *w_pre, int post_norm,
                   float weight_offset, float eps, float x_scale, float u_scale, void *x_out, long long x_out_stride, void *z,
                   long long z_stride, void *stream);

/* Which channels of a head are turned together: i and i + rotary_dim / 2, or 2 i and 2 i + 1. */
enum { POP_ROTARY_HALVES = 0, POP_ROTARY_PAIRS = 1 };
/* How the frequencies base^(-2 i / rotary_dim) are scaled for contexts longer than the trained one, by a factor >= 1:
 *   POP_ROTARY_PLAIN   not at all (factor is not looked at);
 *   POP_ROTARY_LINEAR  divided by the factor;
 *   POP_ROTARY_BASE    base times factor^(R / (R - 2)), R = rotary_dim >= 4: the slowest are divided by the factor, the fastest stay;
 *   POP_ROTARY_BANDS   by the rotations r that a frequency makes over `context` tokens: divided up to `low` of them, as they are from `high` on, and
 *                      in between (1 - s) f / factor + s f with s = (r - low) / (high - low);
 *   POP_ROTARY_RAMP    the same with s falling linearly over i, from the floor of the place where a frequency makes `high` rotations to
 *                      the ceiling of that of `low` (both within 0 .. R - 1); sines and cosines times 1 + ln(factor) / 10. */
enum { POP_ROTARY_PLAIN = 0, POP_ROTARY_LINEAR = 1, POP_ROTARY_BASE = 2, POP_ROTARY_BANDS = 3, POP_ROTARY_RAMP = 4 };
/* Host only.  turns: host [rotary_dim / 2], the frequencies in revolutions a token (f / 2 pi), 64 bits; amplitude (may be NULL): the factor of sines and
 * cosines, 1 but for POP_ROTARY_RAMP.  context, low and high are looked at by the last two only.
 * Errors: NULL turns, an unknown scaling, base not above 1, factor below 1, context or low not above 0, high not above low, numbers that are not
 * finite -> POP_EINVAL; rotary_dim odd, below 2 (4) or above 1024 -> POP_ESHAPE. */
int pop_rotary_frequencies(int rotary_dim, double base, int scaling, double factor, double context, double low, double high, double *turns,
                           float *amplitude);
/* Turns the heads of tokens by their positions: of channels a and b that go together, at an angle t = 2 pi position turns[i],
 *     a' = amplitude (a cos t - b sin t),  b' = amplitude (a sin t + b cos t).
 * The first rotary_dim channels of each head are turned, the others copied.  q, k: dev, rows of [n_heads][head_dim] and [n_kv_heads][head_dim] of
 * dtype, q_stride and k_stride elements apart (so both may be parts of one projection's rows); k may be NULL (with k_out).
 * positions: dev [n_tokens]; rows whose position is negative are left as they were.  turns: dev [rotary_dim / 2], 64 bits.  q_out, k_out:
 * dev, may be q and k themselves (with the same strides), otherwise apart from them.
 * Angles are products in 64 bits, sines and cosines float32.
 * Errors: NULL or misaligned pointers, bad dtype or layout, an amplitude that is not finite, outputs that are inputs with another stride
 * -> POP_EINVAL; sizes, rotary_dim odd or above head_dim, strides below a row -> POP_ESHAPE; rotary_dim > 1024, (n_heads + n_kv_heads) * head_dim
 * >= 2^26, 2^22 tokens or more -> POP_EUNSUPPORTED. */
int pop_rotary(const void *q, const void *k, pop_dtype_t dtype, int n_tokens, int n_heads, int n_kv_heads, int head_dim, int rotary_dim, int layout,
               long long q_stride, long long k_stride, const int *positions, const double *turns, float amplitude, void *q_out, void *k_out,
               long long q_out_stride, long long k_out_stride, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* POP_H */
