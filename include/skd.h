/*
 * skd.h -- C ABI of the SkipDecode decode path for AMD MI355X (gfx950).
 *
 * SkipDecode (arXiv 2307.02628) is a token-level early-exit policy for
 * autoregressive decoders that keeps batching and KV caching intact:
 *   - all sequences of a batch compute the same number of layers n(t) at
 *     sequence position t (one exit point per batch column, Section 2.1);
 *   - n(t) never increases with t (Section 2.2), so a layer that runs at
 *     position t already holds the keys/values of every earlier position and
 *     nothing is ever recomputed;
 *   - n(t) decays linearly from n_max to n_min over the generated positions
 *     and the prompt uses all layers (Section 2.3, the token_idx equation);
 *   - the budget is spent on the TOP layers; lower layers are bypassed, i.e.
 *     the hidden state passes through unchanged and no key/value is stored
 *     (Section 2.4), optionally after `warmup` bottom layers.
 * The model is an OPT-style decoder (Section 3): learned positions,
 * pre-LayerNorm blocks with multi-head causal attention and a ReLU FFN, a
 * final LayerNorm and an LM head tied to the token embedding.
 *
 * Conventions
 *   t, i        0-based sequence position (column) of the token being processed
 *   P, N        prompt_size, sequence_length; T = N - P decode steps
 *   B           batch rows; every call works on one column of B tokens
 *   All functions return 0 (SKD_OK) or a positive count on success and a
 *   negative skd_err on failure; nothing aborts or throws across this boundary.
 *   Unless a parameter says "device", pointers are host memory owned by the
 *   caller and only read/written during the call.
 */
#ifndef SKD_H
#define SKD_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SKD_OK = 0,
  SKD_ERR_NULL = -1,     /* a required pointer is NULL */
  SKD_ERR_SHAPE = -2,    /* inconsistent configuration (see skd_create) */
  SKD_ERR_RANGE = -3,    /* position, layer, token id or size out of range */
  SKD_ERR_ORDER = -4,    /* call out of sequence (prefill missing, wrong t, ...) */
  SKD_ERR_SCHEDULE = -5, /* layer set not monotone / not ascending */
  SKD_ERR_NOMEM = -6,    /* host or device allocation failed, page pool exhausted */
  SKD_ERR_HIP = -7       /* a HIP runtime call failed (skd_last_hip_error) */
} skd_err;

enum { SKD_BF16 = 0, SKD_FP32 = 1, SKD_BF16_KV8 = 2 }; /* skd_config.dtype */
enum { SKD_HOST = 0, SKD_DEVICE = 1 }; /* skd_weights.location            */
enum { SKD_W_FP32 = 0, SKD_W_BF16 = 1 }; /* skd_weights.elem              */

typedef struct skd_state skd_state; /* opaque: device weights, KV pages, workspaces */

typedef struct {
  /* model shape */
  int32_t L;        /* num_decoder_layers                                   */
  int32_t d_model;  /* multiple of n_heads; bf16 path: head_dim 64 or 128, d_model <= 16384 */
  int32_t n_heads;
  int32_t ffn;      /* FFN width; bf16 path: d_model and ffn multiples of 32 */
  int32_t vocab;
  int32_t max_pos;  /* rows of the position table, >= sequence_length       */
  /* workload: the hyper-parameters of the Section 2.3 schedule */
  int32_t batch;            /* B >= 1                                        */
  int32_t prompt_size;      /* P >= 1, the padded prompt length             */
  int32_t sequence_length;  /* N > P                                        */
  int32_t n_min, n_max;     /* 1 <= n_min <= n_max <= L                     */
  int32_t warmup;           /* bottom layers always run, 0 <= warmup <= n_min;
                               they count inside n(t) (Section 2.4)         */
  /* implementation knobs */
  int32_t page_tokens;  /* tokens per KV page, multiple of 32; 0 = 64       */
  int32_t dtype;        /* SKD_BF16: bf16 weights/KV/activations, fp32 residual
                           stream and accumulation (the production path);
                           SKD_FP32: everything fp32, simple kernels (debug);
                           SKD_BF16_KV8: as SKD_BF16, with the cache in 8 bits
                           (SKD_KV_FP8 pages: half the bytes and half the pool;
                           shapes, calls and errors as with SKD_BF16)        */
  int32_t io_on_device; /* 0: token / logit buffers of prefill, decode_step and
                           logits_argmax are host memory and the calls
                           synchronise; 1: they are device memory and the calls
                           only enqueue work on the stream                    */
} skd_config;

/* Model parameters.  Matrices are [out_features][in_features] row-major.
 * `location` and `elem` apply to every tensor; the per-layer members are HOST
 * arrays of L pointers to tensors at `location`.  skd_create copies what it
 * needs (re-laid-out for the kernels); the caller may free everything after
 * it returns.  With dtype SKD_BF16, matrices and embedding tables are rounded
 * to bf16 (nearest even) if given as fp32; vectors (biases, LayerNorm gain and
 * bias) are kept in fp32 with the values given. */
typedef struct {
  int32_t location;    /* SKD_HOST or SKD_DEVICE */
  int32_t elem;        /* SKD_W_FP32 or SKD_W_BF16 (raw bf16 bit patterns)  */
  const void *tok_emb; /* [vocab][d]   */
  const void *pos_emb; /* [max_pos][d] */
  const void *lnf_g, *lnf_b; /* final LayerNorm [d] */
  const void *lm_head; /* [vocab][d] or NULL = tied to tok_emb */
  const void *const *ln1_g, *const *ln1_b;
  const void *const *wqkv, *const *bqkv; /* [3d][d], [3d]: rows q | k | v, head h = rows h*dh.. within each */
  const void *const *wo, *const *bo;     /* [d][d], [d] */
  const void *const *ln2_g, *const *ln2_b;
  const void *const *w1, *const *b1;     /* [ffn][d], [ffn] */
  const void *const *w2, *const *b2;     /* [d][ffn], [d]   */
} skd_weights;

/* n(t): number of layers computed at position t (Section 2.3, token_idx).
 * t < P gives L.  For P <= t <= N the linear interpolation between n_max (at
 * t = P) and n_min (at t = N) is rounded to the nearest integer, halves up,
 * in exact integer arithmetic.  Host only, no device needed.
 * Errors: SKD_ERR_SHAPE if L < 1, n_min < 1, n_min > n_max, n_max > L, P < 0
 * or N <= P;  SKD_ERR_RANGE if t < 0 or t > N. */
int skd_schedule(int32_t t, int32_t prompt_size, int32_t sequence_length, int32_t n_min, int32_t n_max, int32_t L);

/* Active layers at position t (Section 2.4), ascending, into layers_out[0..L):
 * all L layers on the prompt; afterwards the `warmup` bottom layers plus the
 * top n(t) - warmup layers.  Returns their number.  Uses only the schedule
 * fields and L of cfg.  Errors as skd_schedule, plus SKD_ERR_SHAPE if warmup
 * is outside [0, n_min]. */
int skd_active_layers(int32_t t, const skd_config *cfg, int32_t *layers_out);

/* Build a decoding state on the current HIP device: validates cfg, uploads and
 * re-lays-out the weights, reserves the KV page pool.  The pool holds exactly
 * the entries the static schedule will ever write (P*L + sum of n(t) per row,
 * rounded up to pages per layer), not N*L.  `hip_stream` is a hipStream_t (NULL =
 * the default stream) on which every later call of this state enqueues its
 * work.  Errors: SKD_ERR_NULL; SKD_ERR_SHAPE (d % heads, N <= P, P < 1,
 * max_pos < N, schedule fields, page_tokens % 32, bf16-path shape limits
 * above, unknown enum); SKD_ERR_NOMEM; SKD_ERR_HIP. */
int skd_create(const skd_config *cfg, const skd_weights *w, void *hip_stream, skd_state **out);

/* As skd_create, with the layer count of EVERY position supplied by the caller
 * instead of the linear decay: n_table[i], i = 0..N-1 (the paper leaves the
 * decay function open: power law, Section 2.3 / Section 5; decay that already
 * starts inside the prompt, Section 5).  The table must be non-increasing
 * (SKD_ERR_SCHEDULE otherwise: a layer that re-enters would miss keys, Section
 * 2.2), with 1 <= n_table[i] <= L (SKD_ERR_RANGE) and n_table[i] >= warmup
 * (SKD_ERR_SHAPE).  n_min / n_max of cfg must still be valid but are not used;
 * prefill processes prompt column i with n_table[i] layers.  The active set
 * keeps its shape: `warmup` bottom layers plus the top n - warmup. */
int skd_create_with_schedule(const skd_config *cfg, const skd_weights *w, void *hip_stream,
                             const int32_t *n_table, skd_state **out);

/* Active layers of this state at position t (0 <= t < N), ascending, into
 * layers_out[0..L); returns their number.  Equals skd_active_layers for states
 * made by skd_create. */
int skd_state_active_layers(const skd_state *st, int32_t t, int32_t *layers_out);

/* Process the prompt: columns 0..P-1, every one through all L layers
 * (Section 2.3: the prompt uses the full network), filling every layer's KV
 * cache.  tokens [B][P] int32 row-major.  attn_mask [B][P] uint8, 1 = real
 * token, NULL = all real; only LEFT padding is accepted (each row is zeros
 * followed by at least one 1), anything else is SKD_ERR_SHAPE.  Position ids
 * count real tokens; padded entries are never attended to.  Restarts the
 * generation if one was in progress.  With io_on_device = 1, `tokens` is a
 * device pointer laid out [P][B] (column-major) and attn_mask stays a host
 * pointer.  Errors: SKD_ERR_NULL, SKD_ERR_RANGE (host token outside
 * [0, vocab)), SKD_ERR_SHAPE, SKD_ERR_HIP.  Device-resident token ids are
 * not validated; the kernels clamp them into [0, vocab). */
int skd_prefill(skd_state *st, const int32_t *tokens, const uint8_t *attn_mask);

/* One decode step: process column t for all B rows with the layer set of
 * skd_active_layers(t).  Layers outside the set are not launched: the hidden
 * state passes through them and they store no key/value (Section 2.4).
 * tokens_in [B] is the column's input (the tokens generated for position t);
 * NULL = use the tokens the last skd_logits_argmax produced (greedy
 * free-running).  t must equal P + (decode steps done so far) and be < N:
 * the whole batch shares one position (Sections 2.1 and 5).
 * Errors: SKD_ERR_NULL, SKD_ERR_ORDER (no prefill, wrong t, NULL tokens_in
 * with no argmax since the last step), SKD_ERR_RANGE (t >= N, host token id),
 * SKD_ERR_HIP. */
int skd_decode_step(skd_state *st, int32_t t, const int32_t *tokens_in);

/* Several decode steps at once, for tokens that are known: columns t .. t + cols - 1
 * of all B rows, every one with the layer set of skd_active_layers, as `cols` calls of
 * skd_decode_step would process them (another order of the sums: the same values
 * within rounding).  Every weight is read once for up to 4096 rows x columns
 * instead of once per column.  The next turn of a conversation, drafted tokens to
 * be verified; skd_rewind takes columns back.  The heads see the last column.
 * tokens: [B][cols] host memory, or [cols][B] device memory with io_on_device = 1
 * (clamped into [0, vocab)).  The first call allocates its workspace.  Errors:
 * SKD_ERR_NULL, SKD_ERR_ORDER (no prefill, wrong t), SKD_ERR_RANGE (cols < 1,
 * t + cols > N, host token id), SKD_ERR_NOMEM, SKD_ERR_HIP. */
int skd_decode_chunk(skd_state *st, int32_t t, int32_t cols, const int32_t *tokens);

/* Final LayerNorm + LM head + greedy argmax on the hidden state of the last
 * processed column: every column emits a token for the whole batch, whatever
 * number of layers it ran (Section 2.1: one exit point per batch column; the
 * hidden state that leaves the last active layer goes straight to the head,
 * Section 2.4).  The paper leaves the head itself to the base model: the final
 * LayerNorm and the LM head always run and the head is tied to the token
 * embedding unless skd_weights.lm_head is given; the contract path is greedy
 * (beam 1), with the LOWEST index winning ties, and Section 3.2's sampling
 * setting is skd_logits_sample below.  tokens_out [B] (may be NULL) receives, per row, the
 * lowest index attaining the maximum logit; logits_out [B][vocab] fp32 (may be
 * NULL) receives the logits.  The tokens are also kept inside the state for
 * skd_decode_step(.., NULL).  Errors: SKD_ERR_NULL, SKD_ERR_ORDER (nothing
 * processed yet), SKD_ERR_HIP. */
int skd_logits_argmax(skd_state *st, int32_t *tokens_out, float *logits_out);

/* skd_logits_argmax for callers that cannot allocate device memory: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same kernels and the same results, but the LM head's per-workgroup
 * (max, argmax) partials live in a file-scope static device array of 2 MiB
 * (every GPU the library runs on holds its own copy until the process ends)
 * instead of buffers of the state, and the call itself calls no hipMalloc,
 * hipFree or other allocating routine.  Only for states with dtype SKD_BF16
 * or SKD_BF16_KV8 and io_on_device = 1 (SKD_ERR_SHAPE otherwise): tokens_out [B] and
 * logits_out [B][vocab] (either may be NULL) are device memory and the call
 * only enqueues work on the state's stream.  Limit:
 * ceil(vocab / (16 R)) * B_pad <= 262144 partials, R = LM-head tile rows per
 * workgroup (4 for vocabularies above 16320, 1 to 4 below; SKD_R_HEAD),
 * B_pad = batch padded to 16/32/48/64/96/128, i.e. vocabularies
 * up to 131072 at batch 128 and larger ones at smaller batches; beyond the
 * limit SKD_ERR_RANGE and nothing is launched.  All calls on one GPU, from whatever
 * state, share that GPU's array: calls that may overlap there (different
 * streams, different threads) race; calls on one stream are safe.  The array
 * keeps the previous call's contents; nothing in it needs clearing, since the
 * projection of a call writes every partial its final reduction reads.
 * Small heads of wide models (vocab <= 2048, d_model >= 1024) are split along
 * d_model: their partial sums live in a buffer of the state that skd_create has
 * reserved, they use no part of the static array, and calls of different states
 * do not race.
 * Errors otherwise as skd_logits_argmax. */
int skd_logits_argmax_noalloc(skd_state *st, int32_t *tokens_out, float *logits_out);

/* Sampling head (the paper's generation setting: temperature 0.3, top-p 0.7,
 * Section 3.2) in place of the greedy argmax: final LayerNorm + LM head, then
 * per row, with p_i = exp((z_i - max z) / temperature): the nucleus is the
 * smallest set of most likely tokens whose mass reaches top_p (tokens tied with
 * the last admitted one are admitted too), and the token is the first index of
 * the nucleus, in ascending index order, whose running mass exceeds
 * u[b] * mass(nucleus).  u [B] are uniform numbers in [0,1) supplied by the
 * caller (host memory, or device memory with io_on_device = 1): the library
 * draws no random numbers.  Deterministic for given (state, u).  tokens_out [B]
 * and logits_out [B][vocab] may be NULL; the tokens are kept for
 * skd_decode_step(.., NULL).  vocab <= 65536.  Errors: SKD_ERR_NULL,
 * SKD_ERR_ORDER, SKD_ERR_RANGE (temperature <= 0, top_p outside (0,1], host u
 * outside [0,1)), SKD_ERR_SHAPE, SKD_ERR_HIP. */
int skd_logits_sample(skd_state *st, const float *u, float temperature, float top_p, int32_t *tokens_out,
                      float *logits_out);

/* The parameters of a draw, one of each per row: arrays [rows], NULL = off for
 * every row (temperature: 1). */
typedef struct {
  const float *temperature; /* 0: the most likely token, the lowest index of several */
  const int32_t *top_k;     /* 0: off */
  const float *top_p;       /* 1: off */
  const float *min_p;       /* 0: off */
} skd_sampling;

/* skd_logits_sample with parameters per row, and top-k and min-p: final LayerNorm +
 * LM head, then the draw of skd_sample below (vocab <= 262144) from the state's
 * logits.  u [B], the arrays of params (may be NULL: all off) and the outputs are
 * host memory, or device memory with io_on_device = 1.  Errors: SKD_ERR_NULL,
 * SKD_ERR_ORDER, SKD_ERR_SHAPE (vocab), SKD_ERR_RANGE (host values: u outside
 * [0,1), temperature negative or not finite, top_k < 0, top_p outside (0,1],
 * min_p outside [0,1]), SKD_ERR_HIP. */
int skd_logits_sample_rows(skd_state *st, const float *u, const skd_sampling *params, int32_t *tokens_out,
                           float *logits_out);

/* Move the generation back to position t (P <= t <= current position): the
 * next skd_decode_step must be for column t; cache entries at columns >= t are
 * forgotten (they are overwritten when those columns are processed again).
 * The static schedule makes this exact: which layers hold which columns only
 * depends on t.  Used to regenerate from a point and to time a run after a
 * warm-up without repeating the prompt.  Errors: SKD_ERR_NULL, SKD_ERR_ORDER
 * (no prefill), SKD_ERR_RANGE. */
int skd_rewind(skd_state *st, int32_t t);

/* Number of columns layer `layer`'s KV cache holds (host bookkeeping).  For a
 * layer active at t this equals t before the step and t + 1 after it. */
int skd_kv_len(const skd_state *st, int32_t layer);

/* KV pages reserved for the whole state and pages that would be needed
 * without layer-sparse reservation (N tokens in every layer). */
int64_t skd_kv_pages_reserved(const skd_state *st);
int64_t skd_kv_pages_dense(const skd_state *st);

/* Wait until everything enqueued by this state has finished.  SKD_ERR_HIP with
 * skd_last_hip_error() = hipErrorLaunchTimeOut, here and from every other call
 * that computes or hands over results: a kernel of this state had to go on
 * without a workgroup that it had waited for over a second.  What the state
 * holds is then not to be used, and it stays so until skd_destroy. */
int skd_synchronize(skd_state *st);

/* Test / measurement hooks ------------------------------------------------ */

/* Copy the fp32 residual stream of the last processed column to host x_out [B][d]. */
int skd_debug_read_hidden(skd_state *st, float *x_out);

/* Declare columns 0..cols-1 processed (P <= cols < N), as if a prompt of that
 * length had run, and set layer caches from host arrays: for each layer l with
 * Kin[l] != NULL, Kin[l] and Vin[l] are [B][cols][d] fp32 and become that
 * layer's cache (rounded to the path's KV precision); layers with NULL entries
 * hold zeros.  Layers that leave the active window before column `cols` keep
 * only what they reserved.  start [B] (may be NULL = no padding) gives each
 * row's number of left-padding columns, 0 <= start[b] < cols; the entries of
 * Kin / Vin at those columns are ignored.  Used to set up
 * single decode steps at long contexts without running a long prompt.  Kin /
 * Vin are host arrays of L host pointers.  Errors: SKD_ERR_NULL,
 * SKD_ERR_RANGE, SKD_ERR_NOMEM, SKD_ERR_HIP. */
int skd_debug_kv_load(skd_state *st, int32_t cols, const float *const *Kin, const float *const *Vin,
                      const int32_t *start);

/* Read back row b of layer l's cache: k_out, v_out [len][d] fp32 with
 * len = skd_kv_len(l), indexed by column.  Left-padding columns of the row are
 * never attended to; what is returned for them is unspecified (the bf16 path
 * stores nothing for them and returns zeros). */
int skd_debug_kv_read(skd_state *st, int32_t layer, int32_t b, float *k_out, float *v_out);

/* Per-kernel timing.  skd_profile_enable(st, 1): every kernel launch of this
 * state is given its own pair of HIP events that receive the begin and end time
 * stamps of that kernel (what a kernel trace reports as its duration); mode 2
 * instead records one event before and one after the launches of each class
 * on the state's stream, which adds the cost of the two markers to every
 * measurement; 0 switches timing off.  Neither mode serialises anything, but
 * both cost host time per launch, so time whole runs with timing off.  A
 * column that would otherwise run as one launch (narrow bf16 models) runs as
 * separate kernels while timing is on: the same results, other times.
 * skd_profile_read waits for the stream and adds the elapsed milliseconds and
 * launch counts per kernel class into ms[SKD_PROF_CLASSES] and
 * launches[SKD_PROF_CLASSES] (either may be NULL), then clears the internal
 * accumulators.  Classes: see skd_prof_class.  Errors: SKD_ERR_NULL,
 * SKD_ERR_RANGE (mode), SKD_ERR_HIP. */
typedef enum {
  SKD_PROF_EMBED_LN = 0, /* embedding gather + first LayerNorm */
  SKD_PROF_GEMM_QKV = 1, /* q,k,v projection                   */
  SKD_PROF_ATTENTION = 2,/* decode attention over the paged KV (incl. split merge) */
  SKD_PROF_GEMM_OUT = 3, /* attention output projection        */
  SKD_PROF_REDUCE_LN = 4,/* split-K reduce + bias + residual + LayerNorm (with few rows
                            mostly inside GEMM_QKV and GEMM_FFN1) */
  SKD_PROF_GEMM_FFN1 = 5,
  SKD_PROF_GEMM_FFN2 = 6,
  SKD_PROF_LM_HEAD = 7,  /* LM head projection with per-workgroup argmax */
  SKD_PROF_ARGMAX = 8,   /* final argmax reduction, or the sampling head's passes */
  SKD_PROF_OTHER = 9,    /* fp32 debug path kernels            */
  SKD_PROF_CLASSES = 10
} skd_prof_class;
int skd_profile_enable(skd_state *st, int32_t on);
int skd_profile_read(skd_state *st, double *ms, int64_t *launches);

/* Operators outside of a state ------------------------------------------- */

/* A paged cache of keys and values in the caller's memory: a pool of pages, and
 * for every row (sequence) the pages that hold its positions, page_tokens of
 * them each, in a block table.  One layer's; layers have a pool or block tables
 * each.  Everything is device memory of the current device; the calls only
 * enqueue work on hip_stream (NULL: the default stream), allocate nothing, wait
 * for nothing and may be captured into a graph.  Calls that run at the same time
 * (two streams, two graphs) need workspaces of their own; rows of one pool may be
 * appended to and read at the same time if they share no page.
 *
 * SKD_KV_BF16 pages hold bf16 values.  In elements, per kv head h (of
 * page_tokens * 2 * head_dim) and block of 32 positions (of 64 * head_dim):
 *   keys   [half of the block][head_dim / 32][4][16 positions][8]
 *          position 16 half + p, element 32 i + 8 j + e at [half][i][j][p][e]
 *   values [head_dim / 16][4][16][2][4]
 *          position 16 x + 4 j + y, element 16 i + e at [i][j][e][x][y]
 * SKD_KV_FP8 pages hold 8 bits a value: e4m3 codes in bytes, per head and block
 *   keys   [half][head_dim / 64][4][16 positions][2][8]
 *          position 16 half + p, element 64 i + 32 w + 8 j + e at [half][i][j][p][w][e]
 *   values [head_dim / 32][4][16][2][2][4]
 *          position 16 x + 4 j + y, element 32 i + 16 w + e at [i][j][e][w][x][y]
 * and behind the codes of all heads [kv_heads][page_tokens / 32][k | v][32]
 * bytes: the values of a position are code * 2^(byte - 127), where the exponent is
 * the smallest from -127 on with which no magnitude exceeds 448 * 2^exponent, and
 * codes are rounded to nearest even (those of exponent 120 end at 240, so that
 * what is finite stays so).  A position and head whose values held an
 * infinity or NaN has byte 255, codes 0, and reads as NaN.
 * The bf16 pages of a state have the same layout.
 * SKD_KV_FP4 pages hold 4 bits a value (8.5 bits a position and element of keys and values together: 17 / 64 of
 * bf16, a little over half of SKD_KV_FP8): e2m1 codes (bits s e e m: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two in a
 * byte, and for every 32 neighbouring elements of a position one byte that stands for 2^(byte - 127).  The exponent is the smallest
 * from -124 on with which none of the 32 magnitudes exceeds 6 * 2^exponent; codes are rounded to nearest even (those
 * of exponent 126 end at 3, so that what is finite stays so).  32 elements among which was an infinity or NaN have byte
 * 255, codes 0, and read as NaN.  In bytes, per kv head (of page_tokens / 32 * 34 * head_dim) and block of 32 positions
 * (of 34 * head_dim), with G = head_dim / 32; position 16 x + 4 j + y or 16 half + p:
 *   keys   [half * G + c over 4][4][16 positions][half * G + c modulo 4][4]: element 32 c + 8 j + 2 i and the one
 *          behind it (in the upper 4 bits) at [..][j][p][..][i]
 *   values [G / 2][4][16][2][2][4]: elements 32 (2 i + w) + e and (upper 4 bits) + e + 16 at [i][j][e][w][x][y]
 *   bytes of the keys' exponents [16 positions][half][G], of the values' [4][G][2][4] at [j][i][x][y] */
enum { SKD_KV_BF16 = 0, SKD_KV_FP8 = 1, SKD_KV_FP4 = 4 }; /* skd_kv.elem */
typedef struct {
  int32_t elem;
  int32_t kv_heads, head_dim; /* head_dim 64 or 128 */
  int32_t page_tokens;        /* multiple of 32 */
  int32_t pages;              /* of the pool */
  int32_t rows, max_pages;    /* of the block table */
  void *pool;                 /* pages * skd_kv_page_bytes, 16-byte aligned */
  const int32_t *block_table; /* [rows][max_pages]: entries outside [0, pages) are no page: what would be filed there is
                                 dropped, and their positions are neither read nor attended to */
} skd_kv;

/* The tokens of a call: those of row r are tokens first[r] .. first[r + 1] - 1 of
 * the call's arrays and have the positions past[r], past[r] + 1, ... of the row.
 * Rows may have none.  max_new and max_past are upper bounds of the counts and of
 * past[], known to the host: tokens of a row beyond max_new, or beyond max_pages *
 * page_tokens of them, are left out, and max_past only decides how the work is shared
 * out.  Counts that do not fit into [0, tokens) are cut; a row whose past is negative,
 * or more than its pages hold, is left out.  max_pages * page_tokens is below 2^30.
 * Work is shared out as if every row had max_new tokens: one row of hundreds among
 * rows of one token each is better served by two calls, with block tables of the long
 * rows and of the others. */
typedef struct {
  int32_t tokens;             /* rows of the call's arrays */
  int32_t max_new, max_past;
  const int32_t *first;       /* [rows + 1] */
  const int32_t *past;        /* [rows] */
} skd_kv_chunk;

/* Bytes of a page; nothing but the shape is read.  Negative skd_err. */
int64_t skd_kv_page_bytes(const skd_kv *kv);

/* File the keys and values of new tokens: k, v [tokens][kv_heads * head_dim] bf16,
 * strides in elements from token to token (multiples of 8, pointers 16-byte
 * aligned).  What the pages hold at other positions stays.  Errors:
 * SKD_ERR_NULL; SKD_ERR_SHAPE (unknown elem, head_dim, page_tokens, counts below
 * 1, strides, alignment); SKD_ERR_RANGE (negative counts; 2^30 positions of a row,
 * or 2^31 blocks of 32 positions, max_new of every row and kv head, or more; memory
 * that is not the current device's); SKD_ERR_HIP. */
int skd_kv_append(const skd_kv *kv, const skd_kv_chunk *chunk, const void *k, int64_t k_stride, const void *v,
                  int64_t v_stride, void *hip_stream);

/* Read back the keys and values at the tokens' positions (past = 0 and as many
 * tokens as it holds: a whole row) into k_out, v_out [tokens][kv_heads * head_dim],
 * fp32 (SKD_W_FP32: exact) or bf16 (SKD_W_BF16).  Tokens whose positions have no
 * page keep what was there.  Errors as skd_kv_append. */
int skd_kv_read(const skd_kv *kv, const skd_kv_chunk *chunk, int32_t elem, void *k_out, int64_t k_stride, void *v_out,
                int64_t v_stride, void *hip_stream);

/* Attention of new tokens over the cache: query head h of a token at position p of
 * its row attends, with softmax(scale * q . k), to positions 0 .. p of kv head
 * h / (heads / kv_heads).  q, out [tokens][heads * head_dim] bf16, heads a multiple of
 * kv_heads.  k and v (both or neither): the new tokens' keys and values, filed by
 * this call as by skd_kv_append before they are attended to (as they are held, so
 * in 8 bits as rounded); NULL: the cache holds them already.  A query that sees
 * no position, or only such with a score of -infinity, gets zeros.  Positions behind
 * a row's last one may hold anything.  Sums and softmax are in fp32, weights (relative
 * to the largest score met so far, up to 2^8) are rounded to bf16 for the matrix
 * instructions: by 2^-8 of a weight, and times an 8-bit exponent to no less than
 * 2^-133.  The sum of weights times values has to fit fp32: it does for values up to
 * 2^119 over the number of positions, larger ones may give infinity.
 * workspace: skd_kv_attend_workspace bytes for this kv, chunk and heads (16-byte
 * aligned; NULL where that is 0), nothing in it is kept from call to call.  The same
 * call gives the same bits.  Errors as skd_kv_append, and SKD_ERR_SHAPE (heads),
 * SKD_ERR_RANGE (scale not above 0, or above 2.3e38; heads * head_dim of 2^31 or more;
 * 2^32 threads or more, of which 16, 32 or 128 queries of a row and kv head take 256
 * or 512), SKD_ERR_NOMEM (workspace_bytes). */
int skd_kv_attend(const skd_kv *kv, const skd_kv_chunk *chunk, int32_t heads, float scale, const void *q, int64_t q_stride,
                  const void *k, int64_t k_stride, const void *v, int64_t v_stride, void *out, int64_t out_stride,
                  void *workspace, int64_t workspace_bytes, void *hip_stream);
int64_t skd_kv_attend_workspace(const skd_kv *kv, const skd_kv_chunk *chunk, int32_t heads);

/* What becomes of the scores of an attention, and which positions a token sees. */
typedef struct {
  float cap;            /* scores s = scale * q . k become cap * tanh(s / cap), cap from 2^-20 to 1024; 0: they stay */
  const float *slopes;  /* [heads]: slopes[h] * |p - j| is then taken from the score of position j at position p; NULL: nothing */
  int32_t window;       /* a token at position p sees none before p - window + 1; 0: no such bound */
  const int32_t *begin; /* [tokens]: nor any before begin[token] (its document's first position); NULL: from 0 on */
  const int32_t *end;   /* [tokens]: it sees positions up to end[token] - 1, which may lie behind its own (a prefix that sees
                           itself in both directions); NULL: up to its own */
} skd_kv_scores;

/* skd_kv_attend with changed scores and masks (`scores`, device arrays in it; slopes that are finite in fp32, also times the
 * distances and over scale, or over cap where there is one).  Positions seen are cut to those
 * that the row has once the call's tokens are filed, so tokens of one call see each other in both directions where `end`
 * says so; a token that sees none gets zeros.  What positions that a token does not see hold, also infinities and NaN,
 * does not reach it.  A cap's function is off by up to 2^-11.4 of a weight (cap 1024; in proportion to it), a distance above
 * 2^24 by 2^-24 of itself.  Work, memory, workspace (skd_kv_attend_scores_workspace bytes for these arguments) and
 * errors as skd_kv_attend, and SKD_ERR_NULL (scores), SKD_ERR_RANGE (cap, also where 3 * scale / cap is no finite
 * number; window < 0; memory that is not the current device's), SKD_ERR_SHAPE (arrays that are not aligned to their elements). */
int skd_kv_attend_scores(const skd_kv *kv, const skd_kv_chunk *chunk, int32_t heads, float scale, const skd_kv_scores *scores,
                         const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                         void *out, int64_t out_stride, void *workspace, int64_t workspace_bytes, void *hip_stream);
int64_t skd_kv_attend_scores_workspace(const skd_kv *kv, const skd_kv_chunk *chunk, int32_t heads, const skd_kv_scores *scores);

/* The next block table of a batch: rows forked, put into another order, ended, cut and grown.  A page is free if
 * no entry of a table names it; nothing else is kept.  Row r of table_out [rows][max_pages] goes on from row
 * source[r] of kv->block_table (outside [0, rows): from none; NULL: every row from itself), which holds len[r] positions, with
 * more[r] tokens to come (negative: 0; together cut to max_pages * page_tokens).  It has the pages of positions 0 ..
 * len[r] + more[r] - 1, entries behind are -1, and so are entries before len[r] that were no page.  Entries that tokens
 * to come go to are its own: one that has no page gets a free one, and so does one whose page other entries of table_out
 * name too, unless tokens to come go to all of them and it is the first.  Where such a page holds positions below len[r],
 * the pair (page, new page) is listed in copies [rows][2]: skd_kv_copy_pages, before anything is filed, on the pool of
 * every cache that goes by this table.  Pages are dealt out from the lowest free one on, by row and position, copies are listed
 * by row; (-1, -1) follows behind the last.  counts [3]: pages that table_out names; pages that were missing; copies.  If pages
 * were missing nothing is dealt out: rows have the pages of positions below len[r] only, and no copies are listed.
 * No pool is read or written (kv->pool may be NULL).  table_out may be kv->block_table if source is NULL.  All of it is
 * device memory, stream and workspace (skd_kv_assign_workspace bytes) as for the calls above.  Errors: SKD_ERR_NULL;
 * SKD_ERR_SHAPE (kv as for the calls above; arrays that are not aligned to their elements, workspace to 16 bytes);
 * SKD_ERR_RANGE (rows * max_pages from 2^31 on; 2^24 rows, or rows and 1024s of pages, or more; table_out that overlaps the table
 * otherwise; memory that is not the current device's); SKD_ERR_NOMEM (workspace_bytes); SKD_ERR_HIP. */
int skd_kv_assign(const skd_kv *kv, const int32_t *source, const int32_t *len, const int32_t *more, int32_t *table_out,
                  int32_t *copies, int32_t *counts, void *workspace, int64_t workspace_bytes, void *hip_stream);
int64_t skd_kv_assign_workspace(const skd_kv *kv);

/* Moves the pages that a block table names to the lowest places of the pool: with n of them, the k-th one at or
 * behind place n goes to the k-th free place before it.  table_out [rows][max_pages] is the table with the new places (-1 for
 * what is no page) and may be kv->block_table; copies [pages / 2][2] lists the moves in ascending order, then (-1, -1);
 * counts [3]: n, 0, moves.  Pools are moved by skd_kv_copy_pages; memory, workspace and errors as skd_kv_assign. */
int skd_kv_compact(const skd_kv *kv, int32_t *table_out, int32_t *copies, int32_t *counts, void *workspace, int64_t workspace_bytes,
                   void *hip_stream);
int64_t skd_kv_compact_workspace(const skd_kv *kv);

/* Copies whole pages of the pool: page copies[i][0] to page copies[i][1] for i below `most` and, if number is not NULL, below
 * *number (device memory).  A pair with an entry outside [0, pages), or twice the same, is passed over.  No page may be
 * written and named in another pair too.  Nothing but elem, the shape, pages and pool is read of kv.  Errors: SKD_ERR_NULL,
 * SKD_ERR_SHAPE, SKD_ERR_RANGE (most < 0; memory that is not the current device's), SKD_ERR_HIP. */
int skd_kv_copy_pages(const skd_kv *kv, const int32_t *copies, int32_t most, const int32_t *number, void *hip_stream);

/* One token per row of fp32 logits [rows][vocab] (stride: elements from row to
 * row).  With m_i = exp((z_i - max z) / temperature): kept are the tokens with
 * m_i >= min_p that are among the top_k largest logits (those equal to the k-th
 * too), and of these the smallest set of most likely ones whose mass reaches top_p
 * of theirs (those equal to the last too).  The token is the first index, in
 * ascending order, whose running mass over that set exceeds u[row] * its mass.
 * Masses are formed in 64 bits and summed in units of 2^-45 of the largest (a
 * token below half a unit has none and is never drawn), so the same call gives
 * the same tokens.  A NaN is taken for -infinity; where the
 * largest logit is infinite, or temperature is not above 0, the token is the
 * lowest index that has it (0 in a row without a finite logit).  Device values
 * outside their ranges: top_k < 0, top_p >= 1 or NaN, min_p <= 0 or NaN are off,
 * top_p <= 0 keeps the most likely token and those equal to it, min_p >= 1 likewise,
 * u is cut to [0,1).  vocab <= 262144.  All memory is the current device's, with
 * stream and workspace (skd_sample_workspace bytes; NULL where that is 0) as for
 * the calls above.  Errors: SKD_ERR_NULL; SKD_ERR_SHAPE (vocab, stride, pointers not
 * aligned to their elements); SKD_ERR_RANGE (rows < 0 or from 2^22 on, 2^20 of
 * the largest vocab, memory that is not the current device's); SKD_ERR_NOMEM (workspace_bytes); SKD_ERR_HIP. */
int skd_sample(const float *logits, int64_t stride, int32_t rows, int32_t vocab, const skd_sampling *params, const float *u,
               int32_t *tokens_out, void *workspace, int64_t workspace_bytes, void *hip_stream);
int64_t skd_sample_workspace(int32_t rows, int32_t vocab);

void skd_destroy(skd_state *st);
const char *skd_strerror(int err);
/* hipError_t (as int) of the most recent failing HIP call on this thread, 0 if none. */
int skd_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SKD_H */
