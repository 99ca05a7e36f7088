/*
 * dlm.h - C ABI of the MI355X (gfx950) hot path of DepCap block-wise diffusion-LM decoding.
 *
 * The three calls of the method, in the paper's problem statement (Sec. 3, "Two decisions in
 * block-wise inference"):
 *   dlm_step         one denoising step: the masked-diffusion transformer predicts a distribution
 *                    for every position of the active span against a cached prefix, and the
 *                    per-position statistics of Sec. 4.2 / 4.3 are reduced over the vocabulary
 *   block_boundary   DepGA-Block: how far the next block extends (Sec. 4.2, Eq. 3-4)
 *   select_parallel  CAP-Decoding: which masked positions of the block are decoded now
 *                    (Sec. 4.3, Eq. 5-6, Alg. 1), and the token write of Eq. 2
 *
 * Conventions for every function:
 *   - returns DLM_OK (0) or a negative DLM_E* code; never throws, never aborts, never synchronises
 *     the stream; when an error is returned no device memory has been written and no kernel
 *     launched.  dlm_last_error() gives a thread-local message for the last failure.
 *   - "DEVICE" pointers are HIP device memory of the current device; "host" pointers are ordinary
 *     host memory that is read completely before the call returns.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  All work is enqueued
 *     on it; outputs are valid once the caller has synchronised it.
 *   - the caller owns every buffer it passes; the library owns what *_create allocated.
 *   - dtype: DLM_F32 = IEEE binary32, DLM_BF16 = bfloat16; accumulation is always fp32.  DLM_BF16 is what the caller's
 *     weights, embeddings and logits are stored as.  Inside a pass the matrix cores are fed IEEE half: the layer weights are
 *     converted once, by dlm_model_create (exactly, except that a weight below 2^-14 in magnitude keeps an absolute error of
 *     at most 2^-25), and the activations the GEMMs and the attention read are rounded to half (11 significant bits, values
 *     beyond +-65504 saturate) instead of bfloat16 (8 bits); the residual stream is fp32.
 */
#ifndef DLM_H
#define DLM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { DLM_OK = 0, DLM_EINVAL = -1, DLM_ESHAPE = -2, DLM_ECAPACITY = -3, DLM_ENOMEM = -4, DLM_EHIP = -5 };
enum { DLM_F32 = 0, DLM_BF16 = 1 };

const char* dlm_last_error(void);

/* ---- model ------------------------------------------------------------------------------- */

/* Pre-norm transformer without causal mask: RMSNorm, rotary embedding on half-split pairs
 * (i, i + head_dim/2), grouped-query attention (query head h reads kv head h / (n_q/n_kv)),
 * SwiGLU feed-forward, untied LM head, no biases.  Requirements: head_dim in {32, 64, 128};
 * n_q_heads % n_kv_heads == 0; for DLM_BF16 every matrix dimension is a multiple of 32. */
typedef struct {
  int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, vocab, mask_id, dtype;
  float rms_eps, rope_theta;
} dlm_config;

/* DEVICE pointers to row-major [out, in] matrices of the model dtype.  The per-layer members are
 * host arrays of n_layers DEVICE pointers.  wqkv rows: Q heads, then K heads, then V heads.
 * w_gate_up rows: the d_ffn gate rows, then the d_ffn up rows. */
typedef struct {
  const void* embed;              /* [vocab, d_model] */
  const void* const* wqkv;        /* [(n_q + 2 n_kv) * head_dim, d_model] */
  const void* const* wo;          /* [d_model, n_q * head_dim] */
  const void* const* w_gate_up;   /* [2 * d_ffn, d_model] */
  const void* const* w_down;      /* [d_model, d_ffn] */
  const void* const* norm1;       /* [d_model] */
  const void* const* norm2;       /* [d_model] */
  const void* final_norm;         /* [d_model] */
  const void* lm_head;            /* [vocab, d_model] */
} dlm_weights;

typedef struct dlm_model dlm_model;
typedef struct dlm_state dlm_state;

/* Copies the weights into library-owned device memory (bf16 matrices are re-tiled for the matrix
 * cores, in IEEE half, on `stream`).  The caller may release its own tensors once `stream` has been synchronised.
 * bf16 layer matrices are kept twice where the kernel that serves passes of up to 16 to 64 rows has a
 * layout of its own for them (what all workgroups read at the same step adjacent in memory): the
 * model then takes up to twice its layer weights (30 GB for an 8B model).  A copy that does not fit
 * is left out; the environment variable DLM_W_STEPS=0, read by this call, leaves them all out
 * (results are bit-identical either way: the same products are added in the same order).  A bf16 model
 * whose matrices take up to 320 MiB has them read through the memory-side cache, which keeps them from pass to
 * pass, a larger one past it; DLM_W_CACHED=1 or =0, read by this call, says which (bit-identical as well).
 * Errors: DLM_EINVAL (null pointer, bad dtype), DLM_ESHAPE (unsupported dimensions), DLM_ENOMEM. */
int dlm_model_create(const dlm_config* cfg, const dlm_weights* w, void* stream, dlm_model** out);
void dlm_model_destroy(dlm_model* m);

/* Decode state for up to max_seqs independent sequences ("slots"): the prefix KV cache
 * [layer][slot][max_seq_len][n_kv*head_dim] (K after the rotary embedding), the retained
 * look-ahead logits p^prev of Sec. 4.2 (two buffers of max_lookahead rows per slot) and the
 * workspaces of one pass of up to max_rows packed rows.  All slots start empty (kv_len 0).
 * Errors: DLM_EINVAL, DLM_ECAPACITY (a size is not positive, max_seqs > 32), DLM_ENOMEM. */
int dlm_state_create(const dlm_model* m, int max_seqs, int max_seq_len, int max_rows, int max_lookahead,
                     dlm_state** out);
void dlm_state_destroy(dlm_state* s);
/* Forget a slot's cache and retained logits (host bookkeeping only). */
int dlm_state_reset(dlm_state* s, int slot);
/* Cached prefix length of a slot, or a negative error code. */
int dlm_state_kv_len(const dlm_state* s, int slot);

/* ---- dlm_step ------------------------------------------------------------------------------ */

/* One packed pass over n_seqs sequences; sequence b owns rows [row_offsets[b], row_offsets[b+1])
 * of every per-row array, which are the absolute positions span_start[b], span_start[b]+1, ...
 * Each row attends (bidirectionally) to the slot's cached prefix [0, kv_len) and to all rows of
 * its own span; span_start[b] must equal the slot's kv_len.  After the pass the first
 * commit_len[b] rows join the cache (Sec. 5.2: prefix KV cached per decoded block).
 * suffix_len[b] > 0 (dual cache, Sec. 5.2, Q2): the rows also attend to the suffix_len[b] positions right
 * after the span, with the keys and values an earlier pass over those positions left in the cache
 * (every pass writes the K and V of all its rows at their positions; only the committed ones count
 * as prefix).  They are not recomputed.
 *
 * Statistics (Sec. 4.2, 4.3; natural log; the mask token's probability is forced to 0 first;
 * argmax ties go to the lowest token id) are written for every row:
 *   max_logit, lse = log sum exp, conf = max_v p(v), argmax, entropy = H(p),
 *   kl = KL(p^curr || p^prev) (Eq. 3) on the kl_count[b] rows starting at relative row
 *   kl_first[b], where p^prev is the retained distribution of the same absolute position; 0 on
 *   all other rows.
 * The logits of the save_count[b] rows starting at relative row save_first[b] are retained as the
 * slot's new p^prev (replacing the old one after this pass has read it).
 * `tokens` is device memory the host cannot inspect: an id outside [0, vocab) is read as the nearest
 * valid id (clamped), never as an address outside the embedding table.
 *
 * Errors (nothing is launched): DLM_EINVAL (null pointer, n_seqs < 1, offsets not increasing, slot
 * out of range or repeated, span_start != kv_len, commit/kl/save ranges outside the span, a kl row
 * with no retained p^prev, a suffix beyond the positions an earlier pass has covered),
 * DLM_ECAPACITY (rows > max_rows, span beyond max_seq_len, save_count > max_lookahead, n_seqs >
 * max_seqs).  DLM_EHIP: the runtime refused a launch; the state's host bookkeeping is unchanged but
 * what the kernels that did run wrote (uncommitted cache rows, activations) is unspecified. */
typedef struct {
  int32_t n_seqs;
  const int32_t* slot;         /* host [n_seqs] state slot of each sequence (NULL: 0, 1, ...)      */
  const int32_t* row_offsets;  /* host [n_seqs+1]                                                  */
  const int32_t* span_start;   /* host [n_seqs]                                                    */
  const int32_t* commit_len;   /* host [n_seqs]                                                    */
  const int32_t* kl_first;     /* host [n_seqs] (NULL with kl_count: no KL rows)                   */
  const int32_t* kl_count;     /* host [n_seqs]                                                    */
  const int32_t* save_first;   /* host [n_seqs] (NULL with save_count: nothing retained)           */
  const int32_t* save_count;   /* host [n_seqs]                                                    */
  const int32_t* tok_start;    /* host [n_seqs] index into `tokens` of the span's first row        */
  const int32_t* suffix_len;   /* host [n_seqs] (NULL: 0) cached positions after the span to attend */
  const int32_t* tokens;       /* DEVICE token ids (mask_id on undecoded slots)                    */
  void* logits;                /* DEVICE out [rows, vocab], model dtype                            */
  float* max_logit;            /* DEVICE out [rows]                                                */
  float* lse;                  /* DEVICE out [rows]                                                */
  float* entropy;              /* DEVICE out [rows]                                                */
  float* kl;                   /* DEVICE out [rows]                                                */
  float* conf;                 /* DEVICE out [rows]                                                */
  int32_t* argmax;             /* DEVICE out [rows]                                                */
} dlm_step_desc;

int dlm_step(dlm_state* s, const dlm_step_desc* d, void* stream);

/* ---- block_boundary ------------------------------------------------------------------------ */

/* DepGA-Block (Sec. 4.2).  For sequence b the candidate window is the W_b = win_len[b] positions
 * after the frontier, stored at I[win_start[b] ...], H[win_start[b] ...] (the caller sizes it:
 * W = min(L_max, L_remain), 1 <= W_b <= 256); I = last-block influence (Eq. 3), H = entropy of
 * those positions (the kl and entropy outputs of dlm_step can be passed as they are).
 * Both signals are smoothed (centred moving average of radius smooth_radius, truncated at the
 * window edges) and normalised inside the window (norm_mode 0: by the window mean, 1: by the
 * window max, 2: min-max, 3: not at all), S_k = I~_k - lambda H~_k (Eq. 4), and
 *   rule 0: the block ends immediately before the first k with S_k < 0,
 *   rule 1: before the first k whose prefix sum S_0 + ... + S_k < 0 (the cumulative form, Sec. 4.4),
 * whole window if there is none; L is clipped to [l_min, W_b] (the window wins).  cold[b] != 0:
 * first block, L = min(l_min, W_b) and the signals are not read (cold may be NULL).
 * Outputs: L_out DEVICE [n_seqs]; S_out DEVICE, indexed like I (nullable); margin_out DEVICE [n_seqs]
 * (nullable) = the smallest |decision quantity| examined up to the crossing.
 * Errors: DLM_EINVAL (null, n_seqs < 1, lambda <= 0, l_min < 1, bad mode/rule, radius < 0),
 * DLM_ECAPACITY (W_b < 1 or > 256, n_seqs > 32). */
typedef struct {
  float lambda;
  int32_t l_min, smooth_radius, norm_mode, rule;
} dlm_boundary_params;

int block_boundary(const float* I, const float* H, const int32_t* win_start, const int32_t* win_len, const int32_t* cold,
                   int n_seqs, const dlm_boundary_params* p, int32_t* L_out, float* S_out,
                   float* margin_out, void* stream);

/* ---- select_parallel ----------------------------------------------------------------------- */

/* CAP-Decoding (Sec. 4.3, Alg. 1).  The block of sequence b is the block_len[b] <= 256 rows
 * starting at row row_start[b] of logits / lse / conf / argmax, and the same positions start at
 * tokens[tok_start[b]].  A row is eligible iff its token equals mask_id.
 *   mode 0: pool = eligible rows with conf >= tau_low (Eq. 5); i, j conflict iff
 *           (logit_i[y_j] - lse_i) + (logit_j[y_i] - lse_j) > gamma (Eq. 6); phase 1 takes every
 *           pooled row with conf >= tau_high and drops their conflicts; phase 2 walks the rest by
 *           descending conf (ties: lower row first), taking a row and dropping its conflicts;
 *           if nothing was taken, the most confident eligible row alone.
 *   mode 1: every eligible row with conf >= tau_high, else the most confident one (the
 *           confidence-threshold rule of Sec. 5.1);  mode 2: the most confident one only.
 * Outputs: selected_out DEVICE uint8 [same indexing as logits rows; only block rows written];
 * n_selected_out DEVICE [n_seqs]; if apply_tokens != 0, tokens[i] = argmax[i] for the selected
 * rows (Eq. 2); margin_out DEVICE [n_seqs] (nullable) = the smallest distance of an examined
 * quantity from the threshold or neighbour that decides it.  An argmax entry outside [0, vocab) is
 * clamped into it before it indexes the logits.
 * Errors: DLM_EINVAL (null, n_seqs < 1, bad dtype/mode, tau_high < tau_low in mode 0, vocab < 2),
 * DLM_ECAPACITY (block_len < 0 or > 256, n_seqs > 32). */
typedef struct {
  float tau_low, tau_high, gamma;
  int32_t mode;
} dlm_select_params;

int select_parallel(const void* logits, int vocab, int dtype, const float* lse, const float* conf,
                    const int32_t* argmax, int32_t* tokens, const int32_t* row_start,
                    const int32_t* tok_start, const int32_t* block_len, int n_seqs, int mask_id,
                    const dlm_select_params* p, int apply_tokens, uint8_t* selected_out,
                    int32_t* n_selected_out, float* margin_out, void* stream);

/* ---- components of dlm_step, exported for isolated tests and measurement --------------------- */

/* The vocabulary reduction of dlm_step on its own.  logits DEVICE [rows, vocab]; prev (nullable)
 * DEVICE [rows, vocab] of the same dtype gives kl per row (else kl = 0); prev_lse (nullable) DEVICE
 * [rows] fp32: the log-sum-exp of each prev row as an earlier call returned it in `lse` (dlm_step
 * keeps it with the retained logits); NULL: recomputed from prev in the same pass.  Same outputs and
 * definitions as dlm_step.  workspace: DEVICE scratch of at least dlm_vocab_stats_workspace(rows)
 * bytes.  Errors: DLM_EINVAL, DLM_ECAPACITY (rows < 1, workspace too small). */
size_t dlm_vocab_stats_workspace(int rows);
int dlm_vocab_stats(const void* logits, const void* prev, const float* prev_lse, int rows, int vocab, int dtype, int mask_id,
                    float* max_logit, float* lse, float* entropy, float* kl, float* conf,
                    int32_t* argmax, void* workspace, size_t workspace_bytes, void* stream);

/* dlm_vocab_stats for callers that cannot allocate or pass a workspace (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): same arguments, outputs and definitions, but the partial states live in a
 * file-scope device array of the library (4 MiB per GPU the library runs on, held until the process ends), whose address
 * is resolved once per device (at the first dlm_model_create on that device, else at the first call).  No hipMalloc,
 * hipFree or other allocating call is made.  Limit: rows <= 4096 (DLM_ECAPACITY beyond; use dlm_vocab_stats there).
 * All calls on one GPU share the array: calls that overlap on one GPU (different streams, different threads) race;
 * calls on one stream are ordered and safe.  Errors: DLM_EINVAL, DLM_ECAPACITY, DLM_EHIP (address resolution failed). */
int dlm_vocab_stats_static(const void* logits, const void* prev, const float* prev_lse, int rows, int vocab, int dtype, int mask_id,
                           float* max_logit, float* lse, float* entropy, float* kl, float* conf, int32_t* argmax,
                           void* stream);

/* y[M, N] = x[M, K] * w[N, K]^T with fp32 accumulation; all row-major DEVICE, dtype for x, w and y.
 * A test helper around the GEMM kernels of dlm_step: for DLM_BF16 it allocates scratch, re-tiles x
 * and w (dlm_step keeps both tiled) and synchronises the stream before returning; K, N multiples
 * of 32.  Errors: DLM_EINVAL, DLM_ESHAPE, DLM_ENOMEM, DLM_EHIP. */
int dlm_gemm_nt(const void* x, const void* w, void* y, int M, int N, int K, int dtype, void* stream);

/* out[A, n_q, hd] = softmax(q k^T / sqrt(hd)) v without mask; q [A, n_q, hd], k and v [T, n_kv, hd],
 * all DEVICE row-major of `dtype`; the attention kernel of dlm_step on dense operands.
 * Errors: DLM_EINVAL, DLM_ESHAPE. */
int dlm_attention(const void* q, const void* k, const void* v, void* out, int A, int T, int n_q, int n_kv,
                  int head_dim, int dtype, void* stream);

/* ---- an 8-bit KV cache, and what feeds and reads it -------------------------------------------------
 * For callers that keep a cache of their own beside (or instead of) a dlm_state's half-precision one: queries and keys
 * normalised and rotated, K and V quantised as they are written, read back, and the attention of packed rows over them.
 * Sequences are packed as in dlm_step: sequence b owns rows [row_offsets[b], row_offsets[b+1]) of every per-row array (a
 * sequence may have none), host arrays have n_seqs entries (row_offsets one more; row_offsets[0] == 0), slot NULL means
 * 0, 1, ...; at most 32 sequences.  Rows are row-major with a stride in elements, so that they can be columns of a wider
 * matrix (the fused QKV product); DEVICE pointers are 16-byte aligned and strides multiples of 16 bytes (DLM_EINVAL
 * otherwise).  head_dim in {32, 64, 128}; dtype DLM_F32 or DLM_BF16.  None of the calls allocates or synchronises: all can
 * be captured into a graph, with the host arrays as they were at capture. */

/* Queries and keys as an attention reads them.  A row of x holds n_q query heads and then n_kv key heads of head_dim values (either
 * count may be 0; what lies behind them is neither read nor written).  Per head:
 *   y = x * rsqrt(mean(x^2) + eps) * gain          (q_gain / k_gain DEVICE [head_dim] of dtype; NULL: y = x)
 *   out_i = y_i cos a - y_j sin a, out_j = y_j cos a + y_i sin a,   j = i + head_dim/2, a = position * theta^(-2 i / head_dim)
 * positions DEVICE [rows], any int32; the angle is computed in 64 bits, sums are fp32 (the squares of a head that is normalised have to
 * sum within its range), values are rounded once.  out may be x (with the same stride); else the two must not overlap (columns of one
 * matrix do not; with different strides, from the first row to the last).  Errors: DLM_EINVAL (null pointer, alignment, stride shorter
 * than a row, overlap, eps or theta not positive and finite, bad dtype), DLM_ESHAPE (rows < 0, heads, head_dim), DLM_ECAPACITY (more than
 * 67108860 rows), DLM_EHIP. */
int dlm_qk_norm_rope(const void* x, int64_t x_stride, int rows, int n_q, int n_kv, int head_dim, int dtype, const void* q_gain,
                     const void* k_gain, float eps, float theta, const int32_t* positions, void* out, int64_t out_stride, void* stream);

/* A cache of n_slots sequences of up to max_len (at most 2^31 - 256) positions, in caller-owned DEVICE memory of dlm_kv8_bytes(...) bytes (0: an
 * unsupported shape) at a multiple of 16, zero-filled before its first use.  Each vector (K or V of one position and kv head) is held
 * as 8-bit codes and a scale 2^E: E is the smallest integer in [-60, 60] with max|x| <= M 2^E, a code is x 2^-E rounded to the
 * format (ties to even, saturated where E = 60 is not enough).  DLM_KV8_E4M3: 8-bit floating point with 3 fraction bits, M = 448;
 * DLM_KV8_I8: integers, M = 127.  A vector with a NaN or an infinity reads as all NaN; a position never written reads as 0. */
enum { DLM_KV8_E4M3 = 0, DLM_KV8_I8 = 1 };
typedef struct {
  int32_t n_slots, max_len, n_kv, head_dim, format;
  void* data; /* DEVICE */
} dlm_kv8_cache;
size_t dlm_kv8_bytes(int n_slots, int max_len, int n_kv, int head_dim);

/* Row r of sequence b (k and v: [rows, n_kv * head_dim] at row_stride) becomes position start[b] + r of its slot; a slot may be given
 * once.  dlm_kv8_read writes the values the positions stand for (exact in both dtypes) to k and v; slots may repeat, k and v must
 * not overlap (columns of one matrix do not).  Positions outside the spans, and rows behind the last sequence, are left as they are.
 * Errors: DLM_EINVAL (null pointer, alignment, stride, overlap with each other or the cache, bad dtype or format, offsets, slot),
 * DLM_ESHAPE (cache shape), DLM_ECAPACITY (n_seqs > 32, a span beyond max_len, 2^24 blocks of 32 positions of one head or more), DLM_EHIP. */
int dlm_kv8_write(const dlm_kv8_cache* c, const void* k, const void* v, int64_t row_stride, int dtype, const int32_t* row_offsets,
                  const int32_t* start, const int32_t* slot, int n_seqs, void* stream);
int dlm_kv8_read(const dlm_kv8_cache* c, void* k, void* v, int64_t row_stride, int dtype, const int32_t* row_offsets, const int32_t* start,
                 const int32_t* slot, int n_seqs, void* stream);

/* out[rows, n_q, head_dim] (contiguous) = softmax(q K^T / sqrt(head_dim)) V per row and head; query head h reads kv head
 * h / (n_q / n_kv).  mask NULL: every row of sequence b sees positions [0, n_keys[b]) of its slot.  mask DEVICE [rows, mask_words]
 * uint32: the last positions of the n_keys[b] (at least the sequence's row count nr) are its rows' own; a row sees the n_keys[b] - nr
 * before them and position n_keys[b] - nr + j where bit j % 32 of word j / 32 of its mask is set (32 mask_words >= nr): a tree of
 * drafted tokens sets its ancestors' bits and its own, a causal span the bits up to its own.  A row that sees nothing (or n_keys 0)
 * gives zeros; keys and values that a row does not see do not touch it, whatever they are, NaN or infinite ones that it sees make it NaN.
 * Slots may repeat.  q is read as it is (fp32: products to 22 bits of it), probabilities multiply values with 11 bits (fp32: 22), their
 * sum is fp32.  The products of q with the keys that a row sees, element by element and summed, have to be within fp32's range.  Where the
 * scales of two values that it sees lie 2^B apart (at most 2^120), the smaller one counts for nothing below a probability of 2^(B-134) of
 * the other's (fp32: 2^(B-139)).  A position never written that a row sees is a key and a value of zeros (DLM_KV8_I8: up to 2^-53).  out
 * must not overlap what is read, nor the workspace anything else.
 * workspace: DEVICE scratch at a multiple of 16, for calls that share a sequence's keys between workgroups; nothing needs more than
 * dlm_kv8_attention_workspace(rows, n_q, head_dim) bytes, and many calls need none (then it may be NULL).  It is in use until the
 * call's work is done: calls that may overlap need one each.
 * Errors: DLM_EINVAL (null pointer, alignment, stride, overlap, bad dtype or format, offsets, slot, n_keys < 0 or, with a mask, < nr),
 * DLM_ESHAPE (cache shape, n_q), DLM_ECAPACITY (n_seqs > 32, n_keys > max_len, mask_words or workspace too small, more than
 * 65535 tiles of 32 queries of a kv head: rows * n_q / n_kv beyond 2 million), DLM_EHIP. */
size_t dlm_kv8_attention_workspace(int rows, int n_q, int head_dim);
int dlm_kv8_attention(const dlm_kv8_cache* c, const void* q, int64_t q_stride, void* out, int dtype, int n_q, const int32_t* row_offsets,
                      const int32_t* n_keys, const int32_t* slot, int n_seqs, const uint32_t* mask, int mask_words, void* workspace,
                      size_t workspace_bytes, void* stream);

/* ---- linear layers in 8-bit integers -----------------------------------------------------------------
 * For callers that run layers of their own around this library: activations quantised by row, weights by output channel, and products
 * of the two on the 8-bit matrix cores, at half of bf16's weight bytes and twice its matrix rate.
 * A row is held as codes, integers q in [-127, 127], and an fp32 scale s, and stands for s q.  Rows are row-major with a stride in elements
 * (codes: bytes), so that they can be columns of a wider matrix; DEVICE pointers are 16-byte aligned (scales: 4) and strides multiples of 16
 * bytes (DLM_EINVAL otherwise).  Rows of codes that are read own their bytes up to the next multiple of 16: what those hold does not matter, but
 * they have to be readable.  dtypes DLM_F32 or DLM_BF16.  None of the calls allocates or synchronises: all can be captured into a graph. */

/* A row t is quantised as q = 127 t / max|t| rounded to the nearest integer (ties to even, of the exact quotient), s = max|t| / 127; a row of
 * zeros has q = 0 and s = 0.  A row with a NaN or an infinity has q = 0 and s = NaN, so that what is computed from it is NaN.
 * dlm_q8_rows: t = x [rows, width].
 * dlm_add_norm_q8: h = residual + x, rounded once to h_dtype and written to h [rows, width]; y = h rsqrt(mean(h^2) + eps) gain is what is
 * quantised: t = h gain, rounded to fp32 (bf16: exact) gives the codes, and s = max|t| rsqrt(mean(h^2) + eps) / 127.  residual and h are of h_dtype, DLM_F32
 * or x's; both NULL: h = x.  gain DEVICE [width] of dtype.  The squares are summed in fp32: a row whose sum is past its range counts as one with an infinity.  h may be
 * residual or x (with the same stride and type); nothing else that is written may overlap anything.
 * Errors: DLM_EINVAL (null pointer, alignment, stride, overlap, eps not positive and finite, bad dtype), DLM_ESHAPE (rows < 0, width not in
 * 1 .. 1048576), DLM_ECAPACITY (more than 4194303 rows), DLM_EHIP. */
int dlm_q8_rows(const void* x, int64_t x_stride, int rows, int width, int dtype, int8_t* codes, int64_t codes_stride, float* scale, void* stream);
int dlm_add_norm_q8(const void* x, int64_t x_stride, int rows, int width, int dtype, const void* residual, int64_t residual_stride, void* h,
                    int64_t h_stride, int h_dtype, const void* gain, float eps, int8_t* codes, int64_t codes_stride, float* scale, void* stream);

/* A weight of n output channels by k inputs in caller-owned DEVICE memory of dlm_q8_weight_bytes(...) bytes (0: an unsupported shape: n not in
 * 1 .. 16777216, k not in 1 .. 131071, gated and n odd, more than 32 GiB) at a multiple of 16, in the order in which the matrix cores take it; dlm_q8_weight_pack
 * writes it from row-major codes [n, k] (any int8, -128 too) and their scales [n].  gated = 1: the channels are n / 2 gate channels and then n / 2
 * up channels (as w_gate_up), 0: the outputs themselves.  Errors: DLM_EINVAL (null pointer, alignment, stride, overlap, gated), DLM_ESHAPE, DLM_EHIP. */
typedef struct {
  int32_t n, k, gated;
  void* data; /* DEVICE */
} dlm_q8_weight;
size_t dlm_q8_weight_bytes(int n, int k, int gated);
int dlm_q8_weight_pack(const dlm_q8_weight* w, const int8_t* codes, int64_t codes_stride, const float* scale, void* stream);

/* out [rows, n] = x_scale[m] scale[j] sum_k x[m][k] codes[j][k]: the sum exact, converted to fp32 and multiplied by the row's and then the channel's
 * scale.  gated: out [rows, n / 2] = g / (1 + exp(-g)) u of the gate's and the up channel's values.  Before the output's rounding, plain values are off by 3 x 2^-24
 * of themselves, gated ones by (13 + 6 |g|) x 2^-24, and by 2^-125 |g u| at most below g = -87.3, where they may be zero.  Rounded once to out_dtype; columns behind
 * the outputs are left as they are.  x [rows, k] codes (any int8) and x_scale [rows]; nothing may overlap out.
 * workspace: DEVICE scratch at a multiple of 16 of dlm_q8_gemm_workspace(r, n, k, gated) bytes for some r >= rows (0: none is needed, it may be NULL), for
 * products that share K between workgroups (rows up to r; plan[5] KiB of dlm_plan_q8_gemm are enough for those rows alone).  It is in use until the
 * call's work is done: calls that may overlap need one each.
 * Errors: DLM_EINVAL (null pointer, alignment, stride, overlap, bad dtype, gated), DLM_ESHAPE (weight, rows < 0), DLM_ECAPACITY (workspace too small,
 * more than 1048576 rows or 2^38 outputs, or a launch of 2^32 threads: gated, some products of 0.99 x 2^38 outputs and more), DLM_EHIP. */
size_t dlm_q8_gemm_workspace(int rows, int n, int k, int gated);
int dlm_q8_gemm(const dlm_q8_weight* w, const int8_t* x, int64_t x_stride, const float* x_scale, int rows, void* out, int64_t out_stride, int out_dtype,
                void* workspace, size_t workspace_bytes, void* stream);

/* ---- what the GPU achieves on the resources the rooflines are drawn against -------------------
 * For callers that report measurements (bench.py): kernels that do nothing but the one thing, timed
 * with events on `stream`, which is synchronised before the call returns.
 *
 * dlm_probe_hbm_read: streams `bytes` of DEVICE memory at src `reps` times (16-byte loads, every byte
 * once per repetition; use a buffer larger than the 256 MB memory-side cache) and reports the read
 * rate in GB/s.  dlm_probe_mfma: `reps` launches of independent 16x16x32 half-precision products out of
 * registers on every SIMD, on operands of pseudo-random values (what the chip sustains then is set by
 * its power limit, below the published rate, which constant operands reach), reports TFLOP/s.
 * Errors: DLM_EINVAL, DLM_ESHAPE (fewer than 16 MiB), DLM_ENOMEM, DLM_EHIP. */
int dlm_probe_hbm_read(const void* src, size_t bytes, int reps, double* gb_per_s, void* stream);
int dlm_probe_mfma(int reps, double* tflop_per_s, void* stream);

/* Where dlm_step takes the vocabulary statistics of a bf16 model's pass that compares no row with a
 * retained distribution and retains none (kl_count and save_count all zero: the in-block passes of
 * Sec. 4.3) and has at most 64 rows.  enable != 0 (the default of a new state): from the LM-head
 * GEMM's epilogue, which leaves one online-softmax state (maximum, sum of exponentials, their
 * logit-weighted sum, lowest token id of the maximum; Sec. 4.2 entropy, Sec. 4.3 confidence and
 * prediction) per row and column group, finished by a small merge: the logits are written but
 * not read back.  enable == 0: from the streamed reduction over the written logits, as every other
 * pass does.  Both take the logits as written (rounded to the model's dtype) and leave out the mask
 * token; their results differ only in the order of the fp32 sums.  Errors: DLM_EINVAL (null state). */
int dlm_state_fuse_stats(dlm_state* s, int enable);

/* Per-kernel-class timing of dlm_step: the launches of every class whose bit is set in class_mask
 * are bracketed by HIP events on the caller's stream (0 switches the timing off; events cost queue
 * time, so bracket few classes when a class's own duration matters).  dlm_profile_read synchronises
 * those events and returns, per class c < n, the accumulated milliseconds and launch count since the
 * last reset.  Classes: 0 QKV GEMM, 1 O GEMM, 2 gate/up GEMM, 3 down GEMM, 4 LM-head GEMM,
 * 5 attention, 6 vocabulary statistics, 7 other (row tables, embedding, and for fp32 models the
 * row-wise glue). */
int dlm_profile_enable(dlm_state* s, unsigned class_mask);
int dlm_profile_read(dlm_state* s, int n, double* ms_out, int64_t* launches_out, int reset);

/* ---- what the launch rules choose for a shape ---------------------------------------------------
 * Host arithmetic only (no GPU call): for tests that have to reach one variant of a kernel, and for tuning.
 *
 * dlm_plan_attention: a bf16 model's attention over n_seqs spans of which the longest has max_seq_rows
 * rows.  plan[0] wavefronts of a workgroup, plan[1] workgroups that share a head's output dims, plan[2]
 * 16-query tiles of a workgroup.
 * dlm_plan_vocab_stats: the streamed vocabulary reduction.  plan[0] threads of a workgroup, plan[1] chunks
 * a row is cut into (more than one: a second launch merges them).
 * dlm_plan_gemm: a bf16 model's product of M rows with a matrix [N, K] (N and K multiples of 32); epilogue:
 * 0 plain without a workspace (LM head), 1 QKV, 2 gated, 3 residual, 4 plain (dlm_gemm_nt), 5 LM head with
 * statistics (at most 64 rows).  plan[0] kernel (0 skinny, 1 mid, 2 macro), plan[1], plan[2] rows and columns of
 * a workgroup's tile, plan[3] workgroups that share a tile by splitting K, plan[4] parts K is summed in,
 * plan[5] workgroups, plan[6] chunks of the rows' sums of squares per column block (epilogue 3).
 * dlm_plan_q8_gemm: dlm_q8_gemm of `rows` rows (a stride of up to 4 MiB between them) with a weight [n, k].  plan[0] kernel (0 streamed, 1 tiled, 2 banded),
 * plan[1], plan[2] rows and packed channels of a workgroup's tile, plan[3] workgroups that share a tile by splitting K, plan[4] workgroups, plan[5] KiB of
 * workspace.
 * Errors: DLM_EINVAL (null, bad dtype, epilogue or gated), DLM_ESHAPE (a size out of range, head_dim not in {32, 64, 128}). */
int dlm_plan_vocab_stats(int rows, int vocab, int dtype, int32_t plan[2]);
int dlm_plan_gemm(int M, int N, int K, int epilogue, int32_t plan[7]);
int dlm_plan_attention(int max_seq_rows, int n_seqs, int n_q, int head_dim, int32_t plan[3]);
int dlm_plan_q8_gemm(int rows, int n, int k, int gated, int32_t plan[6]);

#ifdef __cplusplus
}
#endif
#endif
