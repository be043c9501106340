/*
 * Kernel-level entry points of libdare: each one enqueues a single stage of the
 * layer step of dare.h on a HIP stream.  dare_layer_step() is built from exactly
 * these stages; they are exported so that each can be checked against its
 * definition and timed on its own.  All data pointers are DEVICE memory owned by
 * the caller; calls are asynchronous and never synchronise.  dtype is a
 * dare_dtype.  Argument errors return DARE_ERR_INVALID_ARG / UNSUPPORTED before
 * anything is enqueued.
 */
#ifndef DARE_KERNELS_H
#define DARE_KERNELS_H

#include <stddef.h>
#include <stdint.h>
#include "dare.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Re-pack a projection weight: wt[n, k] = w[k, n] (w is [rows_k, cols_n]
 * row-major, the Y = X W orientation of Sec. 3.2 eq. 3; wt is [cols_n, rows_k]
 * row-major with leading dimension ldwt >= rows_k).  The GEMM below consumes wt.
 */
dare_status dare_k_pack_weight(int dtype, const void* w, int rows_k, int cols_n,
                               void* wt, int ldwt, void* hip_stream);

/*
 * Row-selected projection (Alg. 1 lines 6-7 and 11; Alg. 2 lines 2, 7, 11):
 *     C[t, 0:n] = A[t, 0:k] . W          for t in rows
 * rows = idx[0 .. m) when idx != NULL (flat token ids; the same id addresses the
 * row of A that is read and the row of C that is written), else 0 .. m-1.
 * m = *m_dev (a device int32, read by the kernel) when m_dev != NULL, else m_max;
 * m_max bounds the launch and must be >= *m_dev.
 *   a    [*, lda] dtype, k contiguous          wt [n, k] dtype (packed weight)
 *   c    column segment s = col / seg_n goes to c[s] (up to 3 segments, each
 *        [*, ldc] dtype); seg_n must divide n; unused entries NULL
 *   c32  optional fp32 copy [*, c32_cols] (leading dimension c32_cols) of output
 *        columns [0, c32_cols), taken from the fp32 accumulators before rounding
 *        to dtype: the input of the drift score.  c may be all NULL when only
 *        c32 is wanted (then n == c32_cols).
 *   k_parts  1, or (bf16, all rows, c all NULL, c32_cols == n) a divisor of k/64: k is
 *        cut into k_parts ranges computed by separate workgroups, and range s writes
 *        its partial products to c32 + s * c32_part_stride (elements).  The sum over s,
 *        taken in order, is the projection; dare_k_score adds the slabs itself.  Meant
 *        for the scored query columns of all rows (few output tiles, long k).
 * k must be a multiple of 64, n of 64 (bf16) / 16 (fp32).
 */
dare_status dare_k_gemm(int dtype, const void* a, int lda, const void* wt, int n,
                        int k, int m_max, const int32_t* idx,
                        const int32_t* m_dev, void* const* c, int ldc, int seg_n,
                        float* c32, int c32_cols, int k_parts, long c32_part_stride,
                        void* hip_stream);

/*
 * Drift score and reuse decision (Sec. 3.1 eq. 1, Sec. 3.2 eq. 2; Alg. 1/2
 * lines 3-5) for n_tokens tokens:
 *   s = 1 - <q, p> / max(sqrt(|q|^2 |p|^2), 1e-30), q = q_new[t, 0:width],
 *   p = q_prev[t, 0:width]; mask = (s <= threshold) unless force_refresh;
 *   then q_prev[t] = q.
 *   q_new [n_tokens, ld_new] fp32, or n_parts such slabs part_stride elements apart
 *   whose sum (taken in slab order) is q; q_prev [n_tokens, width] fp32 in/out;
 *   scores optional [n_tokens] fp32; mask [n_tokens] bytes.
 */
dare_status dare_k_score(const float* q_new, int ld_new, int width, int n_parts,
                         long part_stride, float* q_prev, int n_tokens,
                         float threshold, int force_refresh, float* scores,
                         uint8_t* mask, void* hip_stream);

/*
 * Ordered compaction of the refreshed set (Alg. 1/2 line 5): sel_idx = ascending
 * flat ids b*seq+i with mask == 0; sel_count[b] per sequence; sel_off[b] = number
 * of refreshed tokens in sequences before b, sel_off[batch] = total.
 * sel_idx [batch*seq], sel_count [batch], sel_off [batch+1], all int32; any of
 * the three may be NULL.
 */
dare_status dare_k_compact(const uint8_t* mask, int batch, int seq,
                           int32_t* sel_idx, int32_t* sel_count,
                           int32_t* sel_off, void* hip_stream);

/*
 * Bidirectional multi-head attention for selected query rows (App. E.2; Alg. 1
 * line 10; Alg. 2 line 8):
 *   out[t, h] = softmax(q[t, h] . K_b[:, h]^T / sqrt(head_dim)) V_b[:, h]
 * for every head h and every token t of the row set; b = t / seq is the
 * sequence of t, and keys/values are all seq rows of that sequence.
 * Row set: all tokens when idx == NULL; else idx[sel_off[b] .. sel_off[b+1]) for
 * each sequence b (idx, sel_off as produced by dare_k_compact).
 *   q, k, v, out  [batch*seq, n_heads*head_dim] dtype, token-indexed rows
 */
dare_status dare_k_attention(int dtype, const void* q, const void* k,
                             const void* v, void* out, int batch, int seq,
                             int n_heads, int head_dim, const int32_t* idx,
                             const int32_t* sel_off, void* hip_stream);

/*
 * Row copy between token-indexed buffers: dst[t] = src[t] for t in idx[0..*m_dev)
 * (idx != NULL) or for all n_rows rows (idx == NULL).  row_bytes is a multiple
 * of 16.  Used to mirror the layer output between out and o_cache when they are
 * different buffers (Alg. 2 lines 9-10).
 */
dare_status dare_k_copy_rows(const void* src, void* dst, int n_rows,
                             int row_bytes, const int32_t* idx,
                             const int32_t* m_dev, void* hip_stream);

/*
 * Threshold from a reuse rate and the decision under it (Sec. 3.1 "Reuse rate
 * allocation"; rule as dare_set_threshold_rule in dare.h).  scores [batch, seq] fp32.
 * phi in [0, 1]: per sequence tau = k-th smallest score, k = ceil(phi * seq) in fp32;
 * writes tau_out[batch] (optional) and mask[batch, seq] = (score <= tau), all 0 when
 * force_refresh.  phi < 0: statistics only, mask and tau_out are not touched.
 * stat_sum / stat_count (both or neither): device arrays of [batch] slots; the sum and the
 * number of the non-NaN scores of sequence b are added to slot b (plain read-modify-write by
 * the one workgroup that owns the sequence: no atomics, the same result from run to run).
 */
dare_status dare_k_quantile_mask(const float* scores, int batch, int seq, float phi,
                                 int force_refresh, float* tau_out, uint8_t* mask,
                                 double* stat_sum, uint64_t* stat_count, void* hip_stream);

/*
 * The projection above with the rotary embedding in its epilogue (see dare_block_config
 * in dare.h): output columns [0, rope_cols) are rotated, channel pair (2i, 2i+1) of
 * every head_dim-wide head by the angle whose (cos, sin) is
 * rope_table[(t % seq) * head_dim/2 + i], t the token id of the row; the fp32 copy c32
 * keeps the unrotated values.  rope_table: fp32 [positions, head_dim/2, 2].  rope_cols
 * is a multiple of head_dim; seg_n a multiple of head_dim.  No k_parts.
 */
dare_status dare_k_gemm_rope(int dtype, const void* a, int lda, const void* wt, int n,
                             int k, int m_max, const int32_t* idx,
                             const int32_t* m_dev, void* const* c, int ldc, int seg_n,
                             float* c32, int c32_cols, const float* rope_table,
                             int rope_cols, int head_dim, int seq, void* hip_stream);

/*
 * Rotary table for positions 0 .. n_pos-1: table[p, i] = (cos, sin) of
 * p * base^(-2i / head_dim), computed on the HOST in double precision and copied to
 * the device pointer `table` (fp32 [n_pos, head_dim/2, 2]) with a synchronous copy.
 */
dare_status dare_k_rope_table(float* table, int n_pos, int head_dim, double base);

/*
 * Normalisation of token rows (Alg. 1/2 line 1): kind DARE_NORM_LAYER or
 * DARE_NORM_RMS, formulas as in dare_block_config.  x, out [n_rows, d] dtype (out may
 * be x), gain [d], bias [d] or NULL; d a multiple of 8; fp32 statistics.
 */
dare_status dare_k_norm(int dtype, int kind, const void* x, const void* gain,
                        const void* bias, float eps, int n_rows, int d, void* out,
                        void* hip_stream);

/* Residual sum out = x + o over n_elems elements (a multiple of 8) of dtype. */
dare_status dare_k_residual_add(int dtype, const void* x, const void* o, void* out,
                                long n_elems, void* hip_stream);

/*
 * Operators of a decoder layer whose query heads share key heads, with biases, sequences of different lengths and
 * caches that reach behind the tokens of a call.  Sizes of 0 tokens are fine (nothing is enqueued); every ld is the
 * distance of two rows in elements, and what is read or written by rows lies on 16-byte boundaries (pointers, and ld times
 * the size of an element) unless it says otherwise.  dare_last_error(NULL) has the text of a refusal.
 */
enum { DARE_ACT_NONE = 0, DARE_ACT_SILU = 1, DARE_ACT_GELU = 2, DARE_ACT_GELU_TANH = 3 };

/*
 * Projection with its epilogue, one rounding at the end:
 *     out[t, 0:n] = act(a[t, 0:k] . W + bias) + residual[t, 0:n]        for t in [0, m)
 * act: none; silu z / (1 + e^-z); gelu z Phi(z); its tanh form z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2.
 * Of -infinity gelu is 0, the others are NaN, in both types.
 *   a [m, lda], residual [m, ldr] (or NULL), out [m, ldo] dtype; wt [n, k] (packed weight), bias [n] (or NULL) dtype
 * out may be residual (with the same ld); it must not overlap a.  k and n are multiples of 64.
 * Errors: INVALID_ARG (null pointer, ld below the row's width, alignment, unknown act), UNSUPPORTED (k or n not a
 * multiple of 64, m beyond 2^24, n beyond 2^20, an ld beyond 2^24).
 */
dare_status dare_k_linear(int dtype, const void* a, long lda, const void* wt, int n, int k, int m, const void* bias,
                          int act, const void* residual, long ldr, void* out, long ldo, void* hip_stream);

/*
 * Rotary embedding by positions, with the cache rows it leads to.  Pair i of the first rot_dim channels of every head,
 * (a, b) = channels (2i, 2i + 1) for DARE_ROPE_PAIRS, (i, i + rot_dim / 2) for DARE_ROPE_HALF, becomes
 *     magnitude * (a cos - b sin, b cos + a sin),  angle = pos[t] * freqs[i] (formed and reduced in 64 bits);
 * channels from rot_dim on go through as they are.
 *   pos    [n_tokens] int32, any value           freqs  [rot_dim / 2] fp64 (dare_k_rope_freqs)
 *   q      [n_tokens, ldq], n_heads heads, rotated into q_out [n_tokens, ldqo]
 *   k      [n_tokens, ldk], n_kv_heads heads, rotated into k_out
 *   v      [n_tokens, ldv], n_kv_heads heads, copied into v_out
 *   rows   NULL: k_out and v_out have a row per token.  Else [n_tokens] int32: token t goes to row rows[t] of them, nowhere if that is
 *          outside [0, out_rows); no two tokens to the same row
 * Each of q, k and v may be NULL (with its output).  q_out may be q, and without rows k_out k and v_out v (with the same
 * ld); there is no other overlap.  head_dim is a multiple of 8 up to 256, rot_dim even, 2 .. head_dim, heads 1 .. 65535, n_tokens up to
 * 2^25, an ld up to 2^24.  Rows need no alignment but that of their elements.
 * Errors: INVALID_ARG (struct_size, null pointer, an input without its output, ld below the row's width, alignment, in place with rows or another ld,
 * rows without out_rows, unknown dtype or layout, magnitude not finite, rot_dim, heads out of range), UNSUPPORTED (head_dim, n_tokens or an ld
 * beyond what is said here).
 */
enum { DARE_ROPE_HALF = 0, DARE_ROPE_PAIRS = 1 };
typedef struct {
  uint32_t struct_size; /* = sizeof(dare_rope_call) */
  int32_t dtype, layout, n_tokens, head_dim, rot_dim;
  int32_t n_heads, n_kv_heads;
  int32_t out_rows;
  float magnitude;
  const int32_t* pos;
  const double* freqs;
  const int32_t* rows;
  const void *q, *k, *v;
  void *q_out, *k_out, *v_out;
  int64_t ldq, ldk, ldv, ldqo, ldko, ldvo;
} dare_rope_call;
dare_status dare_k_rope(const dare_rope_call* call, void* hip_stream);

/*
 * Frequencies for dare_k_rope: f_i = base^(-2i / rot_dim), changed for contexts longer than the trained one by `factor`:
 *   DARE_ROPE_SCALE_NONE    as they are
 *   DARE_ROPE_SCALE_LINEAR  f_i / factor (interpolated positions)
 *   DARE_ROPE_SCALE_BASE    base * factor^(rot_dim / (rot_dim - 2)) instead of base (rot_dim above 2): the slowest pair is interpolated,
 *                           the fastest left alone
 *   DARE_ROPE_SCALE_TURNS   f_i (g + (1 - g) / factor), g = clamp((turns_i - low) / (high - low), 0, 1), turns_i = context f_i /
 *                           (2 pi): pairs that turn `high` times in the trained context stay, those that turn `low` times are interpolated
 * Computed on the HOST in double precision and copied to the device pointer `freqs` (fp64 [rot_dim / 2]) with a
 * synchronous copy, which does not wait for other streams: nothing enqueued may still use the memory.
 */
enum { DARE_ROPE_SCALE_NONE = 0, DARE_ROPE_SCALE_LINEAR = 1, DARE_ROPE_SCALE_BASE = 2, DARE_ROPE_SCALE_TURNS = 3 };
dare_status dare_k_rope_freqs(double* freqs, int rot_dim, double base, int scaling, double factor, double context,
                              double low, double high);

/*
 * Attention over packed sequences with shared key heads.  Sequence b has the query tokens q_off[b] .. q_off[b + 1] - 1 and the
 * keys k_begin[b] .. k_end[b] - 1; its queries are the last len_q of its len_k positions (len_q may be the larger one).
 *     out[t, h] = softmax_j(scale q[t, h] . k[j, h / G]) v[j, h / G],   G = n_heads / n_kv_heads,
 * over the keys that the token sees: all of its sequence with causal_block = 0; else those whose position lies in its own
 * block of causal_block positions or in one before (1: causal).  A token that sees no key gets zeros.  What lies in
 * keys that a token does not see does not matter, infinities and NaN included.
 *   q, out       [total_q, ldq or ldo] dtype, n_heads heads of head_dim; out overlaps none of the inputs
 *   k, v         [k_rows, ldk or ldv] dtype, n_kv_heads heads: packed like the queries, or a cache
 *   q_off        [batch + 1] int32, ascending from 0; rows of out from q_off[batch] on are left as they are
 *   k_begin/end  [batch] int32, 0 <= begin <= end <= k_rows.  (Values outside are taken as the nearest inside, so nothing
 *                outside of q, k and v is read, and nothing outside of out written.)
 * max_q and max_k, the largest numbers of query tokens and keys of a sequence, choose how the work is cut: a
 * captured call may be replayed with other lengths.  Longer sequences than they say are right as well, only slower.
 * Logits, maxima and sums are held in fp32.  Probabilities go into the product with the values as fp32 in fp32; in bf16 to 2^-15 of each where
 * max_q G is 32 or less (single tokens), and rounded to bf16 (2^-8 of each, the sum being taken over them as rounded) where it is more.
 * workspace: dare_k_attention_packed_workspace() bytes (for the same call; it does not look at the pointers), 16-byte aligned, needed while the call runs, not
 * initialised and not kept; NULL if that is 0.  Calls that may overlap need one each.
 * Errors: INVALID_ARG (null pointer, ld below the row's width, alignment, n_heads not a multiple of n_kv_heads, scale not above 0 or not
 * finite, workspace too small), UNSUPPORTED (head_dim not 64 or 128; an ld beyond 2^24; total_q * n_heads + 128 batch beyond
 * 2^31; 2^24 blocks and more, of n_kv_heads (total_q G / R + batch), R = 16 in fp32, else 16, 32 or 128: the smallest that max_q G rows fit,
 * or 128).  The query of the workspace looks neither at pointers nor at the number of blocks, and refuses what else the call
 * refuses.
 */
typedef struct {
  uint32_t struct_size; /* = sizeof(dare_packed_call) */
  int32_t dtype, batch, total_q, k_rows, max_q, max_k;
  int32_t n_heads, n_kv_heads, head_dim;
  int32_t causal_block;
  float scale;
  int64_t ldq, ldk, ldv, ldo;
  const void *q, *k, *v;
  void* out;
  const int32_t *q_off, *k_begin, *k_end;
} dare_packed_call;
dare_status dare_k_attention_packed_workspace(const dare_packed_call* call, size_t* bytes);
dare_status dare_k_attention_packed(const dare_packed_call* call, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Operators of a step in 8 bits and of its output end: normalisation into codes, projection of codes, and what decides
 * from logits which positions to unmask.  Sizes of 0 rows are fine (nothing is enqueued), every ld is the distance of
 * two rows in elements, nothing is allocated and nothing kept.  dare_last_error(NULL) has the text of a refusal.
 *
 * Normalisation of token rows into 8-bit codes with a scale per row, behind the residual sum.  For row t of d channels
 *     s = x[t] + o[t], rounded to dtype (x[t] without o); x_out[t] = s
 *     y = s | (s - mean) / sqrt(var + eps) * gain + bias | s / sqrt(mean(s^2) + eps) * gain     (DARE_NORM_NONE | LAYER | RMS)
 *     scales[t] = max |y| / 127 rounded to fp32,  codes[t] = y / scales[t] to the nearest whole number, ties to even, in [-127, 127]
 * so that codes[t] * scales[t] stands for y.  Sums, y and the decision between two codes are formed in 64 bits.  A row
 * of zeros has the scale 0 and codes 0; one with a value that is not finite (zeros under DARE_NORM_RMS with eps 0 are),
 * or with a scale beyond fp32, the scale NaN and codes 0, and its projections are NaN.
 * The codes of a weight: DARE_NORM_NONE of the rows of the packed matrix (dare_k_pack_weight), one scale per output column.
 *   x, o, x_out  [n_rows, ldx | ldo | ldxo] dtype on 16-byte boundaries; o and x_out may be NULL; x_out may be x or o
 *                (with the same ld)
 *   gain, bias   [d] dtype on 16-byte boundaries; gain for both norms, bias (or NULL) for LAYER
 *   codes        [n_rows, ldc], on 8-byte boundaries          scales [n_rows]
 * There is no other overlap.  d is a multiple of 8.
 * Errors: INVALID_ARG (struct_size, null pointer, unknown dtype or kind, sizes, eps, ld below the row's width,
 * alignment, a gain or bias that the kind does not have), UNSUPPORTED (d not a multiple of 8 or beyond 2^24, n_rows
 * beyond 2^23, an ld beyond 2^24).
 */
typedef struct {
  uint32_t struct_size; /* = sizeof(dare_norm_q8_call) */
  int32_t dtype, kind, n_rows, d;
  double eps;
  int64_t ldx, ldo, ldxo, ldc;
  const void *x, *o, *gain, *bias;
  void* x_out;
  int8_t* codes;
  float* scales;
} dare_norm_q8_call;
dare_status dare_k_norm_q8(const dare_norm_q8_call* call, void* hip_stream);

/*
 * Projection of 8-bit codes with scales for each row and each column:
 *     out[t, c] = act(row_scale[t] col_scale[c] sum_k a[t, k] wt[c, k] + bias[c]) + residual[t, c]      for t in [0, m), c in [0, n)
 * The sum is exact, in 32-bit integers (codes -128 .. 127); scales, bias, activation (as in dare_k_linear) and residual
 * sum in fp32, one rounding to dtype, the type of bias, residual and out.
 *   a [m, lda], wt [n, k] codes and col_scale [n] on 16-byte boundaries; row_scale [m]
 *   bias [n] or NULL, residual [m, ldr] or NULL, out [m, ldo] dtype on 16-byte boundaries
 * out may be residual (with the same ld); there is no other overlap.  n is a multiple of 64, k of 128.
 * Errors: INVALID_ARG (struct_size, null pointer, sizes, ld below the row's width, alignment, unknown dtype or act),
 * UNSUPPORTED (n not a multiple of 64, k not of 128, k of 2^17 and more, m beyond 2^24, n beyond 2^20, m n beyond 2^37,
 * an ld beyond 2^24).
 */
typedef struct {
  uint32_t struct_size; /* = sizeof(dare_linear_q8_call) */
  int32_t dtype, m, n, k, act;
  int64_t lda, ldr, ldo;
  const int8_t* a;
  const float* row_scale;
  const int8_t* wt;
  const float* col_scale;
  const void *bias, *residual;
  void* out;
} dare_linear_q8_call;
dare_status dare_k_linear_q8(const dare_linear_q8_call* call, void* hip_stream);

/*
 * Log-probabilities of given tokens, entropy and the largest alternatives of rows of logits, p = softmax(scale logits[t, 0:vocab]):
 *     logprobs[t] = log p[tokens[t]],  entropy[t] = - sum p log p,
 *     top_ids[t, i], top_logprobs[t, i]: the i-th largest logit's id and log p, of equal logits the lower id first
 * A logit of -infinity has the probability 0: its log-probability is -infinity, it adds nothing to the entropy and is
 * no alternative.  Where a row has fewer alternatives than top, ids of -1 and log-probabilities of -infinity fill up; a
 * row without any has the entropy 0.  A token outside [0, vocab) has the log-probability -infinity.  A row with NaN or
 * +infinity: NaN, ids -1.
 * Sums in fp32, of max(64, vocab / 256) terms in a row at most; a log-probability or an entropy is off by a few 2^-23
 * of 1, of its size and of how far, in scaled logits, the probability lies from the largest one on average, whatever
 * the logits' own size, and by what the roundings of such a sum may add.  (Rows whose largest scaled logit is beyond
 * 5.8e6 are read twice where scale is below 65536.)
 *   logits [n_rows, ld] dtype, any alignment of an element; tokens [n_rows] int32 with logprobs [n_rows] fp32, or both
 *   NULL; entropy [n_rows] fp32 or NULL; top_ids [n_rows, top] int32, top_logprobs [n_rows, top] fp32
 * workspace: dare_k_logprobs_workspace() bytes (for the same sizes; it does not look at the pointers), 16-byte aligned,
 * needed while the call runs, not initialised and not kept; NULL if that is 0.  Calls that may overlap need one each.
 * Nothing overlaps.  top is 0 .. 32 and at most vocab; scale (1 / temperature) above 0, at most 1e30.
 * Errors: INVALID_ARG (struct_size, null pointer, unknown dtype, sizes, scale, ld below vocab, alignment, tokens
 * without logprobs or the other way round, workspace too small), UNSUPPORTED (top above 32, n_rows beyond 2^21, vocab
 * beyond 2^28, ld beyond 2^32).
 */
typedef struct {
  uint32_t struct_size; /* = sizeof(dare_logprobs_call) */
  int32_t dtype, n_rows, vocab, top;
  float scale;
  int64_t ld;
  const void* logits;
  const int32_t* tokens;
  float *logprobs, *entropy;
  int32_t* top_ids;
  float* top_logprobs;
} dare_logprobs_call;
dare_status dare_k_logprobs_workspace(const dare_logprobs_call* call, size_t* bytes);
dare_status dare_k_logprobs(const dare_logprobs_call* call, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DARE_KERNELS_H */
