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

#ifdef __cplusplus
}
#endif
#endif /* DARE_KERNELS_H */
