/*
 * mte_proj.h -- C ABI of the operators between the encoder's hidden states and the
 * attention that reads them, on MI355X (gfx950).
 *
 * The encoder (mte.h) ends at its hidden states, and the attentions of mte_cond.h
 * begin at queries, keys and values. Between the two lie the denoiser's projections
 * and, where its heads have one, a rotary embedding; and where all streams of a batch
 * share a long context (an instruction, a history; Sec. III-B's one encode for every frame of a
 * batch) beside each one's own tokens, an attention that reads the shared part once:
 *
 *   mte_i8_quantize_rows   rows as 8-bit integers with a scale each
 *   mte_i8_linear          their product with an 8-bit weight, bias and activation
 *   mte_rotary             rotary positions on queries and keys
 *   mte_prefix_attention   keys shared by all sequences, then each one's own
 *
 * Conventions as in mte_cond.h: device / host pointers, negative mte_status codes,
 * host-side checks before any HIP call, every call only enqueues work on `stream`
 * (graph-capturable) and runs on the current device, which must be the stream's; the
 * caller owns every buffer; workspaces as there. Forward only (the gradient of a
 * rotation is its inverse, which mte_rotary offers).
 */
#ifndef MTE_PROJ_H
#define MTE_PROJ_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#include "mte_cond.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows in 8 bits. Row r of a matrix [rows, cols] is held as codes c (int8, -127 .. 127)
 * and one scale s (float): x ~ c s, with
 *   s = max(max |x| * (1/127), 2^-126), factor and product rounded to fp32 (max |x| / 127, give or take
 *       one unit in the last place: the bits that torch's division by 127 has on this device, so that scales
 *       and codes made there are those made here),
 *   c = x / s rounded to the nearest whole number, ties to the even one (the exact
 *       quotient, not its fp32 rounding).
 * A row that holds an infinity or NaN gets the scale NaN and codes of zero.
 * Codes are stored with mte_i8_pitch(cols) bytes a row, cols rounded up to a multiple
 * of 128; the bytes past cols are zeros. cols is at most MTE_I8_COLS, so that a sum of
 * products of codes (also of -128, which a program that fills codes itself may use) fits 32 bits. */
#define MTE_I8_COLS 131071
int64_t mte_i8_pitch(int32_t cols);       /* or MTE_E_INVALID */

/*  x:      device, dtype (MTE_F32 / MTE_BF16), row r at x + r * x_row elements (x_row >= 0);
 *          aligned like one element.
 *  codes:  device int8 [rows][mte_i8_pitch(cols)], aligned to 16 bytes; scales: device float[rows].
 * Errors: MTE_E_INVALID, MTE_E_HIP. rows == 0 is MTE_OK. */
int mte_i8_quantize_rows(const void *x, int64_t x_row, int32_t rows, int32_t cols, int32_t dtype, int8_t *codes,
                         float *scales, hipStream_t stream);

/* y[i, j] = act(s_i t_j sum_k a[i, k] b[j, k] + bias[j]) for m rows of codes a (scales s) and
 * n of b (scales t): a linear layer whose weight [n, k] and tokens [m, k] are 8-bit rows.
 * The sum is exact (int32); what follows is fp32, rounded once to the result's type.
 *  x:        x_type MTE_I8_CODES: the codes a, with x_scales (x_row is not read).
 *            MTE_F32 / MTE_BF16: rows that the call quantises as mte_i8_quantize_rows does
 *            (x_row as there; x_scales is not read); the codes pass through the workspace.
 *  w:        device int8 [n][mte_i8_pitch(k)] and w_scales float[n].
 *  bias:     device, dtype, [n], or NULL; aligned like one element.
 *  act:      mte_activation.
 *  out:      device, dtype (MTE_F32 / MTE_BF16) [m, n], rows out_row >= n elements apart, aligned
 *            like one element (16 bytes and strides to match are faster); overlaps no input.
 *  workspace: device, at least mte_i8_linear_workspace(...) bytes, aligned to 16; NULL where that is 0.
 * Products are scaled by s_i 2^-31 and t_j 2^31: a row's scale below 2^-95 loses
 * precision there, and a weight's scale beyond 2^96 overflows. A NaN scale gives a row, or a column, of NaN.
 * The result does not depend on how the work is split. m is at most 2^31 - 4097, n likewise.
 * Errors: MTE_E_INVALID, MTE_E_CAPACITY (workspace_bytes), MTE_E_HIP. m == 0 is MTE_OK. */
#define MTE_I8_CODES 2                    /* x_type, beside the mte_dtype values */
int mte_i8_linear(const void *x, int64_t x_row, const float *x_scales, int32_t x_type, int32_t m, int32_t k,
                  const int8_t *w, const float *w_scales, int32_t n, const void *bias, int32_t act, void *out,
                  int64_t out_row, int32_t dtype, void *workspace, int64_t workspace_bytes, hipStream_t stream);
int64_t mte_i8_linear_workspace(int32_t x_type, int32_t m, int32_t k, int32_t n);

/* Rotary positions. Channels 0 .. rot_dim - 1 of every head (rot_dim even) are taken as rot_dim / 2 pairs:
 * pair i is channels (i, i + rot_dim / 2), or with interleaved (2 i, 2 i + 1). For a token
 *   y1 = factor (x1 cos a - x2 sin a),  y2 = factor (x2 cos a + x1 sin a),  a = p[axis(i)] freq[i];
 * inverse: -a in place of a (with the same factor it is the gradient of the rotation). Channels from
 * rot_dim on are copied. The angle is formed and reduced in fp64, so that far positions
 * keep theirs; sine, cosine and products are fp32, rounded once.
 * n_axes positions a token (1 .. 4): the first section[0] pairs take axis 0, the next section[1]
 * axis 1, ..; they sum to rot_dim / 2 (n_axes 1: section is not read). (The encoder's
 * MTE_MROPE_SECTIONS layout: 3 axes t, h, w with freq[i] = theta^(-2 i / d).)
 * Heads: q has n_q_heads, k has n_k_heads (0: no k; then k and k_out are not read). *_row / *_head:
 * strides in elements as in mte_attn_shape (0 or more, multiples of 8, 16-byte aligned bases). head_dim: a
 * multiple of 8, at most 512. q_out may be q (same strides; then channels from rot_dim on stay as they are),
 * k_out may be k; otherwise outputs overlap no input, nor each other. */
typedef struct {
  int32_t n_q_heads, n_k_heads, head_dim, rot_dim;
  int32_t dtype, interleaved, inverse, n_axes;
  int32_t section[4];
  float factor;
  int64_t q_row, q_head, k_row, k_head, qo_row, qo_head, ko_row, ko_head;
} mte_rotary_shape;
/*  positions: device int32, axis a of token i at a * axis_stride + i (n_axes 1: axis_stride is not read); any value.
 *  freq:      device double[rot_dim / 2], aligned to 8 bytes; |p freq| is at most 2^52.
 * Heads are at most 65535 each, tokens times heads 2^31 - 4097. Errors: MTE_E_INVALID, MTE_E_UNSUPPORTED (head_dim),
 * MTE_E_HIP. tokens == 0 is MTE_OK. */
int mte_rotary(const mte_rotary_shape *shape, const void *q, const void *k, const int32_t *positions,
               int64_t axis_stride, const double *freq, int32_t tokens, void *q_out, void *k_out, hipStream_t stream);

/* Attention of packed sequences that share a prefix: sequence i's q_lens[i] queries attend to the
 * prefix_len tokens that all of them share and then to its own kv_lens[i] tokens, in one softmax.
 * causal = 1: query u sees own tokens 0 .. kv_lens[i] - q_lens[i] + u only (the whole prefix in any
 * case). A query that sees nothing gets zeros. What tokens that a query does not see hold (infinities,
 * NaN) does not reach it. An infinite value of one that it sees is the result in its channel; where the weight is
 * below 2^-100 of the heaviest key's, it may be NaN instead.
 *  shape:      heads, types and strides as in mte_cross_attention (k_*, v_*: of the own tokens).
 *  prefix_k/v: device, prefix_len rows at the strides pk_row, pk_head, pv_row, pv_head.
 *  k, v:       device, sum(kv_lens) rows back to back; q, out, workspace as in mte_cross_attention.
 *  q_lens, kv_lens: HOST int32[n], each >= 0; n >= 1.
 * Few rows a sequence: the rows of all sequences are read as one tile over the prefix, which is
 * read once for all of them; many: a tile reads the prefix and its sequence's tokens in one pass.
 * Other sequences may change the last bits of a result. Errors and limits as in mte_cross_attention. */
int mte_prefix_attention(const mte_attn_shape *shape, const void *q, const void *prefix_k, const void *prefix_v,
                         int64_t pk_row, int64_t pk_head, int64_t pv_row, int64_t pv_head, int32_t prefix_len,
                         const void *k, const void *v, const int32_t *q_lens, const int32_t *kv_lens, int32_t n,
                         int32_t causal, void *out, void *workspace, int64_t workspace_bytes, hipStream_t stream);
int64_t mte_prefix_attention_workspace(const mte_attn_shape *shape, int32_t prefix_len, const int32_t *q_lens,
                                       const int32_t *kv_lens, int32_t n);

#ifdef __cplusplus
}
#endif

#endif /* MTE_PROJ_H */
