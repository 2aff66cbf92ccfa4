/*
 * mte_cond.h -- C ABI of the operators that read the encoder's conditioning on
 * MI355X (gfx950).
 *
 * The encoder (mte.h) ends at its hidden states. What the paper's pipeline does
 * with them next, once a frame and its instruction are encoded, is read them:
 * the denoiser's layers normalise their latents and attend from every latent
 * position to the conditioning tokens of its frame (Sec. III-A, where v_theta
 * takes the encoder's output h), and a stream may keep one encode for several
 * calls or for every frame of a batch (Sec. III-B, the optional TE caching
 * modes). This header has those reads:
 *
 *   mte_cross_attention   queries of one length, keys and values of another
 *   mte_kv8_append        keys and values into a cache held in 8 bits
 *   mte_kv8_attention     attention over that cache
 *   mte_kv8_read          cached rows back as bf16 / fp32
 *   mte_group_norm        group norm with an activation, channels last
 *
 * Conventions as in mte.h: device / host pointers, negative mte_status codes,
 * host-side checks before any HIP call, every call only enqueues work on
 * `stream` (no allocation, copy back or synchronisation; graph-capturable) and
 * runs on the device that is current, which must be the stream's. There is no
 * handle: the caller owns every buffer, the workspaces among them, and calls
 * that share no written buffer may overlap in time. A workspace needs no
 * initial value, carries nothing from one call to the next, and may be shared
 * by calls that run one after the other; not by calls (or replays of captured
 * graphs) that overlap in time. Everything is forward: results carry no gradient.
 */
#ifndef MTE_COND_H
#define MTE_COND_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#include "mte.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Heads, types and strides of an attention call.
 *  n_q_heads = Hq, n_kv_heads = Hkv (Hq % Hkv == 0; query head h reads kv head
 *  h / (Hq/Hkv)), head_dim = d.
 *  dtype: mte_dtype of q, k, v and out. Scores, softmax and sums are fp32; with
 *  MTE_BF16 the probabilities are rounded to 16 bits before they meet the values.
 *  scale: multiplies q.k; > 0, and finite also times log2(e).
 *  *_row / *_head: elements from one token's row to the next, and from one head
 *  to the next within a row (the d elements of a head are contiguous). The
 *  halves of a fused key/value projection are row strides of 2 Hkv d; a
 *  head-major tensor [H, T, d] is row d, head T d. A stride is 0 or more and a
 *  multiple of 8; every base address is aligned to 16 bytes. k_* and v_* are not
 *  read by mte_kv8_attention. out's rows and heads must not overlap. out may be q (the same
 *  address and strides: every row is read before it is written), else it overlaps no input. */
typedef struct {
  int32_t n_q_heads, n_kv_heads, head_dim;
  int32_t dtype;
  float scale;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
} mte_attn_shape;

/* Cross attention of packed sequences. For query i of sequence b, head h:
 *   out[i, h] = sum_j softmax_j(scale q[i, h] . k[j, g]) v[j, g],  g = h / (Hq/Hkv),
 * j over the tokens of key/value sequence kv_index[b] whose key_mask is not 0. A
 * query with no such token (an empty sequence, or all masked, or all scores -inf) gets zeros.
 * What a masked token's k and v hold (infinities, NaN) does not reach the output.
 * Sums are of p up to 2^8: values beyond 2^100 may end as infinities.
 *  q, out:   device, sum(q_lens) rows, sequences back to back in q_lens order.
 *  k, v:     device, sum(kv_lens) rows, back to back in kv_lens order.
 *  key_mask: device uint8[sum(kv_lens)], or NULL (all tokens count).
 *  q_lens:   HOST int32[n_q], each >= 0; kv_lens: HOST int32[n_kv], each >= 0; n_q and n_kv at least 1.
 *  kv_index: HOST int32[n_q], the kv sequence of each query sequence (several may
 *            name the same one: one frame's conditioning for all); NULL: b
 *            itself, n_q == n_kv.
 *  workspace: device, at least mte_cross_attention_workspace(...) bytes, aligned to
 *            16; NULL where that is 0.
 * head_dim: a multiple of 8, at most 128. The result does not depend on what else
 * runs. Which kernel takes the rows and how a long key range is split goes by the
 * whole call, so that other sequences may change the last bits of a result.
 * Errors: MTE_E_INVALID (null, negative length, bad index, heads, dtype, scale,
 * strides or alignment, a sum of kv_lens, or of q_lens times heads, beyond 2^31 - 4097), MTE_E_UNSUPPORTED
 * (head_dim), MTE_E_CAPACITY (workspace_bytes), MTE_E_HIP. No query rows at all
 * is MTE_OK and enqueues nothing (then q and out may be NULL, and k and v where
 * there are no key rows). */
int mte_cross_attention(const mte_attn_shape *shape, const void *q, const void *k, const void *v,
                        const uint8_t *key_mask, const int32_t *q_lens, int32_t n_q, const int32_t *kv_lens,
                        int32_t n_kv, const int32_t *kv_index, void *out, void *workspace,
                        int64_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace that such a call needs (0: none; host only, no HIP call), or a
 * negative mte_status. */
int64_t mte_cross_attention_workspace(const mte_attn_shape *shape, const int32_t *q_lens, int32_t n_q,
                                      const int32_t *kv_lens, int32_t n_kv, const int32_t *kv_index);

/* A key/value cache in 8 bits: n_blocks blocks of MTE_KV8_BLOCK tokens, each
 * holding all kv heads. Values are OCP e4m3 codes (as in mte_quantize_e4m3_rows)
 * times one power of two for each block, kv head and tensor. Device memory of the
 * caller, aligned to 16 bytes, of which only blocks that were appended to are read:
 *  k_codes uint8 [n_blocks][Hkv][d / 16][32 tokens][16]
 *  v_codes uint8 [n_blocks][Hkv][d][32], token 16 t + 8 a + 4 h + i (t, a, h < 2, i < 4)
 *          of the block at position 16 h + 8 t + 4 a + i
 *  scales  float [n_blocks][Hkv][2] (key, value); a program that fills blocks itself may use
 *          any normal positive ones, but mte_kv8_append continues only blocks with powers of two
 * (the orders in which the matrix cores take them: a wave's 64 lanes load 1 KB
 * of consecutive codes at a time.) head_dim: 64 or 128.
 *
 * A sequence is a row of block numbers, table[i * table_row + j] (device int32, the
 * block of its tokens 32 j .. 32 j + 31; table_width of them), and a length
 * kv_lens[i] (device int32, so that a captured step can be replayed as the
 * sequence grows). Blocks may appear in several rows (a shared prefix, one
 * frame's conditioning for all) as long as no call appends to a block that
 * another of its sequences appends to or reads, or that the same row names twice. Device values are checked on the
 * device: a length below 0 counts as 0, one beyond 32 table_width as that (attention; append
 * and read: see there), and a block number outside [0, n_blocks) as a block whose
 * tokens are all masked (read: zeros; append: not written). table_width is at most
 * 2^26 - 1. */
#define MTE_KV8_BLOCK 32
typedef struct {
  uint8_t *k_codes, *v_codes;
  float *scales;
  int32_t n_blocks, n_kv_heads, head_dim;
} mte_kv8;

/* Stores the newest new_lens[i] tokens of each sequence: rows of k and v (device,
 * dtype, packed back to back, strides as in mte_attn_shape) become its tokens
 * kv_lens[i] - new_lens[i] .. kv_lens[i] - 1 (kv_lens: the length after the append;
 * a sequence whose length is below new_lens[i], or beyond its table, is not
 * written).
 * The scale of a block and head is 2^e, e >= -126 the smallest integer with
 * max |x| <= 448 * 2^e over the block's new tokens (-126 if they are all zero); where
 * the block holds older tokens, at least its old scale, and if it grows their
 * codes are rounded again to the new one (exact but for codes that become
 * subnormal, which move by at most 2^-10 of the new scale). Code: nearest to x / 2^e,
 * ties to the even one; NaN stays NaN; at the largest scale, 2^120, magnitudes end at
 * 240 * 2^120 (infinities become that), so that every stored value is finite in fp32. Places of a touched block past the length are set to zero.
 * new_lens: HOST int32[n], each >= 0; n >= 1. Errors: MTE_E_INVALID, MTE_E_UNSUPPORTED
 * (head_dim), MTE_E_HIP. */
int mte_kv8_append(const mte_kv8 *cache, const int32_t *table, int32_t table_width, int64_t table_row,
                   const int32_t *kv_lens, const void *k, int64_t k_row, int64_t k_head, const void *v,
                   int64_t v_row, int64_t v_head, int32_t dtype, const int32_t *new_lens, int32_t n,
                   hipStream_t stream);

/* The newest counts[i] tokens of each sequence as rows: k and v (device, dtype,
 * contiguous [sum(counts), Hkv, d], aligned to 16 bytes) receive code * scale (exact,
 * but for bf16 magnitudes below 2^-126: they are rounded to its multiples of 2^-133) of tokens kv_lens[i] - counts[i] .. kv_lens[i] - 1, packed back to
 * back (rows of tokens before the first or beyond the table: zeros). counts: HOST
 * int32[n], each >= 0; n >= 1. Errors as mte_kv8_append. */
int mte_kv8_read(const mte_kv8 *cache, const int32_t *table, int32_t table_width, int64_t table_row,
                 const int32_t *kv_lens, const int32_t *counts, int32_t n, void *k, void *v, int32_t dtype,
                 hipStream_t stream);

/* Attention of packed queries over cached sequences: sequence i's q_lens[i] queries
 * attend to its kv_lens[i] cached tokens; with causal = 1 its query u sees tokens
 * 0 .. kv_lens[i] - q_lens[i] + u only (its own token last: append, then attend).
 * A query that sees nothing gets zeros. Formula, q, out and workspace as in
 * mte_cross_attention (workspace: mte_kv8_attention_workspace); q_lens: HOST int32[n], n >= 1.
 * Rounding: a token's weight, its probability times the scale of its block's values, meets the codes with 11
 * significant bits (MTE_F32: 22), and none below 2^-31 of the largest weight of its row; whatever
 * scales the blocks of lesser weight have. What tokens that a query does not see hold does not reach it; a
 * cached NaN reaches the queries that see its token: a value in its channel, a key everywhere.
 * The work is split for sequences of up to 32 table_width tokens: a table that
 * is much wider than its sequences costs time.
 * Errors: MTE_E_INVALID, MTE_E_UNSUPPORTED (head_dim), MTE_E_CAPACITY
 * (workspace_bytes), MTE_E_HIP, sizes as in mte_cross_attention. */
int mte_kv8_attention(const mte_attn_shape *shape, const mte_kv8 *cache, const int32_t *table,
                      int32_t table_width, int64_t table_row, const int32_t *kv_lens, const void *q,
                      const int32_t *q_lens, int32_t n, int32_t causal, void *out, void *workspace,
                      int64_t workspace_bytes, hipStream_t stream);

int64_t mte_kv8_attention_workspace(const mte_attn_shape *shape, const int32_t *q_lens, int32_t n,
                                    int32_t table_width);

/* Group norm with an activation on channels-last rows:
 *   y = act((x - mean) / sqrt(var + eps) * gamma[c] + beta[c]),
 * mean and biased variance over the pixels and the C / groups channels of a group of
 * one image (fp32: per part the mean, then the squares around it, parts joined by
 * their counts). act: MTE_ACT_NONE, or MTE_ACT_SILU z / (1 + exp(-z)).
 *  x: device, dtype, n images of `pixels` rows of `channels` elements; x_row
 *     elements from one pixel to the next, x_image from one image to the next
 *     (>= 0; rows of a wider buffer may be normalised in place of a copy). y alike;
 *     y may be x (same strides), else they must not overlap.
 *  gamma, beta: device, dtype, [channels], or NULL (1 / 0).
 *  groups divides channels; n and groups are at most 65535. eps >= 0 and finite.
 *  workspace: device, at least mte_group_norm_workspace(...) bytes, aligned to 16; NULL
 *     where that is 0.
 * Buffers need only be aligned like one element (16 bytes and strides that are
 * multiples of 8 elements are faster). Errors: MTE_E_INVALID, MTE_E_CAPACITY
 * (workspace_bytes), MTE_E_HIP. n == 0 or pixels == 0 is MTE_OK. */
typedef enum { MTE_ACT_NONE = 0, MTE_ACT_SILU = 1 } mte_activation;
int mte_group_norm(const void *x, int64_t x_row, int64_t x_image, int32_t n, int32_t pixels, int32_t channels,
                   int32_t groups, const void *gamma, const void *beta, float eps, int32_t act, int32_t dtype,
                   void *y, int64_t y_row, int64_t y_image, void *workspace, int64_t workspace_bytes,
                   hipStream_t stream);
int64_t mte_group_norm_workspace(int32_t n, int32_t pixels, int32_t channels, int32_t groups, int32_t dtype);

#ifdef __cplusplus
}
#endif

#endif /* MTE_COND_H */
