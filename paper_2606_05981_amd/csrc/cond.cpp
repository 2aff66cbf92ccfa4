// C ABI of the operators that read the conditioning (include/mte_cond.h):
// argument checks, all on the host before any HIP call, and the hand-over to the launchers.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/mte_cond.h"
#include "cond_checks.h"

using namespace mte;

namespace {

// MTE_OK, 1 (nothing to do) or an error, for everything of a cross attention but its buffers.
int cross_status(const mte_attn_shape *s, const int32_t *q_lens, int32_t n_q, const int32_t *kv_lens, int32_t n_kv,
                 const int32_t *kv_index, int64_t *q_rows, int64_t *kv_rows) {
  int st = shape_status(s, rows_dim);
  if (st != MTE_OK) return st;
  if (!stride_ok(s->k_row) || !stride_ok(s->k_head) || !stride_ok(s->v_row) || !stride_ok(s->v_head))
    return MTE_E_INVALID;
  *q_rows = query_rows(*s, q_lens, n_q);
  if (*q_rows < 0) return (int)*q_rows;
  if (!kv_lens || n_kv <= 0) return MTE_E_INVALID;
  *kv_rows = total(kv_lens, n_kv);
  if (*kv_rows < 0) return MTE_E_INVALID;
  if (!kv_index && n_q != n_kv) return MTE_E_INVALID;
  if (kv_index)
    for (int32_t i = 0; i < n_q; ++i)
      if (kv_index[i] < 0 || kv_index[i] >= n_kv) return MTE_E_INVALID;
  return MTE_OK;
}

int cache_status(const mte_kv8 *c) {
  if (!c || !c->k_codes || !c->v_codes || !c->scales) return MTE_E_INVALID;
  if (c->n_blocks <= 0 || c->n_kv_heads <= 0 || c->n_kv_heads > kMaxGrid || c->head_dim <= 0) return MTE_E_INVALID;
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes) || !aligned16(c->scales)) return MTE_E_INVALID;
  if (!codes_dim(c->head_dim)) return MTE_E_UNSUPPORTED;
  return MTE_OK;
}

int table_status(const int32_t *table, int32_t width, int64_t row, const int32_t *kv_lens) {
  if (!table || !kv_lens || width <= 0 || width > kMaxWidth || row < 0 || row > kMaxStride) return MTE_E_INVALID;
  return MTE_OK;
}

Kv8View view(const mte_kv8 &c, const int32_t *table, int32_t width, int64_t row, const int32_t *kv_lens) {
  return Kv8View{c.k_codes, c.v_codes, c.scales, table, kv_lens, row, width, c.n_blocks, c.n_kv_heads, c.head_dim};
}

int hip(hipError_t e) { return e == hipSuccess ? MTE_OK : MTE_E_HIP; }

}  // namespace

extern "C" {

int64_t mte_cross_attention_workspace(const mte_attn_shape *shape, const int32_t *q_lens, int32_t n_q,
                                      const int32_t *kv_lens, int32_t n_kv, const int32_t *kv_index) {
  int64_t nq, nk;
  const int st = cross_status(shape, q_lens, n_q, kv_lens, n_kv, kv_index, &nq, &nk);
  if (st != MTE_OK) return st;
  return cross_workspace(problem(*shape, q_lens, n_q), kv_lens, n_kv, kv_index);
}

int mte_cross_attention(const mte_attn_shape *shape, const void *q, const void *k, const void *v,
                        const uint8_t *key_mask, const int32_t *q_lens, int32_t n_q, const int32_t *kv_lens,
                        int32_t n_kv, const int32_t *kv_index, void *out, void *workspace, int64_t workspace_bytes,
                        hipStream_t stream) {
  int64_t nq, nk;
  const int st = cross_status(shape, q_lens, n_q, kv_lens, n_kv, kv_index, &nq, &nk);
  if (st != MTE_OK) return st;
  if (nq == 0) return MTE_OK;
  if (!q || !out || !aligned16(q) || !aligned16(out)) return MTE_E_INVALID;
  if (nk > 0 && (!k || !v || !aligned16(k) || !aligned16(v))) return MTE_E_INVALID;
  AttnProblem p = problem(*shape, q_lens, n_q);
  const int64_t need = cross_workspace(p, kv_lens, n_kv, kv_index);
  if (workspace_bytes < need) return MTE_E_CAPACITY;
  if (need > 0 && (!workspace || !aligned16(workspace))) return MTE_E_INVALID;
  p.c.q = q;
  p.c.out = out;
  p.c.ws = (float *)workspace;
  return hip(launch_cross(p, k, v, key_mask, shape->k_row, shape->k_head, shape->v_row, shape->v_head, kv_lens, n_kv,
                          kv_index, stream));
}

int mte_kv8_append(const mte_kv8 *cache, const int32_t *table, int32_t table_width, int64_t table_row,
                   const int32_t *kv_lens, const void *k, int64_t k_row, int64_t k_head, const void *v, int64_t v_row,
                   int64_t v_head, int32_t dtype, const int32_t *new_lens, int32_t n, hipStream_t stream) {
  int st = cache_status(cache);
  if (st != MTE_OK) return st;
  if ((st = table_status(table, table_width, table_row, kv_lens)) != MTE_OK) return st;
  if (dtype != MTE_F32 && dtype != MTE_BF16) return MTE_E_INVALID;
  if (!new_lens || n <= 0) return MTE_E_INVALID;
  const int64_t rows = total(new_lens, n);
  if (rows < 0 || !stride_ok(k_row) || !stride_ok(k_head) || !stride_ok(v_row) || !stride_ok(v_head))
    return MTE_E_INVALID;
  if (rows == 0) return MTE_OK;
  if (!k || !v || !aligned16(k) || !aligned16(v)) return MTE_E_INVALID;
  return hip(launch_kv8_append(view(*cache, table, table_width, table_row, kv_lens), k, k_row, k_head, v, v_row,
                               v_head, dtype, new_lens, n, stream));
}

int mte_kv8_read(const mte_kv8 *cache, const int32_t *table, int32_t table_width, int64_t table_row,
                 const int32_t *kv_lens, const int32_t *counts, int32_t n, void *k, void *v, int32_t dtype,
                 hipStream_t stream) {
  int st = cache_status(cache);
  if (st != MTE_OK) return st;
  if ((st = table_status(table, table_width, table_row, kv_lens)) != MTE_OK) return st;
  if (dtype != MTE_F32 && dtype != MTE_BF16) return MTE_E_INVALID;
  if (!counts || n <= 0) return MTE_E_INVALID;
  const int64_t rows = total(counts, n);
  if (rows < 0) return MTE_E_INVALID;
  if (rows == 0) return MTE_OK;
  if (!k || !v || !aligned16(k) || !aligned16(v)) return MTE_E_INVALID;
  return hip(launch_kv8_read(view(*cache, table, table_width, table_row, kv_lens), counts, n, k, v, dtype, stream));
}

int64_t mte_kv8_attention_workspace(const mte_attn_shape *shape, const int32_t *q_lens, int32_t n,
                                    int32_t table_width) {
  const int st = shape_status(shape, codes_dim);
  if (st != MTE_OK) return st;
  const int64_t rows = query_rows(*shape, q_lens, n);
  if (rows < 0) return rows;
  if (table_width <= 0 || table_width > kMaxWidth) return MTE_E_INVALID;
  return kv8_workspace(problem(*shape, q_lens, n), table_width);
}

int mte_kv8_attention(const mte_attn_shape *shape, const mte_kv8 *cache, const int32_t *table, int32_t table_width,
                      int64_t table_row, const int32_t *kv_lens, const void *q, const int32_t *q_lens, int32_t n,
                      int32_t causal, void *out, void *workspace, int64_t workspace_bytes, hipStream_t stream) {
  int st = shape_status(shape, codes_dim);
  if (st != MTE_OK) return st;
  const int64_t rows = query_rows(*shape, q_lens, n);
  if (rows < 0) return (int)rows;
  if ((st = cache_status(cache)) != MTE_OK) return st;
  if ((st = table_status(table, table_width, table_row, kv_lens)) != MTE_OK) return st;
  if (cache->n_kv_heads != shape->n_kv_heads || cache->head_dim != shape->head_dim) return MTE_E_INVALID;
  if (causal != 0 && causal != 1) return MTE_E_INVALID;
  if (rows == 0) return MTE_OK;
  if (!q || !out || !aligned16(q) || !aligned16(out)) return MTE_E_INVALID;
  AttnProblem p = problem(*shape, q_lens, n);
  const int64_t need = kv8_workspace(p, table_width);
  if (workspace_bytes < need) return MTE_E_CAPACITY;
  if (need > 0 && (!workspace || !aligned16(workspace))) return MTE_E_INVALID;
  p.c.q = q;
  p.c.out = out;
  p.c.ws = (float *)workspace;
  return hip(launch_kv8_attention(p, view(*cache, table, table_width, table_row, kv_lens), causal, stream));
}

// Sizes of a group norm: MTE_OK or MTE_E_INVALID.
static int norm_status(int32_t n, int32_t pixels, int32_t channels, int32_t groups, int32_t dtype) {
  if (n < 0 || n > kMaxGrid || pixels < 0 || channels <= 0 || groups <= 0 || groups > kMaxGrid || channels % groups)
    return MTE_E_INVALID;
  return dtype == MTE_F32 || dtype == MTE_BF16 ? MTE_OK : MTE_E_INVALID;
}

int64_t mte_group_norm_workspace(int32_t n, int32_t pixels, int32_t channels, int32_t groups, int32_t dtype) {
  const int st = norm_status(n, pixels, channels, groups, dtype);
  if (st != MTE_OK) return st;
  return n == 0 || pixels == 0 ? 0 : group_norm_workspace(n, pixels, channels, groups, dtype);
}

int mte_group_norm(const void *x, int64_t x_row, int64_t x_image, int32_t n, int32_t pixels, int32_t channels,
                   int32_t groups, const void *gamma, const void *beta, float eps, int32_t act, int32_t dtype, void *y,
                   int64_t y_row, int64_t y_image, void *workspace, int64_t workspace_bytes, hipStream_t stream) {
  const int st = norm_status(n, pixels, channels, groups, dtype);
  if (st != MTE_OK) return st;
  if (!(eps >= 0.f) || !std::isfinite(eps) || (act != MTE_ACT_NONE && act != MTE_ACT_SILU)) return MTE_E_INVALID;
  if (x_row < 0 || x_image < 0 || y_row < 0 || y_image < 0 || x_row > kMaxStride || x_image > kMaxStride ||
      y_row > kMaxStride || y_image > kMaxStride)
    return MTE_E_INVALID;
  if (n == 0 || pixels == 0) return MTE_OK;
  const uintptr_t es = dtype == MTE_BF16 ? 2 : 4;
  if (!x || !y || (uintptr_t)x % es || (uintptr_t)y % es || (uintptr_t)gamma % es || (uintptr_t)beta % es)
    return MTE_E_INVALID;
  const int64_t need = group_norm_workspace(n, pixels, channels, groups, dtype);
  if (workspace_bytes < need) return MTE_E_CAPACITY;
  if (need > 0 && (!workspace || !aligned16(workspace))) return MTE_E_INVALID;
  GroupNormArgs a{x, gamma, beta, y, (float *)workspace, x_row, x_image, y_row, y_image, n, pixels, channels, groups,
                  act, eps};
  return hip(launch_group_norm(a, dtype, stream));
}

}  // extern "C"
