// C ABI of the operators between hidden states and attention (include/mte_proj.h): argument
// checks, all on the host before any HIP call, and the hand-over to the launchers.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/mte_proj.h"
#include "cond_checks.h"
#include "proj_launch.h"

using namespace mte;

namespace {

constexpr int32_t kMaxHeads = 65535;

bool aligned(const void *p, uintptr_t n) { return (uintptr_t)p % n == 0; }
bool type_ok(int32_t t) { return t == MTE_F32 || t == MTE_BF16; }
uintptr_t size_of(int32_t t) { return t == MTE_BF16 ? 2 : 4; }
int hip(hipError_t e) { return e == hipSuccess ? MTE_OK : MTE_E_HIP; }

int linear_status(int32_t x_type, int32_t m, int32_t k, int32_t n) {
  if (x_type != MTE_I8_CODES && !type_ok(x_type)) return MTE_E_INVALID;
  if (m < 0 || m > kMaxRows || n <= 0 || n > kMaxRows || k <= 0 || k > MTE_I8_COLS) return MTE_E_INVALID;
  return MTE_OK;
}

// MTE_OK or an error for everything of a prefix attention but its buffers and the prefix's strides.
int prefix_status(const mte_attn_shape *s, int32_t prefix_len, const int32_t *q_lens, const int32_t *kv_lens, int32_t n,
                  int64_t *q_rows, int64_t *kv_rows) {
  const int st = shape_status(s, rows_dim);
  if (st != MTE_OK) return st;
  if (!stride_ok(s->k_row) || !stride_ok(s->k_head) || !stride_ok(s->v_row) || !stride_ok(s->v_head))
    return MTE_E_INVALID;
  *q_rows = query_rows(*s, q_lens, n);
  if (*q_rows < 0) return (int)*q_rows;
  if (!kv_lens || prefix_len < 0) return MTE_E_INVALID;
  *kv_rows = total(kv_lens, n);
  return *kv_rows < 0 || *kv_rows + prefix_len > kMaxRows ? MTE_E_INVALID : MTE_OK;
}

}  // namespace

extern "C" {

int64_t mte_i8_pitch(int32_t cols) {
  return cols <= 0 || cols > MTE_I8_COLS ? (int64_t)MTE_E_INVALID : i8_pitch(cols);
}

int mte_i8_quantize_rows(const void *x, int64_t x_row, int32_t rows, int32_t cols, int32_t dtype, int8_t *codes,
                         float *scales, hipStream_t stream) {
  if (!type_ok(dtype) || rows < 0 || rows > kMaxRows || cols <= 0 || cols > MTE_I8_COLS || x_row < 0 || x_row > kMaxStride)
    return MTE_E_INVALID;
  if (rows == 0) return MTE_OK;
  if (!x || !codes || !scales || !aligned(x, size_of(dtype)) || !aligned(codes, 16) || !aligned(scales, 4))
    return MTE_E_INVALID;
  return hip(launch_i8_quantize(QuantArgs{x, codes, scales, x_row, rows, cols, (int)i8_pitch(cols)}, dtype, stream));
}

int64_t mte_i8_linear_workspace(int32_t x_type, int32_t m, int32_t k, int32_t n) {
  const int st = linear_status(x_type, m, k, n);
  return st != MTE_OK ? st : m == 0 ? 0 : i8_workspace(x_type, m, n, k);
}

int mte_i8_linear(const void *x, int64_t x_row, const float *x_scales, int32_t x_type, int32_t m, int32_t k,
                  const int8_t *w, const float *w_scales, int32_t n, const void *bias, int32_t act, void *out,
                  int64_t out_row, int32_t dtype, void *workspace, int64_t workspace_bytes, hipStream_t stream) {
  const int st = linear_status(x_type, m, k, n);
  if (st != MTE_OK) return st;
  if (!type_ok(dtype) || (act != MTE_ACT_NONE && act != MTE_ACT_SILU)) return MTE_E_INVALID;
  const bool codes = x_type == MTE_I8_CODES;
  if (!codes && (x_row < 0 || x_row > kMaxStride)) return MTE_E_INVALID;
  if (m > 1 && (out_row < n || out_row > kMaxStride)) return MTE_E_INVALID;
  if (m == 0) return MTE_OK;
  if (!x || !w || !w_scales || !out || !aligned(w, 16) || !aligned(w_scales, 4)) return MTE_E_INVALID;
  if (!aligned(out, size_of(dtype)) || !aligned(bias, size_of(dtype))) return MTE_E_INVALID;
  if (codes ? !x_scales || !aligned(x, 16) || !aligned(x_scales, 4) : !aligned(x, size_of(x_type))) return MTE_E_INVALID;
  const int64_t need = i8_workspace(x_type, m, n, k);
  if (workspace_bytes < need) return MTE_E_CAPACITY;
  if (need > 0 && (!workspace || !aligned(workspace, 16))) return MTE_E_INVALID;
  I8Args a{};
  a.b = w;
  a.sb = w_scales;
  a.bias = bias;
  a.out = out;
  a.x_row = m > 1 ? x_row : 0;
  a.out_row = m > 1 ? out_row : 0;
  a.m = m;
  a.n = n;
  a.k = k;
  a.pitch = (int)i8_pitch(k);
  a.act = act;
  if (codes) {
    a.a = (const int8_t *)x;
    a.sa = x_scales;
  } else {
    a.x = x;
  }
  return hip(launch_i8_linear(a, x_type, dtype, workspace, stream));
}

int mte_rotary(const mte_rotary_shape *s, const void *q, const void *k, const int32_t *positions, int64_t axis_stride,
               const double *freq, int32_t tokens, void *q_out, void *k_out, hipStream_t stream) {
  if (!s || s->n_q_heads <= 0 || s->n_k_heads < 0 || s->head_dim <= 0 || s->rot_dim <= 0 || s->rot_dim % 2 ||
      s->rot_dim > s->head_dim || !type_ok(s->dtype) || s->interleaved < 0 || s->interleaved > 1 || s->inverse < 0 ||
      s->inverse > 1 || s->n_axes < 1 || s->n_axes > 4 || !std::isfinite(s->factor) || tokens < 0)
    return MTE_E_INVALID;
  if (s->head_dim % 8 || s->head_dim > 512) return MTE_E_UNSUPPORTED;
  if (s->n_q_heads > kMaxHeads || s->n_k_heads > kMaxHeads ||
      (int64_t)tokens * ((int64_t)s->n_q_heads + s->n_k_heads) > kMaxRows)
    return MTE_E_INVALID;
  for (const int64_t x : {s->q_row, s->q_head, s->qo_row, s->qo_head})
    if (!stride_ok(x)) return MTE_E_INVALID;
  for (const int64_t x : {s->k_row, s->k_head, s->ko_row, s->ko_head})
    if (s->n_k_heads > 0 && !stride_ok(x)) return MTE_E_INVALID;
  RotaryArgs a{};
  int64_t at = 0;
  for (int i = 0; i < 4; ++i) {
    if (i < s->n_axes) {
      const int64_t sec = s->n_axes == 1 ? s->rot_dim / 2 : s->section[i];
      if (sec < 0) return MTE_E_INVALID;
      at += sec;
    }
    a.end[i] = (int)(at < s->rot_dim ? at : s->rot_dim);
  }
  if (at != s->rot_dim / 2) return MTE_E_INVALID;
  if (s->n_axes > 1 && (axis_stride < 0 || axis_stride > kMaxStride)) return MTE_E_INVALID;
  if (tokens == 0) return MTE_OK;
  if (!q || !q_out || !positions || !freq || !aligned(q, 16) || !aligned(q_out, 16) || !aligned(positions, 4) ||
      !aligned(freq, 8))
    return MTE_E_INVALID;
  if (s->n_k_heads > 0 && (!k || !k_out || !aligned(k, 16) || !aligned(k_out, 16))) return MTE_E_INVALID;
  // in place: the same rows
  if (q == q_out && (s->q_row != s->qo_row || s->q_head != s->qo_head)) return MTE_E_INVALID;
  if (s->n_k_heads > 0 && k == k_out && (s->k_row != s->ko_row || s->k_head != s->ko_head)) return MTE_E_INVALID;
  a.q = q;
  a.k = k;
  a.qo = q_out;
  a.ko = k_out;
  a.pos = positions;
  a.freq = freq;
  a.axis_stride = s->n_axes > 1 ? axis_stride : 0;
  a.q_row = s->q_row;
  a.q_head = s->q_head;
  a.k_row = s->k_row;
  a.k_head = s->k_head;
  a.qo_row = s->qo_row;
  a.qo_head = s->qo_head;
  a.ko_row = s->ko_row;
  a.ko_head = s->ko_head;
  a.hq = s->n_q_heads;
  a.hk = s->n_k_heads;
  a.d = s->head_dim;
  a.rot = s->rot_dim;
  a.tokens = tokens;
  a.inter = s->interleaved;
  a.factor = s->factor;
  a.sign = s->inverse ? -1.f : 1.f;
  a.q_tail = q != q_out && s->rot_dim < s->head_dim;
  a.k_tail = s->n_k_heads > 0 && k != k_out && s->rot_dim < s->head_dim;
  return hip(launch_rotary(a, s->dtype, stream));
}

int64_t mte_prefix_attention_workspace(const mte_attn_shape *shape, int32_t prefix_len, const int32_t *q_lens,
                                       const int32_t *kv_lens, int32_t n) {
  int64_t nq, nk;
  const int st = prefix_status(shape, prefix_len, q_lens, kv_lens, n, &nq, &nk);
  return st != MTE_OK ? (int64_t)st : prefix_workspace(problem(*shape, q_lens, n), prefix_len, kv_lens);
}

int mte_prefix_attention(const mte_attn_shape *shape, const void *q, const void *prefix_k, const void *prefix_v,
                         int64_t pk_row, int64_t pk_head, int64_t pv_row, int64_t pv_head, int32_t prefix_len,
                         const void *k, const void *v, const int32_t *q_lens, const int32_t *kv_lens, int32_t n,
                         int32_t causal, void *out, void *workspace, int64_t workspace_bytes, hipStream_t stream) {
  int64_t nq, nk;
  const int st = prefix_status(shape, prefix_len, q_lens, kv_lens, n, &nq, &nk);
  if (st != MTE_OK) return st;
  if (causal != 0 && causal != 1) return MTE_E_INVALID;
  if (!stride_ok(pk_row) || !stride_ok(pk_head) || !stride_ok(pv_row) || !stride_ok(pv_head)) return MTE_E_INVALID;
  if (nq == 0) return MTE_OK;
  if (!q || !out || !aligned16(q) || !aligned16(out)) return MTE_E_INVALID;
  if (prefix_len > 0 && (!prefix_k || !prefix_v || !aligned16(prefix_k) || !aligned16(prefix_v))) return MTE_E_INVALID;
  if (nk > 0 && (!k || !v || !aligned16(k) || !aligned16(v))) return MTE_E_INVALID;
  AttnProblem p = problem(*shape, q_lens, n);
  p.near_rows = p.near_rows && pk_row < (1 << 24) && pv_row < (1 << 24);
  const int64_t need = prefix_workspace(p, prefix_len, kv_lens);
  if (workspace_bytes < need) return MTE_E_CAPACITY;
  if (need > 0 && (!workspace || !aligned16(workspace))) return MTE_E_INVALID;
  p.c.q = q;
  p.c.out = out;
  p.c.ws = (float *)workspace;
  const PrefixRows x{prefix_k, prefix_v, k, v, pk_row, pk_head, pv_row, pv_head,
                     shape->k_row, shape->k_head, shape->v_row, shape->v_head, prefix_len};
  return hip(launch_prefix(p, x, kv_lens, causal, stream));
}

}  // extern "C"
