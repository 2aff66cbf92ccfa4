// C ABI of the operators between hidden states and attention (include/mte_proj.h): argument
// checks, all on the host before any HIP call, and the hand-over to the launchers.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/mte_proj.h"
#include "proj_launch.h"

using namespace mte;

namespace {

constexpr int64_t kMaxRows = 0x7FFFFFFF - 4096;      // a last tile's end stays inside 31 bits
constexpr int64_t kMaxStride = (int64_t)1 << 40;     // row * stride stays inside 64 bits
constexpr int32_t kMaxHeads = 65535;

bool aligned(const void *p, uintptr_t n) { return (uintptr_t)p % n == 0; }
bool type_ok(int32_t t) { return t == MTE_F32 || t == MTE_BF16; }
uintptr_t size_of(int32_t t) { return t == MTE_BF16 ? 2 : 4; }
bool stride_ok(int64_t s) { return s >= 0 && s <= kMaxStride && s % 8 == 0; }
int hip(hipError_t e) { return e == hipSuccess ? MTE_OK : MTE_E_HIP; }

int linear_status(int32_t x_type, int32_t m, int32_t k, int32_t n) {
  if (x_type != MTE_I8_CODES && !type_ok(x_type)) return MTE_E_INVALID;
  if (m < 0 || m > kMaxRows || n <= 0 || n > kMaxRows || k <= 0 || k > MTE_I8_COLS) return MTE_E_INVALID;
  return MTE_OK;
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

}  // extern "C"
