// Argument checks that the entry points of attention share (host).
#pragma once

#include <cmath>
#include <cstdint>

#include "../../include/mte_cond.h"
#include "cond_launch.h"

namespace mte {

constexpr int64_t kMaxRows = 0x7FFFFFFF - 4096;      // a last tile's end, up to 4096 rows on, stays inside 31 bits
constexpr int64_t kMaxStride = (int64_t)1 << 40;     // row * stride stays inside 64 bits
constexpr int32_t kMaxWidth = (1 << 26) - 1;         // 32 * table_width stays inside 31 bits
constexpr int32_t kMaxGrid = 65535;
constexpr float kLog2e = 1.4426950408889634f;

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
inline bool stride_ok(int64_t s) { return s >= 0 && s <= kMaxStride && s % 8 == 0; }

// Sum of n host lengths, or -1 where one is negative or the sum too large.
inline int64_t total(const int32_t *lens, int32_t n) {
  int64_t t = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (lens[i] < 0) return -1;
    t += lens[i];
    if (t > kMaxRows) return -1;
  }
  return t;
}

inline bool rows_dim(int32_t d) { return d % 8 == 0 && d <= 128; }
inline bool codes_dim(int32_t d) { return d == 64 || d == 128; }

inline int shape_status(const mte_attn_shape *s, bool (*built)(int32_t)) {
  if (!s) return MTE_E_INVALID;
  if (s->n_q_heads <= 0 || s->n_kv_heads <= 0 || s->head_dim <= 0 || s->n_q_heads % s->n_kv_heads) return MTE_E_INVALID;
  if (s->n_kv_heads > kMaxGrid) return MTE_E_INVALID;
  if (s->dtype != MTE_F32 && s->dtype != MTE_BF16) return MTE_E_INVALID;
  if (!(s->scale > 0.f) || !std::isfinite(s->scale * kLog2e)) return MTE_E_INVALID;
  if (!built(s->head_dim)) return MTE_E_UNSUPPORTED;
  if (!stride_ok(s->q_row) || !stride_ok(s->q_head) || !stride_ok(s->o_row) || !stride_ok(s->o_head))
    return MTE_E_INVALID;
  return MTE_OK;
}

// Query lengths: their sum, or a negative status. Matrix rows (token, head) are counted in 31 bits.
inline int64_t query_rows(const mte_attn_shape &s, const int32_t *q_lens, int32_t n) {
  if (!q_lens || n <= 0) return MTE_E_INVALID;
  const int64_t t = total(q_lens, n);
  return t < 0 || t * s.n_q_heads > kMaxRows ? (int64_t)MTE_E_INVALID : t;
}

inline AttnProblem problem(const mte_attn_shape &s, const int32_t *q_lens, int32_t n) {
  AttnProblem p;
  p.c.q = nullptr;
  p.c.out = nullptr;
  p.c.ws = nullptr;
  p.c.q_row = s.q_row;
  p.c.q_head = s.q_head;
  p.c.o_row = s.o_row;
  p.c.o_head = s.o_head;
  p.c.sc = s.scale * kLog2e;
  p.c.d = s.head_dim;
  p.c.hkv = s.n_kv_heads;
  p.c.rep = s.n_q_heads / s.n_kv_heads;
  p.c.n_seq = 0;
  p.c.n_split = 1;
  p.c.ws_rows = 0;
  p.c.ws_ml = 0;
  p.c.big = 0;
  p.c.first = 0;
  p.dtype = s.dtype;
  p.near_rows = s.k_row < (1 << 24) && s.v_row < (1 << 24);
  // 31 rows and rep heads: 2^29 + 2^30 elements; rep: what the tiles divide by in fp32 (exact below 2^22)
  const auto near = [&](int64_t row, int64_t head) {
    return p.c.rep <= (1 << 16) && row < (1 << 24) && head < ((int64_t)1 << 30) && (p.c.rep - 1) * head < ((int64_t)1 << 30);
  };
  p.near_tiles = near(s.q_row, s.q_head) && near(s.o_row, s.o_head);
  p.q_lens = q_lens;
  p.n = n;
  return p;
}

}  // namespace mte
