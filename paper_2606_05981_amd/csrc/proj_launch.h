// Host-side launchers of the operators between hidden states and attention (internal to libmte).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/mte_proj.h"
#include "cond_launch.h"

namespace mte {

constexpr int kI8Pitch = 128;        // a row of codes is a multiple of it
inline int64_t i8_pitch(int32_t cols) { return ((int64_t)cols + kI8Pitch - 1) / kI8Pitch * kI8Pitch; }

struct QuantArgs {
  const void *x;
  int8_t *codes;
  float *scales;
  int64_t x_row;
  int rows, cols, pitch;
};
hipError_t launch_i8_quantize(const QuantArgs &a, int dtype, hipStream_t s);

struct I8Args {
  const void *x;                     // rows to quantise, or null
  const int8_t *a, *b;               // codes [m][pitch], [n][pitch] (x: the workspace)
  const float *sa, *sb;
  const void *bias;
  void *out;
  int64_t x_row, out_row;
  int m, n, k, pitch, act;
  int gm, gn, gh;                    // tiles of the launch and their order (GemmArgs)
};
int64_t i8_workspace(int x_type, int m, int n, int k);
hipError_t launch_i8_linear(I8Args a, int x_type, int dtype, void *ws, hipStream_t s);

struct RotaryArgs {
  const void *q, *k;
  void *qo, *ko;
  const int32_t *pos;
  const double *freq;
  int64_t axis_stride, q_row, q_head, k_row, k_head, qo_row, qo_head, ko_row, ko_head;
  int hq, hk, d, rot, tokens, inter;
  int end[4];                        // pairs below end[a] belong to axis a or an earlier one
  float factor, sign;
  int q_tail, k_tail;                // channels from rot on are to be copied (not in place)
};
hipError_t launch_rotary(const RotaryArgs &a, int dtype, hipStream_t s);

struct PrefixRows {
  const void *pk, *pv, *k, *v;
  int64_t pk_row, pk_head, pv_row, pv_head, k_row, k_head, v_row, v_head;
  int p_len;
};
// p.near_rows: of all four sources.
int64_t prefix_workspace(const AttnProblem &p, int p_len, const int32_t *kv_lens);
hipError_t launch_prefix(const AttnProblem &p, const PrefixRows &x, const int32_t *kv_lens, int causal, hipStream_t s);

}  // namespace mte
