// Rows to 8-bit integers on the device (include/mte_proj.h has the definition).
#pragma once

#include "common.h"

namespace mte {

// Elements e .. e + 7 of a row (zeros past its end).
template <typename T, bool VEC> __device__ __forceinline__ void load8(float (&y)[8], const T *row, int e, int cols) {
  if constexpr (VEC) {                               // 16-byte aligned rows
    if (e + 8 <= cols) {
      if constexpr (sizeof(T) == 2) {
        const bf16x8 v = *(const bf16x8 *)(row + e);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (float)v[i];
      } else {
        const f32x4 v = *(const f32x4 *)(row + e), w = *(const f32x4 *)(row + e + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[i] = v[i];
          y[4 + i] = w[i];
        }
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = e + i < cols ? to_f32(row[min(e + i, cols - 1)]) : 0.f;
}

// Largest magnitude so far as the bits of a float (they order like it; NaN lies above infinity).
__device__ __forceinline__ uint32_t top8(const float (&y)[8], uint32_t top) {
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(y[i]) & 0x7FFFFFFFu);
  return top;
}
__device__ __forceinline__ uint32_t wave_top(uint32_t t) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) t = max(t, (uint32_t)__shfl_xor((int)t, m, kWave));
  return t;
}

// Codes are those of the exact quotient: c0 = rint(x * (1/s)) is off by at most one, r = x - c0 s is
// exact in one fma (a multiple of the finer ulp of x and s, and no more than s), and c0 moves by
// one towards r where |r| is more than s / 2, or is s / 2 and c0 odd. A division an element takes twice the
// instructions and still rounds twice.
struct Scale {
  float s, inv;
  bool bad;
  __device__ __forceinline__ explicit Scale(uint32_t top) {
    bad = top >= 0x7F800000u;
    s = fmaxf(__uint_as_float(bad ? 0u : top) * (1.f / 127.f), 0x1p-126f);
    inv = 1.f / s;
  }
  __device__ __forceinline__ float stored() const { return bad ? __uint_as_float(0x7FC00000u) : s; }
  __device__ __forceinline__ int code(float x) const {
    const float c0 = rintf(x * inv), r = fmaf(-c0, s, x);
    int c = (int)c0;
    const float d = fabsf(r) - (s - fabsf(r));       // the sign of 2 |r| - s: the difference is exact
    if (d > 0.f || (d == 0.f && (c & 1))) c += r > 0.f ? 1 : -1;
    return c;
  }
  __device__ __forceinline__ u32x2 codes(const float (&y)[8]) const {
    u32x2 w{0, 0};
    if (bad) return w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2] |= (uint32_t)(code(y[i]) & 0xFF) << (8 * (i & 3));
    return w;
  }
};

}  // namespace mte
