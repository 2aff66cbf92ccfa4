// Rows to 8-bit integers on the device (include/mte_proj.h has the definition).
#pragma once

#include "common.h"

namespace mte {

// Eight consecutive elements of a row as they lie in memory. Rows are aligned like an element: the
// hardware takes loads of 16 bytes at any such address.
typedef uint32_t u32x4e __attribute__((ext_vector_type(4), aligned(2)));
template <typename T> struct Eight;
template <> struct Eight<bf16> {
  u32x4 w;
  __device__ __forceinline__ float get(int i) const {
    return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
  }
  __device__ __forceinline__ void zero() { w = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void load(const bf16 *p) { w = *(const u32x4e *)p; }
  __device__ __forceinline__ void set(int i, bf16 x) {
    const uint32_t b = __builtin_bit_cast(uint16_t, x);
    w[i >> 1] |= i & 1 ? b << 16 : b;
  }
  // itself, another or zeros
  __device__ __forceinline__ void keep(bool mine, bool other, const Eight &y) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = mine ? w[i] : other ? y.w[i] : 0u;
  }
};
template <> struct Eight<float> {
  f32x4 a, b;
  __device__ __forceinline__ float get(int i) const { return i < 4 ? a[i] : b[i - 4]; }
  __device__ __forceinline__ void zero() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void load(const float *p) {
    a = *(const f32x4u *)p;
    b = *(const f32x4u *)(p + 4);
  }
  __device__ __forceinline__ void set(int i, float x) {
    if (i < 4) a[i] = x;
    else b[i - 4] = x;
  }
  __device__ __forceinline__ void keep(bool mine, bool other, const Eight &y) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = mine ? a[i] : other ? y.a[i] : 0.f;
      b[i] = mine ? b[i] : other ? y.b[i] : 0.f;
    }
  }
};

// A row of at least 8 elements in chunks of 8. A load is one instruction in any case, so that many are in flight at
// once (as a branch each, they were waited for one by one: 128 rows of 320 elements a workgroup, 25 us): past the
// last whole chunk it repeats that, and keep() puts in what belongs there once it is needed.
template <typename T> struct RowChunks {
  const T *row;
  int full;                                          // elements of whole chunks
  Eight<T> tail;                                     // the elements after them, then zeros
  __device__ __forceinline__ void open(const T *r, int cols) {
    row = r;
    full = cols & ~7;
    tail.zero();
    if (cols & 7) {                                  // uniform
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < (cols & 7)) tail.set(i, row[full + i]);
    }
  }
  __device__ __forceinline__ void load(Eight<T> &y, int e) const { y.load(row + min(e, full - 8)); }
  __device__ __forceinline__ void keep(Eight<T> &y, int e) const { y.keep(e < full, e == full, tail); }
};

// The largest magnitude of a lane's elements as the bits of a float (they order like it; NaN lies above infinity).
template <typename T> struct Top;
template <> struct Top<bf16> {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u16x2 t{0, 0};
  __device__ __forceinline__ void take(const Eight<bf16> &y) {
#pragma unroll
    for (int i = 0; i < 4; ++i) t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, y.w[i] & 0x7FFF7FFFu));
  }
  __device__ __forceinline__ uint32_t bits() const { return (uint32_t)max(t[0], t[1]) << 16; }
};
template <> struct Top<float> {
  uint32_t t = 0;
  __device__ __forceinline__ void take(const Eight<float> &y) {
#pragma unroll
    for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(y.get(i)) & 0x7FFFFFFFu);
  }
  __device__ __forceinline__ uint32_t bits() const { return t; }
};
// Over 2 STEP lanes that differ in their low bits.
template <int STEP> __device__ __forceinline__ uint32_t lanes_top(uint32_t t) {
#pragma unroll
  for (int m = STEP; m >= 1; m >>= 1) t = max(t, (uint32_t)__shfl_xor((int)t, m, kWave));
  return t;
}

// s is top times the rounded 1 / 127, as torch divides by a number here: 4.7% of fp32 values and 6 of bf16's 128 mantissas
// lie a unit in the last place from the rounded quotient, and beside a half their codes would differ.
// Codes are those of the exact quotient x / s. x times the rounded 1 / s is off by 2^-16 at most, so that its nearest whole
// number (the sum with 1.5 2^23 leaves it in the low bits) is the quotient's, unless it lies next to a half. There,
// c may be off by one: r = x - c s is exact in one fma (a multiple of the finer ulp of x and s, and no more
// than s), and c moves by one towards r where |r| is more than s / 2, or is s / 2 and c odd. 7 instructions an
// element; with the second step for all 20, and quantising 65536 rows of 320 took 25 us where the bytes take 10.
struct Scale {
  float s, inv;
  bool bad;
  __device__ __forceinline__ explicit Scale(uint32_t top) {
    bad = top >= 0x7F800000u;
    s = fmaxf(__uint_as_float(bad ? 0u : top) * (1.f / 127.f), 0x1p-126f);
    inv = 1.f / s;
  }
  __device__ __forceinline__ float stored() const { return bad ? __uint_as_float(0x7FC00000u) : s; }
  __device__ __forceinline__ int exact(float x) const {
    const float c0 = rintf(x * inv), r = fmaf(-c0, s, x);
    int c = (int)c0;
    const float d = fabsf(r) - (s - fabsf(r));       // the sign of 2 |r| - s
    if (d > 0.f || (d == 0.f && (c & 1))) c += r > 0.f ? 1 : -1;
    return c;
  }
  template <typename T> __device__ __forceinline__ u32x2 codes(const Eight<T> &y) const {
    constexpr float kWhole = 0x1.8p23f;
    uint32_t t[8];
    float worst = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = y.get(i), w = fmaf(x, inv, kWhole);
      t[i] = __float_as_uint(w);
      worst = fmaxf(worst, fabsf(fmaf(x, inv, -(w - kWhole))));
    }
    if (worst > 0.5f - 0x1p-15f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = (uint32_t)exact(y.get(i));
    }
    u32x2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      r[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(t[4 * i + 3], t[4 * i + 2], 0x0C0C0400u),
                                   __builtin_amdgcn_perm(t[4 * i + 1], t[4 * i], 0x0C0C0400u), 0x05040100u);
    return bad ? u32x2{0, 0} : r;
  }
};

}  // namespace mte
