// Rows as 8-bit integers with a scale each: s = max |x| (1/127), c = x / s to the nearest whole number.
//
// Codes are those of the exact quotient: c0 = rint(x * (1/s)) is off by at most one, r = x - c0 s is
// exact in one fma (a multiple of the finer ulp of x and s, and no more than s), and c0 moves by
// one towards r where |r| is more than s / 2, or is s / 2 and c0 odd. A division an element takes twice the
// instructions and still rounds twice.
// Bound by bytes: x is read once, into registers where a row is 4096 elements or fewer (a wave a
// row); longer rows (a workgroup a row) are read twice, the second time from the caches.
#include "common.h"
#include "proj_launch.h"

namespace mte {
namespace {

constexpr int kThreads = 256;

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

// A wave a row, NC chunks of 8 elements a lane.
template <typename T, bool VEC, int NC>
__global__ __launch_bounds__(kThreads) void k_i8_rows(QuantArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= a.rows) return;
  const T *row = (const T *)a.x + r * a.x_row;
  float y[NC][8];
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < NC; ++j) load8<T, VEC>(y[j], row, (j * 64 + lane) * 8, a.cols);
#pragma unroll
  for (int j = 0; j < NC; ++j) top = top8(y[j], top);
  const Scale sc(wave_top(top));
  int8_t *out = a.codes + r * a.pitch;
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int e = (j * 64 + lane) * 8;
    if (e < a.pitch) *(u32x2 *)(out + e) = sc.codes(y[j]);
  }
  if (lane == 0) a.scales[r] = sc.stored();
}

// A workgroup a row.
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void k_i8_long_rows(QuantArgs a) {
  __shared__ uint32_t tops[4];
  const int tid = threadIdx.x;
  const int64_t r = blockIdx.x;
  const T *row = (const T *)a.x + r * a.x_row;
  float y[8];
  uint32_t top = 0;
#pragma unroll 4
  for (int e = tid * 8; e < a.cols; e += kThreads * 8) {
    load8<T, VEC>(y, row, e, a.cols);
    top = top8(y, top);
  }
  top = wave_top(top);
  if ((tid & 63) == 0) tops[tid >> 6] = top;
  __syncthreads();
  const Scale sc(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
  int8_t *out = a.codes + r * a.pitch;
#pragma unroll 4
  for (int e = tid * 8; e < a.pitch; e += kThreads * 8) {
    load8<T, VEC>(y, row, e, a.cols);
    *(u32x2 *)(out + e) = sc.codes(y);
  }
  if (tid == 0) a.scales[r] = sc.stored();
}

template <typename T, bool VEC> hipError_t run(const QuantArgs &a, hipStream_t s) {
  const dim3 grid((uint32_t)(((int64_t)a.rows + 3) / 4)), block(kThreads);
  if (a.pitch <= 512) hipLaunchKernelGGL((k_i8_rows<T, VEC, 1>), grid, block, 0, s, a);
  else if (a.pitch <= 1024) hipLaunchKernelGGL((k_i8_rows<T, VEC, 2>), grid, block, 0, s, a);
  else if (a.pitch <= 2048) hipLaunchKernelGGL((k_i8_rows<T, VEC, 4>), grid, block, 0, s, a);
  else if (a.pitch <= 4096) hipLaunchKernelGGL((k_i8_rows<T, VEC, 8>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_i8_long_rows<T, VEC>), dim3(a.rows), block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_i8_quantize(const QuantArgs &a, int dtype, hipStream_t s) {
  const int64_t es = dtype == MTE_BF16 ? 2 : 4;
  const bool vec = ((uintptr_t)a.x & 15) == 0 && (a.rows == 1 || a.x_row * es % 16 == 0);
  if (dtype == MTE_BF16) return vec ? run<bf16, true>(a, s) : run<bf16, false>(a, s);
  return vec ? run<float, true>(a, s) : run<float, false>(a, s);
}

}  // namespace mte
