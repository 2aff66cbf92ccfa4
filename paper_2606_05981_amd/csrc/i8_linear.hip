// Products of 8-bit rows: y = act(s_i t_j sum_k a_ik b_jk + bias_j).
//
// The matrix cores' 8-bit integer form (16x16x64, int32 sums: exact in any order) has twice the
// rate of 16-bit floating point for the same bytes of operands. Codes are rows of a multiple of
// 128 bytes, so that a K stage is 128 bytes of every row and there is no ragged end of K.
// C^T = B A^T: a lane then holds four consecutive columns of one row of the result.
#include "common.h"
#include "proj_launch.h"

namespace mte {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// 16 rows of either operand, 64 of K: lane l supplies row l % 16, bytes 16 (l / 16) .. + 15; register r of
// lane l is row 4 (l / 16) + r of the first operand, column l % 16 (row of the second).
__device__ __forceinline__ void mfma_i8(i32x4 &acc, const i32x4 &x, const i32x4 &y) {
  acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, y, acc, 0, 0, 0);
}

// s_i and t_j as the result needs them: with 2^-31 and 2^31, |acc| 2^-31 s_i is no more than s_i.
__device__ __forceinline__ float row_scale(float s) { return s * 0x1p-31f; }
__device__ __forceinline__ float col_scale(float t) { return t * 0x1p31f; }

template <bool ACT> __device__ __forceinline__ float finish(int acc, float s, float t, float bias) {
  float z = (float)acc * s * t + bias;
  if constexpr (ACT) z *= __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
  return z;
}

// ---- few rows -----------------------------------------------------------------------------------
//
// Bound by the bytes of the weight, or by latency. A workgroup of eight waves takes 16 weight rows and all
// rows of a (MT blocks of 16); the waves take K in turn, 128 bytes of each row at a time, straight from memory
// to the operands, and add up through LDS.
constexpr int kFewWaves = 8;
template <typename TO, int MT, bool ACT>
__global__ __launch_bounds__(64 * kFewWaves) void k_i8_few(I8Args g) {
  __shared__ i32x4 part[kFewWaves][MT][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * MT;
  const int lr = lane & 15, lk = (lane >> 4) * 16;
  const int8_t *bp = g.b + (int64_t)min(n0 + lr, g.n - 1) * g.pitch + lk;
  const int8_t *ap[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) ap[t] = g.a + (int64_t)min(m0 + 16 * t + lr, g.m - 1) * g.pitch + lk;
  i32x4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = i32x4{0, 0, 0, 0};
#pragma unroll 2
  for (int k = wave * 128; k < g.pitch; k += kFewWaves * 128) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const i32x4 b = *(const i32x4 *)(bp + k + 64 * h);
#pragma unroll
      for (int t = 0; t < MT; ++t) mfma_i8(acc[t], b, *(const i32x4 *)(ap[t] + k + 64 * h));
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) part[wave][t][lane] = acc[t];
  __syncthreads();
  // output (row 16 t + i, columns 4 c .. 4 c + 3) is lane 16 c + i of every part
  for (int x = tid; x < MT * 64; x += 64 * kFewWaves) {
    const int t = x >> 6, l = x & 63, m = m0 + 16 * t + (l & 15), n = n0 + 4 * (l >> 4);
    i32x4 s = part[0][t][l];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) s += part[w][t][l];
    if (m >= g.m) continue;
    const float sr = row_scale(g.sa[m]);
    TO *out = (TO *)g.out + (int64_t)m * g.out_row + n;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < g.n)
        out[e] = from_f32<TO>(finish<ACT>(s[e], sr, col_scale(g.sb[n + e]), g.bias ? to_f32(((const TO *)g.bias)[n + e]) : 0.f));
  }
}

template <typename TO, bool ACT> hipError_t run_few(const I8Args &g, hipStream_t s) {
  const dim3 block(64 * kFewWaves), cols((g.n + 15) / 16);
  if (g.m <= 16) hipLaunchKernelGGL((k_i8_few<TO, 1, ACT>), cols, block, 0, s, g);
  else hipLaunchKernelGGL((k_i8_few<TO, 4, ACT>), dim3(cols.x, (g.m + 63) / 64), block, 0, s, g);
  return hipGetLastError();
}

}  // namespace

// Codes and scales of rows that the call quantises itself.
int64_t i8_workspace(int x_type, int m, int, int k) {
  return x_type == MTE_I8_CODES ? 0 : (int64_t)m * i8_pitch(k) + (int64_t)m * 4;
}

hipError_t launch_i8_linear(I8Args a, int x_type, int dtype, void *ws, hipStream_t s) {
  if (x_type != MTE_I8_CODES) {
    int8_t *codes = (int8_t *)ws;
    float *scales = (float *)(codes + (int64_t)a.m * a.pitch);
    const hipError_t e = launch_i8_quantize(QuantArgs{a.x, codes, scales, a.x_row, a.m, a.k, a.pitch}, x_type, s);
    if (e != hipSuccess) return e;
    a.a = codes;
    a.sa = scales;
  }
  if (dtype == MTE_BF16) return a.act ? run_few<bf16, true>(a, s) : run_few<bf16, false>(a, s);
  return a.act ? run_few<float, true>(a, s) : run_few<float, false>(a, s);
}

}  // namespace mte
