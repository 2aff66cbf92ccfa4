// Rows as 8-bit integers with a scale each: s = max |x| (1/127), c = x / s to the nearest whole number.
//
// Bound by bytes: x is read once, into registers where a row is 4096 elements or fewer (a wave a
// row); longer rows (a workgroup a row) are read twice, the second time from the caches. 5120 rows of 2048 bf16: 10
// us, 3.1 TB/s: all rows are resident at once, so that reading, scaling and writing are phases.
#include <algorithm>

#include "i8_device.h"
#include "proj_launch.h"

namespace mte {
namespace {

constexpr int kThreads = 256;

// A wave a row, NC chunks of 8 elements a lane.
template <typename T, int NC>
__global__ __launch_bounds__(kThreads) void k_i8_rows(QuantArgs a) {
  const int lane = threadIdx.x & 63;
  for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < a.rows; r += (int64_t)gridDim.x * 4) {
    RowChunks<T> row;
    Eight<T> y[NC];
    row.open((const T *)a.x + r * a.x_row, a.cols);
#pragma unroll
    for (int j = 0; j < NC; ++j) row.load(y[j], (j * 64 + lane) * 8);
    Top<T> top;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      row.keep(y[j], (j * 64 + lane) * 8);
      top.take(y[j]);
    }
    const Scale sc(lanes_top<32>(top.bits()));
    int8_t *out = a.codes + r * a.pitch;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int e = (j * 64 + lane) * 8;
      if (e < a.pitch) *(u32x2 *)(out + e) = sc.codes(y[j]);
    }
    if (lane == 0) a.scales[r] = sc.stored();
  }
}

// A workgroup a row, four chunks a lane at a time.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_i8_long_rows(QuantArgs a) {
  constexpr int NC = 4;
  __shared__ uint32_t tops[4];
  const int tid = threadIdx.x;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    RowChunks<T> row;
    row.open((const T *)a.x + r * a.x_row, a.cols);
    Eight<T> y[NC];
    Top<T> top;
    for (int e0 = tid * 8; e0 < a.cols; e0 += NC * kThreads * 8) {
#pragma unroll
      for (int j = 0; j < NC; ++j) row.load(y[j], e0 + j * kThreads * 8);
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        row.keep(y[j], e0 + j * kThreads * 8);
        top.take(y[j]);
      }
    }
    const uint32_t mine = lanes_top<32>(top.bits());
    if ((tid & 63) == 0) tops[tid >> 6] = mine;
    __syncthreads();
    const Scale sc(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
    int8_t *out = a.codes + r * a.pitch;
    for (int e0 = tid * 8; e0 < a.pitch; e0 += NC * kThreads * 8) {
#pragma unroll
      for (int j = 0; j < NC; ++j) row.load(y[j], e0 + j * kThreads * 8);
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int e = e0 + j * kThreads * 8;
        row.keep(y[j], e);
        if (e < a.pitch) *(u32x2 *)(out + e) = sc.codes(y[j]);
      }
    }
    if (tid == 0) a.scales[r] = sc.stored();
    __syncthreads();                                 // the maxima are read
  }
}

// Rows of fewer than 8 elements: a lane a row.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_i8_tiny_rows(QuantArgs a) {
  const int64_t r = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (r >= a.rows) return;
  const T *row = (const T *)a.x + r * a.x_row;
  Eight<T> y;
  Top<T> top;
  y.zero();
  for (int i = 0; i < 7; ++i)
    if (i < a.cols) y.set(i, row[i]);
  top.take(y);
  const Scale sc(top.bits());
  u32x4 *out = (u32x4 *)(a.codes + r * a.pitch);
  const u32x2 c = sc.codes(y);
  out[0] = u32x4{c[0], c[1], 0, 0};
  for (int i = 1; i < kI8Pitch / 16; ++i) out[i] = u32x4{0, 0, 0, 0};
  a.scales[r] = sc.stored();
}

template <typename T> hipError_t run(const QuantArgs &a, hipStream_t s) {
  // (the kernels go on in strides of the grid)
  const dim3 grid((uint32_t)std::min<int64_t>(((int64_t)a.rows + 3) / 4, kMostGroups)), block(kThreads);
  if (a.cols < 8) hipLaunchKernelGGL((k_i8_tiny_rows<T>), dim3((uint32_t)(((int64_t)a.rows + kThreads - 1) / kThreads)), block, 0, s, a);
  else if (a.pitch <= 512) hipLaunchKernelGGL((k_i8_rows<T, 1>), grid, block, 0, s, a);
  else if (a.pitch <= 1024) hipLaunchKernelGGL((k_i8_rows<T, 2>), grid, block, 0, s, a);
  else if (a.pitch <= 2048) hipLaunchKernelGGL((k_i8_rows<T, 4>), grid, block, 0, s, a);
  else if (a.pitch <= 4096) hipLaunchKernelGGL((k_i8_rows<T, 8>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_i8_long_rows<T>), dim3((uint32_t)std::min(a.rows, kMostGroups)), block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_i8_quantize(const QuantArgs &a, int dtype, hipStream_t s) {
  return dtype == MTE_BF16 ? run<bf16>(a, s) : run<float>(a, s);
}

}  // namespace mte
