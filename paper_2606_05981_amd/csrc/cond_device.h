// What the kernels of the operators that read the conditioning share on the device.
#pragma once

#include "common.h"
#include "cond_launch.h"

namespace mte {

// The sequence whose tiles hold `tile` (their first tiles ascend). Two sequences a lane, counted: one
// memory latency, where a binary search is one a step (64 sequences: 0.3 us of a launch of 5 to 8).
// All lanes of the wave call it.
__device__ __forceinline__ int find_seq(const CondSeq *seq, int n, int tile) {
  static_assert(kCondSeqs == 128, "two sequences a lane");
  if (n == 1) return 0;
  const int lane = threadIdx.x & 63;
  int before = __popcll(__ballot(lane < n && seq[min(lane, n - 1)].tile0 <= tile));
  if (n > 64) before += __popcll(__ballot(lane + 64 < n && seq[min(lane + 64, n - 1)].tile0 <= tile));
  return __builtin_amdgcn_readfirstlane(before - 1);
}

}  // namespace mte
