// Rotary positions on queries and keys, one launch for both.
//
//   y1 = f (x1 cos a - x2 sin a), y2 = f (x2 cos a + x1 sin a), a = p freq[i] for pair i
//
// Bound by bytes: every channel is read and written once, 3 operations each. A workgroup takes some
// tokens: first the sines and cosines of their pairs (fp64 angle, reduced by whole turns in fp64:
// at position 2^30 an fp32 angle is off by up to 32 radians), which all heads share, into LDS; then
// the heads, V channels of either member of V pairs a thread (interleaved: V channels in a row), two units
// in flight. 65536 tokens of 2 x 10 heads of 64: 63 us, 5.3 TB/s; 5120 of 24 heads of 128: 12 us, 5.2.
#include <algorithm>

#include "common.h"
#include "proj_launch.h"

namespace mte {
namespace {

constexpr int kRotThreads = 256;
constexpr int kTableMax = 2048;      // (sin, cos) pairs of a workgroup's tokens in LDS: 16 KB

template <typename T, int V> struct Vec { typedef T type __attribute__((ext_vector_type(V))); };
template <typename T> struct Vec<T, 1> { typedef T type __attribute__((ext_vector_type(1))); };

// V: channels of a load. tb: tokens of a workgroup.
template <typename T, int V, bool INTER>
__global__ __launch_bounds__(kRotThreads) void k_rotary(RotaryArgs a, int tb) {
  __shared__ __attribute__((aligned(16))) float sines[kTableMax], cosines[kTableMax];
  const int tid = threadIdx.x, pairs = a.rot >> 1;
  const int t0 = blockIdx.x * tb, nt = min(tb, a.tokens - t0);
  for (int i = tid; i < nt * pairs; i += kRotThreads) {
    const int t = i / pairs, p = i - t * pairs;
    const int axis = (p >= a.end[0]) + (p >= a.end[1]) + (p >= a.end[2]);
    const double w = (double)a.pos[axis * a.axis_stride + t0 + t] * a.freq[p];
    // whole turns taken off: 2 pi as the sum of two doubles, so that the rest is exact to 2^-53 of itself or so
    const double n = rint(w * 0.15915494309189535);
    const double r = fma(-n, 2.4492935982947064e-16, fma(-n, 6.283185307179586, w));
    float s, c;
    sincosf((float)r, &s, &c);
    sines[i] = s * a.sign;
    cosines[i] = c;
  }
  __syncthreads();
  // units of a head: of the rotated channels, then of the rest where that is copied. Two units a thread are
  // loaded before the first is used (one by one, 65536 tokens of 20 heads of 64 took 81 us).
  constexpr int W = INTER ? V : 2 * V;                 // channels of a rotating unit
  constexpr int U = 2;
  typedef typename Vec<T, V>::type vec;
  const int heads = a.hq + a.hk, spin = a.rot / W, rest = a.q_tail | a.k_tail ? (a.d - a.rot) / V : 0, units = spin + rest;
  const int per = heads * units, all = nt * per;
  for (int i0 = tid; i0 < all; i0 += U * kRotThreads) {
    T *to[U];
    vec x1[U], x2[U];
    int at[U];                                         // of the unit's first pair in the tables; -1: copied, -2: left
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int i = min(i0 + k * kRotThreads, all - 1);
      const int t = i / per, x = i - t * per, hh = x / units, u = x - hh * units;
      const bool isk = hh >= a.hq, rotates = u < spin;
      const int h = isk ? hh - a.hq : hh, c = rotates ? u * V : a.rot + (u - spin) * V;
      const T *in = (isk ? (const T *)a.k + (t0 + t) * a.k_row + h * a.k_head : (const T *)a.q + (t0 + t) * a.q_row + h * a.q_head) + c;
      to[k] = (isk ? (T *)a.ko + (t0 + t) * a.ko_row + h * a.ko_head : (T *)a.qo + (t0 + t) * a.qo_row + h * a.qo_head) + c;
      at[k] = rotates ? t * pairs + u * (INTER ? V / 2 : V) : (isk ? a.k_tail : a.q_tail) ? -1 : -2;
      if (i0 + k * kRotThreads >= all) at[k] = -2;
      x1[k] = *(const vec *)in;
      if constexpr (!INTER) x2[k] = *(const vec *)(in + (rotates ? pairs : 0));
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (at[k] >= 0) {
        const float *sn = sines + at[k], *cs = cosines + at[k];
        if constexpr (INTER) {
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const float p = to_f32((T)x1[k][e]), q = to_f32((T)x1[k][e + 1]);
            x1[k][e] = from_f32<T>(a.factor * (p * cs[e / 2] - q * sn[e / 2]));
            x1[k][e + 1] = from_f32<T>(a.factor * (q * cs[e / 2] + p * sn[e / 2]));
          }
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float p = to_f32((T)x1[k][e]), q = to_f32((T)x2[k][e]);
            x1[k][e] = from_f32<T>(a.factor * (p * cs[e] - q * sn[e]));
            x2[k][e] = from_f32<T>(a.factor * (q * cs[e] + p * sn[e]));
          }
          *(vec *)(to[k] + pairs) = x2[k];
        }
      }
      if (at[k] >= -1) *(vec *)to[k] = x1[k];
    }
  }
}

template <typename T, int V>
hipError_t run(RotaryArgs a, int tb, hipStream_t s) {
  for (int64_t left = a.tokens; left > 0;) {           // in launches of kMostGroups workgroups
    a.tokens = (int)std::min<int64_t>(left, (int64_t)kMostGroups * tb);
    const dim3 grid((a.tokens + tb - 1) / tb);
    if (a.inter) {
      if constexpr (V > 1) hipLaunchKernelGGL((k_rotary<T, V, true>), grid, dim3(kRotThreads), 0, s, a, tb);
    } else {
      hipLaunchKernelGGL((k_rotary<T, V, false>), grid, dim3(kRotThreads), 0, s, a, tb);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    left -= a.tokens;
    a.pos += a.tokens;
    a.q = (const T *)a.q + a.tokens * a.q_row;
    a.qo = (T *)a.qo + a.tokens * a.qo_row;
    if (a.hk > 0) {
      a.k = (const T *)a.k + a.tokens * a.k_row;
      a.ko = (T *)a.ko + a.tokens * a.ko_row;
    }
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs &a, int dtype, hipStream_t s) {
  // the widest load that the members of a pair allow: strides and bases are multiples of 8 channels
  const int apart = a.inter ? a.rot : a.rot / 2, most = dtype == MTE_BF16 ? 8 : 4;
  int v = a.inter ? 2 : 1;
  while (v < most && apart % (2 * v) == 0) v *= 2;
  const int units = (a.hq + a.hk) * ((a.inter ? a.rot / v : a.rot / 2 / v) + (a.q_tail | a.k_tail ? (a.d - a.rot) / v : 0));
  // tokens of a workgroup: about four units a thread, 512 workgroups at least
  int tb = (4 * kRotThreads + units - 1) / units;
  tb = tb < a.tokens / 512 ? tb : a.tokens / 512;
  tb = tb < kTableMax / (a.rot / 2) ? tb : kTableMax / (a.rot / 2);
  tb = tb < 1 ? 1 : tb;
  if (dtype == MTE_BF16) {
    if (v == 8) return run<bf16, 8>(a, tb, s);
    if (v == 4) return run<bf16, 4>(a, tb, s);
    if (v == 2) return run<bf16, 2>(a, tb, s);
    return run<bf16, 1>(a, tb, s);
  }
  if (v == 4) return run<float, 4>(a, tb, s);
  if (v == 2) return run<float, 2>(a, tb, s);
  return run<float, 1>(a, tb, s);
}

}  // namespace mte
