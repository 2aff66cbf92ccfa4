// Products of 8-bit rows: y = act(s_i t_j sum_k a_ik b_jk + bias_j).
//
// The matrix cores' 8-bit integer form (16x16x64, int32 sums: exact in any order) has twice the
// rate of 16-bit floating point for the same bytes of operands. Codes are rows of a multiple of
// 128 bytes, so that a K stage is 128 bytes of every row and there is no ragged end of K.
// C^T = B A^T: a lane then holds four consecutive columns of one row of the result.
#include <cmath>

#include "gemm_kernel.h"
#include "i8_device.h"
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

// ---- up to 16 rows ------------------------------------------------------------------------------
//
// Bound by the bytes of the weight, or by latency. A workgroup of 16 waves takes blocks of 16 weight rows in
// turn; its waves share K, 128 bytes of each row at a time, straight from memory to the operands (the next
// block's loads are in flight meanwhile), and add up through LDS. The rows of a are few enough to lie in LDS
// whole; every workgroup quantises them for itself, once, while its first weights arrive: a launch less than with
// codes through memory.
// LDS: rows of codes 64 bytes further apart than they are long, so that an operand's 16 rows of 64 bytes
// fill the banks.
constexpr int kFewWaves = 16, kFewRows = 16, kFewThreads = 64 * kFewWaves, kFewLds = 96 * 1024;
int few_lds(int m, int pitch) { return m * (pitch + 64); }

template <typename T, typename TO, bool ACT>
__global__ __launch_bounds__(kFewThreads) void k_i8_few(I8Args g) {
  constexpr int AHEAD = 2;                        // blocks of 128 bytes of K a wave and weight row, ahead
  __shared__ i32x4 part[2][kFewWaves][64];
  __shared__ uint32_t tops[kFewRows];
  __shared__ float sa[kFewRows];
  extern __shared__ u32x4 lds[];
  char *codes = (char *)lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lk = (lane >> 4) * 16, row_bytes = g.pitch + 64;
  const int blocks = (g.n + 15) / 16;
  i32x4 w[2 * AHEAD];
  auto fetch = [&](int nb) {
    const int8_t *bp = g.b + (int64_t)min(nb * 16 + lr, g.n - 1) * g.pitch + lk;
#pragma unroll
    for (int b = 0; b < AHEAD; ++b) {
      const int k = (wave + b * kFewWaves) * 128;
      if (k < g.pitch) {                          // uniform
        w[2 * b] = *(const i32x4 *)(bp + k);
        w[2 * b + 1] = *(const i32x4 *)(bp + k + 64);
      }
    }
  };
  fetch(blockIdx.x);

  if constexpr (sizeof(T) == 1) {
    for (int i = tid; i < g.m * (g.pitch / 16); i += kFewThreads) {
      const int r = i / (g.pitch / 16), c = i - r * (g.pitch / 16);
      *(u32x4 *)(codes + r * row_bytes + c * 16) = *(const u32x4 *)(g.a + (int64_t)r * g.pitch + c * 16);
    }
    if (tid < g.m) sa[tid] = row_scale(g.sa[tid]);
  } else {
    if (tid < kFewRows) tops[tid] = 0;
    __syncthreads();
    // 1024, 512, .. 64 threads a row
    const int per = kFewThreads >> (g.m > 8 ? 4 : g.m > 4 ? 3 : g.m > 2 ? 2 : g.m > 1 ? 1 : 0), r = tid / per, c0 = tid % per;
    const T *row = (const T *)g.x + (int64_t)min(r, g.m - 1) * g.x_row;
    constexpr int KEPT = 4;
    Eight<T> y[KEPT];
    Top<T> top;
    auto read = [&](Eight<T> &z, int c) { load8<T>(z, row, c * 8, g.k); };
#pragma unroll
    for (int j = 0; j < KEPT; ++j) read(y[j], c0 + j * per);
#pragma unroll
    for (int j = 0; j < KEPT; ++j) top.take(y[j]);
    for (int c = c0 + KEPT * per; c * 8 < g.k; c += per) {
      Eight<T> z;
      read(z, c);
      top.take(z);
    }
    const uint32_t t = lanes_top<32>(top.bits());  // a wave is within a row
    if (lane == 0) atomicMax(&tops[r], t);
    __syncthreads();
    const Scale sc(tops[r]);
    if (r < g.m) {
      char *to = codes + r * row_bytes;
#pragma unroll
      for (int j = 0; j < KEPT; ++j)
        if ((c0 + j * per) * 8 < g.pitch) *(u32x2 *)(to + (c0 + j * per) * 8) = sc.codes(y[j]);
      for (int c = c0 + KEPT * per; c * 8 < g.pitch; c += per) {
        Eight<T> z;
        read(z, c);
        *(u32x2 *)(to + c * 8) = sc.codes(z);
      }
      if (c0 == 0) sa[r] = row_scale(sc.stored());
    }
  }
  __syncthreads();

  const char *ap = codes + min(lr, g.m - 1) * row_bytes + lk;
  int buf = 0;
  for (int nb = blockIdx.x; nb < blocks; nb += gridDim.x, buf ^= 1) {
    i32x4 acc{0, 0, 0, 0};
#pragma unroll
    for (int b = 0; b < AHEAD; ++b) {
      const int k = (wave + b * kFewWaves) * 128;
      if (k < g.pitch) {
        mfma_i8(acc, w[2 * b], *(const i32x4 *)(ap + k));
        mfma_i8(acc, w[2 * b + 1], *(const i32x4 *)(ap + k + 64));
      }
    }
    if (g.pitch > AHEAD * kFewWaves * 128) {      // long rows: the rest
      const int8_t *bp = g.b + (int64_t)min(nb * 16 + lr, g.n - 1) * g.pitch + lk;
#pragma unroll 2
      for (int k = (wave + AHEAD * kFewWaves) * 128; k < g.pitch; k += kFewWaves * 128) {
        mfma_i8(acc, *(const i32x4 *)(bp + k), *(const i32x4 *)(ap + k));
        mfma_i8(acc, *(const i32x4 *)(bp + k + 64), *(const i32x4 *)(ap + k + 64));
      }
    }
    part[buf][wave][lane] = acc;
    if (nb + (int)gridDim.x < blocks) fetch(nb + gridDim.x);
    __syncthreads();
    if (tid < 256) {                              // register e of lane l of every part: row l % 16, column 4 (l / 16) + e
      const int l = tid >> 2, e = tid & 3, m = l & 15, n = nb * 16 + 4 * (l >> 4) + e;
      int sum = 0;
#pragma unroll
      for (int v = 0; v < kFewWaves; ++v) sum += ((const int *)&part[buf][v][0])[tid];
      if (m < g.m && n < g.n)
        ((TO *)g.out)[(int64_t)m * g.out_row + n] =
            from_f32<TO>(finish<ACT>(sum, sa[m], col_scale(g.sb[n]), g.bias ? to_f32(((const TO *)g.bias)[n]) : 0.f));
    }
  }
}

template <typename T, typename TO, bool ACT> hipError_t run_few(const I8Args &g, hipStream_t s) {
  const int bytes = few_lds(g.m, g.pitch), blocks = (g.n + 15) / 16;
  auto kern = k_i8_few<T, TO, ACT>;
  if (bytes > 16384) {                            // with the partial sums' 33 KB
    static const hipError_t attr = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, kFewLds);
    if (attr != hipSuccess) return attr;
  }
  hipLaunchKernelGGL(kern, dim3(blocks < 256 ? blocks : 256), dim3(kFewThreads), bytes, s, g);
  return hipGetLastError();
}
bool takes_few(int m, int pitch) { return m <= kFewRows && few_lds(m, pitch) <= kFewLds; }

// ---- many rows ----------------------------------------------------------------------------------
//
// A workgroup takes a BM x BN tile of the result, a wave (BM / WM) x (BN / WN) of it. K goes by in stages of
// 128 bytes a row through a ring of P slots that LDS-direct copies fill (as in the encoder's
// projections, see gemm_kernel.h: swizzle, one barrier a stage, fragments of the longer side of a wave's tile used by
// one row of products each and then replaced, those of the shorter side double-buffered). Rows past the
// last are repeats of it and are not stored.
// The result goes through LDS, 16 rows of a wave at a time, so that it is stored in whole lines and at any
// alignment.
struct I8Tile { int bm, bn, wm, wn, p, occ; double stage_us, tile_us; };

template <typename TO, int BM, int BN, int WM, int WN, int P, int OCC, bool ACT>
__global__ __launch_bounds__(64 * WM * WN, OCC) __attribute__((amdgpu_waves_per_eu((OCC * WM * WN + 3) / 4, (OCC * WM * WN + 3) / 4))) void k_i8_gemm(I8Args g) {
  constexpr int CH = kStageBytes / 16;            // 16-byte chunks of a row and stage
  constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;
  constexpr int NW = WM * WN;
  constexpr int ACH = BM * CH, BCH = BN * CH, AG = ACH / 64, BG = BCH / 64;   // chunks, groups of 64 of them
  constexpr int AR = (AG + NW - 1) / NW, BR = (BG + NW - 1) / NW, LOADS = AR + BR;   // copies of a wave a stage
  constexpr int STAGE = ACH + BCH;
  static_assert(LOADS * (P - 1) < 64 && P >= 2, "vmcnt range");
  extern __shared__ u32x4 lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave / WN, wn = wave % WN, uwave = __builtin_amdgcn_readfirstlane(wave);
  int tn, tm;
  {
    // XCD of this workgroup and its index there -> its place in the tile sequence (GemmArgs)
    const int total = gridDim.x, xcd = blockIdx.x & 7;
    const int t = xcd * (total >> 3) + min(xcd, total & 7) + ((int)blockIdx.x >> 3);
    const int grp = t / (g.gh * g.gn), m1 = grp * g.gh, h = min(g.gh, g.gm - m1), v = t - m1 * g.gn;
    tn = v / h;
    tm = m1 + v - tn * h;
  }
  const int n0 = tn * BN, m0 = tm * BM, M = g.m, N = g.n;
  const int8_t *ab = g.a + (int64_t)m0 * g.pitch, *bb = g.b + (int64_t)n0 * g.pitch;   // wave-uniform
  const int nk = g.pitch / kStageBytes;
  uint32_t pa[AR], pb[BR];                        // a tile's rows are under 2^26 bytes apart
#pragma unroll
  for (int c = 0; c < AR; ++c) {
    const int q = min(c * NW + wave, AG - 1) * 64 + lane, r = q / CH;
    pa[c] = (uint32_t)min(r, M - 1 - m0) * (uint32_t)g.pitch + swz<CH>(r, q % CH) * 16;
  }
#pragma unroll
  for (int c = 0; c < BR; ++c) {
    const int q = min(c * NW + wave, BG - 1) * 64 + lane, r = q / CH;
    pb[c] = (uint32_t)min(r, N - 1 - n0) * (uint32_t)g.pitch + swz<CH>(r, q % CH) * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  auto dma_one = [&](int ks, int slot, int x) {
    const uint32_t st = lds0 + (uint32_t)(slot * STAGE) * 16u;
    const int ko = ks * kStageBytes;
    if (x < AR) dma16(ab + ko, pa[x], st + (uint32_t)(min(x * NW + uwave, AG - 1) * 64) * 16u);
    else dma16(bb + ko, pb[x - AR], st + (uint32_t)(ACH + min((x - AR) * NW + uwave, BG - 1) * 64) * 16u);
  };

  i32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  constexpr int KK = 2;                           // k-steps of 64 a stage
  constexpr bool RA = TM >= TN;                   // rows of products run over the fragments of a
  constexpr int X = RA ? TM : TN, Y = RA ? TN : TM, NM = TM * TN;
  i32x4 fx[X], fy[2][Y];
  const int lc = lane & 15, rg = lane >> 4;
  uint32_t oa[KK], ob[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    oa[kk] = (uint32_t)((wm * WTM + lc) * CH + swz<CH>(lc, 4 * kk + rg)) * 16u;
    ob[kk] = (uint32_t)(ACH + (wn * WTN + lc) * CH + swz<CH>(lc, 4 * kk + rg)) * 16u;
  }
  const char *ldsb = (const char *)lds;
  auto frag = [&](uint32_t st, uint32_t o, int t) { return *(const i32x4 *)(ldsb + (st + o) + t * 16 * CH * 16); };
  auto read_x = [&](uint32_t st, int kk, int o) { fx[o] = frag(st, RA ? oa[kk] : ob[kk], o); };
  auto read_y = [&](uint32_t st, int kk, int b, int y) { fy[b][y] = frag(st, RA ? ob[kk] : oa[kk], y); };
  auto mfma_one = [&](int cur, int m) {
    const int o = m / Y, y = m % Y;
    if constexpr (RA) mfma_i8(acc[o][y], fy[cur][y], fx[o]);
    else mfma_i8(acc[y][o], fx[o], fy[cur][y]);
  };
  constexpr int NPART = (P >= 3) ? KK : 1, PART = (LOADS + NPART - 1) / NPART;
  auto kstep = [&](int cur, uint32_t rst, int rkk, int ks, int slot, int d0, int d1, bool bar) {
    const int b0 = bar ? Y - 1 : 0, nd = d1 - d0;
    auto upto = [&](int m, int n, int w) { return m <= b0 ? 0 : m >= b0 + w ? n : ((m - b0) * n + w - 1) / w; };
    const int wy = (NM - b0 + 1) / 2, wd = NM - b0;
#pragma unroll
    for (int m = 0; m < NM; ++m) {
      mfma_one(cur, m);
      if (bar && m == b0) {
        wait_vm_lds0<(P - 2) * LOADS>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
#pragma unroll
      for (int y = upto(m, Y, wy); y < upto(m + 1, Y, wy); ++y) read_y(rst, rkk, cur ^ 1, y);
      if (m % Y == Y - 1) read_x(rst, rkk, m / Y);
#pragma unroll
      for (int d = upto(m, nd, wd); d < upto(m + 1, nd, wd); ++d) dma_one(ks, slot, d0 + d);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  constexpr int PRE_FULL = (NPART > 1) ? P - 1 : P, PRE_PART = (NPART > 1) ? (PART < LOADS ? PART : LOADS) : 0;
#pragma unroll
  for (int s = 0; s < PRE_FULL; ++s)
#pragma unroll
    for (int x = 0; x < LOADS; ++x) dma_one(min(s, nk - 1), s, x);
#pragma unroll
  for (int x = 0; x < PRE_PART; ++x) dma_one(min(P - 1, nk - 1), P - 1, x);
  wait_vm<(PRE_FULL - 1) * LOADS + PRE_PART>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int y = 0; y < Y; ++y) read_y(0, 0, 0, y);
#pragma unroll
  for (int o = 0; o < X; ++o) read_x(0, 0, o);
  for (int kt = 0; kt < nk; ++kt) {
    const uint32_t st = (uint32_t)((kt % P) * STAGE) * 16u, nx = (uint32_t)(((kt + 1) % P) * STAGE) * 16u;
    const int ksa = min(kt + P - 1, nk - 1), sla = (kt + P - 1) % P, ksb = min(kt + P, nk - 1), slb = kt % P;
    kstep(0, st, 1, ksa, sla, NPART > 1 ? min(PART, LOADS) : 0, NPART > 1 ? LOADS : 0, false);
    kstep(1, nx, 0, ksb, slb, 0, NPART > 1 ? min(PART, LOADS) : LOADS, true);
  }
  wait_vm<0>();
  __syncthreads();                                // every copy has landed, every fragment is read

  // row mw + 16 i + lc, columns cw + 16 j + 4 rg .. + 3
  const int mw = m0 + uwave / WN * WTM, cw = n0 + uwave % WN * WTN;
  if (mw >= M || cw >= N) return;
  constexpr int PITCH = WTN * (int)sizeof(TO) + 32;
  constexpr int CPR = WTN * (int)sizeof(TO) / 16; // 16-byte chunks of a row
  char *box = (char *)lds + uwave * 16 * PITCH;
  static_assert(NW * 16 * PITCH <= P * STAGE * 16, "room to turn the result");
  f32x4 tc[TN], bs[TN];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int n = min(cw + 16 * j + 4 * rg + e, N - 1);
      tc[j][e] = col_scale(g.sb[n]);
      bs[j][e] = g.bias ? to_f32(((const TO *)g.bias)[n]) : 0.f;
    }
  const bool vec = (((uintptr_t)g.out | (uint64_t)(g.out_row * (int64_t)sizeof(TO))) & 15) == 0 && cw + WTN <= N;   // uniform
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int mb = mw + 16 * i;
    if (mb >= M) break;                           // uniform
    const float sr = row_scale(g.sa[min(mb + lc, M - 1)]);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      typedef TO to4 __attribute__((ext_vector_type(4)));
      to4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = from_f32<TO>(finish<ACT>(acc[i][j][e], sr, tc[j][e], bs[j][e]));
      *(to4 *)(box + lc * PITCH + (16 * j + 4 * rg) * (int)sizeof(TO)) = y;
    }
    if (vec) {
#pragma unroll
      for (int x = 0; x < 16 * CPR / 64; ++x) {
        const int q = x * 64 + lane, r = q / CPR, c = q % CPR;
        const u32x4 v = *(const u32x4 *)(box + r * PITCH + c * 16);
        if (mb + r < M) *(u32x4 *)((char *)g.out + ((int64_t)(mb + r) * g.out_row + cw) * (int)sizeof(TO) + c * 16) = v;
      }
    } else {
      for (int q = lane; q < 16 * WTN; q += 64) {
        const int r = q / WTN, c = q % WTN;
        const TO v = *(const TO *)(box + r * PITCH + c * (int)sizeof(TO));
        if (mb + r < M && cw + c < N) ((TO *)g.out)[(int64_t)(mb + r) * g.out_row + cw + c] = v;
      }
    }
  }
}

template <typename TO, bool ACT, int BM, int BN, int WM, int WN, int P, int OCC>
hipError_t run_tile(const I8Args &g, hipStream_t s) {
  constexpr int bytes = P * (BM + BN) * kStageBytes;
  auto kern = k_i8_gemm<TO, BM, BN, WM, WN, P, OCC, ACT>;
  static const hipError_t attr =
      hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL(kern, dim3(g.gm * g.gn), dim3(64 * WM * WN), bytes, s, g);
  return hipGetLastError();
}

// bm, bn, waves, ring, workgroups a compute unit; us of a stage and of a tile.
#define I8_TILES(X)                                     \
  X(0, 256, 256, 4, 2, 2, 1, 1.335, 10.86)              \
  X(1, 192, 384, 2, 4, 2, 1, 1.309, 15.45)              \
  X(2, 128, 256, 4, 2, 3, 1, 0.754, 7.23)               \
  X(3, 128, 128, 4, 2, 4, 1, 0.461, 4.42)               \
  X(4, 96, 128, 2, 4, 4, 1, 0.385, 3.82)                \
  X(5, 64, 128, 2, 4, 5, 1, 0.300, 3.30)                \
  X(6, 64, 64, 2, 2, 6, 1, 0.211, 2.29)                 \
  X(7, 32, 64, 2, 2, 6, 2, 0.196, 1.45)
const I8Tile kTiles[] = {
#define I8_INFO(id, bm, bn, wm, wn, p, occ, su, tu) {bm, bn, wm, wn, p, occ, su, tu},
    I8_TILES(I8_INFO)
#undef I8_INFO
};

// Tile times that a launch takes on 256 compute units (as the encoder's planner counts them).
double rounds_of(int64_t wgs, int occ) {
  const double f = (double)wgs / 256.0, full = std::floor(f / occ), rem = f - occ * full;
  double r = full * (occ == 2 ? 1.5 : 1.0);
  if (rem > 0) r += rem <= 1.0 ? 0.85 + 0.15 * rem : 1.0 + 0.5 * (0.5 + 0.5 * (rem - 1.0));
  return r;
}
int pick_tile(int m, int n, int pitch) {
  int best = 0;
  double least = 1e30;
  for (int i = 0; i < (int)(sizeof(kTiles) / sizeof(kTiles[0])); ++i) {
    const I8Tile &t = kTiles[i];
    const int64_t wgs = (int64_t)((m + t.bm - 1) / t.bm) * ((n + t.bn - 1) / t.bn);
    const double us = rounds_of(wgs, t.occ) * (pitch / kStageBytes * t.stage_us + t.tile_us);
    if (us < least) {
      least = us;
      best = i;
    }
  }
  return best;
}

template <typename TO, bool ACT> hipError_t run_many(I8Args g, hipStream_t s) {
  const int id = pick_tile(g.m, g.n, g.pitch);
  g.gm = (g.m + kTiles[id].bm - 1) / kTiles[id].bm;
  g.gn = (g.n + kTiles[id].bn - 1) / kTiles[id].bn;
  // an XCD's 32 tiles at a time as a block: about as many rows of a as of b
  g.gh = 1;
  while (g.gh < g.gm && g.gh * kTiles[id].bm < 6 * kTiles[id].bn) ++g.gh;
  switch (id) {
#define I8_CASE(idv, bm, bn, wm, wn, p, occ, su, tu) \
  case idv: return run_tile<TO, ACT, bm, bn, wm, wn, p, occ>(g, s);
    I8_TILES(I8_CASE)
#undef I8_CASE
  }
  return hipErrorInvalidValue;
}

// ---- many short rows, quantised on the way ------------------------------------------------------
//
// Rows of up to 1024 elements (fp32: 512, by registers) fit LDS as codes, 128 of them at a time: a workgroup reads its rows of x
// once, quantises them into the layout of the products' operand and goes through all of the weight, which the
// L2 holds, 128 rows and 128 bytes of K at a time (a ring of two slots). x is read once and no codes
// are written or read; the stores of a tile drain beneath the products of the next.
// Eight lanes a row: a lane takes every eighth chunk of 8 elements, maxima are three exchanges.
// LDS: nk stages of [128 rows][8 chunks] of codes, two of the weight's, swizzled as the tiles above.
constexpr int kFusedRows = 128, kFusedCols = 128, kFusedStage = kFusedRows * kStageBytes;
int fused_lds(int pitch) { return (pitch / kStageBytes + 2) * kFusedStage; }

template <typename T, typename TO, int NW, int NJ, bool ACT>
__global__ __launch_bounds__(64 * NW, NW == 4 ? 2 : 1) void k_i8_fused(I8Args g) {
  constexpr int CH = kStageBytes / 16, WN = NW / 2, WTN = kFusedCols / WN, TM = 4, TN = WTN / 16;
  constexpr int BR = kFusedCols * CH / 64 / NW;   // copies of a wave a stage
  extern __shared__ u32x4 lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nk = g.pitch / kStageBytes, M = g.m, N = g.n, m0 = blockIdx.x * kFusedRows;
  const uint32_t ring0 = (uint32_t)nk * kFusedStage;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  char *ldsb = (char *)lds;
  float *sa = (float *)(ldsb + ring0 + kFusedStage);   // the rows' scales, until the second slot is used

  uint32_t pb[BR];
  const int8_t *bb = g.b;
  auto aim = [&](int n0) {                        // at the weight rows of a tile
    bb = g.b + (int64_t)n0 * g.pitch;
#pragma unroll
    for (int c = 0; c < BR; ++c) {
      const int q = (c * NW + wave) * 64 + lane, r = q / CH;
      pb[c] = (uint32_t)min(r, N - 1 - n0) * (uint32_t)g.pitch + swz<CH>(r, q % CH) * 16;
    }
  };
  auto copy = [&](int ks, int slot) {
#pragma unroll
    for (int c = 0; c < BR; ++c)
      dma16(bb + ks * kStageBytes, pb[c], lds0 + ring0 + (uint32_t)(slot * kFusedStage + (c * NW + wave) * 1024));
  };
  aim(0);
  copy(0, 0);

  {
    const int l8 = lane & 7, nj = g.pitch / 64;   // chunks of 8 elements a lane
    constexpr int PASSES = kFusedRows / NW / 8;   // of 8 rows a wave
    Eight<T> next[NJ];
    auto fetch = [&](int pass) {
      const int r = (wave * PASSES + pass) * 8 + (lane >> 3);
      const T *row = (const T *)g.x + (int64_t)min(m0 + r, M - 1) * g.x_row;
#pragma unroll
      for (int j = 0; j < NJ; ++j) load8<T>(next[j], row, (j * 8 + l8) * 8, g.k);
    };
    fetch(0);
#pragma unroll 1
    for (int pass = 0; pass < PASSES; ++pass) {
      const int r = (wave * PASSES + pass) * 8 + (lane >> 3);
      Eight<T> y[NJ];
      Top<T> top;
#pragma unroll
      for (int j = 0; j < NJ; ++j) y[j] = next[j];
      if (pass + 1 < PASSES) fetch(pass + 1);     // in flight meanwhile
#pragma unroll
      for (int j = 0; j < NJ; ++j) top.take(y[j]);
      const Scale sc(lanes_top<4>(top.bits()));
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int e = (j * 8 + l8) * 8, c = (e >> 4) & 7;
        if (j < nj) *(u32x2 *)(ldsb + (e >> 7) * kFusedStage + (r * CH + swz<CH>(r, c)) * 16 + (e & 8)) = sc.codes(y[j]);
      }
      if (l8 == 0) sa[r] = row_scale(sc.stored());
    }
  }

  const int wm = wave / WN, wn = wave % WN, lc = lane & 15, rg = lane >> 4;
  uint32_t oa[2], ob[2];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    oa[kk] = (uint32_t)((wm * 64 + lc) * CH + swz<CH>(lc, 4 * kk + rg)) * 16u;
    ob[kk] = ring0 + (uint32_t)((wn * WTN + lc) * CH + swz<CH>(lc, 4 * kk + rg)) * 16u;
  }
  float sr[TM];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < TM; ++i) sr[i] = sa[wm * 64 + 16 * i + lc];
  __syncthreads();
  const bool vec = (((uintptr_t)g.out | (uint64_t)(g.out_row * (int64_t)sizeof(TO))) & 15) == 0;   // uniform
  int slot = 0;
  bool landed = false;
#pragma unroll 1
  for (int n0 = 0; n0 < N; n0 += kFusedCols) {
    i32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
#pragma unroll 1
    for (int ks = 0; ks < nk; ++ks) {
      if (!landed) wait_vm<0>();
      landed = false;
      __syncthreads();                            // the stage is whole (first: the codes), and the slot beside it read
      if (ks + 1 < nk) {
        copy(ks + 1, slot ^ 1);
      } else if (n0 + kFusedCols < N) {
        aim(n0 + kFusedCols);
        copy(0, slot ^ 1);
      }
      const char *pa = ldsb + ks * kFusedStage, *pw = ldsb + slot * kFusedStage;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        i32x4 fa[TM], fb[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[i] = *(const i32x4 *)(pa + oa[kk] + i * 16 * kStageBytes);
#pragma unroll
        for (int j = 0; j < TN; ++j) fb[j] = *(const i32x4 *)(pw + ob[kk] + j * 16 * kStageBytes);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) mfma_i8(acc[i][j], fb[j], fa[i]);
      }
      slot ^= 1;
    }
    // row mw + 16 i + lc, columns cw + 16 j + 4 rg .. + 3
    const int mw = m0 + wm * 64, cw = n0 + wn * WTN;
    f32x4 tc[TN], bs[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = min(cw + 16 * j + 4 * rg + e, N - 1);
        tc[j][e] = col_scale(g.sb[n]);
        bs[j][e] = g.bias ? to_f32(((const TO *)g.bias)[n]) : 0.f;
      }
    wait_vm<0>();                                 // the next stage's copy: before the stores, not behind them
    landed = true;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int m = mw + 16 * i + lc;
      TO *out = (TO *)g.out + (int64_t)m * g.out_row + cw;
#pragma unroll
      for (int j = 0; j < TN; j += 2) {
        float z[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) z[u][e] = finish<ACT>(acc[i][j + u][e], sr[i], tc[j + u][e], bs[j + u][e]);
        if (vec && cw + WTN <= N) {               // uniform
          if constexpr (sizeof(TO) == 2) {
            // eight columns a lane: of blocks j and j + 1 the 16-lane rows trade places
            const u32x2 x = __builtin_bit_cast(u32x2, bf16x4{(bf16)z[0][0], (bf16)z[0][1], (bf16)z[0][2], (bf16)z[0][3]});
            const u32x2 y = __builtin_bit_cast(u32x2, bf16x4{(bf16)z[1][0], (bf16)z[1][1], (bf16)z[1][2], (bf16)z[1][3]});
            const auto a = __builtin_amdgcn_permlane16_swap(x[0], y[0], false, false);
            const auto b = __builtin_amdgcn_permlane16_swap(x[1], y[1], false, false);
            if (m < M) *(u32x4 *)(out + 16 * (j + (rg & 1)) + 8 * (rg >> 1)) = u32x4{a[0], b[0], a[1], b[1]};
          } else {
#pragma unroll
            for (int u = 0; u < 2; ++u)
              if (m < M) *(f32x4 *)(out + 16 * (j + u) + 4 * rg) = f32x4{z[u][0], z[u][1], z[u][2], z[u][3]};
          }
        } else {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int c = 16 * (j + u) + 4 * rg + e;
              if (m < M && cw + c < N) out[c] = from_f32<TO>(z[u][e]);
            }
        }
      }
    }
  }
}

template <typename T, typename TO, bool ACT> hipError_t run_fused(const I8Args &g, hipStream_t s) {
  const int bytes = fused_lds(g.pitch);
  const bool two = bytes <= 80 * 1024;            // two workgroups a compute unit
  auto kern = two ? k_i8_fused<T, TO, 4, 6, ACT> : k_i8_fused<T, TO, 8, 8, ACT>;
  if constexpr (sizeof(T) == 2)
    if (g.pitch > 512) kern = k_i8_fused<T, TO, 8, 16, ACT>;
  if (bytes > 65536) {
    const hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3((g.m + kFusedRows - 1) / kFusedRows), dim3(two ? 256 : 512), bytes, s, g);
  return hipGetLastError();
}
// How a product is done, by its sizes alone: up to 16 rows and many short rows in one launch from rows as they are,
// others quantised by a launch of their own.
enum Way { FEW, FUSED, TILES };
Way way_of(int x_type, int m, int pitch) {
  if (takes_few(m, pitch)) return FEW;
  return x_type != MTE_I8_CODES && m >= 8192 && pitch <= (x_type == MTE_BF16 ? 1024 : 512) ? FUSED : TILES;
}

template <typename T, typename TO, bool ACT> hipError_t run_rows(const I8Args &g, Way way, hipStream_t s) {
  return way == FEW ? run_few<T, TO, ACT>(g, s) : run_fused<T, TO, ACT>(g, s);
}
template <typename TO, bool ACT> hipError_t run(const I8Args &g, Way way, int x_type, hipStream_t s) {
  if (way == TILES) return run_many<TO, ACT>(g, s);
  if (x_type == MTE_I8_CODES) return run_few<int8_t, TO, ACT>(g, s);
  return x_type == MTE_BF16 ? run_rows<bf16, TO, ACT>(g, way, s) : run_rows<float, TO, ACT>(g, way, s);
}

}  // namespace

// Codes and scales of rows that the call quantises into memory.
int64_t i8_workspace(int x_type, int m, int, int k) {
  const int64_t pitch = i8_pitch(k);
  return x_type == MTE_I8_CODES || way_of(x_type, m, (int)pitch) != TILES ? 0 : m * pitch + (int64_t)m * 4;
}

hipError_t launch_i8_linear(I8Args a, int x_type, int dtype, void *ws, hipStream_t s) {
  const Way way = way_of(x_type, a.m, a.pitch);
  if (way == TILES && x_type != MTE_I8_CODES) {
    int8_t *codes = (int8_t *)ws;
    float *scales = (float *)(codes + (int64_t)a.m * a.pitch);
    const hipError_t e = launch_i8_quantize(QuantArgs{a.x, codes, scales, a.x_row, a.m, a.k, a.pitch}, x_type, s);
    if (e != hipSuccess) return e;
    a.a = codes;
    a.sa = scales;
  }
  if (dtype == MTE_BF16) return a.act ? run<bf16, true>(a, way, x_type, s) : run<bf16, false>(a, way, x_type, s);
  return a.act ? run<float, true>(a, way, x_type, s) : run<float, false>(a, way, x_type, s);
}

}  // namespace mte
