// Products of 8-bit rows: y = act(s_i t_j sum_k a_ik b_jk + bias_j).
//
// The matrix cores' 8-bit integer form (16x16x64, int32 sums: exact in any order) has twice the
// rate of 16-bit floating point for the same bytes of operands. Codes are rows of a multiple of
// 128 bytes, so that a K stage is 128 bytes of every row and there is no ragged end of K.
// C^T = B A^T: a lane then holds four consecutive columns of one row of the result.
#include <algorithm>
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

// ---- up to 32 rows ------------------------------------------------------------------------------
//
// Bound by the bytes of the weight, or by latency. A workgroup of 16 waves takes blocks of 16 weight rows in
// turn; its waves share K, 128 bytes of each row at a time, straight from memory to the operands (the next
// block's loads are in flight meanwhile), and add up through LDS. The rows of a are few enough to lie in LDS
// whole; every workgroup quantises them for itself, once, while its first weights arrive: a launch less than with
// codes through memory (1 x 2048 x 2048: 8.4 us replayed, 14.2 called; so 5.1 and 9.7). 16 x 2048 x 12288: 10.7 us, 2.4
// TB/s, of which launch, quantising and the last sums are about 5; 4 x 6144 x 12288: 20 us, 3.7 TB/s. Three blocks of weights
// ahead instead of one change nothing.
// LDS: rows of codes 64 bytes further apart than they are long, so that an operand's 16 rows of 64 bytes
// fill the banks.
constexpr int kFewWaves = 16, kFewRows = 32, kFewThreads = 64 * kFewWaves, kFewLds = 95 * 1024;
int few_lds(int m, int pitch) { return m * (pitch + 64); }

// MT: blocks of 16 rows of a.
template <typename T, typename TO, bool ACT, int MT>
__global__ __launch_bounds__(kFewThreads) void k_i8_few(I8Args g) {
  constexpr int AHEAD = 2;                        // blocks of 128 bytes of K a wave and weight row, ahead
  __shared__ i32x4 part[2][kFewWaves][MT][64];
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
    // 1024, 512, .. 64 threads a row; MT 2: 32
    const int per = MT == 2 ? 32 : kFewThreads >> (g.m > 8 ? 4 : g.m > 4 ? 3 : g.m > 2 ? 2 : g.m > 1 ? 1 : 0);
    const int r = tid / per, c0 = tid % per;
    constexpr int KEPT = 4 * MT;
    RowChunks<T> row;
    Eight<T> y[KEPT];
    Top<T> top;
    row.open((const T *)g.x + (int64_t)min(r, g.m - 1) * g.x_row, g.k);
#pragma unroll
    for (int j = 0; j < KEPT; ++j) row.load(y[j], (c0 + j * per) * 8);
#pragma unroll
    for (int j = 0; j < KEPT; ++j) {
      row.keep(y[j], (c0 + j * per) * 8);
      top.take(y[j]);
    }
    for (int c = c0 + KEPT * per; c * 8 < g.k; c += per) {
      Eight<T> z;
      row.load(z, c * 8);
      row.keep(z, c * 8);
      top.take(z);
    }
    const uint32_t t = lanes_top<MT == 2 ? 16 : 32>(top.bits());   // a wave, or half of one, is within a row
    if (lane % (MT == 2 ? 32 : 64) == 0) atomicMax(&tops[r], t);
    __syncthreads();
    const Scale sc(tops[r]);
    if (r < g.m) {
      char *to = codes + r * row_bytes;
#pragma unroll
      for (int j = 0; j < KEPT; ++j)
        if ((c0 + j * per) * 8 < g.pitch) *(u32x2 *)(to + (c0 + j * per) * 8) = sc.codes(y[j]);
      for (int c = c0 + KEPT * per; c * 8 < g.pitch; c += per) {
        Eight<T> z;
        row.load(z, c * 8);
        row.keep(z, c * 8);
        *(u32x2 *)(to + c * 8) = sc.codes(z);
      }
      if (c0 == 0) sa[r] = row_scale(sc.stored());
    }
  }
  __syncthreads();

  const char *ap[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) ap[t] = codes + min(16 * t + lr, g.m - 1) * row_bytes + lk;
  int buf = 0;
  for (int nb = blockIdx.x; nb < blocks; nb += gridDim.x, buf ^= 1) {
    i32x4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = i32x4{0, 0, 0, 0};
    auto add = [&](const i32x4 &x, const i32x4 &y, int k) {
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        mfma_i8(acc[t], x, *(const i32x4 *)(ap[t] + k));
        mfma_i8(acc[t], y, *(const i32x4 *)(ap[t] + k + 64));
      }
    };
#pragma unroll
    for (int b = 0; b < AHEAD; ++b) {
      const int k = (wave + b * kFewWaves) * 128;
      if (k < g.pitch) add(w[2 * b], w[2 * b + 1], k);
    }
    if (g.pitch > AHEAD * kFewWaves * 128) {      // long rows: the rest
      const int8_t *bp = g.b + (int64_t)min(nb * 16 + lr, g.n - 1) * g.pitch + lk;
#pragma unroll 2
      for (int k = (wave + AHEAD * kFewWaves) * 128; k < g.pitch; k += kFewWaves * 128)
        add(*(const i32x4 *)(bp + k), *(const i32x4 *)(bp + k + 64), k);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) part[buf][wave][t][lane] = acc[t];
    if (nb + (int)gridDim.x < blocks) fetch(nb + gridDim.x);
    __syncthreads();
    if (tid < 256 * MT) {                         // register e of lane l of every part: row l % 16, column 4 (l / 16) + e
      const int l = tid >> 2 & 63, e = tid & 3, m = (tid >> 8) * 16 + (l & 15), n = nb * 16 + 4 * (l >> 4) + e;
      int sum = 0;
#pragma unroll
      for (int v = 0; v < kFewWaves; ++v) sum += ((const int *)&part[buf][v][0][0])[tid];
      if (m < g.m && n < g.n)
        ((TO *)g.out)[(int64_t)m * g.out_row + n] =
            from_f32<TO>(finish<ACT>(sum, sa[m], col_scale(g.sb[n]), g.bias ? to_f32(((const TO *)g.bias)[n]) : 0.f));
    }
  }
}

template <typename T, typename TO, bool ACT, int MT> hipError_t launch_few(const I8Args &g, hipStream_t s) {
  const int blocks = (g.n + 15) / 16;
  auto kern = k_i8_few<T, TO, ACT, MT>;
  static const hipError_t attr = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, kFewLds);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL(kern, dim3(blocks < 256 ? blocks : 256), dim3(kFewThreads), few_lds(g.m, g.pitch), s, g);
  return hipGetLastError();
}
template <typename T, typename TO, bool ACT> hipError_t run_few(const I8Args &g, hipStream_t s) {
  return g.m <= 16 ? launch_few<T, TO, ACT, 1>(g, s) : launch_few<T, TO, ACT, 2>(g, s);
}
// 17 to 32 rows: where every workgroup has one block of columns, and rows that it quantises itself are short,
// since all of them repeat that. us replayed / called, against tiles: 17 x 640 x 2048 6.7 / 8.6, 7.4 / 14.4; 32 x 640 x
// 2048 7.3 / 8.8, 7.7 / 14.5; 17 x 2048 x 4096 10.7 / 10.0, 10.8 / 14.4; of codes 32 x 2048 x 2048 5.3, 6.1. The line is drawn
// for the call, which gains 3 to 6 everywhere within it; replayed, the longest rows lose near it: 32 x 2048 x 2048
// 11.9 / 11.5, 11.1 / 14.4; 32 x 2048 x 4096 12.2 / 11.6, 11.1 / 14.5 (fp32 rows 11.7 against 9.8, the most). Beyond it
// the call gains nothing: 32 x 2048 x 8192 13.6 / 13.5, 10.9 / 13.7; 32 x 2944 x 2048 16.2 / 15.9, 13.3 / 13.8.
bool takes_few(int m, int pitch, int n, bool codes) {
  if (m > kFewRows || few_lds(m, pitch) > kFewLds) return false;
  return m <= 16 || (n <= 16 * 256 && (codes || pitch <= 2048));
}

// ---- many rows ----------------------------------------------------------------------------------
//
// A workgroup takes a BM x BN tile of the result, a wave (BM / WM) x (BN / WN) of it. K goes by in stages of
// 128 bytes a row through a ring of P slots that LDS-direct copies fill (as in the encoder's
// projections, see gemm_kernel.h: swizzle, one barrier a stage, fragments of the longer side of a wave's tile used by
// one row of products each and then replaced, those of the shorter side double-buffered). Rows past the
// last are repeats of it and are not stored.
// Bound by the matrix cores where K is long, else by prologue and epilogue, which nothing overlaps in the larger tiles
// (5120 x 2048 x 12288: busy 51 of 131 us; SiLU, two quarter-rate instructions an element, makes them 139).
// The result goes through LDS, 16 rows of a wave at a time, so that it is stored in whole lines (at any
// alignment of an element: the hardware takes it).
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
  constexpr int PITCH = WTN * (int)sizeof(TO) + 16;   // 16 rows on 16 sets of 4 banks
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
  const bool whole = cw + WTN <= N;               // uniform
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
    if (whole) {
#pragma unroll
      for (int x = 0; x < 16 * CPR / 64; ++x) {
        const int q = x * 64 + lane, r = q / CPR, c = q % CPR;
        const u32x4 v = *(const u32x4 *)(box + r * PITCH + c * 16);
        if (mb + r < M) *(u32x4e *)((char *)g.out + ((int64_t)(mb + r) * g.out_row + cw) * (int)sizeof(TO) + c * 16) = v;
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

// bm, bn, waves, ring, workgroups a compute unit; us of a stage and of a tile: least squares over 30 products of 5
// to 65536 rows, 128 to 6144 deep and 640 to 12288 wide (10 to 18% rms off; the tile they choose is 0.7% slower
// than the fastest on average, 6% at most). Smaller tiles come two to a compute unit, so that one's products
// hide the other's stores; the largest read the fewest bytes from LDS for a product (5120 x 2048 x 12288 in 131 us, 1.97 P
// operations/s, 4096 cubed in 61, 2.25; a library's 147 and 65 without scales).
#define I8_TILES(X)                                     \
  X(0, 256, 256, 4, 2, 2, 1, 0.957, 12.62)              \
  X(1, 160, 256, 2, 4, 3, 1, 0.714, 8.31)               \
  X(2, 128, 256, 4, 2, 3, 1, 0.561, 7.97)               \
  X(3, 192, 128, 2, 2, 2, 2, 0.637, 6.72)               \
  X(4, 128, 128, 2, 2, 2, 2, 0.576, 4.39)               \
  X(5, 96, 128, 2, 2, 2, 2, 0.488, 3.69)                \
  X(6, 64, 128, 2, 2, 3, 2, 0.318, 2.78)                \
  X(7, 64, 64, 2, 2, 4, 2, 0.204, 1.74)                 \
  X(8, 32, 64, 2, 2, 6, 2, 0.181, 1.31)                 \
  X(9, 128, 128, 4, 2, 4, 1, 0.373, 4.19)
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

template <typename TO, bool ACT> hipError_t run_tiles(const I8Args &g, int id, hipStream_t s) {
  switch (id) {
#define I8_CASE(idv, bm, bn, wm, wn, p, occ, su, tu) \
  case idv: return run_tile<TO, ACT, bm, bn, wm, wn, p, occ>(g, s);
    I8_TILES(I8_CASE)
#undef I8_CASE
  }
  return hipErrorInvalidValue;
}
template <typename TO, bool ACT> hipError_t run_many(const I8Args &all, hipStream_t s) {
  const int id = pick_tile(all.m, all.n, all.pitch), bm = kTiles[id].bm, bn = kTiles[id].bn;
  // in launches of kMostGroups tiles: columns, and rows of them
  const int64_t cols = std::min<int64_t>((all.n + bn - 1) / bn, kMostGroups), rows = kMostGroups / cols;
  for (int64_t n0 = 0; n0 < all.n; n0 += cols * bn)
    for (int64_t m0 = 0; m0 < all.m; m0 += rows * bm) {
      I8Args g = all;
      g.m = (int)std::min(all.m - m0, rows * bm);
      g.n = (int)std::min(all.n - n0, cols * bn);
      g.a += m0 * g.pitch;
      g.sa += m0;
      g.b += n0 * g.pitch;
      g.sb += n0;
      if (g.bias) g.bias = (const TO *)g.bias + n0;
      g.out = (TO *)g.out + m0 * g.out_row + n0;
      g.gm = (g.m + bm - 1) / bm;
      g.gn = (g.n + bn - 1) / bn;
      // an XCD's 32 tiles at a time as a block: about as many rows of a as of b
      g.gh = 1;
      while (g.gh < g.gm && g.gh * bm < 6 * bn) ++g.gh;
      const hipError_t e = run_tiles<TO, ACT>(g, id, s);
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

// ---- many short rows, quantised on the way ------------------------------------------------------
//
// Rows of up to 384 elements: a workgroup of four waves reads 128 of them once, quantises them through LDS into the
// operands of its products, 64 rows a wave, which stay in registers, and goes through all of the weight, which the
// L2 holds, 128 rows and 128 bytes of K at a time. x is read once, and no codes are written or read.
// Eight lanes a row: a lane takes every eighth chunk of 8 elements, maxima are three exchanges.
// LDS: a ring of five stages of the weight, four ahead of the products; the first three hold the codes
// before. All copies are waited for before a tile's stores and not after: the stores then
// drain beneath the next tile's products. They bypass the caches, which hold less than such a result (65536 x 320
// x 640 38 us against 42). Two workgroups a compute unit.
// Bound by the rows in and out, one after the other: all workgroups quantise first (about 10 us) and store then (126
// MB in 38 us, 3.3 TB/s; codes through memory 62). From 32768 rows on: a workgroup alone takes 25 us (32768 x 320 x
// 320 the same 28 either way, 16384 x 320 x 640 32 against 21). With the codes in LDS instead of registers, or rows of
// up to 1024 that way, it was slower than through memory from 640 elements on (65536 x 640 x 640: 96 against 82).
constexpr int kFusedRows = 128, kFusedCols = 128, kFusedStage = kFusedRows * kStageBytes, kFusedRing = 5;

template <typename T, typename TO, int NK, bool ACT>
__global__ __launch_bounds__(256, 2) void k_i8_fused(I8Args g) {
  constexpr int CH = kStageBytes / 16, TM = 4, TN = 4, NJ = 2 * NK, PITCH = NK * kStageBytes;
  static_assert(NK <= 3, "the codes' slots");
  extern __shared__ u32x4 lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int M = g.m, N = g.n, m0 = blockIdx.x * kFusedRows;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  char *ldsb = (char *)lds;

  // copy c of this wave: 8 rows of the stage
  uint32_t pr[4], pc[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int q = (c * 4 + wave) * 64 + lane;
    pr[c] = q / CH;
    pc[c] = swz<CH>(q / CH, q % CH) * 16;
  }
  // stage ks of the columns from n0 on into a slot
  auto copy = [&](int n0, int ks, int slot) {
    const int8_t *bb = g.b + (int64_t)n0 * PITCH + ks * kStageBytes;
    const uint32_t last = (uint32_t)min(N - 1 - n0, kFusedCols - 1);
#pragma unroll
    for (int c = 0; c < 4; ++c)
      dma16(bb, min(pr[c], last) * (uint32_t)PITCH + pc[c], lds0 + (uint32_t)(slot * kFusedStage + (c * 4 + wave) * 1024));
  };
  auto copy_at = [&](int n0, int t, int slot) {   // t stages after the first of n0
    const int n = n0 + t / NK * kFusedCols;
    if (n < N) copy(n, t % NK, slot);
  };
  copy_at(0, 0, 3);
  copy_at(0, 1, 4);

  float rowscale[4];                              // of the rows this lane quantises with its seven neighbours
  {
    const int l8 = lane & 7;
    constexpr int PASSES = kFusedRows / 4 / 8;    // of 8 rows a wave
    Eight<T> next[NJ];
    RowChunks<T> row, ahead;
    auto fetch = [&](int pass) {
      const int r = (wave * PASSES + pass) * 8 + (lane >> 3);
      ahead.open((const T *)g.x + (int64_t)min(m0 + r, M - 1) * g.x_row, g.k);
#pragma unroll
      for (int j = 0; j < NJ; ++j) ahead.load(next[j], (j * 8 + l8) * 8);
    };
    fetch(0);
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
      const int r = (wave * PASSES + pass) * 8 + (lane >> 3);
      Eight<T> y[NJ];
      Top<T> top;
#pragma unroll
      for (int j = 0; j < NJ; ++j) y[j] = next[j];
      row = ahead;
      if (pass + 1 < PASSES) fetch(pass + 1);     // in flight meanwhile
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        row.keep(y[j], (j * 8 + l8) * 8);
        top.take(y[j]);
      }
      const Scale sc(lanes_top<4>(top.bits()));
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int e = (j * 8 + l8) * 8, c = (e >> 4) & 7;
        *(u32x2 *)(ldsb + (e >> 7) * kFusedStage + (r * CH + swz<CH>(r, c)) * 16 + (e & 8)) = sc.codes(y[j]);
      }
      rowscale[pass] = row_scale(sc.stored());
    }
  }
  __syncthreads();
  const int wm = wave >> 1, wn = wave & 1, lc = lane & 15, rg = lane >> 4;
  i32x4 fa[2 * NK][TM];
#pragma unroll
  for (int k = 0; k < 2 * NK; ++k)
#pragma unroll
    for (int i = 0; i < TM; ++i)
      fa[k][i] = *(const i32x4 *)(ldsb + (k >> 1) * kFusedStage +
                                  ((wm * 64 + 16 * i + lc) * CH + swz<CH>(lc, 4 * (k & 1) + rg)) * 16);
  __syncthreads();                                // the codes are read: their slots are free
  float *sa = (float *)ldsb;
  if ((lane & 7) == 0) {
#pragma unroll
    for (int pass = 0; pass < 4; ++pass) sa[(wave * 4 + pass) * 8 + (lane >> 3)] = rowscale[pass];
  }
  __syncthreads();
  float sr[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) sr[i] = sa[wm * 64 + 16 * i + lc];
  __syncthreads();
  copy_at(0, 2, 0);
  copy_at(0, 3, 1);
  uint32_t ob[2];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) ob[kk] = (uint32_t)((wn * 64 + lc) * CH + swz<CH>(lc, 4 * kk + rg)) * 16u;
  int slot = 3;
  wait_vm<0>();
#pragma unroll 1
  for (int n0 = 0; n0 < N; n0 += kFusedCols) {
    const int cw = n0 + wn * 64;
    i32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int ks = 0; ks < NK; ++ks) {
      __syncthreads();                            // this stage is whole (waited for below), the one before it read
      copy_at(n0, ks + 4, slot == 0 ? kFusedRing - 1 : slot - 1);
      const char *pw = ldsb + slot * kFusedStage;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        i32x4 fb[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) fb[j] = *(const i32x4 *)(pw + ob[kk] + j * 16 * kStageBytes);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) mfma_i8(acc[i][j], fb[j], fa[2 * ks + kk][i]);
      }
      slot = slot == kFusedRing - 1 ? 0 : slot + 1;
    }
    wait_vm<0>();
    // row m0 + 64 wm + 16 i + lc (past the last row: the last one again), columns cw + 16 j + 4 rg .. + 3
#pragma unroll
    for (int j = 0; j < TN; j += 2) {
      f32x4 tc[2], bs[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int n = min(cw + 16 * (j + u) + 4 * rg + e, N - 1);
          tc[u][e] = col_scale(g.sb[n]);
          bs[u][e] = g.bias ? to_f32(((const TO *)g.bias)[n]) : 0.f;
        }
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        TO *out = (TO *)g.out + (int64_t)min(m0 + wm * 64 + 16 * i + lc, M - 1) * g.out_row + cw;
        float z[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) z[u][e] = finish<ACT>(acc[i][j + u][e], sr[i], tc[u][e], bs[u][e]);
        if (cw + 64 <= N) {                       // uniform
          if constexpr (sizeof(TO) == 2) {
            // eight columns a lane: of blocks j and j + 1 the 16-lane rows trade places
            const u32x2 x = __builtin_bit_cast(u32x2, bf16x4{(bf16)z[0][0], (bf16)z[0][1], (bf16)z[0][2], (bf16)z[0][3]});
            const u32x2 y = __builtin_bit_cast(u32x2, bf16x4{(bf16)z[1][0], (bf16)z[1][1], (bf16)z[1][2], (bf16)z[1][3]});
            const auto a = __builtin_amdgcn_permlane16_swap(x[0], y[0], false, false);
            const auto b = __builtin_amdgcn_permlane16_swap(x[1], y[1], false, false);
            __builtin_nontemporal_store(u32x4{a[0], b[0], a[1], b[1]}, (u32x4e *)(out + 16 * (j + (rg & 1)) + 8 * (rg >> 1)));
          } else {
#pragma unroll
            for (int u = 0; u < 2; ++u)
              __builtin_nontemporal_store(f32x4{z[u][0], z[u][1], z[u][2], z[u][3]}, (f32x4u *)(out + 16 * (j + u) + 4 * rg));
          }
        } else {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int c = 16 * (j + u) + 4 * rg + e;
              if (cw + c < N) out[c] = from_f32<TO>(z[u][e]);
            }
        }
      }
    }
  }
}

template <typename T, typename TO, bool ACT> hipError_t run_fused(const I8Args &g, hipStream_t s) {
  constexpr int bytes = kFusedRing * kFusedStage;
  auto kern = g.pitch == 384 ? k_i8_fused<T, TO, 3, ACT> : g.pitch == 256 ? k_i8_fused<T, TO, 2, ACT> : k_i8_fused<T, TO, 1, ACT>;
  const hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((g.m + kFusedRows - 1) / kFusedRows), dim3(256), bytes, s, g);
  return hipGetLastError();
}

// How a product is done, by its sizes alone: few rows and many short rows in one launch from rows as they are,
// others quantised by a launch of their own.
enum Way { FEW, FUSED, TILES };
Way way_of(int x_type, int m, int n, int k, int pitch) {
  const bool whole = x_type == MTE_I8_CODES || k >= 8;   // (RowChunks)
  if (whole && takes_few(m, pitch, n, x_type == MTE_I8_CODES)) return FEW;
  return whole && x_type != MTE_I8_CODES && m >= 32768 && pitch <= 384 ? FUSED : TILES;
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
int64_t i8_workspace(int x_type, int m, int n, int k) {
  const int64_t pitch = i8_pitch(k);
  return x_type == MTE_I8_CODES || way_of(x_type, m, n, k, (int)pitch) != TILES ? 0 : m * pitch + (int64_t)m * 4;
}

hipError_t launch_i8_linear(I8Args a, int x_type, int dtype, void *ws, hipStream_t s) {
  const Way way = way_of(x_type, a.m, a.n, a.k, a.pitch);
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
