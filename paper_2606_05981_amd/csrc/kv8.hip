// Rows into and out of the 8-bit key/value cache (layout: include/mte_cond.h).
//
// A workgroup serves one block of 32 tokens and one kv head, keys and values: a
// thread holds 16 consecutive d of one token. The maximum of the block's new rows
// fixes the scale, codes go out 16 bytes a thread; values are turned through LDS
// ([d][32 tokens], the tokens in the matrix core's order). A block that holds older
// tokens is read, merged and written whole (8 KB a head of 128).
// Long appends and reads are bound by the rows and codes, each moved once, and by all workgroups
// being resident at once, so that reading, scaling and writing hardly overlap (16 x 320 tokens of 8
// heads of 128: append 11.0 us, read 9.6 us, 2.9 and 3.3 TB/s); single tokens by the chain of length, table,
// block, maximum, codes (64 sequences: append 6.3 us, read 4.6 us).
#include <algorithm>

#include "../../include/mte.h"
#include "cond_device.h"

namespace mte {

namespace {

constexpr int kThreads = 256;

// Position of token t of a block in a row of the value codes.
__device__ __forceinline__ int v_pos(int t) { return 16 * ((t >> 2) & 1) + 8 * (t >> 4) + 4 * ((t >> 3) & 1) + (t & 3); }

// LDS row of the 32 value codes of one d: 16-byte aligned, and 16 rows (a thread's) and 4 tokens on lie in
// banks of their own (without the last term all pieces of d meet in one: 2 of an append's 12.7 us).
__device__ __forceinline__ int v_row(int d) { return d * 48 + (d >> 4) * 32; }
constexpr int v_bytes(int D) { return D * 48 + (D >> 4) * 32; }

// Exponent of the smallest 2^e >= 2^-126 with amax <= 448 * 2^e (448 = 0.875 * 2^9, amax =
// f * 2^x with f in [0.5, 1)); infinities take the largest, 2^120.
__device__ __forceinline__ int scale_exp(float amax) {
  if (!(amax > 0.f)) return -126;
  if (amax > 3.0e38f) return 120;
  int x = 0;
  const float f = frexpf(amax, &x);
  return max(f <= 0.875f ? x - 9 : x - 8, -126);
}

// Four e4m3 codes of x / 2^e: nearest, ties to even (v_cvt_pk_fp8_f32), NaN kept, magnitudes at
// most `top`.
__device__ __forceinline__ uint32_t code4(const float *x, int e, float top) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = ldexpf(x[i], -e);
    y[i] = fabsf(y[i]) > top ? copysignf(top, y[i]) : y[i];
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
}
__device__ __forceinline__ void value4(uint32_t w, float *x) {
  x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
  x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
  x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
  x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
}

// 16 elements of a row as loaded, and as floats.
template <typename T> struct Row16 { u32x4 w[sizeof(T)]; };
template <typename T> __device__ __forceinline__ void load16(const T *p, Row16<T> &r) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T); ++i) r.w[i] = ((const u32x4 *)p)[i];
}
template <typename T> __device__ __forceinline__ void floats16(const Row16<T> &r, float *x) {
  T t[16];
  __builtin_memcpy(t, &r, sizeof(t));
#pragma unroll
  for (int e = 0; e < 16; ++e) x[e] = to_f32(t[e]);
}
__device__ __forceinline__ void store16(float *p, const float *x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) ((f32x4 *)p)[i] = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
}
__device__ __forceinline__ void store16(bf16 *p, const float *x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    bf16x8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (bf16)x[8 * i + e];
    ((bf16x8 *)p)[i] = v;
  }
}

// The block a workgroup serves: the j-th that the last `n` of its sequence's tokens touch.
struct Where { int start, kv, b; int64_t at; bool ok; };
__device__ __forceinline__ Where block_of(const Kv8View &c, const CondSeq &sq, int j, int g) {
  Where w;
  w.kv = max(c.kv_lens[sq.k0], 0);
  w.start = w.kv - sq.q_len;
  // (the first block of rows that start before the first token is block 0's left neighbour)
  w.b = (w.start >> 5) + j;
  int id = -1;
  if (w.b >= 0 && w.b < c.width && w.b * 32 < w.kv) id = c.table[(int64_t)sq.k0 * c.table_row + w.b];
  w.ok = id >= 0 && id < c.n_blocks;
  w.at = (int64_t)(w.ok ? id : 0) * c.hkv + g;
  return w;
}

// Threads: tensor x token x piece of 16 d. D = 128: 8 pieces a token, keys then values in
// turn; D = 64: 4 pieces, keys in the first 128 threads, values in the others.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void k_kv8_append(Kv8RowsArgs a) {
  constexpr int PC = D / 16;
  constexpr int NT = D == 128 ? 2 : 1;              // tensors a thread serves
  __shared__ __attribute__((aligned(16))) uint8_t sv[v_bytes(D)];
  __shared__ float smax[2][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, blockIdx.x)];
  const int g = blockIdx.y;
  const Where w = block_of(a.c, sq, (int)blockIdx.x - sq.tile0, g);
  // the whole workgroup: a sequence shorter than its new rows, or longer than its table, is not written
  if (w.start < 0 || w.kv > (int64_t)a.c.width * 32) return;
  const int sub = tid % (32 * PC), tok = sub / PC, pc = sub % PC;
  const int first = D == 128 ? 0 : tid / (32 * PC); // tensor of the thread (D = 64)
  const int pos = w.b * 32 + tok;                   // token of the sequence
  const bool fresh = pos >= w.start && pos < w.kv, kept = pos < w.start;
  const bool any_kept = w.b * 32 < w.start;
  // All that is read is in flight at once: the rows, which do not wait for the table, then the block.
  Row16<T> raw[NT] = {};
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int ten = D == 128 ? t : first;
    if (fresh) {
      const int64_t row = sq.q0 + (pos - w.start);
      if (ten == 0) load16((const T *)a.k + row * a.k_row + (int64_t)g * a.k_head + pc * 16, raw[t]);
      else load16((const T *)a.v + row * a.v_row + (int64_t)g * a.v_head + pc * 16, raw[t]);
    }
  }
  if (!w.ok) return;                                // the whole workgroup
  uint8_t *kc = a.c.k_codes + w.at * (32 * D), *vc = a.c.v_codes + w.at * (32 * D);
  const bool turn = any_kept && (D == 128 || first == 1);
  constexpr int VT = D == 128 ? 256 : 128;          // threads that read the block's value codes, 16 bytes each
  const int vi = D == 128 ? tid : tid - 128;
  static_assert(32 * D / 16 == VT, "one chunk a thread");
  u32x4 k_old{0, 0, 0, 0}, v_old{0, 0, 0, 0};
  float s_old[2] = {0.f, 0.f};
  if (any_kept) {                                   // workgroup-uniform
    s_old[0] = a.c.scales[w.at * 2];
    s_old[1] = a.c.scales[w.at * 2 + 1];
    if (kept && (D == 128 || first == 0)) k_old = *(const u32x4 *)(kc + (pc * 32 + tok) * 16);
    if (turn) v_old = ((const u32x4 *)vc)[vi];
  }
  float x[NT][16], mx[2] = {0.f, 0.f};
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    floats16(raw[t], x[t]);
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) m = fmaxf(m, fabsf(x[t][e]));
    if (D == 128) mx[t] = m;
    else mx[first] = m;
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) mx[t] = warp_max_xor(mx[t], s);
    if (lane == 0) smax[t][wave] = mx[t];
  }
  if (turn) *(u32x4 *)(sv + v_row(vi >> 1) + (vi & 1) * 16) = v_old;   // [d][pos]
  __syncthreads();
  int e_new[2], e_old[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    e_new[t] = scale_exp(fmaxf(fmaxf(smax[t][0], smax[t][1]), fmaxf(smax[t][2], smax[t][3])));
    e_old[t] = e_new[t];
    if (any_kept) {
      e_old[t] = (int)((__float_as_uint(s_old[t]) >> 23) & 0xFF) - 127;
      e_new[t] = max(e_new[t], e_old[t]);
    }
  }
  // older tokens: their values in units of the old scale, then like new rows of that size
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int ten = D == 128 ? t : first;
    if (kept) {
      u32x4 o;
      if (ten == 0) {
        o = k_old;
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t b = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) b |= (uint32_t)sv[v_row(pc * 16 + 4 * q + e) + v_pos(tok)] << (8 * e);
          o[q] = b;
        }
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) value4(o[q], &x[t][4 * q]);
    }
    const int e = kept ? e_new[ten] - e_old[ten] : e_new[ten];
    const float top = e_new[ten] == 120 ? 240.f : 448.f;   // 256 * 2^120 is beyond fp32
    u32x4 o;
#pragma unroll
    for (int q = 0; q < 4; ++q) o[q] = code4(&x[t][4 * q], e, top);
    if (ten == 0) {
      *(u32x4 *)(kc + (pc * 32 + tok) * 16) = o;
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) sv[v_row(pc * 16 + 4 * q + i) + v_pos(tok)] = (uint8_t)(o[q] >> (8 * i));
    }
  }
  __syncthreads();
  for (int i = tid; i < 32 * D / 16; i += kThreads)
    ((u32x4 *)vc)[i] = *(const u32x4 *)(sv + v_row(i >> 1) + (i & 1) * 16);
  if (tid < 2) a.c.scales[w.at * 2 + tid] = ldexpf(1.f, tid == 0 ? e_new[0] : e_new[1]);
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void k_kv8_read(Kv8RowsArgs a) {
  constexpr int PC = D / 16;
  constexpr int NT = D == 128 ? 2 : 1;
  __shared__ __attribute__((aligned(16))) uint8_t sv[v_bytes(D)];
  const int tid = threadIdx.x;
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, blockIdx.x)];
  const int g = blockIdx.y;
  const Where w = block_of(a.c, sq, (int)blockIdx.x - sq.tile0, g);
  uint8_t *kc = a.c.k_codes + w.at * (32 * D), *vc = a.c.v_codes + w.at * (32 * D);
  if (w.ok) {
    for (int i = tid; i < 32 * D / 16; i += kThreads)
      *(u32x4 *)(sv + v_row(i >> 1) + (i & 1) * 16) = ((const u32x4 *)vc)[i];
  }
  __syncthreads();
  const int sub = tid % (32 * PC), tok = sub / PC, pc = sub % PC;
  const int first = D == 128 ? 0 : tid / (32 * PC);
  const int64_t pos = (int64_t)w.b * 32 + tok;
  if (pos < w.start || pos >= w.kv) return;
  const int64_t row = (sq.q0 + (pos - w.start)) * a.c.hkv + g;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int ten = D == 128 ? t : first;
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = 0.f;
    if (w.ok) {
      const float s = a.c.scales[w.at * 2 + ten];
      if (ten == 0) {
        const u32x4 o = *(const u32x4 *)(kc + (pc * 32 + tok) * 16);
#pragma unroll
        for (int q = 0; q < 4; ++q) value4(o[q], &x[4 * q]);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          x[e] = __builtin_amdgcn_cvt_f32_fp8((int)sv[v_row(pc * 16 + e) + v_pos(tok)], 0);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] *= s;
    }
    store16((T *)(ten == 0 ? a.ko : a.vo) + row * D + pc * 16, x);
  }
}

// Rows go out in launches of kCondSeqs sequences; a sequence of n rows touches at most
// (n + 30) / 32 + 1 blocks, wherever it starts.
template <typename F>
hipError_t for_rows(Kv8RowsArgs &a, const int32_t *lens, int n, F launch) {
  for (int i = 0, row = 0; i < n;) {
    a.n_seq = 0;
    int tiles = 0;
    for (; i < n && a.n_seq < kCondSeqs; ++i) {
      if (lens[i] == 0) continue;
      a.seq[a.n_seq++] = CondSeq{row, lens[i], i, 0, tiles};
      tiles += (int)(((int64_t)lens[i] + 30) / 32) + 1;
      row += lens[i];
    }
    if (tiles == 0) continue;
    launch(dim3(tiles, a.c.hkv));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_kv8_append(const Kv8View &c, const void *k, int64_t k_row, int64_t k_head, const void *v,
                             int64_t v_row, int64_t v_head, int dtype, const int32_t *new_lens, int n, hipStream_t s) {
  Kv8RowsArgs a;
  a.c = c;
  a.k = k;
  a.v = v;
  a.ko = a.vo = nullptr;
  a.k_row = k_row;
  a.k_head = k_head;
  a.v_row = v_row;
  a.v_head = v_head;
  return for_rows(a, new_lens, n, [&](dim3 grid) {
    if (dtype == MTE_BF16) {
      if (c.d == 64) hipLaunchKernelGGL((k_kv8_append<bf16, 64>), grid, dim3(kThreads), 0, s, a);
      else hipLaunchKernelGGL((k_kv8_append<bf16, 128>), grid, dim3(kThreads), 0, s, a);
    } else {
      if (c.d == 64) hipLaunchKernelGGL((k_kv8_append<float, 64>), grid, dim3(kThreads), 0, s, a);
      else hipLaunchKernelGGL((k_kv8_append<float, 128>), grid, dim3(kThreads), 0, s, a);
    }
  });
}

hipError_t launch_kv8_read(const Kv8View &c, const int32_t *counts, int n, void *k, void *v, int dtype,
                           hipStream_t s) {
  Kv8RowsArgs a;
  a.c = c;
  a.k = a.v = nullptr;
  a.ko = k;
  a.vo = v;
  a.k_row = a.k_head = a.v_row = a.v_head = 0;
  return for_rows(a, counts, n, [&](dim3 grid) {
    if (dtype == MTE_BF16) {
      if (c.d == 64) hipLaunchKernelGGL((k_kv8_read<bf16, 64>), grid, dim3(kThreads), 0, s, a);
      else hipLaunchKernelGGL((k_kv8_read<bf16, 128>), grid, dim3(kThreads), 0, s, a);
    } else {
      if (c.d == 64) hipLaunchKernelGGL((k_kv8_read<float, 64>), grid, dim3(kThreads), 0, s, a);
      else hipLaunchKernelGGL((k_kv8_read<float, 128>), grid, dim3(kThreads), 0, s, a);
    }
  });
}

}  // namespace mte
