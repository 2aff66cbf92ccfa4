// What the kernels of attention over rows of keys and values share: row tiles, their running softmax,
// the two products, rows in and out, partial results. See cond_attention.hip for the forms.
#pragma once

#include "cond_device.h"

namespace mte {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef s16x4 __attribute__((address_space(3))) lds_s16x4;

template <typename T> struct QFrag;   // operand of one 16-byte chunk pair: 32x32x16 (bf16) or 4x 32x32x2 (fp32)
template <> struct QFrag<bf16> { typedef bf16x8 type; };
template <> struct QFrag<float> { typedef f32x4 type; };

constexpr int kThreads = 256;
constexpr int kMaxParts = 512;                      // of a key range

// The workgroup's tile and kv head, heads next to each other: the workgroups that run together then read
// and write whole rows of q and out between them (head-major order: 4 to 10% slower).
struct Unit { int tile, g; };
__device__ __forceinline__ Unit unit_of(const AttnCommon &a) {
  const int flat = a.first + (int)blockIdx.x;
  Unit u;
  u.tile = flat / a.hkv;
  u.g = flat - u.tile * a.hkv;
  return u;
}

// A unit of cross attention: a tile of TR rows over a part of the keys of its sequence. The host cuts every
// key range of nt tiles into parts_of(nt, cut) parts, `cut` for the whole launch; the units of a
// sequence are its row tiles for the first part, then for the next.
__host__ __device__ __forceinline__ int parts_of(int nt, const KeyCut &c) {   // whole, or parts of 4/5 to 5/4 of `per`
  return nt < c.from || nt < 2 * c.per ? 1 : (nt + c.per / 2) / c.per;
}
struct Part { int row_tile, split, used, lo, hi; };     // key tiles [lo, hi)
__device__ __forceinline__ Part part_of(const CondSeq &sq, int local, int rows, int TR, int nt, const KeyCut &cut) {
  Part p;
  p.used = parts_of(nt, cut);
  p.split = 0;
  p.row_tile = local;
  if (p.used > 1) {
    const int tiles = (rows + TR - 1) / TR;
    p.split = local / tiles;
    p.row_tile = local - p.split * tiles;
  }
  const int each = nt / p.used, more = nt % p.used;     // the first `more` parts have one tile more
  p.lo = p.split * each + min(p.split, more);
  p.hi = p.lo + each + (p.split < more);
  return p;
}

// Key tiles [lo, hi) of split `split` of n_split over nt key tiles; used: the splits
// that have any (at least 1). A split takes at least `least` tiles.
struct Span { int lo, hi, used; };
__device__ __forceinline__ Span split_span(int nt, int n_split, int split, int least) {
  const int per = max((nt + n_split - 1) / n_split, least);
  Span s;
  s.used = max(1, (nt + per - 1) / per);
  s.lo = min(split * per, nt);
  s.hi = min(s.lo + per, nt);
  return s;
}

// A reference of scores or sums as a finite number (nothing seen yet: 0, so that exp2(-inf - 0) = 0).
__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.f : m; }

// Running softmax of one row per lane (both halves of the wave hold the same row).
// m is a reference, not quite the maximum: it moves only when some row of the wave has a
// score more than kSlack above it, so that O and l are rescaled in the first step and hardly
// ever after (with random scores every step raises some row's maximum a little, and the 64
// multiplications of a rescaled O of 128 were a fifth of the step's vector work).
// Probabilities are then at most 2^kSlack, and relative precision is what it was.
// Far out, where fp32's step at m is more than 2^-8, m is off the largest product of score and factor by as much, and
// fma(score, factor, -m) with it, up to infinity: there the product is rounded, like m, before m is subtracted, in
// the branch that moves m, which far rows always take (as a branch of its own: 1 to 2% of a call).
constexpr float kSlack = 8.f, kFar = 0x1p16f;
__device__ __forceinline__ void far_scores(f32x16 &s, float factor, float m) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = s[i] * factor - m;
}
template <int ND> struct Rows {
  f32x16 o[ND];
  float m, l;      // m in log2 units; l over this lane's keys only
  float slack;     // kSlack, -inf where some row's m is beyond kFar; wave-uniform
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[n][r] = 0.f;
    m = -INFINITY;
    l = 0.f;
    slack = kSlack;
  }
  // Sets m; whether it is far out.
  __device__ __forceinline__ bool set(float m_new) {
    m = m_new;
    const bool far = __any(fabsf(finite_ref(m)) >= kFar);
    slack = far ? -INFINITY : kSlack;
    return far;
  }
  __device__ __forceinline__ void scale(float f) {
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[n][r] *= f;
  }
  // Takes new scores, their maximum mb (log2 units) and their factor; a probability is then 2^(s factor - ref).
  template <int N> __device__ __forceinline__ void raise(f32x16 (&s)[N], float mb, float &factor, float &ref) {
    ref = finite_ref(m);
    if (__any(mb > m + slack)) {
      const bool far = lift(mb);
      ref = finite_ref(m);
      if (far) {
#pragma unroll
        for (int i = 0; i < N; ++i) far_scores(s[i], factor, ref);
        factor = 1.f;
        ref = 0.f;
      }
    }
  }
  __device__ __forceinline__ bool lift(float mb) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mb), __float_as_uint(mb), false, false);
    const float m_new = fmaxf(m, fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])));
    if (__any(m != -INFINITY)) {                        // else O and l are still zero
      const float alpha = __builtin_amdgcn_exp2f(m - finite_ref(m_new));
      l *= alpha;
      scale(alpha);
    }
    return set(m_new);
  }
};

// Keeps the scores of keys whose bit in `word` (wave-uniform; bit = key of the 32) is set: the lane
// masks of the two halves are scalar work, one select a score.
__device__ __forceinline__ void mask_word(f32x16 &s, uint32_t word) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int k = 8 * (r >> 2) + (r & 3);
    const uint32_t lo = (uint32_t)((int32_t)(word << (31 - k)) >> 31);
    const uint32_t hi = (uint32_t)((int32_t)(word << (27 - k)) >> 31);
    s[r] = __builtin_amdgcn_inverse_ballot_w64((uint64_t)hi << 32 | lo) ? s[r] : -INFINITY;
  }
}
// Keeps the scores of this lane's keys below `n` (of the 32).
__device__ __forceinline__ void mask_below(f32x16 &s, int n, int lane) {
  const int left = n - 4 * (lane >> 5);
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) < left ? s[r] : -INFINITY;
}
__device__ __forceinline__ float max16(const f32x16 &s, float mb) {
#pragma unroll
  for (int i = 0; i < 16; ++i) mb = fmaxf(mb, s[i]);
  return mb;
}

// Memory that is constant while a kernel runs, read at wave-uniform addresses: scalar loads.
template <typename T> __device__ __forceinline__ T uniform_at(const T *p, int64_t i) {
  typedef const T __attribute__((address_space(4))) * ptr;
  return ((ptr)(uintptr_t)p)[i];
}

// Joins the KW waves' states of the same 32 rows through LDS into wave 0's.
// red: (KW - 1) * (2 + 16 ND) * 64 floats.
template <int ND, int KW>
__device__ __forceinline__ void join_waves(Rows<ND> &st, float *red, int kw, int lane) {
  constexpr int NV = 2 + 16 * ND;
  if (kw > 0) {
    float *p = red + (kw - 1) * NV * 64 + lane;
    p[0] = st.m;
    p[64] = st.l;
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) p[(2 + n * 16 + r) * 64] = st.o[n][r];
  }
  __syncthreads();
  if (kw > 0) return;
  float mx = st.m;
#pragma unroll
  for (int v = 0; v < KW - 1; ++v) mx = fmaxf(mx, red[v * NV * 64 + lane]);
  const float mr = finite_ref(mx);
  const float f0 = __builtin_amdgcn_exp2f(st.m - mr);
  st.l *= f0;
  st.scale(f0);
#pragma unroll
  for (int v = 0; v < KW - 1; ++v) {
    const float *p = red + v * NV * 64 + lane;
    const float fv = __builtin_amdgcn_exp2f(p[0] - mr);
    st.l += fv * p[64];
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.o[n][r] += fv * p[(2 + n * 16 + r) * 64];
  }
  st.m = mx;
}

// 8 consecutive d (16 p + 8 h .. of a 32-wide block) of this lane's row as bf16.
__device__ __forceinline__ u32x4 out_chunk(const f32x16 &o, int p, float inv) {
  bf16x4 lo, hi;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    lo[e] = (bf16)(o[8 * p + e] * inv);
    hi[e] = (bf16)(o[8 * p + 4 + e] * inv);
  }
  u32x2 x = __builtin_bit_cast(u32x2, lo), y = __builtin_bit_cast(u32x2, hi);
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    // the upper 32 lanes' x and the lower 32 lanes' y trade places
    const auto r = __builtin_amdgcn_permlane32_swap(x[w], y[w], false, false);
    x[w] = r[0];
    y[w] = r[1];
  }
  return u32x4{x[0], x[1], y[0], y[1]};
}

// Writes a wave's finished rows (lane: row `tok`, head `head`; vscale: factor of O that
// the probabilities did not carry) or, split, their partial state.
template <typename T, int ND>
__device__ __forceinline__ void store_rows(const AttnCommon &a, Rows<ND> &st, float vscale, bool live, int64_t tok,
                                           int head, int lane) {
  const float l = st.l + __shfl_xor(st.l, 32, kWave);
  const float inv = l > 0.f ? vscale / l : 0.f;
  T *row = (T *)a.out + tok * a.o_row + (int64_t)head * a.o_head;
  const int h = lane >> 5;
#pragma unroll
  for (int n = 0; n < ND; ++n) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int c = 32 * n + 8 * b + 4 * h;
        const f32x4 w{st.o[n][4 * b] * inv, st.o[n][4 * b + 1] * inv, st.o[n][4 * b + 2] * inv,
                      st.o[n][4 * b + 3] * inv};
        if (live && c < a.d) *(f32x4 *)(row + c) = w;
      }
    } else {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int c = 32 * n + 16 * p + 8 * h;
        const u32x4 x = out_chunk(st.o[n], p, inv);
        if (live && c < a.d) *(u32x4 *)(row + c) = x;
      }
    }
  }
}

// Partial state of row r of unit (tile, g) and split: O / l (times vscale: no larger than the values,
// so that nothing overflows before the parts are joined), m, l.
template <int ND>
__device__ __forceinline__ void store_part(const AttnCommon &a, Rows<ND> &st, float vscale, bool live, int tile, int g,
                                           int split, int r, int lane) {
  const float l = st.l + __shfl_xor(st.l, 32, kWave);
  const float inv = l > 0.f ? vscale / l : 0.f;
  if (!live) return;
  const int64_t at = (((int64_t)tile * a.hkv + g) * a.n_split + split) * a.ws_rows + r;
  float *o = a.ws + at * (32 * ND) + 4 * (lane >> 5);
#pragma unroll
  for (int n = 0; n < ND; ++n)
#pragma unroll
    for (int b = 0; b < 4; ++b)
      *(f32x4 *)(o + 32 * n + 8 * b) = f32x4{st.o[n][4 * b] * inv, st.o[n][4 * b + 1] * inv, st.o[n][4 * b + 2] * inv,
                                            st.o[n][4 * b + 3] * inv};
  if (lane < 32) {
    float *ml = a.ws + a.ws_ml + at * 2;
    ml[0] = st.m;
    ml[1] = l;
  }
}

// Probabilities of 32 keys, p = 2^(sc s - ref), as the operand of the value product: bf16 (the values'
// type: their range is bf16's; each term off by at most 2^-8 of itself) or fp32.
template <typename T> struct Probs;
template <> struct Probs<bf16> { bf16x8 f[2]; };
template <> struct Probs<float> { float p[16]; };
__device__ __forceinline__ void set_probs(Probs<bf16> &o, const float *p) {
#pragma unroll
  for (int e = 0; e < 16; ++e) o.f[e >> 3][e & 7] = (bf16)p[e];
}
__device__ __forceinline__ void set_probs(Probs<float> &o, const float *p) {
#pragma unroll
  for (int e = 0; e < 16; ++e) o.p[e] = p[e];
}
template <typename T>
__device__ __forceinline__ Probs<T> probs_of(const f32x16 &s, float sc, float ref, float &l) {
  float p[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], sc, -ref));
    l += p[i];
  }
  Probs<T> o;
  set_probs(o, p);
  return o;
}

// O += V^T P^T for the 32 keys of subtile `sub`. Values as rows in LDS at sv, chunks xored.
template <int NCH, bool B16> __device__ __forceinline__ int value_chunk(int row, int c) {
  if constexpr (!B16) return c ^ (8 * ((row >> 2) & 1));
  else if constexpr (NCH == 16) return c ^ (4 * (row & 3));
  else return c ^ (4 * ((row >> 1) & 1));
}
template <typename T, int DP>
__device__ __forceinline__ void add_values(f32x16 (&o)[DP / 32], const Probs<T> &p, const char *sv, int sub, int lane) {
  constexpr int NCH = DP * sizeof(T) / 16, ND = DP / 32;
  const int h = lane >> 5, lrow = lane & 31;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      const int row = sub * 32 + 16 * f + 4 * h + ((lane & 15) >> 2);
#pragma unroll
      for (int n = 0; n < ND; ++n) {
        const int c = 4 * n + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        const char *va = sv + (row * NCH + value_chunk<NCH, true>(row, c)) * 16 + (lane & 1) * 8;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)va);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(va + 8 * NCH * 16));
        mfma32(o[n], __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)), p.f[f]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int row = sub * 32 + 8 * (i >> 2) + 4 * h + (i & 3);
      const float *vr = (const float *)sv + row * DP;
#pragma unroll
      for (int n = 0; n < ND; ++n)
        o[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(vr[32 * (n ^ h) + lrow], p.p[i], o[n], 0, 0, 0);
    }
  }
}

// S^T = K Q^T of subtile `sub`: keys as operand chunks in LDS at sk.
template <typename T, int DP>
__device__ __forceinline__ void key_scores(f32x16 &s, const u32x4 *sk,
                                           const typename QFrag<T>::type (&qf)[DP * sizeof(T) / 32], int sub, int lane) {
  constexpr int NCH = DP * sizeof(T) / 16;
  const int lrow = lane & 31, h = lane >> 5;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
  for (int kk = 0; kk < NCH / 2; ++kk) {
    const int c = 2 * kk + h;
    mfma32(s, __builtin_bit_cast(typename QFrag<T>::type, sk[(sub * NCH + c) * 32 + (lrow ^ (c & 7))]), qf[kk]);
  }
}

constexpr int kBox = 4096;          // a wave's LDS for it
// A store that leaves nothing in L2 (written out: as a branch of two stores of one value the
// compiler makes one plain store of it).
__device__ __forceinline__ void store_past_caches(char *base, uint32_t off, const u32x4 &x) {
  asm volatile("global_store_dwordx4 %0, %1, %2 nt" ::"v"(off), "v"(x), "s"(base) : "memory");
}
// Rows of a tile between memory and the lanes that own them, 128 bytes of a row at a time: a load or
// store takes 8 whole lines (8 lanes each), and 4 KB of LDS of the wave's own turn them (chunks
// xored with the row: neither side meets in a bank). Straight from the owning lanes an access
// would take 32 bytes of 32 rows: on 65536 rows of 10 heads of 64, copied, 40 us against 31.5.
// Place of chunk c of row r in a box.
__device__ __forceinline__ int box_at(int r, int c) { return r * 8 + (c ^ (r & 7)); }
// The rows of the tile: r0 .. of `rows`, token r / rep and head g rep + r % rep. Their addresses are a
// wave-uniform base and 32-bit offsets (the host's AttnProblem::near_tiles): products of 64 bits are
// quarter-rate instructions (16 x 4096 rows of 10 heads of 64: 44.8 us, with them 46.0).
struct TileRows {
  int64_t tok0;        // token of row r0, absolute
  int rem0, left;      // r0 % rep, rows that exist
  float inv;           // 1 / rep
  __device__ __forceinline__ TileRows(const AttnCommon &a, const CondSeq &sq, int r0, int rows) {
    const int t = r0 / a.rep;
    tok0 = sq.q0 + t;
    rem0 = r0 - t * a.rep;
    left = rows - r0;
    inv = 1.f / (float)a.rep;
  }
  template <typename T> __device__ __forceinline__ T *base(T *p, int64_t row, int64_t head, int g, int rep) const {
    const uint64_t x = (uint64_t)(uintptr_t)(p + tok0 * row + (int64_t)(g * rep) * head);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (T *)(uintptr_t)((uint64_t)hi << 32 | lo);
  }
  // elements from the base to row r0 + i
  __device__ __forceinline__ uint32_t offset(int i, int64_t row, int64_t head, int rep) const {
    if (rep == 1) return __umul24(i, (uint32_t)row);
    const int x = rem0 + i, t = (int)(((float)x + 0.5f) * inv);   // exact: rep is 2^16 at most
    return __umul24(t, (uint32_t)row) + (uint32_t)(x - t * rep) * (uint32_t)head;
  }
};
template <typename T, int DP> struct QTile {
  static constexpr int PARTS = DP * sizeof(T) / 128, E = 16 / sizeof(T);
  u32x4 x[PARTS * 4];
  __device__ __forceinline__ void load(const AttnCommon &a, const TileRows &t, int g, int lane) {
    const char *base = (const char *)t.base((const T *)a.q, a.q_row, a.q_head, g, a.rep);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 8 * i + (lane >> 3);
      const uint32_t off = t.offset(r, a.q_row, a.q_head, a.rep);
#pragma unroll
      for (int j = 0; j < PARTS; ++j) {
        const int c = (8 * j + (lane & 7)) * E;
        x[4 * j + i] = u32x4{0, 0, 0, 0};
        if (r < t.left && c < a.d) x[4 * j + i] = *(const u32x4 *)(base + (off + c) * (uint32_t)sizeof(T));
      }
    }
  }
  // part j into the wave's 4 KB; then chunk c (of 8) of this lane's row
  __device__ __forceinline__ void spread(u32x4 *box, int j, int lane) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) box[box_at(8 * i + (lane >> 3), lane & 7)] = x[4 * j + i];
  }
  static __device__ __forceinline__ u32x4 chunk(const u32x4 *box, int c, int lane) {
    return box[box_at(lane & 31, c)];
  }
};
template <typename T, int ND>
__device__ __forceinline__ void store_tile(const AttnCommon &a, Rows<ND> &st, float vscale, const TileRows &t, int g,
                                           u32x4 *box, int lane) {
  constexpr int E = 16 / sizeof(T), PARTS = ND * 32 * sizeof(T) / 128;
  const float l = st.l + __shfl_xor(st.l, 32, kWave);
  const float inv = l > 0.f ? vscale / l : 0.f;
  const int r = lane & 31, h = lane >> 5;
  char *base = (char *)t.base((T *)a.out, a.o_row, a.o_head, g, a.rep);
  uint32_t off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) off[i] = t.offset(8 * i + (lane >> 3), a.o_row, a.o_head, a.rep);
#pragma unroll
  for (int j = 0; j < PARTS; ++j) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int b = 0; b < 4; ++b)
        box[box_at(r, 2 * b + h)] =
            __builtin_bit_cast(u32x4, f32x4{st.o[j][4 * b] * inv, st.o[j][4 * b + 1] * inv, st.o[j][4 * b + 2] * inv,
                                            st.o[j][4 * b + 3] * inv});
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) box[box_at(r, 2 * q + h)] = out_chunk(st.o[2 * j + (q >> 1)], q & 1, inv);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 8 * i + (lane >> 3), c = (8 * j + (lane & 7)) * E;
      const u32x4 x = box[box_at(row, lane & 7)];
      const uint32_t at = (off[i] + c) * (uint32_t)sizeof(T);
      if (row < t.left && c < a.d) {
        if (a.big) store_past_caches(base, at, x);
        else *(u32x4 *)(base + at) = x;
      }
    }
  }
}

// (of 8 chunks, two rows fill the banks: swizzled by the pair, a quarter of the conflicts that r & 7 leaves)
template <int NCH> __device__ __forceinline__ int key_swz(int r, int c) { return c ^ (NCH == 8 ? (r >> 1) & 7 : r & (NCH - 1)); }
template <int DP> struct Stream {
  static constexpr int NCH = DP / 8, TILE = 32 * NCH;     // chunks a row; 16-byte chunks of a tile's keys
  static constexpr int NB = DP == 64 ? 4 : 3;             // two slots for the first tiles, and the waves' kBox
  static constexpr int COPIES = TILE / 64 / 4;            // 1 KB copies of keys (and of values) a wave and tile
  static constexpr int BYTES = NB * 2 * TILE * 16;
  static_assert((NB - 2) * 2 * TILE * 16 >= 4 * kBox, "room to turn the rows");
};

}  // namespace mte
