// Attention of packed queries to conditioning tokens: keys and values as rows (k_cross,
// k_cross_stream), or as e4m3 codes in blocks of 32 tokens (k_kv8_rows, k_kv8_tiles, k_kv8_res).
//
//   o[i, h] = sum_j p_ij v[j, g],  p_ij = exp(s_ij - m_i) / sum_j exp(s_ij - m_i),
//   s_ij = scale q[i, h] . k[j, g],  g = h / rep
//
// Rows. The rep query heads of a kv head read the same keys, so the rows of a matrix tile are (token,
// head) pairs: row r of a sequence is token r / rep, head g rep + r % rep. One query with grouped
// heads fills rep rows, not one.
//
// Matrix core forms (32x32, as in attention.hip): S^T = K Q^T leaves each lane the scores of one row
// (lane % 32) for 16 of 32 keys, key 8 (r / 4) + 4 (lane / 32) + r % 4 in register r, so maxima and
// sums are per-lane loops and one exchange between the wave's halves, and the probabilities are
// already the B operand of O^T = V^T P^T, if V^T is read with its keys in that same order.
//
// One pass over the keys with a running reference m and sum l of each row (fp32, log2 units); O is
// rescaled where m moves. Key ranges may be split: over the waves of a workgroup (joined through
// LDS) and over workgroups (O / l, m, l of each part in the workspace, joined by a second launch).
//
// Roundings to fewer than 32 bits: the probabilities, as the operand of the second product (Probs,
// CodeProbs), and the result. Scores, m, l, O and the joins are fp32.
#include <algorithm>
#include <climits>
#include <cmath>

#include "../../include/mte.h"
#include "cond_device.h"

namespace mte {

namespace {

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
__device__ __forceinline__ Unit unit_of(int hkv) {
  const int flat = blockIdx.x;
  Unit u;
  u.tile = flat / hkv;
  u.g = flat - u.tile * hkv;
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

// ---- keys and values as rows --------------------------------------------------------------------
//
// k_cross: a workgroup of four waves serves 32 RW rows of one sequence and kv head; the other 4 / RW ways of
// its waves split the keys of a tile (few rows: RW = 1). Key tiles go global -> registers -> LDS, the
// next tile's loads issued before one is computed (where the registers hold them: not fp32 tiles of
// 128 keys of 128); rows past the end and masked value rows become zeros as they arrive, so that the loads are
// waited for before that computation, not after it, and with a mask its bytes before the rows.
// Bound by latency: launch, sequence table, each tile's loads, softmax, store, one after the other (16 x 1
// tokens of 2 x 8 heads of 128 over 96: 7.5 us for 6.4 MB); fp32 by the loads and the matrix instructions, a
// ninth of bf16's rate, in turn (12 x 918 rows of 8 heads of 64 over 1610 keys in all: 46 us, 66 of 137 TFLOP/s).
// LDS: keys as 16-byte chunks in the order of the MFMA operand ([32 keys][chunk c]:
// lane = key), the key index xored with the chunk so that neither the row-wise
// writes nor the operand reads meet in a bank; values as rows, chunks xored so that the
// transposing reads (bf16: 4 keys x 16 d per 16 lanes) and the fp32 reads (one d column
// a lane) do not either.
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

template <typename T, int DP, int RW>
__global__ __launch_bounds__(kThreads, 2) void k_cross(CrossArgs a) {
  constexpr bool B16 = sizeof(T) == 2;
  constexpr int KW = 4 / RW;
  constexpr int NS = B16 && RW == 4 ? 2 : 1;        // 32-key subtiles of a wave per tile
  constexpr int KT = 32 * NS * KW;                  // keys per tile
  constexpr int E = 16 / sizeof(T), NCH = DP / E, NK = NCH / 2, ND = DP / 32;
  constexpr int CPT = KT * NCH / kThreads;          // chunks of K (and of V) per thread
  constexpr bool AHEAD = CPT <= 8;                  // next tile in registers meanwhile
  constexpr int STEP = AHEAD ? CPT : 4;
  typedef typename QFrag<T>::type frag_t;
  extern __shared__ u32x4 lds[];
  u32x4 *sk = lds;
  char *sv = (char *)(lds + KT * NCH);
  uint32_t *sm = (uint32_t *)(lds + 2 * KT * NCH);  // validity of the tile's keys, a bit each

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lrow = lane & 31, h = lane >> 5;
  const int rw = wave % RW, kw = wave / RW;
  const Unit un = unit_of(a.hkv);
  const int tile = un.tile, g = un.g;
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, tile)];
  const int klen = sq.k_len, rows = sq.q_len * a.rep;
  const Part span = part_of(sq, tile - sq.tile0, rows, 32 * RW, (klen + KT - 1) / KT, a.cut);
  const int r0 = span.row_tile * 32 * RW + rw * 32; // first row of the wave
  const int r = r0 + lrow;
  const bool live = r < rows;
  const int64_t tok = sq.q0 + (live ? r / a.rep : 0);
  const int head = g * a.rep + (live ? r % a.rep : 0);

  const T *kg = (const T *)a.k + (int64_t)sq.k0 * a.k_row + (int64_t)g * a.k_head;
  const T *vg = (const T *)a.v + (int64_t)sq.k0 * a.v_row + (int64_t)g * a.v_head;
  const uint8_t *mg = a.mask ? a.mask + sq.k0 : nullptr;
  u32x4 kx[STEP], vx[STEP];
  bool see = false;
  auto gload = [&](int kt, int t0) {
#pragma unroll
    for (int t = 0; t < STEP; ++t) {
      const int idx = tid + (t0 + t) * kThreads, c = idx % NCH;
      const int key = kt * KT + idx / NCH;
      const int kc = min(key, klen - 1), cc = c * E < a.d ? c * E : 0;   // an address inside in any case
      const u32x4 x = *(const u32x4 *)(kg + (int64_t)kc * a.k_row + cc);
      const u32x4 y = *(const u32x4 *)(vg + (int64_t)kc * a.v_row + cc);
      const bool ok = key < klen && c * E < a.d;
      const bool vok = ok && (!mg || mg[kc]);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        kx[t][w] = ok ? x[w] : 0;
        vx[t][w] = vok ? y[w] : 0;
      }
    }
  };
  auto gmask = [&](int kt) {
    const int key = kt * KT + tid;
    see = tid < KT && key < klen && (!mg || mg[key]);
  };
  auto lstore = [&](int t0) {
#pragma unroll
    for (int t = 0; t < STEP; ++t) {
      const int idx = tid + (t0 + t) * kThreads, row = idx / NCH, c = idx % NCH;
      sk[((row >> 5) * NCH + c) * 32 + ((row & 31) ^ (c & 7))] = kx[t];
      *(u32x4 *)(sv + (row * NCH + value_chunk<NCH, B16>(row, c)) * 16) = vx[t];
    }
  };
  auto lmask = [&]() {
    const uint64_t b = __ballot(see);
    if (lane == 0 && wave * 64 < KT) {
      sm[wave * 2] = (uint32_t)b;
      if (KT > 32) sm[wave * 2 + 1] = (uint32_t)(b >> 32);
    }
  };

  const bool any = span.lo < span.hi;               // workgroup-uniform
  if (any) {
    gmask(span.lo);
    if constexpr (AHEAD) gload(span.lo, 0);
  }
  frag_t qf[NK];
#pragma unroll
  for (int kk = 0; kk < NK; ++kk) {
    const int c = (2 * kk + h) * E;
    u32x4 x{0, 0, 0, 0};
    if (live && c < a.d) x = *(const u32x4 *)((const T *)a.q + tok * a.q_row + (int64_t)head * a.q_head + c);
    qf[kk] = __builtin_bit_cast(frag_t, x);
  }
  Rows<ND> st;
  st.init();

  auto compute = [&]() {
    f32x16 s[NS];
    float mb = -INFINITY;
#pragma unroll
    for (int u = 0; u < NS; ++u) {
      key_scores<T, DP>(s[u], sk, qf, kw * NS + u, lane);
      const uint32_t word = __builtin_amdgcn_readfirstlane(sm[kw * NS + u]);
      if (word != 0xFFFFFFFFu) mask_word(s[u], word);
      mb = max16(s[u], mb);
    }
    float sc = a.sc, ref;
    st.raise(s, mb * sc, sc, ref);
#pragma unroll
    for (int u = 0; u < NS; ++u)
      add_values<T, DP>(st.o, probs_of<T>(s[u], sc, ref, st.l), sv, kw * NS + u, lane);
  };

  for (int kt = span.lo; kt < span.hi; ++kt) {
    __syncthreads();                                // the tile before is read
    if constexpr (AHEAD) {
      lstore(0);
    } else {
      for (int t0 = 0; t0 < CPT; t0 += STEP) {
        gload(kt, t0);
        lstore(t0);
      }
    }
    lmask();
    __syncthreads();
    if (kt + 1 < span.hi) {
      gmask(kt + 1);
      if constexpr (AHEAD) gload(kt + 1, 0);
    }
    if (r0 < rows) compute();                       // wave-uniform
  }
  if constexpr (KW > 1) {
    __syncthreads();
    join_waves<ND, KW>(st, (float *)lds, kw, lane);
    if (kw > 0) return;
  }
  if (r0 >= rows) return;
  if (span.used == 1) store_rows<T, ND>(a, st, 1.f, live, tok, head, lane);
  else store_part<ND>(a, st, 1.f, live, tile, g, 0, rw * 32 + lrow, lane);
}

// Lane j: which keys of the 32-key tile t0 + j count (a bit each), for up to 64 tiles.
__device__ __forceinline__ uint32_t tile_words(const uint8_t *mask, int klen, int t0, int lane) {
  if (!mask) {
    const int n = klen - (t0 + lane) * 32;
    return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u;
  }
  uint32_t words = 0;
  const int nk = min((klen + 31) / 32 - t0, 64);
  for (int j0 = 0; j0 < nk; j0 += 16) {              // 512 keys a round, their bytes in flight together
    bool see[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int key = (t0 + j0 + 2 * i) * 32 + lane;
      see[i] = mask[min(key, klen - 1)] != 0 && key < klen;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint64_t b = __ballot(see[i]);
      if (lane == j0 + 2 * i) words = (uint32_t)b;
      if (lane == j0 + 2 * i + 1) words = (uint32_t)(b >> 32);
    }
  }
  return words;
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

// Many rows, keys streamed: four waves of 32 rows over a ring of 32-key tiles that the LDS-direct
// copies (dma16) fill two tiles ahead, one barrier a tile. No registers and no vector work for
// the staging, so that three waves fit a SIMD (head_dim 128), and workgroups in different phases
// share a compute unit: rows come and go while others compute.
// Tiles: keys [32][NCH chunks], values the same, chunk c of row r at c ^ key_swz / value_chunk: whole
// rows for the copies, free of bank conflicts for the operand reads. Rows past the end repeat the
// last one; their scores are masked, and value rows that must not count (past the end, masked)
// are overwritten with zeros by the wave that copied them. Chunks past head_dim are not copied and
// stay zero (a lane that skips a copy leaves its 16 bytes alone; no copy is skipped whole).
// The ring's idle slots turn the rows (QTile): before the first barrier the last ones, after the
// last barrier those that the last tile does not use.
// Bound by the rows in and out where the keys are few (16 x 4096 rows of 10 heads of 64 over 96 keys: 44.3 us,
// 3.9 TB/s; the same copies without any arithmetic 40), by both where they are not (32 x 1000 of 2 x 8 heads
// of 128 over 102 to 319: 103 us, 540 TFLOP/s, 2.8 TB/s; rows alone 53, with the key copies 78). Six or eight
// waves a workgroup (125 to 155 us), the keys whole in LDS (129), scores of one tile among the value
// products of the one before (registers spill) and XCD-contiguous tiles (114 to 130) were slower.
// (of 8 chunks, two rows fill the banks: swizzled by the pair, a quarter of the conflicts that r & 7 leaves)
template <int NCH> __device__ __forceinline__ int key_swz(int r, int c) { return c ^ (NCH == 8 ? (r >> 1) & 7 : r & (NCH - 1)); }
template <int DP> struct Stream {
  static constexpr int NCH = DP / 8, TILE = 32 * NCH;     // chunks a row; 16-byte chunks of a tile's keys
  static constexpr int NB = DP == 64 ? 4 : 3;             // two slots for the first tiles, and the waves' kBox
  static constexpr int COPIES = TILE / 64 / 4;            // 1 KB copies of keys (and of values) a wave and tile
  static constexpr int BYTES = NB * 2 * TILE * 16;
  static_assert((NB - 2) * 2 * TILE * 16 >= 4 * kBox, "room to turn the rows");
};
template <int DP>
__global__ __launch_bounds__(kThreads, DP == 64 ? 4 : 3) void k_cross_stream(CrossArgs a) {
  typedef Stream<DP> S;
  constexpr int NCH = S::NCH, NK = NCH / 2, ND = DP / 32, CP = S::COPIES;
  extern __shared__ u32x4 lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lrow = lane & 31, h = lane >> 5;
  const Unit un = unit_of(a.hkv);
  const int tile = un.tile, g = un.g;
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, tile)];
  const int klen = sq.k_len, rows = sq.q_len * a.rep;
  const Part span = part_of(sq, tile - sq.tile0, rows, 128, (klen + 31) >> 5, a.cut);
  const int r0 = span.row_tile * 128 + wave * 32;

  const bf16 *kg = (const bf16 *)a.k + (int64_t)sq.k0 * a.k_row + (int64_t)g * a.k_head;
  const bf16 *vg = (const bf16 *)a.v + (int64_t)sq.k0 * a.v_row + (int64_t)g * a.v_head;
  const uint8_t *mg = a.mask ? a.mask + sq.k0 : nullptr;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  // copy i of this wave: rows RPC (wave CP + i) .. of the tile
  constexpr int RPC = 64 / NCH;
  auto copy_tile = [&](int t) {
    const bf16 *kb = kg + (int64_t)t * 32 * a.k_row, *vb = vg + (int64_t)t * 32 * a.v_row;
    const uint32_t to = lds0 + (uint32_t)(((t - span.lo) % S::NB) * 2 * S::TILE + wave * CP * 64) * 16;
#pragma unroll
    for (int i = 0; i < CP; ++i) {
      const int r = RPC * (wave * CP + i) + lane / NCH, p = lane % NCH;
      const int row = min(r, klen - 1 - t * 32);
      const int kc = key_swz<NCH>(r, p) * 8, vc = value_chunk<NCH, true>(r, p) * 8;
      if (kc < a.d) dma16(kb, (__umul24(row, (uint32_t)a.k_row) + kc) * 2u, to + i * 1024);
      if (vc < a.d) dma16(vb, (__umul24(row, (uint32_t)a.v_row) + vc) * 2u, to + (S::TILE + i * 64) * 16);
    }
  };
  const TileRows rw(a, sq, r0, rows);
  QTile<bf16, DP> qt;
  if (r0 < rows) qt.load(a, rw, g, lane);
  const int t0 = span.lo, t1 = span.hi;
  uint32_t words = tile_words(mg, klen, t0, lane);
  if (t0 < t1) copy_tile(t0);
  if (t0 + 1 < t1) copy_tile(t0 + 1);
  u32x4 *box = lds + (S::NB * 2 * S::TILE - 4 * (kBox / 16)) + wave * (kBox / 16);
  bf16x8 qf[NK];
  if (r0 < rows) {
#pragma unroll
    for (int j = 0; j < qt.PARTS; ++j) {
      qt.spread(box, j, lane);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) qf[4 * j + kk] = __builtin_bit_cast(bf16x8, qt.chunk(box, 2 * kk + h, lane));
    }
  }
  if (a.d < DP) {                                   // uniform
    __syncthreads();                                // the rows are turned
#pragma unroll
    for (int i = 0; i < S::NB * CP; ++i) {          // the rows that this wave copies, of every slot
      const int r = RPC * (wave * CP + i % CP) + lane / NCH, p = lane % NCH;
      u32x4 *at = lds + (i / CP) * 2 * S::TILE + (wave * CP + i % CP) * 64 + lane;
      if (key_swz<NCH>(r, p) * 8 >= a.d) at[0] = u32x4{0, 0, 0, 0};
      if (value_chunk<NCH, true>(r, p) * 8 >= a.d) at[S::TILE] = u32x4{0, 0, 0, 0};
    }
  }
  Rows<ND> st;
  st.init();
  for (int t = t0; t < t1; ++t) {
    const u32x4 *sk = lds + ((t - t0) % S::NB) * 2 * S::TILE, *sv = sk + S::TILE;
    if (t > t0 && (t - t0) % 64 == 0) words = tile_words(mg, klen, t, lane);
    const uint32_t word = (uint32_t)__builtin_amdgcn_readlane((int)words, (t - t0) % 64);
    if (t + 1 < t1) wait_vm<2 * CP>();              // this tile's copies: the next one's are younger
    else wait_vm<0>();
    if (word != 0xFFFFFFFFu) {
#pragma unroll
      for (int i = 0; i < CP; ++i) {
        const int r = RPC * (wave * CP + i) + lane / NCH;
        if (!((word >> r) & 1)) ((u32x4 *)sv)[(wave * CP + i) * 64 + lane] = u32x4{0, 0, 0, 0};
      }
    }
    __syncthreads();                                // the tile is whole, and the one before it read
    if (t + 2 < t1) copy_tile(t + 2);
    if (r0 < rows) {                                // wave-uniform
      f32x16 s[1];
#pragma unroll
      for (int i = 0; i < 16; ++i) s[0][i] = 0.f;
#pragma unroll
      for (int kk = 0; kk < NK; ++kk)
        mfma32(s[0], __builtin_bit_cast(bf16x8, sk[lrow * NCH + key_swz<NCH>(lrow, 2 * kk + h)]), qf[kk]);
      if (word != 0xFFFFFFFFu) mask_word(s[0], word);
      float sc = a.sc, ref;
      st.raise(s, max16(s[0], -INFINITY) * sc, sc, ref);
      add_values<bf16, DP>(st.o, probs_of<bf16>(s[0], sc, ref, st.l), (const char *)sv, 0, lane);
    }
  }
  if (r0 >= rows) return;
  if (span.used > 1) {
    store_part<ND>(a, st, 1.f, r0 + lrow < rows, tile, g, 0, wave * 32 + lrow, lane);
    return;
  }
  // all slots but the last tile's and the one before hold nothing that is still read
  constexpr int ROOM = S::NB * 2 * S::TILE;
  int mine = (t1 - t0) % S::NB * 2 * S::TILE + wave * (kBox / 16);
  if (mine >= ROOM) mine -= ROOM;
  store_tile<bf16, ND>(a, st, 1.f, rw, g, lds + mine, lane);
}

// ---- keys and values as e4m3 codes --------------------------------------------------------------
//
// Codes widen exactly: keys to bf16 (the queries' type: their range is bf16's), values to
// fp16. fp32 queries are three bf16 terms (24 bits).
// Block scales: the key scale multiplies the scores, the value scale the probabilities. Their products,
// weights p_j 2^lv (lv: log2 of the block's value scale), are the operand of the value product: fp16, once
// rounded (2^-11), or for fp32 calls two fp16 terms (2^-22), so that the 16-bit matrix cores serve both. fp16's
// range is short, so weights are relative to a running reference of their own for each row, u:
// the largest is held in [2^7, 2^15], and fp16's smallest step is 2^-31 of it or less, whatever scales other
// blocks have. (In units of the largest scale so far, a row whose weight lies in blocks of scales
// 2^32 smaller, under keys that it hardly weighs, would come out as zero.)
constexpr float kPOff = 15.f - kSlack;

// log2 of a block's value scale: the exponent, exact, and the rest (0 for powers of two).
__device__ __forceinline__ float scale_log(float vs) {
  const uint32_t b = __float_as_uint(vs);
  return (float)((int)(b >> 23) - 127) + __builtin_amdgcn_logf(__uint_as_float((b & 0x7FFFFF) | 0x3F800000));
}

// State of 32 rows over cached codes. With m the reference of the scores (Rows), O is in units of 2^(m + u); both
// lag like m, and are whole numbers, so that rescaling is exact. l and the weights carry 2^kPOff more.
template <int ND> struct CodeRows : Rows<ND> {
  using Rows<ND>::o;
  using Rows<ND>::m;
  using Rows<ND>::l;
  using Rows<ND>::slack;
  float u;
  __device__ __forceinline__ void init() {
    Rows<ND>::init();
    u = -INFINITY;
  }
  // Takes the scores of N blocks of value scales 2^lv, and their factors; a probability is then 2^(s factor - ref).
  template <int N>
  __device__ __forceinline__ void raise(f32x16 (&s)[N], float (&factor)[N], const float (&lv)[N], float &ref) {
    float mb[N];
    bool over = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      mb[i] = max16(s[i], -INFINITY) * factor[i];
      over |= mb[i] - m > fminf(slack, u + kSlack - lv[i]);   // (NaN where nothing is seen yet)
    }
    ref = finite_ref(m);
    if (__any(over)) {
      const bool far = lift<N>(mb, lv);
      ref = finite_ref(m);
      if (far) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          far_scores(s[i], factor[i], ref);
          factor[i] = 1.f;
        }
        ref = 0.f;
      }
    }
  }
  template <int N> __device__ __forceinline__ bool lift(const float (&mb)[N], const float (&lv)[N]) {
    float top[N], m_new = m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mb[i]), __float_as_uint(mb[i]), false, false);
      top[i] = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
      m_new = fmaxf(m_new, floorf(top[i]));
    }
    const float mr = finite_ref(m_new), kept = m - mr + u;
    float u_new = kept;
#pragma unroll
    for (int i = 0; i < N; ++i) u_new = fmaxf(u_new, floorf(top[i] - mr + lv[i]));
    if (__any(m != -INFINITY)) {                        // else O and l are still zero
      l *= __builtin_amdgcn_exp2f(m - mr);
      Rows<ND>::scale(__builtin_amdgcn_exp2f(kept - finite_ref(u_new)));
    }
    u = u_new;
    return Rows<ND>::set(m_new);
  }
  // For the block of value scale 2^lv: a weight is a probability times 2^c, w what their sum counts in l. Weights too
  // far below the row's largest (2^-60, nothing in fp16) are kept from fp32's own limit, for l.
  struct Share { float c, w; };
  __device__ __forceinline__ Share share(float lv) const {
    const float x = fminf(finite_ref(u) - lv, 60.f);
    return Share{kPOff - x, __builtin_amdgcn_exp2f(x)};
  }
  // What O is still to be multiplied by, 2^u: here in part where that is far from 1.
  __device__ __forceinline__ float unit() {
    const float e = finite_ref(u);
    float half = 0.f;
    if (__any(fabsf(e) > 64.f)) {
      half = truncf(0.5f * e);
      Rows<ND>::scale(__builtin_amdgcn_exp2f(half));
    }
    return __builtin_amdgcn_exp2f(e - half);
  }
};

// Brings the KW waves' states of the same rows to one pair of references. red: 2 KW x 64 floats.
template <int ND, int KW>
__device__ __forceinline__ void match_waves(CodeRows<ND> &st, float *red, int wave, int lane) {
  red[wave * 64 + lane] = st.m;
  red[(KW + wave) * 64 + lane] = st.u;
  __syncthreads();
  float m = -INFINITY, u = -INFINITY;
#pragma unroll
  for (int v = 0; v < KW; ++v) m = fmaxf(m, red[v * 64 + lane]);
  const float mr = finite_ref(m);
#pragma unroll
  for (int v = 0; v < KW; ++v) u = fmaxf(u, red[v * 64 + lane] - mr + red[(KW + v) * 64 + lane]);
  st.l *= __builtin_amdgcn_exp2f(st.m - mr);
  st.scale(__builtin_amdgcn_exp2f(st.m - mr + st.u - finite_ref(u)));
  st.m = m;
  st.u = u;
  __syncthreads();
}

// One row tile over n blocks, two at a time.
//   scores(i, s): raw scores;  mask(i, s);  factor(i): what turns them into log2 units;  lv(i): log2 of the value
//   scale;  probs(s, factor, ref, lv): the weights' operand;  values(i, p): O += V^T P^T.
template <int ND, typename P, typename SC, typename MA, typename FA, typename LV, typename PR, typename VA>
__device__ __forceinline__ void attend_blocks(CodeRows<ND> &st, int n, SC scores, MA mask, FA factor, LV lv, PR probs,
                                              VA values) {
  int i = 0;
  float ref;
  for (; i + 2 <= n; i += 2) {
    f32x16 s[2];
    scores(i, s[0]);
    scores(i + 1, s[1]);
    mask(i, s[0]);
    mask(i + 1, s[1]);
    float f[2] = {factor(i), factor(i + 1)};
    const float at[2] = {lv(i), lv(i + 1)};
    st.raise(s, f, at, ref);
    const P p0 = probs(s[0], f[0], ref, at[0]);
    values(i, p0);
    const P p1 = probs(s[1], f[1], ref, at[1]);
    values(i + 1, p1);
  }
  if (i < n) {
    f32x16 s[1];
    scores(i, s[0]);
    mask(i, s[0]);
    float f[1] = {factor(i)};
    const float at[1] = {lv(i)};
    st.raise(s, f, at, ref);
    values(i, probs(s[0], f[0], ref, at[0]));
  }
}

template <typename T, int NK> struct QCodes {      // query operands: NQ bf16 terms
  static constexpr int NQ = sizeof(T) == 4 ? 3 : 1;
  bf16x8 f[NQ][NK];
  // MFMA kk = 2 j + u takes d = 32 j + 16 h + 8 u .. + 7 (the order of the key codes)
  static __device__ __forceinline__ int d_of(int kk, int h) { return 32 * (kk >> 1) + 16 * h + 8 * (kk & 1); }
  __device__ __forceinline__ void set(int kk, const u32x4 &x) { f[0][kk] = __builtin_bit_cast(bf16x8, x); }
  __device__ __forceinline__ void set(int kk, const u32x4 &x0, const u32x4 &x1) {   // 8 floats
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = __uint_as_float(e < 4 ? x0[e & 3] : x1[e & 3]);
      const bf16 a = (bf16)x;
      const float ra = x - (float)a;
      const bf16 b = (bf16)ra;
      f[0][kk][e] = a;
      f[1][kk][e] = b;
      f[2][kk][e] = (bf16)(ra - (float)b);
    }
  }
  __device__ __forceinline__ void load(const T *row, bool live, int h) {
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      const int c = d_of(kk, h);
      u32x4 x{0, 0, 0, 0}, y{0, 0, 0, 0};
      if (live) {
        x = *(const u32x4 *)(row + c);
        if constexpr (sizeof(T) == 4) y = *(const u32x4 *)(row + c + 4);
      }
      if constexpr (sizeof(T) == 4) set(kk, x, y);
      else set(kk, x);
    }
  }
};

__device__ __forceinline__ bf16x8 widen_bf16(uint32_t w0, uint32_t w1) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ f16x8 widen_f16(uint32_t w0, uint32_t w1) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.f, false);
  const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.f, false);
  const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.f, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The bytes of a lane's 16 value codes (half h of a block) whose tokens are below `left`.
__device__ __forceinline__ u32x4 keep_tokens(u32x4 x, int left, int h) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {                     // word 2 t + a: tokens 16 t + 8 a + 4 h + 0..3
    const int n = left - (16 * (w >> 1) + 8 * (w & 1) + 4 * h);
    x[w] &= n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
  }
  return x;
}

// 1 KB of codes (a lane's 16) widened into a block's operand fragments in LDS: piece `sub` of the keys
// (sub < NL) or values.
template <int NL>
__device__ __forceinline__ void widen_to(u32x4 *block, int sub, const u32x4 &x, int lane) {
  u32x4 *to = block + 2 * sub * 64 + lane;
  if (sub < NL) {
    to[0] = __builtin_bit_cast(u32x4, widen_bf16(x[0], x[1]));
    to[64] = __builtin_bit_cast(u32x4, widen_bf16(x[2], x[3]));
  } else {
    to[0] = __builtin_bit_cast(u32x4, widen_f16(x[0], x[1]));
    to[64] = __builtin_bit_cast(u32x4, widen_f16(x[2], x[3]));
  }
}

// Raw scores of one block from its key fragments in LDS (fr: this lane's).
template <typename T, int NK>
__device__ __forceinline__ void kv8_scores(f32x16 &s, const QCodes<T, NK> &q, const u32x4 *fr) {
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
  for (int kk = 0; kk < NK; ++kk) {
    const bf16x8 kf = __builtin_bit_cast(bf16x8, fr[kk * 64]);
#pragma unroll
    for (int t = QCodes<T, NK>::NQ - 1; t >= 0; --t) mfma32(s, kf, q.f[t][kk]);   // small terms first
  }
}

// Weights of one block, 2^(ksc s - ref + c), as fp16 (fp32 calls: two terms); their sum, times w, joins l.
template <typename T> struct CodeProbs { f16x8 f[2], lo[sizeof(T) == 4 ? 2 : 1]; };
template <typename T, int ND>
__device__ __forceinline__ CodeProbs<T> code_probs(const f32x16 &s, float ksc, float ref, float lv, CodeRows<ND> &st) {
  const auto sh = st.share(lv);
  CodeProbs<T> o;
  float sum = 0.f;
  const float c = sh.c - ref;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float p = __builtin_amdgcn_exp2f(fmaf(s[i], ksc, c));
    sum += p;
    o.f[i >> 3][i & 7] = (f16)p;
    if constexpr (sizeof(T) == 4) o.lo[i >> 3][i & 7] = (f16)(p - (float)o.f[i >> 3][i & 7]);
  }
  st.l = fmaf(sum, sh.w, st.l);
  return o;
}
// O += V^T P^T; vf(n, f): value operand of d block n, keys 16 f ..
// 0 x NaN is NaN: a NaN value reaches the rows that do not see its token, too. Where a tile's rows see different
// tokens and its O holds NaN (some_nan), the tile is done again with FINITE, which takes NaN as -448, and
// spread_nan brings NaN to the rows that see them.
template <typename T, int ND, bool FINITE, typename VF>
__device__ __forceinline__ void code_values(f32x16 (&o)[ND], const CodeProbs<T> &p, VF vf) {
#pragma unroll
  for (int f = 0; f < 2; ++f)
#pragma unroll
    for (int n = 0; n < ND; ++n) {
      f16x8 v = vf(n, f);
      if constexpr (FINITE) v = __builtin_elementwise_max(v, f16x8{} - (f16)448.f);   // (of a number and NaN, the number)
      mfma32(o[n], v, p.f[f]);
      if constexpr (sizeof(T) == 4) mfma32(o[n], v, p.lo[f]);
    }
}
template <int ND> __device__ __forceinline__ bool some_nan(const f32x16 (&o)[ND]) {   // of the wave (or infinities of both signs)
  float sum = 0.f;
#pragma unroll
  for (int n = 0; n < ND; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += o[n][r];
  return __any(sum != sum);
}
template <bool X> struct Finite { static constexpr bool value = X; };

// What the rows of a tile see of a sequence: its length; the keys of the tile's first and last row,
// and of this lane's row.
struct Seen {
  int kv, tile_lo, tile_hi, row_hi;
  __device__ __forceinline__ bool uneven(int blocks) const { return tile_lo < min(blocks * 32, kv); }   // some of the first blocks
};
__device__ __forceinline__ Seen seen_of(const Kv8AttnArgs &a, const CondSeq &sq, int first_tok, int last_tok, int tok) {
  Seen v;
  v.kv = min(max(uniform_at(a.c.kv_lens, sq.k0), 0), a.c.width * 32);
  const int before = v.kv - sq.k_len + 1;           // keys of token 0, causal
  v.tile_lo = a.causal ? min(max(before + first_tok, 0), v.kv) : v.kv;
  v.tile_hi = a.causal ? min(max(before + last_tok, 0), v.kv) : v.kv;
  v.row_hi = a.causal ? min(max(before + tok, 0), v.kv) : v.kv;
  return v;
}

// What scores of a block's key codes are multiplied by; never 0 or infinite, so that a masked score stays -inf
// and one of 0 stays 0. (Beyond either end no query that is not 0 has a score within fp32.)
__device__ __forceinline__ float key_factor(float ks, float sc) { return fminf(fmaxf(ks * sc, 0x1p-149f), 0x1.fffffep127f); }

// A block of the pool, or none: its number times heads + g, and its scales (vs < 0: none).
struct BlockRef { int64_t at; float ks, vs; };
__device__ __forceinline__ BlockRef block_ref(const Kv8View &c, int id, int g) {
  const bool ok = id >= 0 && id < c.n_blocks;
  BlockRef b;
  b.at = (int64_t)(ok ? id : 0) * c.hkv + g;
  b.ks = uniform_at(c.scales, b.at * 2);
  b.vs = ok ? uniform_at(c.scales, b.at * 2 + 1) : -1.f;
  return b;
}

// Rows that see a NaN value of block b get NaN in its channel: a product of where they are (1, else 0) and which
// of the block's tokens a row sees, those below `left`.
template <int D>
__device__ __forceinline__ void spread_nan(f32x16 (&o)[D / 32], const Kv8View &c, const int32_t *tab, int b, int g, int left,
                                           int lane) {
  const BlockRef ref = block_ref(c, uniform_at(tab, b), g);
  if (!(ref.vs > 0.f)) return;
  const u32x4 *vp = (const u32x4 *)(c.v_codes + ref.at * (32 * D)) + (lane & 31) * 2 + (lane >> 5);
  f16x8 sees[2];
#pragma unroll
  for (int i = 0; i < 16; ++i) sees[i >> 3][i & 7] = 8 * (i >> 2) + (i & 3) < left - 4 * (lane >> 5) ? (f16)1.f : (f16)0.f;
#pragma unroll
  for (int n = 0; n < D / 32; ++n) {
    const u32x4 x = vp[64 * n];
    f32x16 hits;
#pragma unroll
    for (int i = 0; i < 16; ++i) hits[i] = 0.f;
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      f16x8 at;
#pragma unroll
      for (int e = 0; e < 8; ++e) at[e] = ((x[2 * f + (e >> 2)] >> (8 * (e & 3))) & 0x7F) == 0x7F ? (f16)1.f : (f16)0.f;
      mfma32(hits, at, sees[f]);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) o[n][i] = hits[i] > 0.f ? NAN : o[n][i];
    __builtin_amdgcn_sched_barrier(0);                  // one d block's registers at a time
  }
}

// Least blocks of a split: below that a partial result costs more than its keys.
constexpr int kRowsLeast = 8, kTilesLeast = 4;

// How the few-row kernel cuts its sequences, of lengths only the device knows, into parts of equal
// work: all blocks of the launch over `target` parts (for each kv head) give the blocks of one, every
// sequence has as many as it fills (one at least), and part `at` is found by a running sum over the
// sequences. Every wave computes the same.
struct Cut { int seq, lo, hi, first, used; };       // blocks [lo, hi) of a sequence; its parts: first .. first + used - 1
__device__ __forceinline__ int wave_scan(int x, int lane) {   // inclusive
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d, kWave);
    if (lane >= d) x += y;
  }
  return x;
}
// by_part: the part is `at`; else the cut of sequence `at` as a whole (lo, hi unused).
__device__ __forceinline__ Cut cut_of(const Kv8AttnArgs &a, int target, int at, bool by_part, int lane) {
  static_assert(kCondSeqs == 128, "two sequences a lane");
  int nb[2], c[2];
  double total = 0;                                 // up to 128 sequences of 2^26 blocks
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = lane + 64 * u;
    nb[u] = 0;
    if (i < a.n_seq) {
      const CondSeq &sq = a.seq[i];
      int len = min(max(a.c.kv_lens[sq.k0], 0), a.c.width * 32);
      if (a.causal) len = max(len - (sq.k_len - sq.q_len), 0);   // what its last row sees
      nb[u] = (len + 31) >> 5;
    }
    total += nb[u];
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) total += __shfl_xor(total, m, kWave);
  const int per = max((int)min(ceil(total / target), 0x1p26), kRowsLeast);
  int run[2], before = 0;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    c[u] = lane + 64 * u < a.n_seq ? max(1, (nb[u] + per - 1) / per) : 0;
    run[u] = before + wave_scan(c[u], lane);
    before = __shfl(run[u], 63, kWave);
  }
  Cut w{-1, 0, 0, 0, 0};
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = lane + 64 * u, first = run[u] - c[u];
    const uint64_t hit = __ballot(by_part ? c[u] > 0 && first <= at && at < run[u] : i == at);
    if (hit) {                                      // wave-uniform
      const int l = __builtin_ctzll(hit);
      w.seq = l + 64 * u;
      w.first = __shfl(first, l, kWave);
      w.used = __shfl(c[u], l, kWave);
      const int n = __shfl(nb[u], l, kWave);
      w.lo = min((at - w.first) * per, n);
      w.hi = min(w.lo + per, n);
    }
  }
  w.seq = __builtin_amdgcn_readfirstlane(w.seq);
  w.lo = __builtin_amdgcn_readfirstlane(w.lo);
  w.hi = __builtin_amdgcn_readfirstlane(w.hi);
  w.first = __builtin_amdgcn_readfirstlane(w.first);
  w.used = __builtin_amdgcn_readfirstlane(w.used);
  return w;
}

// Few rows (at most 32 a sequence, or chunk of one): bound by the codes that stream in. Each of the four waves
// takes every fourth block of the split's range and loads its codes straight into MFMA operand
// order, 16 bytes a lane and 1 KB a load, the next block's while one is computed. One token of 2 x 8 heads
// of 128 over 131071: 58.6 us with the join, 4.6 TB/s; 32 over 96 to 8192: 55.8 us, 4.1 TB/s (parts of
// equal tables instead of equal work: 115); in fp32 queries, one wave a SIMD, 70 us.
template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 1 : 2) void k_kv8_rows(Kv8AttnArgs a, int target) {
  constexpr int ND = D / 32, NK = D / 16, NL = D / 32;
  extern __shared__ u32x4 lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lrow = lane & 31, h = lane >> 5;
  const int part = (int)blockIdx.x / a.hkv, g = (int)blockIdx.x - part * a.hkv;
  const Cut span = cut_of(a, target, part, true, lane);
  if (span.seq < 0) return;                         // fewer parts than the grid has room for
  const CondSeq sq = a.seq[span.seq];
  const int rows = sq.q_len * a.rep, r = lrow;
  const bool live = r < rows;
  const int qi = live ? r / a.rep : 0;
  const int head = g * a.rep + (live ? r % a.rep : 0);
  const Seen seen = seen_of(a, sq, 0, sq.q_len - 1, qi);

  const int32_t *tab = a.c.table + (int64_t)sq.k0 * a.c.table_row;
  auto id_at = [&](int b) { return b < span.hi ? uniform_at(tab, b) : -1; };
  struct Block { u32x4 k[NL], v[NL]; BlockRef ref; };
  auto load = [&](int id, Block &x) {
    x.ref = block_ref(a.c, id, g);
    const u32x4 *kp = (const u32x4 *)(a.c.k_codes + x.ref.at * (32 * D)) + lane;
    const u32x4 *vp = (const u32x4 *)(a.c.v_codes + x.ref.at * (32 * D)) + lrow * 2 + h;
#pragma unroll
    for (int i = 0; i < NL; ++i) x.k[i] = kp[64 * i];
#pragma unroll
    for (int i = 0; i < NL; ++i) x.v[i] = vp[64 * i];
  };
  QCodes<T, NK> q;
  CodeRows<ND> st;
  const int b0 = span.lo + wave;
  auto pass = [&](auto finite) {
    typedef decltype(finite) F;
    st.init();
    Block cur, nxt;
    int id = id_at(b0 + 4);
    if (b0 < span.hi) load(id_at(b0), cur);
    if constexpr (!F::value) q.load((const T *)a.q + (int64_t)(sq.q0 + qi) * a.q_row + (int64_t)head * a.q_head, live, h);
    for (int b = b0; b < span.hi; b += 4) {
      if (b + 4 < span.hi) load(id, nxt);
      id = id_at(b + 8);
      if (cur.ref.vs > 0.f) {
        f32x16 s[1];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[0][i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < NK; ++kk) {
          const bf16x8 kf = widen_bf16(cur.k[kk >> 1][2 * (kk & 1)], cur.k[kk >> 1][2 * (kk & 1) + 1]);
#pragma unroll
          for (int t = q.NQ - 1; t >= 0; --t) mfma32(s[0], kf, q.f[t][kk]);   // small terms first
        }
        const int left = seen.kv - b * 32;
        if (left < 32 || b * 32 + 32 > seen.tile_lo) {  // wave-uniform
          mask_below(s[0], seen.row_hi - b * 32, lane);
          if (left < 32) {
#pragma unroll
            for (int i = 0; i < NL; ++i) cur.v[i] = keep_tokens(cur.v[i], left, h);
          }
        }
        float ksc[1] = {key_factor(cur.ref.ks, a.sc)}, ref;
        const float lv[1] = {scale_log(cur.ref.vs)};
        st.raise(s, ksc, lv, ref);
        code_values<T, ND, F::value>(st.o, code_probs<T>(s[0], ksc[0], ref, lv[0], st),
                                     [&](int n, int f) { return widen_f16(cur.v[n][2 * f], cur.v[n][2 * f + 1]); });
      }
      cur = nxt;
    }
  };
  pass(Finite<false>{});
  if (seen.uneven(span.hi) && some_nan<ND>(st.o)) {
    pass(Finite<true>{});
    for (int b = b0; b < span.hi; b += 4) spread_nan<D>(st.o, a.c, tab, b, g, seen.row_hi - b * 32, lane);
  }
  float *red = (float *)lds;
  match_waves<ND, 4>(st, red, wave, lane);
  join_waves<ND, 4>(st, red, wave, lane);
  if (wave > 0) return;
  const float unit = st.unit();
  if (span.used == 1)
    store_rows<T, ND>(a, st, unit, live, sq.q0 + qi, head, lane);
  else
    store_part<ND>(a, st, unit, live, part, g, 0, lrow, lane);
}

// Many rows: four waves of 32 rows; two blocks of codes a step are widened once per
// workgroup on their way into LDS, in MFMA operand order (1 KB of lanes a fragment,
// free of bank conflicts). The next step's codes are loaded into registers before a step is computed, but arrive
// before its products: which block a wave loads goes by its number, so that the block references are kept in
// scratch (80 bytes a lane), and what is read back from there waits for all loads before it. Bound by those
// waits, at one to three waves a SIMD (1000 of 2 x 8 heads of 128 over 1000, causal, in four parts: 31.2 us,
// 131 TFLOP/s; 512 over 4096, causal, 47 us, 342 TFLOP/s).
template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 1 : 2) void k_kv8_tiles(Kv8AttnArgs a) {
  constexpr int ND = D / 32, NK = D / 16, NL = D / 32;
  constexpr int PIECES = 4 * NL;                    // 1 KB loads of a step: 2 blocks x (k, v) x NL
  constexpr int PPW = PIECES / 4;
  extern __shared__ u32x4 lds[];                    // [block][NK key + 2 ND value fragments][64 lanes]
  __shared__ int again[4];                          // waves whose O holds NaN
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lrow = lane & 31, h = lane >> 5;
  const Unit un = unit_of(a.hkv);
  const int tile = un.tile, g = un.g, split = blockIdx.y;
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, tile)];
  const int rows = sq.q_len * a.rep, t0 = (tile - sq.tile0) * 128, r0 = t0 + wave * 32, r = r0 + lrow;
  const bool live = r < rows;
  const int qi = live ? r / a.rep : 0;
  const int head = g * a.rep + (live ? r % a.rep : 0);
  const Seen seen = seen_of(a, sq, min(r0, rows - 1) / a.rep, (min(t0 + 128, rows) - 1) / a.rep, qi);
  const Span span = split_span((seen.tile_hi + 31) >> 5, a.n_split, split, kTilesLeast);
  if (split >= span.used) return;

  const int32_t *tab = a.c.table + (int64_t)sq.k0 * a.c.table_row;
  auto id_at = [&](int b) { return b < span.hi ? uniform_at(tab, b) : -1; };
  u32x4 x[PPW];
  auto gload = [&](int b, const BlockRef (&ref)[2]) {
#pragma unroll
    for (int i = 0; i < PPW; ++i) {
      const int p = wave * PPW + i, blk = p / (2 * NL), sub = p % (2 * NL);
      const BlockRef &r = ref[blk];
      if (sub < NL) {
        x[i] = ((const u32x4 *)(a.c.k_codes + r.at * (32 * D)))[64 * sub + lane];
      } else {
        x[i] = ((const u32x4 *)(a.c.v_codes + r.at * (32 * D)))[64 * (sub - NL) + lrow * 2 + h];
        const int left = seen.kv - (b + blk) * 32;
        if (left < 32) x[i] = keep_tokens(x[i], left, h);
      }
    }
  };
  auto lstore = [&]() {
#pragma unroll
    for (int i = 0; i < PPW; ++i) {
      const int p = wave * PPW + i, blk = p / (2 * NL), sub = p % (2 * NL);
      widen_to<NL>(lds + blk * 4 * NL * 64, sub, x[i], lane);
    }
  };
  QCodes<T, NK> q;
  CodeRows<ND> st;
  auto pass = [&](auto finite) {
    typedef decltype(finite) F;
    BlockRef cur[2], nxt[2];
    int id[2] = {id_at(span.lo + 2), id_at(span.lo + 3)};
    if (span.lo < span.hi) {
#pragma unroll
      for (int u = 0; u < 2; ++u) cur[u] = block_ref(a.c, id_at(span.lo + u), g);
      gload(span.lo, cur);
    }
    if constexpr (!F::value) q.load((const T *)a.q + (int64_t)(sq.q0 + qi) * a.q_row + (int64_t)head * a.q_head, live, h);
    st.init();
    for (int b = span.lo; b < span.hi; b += 2) {
      __syncthreads();
      lstore();
      __syncthreads();
      if (b + 2 < span.hi) {
#pragma unroll
        for (int u = 0; u < 2; ++u) nxt[u] = block_ref(a.c, id[u], g);
        gload(b + 2, nxt);
#pragma unroll
        for (int u = 0; u < 2; ++u) id[u] = id_at(b + 4 + u);
      }
      if (r0 < rows) {                              // wave-uniform: others still load and meet the barriers
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (cur[u].vs > 0.f) {
            const u32x4 *fr = lds + u * 4 * NL * 64 + lane;
            f32x16 s[1];
            kv8_scores<T, NK>(s[0], q, fr);
            if ((b + u) * 32 + 32 > seen.tile_lo) mask_below(s[0], seen.row_hi - (b + u) * 32, lane);
            float ksc[1] = {key_factor(cur[u].ks, a.sc)}, ref;
            const float lv[1] = {scale_log(cur[u].vs)};
            st.raise(s, ksc, lv, ref);
            code_values<T, ND, F::value>(st.o, code_probs<T>(s[0], ksc[0], ref, lv[0], st),
                                         [&](int n, int f) { return __builtin_bit_cast(f16x8, fr[(NK + 2 * n + f) * 64]); });
          }
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) cur[u] = nxt[u];
    }
  };
  pass(Finite<false>{});
  if (a.causal) {                                   // uniform
    const bool mine = r0 < rows && seen.uneven(span.hi) && some_nan<ND>(st.o);
    if (lane == 0) again[wave] = mine;
    __syncthreads();
    if (again[0] | again[1] | again[2] | again[3]) {
      pass(Finite<true>{});
      for (int b = span.lo; r0 < rows && b < span.hi; ++b) spread_nan<D>(st.o, a.c, tab, b, g, seen.row_hi - b * 32, lane);
    }
  }
  if (r0 >= rows) return;
  const float unit = st.unit();
  if (span.used == 1)
    store_rows<T, ND>(a, st, unit, live, sq.q0 + qi, head, lane);
  else
    store_part<ND>(a, st, unit, live, tile, g, split, wave * 32 + lrow, lane);
}

// Many rows over a cache that fits LDS whole once widened. Lane j holds block j's scales and how many of
// its tokens count (none: no such block). A wave takes several row tiles over codes widened once.
// 16 x 1024 of 2 x 8 heads of 128 over 320: 61 to 63 us, 690 TFLOP/s, 2.3 TB/s. Of that the matrix cores are busy 17,
// vector instructions about 23 (4900 a wave, two waves a SIMD; an exponential takes four times as long); the rest
// is the staging that a workgroup waits for, and the next rows' queries, issued ahead but waited for before a
// tile's first product.
template <typename T, int D, int NW, bool BOX>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 4 ? 1 : D == 64 ? 3 : 2) void k_kv8_res(Kv8AttnArgs a, int chunk) {
  constexpr int ND = D / 32, NK = D / 16, NL = D / 32, NF = D / 8;
  extern __shared__ u32x4 lds[];                    // [block][NK key + 2 ND value fragments][64 lanes]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lrow = lane & 31, h = lane >> 5;
  const Unit un = unit_of(a.hkv);
  const int tile = un.tile, g = un.g;
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, tile)];
  const int first = (tile - sq.tile0) * chunk;
  const int rows = min(sq.q_len * a.rep, first + chunk);
  const Seen all = seen_of(a, sq, 0, (rows - 1) / a.rep, 0);
  const int nk = (all.tile_hi + 31) >> 5;
  const int32_t *tab = a.c.table + (int64_t)sq.k0 * a.c.table_row;
  u32x4 *box = lds + wave * (kBox / 16);
  u32x4 *codes = lds + (BOX ? NW * (kBox / 16) : 0);

  struct Own { QCodes<T, NK> f; int64_t tok; int head; bool live; };
  auto load_own = [&](int r0, Own &q) {
    const int r = r0 + lrow;
    q.live = r < rows;
    const int t = q.live ? r / a.rep : 0;
    q.tok = sq.q0 + t;
    q.head = g * a.rep + (q.live ? r - t * a.rep : 0);
    q.f.load((const T *)a.q + q.tok * a.q_row + (int64_t)q.head * a.q_head, q.live, h);
  };
  Own q, qn;
  QTile<T, D> qt;
  int r0 = first + wave * 32;
  if (r0 < rows) {
    if constexpr (BOX) qt.load(a, TileRows(a, sq, r0, rows), g, lane);
    else load_own(r0, q);
  }

  float ks = 1.f, lv = 0.f;
  int count = 0;
  if (lane < nk) {
    const int id = tab[lane];
    if (id >= 0 && id < a.c.n_blocks) {
      const int64_t at = (int64_t)id * a.c.hkv + g;
      ks = key_factor(a.c.scales[at * 2], a.sc);
      lv = scale_log(a.c.scales[at * 2 + 1]);
      count = min(all.kv - lane * 32, 32);
    }
  }
  for (int j = wave; j < nk; j += NW) {
    const int id = uniform_at(tab, j);
    const bool ok = id >= 0 && id < a.c.n_blocks;
    const int64_t at = (int64_t)(ok ? id : 0) * a.c.hkv + g;
    const int left = ok ? all.kv - j * 32 : 0;
    u32x4 x[2 * NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      x[i] = ((const u32x4 *)(a.c.k_codes + at * (32 * D)))[64 * i + lane];
      x[NL + i] = ((const u32x4 *)(a.c.v_codes + at * (32 * D)))[64 * i + lrow * 2 + h];
    }
    if (left < 32) {
#pragma unroll
      for (int i = 0; i < NL; ++i) x[NL + i] = keep_tokens(x[NL + i], left, h);
    }
#pragma unroll
    for (int i = 0; i < 2 * NL; ++i) widen_to<NL>(codes + j * NF * 64, i, x[i], lane);
  }
  __syncthreads();
  for (; r0 < rows; r0 += NW * 32) {                // wave-uniform
    const bool more = r0 + NW * 32 < rows;
    const int r = min(r0 + lrow, rows - 1);
    if constexpr (BOX) {
#pragma unroll
      for (int j = 0; j < qt.PARTS; ++j) {
        qt.spread(box, j, lane);
        if constexpr (sizeof(T) == 4) {             // a part of 32 floats: two steps of 16
#pragma unroll
          for (int u = 0; u < 2; ++u)
            q.f.set(2 * j + u, qt.chunk(box, 4 * h + 2 * u, lane), qt.chunk(box, 4 * h + 2 * u + 1, lane));
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u) q.f.set(4 * j + u, qt.chunk(box, 4 * (u >> 1) + 2 * h + (u & 1), lane));
        }
      }
      if (more) qt.load(a, TileRows(a, sq, r0 + NW * 32, rows), g, lane);
    } else if (sizeof(T) == 2 && more) {
      load_own(r0 + NW * 32, qn);
    }
    const Seen seen = seen_of(a, sq, r0 / a.rep, (min(r0 + 32, rows) - 1) / a.rep, r / a.rep);
    CodeRows<ND> st;
    auto lane_of = [](float x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i)); };
    auto pass = [&](auto finite) {
      typedef decltype(finite) F;
      st.init();
      attend_blocks<ND, CodeProbs<T>>(
          st, (seen.tile_hi + 31) >> 5,
          [&](int i, f32x16 &s) { kv8_scores<T, NK>(s, q.f, codes + i * NF * 64 + lane); },
          [&](int i, f32x16 &s) {
            const int n = __builtin_amdgcn_readlane(count, i), at = i * 32;
            if (n < 32 || at + 32 > seen.tile_lo) mask_below(s, min(seen.row_hi - at, n), lane);
          },
          [&](int i) { return lane_of(ks, i); }, [&](int i) { return lane_of(lv, i); },
          [&](const f32x16 &s, float f, float ref, float at) { return code_probs<T>(s, f, ref, at, st); },
          [&](int i, const CodeProbs<T> &p) {
            const u32x4 *fr = codes + (i * NF + NK) * 64 + lane;
            code_values<T, ND, F::value>(st.o, p,
                                         [&](int n, int f) { return __builtin_bit_cast(f16x8, fr[(2 * n + f) * 64]); });
          });
    };
    pass(Finite<false>{});
    if (seen.uneven(nk) && some_nan<ND>(st.o)) {
      pass(Finite<true>{});
      for (int b = 0; b * 32 < seen.tile_hi; ++b) spread_nan<D>(st.o, a.c, tab, b, g, seen.row_hi - b * 32, lane);
    }
    const float unit = st.unit();
    if constexpr (BOX) {
      store_tile<T, ND>(a, st, unit, TileRows(a, sq, r0, rows), g, box, lane);
    } else {
      store_rows<T, ND>(a, st, unit, q.live, q.tok, q.head, lane);
      if (sizeof(T) == 2) q = qn;
      else if (more) load_own(r0 + NW * 32, q);
    }
  }
}

// ---- joining splits -----------------------------------------------------------------------------
//
// out[row] = sum_s w_s O_s / sum_s w_s, w_s = 2^(m_s - M) l_s, M = max m_s, over the parts that a unit
// (tile or sequence, kv head) used; units of one part wrote their rows themselves. A workgroup a row,
// DP / 4 lanes of four d times as many teams over the parts as it holds, so that the parts of a
// row are read in one go (64 parts read by one team each after the other: 12 us).
constexpr int kMostParts = kMaxParts + 1;
template <typename T>
__device__ __forceinline__ void store_joined(const AttnCommon &a, const CondSeq &sq, int g, int r, int c, const f32x4 &x) {
  T *row = (T *)a.out + (int64_t)(sq.q0 + r / a.rep) * a.o_row + (int64_t)(g * a.rep + r % a.rep) * a.o_head;
  if constexpr (sizeof(T) == 4)
    *(f32x4 *)(row + c) = x;
  else
    *(bf16x4 *)(row + c) = bf16x4{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
}
template <typename T, int DP>
__device__ __forceinline__ void join_row(const AttnCommon &a, const CondSeq &sq, int g, int r, int64_t at, int64_t step,
                                         int used) {
  constexpr int LPR = DP / 4, TEAMS = kThreads / LPR;
  __shared__ float weight[kMostParts];
  __shared__ float red[4];
  __shared__ f32x4 sums[TEAMS][LPR];
  const int tid = threadIdx.x, c = (tid % LPR) * 4, team = tid / LPR;
  const float *ml = a.ws + a.ws_ml + at * 2, *o = a.ws + at * DP + c;
  float M = -INFINITY;
  for (int s = tid; s < used; s += kThreads) {
    weight[s] = ml[s * step * 2];
    M = fmaxf(M, weight[s]);
  }
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) M = warp_max_xor(M, k);
  if ((tid & 63) == 0) red[tid >> 6] = M;
  __syncthreads();
  M = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float mr = M == -INFINITY ? 0.f : M;
  __syncthreads();
  float l = 0.f;
  for (int s = tid; s < used; s += kThreads) {
    weight[s] = __builtin_amdgcn_exp2f(weight[s] - mr) * ml[s * step * 2 + 1];
    l += weight[s];
  }
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) l = warp_sum_xor(l, k);
  if ((tid & 63) == 0) red[tid >> 6] = l;
  __syncthreads();
  l = red[0] + red[1] + red[2] + red[3];
  const float inv = l > 0.f ? 1.f / l : 0.f;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = team; s < used; s += TEAMS) {
    const f32x4 x = *(const f32x4 *)(o + s * step * DP);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += weight[s] * inv * x[e];
  }
  sums[team][tid % LPR] = acc;
  __syncthreads();
  if (team > 0 || c >= a.d) return;
#pragma unroll
  for (int k = 1; k < TEAMS; ++k) {
    const f32x4 x = sums[k][tid];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += x[e];
  }
  store_joined<T>(a, sq, g, r, c, acc);
}
// Few parts of many rows: a row for each DP / 4 lanes, its parts all in flight (10000 rows of two parts: 5 us, a
// workgroup a row 12).
constexpr int kFewParts = 8;
template <typename T, int DP>
__device__ __forceinline__ void join_few(const AttnCommon &a, const CondSeq &sq, int g, int r, int64_t at, int64_t step,
                                         int used) {
  const int c = (threadIdx.x % (DP / 4)) * 4;
  const float *ml = a.ws + a.ws_ml + at * 2, *o = a.ws + at * DP + c;
  float w[kFewParts], lp[kFewParts], M = -INFINITY, l = 0.f;
  f32x4 x[kFewParts], acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < kFewParts; ++s) {
    const int64_t k = min(s, used - 1) * step;
    w[s] = s < used ? ml[k * 2] : -INFINITY;
    lp[s] = s < used ? ml[k * 2 + 1] : 0.f;
    x[s] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (s < used) x[s] = *(const f32x4 *)(o + k * DP);
    M = fmaxf(M, w[s]);
  }
  const float mr = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int s = 0; s < kFewParts; ++s) {
    w[s] = __builtin_amdgcn_exp2f(w[s] - mr) * lp[s];
    l += w[s];
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int s = 0; s < kFewParts; ++s)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += w[s] * inv * x[s][e];
  if (c < a.d) store_joined<T>(a, sq, g, r, c, acc);
}
// The row of a tile of TR that a thread joins, given the grid's y: WIDE, one a workgroup.
template <int DP, bool WIDE> __device__ __forceinline__ int join_index() {
  return WIDE ? blockIdx.y : blockIdx.y * (kThreads / (DP / 4)) + threadIdx.x / (DP / 4);
}

// Grid: x = (row tile, kv head), y = rows of the tile (join_index). The sequences are those that were
// split: k0 = their first unit, k_len = its parts, tile0 = their first tile here.
template <typename T, int DP, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_cross_join(CrossArgs a, int TR) {
  const Unit un = unit_of(a.hkv);
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, un.tile)];
  const int rows = sq.q_len * a.rep, t = un.tile - sq.tile0, i = join_index<DP, WIDE>(), tiles = (rows + TR - 1) / TR;
  if (i >= TR || t * TR + i >= rows) return;
  const int64_t at = ((int64_t)(sq.k0 + t) * a.hkv + un.g) * a.ws_rows + i, step = (int64_t)tiles * a.hkv * a.ws_rows;
  if constexpr (WIDE) join_row<T, DP>(a, sq, un.g, t * TR + i, at, step, sq.k_len);
  else join_few<T, DP>(a, sq, un.g, t * TR + i, at, step, sq.k_len);
}

// Grid: x = (tile, kv head), y = rows of the tile.
template <typename T, int DP, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_kv8_tiles_join(Kv8AttnArgs a) {
  const Unit un = unit_of(a.hkv);
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, un.tile)];
  const int rows = sq.q_len * a.rep, r0 = (un.tile - sq.tile0) * 128, i = join_index<DP, WIDE>();
  if (i >= 128 || r0 + i >= rows) return;
  const int last = (min(r0 + 128, rows) - 1) / a.rep;
  const int used = split_span((seen_of(a, sq, 0, last, 0).tile_hi + 31) >> 5, a.n_split, 0, kTilesLeast).used;
  if (used == 1) return;
  const int64_t at = ((int64_t)un.tile * a.hkv + un.g) * a.n_split * a.ws_rows + i;
  if constexpr (WIDE) join_row<T, DP>(a, sq, un.g, r0 + i, at, a.ws_rows, used);
  else join_few<T, DP>(a, sq, un.g, r0 + i, at, a.ws_rows, used);
}

template <typename T, int DP>
__global__ __launch_bounds__(kThreads) void k_kv8_rows_join(Kv8AttnArgs a, int target) {
  const Unit un = unit_of(a.hkv);
  const CondSeq sq = a.seq[un.tile];
  const int i = blockIdx.y;
  if (i >= sq.q_len * a.rep) return;
  const Cut w = cut_of(a, target, un.tile, false, threadIdx.x & 63);
  if (w.used == 1) return;
  join_row<T, DP>(a, sq, un.g, i, ((int64_t)w.first * a.hkv + un.g) * a.ws_rows + i, (int64_t)a.hkv * a.ws_rows,
                  w.used);
}

// ---- plans --------------------------------------------------------------------------------------

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// How a class of query sequences is launched: TR rows a tile, the same number of splits for all.
struct Plan {
  enum { FEW, COPIES, STREAM, RESIDENT } kind = FEW;
  int TR = 0, KT = 0, n_split = 1, ws_rows = 0;
  KeyCut cut{0, 0};                                 // cross attention: see part_of
  int target = 0;                                   // cached attention with few rows: parts (cut_of), 0: none
  int nw = 4, lds = 0;                              // RESIDENT: waves, LDS bytes,
  bool box = false;                                 // and whether they hold kBox a wave
  bool split = false;                               // cross attention: some sequence has parts
  int64_t tiles = 0;                                // of the launch (of kCondSeqs sequences) with the most
  int64_t floats(int hkv, int dp) const {
    return n_split > 1 || target > 0 || split ? tiles * hkv * n_split * (int64_t)ws_rows * (dp + 2) : 0;
  }
  int64_t ml(int hkv, int dp) const { return tiles * hkv * n_split * (int64_t)ws_rows * dp; }
};

int pad_d(int d) { return d <= 64 ? 64 : 128; }

// Workgroups that fill the 256 compute units with two each; a launch below it splits long key ranges.
constexpr int kFill = 512;
static_assert(kFill <= kMaxParts, "splits of one unit");

}  // namespace

// Row tiles of 32 and the most rows of one query sequence among those that `take` accepts.
template <typename TAKE>
static void count_rows(const AttnProblem &p, int64_t &tiles, int64_t &most, TAKE take) {
  tiles = most = 0;
  for (int i = 0; i < p.n; ++i) {
    const int64_t rows = (int64_t)p.q_lens[i] * p.c.rep;
    if (rows == 0 || !take(i)) continue;
    tiles += ceil_div(rows, 32);
    most = std::max(most, rows);
  }
}

// Tiles of TR rows: of the launch (of kCondSeqs sequences) with the most, and of all.
template <typename TAKE>
static int64_t fill_tiles(const AttnProblem &p, Plan &pl, TAKE take) {
  int64_t all = 0, at = 0;
  int in = 0;
  pl.tiles = 0;
  for (int i = 0; i < p.n; ++i) {
    const int64_t rows = (int64_t)p.q_lens[i] * p.c.rep;
    if (rows == 0 || !take(i)) continue;
    const int t = ceil_div(rows, pl.TR);
    all += t;
    at += t;
    pl.tiles = std::max(pl.tiles, at);
    if (++in == kCondSeqs) in = at = 0;
  }
  return all;
}

// The kernel and its splits:
//  FEW: up to 32 rows a sequence, or fewer than 256 tiles of 32 rows in all: a workgroup per tile, its four
//    waves split the keys (1871 fp32 rows over up to 320 keys: 15 us, against 24 with tiles of 128
//    rows; 1024 bf16 rows of 10 heads, 320 tiles, over 96: 6.5, against 5.6).
//  COPIES (bf16): tiles of 128 rows, keys by LDS-direct copies.
//  STREAM (fp32, or rows too far apart for 32-bit offsets): tiles of 128 rows, keys by registers.
// Key ranges are cut into parts of the work that fills the chip once, kFill workgroups: few rows over long keys
// are cut, and so is one long range among many short ones, whose workgroups would run on alone. Parts
// are of 256 keys at least (fp32 FEW: 128), and ranges are cut from the length at which that saves more than
// the join costs, 4 us of a replayed graph and 6 of an eager call: 2 parts, FEW 1024 keys (fp32, where
// a tile takes 3.5 or 7 us: 512 or 384). us cut / whole, replayed: one token of 2 x 8 heads of 128 over 1024,
// bf16 11.7 / 15.5 (of two parts), fp32 14.3 / 32.3; 1500 rows of 12 heads, 9 sequences over 6 to 963
// keys, those under 12 rows, 15.2 / 27.8; 2500 rows of 8 heads over 356 (below two parts) 18.0 / 13.7; eager: 64
// of 8 heads of 64 over 700 (below 1024) 18.0 / 12.6.
static Plan cross_plan(const AttnProblem &p, const int32_t *kv_lens, const int32_t *kv_index) {
  Plan pl;
  int64_t row_tiles, most;
  const auto any = [](int) { return true; };
  count_rows(p, row_tiles, most, any);
  if (row_tiles == 0) return pl;
  pl.TR = 128;
  int least;
  if (most <= 32 || row_tiles * p.c.hkv < 256) {
    pl.kind = Plan::FEW;
    pl.TR = 32;
    pl.KT = 128;
    least = p.dtype == MTE_BF16 ? 2 : 1;
    pl.cut.from = p.dtype == MTE_BF16 ? 8 : p.c.d > 64 ? 3 : 4;
  } else if (p.dtype == MTE_BF16 && p.near_rows && p.near_tiles) {
    pl.kind = Plan::COPIES;
    pl.KT = 32;
    least = 8;
  } else {
    pl.kind = Plan::STREAM;
    pl.KT = p.dtype == MTE_BF16 ? 64 : 32;
    least = 256 / pl.KT;
  }
  const auto each = [&](auto fn) {                   // row tiles and key tiles of every sequence with rows
    for (int i = 0; i < p.n; ++i)
      if (p.q_lens[i] > 0) fn(ceil_div((int64_t)p.q_lens[i] * p.c.rep, pl.TR), ceil_div(kv_lens[kv_index ? kv_index[i] : i], pl.KT));
  };
  double work = 0;
  each([&](int rows, int keys) { work += (double)rows * keys; });
  pl.cut.per = (int)std::min(std::max((double)least, std::ceil(work * p.c.hkv / kFill)), 0x1p29);
  // no more parts than a join takes
  each([&](int, int keys) { pl.cut.per = std::max(pl.cut.per, ceil_div(keys, kMaxParts - 1)); });
  int64_t at = 0;
  int in = 0;
  each([&](int rows, int keys) {
    const int used = parts_of(keys, pl.cut);
    pl.split |= used > 1;
    if (used > 1) at += (int64_t)rows * used;        // (place_units: the others have no partial results)
    pl.tiles = std::max(pl.tiles, at);
    if (++in == kCondSeqs) in = at = 0;
  });
  pl.ws_rows = (int)std::min<int64_t>(pl.TR, most);
  return pl;
}

// Whether the rows written are more than the caches in front of memory keep until they are read again
// (32 MB of L2): such stores bypass them. 16 x 4096 rows of 10 heads of 64: 46.2 us against 51.3.
static int big_out(const AttnProblem &p) {
  int64_t rows = 0;
  for (int i = 0; i < p.n; ++i) rows += p.q_lens[i];
  return rows * p.c.rep * p.c.hkv * p.c.d * (p.dtype == MTE_BF16 ? 2 : 4) > (32 << 20);
}

int64_t cross_workspace(const AttnProblem &p, const int32_t *kv_lens, int, const int32_t *kv_index) {
  return cross_plan(p, kv_lens, kv_index).floats(p.c.hkv, pad_d(p.c.d)) * 4;
}

// Fills a.seq with the next query sequences that `take` accepts (up to kCondSeqs); returns their tiles.
template <typename A, typename TAKE>
static int next_seqs(A &a, const AttnProblem &p, int &i, int &row, int TR, TAKE take) {
  int tiles = 0;
  a.n_seq = 0;
  for (; i < p.n && a.n_seq < kCondSeqs; ++i) {
    const int len = p.q_lens[i];
    if (len > 0 && take(i, a.seq[a.n_seq])) {
      CondSeq &s = a.seq[a.n_seq++];
      s.q0 = row;
      s.q_len = len;
      s.tile0 = tiles;
      tiles += ceil_div((int64_t)len * a.rep, TR);
    }
    row += len;
  }
  return tiles;
}

template <typename K>
static hipError_t allow_lds(K kern, int bytes) {
  return bytes <= 65536 ? hipSuccess
                        : hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

// Workgroups for the rows of a tile (join_index).
template <int DP> int join_grid(int parts, int rows) { return parts > kFewParts ? rows : ceil_div(rows, kThreads / (DP / 4)); }

// The units of a launch's sequences: first those of split ones (the workspace ends after them), then longest
// first, so that the last workgroups to start are the shortest.
static int place_units(CrossArgs &a, const Plan &pl) {
  const auto rank = [&](const CondSeq &q) {
    const int nt = ceil_div(q.k_len, pl.KT);
    return parts_of(nt, pl.cut) > 1 ? INT_MAX : nt;
  };
  std::stable_sort(a.seq, a.seq + a.n_seq, [&](const CondSeq &x, const CondSeq &y) { return rank(x) > rank(y); });
  int units = 0;
  for (int i = 0; i < a.n_seq; ++i) {
    CondSeq &q = a.seq[i];
    q.tile0 = units;
    units += ceil_div((int64_t)q.q_len * a.rep, pl.TR) * parts_of(ceil_div(q.k_len, pl.KT), pl.cut);
  }
  return units;
}

template <typename T, int DP>
static hipError_t run_cross(CrossArgs &a, const Plan &pl, hipStream_t s) {
  const int units = place_units(a, pl);
  hipError_t e;
  auto kern = pl.kind == Plan::FEW ? k_cross<T, DP, 1> : k_cross<T, DP, 4>;
  int lds = 2 * pl.KT * DP * (int)sizeof(T) + 32;
  if (pl.kind == Plan::FEW) lds = std::max(lds, 3 * (2 + DP / 2) * 64 * 4);
  if constexpr (sizeof(T) == 2) {
    if (pl.kind == Plan::COPIES) {
      kern = k_cross_stream<DP>;
      lds = Stream<DP>::BYTES;
    }
  }
  if ((e = allow_lds(kern, lds)) != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(units * a.hkv), dim3(kThreads), lds, s, a);
  if ((e = hipGetLastError()) != hipSuccess || !pl.split) return e;
  int n = 0, tiles = 0, most = 0;
  for (int i = 0; i < a.n_seq; ++i) {
    CondSeq q = a.seq[i];
    const int used = parts_of(ceil_div(q.k_len, pl.KT), pl.cut);
    if (used == 1) continue;
    q.k0 = q.tile0;
    q.k_len = used;
    most = std::max(most, used);
    q.tile0 = tiles;
    tiles += ceil_div((int64_t)q.q_len * a.rep, pl.TR);
    a.seq[n++] = q;
  }
  if (n == 0) return e;                             // none in this launch
  a.n_seq = n;
  auto join = most > kFewParts ? k_cross_join<T, DP, true> : k_cross_join<T, DP, false>;
  hipLaunchKernelGGL(join, dim3(tiles * a.hkv, join_grid<DP>(most, a.ws_rows)), dim3(kThreads), 0, s, a, pl.TR);
  return hipGetLastError();
}

hipError_t launch_cross(const AttnProblem &p, const void *k, const void *v, const uint8_t *mask, int64_t k_row,
                        int64_t k_head, int64_t v_row, int64_t v_head, const int32_t *kv_lens, int n_kv,
                        const int32_t *kv_index, hipStream_t s) {
  const Plan pl = cross_plan(p, kv_lens, kv_index);
  const int dp = pad_d(p.c.d);
  CrossArgs a;
  (AttnCommon &)a = p.c;
  a.big = big_out(p);
  a.k = k;
  a.v = v;
  a.mask = mask;
  a.k_row = k_row;
  a.k_head = k_head;
  a.v_row = v_row;
  a.v_head = v_head;
  a.cut = pl.cut;
  a.n_split = 1;
  a.ws_rows = pl.ws_rows;
  a.ws_ml = pl.ml(a.hkv, dp);
  // first key row of the sequence a query sequence names: a running sum, taken up again from the
  // start where the index goes back
  int at = 0;
  int64_t first = 0;
  auto take = [&](int i, CondSeq &sq) {
    const int j = kv_index ? kv_index[i] : i;
    if (j < at) { at = 0; first = 0; }
    for (; at < j; ++at) first += kv_lens[at];
    sq.k0 = (int)first;
    sq.k_len = kv_lens[j];
    return true;
  };
  for (int i = 0, row = 0; i < p.n;) {
    const int tiles = next_seqs(a, p, i, row, pl.TR, take);
    if (tiles == 0) continue;
    hipError_t e;
    if (p.dtype == MTE_BF16)
      e = dp == 64 ? run_cross<bf16, 64>(a, pl, s) : run_cross<bf16, 128>(a, pl, s);
    else
      e = dp == 64 ? run_cross<float, 64>(a, pl, s) : run_cross<float, 128>(a, pl, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Few rows stream the codes, in chunks of as many tokens as 32 rows hold, each read as a sequence of its own;
// many stage them, whole where the table is no wider than LDS. A call with both takes both kernels,
// the workspace serving one after the other. Which sequences are few goes by the tiles of 32 rows of
// the call, times kv heads (us few / many):
//   below kFewTiles, all: 508 queries of 2 x 2 heads of 128 over 59 to 682 tokens 16.8 / 29.1; against it,
//     50 of 8 heads of 64 over 257, 11.0 / 9.4; above it 250 of 2 x 8 heads over 320 19.5 / 14.7;
//   below kFill, those of two tiles: 16 x 30 of 2 x 8 heads over 200 9.4 / 10.2, 9 of 1 to 39 of 20
//     heads over 20 to 825 (one kernel instead of two) 15.0 / 24.9;
//   else those of one: 64 x 60 of 10 heads over 100 15.2 / 10.3.
constexpr int kLds = 160 * 1024;                     // of a compute unit
constexpr int kFewTiles = 96;
struct Few {
  int chunk;                                        // tokens of a chunk; 0: one token has more than 32 rows
  int64_t rows;                                     // the most rows of a few sequence
  explicit Few(const AttnProblem &p) : chunk(32 / p.c.rep) {
    int64_t tiles = 0;
    for (int i = 0; chunk > 0 && i < p.n; ++i) tiles += ceil_div(p.q_lens[i], chunk);
    tiles *= p.c.hkv;
    rows = tiles < kFewTiles ? INT64_MAX : tiles < kFill ? 64 : 32;
  }
  bool takes(const AttnProblem &p, int i) const { return chunk > 0 && (int64_t)p.q_lens[i] * p.c.rep <= rows; }
};
// Fills a.seq with the next chunks of few sequences (from query `done` of sequence i); returns how many.
static int next_chunks(Kv8AttnArgs &a, const AttnProblem &p, const Few &fw, int &i, int &row, int &done) {
  a.n_seq = 0;
  while (i < p.n && a.n_seq < kCondSeqs) {
    const int len = p.q_lens[i], left = len - done;
    if (left > 0 && fw.takes(p, i)) {
      const int n = std::min(fw.chunk, left);
      a.seq[a.n_seq] = CondSeq{row + done, n, i, left, a.n_seq};
      ++a.n_seq;
      done += n;
      if (done < len) continue;
    }
    row += len;
    done = 0;
    ++i;
  }
  return a.n_seq;
}
static Plan kv8_plan(const AttnProblem &p, int width, bool few) {
  Plan pl;
  int64_t row_tiles, most;
  const Few fw(p);
  const auto mine = [&](int i) { return fw.takes(p, i) == few; };
  count_rows(p, row_tiles, most, mine);
  if (row_tiles == 0) return pl;
  const int64_t res = (int64_t)width * 32 * p.c.d * 4;
  if (few) {
    pl.TR = 32;
  } else if (res <= kLds) {
    // LDS is shared by two and more workgroups of four waves where that leaves each half of it, else
    // eight waves have it to themselves; rows are turned in LDS where there is room (bf16: fp32 is
    // bound by its products, and has no registers to spare).
    const int room = p.dtype == MTE_BF16 && p.near_tiles ? kBox : 0, simd = p.dtype != MTE_BF16 ? 1 : p.c.d == 64 ? 3 : 2;
    pl.kind = Plan::RESIDENT;
    pl.nw = res + 4 * room <= kLds / 2 ? 4 : 8;
    pl.box = room > 0 && res + pl.nw * room <= kLds;
    pl.lds = (int)res + (pl.box ? pl.nw * room : 0);
    // Row tiles a wave takes one after the other: the keys are staged once for all of them. Whole
    // rounds of the workgroups that the chip holds, a staging at the cost of a tile (16 x 1024
    // queries over 320 tokens, us: 4 tiles in one round 61.5, 2 in two rounds 67).
    const int64_t slots = 256 * std::max(1, std::min(kLds / pl.lds, 4 * simd / pl.nw));
    int64_t best = INT64_MAX;
    int iters = 1;
    for (int i = 1; i <= 16; ++i) {
      pl.TR = 32 * pl.nw * i;
      const int64_t cost = (fill_tiles(p, pl, mine) * p.c.hkv + slots - 1) / slots * (i + 1);
      if (cost < best) { best = cost; iters = i; }
    }
    pl.TR = 32 * pl.nw * iters;
  } else {
    pl.kind = Plan::STREAM;
    pl.TR = 128;
  }
  const int64_t units = fill_tiles(p, pl, mine) * p.c.hkv;
  if (pl.kind == Plan::RESIDENT) return pl;
  pl.ws_rows = (int)std::min<int64_t>(pl.TR, most);
  if (few) {
    int64_t chunks = 0;
    for (int i = 0; i < p.n; ++i)
      if (mine(i)) chunks += ceil_div(p.q_lens[i], fw.chunk);
    pl.tiles = std::min<int64_t>(chunks, kCondSeqs);
    // parts for each kv head: of kFill workgroups, no more than the widest tables fill; the
    // partial results of all that the lengths may lead to
    const int fill = p.dtype == MTE_BF16 ? kFill : kFill / 2;   // fp32: one workgroup a compute unit
    pl.target = (int)std::max<int64_t>(1, std::min<int64_t>(fill / p.c.hkv, pl.tiles * ceil_div(width, kRowsLeast)));
    if (ceil_div(width, kRowsLeast) > 1) pl.tiles += pl.target;
    else pl.target = 0;                             // no sequence is cut
  } else if (units < kFill)
    pl.n_split = (int)std::max<int64_t>(1, std::min<int64_t>(kFill / units, ceil_div(width, 2 * kTilesLeast)));
  return pl;
}

int64_t kv8_workspace(const AttnProblem &p, int width) {
  return std::max(kv8_plan(p, width, true).floats(p.c.hkv, p.c.d), kv8_plan(p, width, false).floats(p.c.hkv, p.c.d)) * 4;
}

template <typename T, int D>
static hipError_t run_kv8(const Kv8AttnArgs &a, int tiles, const Plan &pl, hipStream_t s) {
  const dim3 grid(tiles * a.hkv, a.n_split);
  hipError_t e;
  if (pl.kind == Plan::RESIDENT) {
    constexpr bool B16 = sizeof(T) == 2;
    auto kern = pl.box ? (pl.nw == 4 ? k_kv8_res<T, D, 4, B16> : k_kv8_res<T, D, 8, B16>)
                       : (pl.nw == 4 ? k_kv8_res<T, D, 4, false> : k_kv8_res<T, D, 8, false>);
    if ((e = allow_lds(kern, pl.lds)) != hipSuccess) return e;
    hipLaunchKernelGGL(kern, grid, dim3(64 * pl.nw), pl.lds, s, a, pl.TR);
    return hipGetLastError();
  }
  if (pl.kind == Plan::FEW) {                       // a tile is a chunk
    const int target = std::max(pl.target, 1);
    const dim3 parts((tiles + (pl.target > 0 ? target : 0)) * a.hkv);
    hipLaunchKernelGGL((k_kv8_rows<T, D>), parts, dim3(kThreads), 3 * (2 + D / 2) * 64 * 4, s, a, target);
    if ((e = hipGetLastError()) != hipSuccess || pl.target == 0) return e;
    hipLaunchKernelGGL((k_kv8_rows_join<T, D>), dim3(tiles * a.hkv, a.ws_rows), dim3(kThreads), 0, s, a, target);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((k_kv8_tiles<T, D>), grid, dim3(kThreads), 2 * 4 * (D / 32) * 64 * 16, s, a);
  if ((e = hipGetLastError()) != hipSuccess || a.n_split == 1) return e;
  auto join = a.n_split > kFewParts ? k_kv8_tiles_join<T, D, true> : k_kv8_tiles_join<T, D, false>;
  hipLaunchKernelGGL(join, dim3(tiles * a.hkv, join_grid<D>(a.n_split, a.ws_rows)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_kv8_attention(const AttnProblem &p, const Kv8View &c, int causal, hipStream_t s) {
  const Few fw(p);
  for (const bool few : {true, false}) {
    const Plan pl = kv8_plan(p, c.width, few);
    if (pl.tiles == 0) continue;
    Kv8AttnArgs a;
    (AttnCommon &)a = p.c;
    a.big = big_out(p);
    a.c = c;
    a.causal = causal;
    a.n_split = pl.n_split;
    a.ws_rows = pl.ws_rows;
    a.ws_ml = pl.ml(a.hkv, c.d);
    auto take = [&](int i, CondSeq &sq) {
      sq.k0 = i;
      sq.k_len = p.q_lens[i];
      return fw.takes(p, i) == few;
    };
    for (int i = 0, row = 0, done = 0; i < p.n;) {
      const int tiles = few ? next_chunks(a, p, fw, i, row, done) : next_seqs(a, p, i, row, pl.TR, take);
      if (tiles == 0) continue;
      hipError_t e;
      if (p.dtype == MTE_BF16)
        e = c.d == 64 ? run_kv8<bf16, 64>(a, tiles, pl, s) : run_kv8<bf16, 128>(a, tiles, pl, s);
      else
        e = c.d == 64 ? run_kv8<float, 64>(a, tiles, pl, s) : run_kv8<float, 128>(a, tiles, pl, s);
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace mte
