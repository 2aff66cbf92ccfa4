// Attention of packed queries to conditioning tokens: keys and values as rows
// (k_cross), or as e4m3 codes in blocks of 32 tokens (k_kv8_rows, k_kv8_tiles).
//
//   o[i, h] = sum_j p_ij v[j, g],  p_ij = exp(s_ij - m_i) / sum_j exp(s_ij - m_i),
//   s_ij = scale q[i, h] . k[j, g],  g = h / rep
//
// Rows. The rep query heads of a kv head read the same keys, so the rows of a
// matrix tile are (token, head) pairs: row r of a sequence is token r / rep, head
// g rep + r % rep. One query with grouped heads fills rep rows, not one.
//
// Matrix core forms (32x32, as in attention.hip): S^T = K Q^T leaves each lane the
// scores of one row (lane % 32) for 16 of 32 keys, key 8 (r / 4) + 4 (lane / 32) +
// r % 4 in register r, so maxima and sums are per-lane loops and one exchange between
// the wave's halves, and the probabilities are already the B operand of
// O^T = V^T P^T, if V^T is read with its keys in that same order.
//
// One pass over the keys with the running maximum m and sum l of each row (fp32,
// log2 units); O is rescaled where m moved. Key ranges may be split: over waves of a
// workgroup (joined through LDS) and over workgroups (partial O, m, l in the
// workspace, joined by k_cond_join).
#include <algorithm>

#include "../../include/mte.h"
#include "common.h"
#include "cond_launch.h"

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

__device__ __forceinline__ int find_seq(const CondSeq *seq, int n, int tile) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (seq[mid].tile0 <= tile) lo = mid; else hi = mid - 1;
  }
  return lo;
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

// Running softmax of one row per lane (both halves of the wave hold the same row).
template <int ND> struct Rows {
  f32x16 o[ND];
  float m, l;      // m in log2 units; l over this lane's keys only
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[n][r] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ void scale(float f) {
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[n][r] *= f;
  }
  // takes the maximum mb of new scores (log2 units), returns what to subtract from them
  __device__ __forceinline__ float raise(float mb) {
    const float m_new = fmaxf(m, mb);
    const float ref = m_new == -INFINITY ? 0.f : m_new;   // nothing seen yet: exp2(-inf - 0) = 0
    const float alpha = __builtin_amdgcn_exp2f(m - ref);
    l *= alpha;
    if (__any(alpha != 1.f)) scale(alpha);
    m = m_new;
    return ref;
  }
};

// Keeps the scores of keys whose bit in `word` (bit = key of the 32) is set.
__device__ __forceinline__ void mask_scores(f32x16 &s, uint32_t word, int lane) {
  const uint32_t w = word >> (4 * (lane >> 5));
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = (w >> (8 * (r >> 2) + (r & 3))) & 1 ? s[r] : -INFINITY;
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
  const float mr = mx == -INFINITY ? 0.f : mx;
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
        bf16x4 lo, hi;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo[e] = (bf16)(st.o[n][8 * p + e] * inv);
          hi[e] = (bf16)(st.o[n][8 * p + 4 + e] * inv);
        }
        u32x2 x = __builtin_bit_cast(u32x2, lo), y = __builtin_bit_cast(u32x2, hi);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          // the upper 32 lanes' x and the lower 32 lanes' y trade places: 8 consecutive d a lane
          const auto r = __builtin_amdgcn_permlane32_swap(x[w], y[w], false, false);
          x[w] = r[0];
          y[w] = r[1];
        }
        const int c = 32 * n + 16 * p + 8 * h;
        if (live && c < a.d) *(u32x4 *)(row + c) = u32x4{x[0], x[1], y[0], y[1]};
      }
    }
  }
}

// Partial state of row r of unit (tile, g) and split: O unnormalised (times vscale), m, l.
template <int ND>
__device__ __forceinline__ void store_part(const AttnCommon &a, Rows<ND> &st, float vscale, bool live, int tile, int g,
                                           int split, int r, int lane) {
  const float l = st.l + __shfl_xor(st.l, 32, kWave);
  if (!live) return;
  const int64_t at = (((int64_t)tile * a.hkv + g) * a.n_split + split) * a.ws_rows + r;
  float *o = a.ws + at * (32 * ND) + 4 * (lane >> 5);
#pragma unroll
  for (int n = 0; n < ND; ++n)
#pragma unroll
    for (int b = 0; b < 4; ++b)
      *(f32x4 *)(o + 32 * n + 8 * b) = f32x4{st.o[n][4 * b] * vscale, st.o[n][4 * b + 1] * vscale,
                                            st.o[n][4 * b + 2] * vscale, st.o[n][4 * b + 3] * vscale};
  if (lane < 32) {
    float *ml = a.ws + a.ws_ml + at * 2;
    ml[0] = st.m;
    ml[1] = l;
  }
}

// ---- keys and values as rows --------------------------------------------------------------------
//
// A workgroup of four waves serves 32 RW rows of one sequence and kv head; the other
// 4 / RW ways of its waves split the keys of a tile (few rows: RW = 1). Key tiles go
// global -> registers -> LDS, the next tile's loads in flight while one is computed;
// rows past the end and masked value rows become zeros on the way.
// LDS: keys as 16-byte chunks in the order of the MFMA operand ([32 keys][chunk c]:
// lane = key), the key index xored with the chunk so that neither the row-wise
// writes nor the operand reads meet in a bank; values as rows, chunks xored so that the
// transposing reads (bf16: 4 keys x 16 d per 16 lanes) and the fp32 reads (one d column
// a lane) do not either.
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
  const int tile = blockIdx.x, g = blockIdx.y, split = blockIdx.z;
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, tile)];
  const int klen = sq.k_len, rows = sq.q_len * a.rep;
  const int r0 = (tile - sq.tile0) * 32 * RW + rw * 32;   // first row of the wave
  const Span span = split_span((klen + KT - 1) / KT, a.n_split, split, 1);
  if (split >= span.used) return;                   // the whole workgroup
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
      int vc;
      if constexpr (!B16) vc = c ^ (8 * ((row >> 2) & 1));
      else if constexpr (NCH == 16) vc = c ^ (4 * (row & 3));
      else vc = c ^ (4 * ((row >> 1) & 1));
      *(u32x4 *)(sv + (row * NCH + vc) * 16) = vx[t];
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
      const int sub = kw * NS + u;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[u][i] = 0.f;
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) {
        const int c = 2 * kk + h;
        mfma32(s[u], __builtin_bit_cast(frag_t, sk[(sub * NCH + c) * 32 + (lrow ^ (c & 7))]), qf[kk]);
      }
      const uint32_t word = __builtin_amdgcn_readfirstlane(sm[sub]);
      if (word != 0xFFFFFFFFu) mask_scores(s[u], word, lane);
#pragma unroll
      for (int i = 0; i < 16; ++i) mb = fmaxf(mb, s[u][i]);
    }
    mb = warp_max_xor(mb, 32) * a.sc;
    const float ref = st.raise(mb);
#pragma unroll
    for (int u = 0; u < NS; ++u) {
      const int sub = kw * NS + u;
      float p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(s[u][i], a.sc, -ref));
        st.l += p[i];
      }
      if constexpr (B16) {
        // P in bf16, the values' type (their range is bf16's): each term off by at most 2^-8 of itself
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          bf16x8 pf;
#pragma unroll
          for (int e = 0; e < 8; ++e) pf[e] = (bf16)p[8 * f + e];
          const int i = lane & 15;
          const int row = sub * 32 + 16 * f + 4 * h + (i >> 2);
#pragma unroll
          for (int n = 0; n < ND; ++n) {
            const int c = 4 * n + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
            const int vc = NCH == 16 ? c ^ (4 * (row & 3)) : c ^ (4 * ((row >> 1) & 1));
            const char *va = sv + (row * NCH + vc) * 16 + (lane & 1) * 8;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)va);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(va + 8 * NCH * 16));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            const s16x8 w = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            mfma32(st.o[n], __builtin_bit_cast(bf16x8, w), pf);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int row = sub * 32 + 8 * (i >> 2) + 4 * h + (i & 3);
          const float *vr = (const float *)sv + row * DP;
#pragma unroll
          for (int n = 0; n < ND; ++n)
            st.o[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(vr[32 * (n ^ h) + lrow], p[i], st.o[n], 0, 0, 0);
        }
      }
    }
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
  else store_part<ND>(a, st, 1.f, live, tile, g, split, rw * 32 + lrow, lane);
}

// ---- keys and values as e4m3 codes --------------------------------------------------------------
//
// Codes widen exactly: keys to bf16 (the queries' type: their range is bf16's), values to
// fp16, and the probabilities, at most 2^8 here (an offset in the exponent that
// keeps small ones out of fp16's subnormals), to fp16. fp32 queries are three bf16
// terms (24 bits) and fp32 probabilities two fp16 terms (22 bits), so that the products
// keep fp32's precision on the 16-bit matrix cores.
// Block scales: the key scale multiplies the scores; the value scale, relative to the
// largest one so far (`vref`, a power of two, wave-uniform), multiplies the
// probabilities, and O is in units of vref.
constexpr float kPOff = 8.f;

template <typename T, int NK> struct QCodes {      // query operands: NQ bf16 terms
  static constexpr int NQ = sizeof(T) == 4 ? 3 : 1;
  bf16x8 f[NQ][NK];
  // MFMA 2 j + u takes d = 32 j + 16 h + 8 u .. + 7 (the order of the key codes)
  __device__ __forceinline__ void load(const T *row, bool live, int h) {
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      const int c = 32 * (kk >> 1) + 16 * h + 8 * (kk & 1);
      if constexpr (sizeof(T) == 2) {
        u32x4 x{0, 0, 0, 0};
        if (live) x = *(const u32x4 *)(row + c);
        f[0][kk] = __builtin_bit_cast(bf16x8, x);
      } else {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
        if (live) {
          const f32x4 x0 = *(const f32x4 *)(row + c), x1 = *(const f32x4 *)(row + c + 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) { x[e] = x0[e]; x[4 + e] = x1[e]; }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bf16 a = (bf16)x[e];
          const float ra = x[e] - (float)a;
          const bf16 b = (bf16)ra;
          f[0][kk][e] = a;
          f[1][kk][e] = b;
          f[2][kk][e] = (bf16)(ra - (float)b);
        }
      }
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

// Softmax of one block's scores s (raw, masked) with key factor ksc, and O += V^T P^T.
// vf(n, f): value operand of d block n, keys 16 f ..
template <typename T, int ND, typename VF>
__device__ __forceinline__ void kv8_update(Rows<ND> &st, float &vref, float &vinv, const f32x16 &s, float ksc,
                                           float vsc, VF vf) {
  float mb = -INFINITY;
#pragma unroll
  for (int i = 0; i < 16; ++i) mb = fmaxf(mb, s[i]);
  mb = warp_max_xor(mb, 32) * ksc;
  const float ref = st.raise(mb) - kPOff;
  if (vsc > vref) {                                 // wave-uniform
    st.scale(vref / vsc);                           // 0 at the first block, where O is 0
    vref = vsc;
    vinv = 1.f / vsc;
  }
  const float ratio = vsc * vinv;
  float p[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], ksc, -ref));
    st.l += p[i];
    p[i] *= ratio;
  }
#pragma unroll
  for (int f = 0; f < 2; ++f) {
    f16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi[e] = (f16)p[8 * f + e];
      if constexpr (sizeof(T) == 4) lo[e] = (f16)(p[8 * f + e] - (float)hi[e]);
    }
#pragma unroll
    for (int n = 0; n < ND; ++n) {
      const f16x8 v = vf(n, f);
      mfma32(st.o[n], v, hi);
      if constexpr (sizeof(T) == 4) mfma32(st.o[n], v, lo);
    }
  }
}

// What the rows of a tile see of a sequence.
struct Seen { int kv, tile_hi, row_hi; };           // length; keys of the tile's last row, of this lane's row
__device__ __forceinline__ Seen seen_of(const Kv8AttnArgs &a, const CondSeq &sq, int last_tok, int tok) {
  Seen v;
  v.kv = min(max(a.c.kv_lens[sq.k0], 0), a.c.width * 32);
  v.tile_hi = a.causal ? min(max(v.kv - sq.q_len + last_tok + 1, 0), v.kv) : v.kv;
  v.row_hi = a.causal ? min(max(v.kv - sq.q_len + tok + 1, 0), v.kv) : v.kv;
  return v;
}

// Bits of the block's keys below `hi` (key 0 of the block at `at`).
__device__ __forceinline__ uint32_t bits_below(int hi, int at) {
  const int n = hi - at;
  return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u;
}

// Least blocks of a split: below that a partial result costs more than its keys.
constexpr int kRowsLeast = 8, kTilesLeast = 4;

// Few rows (at most 32 a tile): bound by the codes that stream in. Each of the four waves
// takes every fourth block of the split's range and loads its codes straight into MFMA operand
// order, 16 bytes a lane and 1 KB a load, the next block's while one is computed.
template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 1 : 2) void k_kv8_rows(Kv8AttnArgs a) {
  constexpr int ND = D / 32, NK = D / 16, NL = D / 32;
  extern __shared__ u32x4 lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lrow = lane & 31, h = lane >> 5;
  const int tile = blockIdx.x, g = blockIdx.y, split = blockIdx.z;
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, tile)];
  const int rows = sq.q_len * a.rep, r0 = (tile - sq.tile0) * 32, r = r0 + lrow;
  const bool live = r < rows;
  const int qi = live ? r / a.rep : 0;
  const int head = g * a.rep + (live ? r % a.rep : 0);
  const Seen seen = seen_of(a, sq, (min(r0 + 32, rows) - 1) / a.rep, qi);
  const Span span = split_span((seen.tile_hi + 31) >> 5, a.n_split, split, kRowsLeast);
  if (split >= span.used) return;

  const int32_t *tab = a.c.table + (int64_t)sq.k0 * a.c.table_row;
  struct Block { u32x4 k[NL], v[NL]; float ks, vs; };
  auto load = [&](int b, Block &x) {
    const int id = __builtin_amdgcn_readfirstlane(tab[b]);
    const bool ok = id >= 0 && id < a.c.n_blocks;
    const int64_t at = (int64_t)(ok ? id : 0) * a.c.hkv + g;
    const u32x4 *kp = (const u32x4 *)(a.c.k_codes + at * (32 * D)) + lane;
    const u32x4 *vp = (const u32x4 *)(a.c.v_codes + at * (32 * D)) + lrow * 2 + h;
#pragma unroll
    for (int i = 0; i < NL; ++i) x.k[i] = kp[64 * i];
#pragma unroll
    for (int i = 0; i < NL; ++i) x.v[i] = vp[64 * i];
    x.ks = a.c.scales[at * 2];
    x.vs = ok ? a.c.scales[at * 2 + 1] : -1.f;      // a block that is none
  };
  QCodes<T, NK> q;
  Rows<ND> st;
  st.init();
  float vref = 0.f, vinv = 0.f;
  Block cur, nxt;
  const int b0 = span.lo + wave;
  if (b0 < span.hi) load(b0, cur);
  q.load((const T *)a.q + (int64_t)(sq.q0 + qi) * a.q_row + (int64_t)head * a.q_head, live, h);
  for (int b = b0; b < span.hi; b += 4) {
    if (b + 4 < span.hi) load(b + 4, nxt);
    if (cur.vs > 0.f) {
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) {
        const bf16x8 kf = widen_bf16(cur.k[kk >> 1][2 * (kk & 1)], cur.k[kk >> 1][2 * (kk & 1) + 1]);
#pragma unroll
        for (int t = q.NQ - 1; t >= 0; --t) mfma32(s, kf, q.f[t][kk]);   // small terms first
      }
      const int at = b * 32;
      if (at + 32 > seen.kv || a.causal) {          // wave-uniform
        mask_scores(s, bits_below(seen.row_hi, at), lane);
        const int left = seen.kv - at;
        if (left < 32) {
#pragma unroll
          for (int i = 0; i < NL; ++i) cur.v[i] = keep_tokens(cur.v[i], left, h);
        }
      }
      kv8_update<T, ND>(st, vref, vinv, s, cur.ks * a.sc, cur.vs,
                        [&](int n, int f) { return widen_f16(cur.v[n][2 * f], cur.v[n][2 * f + 1]); });
    }
    cur = nxt;
  }
  // the waves' O in one unit before they are joined
  float *red = (float *)lds;
  if (lane == 0) red[wave] = vref;
  __syncthreads();
  const float top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  if (top > 0.f) st.scale(vref / top);
  __syncthreads();
  join_waves<ND, 4>(st, red, wave, lane);
  if (wave > 0) return;
  if (span.used == 1)
    store_rows<T, ND>(a, st, top, live, sq.q0 + qi, head, lane);
  else
    store_part<ND>(a, st, top, live, tile, g, split, lrow, lane);
}

// Many rows: four waves of 32 rows; two blocks of codes a step are widened once per
// workgroup on their way into LDS, in MFMA operand order (1 KB of lanes a fragment,
// free of bank conflicts), the next step's codes in flight in registers.
template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 1 : 2) void k_kv8_tiles(Kv8AttnArgs a) {
  constexpr int ND = D / 32, NK = D / 16, NL = D / 32;
  constexpr int PIECES = 4 * NL;                    // 1 KB loads of a step: 2 blocks x (k, v) x NL
  constexpr int PPW = PIECES / 4;
  extern __shared__ u32x4 lds[];                    // [block][NK key + 2 ND value fragments][64 lanes]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lrow = lane & 31, h = lane >> 5;
  const int tile = blockIdx.x, g = blockIdx.y, split = blockIdx.z;
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, tile)];
  const int rows = sq.q_len * a.rep, t0 = (tile - sq.tile0) * 128, r0 = t0 + wave * 32, r = r0 + lrow;
  const bool live = r < rows;
  const int qi = live ? r / a.rep : 0;
  const int head = g * a.rep + (live ? r % a.rep : 0);
  const Seen seen = seen_of(a, sq, (min(t0 + 128, rows) - 1) / a.rep, qi);
  const Span span = split_span((seen.tile_hi + 31) >> 5, a.n_split, split, kTilesLeast);
  if (split >= span.used) return;
  const int wave_hi = !a.causal ? seen.kv
                                : min(max(seen.kv - sq.q_len + (min(r0 + 32, rows) - 1) / a.rep + 1, 0), seen.kv);
  const int wave_lo = !a.causal ? seen.kv : min(max(seen.kv - sq.q_len + min(r0, rows - 1) / a.rep + 1, 0), seen.kv);

  const int32_t *tab = a.c.table + (int64_t)sq.k0 * a.c.table_row;
  auto block_at = [&](int b, bool &ok) {
    const int id = b < span.hi ? __builtin_amdgcn_readfirstlane(tab[b]) : -1;
    ok = id >= 0 && id < a.c.n_blocks;
    return (int64_t)(ok ? id : 0) * a.c.hkv + g;
  };
  u32x4 x[PPW];
  auto gload = [&](int b) {
#pragma unroll
    for (int i = 0; i < PPW; ++i) {
      const int p = wave * PPW + i, blk = p / (2 * NL), sub = p % (2 * NL);
      bool ok;
      const int64_t at = block_at(b + blk, ok);
      x[i] = u32x4{0, 0, 0, 0};
      if (ok) {
        if (sub < NL) {
          x[i] = ((const u32x4 *)(a.c.k_codes + at * (32 * D)))[64 * sub + lane];
        } else {
          x[i] = ((const u32x4 *)(a.c.v_codes + at * (32 * D)))[64 * (sub - NL) + lrow * 2 + h];
          const int left = seen.kv - (b + blk) * 32;
          if (left < 32) x[i] = keep_tokens(x[i], left, h);
        }
      }
    }
  };
  auto lstore = [&]() {
#pragma unroll
    for (int i = 0; i < PPW; ++i) {
      const int p = wave * PPW + i, blk = p / (2 * NL), sub = p % (2 * NL);
      u32x4 *to = lds + (blk * 4 * NL + 2 * sub) * 64 + lane;
      if (sub < NL) {
        to[0] = __builtin_bit_cast(u32x4, widen_bf16(x[i][0], x[i][1]));
        to[64] = __builtin_bit_cast(u32x4, widen_bf16(x[i][2], x[i][3]));
      } else {
        to[0] = __builtin_bit_cast(u32x4, widen_f16(x[i][0], x[i][1]));
        to[64] = __builtin_bit_cast(u32x4, widen_f16(x[i][2], x[i][3]));
      }
    }
  };
  if (span.lo < span.hi) gload(span.lo);
  QCodes<T, NK> q;
  q.load((const T *)a.q + (int64_t)(sq.q0 + qi) * a.q_row + (int64_t)head * a.q_head, live, h);
  Rows<ND> st;
  st.init();
  float vref = 0.f, vinv = 0.f;
  for (int b = span.lo; b < span.hi; b += 2) {
    __syncthreads();
    lstore();
    __syncthreads();
    if (b + 2 < span.hi) gload(b + 2);
    if (r0 >= rows) continue;                       // wave-uniform: it still loads and meets the barriers
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int at = (b + u) * 32;
      bool ok;
      const int64_t blk = block_at(b + u, ok);
      if (!ok || at >= wave_hi) continue;
      const u32x4 *fr = lds + u * 4 * NL * 64 + lane;
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) {
        const bf16x8 kf = __builtin_bit_cast(bf16x8, fr[kk * 64]);
#pragma unroll
        for (int t = q.NQ - 1; t >= 0; --t) mfma32(s, kf, q.f[t][kk]);
      }
      if (at + 32 > wave_lo) mask_scores(s, bits_below(seen.row_hi, at), lane);
      kv8_update<T, ND>(st, vref, vinv, s, a.c.scales[blk * 2] * a.sc, a.c.scales[blk * 2 + 1], [&](int n, int f) {
        return __builtin_bit_cast(f16x8, fr[(NK + 2 * n + f) * 64]);
      });
    }
  }
  if (r0 >= rows) return;
  if (span.used == 1)
    store_rows<T, ND>(a, st, vref, live, sq.q0 + qi, head, lane);
  else
    store_part<ND>(a, st, vref, live, tile, g, split, wave * 32 + lrow, lane);
}

// ---- joining splits -----------------------------------------------------------------------------
//
// out[row] = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s, M = max m_s over the splits that a
// unit (tile, kv head) used; units of one split wrote their rows themselves. A row is DP / 4
// lanes of four d.
template <typename T, int DP, typename A, typename SPAN>
__device__ __forceinline__ void join_body(const A &a, int TR, SPAN used_of) {
  constexpr int LPR = DP / 4;
  const int tile = blockIdx.x, g = blockIdx.y;
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, tile)];
  const int rows = sq.q_len * a.rep, r0 = (tile - sq.tile0) * TR;
  const int used = used_of(sq, (min(r0 + TR, rows) - 1) / a.rep);
  if (used == 1) return;
  const int c = (threadIdx.x % LPR) * 4;
  for (int i = threadIdx.x / LPR; i < min(TR, rows - r0); i += kThreads / LPR) {
    const int64_t at = (((int64_t)tile * a.hkv + g) * a.n_split) * a.ws_rows + i;
    const float *ml = a.ws + a.ws_ml + at * 2, *o = a.ws + at * DP + c;
    float M = -INFINITY;
    for (int s = 0; s < used; ++s) M = fmaxf(M, ml[(int64_t)s * a.ws_rows * 2]);
    const float mr = M == -INFINITY ? 0.f : M;
    float l = 0.f;
    f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < used; ++s) {
      const float f = __builtin_amdgcn_exp2f(ml[(int64_t)s * a.ws_rows * 2] - mr);
      l += f * ml[(int64_t)s * a.ws_rows * 2 + 1];
      const f32x4 x = *(const f32x4 *)(o + (int64_t)s * a.ws_rows * DP);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += f * x[e];
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const int r = r0 + i;
    T *row = (T *)a.out + (int64_t)(sq.q0 + r / a.rep) * a.o_row + (int64_t)(g * a.rep + r % a.rep) * a.o_head;
    if (c < a.d) {
      if constexpr (sizeof(T) == 4)
        *(f32x4 *)(row + c) = f32x4{acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
      else
        *(bf16x4 *)(row + c) = bf16x4{(bf16)(acc[0] * inv), (bf16)(acc[1] * inv), (bf16)(acc[2] * inv), (bf16)(acc[3] * inv)};
    }
  }
}

template <typename T, int DP>
__global__ __launch_bounds__(kThreads) void k_cross_join(CrossArgs a, int TR, int KT) {
  join_body<T, DP>(a, TR, [&](const CondSeq &sq, int) {
    return split_span((sq.k_len + KT - 1) / KT, a.n_split, 0, 1).used;
  });
}

template <typename T, int DP>
__global__ __launch_bounds__(kThreads) void k_kv8_join(Kv8AttnArgs a, int TR, int least) {
  join_body<T, DP>(a, TR, [&](const CondSeq &sq, int last_tok) {
    return split_span((seen_of(a, sq, last_tok, 0).tile_hi + 31) >> 5, a.n_split, 0, least).used;
  });
}

// ---- plans --------------------------------------------------------------------------------------

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// How a class of query sequences is launched: TR rows a tile, the same number of splits for all.
struct Plan {
  int TR = 0, n_split = 1, ws_rows = 0;
  int64_t tiles = 0;                                // of the launch (of kCondSeqs sequences) with the most
  int64_t floats(int hkv, int dp) const {
    return n_split > 1 ? tiles * hkv * n_split * (int64_t)ws_rows * (dp + 2) : 0;
  }
  int64_t ml(int hkv, int dp) const { return tiles * hkv * n_split * (int64_t)ws_rows * dp; }
};

int pad_d(int d) { return d <= 64 ? 64 : 128; }

// Workgroups that fill the 256 compute units with two each; a launch below it splits long key ranges.
constexpr int kFill = 512;

}  // namespace

// Rows mode by the longest query sequence: up to 32 rows the four waves of a workgroup share
// them and split the keys.
static Plan cross_plan(const AttnProblem &p, const int32_t *kv_lens, const int32_t *kv_index, int &rw, int &KT) {
  Plan pl;
  int64_t most = 0;
  int kmax = 0;
  for (int i = 0; i < p.n; ++i) {
    most = std::max<int64_t>(most, (int64_t)p.q_lens[i] * p.c.rep);
    if (p.q_lens[i] > 0) kmax = std::max(kmax, kv_lens[kv_index ? kv_index[i] : i]);
  }
  rw = most <= 32 ? 1 : 4;
  KT = rw == 1 ? 128 : p.dtype == MTE_BF16 ? 64 : 32;
  pl.TR = 32 * rw;
  pl.ws_rows = (int)std::min<int64_t>(pl.TR, most);
  int64_t all = 0;
  for (int i = 0, in = 0, at = 0; i < p.n; ++i) {
    if (p.q_lens[i] == 0) continue;
    const int t = ceil_div((int64_t)p.q_lens[i] * p.c.rep, pl.TR);
    all += t;
    at += t;
    pl.tiles = std::max<int64_t>(pl.tiles, at);
    if (++in == kCondSeqs) in = at = 0;
  }
  if (all == 0) return pl;
  // a split of at least 4 key tiles
  const int64_t units = all * p.c.hkv;
  if (units < kFill) pl.n_split = (int)std::max<int64_t>(1, std::min<int64_t>(kFill / units, ceil_div(kmax, KT) / 4));
  return pl;
}

int64_t cross_workspace(const AttnProblem &p, const int32_t *kv_lens, int, const int32_t *kv_index) {
  int rw, KT;
  const Plan pl = cross_plan(p, kv_lens, kv_index, rw, KT);
  return pl.floats(p.c.hkv, pad_d(p.c.d)) * 4;
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

template <typename T, int DP, int RW>
static hipError_t run_cross(const CrossArgs &a, int tiles, int TR, int KT, hipStream_t s) {
  const int lds = std::max(2 * KT * DP * (int)sizeof(T) + 32, RW == 4 ? 0 : 3 * (2 + DP / 2) * 64 * 4);
  auto kern = k_cross<T, DP, RW>;
  hipError_t e = allow_lds(kern, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(tiles, a.hkv, a.n_split), dim3(kThreads), lds, s, a);
  if ((e = hipGetLastError()) != hipSuccess || a.n_split == 1) return e;
  hipLaunchKernelGGL((k_cross_join<T, DP>), dim3(tiles, a.hkv), dim3(kThreads), 0, s, a, TR, KT);
  return hipGetLastError();
}

hipError_t launch_cross(const AttnProblem &p, const void *k, const void *v, const uint8_t *mask, int64_t k_row,
                        int64_t k_head, int64_t v_row, int64_t v_head, const int32_t *kv_lens, int n_kv,
                        const int32_t *kv_index, hipStream_t s) {
  int rw, KT;
  const Plan pl = cross_plan(p, kv_lens, kv_index, rw, KT);
  const int dp = pad_d(p.c.d);
  CrossArgs a;
  (AttnCommon &)a = p.c;
  a.k = k;
  a.v = v;
  a.mask = mask;
  a.k_row = k_row;
  a.k_head = k_head;
  a.v_row = v_row;
  a.v_head = v_head;
  a.n_split = pl.n_split;
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
    if (p.dtype == MTE_BF16) {
      if (dp == 64) e = rw == 1 ? run_cross<bf16, 64, 1>(a, tiles, pl.TR, KT, s) : run_cross<bf16, 64, 4>(a, tiles, pl.TR, KT, s);
      else e = rw == 1 ? run_cross<bf16, 128, 1>(a, tiles, pl.TR, KT, s) : run_cross<bf16, 128, 4>(a, tiles, pl.TR, KT, s);
    } else {
      if (dp == 64) e = rw == 1 ? run_cross<float, 64, 1>(a, tiles, pl.TR, KT, s) : run_cross<float, 64, 4>(a, tiles, pl.TR, KT, s);
      else e = rw == 1 ? run_cross<float, 128, 1>(a, tiles, pl.TR, KT, s) : run_cross<float, 128, 4>(a, tiles, pl.TR, KT, s);
    }
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Query sequences of up to 32 rows stream the codes (few), longer ones stage them (many); a call
// with both takes both kernels. The workspace serves one after the other.
static Plan kv8_plan(const AttnProblem &p, int width, bool few) {
  Plan pl;
  pl.TR = few ? 32 : 128;
  int64_t all = 0, most = 0;
  for (int i = 0, in = 0, at = 0; i < p.n; ++i) {
    const int64_t rows = (int64_t)p.q_lens[i] * p.c.rep;
    if (rows == 0 || (rows <= 32) != few) continue;
    const int t = ceil_div(rows, pl.TR);
    most = std::max(most, rows);
    all += t;
    at += t;
    pl.tiles = std::max<int64_t>(pl.tiles, at);
    if (++in == kCondSeqs) in = at = 0;
  }
  if (all == 0) return pl;
  pl.ws_rows = (int)std::min<int64_t>(pl.TR, most);
  const int64_t units = all * p.c.hkv;
  if (few)
    pl.n_split = (int)std::max<int64_t>(1, std::min<int64_t>(4096 / units, ceil_div(width, 2 * kRowsLeast)));
  else if (units < kFill)
    pl.n_split = (int)std::max<int64_t>(1, std::min<int64_t>(kFill / units, ceil_div(width, 2 * kTilesLeast)));
  return pl;
}

int64_t kv8_workspace(const AttnProblem &p, int width) {
  return std::max(kv8_plan(p, width, true).floats(p.c.hkv, p.c.d), kv8_plan(p, width, false).floats(p.c.hkv, p.c.d)) * 4;
}

template <typename T, int D>
static hipError_t run_kv8(const Kv8AttnArgs &a, int tiles, bool few, hipStream_t s) {
  const dim3 grid(tiles, a.hkv, a.n_split);
  hipError_t e;
  if (few) {
    const int lds = 3 * (2 + D / 2) * 64 * 4;
    hipLaunchKernelGGL((k_kv8_rows<T, D>), grid, dim3(kThreads), lds, s, a);
  } else {
    const int lds = 2 * 4 * (D / 32) * 64 * 16;
    hipLaunchKernelGGL((k_kv8_tiles<T, D>), grid, dim3(kThreads), lds, s, a);
  }
  if ((e = hipGetLastError()) != hipSuccess || a.n_split == 1) return e;
  hipLaunchKernelGGL((k_kv8_join<T, D>), dim3(tiles, a.hkv), dim3(kThreads), 0, s, a, few ? 32 : 128,
                     few ? kRowsLeast : kTilesLeast);
  return hipGetLastError();
}

hipError_t launch_kv8_attention(const AttnProblem &p, const Kv8View &c, int causal, hipStream_t s) {
  for (const bool few : {true, false}) {
    const Plan pl = kv8_plan(p, c.width, few);
    if (pl.tiles == 0) continue;
    Kv8AttnArgs a;
    (AttnCommon &)a = p.c;
    a.c = c;
    a.causal = causal;
    a.n_split = pl.n_split;
    a.ws_rows = pl.ws_rows;
    a.ws_ml = pl.ml(a.hkv, c.d);
    auto take = [&](int i, CondSeq &sq) {
      sq.k0 = i;
      sq.k_len = 0;
      return ((int64_t)p.q_lens[i] * a.rep <= 32) == few;
    };
    for (int i = 0, row = 0; i < p.n;) {
      const int tiles = next_seqs(a, p, i, row, pl.TR, take);
      if (tiles == 0) continue;
      hipError_t e;
      if (p.dtype == MTE_BF16)
        e = c.d == 64 ? run_kv8<bf16, 64>(a, tiles, few, s) : run_kv8<bf16, 128>(a, tiles, few, s);
      else
        e = c.d == 64 ? run_kv8<float, 64>(a, tiles, few, s) : run_kv8<float, 128>(a, tiles, few, s);
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace mte
