// Attention of packed queries to keys that all sequences share and then to their own:
//
//   o[i, h] = sum_j p_ij v[j, g],  p_ij = exp(s_ij - m_i) / sum_j exp(s_ij - m_i),  s_ij = scale q[i, h] . k[j, g],
//
// j over the prefix and the own tokens that query i sees. Row tiles, products and the running softmax are
// those of cross attention (cond_rows.h, cond_attention.hip); the keys are a list of tiles of two
// sources, first those of the prefix, then the sequence's own.
//
// Two ways through the list:
//  one pass: a row tile of one sequence takes the whole list, or a part of it.
//  shared: the rows of all sequences are one more, first sequence, whose list is the prefix alone, so that few
//    rows a sequence still fill tiles and the prefix is read once for a tile of rows and not once
//    a sequence; the sequences' lists are their own tokens. All results are partial (O / l, m, l), and a
//    second launch joins each row's parts of both.
// Which: prefix_plan.
#include <algorithm>
#include <climits>
#include <cmath>

#include "../../include/mte.h"
#include "cond_rows.h"
#include "proj_launch.h"

namespace mte {

namespace {

// Sequences as CondSeq: k0 < 0: the rows of all, over the prefix alone.
struct PrefixArgs : AttnCommon {
  const void *k, *v, *pk, *pv;
  int64_t k_row, k_head, v_row, v_head, pk_row, pk_head, pv_row, pv_head;
  int p_len, causal, shared;
  int unit0;                         // first unit of the launch among the partial results
  KeyCut p_cut, cut;                 // of the prefix alone (shared), of the other lists
  CondSeq seq[kCondSeqs];
};
static_assert(sizeof(PrefixArgs) <= 4096, "kernel arguments");

// The rows of a tile and the list of its keys, in tiles of KT.
struct Keys {
  int np, klen;                      // tiles of the prefix, own keys
  bool cross;                        // rows see different own keys
  int qlen;
  // own keys that query u sees
  __device__ __forceinline__ int seen(int u) const { return cross ? min(max(klen - qlen + u + 1, 0), klen) : klen; }
};
__device__ __forceinline__ Keys keys_of(const PrefixArgs &a, const CondSeq &sq, int KT) {
  const bool alone = sq.k0 < 0;
  Keys k;
  k.np = alone || !a.shared ? (a.p_len + KT - 1) / KT : 0;
  k.klen = alone ? 0 : sq.k_len;
  k.cross = a.causal && !alone;
  k.qlen = sq.q_len;
  return k;
}
__device__ __forceinline__ Part part_in(const PrefixArgs &a, const CondSeq &sq, const Keys &k, int local, int rows, int TR,
                                        int KT) {
  Part p = part_of(sq, local, rows, TR, k.np + (k.klen + KT - 1) / KT, sq.k0 < 0 ? a.p_cut : a.cut);
  if (k.cross) {                                     // nothing past the last row's last key
    const int last = (min((p.row_tile + 1) * TR, rows) - 1) / a.rep;
    p.hi = min(p.hi, k.np + (k.seen(last) + KT - 1) / KT);
  }
  return p;
}

// Infinities and NaN among the values of a tile whose rows see different keys: 0 times infinity in the matrix
// product would reach the rows that do not see them. Such values become zeros on their way to LDS, and rows that
// see them have them added after the last tile and the waves' join (add_wild). An infinity stays one where fp32 holds
// its weight; in a tile that all rows see, or a part of the list, whose weight beside the others' underflows, it is
// zero times infinity. In the loop itself a second path to O would cost a second copy of it, and its registers.
template <typename T> __device__ __forceinline__ bool tame(u32x4 &x) {
  bool wild = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (sizeof(T) == 4) {
      const bool b = (x[w] & 0x7F800000u) == 0x7F800000u;
      x[w] = b ? 0u : x[w];
      wild |= b;
    } else {
      const bool hi = (x[w] & 0x7F800000u) == 0x7F800000u, lo = (x[w] & 0x7F80u) == 0x7F80u;
      x[w] &= (hi ? 0u : 0xFFFF0000u) | (lo ? 0u : 0xFFFFu);
      wild |= hi || lo;
    }
  }
  return wild;
}
// Adds the infinities and NaN among the values of own keys [from, to) to O of the rows that see them; n: keys that
// this lane's row sees.
template <typename T, int ND>
__device__ __forceinline__ void add_wild(f32x16 (&o)[ND], const T *vg, int64_t v_row, int d_all, int from, int to, int n,
                                         int lane) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  const int h = lane >> 5;
#pragma unroll 1
  for (int j = from; j < to; ++j) {
    const T *row = vg + (int64_t)j * v_row;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int c = 32 * d + 8 * b + 4 * h;
        if (c < d_all) {
          const t4 x = *(const t4 *)(row + c);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = to_f32((T)x[e]);
            o[d][4 * b + e] += j < n && (__float_as_uint(v) & 0x7F800000u) == 0x7F800000u ? v : 0.f;
          }
        }
      }
  }
}

// store_part through LDS (`box`, kBox of the wave's own), so that whole lines are written: a lane holds 16 bytes of a row at
// a time, and as partial lines the parts of a step (18 MB, 64 streams over 16384 tokens) took 9 of its 41 us.
// left: rows that exist; row: of the unit, this wave's first.
template <int ND>
__device__ __forceinline__ void store_part_rows(const AttnCommon &a, Rows<ND> &st, int left, int unit, int g, int row,
                                                u32x4 *box, int lane) {
  const float l = st.l + __shfl_xor(st.l, 32, kWave);
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const int r = lane & 31, h = lane >> 5;
  const int64_t at = ((int64_t)unit * a.hkv + g) * a.ws_rows + row;
  if (lane < 32 && r < left) *(float2 *)(a.ws + a.ws_ml + (at + r) * 2) = float2{st.m, l};
  float *to = a.ws + at * (32 * ND);
#pragma unroll
  for (int n = 0; n < ND; ++n) {
#pragma unroll
    for (int b = 0; b < 4; ++b)
      box[box_at(r, 2 * b + h)] =
          __builtin_bit_cast(u32x4, f32x4{st.o[n][4 * b] * inv, st.o[n][4 * b + 1] * inv, st.o[n][4 * b + 2] * inv,
                                          st.o[n][4 * b + 3] * inv});
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int rr = 8 * i + (lane >> 3), c = lane & 7;
      const u32x4 x = box[box_at(rr, c)];
      if (rr < left) *(u32x4 *)(to + rr * (32 * ND) + 32 * n + 4 * c) = x;
    }
  }
}

// As k_cross: four waves, 32 RW rows, 4 / RW ways over the keys of a tile. Serves fp32, rows too far apart for the
// copies of k_prefix_stream, and calls of few rows in one pass. Bound by latency: 110 fp32 queries of 4 heads of 64 over
// 1201 + 7 to 200 tokens 9 us, the join 4.
template <typename T, int DP, int RW>
__global__ __launch_bounds__(kThreads, 2) void k_prefix(PrefixArgs a) {
  constexpr bool B16 = sizeof(T) == 2;
  constexpr int KW = 4 / RW, KT = 32 * KW;          // keys per tile: 32 a wave
  constexpr int E = 16 / sizeof(T), NCH = DP / E, NK = NCH / 2, ND = DP / 32;
  constexpr int CPT = KT * NCH / kThreads;          // chunks of K (and of V) per thread
  constexpr bool AHEAD = CPT <= 8;                  // next tile in registers meanwhile
  constexpr int STEP = AHEAD ? CPT : 4;
  typedef typename QFrag<T>::type frag_t;
  extern __shared__ u32x4 lds[];
  u32x4 *sk = lds;
  char *sv = (char *)(lds + KT * NCH);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lrow = lane & 31, h = lane >> 5;
  const int rw = wave % RW, kw = wave / RW;
  const Unit un = unit_of(a);
  const int tile = un.tile, g = un.g;
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, tile)];
  const Keys ks = keys_of(a, sq, KT);
  const int rows = sq.q_len * a.rep;
  const Part span = part_in(a, sq, ks, tile - sq.tile0, rows, 32 * RW, KT);
  const int r0 = span.row_tile * 32 * RW + rw * 32; // first row of the wave
  const int r = r0 + lrow;
  const bool live = r < rows;
  const int64_t tok = sq.q0 + (live ? r / a.rep : 0);
  const int head = g * a.rep + (live ? r % a.rep : 0);
  const int mine = ks.seen(live ? r / a.rep : sq.q_len - 1), least = ks.seen(r0 / a.rep);
  const int all_see = ks.cross ? ks.seen(span.row_tile * 32 * RW / a.rep) : INT_MAX;   // every row of the tile does
  uint32_t *wild = (uint32_t *)(sv + KT * NCH * 16);   // a word a wave: it found some

  const T *pk = (const T *)a.pk + (int64_t)g * a.pk_head, *pv = (const T *)a.pv + (int64_t)g * a.pv_head;
  const int64_t k0 = max(sq.k0, 0);
  const T *kg = (const T *)a.k + k0 * a.k_row + (int64_t)g * a.k_head;
  const T *vg = (const T *)a.v + k0 * a.v_row + (int64_t)g * a.v_head;
  u32x4 kx[STEP], vx[STEP];
  auto gload = [&](int kt, int t0) {
    const bool pre = kt < ks.np;                    // workgroup-uniform
    const T *kb = pre ? pk : kg, *vb = pre ? pv : vg;
    const int64_t krow = pre ? a.pk_row : a.k_row, vrow = pre ? a.pv_row : a.v_row;
    const int first = (pre ? kt : kt - ks.np) * KT, n = pre ? a.p_len : ks.klen;
#pragma unroll
    for (int t = 0; t < STEP; ++t) {
      const int idx = tid + (t0 + t) * kThreads, c = idx % NCH;
      const int key = first + idx / NCH;
      const int kc = min(key, n - 1), cc = c * E < a.d ? c * E : 0;   // an address inside in any case
      const u32x4 x = *(const u32x4 *)(kb + (int64_t)kc * krow + cc);
      const u32x4 y = *(const u32x4 *)(vb + (int64_t)kc * vrow + cc);
      const bool ok = key < n && c * E < a.d;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        kx[t][w] = ok ? x[w] : 0;
        vx[t][w] = ok ? y[w] : 0;
      }
    }
  };
  auto lstore = [&](int kt, int t0) {
    if (kt >= ks.np && (kt - ks.np + 1) * KT > all_see) {      // workgroup-uniform
      bool any = false;
#pragma unroll
      for (int t = 0; t < STEP; ++t) any |= tame<T>(vx[t]);
      if (any) wild[wave] = 1;
    }
#pragma unroll
    for (int t = 0; t < STEP; ++t) {
      const int idx = tid + (t0 + t) * kThreads, row = idx / NCH, c = idx % NCH;
      sk[((row >> 5) * NCH + c) * 32 + ((row & 31) ^ (c & 7))] = kx[t];
      *(u32x4 *)(sv + (row * NCH + value_chunk<NCH, B16>(row, c)) * 16) = vx[t];
    }
  };

  if (lane == 0) wild[wave] = 0;
  if constexpr (AHEAD)
    if (span.lo < span.hi) gload(span.lo, 0);       // workgroup-uniform
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

  auto compute = [&](int kt) {
    const bool pre = kt < ks.np;
    const int at = (pre ? kt : kt - ks.np) * KT + kw * 32;   // keys of the source before this wave's
    const int every = (pre ? a.p_len : least) - at, n = (pre ? a.p_len : mine) - at;
    f32x16 s[1];
    key_scores<T, DP>(s[0], sk, qf, kw, lane);
    if (every < 32) mask_below(s[0], n, lane);      // wave-uniform
    float sc = a.sc, ref;
    st.raise(s, max16(s[0], -INFINITY) * sc, sc, ref);
    add_values<T, DP>(st.o, probs_of<T>(s[0], sc, ref, st.l), sv, kw, lane);
  };

  for (int kt = span.lo; kt < span.hi; ++kt) {
    __syncthreads();                                // the tile before is read
    if constexpr (AHEAD) {
      lstore(kt, 0);
    } else {
      for (int t0 = 0; t0 < CPT; t0 += STEP) {
        gload(kt, t0);
        lstore(kt, t0);
      }
    }
    __syncthreads();
    if constexpr (AHEAD)
      if (kt + 1 < span.hi) gload(kt + 1, 0);
    if (r0 < rows) compute(kt);                     // wave-uniform
  }
  bool found = false;
  if (ks.cross) {
    __syncthreads();
    found = wild[0] | wild[1] | wild[2] | wild[3];
  }
  if constexpr (KW > 1) {
    __syncthreads();
    join_waves<ND, KW>(st, (float *)lds, kw, lane);
    if (kw > 0) return;
  }
  if (r0 >= rows) return;
  if (found) {                                      // (before the waves are joined, wave 0's weight would reach them)
    const int from = max(max(span.lo - ks.np, 0) * KT, all_see / KT * KT), to = min((span.hi - ks.np) * KT, ks.klen);
    add_wild<T, ND>(st.o, vg, a.v_row, a.d, from, to, mine, lane);
  }
  if (span.used == 1 && !a.shared) store_rows<T, ND>(a, st, 1.f, live, tok, head, lane);
  else store_part<ND>(a, st, 1.f, live, a.unit0 + tile, g, 0, rw * 32 + lrow, lane);
}

// As k_cross_stream: four waves of 32 rows over a ring of 32-key tiles that LDS-direct copies fill.
// One pass over many keys is bound by vector work and its waits: 16 x 1024 rows of 10 heads of 64 over 480 + 320 tokens 54
// to 59 us, 600 TFLOP/s (of the matrix cores 13 us, vector instructions about 33; without products and softmax 34). Shared, by
// bytes: one query of 64 streams over 16384 + 1 to 320 tokens, 2 x 8 heads of 128, 30 us for 113 MB of keys and 20 MB
// of partial results, the join 6. Slower were: two tiles a barrier (56 and 40 us), five workgroups a compute unit at 96
// registers (61), the heads of a key tile on one XCD (59 and 41).
template <int DP>
__global__ __launch_bounds__(kThreads, DP == 64 ? 4 : 3) void k_prefix_stream(PrefixArgs a) {
  typedef Stream<DP> S;
  constexpr int NCH = S::NCH, NK = NCH / 2, ND = DP / 32, CP = S::COPIES;
  extern __shared__ u32x4 lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lrow = lane & 31, h = lane >> 5;
  const Unit un = unit_of(a);
  const int tile = un.tile, g = un.g;
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, tile)];
  const Keys ks = keys_of(a, sq, 32);
  const int rows = sq.q_len * a.rep;
  const Part span = part_in(a, sq, ks, tile - sq.tile0, rows, 128, 32);
  const int r0 = span.row_tile * 128 + wave * 32;
  const int mine = ks.seen(min(r0 + lrow, rows - 1) / a.rep), least = ks.seen(r0 / a.rep);
  const int all_see = ks.cross ? ks.seen(span.row_tile * 128 / a.rep) : INT_MAX;   // every row of the tile does
  uint32_t *wild = (uint32_t *)(lds + S::BYTES / 16);   // a word a wave: it found some
  if (lane == 0) wild[wave] = 0;

  const bf16 *pk = (const bf16 *)a.pk + (int64_t)g * a.pk_head, *pv = (const bf16 *)a.pv + (int64_t)g * a.pv_head;
  const int64_t k0 = max(sq.k0, 0);
  const bf16 *kg = (const bf16 *)a.k + k0 * a.k_row + (int64_t)g * a.k_head;
  const bf16 *vg = (const bf16 *)a.v + k0 * a.v_row + (int64_t)g * a.v_head;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  // copy i of this wave: rows RPC (wave CP + i) .. of the tile
  constexpr int RPC = 64 / NCH;
  auto copy_tile = [&](int t) {
    const bool pre = t < ks.np;
    const int first = (pre ? t : t - ks.np) * 32, n = pre ? a.p_len : ks.klen;
    const uint32_t krow = (uint32_t)(pre ? a.pk_row : a.k_row), vrow = (uint32_t)(pre ? a.pv_row : a.v_row);
    const bf16 *kb = (pre ? pk : kg) + (int64_t)first * krow, *vb = (pre ? pv : vg) + (int64_t)first * vrow;
    const uint32_t to = lds0 + (uint32_t)(((t - span.lo) % S::NB) * 2 * S::TILE + wave * CP * 64) * 16;
#pragma unroll
    for (int i = 0; i < CP; ++i) {
      const int r = RPC * (wave * CP + i) + lane / NCH, p = lane % NCH;
      const int row = min(r, n - 1 - first);
      const int kc = key_swz<NCH>(r, p) * 8, vc = value_chunk<NCH, true>(r, p) * 8;
      if (kc < a.d) dma16(kb, (__umul24(row, krow) + kc) * 2u, to + i * 1024);
      if (vc < a.d) dma16(vb, (__umul24(row, vrow) + vc) * 2u, to + (S::TILE + i * 64) * 16);
    }
  };
  const TileRows rw(a, sq, r0, rows);
  QTile<bf16, DP> qt;
  if (r0 < rows) qt.load(a, rw, g, lane);
  const int t0 = span.lo, t1 = span.hi;
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
    const bool pre = t < ks.np;
    const int first = (pre ? t : t - ks.np) * 32, n = (pre ? a.p_len : ks.klen) - first;
    if (t + 1 < t1) wait_vm<2 * CP>();              // this tile's copies: the next one's are younger
    else wait_vm<0>();
    if (n < 32) {                                   // value rows past the end
#pragma unroll
      for (int i = 0; i < CP; ++i)
        if (RPC * (wave * CP + i) + lane / NCH >= n) ((u32x4 *)sv)[(wave * CP + i) * 64 + lane] = u32x4{0, 0, 0, 0};
    }
    if (!pre && first + 32 > all_see) {             // uniform
#pragma unroll
      for (int i = 0; i < CP; ++i) {
        u32x4 *at = (u32x4 *)sv + (wave * CP + i) * 64 + lane, x = *at;
        if (tame<bf16>(x)) {
          *at = x;
          wild[wave] = 1;
        }
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
      const int every = pre ? n : least - first;
      if (every < 32) mask_below(s[0], pre ? n : mine - first, lane);
      float sc = a.sc, ref;
      st.raise(s, max16(s[0], -INFINITY) * sc, sc, ref);
      add_values<bf16, DP>(st.o, probs_of<bf16>(s[0], sc, ref, st.l), (const char *)sv, 0, lane);
    }
  }
  if (ks.cross) {
    __syncthreads();
    if (r0 < rows && (wild[0] | wild[1] | wild[2] | wild[3]))
      add_wild<bf16, ND>(st.o, vg, a.v_row, a.d, max(max(t0 - ks.np, 0) * 32, all_see / 32 * 32),
                         min((t1 - ks.np) * 32, ks.klen), mine, lane);
  }
  if (r0 >= rows) return;
  // all slots but the last tile's and the one before hold nothing that is still read
  constexpr int ROOM = S::NB * 2 * S::TILE;
  int free0 = t1 > t0 ? (t1 - t0) % S::NB * 2 * S::TILE : 0;
  free0 += wave * (kBox / 16);
  if (free0 >= ROOM) free0 -= ROOM;
  if (span.used > 1 || a.shared) store_part_rows<ND>(a, st, rows - r0, a.unit0 + tile, g, wave * 32, lds + free0, lane);
  else store_tile<bf16, ND>(a, st, 1.f, rw, g, lds + free0, lane);
}

// ---- joining parts ------------------------------------------------------------------------------
//
// out[row] = sum_s w_s O_s / sum_s w_s, w_s = 2^(m_s - M) l_s, M = max m_s, over the parts of the row's list and,
// shared, first those of the prefix. Sequences as for the launch before, but k0: first unit, k_len: parts,
// tile0: first tile of rows here.
struct Parts {
  const float *ws;
  int64_t ml, p_at, p_step, at, step;
  int np, n;
  __device__ __forceinline__ int64_t place(int s) const { return s < np ? p_at + s * p_step : at + (s - np) * step; }
};
struct JoinArgs : AttnCommon {
  int p_parts, p_tiles, TR;
  CondSeq seq[kCondSeqs];
};
__device__ __forceinline__ Parts parts_at(const JoinArgs &a, const CondSeq &sq, int g, int r) {
  const int rows = sq.q_len * a.rep, tiles = (rows + a.TR - 1) / a.TR;
  Parts p;
  p.ws = a.ws;
  p.ml = a.ws_ml;
  const int64_t all = (int64_t)sq.q0 * a.rep + r;   // the row among those of all sequences
  p.p_at = (all / a.TR * a.hkv + g) * a.ws_rows + all % a.TR;
  p.p_step = (int64_t)a.p_tiles * a.hkv * a.ws_rows;
  p.at = ((int64_t)(sq.k0 + r / a.TR) * a.hkv + g) * a.ws_rows + r % a.TR;
  p.step = (int64_t)tiles * a.hkv * a.ws_rows;
  p.np = a.p_parts;
  p.n = a.p_parts + sq.k_len;
  return p;
}
template <typename T>
__device__ __forceinline__ void store_four(const AttnCommon &a, const CondSeq &sq, int g, int r, int c, const f32x4 &x) {
  T *row = (T *)a.out + (int64_t)(sq.q0 + r / a.rep) * a.o_row + (int64_t)(g * a.rep + r % a.rep) * a.o_head;
  if constexpr (sizeof(T) == 4)
    *(f32x4 *)(row + c) = x;
  else
    *(bf16x4 *)(row + c) = bf16x4{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
}

// TEAMS teams of DP / 4 lanes take a row's parts in turn; a workgroup holds 256 / (TEAMS DP / 4) rows.
template <typename T, int DP, int TEAMS>
__global__ __launch_bounds__(kThreads) void k_prefix_join(JoinArgs a) {
  constexpr int LPR = DP / 4, ROWS = kThreads / (LPR * TEAMS);
  __shared__ f32x4 sums[TEAMS > 1 ? kThreads : 1];
  __shared__ float2 tops[TEAMS > 1 ? kThreads / LPR : 1];
  const Unit un = unit_of(a);
  const CondSeq sq = a.seq[find_seq(a.seq, a.n_seq, un.tile)];
  const int rows = sq.q_len * a.rep, tid = threadIdx.x, c = (tid % LPR) * 4, team = tid / LPR % TEAMS;
  const int i = blockIdx.y * ROWS + tid / (LPR * TEAMS), r = (un.tile - sq.tile0) * a.TR + i;
  const bool mine = i < a.TR && r < rows;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  if (mine) {
    const Parts p = parts_at(a, sq, un.g, r);
    // U parts at a time, relative to the largest so far
    constexpr int U = 8;
    for (int s0 = team; s0 < p.n; s0 += U * TEAMS) {
      float ms[U], ls[U];
      f32x4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int s = s0 + u * TEAMS;
        const int64_t at = p.place(min(s, p.n - 1));
        ms[u] = s < p.n ? p.ws[p.ml + at * 2] : -INFINITY;
        ls[u] = s < p.n ? p.ws[p.ml + at * 2 + 1] : 0.f;
        x[u] = *(const f32x4 *)(p.ws + at * DP + c);
      }
      float top = m;
#pragma unroll
      for (int u = 0; u < U; ++u) top = fmaxf(top, ms[u]);
      const float ref = finite_ref(top);
      const float f = __builtin_amdgcn_exp2f(m - ref);
      l *= f;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] *= f;
      m = top;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = __builtin_amdgcn_exp2f(ms[u] - ref) * ls[u];
        l += w;
        if (s0 + u * TEAMS < p.n) {
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] = fmaf(w, x[u][e], acc[e]);
        }
      }
    }
  }
  if constexpr (TEAMS > 1) {
    sums[tid] = acc;
    if (tid % LPR == 0) tops[tid / LPR] = float2{m, l};
    __syncthreads();
    if (team > 0 || !mine) return;
    float top = m;
#pragma unroll
    for (int t = 1; t < TEAMS; ++t) top = fmaxf(top, tops[tid / LPR + t].x);
    const float ref = finite_ref(top), f0 = __builtin_amdgcn_exp2f(m - ref);
    l *= f0;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] *= f0;
#pragma unroll
    for (int t = 1; t < TEAMS; ++t) {
      const float2 o = tops[tid / LPR + t];
      const float f = __builtin_amdgcn_exp2f(o.x - ref);
      const f32x4 x = sums[tid + t * LPR];
      l = fmaf(f, o.y, l);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = fmaf(f, x[e], acc[e]);
    }
  }
  if (!mine || c >= a.d) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] *= inv;
  store_four<T>(a, sq, un.g, r, c, acc);
}

// ---- host ---------------------------------------------------------------------------------------

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
// Tiles of 32 or 128 (a call's plan counts them a dozen times a sequence: no divisions).
int tiles_of(int64_t n, int size) { return (int)(size == 32 ? (n + 31) >> 5 : (n + 127) >> 7); }
int pad_d(int d) { return d <= 64 ? 64 : 128; }

constexpr int kFill = 512;           // workgroups that fill the compute units with two each

// How a call is done; by its sizes alone, so that the workspace can be asked for.
// Shared where that saves more than 2048 steps of a row tile over 32 keys, about what the join costs (us shared / one
// pass: 64 streams of one query over 16384 tokens 38 / 375, over 1024 19 / 34, 8 over 2048 13 / 20, 32 over 512 13 / 18;
// 12 of 20 over 3000 25 / 22; 16 x 1024 over 480 92 / 60). All rows of bf16 then go through tiles of 128, also where 16
// streams fill 32 (16 over 16384: 23 us against 28 in tiles of 32, which split the keys over waves).
// Lists are cut into about kFill workgroups (256 or 1024 instead: 44 and 47 us against 41, before partial results
// were written in whole lines), in parts of 128 keys at least (256: 64 streams over 1024 20 us against 19).
struct Plan {
  enum Kind { FEW, MANY } kind = FEW;
  int TR = 32, KT = 128;             // rows of a tile, keys of the tiles that ranges are cut in
  bool shared = false;
  KeyCut p_cut{1, INT_MAX}, cut{1, INT_MAX};
  int p_tiles = 0, p_parts = 0;      // shared: row tiles of all rows, parts of the prefix
  int64_t units = 0;                 // with partial results, of the launch with the most; p_tiles * p_parts among them
  int most = 0;                      // parts of a row
  int ws_rows = 0;
  int64_t rows_at_once = 0;          // the most rows of one sequence
  int64_t floats(int hkv, int dp) const { return units * hkv * (int64_t)ws_rows * (dp + 2); }
  int64_t ml(int hkv, int dp) const { return units * hkv * (int64_t)ws_rows * dp; }
};

// Cuts of lists of `work` = sum of row tiles x key tiles into about kFill workgroups, parts of `least` tiles at least.
KeyCut cut_for(double work, int hkv, int least, int from, int longest) {
  KeyCut c;
  c.per = (int)std::min(std::max((double)least, std::ceil(work * hkv / kFill)), 0x1p29);
  c.per = std::max(c.per, ceil_div(longest, kMaxParts - 2));
  c.from = from;
  return c;
}

Plan prefix_plan(const AttnProblem &p, int p_len, const int32_t *kv_lens) {
  Plan pl;
  const int rep = p.c.rep, hkv = p.c.hkv;
  int64_t all = 0, tiles32 = 0;
  for (int i = 0; i < p.n; ++i) {
    const int64_t rows = (int64_t)p.q_lens[i] * rep;
    all += rows;
    tiles32 += tiles_of(rows, 32);
    pl.rows_at_once = std::max(pl.rows_at_once, rows);
  }
  if (all == 0) return pl;
  const bool b16 = p.dtype == MTE_BF16;
  // one pass: as cross attention, tiles of 32 rows where the rows are few
  const bool few = pl.rows_at_once <= 32 || tiles32 * hkv < 256;
  // steps of a row tile over 32 keys, both ways
  const int TR1 = few ? 32 : 128, TR2 = all <= 32 && !b16 ? 32 : 128;
  double one = 0, two = (double)tiles_of(all, TR2) * tiles_of(p_len, 32);
  for (int i = 0; i < p.n; ++i) {
    const int64_t rows = (int64_t)p.q_lens[i] * rep;
    if (rows == 0) continue;
    one += (double)tiles_of(rows, TR1) * (tiles_of(p_len, 32) + tiles_of(kv_lens[i], 32));
    two += (double)tiles_of(rows, TR2) * tiles_of(kv_lens[i], 32);
  }
  pl.shared = p_len > 0 && (one - two) * hkv > 2048;
  pl.TR = pl.shared ? TR2 : TR1;
  pl.kind = pl.TR == 32 ? Plan::FEW : Plan::MANY;
  pl.KT = pl.kind == Plan::FEW ? 128 : 32;
  const int least = pl.kind == Plan::FEW ? (b16 ? 2 : 1) : 128 / pl.KT;
  const int from = pl.kind == Plan::FEW ? (b16 ? 8 : p.c.d > 64 ? 3 : 4) : 0;
  const int np = tiles_of(p_len, pl.KT);
  double work = 0;
  int longest = 0;
  const auto list = [&](int i) { return (pl.shared ? 0 : np) + tiles_of(kv_lens[i], pl.KT); };
  for (int i = 0; i < p.n; ++i)
    if (p.q_lens[i] > 0) {
      work += (double)tiles_of((int64_t)p.q_lens[i] * rep, pl.TR) * list(i);
      longest = std::max(longest, list(i));
    }
  if (pl.shared) {
    pl.p_tiles = tiles_of(all, pl.TR);
    work += (double)pl.p_tiles * np;
    pl.p_cut = cut_for(work, hkv, least, 0, np);
    pl.p_parts = parts_of(np, pl.p_cut);
  }
  pl.cut = cut_for(work, hkv, least, pl.shared ? 0 : from, longest);
  // units with partial results of the fullest launch
  int64_t at = 0, top = 0;
  int in = pl.shared ? 1 : 0, own = 0;
  for (int i = 0; i < p.n; ++i) {
    if (p.q_lens[i] == 0) continue;
    const int used = list(i) == 0 ? 0 : parts_of(list(i), pl.cut);
    own = std::max(own, used);
    if (used > 1 || pl.shared) at += (int64_t)tiles_of((int64_t)p.q_lens[i] * rep, pl.TR) * used;
    top = std::max(top, at);
    if (++in == kCondSeqs) in = 0, at = 0;
  }
  pl.units = (int64_t)pl.p_tiles * pl.p_parts + top;
  pl.most = pl.p_parts + own;
  pl.ws_rows = (int)std::min<int64_t>(pl.TR, pl.shared ? all : pl.rows_at_once);
  return pl;
}

template <typename K> hipError_t allow_lds(K kern, int bytes) {
  return bytes <= 65536 ? hipSuccess
                        : hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <typename T, int DP>
hipError_t run(PrefixArgs &a, const Plan &pl, bool copies, hipStream_t s) {
  // units of the launch: the prefix's first, then those with partial results, then longest first
  struct Item { int rank, tiles, used, seq; };
  Item item[kCondSeqs];
  CondSeq seq[kCondSeqs];
  const int np = tiles_of(a.p_len, pl.KT);
  for (int i = 0; i < a.n_seq; ++i) {
    const CondSeq &q = seq[i] = a.seq[i];
    const bool alone = q.k0 < 0;
    const int nt = alone ? np : (pl.shared ? 0 : np) + tiles_of(q.k_len, pl.KT);
    const int used = nt == 0 && pl.shared ? 0 : parts_of(nt, alone ? pl.p_cut : pl.cut);
    item[i] = Item{alone ? INT_MAX : used > 1 ? INT_MAX - 1 : nt, tiles_of((int64_t)q.q_len * a.rep, pl.TR), used, i};
  }
  std::stable_sort(item, item + a.n_seq, [](const Item &x, const Item &y) { return x.rank > y.rank; });
  JoinArgs j;
  (AttnCommon &)j = a;
  j.p_parts = pl.p_parts;
  j.p_tiles = pl.p_tiles;
  j.TR = pl.TR;
  j.n_seq = 0;
  int units = 0, join_tiles = 0, n = 0;
  for (int i = 0; i < a.n_seq; ++i) {
    const Item &it = item[i];
    CondSeq q = seq[it.seq];
    q.tile0 = units;
    if (q.k0 >= 0 && (pl.shared || it.used > 1)) {
      j.seq[j.n_seq++] = CondSeq{q.q0, q.q_len, a.unit0 + units, it.used, join_tiles};
      join_tiles += it.tiles;
    }
    units += it.tiles * it.used;
    if (it.used > 0) a.seq[n++] = q;                 // (no keys at all: nothing but the join)
  }
  a.n_seq = n;
  hipError_t e;
  if (n > 0) {
    auto kern = pl.kind == Plan::FEW ? k_prefix<T, DP, 1> : k_prefix<T, DP, 4>;
    int lds = 2 * pl.KT * DP * (int)sizeof(T) + 16;
    if (pl.kind == Plan::FEW) lds = std::max(lds, 3 * (2 + DP / 2) * 64 * 4);
    if constexpr (sizeof(T) == 2) {
      if (copies) {
        kern = k_prefix_stream<DP>;
        lds = Stream<DP>::BYTES + 16;
      }
    }
    if ((e = allow_lds(kern, lds)) != hipSuccess) return e;
    e = in_launches(a, (int64_t)units * a.hkv,
                    [&](uint32_t n) { hipLaunchKernelGGL(kern, dim3(n), dim3(kThreads), lds, s, a); });
    if (e != hipSuccess) return e;
  }
  if (j.n_seq == 0) return hipSuccess;
  const int most = (int)std::min<int64_t>(pl.TR, pl.rows_at_once);
  const bool teams = pl.most > 8;
  auto join = teams ? k_prefix_join<T, DP, kThreads / (DP / 4)> : k_prefix_join<T, DP, 1>;
  const int across = teams ? most : ceil_div(most, kThreads / (DP / 4));
  return in_launches(j, (int64_t)join_tiles * a.hkv,
                     [&](uint32_t n) { hipLaunchKernelGGL(join, dim3(n, across), dim3(kThreads), 0, s, j); });
}

}  // namespace

int64_t prefix_workspace(const AttnProblem &p, int p_len, const int32_t *kv_lens) {
  return prefix_plan(p, p_len, kv_lens).floats(p.c.hkv, pad_d(p.c.d)) * 4;
}

hipError_t launch_prefix(const AttnProblem &p, const PrefixRows &x, const int32_t *kv_lens, int causal, hipStream_t s) {
  const Plan pl = prefix_plan(p, x.p_len, kv_lens);
  const int dp = pad_d(p.c.d);
  PrefixArgs a;
  (AttnCommon &)a = p.c;
  int64_t rows = 0;
  for (int i = 0; i < p.n; ++i) rows += p.q_lens[i];
  a.big = rows * p.c.rep * p.c.hkv * p.c.d * (p.dtype == MTE_BF16 ? 2 : 4) > (32 << 20);
  a.k = x.k;
  a.v = x.v;
  a.pk = x.pk;
  a.pv = x.pv;
  a.k_row = x.k_row;
  a.k_head = x.k_head;
  a.v_row = x.v_row;
  a.v_head = x.v_head;
  a.pk_row = x.pk_row;
  a.pk_head = x.pk_head;
  a.pv_row = x.pv_row;
  a.pv_head = x.pv_head;
  a.p_len = x.p_len;
  a.causal = causal;
  a.shared = pl.shared;
  a.p_cut = pl.p_cut;
  a.cut = pl.cut;
  a.n_split = 1;
  a.ws_rows = pl.ws_rows;
  a.ws_ml = pl.ml(a.hkv, dp);
  const bool copies = pl.kind == Plan::MANY && p.near_rows && p.near_tiles;
  bool first = pl.shared;
  int64_t q0 = 0, k0 = 0;
  for (int i = 0; i < p.n;) {
    a.n_seq = 0;
    a.unit0 = first || !pl.shared ? 0 : pl.p_tiles * pl.p_parts;
    if (first) a.seq[a.n_seq++] = CondSeq{0, (int)rows, -1, 0, 0};
    first = false;
    for (; i < p.n && a.n_seq < kCondSeqs; ++i) {
      if (p.q_lens[i] > 0) a.seq[a.n_seq++] = CondSeq{(int)q0, p.q_lens[i], (int)k0, kv_lens[i], 0};
      q0 += p.q_lens[i];
      k0 += kv_lens[i];
    }
    if (a.n_seq == 0) break;
    hipError_t e;
    if (p.dtype == MTE_BF16)
      e = dp == 64 ? run<bf16, 64>(a, pl, copies, s) : run<bf16, 128>(a, pl, copies, s);
    else
      e = dp == 64 ? run<float, 64>(a, pl, false, s) : run<float, 128>(a, pl, false, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mte
