// Host-side launchers of the operators that read the conditioning (internal to libmte).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace mte {

// Sequences per launch: their table goes to the kernels by value (kernel
// arguments are at most 4 KB); more sequences take several launches.
constexpr int kCondSeqs = 128;

// Workgroups of a launch, of 512 threads or fewer: a launch counts its threads in 32 bits, and drops
// those beyond without an error.
constexpr int kMostGroups = 1 << 22;

struct CondSeq {
  int q0, q_len;   // first packed query (or appended / read) row, rows
  int k0, k_len;   // first packed key row, key rows; the cache operators: row of the block table; attention
                   // over it: queries of the sequence from q0 on (a chunk's: more than q_len)
  int tile0;       // first tile (or unit: tile and part of the keys) of the sequence in the launch
};

// What the three attention kernels share. Strides in elements.
struct AttnCommon {
  const void *q;
  void *out;
  float *ws;                         // partial results: see join_row
  int64_t q_row, q_head, o_row, o_head;
  float sc;                          // scale * log2(e)
  int d, hkv, rep;
  int n_seq, n_split, ws_rows;       // ws_rows: rows of a tile's partial result
  int64_t ws_ml;                     // float offset of the (m, l) pairs in ws
  int big;                           // out is more than the caches hold
  int first;                         // workgroup of the call that the launch begins with (in_launches)
};

// A call of `groups` workgroups in launches of kMostGroups; launch(workgroups) with a.first set.
template <typename A, typename F> hipError_t in_launches(A &a, int64_t groups, F launch) {
  for (int64_t at = 0; at < groups; at += kMostGroups) {
    a.first = (int)at;
    launch((uint32_t)(groups - at < kMostGroups ? groups - at : kMostGroups));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// How key ranges are cut: key tiles of a part, and of the shortest range that is cut.
struct KeyCut { int per, from; };

struct CrossArgs : AttnCommon {
  const void *k, *v;
  const uint8_t *mask;
  int64_t k_row, k_head, v_row, v_head;
  KeyCut cut;
  CondSeq seq[kCondSeqs];
};

struct Kv8View {
  uint8_t *k_codes, *v_codes;
  float *scales;
  const int32_t *table, *kv_lens;
  int64_t table_row;
  int width, n_blocks, hkv, d;
};

struct Kv8AttnArgs : AttnCommon {
  Kv8View c;
  int causal;
  CondSeq seq[kCondSeqs];
};

struct Kv8RowsArgs {                 // append and read
  Kv8View c;
  const void *k, *v;                 // append: sources
  void *ko, *vo;                     // read: destinations
  int64_t k_row, k_head, v_row, v_head;
  int n_seq;
  int first;                         // tile that the launch begins with (in_launches)
  CondSeq seq[kCondSeqs];
};

// One attention problem as the API has checked it. q_lens, kv_lens, kv_index: host.
struct AttnProblem {
  AttnCommon c;
  int dtype;                         // MTE_F32 / MTE_BF16
  bool near_rows;                    // key and value rows under 2^24 elements apart: 32 of them are 32-bit offsets
  bool near_tiles;                   // the same of the query and result rows of a tile, heads of a group included
  const int32_t *q_lens;
  int n;
};

// Bytes of workspace of the launches below for these lengths.
int64_t cross_workspace(const AttnProblem &p, const int32_t *kv_lens, int n_kv, const int32_t *kv_index);
int64_t kv8_workspace(const AttnProblem &p, int width);

hipError_t launch_cross(const AttnProblem &p, const void *k, const void *v, const uint8_t *mask, int64_t k_row,
                        int64_t k_head, int64_t v_row, int64_t v_head, const int32_t *kv_lens, int n_kv,
                        const int32_t *kv_index, hipStream_t s);
hipError_t launch_kv8_attention(const AttnProblem &p, const Kv8View &c, int causal, hipStream_t s);

hipError_t launch_kv8_append(const Kv8View &c, const void *k, int64_t k_row, int64_t k_head, const void *v,
                             int64_t v_row, int64_t v_head, int dtype, const int32_t *new_lens, int n, hipStream_t s);
hipError_t launch_kv8_read(const Kv8View &c, const int32_t *counts, int n, void *k, void *v, int dtype,
                           hipStream_t s);

struct GroupNormArgs {
  const void *x, *gamma, *beta;
  void *y;
  float *ws;
  int64_t x_row, x_image, y_row, y_image;
  int n, pixels, channels, groups, act;
  float eps;
};
int64_t group_norm_workspace(int n, int pixels, int channels, int groups, int dtype);
hipError_t launch_group_norm(const GroupNormArgs &a, int dtype, hipStream_t s);

}  // namespace mte
