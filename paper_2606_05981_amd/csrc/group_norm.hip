// Group norm with an activation, channels last:
//   y = act((x - mean) / sqrt(var + eps) * gamma[c] + beta[c])
// over the pixels and the cpg = C / G channels of a group of one image.
//
// A thread keeps one column of V channels and walks pixels; sums go through LDS per group, twice:
// the mean first, then the squares around it, so that a large mean cancels nowhere. Two shapes:
//
// k_gn, one launch: a workgroup holds a bundle of whole groups (neighbouring channels, so that rows
// are read in runs) of a whole image in LDS. x is read once, y written once.
//
// k_gn_stats + k_gn_apply, where an image does not fit or its workgroups would be too few:
// workgroups take chunks of pixels over as many groups as they have columns for. A thread runs
// (count, mean, squares around it) per channel over batches of pixels, the workgroup joins its
// threads' and leaves (count, mean, squares) of the part in the workspace; the second launch
// joins the parts while its pixels load. x is read twice, the second time mostly from the caches.
//
// Large images are bound by those bytes (16 x 64 x 64 x 320: 32.7 us for 126 MB, the second read from the caches;
// at the card's copy rate 84 MB take 16.4), small ones by the chain of a launch: loads, two sums through
// LDS, stores (8 x 8 x 1280: 7.4 us). That chain's code runs once per workgroup, so it is kept short: held
// in registers and unrolled (16 vectors a thread), the same 8x8x1280 image took 9.1 us, most of it
// fetching instructions.
#include <algorithm>

#include "../../include/mte_cond.h"
#include "common.h"
#include "cond_launch.h"

namespace mte {

namespace {

template <int BYTES> struct Raw;
template <> struct Raw<16> { typedef u32x4 type; };
template <> struct Raw<8> { typedef u32x2 type; };
template <> struct Raw<4> { typedef uint32_t type; };
template <> struct Raw<2> { typedef uint16_t type; };

constexpr int kBatch = 4;      // vectors of a thread in flight at a time

struct GnArgs : GroupNormArgs {
  int cpg, gb;         // channels per group, groups per bundle
  int ncol;            // columns (of V channels) of a bundle
  int ppi;             // pixels a workgroup takes at a time
  int chunk;           // pixels per workgroup: of k_gn_stats,
  int apply;           // of k_gn_apply
  int parts;           // of k_gn_stats: chunks x column parts
  int colparts;        // a bundle wider than a workgroup (then one group): its parts
  int same;            // a column lies inside one group
};

template <typename T, int V> struct Vec {
  typedef typename Raw<V * sizeof(T)>::type raw;
  static __device__ __forceinline__ raw load(const T *p) { return *(const raw *)p; }
  static __device__ __forceinline__ void unpack(const raw &r, float *x) {
    T t[V];
    __builtin_memcpy(t, &r, sizeof(raw));
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = to_f32(t[e]);
  }
  static __device__ __forceinline__ raw pack(const float *x) {
    T t[V];
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] = from_f32<T>(x[e]);
    raw r;
    __builtin_memcpy(&r, t, sizeof(raw));
    return r;
  }
};

// Where a thread works: its column, pixel lane and first channel.
struct Place { int col0, ncol, g0, col, p0, ch; bool on; };
template <int V, int TH> __device__ __forceinline__ Place place_of(const GnArgs &a, int colpart) {
  Place w;
  w.col0 = colpart * TH;
  w.ncol = min(a.ncol - w.col0, TH);
  w.g0 = blockIdx.y * a.gb;
  w.p0 = threadIdx.x / w.ncol;
  w.col = threadIdx.x - w.p0 * w.ncol;
  w.on = w.p0 < a.ppi;
  w.ch = w.g0 * a.cpg + (w.col0 + w.col) * V;
  return w;
}

// Threads that sum a group, all groups of the bundle at once: a power of two.
template <int TH> __device__ __forceinline__ int team_of(int ng) { return 1 << (31 - __builtin_clz(max(TH / ng, 1))); }
__device__ __forceinline__ float team_sum(float s, int lanes) {   // within a wave
  for (int m = min(lanes, 64) >> 1; m >= 1; m >>= 1) s += __shfl_xor(s, m, kWave);
  return s;
}

// gs[i] = sum over the threads and channels of group i of the bundle of `v` (per thread and
// channel of its column).
template <int V, int TH>
__device__ __forceinline__ void group_sums(const GnArgs &a, const float (&v)[V], const Place &w, float *part, float *gs) {
  const int tid = threadIdx.x;
  // odd: entries of neighbouring lanes in different banks, where a column is one entry (`same`); else they are V
  // pitches apart and V of them meet in a bank (16 x 64 x 64 x 320: two thirds of k_gn_stats's LDS cycles)
  const int pitch = a.ppi | 1;
  const int ng = a.gb;
  int per;                                          // entries of a group, in a run
  __syncthreads();                                  // part and gs are free
  if (a.same) {
    per = (ng == 1 ? w.ncol : a.cpg / V) * pitch;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) s += v[e];
    if (w.on) part[w.col * pitch + w.p0] = s;
    if (w.p0 == 0 && pitch > a.ppi) part[w.col * pitch + a.ppi] = 0.f;
  } else {
    per = a.cpg * pitch;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if (w.on) part[(w.col * V + e) * pitch + w.p0] = v[e];
      if (w.p0 == 0 && pitch > a.ppi) part[(w.col * V + e) * pitch + a.ppi] = 0.f;
    }
  }
  __syncthreads();
  const int team = team_of<TH>(ng), j0 = tid & (team - 1);
  for (int i0 = 0; i0 < ng; i0 += TH / team) {      // one round while ng <= TH
    const int i = i0 + tid / team;
    float s = 0.f;
    if (i < ng) {
#pragma unroll 4
      for (int j = j0; j < per; j += team) s += part[i * per + j];
    }
    s = team_sum(s, team);
    if (team <= 64) {
      if (i < ng && j0 == 0) gs[i] = s;
    } else {                                        // a team of several waves: one round
      __syncthreads();                              // part is read
      if ((tid & 63) == 0) part[tid >> 6] = s;
      __syncthreads();
      const int nw = team / 64;
      if (tid < ng) {
        s = 0.f;
        for (int k = 0; k < nw; ++k) s += part[tid * nw + k];
        gs[tid] = s;
      }
    }
  }
  __syncthreads();
}

template <int V>
__device__ __forceinline__ void normalise(const GnArgs &a, const float *x, const float *mean, const float *rstd,
                                          const float *gam, const float *bet, float *y) {
#pragma unroll
  for (int e = 0; e < V; ++e) y[e] = fmaf((x[e] - mean[e]) * rstd[e], gam[e], bet[e]);
  if (a.act == MTE_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < V; ++e)
      y[e] *= __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * y[e]));
  }
}

template <typename T, int V>
__device__ __forceinline__ void affine(const GnArgs &a, int ch, float *gam, float *bet) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    gam[e] = a.gamma ? to_f32(((const T *)a.gamma)[ch + e]) : 1.f;
    bet[e] = a.beta ? to_f32(((const T *)a.beta)[ch + e]) : 0.f;
  }
}

// One launch. Grid: y = bundle, z = image. LDS: gs [gb], part, then the slab [round][thread].
template <typename T, int V, int TH>
__global__ __launch_bounds__(TH) void k_gn(GnArgs a, int slab) {
  typedef Vec<T, V> vec;
  typedef typename vec::raw raw;
  extern __shared__ float lds[];
  float *gs = lds, *part = lds + a.gb;
  raw *mine = (raw *)((char *)lds + slab) + threadIdx.x;
  const Place w = place_of<V, TH>(a, 0);
  const T *x = (const T *)a.x + (int64_t)blockIdx.z * a.x_image + w.ch;
  const int end = w.on ? a.pixels : 0;
  float sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) sum[e] = 0.f;
  for (int p = w.p0, i = 0; p < end; p += kBatch * a.ppi, i += kBatch) {
    raw r[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k)                // past the end: the last pixel again
      r[k] = vec::load(x + (int64_t)min(p + k * a.ppi, a.pixels - 1) * a.x_row);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (p + k * a.ppi < a.pixels) {
        float f[V];
        vec::unpack(r[k], f);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] += f[e];
        mine[(i + k) * TH] = r[k];
      }
    }
  }
  float gam[V], bet[V];
  affine<T, V>(a, w.ch, gam, bet);
  group_sums<V, TH>(a, sum, w, part, gs);
  const float inv = 1.f / ((float)a.pixels * (float)a.cpg);
  float mean[V], rstd[V];
  int gi[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    gi[e] = a.gb == 1 ? 0 : (w.col * V + e) / a.cpg;
    mean[e] = gs[gi[e]] * inv;
    sum[e] = 0.f;
  }
#pragma unroll 2
  for (int p = w.p0, i = 0; p < end; p += a.ppi, ++i) {
    float f[V];
    vec::unpack(mine[i * TH], f);
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = fmaf(f[e] - mean[e], f[e] - mean[e], sum[e]);
  }
  group_sums<V, TH>(a, sum, w, part, gs);
#pragma unroll
  for (int e = 0; e < V; ++e) rstd[e] = 1.f / sqrtf(gs[gi[e]] * inv + a.eps);
  T *y = (T *)a.y + (int64_t)blockIdx.z * a.y_image + w.ch;
#pragma unroll 2
  for (int p = w.p0, i = 0; p < end; p += a.ppi, ++i) {
    float f[V], o[V];
    vec::unpack(mine[i * TH], f);
    normalise<V>(a, f, mean, rstd, gam, bet, o);
    *(raw *)(y + (int64_t)p * a.y_row) = vec::pack(o);
  }
}

// First of two launches. Grid: x = part (chunk x column part), y = bundle, z = image.
template <typename T, int V, int TH>
__global__ __launch_bounds__(TH) void k_gn_stats(GnArgs a) {
  typedef Vec<T, V> vec;
  extern __shared__ float lds[];
  float *gs = lds, *part = lds + a.gb;
  const int chunk = (int)blockIdx.x / a.colparts;
  const Place w = place_of<V, TH>(a, (int)blockIdx.x - chunk * a.colparts);
  const int px0 = chunk * a.chunk, npx = min(a.chunk, a.pixels - px0);
  const T *x = (const T *)a.x + (int64_t)blockIdx.z * a.x_image + (int64_t)px0 * a.x_row + w.ch;
  // this thread's pixels, a batch at a time: (n, mean, squares) of each channel so far
  float n = 0.f, mean[V], sq[V];
#pragma unroll
  for (int e = 0; e < V; ++e) mean[e] = sq[e] = 0.f;
  constexpr int B = 2 * kBatch;
  for (int p = w.p0; p < (w.on ? npx : 0); p += a.ppi * B) {
    const int left = (npx - p + a.ppi - 1) / a.ppi; // pixels of this batch
    typename vec::raw r[B];
#pragma unroll
    for (int i = 0; i < B; ++i)                     // past the end: the last one again, not counted
      r[i] = vec::load(x + (int64_t)(p + min(i, left - 1) * a.ppi) * a.x_row);
    float s[V], q[V];
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] = q[e] = 0.f;
#pragma unroll
    for (int i = 0; i < B; ++i) {
      float f[V];
      vec::unpack(r[i], f);
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] += i < left ? f[e] : 0.f;
    }
    const float k = (float)min(left, B), ik = 1.f / k, all = n + k;
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] *= ik;
#pragma unroll
    for (int i = 0; i < B; ++i) {
      float f[V];
      vec::unpack(r[i], f);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = i < left ? f[e] - s[e] : 0.f;
        q[e] = fmaf(d, d, q[e]);
      }
    }
    const float share = k / all, cross = n * share;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float d = s[e] - mean[e];
      mean[e] = fmaf(d, share, mean[e]);
      sq[e] += fmaf(d * cross, d, q[e]);            // (the first batch: cross = 0, and d the mean, whose square may overflow)
    }
    n = all;
  }
  float t[V];
#pragma unroll
  for (int e = 0; e < V; ++e) t[e] = n * mean[e];
  group_sums<V, TH>(a, t, w, part, gs);
  const float cnt = (float)npx * (float)(a.gb == 1 ? w.ncol * V : a.cpg), inv = 1.f / cnt;
  float gm[V];
  int gi[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    gi[e] = a.gb == 1 ? 0 : (w.col * V + e) / a.cpg;
    gm[e] = gs[gi[e]] * inv;
    t[e] = fmaf(n * (mean[e] - gm[e]), mean[e] - gm[e], sq[e]);
  }
  for (int i = threadIdx.x; i < a.gb; i += TH) {    // (count, mean, squares) of the part
    float *o = a.ws + (((int64_t)blockIdx.z * a.groups + w.g0 + i) * a.parts + blockIdx.x) * 4;
    o[0] = cnt;
    o[1] = gs[i] * inv;
  }
  group_sums<V, TH>(a, t, w, part, gs);
  for (int i = threadIdx.x; i < a.gb; i += TH)
    a.ws[(((int64_t)blockIdx.z * a.groups + w.g0 + i) * a.parts + blockIdx.x) * 4 + 2] = gs[i];
}

// The second launch: joins the parts of its groups (counts n_i, means m_i, squares S_i:
// mean = sum n_i m_i / N, squares = sum S_i + n_i (m_i - mean)^2), then normalises its pixels.
// Grid: x = chunk of `apply` pixels x column part, y = bundle, z = image. PAST: y is more than the
// 32 MB of L2 and is stored past it (8 x 128 x 128 x 320: 54.4 us against 57.7).
template <typename T, int V, int TH, bool PAST>
__global__ __launch_bounds__(TH) void k_gn_apply(GnArgs a) {
  typedef Vec<T, V> vec;
  extern __shared__ float lds[];                    // [gb][2]
  const int tid = threadIdx.x;
  const int chunk = (int)blockIdx.x / a.colparts;
  const Place w = place_of<V, TH>(a, (int)blockIdx.x - chunk * a.colparts);
  const int px0 = chunk * a.apply, npx = w.on ? min(a.apply, a.pixels - px0) : 0;
  const T *x = (const T *)a.x + (int64_t)blockIdx.z * a.x_image + (int64_t)px0 * a.x_row + w.ch;
  T *y = (T *)a.y + (int64_t)blockIdx.z * a.y_image + (int64_t)px0 * a.y_row + w.ch;
  typename vec::raw r[kBatch], rn[kBatch];
  auto load = [&](int p, typename vec::raw (&to)[kBatch]) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (p + i * a.ppi < npx) to[i] = vec::load(x + (int64_t)(p + i * a.ppi) * a.x_row);
  };
  load(w.p0, r);
  load(w.p0 + kBatch * a.ppi, rn);
  float gam[V], bet[V];
  affine<T, V>(a, w.ch, gam, bet);
  // teams of lanes over the parts of a group, all groups at once; a lane's first PRE parts are in
  // flight together
  constexpr int PRE = 8;
  const int lanes = min(team_of<TH>(a.gb), 64), j0 = tid & (lanes - 1);
  const float inv = 1.f / ((float)a.pixels * (float)a.cpg);
  for (int i0 = 0; i0 < a.gb; i0 += TH / lanes) {
    const int i = i0 + tid / lanes;
    const f32x4 *ws = (const f32x4 *)a.ws + ((int64_t)blockIdx.z * a.groups + w.g0 + min(i, a.gb - 1)) * a.parts;
    f32x4 m[PRE];
#pragma unroll
    for (int k = 0; k < PRE; ++k) m[k] = j0 + k * lanes < a.parts ? ws[j0 + k * lanes] : f32x4{0.f, 0.f, 0.f, 0.f};
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < PRE; ++k) s = fmaf(m[k][0], m[k][1], s);
    for (int j = j0 + PRE * lanes; j < a.parts; j += lanes) s = fmaf(ws[j][0], ws[j][1], s);
    const float mean = team_sum(s, lanes) * inv;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < PRE; ++k) s += fmaf(m[k][0] * (m[k][1] - mean), m[k][1] - mean, m[k][2]);
    for (int j = j0 + PRE * lanes; j < a.parts; j += lanes)
      s += fmaf(ws[j][0] * (ws[j][1] - mean), ws[j][1] - mean, ws[j][2]);
    s = team_sum(s, lanes);
    if (j0 == 0 && i < a.gb) {
      lds[2 * i] = mean;
      lds[2 * i + 1] = 1.f / sqrtf(s * inv + a.eps);
    }
  }
  __syncthreads();
  float mean[V], rstd[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int gi = a.gb == 1 ? 0 : (w.col * V + e) / a.cpg;
    mean[e] = lds[2 * gi];
    rstd[e] = lds[2 * gi + 1];
  }
  for (int p = w.p0; p < npx; p += kBatch * a.ppi) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (p + i * a.ppi < npx) {
        float f[V], o[V];
        vec::unpack(r[i], f);
        normalise<V>(a, f, mean, rstd, gam, bet, o);
        typename vec::raw *to = (typename vec::raw *)(y + (int64_t)(p + i * a.ppi) * a.y_row);
        if constexpr (PAST) __builtin_nontemporal_store(vec::pack(o), to);
        else *to = vec::pack(o);
      }
      r[i] = rn[i];
    }
    load(p + 2 * kBatch * a.ppi, rn);
  }
}

// Two launches: workgroups that keep the chip busy, most parts of an image (every workgroup of the
// second launch reads those of its groups), batches of its pixels a thread of the second launch
// takes. One launch: the largest slab, and what a workgroup can have in all.
constexpr int kFill = 512, kParts = 64, kTurns = 4, kSlab = 128 * 1024, kLds = 160 * 1024;

struct GnPlan {
  int V, TH, gb, ncol, ppi, chunk, apply, colparts, parts;
  bool one;
};

// Widest vector of at most 16 bytes that divides a bundle of n channels and `align` elements.
int vec_of(int n, int align, int esize) {
  int v = 16 / esize;
  while (v > 1 && (n % v || align % v)) v >>= 1;
  return v;
}

// LDS of group_sums: an entry per pixel lane and column, or channel where a column spans groups.
int sums_bytes(int gb, int cpg, int v, int ncol, int ppi) {
  const int entries = (gb == 1 || cpg % v == 0 ? 1 : v) * ncol * (ppi | 1);
  return ((gb + std::max(entries, 16)) * 4 + 15) & ~15;
}

// `align`: the elements that every address and stride is a multiple of.
GnPlan plan_of(int n, int pixels, int channels, int groups, int esize, int align) {
  const int cpg = channels / groups;
  GnPlan p;
  // One launch, if an image of a bundle fits: the fewest groups whose channels are a run of 64 bytes
  // (32 where that leaves fewer than 64 workgroups), and at least 32 workgroups or next to no
  // work. us in one / two launches: 1 x 16 x 16 x 1280 9.2 / 12.2, 1 x 32 x 32 x 640 11.4 / 13.2,
  // 16 x 16 x 16 x 1280 15.0 / 17.8, 16 x 32 x 32 x 640 25.0 / 26.0; 2 x 33 x 31 x 96 (16
  // workgroups) 14.4 / 12.5.
  for (int run = 64; run >= 32; run -= 32) {
    for (int gb = 1; gb <= groups; ++gb) {
      if (groups % gb) continue;
      const int w = gb * cpg, v = vec_of(w, align, esize), ncol = w / v;
      if (w * esize < run && gb < groups) continue;
      const int th = (int64_t)ncol * pixels <= 2048 && ncol <= 256 ? 256 : 1024;
      if (ncol > th) break;
      const int ppi = std::min(th / ncol, pixels);
      const int64_t bytes = ((int64_t)pixels + ppi - 1) / ppi * th * v * esize, wgs = (int64_t)n * (groups / gb);
      if (bytes > kSlab || bytes + sums_bytes(gb, cpg, v, ncol, ppi) > kLds || (wgs < (run == 64 ? 64 : 32) && bytes > 16384)) break;
      return GnPlan{v, th, gb, ncol, ppi, pixels, pixels, 1, 1, true};
    }
  }
  // two launches: as many groups as a workgroup of 256 has columns for
  p.one = false;
  p.TH = 256;
  p.gb = 1;
  for (int gb = 1; gb <= groups; ++gb) {
    if (groups % gb) continue;
    const int w = gb * cpg;
    if (w / vec_of(w, align, esize) > p.TH) continue;
    // wider while that leaves kFill workgroups, or rows shorter than two lines
    if (gb == 1 || p.gb * cpg * esize < 256 || (int64_t)n * (groups / gb) * kParts >= kFill) p.gb = gb;
  }
  p.V = vec_of(p.gb * cpg, align, esize);
  p.ncol = p.gb * cpg / p.V;
  p.colparts = (p.ncol + p.TH - 1) / p.TH;
  p.ppi = p.colparts > 1 ? 1 : std::min(p.TH / p.ncol, pixels);
  // parts of an image: kFill workgroups in all, but at most kParts parts (each workgroup of the
  // second launch reads them all) of at least one batch
  const int64_t bundles = (int64_t)n * (groups / p.gb) * p.colparts;
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(kParts / p.colparts, kFill / bundles));
  const int step = p.ppi * 2 * kBatch;
  p.chunk = (int)std::min<int64_t>(pixels, std::max<int64_t>(1, ((int64_t)pixels + want * step - 1) / (want * step)) * step);
  p.parts = (int)(((int64_t)pixels + p.chunk - 1) / p.chunk) * p.colparts;
  const int64_t turns = std::max<int64_t>(1, std::min<int64_t>(kTurns, (int64_t)pixels * bundles / ((int64_t)p.ppi * kBatch * kFill)));
  p.apply = (int)std::min<int64_t>(pixels, p.ppi * kBatch * turns);
  return p;
}

template <typename K> hipError_t allow_lds(K kern, int bytes) {
  return bytes <= 65536 ? hipSuccess
                        : hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <typename T, int V>
hipError_t run(const GnArgs &a, const GnPlan &p, int esize, hipStream_t s) {
  const int sums = sums_bytes(p.gb, a.cpg, V, std::min(p.ncol, p.TH), p.ppi), bundles = a.groups / p.gb;
  hipError_t e;
  if (p.one) {
    auto kern = p.TH == 256 ? k_gn<T, V, 256> : k_gn<T, V, 1024>;
    const int lds = sums + (a.pixels + p.ppi - 1) / p.ppi * p.TH * V * esize;
    if ((e = allow_lds(kern, lds)) != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3(1, bundles, a.n), dim3(p.TH), lds, s, a, sums);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((k_gn_stats<T, V, 256>), dim3(p.parts, bundles, a.n), dim3(256), sums, s, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const int chunks = (int)(((int64_t)a.pixels + p.apply - 1) / p.apply);
  const bool past = (int64_t)a.n * a.pixels * a.channels * esize > (32 << 20);
  auto apply = past ? k_gn_apply<T, V, 256, true> : k_gn_apply<T, V, 256, false>;
  hipLaunchKernelGGL(apply, dim3(chunks * p.colparts, bundles, a.n), dim3(256), p.gb * 8, s, a);
  return hipGetLastError();
}

}  // namespace

// The largest workspace that any alignment of the buffers leads to.
int64_t group_norm_workspace(int n, int pixels, int channels, int groups, int dtype) {
  const int es = dtype == MTE_BF16 ? 2 : 4;
  int64_t most = 0;
  for (int align = 1; align <= 8; align *= 2) {
    const GnPlan p = plan_of(n, pixels, channels, groups, es, align);
    if (!p.one) most = std::max(most, (int64_t)n * groups * p.parts * 16);
  }
  return most;
}

hipError_t launch_group_norm(const GroupNormArgs &g, int dtype, hipStream_t s) {
  const int es = dtype == MTE_BF16 ? 2 : 4;
  uint64_t bits = (uint64_t)(uintptr_t)g.x / es | (uint64_t)(uintptr_t)g.y / es | (uint64_t)g.x_row | (uint64_t)g.y_row |
                  (uint64_t)g.x_image | (uint64_t)g.y_image | 8;
  const int align = (int)(bits & (~bits + 1));      // lowest set bit
  const GnPlan p = plan_of(g.n, g.pixels, g.channels, g.groups, es, align);
  GnArgs a;
  (GroupNormArgs &)a = g;
  a.cpg = g.channels / g.groups;
  a.gb = p.gb;
  a.ncol = p.ncol;
  a.ppi = p.ppi;
  a.chunk = p.chunk;
  a.apply = p.apply;
  a.parts = p.parts;
  a.colparts = p.colparts;
  a.same = p.gb == 1 || a.cpg % p.V == 0;
  if (dtype == MTE_BF16) {
    if (p.V == 8) return run<bf16, 8>(a, p, es, s);
    if (p.V == 4) return run<bf16, 4>(a, p, es, s);
    if (p.V == 2) return run<bf16, 2>(a, p, es, s);
    return run<bf16, 1>(a, p, es, s);
  }
  if (p.V == 4) return run<float, 4>(a, p, es, s);
  if (p.V == 2) return run<float, 2>(a, p, es, s);
  return run<float, 1>(a, p, es, s);
}

}  // namespace mte
