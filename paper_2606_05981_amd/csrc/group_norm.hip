// Group norm with an activation, channels last:
//   y = act((x - mean) / sqrt(var + eps) * gamma[c] + beta[c])
// over the pixels and the cpg = C / G channels of a group of one image.
//
// A workgroup holds a slab of an image in registers -- a bundle of whole groups
// (neighbouring channels, so that rows are read in runs) times a chunk of pixels; a
// thread keeps one column of V channels and walks the pixels. Sums go through LDS
// per group, twice: the mean first, then the squares around it, so that a large mean
// cancels nowhere. Where the slab is a whole image the same workgroup
// normalises it from its registers: x is read once, y written once, one launch. Else
// the chunks leave (mean, squares) in the workspace and a second launch joins them by
// their counts and normalises. Bound by those bytes.
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

// Vectors a thread holds: 64 registers of 16-byte or 8-byte ones, 32 of shorter ones.
constexpr int hold_of(int bytes) { return bytes == 16 ? 16 : 32; }

struct GnArgs : GroupNormArgs {
  int cpg, gb;         // channels per group, groups per bundle
  int ncol;            // columns (of V channels) of a bundle
  int ppi;             // pixels a workgroup takes at a time
  int chunk;           // pixels per chunk
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

// Sums `v` (per thread and channel of its column) over each group of the bundle: the sum of
// group i is gs[i * wpg] + .. + gs[i * wpg + wpg - 1] afterwards.
template <int V, int TH>
__device__ __forceinline__ void group_sums(const GnArgs &a, float (&v)[V], bool on, int col, int p0, int ncol, int ng,
                                           int wpg, float *part, float *gs) {
  constexpr int NW = TH / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int pitch = a.ppi | 1;                      // odd: columns in different banks
  int per;                                          // entries of a group, in a run
  __syncthreads();                                  // part and gs are free
  if (a.same) {
    per = (ng == 1 ? ncol : a.cpg / V) * pitch;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) s += v[e];
    if (on) part[col * pitch + p0] = s;
    if (on && p0 == 0 && pitch > a.ppi) part[col * pitch + a.ppi] = 0.f;
  } else {
    per = a.cpg * pitch;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if (on) part[(col * V + e) * pitch + p0] = v[e];
      if (on && p0 == 0 && pitch > a.ppi) part[(col * V + e) * pitch + a.ppi] = 0.f;
    }
  }
  __syncthreads();
  for (int i = wave / wpg; i < ng; i += NW / wpg) { // wave-uniform
    float s = 0.f;
    for (int j = (wave % wpg) * 64 + lane; j < per; j += wpg * 64) s += part[i * per + j];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s = warp_sum_xor(s, m);
    if (lane == 0) gs[i * wpg + wave % wpg] = s;
  }
  __syncthreads();
}

template <typename T, int V>
__device__ __forceinline__ void normalise(const GnArgs &a, const float *x, const float *mean, const float *rstd,
                                          const float *gam, const float *bet, float *y) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float z = fmaf((x[e] - mean[e]) * rstd[e], gam[e], bet[e]);
    y[e] = a.act == MTE_ACT_SILU
               ? z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z))
               : z;
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

// Grid: x = part (chunk x column part), y = bundle, z = image. FUSED: one part, y written here; else
// (mean, squares) of the part to ws[image][group][part].
template <typename T, int V, int TH, bool FUSED>
__global__ __launch_bounds__(TH) void k_gn(GnArgs a) {
  typedef Vec<T, V> vec;
  constexpr int HOLD = hold_of(V * sizeof(T));
  extern __shared__ float lds[];
  const int tid = threadIdx.x;
  const int cp = (int)blockIdx.x % a.colparts, chunk = (int)blockIdx.x / a.colparts;
  const int col0 = cp * TH, ncol = min(a.ncol - col0, TH);
  const int g0 = blockIdx.y * a.gb, ng = a.gb;
  const int px0 = chunk * a.chunk, npx = min(a.chunk, a.pixels - px0);
  const int col = tid % ncol, p0 = tid / ncol;
  const bool on = p0 < a.ppi;
  const int ch = g0 * a.cpg + (col0 + col) * V;     // first channel of the column
  const T *x = (const T *)a.x + (int64_t)blockIdx.z * a.x_image + (int64_t)px0 * a.x_row + ch;
  constexpr int NW = TH / 64;
  const int wpg = max(1, NW / ng);
  float *gs = lds, *part = lds + max(NW, ng) ;
  typename vec::raw r[HOLD];
  float sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) sum[e] = 0.f;
#pragma unroll
  for (int i = 0; i < HOLD; ++i) {
    const int p = p0 + i * a.ppi;
    if (on && p < npx) r[i] = vec::load(x + (int64_t)p * a.x_row);
  }
#pragma unroll
  for (int i = 0; i < HOLD; ++i) {
    if (on && p0 + i * a.ppi < npx) {
      float f[V];
      vec::unpack(r[i], f);
#pragma unroll
      for (int e = 0; e < V; ++e) sum[e] += f[e];
    }
  }
  group_sums<V, TH>(a, sum, on, col, p0, ncol, ng, wpg, part, gs);
  const float cnt = (float)npx * (float)(ng == 1 ? ncol * V : a.cpg);
  float mean[V], sq[V];
  int gi[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    gi[e] = ng == 1 ? 0 : ((col0 + col) * V + e) / a.cpg;
    float s = 0.f;
    for (int w = 0; w < wpg; ++w) s += gs[gi[e] * wpg + w];
    mean[e] = s / cnt;
    sq[e] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < HOLD; ++i) {
    if (on && p0 + i * a.ppi < npx) {
      float f[V];
      vec::unpack(r[i], f);
#pragma unroll
      for (int e = 0; e < V; ++e) sq[e] = fmaf(f[e] - mean[e], f[e] - mean[e], sq[e]);
    }
  }
  group_sums<V, TH>(a, sq, on, col, p0, ncol, ng, wpg, part, gs);
  if constexpr (FUSED) {
    float rstd[V], gam[V], bet[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float s = 0.f;
      for (int w = 0; w < wpg; ++w) s += gs[gi[e] * wpg + w];
      rstd[e] = 1.f / sqrtf(s / cnt + a.eps);
    }
    affine<T, V>(a, ch, gam, bet);
    T *y = (T *)a.y + (int64_t)blockIdx.z * a.y_image + (int64_t)px0 * a.y_row + ch;
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
      const int p = p0 + i * a.ppi;
      if (on && p < npx) {
        float f[V], o[V];
        vec::unpack(r[i], f);
        normalise<T, V>(a, f, mean, rstd, gam, bet, o);
        *(typename vec::raw *)(y + (int64_t)p * a.y_row) = vec::pack(o);
      }
    }
  } else {
    // a thread that has an element of the group writes it: the first of its channels
    const int parts = gridDim.x;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int c = (col0 + col) * V + e;
      if (on && p0 == 0 && (ng == 1 ? col == 0 && e == 0 : c % a.cpg == 0)) {
        float s = 0.f;
        for (int w = 0; w < wpg; ++w) s += gs[gi[e] * wpg + w];
        float *o = a.ws + (((int64_t)blockIdx.z * a.groups + g0 + gi[e]) * parts + blockIdx.x) * 2;
        o[0] = mean[e];
        o[1] = s;
      }
    }
  }
}

// The second launch: joins the parts of its groups (counts n_i, means m_i, squares S_i:
// mean = sum n_i m_i / N, squares = sum S_i + n_i (m_i - mean)^2), then normalises its slab.
template <typename T, int V, int TH>
__global__ __launch_bounds__(TH) void k_gn_apply(GnArgs a) {
  typedef Vec<T, V> vec;
  constexpr int HOLD = hold_of(V * sizeof(T));
  extern __shared__ float lds[];                    // [gb][2]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int parts = gridDim.x;
  const int cp = (int)blockIdx.x % a.colparts, chunk = (int)blockIdx.x / a.colparts;
  const int col0 = cp * TH, ncol = min(a.ncol - col0, TH);
  const int g0 = blockIdx.y * a.gb, ng = a.gb;
  const int px0 = chunk * a.chunk, npx = min(a.chunk, a.pixels - px0);
  const int col = tid % ncol, p0 = tid / ncol;
  const bool on = p0 < a.ppi;
  const int ch = g0 * a.cpg + (col0 + col) * V;
  const T *x = (const T *)a.x + (int64_t)blockIdx.z * a.x_image + (int64_t)px0 * a.x_row + ch;
  typename vec::raw r[HOLD];
#pragma unroll
  for (int i = 0; i < HOLD; ++i) {
    const int p = p0 + i * a.ppi;
    if (on && p < npx) r[i] = vec::load(x + (int64_t)p * a.x_row);
  }
  for (int i = wave; i < ng; i += TH / 64) {        // wave-uniform
    const float *w = a.ws + ((int64_t)blockIdx.z * a.groups + g0 + i) * parts * 2;
    auto count = [&](int j) {
      const int n = min(a.chunk, a.pixels - j / a.colparts * a.chunk);
      return (float)n * (float)(a.colparts > 1 ? min(a.ncol - j % a.colparts * TH, TH) * V : a.cpg);
    };
    float s = 0.f;
    for (int j = lane; j < parts; j += 64) s += count(j) * w[2 * j];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s = warp_sum_xor(s, m);
    const float total = (float)a.pixels * (float)a.cpg, mean = s / total;
    float q = 0.f;
    for (int j = lane; j < parts; j += 64) q += w[2 * j + 1] + count(j) * (w[2 * j] - mean) * (w[2 * j] - mean);
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) q = warp_sum_xor(q, m);
    if (lane == 0) {
      lds[2 * i] = mean;
      lds[2 * i + 1] = 1.f / sqrtf(q / total + a.eps);
    }
  }
  __syncthreads();
  float mean[V], rstd[V], gam[V], bet[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int gi = ng == 1 ? 0 : ((col0 + col) * V + e) / a.cpg;
    mean[e] = lds[2 * gi];
    rstd[e] = lds[2 * gi + 1];
  }
  affine<T, V>(a, ch, gam, bet);
  T *y = (T *)a.y + (int64_t)blockIdx.z * a.y_image + (int64_t)px0 * a.y_row + ch;
#pragma unroll
  for (int i = 0; i < HOLD; ++i) {
    const int p = p0 + i * a.ppi;
    if (on && p < npx) {
      float f[V], o[V];
      vec::unpack(r[i], f);
      normalise<T, V>(a, f, mean, rstd, gam, bet, o);
      *(typename vec::raw *)(y + (int64_t)p * a.y_row) = vec::pack(o);
    }
  }
}

struct GnPlan {
  int V, TH, gb, ncol, ppi, chunk, colparts, parts;
  bool fused;
};

// Widest vector of at most 16 bytes that divides a bundle of n channels and `align` elements.
int vec_of(int n, int align, int esize) {
  int v = 16 / esize;
  while (v > 1 && (n % v || align % v)) v >>= 1;
  return v;
}

// `align`: the elements that every address and stride is a multiple of.
GnPlan plan_of(int n, int pixels, int channels, int groups, int esize, int align) {
  const int cpg = channels / groups;
  GnPlan p;
  // one launch: the fewest groups whose channels are a run of 64 bytes, if an image of them fits
  for (int gb = 1; gb <= groups; ++gb) {
    if (groups % gb) continue;
    const int w = gb * cpg, v = vec_of(w, align, esize), ncol = w / v;
    if (w * esize < 64 && gb < groups) continue;
    for (int th : {256, 1024}) {
      if (ncol > th) continue;
      const int ppi = std::min(th / ncol, pixels);
      if ((int64_t)ppi * hold_of(v * esize) < pixels) continue;
      p = GnPlan{v, th, gb, ncol, ppi, pixels, 1, 1, true};
      return p;
    }
    break;
  }
  // two launches: as many groups as a workgroup of 256 has columns for
  p.fused = false;
  p.TH = 256;
  p.gb = 1;
  for (int gb = 1; gb <= groups; ++gb) {
    if (groups % gb) continue;
    const int w = gb * cpg;
    if (w / vec_of(w, align, esize) <= p.TH) p.gb = gb;
  }
  p.V = vec_of(p.gb * cpg, align, esize);
  p.ncol = p.gb * cpg / p.V;
  p.colparts = (p.ncol + p.TH - 1) / p.TH;
  p.ppi = p.colparts > 1 ? 1 : std::min(p.TH / p.ncol, pixels);
  p.chunk = std::min(p.ppi * hold_of(p.V * esize), pixels);
  p.parts = (int)(((int64_t)pixels + p.chunk - 1) / p.chunk) * p.colparts;
  return p;
}

template <typename T, int V, int TH>
hipError_t run(const GnArgs &a, const GnPlan &p, hipStream_t s) {
  const dim3 grid(p.parts, a.groups / p.gb, a.n);
  const int entries = (a.same ? 1 : V) * std::min(p.ncol, TH) * (p.ppi | 1);
  const int lds = (std::max(TH / 64, p.gb) + entries) * 4;
  hipError_t e;
  auto one = k_gn<T, V, TH, true>;
  auto two = k_gn<T, V, TH, false>;
  if (lds > 65536 && (e = hipFuncSetAttribute((const void *)(p.fused ? one : two),
                                              hipFuncAttributeMaxDynamicSharedMemorySize, lds)) != hipSuccess)
    return e;
  if (p.fused) {
    hipLaunchKernelGGL(one, grid, dim3(TH), lds, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(two, grid, dim3(TH), lds, s, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL((k_gn_apply<T, V, TH>), grid, dim3(TH), p.gb * 8, s, a);
  return hipGetLastError();
}

template <typename T, int V>
hipError_t run_th(const GnArgs &a, const GnPlan &p, hipStream_t s) {
  return p.TH == 1024 ? run<T, V, 1024>(a, p, s) : run<T, V, 256>(a, p, s);
}

}  // namespace

// The largest workspace that any alignment of the buffers leads to.
int64_t group_norm_workspace(int n, int pixels, int channels, int groups, int dtype) {
  const int es = dtype == MTE_BF16 ? 2 : 4;
  int64_t most = 0;
  for (int align = 1; align <= 8; align *= 2) {
    const GnPlan p = plan_of(n, pixels, channels, groups, es, align);
    if (!p.fused) most = std::max(most, (int64_t)n * groups * p.parts * 8);
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
  a.colparts = p.colparts;
  a.same = p.gb == 1 || a.cpg % p.V == 0;
  if (dtype == MTE_BF16) {
    if (p.V == 8) return run_th<bf16, 8>(a, p, s);
    if (p.V == 4) return run_th<bf16, 4>(a, p, s);
    if (p.V == 2) return run_th<bf16, 2>(a, p, s);
    return run_th<bf16, 1>(a, p, s);
  }
  if (p.V == 4) return run_th<float, 4>(a, p, s);
  if (p.V == 2) return run_th<float, 2>(a, p, s);
  return run_th<float, 1>(a, p, s);
}

}  // namespace mte
