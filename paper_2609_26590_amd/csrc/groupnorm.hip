// Group norm with an activation over token grids, channels last, and its gradients. Per
// image and group of channels, over all tokens and the group's channels, in float32:
//
//   forward:  mean, rstd = (var + eps)^(-1/2),  xh = (x - mean) rstd,
//             y = act(xh w + b)
//   backward: du = dy act'(xh w + b),  t = du w,
//             dx = rstd (t - mean(t) - xh mean(t xh)) (+ dres)
//             dw = sum over images and tokens of du xh,  db = that of du
//
// What bounds both is memory: each value read once and written once, where an image's
// block of groups fits the registers of one work-group (gn_*_slab_kernel), else read
// twice by two launches (gn_*_sums_kernel, gn_*_rows_kernel).
#include <hip/hip_runtime.h>

#include "ffn_gemm.h"
#include "gtr.h"
#include "gtr_device.h"
#include "gtr_internal.h"
#include "vec_rows.h"

namespace gtr {

// The channels in blocks: kg whole groups each, or where a group is wider than a block
// allows, `pieces` of pw channels (the last may be narrower). The tokens in tiles of R.
struct GnShape {
  int64_t L;
  int B, C, G, Cg;
  int kg, pieces, pw, blocks;
  int tiles, R;
  int team;  // threads that add a group's channels: a power of two, kg teams at most the work-group's threads
};
struct GnBlock {
  int g0, ng, c0, cb, piece;
  __device__ __forceinline__ GnBlock(const GnShape& s, int block) {
    if (s.pieces == 1) {
      g0 = block * s.kg;
      ng = min(s.kg, s.G - g0);
      piece = 0;
      c0 = g0 * s.Cg;
      cb = ng * s.Cg;
    } else {
      g0 = block / s.pieces;
      ng = 1;
      piece = block - g0 * s.pieces;
      c0 = g0 * s.Cg + piece * s.pw;
      cb = min(s.pw, s.Cg - piece * s.pw);
    }
  }
};

// Which tile of which block of which image a work-group takes: the blocks of a tile's rows
// next to each other, image after image; `back`: the last one first (what the launch before
// read last is what the cache still has).
struct GnAt {
  int image, tile, block;
  __device__ __forceinline__ GnAt(const GnShape& s, unsigned id, bool back) {
    if (back) id = (unsigned)s.B * s.tiles * s.blocks - 1 - id;
    const unsigned t = id / (unsigned)s.blocks;
    block = (int)(id - t * (unsigned)s.blocks);
    image = (int)(t / (unsigned)s.tiles);
    tile = (int)(t - (unsigned)image * (unsigned)s.tiles);
  }
};

__device__ __forceinline__ float gn_act(float u, int act) {
  if (act == GTR_ACT_NONE) return u;
  float slope;
  return ffn_act(u, act, slope);
}
__device__ __forceinline__ float gn_slope(float u, int act) {
  if (act == GTR_ACT_NONE) return 1.f;
  float slope;
  ffn_act(u, act, slope);
  return slope;
}

// A work-group's threads on a block: nl lanes hold a row's vectors, rp rows at a time.
// Threads past rp nl are off.
template <int DT, bool TINY>
struct GnLane {
  static constexpr int VE = Ln<DT>::VE;
  int nl, rp, r;
  bool on;
  LnCols<DT, TINY> k;
  __device__ __forceinline__ GnLane(int cb)
      : nl((cb + VE - 1) / VE),
        rp((int)blockDim.x / nl),
        r((int)threadIdx.x / nl),
        on(r < rp),
        k((int)threadIdx.x - r * nl, cb) {}
  // the groups (of the block's) of this lane's channels
  __device__ __forceinline__ void groups(int Cg, int (&g)[VE]) const {
    const int q = k.c / Cg;
    int rem = k.c - q * Cg, i = q;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      g[e] = i;
      if (++rem == Cg) {
        rem = 0;
        ++i;
      }
    }
  }
};

// Sums over a work-group, all in a fixed order. `v`: a value per channel of this thread's,
// zeros in threads that are off; cols: at least blockDim VE floats. What is returned lies in
// cols[0 .. cb): the columns' sums. (Starts and ends with a barrier.)
template <int DT, bool TINY>
__device__ __forceinline__ void gn_columns(const GnLane<DT, TINY>& ln, int cb, const float (&v)[Ln<DT>::VE], float* cols) {
  constexpr int VE = Ln<DT>::VE;
  const int n = blockDim.x, t = threadIdx.x;
  __syncthreads();
  if (ln.on)
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (ln.k.has(e)) cols[ln.r * cb + ln.k.c + e] = v[e];
  __syncthreads();
  if (cb >= n) {
    for (int c = t; c < cb; c += n) {
      float a = 0.f;
      for (int r = 0; r < ln.rp; ++r) a += cols[r * cb + c];
      cols[c] = a;  // (only this thread reads column c)
    }
  } else {
    // slices of the rows, then the slices: each thread adds about VE values
    const int slices = n / cb, s = t / cb, c = t - s * cb;
    float a = 0.f;
    if (s < slices)
      for (int r = s; r < ln.rp; r += slices) a += cols[r * cb + c];
    __syncthreads();
    if (s < slices) cols[s * cb + c] = a;
    __syncthreads();
    if (t < cb) {
      a = cols[t];
      for (int i = 1; i < slices; ++i) a += cols[i * cb + t];
      cols[t] = a;
    }
  }
  __syncthreads();
}
// The groups' sums of cols[0 .. cb) into sums[0 .. ng) (ends with a barrier).
__device__ __forceinline__ void gn_teams(const GnShape& s, const GnBlock& b, const float* cols, float* sums) {
  const int g = threadIdx.x / s.team, i = threadIdx.x - g * s.team;
  const int width = s.pieces == 1 ? s.Cg : b.cb;
  float a = 0.f;
  if (g < b.ng)
    for (int c = i; c < width; c += s.team) a += cols[g * width + c];
  for (int o = 1; o < s.team; o <<= 1) a += __shfl_xor(a, o, kWave);
  if (g < b.ng && i == 0) sums[g] = a;
  __syncthreads();
}

// Mean and sum of squares about it of n values, joined with another's.
struct GnStat {
  float n, mean, m2;
  __device__ __forceinline__ void join(float n2, float mean2, float m22) {
    const float all = n + n2, d = mean2 - mean, f = all > 0.f ? n2 / all : 0.f;
    mean = fmaf(d, f, mean);
    m2 += fmaf(d * d, n * f, m22);
    n = all;
  }
};

// Vectors that are unpacked again from here on: without it the compiler keeps their
// elements, in twice the registers or more.
template <int N>
__device__ __forceinline__ void gn_packed(Vec16 (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) asm volatile("" : "+v"(v[i].u[e]));
}

struct GnFwd {
  GnShape s;
  const char* x;
  const float *w, *b;
  char* y;
  float *mean, *rstd;
  float2* part;  // [B][tiles][pieces][G]: mean and sum of squares
  float eps;
  int act;
};

constexpr int kGnThreads = 256, kGnSlab = 1024;

// Each tile's statistics. A lane takes its channels' sums about the first value it sees of
// each (n values about one of them: their sum of squares loses at most n 2^-24 of itself),
// the work-group the groups' means and then the sums of squares about those.
template <int DT, bool TINY>
__global__ void __launch_bounds__(kGnThreads) gn_fwd_sums_kernel(GnFwd p) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, U = 4;
  __shared__ float cols[kGnThreads * VE], sums[kGnThreads];
  const GnAt wg(p.s, blockIdx.x, false);
  const GnBlock blk(p.s, wg.block);
  const GnLane<DT, TINY> ln(blk.cb);
  const int64_t first = (int64_t)wg.tile * p.s.R, end = min(first + p.s.R, p.s.L), ld = (int64_t)p.s.C * ES;
  const int rows = (int)(end - first);
  const char* x = p.x + ((int64_t)wg.image * p.s.L + first) * ld + (int64_t)blk.c0 * ES;
  float pivot[VE], s1[VE], s2[VE];
  int n = 0;
#pragma unroll
  for (int e = 0; e < VE; ++e) pivot[e] = s1[e] = s2[e] = 0.f;
  if (ln.on && ln.r < rows) {
    n = (rows - ln.r + ln.rp - 1) / ln.rp;
    for (int i = 0; i < n; i += U) {
      Vec16 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = ln.k.load(x + (int64_t)(ln.r + min(i + u, n - 1) * ln.rp) * ld);
      if (i == 0) ln.k.unpack(v[0], pivot);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u >= n) break;
        float a[VE];
        ln.k.unpack(v[u], a);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          a[e] -= pivot[e];
          s1[e] += a[e];
          s2[e] = fmaf(a[e], a[e], s2[e]);
        }
      }
    }
  }
  const float cnt = (float)n, inv = n ? 1.f / cnt : 0.f, all = (float)rows * (float)(p.s.pieces == 1 ? p.s.Cg : blk.cb);
  float v[VE], mean[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    mean[e] = fmaf(s1[e], inv, pivot[e]);
    s2[e] = fmaxf(fmaf(-s1[e] * inv, s1[e], s2[e]), 0.f);
    v[e] = fmaf(cnt, pivot[e], s1[e]);
  }
  gn_columns(ln, blk.cb, v, cols);
  gn_teams(p.s, blk, cols, sums);
  int gi[VE];
  ln.groups(p.s.pieces == 1 ? p.s.Cg : blk.cb, gi);
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    const float d = mean[e] - sums[min(gi[e], blk.ng - 1)] / all;
    v[e] = fmaf(cnt * d, d, s2[e]);
  }
  float m = 0.f;
  if ((int)threadIdx.x < blk.ng) m = sums[threadIdx.x] / all;
  gn_columns(ln, blk.cb, v, cols);
  gn_teams(p.s, blk, cols, sums);
  if ((int)threadIdx.x < blk.ng)
    p.part[(((int64_t)wg.image * p.s.tiles + wg.tile) * p.s.pieces + blk.piece) * p.s.G + blk.g0 + threadIdx.x] =
        float2{m, sums[threadIdx.x]};
}

// The groups' statistics of an image from its tiles', and a tile's rows.
template <int DT, bool TINY>
__global__ void __launch_bounds__(kGnThreads) gn_fwd_rows_kernel(GnFwd p) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, U = 4;
  __shared__ float smean[kGnThreads], srstd[kGnThreads];
  const GnShape& s = p.s;
  const GnAt wg(s, blockIdx.x, true);
  const GnBlock blk(s, wg.block);
  const GnLane<DT, TINY> ln(blk.cb);
  {
    const int g = threadIdx.x / s.team, i = threadIdx.x - g * s.team, entries = s.tiles * s.pieces;
    GnStat st = {0.f, 0.f, 0.f};
    if (g < blk.ng) {
      const float2* q = p.part + (int64_t)wg.image * entries * s.G + blk.g0 + g;
#pragma unroll 4
      for (int j = i; j < entries; j += s.team) {
        const float2 v = q[(int64_t)j * s.G];
        const int tile = s.pieces == 1 ? j : j / s.pieces, piece = s.pieces == 1 ? 0 : j - tile * s.pieces;
        const int rows = (int)min((int64_t)s.R, s.L - (int64_t)tile * s.R);
        const int width = s.pieces == 1 ? s.Cg : min(s.pw, s.Cg - piece * s.pw);
        st.join((float)rows * (float)width, v.x, v.y);
      }
    }
    for (int o = 1; o < s.team; o <<= 1) {
      // (both partners join in the same order, the lower one's first)
      const float n = __shfl_xor(st.n, o, kWave), m = __shfl_xor(st.mean, o, kWave), q = __shfl_xor(st.m2, o, kWave);
      const bool low = (threadIdx.x & o) == 0;
      GnStat a = {low ? st.n : n, low ? st.mean : m, low ? st.m2 : q};
      a.join(low ? n : st.n, low ? m : st.mean, low ? q : st.m2);
      st = a;
    }
    if (g < blk.ng && i == 0) {
      const float rs = 1.f / sqrtf(st.m2 / st.n + p.eps);
      smean[g] = st.mean;
      srstd[g] = rs;
      if (wg.tile == 0 && blk.piece == 0) {
        if (p.mean) p.mean[(int64_t)wg.image * s.G + blk.g0 + g] = st.mean;
        if (p.rstd) p.rstd[(int64_t)wg.image * s.G + blk.g0 + g] = rs;
      }
    }
    __syncthreads();
  }
  const int64_t first = (int64_t)wg.tile * s.R, end = min(first + s.R, s.L), ld = (int64_t)s.C * ES;
  const int rows = (int)(end - first);
  if (!ln.on || ln.r >= rows) return;
  const int64_t at = ((int64_t)wg.image * s.L + first) * ld + (int64_t)blk.c0 * ES;
  int gi[VE];
  ln.groups(s.pieces == 1 ? s.Cg : blk.cb, gi);
  float mean[VE], rs[VE], w[VE], b[VE];
  ln.k.load_f32(p.w ? p.w + blk.c0 : nullptr, 1.f, w);
  ln.k.load_f32(p.b ? p.b + blk.c0 : nullptr, 0.f, b);
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    const int g = min(gi[e], blk.ng - 1);
    mean[e] = smean[g];
    rs[e] = srstd[g];
  }
  const int n = (rows - ln.r + ln.rp - 1) / ln.rp;
  for (int i = 0; i < n; i += U) {
    Vec16 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = ln.k.load(p.x + at + (int64_t)(ln.r + min(i + u, n - 1) * ln.rp) * ld);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= n) break;
      float a[VE];
      ln.k.unpack(v[u], a);
#pragma unroll
      for (int e = 0; e < VE; ++e) a[e] = gn_act(fmaf((a[e] - mean[e]) * rs[e], w[e], b[e]), p.act);
      ln.k.store(p.y + at + (int64_t)(ln.r + (i + u) * ln.rp) * ld, a);
    }
  }
}

// An image's block whole: its rows in the registers of one work-group, NV vectors per
// thread, so that x is read once and the squares are taken about the mean.
template <int DT, int NV>
__global__ void __launch_bounds__(kGnSlab) gn_fwd_slab_kernel(GnFwd p) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES;
  __shared__ float cols[kGnSlab * VE], sums[kGnSlab];
  const GnShape& s = p.s;
  const GnAt wg(s, blockIdx.x, false);
  const GnBlock blk(s, wg.block);
  const GnLane<DT, false> ln(blk.cb);
  const int64_t ld = (int64_t)s.C * ES, at = (int64_t)wg.image * s.L * ld + (int64_t)blk.c0 * ES;
  const int L = (int)s.L;
  Vec16 x[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) x[i] = ln.k.load(p.x + at + (int64_t)min(ln.r + i * ln.rp, L - 1) * ld);
  float v[VE], w[VE], b[VE], mean[VE], rs[VE];
  int gi[VE];
  ln.groups(s.Cg, gi);
  ln.k.load_f32(p.w ? p.w + blk.c0 : nullptr, 1.f, w);
  ln.k.load_f32(p.b ? p.b + blk.c0 : nullptr, 0.f, b);
  const float all = (float)L * (float)s.Cg;
#pragma unroll
  for (int e = 0; e < VE; ++e) v[e] = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float a[VE];
    ln.k.unpack(x[i], a);
    const bool in = ln.on && ln.r + i * ln.rp < L;
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] += in ? a[e] : 0.f;
  }
  gn_columns(ln, blk.cb, v, cols);
  gn_teams(s, blk, cols, sums);
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    mean[e] = sums[min(gi[e], blk.ng - 1)] / all;
    v[e] = 0.f;
  }
  gn_packed(x);
  const float m = (int)threadIdx.x < blk.ng ? sums[threadIdx.x] / all : 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float a[VE];
    ln.k.unpack(x[i], a);
    const bool in = ln.on && ln.r + i * ln.rp < L;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float d = in ? a[e] - mean[e] : 0.f;
      v[e] = fmaf(d, d, v[e]);
    }
  }
  gn_columns(ln, blk.cb, v, cols);
  gn_teams(s, blk, cols, sums);
#pragma unroll
  for (int e = 0; e < VE; ++e) rs[e] = 1.f / sqrtf(sums[min(gi[e], blk.ng - 1)] / all + p.eps);
  if ((int)threadIdx.x < blk.ng) {
    const int64_t g = (int64_t)wg.image * s.G + blk.g0 + threadIdx.x;
    if (p.mean) p.mean[g] = m;
    if (p.rstd) p.rstd[g] = 1.f / sqrtf(sums[threadIdx.x] / all + p.eps);
  }
  if (!ln.on) return;
  gn_packed(x);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (ln.r + i * ln.rp >= L) break;
    float a[VE];
    ln.k.unpack(x[i], a);
#pragma unroll
    for (int e = 0; e < VE; ++e) a[e] = gn_act(fmaf((a[e] - mean[e]) * rs[e], w[e], b[e]), p.act);
    ln.k.store(p.y + at + (int64_t)(ln.r + i * ln.rp) * ld, a);
  }
}

struct GnBwd {
  GnShape s;
  const char *dy, *x;
  const float *mean, *rstd, *w, *b;
  const char* dres;
  char* dx;
  float2* part;  // [B][tiles][pieces][G]: sums of t and t xh
  float* wpart;  // [B tiles][2][C]: sums of du xh and du by column, or null
  float *dw, *db;
  int accumulate, act;
};

// A lane's constants of an image: its channels' statistics and affine weights.
template <int DT, bool TINY>
struct GnConst {
  static constexpr int VE = Ln<DT>::VE;
  float mean[VE], rs[VE], w[VE], b[VE];
  __device__ __forceinline__ GnConst(const GnBwd& p, const GnBlock& blk, const GnLane<DT, TINY>& ln, int image) {
    int gi[VE];
    ln.groups(p.s.pieces == 1 ? p.s.Cg : blk.cb, gi);
    ln.k.load_f32(p.w ? p.w + blk.c0 : nullptr, 1.f, w);
    ln.k.load_f32(p.b ? p.b + blk.c0 : nullptr, 0.f, b);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const int64_t g = (int64_t)image * p.s.G + blk.g0 + min(gi[e], blk.ng - 1);
      mean[e] = p.mean[g];
      rs[e] = p.rstd[g];
    }
  }
  // xh, and du in place of dy
  __device__ __forceinline__ void apply(float (&x)[VE], float (&dy)[VE], int act) const {
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      x[e] = (x[e] - mean[e]) * rs[e];
      dy[e] *= gn_slope(fmaf(x[e], w[e], b[e]), act);
    }
  }
};

// The sums of a tile's (or a whole image's, in one work-group) columns to memory, and
// the groups' sums of t and t xh into LDS.
template <int DT, bool TINY>
__device__ __forceinline__ void gn_bwd_sums(const GnBwd& p, const GnBlock& blk, const GnLane<DT, TINY>& ln,
                                            const float (&sx)[Ln<DT>::VE], const float (&sd)[Ln<DT>::VE], float* out_w,
                                            float* out_b, int add, float* cols, float* s1, float* s2) {
  for (int k = 0; k < 2; ++k) {
    gn_columns(ln, blk.cb, k ? sd : sx, cols);
    float* out = k ? out_b : out_w;
    for (int c = threadIdx.x; c < blk.cb; c += blockDim.x) {
      const float a = cols[c];
      if (out) out[blk.c0 + c] = add ? out[blk.c0 + c] + a : a;
      cols[c] = p.w ? a * p.w[blk.c0 + c] : a;
    }
    __syncthreads();
    gn_teams(p.s, blk, cols, k ? s1 : s2);
  }
}

template <int DT, bool TINY>
__global__ void __launch_bounds__(kGnThreads) gn_bwd_sums_kernel(GnBwd p) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, U = 4;
  __shared__ float cols[kGnThreads * VE], s1[kGnThreads], s2[kGnThreads];
  const GnShape& s = p.s;
  const GnAt wg(s, blockIdx.x, false);
  const GnBlock blk(s, wg.block);
  const GnLane<DT, TINY> ln(blk.cb);
  const int64_t first = (int64_t)wg.tile * s.R, end = min(first + s.R, s.L), ld = (int64_t)s.C * ES;
  const int rows = (int)(end - first);
  const int64_t at = ((int64_t)wg.image * s.L + first) * ld + (int64_t)blk.c0 * ES;
  float sx[VE], sd[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) sx[e] = sd[e] = 0.f;
  if (ln.on && ln.r < rows) {
    const GnConst<DT, TINY> c(p, blk, ln, wg.image);
    const int n = (rows - ln.r + ln.rp - 1) / ln.rp;
    for (int i = 0; i < n; i += U) {
      Vec16 vx[U], vy[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t o = at + (int64_t)(ln.r + min(i + u, n - 1) * ln.rp) * ld;
        vx[u] = ln.k.load(p.x + o);
        vy[u] = ln.k.load(p.dy + o);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u >= n) break;
        float x[VE], dy[VE];
        Ln<DT>::unpack(vx[u], x);
        ln.k.unpack(vy[u], dy);
        c.apply(x, dy, p.act);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          sx[e] = fmaf(dy[e], x[e], sx[e]);
          sd[e] += dy[e];
        }
      }
    }
  }
  const int64_t tile = (int64_t)wg.image * s.tiles + wg.tile;
  float* out = p.wpart ? p.wpart + tile * 2 * s.C : nullptr;
  gn_bwd_sums(p, blk, ln, sx, sd, out, out ? out + s.C : nullptr, 0, cols, s1, s2);
  if (p.part && (int)threadIdx.x < blk.ng)
    p.part[(tile * s.pieces + blk.piece) * s.G + blk.g0 + threadIdx.x] = float2{s1[threadIdx.x], s2[threadIdx.x]};
}

// 32 of the 2 C columns of dw and db from n partial sums.
__device__ __forceinline__ void gn_reduce(const GnBwd& p, int64_t n, int at) {
  __shared__ float t[kGnThreads / 32][33];
  const int cl = threadIdx.x & 31, r = threadIdx.x >> 5, C = p.s.C;
  const int64_t c = (int64_t)at * 32 + cl;
  float a = 0.f;
  if (c < 2 * (int64_t)C) {
#pragma unroll 8
    for (int64_t i = r; i < n; i += kGnThreads / 32) a += p.wpart[i * 2 * C + c];
  }
  t[r][cl] = a;
  __syncthreads();
  if (r == 0 && c < 2 * (int64_t)C) {
    a = 0.f;
#pragma unroll
    for (int i = 0; i < kGnThreads / 32; ++i) a += t[i][cl];
    float* out = c < C ? p.dw : p.db;
    const int64_t o = c < C ? c : c - C;
    if (out) out[o] = p.accumulate ? out[o] + a : a;
  }
}
__global__ void __launch_bounds__(kGnThreads) gn_reduce_kernel(GnBwd p, int64_t n) { gn_reduce(p, n, blockIdx.x); }

template <int DT, bool TINY>
__global__ void __launch_bounds__(kGnThreads) gn_bwd_rows_kernel(GnBwd p) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, U = 2;
  __shared__ float s1[kGnThreads], s2[kGnThreads];
  const GnShape& s = p.s;
  const unsigned tiles = (unsigned)s.B * s.tiles * s.blocks;
  if (blockIdx.x >= tiles) return gn_reduce(p, (int64_t)s.B * s.tiles, (int)(blockIdx.x - tiles));  // (behind the rows)
  const GnAt wg(s, blockIdx.x, true);
  const GnBlock blk(s, wg.block);
  const GnLane<DT, TINY> ln(blk.cb);
  const float all = (float)(int)s.L * (float)s.Cg;
  {
    const int g = threadIdx.x / s.team, i = threadIdx.x - g * s.team, entries = s.tiles * s.pieces;
    float a = 0.f, b = 0.f;
    if (g < blk.ng) {
      const float2* q = p.part + (int64_t)wg.image * entries * s.G + blk.g0 + g;
#pragma unroll 4
      for (int j = i; j < entries; j += s.team) {
        const float2 v = q[(int64_t)j * s.G];
        a += v.x;
        b += v.y;
      }
    }
    for (int o = 1; o < s.team; o <<= 1) {
      a += __shfl_xor(a, o, kWave);
      b += __shfl_xor(b, o, kWave);
    }
    if (g < blk.ng && i == 0) {
      s1[g] = a / all;
      s2[g] = b / all;
    }
    __syncthreads();
  }
  const int64_t first = (int64_t)wg.tile * s.R, end = min(first + s.R, s.L), ld = (int64_t)s.C * ES;
  const int rows = (int)(end - first);
  if (!ln.on || ln.r >= rows) return;
  const int64_t at = ((int64_t)wg.image * s.L + first) * ld + (int64_t)blk.c0 * ES;
  const GnConst<DT, TINY> c(p, blk, ln, wg.image);
  int gi[VE];
  ln.groups(s.pieces == 1 ? s.Cg : blk.cb, gi);
  float m1[VE], m2[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    const int g = min(gi[e], blk.ng - 1);
    m1[e] = s1[g];
    m2[e] = s2[g];
  }
  const int n = (rows - ln.r + ln.rp - 1) / ln.rp;
  for (int i = 0; i < n; i += U) {
    Vec16 vx[U], vy[U], vr[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t o = at + (int64_t)(ln.r + min(i + u, n - 1) * ln.rp) * ld;
      vx[u] = ln.k.load(p.x + o);
      vy[u] = ln.k.load(p.dy + o);
      if (p.dres) vr[u] = ln.k.load(p.dres + o);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= n) break;
      float x[VE], dy[VE];
      Ln<DT>::unpack(vx[u], x);
      ln.k.unpack(vy[u], dy);
      c.apply(x, dy, p.act);
#pragma unroll
      for (int e = 0; e < VE; ++e) dy[e] = c.rs[e] * (fmaf(dy[e], c.w[e], -m1[e]) - x[e] * m2[e]);
      if (p.dres) {
        float z[VE];
        Ln<DT>::unpack(vr[u], z);
#pragma unroll
        for (int e = 0; e < VE; ++e) dy[e] += z[e];
      }
      ln.k.store(p.dx + at + (int64_t)(ln.r + (i + u) * ln.rp) * ld, dy);
    }
  }
}

// An image's block whole, as the forward pass's. With one image dw and db are its sums.
template <int DT, int NV>
__global__ void __launch_bounds__(kGnSlab) gn_bwd_slab_kernel(GnBwd p) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES;
  __shared__ float cols[kGnSlab * VE], s1[kGnSlab], s2[kGnSlab];
  const GnShape& s = p.s;
  const GnAt wg(s, blockIdx.x, false);
  const GnBlock blk(s, wg.block);
  const GnLane<DT, false> ln(blk.cb);
  const int64_t ld = (int64_t)s.C * ES, at = (int64_t)wg.image * s.L * ld + (int64_t)blk.c0 * ES;
  const int L = (int)s.L;
  Vec16 vx[NV], vy[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int64_t o = at + (int64_t)min(ln.r + i * ln.rp, L - 1) * ld;
    vx[i] = ln.k.load(p.x + o);
    vy[i] = ln.k.load(p.dy + o);
  }
  const GnConst<DT, false> c(p, blk, ln, wg.image);
  float sx[VE], sd[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) sx[e] = sd[e] = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float x[VE], dy[VE];
    Ln<DT>::unpack(vx[i], x);
    ln.k.unpack(vy[i], dy);
    c.apply(x, dy, p.act);
    const bool in = ln.on && ln.r + i * ln.rp < L;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      sx[e] += in ? dy[e] * x[e] : 0.f;
      sd[e] += in ? dy[e] : 0.f;
    }
  }
  float* out = p.wpart ? p.wpart + (int64_t)wg.image * 2 * s.C : nullptr;
  gn_bwd_sums(p, blk, ln, sx, sd, out ? out : p.dw, out ? out + s.C : p.db, out ? 0 : p.accumulate, cols, s1, s2);
  if (!ln.on || !p.dx) return;
  gn_packed(vx);
  gn_packed(vy);
  int gi[VE];
  ln.groups(s.Cg, gi);
  const float all = (float)L * (float)s.Cg;
  float m1[VE], m2[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    const int g = min(gi[e], blk.ng - 1);
    m1[e] = s1[g] / all;
    m2[e] = s2[g] / all;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (ln.r + i * ln.rp >= L) break;
    const int64_t o = at + (int64_t)(ln.r + i * ln.rp) * ld;
    float x[VE], dy[VE];
    Ln<DT>::unpack(vx[i], x);
    ln.k.unpack(vy[i], dy);
    c.apply(x, dy, p.act);
#pragma unroll
    for (int e = 0; e < VE; ++e) dy[e] = c.rs[e] * (fmaf(dy[e], c.w[e], -m1[e]) - x[e] * m2[e]);
    if (p.dres) {
      float z[VE];
      Ln<DT>::unpack(ln.k.load(p.dres + o), z);
#pragma unroll
      for (int e = 0; e < VE; ++e) dy[e] += z[e];
    }
    ln.k.store(p.dx + o, dy);
  }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
constexpr int kGnMaxWidth = 16384;

struct GnPlan {
  GnShape s;
  int threads, NV;  // NV 0: two launches
  bool tiny;
  int64_t grid;
};

static int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// kg groups per block, the last block at least a vector wide.
static void gn_blocks(GnShape* s, int64_t kg, int VE) {
  int64_t nb = up(s->G, kg);
  kg = up(s->G, nb);
  while (kg < s->G && (s->G - (up(s->G, kg) - 1) * kg) * s->Cg < VE) ++kg;
  s->kg = (int)kg;
  s->pieces = 1;
  s->pw = s->Cg;
  s->blocks = (int)up(s->G, kg);
}
static void gn_team(GnShape* s, int threads) {
  const int width = s->pieces == 1 ? s->Cg : s->pw;
  s->team = 1;
  while (s->team < 64 && s->team < width && s->team * 2 * s->kg <= threads) s->team *= 2;
}

// An image's block as one work-group's: blocks of at least `bytes` per row.
static bool gn_slab(GnPlan* p, int bytes, int most, int dt) {
  const int VE = dt == GTR_F32 ? 4 : 8, ES = dt == GTR_F32 ? 4 : 2;
  GnShape* s = &p->s;
  gn_blocks(s, up(bytes, (int64_t)s->Cg * ES), VE);
  const int64_t nl = up((int64_t)s->kg * s->Cg, VE);
  if (nl > kGnSlab || s->L > (int64_t)kGnSlab * most) return false;
  int64_t threads = up(s->L * nl, 64) * 64;
  if (threads < up(s->kg, 64) * 64) threads = up(s->kg, 64) * 64;
  p->threads = (int)(threads < kGnSlab ? threads : kGnSlab);
  if (s->kg > p->threads) return false;
  const int64_t nv = up(s->L, p->threads / nl);
  if (nv > most) return false;
  p->NV = nv <= 1 ? 1 : nv <= 2 ? 2 : nv <= 4 ? 4 : nv <= 8 ? 8 : 16;
  s->tiles = 1;
  s->R = 0;
  gn_team(s, p->threads);
  p->grid = (int64_t)s->B * s->blocks;
  return p->grid * p->threads < (int64_t)1 << 32;
}

static gtr_status gn_plan(int32_t B, int64_t L, int32_t C, int32_t G, int dt, bool bwd, GnPlan* p) {
  if (B <= 0 || L <= 0 || C <= 0 || G <= 0 || C % G != 0) return GTR_ERR_SHAPE;
  if (C > kGnMaxWidth || (dt != GTR_F32 && dt != GTR_F16 && dt != GTR_BF16)) return GTR_ERR_UNSUPPORTED;
  if (L >= (int64_t)1 << 31 || B * L >= (int64_t)1 << 40) return GTR_ERR_SHAPE;
  const int VE = dt == GTR_F32 ? 4 : 8;
  *p = GnPlan{};
  GnShape* s = &p->s;
  s->L = L;
  s->B = B;
  s->C = C;
  s->G = G;
  s->Cg = C / G;
  p->tiny = C < VE;
  if (!p->tiny)
    for (int bytes : {128, 64})
      if (gn_slab(p, bytes, bwd ? 4 : 8, dt)) return GTR_OK;
  p->NV = 0;
  p->threads = kGnThreads;
  const int CB = 64 * VE;
  if (s->Cg <= CB) {
    const int kg = CB / s->Cg;
    gn_blocks(s, kg < kGnThreads ? kg : kGnThreads, VE);
  } else {
    s->kg = 1;
    s->pieces = (int)up(s->Cg, CB);
    s->pw = (int)up(s->Cg, s->pieces);
    s->blocks = s->G * s->pieces;
  }
  gn_team(s, kGnThreads);
  const int64_t cb = s->pieces == 1 ? (int64_t)s->kg * s->Cg : s->pw, rp = kGnThreads / up(cb, VE);
  int64_t tiles = up(2048, (int64_t)B * s->blocks);
  if (tiles > up(L, rp * 4)) tiles = up(L, rp * 4);
  if (tiles > 256) tiles = 256;
  s->R = (int)(up(up(L, tiles), rp) * rp);
  s->tiles = (int)up(L, s->R);
  p->grid = (int64_t)B * s->tiles * s->blocks;
  return (p->grid + up(2 * (int64_t)C, 32)) * kGnThreads < (int64_t)1 << 32 ? GTR_OK : GTR_ERR_SHAPE;
}

static size_t gn_stats_bytes(const GnPlan& p) {
  return p.NV ? 0 : (size_t)up((int64_t)p.s.B * p.s.tiles * p.s.pieces * p.s.G * 8, 256) * 256;
}
static size_t gn_weights_bytes(const GnPlan& p) {  // of the columns' partial sums
  return p.NV && p.s.B == 1 ? 0 : (size_t)up((int64_t)p.s.B * p.s.tiles * 2 * p.s.C * 4, 256) * 256;
}

template <int DT>
static void gn_go(const GnPlan& p, const GnFwd& f, hipStream_t st) {
  const dim3 g((unsigned)p.grid), t(p.threads);
  switch (p.NV) {
    case 0:
      if (p.tiny) {
        hipLaunchKernelGGL((gn_fwd_sums_kernel<DT, true>), g, t, 0, st, f);
        hipLaunchKernelGGL((gn_fwd_rows_kernel<DT, true>), g, t, 0, st, f);
      } else {
        hipLaunchKernelGGL((gn_fwd_sums_kernel<DT, false>), g, t, 0, st, f);
        hipLaunchKernelGGL((gn_fwd_rows_kernel<DT, false>), g, t, 0, st, f);
      }
      break;
    case 1: hipLaunchKernelGGL((gn_fwd_slab_kernel<DT, 1>), g, t, 0, st, f); break;
    case 2: hipLaunchKernelGGL((gn_fwd_slab_kernel<DT, 2>), g, t, 0, st, f); break;
    case 4: hipLaunchKernelGGL((gn_fwd_slab_kernel<DT, 4>), g, t, 0, st, f); break;
    case 8: hipLaunchKernelGGL((gn_fwd_slab_kernel<DT, 8>), g, t, 0, st, f); break;
    default: hipLaunchKernelGGL((gn_fwd_slab_kernel<DT, 16>), g, t, 0, st, f); break;
  }
}
template <int DT>
static void gn_go(const GnPlan& p, const GnBwd& f, hipStream_t st) {
  const dim3 g((unsigned)p.grid), t(p.threads);
  const unsigned sums = f.wpart ? (unsigned)up(2 * (int64_t)p.s.C, 32) : 0;
  if (p.NV == 0) {
    const dim3 gr(g.x + sums);
    if (p.tiny)
      hipLaunchKernelGGL((gn_bwd_sums_kernel<DT, true>), g, t, 0, st, f);
    else
      hipLaunchKernelGGL((gn_bwd_sums_kernel<DT, false>), g, t, 0, st, f);
    if (f.dx) {
      if (p.tiny)
        hipLaunchKernelGGL((gn_bwd_rows_kernel<DT, true>), gr, t, 0, st, f);
      else
        hipLaunchKernelGGL((gn_bwd_rows_kernel<DT, false>), gr, t, 0, st, f);
      return;
    }
  } else if (p.NV == 1) {
    hipLaunchKernelGGL((gn_bwd_slab_kernel<DT, 1>), g, t, 0, st, f);
  } else if (p.NV == 2) {
    hipLaunchKernelGGL((gn_bwd_slab_kernel<DT, 2>), g, t, 0, st, f);
  } else if (p.NV == 4) {
    hipLaunchKernelGGL((gn_bwd_slab_kernel<DT, 4>), g, t, 0, st, f);
  } else {
    hipLaunchKernelGGL((gn_bwd_slab_kernel<DT, 8>), g, t, 0, st, f);
  }
  if (sums)
    hipLaunchKernelGGL(gn_reduce_kernel, dim3(sums), dim3(kGnThreads), 0, st, f, (int64_t)p.s.B * p.s.tiles);
}
template <class F>
static gtr_status gn_launch(int dt, const GnPlan& p, const F& f, hipStream_t st) {
  if (dt == GTR_F32)
    gn_go<GTR_F32>(p, f, st);
  else if (dt == GTR_F16)
    gn_go<GTR_F16>(p, f, st);
  else
    gn_go<GTR_BF16>(p, f, st);
  return hipGetLastError() == hipSuccess ? GTR_OK : GTR_ERR_HIP;
}

static bool gn_misaligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }
static bool gn_act_ok(int act) { return act == GTR_ACT_SILU || act == GTR_ACT_GELU || act == GTR_ACT_NONE; }

static gtr_status gn_fwd_check(const gtr_groupnorm_fwd_args* a, GnPlan* p) {
  if (!a) return GTR_ERR_NULL;
  const gtr_status st = gn_plan(a->B, a->L, a->C, a->groups, a->dtype, false, p);
  if (st != GTR_OK) return st;
  return gn_act_ok(a->act) && a->eps >= 0.f && a->eps < 1e30f ? GTR_OK : GTR_ERR_UNSUPPORTED;
}
static gtr_status gn_bwd_check(const gtr_groupnorm_bwd_args* a, GnPlan* p, size_t* need) {
  if (!a) return GTR_ERR_NULL;
  const gtr_status st = gn_plan(a->B, a->L, a->C, a->groups, a->dtype, true, p);
  if (st != GTR_OK) return st;
  *need = (a->dx ? gn_stats_bytes(*p) : 0) + (a->dw || a->db ? gn_weights_bytes(*p) : 0);
  return gn_act_ok(a->act) ? GTR_OK : GTR_ERR_UNSUPPORTED;
}

}  // namespace gtr

using namespace gtr;

extern "C" size_t gtr_groupnorm_fwd_workspace_size(const gtr_groupnorm_fwd_args* a) {
  GnPlan p;
  return gn_fwd_check(a, &p) == GTR_OK ? gn_stats_bytes(p) : 0;
}

extern "C" gtr_status gtr_groupnorm_fwd(const gtr_groupnorm_fwd_args* a, hipStream_t stream) {
  GnPlan p;
  const gtr_status st = gn_fwd_check(a, &p);
  if (st != GTR_OK) return st;
  if (!a->x || !a->y) return GTR_ERR_NULL;
  const size_t es = dtype_size(a->dtype), bytes = (size_t)a->B * a->L * a->C * es, stats = (size_t)a->B * a->groups * 4;
  if (gn_misaligned(a->x, es) || gn_misaligned(a->y, es) || gn_misaligned(a->w, 4) || gn_misaligned(a->b, 4) ||
      gn_misaligned(a->mean, 4) || gn_misaligned(a->rstd, 4))
    return GTR_ERR_UNSUPPORTED;
  const size_t need = gn_stats_bytes(p);
  if (need && (!a->workspace || gn_misaligned(a->workspace, 256) || a->workspace_bytes < need)) return GTR_ERR_WORKSPACE;
  const Bytes ins[] = {{a->x, bytes}, {a->w, (size_t)a->C * 4}, {a->b, (size_t)a->C * 4}};
  const Bytes outs[] = {{a->y, bytes}, {a->mean, stats}, {a->rstd, stats}, {need ? a->workspace : nullptr, need}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 3; ++j)
      if (bytes_meet(outs[i], ins[j]) && !(i == 0 && j == 0 && a->x == a->y)) return GTR_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (bytes_meet(outs[i], outs[j])) return GTR_ERR_ALIAS;
  }
  const GnFwd f = {p.s, static_cast<const char*>(a->x), a->w, a->b, static_cast<char*>(a->y), a->mean, a->rstd,
                   static_cast<float2*>(a->workspace), a->eps, a->act};
  return gn_launch(a->dtype, p, f, stream);
}

extern "C" size_t gtr_groupnorm_bwd_workspace_size(const gtr_groupnorm_bwd_args* a) {
  GnPlan p;
  size_t need;
  return gn_bwd_check(a, &p, &need) == GTR_OK ? need : 0;
}

extern "C" gtr_status gtr_groupnorm_bwd(const gtr_groupnorm_bwd_args* a, hipStream_t stream) {
  GnPlan p;
  size_t need;
  const gtr_status st = gn_bwd_check(a, &p, &need);
  if (st != GTR_OK) return st;
  if (!a->dy || !a->x || !a->mean || !a->rstd || (!a->dx && !a->dw && !a->db)) return GTR_ERR_NULL;
  const size_t es = dtype_size(a->dtype), bytes = (size_t)a->B * a->L * a->C * es, stats = (size_t)a->B * a->groups * 4,
               wide = (size_t)a->C * 4;
  if (gn_misaligned(a->dy, es) || gn_misaligned(a->x, es) || gn_misaligned(a->dres, es) || gn_misaligned(a->dx, es) ||
      gn_misaligned(a->mean, 4) || gn_misaligned(a->rstd, 4) || gn_misaligned(a->w, 4) || gn_misaligned(a->b, 4) ||
      gn_misaligned(a->dw, 4) || gn_misaligned(a->db, 4))
    return GTR_ERR_UNSUPPORTED;
  if (need && (!a->workspace || gn_misaligned(a->workspace, 256) || a->workspace_bytes < need)) return GTR_ERR_WORKSPACE;
  const Bytes ins[] = {{a->dy, bytes}, {a->x, bytes}, {a->dres, bytes}, {a->mean, stats}, {a->rstd, stats},
                       {a->w, wide}, {a->b, wide}};
  const Bytes outs[] = {{a->dx, bytes}, {a->dw, wide}, {a->db, wide}, {need ? a->workspace : nullptr, need}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 7; ++j)
      if (bytes_meet(outs[i], ins[j]) && !(i == 0 && j < 3 && outs[i].p == ins[j].p)) return GTR_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (bytes_meet(outs[i], outs[j])) return GTR_ERR_ALIAS;
  }
  const size_t stat = a->dx ? gn_stats_bytes(p) : 0, sums = a->dw || a->db ? gn_weights_bytes(p) : 0;
  char* ws = static_cast<char*>(a->workspace);
  const GnBwd f = {p.s, static_cast<const char*>(a->dy), static_cast<const char*>(a->x), a->mean, a->rstd, a->w, a->b,
                   static_cast<const char*>(a->dres), static_cast<char*>(a->dx), stat ? reinterpret_cast<float2*>(ws) : nullptr,
                   sums ? reinterpret_cast<float*>(ws + stat) : nullptr, a->dw, a->db, a->accumulate, a->act};
  return gn_launch(a->dtype, p, f, stream);
}
