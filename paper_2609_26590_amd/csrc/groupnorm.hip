// Group norm with an activation over token grids, channels last, and its gradients. Per
// image and group of channels, over all tokens and the group's channels, in float32:
//
//   forward:  mean, rstd = (var + eps)^(-1/2),  xh = (x - mean) rstd,
//             y = act(xh w + b)
//   backward: du = dy act'(xh w + b),  t = du w,
//             dx = rstd (t - mean(t) - xh mean(t xh)) (+ dres)
//             dw = sum over images and tokens of du xh,  db = that of du
//
// What bounds both is memory and, for small images, the chain of loads, sums and stores.
// Where an image's block of groups fits the registers of one work-group, it is read once,
// in one launch (gn_*_image_kernel), else twice by two launches (gn_*_sums_kernel,
// gn_*_rows_kernel): 16 x 16384 x 512 bf16 forward 172 us, 4.7 TB/s of what both read and
// write, 16 x 4096 x 1024 backward with dres 162, 5.0; a large copy reaches 5.0.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "ffn_gemm.h"
#include "gtr.h"
#include "gtr_device.h"
#include "gtr_internal.h"
#include "vec_rows.h"

namespace gtr {

// The channels in blocks: kg whole groups each, or where a group is wider than a block
// allows, `pieces` of pw channels (the last may be narrower). nl lanes, a power of two up to
// 64, hold a block's row, and a work-group rp rows at a time, a row group. Tile t of an image
// has the row groups t, t + tiles, ..: all tiles go through the memory side by side.
struct GnShape {
  int64_t L;
  int B, C, G, Cg;
  int kg, pieces, pw, blocks;
  int nl, shift;  // shift: log2 nl
  int tiles;
  int team, tshift;  // threads that add a group's channels: a power of two, kg teams at most the work-group's threads
  float inv_width, inv_pieces;  // of a group's channels in a block
};
// n / d for 0 <= n < 2^14 and whole d: (n + 1/2) / d is 1 / (2 d) from a whole number or more,
// its rounding errors under 2^-8 / d.
__device__ __forceinline__ int gn_div(int n, float inv) { return (int)(((float)n + 0.5f) * inv); }
struct GnBlock {
  int g0, ng, c0, cb, piece, width;  // width: of a group, or of the piece
  __device__ __forceinline__ GnBlock(const GnShape& s, int block) {
    if (s.pieces == 1) {
      g0 = block * s.kg;
      ng = min(s.kg, s.G - g0);
      piece = 0;
      c0 = g0 * s.Cg;
      cb = ng * s.Cg;
      width = s.Cg;
    } else {
      g0 = block / s.pieces;  // (uniform)
      ng = 1;
      piece = block - g0 * s.pieces;
      c0 = g0 * s.Cg + piece * s.pw;
      cb = width = min(s.pw, s.Cg - piece * s.pw);
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
    const unsigned t = s.blocks == 1 ? id : id / (unsigned)s.blocks;
    block = (int)(id - t * (unsigned)s.blocks);
    image = s.B == 1 ? 0 : (int)(t / (unsigned)s.tiles);
    tile = (int)(t - (unsigned)image * (unsigned)s.tiles);
  }
};

// f with the activation as a constant: one test per loop, not three per value.
template <int ACT>
struct GnAct {
  static __device__ __forceinline__ float value(float u) {
    if constexpr (ACT == GTR_ACT_NONE) return u;
    float slope;
    return ffn_act(u, ACT, slope);
  }
  static __device__ __forceinline__ float slope(float u) {
    if constexpr (ACT == GTR_ACT_NONE) return 1.f;
    float s;
    ffn_act(u, ACT, s);
    return s;
  }
};
template <class F>
__device__ __forceinline__ void gn_by_act(int act, const F& f) {
  if (act == GTR_ACT_SILU)
    f(GnAct<GTR_ACT_SILU>());
  else if (act == GTR_ACT_GELU)
    f(GnAct<GTR_ACT_GELU>());
  else
    f(GnAct<GTR_ACT_NONE>());
}

// A thread's place on a block: its vector of the row, and which of the rows that the
// work-group takes at a time. Lanes past the block's width have nothing.
template <int DT, bool TINY>
struct GnLane {
  static constexpr int VE = Ln<DT>::VE;
  LnCols<DT, TINY> k;
  int r, rp;
  __device__ __forceinline__ GnLane(const GnShape& s, int cb)
      : k((int)threadIdx.x & (s.nl - 1), cb), r((int)threadIdx.x >> s.shift), rp((int)blockDim.x >> s.shift) {}
  // the groups (of the block's) of this lane's channels
  __device__ __forceinline__ void groups(const GnShape& s, const GnBlock& b, int (&g)[VE]) const {
    int i = s.pieces == 1 ? gn_div(k.c, s.inv_width) : 0, rem = k.c - i * b.width;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      g[e] = min(i, b.ng - 1);
      if (++rem == b.width) {
        rem = 0;
        ++i;
      }
    }
  }
};

// An image's row groups over its tiles: each tile has `base`, the first `more` one besides,
// and the last group lacks `lack` rows.
struct GnTiles {
  int base, more, lack, last;
  __device__ __forceinline__ GnTiles(const GnShape& s, int rp) {
    const int L = (int)s.L, groups = (L >> __builtin_ctz(rp)) + ((L & (rp - 1)) != 0);
    base = s.tiles == 1 ? groups : groups / s.tiles;
    more = groups - base * s.tiles;
    lack = (int)((int64_t)groups * rp - s.L);
    last = more ? more - 1 : s.tiles - 1;  // the tile that has it
  }
  __device__ __forceinline__ int groups(int tile) const { return base + (tile < more); }
  __device__ __forceinline__ int rows(int tile, int rp) const { return groups(tile) * rp - (tile == last ? lack : 0); }
  // of which a thread whose row of each group is r has
  __device__ __forceinline__ int rows_of(int tile, int r, int rp) const {
    return groups(tile) - (tile == last && r >= rp - lack);
  }
};

// Sums of N values per lane over the lanes of a wave that hold the same vector of a row, in
// every one of them, in registers: rows of 16 lanes rotate, halves and quarters swap.
template <int ROT>
__device__ __forceinline__ float gn_rot(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x120 + ROT, 0xf, 0xf, false));
}
__device__ __forceinline__ float gn_halves(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const unsigned lo = r[0], hi = r[1];
  return __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
}
__device__ __forceinline__ float gn_quarters(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const unsigned lo = r[0], hi = r[1];
  return __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
}
template <int N>
__device__ __forceinline__ void gn_wave(float (&v)[N], int nl) {
  if (nl <= 32)
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = gn_halves(v[e]);
  if (nl <= 16)
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = gn_quarters(v[e]);
  if (nl <= 8)
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] += gn_rot<8>(v[e]);
  if (nl <= 4)
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] += gn_rot<4>(v[e]);
  if (nl <= 2)
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] += gn_rot<2>(v[e]);
  if (nl <= 1)
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] += gn_rot<1>(v[e]);
}

// The waves' sums of each channel lie in cols[wave][element][lane]: by element first, so
// that writes do not meet in a bank of LDS. gn_column's reads do where nl is large: neighbouring
// threads take neighbouring channels, whose sums lie nl words apart (with nl 64 those of a
// vector are in one bank). Counted over all CUs: 2.6e5 cycles in the sums of 8 x 1600 x 384
// forward, 1.8e6 of 16 x 16384 x 512, 3.7e6 of 16 x 4096 x 1024 backward; none with the few
// lanes per row of an image in one launch.
template <int DT>
__device__ __forceinline__ void gn_put(const GnShape& s, float (&v)[Ln<DT>::VE], float* cols) {
  constexpr int VE = Ln<DT>::VE;
  gn_wave(v, s.nl);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane < s.nl)
#pragma unroll
    for (int e = 0; e < VE; ++e) cols[(wave * VE + e) * s.nl + lane] = v[e];
}
// The work-group's sum of channel c of the block.
template <int DT, bool TINY>
__device__ __forceinline__ float gn_column(const GnShape& s, int cb, int c, const float* cols) {
  constexpr int VE = Ln<DT>::VE;
  const int l = c / VE, e = c - (TINY ? l * VE : min(l * VE, cb - VE)), waves = blockDim.x >> 6;
  float a = 0.f;
  for (int w = 0; w < waves; ++w) a += cols[(w * VE + e) * s.nl + l];
  return a;
}
// Sums over a team's threads, which a wave has whole, in every one of them.
__device__ __forceinline__ float gn_team_sum(float a, int team) {
  for (int o = 1; o < team; o <<= 1) a += __shfl_xor(a, o, kWave);
  return a;
}
// The groups' sums over a work-group of a value per channel (v is used up; values of
// channels that the lane has not, or shares, are not looked at), in a fixed order, divided by
// n, into sums[0 .. ng). Two barriers, the last at the end; cols: 64 VE floats per wave.
template <int DT, bool TINY>
__device__ __forceinline__ void gn_group_sums(const GnShape& s, const GnBlock& b, float (&v)[Ln<DT>::VE], float n,
                                              float* cols, float* sums) {
  gn_put<DT>(s, v, cols);
  __syncthreads();
  const int g = threadIdx.x >> s.tshift, i = threadIdx.x & (s.team - 1);
  float a = 0.f;
  if (g < b.ng)
    for (int c = i; c < b.width; c += s.team) a += gn_column<DT, TINY>(s, b.cb, g * b.width + c, cols);
  a = gn_team_sum(a, s.team);
  if (g < b.ng && i == 0) sums[g] = a / n;
  __syncthreads();
}

// Mean and sum of squares about it of n values, joined with another's.
struct GnStat {
  float n, mean, m2;
  __device__ __forceinline__ void join(float n2, float mean2, float m22) {
    const float all = n + n2, d = mean2 - mean, f = n > 0.f ? n2 * __builtin_amdgcn_rcpf(all) : 1.f;
    mean = fmaf(d, f, mean);
    m2 += fmaf(d * (n * f), d, m22);  // (d d is past float32 where a far mean meets no values, n or n2 = 0)
    n = all;
  }
  // with the lane's across bit o: both in the same order, the lower lane's first
  __device__ __forceinline__ void join_across(int o) {
    const float n2 = __shfl_xor(n, o, kWave), mn = __shfl_xor(mean, o, kWave), q = __shfl_xor(m2, o, kWave);
    const bool low = (threadIdx.x & o) == 0;
    GnStat a = {low ? n : n2, low ? mean : mn, low ? m2 : q};
    a.join(low ? n2 : n, low ? mn : mean, low ? q : m2);
    *this = a;
  }
};

// A vector in four registers next to each other, and unpacked again from here on: without
// that the compiler keeps its elements, in twice the registers or more.
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x4 gn_load(const char* p) {
  return __builtin_bit_cast(u32x4, *reinterpret_cast<const Vec16*>(p));
}
__device__ __forceinline__ Vec16 gn_vec(u32x4 v) { return __builtin_bit_cast(Vec16, v); }
template <int N>
__device__ __forceinline__ void gn_packed(u32x4 (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

// One vector after the other: unpacked side by side they would not fit the registers.
__device__ __forceinline__ void gn_next() { __builtin_amdgcn_sched_barrier(0); }

// To a lane's vector of a row, at its address.
template <int DT>
__device__ __forceinline__ void gn_store(const LnCols<DT, false>& k, char* at, const float (&x)[Ln<DT>::VE]) {
  if (k.skip == 0) {
    *reinterpret_cast<Vec16*>(at) = Ln<DT>::pack(x);
  } else {
#pragma unroll
    for (int e = 0; e < Ln<DT>::VE; ++e)
      if (k.has(e)) Ln<DT>::put(at + e * Ln<DT>::ES, x[e]);
  }
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

constexpr int kGnThreads = 256, kGnImage = 1024;

// An image's block whole: its rows in the registers of one work-group, NV vectors per
// thread, so that x is read once and the squares are taken about the mean.
template <int DT, int NV>
__global__ void __launch_bounds__(kGnImage) gn_fwd_image_kernel(GnFwd p) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES;
  __shared__ float cols[kGnImage * VE], sums[2][kGnImage];
  const GnShape& s = p.s;
  const GnAt wg(s, blockIdx.x, false);
  const GnBlock blk(s, wg.block);
  const GnLane<DT, false> ln(s, blk.cb);
  const int64_t ld = (int64_t)s.C * ES, at = (int64_t)wg.image * s.L * ld + (int64_t)blk.c0 * ES;
  const int L = (int)s.L;
  u32x4 x[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) x[i] = gn_load(p.x + at + (int64_t)min(ln.r + i * ln.rp, L - 1) * ld + ln.k.c * ES);
  float v[VE], w[VE], b[VE], mean[VE];
  int gi[VE];
  ln.groups(s, blk, gi);
  ln.k.load_f32(p.w ? p.w + blk.c0 : nullptr, 1.f, w);
  ln.k.load_f32(p.b ? p.b + blk.c0 : nullptr, 0.f, b);
  const float all = (float)L * (float)s.Cg;
#pragma unroll
  for (int e = 0; e < VE; ++e) v[e] = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float a[VE];
    Ln<DT>::unpack(gn_vec(x[i]), a);
    const bool in = ln.r + i * ln.rp < L;
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] += in ? a[e] : 0.f;
    gn_next();
  }
  gn_packed(x);
  gn_group_sums<DT, false>(s, blk, v, all, cols, sums[0]);
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    mean[e] = sums[0][gi[e]];
    v[e] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float a[VE];
    Ln<DT>::unpack(gn_vec(x[i]), a);
    const bool in = ln.r + i * ln.rp < L;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float d = in ? a[e] - mean[e] : 0.f;
      v[e] = fmaf(d, d, v[e]);
    }
    gn_next();
  }
  gn_packed(x);
  gn_group_sums<DT, false>(s, blk, v, all, cols, sums[1]);
  if ((int)threadIdx.x < blk.ng) {
    const int64_t g = (int64_t)wg.image * s.G + blk.g0 + threadIdx.x;
    if (p.mean) p.mean[g] = sums[0][threadIdx.x];
    if (p.rstd) p.rstd[g] = 1.f / sqrtf(sums[1][threadIdx.x] + p.eps);
  }
  if (ln.k.skip == VE) return;
#pragma unroll
  for (int e = 0; e < VE; ++e) w[e] *= 1.f / sqrtf(sums[1][gi[e]] + p.eps);
  gn_by_act(p.act, [&](auto act) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (ln.r + i * ln.rp < L) {
        float a[VE];
        Ln<DT>::unpack(gn_vec(x[i]), a);
#pragma unroll
        for (int e = 0; e < VE; ++e) a[e] = act.value(fmaf(a[e] - mean[e], w[e], b[e]));
        ln.k.store(p.y + at + (int64_t)(ln.r + i * ln.rp) * ld, a);
      }
      gn_next();
    }
  });
}

// A lane's sums of k values about `pivot` (s1 of their deviations, s2 of those squared),
// moved to their mean. Values that are not finite leave them as they are.
template <int VE>
__device__ __forceinline__ void gn_about_mean(float k, float (&pivot)[VE], float (&s1)[VE], float (&s2)[VE]) {
  const float inv = 1.f / k;
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    const float to = fmaf(s1[e], inv, pivot[e]), by = to - pivot[e], rest = fmaf(-k, by, s1[e]);
    const float sq = fmaf(-by, s1[e] + rest, s2[e]);
    const bool ok = sq == sq;
    pivot[e] = ok ? to : pivot[e];
    s1[e] = ok ? rest : s1[e];
    s2[e] = ok ? fmaxf(sq, 0.f) : s2[e];
  }
}

// Each tile's statistics. A lane takes its channels' sums about the first value that it sees of
// each and, from its 4th, 16th, 64th .. row on, about the mean of those before: so its sum of
// squares is at most 4 times that about its own mean, whatever the values. (About the first
// one throughout it would be up to n times that: with 1,500 equal values behind another one the
// variance was 3 % off.) The work-group takes the groups' means and then the sums of
// squares about those.
template <int DT, bool TINY>
__global__ void __launch_bounds__(kGnThreads) gn_fwd_sums_kernel(GnFwd p) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, U = 4;
  __shared__ float cols[kGnThreads * VE], sums[2][kGnThreads];
  const GnShape& s = p.s;
  const GnAt wg(s, blockIdx.x, false);
  const GnBlock blk(s, wg.block);
  const GnLane<DT, TINY> ln(s, blk.cb);
  const GnTiles tiles(s, ln.rp);
  const int64_t ld = (int64_t)s.C * ES, step = (int64_t)ln.rp * s.tiles * ld;
  const int n = tiles.rows_of(wg.tile, ln.r, ln.rp);
  const char* x = p.x + ((int64_t)wg.image * s.L + (int64_t)ln.rp * wg.tile + ln.r) * ld + (int64_t)blk.c0 * ES;
  float pivot[VE], s1[VE], s2[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) pivot[e] = s1[e] = s2[e] = 0.f;
  if (n > 0) {
    for (int i = 0, move = U; i < n; i += U) {
      Vec16 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = ln.k.load(x + min(i + u, n - 1) * step);
      if (i == 0) ln.k.unpack(v[0], pivot);
      if (i == move) {
        gn_about_mean((float)i, pivot, s1, s2);
        move *= 4;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u < n) {
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
  }
  const float cnt = (float)n, inv = n ? 1.f / cnt : 0.f, all = (float)tiles.rows(wg.tile, ln.rp) * (float)blk.width;
  float v[VE], mean[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    mean[e] = fmaf(s1[e], inv, pivot[e]);
    s2[e] = fmaf(-s1[e] * inv, s1[e], s2[e]);
    s2[e] = s2[e] < 0.f ? 0.f : s2[e];  // (a NaN stays)
    v[e] = fmaf(cnt, pivot[e], s1[e]);
  }
  gn_group_sums<DT, TINY>(s, blk, v, all, cols, sums[0]);
  int gi[VE];
  ln.groups(s, blk, gi);
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    const float d = mean[e] - sums[0][gi[e]];
    v[e] = fmaf(cnt * d, d, s2[e]);
  }
  gn_group_sums<DT, TINY>(s, blk, v, 1.f, cols, sums[1]);
  if ((int)threadIdx.x < blk.ng)
    p.part[(((int64_t)wg.image * s.tiles + wg.tile) * s.pieces + blk.piece) * s.G + blk.g0 + threadIdx.x] =
        float2{sums[0][threadIdx.x], sums[1][threadIdx.x]};
}

// The groups' statistics of an image from its tiles', and a tile's rows.
template <int DT, bool TINY>
__global__ void __launch_bounds__(kGnThreads) gn_fwd_rows_kernel(GnFwd p) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, U = 4;
  __shared__ float smean[kGnThreads], srstd[kGnThreads];
  const GnShape& s = p.s;
  const GnAt wg(s, blockIdx.x, true);
  const GnBlock blk(s, wg.block);
  const GnLane<DT, TINY> ln(s, blk.cb);
  const GnTiles tiles(s, ln.rp);
  const int64_t ld = (int64_t)s.C * ES, step = (int64_t)ln.rp * s.tiles * ld;
  const int n = tiles.rows_of(wg.tile, ln.r, ln.rp);
  const int64_t at = ((int64_t)wg.image * s.L + (int64_t)ln.rp * wg.tile + ln.r) * ld + (int64_t)blk.c0 * ES;
  // the first rows are on their way while the statistics are put together
  Vec16 v[U];
  auto fetch = [&](int i) {
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = ln.k.load(p.x + at + min(i + u, n - 1) * step);
  };
  if (n > 0) fetch(0);
  {
    const int g = threadIdx.x >> s.tshift, i = threadIdx.x & (s.team - 1), entries = s.tiles * s.pieces;
    GnStat st = {0.f, 0.f, 0.f};
    if (g < blk.ng) {
      const float2* q = p.part + (int64_t)wg.image * entries * s.G + blk.g0 + g;
#pragma unroll 4
      for (int j = i; j < entries; j += s.team) {
        const float2 v = q[(int64_t)j * s.G];
        const int tile = s.pieces == 1 ? j : gn_div(j, s.inv_pieces), piece = s.pieces == 1 ? 0 : j - tile * s.pieces;
        const int width = s.pieces == 1 ? s.Cg : min(s.pw, s.Cg - piece * s.pw);
        st.join((float)tiles.rows(tile, ln.rp) * (float)width, v.x, v.y);
      }
    }
    for (int o = 1; o < s.team; o <<= 1) st.join_across(o);
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
  if (ln.k.skip == VE || n <= 0) return;
  int gi[VE];
  ln.groups(s, blk, gi);
  float mean[VE], w[VE], b[VE];
  ln.k.load_f32(p.w ? p.w + blk.c0 : nullptr, 1.f, w);
  ln.k.load_f32(p.b ? p.b + blk.c0 : nullptr, 0.f, b);
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    mean[e] = smean[gi[e]];
    w[e] *= srstd[gi[e]];
  }
  gn_by_act(p.act, [&](auto act) {
    for (int i = 0; i < n; i += U) {
      if (i) fetch(i);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u < n) {
          float a[VE];
          ln.k.unpack(v[u], a);
#pragma unroll
          for (int e = 0; e < VE; ++e) a[e] = act.value(fmaf(a[e] - mean[e], w[e], b[e]));
          ln.k.store(p.y + at + (i + u) * step, a);
        }
      }
    }
  });
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
  int64_t sums;  // partial sums of a column
};

// A lane's constants of an image: its channels' statistics and affine weights.
template <int DT, bool TINY>
struct GnConst {
  static constexpr int VE = Ln<DT>::VE;
  float mean[VE], rs[VE], w[VE], b[VE];
  __device__ __forceinline__ GnConst(const GnBwd& p, const GnBlock& blk, const GnLane<DT, TINY>& ln, int image) {
    int gi[VE];
    ln.groups(p.s, blk, gi);
    ln.k.load_f32(p.w ? p.w + blk.c0 : nullptr, 1.f, w);
    ln.k.load_f32(p.b ? p.b + blk.c0 : nullptr, 0.f, b);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const int64_t g = (int64_t)image * p.s.G + blk.g0 + gi[e];
      mean[e] = p.mean[g];
      rs[e] = p.rstd[g];
    }
  }
  // xh, and du in place of dy
  template <class A>
  __device__ __forceinline__ void apply(float (&x)[VE], float (&dy)[VE], A) const {
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      x[e] = (x[e] - mean[e]) * rs[e];
      dy[e] *= A::slope(fmaf(x[e], w[e], b[e]));
    }
  }
};

// A work-group's sums of its columns (v, used up) to memory, and the groups' sums of those
// times the affine weights into sums (ends with a barrier).
template <int DT, bool TINY>
__device__ __forceinline__ void gn_bwd_column_sums(const GnBwd& p, const GnBlock& blk, float (&v)[Ln<DT>::VE], float* out,
                                                   int add, float* cols, float* sums) {
  const GnShape& s = p.s;
  gn_put<DT>(s, v, cols);
  __syncthreads();
  if (out)
    for (int c = threadIdx.x; c < blk.cb; c += blockDim.x) {
      const float a = gn_column<DT, TINY>(s, blk.cb, c, cols);
      out[blk.c0 + c] = add ? out[blk.c0 + c] + a : a;
    }
  const int g = threadIdx.x >> s.tshift, i = threadIdx.x & (s.team - 1);
  float a = 0.f;
  if (g < blk.ng)
    for (int c = i; c < blk.width; c += s.team)
      a = fmaf(gn_column<DT, TINY>(s, blk.cb, g * blk.width + c, cols), p.w ? p.w[blk.c0 + g * blk.width + c] : 1.f, a);
  a = gn_team_sum(a, s.team);
  if (g < blk.ng && i == 0) sums[g] = a;
  __syncthreads();
}
// Both of a backward pass: sx of du xh, sd of du; the groups' sums of t into s1, of t xh into s2.
template <int DT, bool TINY>
__device__ __forceinline__ void gn_bwd_sums(const GnBwd& p, const GnBlock& blk, float (&sx)[Ln<DT>::VE],
                                            float (&sd)[Ln<DT>::VE], float* out_w, float* out_b, int add, float* cols,
                                            float* s1, float* s2) {
  gn_bwd_column_sums<DT, TINY>(p, blk, sx, out_w, add, cols, s2);
  gn_bwd_column_sums<DT, TINY>(p, blk, sd, out_b, add, cols, s1);
}

// An image's block whole, as the forward pass's. With one image dw and db are its sums.
template <int DT, int NV>
__global__ void __launch_bounds__(kGnImage) gn_bwd_image_kernel(GnBwd p) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES;
  __shared__ float cols[kGnImage * VE], s1[kGnImage], s2[kGnImage];
  const GnShape& s = p.s;
  const GnAt wg(s, blockIdx.x, false);
  const GnBlock blk(s, wg.block);
  const GnLane<DT, false> ln(s, blk.cb);
  const int64_t ld = (int64_t)s.C * ES, at = (int64_t)wg.image * s.L * ld + (int64_t)blk.c0 * ES;
  const int L = (int)s.L;
  u32x4 vx[NV], vy[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int64_t o = at + (int64_t)min(ln.r + i * ln.rp, L - 1) * ld + ln.k.c * ES;
    vx[i] = gn_load(p.x + o);
    vy[i] = gn_load(p.dy + o);
  }
  const GnConst<DT, false> c(p, blk, ln, wg.image);
  float sx[VE], sd[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) sx[e] = sd[e] = 0.f;
  gn_by_act(p.act, [&](auto act) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float x[VE], dy[VE];
      Ln<DT>::unpack(gn_vec(vx[i]), x);
      Ln<DT>::unpack(gn_vec(vy[i]), dy);
      c.apply(x, dy, act);
      const bool in = ln.r + i * ln.rp < L;
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        sx[e] = in ? fmaf(dy[e], x[e], sx[e]) : sx[e];
        sd[e] += in ? dy[e] : 0.f;
      }
      gn_next();
    }
  });
  gn_packed(vx);
  gn_packed(vy);
  float* out = p.wpart ? p.wpart + (int64_t)wg.image * 2 * s.C : nullptr;
  gn_bwd_sums<DT, false>(p, blk, sx, sd, out ? out : p.dw, out ? out + s.C : p.db, out ? 0 : p.accumulate, cols, s1, s2);
  if (!p.dx || ln.k.skip == VE) return;
  int gi[VE];
  ln.groups(s, blk, gi);
  const float inv = 1.f / ((float)L * (float)s.Cg);
  float m1[VE], m2[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    m1[e] = s1[gi[e]] * inv;
    m2[e] = s2[gi[e]] * inv;
  }
  gn_by_act(p.act, [&](auto act) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (ln.r + i * ln.rp < L) {
        const int64_t o = at + (int64_t)(ln.r + i * ln.rp) * ld;
        float x[VE], dy[VE];
        Ln<DT>::unpack(gn_vec(vx[i]), x);
        Ln<DT>::unpack(gn_vec(vy[i]), dy);
        c.apply(x, dy, act);
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
      gn_next();
    }
  });
}

template <int DT, bool TINY>
__global__ void __launch_bounds__(kGnThreads) gn_bwd_sums_kernel(GnBwd p) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, U = 4;
  __shared__ float cols[kGnThreads * VE], s1[kGnThreads], s2[kGnThreads];
  const GnShape& s = p.s;
  const GnAt wg(s, blockIdx.x, false);
  const GnBlock blk(s, wg.block);
  const GnLane<DT, TINY> ln(s, blk.cb);
  const GnTiles tiles(s, ln.rp);
  const int64_t ld = (int64_t)s.C * ES, step = (int64_t)ln.rp * s.tiles * ld;
  const int n = tiles.rows_of(wg.tile, ln.r, ln.rp);
  const int64_t at = ((int64_t)wg.image * s.L + (int64_t)ln.rp * wg.tile + ln.r) * ld + (int64_t)blk.c0 * ES;
  float sx[VE], sd[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) sx[e] = sd[e] = 0.f;
  if (n > 0) {
    const GnConst<DT, TINY> c(p, blk, ln, wg.image);
    gn_by_act(p.act, [&](auto act) {
      for (int i = 0; i < n; i += U) {
        Vec16 vx[U], vy[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t o = at + min(i + u, n - 1) * step;
          vx[u] = ln.k.load(p.x + o);
          vy[u] = ln.k.load(p.dy + o);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (i + u < n) {
            float x[VE], dy[VE];
            Ln<DT>::unpack(vx[u], x);
            Ln<DT>::unpack(vy[u], dy);
            c.apply(x, dy, act);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
              sx[e] = fmaf(dy[e], x[e], sx[e]);
              sd[e] += dy[e];
            }
          }
        }
      }
    });
  }
  const int64_t tile = (int64_t)wg.image * s.tiles + wg.tile;
  float* out = p.wpart ? p.wpart + tile * 2 * s.C : nullptr;
  gn_bwd_sums<DT, TINY>(p, blk, sx, sd, out, out ? out + s.C : nullptr, 0, cols, s1, s2);
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
__global__ void __launch_bounds__(kGnThreads) gn_reduce_kernel(GnBwd p) { gn_reduce(p, p.sums, blockIdx.x); }

template <int DT, bool TINY>
__global__ void __launch_bounds__(kGnThreads) gn_bwd_rows_kernel(GnBwd p) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, U = 2;
  __shared__ float s1[kGnThreads], s2[kGnThreads];
  const GnShape& s = p.s;
  const unsigned tiles = (unsigned)s.B * s.tiles * s.blocks;
  if (blockIdx.x >= tiles) return gn_reduce(p, p.sums, (int)(blockIdx.x - tiles));  // (behind the rows)
  const GnAt wg(s, blockIdx.x, true);
  const GnBlock blk(s, wg.block);
  const GnLane<DT, TINY> ln(s, blk.cb);
  const GnTiles at_tiles(s, ln.rp);
  const int64_t ld = (int64_t)s.C * ES, step = (int64_t)ln.rp * s.tiles * ld;
  const int n = at_tiles.rows_of(wg.tile, ln.r, ln.rp);
  const int64_t at = ((int64_t)wg.image * s.L + (int64_t)ln.rp * wg.tile + ln.r) * ld + (int64_t)blk.c0 * ES;
  // the first rows are on their way while the sums are put together
  Vec16 vx[U], vy[U], vr[U];
  auto fetch = [&](int i) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t o = at + min(i + u, n - 1) * step;
      vx[u] = ln.k.load(p.x + o);
      vy[u] = ln.k.load(p.dy + o);
      if (p.dres) vr[u] = ln.k.load(p.dres + o);
    }
  };
  if (n > 0) fetch(0);
  const float all = (float)(int)s.L * (float)s.Cg;
  {
    const int g = threadIdx.x >> s.tshift, i = threadIdx.x & (s.team - 1), entries = s.tiles * s.pieces;
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
    a = gn_team_sum(a, s.team);
    b = gn_team_sum(b, s.team);
    if (g < blk.ng && i == 0) {
      s1[g] = a / all;
      s2[g] = b / all;
    }
    __syncthreads();
  }
  if (ln.k.skip == VE || n <= 0) return;
  const GnConst<DT, TINY> c(p, blk, ln, wg.image);
  int gi[VE];
  ln.groups(s, blk, gi);
  float m1[VE], m2[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    m1[e] = s1[gi[e]];
    m2[e] = s2[gi[e]];
  }
  gn_by_act(p.act, [&](auto act) {
    for (int i = 0; i < n; i += U) {
      if (i) fetch(i);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u < n) {
          float x[VE], dy[VE];
          Ln<DT>::unpack(vx[u], x);
          Ln<DT>::unpack(vy[u], dy);
          c.apply(x, dy, act);
#pragma unroll
          for (int e = 0; e < VE; ++e) dy[e] = c.rs[e] * (fmaf(dy[e], c.w[e], -m1[e]) - x[e] * m2[e]);
          if (p.dres) {
            float z[VE];
            Ln<DT>::unpack(vr[u], z);
#pragma unroll
            for (int e = 0; e < VE; ++e) dy[e] += z[e];
          }
          ln.k.store(p.dx + at + (i + u) * step, dy);
        }
      }
    }
  });
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
static int pow2_from(int64_t n) {
  int p = 1;
  while (p < n) p *= 2;
  return p;
}

// kg groups per block, the last block at least a vector wide (the groups that this moves to
// the others never make them wider than kg whole groups were allowed to be).
static void gn_blocks(GnShape* s, int64_t kg, int VE) {
  int64_t nb = up(s->G, kg);
  kg = up(s->G, nb);
  while (kg < s->G && (s->G - (up(s->G, kg) - 1) * kg) * s->Cg < VE) ++kg;
  s->kg = (int)kg;
  s->pieces = 1;
  s->pw = s->Cg;
  s->blocks = (int)up(s->G, kg);
}
static void gn_lanes(GnShape* s, int threads, int VE) {
  const int width = s->pieces == 1 ? s->Cg : s->pw;
  s->nl = pow2_from(up((int64_t)s->kg * width, VE));
  s->shift = 0;
  while (1 << s->shift < s->nl) ++s->shift;
  s->team = 1;
  s->tshift = 0;
  while (s->team < 64 && s->team < width && s->team * 2 * s->kg <= threads) {
    s->team *= 2;
    ++s->tshift;
  }
  s->inv_width = 1.f / (float)width;
  s->inv_pieces = 1.f / (float)s->pieces;
}

// An image's block in the registers of one work-group, with blocks of 32 bytes per row or
// more: where the whole batch is small, and a thread has few vectors (4 forward; backward 2,
// with 4 the registers do not hold them), one launch is sooner than two. Us of launches one
// after the other, forward and backward, in one / in two: 1 x 64 x 256 fp16 5.7 / 9.4, 5.9 /
// 11.7; 1 x 256 x 192 8.4 / 9.6, 9.2 / 12.1; 8 x 256 x 384 9.0 / 10.7, 11.7 / 13.4; 1 x 784 x
// 256 9.3 / 11.0, 11.1 / 12.8; 8 x 784 x 256 10.4 / 11.5, 15.2 / 13.7; 1 x 1600 x 512 11.5 /
// 11.6, 25.3 / 14.5; 32 x 256 x 384 15.8 / 13.1, 26.2 / 18.5; 256 x 256 x 384 83 / 38, 156 / 66.
static bool gn_image(GnPlan* p, bool bwd, int dt) {
  constexpr int bytes = 32;
  const int most = bwd ? 2 : 4;
  if ((int64_t)p->s.B * p->s.L > ((int64_t)1 << (bwd ? 20 : 21)) / p->s.C) return false;
  const int VE = dt == GTR_F32 ? 4 : 8, ES = dt == GTR_F32 ? 4 : 2;
  GnShape* s = &p->s;
  gn_blocks(s, up(bytes, (int64_t)s->Cg * ES), VE);
  if (s->kg > 64 || (int64_t)s->kg * s->Cg > 64 * VE) return false;
  gn_lanes(s, kGnImage, VE);
  const int64_t nl = s->nl;
  if (s->L > kGnImage / nl * most) return false;
  p->threads = (int)(s->L * nl >= kGnImage ? kGnImage : up(s->L * nl, 64) * 64);
  gn_lanes(s, p->threads, VE);
  p->NV = pow2_from(up(s->L, p->threads / nl));
  s->tiles = 1;
  p->grid = (int64_t)s->B * s->blocks;
  return p->NV <= most && p->grid * p->threads < (int64_t)1 << 32;
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
  if (!p->tiny && gn_image(p, bwd, dt)) return GTR_OK;
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
  gn_lanes(s, kGnThreads, VE);
  const int64_t rp = kGnThreads / s->nl;
  // Up to 8 work-groups per CU and 8 rows per thread or more, for the most part (8 x 1600 x 384
  // fp16 forward 17.1 us, with 4 rows 21.7; 16 x 16384 x 512 bf16 in 512, 1024, 2048 work-groups
  // 186, 181, 160, backward of 16 x 4096 x 1024 151, 142, 134, of the same inputs each time).
  const int64_t chains = (int64_t)B * s->blocks;
  int64_t tiles = std::min(up(2048, chains), up(L, rp * 8));
  if (tiles * chains < 256) tiles = std::min(up(256, chains), up(L, rp * 4));
  s->tiles = (int)std::min<int64_t>(tiles, 256);
  p->grid = (int64_t)B * s->tiles * s->blocks;
  return (p->grid + up(2 * (int64_t)C, 32)) * kGnThreads < (int64_t)1 << 32 ? GTR_OK : GTR_ERR_SHAPE;
}

// Bytes of workspace: the tiles' sums, and the columns' partial sums.
static size_t gn_stats_bytes(const GnPlan& p) {
  return p.NV ? 0 : (size_t)up((int64_t)p.s.B * p.s.tiles * p.s.pieces * p.s.G * 8, 256) * 256;
}
static size_t gn_weights_bytes(const GnPlan& p) {
  return p.NV && p.s.B == 1 ? 0 : (size_t)up((int64_t)p.s.B * p.s.tiles * 2 * p.s.C * 4, 256) * 256;
}

template <int DT, int NV>
static void gn_go_image(const GnPlan& p, const GnFwd& f, hipStream_t st) {
  hipLaunchKernelGGL((gn_fwd_image_kernel<DT, NV>), dim3((unsigned)p.grid), dim3(p.threads), 0, st, f);
}
template <int DT, int NV>
static void gn_go_image(const GnPlan& p, const GnBwd& f, hipStream_t st) {
  hipLaunchKernelGGL((gn_bwd_image_kernel<DT, NV>), dim3((unsigned)p.grid), dim3(p.threads), 0, st, f);
}
template <int DT, bool TINY>
static void gn_go_tiles(const GnPlan& p, const GnFwd& f, hipStream_t st) {
  const dim3 g((unsigned)p.grid), t(kGnThreads);
  hipLaunchKernelGGL((gn_fwd_sums_kernel<DT, TINY>), g, t, 0, st, f);
  hipLaunchKernelGGL((gn_fwd_rows_kernel<DT, TINY>), g, t, 0, st, f);
}
static unsigned gn_sums_grid(const GnBwd& f) { return f.wpart ? (unsigned)up(2 * (int64_t)f.s.C, 32) : 0; }
template <int DT, bool TINY>
static void gn_go_tiles(const GnPlan& p, const GnBwd& f, hipStream_t st) {
  const dim3 g((unsigned)p.grid), t(kGnThreads);
  hipLaunchKernelGGL((gn_bwd_sums_kernel<DT, TINY>), g, t, 0, st, f);
  if (f.dx) hipLaunchKernelGGL((gn_bwd_rows_kernel<DT, TINY>), dim3(g.x + gn_sums_grid(f)), t, 0, st, f);
}
template <int DT, class F>
static void gn_go(const GnPlan& p, const F& f, hipStream_t st) {
  switch (p.NV) {
    case 0: return p.tiny ? gn_go_tiles<DT, true>(p, f, st) : gn_go_tiles<DT, false>(p, f, st);
    case 1: return gn_go_image<DT, 1>(p, f, st);
    case 2: return gn_go_image<DT, 2>(p, f, st);
    default:
      if constexpr (std::is_same<F, GnFwd>::value) gn_go_image<DT, 4>(p, f, st);
  }
}
template <class F>
static void gn_launch(int dt, const GnPlan& p, const F& f, hipStream_t st) {
  if (dt == GTR_F32)
    gn_go<GTR_F32>(p, f, st);
  else if (dt == GTR_F16)
    gn_go<GTR_F16>(p, f, st);
  else
    gn_go<GTR_BF16>(p, f, st);
}
static gtr_status gn_launched() { return hipGetLastError() == hipSuccess ? GTR_OK : GTR_ERR_HIP; }

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
  gn_launch(a->dtype, p, f, stream);
  return gn_launched();
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
                   sums ? reinterpret_cast<float*>(ws + stat) : nullptr, a->dw, a->db, a->accumulate, a->act,
                   (int64_t)p.s.B * p.s.tiles};
  gn_launch(a->dtype, p, f, stream);
  // the columns' sums, where they are not the rows' launch's
  if (f.wpart && (p.NV || !f.dx))
    hipLaunchKernelGGL(gn_reduce_kernel, dim3(gn_sums_grid(f)), dim3(kGnThreads), 0, stream, f);
  return gn_launched();
}
