// Layer normalisation for training: the forward pass that also leaves the rows'
// statistics, and the backward pass with the reduction of the affine weights'
// gradients. Per row of d channels, in float32:
//
//   forward:  mean = sum x / d,  rstd = (sum (x - mean)^2 / d + eps)^(-1/2),
//             y = (x - mean) rstd w + b
//   backward: xh = (x - mean) rstd,  t = dy w,
//             dx = rstd (t - sum t / d - xh sum (t xh) / d) (+ dres)
//             dw = sum over the rows of dy xh,  db = sum over the rows of dy
//
// What bounds both is memory: each reads its rows once and writes them once (calls one
// after the other, of new inputs: 32768 x 4096 bf16 forward 103 us, 5.2 TB/s; 16384 x
// 4096 bf16 backward with a residual 98 us, 5.5 TB/s; a large copy reaches 5.1), and for
// short batches the launches. A
// row lives in the registers of the lanes that share it (so the forward pass
// takes the squares about the mean, with no second read), in 16-byte vectors at
// whatever address the row starts: the vector loads and stores of this machine
// need no alignment beyond an element's.
#include <hip/hip_runtime.h>

#include "gtr.h"
#include "gtr_device.h"
#include "gtr_internal.h"
#include "vec_rows.h"

namespace gtr {

// A row is shared by T lanes: 16, 32 or 64 of a wave, or (T = 0) by all of a work-group
// of up to 1024. Sums of N values over them, in every one of them. For T = 0 the waves'
// sums meet in `part`, which holds a slot per wave and value and is not written again
// before the next barrier but one.
constexpr int kLnWaves = 16;
template <int T, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float (*part)[T ? 1 : kLnWaves]) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    x[n] = row_bcast<15>(row_inclusive_scan(x[n]));
    if constexpr (T != 16) x[n] += __shfl_xor(x[n], 16, kWave);
    if constexpr (T != 16 && T != 32) x[n] += __shfl_xor(x[n], 32, kWave);
  }
  if constexpr (T == 0) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) part[n][threadIdx.x >> 6] = x[n];
    __syncthreads();
    const int waves = blockDim.x >> 6;
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = 0.f;
    for (int w = 0; w < waves; ++w)
#pragma unroll
      for (int n = 0; n < N; ++n) x[n] += part[n][w];
  }
}

struct LnFwd {
  const char* x;
  const float *w, *b;
  char* y;
  float *mean, *rstd;
  int64_t M;
  int d;
  float eps;
};

// NV vectors per lane. A work-group takes the rows r = its index, + the grid, ..
// (256 / T of them at a time, one if T is 0), keeps the affine weights in registers
// between its rows (for each row they are four times its bytes, from cache) and has the
// next row on its way while it works on one (AHEAD: where that fits the registers).
// One vector per lane takes at most 64 registers: two work-groups of 16 waves per CU
// (8192 x 8192 bf16: 64.5 us, with one 80.5).
template <int DT, int T, int NV, bool TINY>
__global__ void __launch_bounds__(T ? 256 : 64 * kLnWaves) __attribute__((amdgpu_waves_per_eu(NV == 1 ? 8 : 4)))
ln_fwd_kernel(LnFwd g) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, R = T ? 256 / (T ? T : 1) : 1;
  constexpr bool AHEAD = T || NV == 1;
  const int TT = T ? T : blockDim.x;
  __shared__ float part[2][2][T ? 1 : kLnWaves];
  const int l = T ? threadIdx.x % (T ? T : 1) : threadIdx.x, d = g.d;
  const int64_t step = (int64_t)gridDim.x * R;
  int64_t row = (int64_t)blockIdx.x * R + (T ? threadIdx.x / (T ? T : 1) : 0);
  if (row >= g.M) return;  // (T = 0: all threads of the work-group or none, here and in the loop)
  Vec16 next[NV];
  auto fetch = [&](int64_t r) {
#pragma unroll
    for (int q = 0; q < NV; ++q) next[q] = LnCols<DT, TINY>(l + TT * q, d).load(g.x + r * d * ES);
  };
  if (AHEAD) fetch(row);
  float wv[NV][VE], bv[NV][VE];
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    const LnCols<DT, TINY> k(l + TT * q, d);
    k.load_f32(g.w, 1.f, wv[q]);
    k.load_f32(g.b, 0.f, bv[q]);
  }
  const float dn = (float)d;
  for (int flip = 0; row < g.M; row += step, flip ^= 1) {
    float v[NV][VE], s[1] = {0.f};
    if (!AHEAD) fetch(row);
#pragma unroll
    for (int q = 0; q < NV; ++q) LnCols<DT, TINY>(l + TT * q, d).unpack(next[q], v[q]);
    if (AHEAD && row + step < g.M) fetch(row + step);
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
      for (int e = 0; e < VE; ++e) s[0] += v[q][e];
    row_sums<T, 1>(s, &part[flip][0]);
    const float mean = s[0] / dn;  // (a quotient, not a product with 1 / d: the mean of equal values is theirs)
    s[0] = 0.f;
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const LnCols<DT, TINY> k(l + TT * q, d);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        v[q][e] -= mean;
        const float u = k.has(e) ? v[q][e] : 0.f;
        s[0] = fmaf(u, u, s[0]);
      }
    }
    row_sums<T, 1>(s, &part[flip][1]);
    const float rs = 1.f / sqrtf(s[0] / dn + g.eps);
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      float o[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) o[e] = fmaf(v[q][e] * rs, wv[q][e], bv[q][e]);
      LnCols<DT, TINY>(l + TT * q, d).store(g.y + row * d * ES, o);
    }
    if (l == 0) {
      if (g.mean) g.mean[row] = mean;
      if (g.rstd) g.rstd[row] = rs;
    }
  }
}

struct LnBwd {
  const char *dy, *x;
  const float *mean, *rstd, *w;
  const char* dres;
  char* dx;
  float* part;  // [work-groups][2][d]: this call's sums of dy xh and of dy, or null
  int64_t M;
  int d;
  // sums by columns (ln_columns) instead of by partial sums: how many work-groups take
  // the rows, the others take the columns of dw and db
  int rows;  // 0: all of them
  float *dw, *db;
  int accumulate;
};

// Rows as in the forward pass, the sums over them of dy xh and dy in registers: each
// lane's own columns. The sums of the rows that a work-group holds at a time are then
// added in a fixed order, and one partial sum per work-group goes to memory, where
// ln_reduce_kernel adds them in a fixed order too: a call's result does not depend
// on the order in which work-groups run.
//
// A short batch's sums are cheaper the other way (g.rows): work-groups behind those of
// the rows take two vectors' columns each over all rows and read dy and x again, from
// cache, and the call is one launch.
template <int DT, bool TINY>
__device__ __forceinline__ void ln_columns(const LnBwd& g, int pair) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, U = 8;
  __shared__ float sums[kLnWaves][2][2 * VE];
  const LnCols<DT, TINY> k(2 * pair + (threadIdx.x & 1), g.d);
  const int lanes = blockDim.x / 2;  // rows at a time
  const int64_t at = (int64_t)g.d * ES;
  float a[2 * VE];  // sums of dy xh, of dy
#pragma unroll
  for (int e = 0; e < 2 * VE; ++e) a[e] = 0.f;
  for (int64_t r0 = threadIdx.x >> 1; r0 < g.M; r0 += U * lanes) {
    Vec16 vy[U], vx[U];
    float mean[U], rs[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = r0 + u * lanes < g.M ? r0 + u * lanes : r0;
      vy[u] = k.load(g.dy + r * at);
      vx[u] = k.load(g.x + r * at);
      mean[u] = g.mean[r];
      rs[u] = g.rstd[r];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r0 + u * lanes >= g.M) continue;
      float y[VE], h[VE];
      k.unpack(vy[u], y);
      Ln<DT>::unpack(vx[u], h);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        a[e] = fmaf(y[e], (h[e] - mean[u]) * rs[u], a[e]);
        a[VE + e] += y[e];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 2 * VE; ++e) {
#pragma unroll
    for (int o = 2; o < 64; o <<= 1) a[e] += __shfl_xor(a[e], o, kWave);
    if ((threadIdx.x & 63) < 2) sums[threadIdx.x >> 6][threadIdx.x & 1][e] = a[e];
  }
  __syncthreads();
  if (threadIdx.x >= 4 * VE) return;
  const int v = threadIdx.x / (2 * VE), e = threadIdx.x % (2 * VE);
  const LnCols<DT, TINY> kv(2 * pair + v, g.d);
  float t = 0.f;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) t += sums[w][v][e];
  float* out = e < VE ? g.dw : g.db;
  const int c = kv.c + e % VE;
  if (out && kv.has(e % VE)) out[c] = g.accumulate ? out[c] + t : t;
}

template <int DT, int T, int NV, bool TINY>
__global__ void __launch_bounds__(T ? 256 : 64 * kLnWaves) ln_bwd_kernel(LnBwd g) {
  if (g.rows && (int)blockIdx.x >= g.rows) return ln_columns<DT, TINY>(g, blockIdx.x - g.rows);
  if (g.rows && !g.dx) return;
  const int groups = g.rows ? g.rows : gridDim.x;
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, R = T ? 256 / (T ? T : 1) : 1;
  constexpr bool AHEAD = T || NV == 1;
  const int TT = T ? T : blockDim.x;
  __shared__ float part[2][2][T ? 1 : kLnWaves];
  __shared__ float cols[R > 1 ? 2 * T * NV * VE : 1];
  const int l = T ? threadIdx.x % (T ? T : 1) : threadIdx.x, grp = T ? threadIdx.x / (T ? T : 1) : 0, d = g.d;
  const int64_t step = (int64_t)groups * R;
  int64_t row = (int64_t)blockIdx.x * R + grp;
  float wv[NV][VE], aw[NV][VE], ab[NV][VE];
  Vec16 ny[NV], nx[NV], nr[NV];
  float nm = 0.f, ns = 0.f;
  auto fetch = [&](int64_t r) {
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const LnCols<DT, TINY> k(l + TT * q, d);
      ny[q] = k.load(g.dy + r * d * ES);
      nx[q] = k.load(g.x + r * d * ES);
      if (g.dres) nr[q] = k.load(g.dres + r * d * ES);
    }
    nm = g.mean[r];
    ns = g.rstd[r];
  };
  if (AHEAD && row < g.M) fetch(row);
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    LnCols<DT, TINY>(l + TT * q, d).load_f32(g.w, 1.f, wv[q]);
#pragma unroll
    for (int e = 0; e < VE; ++e) aw[q][e] = ab[q][e] = 0.f;
  }
  const float inv = 1.f / (float)d;
  for (int flip = 0; row < g.M; row += step, flip ^= 1) {  // (T = 0: all threads of the work-group or none)
    float y[NV][VE], h[NV][VE];
    Vec16 r[NV];
    if (!AHEAD) fetch(row);
    const float mean = nm, rs = ns;
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      LnCols<DT, TINY>(l + TT * q, d).unpack(ny[q], y[q]);
      Ln<DT>::unpack(nx[q], h[q]);
      r[q] = nr[q];
    }
    if (AHEAD && row + step < g.M) fetch(row + step);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        h[q][e] = (h[q][e] - mean) * rs;  // (of a skipped column dy is 0: every sum gets 0 there)
        aw[q][e] = fmaf(y[q][e], h[q][e], aw[q][e]);
        ab[q][e] += y[q][e];
        y[q][e] *= wv[q][e];
        s[0] += y[q][e];
        s[1] = fmaf(y[q][e], h[q][e], s[1]);
      }
    if (g.dx) {
      row_sums<T, 2>(s, part[flip]);
      const float m1 = s[0] * inv, m2 = s[1] * inv;
#pragma unroll
      for (int q = 0; q < NV; ++q) {
        float o[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) o[e] = rs * (y[q][e] - m1 - h[q][e] * m2);
        if (g.dres) {
          float z[VE];
          Ln<DT>::unpack(r[q], z);
#pragma unroll
          for (int e = 0; e < VE; ++e) o[e] += z[e];
        }
        LnCols<DT, TINY>(l + TT * q, d).store(g.dx + row * d * ES, o);
      }
    }
  }
  if (!g.part) return;
  float* out = g.part + (int64_t)blockIdx.x * 2 * d;
  if constexpr (R > 1) {
#pragma unroll 1
    for (int r = 0; r < R; ++r) {  // the groups add their sums one after the other
      if (grp == r) {
#pragma unroll
        for (int q = 0; q < NV; ++q)
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const int c = (l + T * q) * VE + e;
            if (r) {
              aw[q][e] += cols[2 * c];
              ab[q][e] += cols[2 * c + 1];
            }
            cols[2 * c] = aw[q][e];
            cols[2 * c + 1] = ab[q][e];
          }
      }
      __syncthreads();
    }
    // place c of `cols` is a lane's element, which the row's last vector has later
    for (int c = threadIdx.x; c < d; c += 256) {
      const int last = (d - 1) / VE * VE, at = !TINY && c >= last ? c + (last + VE - d) : c;
      out[c] = cols[2 * at];
      out[d + c] = cols[2 * at + 1];
    }
  } else {
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const LnCols<DT, TINY> k(l + TT * q, d);
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (k.has(e)) {
          out[k.c + e] = aw[q][e];
          out[d + k.c + e] = ab[q][e];
        }
    }
  }
}

// dw and db from the G partial sums: 32 columns per work-group, 32 threads per
// column that take every 32nd partial sum.
__global__ void __launch_bounds__(1024) ln_reduce_kernel(const float* __restrict__ part, int G, int d, float* dw,
                                                         float* db, int accumulate) {
  __shared__ float s[32][33];
  const int cl = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + cl, n = 2 * (int64_t)d;
  float a = 0.f;
  if (c < n) {
#pragma unroll 8
    for (int i = r; i < G; i += 32) a += part[i * n + c];
  }
  s[r][cl] = a;
  __syncthreads();
  if (r == 0 && c < n) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) t += s[i][cl];
    float* out = c < d ? dw : db;
    const int64_t o = c < d ? c : c - d;
    if (out) out[o] = accumulate ? out[o] + t : t;
  }
}

// How a row is shared: by the fewest lanes of a wave that hold it with one vector each,
// a wave with two (no barrier: 25,600 x 768 bf16 backward 26.5 us against 39.2 as two
// waves), the fewest waves of a work-group, or all 16 with more vectors.
constexpr int kLnMaxWidth = 16384;
struct LnShape {
  int T, threads, NV;  // template arguments T and NV, the work-group's size
  bool tiny;
};
static LnShape ln_shape(int d, int dt) {
  const int VE = dt == GTR_F32 ? 4 : 8, n = (d + VE - 1) / VE;
  for (int T : {16, 32, 64})
    if (n <= T) return {T, 256, 1, d < VE};
  if (n <= 128) return {64, 256, 2, false};
  const int nv = (n + 1023) / 1024, lanes = (n + nv - 1) / nv;
  return {0, (lanes + 63) / 64 * 64, nv, false};
}
static int ln_rows(const LnShape& s) { return s.T ? 256 / s.T : 1; }  // of a work-group at a time

// Work-groups of the forward pass: up to 32 waves' per CU four times over. So a batch of
// up to 32768 rows of a wave each has one row per wave, and longer ones share the weights.
// Us of launches one after the other, with these, half, a quarter, an eighth of them:
// 12800 x 384 fp16 6.9, 7.0, 6.9, 7.4; 40000 x 384 fp16 17.7, 17.3, 18.1, 19.6; 30000 x
// 1000 float32 47.4, 48.7, 49.0, 53.9; 32768 x 4096 bf16 103, 108, 112, 118 (with one row
// each 173); but wider rows take less with fewer: 8192 x 8192 bf16 66, 60, 56, 73; 4096 x
// 16384 bf16 74, 66, 62, 60.
static int64_t ln_fwd_groups(int64_t M, const LnShape& s) {
  const int R = ln_rows(s);
  const int64_t all = (M + R - 1) / R, most = 256 * 8192 / s.threads;
  return all < most ? all : most;
}
// Work-groups of the backward pass: 8 waves per CU, which have 6 KB of a 4096-wide
// row's operands each on their way (16384 x 4096 bf16 with a residual: 97 us; with
// twice as many 111, with four times 118, each costing a partial sum); at least 8 rows
// per slot above 256 work-groups, which a short batch needs to fill the chip.
static int64_t ln_bwd_groups(int64_t M, const LnShape& s) {
  const int R = ln_rows(s);
  const int64_t all = (M + R - 1) / R, most = 256 * 512 / s.threads;
  int64_t g = all / 8;
  g = g > most ? most : g;
  g = g < 256 ? 256 : g;
  return g < all ? g : all;
}

// Work-groups that take the columns: two vectors each.
static int ln_column_groups(int d, int dt) {
  const int VE = dt == GTR_F32 ? 4 : 8;
  return (d + 2 * VE - 1) / (2 * VE);
}
// Whether dw and db are summed by columns: where that is sooner for calls one after the
// other, which are paced by the host, by one launch or two (8.5 and 12.9 us), and dx does
// not overwrite what is read. Work-groups that share the columns read every row, so it
// takes longer with the rows (a round of loads per 8) and with the elements: M (d + 540).
// Measured at 32 widths of two types (and 12 of the third, bf16, like fp16) on both sides,
// the two ways are even, in millions of that, at
//   rows of a wave, one vector per lane   fp16 1.2 (unaligned rows) to 2.1, float32 1.8 to 2.0
//   rows of a wave, two vectors           fp16 1.6 to 1.8, float32 1.8 to 1.9
//   rows of a work-group                  fp16 1.75 up to 1536 columns, 2.3 to 3.3 beyond;
//     float32 1.5 to 2.3, and of more than 512 threads (a CU holds one such) 0.65 to 1.0
// and never, or within 3 %, where the columns are more than three rounds of work-groups that
// have a CU for themselves (float32 past 6144 columns, 16 bits past 12288). Us by columns /
// by partial sums below and above the limits taken: fp16 1333 x 300 11.8 / 13.2, 1833 x 300
// 13.8 / 12.9; 923 x 900 10.5 / 12.9, 1555 x 900 14.6 / 12.8; 772 x 2048 11.5 / 12.9, 1159 x
// 2048 15.8 / 13.7; 305 x 6000 17.4 / 19.9, 458 x 6000 21.5 / 20.1; float32 649 x 1000 8.6 /
// 13.0, 1948 x 1000 15.8 / 13.2; 482 x 2048 11.6 / 12.9, 676 x 2048 14.6 / 12.9; 161 x 4096
// 12.7 / 13.0, 215 x 4096 14.9 / 13.2; 1 x 8192 14.0 / 12.2. Recorded into a graph, where no
// host paces them, two launches are ahead from about 0.8 million on (fp16 1333 x 300 11.8 /
// 8.2, 777 x 900 9.6 / 10.9).
static int64_t ln_columns_limit(const LnShape& s, int dt) {
  if (s.T && s.NV == 1) return 1400000;
  if (!s.T && dt != GTR_F32) return 2000000;
  return s.threads > 512 ? 700000 : 1600000;
}
static bool ln_by_columns(const gtr_layernorm_bwd_args* a, const LnShape& s) {
  if (s.threads > 512 && ln_column_groups(a->d, a->dtype) > 3 * 256) return false;
  return a->M * (a->d + 540) <= ln_columns_limit(s, a->dtype) && !(a->dx && (a->dx == a->dy || a->dx == a->x));
}

template <class P>
struct LnLaunch {
  P p;
  LnShape s;
  unsigned grid;
  hipStream_t stream;
};
template <int DT, int T, int NV, bool TINY = false>
static void ln_go(const LnLaunch<LnFwd>& a) {
  hipLaunchKernelGGL((ln_fwd_kernel<DT, T, NV, TINY>), dim3(a.grid), dim3(a.s.threads), 0, a.stream, a.p);
}
template <int DT, int T, int NV, bool TINY = false>
static void ln_go(const LnLaunch<LnBwd>& a) {
  hipLaunchKernelGGL((ln_bwd_kernel<DT, T, NV, TINY>), dim3(a.grid), dim3(a.s.threads), 0, a.stream, a.p);
}
template <int DT, class L>
static void ln_launch_as(const L& a) {
  if (a.s.tiny) return ln_go<DT, 16, 1, true>(a);
  if (a.s.T == 16) return ln_go<DT, 16, 1>(a);
  if (a.s.T == 32) return ln_go<DT, 32, 1>(a);
  if (a.s.T == 64) return a.s.NV == 1 ? ln_go<DT, 64, 1>(a) : ln_go<DT, 64, 2>(a);
  if (a.s.NV == 1) return ln_go<DT, 0, 1>(a);
  if constexpr (DT == GTR_F32) {  // (4 elements per vector: up to 4 of them at the largest width)
    if (a.s.NV == 3) return ln_go<DT, 0, 3>(a);
    if (a.s.NV == 4) return ln_go<DT, 0, 4>(a);
  }
  ln_go<DT, 0, 2>(a);
}
template <class L>
static gtr_status ln_launch(int dt, const L& a) {
  if (dt == GTR_F32)
    ln_launch_as<GTR_F32>(a);
  else if (dt == GTR_F16)
    ln_launch_as<GTR_F16>(a);
  else
    ln_launch_as<GTR_BF16>(a);
  return hipGetLastError() == hipSuccess ? GTR_OK : GTR_ERR_HIP;
}

// The checks that both passes share: sizes, type.
static gtr_status ln_sizes(int64_t M, int32_t d, int dt) {
  if (M <= 0 || d <= 0) return GTR_ERR_SHAPE;
  if (d > kLnMaxWidth || (dt != GTR_F32 && dt != GTR_F16 && dt != GTR_BF16)) return GTR_ERR_UNSUPPORTED;
  if (M >= (int64_t)1 << 31) return GTR_ERR_SHAPE;
  return GTR_OK;
}
static bool ln_misaligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

static gtr_status ln_bwd_check(const gtr_layernorm_bwd_args* a, bool pointers, size_t* need) {
  *need = 0;
  if (!a) return GTR_ERR_NULL;
  const gtr_status st = ln_sizes(a->M, a->d, a->dtype);
  if (st != GTR_OK) return st;
  const LnShape s = ln_shape(a->d, a->dtype);
  *need = ((size_t)ln_bwd_groups(a->M, s) * 2 * a->d * 4 + 255) & ~(size_t)255;
  if (ln_by_columns(a, s)) *need = 0;
  if (!pointers) return GTR_OK;
  if (!a->dy || !a->x || !a->mean || !a->rstd || (!a->dx && !a->dw && !a->db)) return GTR_ERR_NULL;
  const size_t es = dtype_size(a->dtype), bytes = (size_t)a->M * a->d * es;
  if (ln_misaligned(a->dy, es) || ln_misaligned(a->x, es) || ln_misaligned(a->dres, es) || ln_misaligned(a->dx, es) ||
      ln_misaligned(a->mean, 4) || ln_misaligned(a->rstd, 4) || ln_misaligned(a->w, 4) || ln_misaligned(a->dw, 4) ||
      ln_misaligned(a->db, 4))
    return GTR_ERR_UNSUPPORTED;
  const bool sums = a->dw || a->db;
  if (sums && *need && (!a->workspace || ln_misaligned(a->workspace, 256) || a->workspace_bytes < *need))
    return GTR_ERR_WORKSPACE;
  const Bytes ins[] = {{a->dy, bytes}, {a->x, bytes}, {a->dres, bytes}, {a->mean, (size_t)a->M * 4},
                         {a->rstd, (size_t)a->M * 4}, {a->w, (size_t)a->d * 4}};
  const Bytes outs[] = {{a->dx, bytes}, {a->dw, (size_t)a->d * 4}, {a->db, (size_t)a->d * 4},
                          {sums && *need ? a->workspace : nullptr, *need}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 6; ++j)
      if (bytes_meet(outs[i], ins[j]) && !(i == 0 && j < 3 && outs[i].p == ins[j].p)) return GTR_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (bytes_meet(outs[i], outs[j])) return GTR_ERR_ALIAS;
  }
  return GTR_OK;
}

}  // namespace gtr

using namespace gtr;

extern "C" gtr_status gtr_layernorm_fwd(const gtr_layernorm_fwd_args* a, hipStream_t stream) {
  if (!a) return GTR_ERR_NULL;
  const gtr_status st = ln_sizes(a->M, a->d, a->dtype);
  if (st != GTR_OK) return st;
  if (!(a->eps >= 0.f && a->eps < 1e30f)) return GTR_ERR_UNSUPPORTED;
  if (!a->x || !a->y) return GTR_ERR_NULL;
  const size_t es = dtype_size(a->dtype), bytes = (size_t)a->M * a->d * es;
  if (ln_misaligned(a->x, es) || ln_misaligned(a->y, es) || ln_misaligned(a->w, 4) || ln_misaligned(a->b, 4) ||
      ln_misaligned(a->mean, 4) || ln_misaligned(a->rstd, 4))
    return GTR_ERR_UNSUPPORTED;
  const Bytes ins[] = {{a->x, bytes}, {a->w, (size_t)a->d * 4}, {a->b, (size_t)a->d * 4}};
  const Bytes outs[] = {{a->y, bytes}, {a->mean, (size_t)a->M * 4}, {a->rstd, (size_t)a->M * 4}};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 3; ++j)
      if (bytes_meet(outs[i], ins[j]) && !(i == 0 && j == 0 && a->x == a->y)) return GTR_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (bytes_meet(outs[i], outs[j])) return GTR_ERR_ALIAS;
  }
  const LnShape s = ln_shape(a->d, a->dtype);
  const LnFwd p = {static_cast<const char*>(a->x), a->w, a->b, static_cast<char*>(a->y), a->mean, a->rstd, a->M, a->d, a->eps};
  return ln_launch(a->dtype, LnLaunch<LnFwd>{p, s, (unsigned)ln_fwd_groups(a->M, s), stream});
}

extern "C" size_t gtr_layernorm_bwd_workspace_size(const gtr_layernorm_bwd_args* a) {
  size_t need;
  return ln_bwd_check(a, false, &need) == GTR_OK ? need : 0;
}

extern "C" gtr_status gtr_layernorm_bwd(const gtr_layernorm_bwd_args* a, hipStream_t stream) {
  size_t need;
  const gtr_status st = ln_bwd_check(a, true, &need);
  if (st != GTR_OK) return st;
  const LnShape s = ln_shape(a->d, a->dtype);
  const int64_t G = ln_bwd_groups(a->M, s);
  const bool sums = a->dw || a->db, columns = sums && ln_by_columns(a, s);
  LnBwd p = {static_cast<const char*>(a->dy), static_cast<const char*>(a->x), a->mean, a->rstd, a->w,
             static_cast<const char*>(a->dres), static_cast<char*>(a->dx),
             sums && !columns ? static_cast<float*>(a->workspace) : nullptr, a->M, a->d, 0, a->dw, a->db, a->accumulate};
  int64_t grid = G;
  if (columns) {
    // (without dx the rows have nothing to do, but a launch has a work-group for them)
    p.rows = a->dx ? (int)G : 1;
    grid = p.rows + ln_column_groups(a->d, a->dtype);
  }
  const gtr_status run = ln_launch(a->dtype, LnLaunch<LnBwd>{p, s, (unsigned)grid, stream});
  if (run != GTR_OK || !sums || columns) return run;
  hipLaunchKernelGGL(ln_reduce_kernel, dim3((unsigned)((2 * (int64_t)a->d + 31) / 32)), dim3(1024), 0, stream, p.part,
                     (int)G, a->d, a->dw, a->db, a->accumulate);
  return hipGetLastError() == hipSuccess ? GTR_OK : GTR_ERR_HIP;
}
