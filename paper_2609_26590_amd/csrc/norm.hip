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
// What bounds both is memory: each reads its rows once and writes them once. A
// row lives in the registers of the lanes that share it (so the forward pass
// takes the squares about the mean, with no second read), in 16-byte vectors at
// whatever address the row starts: the vector loads and stores of this machine
// need no alignment beyond an element's.
#include <hip/hip_runtime.h>

#include "gtr.h"
#include "gtr_device.h"
#include "gtr_internal.h"

namespace gtr {

// 16 bytes at any element address
struct __attribute__((packed, aligned(2))) Vec16 {
  unsigned u[4];
};

template <int DT>
struct Ln;
template <>
struct Ln<GTR_F32> {
  static constexpr int VE = 4, ES = 4;  // elements per vector, bytes per element
  static __device__ __forceinline__ void unpack(const Vec16& r, float* x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __builtin_bit_cast(float, r.u[e]);
  }
  static __device__ __forceinline__ Vec16 pack(const float* x) {
    Vec16 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r.u[e] = __builtin_bit_cast(unsigned, x[e]);
    return r;
  }
  static __device__ __forceinline__ float get(const char* p) { return *reinterpret_cast<const float*>(p); }
  static __device__ __forceinline__ void put(char* p, float x) { *reinterpret_cast<float*>(p) = x; }
};
template <>
struct Ln<GTR_F16> {
  static constexpr int VE = 8, ES = 2;
  static __device__ __forceinline__ void unpack(const Vec16& r, float* x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = (float)__builtin_bit_cast(_Float16, (unsigned short)(r.u[e] & 0xffffu));
      x[2 * e + 1] = (float)__builtin_bit_cast(_Float16, (unsigned short)(r.u[e] >> 16));
    }
  }
  static __device__ __forceinline__ unsigned bits(float x) {
    return __builtin_bit_cast(unsigned short, (_Float16)x);
  }
  static __device__ __forceinline__ Vec16 pack(const float* x) {
    Vec16 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r.u[e] = bits(x[2 * e]) | bits(x[2 * e + 1]) << 16;
    return r;
  }
  static __device__ __forceinline__ float get(const char* p) { return (float)*reinterpret_cast<const _Float16*>(p); }
  static __device__ __forceinline__ void put(char* p, float x) { *reinterpret_cast<_Float16*>(p) = (_Float16)x; }
};
template <>
struct Ln<GTR_BF16> {
  static constexpr int VE = 8, ES = 2;
  static __device__ __forceinline__ void unpack(const Vec16& r, float* x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __builtin_bit_cast(float, r.u[e] << 16);
      x[2 * e + 1] = __builtin_bit_cast(float, r.u[e] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ Vec16 pack(const float* x) {
    Vec16 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __bf16 lo = (__bf16)x[2 * e], hi = (__bf16)x[2 * e + 1];
      r.u[e] = __builtin_bit_cast(unsigned short, lo) | (unsigned)__builtin_bit_cast(unsigned short, hi) << 16;
    }
    return r;
  }
  static __device__ __forceinline__ float get(const char* p) {
    return bf16_bits_to_f32(*reinterpret_cast<const unsigned short*>(p));
  }
  static __device__ __forceinline__ void put(char* p, float x) {
    *reinterpret_cast<unsigned short*>(p) = f32_to_bf16_bits(x);
  }
};

// Elements c .. c + VE - 1 of a row of d (zeros past its end). The row's last
// vector may be a part of one: its elements go one by one.
template <int DT>
__device__ __forceinline__ void load_vec(const char* row, int c, int d, float (&x)[Ln<DT>::VE]) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES;
  if (c + VE <= d) {
    Ln<DT>::unpack(*reinterpret_cast<const Vec16*>(row + (int64_t)c * ES), x);
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) x[e] = c + e < d ? Ln<DT>::get(row + (int64_t)(c + e) * ES) : 0.f;
  }
}
template <int DT>
__device__ __forceinline__ void store_vec(char* row, int c, int d, const float (&x)[Ln<DT>::VE]) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES;
  if (c + VE <= d) {
    *reinterpret_cast<Vec16*>(row + (int64_t)c * ES) = Ln<DT>::pack(x);
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (c + e < d) Ln<DT>::put(row + (int64_t)(c + e) * ES, x[e]);
  }
}
// Elements c .. c + VE - 1 of a float32 vector of d, `fill` past its end or
// everywhere if there is no vector.
template <int VE>
__device__ __forceinline__ void load_f32(const float* p, int c, int d, float fill, float (&x)[VE]) {
  if (p && c + VE <= d) {
#pragma unroll
    for (int h = 0; h < VE / 4; ++h) {
      const Vec16 r = *reinterpret_cast<const Vec16*>(p + c + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * h + e] = __builtin_bit_cast(float, r.u[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) x[e] = p && c + e < d ? p[c + e] : fill;
  }
}

// Sum over the T lanes that share a row, in every one of them. For a row of a
// whole work-group (T > 64) the waves' sums meet in `part`, which holds one slot per
// wave and is not written again before the next barrier but one.
template <int T>
__device__ __forceinline__ float row_sum(float x, float* part) {
  x = row_bcast<15>(row_inclusive_scan(x));
  if constexpr (T >= 32) x += __shfl_xor(x, 16, kWave);
  if constexpr (T >= 64) x += __shfl_xor(x, 32, kWave);
  if constexpr (T > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) x += part[w];
  }
  return x;
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

// T lanes share a row, NV vectors each.
template <int DT, int T, int NV>
__global__ void __launch_bounds__(T > 64 ? T : 256) ln_fwd_kernel(LnFwd g) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, NT = T > 64 ? T : 256;
  __shared__ float part[2][T > 64 ? T / 64 : 1];
  const int64_t row = (int64_t)blockIdx.x * (NT / T) + threadIdx.x / T;
  const int l = threadIdx.x % T, d = g.d;
  if (row >= g.M) return;  // (T > 64: one row per work-group, all its threads or none)
  const char* xr = g.x + row * d * ES;
  float v[NV][VE], wv[NV][VE], bv[NV][VE];
  float s = 0.f;
#pragma unroll
  for (int q = 0; q < NV; ++q) load_vec<DT>(xr, (l + T * q) * VE, d, v[q]);
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    load_f32<VE>(g.w, (l + T * q) * VE, d, 1.f, wv[q]);
    load_f32<VE>(g.b, (l + T * q) * VE, d, 0.f, bv[q]);
  }
#pragma unroll
  for (int q = 0; q < NV; ++q)
#pragma unroll
    for (int e = 0; e < VE; ++e) s += v[q][e];
  const float mean = row_sum<T>(s, part[0]) / (float)d;
  s = 0.f;
#pragma unroll
  for (int q = 0; q < NV; ++q)
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      v[q][e] -= mean;
      if ((l + T * q) * VE + e < d) s = fmaf(v[q][e], v[q][e], s);
    }
  const float rs = 1.f / sqrtf(row_sum<T>(s, part[1]) / (float)d + g.eps);
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    float o[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) o[e] = fmaf(v[q][e] * rs, wv[q][e], bv[q][e]);
    if ((l + T * q) * VE < d) store_vec<DT>(g.y + row * d * ES, (l + T * q) * VE, d, o);
  }
  if (l == 0) {
    if (g.mean) g.mean[row] = mean;
    if (g.rstd) g.rstd[row] = rs;
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
};

// A work-group takes the rows r = its index, + the grid, .. (NT / T of them at a
// time) and keeps the sums over its rows of dy xh and dy in registers: each
// lane's own columns. The sums of the rows it holds at a time are then added in a
// fixed order, and one partial sum per work-group goes to memory, where
// ln_reduce_kernel adds them in a fixed order too: a call's result does not
// depend on the order in which work-groups run.
template <int DT, int T, int NV>
__global__ void __launch_bounds__(T > 64 ? T : 256) ln_bwd_kernel(LnBwd g) {
  constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES, NT = T > 64 ? T : 256, R = NT / T;
  __shared__ float part[2][2][T > 64 ? T / 64 : 1];
  __shared__ float cols[R > 1 ? 2 * T * NV * VE : 1];
  const int l = threadIdx.x % T, grp = threadIdx.x / T, d = g.d;
  float wv[NV][VE], aw[NV][VE], ab[NV][VE];
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    load_f32<VE>(g.w, (l + T * q) * VE, d, 1.f, wv[q]);
#pragma unroll
    for (int e = 0; e < VE; ++e) aw[q][e] = ab[q][e] = 0.f;
  }
  const float inv = 1.f / (float)d;
  int flip = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * R; r0 < g.M; r0 += (int64_t)gridDim.x * R, flip ^= 1) {
    const int64_t row = r0 + grp;
    if (R == 1 || row < g.M) {
      float y[NV][VE], h[NV][VE];
#pragma unroll
      for (int q = 0; q < NV; ++q) {
        load_vec<DT>(g.dy + row * d * ES, (l + T * q) * VE, d, y[q]);
        load_vec<DT>(g.x + row * d * ES, (l + T * q) * VE, d, h[q]);
      }
      const float mean = g.mean[row], rs = g.rstd[row];
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int q = 0; q < NV; ++q)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          h[q][e] = (h[q][e] - mean) * rs;  // (past the row's end dy is 0, so every sum gets 0 there)
          aw[q][e] = fmaf(y[q][e], h[q][e], aw[q][e]);
          ab[q][e] += y[q][e];
          y[q][e] *= wv[q][e];
          s1 += y[q][e];
          s2 = fmaf(y[q][e], h[q][e], s2);
        }
      if (g.dx) {
        const float m1 = row_sum<T>(s1, part[flip][0]) * inv, m2 = row_sum<T>(s2, part[flip][1]) * inv;
#pragma unroll
        for (int q = 0; q < NV; ++q) {
          const int c = (l + T * q) * VE;
          float o[VE];
#pragma unroll
          for (int e = 0; e < VE; ++e) o[e] = rs * (y[q][e] - m1 - h[q][e] * m2);
          if (g.dres) {
            float z[VE];
            load_vec<DT>(g.dres + row * d * ES, c, d, z);
#pragma unroll
            for (int e = 0; e < VE; ++e) o[e] += z[e];
          }
          if (c < d) store_vec<DT>(g.dx + row * d * ES, c, d, o);
        }
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
    for (int c = threadIdx.x; c < d; c += NT) {
      out[c] = cols[2 * c];
      out[d + c] = cols[2 * c + 1];
    }
  } else {
#pragma unroll
    for (int q = 0; q < NV; ++q)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int c = (l + T * q) * VE + e;
        if (c < d) {
          out[c] = aw[q][e];
          out[d + c] = ab[q][e];
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

// How a row is shared: T lanes (a part of a wave, a wave, or a whole work-group)
// with NV vectors each, at most `most` of them.
struct LnShape {
  int T, NV;
};
static LnShape ln_shape(int d, int VE, int most) {
  const int n = (d + VE - 1) / VE;
  if (n <= 16) return {16, 1};
  if (n <= 32) return {32, 1};
  for (int T : {64, 256})
    if (n <= T * most) return {T, (n + T - 1) / T};
  return {1024, (n + 1023) / 1024};
}
constexpr int kLnMaxWidth = 16384;
static int ln_vec(int dt) { return dt == GTR_F32 ? 4 : 8; }
// Vectors per lane: the backward pass holds five values per element (dy, xh, w and
// both sums), the forward pass three.
static int ln_most(int dt, bool bwd) { return bwd && dt != GTR_F32 ? 2 : 4; }
static int ln_rows(const LnShape& s) { return s.T > 64 ? 1 : 256 / s.T; }  // of a work-group at a time

// Work-groups of the backward pass. Each costs a partial sum (16 bytes per column
// written and read back), each row 6 to 16 bytes per column: at least 8 rows per
// slot above 256 work-groups, which a short batch needs to fill the chip.
static int64_t ln_bwd_groups(int64_t M, const LnShape& s) {
  const int R = ln_rows(s);
  const int64_t all = (M + R - 1) / R;
  int64_t g = all / 8;
  g = g < 256 ? 256 : g > 1024 ? 1024 : g;
  return g < all ? g : all;
}

template <template <int, int, int> class F, class A>
static bool ln_dispatch(int dt, const LnShape& s, const A& a) {
#define GTR_LN_NV(DT, TT)                                       \
  if (s.T == TT) {                                              \
    if (s.NV == 1) return F<DT, TT, 1>::go(a), true;            \
    if (s.NV == 2) return F<DT, TT, 2>::go(a), true;            \
    if constexpr (F<DT, TT, 1>::kMost > 2) {                    \
      if (s.NV == 3) return F<DT, TT, 3>::go(a), true;          \
      if (s.NV == 4) return F<DT, TT, 4>::go(a), true;          \
    }                                                           \
  }
#define GTR_LN_T(DT)                                            \
  if (dt == DT) {                                               \
    if (s.T == 16) return F<DT, 16, 1>::go(a), true;            \
    if (s.T == 32) return F<DT, 32, 1>::go(a), true;            \
    GTR_LN_NV(DT, 64)                                           \
    GTR_LN_NV(DT, 256)                                          \
    GTR_LN_NV(DT, 1024)                                         \
  }
  GTR_LN_T(GTR_F32)
  GTR_LN_T(GTR_F16)
  GTR_LN_T(GTR_BF16)
#undef GTR_LN_T
#undef GTR_LN_NV
  return false;
}

template <class P>
struct LnLaunch {
  P p;
  unsigned grid;
  hipStream_t stream;
};
template <int DT, int T, int NV>
struct LnFwdGo {
  static constexpr int kMost = 4;
  static void go(const LnLaunch<LnFwd>& a) {
    hipLaunchKernelGGL((ln_fwd_kernel<DT, T, NV>), dim3(a.grid), dim3(T > 64 ? T : 256), 0, a.stream, a.p);
  }
};
template <int DT, int T, int NV>
struct LnBwdGo {
  static constexpr int kMost = DT == GTR_F32 ? 4 : 2;
  static void go(const LnLaunch<LnBwd>& a) {
    hipLaunchKernelGGL((ln_bwd_kernel<DT, T, NV>), dim3(a.grid), dim3(T > 64 ? T : 256), 0, a.stream, a.p);
  }
};

struct LnRange {
  const void* p;
  size_t n;
};
static bool ln_overlap(const LnRange& a, const LnRange& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && x < y + b.n && y < x + a.n;
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
  const LnShape s = ln_shape(a->d, ln_vec(a->dtype), ln_most(a->dtype, true));
  *need = ((size_t)ln_bwd_groups(a->M, s) * 2 * a->d * 4 + 255) & ~(size_t)255;
  if (!pointers) return GTR_OK;
  if (!a->dy || !a->x || !a->mean || !a->rstd || (!a->dx && !a->dw && !a->db)) return GTR_ERR_NULL;
  const size_t es = dtype_size(a->dtype), bytes = (size_t)a->M * a->d * es;
  if (ln_misaligned(a->dy, es) || ln_misaligned(a->x, es) || ln_misaligned(a->dres, es) || ln_misaligned(a->dx, es) ||
      ln_misaligned(a->mean, 4) || ln_misaligned(a->rstd, 4) || ln_misaligned(a->w, 4) || ln_misaligned(a->dw, 4) ||
      ln_misaligned(a->db, 4))
    return GTR_ERR_UNSUPPORTED;
  const bool sums = a->dw || a->db;
  if (sums && (!a->workspace || ln_misaligned(a->workspace, 256) || a->workspace_bytes < *need))
    return GTR_ERR_WORKSPACE;
  const LnRange ins[] = {{a->dy, bytes}, {a->x, bytes}, {a->dres, bytes}, {a->mean, (size_t)a->M * 4},
                         {a->rstd, (size_t)a->M * 4}, {a->w, (size_t)a->d * 4}};
  const LnRange outs[] = {{a->dx, bytes}, {a->dw, (size_t)a->d * 4}, {a->db, (size_t)a->d * 4},
                          {sums ? a->workspace : nullptr, *need}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 6; ++j)
      if (ln_overlap(outs[i], ins[j]) && !(i == 0 && j < 3 && outs[i].p == ins[j].p)) return GTR_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (ln_overlap(outs[i], outs[j])) return GTR_ERR_ALIAS;
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
  const LnRange ins[] = {{a->x, bytes}, {a->w, (size_t)a->d * 4}, {a->b, (size_t)a->d * 4}};
  const LnRange outs[] = {{a->y, bytes}, {a->mean, (size_t)a->M * 4}, {a->rstd, (size_t)a->M * 4}};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 3; ++j)
      if (ln_overlap(outs[i], ins[j]) && !(i == 0 && j == 0 && a->x == a->y)) return GTR_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (ln_overlap(outs[i], outs[j])) return GTR_ERR_ALIAS;
  }
  const LnShape s = ln_shape(a->d, ln_vec(a->dtype), ln_most(a->dtype, false));
  const int R = ln_rows(s);
  const LnFwd p = {static_cast<const char*>(a->x), a->w, a->b, static_cast<char*>(a->y), a->mean, a->rstd, a->M, a->d, a->eps};
  const LnLaunch<LnFwd> l = {p, (unsigned)((a->M + R - 1) / R), stream};
  if (!ln_dispatch<LnFwdGo>(a->dtype, s, l)) return GTR_ERR_UNSUPPORTED;
  return hipGetLastError() == hipSuccess ? GTR_OK : GTR_ERR_HIP;
}

extern "C" size_t gtr_layernorm_bwd_workspace_size(const gtr_layernorm_bwd_args* a) {
  size_t need;
  return ln_bwd_check(a, false, &need) == GTR_OK ? need : 0;
}

extern "C" gtr_status gtr_layernorm_bwd(const gtr_layernorm_bwd_args* a, hipStream_t stream) {
  size_t need;
  const gtr_status st = ln_bwd_check(a, true, &need);
  if (st != GTR_OK) return st;
  const LnShape s = ln_shape(a->d, ln_vec(a->dtype), ln_most(a->dtype, true));
  const int64_t G = ln_bwd_groups(a->M, s);
  const bool sums = a->dw || a->db;
  const LnBwd p = {static_cast<const char*>(a->dy), static_cast<const char*>(a->x), a->mean, a->rstd, a->w,
                   static_cast<const char*>(a->dres), static_cast<char*>(a->dx),
                   sums ? static_cast<float*>(a->workspace) : nullptr, a->M, a->d};
  const LnLaunch<LnBwd> l = {p, (unsigned)G, stream};
  if (!ln_dispatch<LnBwdGo>(a->dtype, s, l)) return GTR_ERR_UNSUPPORTED;
  if (hipGetLastError() != hipSuccess) return GTR_ERR_HIP;
  if (sums) {
    hipLaunchKernelGGL(ln_reduce_kernel, dim3((unsigned)((2 * (int64_t)a->d + 31) / 32)), dim3(1024), 0, stream, p.part,
                       (int)G, a->d, a->dw, a->db, a->accumulate);
    if (hipGetLastError() != hipSuccess) return GTR_ERR_HIP;
  }
  return GTR_OK;
}
