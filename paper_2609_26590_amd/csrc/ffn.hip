// The gated feed-forward y = [act(x W_g^T) * (x W_v^T)] W_o^T (+ residual) and its
// backward pass, as products (ffn_gemm.h):
//
//   forward:   h = act(x W_g^T) * (x W_v^T)     one launch: both projections, the activation and the product
//              y = h W_o^T (+ residual)
//   backward:  dh = dy W_o, dg = dh v act'(g), dv = dh act(g), h = act(g) v   one launch
//              dW_g = dg^T x, dW_v = dv^T x, dW_o = dy^T h,
//              dx = dg W_g + dv W_v (one sum over both)                       one launch
//
// A product whose tiles do not fill the chip is cut along K; the partial sums are
// added in a fixed order by a second launch.
#include <hip/hip_runtime.h>

#include "ffn_gemm.h"
#include "gtr.h"
#include "gtr_device.h"
#include "gtr_internal.h"

namespace gtr {

constexpr int kFfnCus = 256;
constexpr int64_t kFfnMaxWidth = 1 << 20;

// Tiles a product can run in: 256 x 256 with one work-group of 8 waves per CU,
// 128 x 128 with two of 4 waves, 64 x 64 with four of 4 waves.
constexpr int kFfnTile[3] = {256, 128, 64}, kFfnPerCu[3] = {1, 2, 4};
enum { kRowRow = 0, kRowCol = 1, kColCol = 2 };  // operands: both along K, A alone, none

struct FfnPlan {
  int tile, ksplit, steps;  // steps: 64-deep steps of a slice
  int64_t tiles;
  float us;  // estimate of a work-group's time, the CU full
};

// Estimates in us, from timings of each tile on its own: a step with `o` work-groups
// on the CU (its matrix cores are shared late: the second costs less than the fourth),
// and what a work-group takes besides its steps, `fill` being the share of the chip's
// places that are taken (the gradients' epilogue moves 10 bytes per element of C, which
// bound it once many do so together). Rows along K that do not start on 128 bytes
// (`skew`) spread each transfer over twice the lines.
static float ffn_step(int tile, int lay, int o, bool skew) {
  static const float one[3][3] = {{1.0f, 1.0f, 1.1f}, {0.41f, 0.42f, 0.45f}, {0.24f, 0.25f, 0.3f}};
  static const float full[3][3] = {{1.42f, 1.45f, 1.35f}, {0.97f, 1.05f, 1.15f}, {0.82f, 1.19f, 1.46f}};
  static const float shared[5] = {0.f, 0.f, 0.19f, 0.54f, 1.f};  // tile 2: ((o - 1) / 3)^1.5
  const float by = skew ? tile == 2 ? 1.5f : 1.4f : 1.f;
  return by * (tile == 0   ? full[0][lay]
               : tile == 1 ? (o > 1 ? full : one)[1][lay]
                           : one[2][lay] + (full[2][lay] - one[2][lay]) * shared[o]);
}
static float ffn_fixed(int tile, int epi, float fill) {
  static const float us[3][3] = {{9.f, 5.f, 4.f}, {9.f, 4.6f, 2.5f}, {8.f, 8.5f, 6.f}}, more[3] = {26.f, 8.5f, 1.5f};
  return us[epi][tile] + (epi == kFfnGateGrad ? more[tile] * (fill < 1.f ? fill : 1.f) : 0.f);
}
static int64_t ffn_tiles(const FfnProd* p, int nprod, int tile, int epi) {
  const int bm = kFfnTile[tile], bn = epi == kFfnGate ? bm / 2 : bm;
  int64_t n = 0;
  for (int i = 0; i < nprod; ++i) n += (int64_t)((p[i].M + bm - 1) / bm) * ((p[i].N + bn - 1) / bn);
  return n;
}
static int ffn_steps(const FfnProd& p) { return (p.K + 63) / 64 * p.nseg; }
static int64_t ffn_elems(const FfnProd* p, int nprod) {
  int64_t n = 0;
  for (int i = 0; i < nprod; ++i) n += (int64_t)p[i].M * p[i].N;
  return n;
}
// Of partial sums: the launch, and their bytes written and read again.
static float ffn_cut_us(int64_t elems, int ks) { return 4.f + (float)elems * (float)(ks + 1) * 4.f / 3e6f; }

// The tile size and the number of K slices with the least estimated time.
static FfnPlan ffn_plan(const FfnProd* p, int nprod, int lay, int epi) {
  FfnPlan best = {};
  float least = 0.f;
  const int steps = ffn_steps(p[0]);
  const int64_t elems = ffn_elems(p, nprod);
  const bool skew = lay == kRowRow && (p[0].lda % 64 || p[0].ldb % 64);
  for (int c = 0; c < 3; ++c) {
    const int64_t tiles = ffn_tiles(p, nprod, c, epi), slots = (int64_t)kFfnCus * kFfnPerCu[c];
    const int most = epi == kFfnStore && steps >= 8 ? (steps / 4 < 32 ? steps / 4 : 32) : 1;
    for (int ks = 1; ks <= most; ++ks) {
      const int per = (steps + ks - 1) / ks;
      if (ks > 1 && (steps + per - 1) / per != ks) continue;  // a slice would be empty
      const int64_t n = tiles * ks;
      const float tile_us = per * ffn_step(c, lay, kFfnPerCu[c], skew) + ffn_fixed(c, epi, 1.f);
      float us;
      if (n <= slots)
        us = per * ffn_step(c, lay, (int)((n + kFfnCus - 1) / kFfnCus), skew) + ffn_fixed(c, epi, (float)n / (float)slots);
      else if (kFfnPerCu[c] == 1)
        us = (float)((n + slots - 1) / slots) * tile_us;
      else  // a CU's work-groups do not start and end together: no whole rounds
        us = (float)n / (float)slots * tile_us;
      if (ks > 1) us += ffn_cut_us(elems, ks);
      if (least == 0.f || us < least) {
        least = us;
        best = {c, ks, per, tiles, tile_us};
      }
    }
  }
  return best;
}

// One tile size for the gradients of the input (nx = 1 or 0 products) and of the
// weights, which share a launch, and the K slices of each: the launch takes the work
// of all tiles spread over the chip, and at least the longest tile; per CU that is
// not full, the tiles run faster.
static void ffn_plan_grads(const FfnProd* x, int nx, const FfnProd* w, int nw, FfnPlan* px, FfnPlan* pw) {
  float least = 0.f;
  const int sx = nx ? ffn_steps(*x) : 0, sw = nw ? ffn_steps(*w) : 0;
  for (int c = 0; c < 3; ++c) {
    const int64_t tx = ffn_tiles(x, nx, c, kFfnStore), tw = ffn_tiles(w, nw, c, kFfnStore), slots = (int64_t)kFfnCus * kFfnPerCu[c];
    const int mx = sx >= 8 ? (sx / 4 < 32 ? sx / 4 : 32) : 1, mw = sw >= 8 ? (sw / 4 < 32 ? sw / 4 : 32) : 1;
    for (int kx = 1; kx <= mx; ++kx) {
      const int perx = (sx + kx - 1) / kx;
      if (kx > 1 && (sx + perx - 1) / perx != kx) continue;
      if (kx > 1 && tx * (kx - 1) >= slots) break;  // cut no further than full
      for (int kw = 1; kw <= mw; ++kw) {
        const int perw = (sw + kw - 1) / kw;
        if (kw > 1 && (sw + perw - 1) / perw != kw) continue;
        if (kw > 1 && tw * (kw - 1) >= slots) break;
        const int64_t n = tx * kx + tw * kw;
        const int o = n >= slots ? kFfnPerCu[c] : (int)((n + kFfnCus - 1) / kFfnCus);
        const float fixed = ffn_fixed(c, kFfnStore, 1.f);
        const float ux = nx ? perx * ffn_step(c, kRowCol, o, false) + fixed : 0.f, uw = nw ? perw * ffn_step(c, kColCol, o, false) + fixed : 0.f;
        const float longest = ux > uw ? ux : uw, shortest = ux < uw && nx ? ux : nw ? uw : ux;
        float us = ((float)(tx * kx) * ux + (float)(tw * kw) * uw) / (float)(kFfnCus * o);
        us = n > slots ? us + 0.5f * shortest : us;
        us = us < longest ? longest : us;
        if (kx > 1 || kw > 1)
          us += ffn_cut_us((kx > 1 ? ffn_elems(x, nx) * (kx + 1) : 0) + (kw > 1 ? ffn_elems(w, nw) * (kw + 1) : 0), 0);
        if (least == 0.f || us < least) {
          least = us;
          *px = {c, kx, perx, tx, ux};
          *pw = {c, kw, perw, tw, uw};
        }
      }
    }
  }
}

// Tile counts and the layout of partial sums.
static void ffn_prepare(FfnGemm& g, const FfnPlan& plan, int epi) {
  const int bm = kFfnTile[plan.tile], bn = epi == kFfnGate ? bm / 2 : bm;
  int64_t off = 0;
  for (int i = 0; i < g.nprod; ++i) {
    g.p[i].gx = (g.p[i].M + bm - 1) / bm;
    g.p[i].gy = (g.p[i].N + bn - 1) / bn;
    g.p[i].part_off = off;
    off += (int64_t)g.p[i].M * g.p[i].N;
  }
  g.ksplit = plan.ksplit;
  g.part_slice = off;
}

static gtr_status ffn_add_slices(const FfnGemm& g, const FfnGemm& h, hipStream_t stream) {
  const int64_t n = (g.ksplit > 1 ? g.part_slice : 0) + (h.ksplit > 1 ? h.part_slice : 0);
  if (!n) return GTR_OK;
  hipLaunchKernelGGL(ffn_reduce_kernel, dim3((unsigned)((n / 8 + 255) / 256)), dim3(256), 0, stream, g, h);
  return hipGetLastError() == hipSuccess ? GTR_OK : GTR_ERR_HIP;
}

template <int DT, int TA, int TB, int EPI>
static void ffn_launch(const FfnGemm& g, int tile, unsigned grid, hipStream_t stream) {
  if (tile == 0)
    hipLaunchKernelGGL((ffn_gemm_kernel<DT, TA, TB, EPI, 256, 256, 2, 4>), dim3(grid), dim3(512), 0, stream, g);
  else if (tile == 1)
    hipLaunchKernelGGL((ffn_gemm_kernel<DT, TA, TB, EPI, 128, 128, 2, 2>), dim3(grid), dim3(256), 0, stream, g);
  else
    hipLaunchKernelGGL((ffn_gemm_kernel<DT, TA, TB, EPI, 64, 64, 2, 2>), dim3(grid), dim3(256), 0, stream, g);
}

// One product in a launch of its own. A plan with K slices needs g.part.
template <int TA, int TB, int EPI>
static gtr_status ffn_run(FfnGemm& g, int dt, const FfnPlan& plan, hipStream_t stream) {
  ffn_prepare(g, plan, EPI);
  const unsigned grid = (unsigned)(plan.tiles * plan.ksplit);
  if (dt == GTR_F16)
    ffn_launch<GTR_F16, TA, TB, EPI>(g, plan.tile, grid, stream);
  else
    ffn_launch<GTR_BF16, TA, TB, EPI>(g, plan.tile, grid, stream);
  if (hipGetLastError() != hipSuccess) return GTR_ERR_HIP;
  FfnGemm none = {};
  return ffn_add_slices(g, none, stream);
}

template <int DT>
static void ffn_launch_grads(const FfnGemm& x, const FfnGemm& w, int tile, int nx, int nw, int x_first, hipStream_t stream) {
  const unsigned grid = (unsigned)(x_first ? (nx + 7) / 8 * 8 + nw : (nw + 7) / 8 * 8 + nx);
  if (tile == 0)
    hipLaunchKernelGGL((ffn_grad_kernel<DT, 256, 256, 2, 4>), dim3(grid), dim3(512), 0, stream, x, w, nx, nw, x_first);
  else if (tile == 1)
    hipLaunchKernelGGL((ffn_grad_kernel<DT, 128, 128, 2, 2>), dim3(grid), dim3(256), 0, stream, x, w, nx, nw, x_first);
  else
    hipLaunchKernelGGL((ffn_grad_kernel<DT, 64, 64, 2, 2>), dim3(grid), dim3(256), 0, stream, x, w, nx, nw, x_first);
}

// The gradients of input and weights (either may have no product), the longer tiles
// first, and their K slices' sums.
static gtr_status ffn_run_grads(FfnGemm& x, FfnGemm& w, int dt, const FfnPlan& px, const FfnPlan& pw, hipStream_t stream) {
  ffn_prepare(x, px, kFfnStore);
  ffn_prepare(w, pw, kFfnStore);
  const int nx = x.nprod ? (int)(px.tiles * px.ksplit) : 0, nw = w.nprod ? (int)(pw.tiles * pw.ksplit) : 0;
  const int x_first = nx && (!nw || px.us >= pw.us);
  if (dt == GTR_F16)
    ffn_launch_grads<GTR_F16>(x, w, px.tile, nx, nw, x_first, stream);
  else
    ffn_launch_grads<GTR_BF16>(x, w, px.tile, nx, nw, x_first, stream);
  if (hipGetLastError() != hipSuccess) return GTR_ERR_HIP;
  return ffn_add_slices(x, w, stream);
}

static FfnProd ffn_prod(const void* a, const void* b, void* c, int64_t lda, int64_t ldb, int64_t M, int64_t N, int64_t K) {
  FfnProd p = {};
  p.a[0] = p.a[1] = static_cast<const char*>(a);
  p.b[0] = p.b[1] = static_cast<const char*>(b);
  p.c = static_cast<char*>(c);
  p.lda = lda;
  p.ldb = ldb;
  p.ldc = N;
  p.M = (int)M;
  p.N = (int)N;
  p.K = (int)K;
  p.nseg = 1;
  return p;
}

struct FfnRange {
  const void* p;
  size_t n;
};
static bool ffn_overlap(const FfnRange& a, const FfnRange& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && x < y + b.n && y < x + a.n;
}
static bool ffn_misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
static size_t ffn_align(size_t n) { return (n + 255) & ~(size_t)255; }

static gtr_status ffn_sizes(int64_t M, int32_t d, int32_t hidden, int dt, int act) {
  if (M <= 0 || d <= 0 || hidden <= 0) return GTR_ERR_SHAPE;
  if (d % 8 || hidden % 8 || d > kFfnMaxWidth || hidden > kFfnMaxWidth || (dt != GTR_F16 && dt != GTR_BF16) ||
      (act != GTR_ACT_SILU && act != GTR_ACT_GELU))
    return GTR_ERR_UNSUPPORTED;
  // rows and work-groups count in 32 bits
  const int64_t w = d > hidden ? d : hidden;
  if (M > ((int64_t)1 << 30) || M * w > ((int64_t)1 << 38)) return GTR_ERR_SHAPE;
  return GTR_OK;
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
// Up to kFewTokens tokens the forward pass runs in ffn_few_kernel, which has columns
// for no more. Kernel times of both launches, in tiles against there: 1 x 1024 x 2816
// 17.0 against 9.7 us, 1 x 192 x 768 13.1 against 6.6.
template <int DT>
static gtr_status ffn_run_few(const gtr_ffn_fwd_args* a, hipStream_t stream) {
  FfnFew up = {}, down = {};
  up.x = static_cast<const char*>(a->x);
  up.w[0] = static_cast<const char*>(a->w_gate);
  up.w[1] = static_cast<const char*>(a->w_value);
  up.c = static_cast<char*>(a->workspace);
  up.gate = static_cast<char*>(a->gate);
  up.value = static_cast<char*>(a->value);
  up.act = a->act;
  up.M = down.M = (int)a->M;
  up.N = down.K = a->hidden;
  up.K = down.N = a->d;
  down.x = up.c;
  down.w[0] = static_cast<const char*>(a->w_out);
  down.c = static_cast<char*>(a->y);
  down.res = static_cast<const char*>(a->residual);
  hipLaunchKernelGGL((ffn_few_kernel<DT, 2>), dim3((up.N + 7) / 8), dim3(64 * few_waves(2)), 0, stream, up);
  hipLaunchKernelGGL((ffn_few_kernel<DT, 1>), dim3((down.N + 7) / 8), dim3(64 * few_waves(1)), 0, stream, down);
  return hipGetLastError() == hipSuccess ? GTR_OK : GTR_ERR_HIP;
}

struct FfnFwdPlan {
  FfnProd up, down;
  FfnPlan pu, pd;
  size_t h_bytes, total;
};

static void ffn_fwd_plan(const gtr_ffn_fwd_args* a, FfnFwdPlan* f) {
  f->up = ffn_prod(a->x, a->w_gate, nullptr, a->d, a->d, a->M, a->hidden, a->d);
  f->up.b[1] = static_cast<const char*>(a->w_value);
  f->down = ffn_prod(nullptr, a->w_out, a->y, a->hidden, a->hidden, a->M, a->d, a->hidden);
  f->down.res = static_cast<const char*>(a->residual);
  f->pu = ffn_plan(&f->up, 1, kRowRow, kFfnGate);
  f->pd = ffn_plan(&f->down, 1, kRowRow, kFfnStore);
  f->h_bytes = ffn_align((size_t)a->M * a->hidden * 2);
  f->total = f->h_bytes + (a->M > kFewTokens && f->pd.ksplit > 1 ? ffn_align((size_t)f->pd.ksplit * a->M * a->d * 4) : 0);
}

static gtr_status ffn_fwd_check(const gtr_ffn_fwd_args* a, const FfnFwdPlan& f) {
  if (!a->x || !a->w_gate || !a->w_value || !a->w_out || !a->y) return GTR_ERR_NULL;
  for (const void* p : {a->x, a->w_gate, a->w_value, a->w_out, a->residual, (const void*)a->y, (const void*)a->gate,
                        (const void*)a->value})
    if (ffn_misaligned(p)) return GTR_ERR_UNSUPPORTED;
  if (!a->workspace || (reinterpret_cast<uintptr_t>(a->workspace) & 255u) || a->workspace_bytes < f.total)
    return GTR_ERR_WORKSPACE;
  const size_t rows = (size_t)a->M * a->d * 2, kept = (size_t)a->M * a->hidden * 2, w = (size_t)a->d * a->hidden * 2;
  const FfnRange ins[] = {{a->x, rows}, {a->w_gate, w}, {a->w_value, w}, {a->w_out, w}, {a->residual, rows}};
  const FfnRange outs[] = {{a->y, rows}, {a->gate, kept}, {a->value, kept}, {a->workspace, f.total}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 5; ++j)
      if (ffn_overlap(outs[i], ins[j]) && !(i == 0 && j == 4 && a->y == a->residual)) return GTR_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (ffn_overlap(outs[i], outs[j])) return GTR_ERR_ALIAS;
  }
  return GTR_OK;
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
struct FfnBwdPlan {
  FfnProd dh, dx, dw[3];
  int ndw;
  FfnPlan ph, px, pw;
  size_t kept, dg_off, dv_off, h_off, part_off, xpart, total;
};

static void ffn_bwd_plan(const gtr_ffn_bwd_args* a, FfnBwdPlan* f) {
  const int64_t M = a->M, d = a->d, h = a->hidden;
  f->kept = ffn_align((size_t)M * h * 2);
  f->dg_off = 0;
  f->dv_off = f->kept;
  f->h_off = 2 * f->kept;
  f->part_off = (a->dw_out ? 3 : 2) * f->kept;
  char* ws = static_cast<char*>(a->workspace);
  char *dg = ws + f->dg_off, *dv = ws + f->dv_off, *hh = ws + f->h_off;
  f->dh = ffn_prod(a->dy, a->w_out, a->dw_out ? hh : nullptr, d, h, M, h, d);
  f->dx = ffn_prod(dg, a->w_gate, a->dx, h, d, M, d, h);
  f->dx.a[1] = dv;
  f->dx.b[1] = static_cast<const char*>(a->w_value);
  f->dx.nseg = 2;
  f->ndw = 0;
  if (a->dw_gate) f->dw[f->ndw++] = ffn_prod(dg, a->x, a->dw_gate, h, d, h, d, M);
  if (a->dw_value) f->dw[f->ndw++] = ffn_prod(dv, a->x, a->dw_value, h, d, h, d, M);
  if (a->dw_out) f->dw[f->ndw++] = ffn_prod(a->dy, hh, a->dw_out, d, h, d, h, M);
  for (int i = 0; i < f->ndw; ++i) f->dw[i].res = a->accumulate ? f->dw[i].c : nullptr;
  f->ph = ffn_plan(&f->dh, 1, kRowCol, kFfnGateGrad);
  f->px = f->pw = FfnPlan{0, 1, 0, 0, 0.f};
  ffn_plan_grads(&f->dx, a->dx ? 1 : 0, f->dw, f->ndw, &f->px, &f->pw);
  f->xpart = a->dx && f->px.ksplit > 1 ? ffn_align((size_t)f->px.ksplit * M * d * 4) : 0;
  const size_t wpart = f->ndw && f->pw.ksplit > 1 ? ffn_align((size_t)f->pw.ksplit * f->ndw * d * h * 4) : 0;
  f->total = f->part_off + f->xpart + wpart;
}

static gtr_status ffn_bwd_check(const gtr_ffn_bwd_args* a, const FfnBwdPlan& f) {
  if (!a->dy || !a->x || !a->w_gate || !a->w_value || !a->w_out || !a->gate || !a->value ||
      (!a->dx && !a->dw_gate && !a->dw_value && !a->dw_out))
    return GTR_ERR_NULL;
  for (const void* p : {a->dy, a->x, a->w_gate, a->w_value, a->w_out, a->gate, a->value, (const void*)a->dx,
                        (const void*)a->dw_gate, (const void*)a->dw_value, (const void*)a->dw_out})
    if (ffn_misaligned(p)) return GTR_ERR_UNSUPPORTED;
  if (!a->workspace || (reinterpret_cast<uintptr_t>(a->workspace) & 255u) || a->workspace_bytes < f.total)
    return GTR_ERR_WORKSPACE;
  const size_t rows = (size_t)a->M * a->d * 2, kept = (size_t)a->M * a->hidden * 2, w = (size_t)a->d * a->hidden * 2;
  const size_t dw = (size_t)a->d * a->hidden * dtype_size(a->dw_dtype);
  const FfnRange ins[] = {{a->dy, rows}, {a->x, rows}, {a->w_gate, w}, {a->w_value, w}, {a->w_out, w}, {a->gate, kept}, {a->value, kept}};
  const FfnRange outs[] = {{a->dx, rows}, {a->dw_gate, dw}, {a->dw_value, dw}, {a->dw_out, dw}, {a->workspace, f.total}};
  for (int i = 0; i < 5; ++i) {
    for (int j = 0; j < 7; ++j)
      if (ffn_overlap(outs[i], ins[j])) return GTR_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (ffn_overlap(outs[i], outs[j])) return GTR_ERR_ALIAS;
  }
  return GTR_OK;
}

static gtr_status ffn_bwd_sizes(const gtr_ffn_bwd_args* a) {
  if (!a) return GTR_ERR_NULL;
  const gtr_status st = ffn_sizes(a->M, a->d, a->hidden, a->dtype, a->act);
  if (st != GTR_OK) return st;
  if (a->dw_dtype != a->dtype && a->dw_dtype != GTR_F32) return GTR_ERR_UNSUPPORTED;
  return GTR_OK;
}

}  // namespace gtr

using namespace gtr;

extern "C" size_t gtr_ffn_fwd_workspace_size(const gtr_ffn_fwd_args* a) {
  if (!a || ffn_sizes(a->M, a->d, a->hidden, a->dtype, a->act) != GTR_OK) return 0;
  FfnFwdPlan f;
  ffn_fwd_plan(a, &f);
  return f.total;
}

extern "C" gtr_status gtr_ffn_fwd(const gtr_ffn_fwd_args* a, hipStream_t stream) {
  if (!a) return GTR_ERR_NULL;
  gtr_status st = ffn_sizes(a->M, a->d, a->hidden, a->dtype, a->act);
  if (st != GTR_OK) return st;
  FfnFwdPlan f;
  ffn_fwd_plan(a, &f);
  st = ffn_fwd_check(a, f);
  if (st != GTR_OK) return st;
  if (a->M <= kFewTokens) return a->dtype == GTR_F16 ? ffn_run_few<GTR_F16>(a, stream) : ffn_run_few<GTR_BF16>(a, stream);
  char* h = static_cast<char*>(a->workspace);
  FfnGemm g = {};
  g.nprod = 1;
  g.cdt = a->dtype;
  g.act = a->act;
  g.p[0] = f.up;
  g.p[0].c = h;
  g.gate = static_cast<char*>(a->gate);
  g.value = static_cast<char*>(a->value);
  st = ffn_run<0, 0, kFfnGate>(g, a->dtype, f.pu, stream);
  if (st != GTR_OK) return st;
  g.p[0] = f.down;
  g.p[0].a[0] = g.p[0].a[1] = h;
  g.part = reinterpret_cast<float*>(h + f.h_bytes);
  return ffn_run<0, 0, kFfnStore>(g, a->dtype, f.pd, stream);
}

extern "C" size_t gtr_ffn_bwd_workspace_size(const gtr_ffn_bwd_args* a) {
  if (ffn_bwd_sizes(a) != GTR_OK) return 0;
  FfnBwdPlan f;
  ffn_bwd_plan(a, &f);
  return f.total;
}

extern "C" gtr_status gtr_ffn_bwd(const gtr_ffn_bwd_args* a, hipStream_t stream) {
  gtr_status st = ffn_bwd_sizes(a);
  if (st != GTR_OK) return st;
  FfnBwdPlan f;
  ffn_bwd_plan(a, &f);
  st = ffn_bwd_check(a, f);
  if (st != GTR_OK) return st;
  char* ws = static_cast<char*>(a->workspace);
  FfnGemm g = {};
  g.nprod = 1;
  g.cdt = a->dtype;
  g.act = a->act;
  g.p[0] = f.dh;
  g.gate = const_cast<char*>(static_cast<const char*>(a->gate));
  g.value = const_cast<char*>(static_cast<const char*>(a->value));
  g.dgate = ws + f.dg_off;
  g.dvalue = ws + f.dv_off;
  st = ffn_run<0, 1, kFfnGateGrad>(g, a->dtype, f.ph, stream);
  if (st != GTR_OK) return st;
  FfnGemm x = {}, w = {};
  x.nprod = a->dx ? 1 : 0;
  x.cdt = a->dtype;
  x.p[0] = f.dx;
  x.part = reinterpret_cast<float*>(ws + f.part_off);
  w.nprod = f.ndw;
  w.cdt = a->dw_dtype;
  for (int i = 0; i < f.ndw; ++i) w.p[i] = f.dw[i];
  w.part = reinterpret_cast<float*>(ws + f.part_off + f.xpart);
  return ffn_run_grads(x, w, a->dtype, f.px, f.pw, stream);
}
