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
#include "ffn_plan.h"
#include "gtr.h"
#include "gtr_device.h"
#include "gtr_internal.h"

namespace gtr {

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

static bool ffn_misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

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

static gtr_status ffn_fwd_check(const gtr_ffn_fwd_args* a, const FfnFwdPlan& f) {
  if (!a->x || !a->w_gate || !a->w_value || !a->w_out || !a->y) return GTR_ERR_NULL;
  for (const void* p : {a->x, a->w_gate, a->w_value, a->w_out, a->residual, (const void*)a->y, (const void*)a->gate,
                        (const void*)a->value})
    if (ffn_misaligned(p)) return GTR_ERR_UNSUPPORTED;
  if (!a->workspace || (reinterpret_cast<uintptr_t>(a->workspace) & 255u) || a->workspace_bytes < f.total)
    return GTR_ERR_WORKSPACE;
  const size_t rows = (size_t)a->M * a->d * 2, kept = (size_t)a->M * a->hidden * 2, w = (size_t)a->d * a->hidden * 2;
  const Bytes ins[] = {{a->x, rows}, {a->w_gate, w}, {a->w_value, w}, {a->w_out, w}, {a->residual, rows}};
  const Bytes outs[] = {{a->y, rows}, {a->gate, kept}, {a->value, kept}, {a->workspace, f.total}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 5; ++j)
      if (bytes_meet(outs[i], ins[j]) && !(i == 0 && j == 4 && a->y == a->residual)) return GTR_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (bytes_meet(outs[i], outs[j])) return GTR_ERR_ALIAS;
  }
  return GTR_OK;
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
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
  const Bytes ins[] = {{a->dy, rows}, {a->x, rows}, {a->w_gate, w}, {a->w_value, w}, {a->w_out, w}, {a->gate, kept}, {a->value, kept}};
  const Bytes outs[] = {{a->dx, rows}, {a->dw_gate, dw}, {a->dw_value, dw}, {a->dw_out, dw}, {a->workspace, f.total}};
  for (int i = 0; i < 5; ++i) {
    for (int j = 0; j < 7; ++j)
      if (bytes_meet(outs[i], ins[j])) return GTR_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (bytes_meet(outs[i], outs[j])) return GTR_ERR_ALIAS;
  }
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
