// The plan of a feed-forward call: its products, the tile and the K slices of each,
// and the workspace. Host only, no HIP call.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "gtr.h"

namespace gtr {

// One product of a launch: C[M][N] = sum over nseg segments of A_s B_s, K deep each.
struct FfnProd {
  const char *a[2], *b[2];  // the segments' operands (gate epilogue: b = the two weights, nseg 1)
  char* c;
  const char* res;  // [M][N] in C's type, added (a residual, or C itself to accumulate), or null
  int64_t lda, ldb, ldc;
  int M, N, K, nseg;
  int gx, gy;  // row and column tiles
  int64_t part_off;  // where its partial sums start within a slice
};

// What an epilogue does with the product.
enum { kFfnStore = 0, kFfnGate = 1, kFfnGateGrad = 2 };

// Up to this many tokens the forward pass runs in ffn_few_kernel.
constexpr int kFewTokens = 8;
constexpr int64_t kFfnMaxWidth = 1 << 20;

constexpr int kFfnCus = 256;

// Tiles a product can run in: 256 x 256 with one work-group of 8 waves per CU,
// 128 x 128 with two of 4 waves, 64 x 64 with four of 4 waves.
constexpr int kFfnTile[3] = {256, 128, 64}, kFfnPerCu[3] = {1, 2, 4};
// A launch takes less than 2^32 threads: of n work-groups of a tile size (small tiles of
// a billion rows are more).
inline bool ffn_fits(int64_t n, int tile) { return n * (tile == 0 ? 512 : 256) < (int64_t)1 << 32; }
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
// (`skew`) spread each transfer over twice the lines; that is counted where both operands
// run along K, not for the rows of dy in dh (1027 x 1000 x 2728: estimate 18.5 us, 21.2).
//
// Against each tile forced, 16 shapes of 640 to 12,800 tokens, four launches each: the
// choice is within 5 % of the best but for 8 of the 64, which lose 6 to 8 % and, at 2048 x
// 1024 x 4096 and 3000 x 512 x 2048, 15 to 19 % (gradients 102 us against 87, 50 against 42;
// gated product 22 against 19).
inline float ffn_step(int tile, int lay, int o, bool skew) {
  static const float one[3][3] = {{1.0f, 1.0f, 1.1f}, {0.41f, 0.42f, 0.45f}, {0.24f, 0.25f, 0.3f}};
  static const float full[3][3] = {{1.42f, 1.45f, 1.35f}, {0.97f, 1.05f, 1.15f}, {0.82f, 1.19f, 1.46f}};
  static const float shared[5] = {0.f, 0.f, 0.19f, 0.54f, 1.f};  // tile 2: ((o - 1) / 3)^1.5
  const float by = skew ? tile == 2 ? 1.5f : 1.4f : 1.f;
  return by * (tile == 0   ? full[0][lay]
               : tile == 1 ? (o > 1 ? full : one)[1][lay]
                           : one[2][lay] + (full[2][lay] - one[2][lay]) * shared[o]);
}
inline float ffn_fixed(int tile, int epi, float fill) {
  static const float us[3][3] = {{9.f, 5.f, 4.f}, {9.f, 4.6f, 2.5f}, {8.f, 8.5f, 6.f}}, more[3] = {26.f, 8.5f, 1.5f};
  return us[epi][tile] + (epi == kFfnGateGrad ? more[tile] * (fill < 1.f ? fill : 1.f) : 0.f);
}
inline int64_t ffn_tiles(const FfnProd* p, int nprod, int tile, int epi) {
  const int bm = kFfnTile[tile], bn = epi == kFfnGate ? bm / 2 : bm;
  int64_t n = 0;
  for (int i = 0; i < nprod; ++i) n += (int64_t)((p[i].M + bm - 1) / bm) * ((p[i].N + bn - 1) / bn);
  return n;
}
inline int ffn_steps(const FfnProd& p) { return (p.K + 63) / 64 * p.nseg; }
inline int64_t ffn_elems(const FfnProd* p, int nprod) {
  int64_t n = 0;
  for (int i = 0; i < nprod; ++i) n += (int64_t)p[i].M * p[i].N;
  return n;
}
// Of partial sums: the launch, and their bytes written and read again.
inline float ffn_cut_us(int64_t elems, int ks) { return 4.f + (float)elems * (float)(ks + 1) * 4.f / 3e6f; }

// The tile size and the number of K slices with the least estimated time.
inline FfnPlan ffn_plan(const FfnProd* p, int nprod, int lay, int epi) {
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
      if (!ffn_fits(n, c)) break;
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
inline void ffn_plan_grads(const FfnProd* x, int nx, const FfnProd* w, int nw, FfnPlan* px, FfnPlan* pw) {
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
        if (!ffn_fits(n + 7, c)) break;
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

inline FfnProd ffn_prod(const void* a, const void* b, void* c, int64_t lda, int64_t ldb, int64_t M, int64_t N, int64_t K) {
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

inline size_t ffn_align(size_t n) { return (n + 255) & ~(size_t)255; }

inline gtr_status ffn_sizes(int64_t M, int32_t d, int32_t hidden, int dt, int act) {
  if (M <= 0 || d <= 0 || hidden <= 0) return GTR_ERR_SHAPE;
  if (d % 8 || hidden % 8 || d > kFfnMaxWidth || hidden > kFfnMaxWidth || (dt != GTR_F16 && dt != GTR_BF16) ||
      (act != GTR_ACT_SILU && act != GTR_ACT_GELU))
    return GTR_ERR_UNSUPPORTED;
  // Rows count in 32 bits, and the largest tiles' launches hold every work-group
  // (activations and weights of 256 and 128 GiB: past what the memory holds).
  const int64_t w = d > hidden ? d : hidden;
  if (M > ((int64_t)1 << 30) || M * w > ((int64_t)1 << 37) || (int64_t)d * hidden > ((int64_t)1 << 36)) return GTR_ERR_SHAPE;
  return GTR_OK;
}

struct FfnFwdPlan {
  FfnProd up, down;
  FfnPlan pu, pd;
  size_t h_bytes, total;
};

inline void ffn_fwd_plan(const gtr_ffn_fwd_args* a, FfnFwdPlan* f) {
  f->up = ffn_prod(a->x, a->w_gate, nullptr, a->d, a->d, a->M, a->hidden, a->d);
  f->up.b[1] = static_cast<const char*>(a->w_value);
  f->down = ffn_prod(nullptr, a->w_out, a->y, a->hidden, a->hidden, a->M, a->d, a->hidden);
  f->down.res = static_cast<const char*>(a->residual);
  f->pu = ffn_plan(&f->up, 1, kRowRow, kFfnGate);
  f->pd = ffn_plan(&f->down, 1, kRowRow, kFfnStore);
  f->h_bytes = ffn_align((size_t)a->M * a->hidden * 2);
  f->total = f->h_bytes + (a->M > kFewTokens && f->pd.ksplit > 1 ? ffn_align((size_t)f->pd.ksplit * a->M * a->d * 4) : 0);
}

struct FfnBwdPlan {
  FfnProd dh, dx, dw[3];
  int ndw;
  FfnPlan ph, px, pw;
  size_t kept, dg_off, dv_off, h_off, part_off, xpart, total;
};

inline void ffn_bwd_plan(const gtr_ffn_bwd_args* a, FfnBwdPlan* f) {
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

inline gtr_status ffn_bwd_sizes(const gtr_ffn_bwd_args* a) {
  if (!a) return GTR_ERR_NULL;
  const gtr_status st = ffn_sizes(a->M, a->d, a->hidden, a->dtype, a->act);
  if (st != GTR_OK) return st;
  if (a->dw_dtype != a->dtype && a->dw_dtype != GTR_F32) return GTR_ERR_UNSUPPORTED;
  return GTR_OK;
}

}  // namespace gtr
