// The gated linear recurrence with a diagonal state, channel by channel along one of the
// four scan orders, and its gradients, in float32:
//
//   la_t = g_t, or logsigmoid(g_t) / tau;   a_t = exp(la_t)
//   h_t = a_t h_{t-1} + b_t,   b_t = x_t, or (1 - a_t) x_t
//
//   Y_t = a_t D_t,  D_t = dh_t + Y_{t+1}   (Y behind the last token: the last state's gradient)
//   dx_t = D_t, or (1 - a_t) D_t;   dla_t = Y_t (h_{t-1} [- x_t]);   dg_t = dla_t, or
//   dla_t sigmoid(-g_t) / tau;   dh_0 = Y_1
//
// Both are a scan of affine maps s -> P s + E, which compose; the backward one runs in
// the reversed order. One launch (behind one that clears its words), every array once: what
// bounds long calls is memory (4 x 16384 x 2048 bf16 backward 317 us, 5.1 TB/s; 16384 x 4096
// float32 forward 156, 5.2; a large copy reaches 5.0) and, in 16-bit types, the gates'
// arithmetic with it, three exponentials or logarithms per logit (32768 x 4096 forward of bf16
// logits 172 us, of fp16 ones with 1 - a 184); short ones the chain of number, rows,
// gates, hand-over and stores.
#include <hip/hip_runtime.h>

#include "gtr.h"
#include "gtr_device.h"
#include "gtr_internal.h"
#include "rec_words.h"

// Products and sums round as they are written: both ways through a wave's steps give the
// same bits.
#pragma clang fp contract(off)

namespace gtr {

// ---------------------------------------------------------------------------
// rows
// ---------------------------------------------------------------------------
// V consecutive elements of a row, at any element address (the machine's vector loads and
// stores need no alignment beyond an element's), in whole words.
template <int BYTES>
struct __attribute__((packed, aligned(2))) RecRaw {
  unsigned u[BYTES / 4];
};
template <>
struct RecRaw<2> {
  unsigned short u[1];
};
template <int DT, int V>
struct RecVec {
  static constexpr int ES = DT == GTR_F32 ? 4 : 2;
  RecRaw<V * ES> r;
  __device__ __forceinline__ void load(const char* p) { r = *reinterpret_cast<const RecRaw<V * ES>*>(p); }
  __device__ __forceinline__ void store(char* p) const { *reinterpret_cast<RecRaw<V * ES>*>(p) = r; }
  __device__ __forceinline__ unsigned short half(int v) const {
    return (unsigned short)(v & 1 ? r.u[v / 2] >> 16 : r.u[v / 2] & 0xffffu);
  }
  __device__ __forceinline__ float get(int v) const {
    if constexpr (DT == GTR_F32)
      return __builtin_bit_cast(float, r.u[v]);
    else if constexpr (DT == GTR_F16)
      return (float)__builtin_bit_cast(_Float16, half(v));
    else if constexpr (V == 1)
      return bf16_bits_to_f32(r.u[0]);
    else
      return __builtin_bit_cast(float, v & 1 ? r.u[v / 2] & 0xffff0000u : r.u[v / 2] << 16);
  }
  __device__ __forceinline__ void set(const float (&x)[V]) {
    if constexpr (DT == GTR_F32) {
#pragma unroll
      for (int v = 0; v < V; ++v) r.u[v] = __builtin_bit_cast(unsigned, x[v]);
    } else if constexpr (V == 1) {
      if constexpr (DT == GTR_F16)
        r.u[0] = __builtin_bit_cast(unsigned short, (_Float16)x[0]);
      else
        r.u[0] = __builtin_bit_cast(unsigned short, (__bf16)x[0]);
    } else {
      typedef _Float16 hh __attribute__((ext_vector_type(2)));
      typedef __bf16 bb __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int v = 0; v < V; v += 2) {  // pairs, which convert in one instruction
        const f2 p = {x[v], x[v + 1]};
        if constexpr (DT == GTR_F16)
          r.u[v / 2] = __builtin_bit_cast(unsigned, __builtin_convertvector(p, hh));
        else
          r.u[v / 2] = __builtin_bit_cast(unsigned, __builtin_convertvector(p, bb));
      }
    }
  }
  __device__ __forceinline__ void store1(char* p, int v) const {
    if constexpr (DT == GTR_F32)
      *reinterpret_cast<unsigned*>(p + 4 * v) = r.u[v];
    else
      *reinterpret_cast<unsigned short*>(p + 2 * v) = half(v);
  }
};

// The rows that a scan visits one after the other, from step s on. Uniform over a wave.
struct RecWalk {
  int64_t row;         // spatial index of the first step
  int64_t step, wrap;  // to the next one, within a grid column and behind its end
  int left, run;       // steps to that end; steps of a whole column less one
  __device__ __forceinline__ RecWalk(int64_t s, int64_t L, int H, int W, int dir) {
    const bool back = dir == GTR_SCAN_ROW_REV || dir == GTR_SCAN_COL_REV;
    const unsigned at = (unsigned)(back ? L - 1 - s : s);  // (L is below 2^31)
    if (dir == GTR_SCAN_ROW || dir == GTR_SCAN_ROW_REV) {
      row = at;
      step = wrap = back ? -1 : 1;
      left = run = 0x7fffffff;
    } else {
      const unsigned j = at / (unsigned)H, i = at - j * (unsigned)H;
      const int64_t to_top = (int64_t)(H - 1) * W - 1;
      row = (int64_t)i * W + j;
      step = back ? -W : W;
      wrap = back ? to_top : -to_top;
      left = back ? (int)i : H - 1 - (int)i;
      run = H - 1;
    }
  }
  // whether the next step is behind a column's end
  __device__ __forceinline__ bool next() {
    const bool end = left == 0;
    left = end ? run : left - 1;
    return end;
  }
};
// One operand's rows along a walk, `ld` bytes apart: a uniform address, to which a lane
// adds its column (the form of address that needs no vector arithmetic).
struct RecRow {
  char* p;
  int64_t step, wrap;
  __device__ __forceinline__ RecRow(const void* base, int64_t first, int64_t ld, const RecWalk& w)
      : p(static_cast<char*>(const_cast<void*>(base)) + (first + w.row) * ld), step(w.step * ld), wrap(w.wrap * ld) {}
  __device__ __forceinline__ void next(bool end) { p += end ? wrap : step; }
};

// ---------------------------------------------------------------------------
// gates
// ---------------------------------------------------------------------------
// In powers of two: a = 2^y with y = g log2(e), or of a logit (min(g, 0) log2(e) - l) / tau
// with l = log2(1 + u), u = exp(-|g|): the machine's exponential and logarithm as they
// are, three of them per logit. w = 1 + u loses the low bits of a small u, of which
// 1 - a would keep the relative error; l takes them back as r / w log2(e), r = u - (w - 1)
// exactly, where w is so close to 1 that it does not divide (r is 2^-24 at most, and l
// at least 0.58 where w is 1.5).
// 1 - 2^y is the exponential's series about 0 up to |y ln 2| = 1/4 (what is left out is
// under 2^-24 of it), else as it stands: 10 roundings of a at most.
// a, 1 - a where KEEP, and d log a / d g where SLOPE.
template <bool LOGITS, bool KEEP, bool SLOPE>
__device__ __forceinline__ void rec_gate(float g, float inv_tau, float& a, float& keep, float& slope) {
  constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
  float y;
  if constexpr (LOGITS) {
    const float u = __builtin_amdgcn_exp2f(-fabsf(g) * kLog2e), w = 1.f + u;
    const float l = fmaf(u - (w - 1.f), kLog2e, __builtin_amdgcn_logf(w));
    y = fmaf(fminf(g, 0.f), kLog2e, -l) * inv_tau;
    if constexpr (SLOPE) slope = (g < 0.f ? 1.f : u) * __builtin_amdgcn_rcpf(w) * inv_tau;
  } else {
    y = g * kLog2e;
  }
  a = __builtin_amdgcn_exp2f(y);
  if constexpr (KEEP) {
    constexpr float l2 = kLn2 * kLn2, l3 = l2 * kLn2, l4 = l2 * l2;
    float s = l4 * l2 / 720.f;
    s = fmaf(s, y, l4 * kLn2 / 120.f);
    s = fmaf(s, y, l4 / 24.f);
    s = fmaf(s, y, l3 / 6.f);
    s = fmaf(s, y, l2 / 2.f);
    s = fmaf(s, y, kLn2);
    keep = fabsf(y) < 0.25f * kLog2e ? -y * s : 1.f - a;
  }
}

// ---------------------------------------------------------------------------
// the scan of a tile
// ---------------------------------------------------------------------------
// A work-group takes a tile: the channels of a block (V per lane), T steps per wave. Each
// wave composes its own steps (P, E), the waves' maps meet in LDS, and the state before
// the tile comes from the tiles before it in one launch, by look-back:
//
//   - every tile hands on its map, in one 64-bit word per channel that is its own flag
//     (rec_words.h). Words travel by device-scope atomic loads and stores, so no cache is
//     written back or dropped for them;
//   - tiles are in groups. The last tile of a group hands on the state behind the group,
//     for which it waits for that of the group before. A tile composes the maps of the tiles
//     before it in its group, shared out over its waves, and applies them to that state.
//
// So a sequence of n tiles has a chain of n / group hand-overs, and the composition is the
// same whatever the order in which work-groups run: results do not depend on it. Tiles are
// numbered by a counter as their work-groups start, the first steps of all of its sequences
// first: what a tile waits for has started before it, and a map is handed on before
// anything is waited for, so every wait ends, whatever else the device is running. (By
// work-group index instead, two calls on two streams could fill each other's chiplets with
// work-groups that wait for ones not started. Waits are bounded all the same: of one that
// runs out its work-group's states are NaN, and the one that it hands on behind a group; its
// own map was handed on before, so others of its group go on.) A counter hands out 80 numbers
// per microsecond. Where that counts, in short calls, there are up to 32, each for sequences of
// its own (8 x 1600 x 384 fp16 17.4 us, with one 19.4; 64 x 400 x 384 21.5, 25.5); in long ones a single counter keeps
// blocks of channels that lie next to each other next to each other in time too, which the
// memory wants (32768 x 4096 bf16 172 us, with 32 counters 220; backward 4 x 16384 x 2048 322, 351).
struct RecTiles {
  unsigned long long* maps;    // [sequences][tiles][64 V]
  unsigned long long* states;  // [sequences][groups][64 V]
  unsigned* counters;          // the next tile of each `share` sequences; null where a sequence is one tile
  int tiles, group, groups, blocks;
  unsigned share, lanes;       // sequences per counter, counters
  unsigned spin;
};

constexpr int kRecWaves = 16;
constexpr unsigned kRecCounters = 32, kRecCounterStep = 32;  // at most; words from one to the next (128 bytes)

struct RecWhere {
  int tile, seq, b, block;  // uniform
};
// Which tile this work-group takes; false if none. Work-groups of index i mod `lanes`
// share counter i, which numbers the tiles of its own sequences.
__device__ __forceinline__ bool rec_where(const RecTiles& t, unsigned sequences, RecWhere& w) {
  unsigned tile, seq;
  if (t.counters) {
    __shared__ unsigned mine;
    const unsigned lane = blockIdx.x % t.lanes;
    if (threadIdx.x == 0) mine = atomicAdd(t.counters + kRecCounterStep * lane, 1u);
    __syncthreads();
    const unsigned id = (unsigned)__builtin_amdgcn_readfirstlane((int)mine);
    tile = id / t.share;
    seq = lane * t.share + (id - tile * t.share);
  } else {
    tile = blockIdx.x / sequences;
    seq = blockIdx.x - tile * sequences;
  }
  w.tile = (int)tile;
  w.seq = (int)seq;
  w.b = w.seq / t.blocks;
  w.block = w.seq - w.b * t.blocks;
  return seq < sequences;
}

// The state s before this wave's steps, of which (P, E) is the map. The first wave of a
// sequence comes with the state before the sequence as s and with the map that leads to its
// last state from anywhere (P = 0), so that nobody else reads the first state: a caller's
// may lie where the last state goes.
template <int V>
__device__ __forceinline__ void rec_carry(const RecTiles& t, const RecWhere& at, int wave, int lane, const float (&P)[V],
                                          const float (&E)[V], float (&s)[V]) {
  constexpr int CB = 64 * V;
  __shared__ float own[kRecWaves][2][CB], before[kRecWaves][2][CB], behind[CB];
  const int waves = blockDim.x >> 6, c = lane * V;
  if (waves == 1 && t.tiles == 1) return;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    own[wave][0][c + v] = P[v];
    own[wave][1][c + v] = E[v];
  }
  __syncthreads();
  const int group = at.tile / t.group, k = at.tile % t.group;  // k tiles before it in its group
  const bool hands_state = k == t.group - 1, last = at.tile == t.tiles - 1;
  float tP[V], tE[V];
  if (wave == 0 && !last) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      tP[v] = 1.f;
      tE[v] = 0.f;
    }
    for (int w = 0; w < waves; ++w)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float p = own[w][0][c + v];
        tE[v] = fmaf(p, tE[v], own[w][1][c + v]);
        tP[v] *= p;
      }
    if (!hands_state) {
      unsigned long long* m = t.maps + ((int64_t)at.seq * t.tiles + at.tile) * CB + c;
#pragma unroll
      for (int v = 0; v < V; ++v)
        __hip_atomic_store(m + v, rec_word(tP[v], tE[v]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  if (at.tile > 0) {
    const int per = (k + waves - 1) / waves, j0 = wave * per, j1 = min(k, j0 + per);
    float bP[V], bE[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      bP[v] = 1.f;
      bE[v] = 0.f;
    }
    constexpr int U = 4;
    const unsigned long long* m = t.maps + ((int64_t)at.seq * t.tiles + (int64_t)group * t.group) * CB + c;
    for (int j = j0; j < j1; j += U) {
      unsigned long long w[U][V];
      const unsigned long long* p[U];
#pragma unroll
      for (int u = 0; u < U; ++u) p[u] = m + (int64_t)min(j + u, j1 - 1) * CB;
      rec_wait<V, U>(w, p, t.spin);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (j + u >= j1) break;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          bE[v] = fmaf(rec_map(w[u][v]), bE[v], rec_add(w[u][v]));
          bP[v] *= rec_map(w[u][v]);
        }
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      before[wave][0][c + v] = bP[v];
      before[wave][1][c + v] = bE[v];
    }
    if (wave == waves - 1) {  // (the wave with the fewest maps)
      float g[V];
#pragma unroll
      for (int v = 0; v < V; ++v) g[v] = 0.f;
      if (group > 0) {
        unsigned long long w[1][V];
        const unsigned long long* p[1] = {t.states + ((int64_t)at.seq * t.groups + group - 1) * CB + c};
        rec_wait<V, 1>(w, p, t.spin);
#pragma unroll
        for (int v = 0; v < V; ++v) g[v] = rec_add(w[0][v]);
      }
#pragma unroll
      for (int v = 0; v < V; ++v) behind[c + v] = g[v];
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = behind[c + v];
    const int used = min(waves, per ? (k + per - 1) / per : 0);
    for (int w = 0; w < used; ++w)
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = fmaf(before[w][0][c + v], s[v], before[w][1][c + v]);
  }
  if (wave == 0 && hands_state && !last) {
    unsigned long long* m = t.states + ((int64_t)at.seq * t.groups + group) * CB + c;
#pragma unroll
    for (int v = 0; v < V; ++v)
      __hip_atomic_store(m + v, rec_word(0.f, fmaf(tP[v], s[v], tE[v])), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
  }
  for (int w = 0; w < wave; ++w)
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = fmaf(own[w][0][c + v], s[v], own[w][1][c + v]);
}

struct RecFwd {
  RecTiles t;
  const char *x, *g;
  char* h;
  const float* h0;
  float* h_final;
  int64_t x_ld, g_ld;  // bytes from row to row
  int64_t L;
  int H, W, d, dir;
  unsigned sequences;
  float inv_tau;
};

// A lane's V channels from c on: the last lane of an odd width starts early and leaves
// the `skip` channels that are another lane's to it; lanes past the width repeat the last
// one's and store nothing.
template <int V>
struct RecCols {
  int c, skip;
  __device__ __forceinline__ RecCols(int block, int lane, int d) {
    const int at = (block * 64 + lane) * V;
    c = min(at, d - V);
    skip = min(V, at - c);
  }
};
template <int DT, int V>
__device__ __forceinline__ void rec_store(const RecVec<DT, V>& r, char* p, int skip) {
  if (skip == 0) {
    r.store(p);
  } else {
#pragma unroll
    for (int v = 1; v < V; ++v)
      if (v >= skip) r.store1(p, v);
  }
}

// Rows' addresses are formed one after the other: the compiler would form all of them
// ahead and spill scalar registers for it.
__device__ __forceinline__ void rec_fence() { __builtin_amdgcn_sched_barrier(0); }

// Both kernels ask for all of a wave's rows at once and keep its gates in registers across
// the look-back. A whole wave (all T steps, no channels that two lanes have) has a way of
// its own without masks and tests per row (32768 x 4096 bf16 forward 172 us, with the other way
// alone 199; 4 x 16384 x 2048 bf16 backward 322, 373; 8 x 1600 x 384 fp16 17.4, 22.7). Odd
// widths have the other way in all of their waves.
template <int DT, int GT, int V, int T, bool LOGITS, bool COMPLEMENT>
__global__ void __launch_bounds__(64 * (T == 1 ? 1 : kRecWaves)) rec_fwd_kernel(RecFwd p) {
  constexpr int ES = RecVec<DT, V>::ES, GS = RecVec<GT, V>::ES;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  RecWhere at;
  if (!rec_where(p.t, p.sequences, at)) return;
  const RecCols<V> k(at.block, lane, p.d);
  const int64_t s0 = ((int64_t)at.tile * waves + wave) * T;
  const int n = (int)min((int64_t)T, p.L - s0);  // this wave's steps (none: 0 or less)
  const bool first = s0 == 0;
  float s[V];
#pragma unroll
  for (int v = 0; v < V; ++v) s[v] = first && p.h0 ? p.h0[(int64_t)at.b * p.d + k.c + v] : 0.f;
  const int64_t row0 = at.b * p.L;
  const unsigned cx = (unsigned)k.c * ES, cg = (unsigned)k.c * GS;
  const bool whole = T > 1 && n == T && p.d % V == 0;
  float a[T][V], b[T][V], P[V], E[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    P[v] = first ? 0.f : 1.f;
    E[v] = s[v];
  }
  auto gate = [&](const RecVec<DT, V>& rx, const RecVec<GT, V>& rg, float (&at)[V], float (&bt)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float keep = 0.f, slope;
      rec_gate<LOGITS, COMPLEMENT, false>(rg.get(v), p.inv_tau, at[v], keep, slope);
      bt[v] = COMPLEMENT ? keep * rx.get(v) : rx.get(v);
    }
  };
  if (whole) {
    RecWalk w(s0, p.L, p.H, p.W, p.dir);
    RecRow x(p.x, row0, p.x_ld, w), g(p.g, row0, p.g_ld, w);
    RecVec<DT, V> rx[T];
    RecVec<GT, V> rg[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      rx[t].load(x.p + cx);
      rg[t].load(g.p + cg);
      const bool end = w.next();
      x.next(end);
      g.next(end);
      rec_fence();
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
      gate(rx[t], rg[t], a[t], b[t]);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        E[v] = fmaf(a[t][v], E[v], b[t][v]);
        P[v] *= a[t][v];
      }
    }
  } else if (n > 0) {
    RecWalk w(s0, p.L, p.H, p.W, p.dir);
    RecRow x(p.x, row0, p.x_ld, w), g(p.g, row0, p.g_ld, w);
    RecVec<DT, V> rx[T];
    RecVec<GT, V> rg[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      rx[t].load(x.p + cx);
      rg[t].load(g.p + cg);
      if (t + 1 < n) {  // (steps past the end read the last row again)
        const bool end = w.next();
        x.next(end);
        g.next(end);
      }
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
      gate(rx[t], rg[t], a[t], b[t]);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        a[t][v] = t < n ? a[t][v] : 1.f;
        b[t][v] = t < n ? b[t][v] : 0.f;
        E[v] = fmaf(a[t][v], E[v], b[t][v]);
        P[v] *= a[t][v];
      }
    }
  }
  if constexpr (T > 1) rec_carry<V>(p.t, at, wave, lane, P, E, s);
  if (n <= 0 || k.skip == V) return;
  RecWalk w(s0, p.L, p.H, p.W, p.dir);
  RecRow h(p.h, row0, (int64_t)p.d * ES, w);
  if (whole) {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      RecVec<DT, V> r;
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = fmaf(a[t][v], s[v], b[t][v]);
      r.set(s);
      r.store(h.p + cx);
      h.next(w.next());
      rec_fence();
    }
  } else {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      // (past the end a = 1 and b = 0: the state stays)
      RecVec<DT, V> r;
#pragma unroll
      for (int v = 0; v < V; ++v) s[v] = fmaf(a[t][v], s[v], b[t][v]);
      r.set(s);
      if (t < n) rec_store(r, h.p + cx, k.skip);
      h.next(w.next());
    }
  }
  if (p.h_final && s0 + n == p.L) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v >= k.skip) p.h_final[(int64_t)at.b * p.d + k.c + v] = s[v];
  }
}

struct RecBwd {
  RecTiles t;
  const char *dh, *g, *h, *x;
  const float *h0, *dh_final;
  char *dx, *dg;
  float* dh0;
  int64_t x_ld, g_ld, dx_ld, dg_ld;
  int64_t L;
  int H, W, d, dir;  // dir: the reversed order
  unsigned sequences;
  float inv_tau;
};

// As the forward pass, in the reversed order: the state is Y, a step's map Y -> a (dh + Y).
template <int DT, int GT, int V, int T, bool LOGITS, bool COMPLEMENT>
__global__ void __launch_bounds__(64 * (T == 1 ? 1 : kRecWaves)) rec_bwd_kernel(RecBwd p) {
  constexpr int ES = RecVec<DT, V>::ES, GS = RecVec<GT, V>::ES;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  RecWhere at;
  if (!rec_where(p.t, p.sequences, at)) return;
  const RecCols<V> k(at.block, lane, p.d);
  const int64_t s0 = ((int64_t)at.tile * waves + wave) * T, state = (int64_t)at.b * p.d + k.c;
  const int n = (int)min((int64_t)T, p.L - s0);
  const bool first = s0 == 0;
  float y[V];
#pragma unroll
  for (int v = 0; v < V; ++v) y[v] = first && p.dh_final ? p.dh_final[state + v] : 0.f;
  const int64_t row0 = at.b * p.L, dense = (int64_t)p.d * ES;
  const unsigned cx = (unsigned)k.c * ES, cg = (unsigned)k.c * GS;
  const bool whole = T > 1 && n == T && p.d % V == 0 && p.dx && p.dg;
  const bool to_start = s0 + n == p.L;  // this wave has the scan's first token, before which the state is h0
  RecVec<DT, V> rd[T];
  float a[T][V], keep[T][V], m[T][V], P[V], E[V], h0[V];  // m: dg over Y
#pragma unroll
  for (int v = 0; v < V; ++v) {
    P[v] = first ? 0.f : 1.f;
    E[v] = y[v];
    h0[v] = to_start && p.h0 ? p.h0[state + v] : 0.f;
  }
  // a step's gate, and the state before it
  auto gate = [&](int t, const RecVec<GT, V>& g, const RecVec<DT, V>& x, const RecVec<DT, V>& h, bool start) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float slope;
      rec_gate<LOGITS, COMPLEMENT, true>(g.get(v), p.inv_tau, a[t][v], keep[t][v], slope);
      m[t][v] = start ? h0[v] : h.get(v);
      if constexpr (COMPLEMENT) m[t][v] -= x.get(v);
      if constexpr (LOGITS) m[t][v] *= slope;
    }
  };
  if (whole) {
    RecWalk w(s0, p.L, p.H, p.W, p.dir);
    RecRow dh(p.dh, row0, dense, w), g(p.g, row0, p.g_ld, w), x(p.x, row0, p.x_ld, w), h(p.h, row0, dense, w);
    RecVec<GT, V> rg[T];
    RecVec<DT, V> rh[T], rx[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      rd[t].load(dh.p + cx);
      rg[t].load(g.p + cg);
      if constexpr (COMPLEMENT) rx[t].load(x.p + cx);
      const bool end = w.next();
      if (t + 1 < T || !to_start) h.next(end);
      rh[t].load(h.p + cx);  // the row before; of the scan's first token its own, which is not used
      dh.next(end);
      g.next(end);
      x.next(end);
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
      gate(t, rg[t], rx[t], rh[t], t + 1 == T && to_start);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        E[v] = a[t][v] * (rd[t].get(v) + E[v]);
        P[v] *= a[t][v];
      }
    }
  } else if (n > 0) {
    RecWalk w(s0, p.L, p.H, p.W, p.dir);
    RecRow dh(p.dh, row0, dense, w), g(p.g, row0, p.g_ld, w), x(p.x, row0, p.x_ld, w), h(p.h, row0, dense, w);
    RecVec<GT, V> rg[T];
    RecVec<DT, V> rh[T], rx[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      rd[t].load(dh.p + cx);
      rg[t].load(g.p + cg);
      if constexpr (COMPLEMENT) rx[t].load(x.p + cx);
      const bool inside = t + 1 < n;  // (steps past the end read the last row again)
      if (inside || (t + 1 == n && !to_start)) {
        const bool end = w.next();
        h.next(end);
        if (inside) {
          dh.next(end);
          g.next(end);
          x.next(end);
        }
      }
      rh[t].load(h.p + cx);
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
      gate(t, rg[t], rx[t], rh[t], t + 1 == n && to_start);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        E[v] = t < n ? a[t][v] * (rd[t].get(v) + E[v]) : E[v];
        P[v] = t < n ? P[v] * a[t][v] : P[v];
      }
    }
  }
  if constexpr (T > 1) rec_carry<V>(p.t, at, wave, lane, P, E, y);
  if (n <= 0 || k.skip == V) return;
  RecWalk w(s0, p.L, p.H, p.W, p.dir);
  RecRow dx(p.dx, row0, p.dx_ld, w), dg(p.dg, row0, p.dg_ld, w);
  // one step's gradients
  auto out = [&](int t, RecVec<DT, V>& ox, RecVec<GT, V>& og) {
    float fx[V], fg[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float D = rd[t].get(v) + y[v];
      y[v] = a[t][v] * D;
      fx[v] = COMPLEMENT ? keep[t][v] * D : D;
      fg[v] = y[v] * m[t][v];
    }
    ox.set(fx);
    og.set(fg);
  };
  if (whole) {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      RecVec<DT, V> ox;
      RecVec<GT, V> og;
      out(t, ox, og);
      ox.store(dx.p + cx);
      og.store(dg.p + cg);
      const bool end = w.next();
      dx.next(end);
      dg.next(end);
    }
  } else {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      if (t < n) {
        RecVec<DT, V> ox;
        RecVec<GT, V> og;
        out(t, ox, og);
        if (p.dx) rec_store(ox, dx.p + cx, k.skip);
        if (p.dg) rec_store(og, dg.p + cg, k.skip);
        const bool end = w.next();
        dx.next(end);
        dg.next(end);
      }
    }
  }
  if (p.dh0 && to_start) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v >= k.skip) p.dh0[state + v] = y[v];
  }
}

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
__global__ void __launch_bounds__(256) rec_clear_kernel(u32x4* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = u32x4{0, 0, 0, 0};
}

}  // namespace gtr

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
namespace gtr {

// Steps of a wave and waves of a tile: what a work-group holds in registers and moves
// while it has them decides how busy it keeps the memory (two work-groups per CU). Us of
// 16, 8 and 4 waves, forward with 16 steps: 32768 x 4096 bf16 178, 172, 231; 16384 x 4096
// float32 175, 156, 172; 8 x 1600 x 384 fp16 19.5, 17.4, 20.2 (8 waves of 8 steps: 244, 170,
// 19.6); backward: 4 x 16384 x 2048 bf16 336, 322, 368; 4 x 16384 x 1024 float32 321, 300, 330;
// 1600 x 192 fp16 14.4, 11.7, 11.6. A sequence that 16 waves take is one tile.
constexpr int kRecFwdSteps = 16, kRecBwdSteps = 8;
// Backward steps of 16-bit types where sequences are several tiles and all together more than
// the CUs: as many as the registers hold (float16 logits with 1 - a keep 7 of them in scratch
// memory). Us with 8 / with these, float16 logits without and with 1 - a: 8 x 1600 x 384 23.7 /
// 20.4, 25.3 / 22.0; 64 x 400 x 384 27.6 / 27.1, 30.9 / 29.6; 1 x 16384 x 1024 60.6 / 52.1, 65.6
// / 61.3; 4 x 16384 x 2048 307 / 277, 332 / 327. Few tiles lose: 1 x 1600 x 384 11.1 / 12.1, 11.9
// / 12.8, and sequences of one tile: 1000 x 64 x 384 44.3 / 58.7, 53.1 / 75.0. (Of 129 to 192 tokens,
// several tiles of 8 steps but one of these, they gain as well: 64 x 129 x 384 15.4 / 11.3, 17.3 /
// 13.8; 64 x 160 x 384 15.4 / 12.3, 17.3 / 13.0; 300 x 129 x 384 46.3 / 37.4, 50.5 / 51.2; 300 x
// 192 x 384 49.4 / 44.9.) In float32 they do
// not fit (4 x 16384 x 1024 log decays with 1 - a 298, with 12 steps 369).
// Short sequences, a few tokens of each of many: fewer steps, so that more waves share them.
// Us forward with 16 / with 4, fp16 logits with 1 - a: 4000 x 2 x 384 61 / 22, 32 x 4 x 2048 6.3
// / 3.5, 512 x 16 x 384 11.4 / 8.0, 512 x 32 x 384 15.3 / 12.5, 512 x 48 x 384 15.6 / 17.3;
// backward with 8 / with 4: 45 / 33, 5.5 / 4.1, 12.7 / 10.3, and 512 x 24 x 384 14.0 / 15.9.
constexpr int kRecFew = 4, kRecFwdFew = 32, kRecBwdFew = 16;  // steps; tokens up to which
constexpr int kRecBwdMore = 12, kRecBwdMoreKeep = 10, kRecCus = 256;
constexpr int kRecTileWaves = 8;
constexpr unsigned kRecSpin = 1u << 22;             // polls of a wait, of a microsecond or less each

static int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct RecPlan {
  int V, T, waves;
  RecTiles t;
  int64_t sequences, grid;
  size_t need, clear;  // bytes of workspace, of which those that are cleared
};

// few: the tokens up to which a wave takes kRecFew steps
static gtr_status rec_plan(int32_t B, int32_t H, int32_t W, int32_t d, int steps, int few, RecPlan* r) {
  // a lane's byte within a row is a 32-bit number
  if (B <= 0 || H <= 0 || W <= 0 || d <= 0 || d > 1 << 29) return GTR_ERR_SHAPE;
  const int64_t L = (int64_t)H * W;
  if (L >= (int64_t)1 << 31) return GTR_ERR_SHAPE;
  r->V = d == 1 ? 1 : 2;
  r->T = L == 1 ? 1 : L <= few ? kRecFew : steps;
  const int64_t waves = (L + r->T - 1) / r->T;
  r->waves = (int)(waves <= kRecWaves ? waves : kRecTileWaves);
  const int64_t tiles = (waves + r->waves - 1) / r->waves;
  r->t = RecTiles{};
  r->t.tiles = (int)tiles;
  r->t.blocks = (d + 64 * r->V - 1) / (64 * r->V);
  r->sequences = (int64_t)B * r->t.blocks;
  if (r->sequences >= (int64_t)1 << 26) return GTR_ERR_SHAPE;  // (more threads than a launch has, see below)
  // a hand-over between groups takes about 2 us, in which the sequences' tiles of a group
  // are read (about 20 ns each): enough of them that the chain does not set the pace, and no
  // more, for maps to be composed again cost more than the hand-over (us forward, backward in
  // groups of 8 / 4, fp16 with 1 - a: 16 x 1600 x 384 23.7 / 22.8, 33.1 / 32.7; 16 x 8192 x 128
  // 37.2 / 35.2, 56.7 / 53.4; 1 x 32768 x 4096 190 / 184, 329 / 323; of 16 sequences of 16384
  // tokens the chain is the longer: 62 / 58, 110 / 113). With one sequence of 65536 x 128 groups
  // of 64, 32, 16 take 31, 38, 51.
  r->t.group = r->sequences >= 16 ? 4 : r->sequences >= 8 ? 16 : r->sequences >= 4 ? 32 : 64;
  r->t.groups = (int)((tiles + r->t.group - 1) / r->t.group);
  r->t.spin = kRecSpin;
  r->t.share = (unsigned)(r->sequences * tiles <= 2048 ? up(r->sequences, kRecCounters) : r->sequences);
  r->t.lanes = (unsigned)up(r->sequences, r->t.share);
  r->grid = tiles > 1 ? (int64_t)r->t.share * r->t.lanes * tiles : r->sequences;
  // a launch's threads stay below 2^32
  if (r->grid > (((int64_t)1 << 32) - 1) / (64 * r->waves)) return GTR_ERR_SHAPE;
  r->need = r->clear = 0;
  if (tiles > 1) {
    const size_t words = (size_t)r->sequences * (size_t)(tiles + r->t.groups) * 64 * r->V;
    r->clear = r->need = kRecCounters * kRecCounterStep * 4 + words * 8;
  }
  return GTR_OK;
}

static gtr_status rec_types(int dtype, int g_dtype, int g_kind, float tau, int scan) {
  if (dtype != GTR_F32 && dtype != GTR_F16 && dtype != GTR_BF16) return GTR_ERR_UNSUPPORTED;
  if (g_dtype != dtype && g_dtype != GTR_F32) return GTR_ERR_UNSUPPORTED;
  if (scan < GTR_SCAN_ROW || scan > GTR_SCAN_COL_REV) return GTR_ERR_UNSUPPORTED;
  if (g_kind != GTR_GATE_LOG_DECAY && g_kind != GTR_GATE_LOGITS) return GTR_ERR_UNSUPPORTED;
  if (g_kind == GTR_GATE_LOGITS && !(tau > 0.f && 1.f / tau <= 3.0e38f && tau <= 3.0e38f)) return GTR_ERR_UNSUPPORTED;
  return GTR_OK;
}

// The rows of an operand: n rows of `width` bytes, `ld` bytes apart.
struct RecRows {
  const void* p;
  int64_t n, ld, width;
};
static bool rec_rows(const void* p, int64_t n, int64_t ld, int32_t d, int es, RecRows* r) {
  if (ld == 0) ld = d;
  int64_t bytes;
  if (ld < d || __builtin_mul_overflow(ld, (int64_t)es, &bytes) || __builtin_mul_overflow(bytes, n, &bytes) ||
      bytes > (int64_t)1 << 62)
    return false;
  *r = RecRows{p, n, ld * es, (int64_t)d * es};
  return true;
}
static Bytes rec_bytes(const RecRows& r) { return {r.p, (size_t)((r.n - 1) * r.ld + r.width)}; }
// Rows that lie between each other's (two halves of one matrix) do not meet.
static bool rows_meet(const RecRows& a, const RecRows& b) {
  if (!bytes_meet(rec_bytes(a), rec_bytes(b))) return false;
  if (a.ld != b.ld) return true;
  const RecRows &lo = a.p <= b.p ? a : b, &hi = a.p <= b.p ? b : a;
  const int64_t off = (int64_t)((reinterpret_cast<uintptr_t>(hi.p) - reinterpret_cast<uintptr_t>(lo.p)) % (uint64_t)a.ld);
  return off < lo.width || off + hi.width > a.ld;
}
static bool same_rows(const RecRows& a, const RecRows& b) { return a.p == b.p && a.ld == b.ld && a.width == b.width; }
static RecRows flat_rows(const void* p, int64_t bytes) { return {p, 1, bytes, bytes}; }
static bool rec_misaligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

static gtr_status rec_workspace(const RecPlan& r, const void* ws, size_t bytes) {
  if (r.need && (!ws || rec_misaligned(ws, 256) || bytes < r.need)) return GTR_ERR_WORKSPACE;
  return GTR_OK;
}

// Lays the tiles' words out and clears them (with a kernel: the call may be captured).
static void rec_words(RecPlan* r, void* ws, uint32_t spin, hipStream_t stream) {
  if (spin) r->t.spin = spin;
  if (!r->need) return;
  r->t.counters = static_cast<unsigned*>(ws);
  r->t.maps = reinterpret_cast<unsigned long long*>(static_cast<char*>(ws) + kRecCounters * kRecCounterStep * 4);
  r->t.states = r->t.maps + r->sequences * r->t.tiles * 64 * r->V;
  const int64_t n = (int64_t)(r->clear / 16), blocks = (n + 255) / 256;
  hipLaunchKernelGGL(rec_clear_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, stream,
                     static_cast<u32x4*>(ws), n);
}

template <class P>
struct RecLaunch {
  P p;
  const RecPlan& r;
  hipStream_t stream;
};
template <int DT, int GT, int V, int T, bool LOGITS, bool COMPLEMENT>
static void rec_go(const RecLaunch<RecFwd>& a) {
  hipLaunchKernelGGL((rec_fwd_kernel<DT, GT, V, T, LOGITS, COMPLEMENT>), dim3((unsigned)a.r.grid), dim3(64 * a.r.waves), 0,
                     a.stream, a.p);
}
template <int DT, int GT, int V, int T, bool LOGITS, bool COMPLEMENT>
static void rec_go(const RecLaunch<RecBwd>& a) {
  hipLaunchKernelGGL((rec_bwd_kernel<DT, GT, V, T, LOGITS, COMPLEMENT>), dim3((unsigned)a.r.grid), dim3(64 * a.r.waves), 0,
                     a.stream, a.p);
}
template <int STEPS, int DT, int GT, bool LOGITS, bool COMPLEMENT, class P>
static void rec_sized(const RecLaunch<P>& a) {
  constexpr int FEW = kRecFew;
  if (a.r.V == 1)
    a.r.T == 1     ? rec_go<DT, GT, 1, 1, LOGITS, COMPLEMENT>(a)
    : a.r.T == FEW ? rec_go<DT, GT, 1, FEW, LOGITS, COMPLEMENT>(a)
                   : rec_go<DT, GT, 1, STEPS, LOGITS, COMPLEMENT>(a);
  else
    a.r.T == 1     ? rec_go<DT, GT, 2, 1, LOGITS, COMPLEMENT>(a)
    : a.r.T == FEW ? rec_go<DT, GT, 2, FEW, LOGITS, COMPLEMENT>(a)
                   : rec_go<DT, GT, 2, STEPS, LOGITS, COMPLEMENT>(a);
}
template <int STEPS, int DT, int GT, class P>
static void rec_kind(const RecLaunch<P>& a, bool logits, bool complement) {
  if constexpr (STEPS == kRecBwdSteps && DT != GTR_F32) {
    if (a.r.T == kRecBwdMore)
      return logits ? rec_sized<kRecBwdMore, DT, GT, true, false>(a) : rec_sized<kRecBwdMore, DT, GT, false, false>(a);
    if (a.r.T == kRecBwdMoreKeep)
      return logits ? rec_sized<kRecBwdMoreKeep, DT, GT, true, true>(a) : rec_sized<kRecBwdMoreKeep, DT, GT, false, true>(a);
  }
  if (logits)
    complement ? rec_sized<STEPS, DT, GT, true, true>(a) : rec_sized<STEPS, DT, GT, true, false>(a);
  else
    complement ? rec_sized<STEPS, DT, GT, false, true>(a) : rec_sized<STEPS, DT, GT, false, false>(a);
}
template <int STEPS, class P>
static gtr_status rec_launch(const RecLaunch<P>& a, int dt, int gt, bool logits, bool complement) {
  if (dt == GTR_F32)
    rec_kind<STEPS, GTR_F32, GTR_F32>(a, logits, complement);
  else if (dt == GTR_F16)
    gt == dt ? rec_kind<STEPS, GTR_F16, GTR_F16>(a, logits, complement) : rec_kind<STEPS, GTR_F16, GTR_F32>(a, logits, complement);
  else
    gt == dt ? rec_kind<STEPS, GTR_BF16, GTR_BF16>(a, logits, complement) : rec_kind<STEPS, GTR_BF16, GTR_F32>(a, logits, complement);
  return hipGetLastError() == hipSuccess ? GTR_OK : GTR_ERR_HIP;
}

static gtr_status rec_fwd_plan(const gtr_recurrence_fwd_args* a, RecPlan* r) {
  if (!a) return GTR_ERR_NULL;
  const gtr_status st = rec_plan(a->B, a->H, a->W, a->d, kRecFwdSteps, kRecFwdFew, r);
  return st != GTR_OK ? st : rec_types(a->dtype, a->g_dtype, a->g_kind, a->gate_tau, a->scan);
}
static gtr_status rec_bwd_plan(const gtr_recurrence_bwd_args* a, RecPlan* r) {
  if (!a) return GTR_ERR_NULL;
  gtr_status st = rec_plan(a->B, a->H, a->W, a->d, kRecBwdSteps, kRecBwdFew, r);
  if (st == GTR_OK && r->t.tiles > 1 && a->dtype != GTR_F32 && r->sequences * r->t.tiles > kRecCus)
    st = rec_plan(a->B, a->H, a->W, a->d, a->complement ? kRecBwdMoreKeep : kRecBwdMore, 0, r);
  return st != GTR_OK ? st : rec_types(a->dtype, a->g_dtype, a->g_kind, a->gate_tau, a->scan);
}

}  // namespace gtr

using namespace gtr;

extern "C" size_t gtr_recurrence_fwd_workspace_size(const gtr_recurrence_fwd_args* a) {
  RecPlan r;
  return rec_fwd_plan(a, &r) == GTR_OK ? r.need : 0;
}

extern "C" gtr_status gtr_recurrence_fwd(const gtr_recurrence_fwd_args* a, hipStream_t stream) {
  RecPlan r;
  gtr_status st = rec_fwd_plan(a, &r);
  if (st != GTR_OK) return st;
  if (!a->x || !a->g || !a->h) return GTR_ERR_NULL;
  const int es = (int)dtype_size(a->dtype), gs = (int)dtype_size(a->g_dtype);
  const int64_t L = (int64_t)a->H * a->W, n = a->B * L, state = (int64_t)a->B * a->d * 4;
  RecRows x, g, h;
  if (!rec_rows(a->x, n, a->x_ld, a->d, es, &x) || !rec_rows(a->g, n, a->g_ld, a->d, gs, &g) ||
      !rec_rows(a->h, n, 0, a->d, es, &h))
    return GTR_ERR_SHAPE;
  if (rec_misaligned(a->x, es) || rec_misaligned(a->g, gs) || rec_misaligned(a->h, es) || rec_misaligned(a->h0, 4) ||
      rec_misaligned(a->h_final, 4))
    return GTR_ERR_UNSUPPORTED;
  st = rec_workspace(r, a->workspace, a->workspace_bytes);
  if (st != GTR_OK) return st;
  const RecRows h0 = flat_rows(a->h0, state), last = flat_rows(a->h_final, state),
                ws = flat_rows(r.need ? a->workspace : nullptr, (int64_t)r.need);
  if ((rows_meet(h, x) && !same_rows(h, x)) || rows_meet(h, g) || rows_meet(h, h0) || rows_meet(h, last) || rows_meet(h, ws) ||
      rows_meet(last, x) || rows_meet(last, g) || (rows_meet(last, h0) && last.p != h0.p) || rows_meet(last, ws) ||
      rows_meet(ws, x) || rows_meet(ws, g) || rows_meet(ws, h0))
    return GTR_ERR_ALIAS;
  rec_words(&r, a->workspace, a->spin_limit, stream);
  RecFwd p = {};
  p.t = r.t;
  p.x = static_cast<const char*>(a->x);
  p.g = static_cast<const char*>(a->g);
  p.h = static_cast<char*>(a->h);
  p.h0 = a->h0;
  p.h_final = a->h_final;
  p.x_ld = x.ld;
  p.g_ld = g.ld;
  p.L = L;
  p.H = a->H;
  p.W = a->W;
  p.d = a->d;
  p.dir = a->scan;
  p.sequences = (unsigned)r.sequences;
  p.inv_tau = a->g_kind == GTR_GATE_LOGITS ? 1.f / a->gate_tau : 1.f;
  return rec_launch<kRecFwdSteps>(RecLaunch<RecFwd>{p, r, stream}, a->dtype, a->g_dtype, a->g_kind == GTR_GATE_LOGITS,
                                  a->complement != 0);
}

extern "C" size_t gtr_recurrence_bwd_workspace_size(const gtr_recurrence_bwd_args* a) {
  RecPlan r;
  return rec_bwd_plan(a, &r) == GTR_OK ? r.need : 0;
}

extern "C" gtr_status gtr_recurrence_bwd(const gtr_recurrence_bwd_args* a, hipStream_t stream) {
  RecPlan r;
  gtr_status st = rec_bwd_plan(a, &r);
  if (st != GTR_OK) return st;
  if (!a->dh || !a->g || !a->h || (a->complement && !a->x) || (!a->dx && !a->dg && !a->dh0)) return GTR_ERR_NULL;
  const int es = (int)dtype_size(a->dtype), gs = (int)dtype_size(a->g_dtype);
  const int64_t L = (int64_t)a->H * a->W, n = a->B * L, state = (int64_t)a->B * a->d * 4;
  RecRows dh, g, h, x, dx, dg;
  if (!rec_rows(a->dh, n, 0, a->d, es, &dh) || !rec_rows(a->g, n, a->g_ld, a->d, gs, &g) ||
      !rec_rows(a->h, n, 0, a->d, es, &h) || !rec_rows(a->complement ? a->x : nullptr, n, a->x_ld, a->d, es, &x) ||
      !rec_rows(a->dx, n, a->dx_ld, a->d, es, &dx) || !rec_rows(a->dg, n, a->dg_ld, a->d, gs, &dg))
    return GTR_ERR_SHAPE;
  if (rec_misaligned(a->dh, es) || rec_misaligned(a->g, gs) || rec_misaligned(a->h, es) || rec_misaligned(x.p, es) ||
      rec_misaligned(a->dx, es) || rec_misaligned(a->dg, gs) || rec_misaligned(a->h0, 4) ||
      rec_misaligned(a->dh_final, 4) || rec_misaligned(a->dh0, 4))
    return GTR_ERR_UNSUPPORTED;
  st = rec_workspace(r, a->workspace, a->workspace_bytes);
  if (st != GTR_OK) return st;
  const RecRows ins[] = {dh, g, x, h, flat_rows(a->h0, state), flat_rows(a->dh_final, state)};
  const RecRows outs[] = {dx, dg, flat_rows(a->dh0, state), flat_rows(r.need ? a->workspace : nullptr, (int64_t)r.need)};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 6; ++j) {
      // a row's gradients may lie where that row of dh, g or x was, and the first state's where the last one's was
      const bool over = (i < 2 && j < 3 && same_rows(outs[i], ins[j])) || (i == 2 && j == 5 && outs[i].p == ins[j].p);
      if (rows_meet(outs[i], ins[j]) && !over) return GTR_ERR_ALIAS;
    }
    for (int j = 0; j < i; ++j)
      if (rows_meet(outs[i], outs[j])) return GTR_ERR_ALIAS;
  }
  rec_words(&r, a->workspace, a->spin_limit, stream);
  RecBwd p = {};
  p.t = r.t;
  p.dh = static_cast<const char*>(a->dh);
  p.g = static_cast<const char*>(a->g);
  p.h = static_cast<const char*>(a->h);
  p.x = static_cast<const char*>(a->x);
  p.h0 = a->h0;
  p.dh_final = a->dh_final;
  p.dx = static_cast<char*>(a->dx);
  p.dg = static_cast<char*>(a->dg);
  p.dh0 = a->dh0;
  p.x_ld = x.ld;
  p.g_ld = g.ld;
  p.dx_ld = dx.ld;
  p.dg_ld = dg.ld;
  p.L = L;
  p.H = a->H;
  p.W = a->W;
  p.d = a->d;
  p.dir = a->scan ^ 2;  // ROW <-> ROW_REV, COL <-> COL_REV
  p.sequences = (unsigned)r.sequences;
  p.inv_tau = a->g_kind == GTR_GATE_LOGITS ? 1.f / a->gate_tau : 1.f;
  return rec_launch<kRecBwdSteps>(RecLaunch<RecBwd>{p, r, stream}, a->dtype, a->g_dtype, a->g_kind == GTR_GATE_LOGITS,
                                  a->complement != 0);
}
