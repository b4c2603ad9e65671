// The matrix products of the gated feed-forward and of its backward pass on
// gfx950: C = A B in work-group tiles, with operands read in the layout that
// they have in memory (rows along K or columns along K) and with the gated
// epilogues. 16-bit operands, float32 accumulation.
#pragma once

#include <hip/hip_runtime.h>

#include "ffn_plan.h"
#include "gemm.h"
#include "gtr.h"
#include "gtr_device.h"

namespace gtr {

typedef int i4 __attribute__((ext_vector_type(4)));
typedef short s16v4 __attribute__((ext_vector_type(4)));

constexpr int kFfnProds = 3;
struct FfnGemm {
  FfnProd p[kFfnProds];
  int nprod, ksplit;
  int cdt;         // type of C (GTR_F32 / GTR_F16 / GTR_BF16)
  float* part;     // ksplit > 1: [ksplit][part_slice] partial sums
  int64_t part_slice;
  int act;
  // gated epilogues, [M][N] in the operands' type: the projections (forward: written where not null;
  // backward: read), and in the backward pass their gradients
  char *gate, *value, *dgate, *dvalue;
};

// Cache policy of stores that nothing reads soon (non-temporal): the projections kept
// for the backward pass leave the caches to the activations that the next product
// reads (12800 x 384 x 1536 fp16, both launches: 57.6 + 37.2 us -> 52.2 + 32.5).
constexpr int kFfnLater = 2;

// What one load or store of a lane moves: 8 16-bit elements, or 4 float32.
struct FfnVec {
  typedef unsigned V __attribute__((ext_vector_type(4)));
  V v;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, unsigned off) { v = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0); }
  template <int AUX = 0>
  __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t r, unsigned off) const {
    __builtin_amdgcn_raw_buffer_store_b128(v, r, off, 0, AUX);
  }
  template <int DT>
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const unsigned u = v[e];
      if constexpr (DT == GTR_F16) {
        x[2 * e] = (float)__builtin_bit_cast(_Float16, (unsigned short)(u & 0xffffu));
        x[2 * e + 1] = (float)__builtin_bit_cast(_Float16, (unsigned short)(u >> 16));
      } else {
        x[2 * e] = __builtin_bit_cast(float, u << 16);
        x[2 * e + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ float f32(int e) const {
    const unsigned u = v[e];
    return __builtin_bit_cast(float, u);
  }
  template <int DT>
  static __device__ __forceinline__ FfnVec pack(const float (&x)[8]) {
    typedef _Float16 hh __attribute__((ext_vector_type(2)));
    typedef __bf16 bb __attribute__((ext_vector_type(2)));
    FfnVec r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // pairs, which convert in one instruction
      const f2 p = {x[2 * e], x[2 * e + 1]};
      if constexpr (DT == GTR_F16)
        r.v[e] = __builtin_bit_cast(unsigned, __builtin_convertvector(p, hh));
      else
        r.v[e] = __builtin_bit_cast(unsigned, __builtin_convertvector(p, bb));
    }
    return r;
  }
  static __device__ __forceinline__ FfnVec bits(const float* x) {
    FfnVec r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r.v[e] = __builtin_bit_cast(unsigned, x[e]);
    return r;
  }
};

// act(g) and its derivative. SiLU: g s(g), s(g) (1 + g (1 - s(g))), s the logistic
// function; GELU: g P(g), P(g) + g phi(g), P and phi the normal distribution
// function and its density. The tail Q(x) = 1 - P(x), x = |g|, is taken as exp(-x^2 /
// 2) t R(t) with t = 1 / (1 + 3 x / 8): Q(x) exp(x^2 / 2) / t is smooth over 0 < t <= 1,
// and R is the polynomial of degree 8 that fits it there by least squares, reweighted
// towards the least largest relative error, 2.6e-7 at any x. In float32 the rounding of
// the exponential's argument comes to it, which grows with x^2: Q is off by at most 1e-6
// + 1.25 x^2 2^-24 of itself (5.3e-7 up to x = 2, 3.8e-6 up to 9, 7.7e-6 up to 13), where a
// 16-bit type's rounding is 4.9e-4 or more. Q shares its exponential with the density.
// (The library's erfc cost 16 us of 101 in the forward pass of 12800 x 384 x 1536.)
__device__ __forceinline__ float ffn_act(float g, int act, float& slope) {
  if (act == GTR_ACT_SILU) {
    const float p = __builtin_amdgcn_rcpf(1.f + __expf(-g));
    slope = p * fmaf(g, 1.f - p, 1.f);
    return g * p;
  }
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(g), 0.375f, 1.f)), e = __expf(-0.5f * g * g);
  float r = -0.0329110212624073f;
  r = fmaf(r, t, 0.13687977194786072f);
  r = fmaf(r, t, -0.18652084469795227f);
  r = fmaf(r, t, 0.050631992518901825f);
  r = fmaf(r, t, 0.015628185123205185f);
  r = fmaf(r, t, 0.08863813430070877f);
  r = fmaf(r, t, 0.12844571471214294f);
  r = fmaf(r, t, 0.14960458874702454f);
  r = fmaf(r, t, 0.14960338175296783f);
  const float q = e * t * r, p = g < 0.f ? q : 1.f - q;
  slope = fmaf(g * 0.39894228040143268f, e, p);
  return g * p;
}

// One lane's 16 bytes at base + voff (descriptor-checked: zeros past the end) to LDS
// byte lds + 16 lane; lds goes on by STEP. As dma16: no register is written and M0 is
// not the compiler's. (The addition is the wait state that M0 needs.)
template <int STEP>
__device__ __forceinline__ void dma16_buf(i4 rsrc, unsigned voff, unsigned& lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_add_u32 %0, %0, %3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               : "+s"(lds)
               : "v"(voff), "s"(rsrc), "n"(STEP)
               : "memory", "scc");
}
// Lane rows (16 lanes) 1 and 3 of a against rows 0 and 2 of b.
__device__ __forceinline__ void swap_rows(float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
  const unsigned lo = r[0], hi = r[1];
  a = __builtin_bit_cast(float, lo);
  b = __builtin_bit_cast(float, hi);
}
// n bytes from `at` on as a buffer descriptor.
__device__ __forceinline__ i4 ffn_rsrc(const char* at, int n) {
  const uint64_t p = reinterpret_cast<uint64_t>(at);
  return i4{__builtin_amdgcn_readfirstlane((int)(uint32_t)p), __builtin_amdgcn_readfirstlane((int)((uint32_t)(p >> 32) & 0xffffu)),
            __builtin_amdgcn_readfirstlane(n), 0x00020000};
}

// A tile of BT rows (or columns) by 64 K elements in LDS.
//
// Rows along K (T = 0): rows of 128 bytes; piece c (16 bytes) of row r sits at c ^ (r
// / 2 mod 8), so that the 16 rows of an operand read take 16 different places
// modulo 256 bytes.
//
// Columns along K (T = 1): 64 rows, one per K element, of BT columns, read with
// the transposing read ds_read_b64_tr_b16 in blocks of 4 K rows x 16 columns. One
// such instruction reads, for the four lane groups kq, the K rows 8 kq + 0..3 (or
// + 4..7), 32 bytes of each, half of the groups at a time. The 32-byte units of a row
// are permuted by XOR with a function of the row that puts those 8 into 8 different
// places modulo 256 bytes.
template <int T, int BT, int NW>
struct FfnTile {
  static constexpr int kBytes = BT * 128;
  static constexpr int P = BT / 8 / NW;  // transfers of 1 KB per wave
  static constexpr int RPC = 512 / BT;   // T = 1: K rows per transfer
  static_assert(BT % (8 * NW) == 0, "the tile splits evenly over the waves");

  static __device__ __forceinline__ int row_swz(int r) { return (r >> 1) & 7; }
  static __device__ __forceinline__ int unit_swz(int k) {
    const int m = k & 3, q = (k >> 3) & 1;
    return BT == 128 ? m | q << 2 : BT == 64 ? m >> 1 | q << 1 : q;
  }
  // byte offset of this lane's piece of transfer c (0 .. BT / 8 - 1), and its first K element
  // (MIX: of a half that is every second 16 of the tile's rows or columns)
  template <bool MIX>
  static __device__ __forceinline__ unsigned voff(int c, int lane, int64_t ld) {
    if constexpr (T == 0) {
      const int row = 8 * c + (lane >> 3), at = MIX ? row + (row & ~15) : row;
      return (unsigned)(at * (int)ld * 2) + 16u * ((lane & 7) ^ row_swz(row));
    } else {
      const int k = RPC * c + lane / (BT / 8), p = lane % (BT / 8);
      return (unsigned)(k * (int)ld * 2) + (MIX ? 64u : 32u) * ((p >> 1) ^ unit_swz(k)) + 16u * (p & 1);
    }
  }
  static __device__ __forceinline__ int piece_k(int c, int lane) {  // T = 0: K elements before this lane's piece
    return 8 * ((lane & 7) ^ row_swz(8 * c + (lane >> 3)));
  }
  // The MFMA operand of rows (columns) r0 + 16 i .. + 15, K elements 32 h .. 32 h + 31,
  // is at one of kAddr LDS addresses of a lane and a constant from it.
  static constexpr int kAddr(int n) { return T == 0 ? 2 : n; }  // n: how many i there are
  static __device__ __forceinline__ unsigned addr(unsigned base, int r0, int x, int lane) {
    const int r16 = lane & 15, kq = lane >> 4;
    if constexpr (T == 0) {
      return base + (r0 + r16) * 128 + (((4 * x + kq) ^ row_swz(r16)) << 4);
    } else {
      const int k = 8 * kq + (r16 >> 2);  // (its swizzle is that of k + 4 and k + 32)
      return base + k * (BT * 2) + ((((r0 >> 4) + x) ^ unit_swz(k)) << 5) + 8 * (r16 & 3);
    }
  }
  template <int N>
  static __device__ __forceinline__ w4 frag(const unsigned (&at)[N], int i, int h) {
    if constexpr (T == 0) {
      typedef __attribute__((address_space(3))) const w4* lp;
      return *(lp)(uintptr_t)(at[h] + i * 2048);
    } else {
      typedef __attribute__((address_space(3))) s16v4* lp;
      const s16v4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(uintptr_t)(at[i] + 64 * BT * h));
      const s16v4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(uintptr_t)(at[i] + 64 * BT * h + 8 * BT));
      return __builtin_bit_cast(w4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

template <int BM, int BN>
constexpr int kFfnLds = 2 * (BM + BN) * 128;

// C = A B. TA = 0: A is [M][K], TA = 1: A is [K][M]; TB = 0: B is [N][K], TB = 1:
// B is [K][N]. WM x WN waves.
//
// A work-group's tile is cut in halves along both sides: A0 and A1 (BM / 2 rows
// each), B0 and B1 (BN / 2 columns each; for the gated epilogue B0 is the gate's
// weight and B1 the value's, so that a lane ends with both projections of the same
// columns). A wave computes TI / 2 x TJ / 2 MFMA tiles of each of the four
// quadrants. Two LDS stages of 64 K elements hold the four halves. A step runs in
// two parts,
//   A0 B0, A0 B1   (meanwhile: reads B1 and A1 of this step from LDS)
//   A1 B0, A1 B1   (meanwhile: reads A0 and B0 of the next step)
// with one barrier after each, so every half is free for the step after next a
// whole step before it is read again: its transfer has three parts' time to
// arrive.
//
// What the epilogue reads (a residual, the projections) is fetched before the first of
// it is used, a half's rows at a time. (Fetched before the products, where the small
// tiles have the registers, it came out the same: 1600 x 192 x 768 backward 23.2 us
// against 23.0.)
//
// b: the work-group's number of T, in the order of dispatch. Work-group b runs on XCD
// b % 8 (round-robin dispatch); each XCD takes a contiguous range of the tiles, in
// groups of 4 row tiles, rows fastest: a patch of 4 x 8 tiles that share operands runs
// on an XCD's 32 CUs at a time (8192 x 4096 x 11008 forward 1568 us; in groups of 8
// 1591, of 16 some 3 % more).
// MANY: the launch may have several products.
template <int DT, int TA, int TB, int EPI, int BM, int BN, int WM, int WN, bool MANY>
__device__ __forceinline__ void ffn_tile(const FfnGemm& g, char* ring, int b, int T) {
  typedef Operand<DT, DT> Op;
  constexpr int NW = WM * WN;
  constexpr int HM = BM / 2, HN = BN / 2;                      // a half's rows, columns
  constexpr int TI = HM / (16 * WM), TJ = HN / (16 * WN);      // MFMA tiles of a wave in a quadrant
  typedef FfnTile<TA, HM, NW> LA;
  typedef FfnTile<TB, HN, NW> LB;
  constexpr int STAGE = 2 * (LA::kBytes + LB::kBytes);
  static_assert(2 * STAGE == kFfnLds<BM, BN>, "two stages");
  constexpr bool DUAL = EPI == kFfnGate;
  constexpr int BC = DUAL ? HN : BN;  // columns of C of a tile
  constexpr bool MIX = TJ == 1 && !DUAL, PAIR = TJ == 1 && DUAL;
  static_assert(TJ == 1 || TJ % 2 == 0, "MFMA tiles of C in pairs");
  static_assert(!DUAL || TB == 0, "the gated epilogue reads linear-layer weights");

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wmi = wave / WN, wni = wave % WN;
  const int r16 = lane & 15, kq = lane >> 4;
  // work-group -> tile
  const int xcd = b & 7, slot = b >> 3;
  int jt = xcd * (T >> 3) + min(xcd, T & 7) + slot;
  int bz = 0, pi = 0;
  if (EPI == kFfnStore && g.ksplit > 1) {
    const int per = T / g.ksplit;
    bz = jt / per;
    jt -= bz * per;
  }
  if (MANY)
    while (pi + 1 < g.nprod && jt >= g.p[pi].gx * g.p[pi].gy) jt -= g.p[pi].gx * g.p[pi].gy, ++pi;
  const FfnProd& p = g.p[pi];
  constexpr int GM = 4;
  const int grp = jt / (GM * p.gy), first = grp * GM, gsz = min(p.gx - first, GM), in = jt - grp * GM * p.gy;
  const int bx = first + in % gsz, by = in / gsz;
  const int mb = bx * BM, nb = by * BC;

  // K steps of this slice; a segment has `sps` steps
  const int K = p.K, sps = (K + 63) / 64, all = sps * p.nseg;
  const int s_per = EPI == kFfnStore && g.ksplit > 1 ? (all + g.ksplit - 1) / g.ksplit : all;
  const int s0 = bz * s_per, steps = max(0, min(s0 + s_per, all) - s0);

  unsigned va[2][LA::P], vb[2][LB::P];  // byte offsets of this lane's transfers
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int q = 0; q < LA::P; ++q)
      va[h][q] = LA::template voff<false>(wave + NW * q, lane, p.lda) + h * HM * 2 * (TA ? 1 : (unsigned)p.lda);
#pragma unroll
    for (int q = 0; q < LB::P; ++q)
      vb[h][q] = LB::template voff<MIX>(wave + NW * q, lane, p.ldb) + (DUAL ? 0 : h * (MIX ? 16 : HN) * 2 * (TB ? 1 : (unsigned)p.ldb));
  }

  // Descriptors of a step's operands: they end where the tile's rows do (rows along
  // K) or with the step's last K row (columns along K; past the last column of a
  // row lies the next one, whose elements only columns that are not stored get).
  const int64_t astep = TA ? 128 * p.lda : 128, bstep = TB ? 128 * p.ldb : 128;
  const int64_t a0 = TA ? 2 * (int64_t)mb : 2 * (int64_t)mb * p.lda, b0 = TB ? 2 * (int64_t)nb : 2 * (int64_t)nb * p.ldb;
  const int ktail = K - 64 * (sps - 1);  // K elements of a segment's last step
  const int aend = TA ? 128 * (int)p.lda - 2 * mb : min(BM, p.M - mb) * (int)p.lda * 2;
  const int bend = TB ? 128 * (int)p.ldb - 2 * nb : min(BC, p.N - nb) * (int)p.ldb * 2;
  const int atail = TA ? ktail * 2 * (int)p.lda - 2 * mb : aend, btail = TB ? ktail * 2 * (int)p.ldb - 2 * nb : bend;
  const int sg = s0 >= sps ? 1 : 0;
  int is = s0 - sg * sps, left = steps;  // the next transfer's step in its segment; steps not transferred yet
  const char *pa = p.a[sg] + a0 + is * astep, *pb = p.b[DUAL ? 0 : sg] + b0 + is * bstep;
  const char *pa1 = p.a[1] + a0, *pb1 = p.b[1] + b0;  // the second segment (DUAL: pb1 - b's start is the second weight)
  const int64_t pv = pb1 - (p.b[0] + b0);
  const unsigned lbase = lds_addr(ring) + wave * 1024;
  i4 ra, rb, rv;
  // In the last step of a segment that is not whole, the next elements of a row along
  // K are another row's: the lanes whose pieces are past the end get offsets past every
  // descriptor's range. (A wave's transfers c are all even or all odd, so a lane's
  // piece is at the same K element in each.)
  const unsigned past = LA::piece_k(wave, lane) >= ktail ? 0x80000000u : 0u;
  const int tailstep = ktail < 64 ? sps - 1 : -1;
  int masked = 0;
  // The next step's operands. Past the last step the descriptors are empty: the
  // transfers write zeros that no product reads, so that the loop has one form.
  auto next = [&]() {
    const bool last = is == sps - 1, more = left > 0;
    --left;
    if ((!TA || !TB) && masked != (is == tailstep ? 1 : 0)) {
      masked ^= 1;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int q = 0; q < LA::P; ++q) va[h][q] ^= TA ? 0u : past;
#pragma unroll
        for (int q = 0; q < LB::P; ++q) vb[h][q] ^= TB ? 0u : past;
      }
    }
    ra = ffn_rsrc(pa, more ? last ? atail : aend : 0);
    rb = ffn_rsrc(pb, more ? last ? btail : bend : 0);
    if (DUAL) rv = ffn_rsrc(pb + pv, more ? bend : 0);
    is = last ? 0 : is + 1;
    pa = last ? pa1 : pa + astep;
    pb = last ? pb1 : pb + bstep;
  };
  // This wave's transfer q of halves A_h and B_h of that step to LDS address l on
  // (transfers in order: l goes on from one to the next).
  constexpr int PL = LA::P + LB::P;
  auto transfer = [&](unsigned& l, int h, int q) {
    constexpr int S = NW * 1024;
    if (q < LA::P - 1)
      dma16_buf<S>(ra, va[h][q], l);
    else if (q == LA::P - 1 && h == 0)
      dma16_buf<2 * LA::kBytes - S*(LA::P - 1)>(ra, va[h][q], l);
    else if (q == LA::P - 1)
      dma16_buf<LA::kBytes + LB::kBytes - S*(LA::P - 1)>(ra, va[h][q], l);
    else
      dma16_buf<S>(DUAL && h ? rv : rb, vb[h][q - LA::P], l);
  };
  auto half_at = [&](int stage, int h) { return lbase + stage * STAGE + h * LA::kBytes; };

  const int wm = wmi * (HM / WM), wn = wni * (HN / WN);
  f4 acc[2][2][TI][TJ];  // quadrant (A half, B half)
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) acc[q >> 1][q & 1][i][j] = f4{0.f, 0.f, 0.f, 0.f};
  w4 fa[2][2 * TI], fb[2][2 * TJ];  // operands of the halves: K elements 0 .. 31, then 32 .. 63
  constexpr int NA = LA::kAddr(TI), NB = LB::kAddr(TJ);
  unsigned aa[NA], ab[NB];  // of A0 and B0 in the current stage; A1 and B1 are a constant further
#pragma unroll
  for (int x = 0; x < NA; ++x) aa[x] = LA::addr(lds_addr(ring), wm, x, lane);
#pragma unroll
  for (int x = 0; x < NB; ++x) ab[x] = LB::addr(lds_addr(ring) + 2 * LA::kBytes, wn, x, lane);
  auto read_a = [&](int h, int q) {
    unsigned at[NA];
#pragma unroll
    for (int x = 0; x < NA; ++x) at[x] = aa[x] + h * LA::kBytes;
    fa[h][q] = LA::frag(at, q % TI, q / TI);
  };
  auto read_b = [&](int h, int q) {
    unsigned at[NB];
#pragma unroll
    for (int x = 0; x < NB; ++x) at[x] = ab[x] + h * LB::kBytes;
    fb[h][q] = LB::frag(at, q % TJ, q / TJ);
  };
  auto other_stage = [&]() {
#pragma unroll
    for (int x = 0; x < NA; ++x) aa[x] ^= STAGE;
#pragma unroll
    for (int x = 0; x < NB; ++x) ab[x] ^= STAGE;
  };

  // A part of a step: the products of A_h with B0, then B1, a row of MFMA tiles at a
  // time, and between the rows the reads and the transfers: the matrix cores work
  // while the wave issues them.
  constexpr int ROWS = 4 * TI;
  constexpr int RR = (2 * TI + 2 * TJ) * 4 / (3 * ROWS) + ((2 * TI + 2 * TJ) * 4 % (3 * ROWS) != 0);  // reads per row
  constexpr int DR = (PL + ROWS - 1) / ROWS;                                                      // transfers per row
  static_assert((2 * TJ + RR - 1) / RR <= ROWS / 2 && (2 * TI + RR - 1) / RR <= ROWS / 2 && RR * ROWS >= 2 * TI + 2 * TJ,
                "every operand is read in time");
  auto part = [&](int h, int stage) {
    unsigned l = half_at(stage, h);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int bh = r / (2 * TI), kh = r / TI & 1, i = r % TI;
#pragma unroll
      for (int j = 0; j < TJ; ++j)
        acc[h][bh][i][j] = mfma(Op::get(fb[bh][kh * TJ + j]), Op::get(fa[h][kh * TI + i]), acc[h][bh][i][j]);  // C^T tiles
      __builtin_amdgcn_sched_barrier(0);
      if (h == 0) {
#pragma unroll
        for (int q = r * RR; q < (r + 1) * RR; ++q) {
          if (q < 2 * TJ)
            read_b(1, q);
          else if (q < 2 * TJ + 2 * TI)
            read_a(1, q - 2 * TJ);
        }
        if (r == ROWS - 1) other_stage();
      } else {
#pragma unroll
        for (int q = r * RR; q < (r + 1) * RR; ++q)
          if (q < 2 * TI) read_a(0, q);
#pragma unroll
        for (int q = (r - ROWS / 2) * RR; q < (r - ROWS / 2 + 1) * RR; ++q)  // B0's registers are free after its products
          if (q >= 0 && q < 2 * TJ) read_b(0, q);
        if (r == ROWS / 2) next();
      }
#pragma unroll
      for (int q = r * DR; q < (r + 1) * DR && q < PL; ++q) transfer(l, h, q);
      __builtin_amdgcn_sched_barrier(0);
    }
    // the transfers that the next part reads have landed, and every wave has read what
    // the next part's transfers overwrite
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0), known to the compiler: no waits for these reads below
    ring_wait<2 * PL>();
  };
  static_assert(PL <= ROWS / 2 * DR, "a part's transfers are issued before its step's descriptors change");

#pragma unroll
  for (int k = 0; k < 2; ++k) {
    next();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      unsigned l = half_at(k, h);
#pragma unroll
      for (int q = 0; q < PL; ++q) transfer(l, h, q);
    }
  }
  next();
  ring_wait<2 * PL>();
#pragma unroll
  for (int q = 0; q < 2 * TI; ++q) read_a(0, q);
#pragma unroll
  for (int q = 0; q < 2 * TJ; ++q) read_b(0, q);
  ring_sync();
  for (int k = 0; k < steps; ++k) {
    part(0, k & 1);
    part(1, k & 1);
  }
  ring_wait<0>();  // no transfer is in flight when the work-group ends

  // Lane (r16, kq) holds, of an MFMA tile of C, row r16 and columns 4 kq .. 4 kq + 3.
  // Two tiles exchange lane rows, so that it holds 8 consecutive columns of one of them,
  // 8 (kq / 2) .. + 7 of tile kq % 2. The two are side by side: column tiles of a half;
  // where a wave has one of those, its tiles of the two halves (MIX: the halves take the
  // tile's columns 16 by 16 in turn); and for the gated epilogue, where the halves are
  // the two projections, the tiles of A0's and A1's rows (PAIR). (1600 x 192 x 768 with
  // 4 columns per lane: gated product 7.8 us, now 7.0; gradients of the projections 12.4,
  // now 11.0; 4150 rows 16.3, now 12.5. Halves that alternate in the larger tiles too, 32
  // columns at a time, cost their transfers more than the stores gain: 12800 x 384 x
  // 1536 gradients of the projections 63.8 us -> 67.9.)
  // Loads and stores go through descriptors of the tile's rows, columns past the last
  // out of range.
  //
  // What goes on to a next product (act(g) v, and dg, dv in the backward pass) is formed
  // in float32 and rounded to the operands' type, which that product's MFMAs take; two
  // MFMAs for an operand's upper and lower parts would keep 32 bits at twice the matrix
  // time, which bounds the large products. It is the whole of the results' distance from
  // a chain in 32 bits: 1.57e-3 relative in bf16 (1 x 1024 x 2816), 2.2e-4 to 3.2e-4 in
  // fp16, under 8e-5 against a chain that rounds there too; to 64 bits it is 1.1 to 1.4
  // times the last rounding's.
  constexpr int NQ = TJ == 1 ? 1 : TJ / 2;       // times 8 columns of a lane in a half
  constexpr int NC = DUAL || MIX ? NQ : 2 * NQ;  // and in the tile
  const int cofs = 8 * (kq >> 1) + (PAIR ? 0 : 16 * (kq & 1)), rofs = r16 + (PAIR ? HM * (kq & 1) : 0);
  const int rows = min(BM, p.M - mb);
  const bool cut = EPI == kFfnStore && g.ksplit > 1;
  const int cdt = cut ? (int)GTR_F32 : EPI == kFfnStore ? g.cdt : DT;
  const unsigned es = cdt == GTR_F32 ? 4 : 2;
  const int64_t ldc = cut ? p.N : p.ldc;
  const int64_t first_at = ((int64_t)mb * ldc + nb) * es;  // the tile's first element
  const int range = (int)((rows * ldc - nb) * es);
  auto tile_of = [&](const char* c) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(c) + first_at, 0, c ? range : 0, 0x00020000); };
  unsigned col[NC];  // a lane's columns, in bytes from the tile's first
#pragma unroll
  for (int q = 0; q < NC; ++q) {
    const int c = q / NQ * HN + (MIX ? 2 : 1) * wn + 32 * (q % NQ) + cofs;
    col[q] = nb + c < p.N ? c * es : 0x80000000u;
  }
  const auto rc = tile_of(cut ? reinterpret_cast<const char*>(g.part + bz * g.part_slice + p.part_off) : p.c);
  const auto rres = tile_of(EPI == kFfnStore && !cut ? p.res : nullptr);
  const auto rg = tile_of(g.gate), rl = tile_of(g.value), rdg = tile_of(g.dgate), rdl = tile_of(g.dvalue);
  const bool res32 = EPI == kFfnStore && p.res && !cut && cdt == GTR_F32, res16 = EPI == kFfnStore && p.res && !cut && cdt != GTR_F32;
  FfnVec e0[TI][NC], e1[TI][NC];  // what the epilogue reads
  auto at = [&](int h, int i, int q) {
    return (unsigned)((h * HM + wm + 16 * i + rofs) * (int)ldc) * es + col[q];
  };
  auto fetch = [&](int h) {
    if (EPI == kFfnGateGrad || res16 || res32) {
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int q = 0; q < NC; ++q) {
          const unsigned o = at(h, i, q);
          if constexpr (EPI == kFfnGateGrad) {
            e0[i][q].load(rg, o);
            e1[i][q].load(rl, o);
          } else {
            e0[i][q].load(rres, o);
            if (res32) e1[i][q].load(rres, o + 16);
          }
        }
    }
  };
#pragma unroll
  for (int h = 0; h < (PAIR ? 1 : 2); ++h) {  // the rows of A_h
    fetch(h);
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      float x[2][NQ][8];
#pragma unroll
      for (int q = 0; q < (MIX ? 1 : 2 * NQ); ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float(&v)[8] = x[q / NQ][q % NQ];
          v[e] = acc[h][q / NQ][i][TJ == 1 ? 0 : 2 * (q % NQ)][e];
          v[4 + e] = MIX ? acc[h][1][i][0][e] : PAIR ? acc[1][q][i][0][e] : acc[h][q / NQ][i][TJ == 1 ? 0 : 2 * (q % NQ) + 1][e];
          swap_rows(v[e], v[4 + e]);
        }
      if constexpr (DUAL) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          const unsigned o = at(h, i, q);
          if (g.gate) FfnVec::pack<DT>(x[0][q]).template store<kFfnLater>(rg, o);
          if (g.value) FfnVec::pack<DT>(x[1][q]).template store<kFfnLater>(rl, o);
          float y[8], s;
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = ffn_act(x[0][q][e], g.act, s) * x[1][q][e];
          FfnVec::pack<DT>(y).store(rc, o);
        }
      } else {
#pragma unroll
        for (int q = 0; q < NC; ++q) {
          float(&v)[8] = x[q / NQ][q % NQ];
          const unsigned o = at(h, i, q);
          if constexpr (EPI == kFfnGateGrad) {
            float gt[8], vl[8], dg[8], dv[8], hh[8];
            e0[i][q].template unpack<DT>(gt);
            e1[i][q].template unpack<DT>(vl);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float s;
              const float a = ffn_act(gt[e], g.act, s);
              dg[e] = v[e] * vl[e] * s;
              dv[e] = v[e] * a;
              hh[e] = a * vl[e];
            }
            FfnVec::pack<DT>(dg).store(rdg, o);
            FfnVec::pack<DT>(dv).store(rdl, o);
            if (p.c) FfnVec::pack<DT>(hh).store(rc, o);
          } else {
            if (res16) {
              float r[8];
              e0[i][q].template unpack<DT>(r);
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] += r[e];
            }
            if (res32) {
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] += e < 4 ? e0[i][q].f32(e) : e1[i][q].f32(e - 4);
            }
            if (cdt == GTR_F32) {
              FfnVec::bits(v).store(rc, o);
              FfnVec::bits(v + 4).store(rc, o + 16);
            } else {
              FfnVec::pack<DT>(v).store(rc, o);
            }
          }
        }
      }
    }
  }
}

template <int DT, int TA, int TB, int EPI, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(2))) ffn_gemm_kernel(FfnGemm g) {
  __shared__ __attribute__((aligned(1024))) char ring[kFfnLds<BM, BN>];
  ffn_tile<DT, TA, TB, EPI, BM, BN, WM, WN, false>(g, ring, blockIdx.x, gridDim.x);
}

// The gradients of the input and of the weights in one launch: neither needs the
// other, and a short batch's products do not fill the chip one by one. The nx
// work-groups of dx and the nw of dw follow each other, dx first or last, the first
// count rounded up to a multiple of 8 for the second's XCDs.
template <int DT, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(2)))
ffn_grad_kernel(FfnGemm dx, FfnGemm dw, int nx, int nw, int x_first) {
  __shared__ __attribute__((aligned(1024))) char ring[kFfnLds<BM, BN>];
  const int n0 = x_first ? nx : nw, r0 = (n0 + 7) & ~7;
  const bool head = (int)blockIdx.x < r0;
  const int b = head ? blockIdx.x : blockIdx.x - r0;
  if (head && b >= n0) return;
  if (head == (x_first != 0))
    ffn_tile<DT, 0, 1, kFfnStore, BM, BN, WM, WN, false>(dx, ring, b, nx);
  else
    ffn_tile<DT, 1, 1, kFfnStore, BM, BN, WM, WN, true>(dw, ring, b, nw);
}

// C = the sum of the slices' partial sums (+ res), 8 elements per thread: of g, then
// of h.
__device__ __forceinline__ void ffn_reduce(const FfnGemm& g, int64_t t) {
  char* c = g.p[0].c;
  const char* res = g.p[0].res;
  int64_t off = t;  // (C is contiguous)
#pragma unroll
  for (int i = 1; i < kFfnProds; ++i)
    if (i < g.nprod && t >= g.p[i].part_off) {
      c = g.p[i].c;
      res = g.p[i].res;
      off = t - g.p[i].part_off;
    }
  float x[8];
  load8(g.part, GTR_F32, t, x);
#pragma unroll 4
  for (int s = 1; s < g.ksplit; ++s) {
    float y[8];
    load8(g.part, GTR_F32, s * g.part_slice + t, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += y[e];
  }
  if (res) {
    float y[8];
    load8(res, g.cdt, off, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += y[e];
  }
  store_n<8>(c, g.cdt, off, x);
}

// ---------------------------------------------------------------------------
// A few tokens (up to kFewTokens): the weights' bytes are the work, each read once,
// and the time is how soon all of them are asked for. A work-group takes 8 columns of
// C, half of what the matrix instruction has rows for, so that a narrow product still
// covers the chip (1,024 columns: 128 work-groups instead of 64). The other 8 rows
// take the same weights' next 32 K elements, and the other 8 of its columns the same
// tokens' there: of the four 8x8 blocks of the result the two on the diagonal are
// halves of the sum, the other two mean nothing. A lane's 16-byte load is its part of
// the operand as it stands; a weight's row is read 128 bytes at a time. The waves take
// the 64-deep pieces of K in turn, kFewFlight of them asked for at once, the tokens'
// rows come from cache, and the waves' sums meet in LDS and are added in their order.
// One token, bf16, gated and down product in us, against 16 columns each with eight
// waves and four pieces in flight: 192 x 768 3.3 + 3.3 (was 4.3 + 4.7), 1024 x 2816
// 5.3 + 4.4 (7.4 + 7.2), 2048 x 5632 10.7 + 5.7 (13.7 + 8.6), 4096 x 11008 37.9 +
// 20.3 (44.3 + 22.8: 4.8 and 4.4 TB/s). Two weights with eight waves and one piece in
// flight: 5.6 and 39.7 at the second and the last; with more in flight the registers
// leave fewer work-groups on a CU.
// ---------------------------------------------------------------------------
constexpr int few_waves(int nb) { return nb == 1 ? 8 : 4; }
constexpr int kFewFlight = 2;
struct FfnFew {
  const char* x;       // [M][K]
  const char* w[2];    // [N][K]: gate and value, or one weight
  char* c;             // [M][N]
  const char* res;     // [M][N] or null (one weight)
  char *gate, *value;  // [M][N] or null (two weights)
  int M, N, K, act;
};

template <int DT, int NB>
__global__ void __launch_bounds__(64 * few_waves(NB)) ffn_few_kernel(FfnFew g) {
  typedef Operand<DT, DT> Op;
  constexpr int U = kFewFlight, NW = few_waves(NB);
  __shared__ f4 sums[NW][NB][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r8 = lane & 7, half = (lane >> 3) & 1, kq = lane >> 4, n0 = blockIdx.x * 8;
  const int K = g.K, pieces = (K + 63) / 64;
  // this lane's rows; past the last one the last one again, which is not stored
  const char *wr[NB], *xr = g.x + (int64_t)min(r8, g.M - 1) * K * 2;
#pragma unroll
  for (int b = 0; b < NB; ++b) wr[b] = g.w[b] + (int64_t)min(n0 + r8, g.N - 1) * K * 2;
  f4 acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = f4{0.f, 0.f, 0.f, 0.f};
  for (int p = wave; p < pieces; p += NW * U) {
    w4 fw[U][NB], fx[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = 64 * (p + NW * u) + 32 * half + 8 * kq;
      const bool in = k < K;  // (K is a multiple of 8)
      const int64_t o = 2 * (int64_t)(in ? k : 0);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        fw[u][b] = *reinterpret_cast<const w4*>(wr[b] + o);
        if (!in) fw[u][b] = w4{0, 0, 0, 0};
      }
      fx[u] = *reinterpret_cast<const w4*>(xr + o);
      if (!in) fx[u] = w4{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b] = mfma(Op::get(fw[u][b]), Op::get(fx[u]), acc[b]);
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) sums[wave][b][lane] = acc[b];
  __syncthreads();
  const int m = r8, n = n0 + 4 * kq;  // columns n .. n + 3 of token m
  if (threadIdx.x >= 32 || half || m >= g.M || n >= g.N) return;
  float s[NB][4];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    f4 v = sums[0][b][lane] + sums[0][b][lane + 40];
#pragma unroll
    for (int i = 1; i < NW; ++i) v += sums[i][b][lane] + sums[i][b][lane + 40];
#pragma unroll
    for (int e = 0; e < 4; ++e) s[b][e] = v[e];
  }
  const int64_t off = (int64_t)m * g.N + n;
  if constexpr (NB == 2) {
    if (g.gate) store_n<4>(g.gate, DT, off, s[0]);
    if (g.value) store_n<4>(g.value, DT, off, s[1]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float slope;
      s[0][e] = ffn_act(s[0][e], g.act, slope) * s[1][e];
    }
  } else if (g.res) {
    float r[4];
    load4(g.res, DT, off, r);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[0][e] += r[e];
  }
  store_n<4>(g.c, DT, off, s[0]);  // (act(g) v in the operands' type, as the tiles leave it)
}

}  // namespace gtr
