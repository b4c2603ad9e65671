// The matrix products of the gated feed-forward and of its backward pass on
// gfx950: C = A B in work-group tiles, with operands read in the layout that
// they have in memory (rows along K or columns along K) and with the gated
// epilogues. 16-bit operands, float32 accumulation.
#pragma once

#include <hip/hip_runtime.h>

#include "gemm.h"
#include "gtr.h"
#include "gtr_device.h"

namespace gtr {

typedef int i4 __attribute__((ext_vector_type(4)));
typedef short s16v4 __attribute__((ext_vector_type(4)));

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

// What an epilogue does with the product.
enum { kFfnStore = 0, kFfnGate = 1, kFfnGateGrad = 2 };

// N (4 or 8) consecutive elements of type DT at p (aligned to all of them, float32 to
// four).
template <int DT, int N>
__device__ __forceinline__ void ffn_load(const char* p, float (&x)[N]) {
  if constexpr (N == 8)
    load8(p, DT, 0, x);
  else
    load4(p, DT, 0, x);
}
template <int DT, int N>
__device__ __forceinline__ void ffn_store(char* p, const float (&x)[N]) {
  if constexpr (DT == GTR_F32) {
    store_n<N>(p, GTR_F32, 0, x);
  } else {
    typedef unsigned v __attribute__((ext_vector_type(N / 2)));
    v r;
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
      if constexpr (DT == GTR_F16) {
        r[e] = __builtin_bit_cast(unsigned short, (_Float16)x[2 * e]) |
               (unsigned)__builtin_bit_cast(unsigned short, (_Float16)x[2 * e + 1]) << 16;
      } else {
        r[e] = __builtin_bit_cast(unsigned short, (__bf16)x[2 * e]) |
               (unsigned)__builtin_bit_cast(unsigned short, (__bf16)x[2 * e + 1]) << 16;
      }
    }
    *reinterpret_cast<v*>(p) = r;
  }
}

// act(g) and its derivative. SiLU: g s(g), s(g) (1 + g (1 - s(g))), s the logistic
// function; GELU: g P(g), P(g) + g phi(g), P and phi the normal distribution
// function and its density.
__device__ __forceinline__ float ffn_act(float g, int act, float& slope) {
  if (act == GTR_ACT_SILU) {
    const float p = __builtin_amdgcn_rcpf(1.f + __expf(-g));
    slope = p * fmaf(g, 1.f - p, 1.f);
    return g * p;
  }
  const float p = 0.5f * erfcf(g * -0.70710678118654752f);  // (1 + erf would lose the lower tail)
  slope = fmaf(g * 0.39894228040143268f, __expf(-0.5f * g * g), p);
  return g * p;
}

// One lane's 16 bytes at base + voff (descriptor-checked: zeros past the end) to LDS
// byte lds + 16 lane. As dma16: no register is written and M0 is not the compiler's.
__device__ __forceinline__ void dma16_buf(i4 rsrc, unsigned voff, unsigned lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(rsrc)
               : "memory");
}
// Lane rows (16 lanes) 1 and 3 of a against rows 0 and 2 of b.
__device__ __forceinline__ void swap_rows(float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
  const unsigned lo = r[0], hi = r[1];
  a = __builtin_bit_cast(float, lo);
  b = __builtin_bit_cast(float, hi);
}
constexpr unsigned kFfnOob = 0x80000000u;  // a byte offset past every descriptor's range

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
// + 4..7): 32 bytes of each of 16 rows. The 32-byte units of a row are permuted by
// XOR with a function of the row that puts those 16 into 16 different places
// modulo 512 bytes.
template <int T, int BT, int NW>
struct FfnTile {
  static constexpr int kBytes = BT * 128;
  static constexpr int P = BT / 8 / NW;  // transfers of 1 KB per wave
  static constexpr int RPC = 512 / BT;   // T = 1: K rows per transfer
  static_assert(BT % (8 * NW) == 0, "the tile splits evenly over the waves");

  static __device__ __forceinline__ int row_swz(int r) { return (r >> 1) & 7; }
  static __device__ __forceinline__ int unit_swz(int k) {
    const int m = k & 3, q = (k >> 3) & 3;
    return BT == 128 ? m >> 1 | q << 1 : BT == 64 ? q : q & 1;  // (32: two of the 16 share a place)
  }
  // byte offset of this lane's piece of transfer c (0 .. BT / 8 - 1), and its first K element
  static __device__ __forceinline__ unsigned voff(int c, int lane, int64_t ld) {
    if constexpr (T == 0) {
      const int row = 8 * c + (lane >> 3);
      return (unsigned)(row * (int)ld * 2) + 16u * ((lane & 7) ^ row_swz(row));
    } else {
      const int k = RPC * c + lane / (BT / 8), p = lane % (BT / 8);
      return (unsigned)(k * (int)ld * 2) + 32u * ((p >> 1) ^ unit_swz(k)) + 16u * (p & 1);
    }
  }
  static __device__ __forceinline__ int piece_k(int c, int lane) {  // T = 0: K elements before this lane's piece
    return 8 * ((lane & 7) ^ row_swz(8 * c + (lane >> 3)));
  }
  // the MFMA operand of rows (columns) r0 .. r0 + 15, K elements 32 h .. 32 h + 31
  static __device__ __forceinline__ w4 frag(const char* s, int r0, int h, int lane) {
    const int r16 = lane & 15, kq = lane >> 4;
    if constexpr (T == 0) {
      const int row = r0 + r16;
      return *reinterpret_cast<const w4*>(s + row * 128 + (((4 * h + kq) ^ row_swz(r16)) << 4));
    } else {
      const int k = 8 * kq + (r16 >> 2);  // (of this half; its swizzle is that of k + 4 and k + 32)
      const char* p = s + (32 * h + k) * (BT * 2) + (((r0 >> 4) ^ unit_swz(k)) << 5) + 8 * (r16 & 3);
      typedef __attribute__((address_space(3))) s16v4* lp;
      const s16v4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)p);
      const s16v4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 4 * BT * 2));
      return __builtin_bit_cast(w4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

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
template <int DT, int TA, int TB, int EPI, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(2))) ffn_gemm_kernel(FfnGemm g) {
  typedef Operand<DT, DT> Op;
  constexpr int NW = WM * WN;
  constexpr int HM = BM / 2, HN = BN / 2;                      // a half's rows, columns
  constexpr int TI = HM / (16 * WM), TJ = HN / (16 * WN);      // MFMA tiles of a wave in a quadrant
  typedef FfnTile<TA, HM, NW> LA;
  typedef FfnTile<TB, HN, NW> LB;
  constexpr int STAGE = 2 * (LA::kBytes + LB::kBytes);
  constexpr bool DUAL = EPI == kFfnGate;
  constexpr int BC = DUAL ? HN : BN;  // columns of C of a tile
  static_assert(!DUAL || TB == 0, "the gated epilogue reads linear-layer weights");
  __shared__ __attribute__((aligned(1024))) char ring[2 * STAGE];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wmi = wave / WN, wni = wave % WN;
  const int r16 = lane & 15, kq = lane >> 4;
  // work-group -> tile
  const int T = gridDim.x, xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  int jt = xcd * (T >> 3) + min(xcd, T & 7) + slot;
  const int per = T / g.ksplit, bz = jt / per;
  jt -= bz * per;
  int pi = 0;
  while (pi + 1 < g.nprod && jt >= g.p[pi].gx * g.p[pi].gy) jt -= g.p[pi].gx * g.p[pi].gy, ++pi;
  const FfnProd& p = g.p[pi];
  constexpr int GM = 8;
  const int grp = jt / (GM * p.gy), first = grp * GM, gsz = min(p.gx - first, GM), in = jt - grp * GM * p.gy;
  const int bx = first + in % gsz, by = in / gsz;
  const int mb = bx * BM, nb = by * BC;

  // K steps of this slice; a segment has `sps` steps
  const int K = p.K, sps = (K + 63) / 64, all = sps * p.nseg;
  const int s_per = (all + g.ksplit - 1) / g.ksplit;
  const int s0 = bz * s_per, steps = max(0, min(s0 + s_per, all) - s0);

  unsigned va[2][LA::P], vb[2][LB::P];  // byte offsets of this lane's transfers
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int q = 0; q < LA::P; ++q)
      va[h][q] = LA::voff(wave + NW * q, lane, p.lda) + h * HM * 2 * (TA ? 1 : (unsigned)p.lda);
#pragma unroll
    for (int q = 0; q < LB::P; ++q)
      vb[h][q] = LB::voff(wave + NW * q, lane, p.ldb) + (DUAL ? 0 : h * HN * 2 * (TB ? 1 : (unsigned)p.ldb));
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
  int kleft = 64;
  // The next step's operands: their descriptors, and how many K elements it has.
  // Past the last step the descriptors are empty: the transfers write zeros that no
  // product reads, so that the loop has one form.
  auto next = [&]() {
    const bool last = is == sps - 1, more = left > 0;
    --left;
    kleft = last ? ktail : 64;
    ra = ffn_rsrc(pa, more ? last ? atail : aend : 0);
    rb = ffn_rsrc(pb, more ? last ? btail : bend : 0);
    if (DUAL) rv = ffn_rsrc(pb + pv, more ? bend : 0);
    is = last ? 0 : is + 1;
    pa = last ? pa1 : pa + astep;
    pb = last ? pb1 : pb + bstep;
  };
  // This wave's transfer q of halves A_h and B_h of that step to a stage. In the last
  // step of a segment a row's next elements are another row's: out of range instead.
  // (A wave's transfers c are all even or all odd, so a lane's piece is at the same K
  // element in each.)
  constexpr int PL = LA::P + LB::P;
  const int pk = LA::piece_k(wave, lane);
  auto transfer = [&](int stage, int h, int q) {
    const unsigned l = lbase + stage * STAGE;
    if (q < LA::P)
      dma16_buf(ra, !TA && pk >= kleft ? kFfnOob : va[h][q], l + h * LA::kBytes + NW * 1024 * q);
    else
      dma16_buf(DUAL && h ? rv : rb, !TB && pk >= kleft ? kFfnOob : vb[h][q - LA::P],
                l + 2 * LA::kBytes + h * LB::kBytes + NW * 1024 * (q - LA::P));
  };

  const int wm = wmi * (HM / WM), wn = wni * (HN / WN);
  f4 acc[2][2][TI][TJ];  // quadrant (A half, B half)
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) acc[q >> 1][q & 1][i][j] = f4{0.f, 0.f, 0.f, 0.f};
  w4 fa[2][2 * TI], fb[2][2 * TJ];  // operands of the halves: K elements 0 .. 31, then 32 .. 63
  auto read_a = [&](int stage, int h, int q) {
    fa[h][q] = LA::frag(ring + stage * STAGE + h * LA::kBytes, wm + 16 * (q % TI), q / TI, lane);
  };
  auto read_b = [&](int stage, int h, int q) {
    fb[h][q] = LB::frag(ring + stage * STAGE + 2 * LA::kBytes + h * LB::kBytes, wn + 16 * (q % TJ), q / TJ, lane);
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
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int b = r / (2 * TI), kh = r / TI & 1, i = r % TI;
#pragma unroll
      for (int j = 0; j < TJ; ++j)
        acc[h][b][i][j] = mfma(Op::get(fb[b][kh * TJ + j]), Op::get(fa[h][kh * TI + i]), acc[h][b][i][j]);  // C^T tiles
      __builtin_amdgcn_sched_barrier(0);
      if (h == 0) {
#pragma unroll
        for (int q = r * RR; q < (r + 1) * RR; ++q) {
          if (q < 2 * TJ)
            read_b(stage, 1, q);
          else if (q < 2 * TJ + 2 * TI)
            read_a(stage, 1, q - 2 * TJ);
        }
      } else {
#pragma unroll
        for (int q = r * RR; q < (r + 1) * RR; ++q)
          if (q < 2 * TI) read_a(stage ^ 1, 0, q);
#pragma unroll
        for (int q = (r - ROWS / 2) * RR; q < (r - ROWS / 2 + 1) * RR; ++q)  // B0's registers are free after its products
          if (q >= 0 && q < 2 * TJ) read_b(stage ^ 1, 0, q);
        if (r == ROWS / 2) next();
      }
#pragma unroll
      for (int q = r * DR; q < (r + 1) * DR && q < PL; ++q)
        if (h == 0 || r < ROWS / 2) transfer(stage, h, q);
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
    for (int q = 0; q < 2 * PL; ++q) transfer(k, q / PL, q % PL);
  }
  next();
  ring_wait<2 * PL>();
#pragma unroll
  for (int q = 0; q < 2 * TI; ++q) read_a(0, 0, q);
#pragma unroll
  for (int q = 0; q < 2 * TJ; ++q) read_b(0, 0, q);
  ring_sync();
  for (int k = 0; k < steps; ++k) {
    part(0, k & 1);
    part(1, k & 1);
  }
  ring_wait<0>();  // no transfer is in flight when the work-group ends

  // Lane (r16, kq) holds, of an MFMA tile of C, row r16 and columns 4 kq .. 4 kq + 3.
  // Two column tiles side by side exchange lane rows, so that it holds 8 consecutive
  // columns of one of them: 16 (kq % 2) + 8 (kq / 2) .. + 7 of the pair.
  const int64_t ldc = p.ldc;
  if (EPI == kFfnStore && g.ksplit > 1) {
    float* out = g.part + bz * g.part_slice + p.part_off;
#pragma unroll
    for (int hi = 0; hi < 2 * TI; ++hi) {
      const int m = mb + hi / TI * HM + wm + 16 * (hi % TI) + r16;
      if (m >= p.M) continue;
#pragma unroll
      for (int hj = 0; hj < 2 * TJ; ++hj) {
        const int n = nb + hj / TJ * HN + wn + 16 * (hj % TJ) + 4 * kq;
        if (n < p.N) *reinterpret_cast<f4*>(out + (int64_t)m * p.N + n) = acc[hi / TI][hj / TJ][hi % TI][hj % TJ];
      }
    }
    return;
  }
  constexpr int CW = TJ % 2 ? 4 : 8, NQ = TJ * 4 / CW;  // consecutive columns of a lane, and how often in a half
  const int cofs = CW == 8 ? 16 * (kq & 1) + 8 * (kq >> 1) : 4 * kq;
#pragma unroll
  for (int hi = 0; hi < 2 * TI; ++hi) {
    float x[2][NQ][CW];
#pragma unroll
    for (int q = 0; q < 2 * NQ; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int h = q / NQ, j = q % NQ;
        if constexpr (CW == 8) {
          x[h][j][e] = acc[hi / TI][h][hi % TI][2 * j][e];
          x[h][j][4 + e] = acc[hi / TI][h][hi % TI][2 * j + 1][e];
          swap_rows(x[h][j][e], x[h][j][4 + e]);
        } else {
          x[h][j][e] = acc[hi / TI][h][hi % TI][j][e];
        }
      }
    const int m = mb + hi / TI * HM + wm + 16 * (hi % TI) + r16;
    if (m >= p.M) continue;
    if constexpr (DUAL) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const int n = nb + wn + 4 * CW * q + cofs;
        if (n >= p.N) continue;
        const int64_t off = 2 * ((int64_t)m * ldc + n);
        if (g.gate) ffn_store<DT, CW>(g.gate + off, x[0][q]);
        if (g.value) ffn_store<DT, CW>(g.value + off, x[1][q]);
        float o[CW], s;
#pragma unroll
        for (int e = 0; e < CW; ++e) o[e] = ffn_act(x[0][q][e], g.act, s) * x[1][q][e];
        ffn_store<DT, CW>(p.c + off, o);
      }
    } else {
#pragma unroll
      for (int hq = 0; hq < 2 * NQ; ++hq) {
        float(&v)[CW] = x[hq / NQ][hq % NQ];
        const int n = nb + hq / NQ * HN + wn + 4 * CW * (hq % NQ) + cofs;
        if (n >= p.N) continue;
        const int64_t off = (int64_t)m * ldc + n;
        if constexpr (EPI == kFfnGateGrad) {
          float gt[CW], vl[CW], dg[CW], dv[CW], hh[CW];
          ffn_load<DT, CW>(g.gate + 2 * off, gt);
          ffn_load<DT, CW>(g.value + 2 * off, vl);
#pragma unroll
          for (int e = 0; e < CW; ++e) {
            float s;
            const float a = ffn_act(gt[e], g.act, s);
            dg[e] = v[e] * vl[e] * s;
            dv[e] = v[e] * a;
            hh[e] = a * vl[e];
          }
          ffn_store<DT, CW>(g.dgate + 2 * off, dg);
          ffn_store<DT, CW>(g.dvalue + 2 * off, dv);
          if (p.c) ffn_store<DT, CW>(p.c + 2 * off, hh);
        } else {
          if (p.res) {
            float r[CW];
            if (g.cdt == GTR_F32)
              ffn_load<GTR_F32, CW>(p.res + 4 * off, r);
            else
              ffn_load<DT, CW>(p.res + 2 * off, r);
#pragma unroll
            for (int e = 0; e < CW; ++e) v[e] += r[e];
          }
          if (g.cdt == GTR_F32)
            ffn_store<GTR_F32, CW>(p.c + 4 * off, v);
          else
            ffn_store<DT, CW>(p.c + 2 * off, v);
        }
      }
    }
  }
}

// C = the sum of the slices' partial sums (+ res), 8 elements per thread.
template <int DT>
__global__ void __launch_bounds__(256) ffn_reduce_kernel(FfnGemm g) {
  int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (t >= g.part_slice) return;
  int pi = 0;
  while (pi + 1 < g.nprod && t >= g.p[pi + 1].part_off) ++pi;
  const FfnProd& p = g.p[pi];
  float x[8];
  load8(g.part, GTR_F32, t, x);
#pragma unroll 4
  for (int s = 1; s < g.ksplit; ++s) {
    float y[8];
    load8(g.part, GTR_F32, s * g.part_slice + t, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += y[e];
  }
  const int64_t off = t - p.part_off;  // (C is contiguous)
  if (p.res) {
    float y[8];
    load8(p.res, g.cdt, off, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += y[e];
  }
  if (g.cdt == GTR_F32)
    ffn_store<GTR_F32, 8>(p.c + 4 * off, x);
  else
    ffn_store<DT, 8>(p.c + 2 * off, x);
}

}  // namespace gtr
