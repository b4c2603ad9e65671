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

// 8 consecutive elements of type dt (16-bit or float32) at p.
template <int DT>
__device__ __forceinline__ void ffn_load8(const char* p, float (&x)[8]) {
  load8(p, DT, 0, x);
}
template <int DT>
__device__ __forceinline__ w4 ffn_pack8(const float (&x)[8]) {
  w4 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (DT == GTR_F16) {
      r[e] = __builtin_bit_cast(unsigned short, (_Float16)x[2 * e]) |
             (unsigned)__builtin_bit_cast(unsigned short, (_Float16)x[2 * e + 1]) << 16;
    } else {
      r[e] = __builtin_bit_cast(unsigned short, (__bf16)x[2 * e]) |
             (unsigned)__builtin_bit_cast(unsigned short, (__bf16)x[2 * e + 1]) << 16;
    }
  }
  return r;
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
    return BT == 256 ? m | q << 2 : BT == 128 ? m >> 1 | q << 1 : q;
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
template <int DT, int TA, int TB, int EPI, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(2))) ffn_gemm_kernel(FfnGemm g) {
  typedef Operand<DT, DT> Op;
  constexpr int NW = WM * WN;
  constexpr int TI = BM / (16 * WM), TJ = BN / (16 * WN);
  typedef FfnTile<TA, BM, NW> LA;
  typedef FfnTile<TB, BN, NW> LB;
  constexpr int STAGE = LA::kBytes + LB::kBytes;
  constexpr bool DUAL = EPI == kFfnGate;
  constexpr int BC = DUAL ? BN / 2 : BN;  // columns of C of a tile
  static_assert(TJ % 2 == 0 && (!DUAL || (TJ == 4 && TB == 0)), "epilogue pairs");
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

  unsigned va[LA::P], vb[LB::P];
#pragma unroll
  for (int q = 0; q < LA::P; ++q) va[q] = LA::voff(wave + NW * q, lane, p.lda);
#pragma unroll
  for (int q = 0; q < LB::P; ++q) vb[q] = LB::voff((wave + NW * q) % (DUAL ? BC / 8 : BN), lane, p.ldb);

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
  // This wave's transfer q of that step to a stage. In the last step of a segment a
  // row's next elements are another row's: out of range instead. (A wave's transfers
  // c are all even or all odd, so a lane's piece is at the same K element in each.)
  const int pk = LA::piece_k(wave, lane);
  auto transfer = [&](int buf, int q) {
    const unsigned l = lbase + buf * STAGE;
    if (q < LA::P) {
      dma16_buf(ra, !TA && pk >= kleft ? kFfnOob : va[q], l + NW * 1024 * q);
    } else {
      const int u = q - LA::P;
      dma16_buf(DUAL && u >= LB::P / 2 ? rv : rb, !TB && pk >= kleft ? kFfnOob : vb[u], l + LA::kBytes + NW * 1024 * u);
    }
  };

  const int wm = wmi * (BM / WM);
  f4 acc[TI][TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
  // operand q of half a step: B's column tiles, then A's row tiles
  auto read = [&](int buf, int h, int q, w4(&fa)[TI], w4(&fb)[TJ]) {
    const char* s = ring + buf * STAGE;
    if (q < TJ) {
      const int r0 = DUAL ? (q >> 1) * BC + wni * (BC / WN) + 16 * (q & 1) : wni * (BN / WN) + 16 * q;
      fb[q] = LB::frag(s + LA::kBytes, r0, h, lane);
    } else {
      fa[q - TJ] = LA::frag(s, wm + 16 * (q - TJ), h, lane);
    }
  };
  // Half a step's products, a row of tiles at a time, and between the rows the reads
  // of the next half's operands and (D) the transfers of a later step: the matrix
  // cores work while the wave issues them.
  constexpr int PL = LA::P + LB::P;
  auto half = [&](const w4(&fa)[TI], const w4(&fb)[TJ], int rbuf, int rh, w4(&na)[TI], w4(&nb)[TJ], int dbuf) {
    constexpr int RR = TI > 1 ? (TI + TJ + TI - 2) / (TI - 1) : TI + TJ;  // reads per row, all of them before the last row
    constexpr int DR = (PL + TI - 1) / TI;
    static_assert(RR * TI >= TI + TJ && DR * TI >= PL, "every read and every transfer has its row");
#pragma unroll
    for (int i = 0; i < TI; ++i) {
#pragma unroll
      for (int j = 0; j < TJ; ++j) acc[i][j] = mfma(Op::get(fb[j]), Op::get(fa[i]), acc[i][j]);  // C^T tiles
      __builtin_amdgcn_sched_barrier(0);
      if (dbuf < 0 && i == TI / 2) next();
#pragma unroll
      for (int q = i * RR; q < (i + 1) * RR && q < TI + TJ; ++q) read(rbuf, rh, q, na, nb);
      if (dbuf >= 0) {
#pragma unroll
        for (int q = i * DR; q < (i + 1) * DR && q < PL; ++q) transfer(dbuf, q);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  w4 fa0[TI], fb0[TJ], fa1[TI], fb1[TJ];
  next();
#pragma unroll
  for (int q = 0; q < PL; ++q) transfer(0, q);
  next();
#pragma unroll
  for (int q = 0; q < PL; ++q) transfer(1, q);
  ring_wait<PL>();
#pragma unroll
  for (int q = 0; q < TI + TJ; ++q) read(0, 0, q, fa0, fb0);
  for (int k = 0; k < steps; ++k) {
    half(fa0, fb0, k & 1, 1, fa1, fb1, -1);
    // every wave has read this stage, and its transfers into the next one have landed
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0), known to the compiler: no waits for these reads below
    ring_wait<0>();
    half(fa1, fb1, (k + 1) & 1, 0, fa0, fb0, k & 1);
  }
  ring_wait<0>();  // no transfer is in flight when the work-group ends

  // Lane (r16, kq) holds C[row 16 i + r16][columns 16 j + 4 kq .. + 3] of its
  // wave's block. Two column tiles exchange lane rows, so that it holds 8
  // consecutive columns of one of them: 16 j' + 8 (kq / 2) .. + 7, j' = j + kq % 2.
  const int64_t ldc = p.ldc;
  if (EPI == kFfnStore && g.ksplit > 1) {
    float* out = g.part + bz * g.part_slice + p.part_off;
#pragma unroll
    for (int i = 0; i < TI; ++i) {
      const int m = mb + wm + 16 * i + r16;
      if (m >= p.M) continue;
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        const int n = nb + wni * (BN / WN) + 16 * j + 4 * kq;
        if (n < p.N) *reinterpret_cast<f4*>(out + (int64_t)m * p.N + n) = acc[i][j];
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < TI; ++i) {
    float x[TJ / 2][8];
#pragma unroll
    for (int q = 0; q < TJ / 2; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[q][e] = acc[i][2 * q][e];
        x[q][4 + e] = acc[i][2 * q + 1][e];
        swap_rows(x[q][e], x[q][4 + e]);
      }
    const int m = mb + wm + 16 * i + r16;
    if (m >= p.M) continue;
    if constexpr (DUAL) {
      const int n = nb + wni * (BC / WN) + 16 * (kq & 1) + 8 * (kq >> 1);
      if (n < p.N) {
        const int64_t off = 2 * ((int64_t)m * ldc + n);
        if (g.gate) *reinterpret_cast<w4*>(g.gate + off) = ffn_pack8<DT>(x[0]);
        if (g.value) *reinterpret_cast<w4*>(g.value + off) = ffn_pack8<DT>(x[1]);
        float o[8], s;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = ffn_act(x[0][e], g.act, s) * x[1][e];
        *reinterpret_cast<w4*>(p.c + off) = ffn_pack8<DT>(o);
      }
    } else {
#pragma unroll
      for (int q = 0; q < TJ / 2; ++q) {
        const int n = nb + wni * (BN / WN) + 32 * q + 16 * (kq & 1) + 8 * (kq >> 1);
        if (n >= p.N) continue;
        const int64_t off = (int64_t)m * ldc + n;
        if constexpr (EPI == kFfnGateGrad) {
          float gt[8], vl[8], dg[8], dv[8], h[8];
          ffn_load8<DT>(g.gate + 2 * off, gt);
          ffn_load8<DT>(g.value + 2 * off, vl);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float s;
            const float a = ffn_act(gt[e], g.act, s);
            dg[e] = x[q][e] * vl[e] * s;
            dv[e] = x[q][e] * a;
            h[e] = a * vl[e];
          }
          *reinterpret_cast<w4*>(g.dgate + 2 * off) = ffn_pack8<DT>(dg);
          *reinterpret_cast<w4*>(g.dvalue + 2 * off) = ffn_pack8<DT>(dv);
          if (p.c) *reinterpret_cast<w4*>(p.c + 2 * off) = ffn_pack8<DT>(h);
        } else {
          if (p.res) {
            float r[8];
            load8(p.res, g.cdt, off, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[q][e] += r[e];
          }
          if (g.cdt == GTR_F32)
            store_n<8>(p.c, GTR_F32, off, x[q]);
          else
            *reinterpret_cast<w4*>(p.c + 2 * off) = ffn_pack8<DT>(x[q]);
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
    store_n<8>(p.c, GTR_F32, off, x);
  else
    *reinterpret_cast<w4*>(p.c + 2 * off) = ffn_pack8<DT>(x);
}

}  // namespace gtr
