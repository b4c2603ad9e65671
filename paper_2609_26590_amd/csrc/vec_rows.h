// Rows of float32, fp16 or bf16 in 16-byte vectors at whatever address they start, for the
// normalisation kernels.
#pragma once

#include <hip/hip_runtime.h>

#include "gtr.h"
#include "gtr_device.h"

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
  static __device__ __forceinline__ void put(char* p, float x) {
    *reinterpret_cast<unsigned short*>(p) = f32_to_bf16_bits(x);
  }
};

// A lane's vector of a row: VE columns from c on. A row whose width is no multiple of
// VE ends with a vector that starts early, at d - VE, and holds `skip` columns that
// are the vector's before it: they count as zeros and are not stored. (Where the whole
// row is shorter than a vector, TINY, its elements go one by one.) Lanes past the
// row's end have the last vector with every column skipped.
template <int DT, bool TINY>
struct LnCols {
  static constexpr int VE = Ln<DT>::VE, ES = Ln<DT>::ES;
  int c, skip;
  __device__ __forceinline__ LnCols(int index, int d) {
    const int at = index * VE;
    c = TINY ? at : min(at, d - VE);
    skip = TINY ? max(0, min(VE, VE - (d - at))) : min(VE, at - c);  // TINY: columns past the end
  }
  __device__ __forceinline__ bool has(int e) const { return TINY ? e < VE - skip : e >= skip; }
  __device__ __forceinline__ Vec16 load(const char* row) const {
    if constexpr (!TINY) {
      return *reinterpret_cast<const Vec16*>(row + (int64_t)c * ES);
    } else {
      Vec16 r = {{0, 0, 0, 0}};
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (has(e)) {
          if constexpr (ES == 4)
            r.u[e] = *reinterpret_cast<const unsigned*>(row + (int64_t)(c + e) * ES);
          else
            r.u[e / 2] |= (unsigned)*reinterpret_cast<const unsigned short*>(row + (int64_t)(c + e) * ES) << (16 * (e & 1));
        }
      return r;
    }
  }
  __device__ __forceinline__ void unpack(const Vec16& r, float (&x)[VE]) const {
    Ln<DT>::unpack(r, x);
#pragma unroll
    for (int e = 0; e < VE; ++e) x[e] = has(e) ? x[e] : 0.f;
  }
  __device__ __forceinline__ void store(char* row, const float (&x)[VE]) const {
    if (skip == 0) {
      *reinterpret_cast<Vec16*>(row + (int64_t)c * ES) = Ln<DT>::pack(x);
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (has(e)) Ln<DT>::put(row + (int64_t)(c + e) * ES, x[e]);
    }
  }
  // of a float32 vector of d, or `fill` everywhere if there is none
  __device__ __forceinline__ void load_f32(const float* p, float fill, float (&x)[VE]) const {
    if (TINY || !p) {
#pragma unroll
      for (int e = 0; e < VE; ++e) x[e] = p && has(e) ? p[c + e] : fill;
    } else {
#pragma unroll
      for (int h = 0; h < VE / 4; ++h) {
        const Vec16 r = *reinterpret_cast<const Vec16*>(p + c + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * h + e] = __builtin_bit_cast(float, r.u[e]);
      }
    }
  }
};

}  // namespace gtr
