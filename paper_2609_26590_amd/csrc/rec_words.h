// The words in which the recurrence's tiles hand on their maps, and the wait for them.
#pragma once

namespace gtr {

// A map s -> P s + E in one 64-bit word that is its own flag: zero until it is written (~P in
// the low half, which no P leaves zero).
__device__ __forceinline__ unsigned long long rec_word(float P, float E) {
  unsigned lo = ~__builtin_bit_cast(unsigned, P);
  lo = lo ? lo : ~0x7fc00000u;  // (a NaN with every bit set becomes another one)
  return (unsigned long long)__builtin_bit_cast(unsigned, E) << 32 | lo;
}
__device__ __forceinline__ float rec_map(unsigned long long w) { return __builtin_bit_cast(float, ~(unsigned)w); }
__device__ __forceinline__ float rec_add(unsigned long long w) { return __builtin_bit_cast(float, (unsigned)(w >> 32)); }

// N words of this lane's V channels each, once all lanes have all of theirs; NaN maps if they
// have not after spin + 1 polls.
template <int V, int N>
__device__ __forceinline__ void rec_wait(unsigned long long (&w)[N][V], const unsigned long long* const (&at)[N],
                                         unsigned spin) {
  for (unsigned n = 0;; ++n) {
    bool all = true;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        w[i][v] = __hip_atomic_load(at[i] + v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        all &= (unsigned)w[i][v] != 0u;
      }
    if (__all(all)) return;
    if (n >= spin) break;
    __builtin_amdgcn_s_sleep(1);
  }
  const float nan = __builtin_bit_cast(float, 0x7fc00000u);
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int v = 0; v < V; ++v) w[i][v] = rec_word(nan, nan);
}

}  // namespace gtr
