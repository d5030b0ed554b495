// Values that do not start on a 16-byte boundary: aligned pieces are read and shifted.
#pragma once
#include "accept_types.cuh"

namespace accept {

// Words `by` bytes (a multiple of 2, the same for the whole warp) into `c`, of which there are N + M.
template <int N, int M>
__device__ __forceinline__ void shifted_words(const uint32_t (&c)[N + M], uint32_t by, uint32_t (&out)[N]) {
  uint32_t w[N + M];
#pragma unroll
  for (int i = 0; i < N + M; ++i) w[i] = c[i];
#pragma unroll
  for (int step = M / 2; step >= 1; step /= 2)  // by / 4 is below M, a power of two
#pragma unroll
    for (int i = 0; i + step < N + M; ++i) w[i] = by & 4 * step ? w[i + step] : w[i];
  const uint32_t pick = by & 2 ? 0x5432u : 0x3210u;
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = __byte_perm(w[i], w[i + 1], pick);
}

// Eight neighbours at p, a 16-bit type's from five 4-byte words: where p is off a word, the value before and the one behind are read too,
// else the two behind.  The words of several units are loaded before the first is used.
template <typename T> struct RawEight { uint32_t c[sizeof(T) == 2 ? 5 : 8]; };
__device__ __forceinline__ uint32_t ld_word(uintptr_t p) {
  uint32_t w = 0;
  if (bounds_ok(reinterpret_cast<const void*>(p), 4, false)) asm volatile("ld.global.u32 %0, [%1];" : "=r"(w) : "l"(p) : "memory");
  return w;
}
template <typename T>
__device__ __forceinline__ void load_raw(const T* p, RawEight<T>& r) {
  const uintptr_t from = reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)3;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r.c) / 4); ++i) r.c[i] = ld_word(from + 4 * i);
}
template <typename T>
__device__ __forceinline__ void words_of(const RawEight<T>& r, const T* p, uint32_t (&w)[2 * sizeof(T)]) {
  const uint32_t pick = reinterpret_cast<uintptr_t>(p) & 2 ? 0x5432u : 0x3210u;
#pragma unroll
  for (int i = 0; i < (int)(2 * sizeof(T)); ++i) w[i] = sizeof(T) == 2 ? __byte_perm(r.c[i], r.c[(i + 1) % (sizeof(r.c) / 4)], pick) : r.c[i];
}
template <typename T>
__device__ __forceinline__ void pairs_of(const uint32_t (&w)[2 * sizeof(T)], Pair (&v)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(T) == 4) v[j] = pair_of(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
    else v[j] = word_to_pair<T>(w[j]);
  }
}
// Those of eight neighbours at p from `lo` on and below `hi`, one by one; zero for the others.
template <typename T>
__device__ __forceinline__ void load_some(const T* p, int lo, int hi, uint32_t (&w)[2 * sizeof(T)]) {
#pragma unroll
  for (int i = 0; i < (int)(2 * sizeof(T)); ++i) w[i] = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (sizeof(T) == 4) {
      if (e >= lo && e < hi) w[e] = __float_as_uint(ld_c(reinterpret_cast<const float*>(p) + e));
    } else {
      uint16_t v = 0;
      if (e >= lo && e < hi) v = ld_c(reinterpret_cast<const uint16_t*>(p) + e);
      w[e / 2] |= (uint32_t)v << 16 * (e % 2);
    }
  }
}

}  // namespace accept
