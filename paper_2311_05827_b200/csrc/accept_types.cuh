// Values of the three floating types the operators beside the codec read and write.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "accept_device.cuh"

namespace accept {

constexpr int kF32 = 0, kBf16 = 1, kF16 = 2;  // accept_dtype

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// ---- pairs: sm_100 adds, multiplies and fuses two fp32 values with one instruction, each rounded as by itself ----
// A pair is one 64-bit register pair from its load to its store.
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair_of(float lo, float hi) {
  Pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 split(Pair b) {
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(b));
  return v;
}
__device__ __forceinline__ Pair both(float v) { return pair_of(v, v); }
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float sum_of(Pair v) {
  const float2 f = split(v);
  return f.x + f.y;
}
// Two 16-bit values of a word, the lower first.
template <typename T> __device__ __forceinline__ Pair word_to_pair(uint32_t w);
template <> __device__ __forceinline__ Pair word_to_pair<__nv_bfloat16>(uint32_t w) {  // bf16 is the upper half of an fp32
  return pair_of(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ Pair word_to_pair<__half>(uint32_t w) {
  __half2 h;
  memcpy(&h, &w, 4);
  const float2 f = __half22float2(h);
  return pair_of(f.x, f.y);
}
template <typename T> __device__ __forceinline__ uint32_t pair_to_word(Pair v);
template <> __device__ __forceinline__ uint32_t pair_to_word<__nv_bfloat16>(Pair p) {
  const float2 v = split(p);
  const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
  uint32_t w;
  memcpy(&w, &h, 4);
  return w;
}
template <> __device__ __forceinline__ uint32_t pair_to_word<__half>(Pair p) {
  const float2 v = split(p);
  const __half2 h = __floats2half2_rn(v.x, v.y);
  uint32_t w;
  memcpy(&w, &h, 4);
  return w;
}

// Eight values as they lie in memory: 16 bytes for the 16-bit types, 32 for fp32.
template <typename T> struct Pack { uint4 w[sizeof(T) / 2]; };

template <typename T>
__device__ __forceinline__ Pack<T> ld_pack(const T* p) {
  Pack<T> v;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
    if (!bounds_ok(reinterpret_cast<const uint4*>(p) + i, 16, false)) { v.w[i] = make_uint4(0, 0, 0, 0); continue; }
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.w[i].x), "=r"(v.w[i].y), "=r"(v.w[i].z), "=r"(v.w[i].w) : "l"(reinterpret_cast<const uint4*>(p) + i));
  }
  return v;
}

}  // namespace accept
