// Dropout with the residual's addition (sm_100a).  Bound by memory: every value is read and written once, the mask is worked
// out from the counters.
#pragma once
#include "accept_drop.cuh"

namespace accept {

struct DropoutArgs {
  const void* x;
  const void* residual;  // may be null
  void* y;
  uint64_t rows, cols, ld_x, ld_y;
  uint64_t per_row, units;  // units of eight neighbours
  Drop drop;
};

// Eight neighbours at p, of which the first n exist.
template <typename T, bool VEC>
__device__ __forceinline__ void load_eight(const T* p, int n, Pair (&v)[4]) {
  if (VEC && n == 8) {
    uint4 w[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = ld_c(reinterpret_cast<const uint4*>(p) + i);
    if constexpr (sizeof(T) == 4) {
      v[0] = pair_of(__uint_as_float(w[0].x), __uint_as_float(w[0].y));
      v[1] = pair_of(__uint_as_float(w[0].z), __uint_as_float(w[0].w));
      v[2] = pair_of(__uint_as_float(w[1].x), __uint_as_float(w[1].y));
      v[3] = pair_of(__uint_as_float(w[1].z), __uint_as_float(w[1].w));
    } else {
      v[0] = word_to_pair<T>(w[0].x); v[1] = word_to_pair<T>(w[0].y); v[2] = word_to_pair<T>(w[0].z); v[3] = word_to_pair<T>(w[0].w);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pair_of(2 * j < n ? to_float(ld_c(p + 2 * j)) : 0.0f, 2 * j + 1 < n ? to_float(ld_c(p + 2 * j + 1)) : 0.0f);
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_eight(T* p, int n, const Pair (&v)[4]) {
  if (VEC && n == 8) {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(T) == 4) { w[2 * j] = __float_as_uint(split(v[j]).x); w[2 * j + 1] = __float_as_uint(split(v[j]).y); }
      else w[j] = pair_to_word<T>(v[j]);
    }
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
      if (bounds_ok(reinterpret_cast<uint4*>(p) + i, 16, true)) __stcs(reinterpret_cast<uint4*>(p) + i, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = split(v[j]);
      if (2 * j < n) st_c(p + 2 * j, from_float<T>(f.x));
      if (2 * j + 1 < n) st_c(p + 2 * j + 1, from_float<T>(f.y));
    }
  }
}

constexpr int kDropThreads = 256;

// A matrix without gaps is one row (the counters run on from row to row): a thread takes UNITS units of eight neighbours, a block's
// width apart, all loads first.
template <typename TX, typename TY, int UNITS>
__global__ void __launch_bounds__(kDropThreads) dropout_flat_kernel(const DropoutArgs a) {
  grid_dependency_handshake();
  constexpr uint32_t kStride = 8 * kDropThreads;
  const uint64_t c0 = ((uint64_t)blockIdx.x * (UNITS * kDropThreads) + threadIdx.x) * 8;
  const TX* x = static_cast<const TX*>(a.x) + c0;
  const TY* residual = static_cast<const TY*>(a.residual) + c0;
  TY* y = static_cast<TY*>(a.y) + c0;
  const uint64_t first = a.drop.offset + c0;
  const DropRow row(a.drop.rng, first, DropKey(a.drop.rng, first));
  if (c0 + (UNITS - 1) * kStride + 8 <= a.cols) {
    Pair v[UNITS][4], add[UNITS][4];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) load_eight<TX, true>(x + i * kStride, 8, v[i]);
    if (a.residual)
#pragma unroll
      for (int i = 0; i < UNITS; ++i) load_eight<TY, true>(residual + i * kStride, 8, add[i]);
    if (a.drop.on) drop_units<8, UNITS>(a.drop, row, 0, kStride, &v[0][0]);
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      if (a.residual)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = add2(v[i][j], add[i][j]);
      store_eight<TY, true>(y + i * kStride, 8, v[i]);
    }
  } else {
#pragma unroll 1
    for (int i = 0; i < UNITS; ++i) {
      const uint64_t c = c0 + i * kStride;
      const int n = c < a.cols ? (int)min(a.cols - c, (uint64_t)8) : 0;
      if (n == 0) break;
      Pair v[4], add[4];
      load_eight<TX, true>(x + i * kStride, n, v);
      if (a.residual) load_eight<TY, true>(residual + i * kStride, n, add);
      if (a.drop.on) drop_units<8, 1>(a.drop, row, i * kStride, 0, v);
      if (a.residual)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = add2(v[j], add[j]);
      store_eight<TY, true>(y + i * kStride, n, v);
    }
  }
}

// Other matrices: the units of all rows in turn, a division for each.
template <typename TX, typename TY, bool VEC, int UNITS>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const DropoutArgs a) {
  grid_dependency_handshake();
  const uint64_t first = (uint64_t)blockIdx.x * (UNITS * kDropThreads) + threadIdx.x;
  Pair v[UNITS][4], add[UNITS][4];
  uint64_t row[UNITS], col[UNITS];
  int n[UNITS];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const uint64_t u = first + i * kDropThreads;
    row[i] = a.units <= 0xffffffffu ? (uint32_t)u / (uint32_t)a.per_row : u / a.per_row;
    col[i] = (u - row[i] * a.per_row) * 8;
    n[i] = u < a.units ? (int)min(a.cols - col[i], (uint64_t)8) : 0;
    if (n[i] == 0) continue;
    load_eight<TX, VEC>(static_cast<const TX*>(a.x) + row[i] * a.ld_x + col[i], n[i], v[i]);
    if (a.residual) load_eight<TY, VEC>(static_cast<const TY*>(a.residual) + row[i] * a.ld_y + col[i], n[i], add[i]);
  }
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    if (n[i] == 0) continue;
    if (a.drop.on) {
      const uint64_t at = a.drop.offset + row[i] * a.cols + col[i];
      drop_units<8, 1>(a.drop, DropRow(a.drop.rng, at, DropKey(a.drop.rng, at)), 0, 0, v[i]);
    }
    if (a.residual)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i][j] = add2(v[i][j], add[i][j]);
    store_eight<TY, VEC>(static_cast<TY*>(a.y) + row[i] * a.ld_y + col[i], n[i], v[i]);
  }
}

}  // namespace accept
