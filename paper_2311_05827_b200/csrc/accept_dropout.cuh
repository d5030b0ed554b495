// Dropout with the residual's addition (sm_100a).  Bound by memory: every value is read and written once, the mask is worked
// out from the counters.
#pragma once
#include "accept_drop.cuh"
#include "accept_shift.cuh"

namespace accept {

struct DropoutArgs {
  const void* x;
  const void* residual;  // may be null
  void* y;
  uint64_t rows, cols, ld_x, ld_y;
  Drop drop;
  int log_units;  // see dropout_kernel
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
    if (sizeof(T) == 4 && (reinterpret_cast<uintptr_t>(p) & 31) == 0) {  // whole 32-byte sectors (fp32 values of 4 bits, 16384 x 4096: 75 -> 52 us)
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
      st_octet(reinterpret_cast<float*>(p), f);
      return;
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

// Other matrices: a block takes 2^log_units units of eight neighbours of ROWS times as many rows as that leaves threads for.  Units
// start on y's 16-byte boundaries; what is read there is shifted, and the ends of a row leave value by value.
// FEW: so few rows that the first and the last count, beside which nothing may be read: there only the units at the very ends are read
// value by value (1 x 30000001 bf16 off a boundary 439 -> 84 us).
template <typename TX, typename TY, int ROWS, bool FEW>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const DropoutArgs a) {
  grid_dependency_handshake();
  constexpr uint32_t kEach = 16 / (uint32_t)sizeof(TY);
  const uint32_t rows_at_once = kDropThreads >> a.log_units;
  const uint64_t unit = ((uint64_t)blockIdx.x << a.log_units) + (threadIdx.x & ((1u << a.log_units) - 1));
  const bool behind_start = unit > 0, before_end = unit * 8 + 9 < a.cols;
  const uint64_t groups = (a.rows + rows_at_once * ROWS - 1) / (rows_at_once * ROWS);
  const DropKey key(a.drop.rng, a.drop.offset + blockIdx.y * (uint64_t)(rows_at_once * ROWS) * a.cols);
  for (uint64_t group = blockIdx.y; group < groups; group += gridDim.y) {
    const uint64_t r0 = group * (rows_at_once * ROWS) + (threadIdx.x >> a.log_units);
    Pair v[ROWS][4], add[ROWS][4];
    int64_t col[ROWS];
    int lo[ROWS], hi[ROWS];
    const TX* x[ROWS];
    const TY* residual[ROWS];
    bool inner = true;  // all eight exist, and the value before and the two behind lie in the matrix
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const uint64_t r = r0 + i * rows_at_once;
      const uint32_t before = (uint32_t)((reinterpret_cast<uintptr_t>(a.y) / sizeof(TY) + r * a.ld_y) % kEach);  // values between the boundary and the row
      col[i] = (int64_t)(unit * 8) - before;
      lo[i] = col[i] < 0 ? (int)-col[i] : 0;
      hi[i] = r < a.rows ? (int)min(max((int64_t)a.cols - col[i], (int64_t)0), (int64_t)8) : 0;
      x[i] = static_cast<const TX*>(a.x) + (int64_t)(r * a.ld_x) + col[i];
      residual[i] = static_cast<const TY*>(a.residual) + (int64_t)(r * a.ld_y) + col[i];
      inner = inner && lo[i] == 0 && hi[i] == 8 && ((FEW && behind_start) || r > 0) && ((FEW && before_end) || r + 1 < a.rows);
    }
    if (inner) {
      RawEight<TX> raw_x[ROWS];
      RawEight<TY> raw_r[ROWS];
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        load_raw<TX>(x[i], raw_x[i]);
        if (a.residual) load_raw<TY>(residual[i], raw_r[i]);
      }
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        uint32_t w[2 * sizeof(TX)], u[2 * sizeof(TY)];
        words_of<TX>(raw_x[i], x[i], w);
        pairs_of<TX>(w, v[i]);
        if (a.residual) {
          words_of<TY>(raw_r[i], residual[i], u);
          pairs_of<TY>(u, add[i]);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        uint32_t w[2 * sizeof(TX)], u[2 * sizeof(TY)];
        load_some<TX>(x[i], lo[i], hi[i], w);
        pairs_of<TX>(w, v[i]);
        if (a.residual) {
          load_some<TY>(residual[i], lo[i], hi[i], u);
          pairs_of<TY>(u, add[i]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      if (hi[i] <= lo[i]) continue;
      const uint64_t r = r0 + i * rows_at_once;
      // (counters before the row's first are drawn and dropped where it starts inside the unit)
      if (a.drop.on) drop_units<8, 1>(a.drop, DropRow(a.drop.rng, a.drop.offset + r * a.cols + (uint64_t)col[i], key), 0, 0, v[i]);
      if (a.residual)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = add2(v[i][j], add[i][j]);
      TY* y = static_cast<TY*>(a.y) + (int64_t)(r * a.ld_y) + col[i];
      if (lo[i] == 0 && hi[i] == 8) {
        store_eight<TY, true>(y, 8, v[i]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 f = split(v[i][e / 2]);
          if (e >= lo[i] && e < hi[i]) st_c(y + e, from_float<TY>(e % 2 ? f.y : f.x));
        }
      }
    }
  }
}

}  // namespace accept
