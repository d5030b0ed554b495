// Quantisation to 8-bit floating point with one power-of-two scale for each block of 128 values (sm_100a).
//
// One block of threads codes a tile of 128 x 128 values, read once and held in registers, along its rows, along its
// columns (through shared memory, so that both outputs leave in runs of 128 bytes), or both.
#pragma once
#include "accept_types.cuh"

namespace accept {

constexpr int kE4m3 = 0, kE5m2 = 1;  // accept_format
constexpr int kTile = 128;           // rows and columns of a tile; also the length of a block

struct BlockArgs {
  const void* x;
  uint8_t* q;        // rows, may be null
  uint8_t* scale;
  uint8_t* qt;       // columns, may be null
  uint8_t* scale_t;
  uint32_t* status;
  uint64_t ld;
  uint32_t rows, cols;
  uint32_t ldq, ldqt;         // bytes between coded rows: cols, rows rounded up to 16
  uint32_t tiles_r, tiles_c;  // tiles over the rows and the columns
  int square;
};

// Exponent e of a block's scale from the bits of its largest magnitude a (finite): the least integer with
// a 2^-e <= F, F = 1.75 * 2^8 (E4M3) or 1.75 * 2^15 (E5M2), held to [-127, 127]; 0 for a = 0.  Subnormal a have
// exponent field 0 and come out below -127.
template <int FORMAT>
__device__ __forceinline__ int scale_exponent(float a) {
  const uint32_t u = __float_as_uint(a);
  const int e = (int)(u >> 23) - 127 - (FORMAT == kE4m3 ? 8 : 15) + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return u == 0 ? 0 : max(e, -127);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }  // -126 <= e <= 127

// Two values to two codes (ties to even; NaN to the format's NaN), lo in the low byte.
template <int FORMAT>
__device__ __forceinline__ uint32_t encode_two(float lo, float hi) {
  uint16_t r;
  if (FORMAT == kE4m3) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
template <int FORMAT>
__device__ __forceinline__ uint2 encode_eight(const float (&v)[8], const float (&scale)[8]) {
  uint32_t p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = encode_two<FORMAT>(v[2 * i] * scale[2 * i], v[2 * i + 1] * scale[2 * i + 1]);
  return make_uint2(p[0] | p[1] << 16, p[2] | p[3] << 16);
}

// Byte of (row, block) in the scales of a matrix whose rows fill `atoms` groups of 128.
__device__ __forceinline__ uint64_t scale_offset(uint32_t row, uint32_t block, uint32_t atoms) {
  return ((uint64_t)(block >> 2) * atoms + (row >> 7)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}
// Writes the byte, and 127 for the blocks that pad the last word.
__device__ __forceinline__ void store_scale(uint8_t* scales, uint32_t row, uint32_t block, uint32_t blocks, uint32_t atoms, int e) {
  uint8_t* p = scales + scale_offset(row, block, atoms);
  st_c(p, (uint8_t)(e + 127));
  if (block + 1 == blocks)
    for (uint32_t b = block + 1; b & 3; ++b) st_c(++p, (uint8_t)127);
}

// Thread t holds columns 8 (t % 16) .. + 7 of rows 8 (t / 16) .. + 7 of the tile.
template <typename T, int FORMAT, bool WHOLE>
__global__ void __launch_bounds__(256) block_quantize_kernel(const BlockArgs a) {
  __shared__ __align__(16) uint8_t turned[kTile * kTile];
  __shared__ float column_most[8][kTile];
  __shared__ __align__(16) float column_scale[kTile];
  __shared__ float tile_most[8];
  grid_dependency_handshake();
  const uint32_t tile_r = blockIdx.x / a.tiles_c, tile_c = blockIdx.x % a.tiles_c;
  const uint32_t t = threadIdx.x, lane = t & 31, warp = t >> 5, part = t & 15;
  const uint32_t r0 = tile_r * kTile + 8 * (t >> 4), c0 = tile_c * kTile + 8 * part;

  float v[8][8];
  {
    Pack<T> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (WHOLE && r0 + i < a.rows && c0 + 8 <= a.cols) raw[i] = ld_pack(static_cast<const T*>(a.x) + (uint64_t)(r0 + i) * a.ld + c0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (WHOLE && r0 + i < a.rows && c0 + 8 <= a.cols) unpack(raw[i], v[i]);
      else ld_some(static_cast<const T*>(a.x) + (uint64_t)(r0 + i) * a.ld + c0, r0 + i < a.rows && c0 < a.cols ? (int)min(a.cols - c0, 8u) : 0, v[i]);
    }
  }

  float row_most[8], col_most[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    row_most[i] = fabsf(v[i][0]);
#pragma unroll
    for (int j = 1; j < 8; ++j) row_most[i] = max_nan(row_most[i], fabsf(v[i][j]));
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    col_most[j] = fabsf(v[0][j]);
#pragma unroll
    for (int i = 1; i < 8; ++i) col_most[j] = max_nan(col_most[j], fabsf(v[i][j]));
  }
  float most = row_most[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) most = max_nan(most, row_most[i]);
  const bool bad = !is_finite_bits(most);
  if (__syncthreads_or(bad)) {
    // rare: the scales are those of the finite values (fmaxf passes over NaN), infinities become NaN
    if (bad) atomicOr(a.status, kDevNonFinite);
    most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) row_most[i] = col_most[i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (!is_finite_bits(v[i][j])) v[i][j] = __uint_as_float(0x7fffffffu);
        const float m = fabsf(v[i][j]);
        row_most[i] = fmaxf(row_most[i], m);
        col_most[j] = fmaxf(col_most[j], m);
        most = fmaxf(most, m);
      }
  }

  int row_e[8];
  if (a.square) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
    if (lane == 0) tile_most[warp] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) most = fmaxf(most, tile_most[w]);
    const int e = scale_exponent<FORMAT>(most);
#pragma unroll
    for (int i = 0; i < 8; ++i) row_e[i] = e;
  } else if (a.q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int d = 8; d >= 1; d >>= 1) row_most[i] = fmaxf(row_most[i], __shfl_xor_sync(0xffffffffu, row_most[i], d));
      row_e[i] = scale_exponent<FORMAT>(row_most[i]);
    }
  }

  if (a.q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float inv = power_of_two(-row_e[i]);
      const float scale[8] = {inv, inv, inv, inv, inv, inv, inv, inv};
      if (r0 + i < a.rows && c0 < a.ldq)
        st_c(reinterpret_cast<uint2*>(a.q + (uint64_t)(r0 + i) * a.ldq + c0), encode_eight<FORMAT>(v[i], scale));
    }
    int mine = row_e[0];  // lane i of the first eight lanes of each half stores the scale of row i
#pragma unroll
    for (int i = 1; i < 8; ++i) mine = part == i ? row_e[i] : mine;
    if (part < 8) store_scale(a.scale, r0 + part, tile_c, a.tiles_c, a.tiles_r, r0 + part < a.rows ? mine : 0);
  }

  if (a.qt) {
    float scale[8];
    if (a.square) {
#pragma unroll
      for (int j = 0; j < 8; ++j) scale[j] = power_of_two(-row_e[0]);
      if (t < kTile) store_scale(a.scale_t, tile_c * kTile + t, tile_r, a.tiles_r, a.tiles_c, tile_c * kTile + t < a.cols ? row_e[0] : 0);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        col_most[j] = fmaxf(col_most[j], __shfl_xor_sync(0xffffffffu, col_most[j], 16));
        if (lane < 16) column_most[warp][8 * part + j] = col_most[j];
      }
      __syncthreads();
      if (t < kTile) {
        float m = column_most[0][t];
#pragma unroll
        for (int w = 1; w < 8; ++w) m = fmaxf(m, column_most[w][t]);
        const int e = scale_exponent<FORMAT>(m);
        column_scale[t] = power_of_two(-e);
        store_scale(a.scale_t, tile_c * kTile + t, tile_r, a.tiles_r, a.tiles_c, e);
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) scale[j] = column_scale[8 * part + j];
    }
    // Column c of the tile is 16 runs of eight bytes (the rows of one thread), run g at place g ^ (c / 8): the sixteen
    // threads that write one run of different columns meet sixteen different places.
    const uint32_t group = t >> 4;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float down[8], same[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) { down[i] = v[i][j]; same[i] = scale[j]; }
      *reinterpret_cast<uint2*>(turned + (8 * part + j) * kTile + 8 * (group ^ part)) = encode_eight<FORMAT>(down, same);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {  // eight threads a column, 16 bytes each
      const uint32_t c = (t >> 3) + 32 * k, u = t & 7, turn = c >> 3;
      uint4 w = *reinterpret_cast<const uint4*>(turned + c * kTile + 16 * (u ^ (turn >> 1)));
      if (turn & 1) w = make_uint4(w.z, w.w, w.x, w.y);
      const uint32_t row = tile_r * kTile + 16 * u;
      if (tile_c * kTile + c < a.cols && row < a.ldqt)
        st_c(reinterpret_cast<uint4*>(a.qt + (uint64_t)(tile_c * kTile + c) * a.ldqt + row), w);
    }
  }
}

}  // namespace accept
