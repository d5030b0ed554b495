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

// ---- eight rows of eight values, as they were read: words of two 16-bit values, or pairs of fp32 ----
template <typename T> struct Held { uint32_t w[8][4]; };
template <> struct Held<float> { Pair w[8][4]; };

template <typename T>
__device__ __forceinline__ Pair held_pair(const Held<T>& h, int i, int j) { return word_to_pair<T>(h.w[i][j]); }
__device__ __forceinline__ Pair held_pair(const Held<float>& h, int i, int j) { return h.w[i][j]; }

// Eight values at p, of which the first n exist (the others are zero).
template <typename T>
__device__ __forceinline__ void hold_row(Held<T>& h, int i, const T* p, bool whole, int n) {
  if (whole) {
    const Pack<T> raw = ld_pack(p);
    if constexpr (sizeof(T) == 4) {
      h.w[i][0] = pair_of(__uint_as_float(raw.w[0].x), __uint_as_float(raw.w[0].y));
      h.w[i][1] = pair_of(__uint_as_float(raw.w[0].z), __uint_as_float(raw.w[0].w));
      h.w[i][2] = pair_of(__uint_as_float(raw.w[1].x), __uint_as_float(raw.w[1].y));
      h.w[i][3] = pair_of(__uint_as_float(raw.w[1].z), __uint_as_float(raw.w[1].w));
    } else {
      h.w[i][0] = raw.w[0].x; h.w[i][1] = raw.w[0].y; h.w[i][2] = raw.w[0].z; h.w[i][3] = raw.w[0].w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      T lo = from_float<T>(0.0f), hi = lo;
      if (2 * j < n) lo = ld_c(p + 2 * j);
      if (2 * j + 1 < n) hi = ld_c(p + 2 * j + 1);
      if constexpr (sizeof(T) == 4) {
        h.w[i][j] = pair_of(lo, hi);
      } else {
        uint16_t a, b;
        memcpy(&a, &lo, 2);
        memcpy(&b, &hi, 2);
        h.w[i][j] = a | (uint32_t)b << 16;
      }
    }
  }
}

// The largest magnitude of each row and of each column; a NaN or an infinity comes out on top.
__device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b, __nv_bfloat16) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b, __half) {
  uint32_t r;
  asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <typename T>
__device__ __forceinline__ void largest(const Held<T>& h, float (&row)[8], float (&col)[8]) {
  uint32_t down[4];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    uint32_t across[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t m[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        m[j] = h.w[i + k][j] & 0x7fff7fffu;
        down[j] = i + k ? max_words(down[j], m[j], T()) : m[j];
      }
      across[k] = max_words(max_words(m[0], m[1], T()), max_words(m[2], m[3], T()), T());
    }
    // two rows in one word: even columns against odd ones
    const float2 f = split(word_to_pair<T>(max_words(__byte_perm(across[0], across[1], 0x5410), __byte_perm(across[0], across[1], 0x7632), T())));
    row[i] = f.x;
    row[i + 1] = f.y;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = split(word_to_pair<T>(down[j]));
    col[2 * j] = f.x;
    col[2 * j + 1] = f.y;
  }
}
__device__ __forceinline__ void largest(const Held<float>& h, float (&row)[8], float (&col)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = split(h.w[i][j]);
      const float x = fabsf(f.x), y = fabsf(f.y);
      row[i] = j ? max3_nan(row[i], x, y) : max_nan(x, y);
      if (i % 2) {
        const float2 g = split(h.w[i - 1][j]);
        col[2 * j] = i > 1 ? max3_nan(col[2 * j], x, fabsf(g.x)) : max_nan(x, fabsf(g.x));
        col[2 * j + 1] = i > 1 ? max3_nan(col[2 * j + 1], y, fabsf(g.y)) : max_nan(y, fabsf(g.y));
      }
    }
  }
}

// Rare: the scales are those of the finite values, and infinities become NaN.
template <typename T>
__device__ __forceinline__ void set_bad_aside(Held<T>& h, float (&row)[8], float (&col)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) row[i] = col[i] = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = split(held_pair(h, i, j));
      const bool x = is_finite_bits(f.x), y = is_finite_bits(f.y);
      if constexpr (sizeof(T) == 4) {
        h.w[i][j] = pair_of(x ? f.x : __uint_as_float(0x7fffffffu), y ? f.y : __uint_as_float(0x7fffffffu));
      } else {
        h.w[i][j] = (x ? h.w[i][j] & 0xffffu : 0x7fffu) | (y ? h.w[i][j] & 0xffff0000u : 0x7fff0000u);
      }
      const float a = x ? fabsf(f.x) : 0.0f, b = y ? fabsf(f.y) : 0.0f;
      row[i] = fmaxf(row[i], fmaxf(a, b));
      col[2 * j] = fmaxf(col[2 * j], a);
      col[2 * j + 1] = fmaxf(col[2 * j + 1], b);
    }
}

// Thread t holds columns 8 (t % 16) .. + 7 of rows 8 (t / 16) .. + 7 of the tile.
template <typename T, int FORMAT, bool WHOLE>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 3 : 2) block_quantize_kernel(const BlockArgs a) {
  __shared__ __align__(16) uint8_t turned[kTile * kTile];
  __shared__ __align__(16) float column_most[8][kTile];
  __shared__ __align__(16) float column_scale[kTile];
  __shared__ float tile_most[8];
  grid_dependency_handshake();
  const uint32_t tile_r = blockIdx.x / a.tiles_c, tile_c = blockIdx.x - tile_r * a.tiles_c;
  const uint32_t t = threadIdx.x, lane = t & 31, warp = t >> 5, part = t & 15;
  const uint32_t r0 = tile_r * kTile + 8 * (t >> 4), c0 = tile_c * kTile + 8 * part;

  Held<T> h;
  {
    const T* p = static_cast<const T*>(a.x) + (uint64_t)r0 * a.ld + c0;
    const int n = c0 < a.cols ? (int)min(a.cols - c0, 8u) : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool there = r0 + i < a.rows;
      hold_row(h, i, p, WHOLE && there && n == 8, there ? n : 0);
      p += a.ld;
    }
  }

  float row_most[8], col_most[8];
  largest(h, row_most, col_most);
  float most = row_most[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) most = max_nan(most, row_most[i]);
  const bool bad = !is_finite_bits(most);
  if (__syncthreads_or(bad)) {
    if (bad) atomicOr(a.status, kDevNonFinite);
    set_bad_aside(h, row_most, col_most);
    most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, row_most[i]);
  }

  int tile_e = 0;
  if (a.square) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
    if (lane == 0) tile_most[warp] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) most = fmaxf(most, tile_most[w]);
    tile_e = scale_exponent<FORMAT>(most);
  }

  if (a.q) {
    // sixteen lanes hold eight rows: each exchange halves the rows that a lane looks after, until two lanes have one
    float m[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float away = part & 8 ? row_most[k] : row_most[k + 4], keep = part & 8 ? row_most[k + 4] : row_most[k];
      m[k] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, away, 8));
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float away = part & 4 ? m[k] : m[k + 2], keep = part & 4 ? m[k + 2] : m[k];
      m[k] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, away, 4));
    }
    {
      const float away = part & 2 ? m[0] : m[1], keep = part & 2 ? m[1] : m[0];
      m[0] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, away, 2));
    }
    m[0] = fmaxf(m[0], __shfl_xor_sync(0xffffffffu, m[0], 1));
    const int e = a.square ? tile_e : scale_exponent<FORMAT>(m[0]);  // of row part / 2
    const uint32_t row = r0 + (part >> 1);
    if (!(part & 1)) store_scale(a.scale, row, tile_c, a.tiles_c, a.tiles_r, row < a.rows ? e : 0);
    const float inverse = power_of_two(-e);
    uint8_t* q = a.q + (uint64_t)r0 * a.ldq + c0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Pair scale = both(__shfl_sync(0xffffffffu, inverse, (lane & 16) | (2 * i)));
      uint32_t code[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = split(mul2(held_pair(h, i, j), scale));
        code[j] = encode_two<FORMAT>(f.x, f.y);
      }
      if (r0 + i < a.rows && c0 < a.ldq) st_c(reinterpret_cast<uint2*>(q), make_uint2(code[0] | code[1] << 16, code[2] | code[3] << 16));
      q += a.ldq;
    }
  }

  if (a.qt) {
    Pair scale[4];
    if (a.square) {
#pragma unroll
      for (int j = 0; j < 4; ++j) scale[j] = both(power_of_two(-tile_e));
      if (t < kTile) store_scale(a.scale_t, tile_c * kTile + t, tile_r, a.tiles_r, a.tiles_c, tile_c * kTile + t < a.cols ? tile_e : 0);
    } else {
      float m[4];  // of the lower or the upper four columns
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float away = lane & 16 ? col_most[k] : col_most[k + 4], keep = lane & 16 ? col_most[k + 4] : col_most[k];
        m[k] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, away, 16));
      }
      *reinterpret_cast<float4*>(&column_most[warp][8 * part + (lane & 16 ? 4 : 0)]) = make_float4(m[0], m[1], m[2], m[3]);
      __syncthreads();
      if (t < kTile) {
        float c = column_most[0][t];
#pragma unroll
        for (int w = 1; w < 8; ++w) c = fmaxf(c, column_most[w][t]);
        const int e = scale_exponent<FORMAT>(c);
        column_scale[t] = power_of_two(-e);
        store_scale(a.scale_t, tile_c * kTile + t, tile_r, a.tiles_r, a.tiles_c, e);
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = *reinterpret_cast<const float2*>(column_scale + 8 * part + 2 * j);
        scale[j] = pair_of(f.x, f.y);
      }
    }
    // Column c of the tile is 16 runs of eight bytes (the rows of one thread), run g at place g ^ (c / 8): the sixteen
    // threads that write one run of different columns meet sixteen different places.
    uint8_t* run = turned + 8 * part * kTile + 8 * ((t >> 4) ^ part);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t left[4], right[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = split(mul2(held_pair(h, 2 * i, j), scale[j])), g = split(mul2(held_pair(h, 2 * i + 1, j), scale[j]));
        left[i] = encode_two<FORMAT>(f.x, g.x);
        right[i] = encode_two<FORMAT>(f.y, g.y);
      }
      *reinterpret_cast<uint2*>(run + 2 * j * kTile) = make_uint2(left[0] | left[1] << 16, left[2] | left[3] << 16);
      *reinterpret_cast<uint2*>(run + (2 * j + 1) * kTile) = make_uint2(right[0] | right[1] << 16, right[2] | right[3] << 16);
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
