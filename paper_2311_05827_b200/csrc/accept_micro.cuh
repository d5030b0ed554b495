// 4-bit floating point (E2M1) with one power-of-two scale for each 32 values: coding and decoding (sm_100a).
//
// Bound by memory.  Coding: one block of threads takes a tile of 128 x 128 values, read once and held in registers, and codes it
// along its rows, along its columns (through shared memory), or both; such a tile's scales are one group of 512 bytes.
#pragma once
#include "accept_block.cuh"
#include "accept_drop.cuh"
#include "accept_dropout.cuh"

namespace accept {

struct MicroArgs {
  const void* x;
  uint8_t* q;        // rows, may be null
  uint8_t* scale;
  uint8_t* qt;       // columns, may be null
  uint8_t* scale_t;
  uint32_t* status;
  uint64_t ld;
  uint64_t offset;   // counter of element 0
  Rng rng;
  uint32_t rows, cols;
  uint32_t ldq, ldqt;         // bytes between coded rows
  uint32_t tiles_r, tiles_c;  // tiles over the rows and the columns
  int square;
};

// Scale byte from the bits of a block's largest magnitude a: e + 127, e the least integer with a 2^-e <= 6 = 1.5 * 2^2 (subnormal a
// have exponent field 0 and come out below -127); 127 for a = 0, 255 for a NaN or an infinity.
__device__ __forceinline__ uint32_t micro_scale_byte(float a) {
  const uint32_t u = __float_as_uint(a);
  const int e = (int)(u >> 23) - 2 + ((u & 0x7fffffu) > 0x400000u ? 1 : 0);
  return u == 0 ? 127u : u >= 0x7f800000u ? 255u : (uint32_t)max(e, 0);
}
// 2^(127 - byte); 0 for 255, which makes every code of the block zero.
__device__ __forceinline__ float micro_inverse(uint32_t byte) { return __uint_as_float(byte == 255u ? 0u : (254u - byte) << 23); }

// Eight values to eight codes, the first in the lowest bits; ties to even.
__device__ __forceinline__ uint32_t micro_encode(const float (&v)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
// One value (|v| <= 6) with stochastic rounding, in exact fixed point: F = the value's place in the list of codes times 2^24,
// rounded up, so that (F + 2^24 - 1 - r) >> 24 is the upper neighbour where r 2^-24 is below the value's share of the step.  From
// 1 on the list is that of fp32's own upper bits; below, steps are 0.5.  `less`: 2^24 - 1 - r.  The code is in the top four
// bits, its sign above it.
__device__ __forceinline__ uint32_t micro_stochastic(float v, uint32_t less) {
  const float size = fabsf(v);
  const uint32_t f = size < 1.0f ? __float2uint_ru(__fmul_rn(size, 0x1p+25f)) : (__float_as_uint(size) << 2) - ((0x3f800000u << 2) - (2u << 24));
  return ((f + less) << 4) | (__float_as_uint(v) & 0x80000000u);
}
// Eight such results to eight codes (each in its top four bits).
__device__ __forceinline__ uint32_t micro_pack(const uint32_t (&w)[8]) {
  uint32_t r = w[7] & 0xf0000000u;
#pragma unroll
  for (int i = 0; i < 7; ++i) r |= (w[i] >> 28) << 4 * i;
  return r;
}

// What a thread's 8 x 8 values need of the generator: word e of row i as `less` above.
struct MicroNumbers {
  uint32_t less[8][8];
};

// Thread t holds columns 8 (t % 16) .. + 7 of rows 8 (t / 16) .. + 7 of the tile.
template <typename T, bool STOCHASTIC, bool WHOLE>
__global__ void __launch_bounds__(256, 2) micro_quantize_kernel(const MicroArgs a) {
  __shared__ __align__(16) uint8_t turned[kTile * (kTile / 2)];
  __shared__ __align__(16) float column_most[8][kTile];
  __shared__ __align__(16) float column_scale[4][kTile];
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
  largest(h, row_most, col_most);  // a NaN or an infinity comes out on top
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) bad |= !is_finite_bits(row_most[i]);
  if (bad) atomicOr(a.status, kDevNonFinite);

  MicroNumbers numbers;
  if (STOCHASTIC) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const DropRow row(a.rng, a.offset + (uint64_t)(r0 + i) * a.cols + c0, 8);
      uint32_t w[8];
      number_unit<8>(a.rng, row, 0, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) numbers.less[i][j] = ~w[j] >> 8;
    }
  }

  uint32_t square_byte = 0;  // of the 32 x 32 block that this thread's values lie in
  if (a.square) {
    float most = row_most[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) most = max_nan(most, row_most[i]);
#pragma unroll
    for (int d = 1; d <= 2; d <<= 1) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, d));
    most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, 16));
    if (lane < 16 && !(lane & 3)) column_most[warp][lane >> 2] = most;
    __syncthreads();
    most = max_nan(column_most[warp & ~1u][part >> 2], column_most[warp | 1u][part >> 2]);
    square_byte = micro_scale_byte(most);
    __syncthreads();
  }

  if (a.q) {
    // four lanes hold eight rows of a block: each exchange halves the rows that a lane looks after, until it has two
    float m[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float away = part & 2 ? row_most[k] : row_most[k + 4], keep = part & 2 ? row_most[k + 4] : row_most[k];
      m[k] = max_nan(keep, __shfl_xor_sync(0xffffffffu, away, 2));
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float away = part & 1 ? m[k] : m[k + 2], keep = part & 1 ? m[k + 2] : m[k];
      m[k] = max_nan(keep, __shfl_xor_sync(0xffffffffu, away, 1));
    }
    uint32_t byte[2];
    float inverse[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {  // rows 2 (part % 4) + k of the eight
      byte[k] = a.square ? square_byte : micro_scale_byte(m[k]);
      inverse[k] = micro_inverse(byte[k]);
      // rows and blocks that do not exist hold zeros: 127 from micro_scale_byte, also beside a square block that ends inside
      const bool there = r0 + 2 * (part & 3) + k < a.rows && (c0 & ~31u) < a.cols;
      uint32_t word = (there ? byte[k] : 127u) << 8 * (part >> 2);
      word |= __shfl_xor_sync(0xffffffffu, word, 4);
      word |= __shfl_xor_sync(0xffffffffu, word, 8);
      const uint32_t row = r0 + 2 * (part & 3) + k;
      if (part < 4) st_c(reinterpret_cast<uint32_t*>(a.scale + scale_offset(row, 4 * tile_c, a.tiles_r)), word);
    }
    uint8_t* q = a.q + (uint64_t)r0 * a.ldq + c0 / 2;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float s = __shfl_sync(0xffffffffu, inverse[i & 1], (lane & ~3u) | (i >> 1));
      float v[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = split(mul2(held_pair(h, i, j), both(s)));
        v[2 * j] = f.x;
        v[2 * j + 1] = f.y;
      }
      uint32_t code;
      if (STOCHASTIC) {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = micro_stochastic(v[j], numbers.less[i][j]);
        code = micro_pack(w);
      } else {
        code = micro_encode(v);
      }
      if (r0 + i < a.rows && c0 / 2 < a.ldq) st_c(reinterpret_cast<uint32_t*>(q), s == 0.0f ? 0u : code);
      q += a.ldq;
    }
  }

  if (a.qt) {
    // the largest of 32 rows: four threads down, in two warps
    if (!a.square) {
      float m[4];  // of the lower or the upper four columns
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float away = lane & 16 ? col_most[k] : col_most[k + 4], keep = lane & 16 ? col_most[k + 4] : col_most[k];
        m[k] = max_nan(keep, __shfl_xor_sync(0xffffffffu, away, 16));
      }
      *reinterpret_cast<float4*>(&column_most[warp][8 * part + (lane & 16 ? 4 : 0)]) = make_float4(m[0], m[1], m[2], m[3]);
    } else if (lane < 16) {
#pragma unroll
      for (int k = 0; k < 8; ++k) column_most[warp][8 * part + k] = __uint_as_float(square_byte);
    }
    __syncthreads();
    if (t < kTile) {
      uint32_t word = 0;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float lower = column_most[2 * g][t], upper = column_most[2 * g + 1][t];
        uint32_t byte = a.square ? __float_as_uint(lower) : micro_scale_byte(max_nan(lower, upper));
        column_scale[g][t] = micro_inverse(byte);
        if (tile_c * kTile + t >= a.cols || tile_r * kTile + 32 * g >= a.rows) byte = 127u;
        word |= byte << 8 * g;
      }
      st_c(reinterpret_cast<uint32_t*>(a.scale_t + scale_offset(tile_c * kTile + t, 4 * tile_r, a.tiles_c)), word);
    }
    __syncthreads();
    const float4 lo = *reinterpret_cast<const float4*>(&column_scale[warp >> 1][8 * part]), hi = *reinterpret_cast<const float4*>(&column_scale[warp >> 1][8 * part + 4]);
    const float scale[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    // Column c of the tile is 16 words (the eight rows of one thread each), word g at place g ^ (c / 8): the sixteen threads that
    // write one word of different columns meet sixteen different places.
    uint8_t* word = turned + 8 * part * (kTile / 2) + 4 * ((t >> 4) ^ part);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 f = split(held_pair(h, i, j / 2));
        v[i] = __fmul_rn(j % 2 ? f.y : f.x, scale[j]);
      }
      uint32_t code;
      if (STOCHASTIC) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = micro_stochastic(v[i], numbers.less[i][j]);
        code = micro_pack(w);
      } else {
        code = micro_encode(v);
      }
      *reinterpret_cast<uint32_t*>(word + j * (kTile / 2)) = scale[j] == 0.0f ? 0u : code;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {  // four threads a column, 16 bytes each
      const uint32_t c = (t >> 2) + 64 * k, u = t & 3, turn = c >> 3;
      const uint4 w = *reinterpret_cast<const uint4*>(turned + c * (kTile / 2) + 16 * (u ^ (turn >> 2)));
      const uint32_t in[4] = {w.x, w.y, w.z, w.w};
      uint32_t out[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) out[i] = (turn & 1 ? (turn & 2 ? in[i ^ 3] : in[i ^ 1]) : (turn & 2 ? in[i ^ 2] : in[i]));
      const uint32_t byte = tile_r * (kTile / 2) + 16 * u;
      if (tile_c * kTile + c < a.cols && byte < a.ldqt)
        st_c(reinterpret_cast<uint4*>(a.qt + (uint64_t)(tile_c * kTile + c) * a.ldqt + byte), make_uint4(out[0], out[1], out[2], out[3]));
    }
  }
}

// ---- decoding ----

struct MicroValueArgs {
  const uint8_t* q;
  const uint8_t* scale;
  void* x;
  uint64_t ld, per_row, units;  // units of eight neighbours
  uint32_t cols, ldq, atoms;
};

// Eight codes as fp32 pairs.  As fp32 bits a code's two exponent and one fraction bits are its value
// times 2^-126 (the smallest, 0.5, a subnormal), so one exact product gives the value and another one applies the scale.
__device__ __forceinline__ void micro_decode(uint32_t codes, float scale, Pair (&v)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t lo = codes >> 8 * j, hi = codes >> (8 * j + 4);
    const Pair raw = pair_of(__uint_as_float((lo << 28 & 0x80000000u) | (lo << 22 & 0x01c00000u)),
                             __uint_as_float((hi << 28 & 0x80000000u) | (hi << 22 & 0x01c00000u)));
    v[j] = mul2(mul2(raw, both(0x1p+126f)), both(scale));
  }
}

constexpr int kValueThreads = 256;
template <typename T, bool VEC, int UNITS>
__global__ void __launch_bounds__(kValueThreads) micro_dequantize_kernel(const MicroValueArgs a) {
  grid_dependency_handshake();
  const uint64_t first = (uint64_t)blockIdx.x * (UNITS * kValueThreads) + threadIdx.x;
  uint32_t codes[UNITS], byte[UNITS], row[UNITS], col[UNITS];
  int n[UNITS];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const uint64_t u = first + i * kValueThreads;
    row[i] = a.units <= 0xffffffffu ? (uint32_t)u / (uint32_t)a.per_row : (uint32_t)(u / a.per_row);
    col[i] = (uint32_t)(u - row[i] * a.per_row) * 8;
    n[i] = u < a.units ? (int)min(a.cols - col[i], 8u) : 0;
    if (n[i] == 0) continue;
    codes[i] = ldg_c(reinterpret_cast<const uint32_t*>(a.q + (uint64_t)row[i] * a.ldq + col[i] / 2));
    byte[i] = ldg_c(a.scale + scale_offset(row[i], col[i] / 32, a.atoms));
  }
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    if (n[i] == 0) continue;
    Pair v[4];
    micro_decode(codes[i], __uint_as_float(byte[i] == 255u ? 0x7fffffffu : byte[i] ? byte[i] << 23 : 1u << 22), v);
    store_eight<T, VEC>(static_cast<T*>(a.x) + (uint64_t)row[i] * a.ld + col[i], n[i], v);
  }
}

}  // namespace accept
