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
// One value (|v| <= 6, v25 = v 2^25) to a code with stochastic rounding, in exact fixed point: F = the value's place in the list of
// codes times 2^24, rounded up, so that F + 2^24 - 1 - r carries into the next place where r 2^-24 is below the value's share of the
// step.  From 1 on the list is that of fp32's own upper bits; below, steps are 0.5.  `less`: the upper 28 bits of the random word's
// complement, 2^24 - 1 - r over four bits that change nothing beside a multiple of 16.  The code is in the top four bits, its sign
// first.  Additions run as multiply-adds beside the logic instructions, which bound this.
__device__ __forceinline__ uint32_t micro_stochastic(float v, float v25, uint32_t less) {
  uint32_t r;
  asm("{\n\t.reg .pred p;\n\t.reg .f32 s, t;\n\t.reg .b32 f;\n\t"
      "abs.f32 s, %1;\n\t"
      "setp.ge.f32 p, s, 0f3F800000;\n\t"
      "abs.f32 t, %2;\n\t"
      "cvt.rpi.u32.f32 f, t;\n\t"
      "@p mad.lo.u32 f, %4, 4, %5;\n\t"
      "mad.lo.u32 f, f, 16, %3;\n\t"
      "lop3.b32 %0, f, %4, 0x80000000, 0xF8;\n\t}"  // f | (v & sign)
      : "=r"(r) : "f"(v), "f"(v25), "r"(less), "r"(__float_as_uint(v)), "r"((2u << 24) - (0x3f800000u << 2)));
  return r;
}
// Eight codes from the top four bits of words, the first in the lowest bits.
__device__ __forceinline__ uint32_t micro_join(const uint32_t (&w)[8]) {
  uint32_t r = w[7] >> 28;
#pragma unroll
  for (int i = 6; i >= 0; --i) r = __funnelshift_l(w[i], r, 4);
  return r;
}

// Thread (warp w, lane l) holds columns 64 (w % 2) + 8 (l % 8) .. + 7 of rows 32 (w / 2) + 8 (l / 8) .. + 7 of the tile: a warp has 32 rows
// of two blocks of columns, so the largest values of all blocks, both ways, are found within it.
//
// Measured on 16384 x 4096 bf16, nearest: see the launch.  Stochastic rounding is bound by instruction issue: some 30 a value for
// both outputs.
// ROUND: nearest, or stochastic where all rows' counters start on a multiple of four (kQuads) or not (kAnywhere).
enum class MicroRound { kNearest, kQuads, kAnywhere };
template <typename T, MicroRound ROUND, bool WHOLE>
__global__ void __launch_bounds__(256, ROUND != MicroRound::kNearest || sizeof(T) == 4 ? 2 : 3) micro_quantize_kernel(const MicroArgs a) {
  constexpr bool STOCHASTIC = ROUND != MicroRound::kNearest;
  __shared__ __align__(16) uint8_t turned[kTile * (kTile / 2)];
  __shared__ __align__(16) uint8_t bytes_t[kTile][4];
  constexpr bool kKept = sizeof(T) == 2;  // the numbers of all values stay in registers; beside fp32 values they are drawn twice
  grid_dependency_handshake();
  const uint32_t tile_r = blockIdx.x / a.tiles_c, tile_c = blockIdx.x - tile_r * a.tiles_c;
  const uint32_t t = threadIdx.x, lane = t & 31, warp = t >> 5, part = lane & 7, down = lane >> 3;
  const uint32_t r_in = 32 * (warp >> 1) + 8 * down, c_in = 64 * (warp & 1) + 8 * part;
  const uint32_t r0 = tile_r * kTile + r_in, c0 = tile_c * kTile + c_in;

  Held<T> h;
  {
    const T* p = static_cast<const T*>(a.x) + (uint64_t)r0 * a.ld + c0;
    const int n = c0 < a.cols ? (int)min(a.cols - c0, 8u) : 0;
    if (!WHOLE && sizeof(T) == 2 && n == 8 && (r0 > 0 || c0 > 0) && (r0 + 8 < a.rows || (r0 + 8 == a.rows && c0 + 8 < a.cols))) {
      RawEight<T> raw[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) load_raw<T>(p + i * a.ld, raw[i]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t w[2 * sizeof(T)];
        words_of<T>(raw[i], p + i * a.ld, w);
#pragma unroll
        for (int j = 0; j < 4; ++j) h.w[i][j] = w[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool there = r0 + i < a.rows;
        hold_row(h, i, p, WHOLE && there && n == 8, there ? n : 0);
        p += a.ld;
      }
    }
  }
  float row_most[8], col_most[8];
  largest(h, row_most, col_most);  // a NaN or an infinity comes out on top
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) bad |= !is_finite_bits(row_most[i]);
  if (bad) atomicOr(a.status, kDevNonFinite);

  uint32_t square_byte = 0;  // of the 32 x 32 block that this thread's values lie in
  if (a.square) {
    float most = row_most[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) most = max_nan(most, row_most[i]);
#pragma unroll
    for (int d = 1; d <= 16; d <<= 1)
      if (d != 4) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, d));
    square_byte = micro_scale_byte(most);
  }

  const uint64_t first = a.offset + (uint64_t)r0 * a.cols + c0;
  const DropKey key(a.rng, first);
  DropRow quads(a.rng, first, key);
  if (ROUND == MicroRound::kQuads) quads.phase = 0;  // known here: the other way of counting falls away
  const auto draw_row = [&](int i, uint32_t (&less)[8]) {
    const auto keep = [&](int, const uint32_t (&w)[8]) {
#pragma unroll
      for (int j = 0; j < 8; ++j) less[j] = w[j] >> 4;
    };
    if (ROUND == MicroRound::kQuads) number_units<8, true, 1>(quads, i * (a.cols & ~3u), 0, keep);
    else number_units<8, true, 1>(DropRow(a.rng, first + (uint64_t)i * a.cols, key), 0, 0, keep);
  };
  uint32_t numbers[STOCHASTIC && kKept ? 8 : 1][8];
  if (STOCHASTIC && kKept)
#pragma unroll
    for (int i = 0; i < 8; ++i) draw_row(i, numbers[i % (STOCHASTIC && kKept ? 8 : 1)]);

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
    float inverse[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {  // rows 2 (part % 4) + k of the eight
      const uint32_t row = r0 + 2 * (part & 3) + k;
      uint32_t byte = a.square ? square_byte : micro_scale_byte(m[k]);
      inverse[k] = micro_inverse(byte);
      if (row >= a.rows || (c0 & ~31u) >= a.cols) byte = 127u;  // rows and blocks that do not exist, beside a square block that ends inside
      const uint32_t next = __shfl_xor_sync(0xffffffffu, byte, 4);
      if (part < 4) st_c(reinterpret_cast<uint16_t*>(a.scale + scale_offset(row, 4 * tile_c + 2 * (warp & 1), a.tiles_r)), (uint16_t)(byte | next << 8));
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
      if constexpr (STOCHASTIC) {
        uint32_t w[8], drawn[8];
        if (!kKept) draw_row(i, drawn);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = split(mul2(pair_of(v[2 * j], v[2 * j + 1]), both(0x1p+25f)));
          w[2 * j] = micro_stochastic(v[2 * j], f.x, kKept ? numbers[i % (kKept ? 8 : 1)][2 * j] : drawn[2 * j]);
          w[2 * j + 1] = micro_stochastic(v[2 * j + 1], f.y, kKept ? numbers[i % (kKept ? 8 : 1)][2 * j + 1] : drawn[2 * j + 1]);
        }
        code = micro_join(w);
      } else {
        code = micro_encode(v);
      }
      if (r0 + i < a.rows && c0 / 2 < a.ldq) st_c(reinterpret_cast<uint32_t*>(q), s == 0.0f ? 0u : code);
      q += a.ldq;
    }
  }

  if (a.qt) {
    // four lanes hold eight columns of a block, 32 rows: as above
    float m[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float away = lane & 16 ? col_most[k] : col_most[k + 4], keep = lane & 16 ? col_most[k + 4] : col_most[k];
      m[k] = max_nan(keep, __shfl_xor_sync(0xffffffffu, away, 16));
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float away = lane & 8 ? m[k] : m[k + 2], keep = lane & 8 ? m[k + 2] : m[k];
      m[k] = max_nan(keep, __shfl_xor_sync(0xffffffffu, away, 8));
    }
    float inverse[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {  // columns 2 down + k of the eight
      uint32_t byte = a.square ? square_byte : micro_scale_byte(m[k]);
      inverse[k] = micro_inverse(byte);
      if (c0 + 2 * down + k >= a.cols || (r0 & ~31u) >= a.rows) byte = 127u;
      bytes_t[c_in + 2 * down + k][warp >> 1] = (uint8_t)byte;
    }
    // Column c of the tile is 16 words (eight rows each), those of 32 rows side by side, u-th four at place u ^ (c / 8 % 4): the lanes
    // that write the words of different columns meet different places.
    uint8_t* word = turned + c_in * (kTile / 2) + 16 * ((warp >> 1) ^ (part & 3)) + 4 * down;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float s0 = __shfl_sync(0xffffffffu, inverse[0], part | j << 3), s1 = __shfl_sync(0xffffffffu, inverse[1], part | j << 3);
      const Pair scale = pair_of(s0, s1);
      float left[8], right[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 f = split(mul2(held_pair(h, i, j), scale));
        left[i] = f.x;
        right[i] = f.y;
      }
      uint32_t code[2];
      if constexpr (STOCHASTIC) {
        uint32_t w[2][8], drawn[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (!kKept) draw_row(i, drawn);  // what this pair of columns does not need falls away
          const float2 f = split(mul2(pair_of(left[i], right[i]), both(0x1p+25f)));
          w[0][i] = micro_stochastic(left[i], f.x, kKept ? numbers[i % (kKept ? 8 : 1)][2 * j] : drawn[2 * j]);
          w[1][i] = micro_stochastic(right[i], f.y, kKept ? numbers[i % (kKept ? 8 : 1)][2 * j + 1] : drawn[2 * j + 1]);
        }
        code[0] = micro_join(w[0]);
        code[1] = micro_join(w[1]);
      } else {
        code[0] = micro_encode(left);
        code[1] = micro_encode(right);
      }
      *reinterpret_cast<uint32_t*>(word + 2 * j * (kTile / 2)) = s0 == 0.0f ? 0u : code[0];
      *reinterpret_cast<uint32_t*>(word + (2 * j + 1) * (kTile / 2)) = s1 == 0.0f ? 0u : code[1];
    }
    __syncthreads();
    if (t < kTile)
      st_c(reinterpret_cast<uint32_t*>(a.scale_t + scale_offset(tile_c * kTile + t, 4 * tile_r, a.tiles_c)), *reinterpret_cast<const uint32_t*>(bytes_t[t]));
#pragma unroll
    for (int k = 0; k < 2; ++k) {  // four threads a column, 16 bytes each
      const uint32_t c = (t >> 2) + 64 * k, u = t & 3;
      const uint4 w = *reinterpret_cast<const uint4*>(turned + c * (kTile / 2) + 16 * (u ^ (c >> 3 & 3)));
      const uint32_t byte = tile_r * (kTile / 2) + 16 * u;
      if (tile_c * kTile + c < a.cols && byte < a.ldqt) st_c(reinterpret_cast<uint4*>(a.qt + (uint64_t)(tile_c * kTile + c) * a.ldqt + byte), w);
    }
  }
}

// ---- decoding ----

struct MicroValueArgs {
  const uint8_t* q;
  const uint8_t* scale;
  void* x;
  uint64_t ld;
  uint32_t rows, cols, ldq, atoms;
  int log_units;  // see micro_dequantize_kernel
};

// Eight codes as fp32 pairs.  As fp32 bits a code's two exponent and one fraction bits are its value times 2^-126 (the smallest,
// 0.5, a subnormal), so one exact product gives the value and another one applies the scale (of the pair's first and second).
__device__ __forceinline__ Pair micro_value(uint32_t codes, int j, Pair scale) {
  const uint32_t lo = codes >> 8 * j, hi = codes >> (8 * j + 4);
  const Pair raw = pair_of(__uint_as_float((lo << 28 & 0x80000000u) | (lo << 22 & 0x01c00000u)),
                           __uint_as_float((hi << 28 & 0x80000000u) | (hi << 22 & 0x01c00000u)));
  return mul2(mul2(raw, both(0x1p+126f)), scale);
}
__device__ __forceinline__ float micro_scale(uint32_t byte) { return __uint_as_float(byte == 255u ? 0x7fffffffu : byte ? byte << 23 : 1u << 22); }

// A unit is eight neighbours of a row that start on a 16-byte boundary of x.  Where rows do not (WHOLE false), a unit's codes are
// shifted out of two words and may have two scales; the ends of a row are written value by value.  (One value a store:
// 4096 x 1001 fp32 27.7 us.)  A block takes 2^log_units units of ROWS times as many rows as that leaves threads for, in turn.
constexpr int kValueThreads = 256;
template <typename T, bool WHOLE, int ROWS>
__global__ void __launch_bounds__(kValueThreads) micro_dequantize_kernel(const MicroValueArgs a) {
  grid_dependency_handshake();
  constexpr uint32_t kEach = 16 / (uint32_t)sizeof(T);
  const uint32_t at_once = kValueThreads >> a.log_units, c = ((blockIdx.x << a.log_units) + (threadIdx.x & ((1u << a.log_units) - 1))) * 8;
  const uint32_t groups = (a.rows + at_once * ROWS - 1) / (at_once * ROWS);
  for (uint32_t group = blockIdx.y; group < groups; group += gridDim.y) {
    const uint32_t r0 = group * (at_once * ROWS) + (threadIdx.x >> a.log_units);
    uint32_t codes[ROWS], byte[ROWS], next[ROWS];
    int col[ROWS];  // of a unit: its first column, below 0 where the row starts inside it
    bool some[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const uint32_t row = r0 + i * at_once;
      uint32_t before = 0;  // values between the 16-byte boundary and the row's start
      if (!WHOLE) before = (uint32_t)((reinterpret_cast<uintptr_t>(a.x) / sizeof(T) + row * a.ld) % kEach);
      col[i] = (int)(c - before);
      some[i] = row < a.rows && row >= r0 && c < a.cols + before;
      codes[i] = byte[i] = next[i] = 0;
      if (!some[i]) continue;
      const uint32_t* q = reinterpret_cast<const uint32_t*>(a.q + (uint64_t)row * a.ldq);
      const uint32_t start = WHOLE ? c : col[i] < 0 ? 0u : (uint32_t)col[i];
      codes[i] = ldg_c(q + start / 8);
      byte[i] = next[i] = ldg_c(a.scale + scale_offset(row, start / 32, a.atoms));
      if (!WHOLE) {
        const uint32_t end = min((uint32_t)(col[i] + 7), a.cols - 1);
        uint32_t more = codes[i];
        if (end / 8 != start / 8) more = ldg_c(q + end / 8);
        if (end / 32 != start / 32) next[i] = ldg_c(a.scale + scale_offset(row, end / 32, a.atoms));
        codes[i] = col[i] < 0 ? codes[i] << 4 * (uint32_t)-col[i] : __funnelshift_r(codes[i], more, 4 * (start % 8));
      }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      if (!some[i]) continue;
      Pair v[4];
      const float s = micro_scale(byte[i]), s2 = WHOLE ? s : micro_scale(next[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int lo = (col[i] + 2 * j) & 31, hi = (col[i] + 2 * j + 1) & 31;  // the second scale from the first boundary on
        const bool second_lo = !WHOLE && col[i] >= 0 && lo < (col[i] & 31), second_hi = !WHOLE && col[i] >= 0 && hi < (col[i] & 31);
        v[j] = micro_value(codes[i], j, pair_of(second_lo ? s2 : s, second_hi ? s2 : s));
      }
      T* x = static_cast<T*>(a.x) + (uint64_t)(r0 + i * at_once) * a.ld;
      if (WHOLE || (col[i] >= 0 && (uint32_t)col[i] + 8 <= a.cols)) {
        store_eight<T, true>(x + col[i], WHOLE ? (int)min(a.cols - (uint32_t)col[i], 8u) : 8, v);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 f = split(v[j / 2]);
          const int at = col[i] + j;
          if (at >= 0 && (uint32_t)at < a.cols) st_c(x + at, from_float<T>(j % 2 ? f.y : f.x));
        }
      }
    }
  }
}

}  // namespace accept
