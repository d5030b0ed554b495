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

// N values (4 or 8) to codes, the first in the lowest bits; ties to even.
template <int N>
__device__ __forceinline__ uint32_t micro_encode(const float (&v)[N]) {
  uint32_t r;
  if constexpr (N == 8) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  } else {
    asm("{\n\t.reg .b8 a, b;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "mov.b32 %0, {a, b, a, b};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]));
    r &= 0xffffu;
  }
  return r;
}
// One value (|v| <= 6, v25 = v 2^25; a value 2^-150 of its block's scale and less has come out as v = 0) to a code with stochastic rounding, in
// exact fixed point: F = the value's place in the list of
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
// N codes from the top four bits of words, the first in the lowest bits.
template <int N>
__device__ __forceinline__ uint32_t micro_join(const uint32_t (&w)[N]) {
  uint32_t r = w[N - 1] >> 28;
#pragma unroll
  for (int i = N - 2; i >= 0; --i) r = __funnelshift_l(w[i], r, 4);
  return r;
}

// The largest magnitude of each of the first ROWS rows, and of each column over them; a NaN or an infinity comes out on top.
template <int ROWS, typename T>
__device__ __forceinline__ void micro_largest(const Held<T>& h, float (&row)[ROWS], float (&col)[8]) {
  uint32_t down[4];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    uint32_t m[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = h.w[i][j] & 0x7fff7fffu;
      down[j] = i ? max_words(down[j], m[j], T()) : m[j];
    }
    const float2 f = split(word_to_pair<T>(max_words(max_words(m[0], m[1], T()), max_words(m[2], m[3], T()), T())));
    row[i] = max_nan(f.x, f.y);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = split(word_to_pair<T>(down[j]));
    col[2 * j] = f.x;
    col[2 * j + 1] = f.y;
  }
}
template <int ROWS>
__device__ __forceinline__ void micro_largest(const Held<float>& h, float (&row)[ROWS], float (&col)[8]) {
#pragma unroll
  for (int i = 0; i < ROWS; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = split(h.w[i][j]);
      const float x = fabsf(f.x), y = fabsf(f.y);
      row[i] = j ? max3_nan(row[i], x, y) : max_nan(x, y);
      col[2 * j] = i ? max_nan(col[2 * j], x) : x;
      col[2 * j + 1] = i ? max_nan(col[2 * j + 1], y) : y;
    }
}

// Each exchange over lane bit BIT halves the values that a lane looks after: N of them to N / 2, the upper half where the bit is set.
template <int N>
__device__ __forceinline__ void halve_most(const float (&m)[N], bool upper, int bit, float (&out)[N / 2]) {
#pragma unroll
  for (int k = 0; k < N / 2; ++k) {
    const float away = upper ? m[k] : m[k + N / 2], keep = upper ? m[k + N / 2] : m[k];
    out[k] = max_nan(keep, __shfl_xor_sync(0xffffffffu, away, bit));
  }
}

// ROUND: nearest, or stochastic where all rows' counters start on a multiple of four (kQuads) or not (kAnywhere).
enum class MicroRound { kNearest, kQuads, kAnywhere };

// A tile is 8 or 16 warps of 32 rows by 64 or 32 columns, a thread has ROWS rows of eight neighbours.  A warp has whole blocks both ways,
// so their largest values are found within it.  Eight rows; four for stochastic rounding of fp32, whose values and random numbers would
// else not fit the registers (16384 x 4096 both ways 151 -> 138 us; no gain for bf16, 97 us).
// Measured on 16384 x 4096 bf16: rows 28.5 us (0.91 of the copy rate), both ways 41 (0.77); stochastic rounding takes
// 35 instructions a value both ways, 97 us: logic pipe 68 %, issue slots 67 % busy with a quarter of the warps that an SM could hold.
template <typename T, MicroRound ROUND> constexpr int kMicroRows = ROUND != MicroRound::kNearest && sizeof(T) == 4 ? 4 : 8;
template <typename T, MicroRound ROUND> constexpr int kMicroThreads = kTile * kTile / 8 / kMicroRows<T, ROUND>;
template <typename T, MicroRound ROUND, bool WHOLE>
__global__ void __launch_bounds__(kMicroThreads<T, ROUND>, kMicroRows<T, ROUND> == 4 ? 1 : ROUND != MicroRound::kNearest || sizeof(T) == 4 ? 2 : 3)
    micro_quantize_kernel(const MicroArgs a) {
  constexpr bool STOCHASTIC = ROUND != MicroRound::kNearest;
  constexpr int ROWS = kMicroRows<T, ROUND>, kAcross = ROWS, kDown = 32 / kAcross;  // lanes side by side, and one below the other
  constexpr int kRowsEach = ROWS / 4, kColsEach = 8 / kDown;                        // that a lane looks after in the end
  constexpr int kWarpsAcross = kTile / (8 * kAcross);
  __shared__ __align__(16) uint8_t turned[kTile * (kTile / 2)];
  __shared__ __align__(16) uint8_t bytes_r[kTile][4], bytes_t[kTile][4];
  grid_dependency_handshake();
  const uint32_t tile_r = blockIdx.x / a.tiles_c, tile_c = blockIdx.x - tile_r * a.tiles_c;
  const uint32_t t = threadIdx.x, lane = t & 31, warp = t >> 5, part = lane % kAcross, down = lane / kAcross;
  const uint32_t warp_r = warp / kWarpsAcross, warp_c = warp % kWarpsAcross;
  const uint32_t r_in = 32 * warp_r + ROWS * down, c_in = 8 * (kAcross * warp_c + part);
  const uint32_t r0 = tile_r * kTile + r_in, c0 = tile_c * kTile + c_in;

  Held<T> h;
  {
    const T* p = static_cast<const T*>(a.x) + (uint64_t)r0 * a.ld + c0;
    const int n = c0 < a.cols ? (int)min(a.cols - c0, 8u) : 0;
    if (!WHOLE && sizeof(T) == 2 && n == 8 && (r0 > 0 || c0 > 0) && (r0 + ROWS < a.rows || (r0 + ROWS == a.rows && c0 + 9 < a.cols))) {
      RawEight<T> raw[ROWS];
#pragma unroll
      for (int i = 0; i < ROWS; ++i) load_raw<T>(p + i * a.ld, raw[i]);
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        uint32_t w[2 * sizeof(T)];
        words_of<T>(raw[i], p + i * a.ld, w);
#pragma unroll
        for (int j = 0; j < 4; ++j) h.w[i][j] = w[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const bool there = r0 + i < a.rows;
        hold_row(h, i, p, WHOLE && there && n == 8, there ? n : 0);
        p += a.ld;
      }
    }
  }
  float row_most[ROWS], col_most[8];
  micro_largest<ROWS>(h, row_most, col_most);
  bool bad = false;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) bad |= !is_finite_bits(row_most[i]);
  if (bad) atomicOr(a.status, kDevNonFinite);

  uint32_t square_byte = 0;  // of the 32 x 32 block that this thread's values lie in
  if (a.square) {
    float most = row_most[0];
#pragma unroll
    for (int i = 1; i < ROWS; ++i) most = max_nan(most, row_most[i]);
#pragma unroll
    for (int d = 1; d <= 16; d <<= 1)
      if (kAcross == 4 || d != 4) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, d));  // eight lanes across are two blocks
    square_byte = micro_scale_byte(most);
  }

  const uint64_t first = a.offset + (uint64_t)r0 * a.cols + c0;
  const DropKey key(a.rng, first);
  DropRow quads(a.rng, first, key);
  if (ROUND == MicroRound::kQuads) quads.phase = 0;  // known here: the other way of counting falls away
  uint32_t numbers[STOCHASTIC ? ROWS : 1][8];  // the upper 28 bits of the words' complements
  if constexpr (STOCHASTIC) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const auto keep = [&](int, const uint32_t (&w)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) numbers[i][j] = w[j] >> 4;
      };
      if (ROUND == MicroRound::kQuads) number_units<8, true, 1>(quads, i * (a.cols / 4), 0, keep);  // below 2^32: columns would wrap
      else number_units<8, true, 1>(DropRow(a.rng, first + (uint64_t)i * a.cols, key), 0, 0, keep);
    }
  }

  if (a.q) {
    float most[kRowsEach], half[ROWS / 2];
    halve_most<ROWS>(row_most, part & 2, 2, half);
    halve_most<ROWS / 2>(half, part & 1, 1, most);
    float inverse[kRowsEach];
#pragma unroll
    for (int k = 0; k < kRowsEach; ++k) {  // rows kRowsEach (part % 4) + k of the thread's
      const uint32_t in = kRowsEach * (part & 3) + k;
      uint32_t byte = a.square ? square_byte : micro_scale_byte(most[k]);
      inverse[k] = micro_inverse(byte);
      if (r0 + in >= a.rows || (c0 & ~31u) >= a.cols) byte = 127u;  // rows and blocks that do not exist, beside a square block that ends inside
      bytes_r[r_in + in][c_in / 32] = (uint8_t)byte;
    }
    uint8_t* q = a.q + (uint64_t)r0 * a.ldq + c0 / 2;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const float s = __shfl_sync(0xffffffffu, inverse[i % kRowsEach], (lane & ~3u) | (i / kRowsEach));
      float v[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = split(mul2(held_pair(h, i, j), both(s)));
        v[2 * j] = f.x;
        v[2 * j + 1] = f.y;
      }
      uint32_t code;
      if constexpr (STOCHASTIC) {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = split(mul2(pair_of(v[2 * j], v[2 * j + 1]), both(0x1p+25f)));
          w[2 * j] = micro_stochastic(v[2 * j], f.x, numbers[i][2 * j]);
          w[2 * j + 1] = micro_stochastic(v[2 * j + 1], f.y, numbers[i][2 * j + 1]);
        }
        code = micro_join<8>(w);
      } else {
        code = micro_encode<8>(v);
      }
      if (r0 + i < a.rows && c0 / 2 < a.ldq) st_c(reinterpret_cast<uint32_t*>(q), s == 0.0f ? 0u : code);
      q += a.ldq;
    }
  }

  if (a.qt) {
    float most[kColsEach];
    {
      float half[4], quarter[2];
      halve_most<8>(col_most, lane & 16, 16, half);
      halve_most<4>(half, lane & 8, 8, quarter);
      if constexpr (kColsEach == 1) halve_most<2>(quarter, lane & 4, 4, most);
      else { most[0] = quarter[0]; most[kColsEach - 1] = quarter[1]; }
    }
    float inverse[kColsEach];
#pragma unroll
    for (int k = 0; k < kColsEach; ++k) {  // columns kColsEach down + k of the eight
      const uint32_t in = kColsEach * down + k;
      uint32_t byte = a.square ? square_byte : micro_scale_byte(most[k]);
      inverse[k] = micro_inverse(byte);
      if (c0 + in >= a.cols || (r0 & ~31u) >= a.rows) byte = 127u;
      bytes_t[c_in + in][warp_r] = (uint8_t)byte;
    }
    // Column c of the tile is 64 bytes, ROWS rows of one thread side by side, 32 rows 16 bytes; u-th 16 at place u ^ (c / 8 % 4): the
    // lanes that write different columns meet different places.
    uint8_t* place = turned + c_in * (kTile / 2) + 16 * (warp_r ^ (part & 3)) + ROWS / 2 * down;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float s0 = __shfl_sync(0xffffffffu, inverse[0], part | (2 * j / kColsEach) * kAcross);
      const float s1 = __shfl_sync(0xffffffffu, inverse[kColsEach - 1], part | ((2 * j + 1) / kColsEach) * kAcross);
      const Pair scale = pair_of(s0, s1);
      float left[ROWS], right[ROWS];
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const float2 f = split(mul2(held_pair(h, i, j), scale));
        left[i] = f.x;
        right[i] = f.y;
      }
      uint32_t code[2];
      if constexpr (STOCHASTIC) {
        uint32_t w[2][ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
          const float2 f = split(mul2(pair_of(left[i], right[i]), both(0x1p+25f)));
          w[0][i] = micro_stochastic(left[i], f.x, numbers[i][2 * j]);
          w[1][i] = micro_stochastic(right[i], f.y, numbers[i][2 * j + 1]);
        }
        code[0] = micro_join<ROWS>(w[0]);
        code[1] = micro_join<ROWS>(w[1]);
      } else {
        code[0] = micro_encode<ROWS>(left);
        code[1] = micro_encode<ROWS>(right);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t w = (k ? s1 : s0) == 0.0f ? 0u : code[k];
        if constexpr (ROWS == 8) *reinterpret_cast<uint32_t*>(place + (2 * j + k) * (kTile / 2)) = w;
        else *reinterpret_cast<uint16_t*>(place + (2 * j + k) * (kTile / 2)) = (uint16_t)w;
      }
    }
  }
  __syncthreads();
  if (t < kTile) {
    if (a.q) st_c(reinterpret_cast<uint32_t*>(a.scale + scale_offset(tile_r * kTile + t, 4 * tile_c, a.tiles_r)), *reinterpret_cast<const uint32_t*>(bytes_r[t]));
    if (a.qt) st_c(reinterpret_cast<uint32_t*>(a.scale_t + scale_offset(tile_c * kTile + t, 4 * tile_r, a.tiles_c)), *reinterpret_cast<const uint32_t*>(bytes_t[t]));
  }
  if (a.qt) {
#pragma unroll
    for (int k = 0; k < kTile / (kMicroThreads<T, ROUND> / 4); ++k) {  // four threads a column, 16 bytes each
      const uint32_t c = (t >> 2) + kMicroThreads<T, ROUND> / 4 * k, u = t & 3;
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
        const uint32_t end = min((uint32_t)col[i] + 7, a.cols - 1);
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
        const int lo = ((uint32_t)col[i] + 2 * j) & 31, hi = ((uint32_t)col[i] + 2 * j + 1) & 31;  // the second scale from the first boundary on
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
          const uint32_t at = (uint32_t)col[i] + j;  // before the row: past every column
          if (at < a.cols) st_c(x + at, from_float<T>(j % 2 ? f.y : f.x));
        }
      }
    }
  }
}

}  // namespace accept
