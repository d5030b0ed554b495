// Root-mean-square norm of a residual stream, forward and backward (sm_100a), with the branch that is added first.
//
// Bound by memory: a row stays in the registers of the threads that share it (16 columns each) from the addition of the branch
// to the output, with one sum over the row between; the next rows are on their way into shared memory meanwhile
// (accept_rows.cuh).  The mask of the branch's dropout is worked out from the counters, twice where there is a backward pass.
#pragma once
#include "accept_block.cuh"
#include "accept_drop.cuh"
#include "accept_dropout.cuh"
#include "accept_rows.cuh"
#include "accept_shift.cuh"

namespace accept {

struct RmsArgs {
  const void* x;         // forward: the stream; backward: the sum that was normalised
  const void* branch;    // forward, may be null
  const void* gamma;     // may be null
  void* sum;             // forward, may be null
  void* y;               // forward, may be null
  uint8_t* q;            // forward, may be null: 8-bit codes of y and their scales
  uint8_t* scale;
  float* rstd_out;       // forward, may be null
  uint32_t* status;      // forward with q
  const float* rstd;     // backward
  const void* dy;
  const void* dsum;      // may be null
  void* dx;              // may be null
  void* dbranch;         // may be null
  float* partials;       // n_partials x cols, or null
  float* dgamma;
  Drop drop;
  uint64_t rows, ld_x, ld_y;
  uint32_t cols, warps;  // warps that share a row
  uint32_t n_partials;
  uint32_t ldq, blocks, atoms;  // of q: bytes between rows, blocks of 128 columns, groups of 128 rows
  float eps, inv_cols;
  int dtype_w, format;
  int whole_weights;     // gamma starts on a 16-byte boundary
  int joins;             // backward: the grid is one cluster, which adds up dgamma itself
};

extern __shared__ __align__(16) uint8_t rms_shared[];

// 1 / sqrt(mean + eps) from the sum of squares.  `again(f)`: the sum of (x f)^2, for rows whose squares leave the range of fp32
// (root mean squares above 2^60, or below 2^-50 where eps does not cover them), f a power of two that brings them back.
template <typename Again>
__device__ __forceinline__ float rms_rstd(const RmsArgs& a, float squares, const Again& again) {
  const float mean = squares * a.inv_cols + a.eps;
  if (mean > 0x1p-100f && mean < 0x1p+120f) return rsqrtf(mean);
  const float f = mean >= 1.0f ? 0x1p-96f : 0x1p+96f;  // sums of up to 2^31 such squares fit (NaN stays NaN either way)
  return rsqrtf(again(f) * a.inv_cols + a.eps * f * f) * f;
}

// The branch's elements after dropout: pairs as column_of deals them.
template <int V, int OWN, int L>
__device__ __forceinline__ void drop_row(const Drop& d, const DropRow& r, uint32_t t, Pair (&v)[OWN / 2]) {
  drop_units<V, OWN / V>(d, r, column_of<V, OWN, L>(t, 0), L * V, v);
}

// ---- rows that start anywhere (LOOSE) ----
// The row lies in shared memory as the 16-byte pieces that hold it, and in the registers of its threads as any other; what is read
// from there, and what is written to a row, is shifted by what the row's start is off: the same for the whole row.  So all loads
// and stores are whole units, but for the two ends of a warp's columns.
// (One or two values a load and store, as layer norm has it: 16384 x 4095 bf16 with a dropped branch 280 us forward.)

template <typename T, int V, int OWN, int L>
__device__ __forceinline__ void take_loose(uint32_t src, const T* row, uint32_t t, Pair (&v)[OWN / 2]) {
  constexpr int kUnit = V * (int)sizeof(T), kWords = kUnit / 4;  // a unit is 16 bytes, or 8
  const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(row) & 15);
  const uint32_t from = src + t / L * (L * OWN * (uint32_t)sizeof(T) + 16) + t % L * kUnit + (off & ~(uint32_t)(kUnit - 1));
#pragma unroll
  for (int i = 0; i < OWN / V; ++i) {
    uint32_t c[2 * kWords], w[kWords];
    if constexpr (kWords == 4) {
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(c[0]), "=r"(c[1]), "=r"(c[2]), "=r"(c[3]) : "r"(from + i * L * kUnit));
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(c[4]), "=r"(c[5]), "=r"(c[6]), "=r"(c[7]) : "r"(from + i * L * kUnit + 16));
    } else {
      asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(c[0]), "=r"(c[1]) : "r"(from + i * L * kUnit));
      asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(c[2]), "=r"(c[3]) : "r"(from + i * L * kUnit + 8));
    }
    shifted_words<kWords, kWords>(c, off & (kUnit - 1), w);
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      if constexpr (sizeof(T) == 4) v[i * V / 2 + j] = pair_of(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
      else v[i * V / 2 + j] = word_to_pair<T>(w[j]);
    }
  }
}

// To a row by way of `place`, the warp's part of a row of this type in shared memory that has been read: laid down as the threads hold
// them, fetched again as units that start on the row's boundaries.  The ends of the warp's columns, less than a unit each, leave value
// by value, the lower one from the first V lanes, the upper one from the next.
template <typename T, int V, bool FULL, int OWN, int L>
__device__ __forceinline__ void store_loose(T* row, uint32_t place, uint32_t cols, uint32_t t, uint32_t mask, const Pair (&v)[OWN / 2]) {
  constexpr int kUnit = V * (int)sizeof(T), kWords = kUnit / 4, kUnits = OWN / V;
  const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(row) & (kUnit - 1)), lane = t % L;
  const uint32_t low = t / L * (L * OWN), have = FULL ? L * OWN : min((uint32_t)(L * OWN), cols - min(low, cols));  // of the warp's columns
  place += t / L * (L * OWN * (uint32_t)sizeof(T) + 16);
  uint32_t mine[kUnits][kWords];
#pragma unroll
  for (int i = 0; i < kUnits; ++i)
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
      if constexpr (sizeof(T) == 4) mine[i][j] = __float_as_uint(j % 2 ? split(v[(i * V + j) / 2]).y : split(v[(i * V + j) / 2]).x);
      else mine[i][j] = pair_to_word<T>(v[i * V / 2 + j]);
    }
  const uint32_t own_place = place + lane * kUnit;
  __syncwarp(mask);  // all lanes have read what lay there
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    if constexpr (kWords == 4) asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(own_place + i * L * kUnit), "r"(mine[i][0]), "r"(mine[i][1]), "r"(mine[i][2]), "r"(mine[i][3]) : "memory");
    else asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(own_place + i * L * kUnit), "r"(mine[i][0]), "r"(mine[i][1]) : "memory");
  }
  __syncwarp(mask);
  T* to = row + low;
  const uint32_t ahead = (kUnit - off) & (kUnit - 1);  // bytes before the first boundary
  const uint32_t bytes = have * (uint32_t)sizeof(T), inner = bytes > ahead ? (bytes - ahead) / kUnit : 0;  // units between the boundaries
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    if (lane + i * L < inner) {
      uint32_t c[2 * kWords], w[kWords];
      const uint32_t from = own_place + i * L * kUnit;  // and the unit behind it: the space of a warp is 16 bytes longer
      if constexpr (kWords == 4) {
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(c[0]), "=r"(c[1]), "=r"(c[2]), "=r"(c[3]) : "r"(from) : "memory");
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(c[4]), "=r"(c[5]), "=r"(c[6]), "=r"(c[7]) : "r"(from + 16) : "memory");
      } else {
        asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(c[0]), "=r"(c[1]) : "r"(from) : "memory");
        asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(c[2]), "=r"(c[3]) : "r"(from + 8) : "memory");
      }
      shifted_words<kWords, kWords>(c, ahead, w);
      uint8_t* p = reinterpret_cast<uint8_t*>(to) + ahead + (lane + i * L) * kUnit;
      if constexpr (kWords == 4) {
        if (bounds_ok(p, 16, true)) __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
      } else {
        if (bounds_ok(p, 8, true)) __stcs(reinterpret_cast<uint2*>(p), make_uint2(w[0], w[1]));
      }
    }
  }
  // below the first boundary (or the end, where that comes first), and behind the last one
  constexpr bool kOnce = L >= 2 * V;
  const uint32_t head = min(ahead / (uint32_t)sizeof(T), have), tail = bytes > ahead ? (ahead + inner * kUnit) / (uint32_t)sizeof(T) : have;
#pragma unroll
  for (int end = 0; end < (kOnce ? 1 : 2); ++end) {
    const bool last = kOnce ? lane >= V : end == 1;
    const uint32_t c = (last ? tail : 0) + lane % V;
    if (lane < (kOnce ? 2 * V : V) && c < (last ? have : head)) {
      if constexpr (sizeof(T) == 4) {
        uint32_t w;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(place + 4 * c) : "memory");
        st_c(reinterpret_cast<uint32_t*>(to + c), w);
      } else {
        uint16_t w;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(place + 2 * c) : "memory");
        st_c(reinterpret_cast<uint16_t*>(to + c), w);
      }
    }
  }
}

// A row's copies, a row that has landed, and a row's values to memory, for rows that start on 16-byte boundaries or anywhere.
template <typename T, int V, bool FULL, int OWN, int L, bool LOOSE>
__device__ __forceinline__ void start_any(uint32_t dst, const T* row, uint32_t cols, uint32_t t, const Own<V, FULL, OWN, L>& own, const T* begin, const T* end) {
  if constexpr (LOOSE) start_row<T, 2, FULL, OWN, L>(dst, row, cols, t, Own<2, FULL, OWN, L>(t, cols), begin, end);
  else start_row<T, V, FULL, OWN, L>(dst, row, cols, t, own, begin, end);
}
template <typename T, int V, bool FULL, int OWN, int L, bool LOOSE>
__device__ __forceinline__ void take_any(uint32_t src, const T* row, uint32_t t, const Own<V, FULL, OWN, L>& own, Pair (&v)[OWN / 2]) {
  if constexpr (LOOSE) {
    take_loose<T, V, OWN, L>(src, row, t, v);
    if (!FULL)  // what lies behind the row's end is dropped
#pragma unroll
      for (int i = 0; i < OWN / V; ++i) {
        if (own.of(i) == V) continue;
#pragma unroll
        for (int j = i * V / 2; j < (i + 1) * V / 2; ++j) {
          const float2 f = split(v[j]);
          v[j] = pair_of(own.has(2 * j) ? f.x : 0.0f, own.has(2 * j + 1) ? f.y : 0.0f);
        }
      }
  } else {
    take_row<T, V, FULL, OWN, L>(src, row, t, own, v);
  }
}
template <typename T, int V, bool FULL, int OWN, int L, bool LOOSE>
__device__ __forceinline__ void store_any(T* row, uint32_t place, uint32_t cols, uint32_t t, uint32_t mask, const Own<V, FULL, OWN, L>& own, const Pair (&v)[OWN / 2]) {
  if constexpr (LOOSE) store_loose<T, V, FULL, OWN, L>(row, place, cols, t, mask, v);
  else store_row<T, V, FULL, OWN, L>(row, t, own, v);
}

// v rounded to T, as it is kept.
template <typename T>
__device__ __forceinline__ Pair rounded(Pair v) {
  if constexpr (sizeof(T) == 4) return v;
  else return word_to_pair<T>(pair_to_word<T>(v));
}

// The largest magnitude of the lanes that share a block, kLanes neighbours; a NaN or an infinity comes out on top.
template <int LANES>
__device__ __forceinline__ float largest_of(float most, uint32_t mask) {
  if constexpr (LANES == 32) {
    float r;
    asm("redux.sync.max.abs.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(most));
    return r;
  }
#pragma unroll
  for (int d = LANES / 2; d >= 1; d >>= 1) most = max_nan(most, __shfl_xor_sync(mask, most, d));
  return most;
}

// The row's values as 8-bit codes with a scale for each 128 columns (accept_block.cuh): a block's columns lie with kLanes lanes
// of a warp, kUnits units of each.  The lanes' columns are the four blocks (or the one) of a word of scales.
template <int FORMAT, int V, int OWN, int L>
__device__ __forceinline__ void store_codes(const RmsArgs& a, uint64_t row, uint32_t t, uint32_t mask, Pair (&v)[OWN / 2]) {
  constexpr int kUnits = 128 / (L * V) > 0 ? 128 / (L * V) : 1, kLanes = 128 / (V * kUnits), kBlocks = OWN / V / kUnits, kPairs = kUnits * V / 2;
  static_assert(kLanes <= L && OWN / V % kUnits == 0 && L * OWN == (L == 32 ? 512 : 128), "a block lies within a warp, a word of scales is one");
  float most[kBlocks];
  bool bad = false;
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
    most[b] = 0.0f;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      const float2 f = split(v[b * kPairs + j]);
      most[b] = max3_nan(most[b], fabsf(f.x), fabsf(f.y));
    }
    most[b] = largest_of<kLanes>(most[b], mask);
    bad |= !is_finite_bits(most[b]);
  }
  if (__any_sync(mask, bad)) {  // rare: scales are those of the finite values, the others become NaN
    bad = false;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      most[b] = 0.0f;
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        const float2 f = split(v[b * kPairs + j]);
        const bool x = is_finite_bits(f.x), y = is_finite_bits(f.y);
        bad |= !x || !y;
        most[b] = fmaxf(most[b], fmaxf(x ? fabsf(f.x) : 0.0f, y ? fabsf(f.y) : 0.0f));
        v[b * kPairs + j] = pair_of(x ? f.x : __uint_as_float(0x7fffffffu), y ? f.y : __uint_as_float(0x7fffffffu));
      }
      most[b] = largest_of<kLanes>(most[b], mask);
    }
    if (bad) atomicOr(a.status, kDevNonFinite);
  }
  uint32_t word = L < 32 ? 0x7f7f7f00u : 0u;
  Pair inverse[kBlocks];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
    const int e = scale_exponent<FORMAT>(most[b]);
    inverse[b] = both(power_of_two(-e));
    word |= (uint32_t)(e + 127) << (kLanes == 16 ? 16 * b : 8 * b);
  }
  if (kLanes == 16) word |= __shfl_xor_sync(mask, word, 16) << 8;  // lane 0: blocks 0 and 2 its own, 1 and 3 of the upper lanes
  if (t % L == 0) {
    const uint32_t r = (uint32_t)row;
    st_c(reinterpret_cast<uint32_t*>(a.scale + ((uint64_t)(t / L) * a.atoms + (r >> 7)) * 512 + (r & 31) * 16 + ((r >> 5) & 3) * 4), word);
  }
  uint8_t* q = a.q + row * a.ldq + column_of<V, OWN, L>(t, 0);
#pragma unroll
  for (int u = 0; u < OWN / V; ++u) {
    if (column_of<V, OWN, L>(t, u * V) >= a.ldq) continue;
    uint32_t code[V / 2];
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      const float2 f = split(mul2(v[u * V / 2 + j], inverse[u / kUnits]));
      code[j] = encode_two<FORMAT>(f.x, f.y);
    }
    uint8_t* to = q + u * (L * V);
    if constexpr (V == 8) st_c(reinterpret_cast<uint2*>(to), make_uint2(code[0] | code[1] << 16, code[2] | code[3] << 16));
    else st_c(reinterpret_cast<uint32_t*>(to), code[0] | code[1] << 16);
  }
}

// Scales of the rows that pad the last group of 128.
__device__ __forceinline__ void pad_scales(const RmsArgs& a) {
  const uint32_t words = (a.blocks + 3) / 4, missing = a.atoms * 128 - (uint32_t)a.rows;
  for (uint32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < missing * words; i += gridDim.x * blockDim.x)
    st_c(reinterpret_cast<uint32_t*>(a.scale + scale_offset((uint32_t)a.rows + i / words, i % words * 4, a.atoms)), 0x7f7f7f7fu);
}

// CODES: with 8-bit codes.  One kernel for both is slower without: 16384 x 4096 bf16 with dropped branch to bf16 97 us against 82.
template <typename TX, typename TY, int V, bool FULL, int OWN, int L, int STAGES, bool LOOSE, bool CODES>
__device__ __forceinline__ void rms_forward_rows(const RmsArgs& a, const Group<L>& g, float (&slots)[3][16], uint32_t shared, uint32_t space, uint32_t space_x,
                                                 uint64_t first, uint32_t step) {
  const uint32_t t = g.t, shared_end = shared + STAGES * space;
  const Own<V, FULL, OWN, L> own(t, a.cols);
  const TX* x = static_cast<const TX*>(a.x);
  const TY* branch = static_cast<const TY*>(a.branch);
  const TX* end_x = x + (a.rows - 1) * a.ld_x + a.cols;
  const TY* end_y = branch + (a.rows - 1) * a.ld_y + a.cols;
  const TX* row = x + first * a.ld_x;
  const TY* brow = branch + first * a.ld_y;
  const uint64_t stride_x = step * a.ld_x, stride_y = step * a.ld_y;
#pragma unroll
  for (int s = 0; s + 1 < STAGES; ++s) {
    if (first + (uint64_t)s * step < a.rows) {
      start_any<TX, V, FULL, OWN, L, LOOSE>(shared + s * space, row + s * stride_x, a.cols, t, own, x, end_x);
      if (branch) start_any<TY, V, FULL, OWN, L, LOOSE>(shared + s * space + space_x, brow + s * stride_y, a.cols, t, own, branch, end_y);
    }
    copy_commit();
  }
  Pair gamma[OWN / 2];
  load_weights<V, FULL, OWN, L>(a, a.gamma, own, 1.0f, t, gamma);
  uint32_t here = shared, ahead = shared + (STAGES - 1) * space, turn = 0;  // where this row lies, and where the one to start goes
  uint64_t r = first;
  const DropKey key(a.drop.rng, a.drop.offset + r * a.cols);
  for (;;) {
    if (r + (STAGES - 1) * (uint64_t)step < a.rows) {
      start_any<TX, V, FULL, OWN, L, LOOSE>(ahead, row + (STAGES - 1) * stride_x, a.cols, t, own, x, end_x);
      if (branch) start_any<TY, V, FULL, OWN, L, LOOSE>(ahead + space_x, brow + (STAGES - 1) * stride_y, a.cols, t, own, branch, end_y);
    }
    copy_commit();
    copy_wait<STAGES - 1>();
    if (LOOSE) __syncwarp(g.mask);  // other lanes of the warp have copied for this one
    Pair v[OWN / 2];
    take_any<TX, V, FULL, OWN, L, LOOSE>(here, row, t, own, v);
    if (branch) {
      Pair b[OWN / 2];
      take_any<TY, V, FULL, OWN, L, LOOSE>(here + space_x, brow, t, own, b);
      if (a.drop.on) drop_row<V, OWN, L>(a.drop, DropRow(a.drop.rng, a.drop.offset + r * a.cols, key), t, b);
#pragma unroll
      for (int i = 0; i < OWN / 2; ++i) v[i] = rounded<TX>(add2(v[i], b[i]));
    }
    if (a.sum) store_any<TX, V, FULL, OWN, L, LOOSE>(static_cast<TX*>(a.sum) + r * a.ld_x, here, a.cols, t, g.mask, own, v);
    Pair squares[2] = {mul2(v[0], v[0]), mul2(v[1], v[1])};
#pragma unroll
    for (int i = 2; i < OWN / 2; ++i) squares[i % 2] = fma2(v[i], v[i], squares[i % 2]);
    const float rstd = rms_rstd(a, g.sum(sum_of(add2(squares[0], squares[1])), slots[turn]), [&](float f) {
      Pair s = both(0.0f);
#pragma unroll
      for (int i = 0; i < OWN / 2; ++i) {
        const Pair w = mul2(v[i], both(f));
        s = fma2(w, w, s);
      }
      return g.sum(sum_of(s), slots[2]);
    });
    turn ^= 1;
#pragma unroll
    for (int i = 0; i < OWN / 2; ++i) v[i] = mul2(mul2(v[i], both(rstd)), gamma[i]);
    if (a.y) store_any<TY, V, FULL, OWN, L, LOOSE>(static_cast<TY*>(a.y) + r * a.ld_y, here + space_x, a.cols, t, g.mask, own, v);
    if (CODES && a.q) {
      if (!FULL)  // zero bytes behind the row's end, whatever its rstd is
#pragma unroll
        for (int i = 0; i < OWN / 2; ++i) {
          const float2 f = split(v[i]);
          v[i] = pair_of(own.has(2 * i) ? f.x : 0.0f, own.has(2 * i + 1) ? f.y : 0.0f);
        }
      if (a.format == kE4m3) store_codes<kE4m3, V, OWN, L>(a, r, t, g.mask, v);
      else store_codes<kE5m2, V, OWN, L>(a, r, t, g.mask, v);
    }
    if (a.rstd_out && t == 0) st_c(a.rstd_out + r, rstd);
    if (LOOSE) __syncwarp(g.mask);  // the row's place, through which it left, is free
    r += step;
    if (r >= a.rows) break;
    row += stride_x;
    brow += stride_y;
    ahead = here;
    here = here + space == shared_end ? shared : here + space;
  }
}

template <typename TX, typename TY, int V, int OWN, int L, int STAGES, bool LOOSE, bool CODES>
__global__ void __launch_bounds__(512) rms_forward_kernel(const RmsArgs a) {
  __shared__ __align__(16) float slots[kMostGroups][3][16];
  const Group<L> g(a.warps);
  const uint32_t groups = blockDim.x / g.threads;
  const uint32_t space_x = row_space<TX>(LOOSE ? 2 : V, OWN, L, a.warps), space = space_x + (a.branch || LOOSE ? row_space<TY>(LOOSE ? 2 : V, OWN, L, a.warps) : 0);
  const uint32_t shared = (uint32_t)__cvta_generic_to_shared(rms_shared) + g.index * STAGES * space;
  const uint64_t first = (uint64_t)blockIdx.x * groups + g.index;
  const uint32_t step = gridDim.x * groups;
  const bool full = lanes_are_full<OWN, L>(g.t, a.cols);
  if (!full) {
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
      clear_row<TX, LOOSE ? 2 : V, OWN, L>(shared + i * space, g.t, a.cols);
      if (a.branch) clear_row<TY, LOOSE ? 2 : V, OWN, L>(shared + i * space + space_x, g.t, a.cols);
    }
  }
  if (L == 32 && a.warps > 1) {
    float* zero = &slots[g.index][0][0];
    for (uint32_t i = g.t; i < 48; i += g.threads) zero[i] = 0.0f;
    g.sync();
  }
  grid_dependency_handshake();
  if (CODES && a.q) pad_scales(a);
  if (first >= a.rows) return;
  if (full) rms_forward_rows<TX, TY, V, true, OWN, L, STAGES, LOOSE, CODES>(a, g, slots[g.index % kMostGroups], shared, space, space_x, first, step);
  else rms_forward_rows<TX, TY, V, false, OWN, L, STAGES, LOOSE, CODES>(a, g, slots[g.index % kMostGroups], shared, space, space_x, first, step);
}

// Backward: dx = rstd (h - xhat mean(h xhat)) + dsum, h = dy gamma, xhat = x rstd; the sum over the rows (dgamma) is held in registers over
// all rows of a group, added up over the block's groups and joined by rms_join_kernel.
template <typename TX, typename TY, int V, bool FULL, int OWN, int L, int STAGES, bool LOOSE>
__device__ __forceinline__ void rms_backward_rows(const RmsArgs& a, const Group<L>& g, float (&slots)[2][16], uint32_t shared, uint32_t space, uint32_t space_x,
                                                  uint32_t space_y, uint64_t first, uint32_t step, Pair (&dgamma)[OWN / 2]) {
  const uint32_t t = g.t, shared_end = shared + STAGES * space;
  const Own<V, FULL, OWN, L> own(t, a.cols);
  const TX* x = static_cast<const TX*>(a.x);
  const TY* dy = static_cast<const TY*>(a.dy);
  const TX* dsum = static_cast<const TX*>(a.dsum);
  const uint64_t last = (a.rows - 1) * a.ld_x + a.cols;
  const TY* end_y = dy + (a.rows - 1) * a.ld_y + a.cols;
  uint64_t at_x = first * a.ld_x, at_y = first * a.ld_y;
  const uint64_t stride_x = step * a.ld_x, stride_y = step * a.ld_y;
  const auto start = [&](uint32_t to, uint64_t from_x, uint64_t from_y) {
    start_any<TX, V, FULL, OWN, L, LOOSE>(to, x + from_x, a.cols, t, own, x, x + last);
    start_any<TY, V, FULL, OWN, L, LOOSE>(to + space_x, dy + from_y, a.cols, t, own, dy, end_y);
    if (dsum) start_any<TX, V, FULL, OWN, L, LOOSE>(to + space_x + space_y, dsum + from_x, a.cols, t, own, dsum, dsum + last);
  };
#pragma unroll
  for (int s = 0; s + 1 < STAGES; ++s) {
    if (first + (uint64_t)s * step < a.rows) start(shared + s * space, at_x + s * stride_x, at_y + s * stride_y);
    copy_commit();
  }
  Pair gamma[OWN / 2];
  load_weights<V, FULL, OWN, L>(a, a.gamma, own, 1.0f, t, gamma);
  uint32_t here = shared, ahead = shared + (STAGES - 1) * space, turn = 0;
  uint64_t r = first;
  float rstd_next = ld_c(a.rstd + r);
  const DropKey key(a.drop.rng, a.drop.offset + r * a.cols);
  for (;;) {
    if (r + (STAGES - 1) * (uint64_t)step < a.rows) start(ahead, at_x + (STAGES - 1) * stride_x, at_y + (STAGES - 1) * stride_y);
    copy_commit();
    const float rstd = rstd_next;
    if (r + step < a.rows) rstd_next = ld_c(a.rstd + r + step);
    copy_wait<STAGES - 1>();
    if (LOOSE) __syncwarp(g.mask);  // other lanes of the warp have copied for this one
    Pair xhat[OWN / 2], h[OWN / 2];
    take_any<TX, V, FULL, OWN, L, LOOSE>(here, x + at_x, t, own, xhat);
    take_any<TY, V, FULL, OWN, L, LOOSE>(here + space_x, dy + at_y, t, own, h);
    Pair along[2] = {both(0.0f), both(0.0f)};
#pragma unroll
    for (int i = 0; i < OWN / 2; ++i) {
      xhat[i] = mul2(xhat[i], both(rstd));
      dgamma[i] = fma2(h[i], xhat[i], dgamma[i]);
      h[i] = mul2(h[i], gamma[i]);
      along[i % 2] = fma2(h[i], xhat[i], along[i % 2]);
    }
    if (a.dx || a.dbranch) {
      const Pair slope = both(-g.sum(sum_of(add2(along[0], along[1])), slots[turn]) * a.inv_cols);
      turn ^= 1;
#pragma unroll
      for (int i = 0; i < OWN / 2; ++i) h[i] = mul2(fma2(xhat[i], slope, h[i]), both(rstd));
      if (dsum) {
        take_any<TX, V, FULL, OWN, L, LOOSE>(here + space_x + space_y, dsum + at_x, t, own, xhat);
#pragma unroll
        for (int i = 0; i < OWN / 2; ++i) h[i] = add2(h[i], xhat[i]);
      }
      if (a.dx) store_any<TX, V, FULL, OWN, L, LOOSE>(static_cast<TX*>(a.dx) + at_x, here, a.cols, t, g.mask, own, h);
      if (a.dbranch) {
        if (a.drop.on) drop_row<V, OWN, L>(a.drop, DropRow(a.drop.rng, a.drop.offset + r * a.cols, key), t, h);
        store_any<TY, V, FULL, OWN, L, LOOSE>(static_cast<TY*>(a.dbranch) + at_y, here + space_x, a.cols, t, g.mask, own, h);
      }
    }
    if (LOOSE) __syncwarp(g.mask);  // the row has been read: its place is free
    r += step;
    if (r >= a.rows) break;
    at_x += stride_x;
    at_y += stride_y;
    ahead = here;
    here = here + space == shared_end ? shared : here + space;
  }
}

template <typename TX, typename TY, int V, int OWN, int L, int STAGES, bool LOOSE>
__global__ void __launch_bounds__(512) rms_backward_kernel(const RmsArgs a) {
  __shared__ __align__(16) float slots[kMostGroups][2][16];
  const Group<L> g(a.warps);
  const uint32_t groups = blockDim.x / g.threads, t = g.t, threads = g.threads;
  const uint32_t space_x = row_space<TX>(LOOSE ? 2 : V, OWN, L, a.warps), space_y = row_space<TY>(LOOSE ? 2 : V, OWN, L, a.warps), space = space_x + space_y + (a.dsum ? space_x : 0);
  const uint32_t shared = (uint32_t)__cvta_generic_to_shared(rms_shared) + g.index * STAGES * space;
  const uint64_t first = (uint64_t)blockIdx.x * groups + g.index;
  const uint32_t step = gridDim.x * groups;
  const bool full = lanes_are_full<OWN, L>(t, a.cols);
  if (!full) {
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
      clear_row<TX, LOOSE ? 2 : V, OWN, L>(shared + i * space, t, a.cols);
      clear_row<TY, LOOSE ? 2 : V, OWN, L>(shared + i * space + space_x, t, a.cols);
      if (a.dsum) clear_row<TX, LOOSE ? 2 : V, OWN, L>(shared + i * space + space_x + space_y, t, a.cols);
    }
  }
  if (L == 32 && a.warps > 1) {
    float* zero = &slots[g.index][0][0];
    for (uint32_t i = t; i < 32; i += threads) zero[i] = 0.0f;
    g.sync();
  }
  grid_dependency_handshake();
  Pair dgamma[OWN / 2];
#pragma unroll
  for (int i = 0; i < OWN / 2; ++i) dgamma[i] = both(0.0f);
  if (first < a.rows) {
    if (full) rms_backward_rows<TX, TY, V, true, OWN, L, STAGES, LOOSE>(a, g, slots[g.index % kMostGroups], shared, space, space_x, space_y, first, step, dgamma);
    else rms_backward_rows<TX, TY, V, false, OWN, L, STAGES, LOOSE>(a, g, slots[g.index % kMostGroups], shared, space, space_x, space_y, first, step, dgamma);
  }
  if (!a.dgamma) return;
  float* out = a.partials + (uint64_t)blockIdx.x * a.cols;
  if (groups == 1 && !a.joins) {
    const bool quads = a.cols % 4 == 0;
#pragma unroll
    for (int i = 0; i < OWN; i += 4) {
      const uint32_t c = column_of<V, OWN, L>(t, i);
      const float2 d0 = split(dgamma[i / 2]), d1 = split(dgamma[i / 2 + 1]);
      if (quads) {
        if (c < a.cols) st_c(reinterpret_cast<float4*>(out + c), make_float4(d0.x, d0.y, d1.x, d1.y));
      } else {
        const float d[4] = {d0.x, d0.y, d1.x, d1.y};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t cj = column_of<V, OWN, L>(t, i + j);
          if (cj < a.cols) st_c(out + cj, d[j]);
        }
      }
    }
    return;
  }
  // the groups of the block lay their sums side by side in shared memory; all threads add them up, group after group
  const uint32_t width = a.warps * L * OWN;
  float* sums = reinterpret_cast<float*>(rms_shared);
  copy_wait<0>();
  __syncthreads();
  float* mine = sums + g.index * width;
#pragma unroll
  for (int i = 0; i < OWN / 2; ++i) {
    const float2 d = split(dgamma[i]);
    mine[column_of<V, OWN, L>(t, 2 * i)] = d.x;
    mine[column_of<V, OWN, L>(t, 2 * i + 1)] = d.y;
  }
  __syncthreads();
#pragma unroll 2
  for (uint32_t c = threadIdx.x; c < a.cols && (groups > 1 || a.joins); c += blockDim.x) {
    float d = 0.0f;
#pragma unroll 4
    for (uint32_t k = 0; k < groups; ++k) d += sums[k * width + c];
    if (a.joins) sums[c] = d;
    else st_c(out + c, d);
  }
  if (!a.joins) return;
  // few rows: the blocks of the one cluster take the columns in turn and add up what each of them has, in their order
  cluster_sync();
  const uint32_t from = smem_address(sums);
#pragma unroll 2
  for (uint32_t c = blockIdx.x * blockDim.x + threadIdx.x; c < a.cols; c += gridDim.x * blockDim.x) {
    float v[8], d = 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) v[k] = k < gridDim.x ? ld_cluster_one(address_in(from + 4 * c, k)) : 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) d += v[k];
    st_c(a.dgamma + c, d);
  }
  cluster_sync();  // no block leaves while others read its sums
}

// ---- rows of more than 8192 columns: a block a row, which is read again for the output (it lies in the caches by then) ----

__device__ __forceinline__ float rms_block_sum(float v, float* slot) {  // a barrier lies between two uses of a slot
  v = warp_sum(v);
  const uint32_t lane = threadIdx.x & 31;
  if (lane == 0) slot[threadIdx.x >> 5] = v;
  __syncthreads();
  return warp_sum(lane < blockDim.x >> 5 ? slot[lane] : 0.0f);
}

constexpr int kWideThreads = 512;

template <typename T>
__device__ __forceinline__ void weights_eight(const T* w, bool whole, int n, Pair (&v)[4]) {
  if (whole) load_eight<T, true>(w, n, v);
  else load_eight<T, false>(w, n, v);
}
__device__ __forceinline__ void gamma_eight(const RmsArgs& a, uint32_t c, int n, Pair (&v)[4]) {
  if (!a.gamma) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = both(1.0f);
  } else if (a.dtype_w == kF32) weights_eight(static_cast<const float*>(a.gamma) + c, a.whole_weights, n, v);
  else if (a.dtype_w == kBf16) weights_eight(static_cast<const __nv_bfloat16*>(a.gamma) + c, a.whole_weights, n, v);
  else weights_eight(static_cast<const __half*>(a.gamma) + c, a.whole_weights, n, v);
}

template <int FORMAT>
__device__ __forceinline__ void store_codes_eight(const RmsArgs& a, uint64_t row, uint32_t c, Pair (&v)[4]) {  // by whole warps: 16 lanes hold a block
  float most = 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = split(v[j]);
    most = max3_nan(most, fabsf(f.x), fabsf(f.y));
  }
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, d));
  if (__any_sync(0xffffffffu, !is_finite_bits(most))) {
    bool bad = false;
    most = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = split(v[j]);
      const bool x = is_finite_bits(f.x), y = is_finite_bits(f.y);
      bad |= !x || !y;
      most = fmaxf(most, fmaxf(x ? fabsf(f.x) : 0.0f, y ? fabsf(f.y) : 0.0f));
      v[j] = pair_of(x ? f.x : __uint_as_float(0x7fffffffu), y ? f.y : __uint_as_float(0x7fffffffu));
    }
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
    if (bad) atomicOr(a.status, kDevNonFinite);
  }
  const int e = scale_exponent<FORMAT>(most);
  const Pair inverse = both(power_of_two(-e));
  if ((threadIdx.x & 15) == 0 && c < a.cols) store_scale(a.scale, (uint32_t)row, c / 128, a.blocks, a.atoms, e);
  uint32_t code[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = split(mul2(v[j], inverse));
    code[j] = encode_two<FORMAT>(f.x, f.y);
  }
  if (c < a.ldq) st_c(reinterpret_cast<uint2*>(a.q + row * a.ldq + c), make_uint2(code[0] | code[1] << 16, code[2] | code[3] << 16));
}

template <typename TX, typename TY, bool VEC>
__global__ void __launch_bounds__(kWideThreads) rms_forward_wide_kernel(const RmsArgs a) {
  __shared__ float slots[3][32];
  grid_dependency_handshake();
  if (a.q) pad_scales(a);
  uint32_t turn = 0;
  const DropKey key(a.drop.rng, a.drop.offset + blockIdx.x * (uint64_t)a.cols);
  for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
    const TX* row = static_cast<const TX*>(a.x) + r * a.ld_x;
    const TY* branch = a.branch ? static_cast<const TY*>(a.branch) + r * a.ld_y : nullptr;
    TX* kept = a.sum ? static_cast<TX*>(a.sum) + r * a.ld_x : nullptr;
    const DropRow numbers(a.drop.rng, a.drop.offset + r * a.cols, key);
    const auto sum_of_eight = [&](uint32_t c, int n, Pair (&v)[4]) {
      load_eight<TX, VEC>(row + c, n, v);
      if (branch) {
        Pair b[4];
        load_eight<TY, VEC>(branch + c, n, b);
        if (a.drop.on) drop_units<8, 1>(a.drop, numbers, c, 0, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = rounded<TX>(add2(v[j], b[j]));
      }
    };
    Pair squares = both(0.0f);
    for (uint32_t c = 8 * threadIdx.x; c < a.cols; c += 8 * kWideThreads) {
      const int n = (int)min(a.cols - c, 8u);
      Pair v[4];
      sum_of_eight(c, n, v);
      if (kept) store_eight<TX, VEC>(kept + c, n, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) squares = fma2(v[j], v[j], squares);
    }
    // what this thread has written it reads again itself
    const auto again_eight = [&](uint32_t c, int n, Pair (&v)[4]) {
      if (kept) load_eight<TX, VEC>(kept + c, n, v);
      else sum_of_eight(c, n, v);
    };
    const float rstd = rms_rstd(a, rms_block_sum(sum_of(squares), slots[turn]), [&](float f) {
      Pair s = both(0.0f);
      for (uint32_t c = 8 * threadIdx.x; c < a.cols; c += 8 * kWideThreads) {
        Pair v[4];
        again_eight(c, (int)min(a.cols - c, 8u), v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const Pair w = mul2(v[j], both(f));
          s = fma2(w, w, s);
        }
      }
      return rms_block_sum(sum_of(s), slots[2]);
    });
    for (uint32_t base = 0; base < a.cols; base += 8 * kWideThreads) {  // whole warps: the codes' maxima are taken over lanes
      const uint32_t c = base + 8 * threadIdx.x;
      const int n = c < a.cols ? (int)min(a.cols - c, 8u) : 0;
      Pair v[4], w[4];
      if (n) {
        again_eight(c, n, v);
        gamma_eight(a, c, n, w);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = n ? mul2(mul2(v[j], both(rstd)), w[j]) : both(0.0f);
      if (a.y && n) store_eight<TY, VEC>(static_cast<TY*>(a.y) + r * a.ld_y + c, n, v);
      if (a.q) {
        if (n < 8)  // zero bytes behind the row's end, whatever its rstd is
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 f = split(v[j]);
            v[j] = pair_of(2 * j < n ? f.x : 0.0f, 2 * j + 1 < n ? f.y : 0.0f);
          }
        if (a.format == kE4m3) store_codes_eight<kE4m3>(a, r, c, v);
        else store_codes_eight<kE5m2>(a, r, c, v);
      }
    }
    if (a.rstd_out && threadIdx.x == 0) st_c(a.rstd_out + r, rstd);
  }
}

template <typename TX, typename TY, bool VEC>
__global__ void __launch_bounds__(kWideThreads) rms_backward_wide_kernel(const RmsArgs a) {
  __shared__ float slots[2][32];
  grid_dependency_handshake();
  uint32_t turn = 0;
  const DropKey key(a.drop.rng, a.drop.offset + blockIdx.x * (uint64_t)a.cols);
  for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
    const TX* row = static_cast<const TX*>(a.x) + r * a.ld_x;
    const TY* drow = static_cast<const TY*>(a.dy) + r * a.ld_y;
    const float rstd = ld_c(a.rstd + r);
    const auto take = [&](uint32_t c, int n, Pair (&xhat)[4], Pair (&h)[4]) {
      Pair w[4];
      load_eight<TX, VEC>(row + c, n, xhat);
      load_eight<TY, VEC>(drow + c, n, h);
      gamma_eight(a, c, n, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        xhat[j] = mul2(xhat[j], both(rstd));
        h[j] = mul2(h[j], w[j]);
      }
    };
    Pair along = both(0.0f);
    for (uint32_t c = 8 * threadIdx.x; c < a.cols; c += 8 * kWideThreads) {
      Pair xhat[4], h[4];
      take(c, (int)min(a.cols - c, 8u), xhat, h);
#pragma unroll
      for (int j = 0; j < 4; ++j) along = fma2(h[j], xhat[j], along);
    }
    const Pair slope = both(-rms_block_sum(sum_of(along), slots[turn]) * a.inv_cols);
    const DropRow numbers(a.drop.rng, a.drop.offset + r * a.cols, key);
    for (uint32_t c = 8 * threadIdx.x; c < a.cols; c += 8 * kWideThreads) {
      const int n = (int)min(a.cols - c, 8u);
      Pair xhat[4], h[4];
      take(c, n, xhat, h);
#pragma unroll
      for (int j = 0; j < 4; ++j) h[j] = mul2(fma2(xhat[j], slope, h[j]), both(rstd));
      if (a.dsum) {
        load_eight<TX, VEC>(static_cast<const TX*>(a.dsum) + r * a.ld_x + c, n, xhat);
#pragma unroll
        for (int j = 0; j < 4; ++j) h[j] = add2(h[j], xhat[j]);
      }
      if (a.dx) store_eight<TX, VEC>(static_cast<TX*>(a.dx) + r * a.ld_x + c, n, h);
      if (a.dbranch) {
        if (a.drop.on) drop_units<8, 1>(a.drop, numbers, c, 0, h);
        store_eight<TY, VEC>(static_cast<TY*>(a.dbranch) + r * a.ld_y + c, n, h);
      }
    }
  }
}

// dgamma of such rows: 256 columns a block, the rows of its slab (blockIdx.y) dealt over eight warps, four rows on their way for
// each.  With one slab the sums are the results.
template <typename TX, typename TY, bool VEC>
__global__ void __launch_bounds__(256) rms_column_sums_kernel(const RmsArgs a) {
  __shared__ float part[8][256 + 1];
  constexpr int kAtOnce = 4;
  grid_dependency_handshake();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t c = ((uint64_t)blockIdx.x * 32 + lane) * 8;
  const int n = c < a.cols ? (int)min(a.cols - c, (uint64_t)8) : 0;
  Pair sums[4] = {both(0.0f), both(0.0f), both(0.0f), both(0.0f)};
  if (n) {
    const uint64_t step = 8ull * gridDim.y;
#pragma unroll 1
    for (uint64_t r = blockIdx.y * 8 + warp; r < a.rows; r += kAtOnce * step) {
      Pair u[kAtOnce][4], v[kAtOnce][4];
      float rstd[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const uint64_t row = r + j * step;
        rstd[j] = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) u[j][k] = v[j][k] = both(0.0f);
        if (row < a.rows) {
          const TY* drow = static_cast<const TY*>(a.dy) + row * a.ld_y;
          const TX* xrow = static_cast<const TX*>(a.x) + row * a.ld_x;
          load_eight<TY, VEC>(drow + c, n, u[j]);
          load_eight<TX, VEC>(xrow + c, n, v[j]);
          rstd[j] = ld_c(a.rstd + row);
        }
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) sums[k] = fma2(u[j][k], mul2(v[j][k], both(rstd[j])), sums[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 f = split(sums[k]);
    part[warp][lane * 8 + 2 * k] = f.x;
    part[warp][lane * 8 + 2 * k + 1] = f.y;
  }
  __syncthreads();
  const uint64_t col = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (col < a.cols) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += part[w][threadIdx.x];
    st_c((gridDim.y > 1 ? a.partials + (uint64_t)blockIdx.y * a.cols : a.dgamma) + col, s);
  }
}

// dgamma from the blocks' partial sums: 32 columns a block, the partials dealt over its sixteen warps, all of a warp's loads on
// their way at once, and added in a fixed order.
constexpr int kRmsJoinWarps = 16;
template <int WARPS>
__global__ void __launch_bounds__(32 * WARPS) rms_join_kernel(const RmsArgs a) {
  __shared__ float part[WARPS][33];
  grid_dependency_handshake();
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t c = (uint64_t)blockIdx.x * 32 + lane;
  float s = 0.0f;
  if (c < a.cols) {
    const float* p = a.partials + c;
    constexpr int kAtOnce = 10;  // 148 blocks over 16 warps
    for (uint32_t i = warp; i < a.n_partials; i += kAtOnce * WARPS) {
      float v[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) v[j] = i + j * WARPS < a.n_partials ? ld_c(p + (uint64_t)(i + j * WARPS) * a.cols) : 0.0f;
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) s += v[j];
    }
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < a.cols) {
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) s += part[w][lane];
    st_c(a.dgamma + c, s);
  }
}

}  // namespace accept
