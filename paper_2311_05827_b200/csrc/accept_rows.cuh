// Rows of a matrix shared by the threads of a warp or of several (sm_100a): how their columns are dealt, copies into shared
// memory that run ahead, and sums over a row.  What layer norm and the root-mean-square norm are made of.
#pragma once
#include "accept_tensor.cuh"
#include "accept_types.cuh"

namespace accept {

// How the columns of a row lie over the threads that share it: L lanes (a warp, or eight lanes where a row is short) hold
// L OWN neighbours, as units of V neighbours dealt over them, so that all addresses of a thread are one base and constants.  V = 8 where both tensors are 16-bit types,
// 4 where one is fp32 (16 bytes at most for a thread, neighbours side by side); where rows do not start on 16-byte
// boundaries, 2 if those of the 16-bit tensors start on 4-byte ones, else 1.
template <int V, int OWN, int L>
__device__ __forceinline__ uint32_t column_of(uint32_t t, int own) {
  return t / L * (L * OWN) + V * (t % L) + own / V * (L * V) + own % V;
}
template <int OWN, int L>  // all columns of the L lanes exist
__device__ __forceinline__ bool lanes_are_full(uint32_t t, uint32_t cols) { return (t / L + 1) * (L * OWN) <= cols; }

// How many values of each of the thread's units exist (V = 1 and 2: a bit for each value).  FULL: all of them.
template <int V, bool FULL, int OWN, int L>
struct Own {
  static constexpr int kUnits = V > 2 ? OWN / V : 1;
  uint32_t count[kUnits];
  __device__ __forceinline__ Own(uint32_t t, uint32_t cols) {
    if (V > 2) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const uint32_t c = column_of<V, OWN, L>(t, V * i);
        count[i] = c < cols ? min(cols - c, (uint32_t)V) : 0;
      }
    } else {
      count[0] = 0;
#pragma unroll
      for (int j = 0; j < OWN; ++j) count[0] |= column_of<V, OWN, L>(t, j) < cols ? 1u << j : 0u;
    }
  }
  __device__ __forceinline__ uint32_t of(int unit) const {
    return FULL ? V : V > 2 ? count[unit % kUnits] : V == 2 ? (count[0] >> 2 * unit & 1) + (count[0] >> (2 * unit + 1) & 1) : count[0] >> unit & 1;
  }
  __device__ __forceinline__ bool has(int value) const {  // value of the thread's OWN
    return FULL || (V > 2 ? (uint32_t)(value % V) < count[value / V % kUnits] : (count[0] >> value & 1) != 0);
  }
};

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, uint32_t bytes) {  // the rest of BYTES is zero
  if (!bounds_ok(src, bytes, false)) bytes = 0;
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// With offsets from the two addresses that the instruction holds.
template <int BYTES, int TO, int FROM>
__device__ __forceinline__ void copy_async_at(uint32_t dst, const void* src) {
  if (!bounds_ok(static_cast<const uint8_t*>(src) + FROM, BYTES, false)) return;
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0+%2], [%1+%3], 16;" ::"r"(dst), "l"(src), "n"(TO), "n"(FROM) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0+%2], [%1+%3], 8;" ::"r"(dst), "l"(src), "n"(TO), "n"(FROM) : "memory");
}
template <int BYTES, int TO, int FROM>
__device__ __forceinline__ void copy_async_at(uint32_t dst, const void* src, uint32_t bytes) {  // the rest of BYTES is zero
  if (!bounds_ok(static_cast<const uint8_t*>(src) + FROM, bytes, false)) return;
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0+%2], [%1+%3], 16, %4;" ::"r"(dst), "l"(src), "n"(TO), "n"(FROM), "r"(bytes) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0+%2], [%1+%3], 8, %4;" ::"r"(dst), "l"(src), "n"(TO), "n"(FROM), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING>  // all but the last PENDING groups have landed
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }

// Bytes of shared memory that a row of T takes for `warps` times `lanes` threads (V = 1 and 2: for each of the warps the
// 16-byte pieces that hold its columns).
template <typename T>
__host__ __device__ constexpr uint32_t row_space(int v, int own, uint32_t lanes, uint32_t warps) {
  return warps * (lanes * own * (uint32_t)sizeof(T) + (v > 2 ? 0 : 16));
}

// Starts the copies of a row into `dst` (shared).  `begin` and `end` bound the values of the matrix.  Units that do not
// exist are not copied: their places hold zeros from the start (clear_row).
template <typename T, int V, bool FULL, int OWN, int L, int I = 0>
__device__ __forceinline__ void start_units(uint32_t to, const T* from, const Own<V, FULL, OWN, L>& own) {
  constexpr int kBytes = V * (int)sizeof(T), kTo = I * L * kBytes, kFrom = I * L * V * (int)sizeof(T);
  static_assert(kBytes == 8 || kBytes == 16, "a unit is one copy");
  if (FULL) copy_async_at<kBytes, kTo, kFrom>(to, from);
  else if (own.of(I)) copy_async_at<kBytes, kTo, kFrom>(to, from, own.of(I) * (uint32_t)sizeof(T));
  if constexpr (I + 1 < OWN / V) start_units<T, V, FULL, OWN, L, I + 1>(to, from, own);
}
template <typename T, int V, bool FULL, int OWN, int L>
__device__ __forceinline__ void start_row(uint32_t dst, const T* row, uint32_t cols, uint32_t t, const Own<V, FULL, OWN, L>& own,
                                          const T* begin, const T* end) {
  if constexpr (V > 2) {
    const uint32_t first = column_of<V, OWN, L>(t, 0), to = dst + first * (uint32_t)sizeof(T);
    const T* from = row + first;
    start_units(to, from, own);
  } else {
    // the 16-byte pieces that hold the L lanes' columns; what lies outside the matrix is not read
    constexpr uint32_t kBytes = L * OWN * (uint32_t)sizeof(T);
    const uint32_t part = t / L, lane = t % L;
    dst += part * (kBytes + 16) + 16 * lane;
    const T* begins = row + part * (L * OWN);
    const uintptr_t from = (reinterpret_cast<uintptr_t>(begins) & ~(uintptr_t)15) + 16 * lane;
    if (FULL && row != begin && row + cols != end) {
      const void* p = reinterpret_cast<const void*>(from);
      copy_async_at<16, 0, 0>(dst, p);
      copy_async_at<16, 16 * L, 16 * L>(dst, p);
      if constexpr (kBytes > 32 * L) {
        copy_async_at<16, 32 * L, 32 * L>(dst, p);
        copy_async_at<16, 48 * L, 48 * L>(dst, p);
      }
      if constexpr (kBytes > 64 * L) {
        copy_async_at<16, 64 * L, 64 * L>(dst, p);
        copy_async_at<16, 80 * L, 80 * L>(dst, p);
        copy_async_at<16, 96 * L, 96 * L>(dst, p);
        copy_async_at<16, 112 * L, 112 * L>(dst, p);
      }
      if (lane == 0) copy_async_at<16, kBytes, kBytes>(dst, p);  // the columns end inside one more piece, or before it
    } else {
      const T* ends = part * (L * OWN) + L * OWN < cols ? begins + L * OWN : row + cols;
      for (uintptr_t at = from; at < reinterpret_cast<uintptr_t>(ends); at += 16 * L, dst += 16 * L) {
        if (at >= reinterpret_cast<uintptr_t>(begin)) {
          const uint64_t left = reinterpret_cast<uintptr_t>(end) - at;
          copy_async<16>(dst, reinterpret_cast<const void*>(at), left < 16 ? (uint32_t)left : 16u);
        } else {  // the matrix starts inside this piece
          for (const T* p = begin; reinterpret_cast<uintptr_t>(p) < at + 16 && p < end; ++p) {
            const T v = ld_c(p);
            const uint32_t to_byte = dst + (uint32_t)(reinterpret_cast<uintptr_t>(p) - at);
            if (sizeof(T) == 4) {
              uint32_t w;
              memcpy(&w, &v, sizeof(T));
              asm volatile("st.shared.u32 [%0], %1;" ::"r"(to_byte), "r"(w) : "memory");
            } else {
              uint16_t w;
              memcpy(&w, &v, 2);
              asm volatile("st.shared.u16 [%0], %1;" ::"r"(to_byte), "h"(w) : "memory");
            }
          }
        }
      }
    }
  }
}

// Zeros where this thread's units that do not exist would lie.
template <typename T, int V, int OWN, int L>
__device__ __forceinline__ void clear_row(uint32_t dst, uint32_t t, uint32_t cols) {
  if (V <= 2) return;
#pragma unroll
  for (int i = 0; i < OWN; i += V) {
    if (column_of<V, OWN, L>(t, i) < cols) continue;
    const uint32_t at = dst + column_of<V, OWN, L>(t, i) * (uint32_t)sizeof(T);
#pragma unroll
    for (int j = 0; j < V * (int)sizeof(T); j += 8) asm volatile("st.shared.u64 [%0], %1;" ::"r"(at + j), "l"(0ull) : "memory");
  }
}

// Units I and after of the thread from shared memory.
template <typename T, int V, int OWN, int L, int I = 0>
__device__ __forceinline__ void take_units(uint32_t from, Pair (&v)[OWN / 2]) {
  constexpr int kFirst = V * I / 2;
  if constexpr (sizeof(T) == 4) {
    asm volatile("ld.shared.v2.u64 {%0,%1}, [%2+%3];" : "=l"(v[kFirst % (OWN / 2)]), "=l"(v[(kFirst + 1) % (OWN / 2)]) : "r"(from), "n"(I * L * 16));
  } else if constexpr (V == 8) {
    uint32_t w[4];
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4+%5];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(from), "n"(I * L * 16));
#pragma unroll
    for (int j = 0; j < 4; ++j) v[(kFirst + j) % (OWN / 2)] = word_to_pair<T>(w[j]);
  } else {
    uint32_t w[2];
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2+%3];" : "=r"(w[0]), "=r"(w[1]) : "r"(from), "n"(I * L * 8));
    v[kFirst % (OWN / 2)] = word_to_pair<T>(w[0]);
    v[(kFirst + 1) % (OWN / 2)] = word_to_pair<T>(w[1]);
  }
  if constexpr (I + 1 < OWN / V) take_units<T, V, OWN, L, I + 1>(from, v);
}

// Takes a row that has landed at `src` (shared) into registers; columns that do not exist are zero.
template <typename T, int V, bool FULL, int OWN, int L>
__device__ __forceinline__ void take_row(uint32_t src, const T* row, uint32_t t, const Own<V, FULL, OWN, L>& own, Pair (&v)[OWN / 2]) {
  if constexpr (V > 2) {
    const uint32_t from = src + column_of<V, OWN, L>(t, 0) * (uint32_t)sizeof(T);
    take_units<T, V, OWN, L>(from, v);
  } else {
    const uint32_t from = src + t / L * (L * OWN * (uint32_t)sizeof(T) + 16) + (uint32_t)(reinterpret_cast<uintptr_t>(row) & 15) + V * (t % L) * (uint32_t)sizeof(T);
    // what lies where a column does not exist (it is inside the warp's space) is read and dropped
#pragma unroll
    for (int i = 0; i < OWN; i += 2) {
      float lo, hi;
      if constexpr (sizeof(T) == 4) {
        constexpr int kNext = V == 2 ? 4 : 4 * L;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(lo) : "r"(from + i / V * (L * V) * 4));
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(hi) : "r"(from + i / V * (L * V) * 4 + kNext));
      } else if constexpr (V == 2) {
        uint32_t w;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(from + i * L * 2));
        const float2 f = split(word_to_pair<T>(w));
        lo = f.x;
        hi = f.y;
      } else {
        uint16_t w0, w1;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w0) : "r"(from + i * L * 2));
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w1) : "r"(from + (i + 1) * L * 2));
        const float2 f = split(word_to_pair<T>(w0 | (uint32_t)w1 << 16));
        lo = f.x;
        hi = f.y;
      }
      v[i / 2] = FULL ? pair_of(lo, hi) : pair_of(own.has(i) ? lo : 0.0f, own.has(i + 1) ? hi : 0.0f);
    }
  }
}

template <typename T, int V, bool FULL, int OWN, int L>
__device__ __forceinline__ void store_row(T* row, uint32_t t, const Own<V, FULL, OWN, L>& own, const Pair (&v)[OWN / 2]) {
  T* to = row + column_of<V, OWN, L>(t, 0);
#pragma unroll
  for (int i = 0; i < OWN / V; ++i) {
    T* p = to + i * L * V;
    if (V == 2 && own.of(i) == 2) {
      if constexpr (sizeof(T) == 2) {
        st_c(reinterpret_cast<uint32_t*>(p), pair_to_word<T>(v[i % (OWN / 2)]));
      } else {
        const float2 f = split(v[i % (OWN / 2)]);
        st_c(p, from_float<T>(f.x));
        st_c(p + 1, from_float<T>(f.y));
      }
    } else if (V > 2 && own.of(i) == V) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < V / 2; ++j) {
        const Pair f = v[(V * i / 2 + j) % (OWN / 2)];
        if constexpr (sizeof(T) == 4) { w[(2 * j) % 4] = __float_as_uint(split(f).x); w[(2 * j + 1) % 4] = __float_as_uint(split(f).y); }
        else w[j % 4] = pair_to_word<T>(f);
      }
      if (V * sizeof(T) == 16) {
        if (bounds_ok(p, 16, true)) __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
      } else {
        if (bounds_ok(p, 8, true)) __stcs(reinterpret_cast<uint2*>(p), make_uint2(w[0], w[1]));
      }
    } else if (V == 1 || own.of(i) != 0) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float2 f = split(v[(V * i + j) / 2]);
        if (own.has(V * i + j)) st_c(p + j, from_float<T>((V * i + j) % 2 ? f.y : f.x));
      }
    }
  }
}

// Value c of gamma or beta, in whichever type it has.
__device__ __forceinline__ float weight_at(const void* w, int dtype, float absent, uint32_t c) {
  if (!w) return absent;
  if (dtype == kF32) return ld_c(static_cast<const float*>(w) + c);
  if (dtype == kBf16) return to_float(ld_c(static_cast<const __nv_bfloat16*>(w) + c));
  return to_float(ld_c(static_cast<const __half*>(w) + c));
}

// gamma or beta for this thread's columns: read once for all rows that it takes, all loads on their way at once.
template <typename T, int V, bool FULL, int OWN, int L>
__device__ __forceinline__ void load_weights_of(const T* w, bool whole, const Own<V, FULL, OWN, L>& own, float absent, uint32_t t, Pair (&v)[OWN / 2]) {
  w += column_of<V, OWN, L>(t, 0);
  if (V > 2 && FULL && whole) {
    uint4 raw[OWN * sizeof(T) / 16];
    constexpr int kEach = 16 / (int)sizeof(T), kOf = V >= kEach ? V / kEach : 1;  // values of a load, loads of a unit
    if constexpr (V >= kEach) {
#pragma unroll
      for (int i = 0; i < OWN / kEach; ++i) raw[i] = ld_c(reinterpret_cast<const uint4*>(w + i / kOf * (L * V) + i % kOf * kEach));
    } else {  // units of four 16-bit values
#pragma unroll
      for (int i = 0; i < OWN / V; i += 2) {
        const uint2 lo = ld_c(reinterpret_cast<const uint2*>(w + i * (L * V))), hi = ld_c(reinterpret_cast<const uint2*>(w + (i + 1) * (L * V)));
        raw[i / 2] = make_uint4(lo.x, lo.y, hi.x, hi.y);
      }
    }
#pragma unroll
    for (int i = 0; i < OWN / kEach; ++i) {
      if constexpr (sizeof(T) == 4) {
        v[2 * i] = pair_of(__uint_as_float(raw[i].x), __uint_as_float(raw[i].y));
        v[2 * i + 1] = pair_of(__uint_as_float(raw[i].z), __uint_as_float(raw[i].w));
      } else {
        v[4 * i] = word_to_pair<T>(raw[i].x);
        v[4 * i + 1] = word_to_pair<T>(raw[i].y);
        v[4 * i + 2] = word_to_pair<T>(raw[i].z);
        v[4 * i + 3] = word_to_pair<T>(raw[i].w);
      }
    }
  } else {
    T raw[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i)
      if (own.has(i)) raw[i] = ld_c(w + i / V * (L * V) + i % V);
#pragma unroll
    for (int i = 0; i < OWN; i += 2) v[i / 2] = pair_of(own.has(i) ? to_float(raw[i]) : absent, own.has(i + 1) ? to_float(raw[i + 1]) : absent);
  }
}
template <int V, bool FULL, int OWN, int L, typename Args>  // Args: dtype_w and whole_weights say how w lies
__device__ __forceinline__ void load_weights(const Args& a, const void* w, const Own<V, FULL, OWN, L>& own, float absent, uint32_t t, Pair (&v)[OWN / 2]) {
  if (!w) {
#pragma unroll
    for (int i = 0; i < OWN / 2; ++i) v[i] = both(absent);
  } else if (a.dtype_w == kF32) {
    load_weights_of<float, V, FULL, OWN, L>(static_cast<const float*>(w), a.whole_weights, own, absent, t, v);
  } else if (a.dtype_w == kBf16) {
    load_weights_of<__nv_bfloat16, V, FULL, OWN, L>(static_cast<const __nv_bfloat16*>(w), a.whole_weights, own, absent, t, v);
  } else {
    load_weights_of<__half, V, FULL, OWN, L>(static_cast<const __half*>(w), a.whole_weights, own, absent, t, v);
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// The threads that share a row, one of the block's groups: `warps` warps (L = 32), or eight lanes of a warp (L = 8).
template <int L>
struct Group {
  uint32_t index, warps, threads, t, mask;  // mask: the lanes that take part in an exchange
  __device__ __forceinline__ explicit Group(uint32_t warps_) : warps(warps_), threads(L * warps_) {
    index = L == 32 ? (threadIdx.x >> 5) / warps : threadIdx.x / L;
    t = threadIdx.x - index * threads;
    mask = L == 32 ? 0xffffffffu : ((1u << L % 32) - 1) << (threadIdx.x & 31 & ~(L - 1));
  }
  __device__ __forceinline__ void sync() const {
    if (L < 32 || warps == 1) __syncwarp(mask);
    else asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(threads) : "memory");
  }
  // Sum over the group.  `slot`: 16 floats of the group, zero past its warps, used in turn with others (a barrier lies
  // between two uses); every thread adds the warps' values up for itself.
  __device__ __forceinline__ float sum(float v, float* slot) const {
#pragma unroll
    for (int d = L / 2; d >= 1; d >>= 1) v += __shfl_xor_sync(mask, v, d);
    if (L < 32 || warps == 1) return v;
    if ((t & 31) == 0) slot[t >> 5] = v;
    sync();
    float4 s = *reinterpret_cast<const float4*>(slot);
#pragma unroll
    for (uint32_t w = 4; w < 16; w += 4) {
      if (w >= warps) break;
      const float4 m = *reinterpret_cast<const float4*>(slot + w);
      s.x += m.x; s.y += m.y; s.z += m.z; s.w += m.w;
    }
    return (s.x + s.y) + (s.z + s.w);
  }
  // Two sums with one barrier: after the first exchange the lower half of the lanes adds up one of them, the upper half the
  // other.  `slot`: 32 floats, pairs of both.
  __device__ __forceinline__ float2 sum_two(float2 v, float* slot) const {
    constexpr int kHalf = L / 2;
    const bool upper = (t & kHalf) != 0;
    float mine = upper ? v.y : v.x;
    mine += __shfl_xor_sync(mask, upper ? v.x : v.y, kHalf);
#pragma unroll
    for (int d = kHalf / 2; d >= 1; d >>= 1) mine += __shfl_xor_sync(mask, mine, d);
    if (L < 32 || warps == 1) {
      const float other = __shfl_xor_sync(mask, mine, kHalf);
      return upper ? make_float2(other, mine) : make_float2(mine, other);
    }
    if ((t & 15) == 0) slot[t >> 4] = mine;
    sync();
    float4 s = *reinterpret_cast<const float4*>(slot);
#pragma unroll
    for (uint32_t w = 2; w < 16; w += 2) {
      if (w >= warps) break;
      const float4 m = *reinterpret_cast<const float4*>(slot + 2 * w);
      s.x += m.x; s.y += m.y; s.z += m.z; s.w += m.w;
    }
    return make_float2(s.x + s.z, s.y + s.w);
  }
};

constexpr int kMostGroups = 8;  // of several warps

}  // namespace accept
