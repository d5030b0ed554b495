// Dropout numbers: which elements of a matrix are kept, from the codec's counter-based generator (accept_device.cuh).  The
// mask is a function of seed, counter and element, so a backward pass works it out again and nothing is stored.
#pragma once
#include "accept_types.cuh"

namespace accept {

// An element is kept where the upper 24 bits of its word are at least T = ceil(p 2^24): word > 256 T - 1 (T >= 1).
struct Drop {
  Rng rng;
  uint64_t offset;   // counter of element 0
  uint32_t limit;    // 256 T - 1
  float scale;       // 1 / (1 - p), of what is kept
  int on;            // p > 0
};

// What counters share while the upper 30 bits of the counter stay, and the next such.
struct DropKey {
  uint32_t high, key, next;
  __device__ __forceinline__ DropKey(const Rng& rng, uint64_t first) : high((uint32_t)(first >> 34)), key(rng.key(high)), next(rng.key((high + 1) & 0x3fffffffu)) {}
};

// The counters from `first` on, 2^33 of them at most; `known`: the keys of counters near by.
struct DropRow {
  uint32_t quad, key, next, phase;
  __device__ __forceinline__ DropRow(const Rng& rng, uint64_t first, const DropKey& known) {
    quad = (uint32_t)(first >> 2);
    key = known.key;
    next = known.next;
    if ((uint32_t)(first >> 34) != known.high) {
      const DropKey own(rng, first);
      key = own.key;
      next = own.next;
    }
    phase = (uint32_t)first & 3;
  }
  __device__ __forceinline__ uint32_t hash(uint32_t ahead) const {  // of the ahead-th quad
    const uint32_t q = quad + ahead;
    return Rng::quad_hash(q, q < quad ? next : key);
  }
};

__device__ __forceinline__ uint32_t lane_factor(uint32_t m) { return m == 0 ? 1u : m == 1 ? 0x9E3779B1u : m == 2 ? 0x85EBCA77u : 0xC2B2AE3Du; }

static __constant__ uint32_t kLaneFactors[8] = {1u, 0x9E3779B1u, 0x85EBCA77u, 0xC2B2AE3Du, 1u, 0x9E3779B1u, 0x85EBCA77u, 0xC2B2AE3Du};

// Random words of UNITS units of N neighbours (or their complements, NOT: ~(h M) = -h M - 1 costs nothing more), the first from the
// quad-th four columns on (columns themselves may pass 32 bits) and `step` columns apart (a multiple of four), for take(unit, words).  A hash
// serves four counters; where the row's counters do not start on a multiple of four, four columns take theirs from two hashes, split at
// the same place in the whole row.
template <int N, bool NOT, int UNITS, typename Take>
__device__ __forceinline__ void number_units(const DropRow& r, uint32_t quad, uint32_t step, const Take& take) {
  constexpr uint32_t kAdd = NOT ? 0xffffffffu : 0u;
  if (r.phase == 0) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      uint32_t w[N];
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        uint32_t h = r.hash(quad + u * (step / 4) + i / 4);
        if (NOT) h = 0u - h;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[i + e] = h * lane_factor(e) + kAdd;
      }
      take(u, w);
    }
  } else {
    uint32_t times[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) times[e] = kLaneFactors[r.phase + e];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      uint32_t w[N], h[N / 4 + 1];
#pragma unroll
      for (int i = 0; i <= N / 4; ++i) {
        h[i] = r.hash(quad + u * (step / 4) + i);
        if (NOT) h[i] = 0u - h[i];
      }
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = (r.phase + i % 4 >= 4 ? h[i / 4 + 1] : h[i / 4]) * times[i % 4] + kAdd;
      take(u, w);
    }
  }
}
// v / (1 - p) where kept, else 0.
template <int N>
__device__ __forceinline__ void drop_values(const Drop& d, const uint32_t (&w)[N], Pair* v) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const float2 f = split(mul2(v[i], both(d.scale)));
    v[i] = pair_of(w[2 * i] > d.limit ? f.x : 0.0f, w[2 * i + 1] > d.limit ? f.y : 0.0f);
  }
}
// UNITS units of N values each, the first from column `col` on, a multiple of four.
template <int N, int UNITS>
__device__ __forceinline__ void drop_units(const Drop& d, const DropRow& r, uint32_t col, uint32_t step, Pair* v) {
  number_units<N, false, UNITS>(r, col / 4, step, [&](int u, const uint32_t (&w)[N]) { drop_values<N>(d, w, v + u * (N / 2)); });
}

}  // namespace accept
