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

// Random word of any counter.
static __device__ __noinline__ uint32_t drop_word_far(uint32_t seed_lo, uint32_t seed_hi, uint64_t ctr) { return Rng{seed_lo, seed_hi}.word(ctr); }

// What counters share while the upper 30 bits of the counter stay.
struct DropKey {
  uint32_t high, key;
  __device__ __forceinline__ DropKey(const Rng& rng, uint64_t first) : high((uint32_t)(first >> 34)), key(rng.key(high)) {}
};

// The counters from `first` on, `span` of them at most; `known`: the key of counters near by.
struct DropRow {
  uint64_t first;
  uint32_t quad, key, phase;
  bool wraps;  // the low word of the quad index wraps inside: every element by itself
  __device__ __forceinline__ DropRow(const Rng& rng, uint64_t first_, uint32_t span, const DropKey& known) : first(first_) {
    const uint64_t q = first >> 2;
    quad = (uint32_t)q;
    key = known.key;
    if ((uint32_t)(q >> 32) != known.high) key = rng.key((uint32_t)(q >> 32));
    phase = (uint32_t)first & 3;
    wraps = quad > 0xffffffffu - (span / 4 + 2);
  }
  __device__ __forceinline__ uint32_t word(const Drop& d, uint32_t col) const {  // one element's
    if (wraps) return drop_word_far(d.rng.seed_lo, d.rng.seed_hi, first + col);
    const uint32_t at = phase + col, m = at & 3, h = Rng::quad_hash(quad + (at >> 2), key);
    return h * (m == 0 ? 1u : m == 1 ? 0x9E3779B1u : m == 2 ? 0x85EBCA77u : 0xC2B2AE3Du);
  }
};

// Random words of the N counters (or their complements, NOT: ~(h M) = -h M - 1 costs nothing more) from a multiple of four on: a hash
// serves four.
template <int N, bool NOT>
__device__ __forceinline__ void number_quads(uint32_t quad, uint32_t key, uint32_t (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    uint32_t h = Rng::quad_hash(quad + i / 4, key);
    if (NOT) h = 0u - h;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[i + e] = h * (e == 0 ? 1u : e == 1 ? 0x9E3779B1u : e == 2 ? 0x85EBCA77u : 0xC2B2AE3Du) + (NOT ? 0xffffffffu : 0u);
  }
}

// Those of UNITS units of N neighbours, the first from column `col` on and `step` columns apart (multiples of four), for take(unit, words).
// Where the row's counters do not start on a multiple of four, four columns take theirs from two hashes, split at the same place in
// the whole row.
template <int N, bool NOT, int UNITS, typename Take>
__device__ __forceinline__ void number_units(const Rng& rng, const DropRow& r, uint32_t col, uint32_t step, const Take& take) {
  constexpr uint32_t kAdd = NOT ? 0xffffffffu : 0u;
  if (r.wraps) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      uint32_t w[N];
#pragma unroll
      for (int e = 0; e < N; ++e) w[e] = drop_word_far(rng.seed_lo, rng.seed_hi, r.first + col + u * step + e) ^ kAdd;
      take(u, w);
    }
  } else if (r.phase == 0) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      uint32_t w[N];
      number_quads<N, NOT>(r.quad + (col + u * step) / 4, r.key, w);
      take(u, w);
    }
  } else {
    uint32_t times[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t m = (r.phase + e) & 3;
      times[e] = m == 0 ? 1u : m == 1 ? 0x9E3779B1u : m == 2 ? 0x85EBCA77u : 0xC2B2AE3Du;
    }
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      uint32_t w[N], h[N / 4 + 1];
#pragma unroll
      for (int i = 0; i <= N / 4; ++i) {
        h[i] = Rng::quad_hash(r.quad + (col + u * step) / 4 + i, r.key);
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
// UNITS units of N values each, as above.
template <int N, int UNITS>
__device__ __forceinline__ void drop_units(const Drop& d, const DropRow& r, uint32_t col, uint32_t step, Pair* v) {
  number_units<N, false, UNITS>(d.rng, r, col, step, [&](int u, const uint32_t (&w)[N]) { drop_values<N>(d, w, v + u * (N / 2)); });
}

}  // namespace accept
