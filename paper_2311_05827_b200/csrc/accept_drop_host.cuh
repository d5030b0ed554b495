// Host side of the dropout numbers: what a rate, a seed and a counter become for the kernels.
#pragma once
#include <cmath>

#include "accept_drop.cuh"
#include "accept_host.cuh"

namespace accept {

inline bool is_drop_rate(float p) { return p >= 0.0f && p <= 1.0f; }  // not NaN

// Kept: U >= p for U = r 2^-24, that is r >= T = ceil(p 2^24).  Everything is dropped where p = 1.
inline Drop drop_of(float p, uint64_t seed, uint64_t offset) {
  Drop d{};
  const uint32_t least = (uint32_t)std::ceil((double)p * 16777216.0);
  d.rng.seed_lo = (uint32_t)seed;
  d.rng.seed_hi = (uint32_t)(seed >> 32);
  d.offset = offset;
  d.limit = least * 256u - 1u;  // p = 1: 2^32 - 1, which no word is above
  d.scale = p < 1.0f ? (float)(1.0 / (1.0 - (double)p)) : 0.0f;
  d.on = p > 0.0f;
  return d;
}

}  // namespace accept
