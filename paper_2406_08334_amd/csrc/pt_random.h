// Dropout from a counter: which elements of a row of an array are kept (splitmix64 of a counter: Steele, Lea, Flood, 2014).
#pragma once

#include "pt_common.h"

#include <cmath>

namespace pt_random {

constexpr uint64_t PHI = 0x9E3779B97F4A7C15ull;

__device__ __forceinline__ uint64_t mix64(uint64_t x) {
  x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9ull;
  x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
  return x ^ (x >> 31);
}

struct Drop {
  uint64_t seed;
  const uint64_t* step;
  uint32_t off;              // of 65536; 0: no dropout
  float scale;

  __device__ __forceinline__ uint64_t key() const { return off ? mix64(seed + (step ? *(const PT_GLOBAL uint64_t*)step : 0) * PHI) : 0; }
  // Element c (0 to 3) of the four that share word z: x scaled, or 0.
  __device__ __forceinline__ float of(uint64_t z, int c, float x) const { return (uint32_t(z >> (16 * c)) & 0xffffu) < off ? 0.0f : x * scale; }
  // Four elements whose word has the counter key + (word + 1) PHI.
  __device__ __forceinline__ void apply(uint64_t counter, float* x) const {
    const uint64_t z = mix64(counter);
#pragma unroll
    for (int c = 0; c < 4; ++c) x[c] = of(z, c, x[c]);
  }
};

inline bool valid(const pt_drop& d) { return d.p >= 0.0 && d.p < 1.0; }
inline Drop make(const pt_drop& d) {
  const uint32_t off = uint32_t(std::fmin(65535.0, std::nearbyint(d.p * 65536.0)));
  return {d.seed, d.step, off, float(65536.0 / (65536 - off))};
}

}  // namespace pt_random
