// Dropout whose mask is a function of counters, so that it is drawn again where it is needed and never stored:
// entry c of row r is kept iff half c mod 8 (the low half of word 0 first) of Philox4x32-10 of counter (c / 8, r, layer, step) is at least
// `threshold`; one call serves eight neighbours.  Key: the seed, its high word xored with a constant, so that the draws of a compressed step with the same seed
// are others.  Sixteen bits an entry: probabilities are multiples of 2^-16, and the scale is exactly the reciprocal of what is kept.
#pragma once
#include "dsq_internal.h"

namespace dsq {

struct Drop {
  PhiloxKeys keys;
  uint32_t threshold, layer, step;      // threshold 0: nothing is dropped
  float scale;
};
constexpr uint32_t kDropKey = 0x44524F50u;

inline Drop make_drop(uint32_t threshold, uint64_t seed, uint32_t layer, uint32_t step) {
  return {philox_key_schedule((uint32_t)seed, (uint32_t)(seed >> 32) ^ kDropKey), threshold, layer, step, (float)(65536.0 / (65536.0 - threshold))};
}

// Bit j: entry c + j of the row is kept (c a multiple of 8).
__device__ __forceinline__ uint32_t kept8(const Drop& d, uint32_t row, uint32_t c) {
  const uint4 r = philox4x32_10(make_uint4(c >> 3, row, d.layer, d.step), d.keys);
  const uint32_t top = d.threshold << 16;
  uint32_t m = 0;
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) m |= (uint32_t)(w[i] << 16 >= top) << (2 * i) | (uint32_t)(w[i] >= top) << (2 * i + 1);
  return m;
}
__device__ __forceinline__ void drop8(const Drop& d, uint32_t kept, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = kept >> j & 1 ? v[j] * d.scale : 0.f;
}

}  // namespace dsq
