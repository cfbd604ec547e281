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

// The random words of entries c .. c + 7 of a row (c a multiple of 8).
__device__ __forceinline__ uint4 draw8(const Drop& d, uint32_t row, uint32_t c) { return philox4x32_10(make_uint4(c >> 3, row, d.layer, d.step), d.keys); }
// An entry's half in the upper half of a word against the threshold there: the lower half below it makes no difference.
__device__ __forceinline__ void drop8(const Drop& d, const uint4& r, float (&v)[8]) {
  const uint32_t top = d.threshold << 16, w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = w[i] << 16 >= top ? v[2 * i] * d.scale : 0.f;
    v[2 * i + 1] = w[i] >= top ? v[2 * i + 1] * d.scale : 0.f;
  }
}

}  // namespace dsq
