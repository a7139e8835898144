// The order of logits among the largest, and the bar that a piece's logits have to reach: what the join of the scores (gensor_lm.cpp) takes for one of
// the largest, and what the product (lm_kernel.hpp, Score) has stored.
#pragma once
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

namespace gensor {

// Score stores the logits of a set (a run of rows of a piece) only where the set's maximum is above the bar that earlier pieces have left for the token.
// The bar is NaN where they have left none: then all of them are stored.
__host__ __device__ inline bool set_is_stored(float set_max, float bar) { return !(set_max <= bar); }

// A logit and its entry as one number, the larger the earlier it is among the largest: the value's order in front, then the lower entry.  0: none.
__host__ __device__ inline uint64_t rank_key(float v, int entry) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.f);            // (minus zero is zero)
  return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)~entry;
}
__host__ __device__ inline float key_value(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __builtin_bit_cast(float, u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__host__ __device__ inline int key_entry(uint64_t key) { return (int)~(uint32_t)key; }

// The smallest number above a number (NaN above infinity, which no number reaches)
__host__ __device__ inline float next_above(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);
  return __builtin_bit_cast(float, u & 0x80000000u ? u - 1 : u + 1);
}

// The largest number of 20 bits that n values reach, so at or up to 2^-11 of its size below the n'th largest; minus infinity where there are fewer.
// reach(key): how many values' keys (the upper halves of rank_key) are `key` at least.
template <typename Reach>
__host__ __device__ __attribute__((always_inline)) inline float nth_reached(int n, Reach&& reach) {
  uint32_t found = 0;
#pragma unroll
  for (int bit = 31; bit >= 12; --bit) {
    const uint32_t higher = found | 1u << bit;
    if (reach(higher) >= n) found = higher;
  }
  return found > 0x007fffffu ? key_value((uint64_t)found << 32) : -INFINITY;
}

// What one of a piece's logits has to reach.  bar: the `top`'th largest so far, which it has to exceed, or NaN; enough: `top` of the piece's group maxima do
// that; nth(): nth_reached of those maxima, of which `top` logits are no smaller.  nth() is cut to fewer bits and may lie at or below the bar that the maxima
// themselves exceed.  But sets that are not above the bar have not been stored, so the result is above it always: a set whose maximum reaches it is one
// that set_is_stored.
template <typename Nth>
__host__ __device__ __attribute__((always_inline)) inline float least_wanted(float bar, bool enough, Nth&& nth) {
  const float above = next_above(bar);
  if (bar == bar && !enough) return above;
  const float least = nth();
  return bar == bar && !(least >= above) ? above : least;
}

}  // namespace gensor
