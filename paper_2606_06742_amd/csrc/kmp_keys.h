// Keys that order tokens by their logits (logprobs.hip, sample.hip).
#pragma once

#include "kmp_operators.h"

namespace kmp {

// Order of tokens (value descending, index ascending) as one unsigned number: the
// value's bits mapped to increasing order (NaN highest, -0 as 0) above the complemented
// index. No value has key 0.
typedef unsigned long long key_t;
__device__ __forceinline__ uint32_t value_key(float v) {
  if (v != v) return 0xFFFFFFFFu;
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return k == 0xFFFFFFFFu ? __builtin_nanf("") : __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ key_t key_of(float v, uint32_t index) { return (key_t)value_key(v) << 32 | (uint32_t)~index; }

}  // namespace kmp
