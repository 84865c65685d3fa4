// What the vocabulary layer's kernels share beside the contraction (gfx950, wave64).
#pragma once

#include "contraction.hpp"
#include "vocab.hpp"

namespace vtrace {
namespace {

constexpr float kLog2eF = 1.44269504088896340736f;

// Sums (or maxima) over the four lane groups, the same in all of them.
template <typename Op>
__device__ __forceinline__ float over_groups(float x, Op op) {
  const v2u p = __builtin_bit_cast(
      v2u, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  x = op(__uint_as_float(p.x), __uint_as_float(p.y));
  const v2u q = __builtin_bit_cast(
      v2u, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return op(__uint_as_float(q.x), __uint_as_float(q.y));
}
__device__ __forceinline__ float group_max(float x) {
  return over_groups(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float group_sum(float x) {
  return over_groups(x, [](float a, float b) { return a + b; });
}

// Where a token's logit starts: its bias.  Behind the vocabulary's end, and for a bias
// so low that the logit's scaling could overflow, the token is ruled out.  (A buffer without
// a bias is empty and reads 0.)
constexpr float kRuledOut = -1e37f;
__device__ __forceinline__ float start_of_logit(const VocabArgs& a, int64_t v) {
  const Rsrc bias = make_rsrc(a.bias, a.bias ? a.V * 4 : 0);
  const float b = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(bias, static_cast<uint32_t>(v) * 4, 0, 0));
  return v >= a.V || b < kRuledOut ? -INFINITY : b;
}
// A token ruled out adds p log p = 0, not 0 * -inf.
constexpr float kLeastLog = -1e30f;
// A logit's exponent about another one, in log2 units.  The difference comes first: scaled
// each for itself, logits near 1e10 (a finite mask's) round to hundreds of units off, and
// 2^hundreds overflows.
__device__ __forceinline__ float log2_ratio(float z, float about) { return (z - about) * kLog2eF; }
}  // namespace
}  // namespace vtrace
