// What the kernels of attention with shaped scores share (device code): operand types, row
// reductions over the two lanes that hold a row, and the exponent of a score.
//
//   x_j = scale q k_j;  with a cap: x_j <- cap tanh(x_j / cap);  x_j <- x_j - slope_h |p - j|
//   key j counts where lo <= j < lim:  lo the larger of the token's first visible position and
//   p - window + 1, lim the larger of p + 1 and the length of the sequence's prefix mask
//   out = sum_j w_j v_j / sum_j w_j, w_j = 2^(x_j log2 e - m)
//
// tanh(u) = 1 - 2 / (1 + e^2u), so the capped exponent is cap2 - 2 cap2 / (1 + 2^(s c)) with cap2 =
// cap log2 e and c = 2 scale log2 e / cap: two transcendentals and one fma that also takes the
// bias and the running max.  Its error is absolute, some 2^-22 of the cap (1.2e-5 at 50), and
// both ends saturate without a case: 2^(s c) overflows to inf, whose reciprocal is 0.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../cw_internal.h"

namespace cw {
namespace shaped {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
// The running max of a row that has seen no key.
constexpr float kNegBig = -1.0e30f;
// A half-row weight sum above this (or not finite) makes a block raise the running max:
// weights then stay below 2^16 and fp32 accumulators far from overflow.
constexpr float kSumLimit = 65536.f;
// The running max is set this much (in log2 units) below a row's largest score, so that fp16
// weights down to 2^-22 of the largest are normal numbers.
constexpr float kHeadroom = 8.f;

__device__ __forceinline__ int swap_bits_2_3(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

// Sum / maximum of a value over the two lanes (l and l + 32) that hold a row.
__device__ __forceinline__ float row_sum(float x) {
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}
__device__ __forceinline__ float row_max(float x) {
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}

// The exponent of a score s (times c), given its bias less the running max.
template <bool CAP>
__device__ __forceinline__ float exponent(float s, float c, float cap2, float bias) {
  if constexpr (CAP)
    return fmaf(__builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(s * c)), -2.f * cap2, cap2 + bias);
  else
    return fmaf(s, c, bias);
}

// How far a block raises a row's running max.  An exponent is held to some 2^-22 of the score and the bias
// that are in it, which from about 2^26 on is more than kHeadroom: taken against the largest exponent as
// it came out against m = 0, none need come out near 0, and the weights would overflow or all vanish.  So
// that one gives the new max roughly (`near`), and where the exponents against `near` are off, the largest of
// them is taken out of them once more (`settle`): the row's largest weight is then in [2^kHeadroom,
// 2^(kHeadroom + 1)) whatever was rounded before.  What comes in is rounded down to whole numbers, and m stays
// one.  (A row that sees none of the keys has -inf, and keeps its max.)
struct RunningMax {
  float near, from;
  __device__ __forceinline__ RunningMax(float m_run, float top) : near(fmaxf(top - kHeadroom, m_run)), from(kHeadroom) {}
  // `top`: the largest exponent against `near`.  (The max never falls.)
  __device__ __forceinline__ void settle(float m_run, float top) { from = fmaxf(top, m_run - near + kHeadroom); }
  // An exponent against `near`, against the settled max.
  __device__ __forceinline__ float exponent(float f) const { return f - from + kHeadroom; }
  // Raises m_run and returns the factor of what was summed against the old one.
  __device__ __forceinline__ float raise(float& m_run) const {
    const float m = fmaxf(near + (from - kHeadroom), m_run);
    const float alpha = __builtin_amdgcn_exp2f(m_run - m);
    m_run = m;
    return alpha;
  }
};

}  // namespace shaped
}  // namespace cw
