// What the differential attention kernels share (device code): tile swizzles, operand
// conversions, and the difference of the two maps with its norm.
//
//   out_h = ((softmax(c q1 K1^T) - lam_h softmax(c q2 K2^T)) [Va | Vb]) [/ rms * weight] * after
//
// Key heads 2 j and 2 j + 1 of a pool are the keys of pair j's two maps, value heads 2 j
// and 2 j + 1 the halves of its 2 D-wide value; query heads 2 h and 2 h + 1 are those of
// query pair h, which uses pair h / G.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../cw_internal.h"

namespace cw {
namespace diff {

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

constexpr float kNegBig = -1.0e30f;
// A half-row weight sum above this (or not finite) makes a block raise the running max:
// weights then stay below 2^16 and fp32 accumulators far from overflow.
constexpr float kSumLimit = 65536.f;

__device__ __forceinline__ int swap_bits_2_3(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

// The running max is set this much (in log2 units) below a row's largest score, so that fp16
// weights down to 2^-22 of the largest are normal numbers (where a few keys take most of
// the weight and many share the rest).
constexpr float kHeadroom = 8.f;

// Sum / maximum of a value over the two lanes (l and l + 32) that hold a row.
__device__ __forceinline__ float row_sum(float x) {
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}
__device__ __forceinline__ float row_max(float x) {
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}

// What a row's values are multiplied with after the difference: out_scale, and with a
// norm 1 / sqrt(mean + eps) of its 2 D values, whose squares sum to ss.
__device__ __forceinline__ float row_factor(const DiffParams& p, float ss, int head_dim) {
  return p.weight == nullptr ? p.out_scale : p.out_scale / sqrtf(ss / static_cast<float>(2 * head_dim) + p.eps);
}

// Stores a row's values (element 4 q4 + e of block b: dim 32 b + 8 q4 + 4 h + e) with the
// norm: `o` holds the differences.
template <int VB>
__device__ __forceinline__ void store_row(const DiffParams& p, uint16_t* row, int h, const f32x16 (&o)[VB]) {
  float ss = 0.f;
#pragma unroll
  for (int b = 0; b < VB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) ss = fmaf(o[b][i], o[b][i], ss);
  const float f = row_factor(p, row_sum(ss), 16 * VB);
#pragma unroll
  for (int b = 0; b < VB; ++b) {
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const int d = 32 * b + 8 * q4 + 4 * h;
      f32x4 w = {1.f, 1.f, 1.f, 1.f};
      if (p.weight != nullptr) w = *reinterpret_cast<const f32x4*>(p.weight + d);
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = static_cast<__bf16>(o[b][4 * q4 + e] * f * w[e]);
      *reinterpret_cast<u32x2*>(row + d) = __builtin_bit_cast(u32x2, v);
    }
  }
}

}  // namespace diff
}  // namespace cw
