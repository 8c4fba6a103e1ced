// What the attention kernels share: operand types, conversions, the bounds of a weight.
#pragma once

#include "tq_device.hpp"

namespace tq {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef uint16_t s2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef const int32_t __attribute__((address_space(4))) const_i32;

constexpr float kLog2e = 1.4426950408889634f;

// The largest weight that a step may have (fp16's largest value), and the power of two at
// which the largest one is put when the reference moves.
constexpr float kTopWeight = 65504.0f, kHeadroom = 12.0f;
// With bf16 rows, whose values fp32 itself just holds, the weights of a range of fewer than
// 2^e tokens stay at 2^-e or below, so that no sum passes the largest value; the largest
// weight is put kBelow binades lower.
constexpr int kBelow = 8;
constexpr float kLeastScale = 0x1p-24f;    // fp16's smallest number

// four e4m3 bytes times `scale` (a power of two) as two words of 16-bit values
template <bool BF16>
__device__ __forceinline__ void widen4(uint32_t w, float scale, uint32_t &lo, uint32_t &hi) {
  if constexpr (BF16) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
  } else {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true));
  }
}

// two fp32 values rounded to a word of 16-bit ones
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const f2 v = {x, y};
  if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, h2));
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Scores under a cap, in binades: cap tanh x = cap (1 - 2 / (e^2x + 1)), good to 2^-22 of the
// cap.  `in` turns a product of a query and a key into the exponent, log2(e) 2 x.
struct Shape {
  float in, out;
};
__device__ __forceinline__ Shape shape_of(float scale, float cap, float unit) {
  return {cap > 0.0f ? 2.0f * kLog2e * (fabsf(scale) / cap) * unit : 0.0f, cap * kLog2e};
}
__device__ __forceinline__ float capped(float product, const Shape &s) {
  return fmaf(__builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(product * s.in) + 1.0f), -2.0f * s.out, s.out);
}

// log-sum-exp in natural units from the reference m and the sum l of exp2(score - m)
// (m and l's binade all but cancel: they go together first)
__device__ __forceinline__ float log_sum(float m, float l) {
  return (m + (float)__builtin_amdgcn_frexp_expf(l) + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(l))) * (1.0f / kLog2e);
}

}  // namespace tq
