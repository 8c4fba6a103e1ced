// What the attention kernels share: operand types, conversions, the bounds of a weight.
#pragma once

#include <cfloat>

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

// Scores under a cap, in binades: cap tanh x, where a product z of a query and a key has the score
// z * c before the cap and x = z * `x`.
//   |x| < 1/2: z c tanh(x) / x, a series in x^2 (fitted for the least relative error, 2^-26)
//   else cap (1 - 2 / (e^2x + 1)), whose difference cancels below that
// is good to 2^-20 of itself.  Caps up to 64 take the second everywhere, good to 2^-21 of the cap:
// no more than the sums in front of it leave a score off by.  (Both for them too: a prompt of 4096, 16
// / 4 heads of 64, 99 us for 86 while all scores are below half of the cap, 170 where some are not.)
constexpr float kWide = 64.0f;
struct Shape {
  float x, in, out, c;        // in: of e^2x as a power of two
};
__device__ __forceinline__ Shape shape_of(float scale, float cap, float c, float unit) {
  // (finite, so that a product of zero stays one)
  const float x = cap > 0.0f ? fminf(fabsf(scale) / cap * unit, 0x1p126f) : 0.0f;
  return {x, 2.0f * kLog2e * x, fminf(cap * kLog2e, FLT_MAX), c};
}
constexpr float kNear = 0.5f;
__device__ __forceinline__ float capped_near(float z, const Shape &s) {
  const float x = z * s.x, u = x * x, y = z * s.c;
  const float r = fmaf(fmaf(fmaf(0.01724149f, u, -0.05304549f), u, 0.13325879f), u, -0.33333144f);
  return fmaf(y, u * r, y);
}
// 1 / (e^2x + 1)
__device__ __forceinline__ float capped_rest(float z, const Shape &s) {
  return __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(z * s.in) + 1.0f);
}
// N scores, by at(i) and set(i, score); WIDE: of a cap past 64
template <int N, bool WIDE, typename At, typename Set>
__device__ __forceinline__ void cap_scores(At at, Set set, const Shape &s) {
  if constexpr (!WIDE) {
#pragma unroll
    for (int i = 0; i < N; i++) set(i, fmaf(capped_rest(at(i), s), -2.0f * s.out, s.out));
    return;
  }
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < N; i++) top = fmaxf(top, fabsf(at(i)));
  if (__any(!(top * s.x < kNear))) {
    // (2 out may pass fp32's range)
#pragma unroll
    for (int i = 0; i < N; i++)
      set(i, fabsf(at(i) * s.x) < kNear ? capped_near(at(i), s) : s.out * fmaf(capped_rest(at(i), s), -2.0f, 1.0f));
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) set(i, capped_near(at(i), s));
  }
}

// log-sum-exp in natural units from the reference m and the sum l of exp2(score - m)
// (m and l's binade all but cancel: they go together first)
__device__ __forceinline__ float log_sum(float m, float l) {
  return (m + (float)__builtin_amdgcn_frexp_expf(l) + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(l))) * (1.0f / kLog2e);
}

}  // namespace tq
