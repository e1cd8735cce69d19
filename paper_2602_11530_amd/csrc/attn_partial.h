// Partial attention results of one query row: what the stream pass and the reduce pass fold
// together (reference maximum in log2 units, partial sum, un-normalised row).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pkv {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kNegInf = -__builtin_huge_valf();
// A reference maximum before any score.  Finite, so that weights of minus infinity are zeros, those of what is masked and those of infinite keys; a result
// that has seen tokens keeps at least this, one that has not has minus infinity.
constexpr float kLeast = -3e38f;

// Two fp32 -> packed bf16, round to nearest even (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const f32x2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}
// A row's partial result while records are folded into it.
struct Partial {
  float m, l;
  f32x4 x;
};
constexpr Partial kNothing = {kNegInf, 0.f, {0.f, 0.f, 0.f, 0.f}};
constexpr f32x2 kNoStats = {kNegInf, 0.f};   // of a result that is not there

// Folds kN partial results into p: one common maximum first, so that the weights do not wait for
// each other.  A side whose sum is exactly zero has seen nothing and is left out, whatever its row holds.  Every other one
// counts, also with a weight of zero: one whose scores were all NaN has a sum of NaN and no maximum, and a NaN among values
// that weigh nothing makes a NaN of the whole.
template <int kN>
__device__ __forceinline__ void fold(Partial& p, const f32x2 (&ml)[kN], const f32x4 (&x)[kN]) {
  float M = p.m;
#pragma unroll
  for (int z = 0; z < kN; ++z) M = fmaxf(M, ml[z].x);
  const float w = __builtin_amdgcn_exp2f(p.m - M);   // NaN where both are -inf: then the sum is zero or NaN
  const bool some = p.l != 0.f;
  p.m = M;
  p.l = some ? w * p.l : 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) p.x[e] = some ? w * p.x[e] : 0.f;
#pragma unroll
  for (int z = 0; z < kN; ++z) {
    const float wz = __builtin_amdgcn_exp2f(ml[z].x - M);
    const bool there = ml[z].y != 0.f;
    p.l = there ? __builtin_fmaf(wz, ml[z].y, p.l) : p.l;
#pragma unroll
    for (int e = 0; e < 4; ++e) p.x[e] = there ? __builtin_fmaf(wz, x[z][e], p.x[e]) : p.x[e];
  }
}
// Normalise, scale and round once to bf16.
__device__ __forceinline__ u32x2 finish_row4(f32x4 x, float inv) {
  return u32x2{pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
}
// Zeros where nothing was seen.  Where none of the tokens that were seen has a weight, the row of zeros is multiplied by infinity, which is NaN: the quotient
// of two zeros.
__device__ __forceinline__ float inverse(float m, float l, float out_scale) {
  return m > kNegInf ? out_scale / l : 0.f;
}

}  // namespace pkv
