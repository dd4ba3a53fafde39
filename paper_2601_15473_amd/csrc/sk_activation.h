// The activations of the dense layers and their derivatives, in fp32.
#pragma once
#include "sk_common.h"

namespace sk {

enum Activation : int { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4, ACT_COUNT = 5 };

// The normal distribution's Phi(-a) for a >= 0 and exp(-a^2 / 2): their quotient, erfcx(a / sqrt 2) / 2, is smooth and falls like 1 / a, here a polynomial
// in t = 1 / (1 + p a) without a constant, fitted to it over 0 .. 14 for the least relative error: 4.6e-6 at degree 6 (4.9e-6 as evaluated), far below a
// rounding to bf16, 1.5e-7 at degree 8 (4.3e-7).  Phi has that and the exponential's, whose argument is rounded: with degree 8 1.5e-6 of itself up to a = 5, 8e-6 at 12, where Phi is 1e-33.
// One exponential serves value and derivative.
template <bool PRECISE>
__device__ __forceinline__ float phi_below(float a, float& bell) {
  bell = __builtin_amdgcn_exp2f(a * a * -0.72134752044f);
  float t, q;
  if constexpr (PRECISE) {
    t = 1.f / (1.f + 0.3f * a);
    q = 0.0356747359f;
    q = fmaf(q, t, -0.157202899f);
    q = fmaf(q, t, 0.206353143f);
    q = fmaf(q, t, -0.053683307f);
    q = fmaf(q, t, 0.128561452f);
    q = fmaf(q, t, 0.0999135524f);
    q = fmaf(q, t, 0.120753951f);
    q = fmaf(q, t, 0.119629301f);
  } else {
    t = __builtin_amdgcn_rcpf(1.f + 0.31f * a);
    q = -0.0739290193f;
    q = fmaf(q, t, 0.180450007f);
    q = fmaf(q, t, 0.0157450773f);
    q = fmaf(q, t, 0.133429602f);
    q = fmaf(q, t, 0.120441318f);
    q = fmaf(q, t, 0.123860702f);
  }
  return q * t * bell;
}
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.4426950409f)); }
// ... and what it leaves to 1 (where that is little, not as a difference from 1)
__device__ __forceinline__ float logistic(float x, float& rest) {
  const float e = __builtin_amdgcn_exp2f(x * -1.4426950409f), p = __builtin_amdgcn_rcpf(1.f + e);
  rest = x > 0.f ? e * p : 1.f - p;
  return p;
}
// z / 2 (1 + tanh u) = z / (1 + exp(-2 u)), u = sqrt(2 / pi) (z + 0.044715 z^3): 2 u and its slope; past 100 (where the gate is 0 or 1) they stay what they are there
__device__ __forceinline__ float tanh_argument(float z, float& slope) {
  const float c = fminf(fmaxf(z, -100.f), 100.f), cc = c * c;
  slope = fmaf(0.2140644488f, cc, 1.5957691216f);
  return c * fmaf(0.0713548162726f, cc, 1.5957691216f);
}

template <int ACT, bool PRECISE>
__device__ __forceinline__ float activation(float z) {
  if constexpr (ACT == ACT_RELU) return z < 0.f ? 0.f : z;      // (NaN stays)
  if constexpr (ACT == ACT_GELU) {
    float bell;
    const float h = phi_below<PRECISE>(fabsf(z), bell);
    return z * (z < 0.f ? h : 1.f - h);
  }
  if constexpr (ACT == ACT_GELU_TANH) {
    float slope;
    return z * logistic(tanh_argument(z, slope));
  }
  if constexpr (ACT == ACT_SILU) return z * logistic(z);
  return z;
}
// ... by a number that is the same in all lanes, where an activation is not worth a kernel
template <bool PRECISE>
__device__ __forceinline__ float activation(int act, float z) {
  switch (act) {
    case ACT_RELU: return activation<ACT_RELU, PRECISE>(z);
    case ACT_GELU: return activation<ACT_GELU, PRECISE>(z);
    case ACT_GELU_TANH: return activation<ACT_GELU_TANH, PRECISE>(z);
    case ACT_SILU: return activation<ACT_SILU, PRECISE>(z);
    default: return z;
  }
}
template <int ACT, bool PRECISE>
__device__ __forceinline__ float activation_slope(float z) {
  if constexpr (ACT == ACT_RELU) return z <= 0.f ? 0.f : 1.f;
  if constexpr (ACT == ACT_GELU) {
    float bell;
    const float h = phi_below<PRECISE>(fabsf(z), bell);
    return (z < 0.f ? h : 1.f - h) + z * bell * 0.3989422804f;
  }
  if constexpr (ACT == ACT_GELU_TANH) {
    float slope, rest;
    const float u = tanh_argument(z, slope), p = logistic(u, rest);
    return p + z * (p * rest * slope);
  }
  if constexpr (ACT == ACT_SILU) {
    float rest;
    const float p = logistic(z, rest);
    return p * (1.f + z * rest);
  }
  return 1.f;
}

}  // namespace sk
