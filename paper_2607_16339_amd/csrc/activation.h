// Activations of the bf16 projections, in fp32.
#pragma once

#include "device.h"
#include "lacache.h"

namespace lacache {

// exp(-x) and 1 / x by the hardware's exp2 and reciprocal (1 ulp each).
__device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(x * -1.44269504088896341f); }
__device__ __forceinline__ float silu(float x) { return x * fast_rcp(1.0f + exp_neg(x)); }
// gelu(x) = x Phi(x), Phi(x) = erfc(-x / sqrt 2) / 2, with erfc(z), z >= 0, by formula
// 7.1.26 of Abramowitz and Stegun (t = 1 / (1 + 0.3275911 z), t times a polynomial of
// degree 4 in t, times exp(-z^2)): 13 instructions where the library's erfc takes several
// times that, and it is applied to every output. The formula is off by at most 1.5e-7,
// so gelu by 0.75e-7 |x|; its steps in fp32 add up to 6.9e-7 |x| (the polynomial's
// partial sums and the reciprocal's error are as large as erfc). Found: 4.1e-7 |x|. In
// the far negative tail the formula's relative error grows: 4e-3 of gelu(x) at x = -6.
__device__ __forceinline__ float gelu(float x) {
  const float z = __builtin_fabsf(x) * 0.70710678118654752f;
  const float t = fast_rcp(__builtin_fmaf(0.3275911f, z, 1.0f));
  float p = __builtin_fmaf(1.061405429f, t, -1.453152027f);
  p = __builtin_fmaf(p, t, 1.421413741f);
  p = __builtin_fmaf(p, t, -0.284496736f);
  p = __builtin_fmaf(p, t, 0.254829592f);
  const float e = 0.5f * p * t * exp_neg(z * z);  // erfc(z) / 2
  return x * (x >= 0.0f ? 1.0f - e : e);
}
// 0.5 x (1 + tanh u) = x / (1 + exp(-2 u)), u = sqrt(2 / pi) (x + 0.044715 x^3)
__device__ __forceinline__ float gelu_tanh(float x) {
  const float u = 1.5957691216057308f * __builtin_fmaf(0.044715f * x * x, x, x);
  return x * fast_rcp(1.0f + exp_neg(u));
}
// N values at once (act is the same for the whole call).
template <int N>
__device__ __forceinline__ void activate(int act, float (&v)[N]) {
  switch (act) {
    case LACACHE_ACT_RELU:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];
      break;
    case LACACHE_ACT_SILU:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = silu(v[i]);
      break;
    case LACACHE_ACT_GELU:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = gelu(v[i]);
      break;
    case LACACHE_ACT_GELU_TANH:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = gelu_tanh(v[i]);
      break;
    default: break;
  }
}

// What follows a sum: the bias before the activation, the residual after it.
struct ActArgs {
  const uint16_t* bias;      // [weight rows], nullable
  const uint16_t* residual;  // [M x columns], nullable; may be the output
  int act;                   // a LACACHE_ACT_ value
};

}  // namespace lacache
