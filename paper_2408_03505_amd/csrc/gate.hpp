// GELU, SiLU and their derivatives, for the epilogues of the MLP's and the gated
// feed-forward block's products.
#pragma once

#include "common.hpp"

namespace optimus {

// Phi(-|u|) = erfc(|u| / sqrt 2) / 2 for the GELU epilogues, from Abramowitz &
// Stegun, Handbook of Mathematical Functions (1964), formula 7.1.26: for
// x >= 0, erfc(x) = (a1 t + a2 t^2 + a3 t^3 + a4 t^4 + a5 t^5) e^(-x^2) with
// t = 1 / (1 + p x), absolute error <= 1.5e-7 (here halved, the halves taken
// into a1..a5 and 1 / sqrt 2 into p).  The tail is computed directly, so the
// negative side does not cancel in fp32.  On the hardware reciprocal and
// exponential this is a fraction of the library erff's instructions; the
// epilogue evaluates it for every output element and is bound by it (two
// quarter-rate instructions and a dozen others), and results are rounded to bf16.
// Also returns e^(-u^2 / 2), which GELU' needs as well.
__device__ __forceinline__ float phi_tail(float u, float &ex2) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678118654752f, fabsf(u), 1.0f));
  const float v = u * 0.84932180028801904f;  // sqrt(log2(e) / 2)
  ex2 = __builtin_amdgcn_exp2f(-(v * v));
  const float poly = fmaf(
      t, fmaf(t, fmaf(t, fmaf(t, 0.5f * 1.061405429f, -0.5f * 1.453152027f), 0.5f * 1.421413741f), -0.5f * 0.284496736f),
      0.5f * 0.254829592f);
  return poly * (t * ex2);
}

// GELU(u) = u Phi(u) and GELU'(u) = Phi(u) + u phi(u), with Phi(u) =
// 1 - Phi(-u) and phi(u) = e^(-u^2 / 2) / sqrt(2 pi).
__device__ __forceinline__ float gelu_f(float u) {
  float ex2;
  const float h = phi_tail(u, ex2);
  return u * (u >= 0.0f ? 1.0f - h : h);
}

__device__ __forceinline__ float gelu_grad_f(float u) {
  float ex2;
  const float h = phi_tail(u, ex2);
  return fmaf(u * 0.39894228040143268f, ex2, u >= 0.0f ? 1.0f - h : h);
}

// The gate's activation of a gated feed-forward block, and with its derivative:
// SiLU(g) = g s, SiLU'(g) = s (1 + g (1 - s)), s = 1 / (1 + e^-g), or GELU.
__device__ __forceinline__ float sigmoid_f(float g) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f));
}

__device__ __forceinline__ float gate_f(float g, int act) {
  if (act) return gelu_f(g);
  return g * sigmoid_f(g);
}

__device__ __forceinline__ float gate_grad_f(float g, int act, float &value) {
  if (act) {
    float ex2;
    const float h = phi_tail(g, ex2), phi = g >= 0.0f ? 1.0f - h : h;
    value = g * phi;
    return fmaf(g * 0.39894228040143268f, ex2, phi);
  }
  const float s = sigmoid_f(g);
  value = g * s;
  return s * fmaf(g, 1.0f - s, 1.0f);
}

}  // namespace optimus
