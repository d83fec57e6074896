// Activations of the layers (include/layers.h) with their derivatives, and what the
// matrix products take for a dense layer (dense.hip).
#pragma once

#include <type_traits>

#include "common.h"

namespace ot {

// A dense layer's epilogue: C = act(acc + bias) + residual.
struct LayerArgs {
  const void* residual;     // C's type (nullable)
  int64_t ldr;
  void* pre;                // receives acc + bias in the operands' type (nullable)
  int64_t ldp;
  int32_t act;              // OT_ACT_*
  int32_t planes;           // bf16: A is the sum of so many matrices, plane_stride elements apart
  int64_t plane_stride;
};

constexpr int kActNone = 0, kActRelu = 1, kActSilu = 2, kActGelu = 3;

// exp(x + lo) for |lo| far below |x|: the exponent's rounding is put right by a first-order term.
__device__ __forceinline__ float act_exp(float x, float lo = 0.f) {
  const float t = x * 1.44269504088896341f;
  const float rest = fmaf(x, 1.44269504088896341f, -t) + fmaf(x, 1.925963033500011e-8f, lo * 1.44269504088896341f);
  const float e = __builtin_amdgcn_exp2f(t);
  return fabsf(t) < 126.f ? fmaf(e, 0.69314718055994531f * rest, e) : e;   // (also where x is infinite)
}
__device__ __forceinline__ float act_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + act_exp(-z)); }

// The normal distribution's integral Phi(z) = erfc(-z / sqrt 2) / 2 and e = exp(-z^2 / 2).  With t = |z| / sqrt 2
// and s = 1 / (1 + 0.3 t), exp(t^2) erfc(t) / s is a polynomial of degree 8 in s to 2e-8 of its value for t up to
// 10.5 (coefficients by iterated least squares against 64-bit values); past that e is 0.  z Phi(z) is off by at most
// 9.8 units of 2^-24 of its value in 3 x 10^8 values of -12.5 .. 12.5, the lower tail included, where 1 + erf would cancel.
__device__ __forceinline__ float act_phi(float z, float& e) {
  const float q = z * z;
  e = act_exp(-0.5f * q, -0.5f * fmaf(z, z, -q));
  const float s = __builtin_amdgcn_rcpf(fmaf(0.21213203435596426f, fabsf(z), 1.f));
  float p = -0.12955424189567566f;
  p = fmaf(p, s, 0.4857277274131775f);
  p = fmaf(p, s, -0.5126484036445618f);
  p = fmaf(p, s, 0.5481860637664795f);
  p = fmaf(p, s, -0.09500878304243088f);
  p = fmaf(p, s, 0.21509777009487152f);
  p = fmaf(p, s, 0.1482890546321869f);
  p = fmaf(p, s, 0.1707233488559723f);
  p = fmaf(p, s, 0.16918744146823883f);
  const float h = 0.5f * e * (s * p);
  return z > 0.f ? 1.f - h : h;
}

// NaN stays NaN.
template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if constexpr (ACT == kActRelu) return z < 0.f ? 0.f : z;
  if constexpr (ACT == kActSilu) return z * act_sigmoid(z);
  if constexpr (ACT == kActGelu) {
    float e;
    return z * act_phi(z, e);
  }
  return z;
}

// dy act'(z).  relu: a choice and no product, so that a dropped infinity leaves no NaN.
template <int ACT>
__device__ __forceinline__ float act_back(float dy, float z) {
  if constexpr (ACT == kActRelu) return z > 0.f ? dy : 0.f;
  if constexpr (ACT == kActSilu) {
    const float s = act_sigmoid(z);
    return dy * (s * fmaf(z, 1.f - s, 1.f));
  }
  if constexpr (ACT == kActGelu) {
    float e;
    const float phi = act_phi(z, e);
    return dy * fmaf(z, 0.39894228040143268f * e, phi);
  }
  return dy;
}

// The activation of N values (the same for all lanes), one choice for all of them.
template <int N, class V>
__device__ __forceinline__ void act_values(V& v, int act) {
  if (act == kActRelu) {
#pragma unroll
    for (int c = 0; c < N; ++c) v[c] = act_value<kActRelu>(v[c]);
  } else if (act == kActSilu) {
#pragma unroll
    for (int c = 0; c < N; ++c) v[c] = act_value<kActSilu>(v[c]);
  } else if (act == kActGelu) {
#pragma unroll
    for (int c = 0; c < N; ++c) v[c] = act_value<kActGelu>(v[c]);
  }
}

#ifdef __HIPCC__
// f(std::integral_constant<int, act>()).
template <class F>
void with_act(int act, F f) {
  switch (act) {
    case kActNone: f(std::integral_constant<int, kActNone>()); break;
    case kActRelu: f(std::integral_constant<int, kActRelu>()); break;
    case kActSilu: f(std::integral_constant<int, kActSilu>()); break;
    default: f(std::integral_constant<int, kActGelu>()); break;
  }
}
#endif

}  // namespace ot
