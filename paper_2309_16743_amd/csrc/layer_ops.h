// Activations of the layers (include/layers.h) with their derivatives, and what the
// matrix products take for a dense layer (dense.hip).
#pragma once

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

// NaN stays NaN.  Phi(z) = erfc(-z / sqrt 2) / 2, which keeps its digits in the lower
// tail where 1 + erf would cancel.
__device__ __forceinline__ float act_value(float z, int act) {
  if (act == kActRelu) return z < 0.f ? 0.f : z;
  if (act == kActSilu) return z / (1.f + expf(-z));
  if (act == kActGelu) return 0.5f * z * erfcf(-0.70710678118654752f * z);
  return z;
}

__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == kActRelu) return z > 0.f ? 1.f : 0.f;
  if (act == kActSilu) {
    const float s = 1.f / (1.f + expf(-z));
    return s * (1.f + z * (1.f - s));
  }
  if (act == kActGelu)
    return 0.5f * erfcf(-0.70710678118654752f * z) + z * (0.39894228040143268f * expf(-0.5f * z * z));
  return 1.f;
}

// dy act'(z).  relu: a choice and no product, so that a dropped infinity leaves no NaN.
__device__ __forceinline__ float act_back(float dy, float z, int act) {
  if (act == kActNone) return dy;
  if (act == kActRelu) return z > 0.f ? dy : 0.f;
  return dy * act_slope(z, act);
}

}  // namespace ot
