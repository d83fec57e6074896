// 8 values of a row of a matrix whose rows are padded to whole 16-byte pieces, as fp32, and the thread layout
// of kernels that walk such rows.
#pragma once

#include "lowrank_ops.h"

namespace ot {

// Values p[0 .. 7], zeros from `left` on.
__device__ __forceinline__ void load8(const uint16_t* p, int64_t left, float (&v)[8]) {
  const lr_u32x4 q = lr_load16(p, left);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    v[2 * w] = __uint_as_float(q[w] << 16);
    v[2 * w + 1] = __uint_as_float(q[w] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, int64_t left, float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const lr_u32x4 q = lr_load16(p + 4 * h, left - 4 * h);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * h + e] = __uint_as_float(q[e]);
  }
}

// The first min(left, 8) of them to p, rounded to nearest even.
__device__ __forceinline__ void store8(uint16_t* p, int64_t left, const float (&v)[8]) {
  if (left >= 8) {
    lr_u32x4 t;
#pragma unroll
    for (int q = 0; q < 4; ++q) t[q] = (uint32_t)lr_bf16(v[2 * q]) | ((uint32_t)lr_bf16(v[2 * q + 1]) << 16);
    *reinterpret_cast<lr_u32x4*>(p) = t;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e] = lr_bf16(v[e]);
  }
}
__device__ __forceinline__ void store8(float* p, int64_t left, const float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (left >= 4 * h + 4) *reinterpret_cast<f32x4*>(p + 4 * h) = f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
    else
#pragma unroll
      for (int e = 4 * h; e < 4 * h + 4; ++e)
        if (e < left) p[e] = v[e];
  }
}

// a / b and a - a / b * b of numbers that mostly fit 32 bits (a 64-bit division takes a hundred instructions).
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b, int64_t& rest) {
  if (((a | b) >> 32) == 0) {
    const uint32_t q = (uint32_t)a / (uint32_t)b;
    rest = (uint32_t)a - q * (uint32_t)b;
    return q;
  }
  const int64_t q = a / b;
  rest = a - q * b;
  return q;
}

// A thread's rows r, r + step, .. below end in groups of U: load(slot, row) of a whole group comes before
// use(slot, row), since the compiler keeps loads behind stores that may alias them.
template <int U, class Load, class Use>
__device__ __forceinline__ void rows_in_groups(int64_t r, int64_t end, int64_t step, Load load, Use use) {
  for (; r + (U - 1) * step < end; r += U * step) {
#pragma unroll
    for (int u = 0; u < U; ++u) load(u, r + u * step);
#pragma unroll
    for (int u = 0; u < U; ++u) use(u, r + u * step);
  }
  for (; r < end; r += step) {
    load(0, r);
    use(0, r);
  }
}

}  // namespace ot
