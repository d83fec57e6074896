// What the matrix products take for low-rank adapters (adapters.hip), and device
// helpers of the low-rank products: values of 16 or 32 bits, 16-byte
// pieces with a ragged end, and fp32 values as sums of bf16 terms.
#pragma once

#include "common.h"

namespace ot {

// Sorted rows of a batch and their adapters (adapters.hip).
struct AdaptRows {
  const int32_t* perm;      // sorted position -> row
  const int32_t* gid;       // sorted position -> adapter (G: none, these come last)
  const int32_t* off;       // adapter -> its first sorted position
  const float* ts;          // low-rank values of the sorted rows, pitch RP (R rounded up to 16, zeros past R)
  const void* mat;          // G x R rows of N values (the operands' type)
  int64_t ldm;
  int32_t G, R, RP;
  int32_t relu;
  const void* mask;         // rows by row number, in the operands' type (nullable)
  int64_t ldmask;
};

constexpr float kBf16Max = 3.3895313892515355e38f;   // larger finite fp32 values may round to infinity in bf16

typedef __bf16 lr_bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t lr_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t lr_u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float lr_value(const float* p) { return *p; }
__device__ __forceinline__ float lr_value(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
// round to nearest even, NaN stays NaN
__device__ __forceinline__ uint16_t lr_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ void lr_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void lr_store(uint16_t* p, float v) { *p = lr_bf16(v); }

// 16 bytes at p of which the first `valid` elements (of 2 or 4 bytes) exist, zeros past them.  The
// piece is 16-byte aligned, so it may be read whole if one element exists.
template <class T>
__device__ __forceinline__ lr_u32x4 lr_load16(const T* p, int64_t valid) {
  constexpr int V = 16 / (int)sizeof(T);
  if (valid <= 0) return lr_u32x4{0, 0, 0, 0};
  lr_u32x4 q = *reinterpret_cast<const lr_u32x4*>(p);
  if (valid < V) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (sizeof(T) == 2) {
        if (2 * w >= valid) q[w] = 0;
        else if (2 * w + 1 >= valid) q[w] &= 0xffffu;
      } else {
        if (w >= valid) q[w] = 0;
      }
    }
  }
  return q;
}

// x as a sum of three bf16 values, packed in pairs: t[q] holds term q of 8 values.
// Three terms hold the 24 bits of x (two would leave 2^-18 of it).  Infinities and NaN: the first term
// holds them, later ones are zero (inf - inf would be NaN).
__device__ __forceinline__ void lr_split8(const float (&x)[8], lr_u32x4 (&t)[3]) {
  constexpr int TERMS = 3;
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = x[e];
#pragma unroll
  for (int q = 0; q < TERMS; ++q)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const bf16x2 h = __builtin_convertvector(f32x2{rest[2 * w], rest[2 * w + 1]}, bf16x2);
      t[q][w] = __builtin_bit_cast(uint32_t, h);
      if (q + 1 < TERMS) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float hi = __uint_as_float(e ? (t[q][w] & 0xffff0000u) : (t[q][w] << 16));
          const float r = rest[2 * w + e] - hi;
          rest[2 * w + e] = fabsf(hi) <= 3.402823466e38f ? r : 0.f;
        }
      }
    }
}

}  // namespace ot
