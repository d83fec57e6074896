// The matrix products of a dense layer (dense.hip), compiled in files of their own per precision.
#pragma once

#include <cstdint>

#include "common.h"
#include "layer_ops.h"
#include "layer_plan.h"

namespace ot {

// C = A B^T over K.  Forward: the layer (A = x, B = W, both KMajor); InputGrad: A = dz KMajor, B = W MNMajor;
// WeightGrad: A = dz, B = x, both MNMajor.
struct ProductArgs {
  const void* A;
  int64_t lda;
  const void* B;
  int64_t ldb;
  int64_t M, N, K;
  const float* bias;        // Forward (nullable)
  void* C;
  int64_t ldc;
  int32_t c_type;           // OT_FP32 or OT_BF16
  LayerArgs ly;
  float* part;              // partial sums of split products
};

// Launches the product (and the pass that joins its splits); an OT_* status.
int run_product_bf16(Product p, const ProductArgs& a, hipStream_t st);
int run_product_f32(Product p, const ProductArgs& a, hipStream_t st);

#ifdef __HIPCC__
// C[m][n] = sum of the splits' partials [split][m][n] in order; four columns per thread.
template <class T>
__global__ __launch_bounds__(256) void layer_reduce_kernel(const float* __restrict__ part, int32_t splits,
                                                           int64_t stride, int64_t M, int64_t N, int64_t ldp,
                                                           T* __restrict__ C, int64_t ldc) {
  const int64_t groups = (N + 3) / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= M * groups) return;
  const int64_t m = i / groups, n = i % groups * 4;
  const float* p = part + m * ldp + n;
  f32x4 v = *reinterpret_cast<const f32x4*>(p);
  int s = 1;
  for (; s + 8 <= splits; s += 8) {                    // eight loads in flight, added in order
    f32x4 t[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) t[u] = *reinterpret_cast<const f32x4*>(p + (s + u) * stride);
#pragma unroll
    for (int u = 0; u < 8; ++u) v += t[u];
  }
  for (; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(p + s * stride);
  const int cnt = (int)min((int64_t)4, N - n);
  T* out = C + m * ldc + n;
  if constexpr (sizeof(T) == 4) {
    if (cnt == 4) *reinterpret_cast<f32x4*>(out) = v;
    else
      for (int c = 0; c < cnt; ++c) out[c] = v[c];
  } else {
    for (int c = 0; c < cnt; ++c) out[c] = __builtin_bit_cast(uint16_t, (__bf16)v[c]);
  }
}

template <class T>
inline int join_splits(const ProductArgs& a, int64_t splits, int64_t stride, int64_t ldp, hipStream_t st) {
  hipLaunchKernelGGL(layer_reduce_kernel<T>, dim3((unsigned)ceil_div(a.M * ((a.N + 3) / 4), 256)), dim3(256), 0, st,
                     a.part, (int32_t)splits, stride, a.M, a.N, ldp, static_cast<T*>(a.C), a.ldc);
  OT_LAUNCHED("layer_reduce_kernel");
  return OT_OK;
}
#endif

}  // namespace ot
