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
  float* part;              // partial sums, if the product is split
};

// A sum still to be formed: C[m][n] = the sum of part[split][m][n] over the splits in a fixed order, rounded to c_type.
struct JoinJob {
  const float* part;        // rows of ldp values (whole vectors of 4), splits `stride` values apart
  int64_t stride, ldp;
  int32_t splits;           // 0: no job
  int32_t lanes;            // threads that share an output's splits
  int64_t M, N;
  void* C;
  int64_t ldc;
  int32_t c_type;
};

// Launches the product; an OT_* status.  A split one leaves its join to the caller.
int run_product_bf16(Product p, const ProductArgs& a, JoinJob* join, hipStream_t st);
int run_product_f32(Product p, const ProductArgs& a, JoinJob* join, hipStream_t st);

inline JoinJob split_join(const ProductArgs& a, int64_t splits, int64_t stride, int64_t ldp) {
  // few outputs of many splits: a thread's loads would come one after the other (2 x 5 in 512 splits: 22 us)
  return JoinJob{a.part, stride, ldp, (int32_t)splits, splits > 64 ? 16 : 1, a.M, a.N, a.C, a.ldc, a.c_type};
}

}  // namespace ot
