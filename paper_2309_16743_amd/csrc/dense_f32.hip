// Products of an fp32 dense layer: gemm_f32x3.h's kernel with its Layer epilogues.
#include "dense_products.h"
#include "gemm_f32x3.h"
#include "layer_plan.h"
#include "surrogate.h"

namespace ot {
namespace {

constexpr Lay KM = Lay::KMajor, MN = Lay::MNMajor;

// The tiles that plan_dense gives for each product, whole or split.
template <Product P, Epi E>
hipError_t launch(int tile, const GemmArgs& g, int64_t splits, hipStream_t st) {
  constexpr Lay LA = P == Product::WeightGrad ? MN : KM, LB = P == Product::Forward ? KM : MN;
  constexpr bool split = E == Epi::SplitK;
  if (tile == kF64x64) return launch_gemm_f32x3<2, 2, 1, 1, LA, LB, E>(g, splits, st);
  if constexpr (P != Product::WeightGrad) {
    if (tile == kF32x256) return launch_gemm_f32x3<1, 4, 1, 2, LA, LB, E>(g, splits, st);
    if (tile == kF64x256) return launch_gemm_f32x3<1, 4, 2, 2, LA, LB, E>(g, splits, st);
  }
  if constexpr (P == Product::Forward) {
    if (tile == kF64x128) return launch_gemm_f32x3<2, 2, 1, 2, LA, LB, E>(g, splits, st);
  } else if constexpr (!(P == Product::WeightGrad && split)) {
    if (tile == kF128x128) return launch_gemm_f32x3<2, 2, 2, 2, LA, LB, E>(g, splits, st);
  }
  if constexpr (P == Product::WeightGrad) {
    if (tile == kF128x64) return launch_gemm_f32x3<4, 1, 1, 2, LA, LB, E>(g, splits, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace

int run_product_f32(Product p, const ProductArgs& a, JoinJob* join, hipStream_t st) {
  const AdaptPlan plan = split_dense(plan_dense(false, p, a.M, a.N, a.K, 1), a.K);
  GemmArgs g{};
  g.A = static_cast<const float*>(a.A);
  g.lda = a.lda;
  g.B = static_cast<const float*>(a.B);
  g.ldb = a.ldb;
  g.C = static_cast<float*>(a.C);
  g.ldc = a.ldc;
  g.M = a.M;
  g.N = a.N;
  g.K = a.K;
  g.k_chunk = plan.k_chunk;
  g.bias = a.bias;
  g.ly = a.ly;
  const bool split = plan.splits > 1;
  if (split) {
    g.C = a.part;
    g.ldc = (a.N + 3) / 4 * 4;
    g.split_stride = a.M * g.ldc;
  }
  hipError_t rc;
  if (p == Product::Forward)
    rc = a.c_type == OT_BF16 ? launch<Product::Forward, Epi::LayerBf>(plan.tile, g, 1, st)
                             : launch<Product::Forward, Epi::LayerF32>(plan.tile, g, 1, st);
  else if (p == Product::InputGrad)
    rc = split ? launch<Product::InputGrad, Epi::SplitK>(plan.tile, g, plan.splits, st)
               : launch<Product::InputGrad, Epi::Store>(plan.tile, g, 1, st);
  else
    rc = split ? launch<Product::WeightGrad, Epi::SplitK>(plan.tile, g, plan.splits, st)
               : launch<Product::WeightGrad, Epi::Store>(plan.tile, g, 1, st);
  if (rc != hipSuccess)
    return set_error(OT_E_HIP, "launch of the dense product failed: %s", hipGetErrorString(rc));
  if (split) *join = split_join(a, plan.splits, g.split_stride, g.ldc);
  return OT_OK;
}

}  // namespace ot
