// Products of a bf16 dense layer: gemm_bf16.h's kernels with their Layer epilogues.
#include "dense_products.h"
#include "gemm_bf16.h"
#include "layer_plan.h"
#include "surrogate.h"

namespace ot {
namespace {

constexpr LayB KM = LayB::KMajor, MN = LayB::MNMajor;

// The tiles that plan_dense gives for each product, whole or split.
template <Product P, EpiB E>
hipError_t launch(int tile, const GemmBArgs& g, int64_t splits, hipStream_t st) {
  constexpr LayB LA = P == Product::WeightGrad ? MN : KM, LB = P == Product::Forward ? KM : MN;
  constexpr bool split = E == EpiB::LayerSplit;
  if constexpr (P == Product::Forward) {
    if (tile == kT64x64) return launch_gemm_bf16_pipe<64, 64, 64, 4, 2, LA, LB, E>(g, splits, st);
  }
  if constexpr (P != Product::WeightGrad) {
    if (tile == kT64x128) return launch_gemm_bf16_pipe<64, 128, 64, 3, 4, LA, LB, E, 4>(g, splits, st);
  }
  if constexpr (!split) {
    if (tile == kT128k32) return launch_gemm_bf16_pipe<128, 128, 32, 3, 3, LA, LB, E>(g, splits, st);
  }
  if constexpr (P == Product::InputGrad && !split) {
    if (tile == kT128k64) return launch_gemm_bf16_pipe<128, 128, 64, 2, 2, LA, LB, E>(g, splits, st);
  }
  if constexpr (P != Product::Forward) {
    if (tile == kT128w8) return launch_gemm_bf16_pipe<128, 128, 64, 2, 2, LA, LB, E, 4>(g, splits, st);
  }
  if constexpr (split == (P == Product::InputGrad)) {
    if (tile == kT256) return launch_gemm_bf16_pp<4, LA, LB, E>(g, splits, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace

int run_product_bf16(Product p, const ProductArgs& a, JoinJob* join, hipStream_t st) {
  const AdaptPlan plan = split_dense(plan_dense(true, p, a.M, a.N, a.K, a.ly.planes), a.K);
  GemmBArgs g{};
  g.A = static_cast<const uint16_t*>(a.A);
  g.lda = a.lda;
  g.B = static_cast<const uint16_t*>(a.B);
  g.ldb = a.ldb;
  g.C = a.C;
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
    rc = a.c_type == OT_BF16 ? launch<Product::Forward, EpiB::LayerBf>(plan.tile, g, 1, st)
                             : launch<Product::Forward, EpiB::LayerF32>(plan.tile, g, 1, st);
  else if (p == Product::InputGrad)
    rc = split ? launch<Product::InputGrad, EpiB::LayerSplit>(plan.tile, g, plan.splits, st)
               : launch<Product::InputGrad, EpiB::LayerBf>(plan.tile, g, 1, st);
  else
    rc = split ? launch<Product::WeightGrad, EpiB::LayerSplit>(plan.tile, g, plan.splits, st)
               : launch<Product::WeightGrad, EpiB::LayerF32>(plan.tile, g, 1, st);
  if (rc != hipSuccess)
    return set_error(OT_E_HIP, "launch of the dense product failed: %s", hipGetErrorString(rc));
  if (split) *join = split_join(a, plan.splits, g.split_stride, g.ldc);
  return OT_OK;
}

}  // namespace ot
