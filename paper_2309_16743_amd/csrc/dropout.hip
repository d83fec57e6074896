// Dropout with a residual (include/layers.h); the mask is generated where it is needed.
#include <cmath>
#include <new>

#include "layer_host.h"
#include "layer_plan.h"
#include "layers.h"
#include "philox32.h"
#include "row_ops.h"
#include "surrogate.h"

namespace ot {

struct DropoutArgs {
  const void* x;
  int64_t ldx;
  const void* residual;     // nullable
  int64_t ldr;
  void* y;
  int64_t ldy;
  int64_t n, cols;
  uint32_t k0, k1, site, step;
  const int64_t* step_dev;  // nullable
  uint32_t below;           // bits under this drop the value
  float scale;
  int32_t col_threads;
};

// A thread makes 8 columns of a row from one counter: ten rounds of two 32 x 32 -> 64 bit products for 8
// values, hidden behind the memory (640000 x 64 bf16: 28 us, 5.9 TB/s; with the loads of four rows ahead of
// their stores, and so fewer threads on a CU, 36).
template <class T>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a) {
  const int w = a.col_threads, lanes = 256 / w;
  const int64_t j = (int64_t)blockIdx.x * w + threadIdx.x % w, c = 8 * j;
  if (c >= a.cols) return;
  const uint32_t step = a.step + (a.step_dev ? (uint32_t)*a.step_dev : 0u);
  for (int64_t r = (int64_t)blockIdx.y * lanes + threadIdx.x / w; r < a.n; r += (int64_t)gridDim.y * lanes) {
    float v[8], res[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    load8(static_cast<const T*>(a.x) + r * a.ldx + c, a.cols - c, v);
    if (a.residual) load8(static_cast<const T*>(a.residual) + r * a.ldr + c, a.cols - c, res);
    const Words4 b = philox4x32_10((uint32_t)j, (uint32_t)r, a.site, step, a.k0, a.k1);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t bits = e % 2 ? b.w[e / 2] >> 16 : b.w[e / 2] & 0xffffu;
      v[e] = bits < a.below ? res[e] : fmaf(v[e], a.scale, res[e]);
    }
    store8(static_cast<T*>(a.y) + r * a.ldy + c, a.cols - c, v);
  }
}

}  // namespace ot

struct ot_dropout {
  uint64_t seed;
  uint32_t site, below;
  float scale;
  int32_t precision;
  int device;
};

namespace {

int run(const ot_dropout* d, const void* x, int64_t ldx, const char* name_x, const void* residual, int64_t ldr,
        int64_t n, int64_t cols, void* y, int64_t ldy, const char* name_y, int64_t step, const int64_t* step_dev,
        void* stream, const char* what) {
  ot::clear_error();
  OT_REQUIRE(d != nullptr, "%s: NULL dropout", what);
  OT_REQUIRE(n >= 0 && n < (1LL << 31) && cols >= 0 && cols < (1LL << 31), "%s: n or cols outside [0, 2^31)", what);
  if (n == 0 || cols == 0) return OT_OK;
  const int e = d->precision == OT_BF16 ? 2 : 4;
  int rc;
  if ((rc = ot::check_rows(x, ldx, n, cols, e, what, name_x))) return rc;
  if (residual && (rc = ot::check_rows(residual, ldr, n, cols, e, what, "residual"))) return rc;
  if ((rc = ot::check_rows(y, ldy, n, cols, e, what, name_y))) return rc;
  if ((rc = ot::check_values(step_dev, 8, what, "step_dev"))) return rc;
  if ((rc = ot::check_device(d->device, what))) return rc;
  const int64_t groups = ot::ceil_div(cols, 8);
  int32_t w = 1;
  while (w < 256 && w < groups) w *= 2;
  const int64_t bx = ot::ceil_div(groups, w), rows = ot::ceil_div(n, 256 / w);
  const int64_t by = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(rows, 65535), 8192 / bx));
  const ot::DropoutArgs a{x, ldx, residual, ldr, y, ldy, n, cols, (uint32_t)d->seed, (uint32_t)(d->seed >> 32),
                          d->site, (uint32_t)step, step_dev, d->below, d->scale, w};
  const dim3 grid((unsigned)bx, (unsigned)by);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (e == 2) hipLaunchKernelGGL(ot::dropout_kernel<uint16_t>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(ot::dropout_kernel<float>, grid, dim3(256), 0, st, a);
  OT_LAUNCHED("dropout_kernel");
  return OT_OK;
}

}  // namespace

extern "C" int dropout_create(ot_dropout** out, double p, uint64_t seed, uint32_t site, int32_t precision) {
  ot::clear_error();
  OT_REQUIRE(out != nullptr, "dropout_create: NULL out");
  *out = nullptr;
  OT_REQUIRE(p >= 0.0 && p <= 1.0, "dropout_create: p outside [0, 1]");
  OT_REQUIRE(precision == OT_FP32 || precision == OT_BF16, "dropout_create: unknown precision");
  int device = -1;
  OT_HIP(hipGetDevice(&device));
  ot_dropout* d = new (std::nothrow) ot_dropout();
  if (!d) return ot::set_error(OT_E_NOMEM, "dropout_create: out of host memory");
  const uint32_t t = (uint32_t)std::nearbyint(65536.0 * p);
  *d = ot_dropout{seed, site, t, t < 65536 ? (float)(65536.0 / (65536 - t)) : 0.f, precision, device};
  *out = d;
  return OT_OK;
}

extern "C" int dropout_forward(ot_dropout* d, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                               int64_t n, int64_t cols, void* y, int64_t ldy, int64_t step, const int64_t* step_dev,
                               void* stream) {
  return run(d, x, ldx, "x", residual, ldr, n, cols, y, ldy, "y", step, step_dev, stream, "dropout_forward");
}

extern "C" int dropout_backward(ot_dropout* d, const void* dy, int64_t lddy, int64_t n, int64_t cols, void* dx,
                                int64_t lddx, int64_t step, const int64_t* step_dev, void* stream) {
  return run(d, dy, lddy, "dy", nullptr, 0, n, cols, dx, lddx, "dx", step, step_dev, stream, "dropout_backward");
}

extern "C" int dropout_destroy(ot_dropout* d) {
  ot::clear_error();
  delete d;
  return OT_OK;
}
