// Dense layer with bias, activation and residual (include/layers.h): entry points, the
// activation's backward and the column sums.  The products are in dense_bf16.hip and dense_f32.hip.
#include <cmath>
#include <new>

#include "dense_products.h"
#include "dense_rows.h"
#include "layer_host.h"
#include "layer_plan.h"
#include "layers.h"
#include "row_ops.h"
#include "surrogate.h"

namespace ot {

struct SlopeArgs {
  const void* dy;
  int64_t lddy;
  const void* pre;          // nullable: dz = dy
  int64_t ldp;
  void* dz;                 // rows of lddz values, planes plane_stride elements apart
  int64_t lddz, plane_stride;
  int64_t n, cols;
  float* sums;              // [chunk] rows of sums_ld values (nullable)
  int64_t sums_ld;
  ColumnPlan plan;
};

// dz = dy act'(pre) and its column sums.  Bound by memory where it is long (sums alone of 512 x 1000000 bf16: 160 us,
// 6.4 TB/s) and by its own latency where it is short (1024 x 2048 bf16, gelu in three terms: 9 us).  PLANES: what is written of dz (0: nothing, dz is dy): one matrix, or in
// bf16 the three terms whose sum is dz in 24 bits.
template <class T, int PLANES, int ACT>
__global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a) {
  __shared__ float s[256][9];
  const int w = a.plan.col_threads, cx = threadIdx.x % w, rx = threadIdx.x / w, lanes = 256 / w;
  const int64_t c = ((int64_t)blockIdx.x * w + cx) * 8;
  const int64_t r0 = (int64_t)blockIdx.y * a.plan.rows, r1 = min(a.n, r0 + a.plan.rows);
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (c < a.cols) {
    constexpr int U = 4;
    float v[U][8], z[U][8];
    rows_in_groups<U>(
        r0 + rx, r1, lanes,
        [&](int u, int64_t r) {
          load8(static_cast<const T*>(a.dy) + r * a.lddy + c, a.cols - c, v[u]);
          if constexpr (PLANES > 0) load8(static_cast<const T*>(a.pre) + r * a.ldp + c, a.cols - c, z[u]);
        },
        [&](int u, int64_t r) {
          if constexpr (PLANES > 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] = act_back<ACT>(v[u][e], z[u][e]);
            T* out = static_cast<T*>(a.dz) + r * a.lddz + c;
            if constexpr (PLANES == 3) {
              lr_u32x4 t[3];
              lr_split8(v[u], t);
#pragma unroll
              for (int p = 0; p < 3; ++p) *reinterpret_cast<lr_u32x4*>(out + p * a.plane_stride) = t[p];
            } else {
              store8(out, 8, v[u]);                      // (rows of dz are padded to 8 values)
            }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[e] += v[u][e];
        });
  }
  if (!a.sums) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) s[threadIdx.x][e] = sum[e];
  for (int h = lanes / 2; h > 0; h /= 2) {
    __syncthreads();
    if (rx < h)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[threadIdx.x][e] += s[threadIdx.x + h * w][e];
  }
  if (rx == 0)
    for (int e = 0; e < 8; ++e)
      if (c + e < a.cols) a.sums[blockIdx.y * a.sums_ld + c + e] = s[threadIdx.x][e];
}

// All the sums that a backward leaves: of the split products, and of the chunks' column sums.  A thread sums four
// neighbouring values; where the splits are many, `lanes` threads share them.  One launch, since each costs 4 us and more
// by itself (331 x 437 x 6561 fp32: 13 us for 58 MB of partial sums, 17 in three).
struct JoinJobs {
  JoinJob job[3];
  int64_t blocks[3];
};
__global__ __launch_bounds__(256) void dense_join_kernel(JoinJobs jobs) {
  __shared__ f32x4 s[256];
  int64_t b = blockIdx.x;
  int k = 0;
  while (b >= jobs.blocks[k]) b -= jobs.blocks[k++];
  const JoinJob& j = jobs.job[k];
  const int per = 256 / j.lanes, lane = threadIdx.x / per;
  const int64_t groups = (j.N + 3) / 4, i = b * per + threadIdx.x % per;
  const bool in = i < j.M * groups;
  int64_t col;
  const int64_t m = quotient(in ? i : 0, groups, col), n = 4 * col;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (in) {
    const float* p = j.part + m * j.ldp + n;
    int q = lane;
    for (; q + 7 * j.lanes < j.splits; q += 8 * j.lanes) {   // eight loads in flight, added in order
      f32x4 t[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) t[u] = *reinterpret_cast<const f32x4*>(p + (q + u * j.lanes) * j.stride);
#pragma unroll
      for (int u = 0; u < 8; ++u) v += t[u];
    }
    for (; q < j.splits; q += j.lanes) v += *reinterpret_cast<const f32x4*>(p + q * j.stride);
  }
  if (j.lanes > 1) {                                     // the same for the whole block
    s[threadIdx.x] = v;
    for (int h = j.lanes / 2; h > 0; h /= 2) {
      __syncthreads();
      if (lane < h) s[threadIdx.x] += s[threadIdx.x + h * per];
    }
    v = s[threadIdx.x];
  }
  if (!in || lane > 0) return;
  const int cnt = (int)min((int64_t)4, j.N - n);
  if (j.c_type == OT_BF16) {
    uint16_t* out = static_cast<uint16_t*>(j.C) + m * j.ldc + n;
    for (int c = 0; c < cnt; ++c) out[c] = lr_bf16(v[c]);
  } else {
    float* out = static_cast<float*>(j.C) + m * j.ldc + n;
    if (cnt == 4 && reinterpret_cast<uintptr_t>(out) % 16 == 0) *reinterpret_cast<f32x4*>(out) = v;
    else
      for (int c = 0; c < cnt; ++c) out[c] = v[c];
  }
}

__global__ __launch_bounds__(256) void zero_rows_kernel(float* p, int64_t ld, int64_t rows, int64_t cols) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  for (int64_t k = i; k < rows * cols; k += step) p[k / cols * ld + k % cols] = 0.f;
}

}  // namespace ot

struct ot_dense {
  int64_t in, out;
  int32_t precision, act;
  int device;
  ot::Workspace ws;
  ot::DenseSizes sizes() const {
    const bool bf16 = precision == OT_BF16;
    const int32_t planes = act == OT_ACT_NONE ? 0 : bf16 && act != OT_ACT_RELU ? 3 : 1;
    return {in, out, bf16, planes};
  }
  int64_t bytes(int64_t n) const { return n < 1 ? 0 : ot::dz_bytes(sizes(), n) + 4 * ot::dense_values(sizes(), n); }
};

namespace {

constexpr int64_t kMost = 1LL << 26, kMostValues = 1LL << 36;

int run_product(ot::Product p, const ot_dense* d, const ot::ProductArgs& a, ot::JoinJob* join, hipStream_t st) {
  return d->precision == OT_BF16 ? ot::run_product_bf16(p, a, join, st) : ot::run_product_f32(p, a, join, st);
}

// The layer straight from memory (direct_layer).
template <class T, class Y>
int run_rows(const ot_dense* d, const ot::RowsArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)ot::ceil_div(a.N, 16), (unsigned)ot::ceil_div(a.M, 32)), block(256);
  if (a.M <= 16) hipLaunchKernelGGL((ot::dense_rows_kernel<T, Y, 1>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((ot::dense_rows_kernel<T, Y, 2>), grid, block, 0, st, a);
  OT_LAUNCHED("dense_rows_kernel");
  return OT_OK;
}

// dz and the column sums; where those are partial, their join is left to the caller.
int run_slope(const ot_dense* d, ot::SlopeArgs a, float* dbias, float* part, ot::JoinJob* join, hipStream_t st) {
  a.plan = ot::plan_columns(a.n, a.cols);
  const bool split = a.plan.chunks > 1;
  a.sums = dbias && split ? part : dbias;
  a.sums_ld = ot::round_up(a.cols, 4);
  const dim3 grid((unsigned)a.plan.blocks_x, (unsigned)a.plan.chunks), block(256);
  ot::with_act(d->act, [&](auto act) {
    constexpr int A = decltype(act)::value;
    constexpr int PLANES = A == ot::kActNone ? 0 : 1, TERMS = A == ot::kActNone ? 0 : A == ot::kActRelu ? 1 : 3;
    if (d->precision == OT_FP32) hipLaunchKernelGGL((ot::slope_kernel<float, PLANES, A>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((ot::slope_kernel<uint16_t, TERMS, A>), grid, block, 0, st, a);
  });
  OT_LAUNCHED("slope_kernel");
  if (dbias && split)
    *join = ot::JoinJob{part, a.sums_ld, a.sums_ld, (int32_t)a.plan.chunks, 16, 1, a.cols, dbias, a.cols, OT_FP32};
  return OT_OK;
}

int run_joins(const ot::JoinJob (&job)[3], hipStream_t st) {
  ot::JoinJobs jobs{};
  int64_t blocks = 0;
  for (int k = 0; k < 3; ++k) {
    jobs.job[k] = job[k];
    if (job[k].splits) jobs.blocks[k] = ot::ceil_div(job[k].M * ot::ceil_div(job[k].N, 4), 256 / job[k].lanes);
    blocks += jobs.blocks[k];
  }
  if (blocks == 0) return OT_OK;
  hipLaunchKernelGGL(ot::dense_join_kernel, dim3((unsigned)blocks), dim3(256), 0, st, jobs);
  OT_LAUNCHED("dense_join_kernel");
  return OT_OK;
}

int zero_rows(float* p, int64_t ld, int64_t rows, int64_t cols, hipStream_t st) {
  const int64_t blocks = std::min<int64_t>(4096, ot::ceil_div(rows * cols, 256));
  hipLaunchKernelGGL(ot::zero_rows_kernel, dim3((unsigned)blocks), dim3(256), 0, st, p, ld, rows, cols);
  OT_LAUNCHED("zero_rows_kernel");
  return OT_OK;
}

}  // namespace

extern "C" int dense_create(ot_dense** out, int64_t in, int64_t out_dim, int32_t precision, int32_t activation,
                            int64_t max_rows) {
  ot::clear_error();
  OT_REQUIRE(out != nullptr, "dense_create: NULL out");
  *out = nullptr;
  OT_REQUIRE(in >= 1 && in <= kMost && out_dim >= 1 && out_dim <= kMost, "dense_create: in or out outside [1, 2^26]");
  OT_REQUIRE(in * out_dim <= kMostValues, "dense_create: more than 2^36 weights");
  OT_REQUIRE(precision == OT_FP32 || precision == OT_BF16, "dense_create: unknown precision");
  OT_REQUIRE(activation >= OT_ACT_NONE && activation <= OT_ACT_GELU, "dense_create: unknown activation");
  OT_REQUIRE(max_rows >= 0 && max_rows <= kMost, "dense_create: max_rows outside [0, 2^26]");
  OT_REQUIRE(max_rows * std::max(in, out_dim) <= kMostValues, "dense_create: more than 2^36 values in max_rows rows");
  int device = -1;
  OT_HIP(hipGetDevice(&device));
  ot_dense* d = new (std::nothrow) ot_dense();
  if (!d) return ot::set_error(OT_E_NOMEM, "dense_create: out of host memory");
  d->in = in;
  d->out = out_dim;
  d->precision = precision;
  d->act = activation;
  d->device = device;
  const int rc = d->ws.allocate(max_rows, d->bytes(max_rows), "dense_create");
  if (rc) {
    delete d;
    return rc;
  }
  *out = d;
  return OT_OK;
}

extern "C" int dense_forward(ot_dense* d, const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias,
                             const void* residual, int64_t ldr, int64_t n, void* y, int64_t ldy, int32_t y_type,
                             void* pre, int64_t ldp, void* stream) {
  ot::clear_error();
  const char* what = "dense_forward";
  OT_REQUIRE(d != nullptr, "%s: NULL layer", what);
  OT_REQUIRE(n >= 0 && n <= kMost, "%s: n outside [0, 2^26]", what);
  OT_REQUIRE(n * std::max(d->in, d->out) <= kMostValues, "%s: more than 2^36 values", what);
  OT_REQUIRE(y_type == OT_FP32 || y_type == OT_BF16, "%s: y_type is neither OT_FP32 nor OT_BF16", what);
  if (n == 0) return OT_OK;
  const int e = d->precision == OT_BF16 ? 2 : 4, ey = y_type == OT_BF16 ? 2 : 4;
  int rc;
  if ((rc = ot::check_rows(x, ldx, n, d->in, e, what, "x"))) return rc;
  if ((rc = ot::check_rows(w, ldw, d->out, d->in, e, what, "w"))) return rc;
  if ((rc = ot::check_rows(y, ldy, n, d->out, ey, what, "y"))) return rc;
  if (residual && (rc = ot::check_rows(residual, ldr, n, d->out, ey, what, "residual"))) return rc;
  if (pre && (rc = ot::check_rows(pre, ldp, n, d->out, e, what, "pre"))) return rc;
  if ((rc = ot::check_values(bias, 4, what, "bias"))) return rc;
  if ((rc = ot::check_device(d->device, what))) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const ot::LayerArgs ly{residual, ldr, pre, ldp, d->act, 1, 0};
  if (ot::direct_layer(e == 2, n, d->out, d->in)) {
    const ot::RowsArgs a{x, ldx, w, ldw, n, d->out, d->in, bias, y, ldy, ly};
    if (e == 2) return ey == 2 ? run_rows<uint16_t, uint16_t>(d, a, st) : run_rows<uint16_t, float>(d, a, st);
    return ey == 2 ? run_rows<float, uint16_t>(d, a, st) : run_rows<float, float>(d, a, st);
  }
  const ot::ProductArgs a{x, ldx, w, ldw, n, d->out, d->in, bias, y, ldy, y_type, ly, nullptr};
  return run_product(ot::Product::Forward, d, a, nullptr, st);
}

extern "C" int dense_backward(ot_dense* d, const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t n,
                              const void* dy, int64_t lddy, const void* pre, int64_t ldp, void* dx, int64_t lddx,
                              float* dw, int64_t lddw, float* dbias, void* stream) try {
  ot::clear_error();
  const char* what = "dense_backward";
  OT_REQUIRE(d != nullptr, "%s: NULL layer", what);
  OT_REQUIRE(n >= 0 && n <= kMost, "%s: n outside [0, 2^26]", what);
  OT_REQUIRE(n * std::max(d->in, d->out) <= kMostValues, "%s: more than 2^36 values", what);
  const int e = d->precision == OT_BF16 ? 2 : 4;
  const ot::DenseSizes sz = d->sizes();
  int rc;
  if (dw && (rc = ot::check_rows(dw, lddw, d->out, d->in, 4, what, "dw"))) return rc;
  if ((rc = ot::check_values(dbias, 4, what, "dbias"))) return rc;
  if (n > 0) {
    if ((rc = ot::check_rows(dy, lddy, n, d->out, e, what, "dy"))) return rc;
    if (sz.planes && (rc = ot::check_rows(pre, ldp, n, d->out, e, what, "pre"))) return rc;
    if (dw && (rc = ot::check_rows(x, ldx, n, d->in, e, what, "x"))) return rc;
    if (dx) {
      if ((rc = ot::check_rows(w, ldw, d->out, d->in, e, what, "w"))) return rc;
      if ((rc = ot::check_rows(dx, lddx, n, d->in, e, what, "dx"))) return rc;
    }
  }
  if ((rc = ot::check_device(d->device, what))) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (n == 0) {
    if (dw && (rc = zero_rows(dw, lddw, d->out, d->in, st))) return rc;
    return dbias ? zero_rows(dbias, d->out, 1, d->out, st) : OT_OK;
  }
  if (!dx && !dw && !dbias) return OT_OK;
  // without dz and partial sums a call keeps nothing between its launches
  if ((sz.planes || (dw && ot::dw_values(sz, n)) || (dx && ot::dx_values(sz, n)) ||
       (dbias && ot::column_values(n, d->out))) &&
      (rc = d->ws.begin(n, st, what, [&](int64_t rows) { return d->bytes(rows); })))
    return rc;
  const int64_t ldz = sz.planes ? ot::dz_ld(sz) : lddy;
  void* dz = sz.planes ? d->ws.p : const_cast<void*>(dy);
  float* const dw_part = reinterpret_cast<float*>(d->ws.p + ot::dz_bytes(sz, n));
  float* const dx_part = dw_part + ot::round_up(ot::dw_values(sz, n), 4);
  float* const db_part = dx_part + ot::round_up(ot::dx_values(sz, n), 4);
  ot::JoinJob join[3] = {};                              // dw, dx, dbias
  if (sz.planes || dbias) {
    const ot::SlopeArgs s{dy, lddy, pre, ldp, dz, ldz, n * ldz, n, d->out, nullptr, 0, {}};
    if ((rc = run_slope(d, s, dbias, db_part, &join[2], st))) return rc;
  }
  ot::LayerArgs ly{};
  ly.planes = std::max(1, sz.planes);                    // all of dz: in dx two terms would leave 2^-18 of each
                                                         // product, which shows where a sum cancels (1024 x 2048 x
                                                         // 2048: 40 us, 29 with two)
  ly.plane_stride = n * ldz;
  if (dw) {
    const ot::ProductArgs a{dz, ldz, x, ldx, d->out, d->in, n, nullptr, dw, lddw, OT_FP32, ly, dw_part};
    if ((rc = run_product(ot::Product::WeightGrad, d, a, &join[0], st))) return rc;
  }
  if (dx) {
    const ot::ProductArgs a{dz, ldz, w, ldw, n, d->in, d->out, nullptr, dx, lddx, d->precision, ly, dx_part};
    if ((rc = run_product(ot::Product::InputGrad, d, a, &join[1], st))) return rc;
  }
  return run_joins(join, st);
} catch (const std::bad_alloc&) {
  return ot::set_error(OT_E_NOMEM, "dense_backward: out of host memory");
}

extern "C" int dense_destroy(ot_dense* d) {
  ot::clear_error();
  if (!d) return OT_OK;
  d->ws.release();
  delete d;
  return OT_OK;
}
