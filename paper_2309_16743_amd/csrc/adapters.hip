// Low-rank adapters beside a frozen projection (include/adapters.h).
//
// A call first sorts its rows by adapter (group_rows_kernel): position p of the
// sorted order is row perm[p] with adapter gid[p] (G: none).  Every later kernel
// works in sorted order and reads and writes the caller's rows through perm, so that rows of
// one adapter lie next to each other whatever order they came in.
#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>
#include <vector>

#include "adapt_plan.h"
#include "adapters.h"
#include "common.h"
#include "gemm_bf16.h"
#include "gemm_f32x3.h"
#include "intmath.h"
#include "lowrank.h"
#include "surrogate.h"

namespace ot {

// Block g collects the rows of adapter g (block G: rows without one) in their
// order: it counts the rows of smaller keys, which is where its own start, and
// then writes them.  Every block reads all ids (n G / 64 wavefront reads from
// the caches) and none waits for another.  Slots: adapter g's first is
// start / slot_rows + g, which leaves room for those of the adapters before it; those
// that stay unused get count 0.
__global__ __launch_bounds__(256) void group_rows_kernel(const int32_t* __restrict__ ids, int32_t n, int32_t G,
                                                         int32_t* __restrict__ perm, int32_t* __restrict__ gid,
                                                         int32_t* __restrict__ off, RowSlot* __restrict__ slots,
                                                         int32_t slot_rows) {
  __shared__ int32_t s_less[4], s_same[4];
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  auto key = [&](int i) {
    const int32_t k = ids[i];
    return (k < 0 || k >= G) ? G : k;
  };
  int less = 0, same = 0;
  for (int i = tid; i < n; i += 256) {
    const int k = key(i);
    less += k < g;
    same += k == g;
  }
  for (int o = 32; o > 0; o >>= 1) {
    less += __shfl_xor(less, o, 64);
    same += __shfl_xor(same, o, 64);
  }
  if (lane == 0) {
    s_less[wid] = less;
    s_same[wid] = same;
  }
  __syncthreads();
  const int start = (s_less[0] + s_less[1]) + (s_less[2] + s_less[3]);
  const int count = (s_same[0] + s_same[1]) + (s_same[2] + s_same[3]);
  if (tid == 0) {
    off[g] = start;
    if (g == G) off[G + 1] = n;
  }
  const int slot0 = start / slot_rows + g, slot1 = (start + count) / slot_rows + g + 1;
  for (int s = slot0 + tid; s < slot1; s += 256) {
    const int r = (s - slot0) * slot_rows;
    slots[s] = RowSlot{start + r, max(0, min(slot_rows, count - r)), g, 0};
  }
  int at = start;
  for (int i0 = 0; i0 < n && at < start + count; i0 += 256) {   // the same for all threads: at is uniform
    const int i = i0 + tid;
    const bool mine = i < n && key(i) == g;
    const uint64_t mask = __ballot(mine);
    __syncthreads();
    if (lane == 0) s_same[wid] = __popcll(mask);
    __syncthreads();
    int p = at;
    for (int w = 0; w < wid; ++w) p += s_same[w];
    if (mine) {
      p += __popcll(mask & ((1ull << lane) - 1));
      perm[p] = i;
      gid[p] = g;
    }
    at += (s_same[0] + s_same[1]) + (s_same[2] + s_same[3]);
  }
}

// C[row of m][n] = sum of the splits' partials [split][m][n] in order, 0 where mask is not above 0; four columns
// per thread.
template <class T>
__global__ __launch_bounds__(256) void adapt_reduce_kernel(const float* __restrict__ ws, int32_t splits,
                                                           int64_t stride, int64_t M, int64_t N, int64_t ldws,
                                                           const int32_t* __restrict__ perm,
                                                           const T* __restrict__ mask, int64_t ldmask,
                                                           T* __restrict__ C, int64_t ldc) {
  const int64_t groups = (N + 3) / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= M * groups) return;
  const int64_t m = i / groups, n = i % groups * 4, row = perm[m];
  const float* p = ws + m * ldws + n;
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
  for (int c = 0; c < cnt; ++c) {
    if (mask && !(lr_value(mask + row * ldmask + n + c) > 0.f)) v[c] = 0.f;
    lr_store(C + row * ldc + n + c, v[c]);
  }
}

}  // namespace ot

struct ot_adapters {
  int64_t in, out;
  int32_t R, RP, G, precision;
  int device;
  int64_t max_rows;
  ot::AdaptSizes sizes() const { return {in, out, RP, G, precision == OT_BF16}; }
  // workspaces of calls of up to max_rows rows, in one allocation
  unsigned char* ws = nullptr;
  bool captured = false;                    // a captured call may name ws
  std::vector<unsigned char*> kept;         // workspaces replaced after such a call
};

namespace {

constexpr int64_t kMaxRows = 1LL << 20;

struct Work {
  int32_t* perm;
  int32_t* gid;
  int32_t* off;
  ot::RowSlot* slots;
  float* ts;
  float* part;            // partial sums of split products, one after another
  int64_t n_slots;
};

constexpr int kMinSlotRows = 16;

// Rows of a slot for a product over L values: short ranges are not split, so smaller slots
// give the blocks that fill the card (1024 rows of 2048 values: 9.3 us with 16, 11.5 with 32); long ones
// read the adapter's matrix once per slot.
int slot_rows(int64_t L) { return L <= 4096 ? kMinSlotRows : ot::kSlotRows; }

int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

// Workspace of a call of n rows at `base`; returns the size of what comes before the partial sums, whose
// size only allocate() needs (part_values looks at every group of 32 rows: 0.1 ms and more at 2^20).
int64_t layout(const ot_adapters* a, int64_t n, unsigned char* base, Work* w) {
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    unsigned char* p = base + at;
    at += up256(bytes);
    return p;
  };
  Work t;
  t.n_slots = n / kMinSlotRows + a->G + 1;       // most of either slot size
  t.perm = reinterpret_cast<int32_t*>(take(4 * n));
  t.gid = reinterpret_cast<int32_t*>(take(4 * n));
  t.off = reinterpret_cast<int32_t*>(take(4 * (a->G + 2)));
  t.slots = reinterpret_cast<ot::RowSlot*>(take((int64_t)sizeof(ot::RowSlot) * t.n_slots));
  t.ts = reinterpret_cast<float*>(take(4 * n * a->RP));
  t.part = reinterpret_cast<float*>(base + at);
  if (w) *w = t;
  return at;
}

int allocate(ot_adapters* a, int64_t rows, const char* what) {
  unsigned char* p = nullptr;
  const int64_t bytes = layout(a, rows, nullptr, nullptr) + 4 * ot::part_values(a->sizes(), rows);
  const hipError_t e = hipMalloc(reinterpret_cast<void**>(&p), (size_t)bytes);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return ot::set_error(OT_E_NOMEM, "%s: hipMalloc of %lld bytes failed: %s", what, (long long)bytes,
                         hipGetErrorString(e));
  }
  if (a->ws) {
    if (a->captured) {
      a->kept.push_back(a->ws);             // (reserved before: cannot throw)
      a->captured = false;
    } else {
      (void)hipFree(a->ws);                 // waits for the device
    }
  }
  a->ws = p;
  a->max_rows = rows;
  return OT_OK;
}

// Device, capture state and workspaces of a call of n rows.
int begin_call(ot_adapters* a, int64_t n, hipStream_t st, const char* what) {
  int device = -1;
  OT_HIP(hipGetDevice(&device));
  if (device != a->device)
    return ot::set_error(OT_E_STATE, "%s: device %d is current, the adapters live on %d", what, device, a->device);
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  OT_HIP(hipStreamIsCapturing(st, &cap));
  if (n > a->max_rows) {
    if (cap != hipStreamCaptureStatusNone)
      return ot::set_error(OT_E_STATE, "%s: %lld rows under capture, workspaces hold %lld", what, (long long)n,
                           (long long)a->max_rows);
    a->kept.reserve(a->kept.size() + 1);
    const int rc = allocate(a, n, what);
    if (rc) return rc;
  }
  if (cap != hipStreamCaptureStatusNone) a->captured = true;
  return OT_OK;
}

int check_rows(const void* p, int64_t ld, int64_t rows, int64_t len, int elem, const char* what, const char* name) {
  OT_REQUIRE(p != nullptr, "%s: NULL %s", what, name);
  OT_REQUIRE(reinterpret_cast<uintptr_t>(p) % 16 == 0, "%s: %s is not 16-byte aligned", what, name);
  OT_REQUIRE(rows <= 1 || (ld >= len && ld % (16 / elem) == 0),
             "%s: leading dimension %lld of %s is not a multiple of %d of at least %lld", what, (long long)ld, name,
             16 / elem, (long long)len);
  return OT_OK;
}

int check_values(const void* p, int align, const char* what, const char* name) {
  OT_REQUIRE(reinterpret_cast<uintptr_t>(p) % align == 0, "%s: %s is not aligned to its elements", what, name);
  return OT_OK;
}

// Whether the shrink's blocks sort the ids themselves (lowrank.h).
bool self_sorted(int64_t n, int32_t G) { return n <= ot::kSelfRows && G < ot::kSelfKeys; }

int run_group(const ot_adapters* a, const int32_t* ids, int64_t n, int64_t L, const Work& w, hipStream_t st) {
  hipLaunchKernelGGL(ot::group_rows_kernel, dim3((unsigned)(a->G + 1)), dim3(256), 0, st, ids, (int32_t)n, a->G,
                     w.perm, w.gid, w.off, w.slots, slot_rows(L));
  OT_LAUNCHED("group_rows_kernel");
  return OT_OK;
}

// Sorts the rows by adapter, then the low-rank values of every row.
template <class T>
int run_shrink(const ot_adapters* a, ot::ShrinkArgs s, const int32_t* ids, int64_t n, const Work& w, hipStream_t st) {
  const bool self = self_sorted(n, s.G);
  int rc;
  if (!self && (rc = run_group(a, ids, n, s.L, w, st))) return rc;
  const int64_t splits = ot::shrink_splits(n, s.L, s.G);
  s.k_chunk = ot::ceil_div(ot::ceil_div(s.L, splits), ot::kShrinkUnit) * ot::kShrinkUnit;
  s.splits = (int32_t)ot::ceil_div(s.L, s.k_chunk);
  s.n = n;
  s.part = w.part;
  const unsigned n_slots = (unsigned)(n / slot_rows(s.L) + s.G + 1);
  const dim3 grid(n_slots, (unsigned)s.splits);
  const ot::SelfSort o{ids, w.perm, w.gid, w.off, w.slots, slot_rows(s.L)};
  auto go = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    if (self) hipLaunchKernelGGL((ot::shrink_kernel<T, NT, true>), grid, dim3(ot::kShrinkThreads), 0, st, s, o);
    else hipLaunchKernelGGL((ot::shrink_kernel<T, NT, false>), grid, dim3(ot::kShrinkThreads), 0, st, s, o);
  };
  switch (s.RP / 16) {
    case 1: go(std::integral_constant<int, 1>()); break;
    case 2: go(std::integral_constant<int, 2>()); break;
    case 3: go(std::integral_constant<int, 3>()); break;
    default: go(std::integral_constant<int, 4>()); break;
  }
  OT_LAUNCHED("shrink_kernel");
  if (s.splits > 1) {
    hipLaunchKernelGGL(ot::shrink_reduce_kernel, dim3(n_slots), dim3(256), 0, st, s);
    OT_LAUNCHED("shrink_reduce_kernel");
  }
  return OT_OK;
}

template <class T>
int run_pass(const ot_adapters* a, const ot::OuterArgs& o, const void* up, int64_t ldu, int64_t n, const Work& w,
             hipStream_t st) {
  const int chunks = ot::pass_chunks(a->sizes(), n);
  const int64_t ranges = ot::pass_ranges(a->sizes(), n);
  const ot::PassArgs p{o, up, ldu, w.part, n, ranges, a->RP, chunks};
  const dim3 grid((unsigned)(ot::ceil_div(ranges, 8) * 16), (unsigned)a->G), block(ot::kPassThreads);
  switch (a->RP / 16) {
    case 1: hipLaunchKernelGGL((ot::pass_kernel<T, 1>), grid, block, 0, st, p); break;
    case 2: hipLaunchKernelGGL((ot::pass_kernel<T, 2>), grid, block, 0, st, p); break;
    case 3: hipLaunchKernelGGL((ot::pass_kernel<T, 3>), grid, block, 0, st, p); break;
    default: hipLaunchKernelGGL((ot::pass_kernel<T, 4>), grid, block, 0, st, p); break;
  }
  OT_LAUNCHED("pass_kernel");
  hipLaunchKernelGGL(ot::pass_reduce_kernel, dim3((unsigned)ot::ceil_div(n * a->RP, 16)), dim3(256), 0, st, w.part,
                     (int32_t)ranges, n, a->RP, a->G, w.gid, o.scale, w.ts);
  OT_LAUNCHED("pass_reduce_kernel");
  return OT_OK;
}

// Both gradients of the bank (only_down: the second alone).
template <class T>
int run_outer(ot::OuterArgs up, ot::OuterArgs down, int64_t n, int32_t G, hipStream_t st, bool only_down = false) {
  // short rows and many rows per adapter: the wavefronts of a block share its columns and split the rows
  auto blocks = [&](ot::OuterArgs& o) {
    o.split_rows = ot::ceil_div(o.L, 256) * G < 1024 && n > 64 * (int64_t)G;
    return ot::ceil_div(o.L, o.split_rows ? 64 : 256);
  };
  const int64_t b1 = blocks(down), b0 = only_down ? 0 : blocks(up);
  const dim3 grid((unsigned)(b0 + b1), (unsigned)G);
  switch ((up.R + 15) / 16) {
    case 1: hipLaunchKernelGGL((ot::outer_kernel<T, 1>), grid, dim3(256), 0, st, up, down, b0); break;
    case 2: hipLaunchKernelGGL((ot::outer_kernel<T, 2>), grid, dim3(256), 0, st, up, down, b0); break;
    case 3: hipLaunchKernelGGL((ot::outer_kernel<T, 3>), grid, dim3(256), 0, st, up, down, b0); break;
    default: hipLaunchKernelGGL((ot::outer_kernel<T, 4>), grid, dim3(256), 0, st, up, down, b0); break;
  }
  OT_LAUNCHED("outer_kernel");
  return OT_OK;
}

// The adapted product C[row] = B A[row] (+ bias) + sum_r ts[r] mat_g[r] (ReLU or mask): the
// layer itself (B = W, KMajor) or its input gradient (B = W, MNMajor).
struct Expand {
  const void* A;
  int64_t lda;
  const void* B;
  int64_t ldb;
  int64_t M, N, K;
  const float* bias;
  void* C;
  int64_t ldc;
  int32_t c_type;         // OT_FP32 or OT_BF16
  ot::AdaptRows lr;
};

// The tiles that plan_expand gives for each layout.
template <ot::LayB LB, ot::EpiB E>
hipError_t launch_b(int tile, const ot::GemmBArgs& g, int64_t splits, hipStream_t st) {
  constexpr ot::LayB KM = ot::LayB::KMajor;
  if constexpr (LB == KM) {
    if (tile == ot::kB64x64) return ot::launch_gemm_bf16_pipe<64, 64, 64, 4, 2, KM, LB, E>(g, splits, st);
  }
  if (tile == ot::kB64x128) return ot::launch_gemm_bf16_pipe<64, 128, 64, 3, 4, KM, LB, E, 4>(g, splits, st);
  if (tile == ot::kB128x128) return ot::launch_gemm_bf16_pipe<128, 128, 32, 4, 2, KM, LB, E>(g, splits, st);
  if (tile == ot::kB256x256) return ot::launch_gemm_bf16_pp<4, KM, LB, E>(g, splits, st);
  return hipErrorInvalidValue;
}

template <ot::Lay LB, ot::Epi E>
hipError_t launch_x(int tile, const ot::GemmArgs& g, int64_t splits, hipStream_t st) {
  constexpr ot::Lay KM = ot::Lay::KMajor;
  if (tile == ot::kX64x64) return ot::launch_gemm_f32x3<2, 2, 1, 1, KM, LB, E>(g, splits, st);
  if (tile == ot::kX32x256) return ot::launch_gemm_f32x3<1, 4, 1, 2, KM, LB, E>(g, splits, st);
  if (tile == ot::kX64x256) return ot::launch_gemm_f32x3<1, 4, 2, 2, KM, LB, E>(g, splits, st);
  if constexpr (LB == KM) {
    if (tile == ot::kX64x128) return ot::launch_gemm_f32x3<2, 2, 1, 2, KM, LB, E>(g, splits, st);
  } else {
    if (tile == ot::kX128x128) return ot::launch_gemm_f32x3<2, 2, 2, 2, KM, LB, E>(g, splits, st);
  }
  return hipErrorInvalidValue;
}

template <class T, class G>
int reduce_splits(const Expand& e, const G& g, const ot::AdaptPlan& p, const float* part, hipStream_t st) {
  hipLaunchKernelGGL(ot::adapt_reduce_kernel<T>, dim3((unsigned)ot::ceil_div(e.M * ((e.N + 3) / 4), 256)), dim3(256), 0,
                     st, part, (int32_t)p.splits, g.split_stride, e.M, e.N, g.ldc, e.lr.perm,
                     static_cast<const T*>(e.lr.mask), e.lr.ldmask, static_cast<T*>(e.C), e.ldc);
  OT_LAUNCHED("adapt_reduce_kernel");
  return OT_OK;
}

// part: workspace of plan_values() floats.  Split products only as input gradients.
template <class G>
void fill_expand(G& g, const Expand& e, const ot::AdaptPlan& p, float* part) {
  g.lda = e.lda;
  g.ldb = e.ldb;
  g.ldc = e.ldc;
  g.M = e.M;
  g.N = e.N;
  g.K = e.K;
  g.bias = e.bias;
  g.lr = e.lr;
  g.k_chunk = p.k_chunk;
  if (p.splits > 1) {
    g.ldc = (e.N + 3) / 4 * 4;
    g.split_stride = e.M * g.ldc;
  }
}

int run_expand(const Expand& e, bool bf16, bool kmajor, float* part, hipStream_t st) {
  const ot::AdaptPlan p = ot::plan_expand(bf16, kmajor, e.M, e.N, e.K);
  hipError_t rc;
  if (bf16) {
    ot::GemmBArgs g{};
    fill_expand(g, e, p, part);
    g.A = static_cast<const uint16_t*>(e.A);
    g.B = static_cast<const uint16_t*>(e.B);
    g.C = p.splits > 1 ? part : e.C;
    if (kmajor)
      rc = e.c_type == OT_BF16 ? launch_b<ot::LayB::KMajor, ot::EpiB::AdaptBf>(p.tile, g, 1, st)
                               : launch_b<ot::LayB::KMajor, ot::EpiB::AdaptF32>(p.tile, g, 1, st);
    else if (p.splits > 1)
      rc = launch_b<ot::LayB::MNMajor, ot::EpiB::AdaptSplit>(p.tile, g, p.splits, st);
    else
      rc = launch_b<ot::LayB::MNMajor, ot::EpiB::AdaptBf>(p.tile, g, 1, st);
    if (rc == hipSuccess && p.splits > 1) return reduce_splits<uint16_t>(e, g, p, part, st);
  } else {
    ot::GemmArgs g{};
    fill_expand(g, e, p, part);
    g.A = static_cast<const float*>(e.A);
    g.B = static_cast<const float*>(e.B);
    g.C = p.splits > 1 ? part : static_cast<float*>(e.C);
    if (kmajor)
      rc = e.c_type == OT_BF16 ? launch_x<ot::Lay::KMajor, ot::Epi::AdaptBf>(p.tile, g, 1, st)
                               : launch_x<ot::Lay::KMajor, ot::Epi::AdaptF32>(p.tile, g, 1, st);
    else if (p.splits > 1)
      rc = launch_x<ot::Lay::MNMajor, ot::Epi::AdaptSplit>(p.tile, g, p.splits, st);
    else
      rc = launch_x<ot::Lay::MNMajor, ot::Epi::AdaptF32>(p.tile, g, 1, st);
    if (rc == hipSuccess && p.splits > 1) return reduce_splits<float>(e, g, p, part, st);
  }
  if (rc != hipSuccess)
    return ot::set_error(OT_E_HIP, "launch of the adapted product failed: %s", hipGetErrorString(rc));
  return OT_OK;
}

}  // namespace

extern "C" int adapters_create(ot_adapters** out, int64_t in, int64_t out_dim, int32_t rank, int32_t n_adapters,
                               int32_t precision, int64_t max_rows) {
  ot::clear_error();
  OT_REQUIRE(out != nullptr, "adapters_create: NULL out");
  *out = nullptr;
  OT_REQUIRE(in >= 1 && in <= (1LL << 26) && out_dim >= 1 && out_dim <= (1LL << 26),
             "adapters_create: in or out outside [1, 2^26]");
  OT_REQUIRE(rank >= 1 && rank <= 64, "adapters_create: rank outside [1, 64]");
  OT_REQUIRE(n_adapters >= 1 && n_adapters <= 4096, "adapters_create: n_adapters outside [1, 4096]");
  OT_REQUIRE(precision == OT_FP32 || precision == OT_BF16, "adapters_create: unknown precision");
  OT_REQUIRE(max_rows >= 1 && max_rows <= kMaxRows, "adapters_create: max_rows outside [1, 2^20]");
  int device = -1;
  OT_HIP(hipGetDevice(&device));
  ot_adapters* a = new (std::nothrow) ot_adapters();
  if (!a) return ot::set_error(OT_E_NOMEM, "adapters_create: out of host memory");
  a->in = in;
  a->out = out_dim;
  a->R = rank;
  a->RP = (rank + 15) / 16 * 16;
  a->G = n_adapters;
  a->precision = precision;
  a->device = device;
  a->max_rows = 0;
  const int rc = allocate(a, max_rows, "adapters_create");
  if (rc) {
    delete a;
    return rc;
  }
  *out = a;
  return OT_OK;
}

extern "C" int adapters_forward(ot_adapters* a, const void* x, int64_t ldx, const void* w, int64_t ldw,
                                const float* bias, const void* down, int64_t ldd, const void* up, int64_t ldu,
                                const float* scale, const int32_t* ids, int64_t n, void* y, int64_t ldy,
                                int32_t y_type, float* t, int64_t ldt, uint32_t flags, void* stream) try {
  ot::clear_error();
  const char* what = "adapters_forward";
  OT_REQUIRE(a != nullptr, "%s: NULL adapters", what);
  OT_REQUIRE(n >= 0 && n <= kMaxRows, "%s: n outside [0, 2^20]", what);
  OT_REQUIRE((flags & ~(uint32_t)OT_ADAPTERS_RELU) == 0, "%s: unknown flags", what);
  OT_REQUIRE(y_type == OT_FP32 || y_type == OT_BF16, "%s: y_type is neither OT_FP32 nor OT_BF16", what);
  if (n == 0) return OT_OK;
  const int e = a->precision == OT_BF16 ? 2 : 4;
  int rc;
  if ((rc = check_rows(x, ldx, n, a->in, e, what, "x"))) return rc;
  if ((rc = check_rows(w, ldw, a->out, a->in, e, what, "w"))) return rc;
  if ((rc = check_rows(down, ldd, (int64_t)a->G * a->R, a->in, e, what, "down"))) return rc;
  if ((rc = check_rows(up, ldu, (int64_t)a->G * a->R, a->out, e, what, "up"))) return rc;
  if ((rc = check_rows(y, ldy, n, a->out, y_type == OT_BF16 ? 2 : 4, what, "y"))) return rc;
  OT_REQUIRE(ids != nullptr, "%s: NULL ids", what);
  if ((rc = check_values(ids, 4, what, "ids"))) return rc;
  if ((rc = check_values(bias, 4, what, "bias"))) return rc;
  if ((rc = check_values(scale, 4, what, "scale"))) return rc;
  if ((rc = check_values(t, 4, what, "t"))) return rc;
  OT_REQUIRE(t == nullptr || n == 1 || ldt >= a->R, "%s: leading dimension of t below the rank", what);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if ((rc = begin_call(a, n, st, what))) return rc;
  Work wk;
  layout(a, n, a->ws, &wk);
  const ot::ShrinkArgs s{x,     ldx,     down,     ldd,     a->in, 0, a->G, a->R, a->RP, 0, 0,
                         scale, wk.perm, wk.slots, nullptr, wk.ts, t, ldt};
  rc = e == 2 ? run_shrink<uint16_t>(a, s, ids, n, wk, st) : run_shrink<float>(a, s, ids, n, wk, st);
  if (rc) return rc;
  const ot::AdaptRows lr{wk.perm, wk.gid, wk.off, wk.ts, up, ldu, a->G, a->R, a->RP,
                         (int32_t)(flags & OT_ADAPTERS_RELU ? 1 : 0), nullptr, 0};
  return run_expand(Expand{x, ldx, w, ldw, n, a->out, a->in, bias, y, ldy, y_type, lr}, e == 2, true, wk.part, st);
} catch (const std::bad_alloc&) {
  return ot::set_error(OT_E_NOMEM, "adapters_forward: out of host memory");
}

extern "C" int adapters_backward(ot_adapters* a, const void* x, int64_t ldx, const void* w, int64_t ldw,
                                 const void* down, int64_t ldd, const void* up, int64_t ldu, const float* scale,
                                 const int32_t* ids, int64_t n, const void* dy, int64_t lddy, const float* t,
                                 int64_t ldt, float* ddown, int64_t lddd, float* dup, int64_t lddu, void* dx,
                                 int64_t lddx, uint32_t flags, void* stream) try {
  ot::clear_error();
  const char* what = "adapters_backward";
  OT_REQUIRE(a != nullptr, "%s: NULL adapters", what);
  OT_REQUIRE(n >= 0 && n <= kMaxRows, "%s: n outside [0, 2^20]", what);
  OT_REQUIRE((flags & ~(uint32_t)OT_ADAPTERS_RELU_INPUT) == 0, "%s: unknown flags", what);
  const int e = a->precision == OT_BF16 ? 2 : 4;
  const int64_t gr = (int64_t)a->G * a->R;
  int rc;
  if ((rc = check_rows(ddown, lddd, gr, a->in, 4, what, "ddown"))) return rc;
  if ((rc = check_rows(dup, lddu, gr, a->out, 4, what, "dup"))) return rc;
  if (n > 0) {
    if ((rc = check_rows(x, ldx, n, a->in, e, what, "x"))) return rc;
    if ((rc = check_rows(up, ldu, gr, a->out, e, what, "up"))) return rc;
    if ((rc = check_rows(dy, lddy, n, a->out, e, what, "dy"))) return rc;
    if (dx) {
      if ((rc = check_rows(w, ldw, a->out, a->in, e, what, "w"))) return rc;
      if ((rc = check_rows(down, ldd, gr, a->in, e, what, "down"))) return rc;
      if ((rc = check_rows(dx, lddx, n, a->in, e, what, "dx"))) return rc;
    }
    OT_REQUIRE(ids != nullptr, "%s: NULL ids", what);
    OT_REQUIRE(t != nullptr, "%s: NULL t", what);
    OT_REQUIRE(n == 1 || ldt >= a->R, "%s: leading dimension of t below the rank", what);
    if ((rc = check_values(ids, 4, what, "ids"))) return rc;
    if ((rc = check_values(t, 4, what, "t"))) return rc;
    if ((rc = check_values(scale, 4, what, "scale"))) return rc;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  if ((rc = begin_call(a, n, st, what))) return rc;
  Work wk;
  layout(a, n, a->ws, &wk);
  const ot::OuterArgs ou{dy, lddy, a->out, t, ldt, 1, scale, a->R, wk.perm, wk.off, dup, lddu, 0};
  const ot::OuterArgs od{x, ldx, a->in, wk.ts, a->RP, 0, nullptr, a->R, wk.perm, wk.off, ddown, lddd, 0};
  if (n == 0) {
    if ((rc = run_group(a, ids, n, a->out, wk, st))) return rc;
    return e == 2 ? run_outer<uint16_t>(ou, od, n, a->G, st) : run_outer<float>(ou, od, n, a->G, st);
  }
  const bool pass = ot::pass_chunks(a->sizes(), n) > 0;
  if (pass) {
    if ((rc = run_group(a, ids, n, a->out, wk, st))) return rc;
    rc = e == 2 ? run_pass<uint16_t>(a, ou, up, ldu, n, wk, st) : run_pass<float>(a, ou, up, ldu, n, wk, st);
    if (rc) return rc;
    rc = e == 2 ? run_outer<uint16_t>(od, od, n, a->G, st, true) : run_outer<float>(od, od, n, a->G, st, true);
  } else {
    const ot::ShrinkArgs s{dy,    lddy,    up,       ldu,     a->out, 0, a->G, a->R, a->RP, 0, 0,
                           scale, wk.perm, wk.slots, nullptr, wk.ts, nullptr, 0};
    rc = e == 2 ? run_shrink<uint16_t>(a, s, ids, n, wk, st) : run_shrink<float>(a, s, ids, n, wk, st);
    if (rc) return rc;
    rc = e == 2 ? run_outer<uint16_t>(ou, od, n, a->G, st) : run_outer<float>(ou, od, n, a->G, st);
  }
  if (rc) return rc;
  if (!dx) return OT_OK;
  const ot::AdaptRows lr{wk.perm, wk.gid, wk.off, wk.ts, down, ldd, a->G, a->R, a->RP, 0,
                         flags & OT_ADAPTERS_RELU_INPUT ? x : nullptr, ldx};
  return run_expand(Expand{dy, lddy, w, ldw, n, a->in, a->out, nullptr, dx, lddx, a->precision, lr}, e == 2, false,
                    wk.part, st);
} catch (const std::bad_alloc&) {
  return ot::set_error(OT_E_NOMEM, "adapters_backward: out of host memory");
}

extern "C" int adapters_destroy(ot_adapters* a) {
  ot::clear_error();
  if (!a) return OT_OK;
  if (a->ws) (void)hipFree(a->ws);          // waits for the device
  for (unsigned char* p : a->kept) (void)hipFree(p);
  delete a;
  return OT_OK;
}
