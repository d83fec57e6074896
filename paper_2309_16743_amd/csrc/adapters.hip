// Low-rank adapters beside a frozen projection (include/adapters.h).
//
// A call first sorts its rows by adapter (group_rows_kernel): position p of the
// sorted order is row perm[p] with adapter gid[p] (G: none).  Every later kernel
// works in sorted order and reads and writes the caller's rows through perm, so that rows of
// one adapter lie next to each other whatever order they came in.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "adapters.h"
#include "common.h"
#include "intmath.h"
#include "lowrank.h"
#include "surrogate.h"

namespace ot {

// Block g collects the rows of adapter g (block G: rows without one) in their
// order: it counts the rows of smaller keys, which is where its own start, and
// then writes them.  Every block reads all ids (n G / 64 wavefront reads from
// the caches) and none waits for another.  Slots: adapter g's first is
// start / kSlotRows + g, which leaves room for those of the adapters before it; those
// that stay unused get count 0.
__global__ __launch_bounds__(256) void group_rows_kernel(const int32_t* __restrict__ ids, int32_t n, int32_t G,
                                                         int32_t* __restrict__ perm, int32_t* __restrict__ gid,
                                                         int32_t* __restrict__ off, RowSlot* __restrict__ slots) {
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
  const int slot0 = start / kSlotRows + g, slot1 = (start + count) / kSlotRows + g + 1;
  for (int s = slot0 + tid; s < slot1; s += 256) {
    const int r = (s - slot0) * kSlotRows;
    slots[s] = RowSlot{start + r, max(0, min(kSlotRows, count - r)), g, 0};
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

struct ExpandArgs {
  const void* A;          // rows (through perm) of K values
  int64_t lda;
  const void* B;          // KMajor: N rows of K values; else K rows of N values
  int64_t ldb;
  int64_t M, N, K;
  const float* ts;        // sorted low-rank values, pitch RP
  const void* L;          // G x R rows of N values
  int64_t ldl;
  int32_t G, R, RP;
  const int32_t* perm;
  const int32_t* gid;
  const float* bias;      // nullable
  int32_t relu;
  const void* mask;       // rows by row number; the output is 0 where it is not above 0 (nullable)
  int64_t ldmask;
  void* C;
  int64_t ldc;
};

// C[row] = B A[row] (+ bias) + sum_r ts[r] L_g[r], 64 x 64 per block.
template <class T, class TC, bool KMAJOR>
__global__ __launch_bounds__(256) void expand_kernel(ExpandArgs a) {
  __shared__ float sa[16][65], sb[16][65];
  const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
  const int64_t tiles_m = (a.M + 63) / 64;
  const int64_t m0 = (blockIdx.x % tiles_m) * 64, n0 = (blockIdx.x / tiles_m) * 64;
  const T* A = static_cast<const T*>(a.A);
  const T* B = static_cast<const T*>(a.B);
  float acc[4][4] = {};
  for (int64_t k0 = 0; k0 < a.K; k0 += 16) {
    for (int i = tid; i < 1024; i += 256) {
      const int r = i / 16, k = i % 16;
      sa[k][r] = (m0 + r < a.M && k0 + k < a.K) ? lr_value(A + a.perm[m0 + r] * a.lda + k0 + k) : 0.f;
      if (KMAJOR) {
        sb[k][r] = (n0 + r < a.N && k0 + k < a.K) ? lr_value(B + (n0 + r) * a.ldb + k0 + k) : 0.f;
      } else {
        const int kk = i / 64, c = i % 64;
        sb[kk][c] = (n0 + c < a.N && k0 + kk < a.K) ? lr_value(B + (k0 + kk) * a.ldb + n0 + c) : 0.f;
      }
    }
    __syncthreads();
    for (int k = 0; k < 16; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][4 * ty + i], sb[k][tx + 16 * j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i) {
    const int64_t p = m0 + 4 * ty + i;
    if (p >= a.M) continue;
    const int64_t row = a.perm[p];
    const int g = a.gid[p];
    for (int j = 0; j < 4; ++j) {
      const int64_t n = n0 + tx + 16 * j;
      if (n >= a.N) continue;
      float v = acc[i][j];
      if (g < a.G)
        for (int r = 0; r < a.R; ++r)
          v = fmaf(a.ts[p * a.RP + r], lr_value(static_cast<const T*>(a.L) + ((int64_t)g * a.R + r) * a.ldl + n), v);
      if (a.bias) v += a.bias[n];
      if (a.relu) v = v > 0.f ? v : (v != v ? v : 0.f);
      if (a.mask && !(lr_value(static_cast<const T*>(a.mask) + row * a.ldmask + n) > 0.f)) v = 0.f;
      lr_store(static_cast<TC*>(a.C) + row * a.ldc + n, v);
    }
  }
}

}  // namespace ot

struct ot_adapters {
  int64_t in, out;
  int32_t R, RP, G, precision;
  int device;
  int64_t max_rows;
  // workspaces of calls of up to max_rows rows, in one allocation
  unsigned char* ws = nullptr;
  bool captured = false;                    // a captured call may name ws
  std::vector<unsigned char*> kept;         // workspaces replaced after such a call
};

namespace {

constexpr int64_t kMaxRows = 1LL << 20;

// Splits of the shrink's k range (length L) for n rows: enough blocks to fill the
// card, each with at least 16 steps per wavefront; one when the range is short,
// since the join costs a launch.  Blocks of unused slots (a large bank, few rows) are
// not multiplied without bound.
constexpr int64_t kShrinkBlocks = 1024;
int64_t shrink_splits(int64_t n, int64_t L, int32_t G) {
  if (L <= 4096) return 1;
  const int64_t slots = ot::ceil_div(n, ot::kSlotRows) + std::min<int64_t>(G, n) / 2;
  return std::max<int64_t>(1, std::min(std::min(ot::ceil_div(kShrinkBlocks, slots), L / 2048),
                                       32768 / (n / ot::kSlotRows + G + 1)));
}

struct Work {
  int32_t* perm;
  int32_t* gid;
  int32_t* off;
  ot::RowSlot* slots;
  float* ts;
  float* part;
  int64_t n_slots;
};

int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

// Workspace of a call of n rows at `base`; returns its size.
int64_t layout(const ot_adapters* a, int64_t n, unsigned char* base, Work* w) {
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    unsigned char* p = base + at;
    at += up256(bytes);
    return p;
  };
  Work t;
  t.n_slots = n / ot::kSlotRows + a->G + 1;
  t.perm = reinterpret_cast<int32_t*>(take(4 * n));
  t.gid = reinterpret_cast<int32_t*>(take(4 * n));
  t.off = reinterpret_cast<int32_t*>(take(4 * (a->G + 2)));
  t.slots = reinterpret_cast<ot::RowSlot*>(take((int64_t)sizeof(ot::RowSlot) * t.n_slots));
  t.ts = reinterpret_cast<float*>(take(4 * n * a->RP));
  // splits * rows of any call of up to n rows: splits <= kShrinkBlocks / (rows / 32) + 1
  const bool split = std::max(a->in, a->out) > 4096;
  t.part = reinterpret_cast<float*>(take(split ? 4 * (kShrinkBlocks * ot::kSlotRows + n) * a->RP : 0));
  if (w) *w = t;
  return at;
}

int allocate(ot_adapters* a, int64_t rows, const char* what) {
  unsigned char* p = nullptr;
  const int64_t bytes = layout(a, rows, nullptr, nullptr);
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

template <class T>
int run_shrink(ot::ShrinkArgs s, int64_t n, const Work& w, hipStream_t st) {
  const int64_t splits = shrink_splits(n, s.L, s.G);
  s.k_chunk = ot::ceil_div(ot::ceil_div(s.L, splits), ot::kShrinkUnit) * ot::kShrinkUnit;
  s.splits = (int32_t)ot::ceil_div(s.L, s.k_chunk);
  s.n = n;
  s.part = w.part;
  const dim3 grid((unsigned)w.n_slots, (unsigned)s.splits);
  switch (s.RP / 16) {
    case 1: hipLaunchKernelGGL((ot::shrink_kernel<T, 1>), grid, dim3(256), 0, st, s); break;
    case 2: hipLaunchKernelGGL((ot::shrink_kernel<T, 2>), grid, dim3(256), 0, st, s); break;
    case 3: hipLaunchKernelGGL((ot::shrink_kernel<T, 3>), grid, dim3(256), 0, st, s); break;
    default: hipLaunchKernelGGL((ot::shrink_kernel<T, 4>), grid, dim3(256), 0, st, s); break;
  }
  OT_LAUNCHED("shrink_kernel");
  if (s.splits > 1) {
    hipLaunchKernelGGL(ot::shrink_reduce_kernel, dim3((unsigned)w.n_slots), dim3(256), 0, st, s);
    OT_LAUNCHED("shrink_reduce_kernel");
  }
  return OT_OK;
}

template <class T, class TC, bool KMAJOR>
int run_expand(const ot::ExpandArgs& e, hipStream_t st) {
  const int64_t tiles = ot::ceil_div(e.M, 64) * ot::ceil_div(e.N, 64);
  hipLaunchKernelGGL((ot::expand_kernel<T, TC, KMAJOR>), dim3((unsigned)tiles), dim3(256), 0, st, e);
  OT_LAUNCHED("expand_kernel");
  return OT_OK;
}

template <class T, int NT>
int launch_outer(const ot::OuterArgs& o, int32_t G, hipStream_t st) {
  // short rows: the wavefronts of a block share its columns and split the rows
  const int64_t blocks = ot::ceil_div(o.L, 256) * G;
  if (blocks < 1024)
    hipLaunchKernelGGL((ot::outer_kernel<T, NT, true>), dim3((unsigned)ot::ceil_div(o.L, 64), (unsigned)G), dim3(256),
                       0, st, o);
  else
    hipLaunchKernelGGL((ot::outer_kernel<T, NT, false>), dim3((unsigned)ot::ceil_div(o.L, 256), (unsigned)G), dim3(256),
                       0, st, o);
  OT_LAUNCHED("outer_kernel");
  return OT_OK;
}

template <class T>
int run_outer(const ot::OuterArgs& o, int32_t G, hipStream_t st) {
  switch ((o.R + 15) / 16) {
    case 1: return launch_outer<T, 1>(o, G, st);
    case 2: return launch_outer<T, 2>(o, G, st);
    case 3: return launch_outer<T, 3>(o, G, st);
    default: return launch_outer<T, 4>(o, G, st);
  }
}

int run_group(const ot_adapters* a, const int32_t* ids, int64_t n, const Work& w, hipStream_t st) {
  hipLaunchKernelGGL(ot::group_rows_kernel, dim3((unsigned)(a->G + 1)), dim3(256), 0, st, ids, (int32_t)n, a->G,
                     w.perm, w.gid, w.off, w.slots);
  OT_LAUNCHED("group_rows_kernel");
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
  if ((rc = run_group(a, ids, n, wk, st))) return rc;
  const ot::ShrinkArgs s{x,     ldx,     down,     ldd,     a->in, 0, a->G, a->R, a->RP, 0, 0,
                         scale, wk.perm, wk.slots, nullptr, wk.ts, t, ldt};
  rc = e == 2 ? run_shrink<uint16_t>(s, n, wk, st) : run_shrink<float>(s, n, wk, st);
  if (rc) return rc;
  const ot::ExpandArgs ex{x,    ldx,     w,       ldw,  n,  a->out, a->in, wk.ts, up, ldu, a->G, a->R, a->RP,
                          wk.perm, wk.gid, bias, (int32_t)(flags & OT_ADAPTERS_RELU ? 1 : 0), nullptr, 0, y, ldy};
  if (e == 2)
    return y_type == OT_BF16 ? run_expand<uint16_t, uint16_t, true>(ex, st) : run_expand<uint16_t, float, true>(ex, st);
  return y_type == OT_BF16 ? run_expand<float, uint16_t, true>(ex, st) : run_expand<float, float, true>(ex, st);
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
  if ((rc = run_group(a, ids, n, wk, st))) return rc;
  if (n > 0) {
    const ot::ShrinkArgs s{dy,    lddy,    up,       ldu,     a->out, 0, a->G, a->R, a->RP, 0, 0,
                           scale, wk.perm, wk.slots, nullptr, wk.ts, nullptr, 0};
    rc = e == 2 ? run_shrink<uint16_t>(s, n, wk, st) : run_shrink<float>(s, n, wk, st);
    if (rc) return rc;
  }
  const ot::OuterArgs ou{dy, lddy, a->out, t, ldt, 1, scale, a->R, wk.perm, wk.off, dup, lddu};
  const ot::OuterArgs od{x, ldx, a->in, wk.ts, a->RP, 0, nullptr, a->R, wk.perm, wk.off, ddown, lddd};
  if ((rc = e == 2 ? run_outer<uint16_t>(ou, a->G, st) : run_outer<float>(ou, a->G, st))) return rc;
  if ((rc = e == 2 ? run_outer<uint16_t>(od, a->G, st) : run_outer<float>(od, a->G, st))) return rc;
  if (n == 0 || !dx) return OT_OK;
  const ot::ExpandArgs ex{dy,      lddy,   w,       ldw, n,
                          a->in,   a->out, wk.ts,   down, ldd,
                          a->G,    a->R,   a->RP,   wk.perm, wk.gid,
                          nullptr, 0,      flags & OT_ADAPTERS_RELU_INPUT ? x : nullptr, ldx, dx,
                          lddx};
  return e == 2 ? run_expand<uint16_t, uint16_t, false>(ex, st) : run_expand<float, float, false>(ex, st);
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
