// Global gradient norm over a list of tensors, clipping by it, and Adam with
// the clipped gradients (include/gradients.h).
//
// The list is cut into chunks of up to kChunk elements when it is created; a
// chunk is one block's unit of work, so a list of many small tensors and one
// of few large ones take the same two launches: partial sums of squares, then
// the elementwise pass, whose blocks each add the partials up themselves in the
// same fixed order (at most kParts of them, from the caches: cheaper than a
// third launch between the two, and nothing waits on another block).
//
// Bound by HBM: the norm reads every gradient once, clipping reads it again
// and writes it, Adam reads it again and reads and writes p, m, v.  103.6 M fp32 elements: norm 67 us
// (6.2 TB/s), clipping 122 (6.8 TB/s), Adam 485 (6.0 TB/s; a copy of 1 GiB reaches 5.2).  Chunks of
// 2048 elements slow the norm to 92 us, 1024 to 113 (two dependent loads ahead of each
// chunk's own).  96 tensors of 1.4 M elements in all: norm 3.2, clipping 4.7, Adam 11.9
// us, each a chain of dependent loads (partials or chunk, tensor, data).
// The squares are summed in 64 bits: the products are exact, cannot overflow or
// underflow, and the vector units have the rate to spare.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "adam.h"
#include "common.h"
#include "gradients.h"
#include "surrogate.h"

namespace ot {

constexpr int kChunk = 4096;      // elements
constexpr int kParts = 1024;      // partial sums, one per block of the norm's launch

struct ListTensor {
  const void* g;
  void* out;        // clip: destination
  float* p;         // Adam: parameters, moments, bf16 copy (nullable)
  float* m;
  float* v;
  uint16_t* copy;
  int32_t type;     // of g and out
  int32_t vec;      // elements that must precede the first 16-byte boundary of every array, or -1: none is common
};

struct ListChunk {
  int64_t offset;
  int32_t tensor;
  int32_t count;
};

// State that calls leave for later ones, in device memory: the steps taken, and
// whether the last enqueued step was one (added at the start of the next).
struct ListState {
  long long steps;
  long long pending;
};

__device__ __forceinline__ float list_bf2f(uint16_t h) { return __uint_as_float((uint32_t)h << 16); }
// round to nearest even, NaN stays NaN
__device__ __forceinline__ uint16_t list_f2bf(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

__device__ __forceinline__ double block_sum_256(double s, double* red) {
  s = warp_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  const double t = (red[0] + red[1]) + (red[2] + red[3]);
  __syncthreads();
  return t;
}

// Norm from the partials, the same bits in every block and call.
__device__ __forceinline__ float norm_from(const double* __restrict__ part, int n, double* red) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) s += part[i];
  return (float)sqrt(block_sum_256(s, red));
}

// min(1, max_norm / norm); 1 where the norm is 0 or not finite.
__device__ __forceinline__ float clip_coefficient(float norm, float max_norm) {
  return (norm > max_norm && norm <= 3.402823466e38f) ? max_norm / norm : 1.f;
}

// Elements [0, count) of a chunk as whole vectors of V (from index `head` on) and
// single elements around them.
struct Walk {
  int head, nv;
  __device__ __forceinline__ Walk(const ListTensor& t, const ListChunk& c, int V) {
    if (t.vec < 0) {
      head = c.count;
      nv = 0;
      return;
    }
    // chunks after a tensor's first start on a boundary
    head = min(c.offset == 0 ? t.vec : 0, c.count);
    nv = (c.count - head) / V;
  }
};

template <bool BF16>
__device__ __forceinline__ double chunk_squares(const ListTensor& t, const ListChunk& c) {
  constexpr int V = BF16 ? 8 : 4;
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const uint16_t* g16 = static_cast<const uint16_t*>(t.g) + c.offset;
  const float* g32 = static_cast<const float*>(t.g) + c.offset;
  const Walk w(t, c, V);
  double s = 0.0;
  auto one = [&](int i) {
    const double x = BF16 ? list_bf2f(g16[i]) : g32[i];
    s = fma(x, x, s);
  };
  auto add = [&](const u32x4 q) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (BF16) {
        const double a = __uint_as_float(q[e] << 16), b = __uint_as_float(q[e] & 0xffff0000u);
        s = fma(a, a, s);
        s = fma(b, b, s);
      } else {
        const double a = __uint_as_float(q[e]);
        s = fma(a, a, s);
      }
    }
  };
  const u32x4* v = reinterpret_cast<const u32x4*>(BF16 ? (const void*)(g16 + w.head) : (const void*)(g32 + w.head));
  int i = threadIdx.x;
  for (; i + 3 * 256 < w.nv; i += 4 * 256) {      // four loads in flight
    u32x4 q[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) q[u] = v[i + 256 * u];
#pragma unroll
    for (int u = 0; u < 4; ++u) add(q[u]);
  }
  for (; i < w.nv; i += 256) add(v[i]);
  for (int j = threadIdx.x; j < w.head; j += 256) one(j);
  for (int j = w.head + w.nv * V + threadIdx.x; j < c.count; j += 256) one(j);
  return s;
}

// part[block] = sum of squares of this block's chunks; block 0 also counts the
// step that the last call took (st, Adam lists).
__global__ __launch_bounds__(256) void norm_partial_kernel(const ListTensor* __restrict__ tensors,
                                                           const ListChunk* __restrict__ chunks, int64_t n_chunks,
                                                           double* __restrict__ part, ListState* __restrict__ st) {
  __shared__ double red[4];
  if (st && blockIdx.x == 0 && threadIdx.x == 0) {
    st->steps += st->pending;
    st->pending = 0;
  }
  double s = 0.0;
  for (int64_t k = blockIdx.x; k < n_chunks; k += gridDim.x) {
    const ListChunk c = chunks[k];
    const ListTensor t = tensors[c.tensor];
    s += t.type == OT_BF16 ? chunk_squares<true>(t, c) : chunk_squares<false>(t, c);
  }
  s = block_sum_256(s, red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(256) void norm_finish_kernel(const double* __restrict__ part, int n_parts,
                                                          float* __restrict__ norm_out) {
  __shared__ double red[4];
  const float norm = norm_from(part, n_parts, red);
  if (threadIdx.x == 0) *norm_out = norm;
}

template <bool BF16>
__device__ __forceinline__ void chunk_scale(const ListTensor& t, const ListChunk& c, float k) {
  constexpr int V = BF16 ? 8 : 4;
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const uint16_t* g16 = static_cast<const uint16_t*>(t.g) + c.offset;
  const float* g32 = static_cast<const float*>(t.g) + c.offset;
  uint16_t* o16 = static_cast<uint16_t*>(t.out) + c.offset;
  float* o32 = static_cast<float*>(t.out) + c.offset;
  const Walk w(t, c, V);
  auto one = [&](int i) {
    // k = 1 copies the bits as they are
    if constexpr (BF16) o16[i] = k == 1.f ? g16[i] : list_f2bf(k * list_bf2f(g16[i]));
    else o32[i] = k == 1.f ? g32[i] : k * g32[i];
  };
  auto scaled = [&](u32x4 q) {
    if (k == 1.f) return q;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (BF16) {
        const float a = __uint_as_float(q[e] << 16), b = __uint_as_float(q[e] & 0xffff0000u);
        q[e] = (uint32_t)list_f2bf(k * a) | ((uint32_t)list_f2bf(k * b) << 16);
      } else {
        q[e] = __float_as_uint(k * __uint_as_float(q[e]));
      }
    }
    return q;
  };
  const u32x4* v = reinterpret_cast<const u32x4*>(BF16 ? (const void*)(g16 + w.head) : (const void*)(g32 + w.head));
  u32x4* o = reinterpret_cast<u32x4*>(BF16 ? (void*)(o16 + w.head) : (void*)(o32 + w.head));
  int i = threadIdx.x;
  for (; i + 3 * 256 < w.nv; i += 4 * 256) {
    u32x4 q[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) q[u] = __builtin_nontemporal_load(v + i + 256 * u);
#pragma unroll
    for (int u = 0; u < 4; ++u) __builtin_nontemporal_store(scaled(q[u]), o + i + 256 * u);
  }
  for (; i < w.nv; i += 256) o[i] = scaled(v[i]);
  for (int j = threadIdx.x; j < w.head; j += 256) one(j);
  for (int j = w.head + w.nv * V + threadIdx.x; j < c.count; j += 256) one(j);
}

__global__ __launch_bounds__(256) void clip_kernel(const ListTensor* __restrict__ tensors,
                                                   const ListChunk* __restrict__ chunks, int64_t n_chunks,
                                                   const double* __restrict__ part, int n_parts, float max_norm,
                                                   float* __restrict__ norm_out) {
  __shared__ double red[4];
  const float norm = norm_from(part, n_parts, red);
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
  const float k = clip_coefficient(norm, max_norm);
  for (int64_t q = blockIdx.x; q < n_chunks; q += gridDim.x) {
    const ListChunk c = chunks[q];
    const ListTensor t = tensors[c.tensor];
    if (k == 1.f && t.out == t.g) continue;            // nothing to write
    if (t.type == OT_BF16) chunk_scale<true>(t, c, k);
    else chunk_scale<false>(t, c, k);
  }
}

// Counts the last call's step where no norm is formed.
__global__ void steps_kernel(ListState* __restrict__ st) {
  st->steps += st->pending;
  st->pending = 0;
}

// Adam over the list with gradients scaled by the coefficient.  n_parts = 0:
// no norm, no clipping.  The moments and parameters are touched once per step:
// non-temporal; four vectors of each array are in flight per thread.
__global__ __launch_bounds__(256) void adam_list_kernel(const ListTensor* __restrict__ tensors,
                                                        const ListChunk* __restrict__ chunks, int64_t n_chunks,
                                                        const double* __restrict__ part, int n_parts, float max_norm,
                                                        float* __restrict__ norm_out, ListState* __restrict__ st,
                                                        AdamArgs a) {
  __shared__ double red[4];
  float k = 1.f;
  if (n_parts > 0) {
    const float norm = norm_from(part, n_parts, red);
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
    if (!(norm <= 3.402823466e38f)) return;            // the same in every block: no step
    if (max_norm > 0.f) k = clip_coefficient(norm, max_norm);
  }
  // read by every block, advanced only by the next call's first launch
  const long long now = st->steps + 1;
  if (blockIdx.x == 0 && threadIdx.x == 0) st->pending = 1;
  a.c1 = bias_correction(a.b1, now);
  a.c2 = bias_correction(a.b2, now);

  for (int64_t q = blockIdx.x; q < n_chunks; q += gridDim.x) {
    const ListChunk c = chunks[q];
    const ListTensor t = tensors[c.tensor];
    const float* g = static_cast<const float*>(t.g) + c.offset;
    float* p = t.p + c.offset;
    float* m = t.m + c.offset;
    float* v = t.v + c.offset;
    uint16_t* pb = t.copy ? t.copy + c.offset : nullptr;
    const Walk w(t, c, 4);
    auto one = [&](int i) {
      float pi = p[i], mi = m[i], vi = v[i];
      adam1(pi, k * g[i], mi, vi, a);
      p[i] = pi;
      m[i] = mi;
      v[i] = vi;
      if (pb) pb[i] = list_f2bf(pi);
    };
    // w.head also aligns the copy to 8 bytes where there is one
    const f32x4* G = reinterpret_cast<const f32x4*>(g + w.head);
    f32x4* P = reinterpret_cast<f32x4*>(p + w.head);
    f32x4* M = reinterpret_cast<f32x4*>(m + w.head);
    f32x4* V = reinterpret_cast<f32x4*>(v + w.head);
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
    u16x4* PB = reinterpret_cast<u16x4*>(pb + w.head);
    constexpr int U = 4;
    for (int i = threadIdx.x; i < w.nv; i += U * 256) {
      f32x4 gg[U], pp[U], mm[U], vv[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int j = i + 256 * u;
        if (j < w.nv) {
          gg[u] = __builtin_nontemporal_load(G + j);
          pp[u] = __builtin_nontemporal_load(P + j);
          mm[u] = __builtin_nontemporal_load(M + j);
          vv[u] = __builtin_nontemporal_load(V + j);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int j = i + 256 * u;
        if (j < w.nv) {
          adam4(pp[u], k * gg[u], mm[u], vv[u], a);
          __builtin_nontemporal_store(pp[u], P + j);
          __builtin_nontemporal_store(mm[u], M + j);
          __builtin_nontemporal_store(vv[u], V + j);
          if (pb) PB[j] = u16x4{list_f2bf(pp[u][0]), list_f2bf(pp[u][1]), list_f2bf(pp[u][2]), list_f2bf(pp[u][3])};
        }
      }
    }
    for (int j = threadIdx.x; j < w.head; j += 256) one(j);
    for (int j = w.head + 4 * w.nv + threadIdx.x; j < c.count; j += 256) one(j);
  }
}

// What both kinds of list hold.
struct TensorList {
  int device = -1;
  int64_t n_chunks = 0;
  int parts = 0;                 // blocks of the norm's launch
  int blocks = 0;                // blocks of the elementwise pass
  unsigned char* mem = nullptr;  // one allocation: partials, state, tensors, chunks
  double* part = nullptr;
  ListState* state = nullptr;
  ListTensor* tensors = nullptr;
  ListChunk* chunks = nullptr;
};

// Elements before the first 16-byte boundary that all the given arrays share
// (element sizes 4 or 2), or -1.
struct SharedAlign {
  int head = -2;
  void add(const void* p, int elem, int align) {
    const int h = (int)((align - (int)(reinterpret_cast<uintptr_t>(p) % align)) % align) / elem;
    const int n = align / elem;      // heads that differ by whole vectors are alike
    if (head == -2) { head = h; period = n; }
    else if (n != period || h != head) head = -1;
  }
  int period = 0;
};

int list_build(TensorList& l, std::vector<ListTensor>& t, const int64_t* counts, const char* what) {
  std::vector<ListChunk> chunks;
  for (size_t i = 0; i < t.size(); ++i) {
    int64_t at = 0;
    while (at < counts[i]) {
      // the first chunk ends where the tensor's vectors do, so that later ones start on a boundary
      const int64_t want = at == 0 && t[i].vec > 0 ? kChunk - 8 + t[i].vec : kChunk;
      const int64_t c = std::min(want, counts[i] - at);
      chunks.push_back(ListChunk{at, (int32_t)i, (int32_t)c});
      at += c;
    }
  }
  l.n_chunks = (int64_t)chunks.size();
  l.parts = (int)std::max<int64_t>(1, std::min<int64_t>(kParts, l.n_chunks));
  l.blocks = (int)std::max<int64_t>(1, std::min<int64_t>(2048, l.n_chunks));
  OT_HIP(hipGetDevice(&l.device));
  const size_t bp = kParts * sizeof(double), bs = 256, bt = (t.size() * sizeof(ListTensor) + 255) / 256 * 256,
               bc = chunks.size() * sizeof(ListChunk) + 16;
  const hipError_t e = hipMalloc(reinterpret_cast<void**>(&l.mem), bp + bs + bt + bc);
  if (e != hipSuccess) {
    l.mem = nullptr;
    (void)hipGetLastError();
    return set_error(OT_E_NOMEM, "%s: hipMalloc of %zu bytes failed: %s", what, bp + bs + bt + bc, hipGetErrorString(e));
  }
  l.part = reinterpret_cast<double*>(l.mem);
  l.state = reinterpret_cast<ListState*>(l.mem + bp);
  l.tensors = reinterpret_cast<ListTensor*>(l.mem + bp + bs);
  l.chunks = reinterpret_cast<ListChunk*>(l.mem + bp + bs + bt);
  const ListState zero{0, 0};
  OT_HIP(hipMemcpy(l.state, &zero, sizeof zero, hipMemcpyHostToDevice));
  OT_HIP(hipMemcpy(l.tensors, t.data(), t.size() * sizeof(ListTensor), hipMemcpyHostToDevice));
  if (!chunks.empty())
    OT_HIP(hipMemcpy(l.chunks, chunks.data(), chunks.size() * sizeof(ListChunk), hipMemcpyHostToDevice));
  return OT_OK;
}

void list_free(TensorList& l) {
  if (l.mem) (void)hipFree(l.mem);
  l.mem = nullptr;
}

int list_device(const TensorList& l, const char* what) {
  int device = -1;
  OT_HIP(hipGetDevice(&device));
  if (device != l.device)
    return set_error(OT_E_STATE, "%s: device %d is current, the list was created on %d", what, device, l.device);
  return OT_OK;
}

// counts, and the total of all lists
int check_counts(int32_t n, const int64_t* counts, const char* what) {
  OT_REQUIRE(n >= 1 && n <= 65536, "%s: n outside [1, 65536]", what);
  OT_REQUIRE(counts != nullptr, "%s: NULL counts", what);
  int64_t total = 0;
  for (int32_t i = 0; i < n; ++i) {
    OT_REQUIRE(counts[i] >= 0 && counts[i] <= (1LL << 40), "%s: counts[%d] outside [0, 2^40]", what, i);
    total += counts[i];
    OT_REQUIRE(total <= (1LL << 40), "%s: more than 2^40 elements", what);
  }
  return OT_OK;
}

int check_array(const void* p, int64_t count, int elem, const char* what, const char* name, int32_t i) {
  if (count == 0) return OT_OK;
  OT_REQUIRE(p != nullptr, "%s: %s[%d] is NULL", what, name, i);
  OT_REQUIRE(reinterpret_cast<uintptr_t>(p) % elem == 0, "%s: %s[%d] is not aligned to its elements", what, name, i);
  return OT_OK;
}

int launch_norm(const TensorList& l, bool count_step, hipStream_t st) {
  hipLaunchKernelGGL(norm_partial_kernel, dim3(l.parts), dim3(256), 0, st, l.tensors, l.chunks, l.n_chunks, l.part,
                     count_step ? l.state : nullptr);
  OT_LAUNCHED("norm_partial_kernel");
  return OT_OK;
}

}  // namespace ot

struct ot_clip {
  ot::TensorList list;
};

struct ot_adam {
  ot::TensorList list;
  float lr, b1, b2, eps;
};

extern "C" int clip_create(ot_clip** out, int32_t n, const void* const* grads, void* const* outs,
                           const int64_t* counts, const int32_t* types) try {
  ot::clear_error();
  OT_REQUIRE(out != nullptr, "clip_create: NULL out");
  *out = nullptr;
  int rc = ot::check_counts(n, counts, "clip_create");
  if (rc) return rc;
  OT_REQUIRE(grads != nullptr, "clip_create: NULL grads");
  std::vector<ot::ListTensor> t((size_t)n);
  for (int32_t i = 0; i < n; ++i) {
    const int32_t type = types ? types[i] : (int32_t)OT_FP32;
    OT_REQUIRE(type == OT_FP32 || type == OT_BF16, "clip_create: types[%d] is neither OT_FP32 nor OT_BF16", i);
    const int elem = type == OT_BF16 ? 2 : 4;
    void* o = outs ? outs[i] : const_cast<void*>(grads[i]);
    if ((rc = ot::check_array(grads[i], counts[i], elem, "clip_create", "grads", i))) return rc;
    if ((rc = ot::check_array(o, counts[i], elem, "clip_create", "outs", i))) return rc;
    ot::SharedAlign a;
    a.add(grads[i], elem, 16);
    a.add(o, elem, 16);
    t[i] = ot::ListTensor{grads[i], o, nullptr, nullptr, nullptr, nullptr, type, a.head};
  }
  ot_clip* c = new ot_clip();
  if ((rc = ot::list_build(c->list, t, counts, "clip_create"))) {
    ot::list_free(c->list);
    delete c;
    return rc;
  }
  *out = c;
  return OT_OK;
} catch (const std::bad_alloc&) {
  return ot::set_error(OT_E_NOMEM, "clip_create: out of host memory");
}

extern "C" int clip_norm(ot_clip* c, float* norm_dev, void* stream) {
  ot::clear_error();
  OT_REQUIRE(c != nullptr, "clip_norm: NULL list");
  OT_REQUIRE(norm_dev != nullptr, "clip_norm: NULL norm_dev");
  int rc = ot::list_device(c->list, "clip_norm");
  if (rc) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if ((rc = ot::launch_norm(c->list, false, st))) return rc;
  hipLaunchKernelGGL(ot::norm_finish_kernel, dim3(1), dim3(256), 0, st, c->list.part, c->list.parts, norm_dev);
  OT_LAUNCHED("norm_finish_kernel");
  return OT_OK;
}

extern "C" int clip_apply(ot_clip* c, float max_norm, float* norm_dev, void* stream) {
  ot::clear_error();
  OT_REQUIRE(c != nullptr, "clip_apply: NULL list");
  OT_REQUIRE(std::isfinite(max_norm) && max_norm > 0.f, "clip_apply: max_norm is not a finite number above 0");
  int rc = ot::list_device(c->list, "clip_apply");
  if (rc) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if ((rc = ot::launch_norm(c->list, false, st))) return rc;
  hipLaunchKernelGGL(ot::clip_kernel, dim3(c->list.blocks), dim3(256), 0, st, c->list.tensors, c->list.chunks,
                     c->list.n_chunks, c->list.part, c->list.parts, max_norm, norm_dev);
  OT_LAUNCHED("clip_kernel");
  return OT_OK;
}

extern "C" int clip_destroy(ot_clip* c) {
  ot::clear_error();
  if (!c) return OT_OK;
  ot::list_free(c->list);        // hipFree waits for the device
  delete c;
  return OT_OK;
}

extern "C" int adam_create(ot_adam** out, int32_t n, float* const* params, const float* const* grads, float* const* m,
                           float* const* v, uint16_t* const* copies, const int64_t* counts, float lr, float beta1,
                           float beta2, float eps, int64_t steps) try {
  ot::clear_error();
  OT_REQUIRE(out != nullptr, "adam_create: NULL out");
  *out = nullptr;
  int rc = ot::check_counts(n, counts, "adam_create");
  if (rc) return rc;
  OT_REQUIRE(params && grads && m && v, "adam_create: NULL array");
  OT_REQUIRE(std::isfinite(lr), "adam_create: lr is not finite");
  OT_REQUIRE(beta1 >= 0.f && beta1 < 1.f && beta2 >= 0.f && beta2 < 1.f, "adam_create: betas outside [0, 1)");
  OT_REQUIRE(eps >= 0.f && std::isfinite(eps), "adam_create: eps is not a finite number of at least 0");
  OT_REQUIRE(steps >= 0, "adam_create: steps < 0");
  std::vector<ot::ListTensor> t((size_t)n);
  for (int32_t i = 0; i < n; ++i) {
    uint16_t* copy = copies ? copies[i] : nullptr;
    if ((rc = ot::check_array(params[i], counts[i], 4, "adam_create", "params", i))) return rc;
    if ((rc = ot::check_array(grads[i], counts[i], 4, "adam_create", "grads", i))) return rc;
    if ((rc = ot::check_array(m[i], counts[i], 4, "adam_create", "m", i))) return rc;
    if ((rc = ot::check_array(v[i], counts[i], 4, "adam_create", "v", i))) return rc;
    if (copy && (rc = ot::check_array(copy, counts[i], 2, "adam_create", "copies", i))) return rc;
    ot::SharedAlign a;
    a.add(params[i], 4, 16);
    a.add(grads[i], 4, 16);
    a.add(m[i], 4, 16);
    a.add(v[i], 4, 16);
    if (copy) a.add(copy, 2, 8);
    t[i] = ot::ListTensor{grads[i], nullptr, params[i], m[i], v[i], copy, (int32_t)OT_FP32, a.head};
  }
  ot_adam* o = new ot_adam();
  o->lr = lr;
  o->b1 = beta1;
  o->b2 = beta2;
  o->eps = eps;
  rc = ot::list_build(o->list, t, counts, "adam_create");
  if (rc == OT_OK) {
    const ot::ListState s{(long long)steps, 0};
    const hipError_t e = hipMemcpy(o->list.state, &s, sizeof s, hipMemcpyHostToDevice);
    if (e != hipSuccess) rc = ot::set_error(OT_E_HIP, "adam_create: hipMemcpy failed: %s", hipGetErrorString(e));
  }
  if (rc) {
    ot::list_free(o->list);
    delete o;
    return rc;
  }
  *out = o;
  return OT_OK;
} catch (const std::bad_alloc&) {
  return ot::set_error(OT_E_NOMEM, "adam_create: out of host memory");
}

extern "C" int adam_step(ot_adam* a, float max_norm, float* norm_dev, void* stream) {
  ot::clear_error();
  OT_REQUIRE(a != nullptr, "adam_step: NULL list");
  OT_REQUIRE(std::isfinite(max_norm) && max_norm >= 0.f, "adam_step: max_norm is not a finite number of at least 0");
  int rc = ot::list_device(a->list, "adam_step");
  if (rc) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool norm = max_norm > 0.f || norm_dev != nullptr;
  if (norm) {
    if ((rc = ot::launch_norm(a->list, true, st))) return rc;
  } else {
    hipLaunchKernelGGL(ot::steps_kernel, dim3(1), dim3(1), 0, st, a->list.state);
    OT_LAUNCHED("steps_kernel");
  }
  const ot::AdamArgs args{a->lr, a->b1, a->b2, a->eps, 0.f, 0.f, nullptr};
  hipLaunchKernelGGL(ot::adam_list_kernel, dim3(a->list.blocks), dim3(256), 0, st, a->list.tensors, a->list.chunks,
                     a->list.n_chunks, a->list.part, norm ? a->list.parts : 0, max_norm, norm_dev, a->list.state, args);
  OT_LAUNCHED("adam_list_kernel");
  return OT_OK;
}

extern "C" int adam_set_lr(ot_adam* a, float lr) {
  ot::clear_error();
  OT_REQUIRE(a != nullptr, "adam_set_lr: NULL list");
  OT_REQUIRE(std::isfinite(lr), "adam_set_lr: lr is not finite");
  a->lr = lr;
  return OT_OK;
}

extern "C" int adam_get_steps(ot_adam* a, int64_t* steps) {
  ot::clear_error();
  OT_REQUIRE(a != nullptr && steps != nullptr, "adam_get_steps: NULL argument");
  int rc = ot::list_device(a->list, "adam_get_steps");
  if (rc) return rc;
  OT_HIP(hipDeviceSynchronize());
  ot::ListState s{0, 0};
  OT_HIP(hipMemcpy(&s, a->list.state, sizeof s, hipMemcpyDeviceToHost));
  *steps = (int64_t)(s.steps + s.pending);
  return OT_OK;
}

extern "C" int adam_set_steps(ot_adam* a, int64_t steps) {
  ot::clear_error();
  OT_REQUIRE(a != nullptr, "adam_set_steps: NULL list");
  OT_REQUIRE(steps >= 0, "adam_set_steps: steps < 0");
  int rc = ot::list_device(a->list, "adam_set_steps");
  if (rc) return rc;
  OT_HIP(hipDeviceSynchronize());
  const ot::ListState s{(long long)steps, 0};
  OT_HIP(hipMemcpy(a->list.state, &s, sizeof s, hipMemcpyHostToDevice));
  return OT_OK;
}

extern "C" int adam_destroy(ot_adam* a) {
  ot::clear_error();
  if (!a) return OT_OK;
  ot::list_free(a->list);        // hipFree waits for the device
  delete a;
  return OT_OK;
}
