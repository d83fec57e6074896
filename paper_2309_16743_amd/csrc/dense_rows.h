// Dense layer on few rows or few outputs (a request, a small batch, a narrow layer): the matrix instructions work
// straight from memory, without LDS; a block takes 16 outputs of up to 32 rows.
//
// The weights are the first operand of a 16 x 16 product, the rows of x the second: a lane reads 16 bytes of
// weight row n0 + l % 16 and 16 bytes of row l % 16 of x, and holds 4 neighbouring outputs 4 (l / 16) .. of one
// row.  (fp32: v_mfma_f32_16x16x4_f32 takes one k of a lane at a time; k = 4 (l / 16) + e in the e-th product, for
// both operands alike.)  The four wavefronts of a block share 16 outputs and take a quarter of k each, joined
// through LDS in a fixed order: many blocks from few outputs, and the latency of a long k in parallel.
// Measured (us, this and the tiled products): 1, 32 rows of 2048 x 2048 bf16 7 and 15, 9 and 17; 1 row of
// 2048 x 2048 fp32 9 and 57, of 1024 x 200000 fp32 139 and 198 (5.9 TB/s), of 65536 inputs and 64 outputs bf16
// 76 and 347.  With more rows the loads of x, once for every 16 outputs, bound it (1000000 x 1024 bf16 on 1, 4, 16, 32
// rows 325, 376, 515, 760, tiled 350, 351, 393, 419), so direct_layer bounds them; a piece of x for 64
// outputs at once was no faster than the tiles (391 on 4 rows, 485 on 32).
#pragma once

#include "layer_ops.h"
#include "lowrank_ops.h"

namespace ot {

struct RowsArgs {
  const void* x;
  int64_t ldx;
  const void* w;
  int64_t ldw;
  int64_t M, N, K;
  const float* bias;        // nullable
  void* y;
  int64_t ldy;
  LayerArgs ly;
};

template <class T>
struct RowsStep;
template <>
struct RowsStep<uint16_t> {
  static constexpr int K = 32;                           // k of one step, 16 bytes a lane
  typedef lr_bf16x8 V;
  static __device__ __forceinline__ void mul(V w, V x, f32x4& acc) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, acc, 0, 0, 0);
  }
};
template <>
struct RowsStep<float> {
  static constexpr int K = 16;
  typedef f32x4 V;
  static __device__ __forceinline__ void mul(V w, V x, f32x4& acc) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x[e], acc, 0, 0, 0);
  }
};

// MB: 16-row blocks of x; Y: type of y.
template <class T, class Y, int MB>
__global__ __launch_bounds__(256) void dense_rows_kernel(RowsArgs a) {
  typedef RowsStep<T> S;
  typedef typename S::V V;
  constexpr int E = 16 / sizeof(T), KS = 4, U = 8;
  __shared__ f32x4 s_acc[KS - 1][MB][64];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = 16 * (int64_t)blockIdx.x, m0 = 16 * MB * (int64_t)blockIdx.y;
  const int64_t steps = (a.K + S::K - 1) / S::K, each = (steps + KS - 1) / KS;
  const int64_t k0 = min(a.K, wid * each * S::K), k1 = min(a.K, k0 + each * S::K);
  const int kl = E * (lane / 16);
  const T* w = static_cast<const T*>(a.w) + min(n0 + lane % 16, a.N - 1) * a.ldw + kl;
  const T* x[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) x[b] = static_cast<const T*>(a.x) + min(m0 + 16 * b + lane % 16, a.M - 1) * a.ldx + kl;
  f32x4 acc[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  int64_t k = k0;
  for (; k + U * S::K <= k1; k += U * S::K) {
    V wv[U], xv[U][MB];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      wv[u] = *reinterpret_cast<const V*>(w + k + u * S::K);
#pragma unroll
      for (int b = 0; b < MB; ++b) xv[u][b] = *reinterpret_cast<const V*>(x[b] + k + u * S::K);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int b = 0; b < MB; ++b) S::mul(wv[u], xv[u][b], acc[b]);
  }
  for (; k < k1; k += S::K) {                            // the rest; zeros past the rows' ends
    const V wv = __builtin_bit_cast(V, lr_load16(w + k, a.K - k - kl));
#pragma unroll
    for (int b = 0; b < MB; ++b) S::mul(wv, __builtin_bit_cast(V, lr_load16(x[b] + k, a.K - k - kl)), acc[b]);
  }
  if (wid > 0)
#pragma unroll
    for (int b = 0; b < MB; ++b) s_acc[wid - 1][b][lane] = acc[b];
  __syncthreads();
  if (wid > 0) return;
#pragma unroll
  for (int b = 0; b < MB; ++b)
#pragma unroll
    for (int q = 0; q < KS - 1; ++q) acc[b] += s_acc[q][b][lane];
  const int64_t n = n0 + 4 * (lane / 16);
  if (n >= a.N) return;
  const int cnt = (int)min((int64_t)4, a.N - n);
  float bias[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) bias[c] = a.bias && c < cnt ? a.bias[n + c] : 0.f;
  auto put = [&](auto* p, const f32x4& v) {
    if constexpr (sizeof(*p) == 4) {
      if (cnt == 4) *reinterpret_cast<f32x4*>(p) = v;
      else
        for (int c = 0; c < cnt; ++c) p[c] = v[c];
    } else {
      if (cnt == 4) {
        *reinterpret_cast<lr_u32x2*>(p) = lr_u32x2{(uint32_t)lr_bf16(v[0]) | ((uint32_t)lr_bf16(v[1]) << 16),
                                                   (uint32_t)lr_bf16(v[2]) | ((uint32_t)lr_bf16(v[3]) << 16)};
      } else {
        for (int c = 0; c < cnt; ++c) p[c] = lr_bf16(v[c]);
      }
    }
  };
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const int64_t m = m0 + 16 * b + lane % 16;
    if (m >= a.M) continue;
    f32x4 v = acc[b];
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] += bias[c];
    if (a.ly.pre) put(static_cast<T*>(a.ly.pre) + m * a.ly.ldp + n, v);
    act_values<4>(v, a.ly.act);
    if (a.ly.residual) {
      const Y* r = static_cast<const Y*>(a.ly.residual) + m * a.ly.ldr + n;
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (c < cnt) v[c] += lr_value(r + c);
    }
    put(static_cast<Y*>(a.y) + m * a.ldy + n, v);
  }
}

}  // namespace ot
