// Group norm with an activation over channels-last data (include/layers.h).
//
// Three forms (norm_plan.h).  Up to 4 positions, groups of whole vectors of 8 channels: in registers of a team of
// lanes.  Few positions otherwise: a block keeps some of a sample's groups in LDS.  Both read x once: mean, the
// squares of the differences from it, the results.  Many positions, or longer groups, take three launches: partial
// moments per chunk of positions and channel, their join per sample and group, the results (x is read twice,
// the second time from the Infinity Cache where it fits).  No atomics: every sum has a fixed order.
#include <cmath>
#include <new>

#include "layer_host.h"
#include "layer_ops.h"
#include "layers.h"
#include "norm_plan.h"
#include "row_ops.h"
#include "surrogate.h"

namespace ot {

struct NormArgs {
  const void* x;
  int64_t ldx;
  const void* dy;           // backward
  int64_t lddy;
  void* out;                // y or dx (backward: nullable)
  int64_t ldo;
  const float* weight;      // nullable
  const float* bias;        // nullable
  const float* stats;       // backward: mean and rstd per sample and group
  float* stats_out;         // forward (nullable)
  int64_t n, positions, channels;
  int32_t groups, per;
  float eps;
};

// Sum over a team of S threads (S a power of two up to 256, teams aligned in the block), the same value to all; s:
// four values per block, for teams of several wavefronts.  All threads of the block call it together.
template <class V>
__device__ __forceinline__ V team_sum(V v, int S, V* s) {
  for (int o = 1; o < S && o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
  if (S > 64) {                                          // the same for the whole block
    const int wid = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) s[wid] = v;
    __syncthreads();
    if (S == 256) v = (s[0] + s[1]) + (s[2] + s[3]);
    else v = s[wid & 2] + s[(wid & 2) + 1];
    __syncthreads();
  }
  return v;
}

// What a block over slabs does with its groups: teams of S threads take one group after the
// other; in a team CL threads lie side by side along the channels.
struct Teams {
  int S, CL, teams;
  __device__ __forceinline__ Teams(int groups, int per) {
    S = 256;
    while (S > 1 && 256 / S < groups) S >>= 1;
    CL = 1;
    while (CL < S && CL < per) CL <<= 1;
    teams = 256 / S;
  }
};

// f(element index in the slab, channel in the block) over the values of group gi.
template <class F>
__device__ __forceinline__ void team_each(const Teams& t, int gi, int per, int positions, int width, F f) {
  const int me = threadIdx.x % t.S, c0 = me % t.CL, p0 = me / t.CL, dp = t.S / t.CL;
  for (int p = p0; p < positions; p += dp)
    for (int c = c0; c < per; c += t.CL) f(p * width + gi * per + c, gi * per + c);
}

// 8 values of a parameter (any alignment), or 8 times `missing`.
__device__ __forceinline__ void load_param(const float* p, int64_t c, float missing, float (&v)[8]) {
  if (p == nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = missing;
  } else if (reinterpret_cast<uintptr_t>(p) % 16 == 0) {  // the same for all
    load8(p + c, 8, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = p[c + e];
  }
}

// Groups of whole vectors of 8 channels, up to 4 vectors a lane: a team of S lanes keeps a sample's group in
// registers, since LDS would add its latency to each of three sums.  1024 x 2048 bf16 in 32 groups, silu: 6.0 us, 19
// over slabs; what is left is one latency of memory and three of shuffles.
template <class T, int ACT, int V>
__global__ __launch_bounds__(256) void norm_team_kernel(NormArgs a, int S) {
  const int lane = threadIdx.x % S, pv = a.per / 8, vecs = (int)a.positions * pv;
  const float inv = 1.f / (float)(a.per * (int)a.positions);
  const int64_t teams = a.n * a.groups;
  // all lanes of a wavefront take part in every turn
  for (int64_t t0 = (int64_t)blockIdx.x * (256 / S); t0 < teams; t0 += (int64_t)gridDim.x * (256 / S)) {
    const int64_t q = t0 + threadIdx.x / S;
    const bool in = q < teams;
    int64_t g;
    const int64_t s = quotient(in ? q : 0, a.groups, g);
    float v[V][8];
    int64_t at[V];                                       // row, channel of each vector
    int ch[V];
    bool has[V];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int k = lane + S * i;
      has[i] = in && k < vecs;
      const int p = has[i] ? k / pv : 0;
      at[i] = s * a.positions + p;
      ch[i] = (int)g * a.per + 8 * (has[i] ? k - p * pv : 0);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
      if (has[i]) load8(static_cast<const T*>(a.x) + at[i] * a.ldx + ch[i], 8, v[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += v[i][e];
    }
    float w[V][8], b[V][8];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      load_param(a.weight, ch[i], 1.f, w[i]);
      load_param(a.bias, ch[i], 0.f, b[i]);
    }
    auto total = [&](float x) {
      for (int o = 1; o < S; o <<= 1) x += __shfl_xor(x, o, 64);
      return x;
    };
    float mean = total(sum) * inv;
    sum = 0.f;                                           // what the rounded sum left
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (has[i])
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[i][e] - mean;
    mean += total(sum) * inv;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (has[i])
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[i][e] -= mean;
          sum = fmaf(v[i][e], v[i][e], sum);
        }
    const float rstd = 1.f / sqrtf(total(sum) * inv + a.eps);
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (has[i]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = act_value<ACT>(fmaf(v[i][e] * rstd, w[i][e], b[i][e]));
        store8(static_cast<T*>(a.out) + at[i] * a.ldo + ch[i], 8, v[i]);
      }
    if (in && lane == 0 && a.stats_out) {
      a.stats_out[2 * q] = mean;
      a.stats_out[2 * q + 1] = rstd;
    }
  }
}

// The same for the backward, with one position: a block takes tg groups, its 256 / (S tg) rows of teams each their
// samples of the range; sums[0 / 1][range][channel] receive the range's sums of dp xh and dp (nullable).  The next
// sample's values are under way while one is worked on.
template <class T, int ACT, int V>
__global__ __launch_bounds__(256) void norm_team_back_kernel(NormArgs a, int S, int tg, int64_t tiles, int64_t ranges,
                                                             float* sums) {
  __shared__ float s_part[256][8];
  const int lane = threadIdx.x % S, team = threadIdx.x / S, pv = a.per / 8;
  const int ts = 256 / S / tg, row = team / tg;
  const int64_t tile = blockIdx.x % tiles, range = blockIdx.x / tiles;
  const int64_t g = tile * tg + team % tg;
  const bool in = g < a.groups;
  const float inv = 1.f / (float)a.per;
  int64_t ch[V];
  bool has[V];
  float w[V][8], b[V][8], sw[V][8], sb[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    has[i] = in && lane + S * i < pv;
    ch[i] = has[i] ? g * a.per + 8 * (lane + S * i) : 0;
    load_param(a.weight, ch[i], 1.f, w[i]);
    load_param(a.bias, ch[i], 0.f, b[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (!has[i]) w[i][e] = 1.f;                        // (idle lanes join the team's sums: 0 times channel 0's infinity)
      sw[i][e] = sb[i][e] = 0.f;
    }
  }
  auto total = [&](float x) {
    for (int o = 1; o < S; o <<= 1) x += __shfl_xor(x, o, 64);
    return x;
  };
  float x[V][8], d[V][8], mean = 0.f, rstd = 0.f;
  auto load = [&](int64_t s) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = d[i][e] = 0.f;
      if (has[i]) {
        load8(static_cast<const T*>(a.x) + s * a.ldx + ch[i], 8, x[i]);
        load8(static_cast<const T*>(a.dy) + s * a.lddy + ch[i], 8, d[i]);
      }
    }
    if (in) {
      mean = a.stats[(s * a.groups + g) * 2];
      rstd = a.stats[(s * a.groups + g) * 2 + 1];
    }
  };
  const int64_t s0 = a.n * range / ranges, s1 = a.n * (range + 1) / ranges;
  // every team takes part in every turn; past the range it works on zeros
  int64_t s = s0 + row;
  if (s < s1) load(s);
  for (int64_t turn = s0; turn < s1; turn += ts, s += ts) {
    const bool live = s < s1;
    const float r = rstd;
    float xh[V][8], dp[V][8], c1 = 0.f, c2 = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool use = live && has[i];
        xh[i][e] = use ? (x[i][e] - mean) * r : 0.f;
        dp[i][e] = use ? act_back<ACT>(d[i][e], fmaf(xh[i][e], w[i][e], b[i][e])) : 0.f;
      }
    if (s + ts < s1) load(s + ts);
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sw[i][e] = fmaf(dp[i][e], xh[i][e], sw[i][e]);
        sb[i][e] += dp[i][e];
        dp[i][e] *= w[i][e];
        c1 += dp[i][e];
        c2 = fmaf(dp[i][e], xh[i][e], c2);
      }
    if (a.out) {
      c1 = total(c1) * inv;
      c2 = total(c2) * inv;
      if (live)
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (has[i]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) dp[i][e] = r * ((dp[i][e] - c1) - xh[i][e] * c2);
            store8(static_cast<T*>(a.out) + s * a.ldo + ch[i], 8, dp[i]);
          }
    }
  }
  if (!sums) return;
  // rows of teams hold the same channels: joined pairwise
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float (&v)[8] = k ? sb[i] : sw[i];
      for (int h = ts / 2; h > 0; h /= 2) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) s_part[threadIdx.x][e] = v[e];
        __syncthreads();
        if (row < h)
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += s_part[threadIdx.x + h * tg * S][e];
      }
      if (row == 0 && has[i]) {
        float* o = sums + (k * ranges + range) * a.channels + ch[i];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = v[e];
      }
    }
}

// A block's slab: sample s, groups g0 .., `width` channels from c0 on.  f(row, vector's channel in the block, values
// of it that exist) over its vectors of 8 channels.
template <class F>
__device__ __forceinline__ void slab_each(int width, int positions, F f) {
  const int vecs = (width + 7) / 8;
  for (int i = threadIdx.x; i < vecs * positions; i += 256) {
    const int p = i / vecs, c = i % vecs * 8;
    f(p, c, width - c);
  }
}

template <class T>
__device__ __forceinline__ void slab_load(const T* p, bool aligned, int left, float (&v)[8]) {
  if (aligned) {
    load8(p, left, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? lr_value(p + e) : 0.f;
  }
}
template <class T>
__device__ __forceinline__ void slab_store(T* p, bool aligned, int left, const float (&v)[8]) {
  if (aligned) {
    store8(p, left, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) lr_store(p + e, v[e]);
  }
}

template <class T, int ACT>
__global__ __launch_bounds__(256) void norm_slab_kernel(NormArgs a, int gb, int64_t parts) {
  extern __shared__ float s_dyn[];                         // slab_values()
  __shared__ float s_red[4];
  const int P = (int)a.positions;
  float* const tile = s_dyn;
  float* const s_mean = tile + gb * a.per * P;
  float* const s_rstd = s_mean + gb;
  for (int64_t b = blockIdx.x; b < a.n * parts; b += gridDim.x) {
    const int64_t s = b / parts, g0 = b % parts * gb;
    const int groups = (int)min((int64_t)gb, a.groups - g0), width = groups * a.per;
    const int64_t c0 = g0 * a.per;
    const bool aligned = c0 % 8 == 0;
    const T* x = static_cast<const T*>(a.x) + s * P * a.ldx + c0;
    slab_each(width, P, [&](int p, int c, int left) {
      float v[8];
      slab_load(x + p * a.ldx + c, aligned, left, v);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) tile[p * width + c + e] = v[e];
    });
    __syncthreads();
    const Teams t(groups, a.per);
    const float inv = 1.f / (float)(a.per * P);
    for (int i = 0; i < groups; i += t.teams) {            // every team takes part in every turn
      const int gi = i + threadIdx.x / t.S;
      const bool in = gi < groups;
      float sum = 0.f;
      if (in) team_each(t, gi, a.per, P, width, [&](int k, int) { sum += tile[k]; });
      float mean = team_sum(sum, t.S, s_red) * inv;
      // what the rounded sum left: the mean of the differences
      sum = 0.f;
      if (in) team_each(t, gi, a.per, P, width, [&](int k, int) { sum += tile[k] - mean; });
      mean += team_sum(sum, t.S, s_red) * inv;
      sum = 0.f;
      if (in)
        team_each(t, gi, a.per, P, width, [&](int k, int) {
          const float d = tile[k] - mean;
          sum = fmaf(d, d, sum);
        });
      const float var = team_sum(sum, t.S, s_red) * inv;
      if (in && threadIdx.x % t.S == 0) {
        const float rstd = 1.f / sqrtf(var + a.eps);
        s_mean[gi] = mean;
        s_rstd[gi] = rstd;
        if (a.stats_out) {
          float* o = a.stats_out + (s * a.groups + g0 + gi) * 2;
          o[0] = mean;
          o[1] = rstd;
        }
      }
    }
    __syncthreads();
    T* y = static_cast<T*>(a.out) + s * P * a.ldo + c0;
    slab_each(width, P, [&](int p, int c, int left) {
      float v[8];
      int gi = c / a.per, end = (gi + 1) * a.per;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = 0.f;
        if (e < left) {
          if (c + e >= end) {
            ++gi;
            end += a.per;
          }
          const float xh = (tile[p * width + c + e] - s_mean[gi]) * s_rstd[gi];
          const int64_t ch = c0 + c + e;
          v[e] = act_value<ACT>(fmaf(xh, a.weight ? a.weight[ch] : 1.f, a.bias ? a.bias[ch] : 0.f));
        }
      }
      slab_store(y + p * a.ldo + c, aligned, left, v);
    });
    __syncthreads();
  }
}

// Block (range r of `ranges`, part of the groups): its samples one after the other; sums[0 / 1][range][channel]
// receive the range's sums of dp xh and dp (nullable).
template <class T, int ACT>
__global__ __launch_bounds__(256) void norm_slab_back_kernel(NormArgs a, int gb, int64_t parts, int64_t ranges,
                                                             float* sums) {
  extern __shared__ float s_dyn[];                         // slab_values()
  __shared__ float s_red[4];
  const int P = (int)a.positions, full = gb * a.per;
  float* const t_dp = s_dyn;
  float* const t_xh = t_dp + full * P;
  float* const s_w = t_xh + full * P;                      // sums of the range so far
  float* const s_b = s_w + full;
  float* const s_c1 = s_b + full;
  float* const s_c2 = s_c1 + gb;
  const int64_t part = blockIdx.x % parts, range = blockIdx.x / parts;
  const int64_t g0 = part * gb, c0 = g0 * a.per;
  const int groups = (int)min((int64_t)gb, a.groups - g0), width = groups * a.per;
  const bool aligned = c0 % 8 == 0;
  const int64_t s0 = a.n * range / ranges, s1 = a.n * (range + 1) / ranges;
  const Teams t(groups, a.per);
  const float inv = 1.f / (float)(a.per * P);
  for (int c = threadIdx.x; c < width; c += 256) s_w[c] = s_b[c] = 0.f;
  for (int64_t s = s0; s < s1; ++s) {
    const T* x = static_cast<const T*>(a.x) + s * P * a.ldx + c0;
    const T* dy = static_cast<const T*>(a.dy) + s * P * a.lddy + c0;
    const float* st = a.stats + (s * a.groups + g0) * 2;
    __syncthreads();
    slab_each(width, P, [&](int p, int c, int left) {
      float v[8], d[8];
      slab_load(x + p * a.ldx + c, aligned, left, v);
      slab_load(dy + p * a.lddy + c, aligned, left, d);
      int gi = c / a.per, end = (gi + 1) * a.per;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) {
          if (c + e >= end) {
            ++gi;
            end += a.per;
          }
          const int64_t ch = c0 + c + e;
          const float xh = (v[e] - st[2 * gi]) * st[2 * gi + 1];
          t_xh[p * width + c + e] = xh;
          t_dp[p * width + c + e] =
              act_back<ACT>(d[e], fmaf(xh, a.weight ? a.weight[ch] : 1.f, a.bias ? a.bias[ch] : 0.f));
        }
    });
    __syncthreads();
    if (sums)
      for (int c = threadIdx.x; c < width; c += 256) {
        float w = s_w[c], bsum = s_b[c];
        for (int p = 0; p < P; ++p) {
          const float d = t_dp[p * width + c];
          w = fmaf(d, t_xh[p * width + c], w);
          bsum += d;
        }
        s_w[c] = w;
        s_b[c] = bsum;
      }
    if (!a.out) continue;
    for (int i = 0; i < groups; i += t.teams) {
      const int gi = i + threadIdx.x / t.S;
      const bool in = gi < groups;
      float c1 = 0.f, c2 = 0.f;
      if (in)
        team_each(t, gi, a.per, P, width, [&](int k, int c) {
          const float d = t_dp[k] * (a.weight ? a.weight[c0 + c] : 1.f);
          c1 += d;
          c2 = fmaf(d, t_xh[k], c2);
        });
      c1 = team_sum(c1, t.S, s_red) * inv;
      c2 = team_sum(c2, t.S, s_red) * inv;
      if (in && threadIdx.x % t.S == 0) {
        s_c1[gi] = c1;
        s_c2[gi] = c2;
      }
    }
    __syncthreads();
    T* dx = static_cast<T*>(a.out) + s * P * a.ldo + c0;
    slab_each(width, P, [&](int p, int c, int left) {
      float v[8];
      int gi = c / a.per, end = (gi + 1) * a.per;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = 0.f;
        if (e < left) {
          if (c + e >= end) {
            ++gi;
            end += a.per;
          }
          const int k = p * width + c + e;
          const float d = t_dp[k] * (a.weight ? a.weight[c0 + c + e] : 1.f);
          v[e] = st[2 * gi + 1] * ((d - s_c1[gi]) - t_xh[k] * s_c2[gi]);
        }
      }
      slab_store(dx + p * a.ldo + c, aligned, left, v);
    });
  }
  if (sums) {
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += 256) {
      sums[range * a.channels + c0 + c] = s_w[c];
      sums[(ranges + range) * a.channels + c0 + c] = s_b[c];
    }
  }
}

// Where block b of a split pass stands.
struct NormSpot {
  int64_t tile, sample, chunk, r0, r1, c;      // rows r0 .. r1 of the data; this thread's first channel
  int rx, lanes;                         // its row among those side by side
  __device__ __forceinline__ NormSpot(const NormArgs& a, const NormPlan& p, int64_t b) {
    const int64_t q = quotient(b, p.tiles, tile);
    sample = quotient(q, p.chunks, chunk);
    lanes = 256 / p.col_threads;
    rx = threadIdx.x / p.col_threads;
    c = 8 * (tile * p.col_threads + threadIdx.x % p.col_threads);
    r0 = sample * a.positions + chunk * p.rows;
    r1 = sample * a.positions + min(a.positions, (chunk + 1) * p.rows);
  }
};

// Mean and sum of squared differences of `na` and `nb` values (Chan, Golub, LeVeque: updating formulae for
// sample variances).
__device__ __forceinline__ void join_moments(float& mean, float& m2, float na, float mean_b, float m2_b, float nb) {
  const float d = mean_b - mean, f = nb / (na + nb);
  mean = fmaf(d, f, mean);
  m2 = m2 + m2_b + d * d * (na * f);
}

// The split passes stream x (and dy) in rows of 16-byte pieces.  64 x 10000 x 64 bf16, relu: moments 18 us
// (4.5 TB/s), results 30 (5.4 TB/s); sums of the backward 46, dx 44 (5.6 TB/s).  Joining the partial sums at the start of every
// block that needs them took 11 us more than the launch it saved.
// Moments of every channel of a chunk: [sample][chunk][channel] mean, then the sums of squares.  A thread's
// rows are few, and it sums differences from the first of them, so that little cancels.
template <class T>
__global__ __launch_bounds__(256) void norm_moments_kernel(NormArgs a, NormPlan p, float* part) {
  __shared__ float s_m[256][9], s_q[256][9];
  const int64_t blocks = a.n * p.chunks * p.tiles;
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const NormSpot at(a, p, b);
    const int64_t left = a.channels - at.c;
    float first[8], s1[8], s2[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) first[e] = s1[e] = s2[e] = 0.f;
    int mine = 0;
    if (left > 0) {
      const T* x = static_cast<const T*>(a.x) + at.c;
      const int64_t r0 = at.r0 + at.rx;
      if (r0 < at.r1) load8(x + r0 * a.ldx, left, first);
      constexpr int U = 4;
      float v[U][8];
      rows_in_groups<U>(
          r0, at.r1, at.lanes, [&](int u, int64_t r) { load8(x + r * a.ldx, left, v[u]); },
          [&](int u, int64_t) {
            ++mine;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float d = v[u][e] - first[e];
              s1[e] += d;
              s2[e] = fmaf(d, d, s2[e]);
            }
          });
    }
    const float inv = mine > 0 ? 1.f / (float)mine : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float m = s1[e] * inv;
      s_m[threadIdx.x][e] = first[e] + m;
      s_q[threadIdx.x][e] = fmaxf(0.f, fmaf(-s1[e], m, s2[e]));
    }
    // rows of lane rx: rx, rx + lanes, ..; joined pairwise
    const int rows = (int)(at.r1 - at.r0);
    auto count = [&](int rx, int step) { return rx < rows ? (rows - rx + step - 1) / step : 0; };
    for (int h = at.lanes / 2; h > 0; h /= 2) {
      __syncthreads();
      if (at.rx < h) {
        // after this turn lane rx holds the rows that are rx modulo h
        const float na = (float)count(at.rx, 2 * h), nb = (float)count(at.rx + h, 2 * h);
        if (nb > 0.f)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            join_moments(s_m[threadIdx.x][e], s_q[threadIdx.x][e], na, s_m[threadIdx.x + h * p.col_threads][e],
                         s_q[threadIdx.x + h * p.col_threads][e], nb);
      }
    }
    if (at.rx == 0) {
      const int64_t o = (at.sample * p.chunks + at.chunk) * a.channels + at.c;
      const int64_t q = a.n * p.chunks * a.channels;
      for (int e = 0; e < 8; ++e)
        if (e < left) {
          part[o + e] = s_m[threadIdx.x][e];
          part[q + o + e] = s_q[threadIdx.x][e];
        }
    }
    __syncthreads();
  }
}

// Sums over a group's partial values in 64 bits by a team of S threads: f(chunk, channel, u, v) adds to u and v.  All
// threads of the block call it together.
template <int S, class F>
__device__ __forceinline__ void group_sums(const NormArgs& a, const NormPlan& p, bool in, double* s_red, double& u,
                                           double& v, F f) {
  int CL = 1;                                            // threads side by side along the channels
  while (CL < S && CL < a.per) CL <<= 1;
  const int me = threadIdx.x % S, dk = S / CL;
  u = v = 0.0;
  if (in)
    for (int64_t k = me / CL; k < p.chunks; k += dk)
      for (int c = me % CL; c < a.per; c += CL) f(k, c, u, v);
  u = team_sum(u, S, s_red);
  v = team_sum(v, S, s_red);
}

// Team per sample and group: mean and rstd from the partial moments, to out and (nullable) stats_out.
template <int S>
__global__ __launch_bounds__(256) void norm_join_kernel(NormArgs a, NormPlan p, const float* part, float* out) {
  __shared__ double s_red[4];
  const int64_t q = a.n * p.chunks * a.channels, all = a.n * a.groups;
  const double total = (double)a.per * (double)a.positions;
  auto rows = [&](int64_t k) { return (double)(min(a.positions, (k + 1) * p.rows) - k * p.rows); };
  for (int64_t b0 = (int64_t)blockIdx.x * (256 / S); b0 < all; b0 += (int64_t)gridDim.x * (256 / S)) {
    const int64_t b = b0 + threadIdx.x / S;
    const bool in = b < all;
    int64_t g;
    const int64_t s = quotient(in ? b : 0, a.groups, g);
    const float* mean_p = part + s * p.chunks * a.channels + g * a.per;
    double sum, m2, none;
    group_sums<S>(a, p, in, s_red, sum, none, [&](int64_t k, int c, double& u, double&) {
      u += rows(k) * (double)mean_p[k * a.channels + c];
    });
    const double mean = sum / total;
    group_sums<S>(a, p, in, s_red, m2, none, [&](int64_t k, int c, double& u, double&) {
      const double d = (double)mean_p[k * a.channels + c] - mean;
      u += (double)mean_p[q + k * a.channels + c] + rows(k) * d * d;
    });
    if (in && threadIdx.x % S == 0) {
      const float m = (float)mean, rstd = (float)(1.0 / sqrt(m2 / total + (double)a.eps));
      out[2 * b] = m;
      out[2 * b + 1] = rstd;
      if (a.stats_out) {
        a.stats_out[2 * b] = m;
        a.stats_out[2 * b + 1] = rstd;
      }
    }
  }
}

// Team per sample and group: the means of weight dp and weight dp xh from the partial sums.
template <int S>
__global__ __launch_bounds__(256) void norm_coef_kernel(NormArgs a, NormPlan p, const float* part, float* coef) {
  __shared__ double s_red[4];
  const int64_t q = a.n * p.chunks * a.channels, all = a.n * a.groups;
  const double total = (double)a.per * (double)a.positions;
  for (int64_t b0 = (int64_t)blockIdx.x * (256 / S); b0 < all; b0 += (int64_t)gridDim.x * (256 / S)) {
    const int64_t b = b0 + threadIdx.x / S;
    const bool in = b < all;
    int64_t g;
    const int64_t s = quotient(in ? b : 0, a.groups, g);
    const float* pw = part + s * p.chunks * a.channels + g * a.per;
    double c1, c2;
    group_sums<S>(a, p, in, s_red, c1, c2, [&](int64_t k, int c, double& u, double& v) {
      const double w = a.weight ? (double)a.weight[g * a.per + c] : 1.0;
      u += w * (double)pw[q + k * a.channels + c];
      v += w * (double)pw[k * a.channels + c];
    });
    if (in && threadIdx.x % S == 0) {
      coef[2 * b] = (float)(c1 / total);
      coef[2 * b + 1] = (float)(c2 / total);
    }
  }
}

// What a thread of a split pass keeps of its 8 channels: with d = x - mean, p = wr d + bias (wr = weight rstd).
struct Channels {
  float mean[8], wr[8], b[8];
  // each(e, rstd, group of the sample) for what else is wanted
  template <class Each>
  __device__ __forceinline__ Channels(const NormArgs& a, const float* stats, int64_t sample, int64_t c, Each each) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t ch = (uint32_t)min(c + e, a.channels - 1);
      const int64_t g = sample * a.groups + ch / (uint32_t)a.per;
      mean[e] = stats[2 * g];
      const float rstd = stats[2 * g + 1];
      wr[e] = (a.weight ? a.weight[ch] : 1.f) * rstd;
      b[e] = a.bias ? a.bias[ch] : 0.f;
      each(e, rstd, g);
    }
  }
};

template <class T, int ACT>
__global__ __launch_bounds__(256) void norm_apply_kernel(NormArgs a, NormPlan p, const float* stats) {
  const int64_t blocks = a.n * p.chunks * p.tiles;
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const NormSpot at(a, p, b);
    const int64_t left = a.channels - at.c;
    if (left <= 0) continue;
    const Channels k(a, stats, at.sample, at.c, [](int, float, int64_t) {});
    const T* x = static_cast<const T*>(a.x) + at.c;
    T* y = static_cast<T*>(a.out) + at.c;
    constexpr int U = 4;
    float v[U][8];
    rows_in_groups<U>(
        at.r0 + at.rx, at.r1, at.lanes, [&](int u, int64_t r) { load8(x + r * a.ldx, left, v[u]); },
        [&](int u, int64_t r) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[u][e] = act_value<ACT>(fmaf(v[u][e] - k.mean[e], k.wr[e], k.b[e]));
          store8(y + r * a.ldo, left, v[u]);
        });
  }
}

// Sums of dp xh and dp over a chunk's rows: [sample][chunk][channel] of each.
template <class T, int ACT>
__global__ __launch_bounds__(256) void norm_sums_kernel(NormArgs a, NormPlan p, float* part) {
  __shared__ float s_w[256][9], s_b[256][9];
  const int64_t blocks = a.n * p.chunks * p.tiles;
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const NormSpot at(a, p, b);
    const int64_t left = a.channels - at.c;
    float sw[8], sb[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sw[e] = sb[e] = 0.f;
    if (left > 0) {
      float rstd[8];
      const Channels k(a, a.stats, at.sample, at.c, [&](int e, float r, int64_t) { rstd[e] = r; });
      const T* x = static_cast<const T*>(a.x) + at.c;
      const T* dy = static_cast<const T*>(a.dy) + at.c;
      constexpr int U = 2;
      float v[U][8], d[U][8];
      rows_in_groups<U>(
          at.r0 + at.rx, at.r1, at.lanes,
          [&](int u, int64_t r) {
            load8(x + r * a.ldx, left, v[u]);
            load8(dy + r * a.lddy, left, d[u]);
          },
          [&](int u, int64_t) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float diff = v[u][e] - k.mean[e];
              const float dp = act_back<ACT>(d[u][e], fmaf(diff, k.wr[e], k.b[e]));
              sw[e] = fmaf(dp, diff, sw[e]);
              sb[e] += dp;
            }
          });
#pragma unroll
      for (int e = 0; e < 8; ++e) sw[e] *= rstd[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s_w[threadIdx.x][e] = sw[e];
      s_b[threadIdx.x][e] = sb[e];
    }
    for (int h = at.lanes / 2; h > 0; h /= 2) {
      __syncthreads();
      if (at.rx < h)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s_w[threadIdx.x][e] += s_w[threadIdx.x + h * p.col_threads][e];
          s_b[threadIdx.x][e] += s_b[threadIdx.x + h * p.col_threads][e];
        }
    }
    if (at.rx == 0) {
      const int64_t o = (at.sample * p.chunks + at.chunk) * a.channels + at.c;
      const int64_t q = a.n * p.chunks * a.channels;
      for (int e = 0; e < 8; ++e)
        if (e < left) {
          part[o + e] = s_w[threadIdx.x][e];
          part[q + o + e] = s_b[threadIdx.x][e];
        }
    }
    __syncthreads();
  }
}

// Sums over the rows of part[0 / 1][row][channel] in a fixed order, dweight's and dbias's (nullable): block b of
// gradient_blocks() takes 8 channels of one of them, its threads 32 rows side by side.  In 64 bits, as the other joins:
// the rows grow with the samples, and 4096 equal ones added one by one in fp32 are off by up to 700 u of their sum.
__device__ __forceinline__ void gradient_block(int64_t b, const float* part, int64_t rows, int64_t channels,
                                               float* dweight, float* dbias) {
  __shared__ double s[256];
  const int64_t tiles = (channels + 7) / 8, which = b / tiles;
  float* out = which ? dbias : dweight;
  if (!out) return;                                      // the same for the whole block
  const int lane = threadIdx.x / 8;
  const int64_t c = b % tiles * 8 + threadIdx.x % 8;
  const float* p = part + which * rows * channels + c;
  double sum = 0.0;
  if (c < channels)
#pragma unroll 8
    for (int64_t k = lane; k < rows; k += 32) sum += (double)p[k * channels];
  s[threadIdx.x] = sum;
  for (int h = 16; h > 0; h /= 2) {
    __syncthreads();
    if (lane < h) s[threadIdx.x] += s[threadIdx.x + 8 * h];
  }
  if (lane == 0 && c < channels) out[c] = (float)s[threadIdx.x];
}
__global__ __launch_bounds__(256) void norm_gradient_kernel(const float* part, int64_t rows, int64_t channels,
                                                            float* dweight, float* dbias) {
  gradient_block(blockIdx.x, part, rows, channels, dweight, dbias);
}

// The first `extra` blocks sum dweight and dbias from norm_sums_kernel's partials beside the others.
template <class T, int ACT>
__global__ __launch_bounds__(256) void norm_apply_back_kernel(NormArgs a, NormPlan p, const float* coef,
                                                              const float* part, int extra, float* dweight,
                                                              float* dbias) {
  if ((int)blockIdx.x < extra) {
    gradient_block(blockIdx.x, part, a.n * p.chunks, a.channels, dweight, dbias);
    return;
  }
  const int64_t blocks = a.n * p.chunks * p.tiles;
  for (int64_t b = blockIdx.x - extra; b < blocks; b += gridDim.x - extra) {
    const NormSpot at(a, p, b);
    const int64_t left = a.channels - at.c;
    if (left <= 0) continue;
    // dx = rstd (w dp - c1 - xh c2) = wr dp - rstd c1 - (rstd^2 c2) d
    float c1[8], c2[8];
    const Channels k(a, a.stats, at.sample, at.c, [&](int e, float rstd, int64_t g) {
      c1[e] = rstd * coef[2 * g];
      c2[e] = rstd * (rstd * coef[2 * g + 1]);
    });
    const T* x = static_cast<const T*>(a.x) + at.c;
    const T* dy = static_cast<const T*>(a.dy) + at.c;
    T* dx = static_cast<T*>(a.out) + at.c;
    constexpr int U = 2;
    float v[U][8], d[U][8];
    rows_in_groups<U>(
        at.r0 + at.rx, at.r1, at.lanes,
        [&](int u, int64_t r) {
          load8(x + r * a.ldx, left, v[u]);
          load8(dy + r * a.lddy, left, d[u]);
        },
        [&](int u, int64_t r) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float diff = v[u][e] - k.mean[e];
            const float dp = act_back<ACT>(d[u][e], fmaf(diff, k.wr[e], k.b[e]));
            v[u][e] = fmaf(-diff, c2[e], fmaf(dp, k.wr[e], -c1[e]));
          }
          store8(dx + r * a.ldo, left, v[u]);
        });
  }
}

}  // namespace ot

struct ot_norm {
  ot::NormSizes sizes;
  int32_t precision, act;
  float eps;
  int device;
  ot::Workspace ws;
  int64_t bytes(int64_t n) const { return 4 * ot::norm_values(sizes, n); }
};

namespace {

constexpr int64_t kMostSamples = 1LL << 26, kMostValues = 1LL << 36;
constexpr int64_t kMostBlocks = 1LL << 20;              // kernels loop over what is more

unsigned grid_of(int64_t blocks) { return (unsigned)std::min(blocks, kMostBlocks); }

ot::NormArgs args_of(const ot_norm* d, int64_t n) {
  ot::NormArgs a{};
  a.n = n;
  a.positions = d->sizes.positions;
  a.channels = d->sizes.channels;
  a.groups = d->sizes.groups;
  a.per = (int32_t)d->sizes.per();
  a.eps = d->eps;
  return a;
}

template <class T, int ACT>
int forward(const ot_norm* d, const ot::NormArgs& a, hipStream_t st) {
  if (const int lanes = ot::team_lanes(d->sizes)) {
    const dim3 grid(grid_of(ot::ceil_div(a.n * a.groups, 256 / lanes)));
    switch (ot::team_vectors(d->sizes)) {
      case 1: hipLaunchKernelGGL((ot::norm_team_kernel<T, ACT, 1>), grid, dim3(256), 0, st, a, lanes); break;
      case 2: hipLaunchKernelGGL((ot::norm_team_kernel<T, ACT, 2>), grid, dim3(256), 0, st, a, lanes); break;
      default: hipLaunchKernelGGL((ot::norm_team_kernel<T, ACT, 4>), grid, dim3(256), 0, st, a, lanes); break;
    }
    OT_LAUNCHED("norm_team_kernel");
    return OT_OK;
  }
  const int gb = ot::slab_groups(d->sizes);
  if (gb > 0) {
    const int64_t parts = ot::ceil_div(a.groups, gb);
    hipLaunchKernelGGL((ot::norm_slab_kernel<T, ACT>), dim3(grid_of(a.n * parts)), dim3(256),
                       (unsigned)(4 * ot::slab_values(d->sizes, false)), st, a, gb, parts);
    OT_LAUNCHED("norm_slab_kernel");
    return OT_OK;
  }
  const ot::NormPlan p = ot::plan_norm(d->sizes, a.n);
  float* stats = reinterpret_cast<float*>(d->ws.p);
  float* part = stats + 2 * a.n * a.groups;
  const dim3 grid(grid_of(a.n * p.chunks * p.tiles));
  hipLaunchKernelGGL(ot::norm_moments_kernel<T>, grid, dim3(256), 0, st, a, p, part);
  OT_LAUNCHED("norm_moments_kernel");
  if (ot::long_join(d->sizes, p))
    hipLaunchKernelGGL(ot::norm_join_kernel<256>, dim3(grid_of(a.n * a.groups)), dim3(256), 0, st, a, p, part, stats);
  else
    hipLaunchKernelGGL(ot::norm_join_kernel<64>, dim3(grid_of(ot::ceil_div(a.n * a.groups, 4))), dim3(256), 0, st, a, p,
                       part, stats);
  OT_LAUNCHED("norm_join_kernel");
  hipLaunchKernelGGL((ot::norm_apply_kernel<T, ACT>), grid, dim3(256), 0, st, a, p, stats);
  OT_LAUNCHED("norm_apply_kernel");
  return OT_OK;
}

int64_t gradient_blocks(int64_t channels) { return 2 * ot::ceil_div(channels, 8); }

int gradients(const float* sums, int64_t rows, int64_t channels, float* dweight, float* dbias, hipStream_t st) {
  hipLaunchKernelGGL(ot::norm_gradient_kernel, dim3((unsigned)gradient_blocks(channels)), dim3(256), 0, st, sums, rows,
                     channels, dweight, dbias);
  OT_LAUNCHED("norm_gradient_kernel");
  return OT_OK;
}

template <class T, int ACT>
int backward(const ot_norm* d, const ot::NormArgs& a, float* dweight, float* dbias, hipStream_t st) {
  const int gb = ot::slab_groups(d->sizes);
  const bool want = dweight || dbias;
  float* ws = reinterpret_cast<float*>(d->ws.p);
  if (d->sizes.positions == 1 && ot::team_lanes(d->sizes)) {
    const ot::TeamPlan t = ot::plan_team_back(d->sizes, a.n);
    const dim3 grid((unsigned)(t.tiles * t.ranges));
    float* sums = want ? ws : nullptr;
    switch (ot::team_vectors(d->sizes)) {
      case 1:
        hipLaunchKernelGGL((ot::norm_team_back_kernel<T, ACT, 1>), grid, dim3(256), 0, st, a, t.lanes, t.groups, t.tiles,
                           t.ranges, sums);
        break;
      case 2:
        hipLaunchKernelGGL((ot::norm_team_back_kernel<T, ACT, 2>), grid, dim3(256), 0, st, a, t.lanes, t.groups, t.tiles,
                           t.ranges, sums);
        break;
      default:
        hipLaunchKernelGGL((ot::norm_team_back_kernel<T, ACT, 4>), grid, dim3(256), 0, st, a, t.lanes, t.groups, t.tiles,
                           t.ranges, sums);
        break;
    }
    OT_LAUNCHED("norm_team_back_kernel");
    return want ? gradients(ws, t.ranges, a.channels, dweight, dbias, st) : OT_OK;
  }
  if (gb > 0) {
    const int64_t parts = ot::ceil_div(a.groups, gb), ranges = ot::slab_ranges(d->sizes, a.n);
    hipLaunchKernelGGL((ot::norm_slab_back_kernel<T, ACT>), dim3((unsigned)(parts * ranges)), dim3(256),
                       (unsigned)(4 * ot::slab_values(d->sizes, true)), st, a, gb, parts, ranges, want ? ws : nullptr);
    OT_LAUNCHED("norm_slab_back_kernel");
    return want ? gradients(ws, ranges, a.channels, dweight, dbias, st) : OT_OK;
  }
  const ot::NormPlan p = ot::plan_norm(d->sizes, a.n);
  float* coef = ws;
  float* part = coef + 2 * a.n * a.groups;
  const unsigned blocks = grid_of(a.n * p.chunks * p.tiles);
  hipLaunchKernelGGL((ot::norm_sums_kernel<T, ACT>), dim3(blocks), dim3(256), 0, st, a, p, part);
  OT_LAUNCHED("norm_sums_kernel");
  if (!a.out) return gradients(part, a.n * p.chunks, a.channels, dweight, dbias, st);
  if (ot::long_join(d->sizes, p))
    hipLaunchKernelGGL(ot::norm_coef_kernel<256>, dim3(grid_of(a.n * a.groups)), dim3(256), 0, st, a, p, part, coef);
  else
    hipLaunchKernelGGL(ot::norm_coef_kernel<64>, dim3(grid_of(ot::ceil_div(a.n * a.groups, 4))), dim3(256), 0, st, a, p,
                       part, coef);
  OT_LAUNCHED("norm_coef_kernel");
  const int extra = want ? (int)gradient_blocks(a.channels) : 0;
  hipLaunchKernelGGL((ot::norm_apply_back_kernel<T, ACT>), dim3(blocks + extra), dim3(256), 0, st, a, p, coef,
                     part, extra, dweight, dbias);
  OT_LAUNCHED("norm_apply_back_kernel");
  return OT_OK;
}

}  // namespace

extern "C" int norm_create(ot_norm** out, int64_t channels, int32_t groups, int64_t positions, int32_t precision,
                           int32_t activation, float eps, int64_t max_samples) {
  ot::clear_error();
  OT_REQUIRE(out != nullptr, "norm_create: NULL out");
  *out = nullptr;
  OT_REQUIRE(channels >= 1 && channels <= 65536, "norm_create: channels outside [1, 65536]");
  OT_REQUIRE(groups >= 1 && groups <= channels && channels % groups == 0, "norm_create: groups do not divide channels");
  OT_REQUIRE(positions >= 1 && positions <= (1LL << 26), "norm_create: positions outside [1, 2^26]");
  OT_REQUIRE(precision == OT_FP32 || precision == OT_BF16, "norm_create: unknown precision");
  OT_REQUIRE(activation >= OT_ACT_NONE && activation <= OT_ACT_GELU, "norm_create: unknown activation");
  OT_REQUIRE(std::isfinite(eps) && eps > 0.f, "norm_create: eps is not finite and above 0");
  OT_REQUIRE(max_samples >= 0 && max_samples <= kMostSamples, "norm_create: max_samples outside [0, 2^26]");
  OT_REQUIRE(channels * positions <= kMostValues && max_samples <= kMostValues / (channels * positions),
             "norm_create: more than 2^36 values");
  int device = -1;
  OT_HIP(hipGetDevice(&device));
  ot_norm* d = new (std::nothrow) ot_norm();
  if (!d) return ot::set_error(OT_E_NOMEM, "norm_create: out of host memory");
  d->sizes = ot::NormSizes{channels, positions, groups};
  d->precision = precision;
  d->act = activation;
  d->eps = eps;
  d->device = device;
  const int rc = d->ws.allocate(max_samples, d->bytes(max_samples), "norm_create");
  if (rc) {
    delete d;
    return rc;
  }
  *out = d;
  return OT_OK;
}

namespace {

// Checks that forward and backward share.
int check_call(const ot_norm* d, const void* x, int64_t ldx, const float* weight, const float* bias, int64_t n,
               const char* what) {
  OT_REQUIRE(n >= 0 && n <= kMostSamples, "%s: n outside [0, 2^26]", what);
  OT_REQUIRE(n <= kMostValues / (d->sizes.channels * d->sizes.positions), "%s: more than 2^36 values", what);
  if (n == 0) return OT_OK;
  const int e = d->precision == OT_BF16 ? 2 : 4;
  int rc;
  if ((rc = ot::check_rows(x, ldx, n * d->sizes.positions, d->sizes.channels, e, what, "x"))) return rc;
  if ((rc = ot::check_values(weight, 4, what, "weight"))) return rc;
  return ot::check_values(bias, 4, what, "bias");
}

}  // namespace

extern "C" int norm_forward(ot_norm* d, const void* x, int64_t ldx, const float* weight, const float* bias, int64_t n,
                            void* y, int64_t ldy, float* stats, void* stream) try {
  ot::clear_error();
  const char* what = "norm_forward";
  OT_REQUIRE(d != nullptr, "%s: NULL norm", what);
  int rc;
  if ((rc = check_call(d, x, ldx, weight, bias, n, what)) || n == 0) return rc;
  const int e = d->precision == OT_BF16 ? 2 : 4;
  if ((rc = ot::check_rows(y, ldy, n * d->sizes.positions, d->sizes.channels, e, what, "y"))) return rc;
  if ((rc = ot::check_values(stats, 4, what, "stats"))) return rc;
  if ((rc = ot::check_device(d->device, what))) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  // only split passes keep something between launches
  if (ot::slab_groups(d->sizes) == 0 && (rc = d->ws.begin(n, st, what, [&](int64_t k) { return d->bytes(k); })))
    return rc;
  ot::NormArgs a = args_of(d, n);
  a.x = x;
  a.ldx = ldx;
  a.out = y;
  a.ldo = ldy;
  a.weight = weight;
  a.bias = bias;
  a.stats_out = stats;
  ot::with_act(d->act, [&](auto act) {
    constexpr int A = decltype(act)::value;
    rc = e == 2 ? forward<uint16_t, A>(d, a, st) : forward<float, A>(d, a, st);
  });
  return rc;
} catch (const std::bad_alloc&) {
  return ot::set_error(OT_E_NOMEM, "norm_forward: out of host memory");
}

extern "C" int norm_backward(ot_norm* d, const void* x, int64_t ldx, const float* weight, const float* bias,
                             int64_t n, const float* stats, const void* dy, int64_t lddy, void* dx, int64_t lddx,
                             float* dweight, float* dbias, void* stream) try {
  ot::clear_error();
  const char* what = "norm_backward";
  OT_REQUIRE(d != nullptr, "%s: NULL norm", what);
  int rc;
  if ((rc = check_call(d, x, ldx, weight, bias, n, what))) return rc;
  if ((rc = ot::check_values(dweight, 4, what, "dweight"))) return rc;
  if ((rc = ot::check_values(dbias, 4, what, "dbias"))) return rc;
  const int e = d->precision == OT_BF16 ? 2 : 4;
  if (n > 0) {
    OT_REQUIRE(stats != nullptr, "%s: NULL stats", what);
    if ((rc = ot::check_values(stats, 4, what, "stats"))) return rc;
    if ((rc = ot::check_rows(dy, lddy, n * d->sizes.positions, d->sizes.channels, e, what, "dy"))) return rc;
    if (dx && (rc = ot::check_rows(dx, lddx, n * d->sizes.positions, d->sizes.channels, e, what, "dx"))) return rc;
  }
  if ((rc = ot::check_device(d->device, what))) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (n == 0) return dweight || dbias ? gradients(nullptr, 0, d->sizes.channels, dweight, dbias, st) : OT_OK;
  if (!dx && !dweight && !dbias) return OT_OK;
  // dx of groups that one launch holds keeps nothing
  if ((ot::slab_groups(d->sizes) == 0 || dweight || dbias) &&
      (rc = d->ws.begin(n, st, what, [&](int64_t k) { return d->bytes(k); })))
    return rc;
  ot::NormArgs a = args_of(d, n);
  a.x = x;
  a.ldx = ldx;
  a.dy = dy;
  a.lddy = lddy;
  a.out = dx;
  a.ldo = lddx;
  a.weight = weight;
  a.bias = bias;
  a.stats = stats;
  ot::with_act(d->act, [&](auto act) {
    constexpr int A = decltype(act)::value;
    rc = e == 2 ? backward<uint16_t, A>(d, a, dweight, dbias, st) : backward<float, A>(d, a, dweight, dbias, st);
  });
  return rc;
} catch (const std::bad_alloc&) {
  return ot::set_error(OT_E_NOMEM, "norm_backward: out of host memory");
}

extern "C" int norm_destroy(ot_norm* d) {
  ot::clear_error();
  if (!d) return OT_OK;
  d->ws.release();
  delete d;
  return OT_OK;
}
