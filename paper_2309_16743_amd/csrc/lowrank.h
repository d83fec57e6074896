// Products with one short side for the adapters (adapters.hip): rows of a batch,
// sorted by adapter, times rank x length matrices.
//
//   shrink: t[p][r]     = sum_k src[row(p)][k] mat_g[r][k]       (reduction over the long axis)
//   outer:  out_g[r][c] = sum over adapter g's rows of coef[p][r] src[row(p)][c]
//
// Both read every src value once and use each for `rank` products, so they are
// bound by HBM (rank 16 in bf16: 16 flops a byte).  Matrix instructions keep the vector units free for addresses;
// operands go from memory to registers in the lane layout of the instruction, without LDS:
// v_mfma_f32_16x16x32_bf16: lane l supplies A[l%16][8 (l/16) + e], B[8 (l/16) + e][l%16], e = 0..7;
// v_mfma_f32_16x16x4_f32:   lane l supplies A[l%16][l/16], B[l/16][l%16];
// both: accumulator element e of lane l is D[4 (l/16) + e][l%16].
// The order of k inside an instruction is free as long as A and B agree, so a
// lane's consecutive values in memory serve as its consecutive k.
#pragma once

#include "common.h"
#include "intmath.h"
#include "lowrank_ops.h"

namespace ot {

constexpr int kSlotRows = 32;       // sorted rows of one adapter that a block takes together

// Rows [start, start + count) of the sorted order, all of adapter g.
struct RowSlot {
  int32_t start, count, g, pad;
};

// D += A B with the 16 bytes that lane l holds of each operand as its k values.
template <class T>
__device__ __forceinline__ f32x4 lr_mfma(lr_u32x4 a, lr_u32x4 b, f32x4 d) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(lr_bf16x8, a), __builtin_bit_cast(lr_bf16x8, b), d,
                                                   0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      d = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), d, 0, 0, 0);
    return d;
  }
}

// ------------------------------------------------------------------ shrink
struct ShrinkArgs {
  const void* src;        // rows of L values
  int64_t lds;
  const void* mat;        // G x R rows of L values
  int64_t ldm;
  int64_t L;
  int64_t k_chunk;        // of one split (a multiple of kShrinkUnit)
  int32_t G, R, RP;       // RP: R rounded up to 16
  int32_t splits;
  int64_t n;
  const float* scale;     // nullable
  const int32_t* perm;
  const RowSlot* slots;
  float* part;            // splits > 1: [split][sorted row][RP]
  float* ts;              // sorted, pitch RP: scaled
  float* t;               // by row, pitch ldt: unscaled (nullable)
  int64_t ldt;
};

constexpr int kShrinkUnit = 128;    // k values of four steps (bf16) or eight (fp32)

// Row i of slot s: sums over rank tile q of this thread's values, to their destinations.
__device__ __forceinline__ void shrink_finish(const ShrinkArgs& a, const RowSlot& s, int i, int r, float v) {
  if (a.t && r < a.R) a.t[(int64_t)a.perm[s.start + i] * a.ldt + r] = v;
  if (s.g < a.G) a.ts[(int64_t)(s.start + i) * a.RP + r] = a.scale ? a.scale[s.g] * v : v;
}

// grid = (slots, splits), 256 threads: the four wavefronts take neighbouring
// quarters of the split's k range and join their sums in LDS in a fixed order.
template <class T, int NT>
__global__ __launch_bounds__(256) void shrink_kernel(ShrinkArgs a) {
  constexpr int V = 16 / (int)sizeof(T);          // values per lane and step
  constexpr int STEP = 4 * V;                     // k values per step
  constexpr int U = sizeof(T) == 2 ? 4 : (NT > 2 ? 2 : 4);   // steps whose loads are in flight together
  constexpr int RP = 16 * NT;
  __shared__ float red[4][32][RP + 1];
  const RowSlot s = a.slots[blockIdx.x];
  if (s.count <= 0) return;                       // the same for the whole block
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int64_t split = blockIdx.y;
  if (s.g >= a.G) {                               // rows without an adapter
    if (split == 0 && a.t)
      for (int i = threadIdx.x; i < s.count * a.R; i += 256)
        a.t[(int64_t)a.perm[s.start + i / a.R] * a.ldt + i % a.R] = 0.f;
    return;
  }
  const int64_t kb = split * a.k_chunk, ke = min(a.L, kb + a.k_chunk);
  const int64_t quarter = ((ke - kb + 4 * STEP - 1) / (4 * STEP)) * STEP;
  const int64_t b = kb + wid * quarter, e = min(ke, b + quarter);
  const int i = lane % 16, kq = V * (lane / 16);
  const bool two = s.count > 16;
  const T* x0 = static_cast<const T*>(a.src) + (int64_t)a.perm[s.start + min(i, s.count - 1)] * a.lds;
  const T* x1 = static_cast<const T*>(a.src) + (int64_t)a.perm[s.start + min(16 + i, s.count - 1)] * a.lds;
  const T* m[NT];
#pragma unroll
  for (int q = 0; q < NT; ++q)                    // ranks past R read the last one; their sums are dropped
    m[q] = static_cast<const T*>(a.mat) + ((int64_t)s.g * a.R + min(16 * q + i, a.R - 1)) * a.ldm;
  f32x4 acc[2][NT];
#pragma unroll
  for (int f = 0; f < 2; ++f)
#pragma unroll
    for (int q = 0; q < NT; ++q) acc[f][q] = f32x4{0.f, 0.f, 0.f, 0.f};
  int64_t k = b;
  for (; k + U * STEP <= e; k += U * STEP) {
    lr_u32x4 va[U], vb[U], vm[U][NT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t o = k + u * STEP + kq;
      va[u] = *reinterpret_cast<const lr_u32x4*>(x0 + o);
      if (two) vb[u] = *reinterpret_cast<const lr_u32x4*>(x1 + o);
#pragma unroll
      for (int q = 0; q < NT; ++q) vm[u][q] = *reinterpret_cast<const lr_u32x4*>(m[q] + o);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int q = 0; q < NT; ++q) {
        acc[0][q] = lr_mfma<T>(va[u], vm[u][q], acc[0][q]);
        if (two) acc[1][q] = lr_mfma<T>(vb[u], vm[u][q], acc[1][q]);
      }
  }
  for (; k < e; k += STEP) {
    const int64_t o = k + kq, valid = e - o;
    const lr_u32x4 va = lr_load16(x0 + o, valid), vb = lr_load16(x1 + o, two ? valid : 0);
#pragma unroll
    for (int q = 0; q < NT; ++q) {
      const lr_u32x4 vm = lr_load16(m[q] + o, valid);
      acc[0][q] = lr_mfma<T>(va, vm, acc[0][q]);
      if (two) acc[1][q] = lr_mfma<T>(vb, vm, acc[1][q]);
    }
  }
#pragma unroll
  for (int f = 0; f < 2; ++f)
#pragma unroll
    for (int q = 0; q < NT; ++q)
#pragma unroll
      for (int r = 0; r < 4; ++r) red[wid][16 * f + 4 * (lane / 16) + r][16 * q + i] = acc[f][q][r];
  __syncthreads();
  for (int j = threadIdx.x; j < s.count * RP; j += 256) {
    const int row = j / RP, r = j % RP;
    float v = (red[0][row][r] + red[1][row][r]) + (red[2][row][r] + red[3][row][r]);
    if (r >= a.R) v = 0.f;
    if (a.splits > 1) a.part[(split * a.n + s.start + row) * RP + r] = v;
    else shrink_finish(a, s, row, r, v);
  }
}

// Sums of the splits in order; grid = slots.
__global__ __launch_bounds__(256) void shrink_reduce_kernel(ShrinkArgs a) {
  const RowSlot s = a.slots[blockIdx.x];
  if (s.count <= 0 || s.g >= a.G) return;
  for (int j = threadIdx.x; j < s.count * a.RP; j += 256) {
    const int64_t step = a.n * a.RP;
    const float* p = a.part + (int64_t)s.start * a.RP + j;
    float v = 0.f;
    int q = 0;
    for (; q + 8 <= a.splits; q += 8) {           // eight loads in flight, added in order
      float w[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) w[u] = p[(q + u) * step];
#pragma unroll
      for (int u = 0; u < 8; ++u) v += w[u];
    }
    for (; q < a.splits; ++q) v += p[q * step];
    shrink_finish(a, s, j / a.RP, j % a.RP, v);
  }
}

// ------------------------------------------------------------------ outer
struct OuterArgs {
  const void* src;        // rows of L values
  int64_t lds;
  int64_t L;
  const float* coef;      // sorted rows (pitch RP) or, by_row, the caller's rows (pitch ldc)
  int64_t ldc;
  int32_t by_row;
  const float* scale;     // by_row: factor of adapter g (nullable)
  int32_t R;
  const int32_t* perm;
  const int32_t* off;
  float* out;             // G x R rows of L values
  int64_t ldo;
};

// A wavefront holds rank x 64 outputs: lane l covers columns 4 (l%16) .. + 3, so
// that it reads 8 or 16 bytes of a row and writes 16 bytes of an output row; column
// q of the four is one matrix product.  In bf16 the rows' coefficients enter as
// three bf16 terms (they are fp32), 32 rows to a step; in fp32 4 rows to a product.
//
// ROWSPLIT false: the block's wavefronts take 64 columns each (long rows: enough
// blocks).  true: they take the same 64 columns and every fourth step of 32
// rows, and join in LDS (short rows: four times the wavefronts).
// grid = (column blocks, adapters).
template <class T, int NT, bool ROWSPLIT>
__global__ __launch_bounds__(256) void outer_kernel(OuterArgs a) {
  constexpr int TERMS = 3;
  __shared__ float red[ROWSPLIT ? 3 : 1][ROWSPLIT ? 16 * NT : 1][ROWSPLIT ? 68 : 1];
  const int g = blockIdx.y, lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int64_t c0 = ((int64_t)blockIdx.x * (ROWSPLIT ? 1 : 4) + (ROWSPLIT ? 0 : wid)) * 64;
  if (!ROWSPLIT && c0 >= a.L) return;             // no barriers follow
  const int pb = a.off[g], pe = a.off[g + 1];
  const int i = lane % 16, kg = lane / 16;
  const int64_t c = c0 + 4 * i;
  const int64_t cl = c < a.L ? c : 0;             // lanes past the row read its start; they store nothing
  const float sc = a.by_row && a.scale ? a.scale[g] : 1.f;
  f32x4 acc[NT][4];
#pragma unroll
  for (int q = 0; q < NT; ++q)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[q][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // coefficient of sorted row p, rank 16 q + i
  auto coef = [&](int p, int64_t row, int q) {
    const int r = 16 * q + i;
    return r < a.R ? sc * a.coef[(a.by_row ? row : (int64_t)p) * a.ldc + r] : 0.f;
  };
  for (int p0 = pb + (ROWSPLIT ? 32 * wid : 0); p0 < pe; p0 += ROWSPLIT ? 128 : 32) {
    int64_t row[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int p = p0 + (sizeof(T) == 2 ? 8 * kg + e : 4 * e + kg);
      row[e] = a.perm[min(p, pe - 1)];
    }
    if constexpr (sizeof(T) == 2) {
      lr_u32x2 v[8];
      const uint16_t* src = static_cast<const uint16_t*>(a.src) + cl;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const lr_u32x2*>(src + row[e] * a.lds);
      if (p0 + 32 > pe) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (p0 + 8 * kg + e >= pe) v[e] = lr_u32x2{0, 0};
      }
      lr_u32x4 b[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) {               // rows 2 w and 2 w + 1 of each column
        b[0][w] = __builtin_amdgcn_perm(v[2 * w + 1][0], v[2 * w][0], 0x05040100);
        b[1][w] = __builtin_amdgcn_perm(v[2 * w + 1][0], v[2 * w][0], 0x07060302);
        b[2][w] = __builtin_amdgcn_perm(v[2 * w + 1][1], v[2 * w][1], 0x05040100);
        b[3][w] = __builtin_amdgcn_perm(v[2 * w + 1][1], v[2 * w][1], 0x07060302);
      }
#pragma unroll
      for (int q = 0; q < NT; ++q) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int p = p0 + 8 * kg + e;
          x[e] = p < pe ? coef(p, row[e], q) : 0.f;
        }
        lr_u32x4 t[TERMS];
        lr_split8<TERMS>(x, t);
#pragma unroll
        for (int z = TERMS - 1; z >= 0; --z)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[q][j] = lr_mfma<uint16_t>(t[z], b[j], acc[q][j]);
      }
    } else {
      f32x4 v[8];
      const float* src = static_cast<const float*>(a.src) + cl;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const f32x4*>(src + row[e] * a.lds);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int p = p0 + 4 * e + kg;
        const bool in = p < pe;
#pragma unroll
        for (int q = 0; q < NT; ++q) {
          const float x = in ? coef(p, row[e], q) : 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[q][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, in ? v[e][j] : 0.f, acc[q][j], 0, 0, 0);
        }
      }
    }
  }
  // element r of acc[q][j]: rank 16 q + 4 kg + r, column c + j
  if constexpr (ROWSPLIT) {
    if (wid > 0) {
#pragma unroll
      for (int q = 0; q < NT; ++q)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < 4; ++j) red[wid - 1][16 * q + 4 * kg + r][4 * i + j] = acc[q][j][r];
    }
    __syncthreads();
    if (wid > 0) return;
#pragma unroll
    for (int q = 0; q < NT; ++q)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int rr = 16 * q + 4 * kg + r, cc = 4 * i + j;
          acc[q][j][r] = ((acc[q][j][r] + red[0][rr][cc]) + red[1][rr][cc]) + red[2][rr][cc];
        }
  }
#pragma unroll
  for (int q = 0; q < NT; ++q)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int rank = 16 * q + 4 * kg + r;
      if (rank >= a.R || c >= a.L) continue;
      float* o = a.out + ((int64_t)g * a.R + rank) * a.ldo + c;
      if (c + 4 <= a.L) {
        *reinterpret_cast<f32x4*>(o) = f32x4{acc[q][0][r], acc[q][1][r], acc[q][2][r], acc[q][3][r]};
      } else {
        for (int j = 0; c + j < a.L; ++j) o[j] = j == 0 ? acc[q][0][r] : j == 1 ? acc[q][1][r] : acc[q][2][r];
      }
    }
}

}  // namespace ot
