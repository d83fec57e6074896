// Products with one short side for the adapters (adapters.hip): rows of a batch,
// sorted by adapter, times rank x length matrices.
//
//   shrink: t[p][r]     = sum_k src[row(p)][k] mat_g[r][k]       (reduction over the long axis)
//   outer:  out_g[r][c] = sum over adapter g's rows of coef[p][r] src[row(p)][c]
//
// Both read every src value once and use each for `rank` products, so they are
// bound by HBM (rank 16 in bf16: 16 flops a byte), and for a batch of hidden rows by latency: 1024 rows of
// 2048 bf16 values, rank 16, 32 adapters: shrink 8.5 us, of which 4 sort the ids, both gradients 9.5.  Matrix instructions keep the vector units free for addresses;
// operands go from memory to registers in the lane layout of the instruction, without LDS:
// v_mfma_f32_16x16x32_bf16: lane l supplies A[l%16][8 (l/16) + e], B[8 (l/16) + e][l%16], e = 0..7;
// v_mfma_f32_16x16x4_f32:   lane l supplies A[l%16][l/16], B[l/16][l%16];
// both: accumulator element e of lane l is D[4 (l/16) + e][l%16].
// The order of k inside an instruction is free as long as A and B agree, so a
// lane's consecutive values in memory serve as its consecutive k.
#pragma once

#include <type_traits>

#include "adapt_plan.h"
#include "common.h"
#include "intmath.h"
#include "lowrank_ops.h"

namespace ot {

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
constexpr int kShrinkThreads = 512;
// Up to this many rows and keys (adapters and "none") the blocks of the shrink sort the ids themselves.
constexpr int kSelfRows = 2048, kSelfKeys = 1024;

struct SelfSort {
  const int32_t* ids;
  int32_t* perm;          // written: what group_rows_kernel would write
  int32_t* gid;
  int32_t* off;
  RowSlot* slots;
  int32_t slot_rows;
};

// Slot b of the batch's rows sorted by adapter, found by the block itself (512
// threads): every block counts all ids and scans the counts in LDS, so no launch has to
// come before.  About 2 us of latency against 4.5 us for a launch of its own (1024 rows).
// s_rows receives the slot's row numbers; `publish`: the block writes its part of the sorted order (slot 0's block
// the adapters' offsets) for the kernels that follow.
struct SelfScratch {
  int32_t cnt[kSelfKeys];
  int32_t sum[2][8];
  RowSlot slot;
};
__device__ __forceinline__ RowSlot self_slot(const SelfSort& o, int n, int G, int b, bool publish, SelfScratch& sh,
                                             int32_t* s_rows) {
  constexpr int PER = kSelfRows / kShrinkThreads;
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  int key[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = PER * tid + j;
    const int k = i < n ? o.ids[i] : 0;
    key[j] = i < n ? (k < 0 || k >= G ? G : k) : -1;
  }
  for (int k = tid; k < kSelfKeys; k += kShrinkThreads) sh.cnt[k] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (key[j] >= 0) atomicAdd(&sh.cnt[key[j]], 1);          // integer counts: any order gives the same
  __syncthreads();
  // sum over the threads before this one, in thread order
  auto before = [&](int v, int32_t* part) {
    int x = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(x, d, 64);
      if (lane >= d) x += y;
    }
    if (lane == 63) part[wid] = x;
    __syncthreads();
    int base = 0;
    for (int w = 0; w < wid; ++w) base += part[w];
    return base + x - v;
  };
  const int c0 = sh.cnt[2 * tid], c1 = sh.cnt[2 * tid + 1];
  const int start0 = before(c0 + c1, sh.sum[0]);
  static_assert(kSelfKeys == 2 * kShrinkThreads, "two keys per thread");
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int k = 2 * tid + j, start = j ? start0 + c0 : start0, count = j ? c1 : c0;
    if (k > G) break;
    if (b == 0 && publish) {
      o.off[k] = start;
      if (k == G) o.off[G + 1] = n;
    }
    const int first = start / o.slot_rows + k;
    if (b >= first && b < (start + count) / o.slot_rows + k + 1) {
      const int r = (b - first) * o.slot_rows;
      sh.slot = RowSlot{start + r, max(0, min(o.slot_rows, count - r)), k, r};
    }
  }
  __syncthreads();
  RowSlot s = sh.slot;
  if (publish && tid == 0) o.slots[b] = s;
  if (s.count <= 0) return s;
  int mine = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) mine += key[j] == s.g;
  int at = before(mine, sh.sum[1]) - s.pad;                  // rank within the adapter, from the slot's first
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (key[j] == s.g) {
      if (at >= 0 && at < s.count) {
        s_rows[at] = PER * tid + j;
        if (publish) {
          o.perm[s.start + at] = PER * tid + j;
          o.gid[s.start + at] = s.g;
        }
      }
      ++at;
    }
  __syncthreads();
  return s;
}

// Row number `row`, sorted position p: value v of rank r to its destinations.
__device__ __forceinline__ void shrink_finish(const ShrinkArgs& a, int g, int64_t p, int64_t row, int r, float v) {
  if (a.t && r < a.R) a.t[row * a.ldt + r] = v;
  if (g < a.G) a.ts[p * a.RP + r] = a.scale ? a.scale[g] * v : v;
}

// grid = (slots, splits), 512 threads: the eight wavefronts take neighbouring
// parts of the split's k range and join their sums in LDS in a fixed order.
// SELF: the blocks sort the ids (self_slot); otherwise group_rows_kernel has.
template <class T, int NT, bool SELF>
__global__ __launch_bounds__(kShrinkThreads) void shrink_kernel(ShrinkArgs a, SelfSort self) {
  constexpr int V = 16 / (int)sizeof(T);          // values per lane and step
  constexpr int STEP = 4 * V;                     // k values per step
  constexpr int U = sizeof(T) == 2 ? 4 : (NT > 2 ? 2 : 4);   // steps whose loads are in flight together
  constexpr int RP = 16 * NT, NW = kShrinkThreads / 64;
  __shared__ float red[NW][32][RP + 1];
  __shared__ int32_t s_rows[kSlotRows];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int64_t split = blockIdx.y;
  RowSlot s;
  if constexpr (SELF) {
    __shared__ SelfScratch sh;
    s = self_slot(self, (int)a.n, a.G, blockIdx.x, split == 0, sh, s_rows);
    if (s.count <= 0) return;                     // the same for the whole block
  } else {
    s = a.slots[blockIdx.x];
    if (s.count <= 0) return;
    if ((int)threadIdx.x < s.count) s_rows[threadIdx.x] = a.perm[s.start + threadIdx.x];
    __syncthreads();
  }
  if (s.g >= a.G) {                               // rows without an adapter
    if (split == 0 && a.t)
      for (int i = threadIdx.x; i < s.count * a.R; i += kShrinkThreads)
        a.t[(int64_t)s_rows[i / a.R] * a.ldt + i % a.R] = 0.f;
    return;
  }
  const int64_t kb = split * a.k_chunk, ke = min(a.L, kb + a.k_chunk);
  const int64_t share = ((ke - kb + NW * STEP - 1) / (NW * STEP)) * STEP;
  const int64_t b = kb + wid * share, e = min(ke, b + share);
  const int i = lane % 16, kq = V * (lane / 16);
  const bool two = s.count > 16;
  const T* x0 = static_cast<const T*>(a.src) + (int64_t)s_rows[min(i, s.count - 1)] * a.lds;
  const T* x1 = static_cast<const T*>(a.src) + (int64_t)s_rows[min(16 + i, s.count - 1)] * a.lds;
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
  for (int j = threadIdx.x; j < s.count * RP; j += kShrinkThreads) {
    const int row = j / RP, r = j % RP;
    float v = red[0][row][r];
#pragma unroll
    for (int w = 1; w < NW; ++w) v += red[w][row][r];
    if (r >= a.R) v = 0.f;
    if (a.splits > 1) a.part[(split * a.n + s.start + row) * RP + r] = v;
    else shrink_finish(a, s.g, s.start + row, s_rows[row], r, v);
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
    shrink_finish(a, s.g, s.start + j / a.RP, a.perm[s.start + j / a.RP], j % a.RP, v);
  }
}

// ------------------------------------------------------------------ outer
// Pairs of bf16 values with infinities and NaN as zeros.
__device__ __forceinline__ lr_u32x4 lr_finite(lr_u32x4 v) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t bad = ((v[w] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;   // exponents of all ones carry out
    v[w] &= ~((bad >> 15) * 0xffffu);
  }
  return v;
}

// Whether any sum of the wavefront is NaN (the same for all its lanes).
template <int NT>
__device__ __forceinline__ bool lr_any_nan(const f32x4 (&acc)[NT][4]) {
  bool nan = false;
#pragma unroll
  for (int q = 0; q < NT; ++q)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) nan |= acc[q][j][r] != acc[q][j][r];
  return __ballot(nan) != 0;
}

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
  int32_t split_rows;
};

// A wavefront holds rank x 64 outputs: lane l covers columns 4 (l%16) .. + 3, so
// that it reads 8 or 16 bytes of a row and writes 16 bytes of an output row; column
// q of the four is one matrix product.  In bf16 the rows' coefficients enter as
// three bf16 terms (they are fp32), 32 rows to a step; in fp32 4 rows to a product.
// An infinite src times a coefficient's later terms (zero, or of the other sign) would
// be a NaN that the product itself is not: sums that end as NaN are formed again with
// such values against the first term alone, which also gives the NaN that are right.
//
// Sums of a wavefront's 64 columns from c0 over the adapter's sorted rows p0, p0 + 1 .. p0 + 31, then from p0 + STRIDE
// on.  AGAIN: infinities and NaN of src meet the first term only.
template <class T, int NT, int STRIDE, bool AGAIN>
__device__ __forceinline__ void outer_sums(const OuterArgs& a, int64_t c0, int g, int p0, f32x4 (&acc)[NT][4]) {
  constexpr int TERMS = 3;
  const int lane = threadIdx.x & 63, i = lane % 16, kg = lane / 16;
  const int pe = a.off[g + 1];
  const int64_t c = c0 + 4 * i;
  const int64_t cl = c < a.L ? c : 0;             // lanes past the row read its start; they store nothing
  const float sc = a.by_row && a.scale ? a.scale[g] : 1.f;
#pragma unroll
  for (int q = 0; q < NT; ++q)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[q][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // coefficient of sorted row p, rank 16 q + i
  auto coef = [&](int p, int64_t row, int q) {
    const int r = 16 * q + i;
    return r < a.R ? sc * a.coef[(a.by_row ? row : (int64_t)p) * a.ldc + r] : 0.f;
  };
  for (; p0 < pe; p0 += STRIDE) {
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
        lr_split8(x, t);
#pragma unroll
        for (int z = TERMS - 1; z >= 0; --z)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[q][j] = lr_mfma<uint16_t>(t[z], AGAIN && z > 0 ? lr_finite(b[j]) : b[j], acc[q][j]);
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
}

// Element r of acc[q][j] is rank 16 q + 4 (l/16) + r, column c0 + 4 (l%16) + j.
template <int NT>
__device__ __forceinline__ void outer_store(const OuterArgs& a, int64_t c0, int g, const f32x4 (&acc)[NT][4]) {
  const int lane = threadIdx.x & 63, kg = lane / 16;
  const int64_t c = c0 + 4 * (lane % 16);
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

// split_rows false: the block's wavefronts take 64 columns each (long rows: enough
// blocks).  true: they take the same 64 columns and every fourth step of 32
// rows, and join in LDS (short rows: four times the wavefronts).
template <class T, int NT, bool ROWSPLIT>
__device__ __forceinline__ void outer_block(const OuterArgs& a, int64_t block, int g, float (*red)[16 * NT][68]) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, i = lane % 16, kg = lane / 16;
  const int64_t c0 = (block * (ROWSPLIT ? 1 : 4) + (ROWSPLIT ? 0 : wid)) * 64;
  if (!ROWSPLIT && c0 >= a.L) return;             // no barriers follow
  constexpr int STRIDE = ROWSPLIT ? 128 : 32;
  const int p0 = a.off[g] + (ROWSPLIT ? 32 * wid : 0);
  f32x4 acc[NT][4];
  outer_sums<T, NT, STRIDE, false>(a, c0, g, p0, acc);
  if constexpr (sizeof(T) == 2) {
    if (lr_any_nan(acc)) outer_sums<T, NT, STRIDE, true>(a, c0, g, p0, acc);
  }
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
  outer_store<NT>(a, c0, g, acc);
}

// Both low-rank products of a long dy in one launch (its rows are the largest array of a
// backward): dup_g = sum of t dy, and the partial sums of dt = up_g dy.  Two blocks
// take the same columns of the same adapter's rows, one for each product; their
// numbers differ by 8, so they run on one XCD at about the same time and the second to
// read a line finds it in that XCD's L2 (1000000 columns, 512 rows, 8 adapters of rank 16 in
// bf16: 1.2 GB fetched for 1.3 GB of operands).  405 us there, 4.3 TB/s; two launches one
// after the other 690; one block doing both 501 (209 registers, two wavefronts per SIMD).
// dup: a wavefront holds rank x 64 sums; coefficients of kPassRows rows lie in
//   LDS as operands (bf16: three terms); adapters with more rows take further rounds, which add to dup.
// dt: a wavefront takes 32 rows and its part of the columns, the block joins in LDS, and
//   one partial per block goes to memory.
// grid = (16 per 8 column ranges, adapters), 512 threads.
constexpr int kPassRows = 128;
struct PassArgs {
  OuterArgs o;            // src = dy, coef = t by row, out = dup
  const void* up;         // G x R rows of L values
  int64_t ldm;
  float* part;            // [range][sorted row][RP]
  int64_t n, ranges;
  int32_t RP, chunks;     // chunks: pieces of 64 columns per wavefront
};

template <class T, int NT>
struct PassShared {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int S = kPassRows / 32, TERMS = BF ? 3 : 2;
  union {
    // operands of one step of 32 rows: bf16: [term][lane] of 16 bytes; fp32: [half][lane] of 4 values
    lr_u32x4 coef[S][NT][TERMS][64];
    float dt[kPassThreads / 64][32][16 * NT + 1];
  };
  int32_t rows[kPassRows];
};

template <class T, int NT>
__device__ __forceinline__ void pass_outer(const PassArgs& a, int64_t range, int g, PassShared<T, NT>& sh) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int NW = kPassThreads / 64, S = kPassRows / 32;
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int pb = a.o.off[g], pe = a.o.off[g + 1];
  const int i = lane % 16, kg = lane / 16;
  // the wavefronts take neighbouring pieces, so that the block reads 8 of them of a row at about the same time
  const int64_t w0 = range * a.chunks * NW * 64 + wid * 64;
  const float sc = a.o.scale ? a.o.scale[g] : 1.f;
  const T* const src = static_cast<const T*>(a.o.src);
  bool nan = false;                                // the same for the wavefront
  for (int p0 = pb; p0 < pe || p0 == pb; p0 += kPassRows) {    // also once for an adapter without rows
    const int cnt = min(kPassRows, pe - p0);
    __syncthreads();                               // the last round's coefficients have been read
    if ((int)threadIdx.x < kPassRows && cnt > 0) sh.rows[threadIdx.x] = a.o.perm[p0 + min((int)threadIdx.x, cnt - 1)];
    __syncthreads();
    for (int j = threadIdx.x; j < S * NT * 64; j += kPassThreads) {
      const int s = j / (NT * 64), q = j / 64 % NT, l = j % 64;
      if (32 * s >= cnt) break;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int p = 32 * s + (BF ? 8 * (l / 16) + e : 4 * e + l / 16), r = 16 * q + l % 16;
        x[e] = p < cnt && r < a.o.R ? sc * a.o.coef[(int64_t)sh.rows[p] * a.o.ldc + r] : 0.f;
      }
      if constexpr (BF) {
        lr_u32x4 t[3];
        lr_split8(x, t);
#pragma unroll
        for (int z = 0; z < 3; ++z) sh.coef[s][q][z][l] = t[z];
      } else {
#pragma unroll
        for (int z = 0; z < 2; ++z)
          sh.coef[s][q][z][l] = lr_u32x4{__float_as_uint(x[4 * z]), __float_as_uint(x[4 * z + 1]),
                                         __float_as_uint(x[4 * z + 2]), __float_as_uint(x[4 * z + 3])};
      }
    }
    __syncthreads();
    // steps of 32 rows by 64 columns, rows first; the loads of the next two (fp32: one) are in
    // flight while one is multiplied
    typedef typename std::conditional<BF, lr_u32x2, f32x4>::type Piece;
    const int steps = (max(cnt, 1) + 31) / 32;
    const int64_t left = a.o.L - w0;
    const int pieces = left <= 0 ? 0 : (int)min((int64_t)a.chunks, (left + NW * 64 - 1) / (NW * 64));
    auto load = [&](int ch, int s, Piece (&v)[8]) {
      const int64_t c0 = w0 + NW * 64 * ch, c = c0 + 4 * i;
      const T* p = src + (c < a.o.L ? c : c0);     // lanes past the row read inside it; they store nothing
#pragma unroll
      for (int e = 0; e < 8; ++e)
        v[e] = *reinterpret_cast<const Piece*>(p + (int64_t)sh.rows[32 * s + (BF ? 8 * kg + e : 4 * e + kg)] * a.o.lds);
    };
    f32x4 acc[NT][4];
    auto clear = [&] {
#pragma unroll
      for (int q = 0; q < NT; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[q][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    auto multiply = [&](int s, Piece (&v)[8]) {
      if constexpr (BF) {
        if (32 * s + 32 > cnt) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (32 * s + 8 * kg + e >= cnt) v[e] = lr_u32x2{0, 0};
        }
        lr_u32x4 b[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {              // rows 2 w and 2 w + 1 of each column
          b[0][w] = __builtin_amdgcn_perm(v[2 * w + 1][0], v[2 * w][0], 0x05040100);
          b[1][w] = __builtin_amdgcn_perm(v[2 * w + 1][0], v[2 * w][0], 0x07060302);
          b[2][w] = __builtin_amdgcn_perm(v[2 * w + 1][1], v[2 * w][1], 0x05040100);
          b[3][w] = __builtin_amdgcn_perm(v[2 * w + 1][1], v[2 * w][1], 0x07060302);
        }
#pragma unroll
        for (int q = 0; q < NT; ++q)
#pragma unroll
          for (int z = 2; z >= 0; --z) {
            const lr_u32x4 t = sh.coef[s][q][z][lane];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[q][j] = lr_mfma<uint16_t>(t, b[j], acc[q][j]);
          }
      } else {
#pragma unroll
        for (int q = 0; q < NT; ++q) {
          const lr_u32x4 lo = sh.coef[s][q][0][lane], hi = sh.coef[s][q][1][lane];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = __uint_as_float(e < 4 ? lo[e] : hi[e - 4]);
            const bool in = 32 * s + 4 * e + kg < cnt;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              acc[q][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, in ? v[e][j] : 0.f, acc[q][j], 0, 0, 0);
          }
        }
      }
    };
    // element r of acc[q][j]: rank 16 q + 4 kg + r, column c + j
    auto store = [&](int ch) {
      const int64_t c = w0 + NW * 64 * ch + 4 * i;
#pragma unroll
      for (int q = 0; q < NT; ++q)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int rank = 16 * q + 4 * kg + r;
          if (rank >= a.o.R || c >= a.o.L) continue;
          float* o = a.o.out + ((int64_t)g * a.o.R + rank) * a.o.ldo + c;
          if (c + 4 <= a.o.L) {
            f32x4 x = {acc[q][0][r], acc[q][1][r], acc[q][2][r], acc[q][3][r]};
            if (p0 > pb) x += *reinterpret_cast<const f32x4*>(o);
            *reinterpret_cast<f32x4*>(o) = x;
          } else {
            for (int j = 0; c + j < a.o.L; ++j)
              o[j] = (p0 > pb ? o[j] : 0.f) + (j == 0 ? acc[q][0][r] : j == 1 ? acc[q][1][r] : acc[q][2][r]);
          }
        }
    };
    if (cnt <= 0) {                                // an adapter without rows: zeros
      clear();
      for (int ch = 0; ch < pieces; ++ch) store(ch);
      break;
    }
    constexpr int D = BF ? 3 : 2;
    Piece v[D][8];
    const int total = pieces * steps;
    int lch = 0, ls = 0, mch = 0, ms = 0, loaded = 0;
    auto next = [&](Piece (&x)[8]) {
      if (loaded >= total) return;
      load(lch, ls, x);
      ++loaded;
      if (++ls == steps) { ls = 0; ++lch; }
    };
#pragma unroll
    for (int u = 0; u < D - 1; ++u) next(v[u]);
    for (int it = 0; it < total; it += D) {
#pragma unroll
      for (int u = 0; u < D; ++u) {
        if (it + u < total) {
          next(v[(u + D - 1) % D]);
          if (ms == 0) clear();
          multiply(ms, v[u]);
          if (++ms == steps) {
            if constexpr (BF) nan |= lr_any_nan(acc);
            store(mch);
            ms = 0;
            ++mch;
          }
        }
      }
    }
  }
  if constexpr (BF) {
    if (nan) {                                     // as in outer_block: rare, so each piece again, over all its rows
      f32x4 acc[NT][4];
      for (int64_t c0 = w0; c0 < min(a.o.L, w0 + NW * 64 * a.chunks); c0 += NW * 64) {
        outer_sums<T, NT, 32, true>(a.o, c0, g, pb, acc);
        outer_store<NT>(a.o, c0, g, acc);
      }
    }
  }
}

template <class T, int NT>
__device__ __forceinline__ void pass_shrink(const PassArgs& a, int64_t range, int g, PassShared<T, NT>& sh) {
  constexpr int NW = kPassThreads / 64, RP = 16 * NT;
  constexpr int V = 16 / (int)sizeof(T), STEP = 4 * V;
  constexpr int F = NT == 1 ? 4 : 2;              // 16-row fragments of a round
  constexpr int U = (sizeof(T) == 2 ? 64 : 32) / STEP;   // steps whose loads are in flight together
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int pb = a.o.off[g], pe = a.o.off[g + 1];
  const int i = lane % 16, kq = V * (lane / 16);
  // neighbouring pieces of U steps, as the other product's wavefronts sweep the range
  const int64_t b = range * a.chunks * NW * 64, e = min(a.o.L, b + a.chunks * NW * 64);
  const T* m[NT];
#pragma unroll
  for (int q = 0; q < NT; ++q)                    // ranks past R read the last one; their sums are dropped
    m[q] = static_cast<const T*>(a.up) + ((int64_t)g * a.o.R + min(16 * q + i, a.o.R - 1)) * a.ldm;
  for (int p0 = pb; p0 < pe; p0 += 16 * F) {
    const int cnt = min(16 * F, pe - p0);
    const T* x[F];
    f32x4 acc[F][NT];
#pragma unroll
    for (int f = 0; f < F; ++f) {
      x[f] = static_cast<const T*>(a.o.src) + (int64_t)a.o.perm[p0 + min(16 * f + i, cnt - 1)] * a.o.lds;
#pragma unroll
      for (int q = 0; q < NT; ++q) acc[f][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    int64_t k = b + wid * U * STEP;
    for (; k + U * STEP <= e; k += NW * U * STEP) {
      lr_u32x4 vx[F][U], vm[U][NT];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < NT; ++q) vm[u][q] = *reinterpret_cast<const lr_u32x4*>(m[q] + k + u * STEP + kq);
#pragma unroll
      for (int f = 0; f < F; ++f)
        if (16 * f < cnt) {
#pragma unroll
          for (int u = 0; u < U; ++u) vx[f][u] = *reinterpret_cast<const lr_u32x4*>(x[f] + k + u * STEP + kq);
        }
#pragma unroll
      for (int f = 0; f < F; ++f)
        if (16 * f < cnt) {
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < NT; ++q) acc[f][q] = lr_mfma<T>(vx[f][u], vm[u][q], acc[f][q]);
        }
    }
    for (; k < e; k += STEP) {                     // (the one wavefront whose piece holds the end)
      const int64_t o = k + kq, valid = e - o;
#pragma unroll
      for (int f = 0; f < F; ++f) {
        const lr_u32x4 vx = lr_load16(x[f] + o, valid);
#pragma unroll
        for (int q = 0; q < NT; ++q) acc[f][q] = lr_mfma<T>(vx, lr_load16(m[q] + o, valid), acc[f][q]);
      }
    }
#pragma unroll
    for (int h = 0; h < F / 2; ++h) {              // 32 rows at a time through LDS
      __syncthreads();                             // the last sums have been read
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int q = 0; q < NT; ++q)
#pragma unroll
          for (int r = 0; r < 4; ++r) sh.dt[wid][16 * f + 4 * (lane / 16) + r][16 * q + i] = acc[2 * h + f][q][r];
      __syncthreads();
      for (int j = threadIdx.x; j < 32 * RP; j += kPassThreads) {
        const int row = j / RP, r = j % RP;
        if (32 * h + row >= cnt) break;
        float v = sh.dt[0][row][r];
#pragma unroll
        for (int w = 1; w < NW; ++w) v += sh.dt[w][row][r];
        a.part[(range * a.n + p0 + 32 * h + row) * RP + r] = r < a.o.R ? v : 0.f;
      }
    }
  }
}

template <class T, int NT>
__global__ __launch_bounds__(kPassThreads, NT == 1 ? 4 : 2) void pass_kernel(PassArgs a) {
  __shared__ PassShared<T, NT> sh;
  const int64_t range = (int64_t)(blockIdx.x / 16) * 8 + blockIdx.x % 8;
  if (range >= a.ranges) return;
  if (blockIdx.x / 8 % 2) pass_shrink<T, NT>(a, range, blockIdx.y, sh);
  else pass_outer<T, NT>(a, range, blockIdx.y, sh);
}

// dt of the sorted rows [0, off[G]) from the ranges' partials, added in order; one thread per value.
__global__ __launch_bounds__(256) void pass_reduce_kernel(const float* __restrict__ part, int32_t ranges, int64_t n,
                                                          int32_t RP, int32_t G, const int32_t* __restrict__ gid,
                                                          const float* __restrict__ scale, float* __restrict__ ts) {
  // a block takes 16 values, 16 threads each: thread k adds every 16th range, then they join in order
  __shared__ float red[16][17];
  const int v = threadIdx.x % 16, k = threadIdx.x / 16;
  const int64_t at = (int64_t)blockIdx.x * 16 + v, total = n * RP;
  float x = 0.f;
  if (at < total && gid[at / RP] < G) {
    int q = k;
    for (; q + 48 < ranges; q += 64) {            // four loads in flight
      float w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) w[u] = part[(q + 16 * u) * total + at];
#pragma unroll
      for (int u = 0; u < 4; ++u) x += w[u];
    }
    for (; q < ranges; q += 16) x += part[q * total + at];
  }
  red[k][v] = x;
  __syncthreads();
  if (k || at >= total) return;
  const int g = gid[at / RP];
  if (g >= G) return;
#pragma unroll
  for (int u = 1; u < 16; ++u) x += red[u][v];
  ts[at] = scale ? scale[g] * x : x;
}

// Both gradients of a bank in one launch: blocks [0, blocks0) of the first, then the second.
// grid = (blocks0 + blocks1, adapters).
template <class T, int NT>
__global__ __launch_bounds__(256) void outer_kernel(OuterArgs a0, OuterArgs a1, int64_t blocks0) {
  __shared__ float red[3][16 * NT][68];
  const bool second = blockIdx.x >= blocks0;
  const OuterArgs& a = second ? a1 : a0;
  const int64_t block = second ? blockIdx.x - blocks0 : blockIdx.x;
  if (a.split_rows) outer_block<T, NT, true>(a, block, blockIdx.y, red);
  else outer_block<T, NT, false>(a, block, blockIdx.y, red);
}

}  // namespace ot
