// Product of few rows with a weight that is streamed once, shared by the dense
// gated feed-forward and the matrix product with an epilogue.  Internal to libcep.
#pragma once

#include "block_ops.h"
#include "gemm_common.h"

namespace cep {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr int kCols = 128;   // columns of a workgroup
constexpr int kUnit = 32;    // K of a unit
constexpr int kPitch = 132;  // floats of a row of the waves' sums in LDS

struct RowsArgs {
  const __bf16 *A[2];  // the rows (their hi and lo terms)
  const __bf16 *B0, *B1;
  int64_t lda, ldb;
  int M, N, K;
  int splits, col_blocks;
  const float *gu;  // kFused: the shares [gu_splits][M][2 K] of g and u
  int gu_splits;
};

// Where the rows come from: kRows memory; kTerms memory, as hi and lo; kFused
// silu(g) u of the g and u sums, computed for the workgroup's share of K and
// kept in LDS as hi and lo.
enum Source { kRows, kTerms, kFused };
constexpr int kFusedBytes = 32768;  // of those terms

__device__ inline void split_hidden(const f32x4 &g, const f32x4 &u, bf16x4 *hi, bf16x4 *lo) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const float h = silu_mul(g[r], u[r]);
    (*hi)[r] = (__bf16)h;
    (*lo)[r] = (__bf16)(__builtin_isinf((float)(*hi)[r]) ? 0.f : h - (float)(*hi)[r]);
  }
}

// Four columns of g and u of a row, the shares added in order, the loads of eight
// on the way at once (of one after the other, 32 shares took 12 us).
__device__ inline void sum_gu(const float *part, int splits, int M, int I, int64_t row, int col,
                              f32x4 *g, f32x4 *u) {
  *g = *u = f32x4{};
  const float *p = part + row * 2 * I + col;
  const int64_t share = (int64_t)M * 2 * I;
  for (int i0 = 0; i0 < splits; i0 += 8) {
    f32x4 a[8], b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float *q = p + min(i0 + i, splits - 1) * share;
      a[i] = *(const f32x4 *)q;
      b[i] = *(const f32x4 *)(q + I);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      *g += i0 + i < splits ? a[i] : f32x4{};
      *u += i0 + i < splits ? b[i] : f32x4{};
    }
  }
}

// LDS of a workgroup.
template <int MF, Source SRC>
struct RowsLds {
  static constexpr int NA = SRC == kRows ? MF : 2 * MF;       // fragments of A
  static constexpr int LOADS = 8 + (SRC == kFused ? 0 : NA);  // 1 KB loads of a unit
  static constexpr int DEPTH = 3;                             // units on the way
  static constexpr int RING = LOADS * 1024 * DEPTH;
  static constexpr int SUMS = MF * 16 * kPitch * 4;
  __attribute__((aligned(1024))) uint8_t ring[4 * (RING > SUMS ? RING : SUMS)];
  __attribute__((aligned(16))) uint8_t terms[SRC == kFused ? kFusedBytes : 16];
};

// MF row fragments of 16; DUAL: gate and up columns; column block cb, share sp.
// out(row, col, v) takes the share's sums of four columns from col (DUAL: those
// of the up projection from a.N on).
template <int MF, Source SRC, bool DUAL, class Out>
__device__ inline void rows_tile(const RowsArgs &a, int cb, int sp, RowsLds<MF, SRC> &mem, Out out) {
  typedef RowsLds<MF, SRC> L;
  constexpr int NF = kCols / 16, NA = L::NA, LOADS = L::LOADS, DEPTH = L::DEPTH, RING = L::RING;
  uint8_t *lds = mem.ring, *terms = mem.terms;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l15 = lane & 15, g4 = lane >> 4;
  const int n0 = cb * (DUAL ? 64 : kCols);
  const int units = a.K / kUnit;
  const int u0 = (int)((int64_t)units * sp / a.splits), u1 = (int)((int64_t)units * (sp + 1) / a.splits);
  const int mine = u1 - u0 > wave ? (u1 - u0 - wave + 3) / 4 : 0;  // units u0 + wave + 4 i

  // Loads of a unit: 8 pieces of B, four lines of k x 128 columns each
  // (16-byte chunk pair p of line k at p ^ (k % 4 + k / 8 % 2 * 4)), then 16
  // rows x 32 of k a piece of A (chunk c of row r at c ^ (r / 4 % 4)).
  const char *srcB[2];
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const int pos = l15, chunk = ((((pos >> 1) ^ g4 ^ (v << 2)) << 1) | (pos & 1));
    const bool up = DUAL && chunk >= 8;
    const int col = min(n0 + (DUAL ? chunk & 7 : chunk) * 8, a.N - 8);
    srcB[v] = (const char *)((up ? a.B1 : a.B0) + (int64_t)g4 * a.ldb + col);
  }
  const char *srcA[NA];
#pragma unroll
  for (int i = 0; i < (SRC == kFused ? 0 : NA); ++i) {
    const int r = lane >> 2;
    const int row = min((i % MF) * 16 + r, a.M - 1);
    srcA[i] = (const char *)(a.A[i / MF] + row * a.lda + ((lane & 3) ^ ((r >> 2) & 3)) * 8);
  }
  uint8_t *ring = lds + wave * RING;
  const uint32_t ring0 = lds_offset(ring);
  auto issue = [&](int i) {
    const int64_t u = u0 + wave + 4 * i;
    const uint32_t to = ring0 + (i % DEPTH) * LOADS * 1024;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      dma16(srcB[(e >> 1) & 1] + (u * kUnit + e * 4) * a.ldb * 2, to + e * 1024);
#pragma unroll
    for (int p = 0; p < LOADS - 8; ++p) dma16(srcA[p] + u * kUnit * 2, to + (8 + p) * 1024);
  };
  f32x4 acc[MF][NF] = {};
  // kFused: rows [M][pitch] of hi, then of lo, from column u0 * 32 on; a row's
  // pitch is the share's whole units and room for a shorter one
  const int pitch = (u1 - u0 + 1) * kUnit;
  const int lrow = min(l15, a.M - 1) * pitch + g4 * 8;
  auto multiply = [&](const uint8_t *at, int u) {
    bf16x8 fa[NA];
#pragma unroll
    for (int p = 0; p < NA; ++p)
      if (SRC == kFused)
        fa[p] = *(const bf16x8 *)((const __bf16 *)terms + p * a.M * pitch + lrow + (u - u0) * kUnit);
      else fa[p] = *(const bf16x8 *)(at + (8 + p) * 1024 + l15 * 64 + (g4 ^ (l15 >> 2)) * 16);
    const int k = g4 * 8 + (l15 >> 2), f = (k & 3) | ((k >> 3) & 1) << 2;
#pragma unroll
    for (int n = 0; n < NF; ++n) {
      union { bf16x8 v; bf16x4 h[2]; } b;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        b.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
            (__attribute__((address_space(3))) bf16x4 *)(at + (k + h * 4) * 256 + ((n ^ f) << 5) +
                                                          (l15 & 3) * 8));
#pragma unroll
      for (int p = 0; p < NA; ++p)
        acc[p % MF][n] =
            __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v, fa[p], acc[p % MF][n], 0, 0, 0);
    }
  };
#pragma unroll
  for (int i = 0; i < DEPTH; ++i)
    if (i < mine) issue(i);
  if (SRC == kFused) {
    const int k0 = u0 * kUnit, k1 = sp == a.splits - 1 ? a.K : u1 * kUnit;
    for (int q = tid; q < a.M * pitch / 4; q += 256) {
      const int row = q / (pitch / 4), c = (q % (pitch / 4)) * 4;
      bf16x4 hi = {}, lo = {};
      if (k0 + c < k1) {
        f32x4 g, u;
        sum_gu(a.gu, a.gu_splits, a.M, a.K, row, k0 + c, &g, &u);
        split_hidden(g, u, &hi, &lo);
      }
      *(bf16x4 *)((__bf16 *)terms + row * pitch + c) = hi;
      *(bf16x4 *)((__bf16 *)terms + (a.M + row) * pitch + c) = lo;
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  }
  for (int i = 0; i < mine; ++i) {
    wait_stages<LOADS, DEPTH - 1>(min(DEPTH - 1, mine - 1 - i));
    asm volatile("" ::: "memory");
    multiply(ring + (i % DEPTH) * LOADS * 1024, u0 + wave + 4 * i);
    // the reads of this unit are done before its place is filled again
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (i + DEPTH < mine) issue(i + DEPTH);
  }
  if (a.K % kUnit && sp == a.splits - 1 && wave == (units - u0) % 4) {
    // the last, shorter unit, zeros past K
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      const int64_t k0 = (int64_t)units * kUnit + e * 4;
      if (k0 + g4 < a.K) v = *(const uint4 *)(srcB[(e >> 1) & 1] + k0 * a.ldb * 2);
      *(uint4 *)(ring + e * 1024 + lane * 16) = v;
    }
#pragma unroll
    for (int p = 0; p < LOADS - 8; ++p) {
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      const int chunk = (lane & 3) ^ ((lane >> 4) & 3);
      if (units * kUnit + chunk * 8 < a.K) v = *(const uint4 *)(srcA[p] + (int64_t)units * kUnit * 2);
      *(uint4 *)(ring + (8 + p) * 1024 + lane * 16) = v;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    multiply(ring, units);
  }
  __syncthreads();
  // the four waves' sums, added in wave order
  float *sums = (float *)lds;
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int n = 0; n < NF; ++n)
      *(f32x4 *)(sums + ((wave * MF + i) * 16 + l15) * kPitch + n * 16 + g4 * 4) = acc[i][n];
  __syncthreads();
  // four columns of a row each; returns false outside the product
  auto place = [&](int q, int *row, int *col) {
    const int c = (q % (kCols / 4)) * 4;
    *row = q / (kCols / 4);
    const int n = n0 + (DUAL ? c & 63 : c);
    *col = DUAL && c >= 64 ? a.N + n : n;
    return *row < a.M && n < a.N;
  };
  for (int q = tid; q < MF * 16 * kCols / 4; q += 256) {
    int row, col;
    if (!place(q, &row, &col)) continue;
    const float *p = sums + (q / (kCols / 4)) * kPitch + (q % (kCols / 4)) * 4;
    f32x4 v = *(const f32x4 *)p;
#pragma unroll
    for (int w = 1; w < 4; ++w) v += *(const f32x4 *)(p + w * MF * 16 * kPitch);
    out(row, col, v);
  }
}

}  // namespace cep
