// Dense gated feed-forward of few rows for gfx950: the weights are streamed
// once, and the rows ride along.
//
// Measured: one row of 4096 x 2048 (50 MB of weights) 17.7 us from HBM (forty sets
// of weights in turn), 15.6 with the weights in the last-level cache (three sets):
// of the three launches' 7.7, 5.8 and 1.8 us the start and end are the larger part,
// not memory's rate.
//
// A workgroup takes all rows (up to 32), 128 columns (64 of the gate and the
// same 64 of the up projection, or 128 of the down projection) and a share of
// K; its four waves take the share's 32-wide units in turn, each with
// a ring of its own in LDS and no barrier between them.  The waves' sums meet
// in LDS, the shares' in a float32 scratch.  The shares are added in order by
// the launch that follows: those of g and u by k_rows_hidden, which applies
// silu(g) u, or with very few rows by the workgroups of the down projection,
// each for its share of K; those of y by k_rows_sum.  (Having the workgroup
// that comes last to its columns add them instead, behind a device-wide fence,
// cost 10 us a launch: the fence writes back a whole L2.)
//
// The hidden row is kept as two bf16 terms, h = hi + lo (16 bits of mantissa):
// the second costs matrix instructions that a weight-bound product has to
// spare, and the one rounding of h would show in y.
#include "block_ops.h"
#include "dense.h"
#include "gemm_common.h"

#include <algorithm>

namespace cep {
namespace {

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
  float *part;  // [splits][M][columns]; unused with one share of a plain product
  __bf16 *y;    // its output
  int64_t ldy;
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

// MF row fragments of 16; DUAL: gate and up columns.
template <int MF, Source SRC, bool DUAL>
__global__ __launch_bounds__(256) void k_rows(RowsArgs a) {
  constexpr int NF = kCols / 16;
  constexpr int NA = SRC == kRows ? MF : 2 * MF;            // fragments of A
  constexpr int LOADS = 8 + (SRC == kFused ? 0 : NA);       // 1 KB loads of a unit
  constexpr int DEPTH = 3;                                  // units on the way
  constexpr int RING = LOADS * 1024 * DEPTH;
  constexpr int SUMS = MF * 16 * kPitch * 4;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * (RING > SUMS ? RING : SUMS)];
  __shared__ __attribute__((aligned(16))) uint8_t terms[SRC == kFused ? kFusedBytes : 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l15 = lane & 15, g4 = lane >> 4;
  const int cb = blockIdx.x % a.col_blocks, sp = blockIdx.x / a.col_blocks;
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
  const int64_t width = DUAL ? 2 * a.N : a.N;
  const bool direct = !DUAL && a.splits == 1;
  // four columns of a row each; returns false outside the product
  auto place = [&](int q, int *row, int *col) {
    const int c = (q % (kCols / 4)) * 4;
    *row = q / (kCols / 4);
    const int n = n0 + (DUAL ? c & 63 : c);
    *col = DUAL && c >= 64 ? a.N + n : n;
    return *row < a.M && n < a.N;
  };
  auto to_y = [&](int row, int col, const f32x4 &v) {
    *(uint2 *)(a.y + row * a.ldy + col) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
  };
  for (int q = tid; q < MF * 16 * kCols / 4; q += 256) {
    int row, col;
    if (!place(q, &row, &col)) continue;
    const float *p = sums + (q / (kCols / 4)) * kPitch + (q % (kCols / 4)) * 4;
    f32x4 v = *(const f32x4 *)p;
#pragma unroll
    for (int w = 1; w < 4; ++w) v += *(const f32x4 *)(p + w * MF * 16 * kPitch);
    if (direct) to_y(row, col, v);
    else *(f32x4 *)(a.part + ((int64_t)sp * a.M + row) * width + col) = v;
  }
}

// h = silu(g) u from the shares of g and u, as hi + lo.
__global__ __launch_bounds__(256) void k_rows_hidden(const float *part, int splits, int M, int I,
                                                     float *pre, __bf16 *hi, __bf16 *lo) {
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = q / (I / 4);
  const int col = (int)(q % (I / 4)) * 4;
  if (row >= M) return;
  f32x4 g, u;
  sum_gu(part, splits, M, I, row, col, &g, &u);
  if (pre) {
    *(f32x4 *)(pre + row * 2 * I + col) = g;
    *(f32x4 *)(pre + row * 2 * I + I + col) = u;
  }
  bf16x4 a, b;
  split_hidden(g, u, &a, &b);
  *(bf16x4 *)(hi + row * I + col) = a;
  *(bf16x4 *)(lo + row * I + col) = b;
}

// y from its shares.
__global__ __launch_bounds__(256) void k_rows_sum(const float *part, int splits, int M, int N,
                                                  __bf16 *y, int64_t ldy) {
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = q / (N / 4);
  const int col = (int)(q % (N / 4)) * 4;
  if (row >= M) return;
  f32x4 v = {};
#pragma unroll 8
  for (int i = 0; i < splits; ++i) v += *(const f32x4 *)(part + ((int64_t)i * M + row) * N + col);
  *(uint2 *)(y + row * ldy + col) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
}

int blocks_of(int n, int per) { return (n + per - 1) / per; }

template <Source SRC, bool DUAL>
void launch_rows(const RowsArgs &a, hipStream_t s) {
  const dim3 grid(a.col_blocks * a.splits);
  auto *k = k_rows<1, SRC, DUAL>;
  if constexpr (SRC != kFused)
    if (a.M > 16) k = k_rows<2, SRC, DUAL>;
  hipLaunchKernelGGL(k, grid, dim3(256), 0, s, a);
}

unsigned grid_of(int64_t elements) { return (unsigned)((elements / 4 + 255) / 256); }

}  // namespace

// Rows up to which the weights are streamed.  Above it the tiled product with
// K shares is as fast (both products, us here and tiled, h in two terms; d 4096,
// d_ff 2048: 1 row 15.9, 21.4; 16 rows 19.0, 22.4; 32 rows 21.1, 23.8; 33 rows 23.8,
// 24.0; d 7168: 16 rows 27.2, 29.4; 32 rows 30.3, 31.4; 64 rows 37.0, 35.8; 32 rows
// of 256 x 128 11.3, 10.3).
constexpr int kRowsMost = 32;

RowsPlan rows_plan(int rows, int d, int I) {
  RowsPlan p{};
  p.use = rows > 0 && rows <= kRowsMost;
  if (!p.use) return p;
  // one workgroup a compute unit (a ring takes most of its LDS), at least a
  // unit for each wave
  auto splits = [&](int cols, int K) {
    return std::max(1, std::min(256 / cols, K / kUnit / 4));
  };
  p.splits1 = splits(blocks_of(I, 64), d);
  p.splits2 = splits(blocks_of(d, kCols), I);
  return p;
}

namespace {
struct RowsSpace {
  size_t part2, hi, lo, bytes;  // the shares of g and u first
};
RowsSpace rows_space(const RowsPlan &p, int rows, int d, int I) {
  RowsSpace w;
  w.part2 = align_up((size_t)p.splits1 * rows * 2 * I * 4, 256);
  w.hi = w.part2 + align_up((size_t)p.splits2 * rows * d * 4, 256);
  w.lo = w.hi + align_up((size_t)rows * I * 2, 256);
  w.bytes = w.lo + align_up((size_t)rows * I * 2, 256);
  return w;
}
}  // namespace

size_t rows_workspace(const RowsPlan &p, int rows, int d, int I) {
  return rows_space(p, rows, d, I).bytes;
}

void launch_rows_ffn(const RowsPlan &p, int rows, int d, int I, const __bf16 *x, int64_t ld_x,
                     const __bf16 *wg, const __bf16 *wu, const __bf16 *wd, __bf16 *y, int64_t ld_y,
                     float *pre, uint8_t *workspace, hipStream_t s) {
  const RowsSpace w = rows_space(p, rows, d, I);
  float *part = (float *)workspace, *part2 = (float *)(workspace + w.part2);
  __bf16 *hi = (__bf16 *)(workspace + w.hi), *lo = (__bf16 *)(workspace + w.lo);
  RowsArgs a{};
  a.A[0] = x;
  a.B0 = wg, a.B1 = wu;
  a.lda = ld_x, a.ldb = I;
  a.M = rows, a.N = I, a.K = d;
  a.splits = p.splits1, a.col_blocks = blocks_of(I, 64);
  a.part = part;
  launch_rows<kRows, true>(a, s);
  RowsArgs b{};
  b.A[0] = hi, b.A[1] = lo;
  b.B0 = wd;
  b.lda = I, b.ldb = d;
  b.M = rows, b.N = d, b.K = I;
  b.splits = p.splits2, b.col_blocks = blocks_of(d, kCols);
  b.part = part2;
  b.y = y, b.ldy = ld_y;
  b.gu = part, b.gu_splits = p.splits1;
  // Each workgroup of the down projection adds its share's g and u itself while
  // that reads up to 128 KB, which saves a launch (us, saved and not: one row of
  // 4096 x 2048, 18 KB, 15.9, 17.7; one of 7168 x 2048, 35 KB, 23.4, 25.1; four,
  // 139 KB, 26.0, 25.7; eight, 279 KB, 28.6, 26.0).
  const int share = (blocks_of(I / kUnit, p.splits2) + 1) * kUnit;
  if (rows <= 16 && rows * share * 4 <= kFusedBytes &&
      (int64_t)rows * share * 8 * p.splits1 <= 128 << 10 && !pre) {
    launch_rows<kFused, false>(b, s);
  } else {
    hipLaunchKernelGGL(k_rows_hidden, dim3(grid_of((int64_t)rows * I)), dim3(256), 0, s, part,
                       p.splits1, rows, I, pre, hi, lo);
    launch_rows<kTerms, false>(b, s);
  }
  if (p.splits2 > 1)
    hipLaunchKernelGGL(k_rows_sum, dim3(grid_of((int64_t)rows * d)), dim3(256), 0, s, part2,
                       p.splits2, rows, d, y, ld_y);
}

}  // namespace cep
