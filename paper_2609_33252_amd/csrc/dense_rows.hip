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
#include "dense.h"
#include "rows_tile.h"

#include <algorithm>

namespace cep {
namespace {

struct FfnRowsArgs : RowsArgs {
  float *part;  // [splits][M][columns]; unused with one share of a plain product
  __bf16 *y;    // its output
  int64_t ldy;
};

template <int MF, Source SRC, bool DUAL>
__global__ __launch_bounds__(256) void k_rows(FfnRowsArgs a) {
  __shared__ RowsLds<MF, SRC> lds;
  const int cb = blockIdx.x % a.col_blocks, sp = blockIdx.x / a.col_blocks;
  const int64_t width = DUAL ? 2 * a.N : a.N;
  rows_tile<MF, SRC, DUAL>(a, cb, sp, lds, [&](int row, int col, const f32x4 &v) {
    if (!DUAL && a.splits == 1)
      *(uint2 *)(a.y + row * a.ldy + col) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
    else *(f32x4 *)(a.part + ((int64_t)sp * a.M + row) * width + col) = v;
  });
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
void launch_rows(const FfnRowsArgs &a, hipStream_t s) {
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
  FfnRowsArgs a{};
  a.A[0] = x;
  a.B0 = wg, a.B1 = wu;
  a.lda = ld_x, a.ldb = I;
  a.M = rows, a.N = I, a.K = d;
  a.splits = p.splits1, a.col_blocks = blocks_of(I, 64);
  a.part = part;
  launch_rows<kRows, true>(a, s);
  FfnRowsArgs b{};
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
