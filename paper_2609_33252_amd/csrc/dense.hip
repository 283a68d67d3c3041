// Dense gated feed-forward, y = (silu(x Wg) * (x Wu)) Wd, and its gradient, in
// bf16 with float32 accumulation, for gfx950.
//
//   g = x Wg, u = x Wu, h = silu(g) u, y = h Wd
//   dh = dy Wd^T, du = dh silu(g), dg = dh u sigma (1 + g (1 - sigma))
//   dx = dg Wg^T + du Wu^T, dWg = x^T dg, dWu = x^T du, dWd = h^T dy
//
// Six products of three layouts, C[m][n] = sum over k of A(m, k) B(k, n): A
// has k or m contiguous, B k or n.
#include "dense.h"
#include "dense_tile.h"

namespace cep {
namespace {

// What happens to the accumulated tile.
enum Epilogue {
  kStore,   // bf16 to out0
  kStore2,  // two products over the same A: bf16 to out0 and out1
  kSwiGlu,  // two products g, u: h = silu(g) u to out0 (what that rounds off to out1),
            // g and u to pre
  kGrad     // dh: with g, u from pre, [dg | du] to out0 and h to out1
};
constexpr bool is_dual(int epi) { return epi == kStore2 || epi == kSwiGlu; }

struct DenseArgs : TileArgs {
  __bf16 *out0, *out1;
  int64_t ldo;
  float *pre;   // [M][2][N]
  float *part;  // above one K share their sums: [splits][M][N, or 2 N of two products]
};

// Four consecutive outputs of row m from their sums v (and w, of the second
// product).
template <int EPI>
__device__ inline void finish(const DenseArgs &a, int64_t m, int n, const f32x4 &v, const f32x4 &w) {
  if (EPI == kStore || EPI == kStore2) store_bf16(a.out0 + m * a.ldo + n, v);
  if (EPI == kStore2) store_bf16(a.out1 + m * a.ldo + n, w);
  if (EPI == kSwiGlu) {
    f32x4 h;
#pragma unroll
    for (int r = 0; r < 4; ++r) h[r] = v[r] * sigma(v[r]) * w[r];
    store_bf16(a.out0 + m * a.ldo + n, h);
    if (a.out1) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float hi = (float)(__bf16)h[r];
        h[r] = __builtin_isinf(hi) ? 0.f : h[r] - hi;
      }
      store_bf16(a.out1 + m * a.ldo + n, h);
    }
    if (a.pre) {
      *(f32x4 *)(a.pre + m * 2 * a.N + n) = v;
      *(f32x4 *)(a.pre + m * 2 * a.N + a.N + n) = w;
    }
  }
  if (EPI == kGrad) {
    const f32x4 g = *(const f32x4 *)(a.pre + m * 2 * a.N + n);
    const f32x4 u = *(const f32x4 *)(a.pre + m * 2 * a.N + a.N + n);
    f32x4 dg, du, h;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float s = sigma(g[r]);
      dg[r] = v[r] * u[r] * s * (1.0f + g[r] * (1.0f - s));
      du[r] = v[r] * g[r] * s;
      h[r] = g[r] * s * u[r];
    }
    store_bf16(a.out0 + m * 2 * a.N + n, dg);
    store_bf16(a.out0 + m * 2 * a.N + a.N + n, du);
    store_bf16(a.out1 + m * a.N + n, h);
  }
}

// The shares' sums, added in order, and what becomes of them.
template <int EPI>
__global__ __launch_bounds__(256) void k_dense_finish(DenseArgs a) {
  const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t m = q / (a.N / 4);
  const int n = (int)(q % (a.N / 4)) * 4;
  if (m >= a.M) return;
  const int64_t width = is_dual(EPI) ? 2 * a.N : a.N;
  f32x4 v = {}, w = {};
#pragma unroll 4
  for (int i = 0; i < a.splits; ++i) {
    const float *p = a.part + ((int64_t)i * a.M + m) * width + n;
    v += *(const f32x4 *)p;
    if (is_dual(EPI)) w += *(const f32x4 *)(p + a.N);
  }
  finish<EPI>(a, m, n, v, w);
}

// Item `at` of XCD x's: its tile and share.
template <int HALF, int WM, int WN, bool A_K, bool B_K, int EPI>
__device__ inline void dense_item(const DenseArgs &a, int x, int at, uint8_t *lds) {
  constexpr bool DUAL = is_dual(EPI);
  constexpr int TN = DUAL ? HALF : 2 * HALF;
  const int n_tm = (a.M + 2 * HALF - 1) / (2 * HALF), n_tn = (a.N + TN - 1) / TN;
  // the items: the shares of a tile are separate ones, share by share
  const int items = n_tm * a.splits * n_tn;
  if (at >= piece_of(items, x)) return;
  int mt, nt;
  tile_of<kGroupM>(x * (items / 8) + min(x, items % 8) + at, n_tm * a.splits, n_tn, &mt, &nt);
  const int share = mt / n_tm;
  dense_tile<HALF, WM, WN, A_K, B_K, DUAL>(
      a, (mt - share * n_tm) * 2 * HALF, nt * TN, share, lds,
      [&](int64_t m, int n, const f32x4 &v, const f32x4 &w) {
        if (a.splits == 1) {
          finish<EPI>(a, m, n, v, w);
        } else {
          float *p = a.part + ((int64_t)share * a.M + m) * (DUAL ? 2 * a.N : a.N) + n;
          *(f32x4 *)p = v;
          if (DUAL) *(f32x4 *)(p + a.N) = w;
        }
      });
}

template <int HALF, int WM, int WN, bool A_K, bool B_K, int EPI>
__global__ __launch_bounds__(WM * WN * 64, 2) void k_dense(DenseArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[HALF * 1024];
  dense_item<HALF, WM, WN, A_K, B_K, EPI>(a, blockIdx.x & 7, blockIdx.x >> 3, lds);
}

// dx, dWg and dWu, and dWd in one launch, those with the longest tiles first:
// the tiles of one fill the compute units that the others' last round leaves.
struct GradArgs {
  DenseArgs dx, dwgu, dwd;
  int order[3], tiles[3];  // which of the three comes first, ..., and its tiles
};
template <int HALF, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64, 2) void k_dense_grads(GradArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[HALF * 1024];
  // An XCD's workgroups take its piece of the first product, then of the second,
  // ...; where one product's longer pieces end, the next one's begin.  (Workgroups
  // with nothing to do between them unbalance the dispatch: 252 tiles then took
  // two rounds.)
  int x = blockIdx.x & 7, at = blockIdx.x >> 3, which = -1;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int n = piece_of(a.tiles[i], x);
    if (which < 0) {
      if (at < n) {
        which = a.order[i];
      } else {
        at -= n;
        x = (x - a.tiles[i]) & 7;
      }
    }
  }
  if (which == 0) dense_item<HALF, WM, WN, true, true, kStore>(a.dx, x, at, lds);
  if (which == 1) dense_item<HALF, WM, WN, false, false, kStore2>(a.dwgu, x, at, lds);
  if (which == 2) dense_item<HALF, WM, WN, false, false, kStore>(a.dwd, x, at, lds);
}

// Tile and K shares of a product.
struct DensePlan {
  int tile;  // 0: 256 x 256, 1: 128 x 128 (of both products' columns)
  int splits;
  double us;  // estimated
};
constexpr int kTile[2] = {256, 128};

int64_t dense_tiles(int t, int M, int N) {
  return (int64_t)((M + kTile[t] - 1) / kTile[t]) * ((N + kTile[t] - 1) / kTile[t]);
}

// Tile and shares by an estimate of the time, in us, from these measurements
// (a product alone, steps of 64 of K):
//   256-wide tiles, one a compute unit: 12 and 1.4 a step, a round of up to 256
//     (777 x 5120 x 6144, 80 tiles: in two shares 71, in three 57)
//   128-wide ones: 3 and a step of 0.55 with one a unit (777 x 4096 x 4096, 224
//     tiles: 37), 0.85 to 1.0 with two (280 tiles of 96 steps 84, 512 tiles of
//     64 steps 64), 1.2 a round of several (1024 tiles of 64 steps 146)
//   the shares' second launch: 4, and their sums at 9 TB/s (three of 777 x 5120: 9)
// Shares have six steps at least and fit one round; they have to win by a tenth.
// Layouts and epilogues are not told apart: of 512 128-wide tiles of 64 steps,
// estimated at 67, dh (4095 x 2048 x 4096) takes 96 with its reads of g and u, and
// dWd 76.
// (A 256 x 128 tile, in four or eight waves, was no faster than two 128-wide
// ones: 4095 x 2048 x 4096 118 and 108 against 104.)
DensePlan dense_plan(int M, int n, int K, bool dual) {
  const int N = dual ? 2 * n : n, steps = K / 64;
  DensePlan best{};
  for (int t = 0; t < 2; ++t) {
    const int64_t tiles = dense_tiles(t, M, N);
    for (int s = 1; s <= 16; ++s) {
      if (s > 1 && (tiles * s > 256 || steps / s < 6)) break;
      const int64_t items = tiles * s, rest = items % 512;
      const double step = (double)steps / s;
      double us = t == 0 ? (double)((items + 255) / 256) * (12 + 1.4 * step)
                         : 3 + step * ((items > 512 ? 1.2 : 1.0) * (double)(items / 512) +
                                       (rest == 0     ? 0.0
                                        : rest <= 256 ? 0.55
                                                      : 0.85 + 0.15 * (double)(rest - 256) / 256));
      if (s > 1) us = (us + 4 + (double)s * M * N * 4 / 9e6) / 0.9;
      if ((t == 0 && s == 1) || us < best.us) best = {t, s, us};
    }
  }
  return best;
}

// Scratch of a product's shares.
size_t part_bytes(int M, int n, int K, bool dual) {
  const DensePlan p = dense_plan(M, n, K, dual);
  return p.splits > 1 ? (size_t)p.splits * M * n * (dual ? 8 : 4) : 0;
}

template <bool A_K, bool B_K, int EPI>
void launch_dense(DenseArgs a, float *part, hipStream_t s) {
  const DensePlan p = dense_plan(a.M, a.N, a.K * a.segs, is_dual(EPI));
  a.splits = p.splits;
  a.part = part;
  const int N = is_dual(EPI) ? 2 * a.N : a.N;
  const int64_t items = dense_tiles(p.tile, a.M, N) * p.splits;
  const dim3 grid((unsigned)((items + 7) / 8 * 8));
  if (p.tile == 0)
    hipLaunchKernelGGL((k_dense<128, 2, 4, A_K, B_K, EPI>), grid, dim3(512), 0, s, a);
  else
    hipLaunchKernelGGL((k_dense<64, 2, 2, A_K, B_K, EPI>), grid, dim3(256), 0, s, a);
  if (p.splits > 1)
    hipLaunchKernelGGL((k_dense_finish<EPI>),
                       dim3((unsigned)(((int64_t)a.M * (a.N / 4) + 255) / 256)), dim3(256), 0, s, a);
}

// The tile with which dx, dWg and dWu, and dWd run in one launch, -1: a launch
// each.  One launch saves the others' starts and joins their last rounds;
// launches of their own can share K and take different tiles.  Kernels' us, one
// launch of 256-wide tiles / of 128-wide ones / a launch each:
//   T 2621, d 2304, d_ff 1328 (252 tiles): 76 / 104 / 131
//   8192, 4096, 1408: 378 / 446 / 433       2048, 4096, 2048: 143 / 157 / 156
//   700, 2048, 1024: 42 / 24 / 45           39, 256, 128: 12 / 7 / 16
//   4095, 4096, 2048 (640 tiles in 2.5 rounds): 335 / 358 / 332
//   100, 2048, 8192 (dx: 16 tiles of 256 steps): 254 / 148 / 76
//   128, 4096, 2048 (dx: 32 of 64), the backward pass: 95 / 76 / 64
int grads_tile(int T, int D, int I) {
  auto steps = [](int K, int segs) { return 2 + segs * (K / 64 + (K % 64 ? 3.0 : 0.0)); };
  const int M[3] = {T, D, I}, N[3] = {D, 2 * I, D};
  const double st[3] = {steps(I, 2), steps(T, 1), steps(T, 1)};
  const DensePlan each[3] = {dense_plan(T, D, 2 * I, false), dense_plan(D, I, T, true),
                             dense_plan(I, D, T, false)};
  double least = 0;
  for (int i = 0; i < 3; ++i) {
    const int64_t tiles = dense_tiles(each[i].tile, M[i], N[i]);
    least += each[i].splits > 1 ? each[i].us + 3 : tiles_us(each[i].tile, 1, &tiles, &st[i]);
  }
  int best = -1;
  for (int t = 0; t < 2; ++t) {
    int64_t tiles[3];
    for (int i = 0; i < 3; ++i) tiles[i] = dense_tiles(t, M[i], N[i]);
    const double us = tiles_us(t, 3, tiles, st);
    if (us < least) best = t, least = us;
  }
  return best;
}

void launch_grads(int tile, const DenseArgs &dx, const DenseArgs &dwgu, const DenseArgs &dwd,
                  hipStream_t s) {
  GradArgs a{dx, dwgu, dwd, {0, 1, 2}, {}};
  a.dx.splits = a.dwgu.splits = a.dwd.splits = 1;
  if (dx.K * dx.segs < dwd.K) std::rotate(a.order, a.order + 1, a.order + 3);
  const int64_t tiles[3] = {dense_tiles(tile, dx.M, dx.N), dense_tiles(tile, dwgu.M, 2 * dwgu.N),
                            dense_tiles(tile, dwd.M, dwd.N)};
  int64_t all = 0;
  for (int i = 0; i < 3; ++i) {
    a.tiles[i] = (int)tiles[a.order[i]];
    all += a.tiles[i];
  }
  const unsigned at = (unsigned)((all + 7) / 8 * 8);
  if (tile == 0) hipLaunchKernelGGL((k_dense_grads<128, 2, 4>), dim3(at), dim3(512), 0, s, a);
  else hipLaunchKernelGGL((k_dense_grads<64, 2, 2>), dim3(at), dim3(256), 0, s, a);
}

// a tile's offsets from its base stay below 2^31 bytes
constexpr int64_t kMaxStride = 1 << 21;

const char *bad_desc(const cep_gated_ffn_desc *d) {
  if (!d) return "desc is NULL";
  if (d->rows < 0 || d->rows > kMaxOpRows) return "rows must be in 0..2^21";
  for (int w : {d->d_model, d->d_ff})
    if (w < 8 || w > kMaxDim || w % 8) return "d_model and d_ff must be multiples of 8, up to 32768";
  for (int64_t ld : {d->ld_x, d->ld_y, d->ld_dx})
    if (ld && (ld < d->d_model || ld % 8 || ld > kMaxStride))
      return "row strides must be multiples of 8, at least d_model, at most 2^21";
  return nullptr;
}

// bf16 terms of h in the forward pass.  Up to 64 rows a call is bound by its
// weights, and h goes to the down projection as hi + lo (16 bits of mantissa), as
// two segments of K over the same weights, so that of y only its own rounding is
// left (relative RMS error 1.7e-3, 2.4e-3 with one term).  us with two and one: 33
// rows of 4096 x 2048 24.2, 22.8; 61 of 7168 x 2048 36.1, 32.9; 54 of 4096 x 264
// 19.9, 17.5.  Larger calls round h once: bound by matrix instructions, they would
// pay a third more of them.
constexpr int kTwoTermRows = 64;
int hidden_terms(int rows) { return rows <= kTwoTermRows ? 2 : 1; }

// [dg | du] and h of the backward pass, the terms of h of the forward one
size_t hidden_bytes(const cep_gated_ffn_desc *d, int backward) {
  return align_up((size_t)d->rows * d->d_ff * (backward ? 6 : 2 * hidden_terms(d->rows)), 256);
}

}  // namespace
}  // namespace cep

using namespace cep;

CEP_API size_t cep_gated_ffn_workspace(const cep_gated_ffn_desc *d, int backward) {
  if (bad_desc(d)) return 0;
  const int T = d->rows, D = d->d_model, I = d->d_ff;
  // forward: h, or the row blocks' scratch; backward: [dg | du] and h; then the
  // K shares of the products
  const RowsPlan p = rows_plan(T, D, I);
  size_t part = 0;
  if (backward)
    part = std::max({part_bytes(T, I, D, false), part_bytes(T, D, 2 * I, false),
                     part_bytes(D, I, T, true), part_bytes(I, D, T, false)});
  if (!p.use)
    part = std::max({part, part_bytes(T, I, D, true),
                     part_bytes(T, D, I * hidden_terms(T), false)});
  const size_t rows = p.use ? rows_workspace(p, T, D, I) : 0;
  return std::max(std::max<size_t>(hidden_bytes(d, backward) + part, rows), (size_t)256);
}

CEP_API int cep_gated_ffn(const cep_gated_ffn_desc *d, const void *x, const void *w_gate,
                          const void *w_up, const void *w_down, void *y, float *preact,
                          void *workspace, size_t workspace_bytes, hipStream_t s) {
  const char *fn = "cep_gated_ffn";
  if (const char *why = bad_desc(d)) return refuse(CEP_EINVAL, "%s: %s", fn, why);
  if (d->rows == 0) return CEP_OK;
  if (!x || !w_gate || !w_up || !w_down || !y) return refuse(CEP_EINVAL, "%s: NULL array", fn);
  for (const void *p : {x, w_gate, w_up, w_down, (const void *)y, (const void *)preact,
                        (const void *)workspace})
    if (!aligned(p, 16)) return refuse(CEP_EINVAL, "%s: pointers must be 16-byte aligned", fn);
  if (!workspace || workspace_bytes < cep_gated_ffn_workspace(d, 0))
    return refuse(workspace ? CEP_ENOMEM : CEP_EINVAL, "%s: needs a workspace of %zu bytes", fn,
                  cep_gated_ffn_workspace(d, 0));
  const int T = d->rows, D = d->d_model, I = d->d_ff;
  if (const RowsPlan p = rows_plan(T, D, I); p.use) {
    launch_rows_ffn(p, T, D, I, (const __bf16 *)x, d->ld_x ? d->ld_x : D, (const __bf16 *)w_gate,
                    (const __bf16 *)w_up, (const __bf16 *)w_down, (__bf16 *)y,
                    d->ld_y ? d->ld_y : D, preact, (uint8_t *)workspace, s);
    return launched(fn);
  }
  DenseArgs a{};
  a.A = (const __bf16 *)x;
  a.B0 = (const __bf16 *)w_gate;
  a.B1 = (const __bf16 *)w_up;
  a.lda = d->ld_x ? d->ld_x : D;
  a.ldb = I;
  a.M = T, a.N = I, a.K = D, a.segs = 1;
  const int terms = hidden_terms(T);
  a.out0 = (__bf16 *)workspace;
  if (terms == 2) a.out1 = a.out0 + I;
  a.ldo = terms * I;
  a.pre = preact;
  float *part = (float *)((uint8_t *)workspace + hidden_bytes(d, 0));
  launch_dense<true, false, kSwiGlu>(a, part, s);
  DenseArgs b{};
  b.A = (const __bf16 *)workspace;
  b.B0 = b.B1 = (const __bf16 *)w_down;
  b.lda = terms * I, b.ldb = D;
  b.M = T, b.N = D, b.K = I, b.segs = terms;
  b.out0 = (__bf16 *)y;
  b.ldo = d->ld_y ? d->ld_y : D;
  launch_dense<true, false, kStore>(b, part, s);
  return launched(fn);
}

CEP_API int cep_gated_ffn_backward(const cep_gated_ffn_desc *d, const void *dy, const void *x,
                                   const void *w_gate, const void *w_up, const void *w_down,
                                   const float *preact, void *dx, void *dw_gate, void *dw_up,
                                   void *dw_down, void *workspace, size_t workspace_bytes,
                                   hipStream_t s) {
  const char *fn = "cep_gated_ffn_backward";
  if (const char *why = bad_desc(d)) return refuse(CEP_EINVAL, "%s: %s", fn, why);
  if (!dw_gate || !dw_up || !dw_down ||
      (d->rows && (!dy || !x || !w_gate || !w_up || !w_down || !preact || !dx)))
    return refuse(CEP_EINVAL, "%s: NULL array", fn);
  for (const void *p : {dy, x, w_gate, w_up, w_down, (const void *)preact, (const void *)dx,
                        (const void *)dw_gate, (const void *)dw_up, (const void *)dw_down,
                        (const void *)workspace})
    if (!aligned(p, 16)) return refuse(CEP_EINVAL, "%s: pointers must be 16-byte aligned", fn);
  if (!workspace || workspace_bytes < cep_gated_ffn_workspace(d, 1))
    return refuse(workspace ? CEP_ENOMEM : CEP_EINVAL, "%s: needs a workspace of %zu bytes", fn,
                  cep_gated_ffn_workspace(d, 1));
  const int T = d->rows, D = d->d_model, I = d->d_ff;
  const int64_t ld_x = d->ld_x ? d->ld_x : D, ld_y = d->ld_y ? d->ld_y : D;
  __bf16 *dgu = (__bf16 *)workspace, *h = dgu + (size_t)T * 2 * I;
  float *part = (float *)((uint8_t *)workspace + hidden_bytes(d, 1));
  DenseArgs b{};  // dx
  if (T) {
    DenseArgs a{};  // dh, and from it dg, du and h
    a.A = (const __bf16 *)dy;
    a.B0 = (const __bf16 *)w_down;
    a.lda = ld_y, a.ldb = D;
    a.M = T, a.N = I, a.K = D, a.segs = 1;
    a.out0 = dgu, a.out1 = h;
    a.pre = const_cast<float *>(preact);
    launch_dense<true, true, kGrad>(a, part, s);
    b.A = dgu;
    b.B0 = (const __bf16 *)w_gate;
    b.B1 = (const __bf16 *)w_up;
    b.lda = 2 * I, b.ldb = I;
    b.M = T, b.N = D, b.K = I, b.segs = 2;
    b.out0 = (__bf16 *)dx;
    b.ldo = d->ld_dx ? d->ld_dx : D;
  }
  DenseArgs c{};  // dWg, dWu
  c.A = (const __bf16 *)x;
  c.B0 = dgu;
  c.B1 = dgu + I;
  c.lda = ld_x, c.ldb = 2 * I;
  c.M = D, c.N = I, c.K = T, c.segs = 1;
  c.out0 = (__bf16 *)dw_gate, c.out1 = (__bf16 *)dw_up;
  c.ldo = I;
  DenseArgs e{};  // dWd
  e.A = h;
  e.B0 = (const __bf16 *)dy;
  e.lda = I, e.ldb = ld_y;
  e.M = I, e.N = D, e.K = T, e.segs = 1;
  e.out0 = (__bf16 *)dw_down;
  e.ldo = D;
  const int tile = T ? grads_tile(T, D, I) : -1;
  if (tile >= 0) {
    launch_grads(tile, b, c, e, s);
  } else {
    if (T) launch_dense<true, true, kStore>(b, part, s);
    launch_dense<false, false, kStore2>(c, part, s);
    launch_dense<false, false, kStore>(e, part, s);
  }
  return launched(fn);
}
