// Matrix product with bias, activation, factor and residual in its epilogue, of one
// weight or of one per group of rows, and its gradient, in bf16 with float32
// accumulation, for gfx950.
//
//   z = x W + b, y = act(z) m + r
//   dz = dy m act'(z), dm = dy act(z), db = sum of dz, dx = dz W^T + a, dW = x^T dz
//
// Few rows a group stream the weights (rows_tile.h), more run the tiled product
// (dense_tile.h); the tiles of grouped rows are found on the device from the
// groups' offsets, the grid covers their most.  Bound by HBM with few rows (24 rows on
// eight weights of 4096 x 2048 25 us, 5.4 TB/s), else by the matrix instructions (8192 x
// 2048 x 7168 with bias and GELU 179 us among others, 1.34 PFLOP/s, 186 in a trace) and,
// where the epilogue reads a factor or keeps z, by its bytes (eight groups of 8192 x 2048
// x 4096 with both 166 us).
#include "dense_tile.h"
#include "rows_tile.h"

namespace cep {
namespace {

constexpr int kMaxGroups = 1024;

struct Groups {
  const int32_t *offsets;  // [n + 1]
  int n;                   // 0: one weight
  int rows;
};

// Rows [lo, lo + n) of group g, inside the arrays whatever the offsets hold.
struct Span {
  int lo, n;
};
__device__ inline Span span_of(const Groups &gr, int g) {
  const int lo = min(max(gr.offsets[g], 0), gr.rows);
  return {lo, min(max(gr.offsets[g + 1], lo), gr.rows) - lo};
}

// Tiles of TILE rows of the groups g0 + lane and those before it from g0 on.
template <int TILE>
__device__ inline int tiles_upto(const Groups &gr, int g0) {
  const int lane = threadIdx.x & 63;
  int v = g0 + lane < gr.n ? (span_of(gr, g0 + lane).n + TILE - 1) / TILE : 0;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  return v;
}
template <int TILE>
__device__ inline int tiles_of(const Groups &gr) {
  if (gr.n == 0) return (gr.rows + TILE - 1) / TILE;
  int all = 0;
  for (int g0 = 0; g0 < gr.n; g0 += 64)
    all += __builtin_amdgcn_readlane(tiles_upto<TILE>(gr, g0), 63);
  return all;
}
// Tile mt of them: its group, that group's rows, and the row of it where it starts.
struct RowTile {
  int g, m0;
  Span rows;
};
template <int TILE>
__device__ inline RowTile tile_at(const Groups &gr, int mt) {
  if (gr.n == 0) return {0, mt * TILE, {0, gr.rows}};
  for (int g0 = 0;; g0 += 64) {
    const int upto = tiles_upto<TILE>(gr, g0), all = __builtin_amdgcn_readlane(upto, 63);
    if (mt < all) {
      const int i = (int)__popcll(__ballot(upto <= mt));
      const int first = i ? __builtin_amdgcn_readlane(upto, i - 1) : 0;
      const Span s = span_of(gr, g0 + i);
      return {__builtin_amdgcn_readfirstlane(g0 + i),
              __builtin_amdgcn_readfirstlane((mt - first) * TILE),
              {__builtin_amdgcn_readfirstlane(s.lo), __builtin_amdgcn_readfirstlane(s.n)}};
    }
    mt -= all;
  }
}
// The group of a row, gr.n: none (the first whose end is behind it).
__device__ inline int group_of(const Groups &gr, int row) {
  const int lane = threadIdx.x & 63;
  int g = 0;
  for (int g0 = 0; g0 < gr.n; g0 += 64) {
    const bool past = g0 + lane < gr.n && gr.offsets[g0 + lane + 1] <= row;
    const int n = (int)__popcll(__ballot(past));
    g += n;
    if (n < 64) break;
  }
  return g;
}

// ---- epilogue

// Phi(z), the normal distribution, and *density, its slope.  Phi(-x) = exp(-x^2 / 2) t
// P(t) for x >= 0 with t = 1 / (1 + 0.31 x): P, of degree 7, fits erfcx(x / sqrt 2) / (2
// t) within 1.7e-7 of its value for x up to 14, where float32 has no smaller result
// (weighted least squares, the weights raised where the error is largest, one coefficient
// after the other rounded to float32 and the rest fitted anew).  2^(x^2 c) takes the
// rounding errors of x^2, of c = -log2(e) / 2 and of their product back as a factor 1 + r
// ln(2): without, they are 7.5e-6 of the value at x = 13 (8192 x 2048 x 7168 with GELU 168
// us, 170 with).  As evaluated, Phi and the density are within 2^-20 of their values for x
// up to 12.9, where Phi(-x) becomes subnormal.  With the library's erfc the gradient of
// 4095 x 2048 GELUs took 24 us, bound by its instructions.
__device__ inline float normal_cdf(float z, float *density = nullptr) {
  constexpr float kC = -0.721347511f, kCRest = -9.62981506e-9f;
  const float x = fabsf(z), t = __builtin_amdgcn_rcpf(fmaf(0.31f, x, 1.0f));
  const float q = fminf(x, 16.0f);  // past which e is 0 (a square without end has no remainder)
  const float s = q * q, v = s * kC;
  const float r = fmaf(fmaf(q, q, -s), kC, fmaf(s, kCRest, fmaf(s, kC, -v)));
  const float e = __builtin_amdgcn_exp2f(v) * fmaf(r, 0.693147182f, 1.0f);
  float p = fmaf(t, 0.035841763f, -0.141604379f);
  p = fmaf(t, p, 0.155067414f);
  p = fmaf(t, p, -0.0149032548f);
  p = fmaf(t, p, 0.110110231f);
  p = fmaf(t, p, 0.107771069f);
  p = fmaf(t, p, 0.124060325f);
  p = fmaf(t, p, 0.123656914f);
  const float below = e * t * p;
  if (density) *density = 0.398942280f * e;
  return z > 0.f ? 1.0f - below : below;
}
// The two operands of the tangent's logistic form: z (1 + tanh(u)) / 2 = z sigma(2 u),
// where z beyond 30 in magnitude changes nothing any more but could overflow.
__device__ inline float tanh_arg(float z, float *slope) {
  constexpr float kA = 1.59576912f, kB = 0.044715f;  // 2 sqrt(2 / pi)
  const float c = z != z ? z : fminf(fmaxf(z, -30.0f), 30.0f), q = c * c;
  if (slope) *slope = kA * fmaf(3.0f * kB, q, 1.0f);
  return kA * c * fmaf(kB, q, 1.0f);
}
template <int ACT>
__device__ inline float act_of(float z) {
  if (ACT == CEP_RELU) return z > 0.f ? z : z != z ? z : 0.f;
  if (ACT == CEP_SILU) return z * sigma(z);
  if (ACT == CEP_GELU) return z * normal_cdf(z);
  if (ACT == CEP_GELU_TANH) return z * sigma(tanh_arg(z, nullptr));
  return z;
}
// act(z), and its slope
template <int ACT>
__device__ inline float slope_of(float z, float *value) {
  if (ACT == CEP_SILU) {
    const float s = sigma(z);
    *value = z * s;
    return s * (1.0f + z * (1.0f - s));
  }
  if (ACT == CEP_GELU) {
    float density;
    const float phi = normal_cdf(z, &density);
    *value = z * phi;
    return fmaf(z, density, phi);
  }
  if (ACT == CEP_GELU_TANH) {
    float slope;
    const float s = sigma(tanh_arg(z, &slope));
    *value = z * s;
    const float c = fminf(fmaxf(z, -30.0f), 30.0f);  // (s is NaN where z is)
    return fmaf(c * s * (1.0f - s), slope, s);
  }
  *value = act_of<ACT>(z);
  return ACT == CEP_RELU ? (z > 0.f ? 1.0f : z != z ? z : 0.f) : 1.0f;
}
// f(std::integral_constant) of an activation
template <class F>
__device__ inline void with_act(int act, F f) {
  switch (act) {
    case CEP_RELU: return f(std::integral_constant<int, CEP_RELU>{});
    case CEP_SILU: return f(std::integral_constant<int, CEP_SILU>{});
    case CEP_GELU: return f(std::integral_constant<int, CEP_GELU>{});
    case CEP_GELU_TANH: return f(std::integral_constant<int, CEP_GELU_TANH>{});
    default: return f(std::integral_constant<int, CEP_IDENTITY>{});
  }
}

struct Finish {
  const float *bias;   // [groups][N]
  const __bf16 *mul;
  const void *res;
  void *y;
  float *pre;          // [rows][N]
  int64_t ld_mul, ld_res, ld_y;
  int N, act, res_dtype, y_dtype;
};

__device__ inline f32x4 from_bf16(uint32_t a, uint32_t b) {
  return f32x4{__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u),
               __uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u)};
}
__device__ inline f32x4 load4(const void *p, int dtype, int64_t at) {
  if (dtype == CEP_F32) return *(const f32x4 *)((const float *)p + at);
  const uint2 u = *(const uint2 *)((const __bf16 *)p + at);
  return from_bf16(u.x, u.y);
}
__device__ inline void store4(void *p, int dtype, int64_t at, const f32x4 &v) {
  if (dtype == CEP_F32) *(f32x4 *)((float *)p + at) = v;
  else store_bf16((__bf16 *)p + at, v);
}

// Four columns from n of row m, of group g, from their sums.
template <int ACT>
__device__ inline void finish(const Finish &f, int64_t m, int n, int g, f32x4 z) {
  if (f.bias) z += *(const f32x4 *)(f.bias + (int64_t)g * f.N + n);
  if (f.pre) *(f32x4 *)(f.pre + m * f.N + n) = z;
  f32x4 v;
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = act_of<ACT>(z[r]);
  if (f.mul) v *= load4(f.mul, CEP_BF16, m * f.ld_mul + n);
  if (f.res) v += load4(f.res, f.res_dtype, m * f.ld_res + n);
  store4(f.y, f.y_dtype, m * f.ld_y + n, v);
}

// The same for eight columns, in steps: what a column needs, what a row's columns need.
struct Column {
  f32x4 bias[2];
};
__device__ inline Column column_of(const Finish &f, int n, int g) {
  Column c{};
  if (f.bias)
#pragma unroll
    for (int h = 0; h < 2; ++h) c.bias[h] = *(const f32x4 *)(f.bias + (int64_t)g * f.N + n + 4 * h);
  return c;
}
struct Loaded {
  Vec16 mul, res[2];
};
__device__ inline Loaded load_eight(const Finish &f, int64_t m, int n) {
  Loaded in;
  if (f.mul) in.mul = *(const Vec16 *)(f.mul + m * f.ld_mul + n);
  if (f.res) {
    const char *p = (const char *)f.res + (m * f.ld_res + n) * (f.res_dtype == CEP_F32 ? 4 : 2);
    in.res[0] = *(const Vec16 *)p;
    if (f.res_dtype == CEP_F32) in.res[1] = *(const Vec16 *)(p + 16);
  }
  return in;
}
__device__ inline f32x4 half_of(const Vec16 &v, int h) {  // four of eight bf16 values
  return from_bf16(v[2 * h], v[2 * h + 1]);
}
template <int ACT>
__device__ inline void finish_eight(const Finish &f, int64_t m, int n, const f32x4 &lo,
                                    const f32x4 &hi, const Loaded &in, const Column &c) {
  f32x4 v[2] = {lo, hi};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (f.bias) v[h] += c.bias[h];
    if (f.pre) *(f32x4 *)(f.pre + m * f.N + n + 4 * h) = v[h];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[h][r] = act_of<ACT>(v[h][r]);
    if (f.mul) v[h] *= half_of(in.mul, h);
    if (f.res) v[h] += f.res_dtype == CEP_F32 ? __builtin_bit_cast(f32x4, in.res[h]) : half_of(in.res[0], h);
  }
  if (f.y_dtype == CEP_F32) {
    *(f32x4 *)((float *)f.y + m * f.ld_y + n) = v[0];
    *(f32x4 *)((float *)f.y + m * f.ld_y + n + 4) = v[1];
  } else {
    *(Vec16 *)((__bf16 *)f.y + m * f.ld_y + n) =
        Vec16{bf16_pair(v[0][0], v[0][1]), bf16_pair(v[0][2], v[0][3]), bf16_pair(v[1][0], v[1][1]),
              bf16_pair(v[1][2], v[1][3])};
  }
}

// Where a tile's sums go, row 0 of the tile's matrix being row `row0` of the
// epilogue's: the epilogue, or with K shares their lines of part.
template <int ACT>
struct TileOut {
  const Finish &f;
  int64_t row0;
  int g;
  float *part;  // of this share, null: one share
  __device__ inline Loaded load(int64_t m, int n) const {
    return part ? Loaded{} : load_eight(f, row0 + m, n);
  }
  __device__ inline Column column(int n) const { return part ? Column{} : column_of(f, n, g); }
  __device__ inline void store(int64_t m, int n, const f32x4 &lo, const f32x4 &hi, const Loaded &in,
                               const Column &c) const {
    if (part) {
      float *p = part + (row0 + m) * f.N + n;
      *(f32x4 *)p = lo;
      *(f32x4 *)(p + 4) = hi;
    } else {
      finish_eight<ACT>(f, row0 + m, n, lo, hi, in, c);
    }
  }
  __device__ inline void operator()(int64_t m, int n, const f32x4 &v, const f32x4 &) const {
    if (part) *(f32x4 *)(part + (row0 + m) * f.N + n) = v;
    else finish<ACT>(f, row0 + m, n, g, v);
  }
};

// ---- tiled product

struct LinearArgs : TileArgs {  // M: unused with groups
  Groups groups;
  int64_t w_stride;  // elements of a group's weight
  float *part;       // above one K share their sums: [splits][rows][N]
  Finish f;
};

// Tile L of an order of tiles: its rows, columns and share.
template <int SIZE, bool B_K, bool STAGED, int ACT>
struct TileWork {
  const LinearArgs &a;
  int n_tm, n_tn;
  uint8_t *lds;
  // PART of the tile's height and width from row m0 + SIZE / PART * row, ...
  template <int HALF, int WM, int WN>
  __device__ inline void run(int L, int row, int col) const {
    int mt, nt;
    tile_of<kGroupM>(L, n_tm * a.splits, n_tn, &mt, &nt);
    const int share = mt / n_tm;
    const RowTile tile = tile_at<SIZE>(a.groups, mt - share * n_tm);
    TileArgs t = a;
    t.A += tile.rows.lo * a.lda;
    t.B0 += tile.g * a.w_stride;
    t.M = tile.rows.n;
    const int m0 = tile.m0 + row * 2 * HALF, n0 = nt * SIZE + col * 2 * HALF;
    if (m0 >= t.M || n0 >= t.N) return;
    const TileOut<ACT> out{a.f, tile.rows.lo, tile.g,
                           a.splits > 1 ? a.part + (int64_t)share * a.groups.rows * a.N : nullptr};
    dense_tile<HALF, WM, WN, true, B_K, false, STAGED>(t, m0, n0, share, lds, out);
  }
};

// y (B_K false) or dx (true: N is d_in) in 128-wide tiles of whole groups' rows, two
// workgroups of eight waves a compute unit.  4095 x 2048 x 4096 with GELU and z kept 87 to
// 94 us from machine to machine, 0.73 to 0.79 PFLOP/s: one round, whose tiles all store at
// its end.  (us, eight and four
// waves: 777 x 6144 x 2560 with a residual 38.7, 39.7; 3000 x 1408 x 2048 in 16 groups
// 41.4, 43.9; 378 x 1896 x 976 in two shares 11.2, 12.7; one workgroup a unit 50 for the
// second)
template <bool B_K, bool STAGED, int ACT>
__global__ __launch_bounds__(512, 4) void k_linear_128(LinearArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[65536];
  const int x = blockIdx.x & 7, at = blockIdx.x >> 3;
  const TileWork<128, B_K, STAGED, ACT> work{a, tiles_of<128>(a.groups), (a.N + 127) / 128, lds};
  const int items = work.n_tm * a.splits * work.n_tn;
  if (at >= piece_of(items, x)) return;
  work.template run<64, 2, 4>(x * (items / 8) + min(x, items % 8) + at, 0, 0);
}

// ... in 256-wide ones, one a compute unit.  Where a few are left after the last full
// round, those are cut into quarters: up to two rounds of them (of 64 steps 38 us each)
// cost less than one of whole tiles (101 us).
constexpr int kUnits = 256;
__host__ __device__ inline int whole_tiles(int items) {
  const int full = items / kUnits * kUnits;
  return full && (items - full) * 4 <= 2 * kUnits ? full : items;
}
template <bool B_K, bool STAGED, int ACT>
__global__ __launch_bounds__(512, 2) void k_linear_256(LinearArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[131072];
  const TileWork<256, B_K, STAGED, ACT> work{a, tiles_of<256>(a.groups), (a.N + 255) / 256, lds};
  const int items = work.n_tm * a.splits * work.n_tn, whole = whole_tiles(items);
  const int x = blockIdx.x & 7, at = blockIdx.x >> 3;
  if (at < piece_of(whole, x)) {
    work.template run<128, 2, 4>(x * (whole / 8) + min(x, whole % 8) + at, 0, 0);
  } else if (whole < items) {  // `whole` is then a multiple of 8
    const int quarters = (items - whole) * 4, q = at - whole / 8;
    if (q >= piece_of(quarters, x)) return;
    const int i = x * (quarters / 8) + min(x, quarters % 8) + q;
    work.template run<64, 2, 4>(whole + i / 4, i & 1, i >> 1 & 1);
  }
}

// The shares' sums of a row, added in order, eight on the way at once, and what becomes
// of them.  A launch's start and a trip to memory: one row of 2048 3.0 us, 24 rows of
// groups 4.7.
constexpr int kFinishThreads = 128;
__global__ __launch_bounds__(kFinishThreads) void k_linear_finish(const float *part, int splits,
                                                                  Groups groups, Finish f) {
  const int64_t m = blockIdx.x;
  const int n = ((int)blockIdx.y * kFinishThreads + threadIdx.x) * 4;
  int g = 0;
  if (groups.n) {
    g = group_of(groups, (int)m);
    if (g == groups.n || m < span_of(groups, g).lo) return;  // no group's
  }
  if (n >= f.N) return;
  const float *p = part + m * f.N + n;
  const int64_t share = (int64_t)groups.rows * f.N;
  f32x4 v = {};
  for (int i0 = 0; i0 < splits; i0 += 8) {
    f32x4 w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = *(const f32x4 *)(p + min(i0 + i, splits - 1) * share);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 8; ++i) v += i0 + i < splits ? w[i] : f32x4{};
  }
  with_act(f.act, [&](auto act) { finish<decltype(act)::value>(f, m, n, g, v); });
}

struct WgradArgs : TileArgs {  // K: unused with groups
  Groups groups;
  float *part;  // above one K share (one weight): [splits][M][N]
  Finish f;     // of one weight's gradient
};

// The r-th largest group, the lower of equals first (up to 64 groups, past which they
// come in their own order): a launch's longest tiles go first.
constexpr int kOrderedGroups = 64;
__device__ inline int ranked_group(const Groups &gr, int r) {
  if (gr.n > kOrderedGroups) return r;
  const int lane = threadIdx.x & 63, n = lane < gr.n ? span_of(gr, lane).n : -1;
  int rank = 0;
  for (int h = 0; h < gr.n; ++h) {
    const int o = __builtin_amdgcn_readlane(n, h);
    rank += o > n || (o == n && h < lane);
  }
  return (int)__builtin_ctzll(__ballot(lane < gr.n && rank == r));
}

// A group's tiles are dealt to all XCDs: those of XCD x, and item `at` of its order,
// groups by size.  False: none.
struct WgradTile {
  int g, m0, n0, share;
};
template <int SIZE>
__device__ inline int wgrad_room(const WgradArgs &a) {  // of an XCD, a group
  return ((a.M + SIZE - 1) / SIZE * ((a.N + SIZE - 1) / SIZE) * a.splits + 7) / 8;
}
// (ordered only where tiles are long: of 128-wide ones, a few steps each, finding the
// order costs more than it gives, 16 groups of 3000 rows 77 us with it, 69 without)
template <int SIZE>
__device__ inline bool wgrad_item(const WgradArgs &a, int x, int at, WgradTile *t) {
  const int n_tm = (a.M + SIZE - 1) / SIZE, n_tn = (a.N + SIZE - 1) / SIZE;
  const int items = n_tm * a.splits * n_tn, room = wgrad_room<SIZE>(a);
  const int r = at / room, in = at - r * room;
  if (in >= piece_of(items, x)) return false;
  int mt, nt;
  tile_of<kGroupM>(x * (items / 8) + min(x, items % 8) + in, n_tm * a.splits, n_tn, &mt, &nt);
  t->share = mt / n_tm;
  t->m0 = (mt - t->share * n_tm) * SIZE;
  t->n0 = nt * SIZE;
  t->g = a.groups.n && SIZE == 256 ? __builtin_amdgcn_readfirstlane(ranked_group(a.groups, r)) : r;
  return true;
}
template <int HALF, int WM, int WN>
__device__ inline void wgrad_run(const WgradArgs &a, const WgradTile &w, uint8_t *lds) {
  TileArgs t = a;
  if (a.groups.n) {
    const Span s = span_of(a.groups, w.g);
    const int lo = __builtin_amdgcn_readfirstlane(s.lo);
    t.A += lo * a.lda;
    t.B0 += lo * a.ldb;
    t.K = __builtin_amdgcn_readfirstlane(s.n);
  }
  const TileOut<CEP_IDENTITY> out{a.f, (int64_t)w.g * a.M, 0,
                                  a.splits > 1 ? a.part + (int64_t)w.share * a.M * a.N : nullptr};
  dense_tile<HALF, WM, WN, false, false, false>(t, w.m0, w.n0, w.share, lds, out);
}

// dW of each group, its rows as K, both operands read across: 4096 x 2048 of 4095 rows in
// 128-wide tiles 72 us, 0.95 PFLOP/s; 976 x 1896 of 378 rows 9.1 (with four waves 12.1).
template <int HALF, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64, HALF == 64 ? 4 : 2) void k_linear_wgrad(WgradArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[HALF * 1024];
  WgradTile t;
  if (wgrad_item<2 * HALF>(a, blockIdx.x & 7, blockIdx.x >> 3, &t)) wgrad_run<HALF, WM, WN>(a, t, lds);
}

// dW of groups of few rows, in 128-wide tiles by 2 x 4 waves: a tile is mostly its start
// and its store, so that several share a compute unit (32 KB of LDS) instead of one
// running ahead of itself.  64 rows at a time, [64 rows][128 columns] of each operand,
// 16-byte chunk pair p of line k at p ^ f(k); lines past the group's rows are zeros.
// Measured: 32 groups of 34 rows of 4096 x 2048 147 us, 3.7 TB/s of stores
// (k_linear_wgrad 262); 16 of 128 rows 108 (175).  By 2 x 2 waves 154 and 110, those
// stored straight from the accumulators 177 and 124; four workgroups a unit spill.
__global__ __launch_bounds__(512, 6) void k_linear_wgrad_few(WgradArgs a) {
  constexpr int MF = 4, NF = 2;  // fragments of a wave
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2][16384];
  WgradTile w;
  if (!wgrad_item<128>(a, blockIdx.x & 7, blockIdx.x >> 3, &w)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l15 = lane & 15, g4 = lane >> 4, wm = wave & 1, wn = wave >> 1;
  int lo = 0, K = a.K;
  if (a.groups.n) {
    const Span s = span_of(a.groups, w.g);
    lo = __builtin_amdgcn_readfirstlane(s.lo);
    K = __builtin_amdgcn_readfirstlane(s.n);
  }
  auto f_of = [](int k) { return (k & 3) | ((k >> 3) & 1) << 2; };
  // a thread's 16 bytes of lines k0 + tid / 16, and every 16th from there
  const int chunk = tid & 15;
  const __bf16 *srcA = a.A + lo * a.lda + min(w.m0 + chunk * 8, a.M - 8);
  const __bf16 *srcB = a.B0 + lo * a.ldb + min(w.n0 + chunk * 8, a.N - 8);
  f32x4 acc[MF][NF] = {};
  for (int k0 = 0; k0 < K; k0 += 64) {
    uint4 v[2][2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int64_t k = k0 + e * 32 + (tid >> 4);
      v[0][e] = v[1][e] = make_uint4(0u, 0u, 0u, 0u);
      if (k < K) {
        v[0][e] = *(const uint4 *)(srcA + k * a.lda);
        v[1][e] = *(const uint4 *)(srcB + k * a.ldb);
      }
    }
    if (k0) __syncthreads();
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int k = e * 32 + (tid >> 4);
      const int to = k * 256 + (((chunk >> 1) ^ f_of(k)) << 5) + (chunk & 1) * 16;
      *(uint4 *)(lds[0] + to) = v[0][e];
      *(uint4 *)(lds[1] + to) = v[1][e];
    }
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int k = ks * 32 + g4 * 8 + (l15 >> 2);
      auto read = [&](const uint8_t *at, int row0, int i) {
        union { bf16x8 v; bf16x4 h[2]; } o;
#pragma unroll
        for (int h = 0; h < 2; ++h)
          o.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              (__attribute__((address_space(3))) bf16x4 *)(at + (k + h * 4) * 256 +
                                                            (((row0 >> 4) + i) ^ f_of(k)) * 32 +
                                                            (l15 & 3) * 8));
        return o.v;
      };
      bf16x8 fa[MF], fb[NF];
#pragma unroll
      for (int j = 0; j < NF; ++j) fb[j] = read(lds[1], wn * 32, j);
#pragma unroll
      for (int i = 0; i < MF; ++i) fa[i] = read(lds[0], wm * 64, i);
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
  }
  // a row fragment of both halves at a time through LDS, [32 rows][128] float32, 16-byte
  // chunk c of row r at c ^ (r % 16), so that whole cache lines are written
  auto at = [&](int i, int r, int c) {
    return (f32x4 *)(lds[i & 1] + r * 512 + ((c ^ (r & 15)) << 4));
  };
  __syncthreads();
#pragma unroll
  for (int i = 0; i < MF; ++i) {
#pragma unroll
    for (int j = 0; j < NF; ++j) *at(i, wm * 16 + l15, wn * 8 + j * 4 + g4) = acc[i][j];
    wait_lgkm0();
    asm volatile("s_barrier" ::: "memory");
    const int r = tid >> 4, n = w.n0 + chunk * 8;
    const int64_t m = w.m0 + (r >> 4) * 64 + i * 16 + (r & 15);
    if (m < a.M && n < a.N)
      finish_eight<CEP_IDENTITY>(a.f, (int64_t)w.g * a.M + m, n, *at(i, r, 2 * chunk),
                                 *at(i, r, 2 * chunk + 1), Loaded{}, Column{});
  }
}

// dW and dx in one launch, so that the tiles of one fill the compute units that the others'
// last round leaves: weights' gradients, as many groups' as have more rows than dx has
// columns to sum over, then dx, then the other weights'.  Of 256-wide tiles the groups go
// by size, so that the longest come first; of 128-wide ones in their own order, whichever
// are the large ones (wgrad_item).
template <int HALF, int WM, int WN, bool STAGED>
__global__ __launch_bounds__(WM * WN * 64, HALF == 64 ? 4 : 2) void k_linear_grads(LinearArgs dx, WgradArgs dw) {
  constexpr int SIZE = 2 * HALF;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[HALF * 1024];
  const int x = blockIdx.x & 7, room = wgrad_room<SIZE>(dw);
  int at = blockIdx.x >> 3, first = dw.K > dx.K;  // of one weight
  if (dw.groups.n > kOrderedGroups) {
    first = dw.K / dw.groups.n > dx.K ? dw.groups.n : 0;
  } else if (dw.groups.n) {
    const int lane = threadIdx.x & 63;
    first = (int)__popcll(__ballot(lane < dw.groups.n && span_of(dw.groups, min(lane, dw.groups.n - 1)).n > dx.K));
  }
  const TileWork<SIZE, true, STAGED, CEP_IDENTITY> work{dx, tiles_of<SIZE>(dx.groups),
                                                        (dx.N + SIZE - 1) / SIZE, lds};
  const int items = work.n_tm * work.n_tn, mine = piece_of(items, x);
  if (at >= first * room && at < first * room + mine) {
    work.template run<HALF, WM, WN>(x * (items / 8) + min(x, items % 8) + at - first * room, 0, 0);
    return;
  }
  if (at >= first * room) at -= mine;
  WgradTile t;
  if (at < room * max(dw.groups.n, 1) && wgrad_item<SIZE>(dw, x, at, &t))
    wgrad_run<HALF, WM, WN>(dw, t, lds);
}

// ---- few rows: the weights are streamed

struct LinearRowsArgs : RowsArgs {
  Groups groups;
  int64_t w_stride;
  float *part;
  Finish f;
};

// Few rows, MF * 16 of a group at a time, the weights read past them once.  Bound by HBM:
// one row of 7168 x 2048 7.9 us with its start and end, 24 rows of eight groups of 4096 x
// 2048 25 us, 5.4 TB/s.
template <int MF>
__global__ __launch_bounds__(256) void k_linear_rows(LinearRowsArgs a) {
  __shared__ RowsLds<MF, kRows> lds;
  const int cb = blockIdx.x % a.col_blocks, sp = blockIdx.x / a.col_blocks % a.splits;
  const int mt = blockIdx.x / (a.col_blocks * a.splits);
  if (mt >= tiles_of<MF * 16>(a.groups)) return;
  const RowTile tile = tile_at<MF * 16>(a.groups, mt);
  const int64_t row0 = tile.rows.lo + tile.m0;
  RowsArgs t = a;
  t.A[0] += row0 * a.lda;
  t.B0 += tile.g * a.w_stride;
  t.M = min(tile.rows.n - tile.m0, MF * 16);
  rows_tile<MF, kRows, false>(t, cb, sp, lds, [&](int row, int col, const f32x4 &v) {
    const int64_t m = row0 + row;
    if (a.splits == 1)
      with_act(a.f.act, [&](auto act) { finish<decltype(act)::value>(a.f, m, col, tile.g, v); });
    else *(f32x4 *)(a.part + ((int64_t)sp * a.groups.rows + m) * a.N + col) = v;
  });
}

// ---- the gradient of the epilogue

constexpr int kDzCols = 256;  // columns of a k_linear_dz block: 32 lanes of eight
// Its rows, eight at a time: one round of them where blocks are few (us, 8 and 32 rows:
// 109 x 1408 3.5, 6.2; 378 x 1896 4.7, 8.1; 1116 x 2048 6.6, 12.0), four elsewhere, which
// leaves fewer sums.
inline int dz_rows(int rows, int N) {
  return (int64_t)((rows + 31) / 32) * ((N + kDzCols - 1) / kDzCols) < 512 ? 8 : 32;
}

struct DzArgs {
  const void *dy;
  const float *pre;
  const __bf16 *mul;
  __bf16 *dz, *dmul;  // dz [rows][N]
  float *part;        // column sums of a block's rows of a group: [blocks + groups][N]
  int64_t ld_y, ld_mul;
  int N, y_dtype;
  Groups groups;
};

// dz and dm of a block's rows, and their sums over each group's rows there: those of
// group g go to line blockIdx.x + g of `part` (from one pair of block and group to the
// next, one of the two grows, so no line is written twice).  With one block the lines
// are db, and those of groups without rows get zeros.  dz is rounded to bf16, which the
// matrix instructions of dx and dW take beside bf16 weights and rows: their error against
// 64 bits is 2.34e-3 of their size, where their own rounding alone is 1.66e-3.  A second
// term of dz would take those instructions twice (dx and dW of 4095 x 4096 x 2048: 110 us
// of a step of 214).  Bound by HBM: 4095 x 2048 from bf16 with GELU and sums 16.6 us, 4.0
// TB/s; 8192 x 2048 with SiLU and a factor 40, 5.0.  (Eight rows of four columns a lane at
// once, in fewer waves: 23 and 56.)
template <int ACT, int ROWS>
__global__ __launch_bounds__(256) void k_linear_dz(DzArgs a) {
  __shared__ float sums[ROWS][kDzCols];
  __shared__ int group[ROWS];  // of a row
  const int tid = threadIdx.x, lane = tid & 31, rl = tid >> 5;
  const int n = (int)blockIdx.y * kDzCols + lane * 8;
  const int row0 = blockIdx.x * ROWS;
  const int end = min(row0 + ROWS, a.groups.rows);
  int from = row0, to = end;  // the rows of some group, inside the block's whatever the offsets hold
  if (a.groups.n) {
    from = min(max(a.groups.offsets[0], row0), end);
    to = min(max(a.groups.offsets[a.groups.n], from), end);
  }
  if (n < a.N) {
    for (int r = rl; r < ROWS; r += 8) {
      const int64_t m = row0 + r;
      float out[8] = {};
      if (m >= from && m < to) {
        float dy[8], z[8], f[8], dm[8];
        load8(a.dy, a.y_dtype, m * a.ld_y + n, 8, dy);
        if (a.pre) load8(a.pre, CEP_F32, m * a.N + n, 8, z);
        if (a.mul) load8(a.mul, CEP_BF16, m * a.ld_mul + n, 8, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float value = 0.f, slope = 1.0f;
          if (a.pre) slope = slope_of<ACT>(z[i], &value);
          out[i] = (a.mul ? dy[i] * f[i] : dy[i]) * slope;
          dm[i] = dy[i] * value;
        }
        if (a.dz) store8(a.dz, CEP_BF16, m * a.N + n, 8, out);
        if (a.dmul) store8(a.dmul, CEP_BF16, m * a.ld_mul + n, 8, dm);
      }
      if (a.part) {
        *(f32x4 *)&sums[r][lane * 8] = f32x4{out[0], out[1], out[2], out[3]};
        *(f32x4 *)&sums[r][lane * 8 + 4] = f32x4{out[4], out[5], out[6], out[7]};
      }
    }
  }
  if (!a.part) return;
  if (a.groups.n && tid < 64) {
    int mine = 0;  // of row row0 + tid: how many groups end up to it
    for (int g0 = 0; g0 < a.groups.n; g0 += 64) {
      const int stop = g0 + tid < a.groups.n ? a.groups.offsets[g0 + tid + 1] : INT32_MAX;
      for (int r = 0; r < ROWS; ++r) {
        const int n_ended = (int)__popcll(__ballot(stop <= row0 + r));
        if (tid == r) mine += n_ended;
      }
    }
    if (tid < ROWS) group[tid] = mine;
  }
  __syncthreads();
  const int c = (int)blockIdx.y * kDzCols + tid;  // a column a thread
  if (c >= a.N) return;
  float *line = a.part + (int64_t)blockIdx.x * a.N + c;
  if (a.groups.n == 0) {
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) sum += sums[r][tid];
    *line = sum;
    return;
  }
  const bool whole = gridDim.x == 1;
  int next = 0;  // the first line not written yet, of one block
  for (int r = from - row0; r < to - row0;) {
    const int g = group[r];
    if (g >= a.groups.n) break;
    float sum = 0.f;
    for (; r < to - row0 && group[r] == g; ++r) sum += sums[r][tid];
    if (whole)
      for (; next < g; ++next) line[(int64_t)next * a.N] = 0.f;
    line[(int64_t)g * a.N] = sum;
    next = g + 1;
  }
  if (whole)
    for (; next < a.groups.n; ++next) line[(int64_t)next * a.N] = 0.f;
}

// db of a group: its lines of `part`, added in order by 16 lanes of columns' fours.
__global__ __launch_bounds__(256) void k_linear_dbias(const float *part, int rows, int N,
                                                      Groups groups, float *db) {
  __shared__ f32x4 sums[16][16];
  const int lane = threadIdx.x & 15, sl = threadIdx.x >> 4, g = blockIdx.y;
  const int n = ((int)blockIdx.x * 16 + lane) * 4;
  const Span s = groups.n ? span_of(groups, g) : Span{0, groups.rows};
  f32x4 v = {};
  if (s.n && n < N) {
    const int last = (s.lo + s.n - 1) / rows;
#pragma unroll 4
    for (int c = s.lo / rows + sl; c <= last; c += 16)
      v += *(const f32x4 *)(part + (int64_t)(c + g) * N + n);
  }
  sums[sl][lane] = v;
  __syncthreads();
  if (sl || n >= N) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) v += sums[i][lane];
  *(f32x4 *)(db + (int64_t)g * N + n) = v;
}

// ---- host

constexpr int64_t kMaxStride = 1 << 21;  // a tile's offsets stay below 2^31 bytes

const char *bad_desc(const cep_linear_desc *d) {
  if (!d) return "desc is NULL";
  if (d->rows < 0 || d->rows > kMaxOpRows) return "rows must be in 0..2^21";
  for (int w : {d->d_in, d->d_out})
    if (w < 8 || w > kMaxDim || w % 8) return "d_in and d_out must be multiples of 8, up to 32768";
  if (d->n_groups < 0 || d->n_groups > kMaxGroups) return "n_groups must be in 0..1024";
  if (d->act < CEP_IDENTITY || d->act > CEP_GELU_TANH) return "unknown act";
  for (int t : {d->y_dtype, d->res_dtype, d->dx_dtype, d->dw_dtype})
    if (!is_float_dtype(t)) return "types must be CEP_F32 or CEP_BF16";
  for (int64_t ld : {d->ld_x, d->ld_dx})
    if (ld && (ld < d->d_in || ld % 8 || ld > kMaxStride))
      return "row strides must be multiples of 8, at least a row, at most 2^21";
  for (int64_t ld : {d->ld_y, d->ld_mul, d->ld_res})
    if (ld && (ld < d->d_out || ld % 8 || ld > kMaxStride))
      return "row strides must be multiples of 8, at least a row, at most 2^21";
  return nullptr;
}

// How a product of `rows` rows (in groups) runs.
struct Plan {
  bool stream;  // in row blocks of 16 or 32 (MF fragments)
  int mf;
  int tile, splits;
  double us;  // estimated
};

// Rows of one weight, and of a group on average, up to which the weights are streamed:
// the tiled product reads each weight once for all its rows, with fewer loads on the way
// at a time (4096 x 2048, us streamed and tiled: 16 rows 6.4, 8.3; 32 7.5, 8.6; 48 11.3,
// 9.2; of eight groups 3 rows each 24.9, 29.4; 8 30.4, 34.8; 12 40.2, 35.2; 32 42, 34).
// The host knows the groups' mean alone, and these are of even groups.  With all rows in
// one of many groups the streamed form reads that weight for every 16 of them: 10 rows a
// group on average in one of 32 groups 35 us, tiled 33; in one of 256 208 and 60.
constexpr int kStreamRows = 32, kStreamGroup = 10;

Plan plan_of(int rows, int N, int K, int groups, bool may_stream) {
  Plan p{};
  const int g = std::max(groups, 1);
  if (may_stream && rows <= (int64_t)(groups ? kStreamGroup : kStreamRows) * g) {
    p.stream = true;
    p.mf = rows <= 16 * g ? 1 : 2;  // (16 rows 6.4, 32 in one block 7.5)
    // one workgroup a compute unit (a ring takes most of its LDS), at least a unit
    // for each wave
    const int cols = (N + kCols - 1) / kCols, blocks = cols * std::min(g, std::max(rows, 1));
    p.splits = std::max(1, std::min(256 / blocks, K / kUnit / 4));
    return p;
  }
  int64_t tiles[2];
  for (int t = 0; t < 2; ++t) {
    // a group's last tile is half full on average
    const int64_t n_tm = groups ? rows / kTile[t] + (groups + 1) / 2 : (rows + kTile[t] - 1) / kTile[t];
    tiles[t] = std::max<int64_t>(n_tm, 1) * ((N + kTile[t] - 1) / kTile[t]);
  }
  const DensePlan d = plan_tiles(tiles, K / 64, (double)rows * N, 16);
  p.tile = d.tile, p.splits = d.splits, p.us = d.us;
  // 256-wide tiles with quarters, which that estimate does not know
  const int whole = whole_tiles((int)tiles[0]), quarters = ((int)tiles[0] - whole) * 4;
  const double us = (double)((whole + kUnits - 1) / kUnits) * (12 + 1.4 * (K / 64)) +
                    (double)((quarters + kUnits - 1) / kUnits) * (3 + 0.55 * (K / 64));
  if (us < d.us) p.tile = 0, p.splits = 1, p.us = us;
  // Few 128-wide tiles of one weight share K in shorter pieces than that estimate takes
  // (us, shared and not: 378 x 1896 x 976 with a factor and z kept 17.3, 21.0; 648 x 632 x
  // 1024 13.6, 13.9; 64 x 1024 x 1024 9.3, 11.3; of eight groups 700 x 1024 x 1024 16.4,
  // 14.4)
  if (!groups && tiles[1] <= 128) {
    double least = 7 + 0.65 * (K / 64.0);
    for (int s = 2; s <= 16 && tiles[1] * s <= 256 && K / 64 / s >= 4; ++s) {
      const double split = 9 + 0.6 * (K / 64.0 / s) + (double)s * rows * N * 4 / 9e6;
      if (split < least) least = split, p.tile = 1, p.splits = s, p.us = split;
    }
  }
  return p;
}

// dW: 256- or 128-wide tiles (0, 1), or k_linear_wgrad_few (2), by estimates of the time
// for K in steps of 64 (us; measured, 4096 x 2048 a group):
//   256-wide: 12 + 1.4 a step, a round of 256; groups of unlike sizes a tenth more
//   128-wide, more than a round: 6 + 1.3 a step, a round of 512 (32 groups of 34 rows 262,
//     16 of 128 rows 175)
//   few: 5 + 2 a step, a round of 768, three a compute unit (the same two 147 and 108, 16
//     of 256 rows 143, eight of 512 109, eight of 1024 198); two of them 1.5 a step, one 1
constexpr int kFewTile = 2;
Plan wgrad_plan(const cep_linear_desc *d) {
  const int g = std::max(d->n_groups, 1);
  const int64_t tiles[2] = {g * dense_tiles(0, d->d_in, d->d_out),
                            g * dense_tiles(1, d->d_in, d->d_out)};
  const double steps = std::max(1.0, (double)d->rows / g / 64);
  DensePlan w = plan_tiles(tiles, d->rows / g / 64, (double)d->d_in * d->d_out, d->n_groups ? 1 : 16);
  if (w.tile == 1 && tiles[1] > 512) w.us = (double)tiles[1] / 512 * (6 + 1.3 * steps);
  Plan p{};
  p.tile = w.tile, p.splits = w.splits, p.us = w.us;
  const double wide = (double)((tiles[0] + 255) / 256) * (12 + 1.4 * steps) * (d->n_groups ? 1.1 : 1.0);
  if (wide < p.us) p.tile = 0, p.splits = 1, p.us = wide;
  const double few = tiles[1] > 768 ? (double)tiles[1] / 768 * (5 + 2 * steps)
                                    : 5 + steps * (0.5 + 0.5 * (double)((tiles[1] + 255) / 256));
  if (few < p.us) p.tile = kFewTile, p.splits = 1, p.us = few;
  return p;
}

// Tiles that the groups' rows are in, on average (a group's last is half full).
int64_t row_tiles(const cep_linear_desc *d, int size) {
  if (!d->n_groups) return (d->rows + size - 1) / size;
  return std::max<int64_t>(d->rows / size + (d->n_groups + 1) / 2, 1);
}

// The tile with which dx and dW run in one launch, -1: a launch each.
int grads_tile(const cep_linear_desc *d) {
  if (d->rows == 0) return -1;
  const int g = std::max(d->n_groups, 1);
  // Launches of their own for groups take longer than estimated, with the tiles of unlike
  // sizes that they wait for (us, one launch and two: 8192 rows of 4096 x 2048 in eight
  // groups 284, 288, and with some popular 292, 306; 2048 x 4096 in four 246, 260; one
  // weight, 4095 x 4096 x 2048, 125, 140)
  const Plan own = wgrad_plan(d);
  double least = plan_of(d->rows, d->d_in, d->d_out, d->n_groups, false).us +
                 own.us * (d->n_groups && own.tile == 0 ? 1.2 : 1.0);
  int best = -1;
  auto steps = [](int K) { return 2 + K / 64 + (K % 64 ? 3.0 : 0.0); };
  const double st[2] = {steps(d->d_out), steps(d->rows / g)};
  for (int t = 0; t < 2; ++t) {
    const int64_t tiles[2] = {row_tiles(d, kTile[t]) * ((d->d_in + kTile[t] - 1) / kTile[t]),
                              g * dense_tiles(t, d->d_in, d->d_out)};
    double us = tiles_us(t, 2, tiles, st);
    if (t == 1 && tiles[0] + tiles[1] > 512)
      us = std::max(us, ((double)tiles[0] * (6 + 1.3 * st[0]) + (double)tiles[1] * (6 + 1.3 * st[1])) / 512);
    if (us < least) best = t, least = us;
  }
  return best;
}

size_t part_bytes(const Plan &p, int rows, int N) {
  return p.splits > 1 ? (size_t)p.splits * rows * N * 4 : 0;
}

int dz_chunks(const cep_linear_desc *d) {
  const int rows = dz_rows(d->rows, d->d_out);
  return (d->rows + rows - 1) / rows;
}

// Scratch of the backward pass: dz, the parts of db, the K shares of a product.
struct Space {
  size_t bias, part, bytes;
};
Space space_of(const cep_linear_desc *d, int backward) {
  Space s{};
  size_t most = part_bytes(plan_of(d->rows, d->d_out, d->d_in, d->n_groups, true), d->rows, d->d_out);
  if (backward) {
    s.bias = align_up((size_t)d->rows * d->d_out * 2, 256);
    s.part = s.bias + align_up((size_t)(dz_chunks(d) + d->n_groups) * d->d_out * 4, 256);
    most = std::max({most,
                     s.part + part_bytes(plan_of(d->rows, d->d_in, d->d_out, d->n_groups, false),
                                         d->rows, d->d_in),
                     s.part + part_bytes(wgrad_plan(d), d->d_in, d->d_out)});
  }
  s.bytes = std::max<size_t>(most, 256);
  return s;
}

void launch_finish(const float *part, int splits, const Groups &g, const Finish &f, int rows,
                   hipStream_t s) {
  hipLaunchKernelGGL(k_linear_finish, dim3(rows, (f.N / 4 + kFinishThreads - 1) / kFinishThreads),
                     dim3(kFinishThreads), 0, s, part, splits, g, f);
}

// The epilogue is staged, but for a dx that nothing is added to (us, staged and not: 777 x
// 6144 x 2560 with bias and residual 42, 47; 8192 x 2048 x 4096 in eight groups with a
// factor 212, 229; dx of 4095 x 4096 x 2048 68, 64).  Plain stores of y gain on neither
// side (4095 x 4096 x 2048 55.8, 53.8; 8192 x 2048 x 4096 in eight groups 128, 127; 8192 x
// 2048 x 7168 161, 159; 777 x 6144 x 2560 35.5, 36.7; 3000 x 1408 x 2048 in 16 30.3, 31.1).
template <int TILE, bool B_K, bool STAGED, int ACT>
void launch_kind(const LinearArgs &a, int64_t items, hipStream_t s) {
  // with groups fewer tiles may be live, and then quarters
  const int64_t blocks = TILE == 0 && items > kUnits ? items + 2 * kUnits : items;
  const dim3 grid((unsigned)((blocks + 7) / 8 * 8));
  if constexpr (TILE == 0) hipLaunchKernelGGL((k_linear_256<B_K, STAGED, ACT>), grid, dim3(512), 0, s, a);
  else hipLaunchKernelGGL((k_linear_128<B_K, STAGED, ACT>), grid, dim3(512), 0, s, a);
}
template <int TILE, bool B_K>
void launch_tiles(const LinearArgs &a, int64_t items, hipStream_t s) {
  auto *launch = launch_kind<TILE, B_K, true, CEP_IDENTITY>;
  if constexpr (B_K) {
    if (!a.f.res) launch = launch_kind<TILE, B_K, false, CEP_IDENTITY>;
  } else {
    if (a.f.act == CEP_RELU) launch = launch_kind<TILE, B_K, true, CEP_RELU>;
    if (a.f.act == CEP_SILU) launch = launch_kind<TILE, B_K, true, CEP_SILU>;
    if (a.f.act == CEP_GELU) launch = launch_kind<TILE, B_K, true, CEP_GELU>;
    if (a.f.act == CEP_GELU_TANH) launch = launch_kind<TILE, B_K, true, CEP_GELU_TANH>;
  }
  launch(a, items, s);
}

// The most tiles that the groups' rows can be in.
int64_t most_tiles(const Groups &g, int tile) {
  return g.n ? std::min<int64_t>(g.rows, g.rows / tile + g.n) : (g.rows + tile - 1) / tile;
}

LinearArgs linear_args(const Groups &g, const __bf16 *A, int64_t lda, const __bf16 *W, int64_t ldb,
                       int N, int K, const Finish &f) {
  LinearArgs a{};
  a.A = A, a.lda = lda;
  a.B0 = W, a.ldb = ldb;
  a.N = N, a.K = K, a.segs = 1, a.splits = 1;
  a.groups = g, a.f = f;
  a.w_stride = g.n ? (int64_t)N * K : 0;
  return a;
}

void launch_grads(int tile, const LinearArgs &dx, WgradArgs dw, hipStream_t s) {
  dw.splits = 1;
  const int64_t items = most_tiles(dx.groups, kTile[tile]) * ((dx.N + kTile[tile] - 1) / kTile[tile]);
  const int64_t room = (dense_tiles(tile, dw.M, dw.N) + 7) / 8 * std::max(dw.groups.n, 1);
  const dim3 grid((unsigned)(((items + 7) / 8 + room) * 8));
  auto *k = tile == 0 ? k_linear_grads<128, 2, 4, false> : k_linear_grads<64, 2, 4, false>;
  if (dx.f.res) k = tile == 0 ? k_linear_grads<128, 2, 4, true> : k_linear_grads<64, 2, 4, true>;
  hipLaunchKernelGGL(k, grid, dim3(512), 0, s, dx, dw);
}

// A product over the groups' rows: A [rows][K], W as B, the epilogue's output [rows][N].
template <bool B_K>
void launch_linear(const Plan &p, const Groups &g, const __bf16 *A, int64_t lda, const __bf16 *W,
                   int64_t ldb, int N, int K, const Finish &f, float *part, hipStream_t s) {
  if (p.stream) {
    LinearRowsArgs a{};
    a.A[0] = A, a.lda = lda;
    a.B0 = W, a.ldb = ldb;
    a.N = N, a.K = K;
    a.splits = p.splits, a.col_blocks = (N + kCols - 1) / kCols;
    a.groups = g, a.w_stride = g.n ? (int64_t)N * K : 0, a.part = part, a.f = f;
    const dim3 grid((unsigned)(most_tiles(g, p.mf * 16) * a.col_blocks * a.splits));
    if (p.mf == 1) hipLaunchKernelGGL(k_linear_rows<1>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(k_linear_rows<2>, grid, dim3(256), 0, s, a);
  } else {
    LinearArgs a = linear_args(g, A, lda, W, ldb, N, K, f);
    a.splits = p.splits, a.part = part;
    const int64_t items =
        most_tiles(g, kTile[p.tile]) * p.splits * ((N + kTile[p.tile] - 1) / kTile[p.tile]);
    if (p.tile == 0) launch_tiles<0, B_K>(a, items, s);
    else launch_tiles<1, B_K>(a, items, s);
  }
  if (p.splits > 1) launch_finish(part, p.splits, g, f, g.rows, s);
}

template <int ROWS>
auto dz_kernel(int act) {
  return act == CEP_RELU        ? k_linear_dz<CEP_RELU, ROWS>
         : act == CEP_SILU      ? k_linear_dz<CEP_SILU, ROWS>
         : act == CEP_GELU      ? k_linear_dz<CEP_GELU, ROWS>
         : act == CEP_GELU_TANH ? k_linear_dz<CEP_GELU_TANH, ROWS>
                                : k_linear_dz<CEP_IDENTITY, ROWS>;
}

int check_shared(const char *fn, const cep_linear_desc *d, const int32_t *offsets) {
  if (const char *why = bad_desc(d)) return refuse(CEP_EINVAL, "%s: %s", fn, why);
  if (!offsets != !d->n_groups)
    return refuse(CEP_EINVAL, "%s: offsets go with n_groups", fn);
  if (!aligned(offsets, 4)) return refuse(CEP_EINVAL, "%s: offsets are not aligned to their type", fn);
  return CEP_OK;
}

}  // namespace
}  // namespace cep

using namespace cep;

CEP_API size_t cep_linear_workspace(const cep_linear_desc *d, int backward) {
  return bad_desc(d) ? 0 : space_of(d, backward).bytes;
}

CEP_API int cep_linear(const cep_linear_desc *d, const void *x, const void *w, const float *bias,
                       const void *mul, const void *residual, const int32_t *offsets, void *y,
                       float *preact, void *workspace, size_t workspace_bytes, hipStream_t s) {
  const char *fn = "cep_linear";
  if (const int rc = check_shared(fn, d, offsets)) return rc;
  if (d->rows == 0) return CEP_OK;
  if (!x || !w || !y) return refuse(CEP_EINVAL, "%s: NULL array", fn);
  for (const void *p : {x, w, (const void *)bias, mul, residual, (const void *)y,
                        (const void *)preact, (const void *)workspace})
    if (!aligned(p, 16)) return refuse(CEP_EINVAL, "%s: pointers must be 16-byte aligned", fn);
  if (!workspace || workspace_bytes < cep_linear_workspace(d, 0))
    return refuse(workspace ? CEP_ENOMEM : CEP_EINVAL, "%s: needs a workspace of %zu bytes", fn,
                  cep_linear_workspace(d, 0));
  for (const void *p : {x, w, (const void *)bias})
    if (p && (y == p || preact == p))
      return refuse(CEP_EINVAL, "%s: y or preact overlaps x, w or bias", fn);
  if (preact && (preact == y || preact == mul || preact == residual))
    return refuse(CEP_EINVAL, "%s: preact overlaps y, mul or residual", fn);
  const int D = d->d_in, N = d->d_out;
  Finish f{};
  f.bias = bias, f.mul = (const __bf16 *)mul, f.res = residual, f.y = y, f.pre = preact;
  f.ld_mul = d->ld_mul ? d->ld_mul : N;
  f.ld_res = d->ld_res ? d->ld_res : N;
  f.ld_y = d->ld_y ? d->ld_y : N;
  f.N = N, f.act = d->act, f.res_dtype = d->res_dtype, f.y_dtype = d->y_dtype;
  const Groups g{offsets, d->n_groups, d->rows};
  launch_linear<false>(plan_of(d->rows, N, D, d->n_groups, true), g, (const __bf16 *)x,
                       d->ld_x ? d->ld_x : D, (const __bf16 *)w, N, N, D, f, (float *)workspace, s);
  return launched(fn);
}

CEP_API int cep_linear_backward(const cep_linear_desc *d, const void *dy, const void *x,
                                const void *w, const void *mul, const int32_t *offsets,
                                const float *preact, const void *dx_add, void *dx, void *dw,
                                float *dbias, void *dmul, void *workspace, size_t workspace_bytes,
                                hipStream_t s) {
  const char *fn = "cep_linear_backward";
  if (const int rc = check_shared(fn, d, offsets)) return rc;
  if (!dx && !dw && !dbias && !dmul) return refuse(CEP_EINVAL, "%s: no output", fn);
  if (dx_add && !dx) return refuse(CEP_EINVAL, "%s: dx_add goes with dx", fn);
  if (dmul && !mul) return refuse(CEP_EINVAL, "%s: dmul goes with mul", fn);
  const bool curved = d->act != CEP_IDENTITY || dmul;
  if (d->rows && (!dy || (dx && !w) || (dw && !x) || (curved && !preact)))
    return refuse(CEP_EINVAL, "%s: NULL array", fn);
  for (const void *p : {dy, x, w, mul, (const void *)preact, dx_add, (const void *)dx,
                        (const void *)dw, (const void *)dbias, (const void *)dmul,
                        (const void *)workspace})
    if (!aligned(p, 16)) return refuse(CEP_EINVAL, "%s: pointers must be 16-byte aligned", fn);
  if (!workspace || workspace_bytes < cep_linear_workspace(d, 1))
    return refuse(workspace ? CEP_ENOMEM : CEP_EINVAL, "%s: needs a workspace of %zu bytes", fn,
                  cep_linear_workspace(d, 1));
  for (const void *p : {dy, x, w})
    if (p && (dx == p || dw == p || dbias == p))
      return refuse(CEP_EINVAL, "%s: dx, dw or dbias overlaps dy, x or w", fn);
  for (const void *p : {mul, (const void *)preact})
    if (p && dbias == p) return refuse(CEP_EINVAL, "%s: dbias overlaps mul or preact", fn);
  const int D = d->d_in, N = d->d_out, T = d->rows, n_groups = std::max(d->n_groups, 1);
  const Space space = space_of(d, 1);
  const Groups g{offsets, d->n_groups, T};
  uint8_t *ws = (uint8_t *)workspace;
  float *part = (float *)(ws + space.part), *sums = (float *)(ws + space.bias);
  // dy is dz already where nothing lies between them but a bias
  const __bf16 *dz = (const __bf16 *)dy;
  int64_t ld_z = d->ld_y ? d->ld_y : N;
  const bool same = d->act == CEP_IDENTITY && !mul && d->y_dtype == CEP_BF16;
  if (T && (dbias || dmul || (!same && (dx || dw)))) {
    DzArgs a{};
    a.dy = dy, a.ld_y = ld_z, a.y_dtype = d->y_dtype;
    a.pre = curved ? preact : nullptr;
    a.mul = (const __bf16 *)mul, a.ld_mul = d->ld_mul ? d->ld_mul : N;
    a.dz = !same && (dx || dw) ? (__bf16 *)ws : nullptr;
    a.dmul = (__bf16 *)dmul;
    a.part = dbias ? (dz_chunks(d) == 1 ? dbias : sums) : nullptr;
    a.N = N, a.groups = g;
    const dim3 grid(dz_chunks(d), (N + kDzCols - 1) / kDzCols);
    auto *k = dz_rows(T, N) == 8 ? dz_kernel<8>(d->act) : dz_kernel<32>(d->act);
    hipLaunchKernelGGL(k, grid, dim3(256), 0, s, a);
  }
  if (!same) dz = (const __bf16 *)ws, ld_z = N;
  if (dbias && dz_chunks(d) != 1)
    hipLaunchKernelGGL(k_linear_dbias, dim3((N + 63) / 64, n_groups), dim3(256), 0, s, sums,
                       dz_rows(T, N), N, g, dbias);
  Finish f{};
  f.res = dx_add, f.y = dx, f.N = D, f.res_dtype = f.y_dtype = d->dx_dtype;
  f.ld_res = f.ld_y = d->ld_dx ? d->ld_dx : D;
  const Plan p = wgrad_plan(d);
  WgradArgs a{};
  a.A = (const __bf16 *)x, a.lda = d->ld_x ? d->ld_x : D;
  a.B0 = dz, a.ldb = ld_z;
  a.M = D, a.N = N, a.K = T, a.segs = 1, a.splits = p.splits;
  a.groups = g, a.part = part;
  a.f.y = dw, a.f.N = N, a.f.y_dtype = d->dw_dtype, a.f.ld_y = N;
  if (const int tile = dx && dw ? grads_tile(d) : -1; tile >= 0) {
    launch_grads(tile, linear_args(g, dz, ld_z, (const __bf16 *)w, N, D, N, f), a, s);
    return launched(fn);
  }
  if (dx && T)
    launch_linear<true>(plan_of(T, D, N, d->n_groups, false), g, dz, ld_z, (const __bf16 *)w, N, D, N,
                        f, part, s);
  if (dw && p.tile == kFewTile) {
    const int64_t items = dense_tiles(1, D, N);
    hipLaunchKernelGGL(k_linear_wgrad_few, dim3((unsigned)((items + 7) / 8 * 8 * n_groups)), dim3(512),
                       0, s, a);
  } else if (dw) {
    const int64_t items = dense_tiles(p.tile, D, N) * p.splits;
    const dim3 grid((unsigned)((items + 7) / 8 * 8 * n_groups));
    if (p.tile == 0)
      hipLaunchKernelGGL((k_linear_wgrad<128, 2, 4>), grid, dim3(512), 0, s, a);
    else hipLaunchKernelGGL((k_linear_wgrad<64, 2, 4>), grid, dim3(512), 0, s, a);
    if (p.splits > 1) launch_finish(part, p.splits, Groups{nullptr, 0, D}, a.f, D, s);
  }
  return launched(fn);
}
