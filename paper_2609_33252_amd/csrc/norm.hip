// Root-mean-square norm of token rows with the residual's addition and an
// MXFP8 copy of the result, and its gradient, for gfx950.
//
//   s = x + r                         (float32; stored as the new residual)
//   y = s * w / sqrt(mean(s^2) + eps)
//   MXFP8(y): e4m3 codes, one E8M0 scale per 32 channels
// and with n = s / sqrt(mean(s^2) + eps), a = dy * w:
//   dx = (a - n * mean(a * n)) / sqrt(mean(s^2) + eps) + dres
//   dw = sum over rows of dy * n
//
// Both read every input once and write every output once: bound by HBM.
// A row stays in registers between the sum of its squares and its scaling.
// Measured: 8191 float32 rows of 6144 with a bf16 residual, y and MXFP8 107 us,
// 5.2 TB/s (a large copy 4.9); gradient of 4096 bf16 rows of 7168 52.6 us,
// 4.5 TB/s, 5 of it the sum of dw's parts; one row of 7168 4.1 to 4.8 us, where
// an empty launch takes 3.5 to 4.
#include "block_ops.h"

#include <algorithm>
#include <type_traits>

namespace cep {
namespace {

struct NormArgs {
  const void *x, *res, *w;
  void *res_out, *y;
  uint8_t *codes, *scales;
  int64_t ld_x, ld_res, ld_y, ld_codes, ld_scales;
  int rows, d, x_dtype, res_dtype, w_dtype, y_dtype;
  float eps;
};

// Sum over the LANES threads of a row (a wave, or the whole block).
template <int LANES>
__device__ inline float row_sum(float v, float *lds) {
  v = wave_sum(v);
  if (LANES > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < LANES / 64; ++i) v += lds[i];
  }
  return v;
}

// Eight channels of a 32-channel block in each of four neighbouring lanes:
// E8M0 scale 2^(floor(log2 amax) - 8), codes e4m3(v / scale) saturated at 448.
// A block with an infinity or NaN gets the scale code 255 (NaN).  Returns the
// lane's codes; *code gets the scale's code.
__device__ inline uint2 mxfp8_block(const float v[8], int *code) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
  m = max(m, (uint32_t)__shfl_xor((int)m, 1, 4));
  m = max(m, (uint32_t)__shfl_xor((int)m, 2, 4));
  const int ex = (int)(m >> 23);
  *code = ex == 255 ? 255 : max(ex - 8, 0);
  const int e = 127 - max(ex - 8, 0);
  int w[2] = {0, 0};
  float q[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) q[j] = fminf(fmaxf(ldexpf(v[j], e), -448.0f), 448.0f);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h], q[4 * h + 1], w[h], false);
    w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * h + 2], q[4 * h + 3], w[h], true);
  }
  return make_uint2((uint32_t)w[0], (uint32_t)w[1]);
}

// LANES threads a row, NV groups of eight channels each.  With one group of
// 1024 threads (a few rows) the weight is loaded before the sum, so that the row
// waits for memory once; elsewhere the registers are worth more as waves (8192
// rows of 7168: 109 us, 114 with the weight ahead).
template <int LANES, int NV>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void k_rms_norm(NormArgs a) {
  constexpr bool AHEAD = LANES == 1024 && NV == 1;
  __shared__ float lds[LANES > 64 ? LANES / 64 : 1];
  const int lane = threadIdx.x % LANES;
  const int row = LANES < 256 ? blockIdx.x * (256 / LANES) + threadIdx.x / LANES : blockIdx.x;
  if (row >= a.rows) return;  // uniform over the row's threads
  auto col = [&](int u) { return (u * LANES + lane) * 8; };
  float s[NV][8], ahead[8];
#pragma unroll
  for (int u = 0; u < NV; ++u) load8(a.x, a.x_dtype, row * a.ld_x + col(u), a.d - col(u), s[u]);
  if (AHEAD) load8(a.w, a.w_dtype, col(0), a.d - col(0), ahead);
  if (a.res) {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      float r[8];
      load8(a.res, a.res_dtype, row * a.ld_res + col(u), a.d - col(u), r);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[u][j] += r[j];
      if (a.res_out)
        store8(a.res_out, a.res_dtype, row * a.ld_res + col(u), a.d - col(u), s[u]);
    }
  }
  float sq = 0.f;
#pragma unroll
  for (int u = 0; u < NV; ++u)
#pragma unroll
    for (int j = 0; j < 8; ++j) sq = fmaf(s[u][j], s[u][j], sq);
  const float inv = 1.0f / sqrtf(row_sum<LANES>(sq, lds) / (float)a.d + a.eps);
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int c = col(u);
    if (c >= a.d) continue;
    float w[8], y[8];
    if (!AHEAD) load8(a.w, a.w_dtype, c, a.d - c, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = s[u][j] * inv * (AHEAD ? ahead[j] : w[j]);
    if (a.y) store8(a.y, a.y_dtype, row * a.ld_y + c, a.d - c, y);
    if (a.codes) {  // d is a multiple of 32: whole blocks
      int code;
      const uint2 q = mxfp8_block(y, &code);
      *(uint2 *)(a.codes + row * a.ld_codes + c) = q;
      if ((lane & 3) == 0) a.scales[row * a.ld_scales + c / kMxBlock] = (uint8_t)code;
    }
  }
}

struct NormGradArgs {
  const void *s, *w, *dy, *dres;
  void *dx;
  float *part;  // [blocks][d] partial sums of dw
  int64_t ld_s, ld_dy, ld_dx;
  int rows, d, s_dtype, dx_dtype, w_dtype, dy_dtype;
  float eps;
};

// Eight values of a row as they are in memory (BF: bf16, else widened).
template <bool BF>
struct Raw8 {
  Vec16 v[BF ? 1 : 2];
  // whole: the row has eight values at least
  template <bool SHIFT>
  __device__ void load(const void *row, int dtype, int64_t at, int n, bool whole) {
    if (BF && n >= 8) {
      v[0] = *(const Any16 *)((const char *)row + at * 2);
      return;
    }
    if (BF && SHIFT && whole) {  // the row's last few: its last eight, shifted down
      v[0] = Vec16{};
      if (n <= 0) return;
      const Vec16 t = *(const Any16 *)((const char *)row + (at + n - 8) * 2);
      const int bits = (8 - n) * 16;
      uint64_t lo = t[0] | (uint64_t)t[1] << 32, hi = t[2] | (uint64_t)t[3] << 32;
      lo = bits >= 64 ? hi >> (bits - 64) : lo >> bits | hi << (64 - bits);
      hi = bits >= 64 ? 0 : hi >> bits;
      v[0] = Vec16{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
      return;
    }
    float f[8];
    load8(row, dtype, at, n, f);
    if (BF)
      v[0] = Vec16{bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]),
                   bf16_pair(f[6], f[7])};
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j / 4][j % 4] = __float_as_uint(f[j]);
  }
  __device__ float operator[](int j) const {
    if (!BF) return __uint_as_float(v[j / 4][j % 4]);
    const uint32_t u = v[0][j / 2];
    return __uint_as_float(j % 2 ? u & 0xffff0000u : u << 16);
  }
};
// A row of the backward pass in registers.
template <bool BF, int NV>
struct GradRow {
  Raw8<BF> s[NV], dy[NV], dres[NV];
};

// Block b takes rows b, b + gridDim.x, ... and keeps its part of dw in
// registers; the parts are summed in block order by k_rms_norm_dw, so dw does
// not depend on which block ran first.  Rows of one wave go to the four waves
// of a block in turn, whose parts meet in LDS.  AHEAD: the next row is loaded
// while this one's sums meet, and the weight stays in registers (4096 rows of
// 7168: 56 us, 141 with each row loaded when its turn comes).  BF: the rows are
// all bf16 and are kept so until they are used.
template <int LANES, int NV, bool BF, bool AHEAD>
__global__ __launch_bounds__(LANES == 64 ? 256 : LANES,
                             LANES == 512 && !AHEAD ? 4 : 1) void k_rms_norm_grad(NormGradArgs a) {
  constexpr int SIDE = LANES == 64 ? 4 : 1;  // rows side by side in a block
  __shared__ float lds[2][2][LANES / 64];
  const int lane = SIDE > 1 ? threadIdx.x % LANES : threadIdx.x;
  const int64_t first = (int64_t)blockIdx.x * SIDE + (SIDE > 1 ? threadIdx.x / LANES : 0);
  const int64_t stride = (int64_t)gridDim.x * SIDE;
  const bool whole = a.d >= 8;
  auto load = [&](GradRow<BF, NV> &r, int64_t row) {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = (u * LANES + lane) * 8;
      r.s[u].template load<AHEAD>(a.s, a.s_dtype, row * a.ld_s + c, a.d - c, whole);
      r.dy[u].template load<AHEAD>(a.dy, a.dy_dtype, row * a.ld_dy + c, a.d - c, whole);
      if (AHEAD && a.dres)
        r.dres[u].template load<AHEAD>(a.dres, a.dx_dtype, row * a.ld_dx + c, a.d - c, whole);
    }
  };
  float w[NV][8], dw[NV][8] = {};
  auto load_w = [&](int u) {
    const int c = (u * LANES + lane) * 8;
    load8(a.w, a.w_dtype, c, a.d - c, w[u]);
  };
  if (AHEAD)
#pragma unroll
    for (int u = 0; u < NV; ++u) load_w(u);
  GradRow<BF, NV> cur = {}, next = {};
  if (AHEAD && first < a.rows) load(next, first);
  int turn = 0;
  for (int64_t row = first; row < a.rows; row += stride, turn ^= 1) {
    if (AHEAD) {
      cur = next;
      if (row + stride < a.rows) load(next, row + stride);
    } else {
      load(cur, row);
    }
    float sq = 0.f, dot = 0.f;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (!AHEAD) load_w(u);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sq = fmaf(cur.s[u][j], cur.s[u][j], sq);
        dot = fmaf(cur.dy[u][j] * w[u][j], cur.s[u][j], dot);
      }
    }
    sq = wave_sum(sq);
    dot = wave_sum(dot);
    if (LANES > 64) {  // two places in turn: one barrier a row
      if ((lane & 63) == 0) {
        lds[turn][0][lane >> 6] = sq;
        lds[turn][1][lane >> 6] = dot;
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      sq = dot = 0.f;
#pragma unroll
      for (int i = 0; i < LANES / 64; ++i) {
        sq += lds[turn][0][i];
        dot += lds[turn][1][i];
      }
    }
    const float inv = 1.0f / sqrtf(sq / (float)a.d + a.eps);
    const float mean = dot * inv / (float)a.d;  // of a * n
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = (u * LANES + lane) * 8;
      if (c >= a.d) continue;
      float dx[8];
      if (!AHEAD) {
        asm volatile("" ::: "memory");  // not kept from the sums above
        load_w(u);
        if (a.dres)
          cur.dres[u].template load<AHEAD>(a.dres, a.dx_dtype, row * a.ld_dx + c, a.d - c, whole);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = cur.s[u][j] * inv;
        dx[j] = inv * (cur.dy[u][j] * w[u][j] - n * mean) + cur.dres[u][j];
        dw[u][j] = fmaf(cur.dy[u][j], n, dw[u][j]);
      }
      store8(a.dx, a.dx_dtype, row * a.ld_dx + c, a.d - c, dx);
    }
  }
  if (SIDE > 1) {
    __shared__ float sums[SIDE > 1 ? SIDE : 1][SIDE > 1 ? LANES * 8 : 1];
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[threadIdx.x / LANES][lane * 8 + j] = dw[0][j];
    __syncthreads();
    if (threadIdx.x >= LANES) return;
    for (int i = 1; i < SIDE; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) dw[0][j] += sums[i][lane * 8 + j];
  }
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int c = (u * LANES + lane) * 8;
    store8(a.part, CEP_F32, (int64_t)blockIdx.x * a.d + c, a.d - c, dw[u]);
  }
}

// dw: 64 columns a block, 16 strands of the parts each, summed in a fixed
// order.
__global__ __launch_bounds__(1024) void k_rms_norm_dw(const float *part, int n, int d, int w_dtype,
                                                      void *dw) {
  __shared__ float lds[16][64];
  const int col = blockIdx.x * 64 + (threadIdx.x & 63), strand = threadIdx.x >> 6;
  float v = 0.f;
  if (col < d) {
#pragma unroll 8
    for (int i = strand; i < n; i += 16) v += part[(size_t)i * d + col];
  }
  lds[strand][threadIdx.x & 63] = v;
  __syncthreads();
  if (strand == 0 && col < d) {
#pragma unroll
    for (int i = 1; i < 16; ++i) v += lds[i][threadIdx.x];
    if (w_dtype == CEP_BF16) ((__bf16 *)dw)[col] = (__bf16)v;
    else ((float *)dw)[col] = v;
  }
}

// Calls f with the threads a row takes and the groups of eight channels each
// of them holds: a wave up to 1024 channels (no barrier), else 256 threads.
// Rows beyond 8192 channels take 1024, as do up to 256 rows, one workgroup a
// compute unit (7168 channels, one row 6.3 us with 256 threads, 4.6 with 1024;
// 256 rows 8.4 and 5.9).
template <class F>
void by_width(int d, int rows, F f) {
  using std::integral_constant;
  const bool few = rows <= 256;
  if (d <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (d <= 1024) f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  else if (d <= 2048) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (d <= 8192 && few) f(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
  else if (d <= 4096) f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (d <= 8192) f(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  else if (d <= 16384) f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  else f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

// Blocks of the backward pass: the most that run at once are two a compute
// unit (512), and each writes a part of dw.
int grad_blocks(int rows, int d) { return std::min(d <= 512 ? (rows + 3) / 4 : rows, 512); }

// Threads and groups of the backward pass, which keeps three rows, the weight
// and dw.  Rows that are not all bf16 are not loaded ahead: twice as wide, they
// run at memory's rate without it (4096 float32 rows with dres, of 4096 channels
// 56 us, of 7168 97, both 4.8 TB/s; 7168 in bf16 with a float32 dy 67 us, 4.4
// TB/s).  Nor are rows past 8192 channels (the registers of two rows would not
// hold four waves a unit).
template <class F>
void by_width_grad(int d, bool bf, F f) {
  using std::integral_constant;
  auto with = [&](auto lanes, auto nv, auto ahead) {
    if (bf) f(lanes, nv, std::true_type{}, ahead);
    else f(lanes, nv, std::false_type{}, std::false_type{});
  };
  if (d <= 512) with(integral_constant<int, 64>{}, integral_constant<int, 1>{}, std::true_type{});
  else if (d <= 2048) with(integral_constant<int, 256>{}, integral_constant<int, 1>{}, std::true_type{});
  else if (d <= 4096) with(integral_constant<int, 512>{}, integral_constant<int, 1>{}, std::true_type{});
  else if (d <= 8192) with(integral_constant<int, 512>{}, integral_constant<int, 2>{}, std::true_type{});
  else if (d <= 16384) with(integral_constant<int, 1024>{}, integral_constant<int, 2>{}, std::false_type{});
  else with(integral_constant<int, 1024>{}, integral_constant<int, 4>{}, std::false_type{});
}

// nullptr, or what is wrong with a descriptor
const char *bad_desc(const cep_norm_desc *n) {
  if (!n) return "desc is NULL";
  if (n->rows < 0 || n->rows > kMaxOpRows) return "rows must be in 0..2^21";
  if (n->d < 1 || n->d > kMaxDim) return "d must be in 1..32768";
  if (!is_float_dtype(n->x_dtype) || !is_float_dtype(n->res_dtype) ||
      !is_float_dtype(n->w_dtype) || !is_float_dtype(n->y_dtype))
    return "dtypes must be CEP_F32 or CEP_BF16";
  if (!(n->eps >= 0.f)) return "eps must be >= 0";
  for (int64_t ld : {n->ld_x, n->ld_res, n->ld_y})
    if (ld != 0 && ld < n->d) return "a row stride is shorter than a row";
  return nullptr;
}

int64_t stride_of(int64_t ld, int64_t dense) { return ld ? ld : dense; }

}  // namespace
}  // namespace cep

using namespace cep;

CEP_API int cep_rms_norm(const cep_norm_desc *n, const void *x, const void *residual,
                         const void *w, void *res_out, void *y, uint8_t *codes, uint8_t *scales,
                         hipStream_t s) {
  if (const char *why = bad_desc(n)) return refuse(CEP_EINVAL, "cep_rms_norm: %s", why);
  if (!w || (!x && n->rows)) return refuse(CEP_EINVAL, "cep_rms_norm: NULL x or w");
  if (!y && !codes) return refuse(CEP_EINVAL, "cep_rms_norm: neither y nor codes is asked for");
  if ((codes != nullptr) != (scales != nullptr))
    return refuse(CEP_EINVAL, "cep_rms_norm: codes and scales come together");
  if (res_out && !residual) return refuse(CEP_EINVAL, "cep_rms_norm: res_out without residual");
  const int64_t ld_codes = stride_of(n->ld_codes, n->d);
  if (codes && (n->d % kMxBlock || ld_codes < n->d || ld_codes % 8 || !aligned(codes, 8) ||
                (n->ld_scales && n->ld_scales < n->d / kMxBlock)))
    return refuse(CEP_EINVAL, "cep_rms_norm: MXFP8 rows need d a multiple of 32, 8-byte aligned "
                              "codes and row strides of at least a row");
  if (!aligned(x, dtype_bytes(n->x_dtype)) || !aligned(residual, dtype_bytes(n->res_dtype)) ||
      !aligned(res_out, dtype_bytes(n->res_dtype)) || !aligned(w, dtype_bytes(n->w_dtype)) ||
      !aligned(y, dtype_bytes(n->y_dtype)))
    return refuse(CEP_EINVAL, "cep_rms_norm: a pointer is not aligned to its type");
  if (n->rows == 0) return CEP_OK;
  const NormArgs a{x, residual, w, res_out, y, codes, scales, stride_of(n->ld_x, n->d),
                   stride_of(n->ld_res, n->d), stride_of(n->ld_y, n->d), ld_codes,
                   stride_of(n->ld_scales, n->d / kMxBlock), n->rows, n->d, n->x_dtype,
                   n->res_dtype, n->w_dtype, n->y_dtype, n->eps};
  by_width(n->d, n->rows, [&](auto lanes, auto nv) {
    constexpr int L = decltype(lanes)::value, NV = decltype(nv)::value;
    const int per = L < 256 ? 256 / L : 1;
    hipLaunchKernelGGL((k_rms_norm<L, NV>), dim3((n->rows + per - 1) / per),
                       dim3(L < 256 ? 256 : L), 0, s, a);
  });
  return launched("cep_rms_norm");
}

CEP_API size_t cep_rms_norm_workspace(const cep_norm_desc *n) {
  if (bad_desc(n)) return 0;
  return std::max<size_t>((size_t)grad_blocks(n->rows, n->d) * n->d * 4, 256);
}

CEP_API int cep_rms_norm_backward(const cep_norm_desc *n, const void *x, const void *w,
                                  const void *dy, const void *dres, void *dx, void *dw,
                                  void *workspace, size_t workspace_bytes, hipStream_t s) {
  const char *fn = "cep_rms_norm_backward";
  if (const char *why = bad_desc(n)) return refuse(CEP_EINVAL, "%s: %s", fn, why);
  if (!w || !dw || (n->rows && (!x || !dy || !dx)))
    return refuse(CEP_EINVAL, "%s: NULL x, w, dy, dx or dw", fn);
  if (!workspace || !aligned(workspace, 4) || workspace_bytes < cep_rms_norm_workspace(n))
    return refuse(workspace ? CEP_ENOMEM : CEP_EINVAL, "%s: needs a workspace of %zu bytes", fn,
                  cep_rms_norm_workspace(n));
  if (!aligned(x, dtype_bytes(n->x_dtype)) || !aligned(dres, dtype_bytes(n->res_dtype)) ||
      !aligned(dx, dtype_bytes(n->res_dtype)) || !aligned(w, dtype_bytes(n->w_dtype)) ||
      !aligned(dw, dtype_bytes(n->w_dtype)) || !aligned(dy, dtype_bytes(n->y_dtype)))
    return refuse(CEP_EINVAL, "%s: a pointer is not aligned to its type", fn);
  const int blocks = grad_blocks(n->rows, n->d);
  const NormGradArgs a{x, w, dy, dres, dx, (float *)workspace, stride_of(n->ld_x, n->d),
                       stride_of(n->ld_y, n->d), stride_of(n->ld_res, n->d), n->rows, n->d,
                       n->x_dtype, n->res_dtype, n->w_dtype, n->y_dtype, n->eps};
  if (blocks)
    by_width_grad(n->d, n->x_dtype == CEP_BF16 && n->y_dtype == CEP_BF16 &&
                            (!dres || n->res_dtype == CEP_BF16),
                  [&](auto lanes, auto nv, auto bf, auto ahead) {
                    constexpr int L = decltype(lanes)::value, NV = decltype(nv)::value;
                    hipLaunchKernelGGL(
                        (k_rms_norm_grad<L, NV, decltype(bf)::value, decltype(ahead)::value>),
                        dim3(blocks), dim3(L == 64 ? 256 : L), 0, s, a);
                  });
  hipLaunchKernelGGL(k_rms_norm_dw, dim3((n->d + 63) / 64), dim3(1024), 0, s, a.part, blocks, n->d,
                     n->w_dtype, dw);
  return launched(fn);
}
