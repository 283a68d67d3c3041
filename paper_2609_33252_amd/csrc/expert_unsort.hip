// The experts' rows back to their tokens, weighted and summed, and its gradient,
// for gfx950.
//
//   y[t] = r[t] + sum over j of w[t][j] ys[place[t][j]]
//   dys[place[t][j]] = w[t][j] dy[t];  dw[t][j] = <dy[t], ys[place[t][j]]>
//
// Every row is read and written once: bound by HBM (8192 tokens of 6 rows of 4096, bf16:
// 106 us, 536 MB, 5.1 TB/s; the gradient 168 us, 870 MB, 5.2 TB/s).  The sum over the slots and the
// product over the channels have a fixed order, so results do not depend on timing.
#include "block_ops.h"

#include <algorithm>

namespace cep {
namespace {

struct UnsortArgs {
  const void *ys;
  const int32_t *place;
  const float *w;
  const void *res;
  void *y;
  const void *dy;
  void *dys;
  float *dw;
  int64_t ld_ys, ld_res, ld_y;
  int rows, k, d, sorted, ys_dtype, res_dtype, y_dtype;
  int waves;  // of a row
};

// The slot's sorted row, -1: none.
__device__ inline int place_of(const UnsortArgs &a, int64_t pair) {
  const int p = a.place[pair];
  return p < a.sorted ? p : -1;
}

// Eight consecutive values of a row as they are in memory, so that a row on the way
// takes no more registers than bytes (n: those inside the row, the others zero).  A
// row is read once: loaded past the caches' retention (8192 x 6 rows of 4096 to their
// tokens 106 us, 121 with plain loads).
template <bool F32>
struct Eight {
  Vec16 v[F32 ? 2 : 1];
  __device__ inline void load(const void *row, int64_t at, int n) {
    if (n >= 8) {
#pragma unroll
      for (int h = 0; h < (F32 ? 2 : 1); ++h)
        v[h] = __builtin_nontemporal_load((const Any16 *)((const char *)row + at * (F32 ? 4 : 2) + 16 * h));
      return;
    }
#pragma unroll
    for (int i = 0; i < (F32 ? 8 : 4); ++i) {
      uint32_t u = 0;
      if (F32) {
        if (i < n) u = ((const uint32_t *)row)[at + i];
      } else {
        if (2 * i < n) u = ((const uint16_t *)row)[at + 2 * i];
        if (2 * i + 1 < n) u |= (uint32_t)((const uint16_t *)row)[at + 2 * i + 1] << 16;
      }
      v[i / 4][i % 4] = u;
    }
  }
  __device__ inline float operator[](int i) const {
    if (F32) return __uint_as_float(v[i / 4][i % 4]);
    const uint32_t u = v[0][i / 2];
    return __uint_as_float(i % 2 ? u & 0xffff0000u : u << 16);
  }
};

// A wave a token and 512 channels of it; the rows of all slots on the way at once.
template <int KM, bool YS32>
__global__ __launch_bounds__(256) void k_unsort(UnsortArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  const int64_t item = block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = item / a.waves;
  if (t >= a.rows) return;
  const int c = ((int)(item % a.waves) * 64 + lane) * 8, n = a.d - c;
  const bool slot = lane < a.k;
  const int my = slot ? place_of(a, t * a.k + lane) : -1;
  const float mw = slot && a.w ? a.w[t * a.k + lane] : 1.0f;
  float s[8] = {};
  Eight<YS32> v[KM];
  if (a.res) load8(a.res, a.res_dtype, t * a.ld_res + c, n, s);
#pragma unroll
  for (int j = 0; j < KM; ++j) {
    const int p = __builtin_amdgcn_readlane(my, j);
    if (j < a.k && p >= 0) v[j].load(a.ys, p * a.ld_ys + c, n);
  }
#pragma unroll
  for (int j = 0; j < KM; ++j) {
    const int p = __builtin_amdgcn_readlane(my, j);
    if (j >= a.k || p < 0) continue;
    const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mw), j));
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = fmaf(w, v[j][i], s[i]);
  }
  if (n > 0) store8(a.y, a.y_dtype, t * a.ld_y + c, n, s);
}

// LANES threads a token, 8 channels each at a time.
template <int LANES, int KM, bool YS32>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void k_unsort_grad(UnsortArgs a) {
  __shared__ float part[LANES > 64 ? LANES / 64 : 1][KM];
  const int lane = threadIdx.x & 63, at = threadIdx.x % LANES;
  const int64_t t = LANES < 256 ? (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES : blockIdx.x;
  if (t >= a.rows) return;  // uniform over the token's threads
  const bool slot = lane < a.k;
  const int my = slot ? place_of(a, t * a.k + lane) : -1;
  const float mw = slot && a.w ? a.w[t * a.k + lane] : 1.0f;
  float dot[KM] = {};
  for (int c = at * 8; c < (a.d + LANES * 8 - 1) / (LANES * 8) * (LANES * 8); c += LANES * 8) {
    const int n = a.d - c;
    float g[8];
    load8(a.dy, a.y_dtype, t * a.ld_y + c, n, g);
    Eight<YS32> v[KM];
    if (a.dw) {
#pragma unroll
      for (int j = 0; j < KM; ++j) {
        const int p = __builtin_amdgcn_readlane(my, j);
        if (j < a.k && p >= 0) v[j].load(a.ys, p * a.ld_ys + c, n);
      }
    }
#pragma unroll
    for (int j = 0; j < KM; ++j) {
      const int p = __builtin_amdgcn_readlane(my, j);
      if (j >= a.k || p < 0) continue;
      if (a.dw) {
#pragma unroll
        for (int i = 0; i < 8; ++i) dot[j] = fmaf(g[i], v[j][i], dot[j]);
      }
      if (a.dys && n > 0) {
        const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mw), j));
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = w * g[i];
        store8(a.dys, YS32 ? CEP_F32 : CEP_BF16, p * a.ld_ys + c, n, o);
      }
    }
  }
  if (!a.dw) return;
#pragma unroll
  for (int j = 0; j < KM; ++j) {
    dot[j] = wave_sum(dot[j]);
    if (LANES > 64 && lane == 0) part[threadIdx.x >> 6][j] = dot[j];
  }
  if (LANES > 64) __syncthreads();
  if (at >= a.k) return;
  float sum = 0.f;
  if (LANES > 64) {
#pragma unroll
    for (int i = 0; i < LANES / 64; ++i) sum += part[i][at];
  } else {
#pragma unroll
    for (int j = 0; j < KM; ++j) sum = at == j ? dot[j] : sum;
  }
  a.dw[t * a.k + at] = my >= 0 ? sum : 0.f;
}

template <int KM, bool YS32>
void launch_unsort(const UnsortArgs &a, hipStream_t s) {
  // (a launch holds fewer than 2^32 threads in x)
  constexpr int64_t kMost = 1 << 22;
  const int64_t blocks = ((int64_t)a.rows * a.waves + 3) / 4;
  const dim3 grid((unsigned)std::min(blocks, kMost), (unsigned)((blocks + kMost - 1) / kMost));
  hipLaunchKernelGGL((k_unsort<KM, YS32>), grid, dim3(256), 0, s, a);
}
template <int KM, bool YS32>
void launch_grad(const UnsortArgs &a, hipStream_t s) {
  // A wave a row, or a workgroup: its waves each start anew for a token, which short rows
  // do not repay, and more of them are on the way with few tokens (8192 tokens of 6 rows,
  // us, wave and workgroup: of 256 values 18, 51; 512 22, 50; 1024 47, 60; 2048 102, 93;
  // 60 tokens: of 512 5.7, 6.4; 2048 13, 6.7)
  if (a.d <= 1024)
    hipLaunchKernelGGL((k_unsort_grad<64, KM, YS32>), dim3((a.rows + 3) / 4), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_unsort_grad<256, KM, YS32>), dim3(a.rows), dim3(256), 0, s, a);
}

const char *bad_desc(const cep_expert_unsort_desc *d) {
  if (!d) return "desc is NULL";
  if (d->rows < 0 || d->rows > kMaxOpRows) return "rows must be in 0..2^21";
  if (d->top_k < 1 || d->top_k > kMaxTopK) return "top_k must be in 1..16";
  if (d->d < 1 || d->d > kMaxDim) return "d must be in 1..32768";
  if (d->sorted_rows < 0) return "sorted_rows must be >= 0";
  if (!is_float_dtype(d->ys_dtype) || !is_float_dtype(d->res_dtype) || !is_float_dtype(d->y_dtype))
    return "types must be CEP_F32 or CEP_BF16";
  for (int64_t ld : {d->ld_ys, d->ld_res, d->ld_y})
    if (ld && ld < d->d) return "a row stride is shorter than a row";
  return nullptr;
}

UnsortArgs args_of(const cep_expert_unsort_desc *d) {
  UnsortArgs a{};
  a.ld_ys = d->ld_ys ? d->ld_ys : d->d;
  a.ld_res = d->ld_res ? d->ld_res : d->d;
  a.ld_y = d->ld_y ? d->ld_y : d->d;
  a.rows = d->rows, a.k = d->top_k, a.d = d->d, a.sorted = d->sorted_rows;
  a.ys_dtype = d->ys_dtype, a.res_dtype = d->res_dtype, a.y_dtype = d->y_dtype;
  a.waves = (d->d + 511) / 512;
  return a;
}

}  // namespace
}  // namespace cep

using namespace cep;

CEP_API int cep_expert_unsort(const cep_expert_unsort_desc *d, const void *ys, const int32_t *place,
                              const float *w, const void *residual, void *y, hipStream_t s) {
  const char *fn = "cep_expert_unsort";
  if (const char *why = bad_desc(d)) return refuse(CEP_EINVAL, "%s: %s", fn, why);
  if (d->rows == 0) return CEP_OK;
  if (!place || !y || (d->sorted_rows && !ys)) return refuse(CEP_EINVAL, "%s: NULL array", fn);
  if (!aligned(place, 4) || !aligned(w, 4) || !aligned(ys, dtype_bytes(d->ys_dtype)) ||
      !aligned(residual, dtype_bytes(d->res_dtype)) || !aligned(y, dtype_bytes(d->y_dtype)))
    return refuse(CEP_EINVAL, "%s: a pointer is not aligned to its type", fn);
  if (y == ys) return refuse(CEP_EINVAL, "%s: y overlaps ys", fn);
  UnsortArgs a = args_of(d);
  a.ys = ys, a.place = place, a.w = w, a.res = residual, a.y = y;
  auto *launch = a.k <= 8 ? launch_unsort<8, false> : launch_unsort<16, false>;
  if (a.ys_dtype == CEP_F32) launch = a.k <= 8 ? launch_unsort<8, true> : launch_unsort<16, true>;
  launch(a, s);
  return launched(fn);
}

CEP_API int cep_expert_unsort_backward(const cep_expert_unsort_desc *d, const void *dy,
                                       const void *ys, const int32_t *place, const float *w,
                                       void *dys, float *dw, hipStream_t s) {
  const char *fn = "cep_expert_unsort_backward";
  if (const char *why = bad_desc(d)) return refuse(CEP_EINVAL, "%s: %s", fn, why);
  if (d->rows == 0) return CEP_OK;
  if (!dy || !place || (!dys && !dw) || (dw && d->sorted_rows && !ys))
    return refuse(CEP_EINVAL, "%s: NULL array", fn);
  if (!aligned(place, 4) || !aligned(w, 4) || !aligned(dw, 4) ||
      !aligned(ys, dtype_bytes(d->ys_dtype)) || !aligned(dys, dtype_bytes(d->ys_dtype)) ||
      !aligned(dy, dtype_bytes(d->y_dtype)))
    return refuse(CEP_EINVAL, "%s: a pointer is not aligned to its type", fn);
  if (dys == dy) return refuse(CEP_EINVAL, "%s: dys overlaps dy", fn);
  UnsortArgs a = args_of(d);
  a.dy = dy, a.ys = ys, a.place = place, a.w = w, a.dys = dys, a.dw = dw;
  auto *launch = a.k <= 8 ? launch_grad<8, false> : launch_grad<16, false>;
  if (a.ys_dtype == CEP_F32) launch = a.k <= 8 ? launch_grad<8, true> : launch_grad<16, true>;
  launch(a, s);
  return launched(fn);
}
