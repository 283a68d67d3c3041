// Dense gated feed-forward, y = (silu(x Wg) * (x Wu)) Wd, and its gradient, in
// bf16 with float32 accumulation, for gfx950.
//
//   g = x Wg, u = x Wu, h = silu(g) u, y = h Wd
//   dh = dy Wd^T, du = dh silu(g), dg = dh u sigma (1 + g (1 - sigma))
//   dx = dg Wg^T + du Wu^T, dWg = x^T dg, dWu = x^T du, dWd = h^T dy
//
// Six products of three layouts, C[m][n] = sum over k of A(m, k) B(k, n): A
// has k or m contiguous, B k or n.
#include "block_ops.h"

#include <algorithm>

namespace cep {
namespace {

typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// What happens to the accumulated tile.
enum Epilogue {
  kStore,   // bf16 to out0
  kStore2,  // two products over the same A: bf16 to out0 and out1
  kSwiGlu,  // two products g, u: h = silu(g) u to out0, g and u to pre
  kGrad     // dh: with g, u from pre, [dg | du] to out0 and h to out1
};

struct DenseArgs {
  const __bf16 *A, *B0, *B1;
  int64_t lda, ldb;
  int M, N, K;
  int segs;       // K segments: A advances by K columns, B0 then B1 (dx)
  __bf16 *out0, *out1;
  int64_t ldo;
  float *pre;     // [M][2][N]
};

__device__ inline float sigma(float g) { return 1.0f / (1.0f + __expf(-g)); }

template <bool A_K, bool B_K, int EPI>
__global__ __launch_bounds__(256) void k_dense(DenseArgs a) {
  constexpr bool DUAL = EPI == kStore2 || EPI == kSwiGlu;
  constexpr int NB = DUAL ? 2 : 1;
  __shared__ __bf16 As[64][40], Bs[NB][64][40];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  const int wm = (wave & 1) * 32, wn = (wave >> 1) * 32;
  f32x4 acc[NB][2][2] = {};
  for (int seg = 0; seg < a.segs; ++seg) {
    const __bf16 *A = a.A + (int64_t)seg * a.K;
    for (int k0 = 0; k0 < a.K; k0 += 32) {
      for (int i = tid; i < 64 * 32; i += 256) {
        const int r = A_K ? i / 32 : i % 64, k = A_K ? i % 32 : i / 64;
        const int m = m0 + r, kk = k0 + k;
        __bf16 v = (__bf16)0.f;
        if (m < a.M && kk < a.K) v = A_K ? A[m * a.lda + kk] : A[kk * a.lda + m];
        As[r][k] = v;
      }
      for (int b = 0; b < NB; ++b) {
        const __bf16 *B = (DUAL ? b : seg) ? a.B1 : a.B0;
        for (int i = tid; i < 64 * 32; i += 256) {
          const int c = B_K ? i / 32 : i % 64, k = B_K ? i % 32 : i / 64;
          const int n = n0 + c, kk = k0 + k;
          __bf16 v = (__bf16)0.f;
          if (n < a.N && kk < a.K) v = B_K ? B[n * a.ldb + kk] : B[kk * a.ldb + n];
          Bs[b][c][k] = v;
        }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const b16x8 fa = *(const b16x8 *)&As[wm + i * 16 + (lane & 15)][(lane >> 4) * 8];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const b16x8 fb = *(const b16x8 *)&Bs[b][wn + j * 16 + (lane & 15)][(lane >> 4) * 8];
            acc[b][i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb, fa, acc[b][i][j], 0, 0, 0);
          }
      }
      __syncthreads();
    }
  }
  // lane: row lane % 16 of a fragment, four columns from 4 (lane / 16)
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t m = m0 + wm + i * 16 + (lane & 15);
        const int n = n0 + wn + j * 16 + (lane >> 4) * 4 + r;
        if (m >= a.M || n >= a.N) continue;
        const float v = acc[0][i][j][r];
        if (EPI == kStore) a.out0[m * a.ldo + n] = (__bf16)v;
        if (EPI == kStore2) {
          a.out0[m * a.ldo + n] = (__bf16)v;
          a.out1[m * a.ldo + n] = (__bf16)acc[NB - 1][i][j][r];
        }
        if (EPI == kSwiGlu) {
          const float u = acc[NB - 1][i][j][r];
          a.out0[m * a.ldo + n] = (__bf16)(v * sigma(v) * u);
          if (a.pre) {
            a.pre[m * 2 * a.N + n] = v;
            a.pre[m * 2 * a.N + a.N + n] = u;
          }
        }
        if (EPI == kGrad) {
          const float g = a.pre[m * 2 * a.N + n], u = a.pre[m * 2 * a.N + a.N + n];
          const float s = sigma(g);
          a.out0[m * 2 * a.N + n] = (__bf16)(v * u * s * (1.0f + g * (1.0f - s)));
          a.out0[m * 2 * a.N + a.N + n] = (__bf16)(v * g * s);
          a.out1[m * a.N + n] = (__bf16)(g * s * u);
        }
      }
}

template <bool A_K, bool B_K, int EPI>
void launch_dense(const DenseArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((k_dense<A_K, B_K, EPI>), dim3((a.N + 63) / 64, (a.M + 63) / 64), dim3(256),
                     0, s, a);
}

const char *bad_desc(const cep_gated_ffn_desc *d) {
  if (!d) return "desc is NULL";
  if (d->rows < 0 || d->rows > kMaxOpRows) return "rows must be in 0..2^24";
  for (int w : {d->d_model, d->d_ff})
    if (w < 8 || w > kMaxDim || w % 8) return "d_model and d_ff must be multiples of 8, up to 32768";
  for (int64_t ld : {d->ld_x, d->ld_y, d->ld_dx})
    if (ld && (ld < d->d_model || ld % 8))
      return "row strides must be multiples of 8 and at least d_model";
  return nullptr;
}

}  // namespace
}  // namespace cep

using namespace cep;

CEP_API size_t cep_gated_ffn_workspace(const cep_gated_ffn_desc *d, int backward) {
  if (bad_desc(d)) return 0;
  // forward: h; backward: [dg | du] and h
  return std::max<size_t>((size_t)d->rows * d->d_ff * (backward ? 6 : 2), 256);
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
  DenseArgs a{};
  a.A = (const __bf16 *)x;
  a.B0 = (const __bf16 *)w_gate;
  a.B1 = (const __bf16 *)w_up;
  a.lda = d->ld_x ? d->ld_x : D;
  a.ldb = I;
  a.M = T, a.N = I, a.K = D, a.segs = 1;
  a.out0 = (__bf16 *)workspace;
  a.ldo = I;
  a.pre = preact;
  launch_dense<true, false, kSwiGlu>(a, s);
  DenseArgs b{};
  b.A = (const __bf16 *)workspace;
  b.B0 = (const __bf16 *)w_down;
  b.lda = I, b.ldb = D;
  b.M = T, b.N = D, b.K = I, b.segs = 1;
  b.out0 = (__bf16 *)y;
  b.ldo = d->ld_y ? d->ld_y : D;
  launch_dense<true, false, kStore>(b, s);
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
  if (T) {
    DenseArgs a{};  // dh, and from it dg, du and h
    a.A = (const __bf16 *)dy;
    a.B0 = (const __bf16 *)w_down;
    a.lda = ld_y, a.ldb = D;
    a.M = T, a.N = I, a.K = D, a.segs = 1;
    a.out0 = dgu, a.out1 = h;
    a.pre = const_cast<float *>(preact);
    launch_dense<true, true, kGrad>(a, s);
    DenseArgs b{};  // dx
    b.A = dgu;
    b.B0 = (const __bf16 *)w_gate;
    b.B1 = (const __bf16 *)w_up;
    b.lda = 2 * I, b.ldb = I;
    b.M = T, b.N = D, b.K = I, b.segs = 2;
    b.out0 = (__bf16 *)dx;
    b.ldo = d->ld_dx ? d->ld_dx : D;
    launch_dense<true, true, kStore>(b, s);
  }
  DenseArgs c{};  // dWg, dWu
  c.A = (const __bf16 *)x;
  c.B0 = dgu;
  c.B1 = dgu + I;
  c.lda = ld_x, c.ldb = 2 * I;
  c.M = D, c.N = I, c.K = T, c.segs = 1;
  c.out0 = (__bf16 *)dw_gate, c.out1 = (__bf16 *)dw_up;
  c.ldo = I;
  launch_dense<false, false, kStore2>(c, s);
  DenseArgs e{};  // dWd
  e.A = h;
  e.B0 = (const __bf16 *)dy;
  e.lda = I, e.ldb = ld_y;
  e.M = I, e.N = D, e.K = T, e.segs = 1;
  e.out0 = (__bf16 *)dw_down;
  e.ldo = D;
  launch_dense<false, false, kStore>(e, s);
  return launched(fn);
}
