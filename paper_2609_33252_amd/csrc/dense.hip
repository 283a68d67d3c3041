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
#include "dense.h"
#include "gemm_common.h"

#include <algorithm>

namespace cep {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

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

// p, the same in every lane, in scalar registers
__device__ inline const char *uniform(const char *p) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (const char *)((uint64_t)hi << 32 | lo);
}

// The product in tiles of 2 HALF x 2 HALF, K in steps of 64, HALF / 16 waves.
//
// Each operand's 64-wide step is two halves of HALF rows (columns), loaded
// straight to LDS; the two operand halves meet in four quadrants, one phase
// each, in which a wave multiplies HALF/2 x 32 outputs (16 matrix
// instructions at HALF 128).  Quadrants follow a snake (A0 B0, A0 B1, A1 B1,
// A1 B0, then B swapped in the next step), so that only one operand half
// changes from phase to phase.  A half of A is read into the registers of the
// one before as soon as their last matrix instruction has issued, a half of B
// one phase ahead; a phase also loads one half, four to five phases ahead of
// its use.  A barrier ends each phase: behind it, the loads the next phase
// reads have landed in every wave, and the halves read in the phase before
// have been consumed and may be refilled.
//
// LDS layout of a half, in 16-byte chunks so that every fragment read spreads
// over all banks:
//   k contiguous: [row][64 k], chunk c of row r at c ^ (r / 2 % 8); a fragment
//     is one 16-byte read a lane
//   row contiguous: [64 k][row], chunk pair p (16 rows) of line k at p ^ f(k);
//     a fragment is two transposing 8-byte reads of four lines of k
// Measured (kernel alone): 8192 x 7168 x 2 x 2048 with SwiGLU 337 us, 1.43
// PFLOP/s; bound by the matrix cores' issue and the loads that miss L2.
template <int HALF, bool A_K, bool B_K, int EPI>
__global__ __launch_bounds__(HALF * 4, 2) void k_dense(DenseArgs a) {
  constexpr bool DUAL = EPI == kStore2 || EPI == kSwiGlu;
  constexpr int MF = HALF / 32, NF = 2;   // fragments of a wave in a half
  constexpr int HB = HALF * 128;          // bytes of a half
  constexpr int STAGE = 4 * HB;           // A0, A1, B0, B1
  constexpr int TN = DUAL ? HALF : 2 * HALF;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l15 = lane & 15, g4 = lane >> 4;
  const int wm = wave & 1, wn = wave >> 1;
  const int n_tn = (a.N + TN - 1) / TN;
  int mt, nt;
  if (!work_item<kGroupM, false>(0, (a.M + 2 * HALF - 1) / (2 * HALF), n_tn, &mt, &nt)) return;
  const int m0 = mt * 2 * HALF, n0 = nt * TN;

  // ---- loads: per half two 1 KB pieces a wave, lane offsets from a base that
  // advances with k; rows and columns past the end read the last ones
  auto f_of = [](int k) {
    return HALF == 128 ? (k & 3) | ((k >> 3) & 1) << 2 : ((k >> 1) & 1) | ((k >> 3) & 1) << 1;
  };
  constexpr int LPR = HALF / 8;  // lanes of a line of the row-contiguous layout
  auto offset = [&](bool kc, int half, int e, int at0, int end, int64_t ld) -> uint32_t {
    const int piece = wave * 2 + e;
    if (kc) {
      const int r = piece * 8 + (lane >> 3);
      const int row = min(at0 + half * HALF + r, end - 1) - at0;
      return (uint32_t)(row * (int)ld * 2 + ((lane & 7) ^ ((r >> 1) & 7)) * 16);
    }
    const int k = piece * (64 / LPR) + lane / LPR, pos = lane % LPR;
    const int chunk = (((pos >> 1) ^ f_of(k)) << 1) | (pos & 1);
    const int col = min(at0 + half * HALF + chunk * 8, end - 8) - at0;
    return (uint32_t)(k * (int)ld * 2 + col * 2);
  };
  uint32_t offA[2][2], offB[2][2];
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      offA[h][e] = offset(A_K, h, e, m0, a.M, a.lda);
      offB[h][e] = offset(B_K, DUAL ? 0 : h, e, n0, a.N, a.ldb);
    }
  const int full = a.K / 64, S = full * a.segs;  // whole steps
  const char *baseA = (const char *)(a.A + (A_K ? m0 * a.lda : m0));
  const char *baseB0 = (const char *)(a.B0 + (B_K ? n0 * a.ldb : n0));
  const char *baseB1 = a.B1 ? (const char *)(a.B1 + (B_K ? n0 * a.ldb : n0)) : nullptr;
  const int64_t stepA = A_K ? 128 : 128 * a.lda, stepB = B_K ? 128 : 128 * a.ldb;
  auto ptrA = [&](int seg, int step) { return baseA + (int64_t)seg * a.K * 2 + step * stepA; };
  auto ptrB = [&](int half, int seg, int step) {
    return ((DUAL ? half : seg) ? baseB1 : baseB0) + step * stepB;
  };
  const uint32_t lds0 = lds_offset(lds) + wave * 2048;
  // half `which` (0 A0, 1 first B, 2 second B, 3 A1) of step s, whose parity
  // is P; the first B half is half P
  auto issue = [&](int s, auto which, auto parity) {
    constexpr int W = decltype(which)::value, P = decltype(parity)::value;
    constexpr bool IS_A = W == 0 || W == 3;
    constexpr int H = W == 0 ? 0 : W == 3 ? 1 : W == 1 ? P : 1 - P;
    const int from = min(s, S - 1);
    const int seg = from >= full ? 1 : 0, step = from - (seg ? full : 0);
    const char *src = uniform(IS_A ? ptrA(seg, step) : ptrB(H, seg, step));
#pragma unroll
    for (int e = 0; e < 2; ++e)
      dma16_s(src, IS_A ? offA[H][e] : offB[H][e],
              lds0 + P * STAGE + (IS_A ? H : 2 + H) * HB + e * 1024);
  };

  // ---- fragments
  // a lane's byte offsets in a half: k contiguous, of its chunk of each 32 of
  // k (a fragment of 16 rows further on: + 2 KB); row contiguous, of its piece
  // of each fragment (4 lines of k: + 4 lines)
  constexpr int LINE = HALF * 2;
  int ra[A_K ? 2 : MF], rb[B_K ? 2 : NF];
  auto place = [&](bool kc, int row0, int i) {
    if (kc) return (row0 + l15) * 128 + ((g4 + 4 * i) ^ (l15 >> 1)) * 16;
    const int k = g4 * 8 + (l15 >> 2);
    return k * LINE + (((row0 >> 4) + i) ^ f_of(k)) * 32 + (l15 & 3) * 8;
  };
#pragma unroll
  for (int i = 0; i < (A_K ? 2 : MF); ++i) ra[i] = place(A_K, wm * (HALF / 2), i);
#pragma unroll
  for (int i = 0; i < (B_K ? 2 : NF); ++i) rb[i] = place(B_K, wn * 32, i);
  auto read = [&](bool kc, const int *r, int base, int i, int ks) {
    if (kc) return *(const bf16x8 *)(lds + r[ks] + (base + i * 2048));
    union { bf16x8 v; bf16x4 h[2]; } o;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      o.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
          (__attribute__((address_space(3))) bf16x4 *)(lds + r[i] +
                                                        (base + (ks * 32 + h * 4) * LINE)));
    return o.v;
  };
  bf16x8 fa[MF][2], fb[2][NF][2];
  f32x4 acc[2][2][MF][NF] = {};
  auto read_a = [&](int half, int stage, int ks) {
#pragma unroll
    for (int i = 0; i < MF; ++i)
      fa[i][ks] = read(A_K, ra, stage * STAGE + half * HB, i, ks);
  };
  auto read_b = [&](auto half, int stage) {
    constexpr int H = decltype(half)::value;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int j = 0; j < NF; ++j)
        fb[H][j][ks] = read(B_K, rb, stage * STAGE + (2 + H) * HB, j, ks);
  };
  // half of a quadrant's products
  auto mul = [&](auto mh, auto nh, int ks) {
    constexpr int P = decltype(mh)::value, Q = decltype(nh)::value;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
      for (int j = 0; j < NF; ++j)
        acc[P][Q][i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[Q][j][ks], fa[i][ks],
                                                                  acc[P][Q][i][j], 0, 0, 0);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using I2 = std::integral_constant<int, 2>;
  using I3 = std::integral_constant<int, 3>;
  auto sync = [&] { asm volatile("s_barrier" ::: "memory"); };
  // Halves are loaded in the order A0, first B, second B, A1 of each step;
  // phase n (four a step) loads half n + 7, and the phase after it reads up
  // to half n + 3.  Past the last step the loads repeat it, unread, so that
  // the count in flight stays the same.
  auto phase = [&](int t, auto phase_c, auto parity_c) {
    constexpr int Q = decltype(phase_c)::value, P = decltype(parity_c)::value;
    using M = std::integral_constant<int, Q / 2>;
    using G = std::integral_constant<int, 1 - P>;  // this step's second B half, the next one's first
    using N = std::integral_constant<int, Q == 0 || Q == 3 ? P : 1 - P>;
    if (Q == 0) read_b(G{}, P);
    if (Q == 3) read_b(G{}, 1 - P);
    issue(t + (Q == 0 ? 1 : 2), std::integral_constant<int, (Q + 3) % 4>{},
          std::integral_constant<int, Q == 0 ? 1 - P : P>{});
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      mul(M{}, N{}, ks);
      if (Q == 1) read_a(1, P, ks);
      if (Q == 3) read_a(0, 1 - P, ks);
      __builtin_amdgcn_sched_barrier(0);
    }
    wait_vmcnt<8>();
    sync();
  };
  auto whole_step = [&](int t, auto parity) {
    phase(t, I0{}, parity);
    phase(t, I1{}, parity);
    phase(t, I2{}, parity);
    phase(t, I3{}, parity);
  };
  if (S > 0) {
    issue(0, I0{}, I0{});
    issue(0, I1{}, I0{});
    issue(0, I2{}, I0{});
    issue(0, I3{}, I0{});
    issue(1, I0{}, I1{});
    issue(1, I1{}, I1{});
    issue(1, I2{}, I1{});
    wait_vmcnt<10>();
    sync();
    read_a(0, 0, 0);
    read_a(0, 0, 1);
    read_b(I0{}, 0);
    wait_vmcnt<8>();
    sync();
    for (int t = 0;;) {
      whole_step(t, I0{});
      if (++t == S) break;
      whole_step(t, I1{});
      if (++t == S) break;
    }
    wait_vmcnt<0>();
    sync();
  }
  if (a.K % 64) {  // the last, shorter step of each segment, zeros past K
    for (int seg = 0; seg < a.segs; ++seg) {
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const bool is_a = h < 2;
        const bool kc = is_a ? A_K : B_K;
        const char *src = is_a ? ptrA(seg, full) : ptrB(h & 1, seg, full);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int piece = wave * 2 + e;
          const int r = piece * 8 + (lane >> 3);
          const int k = full * 64 + (kc ? ((lane & 7) ^ ((r >> 1) & 7)) * 8
                                        : piece * (64 / LPR) + lane / LPR);
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (k < a.K) v = *(const uint4 *)(src + (is_a ? offA[h & 1][e] : offB[h & 1][e]));
          *(uint4 *)(lds + h * HB + piece * 1024 + lane * 16) = v;
        }
      }
      __syncthreads();
      read_b(I0{}, 0);
      read_b(I1{}, 0);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        read_a(0, 0, ks);
        mul(I0{}, I0{}, ks);
        mul(I0{}, I1{}, ks);
        read_a(1, 0, ks);
        mul(I1{}, I0{}, ks);
        mul(I1{}, I1{}, ks);
      }
      __syncthreads();
    }
  }

  // lane: row lane % 16 of a fragment, four columns from 4 (lane / 16)
  auto store4 = [](__bf16 *p, const f32x4 &v) {
    *(uint2 *)p = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
  };
#pragma unroll
  for (int mh = 0; mh < 2; ++mh)
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      const int64_t m = m0 + mh * HALF + wm * (HALF / 2) + i * 16 + l15;
      if (m >= a.M) continue;
#pragma unroll
      for (int nh = 0; nh < (DUAL ? 1 : 2); ++nh)
#pragma unroll
        for (int j = 0; j < NF; ++j) {
          const int n = n0 + nh * HALF + wn * 32 + j * 16 + g4 * 4;
          if (n >= a.N) continue;
          const f32x4 v = acc[mh][nh][i][j];
          if (EPI == kStore) store4(a.out0 + m * a.ldo + n, v);
          if (EPI == kStore2) {
            store4(a.out0 + m * a.ldo + n, v);
            store4(a.out1 + m * a.ldo + n, acc[mh][1][i][j]);
          }
          if (EPI == kSwiGlu) {
            const f32x4 u = acc[mh][1][i][j];
            f32x4 h;
#pragma unroll
            for (int r = 0; r < 4; ++r) h[r] = v[r] * sigma(v[r]) * u[r];
            store4(a.out0 + m * a.ldo + n, h);
            if (a.pre) {
              *(f32x4 *)(a.pre + m * 2 * a.N + n) = v;
              *(f32x4 *)(a.pre + m * 2 * a.N + a.N + n) = u;
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
            store4(a.out0 + m * 2 * a.N + n, dg);
            store4(a.out0 + m * 2 * a.N + a.N + n, du);
            store4(a.out1 + m * a.N + n, h);
          }
        }
    }
}

template <bool A_K, bool B_K, int EPI>
void launch_dense(const DenseArgs &a, hipStream_t s) {
  constexpr bool DUAL = EPI == kStore2 || EPI == kSwiGlu;
  auto tiles = [&](int half) {
    const int tn = DUAL ? half : 2 * half;
    return (long long)((a.M + 2 * half - 1) / (2 * half)) * ((a.N + tn - 1) / tn);
  };
  // 256-wide tiles when they occupy most compute units, else 128-wide ones
  const bool large = tiles(128) >= 160;
  const dim3 grid((unsigned)((tiles(large ? 128 : 64) + 7) / 8 * 8));
  if (large)
    hipLaunchKernelGGL((k_dense<128, A_K, B_K, EPI>), grid, dim3(512), 0, s, a);
  else
    hipLaunchKernelGGL((k_dense<64, A_K, B_K, EPI>), grid, dim3(256), 0, s, a);
}

// a tile's offsets from its base stay below 2^31 bytes
constexpr int64_t kMaxStride = 1 << 21;

const char *bad_desc(const cep_gated_ffn_desc *d) {
  if (!d) return "desc is NULL";
  if (d->rows < 0 || d->rows > kMaxOpRows) return "rows must be in 0..2^24";
  for (int w : {d->d_model, d->d_ff})
    if (w < 8 || w > kMaxDim || w % 8) return "d_model and d_ff must be multiples of 8, up to 32768";
  for (int64_t ld : {d->ld_x, d->ld_y, d->ld_dx})
    if (ld && (ld < d->d_model || ld % 8 || ld > kMaxStride))
      return "row strides must be multiples of 8, at least d_model, at most 2^21";
  return nullptr;
}

}  // namespace
}  // namespace cep

using namespace cep;

CEP_API size_t cep_gated_ffn_workspace(const cep_gated_ffn_desc *d, int backward) {
  if (bad_desc(d)) return 0;
  // forward: h, or the row blocks' scratch; backward: [dg | du] and h
  const RowsPlan p = rows_plan(d->rows, d->d_model, d->d_ff);
  const size_t rows = p.use ? rows_workspace(p, d->rows, d->d_model, d->d_ff) : 0;
  return std::max<size_t>({(size_t)d->rows * d->d_ff * (backward ? 6 : 2), rows, 256});
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
