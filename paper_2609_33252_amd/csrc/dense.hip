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
  kSwiGlu,  // two products g, u: h = silu(g) u to out0 (what that rounds off to out1),
            // g and u to pre
  kGrad     // dh: with g, u from pre, [dg | du] to out0 and h to out1
};
constexpr bool is_dual(int epi) { return epi == kStore2 || epi == kSwiGlu; }

struct DenseArgs {
  const __bf16 *A, *B0, *B1;
  int64_t lda, ldb;
  int M, N, K;
  int segs;       // K segments: A advances by K columns, B0 then B1 (dx; h in two terms)
  __bf16 *out0, *out1;
  int64_t ldo;
  float *pre;     // [M][2][N]
  int splits;     // K shares; above one, their sums go to part
  float *part;    // [splits][M][N, or 2 N of two products]
};

__device__ inline float sigma(float g) { return 1.0f / (1.0f + __expf(-g)); }

__device__ inline void store_bf16(__bf16 *p, const f32x4 &v) {
  *(uint2 *)p = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
}

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

// p, the same in every lane, in scalar registers
__device__ inline const char *uniform(const char *p) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (const char *)((uint64_t)hi << 32 | lo);
}

// Items are dealt in eight contiguous pieces, one an XCD (to which workgroups go
// round-robin), so that an XCD's tiles share panels in its L2: those in piece x.
__device__ inline int piece_of(int items, int x) { return items / 8 + (x < items % 8); }

// The product in tiles of 2 HALF x 2 HALF outputs, K in steps of 64, by WM x WN
// waves.
//
// Each operand's 64-wide step is two halves of HALF rows (columns), loaded
// straight to LDS; the operands' halves meet in four quadrants, one phase
// each, in which a wave multiplies HALF/WM x HALF/WN outputs (16 matrix
// instructions in the larger tile).  Quadrants follow a snake (A0 B0, A0 B1,
// A1 B1, A1 B0, then B swapped in the next step), so that only one operand half
// changes from phase to phase.  Fragments are read at least half a phase ahead
// and spread over the phases; a phase also loads one half, three to five phases
// ahead of its use.  A barrier ends each phase: behind it, the loads the next
// phase reads have landed in every wave, and the halves read in the phase before
// have been consumed and may be refilled.  (The scheduling barriers keep the
// matrix instructions, and with them the waits for their fragments, on their
// side of the phase's end.)
//
// LDS layout of a half, in 16-byte chunks so that every fragment read spreads
// over all banks:
//   k contiguous: [row][64 k], chunk c of row r at c ^ (r / 2 % 8); a fragment
//     is one 16-byte read a lane
//   row contiguous: [64 k][row], chunk pair p (16 rows) of line k at p ^ f(k);
//     a fragment is two transposing 8-byte reads of four lines of k
//
// Measured (kernel alone, 256-wide): 8192 x 7168 x 2 x 2048 with SwiGLU 321 to 329
// us from machine to machine, 1.46 to 1.50 PFLOP/s, the matrix pipe busy 65 % of
// the time at 2.1 GHz.  Bound inside the CU: without the loads the pass is 15 %
// shorter, without the LDS reads 18 %, with neither 31 %, with every load an L2
// hit 4 %.
template <int HALF, int WM, int WN, bool A_K, bool B_K, int EPI>
__device__ inline void dense_tile(const DenseArgs &a, int x, int at, uint8_t *lds) {
  constexpr bool DUAL = is_dual(EPI);
  constexpr int MF = HALF / 16 / WM, NF = HALF / 16 / WN;  // fragments of a wave in a half
  constexpr int HB = HALF * 128;                           // bytes of a half
  constexpr int STAGE = 2 * HB;                            // one operand's two halves
  constexpr int LOADS = HB / 1024 / (WM * WN);             // 1 KB loads of a wave of a half
  constexpr int TN = DUAL ? HALF : 2 * HALF;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l15 = lane & 15, g4 = lane >> 4;
  const int wm = wave % WM, wn = wave / WM;
  const int n_tm = (a.M + 2 * HALF - 1) / (2 * HALF), n_tn = (a.N + TN - 1) / TN;
  // the items: the shares of a tile are separate ones, share by share
  const int items = n_tm * a.splits * n_tn;
  if (at >= piece_of(items, x)) return;
  int mt, nt;
  tile_of<kGroupM>(x * (items / 8) + min(x, items % 8) + at, n_tm * a.splits, n_tn, &mt, &nt);
  const int share = mt / n_tm;
  const int m0 = (mt - share * n_tm) * 2 * HALF, n0 = nt * TN;

  // ---- loads: lane offsets from a base that advances with k; rows and columns
  // past the end read the last ones
  auto f_of = [](int k) {
    return HALF == 128 ? (k & 3) | ((k >> 3) & 1) << 2 : ((k >> 1) & 1) | ((k >> 3) & 1) << 1;
  };
  // piece e of this wave's loads of a half; its line of k (row contiguous)
  auto line_of = [&](int piece) { return piece * (512 / HALF) + lane / (HALF / 8); };
  auto offset = [&](bool kc, int half, int piece, int at0, int end, int64_t ld) {
    if (kc) {
      const int r = piece * 8 + (lane >> 3);
      const int row = min(at0 + half * HALF + r, end - 1) - at0;
      return (uint32_t)(row * (int)ld * 2 + ((lane & 7) ^ ((r >> 1) & 7)) * 16);
    }
    const int k = line_of(piece), pos = lane % (HALF / 8);
    const int chunk = (((pos >> 1) ^ f_of(k)) << 1) | (pos & 1);
    const int col = min(at0 + half * HALF + chunk * 8, end - 8) - at0;
    return (uint32_t)(k * (int)ld * 2 + col * 2);
  };
  uint32_t offA[2][LOADS], offB[2][LOADS];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < LOADS; ++e) {
      offA[h][e] = offset(A_K, h, wave * LOADS + e, m0, a.M, a.lda);
      offB[h][e] = offset(B_K, DUAL ? 0 : h, wave * LOADS + e, n0, a.N, a.ldb);
    }
  const int full = a.K / 64;  // whole steps of a segment
  const int s0 = (int)((int64_t)full * a.segs * share / a.splits);
  const int S = (int)((int64_t)full * a.segs * (share + 1) / a.splits) - s0;  // this share's
  const char *baseA = (const char *)(a.A + (A_K ? m0 * a.lda : m0));
  const char *baseB0 = (const char *)(a.B0 + (B_K ? n0 * a.ldb : n0));
  const char *baseB1 = a.B1 ? (const char *)(a.B1 + (B_K ? n0 * a.ldb : n0)) : nullptr;
  const int64_t stepA = A_K ? 128 : 128 * a.lda, stepB = B_K ? 128 : 128 * a.ldb;
  auto ptrA = [&](int seg, int step) { return baseA + (int64_t)seg * a.K * 2 + step * stepA; };
  auto ptrB = [&](int half, int seg, int step) {
    return ((DUAL ? half : seg) ? baseB1 : baseB0) + step * stepB;
  };
  const uint32_t lds0 = lds_offset(lds);
  // piece e of half `which` (0 A0, 1 first B, 2 second B, 3 A1) of the share's
  // step s, whose parity is P; the first B half is half P
  auto issue = [&](int s, auto which, auto parity, int e) {
    constexpr int W = decltype(which)::value, P = decltype(parity)::value;
    constexpr bool IS_A = W == 0 || W == 3;
    constexpr int H = W == 0 ? 0 : W == 3 ? 1 : W == 1 ? P : 1 - P;
    const int from = s0 + min(s, S - 1);
    const int seg = from >= full ? 1 : 0, step = from - (seg ? full : 0);
    const char *src = uniform(IS_A ? ptrA(seg, step) : ptrB(H, seg, step));
    const uint32_t to = lds0 + (IS_A ? P : 2 + P) * STAGE + H * HB + wave * LOADS * 1024;
    dma16_s(src, IS_A ? offA[H][e] : offB[H][e], to + e * 1024);
  };
  auto issue_half = [&](int s, auto which, auto parity) {
#pragma unroll
    for (int e = 0; e < LOADS; ++e) issue(s, which, parity, e);
  };

  // ---- fragments
  // a lane's byte offsets in a half: k contiguous, of its chunk of each 32 of
  // k (a fragment of 16 rows further on: + 2 KB); row contiguous, of its piece
  // of each fragment (4 lines of k: + 4 lines)
  int ra[A_K ? 2 : MF], rb[B_K ? 2 : NF];
  auto place = [&](bool kc, int row0, int i) {
    if (kc) return (row0 + l15) * 128 + ((g4 + 4 * i) ^ (l15 >> 1)) * 16;
    const int k = g4 * 8 + (l15 >> 2);
    return k * HALF * 2 + (((row0 >> 4) + i) ^ f_of(k)) * 32 + (l15 & 3) * 8;
  };
#pragma unroll
  for (int i = 0; i < (A_K ? 2 : MF); ++i) ra[i] = place(A_K, wm * MF * 16, i);
#pragma unroll
  for (int i = 0; i < (B_K ? 2 : NF); ++i) rb[i] = 2 * STAGE + place(B_K, wn * NF * 16, i);
  auto read = [&](bool kc, const int *r, int base, int i, int ks) {
    if (kc) return *(const bf16x8 *)(lds + r[ks] + (base + i * 2048));
    union { bf16x8 v; bf16x4 h[2]; } o;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      o.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
          (__attribute__((address_space(3))) bf16x4 *)(lds + r[i] +
                                                        (base + (ks * 32 + h * 4) * HALF * 2)));
    return o.v;
  };
  // Fragments: of A three sets of a half's 32 of k, taken in turn by the pieces
  // A0 (first and second 32 of k), A1, A0 of the next step, ...; of B two halves.
  bf16x8 fa[3][MF], fb[2][NF][2];
  f32x4 acc[2][2][MF][NF] = {};
  auto read_a = [&](auto set, int half, int stage, int ks, int i) {
    fa[decltype(set)::value][i] = read(A_K, ra, stage * STAGE + half * HB, i, ks);
  };
  auto read_b = [&](auto half, int stage, int item) {  // item: fragment and 32 of k
    constexpr int H = decltype(half)::value;
    fb[H][item % NF][item / NF] = read(B_K, rb, stage * STAGE + H * HB, item % NF, item / NF);
  };
  // the products of one fragment of A in a quadrant
  auto mul = [&](auto mh, auto nh, auto set, int ks, int i) {
    constexpr int P = decltype(mh)::value, Q = decltype(nh)::value, Z = decltype(set)::value;
#pragma unroll
    for (int j = 0; j < NF; ++j)
      acc[P][Q][i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[Q][j][ks], fa[Z][i],
                                                                acc[P][Q][i][j], 0, 0, 0);
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using I2 = std::integral_constant<int, 2>;
  using I3 = std::integral_constant<int, 3>;
  auto sync = [&] { asm volatile("s_barrier" ::: "memory"); };
  // Halves are loaded in the order A0, first B, second B, A1 of each step;
  // phase n (four a step) loads half n + 7, and the phase after it reads up
  // to half n + 3 (n + 4 after a step's last phase).  Past the last step the
  // loads repeat it, unread, so that the count in flight stays the same.  TURN:
  // the step modulo 6, the period of the stages and the fragment sets.
  auto phase = [&](int t, auto phase_c, auto turn_c) {
    constexpr int Q = decltype(phase_c)::value, TURN = decltype(turn_c)::value, P = TURN % 2;
    using M = std::integral_constant<int, Q / 2>;
    using G = std::integral_constant<int, 1 - P>;  // this step's second B half, the next one's first
    using N = std::integral_constant<int, Q == 0 || Q == 3 ? P : 1 - P>;
    using Z0 = std::integral_constant<int, (TURN + Q / 2 * 2) % 3>;      // this half's sets
    using Z1 = std::integral_constant<int, (TURN + Q / 2 * 2 + 1) % 3>;
    using Z2 = std::integral_constant<int, (TURN + Q / 2 * 2 + 2) % 3>;  // the free one
    const int to = t + (Q == 0 ? 1 : 2);
    using W = std::integral_constant<int, (Q + 3) % 4>;
    using TO = std::integral_constant<int, Q == 0 ? 1 - P : P>;
    // The reads and loads are dealt out between the matrix instructions: at the
    // head of the phase they would hold up the instructions behind them for as
    // long as the LDS queue is full.
    constexpr int NG = 2 * MF, NB = 2 * NF;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      if (g < MF) mul(M{}, N{}, Z0{}, 0, g);
      else mul(M{}, N{}, Z1{}, 1, g - MF);
      if (Q == 0 || Q == 3) {
#pragma unroll
        for (int r = 0; r < NB; ++r)
          if (r * MF / NB == g) read_b(G{}, Q == 0 ? P : 1 - P, r);
        if (Q == 0 && g >= MF) read_a(Z2{}, 1, P, 0, g - MF);
        if (Q == 3 && g >= MF) read_a(Z0{}, 0, 1 - P, 1, g - MF);
      }
      if (Q == 1 && g % 2 == 1) read_a(Z0{}, 1, P, 1, g / 2);
      if (Q == 2 && g % 2 == 1) read_a(Z2{}, 0, 1 - P, 0, g / 2);
#pragma unroll
      for (int e = 0; e < LOADS; ++e)
        if ((2 * e + 1) * NG / (2 * LOADS) == g) issue(to, W{}, TO{}, e);
      __builtin_amdgcn_sched_barrier(0);
    }
    wait_vmcnt<(Q == 3 ? 3 : 4) * LOADS>();
    sync();
  };
  auto whole_step = [&](int t, auto turn) {
    phase(t, I0{}, turn);
    phase(t, I1{}, turn);
    phase(t, I2{}, turn);
    phase(t, I3{}, turn);
  };
  if (S > 0) {
    issue_half(0, I0{}, I0{});
    issue_half(0, I1{}, I0{});
    issue_half(0, I2{}, I0{});
    issue_half(0, I3{}, I0{});
    issue_half(1, I0{}, I1{});
    issue_half(1, I1{}, I1{});
    issue_half(1, I2{}, I1{});
    wait_vmcnt<5 * LOADS>();
    sync();
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      read_a(I0{}, 0, 0, 0, i);
      read_a(I1{}, 0, 0, 1, i);
    }
#pragma unroll
    for (int r = 0; r < 2 * NF; ++r) read_b(I0{}, 0, r);
    wait_vmcnt<3 * LOADS>();
    sync();
    for (int t = 0;;) {
      whole_step(t, I0{});
      if (++t == S) break;
      whole_step(t, I1{});
      if (++t == S) break;
      whole_step(t, I2{});
      if (++t == S) break;
      whole_step(t, I3{});
      if (++t == S) break;
      whole_step(t, std::integral_constant<int, 4>{});
      if (++t == S) break;
      whole_step(t, std::integral_constant<int, 5>{});
      if (++t == S) break;
    }
    wait_vmcnt<0>();
    sync();
  }
  if (a.K % 64 && share == a.splits - 1) {  // each segment's last, shorter step: zeros past K
    for (int seg = 0; seg < a.segs; ++seg) {
      auto piece_in = [&](bool kc, int piece, const char *src, int half) {
        const int r = piece * 8 + (lane >> 3);
        const int k = full * 64 + (kc ? ((lane & 7) ^ ((r >> 1) & 7)) * 8 : line_of(piece));
        const uint4 v = k < a.K ? *(const uint4 *)src : make_uint4(0u, 0u, 0u, 0u);
        *(uint4 *)(lds + half * HB + piece * 1024 + lane * 16) = v;
      };
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < LOADS; ++e) {
          piece_in(A_K, wave * LOADS + e, ptrA(seg, full) + offA[h][e], h);
          piece_in(B_K, wave * LOADS + e, ptrB(h, seg, full) + offB[h][e], 4 + h);
        }
      __syncthreads();
#pragma unroll
      for (int r = 0; r < 2 * NF; ++r) {
        read_b(I0{}, 0, r);
        read_b(I1{}, 0, r);
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int i = 0; i < MF; ++i) {
          read_a(I0{}, 0, 0, ks, i);
          read_a(I1{}, 1, 0, ks, i);
          mul(I0{}, I0{}, I0{}, ks, i);
          mul(I0{}, I1{}, I0{}, ks, i);
          mul(I1{}, I0{}, I1{}, ks, i);
          mul(I1{}, I1{}, I1{}, ks, i);
        }
      __syncthreads();
    }
  }

  // lane: row lane % 16 of a fragment, four columns from 4 (lane / 16)
#pragma unroll
  for (int mh = 0; mh < 2; ++mh)
#pragma unroll
    for (int i = 0; i < MF; ++i) {
      const int64_t m = m0 + mh * HALF + (wm * MF + i) * 16 + l15;
      if (m >= a.M) continue;
#pragma unroll
      for (int nh = 0; nh < (DUAL ? 1 : 2); ++nh)
#pragma unroll
        for (int j = 0; j < NF; ++j) {
          const int n = n0 + nh * HALF + (wn * NF + j) * 16 + g4 * 4;
          if (n >= a.N) continue;
          if (a.splits == 1) {
            finish<EPI>(a, m, n, acc[mh][nh][i][j], acc[mh][1][i][j]);
          } else {
            float *p = a.part + ((int64_t)share * a.M + m) * (DUAL ? 2 * a.N : a.N) + n;
            *(f32x4 *)p = acc[mh][nh][i][j];
            if (DUAL) *(f32x4 *)(p + a.N) = acc[mh][1][i][j];
          }
        }
    }
}

template <int HALF, int WM, int WN, bool A_K, bool B_K, int EPI>
__global__ __launch_bounds__(WM * WN * 64, 2) void k_dense(DenseArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[HALF * 1024];
  dense_tile<HALF, WM, WN, A_K, B_K, EPI>(a, blockIdx.x & 7, blockIdx.x >> 3, lds);
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
  if (which == 0) dense_tile<HALF, WM, WN, true, true, kStore>(a.dx, x, at, lds);
  if (which == 1) dense_tile<HALF, WM, WN, false, false, kStore2>(a.dwgu, x, at, lds);
  if (which == 2) dense_tile<HALF, WM, WN, false, false, kStore>(a.dwd, x, at, lds);
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

// Estimated time, in us, of the tiles of n products in one launch, the longest
// first; steps: of 64 of K, with 2 for a tile's start and end and 3 for each
// ragged end of K.
double tiles_us(int t, int n, const int64_t *tiles, const double *steps) {
  if (t == 0) {  // one a compute unit, on the one that is free first
    int order[3] = {0, 1, 2};
    std::sort(order, order + n, [&](int i, int j) { return steps[i] > steps[j]; });
    // units that are free at a time: a product splits one group at most
    struct { double at; int64_t units; } group[4] = {{0.0, 256}};
    int groups = 1;
    double whole = 0, end = 0;
    for (int o = 0; o < n; ++o) {
      const int i = order[o];
      const double us = 10 + 1.4 * steps[i];
      const int64_t rounds = std::max<int64_t>(tiles[i] / 256 - 64, 0);
      whole += (double)rounds * us;
      for (int64_t left = tiles[i] - rounds * 256; left > 0;) {
        auto *first = &group[0];
        for (int g = 1; g < groups; ++g)
          if (group[g].at < first->at) first = &group[g];
        if (left < first->units) {
          first->units -= left;
          group[groups++] = {first->at + us, left};
          end = std::max(end, first->at + us);
          left = 0;
        } else {
          left -= first->units;
          first->at += us;
          end = std::max(end, first->at);
        }
      }
    }
    return whole + end;
  }
  // two a unit share it, so that its work counts, and the last round's gaps
  int64_t all = 0;
  double work = 0, longest = 0, shortest = steps[0];
  for (int i = 0; i < n; ++i) {
    all += tiles[i];
    work += (double)tiles[i] * steps[i] / 512;
    longest = std::max(longest, steps[i]);
    shortest = std::min(shortest, steps[i]);
  }
  const double part = (double)(all % 512) / 512;
  const double last = part == 0 ? 0 : part <= 0.5 ? 0.5 : 0.85 + 0.3 * (part - 0.5);
  return 4 + std::max(0.55 * longest, work + shortest * (last - part) * (all < 512 ? 1.0 : 0.5));
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
