// Tile of a bf16 product with float32 accumulation, C[m][n] = sum over k of
// A(m, k) B(k, n), shared by the dense gated feed-forward and the matrix product
// with an epilogue.  Internal to libcep.
#pragma once

#include "block_ops.h"
#include "gemm_common.h"

#include <algorithm>

namespace cep {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

struct TileArgs {
  const __bf16 *A, *B0, *B1;
  int64_t lda, ldb;
  int M, N, K;
  int segs;    // K segments: A advances by K columns, B0 then B1 (dx; h in two terms)
  int splits;  // K shares
};

__device__ inline float sigma(float g) { return 1.0f / (1.0f + __expf(-g)); }

__device__ inline void store_bf16(__bf16 *p, const f32x4 &v) {
  *(uint2 *)p = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
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

// A tile of 2 HALF x 2 HALF outputs from row m0 and column n0 (DUAL: HALF columns
// of each of two products over the same A), K in steps of 64, by WM x WN waves.
// out(m, n, v, w) takes the sums of four columns from n of row m, w those of the
// second product.  A has k or m contiguous (A_K), B k or n (B_K).
//
// STAGED: the sums go through LDS first, and out.load(m, n) and out.store(m, n, v, w,
// loaded, out.column(n)) take eight columns of a row, four rows' loads on the way at
// once: for an epilogue that reads a matrix of its own.
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
template <int HALF, int WM, int WN, bool A_K, bool B_K, bool DUAL, bool STAGED = false, class Out>
__device__ inline void dense_tile(const TileArgs &a, int m0, int n0, int share, uint8_t *lds,
                                  Out out) {
  constexpr int MF = HALF / 16 / WM, NF = HALF / 16 / WN;  // fragments of a wave in a half
  constexpr int HB = HALF * 128;                           // bytes of a half
  constexpr int STAGE = 2 * HB;                            // one operand's two halves
  constexpr int LOADS = HB / 1024 / (WM * WN);             // 1 KB loads of a wave of a half
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l15 = lane & 15, g4 = lane >> 4;
  const int wm = wave % WM, wn = wave / WM;

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

  if constexpr (STAGED) {
    static_assert(!DUAL, "one product");
    // half of the rows at a time: [HALF][2 HALF] float32, 16-byte chunk c of row r at c ^
    // (r % 16)
    constexpr int TN = 2 * HALF, PER = TN / 8, ROWS = WM * WN * 64 / PER;
    constexpr int AT_ONCE = HALF / ROWS < 4 ? HALF / ROWS : 4;
    auto at = [&](int r, int chunk) { return (f32x4 *)(lds + r * TN * 4 + ((chunk ^ (r & 15)) << 4)); };
    auto meet = [] {
      wait_lgkm0();
      asm volatile("s_barrier" ::: "memory");
    };
#pragma unroll
    for (int mh = 0; mh < 2; ++mh) {
      if (mh) meet();
#pragma unroll
      for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int nh = 0; nh < 2; ++nh)
#pragma unroll
          for (int j = 0; j < NF; ++j)
            *at((wm * MF + i) * 16 + l15, (nh * HALF + (wn * NF + j) * 16) / 4 + g4) = acc[mh][nh][i][j];
      meet();
      const int c8 = tid % PER, n = n0 + c8 * 8;
      if (n < a.N) {
        const auto column = out.column(n);
        for (int r0 = tid / PER; r0 < HALF; r0 += AT_ONCE * ROWS) {
          decltype(out.load(0, 0)) in[AT_ONCE];
#pragma unroll
          for (int u = 0; u < AT_ONCE; ++u) {
            const int64_t m = m0 + mh * HALF + r0 + u * ROWS;
            if (m < a.M) in[u] = out.load(m, n);
          }
#pragma unroll
          for (int u = 0; u < AT_ONCE; ++u) {
            const int r = r0 + u * ROWS;
            const int64_t m = m0 + mh * HALF + r;
            if (m < a.M) out.store(m, n, *at(r, 2 * c8), *at(r, 2 * c8 + 1), in[u], column);
          }
        }
      }
    }
  } else {
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
            out(m, n, acc[mh][nh][i][j], acc[mh][1][i][j]);
          }
      }
  }
}

// Tile and K shares of a product.
struct DensePlan {
  int tile;  // 0: 256 x 256, 1: 128 x 128 (of both products' columns)
  int splits;
  double us;  // estimated
};
constexpr int kTile[2] = {256, 128};

inline int64_t dense_tiles(int t, int M, int N) {
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
// tiles: of each kind, none 0; sums: outputs of a share; most: shares.
inline DensePlan plan_tiles(const int64_t tiles[2], int steps, double sums, int most) {
  DensePlan best{};
  for (int t = 0; t < 2; ++t) {
    for (int s = 1; s <= most; ++s) {
      if (s > 1 && (tiles[t] * s > 256 || steps / s < 6)) break;
      const int64_t items = tiles[t] * s, rest = items % 512;
      const double step = (double)steps / s;
      double us = t == 0 ? (double)((items + 255) / 256) * (12 + 1.4 * step)
                         : 3 + step * ((items > 512 ? 1.2 : 1.0) * (double)(items / 512) +
                                       (rest == 0     ? 0.0
                                        : rest <= 256 ? 0.55
                                                      : 0.85 + 0.15 * (double)(rest - 256) / 256));
      if (s > 1) us = (us + 4 + (double)s * sums * 4 / 9e6) / 0.9;
      if ((t == 0 && s == 1) || us < best.us) best = {t, s, us};
    }
  }
  return best;
}
inline DensePlan dense_plan(int M, int n, int K, bool dual) {
  const int N = dual ? 2 * n : n;
  const int64_t tiles[2] = {dense_tiles(0, M, N), dense_tiles(1, M, N)};
  return plan_tiles(tiles, K / 64, (double)M * N, 16);
}

// Estimated time, in us, of the tiles of n products in one launch, the longest
// first; steps: of 64 of K, with 2 for a tile's start and end and 3 for each
// ragged end of K.
inline double tiles_us(int t, int n, const int64_t *tiles, const double *steps) {
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

}  // namespace cep
