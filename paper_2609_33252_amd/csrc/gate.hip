// Choice of each token's experts from the gate's logits, and their routing
// coefficients, for gfx950.
//
// A row's keys are the logits (softmax) or sigmoid(logit) + bias; the k
// largest keys win, the lowest expert on ties, experts whose logit is -inf or
// NaN never.  With groups, only the experts of the topk_groups groups with the
// largest sum of their two best keys take part.
//
// A handful of lanes share a row.  Each lane sorts its keys in registers, and
// a round of the choice is a maximum over the lanes' heads.  A key and its
// expert travel as one double: the key's float32 bits are the high word (every
// number and -inf is then a finite double of the same order) and the expert
// the low word, so that one v_max_f64 compares both.
//
// Measured: 65536 rows of 160 logits, k 8, softmax 11.5 us, 4 TB/s, bound by
// the sorts' instructions; 9 rows of 256 in eight groups, sigmoid, 4.2 us, where
// an empty launch takes 3.5 to 4.
#include "block_ops.h"

#include <cfloat>
#include <type_traits>

namespace cep {
namespace {

constexpr int kMaxGateExperts = 1024;
constexpr int kMaxGroups = 64;

struct GateArgs {
  const void *logits;
  const float *bias;
  int32_t *ids;
  float *w;
  int64_t ld;
  int rows, E, k, dtype, sigmoid, groups, topg, normalize;
  float scale;
};

__device__ inline double dmax(double a, double b) {
  double r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ inline double dmin(double a, double b) {
  double r;
  asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}

// Larger for a larger key, and among equal keys for the lower expert: a
// double's low word adds to the magnitude, so a negative key takes the expert
// itself.  key + 0 makes -0 and +0 one key.
__device__ inline double pack_key(float key, int expert) {
  const uint32_t hi = __float_as_uint(key + 0.0f);
  return __hiloint2double((int)hi, (hi >> 31) ? expert : ~expert);
}
__device__ inline float key_of(double p) { return __int_as_float(__double2hiint(p)); }
__device__ inline int expert_of(double p) {
  const int lo = __double2loint(p);
  return __double2hiint(p) < 0 ? lo : ~lo;
}

// Maximum over the LPR lanes of a row, in each of them.
template <int CTRL>
__device__ inline double dpp_max(double v) {
  const int lo = __builtin_amdgcn_mov_dpp(__double2loint(v), CTRL, 0xf, 0xf, false);
  const int hi = __builtin_amdgcn_mov_dpp(__double2hiint(v), CTRL, 0xf, 0xf, false);
  return dmax(v, __hiloint2double(hi, lo));
}
template <int LPR>
__device__ inline double row_max(double v) {
  v = dpp_max<0xB1>(v);   // lanes 1 0 3 2
  v = dpp_max<0x4E>(v);   // lanes 2 3 0 1
  v = dpp_max<0x141>(v);  // half row mirrored: lane 7 - i
  if (LPR == 64) {
    v = dpp_max<0x140>(v);  // row mirrored: lane 15 - i
    v = dmax(v, __shfl_xor(v, 16));
    v = dmax(v, __shfl_xor(v, 32));
  }
  return v;
}
// The two largest of eight lanes' pairs best >= second, in each of them.
template <int CTRL>
__device__ inline void dpp_top2(float *best, float *second) {
  const float b = __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(*best), CTRL, 0xf, 0xf, false));
  const float s = __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(*second), CTRL, 0xf, 0xf, false));
  *second = fmaxf(fminf(*best, b), fmaxf(*second, s));
  *best = fmaxf(*best, b);
}
__device__ inline void lanes_top2(float *best, float *second) {
  dpp_top2<0xB1>(best, second);
  dpp_top2<0x4E>(best, second);
  dpp_top2<0x141>(best, second);
}
template <int LPR>
__device__ inline float row_add(float v) {
#pragma unroll
  for (int o = 1; o < LPR; o <<= 1) v += __shfl_xor(v, o);
  return v;
}

// Merge-exchange sort (Batcher), descending, of N register values.
template <int N>
__device__ inline void sort_desc(double (&v)[N]) {
  constexpr int T = N <= 8 ? 3 : N <= 16 ? 4 : 5;
#pragma unroll
  for (int pi = T - 1; pi >= 0; --pi) {
#pragma unroll
    for (int pass = 0; pass < T - pi; ++pass) {
      const int p = 1 << pi, d = pass == 0 ? p : (1 << (T - pass)) - p, r = pass == 0 ? 0 : p;
#pragma unroll
      for (int i = 0; i < N - d; ++i)
        if ((i & p) == r) {
          const double a = v[i], b = v[i + d];
          v[i] = dmax(a, b);
          v[i + d] = dmin(a, b);
        }
    }
  }
}

// NaN: as masked; +inf: the largest number
__device__ inline float unmasked(float l) { return l != l ? -INFINITY : fminf(l, FLT_MAX); }
__device__ inline float logit(const GateArgs &a, int64_t row, int e) {
  return unmasked(a.dtype == CEP_BF16 ? (float)((const __bf16 *)a.logits)[row * a.ld + e]
                                      : ((const float *)a.logits)[row * a.ld + e]);
}
// 1 / (1 + 2^t), t = -l log2(e), with t's rounding error r put back as 2^r ~ 1 +
// r ln(2): the exponential and reciprocal instructions are within one unit of
// the last place.  Past 2^125, where the reciprocal would be subnormal, both are
// taken of 2^(t - 64) (an exact difference, beside which the 1 is nothing), and
// the last factor keeps the steps of subnormal numbers: experts are told apart
// down to where float32 has no smaller score (a logit of -104).
__device__ inline float sigmoid(float l) {
  constexpr float kLog2e = 1.44269502f, kLog2eRest = 1.92596303e-8f;
  const float c = fminf(fmaxf(-l, -90.0f), 105.0f), t = c * kLog2e;
  const float r = fmaf(c, kLog2eRest, fmaf(c, kLog2e, -t));
  const bool far = t > 125.0f;
  const float q = __builtin_amdgcn_exp2f(t - (far ? 64.0f : 0.0f)) * fmaf(r, 0.693147182f, 1.0f);
  return __builtin_amdgcn_rcpf(1.0f + q) * (far ? 0x1p-64f : 1.0f);
}

// How groups are found: none; any size, through LDS; 32 experts, in eight lanes'
// registers.
enum Groups { kNoGroups, kAnyGroups, kGroupsOf32 };

// LPR lanes a row, V experts a lane (V a multiple of 4: chunk j of a lane is
// the four experts from (j * LPR + lane) * 4), at most KM chosen.
template <int LPR, int V, int KM, bool SIGMOID, Groups GROUPS>
__global__ __launch_bounds__(256) void k_gate(GateArgs a) {
  constexpr int ROWS = 256 / LPR;  // rows of a block
  const int lane = threadIdx.x % LPR, sub = threadIdx.x / LPR;
  const int64_t row0 = (int64_t)blockIdx.x * ROWS + sub;
  const bool live = row0 < a.rows;
  const int64_t row = live ? row0 : a.rows - 1;
  float key[V];
#pragma unroll
  for (int j = 0; j < V / 4; ++j) {
    const int e0 = (j * LPR + lane) * 4;
    Vec16 l = {}, b = {};
    if (e0 + 4 <= a.E) {
      if (a.dtype == CEP_F32) {
        l = *(const Any16 *)((const float *)a.logits + row * a.ld + e0);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          l[i] = (uint32_t)((const uint16_t *)a.logits)[row * a.ld + e0 + i] << 16;
      }
      if (SIGMOID && a.bias) b = *(const Any16 *)(a.bias + e0);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        l[i] = __float_as_uint(e0 + i < a.E ? logit(a, row, e0 + i) : -INFINITY);
        if (SIGMOID && a.bias && e0 + i < a.E) b[i] = __float_as_uint(a.bias[e0 + i]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v = unmasked(__uint_as_float(l[i]));
      float q = v;
      if (SIGMOID) {
        q = sigmoid(v) + __uint_as_float(b[i]);
        if (v == -INFINITY || q != q) q = -INFINITY;
      }
      key[4 * j + i] = q;
    }
  }
  if constexpr (GROUPS == kGroupsOf32) {
    // a chunk of 32 experts is a group: chunk j of the row's eight lanes, or (a
    // wave a row, one chunk) of the eight lanes around this one
    static_assert(LPR == 8 || V == 4, "one chunk a lane");
    float total[V / 4];
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      const float *v = key + 4 * j;
      const float lo = fminf(v[0], v[1]), hi = fminf(v[2], v[3]);
      const float a0 = fmaxf(v[0], v[1]), a1 = fmaxf(v[2], v[3]);
      float best = fmaxf(a0, a1), second = fmaxf(fminf(a0, a1), fmaxf(lo, hi));
      lanes_top2(&best, &second);
      total[j] = second > -INFINITY ? best + second : best;
    }
    // the groups past the last have nothing and come last
    if (LPR == 8) {
      float own = -INFINITY;  // group `lane`
#pragma unroll
      for (int c = 0; c < V / 4; ++c) own = lane == c ? total[c] : own;
      int rank = 0;
#pragma unroll
      for (int c = 0; c < V / 4; ++c) rank += total[c] > own || (total[c] == own && c < lane);
      const uint64_t keep = __ballot(rank < a.topg) >> (threadIdx.x & 56);
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (!((keep >> (j / 4)) & 1)) key[j] = -INFINITY;
    } else {
      int rank = 0;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float t = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(total[0]), 8 * c));
        rank += t > total[0] || (t == total[0] && c < lane / 8);
      }
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (rank >= a.topg) key[j] = -INFINITY;
    }
  }
  if constexpr (GROUPS == kAnyGroups) {
    // rows 8 words apart modulo the banks, and one word between groups, so that
    // the lanes of a wave, at the same place of their groups, read 64 banks
    __shared__ float keys[ROWS][LPR * V + kMaxGroups + 8];
    __shared__ float total[ROWS][kMaxGroups + 1];
    const int per = a.E / a.groups;
    const float inv = 1.0f / (float)per;
    // e / per: exact, the quotient of e + 1/2 lies 1 / (2 per) off a whole number
    auto group_of = [&](int e) { return (int)(((float)e + 0.5f) * inv); };
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int e = (j / 4 * LPR + lane) * 4 + j % 4;
      if (e < a.E) keys[sub][e + group_of(e)] = key[j];
    }
    __syncthreads();
    for (int g = lane; g < a.groups; g += LPR) {
      float best = -INFINITY, second = -INFINITY;
#pragma unroll 8
      for (int e = g * per; e < (g + 1) * per; ++e) {
        const float v = keys[sub][e + g];
        second = fmaxf(second, fminf(best, v));
        best = fmaxf(best, v);
      }
      // a group's only expert counts alone
      total[sub][g] = second > -INFINITY ? best + second : best;
    }
    __syncthreads();
    uint64_t keep = 0;  // this row's kept groups
    for (int g = lane; g < a.groups; g += LPR) {
      const float v = total[sub][g];
      int rank = 0;
#pragma unroll 8
      for (int h = 0; h < a.groups; ++h) rank += total[sub][h] > v || (total[sub][h] == v && h < g);
      keep |= (uint64_t)(rank < a.topg) << g;
    }
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) keep |= __shfl_xor((unsigned long long)keep, o);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int e = (j / 4 * LPR + lane) * 4 + j % 4;
      if (e < a.E && !((keep >> group_of(e)) & 1)) key[j] = -INFINITY;
    }
  }
  double s[V];
#pragma unroll
  for (int j = 0; j < V; ++j) s[j] = pack_key(key[j], (j / 4 * LPR + lane) * 4 + j % 4);
  sort_desc(s);
  // the choice of round r is kept by lane r % LPR
  constexpr int OWN = (KM + LPR - 1) / LPR;
  double mine[OWN];
#pragma unroll
  for (int i = 0; i < OWN; ++i) mine[i] = pack_key(-INFINITY, 0);
  float top = -INFINITY;
#pragma unroll
  for (int r = 0; r < KM; ++r) {
    if (r < a.k) {
      const double best = row_max<LPR>(s[0]);
      if (r == 0) top = key_of(best);
      if (lane == r % LPR) mine[r / LPR] = best;
      const bool won = s[0] == best;
#pragma unroll
      for (int i = 0; i + 1 < V && i < KM - 1 - r; ++i) s[i] = won ? s[i + 1] : s[i];
      if (V - 1 < KM - 1 - r) s[V - 1] = won ? pack_key(-INFINITY, 0) : s[V - 1];
    }
  }
  // coefficients: the scores of the chosen, over their sum or (softmax) over
  // every expert's
  float w[OWN], sum = 0.f;
#pragma unroll
  for (int i = 0; i < OWN; ++i) {
    const int r = i * LPR + lane;
    const bool some = r < a.k && key_of(mine[i]) > -INFINITY;
    w[i] = 0.f;
    if (some) w[i] = SIGMOID ? sigmoid(logit(a, row, expert_of(mine[i]))) : expf(key_of(mine[i]) - top);
    sum += w[i];
  }
  if (!SIGMOID && !a.normalize) {
    sum = 0.f;
    for (int e = lane; e < a.E; e += LPR) {
      const float l = logit(a, row, e);
      if (l > -INFINITY) sum += expf(l - top);
    }
  }
  sum = row_add<LPR>(sum);
  const bool over = a.normalize || !SIGMOID;
#pragma unroll
  for (int i = 0; i < OWN; ++i) {
    const int r = i * LPR + lane;
    if (!live || r >= a.k) continue;
    const bool some = key_of(mine[i]) > -INFINITY;
    a.ids[row * a.k + r] = some ? expert_of(mine[i]) : -1;
    a.w[row * a.k + r] = over ? (sum > 0.f ? w[i] / sum * a.scale : 0.f) : w[i] * a.scale;
  }
}

template <int LPR, int V, int KM>
void launch_gate(const GateArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)a.rows * LPR + 255) / 256));
  auto *k = !a.sigmoid ? k_gate<LPR, V, KM, false, kNoGroups>
            : a.groups > 1 ? k_gate<LPR, V, KM, true, kAnyGroups>
                           : k_gate<LPR, V, KM, true, kNoGroups>;
  if constexpr (LPR == 8 || V == 4)
    if (a.groups > 1 && a.E == 32 * a.groups) k = k_gate<LPR, V, KM, true, kGroupsOf32>;
  hipLaunchKernelGGL(k, grid, dim3(256), 0, s, a);
}

// Few rows: a wave a row, four experts a lane, for the latency of one row;
// more rows: eight lanes a row, which takes fewer instructions a row.  256
// experts, k 8, us a call of 64 / 2048 / 4096 / 65536 rows: softmax 4.0 / 4.2 /
// 5.3 / 43 with a wave, 4.0 / 4.3 / 4.4 / 16.4 with eight lanes; sigmoid in
// eight groups of 32 4.4 / 5.1 / 6.8 / 58 and 5.8 / 6.1 / 6.1 / 26; 96 in
// four of 24, through LDS, 6.6 / 6.5 / 8.4 / 72 and 7.9 / 8.3 / 8.4 / 31.
// (Groups of 32 through LDS, as those of any size are: 38 us for 65536 rows with
// eight lanes, 24 so at the time.)  129 to 160 experts have 20 a lane: 65536 rows
// of 160 11.8 us, 15.4 with 32 a lane; sigmoid 15.2, 21.4.  Above 256 every row
// takes a wave: 65536 rows of 384 81 us, of 1024 152, where their bytes take 20
// and 55.
template <int KM>
void launch_by_experts(const GateArgs &a, hipStream_t s) {
  if (a.E <= 256 && a.rows <= (a.groups > 1 && a.E != 32 * a.groups ? 4096 : 2048)) launch_gate<64, 4, KM>(a, s);
  else if (a.E <= 64) launch_gate<8, 8, KM>(a, s);
  else if (a.E <= 128) launch_gate<8, 16, KM>(a, s);
  else if (a.E <= 160) launch_gate<8, 20, KM>(a, s);
  else if (a.E <= 256) launch_gate<8, 32, KM>(a, s);
  else if (a.E <= 512) launch_gate<64, 8, KM>(a, s);
  else launch_gate<64, 16, KM>(a, s);
}

}  // namespace
}  // namespace cep

using namespace cep;

CEP_API int cep_gate_topk(const cep_gate_desc *g, const void *logits, const float *bias,
                          int32_t *topk_id, float *topk_w, hipStream_t s) {
  const char *fn = "cep_gate_topk";
  if (!g) return refuse(CEP_EINVAL, "%s: desc is NULL", fn);
  if (g->rows < 0 || g->rows > kMaxOpRows) return refuse(CEP_EINVAL, "%s: rows must be in 0..2^21", fn);
  if (g->n_experts < 1 || g->n_experts > kMaxGateExperts)
    return refuse(CEP_EINVAL, "%s: n_experts must be in 1..1024", fn);
  if (g->top_k < 1 || g->top_k > kMaxTopK || g->top_k > g->n_experts)
    return refuse(CEP_EINVAL, "%s: top_k must be in 1..16 and at most n_experts", fn);
  if (!is_float_dtype(g->logit_dtype))
    return refuse(CEP_EINVAL, "%s: logit_dtype must be CEP_F32 or CEP_BF16", fn);
  if (g->score != CEP_SOFTMAX && g->score != CEP_SIGMOID)
    return refuse(CEP_EINVAL, "%s: unknown score %d", fn, g->score);
  const int groups = g->n_groups ? g->n_groups : 1;
  const int topg = g->n_groups ? g->topk_groups : 1;
  if (groups < 1 || groups > kMaxGroups || g->n_experts % groups || topg < 1 || topg > groups)
    return refuse(CEP_EINVAL, "%s: n_groups (up to 64) must divide n_experts, topk_groups be in "
                  "1..n_groups", fn);
  if (g->score == CEP_SOFTMAX && (bias || groups > 1))
    return refuse(CEP_EINVAL, "%s: a bias and groups go with CEP_SIGMOID", fn);
  if (g->ld && g->ld < g->n_experts) return refuse(CEP_EINVAL, "%s: ld is shorter than a row", fn);
  if (!(g->scale == g->scale)) return refuse(CEP_EINVAL, "%s: scale is NaN", fn);
  if (g->rows == 0) return CEP_OK;
  if (!logits || !topk_id || !topk_w) return refuse(CEP_EINVAL, "%s: NULL array", fn);
  if (!aligned(logits, dtype_bytes(g->logit_dtype)) || !aligned(bias, 4) || !aligned(topk_id, 4) ||
      !aligned(topk_w, 4))
    return refuse(CEP_EINVAL, "%s: a pointer is not aligned to its type", fn);
  const GateArgs a{logits, bias, topk_id, topk_w, g->ld ? g->ld : g->n_experts, g->rows,
                   g->n_experts, g->top_k, g->logit_dtype, g->score == CEP_SIGMOID, groups, topg,
                   g->normalize != 0, g->scale};
  if (g->top_k <= 8) launch_by_experts<8>(a, s);
  else launch_by_experts<16>(a, s);
  return launched(fn);
}
