// Packing of routed tokens into one send buffer, expert-parallel rank by rank,
// for gfx950 (Appendix C, "Asynchronous dispatch": a source lane's rows travel
// to the rank that holds their experts).
//
// The tokens of a rank keep their order.  A token's place in a rank's segment
// is the number of earlier tokens that go there too: k_send_count writes it
// per tile of tokens and block, k_send adds the blocks before it, and copies
// each row once from memory to all of its places.  Bound by HBM: every row is
// read once and written once per rank it goes to.
#include "block_ops.h"

#include <algorithm>

namespace cep {
namespace {

constexpr int kMaxRanks = 64;     // one lane each
constexpr int kCountTokens = 256;  // tokens of a k_send_count block (one wave)
constexpr int kSendTokens = 16;    // tokens of a k_send block (a tile)
constexpr int kTiles = kCountTokens / kSendTokens;

struct SendArgs {
  const int32_t *ids;  // [rows][k]
  const float *w;      // [rows][k]
  const char *x;
  int64_t ld_x;
  int32_t *plan;  // [R + 1] segment offsets, [R] pairs, [1] ids out of range
  int32_t *token;
  int32_t *out_id;
  float *out_w;
  char *out_x;
  // tile_at [tiles][R]: earlier tokens of the tile's block that go to a rank;
  // tot, pairs [blocks][R]; bad [blocks]
  int32_t *tile_at, *tot, *pairs, *bad;
  int rows, k, R, per, blocks, capacity;
  int64_t row_bytes;
};

// The ranks (a bit each) that hold the token's experts; *bad counts ids that
// no rank has, apart from -1 (no expert).
__device__ inline uint64_t ranks_of(const SendArgs &a, int64_t t, int *bad) {
  uint64_t m = 0;
  for (int j = 0; j < a.k; ++j) {
    const int id = a.ids[t * a.k + j];
    if (id >= 0 && id < a.R * a.per) m |= 1ull << (id / a.per);
    else if (id != -1) ++*bad;
  }
  return m;
}

// Wave: the tokens [256 b, 256 b + 256), 64 at a time.  Lane r keeps rank r's
// count.
__device__ inline void count_block(const SendArgs &a, int b, int32_t *tile_at, int32_t *tot,
                                   int32_t *pairs, int32_t *bad_out, int32_t *lds_pairs) {
  const int lane = threadIdx.x & 63;
  lds_pairs[lane] = 0;
  int run = 0, bad = 0;
  for (int q = 0; q < kCountTokens / 64; ++q) {
    const int64_t t = (int64_t)b * kCountTokens + q * 64 + lane;
    uint64_t m = 0;
    if (t < a.rows) {
      m = ranks_of(a, t, &bad);
      for (int j = 0; j < a.k; ++j) {
        const int id = a.ids[t * a.k + j];
        if (id >= 0 && id < a.R * a.per) atomicAdd(&lds_pairs[id / a.per], 1);
      }
    }
    uint64_t there = 0;  // of rank `lane`: the round's tokens that go there
    for (int r = 0; r < a.R; ++r) {
      const uint64_t v = __ballot((m >> r) & 1);
      if (lane == r) there = v;
    }
    if (lane < a.R) {
#pragma unroll
      for (int i = 0; i < 64 / kSendTokens; ++i)
        tile_at[(q * (64 / kSendTokens) + i) * a.R + lane] =
            run + (int)__popcll(there & ((1ull << (i * kSendTokens)) - 1));
    }
    run += (int)__popcll(there);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) bad += __shfl_xor(bad, o);
  if (lane < a.R) {
    tot[lane] = run;
    pairs[lane] = lds_pairs[lane];
  }
  if (lane == 0) *bad_out = bad;
}

__global__ __launch_bounds__(64) void k_send_count(SendArgs a) {
  __shared__ int32_t lds_pairs[64];
  const size_t b = blockIdx.x;
  count_block(a, b, a.tile_at + b * kTiles * a.R, a.tot + b * a.R, a.pairs + b * a.R, a.bad + b,
              lds_pairs);
}

// One block per tile of tokens.  ONE: all tokens are one counting block, which
// every workgroup counts for itself (one launch).
template <bool ONE>
__global__ __launch_bounds__(256) void k_send(SendArgs a) {
  __shared__ int32_t all[kMaxRanks], before[kMaxRanks], pairs[kMaxRanks], first[kMaxRanks + 1];
  __shared__ int32_t at[kMaxRanks];
  __shared__ int32_t one_at[ONE ? kTiles * kMaxRanks : 1], one_pairs[64], n_bad;
  __shared__ uint64_t mask[kSendTokens];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tile = blockIdx.x, block = tile / kTiles;
  if (tid < a.R) all[tid] = before[tid] = pairs[tid] = 0;
  if (tid == 0) n_bad = 0;
  __syncthreads();
  if (ONE) {
    if (wave == 0) count_block(a, 0, one_at, all, pairs, &n_bad, one_pairs);
  } else {
    for (int i = tid; i < a.blocks * a.R; i += 256) {
      const int r = i % a.R, v = a.tot[i];
      atomicAdd(&all[r], v);
      if (i < block * a.R) atomicAdd(&before[r], v);
      if (tile == 0) atomicAdd(&pairs[r], a.pairs[i]);
    }
    if (tile == 0)
      for (int i = tid; i < a.blocks; i += 256) atomicAdd(&n_bad, a.bad[i]);
  }
  // the tile's tokens: where each goes
  const int64_t t0 = (int64_t)tile * kSendTokens;
  if (wave == 1 && lane < kSendTokens) {
    int bad = 0;
    mask[lane] = t0 + lane < a.rows ? ranks_of(a, t0 + lane, &bad) : 0;
  }
  __syncthreads();
  if (tid == 0) {
    int n = 0;
    for (int r = 0; r < a.R; ++r) {
      first[r] = n;
      n += all[r];
    }
    first[a.R] = n;
  }
  __syncthreads();
  if (tid < a.R)
    at[tid] = first[tid] + before[tid] +
              (ONE ? one_at[tile * a.R + tid] : a.tile_at[(size_t)tile * a.R + tid]);
  if (tile == 0) {
    if (tid <= a.R) a.plan[tid] = first[tid];
    if (tid < a.R) a.plan[a.R + 1 + tid] = pairs[tid];
    if (tid == 0) a.plan[2 * a.R + 1] = n_bad;
  }
  __syncthreads();
  const int64_t chunks = a.row_bytes / 16;
  const int tail = (int)(a.row_bytes % 16);
  for (int i = wave; i < kSendTokens; i += 4) {
    const int64_t t = t0 + i;
    if (t >= a.rows) return;
    const uint64_t m = mask[i];
    if (!m) continue;
    // lane r: the token's place in rank r's segment, -1 if it does not go there
    int place = -1;
    if (lane < a.R && ((m >> lane) & 1)) {
      place = at[lane];
      for (int j = 0; j < i; ++j) place += (int)((mask[j] >> lane) & 1);
      if (place >= a.capacity) place = -1;
    }
    const uint64_t go = __ballot(place >= 0);
    for (uint64_t g = go; g; g &= g - 1) {
      const int r = __builtin_ctzll(g);
      const int64_t p = __shfl(place, r);
      if (lane == 0) a.token[p] = (int32_t)t;
      if (lane < a.k) {
        const int id = a.ids[t * a.k + lane];
        const bool here = id >= 0 && id / a.per == r;
        a.out_id[p * a.k + lane] = here ? id - r * a.per : -1;
        a.out_w[p * a.k + lane] = here ? a.w[t * a.k + lane] : 0.f;
      }
    }
    const char *src = a.x + t * a.ld_x;
    constexpr int U = 8;
    for (int64_t c0 = 0; c0 < chunks; c0 += 64 * U) {
      Any16 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t c = c0 + u * 64 + lane;
        if (c < chunks) v[u] = *(const Any16 *)(src + c * 16);
      }
      for (uint64_t g = go; g; g &= g - 1) {
        char *dst = a.out_x + (int64_t)__shfl(place, __builtin_ctzll(g)) * a.row_bytes;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t c = c0 + u * 64 + lane;
          if (c < chunks) *(Any16 *)(dst + c * 16) = v[u];
        }
      }
    }
    if (tail) {
      const char v = lane < tail ? src[chunks * 16 + lane] : 0;
      for (uint64_t g = go; g; g &= g - 1) {
        const int64_t p = __shfl(place, __builtin_ctzll(g));  // every lane takes part
        if (lane < tail) a.out_x[p * a.row_bytes + chunks * 16 + lane] = v;
      }
    }
  }
}

const char *bad_desc(const cep_dispatch_desc *d) {
  if (!d) return "desc is NULL";
  if (d->rows < 0 || d->rows > kMaxOpRows) return "rows must be in 0..2^24";
  if (d->top_k < 1 || d->top_k > kMaxTopK) return "top_k must be in 1..16";
  if (d->n_ranks < 1 || d->n_ranks > kMaxRanks) return "n_ranks must be in 1..64";
  if (d->experts_per_rank < 1 || d->experts_per_rank > 1 << 20)
    return "experts_per_rank must be in 1..2^20";
  if (d->row_bytes < 1 || d->row_bytes > 4 * kMaxDim) return "row_bytes must be in 1..131072";
  if (d->ld_x && d->ld_x < d->row_bytes) return "ld_x is shorter than a row";
  if (d->capacity < 0) return "capacity must be >= 0";
  const int64_t most = (int64_t)d->rows * (d->top_k < d->n_ranks ? d->top_k : d->n_ranks);
  if (most > INT32_MAX) return "rows * min(top_k, n_ranks) is too large";
  return nullptr;
}

int count_blocks(int rows) { return (rows + kCountTokens - 1) / kCountTokens; }

}  // namespace
}  // namespace cep

using namespace cep;

CEP_API size_t cep_dispatch_workspace(const cep_dispatch_desc *d) {
  if (bad_desc(d)) return 0;
  const size_t b = count_blocks(d->rows);
  return std::max<size_t>(4 * (b * d->n_ranks * (kTiles + 2) + b), 256);
}

CEP_API int cep_dispatch(const cep_dispatch_desc *d, const int32_t *topk_id, const float *topk_w,
                         const void *x, int32_t *plan, int32_t *token_idx, int32_t *out_id,
                         float *out_w, void *out_x, void *workspace, size_t workspace_bytes,
                         hipStream_t s) {
  const char *fn = "cep_dispatch";
  if (const char *why = bad_desc(d)) return refuse(CEP_EINVAL, "%s: %s", fn, why);
  const int64_t most = (int64_t)d->rows * std::min(d->top_k, d->n_ranks);
  if (d->capacity < most)
    return refuse(CEP_ENOMEM, "%s: capacity %d, up to %lld rows are sent", fn, d->capacity,
                  (long long)most);
  if (!plan || (d->rows && (!topk_id || !topk_w || !x || !token_idx || !out_id || !out_w || !out_x)))
    return refuse(CEP_EINVAL, "%s: NULL array", fn);
  if (!aligned(topk_id, 4) || !aligned(topk_w, 4) || !aligned(plan, 4) || !aligned(token_idx, 4) ||
      !aligned(out_id, 4) || !aligned(out_w, 4))
    return refuse(CEP_EINVAL, "%s: a pointer is not aligned to its type", fn);
  if (!workspace || !aligned(workspace, 4) || workspace_bytes < cep_dispatch_workspace(d))
    return refuse(workspace ? CEP_ENOMEM : CEP_EINVAL, "%s: needs a workspace of %zu bytes", fn,
                  cep_dispatch_workspace(d));
  const int blocks = count_blocks(d->rows), R = d->n_ranks;
  int32_t *ws = (int32_t *)workspace;
  SendArgs a{topk_id, topk_w, (const char *)x, d->ld_x ? d->ld_x : d->row_bytes, plan, token_idx,
             out_id, out_w, (char *)out_x, ws, ws + (size_t)blocks * kTiles * R,
             ws + (size_t)blocks * (kTiles + 1) * R, ws + (size_t)blocks * (kTiles + 2) * R,
             d->rows, d->top_k, R, d->experts_per_rank, blocks, d->capacity, d->row_bytes};
  const dim3 grid(std::max(1, (d->rows + kSendTokens - 1) / kSendTokens));
  if (blocks <= 1) {
    hipLaunchKernelGGL(k_send<true>, grid, dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL(k_send_count, dim3(blocks), dim3(64), 0, s, a);
    hipLaunchKernelGGL(k_send<false>, grid, dim3(256), 0, s, a);
  }
  return launched(fn);
}
