// Packing of routed tokens into one send buffer, expert-parallel rank by rank,
// for gfx950 (Appendix C, "Asynchronous dispatch": a source lane's rows travel
// to the rank that holds their experts).
//
// The tokens of a rank keep their order: a token's place in a rank's segment
// is the number of earlier tokens that go there too.  A few tokens are packed
// by one launch, a workgroup a token, each of which counts for itself
// (k_send_few).  More take three: the counts per block of 256 tokens
// (k_send_count), their prefix sums and the plan (k_send_scan), and the rows
// (k_send), a wave a token, which reads its row once, before it knows where the
// row goes, and writes it to each of its places.  Bound by HBM: 8192
// rows of 6336 bytes to ten ranks, 5.8 places each, 85 us, 4.2 TB/s, of which
// k_send 74; 13 rows of 14336 bytes 6.2 us, the latency of ids, counts and
// places.  (One launch for all with four tokens a wave: 189 us for 8192
// rows, 78 us for 13, too few loads in flight.)
#include "block_ops.h"

#include <algorithm>

namespace cep {
namespace {

constexpr int kMaxRanks = 64;      // one lane each
// Packed by one launch.  Rows of 6336 bytes to eight ranks, us in one launch and in
// three: 300 rows 10.4, 18.3; 512 11.9, 19.1; 1024 25.8, 20.0; 512 rows to 64
// ranks 17.1, 20.7.
constexpr int kFewTokens = 512;
constexpr int kCountTokens = 256;  // tokens of a k_send_count block
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
  // tot (after the scan: of the blocks before), pairs [blocks][R]; bad [blocks]
  int32_t *tile_at, *tot, *pairs, *bad;
  int rows, k, R, per, blocks;
  int64_t row_bytes;
  uint32_t mul, shift;  // id / per = id * mul >> shift
};

// The rank that holds an expert, -1: none.  mul = 2^shift / per rounded up and
// shift = 26 + log2(per) rounded up give the whole quotient of any id below
// 2^26, which those of 64 ranks of 2^20 experts are.
__device__ inline int rank_of(const SendArgs &a, int id) {
  return id >= 0 && id < a.R * a.per ? (int)(((uint64_t)(uint32_t)id * a.mul) >> a.shift) : -1;
}

// The ranks (a bit each) that hold the experts of token t; COUNT: counts its
// pairs per rank, and its ids that no rank has (apart from -1), in LDS.
template <bool COUNT>
__device__ inline uint64_t ranks_of(const SendArgs &a, int64_t t, int32_t *pairs, int32_t *bad) {
  int32_t id[kMaxTopK];
#pragma unroll
  for (int j = 0; j < kMaxTopK; ++j) id[j] = j < a.k ? a.ids[t * a.k + j] : -1;
  uint64_t m = 0;
#pragma unroll
  for (int j = 0; j < kMaxTopK; ++j) {
    if (j >= a.k) continue;
    const int r = rank_of(a, id[j]);
    if (r >= 0) {
      m |= 1ull << r;
      if (COUNT) atomicAdd(&pairs[r], 1);
    } else if (COUNT && id[j] != -1) {
      atomicAdd(bad, 1);
    }
  }
  return m;
}

// Sum over the lanes before this one.
__device__ inline int wave_before(int v) {
  const int lane = threadIdx.x & 63;
  int s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(s, o);
    if (lane >= o) s += u;
  }
  return s - v;
}

// Thread t counts token t of a block; lane r of a wave keeps rank r's count.
__global__ __launch_bounds__(kCountTokens) void k_send_count(SendArgs a) {
  __shared__ int32_t pairs[kMaxRanks], bad, sent[4][kMaxRanks];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = blockIdx.x, t = b * kCountTokens + tid;
  if (tid < kMaxRanks) pairs[tid] = 0;
  if (tid == 0) bad = 0;
  __syncthreads();
  const uint64_t m = t < a.rows ? ranks_of<true>(a, t, pairs, &bad) : 0;
  uint64_t there = 0;  // the wave's tokens that go to rank `lane`
  for (int r = 0; r < a.R; ++r) {
    const uint64_t v = __ballot((m >> r) & 1);
    if (lane == r) there = v;
  }
  sent[wave][lane] = (int)__popcll(there);
  __syncthreads();
  int run = 0;
  for (int i = 0; i < wave; ++i) run += sent[i][lane];
  if (lane < a.R) {
#pragma unroll
    for (int i = 0; i < 64 / kSendTokens; ++i)
      a.tile_at[(b * kTiles + wave * (64 / kSendTokens) + i) * a.R + lane] =
          run + (int)__popcll(there & ((1ull << (i * kSendTokens)) - 1));
    if (wave == 3) {
      a.tot[b * a.R + lane] = run + sent[3][lane];
      a.pairs[b * a.R + lane] = pairs[lane];
    }
  }
  if (tid == 0) a.bad[b] = bad;
}

// The plan from its counts (one block): wave 0 of a workgroup.
__device__ inline void write_plan(const SendArgs &a, const int32_t *sent, const int32_t *pairs,
                                  int bad) {
  const int lane = threadIdx.x & 63;
  const int n = lane < a.R ? sent[lane] : 0, at = wave_before(n);
  if (lane < a.R) {
    a.plan[lane] = at;
    a.plan[a.R + 1 + lane] = pairs[lane];
  }
  if (lane == a.R - 1) a.plan[a.R] = at + n;
  if (lane == 0) a.plan[2 * a.R + 1] = bad;
}

// Per rank (a wave takes every 16th): the block counts become the sums of the
// blocks before; then the plan.
__global__ __launch_bounds__(1024) void k_send_scan(SendArgs a) {
  __shared__ int32_t sent[kMaxRanks], pairs[kMaxRanks], bad;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  for (int r = wave; r < a.R; r += 16) {
    int run = 0, p = 0;
    for (int64_t b0 = 0; b0 < a.blocks; b0 += 64) {
      const bool in = b0 + lane < a.blocks;
      const int v = in ? a.tot[(b0 + lane) * a.R + r] : 0;
      p += in ? a.pairs[(b0 + lane) * a.R + r] : 0;
      const int before = wave_before(v);
      if (in) a.tot[(b0 + lane) * a.R + r] = run + before;
      run += __shfl(before + v, 63);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) p += __shfl_xor(p, o);
    if (lane == 0) {
      sent[r] = run;
      pairs[r] = p;
    }
  }
  for (int b = threadIdx.x; b < a.blocks; b += 1024) atomicAdd(&bad, a.bad[b]);
  __syncthreads();
  if (wave == 0) write_plan(a, sent, pairs, bad);
}

// The token's metadata at its places: lane r holds the place in rank r's
// segment, `go` the ranks it goes to; lanes below k its ids and weights.
__device__ inline void write_meta(const SendArgs &a, int t, int place, uint64_t go, int id,
                                  float w) {
  const int lane = threadIdx.x & 63, r_id = rank_of(a, id);
  for (uint64_t g = go; g; g &= g - 1) {
    const int r = __builtin_ctzll(g);
    const int64_t p = __shfl(place, r);
    if (lane == 0) a.token[p] = t;
    if (lane < a.k) {
      a.out_id[p * a.k + lane] = r_id == r ? id - r * a.per : -1;
      a.out_w[p * a.k + lane] = r_id == r ? w : 0.f;
    }
  }
}

// A row's 16-byte chunks c0 + lane, and every STEP from there, kChunks in all
// (past the row's last whole chunk the lane reads that one again).
constexpr int kChunks = 8;
template <int STEP>
__device__ inline void load_row(const SendArgs &a, const char *src, int c0, Vec16 (&v)[kChunks]) {
  const int lane = threadIdx.x & 63, n = (int)(a.row_bytes / 16);
  if (n == 0) return;
#pragma unroll
  for (int u = 0; u < kChunks; ++u)
    v[u] = *(const Any16 *)(src + (int64_t)min(c0 + u * STEP + lane, n - 1) * 16);
}
template <int STEP>
__device__ inline void store_row(const SendArgs &a, int place, uint64_t go, int c0,
                                 const Vec16 (&v)[kChunks]) {
  const int lane = threadIdx.x & 63, n = (int)(a.row_bytes / 16);
  for (uint64_t g = go; g; g &= g - 1) {
    char *dst = a.out_x + (int64_t)__shfl(place, __builtin_ctzll(g)) * a.row_bytes;
#pragma unroll
    for (int u = 0; u < kChunks; ++u) {
      const int c = c0 + u * STEP + lane;
      if (c < n) *(Any16 *)(dst + (int64_t)c * 16) = v[u];
    }
  }
}
__device__ inline void copy_tail(const SendArgs &a, const char *src, int place, uint64_t go) {
  const int lane = threadIdx.x & 63, tail = (int)(a.row_bytes % 16);
  if (!tail) return;  // uniform
  const int64_t at = a.row_bytes - tail + lane;
  const char v = lane < tail ? src[at] : 0;
  for (uint64_t g = go; g; g &= g - 1) {
    const int64_t p = __shfl(place, __builtin_ctzll(g));  // every lane takes part
    if (lane < tail) a.out_x[p * a.row_bytes + at] = v;
  }
}

// A wave a token.
__global__ __launch_bounds__(64 * kSendTokens) void k_send(SendArgs a) {
  __shared__ uint64_t mask[kSendTokens];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t tile = blockIdx.x, t = tile * kSendTokens + wave;
  const bool live = t < a.rows;
  const char *src = a.x + (live ? t : 0) * a.ld_x;
  Vec16 v[kChunks] = {};
  if (live) load_row<64>(a, src, 0, v);
  const int id = live && lane < a.k ? a.ids[t * a.k + lane] : -1;
  const float w = live && lane < a.k ? a.w[t * a.k + lane] : 0.f;
  int place = 0;
  if (lane < a.R)
    place = a.plan[lane] + a.tot[tile / kTiles * a.R + lane] + a.tile_at[tile * a.R + lane];
  const int r_id = rank_of(a, id);
  uint64_t go = 0;
  for (int j = 0; j < a.k; ++j) {
    const int r = __shfl(r_id, j);
    if (r >= 0) go |= 1ull << r;
  }
  if (lane == 0) mask[wave] = go;
  __syncthreads();
  if (!live) return;
  for (int i = 0; i < wave; ++i) place += (int)((mask[i] >> lane) & 1);
  write_meta(a, (int)t, place, go, id, w);
  store_row<64>(a, place, go, 0, v);
  for (int c0 = 64 * kChunks; c0 < a.row_bytes / 16; c0 += 64 * kChunks) {
    load_row<64>(a, src, c0, v);
    store_row<64>(a, place, go, c0, v);
  }
  copy_tail(a, src, place, go);
}

// Workgroup i packs token i, its four waves every fourth 1 KB of the row; its
// threads count every token first.  One workgroup more writes the plan.
__global__ __launch_bounds__(256) void k_send_few(SendArgs a) {
  __shared__ int32_t sent[4][kMaxRanks], before[4][kMaxRanks], pairs[kMaxRanks], bad;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int token = blockIdx.x;
  const bool packs = token < a.rows;  // the same in the whole workgroup
  const char *src = a.x + (packs ? token : 0) * a.ld_x;
  const int chunks = (int)(a.row_bytes / 16);
  Vec16 v[kChunks] = {};
  if (packs) load_row<256>(a, src, wave * 64, v);
  const int id = packs && lane < a.k ? a.ids[(int64_t)token * a.k + lane] : -1;
  const float w = packs && lane < a.k ? a.w[(int64_t)token * a.k + lane] : 0.f;
  if (!packs) {
    if (tid < kMaxRanks) pairs[tid] = 0;
    if (tid == 0) bad = 0;
    __syncthreads();
  }
  int n_sent = 0, n_before = 0;  // of the wave's tokens, to rank `lane`
  for (int t0 = 0; t0 < a.rows; t0 += 256) {
    const int t = t0 + tid, rel = token - t0 - wave * 64;  // this token among the wave's
    uint64_t m = 0;
    if (t < a.rows)
      m = packs ? ranks_of<false>(a, t, pairs, &bad) : ranks_of<true>(a, t, pairs, &bad);
    const uint64_t earlier = rel <= 0 ? 0 : rel >= 64 ? ~0ull : (1ull << rel) - 1;
    for (int r = 0; r < a.R; ++r) {
      const uint64_t there = __ballot((m >> r) & 1);
      if (lane == r) {
        n_sent += (int)__popcll(there);
        n_before += (int)__popcll(there & earlier);
      }
    }
  }
  sent[wave][lane] = n_sent;
  before[wave][lane] = n_before;
  __syncthreads();
  int all = 0, place = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    all += sent[i][lane];
    place += before[i][lane];
  }
  if (!packs) {
    __syncthreads();  // before wave 0 replaces its counts by the sums
    if (wave == 0) {
      sent[0][lane] = all;
      write_plan(a, sent[0], pairs, bad);
    }
    return;
  }
  place += wave_before(all);
  const int r_id = rank_of(a, id);
  uint64_t go = 0;
  for (int j = 0; j < a.k; ++j) {
    const int r = __shfl(r_id, j);
    if (r >= 0) go |= 1ull << r;
  }
  if (wave == 0) write_meta(a, token, place, go, id, w);
  for (int c0 = wave * 64;; c0 += 256 * kChunks) {
    store_row<256>(a, place, go, c0, v);
    if (c0 + 256 * kChunks >= chunks) break;
    load_row<256>(a, src, c0 + 256 * kChunks, v);
  }
  if (wave == 3) copy_tail(a, src, place, go);
}

const char *bad_desc(const cep_dispatch_desc *d) {
  if (!d) return "desc is NULL";
  if (d->rows < 0 || d->rows > kMaxOpRows) return "rows must be in 0..2^21";
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
             d->rows, d->top_k, R, d->experts_per_rank, blocks, d->row_bytes, 0, 26};
  while ((1 << (a.shift - 26)) < a.per) ++a.shift;
  a.mul = (uint32_t)(((uint64_t)1 << a.shift) / a.per + 1);
  if (d->rows <= kFewTokens) {
    hipLaunchKernelGGL(k_send_few, dim3(d->rows + 1), dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL(k_send_count, dim3(blocks), dim3(kCountTokens), 0, s, a);
    hipLaunchKernelGGL(k_send_scan, dim3(1), dim3(1024), 0, s, a);
    hipLaunchKernelGGL(k_send, dim3((d->rows + kSendTokens - 1) / kSendTokens),
                       dim3(64 * kSendTokens), 0, s, a);
  }
  return launched(fn);
}
