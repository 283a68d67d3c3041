// Stable sort of routed (token, slot) pairs by expert, with the token rows, for
// gfx950.
//
// A pair's place is its expert's offset plus the number of earlier pairs of that
// expert.  A few pairs are placed by one launch, a workgroup a token: its threads
// count, for each of the token's slots, the pairs that come first, (id, index)
// compared as a whole.  More take two: each block's counts and every pair's place
// among its expert's in the block (k_sort_count), and the places and rows
// (k_sort_rows), a wave a token, which reads its row once and writes it to each of its
// places.  It sums the blocks' counts itself, those of many blocks a launch between (k_sort_scan).
// Bound by HBM, mostly the sorted rows' writes: 8191 tokens of 8 KB, eight places each,
// 116 us for 604 MB, 5.2 TB/s (nontemporal stores: 17 % slower).
#include "block_ops.h"

#include <algorithm>

namespace cep {
namespace {

constexpr int kMaxSortExperts = 1024;
// Pairs placed by one launch (8 a token, 64 experts, us in one and in two: 512 tokens 8.7,
// 12.7; 768 13.0, 13.9; 1024 16.6, 14.0)
constexpr int kFewPairs = 4096;
constexpr int kSortPairs = 1024;    // pairs of a k_sort_count block, a quarter a wave
constexpr int kSortTokens = 4;      // tokens of a k_sort_rows block, one a wave
// Blocks whose counts k_sort_rows sums itself, a thread 256 buckets apart, and buckets.  A
// scan is a launch, nearly the same for any blocks; the sums are a walk over them in every
// workgroup, twice as long past 256 buckets (8 a token, 256-byte rows, us with the sums and
// with the scan: eight experts 8 blocks 8.6, 9.5; 16 9.9, 10.3; 24 11.4, 11.1; 64 20.2, 15.2;
// 256 118, 33.  64 experts 16 blocks 11.2, 11.4; 24 13.2, 12.1.  300 experts 8 blocks 12.1,
// 13.0; 12 14.3, 13.5)
constexpr int kFusedBlocks = 16, kFusedCounts = 512;

struct SortArgs {
  const int32_t *ids;  // [rows][k]
  const char *x;
  int64_t ld_x, row_bytes;
  int32_t *plan, *pair, *place;
  char *out_x;
  int32_t *counts;  // [blocks][E + 1], the last of ids out of range; after the scan of blocks before
  int32_t *total;   // [E + 1]
  int rows, k, E, blocks;
};

// The bucket of an id: its expert; E: out of range; -1: an empty slot.
__device__ inline int bucket_of(int id, int E) { return id < -1 || id >= E ? E : id; }

// Sum over the lanes up to this one.
__device__ inline int wave_upto(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  return v;
}

// Sum over the wave, by adds that read neighbouring lanes: within rows of 16, then a
// row's last lane into the next rows.
template <int CTRL, int ROWS>
__device__ inline int dpp_add(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ inline int wave_total(int v) {
  v = dpp_add<0x111, 0xf>(v);
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  v = dpp_add<0x118, 0xf>(v);
  v = dpp_add<0x142, 0xa>(v);
  v = dpp_add<0x143, 0xc>(v);
  return __builtin_amdgcn_readlane(v, 63);
}

// A wave walks its quarter of the block's pairs 64 at a time, lanes with the same
// bucket found by ballots over its bits, and keeps its own counts.  A pair's place
// in the block goes to `place`.
__global__ __launch_bounds__(256) void k_sort_count(SortArgs a) {
  constexpr int kRounds = kSortPairs / 256;
  __shared__ int32_t count[4][kMaxSortExperts + 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int e = tid; e <= a.E; e += 256)
#pragma unroll
    for (int w = 0; w < 4; ++w) count[w][e] = 0;
  __syncthreads();
  const int64_t pairs = (int64_t)a.rows * a.k;
  const int64_t p0 = (int64_t)blockIdx.x * kSortPairs + wave * (kRounds * 64) + lane;
  int bucket[kRounds], at[kRounds];
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int64_t p = p0 + i * 64;
    bucket[i] = p < pairs ? bucket_of(a.ids[p], a.E) : -1;
  }
  const int bits = 32 - __clz(a.E);  // of a bucket
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int b = bucket[i];
    uint64_t same = __ballot(b >= 0);
    for (int j = 0; j < bits; ++j) {
      const uint64_t one = __ballot((b >> j) & 1);
      same &= (b >> j) & 1 ? one : ~one;
    }
    const int before = (int)__popcll(same & ((1ull << lane) - 1));
    at[i] = 0;
    if (b >= 0) {
      at[i] = count[wave][b] + before;
      // the bucket's last lane, behind every lane's read (a wave's LDS operations
      // keep their order)
      if ((same >> lane) == 1) count[wave][b] = at[i] + 1;
    }
  }
  __syncthreads();
  for (int e = tid; e <= a.E; e += 256) {
    int run = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int n = count[w][e];
      count[w][e] = run;
      run += n;
    }
    a.counts[(int64_t)blockIdx.x * (a.E + 1) + e] = run;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int64_t p = p0 + i * 64;
    if (p >= pairs) continue;
    const int b = bucket[i];
    a.place[p] = b >= 0 && b < a.E ? at[i] + count[wave][b] : -1;
  }
}

// A wave a bucket: the blocks' counts become the sums of the blocks before.
__global__ __launch_bounds__(256) void k_sort_scan(SortArgs a) {
  const int lane = threadIdx.x & 63, e = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (e > a.E) return;  // uniform over the wave
  int run = 0;
  for (int64_t b0 = 0; b0 < a.blocks; b0 += 64) {
    const bool in = b0 + lane < a.blocks;
    int32_t *c = a.counts + (b0 + lane) * (a.E + 1) + e;
    const int v = in ? *c : 0, upto = wave_upto(v);
    if (in) *c = run + upto - v;
    run += __shfl(upto, 63);
  }
  if (lane == 0) a.total[e] = run;
}

// Offsets of the experts' segments from their totals in LDS, `off` [E + 1], by wave 0.
__device__ inline void scan_totals(const int32_t *total, int E, int32_t *off) {
  const int lane = threadIdx.x & 63;
  int run = 0;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int v = e0 + lane < E ? total[e0 + lane] : 0, upto = wave_upto(v);
    if (e0 + lane < E) off[e0 + lane] = run + upto - v;
    run += __shfl(upto, 63);
  }
  if (lane == 0) off[E] = run;
}

// A row's 16-byte chunks c0 + lane, and every STEP from there, kChunks in all
// (past the row's last whole chunk the lane reads that one again).
constexpr int kChunks = 8;
template <int STEP>
__device__ inline void load_row(const SortArgs &a, const char *src, int c0, Vec16 (&v)[kChunks]) {
  const int lane = threadIdx.x & 63, n = (int)(a.row_bytes / 16);
  if (n == 0) return;
#pragma unroll
  for (int u = 0; u < kChunks; ++u)
    v[u] = *(const Any16 *)(src + (int64_t)min(c0 + u * STEP + lane, n - 1) * 16);
}
// ... to the places that lanes below k hold (-1: none)
template <int STEP>
__device__ inline void store_row(const SortArgs &a, int place, int c0, const Vec16 (&v)[kChunks]) {
  const int lane = threadIdx.x & 63, n = (int)(a.row_bytes / 16);
  for (int j = 0; j < a.k; ++j) {
    const int to = __builtin_amdgcn_readlane(place, j);
    if (to < 0) continue;
    char *dst = a.out_x + (int64_t)to * a.row_bytes;
#pragma unroll
    for (int u = 0; u < kChunks; ++u) {
      const int c = c0 + u * STEP + lane;
      if (c < n) *(Any16 *)(dst + (int64_t)c * 16) = v[u];
    }
  }
}
__device__ inline void copy_tail(const SortArgs &a, const char *src, int place) {
  const int lane = threadIdx.x & 63, tail = (int)(a.row_bytes % 16);
  if (!tail) return;  // uniform
  const int64_t at = a.row_bytes - tail + lane;
  const char v = lane < tail ? src[at] : 0;
  for (int j = 0; j < a.k; ++j) {
    const int to = __builtin_amdgcn_readlane(place, j);
    if (to >= 0 && lane < tail) a.out_x[(int64_t)to * a.row_bytes + at] = v;
  }
}

// SCANNED: k_sort_scan ran.  Otherwise the workgroup sums the blocks' counts itself,
// while its rows are on the way.
template <bool SCANNED>
__global__ __launch_bounds__(64 * kSortTokens) void k_sort_rows(SortArgs a) {
  __shared__ int32_t off[kMaxSortExperts + 1];
  __shared__ int32_t sums[SCANNED ? 1 : 3][SCANNED ? 1 : kFusedCounts];  // all, before the
                                                                         // first pair's block
                                                                         // and the one after
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = (int64_t)blockIdx.x * kSortTokens + wave;
  const bool live = t < a.rows, copies = live && a.x;
  const char *src = a.x + (live ? t : 0) * a.ld_x;
  Vec16 v[kChunks] = {};
  if (copies) load_row<64>(a, src, 0, v);
  int at = -1, id = 0, before = 0;
  const int64_t p = t * a.k + lane;
  if (live && lane < a.k) {
    at = a.place[p];
    if (at >= 0) {
      id = a.ids[p];
      if (SCANNED) before = a.counts[p / kSortPairs * (a.E + 1) + id];
    }
  }
  // (the workgroup's pairs are fewer than a block's, so they lie in two at most)
  const int b0 = (int)((int64_t)blockIdx.x * kSortTokens * a.k / kSortPairs);
  if (!SCANNED) {
    for (int e = tid; e <= a.E; e += 64 * kSortTokens) {
      int run = 0, before0 = 0, before1 = 0;
#pragma unroll 8
      for (int b = 0; b < a.blocks; ++b) {
        const int n = a.counts[b * (a.E + 1) + e];
        run += n;
        before0 += b < b0 ? n : 0;
        before1 += b <= b0 ? n : 0;
      }
      sums[0][e] = run, sums[1][e] = before0, sums[2][e] = before1;
    }
    __syncthreads();
    if (at >= 0) before = sums[p / kSortPairs > b0 ? 2 : 1][id];
  }
  const int32_t *total = SCANNED ? a.total : sums[0];
  if (wave == 0) scan_totals(total, a.E, off);
  __syncthreads();
  if (blockIdx.x == 0) {
    for (int e = tid; e <= a.E; e += 64 * kSortTokens) a.plan[e] = off[e];
    if (tid == 0) a.plan[a.E + 1] = total[a.E];
  }
  if (!live) return;
  int place = -1;
  if (lane < a.k) {
    if (at >= 0) {
      place = off[id] + before + at;
      a.pair[place] = (int32_t)p;
    }
    a.place[p] = place;
  }
  if (!copies) return;
  store_row<64>(a, place, 0, v);
  for (int c0 = 64 * kChunks; c0 < a.row_bytes / 16; c0 += 64 * kChunks) {
    load_row<64>(a, src, c0, v);
    store_row<64>(a, place, c0, v);
  }
  copy_tail(a, src, place);
}

// Workgroup i places token i's pairs, its four waves every fourth 1 KB of the row.
// One workgroup more writes the plan.
__global__ __launch_bounds__(256) void k_sort_few(SortArgs a) {
  __shared__ int32_t sum[4][kMaxTopK], total[kMaxSortExperts + 1], off[kMaxSortExperts + 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int token = blockIdx.x, pairs = a.rows * a.k;
  if (token == a.rows) {  // uniform over the workgroup
    for (int e = tid; e <= a.E; e += 256) total[e] = 0;
    __syncthreads();
    constexpr int kOnTheWay = 8;  // loads
    for (int p0 = tid; p0 < pairs; p0 += 256 * kOnTheWay) {
      int b[kOnTheWay];
#pragma unroll
      for (int u = 0; u < kOnTheWay; ++u)
        b[u] = p0 + u * 256 < pairs ? a.ids[p0 + u * 256] : -1;
#pragma unroll
      for (int u = 0; u < kOnTheWay; ++u) {
        const int e = bucket_of(b[u], a.E);
        if (e >= 0) atomicAdd(&total[e], 1);
      }
    }
    __syncthreads();
    if (wave == 0) scan_totals(total, a.E, off);
    __syncthreads();
    for (int e = tid; e <= a.E; e += 256) a.plan[e] = off[e];
    if (tid == 0) a.plan[a.E + 1] = total[a.E];
    return;
  }
  const char *src = a.x + token * a.ld_x;
  const int chunks = (int)(a.row_bytes / 16);
  Vec16 v[kChunks] = {};
  if (a.x) load_row<256>(a, src, wave * 64, v);
  const int own = lane < a.k ? a.ids[token * a.k + lane] : -1;
  // (id, index) as one number, below 2^22
  const int mine = own >= 0 && own < a.E ? own * pairs + token * a.k + lane : 0;
  int first[kMaxTopK] = {};  // of the lane's pairs, those that come before slot j's
  constexpr int kAhead = 4;  // loads on the way
  for (int p0 = tid; p0 < pairs; p0 += 256 * kAhead) {
    int key[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int p = p0 + u * 256, id = p < pairs ? a.ids[p] : -1;
      key[u] = id >= 0 && id < a.E ? id * pairs + p : INT32_MAX;
    }
#pragma unroll
    for (int j = 0; j < kMaxTopK; ++j) {
      if (j >= a.k) continue;
      const int at = __builtin_amdgcn_readlane(mine, j);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) first[j] += key[u] < at;
    }
  }
#pragma unroll
  for (int j = 0; j < kMaxTopK; ++j) {
    if (j >= a.k) continue;
    const int n = wave_total(first[j]);
    if (lane == 0) sum[wave][j] = n;
  }
  __syncthreads();
  int place = -1;
  if (lane < a.k && own >= 0 && own < a.E)
    place = sum[0][lane] + sum[1][lane] + sum[2][lane] + sum[3][lane];
  if (wave == 0 && lane < a.k) {
    a.place[token * a.k + lane] = place;
    if (place >= 0) a.pair[place] = token * a.k + lane;
  }
  if (!a.x) return;
  for (int c0 = wave * 64;; c0 += 256 * kChunks) {
    store_row<256>(a, place, c0, v);
    if (c0 + 256 * kChunks >= chunks) break;
    load_row<256>(a, src, c0 + 256 * kChunks, v);
  }
  if (wave == 3) copy_tail(a, src, place);
}

const char *bad_desc(const cep_expert_sort_desc *d) {
  if (!d) return "desc is NULL";
  if (d->rows < 0 || d->rows > kMaxOpRows) return "rows must be in 0..2^21";
  if (d->top_k < 1 || d->top_k > kMaxTopK) return "top_k must be in 1..16";
  if (d->n_experts < 1 || d->n_experts > kMaxSortExperts) return "n_experts must be in 1..1024";
  if (d->row_bytes < 1 || d->row_bytes > 4 * kMaxDim) return "row_bytes must be in 1..131072";
  if (d->ld_x && d->ld_x < d->row_bytes) return "ld_x is shorter than a row";
  if (d->capacity < 0) return "capacity must be >= 0";
  return nullptr;
}

int sort_blocks(const cep_expert_sort_desc *d) {
  return (int)(((int64_t)d->rows * d->top_k + kSortPairs - 1) / kSortPairs);
}

}  // namespace
}  // namespace cep

using namespace cep;

CEP_API size_t cep_expert_sort_workspace(const cep_expert_sort_desc *d) {
  if (bad_desc(d)) return 0;
  return std::max<size_t>(4 * ((size_t)sort_blocks(d) + 1) * (d->n_experts + 1), 256);
}

CEP_API int cep_expert_sort(const cep_expert_sort_desc *d, const int32_t *topk_id, const void *x,
                            int32_t *plan, int32_t *pair, int32_t *place, void *out_x,
                            void *workspace, size_t workspace_bytes, hipStream_t s) {
  const char *fn = "cep_expert_sort";
  if (const char *why = bad_desc(d)) return refuse(CEP_EINVAL, "%s: %s", fn, why);
  const int64_t pairs = (int64_t)d->rows * d->top_k;
  if (d->capacity < pairs)
    return refuse(CEP_ENOMEM, "%s: capacity %d, up to %lld rows are sorted", fn, d->capacity,
                  (long long)pairs);
  if (!plan || (d->rows && (!topk_id || !pair || !place)))
    return refuse(CEP_EINVAL, "%s: NULL array", fn);
  if (d->rows && !x != !out_x)
    return refuse(CEP_EINVAL, "%s: x and out_x go together", fn);
  if (!aligned(topk_id, 4) || !aligned(plan, 4) || !aligned(pair, 4) || !aligned(place, 4))
    return refuse(CEP_EINVAL, "%s: a pointer is not aligned to its type", fn);
  if (!workspace || !aligned(workspace, 4) || workspace_bytes < cep_expert_sort_workspace(d))
    return refuse(workspace ? CEP_ENOMEM : CEP_EINVAL, "%s: needs a workspace of %zu bytes", fn,
                  cep_expert_sort_workspace(d));
  if (d->rows && x && x == out_x) return refuse(CEP_EINVAL, "%s: out_x overlaps x", fn);
  const int blocks = sort_blocks(d), E = d->n_experts;
  int32_t *counts = (int32_t *)workspace;
  const SortArgs a{topk_id, (const char *)x, d->ld_x ? d->ld_x : d->row_bytes, d->row_bytes, plan,
                   pair, place, (char *)out_x, counts, counts + (size_t)blocks * (E + 1), d->rows,
                   d->top_k, E, blocks};
  if (pairs <= kFewPairs) {
    hipLaunchKernelGGL(k_sort_few, dim3(d->rows + 1), dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL(k_sort_count, dim3(blocks), dim3(256), 0, s, a);
    const dim3 grid((d->rows + kSortTokens - 1) / kSortTokens), threads(64 * kSortTokens);
    if (E < kFusedCounts && blocks * (E / 256 + 1) <= kFusedBlocks) {
      hipLaunchKernelGGL(k_sort_rows<false>, grid, threads, 0, s, a);
    } else {
      hipLaunchKernelGGL(k_sort_scan, dim3(E / 4 + 1), dim3(256), 0, s, a);
      hipLaunchKernelGGL(k_sort_rows<true>, grid, threads, 0, s, a);
    }
  }
  return launched(fn);
}
