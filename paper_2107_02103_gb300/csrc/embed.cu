// Embedding of ids (atom types) and its gradient.
//   y[t]  = add[t] + scale W[id_t]                 an id outside [0, nvocab) adds nothing
//   dW[v] = (dW[v] +) scale sum_{t: id_t = v} dy[t]
// The gradient's sums run over the tokens sorted by id, in their order, cut at multiples of a number of rows that
// the sizes alone give, and the pieces of a cut run are added in order: no atomics, results repeat bit for bit.
// The rows are bound by memory: 65,536 x 1600 bf16 plus embedding in 74 us (5.7 TB/s), f32 in 130 (6.4); gradient of
// 65,536 x 1600 f32 to four rows in 68 (6.2 TB/s) and 10 for the join, of 24,571 x 1003 f16 to 30,011 in 34 and 12.  The plan
// is bound by latency, some 10 us a digit: 65,536 ids of four in 13 us, 24,571 of 30,011 in 24.
#include <cooperative_groups.h>

#include "rows.cuh"
#include "search.cuh"

namespace dpc {
namespace {

constexpr int kMaxVocab = (1 << 24) - 1, kMaxH = 1 << 20;

// ------------------------------------------------------------------ the plan: a stable radix sort of the ids
// Up to 4096 tokens in one block, up to 65,536 in a cluster of up to eight blocks that read one another's counts (one launch
// either way), more in three launches a digit.
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortPer = 4, kSortBlock = kSortThreads * kSortPer;
constexpr int kDigits = 256;

// Ids as sort keys: nvocab for those that stand for no row.
__device__ __forceinline__ uint32_t sort_key(int32_t id, int nvocab) {
  return (uint32_t)id < (uint32_t)nvocab ? (uint32_t)id : (uint32_t)nvocab;
}

// A thread's kPer items of a block in order by warp, 32 apart: the warp counts them by digit.
template <int kPer>
struct SortItems {
  uint32_t key[kPer];
  int64_t first;
};

// The place of every item of a block in a digit, after the warps before it and those before it in its warp.  cnt: a row
// of kDigits counters a warp, from counts to the warp's next place.
template <int kPer>
__device__ __forceinline__ void count_digits(const SortItems<kPer> &it, int64_t n, int shift, int mask, int *mine) {
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (it.first + 32 * i < n) atomicAdd(mine + (it.key[i] >> shift & mask), 1);  // integers: any order gives the same
}

// (Voting on each bit of the digit instead of the match, once for the count and the place: 12 -> 15 us for 65,536 ids.)
__device__ __forceinline__ int take_place(uint32_t d, bool have, int lane, int *mine) {
  const unsigned same = __match_any_sync(0xffffffffu, have ? d : 0xffffffffu);
  const int p = have ? mine[d] + __popc(same & ((1u << lane) - 1)) : 0;
  __syncwarp();
  if (have && lane == __ffs(same) - 1) mine[d] += __popc(same);
  __syncwarp();
  return p;
}

// An exclusive scan of 256 values by the first 256 threads of a block (all threads call).
__device__ __forceinline__ int scan_digits(int v, int *sums) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int inc = v;
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += up;
  }
  if (lane == 31 && warp < kDigits / 32) sums[warp] = inc;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < kDigits / 32; ++w) before += w < warp ? sums[w] : 0;
  __syncthreads();
  return before + inc - v;
}

// start[v] = the first of n sorted keys that is at least v.
__device__ __forceinline__ int lower_bound(const uint32_t *keys, int n, uint32_t v) {
  return dpc::lower_bound([keys](int i) { return keys[i]; }, n, v);
}

// Up to kSortBlock ids in one block, all digits in shared memory.
constexpr size_t kSmallSmem = (size_t)(kSortWarps * kDigits + 4 * kSortBlock + kSortWarps) * sizeof(int);
__global__ void __launch_bounds__(kSortThreads)
    embed_plan_small_kernel(const int32_t *__restrict__ ids, int n, int nvocab, int passes, int bits,
                            int64_t *__restrict__ start, int32_t *__restrict__ src) {
  extern __shared__ int smem[];
  int *cnt = smem, *sums = cnt + kSortWarps * kDigits;
  uint32_t *keys = (uint32_t *)(sums + kSortWarps);
  int *idx = (int *)(keys + 2 * kSortBlock);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, mask = (1 << bits) - 1;
  SortItems<kSortPer> it;
  int id[kSortPer];
  it.first = warp * kSortPer * 32 + lane;
#pragma unroll
  for (int i = 0; i < kSortPer; ++i) {
    id[i] = (int)it.first + 32 * i;
    it.key[i] = id[i] < n ? sort_key(__ldg(ids + id[i]), nvocab) : 0u;
  }
  for (int pass = 0; pass < passes; ++pass) {
    for (int i = threadIdx.x; i < kSortWarps * kDigits; i += kSortThreads) cnt[i] = 0;
    __syncthreads();
    int *mine = cnt + warp * kDigits;
    const int shift = pass * bits;
    count_digits(it, n, shift, mask, mine);
    __syncthreads();
    int total = 0;
    if (threadIdx.x < kDigits)
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) total += cnt[w * kDigits + threadIdx.x];
    int run = scan_digits(total, sums);
    if (threadIdx.x < kDigits)
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) {
        const int c = cnt[w * kDigits + threadIdx.x];
        cnt[w * kDigits + threadIdx.x] = run;
        run += c;
      }
    __syncthreads();
    uint32_t *to_k = keys + (pass & 1) * kSortBlock;
    int *to_i = idx + (pass & 1) * kSortBlock;
#pragma unroll
    for (int i = 0; i < kSortPer; ++i) {
      const bool have = it.first + 32 * i < n;
      const int p = take_place(it.key[i] >> shift & mask, have, lane, mine);
      if (have) {
        to_k[p] = it.key[i];
        to_i[p] = id[i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortPer; ++i)
      if (it.first + 32 * i < n) {
        it.key[i] = to_k[it.first + 32 * i];
        id[i] = to_i[it.first + 32 * i];
      }
  }
#pragma unroll
  for (int i = 0; i < kSortPer; ++i)
    if (it.first + 32 * i < n) src[it.first + 32 * i] = it.key[i] < (uint32_t)nvocab ? id[i] : -1;
  const uint32_t *sorted = keys + ((passes - 1) & 1) * kSortBlock;
  for (int v = threadIdx.x; v <= nvocab; v += kSortThreads) start[v] = lower_bound(sorted, n, v);
}

// The digits' places in global memory (keys and idx: two of each), blocks of a cluster.  A block's counts of a digit's
// pass lie in its shared memory until all have read them.  start: with one digit its scan, else each block searches the
// ids between its sorted keys.
constexpr int kClusterBlocks = 8, kClusterStart = 1 << 16;
template <int kPer>
__global__ void __launch_bounds__(kSortThreads)
    embed_plan_cluster_kernel(const int32_t *__restrict__ ids, int n, int nvocab, int passes, int bits, uint32_t *keys, int *idx,
                              int64_t *__restrict__ start, int32_t *src) {
  namespace cg = cooperative_groups;
  constexpr int kItems = kSortThreads * kPer;
  __shared__ int cnt[kSortWarps * kDigits], block[kDigits], sums[kDigits / 32];
  static_assert(kItems <= kSortWarps * kDigits, "a block's keys in the counters' place");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, mask = (1 << bits) - 1, d = threadIdx.x;
  SortItems<kPer> it;
  int id[kPer];
  it.first = (int64_t)blockIdx.x * kItems + warp * kPer * 32 + lane;
  for (int pass = 0; pass < passes; ++pass) {
    const uint32_t *from_k = keys + (int64_t)((pass - 1) & 1) * n;
    const int *from_i = idx + (int64_t)((pass - 1) & 1) * n;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {  // written by other blocks in the pass before: not through L1
      const int64_t q = it.first + 32 * i;
      it.key[i] = q >= n ? 0u : pass ? __ldcg(from_k + q) : sort_key(__ldg(ids + q), nvocab);
      id[i] = q >= n ? 0 : pass ? __ldcg(from_i + q) : (int)q;
    }
    for (int i = threadIdx.x; i < kSortWarps * kDigits; i += kSortThreads) cnt[i] = 0;
    __syncthreads();
    int *mine = cnt + warp * kDigits;
    const int shift = pass * bits;
    count_digits(it, n, shift, mask, mine);
    __syncthreads();
    if (d < kDigits) {
      int c = 0;
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) c += cnt[w * kDigits + d];
      block[d] = c;
    }
    cg::this_cluster().sync();
    int total = 0, before = 0;
    if (d < kDigits)
#pragma unroll
      for (int b = 0; b < kClusterBlocks; ++b) {
        const int c = b < (int)gridDim.x ? cg::this_cluster().map_shared_rank(block, b)[d] : 0;
        before += b < (int)blockIdx.x ? c : 0;
        total += c;
      }
    int run = scan_digits(total, sums);
    if (passes == 1 && blockIdx.x == 0 && d <= nvocab) start[d] = run;
    if (d < kDigits) {
      run += before;
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) {
        const int c = cnt[w * kDigits + d];
        cnt[w * kDigits + d] = run;
        run += c;
      }
    }
    __syncthreads();
    const bool last = pass == passes - 1;
    uint32_t *to_k = keys + (int64_t)(pass & 1) * n;
    int *to_i = last ? src : idx + (int64_t)(pass & 1) * n;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const bool have = it.first + 32 * i < n;
      const int p = take_place(it.key[i] >> shift & mask, have, lane, mine);
      if (have) {
        if (!last || passes > 1) to_k[p] = it.key[i];
        to_i[p] = last && it.key[i] >= (uint32_t)nvocab ? -1 : id[i];
      }
    }
    cg::this_cluster().sync();  // the counts are read, the places written
  }
  if (passes == 1 || nvocab > kClusterStart) return;
  uint32_t *sorted = (uint32_t *)cnt;
  const uint32_t *from = keys + (int64_t)((passes - 1) & 1) * n;
  const int first = blockIdx.x * kItems, own = min(kItems, n - first);
  for (int i = threadIdx.x; i < own; i += kSortThreads) sorted[i] = __ldcg(from + first + i);
  const int low = first ? (int)__ldcg(from + first - 1) + 1 : 0;
  __syncthreads();
  const int high = first + own == n ? nvocab : (int)sorted[own - 1];
  for (int v = low + threadIdx.x; v <= high; v += kSortThreads) start[v] = first + lower_bound(sorted, own, v);
}

// More ids, a pass of a digit: counts[d][block], each digit's scan over the blocks with its total behind, and the move.
__global__ void __launch_bounds__(kSortThreads)
    sort_count_kernel(const int32_t *__restrict__ ids, const uint32_t *__restrict__ keys, int64_t n, int nvocab, int shift,
                      int mask, int *__restrict__ counts) {
  __shared__ int cnt[kDigits];
  if (threadIdx.x < kDigits) cnt[threadIdx.x] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * kSortBlock + threadIdx.x;
#pragma unroll
  for (int i = 0; i < kSortPer; ++i) {
    const int64_t q = first + (int64_t)i * kSortThreads;
    if (q < n) atomicAdd(cnt + ((keys ? __ldg(keys + q) : sort_key(__ldg(ids + q), nvocab)) >> shift & mask), 1);
  }
  __syncthreads();
  if (threadIdx.x < kDigits) counts[(int64_t)threadIdx.x * gridDim.x + blockIdx.x] = cnt[threadIdx.x];
}

__global__ void __launch_bounds__(kDigits) sort_scan_kernel(int *__restrict__ counts, int nb, int *__restrict__ totals) {
  __shared__ int sums[kDigits / 32], chunk;
  int *row = counts + (int64_t)blockIdx.x * nb;
  int base = 0;
  for (int b0 = 0; b0 < nb; b0 += kDigits) {
    const int b = b0 + threadIdx.x, c = b < nb ? row[b] : 0;
    const int before = scan_digits(c, sums);
    if (b < nb) row[b] = base + before;
    if (threadIdx.x == kDigits - 1) chunk = before + c;
    __syncthreads();
    base += chunk;
    __syncthreads();
  }
  if (threadIdx.x == 0) totals[blockIdx.x] = base;
}

__global__ void __launch_bounds__(kSortThreads)
    sort_place_kernel(const int32_t *__restrict__ ids, const uint32_t *__restrict__ keys, const int *__restrict__ idx,
                      int64_t n, int nvocab, int shift, int bits, const int *__restrict__ counts,
                      const int *__restrict__ totals, uint32_t *__restrict__ to_key, int *__restrict__ to_idx, bool last) {
  __shared__ int cnt[kSortWarps * kDigits], sums[kSortWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, mask = (1 << bits) - 1;
  for (int i = threadIdx.x; i < kSortWarps * kDigits; i += kSortThreads) cnt[i] = 0;
  SortItems<kSortPer> it;
  int id[kSortPer];
  it.first = (int64_t)blockIdx.x * kSortBlock + warp * kSortPer * 32 + lane;
#pragma unroll
  for (int i = 0; i < kSortPer; ++i) {
    const int64_t q = it.first + 32 * i;
    it.key[i] = q >= n ? 0u : keys ? __ldg(keys + q) : sort_key(__ldg(ids + q), nvocab);
    id[i] = q >= n ? 0 : idx ? __ldg(idx + q) : (int)q;
  }
  __syncthreads();
  int *mine = cnt + warp * kDigits;
  count_digits(it, n, shift, mask, mine);
  __syncthreads();
  const int d = threadIdx.x;
  int run = scan_digits(d < kDigits ? __ldg(totals + d) : 0, sums);
  if (d < kDigits) {
    run += __ldg(counts + (int64_t)d * gridDim.x + blockIdx.x);
#pragma unroll 8
    for (int w = 0; w < kSortWarps; ++w) {
      const int c = cnt[w * kDigits + d];
      cnt[w * kDigits + d] = run;
      run += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortPer; ++i) {
    const bool have = it.first + 32 * i < n;
    const int p = take_place(it.key[i] >> shift & mask, have, lane, mine);
    if (have) {
      to_key[p] = it.key[i];
      to_idx[p] = last && it.key[i] >= (uint32_t)nvocab ? -1 : id[i];
    }
  }
}

__global__ void __launch_bounds__(256)
    embed_start_kernel(const uint32_t *__restrict__ keys, int n, int nvocab, int64_t *__restrict__ start) {
  const int v = blockIdx.x * 256 + threadIdx.x;
  if (v <= nvocab) start[v] = lower_bound(keys, n, v);
}

struct SortShape {
  int blocks, passes, bits;
};
SortShape sort_shape(int64_t n, int nvocab) {
  int bits = 1;
  while (nvocab >> bits) ++bits;  // keys up to nvocab
  SortShape s;
  s.passes = (bits + 7) / 8;
  s.bits = (bits + s.passes - 1) / s.passes;
  s.blocks = (int)((n + kSortBlock - 1) / kSortBlock);
  return s;
}

// Whether one block does it all, start included: not where there are many more ids than its threads can search for.
bool plan_is_small(int64_t ntok, int nvocab) { return ntok == 0 || (ntok <= kSortBlock && nvocab <= kClusterStart); }

// ------------------------------------------------------------------ the rows
// V elements an access.  Long rows: a warp takes kFwdPart packs a lane of a token's row.  Short ones (Flat, fewer packs than
// lanes): a thread takes one pack, the packs in order over the tokens.
constexpr int kFwdThreads = 128;
template <int V>
constexpr int kFwdPart = V > 1 ? 2 : 8;  // accesses of a lane
template <typename T, int V, bool Flat>
__global__ void __launch_bounds__(kFwdThreads)
    embed_fwd_kernel(const T *__restrict__ W, const int32_t *__restrict__ ids, int64_t ntok, int nvocab, int H, int np,
                     acc_t<T> scale, const T *add, T *y) {  // y may be add
  using A = acc_t<T>;
  constexpr int kP = Flat ? 1 : kFwdPart<V>;
  int64_t t;
  int c;
  if constexpr (Flat) {
    const int64_t base = (int64_t)blockIdx.x * kFwdThreads, t0 = base / np;
    const uint32_t off = (uint32_t)(base - t0 * np) + threadIdx.x, dt = off / (uint32_t)np;
    t = t0 + dt;
    c = (int)(off - dt * np);
  } else {
    t = (int64_t)blockIdx.x * (kFwdThreads / 32) + (threadIdx.x >> 5);
    c = (int)(blockIdx.y * 32 * kP + (threadIdx.x & 31));
  }
  if (t >= ntok) return;
  Pack<T, V> a[kP], w[kP];
#pragma unroll
  for (int i = 0; i < kP; ++i)
    if (add && c + 32 * i < np) a[i] = load_pack<T, V>(add + t * H + (c + 32 * i) * V);
  const int32_t id = __ldg(ids + t);
  const bool have = (uint32_t)id < (uint32_t)nvocab;
  const T *row = W + (int64_t)id * H;
#pragma unroll
  for (int i = 0; i < kP; ++i)
    if (have && c + 32 * i < np) w[i] = load_pack<T, V>(row + (c + 32 * i) * V);
#pragma unroll
  for (int i = 0; i < kP; ++i)
    if (c + 32 * i < np) {
      Pack<T, V> o;
#pragma unroll
      for (int l = 0; l < V; ++l) {
        const A from = add ? to_acc(a[i].v[l]) : A(0);
        o.v[l] = from_acc<T>(have ? fma(scale, to_acc(w[i].v[l]), from) : from);
      }
      store_pack<T, V>(y + t * H + (c + 32 * i) * V, o);
    }
}

// A group of `width` threads sums a chunk of R sorted rows over a strip of columns: runs of an id that lie in the chunk go
// to dW, what continues from the chunk before or into the next to `part` ([chunk][2][H]: the piece that begins at the
// chunk's first row, and the one after it); cut[chunk] is the id of the run that begins in the chunk and goes on, else -1.
// Further blocks clear the rows of ids that no token has.  The chunk's tokens and ids are read first, so that the rows'
// addresses wait for shared memory alone.
constexpr int kSumThreads = 256, kMaxRows = 256, kMaxGroups = 8, kClearRows = 32;
// Rows of a thread on their way, and its accesses of a row: a row's bookkeeping costs more than one element's sum.
template <int V>
constexpr int kSumAhead = V > 1 ? 8 : 4;
template <int V>
constexpr int kSumCols = V > 1 ? 1 : 4;
constexpr int kMostAhead = 8;
struct SumShape {
  int R, chunks, strips, width, groups;
  int64_t blocks;  // that sum
};
template <typename T, int V>
__global__ void __launch_bounds__(kSumThreads)
    embed_grad_kernel(const T *__restrict__ dy, const int32_t *__restrict__ ids, const int64_t *__restrict__ start,
                      const int32_t *__restrict__ src, int64_t ntok, int nvocab, int H, const __grid_constant__ SumShape s,
                      acc_t<T> scale, bool accumulate, acc_t<T> *__restrict__ dW, acc_t<T> *__restrict__ part,
                      int *__restrict__ cut) {
  using A = acc_t<T>;
  constexpr int kAhead = kSumAhead<V>, kCols = kSumCols<V>;
  if ((int64_t)blockIdx.x >= s.blocks) {  // (in turn with the others instead: 48 -> 56 us for 24,571 x 1003 f16 to 30,011 rows)
    const int64_t v0 = ((int64_t)blockIdx.x - s.blocks) * kClearRows;
    const int lane = threadIdx.x & 31;
    const bool in = v0 + lane < nvocab;
    const int64_t at = in ? __ldg(start + v0 + lane) : 0, end = in ? __ldg(start + v0 + lane + 1) : 1;
    unsigned empty = __ballot_sync(0xffffffffu, at == end);
    for (int n = 0; empty; empty &= empty - 1, ++n)
      if (n % (int)(blockDim.x / 32) == (int)threadIdx.x / 32) {
        A *row = dW + (v0 + __ffs(empty) - 1) * H;
        if ((((uintptr_t)dW | (uintptr_t)(H * sizeof(A))) & 15) == 0) {
          for (int c = lane; c < H / (16 / (int)sizeof(A)); c += 32)
            reinterpret_cast<uint4 *>(row)[c] = make_uint4(0, 0, 0, 0);
        } else {
          for (int c = lane; c < H; c += 32) row[c] = A(0);
        }
      }
    return;
  }
  __shared__ int froms[kMaxGroups * (kMaxRows + kMostAhead)], idsm[kMaxGroups * (kMaxRows + 2)];
  const int group = threadIdx.x / s.width, tid = threadIdx.x - group * s.width;
  const int64_t unit = (int64_t)blockIdx.x * s.groups + group, chunk = unit / s.strips;
  const int strip = (int)(unit - chunk * s.strips);
  // a row's token (-1: none), and its id, of one row before, and one behind
  int *from = froms + group * (s.R + kMostAhead), *id = idsm + group * (s.R + 2);
  const int64_t kept = min(max(__ldg(start + nvocab), (int64_t)0), ntok), r0 = chunk * s.R;
  const int rows = chunk < s.chunks ? (int)min((int64_t)s.R, max(kept - r0, (int64_t)0)) : 0;
  for (int r = tid - 1; r < rows + kAhead; r += s.width) {
    const int64_t p = r0 + r;
    const int q = p >= 0 && p < kept && r <= rows ? __ldg(src + p) : -1;
    const bool have = q >= 0 && q < ntok;  // the plan may not be one of these ids
    if (r <= rows) id[r + 1] = have ? __ldg(ids + q) : -1;
    if (r >= 0) from[r] = have && r < rows ? q : -1;
  }
  __syncthreads();
  if (chunk >= s.chunks) return;
  if (rows == 0) {
    if (strip == 0 && tid == 0) cut[chunk] = -1;
    return;
  }
  const int c = (strip * s.width * kCols + tid) * V, step = s.width * V;  // its accesses are `step` apart
  if (c >= H) return;
  const int before = id[0], after = id[rows + 1];
  A sum[kCols][V] = {};
  int run = id[1], first = 0;  // the run at hand and its first row
  auto put = [&](int end) {    // its rows end before `end`
    if ((uint32_t)run < (uint32_t)nvocab) {
      const bool is_cut = (first == 0 && before == run) || (end == rows && after == run);
      A *to = is_cut ? part + (chunk * 2 + (first ? 1 : 0)) * H + c : dW + (int64_t)run * H + c;
#pragma unroll
      for (int u = 0; u < kCols; ++u, to += step)
        if (kCols == 1 || c + u * step < H)
#pragma unroll
          for (int l = 0; l < V; ++l)
            to[l] = is_cut ? sum[u][l] : accumulate ? fma(scale, sum[u][l], to[l]) : scale * sum[u][l];
    }
#pragma unroll
    for (int u = 0; u < kCols; ++u)
#pragma unroll
      for (int l = 0; l < V; ++l) sum[u][l] = A(0);
  };
  for (int r = 0; r < rows; r += kAhead) {
    Pack<T, V> v[kAhead][kCols];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int q = from[r + i];
      const T *row = dy + (int64_t)q * H + c;
#pragma unroll
      for (int u = 0; u < kCols; ++u) {
        v[i][u] = Pack<T, V>{};
        if (q >= 0 && (kCols == 1 || c + u * step < H)) v[i][u] = load_pack<T, V>(row + u * step);
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (r + i < rows) {
        const int now = id[r + i + 1];
        if (now != run) {
          put(r + i);
          run = now;
          first = r + i;
        }
#pragma unroll
        for (int u = 0; u < kCols; ++u)
#pragma unroll
          for (int l = 0; l < V; ++l) sum[u][l] += to_acc(v[i][u].v[l]);
      }
  }
  if (c == 0) cut[chunk] = (uint32_t)run < (uint32_t)nvocab && after == run && !(first == 0 && before == run) ? run : -1;
  put(rows);
}

// The runs that chunks cut, four chunks a block: a run's pieces are added in four parts of neighbouring ones, each in
// order, and the parts in order.  (One part: a run of a tenth of 24,571 tokens, 50 pieces, took 21 us.)
constexpr int kJoinSlots = 4, kJoinParts = 4;
template <int V>
constexpr int kJoinCols = V > 1 ? 1 : 4;
template <typename A, int V>
__global__ void __launch_bounds__(kJoinSlots *kJoinParts * 32)
    embed_join_kernel(const int64_t *__restrict__ start, int64_t ntok, int nvocab, int H, int R, int chunks, A scale,
                      bool accumulate, A *__restrict__ dW, const A *__restrict__ part, const int *__restrict__ cut) {
  __shared__ Pack<A, V> sums[kJoinSlots][kJoinParts][kJoinCols<V>][32];
  constexpr int kCols = kJoinCols<V>;  // accesses of a thread, 32 apart
  const int lane = threadIdx.x % 32, which = threadIdx.x / 32 % kJoinParts, slot = threadIdx.x / (32 * kJoinParts);
  const int chunk = blockIdx.x * kJoinSlots + slot, c = (blockIdx.y * 32 * kCols + lane) * V;
  const int v = chunk < chunks ? __ldg(cut + chunk) : -1;
  if (!__syncthreads_or(v >= 0)) return;
  Pack<A, V> sum[kCols] = {};
  if (v >= 0 && v < nvocab) {
    const int s0 = (int)__ldg(start + v), s1 = (int)min(__ldg(start + v + 1), ntok);  // below 2^31
    const int n = min((s1 - 1) / R, chunks - 1) - chunk + 1, each = (n + kJoinParts - 1) / kJoinParts;  // pieces
    const int first = which * each, end = min(n, first + each);
    constexpr int kAhead = kCols > 1 ? 4 : 8;  // pieces on their way
    const A *from = part + (int64_t)(chunk + first) * 2 * H + c;
    for (int k = first; k < end; k += kAhead, from += (int64_t)2 * kAhead * H) {
      Pack<A, V> p[kAhead][kCols];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
#pragma unroll
        for (int u = 0; u < kCols; ++u)
          if (k + i < end && c + 32 * V * u < H)
            p[i][u] = load_pack<A, V>(from + 32 * V * u + (int64_t)2 * i * H + (k + i == 0 && s0 != chunk * R ? H : 0));
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
#pragma unroll
        for (int u = 0; u < kCols; ++u)
          if (k + i < end && c + 32 * V * u < H)
#pragma unroll
            for (int l = 0; l < V; ++l) sum[u].v[l] += p[i][u].v[l];
    }
  }
#pragma unroll
  for (int u = 0; u < kCols; ++u) sums[slot][which][u][lane] = sum[u];
  __syncthreads();
  if (which || v < 0 || v >= nvocab) return;
#pragma unroll
  for (int u = 0; u < kCols; ++u) {
    if (c + 32 * V * u >= H) break;
#pragma unroll
    for (int k = 1; k < kJoinParts; ++k)
#pragma unroll
      for (int l = 0; l < V; ++l) sum[u].v[l] += sums[slot][k][u][lane].v[l];
    A *to = dW + (int64_t)v * H + c + 32 * V * u;
#pragma unroll
    for (int l = 0; l < V; ++l) to[l] = accumulate ? fma(scale, sum[u].v[l], to[l]) : scale * sum[u].v[l];
  }
}

// Strips of at most kSumThreads packs, whole warps a group, as many groups a block as fit, chunks of 16 to 256 rows.
SumShape sum_shape(int64_t ntok, int np, bool packs) {
  SumShape s;
  const int cols = packs ? 1 : kSumCols<1>, threads = (np + cols - 1) / cols;  // of a row
  s.strips = (threads + kSumThreads - 1) / kSumThreads;
  s.width = ((threads + s.strips - 1) / s.strips + 31) / 32 * 32;
  s.groups = kSumThreads / s.width;
  int64_t want = (int64_t)152 * 4 * s.groups / s.strips;  // chunks of four blocks an SM, all resident
  if (want < 1) want = 1;
  int64_t R = ((ntok + want - 1) / want + 15) / 16 * 16;
  s.R = (int)(R < 16 ? 16 : R > kMaxRows ? kMaxRows : R);
  s.chunks = (int)((ntok + s.R - 1) / s.R);
  s.blocks = ((int64_t)s.chunks * s.strips + s.groups - 1) / s.groups;
  return s;
}
// The pieces of the chunks of rows of H elements, whether they move in packs or not, then the chunks' cut.
size_t part_chunks(int64_t ntok, int H, int elem) {
  const int V = 16 / elem;
  const SumShape a = sum_shape(ntok, (H + V - 1) / V, true), b = sum_shape(ntok, H, false);
  return (size_t)(a.chunks > b.chunks ? a.chunks : b.chunks);
}
size_t part_bytes(int64_t ntok, int H, int elem) {
  return part_chunks(ntok, H, elem) * ((size_t)2 * H * (elem == 8 ? 8 : 4) + sizeof(int));
}

int embed_check(int64_t ntok, int nvocab, const char *who) {
  if (ntok < 0 || ntok > 0x7fffffffLL - kSortBlock) return set_error(DP_ERR_SHAPE, "%s: ntok = %lld", who, (long long)ntok);
  if (nvocab < 1) return set_error(DP_ERR_SHAPE, "%s: nvocab = %d", who, nvocab);
  if (nvocab > kMaxVocab) return set_error(DP_ERR_UNSUPPORTED, "%s: nvocab = %d > %d", who, nvocab, kMaxVocab);
  return DP_OK;
}
template <typename A>
int embed_check(int64_t ntok, int nvocab, int H, double scale, const char *who) {
  const int rc = embed_check(ntok, nvocab, who);
  if (rc) return rc;
  if (H < 1 || H > kMaxH) return set_error(DP_ERR_SHAPE, "%s: row length %d outside [1, 2^20]", who, H);
  if (!scale_fits<A>(scale)) return set_error(DP_ERR_SHAPE, "%s: scale = %g", who, scale);
  return DP_OK;
}

template <typename T>
int embed_fwd(const T *W, const int32_t *ids, int64_t ntok, int nvocab, int H, double scale, const T *add, T *y,
              void *stream, const char *who) {
  clear_error();
  const int rc = embed_check<acc_t<T>>(ntok, nvocab, H, scale, who);
  if (rc || ntok == 0) return rc;
  if (!W || !ids || !y) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (!at_elements(W, add, y) || !at_elements(ids)) return misaligned(who);
  constexpr int V = 16 / (int)sizeof(T);
  const bool whole = pack_width<T>(H, W, add, y) >= V;
  const int np = whole ? H / V : H;
  const bool flat = np < 32;
  const int64_t bx = flat ? (ntok * np + kFwdThreads - 1) / kFwdThreads : (ntok + kFwdThreads / 32 - 1) / (kFwdThreads / 32);
  const int part = 32 * (whole ? kFwdPart<V> : kFwdPart<1>), by = flat ? 1 : (np + part - 1) / part;
  if (bx > 0x7fffffffLL || by > 65535) return set_error(DP_ERR_SHAPE, "%s: %lld rows of %d", who, (long long)ntok, H);
  auto k = flat ? (whole ? embed_fwd_kernel<T, V, true> : embed_fwd_kernel<T, 1, true>)
                : (whole ? embed_fwd_kernel<T, V, false> : embed_fwd_kernel<T, 1, false>);
  k<<<dim3((unsigned)bx, (unsigned)by), kFwdThreads, 0, (cudaStream_t)stream>>>(W, ids, ntok, nvocab, H, np,
                                                                                     (acc_t<T>)scale, add, y);
  return launch_status(who);
}

template <typename T>
int embed_grad(const T *dy, const int32_t *ids, const int64_t *start, const int32_t *src, int64_t ntok, int nvocab, int H,
               double scale, int accumulate, acc_t<T> *dW, void *work, size_t work_bytes, void *stream, const char *who) {
  using A = acc_t<T>;
  clear_error();
  const int rc = embed_check<A>(ntok, nvocab, H, scale, who);
  if (rc) return rc;
  if (!start || !dW || (ntok > 0 && (!dy || !ids || !src))) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (!at_elements(dy) || !at_elements(ids, src) || !at_elements(start) || !at_elements(dW)) return misaligned(who);
  constexpr int V = 16 / (int)sizeof(T);
  const bool whole = pack_width<T>(H, dy) >= V;
  const int np = whole ? H / V : H;
  const SumShape s = sum_shape(ntok, np, whole);
  if (s.chunks > 0) {
    if (!work) return set_error(DP_ERR_NULL, "%s: work is NULL", who);
    if (work_bytes < part_bytes(ntok, H, sizeof(T)) || ((uintptr_t)work & 15))
      return set_error(DP_ERR_SHAPE, "%s: work buffer of %zu bytes is too short or misaligned", who, work_bytes);
  }
  const int64_t blocks = s.blocks + (accumulate ? 0 : (nvocab + kClearRows - 1) / kClearRows);
  if (blocks == 0) return DP_OK;
  if (blocks > 0x7fffffffLL) return set_error(DP_ERR_SHAPE, "%s: %lld rows of %d", who, (long long)ntok, H);
  const cudaStream_t st = (cudaStream_t)stream;
  A *part = (A *)work;
  int *cut = s.chunks ? (int *)(part + part_chunks(ntok, H, sizeof(T)) * 2 * H) : nullptr;
  auto k = whole ? embed_grad_kernel<T, V> : embed_grad_kernel<T, 1>;
  k<<<(unsigned)blocks, s.groups * s.width, 0, st>>>(dy, ids, start, src, ntok, nvocab, H, s, (A)scale,
                                                      accumulate != 0, dW, part, cut);
  if (s.chunks > 1) {
    constexpr int VA = 16 / (int)sizeof(A);
    const bool packs = pack_width<A>(H, dW) >= VA;
    const int cols = 32 * (packs ? VA : kJoinCols<1>);  // of a block
    const dim3 grid((s.chunks + kJoinSlots - 1) / kJoinSlots, (H + cols - 1) / cols);
    auto join = packs ? embed_join_kernel<A, VA> : embed_join_kernel<A, 1>;
    join<<<grid, kJoinSlots * kJoinParts * 32, 0, st>>>(start, ntok, nvocab, H, s.R, s.chunks, (A)scale,
                                                          accumulate != 0, dW, part, cut);
  }
  return launch_status(who);
}

}  // namespace
}  // namespace dpc

extern "C" {

size_t dp_embed_plan_work_bytes(int64_t ntok, int nvocab) {
  if (ntok < 0 || ntok > 0x7fffffffLL - dpc::kSortBlock || nvocab < 1 || nvocab > dpc::kMaxVocab) return 0;
  const dpc::SortShape s = dpc::sort_shape(ntok, nvocab);
  if (dpc::plan_is_small(ntok, nvocab)) return 1;
  return ((size_t)ntok * 4 + (size_t)(s.blocks + 1) * dpc::kDigits) * sizeof(int);
}

int dp_embed_plan(const int32_t *ids, int64_t ntok, int nvocab, int64_t *start, int32_t *src, void *work,
                  size_t work_bytes, void *stream) {
  using namespace dpc;
  const char *who = "dp_embed_plan";
  clear_error();
  int rc = embed_check(ntok, nvocab, who);
  if (rc) return rc;
  if (!start || (ntok > 0 && (!ids || !src))) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (!at_elements(ids, src) || !at_elements(start)) return misaligned(who);
  const SortShape s = sort_shape(ntok, nvocab);
  const cudaStream_t st = (cudaStream_t)stream;
  if (plan_is_small(ntok, nvocab)) {
    rc = allow_smem((const void *)embed_plan_small_kernel, kSmallSmem, who);
    if (rc) return rc;
    embed_plan_small_kernel<<<1, kSortThreads, kSmallSmem, st>>>(ids, (int)ntok, nvocab, s.passes, s.bits, start, src);
    return launch_status(who);
  }
  if (!work) return set_error(DP_ERR_NULL, "%s: work is NULL", who);
  if (work_bytes < dp_embed_plan_work_bytes(ntok, nvocab) || ((uintptr_t)work & 15))
    return set_error(DP_ERR_SHAPE, "%s: work buffer of %zu bytes is too short or misaligned", who, work_bytes);
  if (ntok <= (int64_t)kClusterBlocks * 8 * kSortThreads) {
    const int per = ntok <= (int64_t)kClusterBlocks * 4 * kSortThreads ? 4 : 8;
    cudaLaunchAttribute cluster{};
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = (unsigned)((ntok + per * kSortThreads - 1) / (per * kSortThreads));
    cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(cluster.val.clusterDim.x);
    cfg.blockDim = dim3(kSortThreads);
    cfg.stream = st;
    cfg.attrs = &cluster;
    cfg.numAttrs = 1;
    auto k = per == 4 ? embed_plan_cluster_kernel<4> : embed_plan_cluster_kernel<8>;
    uint32_t *keys = (uint32_t *)work;
    cudaLaunchKernelEx(&cfg, k, ids, (int)ntok, nvocab, s.passes, s.bits, keys, (int *)work + 2 * ntok, start, src);
    if (s.passes > 1 && nvocab > kClusterStart)
      embed_start_kernel<<<(nvocab + 256) / 256, 256, 0, st>>>(keys + (int64_t)((s.passes - 1) & 1) * ntok, (int)ntok,
                                                                 nvocab, start);
    return launch_status(who);
  }
  uint32_t *keys[2] = {(uint32_t *)work, (uint32_t *)work + ntok};
  int *idx[2] = {(int *)work + 2 * ntok, (int *)work + 3 * ntok}, *counts = (int *)work + 4 * ntok;
  int *totals = counts + (int64_t)s.blocks * kDigits;
  const int mask = (1 << s.bits) - 1;
  for (int pass = 0; pass < s.passes; ++pass) {
    const uint32_t *from = pass ? keys[(pass - 1) & 1] : nullptr;
    const int *from_idx = pass ? idx[(pass - 1) & 1] : nullptr;
    const bool last = pass == s.passes - 1;
    sort_count_kernel<<<s.blocks, kSortThreads, 0, st>>>(ids, from, ntok, nvocab, pass * s.bits, mask, counts);
    sort_scan_kernel<<<kDigits, kDigits, 0, st>>>(counts, s.blocks, totals);
    sort_place_kernel<<<s.blocks, kSortThreads, 0, st>>>(ids, from, from_idx, ntok, nvocab, pass * s.bits, s.bits, counts, totals,
                                                         keys[pass & 1], last ? src : idx[pass & 1], last);
  }
  embed_start_kernel<<<(nvocab + 256) / 256, 256, 0, st>>>(keys[(s.passes - 1) & 1], (int)ntok, nvocab, start);
  return launch_status(who);
}

size_t dp_embed_grad_work_bytes(int64_t ntok, int H, int elem_bytes) {
  if (ntok < 0 || ntok > 0x7fffffffLL - dpc::kSortBlock || H < 1 || H > dpc::kMaxH) return 0;
  if (elem_bytes != 2 && elem_bytes != 4 && elem_bytes != 8) return 0;
  const size_t n = dpc::part_bytes(ntok, H, elem_bytes);
  return n ? n : 1;
}

#define DP_EMBED(X, C, T, W_)                                                                                        \
  int dp_embed_fwd_##X(const C *W, const int32_t *ids, int64_t ntok, int nvocab, int H, double scale, const C *add,  \
                       C *y, void *stream) {                                                                         \
    return dpc::embed_fwd<T>((const T *)W, ids, ntok, nvocab, H, scale, (const T *)add, (T *)y, stream,              \
                             "dp_embed_fwd_" #X);                                                                    \
  }                                                                                                                  \
  int dp_embed_grad_##X(const C *dy, const int32_t *ids, const int64_t *start, const int32_t *src, int64_t ntok,     \
                        int nvocab, int H, double scale, int accumulate, W_ *dW, void *work, size_t work_bytes,      \
                        void *stream) {                                                                              \
    return dpc::embed_grad<T>((const T *)dy, ids, start, src, ntok, nvocab, H, scale, accumulate, dW, work,          \
                              work_bytes, stream, "dp_embed_grad_" #X);                                              \
  }
DP_EMBED(f64, double, double, double)
DP_EMBED(f32, float, float, float)
DP_EMBED(bf16, uint16_t, __nv_bfloat16, float)
DP_EMBED(f16, uint16_t, __half, float)

}  // extern "C"
