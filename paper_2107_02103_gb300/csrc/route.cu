// Tokens (atoms' feature rows) sorted by expert and back.  Pair q = t topk + j sends token t to expert
// expert[q]; an id outside [0, nexp) drops the pair.  The plan is a stable counting sort of the pairs by
// expert: start[e] the first sorted row of expert e, src[p] the pair at sorted row p (-1 past the kept
// ones), pos[q] the sorted row of pair q (-1 for a dropped one).  Then
//   gather   xs[p] = x[src[p] / topk]
//   combine  y[t]  = sum_j w[t][j] z[pos[t][j]]            (dropped pairs add nothing)
//   backward dz[p] = w_q dy[t],  dw_q = <dy[t], z[p]>;  the gather's backward is combine without weights.
// No atomics on the data: every output row has one writer and every sum a fixed order, so results repeat
// bit for bit.
// All are bound by memory.  Measured (12,288 x 2 rows of 1600 bf16): plan 8 us, gather 19 us (6.3 TB/s),
// combine 25 us (4.8 TB/s; 6.1 in f32, whose rows are longer), gradient 48 us; 16,384 x 2 x 1600 f32: 51, 51, 87 us.
// f64 12,288 x 2 x 1600: gather 74 (6.4 TB/s), combine 80 (5.9), gradient 247 us (3.2).
#include <cooperative_groups.h>

#include "rows.cuh"

namespace dpc {
namespace {

constexpr int kMaxExperts = 1024, kMaxTopk = 64;
constexpr int kPlanWarps = 32;

// The placing kernel's counters: a row of them a warp, the scan's sums, the block's counts.
constexpr size_t plan_smem(int nexp) { return (size_t)(kPlanWarps * nexp + kPlanWarps + nexp) * sizeof(int); }

// A thread's kPer expert ids, -1 for a dropped pair or past the end; warp w of a block has 32 kPer pairs in order.
template <int kPer>
struct PlanIds {
  int64_t first;  // the lane's first pair; the next are 32 apart
  int e[kPer];
  __device__ __forceinline__ PlanIds(const int32_t *expert, int64_t n, int nexp) {
    first = (((int64_t)blockIdx.x * kPlanWarps + (threadIdx.x >> 5)) * kPer) * 32 + (threadIdx.x & 31);
#pragma unroll
    for (int i = 0; i < kPer; ++i) e[i] = first + 32 * i < n ? __ldg(expert + first + 32 * i) : -1;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (e[i] >= nexp || e[i] < 0) e[i] = -1;
  }
};

// counts[b][e]: the kept pairs of expert e in block b's pairs (integer atomics: any order gives the same).
template <int kPer>
__global__ void __launch_bounds__(kPlanWarps * 32)
    plan_count_kernel(const int32_t *__restrict__ expert, int64_t n, int nexp, int *__restrict__ counts) {
  extern __shared__ int cnt[];
  for (int e = threadIdx.x; e < nexp; e += blockDim.x) cnt[e] = 0;
  __syncthreads();
  const PlanIds<kPer> ids(expert, n, nexp);
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (ids.e[i] >= 0) atomicAdd(cnt + ids.e[i], 1);
  __syncthreads();
  for (int e = threadIdx.x; e < nexp; e += blockDim.x) counts[(int64_t)blockIdx.x * nexp + e] = cnt[e];
}

// Every block sums the blocks' counts (its own prefix and the totals), scans the experts, then gives its pairs their
// places: a warp's pairs of an expert follow those of the warps before it, and lanes with the same expert are found
// with a match, so that a warp moves each counter once per 32 pairs.  One block counts by itself, up to eight form a
// cluster and read one another's counts (a single launch either way), more read a table that a launch before filled.
// That table's sums are taken anew by every block, nexp threads at work: 202 us for 2^23 pairs of 8 experts.
enum PlanCounts { kOwn, kCluster, kTable };
template <int kPer, PlanCounts kFrom>
__global__ void __launch_bounds__(kPlanWarps * 32)
    plan_place_kernel(const int32_t *__restrict__ expert, int64_t n, int nexp, const int *__restrict__ counts,
                      int64_t *__restrict__ start, int32_t *__restrict__ src, int32_t *__restrict__ pos) {
  extern __shared__ int cnt[];  // [warps][nexp], then the scan's warp sums, then the block's counts
  int *sums = cnt + kPlanWarps * nexp, *block = sums + kPlanWarps;
  namespace cg = cooperative_groups;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kPlanWarps * nexp; i += blockDim.x) cnt[i] = 0;
  const PlanIds<kPer> ids(expert, n, nexp);
  __syncthreads();
  int *mine = cnt + warp * nexp;
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (ids.e[i] >= 0) atomicAdd(mine + ids.e[i], 1);
  __syncthreads();
  if constexpr (kFrom == kCluster) {
    for (int e = threadIdx.x; e < nexp; e += blockDim.x) {
      int c = 0;
#pragma unroll 8
      for (int w = 0; w < kPlanWarps; ++w) c += cnt[w * nexp + e];
      block[e] = c;
    }
    cg::this_cluster().sync();
  }
  // an exclusive scan of the totals, an expert a thread
  static_assert(kMaxExperts <= kPlanWarps * 32, "an expert a thread");
  const int e = threadIdx.x;
  int total = 0, before = 0;
  if (e < nexp) {
    if constexpr (kFrom != kOwn) {
#pragma unroll 8
      for (int b = 0; b < (int)gridDim.x; ++b) {
        int c;
        if constexpr (kFrom == kTable) c = __ldg(counts + (int64_t)b * nexp + e);
        else c = cg::this_cluster().map_shared_rank(block, b)[e];
        before += b < (int)blockIdx.x ? c : 0;
        total += c;
      }
    } else {
#pragma unroll 8
      for (int w = 0; w < kPlanWarps; ++w) total += cnt[w * nexp + e];
    }
  }
  int inc = total;
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += up;
  }
  if (lane == 31) sums[warp] = inc;
  __syncthreads();
  const int before_warp = __reduce_add_sync(0xffffffffu, lane < warp ? sums[lane] : 0);
  const int kept = __reduce_add_sync(0xffffffffu, sums[lane]);
  if (e < nexp) {
    const int first = before_warp + inc - total;
    if (blockIdx.x == 0) start[e] = first;
    int run = first + before;  // from counts to each warp's next row of the expert
#pragma unroll 8
    for (int w = 0; w < kPlanWarps; ++w) {
      const int c = cnt[w * nexp + e];
      cnt[w * nexp + e] = run;
      run += c;
    }
  }
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) start[nexp] = kept;
  if constexpr (kFrom == kCluster) cg::this_cluster().sync();  // nobody leaves while its counts are read
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int64_t q = ids.first + 32 * i;
    if (q - lane >= n) break;  // warp-uniform
    const int own = ids.e[i];
    const unsigned same = __match_any_sync(0xffffffffu, own);
    const int p = own >= 0 ? mine[own] + __popc(same & ((1u << lane) - 1)) : -1;
    __syncwarp();
    if (own >= 0 && lane == __ffs(same) - 1) mine[own] += __popc(same);
    __syncwarp();
    if (q < n) {
      pos[q] = p;
      if (p >= 0) src[p] = (int32_t)q;
      if (q >= kept) src[q] = -1;
    }
  }
}

// Two ways over the rows.  Long rows: a warp takes one part of a token's row, kPart packs a lane, so that the
// token's pairs are read once by the warp and its loads are long.  Short rows (fewer packs than lanes): a thread
// takes one pack of any token, the packs in order over the tokens.
constexpr int kMoveThreads = 128, kPart = 4;

struct Unit {
  int64_t t;  // the token
  int c;      // the lane's first pack; further ones 32 apart
};
template <bool Flat, int kP = kPart>
__device__ __forceinline__ Unit unit_of(int np) {
  if constexpr (Flat) {
    const int64_t base = (int64_t)blockIdx.x * kMoveThreads, t0 = base / np;
    const uint32_t off = (uint32_t)(base - t0 * np) + threadIdx.x, dt = off / (uint32_t)np;
    return {t0 + dt, (int)(off - dt * np)};
  } else {
    return {(int64_t)blockIdx.x * (kMoveThreads / 32) + (threadIdx.x >> 5), (int)(blockIdx.y * 32 * kP + (threadIdx.x & 31))};
  }
}

// Accesses a lane has in flight of a row, V elements each: whole rows' packs, or single elements of other rows.  Reading
// the two aligned words under every 16 bytes of such rows instead (us, words and elements): combine of 30,011 x 3 x 1003
// f16 75, 48; gather of 20,000 x 2 x 701 bf16 19, 17, x 1003 f32 53, 43, but of 30,011 x 3 x 1003 f16 52, 60.
template <int V>
constexpr int kRowPart = V > 1 ? kPart : 8;

// xs rows of token t from one read of x[t]; also clears the rows past the kept ones that carry t's pair numbers.
template <typename T, int V, bool Flat>
__global__ void __launch_bounds__(kMoveThreads)
    gather_kernel(const T *__restrict__ x, const int32_t *__restrict__ src, const int32_t *__restrict__ pos,
                  int64_t ntok, int topk, int H, int np, T *__restrict__ xs) {
  constexpr int kP = Flat ? 1 : kRowPart<V>;
  const int64_t n = ntok * topk;
  const Unit u = unit_of<Flat, kRowPart<V>>(np);
  if (u.t >= ntok) return;
  const T *row = x + u.t * H;
  Pack<T, V> v[kP];
#pragma unroll
  for (int i = 0; i < kP; ++i)
    if (u.c + 32 * i < np) v[i] = load_pack<T, V>(row + (u.c + 32 * i) * V);
  for (int j = 0; j < topk; ++j) {
    const int64_t q = u.t * topk + j, p = __ldg(pos + q);
    if (p >= 0 && p < n)
#pragma unroll
      for (int i = 0; i < kP; ++i)
        if (u.c + 32 * i < np) store_pack<T, V>(xs + p * H + (u.c + 32 * i) * V, v[i]);
    if (__ldg(src + q) < 0)
#pragma unroll
      for (int i = 0; i < kP; ++i)
        if (u.c + 32 * i < np) store_pack<T, V>(xs + q * H + (u.c + 32 * i) * V, Pack<T, V>{});
  }
}

template <typename T, int V, bool Flat>
__global__ void __launch_bounds__(kMoveThreads)
    combine_kernel(const T *__restrict__ z, const int32_t *__restrict__ pos, const acc_t<T> *__restrict__ w,
                   int64_t ntok, int topk, int H, int np, T *__restrict__ y) {
  using A = acc_t<T>;
  constexpr int kP = Flat ? 1 : kRowPart<V>;
  const int64_t n = ntok * topk;
  const Unit u = unit_of<Flat, kRowPart<V>>(np);
  if (u.t >= ntok) return;
  A sum[kP][V] = {};
  for (int j = 0; j < topk; ++j) {
    const int64_t q = u.t * topk + j, p = __ldg(pos + q);
    if (p < 0 || p >= n) continue;
    const A wj = w ? __ldg(w + q) : A(1);
    const T *row = z + p * H;
    Pack<T, V> v[kP];
#pragma unroll
    for (int i = 0; i < kP; ++i)
      if (u.c + 32 * i < np) v[i] = load_pack<T, V>(row + (u.c + 32 * i) * V);
#pragma unroll
    for (int i = 0; i < kP; ++i)
#pragma unroll
      for (int l = 0; l < V; ++l) sum[i][l] = fma(wj, to_acc(v[i].v[l]), sum[i][l]);
  }
  T *to = y + u.t * H;
#pragma unroll
  for (int i = 0; i < kP; ++i)
    if (u.c + 32 * i < np) {
      Pack<T, V> o;
#pragma unroll
      for (int l = 0; l < V; ++l) o.v[l] = from_acc<T>(sum[i][l]);
      store_pack<T, V>(to + (u.c + 32 * i) * V, o);
    }
}

// Accesses a lane has in flight of either row.
template <int V>
constexpr int kGradPacks = V > 1 ? 4 : 8;

// Threads a block: more of a token's pairs in one block let rows read by elements find dy in L1 (30,011 x 3 rows of
// 1003 f16: 136 us against 183 in blocks of 128); whole rows do better in small blocks (48 us against 58 for 12,288
// x 2 of 1600 bf16).
template <int V>
constexpr int kGradThreads = V > 1 ? 128 : 256;

// G lanes a pair (8 to 256): its dz row and dot product (each lane's partial in order, then a
// fixed tree).  A token's pairs are neighbours, so that dy comes from memory once; a pair to itself leaves nothing
// to wait for but its own rows.
template <typename T, int V, int G>
__global__ void __launch_bounds__(G > kGradThreads<V> ? G : kGradThreads<V>)
    combine_grad_kernel(const T *__restrict__ z, const int32_t *__restrict__ src, const int32_t *__restrict__ pos,
                        const acc_t<T> *__restrict__ w, const T *__restrict__ dy, int64_t ntok, int topk, int H, int np,
                        T *__restrict__ dz, acc_t<T> *__restrict__ dw) {
  using A = acc_t<T>;
  constexpr int kPairs = G > kGradThreads<V> ? 1 : kGradThreads<V> / G, kW = G <= 32 ? 1 : G / 32, kP = kGradPacks<V>;
  __shared__ A part[kPairs][kW];
  const int tid = threadIdx.x % G, slot = threadIdx.x / G;
  const int64_t n = ntok * topk, q = (int64_t)blockIdx.x * kPairs + slot;
  A dot = A(0);
  if (q < n) {
    const T *g = dy + q / topk * H;
    Pack<T, V> gv[kP], zv[kP];
    auto upstream = [&](int s) {
#pragma unroll
      for (int i = 0; i < kP; ++i)
        if (s + i * G < np) gv[i] = load_pack<T, V>(g + (s + i * G) * V);
    };
    upstream(tid);  // on its way while the pair's place is read
    const int64_t p = __ldg(pos + q);
    if (p >= 0 && p < n) {
      const A wq = w ? __ldg(w + q) : A(1);
      const T *from = z + p * H;
      T *to = dz + p * H;
      for (int s = tid; s < np; s += kP * G) {
        if (s != tid) upstream(s);
        if (dw)
#pragma unroll
          for (int i = 0; i < kP; ++i)
            if (s + i * G < np) zv[i] = load_pack<T, V>(from + (s + i * G) * V);
#pragma unroll
        for (int i = 0; i < kP; ++i)
          if (s + i * G < np) {
            Pack<T, V> o;
#pragma unroll
            for (int l = 0; l < V; ++l) {
              if (dw) dot = fma(to_acc(gv[i].v[l]), to_acc(zv[i].v[l]), dot);
              o.v[l] = from_acc<T>(wq * to_acc(gv[i].v[l]));
            }
            store_pack<T, V>(to + (s + i * G) * V, o);
          }
      }
    }
    if (__ldg(src + q) < 0)
      for (int s = tid; s < np; s += G) store_pack<T, V>(dz + q * H + s * V, Pack<T, V>{});
  }
  if (dw) {  // launch-uniform; the dot of a dropped pair is 0
#pragma unroll
    for (int o = (G < 32 ? G : 32) / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
    if constexpr (G > 32) {
      if (threadIdx.x % 32 == 0) part[slot][tid / 32] = dot;
      __syncthreads();
      if (tid == 0) {
        dot = part[slot][0];
#pragma unroll
        for (int k = 1; k < kW; ++k) dot += part[slot][k];
      }
    }
    if (tid == 0 && q < n) dw[q] = dot;
  }
}

int route_check(int64_t ntok, int topk, const char *who) {
  if (ntok < 0) return set_error(DP_ERR_SHAPE, "%s: ntok = %lld", who, (long long)ntok);
  if (topk < 1 || topk > kMaxTopk) return set_error(DP_ERR_SHAPE, "%s: topk = %d outside [1, %d]", who, topk, kMaxTopk);
  if (ntok > 0x7fffffffLL / topk)
    return set_error(DP_ERR_SHAPE, "%s: %lld tokens x %d pairs exceed 2^31", who, (long long)ntok, topk);
  return DP_OK;
}

int row_check(int64_t ntok, int topk, int H, const char *who) {
  const int rc = route_check(ntok, topk, who);
  if (rc) return rc;
  if (H < 1 || H > (1 << 20)) return set_error(DP_ERR_SHAPE, "%s: row length %d outside [1, 2^20]", who, H);
  return DP_OK;
}

// Blocks of the plan and pairs a thread (whose walk costs 0.3 us each): a cluster of up to eight blocks where that
// holds the pairs, else two launches (24,576 pairs: 8 us in a cluster, 11 in two launches).
struct PlanShape {
  int blocks, per;
};
PlanShape plan_shape(int64_t n) {
  if (n <= 8 * 4096) return {(int)((n + 4095) / 4096 < 1 ? 1 : (n + 4095) / 4096), 4};
  if (n <= 304 * 4096) return {(int)((n + 4095) / 4096), 4};
  return {(int)((n + 8191) / 8192), 8};
}

template <typename T>
bool whole_rows(int H, const void *a, const void *b, const void *c = nullptr) {
  return ((((uintptr_t)a | (uintptr_t)b | (uintptr_t)c) | (uintptr_t)(H * sizeof(T))) & 15) == 0;
}
// The grid of a move over rows of np packs; false where it is too large.
bool move_grid(int64_t ntok, int np, bool flat, int part, dim3 *grid) {
  const int64_t x = flat ? (ntok * np + kMoveThreads - 1) / kMoveThreads : (ntok + kMoveThreads / 32 - 1) / (kMoveThreads / 32);
  const int64_t y = flat ? 1 : (np + 32 * part - 1) / (32 * part);
  *grid = dim3((unsigned)x, (unsigned)y);
  return x <= 0x7fffffffLL && y <= 65535;
}

template <typename T>
int gather(const T *x, const int32_t *src, const int32_t *pos, int64_t ntok, int topk, int H, T *xs, void *stream,
           const char *who) {
  clear_error();
  int rc = row_check(ntok, topk, H, who);
  if (rc || ntok == 0) return rc;
  if (!x || !src || !pos || !xs) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (!at_elements(x, xs, src, pos)) return misaligned(who);
  constexpr int V = 16 / (int)sizeof(T);
  const bool whole = whole_rows<T>(H, x, xs);
  const int np = whole ? H / V : H;
  dim3 grid;
  if (!move_grid(ntok, np, np < 32, whole ? kRowPart<V> : kRowPart<1>, &grid))
    return set_error(DP_ERR_SHAPE, "%s: %lld rows of %d", who, (long long)ntok, H);
  auto k = np < 32 ? (whole ? gather_kernel<T, V, true> : gather_kernel<T, 1, true>)
                   : (whole ? gather_kernel<T, V, false> : gather_kernel<T, 1, false>);
  k<<<grid, kMoveThreads, 0, (cudaStream_t)stream>>>(x, src, pos, ntok, topk, H, np, xs);
  return launch_status(who);
}

template <typename T>
int combine(const T *z, const int32_t *pos, const acc_t<T> *w, int64_t ntok, int topk, int H, T *y, void *stream,
            const char *who) {
  clear_error();
  int rc = row_check(ntok, topk, H, who);
  if (rc || ntok == 0) return rc;
  if (!z || !pos || !y) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (!at_elements(z, y, pos, w)) return misaligned(who);
  constexpr int V = 16 / (int)sizeof(T);
  const bool whole = whole_rows<T>(H, z, y);
  const int np = whole ? H / V : H;
  dim3 grid;
  if (!move_grid(ntok, np, np < 32, whole ? kRowPart<V> : kRowPart<1>, &grid))
    return set_error(DP_ERR_SHAPE, "%s: %lld rows of %d", who, (long long)ntok, H);
  auto k = np < 32 ? (whole ? combine_kernel<T, V, true> : combine_kernel<T, 1, true>)
                   : (whole ? combine_kernel<T, V, false> : combine_kernel<T, 1, false>);
  k<<<grid, kMoveThreads, 0, (cudaStream_t)stream>>>(z, pos, w, ntok, topk, H, np, y);
  return launch_status(who);
}

template <typename T>
int combine_grad(const T *z, const int32_t *src, const int32_t *pos, const acc_t<T> *w, const T *dy, int64_t ntok,
                 int topk, int H, T *dz, acc_t<T> *dw, void *stream, const char *who) {
  clear_error();
  int rc = row_check(ntok, topk, H, who);
  if (rc || ntok == 0) return rc;
  if (!src || !pos || !dy || !dz || (dw && !z)) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  const T *zr = dw ? z : nullptr;
  if (!at_elements(zr, dy, dz, dw) || !at_elements(src, pos, w)) return misaligned(who);
  constexpr int V = 16 / (int)sizeof(T);
  const bool whole = whole_rows<T>(H, zr, dy, dz);
  const int np = whole ? H / V : H, each = whole ? kGradPacks<V> : kGradPacks<1>;
  auto go = [&](auto G) {
    constexpr int g_ = decltype(G)::value;
    int threads = whole ? kGradThreads<V> : kGradThreads<1>;
    threads = threads < g_ ? g_ : threads;
    const int pairs = threads / g_;
    auto k = whole ? combine_grad_kernel<T, V, g_> : combine_grad_kernel<T, 1, g_>;
    k<<<(unsigned)((ntok * topk + pairs - 1) / pairs), threads, 0, (cudaStream_t)stream>>>(z, src, pos, w, dy, ntok, topk,
                                                                                           H, np, dz, dw);
  };
  if (np <= 8 * each) go(std::integral_constant<int, 8>{});  // as many lanes as hold the row
  else if (np <= 32 * each) go(std::integral_constant<int, 32>{});
  else if (np <= 64 * each) go(std::integral_constant<int, 64>{});
  else if (np <= 128 * each) go(std::integral_constant<int, 128>{});
  else go(std::integral_constant<int, 256>{});
  return launch_status(who);
}

}  // namespace
}  // namespace dpc

extern "C" {

size_t dp_route_work_bytes(int64_t ntok, int topk, int nexp) {
  if (ntok < 0 || topk < 1 || topk > dpc::kMaxTopk || nexp < 1 || nexp > dpc::kMaxExperts || ntok > 0x7fffffffLL / topk)
    return 0;
  const dpc::PlanShape s = dpc::plan_shape(ntok * topk);
  return s.blocks > 8 ? (size_t)s.blocks * nexp * sizeof(int) : 1;
}

int dp_route_plan(const int32_t *expert, int64_t ntok, int topk, int nexp, int64_t *start, int32_t *src, int32_t *pos,
                  void *work, size_t work_bytes, void *stream) {
  using namespace dpc;
  const char *who = "dp_route_plan";
  clear_error();
  int rc = route_check(ntok, topk, who);
  if (rc) return rc;
  if (nexp < 1) return set_error(DP_ERR_SHAPE, "%s: nexp = %d", who, nexp);
  if (nexp > kMaxExperts) return set_error(DP_ERR_UNSUPPORTED, "%s: nexp = %d > %d", who, nexp, kMaxExperts);
  if (!start || (ntok > 0 && (!expert || !src || !pos))) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (!at_elements(expert, start, src, pos)) return misaligned(who);
  const PlanShape s = plan_shape(ntok * topk);
  if (s.blocks > 8) {
    if (!work) return set_error(DP_ERR_NULL, "%s: work is NULL", who);
    if (work_bytes < dp_route_work_bytes(ntok, topk, nexp) || ((uintptr_t)work & 15))
      return set_error(DP_ERR_SHAPE, "%s: work buffer of %zu bytes is too short or misaligned", who, work_bytes);
  }
  const size_t smem = plan_smem(nexp);
  const cudaStream_t st = (cudaStream_t)stream;
  const int64_t n = ntok * topk;
  int *counts = s.blocks > 8 ? (int *)work : nullptr;
  auto place = s.blocks == 1  ? plan_place_kernel<4, kOwn>
               : !counts      ? plan_place_kernel<4, kCluster>
               : s.per == 4   ? plan_place_kernel<4, kTable>
                              : plan_place_kernel<8, kTable>;
  if (smem > 48 * 1024) {
    rc = allow_smem((const void *)place, plan_smem(kMaxExperts), who);
    if (rc) return rc;
  }
  if (counts) {
    auto count = s.per == 8 ? plan_count_kernel<8> : plan_count_kernel<4>;
    count<<<s.blocks, kPlanWarps * 32, nexp * sizeof(int), st>>>(expert, n, nexp, counts);
  }
  if (s.blocks == 1 || counts) {
    place<<<s.blocks, kPlanWarps * 32, smem, st>>>(expert, n, nexp, counts, start, src, pos);
  } else {
    cudaLaunchAttribute cluster{};
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = s.blocks;
    cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(s.blocks);
    cfg.blockDim = dim3(kPlanWarps * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &cluster;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, place, expert, n, nexp, (const int *)counts, start, src, pos);
  }
  return launch_status(who);
}

#define DP_ROUTE(X, C, T, W)                                                                                          \
  int dp_route_gather_##X(const C *x, const int32_t *src, const int32_t *pos, int64_t ntok, int topk, int H, C *xs,   \
                          void *stream) {                                                                             \
    return dpc::gather<T>((const T *)x, src, pos, ntok, topk, H, (T *)xs, stream, "dp_route_gather_" #X);             \
  }                                                                                                                   \
  int dp_route_combine_##X(const C *z, const int32_t *pos, const W *w, int64_t ntok, int topk, int H, C *y,           \
                           void *stream) {                                                                            \
    return dpc::combine<T>((const T *)z, pos, w, ntok, topk, H, (T *)y, stream, "dp_route_combine_" #X);              \
  }                                                                                                                   \
  int dp_route_combine_grad_##X(const C *z, const int32_t *src, const int32_t *pos, const W *w, const C *dy,          \
                                int64_t ntok, int topk, int H, C *dz, W *dw, void *stream) {                          \
    return dpc::combine_grad<T>((const T *)z, src, pos, w, (const T *)dy, ntok, topk, H, (T *)dz, dw, stream,         \
                                "dp_route_combine_grad_" #X);                                                         \
  }
DP_ROUTE(f64, double, double, double)
DP_ROUTE(f32, float, float, float)
DP_ROUTE(bf16, uint16_t, __nv_bfloat16, float)
DP_ROUTE(f16, uint16_t, __half, float)

}  // extern "C"
