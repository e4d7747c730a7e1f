// Tokens (atoms' feature rows) sorted by expert and back.  Pair q = t topk + j sends token t to expert
// expert[q]; an id outside [0, nexp) drops the pair.  The plan is a stable counting sort of the pairs by
// expert: start[e] the first sorted row of expert e, src[p] the pair at sorted row p (-1 past the kept
// ones), pos[q] the sorted row of pair q (-1 for a dropped one).  Then
//   gather   xs[p] = x[src[p] / topk]
//   combine  y[t]  = sum_j w[t][j] z[pos[t][j]]            (dropped pairs add nothing)
//   backward dz[p] = w_q dy[t],  dw_q = <dy[t], z[p]>;  the gather's backward is combine without weights.
// No atomics on the data: every output row has one writer and every sum a fixed order, so results repeat
// bit for bit.
#include "rows.cuh"

namespace dpc {
namespace {

constexpr int kMaxExperts = 1024, kMaxTopk = 64;
constexpr int kPlanWarps = 16;

// One warp's part of a block's pairs: cnt[e] += the pairs of expert e among [lo, hi).  Lanes with the same
// expert are found with a match, so that a warp adds each expert once per 32 pairs, without atomics.
__device__ __forceinline__ void warp_count(const int32_t *expert, int64_t lo, int64_t hi, int nexp, int *cnt, int lane) {
  for (int64_t q0 = lo; q0 < hi; q0 += 32) {
    const int64_t q = q0 + lane;
    int e = q < hi ? __ldg(expert + q) : -1;
    if (e < 0 || e >= nexp) e = -1;
    const unsigned same = __match_any_sync(0xffffffffu, e);
    if (e >= 0 && lane == __ffs(same) - 1) cnt[e] += __popc(same);
    __syncwarp();
  }
}

// counts[b][e]: the kept pairs of expert e in block b's chunk.
__global__ void __launch_bounds__(kPlanWarps * 32)
    plan_count_kernel(const int32_t *__restrict__ expert, int64_t n, int64_t chunk, int nexp, int *__restrict__ counts) {
  extern __shared__ int cnt[];  // [warps][nexp]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kPlanWarps * nexp; i += blockDim.x) cnt[i] = 0;
  __syncthreads();
  const int64_t b0 = blockIdx.x * chunk, b1 = min(b0 + chunk, n), part = chunk / kPlanWarps;
  warp_count(expert, b0 + warp * part, min(b0 + (warp + 1) * part, b1), nexp, cnt + warp * nexp, lane);
  __syncthreads();
  for (int e = threadIdx.x; e < nexp; e += blockDim.x) {
    int s = 0;
    for (int w = 0; w < kPlanWarps; ++w) s += cnt[w * nexp + e];
    counts[(int64_t)blockIdx.x * nexp + e] = s;
  }
}

// Every block sums the count table again (its own prefix and the totals), scans the experts, then walks its
// pairs in order and writes src and pos.  With one block (counts NULL) it counts by itself: a single launch.
__global__ void __launch_bounds__(kPlanWarps * 32)
    plan_place_kernel(const int32_t *__restrict__ expert, int64_t n, int64_t chunk, int nexp,
                      const int *__restrict__ counts, int64_t *__restrict__ start, int32_t *__restrict__ src,
                      int32_t *__restrict__ pos) {
  extern __shared__ int cnt[];  // [warps][nexp], then base[nexp + 1], then the scan's warp sums
  int *base = cnt + kPlanWarps * nexp, *sums = base + nexp + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kPlanWarps * nexp; i += blockDim.x) cnt[i] = 0;
  __syncthreads();
  const int64_t b0 = blockIdx.x * chunk, b1 = min(b0 + chunk, n), part = chunk / kPlanWarps;
  const int64_t w0 = b0 + warp * part, w1 = min(w0 + part, b1);
  warp_count(expert, w0, w1, nexp, cnt + warp * nexp, lane);
  __syncthreads();
  // totals and this block's prefix per expert; an exclusive scan of the totals, kPlanWarps * 32 experts at a time
  int carry = 0;
  for (int e0 = 0; e0 < nexp; e0 += kPlanWarps * 32) {
    const int e = e0 + threadIdx.x;
    int total = 0, before = 0;
    if (e < nexp) {
      if (counts) {
        for (int b = 0; b < (int)gridDim.x; ++b) {
          const int c = __ldg(counts + (int64_t)b * nexp + e);
          before += b < (int)blockIdx.x ? c : 0;
          total += c;
        }
      } else {
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
    int off = carry;
    for (int w = 0; w < kPlanWarps; ++w) {
      off += w < warp ? sums[w] : 0;
      carry += sums[w];
    }
    if (e < nexp) {
      const int first = off + inc - total;
      if (blockIdx.x == 0) start[e] = first;
      int run = first + before;  // from counts to each warp's next row of the expert
      for (int w = 0; w < kPlanWarps; ++w) {
        const int c = cnt[w * nexp + e];
        cnt[w * nexp + e] = run;
        run += c;
      }
    }
    __syncthreads();
  }
  const int kept = carry;
  if (blockIdx.x == 0 && threadIdx.x == 0) start[nexp] = kept;
  int *next = cnt + warp * nexp;
  for (int64_t q0 = w0; q0 < w1; q0 += 32) {
    const int64_t q = q0 + lane;
    int e = q < w1 ? __ldg(expert + q) : -1;
    if (e < 0 || e >= nexp) e = -1;
    const unsigned same = __match_any_sync(0xffffffffu, e);
    const int p = e >= 0 ? next[e] + __popc(same & ((1u << lane) - 1)) : -1;
    __syncwarp();
    if (e >= 0 && lane == __ffs(same) - 1) next[e] += __popc(same);
    __syncwarp();
    if (q < w1) {
      pos[q] = p;
      if (p >= 0) src[p] = (int32_t)q;
      if (q >= kept) src[q] = -1;
    }
  }
}

constexpr int kRowWarps = 4, kSegPacks = 4;  // packs a lane has in flight; a warp moves 32 * kSegPacks of a row

// xs rows of token t from one read of x[t]; also clears the rows past the kept ones that carry t's pair numbers.
template <typename T, int V>
__global__ void __launch_bounds__(kRowWarps * 32)
    gather_kernel(const T *__restrict__ x, const int32_t *__restrict__ src, const int32_t *__restrict__ pos,
                  int64_t ntok, int topk, int H, T *__restrict__ xs) {
  const int lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * kRowWarps + (threadIdx.x >> 5), n = ntok * topk;
  if (t >= ntok) return;
  const int np = H / V, c0 = blockIdx.y * (32 * kSegPacks) + lane;
  Pack<T, V> v[kSegPacks];
#pragma unroll
  for (int i = 0; i < kSegPacks; ++i)
    if (c0 + 32 * i < np) v[i] = load_pack<T, V>(x + t * H + (int64_t)(c0 + 32 * i) * V);
  for (int j = 0; j < topk; ++j) {
    const int64_t p = __ldg(pos + t * topk + j);
    if (p >= 0 && p < n)
#pragma unroll
      for (int i = 0; i < kSegPacks; ++i)
        if (c0 + 32 * i < np) store_pack<T, V>(xs + p * H + (int64_t)(c0 + 32 * i) * V, v[i]);
  }
  for (int j = 0; j < topk; ++j) {
    const int64_t p = t * topk + j;
    if (__ldg(src + p) < 0)
#pragma unroll
      for (int i = 0; i < kSegPacks; ++i)
        if (c0 + 32 * i < np) store_pack<T, V>(xs + p * H + (int64_t)(c0 + 32 * i) * V, Pack<T, V>{});
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(kRowWarps * 32)
    combine_kernel(const T *__restrict__ z, const int32_t *__restrict__ pos, const acc_t<T> *__restrict__ w,
                   int64_t ntok, int topk, int H, T *__restrict__ y) {
  using A = acc_t<T>;
  const int lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * kRowWarps + (threadIdx.x >> 5), n = ntok * topk;
  if (t >= ntok) return;
  const int np = H / V, c0 = blockIdx.y * (32 * kSegPacks) + lane;
  A sum[kSegPacks][V];
#pragma unroll
  for (int i = 0; i < kSegPacks; ++i)
#pragma unroll
    for (int l = 0; l < V; ++l) sum[i][l] = A(0);
  for (int j = 0; j < topk; ++j) {
    const int64_t p = __ldg(pos + t * topk + j);
    if (p < 0 || p >= n) continue;
    const A wj = w ? __ldg(w + t * topk + j) : A(1);
    Pack<T, V> v[kSegPacks];
#pragma unroll
    for (int i = 0; i < kSegPacks; ++i)
      if (c0 + 32 * i < np) v[i] = load_pack<T, V>(z + p * H + (int64_t)(c0 + 32 * i) * V);
#pragma unroll
    for (int i = 0; i < kSegPacks; ++i)
#pragma unroll
      for (int l = 0; l < V; ++l) sum[i][l] = fma(wj, to_acc(v[i].v[l]), sum[i][l]);
  }
#pragma unroll
  for (int i = 0; i < kSegPacks; ++i)
    if (c0 + 32 * i < np) {
      Pack<T, V> o;
#pragma unroll
      for (int l = 0; l < V; ++l) o.v[l] = from_acc<T>(sum[i][l]);
      store_pack<T, V>(y + t * H + (int64_t)(c0 + 32 * i) * V, o);
    }
}

constexpr int kGradThreads = 128;

// A block per token: dz rows and the dot products for dw (each lane's partial in order, then a fixed tree).
template <typename T, int V>
__global__ void __launch_bounds__(kGradThreads)
    combine_grad_kernel(const T *__restrict__ z, const int32_t *__restrict__ src, const int32_t *__restrict__ pos,
                        const acc_t<T> *__restrict__ w, const T *__restrict__ dy, int64_t ntok, int topk, int H,
                        T *__restrict__ dz, acc_t<T> *__restrict__ dw) {
  using A = acc_t<T>;
  __shared__ A part[kGradThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, np = H / V;
  const int64_t t = blockIdx.x, n = ntok * topk;
  for (int j = 0; j < topk; ++j) {
    const int64_t p = __ldg(pos + t * topk + j);
    const bool in = p >= 0 && p < n;
    A dot = A(0);
    if (in) {
      const A wj = w ? __ldg(w + t * topk + j) : A(1);
      for (int c = threadIdx.x; c < np; c += kGradThreads) {
        const Pack<T, V> g = load_pack<T, V>(dy + t * H + (int64_t)c * V);
        Pack<T, V> o;
        if (dw) {
          const Pack<T, V> v = load_pack<T, V>(z + p * H + (int64_t)c * V);
#pragma unroll
          for (int l = 0; l < V; ++l) dot = fma(to_acc(g.v[l]), to_acc(v.v[l]), dot);
        }
#pragma unroll
        for (int l = 0; l < V; ++l) o.v[l] = from_acc<T>(wj * to_acc(g.v[l]));
        store_pack<T, V>(dz + p * H + (int64_t)c * V, o);
      }
    }
    if (dw) {  // launch-uniform
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
      if (lane == 0) part[warp] = dot;
      __syncthreads();
      if (threadIdx.x == 0) {
        A s = part[0];
        for (int k = 1; k < kGradThreads / 32; ++k) s += part[k];
        dw[t * topk + j] = in ? s : A(0);
      }
      __syncthreads();
    }
    const int64_t q = t * topk + j;
    if (__ldg(src + q) < 0)
      for (int c = threadIdx.x; c < np; c += kGradThreads) store_pack<T, V>(dz + q * H + (int64_t)c * V, Pack<T, V>{});
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

// Calls f(std::integral_constant<int, V>) for the pack width V in {16, 8, 4, 2, 1 bytes} / sizeof(T).
template <typename T, typename F>
void with_pack(int v, F f) {
  if constexpr (sizeof(T) == 2)
    if (v == 8) return f(std::integral_constant<int, 8>{});
  if constexpr (sizeof(T) <= 4)
    if (v == 4) return f(std::integral_constant<int, 4>{});
  if (v == 2) return f(std::integral_constant<int, 2>{});
  f(std::integral_constant<int, 1>{});
}

// Blocks of the plan: one while a block's pass over the pairs costs less than a second launch, else chunks of
// at least 2048 pairs, at most 304 blocks (two per SM; each reads the whole count table).
struct PlanShape {
  int blocks;
  int64_t chunk;
};
PlanShape plan_shape(int64_t n) {
  int64_t blocks = n <= 8192 ? 1 : (n + 2047) / 2048;
  blocks = blocks > 304 ? 304 : blocks < 1 ? 1 : blocks;
  int64_t chunk = (n + blocks - 1) / blocks;
  chunk = (chunk + kPlanWarps * 32 - 1) / (kPlanWarps * 32) * (kPlanWarps * 32);
  if (chunk < kPlanWarps * 32) chunk = kPlanWarps * 32;
  return {(int)((n + chunk - 1) / chunk < 1 ? 1 : (n + chunk - 1) / chunk), chunk};
}

template <typename T>
int gather(const T *x, const int32_t *src, const int32_t *pos, int64_t ntok, int topk, int H, T *xs, void *stream,
           const char *who) {
  clear_error();
  int rc = row_check(ntok, topk, H, who);
  if (rc || ntok == 0) return rc;
  if (!x || !src || !pos || !xs) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  const int v = pack_width<T>(H, x, xs);
  if (!v) return set_error(DP_ERR_SHAPE, "%s: an array is not aligned to its elements", who);
  with_pack<T>(v, [&](auto V) {
    const dim3 grid((unsigned)((ntok + kRowWarps - 1) / kRowWarps), (H / V + 32 * kSegPacks - 1) / (32 * kSegPacks));
    gather_kernel<T, V><<<grid, kRowWarps * 32, 0, (cudaStream_t)stream>>>(x, src, pos, ntok, topk, H, xs);
  });
  return launch_status(who);
}

template <typename T>
int combine(const T *z, const int32_t *pos, const acc_t<T> *w, int64_t ntok, int topk, int H, T *y, void *stream,
            const char *who) {
  clear_error();
  int rc = row_check(ntok, topk, H, who);
  if (rc || ntok == 0) return rc;
  if (!z || !pos || !y) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  const int v = pack_width<T>(H, z, y);
  if (!v) return set_error(DP_ERR_SHAPE, "%s: an array is not aligned to its elements", who);
  with_pack<T>(v, [&](auto V) {
    const dim3 grid((unsigned)((ntok + kRowWarps - 1) / kRowWarps), (H / V + 32 * kSegPacks - 1) / (32 * kSegPacks));
    combine_kernel<T, V><<<grid, kRowWarps * 32, 0, (cudaStream_t)stream>>>(z, pos, w, ntok, topk, H, y);
  });
  return launch_status(who);
}

template <typename T>
int combine_grad(const T *z, const int32_t *src, const int32_t *pos, const acc_t<T> *w, const T *dy, int64_t ntok,
                 int topk, int H, T *dz, acc_t<T> *dw, void *stream, const char *who) {
  clear_error();
  int rc = row_check(ntok, topk, H, who);
  if (rc || ntok == 0) return rc;
  if (!src || !pos || !dy || !dz || (dw && !z)) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  const int v = pack_width<T>(H, dw ? z : nullptr, dy, dz);
  if (!v) return set_error(DP_ERR_SHAPE, "%s: an array is not aligned to its elements", who);
  with_pack<T>(v, [&](auto V) {
    combine_grad_kernel<T, V><<<(unsigned)ntok, kGradThreads, 0, (cudaStream_t)stream>>>(z, src, pos, w, dy, ntok, topk,
                                                                                         H, dz, dw);
  });
  return launch_status(who);
}

}  // namespace
}  // namespace dpc

extern "C" {

size_t dp_route_work_bytes(int64_t ntok, int topk, int nexp) {
  if (ntok < 0 || topk < 1 || topk > dpc::kMaxTopk || nexp < 1 || nexp > dpc::kMaxExperts || ntok > 0x7fffffffLL / topk)
    return 0;
  const dpc::PlanShape s = dpc::plan_shape(ntok * topk);
  return s.blocks > 1 ? (size_t)s.blocks * nexp * sizeof(int) : 16;
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
  const PlanShape s = plan_shape(ntok * topk);
  if (s.blocks > 1) {
    if (!work) return set_error(DP_ERR_NULL, "%s: work is NULL", who);
    if (work_bytes < dp_route_work_bytes(ntok, topk, nexp) || ((uintptr_t)work & 15))
      return set_error(DP_ERR_SHAPE, "%s: work buffer of %zu bytes is too short or misaligned", who, work_bytes);
  }
  const size_t smem = (size_t)(kPlanWarps * nexp + nexp + 1 + kPlanWarps) * sizeof(int);
  const cudaStream_t st = (cudaStream_t)stream;
  if (smem > 48 * 1024) {
    const cudaError_t a = cudaFuncSetAttribute(plan_count_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    const cudaError_t b = cudaFuncSetAttribute(plan_place_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (a != cudaSuccess || b != cudaSuccess) return set_error(DP_ERR_CUDA, "%s: %zu bytes of shared memory", who, smem);
  }
  int *counts = s.blocks > 1 ? (int *)work : nullptr;
  if (counts) plan_count_kernel<<<s.blocks, kPlanWarps * 32, smem, st>>>(expert, ntok * topk, s.chunk, nexp, counts);
  plan_place_kernel<<<s.blocks, kPlanWarps * 32, smem, st>>>(expert, ntok * topk, s.chunk, nexp, counts, start, src, pos);
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
