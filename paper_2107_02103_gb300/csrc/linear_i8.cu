// Matrix product in 8-bit integers with a scale for each token (row of x) and each output channel (row of W),
// for one net or for several experts over rows sorted by expert:
//   amax_i = max_k |x_ik|, r_i = 127 / amax_i, q_ik = rint(x_ik r_i), sx_i = amax_i / 127        (f32 arithmetic)
//   y_in = act(float(sum_k q_ik w_nk) sx_i sw_n + b_n)
// The integer sum is exact.
#include "rows.cuh"

namespace dpc {
namespace {

constexpr int kMaxTopk = 64;
constexpr int kMaxK = 65536;  // |q w| <= 2^14: int32 sums hold 2^17 of them

// ------------------------------------------------------------------ rows to 8 bits
constexpr int kQuantKeep = 4;  // packs a thread keeps in registers; longer rows are read again (from L2)

// A row per block of TPR threads.  With pos, token t's row goes to the topk sorted rows pos[t][.], and the
// rows past the kept ones (src < 0) are cleared.
template <typename T, int V>
__global__ void quant_rows_kernel(const T *__restrict__ x, const int32_t *__restrict__ src,
                                  const int32_t *__restrict__ pos, int64_t ntok, int topk, int K, int ldq,
                                  int8_t *__restrict__ xq, float *__restrict__ sx) {
  __shared__ unsigned part[32];
  const int64_t t = blockIdx.x, n = ntok * topk;
  const T *row = x + t * K;
  const int np = K / V;
  Pack<T, V> keep[kQuantKeep];
  unsigned most = 0;  // the largest |x| as bits: infinities and NaN come out on top
#pragma unroll
  for (int i = 0; i < kQuantKeep; ++i) {
    const int c = threadIdx.x + i * blockDim.x;
    if (c < np) keep[i] = load_pack<T, V>(row + (int64_t)c * V);
  }
#pragma unroll
  for (int i = 0; i < kQuantKeep; ++i)
    if (threadIdx.x + i * blockDim.x < np)
#pragma unroll
      for (int l = 0; l < V; ++l) most = max(most, __float_as_uint((float)to_acc(keep[i].v[l])) & 0x7fffffffu);
  for (int c = threadIdx.x + kQuantKeep * blockDim.x; c < np; c += blockDim.x) {
    const Pack<T, V> v = load_pack<T, V>(row + (int64_t)c * V);
#pragma unroll
    for (int l = 0; l < V; ++l) most = max(most, __float_as_uint((float)to_acc(v.v[l])) & 0x7fffffffu);
  }
  most = __reduce_max_sync(0xffffffffu, most);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = most;
  __syncthreads();
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) most = max(most, part[w]);
  const float amax = __uint_as_float(most);
  const bool fine = most < 0x7f800000u && amax >= 0x1p-100f;
  const float r = fine ? __fdiv_rn(127.0f, amax) : 0.0f;
  const float s = fine ? __fdiv_rn(amax, 127.0f) : most < 0x7f800000u ? 0.0f : __uint_as_float(0x7fc00000u);
  auto put = [&](int64_t p, int c, const Pack<int8_t, V> &q) { store_pack<int8_t, V>(xq + p * ldq + (int64_t)c * V, q); };
  for (int c = threadIdx.x, i = 0; c < np; c += blockDim.x, ++i) {
    Pack<T, V> v;
    if (i < kQuantKeep) {
#pragma unroll
      for (int k = 0; k < kQuantKeep; ++k)
        if (k == i) v = keep[k];
    } else {
      v = load_pack<T, V>(row + (int64_t)c * V);
    }
    Pack<int8_t, V> q;
#pragma unroll
    for (int l = 0; l < V; ++l) q.v[l] = fine ? (int8_t)__float2int_rn((float)to_acc(v.v[l]) * r) : (int8_t)0;
    if (!pos) put(t, c, q);
    else
      for (int j = 0; j < topk; ++j) {
        const int64_t p = __ldg(pos + t * topk + j);
        if (p >= 0 && p < n) put(p, c, q);
      }
  }
  // the padding columns, the scales, and the rows past the kept ones
  const int64_t rows = pos ? topk : 1;
  for (int64_t j = 0; j < rows; ++j) {
    const int64_t q = t * rows + j, p = pos ? __ldg(pos + q) : t;
    if (p >= 0 && p < n) {
      for (int c = K + threadIdx.x; c < ldq; c += blockDim.x) xq[p * ldq + c] = 0;
      if (threadIdx.x == 0) sx[p] = s;
    }
    if (pos && __ldg(src + q) < 0) {
      for (int c = threadIdx.x; c < ldq / 16; c += blockDim.x) reinterpret_cast<uint4 *>(xq + q * ldq)[c] = make_uint4(0, 0, 0, 0);
      if (threadIdx.x == 0) sx[q] = 0.0f;
    }
  }
}

// ------------------------------------------------------------------ the product
struct I8Args {
  const int8_t *xq, *wq;
  const float *sx, *sw, *bias;
  const int64_t *start;  // [nexp + 1], or NULL: one expert for all rows
  int64_t rows;
  int K, N, nexp, act;
  void *y;
};

template <typename T>
__device__ __forceinline__ void put_out(T *y, float v) {
  if constexpr (sizeof(T) == 8) *y = (double)v;
  else *y = from_acc<T>(v);
}

// Row tile `tile` of the sorted rows cut into tiles of at most R rows that lie in one expert: the expert (nexp for
// the rows past start[nexp]) and its rows [r0, r1).  A warp looks at 32 experts at a time.
__device__ __forceinline__ bool find_tile(const I8Args &p, int64_t tile, int R, int &e, int64_t &r0, int64_t &r1) {
  if (!p.start) {
    e = 0;
    r0 = tile * R;
    r1 = min(r0 + R, p.rows);
    return r0 < p.rows;
  }
  const int lane = threadIdx.x & 31;
  int64_t before = 0;
  for (int e0 = 0; e0 <= p.nexp; e0 += 32) {
    const int k = e0 + lane;
    int64_t lo = 0, hi = 0;
    if (k <= p.nexp) {
      lo = k ? min(max(__ldg(p.start + k), (int64_t)0), p.rows) : 0;
      hi = k < p.nexp ? min(max(__ldg(p.start + k + 1), lo), p.rows) : p.rows;
    }
    const int64_t mine = (hi - lo + R - 1) / R;
    int64_t inc = mine;
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, before + inc > tile);
    if (hit) {
      const int who = __ffs(hit) - 1;
      const int64_t first = lo + (tile - (before + inc - mine)) * R;
      e = e0 + who;
      r0 = __shfl_sync(0xffffffffu, first, who);
      r1 = min(r0 + R, __shfl_sync(0xffffffffu, hi, who));
      return true;
    }
    before += __shfl_sync(0xffffffffu, inc, 31);
  }
  return false;
}

constexpr int kFewWarps = 8, kFewRows = 8;

// A warp per output channel and tile of up to eight rows: weights read once per tile, 16 bytes a lane, four
// products an instruction.
template <typename T>
__global__ void __launch_bounds__(kFewWarps * 32) linear_i8_few_kernel(const I8Args p) {
  int e;
  int64_t r0, r1;
  if (!find_tile(p, blockIdx.x, kFewRows, e, r0, r1)) return;
  const int lane = threadIdx.x & 31, n = blockIdx.y * kFewWarps + (threadIdx.x >> 5), nr = (int)(r1 - r0);
  if (n >= p.N) return;
  T *y = (T *)p.y;
  if (e == p.nexp) {
    if (lane < nr) put_out(y + (r0 + lane) * p.N + n, 0.0f);
    return;
  }
  const int8_t *w = p.wq + ((int64_t)e * p.N + n) * p.K, *x = p.xq + r0 * p.K;
  int acc[kFewRows] = {};
  for (int k = lane * 16; k < p.K; k += 512) {
    const int4 a = __ldg(reinterpret_cast<const int4 *>(w + k));
#pragma unroll
    for (int i = 0; i < kFewRows; ++i)
      if (i < nr) {
        const int4 b = __ldg(reinterpret_cast<const int4 *>(x + (int64_t)i * p.K + k));
        acc[i] = __dp4a(a.x, b.x, __dp4a(a.y, b.y, __dp4a(a.z, b.z, __dp4a(a.w, b.w, acc[i]))));
      }
  }
  int mine = 0;
#pragma unroll
  for (int i = 0; i < kFewRows; ++i) {
    const int s = __reduce_add_sync(0xffffffffu, acc[i]);
    if (lane == i) mine = s;
  }
  if (lane < nr) {
    const int64_t c = (int64_t)e * p.N + n;
    float v = fmaf((float)mine * __ldg(p.sx + r0 + lane), __ldg(p.sw + c), p.bias ? __ldg(p.bias + c) : 0.0f);
    if (p.act == DP_ACT_TANH) v = tanhf(v);
    put_out(y + (r0 + lane) * p.N + n, v);
  }
}

template <typename T>
int quant_rows(const T *x, const int32_t *src, const int32_t *pos, int64_t ntok, int topk, int K, int8_t *xq, float *sx,
               void *stream, const char *who) {
  clear_error();
  if (ntok < 0) return set_error(DP_ERR_SHAPE, "%s: ntok = %lld", who, (long long)ntok);
  if (topk < 1 || topk > kMaxTopk || ntok > 0x7fffffffLL / topk)
    return set_error(DP_ERR_SHAPE, "%s: topk = %d for %lld tokens", who, topk, (long long)ntok);
  if (K < 1) return set_error(DP_ERR_SHAPE, "%s: K = %d", who, K);
  if (K > kMaxK) return set_error(DP_ERR_UNSUPPORTED, "%s: K = %d > %d", who, K, kMaxK);
  if (!pos != !src) return set_error(DP_ERR_NULL, "%s: src and pos come together", who);
  if (!pos && topk != 1) return set_error(DP_ERR_SHAPE, "%s: topk = %d without a plan", who, topk);
  if (ntok == 0) return DP_OK;
  if (!x || !xq || !sx) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if ((uintptr_t)xq & 15) return set_error(DP_ERR_SHAPE, "%s: xq is not 16-byte aligned", who);
  const int v = pack_width<T>(K, x);
  if (!v) return set_error(DP_ERR_SHAPE, "%s: x is not aligned to its elements", who);
  const int ldq = (K + 15) / 16 * 16;
  auto go = [&](auto V) {
    int threads = ((K / V + kQuantKeep - 1) / kQuantKeep + 31) / 32 * 32;
    threads = threads < 32 ? 32 : threads > 512 ? 512 : threads;
    quant_rows_kernel<T, V><<<(unsigned)ntok, threads, 0, (cudaStream_t)stream>>>(x, src, pos, ntok, topk, K, ldq, xq, sx);
  };
  if (v == 16 / (int)sizeof(T)) go(std::integral_constant<int, 16 / (int)sizeof(T)>{});
  else go(std::integral_constant<int, 1>{});
  return launch_status(who);
}

template <typename T>
int linear(const int8_t *xq, const float *sx, int64_t rows, int K, const int8_t *wq, const float *sw, const float *bias,
           int nexp, int N, const int64_t *start, int act, T *y, void *stream, const char *who) {
  clear_error();
  if (rows < 0 || rows > 0x7fffffffLL) return set_error(DP_ERR_SHAPE, "%s: rows = %lld", who, (long long)rows);
  if (K < 16 || K % 16) return set_error(DP_ERR_SHAPE, "%s: K = %d is not a positive multiple of 16", who, K);
  if (K > kMaxK) return set_error(DP_ERR_UNSUPPORTED, "%s: K = %d > %d", who, K, kMaxK);
  if (N < 1 || N > (1 << 18)) return set_error(DP_ERR_SHAPE, "%s: N = %d outside [1, 2^18]", who, N);
  if (nexp < 1 || nexp > 1024) return set_error(DP_ERR_SHAPE, "%s: nexp = %d outside [1, 1024]", who, nexp);
  if (act != DP_ACT_NONE && act != DP_ACT_TANH) return set_error(DP_ERR_SHAPE, "%s: act = %d", who, act);
  if (nexp > 1 && !start) return set_error(DP_ERR_NULL, "%s: start is NULL with %d experts", who, nexp);
  if (rows == 0) return DP_OK;
  if (!xq || !sx || !wq || !sw || !y) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (((uintptr_t)xq | (uintptr_t)wq) & 15) return set_error(DP_ERR_SHAPE, "%s: xq or wq is not 16-byte aligned", who);
  const I8Args p{xq, wq, sx, sw, bias, start, rows, K, N, nexp, act, y};
  const int64_t tiles = (rows + kFewRows - 1) / kFewRows + (start ? (nexp + 1 < rows ? nexp + 1 : rows) : 0);
  const dim3 grid((unsigned)tiles, (N + kFewWarps - 1) / kFewWarps);
  linear_i8_few_kernel<T><<<grid, kFewWarps * 32, 0, (cudaStream_t)stream>>>(p);
  return launch_status(who);
}

}  // namespace
}  // namespace dpc

extern "C" {

#define DP_I8(X, C, T)                                                                                                 \
  int dp_quant_rows_i8_##X(const C *x, const int32_t *src, const int32_t *pos, int64_t ntok, int topk, int K,          \
                           int8_t *xq, float *sx, void *stream) {                                                      \
    return dpc::quant_rows<T>((const T *)x, src, pos, ntok, topk, K, xq, sx, stream, "dp_quant_rows_i8_" #X);          \
  }                                                                                                                    \
  int dp_linear_i8_##X(const int8_t *xq, const float *sx, int64_t rows, int K, const int8_t *wq, const float *sw,      \
                       const float *bias, int nexp, int N, const int64_t *start, int act, C *y, void *stream) {        \
    return dpc::linear<T>(xq, sx, rows, K, wq, sw, bias, nexp, N, start, act, (T *)y, stream, "dp_linear_i8_" #X);     \
  }
DP_I8(f64, double, double)
DP_I8(f32, float, float)
DP_I8(bf16, uint16_t, __nv_bfloat16)
DP_I8(f16, uint16_t, __half)

}  // extern "C"
