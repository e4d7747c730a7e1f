// Matrix product in microscaled 4-bit floating point, for one net or for several experts over rows sorted by expert.
// 32 neighbours of a row along K share a power of two:
//   amax = max_k |x_k|,  e = max(floor(log2 amax) - 2, -127),  q_k = the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (and their
//   negatives) to x_k 2^-e, ties to the even code, 6 for what lies above (amax 2^-e is below 8);  x_k ~ q_k 2^e
//   y_in = act(sum_b 2^(e_ib + e_nb) sum_(k in b) q_ik w_nk + b_n)
// Codes are sign, two exponent bits, one mantissa bit, two a byte with the lower four bits first; a scale is e + 127 in a byte.
#include "rows.cuh"

namespace dpc {
namespace {

constexpr int kMaxTopk = 64, kMaxK = 65536;
constexpr int kBlock = 32;  // elements of a scale

__host__ __device__ constexpr int code_cols(int K) { return (K + 63) / 64 * 64; }        // elements of a row of codes
__host__ __device__ constexpr int scale_cols(int K) { return (K + 255) / 256 * 8; }      // scales of a row

// ------------------------------------------------------------------ rows to 4 bits
// The codes of eight values, the first in the lowest bits.
__device__ __forceinline__ uint32_t to_codes(const float (&v)[8]) {
  uint32_t r;
  asm("{\n .reg .b8 a, b, c, d;\n"
      " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n"
      " cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n"
      " cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
      " mov.b32 %0, {a, b, c, d};\n}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}

// A warp takes 256 elements of a token's row, eight a lane, four lanes a scale.  With pos the row goes to the topk sorted
// rows pos[t][.], and the rows past the kept ones (src < 0) are cleared.  Whole: rows of whole aligned packs.
template <typename T, bool Whole>
__global__ void __launch_bounds__(128)
    quant_rows_mx4_kernel(const T *__restrict__ x, const int32_t *__restrict__ src, const int32_t *__restrict__ pos,
                          int64_t ntok, int topk, int K, int parts, uint8_t *__restrict__ xq, uint8_t *__restrict__ sx) {
  constexpr int V = 16 / (int)sizeof(T), kP = 8 / V;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5), t = unit / parts, n = ntok * topk;
  const int part = (int)(unit - t * parts), lane = threadIdx.x & 31, c = part * 256 + lane * 8;
  if (t >= ntok) return;
  const int ldq = code_cols(K), lds = scale_cols(K);
  const T *row = x + t * K;
  float v[8], amax = 0.0f;
#pragma unroll
  for (int i = 0; i < kP; ++i) {
    Pack<T, V> q{};
    if (c + i * V < K) {
      if constexpr (Whole) q = load_pack<T, V>(row + c + i * V);
      else q = load_any<T>(row + c + i * V, x, x + ntok * K);
    }
#pragma unroll
    for (int l = 0; l < V; ++l) v[i * V + l] = Whole || c + i * V + l < K ? (float)to_acc(q.v[l]) : 0.0f;
  }
#pragma unroll
  for (int l = 0; l < 8; ++l) amax = max_nan(amax, fabsf(v[l]));
  amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
  amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
  const uint32_t exponent = __float_as_uint(amax) >> 23;  // 255: an infinity or NaN in the block
  const uint32_t scale = exponent == 255 ? 255u : exponent < 2 ? 0u : exponent - 2;
  const float r = __uint_as_float((254u - scale) << 23);  // 2^-e
#pragma unroll
  for (int l = 0; l < 8; ++l) v[l] *= r;  // exact, but where it is far below the least code
  const uint32_t codes = scale == 255 ? 0u : to_codes(v);
  for (int j = 0; j < topk; ++j) {
    const int64_t q = t * topk + j, p = pos ? __ldg(pos + q) : t;
    if (p >= 0 && p < n) {
      if (c < ldq) reinterpret_cast<uint32_t *>(xq + p * (ldq / 2))[c / 8] = codes;
      if (lane % 4 == 0) sx[p * lds + c / kBlock] = (uint8_t)scale;
    }
    if (pos && __ldg(src + q) < 0) {
      if (c < ldq) reinterpret_cast<uint32_t *>(xq + q * (ldq / 2))[c / 8] = 0u;
      if (lane % 4 == 0) sx[q * lds + c / kBlock] = 0;
    }
  }
}

// ------------------------------------------------------------------ the product
struct Mx4Args {
  const uint8_t *xq, *sx, *wq, *sw;
  const float *bias;
  const int64_t *start;  // [nexp + 1], or NULL: one expert for all rows
  int rows, K, N, nexp, act;  // K: of the codes, a multiple of 64
  void *y;
};

// Four codes (the lower 16 bits) as four int8, twice their values: a byte permutation looks up the magnitudes, and gives
// zero where the selector's top bit, the code's sign, is set (it repeats the sign of the byte it selects).
__device__ __forceinline__ uint32_t four(uint32_t codes) {
  constexpr uint32_t lo = 0x03020100u, hi = 0x0c080604u;
  uint32_t p, m;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(p) : "r"(lo), "r"(hi), "r"(codes));
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(m) : "r"(lo), "r"(hi), "r"(codes ^ 0x8888u));
  return ((p | 0x80808080u) - m) ^ 0x80808080u;  // bytewise p - m: no borrow crosses a byte
}
struct Block32 {
  uint32_t v[8];
  __device__ __forceinline__ explicit Block32(const uint4 &q) {
    v[0] = four(q.x);
    v[1] = four(q.x >> 16);
    v[2] = four(q.y);
    v[3] = four(q.y >> 16);
    v[4] = four(q.z);
    v[5] = four(q.z >> 16);
    v[6] = four(q.w);
    v[7] = four(q.w >> 16);
  }
};
__device__ __forceinline__ int dot(const Block32 &a, const Block32 &b) {  // four times the sum, exact
  int s = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) s = __dp4a((int)a.v[i], (int)b.v[i], s);
  return s;
}
__device__ __forceinline__ float pow2_of(uint32_t code) {
  return __uint_as_float(code == 0 ? 0x00400000u : code == 255 ? 0x7fc00000u : code << 23);
}

constexpr int kFewWarps = 8, kFewRows = 8;

// A warp per output channel and tile of up to eight rows, a scale's block a lane: the block's sum is exact in integers.
template <typename T>
__global__ void __launch_bounds__(kFewWarps * 32) linear_mx4_few_kernel(const Mx4Args p) {
  int e, r0, r1;
  if (!find_tile(p.start, p.rows, p.nexp, blockIdx.x, kFewRows, e, r0, r1)) return;
  const int lane = threadIdx.x & 31, n = blockIdx.y * kFewWarps + (threadIdx.x >> 5), nr = r1 - r0;
  if (n >= p.N) return;
  T *y = (T *)p.y;
  if (e == p.nexp) {
    if (lane < nr) put_out(y + (int64_t)(r0 + lane) * p.N + n, 0.0f);
    return;
  }
  const int nb = p.K / kBlock, lds = scale_cols(p.K);
  const int64_t c = (int64_t)e * p.N + n;
  const uint4 *w = reinterpret_cast<const uint4 *>(p.wq + c * (p.K / 2)), *x = reinterpret_cast<const uint4 *>(p.xq + (int64_t)r0 * (p.K / 2));
  float acc[kFewRows] = {};
  for (int b = lane; b < nb; b += 32) {
    const Block32 wb(__ldg(w + b));
    const float s = pow2_of(__ldg(p.sw + c * lds + b));
#pragma unroll
    for (int i = 0; i < kFewRows; ++i)
      if (i < nr) {
        const Block32 xb(__ldg(x + (int64_t)i * nb + b));
        acc[i] = fmaf((float)dot(wb, xb), s * pow2_of(__ldg(p.sx + (int64_t)(r0 + i) * lds + b)), acc[i]);
      }
  }
  float mine = 0.0f;
#pragma unroll
  for (int i = 0; i < kFewRows; ++i) {
    float s = acc[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == i) mine = s;
  }
  if (lane < nr) {
    float v = fmaf(mine, 0.25f, p.bias ? __ldg(p.bias + c) : 0.0f);
    if (p.act == DP_ACT_TANH) v = tanhf(v);
    put_out(y + (int64_t)(r0 + lane) * p.N + n, v);
  }
}

template <typename T>
int quant_rows(const T *x, const int32_t *src, const int32_t *pos, int64_t ntok, int topk, int K, uint8_t *xq, uint8_t *sx,
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
  if (((uintptr_t)xq & 15) || ((uintptr_t)sx & 7)) return set_error(DP_ERR_SHAPE, "%s: xq or sx is not aligned", who);
  if (!at_elements(x) || !at_elements(src, pos)) return misaligned(who);
  const int parts = (K + 255) / 256;
  const int64_t blocks = (ntok * parts + 3) / 4;
  if (blocks > 0x7fffffffLL) return set_error(DP_ERR_SHAPE, "%s: %lld rows of %d", who, (long long)ntok, K);
  const bool whole = (((uintptr_t)x | (uintptr_t)(K * sizeof(T))) & 15) == 0;
  auto k = whole ? quant_rows_mx4_kernel<T, true> : quant_rows_mx4_kernel<T, false>;
  k<<<(unsigned)blocks, 128, 0, (cudaStream_t)stream>>>(x, src, pos, ntok, topk, K, parts, xq, sx);
  return launch_status(who);
}

template <typename T>
int linear(const uint8_t *xq, const uint8_t *sx, int64_t rows, int K, const uint8_t *wq, const uint8_t *sw, const float *bias,
           int nexp, int N, const int64_t *start, int act, T *y, void *stream, const char *who) {
  clear_error();
  if (rows < 0 || rows > 0x7fffffffLL - 1024) return set_error(DP_ERR_SHAPE, "%s: rows = %lld", who, (long long)rows);
  if (K < 64 || K % 64) return set_error(DP_ERR_SHAPE, "%s: K = %d is not a positive multiple of 64", who, K);
  if (K > kMaxK) return set_error(DP_ERR_UNSUPPORTED, "%s: K = %d > %d", who, K, kMaxK);
  if (N < 1 || N > (1 << 18)) return set_error(DP_ERR_SHAPE, "%s: N = %d outside [1, 2^18]", who, N);
  if (nexp < 1 || nexp > 1024) return set_error(DP_ERR_SHAPE, "%s: nexp = %d outside [1, 1024]", who, nexp);
  if (act != DP_ACT_NONE && act != DP_ACT_TANH) return set_error(DP_ERR_SHAPE, "%s: act = %d", who, act);
  if (nexp > 1 && !start) return set_error(DP_ERR_NULL, "%s: start is NULL with %d experts", who, nexp);
  if (rows == 0) return DP_OK;
  if (!xq || !sx || !wq || !sw || !y) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if ((((uintptr_t)xq | (uintptr_t)wq) & 15) || (((uintptr_t)sx | (uintptr_t)sw) & 7))
    return set_error(DP_ERR_SHAPE, "%s: xq, wq, sx or sw is not aligned", who);
  if (!at_elements(y) || !at_elements(bias) || !at_elements(start)) return misaligned(who);
  const Mx4Args p{xq, sx, wq, sw, bias, start, (int)rows, K, N, nexp, act, y};
  const cudaStream_t st = (cudaStream_t)stream;
  const int64_t pieces = start ? (nexp + 1 < rows ? nexp + 1 : rows) : 0;  // a tile more for each expert's remainder
  auto tiles = [&](int R) { return (rows + R - 1) / R + pieces; };
  const dim3 grid((unsigned)tiles(kFewRows), (N + kFewWarps - 1) / kFewWarps);
  linear_mx4_few_kernel<T><<<grid, kFewWarps * 32, 0, st>>>(p);
  return launch_status(who);
}

}  // namespace
}  // namespace dpc

extern "C" {

#define DP_MX4(X, C, T)                                                                                                \
  int dp_quant_rows_mx4_##X(const C *x, const int32_t *src, const int32_t *pos, int64_t ntok, int topk, int K,         \
                            uint8_t *xq, uint8_t *sx, void *stream) {                                                  \
    return dpc::quant_rows<T>((const T *)x, src, pos, ntok, topk, K, xq, sx, stream, "dp_quant_rows_mx4_" #X);         \
  }                                                                                                                    \
  int dp_linear_mx4_##X(const uint8_t *xq, const uint8_t *sx, int64_t rows, int K, const uint8_t *wq,                  \
                        const uint8_t *sw, const float *bias, int nexp, int N, const int64_t *start, int act, C *y,    \
                        void *stream) {                                                                                \
    return dpc::linear<T>(xq, sx, rows, K, wq, sw, bias, nexp, N, start, act, (T *)y, stream, "dp_linear_mx4_" #X);    \
  }
DP_MX4(f64, double, double)
DP_MX4(f32, float, float)
DP_MX4(bf16, uint16_t, __nv_bfloat16)
DP_MX4(f16, uint16_t, __half)

}  // extern "C"
