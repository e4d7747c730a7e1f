// Matrix product in microscaled 4-bit floating point, for one net or for several experts over rows sorted by expert.
// 32 neighbours of a row along K share a power of two:
//   amax = max_k |x_k|,  e = max(floor(log2 amax) - 2, -127),  q_k = the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (and their
//   negatives) to x_k 2^-e, ties to the even code, 6 for what lies above (amax 2^-e is below 8);  x_k ~ q_k 2^e
//   y_in = act(sum_b 2^(e_ib + e_nb) sum_(k in b) q_ik w_nk + b_n)
// Codes are sign, two exponent bits, one mantissa bit, two a byte with the lower four bits first; a
// scale is e + 127 in a byte.
#include <cuda.h>

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

// Eight neighbouring elements of a row, as many as a lane takes at a time; four lanes have a scale.
template <typename T>
struct Eight {
  static constexpr int V = 16 / (int)sizeof(T), kN = 8 / V;
  Pack<T, V> p[kN];
  __device__ __forceinline__ float at(int l) const { return (float)to_acc(p[l / V].v[l % V]); }
  // The bits of their largest |x| as an f32, NaN above all: without the sign the bits are ordered as the numbers are.
  __device__ __forceinline__ uint32_t amax() const {
    if constexpr (sizeof(T) == 2) {
      uint32_t w[4], m;
      memcpy(w, p, 16);
      m = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
      m = max(m >> 16, m & 0xffffu);
      if constexpr (std::is_same<T, __nv_bfloat16>::value) return m << 16;
      else return __float_as_uint(__half2float(__ushort_as_half((unsigned short)m)));
    } else {
      uint32_t m = 0;
#pragma unroll
      for (int l = 0; l < 8; ++l) m = max(m, __float_as_uint(at(l)) & 0x7fffffffu);
      return m;
    }
  }
};

template <typename T>
constexpr int kQuantEights = sizeof(T) == 8 ? 2 : 4;  // a lane has 64 (16 bits) or 128 bytes on their way

// A warp takes `part` eights of a token's row; `slices` warps side by side a token, about four of them or more in a
// block.  With pos the row goes to the topk sorted rows pos[t][.], and the rows past the kept ones (src < 0) are cleared.
// Rows: kExact, whole aligned packs and whole blocks of 64 elements; kWhole, whole aligned packs; kAny.
// Bound by memory: 65,536 x 1600 f32 to sorted places in 70 us (6.8 TB/s), 32,768 x 2048 bf16 in 31 (5.4).  Instructions come
// second: four elements a lane at a time, with three exchanges of the largest instead of two and codes in two bytes, took
// 98, and half as many bytes a warp 85.  Rows of odd length come as shifted words: 65,536 x 1003 f16 in 58 us (2.8 TB/s).
enum QuantRows { kExact, kWhole, kAny };
template <typename T, QuantRows kRows>
__global__ void __launch_bounds__(256)
    quant_rows_mx4_kernel(const T *__restrict__ x, const int32_t *__restrict__ src, const int32_t *__restrict__ pos,
                          int64_t ntok, int topk, int K, int part, int token_bits, uint8_t *__restrict__ xq,
                          uint8_t *__restrict__ sx) {
  constexpr int V = 16 / (int)sizeof(T), kE = kQuantEights<T>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ldq = code_cols(K), lds = scale_cols(K);
  const int slice = (int)(blockIdx.y * (blockDim.x >> 5 >> token_bits)) + (warp >> token_bits);
  const int64_t t = ((int64_t)blockIdx.x << token_bits) + (warp & ((1 << token_bits) - 1)), n = ntok * topk;
  if (t >= ntok) return;
  const int first = slice * part, total = min(part, ldq / 8 - first), count = total - lane;  // of this lane on, 32 apart
  // where the first two pairs go, read beside the row
  int place[2] = {-1, -1}, kept[2] = {0, 0};
  if (pos)
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (j < topk) {
        place[j] = __ldg(pos + t * topk + j);
        kept[j] = __ldg(src + t * topk + j);
      }
  const int c0 = (first + lane) * 8;
  const T *row = x + t * K + c0;
  Eight<T> in[kE];
#pragma unroll
  for (int i = 0; i < kE; ++i)
#pragma unroll
    for (int h = 0; h < Eight<T>::kN; ++h) {
      const int d = i * 256 + h * V;
      Pack<T, V> &q = in[i].p[h];
      if constexpr (kRows == kExact) {
        if (i * 32 < count) q = load_pack<T, V>(row + d);
      } else {
        q = Pack<T, V>{};
        if (i * 32 < count && c0 + d < K) {
          if constexpr (kRows == kWhole) q = load_pack<T, V>(row + d);
          else q = load_any<T>(row + d, x, x + ntok * K);
        }
        if constexpr (kRows == kAny) {
          const T zero = from_acc<T>(acc_t<T>(0));
#pragma unroll
          for (int l = 0; l < V; ++l)
            if (c0 + d + l >= K) q.v[l] = zero;
        }
      }
    }
  uint32_t codes[kE], scales[kE];
#pragma unroll
  for (int i = 0; i < kE; ++i) {
    if (i * 32 >= total) break;  // for the warp
    uint32_t amax = in[i].amax();
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    // 2^-e from the exponent's bits, which are at least two (e >= -127)
    const uint32_t top = max(amax & 0x7f800000u, 2u << 23);
    const float r = __uint_as_float(0x80000000u - top);
    float v[8];
#pragma unroll
    for (int l = 0; l < 8; ++l) v[l] = in[i].at(l) * r;  // exact, but where it is far below the least code
    codes[i] = to_codes(v);
    scales[i] = (top >> 23) - 2;
    if (amax >= 0x7f800000u) {  // an infinity or NaN in the block
      codes[i] = 0;
      scales[i] = 255;
    }
  }
  const bool leads = lane % 4 == 0;
  const int pad = slice == 0 && lane < lds - ldq / kBlock ? ldq / kBlock + lane : -1;  // scales past the last block
  for (int j = 0; j < topk; ++j) {
    const int64_t q = t * topk + j, p = !pos ? t : j == 0 ? place[0] : j == 1 ? place[1] : __ldg(pos + q);
    if (p >= 0 && p < n) {
      uint32_t *to = reinterpret_cast<uint32_t *>(xq + p * (ldq / 2)) + first + lane;
      uint8_t *ts = sx + p * lds + (first + lane) / 4;
#pragma unroll
      for (int i = 0; i < kE; ++i)
        if (i * 32 < count) {
          to[i * 32] = codes[i];
          if (leads) ts[i * 8] = (uint8_t)scales[i];
        }
      if (pad >= 0) sx[p * lds + pad] = 0;
    }
    if (pos && (j == 0 ? kept[0] : j == 1 ? kept[1] : __ldg(src + q)) < 0) {
      for (int i = 0; i < count; i += 32) {
        (reinterpret_cast<uint32_t *>(xq + q * (ldq / 2)) + first + lane)[i] = 0;
        if (leads) (sx + q * lds + (first + lane) / 4)[i / 4] = 0;
      }
      if (pad >= 0) sx[q * lds + pad] = 0;
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
  int give_up;  // the stage of a block whose wait gives up (dp_give_up_at)
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

constexpr int kFewWarps = 8, kFewRows = 2;

// A warp per output channel and tile of up to two rows, a scale's block a lane: the block's sum is exact in integers.
// Bound by latency: 2 rows of 1600 -> 2048 in two of eight nets 8 us, of which 5 are the launch.
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
  const uint4 *w = reinterpret_cast<const uint4 *>(p.wq + c * (p.K / 2));
  const uint4 *x = reinterpret_cast<const uint4 *>(p.xq + (int64_t)r0 * (p.K / 2));
  float acc[kFewRows] = {};
  for (int b = lane; b < nb; b += 32) {
    const Block32 wb(__ldg(w + b));
    const uint32_t cw = __ldg(p.sw + c * lds + b);
#pragma unroll
    for (int i = 0; i < kFewRows; ++i)
      if (i < nr) {
        const Block32 xb(__ldg(x + (int64_t)i * nb + b));
        // the scales' product as two powers of two of equal size: neither the sum's product with the first (exact) nor
        // the powers leave f32's range unless the block's sum does
        const uint32_t cx = __ldg(p.sx + (int64_t)(r0 + i) * lds + b);
        const uint32_t half = cw == 255 || cx == 255 ? 255 : (cw + cx) / 2;
        acc[i] = fmaf(0.25f * (float)dot(wb, xb) * pow2_of(half), pow2_of(cw + cx - half), acc[i]);
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
    float v = mine + (p.bias ? __ldg(p.bias + c) : 0.0f);
    if (p.act == DP_ACT_TANH) v = tanhf(v);
    put_out(y + (int64_t)(r0 + lane) * p.N + n, v);
  }
}

// ------------------------------------------------------------------ the product on the tensor cores
// A tile is 128 output channels (the MMA's rows) by up to TN sorted rows of one expert (its columns), so that an epilogue
// warp holds 32 neighbouring channels of a row and stores them side by side.  The block-scaled MMA takes codes and scales
// as they are: K 64 an instruction, a scale for 32.
//   One lane copies a stage's codes, 256 of K, by tensor-map copies into K-major rows of 128 bytes in the 128-byte swizzle
//   (a map reads zeros past the arrays; rows of another expert or past N land in columns and rows that nobody reads).
//   Two sets of four warps bring the scales, of four stages at a time in turn, four lanes a row, through shared memory
//   (one set: 156 us for 32,768 x 2048 x 4096).  There 128 rows' four scales of 128 of K are 512 bytes, row r at
//   16 (r % 32) + 4 (r / 32), so that lane r of each of a set's warps finds the words that its quadrant of tensor memory
//   holds in lane r, and writes them there with tcgen05.st, two stages at a time.
//   Two stages' scales have three places, taken in turn; a place is written again when the MMAs that read it have completed.
//   (Copies from shared to tensor memory by the MMAs' own thread, tcgen05.cp, take turns with the MMAs: a stage took 2000
//   cycles whatever its tile, 32,768 x 2048 x 4096 264 us; stages one by one 220 us.)
//   One lane issues the MMAs; its warp walks the stages together, so that addresses and descriptors stay in uniform
//   registers (in a branch for one lane a stage's issue took 600 cycles), and waits once for two stages: the scales'
//   warps have waited for their codes.
//   Eight epilogue warps (two per lane quadrant, half the columns each) finish a tile while the next one runs.
// A block per SM walks the tiles; every wait is bounded, a block that gives up writes NaN and is counted.
// Measured: 32,768 x 2048 x 4096 bf16 in 139 us (4.0 PFLOP/s, 2.1 times the measured bf16 rate), 8192 cubed 228 us (4.8),
// 65,536 x 1600 x 240 f32 with four nets 37 us.  A stage of 8192 cubed takes 390 ns for 192 rows, 310 for 128, 280 for 64,
// and with one of its four MMAs 355: what bounds it are the barriers between the roles.  Without the output 212 us, the wide
// product 119 (stages and these without the wait for a stage's turn before, which costs some 2 %).
namespace mx4 {
constexpr int kTM = 128, kKB = 256, kRowBytes = kKB / 2;
constexpr int kEpiWarps = 8, kScaleWarps = 4, kScaleSets = 2;
constexpr int kCopyWarp = kEpiWarps + kScaleWarps * kScaleSets, kMmaWarp = kCopyWarp + 1;
constexpr int kThreads = (kMmaWarp + 1) * 32;
constexpr int kGroup = 4;  // stages whose scales come together

template <int TN>
struct Shape {
  static constexpr int kA = kTM * kRowBytes, kB = TN * kRowBytes, kStageBytes = kA + kB;
  static constexpr int kSA = 1024, kBlocksB = (TN + 127) / 128, kScaleBytes = kSA + 1024 * kBlocksB;  // of a stage
  static constexpr int kStages = TN > 128 ? 5 : TN > 64 ? 6 : 8;
  static constexpr uint32_t kColsA = 4, kColsB = TN / 32;  // of 128 of K
  // two accumulators, then the scales' places
  static constexpr int kPlaces = 3;
  static constexpr uint32_t kStageCols = 2 * (kColsA + kColsB), kPlaceCols = 2 * kStageCols, kScaleAt = 2 * TN;
  static constexpr uint32_t kTmemCols = TN > 64 ? 512 : 256;
  static constexpr int kBarriers = 2 * kStages + kPlaces + 9;
  static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + 2 * kGroup * kScaleBytes + kBarriers * 8 + 16;
  static_assert(kStageBytes % 1024 == 0 && kSmem <= 227 * 1024 && TN % 32 == 0, "tile");
  static_assert(kScaleAt + kPlaces * kPlaceCols <= kTmemCols, "accumulators and scales");
};

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool elect_one() {  // one lane of a converged warp
  uint32_t is;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(is));
  return is != 0;
}
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Shared-memory descriptor, version 1: codes K-major in the 128-byte swizzle (8 rows are 1024 bytes).
__device__ __forceinline__ uint64_t code_desc(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFF) >> 4) | (1ull << 16) | ((uint64_t)(8 * kRowBytes >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void tmem_st2(uint32_t addr, const uint4 &v) {  // two columns
  asm volatile("tcgen05.st.sync.aligned.32x32b.x2.b32 [%0], {%1,%2};" ::"r"(addr), "r"(v.x), "r"(v.y));
}
__device__ __forceinline__ void tmem_st(uint32_t addr, const uint4 &v) {  // four
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w));
}
__device__ __forceinline__ void tmem_ld(uint32_t addr, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
        "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(addr));
}
__device__ __forceinline__ void copy_tile(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
               " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"((uint64_t)map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}

// Where a role stands: the tile, and the expert, rows and channels it means.
struct Tile {
  int tile, r0, r1, e, n0;
  bool have;
};
__device__ __forceinline__ void seek(const Mx4Args &p, int TN, int nct, Tile &t) {
  const int rt = t.tile / nct;
  t.n0 = (t.tile - rt * nct) * kTM;
  t.have = find_tile(p.start, p.rows, p.nexp, rt, TN, t.e, t.r0, t.r1);
}
// The next tile with products, from t on.
__device__ __forceinline__ void seek_work(const Mx4Args &p, int TN, int nct, Tile &t) {
  for (;; t.tile += gridDim.x) {
    seek(p, TN, nct, t);
    if (!t.have || t.e < p.nexp) return;
  }
}

template <typename T, int TN>
__global__ void __launch_bounds__(kThreads, 1)
    linear_mx4_tc_kernel(const Mx4Args p, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap wmap) {
  using S = Shape<TN>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char *smem = smem_raw + (1024 - (smem_u32(smem_raw) & 1023)) % 1024;
  unsigned char *scale_room = smem + S::kStages * S::kStageBytes;
  uint64_t *codes = reinterpret_cast<uint64_t *>(scale_room + 2 * kGroup * S::kScaleBytes), *empty = codes + S::kStages;
  uint64_t *scales = empty + S::kStages, *staged = scales + S::kPlaces, *unstaged = staged + 2;
  uint64_t *acc_full = unstaged + 2;
  uint64_t *acc_empty = acc_full + 2;
  uint64_t *done = acc_empty + 2;
  uint32_t *holder = reinterpret_cast<uint32_t *>(done + 1);
  volatile int *stop = reinterpret_cast<int *>(holder + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int nct = (p.N + kTM - 1) / kTM, nkb = (p.K + kKB - 1) / kKB;
  auto wait = [&](uint64_t *bar, uint32_t parity) {  // gives up with any other wait of the block
    return bounded_wait(smem_u32(bar), parity, [&] { return *stop != 0; });
  };
  auto wait_on = [&](uint64_t *bar, uint32_t parity) {  // for what is in flight, come what may
    return bounded_wait(smem_u32(bar), parity, [] { return false; });
  };

  if (threadIdx.x == 0) {
    auto init = [](uint64_t *b, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(n)); };
    for (int s = 0; s < S::kStages; ++s) {
      init(codes + s, 1);
      init(empty + s, 1);
    }
    for (int b = 0; b < S::kPlaces; ++b) init(scales + b, kScaleWarps);
    for (int b = 0; b < 2; ++b) {
      init(staged + b, kScaleWarps);
      init(unstaged + b, kScaleWarps);
      init(acc_full + b, 1);
      init(acc_empty + b, kEpiWarps);
    }
    init(done, 1);
    *stop = 0;
    asm volatile("fence.mbarrier_init.release.cluster;");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(holder)),
                 "r"(S::kTmemCols));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  asm volatile("tcgen05.fence::before_thread_sync;");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;");
  const uint32_t tmem = *holder;
  bool ok = true;
  int copied = 0;  // stages copied

  if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- the MMAs
    int j = 0, unit = 0;     // stages, tiles
    int st = 0, place = 0;   // j's place, its scales' place
    uint32_t turn = 0;       // the parity of the latter's turn
    const bool leader = elect_one();
    const uint64_t a_at = code_desc(smem_u32(smem)), b_at = a_at + (S::kA >> 4);
    Tile t{(int)blockIdx.x, 0, 0, 0, 0, false};
    for (; ok; t.tile += gridDim.x, ++unit) {
      seek_work(p, TN, nct, t);
      if (!t.have) break;
      const uint32_t cols = (uint32_t)(t.r1 - t.r0 + 15) / 16 * 16;
      // fp4 operands, K-major; scales are powers of two, a word's lower two or upper two
      const uint32_t low = (1u << 7) | (1u << 10) | ((cols >> 3) << 17) | (1u << 23) | ((uint32_t)(kTM >> 7) << 27);
      const uint32_t high = low | (2u << 4) | (2u << 29);
      const int buf = unit & 1;
      auto all = [&](uint64_t *bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
      if (unit >= 2) ok = all(acc_empty + buf, ((unit >> 1) - 1) & 1);
      const int end = min(nkb, p.give_up - j);
      const uint32_t acc = tmem + buf * TN;
      auto mma = [&](int k, uint64_t a, uint64_t b, uint32_t ta, bool add) {
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(acc),
            "l"(a + (uint64_t)(k * 2)), "l"(b + (uint64_t)(k * 2)), "r"(k & 1 ? high : low), "r"(ta + (k >> 1) * S::kColsA),
            "r"(ta + 2 * S::kColsA + (k >> 1) * S::kColsB), "r"(add ? 1u : 0u)
            : "memory");
      };
      for (int kb = 0; kb < nkb; kb += 2) {
        const int n = min(2, nkb - kb);
        ok = ok && kb + n <= end && all(scales + place, turn);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;");
        const uint32_t ta = tmem + S::kScaleAt + place * S::kPlaceCols;
        if (++place == S::kPlaces) {
          place = 0;
          turn ^= 1;
        }
        for (int i = 0; i < n; ++i, ++j) {
          const uint64_t place_of = (uint64_t)(st * (S::kStageBytes >> 4)), a = a_at + place_of, b = b_at + place_of;
          const uint32_t tai = ta + i * S::kStageCols;
          if (leader) {
            if ((kb + i + 1) * kKB <= p.K) {
              mma(0, a, b, tai, kb + i > 0);
              mma(1, a, b, tai, true);
              mma(2, a, b, tai, true);
              mma(3, a, b, tai, true);
            } else {
#pragma unroll
              for (int k = 0; k < kKB / 64 - 1; ++k)
                if ((kb + i) * kKB + k * 64 < p.K) mma(k, a, b, tai, kb + i > 0 || k > 0);
            }
            commit(smem_u32(empty + st));
            if (kb + i == nkb - 1) commit(smem_u32(acc_full + buf));
          }
          if (++st == S::kStages) st = 0;
        }
        __syncwarp();
      }
    }
    if (leader) commit(smem_u32(done));  // completes when every MMA issued above has
    if (!ok) *stop = 1;
  } else if (warp == kCopyWarp) {
    // ---------------------------------------------------------------- the codes
    Tile t{(int)blockIdx.x, 0, 0, 0, 0, false};
    for (; ok; t.tile += gridDim.x) {
      seek_work(p, TN, nct, t);
      if (!t.have) break;
      if (lane == 0) {
        for (int kb = 0; kb < nkb; ++kb) {
          const int st = copied % S::kStages;
          ok = wait(empty + st, (copied / S::kStages & 1) ^ 1);
          if (!ok) break;
          const uint32_t bar = smem_u32(codes + st), dst = smem_u32(smem) + st * S::kStageBytes;
          asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)(S::kA + S::kB))
                       : "memory");
          copy_tile(dst, &wmap, kb * kRowBytes, t.e * p.N + t.n0, bar);
          copy_tile(dst + S::kA, &xmap, kb * kRowBytes, t.r0, bar);
          ++copied;
        }
      }
      ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
    }
    if (!ok) *stop = 1;
  } else if (warp >= kEpiWarps) {
    // ---------------------------------------------------------------- the scales
    constexpr int kRA = kTM / 32, kRB = TN / 32;  // rows of a thread
    const int set = (warp - kEpiWarps) / kScaleWarps, at = threadIdx.x - (kEpiWarps + set * kScaleWarps) * 32;
    const int row = at / 4, s = at % 4, lds = scale_cols(p.K);
    Tile t{(int)blockIdx.x, 0, 0, 0, 0, false};
    int kb = 0;
    uint2 v[kRA + kRB];
    auto read = [&] {  // of stage kb + s
      const uint8_t *a = p.sw + ((int64_t)t.e * p.N + t.n0 + row) * lds, *b = p.sx + (int64_t)(t.r0 + row) * lds;
      const int na = kb + s < nkb ? p.N - t.n0 - row : 0, nb = kb + s < nkb ? t.r1 - t.r0 - row : 0, k = (kb + s) * 8;
#pragma unroll
      for (int i = 0; i < kRA + kRB; ++i) {
        const int r = 32 * (i < kRA ? i : i - kRA);
        v[i] = make_uint2(0, 0);
        if (r < (i < kRA ? na : nb)) v[i] = __ldg(reinterpret_cast<const uint2 *>((i < kRA ? a : b) + (int64_t)r * lds + k));
      }
    };
    // the groups of four stages go to the two sets of warps in turn, each with a place of its own in shared memory
    int j = 0, place = 0;                    // the stage, its pair's place in tensor memory
    int last0 = -1, last1 = -1, last2 = -1;  // the last stages of the pairs before, the latest first
    static_assert(S::kPlaces == 3 && kScaleSets == 2, "as many pairs before; a place a set");
    static_assert(S::kStages > 2 * (S::kPlaces - 1), "a last stage's barrier does not turn again before this pair's MMAs");
    auto next_pair = [&](int n) {
      if (++place == S::kPlaces) place = 0;
      j += n;
      last2 = last1;
      last1 = last0;
      last0 = j - 1;
    };
    auto next_group = [&] {
      kb += kGroup;
      if (kb >= nkb) {
        kb = 0;
        t.tile += gridDim.x;
        seek_work(p, TN, nct, t);
      }
    };
    auto skip_group = [&] {  // the other set's
      if (!t.have) return;
      const int stages = min(kGroup, nkb - kb);
      for (int i = 0; i < stages; i += 2) next_pair(min(2, stages - i));
      next_group();
    };
    seek_work(p, TN, nct, t);
    if (set) skip_group();
    if (t.have) read();
    const uint32_t room = smem_u32(scale_room) + set * kGroup * S::kScaleBytes, to = room + s * S::kScaleBytes + row * 16;
    const uint32_t quadrant = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + S::kScaleAt;
    auto all_wait = [&](uint64_t *bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
    for (uint32_t turn = 0; ok && t.have; turn ^= 1) {
      ok = all_wait(unstaged + set, turn ^ 1);  // the set's warps have read what lay there
      if (!ok) break;
#pragma unroll
      for (int i = 0; i < kRA + kRB; ++i) {  // row r of an operand: block r / 128 of each 128 of K, word r / 32 % 4
        const int q = i < kRA ? i : i - kRA, nblk = i < kRA ? 1 : S::kBlocksB;
        const uint32_t d = to + (i < kRA ? 0 : S::kSA) + q / 4 * 512 + q % 4 * 4;
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(d), "r"(v[i].x) : "memory");
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(d + 512 * nblk), "r"(v[i].y) : "memory");
      }
      __syncwarp();
      if (lane == 0) arrive(smem_u32(staged + set));
      const int stages = min(kGroup, nkb - kb);
      ok = all_wait(staged + set, turn);
      for (int i = 0; ok && i < stages; i += 2) {
        const uint32_t from = room + i * S::kScaleBytes + lane * 16;
        constexpr int kBlocks = S::kScaleBytes / 512;  // an operand's 128 rows by 128 of K, in the order of the columns
        uint4 w[2 * kBlocks];
#pragma unroll
        for (int b = 0; b < 2 * kBlocks; ++b)  // of a last stage alone: what lay there before, for columns that are not read
          asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
                       : "=r"(w[b].x), "=r"(w[b].y), "=r"(w[b].z), "=r"(w[b].w)
                       : "r"(from + b * 512));
        const int n = min(2, stages - i);
        if (last2 >= 0) ok = all_wait(empty + last2 % S::kStages, last2 / S::kStages & 1);  // the place's MMAs are through
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;");
        uint32_t at = quadrant + place * S::kPlaceCols;
#pragma unroll
        for (int b = 0; b < 2 * kBlocks; ++b) {
          const int in = b % kBlocks;  // A of both 128 of K, then B's blocks of both, the last of them as far as TN goes
          const bool whole = in < 2 || (in - 2) % S::kBlocksB < S::kBlocksB - 1;
          const uint32_t cols = whole ? 4 : S::kColsB - 4 * (S::kBlocksB - 1);
          if (cols == 4) tmem_st(at, w[b]);
          else tmem_st2(at, w[b]);
          at += cols;
        }
        static_assert(S::kColsB % 2 == 0 && (S::kColsB % 4 == 0 || S::kColsB % 4 == 2), "two or four columns");
        // One of the warps waits for the codes too.  A parity tells a turn from the next, not from the one after that: the
        // place's turn before, which the other set may have waited for, must be over.  It is if its MMAs are through: those
        // up to last2 are, and with fewer stages than three pairs have, the others are waited for (the codes are copied after
        // them anyway) while the scales are on their way.
        const bool brings_codes = (warp - kEpiWarps) % kScaleWarps == 0;
        if (S::kStages < 2 * S::kPlaces && brings_codes)
          for (int k = max(j, last2 + 1 + S::kStages); ok && k < j + n; ++k)
            ok = all_wait(empty + k % S::kStages, (k / S::kStages - 1) & 1);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;");
        if (brings_codes)
          for (int k = j; ok && k < j + n; ++k) ok = all_wait(codes + k % S::kStages, k / S::kStages & 1);
        if (!ok) break;
        __syncwarp();
        if (lane == 0) arrive(smem_u32(scales + place));
        next_pair(n);
      }
      __syncwarp();
      if (lane == 0) arrive(smem_u32(unstaged + set));
      next_group();
      skip_group();
      if (t.have) read();  // on its way while the other set works
    }
    if (!ok) *stop = 1;
  } else {
    // ---------------------------------------------------------------- epilogue
    constexpr int CW = TN / 2;  // columns of this warp
    const int quad = warp & 3, c0 = (warp >> 2) * CW;
    const uint32_t trow = tmem + ((uint32_t)(32 * quad) << 16) + c0;
    T *y = (T *)p.y;
    int unit = 0;
    Tile t{(int)blockIdx.x, 0, 0, 0, 0, false};
    for (;; t.tile += gridDim.x) {
      seek(p, TN, nct, t);
      if (!t.have) break;
      const int n = t.n0 + 32 * quad + lane, nr = t.r1 - t.r0;
      const bool mine = n < p.N;
      if (t.e == p.nexp) {
        if (mine)
          for (int c = c0; c < min(nr, c0 + CW); ++c) put_out(y + (int64_t)(t.r0 + c) * p.N + n, 0.0f);
        continue;
      }
      const float bias = mine && p.bias ? __ldg(p.bias + (int64_t)t.e * p.N + n) : 0.0f;
      ok = __all_sync(0xffffffffu, ok && wait(acc_full + (unit & 1), (unit >> 1) & 1));
      asm volatile("tcgen05.fence::after_thread_sync;");
      T *out = y + (int64_t)(t.r0 + c0) * p.N + n;
#pragma unroll 1
      for (int g = 0; g < CW && c0 + g < nr; g += 16, out += (int64_t)16 * p.N) {
        const int left = nr - c0 - g;
        float v[16];
        if (ok) {
          tmem_ld(trow + (unit & 1) * TN + g, v);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = ok ? v[i] + bias : __uint_as_float(0x7fc00000u);
        if (p.act == DP_ACT_TANH) {
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = tanhf(v[i]);
        }
        T *o = out;
        if (mine) {
          if (left >= 16) {
#pragma unroll
            for (int i = 0; i < 16; ++i, o += p.N) put_out(o, v[i]);
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i, o += p.N)
              if (i < left) put_out(o, v[i]);
          }
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;");
      __syncwarp();
      if (lane == 0) arrive(smem_u32(acc_empty + (unit & 1)));
      ++unit;
    }
    if (!ok) *stop = 1;
  }
  __syncwarp();
  __syncthreads();
  ok = wait_on(done, 0) && !*stop;  // no MMA is in flight when the accumulators go
  if (!__syncthreads_and(ok)) {
    if (threadIdx.x == 0) atomicAdd(&g_wait_timeouts, 1u);
    if (warp == kCopyWarp && lane == 0)  // nor any copy
      for (int i = max(0, copied - S::kStages); i < copied; ++i) wait_on(codes + i % S::kStages, i / S::kStages & 1);
    __syncthreads();
  }
  asm volatile("tcgen05.fence::after_thread_sync;");
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmemCols));
}

// The driver's encoder of tensor maps, looked up once.
using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                              const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encoder() {
  static const EncodeFn fn = [] {
    void *f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      f = nullptr;
    return (EncodeFn)f;
  }();
  return fn;
}

// Rows of `bytes` bytes, in boxes of `box` rows by 128 bytes.
bool make_map(CUtensorMap *m, const void *base, int64_t rows, int bytes, int box) {
  const EncodeFn fn = encoder();
  const cuuint64_t dims[2] = {(cuuint64_t)bytes, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)bytes};
  const cuuint32_t boxes[2] = {(cuuint32_t)kRowBytes, (cuuint32_t)box}, steps[2] = {1, 1};
  return fn && fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, boxes, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int TN>
int launch_tc(const Mx4Args &p, int64_t row_tiles, cudaStream_t st, const char *who) {
  using S = Shape<TN>;
  auto k = linear_mx4_tc_kernel<T, TN>;
  const int rc = allow_smem((const void *)k, S::kSmem, who);
  if (rc) return rc;
  CUtensorMap xmap, wmap;
  if (!make_map(&xmap, p.xq, p.rows, p.K / 2, TN) || !make_map(&wmap, p.wq, (int64_t)p.nexp * p.N, p.K / 2, kTM))
    return set_error(DP_ERR_CUDA, "%s: no tensor map", who);
  const int64_t tiles = row_tiles * ((p.N + kTM - 1) / kTM);
  k<<<(unsigned)(tiles < 152 ? tiles : 152), kThreads, S::kSmem, st>>>(p, xmap, wmap);
  return DP_OK;
}
}  // namespace mx4

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
  const int eights = code_cols(K) / 8, most = 32 * kQuantEights<T>, slices = (eights + most - 1) / most;
  const int part = ((eights + slices - 1) / slices + 31) / 32 * 32;  // all lanes of a warp, and whole blocks of 32 elements
  const bool whole = (((uintptr_t)x | (uintptr_t)(K * sizeof(T))) & 15) == 0;
  auto k = !whole   ? quant_rows_mx4_kernel<T, kAny>
           : K % 64 ? quant_rows_mx4_kernel<T, kWhole>
                    : quant_rows_mx4_kernel<T, kExact>;
  const int token_bits = slices == 1 ? 2 : slices == 2 ? 1 : 0, tokens = 1 << token_bits;  // of a block
  const int warps = slices * tokens < 8 ? slices * tokens : 8;
  const dim3 grid((unsigned)((ntok + tokens - 1) / tokens), (unsigned)((slices + 7) / 8));
  k<<<grid, warps * 32, 0, (cudaStream_t)stream>>>(x, src, pos, ntok, topk, K, part, token_bits, xq, sx);
  return launch_status(who);
}

// Which kernel.  One or two rows: the tiles' start costs 2 us more than a short dot product (back to back, us, few and
// tiles of 64: 1 row of 1600 -> 2048 6.2 and 8.2, 2 rows of it in two experts 8.3 and 8.3, 2 rows of 4096 -> 4096 12.9 and
// 11.1, 1 row of 8192 -> 8192 20.6 and 16.4, 4 rows of 1600 -> 2048 8.2 and 8.2).  Tiles of more rows need fewer rounds over
// 152 SMs, and a round of them takes little longer: 2.8, 3.2 and 3.8 us at K 2048 for 64, 128 and 192 rows.
enum Mx4Form { kFew, kTiles64, kTiles128, kTiles192 };
Mx4Form form_of(int64_t rows, int K, int N, int nexp) {
  if (rows <= kFewRows && rows * K * N <= 1 << 23) return kFew;
  auto cost = [&](int R) {
    const int64_t rounds = (((rows + R - 1) / R + nexp / 2) * ((N + mx4::kTM - 1) / mx4::kTM) + 151) / 152;
    return rounds * (R + 280);
  };
  const int64_t c64 = cost(64), c128 = cost(128), c192 = cost(192);
  return c192 < c128 && c192 < c64 ? kTiles192 : c128 < c64 ? kTiles128 : kTiles64;
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
  const Mx4Args p{xq, sx, wq, sw, bias, start, (int)rows, K, N, nexp, act, y, give_up_at()};
  const cudaStream_t st = (cudaStream_t)stream;
  const int64_t pieces = start ? (nexp + 1 < rows ? nexp + 1 : rows) : 0;  // a tile more for each expert's remainder
  auto tiles = [&](int R) { return (rows + R - 1) / R + pieces; };
  int rc = DP_OK;
  switch (form_of(rows, K, N, nexp)) {
    case kFew: {
      const dim3 grid((unsigned)tiles(kFewRows), (N + kFewWarps - 1) / kFewWarps);
      linear_mx4_few_kernel<T><<<grid, kFewWarps * 32, 0, st>>>(p);
      break;
    }
    case kTiles64: rc = mx4::launch_tc<T, 64>(p, tiles(64), st, who); break;
    case kTiles128: rc = mx4::launch_tc<T, 128>(p, tiles(128), st, who); break;
    case kTiles192: rc = mx4::launch_tc<T, 192>(p, tiles(192), st, who); break;
  }
  if (rc) return rc;
  return launch_status(who);
}

}  // namespace

int take_wait_timeouts_linear_mx4(unsigned int *count) { return take_unit_timeouts(count); }

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
