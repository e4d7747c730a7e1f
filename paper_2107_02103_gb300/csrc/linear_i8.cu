// Matrix product in 8-bit integers with a scale for each token (row of x) and each output channel (row of W),
// for one net or for several experts over rows sorted by expert:
//   amax_i = max_k |x_ik|, r_i = 127 / amax_i, q_ik = rint(x_ik r_i), sx_i = amax_i / 127        (f32 arithmetic)
//   y_in = act(float(sum_k q_ik w_nk) sx_i sw_n + b_n)
// The integer sum is exact.  Rows to 8 bits are bound by memory: 65,536 x 1600 f32 in 80 us (6.5 TB/s), to their sorted
// places in 87.
#include "rows.cuh"

namespace dpc {
namespace {

constexpr int kMaxTopk = 64;
constexpr int kMaxK = 65536;  // |q w| <= 2^14: int32 sums hold 2^17 of them

// ------------------------------------------------------------------ rows to 8 bits
constexpr int kQuantKeep = 4;  // packs a lane keeps in registers; longer rows are read again (from L2)

__device__ __forceinline__ float max_nan(float a, float b) {  // NaN wins
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// rint(x r) as the low byte of a float: the product is rounded, then adding 1.5 2^23 leaves its nearest integer
// (ties to even) in the low bits, without the slow conversions.
__device__ __forceinline__ uint32_t to_byte(float x, float r) {
  return __float_as_uint(__fadd_rn(__fmul_rn(x, r), 12582912.0f));
}

// G lanes a row (8 to 256; blocks of 128, or 256).  With pos, token t's row goes to the topk sorted rows pos[t][.],
// and the rows past the kept ones (src < 0) are cleared.  Whole: rows of whole aligned packs.
template <typename T, bool Whole, int G>
__global__ void __launch_bounds__(G == 256 ? 256 : 128)
    quant_rows_kernel(const T *__restrict__ x, const int32_t *__restrict__ src, const int32_t *__restrict__ pos,
                      int64_t ntok, int topk, int K, int ldq, int8_t *__restrict__ xq, float *__restrict__ sx) {
  constexpr int V = 16 / (int)sizeof(T), kTok = G == 256 ? 1 : 128 / G, kStep = G, kW = G <= 32 ? 1 : G / 32;
  __shared__ float part[kTok][kW];
  const int tid = threadIdx.x % G, slot = threadIdx.x / G;
  const int64_t t = (int64_t)blockIdx.x * kTok + slot, n = ntok * topk;
  const bool have = t < ntok;
  const T *row = x + (have ? t : 0) * K;
  const int np = ldq / V;  // packs of the row written, those past K zero
  auto load = [&](int c, float (&v)[V]) {
    Pack<T, V> q{};
    if (have && c * V < K) {
      if constexpr (Whole) q = load_pack<T, V>(row + c * V);
      else q = load_any<T>(row + c * V, x, x + ntok * K);
    }
#pragma unroll
    for (int l = 0; l < V; ++l) v[l] = Whole || c * V + l < K ? (float)to_acc(q.v[l]) : 0.0f;
  };
  // where the first two pairs go, read beside the row
  int place[2] = {-1, -1}, kept[2] = {0, 0};
  if (pos && have)
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (j < topk) {
        place[j] = __ldg(pos + t * topk + j);
        kept[j] = __ldg(src + t * topk + j);
      }
  float keep[kQuantKeep][V], amax = 0.0f;
#pragma unroll
  for (int i = 0; i < kQuantKeep; ++i) load(tid + i * kStep, keep[i]);
#pragma unroll
  for (int i = 0; i < kQuantKeep; ++i)
#pragma unroll
    for (int l = 0; l < V; ++l) amax = max_nan(amax, fabsf(keep[i][l]));
  for (int c = tid + kQuantKeep * kStep; c < np; c += kStep) {
    float v[V];
    load(c, v);
#pragma unroll
    for (int l = 0; l < V; ++l) amax = max_nan(amax, fabsf(v[l]));
  }
#pragma unroll
  for (int o = (G < 32 ? G : 32) / 2; o > 0; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if constexpr (G > 32) {
    if (threadIdx.x % 32 == 0) part[slot][tid / 32] = amax;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kW; ++k) amax = max_nan(amax, part[slot][k]);
  }
  if (!have) return;
  const bool fine = amax >= 0x1p-100f && amax < __uint_as_float(0x7f800000u);
  const float r = fine ? __fdiv_rn(127.0f, amax) : 0.0f;
  const float s = fine ? __fdiv_rn(amax, 127.0f) : amax < 1.0f ? 0.0f : __uint_as_float(0x7fc00000u);
  auto put = [&](int64_t p, int c, const float (&v)[V]) {
    uint32_t b[V];
#pragma unroll
    for (int l = 0; l < V; ++l) b[l] = fine ? to_byte(v[l], r) : 0u;
    int8_t *to = xq + p * ldq + c * V;
    if constexpr (V == 2) {
      *reinterpret_cast<uint16_t *>(to) = (uint16_t)__byte_perm(b[0], b[1], 0x40);
    } else {
      uint32_t w[V / 4];
#pragma unroll
      for (int l = 0; l < V; l += 4)
        w[l / 4] = __byte_perm(__byte_perm(b[l], b[l + 1], 0x40), __byte_perm(b[l + 2], b[l + 3], 0x40), 0x5410);
      if constexpr (V == 4) *reinterpret_cast<uint32_t *>(to) = w[0];
      else *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[V / 4 - 1]);
    }
  };
  for (int j = 0; j < topk; ++j) {
    const int64_t q = t * topk + j, p = !pos ? t : j == 0 ? place[0] : j == 1 ? place[1] : __ldg(pos + q);
    if (p >= 0 && p < n) {
#pragma unroll
      for (int i = 0; i < kQuantKeep; ++i)
        if (tid + i * kStep < np) put(p, tid + i * kStep, keep[i]);
      for (int c = tid + kQuantKeep * kStep; c < np; c += kStep) {
        float v[V];
        load(c, v);
        put(p, c, v);
      }
      if (tid == 0) sx[p] = s;
    }
    if (pos && (j == 0 ? kept[0] : j == 1 ? kept[1] : __ldg(src + q)) < 0) {
      for (int c = tid; c < ldq / 16; c += kStep) reinterpret_cast<uint4 *>(xq + q * ldq)[c] = make_uint4(0, 0, 0, 0);
      if (tid == 0) sx[q] = 0.0f;
    }
  }
}

// ------------------------------------------------------------------ the product
struct I8Args {
  const int8_t *xq, *wq;
  const float *sx, *sw, *bias;
  const int64_t *start;  // [nexp + 1], or NULL: one expert for all rows
  int rows, K, N, nexp, act;
  void *y;
  unsigned char *image;  // the wide form's weights (linear_i8_tc_kernel)
  int give_up;           // the stage of a block whose wait gives up (dp_give_up_at)
};

template <typename T>
__device__ __forceinline__ void put_out(T *y, float v) {
  if constexpr (sizeof(T) == 8) *y = (double)v;
  else *y = from_acc<T>(v);
}

// Row tile `tile` of the sorted rows cut into tiles of at most R rows that lie in one expert: the expert (nexp for
// the rows past start[nexp]) and its rows [r0, r1).  A warp looks at 32 experts at a time.
__device__ __forceinline__ bool find_tile(const I8Args &p, int tile, int R, int &e, int &r0, int &r1) {
  const int rows = p.rows;
  if (!p.start) {
    if (tile >= (rows + R - 1) / R) return false;
    e = 0;
    r0 = tile * R;
    r1 = min(R, rows - r0) + r0;
    return true;
  }
  const int lane = threadIdx.x & 31;
  int before = 0;
  for (int e0 = 0; e0 <= p.nexp; e0 += 32) {
    const int k = e0 + lane;
    int lo = 0, hi = 0;
    if (k <= p.nexp) {
      lo = k ? (int)min(max(__ldg(p.start + k), (int64_t)0), (int64_t)rows) : 0;
      hi = k < p.nexp ? (int)min(max(__ldg(p.start + k + 1), (int64_t)lo), (int64_t)rows) : rows;
    }
    const int mine = (hi - lo + R - 1) / R;
    int inc = mine;
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, before + inc > tile);
    if (hit) {
      const int who = __ffs(hit) - 1;
      const int first = lo + (tile - (before + inc - mine)) * R;
      e = e0 + who;
      r0 = __shfl_sync(0xffffffffu, first, who);
      r1 = min(R, __shfl_sync(0xffffffffu, hi, who) - r0) + r0;
      return true;
    }
    before += __shfl_sync(0xffffffffu, inc, 31);
  }
  return false;
}

constexpr int kFewWarps = 8, kFewRows = 8;

// A warp per output channel and tile of up to eight rows: weights read once per tile, 16 bytes a lane, four products an
// instruction.  Bound by latency: 4 rows of 1600 -> 2432 in 8 us, of which 5 are the launch.
template <typename T>
__global__ void __launch_bounds__(kFewWarps * 32) linear_i8_few_kernel(const I8Args p) {
  int e, r0, r1;
  if (!find_tile(p, blockIdx.x, kFewRows, e, r0, r1)) return;
  const int lane = threadIdx.x & 31, n = blockIdx.y * kFewWarps + (threadIdx.x >> 5), nr = r1 - r0;
  if (n >= p.N) return;
  T *y = (T *)p.y;
  if (e == p.nexp) {
    if (lane < nr) put_out(y + (int64_t)(r0 + lane) * p.N + n, 0.0f);
    return;
  }
  const int8_t *w = p.wq + ((int64_t)e * p.N + n) * p.K, *x = p.xq + (int64_t)r0 * p.K;
  int acc[kFewRows] = {};
  constexpr int kStep = 4;  // 2 KB of the channel on its way at a time
  for (int k0 = lane * 16; k0 < p.K; k0 += kStep * 512) {
    int4 a[kStep];
#pragma unroll
    for (int u = 0; u < kStep; ++u)
      a[u] = k0 + 512 * u < p.K ? __ldg(reinterpret_cast<const int4 *>(w + k0 + 512 * u)) : make_int4(0, 0, 0, 0);
#pragma unroll
    for (int u = 0; u < kStep; ++u)
      if (k0 + 512 * u < p.K)
#pragma unroll
        for (int i = 0; i < kFewRows; ++i)
          if (i < nr) {
            const int4 b = __ldg(reinterpret_cast<const int4 *>(x + (int64_t)i * p.K + k0 + 512 * u));
            acc[i] = __dp4a(a[u].x, b.x, __dp4a(a[u].y, b.y, __dp4a(a[u].z, b.z, __dp4a(a[u].w, b.w, acc[i]))));
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
    put_out(y + (int64_t)(r0 + lane) * p.N + n, v);
  }
}

// ------------------------------------------------------------------ the product on the tensor cores
// A tile is 128 output channels (the MMA's rows) by up to TN sorted rows of one expert (its columns), so that an
// epilogue warp holds 32 neighbouring channels of a row and stores them side by side.  sm_103a multiplies 8-bit
// integers slowly; fp16 holds them exactly, and fp32 sums of their products are exact while K <= 1024
// (1024 * 2^14 = 2^24): longer K is cut into chunks of 1024 whose sums are added as int32.
//   Loader warps read the 8-bit rows from global memory into registers a stage ahead, turn them into fp16
//   (byte q + 128 under the exponent of 1024, less 1152) and write the stage's operands, K-major rows of 128 bytes in
//   the 128-byte swizzle: four neighbouring lanes read 64 bytes of a row (lanes along the rows instead, each in a line
//   of its own, kept L1 busy: 955 us where this took 750), and the swizzle spreads their stores over all banks.
//   One lane of a warp of its own issues a stage's MMAs (M 128, K 16 each).
//   Epilogue warps (two per TMEM lane quadrant, half the columns each) keep the chunks' int32 sums in registers and
//   finish a tile while the next one runs in the other TMEM buffer.
// Two forms.  Up to 128 rows a tile both operands are widened on the way.  Wide tiles of 256 rows, for many rows an
// expert, take the weights widened once (widen_weights_kernel) by bulk copies.
// A block per SM walks the tiles; every wait is bounded, a block that gives up writes NaN and is counted.
// Measured: 32,768 x 2048 x 4096 in 517 us, 1,063 TFLOP/s (55 % of the measured bf16 rate); 65,536 x 1600 x 240 with
// four nets in 92 us, with as many rows each in 87.  Without the epilogue 471 and 74 us, without the loads of x 491 and
// 81: what is left is shared memory: at 128 bytes a cycle a stage's operand writes and MMA reads (48 KB each) take 768
// cycles where its MMAs take 512.  The wide form spills 116 bytes of a thread's registers.
namespace i8 {
constexpr int kTM = 128, kKB = 64, kChunkK = 1024;
constexpr int kEpiWarps = 8;
// The wide form's warpgroups move registers from the loaders and the last group to the epilogue's 128 sums; the
// shares of a scheduler's five warps come to what they were launched with.
constexpr int kRegs = 96, kEpiRegs = 152, kLoadRegs = 72, kMmaRegs = 32;
static_assert(2 * kEpiRegs + 2 * kLoadRegs + kMmaRegs <= 5 * kRegs, "register split");
constexpr uint32_t kRowBytes = kKB * 2, kSBO = 8 * kRowBytes;  // a slice's row; the next 8 rows

template <int TN>
struct Shape {
  static constexpr bool kWide = TN == 256;  // weights come widened, by bulk copies
  // the narrow forms' 13 warps leave 128 registers a thread
  static constexpr int kLoadWarps = kWide ? 8 : 4, kMmaWarp = kEpiWarps + kLoadWarps;
  static constexpr int kThreads = (kMmaWarp + (kWide ? 4 : 1)) * 32;
  static constexpr int kStageA = kTM * kKB * 2, kStageBytes = kStageA + TN * kKB * 2;
  static constexpr int kStages = kWide ? 4 : 6;
  // Two groups of loader warps take the stages in turn: a stage costs a warp some 900 cycles of waiting (barrier,
  // stores, proxy fence) whatever it holds, which the other group's stage hides.  A group holds its next stage in registers.
  static constexpr int kGroups = 2;
  static constexpr uint32_t kTmemCols = 2 * TN;
  static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + (2 * kStages + 5) * 8 + 16;  // aligned within
  static_assert(kSmem <= 227 * 1024 && TN % 64 == 0 && TN <= 256, "tile");
  static_assert(!kWide || (kEpiWarps % 4 == 0 && kLoadWarps % 4 == 0 && kThreads % 128 == 0), "roles of whole warpgroups");
};

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint64_t smem_desc(uint32_t saddr) {  // K-major, 128-byte swizzle, version 1
  return (uint64_t)((saddr & 0x3FFFF) >> 4) | (1ull << 16) | ((uint64_t)(kSBO >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// Byte of the 16-byte chunk c of row r in an operand whose first byte is 1024-byte aligned.
__device__ __forceinline__ uint32_t chunk_at(int r, int c) { return r * kRowBytes + ((c ^ (r & 7)) << 4); }

// Four int8 as two fp16 pairs.
__device__ __forceinline__ void widen(uint32_t q, uint32_t &lo, uint32_t &hi) {
  const uint32_t u = q ^ 0x80808080u;  // q + 128
  lo = __byte_perm(u, 0x64646464u, 0x4140);
  hi = __byte_perm(u, 0x64646464u, 0x4342);  // 1024 + q + 128
  asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(lo) : "r"(0x64806480u));
  asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(hi) : "r"(0x64806480u));
}

// Where a role stands: the tile, and the expert, rows and channels it means.
struct Tile {
  int tile, r0, r1, e, n0;
  bool have;
};
__device__ __forceinline__ void seek(const I8Args &p, int TN, int nct, Tile &t) {
  const int rt = t.tile / nct;
  t.n0 = (t.tile - rt * nct) * kTM;
  t.have = find_tile(p, rt, TN, t.e, t.r0, t.r1);
}

__device__ __forceinline__ void tmem_ld(uint32_t addr, float (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
               : "r"(addr));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st(uint32_t addr, const float (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr), "f"(v[0]), "f"(v[1]),
               "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
}

template <typename T, int TN>
__global__ void __launch_bounds__(Shape<TN>::kThreads, 1) linear_i8_tc_kernel(const I8Args p) {
  using S = Shape<TN>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char *smem = smem_raw + (1024 - (smem_u32(smem_raw) & 1023)) % 1024;
  uint64_t *full = reinterpret_cast<uint64_t *>(smem + S::kStages * S::kStageBytes), *empty = full + S::kStages;
  uint64_t *acc_full = empty + S::kStages, *acc_empty = acc_full + 2, *done = acc_empty + 2;
  uint32_t *holder = reinterpret_cast<uint32_t *>(done + 1);
  volatile int *stop = reinterpret_cast<int *>(holder + 1), *issued = stop + 1;
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
      init(full + s, S::kLoadWarps / S::kGroups + (S::kWide ? 1 : 0));
      init(empty + s, 1);
    }
    for (int b = 0; b < 2; ++b) {
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
  int next = 0;  // stages copied, or a loader's next one

  if (warp >= S::kMmaWarp) {  // in the wide form a warpgroup: one setmaxnreg for all four of its warps
    if constexpr (S::kWide) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kMmaRegs));
    if (warp == S::kMmaWarp) {
      // -------------------------------------------------------------- the MMAs
      int j = 0, unit = 0;  // stages, accumulator uses
      Tile t{(int)blockIdx.x, 0, 0, 0, 0, false};
      for (; ok; t.tile += gridDim.x) {
        seek(p, TN, nct, t);
        if (!t.have) break;
        if (t.e == p.nexp) continue;
        const uint32_t cols = (uint32_t)(t.r1 - t.r0 + 15) / 16 * 16;
        const uint32_t idesc = (1u << 4) | ((uint32_t)(kTM >> 4) << 24) | ((cols >> 3) << 17);
        if (lane == 0) {
          const int end = min(nkb, p.give_up - j);  // outside the loop: inside it costs 7 % of the narrow forms' time
          for (int kb = 0; kb < end && ok; ++kb, ++j) {
            const int st = j % S::kStages, buf = unit & 1, slice = kb % (kChunkK / kKB);
            if (slice == 0 && unit >= 2) ok = wait(acc_empty + buf, ((unit >> 1) - 1) & 1);
            ok = ok && wait(full + st, (j / S::kStages) & 1);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;");
            const uint32_t base = smem_u32(smem) + st * S::kStageBytes;
            const uint64_t a0 = smem_desc(base), b0 = smem_desc(base + S::kStageA);
  #pragma unroll
            for (int k = 0; k < kKB / 16; ++k) {
              const uint32_t acc = slice > 0 || k > 0 ? 1u : 0u;
              asm volatile(
                  "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
                  " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(tmem + (uint32_t)(buf * TN)),
                  "l"(a0 + (uint64_t)(k * 2)), "l"(b0 + (uint64_t)(k * 2)), "r"(idesc), "r"(acc));
            }
            commit(smem_u32(empty + st));
            if (slice == kChunkK / kKB - 1 || kb == nkb - 1) {
              commit(smem_u32(acc_full + buf));
              ++unit;
            }
          }
          ok = ok && end == nkb;
        }
        ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
      }
      if (lane == 0) commit(smem_u32(done));  // completes when every MMA issued above has
      if (!ok) *stop = 1;
    } else if constexpr (S::kWide) {
      // -------------------------------------------------------------- the weights' copies, by one warp; two are idle
      if (warp == S::kMmaWarp + 1) {
        Tile t{(int)blockIdx.x, 0, 0, 0, 0, false};
        for (; ok; t.tile += gridDim.x) {
          seek(p, TN, nct, t);
          if (!t.have) break;
          if (t.e == p.nexp) continue;
          const unsigned char *src = p.image + ((int64_t)t.e * nct + t.n0 / kTM) * nkb * S::kStageA;
          if (lane == 0) {
            for (int kb = 0; kb < nkb; ++kb) {
              const int st = next % S::kStages;
              ok = wait(empty + st, (next / S::kStages & 1) ^ 1);
              if (!ok) break;
              const uint32_t bar = smem_u32(full + st);
              asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)S::kStageA)
                           : "memory");
              asm volatile(
                  "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                      smem_u32(smem) + st * S::kStageBytes),
                  "l"(src + (int64_t)kb * S::kStageA), "r"((uint32_t)S::kStageA), "r"(bar)
                  : "memory");
              ++next;
            }
          }
          ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
        }
        if (!ok) *stop = 1;
        if (lane == 0) *issued = next;
      }
    }
  } else if (warp >= kEpiWarps) {
    // ---------------------------------------------------------------- loaders
    if constexpr (S::kWide) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kLoadRegs));
    constexpr int kLR = S::kLoadWarps / S::kGroups * 8;  // rows a group covers at once
    constexpr int kA = S::kWide ? 0 : kTM / kLR, kB = TN / kLR, kU = kA + kB;
    const int kp = lane & 3, lw = warp - kEpiWarps, row = (lw / S::kGroups) * 8 + (lane >> 2);
    const uint32_t put = smem_u32(smem), put0 = chunk_at(row, 2 * kp), put1 = chunk_at(row, 2 * kp + 1);
    int tile = blockIdx.x, k = 0;             // where the loads stand: the tile, this thread's column in it,
    int now = 0;                              // its columns (rows of x, whole sixteens), 0 past the last tile,
    uint32_t rows = 0;                        // which of this thread's rows exist,
    const int8_t *w = nullptr, *x = nullptr;  // and its first row of either operand at column k
    const int step = kLR * p.K;               // bytes to the thread's next row
    auto next_tile = [&] {                    // to the next tile with work, from `tile` on
      now = 0;
      for (;; tile += gridDim.x) {
        Tile t{tile, 0, 0, 0, 0, false};
        seek(p, TN, nct, t);
        if (!t.have) return;
        if (t.e == p.nexp) continue;
        k = kp * 16;
        if constexpr (kA > 0) w = p.wq + ((int64_t)t.e * p.N + t.n0 + row) * p.K + k;
        x = p.xq + (int64_t)(t.r0 + row) * p.K + k;
        rows = 0;
#pragma unroll
        for (int i = 0; i < kU; ++i)
          rows |= (uint32_t)(i < kA ? t.n0 + row + kLR * i < p.N : row + kLR * (i - kA) < t.r1 - t.r0) << i;
        now = (t.r1 - t.r0 + 15) / 16 * 16;
        return;
      }
    };
    next_tile();
    uint4 raw[kU];
    uint32_t wanted = 0;  // this thread's rows of the stage where the loads stand
    auto load = [&](int i) {
      raw[i] = make_uint4(0, 0, 0, 0);
      if (wanted >> i & 1) raw[i] = __ldg(reinterpret_cast<const uint4 *>((i < kA ? w : x) + (int64_t)step * (i < kA ? i : i - kA)));
    };
    auto advance = [&] {  // one slice on
      if (!now) return;
      k += kKB;
      if constexpr (kA > 0) w += kKB;
      x += kKB;
      if (k - kp * 16 >= p.K) {
        tile += gridDim.x;
        next_tile();
      }
    };
    int st = lw % S::kGroups, round = 0;  // the stage, and its turn (the wait of the first passes)
    for (int g = 0; g < st; ++g) advance();
    static_assert(S::kGroups == 2 && S::kStages % S::kGroups == 0, "stages in turn");
    int c = now;
    wanted = now && k < p.K ? rows : 0u;
#pragma unroll
    for (int i = 0; i < kU; ++i) load(i);
    while (c) {
      ok = __all_sync(0xffffffffu, wait(empty + st, (round & 1) ^ 1));
      if (!ok) break;
      const uint32_t dst = put + st * S::kStageBytes;
      const int cols = c;
      advance();
      advance();
      c = now;
      wanted = now && k < p.K ? rows : 0u;
#pragma unroll
      for (int i = 0; i < kU; ++i) {
        if (i < kA || row + kLR * (i - kA) < cols) {
          uint32_t h[8];
          widen(raw[i].x, h[0], h[1]);
          widen(raw[i].y, h[2], h[3]);
          widen(raw[i].z, h[4], h[5]);
          widen(raw[i].w, h[6], h[7]);
          const uint32_t d = dst + (i < kA ? i * (kLR / 8) * kSBO : S::kStageA + (i - kA) * (kLR / 8) * kSBO);
          asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(d + put0), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
          asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(d + put1), "r"(h[4]), "r"(h[5]), "r"(h[6]), "r"(h[7]) : "memory");
        }
        load(i);  // the group's next stage, on its way during the fence and the next wait
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) arrive(smem_u32(full + st));
      if ((st += S::kGroups) >= S::kStages) {
        st -= S::kStages;
        ++round;
      }
    }
    next = round * S::kStages + st;
    if (!ok) *stop = 1;
  } else {
    // ---------------------------------------------------------------- epilogue
    if constexpr (S::kWide) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kEpiRegs));
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
      const int chunks = (nkb * kKB + kChunkK - 1) / kChunkK;
      if (chunks > 1) {
        int sum[CW];
#pragma unroll
        for (int i = 0; i < CW; ++i) sum[i] = 0;
#pragma unroll 1
        for (int c = chunks;; ++unit) {
          ok = __all_sync(0xffffffffu, ok && wait(acc_full + (unit & 1), (unit >> 1) & 1));
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;");
          const uint32_t col = trow + (unit & 1) * TN;
#pragma unroll
          for (int g = 0; g < CW; g += 8) {
            float v[8];
            tmem_ld(col + g, v);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[g + i] += __float2int_rn(v[i]);
          }
          if (--c == 0) {  // the sums go back to be finished below
#pragma unroll
            for (int g = 0; g < CW; g += 8) {
              float v[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) v[i] = __int2float_rn(sum[g + i]);
              tmem_st(col + g, v);
            }
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            break;
          }
          asm volatile("tcgen05.fence::before_thread_sync;");
          __syncwarp();
          if (lane == 0) arrive(smem_u32(acc_empty + (unit & 1)));
        }
      } else {
        ok = __all_sync(0xffffffffu, ok && wait(acc_full + (unit & 1), (unit >> 1) & 1));
        asm volatile("tcgen05.fence::after_thread_sync;");
      }
      const float sw = mine ? __ldg(p.sw + (int64_t)t.e * p.N + n) : 0.0f;
      const float bias = mine && p.bias ? __ldg(p.bias + (int64_t)t.e * p.N + n) : 0.0f;
      T *out = y + (int64_t)(t.r0 + c0) * p.N + n;
#pragma unroll 1
      for (int g = 0; g < CW && c0 + g < nr; g += 16, out += (int64_t)16 * p.N) {
        const int left = nr - c0 - g;
        const float scale = lane < min(left, 16) ? __ldg(p.sx + t.r0 + c0 + g + lane) : 0.0f;
        float v[16], v1[8];
        if (ok) {
          tmem_ld(trow + (unit & 1) * TN + g, reinterpret_cast<float(&)[8]>(v));
          tmem_ld(trow + (unit & 1) * TN + g + 8, v1);
          tmem_wait_ld();
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[8 + i] = v1[i];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = fmaf(v[i] * __shfl_sync(0xffffffffu, scale, i), sw, bias);
        if (p.act == DP_ACT_TANH) {
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = tanhf(v[i]);
        }
        T *o = out;
        if (ok && left >= 16) {
          if (mine)
#pragma unroll
            for (int i = 0; i < 16; ++i, o += p.N) put_out(o, v[i]);
        } else if (mine) {
#pragma unroll
          for (int i = 0; i < 16; ++i, o += p.N)
            if (i < left) put_out(o, ok ? v[i] : __uint_as_float(0x7fc00000u));
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
    if constexpr (S::kWide) {  // nor any copy: the loaders' arrivals that its stage lacks, then the copy
      if (lane == 0 && warp >= kEpiWarps && warp < S::kMmaWarp)
        for (; next < *issued; next += S::kGroups) arrive(smem_u32(full + next % S::kStages));
      if (lane == 0 && warp == S::kMmaWarp + 1)
        for (int i = max(0, next - S::kStages); i < next; ++i) wait_on(full + i % S::kStages, i / S::kStages & 1);
      __syncthreads();
    }
  }
  asm volatile("tcgen05.fence::after_thread_sync;");
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmemCols));
}

// The wide form's weights: fp16 as the shared-memory image of each (128 channels, 64 of K) block, 16 KB apiece,
// channels and columns past the end zero.  A warp widens eight channels' 64 columns.
__global__ void __launch_bounds__(256) widen_weights_kernel(const int8_t *__restrict__ wq, int K, int N, int nexp,
                                                            unsigned char *__restrict__ image) {
  const int nct = (N + kTM - 1) / kTM, nkb = (K + kKB - 1) / kKB, lane = threadIdx.x & 31, r8 = lane >> 2, kp = lane & 3;
  const int64_t groups = (int64_t)nexp * nct * (kTM / 8) * nkb;
  for (int64_t g = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); g < groups; g += (int64_t)gridDim.x * 8) {
    const int kb = (int)(g % nkb), rg = (int)(g / nkb % (kTM / 8));
    const int64_t ect = g / nkb / (kTM / 8);
    const int n = (int)(ect % nct) * kTM + rg * 8 + r8, k = kb * kKB + kp * 16;
    uint4 q = make_uint4(0, 0, 0, 0);
    if (n < N && k < K) q = __ldg(reinterpret_cast<const uint4 *>(wq + ((ect / nct) * N + n) * K + k));
    uint4 lo, hi;
    widen(q.x, lo.x, lo.y);
    widen(q.y, lo.z, lo.w);
    widen(q.z, hi.x, hi.y);
    widen(q.w, hi.z, hi.w);
    unsigned char *dst = image + (ect * nkb + kb) * (kTM * kKB * 2) + rg * kSBO;
    *reinterpret_cast<uint4 *>(dst + chunk_at(r8, 2 * kp)) = lo;
    *reinterpret_cast<uint4 *>(dst + chunk_at(r8, 2 * kp + 1)) = hi;
  }
}

size_t image_bytes(int K, int N, int nexp) {
  return (size_t)nexp * ((N + kTM - 1) / kTM) * ((K + kKB - 1) / kKB) * (kTM * kKB * 2);
}

template <typename T, int TN>
int launch_tc(const I8Args &p, int64_t row_tiles, cudaStream_t st, const char *who) {
  using S = Shape<TN>;
  auto k = linear_i8_tc_kernel<T, TN>;
  cudaFuncAttributes a{};
  cudaError_t e = cudaSuccess;
  if (S::kWide) e = cudaFuncGetAttributes(&a, k);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem);
  if (e != cudaSuccess) return set_error(DP_ERR_CUDA, "%s: %s", who, cudaGetErrorString(e));
  // the epilogue's registers come out of what the block is launched with
  if (S::kWide && a.numRegs < kRegs) return set_error(DP_ERR_CUDA, "%s: kernel of %d registers", who, a.numRegs);
  if (S::kWide) {
    const int64_t warps = (int64_t)p.nexp * ((p.N + kTM - 1) / kTM) * (kTM / 8) * ((p.K + kKB - 1) / kKB);
    const int64_t blocks = (warps + 7) / 8;
    widen_weights_kernel<<<(unsigned)(blocks < 152 * 8 ? blocks : 152 * 8), 256, 0, st>>>(p.wq, p.K, p.N, p.nexp, p.image);
  }
  const int64_t tiles = row_tiles * ((p.N + kTM - 1) / kTM);
  k<<<(unsigned)(tiles < 152 ? tiles : 152), S::kThreads, S::kSmem, st>>>(p);
  return DP_OK;
}
}  // namespace i8

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
  if (!at_elements(x, sx, src, pos)) return misaligned(who);
  const int ldq = (K + 15) / 16 * 16, packs = ldq / (16 / (int)sizeof(T));
  const bool whole = (((uintptr_t)x | (uintptr_t)(K * sizeof(T))) & 15) == 0;
  auto go = [&](auto G) {
    constexpr int g_ = decltype(G)::value, threads = g_ == 256 ? 256 : 128, tok = threads / g_;
    auto k = whole ? quant_rows_kernel<T, true, g_> : quant_rows_kernel<T, false, g_>;
    k<<<(unsigned)((ntok + tok - 1) / tok), threads, 0, (cudaStream_t)stream>>>(x, src, pos, ntok, topk, K, ldq, xq, sx);
  };
  if (packs <= 8 * kQuantKeep) go(std::integral_constant<int, 8>{});  // as many lanes as hold the row
  else if (packs <= 32 * kQuantKeep) go(std::integral_constant<int, 32>{});
  else if (packs <= 64 * kQuantKeep) go(std::integral_constant<int, 64>{});
  else if (packs <= 128 * kQuantKeep) go(std::integral_constant<int, 128>{});
  else go(std::integral_constant<int, 256>{});
  return launch_status(who);
}

// Which kernel.  Measured (us, one net of 2048 -> 4096, bf16): 16 rows 17 few, 21 tiles of 64; 32 rows 27 and 21; 256
// rows 22 by 64, 24 by 128; 512 rows 36 by 64, 25 by 128, 37 wide; 1024 rows 42 by 128, 38 wide; 4096 rows 125 by 128,
// 93 wide.  Below 2^33 products the widening launch costs more than it saves (16,384 rows of 240 -> 240: 13 by 128, 21
// wide).  Between 64 and 128 by their rounds over 152 SMs, one of 128 costing a fifth more.
enum I8Form { kFew, kTiles64, kTiles128, kWideTiles };
I8Form form_of(int64_t rows, int K, int N, int nexp) {
  if (rows <= 16) return kFew;
  if (rows / nexp >= 512 && (double)rows * K * N >= 8589934592.0) return kWideTiles;
  auto rounds = [&](int R) { return (((rows + R - 1) / R + nexp / 2) * ((N + i8::kTM - 1) / i8::kTM) + 151) / 152; };
  return 6 * rounds(128) < 5 * rounds(64) ? kTiles128 : kTiles64;
}

template <typename T>
int linear(const int8_t *xq, const float *sx, int64_t rows, int K, const int8_t *wq, const float *sw, const float *bias,
           int nexp, int N, const int64_t *start, int act, T *y, void *work, size_t work_bytes, void *stream,
           const char *who) {
  clear_error();
  if (rows < 0 || rows > 0x7fffffffLL - 1024) return set_error(DP_ERR_SHAPE, "%s: rows = %lld", who, (long long)rows);
  if (K < 16 || K % 16) return set_error(DP_ERR_SHAPE, "%s: K = %d is not a positive multiple of 16", who, K);
  if (K > kMaxK) return set_error(DP_ERR_UNSUPPORTED, "%s: K = %d > %d", who, K, kMaxK);
  if (N < 1 || N > (1 << 18)) return set_error(DP_ERR_SHAPE, "%s: N = %d outside [1, 2^18]", who, N);
  if (nexp < 1 || nexp > 1024) return set_error(DP_ERR_SHAPE, "%s: nexp = %d outside [1, 1024]", who, nexp);
  if (act != DP_ACT_NONE && act != DP_ACT_TANH) return set_error(DP_ERR_SHAPE, "%s: act = %d", who, act);
  if (nexp > 1 && !start) return set_error(DP_ERR_NULL, "%s: start is NULL with %d experts", who, nexp);
  if (rows == 0) return DP_OK;
  if (!xq || !sx || !wq || !sw || !y) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (((uintptr_t)xq | (uintptr_t)wq) & 15) return set_error(DP_ERR_SHAPE, "%s: xq or wq is not 16-byte aligned", who);
  if (!at_elements(y, sx, sw, bias, start)) return misaligned(who);
  const I8Form form = form_of(rows, K, N, nexp);
  if (form == kWideTiles) {
    if (!work) return set_error(DP_ERR_NULL, "%s: work is NULL", who);
    if (work_bytes < i8::image_bytes(K, N, nexp) || ((uintptr_t)work & 15))
      return set_error(DP_ERR_SHAPE, "%s: work buffer of %zu bytes is too short or misaligned", who, work_bytes);
  }
  const I8Args p{xq, wq, sx, sw, bias, start, (int)rows, K, N, nexp, act, y, (unsigned char *)work, give_up_at()};
  const cudaStream_t st = (cudaStream_t)stream;
  const int64_t pieces = start ? (nexp + 1 < rows ? nexp + 1 : rows) : 0;  // a tile more for each expert's remainder
  auto tiles = [&](int R) { return (rows + R - 1) / R + pieces; };
  int rc = DP_OK;
  switch (form) {
    case kFew: {
      const dim3 grid((unsigned)tiles(kFewRows), (N + kFewWarps - 1) / kFewWarps);
      linear_i8_few_kernel<T><<<grid, kFewWarps * 32, 0, st>>>(p);
      break;
    }
    case kTiles64: rc = i8::launch_tc<T, 64>(p, tiles(64), st, who); break;
    case kTiles128: rc = i8::launch_tc<T, 128>(p, tiles(128), st, who); break;
    case kWideTiles: rc = i8::launch_tc<T, 256>(p, tiles(256), st, who); break;
  }
  if (rc) return rc;
  return launch_status(who);
}

}  // namespace

int take_wait_timeouts_linear_i8(unsigned int *count) { return take_unit_timeouts(count); }

}  // namespace dpc

extern "C" {

size_t dp_linear_i8_work_bytes(int64_t rows, int K, int N, int nexp) {
  if (rows < 0 || K < 1 || N < 1 || nexp < 1 || dpc::form_of(rows, K, N, nexp) != dpc::kWideTiles) return 0;
  return dpc::i8::image_bytes(K, N, nexp);
}

#define DP_I8(X, C, T)                                                                                                 \
  int dp_quant_rows_i8_##X(const C *x, const int32_t *src, const int32_t *pos, int64_t ntok, int topk, int K,          \
                           int8_t *xq, float *sx, void *stream) {                                                      \
    return dpc::quant_rows<T>((const T *)x, src, pos, ntok, topk, K, xq, sx, stream, "dp_quant_rows_i8_" #X);          \
  }                                                                                                                    \
  int dp_linear_i8_##X(const int8_t *xq, const float *sx, int64_t rows, int K, const int8_t *wq, const float *sw,      \
                       const float *bias, int nexp, int N, const int64_t *start, int act, C *y, void *work,            \
                       size_t work_bytes, void *stream) {                                                              \
    return dpc::linear<T>(xq, sx, rows, K, wq, sw, bias, nexp, N, start, act, (T *)y, work, work_bytes, stream,        \
                          "dp_linear_i8_" #X);                                                                         \
  }
DP_I8(f64, double, double)
DP_I8(f32, float, float)
DP_I8(bf16, uint16_t, __nv_bfloat16)
DP_I8(f16, uint16_t, __half)

}  // extern "C"
