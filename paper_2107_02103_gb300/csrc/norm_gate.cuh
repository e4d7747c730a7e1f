// The norms before and after a block, fused with the block's gate and residual scale, and their backward.
// With x^ = (v - m) s over a row of H (root-mean-square norm: m = 0, s = (mean v^2 + eps)^-1/2; layer norm:
// m = mean v, s = (mean (v - m)^2 + eps)^-1/2):
//   p = f^ w1 (+ b1)          the norm after the block, of the block's output f
//   r2 = r + a G p            gate G ([ntok][H], [ntok] or none), residual scale a [H]
//   u = r2^ w2 (+ b2)         the norm before the next block, of the new residual stream
// Backward, from dr2 and du:
//   t = du w2;   dr = dr2 + s2 (t - r2^ mean(t r2^) - mean t)            (mean t for the layer norm only)
//   dp = dr a G; t1 = dp w1;  df = s1 (t1 - f^ mean(t1 f^) - mean t1);   dG = dr a p
//   da = sum_t dr G p, dw1 = sum_t dp f^, db1 = sum_t dp, dw2 = sum_t du r2^, db2 = sum_t du
// A row lives in the registers of one warp (short rows) or one block, so each array is moved once; the layer
// norm's variance is taken around the mean in a second sweep of the registers.
// f32 is bound by memory: 24,576 x 2048 with a full gate 154 us forward (6.5 TB/s), 272 us backward (5.9 TB/s).  16-bit
// rows, twice the elements a byte, are bound by instructions and the waits of a row's four block sums: layer norm of
// 65,536 x 1600 bf16 248 us (4.2 TB/s) and 396 us (4.2 TB/s).  The registers do not hold everything in the backward of
// rows past 4096 elements (64 a thread; 0.1 to 0.4 KB of them spilled, 0.9 to 1.9 KB past 8192) nor in f64 (forward 50 to
// 150 bytes, backward 0.2 to 0.6 KB, up to 3.3 KB past 8192): 8,000 x 6000 f32 152 and 338 us, 4,000 x 16384 f32 400 and
// 1,653 us with layer norm.  f64 is bound by the FP64 pipe's instructions, of which the elements' own, some 12 each
// forward, are 0.6 of 1.60 ms for a layer norm of 20,000 x 1600; the rest is that every thread finishes a row's sums,
// root and division for itself.  Backward 2.39 ms; root-mean-square norm without a gate 1.01 and 1.68 ms.
#pragma once

#include <algorithm>

#include "rows.cuh"

namespace dpc {
namespace {

constexpr int kNormMaxH = 16384;
constexpr int kNormVectors = 5;  // da, dw1, dw2, db1, db2

// The warps' partial sums of a block, two sets used in turn (one barrier a sum); a value's partials lie side by side
// and are read as vectors, unused warps' stay zero.
template <typename A, int kWarps>
struct SumBuf {
  alignas(16) A v[2][3][(kWarps + 3) / 4 * 4];
};

// Sums of NV values over the row's threads (a warp, or the block), the same bits in every thread.
template <int NV, bool kWarpRow, typename A, int kWarps>
__device__ __forceinline__ void row_sum(A (&v)[NV], SumBuf<A, kWarps> &buf, int &phase) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if constexpr (!kWarpRow) {
    constexpr int kP = 16 / (int)sizeof(A);
    if ((threadIdx.x & 31) == 0)
#pragma unroll
      for (int i = 0; i < NV; ++i) buf.v[phase][i][threadIdx.x >> 5] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      A s[kP] = {};
#pragma unroll
      for (int w = 0; w < (kWarps + 3) / 4 * 4; w += kP) {
        const Pack<A, kP> x = load_pack<A, kP>(buf.v[phase][i] + w);
#pragma unroll
        for (int k = 0; k < kP; ++k) s[k] += x.v[k];
      }
      v[i] = kP == 4 ? (s[0] + s[1]) + (s[kP / 2] + s[kP - 1]) : s[0] + s[1];
    }
    phase ^= 1;
  }
}

template <typename A>
__device__ __forceinline__ A inv_sqrt(A x) {
  if constexpr (sizeof(A) == 8) return 1.0 / sqrt(x);
  else return rsqrtf(x);
}

template <typename A>
__device__ __forceinline__ A nan_of() {
  return A(__int_as_float(0x7fc00000));
}

// Means m and inverse deviations s of R rows held as v[R][EPT] per thread; v becomes v - m.  A row that is not ok in
// any of its threads gets s (and a layer norm's m) NaN in all of them.
template <int R, int EPT, bool kWarpRow, bool kLayer, typename Map, typename A, typename Buf>
__device__ __forceinline__ void row_stats(const Map &map, A (&v)[R][EPT], const bool (&ok)[R], A inv, A eps, A (&m)[R],
                                          A (&s)[R], Buf &buf, int &phase) {
  A sum[R];
#pragma unroll
  for (int k = 0; k < R; ++k) m[k] = A(0);
  if constexpr (kLayer) {
#pragma unroll
    for (int k = 0; k < R; ++k) sum[k] = ok[k] ? map.total([&](int i) { return v[k][i]; }) : nan_of<A>();
    row_sum<R, kWarpRow>(sum, buf, phase);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      m[k] = sum[k] * inv;
#pragma unroll
      for (int i = 0; i < EPT; ++i) v[k][i] -= m[k];
    }
  }
#pragma unroll
  for (int k = 0; k < R; ++k) sum[k] = ok[k] || kLayer ? map.total([&](int i) { return v[k][i] * v[k][i]; }) : nan_of<A>();
  row_sum<R, kWarpRow>(sum, buf, phase);
#pragma unroll
  for (int k = 0; k < R; ++k) s[k] = inv_sqrt(fma(sum[k], inv, eps));
}

// A thread's elements of a row: packs first + i * step, i < EPT / V.  Packs past the row's end repeat its last one
// (so that loads need no zeros) and are left out of sums and stores.
//
// Cut rows (of a length that is no multiple of 16 bytes, in arrays that begin at one): the packs are the aligned words
// under the row, `off` elements of the first lie before it, and the ends' packs are partly the neighbours'.  Blocks
// take rows a multiple of eight apart, which all begin at the same place in their word, so that off, the columns a
// thread sums and the weights beside its elements stay the same for all of a block's rows.
template <typename T, int V, int EPT, bool kCut>
struct RowMap {
  static constexpr int kN = EPT / V;
  int first, step, np;  // first pack, stride between packs, packs in the row
  int off, H;           // cut rows only
  __device__ __forceinline__ bool in(int i) const { return first + i * step < np; }
  __device__ __forceinline__ int at(int i) const { return min(first + i * step, np - 1) * V; }
  // Whether element l of pack i is the row's; its pack must be in.
  __device__ __forceinline__ bool mine(int i, int l) const {
    return !kCut || (unsigned)(at(i) + l - off) < (unsigned)H;
  }
  template <typename S, typename A>
  __device__ __forceinline__ void load(const S *row, A (&v)[EPT]) const {
    Pack<S, V> x[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) x[i] = load_pack<S, V>(row + at(i));
#pragma unroll
    for (int i = 0; i < EPT; ++i) v[i] = to_acc(x[i / V].v[i % V]);
  }
  // The shared weights, read for every row again: they stay in L1 (cut rows: in shared memory, moved by off) and would
  // cost 40 registers otherwise.  Vec: their arrays are 16-byte aligned and V elements a multiple of 16 bytes.
  template <bool Vec, typename A>
  __device__ __forceinline__ void weights(const A *w, A (&v)[EPT]) const {
    constexpr int kP = Vec ? 16 / (int)sizeof(A) : 1;
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int l = 0; l < V; l += kP) {
        const Pack<A, kP> x = load_pack<A, kP>(w + at(i) + l);
#pragma unroll
        for (int k = 0; k < kP; ++k) v[i * V + l + k] = x.v[k];
      }
  }
  template <typename A>
  __device__ __forceinline__ void store(T *row, const A (&v)[EPT]) const {
    if constexpr (kCut) row -= off;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      Pack<T, V> x;
#pragma unroll
      for (int l = 0; l < V; ++l) x.v[l] = from_acc<T>(v[i * V + l]);
      if (!in(i)) continue;
      if (mine(i, 0) && mine(i, V - 1)) store_pack<T, V>(row + at(i), x);
      else
#pragma unroll
        for (int l = 0; l < V; ++l)
          if (mine(i, l)) row[at(i) + l] = x.v[l];
    }
  }
  // The sum of f(i) over the elements that are in the row.
  template <typename F>
  __device__ __forceinline__ auto total(F f) const {
    using A = decltype(f(0));
    A s = 0;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      A q = mine(i, 0) ? f(i * V) : A(0);
#pragma unroll
      for (int l = 1; l < V; ++l) q += mine(i, l) ? f(i * V + l) : A(0);
      s += in(i) ? q : A(0);
    }
    return s;
  }
};

// Bytes a cut row of H may lie under.
template <typename T>
__host__ __device__ constexpr uint32_t cut_bytes(int H) {
  return (uint32_t)((H * sizeof(T) + 30) / 16 * 16);
}

template <typename T>
struct NormArgs {
  const T *in[5];  // the arrays a row is read from: forward f, r, gate; backward r2, du, dr2, f, gate
  int nin;         // how many of them (the gate only if it has a value for each element)
  const T *gate;   // a value for each token, or NULL
  const acc_t<T> *a, *w1, *b1, *w2, *b2;
  int64_t ntok;
  int H, stages;  // stages: rows a block of the bulk form has in shared memory
  int64_t fetched;  // rows that bulk copies fetch: ntok, or fewer for a test of waits that give up (dp_give_up_at)
  acc_t<T> eps;
  T *r2, *u;
  acc_t<T> *stats;  // [ntok][4]: m1, s1, m2, s2
  T *dr, *df, *dgate;
  acc_t<T> *part;  // [blocks][5][H] partial column sums
};

// How rows reach a block: plain loads, or whole rows copied ahead into shared memory in bulk, `stages` rows deep
// (kCut: the aligned words under the rows).  A stage may be refilled once every thread has read it, which the first
// block sum of a row implies.
//
// Waits are bounded.  A thread whose wait gives up puts NaN into the row's first sum, which all threads of the block
// see, and raises `lost`, which tells that NaN from one of the data.  The block then leaves its loop, before it fetches
// anything more, waits once more for what is in flight, and fills this row and its later ones with NaN.
enum Feed { kPlain, kBulkRows, kCutRows };
constexpr int kMaxStages = 4;
constexpr unsigned kNoRow = 0xffffffffu;
constexpr int kRowPolls = 1 << 16;  // of a wait for a row: 0.3 s

template <typename T, int V, int EPT, Feed kFeed>
struct RowFeed {
  static constexpr bool kBulk = kFeed != kPlain, kCut = kFeed == kCutRows;
  const NormArgs<T> &p;
  const RowMap<T, V, EPT, kCut> &map;
  int64_t t, step;  // the row at hand, and to the next one
  unsigned char *smem;
  uint64_t *bars;
  volatile unsigned *lost;
  int st = 0, phase = 0;

  __device__ __forceinline__ uint32_t row_bytes() const {  // of a place in a stage
    return kCut ? cut_bytes<T>(p.H) : (uint32_t)p.H * sizeof(T);
  }
  __device__ __forceinline__ uint32_t bar(int s) const { return (uint32_t)__cvta_generic_to_shared(bars + s); }
  // Called by lane 0 of each warp, which copies its arrays of the row, counted on the stage's barrier (one warp copying
  // all of them kept the others waiting).
  __device__ __forceinline__ void fetch(int64_t row, int s) const {
    const uint32_t place = row_bytes(), dst = (uint32_t)__cvta_generic_to_shared(smem) + s * p.nin * place;
    uint32_t bytes = place;
    if constexpr (kCut)  // the last row's last word may reach past the array: load() takes what is left out here
      bytes = row == p.ntok - 1 ? (uint32_t)(map.off + p.H) * sizeof(T) & ~15u : (uint32_t)map.np * 16u;
    for (int i = threadIdx.x >> 5; i < p.nin; i += blockDim.x >> 5) {
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar(s)), "r"(bytes) : "memory");
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                       dst + i * place),
                   "l"(p.in[i] + row * p.H - (kCut ? map.off : 0)), "r"(bytes), "r"(bar(s))
                   : "memory");
    }
  }
  __device__ __forceinline__ void begin() {
    if constexpr (kBulk) {
      if (threadIdx.x == 0) {
        *lost = kNoRow;
        for (int s = 0; s < p.stages; ++s) asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar(s)), "r"(p.nin));
        asm volatile("fence.mbarrier_init.release.cluster;");
      }
      __syncthreads();
      for (int s = 0; s < p.stages; ++s)
        if ((threadIdx.x & 31) == 0 && t + s * step < p.fetched) fetch(t + s * step, s);
    }
  }
  // The stage k rows on, and the parity of its barrier.
  __device__ __forceinline__ int stage(int k) const { return st + k < p.stages ? st + k : st + k - p.stages; }
  __device__ __forceinline__ uint32_t parity(int k) const { return phase ^ (st + k >= p.stages); }
  __device__ __forceinline__ bool arrived(int k = 0) const {
    if constexpr (kBulk) {
      const bool ok = bounded_wait<kRowPolls>(bar(stage(k)), parity(k), [] { return false; });
      if (!ok) *lost = (unsigned)t;
      return ok;
    }
    return true;
  }
  // Whether a wait of the rows at hand gave up in any thread of the block; first: their first sum, or what follows from it.
  template <typename A>
  __device__ __forceinline__ bool given_up(A first) const {
    if constexpr (kBulk) return first != first && *lost <= (unsigned)t;
    return false;
  }
  template <typename A>
  __device__ __forceinline__ void load(int i, A (&v)[EPT], int k = 0) const {
    if constexpr (kBulk) map.load(reinterpret_cast<const T *>(smem + (stage(k) * p.nin + i) * row_bytes()), v);
    else map.load(p.in[i] + (t + k * step) * p.H, v);
    if constexpr (kCut) {
      if (t + k * step == p.ntok - 1) {
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
          const int q = e / V, l = e % V;
          if (map.in(q) && map.at(q) == (map.np - 1) * V && map.mine(q, l))
            v[e] = to_acc(p.in[i][(t + k * step) * p.H + map.at(q) + l - map.off]);
        }
      }
    }
  }
  template <int kRows>
  __device__ __forceinline__ void read() const {  // after a block barrier that follows the rows' loads
    if constexpr (kBulk)
      if ((threadIdx.x & 31) == 0 && t + p.stages * step < p.fetched)
#pragma unroll
        for (int k = 0; k < kRows; ++k)
          if (t + (k + p.stages) * step < p.fetched) fetch(t + (k + p.stages) * step, stage(k));
  }
  __device__ __forceinline__ void next(int rows = 1) {
    t += rows * step;
    if constexpr (kBulk)
      if ((st += rows) >= p.stages) {
        st -= p.stages;
        phase ^= 1;
      }
  }
};

constexpr size_t kBulkRoom = 200 * 1024;  // shared memory that an SM's blocks of a bulk form divide

// Cut rows' weights into shared memory, beside the packs of a row that begins at `off`: vector i at out + i * room.
template <int N, typename A>
__device__ __forceinline__ void move_weights(const A *const (&from)[5], int off, int H, int room, A *out) {
#pragma unroll 2
  for (int c = threadIdx.x; c < room; c += blockDim.x) {
    const bool in = (unsigned)(c - off) < (unsigned)H;
    A v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = in ? __ldg(from[i] + c - off) : A(0);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i * room + c] = v[i];
  }
}

// The block's threads fill n elements with NaN.
template <typename T>
__device__ __forceinline__ void fill_nan(T *to, int n) {
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += blockDim.x) to[i] = from_acc<T>(nan_of<acc_t<T>>());
}

// A block that gave up at its row `first` (RowFeed): waits once more for the rows in flight, fills this row and its later
// ones of a, b [ntok][H] and c [ntok][nc] (or NULL) with NaN, and is counted.  Out of line, and with nothing from the
// loop over the rows: what stays alive for it there costs registers (backward of 65,536 x 1600 bf16: 423 us against 396).
template <typename T, typename C>
__device__ __noinline__ void leave_rows(uint64_t *bars, int stages, unsigned first, int64_t fetched, int64_t ntok, int H,
                                        T *a, T *b, C *c, int nc) {
  const unsigned step = gridDim.x, at = (first - blockIdx.x) / step;
  if (threadIdx.x == 0) {
    atomicAdd(&g_wait_timeouts, 1u);
    for (unsigned i = at; i < at + stages && blockIdx.x + (int64_t)i * step < fetched; ++i)
      bounded_wait((uint32_t)__cvta_generic_to_shared(bars + i % stages), i / stages & 1, [] { return false; });
  }
  for (int64_t t = first; t < ntok; t += step) {
    fill_nan(a + t * H, H);
    fill_nan(b + t * H, H);
    if (c) fill_nan(c + t * nc, nc);
  }
  __syncthreads();  // nobody's copies into shared memory outlive the block, nobody's stores follow these
}

// Rows a block of the forward works on at once: two of 16-bit elements by bulk copies (the waits of their block sums
// overlap, and the weights are read once for both: layer norm of 65,536 x 1600 bf16 in 248 us against 277), else one.
template <typename T, bool kBulk, int kThreads>
constexpr int kFwdRows = kBulk && sizeof(T) == 2 && kThreads <= 512 ? 2 : 1;

template <typename T, int V, int EPT, bool kWarpRow, Feed kFeed, bool kLayer, int kThreads, int kMinBlocks>
__global__ void __launch_bounds__(kThreads, kMinBlocks) norm_fwd_kernel(const NormArgs<T> p) {
  using A = acc_t<T>;
  constexpr bool kBulk = kFeed != kPlain, kCut = kFeed == kCutRows;
  constexpr int R = kFwdRows<T, kBulk, kThreads>;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ uint64_t bars[kMaxStages];
  __shared__ unsigned lost;
  __shared__ SumBuf<A, kThreads / 32> buf;
  int phase = 0;
  for (int i = threadIdx.x; i < (int)(sizeof buf / sizeof(A)); i += blockDim.x) (&buf.v[0][0][0])[i] = A(0);
  __syncthreads();
  const int off = kCut ? (int)((uint64_t)blockIdx.x * p.H % V) : 0;
  const RowMap<T, V, EPT, kCut> map{kWarpRow ? (int)(threadIdx.x & 31) : (int)threadIdx.x,
                                    kWarpRow ? 32 : (int)blockDim.x, kCut ? (off + p.H + V - 1) / V : p.H / V, off, p.H};
  RowFeed<T, V, EPT, kFeed> feed{
      p, map, kWarpRow ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : (int64_t)blockIdx.x,
      kWarpRow ? (int64_t)gridDim.x * (blockDim.x >> 5) : (int64_t)gridDim.x, smem, bars, &lost};
  const A inv = A(1) / A(p.H);
  feed.begin();
  const A *wa = p.a, *w1 = p.w1, *w2 = p.w2, *b1 = p.b1, *b2 = p.b2;
  if constexpr (kCut) {
    A *ws = reinterpret_cast<A *>(smem + p.stages * p.nin * feed.row_bytes());
    const int room = cut_bytes<T>(p.H) / sizeof(T);
    move_weights<kLayer ? 5 : 3, A>({p.a, p.w1, p.w2, p.b1, p.b2}, off, p.H, room, ws);
    wa = ws, w1 = ws + room, w2 = ws + 2 * room, b1 = ws + 3 * room, b2 = ws + 4 * room;
    __syncthreads();
  }
  T gate_next[R];
  auto peek = [&](int64_t t) {  // the next rows' gates
    if (p.gate)
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (t + k * feed.step < p.ntok) gate_next[k] = p.gate[t + k * feed.step];
  };
  peek(feed.t);
  for (; feed.t < p.ntok; feed.next(R)) {
    A f[R][EPT], r[R][EPT], g[R][EPT], w[EPT], b[EPT], gate[R], m1[R], s1[R], m2[R], s2[R];
    bool have[R], ok[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      have[k] = k == 0 || feed.t + k * feed.step < p.ntok;  // the last row alone: its place holds an older row
      gate[k] = p.gate && have[k] ? to_acc(gate_next[k]) : A(1);
    }
    peek(feed.t + R * feed.step);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      ok[k] = !have[k] || feed.arrived(k);
      const int at = have[k] ? k : 0;
      feed.load(0, f[k], at);
      feed.load(1, r[k], at);
      if (p.nin > 2) feed.load(2, g[k], at);
    }
    row_stats<R, EPT, kWarpRow, kLayer>(map, f, ok, inv, p.eps, m1, s1, buf, phase);
    if (feed.given_up(kLayer ? m1[0] + m1[R - 1] : s1[0] + s1[R - 1])) break;
    feed.template read<R>();
    map.template weights<kBulk>(w1, w);
    if constexpr (kLayer) map.template weights<kBulk>(b1, b);
#pragma unroll
    for (int k = 0; k < R; ++k) {
#pragma unroll
      for (int i = 0; i < EPT; ++i) f[k][i] = kLayer ? fma(f[k][i] * s1[k], w[i], b[i]) : f[k][i] * s1[k] * w[i];
      if (p.nin > 2) {
#pragma unroll
        for (int i = 0; i < EPT; ++i) f[k][i] *= g[k][i];
      } else if (p.gate) {
#pragma unroll
        for (int i = 0; i < EPT; ++i) f[k][i] *= gate[k];
      }
    }
    map.template weights<kBulk>(wa, w);
#pragma unroll
    for (int k = 0; k < R; ++k) {
#pragma unroll
      for (int i = 0; i < EPT; ++i) r[k][i] = fma(w[i], f[k][i], r[k][i]);
      if (have[k]) map.store(p.r2 + (feed.t + k * feed.step) * p.H, r[k]);
    }
    row_stats<R, EPT, kWarpRow, kLayer>(map, r, ok, inv, p.eps, m2, s2, buf, phase);
    map.template weights<kBulk>(w2, w);
    if constexpr (kLayer) map.template weights<kBulk>(b2, b);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t t = feed.t + k * feed.step;
#pragma unroll
      for (int i = 0; i < EPT; ++i) r[k][i] = kLayer ? fma(r[k][i] * s2[k], w[i], b[i]) : r[k][i] * s2[k] * w[i];
      if (!have[k]) continue;
      map.store(p.u + t * p.H, r[k]);
      if (map.first == 0) {
        A *st = p.stats + t * 4;
        st[0] = m1[k];
        st[1] = s1[k];
        st[2] = m2[k];
        st[3] = s2[k];
      }
    }
  }
  if constexpr (kBulk)
    if (lost != kNoRow) leave_rows<T>(bars, p.stages, lost, p.fetched, p.ntok, p.H, p.r2, p.u, p.stats, 4);
}

// The forward for 16-bit rows of 257 to 512 elements: a warp a row, the row's one array in registers (f, then p, then
// r2), r and the gate read from shared memory where they are used.  No block barriers, and a row costs a third of the
// instructions that it costs a block, whose sums' shuffles and barriers every warp repeats.  Each warp has two rows in
// shared memory, the next on its way while it works on one.  65,536 x 512 bf16 layer norm: 60 us against 78 by blocks;
// longer rows leave too few warps on an SM (1024 when it was tried: 161 against 140).
constexpr int kWarpStages = 2, kWarpEpt = 16;  // the stages' order below holds for two

// Warps a block: two for whole rows; cut rows share the block's weights, one block an SM.
template <Feed kFeed>
constexpr int kRowWarpsMost = kFeed == kBulkRows ? 2 : 16;
template <Feed kFeed>
constexpr int kRowBlocks = kFeed == kCutRows ? 1 : 10;

template <typename T, Feed kFeed, bool kLayer>
__global__ void __launch_bounds__(kRowWarpsMost<kFeed> * 32, kRowBlocks<kFeed>)
    norm_fwd_rows_kernel(const NormArgs<T> p) {
  using A = acc_t<T>;
  constexpr int EPT = kWarpEpt, V = 8 / (int)sizeof(T);  // neighbouring lanes read neighbouring 16 bytes of the weights
  constexpr bool kCut = kFeed == kCutRows;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ uint64_t bars[kRowWarpsMost<kFeed>][kWarpStages];
  __shared__ SumBuf<A, 4> unused;
  int phase = 0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, wpb = blockDim.x >> 5;
  const int64_t step = (int64_t)gridDim.x * wpb;
  // cut rows: a block's warps begin a multiple of eight rows apart (the grid is one), at the same place in a word
  int64_t t = kCut ? (int64_t)warp * gridDim.x + blockIdx.x : (int64_t)blockIdx.x * wpb + warp;
  const uint32_t place = kCut ? cut_bytes<T>(p.H) : (uint32_t)p.H * sizeof(T);
  const int off = kCut ? (int)((uint64_t)t * p.H % (16 / sizeof(T))) : 0;
  const RowMap<T, V, EPT, kCut> map{lane, 32, (off + p.H + V - 1) / V, off, p.H};
  unsigned char *mine = smem + (size_t)warp * kWarpStages * p.nin * place;
  const A inv = A(1) / A(p.H);
  auto bar = [&](int s) { return (uint32_t)__cvta_generic_to_shared(&bars[warp][s]); };
  auto fetch = [&](int64_t row, int s) {  // a lane an array
    if (row >= p.ntok || lane >= p.nin) return;
    // the last row's last word may reach past the array: what is left out here is read below
    const uint32_t bytes = !kCut ? place : row == p.ntok - 1 ? (uint32_t)(off + p.H) * sizeof(T) & ~15u : (uint32_t)((off + p.H) * sizeof(T) + 15) & ~15u;
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar(s)), "r"(bytes) : "memory");
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                     (uint32_t)__cvta_generic_to_shared(mine) + (s * p.nin + lane) * place),
                 "l"(p.in[lane] + row * p.H - off), "r"(bytes), "r"(bar(s))
                 : "memory");
  };
  if (lane == 0) {
    for (int s = 0; s < kWarpStages; ++s) asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar(s)), "r"(p.nin));
    asm volatile("fence.mbarrier_init.release.cluster;");
  }
  const A *wa = p.a, *w1 = p.w1, *w2 = p.w2, *b1 = p.b1, *b2 = p.b2;
  if constexpr (kCut) {
    A *ws = reinterpret_cast<A *>(smem + (size_t)wpb * kWarpStages * p.nin * place);
    const int room = place / sizeof(T);
    move_weights<kLayer ? 5 : 3, A>({p.a, p.w1, p.w2, p.b1, p.b2}, off, p.H, room, ws);
    wa = ws, w1 = wa + room, w2 = w1 + room, b1 = w2 + room, b2 = b1 + room;
  }
  __syncthreads();
  for (int s = 0; s < kWarpStages; ++s) fetch(t + s * step, s);
  T gate_next = p.gate && t < p.ntok ? p.gate[t] : T(0.0f);
  int st = 0, parity = 0;
  auto never = [] { return false; };
  for (; t < p.ntok; t += step) {
    const A gate = p.gate ? to_acc(gate_next) : A(1);
    if (p.gate && t + step < p.ntok) gate_next = p.gate[t + step];
    const bool ok[1] = {t < p.fetched && bounded_wait<kRowPolls>(bar(st), parity, never)};
    const unsigned char *row = mine + (size_t)st * p.nin * place;
    auto pack = [&](int array, int i, A (&x)[V]) {
      const Pack<T, V> q = load_pack<T, V>(reinterpret_cast<const T *>(row + array * place) + map.at(i));
      const bool late = kCut && t == p.ntok - 1 && (map.at(i) + V) * (int)sizeof(T) > (((off + p.H) * (int)sizeof(T)) & ~15);
#pragma unroll
      for (int l = 0; l < V; ++l) {
        x[l] = to_acc(q.v[l]);
        if (late && map.mine(i, l)) x[l] = to_acc(p.in[array][t * p.H + map.at(i) + l - off]);
      }
    };
    auto vec = [&](const A *w, int i, A (&x)[V]) {
      const Pack<A, V> q = load_pack<A, V>(w + map.at(i));
#pragma unroll
      for (int l = 0; l < V; ++l) x[l] = q.v[l];
    };
    A v[1][EPT], m1[1], s1[1], m2[1], s2[1], x[V];
#pragma unroll
    for (int i = 0; i < map.kN; ++i) {
      pack(0, i, x);
#pragma unroll
      for (int l = 0; l < V; ++l) v[0][i * V + l] = x[l];
    }
    row_stats<1, EPT, true, kLayer>(map, v, ok, inv, p.eps, m1, s1, unused, phase);
    if (s1[0] != s1[0] && __any_sync(0xffffffffu, !ok[0])) break;  // the warp gives up
#pragma unroll
    for (int i = 0; i < map.kN; ++i) {
      A w[V], b[V], r[V], a[V];
      vec(w1, i, w);
      if constexpr (kLayer) vec(b1, i, b);
      vec(wa, i, a);
      pack(1, i, r);
      if (p.nin > 2) {
        pack(2, i, x);
      } else {
#pragma unroll
        for (int l = 0; l < V; ++l) x[l] = gate;
      }
#pragma unroll
      for (int l = 0; l < V; ++l) {
        const A n = v[0][i * V + l] * s1[0], q = kLayer ? fma(n, w[l], b[l]) : n * w[l];
        v[0][i * V + l] = fma(a[l], q * x[l], r[l]);
      }
    }
    __syncwarp();  // the row has been read
    fetch(t + kWarpStages * step, st);
    if (++st == kWarpStages) {
      st = 0;
      parity ^= 1;
    }
    map.store(p.r2 + t * p.H, v[0]);
    row_stats<1, EPT, true, kLayer>(map, v, ok, inv, p.eps, m2, s2, unused, phase);
#pragma unroll
    for (int i = 0; i < map.kN; ++i) {
      A w[V], b[V];
      vec(w2, i, w);
      if constexpr (kLayer) vec(b2, i, b);
#pragma unroll
      for (int l = 0; l < V; ++l) {
        const A n = v[0][i * V + l] * s2[0];
        v[0][i * V + l] = kLayer ? fma(n, w[l], b[l]) : n * w[l];
      }
    }
    map.store(p.u + t * p.H, v[0]);
    if (lane == 0) {
      A *out = p.stats + t * 4;
      out[0] = m1[0], out[1] = s1[0], out[2] = m2[0], out[3] = s2[0];
    }
  }
  if (t < p.ntok) {  // given up: once what is in flight has landed, NaN into this row and its later ones
    if (lane == 0) atomicAdd(&g_wait_timeouts, 1u);
    bounded_wait(bar(st), parity, never);
    if (t + step < p.ntok) bounded_wait(bar(st ^ 1), parity ^ st, never);
    A none[EPT];
#pragma unroll
    for (int i = 0; i < EPT; ++i) none[i] = nan_of<A>();
    for (; t < p.ntok; t += step) {
      map.store(p.r2 + t * p.H, none);
      map.store(p.u + t * p.H, none);
      if (lane < 4) p.stats[t * 4 + lane] = none[0];
    }
  }
}

// A thread keeps its columns' sums over the rows of its block (or warp) in registers.
template <typename T, int V, int EPT, bool kWarpRow, Feed kFeed, bool kLayer, int kThreads, int kMinBlocks>
__global__ void __launch_bounds__(kThreads, kMinBlocks) norm_grad_kernel(const NormArgs<T> p) {
  using A = acc_t<T>;
  constexpr bool kBulk = kFeed != kPlain, kCut = kFeed == kCutRows;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ uint64_t bars[kMaxStages];
  __shared__ unsigned lost;
  __shared__ SumBuf<A, kThreads / 32> buf;
  int phase = 0;
  for (int i = threadIdx.x; i < (int)(sizeof buf / sizeof(A)); i += blockDim.x) (&buf.v[0][0][0])[i] = A(0);
  __syncthreads();
  const int off = kCut ? (int)((uint64_t)blockIdx.x * p.H % V) : 0;
  const RowMap<T, V, EPT, kCut> map{kWarpRow ? (int)(threadIdx.x & 31) : (int)threadIdx.x,
                                    kWarpRow ? 32 : (int)blockDim.x, kCut ? (off + p.H + V - 1) / V : p.H / V, off, p.H};
  RowFeed<T, V, EPT, kFeed> feed{
      p, map, kWarpRow ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : (int64_t)blockIdx.x,
      kWarpRow ? (int64_t)gridDim.x * (blockDim.x >> 5) : (int64_t)gridDim.x, smem, bars, &lost};
  A sa[EPT], sw1[EPT], sw2[EPT], sb1[EPT], sb2[EPT];
#pragma unroll
  for (int i = 0; i < EPT; ++i) sa[i] = sw1[i] = sw2[i] = sb1[i] = sb2[i] = A(0);
  const A inv = A(1) / A(p.H);
  feed.begin();
  const A *wa = p.a, *w1 = p.w1, *w2 = p.w2, *b1 = p.b1;
  if constexpr (kCut) {
    A *ws = reinterpret_cast<A *>(smem + p.stages * p.nin * feed.row_bytes());
    const int room = cut_bytes<T>(p.H) / sizeof(T);
    move_weights<kLayer ? 4 : 3, A>({p.a, p.w1, p.w2, p.b1, nullptr}, off, p.H, room, ws);
    wa = ws, w1 = ws + room, w2 = ws + 2 * room, b1 = ws + 3 * room;
    __syncthreads();
  }
  const bool each = p.nin > 4;  // a gate value for each element
  A st_next[4] = {};
  T gate_next = T(0.0f);
  auto peek = [&](int64_t t) {  // the next row's few numbers
    if (t >= p.ntok) return;
    if (p.gate) gate_next = p.gate[t];
#pragma unroll
    for (int i = 0; i < 4; ++i) st_next[i] = __ldg(p.stats + t * 4 + i);
  };
  peek(feed.t);
  for (; feed.t < p.ntok; feed.next()) {
    const int64_t t = feed.t;
    const A m1 = st_next[0], s1 = st_next[1], m2 = st_next[2], s2 = st_next[3], gt = p.gate ? to_acc(gate_next) : A(1);
    peek(t + feed.step);
    const bool ok = feed.arrived();
    A f[EPT], n2[EPT], du[EPT], dr[EPT], g[EPT], w[EPT];
    feed.load(0, n2);
    feed.load(1, du);
    feed.load(2, dr);
    feed.load(3, f);
    if (each) feed.load(4, g);
    else
#pragma unroll
      for (int i = 0; i < EPT; ++i) g[i] = gt;
    map.template weights<kBulk>(w2, w);
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      n2[i] = (n2[i] - m2) * s2;
      f[i] = (f[i] - m1) * s1;
      sw2[i] = fma(du[i], n2[i], sw2[i]);
      if constexpr (kLayer) sb2[i] += du[i];
      du[i] *= w[i];
    }
    constexpr int kOne = kLayer ? 2 : 1;
    A one[kOne];
    one[0] = ok ? map.total([&](int i) { return du[i] * n2[i]; }) : nan_of<A>();
    if constexpr (kLayer) one[1] = map.total([&](int i) { return du[i]; });
    row_sum<kOne, kWarpRow>(one, buf, phase);
    if (feed.given_up(one[0])) break;
    feed.template read<1>();
    A along = one[0] * inv, mean = kLayer ? one[kOne - 1] * inv : A(0);
#pragma unroll
    for (int i = 0; i < EPT; ++i) dr[i] = fma(s2, du[i] - (kLayer ? fma(n2[i], along, mean) : n2[i] * along), dr[i]);
    map.store(p.dr + t * p.H, dr);
    map.template weights<kBulk>(w1, w);
    if constexpr (kLayer) map.template weights<kBulk>(b1, n2);
#pragma unroll
    for (int i = 0; i < EPT; ++i) {  // du: p from here on
      du[i] = kLayer ? fma(f[i], w[i], n2[i]) : f[i] * w[i];
      sa[i] = fma(dr[i] * g[i], du[i], sa[i]);
    }
    map.template weights<kBulk>(wa, n2);
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      const A dra = dr[i] * n2[i], dp = dra * g[i];
      sw1[i] = fma(dp, f[i], sw1[i]);
      if constexpr (kLayer) sb1[i] += dp;
      g[i] = dra * du[i];  // dG
      dr[i] = dp * w[i];
    }
    A sums[3];
    sums[0] = map.total([&](int i) { return dr[i] * f[i]; });
    sums[1] = kLayer ? map.total([&](int i) { return dr[i]; }) : A(0);
    sums[2] = p.gate ? map.total([&](int i) { return g[i]; }) : A(0);
    if (kLayer || p.gate) {
      row_sum<3, kWarpRow>(sums, buf, phase);
    } else {
      A two[1] = {sums[0]};
      row_sum<1, kWarpRow>(two, buf, phase);
      sums[0] = two[0];
    }
    along = sums[0] * inv, mean = kLayer ? sums[1] * inv : A(0);
    if (p.dgate) {
      if (each) map.store(p.dgate + t * p.H, g);
      else if (map.first == 0) p.dgate[t] = from_acc<T>(sums[2]);
    }
#pragma unroll
    for (int i = 0; i < EPT; ++i) dr[i] = s1 * (dr[i] - (kLayer ? fma(f[i], along, mean) : f[i] * along));
    map.store(p.df + t * p.H, dr);
  }
  constexpr int kVec = kLayer ? 5 : 3;
  A *out = p.part + (int64_t)blockIdx.x * kNormVectors * p.H;
  if constexpr (kWarpRow) {  // the block's warps hold the same columns: one partial for the block
    A *all = reinterpret_cast<A *>(smem), *mine = all + (threadIdx.x >> 5) * kVec * p.H;
#pragma unroll
    for (int i = 0; i < EPT; ++i)
      if (map.in(i / V) && map.mine(i / V, i % V)) {
        A *o = mine + map.at(i / V) + i % V - off;
        o[0] = sa[i], o[p.H] = sw1[i], o[2 * p.H] = sw2[i];
        if constexpr (kLayer) o[3 * p.H] = sb1[i], o[4 * p.H] = sb2[i];
      }
    __syncthreads();
    for (int i = threadIdx.x; i < kVec * p.H; i += blockDim.x) {
      A v = all[i];
      for (int k = 1; k < (int)(blockDim.x >> 5); ++k) v += all[k * kVec * p.H + i];
      out[i] = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPT; ++i)
      if (map.in(i / V) && map.mine(i / V, i % V)) {
        A *o = out + map.at(i / V) + i % V - off;
        o[0] = sa[i], o[p.H] = sw1[i], o[2 * p.H] = sw2[i];
        if constexpr (kLayer) o[3 * p.H] = sb1[i], o[4 * p.H] = sb2[i];
      }
    if constexpr (kBulk)
      if (lost != kNoRow) {
        leave_rows<T>(bars, p.stages, lost, p.fetched, p.ntok, p.H, p.dr, p.df, p.dgate, each ? p.H : 1);
        fill_nan(out, kVec * p.H);
      }
  }
}

// Column sums of the blocks' partials: a block per 32 columns of one vector, 32 rows of threads, fixed order.
template <typename A>
__global__ void __launch_bounds__(1024) norm_finish_kernel(const A *__restrict__ part, int blocks, int H, A *da, A *dw1,
                                                           A *dw2, A *db1, A *db2) {
  __shared__ A s[32][33];
  A *const outs[kNormVectors] = {da, dw1, dw2, db1, db2};
  A *out = outs[blockIdx.y];
  const int lane = threadIdx.x & 31, row = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  A v = A(0);
  for (int k0 = row; k0 < blocks; k0 += 32 * 10) {  // ten partials on their way at a time
    A x[10];
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const int k = k0 + 32 * i;
      x[i] = c < H && k < blocks ? __ldg(part + ((int64_t)k * kNormVectors + blockIdx.y) * H + c) : A(0);
    }
#pragma unroll
    for (int i = 0; i < 10; ++i) v += x[i];
  }
  s[row][lane] = v;
  __syncthreads();
  v = s[lane][row];  // a warp a column
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lane == 0 && blockIdx.x * 32 + row < H) out[blockIdx.x * 32 + row] = v;
}

constexpr int kRowWarps = 4;      // rows (warps) per block where a warp holds a row,
constexpr int kWarpRowMax = 256;  // which is up to this length

// Launch shape, by the row length alone: a warp per row up to 256 elements, else a block with 8 elements a thread (16
// past 8192).  The blocks that an SM's registers hold (64 a thread forward, 128 backward) stay and take rows in turn.
struct NormShape {
  int ept, threads, blocks;  // elements a thread, threads a block, blocks an SM
};
inline NormShape norm_shape(int H, bool grad) {
  if (H <= kWarpRowMax) return {8, kRowWarps * 32, grad ? 3 : 8};
  const int ept = H <= 8192 ? 8 : 16, threads = (H + ept * 32 - 1) / (ept * 32) * 32;
  const int blocks = (grad ? 512 : 1024) / threads;
  return {ept, threads, blocks < 1 ? 1 : blocks};
}

// Two rows at once (kFwdRows) take 80 registers a thread: six warps of a scheduler's 16,384, 768 threads an SM.  Held to
// 72 they leave room for seven, 896.  What that costs each warp pays where a fourth block comes to three, not where the
// blocks were more already (us at 80 and 72, layer norm of 105 M bf16 elements: rows of 600 272, 292; 1000 224, 231; 1200
// 240, 254; 1400 239, 254; 1600 264, 248; 1792 237, 228).
constexpr int kTwoHeld = 768, kTightHeld = 896, kTightThreads = kTightHeld / 4;

// Rows whose bytes and addresses are multiples of 16 come by bulk copies, as many rows ahead as fit; so do rows of other
// lengths up to 2048 in arrays that begin at a multiple of 16 (cut rows); the rest by plain loads, element by
// element unless their packs are whole.
template <typename T, bool kGrad, bool kLayer>
int launch(NormArgs<T> &p, int v, bool weights16, bool bases16, cudaStream_t st, const char *who) {
  using std::integral_constant;
  using no = std::false_type;
  using yes = std::true_type;
  const NormShape n = norm_shape(p.H, kGrad);
  int rc = DP_OK;
  auto go = [&](auto V, auto E, auto W, auto B, auto M, auto N) {
    constexpr int v_ = decltype(V)::value, e_ = decltype(E)::value, m_ = decltype(M)::value, n_ = decltype(N)::value;
    constexpr bool w_ = decltype(W)::value, b_ = decltype(B)::value != kPlain;
    constexpr Feed f_ = decltype(B)::value;
    void (*k)(const NormArgs<T>);
    if constexpr (kGrad) k = norm_grad_kernel<T, v_, e_, w_, f_, kLayer, m_, n_>;
    else k = norm_fwd_kernel<T, v_, e_, w_, f_, kLayer, m_, n_>;
    constexpr bool two = !kGrad && kFwdRows<T, b_, m_> == 2;
    int blocks = two ? std::max(1, (m_ == kTightThreads ? kTightHeld : kTwoHeld) / n.threads) : n.blocks;
    size_t smem = kGrad && w_ ? (size_t)kRowWarps * kNormVectors * p.H * sizeof(acc_t<T>) : 0;
    if (b_) {
      const size_t row = (size_t)p.nin * (f_ == kCutRows ? cut_bytes<T>(p.H) : p.H * sizeof(T));
      const size_t weights = f_ == kCutRows ? cut_bytes<T>(p.H) / sizeof(T) * kNormVectors * sizeof(acc_t<T>) : 0;
      for (;; --blocks) {  // fewer blocks an SM where their rows would not fit
        const int64_t room = (int64_t)kBulkRoom / blocks - (int64_t)weights;
        p.stages = room < 0 ? 0 : room / (int64_t)row > kMaxStages ? kMaxStages : (int)(room / (int64_t)row);
        if (two) p.stages &= ~1;  // pairs of rows keep to pairs of stages
        if (p.stages > 0 || blocks == 1) break;
      }
      smem = row * p.stages + weights;
    }
    constexpr size_t kMost = b_ ? kBulkRoom : (size_t)kRowWarps * kNormVectors * kWarpRowMax * sizeof(acc_t<T>);
    if (smem > 32 * 1024) rc = allow_smem((const void *)k, kMost, who);  // the static part counts too
    const int64_t units = w_ ? (p.ntok + kRowWarps - 1) / kRowWarps : p.ntok, most = 152 * (kGrad ? n.blocks : blocks);
    if (!rc) k<<<(unsigned)(kGrad || units > most ? most : units), n.threads, smem, st>>>(p);
  };
  if constexpr (!kGrad && sizeof(T) == 2) {
    const bool whole = v == 8 && weights16, cut = v < 8 && bases16;
    const int need = p.H + (cut ? 10 : 0);  // places for the packs of a row that begins inside a word
    auto rows = [&](auto F) {
      constexpr Feed f_ = decltype(F)::value;
      const size_t place = f_ == kCutRows ? cut_bytes<T>(p.H) : (size_t)p.H * sizeof(T), row = kWarpStages * p.nin * place;
      const size_t weights = f_ == kCutRows ? place / sizeof(T) * (kLayer ? 5 : 3) * sizeof(acc_t<T>) : 0;
      const int fit = (int)((kBulkRoom - weights) / row), warps = fit < kRowWarpsMost<f_> ? fit : kRowWarpsMost<f_>;
      const int64_t held = f_ == kCutRows ? 1 : fit / 2 < kRowBlocks<f_> ? fit / 2 : kRowBlocks<f_>;
      const int64_t units = f_ == kCutRows ? 152 : (p.ntok + warps - 1) / warps, most = 152 * held;
      const size_t smem = row * warps + weights;
      auto k = norm_fwd_rows_kernel<T, f_, kLayer>;
      rc = allow_smem((const void *)k, kBulkRoom, who);
      if (!rc) k<<<(unsigned)(units > most ? most : units), warps * 32, smem, st>>>(p);
      return rc;
    };
    if (p.H > kWarpRowMax && need <= 32 * kWarpEpt) {
      if (whole) return rows(integral_constant<Feed, kBulkRows>{});
      if (cut) return rows(integral_constant<Feed, kCutRows>{});
    }
  }
  auto shape = [&](auto V) {
    constexpr integral_constant<int, 8> e8{};
    constexpr int kFew = kGrad ? 2 : 4, kHalf = kGrad ? 1 : 2;
    constexpr integral_constant<Feed, kPlain> plain{};
    constexpr integral_constant<Feed, kBulkRows> bulk{};
    if (p.H <= kWarpRowMax)
      return go(V, e8, yes{}, plain, integral_constant<int, kRowWarps * 32>{}, integral_constant<int, kGrad ? 3 : 8>{});
    if constexpr (decltype(V)::value * sizeof(T) == 16) {
      if (weights16 && (size_t)p.nin * p.H * sizeof(T) * n.blocks <= kBulkRoom) {
        constexpr int kTwo = !kGrad && sizeof(T) == 2 ? 3 : kFew, kTwoHalf = !kGrad && sizeof(T) == 2 ? 1 : kHalf;
        if constexpr (!kGrad && sizeof(T) == 2)
          if (kTwoHeld / n.threads == 3 && kTightHeld / n.threads == 4)
            return go(V, e8, no{}, bulk, integral_constant<int, kTightThreads>{}, integral_constant<int, 4>{});
        if (p.H <= 2048) return go(V, e8, no{}, bulk, integral_constant<int, 256>{}, integral_constant<int, kTwo>{});
        if (p.H <= 4096) return go(V, e8, no{}, bulk, integral_constant<int, 512>{}, integral_constant<int, kTwoHalf>{});
        if (p.H <= 8192) return go(V, e8, no{}, bulk, integral_constant<int, 1024>{}, integral_constant<int, 1>{});
      }
    }
    if constexpr (sizeof(T) < 8) {  // apart from the next, which depends on V: or f64's cut form would be compiled too
      if constexpr (decltype(V)::value * sizeof(T) != 16) {
        constexpr int kTwo = !kGrad && sizeof(T) == 2 ? 3 : kFew;
        // A block sets its weights up first, which pays from some 8 rows on, in the backward of 16-bit rows 20 (us, plain
        // and cut, rows of 1003: backward f16 5,000 35, 43; 9,973 63, 66; 20,000 111, 103; f32 5,000 42, 43).
        constexpr int kPays = kGrad && sizeof(T) == 2 ? 20 : 8;
        const bool places = cut_bytes<T>(p.H) / sizeof(T) <= (size_t)n.threads * 8;  // one for every pack
        if (bases16 && p.H <= 2048 && p.ntok >= (int64_t)152 * kPays * n.blocks && places)
          return go(integral_constant<int, 16 / (int)sizeof(T)>{}, e8, no{}, integral_constant<Feed, kCutRows>{},
                    integral_constant<int, 256>{}, integral_constant<int, kTwo>{});
      }
    }
    if (p.H <= 2048) return go(V, e8, no{}, plain, integral_constant<int, 256>{}, integral_constant<int, kFew>{});
    if (p.H <= 4096) return go(V, e8, no{}, plain, integral_constant<int, 512>{}, integral_constant<int, kHalf>{});
    if (p.H <= 8192) return go(V, e8, no{}, plain, integral_constant<int, 1024>{}, integral_constant<int, 1>{});
    go(V, integral_constant<int, 16>{}, no{}, plain, integral_constant<int, 1024>{}, integral_constant<int, 1>{});
  };
  constexpr int kFull = 16 / (int)sizeof(T);
  if (v == kFull) shape(integral_constant<int, kFull>{});
  else shape(integral_constant<int, 1>{});
  return rc;
}

template <typename... P>
bool aligned16(P... ptrs) {
  return (((uintptr_t)ptrs | ...) & 15) == 0;
}

inline int norm_check(int64_t ntok, int H, int kind, int gate_kind, const char *who) {
  if (ntok < 0 || ntok > 0x7fffffffLL) return set_error(DP_ERR_SHAPE, "%s: ntok = %lld", who, (long long)ntok);
  if (H < 1) return set_error(DP_ERR_SHAPE, "%s: row length %d", who, H);
  if (H > kNormMaxH) return set_error(DP_ERR_UNSUPPORTED, "%s: row length %d > %d", who, H, kNormMaxH);
  if (kind != DP_NORM_RMS && kind != DP_NORM_LAYER) return set_error(DP_ERR_SHAPE, "%s: kind = %d", who, kind);
  if (gate_kind < DP_GATE_NONE || gate_kind > DP_GATE_FULL)
    return set_error(DP_ERR_SHAPE, "%s: gate_kind = %d", who, gate_kind);
  return DP_OK;
}


}  // namespace
}  // namespace dpc
