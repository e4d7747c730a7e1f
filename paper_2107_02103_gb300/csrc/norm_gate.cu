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
// A row lives in the registers of one warp (H <= 256) or one block, so each array is moved once; the layer
// norm's variance is taken around the mean in a second sweep of the registers.
#include "rows.cuh"

namespace dpc {
namespace {

constexpr int kNormMaxH = 16384;
constexpr int kNormVectors = 5;  // da, dw1, dw2, db1, db2

// Sums of NV values over the row's threads (a warp, or the block through `buf`), the same bits in every thread.
template <int NV, bool kWarpRow, typename A>
__device__ __forceinline__ void row_sum(A (&v)[NV], A *buf, int &phase) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if constexpr (!kWarpRow) {
    const int warp = threadIdx.x >> 5, nwarp = blockDim.x >> 5;
    A *b = buf + phase * (32 * 3);  // alternate halves: one barrier per sum
    phase ^= 1;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
      for (int i = 0; i < NV; ++i) b[warp * 3 + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = b[i];
    for (int w = 1; w < nwarp; ++w)
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] += b[w * 3 + i];
  }
}

template <typename A>
__device__ __forceinline__ A inv_sqrt(A x) {
  if constexpr (sizeof(A) == 8) return 1.0 / sqrt(x);
  else return rsqrtf(x);
}

// Mean and inverse deviation of a row held as v[EPT] per thread (0 past the row's end, in[] says which).
template <int EPT, bool kWarpRow, typename A>
__device__ __forceinline__ void row_stats(const A (&v)[EPT], int have, int H, bool layer, A eps, A &m, A &s, A *buf,
                                          int &phase) {
  A sum[1];
  m = A(0);
  if (layer) {
    sum[0] = A(0);
#pragma unroll
    for (int i = 0; i < EPT; ++i) sum[0] += v[i];
    row_sum<1, kWarpRow>(sum, buf, phase);
    m = sum[0] / A(H);
  }
  sum[0] = A(0);
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    const A d = i < have ? v[i] - m : A(0);
    sum[0] = fma(d, d, sum[0]);
  }
  row_sum<1, kWarpRow>(sum, buf, phase);
  s = inv_sqrt(sum[0] / A(H) + eps);
}

// A thread's elements of a row: packs threadIdx + i * threads, i < EPT / V.
template <typename T, int V, int EPT>
struct RowMap {
  int first, step, np;  // first pack, stride between packs, packs in the row
  template <typename S, typename A>
  __device__ __forceinline__ void load(const S *row, A (&v)[EPT]) const {
#pragma unroll
    for (int i = 0; i < EPT / V; ++i) {
      const int c = first + i * step;
      if (c < np) {
        const Pack<S, V> x = load_pack<S, V>(row + (int64_t)c * V);
#pragma unroll
        for (int l = 0; l < V; ++l) v[i * V + l] = to_acc(x.v[l]);
      } else {
#pragma unroll
        for (int l = 0; l < V; ++l) v[i * V + l] = A(0);
      }
    }
  }
  template <typename A>
  __device__ __forceinline__ void load_weights(const A *w, A (&v)[EPT]) const {  // f32 or f64, any alignment
#pragma unroll
    for (int i = 0; i < EPT / V; ++i)
#pragma unroll
      for (int l = 0; l < V; ++l) {
        const int c = first + i * step;
        v[i * V + l] = c < np && w ? __ldg(w + c * V + l) : A(0);
      }
  }
  template <typename A>
  __device__ __forceinline__ void store(T *row, const A (&v)[EPT]) const {
#pragma unroll
    for (int i = 0; i < EPT / V; ++i) {
      const int c = first + i * step;
      if (c < np) {
        Pack<T, V> x;
#pragma unroll
        for (int l = 0; l < V; ++l) x.v[l] = from_acc<T>(v[i * V + l]);
        store_pack<T, V>(row + (int64_t)c * V, x);
      }
    }
  }
  __device__ __forceinline__ int have() const {  // elements of this thread inside the row (whole packs)
    int n = 0;
#pragma unroll
    for (int i = 0; i < EPT / V; ++i) n += first + i * step < np ? V : 0;
    return n;
  }
};

template <typename T>
struct NormArgs {
  const T *r, *f, *gate;  // r: the residual stream (backward: r2)
  const acc_t<T> *a, *w1, *b1, *w2, *b2;
  int64_t ntok;
  int H, layer, gate_token;
  acc_t<T> eps;
  T *r2, *u;
  acc_t<T> *stats;  // [ntok][4]: m1, s1, m2, s2
  const T *dr2, *du;
  T *dr, *df, *dgate;
  acc_t<T> *part;  // [blocks or warps][5][H] partial column sums
};

template <typename T, int V, int EPT, bool kWarpRow, int kThreads>
__global__ void __launch_bounds__(kThreads) norm_fwd_kernel(const NormArgs<T> p) {
  using A = acc_t<T>;
  __shared__ A buf[2 * 32 * 3];
  int phase = 0;
  const int64_t t = kWarpRow ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  if (kWarpRow && t >= p.ntok) return;
  const RowMap<T, V, EPT> map{kWarpRow ? (int)(threadIdx.x & 31) : (int)threadIdx.x,
                              kWarpRow ? 32 : (int)blockDim.x, p.H / V};
  const int have = map.have();
  A f[EPT], r[EPT], w[EPT], m1, s1, m2, s2;
  map.load(p.f + t * p.H, f);
  map.load(p.r + t * p.H, r);
  row_stats<EPT, kWarpRow>(f, have, p.H, p.layer, p.eps, m1, s1, buf, phase);
  map.load_weights(p.w1, w);
#pragma unroll
  for (int i = 0; i < EPT; ++i) f[i] = (f[i] - m1) * s1 * w[i];
  if (p.b1) {
    map.load_weights(p.b1, w);
#pragma unroll
    for (int i = 0; i < EPT; ++i) f[i] += w[i];
  }
  if (p.gate) {
    if (p.gate_token) {
      const A g = to_acc(p.gate[t]);
#pragma unroll
      for (int i = 0; i < EPT; ++i) f[i] *= g;
    } else {
      map.load(p.gate + t * p.H, w);
#pragma unroll
      for (int i = 0; i < EPT; ++i) f[i] *= w[i];
    }
  }
  map.load_weights(p.a, w);
#pragma unroll
  for (int i = 0; i < EPT; ++i) r[i] = i < have ? fma(w[i], f[i], r[i]) : A(0);
  map.store(p.r2 + t * p.H, r);
  row_stats<EPT, kWarpRow>(r, have, p.H, p.layer, p.eps, m2, s2, buf, phase);
  map.load_weights(p.w2, w);
#pragma unroll
  for (int i = 0; i < EPT; ++i) r[i] = (r[i] - m2) * s2 * w[i];
  if (p.b2) {
    map.load_weights(p.b2, w);
#pragma unroll
    for (int i = 0; i < EPT; ++i) r[i] += w[i];
  }
  map.store(p.u + t * p.H, r);
  if (map.first == 0) {
    A *st = p.stats + t * 4;
    st[0] = m1;
    st[1] = s1;
    st[2] = m2;
    st[3] = s2;
  }
}

// Rows in turn over a fixed number of blocks (or warps): a thread keeps its columns' five sums in registers.
template <typename T, int V, int EPT, bool kWarpRow, int kThreads>
__global__ void __launch_bounds__(kThreads) norm_grad_kernel(const NormArgs<T> p) {
  using A = acc_t<T>;
  __shared__ A buf[2 * 32 * 3];
  int phase = 0;
  const int64_t unit = kWarpRow ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  const int64_t units = kWarpRow ? (int64_t)gridDim.x * (blockDim.x >> 5) : gridDim.x;
  const RowMap<T, V, EPT> map{kWarpRow ? (int)(threadIdx.x & 31) : (int)threadIdx.x,
                              kWarpRow ? 32 : (int)blockDim.x, p.H / V};
  A a[EPT], w1[EPT], b1[EPT], w2[EPT];
  map.load_weights(p.a, a);
  map.load_weights(p.w1, w1);
  map.load_weights(p.b1, b1);
  map.load_weights(p.w2, w2);
  A sa[EPT], sw1[EPT], sw2[EPT], sb1[EPT], sb2[EPT];
#pragma unroll
  for (int i = 0; i < EPT; ++i) sa[i] = sw1[i] = sw2[i] = sb1[i] = sb2[i] = A(0);
  const A inv = A(1) / A(p.H);
  const int have = map.have();
  for (int64_t t = unit; t < p.ntok; t += units) {
    const A *st = p.stats + t * 4;
    const A m1 = __ldg(st), s1 = __ldg(st + 1), m2 = __ldg(st + 2), s2 = __ldg(st + 3);
    A f[EPT], n2[EPT], du[EPT], dr[EPT], g[EPT];
    map.load(p.r + t * p.H, n2);
    map.load(p.du + t * p.H, du);
    map.load(p.dr2 + t * p.H, dr);
    map.load(p.f + t * p.H, f);
    if (p.gate && !p.gate_token) map.load(p.gate + t * p.H, g);
    else {
      const A gt = p.gate ? to_acc(p.gate[t]) : A(1);
#pragma unroll
      for (int i = 0; i < EPT; ++i) g[i] = gt;
    }
    A sums[3] = {A(0), A(0), A(0)};
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      n2[i] = i < have ? (n2[i] - m2) * s2 : A(0);
      f[i] = i < have ? (f[i] - m1) * s1 : A(0);
      sw2[i] = fma(du[i], n2[i], sw2[i]);
      sb2[i] += du[i];
      du[i] *= w2[i];
      sums[0] += du[i];
      sums[1] = fma(du[i], n2[i], sums[1]);
    }
    row_sum<3, kWarpRow>(sums, buf, phase);
    A mean = p.layer ? sums[0] * inv : A(0), along = sums[1] * inv;
#pragma unroll
    for (int i = 0; i < EPT; ++i) dr[i] = i < have ? fma(s2, du[i] - fma(n2[i], along, mean), dr[i]) : A(0);
    map.store(p.dr + t * p.H, dr);
    sums[0] = sums[1] = sums[2] = A(0);
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      const A pp = fma(f[i], w1[i], b1[i]);
      const A dra = dr[i] * a[i], dp = dra * g[i];
      sa[i] = fma(dr[i] * g[i], pp, sa[i]);
      sw1[i] = fma(dp, f[i], sw1[i]);
      sb1[i] += dp;
      g[i] = dra * pp;  // dG
      sums[2] += g[i];
      dr[i] = dp * w1[i];
      sums[0] += dr[i];
      sums[1] = fma(dr[i], f[i], sums[1]);
    }
    row_sum<3, kWarpRow>(sums, buf, phase);
    mean = p.layer ? sums[0] * inv : A(0), along = sums[1] * inv;
    if (p.dgate) {
      if (!p.gate_token) map.store(p.dgate + t * p.H, g);
      else if (map.first == 0) p.dgate[t] = from_acc<T>(sums[2]);
    }
#pragma unroll
    for (int i = 0; i < EPT; ++i) dr[i] = s1 * (dr[i] - fma(f[i], along, mean));
    map.store(p.df + t * p.H, dr);
  }
  A *out = p.part + unit * kNormVectors * p.H;
  const int nvec = p.layer ? kNormVectors : 3;
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    const int c = map.first + (i / V) * map.step;
    if (c < map.np) {
      A *o = out + c * V + i % V;
      o[0] = sa[i];
      o[p.H] = sw1[i];
      o[2 * p.H] = sw2[i];
      if (nvec == kNormVectors) {
        o[3 * p.H] = sb1[i];
        o[4 * p.H] = sb2[i];
      }
    }
  }
}

// Column sums of the units' partials: a block per 32 columns of one vector, eight rows of threads, fixed order.
template <typename A>
__global__ void __launch_bounds__(256) norm_finish_kernel(const A *__restrict__ part, int units, int H, A *da, A *dw1,
                                                          A *dw2, A *db1, A *db2) {
  __shared__ A s[8][33];
  A *const outs[kNormVectors] = {da, dw1, dw2, db1, db2};
  A *out = outs[blockIdx.y];
  const int lane = threadIdx.x & 31, row = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  A v = A(0);
  if (c < H)
    for (int k = row; k < units; k += 8) v += part[((int64_t)k * kNormVectors + blockIdx.y) * H + c];
  s[row][lane] = v;
  __syncthreads();
  if (row == 0 && c < H) {
    for (int k = 1; k < 8; ++k) v += s[k][lane];
    out[c] = v;
  }
}

constexpr int kRowWarps = 4;     // rows (warps) per block where a warp holds a row
constexpr int kGradUnits = 304;  // blocks of the backward (two per SM); four times that in warps for short rows

// Launch shape: a warp per row up to 256 elements, else a block with 8 (16 past 4096) elements a thread.
template <typename T, bool kGrad>
void launch(const NormArgs<T> &p, int v, cudaStream_t st) {
  auto go = [&](auto V, auto E, auto W, auto M) {
    constexpr int v_ = decltype(V)::value, e_ = decltype(E)::value, m_ = decltype(M)::value;
    constexpr bool w_ = decltype(W)::value;
    const int threads = w_ ? kRowWarps * 32 : (p.H + e_ * 32 - 1) / (e_ * 32) * 32;
    if constexpr (kGrad) {
      norm_grad_kernel<T, v_, e_, w_, m_><<<kGradUnits, threads, 0, st>>>(p);
    } else {
      const int64_t blocks = w_ ? (p.ntok + kRowWarps - 1) / kRowWarps : p.ntok;
      norm_fwd_kernel<T, v_, e_, w_, m_><<<(unsigned)blocks, threads, 0, st>>>(p);
    }
  };
  auto shape = [&](auto V) {
    using std::integral_constant;
    if (p.H <= 256) go(V, integral_constant<int, 8>{}, std::true_type{}, integral_constant<int, kRowWarps * 32>{});
    else if (p.H <= 4096) go(V, integral_constant<int, 8>{}, std::false_type{}, integral_constant<int, 512>{});
    else go(V, integral_constant<int, 16>{}, std::false_type{}, integral_constant<int, 1024>{});
  };
  if constexpr (sizeof(T) == 2)
    if (v == 8) return shape(std::integral_constant<int, 8>{});
  if constexpr (sizeof(T) <= 4)
    if (v == 4) return shape(std::integral_constant<int, 4>{});
  if (v == 2) return shape(std::integral_constant<int, 2>{});
  shape(std::integral_constant<int, 1>{});
}

int norm_check(int64_t ntok, int H, int kind, int gate_kind, const char *who) {
  if (ntok < 0 || ntok > 0x7fffffffLL) return set_error(DP_ERR_SHAPE, "%s: ntok = %lld", who, (long long)ntok);
  if (H < 1) return set_error(DP_ERR_SHAPE, "%s: row length %d", who, H);
  if (H > kNormMaxH) return set_error(DP_ERR_UNSUPPORTED, "%s: row length %d > %d", who, H, kNormMaxH);
  if (kind != DP_NORM_RMS && kind != DP_NORM_LAYER) return set_error(DP_ERR_SHAPE, "%s: kind = %d", who, kind);
  if (gate_kind < DP_GATE_NONE || gate_kind > DP_GATE_FULL)
    return set_error(DP_ERR_SHAPE, "%s: gate_kind = %d", who, gate_kind);
  return DP_OK;
}

template <typename T>
int norm_fwd(const T *r, const T *f, const T *gate, int gate_kind, const acc_t<T> *a, const acc_t<T> *w1,
             const acc_t<T> *b1, const acc_t<T> *w2, const acc_t<T> *b2, int64_t ntok, int H, int kind, double eps,
             T *r2, T *u, acc_t<T> *stats, void *stream, const char *who) {
  clear_error();
  const int rc = norm_check(ntok, H, kind, gate_kind, who);
  if (rc) return rc;
  if (!(eps > 0.0) || !std::isfinite(eps) || !((acc_t<T>)eps > acc_t<T>(0)))
    return set_error(DP_ERR_SHAPE, "%s: eps = %g must be positive", who, eps);
  if (ntok == 0) return DP_OK;
  if (!r || !f || !a || !w1 || !w2 || !r2 || !u || !stats || (gate_kind != DP_GATE_NONE && !gate) ||
      (kind == DP_NORM_LAYER && (!b1 || !b2)))
    return set_error(DP_ERR_NULL, "%s: NULL array", who);
  NormArgs<T> p{};
  p.r = r, p.f = f, p.gate = gate_kind == DP_GATE_NONE ? nullptr : gate;
  p.a = a, p.w1 = w1, p.w2 = w2;
  p.layer = kind == DP_NORM_LAYER;
  p.b1 = p.layer ? b1 : nullptr, p.b2 = p.layer ? b2 : nullptr;
  p.ntok = ntok, p.H = H, p.gate_token = gate_kind == DP_GATE_TOKEN, p.eps = (acc_t<T>)eps;
  p.r2 = r2, p.u = u, p.stats = stats;
  const int v = pack_width<T>(H, r, f, gate_kind == DP_GATE_FULL ? gate : nullptr, r2, u);
  if (!v) return set_error(DP_ERR_SHAPE, "%s: an array is not aligned to its elements", who);
  launch<T, false>(p, v, (cudaStream_t)stream);
  return launch_status(who);
}

int64_t grad_units(int H) { return H <= 256 ? (int64_t)kGradUnits * kRowWarps : kGradUnits; }

template <typename T>
int norm_grad(const T *r2, const T *f, const T *gate, int gate_kind, const acc_t<T> *a, const acc_t<T> *w1,
              const acc_t<T> *b1, const acc_t<T> *w2, const acc_t<T> *stats, const T *dr2, const T *du, int64_t ntok,
              int H, int kind, T *dr, T *df, T *dgate, acc_t<T> *da, acc_t<T> *dw1, acc_t<T> *dw2, acc_t<T> *db1,
              acc_t<T> *db2, void *work, size_t work_bytes, void *stream, const char *who) {
  clear_error();
  const int rc = norm_check(ntok, H, kind, gate_kind, who);
  if (rc) return rc;
  const bool layer = kind == DP_NORM_LAYER;
  if (!da || !dw1 || !dw2 || !a || !w1 || !w2 || (layer && (!b1 || !db1 || !db2)) || !work ||
      (ntok > 0 && (!r2 || !f || !stats || !dr2 || !du || !dr || !df)) ||
      (ntok > 0 && gate_kind != DP_GATE_NONE && (!gate || !dgate)))
    return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (work_bytes < (size_t)grad_units(H) * kNormVectors * H * sizeof(acc_t<T>) || ((uintptr_t)work & 15))
    return set_error(DP_ERR_SHAPE, "%s: work buffer of %zu bytes is too short or misaligned", who, work_bytes);
  NormArgs<T> p{};
  p.r = r2, p.f = f, p.gate = gate_kind == DP_GATE_NONE ? nullptr : gate;
  p.a = a, p.w1 = w1, p.w2 = w2, p.layer = layer, p.b1 = layer ? b1 : nullptr;
  p.ntok = ntok, p.H = H, p.gate_token = gate_kind == DP_GATE_TOKEN;
  p.stats = const_cast<acc_t<T> *>(stats), p.dr2 = dr2, p.du = du, p.dr = dr, p.df = df;
  p.dgate = gate_kind == DP_GATE_NONE ? nullptr : dgate;
  p.part = (acc_t<T> *)work;
  const bool full = gate_kind == DP_GATE_FULL;
  const int v = pack_width<T>(H, r2, f, full ? gate : nullptr, dr2, du, dr, df, full ? dgate : nullptr);
  if (!v) return set_error(DP_ERR_SHAPE, "%s: an array is not aligned to its elements", who);
  const cudaStream_t st = (cudaStream_t)stream;
  launch<T, true>(p, v, st);
  norm_finish_kernel<acc_t<T>><<<dim3((H + 31) / 32, layer ? kNormVectors : 3), 256, 0, st>>>(
      p.part, (int)grad_units(H), H, da, dw1, dw2, db1, db2);
  return launch_status(who);
}

}  // namespace
}  // namespace dpc

extern "C" {

size_t dp_norm_gate_work_bytes(int H, int elem_bytes) {
  if (H < 1 || H > dpc::kNormMaxH || (elem_bytes != 2 && elem_bytes != 4 && elem_bytes != 8)) return 0;
  return (size_t)dpc::grad_units(H) * dpc::kNormVectors * H * (elem_bytes == 8 ? 8 : 4);
}

#define DP_NORM(X, C, T, W)                                                                                            \
  int dp_norm_gate_fwd_##X(const C *r, const C *f, const C *gate, int gate_kind, const W *a, const W *w1, const W *b1, \
                           const W *w2, const W *b2, int64_t ntok, int H, int kind, double eps, C *r2, C *u, W *stats, \
                           void *stream) {                                                                             \
    return dpc::norm_fwd<T>((const T *)r, (const T *)f, (const T *)gate, gate_kind, a, w1, b1, w2, b2, ntok, H, kind,  \
                            eps, (T *)r2, (T *)u, stats, stream, "dp_norm_gate_fwd_" #X);                              \
  }                                                                                                                    \
  int dp_norm_gate_grad_##X(const C *r2, const C *f, const C *gate, int gate_kind, const W *a, const W *w1,            \
                            const W *b1, const W *w2, const W *stats, const C *dr2, const C *du, int64_t ntok, int H,  \
                            int kind, C *dr, C *df, C *dgate, W *da, W *dw1, W *dw2, W *db1, W *db2, void *work,       \
                            size_t work_bytes, void *stream) {                                                         \
    return dpc::norm_grad<T>((const T *)r2, (const T *)f, (const T *)gate, gate_kind, a, w1, b1, w2, stats,            \
                             (const T *)dr2, (const T *)du, ntok, H, kind, (T *)dr, (T *)df, (T *)dgate, da, dw1, dw2, \
                             db1, db2, work, work_bytes, stream, "dp_norm_gate_grad_" #X);                             \
  }
DP_NORM(f64, double, double, double)
DP_NORM(f32, float, float, float)
DP_NORM(bf16, uint16_t, __nv_bfloat16, float)
DP_NORM(f16, uint16_t, __half, float)

}  // extern "C"
