// Experts of each token from a router's logits, and the gradient of their weights.  For a row x of E logits and a bias b:
//   s = softmax(x) or sigmoid(x),  c = s + b
//   groups of E/G neighbours, each scored by the sum of its one or two largest c: the `keep` best stay
//   expert[j] = the j-th largest c left,  w_j = scale s_ej, or scale s_ej / sum_i s_ei
// Without a bias the experts are ordered by x itself, which has the order of s and no rounding.  Ties go to the lowest
// index, a NaN stands above all numbers, an expert with x = -inf or b = -inf is never chosen (-1, weight 0).
// The choice is that of exact arithmetic: c is computed in f32, and a token in which two neighbours of the order (the
// first one left out included) or the last group kept and the first one dropped are nearer than their error bounds is
// done again in f64.
// Backward, the choice held fixed, n_j = s_ej / sum_i s_ei:
//   renormalised  g_j = scale n_j (dw_j - sum_i n_i dw_i)   softmax dx_ej += g_j,  sigmoid dx_ej += g_j (1 - s_ej)
//   plain         softmax dx_e = sum_(j: e_j = e) g_j - s_e sum_j g_j with g_j = scale dw_j s_ej
//                 sigmoid dx_ej += scale dw_j s_ej (1 - s_ej)
#include <climits>

#include "rows.cuh"

namespace dpc {
namespace {

constexpr int kMaxExperts = 1024, kMaxTopk = 64;
constexpr int kThreads = 128;

struct TopkArgs {
  const void *x, *bias;
  int64_t ntok;
  int E, k, sigmoid, G, keep, gtop, renorm;
  double scale;
  int32_t *expert;
  void *w;
};

template <typename A>
struct KeyOf {
  using type = uint32_t;
};
template <>
struct KeyOf<double> {
  using type = unsigned long long;
};
template <typename A>
using key_t_ = typename KeyOf<A>::type;

// Numbers to integers of the same order; 0 is no candidate (-inf), all ones a NaN, and -0 is 0.
__device__ __forceinline__ uint32_t to_key(float c) {
  const uint32_t u = __float_as_uint(c + 0.0f);
  if (c != c) return 0xffffffffu;
  return u == 0xff800000u ? 0u : (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ unsigned long long to_key(double c) {
  const unsigned long long u = (unsigned long long)__double_as_longlong(c + 0.0);
  if (c != c) return ~0ull;
  return u == 0xfff0000000000000ull ? 0ull : (u >> 63) ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ float from_key(uint32_t k) {
  return __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k);  // all ones: a NaN
}
__device__ __forceinline__ double from_key(unsigned long long k) {
  return __longlong_as_double((long long)((k >> 63) ? k & 0x7fffffffffffffffull : ~k));
}

// Reductions over the L lanes of a token (mask: those lanes).
template <int L, typename V, typename F>
__device__ __forceinline__ V over(unsigned mask, V v, F f) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(mask, v, o));
  return v;
}
template <int L, typename V>
__device__ __forceinline__ V max_over(unsigned mask, V v) {
  if constexpr (L == 32 && std::is_same<V, uint32_t>::value) return __reduce_max_sync(mask, v);
  return over<L>(mask, v, [](V a, V b) { return a > b ? a : b; });
}
template <int L>
__device__ __forceinline__ int min_over(unsigned mask, int v) {
  if constexpr (L == 32) return __reduce_min_sync(mask, v);
  return over<L>(mask, v, [](int a, int b) { return a < b ? a : b; });
}
template <int L, typename V>
__device__ __forceinline__ V sum_over(unsigned mask, V v) {
  return over<L>(mask, v, [](V a, V b) { return a + b; });
}
// The largest of the lanes' values, NaN above all.
template <int L, typename A>
__device__ __forceinline__ A most_over(unsigned mask, A v) {
  return over<L>(mask, v, [](A a, A b) { return a != a || a > b ? a : b; });
}

__device__ __forceinline__ float exp_(float x) { return expf(x); }
__device__ __forceinline__ double exp_(double x) { return exp(x); }
template <typename A>
__device__ __forceinline__ A sigmoid(A x) {
  const A e = exp_(x < A(0) ? x : -x), r = A(1) / (A(1) + e);  // e <= 1
  return x < A(0) ? e * r : r;
}
template <typename A>
__device__ __forceinline__ A none() { return -A(INFINITY); }

// Scores of chosen logits up to a factor common to the row that keeps their sum from underflowing: for a softmax
// exp(x - m), for a sigmoid s exp(-m) with m = min(0, largest x).
template <typename A>
__device__ __forceinline__ A relative_score(A x, A most, bool sigm) {
  if (!sigm) return exp_(x - most);
  if (x >= A(0)) return A(1) / (A(1) + exp_(-x));
  return exp_(x - (most < A(0) ? most : A(0))) / (A(1) + exp_(x));
}

// One token on L lanes, N logits a lane: lane's i-th is expert i L + lane.  True: two scores are too near to tell apart
// in A, and nothing is written.  `room`: shared memory of the token, E + 2 G words of 8 bytes, for the groups.
template <typename T, typename A, int L, int N>
__device__ bool choose(const TopkArgs &p, int64_t t, int lane, unsigned mask, unsigned char *room) {
  using U = key_t_<A>;
  constexpr bool kExact = sizeof(A) == 8;
  constexpr int kSlots = (kMaxTopk < L * N ? kMaxTopk : L * N) / L;
  const T *x = (const T *)p.x + t * p.E;
  const acc_t<T> *bias = (const acc_t<T> *)p.bias;
  const bool grouped = p.keep < p.G, by_score = p.bias || (grouped && p.gtop == 2);
  A v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = i * L + lane < p.E ? (A)to_acc(x[i * L + lane]) : none<A>();
  A most = none<A>(), total = A(0);
  if (!p.sigmoid && (by_score || !p.renorm)) {
#pragma unroll
    for (int i = 0; i < N; ++i) most = v[i] != v[i] || v[i] > most ? v[i] : most;
    most = most_over<L>(mask, most);
#pragma unroll
    for (int i = 0; i < N; ++i) total += v[i] == none<A>() ? A(0) : exp_(v[i] - most);
    total = sum_over<L>(mask, total);
  }
  auto score = [&](A xe) { return p.sigmoid ? sigmoid(xe) : exp_(xe - most) / total; };

  U key[N];
  A *room_c = (A *)room;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * L + lane;
    A c = v[i], by = v[i];
    if (by_score && e < p.E) {
      const A b = bias ? (A)__ldg(bias + e) : A(0);
      const bool out = v[i] == none<A>() || b == none<A>();
      c = out ? none<A>() : score(v[i]) + b;
      by = bias ? c : v[i];
    }
    key[i] = to_key(by);
    if (grouped && e < p.E) room_c[e] = c;
  }
  bool near = false;
  if (grouped) {
    U *gkey = (U *)(room + (size_t)p.E * 8), *kept = (U *)(room + (size_t)(p.E + p.G) * 8);
    const int per = p.E / p.G;
    __syncwarp(mask);
    for (int g = lane; g < p.G; g += L) {
      U a = 0, b = 0;
      for (int i = 0; i < per; ++i) {
        const U c = to_key(room_c[g * per + i]);
        b = c > a ? a : c > b ? c : b;
        a = c > a ? c : a;
      }
      gkey[g] = p.gtop == 2 && b ? to_key(from_key(a) + from_key(b)) : a;
    }
    __syncwarp(mask);
    U last = ~(U)0, first = 0;  // the least group kept, the best one dropped
    for (int g = lane; g < p.G; g += L) {
      const U mine = gkey[g];
      int rank = 0;
      for (int o = 0; o < p.G; ++o) rank += gkey[o] > mine || (gkey[o] == mine && o < g);
      kept[g] = rank < p.keep;
      if (rank < p.keep) last = mine < last ? mine : last;
      else first = mine > first ? mine : first;
    }
    __syncwarp(mask);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = i * L + lane;
      if (e < p.E && !kept[e / per]) key[i] = 0;
    }
    if (!kExact && by_score) {
      last = ~max_over<L>(mask, (U)~last);
      first = max_over<L>(mask, first);
      const A a = from_key(last), b = from_key(first);
      // an s is within 2^-20 of its value (s <= 1: 2 ulp of the exponential, its argument's rounding, sum and quotient)
      near = first != 0 && !(a - b > A(0x1p-18) * (A(1) + fabs((double)b)));
    }
  }

  // the best of each lane, then of the token, k times and once more for the first one left out
  U best;
  int at;
  A bx;
  auto rescan = [&] {
    best = 0;
    at = 0;
    bx = A(0);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (key[i] > best) {
        best = key[i];
        at = i;
        bx = v[i];
      }
  };
  rescan();
  int se[kSlots];
  A sx[kSlots], sc[kSlots];
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    se[s] = -1;
    sx[s] = none<A>();
    sc[s] = none<A>();
  }
  const bool check = !kExact && p.bias;
  int left_e = -1;
  A left_x = A(0), left_c = none<A>();
  for (int j = 0; j < p.k + (check ? 1 : 0); ++j) {
    const U m = max_over<L>(mask, best);
    if (m == 0) break;
    const int e = min_over<L>(mask, best == m ? at * L + lane : INT_MAX);
    const A xe = __shfl_sync(mask, bx, e % L, L);
    if (e % L == lane) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i == at) key[i] = 0;
      rescan();
    }
    if (j == p.k) {
      left_e = e;
      left_x = xe;
      left_c = from_key(m);
    } else {
#pragma unroll
      for (int s = 0; s < kSlots; ++s)
        if (j == s * L + lane) {
          se[s] = e;
          sx[s] = xe;
          sc[s] = from_key(m);
        }
    }
  }
  if (check) {
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const int up = lane + 1 < L ? s : s + 1;  // whose next one is where
      int ne = __shfl_sync(mask, se[s], (lane + 1) % L, L);
      A nx = __shfl_sync(mask, sx[s], (lane + 1) % L, L), nc = __shfl_sync(mask, sc[s], (lane + 1) % L, L);
      const int s1 = s + 1 < kSlots ? s + 1 : s;
      const int ne1 = __shfl_sync(mask, se[s1], 0, L);
      const A nx1 = __shfl_sync(mask, sx[s1], 0, L), nc1 = __shfl_sync(mask, sc[s1], 0, L);
      if (up != s) {
        ne = ne1;
        nx = nx1;
        nc = nc1;
      }
      if (s * L + lane == p.k - 1) {
        ne = left_e;
        nx = left_x;
        nc = left_c;
      }
      if (s * L + lane < p.k && se[s] >= 0 && ne >= 0) {
        const A b0 = (A)__ldg(bias + se[s]), b1 = (A)__ldg(bias + ne);
        // s is off by less than 2^-21 of itself (2 ulp of the exponential, quotient, sum) and, in a softmax, by its
        // argument's rounding; s <= |c| + |b|
        A eps = A(0x1p-20);
        if (!p.sigmoid) eps += A(0x1p-23) * (most - (sx[s] < nx ? sx[s] : nx));
        const A tol = eps * (fabsf(sc[s]) + fabsf(nc) + fabsf(b0) + fabsf(b1));
        near |= !(sx[s] == nx && b0 == b1) && !(sc[s] - nc > tol);
      }
    }
  }
  if (!kExact && by_score && __any_sync(mask, near)) return true;

  A wsum = A(1), top = A(0);
  A ws[kSlots];
  if (p.renorm) {
    top = none<A>();
#pragma unroll
    for (int s = 0; s < kSlots; ++s) top = sx[s] != sx[s] || sx[s] > top ? sx[s] : top;
    top = most_over<L>(mask, top);
    wsum = A(0);
  }
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    ws[s] = se[s] < 0 ? A(0) : p.renorm ? relative_score(sx[s], top, p.sigmoid) : score(sx[s]);
    if (p.renorm) wsum += ws[s];
  }
  // total * 0: a NaN or +inf anywhere makes every score of a softmax NaN, also where the chosen logits are numbers
  if (p.renorm) wsum = sum_over<L>(mask, wsum) + (by_score ? total * A(0) : A(0));
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    const int j = s * L + lane;
    if (j < p.k) {
      p.expert[t * p.k + j] = se[s];
      ((acc_t<T> *)p.w)[t * p.k + j] = se[s] < 0 ? acc_t<T>(0) : (acc_t<T>)((A)p.scale * (ws[s] / wsum));
    }
  }
  return false;
}

template <typename T, int L, int N>
__device__ __noinline__ void choose_exact(const TopkArgs &p, int64_t t, int lane, unsigned mask, unsigned char *room) {
  choose<T, double, L, N>(p, t, lane, mask, room);
}

template <typename T, int L, int N>
__global__ void __launch_bounds__(kThreads) topk_kernel(const __grid_constant__ TopkArgs p) {
  extern __shared__ __align__(16) unsigned char rooms[];
  const int slot = threadIdx.x / L, lane = threadIdx.x % L;
  const int64_t t = (int64_t)blockIdx.x * (kThreads / L) + slot;
  if (t >= p.ntok) return;
  const unsigned mask = L == 32 ? 0xffffffffu : ((1u << (L % 32)) - 1) << (threadIdx.x % 32 / L * L);
  unsigned char *room = rooms + (size_t)slot * (p.E + 2 * p.G) * 8;
  if (choose<T, acc_t<T>, L, N>(p, t, lane, mask, room))
    if constexpr (sizeof(T) < 8) {
      __syncwarp(mask);
      choose_exact<T, L, N>(p, t, lane, mask, room);
    }
}

struct TopkGradArgs {
  const void *x;
  const int32_t *expert;
  const void *dw;
  int64_t ntok;
  int E, k, sigmoid, renorm;
  double scale;
  void *dx;
};

template <typename T, int L, int N>
__global__ void __launch_bounds__(kThreads) topk_grad_kernel(const __grid_constant__ TopkGradArgs p) {
  using A = acc_t<T>;
  constexpr int kSlots = (kMaxTopk < L * N ? kMaxTopk : L * N) / L;
  const int lane = threadIdx.x % L;
  const int64_t t = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  if (t >= p.ntok) return;
  const unsigned mask = L == 32 ? 0xffffffffu : ((1u << (L % 32)) - 1) << (threadIdx.x % 32 / L * L);
  const T *x = (const T *)p.x + t * p.E;
  const A scale = (A)p.scale;
  int e[kSlots];
  A xe[kSlots], g[kSlots];
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    const int j = s * L + lane;
    e[s] = j < p.k ? __ldg(p.expert + t * p.k + j) : -1;
    if ((unsigned)e[s] >= (unsigned)p.E) e[s] = -1;
    xe[s] = e[s] >= 0 ? to_acc(x[e[s]]) : none<A>();
    if (xe[s] == none<A>()) e[s] = -1;
    g[s] = e[s] >= 0 ? scale * __ldg((const A *)p.dw + t * p.k + j) : A(0);
  }
  A out[N];
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = A(0);
  if (p.renorm) {
    A top = none<A>();
#pragma unroll
    for (int s = 0; s < kSlots; ++s) top = xe[s] != xe[s] || xe[s] > top ? xe[s] : top;
    top = most_over<L>(mask, top);
    A n[kSlots], sum = A(0), mean = A(0);
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      n[s] = e[s] >= 0 ? relative_score(xe[s], top, p.sigmoid) : A(0);
      sum += n[s];
    }
    sum = sum_over<L>(mask, sum);
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      n[s] = e[s] >= 0 ? n[s] / sum : A(0);
      mean += n[s] * g[s];
    }
    mean = sum_over<L>(mask, mean);
#pragma unroll
    for (int s = 0; s < kSlots; ++s)
      if (e[s] >= 0) g[s] = n[s] * (g[s] - mean) * (p.sigmoid ? sigmoid(-xe[s]) : A(1));
  } else if (p.sigmoid) {
#pragma unroll
    for (int s = 0; s < kSlots; ++s)
      if (e[s] >= 0) g[s] *= sigmoid(xe[s]) * sigmoid(-xe[s]);
  } else {
    A most = none<A>(), total = A(0), sum = A(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      out[i] = i * L + lane < p.E ? to_acc(x[i * L + lane]) : none<A>();
      most = out[i] != out[i] || out[i] > most ? out[i] : most;
    }
    most = most_over<L>(mask, most);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      out[i] = out[i] == none<A>() ? A(0) : exp_(out[i] - most);
      total += out[i];
    }
    total = sum_over<L>(mask, total);
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      if (e[s] >= 0) g[s] *= exp_(xe[s] - most) / total;
      sum += g[s];
    }
    sum = sum_over<L>(mask, sum);
    const A f = total > A(0) || total != total ? sum / total : A(0);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = -out[i] * f;
  }
#pragma unroll
  for (int s = 0; s < kSlots; ++s)
    for (int l = 0; l < L && s * L + l < p.k; ++l) {
      const int ej = __shfl_sync(mask, e[s], l, L);
      const A gj = __shfl_sync(mask, g[s], l, L);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (ej == i * L + lane) out[i] += gj;
    }
  T *dx = (T *)p.dx + t * p.E;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i * L + lane < p.E) dx[i * L + lane] = from_acc<T>(out[i]);
}

int topk_check(int64_t ntok, int E, int k, int score, const char *who) {
  if (E < 1) return set_error(DP_ERR_SHAPE, "%s: nexp = %d", who, E);
  if (E > kMaxExperts) return set_error(DP_ERR_UNSUPPORTED, "%s: nexp = %d > %d", who, E, kMaxExperts);
  if (k < 1 || k > kMaxTopk || k > E) return set_error(DP_ERR_SHAPE, "%s: topk = %d of %d experts", who, k, E);
  if (ntok < 0 || ntok > 0x7fffffffLL / k)
    return set_error(DP_ERR_SHAPE, "%s: %lld tokens x %d experts", who, (long long)ntok, k);
  if (score != DP_SCORE_SOFTMAX && score != DP_SCORE_SIGMOID) return set_error(DP_ERR_SHAPE, "%s: score = %d", who, score);
  return DP_OK;
}

// Lanes a token and logits a lane.
template <typename F>
void with_shape(int E, F f) {
  if (E <= 32) f(std::integral_constant<int, 8>{}, std::integral_constant<int, 4>{});
  else if (E <= 128) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 8>{});
  else if (E <= 512) f(std::integral_constant<int, 32>{}, std::integral_constant<int, 16>{});
  else f(std::integral_constant<int, 32>{}, std::integral_constant<int, 32>{});
}

template <typename T>
int topk(const T *x, const acc_t<T> *bias, int64_t ntok, int E, int k, int score, int G, int keep, int gtop, int renorm,
         double scale, int32_t *expert, acc_t<T> *w, void *stream, const char *who) {
  clear_error();
  int rc = topk_check(ntok, E, k, score, who);
  if (rc) return rc;
  if (G < 1 || E % G) return set_error(DP_ERR_SHAPE, "%s: %d experts in %d groups", who, E, G);
  if (keep < 1 || keep > G || keep * (E / G) < k)
    return set_error(DP_ERR_SHAPE, "%s: %d experts of %d groups of %d", who, k, keep, E / G);
  if (gtop != 1 && gtop != 2) return set_error(DP_ERR_SHAPE, "%s: group_top = %d", who, gtop);
  if (!std::isfinite(scale)) return set_error(DP_ERR_SHAPE, "%s: scale = %g", who, scale);
  if (ntok == 0) return DP_OK;
  if (!x || !expert || !w) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (!at_elements(x, bias, w) || !at_elements(expert)) return misaligned(who);
  const TopkArgs p{x, bias, ntok, E, k, score == DP_SCORE_SIGMOID, G, keep, E / G == 1 ? 1 : gtop, renorm != 0, scale, expert, w};
  with_shape(E, [&](auto L_, auto N_) {
    constexpr int L = decltype(L_)::value, N = decltype(N_)::value, tok = kThreads / L;
    const size_t smem = keep < G ? (size_t)tok * (E + 2 * G) * 8 : 0;
    auto kernel = topk_kernel<T, L, N>;
    if (smem > 48 * 1024 && (rc = allow_smem((const void *)kernel, (size_t)kThreads * N * 3 * 8, who))) return;
    kernel<<<(unsigned)((ntok + tok - 1) / tok), kThreads, smem, (cudaStream_t)stream>>>(p);
  });
  return rc ? rc : launch_status(who);
}

template <typename T>
int topk_grad(const T *x, const int32_t *expert, const acc_t<T> *dw, int64_t ntok, int E, int k, int score, int renorm,
              double scale, T *dx, void *stream, const char *who) {
  clear_error();
  const int rc = topk_check(ntok, E, k, score, who);
  if (rc) return rc;
  if (!std::isfinite(scale)) return set_error(DP_ERR_SHAPE, "%s: scale = %g", who, scale);
  if (ntok == 0) return DP_OK;
  if (!x || !expert || !dw || !dx) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (!at_elements(x, dx) || !at_elements(expert) || !at_elements(dw)) return misaligned(who);
  const TopkGradArgs p{x, expert, dw, ntok, E, k, score == DP_SCORE_SIGMOID, renorm != 0, scale, dx};
  with_shape(E, [&](auto L_, auto N_) {
    constexpr int L = decltype(L_)::value, N = decltype(N_)::value, tok = kThreads / L;
    topk_grad_kernel<T, L, N><<<(unsigned)((ntok + tok - 1) / tok), kThreads, 0, (cudaStream_t)stream>>>(p);
  });
  return launch_status(who);
}

}  // namespace
}  // namespace dpc

extern "C" {

#define DP_TOPK(X, C, T, W)                                                                                          \
  int dp_route_topk_##X(const C *logits, const W *bias, int64_t ntok, int nexp, int topk, int score, int ngroup,     \
                        int keep_groups, int group_top, int renorm, double scale, int32_t *expert, W *w,             \
                        void *stream) {                                                                              \
    return dpc::topk<T>((const T *)logits, bias, ntok, nexp, topk, score, ngroup, keep_groups, group_top, renorm,    \
                        scale, expert, w, stream, "dp_route_topk_" #X);                                              \
  }                                                                                                                  \
  int dp_route_topk_grad_##X(const C *logits, const int32_t *expert, const W *dw, int64_t ntok, int nexp, int topk,  \
                             int score, int renorm, double scale, C *dlogits, void *stream) {                        \
    return dpc::topk_grad<T>((const T *)logits, expert, dw, ntok, nexp, topk, score, renorm, scale, (T *)dlogits,    \
                             stream, "dp_route_topk_grad_" #X);                                                      \
  }
DP_TOPK(f64, double, double, double)
DP_TOPK(f32, float, float, float)
DP_TOPK(bf16, uint16_t, __nv_bfloat16, float)
DP_TOPK(f16, uint16_t, __half, float)

}  // extern "C"
