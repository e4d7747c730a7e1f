// Experts of each token from a router's logits, and the gradient of their weights.  For a row x of E logits and a bias b:
//   s = softmax(x) or sigmoid(x),  c = s + b
//   groups of E/G neighbours, each scored by the sum of its one or two largest c: the `keep` best stay
//   expert[j] = the j-th largest c left,  w_j = scale s_ej, or scale s_ej / sum_i s_ei
// Without a bias the experts are ordered by x itself, which has the order of s and no rounding.  Scores that are equal in
// f64 go by the larger logit, equal logits by the lowest index, a NaN stands above all numbers, an expert with x = -inf or
// b = -inf is never chosen (-1, weight 0).
// The choice is that of exact arithmetic as far as f64 has it, in up to three steps: first on f32 scores cut to leave
// room for the expert's index in the same word (one integer is compared and moved, and no two are equal); a token in
// which two neighbours of the chosen ones, the last of them and any that is left out (whose error may be far larger
// than a neighbour's: an s near 1 that a bias cancels), or the last group kept and the first one dropped are nearer
// than their error bounds is settled in f64 on those in question (eight lanes a token), or done again on whole f32
// scores and then in f64 (a warp a token).
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
  uint32_t mask;  // the bits of an expert's index
  uint32_t inv_per;  // floor(e inv_per / 2^32) is the group of expert e
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

// Whether equal scores c go by their logits: a sigmoid of 40 is 1 in f64, and c grows with x where the biases are equal.
// NaN and +inf are equal ones.
__device__ __forceinline__ bool goes_by_logit(unsigned long long key) { return key != 0 && key < 0xfff0000000000000ull; }

// Reductions over the L lanes of a token (mask: those lanes).
template <int L, typename V, typename F>
__device__ __forceinline__ V over(unsigned mask, V v, F f) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(mask, v, o));
  return v;
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
constexpr unsigned kAll = 0xffffffffu;
__device__ __forceinline__ uint32_t warp_max(uint32_t v) { return __reduce_max_sync(kAll, v); }
__device__ __forceinline__ unsigned long long warp_max(unsigned long long v) {
  return over<32>(kAll, v, [](unsigned long long a, unsigned long long b) { return a > b ? a : b; });
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

// s of a logit, from the row's largest and the sum of exp(x - most) for a softmax.
template <typename A>
__device__ __forceinline__ A score_of(A x, bool sigm, A most, A total) { return sigm ? sigmoid(x) : exp_(x - most) / total; }
// Scores of chosen logits up to a factor common to the row that keeps their sum from underflowing: for a softmax
// exp(x - m), for a sigmoid s exp(-m) with m = min(0, largest x).
template <typename A>
__device__ __forceinline__ A relative_score(A x, A most, bool sigm) {
  if (!sigm) return exp_(x - most);
  if (x >= A(0)) return A(1) / (A(1) + exp_(-x));
  return exp_(x - (most < A(0) ? most : A(0))) / (A(1) + exp_(x));
}

// f32 scores for the order: the relative error of s in ulp of 2^-23 (an exponential 2, a quotient, sum or difference 0.5;
// `range` the size of the softmax's argument x - m):
//   sigmoid  2 of the exponential, its product with the reciprocal, that and 1 + e: below 4
//   softmax  2, the argument's rounding 0.5 range, the quotient; the total: its terms' 2 and their arguments' roundings
//            (in the mean below 4), and (32 + 5) / 2 of its additions: below 28 + 0.5 range
__device__ __forceinline__ float score_error(float range, bool sigm) {
  return sigm ? 0x1p-21f : 0x1p-18f + 0x1p-24f * fminf(range, 128.0f);
}
// And absolutely, for exponentials and scores below the normal range, which the hardware's instructions flush.
constexpr float kFlushed = 0x1p-125f;
// Two scores that f32 cannot order: x the logits, b the biases (c = s + b), range the larger |argument|.  Equal inputs
// give equal scores; else s <= |c| + |b|, and the sum's own rounding is half an ulp.
__device__ __forceinline__ bool too_near(float c0, float c1, float x0, float x1, float b0, float b1, float range,
                                         bool sigm) {
  if (x0 == x1 && b0 == b1) return false;
  return !(c0 - c1 > (score_error(range, sigm) + 0x1p-23f) * (fabsf(c0) + fabsf(c1) + fabsf(b0) + fabsf(b1)) + kFlushed);
}
// A group's score from its two best (0 in the place of none), at half its size: no sum leaves the type's range.
template <typename A>
__device__ __forceinline__ A half_sum(A a, A b) { return A(0.5) * a + A(0.5) * b; }
// The least and the largest that a group's score may be, `spread` the sum of the |c| that it is made of (which may cancel in
// it): half of two s' errors or one s' error come to less than 2^-18 (a softmax's s to at most 1 together, and
// s ln(1 / s) to 0.37 each), the roundings of s + b and of the score to 2^-24 of the spread.
__device__ __forceinline__ float group_error(float spread) { return 0x1p-18f + 0x1p-23f * spread; }
__device__ __forceinline__ float group_least(float score, float spread) {
  const float v = score - group_error(spread);
  return score != score ? INFINITY : v == v ? v : -INFINITY;
}
__device__ __forceinline__ float group_most(float score, float spread) {
  const float v = score + group_error(spread);
  return v == v ? v : INFINITY;
}

// The first step's scores, by the hardware's base-two exponential (documented error 2^-22, its argument's roundings |x| ulp)
// and reciprocal (1 ulp).
__device__ __forceinline__ float rough_exp(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * 1.442695041f));
  return y;
}
__device__ __forceinline__ float rough_rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rough_sigmoid(float x) {
  const float e = rough_exp(-fabsf(x)), r = rough_rcp(1.0f + e);
  return x < 0.0f ? e * r : r;
}
__device__ __forceinline__ float rough_error(float range, bool sigm) {
  return (sigm ? 0x1p-20f : 0x1p-18f) + 0x1p-21f * fminf(range, 128.0f);
}
// A key with the index of its expert in the low bits (mask: all of them), the lower index the larger; 0 stays 0.
__device__ __forceinline__ uint32_t pack_key(uint32_t key, uint32_t mask, int e) {
  return key ? (key & ~mask) | (mask - e) : 0u;
}
__device__ __forceinline__ int packed_expert(uint32_t key, uint32_t mask) { return key ? (int)(mask - (key & mask)) : -1; }
// The size of the exponential's argument in a score.
__device__ __forceinline__ float range_of(float x0, float x1, float most, bool sigm) {
  return sigm ? fmaxf(fabsf(x0), fabsf(x1)) : most - fminf(x0, x1);
}
// Neighbours of the packed order that it may have wrong: their cut scores as intervals.
__device__ __forceinline__ bool packed_near(uint32_t k0, uint32_t k1, uint32_t mask, float x0, float x1, float b0, float b1,
                                            float range, bool sigm) {
  if (x0 == x1 && b0 == b1) return false;
  const float c0 = from_key(k0 & ~mask), c1 = from_key(k1 | mask);
  return !(c0 - c1 > (rough_error(range, sigm) + 0x1p-23f) * (fabsf(c0) + fabsf(c1) + fabsf(b0) + fabsf(b1)) + kFlushed);
}

// The largest c that an expert whose f32 score is at most c1 may have: s = c - b is at most |c1| + bmost (the largest finite
// |b|) and 1, the size of its exponential's argument at most ln(1 / s), and s ln(1 / s) grows up to s = 1/e.
__device__ __forceinline__ float reach_of(float c1, float bmost, bool sigm) {
  const float s = fminf(1.0f, fabsf(c1) + bmost);
  const float range = fmaxf(1.0f, 0.6932f * (float)(127 - (int)(__float_as_uint(s) >> 23)));
  return c1 + (rough_error(range, sigm) * s + 0x1p-22f * fabsf(c1) + kFlushed);
}
// The least c that a chosen one may have.
__device__ __forceinline__ float least_of(float c, float x, float b, float most, bool sigm) {
  return c - (rough_error(range_of(x, x, most, sigm), sigm) + 0x1p-23f) * (fabsf(c) + fabsf(b));
}

// Whether the warp's least group kept and largest one dropped leave the choice of groups open.
__device__ __forceinline__ bool groups_near(float least, float next) {
  least = over<32>(kAll, least, [](float a, float b) { return fminf(a, b); });
  next = over<32>(kAll, next, [](float a, float b) { return fmaxf(a, b); });
  return next > -INFINITY && !(least > next);
}

// The value of pair k - 1 of a warp's pairs.
template <int S, typename V>
__device__ __forceinline__ V of_last(int k, const V (&v)[S]) {
  V at = v[0];
#pragma unroll
  for (int s = 1; s < S; ++s)
    if ((k - 1) / 32 == s) at = v[s];
  return __shfl_sync(kAll, at, (k - 1) % 32);
}

// One token on a warp, N logits a lane: the i-th is expert 32 i + lane.  S chosen pairs a lane.  True: two scores are too near to tell apart in A, and nothing is written.  `room`: shared memory of the token,
// E + 3 G words of 8 bytes, for the groups.
template <typename T, typename A, int N, int S>
__device__ bool choose(const TopkArgs &p, int64_t t, unsigned char *room) {
  using U = key_t_<A>;
  constexpr bool kExact = sizeof(A) == 8;
  const int lane = threadIdx.x & 31;
  const T *x = (const T *)p.x + t * p.E;
  const acc_t<T> *bias = (const acc_t<T> *)p.bias;
  const bool grouped = p.keep < p.G, by_score = p.bias || (grouped && p.gtop == 2);
  A v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = i * 32 + lane < p.E ? (A)to_acc(x[i * 32 + lane]) : none<A>();
  A most = none<A>(), total = A(0);
  if (!p.sigmoid && (by_score || !p.renorm)) {
#pragma unroll
    for (int i = 0; i < N; ++i) most = v[i] != v[i] || v[i] > most ? v[i] : most;
    most = most_over<32>(kAll, most);
#pragma unroll
    for (int i = 0; i < N; ++i) total += v[i] == none<A>() ? A(0) : exp_(v[i] - most);
    total = sum_over<32>(kAll, total);
  }

  U key[N];
  const int per = p.E / p.G;
  U *ckey = (U *)room;  // of group g from g (per + 1) on: lanes of neighbouring groups fall on different banks
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * 32 + lane;
    A c = v[i], by = v[i];
    if (by_score && e < p.E) {
      const A b = bias ? (A)__ldg(bias + e) : A(0);
      const A s = p.sigmoid ? sigmoid(v[i]) : exp_(v[i] - most) / total;
      c = v[i] == none<A>() || b == none<A>() ? none<A>() : s + b;
      by = bias ? c : v[i];
    }
    key[i] = to_key(by);
    if (grouped && e < p.E) ckey[e + e / per] = to_key(c);
  }
  bool near = false;
  if (grouped) {
    U *gkey = (U *)(room + (size_t)(p.E + p.G) * 8), *kept = gkey + p.G;
    __syncwarp();
    for (int g = lane; g < p.G; g += 32) {
      U a = 0, b = 0;
      for (int i = 0; i < per; ++i) {
        const U c = ckey[g * (per + 1) + i];
        const U less = c < a ? c : a;
        b = less > b ? less : b;
        a = c > a ? c : a;
      }
      const A ca = a ? from_key(a) : A(0), cb = p.gtop == 2 && b ? from_key(b) : A(0);
      gkey[g] = p.gtop == 2 && a ? to_key(half_sum(ca, cb)) : a;
      if constexpr (!kExact) kept[g] = __float_as_uint(fabsf(ca) + fabsf(cb));  // until it is ranked, by this lane
    }
    __syncwarp();
    [[maybe_unused]] float least = INFINITY, next = -INFINITY;  // of the groups kept, and the largest of those dropped
    for (int g = lane; g < p.G; g += 32) {
      const U mine = gkey[g];
      int rank = 0;
      for (int o = 0; o < p.G; ++o) rank += gkey[o] > mine || (gkey[o] == mine && o < g);
      if constexpr (!kExact)
        if (mine) {
          const float spread = __uint_as_float(kept[g]);
          if (rank < p.keep) least = fminf(least, group_least(from_key(mine), spread));
          else next = fmaxf(next, group_most(from_key(mine), spread));
        }
      kept[g] = rank < p.keep;
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = i * 32 + lane;
      if (e < p.E && !kept[e / per]) key[i] = 0;
    }
    if constexpr (!kExact) near = by_score && groups_near(least, next);
  }

  // the best of each lane, then of the warp, k times; the keys of those that are left out stay
  int se[S];
  U sk[S];
  U best;
  auto pick = [&](auto by_logit) {
    constexpr bool kByLogit = decltype(by_logit)::value;
    int at;
    auto rescan = [&] {
      best = 0;
      at = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        bool first = key[i] > best;
        if constexpr (kByLogit)
          if (key[i] == best && bias && goes_by_logit(best)) first = to_acc(x[i * 32 + lane]) > to_acc(x[at * 32 + lane]);
        if (first) {
          best = key[i];
          at = i;
        }
      }
    };
    rescan();
#pragma unroll
    for (int s = 0; s < S; ++s) {
      se[s] = -1;
      sk[s] = 0;
    }
    for (int j = 0; j < p.k; ++j) {
      const U m = warp_max(best);
      if (m == 0) break;
      bool mine = best == m;
      if constexpr (kByLogit)
        if (bias && goes_by_logit(m) && __popc(__ballot_sync(kAll, mine)) > 1) {
          const A xm = mine ? (A)to_acc(x[at * 32 + lane]) : none<A>(), largest = most_over<32>(kAll, xm);  // by all lanes
          mine = mine && xm == largest;
        }
      const int e = __reduce_min_sync(kAll, mine ? at * 32 + lane : INT_MAX);
      if (e % 32 == lane) {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (i == at) key[i] = 0;
        rescan();
      }
#pragma unroll
      for (int s = 0; s < S; ++s)
        if (j == s * 32 + lane) {
          se[s] = e;
          sk[s] = m;
        }
    }
  };
  // Ties in f64 go by the logit in the same pass, but where 32 keys a lane leave no registers for it (8192 x 1024 f32 with 40
  // chosen, a few tokens of which come here: 513 us with, 472 without): there in a second one.
  pick(std::bool_constant<kExact && N <= 8>{});
  if constexpr (kExact && N > 8)
    if (bias) {  // equal scores of unequal logits, among the chosen ones or across their end
      const U kl = of_last(p.k, sk);
      const A xl = kl ? (A)to_acc(x[of_last(p.k, se)]) : A(0);
      bool tie = false;
#pragma unroll
      for (int i = 0; i < N; ++i) tie |= goes_by_logit(kl) && key[i] == kl && (A)to_acc(x[i * 32 + lane]) != xl;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const int from = (lane + 1) % 32, s1 = s + 1 < S ? s + 1 : s;
        const U k0 = __shfl_sync(kAll, sk[s], from), k1 = __shfl_sync(kAll, sk[s1], from);
        const int e0 = __shfl_sync(kAll, se[s], from), e1 = __shfl_sync(kAll, se[s1], from);
        const bool wrap = lane == 31;
        const U nk = wrap ? (S > 1 ? k1 : 0) : k0;
        if (goes_by_logit(sk[s]) && sk[s] == nk) tie |= to_acc(x[se[s]]) != to_acc(x[wrap ? e1 : e0]);
      }
      if (__any_sync(kAll, tie)) {
        for (int j = 0; j < p.k; ++j) {
          int e = se[0];
          U m = sk[0];
#pragma unroll
          for (int s = 1; s < S; ++s)
            if (j / 32 == s) {
              e = se[s];
              m = sk[s];
            }
          e = __shfl_sync(kAll, e, j % 32);
          m = __shfl_sync(kAll, m, j % 32);
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (e == i * 32 + lane) key[i] = m;
        }
        pick(std::true_type{});
      }
    }
  const bool check = !kExact && p.bias;
  A sx[S];
#pragma unroll
  for (int s = 0; s < S; ++s) sx[s] = se[s] >= 0 ? (A)to_acc(x[se[s]]) : none<A>();
  if constexpr (!kExact) {
    if (check) {
      float c[S], b[S];
#pragma unroll
      for (int s = 0; s < S; ++s) {
        c[s] = from_key(sk[s]);
        b[s] = se[s] >= 0 ? __ldg(bias + se[s]) : 0.0f;
      }
#pragma unroll
      for (int s = 0; s < S; ++s) {  // a pair and the next one: the next lane's, of the last lane the first lane's next
        const int from = (lane + 1) % 32, s1 = s + 1 < S ? s + 1 : s;
        const float c0 = __shfl_sync(kAll, c[s], from), c1 = __shfl_sync(kAll, c[s1], from);
        const float x0 = __shfl_sync(kAll, sx[s], from), x1 = __shfl_sync(kAll, sx[s1], from);
        const float b0 = __shfl_sync(kAll, b[s], from), b1 = __shfl_sync(kAll, b[s1], from);
        const int e0 = __shfl_sync(kAll, se[s], from), e1 = __shfl_sync(kAll, se[s1], from);
        const bool wrap = lane == 31;
        const float nx = wrap ? x1 : x0;
        if (s * 32 + lane < p.k && se[s] >= 0 && (wrap ? (S > 1 ? e1 : -1) : e0) >= 0) {
          const float range = most - fminf(sx[s], nx);
          near |= too_near(c[s], wrap ? c1 : c0, sx[s], nx, b[s], wrap ? b1 : b0, range, p.sigmoid);
        }
      }
      const int el = of_last(p.k, se);
      if (el >= 0) {
        const float cl = from_key(of_last(p.k, sk)), xl = to_acc(x[el]), bl = __ldg(bias + el);
        if (best && !(least_of(cl, xl, bl, most, p.sigmoid) > reach_of(from_key(best), 1.0f, p.sigmoid)))
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (key[i]) {
              const int e = i * 32 + lane;
              const float xe = to_acc(x[e]);
              near |= too_near(cl, from_key(key[i]), xl, xe, bl, __ldg(bias + e), most - fminf(xl, xe), p.sigmoid);
            }
      }
    }
    if (by_score && __any_sync(kAll, near)) return true;
  }

  A wsum = A(1), top = A(0);
  A ws[S];
  if (p.renorm) {
    top = none<A>();
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (se[s] >= 0) top = sx[s] != sx[s] || sx[s] > top ? sx[s] : top;
    }
    top = most_over<32>(kAll, top);
    wsum = A(0);
  }
#pragma unroll
  for (int s = 0; s < S; ++s) {
    ws[s] = se[s] < 0 ? A(0) : p.renorm ? relative_score(sx[s], top, p.sigmoid) : score_of(sx[s], p.sigmoid, most, total);
    if (p.renorm) wsum += ws[s];
  }
  // total * 0: a NaN or +inf anywhere makes every score of a softmax NaN, also where the chosen logits are numbers
  if (p.renorm) wsum = sum_over<32>(kAll, wsum) + (by_score ? total * A(0) : A(0));
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int j = s * 32 + lane;
    if (j < p.k) {
      p.expert[t * p.k + j] = se[s];
      ((acc_t<T> *)p.w)[t * p.k + j] = se[s] < 0 ? acc_t<T>(0) : (acc_t<T>)((A)p.scale * (ws[s] / wsum));
    }
  }
  return false;
}

// The later steps, rarely taken.
template <typename T, int N, int S>
__device__ __noinline__ void choose_again(const TopkArgs &p, int64_t t, unsigned char *room) {
  __syncwarp();
  if (!choose<T, float, N, S>(p, t, room)) return;
  __syncwarp();
  choose<T, double, N, S>(p, t, room);
}

// What the eight lanes of a token could not settle, whose bounds are those of f32 scores: in f64 at once.
template <typename T, int N>
__device__ __noinline__ void choose_exact(const TopkArgs &p, int64_t t, unsigned char *room) {
  __syncwarp();
  choose<T, double, N, 1>(p, t, room);
}

// The first step for a token on a warp; true: not sure.
template <typename T, int N, int S>
__device__ __forceinline__ bool choose_packed(const TopkArgs &p, int64_t t, unsigned char *room) {
  const int lane = threadIdx.x & 31;
  const T *x = (const T *)p.x + t * p.E;
  const float *bias = (const float *)p.bias;
  const bool grouped = p.keep < p.G, by_score = p.bias || (grouped && p.gtop == 2);
  const uint32_t mask = p.mask;
  float v[N], most = none<float>(), total = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = i * 32 + lane < p.E ? to_acc(x[i * 32 + lane]) : none<float>();
  if (!p.sigmoid && (by_score || !p.renorm)) {
#pragma unroll
    for (int i = 0; i < N; ++i) most = v[i] != v[i] || v[i] > most ? v[i] : most;
    most = most_over<32>(kAll, most);
#pragma unroll
    for (int i = 0; i < N; ++i) total += v[i] == none<float>() ? 0.0f : expf(v[i] - most);
    total = sum_over<32>(kAll, total);
  }
  uint32_t key[N], best = 0;
  const int per = p.E / p.G;
  uint32_t *ckey = (uint32_t *)room, *gkey = ckey + p.E + p.G, *kept = gkey + p.G;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * 32 + lane;
    uint32_t by = to_key(v[i]), c = by;
    if (by_score && e < p.E) {
      const float b = bias ? __ldg(bias + e) : 0.0f;
      const float s = p.sigmoid ? rough_sigmoid(v[i]) : rough_exp(v[i] - most) * rough_rcp(total);
      c = v[i] == none<float>() || b == none<float>() ? 0u : to_key(s + b);
      by = bias ? c : by;
    }
    if (grouped && e < p.E) ckey[e + e / per] = c;
    key[i] = pack_key(by, mask, e);
  }
  bool near = false;
  if (grouped) {
    __syncwarp();
    for (int g = lane; g < p.G; g += 32) {
      uint32_t a = 0, b = 0;
      const uint32_t *from = ckey + g * (per + 1);
#pragma unroll 4
      for (int i = 0; i < per; ++i) {
        const uint32_t c = from[i];
        b = max(b, min(a, c));
        a = max(a, c);
      }
      const float ca = a ? from_key(a) : 0.0f, cb = p.gtop == 2 && b ? from_key(b) : 0.0f;
      gkey[g] = p.gtop == 2 && a ? to_key(half_sum(ca, cb)) : a;
      kept[g] = __float_as_uint(fabsf(ca) + fabsf(cb));  // until it is ranked, by this lane
    }
    __syncwarp();
    float least = INFINITY, next = -INFINITY;  // as in choose()
    for (int g = lane; g < p.G; g += 32) {
      const uint32_t mine = gkey[g];
      int rank = 0;
#pragma unroll 4
      for (int o = 0; o < p.G; ++o) rank += gkey[o] > mine || (gkey[o] == mine && o < g);
      if (mine) {
        const float spread = __uint_as_float(kept[g]);
        if (rank < p.keep) least = fminf(least, group_least(from_key(mine), spread));
        else next = fmaxf(next, group_most(from_key(mine), spread));
      }
      kept[g] = rank < p.keep;
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = i * 32 + lane;
      if (e < p.E && !kept[e / per]) key[i] = 0;
    }
    near = by_score && groups_near(least, next);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) best = max(best, key[i]);
  uint32_t sk[S];
#pragma unroll
  for (int s = 0; s < S; ++s) sk[s] = 0;
  const bool check = p.bias || (sizeof(T) == 4);  // 16-bit logits are whole beside the index
  for (int j = 0; j < p.k; ++j) {
    const uint32_t m = warp_max(best);
    if (m == 0) break;
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (j == s * 32 + lane) sk[s] = m;
    if (m == best) {
      best = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        key[i] = key[i] == m ? 0u : key[i];
        best = max(best, key[i]);
      }
    }
  }
  int se[S];
  float sx[S];
#pragma unroll
  for (int s = 0; s < S; ++s) {
    se[s] = packed_expert(sk[s], mask);
    sx[s] = se[s] >= 0 ? to_acc(x[se[s]]) : none<float>();
  }
  if (check) {
    float b[S];
#pragma unroll
    for (int s = 0; s < S; ++s) b[s] = bias && se[s] >= 0 ? __ldg(bias + se[s]) : 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s) {  // a pair and the next one: the next lane's, of the last lane the first lane's next
      const int from = (lane + 1) % 32;
      uint32_t nk = __shfl_sync(kAll, sk[s], from);
      float nx = __shfl_sync(kAll, sx[s], from), nb = __shfl_sync(kAll, b[s], from);
      if constexpr (S > 1) {
        const int s1 = s + 1 < S ? s + 1 : s;
        const uint32_t k1 = __shfl_sync(kAll, sk[s1], from);
        const float x1 = __shfl_sync(kAll, sx[s1], from), b1 = __shfl_sync(kAll, b[s1], from);
        if (lane == 31) {
          nk = k1;
          nx = x1;
          nb = b1;
        }
      } else {
        if (lane == 31) nk = 0;
      }
      if (s * 32 + lane < p.k && sk[s] != 0 && nk != 0) {
        const float range = range_of(sx[s], nx, most, p.sigmoid);
        if (bias) near |= packed_near(sk[s], nk, mask, sx[s], nx, b[s], nb, range, p.sigmoid);
        else near |= ((sk[s] ^ nk) & ~mask) == 0 && sx[s] != nx;
      }
    }
    const uint32_t kl = of_last(p.k, sk);
    if (kl) {
      const int el = packed_expert(kl, mask);
      const float xl = to_acc(x[el]), bl = bias ? __ldg(bias + el) : 0.0f;
      // the lane's best by the widest bounds, its others by their own only where those do not do
      if (best && (bias ? !(least_of(from_key(kl & ~mask), xl, bl, most, p.sigmoid) > reach_of(from_key(best | mask), 1.0f, p.sigmoid))
                        : ((kl ^ best) & ~mask) == 0))
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (key[i]) {
            const int e = i * 32 + lane;
            const float xe = to_acc(x[e]);
            if (bias) near |= packed_near(kl, key[i], mask, xl, xe, bl, __ldg(bias + e), range_of(xl, xe, most, p.sigmoid), p.sigmoid);
            else near |= ((kl ^ key[i]) & ~mask) == 0 && xl != xe;
          }
    }
  }
  if (__any_sync(kAll, near)) return true;

  float wsum = 1.0f, top = none<float>(), ws[S];
#pragma unroll
  for (int s = 0; s < S; ++s) {
    if (se[s] >= 0) top = sx[s] != sx[s] || sx[s] > top ? sx[s] : top;
  }
  if (p.renorm) {
    top = most_over<32>(kAll, top);
    wsum = 0.0f;
  }
#pragma unroll
  for (int s = 0; s < S; ++s) {
    ws[s] = se[s] < 0 ? 0.0f : p.renorm ? relative_score(sx[s], top, p.sigmoid) : score_of(sx[s], p.sigmoid, most, total);
    if (p.renorm) wsum += ws[s];
  }
  if (p.renorm) wsum = sum_over<32>(kAll, wsum) + (by_score ? total * 0.0f : 0.0f);  // as in choose()
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int j = s * 32 + lane;
    if (j < p.k) {
      p.expert[t * p.k + j] = se[s];
      ((float *)p.w)[t * p.k + j] = se[s] < 0 ? 0.0f : (float)p.scale * (ws[s] / wsum);
    }
  }
  return false;
}

// Words of 8 bytes of a token's groups.
__host__ __device__ constexpr int room_words(int E, int G) { return E + 3 * G; }

// Four or eight blocks an SM: at the 134 registers that 32 logits a lane else take, 8192 x 1024 with 40 chosen took 506 us,
// not 461; with fewer logits it is the later steps that would take more than 64.
template <typename T, int N, int S>
__global__ void __launch_bounds__(kThreads, N == 32 ? 4 : 8) topk_kernel(const __grid_constant__ TopkArgs p) {
  extern __shared__ __align__(16) unsigned char rooms[];
  const int64_t t = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
  if (t >= p.ntok) return;
  unsigned char *room = rooms + (size_t)(threadIdx.x / 32) * room_words(p.E, p.G) * 8;
  if constexpr (sizeof(T) == 8) {
    choose<T, double, N, S>(p, t, room);
  } else {
    if (choose_packed<T, N, S>(p, t, room)) choose_again<T, N, S>(p, t, room);
  }
}

// Up to eight experts a token, the usual case: eight lanes a token.  Each lane sorts eight packed keys at a time in
// registers (19 exchanges) and merges them into its list of the best eight; three exchanges of lists between lanes leave
// the token's in all of them, and lane j works out pair j.  Bound by instructions: 220 a token for the best eight of 128
// logits, 65,536 tokens bf16 in 23 us (a warp a token as above, whose reductions, one an expert, leave most lanes idle: 550
// and 42; a thread a token with its column in shared memory: 400, 72), 480 with scores, a bias and four of eight groups, 46
// us (103, 115).  Eight blocks an SM at 64 registers, some 30 of a thread's spilled: with five at 96 it took 54.
constexpr int kList = 8;
__device__ __forceinline__ void exchange(uint32_t &a, uint32_t &b) {
  const uint32_t most = max(a, b);
  b = min(a, b);
  a = most;
}
__device__ __forceinline__ void sort8(uint32_t (&k)[8]) {  // descending
  constexpr int net[19][2] = {{0, 1}, {2, 3}, {4, 5}, {6, 7}, {0, 2}, {1, 3}, {4, 6}, {5, 7}, {1, 2}, {5, 6},
                              {0, 4}, {3, 7}, {1, 5}, {2, 6}, {1, 4}, {3, 6}, {2, 4}, {3, 5}, {3, 4}};
#pragma unroll
  for (int i = 0; i < 19; ++i) exchange(k[net[i][0]], k[net[i][1]]);
}
// The best eight of two descending lists, and the best of the others.
__device__ __forceinline__ void merge8(uint32_t (&a)[8], const uint32_t (&b)[8], uint32_t &left) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    left = max(left, min(a[i], b[7 - i]));
    a[i] = max(a[i], b[7 - i]);
  }
#pragma unroll
  for (int h = 4; h > 0; h >>= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!(i & h)) exchange(a[i], a[i + h]);
}
constexpr uint32_t kNoKey = 0x007fffffu;  // to_bits(-inf): no candidate, nor is what lies below
__device__ __forceinline__ uint32_t to_bits(float c) {  // as to_key in three instructions; the sum makes -0 and NaN positive
  const uint32_t u = __float_as_uint(c + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// What the packed keys leave open is settled in f64, on the few scores in question, by a token's eight lanes (m8).
__device__ __noinline__ double exact_score(double x, bool sigm, double most, double total) {
  if (!sigm) return exp(x - most) / total;
  const double e = exp(x < 0.0 ? x : -x);
  return (x < 0.0 ? e : 1.0) / (1.0 + e);
}
template <typename T>
__device__ __noinline__ double exact_total(const T *x, int E, float most, unsigned m8) {
  double total = 0.0;
  for (int e0 = threadIdx.x % 8; e0 < E; e0 += 32) {  // four exponentials on their way
    double part[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double v = e0 + 8 * i < E ? (double)to_acc(x[e0 + 8 * i]) : -INFINITY;
      part[i] = v == -INFINITY ? 0.0 : exp(v - most);
    }
    total += (part[0] + part[1]) + (part[2] + part[3]);
  }
  return sum_over<8>(m8, total);
}
// c as an ordered integer (to_key), 0 for an expert that is never chosen.
template <typename T>
__device__ __forceinline__ unsigned long long exact_key(const TopkArgs &p, const T *x, int e, float most, double total) {
  const double v = to_acc(x[e]), b = p.bias ? (double)__ldg((const float *)p.bias + e) : 0.0;
  return v == -INFINITY || b == -INFINITY ? 0ull : to_key(exact_score(v, p.sigmoid, most, total) + b);
}
// The groups to keep of a token: those surely above the border stay, the ones near it (up to eight) by their exact
// scores.  gkey, spread: the groups' f32 scores and what they are made of, least, next: as in choose().  False: too many.
template <typename T>
__device__ __noinline__ bool settle_groups(const TopkArgs &p, const T *x, const uint32_t *gkey, const float *spread,
                                           uint32_t *kept, float least, float next, float most, unsigned m8) {
  const int sub = threadIdx.x % 8, per = p.E / p.G;
  const double total = p.sigmoid ? 1.0 : exact_total(x, p.E, most, m8);
  int sure = 0, n = 0, g_of = -1;
  unsigned long long of = 0;
  for (int g = 0; g < p.G; ++g) {
    const float s = from_key(gkey[g]);
    const bool stays = kept[g];
    const bool open = gkey[g] > kNoKey && !(stays ? group_least(s, spread[g]) > next : group_most(s, spread[g]) < least);
    if (!open) {
      sure += stays;
      continue;
    }
    unsigned long long k0 = 0, k1 = 0;  // the group's two best
    for (int i = sub; i < per; i += 8) {
      const unsigned long long k = exact_key(p, x, g * per + i, most, total);
      k1 = k > k0 ? k0 : k > k1 ? k : k1;
      k0 = k > k0 ? k : k0;
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
      const unsigned long long q0 = __shfl_xor_sync(m8, k0, o), q1 = __shfl_xor_sync(m8, k1, o);
      const unsigned long long low = k0 < q0 ? k0 : q0, high = k1 > q1 ? k1 : q1;
      k1 = low > high ? low : high;
      k0 = k0 > q0 ? k0 : q0;
    }
    if (n == sub) {
      g_of = g;
      of = p.gtop == 2 && k0 ? to_key(half_sum(from_key(k0), k1 ? from_key(k1) : 0.0)) : k0;
    }
    ++n;
  }
  if (n > 8) return false;
  int rank = 0;
  for (int o = 0; o < n; ++o) {
    const unsigned long long k = __shfl_sync(m8, of, o, 8);
    rank += k > of || (k == of && o < sub);
  }
  __syncwarp(m8);  // all lanes have read the flags
  if (g_of >= 0) kept[g_of] = rank < p.keep - sure;
  return true;
}
// Whether an expert beside the lanes' e and e9 may have a larger c than `low`, the least of the k-th one, el.  kept: the
// groups' flags, or NULL.
template <typename T>
__device__ __noinline__ bool one_ahead(const TopkArgs &p, const T *x, int e, int e9, int el, double low, const uint32_t *kept,
                                       float most, float total, unsigned m8) {
  const float *bias = (const float *)p.bias;
  const float xl = to_acc(x[el]), bl = bias ? __ldg(bias + el) : 0.0f;
  const int per = p.E / p.G;
  int listed[8];
#pragma unroll
  for (int o = 0; o < 8; ++o) listed[o] = __shfl_sync(m8, e, o, 8);
  bool ahead = false;
#pragma unroll 2
  for (int i = threadIdx.x % 8; i < p.E; i += 8) {
    const float v = to_acc(x[i]), b = bias ? __ldg(bias + i) : 0.0f;
    bool out = i == e9 || v == none<float>() || b == none<float>() || (v == xl && b == bl && i > el);
#pragma unroll
    for (int o = 0; o < 8; ++o) out |= i == listed[o];
    if (out || (kept && !kept[i / per])) continue;
    const float c = bias ? score_of(v, p.sigmoid, most, total) + b : v;
    const float tol = bias ? (score_error(most - v, p.sigmoid) + 0x1p-23f) * (fabsf(c) + fabsf(b)) + kFlushed : 0.0f;
    ahead |= !(low - c > tol);
  }
  return __any_sync(m8, ahead);
}
// The list's experts and the best beyond it in their exact order: lane j's e (-1: none) becomes the j-th.  left: the best
// packed key beyond the list; kept as above.  False: one beyond them may belong to the first k.
template <typename T>
__device__ __noinline__ bool settle_list(const TopkArgs &p, const T *x, int &e, uint32_t left, const uint32_t *kept, float most,
                                         unsigned m8) {
  const int sub = threadIdx.x % 8;
  const double total = p.sigmoid || !p.bias ? 1.0 : exact_total(x, p.E, most, m8);
  auto exact = [&](int of) {
    return of < 0 ? 0ull : p.bias ? exact_key(p, x, of, most, total) : to_key((double)to_acc(x[of]));
  };
  const int e9 = left > kNoKey ? (int)(p.mask - (left & p.mask)) : -1;
  const unsigned long long key = exact(e), key9 = exact(e9);
  const float xe = e >= 0 ? to_acc(x[e]) : 0.0f, x9 = e9 >= 0 ? to_acc(x[e9]) : 0.0f;
  auto before = [](unsigned long long k0, float x0, int e0, unsigned long long k1, float x1, int e1) {  // k1 not 0
    return k0 > k1 || (k0 == k1 && (goes_by_logit(k1) && x0 != x1 ? x0 > x1 : e0 < e1));
  };
  const bool after9 = key9 && before(key9, x9, e9, key, xe, e);
  const int listed = e;
  int rank = after9;
#pragma unroll
  for (int o = 0; o < 8; ++o) {
    const unsigned long long k = __shfl_sync(m8, key, o, 8);
    const int eo = __shfl_sync(m8, e, o, 8);
    const float xo = __shfl_sync(m8, xe, o, 8);
    rank += k | key ? before(k, xo, eo, key, xe, e) : o < sub;  // those without an expert stay in order at the end
  }
  const int rank9 = 8 - __popc(__ballot_sync(m8, after9));
  unsigned long long last = rank9 == p.k - 1 ? key9 : 0ull;  // the k-th
  int sorted = rank9 == sub ? e9 : -1;
#pragma unroll
  for (int o = 0; o < 8; ++o) {
    const int r = __shfl_sync(m8, rank, o, 8), eo = __shfl_sync(m8, e, o, 8);
    const unsigned long long k = __shfl_sync(m8, key, o, 8);
    if (r == sub) sorted = eo;
    if (r == p.k - 1) last = k;
  }
  e = sorted;
  const int el = __shfl_sync(m8, e, p.k - 1, 8);
  if (el < 0) return true;  // all that may be chosen are
  const float beyond = from_key(left | p.mask);  // those are behind it in the packed order
  if (left <= kNoKey || from_key(last) > (p.bias ? reach_of(beyond, 1.0f, p.sigmoid) : beyond)) return true;
  return !one_ahead(p, x, listed, e9, el, from_key(last), kept, most, (float)total, m8);
}

__host__ __device__ constexpr int list_words(int E, int G) { return (E + E / 8 + 1 + 3 * G) | 1; }

template <typename T, bool Whole>
__global__ void __launch_bounds__(kThreads, 8) topk_lists_kernel(const __grid_constant__ TopkArgs p) {
  extern __shared__ __align__(16) unsigned char rooms[];
  constexpr int V = 16 / (int)sizeof(T);
  const int sub = threadIdx.x % 8, slot = threadIdx.x / 8;
  const int64_t t_ = (int64_t)blockIdx.x * (kThreads / 8) + slot, t = t_ < p.ntok ? t_ : p.ntok - 1;
  const bool mine = t_ < p.ntok;
  const T *x = (const T *)p.x + t * p.E;
  const float *bias = (const float *)p.bias;
  const bool grouped = p.keep < p.G, by_score = p.bias || (grouped && p.gtop == 2);
  const uint32_t mask = p.mask;
  auto load = [&](int e0, float (&v)[8]) {  // -inf past the last expert
    if constexpr (Whole) {
#pragma unroll
      for (int i = 0; i < 8; i += V) {
        Pack<T, V> q;
        if (e0 + i < p.E) q = load_pack<T, V>(x + e0 + i);
#pragma unroll
        for (int l = 0; l < V; ++l) v[i + l] = e0 + i < p.E ? to_acc(q.v[l]) : none<float>();
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = e0 + i < p.E ? to_acc(x[e0 + i]) : none<float>();
    }
  };
  const int first = sub * 8;
  float most = none<float>(), total = 0.0f;
  if (!p.sigmoid && (by_score || !p.renorm)) {
    for (int e0 = first; e0 < p.E; e0 += 64) {
      float v[8];
      load(e0, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) most = v[i] != v[i] || v[i] > most ? v[i] : most;
    }
    most = most_over<8>(kAll, most);
    for (int e0 = first; e0 < p.E; e0 += 64) {  // at most 16 parts of eight terms
      float v[8], part = 0.0f;
      load(e0, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) part += v[i] == none<float>() ? 0.0f : expf(v[i] - most);
      total += part;
    }
    total = sum_over<8>(kAll, total);
  }
  auto biases = [&](int e0, float (&b)[8]) {
    if (bias && e0 + 8 <= p.E && !((uintptr_t)bias & 15)) {
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        const float4 q = __ldg(reinterpret_cast<const float4 *>(bias + e0 + i));
        b[i] = q.x;
        b[i + 1] = q.y;
        b[i + 2] = q.z;
        b[i + 3] = q.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) b[i] = bias && e0 + i < p.E ? __ldg(bias + e0 + i) : 0.0f;
    }
  };
  auto bits = [&](float v, float b) {  // the order of c
    const float s = p.sigmoid ? rough_sigmoid(v) : rough_exp(v - most) * rough_rcp(total);
    return v == none<float>() || b == none<float>() ? kNoKey : to_bits(s + b);
  };
  bool lost = false;  // not to be settled here
  const unsigned m8 = 0xffu << (threadIdx.x & 24);
  // the token's keys (a word more for eight: lanes and groups begin on different banks), the groups' scores
  uint32_t *ckey = (uint32_t *)rooms + slot * list_words(p.E, p.G), *gkey = ckey + p.E + p.E / 8 + 1, *kept = gkey + p.G;
  float *spread = (float *)(kept + p.G);
  const int per = p.E / p.G;
  if (grouped) {
    for (int e0 = first; e0 < p.E; e0 += 64) {
      float v[8], b[8];
      load(e0, v);
      if (by_score) biases(e0, b);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (e0 + i < p.E) ckey[e0 + e0 / 8 + i] = by_score ? bits(v[i], b[i]) : to_bits(v[i]);
    }
    __syncwarp();
    for (int g = sub; g < p.G; g += 8) {
      uint32_t a = kNoKey, b = kNoKey;
#pragma unroll 4
      for (int i = g * per; i < (g + 1) * per; ++i) {
        const uint32_t k = ckey[i + i / 8];
        b = max(b, min(a, k));
        a = max(a, k);
      }
      const float ca = a > kNoKey ? from_key(a) : 0.0f, cb = p.gtop == 2 && b > kNoKey ? from_key(b) : 0.0f;
      gkey[g] = p.gtop == 2 && a > kNoKey ? to_bits(half_sum(ca, cb)) : a;
      spread[g] = fabsf(ca) + fabsf(cb);
    }
    __syncwarp();
    float least = INFINITY, next = -INFINITY;  // as in choose()
    for (int g = sub; g < p.G; g += 8) {
      const uint32_t k = gkey[g];
      int rank = 0;
#pragma unroll 4
      for (int o = 0; o < p.G; ++o) rank += gkey[o] > k || (gkey[o] == k && o < g);
      kept[g] = rank < p.keep;
      if (k > kNoKey) {
        if (rank < p.keep) least = fminf(least, group_least(from_key(k), spread[g]));
        else next = fmaxf(next, group_most(from_key(k), spread[g]));
      }
    }
    __syncwarp();  // settle_groups reads the flags of all lanes' groups
    least = over<8>(kAll, least, [](float a, float b) { return fminf(a, b); });
    next = over<8>(kAll, next, [](float a, float b) { return fmaxf(a, b); });
    if (by_score && next > -INFINITY && !(least > next))
      lost = !settle_groups(p, x, gkey, spread, kept, least, next, most, m8);
    __syncwarp();
  }
  uint32_t list[8], left = 0;  // the best beyond the list
#pragma unroll
  for (int i = 0; i < 8; ++i) list[i] = 0;
#pragma unroll 1
  for (int e0 = first; e0 < p.E; e0 += 64) {
    uint32_t k[8];
    float v[8], b[8];
    if (!(grouped && bias)) load(e0, v);
    if (!grouped && bias) biases(e0, b);
    const bool same = per % 8 == 0;  // eight neighbours of one group
    const bool in = grouped && same && e0 < p.E && kept[__umulhi(e0, p.inv_per)];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = e0 + i;
      if (!grouped) k[i] = bias ? bits(v[i], b[i]) : to_bits(v[i]);
      else k[i] = !(same ? in : e < p.E && kept[__umulhi(e, p.inv_per)]) ? 0u : bias ? ckey[e0 + e0 / 8 + i] : to_bits(v[i]);
      k[i] = (k[i] & ~mask) | ((mask - e) & mask);  // past the last expert: no candidate
    }
    sort8(k);
    if (e0 == first) {
#pragma unroll
      for (int i = 0; i < 8; ++i) list[i] = k[i];
    } else {
      merge8(list, k, left);
    }
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = __shfl_xor_sync(kAll, list[i], o);
    left = max(left, __shfl_xor_sync(kAll, left, o));
    merge8(list, b, left);
  }
  uint32_t key = 0, next = left;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i == sub) key = list[i];
    if (i == sub + 1) next = list[i];
  }
  int e = key > kNoKey ? (int)(mask - (key & mask)) : -1;
  float xe = e >= 0 ? to_acc(x[e]) : none<float>();
  if (bias || sizeof(T) == 4) {  // 16-bit logits are whole beside the index
    // Neighbours in the order: the chosen ones each with the next, the last of them with all that follow.  Those may begin
    // with its equals, which are rightly behind it: the first pair that differs, its lane `border`, decides.
    const bool pair = e >= 0 && next > kNoKey;
    const int en = pair ? (int)(mask - (next & mask)) : 0;
    const float xn = pair ? to_acc(x[en]) : 0.0f;
    const float b0 = bias && pair ? __ldg(bias + e) : 0.0f, b1 = bias && pair ? __ldg(bias + en) : 0.0f;
    const bool same = pair && xe == xn && b0 == b1;
    const unsigned at = threadIdx.x & 24;
    const int border = __ffs((~__ballot_sync(kAll, same) >> at & 255) >> (p.k - 1)) + p.k - 2;  // k - 2: none
    bool near = false;
    float low = 0.0f;  // the least that c may be
    if (pair && !same) {
      if (!bias) {
        near = (sub < p.k - 1 || sub == border) && ((key ^ next) & ~mask) == 0;
      } else if (sub < p.k - 1) {
        near = packed_near(key, next, mask, xe, xn, b0, b1, range_of(xe, xn, most, p.sigmoid), p.sigmoid);
      } else if (sub == border) {
        low = least_of(from_key(key & ~mask), xe, b0, most, p.sigmoid);
        near = !(low > reach_of(from_key(next | mask), 1.0f, p.sigmoid));
      }
    }
    if (bias && __any_sync(kAll, near)) {  // looked at again with the largest |b|, where scores are far below 1
      float bmost = 0.0f;
      for (int i = sub; i < p.E; i += 8) {
        const float b = fabsf(__ldg(bias + i));
        bmost = b < INFINITY ? fmaxf(bmost, b) : bmost;  // -inf is out, +inf comes first
      }
      bmost = over<8>(kAll, bmost, [](float a, float b) { return fmaxf(a, b); });
      if (near && sub == border) near = !(low > reach_of(from_key(next | mask), bmost, p.sigmoid));
    }
    bool unsure = __ballot_sync(kAll, near) & m8;
    if (!unsure && border < p.k - 1) {  // its equals fill the list
      if (bias) low = least_of(from_key(key & ~mask), xe, b0, most, p.sigmoid);
      unsure = one_ahead(p, x, e, -1, __shfl_sync(m8, e, p.k - 1, 8), __shfl_sync(m8, bias ? low : xe, p.k - 1, 8),
                         grouped ? kept : nullptr, most, total, m8);
    }
    if (unsure) {
      lost |= !settle_list(p, x, e, left, grouped ? kept : nullptr, most, m8);
      xe = e >= 0 ? to_acc(x[e]) : none<float>();
    }
    __syncwarp();
  }
  const bool have = sub < p.k && e >= 0;
  if (!have) xe = none<float>();
  const float top = p.renorm ? most_over<8>(kAll, xe) : 0.0f;
  const float w = !have ? 0.0f : p.renorm ? relative_score(xe, top, p.sigmoid) : score_of(xe, p.sigmoid, most, total);
  const float sum = p.renorm ? sum_over<8>(kAll, w) + (by_score ? total * 0.0f : 0.0f) : 1.0f;  // as in choose()
  const unsigned unsure = __ballot_sync(kAll, lost && mine);
  if (mine && sub < p.k && !lost) {
    p.expert[t * p.k + sub] = have ? e : -1;
    ((float *)p.w)[t * p.k + sub] = have ? (float)p.scale * (w / sum) : 0.0f;
  }
  if (unsure) {  // the warp's rooms are read no more
    unsigned char *room = (unsigned char *)((uint32_t *)rooms + (threadIdx.x / 32) * 4 * list_words(p.E, p.G));
    for (int i = 0; i < 4; ++i)
      if (unsure >> (8 * i) & 255) {
        const int64_t again = (int64_t)blockIdx.x * (kThreads / 8) + (threadIdx.x / 32) * 4 + i;
        if (p.E <= 256) choose_exact<T, 8>(p, again, room);
        else choose_exact<T, 32>(p, again, room);
      }
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

// The gradient where it reaches the chosen logits alone: a warp takes `tokens` (up to 32) neighbouring ones, a thread
// works out a token's few values and adds them into a tile of zeros in shared memory, which the warp then stores: 65,536 x
// 128 f32 of six pairs in 18 us.  The zeros' way to memory would take 6; what is left is the latency of ids, then logits.
template <typename T, int V>
__global__ void __launch_bounds__(64) topk_grad_sparse_kernel(const __grid_constant__ TopkGradArgs p, int tokens) {
  using A = acc_t<T>;
  extern __shared__ __align__(16) unsigned char tiles[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const int64_t t0 = ((int64_t)blockIdx.x * 2 + warp) * tokens, t = t0 + lane;
  if (t0 >= p.ntok) return;
  const int have = (int)min((int64_t)tokens, p.ntok - t0), n = have * p.E;
  A *tile = (A *)tiles + (size_t)warp * ((tokens * p.E + 15) / 16 * 16);
  constexpr int kVA = 16 / (int)sizeof(A);
  for (int c = lane * kVA; c < n; c += 32 * kVA) store_pack<A, kVA>(tile + c, Pack<A, kVA>{});  // in whole packs
  __syncwarp();
  if (lane < have) {
    constexpr int kAtOnce = 8;  // pairs whose logits are on their way
    const T *x = (const T *)p.x + t * p.E;
    const A scale = (A)p.scale;
    A *to = tile + lane * p.E;
    int e[kAtOnce];
    A v[kAtOnce], d[kAtOnce];
    auto read = [&](int j0) {  // -inf: no pair
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        e[i] = j0 + i < p.k ? __ldg(p.expert + t * p.k + j0 + i) : -1;
        d[i] = j0 + i < p.k ? scale * __ldg((const A *)p.dw + t * p.k + j0 + i) : A(0);
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) v[i] = (unsigned)e[i] < (unsigned)p.E ? to_acc(x[e[i]]) : none<A>();
    };
    A sum = A(1), mean = A(0), top = none<A>(), q[kAtOnce], rest[kAtOnce];
    // a pair's score as relative_score has it and, for a sigmoid, 1 - s, from one exponential and one quotient
    auto terms = [&] {
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (p.sigmoid) {
          const A x = exp_(v[i] < A(0) ? v[i] : -v[i]), r = A(1) / (A(1) + x);
          q[i] = (p.renorm && top < A(0) ? exp_(v[i] - top) : v[i] < A(0) ? x : A(1)) * r;
          rest[i] = v[i] < A(0) ? r : x * r;
        } else {
          q[i] = exp_(v[i] - top);
          rest[i] = A(1);
        }
      }
    };
    const bool once = p.k <= kAtOnce;
    read(0);
    if (p.renorm) {
      for (int j0 = 0; j0 < p.k; j0 += kAtOnce) {
        if (j0) read(j0);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) top = v[i] != v[i] || v[i] > top ? v[i] : top;
      }
      sum = A(0);
      for (int j0 = 0; j0 < p.k; j0 += kAtOnce) {
        if (!once) read(j0);
        terms();
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          if (v[i] != none<A>()) {
            sum += q[i];
            mean += q[i] * d[i];
          }
      }
      mean /= sum;
    }
    for (int j0 = 0; j0 < p.k; j0 += kAtOnce) {
      if (!once) read(j0);
      if (!once || !p.renorm) terms();
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (v[i] != none<A>()) to[e[i]] += (p.renorm ? q[i] / sum : q[i]) * (d[i] - mean) * rest[i];
    }
  }
  __syncwarp();
  T *dx = (T *)p.dx + t0 * p.E;
  for (int c = lane * V; c < n; c += 32 * V) {
    if (c + V <= n) {
      Pack<T, V> o;
#pragma unroll
      for (int l = 0; l < V; ++l) o.v[l] = from_acc<T>(tile[c + l]);
      store_pack<T, V>(dx + c, o);
    } else {
      for (int l = c; l < n; ++l) dx[l] = from_acc<T>(tile[l]);
    }
  }
}

// A softmax without renormalisation reaches every logit: L lanes a token, N logits a lane.  30,011 x 61 f16 in 13 us.
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
  if (!scale_fits<acc_t<T>>(scale)) return set_error(DP_ERR_SHAPE, "%s: scale = %g", who, scale);
  if (ntok == 0) return DP_OK;
  if (!x || !expert || !w) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (!at_elements(x, bias, w) || !at_elements(expert)) return misaligned(who);
  if (G == E) G = keep = 1;  // groups of one: their best are the best experts
  TopkArgs p{x, bias, ntok, E, k, score == DP_SCORE_SIGMOID, G, keep, gtop, renorm != 0, scale, expert, w, 0, 0};
  p.inv_per = (uint32_t)(((1ull << 32) + E / G - 1) / (E / G));
  while ((int)p.mask < E - 1) p.mask = 2 * p.mask + 1;
  const cudaStream_t st = (cudaStream_t)stream;
  if constexpr (sizeof(T) < 8)
    if (k <= kList) {
      constexpr int tok = kThreads / 8;
      const bool whole = (((uintptr_t)x | (uintptr_t)(E * sizeof(T))) & 15) == 0;
      auto kernel = whole ? topk_lists_kernel<T, true> : topk_lists_kernel<T, false>;
      const size_t smem = keep < G ? (size_t)tok * list_words(E, G) * 4 : 0;
      constexpr size_t most = (size_t)tok * list_words(kMaxExperts, kMaxExperts / 2) * 4;
      if (smem > 48 * 1024 && (rc = allow_smem((const void *)kernel, most, who))) return rc;
      kernel<<<(unsigned)((ntok + tok - 1) / tok), kThreads, smem, st>>>(p);
      return launch_status(who);
    }
  auto go = [&](auto N_, auto S_) {
    constexpr int N = decltype(N_)::value, S = decltype(S_)::value, tok = kThreads / 32;
    const size_t smem = keep < G ? (size_t)tok * room_words(E, G) * 8 : 0;
    auto kernel = topk_kernel<T, N, S>;
    constexpr size_t most = (size_t)tok * room_words(32 * N, 16 * N) * 8;
    if (smem > 48 * 1024 && (rc = allow_smem((const void *)kernel, most, who))) return;
    kernel<<<(unsigned)((ntok + tok - 1) / tok), kThreads, smem, st>>>(p);
  };
  using std::integral_constant;
  if (k < 32) {
    if (E <= 32) go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    else if (E <= 128) go(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    else if (E <= 256) go(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  } else {
    if (E <= 256) go(integral_constant<int, 8>{}, integral_constant<int, 3>{});
    else go(integral_constant<int, 32>{}, integral_constant<int, 3>{});
  }
  return rc ? rc : launch_status(who);
}

template <typename T>
int topk_grad(const T *x, const int32_t *expert, const acc_t<T> *dw, int64_t ntok, int E, int k, int score, int renorm,
              double scale, T *dx, void *stream, const char *who) {
  clear_error();
  const int rc = topk_check(ntok, E, k, score, who);
  if (rc) return rc;
  if (!scale_fits<acc_t<T>>(scale)) return set_error(DP_ERR_SHAPE, "%s: scale = %g", who, scale);
  if (ntok == 0) return DP_OK;
  if (!x || !expert || !dw || !dx) return set_error(DP_ERR_NULL, "%s: NULL array", who);
  if (!at_elements(x, dx) || !at_elements(expert) || !at_elements(dw)) return misaligned(who);
  const TopkGradArgs p{x, expert, dw, ntok, E, k, score == DP_SCORE_SIGMOID, renorm != 0, scale, dx};
  if (renorm || score == DP_SCORE_SIGMOID) {
    const int most = 8192 / (int)sizeof(acc_t<T>) / E;  // tokens of a tile of 8 KB
    const int tokens = most >= 32 ? 32 : most >= 8 ? most / 8 * 8 : most < 1 ? 1 : most;
    const size_t smem = (size_t)(tokens * E + 15) / 16 * 16 * sizeof(acc_t<T>) * 2;
    constexpr int V = 16 / (int)sizeof(T);
    // a warp's tile begins at whole packs
    const bool whole = (((uintptr_t)dx | (uintptr_t)(tokens * E * sizeof(T))) & 15) == 0;
    auto k_ = whole ? topk_grad_sparse_kernel<T, V> : topk_grad_sparse_kernel<T, 1>;
    const int64_t blocks = (ntok + 2 * tokens - 1) / (2 * tokens);
    k_<<<(unsigned)blocks, 64, smem, (cudaStream_t)stream>>>(p, tokens);
    return launch_status(who);
  }
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
