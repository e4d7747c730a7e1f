// The forward calls of the norms around a block (norm_gate.cuh).
#include "norm_gate.cuh"

namespace dpc {
namespace {

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
  const bool layer = kind == DP_NORM_LAYER, full = gate_kind == DP_GATE_FULL;
  NormArgs<T> p{};
  p.in[0] = f, p.in[1] = r, p.in[2] = full ? gate : nullptr, p.nin = full ? 3 : 2;
  p.gate = gate_kind == DP_GATE_TOKEN ? gate : nullptr;
  p.a = a, p.w1 = w1, p.w2 = w2, p.b1 = layer ? b1 : nullptr, p.b2 = layer ? b2 : nullptr;
  p.fetched = ntok < give_up_at() ? ntok : give_up_at(), p.ntok = ntok, p.H = H, p.eps = (acc_t<T>)eps;
  p.r2 = r2, p.u = u, p.stats = stats;
  const int v = pack_width<T>(H, r, f, p.in[2], r2, u);
  if (!v || !at_elements(p.gate, a, w1, w2, p.b1, p.b2, stats)) return misaligned(who);
  const bool w16 = aligned16(a, w1, w2, p.b1, p.b2);
  const bool bases = aligned16(r, f, p.in[2], r2, u);
  const int lrc = layer ? launch<T, false, true>(p, v, w16, bases, (cudaStream_t)stream, who)
                        : launch<T, false, false>(p, v, w16, bases, (cudaStream_t)stream, who);
  return lrc ? lrc : launch_status(who);
}

}  // namespace

int take_wait_timeouts_norm_fwd(unsigned int *count) { return take_unit_timeouts(count); }

}  // namespace dpc

extern "C" {

#define DP_NORM(X, C, T, W)                                                                                            \
  int dp_norm_gate_fwd_##X(const C *r, const C *f, const C *gate, int gate_kind, const W *a, const W *w1, const W *b1, \
                           const W *w2, const W *b2, int64_t ntok, int H, int kind, double eps, C *r2, C *u, W *stats, \
                           void *stream) {                                                                             \
    return dpc::norm_fwd<T>((const T *)r, (const T *)f, (const T *)gate, gate_kind, a, w1, b1, w2, b2, ntok, H, kind,  \
                            eps, (T *)r2, (T *)u, stats, stream, "dp_norm_gate_fwd_" #X);                              \
  }
DP_NORM(f64, double, double, double)
DP_NORM(f32, float, float, float)
DP_NORM(bf16, uint16_t, __nv_bfloat16, float)
DP_NORM(f16, uint16_t, __half, float)

}  // extern "C"
