// The backward calls of the norms around a block (norm_gate.cuh).
#include "norm_gate.cuh"

namespace dpc {
namespace {

int grad_blocks(int H) { return 152 * norm_shape(H, true).blocks; }

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
  if (work_bytes < (size_t)grad_blocks(H) * kNormVectors * H * sizeof(acc_t<T>) || ((uintptr_t)work & 15))
    return set_error(DP_ERR_SHAPE, "%s: work buffer of %zu bytes is too short or misaligned", who, work_bytes);
  const bool full = gate_kind == DP_GATE_FULL;
  NormArgs<T> p{};
  p.in[0] = r2, p.in[1] = du, p.in[2] = dr2, p.in[3] = f, p.in[4] = full ? gate : nullptr, p.nin = full ? 5 : 4;
  p.gate = gate_kind == DP_GATE_TOKEN ? gate : nullptr;
  p.a = a, p.w1 = w1, p.w2 = w2, p.b1 = layer ? b1 : nullptr;
  p.fetched = ntok < give_up_at() ? ntok : give_up_at(), p.ntok = ntok, p.H = H;
  p.stats = const_cast<acc_t<T> *>(stats), p.dr = dr, p.df = df;
  p.dgate = gate_kind == DP_GATE_NONE ? nullptr : dgate;
  p.part = (acc_t<T> *)work;
  const int v = pack_width<T>(H, r2, f, p.in[4], dr2, du, dr, df, full ? dgate : nullptr);
  if (!v || !at_elements(p.gate, p.dgate, a, w1, w2, p.b1, stats, da, dw1, dw2) ||
      (layer && !at_elements(db1, db2)))
    return misaligned(who);
  const cudaStream_t st = (cudaStream_t)stream;
  const bool w16 = aligned16(a, w1, w2, p.b1);
  const bool bases = aligned16(r2, f, p.in[4], dr2, du, dr, df, full ? dgate : nullptr);
  const int lrc = layer ? launch<T, true, true>(p, v, w16, bases, st, who)
                        : launch<T, true, false>(p, v, w16, bases, st, who);
  if (lrc) return lrc;
  norm_finish_kernel<acc_t<T>><<<dim3((H + 31) / 32, layer ? kNormVectors : 3), 1024, 0, st>>>(
      p.part, grad_blocks(H), H, da, dw1, dw2, db1, db2);
  return launch_status(who);
}

}  // namespace

int take_wait_timeouts_norm_grad(unsigned int *count) { return take_unit_timeouts(count); }

}  // namespace dpc

extern "C" {

size_t dp_norm_gate_work_bytes(int H, int elem_bytes) {
  if (H < 1 || H > dpc::kNormMaxH || (elem_bytes != 2 && elem_bytes != 4 && elem_bytes != 8)) return 0;
  return (size_t)dpc::grad_blocks(H) * dpc::kNormVectors * H * (elem_bytes == 8 ? 8 : 4);
}

#define DP_NORM(X, C, T, W)                                                                                            \
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
