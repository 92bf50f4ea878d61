// Log-probabilities of given classes and the losses made from them: what the kernels share (the formulas: fw_logprob.cu).
#ifndef FW_LOGPROB_CUH_
#define FW_LOGPROB_CUH_

#include "fw_internal.h"
#include "fw_rows.cuh"

namespace fw {
namespace logprob {

using namespace rows;

constexpr int kMaxV = 1 << 20;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLow = -3.402823466e38f;   // the lowest finite value: the largest of nothing, beside a sum of 0
enum { LP_FORWARD = 0, LP_BOTH = 1, LP_BACKWARD = 2 };

struct Logprob {
  const void* Z;
  void* dZ;
  const void* id;
  const float *stat_in, *dlogp_in;                                // backward
  float *logp, *stat;                                             // each may be null
  const float *logp_old, *logp_ref, *adv, *weight;                // policy: loss is not null
  float *loss, *dlogp;
  int64_t rows, ldz, lddz;
  int32_t V, i64;
  float inv_tau, low, high, kl;                                   // 1 - clip_low, 1 + clip_high
};

// What a row needs besides its logits; z: the logit of its class
struct Head {
  int id;                                                         // -1: the row does not count
  float z, a, b, c, d;                                            // policy: adv, logp_old, logp_ref, weight; backward: dlogp, stat
};
template <class T, int MODE>
__device__ __forceinline__ Head head_of(const Logprob& p, int64_t row) {
  Head h = {-1, 0.f, 0.f, 0.f, 0.f, 1.f};
  if (row >= p.rows) return h;
  const int64_t i = p.i64 ? static_cast<const int64_t*>(p.id)[row] : static_cast<const int32_t*>(p.id)[row];
  bool live = i >= 0 && i < p.V;
  if (MODE == LP_BACKWARD) {
    h.a = p.dlogp_in[row];
    live = live && h.a != 0.f;
    h.b = p.stat_in[2 * row];
    h.c = p.stat_in[2 * row + 1];
  } else if (p.loss) {
    if (p.weight) h.d = p.weight[row];
    live = live && h.d != 0.f;
    h.a = p.adv[row];
    h.b = p.logp_old[row];
    if (p.logp_ref) h.c = p.logp_ref[row];
  }
  if (live) {
    h.id = (int)i;
    h.z = to_f(static_cast<const T*>(p.Z)[row * p.ldz + i]);
  }
  return h;
}

// Largest logit m and the sum of exp((z - m) / tau).  Differences of logits are scaled, not logits: near the largest, where the
// mass is, their rounding is small.  c2 = log2(e) / tau.
struct MaxSum { float m, l; };
__device__ __forceinline__ MaxSum merge(MaxSum a, MaxSum b, float c2) {
  const float m = fmaxf(a.m, b.m);
  return {m, fmaf(a.l, ex2((a.m - m) * c2), __fmul_rn(b.l, ex2((b.m - m) * c2)))};
}
__device__ __forceinline__ MaxSum merge_lanes(MaxSum s, float c2) {
  float m;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(s.m));
  return {m, warp_sum(s.l * ex2((s.m - m) * c2))};
}

// The row's numbers from those of the classes other than its own.
struct Row {
  float m, others, all;                                           // largest logit; sums of exp((z - m) / tau)
  float logp;
  bool empty;                                                     // no class has mass
};
__device__ __forceinline__ Row row_of(MaxSum o, float z, float c2, float inv_tau) {
  Row r;
  r.m = fmaxf(o.m, z);
  r.others = o.l * ex2((o.m - r.m) * c2);
  const float e = z == -INFINITY ? 0.f : ex2((z - r.m) * c2);
  r.all = r.others + e;
  r.empty = r.all == 0.f;
  // of a class that has most of the mass 1 - q is what matters, and it is the others' sum
  r.logp = r.empty ? 0.f : r.others < e ? -log1pf(r.others / e) : fmaf(z - r.m, inv_tau, -logf(r.all));
  return r;
}

// Loss and d loss / d logp of one row
struct Slope { float loss, dlogp; };
__device__ __forceinline__ Slope policy_of(const Logprob& p, const Head& h, float logp) {
  const float ratio = expf(logp - h.b), free = ratio * h.a, held = fminf(fmaxf(ratio, p.low), p.high) * h.a;
  Slope s = {-fminf(free, held), free <= held ? -free : 0.f};
  if (ratio != ratio || free != free) s = {free + ratio, free + ratio};
  if (p.logp_ref) {
    const float k = h.c - logp, e1 = expm1f(k);
    // exp(k) - 1 - k of a small k by its series (below 1/4: the seventh term is 2e-8 of the first)
    const float low = k * k * fmaf(k, fmaf(k, fmaf(k, fmaf(k, fmaf(k, 1.f / 5040.f, 1.f / 720.f), 1.f / 120.f), 1.f / 24.f), 1.f / 6.f), 0.5f);
    s.loss = fmaf(p.kl, fabsf(k) < 0.25f ? low : e1 - k, s.loss);
    s.dlogp = fmaf(-p.kl, e1, s.dlogp);
  }
  return {h.d * s.loss, h.d * s.dlogp};
}

}  // namespace logprob
}  // namespace fw
#endif
