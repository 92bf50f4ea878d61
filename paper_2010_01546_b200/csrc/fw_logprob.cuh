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
  const float ratio = expf(logp - h.b), held = fminf(fmaxf(ratio, p.low), p.high) * h.a;
  const float free = ratio == INFINITY && h.a == 0.f ? 0.f : ratio * h.a;      // the ratio is a number, though beyond fp32
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

// 16 bytes of a row
template <class T> struct Group;
template <> struct Group<float> {
  static constexpr int VEC = 4;
  static constexpr uint32_t kNone = 0xff800000u;             // -inf
  // the larger of m and the largest of the group
  static __device__ __forceinline__ float top(uint4 q, float m) {
    return fmaxf(fmaxf(m, fmaxf(__uint_as_float(q.x), __uint_as_float(q.y))), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w)));
  }
  static __device__ __forceinline__ void open(uint4 q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
  }
  static __device__ __forceinline__ uint4 close(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};
template <> struct Group<__nv_bfloat16> {
  static constexpr int VEC = 8;
  static constexpr uint32_t kNone = 0xff80ff80u;
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {      // of both halves; a NaN gives way
    const __nv_bfloat162 r = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ float top(uint4 q, float m) {
    const uint32_t w = larger(larger(q.x, q.y), larger(q.z, q.w));
    return fmaxf(m, fmaxf(bf16_lo(w), bf16_hi(w)));
  }
  static __device__ __forceinline__ void open(uint4 q, float (&v)[8]) {
    v[0] = bf16_lo(q.x); v[1] = bf16_hi(q.x); v[2] = bf16_lo(q.y); v[3] = bf16_hi(q.y);
    v[4] = bf16_lo(q.z); v[5] = bf16_hi(q.z); v[6] = bf16_lo(q.w); v[7] = bf16_hi(q.w);
  }
  static __device__ __forceinline__ uint4 close(const float (&v)[8]) {
    return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
};

// A row's place: its groups of 16 aligned bytes, of which the first and the last may be shared with other rows
template <class T>
struct Place {
  static constexpr int VEC = Group<T>::VEC;
  uintptr_t base;                                            // of the first group
  int shift, groups;                                         // elements before the row in it
  int own, V;                                                // the group of its class
  int edge0, edge1;                                          // groups that hold other rows' elements, -1: none
  __device__ __forceinline__ Place(const void* matrix, int64_t row, int64_t ld, int V_, int id) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(matrix) + (uint64_t)row * (uint64_t)ld * sizeof(T);
    base = a & ~(uintptr_t)15;
    shift = (int)(a & 15) / (int)sizeof(T);
    V = V_;
    groups = (V + shift + VEC - 1) / VEC;
    own = id < 0 ? -1 : (id + shift) / VEC;
    edge0 = shift != 0 ? 0 : -1;
    edge1 = (V + shift) % VEC != 0 ? groups - 1 : -1;
  }
  __device__ __forceinline__ const uint4* at(int g) const { return reinterpret_cast<const uint4*>(base) + g; }
  __device__ __forceinline__ int first(int g) const { return g * VEC - shift; }        // the group's first element
  __device__ __forceinline__ bool edge(int g) const { return g == edge0 || g == edge1; }
  __device__ __forceinline__ bool special(int g) const { return g == own || edge(g); }
  // the group with -inf in the place of its class and of other rows' elements
  __device__ __forceinline__ uint4 others(uint4 q, int g, int id) const {
    uint32_t w[4] = {q.x, q.y, q.z, q.w};
    const int c = first(g);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const bool out = c + e == id || (unsigned)(c + e) >= (unsigned)V;
      if (sizeof(T) == 4) {
        if (out) w[e % 4] = Group<T>::kNone;
      } else if (out) {
        w[e / 2] = e % 2 ? (w[e / 2] & 0xffffu) | 0xff800000u : (w[e / 2] & 0xffff0000u) | 0xff80u;
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// s and U groups more, which may be -inf throughout
template <class T, int U>
__device__ __forceinline__ MaxSum add_groups(MaxSum s, const uint4 (&raw)[U], float c2) {
  constexpr int VEC = Group<T>::VEC;
  float m = s.m;
#pragma unroll
  for (int u = 0; u < U; ++u) m = Group<T>::top(raw[u], m);
  const u64 minus = pack2(-m, -m), cc = pack2(c2, c2);
  u64 l[2] = {pack2(s.l * ex2((s.m - m) * c2), 0.f), pack2(0.f, 0.f)};
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float v[VEC];
    Group<T>::open(raw[u], v);
#pragma unroll
    for (int e = 0; e < VEC; e += 2) {
      float a, b;
      unpack2(times2(add2(pack2(v[e], v[e + 1]), minus), cc), a, b);
      l[(e >> 1) & 1] = add2(l[(e >> 1) & 1], pack2(ex2(a), ex2(b)));
    }
  }
  float a, b;
  unpack2(add2(l[0], l[1]), a, b);
  return {m, a + b};
}

// The row that unit u of n (warps, CTAs, clusters) takes in its it-th turn: every turn the units take n rows that follow one another, each
// time with another beginning, since rows that do not count often lie a power of two apart.  (Dealing out the rows that count by lists that
// every CTA makes first cost 6 to 20 us and gave 6 of 400.)
__device__ __forceinline__ int64_t row_at(int it, int u, int n) {
  return (int64_t)it * n + (unsigned)(u + (it & 0xffff) * 7) % (unsigned)n;
}

// What the gradient of a row is formed with: dZ_j = f exp((Z_j - m) / tau), own for its class
struct Scale { float m, f, own; int zero; };
__device__ __forceinline__ Scale scale_of(const Row& r, float dlogp, float inv_tau) {
  const float coef = r.empty ? 0.f : dlogp * inv_tau;
  return {r.m, -coef / r.all, coef * (r.others / r.all), r.empty || coef == 0.f};
}

// The group's gradient, but for the row's class
template <class T, int VEC>
__device__ __forceinline__ void slopes(uint4 raw, const Scale& s, float c2, float (&v)[VEC]) {
  const u64 minus = pack2(-s.m, -s.m), cc = pack2(c2, c2), ff = pack2(s.f, s.f);
  Group<T>::open(raw, v);
#pragma unroll
  for (int e = 0; e < VEC; e += 2) {
    float a, b;
    unpack2(times2(add2(pack2(v[e], v[e + 1]), minus), cc), a, b);
    unpack2(times2(pack2(ex2(a), ex2(b)), ff), v[e], v[e + 1]);
  }
}

// Group g of a row to dZ, one by one: it may hold other rows' elements, or lie otherwise past 16 bytes in dZ.  (Not inline: within the
// loops its comparisons were carried out for every group.)
template <class T>
__device__ __noinline__ void put_singly(Place<T> z, int g, uint4 raw, Scale s, float c2, T* out) {
  constexpr int VEC = Group<T>::VEC;
  float v[VEC] = {};
  if (!s.zero) slopes<T, VEC>(raw, s, c2, v);
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const int j = z.first(g) + e;
    if (j >= 0 && j < z.V) put(out + j, v[e]);
  }
}

// The row's class, -1 if the row is not read
template <int MODE>
__device__ __forceinline__ int id_of(const Logprob& p, int64_t row) {
  if (row >= p.rows) return -1;
  const int64_t i = p.i64 ? static_cast<const int64_t*>(p.id)[row] : static_cast<const int32_t*>(p.id)[row];
  const float w = MODE == LP_BACKWARD ? p.dlogp_in[row] : p.weight ? p.weight[row] : 1.f;
  return i >= 0 && i < p.V && w != 0.f ? (int)i : -1;
}

// Results of a row, by one thread; the slope of the loss
template <int MODE>
__device__ __forceinline__ float finish(const Logprob& p, int64_t row, const Head& h, const Row& r, bool keep) {
  if (MODE == LP_BACKWARD) return h.a;
  Slope sl = {0.f, 0.f};
  if (p.loss && !r.empty) sl = policy_of(p, h, r.logp);
  if (keep) {
    if (p.logp) p.logp[row] = r.empty ? 0.f : r.logp;
    if (p.stat) {
      p.stat[2 * row] = r.empty ? 0.f : r.m;
      p.stat[2 * row + 1] = r.empty ? 0.f : r.others;
    }
    if (p.loss) p.loss[row] = sl.loss;
    if (p.dlogp) p.dlogp[row] = sl.dlogp;
  }
  return sl.dlogp;
}
// The row as its statistics have it
__device__ __forceinline__ Row row_of_stat(const Head& h, float c2) {
  const float e = h.z == -INFINITY ? 0.f : ex2((h.z - h.b) * c2);
  return {h.b, h.c, h.c + e, 0.f, h.c + e == 0.f};
}

// ---- a CTA of several warps for the logits and one, the last, for what a row has besides them ----
// With every warp forming the row's numbers from the sums, they were more instructions than the logits (29 for a logit of 4096 x 20000
// bf16, of which 11 for exponentials and sums).  The warps meet on the CTA's numbered barriers, where those that only tell do not wait.
template <int BAR>
__device__ __forceinline__ void meet(int turn, int threads) {
  __syncwarp();
  if (turn & 1) asm volatile("bar.sync %0, %1;" ::"n"(BAR + 1), "r"(threads) : "memory");
  else asm volatile("bar.sync %0, %1;" ::"n"(BAR), "r"(threads) : "memory");
}
template <int BAR>
__device__ __forceinline__ void tell(int turn, int threads) {
  __syncwarp();
  if (turn & 1) asm volatile("bar.arrive %0, %1;" ::"n"(BAR + 1), "r"(threads) : "memory");
  else asm volatile("bar.arrive %0, %1;" ::"n"(BAR), "r"(threads) : "memory");
}
enum { BAR_SUMS = 1, BAR_SCALE = 3, BAR_READ = 5 };          // each two that take turns

// The last warp's rows.  red: two places for the sums of `warps` warps; out: two for the scale.  FORWARD: sums come, nothing goes back, so the
// others are up to two rows ahead; BACKWARD: the scale goes out up to two rows ahead; BOTH: sums, then the scale.
template <class T, int MODE, class Combine>
__device__ __forceinline__ void numbers(const Logprob& p, int unit, int units, int threads, int warps, const MaxSum* red, Scale* out, bool keep,
                                        Combine combine) {
  const int lane = threadIdx.x & 31;
  const float c2 = p.inv_tau * kLog2e;
  int64_t later = row_at(0, unit, units);
  Head next = head_of<T, MODE>(p, later);
  int n = 0;
  for (int it = 0; (int64_t)it * units < p.rows; ++it) {
    const Head h = next;
    const int64_t row = later;
    later = row_at(it + 1, unit, units);
    next = head_of<T, MODE>(p, later);
    if (row >= p.rows) continue;
    Row r = {0.f, 0.f, 0.f, 0.f, true};
    if (h.id >= 0) {
      if (MODE == LP_BACKWARD) {
        r = row_of_stat(h, c2);
        if (n >= 2) meet<BAR_READ>(n, threads);
      } else {
        meet<BAR_SUMS>(n, threads);
        const MaxSum s = merge_lanes(lane < warps ? red[(n & 1) * 32 + lane] : MaxSum{kLow, 0.f}, c2);
        if (MODE == LP_FORWARD) tell<BAR_READ>(n, threads);
        r = row_of(combine(s, n), h.z, c2, p.inv_tau);
      }
    }
    const float dlogp = finish<MODE>(p, row, h, r, keep && lane == 0);
    if (MODE != LP_FORWARD && h.id >= 0) {
      if (lane == 0) out[n & 1] = scale_of(r, dlogp, p.inv_tau);
      tell<BAR_SCALE>(n, threads);
    }
    if (h.id >= 0) ++n;
  }
  // what the others have told is taken in
  if (MODE == LP_BACKWARD)
    for (int k = n > 2 ? n - 2 : 0; k < n; ++k) meet<BAR_READ>(k, threads);
}

// Loss and gradient of long rows whose Z and dZ lie equally past 16 bytes; *taken: the shape is one of them (fw_logprob_resident.cu)
template <class T>
cudaError_t launch_resident(const Logprob& p, cudaStream_t s, bool* taken);

}  // namespace logprob
}  // namespace fw
#endif
