// Distillation loss: what its kernels share (the formulas: fw_distill.cu).
#ifndef FW_DISTILL_CUH_
#define FW_DISTILL_CUH_

#include "fw_internal.h"
#include "fw_rows.cuh"

namespace fw {
namespace distill {

using namespace rows;

constexpr int kMaxK = 1024;
constexpr int kMaxV = 1 << 20;             // a cluster's bit sets and entries stay below 48 KB of shared memory a CTA
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLow = -3.402823466e38f;   // the lowest finite value: the largest of nothing, beside a sum of 0
// Logarithms are summed times 2^-21 (exact), so that a logit at the lowest finite value (a mask) times log2(e) / tau stays in
// fp32 for every tau; kUp = 2^21 ln 2 makes the loss of them.
constexpr float kDown = 4.76837158203125e-07f, kUp = 2097152.f * kLn2;
enum { DIST_LOSS = 0, DIST_BOTH = 1, DIST_BACKWARD = 2 };
// The gradient alone takes a row's normalisers from the forward call, as far as they are fine: beyond 1024 their rounding to fp32
// is more than 2^-15 of every exponential, and at -3e38 (a row of the lowest finite value) nothing is left of the classes' number.  Such
// a row's sums are formed again from Z.
constexpr float kFineStat = 1024.f;
__device__ __forceinline__ bool coarse(float s0, float s1) { return !(fabsf(s0) <= kFineStat && fabsf(s1) <= kFineStat); }

struct Distill {
  const void* Z;
  const void* T;
  const void* I;
  const float *t_lse, *weight;
  const float* stat_in;
  float *loss, *stat;
  void* dZ;
  int64_t ldz, lddz;
  int32_t V, K;
  int32_t t_bf16, i64;
  int32_t slice;          // classes of a CTA, a multiple of the CTA's accesses
  float inv_tau;
};

// Largest logit m and the sum of exp((z - m) / tau).  Differences of logits are scaled, not logits: near the largest, where the
// mass is, their rounding is small.  c2 = log2(e) / tau.
// (The roundings are written out: the loss alone and the loss with the gradient are the same number.)
struct MaxSum { float m, l; };
__device__ __forceinline__ MaxSum merge(MaxSum a, MaxSum b, float c2) {
  const float m = fmaxf(a.m, b.m);
  return {m, fmaf(a.l, ex2((a.m - m) * c2), __fmul_rn(b.l, ex2((b.m - m) * c2)))};
}
__device__ __forceinline__ float lanes_max(float v) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// The whole warp's: its largest first, so that the chain is one exponential and five additions long (five merges took twice that)
__device__ __forceinline__ MaxSum merge_lanes(MaxSum s, float c2) {
  const float m = lanes_max(s.m);
  return {m, lanes_sum(s.l * ex2((s.m - m) * c2))};
}

// Two and three of them at once: the chains run beside each other.
__device__ __forceinline__ void merge_lanes2(MaxSum& a, MaxSum& b, float c2) {
  const float ma = lanes_max(a.m), mb = lanes_max(b.m);
  a = {ma, a.l * ex2((a.m - ma) * c2)};
  b = {mb, b.l * ex2((b.m - mb) * c2)};
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float x = __shfl_xor_sync(0xffffffffu, a.l, o), y = __shfl_xor_sync(0xffffffffu, b.l, o);
    a.l += x;
    b.l += y;
  }
}
__device__ __forceinline__ void merge_lanes3(MaxSum& a, MaxSum& b, MaxSum& c, float c2) {
  const float ma = lanes_max(a.m), mb = lanes_max(b.m), mc = lanes_max(c.m);
  a = {ma, a.l * ex2((a.m - ma) * c2)};
  b = {mb, b.l * ex2((b.m - mb) * c2)};
  c = {mc, c.l * ex2((c.m - mc) * c2)};
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float x = __shfl_xor_sync(0xffffffffu, a.l, o), y = __shfl_xor_sync(0xffffffffu, b.l, o), z = __shfl_xor_sync(0xffffffffu, c.l, o);
    a.l += x;
    b.l += y;
    c.l += z;
  }
}

// With P of the teacher's mass and Q of the student's on the named classes: log p_t - log q_t (base 2, times kDown), and A q_t - p_t, from the masses
// that are small.  Where both lie almost wholly on the other classes the loss is what is left of two logarithms near 0.
// log q_t comes from logarithms, and the others' exponentials are relative to the largest of the others: a named class 90 tau ahead
// takes their mass out of fp32, not the loss nor their gradient (A q_t - p_t times their shares of q_t).
__device__ __forceinline__ float log_rest(float pt, MaxSum others, MaxSum all, float c2, float P, float Q) {
  if (P < 0.5f && Q < 0.5f) return (log1pf(-P) - log1pf(-Q)) * (kLog2e * kDown);
  return kDown * log2f(pt) - fmaf(others.m - all.m, c2 * kDown, kDown * (log2f(others.l) - log2f(all.l)));
}
__device__ __forceinline__ float excess_rest(float A, float pt, float qt, float P, float Q) {
  return pt > 0.f ? (P < 0.5f && Q < 0.5f ? P - Q : fmaf(A, qt, -pt)) : A * qt;
}

// The gradient of a row whose statistics are coarse, by a warp, or by a CTA for which red has two floats a warp.  bits: one for each
// class.  Z is read twice for the sums and written over at the end, dZ = Z or not; entries are looked at where they lie.  Few
// registers and no speed: it is called beside kernels that hardly ever meet such a row, and costs them a branch (with the
// sums in their own loops the gradient alone of 1024 x 131072 bf16 took 126-145 us for 98).
template <class T, int VEC, bool CTA>
__device__ __noinline__ void coarse_row(Distill p, int64_t row, uint32_t* bits, float* red) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int tid = CTA ? (int)threadIdx.x : lane, nt = CTA ? (int)blockDim.x : 32;
  const float c2 = p.inv_tau * kLog2e, wt = p.weight ? p.weight[row] : 1.f, t_lse = p.t_lse ? p.t_lse[row] : 0.f;
  const T* z = static_cast<const T*>(p.Z) + row * p.ldz;
  T* dz = static_cast<T*>(p.dZ) + row * p.lddz;
  auto sync = [&]() { if (CTA) __syncthreads(); else __syncwarp(); };
  auto whole_group = [&](MaxSum s) {                  // warps in order
    s = merge_lanes(s, c2);
    if (!CTA) return s;
    __syncthreads();
    if (lane == 0) { red[2 * warp] = s.m; red[2 * warp + 1] = s.l; }
    __syncthreads();
    s = {red[0], red[1]};
    for (int k = 1; k < nt / 32; ++k) s = merge(s, {red[2 * k], red[2 * k + 1]}, c2);
    return s;
  };
  auto cls = [&](int k) {
    const int64_t at = row * p.K + k, i = p.i64 ? static_cast<const int64_t*>(p.I)[at] : static_cast<const int32_t*>(p.I)[at];
    return i >= 0 && i < p.V ? (int)i : -1;
  };
  auto t_of = [&](int k) {
    const int64_t at = row * p.K + k;
    return p.t_bf16 ? to_f(static_cast<const __nv_bfloat16*>(p.T)[at]) : static_cast<const float*>(p.T)[at];
  };
  for (int i = tid; i < (p.V + 31) / 32; i += nt) bits[i] = 0;
  sync();
  uint32_t mine = 0;                                  // which of this thread's entries count
  float tm = kLow;
  MaxSum named = {kLow, 0.f}, others = {kLow, 0.f};
  for (int k = tid, b = 0; k < p.K; k += nt, ++b) {
    const int i = cls(k);
    bool out = i < 0;
    for (int j = 0; j < k && !out; ++j) out = cls(j) == i;
    if (out) continue;
    mine |= 1u << b;
    atomicOr(&bits[i >> 5], 1u << (i & 31));
    tm = fmaxf(tm, t_of(k));
    const float v = to_f(z[i]);
    named = merge(named, {fmaxf(v, kLow), v == -INFINITY ? 0.f : v != v ? v : 1.f}, c2);
  }
  sync();
  for (int c = tid * VEC; c < p.V; c += nt * VEC) {
    const uint32_t is = bits[c >> 5] >> (c & 31);
    float v[VEC];
    load<VEC>(z + c, p.V - c, -INFINITY, v);
    MaxSum now = {kLow, 0.f};
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      if ((is >> e) & 1u) v[e] = -INFINITY;
      now.m = fmaxf(now.m, v[e]);
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) now.l += ex2((v[e] - now.m) * c2);
    others = merge(others, now, c2);
  }
  others = whole_group(others);
  named = whole_group(named);
  tm = whole_group({tm, 0.f}).m;
  auto teacher2 = [&](float t) { return p.t_lse ? fmaf(t, p.inv_tau, -t_lse) * kLog2e : (t - tm) * c2; };
  MaxSum t = {0.f, 0.f};
  for (int k = tid, b = 0; k < p.K; k += nt, ++b)
    if ((mine >> b) & 1u) t.l += ex2(teacher2(t_of(k)));
  const float ts = whole_group(t).l;
  const float scale_p = p.t_lse ? 1.f : (ts > 0.f ? 1.f / ts : (ts == 0.f ? 0.f : ts));
  const float whole = ts * scale_p;
  float pt = 0.f;
  if (p.t_lse) pt = 1.f - whole < 0.f ? 0.f : 1.f - whole;
  const float A = whole + pt;
  const MaxSum all = merge(others, named, c2);
  const float inv = 1.f / all.l, qt = others.l * ex2((others.m - all.m) * c2) * inv, Q = named.l * ex2((named.m - all.m) * c2) * inv;
  const float ws = all.l == 0.f ? 0.f : wt * p.inv_tau;
  const float f = ws == 0.f || others.l == 0.f ? 0.f : ws * excess_rest(A, pt, qt, whole, Q) / others.l;
  for (int c = tid * VEC; c < p.V; c += nt * VEC) {
    const uint32_t is = bits[c >> 5] >> (c & 31);
    float v[VEC];
    load<VEC>(z + c, p.V - c, -INFINITY, v);
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (!((is >> e) & 1u)) v[e] = f == 0.f ? 0.f : f * ex2((v[e] - others.m) * c2);      // a named class keeps its logit: it is read once more
    store<VEC>(dz + c, p.V - c, v);
  }
  sync();
  for (int k = tid, b = 0; k < p.K; k += nt, ++b) {
    if (!((mine >> b) & 1u)) continue;
    const int i = cls(k);
    const float q = ex2((to_f(z[i]) - all.m) * c2) * inv;
    put(dz + i, ws == 0.f ? 0.f : ws * (A * q - ex2(teacher2(t_of(k))) * scale_p));
  }
  sync();
}

// Launchers of a kernel for rows of one kind; *taken: the shape is one of its own
template <class T, int VEC, int MODE>
cudaError_t launch_ring(const Distill& p, int64_t rows, cudaStream_t s, bool* taken);      // fw_distill_ring.cu
template <class T, int VEC, int MODE>
cudaError_t launch_warp(const Distill& p, int64_t rows, cudaStream_t s, bool* taken);      // fw_distill_warp.cu

}  // namespace distill
}  // namespace fw
#endif
